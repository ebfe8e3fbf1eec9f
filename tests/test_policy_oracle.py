"""Pins of the oracle's 4-bit formats and changed logits: values by hand, brute force, autograd and differences."""

import itertools
import math

import numpy as np
import pytest
import torch

import oracle

VALUES = [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]


def test_code_values():
    assert oracle.mxfp4_code_values().tolist() == VALUES
    assert np.signbit(oracle.mxfp4_code_values()[8])


def test_every_code_and_scale_quantises_to_itself():
    """A block that holds a magnitude in [4, 8) keeps its scale and codes."""
    codes = np.tile(np.arange(16, dtype=np.uint8), 2)[None].repeat(253, 0)
    scales = np.arange(0, 253, dtype=np.uint8)[:, None]
    c, s = oracle.mxfp4_quantize(oracle.mxfp4_values(codes, scales))
    assert (c == codes).all() and (s == scales).all()


def test_nearest_by_brute_force():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 64)) * np.exp(rng.standard_normal((40, 64)))
    c, s = oracle.mxfp4_quantize(x)
    got = oracle.mxfp4_values(c, s)
    for i, k in itertools.product(range(40), range(64)):
        scale = 2.0 ** (math.floor(math.log2(np.abs(x[i, k // 32 * 32:k // 32 * 32 + 32]).max())) - 2)
        assert 2.0 ** (float(s[i, k // 32]) - 127) == scale
        best = min(abs(x[i, k] - scale * v) for v in VALUES)
        assert abs(x[i, k] - got[i, k]) == pytest.approx(best, abs=0)


@pytest.mark.parametrize("x,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6),
                                    (0.2500001, 1), (7.99, 7), (-0.75, 10), (-0.1, 8), (-0.0, 8)])
def test_ties_go_to_the_even_code(x, code):
    row = np.zeros((1, 32))
    row[0, 0], row[0, 1] = 4.0, x  # the scale is 1
    c, s = oracle.mxfp4_quantize(row)
    assert s[0, 0] == 127 and c[0, 1] == code


def test_zero_tiny_and_bad_blocks():
    x = np.zeros((1, 128))
    x[0, 32] = 2.0 ** -149
    x[0, 64], x[0, 96] = np.nan, -np.inf
    c, s = oracle.mxfp4_quantize(x)
    assert s.tolist() == [[0, 0, 255, 255]] and (c == 0).all()
    v = oracle.mxfp4_values(c, s)
    assert (v[0, :64] == 0).all() and np.isnan(v[0, 64:]).all()


def test_pack_and_logits():
    rng = np.random.default_rng(2)
    codes = rng.integers(0, 16, (3, 64)).astype(np.uint8)
    packed = oracle.mxfp4_pack(codes)
    assert packed[1, 5] == codes[1, 10] + 16 * codes[1, 11]
    assert (oracle.mxfp4_unpack(packed) == codes).all()
    w = rng.standard_normal((2, 64))
    h = oracle.mxfp4_values(codes, np.full((3, 2), 126, np.uint8))
    z = oracle.mxfp4_logits(h, w, 0.5)
    for t, v in itertools.product(range(3), range(2)):
        assert z[t, v] == pytest.approx(2 * math.fsum(h[t, k] * w[v, k] for k in range(64)), rel=1e-13)


# ------------------------------------------------------------------ changed logits


def test_rules_by_hand():
    z = np.array([[2.0, -2.0, 4.0, 0.0, 1.0]])
    rule = {"prompt": [0, 1, 9, -1], "output": [2, 2, 1, 77], "repetition": 2.0, "frequency": 0.25, "presence": 0.5,
            "bias": [(3, 7.0), (4, 1.0), (3, -3.0), (5, 9.0)], "allowed": np.array([1, 1, 1, 1, 0], bool)}
    x, slope = oracle.change_logits(z, [rule], 0.5)
    # 2/2; -2*2 - .25 - .5; 4/2 - 2*.25 - .5; 0 - 3; masked
    assert x.tolist() == [[2.0, -9.5, 2.0, -6.0, -math.inf]]
    assert slope.tolist() == [[1.0, 4.0, 1.0, 2.0, 0.0]]


def _rule_cases():
    rng = np.random.default_rng(3)
    z = 2 * rng.standard_normal((5, 11))
    z[1, 4] = np.nan
    rules = [{}, {"prompt": [1, 2], "output": [3, 3, 5], "repetition": 1.3, "frequency": 0.2, "presence": 0.4,
                  "allowed": np.arange(11) != 4},
             {"bias": [(2, 1.5)], "output": [0] * 7, "frequency": 0.1},
             {"allowed": np.arange(11) == 6}, {"allowed": np.zeros(11, bool)}]
    return z, rules, np.array([3, 5, -1, 6, 0]), rng.standard_normal(5), rng.standard_normal(5)


def test_changed_logprobs_and_grad_against_autograd():
    z, rules, tok, g, e = _rule_cases()
    lp, H, lse = oracle.changed_logprobs(z, tok, rules, 0.8)
    grad = oracle.changed_logprobs_grad(z, tok, rules, g, e, 0.8)
    for i in range(4):
        keep = rules[i].get("allowed", np.ones(11, bool))
        zi = torch.tensor(z[i], requires_grad=True)
        x = zi
        rule = rules[i]
        seen = np.isin(np.arange(11), list(rule.get("prompt", [])) + list(rule.get("output", [])))
        c = torch.tensor([float(list(rule.get("output", [])).count(v)) for v in range(11)], dtype=torch.float64)
        rho = rule.get("repetition", 1.0)
        x = torch.where(torch.tensor(seen), torch.where(x > 0, x / rho, x * rho), x)
        x = x - rule.get("frequency", 0.0) * c - rule.get("presence", 0.0) * (c > 0).double()
        for t, b in rule.get("bias", ()):
            x = x + b * (torch.arange(11) == t)
        x = (x / 0.8)[torch.tensor(keep)]
        logp = torch.log_softmax(x, 0)
        ent = -(logp.exp() * logp).sum()
        at = np.nonzero(np.nonzero(keep)[0] == tok[i])[0]
        loss = e[i] * ent + (g[i] * logp[int(at[0])] if len(at) else 0.0)
        loss.backward()
        assert H[i] == pytest.approx(ent.item(), abs=1e-13)
        assert lse[i] == pytest.approx(torch.logsumexp(x, 0).item(), abs=1e-13)
        assert np.isnan(lp[i]) if tok[i] < 0 else lp[i] == pytest.approx(logp[int(at[0])].item(), abs=1e-13)
        np.testing.assert_allclose(grad[i][keep], zi.grad.numpy()[keep], atol=1e-13)
        assert (grad[i][~keep] == 0).all()
    assert (lp[4], H[4], lse[4]) == (-math.inf, 0.0, -math.inf) and (grad[4] == 0).all()


def test_changed_grad_against_differences():
    z, rules, tok, g, e = _rule_cases()
    z[1, 4] = 0.3
    grad = oracle.changed_logprobs_grad(z, tok, rules, g, e, 0.8)

    def loss(zz):
        lp, H, _ = oracle.changed_logprobs(zz, tok, rules, 0.8)
        return np.where(np.isfinite(lp), g * np.where(np.isfinite(lp), lp, 0), 0).sum() + (e * H).sum()

    for i, v in itertools.product(range(4), range(11)):
        step = np.zeros_like(z)
        step[i, v] = 1e-6
        assert (loss(z + step) - loss(z - step)) / 2e-6 == pytest.approx(grad[i, v], abs=1e-8)


def test_no_rules_is_the_plain_log_softmax():
    rng = np.random.default_rng(4)
    z, tok = 3 * rng.standard_normal((4, 9)), np.array([0, 8, 3, 9])
    lp, H, lse = oracle.changed_logprobs(z, tok, [{}] * 4, 1.7)
    ref = torch.log_softmax(torch.tensor(z) / 1.7, 1)
    np.testing.assert_allclose(lp[:3], ref[torch.arange(3), torch.tensor(tok[:3])], atol=1e-13)
    assert np.isnan(lp[3])
    np.testing.assert_allclose(H, -(ref.exp() * ref).sum(1), atol=1e-13)
    np.testing.assert_allclose(lse, torch.logsumexp(torch.tensor(z) / 1.7, 1), atol=1e-13)


MUTATIONS = [  # a mistake in the oracle must show in the pins above
    ("mxfp4", "- 1 - 2, -127)", "- 1 - 1, -127)"),
    ("mxfp4", "[0, 2, 4, 6, 1, 3, 5, 7]", "[1, 3, 5, 7, 0, 2, 4, 6]"),
    ("mxfp4", "np.signbit(b), code + 8", "b < 0, code + 8"),
    ("mxfp4", "(codes[:, 1::2] << 4)", "(codes[:, 1::2] << 3)"),
    ("mxfp4", "/ float(temperature)", "* float(temperature)"),
    ("rules", "z[i, t] / rho if z[i, t] > 0", "z[i, t] / rho if z[i, t] < 0"),
    ("rules", "slope[i, t] = k", "slope[i, t] = 1.0"),
    ("rules", "* c + float(rule", "+ float(rule"),
    ("rules", "dict(rule.get(\"bias\", ())).items()", "list(rule.get(\"bias\", ()))"),
    ("rules", "slope[i][~rule[\"allowed\"]] = 0.0", "pass"),
    ("rules", "(logp_all + H[:, None])", "(logp_all - H[:, None])"),
    ("rules", "g = np.where(ok,", "g = np.where(ok | True,"),
    ("rules", "slope[i] /= float(temperature)", "pass"),
]


@pytest.mark.parametrize("module,old,new", MUTATIONS)
def test_pins_reject_mistakes(module, old, new, monkeypatch):
    import importlib
    import types

    real = importlib.import_module(f"oracle.{module}")
    source = open(real.__file__).read()
    assert source.count(old) == 1
    mutant = types.ModuleType("mutant")
    exec(compile(source.replace(old, new), "mutant", "exec"), mutant.__dict__)
    for name in ("mxfp4_quantize", "mxfp4_pack", "mxfp4_logits", "change_logits", "changed_logprobs",
                 "changed_logprobs_grad"):
        if hasattr(mutant, name):
            monkeypatch.setattr(oracle, name, getattr(mutant, name))
    failed = 0
    for check in (test_every_code_and_scale_quantises_to_itself, test_nearest_by_brute_force, test_pack_and_logits,
                  test_rules_by_hand, test_changed_logprobs_and_grad_against_autograd, test_changed_grad_against_differences,
                  lambda: test_ties_go_to_the_even_code(0.25, 0), lambda: test_ties_go_to_the_even_code(-0.0, 8)):
        try:
            check()
        except Exception:
            failed += 1
    assert failed


@pytest.mark.parametrize("offset", [0.0, 1e6, -1e12, -3.4028234663852886e38, 3.4028234663852886e38])
def test_offsets_common_to_a_row_do_not_enter(offset):
    """n equal logits: p = 1 / n, H = log n, gradient g ([v = token] - 1 / n), whatever lse can hold."""
    n = 37
    z = np.full((2, n), offset)
    allowed = np.arange(n) < 11
    rules = [{}, {"allowed": allowed}]
    lp, H, _ = oracle.changed_logprobs(z, [3, 4], rules, 0.7)
    assert np.allclose(lp, [-math.log(n), -math.log(11)]) and np.allclose(H, [math.log(n), math.log(11)])
    g = oracle.changed_logprobs_grad(z, [3, 4], rules, [1.0, -2.0], [5.0, 5.0], 0.7)
    want = np.zeros((2, n))
    want[0], want[1, :11] = -1 / n, 2 / 11
    want[0, 3] += 1.0
    want[1, 4] -= 2.0
    assert np.allclose(g, want / 0.7, rtol=1e-12, atol=1e-12)
