"""GPU parity of the changed logits (tim_logits_adjust, tim_logits_logprobs and its backward).

adjust: every step is one fp32 operation, so the outputs are compared bit for bit with the same steps in numpy's fp32,
rounded once to the output type.

logprobs and backward, against the fp64 oracle, u = 2^-24. With M the largest magnitude an entry of the row takes on
its way (logit times the penalties, plus bias), each x is within 6 u M / tau =: D of its exact value (six roundings).
  lse, logp: a softmax average of D, the exponentials' argument (2 u |q| each, a p-weighted mean of |q| is at most
    ln V + 1 < 16), a sum of 16 + 6 + 8 + 6 terms in chains and trees, the logarithm and the last additions:
    2 D + (64 + 32 + 4 |result|) u
  entropy: dH/dx = -p (log p + H), whose absolute values sum to at most 2 (ln V + 1): 2 D (ln V + 1) + 128 (ln V + 1) u
  grad: p = e^(x - lse) is relatively within D + 4 u |q| + 8 u, q = x - lse absolutely within D + u |q|:
    slope p (|g| + |e| (|q| + |H| + 1)) (D + (4 |q| + 12) u) + 4 u |ref| + 4 u slope |g| [v = tok] + the output type's
    half step; where the entry's logit sits at a penalty's corner (0) both sides take the same branch."""

import math

import numpy as np
import pytest
import torch

import oracle
import paper_2605_14220_amd as tim
from tim_testutil import require_gpu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = {torch.float32: 2.0 ** -120, torch.bfloat16: 2.0 ** -120, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


class Case:
    """Random logits and rules of T rows: lists for the oracle, tensors for the library."""

    def __init__(self, T, V, seed, dtype=torch.float32, history=40, packed=False, bias=0, masks=0, penalties=True,
                 pad=0, scale=3.0, heavy=False):
        rng = np.random.default_rng(seed)
        self.T, self.V = T, V
        z = torch.as_tensor(scale * rng.standard_normal((T, V + pad)), dtype=torch.float32).to(dtype)
        self.z = z.cuda()[:, :V]
        self.tokens = rng.integers(0, V, T).astype(np.int32)
        self.rules = [{} for _ in range(T)]
        kw = {}
        if history is not None:
            n = max(1, history) * (1 if packed else T) + (T if packed else 0) + 7
            # few distinct tokens, so that they repeat; some outside the vocabulary
            stream = rng.choice(np.concatenate([rng.integers(0, V, 4 if heavy else 60), [-1, V, 2 ** 31 - 1, -2 ** 31]]), n)
            stream = np.where(rng.random(n) < (0.1 if heavy else 0.5), rng.integers(0, V, n), stream).astype(np.int32)
            if packed:
                begin = np.zeros(T, np.int64) + 3
                split = begin + history
                end = split + np.arange(T)
            else:
                begin = rng.integers(0, n - history + 1, T)
                end = begin + rng.integers(0, history + 1, T)
                split = begin + ((end - begin) * rng.random(T)).astype(np.int64)
            for i in range(T):
                self.rules[i]["prompt"] = stream[begin[i]:split[i]].tolist()
                self.rules[i]["output"] = stream[split[i]:end[i]].tolist()
            kw.update(history=torch.as_tensor(stream).cuda(), hist_begin=torch.as_tensor(begin).cuda(),
                      hist_split=torch.as_tensor(split).cuda(), hist_end=torch.as_tensor(end).cuda())
            if penalties:
                for name, lo, hi in (("repetition", 0.5, 2.0), ("frequency", -0.5, 1.0), ("presence", -1.0, 1.0)):
                    x = rng.uniform(lo, hi, T).astype(np.float32)
                    kw[name] = torch.as_tensor(x).cuda()
                    for i in range(T):
                        self.rules[i][name] = float(x[i])
        if bias:
            n = 3 * bias
            ids = rng.integers(-2, V + 2, n).astype(np.int32)
            ids[: n // 2] = ids[n - n // 2:]  # the same ids twice
            vals = rng.uniform(-5, 5, n).astype(np.float32)
            vals[rng.random(n) < 0.05] = -np.inf
            b = rng.integers(0, n + 1, T)
            e = np.minimum(n, b + rng.integers(0, 2 * bias + 1, T))
            for i in range(T):
                self.rules[i]["bias"] = list(zip(ids[b[i]:e[i]].tolist(), vals[b[i]:e[i]].tolist()))
            kw.update(bias_ids=torch.as_tensor(ids).cuda(), bias_values=torch.as_tensor(vals).cuda(),
                      bias_begin=torch.as_tensor(b).cuda(), bias_end=torch.as_tensor(e).cuda())
        if masks:
            words = (V + 31) // 32 + 2
            allowed = rng.random((masks, V)) < np.where(np.arange(masks) % 2 == 0, 0.9, min(1.0, 8 / V))[:, None]
            allowed[0] = False  # a mask that leaves nothing
            if masks > 1:
                allowed[1] = False
                allowed[1, V - 1] = True
            rows = rng.integers(-1, masks + 1, T).astype(np.int32)
            bits = np.zeros((masks, words * 32), dtype=bool)
            bits[:, :V] = allowed
            bits[:, V:] = rng.random((masks, words * 32 - V)) < 0.5  # bits past V mean nothing
            packed_words = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
            for i in range(T):
                if 0 <= rows[i] < masks:
                    self.rules[i]["allowed"] = allowed[rows[i]]
            kw.update(mask=torch.as_tensor(packed_words).cuda(), mask_rows=torch.as_tensor(rows).cuda())
        self.lib = tim.LogitRules(**kw)
        self.tok = torch.as_tensor(self.tokens).cuda()

    def rows(self, a, b):
        """The rules of rows a .. b."""
        kw = {}
        for f in ("hist_begin", "hist_split", "hist_end", "repetition", "frequency", "presence", "bias_begin",
                  "bias_end", "mask_rows"):
            t = getattr(self.lib, f)
            if t is not None:
                kw[f] = t[a:b].contiguous()
        return tim.LogitRules(**{f: getattr(self.lib, f) for f in ("history", "bias_ids", "bias_values", "mask")}, **kw)


def fp32_steps(case, z, tau):
    """The documented steps in numpy fp32, and the largest magnitude on the way per row."""
    f = np.float32
    z = z.float().cpu().numpy()
    inv = f(1.0 / np.float64(f(tau)))
    out, top = z.copy(), np.zeros(case.T)
    with np.errstate(all="ignore"):
        for i, rule in enumerate(case.rules):
            x = out[i]
            big = np.abs(np.where(np.isfinite(x), x, 0)).max() * max(rule.get("repetition", 1), 1 / rule.get("repetition", 1))
            output = [t for t in rule.get("output", ()) if 0 <= t < case.V]
            count = np.bincount(output, minlength=case.V)
            seen = count > 0
            seen[[t for t in rule.get("prompt", ()) if 0 <= t < case.V]] = True
            if "repetition" in rule:
                rho = f(rule["repetition"])
                x[seen] = np.where(x[seen] > 0, x[seen] / rho, x[seen] * rho)
            has = count > 0
            if "frequency" in rule:
                x[has] = x[has] - f(rule["frequency"]) * count[has].astype(f)
                x[has] = x[has] - f(rule["presence"])
                big += abs(rule["frequency"]) * count.max() + abs(rule["presence"])
            for t, b in dict(rule.get("bias", ())).items():
                if 0 <= t < case.V:
                    x[t] = x[t] + f(b)
                    big += abs(b) if np.isfinite(b) else 0
            out[i] = x * inv
            if "allowed" in rule:
                out[i][~rule["allowed"]] = -np.inf
            top[i] = big
    return out, top


def check_adjust(case, tau, **kw):
    want = torch.as_tensor(fp32_steps(case, case.z, tau)[0]).to(case.z.dtype)
    got = tim.logits_adjust(case.z, case.lib, tau, **kw).cpu()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    assert same.all(), (same.logical_not().nonzero()[:5], got[~same][:5], want[~same][:5])
    return got


def check_logprobs(case, tau):
    lp, H, lse = (x.double().cpu().numpy() for x in tim.logits_logprobs(case.z, case.tok, case.lib, tau, lse=True))
    z64 = case.z.double().cpu().numpy()
    inv = float(np.float32(1.0 / np.float64(np.float32(tau))))
    r_lp, r_H, r_lse = oracle.changed_logprobs(z64, case.tokens, case.rules, 1.0 / inv)
    _, top = fp32_steps(case, case.z, tau)
    D = 6 * U * top * inv
    lnv = math.log(case.V) + 1
    for name, got, ref, tol in (("logp", lp, r_lp, 2 * D + (96 + 4 * np.abs(r_lp)) * U),
                                ("lse", lse, r_lse, 2 * D + (96 + 4 * np.abs(r_lse)) * U),
                                ("entropy", H, r_H, 2 * D * lnv + 128 * lnv * U)):
        special = ~np.isfinite(ref)
        assert (np.isnan(got) == np.isnan(ref)).all() and (got[np.isinf(ref)] == ref[np.isinf(ref)]).all(), name
        err, lim = np.abs(got[~special] - ref[~special]), np.broadcast_to(tol, ref.shape)[~special]
        if len(err):
            print(f"[parity] {name}: max|err| {err.max():.2e}, {np.max(err / lim):.3f} of the bound")
            assert (err <= lim).all(), (name, np.argmax(err / lim))
    return r_lp, r_H, r_lse


def check_backward(case, tau, entropy, grad=None, **kw):
    rng = np.random.default_rng(case.T + 99)
    g = rng.standard_normal(case.T).astype(np.float32)
    e = rng.standard_normal(case.T).astype(np.float32) if entropy else None
    g[case.T // 2] = 0.0
    if entropy:
        e[case.T // 3] = 0.0
    inv = float(np.float32(1.0 / np.float64(np.float32(tau))))
    z64 = case.z.double().cpu().numpy()
    _, H, lse = oracle.changed_logprobs(z64, case.tokens, case.rules, 1.0 / inv)
    as_gpu = lambda x: None if x is None else torch.as_tensor(x.astype(np.float32)).cuda()  # noqa: E731
    got = tim.logits_logprobs_backward(case.z, case.tok, as_gpu(lse), as_gpu(g), case.lib, tau, entropy=as_gpu(H),
                                       grad_entropy=as_gpu(e), dtype=grad, **kw)
    ref = oracle.changed_logprobs_grad(z64, case.tokens, case.rules, g, e, 1.0 / inv)
    x, slope = oracle.change_logits(z64, case.rules, 1.0 / inv)
    _, top = fp32_steps(case, case.z, tau)
    # lse and H reach the kernel rounded to fp32: one more rounding of q and of H
    D = (6 * top * inv + np.abs(np.where(np.isfinite(lse), lse, 0)))[:, None] * U
    q = np.where(np.isfinite(x), x - np.where(np.isfinite(lse), lse, 0)[:, None], 0.0)
    p = np.where(np.isfinite(x), np.exp(q), 0.0)
    eg = 0.0 if e is None else np.abs(e)[:, None]
    a = np.abs(g)[:, None] + eg * (np.abs(q) + np.abs(H)[:, None] + 1)
    onehot = np.zeros_like(z64)
    ok = (case.tokens >= 0) & (case.tokens < case.V)
    onehot[np.nonzero(ok)[0], case.tokens[ok]] = 1.0
    bound = slope * (p * a * (D + (4 * np.abs(q) + 12) * U) + 4 * U * np.abs(g)[:, None] * onehot) + 4 * U * np.abs(ref)
    # the hardware exponential gives 0 where e^q is below the smallest normal number, 2^-126: p is off by up to that
    bound += slope * a * 2.0 ** -126
    bound += torch.finfo(got.dtype).eps / 2 * (np.abs(ref) + bound) + TINY[got.dtype]
    err = np.abs(got.double().cpu().numpy() - ref)
    assert np.isfinite(err).all()
    print(f"[parity] grad: max|err| {err.max():.2e}, {np.max(err / bound):.3f} of the bound")
    assert (err <= bound).all(), np.argwhere(err > bound)[:5]
    assert (got[case.T // 2].abs().sum() == 0) or entropy
    return got


CASES = {
    "one_entry": dict(T=3, V=1, history=3, masks=2),
    "one_row": dict(T=1, V=1000, history=50, bias=20, masks=3),
    "odd": dict(T=13, V=1237, history=100, bias=40, masks=5, pad=3),
    "chunk_end": dict(T=4, V=8191, history=300, bias=100, masks=4),
    "chunk": dict(T=4, V=8192, history=300, bias=100, masks=4),
    "chunk_and_one": dict(T=4, V=8193, history=300, bias=100, masks=4, pad=1),
    "three_chunks": dict(T=6, V=20003, history=2000, bias=300, masks=6),
    "packed": dict(T=70, V=9001, history=30, packed=True),
    "packed_heavy": dict(T=600, V=300, history=5, packed=True, heavy=True, bias=9, masks=7),
    "no_penalties": dict(T=5, V=3000, history=100, penalties=False),
    "bias_only": dict(T=9, V=500, history=None, bias=1000),
    "masks_only": dict(T=9, V=4099, history=None, masks=9),
    "nothing": dict(T=9, V=4099, history=None),
    "empty_history": dict(T=3, V=100, history=0),
}


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("name", list(CASES))
def test_adjust(name, dtype):
    print(f"case {name} {dtype}", flush=True)
    check_adjust(Case(seed=len(name), dtype=DTYPES[dtype], **CASES[name]), 0.7)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("name", list(CASES))
def test_logprobs(name, dtype):
    print(f"case {name} {dtype}", flush=True)
    check_logprobs(Case(seed=len(name) + 1, dtype=DTYPES[dtype], **CASES[name]), 0.7)


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("bf16", "f32"),
                                        ("bf16", "f16"), ("f16", "f16"), ("f16", "f32"), ("f16", "bf16")])
@pytest.mark.parametrize("name", list(CASES))
def test_backward(name, dtype, grad):
    print(f"case {name} {dtype} -> {grad}", flush=True)
    case = Case(seed=len(name) + 2, dtype=DTYPES[dtype], **CASES[name])
    check_backward(case, 0.7, entropy=(len(name) + len(grad)) % 2 == 0, grad=DTYPES[grad])


def test_gradient_against_differences():
    """The gradient of the fp64 oracle's loss by central differences, on the rows' most likely entries."""
    case = Case(4, 50, 3, history=30, bias=10)
    case.rules[2].pop("bias")
    case.lib.bias_end[2] = case.lib.bias_begin[2]
    for r in case.rules:  # no entry at -inf, where differences do not exist
        r["bias"] = [(t, b) for t, b in r.get("bias", ()) if np.isfinite(b)]
    case.lib.bias_values[torch.isinf(case.lib.bias_values)] = 0.0
    for i, r in enumerate(case.rules):
        b, e = int(case.lib.bias_begin[i]), int(case.lib.bias_end[i])
        r["bias"] = list(zip(case.lib.bias_ids[b:e].tolist(), case.lib.bias_values[b:e].tolist()))
    z = case.z.double().cpu().numpy()
    g, e = np.array([1.0, -2.0, 0.5, 0.3]), np.array([0.2, 0.0, -1.0, 0.4])

    def loss(zz):
        lp, H, _ = oracle.changed_logprobs(zz, case.tokens, case.rules)
        return (g * lp).sum() + (e * H).sum()

    lp, H, lse = tim.logits_logprobs(case.z, case.tok, case.lib, lse=True)
    got = tim.logits_logprobs_backward(case.z, case.tok, lse, torch.tensor(g).float().cuda(), case.lib, entropy=H,
                                       grad_entropy=torch.tensor(e).float().cuda()).double().cpu().numpy()
    for i in range(4):
        for v in np.argsort(-np.abs(z[i]))[:10]:
            d = np.zeros_like(z)
            d[i, v] = 1e-5
            assert (loss(z + d) - loss(z - d)) / 2e-5 == pytest.approx(got[i, v], abs=2e-5)


@pytest.mark.parametrize("tau", [1.0, 0.01, 50.0])
def test_temperatures(tau):
    case = Case(6, 3001, 5, history=60, bias=20, masks=4)
    check_adjust(case, tau)
    check_logprobs(case, tau)
    check_backward(case, tau, True)


def test_penalties_one_at_a_time():
    for keep in ("repetition", "frequency", "presence"):
        case = Case(5, 700, 11, history=80)
        for other in {"repetition", "frequency", "presence"} - {keep}:
            setattr(case.lib, other, None)
            for r in case.rules:
                r[other] = 1.0 if other == "repetition" else 0.0
        check_adjust(case, 1.0)
        check_logprobs(case, 1.0)
        check_backward(case, 1.0, False)


def test_no_split_counts_everything_as_output():
    case = Case(5, 700, 12, history=80)
    case.lib.hist_split = None
    for r in case.rules:
        r["output"] = r.pop("prompt") + r["output"]
    check_adjust(case, 1.0)


def test_offsets_out_of_range_and_out_of_order_are_clamped():
    case = Case(6, 300, 13, history=50)
    h = case.lib.history.tolist()
    N = len(h)
    begin = [-5, 10, N - 3, N + 9, 20, -2 ** 62]
    split = [3, 5, N + 7, 0, 25, -9]
    end = [8, 30, 2 ** 62, N + 20, 22, 2 ** 62]
    spans = [(0, 3, 8), (10, 10, 30), (N - 3, N, N), (N, N, N), (20, 25, 25), (0, 0, N)]
    for f, x in (("hist_begin", begin), ("hist_split", split), ("hist_end", end)):
        setattr(case.lib, f, torch.tensor(x, dtype=torch.int64).cuda())
    for r, (b, s, e) in zip(case.rules, spans):
        r["prompt"], r["output"] = h[b:s], h[s:e]
    check_adjust(case, 1.0)
    check_logprobs(case, 1.0)


def test_rows_that_extend_shrink_and_repeat_their_history():
    """Consecutive rows share their counts only where the history grows; every other order recounts. Enough rows that a
    workgroup takes several."""
    T = 8300
    case = Case(T, 97, 14, history=64, packed=True, heavy=True)
    rng = np.random.default_rng(2)
    n = case.lib.history.shape[0]
    begin = np.where(rng.random(T) < 0.9, 5, rng.integers(0, 40, T))
    split = begin + np.where(rng.random(T) < 0.9, 7, rng.integers(0, 9, T))
    end = np.minimum(n, split + np.cumsum(rng.integers(0, 2, T)) % 50)  # grows, falls back, stays
    h = case.lib.history.tolist()
    for f, x in (("hist_begin", begin), ("hist_split", split), ("hist_end", end)):
        setattr(case.lib, f, torch.as_tensor(x.astype(np.int64)).cuda())
    for i, r in enumerate(case.rules):
        r["prompt"], r["output"] = h[begin[i]:split[i]], h[split[i]:end[i]]
    check_adjust(case, 1.0)
    check_logprobs(case, 1.0)


def test_tokens_outside_the_vocabulary_and_masked_tokens():
    case = Case(8, 1000, 15, history=20, masks=4, bias=10)
    case.lib.mask_rows[:] = 2
    for r in case.rules:
        r["allowed"] = np.unpackbits(case.lib.mask[2].cpu().numpy().view(np.uint8), bitorder="little")[:1000] > 0
    off = np.nonzero(~case.rules[0]["allowed"])[0]
    case.tokens[:] = [-1, 1000, 2 ** 31 - 1, -2 ** 31, off[0], off[-1], 0, 999]
    case.tok = torch.as_tensor(case.tokens).cuda()
    lp, _, _ = check_logprobs(case, 0.8)
    assert np.isnan(lp[:4]).all() and np.isneginf(lp[4:6]).all()
    check_backward(case, 0.8, True)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_lowest_values_infinities_and_nan(dtype):
    """Rows of the type's lowest value, of -inf, with +inf or NaN in the open and behind the mask."""
    t = DTYPES[dtype]
    V = 9000
    case = Case(8, V, 16, dtype=t, history=None, masks=1)
    lowest = torch.finfo(t).min
    allowed = np.ones(V, bool)
    allowed[100:200] = False
    words = np.packbits(np.pad(allowed, (0, -V % 32)), bitorder="little").view(np.int32)
    case.lib.mask = torch.as_tensor(words).cuda()[None]
    case.lib.mask_rows = torch.zeros(8, dtype=torch.int32, device="cuda")
    for r in case.rules:
        r["allowed"] = allowed
    case.z[0] = lowest                     # uniform
    case.z[1, 10:] = lowest                # ten entries left
    case.z[2] = -math.inf                  # nothing left
    case.z[3, 7] = -math.inf
    case.z[4, 150] = math.nan              # masked
    case.z[5, 120], case.z[5, 130] = math.inf, -math.inf  # masked
    case.z[6, 50] = math.nan               # in the open
    case.z[7, 8999] = math.inf             # in the open
    case.tokens[:] = [5, 3, 9, 7, 20, 30, 40, 50]
    case.tok = torch.as_tensor(case.tokens).cuda()
    check_adjust(case, 1.0)
    lp, H, lse = (x.cpu() for x in tim.logits_logprobs(case.z, case.tok, case.lib, lse=True))
    n = V - 100
    assert lp[0].item() == pytest.approx(-math.log(n), abs=1e-5) and H[0].item() == pytest.approx(math.log(n), abs=1e-4)
    assert (lp[2].item(), H[2].item(), lse[2].item()) == (-math.inf, 0.0, -math.inf)
    assert lp[3].item() == -math.inf and math.isfinite(H[3].item())
    assert torch.isnan(lp[6:]).all() and torch.isnan(H[6:]).all() and torch.isnan(lse[6]).all()
    z64 = case.z.double().cpu().numpy()
    ref = oracle.changed_logprobs(z64[[1, 3, 4, 5]], case.tokens[[1, 3, 4, 5]], [case.rules[0]] * 4)
    for got, want in zip((lp, H, lse), ref):
        got = got.double().numpy()[[1, 3, 4, 5]]
        fin = np.isfinite(want)
        assert (got[~fin] == want[~fin]).all() and np.allclose(got[fin], want[fin], rtol=1e-6, atol=1e-4)
    g = tim.logits_logprobs_backward(case.z, case.tok, lse.cuda(), torch.ones(8, device="cuda"), case.lib, entropy=H.cuda(),
                                     grad_entropy=torch.full((8,), 0.1, device="cuda"), dtype=torch.float32).cpu()
    assert torch.isfinite(g[:6]).all() and (g[2] == 0).all() and (g[:, 100:200] == 0).all()
    assert g[3, 7] == 1.0  # an entry at -inf: p = 0
    assert torch.isnan(g[6, 0])


@pytest.mark.parametrize("lowest", [-3.4028234663852886e38, -1e30, -65504.0])
def test_additive_masks(lowest):
    """A mask added to the logits as a very low number leaves finite outputs, whatever the temperature."""
    case = Case(3, 5000, 17, history=30)
    case.z[:, 100:] = lowest
    case.tokens[:] = [5, 50, 99]
    case.tok = torch.as_tensor(case.tokens).cuda()
    for tau in (0.1, 1.0):
        lp, H, lse = tim.logits_logprobs(case.z, case.tok, case.lib, tau, lse=True)
        assert torch.isfinite(lp).all() and torch.isfinite(H).all() and torch.isfinite(lse).all()
        g = tim.logits_logprobs_backward(case.z, case.tok, lse, torch.ones(3, device="cuda"), case.lib, tau, entropy=H,
                                         grad_entropy=torch.ones(3, device="cuda"))
        assert torch.isfinite(g).all() and (g[:, 200:] == 0).all()


def test_rows_do_not_depend_on_the_batch():
    """Outputs of a row have the same bits in any batch, position, stride and order of the history's use."""
    T, V = 700, 17001
    case = Case(T, V, 18, history=90, packed=True, bias=20, masks=5, pad=2)
    whole = tim.logits_logprobs(case.z, case.tok, case.lib, 0.7, lse=True)
    adj = tim.logits_adjust(case.z, case.lib, 0.7)
    g = torch.randn(T, device="cuda")
    grad = tim.logits_logprobs_backward(case.z, case.tok, whole[2], g, case.lib, 0.7)
    for a, b in ((0, 1), (699, 700), (17, 300)):
        part = case.z[a:b].contiguous()
        rules = case.rows(a, b)
        for x, y in zip(tim.logits_logprobs(part, case.tok[a:b], rules, 0.7, lse=True), whole):
            assert torch.equal(x.view(torch.int32), y[a:b].view(torch.int32))
        assert torch.equal(tim.logits_adjust(part, rules, 0.7), adj[a:b])
        out = tim.logits_logprobs_backward(part, case.tok[a:b], whole[2][a:b], g[a:b], rules, 0.7)
        assert torch.equal(out, grad[a:b])


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_in_place_and_padded_outputs(dtype):
    t = DTYPES[dtype]
    case = Case(50, 9003, 19, dtype=t, history=40, bias=10, masks=3)
    want = tim.logits_adjust(case.z, case.lib, 0.9)
    _, H, lse = tim.logits_logprobs(case.z, case.tok, case.lib, 0.9, lse=True)
    g = torch.randn(50, device="cuda")
    grad = tim.logits_logprobs_backward(case.z, case.tok, lse, g, case.lib, 0.9)
    wide = torch.full((52, 9010), 7.0, dtype=t, device="cuda")
    tim.logits_adjust(case.z, case.lib, 0.9, out=wide[1:51, 3:9006])
    assert torch.equal(wide[1:51, 3:9006], want)
    wide[1:51, 3:9006] = 7.0
    assert (wide == 7.0).all()
    tim.logits_logprobs_backward(case.z, case.tok, lse, g, case.lib, 0.9, out=wide[1:51, 3:9006])
    assert torch.equal(wide[1:51, 3:9006], grad)
    wide[1:51, 3:9006] = 7.0
    assert (wide == 7.0).all()
    z = case.z.clone()
    assert tim.logits_logprobs_backward(z, case.tok, lse, g, case.lib, 0.9, out=z) is z and torch.equal(z, grad)
    z = case.z.clone()
    assert tim.logits_adjust(z, case.lib, 0.9, out=z) is z and torch.equal(z, want)


def test_optional_outputs():
    case = Case(7, 500, 20)
    lp, H, lse = tim.logits_logprobs(case.z, case.tok, case.lib, lse=True)
    a = tim.logits_logprobs(case.z, case.tok, case.lib, entropy=False)
    assert torch.equal(a[0], lp) and a[1] is None and a[2] is None
    out = (torch.empty(7, device="cuda"), None, torch.empty(7, device="cuda"))
    tim.logits_logprobs(case.z, case.tok, case.lib, out=out)
    assert torch.equal(out[0], lp) and torch.equal(out[2], lse)


def test_no_rows():
    z = torch.empty(0, 100, device="cuda")
    tok = torch.empty(0, dtype=torch.int32, device="cuda")
    assert tim.logits_adjust(z).shape == (0, 100)
    assert tim.logits_logprobs(z, tok)[0].shape == (0,)
    e = torch.empty(0, device="cuda")
    assert tim.logits_logprobs_backward(z, tok, e, e).shape == (0, 100)


def test_padded_batch_rows_get_zeros_whatever_they_hold():
    """Rows of padding (token -1, no upstream gradient) hold NaN: their gradients are zeros, the others untouched."""
    case = Case(6, 2000, 21, history=30)
    _, H, lse = tim.logits_logprobs(case.z, case.tok, case.lib, lse=True)
    g = torch.randn(6, device="cuda")
    want = tim.logits_logprobs_backward(case.z, case.tok, lse, g, case.lib)
    case.z[4:] = math.nan
    lse[4:] = math.nan
    case.tok[4:] = -1
    got = tim.logits_logprobs_backward(case.z, case.tok, lse, g, case.lib)
    assert torch.equal(got[:4], want[:4]) and (got[4:] == 0).all()


def test_long_history():
    """One row with 300000 tokens, most of them one token: its count passes 16 bits."""
    V = 12000
    case = Case(2, V, 22, history=10)
    n = 300000
    h = torch.full((n,), 77, dtype=torch.int32)
    h[::3] = torch.randint(0, V, (n // 3,), dtype=torch.int32, generator=torch.Generator().manual_seed(1))
    case.lib.history = h.cuda()
    spans = [(0, 1000, n), (5, 5, 70000)]
    for j, f in enumerate(("hist_begin", "hist_split", "hist_end")):
        setattr(case.lib, f, torch.tensor([s[j] for s in spans], dtype=torch.int64).cuda())
    for r, (b, s, e) in zip(case.rules, spans):
        r["prompt"], r["output"] = h[b:s].tolist(), h[s:e].tolist()
        r["frequency"] = 2.0 ** -14
    case.lib.frequency[:] = 2.0 ** -14
    check_adjust(case, 1.0)


def test_largest_vocabulary():
    V = tim.MAX_VOCAB
    case = Case(2, V, 23, history=500, bias=50, masks=3)
    check_adjust(case, 1.0)
    check_logprobs(case, 1.0)
    check_backward(case, 1.0, True)


def test_rows_past_32_bit_offsets():
    """A matrix of more than 2^32 bytes and 2^31 elements: the last rows against the same rows alone."""
    T, V = 14500, 151936
    z = torch.empty(T, V, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    for a in (0, T - 3):
        z[a:a + 3] = torch.randn(3, V, generator=g, device="cuda").to(torch.bfloat16)
    z[3:T - 3] = 0.0
    tok = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    whole = tim.logits_logprobs(z, tok, lse=True)
    alone = tim.logits_logprobs(z[T - 3:].clone(), tok[T - 3:], lse=True)
    for a, b in zip(whole, alone):
        assert torch.equal(a[T - 3:], b)
    assert torch.equal(tim.logits_adjust(z, None, 0.5)[T - 3:], tim.logits_adjust(z[T - 3:].clone(), None, 0.5))


def _packed_rules(T, V, seed, masks):
    """Histories of many short responses in one stream, some rows out of order, as tensors only."""
    g = torch.Generator().manual_seed(seed)
    n = T + 100
    resp = torch.randint(1, 30, (T,), generator=g)
    start = torch.cumsum(resp, 0) - resp
    row = torch.arange(T)
    first = torch.searchsorted(start, row, right=True) - 1
    begin = start[first]
    end = row.clone()
    odd = torch.rand(T, generator=g) < 0.03
    end[odd] = begin[odd] + torch.randint(0, 40, (int(odd.sum()),), generator=g)
    split = begin + torch.randint(0, 3, (T,), generator=g)[first]
    kw = dict(history=torch.randint(0, V, (n,), dtype=torch.int32, generator=g), hist_begin=begin, hist_split=split,
              hist_end=end, repetition=0.5 + torch.rand(T, generator=g), frequency=torch.rand(T, generator=g),
              presence=torch.rand(T, generator=g), bias_ids=torch.randint(0, V, (50,), dtype=torch.int32, generator=g),
              bias_values=torch.randn(50, generator=g), bias_begin=first % 40, bias_end=first % 40 + first % 7)
    if masks:
        kw["mask"] = torch.randint(-2 ** 31, 2 ** 31, (T, (V + 31) // 32), dtype=torch.int64, generator=g).to(torch.int32)
    return {k: v.cuda() for k, v in kw.items()}


def _slice(kw, a, b):
    rows = ("hist_begin", "hist_split", "hist_end", "repetition", "frequency", "presence", "bias_begin", "bias_end", "mask")
    return tim.LogitRules(**{k: v[a:b].contiguous() if k in rows else v for k, v in kw.items()})


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_many_rows_to_a_workgroup(dtype):
    """Rows enough for sixteen to a workgroup give the bits of calls with one row to each."""
    T, V = 70001, 67
    kw = _packed_rules(T, V, 31, True)
    z = torch.randn(T, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(DTYPES[dtype])
    tok = torch.randint(-1, V, (T,), device="cuda", dtype=torch.int32)
    g = torch.randn(T, device="cuda")
    g[::11] = 0.0
    adj = tim.logits_adjust(z, _slice(kw, 0, T), 0.8)
    lp, H, lse = tim.logits_logprobs(z, tok, _slice(kw, 0, T), 0.8, lse=True)
    dz = tim.logits_logprobs_backward(z, tok, lse, g, _slice(kw, 0, T), 0.8)
    for a in range(0, T, 4000):
        b = min(T, a + 4000)
        r = _slice(kw, a, b)
        assert torch.equal(tim.logits_adjust(z[a:b], r, 0.8), adj[a:b])
        for x, y in zip(tim.logits_logprobs(z[a:b], tok[a:b], r, 0.8, lse=True), (lp, H, lse)):
            assert torch.equal(x.view(torch.int32), y[a:b].view(torch.int32))
        assert torch.equal(tim.logits_logprobs_backward(z[a:b], tok[a:b], lse[a:b], g[a:b], r, 0.8), dz[a:b])


def test_more_rows_than_a_launch():
    """More rows than one launch takes (2^22 of one chunk), each with a mask of its own: the last rows against the same
    rows alone."""
    T, V = (1 << 22) + 5000, 5
    kw = _packed_rules(T, V, 32, True)
    z = torch.randn(T, V, device="cuda")
    tok = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    g = torch.randn(T, device="cuda")
    adj = tim.logits_adjust(z, _slice(kw, 0, T))
    whole = tim.logits_logprobs(z, tok, _slice(kw, 0, T), lse=True)
    dz = tim.logits_logprobs_backward(z, tok, whole[2], g, _slice(kw, 0, T))
    for a, b in ((0, 100), ((1 << 22) - 50, (1 << 22) + 50), (T - 100, T)):
        r = _slice(kw, a, b)
        assert torch.equal(tim.logits_adjust(z[a:b], r), adj[a:b])
        for x, y in zip(tim.logits_logprobs(z[a:b], tok[a:b], r, lse=True), whole):
            assert torch.equal(x.view(torch.int32), y[a:b].view(torch.int32))
        assert torch.equal(tim.logits_logprobs_backward(z[a:b], tok[a:b], whole[2][a:b], g[a:b], r), dz[a:b])


def test_a_bias_for_the_whole_vocabulary():
    """A list of every id, twice: the second entry of each wins."""
    V = 20001
    case = Case(2, V, 33, history=20)
    ids = torch.cat([torch.randperm(V, generator=torch.Generator().manual_seed(k)) for k in (1, 2)]).to(torch.int32)
    vals = torch.randn(2 * V, generator=torch.Generator().manual_seed(3))
    case.lib.bias_ids, case.lib.bias_values = ids.cuda(), vals.cuda()
    case.lib.bias_begin = torch.tensor([0, 7], device="cuda")
    case.lib.bias_end = torch.tensor([2 * V, V + 7], device="cuda")
    for r, (b, e) in zip(case.rules, ((0, 2 * V), (7, V + 7))):
        r["bias"] = list(zip(ids[b:e].tolist(), vals[b:e].tolist()))
    check_adjust(case, 0.7)
    check_logprobs(case, 0.7)
    check_backward(case, 0.7, True)


def test_empty_rules():
    """A rule set without anything, or with empty arrays, changes nothing but the temperature."""
    z = torch.randn(3, 100, device="cuda")
    none = torch.zeros(3, dtype=torch.int64, device="cuda")
    empty = tim.LogitRules(history=torch.empty(0, dtype=torch.int32, device="cuda"), hist_begin=none, hist_end=none,
                           repetition=torch.full((3,), 2.0, device="cuda"),
                           bias_ids=torch.empty(0, dtype=torch.int32, device="cuda"),
                           bias_values=torch.empty(0, device="cuda"), bias_begin=none, bias_end=none,
                           mask=torch.empty((0, 4), dtype=torch.int32, device="cuda"),
                           mask_rows=torch.zeros(3, dtype=torch.int32, device="cuda"))
    want = tim.logits_adjust(z, None, 0.5)
    assert torch.equal(tim.logits_adjust(z, empty, 0.5), want) and torch.equal(want, z * 2.0)
    assert torch.equal(tim.logits_adjust(z, tim.LogitRules(), 0.5), want)


@pytest.mark.parametrize("dtype,grad,T,V", [("f32", "f32", 570, 120001), ("bf16", "f32", 570, 120003),
                                            ("f32", "bf16", 1200, 120001), ("f16", "f16", 1150, 120002)])
def test_outputs_larger_than_the_caches(dtype, grad, T, V):
    """Outputs of more than 256 MB in rows of odd lengths: the same bits as the rows a few at a time."""
    kw = _packed_rules(T, V, 34, False)
    gen = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randn(T, V, device="cuda", generator=gen).to(DTYPES[dtype])
    tok = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=gen)
    g, e = (torch.randn(T, device="cuda", generator=gen) for _ in range(2))
    r = _slice(kw, 0, T)
    _, H, lse = tim.logits_logprobs(z, tok, r, 0.9, lse=True)
    dz = tim.logits_logprobs_backward(z, tok, lse, g, r, 0.9, entropy=H, grad_entropy=e, dtype=DTYPES[grad])
    adj = tim.logits_adjust(z, r, 0.9)
    for a, b in ((0, 5), (T // 2, T // 2 + 3), (T - 7, T)):
        r = _slice(kw, a, b)
        assert torch.equal(tim.logits_adjust(z[a:b], r, 0.9), adj[a:b])
        assert torch.equal(tim.logits_logprobs_backward(z[a:b], tok[a:b], lse[a:b], g[a:b], r, 0.9, entropy=H[a:b],
                                                        grad_entropy=e[a:b], dtype=DTYPES[grad]), dz[a:b])


# Rows far from 0. lse holds its row's normaliser to |lse| 2^-24 only, so from |lse| = 1024 on the gradient forms it anew
# from the logits, as their largest y and log S. Without penalties and biases y is exact there, and p off by what S and
# the exponentials are: S is a sum of V / 512 < 42 terms a thread, each step an exponential, a product and an addition,
# then 17 additions and the logarithm, its exponentials within (2 + 2 |t|) u and a p-weighted mean of |t| below
# ln V + 1 < 12: at most (3 * 42 + 17 + 8 + 26) u < 180 u. With penalties and biases every y is within 6 u M of its exact
# value, and so is the softmax average of them. Short of 1024 the given lse's half step enters p instead.


def check_far_backward(case, tau, entropy, grad=None, **kw):
    rng = np.random.default_rng(case.T + 7)
    g = rng.standard_normal(case.T).astype(np.float32)
    e = rng.standard_normal(case.T).astype(np.float32) if entropy else None
    inv = float(np.float32(1.0 / np.float64(np.float32(tau))))
    z64 = case.z.double().cpu().numpy()
    _, H, lse64 = oracle.changed_logprobs(z64, case.tokens, case.rules, 1.0 / inv)
    with np.errstate(over="ignore"):
        lse = lse64.astype(np.float32)  # infinite past fp32's range
    as_gpu = lambda x: None if x is None else torch.as_tensor(x.astype(np.float32)).cuda()  # noqa: E731
    x, slope = oracle.change_logits(z64, case.rules, 1.0 / inv)
    ref = oracle.changed_logprobs_grad(z64, case.tokens, case.rules, g, e, 1.0 / inv)
    changed = any(r.get("prompt") or r.get("output") or r.get("bias") for r in case.rules)
    _, top = fp32_steps(case, case.z, tau)
    got = tim.logits_logprobs_backward(case.z, case.tok, as_gpu(lse), as_gpu(g), case.lib, tau, entropy=as_gpu(H),
                                       grad_entropy=as_gpu(e), dtype=grad, **kw)
    D = 12 * U * top * inv if changed else np.zeros(case.T)
    D = (D + np.where(np.abs(lse64) < 1024.5, np.abs(lse64), 0) * U + 180 * U)[:, None]
    none = np.isneginf(x).all(1)[:, None]
    with np.errstate(invalid="ignore", divide="ignore"):
        m = x.max(1, keepdims=True)
        q = np.where(np.isfinite(x) & ~none, x - m - np.log(np.exp(x - m).sum(1, keepdims=True)), 0.0)
    p = np.where(np.isfinite(x) & ~none, np.exp(q), 0.0)
    a = np.abs(g)[:, None] + (0.0 if e is None else np.abs(e)[:, None]) * (np.abs(q) + np.abs(H)[:, None] + 1)
    onehot = np.zeros_like(z64)
    ok = (case.tokens >= 0) & (case.tokens < case.V)
    onehot[np.nonzero(ok)[0], case.tokens[ok]] = 1.0
    bound = slope * (p * a * (D + (4 * np.abs(q) + 12) * U) + 4 * U * np.abs(g)[:, None] * onehot) + 4 * U * np.abs(ref)
    bound += slope * a * 2.0 ** -126
    bound += torch.finfo(got.dtype).eps / 2 * (np.abs(ref) + bound) + TINY[got.dtype]
    err = np.abs(got.double().cpu().numpy() - ref)
    assert np.isfinite(err).all()
    print(f"[parity] far grad: max|err| {err.max():.2e}, {np.max(err / bound):.3f} of the bound")
    assert (err <= bound).all(), np.argwhere(err > bound)[:5]
    return got, g


@pytest.mark.parametrize("tau", [1.0, 0.7, 0.3])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_gradient_of_rows_of_lowest_values(dtype, tau):
    """Rows of the type's lowest and largest value: p is 1 / n, also where lse holds no log n or is past fp32's range."""
    V, n = 20003, 20003 - 9000
    case = Case(6, V, 41, dtype=DTYPES[dtype], history=None, masks=2)
    allowed = np.ones(V, bool)
    allowed[100:9100] = False
    for m, bits in ((0, allowed), (1, np.zeros(V, bool))):
        case.lib.mask[m] = torch.as_tensor(np.packbits(np.pad(bits, (0, case.lib.mask.shape[1] * 32 - V)),
                                                       bitorder="little").view(np.int32)).cuda()
    lowest = torch.finfo(DTYPES[dtype]).min
    case.z[0] = lowest
    case.z[1] = lowest
    case.z[2] = -lowest
    case.z[3] = lowest
    case.z[3, 9500:9510] = lowest / 2      # ten entries left
    case.z[4] = -math.inf                  # nothing left
    case.z[5] = lowest                     # nothing allowed
    case.lib.mask_rows[:] = torch.tensor([0, -1, 0, 0, 0, 1], dtype=torch.int32)
    for r, m in zip(case.rules, (allowed, None, allowed, allowed, allowed, np.zeros(V, bool))):
        r.pop("allowed", None)
        if m is not None:
            r["allowed"] = m
    case.tokens[:] = [5, 30, 20002, 9501, 3, 4]
    case.tok = torch.as_tensor(case.tokens).cuda()
    lp, H, lse = (x.double().cpu() for x in tim.logits_logprobs(case.z, case.tok, case.lib, tau, lse=True))
    assert lp[0].item() == pytest.approx(-math.log(n), abs=1e-5) and H[0].item() == pytest.approx(math.log(n), abs=1e-4)
    for entropy in (False, True):
        got, g = check_far_backward(case, tau, entropy, grad=torch.float32)
        if not entropy:  # each row's gradient sums to 0, each of its entries within the bound above of p g / tau
            for i in range(4):
                assert abs(got[i].double().sum().item()) <= 600 * U * abs(g[i]) / tau
        assert (got[4:] == 0).all() and (got[0, 100:9100] == 0).all()


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("V", [1, 700, 8193, 20003])
def test_gradient_of_rows_far_from_zero(dtype, grad, V):
    """Offsets common to a row, on both sides of where lse becomes too coarse: the gradient does not feel them."""
    offsets = [0.0, 900.0, 1020.0, -1020.0, 1030.0, -1030.0, 5000.0, -20000.0]
    if dtype != "f16":
        offsets += [1e5, -1e6, 3e7, -1e12]
    print(f"case {dtype} -> {grad} V={V}", flush=True)
    case = Case(len(offsets), V, 42, dtype=DTYPES[dtype], history=None, masks=3, pad=1)
    case.z += torch.tensor(offsets, device="cuda")[:, None].to(case.z.dtype)
    for entropy in (False, True):
        check_far_backward(case, 0.9, entropy, grad=DTYPES[grad])


@pytest.mark.parametrize("bias", [0, 30])
@pytest.mark.parametrize("V", [500, 20003])
def test_gradient_of_changed_rows_far_from_zero(V, bias):
    """Penalties, biases and masks on rows at an offset, whose changes are of its size."""
    case = Case(9, V, 43, history=60, bias=bias, masks=5)
    case.z[::2] += 3000.0
    case.z[1::4] -= 3000.0
    for entropy in (False, True):
        check_far_backward(case, 1.0, entropy)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_far_rows_beside_others_in_a_workgroup(dtype):
    """Far, padded, empty and ordinary rows in turn, several to a workgroup, their histories extending one another: each
    row has the bits it has alone, in place too."""
    T, V = 4200, 17001
    kw = _packed_rules(T, V, 44, True)
    kw["mask"][10::97] = 0
    gen = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn(T, V, device="cuda", generator=gen)
    z[::5] += 4000.0
    z[2::7] -= 4000.0
    z = z.to(DTYPES[dtype])
    tok = torch.randint(-1, V, (T,), device="cuda", dtype=torch.int32, generator=gen)
    g, e = (torch.randn(T, device="cuda", generator=gen) for _ in range(2))
    g[::11] = 0.0
    e[::11] = 0.0
    r = _slice(kw, 0, T)
    _, H, lse = tim.logits_logprobs(z, tok, r, 0.9, lse=True)
    assert (lse.abs() > 1024).sum() > T // 4 and torch.isinf(lse).sum() > T // 100
    dz = tim.logits_logprobs_backward(z, tok, lse, g, r, 0.9, entropy=H, grad_entropy=e)
    assert torch.isfinite(dz).all()
    for a in (0, 1, 2, 5, 10, 11, 2000, 2005, 2100, T - 3):
        one = tim.logits_logprobs_backward(z[a:a + 1], tok[a:a + 1], lse[a:a + 1], g[a:a + 1], _slice(kw, a, a + 1), 0.9,
                                           entropy=H[a:a + 1], grad_entropy=e[a:a + 1])
        assert torch.equal(one, dz[a:a + 1]), a
    for a in range(0, T, 600):
        part = _slice(kw, a, a + 600)
        assert torch.equal(tim.logits_logprobs_backward(z[a:a + 600], tok[a:a + 600], lse[a:a + 600], g[a:a + 600], part,
                                                        0.9, entropy=H[a:a + 600], grad_entropy=e[a:a + 600]),
                           dz[a:a + 600]), a
    tim.logits_logprobs_backward(z, tok, lse, g, r, 0.9, entropy=H, grad_entropy=e, out=z)
    assert torch.equal(z, dz)


def test_biases_before_the_penalties_by_two_calls():
    """The other order of bias and penalties: a call with the bias alone, the rest on its fp32 output."""
    case = Case(7, 9001, 45, history=80, bias=30, masks=4, scale=1.0)
    bias = tim.LogitRules(**{f: getattr(case.lib, f) for f in ("bias_ids", "bias_values", "bias_begin", "bias_end")})
    first = tim.logits_adjust(case.z, bias)
    want = case.z.cpu().numpy().copy()
    for row, r in zip(want, case.rules):
        for t, b in dict(r.pop("bias", ())).items():
            if 0 <= t < case.V:
                row[t] = row[t] + np.float32(b)
    assert torch.equal(first.cpu(), torch.as_tensor(want))
    one = tim.logits_adjust(case.z, case.lib, 0.7)
    case.z = first
    for f in ("bias_ids", "bias_values", "bias_begin", "bias_end"):
        setattr(case.lib, f, None)
    assert not torch.equal(check_adjust(case, 0.7), one.cpu())
    check_logprobs(case, 0.7)
    check_backward(case, 0.7, True)


def test_far_rows_captured_and_on_two_streams():
    """A captured gradient whose rows become far and near between replays, and two at once, give the eager bits."""
    T, V = 40, 17001
    kw = _packed_rules(T, V, 46, True)
    rules, gen = _slice(kw, 0, T), torch.Generator(device="cuda").manual_seed(4)
    base = torch.randn(T, V, device="cuda", generator=gen)
    z, tok = base.clone(), torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=gen)
    g, e = (torch.randn(T, device="cuda", generator=gen) for _ in range(2))
    out = tuple(torch.empty(T, device="cuda") for _ in range(3))
    ws = torch.empty(tim.logits_logprobs_workspace_size(T, V), dtype=torch.uint8, device="cuda")
    dz = torch.empty_like(z)

    def step(z, out, ws, dz):
        tim.logits_logprobs(z, tok, rules, 0.8, workspace=ws, out=out)
        tim.logits_logprobs_backward(z, tok, out[2], g, rules, 0.8, entropy=out[1], grad_entropy=e, out=dz)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(z, out, ws, dz)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(z, out, ws, dz)
    other = [(torch.empty_like(z), tuple(torch.empty_like(t) for t in out), torch.empty_like(ws), torch.empty_like(dz))
             for _ in range(3)]
    for k in range(4):
        z.copy_(base + 5000.0 * ((torch.arange(T, device="cuda") + k) % 3 - 1)[:, None])
        for a in other:
            a[0].copy_(z)
        step(*other[0])
        want = other[0][3].clone()
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(dz, want), k
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for s, a in zip(streams, other[1:]):
            with torch.cuda.stream(s):
                step(*a)
        torch.cuda.synchronize()
        assert all(torch.equal(a[3], want) for a in other[1:]), k
