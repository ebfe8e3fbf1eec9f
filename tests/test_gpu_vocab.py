"""The embedding, the adapters and the calls beside them together, as a rollout engine and a trainer make them: a tied
model's tail with adapters on its head, captured and replayed, on two streams, on tensors of another stream, through
autograd, and with tensors that change in place."""

import numpy as np
import pytest
import torch

import oracle
import paper_2605_14220_amd as tim
from tim_testutil import bits_equal, require_gpu

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _model(T=96, d=256, V=3000, n=3, r=8, seed=0):
    g = torch.Generator().manual_seed(seed)
    m = dict(W=(0.05 * torch.randn(V, d, generator=g)).to(BF16).cuda(),
             gamma=(1 + 0.1 * torch.randn(d, generator=g)).to(BF16).cuda(),
             a=(torch.randn(n, r, d, generator=g) / d ** 0.5).to(BF16).cuda(),
             b=(0.05 * torch.randn(n, V, r, generator=g)).to(BF16).cuda(),
             s=(torch.rand(n, generator=g) + 0.5).cuda(),
             inp=torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda(),
             out=torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda(),
             rows=(torch.arange(T) * (n + 1) // T - 1).to(torch.int32).cuda(),
             g=torch.randn(T, generator=g).cuda())
    m["inp"][-3:] = -1  # padding
    m["ad"] = tim.Adapters(m["a"], m["b"], m["s"])
    return m


def _step(m, grad_w):
    """Forward and backward of embedding -> norm -> tied head with adapters -> log-probs."""
    x = tim.embedding(m["W"], m["inp"], 16.0)
    h, rstd = tim.rmsnorm(x, m["gamma"])
    z = tim.logits(h, m["W"])
    y = tim.adapters_add(z, h, m["rows"], m["ad"])
    logp, _, lse = tim.logits_logprobs(y, m["out"], lse=True)
    dy = tim.logits_logprobs_backward(y, m["out"], lse, m["g"], dtype=BF16)
    gh = dy.float() @ m["W"].float()
    base = gh.clone()
    tim.adapters_backward(dy, h, m["rows"], m["ad"], grad_x=gh, accumulate_x=True, grad_a=m.get("ga"), grad_b=m.get("gb"))
    _, ga, gb = tim.adapters_backward(dy, h, m["rows"], m["ad"], want_x=False)
    gx, _ = tim.rmsnorm_backward(x, m["gamma"], rstd, gh)
    torch.mm(dy.float().T, h.float(), out=grad_w)
    head = grad_w.clone()
    tim.embedding_backward(gx, m["inp"], m["W"].shape[0], 16.0, grad_table=grad_w, accumulate=True)
    return dict(x=x, h=h, z=z, y=y, logp=logp, dy=dy, base=base, gh=gh, ga=ga, gb=gb, gx=gx, head=head, grad_w=grad_w)


def _np(t):
    return t.detach().double().cpu().numpy()


def test_tied_model_with_adapters():
    """Each new stage against the oracle on the tensors it was given, within the bounds of its own tests: out and grad_h
    (d or V + r + 3) 2^-23 of the magnitudes, grad_a (V + T + 3), grad_b (d + T + 3), the embedding's gradient
    (n + 2) 2^-24, each with its type's half step. The log-probs' error is at most twice the logits'."""
    m = _model()
    V, d = m["W"].shape
    T, r = len(m["inp"]), m["a"].shape[1]
    t = _step(m, torch.empty(V, d, device="cuda"))
    rows, slack = m["rows"].cpu().numpy(), 1 + 2.0 ** -8
    A, B, S = _np(m["a"]), _np(m["b"]), _np(m["s"])

    def near(got, want, size, terms, eps=2.0 ** -24):
        assert (np.abs(_np(got) - want) <= (terms * 2.0 ** -23 * size + eps * np.abs(want)) * slack).all()

    e = oracle.embedding(_np(m["W"]), m["inp"].cpu().numpy(), 16.0)
    assert np.array_equal(_np(t["x"]), e)  # a power of two
    want, size = oracle.adapters_add(_np(t["z"]), _np(t["h"]), rows, A, B, S)
    near(t["y"], want, size, d + r + 3)
    zref = torch.as_tensor(want)
    lp = torch.log_softmax(zref, 1).gather(1, m["out"].cpu().long()[:, None])[:, 0].numpy()
    worst = ((d + r + 3) * 2.0 ** -23 * size + 2.0 ** -24 * np.abs(want)).max() * slack
    # beside the logits' error that of the log-probs' own fp32 statistics: V terms, and the values' rounding
    assert np.abs(_np(t["logp"]) - lp).max() <= 2 * worst + 1e-5 + 2.0 ** -22 * np.abs(lp).max()
    (wx, wa, wb), (sx, sa, sb) = oracle.adapters_backward(_np(t["dy"]), _np(t["h"]), rows, A, B, S)
    near(t["gh"], _np(t["base"]) + wx, np.abs(_np(t["base"])) + sx, V + r + 3)
    near(t["ga"], wa, sa, V + T + 3)
    near(t["gb"], wb, sb, d + T + 3)
    we, se, n = oracle.embedding_backward(_np(t["gx"]), m["inp"].cpu().numpy(), V, 16.0)
    old = _np(t["head"])
    bound = (n + 2)[:, None] * 2.0 ** -24 * (se + np.abs(old)) * slack
    assert (np.abs(_np(t["grad_w"]) - (old + we)) <= bound).all()
    assert np.array_equal(_np(t["grad_w"])[n == 0], old[n == 0])


def test_quantised_head_with_adapters():
    """Adapters beside the logits of a 4-bit head, in place."""
    m = _model()
    h, _ = tim.rmsnorm(tim.embedding(m["W"], m["inp"].clamp(min=0), 16.0), m["gamma"])
    z = tim.mxfp4_logits(tim.mxfp4_quantize(h), tim.mxfp4_quantize(m["W"]))
    want, size = oracle.adapters_add(_np(z), _np(h), m["rows"].cpu().numpy(), _np(m["a"]), _np(m["b"]), _np(m["s"]))
    y = tim.adapters_add(z, h, m["rows"], m["ad"], out=z)
    assert y is z
    assert (np.abs(_np(y) - want) <= (256 + 8 + 3) * 2.0 ** -23 * size * (1 + 2.0 ** -8) + 2.0 ** -23 * np.abs(want)).all()


SMALL, LARGE = dict(T=70, n=3, r=8), dict(T=1500, n=2, r=20)  # rows by themselves beside the grouping; grouped first


@pytest.mark.parametrize("sizes", [SMALL, LARGE])
def test_captured_and_replayed(sizes):
    """A graph of all four calls, replayed with other inputs in the same buffers, with eager work between the replays."""
    m = _model(V=1000, **sizes)
    T, d, V = len(m["inp"]), 256, 1000
    n, r = m["a"].shape[:2]
    z, dy = torch.randn(T, V, device="cuda"), torch.randn(T, V, device="cuda").to(BF16)
    ws = [torch.empty(s, dtype=torch.uint8, device="cuda") for s in
          (tim.embedding_backward_workspace_size(T, V, d), tim.adapters_add_workspace_size(T, d, V, n, r),
           tim.adapters_backward_workspace_size(T, d, V, n, r))]
    out = dict(x=torch.empty(T, d, dtype=BF16, device="cuda"), y=torch.empty_like(z),
               gx=torch.empty(T, d, device="cuda"), ga=torch.empty(n, r, d, device="cuda"),
               gb=torch.empty(n, V, r, device="cuda"), gw=torch.empty(V, d, device="cuda"))

    def calls(o, ws):
        tim.embedding(m["W"], m["inp"], 2.0, out=o["x"])
        tim.adapters_add(z, o["x"], m["rows"], m["ad"], out=o["y"], workspace=ws[1])
        tim.adapters_backward(dy, o["x"], m["rows"], m["ad"], grad_x=o["gx"], grad_a=o["ga"], grad_b=o["gb"],
                              workspace=ws[2])
        tim.embedding_backward(o["gx"], m["inp"], V, 2.0, grad_table=o["gw"], workspace=ws[0])
        tim.embedding_backward(o["gx"], m["inp"], V, 2.0, grad_table=o["gw"], accumulate=True, workspace=ws[0])

    calls(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(out, ws)
    g = torch.Generator(device="cuda").manual_seed(1)
    for k in range(4):
        m["inp"].copy_(torch.randint(-1, V, (T,), generator=g, device="cuda"))
        m["rows"].copy_(torch.randint(-1, n, (T,), generator=g, device="cuda") if k < 3 else torch.full((T,), -1))
        z.copy_(torch.randn(T, V, generator=g, device="cuda"))
        eager = {f: torch.empty_like(t) for f, t in out.items()}
        calls(eager, [torch.empty_like(w) for w in ws])
        for t in out.values():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for f in out:
            assert torch.equal(out[f], eager[f]), (k, f)


def test_two_streams():
    """Calls on two streams at once, each with its own workspace, whose inputs are made there."""
    ms = [_model(seed=s, T=t) for s, t in ((1, 90), (2, 2000))]
    want = [_step(m, torch.empty(m["W"].shape, device="cuda")) for m in ms]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for m, s in zip(ms, streams):
            with torch.cuda.stream(s):
                got.append(_step(m, torch.empty(m["W"].shape, device="cuda")))
        torch.cuda.synchronize()
        for w, t in zip(want, got):
            for f in ("y", "gh", "ga", "gb", "gx"):
                assert torch.equal(w[f], t[f]), f


def test_repeated_calls_give_the_same_bits():
    m = _model(T=1800, n=2, r=40)
    dy = torch.randn(1800, 3000, device="cuda").to(BF16)
    x = tim.embedding(m["W"], m["inp"])
    first = None
    for _ in range(3):
        got = tim.adapters_backward(dy, x, m["rows"], m["ad"], dtype=F32)
        table = tim.embedding_backward(got[0], m["inp"] % 50, 3000)
        if first is None:
            first = (*got, table)
        for a, b in zip(first, (*got, table)):
            assert bits_equal(a, b)


def test_adapters_that_change():
    """New values in the same tensors are read; another tensor, type or size in a field is checked anew."""
    m = _model(T=20)
    x = tim.embedding(m["W"], m["inp"])
    y0 = tim.adapters_add(None, x, m["rows"], m["ad"], dtype=F32)
    m["b"].mul_(2)
    assert torch.equal(tim.adapters_add(None, x, m["rows"], m["ad"], dtype=F32), 2 * y0)
    m["ad"].scales = None
    want = tim.adapters_add(None, x, m["rows"], tim.Adapters(m["a"], m["b"]), dtype=F32)
    assert torch.equal(tim.adapters_add(None, x, m["rows"], m["ad"], dtype=F32), want)
    m["ad"].b = m["b"][:2]
    with pytest.raises(ValueError):
        tim.adapters_add(None, x, m["rows"], m["ad"])
    m["ad"].a = m["a"][:2]
    got = tim.adapters_add(None, x, m["rows"], m["ad"], dtype=F32)
    keep = m["rows"] < 2
    assert torch.equal(got[keep], want[keep]) and (got[~keep] == 0).all()
    m["ad"].a = m["a"][:2].half()
    with pytest.raises(TypeError):
        tim.adapters_add(None, x, m["rows"], m["ad"])


class _Adapt(torch.autograd.Function):
    @staticmethod
    def forward(ctx, base, x, a, b, scales, rows):
        ctx.save_for_backward(x, a, b, scales, rows)
        return tim.adapters_add(base, x, rows, tim.Adapters(a, b, scales))

    @staticmethod
    def backward(ctx, g):
        x, a, b, scales, rows = ctx.saved_tensors
        gx, ga, gb = tim.adapters_backward(g.contiguous(), x, rows, tim.Adapters(a, b, scales))
        return g, gx, ga.to(a.dtype), gb.to(b.dtype), None, None


def test_through_autograd():
    """Whole numbers, so that the gradients of a quadratic loss equal float64 autograd's through the textbook form."""
    g = torch.Generator().manual_seed(7)
    T, d, N, n, r = 30, 6, 9, 2, 2
    ints = lambda *s: torch.randint(-1, 2, s, generator=g).float()
    x, a, b, base = ints(T, d), ints(n, r, d), ints(n, N, r), ints(T, N)
    rows = torch.randint(-1, n, (T,), generator=g, dtype=torch.int32)
    leaves = [t.cuda().requires_grad_() for t in (base, x.to(BF16), a.to(BF16), b.to(BF16))]
    y = _Adapt.apply(*leaves, torch.tensor([1.0, 2.0], device="cuda"), rows.cuda())
    (y * y).sum().backward()
    ref = [t.double().requires_grad_() for t in (base, x, a, b)]
    s = torch.tensor([1.0, 2.0], dtype=torch.float64)
    z = ref[0]
    for k in range(n):
        z = z + (rows == k).double()[:, None] * s[k] * (ref[1] @ ref[2][k].T @ ref[3][k].T)
    (z * z).sum().backward()
    for got, want in zip(leaves, ref):
        assert torch.equal(got.grad.cpu(), want.grad.to(got.dtype))


def test_embedding_many_distinct_and_sorted_inputs():
    """Every token once, in order and in reverse, over the single workgroup's limit and under it."""
    for V in (4096, 4097, 20000):
        g = torch.Generator().manual_seed(V)
        grad = torch.randn(V, 12, generator=g).cuda()
        for tok in (torch.arange(V), torch.arange(V).flip(0), torch.randperm(V, generator=g)):
            tok = tok.to(torch.int32).cuda()
            got = tim.embedding_backward(grad, tok, V)
            assert torch.equal(got[tok.long()], grad)


@pytest.mark.parametrize("T", [5, 90, 2000, 17000])
def test_whatever_the_workspace_holds(T):
    """A workspace of NaN bits and one of zeros give the same bits: everything read from it was written by the call."""
    m = _model(T=T, V=520, n=3, r=20)
    d, V, n, r = 256, 520, 3, 20
    x = tim.embedding(m["W"], m["inp"], 16.0)
    dy = torch.randn(T, V, device="cuda")
    sizes = (tim.adapters_add_workspace_size(T, d, V, n, r), tim.adapters_backward_workspace_size(T, d, V, n, r),
             tim.embedding_backward_workspace_size(T, V, d))
    results = []
    for byte in (0, 255):
        ws = [torch.full((s,), byte, dtype=torch.uint8, device="cuda") for s in sizes]
        out = [tim.adapters_add(dy, x, m["rows"], m["ad"], workspace=ws[0])]
        for g in (dy, dy.to(BF16)):
            out += tim.adapters_backward(g, x, m["rows"], m["ad"], dtype=F32, workspace=ws[1].fill_(byte))
        out += [tim.embedding_backward(out[1], m["inp"], V, workspace=ws[2]),
                tim.embedding_backward(out[1], m["inp"], V, grad_table=torch.ones(V, d, device="cuda"), accumulate=True,
                                       workspace=ws[2].fill_(byte))]
        results.append(out)
    for a, b in zip(*results):
        assert bits_equal(a, b)
