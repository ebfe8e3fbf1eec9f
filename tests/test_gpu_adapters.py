"""GPU parity of low-rank adapters and their gradients (tim_adapters_*) against the fp64 oracle.

Whole numbers. Small whole numbers keep every sum exact in fp32 in any order, so outputs are compared for equality with
the exact result rounded once: that pins the grouping, every index and the ends of odd sizes, in every rank's kernel.

Other numbers. Sums of k terms in fp32 are off by at most k 2^-23 of their terms' magnitudes (one rounding of at most 2^-23
a term, whatever the order, for the matrix instructions may truncate). With S the oracle's sum of magnitudes:
  out     d + r + 3 additions and multiplications behind an element: (d + r + 3) 2^-23 S, then eps / 2 of the output type
  grad_x  N + r + 3: the same with N
  grad_a  N + rows + 3,  grad_b  d + rows + 3, fp32 outputs
times (1 + 2^-8) for the products of those factors (the counts stay below 2^14)."""

import numpy as np
import pytest
import torch

import oracle
import paper_2605_14220_amd as tim
from tim_testutil import require_gpu

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _padded(t, pad):
    if not pad:
        return t
    rows, cols = t.shape
    big = torch.full((rows * (cols + pad) + 1,), 77.0, dtype=t.dtype, device=t.device)
    view = big[1:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


def _rows(T, n, kind, g):
    if kind == "one":
        return torch.full((T,), n - 1, dtype=torch.int32)
    if kind == "runs":
        return (torch.arange(T) * 3 // max(T, 1) % n).to(torch.int32)
    if kind == "none":
        return torch.full((T,), -1, dtype=torch.int32)
    r = torch.randint(-1, n, (T,), generator=g)
    odd = torch.tensor([n, 2 ** 31 - 1, -2 ** 31])
    return torch.where(r < 0, odd[torch.randint(0, 3, (T,), generator=g)], r).to(torch.int32)


# T, d, N, n, r, rows, padding of strides
SIZES = [(1, 1, 1, 1, 1, "one", 0), (1, 2048, 1000, 4, 16, "one", 0), (2, 33, 7, 3, 2, "mixed", 0),
         (16, 64, 64, 2, 16, "mixed", 0), (17, 100, 65, 2, 9, "mixed", 3), (48, 130, 300, 32, 16, "mixed", 0),
         (63, 40, 257, 1, 17, "one", 0), (64, 1024, 256, 1, 32, "one", 1), (65, 1025, 255, 1, 33, "one", 0),
         (130, 257, 1031, 2, 64, "runs", 0), (200, 96, 64, 5, 65, "mixed", 2), (37, 72, 130, 2, 100, "mixed", 0),
         (70, 40, 90, 2, 256, "mixed", 0), (333, 500, 130, 3, 8, "runs", 0), (700, 64, 70, 2, 5, "mixed", 0),
         (1500, 40, 66, 1, 12, "one", 0), (5000, 24, 33, 7, 3, "mixed", 0), (100, 48, 40, 3, 4, "none", 0),
         (4097, 20, 16, 1000, 2, "mixed", 0), (40, 3001, 20, 2, 1, "mixed", 0),
         (70, 24, 33001, 2, 16, "mixed", 1), (150, 24, 32768, 2, 20, "runs", 0),
         (17000, 12, 20, 3, 2, "mixed", 0), (1025, 520, 600, 3, 48, "runs", 1),
         (40, 24, 33001, 31, 16, "mixed", 1), (45, 24, 33001, 31, 27, "mixed", 0)]


def _whole(T, d, N, n, r, kind, dtype, seed):
    g = torch.Generator().manual_seed(seed)

    def ints(*shape, top=2, keep=1.0):
        z = torch.randint(-top, top + 1, shape, generator=g).float()
        return z * (torch.rand(shape, generator=g) < keep)

    # few nonzero elements, so that sums of products of three stay far below 2^24
    x = ints(T, d, keep=min(1.0, 40 / d))
    a, b = ints(n, r, d), ints(n, N, r, keep=min(1.0, 16 / r))
    grad = ints(T, N, keep=min(1.0, 40 / N))
    scales = 2.0 ** torch.randint(-1, 3, (n,), generator=g).float()
    rows = _rows(T, n, kind, g)
    return [t.to(dtype) for t in (x, a, b, grad)] + [scales, rows]


@pytest.mark.parametrize("case", range(len(SIZES)))
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F16), (F16, BF16)])
def test_whole_numbers(case, dtype, out):
    T, d, N, n, r, kind, pad = SIZES[case]
    x, a, b, grad, scales, rows = _whole(T, d, N, n, r, kind, dtype, 7 * case)
    g = torch.Generator().manual_seed(case)
    base = torch.randint(-100, 101, (T, N), generator=g).to(out)
    dev = [t.cuda() for t in (a, b, scales)]
    ad = tim.Adapters(*dev)
    xd, rd = _padded(x.cuda(), pad), rows.cuda()
    print(SIZES[case], dtype, out, flush=True)

    want, size = oracle.adapters_add(_np(base), _np(x), rows.numpy(), _np(a), _np(b), _np(scales))
    assert size.max() < 2 ** 24
    bd = _padded(base.cuda(), pad)
    got = tim.adapters_add(bd, xd, rd, ad)
    assert torch.equal(got.cpu(), torch.as_tensor(want).to(out))
    got = tim.adapters_add(bd, xd, rd, ad, out=bd)  # in place
    assert got is bd and torch.equal(bd.cpu(), torch.as_tensor(want).to(out))
    if pad:
        assert (bd._base[1:].view(T, N + pad)[:, N:] == 77).all()
    want, _ = oracle.adapters_add(None, _np(x), rows.numpy(), _np(a), _np(b), None)
    got = tim.adapters_add(None, xd, rd, tim.Adapters(dev[0], dev[1]), dtype=out)
    assert torch.equal(got.cpu(), torch.as_tensor(want).to(out))

    (wx, wa, wb), sizes = oracle.adapters_backward(_np(grad), _np(x), rows.numpy(), _np(a), _np(b), _np(scales))
    assert all(s.max() < 2 ** 24 for s in sizes)
    gd = _padded(grad.to(out).cuda(), pad)
    gx, ga, gb = tim.adapters_backward(gd, xd, rd, ad, dtype=out)
    assert torch.equal(gx.cpu(), torch.as_tensor(wx).to(out))
    assert torch.equal(ga.cpu().double(), torch.as_tensor(wa))
    assert torch.equal(gb.cpu().double(), torch.as_tensor(wb))
    # accumulated, into rows with gaps
    old = torch.randint(-9, 10, (T, d), generator=g).float()
    acc = _padded(old.to(out).cuda(), pad)
    pa, pb = torch.ones_like(ga), torch.ones_like(gb)
    tim.adapters_backward(gd, xd, rd, ad, grad_x=acc, accumulate_x=True, grad_a=pa, grad_b=pb, accumulate=True)
    assert torch.equal(acc.cpu(), (torch.as_tensor(wx) + old).to(out))
    assert torch.equal(pa.cpu().double(), torch.as_tensor(wa) + 1) and torch.equal(pb.cpu().double(), torch.as_tensor(wb) + 1)


NUMBERS = [(5, 4096, 700, 3, 16, "mixed"), (200, 300, 257, 4, 9, "mixed"), (90, 1500, 1100, 2, 64, "runs"),
           (600, 128, 80, 1, 40, "one"), (21, 60, 3000, 2, 130, "mixed")]


@pytest.mark.parametrize("case", range(len(NUMBERS)))
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F32), (BF16, BF16), (F16, F16)])
def test_numbers(case, dtype, out):
    T, d, N, n, r, kind = NUMBERS[case]
    g = torch.Generator().manual_seed(case)
    x = (torch.randn(T, d, generator=g) * torch.exp(torch.randn(T, 1, generator=g))).to(dtype)
    a = (torch.randn(n, r, d, generator=g) / d ** 0.5).to(dtype)
    b = (torch.randn(n, N, r, generator=g) * 0.02).to(dtype)
    scales = torch.rand(n, generator=g) + 0.5
    rows = _rows(T, n, kind, g)
    base = (2.5 * torch.randn(T, N, generator=g)).to(out)
    grad = (0.1 * torch.randn(T, N, generator=g)).to(out)
    ad = tim.Adapters(a.cuda(), b.cuda(), scales.cuda())
    eps = torch.finfo(out).eps / 2
    tiny = 2.0 ** -25 if out == F16 else 0.0  # half the step of fp16's subnormal numbers

    def check(name, got, want, size, terms, eps):
        err, bound = np.abs(_np(got) - want), terms * 2.0 ** -23 * size * (1 + 2.0 ** -8) + eps * np.abs(want) * (
            1 + 2.0 ** -8) + tiny * (eps > 2.0 ** -24)
        print(f"{name}: max err / bound {np.max(err / np.maximum(bound, 1e-300)):.3f}")
        assert (err <= bound).all()

    want, size = oracle.adapters_add(_np(base), _np(x), rows.numpy(), _np(a), _np(b), _np(scales))
    check("out", tim.adapters_add(base.cuda(), x.cuda(), rows.cuda(), ad), want, size, d + r + 3, eps)
    want, size = oracle.adapters_backward(_np(grad), _np(x), rows.numpy(), _np(a), _np(b), _np(scales))
    got = tim.adapters_backward(grad.cuda(), x.cuda(), rows.cuda(), ad, dtype=out)
    check("grad_x", got[0], want[0], size[0], N + r + 3, eps)
    check("grad_a", got[1], want[1], size[1], N + T + 3, 2.0 ** -24)
    check("grad_b", got[2], want[2], size[2], d + T + 3, 2.0 ** -24)


@pytest.mark.parametrize("r", [16, 24, 40])
def test_many_rows_of_a_projection(r):
    """Runs and columns enough for every kernel's widest shape, in whole numbers against float64 products on the GPU."""
    T, d, N, n = 8200, 4100, 2052, 2
    g = torch.Generator(device="cuda").manual_seed(r)
    ints = lambda *s: torch.randint(-1, 2, s, generator=g, device="cuda").to(BF16)
    x, a, b, grad = ints(T, d), ints(n, r, d), ints(n, N, r), ints(T, N)
    x *= torch.rand(T, d, generator=g, device="cuda") < 0.01
    grad *= torch.rand(T, N, generator=g, device="cuda") < 0.02
    rows = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    ad = tim.Adapters(a, b)
    y = tim.adapters_add(None, x, rows, ad, dtype=F32)
    gx, ga, gb = tim.adapters_backward(grad, x, rows, ad, dtype=F32)
    wy, wx = torch.zeros(T, N, dtype=torch.float64, device="cuda"), torch.zeros(T, d, dtype=torch.float64, device="cuda")
    X, G = x.double(), grad.double()
    for k in range(n):
        m = (rows == k).double()[:, None]
        A, B = a[k].double(), b[k].double()
        u, v = m * (X @ A.T), m * (G @ B)
        wy += u @ B.T
        wx += v @ A
        assert torch.equal(ga[k].double(), v.T.contiguous() @ X)
        assert torch.equal(gb[k].double(), G.T.contiguous() @ u)
    assert torch.equal(y.double(), wy) and torch.equal(gx.double(), wx)
    assert torch.equal(tim.adapters_backward(grad, x, rows, ad, want_a=False, want_b=False)[0], wx.to(BF16))


def test_more_elements_than_31_bits():
    """Outputs and gradients of 2.25e9 elements, past the caches and in whole numbers: every row against its own few
    values, the weights' gradients against exact sums."""
    T, N, d, r = 15000, 150001, 8, 1
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randint(-2, 3, (T, d), generator=g, device="cuda").to(BF16)
    a = torch.randint(-1, 2, (1, r, d), generator=g, device="cuda").to(BF16)
    b = torch.randint(-2, 3, (1, N, r), generator=g, device="cuda").to(BF16)
    rows = torch.zeros(T, dtype=torch.int32, device="cuda")
    rows[::7] = -1
    u = (x.double() @ a[0].double().T)[:, 0] * (rows == 0)
    y = tim.adapters_add(None, x, rows, tim.Adapters(a, b))  # at most 16 * 2 in magnitude: exact in bf16
    for t in range(0, T, 1000):
        want = u[t:t + 1000, None] * b[0, :, 0].double()
        assert torch.equal(y[t:t + 1000].double(), want)
    base = tim.adapters_add(y, x, rows, tim.Adapters(a, b), out=y)
    assert torch.equal(base[T - 1].double(), 2 * u[T - 1] * b[0, :, 0].double())
    # gradients: y itself, as whole numbers
    gx, ga, gb = tim.adapters_backward(y, x, rows, tim.Adapters(a, b), dtype=F32)
    bb = (b.double() ** 2).sum()
    v = 2 * u * bb  # exact in fp64; in fp32 below 2^24 times a power of two only if bb is small, so bounds instead
    assert ((gx.double() - v[:, None] * a[0, 0].double()).abs() <= 2.0 ** -23 * N * (v[:, None] * a[0, 0].double()).abs()).all()
    assert torch.equal(gb[0, :, 0].double(), 2 * (u * u).sum() * b[0, :, 0].double())
    want = v @ x.double()
    size = (v.abs()[:, None] * x.double().abs()).sum(0)
    assert ((ga[0, 0].double() - want).abs() <= (N + T + 3) * 2.0 ** -23 * size * (1 + 2.0 ** -5)).all()


def test_gradients_are_the_derivative():
    """Against central differences of sum(out * c) with whole numbers: out is linear in each of x, a and b, so the
    differences are exact."""
    T, d, N, n, r = 11, 5, 6, 2, 3
    x, a, b, c, scales, rows = [t.cuda() for t in _whole(T, d, N, n, r, "mixed", BF16, 1)]

    def loss(x, a, b):
        return (tim.adapters_add(None, x, rows, tim.Adapters(a, b, scales), dtype=F32).double() * c.double()).sum().item()

    grads = tim.adapters_backward(c.float(), x, rows, tim.Adapters(a, b, scales), dtype=F32)
    for i, t in enumerate((x, a, b)):
        flat = grads[i].flatten()
        for k in range(t.numel()):
            args = [[x, a, b][j].clone() for j in range(3)]
            args[i].view(-1)[k] += 1
            up = loss(*args)
            args[i].view(-1)[k] -= 2
            assert (up - loss(*args)) / 2 == flat[k].item()


def test_a_row_depends_on_itself_only():
    """out and grad_x bit for bit, in batches of other sizes, other neighbours and other places."""
    d, N, n, r = 2100, 1500, 5, 24
    g = torch.Generator().manual_seed(2)
    a = (torch.randn(n, r, d, generator=g) / d ** 0.5).to(BF16).cuda()
    b = (torch.randn(n, N, r, generator=g) * 0.1).to(BF16).cuda()
    ad = tim.Adapters(a, b, torch.rand(n, generator=g).cuda())
    x, base, grad = torch.randn(1, d, generator=g).to(BF16), torch.randn(1, N, generator=g), torch.randn(1, N, generator=g)
    one = torch.tensor([3], dtype=torch.int32).cuda()
    y0 = tim.adapters_add(base.cuda(), x.cuda(), one, ad)
    x0 = tim.adapters_backward(grad.cuda(), x.cuda(), one, ad, dtype=F32)[0]
    for T in (2, 17, 65, 500, 4100):
        at = T * 2 // 3
        X, Y, G = torch.randn(T, d, generator=g).to(BF16), torch.randn(T, N, generator=g), torch.randn(T, N, generator=g)
        X[at], Y[at], G[at] = x[0], base[0], grad[0]
        rows = torch.randint(-1, n, (T,), generator=g, dtype=torch.int32)
        rows[at] = 3
        X, Y, G, rows = X.cuda(), Y.cuda(), G.cuda(), rows.cuda()
        assert torch.equal(tim.adapters_add(Y, X, rows, ad)[at], y0[0])
        assert torch.equal(tim.adapters_backward(G, X, rows, ad, dtype=F32)[0][at], x0[0])


def test_nan_and_infinity_stay_in_their_rows():
    T, d, N, n, r = 40, 70, 90, 3, 5
    g = torch.Generator().manual_seed(4)
    x = torch.randn(T, d, generator=g).to(BF16).cuda()
    a, b = torch.randn(n, r, d, generator=g).to(BF16).cuda(), torch.randn(n, N, r, generator=g).to(BF16).cuda()
    rows = (torch.arange(T) % 4 - 1).to(torch.int32).cuda()  # -1 .. 2
    base = torch.randn(T, N, generator=g).cuda()
    grad = torch.randn(T, N, generator=g).cuda()
    ad = tim.Adapters(a, b)
    good = tim.adapters_add(base, x, rows, ad)
    gx = tim.adapters_backward(grad, x, rows, ad, dtype=F32)[0]
    x[6, 3] = float("nan")   # adapter 1
    x[10, 0] = float("inf")  # adapter 1
    grad[13, 2] = float("nan")  # adapter 0
    x[4], grad[4] = float("nan"), float("inf")  # no adapter
    got = tim.adapters_add(base, x, rows, ad)
    bad = torch.zeros(T, dtype=torch.bool)
    bad[6] = bad[10] = True
    assert torch.equal((~torch.isfinite(got)).any(1).cpu(), bad)
    assert torch.equal(got[~bad.cuda()], good[~bad.cuda()])
    hx, ha, hb = tim.adapters_backward(grad, x, rows, ad, dtype=F32)
    keep = torch.arange(T).cuda() != 13
    assert torch.isnan(hx[13]).all() and torch.equal(hx[keep], gx[keep])
    assert torch.isfinite(ha[2]).all() and torch.isfinite(hb[2]).all()  # other adapters
    # an adapter that holds NaN reaches its own rows only
    a[0] = float("nan")
    got = tim.adapters_add(base, x, rows, ad)
    assert torch.isnan(got[rows == 0]).all() and torch.equal(got[rows == 2], good[rows == 2])


def test_rows_without_adapter_keep_the_bits_of_base():
    base = torch.tensor([[-0.0, float("nan"), float("inf"), 1e-45, 3.0]], device="cuda")
    x = torch.full((1, 4), float("nan"), dtype=BF16, device="cuda")
    ad = tim.Adapters(torch.ones(2, 3, 4, dtype=BF16, device="cuda"), torch.ones(2, 5, 3, dtype=BF16, device="cuda"))
    for k in (-1, 2):
        got = tim.adapters_add(base, x, torch.tensor([k], dtype=torch.int32, device="cuda"), ad)
        assert torch.equal(got.view(torch.int32), base.view(torch.int32))


def test_parts_of_the_backward():
    x, a, b, grad, scales, rows = [t.cuda() for t in _whole(90, 50, 60, 2, 6, "mixed", BF16, 3)]
    ad = tim.Adapters(a, b, scales)
    full = tim.adapters_backward(grad, x, rows, ad)
    for want in range(8):
        flags = [bool(want >> i & 1) for i in range(3)]
        got = tim.adapters_backward(grad, x, rows, ad, want_x=flags[0], want_a=flags[1], want_b=flags[2])
        for f, t, u in zip(flags, got, full):
            assert torch.equal(t, u) if f else t is None


def test_no_rows():
    ad = tim.Adapters(torch.ones(2, 3, 4, dtype=BF16, device="cuda"), torch.ones(2, 5, 3, dtype=BF16, device="cuda"))
    x = torch.empty(0, 4, dtype=BF16, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert tim.adapters_add(torch.empty(0, 5, device="cuda"), x, none, ad).shape == (0, 5)
    old = torch.ones(2, 3, 4, device="cuda")
    gx, ga, gb = tim.adapters_backward(torch.empty(0, 5, device="cuda"), x, none, ad, grad_a=old)
    assert gx.shape == (0, 4) and (ga == 0).all() and (gb == 0).all()
    tim.adapters_backward(torch.empty(0, 5, device="cuda"), x, none, ad, grad_a=old.fill_(1), grad_b=gb, accumulate=True)
    assert (old == 1).all()


def _formula(base, x, rows, a, b, scales, grad):
    """(out, grad_x, grad_a, grad_b) in float64, every product taken: 0 times an infinity is NaN in it."""
    T, (n, r, d), N = x.shape[0], a.shape, b.shape[1]
    x, a, b, grad, s = x.double(), a.double(), b.double(), grad.double(), scales.double()
    out, gx = base.double().clone(), torch.zeros(T, d, dtype=torch.float64)
    ga, gb = torch.zeros(n, r, d, dtype=torch.float64), torch.zeros(n, N, r, dtype=torch.float64)
    for t in range(T):
        k = int(rows[t])
        if 0 <= k < n:
            u, v = s[k] * (a[k] * x[t]).sum(1), s[k] * (b[k] * grad[t][:, None]).sum(0)
            out[t] += (b[k] * u).sum(1)
            gx[t] = (a[k] * v[:, None]).sum(0)
            ga[k] += v[:, None] * x[t]
            gb[k] += grad[t][:, None] * u
    return out, gx, ga, gb


# every kernel of the products: ranks of 1, 2, 4 and more blocks of 16, several tiles a wave, several blocks of rows
INFINITE = [(40, 70, 90, 3, 5, "mixed"), (70, 40, 300, 1, 16, "one"), (33, 130, 600, 2, 25, "mixed"),
            (90, 64, 80, 2, 44, "runs"), (20, 50, 70, 2, 64, "mixed"), (18, 40, 66, 2, 100, "mixed"),
            (40, 24, 33001, 31, 16, "mixed"), (45, 24, 33001, 31, 27, "mixed")]


@pytest.mark.parametrize("case", range(len(INFINITE)))
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (BF16, BF16), (F16, F32)])
@pytest.mark.parametrize("where", ["a", "b", "x", "grad"])
def test_infinities_give_what_the_formula_gives(case, dtype, out, where):
    """An infinity times a number is an infinity, times 0 NaN, and nothing else changes: in whole numbers, which are exact."""
    T, d, N, n, r, kind = INFINITE[case]
    x, a, b, grad, scales, rows = _whole(T, d, N, n, r, kind, dtype, 31 * case)
    g = torch.Generator().manual_seed(case)
    base = torch.randint(-100, 101, (T, N), generator=g).to(out)
    t = {"a": a, "b": b, "x": x, "grad": grad}[where].view(-1)
    some = lambda t, n: torch.randint(0, t.numel(), (n,), generator=g)
    for value in (float("inf"), float("-inf")):
        t[some(t, 6)] = value
        base.view(-1)[some(base, 6)] = value
    base.view(-1)[some(base, 6)] = float("nan")
    print(INFINITE[case], dtype, out, where, flush=True)
    want = _formula(base, x, rows, a, b, scales, grad)
    ad = tim.Adapters(a.cuda(), b.cuda(), scales.cuda())
    xd, rd, gd = x.cuda(), rows.cuda(), grad.to(out).cuda()
    got = (tim.adapters_add(base.cuda(), xd, rd, ad), *tim.adapters_backward(gd, xd, rd, ad, dtype=out))
    place = base.cuda()
    tim.adapters_add(place, xd, rd, ad, out=place)
    old = [torch.ones_like(t) for t in got[1:]]
    for o in old:
        o.view(-1)[some(o, 4)] = float("inf")
        o.view(-1)[some(o, 4)] = float("nan")
    sums = [o.cpu().double() + w for o, w in zip(old, want[1:])]
    tim.adapters_backward(gd, xd, rd, ad, grad_x=old[0], accumulate_x=True, grad_a=old[1], grad_b=old[2], accumulate=True)
    names = ("out", "grad_x", "grad_a", "grad_b", "out in place", "grad_x added", "grad_a added", "grad_b added")
    for name, y, w in zip(names, (*got, place, *old), (*want, want[0], *sums)):
        y, w = y.cpu(), w.to(y.dtype)
        wrong = ~((y == w) | (torch.isnan(y) & torch.isnan(w)))
        assert not wrong.any(), (name, int(wrong.sum()), y[wrong][:4], w[wrong][:4])


def test_outputs_beside_and_over_inputs():
    """grad_x in the columns beside x and out beside base, in one buffer each: as apart. Over an input: refused, with nothing
    written."""
    T, d, N = 70, 24, 40
    x, a, b, grad, scales, rows = [t.cuda() for t in _whole(T, d, N, 3, 5, "mixed", BF16, 9)]
    ad = tim.Adapters(a, b, scales)
    base = torch.randn(T, N, device="cuda").to(BF16)
    want = tim.adapters_backward(grad, x, rows, ad)
    out = tim.adapters_add(base, x, rows, ad)
    both, two = torch.zeros(T, 2 * d, dtype=BF16, device="cuda"), torch.zeros(T, 2 * N, dtype=BF16, device="cuda")
    both[:, :d], two[:, N:] = x, base
    got = tim.adapters_backward(grad, both[:, :d], rows, ad, grad_x=both[:, d:])
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and torch.equal(both[:, :d], x)
    assert torch.equal(tim.adapters_add(two[:, N:], x, rows, ad, out=two[:, :N]), out) and torch.equal(two[:, N:], base)
    kept = x.clone(), grad.clone(), base.clone()
    with pytest.raises(RuntimeError):
        tim.adapters_backward(grad, x, rows, ad, grad_x=x)
    with pytest.raises(RuntimeError):
        tim.adapters_add(base[1:], x[1:], rows[1:], ad, out=base[:-1])
    assert torch.equal(x, kept[0]) and torch.equal(grad, kept[1]) and torch.equal(base, kept[2])


@pytest.mark.parametrize("T,d,r", [(70, 48, 5), (1500, 600, 24), (300, 260, 80)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_a_residual_in_place(T, d, r, dtype):
    """x + its adapter over x, and its gradient over grad: as out of place."""
    x, a, b, grad, scales, rows = [t.cuda() for t in _whole(T, d, d, 3, r, "mixed", dtype, T)]
    ad = tim.Adapters(a, b, scales)
    out = tim.adapters_add(x, x, rows, ad)
    gx = tim.adapters_backward(grad, x, rows, ad, grad_x=grad.clone(), accumulate_x=True)
    plain = tim.adapters_backward(grad, x, rows, ad)
    assert torch.equal(gx[0], (grad.float() + tim.adapters_backward(grad, x, rows, ad, dtype=F32)[0]).to(dtype))
    ga, gb = torch.empty_like(gx[1]), torch.empty_like(gx[2])
    place = grad.clone()
    tim.adapters_backward(place, x, rows, ad, grad_x=place, accumulate_x=True, grad_a=ga, grad_b=gb)
    assert torch.equal(place, gx[0]) and torch.equal(ga, gx[1]) and torch.equal(gb, gx[2])
    place = grad.clone()
    tim.adapters_backward(place, x, rows, ad, grad_x=place)
    assert torch.equal(place, plain[0])
    y = x.clone()
    tim.adapters_add(y, y, rows, ad, out=y)
    assert torch.equal(y, out)


def _few(rows, cols, top, keep, dtype, g):
    """Whole numbers up to top in magnitude, a share `keep` of them not 0, made on the GPU."""
    z = torch.randint(-top, top + 1, (rows, cols), generator=g, device="cuda", dtype=torch.int8)
    return z.to(dtype).mul_(torch.rand(rows, cols, generator=g, device="cuda") < keep)


def _check_exact(grad, x, rows, a, b, got, step):
    """Gradients of whole numbers against float64 products, `step` rows of grad at a time."""
    for k in range(a.shape[0]):
        mine = (rows == k).nonzero()[:, 0]
        A, B = a[k].double(), b[k].double()
        ga, gb = torch.zeros_like(A), torch.zeros_like(B)
        for t in range(0, len(mine), step):
            i = mine[t:t + step]
            X, G = x[i].double(), grad[i].double()
            u, v = X @ A.T.contiguous(), G @ B
            assert torch.equal(got[0][i].double(), v @ A)
            ga += v.T.contiguous() @ X
            gb += G.T.contiguous() @ u
        assert ga.abs().max() < 2 ** 24 and gb.abs().max() < 2 ** 24
        assert torch.equal(got[1][k].double(), ga) and torch.equal(got[2][k].double(), gb)


@pytest.mark.parametrize("T", [700, 1500])
@pytest.mark.parametrize("r", [9, 16])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (BF16, F16), (F16, F16), (F16, F32)])
def test_long_runs_on_a_wide_head(T, r, dtype, out):
    """Two tiles of columns a workgroup beside runs of several blocks of 64 rows (256 or 512 rows, as T is), with gradients
    that the caches hold and larger ones; to the last bit, for sums of few small whole numbers are exact in any order."""
    d, N, n = 72, 100003, 2
    g = torch.Generator(device="cuda").manual_seed(r)
    x, a = _few(T, d, 2, 0.3, dtype, g), _few(n * r, d, 2, 1.0, dtype, g).view(n, r, d)
    b, grad = _few(n * N, r, 2, 0.5, dtype, g).view(n, N, r), _few(T, N, 2, 40 / N, out, g)
    rows = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    grad[:, N - 1] = 1  # the last tile's end
    grad[rows < 0] = float("nan")
    print(T, r, dtype, out, flush=True)
    got = tim.adapters_backward(grad, x, rows, tim.Adapters(a, b), dtype=F32)
    assert (got[0][rows < 0] == 0).all()
    _check_exact(grad, x, rows, a, b, got, 400)


@pytest.mark.parametrize("out", [BF16, F32])
def test_gradients_of_more_than_31_bits_of_elements(out):
    T, d, N, n, r = 15000, 40, 150001, 2, 16
    g = torch.Generator(device="cuda").manual_seed(3)
    x, a = _few(T, d, 1, 0.2, BF16, g), _few(n * r, d, 1, 1.0, BF16, g).view(n, r, d)
    b = _few(n * N, r, 1, 0.02, BF16, g).view(n, N, r)
    grad = torch.empty(T, N, dtype=out, device="cuda")
    for t in range(0, T, 1000):
        grad[t:t + 1000] = _few(1000, N, 1, 0.01, out, g)
    rows = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    got = tim.adapters_backward(grad, x, rows, tim.Adapters(a, b), dtype=F32)
    _check_exact(grad, x, rows, a, b, got, 1000)


@pytest.mark.parametrize("r", [16, 27])
@pytest.mark.parametrize("out", [BF16, F32])
def test_a_row_depends_on_itself_only_whatever_kernels_are_chosen(r, out):
    """out and grad_x bit for bit for row counts on both sides of every choice: tiles of columns a workgroup (two from few
    rows of many adapters on), tiles a wave in the forward (several for runs of few rows) and in grad_x's product (two for
    many runs)."""
    d, N, n = 4100, 50257, 40
    g = torch.Generator(device="cuda").manual_seed(r)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    ad = tim.Adapters((normal(n, r, d) / d ** 0.5).to(BF16), (0.1 * normal(n, N, r)).to(BF16), torch.rand(n, generator=g, device="cuda"))
    x, base, grad = normal(1, d).to(BF16), normal(1, N).to(out), normal(1, N).to(out)
    one = torch.full((1,), 3, dtype=torch.int32, device="cuda")
    y0 = tim.adapters_add(base, x, one, ad)
    x0 = tim.adapters_backward(grad, x, one, ad, dtype=F32, want_a=False, want_b=False)[0]
    for T in (2, 5, 65, 700, 8200):
        at = T * 2 // 3
        X, Y, G = normal(T, d).to(BF16), normal(T, N).to(out), normal(T, N).to(out)
        X[at], Y[at], G[at] = x[0], base[0], grad[0]
        rows = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
        rows[at] = 3
        print(T, r, out, flush=True)
        assert torch.equal(tim.adapters_add(Y, X, rows, ad)[at], y0[0])
        for want in (False, True):
            got = tim.adapters_backward(G, X, rows, ad, dtype=F32, want_a=want, want_b=want)
            assert torch.equal(got[0][at], x0[0])


@pytest.mark.parametrize("r,N,dtype,out", [(16, 3000, BF16, BF16), (16, 33001, BF16, F32), (40, 3000, BF16, BF16),
                                           (9, 700, F16, F16)])
def test_an_adapters_gradients_depend_on_its_rows_only(r, N, dtype, out):
    """grad_a and grad_b bit for bit when the other adapters' rows hold other values, NaN, or change their adapter."""
    T, d, n = 1500, 600, 4
    g = torch.Generator(device="cuda").manual_seed(r)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    ad = tim.Adapters((normal(n, r, d) / d ** 0.5).to(dtype), (0.1 * normal(n, N, r)).to(dtype), torch.rand(n, generator=g, device="cuda"))
    x, grad = normal(T, d).to(dtype), normal(T, N).to(out)
    rows = torch.randint(-1, n, (T,), generator=g, device="cuda", dtype=torch.int32)
    rows[torch.rand(T, generator=g, device="cuda") < 0.5] = 2  # runs of more than a workgroup takes
    first = tim.adapters_backward(grad, x, rows, ad, want_x=False)
    mine = (rows == 2)[:, None]
    others = torch.randint(-1, 2, (T,), generator=g, device="cuda", dtype=torch.int32)  # none is left with adapter 3
    for fill in (normal(T, N), torch.full((T, N), float("nan"), device="cuda")):
        got = tim.adapters_backward(torch.where(mine, grad, fill.to(out)), torch.where(mine, x, normal(T, d).to(dtype)),
                                    torch.where(mine[:, 0], rows, others), ad, want_x=False)
        assert torch.equal(got[1][2], first[1][2]) and torch.equal(got[2][2], first[2][2])
        assert (got[1][3] == 0).all() and (got[2][3] == 0).all()


@pytest.mark.parametrize("out", [BF16, F32])
def test_adapters_without_rows_change_no_row(out):
    """out and grad_x bit for bit with a set of 2 adapters and the same two among 60, where the set's size chooses other
    kernels; the gradients of those without rows are zeros."""
    T, d, N, r = 150, 700, 33000, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    a, b = (normal(60, r, d) / d ** 0.5).to(BF16), (0.1 * normal(60, N, r)).to(BF16)
    x, base, grad = normal(T, d).to(BF16), normal(T, N).to(out), normal(T, N).to(out)
    rows = torch.randint(-1, 2, (T,), generator=g, device="cuda", dtype=torch.int32)
    few, many = tim.Adapters(a[:2].contiguous(), b[:2].contiguous()), tim.Adapters(a, b)
    assert torch.equal(tim.adapters_add(base, x, rows, few), tim.adapters_add(base, x, rows, many))
    one, all_ = (tim.adapters_backward(grad, x, rows, ad, dtype=F32) for ad in (few, many))
    assert torch.equal(one[0], all_[0])
    assert (all_[1][2:] == 0).all() and (all_[2][2:] == 0).all()
