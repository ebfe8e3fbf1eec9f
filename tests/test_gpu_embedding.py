"""GPU parity of the token embedding and its gradient (tim_embedding*) against the fp64 oracle.

Lookup. An element is one fp32 product rounded once to the output type, so it is compared for equality with that.

Gradient. With whole numbers below 2^24 in all sums, fp32 addition is exact in any order and the gradient is compared for
equality: that pins the grouping, every index, the ends of odd sizes and the joining of runs. With other numbers an
element behind which n rows stand is a sum of at most n additions, then one multiplication and with accumulation one
addition more, each off by at most 2^-24 relative: |err| <= (n + 2) 2^-24 (sum |g| |scale| + |old|), to which (1 + 2^-10)
allows for the products of those factors."""

import numpy as np
import pytest
import torch

import oracle
import paper_2605_14220_amd as tim
from tim_testutil import require_gpu

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _np(t):
    return t.detach().double().cpu().numpy()


def _padded(t, pad):
    """The matrix with `pad` elements between its rows, one element off the allocation's start."""
    if not pad:
        return t
    rows, cols = t.shape
    big = torch.full((rows * (cols + pad) + 1,), 77.0, dtype=t.dtype, device=t.device)
    view = big[1:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


def _tokens(T, V, seed, kind):
    g = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        return torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    if kind == "few":     # long runs, some of them ending exactly at a run's length
        return torch.randint(0, min(3, V), (T,), generator=g, dtype=torch.int32)
    if kind == "one":
        return torch.full((T,), V - 1, dtype=torch.int32)
    t = (V ** torch.rand(T, generator=g, dtype=torch.float64)).long().clamp(1, V).sub(1).to(torch.int32)  # heavy head
    bad = torch.rand(T, generator=g) < 0.1
    odd = torch.tensor([-1, V, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64).to(torch.int32)
    return torch.where(bad, odd[torch.randint(0, 4, (T,), generator=g)], t)


@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V,d,pad", [(1, 1, 1, 0), (1, 50257, 4096, 0), (7, 100, 5, 0), (48, 1000, 5120, 0),
                                       (129, 333, 257, 3), (1000, 77, 96, 1), (3, 10, 20001, 0), (65, 64, 8, 5)])
def test_lookup(T, V, d, pad, dtype, out):
    g = torch.Generator().manual_seed(T + d)
    table = _padded(torch.randn(V, d, generator=g).to(dtype).cuda(), pad)
    tok = _tokens(T, V, T, "mixed")
    dst = _padded(torch.full((T, d), 5.0, dtype=out, device="cuda"), pad)
    for scale in (1.0, 64.0, -0.3, 0.0):
        got = tim.embedding(table, tok.cuda(), scale, out=dst)
        there = (tok >= 0) & (tok < V)
        want = (table.float().cpu()[torch.where(there, tok, 0).long()] * scale).to(out)
        want[~there] = 0
        assert torch.equal(got.cpu(), want)
        if out == torch.float32:
            exact = oracle.embedding(_np(table), tok.numpy(), float(np.float32(scale)))
            assert (np.abs(_np(got) - exact) <= 2.0 ** -24 * np.abs(exact)).all()
    if pad:  # what lies between the rows stays
        assert (dst._base[1:].view(T, d + pad)[:, d:] == 77).all()


def test_lookup_keeps_specials():
    table = torch.tensor([[float("nan"), float("inf"), -float("inf"), -0.0, 3.0e38]], device="cuda")
    got = tim.embedding(table, torch.zeros(2, dtype=torch.int32, device="cuda"), 1.0)
    assert torch.equal(got.view(torch.int32), table.expand(2, -1).contiguous().view(torch.int32))
    z = tim.embedding(table, torch.tensor([-1], dtype=torch.int32, device="cuda"), 2.0)
    assert (z == 0).all()  # padding is zeros whatever the table holds


SIZES = [(1, 1, 1, 0), (1, 50257, 4096, 0), (2, 3, 5, 0), (63, 7, 33, 0), (64, 7, 33, 2), (65, 7, 1030, 0),
         (129, 5000, 257, 3), (1000, 77, 96, 0), (1025, 300, 512, 0), (4095, 1023, 40, 0), (4096, 1024, 24, 1),
         (4097, 255, 17, 0), (4097, 151936, 8, 0), (5000, 1, 64, 0), (9000, 1500, 130, 0), (70000, 50257, 16, 0),
         (300001, 3001, 5, 0)]


@pytest.mark.parametrize("kind", ["uniform", "few", "one", "mixed"])
@pytest.mark.parametrize("T,V,d,pad", SIZES)
def test_gradient_of_whole_numbers(T, V, d, pad, kind):
    dtype = DTYPES[(T + d) % 3]
    g = torch.Generator().manual_seed(T + V + d)
    grad = torch.randint(-8, 9, (T, d), generator=g).float()  # 8 * 300001 * 4 < 2^24
    tok = _tokens(T, V, T + V, kind)
    old = torch.randint(-50, 51, (V, d), generator=g).float()
    want = torch.zeros(V, d, dtype=torch.float64)
    there = (tok >= 0) & (tok < V)
    want.index_add_(0, tok[there].long(), grad[there].double())
    if T * d < 50000:
        assert np.array_equal(want.numpy(), oracle.embedding_backward(_np(grad), tok.numpy(), V, 1.0)[0])
    dev = _padded(grad.to(dtype).cuda(), pad)
    dst = _padded(torch.full((V, d), float("nan"), device="cuda"), pad)
    print(T, V, d, kind, flush=True)
    tim.embedding_backward(dev, tok.cuda(), V, 4.0, grad_table=dst)
    assert torch.equal(dst.cpu().double(), 4.0 * want)
    dst.copy_(old)
    tim.embedding_backward(dev, tok.cuda(), V, -2.0, grad_table=dst, accumulate=True)
    assert torch.equal(dst.cpu().double(), old - 2.0 * want)
    if pad:
        assert (dst._base[1:].view(V, d + pad)[:, d:] == 77).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V,d,kind", [(301, 500, 1536, "mixed"), (4096, 9000, 100, "mixed"), (20000, 3000, 60, "mixed"),
                                        (2000, 4, 300, "few"), (513, 2, 7, "one")])
def test_gradient(T, V, d, kind, dtype):
    g = torch.Generator().manual_seed(T)
    grad = (torch.randn(T, d, generator=g) * torch.exp(2 * torch.randn(T, 1, generator=g))).to(dtype)
    old = torch.randn(V, d, generator=g)
    tok = _tokens(T, V, T, kind)
    scale = 0.37
    want, size, n = oracle.embedding_backward(_np(grad), tok.numpy(), V, float(np.float32(scale)))
    dst = old.cuda()
    for acc in (False, True):
        got = _np(tim.embedding_backward(grad.cuda(), tok.cuda(), V, scale, grad_table=dst, accumulate=acc))
        w = want + acc * prev if acc else want
        s = size + np.abs(prev) if acc else size
        bound = (n + 2)[:, None] * 2.0 ** -24 * s * (1 + 2.0 ** -10)
        err = np.abs(got - w)
        print(f"max err / bound {np.max(err / np.maximum(bound, 1e-300)):.3f}")
        assert (err <= bound).all()
        prev = got


def test_gradient_is_the_lookups_derivative():
    """Against central differences of sum(out * c) in fp64 arithmetic on the lookup's own fp32 output: the lookup is
    linear, so differences of steps that are powers of two are exact."""
    V, d, T = 9, 6, 40
    g = torch.Generator().manual_seed(3)
    table = torch.randint(-8, 9, (V, d), generator=g).float().cuda()
    c = torch.randint(-8, 9, (T, d), generator=g).float().cuda()
    tok = _tokens(T, V, 1, "mixed").cuda()
    grad = tim.embedding_backward(c, tok, V, 0.5)
    for v in range(V):
        for k in range(d):
            up, down = table.clone(), table.clone()
            up[v, k] += 0.5
            down[v, k] -= 0.5
            diff = (tim.embedding(up, tok, 0.5).double() * c).sum() - (tim.embedding(down, tok, 0.5).double() * c).sum()
            assert diff.item() == grad[v, k].item()


def test_a_tokens_gradient_depends_on_its_own_rows_only():
    """Bit for bit the same alone, among others, and further back in a longer batch: runs start at the token's first row."""
    d, V = 130, 4000
    g = torch.Generator().manual_seed(5)
    rows = (torch.randn(700, d, generator=g) * 0.1).cuda()
    alone = tim.embedding_backward(rows, torch.full((700,), 17, dtype=torch.int32, device="cuda"), V)[17]
    for T in (701, 1500, 4500, 9000):
        where = torch.sort(torch.randperm(T, generator=g)[:700])[0].cuda()
        tok = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda()
        tok[tok == 17] = 16
        tok[where] = 17
        grad = torch.randn(T, d, generator=g).cuda()
        grad[where] = rows
        got = tim.embedding_backward(grad, tok, V)[17]
        assert torch.equal(got.view(torch.int32), alone.view(torch.int32))


def test_gradient_nan_stays_in_its_token():
    grad = torch.ones(200, 33, device="cuda")
    grad[5, 7] = float("nan")
    grad[8, 1] = float("inf")
    tok = (torch.arange(200) % 50).to(torch.int32).cuda()
    got = tim.embedding_backward(grad, tok, 60)
    bad = ~torch.isfinite(got)
    assert bad.sum() == 2 and bool(bad[5, 7]) and bool(bad[8, 1])
    grad[5] = float("nan")
    tok[5] = -1  # padding rows may hold anything
    assert torch.isfinite(tim.embedding_backward(grad, tok, 60)).sum() == 60 * 33 - 1


def test_no_rows():
    empty = torch.empty(0, 8, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert (tim.embedding_backward(empty, none, 5, grad_table=torch.ones(5, 8, device="cuda")) == 0).all()
    assert (tim.embedding_backward(empty, none, 5, grad_table=torch.ones(5, 8, device="cuda"), accumulate=True) == 1).all()
    assert tim.embedding(torch.ones(3, 8, device="cuda"), none).shape == (0, 8)


def test_offsets_past_32_bits():
    """A table whose last rows lie beyond 2^32 bytes and 2^31 elements."""
    V, d = 300000, 8192
    table = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    table[V - 1] = torch.arange(d, device="cuda") % 128
    tok = torch.tensor([V - 1, 0, V - 1], dtype=torch.int32, device="cuda")
    got = tim.embedding(table, tok)
    assert torch.equal(got[0], table[V - 1]) and torch.equal(got[2], table[V - 1]) and (got[1] == 0).all()
    del table
    grad = tim.embedding_backward(got, tok, V, 1.0)
    assert torch.equal(grad[V - 1], 2.0 * got[0].float()) and grad[V - 2].abs().sum() == 0
    assert float(grad[V - 1].double().sum()) == float(grad.sum(dtype=torch.float64))
