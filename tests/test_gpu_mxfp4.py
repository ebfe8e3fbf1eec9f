"""GPU parity of the 4-bit microscaled formats and the quantised head (tim_mxfp4_*) against the fp64 oracle.

Codes, scales and values are exact, so they are compared for equality: on every bf16 value, on ties, on blocks of
zeros, of the smallest numbers, of NaN and infinities, for each input type, row stride and odd row count.

Logits. Where all scales are equal every partial sum is a multiple of one unit below 2^24 units, so fp32 accumulation
is exact in any order and the logits are compared for equality: that pins layout, indices and the ends of odd sizes.
With scales that differ, each logit is a sum of d products with at most one rounding of at most 2^-23 relative per
addition whatever the order: |err| <= d 2^-23 sum |h w| / tau, then eps / 2 of the output type."""

import numpy as np
import pytest
import torch

import oracle
import paper_2605_14220_amd as tim
from plan_shim import fp4_kernel
from tim_testutil import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _check_quant(x, q):
    codes, scales = oracle.mxfp4_quantize(x.double().cpu().numpy())
    assert (q.scales.cpu().numpy() == scales).all()
    got = oracle.mxfp4_unpack(q.codes.cpu().numpy())
    bad = np.argwhere(got != codes)
    assert not len(bad), (bad[:4], x.flatten()[:1])


def test_every_bf16_value_beside_every_scale():
    """Each of the 2^16 bit patterns, in blocks whose largest value is the pattern itself and in blocks led by values
    up to 2^8 larger."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(torch.bfloat16)
    for lead in (0.0, 1.0, 1.5, 3.0, 40.0, 256.0):
        x = torch.zeros(65536, 32, dtype=torch.bfloat16)
        x[:, 0] = bits
        x[:, 5] = (bits.float() * lead).to(torch.bfloat16)
        print(f"lead {lead}", flush=True)
        _check_quant(x, tim.mxfp4_quantize(x.cuda()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,d,pad", [(1, 32, 0), (3, 96, 0), (7, 160, 5), (65, 4096, 0), (33, 256, 8), (1, 64, 7),
                                        (1000, 128, 1)])
def test_quantise_rows(dtype, rows, d, pad):
    g = torch.Generator().manual_seed(rows + d)
    x = torch.randn(rows, d + pad, generator=g) * torch.exp(3 * torch.randn(rows, d + pad, generator=g))
    x = x.to(dtype).cuda()[:, :d]
    _check_quant(x, tim.mxfp4_quantize(x))


def test_quantise_ties_and_extremes():
    row = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -7.999, 0.0, -0.0,
           7.0, 6.9, 0.24999999, 0.25000003, 4.9999995, 5.0000005, 2.4999998, 2.5000002] + [0.0] * 6
    rows = [torch.tensor(row) * 2.0 ** k for k in (0, 1, -1, 20, -60, 100, -120, 125)]
    rows += [torch.full((32,), v) for v in (2.0 ** -149, 2.0 ** -127, 3.4028234663852886e38, -2.0 ** -126, 0.0, -0.0)]
    for bad in (float("nan"), float("inf"), -float("inf")):
        r = torch.ones(32)
        r[31] = bad
        rows.append(r)
    x = torch.stack(rows)
    _check_quant(x, tim.mxfp4_quantize(x.cuda()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_dequantise_every_code_and_scale(dtype):
    codes = np.tile(np.arange(16, dtype=np.uint8), 2)[None].repeat(256, 0)
    scales = np.arange(256, dtype=np.uint8)[:, None]
    q = tim.Mxfp4(torch.as_tensor(oracle.mxfp4_pack(codes)).cuda(), torch.as_tensor(scales).cuda())
    got = tim.mxfp4_dequantize(q, dtype).cpu()
    want = torch.as_tensor(oracle.mxfp4_values(codes, scales))
    assert torch.equal(got[:253].double(), want[:253])       # 6 * 2^125 is the largest that always fits
    assert torch.equal(got[253:255], want[253:255].to(dtype))  # values past the range are infinite
    assert torch.isnan(got[255]).all()
    assert torch.signbit(got[100, 8]) and not torch.signbit(got[100, 0])


def test_quantise_into_a_slice_leaves_the_rest():
    x = torch.randn(5, 64, device="cuda")
    codes = torch.full((9, 32), 77, dtype=torch.uint8, device="cuda")
    scales = torch.full((9, 2), 77, dtype=torch.uint8, device="cuda")
    tim.mxfp4_quantize(x, out=tim.Mxfp4(codes[2:7], scales[2:7]))
    assert (codes[:2] == 77).all() and (codes[7:] == 77).all()
    assert (scales[:2] == 77).all() and (scales[7:] == 77).all()
    _check_quant(x, tim.Mxfp4(codes[2:7], scales[2:7]))


def test_quantise_nothing():
    q = tim.mxfp4_quantize(torch.empty(0, 64, device="cuda"))
    assert q.codes.shape == (0, 32) and q.scales.shape == (0, 2)
    assert tim.mxfp4_dequantize(q).shape == (0, 64)


# ------------------------------------------------------------------ logits


def _random(rows, d, seed, spread):
    """Random codes; scales 127 everywhere (spread 0) or 127 +- spread."""
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 16, (rows, d)).astype(np.uint8)
    scales = (127 + rng.integers(-spread, spread + 1, (rows, d // 32))).astype(np.uint8)
    q = tim.Mxfp4(torch.as_tensor(oracle.mxfp4_pack(codes)).cuda(), torch.as_tensor(scales).cuda())
    return q, torch.as_tensor(oracle.mxfp4_values(codes, scales)).cuda()


SHAPES = [(1, 128, 1), (1, 256, 16), (2, 384, 100), (5, 512, 1000), (16, 640, 257), (17, 256, 4097), (31, 128, 333),
          (33, 896, 515), (64, 1024, 1111), (65, 1152, 640), (127, 256, 259), (129, 384, 2050), (200, 2048, 777),
          (256, 128, 256), (257, 640, 513), (300, 1536, 1025), (513, 256, 130), (1030, 384, 300)]


@pytest.mark.parametrize("T,d,V", SHAPES)
def test_logits_exact(T, d, V):
    print(f"case T={T} d={d} V={V}", flush=True)
    h, hv = _random(T, d, 1, 0)
    w, wv = _random(V, d, 2, 0)
    z = tim.mxfp4_logits(h, w)
    assert torch.equal(z.double(), hv @ wv.T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,d,V,tau,spread", [(3, 256, 500, 1.0, 3), (40, 1152, 777, 0.7, 4), (260, 640, 1031, 1.3, 6),
                                              (1, 4096, 300, 0.6, 20), (600, 256, 520, 1.0, 9)])
def test_logits_within_the_bound(T, d, V, tau, spread, dtype):
    print(f"case T={T} d={d} V={V} {dtype}", flush=True)
    h, hv = _random(T, d, 3, spread)
    w, wv = _random(V, d, 4, spread)
    scale = 2.0 ** -12 / d  # towards fp16's range: the rows' scales are moved by a power of two
    k = int(np.floor(np.log2(scale)))
    h = tim.Mxfp4(h.codes, (h.scales.int() + k).to(torch.uint8))
    hv = hv * 2.0 ** k
    z = tim.mxfp4_logits(h, w, tau, dtype=dtype).double()
    inv = float(np.float32(1.0 / np.float64(np.float32(tau))))
    ref = (hv @ wv.T) * inv
    bound = d * 2.0 ** -23 * (hv.abs() @ wv.abs().T) * inv + 2.0 ** -24 * ref.abs()
    tiny = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}[dtype]
    bound = bound + torch.finfo(dtype).eps / 2 * (ref.abs() + bound) + tiny
    # with scales 2^20 apart on both sides a logit reaches 36 * 2^40 * 2^-24 / 0.6 > 65504: past fp16 it is infinite
    top = torch.finfo(dtype).max
    past = ref.abs() - bound > top * (1 + torch.finfo(dtype).eps)
    assert torch.equal(z[past], torch.sign(ref[past]) * float("inf"))
    inside = ref.abs() + bound < top
    assert (inside | past).float().mean() > 0.9
    worst = ((z - ref).abs() / bound)[inside].max().item()
    print(f"worst error {worst:.3f} of the bound")
    assert worst <= 1


@pytest.mark.parametrize("T", [1, 16, 17, 64, 65, 128, 129, 300])
def test_rows_do_not_depend_on_the_batch(T):
    """A row's logits have the same bits alone, in any batch, at any position, in a padded output."""
    V, d = 1000, 1152
    h, _ = _random(300, d, 5, 5)
    w, _ = _random(V, d, 6, 5)
    whole = tim.mxfp4_logits(h, w, 0.7)
    out = torch.full((T + 1, V + 13), 5.0, device="cuda")
    part = tim.Mxfp4(h.codes[300 - T:], h.scales[300 - T:])
    tim.mxfp4_logits(part, w, 0.7, out=out[:T, :V])
    assert torch.equal(out[:T, :V], whole[300 - T:])
    assert (out[T] == 5.0).all() and (out[:, V:] == 5.0).all()


def test_columns_do_not_depend_on_the_vocabulary():
    h, _ = _random(40, 640, 7, 5)
    w, _ = _random(900, 640, 8, 5)
    whole = tim.mxfp4_logits(h, w)
    for a, b in ((0, 1), (5, 300), (899, 900), (131, 900)):
        part = tim.Mxfp4(w.codes[a:b].contiguous(), w.scales[a:b].contiguous())
        assert torch.equal(tim.mxfp4_logits(h, part), whole[:, a:b])


@pytest.mark.parametrize("T", [2, 40, 300])
def test_nan_blocks_reach_their_logits_only(T):
    h, _ = _random(T, 384, 9, 2)
    w, _ = _random(300, 384, 10, 2)
    clean = tim.mxfp4_logits(h, w)
    h.scales[1, 3] = 255
    w.scales[77, 11] = 255
    w.codes[77] = 0
    z = tim.mxfp4_logits(h, w)
    bad = torch.zeros_like(z, dtype=torch.bool)
    bad[1] = True
    bad[:, 77] = True
    assert torch.equal(torch.isnan(z), bad)
    assert torch.equal(z[~bad], clean[~bad])


@pytest.mark.parametrize("T,V", [(3, 200), (200, 300)])
def test_extreme_scales(T, V):
    """Scales at both ends: products of values near 2^60 and 2^-60 on both sides stay exact powers of two."""
    codes = np.zeros((T, 256), np.uint8)
    codes[:, 7], codes[:, 200] = 2, 5
    hs = np.full((T, 8), 187, np.uint8)
    wc = np.zeros((V, 256), np.uint8)
    wc[:, 7], wc[:, 200] = 4, 10
    ws = np.full((V, 8), 67, np.uint8)
    h = tim.Mxfp4(torch.as_tensor(oracle.mxfp4_pack(codes)).cuda(), torch.as_tensor(hs).cuda())
    w = tim.Mxfp4(torch.as_tensor(oracle.mxfp4_pack(wc)).cuda(), torch.as_tensor(ws).cuda())
    assert (tim.mxfp4_logits(h, w) == -1.0).all()  # 1 * 2 + 3 * -1


def test_logits_of_quantised_rows_against_the_bf16_head():
    """The values a 4-bit head stands for, scored by the bf16 path, differ only by the order of the sums."""
    g = torch.Generator(device="cuda").manual_seed(1)
    h = tim.mxfp4_quantize(torch.randn(50, 512, device="cuda", generator=g))
    w = tim.mxfp4_quantize(0.02 * torch.randn(600, 512, device="cuda", generator=g))
    z = tim.mxfp4_logits(h, w, 0.7)
    hv, wv = tim.mxfp4_dequantize(h), tim.mxfp4_dequantize(w)
    bound = 2 * 512 * 2.0 ** -23 / 0.7 * (hv.double().abs() @ wv.double().abs().T)
    assert ((z.double() - tim.logits(hv, wv, 0.7).double()).abs() <= bound).all()


def test_no_rows():
    h, _ = _random(1, 256, 1, 0)
    w, _ = _random(40, 256, 2, 0)
    assert tim.mxfp4_logits(tim.Mxfp4(h.codes[:0], h.scales[:0]), w).shape == (0, 40)


@pytest.mark.parametrize("dtype,T,V", [(torch.float32, 600, 131071), (torch.bfloat16, 1100, 131073), (torch.float16, 1030, 140002)])
def test_logits_larger_than_the_caches(dtype, T, V):
    """More than 256 MB of logits in rows of odd lengths: the same bits as the rows a few at a time."""
    h, _ = _random(T, 512, 11, 3)
    w, _ = _random(V, 512, 12, 3)
    z = tim.mxfp4_logits(h, w, 0.9, dtype=dtype)
    for a, b in ((0, 64), (T - 40, T), (T // 2, T // 2 + 3)):
        part = tim.mxfp4_logits(tim.Mxfp4(h.codes[a:b], h.scales[a:b]), w, 0.9, dtype=dtype)
        assert torch.equal(z[a:b], part)


@pytest.mark.parametrize("d", [512, 640, 768, 896, 1024, 1152, 1280, 1408, 1536, 1664, 2048 + 128])
@pytest.mark.parametrize("T", [9, 30, 50, 100, 300])
def test_every_end_of_a_row(T, d):
    """Rows that end after each k-step of a scale group, in every tile shape: exact."""
    print(f"case T={T} d={d}", flush=True)
    h, hv = _random(T, d, T, 0)
    w, wv = _random(331, d, d, 0)
    hs = torch.randint(126, 129, h.scales.shape, generator=torch.Generator().manual_seed(1)).to(torch.uint8).cuda()
    h = tim.Mxfp4(h.codes, hs)  # scales that differ from block to block show a misplaced one
    hv = hv * torch.exp2(hs.double() - 127).repeat_interleave(32, 1)
    # sums of multiples of 1/8 below 36 * 2 * d < 2^21 units: exact in fp32
    assert torch.equal(tim.mxfp4_logits(h, w).double(), hv @ wv.T)


@pytest.mark.parametrize("T,d", [(2, 640), (40, 1024), (100, 512), (300, 1152)])
def test_nan_blocks_in_every_tile(T, d):
    """As above with rows of a whole scale group and more, the NaN in the first, a middle and the last block."""
    h, _ = _random(T, d, 13, 2)
    w, _ = _random(300, d, 14, 2)
    clean = tim.mxfp4_logits(h, w)
    h.scales[1, 0] = 255
    w.scales[77, d // 64] = 255
    w.scales[299, d // 32 - 1] = 255
    z = tim.mxfp4_logits(h, w)
    bad = torch.zeros_like(z, dtype=torch.bool)
    bad[1] = True
    bad[:, [77, 299]] = True
    assert torch.equal(torch.isnan(z), bad)
    assert torch.equal(z[~bad], clean[~bad])


@pytest.mark.parametrize("T", [3, 50, 100, 300])
def test_scales_at_both_ends(T):
    """One block of 2^60, the others of the smallest scale, against 2^-60: the small ones vanish, the rest is exact."""
    d, V = 768, 200
    codes = np.full((T, d), 2, np.uint8)  # 1.0 everywhere
    hs = np.zeros((T, d // 32), np.uint8)
    hs[:, 13] = 187
    wc = np.full((V, d), 10, np.uint8)    # -1.0
    ws = np.full((V, d // 32), 67, np.uint8)
    h = tim.Mxfp4(torch.as_tensor(oracle.mxfp4_pack(codes)).cuda(), torch.as_tensor(hs).cuda())
    w = tim.Mxfp4(torch.as_tensor(oracle.mxfp4_pack(wc)).cuda(), torch.as_tensor(ws).cuda())
    assert (tim.mxfp4_logits(h, w) == -32.0).all()  # 32 products of 2^60 * -2^-60; the others sum to 736 * 2^-187


def test_one_wide_row():
    """A long d, one row: offsets along a row and the scale groups at their largest common size."""
    d = 65536 + 128
    h, hv = _random(1, d, 15, 0)
    w, wv = _random(5, d, 16, 0)
    # 36 * d * 4 units < 2^24: exact
    assert torch.equal(tim.mxfp4_logits(h, w).double(), hv @ wv.T)


@pytest.mark.parametrize("T,d,dtype", [(129, 640, torch.float32), (200, 512, torch.bfloat16), (256, 1152, torch.float32)])
def test_one_large_tile_of_rows(T, d, dtype):
    """All rows in one tile of 256 of them, W read once: the same bits as the rows a few at a time."""
    print(f"case T={T} d={d}", flush=True)
    h, _ = _random(T, d, 15, 3)
    w, _ = _random(150001, d, 16, 3)
    z = tim.mxfp4_logits(h, w, 0.9, dtype=dtype)
    for a, b in ((0, 64), (T - 40, T), (T // 2, T // 2 + 3)):
        part = tim.Mxfp4(h.codes[a:b].contiguous(), h.scales[a:b].contiguous())
        assert torch.equal(tim.mxfp4_logits(part, w, 0.9, dtype=dtype), z[a:b])


# ------------------------------------------------------------------ every kernel of the product, by the rule's own name

KERNELS = {  # (T, V, type): rows and vocabulary end inside a tile
    "rows16": [(9, 331, torch.float32)], "rows32": [(30, 331, torch.bfloat16)], "rows64": [(50, 331, torch.float32)],
    "rows128": [(100, 331, torch.float16)], "small": [(300, 331, torch.float32)],
    "large_once": [(200, 50257, torch.float32), (131, 50257, torch.bfloat16)],
    "large": [(500, 32001, torch.float32), (499, 32003, torch.bfloat16), (500, 32001, torch.float16)],
    "large_past": [(500, 140001, torch.float32), (999, 140003, torch.bfloat16), (1000, 140001, torch.float16)],
}


def _on_gpu(rows, d, seed):
    """Random codes, scales of 126 to 128, and the values they stand for."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (rows, d // 2), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.randint(126, 129, (rows, d // 32), dtype=torch.int32, device="cuda", generator=g).to(torch.uint8)
    table = torch.as_tensor(oracle.mxfp4_code_values()).cuda()
    v = table[torch.stack((codes & 15, codes >> 4), 2).view(rows, d).int()]
    return tim.Mxfp4(codes, scales), v * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)


@pytest.mark.parametrize("d", [512, 640, 768, 896, 1024, 1152, 1408, 2048])
@pytest.mark.parametrize("kernel,T,V,dtype", [(k, *c) for k, cases in KERNELS.items() for c in cases])
def test_every_kernel_at_every_end_of_a_row(kernel, T, V, dtype, d):
    """Exact logits where rows of one scale group and of several end after each of its k-steps, then the same bits
    around NaN blocks at the first, a middle and the last block of rows and entries in different tiles."""
    esize = torch.empty((), dtype=dtype).element_size()
    assert fp4_kernel(T, d, V, esize, torch.cuda.get_device_properties(0).multi_processor_count) == kernel
    print(f"case {kernel} T={T} d={d} V={V} {dtype}", flush=True)
    h, hv = _on_gpu(T, d, d)
    w, wv = _on_gpu(V, d, d + 1)
    # sums of multiples of 1/16 below 36 * 4 * d < 2^23 units: exact in fp32, rounded once on the way out
    z = tim.mxfp4_logits(h, w, dtype=dtype)
    assert torch.equal(z, (hv @ wv.T).to(dtype))
    rows, entries, blocks = (0, T // 2, T - 1), (1, V // 2, V - 1), (0, d // 64, d // 32 - 1)
    for r, v, b in zip(rows, entries, blocks):
        h.scales[r, b] = 255
        w.scales[v, d // 32 - 1 - b] = 255
    y = tim.mxfp4_logits(h, w, dtype=dtype)
    bad = torch.zeros_like(z, dtype=torch.bool)
    bad[list(rows)] = True
    bad[:, list(entries)] = True
    assert torch.equal(torch.isnan(y), bad)
    assert torch.equal(torch.where(bad, 0.0, y), torch.where(bad, 0.0, z))


def test_more_short_rows_than_a_launch():
    """More rows than one launch of the kernel for short rows takes (65535 blocks of 16): the rows about its end."""
    T, d, V = 65535 * 16 + 50, 384, 3
    h, _ = _on_gpu(T, d, 1)
    w, wv = _on_gpu(V, d, 2)
    z = tim.mxfp4_logits(h, w)
    for a, b in ((0, 40), (65535 * 16 - 20, 65535 * 16 + 20), (T - 33, T)):
        part = tim.Mxfp4(h.codes[a:b], h.scales[a:b])
        assert torch.equal(z[a:b].double(), tim.mxfp4_dequantize(part, torch.float32).double() @ wv.T)
