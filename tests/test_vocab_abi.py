"""The entry points of include/tim_vocab.h on the host: exported, sized, and refusing every bad argument with the
documented status before anything is enqueued. No call here reaches a launch."""

import copy
import ctypes
import os
import pickle
import re
import subprocess

import pytest
import torch

import paper_2605_14220_amd as tim
from paper_2605_14220_amd import Status

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_14220_amd", "csrc")
FAKE, MIS8, MIS2, MIS1 = 0x10000, 0x10008, 0x10002, 0x10001  # never dereferenced
F32, BF16, F16 = 0, 1, 2
SHAPE, VALUE, NULL, WORKSPACE = Status.ERR_SHAPE, Status.ERR_VALUE, Status.ERR_NULL, Status.ERR_WORKSPACE
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return tim.load_library()


def test_every_declared_function_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "tim_vocab.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"^\s*\w+\s+(tim_\w+)\s*\(", text, flags=re.M)))
    assert names == ["tim_adapters_add", "tim_adapters_add_workspace_size", "tim_adapters_backward",
                     "tim_adapters_backward_workspace_size", "tim_embedding", "tim_embedding_backward",
                     "tim_embedding_backward_workspace_size"]
    out = subprocess.run(["nm", "-D", "--defined-only", tim.LIB_PATH], capture_output=True, text=True, check=True).stdout
    assert set(names) <= set(re.findall(r"\bT\s+(\w+)$", out, flags=re.M))


def test_header_is_c_and_the_struct_matches(tmp_path):
    fields = [f for f, _ in tim._Adapters._fields_]
    src = tmp_path / "use.c"
    src.write_text('#define __HIP_PLATFORM_AMD__ 1\n#include <stdio.h>\n#include "tim_vocab.h"\nint main(void) {\n'
                   + "".join(f'printf("%zu ", offsetof(tim_adapters, {f}));\n' for f in fields)
                   + 'printf("%zu", sizeof(tim_adapters)); return 0; }\n')
    exe = str(tmp_path / "use")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-I",
                    "/opt/rocm/include", str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(tim._Adapters, f).offset for f in fields] + [ctypes.sizeof(tim._Adapters)]


def test_workspace_sizes(lib):
    """Nothing for nothing or for bad sizes; otherwise at least the lists, the order and the partial sums, and no less
    for more rows."""
    for T, V, d in ((0, 10, 8), (-1, 10, 8), (4, 0, 8), (4, tim.MAX_VOCAB + 1, 8), (4, 10, 0), (4, 10, 2 ** 20 + 1),
                    (2 ** 23 + 1, 10, 8)):
        assert tim.embedding_backward_workspace_size(T, V, d) == 0
    last = 0
    for T in (1, 64, 65, 4096, 4097, 16384, 16385, 300000, 2 ** 23):
        n = tim.embedding_backward_workspace_size(T, 50257, 64)
        assert n >= last and n >= T * 4 + 50257 + (T // 64) * 2 * 64 * 4 * (T > 64)
        last = n
    for size in (tim.adapters_add_workspace_size, tim.adapters_backward_workspace_size):
        for T, d, N, n, r in ((0, 8, 8, 1, 1), (-1, 8, 8, 1, 1), (2 ** 23 + 1, 8, 8, 1, 1), (4, 0, 8, 1, 1),
                              (4, 8, 0, 1, 1), (4, 8, 8, 0, 1), (4, 8, 8, 1, 0), (4, 8, 8, 1, 257),
                              (4, 2 ** 20 + 1, 8, 1, 1), (4, 8, 2 ** 20 + 1, 1, 1), (4, 8, 8, tim.MAX_VOCAB + 1, 1)):
            assert size(T, d, N, n, r) == 0
        assert size(5, 1000, 100, 3, 9) >= 5 * 4 + 2 * 5 * 16 * 4
    assert tim.adapters_backward_workspace_size(5, 8, 8, 1, 1) > tim.adapters_add_workspace_size(5, 8, 8, 1, 1)


def test_runs_fit_their_lists_and_slots(tmp_path):
    """The sizes a grouping is planned with, against runs made by hand: their number, the joins' number, and that no two
    partial results share a slot or lie past the slots."""
    src = tmp_path / "shim.cpp"
    src.write_text("""
#include "grouping.h"
extern "C" int64_t plan(int64_t T, int32_t n, int log_C, int what) {
  const int l[1] = {log_C};
  const tim::Grouping g = tim::plan_grouping(T, n, 1, l);
  return what == 0 ? g.max_runs[0] : what == 1 ? g.max_joins[0] : what == 2 ? tim::run_slots(T, log_C)
       : what == 3 ? (int64_t)1 << (g.passes * g.digit) : what == 4 ? (int64_t)g.blocks * g.per_block : what == 5 ? g.blocks : what == 6 ? g.small : g.digit;
}
extern "C" int32_t slot(int32_t first, int log_C, int last) { return tim::run_slot(first, log_C, last); }
""")
    so = str(tmp_path / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__=1", "-shared", "-fPIC", "-I", CSRC, "-I",
                    os.path.join(ROOT, "include"), "-isystem", "/opt/rocm/include", "-o", so, str(src)], check=True)
    shim = ctypes.CDLL(so)
    shim.plan.restype = ctypes.c_int64
    shim.plan.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int, ctypes.c_int]
    import random
    rng = random.Random(0)
    for _ in range(400):
        log_C = rng.choice([6, 7, 8, 9])
        C = 1 << log_C
        lengths = [rng.choice([1, 2, C - 1, C, C + 1, 2 * C, 2 * C + 1, rng.randint(1, 4 * C)])
                   for _ in range(rng.randint(1, 12))]
        n, T = rng.choice([len(lengths), len(lengths) - 1 or 1]), sum(lengths)
        if n + 1 < len(lengths):
            continue
        runs = joins = first = 0
        slots = set()
        for L in lengths:
            k = -(-L // C)
            runs += k
            joins += k > 1
            for q in range(k):
                if k > 1:
                    s = shim.slot(first + q * C, log_C, int(q == k - 1))
                    assert s == shim.slot(first, log_C, 0) + 2 * q + (q == k - 1)  # as the joins read them
                    assert s not in slots and 0 <= s < shim.plan(T, n, log_C, 2)
                    slots.add(s)
            first += L
        assert runs <= shim.plan(T, n, log_C, 0) and joins <= shim.plan(T, n, log_C, 1)
    for T in (1, 4096, 4097, 16384, 16385, 100000, 2 ** 23):
        for n in (1, 255, 256, 1023, 1024, 65535, 524288):
            assert shim.plan(T, n, 6, 3) > n                      # the digits hold every key, n included
            assert shim.plan(T, n, 6, 4) >= T                     # the blocks hold every row
            assert 1 <= shim.plan(T, n, 6, 5) <= 256
            if shim.plan(T, n, 6, 6):  # one workgroup: its LDS holds 256 digits, and key and index fit 32 bits
                assert shim.plan(T, n, 6, 7) <= 8 and T <= 16384 and n < 1 << (20 if T <= 4096 else 18)
            else:
                assert shim.plan(T, n, 6, 7) <= 10 and T > 4096


def test_shapes_of_the_pass_over_grad(tmp_path):
    """The workgroups' tiles and rows: of tiles and rows that the kernels have, two tiles only where one tile a workgroup
    would be more than 768 workgroups and for ranks up to 16, rows that leave 512 workgroups where 128 would; partial sums
    of grad b for every pair of tiles; a workspace that holds the plans of both kinds of instructions."""
    src = tmp_path / "shim.cpp"
    src.write_text("""
#include "adapters_plan.h"
extern "C" int shape(int64_t T, int64_t N, int n, int cols, int rp, int contract, int what) {
  const tim::PassShape s = tim::pass_shape(T, N, n, cols, rp, contract);
  return what ? s.log_rows : s.tiles;
}
extern "C" int64_t plan(int64_t T, int d, int N, int n, int r, int cols, int what) {
  const tim::AdapterPlan p = tim::plan_adapters(T, d, N, n, r, cols);
  return what == 0 ? (int64_t)p.bytes : what == 1 ? p.g_chunks : p.of_grad.tiles;
}
""")
    so = str(tmp_path / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__=1", "-shared", "-fPIC", "-I", CSRC, "-I",
                    os.path.join(ROOT, "include"), "-isystem", "/opt/rocm/include", "-o", so, str(src)], check=True)
    shim = ctypes.CDLL(so)
    i64, i32 = ctypes.c_int64, ctypes.c_int
    shim.shape.argtypes, shim.plan.restype, shim.plan.argtypes = [i64, i64, i32, i32, i32, i32, i32], i64, [i64] + [i32] * 6
    import random
    rng = random.Random(2)
    two = 0
    for _ in range(4000):
        T, N = int(2 ** rng.uniform(0, 23)), int(2 ** rng.uniform(0, 20))
        n, r, cols = int(2 ** rng.uniform(0, 12)), rng.randint(1, 256), rng.choice([128, 256])
        rp = (r + 15) // 16 * 16
        tiles, log_rows = (shim.shape(T, N, n, cols, rp, 1, w) for w in (0, 1))
        one_each = ((T >> 9) + min(n, T)) * -(-N // cols)
        assert tiles == (2 if rp == 16 and one_each > 768 else 1) and 7 <= log_rows <= 9
        count = lambda log: ((T >> log) + 1) * -(-N // (tiles * cols))
        assert log_rows == 7 or count(log_rows) >= 512
        assert log_rows == 9 or count(log_rows + 1) < 512
        assert shim.shape(T, N, n, cols, rp, 0, 0) == 1
        two += tiles == 2
        d = int(2 ** rng.uniform(0, 14))
        assert shim.plan(T, d, N, n, r, cols, 2) == tiles and shim.plan(T, d, N, n, r, cols, 1) == -(-N // (tiles * cols))
        assert tim.adapters_backward_workspace_size(T, d, N, n, r) == max(shim.plan(T, d, N, n, r, c, 0) for c in (128, 256))
        assert tim.adapters_add_workspace_size(T, d, N, n, r) == shim.plan(T, d, N, n, r, 0, 0)
    assert two > 50
    # both sides of the limit, each with an adapter more in the set
    for cols in (128, 256):
        assert [shim.shape(150, 384 * cols + k, 2, cols, 16, 1, 0) for k in (0, 1)] == [1, 2]
        assert [shim.shape(150, 256 * cols, n, cols, 16, 1, 0) for n in (3, 4)] == [1, 2]


def _embed(lib, table=FAKE, dtype=BF16, V=10, d=8, ld=8, tokens=FAKE, T=4, scale=1.0, out=FAKE, out_dtype=F32, out_ld=8):
    return lib.tim_embedding(table, dtype, V, d, ld, tokens, T, scale, out, out_dtype, out_ld, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(T=-1), SHAPE), (dict(V=0), SHAPE), (dict(V=tim.MAX_VOCAB + 1), SHAPE), (dict(d=0), SHAPE),
    (dict(d=2 ** 20 + 1, ld=BIG, out_ld=BIG), SHAPE), (dict(ld=7), SHAPE), (dict(out_ld=7), SHAPE),
    (dict(dtype=3), VALUE), (dict(out_dtype=-1), VALUE), (dict(scale=float("nan")), VALUE),
    (dict(scale=float("inf")), VALUE), (dict(table=None), NULL), (dict(tokens=None), NULL), (dict(out=None), NULL),
    (dict(table=MIS1), VALUE), (dict(tokens=MIS2), VALUE), (dict(out=MIS2), VALUE),
    (dict(T=0, table=None, tokens=None, out=None), Status.OK), (dict(T=0, d=0), SHAPE)])
def test_embedding_refusals(lib, kw, expect):
    assert _embed(lib, **kw) == expect


def _embed_back(lib, grad=FAKE, dtype=BF16, T=4, d=8, ld=8, tokens=FAKE, V=10, scale=1.0, table=FAKE, table_ld=8, acc=0,
                ws=FAKE, size=1 << 30):
    return lib.tim_embedding_backward(grad, dtype, T, d, ld, tokens, V, scale, table, table_ld, acc, ws, size, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(T=-1), SHAPE), (dict(T=2 ** 23 + 1), SHAPE), (dict(V=0), SHAPE), (dict(V=tim.MAX_VOCAB + 1), SHAPE),
    (dict(d=0), SHAPE), (dict(ld=7), SHAPE), (dict(table_ld=7), SHAPE), (dict(dtype=3), VALUE),
    (dict(scale=float("nan")), VALUE), (dict(acc=2), VALUE), (dict(acc=-1), VALUE), (dict(grad=None), NULL),
    (dict(tokens=None), NULL), (dict(table=None), NULL), (dict(grad=MIS1), VALUE), (dict(grad=MIS2, dtype=F32), VALUE),
    (dict(tokens=MIS2), VALUE), (dict(table=MIS2), VALUE), (dict(ws=None), WORKSPACE), (dict(ws=MIS8), WORKSPACE),
    (dict(size=100), WORKSPACE), (dict(T=0, acc=1, grad=None, tokens=None, ws=None), Status.OK)])
def test_embedding_backward_refusals(lib, kw, expect):
    assert _embed_back(lib, **kw) == expect


def _ad(a=FAKE, b=FAKE, scales=FAKE, dtype=BF16, n=3, r=4, d=8, N=16):
    return tim._Adapters(a, b, scales, dtype, n, r, d, N)


AD = [(dict(a=None), NULL), (dict(b=None), NULL), (dict(dtype=F32), VALUE), (dict(dtype=3), VALUE), (dict(n=0), SHAPE),
      (dict(n=tim.MAX_VOCAB + 1), SHAPE), (dict(r=0), SHAPE), (dict(r=257), SHAPE), (dict(d=0), SHAPE),
      (dict(N=0), SHAPE), (dict(d=2 ** 20 + 1), SHAPE), (dict(N=2 ** 20 + 1), SHAPE), (dict(a=MIS1), VALUE),
      (dict(b=MIS1), VALUE), (dict(scales=MIS2), VALUE)]


def _add(lib, ad=None, x=FAKE, x_ld=8, rows=FAKE, T=5, base=FAKE, base_ld=16, out=FAKE, out_dtype=F32, out_ld=16, ws=FAKE,
         size=1 << 30, null=False):
    ad = None if null else ctypes.byref(_ad(**(ad or {})))
    return lib.tim_adapters_add(ad, x, x_ld, rows, T, base, base_ld, out, out_dtype, out_ld, ws, size, None)


@pytest.mark.parametrize("kw,expect", [(dict(ad=a, x_ld=BIG, base_ld=BIG, out_ld=BIG), e) for a, e in AD] + [
    (dict(null=True), NULL), (dict(T=-1), SHAPE), (dict(T=2 ** 23 + 1), SHAPE), (dict(x_ld=7), SHAPE),
    (dict(base_ld=15), SHAPE), (dict(out_ld=15), SHAPE), (dict(out_ld=17), SHAPE),  # in place with another stride
    (dict(x=None), NULL), (dict(rows=None), NULL), (dict(out=None), NULL), (dict(out_dtype=3), VALUE),
    (dict(x=MIS1), VALUE), (dict(rows=MIS2), VALUE), (dict(base=MIS2, out=FAKE), VALUE), (dict(out=MIS2), VALUE),
    (dict(ws=None), WORKSPACE), (dict(ws=MIS8), WORKSPACE), (dict(size=10), WORKSPACE),
    (dict(T=0, x=None, rows=None, out=None, ws=None), Status.OK)])
def test_add_refusals(lib, kw, expect):
    assert _add(lib, **kw) == expect


def _back(lib, ad=None, x=FAKE, x_ld=8, rows=FAKE, T=5, grad=FAKE, grad_dtype=F32, grad_ld=16, gx=FAKE, gx_dtype=F32,
          gx_ld=8, acc_x=0, ga=FAKE, gb=FAKE, acc=0, ws=FAKE, size=1 << 30, null=False):
    ad = None if null else ctypes.byref(_ad(**(ad or {})))
    return lib.tim_adapters_backward(ad, x, x_ld, rows, T, grad, grad_dtype, grad_ld, gx, gx_dtype, gx_ld, acc_x, ga, gb,
                                     acc, ws, size, None)


@pytest.mark.parametrize("kw,expect", [(dict(ad=a, x_ld=BIG, grad_ld=BIG, gx_ld=BIG), e) for a, e in AD] + [
    (dict(null=True), NULL), (dict(T=-1), SHAPE), (dict(T=2 ** 23 + 1), SHAPE), (dict(x_ld=7), SHAPE),
    (dict(grad_ld=15), SHAPE), (dict(gx_ld=7), SHAPE), (dict(x=None), NULL), (dict(rows=None), NULL),
    (dict(grad=None), NULL), (dict(grad_dtype=3), VALUE), (dict(gx_dtype=3), VALUE), (dict(acc_x=2), VALUE),
    (dict(acc=2), VALUE), (dict(grad=MIS2), VALUE), (dict(gx=MIS2), VALUE), (dict(ga=MIS2), VALUE),
    (dict(gb=MIS2), VALUE), (dict(ws=None), WORKSPACE), (dict(ws=MIS8), WORKSPACE), (dict(size=10), WORKSPACE),
    (dict(gx=None, ga=None, gb=None), Status.OK), (dict(T=0, acc=1, x=None, rows=None, grad=None, ws=None), Status.OK)])
def test_backward_refusals(lib, kw, expect):
    assert _back(lib, **kw) == expect


# ------------------------------------------------------------------ the binding


def _refused(error, f, *a, **kw):
    with pytest.raises(error) as e:
        f(*a, **kw)
    assert "tim" in str(e.value)


def _cuda_like(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_refuses(lib):
    z, tok = _cuda_like, torch.zeros(4, dtype=torch.int32)
    _refused(ValueError, tim.embedding, z(10, 8), tok)  # on the CPU
    _refused(TypeError, tim.embedding, z(10, 8, dtype=torch.int32), tok)
    _refused(TypeError, tim.embedding, z(10, 8), tok.long())
    _refused(ValueError, tim.embedding, z(10, 8), tok[None])
    _refused(ValueError, tim.embedding, z(8, 10).T, tok)
    _refused(ValueError, tim.embedding, z(10, 8, 1), tok)
    back = tim.embedding_backward
    _refused(TypeError, back, z(4, 8, dtype=torch.float64), tok, 10)
    _refused(ValueError, back, z(5, 8), tok, 10)
    _refused(ValueError, back, z(4, 8), tok, 1 << 32)  # not the 32 bits that are left of it
    ad = tim.Adapters(z(3, 4, 8), z(3, 16, 4))
    rows = torch.zeros(5, dtype=torch.int32)
    for bad in (tim.Adapters(z(3, 4, 8, dtype=torch.float32), z(3, 16, 4)), tim.Adapters(z(3, 4, 8), z(3, 16, 4).half()),
                tim.Adapters(z(3, 4, 8), z(3, 16, 4), z(3))):
        _refused(TypeError, tim.adapters_add, None, z(5, 8), rows, bad)
    for bad in (tim.Adapters(z(3, 4, 8), z(2, 16, 4)), tim.Adapters(z(3, 4, 8), z(3, 16, 5)),
                tim.Adapters(z(4, 8), z(16, 4)), tim.Adapters(z(3, 4, 8), z(3, 16, 4), torch.zeros(2)), ad):
        _refused(ValueError, tim.adapters_add, None, z(5, 8), rows, bad)
    _refused(ValueError, tim.adapters_backward, z(5, 16), z(5, 8), rows, ad)


def test_adapters_can_be_copied_and_pickled():
    ad = tim.Adapters(torch.ones(3, 4, 8), torch.ones(3, 16, 4), torch.ones(3))
    object.__setattr__(ad, "_built", (tim._Adapters(), None))  # as after a call
    for c in (copy.deepcopy(ad), copy.copy(ad), pickle.loads(pickle.dumps(ad))):
        assert torch.equal(c.a, ad.a) and torch.equal(c.b, ad.b) and torch.equal(c.scales, ad.scales)
        assert c._built is None


# ------------------------------------------------------------------ outputs over inputs


def test_rows_that_share_bytes(tmp_path):
    """Against the bytes themselves, written out."""
    src = tmp_path / "shim.cpp"
    src.write_text("""
#include "overlap.h"
extern "C" int share(int64_t a, int64_t rows_a, int64_t width_a, int64_t ld_a, int64_t b, int64_t rows_b, int64_t width_b,
                     int64_t ld_b) {
  return tim::share_bytes({(const void*)a, rows_a, width_a, ld_a}, {(const void*)b, rows_b, width_b, ld_b});
}
""")
    so = str(tmp_path / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", so, str(src)], check=True)
    share = ctypes.CDLL(so).share
    share.argtypes = [ctypes.c_int64] * 8
    import random
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(20000):
        def rows():
            width = rng.randint(1, 9)
            return rng.randint(100, 160), rng.randint(1, 6), width, width + rng.choice([0, 1, 2, 7, 13])
        a, b = rows(), rows()
        if rng.random() < 0.4:
            b = (*b[:3], max(a[3], b[2]))
        of = lambda p, n, width, ld: {p + i * ld + k for i in range(n) for k in range(width)}
        want = bool(of(*a) & of(*b))
        seen[want] += 1
        assert share(*a, *b) == share(*b, *a) == want, (a, b)
    assert min(seen) > 2000
    assert not share(0, 5, 4, 4, 100, 5, 4, 4) and not share(100, 0, 4, 4, 100, 5, 4, 4)  # nothing there
    far = 1 << 46
    assert not share(far, 1 << 23, 1 << 20, 1 << 40, 1 << 45, 1, 8, 8) and share(far, 1 << 23, 8, 1 << 40, far + (5 << 40) + 7, 1, 1, 1)


AT = {k: (i + 1) << 24 for i, k in enumerate(("x", "rows", "grad", "base", "out", "gx", "ga", "gb", "ws"))}  # 16 MiB apart
AT_AD = dict(a=20 << 24, b=21 << 24, scales=22 << 24)


@pytest.mark.parametrize("over", ["x", "rows", "a", "b", "scales"])
def test_outputs_over_inputs_are_refused(lib, over):
    there = {**AT, **AT_AD}[over]
    add = {k: AT[k] for k in ("x", "rows", "base", "out", "ws")}
    if over != "x":
        assert _add(lib, ad=AT_AD, **{**add, "out": there}) == VALUE
    back = {k: AT[k] for k in ("x", "rows", "grad", "gx", "ga", "gb", "ws")}
    for k in ("gx", "ga", "gb"):
        assert _back(lib, ad=AT_AD, **{**back, k: there}) == VALUE
        if k != "gx":
            assert _back(lib, ad=AT_AD, **{**back, k: AT["grad"] + 4}) == VALUE
        for m in ("gx", "ga", "gb"):
            if k != m:
                assert _back(lib, ad=AT_AD, **{**back, k: AT[m]}) == VALUE


def test_shifted_outputs_are_refused(lib):
    add = {k: AT[k] for k in ("x", "rows", "base", "out", "ws")}
    for shift in (4, 64, -64, 4 * 5 * 16 - 4):  # base's rows one on, and its last element
        assert _add(lib, ad=AT_AD, **{**add, "out": AT["base"] + shift}) == VALUE
    assert _embed(lib, table=AT["x"], tokens=AT["rows"], out=AT["x"] + 10 * 8 * 2 - 4) == VALUE
    assert _embed(lib, table=AT["x"], tokens=AT["rows"], out=AT["rows"] + 12) == VALUE
    assert _embed_back(lib, grad=AT["x"], tokens=AT["rows"], table=AT["x"], ws=AT["ws"]) == VALUE
    assert _embed_back(lib, grad=AT["x"], tokens=AT["rows"], table=AT["rows"] - 4, ws=AT["ws"]) == VALUE
