"""The entry points of include/tim_policy.h on the host: exported, sized by the documented formula, and refusing every
bad argument with the documented status before anything is enqueued. No call here reaches a launch."""

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
FAKE, MIS8, MIS2, MIS1 = 0x10000, 0x10008, 0x10002, 0x10001  # never dereferenced
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    return tim.load_library()


def test_every_declared_function_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "tim_policy.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"^\s*\w+\s+(tim_\w+)\s*\(", text, flags=re.M)))
    assert names == ["tim_logits_adjust", "tim_logits_logprobs", "tim_logits_logprobs_backward",
                     "tim_logits_logprobs_workspace_size", "tim_mxfp4_dequantize", "tim_mxfp4_logits",
                     "tim_mxfp4_quantize"]
    out = subprocess.run(["nm", "-D", "--defined-only", tim.LIB_PATH], capture_output=True, text=True, check=True).stdout
    exported = set(re.findall(r"\bT\s+(\w+)$", out, flags=re.M))
    assert set(names) <= exported


def test_header_is_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#define __HIP_PLATFORM_AMD__ 1\n#include "tim_policy.h"\n'
                   "int main(void) { tim_logit_rules r = {0}; return (int)sizeof(r); }\n")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), "-I",
                    "/opt/rocm/include", str(src)], check=True)


def test_rules_struct_matches_the_header(tmp_path):
    """The binding's struct has the header's fields in order, sizes and offsets."""
    fields = [f for f, _ in tim._LogitRules._fields_]
    src = tmp_path / "use.c"
    src.write_text('#define __HIP_PLATFORM_AMD__ 1\n#include <stdio.h>\n#include "tim_policy.h"\nint main(void) {\n'
                   + "".join(f'printf("%zu ", offsetof(tim_logit_rules, {f}));\n' for f in fields)
                   + 'printf("%zu", sizeof(tim_logit_rules)); return 0; }\n')
    exe = str(tmp_path / "use")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", str(src), "-o",
                    exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(tim._LogitRules, f).offset for f in fields] + [ctypes.sizeof(tim._LogitRules)]


def test_workspace_size(lib):
    assert tim.logits_logprobs_workspace_size(5, 151936) == 5 * 19 * 16
    assert tim.logits_logprobs_workspace_size(3, 8192) == 3 * 16
    assert tim.logits_logprobs_workspace_size(3, 8193) == 3 * 32
    for T, V in ((0, 10), (-1, 10), (4, 0), (4, tim.MAX_VOCAB + 1)):
        assert tim.logits_logprobs_workspace_size(T, V) == 0


def _quant(lib, x=FAKE, dtype=BF16, rows=4, d=64, ld=64, codes=FAKE, scales=FAKE):
    return lib.tim_mxfp4_quantize(x, dtype, rows, d, ld, codes, scales, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(rows=-1), Status.ERR_SHAPE), (dict(d=0), Status.ERR_SHAPE), (dict(d=33, ld=64), Status.ERR_SHAPE),
    (dict(d=-32), Status.ERR_SHAPE), (dict(ld=63), Status.ERR_SHAPE), (dict(dtype=3), Status.ERR_VALUE),
    (dict(dtype=-1), Status.ERR_VALUE), (dict(x=None), Status.ERR_NULL), (dict(codes=None), Status.ERR_NULL),
    (dict(scales=None), Status.ERR_NULL), (dict(x=MIS1), Status.ERR_VALUE), (dict(x=MIS2, dtype=F32), Status.ERR_VALUE),
    (dict(rows=0, x=None, codes=None, scales=None), Status.OK)])
def test_quantize_refusals(lib, kw, expect):
    assert _quant(lib, **kw) == expect


def _dequant(lib, codes=FAKE, scales=FAKE, rows=4, d=64, out=FAKE, dtype=BF16):
    return lib.tim_mxfp4_dequantize(codes, scales, rows, d, out, dtype, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(rows=-1), Status.ERR_SHAPE), (dict(d=16), Status.ERR_SHAPE), (dict(dtype=F16), Status.ERR_VALUE),
    (dict(dtype=9), Status.ERR_VALUE), (dict(codes=None), Status.ERR_NULL), (dict(scales=None), Status.ERR_NULL),
    (dict(out=None), Status.ERR_NULL), (dict(out=MIS1), Status.ERR_VALUE), (dict(out=MIS2, dtype=F32), Status.ERR_VALUE),
    (dict(rows=0, out=None), Status.OK)])
def test_dequantize_refusals(lib, kw, expect):
    assert _dequant(lib, **kw) == expect


def _product(lib, hc=FAKE, hs=FAKE, wc=FAKE, ws=FAKE, T=4, d=256, V=100, tau=1.0, z=FAKE, dtype=F32, ld=100):
    return lib.tim_mxfp4_logits(hc, hs, wc, ws, T, d, V, tau, z, dtype, ld, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(T=-1), Status.ERR_SHAPE), (dict(d=0), Status.ERR_SHAPE), (dict(d=64), Status.ERR_SHAPE),
    (dict(d=192), Status.ERR_SHAPE), (dict(d=2 ** 20 + 128), Status.ERR_SHAPE), (dict(V=0), Status.ERR_SHAPE), (dict(V=2048 * 256 + 1, ld=1 << 20), Status.ERR_SHAPE),
    (dict(ld=99), Status.ERR_SHAPE), (dict(tau=0.0), Status.ERR_VALUE), (dict(tau=float("nan")), Status.ERR_VALUE),
    (dict(tau=float("inf")), Status.ERR_VALUE), (dict(tau=-1.0), Status.ERR_VALUE), (dict(dtype=3), Status.ERR_VALUE),
    (dict(hc=None), Status.ERR_NULL), (dict(hs=None), Status.ERR_NULL), (dict(wc=None), Status.ERR_NULL),
    (dict(ws=None), Status.ERR_NULL), (dict(z=None), Status.ERR_NULL), (dict(hc=MIS8), Status.ERR_VALUE),
    (dict(wc=MIS8), Status.ERR_VALUE), (dict(hs=MIS2), Status.ERR_VALUE), (dict(ws=MIS1), Status.ERR_VALUE),
    (dict(z=MIS2), Status.ERR_VALUE), (dict(z=MIS1, dtype=BF16), Status.ERR_VALUE),
    (dict(T=0, hc=None, z=None), Status.OK)])
def test_product_refusals(lib, kw, expect):
    assert _product(lib, **kw) == expect


CALLS = ["adjust", "logprobs", "backward"]


def _changed(lib, call, rules=None, logits=FAKE, dtype=F32, T=4, V=100, ld=100, tau=1.0, **kw):
    r = None if rules is None else ctypes.byref(tim._LogitRules(**rules))
    a = (logits, dtype, T, V, ld)
    if call == "adjust":
        return lib.tim_logits_adjust(*a, r, tau, kw.get("out", FAKE + 4096), kw.get("out_ld", 100), None)
    if call == "logprobs":
        return lib.tim_logits_logprobs(*a, kw.get("tokens", FAKE), r, tau, kw.get("logp", FAKE), None, None,
                                       kw.get("ws", FAKE), kw.get("ws_bytes", 1 << 40), None)
    return lib.tim_logits_logprobs_backward(*a, kw.get("tokens", FAKE), r, tau, kw.get("lse", FAKE),
                                            kw.get("entropy"), kw.get("grad_logp", FAKE), kw.get("grad_entropy"),
                                            kw.get("out", FAKE + 4096), kw.get("out_dtype", F32),
                                            kw.get("out_ld", 100), None)


HIST = dict(history=FAKE, history_len=8, hist_begin=FAKE, hist_end=FAKE)
BIAS = dict(bias_ids=FAKE, bias_values=FAKE, bias_len=4, bias_begin=FAKE, bias_end=FAKE)
MASK = dict(mask=FAKE, n_masks=2, mask_ld=4)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw,expect", [
    (dict(T=-1), Status.ERR_SHAPE), (dict(V=0), Status.ERR_SHAPE), (dict(ld=99), Status.ERR_SHAPE),
    (dict(V=2048 * 256 + 1, ld=1 << 20, out_ld=1 << 20), Status.ERR_SHAPE), (dict(tau=0.0), Status.ERR_VALUE),
    (dict(tau=float("nan")), Status.ERR_VALUE), (dict(dtype=5), Status.ERR_VALUE), (dict(logits=None), Status.ERR_NULL),
    (dict(logits=MIS2), Status.ERR_VALUE), (dict(logits=MIS1, dtype=F16, out_dtype=F16), Status.ERR_VALUE),
    (dict(rules=HIST | dict(history_len=-1)), Status.ERR_SHAPE), (dict(rules=HIST | dict(hist_begin=None)), Status.ERR_NULL),
    (dict(rules=HIST | dict(hist_end=None)), Status.ERR_NULL), (dict(rules=HIST | dict(history=MIS2)), Status.ERR_VALUE),
    (dict(rules=BIAS | dict(bias_len=-1)), Status.ERR_SHAPE), (dict(rules=BIAS | dict(bias_len=2 ** 31 - 1)), Status.ERR_SHAPE),
    (dict(rules=BIAS | dict(bias_values=None)), Status.ERR_NULL), (dict(rules=BIAS | dict(bias_begin=None)), Status.ERR_NULL),
    (dict(rules=BIAS | dict(bias_end=None)), Status.ERR_NULL), (dict(rules=MASK | dict(n_masks=-1)), Status.ERR_SHAPE),
    (dict(rules=MASK | dict(mask_ld=3)), Status.ERR_SHAPE), (dict(rules=MASK | dict(mask=MIS2)), Status.ERR_VALUE),
    (dict(T=0, logits=None, rules=HIST | dict(history_len=-1)), Status.OK)])
def test_changed_refusals(lib, call, kw, expect):
    assert _changed(lib, call, **kw) == expect


@pytest.mark.parametrize("call,kw,expect", [
    ("adjust", dict(out=None), Status.ERR_NULL), ("adjust", dict(out_ld=99), Status.ERR_SHAPE),
    ("adjust", dict(out=FAKE, ld=101), Status.ERR_SHAPE), ("adjust", dict(out=MIS2), Status.ERR_VALUE),
    ("logprobs", dict(tokens=None), Status.ERR_NULL), ("logprobs", dict(logp=None), Status.ERR_NULL),
    ("logprobs", dict(ws=None), Status.ERR_WORKSPACE), ("logprobs", dict(ws=MIS8), Status.ERR_WORKSPACE),
    ("logprobs", dict(ws_bytes=4 * 16 - 1), Status.ERR_WORKSPACE),
    ("backward", dict(tokens=None), Status.ERR_NULL), ("backward", dict(lse=None), Status.ERR_NULL),
    ("backward", dict(grad_logp=None), Status.ERR_NULL), ("backward", dict(out=None), Status.ERR_NULL),
    ("backward", dict(grad_entropy=FAKE), Status.ERR_NULL), ("backward", dict(out_dtype=7), Status.ERR_VALUE),
    ("backward", dict(out=MIS2), Status.ERR_VALUE), ("backward", dict(out_ld=99), Status.ERR_SHAPE),
    ("backward", dict(out=FAKE, ld=101), Status.ERR_SHAPE),
    ("backward", dict(out=FAKE, out_dtype=BF16), Status.ERR_SHAPE)])
def test_refusals_of_one_call(lib, call, kw, expect):
    assert _changed(lib, call, **kw) == expect


# ------------------------------------------------------------------ the binding's own checks, on CPU tensors


def _q(rows, d):
    return tim.Mxfp4(torch.zeros(rows, d // 2, dtype=torch.uint8), torch.zeros(rows, d // 32, dtype=torch.uint8))


@pytest.mark.parametrize("call,error", [
    (lambda: tim.mxfp4_quantize(torch.zeros(2, 64)), ValueError),                      # not on the GPU
    (lambda: tim.mxfp4_quantize(torch.zeros(2, 64, dtype=torch.float64)), TypeError),
    (lambda: tim.mxfp4_quantize(torch.zeros(2, 33)), ValueError),
    (lambda: tim.mxfp4_quantize(torch.zeros(2, 0)), ValueError),
    (lambda: tim.mxfp4_quantize(torch.zeros(64)), ValueError),
    (lambda: tim.mxfp4_quantize(torch.zeros(64, 64).T), ValueError),
    (lambda: tim.mxfp4_quantize(torch.zeros(1, 64).expand(4, 64)), ValueError),        # rows share elements
    (lambda: tim.mxfp4_dequantize(_q(2, 64)), ValueError),
    (lambda: tim.mxfp4_dequantize(tim.Mxfp4(torch.zeros(2, 32), torch.zeros(2, 2))), TypeError),
    (lambda: tim.mxfp4_logits(_q(2, 128), _q(3, 128)), ValueError),
    (lambda: tim.logits_adjust(torch.zeros(2, 8)), ValueError),
    (lambda: tim.logits_adjust(torch.zeros(2, 8, dtype=torch.float64)), TypeError),
    (lambda: tim.logits_adjust(torch.zeros(8, 2).T), ValueError),
    (lambda: tim.logits_logprobs(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)), ValueError),
    (lambda: tim.logits_logprobs_backward(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2),
                                          torch.zeros(2)), ValueError),
])
def test_binding_refuses(call, error):
    with pytest.raises(error):
        call()


@pytest.mark.parametrize("rules,error", [
    (dict(history=torch.zeros(3, dtype=torch.int32)), ValueError),
    (dict(history=torch.zeros(3), hist_begin=torch.zeros(2, dtype=torch.int64), hist_end=torch.zeros(2, dtype=torch.int64)), TypeError),
    (dict(history=torch.zeros(3, dtype=torch.int32), hist_begin=torch.zeros(2, dtype=torch.int32),
          hist_end=torch.zeros(2, dtype=torch.int64)), TypeError),
    (dict(history=torch.zeros(3, dtype=torch.int32), hist_begin=torch.zeros(2, dtype=torch.int64),
          hist_end=torch.zeros(3, dtype=torch.int64)), ValueError),
    (dict(repetition=torch.ones(3)), ValueError), (dict(presence=torch.ones(2, dtype=torch.float64)), TypeError),
    (dict(frequency=torch.ones(4)[::2]), ValueError),
    (dict(bias_ids=torch.zeros(3, dtype=torch.int32)), ValueError),
    (dict(bias_ids=torch.zeros(3, dtype=torch.int32), bias_values=torch.zeros(2), bias_begin=torch.zeros(2, dtype=torch.int64),
          bias_end=torch.zeros(2, dtype=torch.int64)), ValueError),
    (dict(mask=torch.zeros(2, 1, dtype=torch.int64)), TypeError), (dict(mask=torch.zeros(2, 1, dtype=torch.int32)), ValueError),
    (dict(mask=torch.zeros(3, 2, dtype=torch.int32)), ValueError),
    (dict(mask=torch.zeros(3, 2, dtype=torch.int32), mask_rows=torch.zeros(2, dtype=torch.int64)), TypeError),
])
def test_binding_refuses_rules(rules, error):
    with pytest.raises(error):
        tim.LogitRules(**rules)._struct("logits_adjust", 2, 40, torch.device("cpu"))


def test_rules_are_filled_again_when_a_field_or_its_storage_changes():
    cpu = torch.device("cpu")
    r = tim.LogitRules(repetition=torch.ones(3), mask=torch.zeros(3, 2, dtype=torch.int32))
    s = r._struct("logits_adjust", 3, 40, cpu)
    assert r._struct("logits_adjust", 3, 64, cpu) is s and s.repetition == r.repetition.data_ptr()
    r.repetition.mul_(2.0)  # contents may change
    assert r._struct("logits_adjust", 3, 40, cpu) is s
    with pytest.raises(ValueError):
        r._struct("logits_adjust", 3, 65, cpu)   # the masks are too short
    with pytest.raises(ValueError):
        r._struct("logits_adjust", 4, 40, cpu)
    r.repetition = torch.full((3,), 3.0)
    t = r._struct("logits_adjust", 3, 40, cpu)
    assert t is not s and t.repetition == r.repetition.data_ptr()
    r.repetition.data = torch.full((3,), 4.0)
    assert r._struct("logits_adjust", 3, 40, cpu).repetition == r.repetition.data_ptr()
    r.repetition.data = torch.ones(3, dtype=torch.float64)
    with pytest.raises(TypeError):
        r._struct("logits_adjust", 3, 40, cpu)
    r.repetition = None
    assert r._struct("logits_adjust", 3, 40, cpu).repetition is None


def test_rules_are_filled_again_when_a_tensor_is_cut_in_place():
    cpu = torch.device("cpu")
    r = tim.LogitRules(history=torch.zeros(9, dtype=torch.int32), hist_begin=torch.zeros(2, dtype=torch.int64),
                       hist_end=torch.zeros(2, dtype=torch.int64), mask=torch.zeros(8, 2, dtype=torch.int32),
                       mask_rows=torch.zeros(2, dtype=torch.int32))
    s = r._struct("logits_adjust", 2, 40, cpu)
    assert (s.history_len, s.n_masks, s.mask_ld) == (9, 8, 2)
    r.history.data = r.history[:5]
    r.mask.data = r.mask[::2]
    s = r._struct("logits_adjust", 2, 40, cpu)
    assert (s.history_len, s.n_masks, s.mask_ld) == (5, 4, 4)
    r.hist_end.resize_(1)
    with pytest.raises(ValueError):
        r._struct("logits_adjust", 2, 40, cpu)


@pytest.mark.parametrize("relaid,error", [
    (lambda t, spare: setattr(t, "data", spare[::2]), ValueError),             # every other element, the same address and count
    (lambda t, spare: t.as_strided_((4,), (0,)), ValueError),                  # one element four times
    (lambda t, spare: setattr(t, "data", t.data.view(torch.int32)), TypeError),  # the same bytes as another type
])
@pytest.mark.parametrize("mutated", ["repetition", "presence"])
def test_rules_refuse_a_tensor_laid_out_anew_in_place(relaid, error, mutated):
    """A used rule set refuses what a fresh one refuses: the address and the element count do not show the change."""
    cpu = torch.device("cpu")
    spare = torch.arange(8, dtype=torch.float32)
    r = tim.LogitRules(frequency=torch.ones(4), **{mutated: spare[:4]})
    s = r._struct("logits_adjust", 4, 40, cpu)
    t = getattr(r, mutated)
    relaid(t, spare)
    assert t.data_ptr() == getattr(s, mutated) and t.numel() == 4
    for rules in (r, tim.LogitRules(frequency=torch.ones(4), **{mutated: t})):
        with pytest.raises(error):
            rules._struct("logits_adjust", 4, 40, cpu)


def test_masks_laid_out_anew_in_place():
    cpu = torch.device("cpu")
    words = torch.zeros(4, 4, dtype=torch.int32)
    r = tim.LogitRules(mask=words, mask_rows=torch.zeros(3, dtype=torch.int32))
    assert r._struct("logits_adjust", 3, 128, cpu).mask_ld == 4
    r.mask.data = torch.as_strided(words, (2, 8), (8, 1))  # as many elements at the same address
    s = r._struct("logits_adjust", 3, 128, cpu)
    assert (s.n_masks, s.mask_ld) == (2, 8)
    r.mask.data = r.mask.view(torch.float32)
    with pytest.raises(TypeError):
        r._struct("logits_adjust", 3, 128, cpu)


@pytest.mark.parametrize("copied", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r))])
def test_rules_are_copied_after_a_call(copied):
    cpu = torch.device("cpu")
    r = tim.LogitRules(repetition=torch.ones(3), mask=torch.zeros(3, 2, dtype=torch.int32))
    r._struct("logits_adjust", 3, 40, cpu)
    c = copied(r)
    s = c._struct("logits_adjust", 3, 40, cpu)
    assert s.repetition == c.repetition.data_ptr() and s.mask == c.mask.data_ptr()
    assert torch.equal(c.repetition, r.repetition) and c.presence is None
