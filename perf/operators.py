"""Timed cases of the 4-bit head and of the changed logits, each in two forms.

`own` chooses the form: the package's calls (true) or the same mathematics in elementary torch operations in 32 bits
(false). A case is one call, or the two that belong together, as a rollout engine or a trainer makes it:

  quant     hidden rows or head weights to 4-bit microscaled floating point and back to the values they stand for
  product   logits of 4-bit hidden rows against a 4-bit head
  adjust    logits changed by penalties, biases and grammar masks, as a sampler reads them
  logprobs  log-probs, entropies and log-normalisers of sampled tokens under the changed logits
  backward  their gradient with respect to the logits

Inputs are synthetic and made from the seed alone. Token streams follow Zipf's law, so tokens repeat as text does;
logits are normal with the sampled token lifted, as a trained model's are; half of the grammar states allow nearly all
of the vocabulary and half a few tokens. The listed cases stand for the ranges `draw` samples from.
"""

from __future__ import annotations

import math

import torch

own = False

W_STD = 0.02           # usual initialiser range of head weights
LIFT = 9.0             # of the sampled token's logit
BLOCK = 32             # elements per shared scale
ELEMENTS = 1 << 26     # of a block of rows in the plain forms
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the hidden rows of a small decode step: launch latency
        {"name": "quant_64", "kind": "quant", "rows": 64, "d": 2048, "dtype": "bf16"},
        # the whole head after a policy update, as the rollout engine reloads it
        {"name": "quant_head", "kind": "quant", "rows": 151936, "d": 4096, "dtype": "bf16"},
        # one response in flight
        {"name": "product_1", "kind": "product", "T": 1, "d": 2048, "V": 151936, "tau": 1.0, "dtype": "f32"},
        # an ordinary decode step at temperature 0.7, the widest configuration
        {"name": "product_48", "kind": "product", "T": 48, "d": 5120, "V": 152064, "tau": 0.7, "dtype": "f32"},
        # a chunk of a short prompt scored by the engine, an odd vocabulary, logits kept in bf16
        {"name": "product_333", "kind": "product", "T": 333, "d": 1536, "V": 50257, "tau": 1.0, "dtype": "bf16"},
        # a packed stream scored by the engine, for the mismatch between it and the trainer
        {"name": "product_2000", "kind": "product", "T": 2000, "d": 4096, "V": 151936, "tau": 1.0, "dtype": "f32"},
        # a few long responses with penalties and a bias list, logits in bf16
        {"name": "adjust_7", "kind": "adjust", "T": 7, "V": 151936, "tau": 0.7, "dtype": "bf16", "history": 8192,
         "masks": 0, "bias": 16, "packed": False},
        # a full decode step under tool-call grammars
        {"name": "adjust_200", "kind": "adjust", "T": 200, "V": 151936, "tau": 1.0, "dtype": "f32", "history": 2048,
         "masks": 24, "bias": 0, "packed": False},
        # the log-probs that a decode step reports for its sampled tokens
        {"name": "logprobs_64", "kind": "logprobs", "T": 64, "V": 151936, "tau": 1.0, "dtype": "f32", "history": 1024,
         "masks": 8, "bias": 0, "packed": False},
        # the trainer scoring a packed stream of four responses under the sampler's penalties
        {"name": "logprobs_4096", "kind": "logprobs", "T": 4096, "V": 151936, "tau": 1.0, "dtype": "f32",
         "history": 1024, "masks": 0, "bias": 0, "packed": True},
        # a short batch with an entropy bonus under grammar masks, logits in fp16
        {"name": "backward_150", "kind": "backward", "T": 150, "V": 50257, "tau": 0.7, "dtype": "f16", "grad": "f32",
         "history": 150, "masks": 6, "bias": 8, "packed": True, "entropy": True},
        # gradients of the policy loss over a packed stream, handed on in bf16
        {"name": "backward_2047", "kind": "backward", "T": 2047, "V": 151936, "tau": 1.0, "dtype": "f32",
         "grad": "bf16", "history": 1024, "masks": 0, "bias": 0, "packed": True, "entropy": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["quant", "product", "product", "adjust", "logprobs", "logprobs", "backward", "backward"])
    if kind == "quant":
        d = rng.choice([256, 1024, 1536, 2048, 3584, 4096, 5120, 8192])
        return {"kind": kind, "rows": _log_int(rng, 1, min(152064, 151936 * 4096 // d)), "d": d,
                "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
    tau = rng.choice([1.0, 1.0, 0.7, 0.6])
    V = rng.choice([32000, 50257, 131072, 151936, 152064, _log_int(rng, 1000, 20000)])
    if kind == "product":
        d = 128 * _log_int(rng, 2, 64)
        top = 2000 * 4096 * 151936 // (d * V)
        return {"kind": kind, "T": _log_int(rng, 1, min(2000, top)), "d": d, "V": V, "tau": tau,
                "dtype": rng.choice(["f32", "f32", "bf16", "f16"])}
    packed = kind == "backward" or (kind == "logprobs" and rng.random() < 0.5)
    T = _log_int(rng, 1, 2000 if packed else 256)
    case = {"kind": kind, "T": T, "V": V, "tau": tau, "dtype": rng.choice(["f32", "f32", "bf16", "f16"]),
            "history": _log_int(rng, 1, 2048 if packed else 32768), "masks": rng.choice([0, 0, _log_int(rng, 1, 64)]),
            "bias": rng.choice([0, 0, _log_int(rng, 1, 300)]), "packed": packed}
    if kind == "backward":
        case["grad"] = rng.choice(["f32", "bf16", case["dtype"]])
        case["entropy"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------ inputs


def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 32 + k)
    return g


def _rows(n, d, dtype, std, g):
    """n rows of d normal values in dtype; with std None, rows of root mean square one whose elements differ in scale."""
    x = torch.empty((n, d), dtype=dtype, device="cuda")
    step = max(1, ELEMENTS // d)
    gain = None if std is not None else torch.exp(0.5 * torch.randn(d, generator=g, device="cuda"))
    for r in range(0, n, step):
        y = torch.randn((min(step, n - r), d), generator=g, device="cuda")
        y = y * std if std is not None else y * gain
        x[r:r + step] = (y if std is not None else y * torch.rsqrt(y.square().mean(1, keepdim=True))).to(dtype)
    return x


def _zipf(n, V, g):
    """n token ids whose ranks follow p(rank) ~ 1 / rank, spread over the vocabulary."""
    rank = torch.exp(torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * math.log(V + 1.0)).long() - 1
    return (rank.clamp_(0, V - 1) * 7919 % V).to(torch.int32)


def _spans(case, seed):
    """(begin, split, end, stream length) of the rows' histories: prompt [begin, split), output [split, end).

    Packed rows are the tokens of responses of `history` tokens behind a prompt of a quarter of that, each row's output
    all before it; the others are the requests of a decode step, histories from a quarter of `history` to all of it."""
    T, top = case["T"], case["history"]
    if case["packed"]:
        prompt = max(1, top // 4)
        t = torch.arange(T)
        begin = t // top * (top + prompt)
        split = begin + prompt
        return begin, split, split + t % top, (T + top - 1) // top * (top + prompt)
    length = torch.linspace(max(1, top // 4), top, T).round().long() if T > 1 else torch.tensor([top])
    length = length[torch.randperm(T, generator=torch.Generator().manual_seed(int(seed)))]
    end = torch.cumsum(length, 0)
    begin = end - length
    return begin, begin + length // 3, end, int(end[-1])


def _masks(case, tokens, g):
    """(int32 words [masks, ceil(V / 32)], int32 mask of each row, -1 for none); every row's token is allowed."""
    T, V, n = case["T"], case["V"], case["masks"]
    row = torch.randint(-1, n, (T,), generator=g, device="cuda")
    keep = torch.where(torch.arange(n, device="cuda") % 2 == 0, 0.9, min(1.0, 40.0 / V))
    allowed = torch.rand((n, V), generator=g, device="cuda") < keep[:, None]
    has = (row >= 0).nonzero()[:, 0]
    allowed[row[has], tokens[has].long()] = True
    words = (V + 31) // 32
    bits = torch.zeros((n, words * 32), dtype=torch.int64, device="cuda")
    bits[:, :V] = allowed
    packed = (bits.view(n, words, 32) << torch.arange(32, device="cuda")).sum(2)
    packed = torch.where(packed >= 1 << 31, packed - (1 << 32), packed)
    return packed.to(torch.int32), row.to(torch.int32)


def _prepare_logits(case, seed):
    T, V, kind = case["T"], case["V"], case["kind"]
    g = [_gen(seed, k) for k in range(10)]
    st = {"kind": kind, "tau": case["tau"], "V": V, "packed": case["packed"]}
    begin, split, end, n = _spans(case, seed)
    st["longest"] = int((end - begin).max())
    st["history"] = _zipf(n, V, g[0])
    st["begin"], st["split"], st["end"] = (x.cuda() for x in (begin, split, end))
    if case["packed"]:  # row t scores the token that follows its history
        st["tokens"] = st["history"][st["end"]].contiguous()
    else:
        st["tokens"] = _zipf(T, V, g[1])
    if case["packed"]:  # one policy: the same penalties on every row
        rho, f, p = (torch.full((T,), x, device="cuda") for x in (1.1, 0.1, 0.2))
    else:               # requests with settings of their own, some with none
        pick = torch.rand((3, T), generator=g[2], device="cuda")
        rho = torch.where(pick[0] < 0.5, 1.0, 1.0 + 0.3 * pick[0])
        f, p = (torch.where(x < 0.3, 0.0, 0.5 * x) for x in pick[1:])
    st["rho"], st["f"], st["p"] = rho, f, p
    dtype = DTYPES[case["dtype"]]
    z = torch.empty((T, V), dtype=dtype, device="cuda")
    step = max(1, ELEMENTS // V)
    for r in range(0, T, step):
        x = 2.5 * torch.randn((min(step, T - r), V), generator=g[3], device="cuda")
        x.scatter_add_(1, st["tokens"][r:r + step].long()[:, None], torch.full((x.shape[0], 1), LIFT, device="cuda"))
        z[r:r + step] = x.to(dtype)
    st["logits"] = z
    st["mask"] = st["mask_rows"] = None
    if case["masks"]:
        st["mask"], st["mask_rows"] = _masks(case, st["tokens"], g[4])
    st["bias_ids"] = None
    if case["bias"]:  # four lists, each shared by the rows that use it: some tokens banned, others moved
        n = min(case["bias"], V)
        st["bias_ids"] = torch.cat([torch.randperm(V, generator=g[5], device="cuda")[:n] for _ in range(4)]).to(
            torch.int32)
        v = 2.0 * torch.randn(4 * n, generator=g[6], device="cuda")
        st["bias_values"] = torch.where(torch.rand(4 * n, generator=g[7], device="cuda") < 0.3, -100.0, v)
        st["bias_begin"] = n * torch.randint(0, 4, (T,), generator=g[8], device="cuda")
        st["bias_end"] = st["bias_begin"] + n
        st["bias_n"] = n
    if kind == "backward":
        st["grad"] = DTYPES[case["grad"]]
        _, st["ent"], st["lse"] = _plain_logprobs(st)
        st["g"] = torch.randn(T, generator=g[9], device="cuda")
        st["e"] = torch.full((T,), -0.05, device="cuda") if case["entropy"] else None
    if own:
        import paper_2605_14220_amd as tim

        st["rules"] = tim.LogitRules(
            history=st["history"], hist_begin=st["begin"], hist_split=st["split"], hist_end=st["end"],
            repetition=rho, frequency=f, presence=p, bias_ids=st["bias_ids"], bias_values=st.get("bias_values"),
            bias_begin=st.get("bias_begin"), bias_end=st.get("bias_end"), mask=st["mask"], mask_rows=st["mask_rows"])
        if kind == "logprobs":
            st["ws"] = torch.empty(tim.logits_logprobs_workspace_size(T, V), dtype=torch.uint8, device="cuda")
    return st


def prepare(case, seed):
    kind = case["kind"]
    if kind == "quant":
        std = W_STD if case["rows"] > 4096 else None
        return {"kind": kind, "x": _rows(case["rows"], case["d"], DTYPES[case["dtype"]], std, _gen(seed, 0))}
    if kind != "product":
        return _prepare_logits(case, seed)
    st = {"kind": kind, "tau": case["tau"], "dtype": DTYPES[case["dtype"]]}
    for name, n, std, k in (("h", case["T"], None, 0), ("w", case["V"], W_STD, 1)):
        x = _rows(n, case["d"], torch.bfloat16, std, _gen(seed, k))
        codes = torch.empty((n, case["d"] // 2), dtype=torch.uint8, device="cuda")
        scales = torch.empty((n, case["d"] // BLOCK), dtype=torch.uint8, device="cuda")
        step = max(1, ELEMENTS // case["d"])
        for r in range(0, n, step):
            e, q = _quantise(x[r:r + step].float())
            nearest = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda")
            c = torch.bucketize(q.abs(), nearest) + 8 * (q < 0)
            codes[r:r + step] = (c[:, 0::2] + 16 * c[:, 1::2]).to(torch.uint8)
            scales[r:r + step] = (e + 127).to(torch.uint8)
        st[name + "_codes"], st[name + "_scales"] = codes, scales
    if own:
        import paper_2605_14220_amd as tim

        st["h"] = tim.Mxfp4(st["h_codes"], st["h_scales"])
        st["w"] = tim.Mxfp4(st["w_codes"], st["w_scales"])
    return st


# ------------------------------------------------------------------ plain forms


def _quantise(x):
    """(exponent of each block's scale [rows, d / 32], elements in units of their scale [rows, d]) of fp32 rows."""
    rows, d = x.shape
    b = x.view(rows, d // BLOCK, BLOCK)
    top = b.abs().amax(2)
    _, e = torch.frexp(top)  # top = m 2^e with m in [1/2, 1)
    e = torch.where(top > 0, (e - 3).clamp(min=-127), -127)
    v = torch.ldexp(b, -e[:, :, None])
    a = v.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    q = torch.copysign((torch.round(a / step) * step).clamp(max=6.0), v)
    return e, q.view(rows, d)


def _plain_quant(x):
    out = torch.empty_like(x, dtype=torch.bfloat16)
    step = max(1, ELEMENTS // x.shape[1])
    for r in range(0, x.shape[0], step):
        e, q = _quantise(x[r:r + step].float())
        out[r:r + step] = torch.ldexp(q.view(*e.shape, BLOCK), e[:, :, None]).view(q.shape).to(torch.bfloat16)
    return out


def _values(codes, scales):
    """fp32 values of 4-bit codes and their scales."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                         device=codes.device)
    out = torch.empty((codes.shape[0], codes.shape[1] * 2), device=codes.device)
    out[:, 0::2] = table[(codes & 15).int()]
    out[:, 1::2] = table[(codes >> 4).int()]
    scale = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    return (out.view(*scales.shape, BLOCK) * scale[:, :, None]).view(out.shape)


def _plain_product(st):
    z = _values(st["h_codes"], st["h_scales"]) @ _values(st["w_codes"], st["w_scales"]).T
    return z.mul_(1.0 / st["tau"]).to(st["dtype"])


def _adjusted(st, r0, r1):
    """(changed logits fp32, slope of each with respect to its logit) of rows r0 .. r1."""
    V, s = st["V"], slice(r0, r1)
    z = st["logits"][s].float()
    idx = st["begin"][s, None] + torch.arange(st["longest"], device=z.device)
    tok = st["history"][idx.clamp(max=st["history"].numel() - 1)].long()
    there = idx < st["end"][s, None]
    seen = torch.zeros_like(z).scatter_add_(1, tok, there.float()) > 0
    count = torch.zeros_like(z).scatter_add_(1, tok, (there & (idx >= st["split"][s, None])).float())
    rho = st["rho"][s, None]
    x = torch.where(seen, torch.where(z > 0, z / rho, z * rho), z)
    x = x - st["f"][s, None] * count - st["p"][s, None] * (count > 0)
    slope = torch.where(seen, torch.where(z > 0, 1.0 / rho, rho), 1.0) * (1.0 / st["tau"])
    if st["bias_ids"] is not None:
        k = st["bias_begin"][s, None] + torch.arange(st["bias_n"], device=z.device)
        x.scatter_add_(1, st["bias_ids"][k].long(), st["bias_values"][k])
    x = x * (1.0 / st["tau"])
    if st["mask"] is not None:
        m = st["mask_rows"][s].long()
        bits = (st["mask"][m.clamp(min=0)][:, :, None] >> torch.arange(32, device=z.device, dtype=torch.int32)) & 1
        off = (bits.view(m.shape[0], -1)[:, :V] == 0) & (m >= 0)[:, None]
        x = x.masked_fill(off, -math.inf)
        slope = slope.masked_fill(off, 0.0)
    return x, slope


def _row_blocks(st):
    T = st["logits"].shape[0]
    step = max(1, ELEMENTS // st["V"])
    return [(r, min(r + step, T)) for r in range(0, T, step)]


def _plain_adjust(st):
    out = torch.empty_like(st["logits"])
    for r0, r1 in _row_blocks(st):
        out[r0:r1] = _adjusted(st, r0, r1)[0].to(out.dtype)
    return out


def _plain_logprobs(st):
    T = st["logits"].shape[0]
    logp, ent, lse = (torch.empty(T, device=st["logits"].device) for _ in range(3))
    for r0, r1 in _row_blocks(st):
        x = _adjusted(st, r0, r1)[0]
        m = x.amax(1)
        q = x - m[:, None]
        e = torch.exp(q)
        s = e.sum(1)
        log_s = torch.log(s)
        logp[r0:r1] = q.gather(1, st["tokens"][r0:r1].long()[:, None])[:, 0] - log_s
        ent[r0:r1] = log_s - torch.where(e > 0, e * q, 0.0).sum(1) / s
        lse[r0:r1] = m + log_s
    return logp, ent, lse


def _plain_backward(st):
    out = torch.empty_like(st["logits"], dtype=st["grad"])
    for r0, r1 in _row_blocks(st):
        s = slice(r0, r1)
        x, slope = _adjusted(st, r0, r1)
        g = st["g"][s, None]
        q = x - st["lse"][s, None]
        p = torch.exp(q)
        up = -p * g if st["e"] is None else -p * (
            g + st["e"][s, None] * (torch.where(p > 0, q, 0.0) + st["ent"][s, None]))
        up.scatter_add_(1, st["tokens"][s].long()[:, None], g)
        out[s] = (up * slope).to(out.dtype)
    return out


def run(st):
    kind = st["kind"]
    if not own:
        return {"quant": lambda s: _plain_quant(s["x"]), "product": _plain_product, "adjust": _plain_adjust,
                "logprobs": _plain_logprobs, "backward": _plain_backward}[kind](st)
    import paper_2605_14220_amd as tim

    if kind == "quant":
        return tim.mxfp4_dequantize(tim.mxfp4_quantize(st["x"]))
    if kind == "product":
        return tim.mxfp4_logits(st["h"], st["w"], st["tau"], dtype=st["dtype"])
    if kind == "adjust":
        return tim.logits_adjust(st["logits"], st["rules"], st["tau"])
    if kind == "logprobs":
        return tim.logits_logprobs(st["logits"], st["tokens"], st["rules"], st["tau"], lse=True, workspace=st["ws"])
    return tim.logits_logprobs_backward(st["logits"], st["tokens"], st["lse"], st["g"], st["rules"], st["tau"],
                                        entropy=st["ent"], grad_entropy=st["e"], dtype=st["grad"])


def work(case):
    if case["kind"] == "quant":  # rows read, codes and scales written, values written
        n = case["rows"] * case["d"]
        return {"bytes": n * (SIZES[case["dtype"]] + 2) + n // 2 + n // BLOCK, "flops": 4 * n}
    T, V = case["T"], case["V"]
    if case["kind"] == "product":
        d = case["d"]
        return {"bytes": (T + V) * (d // 2 + d // BLOCK) + T * V * SIZES[case["dtype"]], "flops": 2 * T * V * d}
    _, _, _, n = _spans(case, 0)
    size = T * V * SIZES[case["dtype"]] + 4 * n + 40 * T + case["masks"] * ((V + 31) // 32) * 4 + 32 * case["bias"]
    if case["kind"] == "adjust":
        return {"bytes": size + T * V * SIZES[case["dtype"]], "flops": 2 * T * V}
    if case["kind"] == "logprobs":
        return {"bytes": size + 16 * T, "flops": 6 * T * V}
    return {"bytes": size + T * V * SIZES[case["grad"]] + 20 * T, "flops": 6 * T * V}


# ------------------------------------------------------------------ in 64 bits, from the definitions


def _exact_values(codes, scales):
    """Sign, two exponent bits, one mantissa bit: (-1)^s 2^(e - 1) (1 + m / 2), or m / 2 where e = 0; times 2^(scale - 127)."""
    c = torch.stack((codes & 15, codes >> 4), 2).view(codes.shape[0], -1).long()
    sign = 1.0 - 2.0 * (c >> 3).double()
    e, m = (c >> 1) & 3, (c & 1).double()
    v = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.exp2((e - 1).double()))
    return sign * v * torch.exp2(scales.double() - 127.0).repeat_interleave(BLOCK, 1)


def _exact_quant(x):
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    step = max(1, (ELEMENTS >> 2) // x.shape[1])
    powers = torch.exp2(torch.arange(-160, 129, device=x.device).double())
    for r in range(0, x.shape[0], step):
        b = x[r:r + step].double().unflatten(1, (-1, BLOCK))
        top = b.abs().max(2).values
        low = powers[torch.searchsorted(powers, top.contiguous(), right=True).clamp(min=1) - 1]  # largest power <= top
        scale = (low / 4.0).clamp(min=2.0 ** -127)[:, :, None]
        a = b.abs() / scale
        hi = torch.searchsorted(grid, a.contiguous()).clamp(max=7)
        lo = (hi - 1).clamp(min=0)
        below, above = a - grid[lo], grid[hi] - a
        # halfway goes to the even code; beyond the largest value hi is that value
        pick = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
        pick = torch.where(a > 6.0, 7, pick)
        out[r:r + step] = (torch.sign(b) * grid[pick] * scale).flatten(1)
    return out


def _exact_rows(st, r0, r1):
    """The changed logits and their slopes of rows r0 .. r1, each distinct (row, token) of a history changed once."""
    V, n = st["V"], r1 - r0
    z = st["logits"][r0:r1].double().contiguous()
    slope = torch.ones_like(z)
    begin, split, end = (st[k][r0:r1] for k in ("begin", "split", "end"))
    rho, f, p = (st[k][r0:r1].double() for k in ("rho", "f", "p"))

    def pairs(a, b):
        length = b - a
        row = torch.repeat_interleave(torch.arange(n, device=z.device), length)
        at = torch.arange(row.numel(), device=z.device) - (torch.cumsum(length, 0) - length)[row] + a[row]
        return torch.unique(row * V + st["history"][at].long(), return_counts=True)

    flat, sl = z.view(-1), slope.view(-1)
    keys, _ = pairs(begin, end)
    row, v = keys // V, flat[keys]
    flat[keys] = torch.where(v > 0, v / rho[row], v * rho[row])
    sl[keys] = torch.where(v > 0, 1.0 / rho[row], rho[row])
    keys, c = pairs(split, end)
    flat[keys] -= f[keys // V] * c.double() + p[keys // V]
    if st["bias_ids"] is not None:
        for i in range(n):
            b = slice(int(st["bias_begin"][r0 + i]), int(st["bias_end"][r0 + i]))
            z[i, st["bias_ids"][b].long()] += st["bias_values"][b].double()
    inv = float(torch.tensor(1.0 / st["tau"], dtype=torch.float32))
    z *= inv
    slope *= inv
    if st["mask"] is not None:
        v = torch.arange(V, device=z.device)
        for i in range(n):
            m = int(st["mask_rows"][r0 + i])
            if m >= 0:
                off = (st["mask"][m][v // 32].long() >> (v % 32)) % 2 == 0
                z[i, off] = -math.inf
                slope[i, off] = 0.0
    return z, slope


def exact(case, seed):
    kind = case["kind"]
    st = prepare(case, seed)
    if kind == "quant":
        return _exact_quant(st["x"])
    if kind == "product":
        h = _exact_values(st["h_codes"], st["h_scales"])
        z = torch.empty((case["T"], case["V"]), dtype=torch.float64, device="cuda")
        step = max(1, (ELEMENTS >> 1) // case["d"])
        for v in range(0, case["V"], step):
            z[:, v:v + step] = h @ _exact_values(st["w_codes"][v:v + step], st["w_scales"][v:v + step]).T
        return z.mul_(float(torch.tensor(1.0 / st["tau"], dtype=torch.float32)))
    T, V = case["T"], case["V"]
    rows = [torch.empty(T, dtype=torch.float64, device="cuda") for _ in range(3)]
    whole = None if kind == "logprobs" else torch.empty((T, V), dtype=torch.float64, device="cuda")
    step = max(1, (ELEMENTS >> 1) // V)
    for r in range(0, T, step):
        n = min(step, T - r)
        x, slope = _exact_rows(st, r, r + n)
        if kind == "adjust":
            whole[r:r + n] = x
            continue
        tok = st["tokens"][r:r + n].long()
        if kind == "logprobs":
            lse = torch.logsumexp(x, 1)
            q = x - lse[:, None]
            rows[0][r:r + n] = q[torch.arange(n, device="cuda"), tok]
            rows[1][r:r + n] = -torch.nan_to_num(q * q.exp(), nan=0.0).sum(1)
            rows[2][r:r + n] = lse
            continue
        q = x - st["lse"][r:r + n, None].double()
        p = q.exp()
        up = torch.zeros_like(x)
        up[torch.arange(n, device="cuda"), tok] = st["g"][r:r + n].double()
        up -= p * st["g"][r:r + n, None].double()
        if st["e"] is not None:
            h = st["ent"][r:r + n, None].double()
            up -= st["e"][r:r + n, None].double() * torch.nan_to_num(p * (q + h), nan=0.0)
        whole[r:r + n] = up * slope
    return tuple(rows) if kind == "logprobs" else whole
