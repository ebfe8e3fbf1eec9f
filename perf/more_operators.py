"""Timed cases of the embedding and of low-rank adapters, each in two forms.

`own` chooses the form: the package's calls (true) or the same mathematics in elementary torch operations in 32 bits
(false). A case is one call, or the two that belong together, as a rollout engine or a trainer makes it:

  lookup    rows of the vocabulary's matrix for token ids, scaled: the other end of a tied head
  scatter   the gradient of that matrix from the gradients of its looked-up rows, over one micro-batch or two that
            accumulate
  adapt     the output of a shared projection (the head's logits among them) plus each row's own low-rank adapter
  train     the gradients of the rows and of the adapters' two matrices from the gradient of that output

Inputs are synthetic and made from the seed alone. Tokens follow Zipf's law, so a few of them repeat in a large part of
a batch, and a fiftieth of a packed batch is padding (token -1). Decode rows belong to requests whose adapters are mixed,
some with none; the rows of a packed stream come in one run per response. The listed cases stand for the ranges `draw`
samples from.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

B_STD = 0.02           # of a trained adapter's second matrix
TABLE_STD = 0.02       # usual initialiser range of vocabulary weights
LIFT = 9.0             # of the sampled token's logit
ELEMENTS = 1 << 26     # of a block of rows
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the tokens of a decode step, the widest configuration: launch latency
        {"name": "lookup_48", "kind": "lookup", "T": 48, "d": 5120, "V": 152064, "scale": 1.0, "dtype": "bf16",
         "out": "bf16", "pad": False},
        # a packed micro-batch of the trainer, rows scaled by the root of d
        {"name": "lookup_16384", "kind": "lookup", "T": 16384, "d": 4096, "V": 151936, "scale": 64.0, "dtype": "bf16",
         "out": "bf16", "pad": True},
        # two short micro-batches of odd length whose fp32 gradients accumulate, a small model
        {"name": "scatter_301", "kind": "scatter", "T": 301, "d": 1536, "V": 50257, "scale": 1.0, "dtype": "f32",
         "steps": 2, "pad": True},
        # the packed micro-batch's gradient in bf16, the whole matrix written
        {"name": "scatter_16384", "kind": "scatter", "T": 16384, "d": 4096, "V": 151936, "scale": 64.0, "dtype": "bf16",
         "steps": 1, "pad": True},
        # one response in flight with an adapter on the head
        {"name": "adapt_1", "kind": "adapt", "T": 1, "d": 2048, "N": 151936, "n": 4, "r": 16, "dtype": "bf16",
         "out": "f32", "packed": False},
        # a decode step through an ordinary projection, many requests on few adapters of high rank
        {"name": "adapt_200", "kind": "adapt", "T": 200, "d": 4096, "N": 4096, "n": 8, "r": 64, "dtype": "bf16",
         "out": "bf16", "packed": False},
        # a decode step whose requests hardly share adapters, on the widest head
        {"name": "adapt_48", "kind": "adapt", "T": 48, "d": 5120, "N": 152064, "n": 32, "r": 16, "dtype": "bf16",
         "out": "f32", "packed": False},
        # a chunk of a short prompt, an odd vocabulary and an odd rank, fp16
        {"name": "adapt_333", "kind": "adapt", "T": 333, "d": 1536, "N": 50257, "n": 3, "r": 9, "dtype": "f16",
         "out": "f16", "packed": True},
        # the trainer's packed stream under four policies' adapters on the head, logits in fp32
        {"name": "adapt_4096", "kind": "adapt", "T": 4096, "d": 4096, "N": 151936, "n": 4, "r": 16, "dtype": "bf16",
         "out": "f32", "packed": True},
        # gradients of a short batch, an odd vocabulary and an odd rank, fp32 gradients of the logits
        {"name": "train_150", "kind": "train", "T": 150, "d": 1536, "N": 50257, "n": 2, "r": 9, "dtype": "bf16",
         "out": "f32", "packed": True},
        # an ordinary projection's adapters over a long packed stream
        {"name": "train_8192", "kind": "train", "T": 8192, "d": 4096, "N": 4096, "n": 2, "r": 32, "dtype": "bf16",
         "out": "bf16", "packed": True},
        # the head's adapters over the packed stream, gradients of the logits in bf16
        {"name": "train_2047", "kind": "train", "T": 2047, "d": 4096, "N": 151936, "n": 4, "r": 16, "dtype": "bf16",
         "out": "bf16", "packed": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["lookup", "scatter", "adapt", "adapt", "train", "train"])
    vocab = [32000, 50257, 131072, 151936, 152064, _log_int(rng, 1000, 20000)]
    if kind in ("lookup", "scatter"):
        d = rng.choice([256, 1024, 1536, 2048, 3584, 4096, 5120, _log_int(rng, 200, 4096)])
        case = {"kind": kind, "T": _log_int(rng, 1, min(16384, 16384 * 4096 // d)), "d": d,
                "V": min(rng.choice(vocab), 151936 * 4096 // d), "scale": rng.choice([1.0, 1.0, d ** 0.5]),
                "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "pad": rng.random() < 0.5}
        if kind == "lookup":
            case["out"] = rng.choice([case["dtype"], case["dtype"], "f32", "bf16"])
        else:
            case["T"] = min(case["T"], 8192)
            case["steps"] = rng.choice([1, 1, 2])
        return case
    packed = kind == "train" or rng.random() < 0.4
    d = rng.choice([256, 1024, 1536, 2048, 3584, 4096, 5120, _log_int(rng, 200, 4096)])
    N = rng.choice([rng.choice(vocab), _log_int(rng, 512, 16384), d])
    n = _log_int(rng, 1, 8 if packed else 32)
    r = rng.choice([8, 16, 16, 32, 64, _log_int(rng, 1, 64)])
    top = 2047 * 151936 * 64 // (max(N, d) * max(64, n * r))
    return {"kind": kind, "T": _log_int(rng, 1, min(top, 4096 if packed else 256)), "d": d, "N": N, "n": n, "r": r,
            "dtype": rng.choice(["bf16", "bf16", "f16"]), "out": rng.choice(["f32", "bf16", "f16"]), "packed": packed}


# ------------------------------------------------------------------ inputs


def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 32 + k)
    return g


def _normal(n, m, dtype, std, g):
    """[n, m] normal values in dtype, made in blocks of rows."""
    x = torch.empty((n, m), dtype=dtype, device="cuda")
    step = max(1, ELEMENTS // m)
    for r in range(0, n, step):
        x[r:r + step] = (torch.randn((min(step, n - r), m), generator=g, device="cuda") * std).to(dtype)
    return x


def _hidden(n, d, dtype, g):
    """Hidden rows of root mean square one whose elements differ in scale."""
    x = _normal(n, d, torch.float32, 1.0, g) * torch.exp(0.5 * torch.randn(d, generator=g, device="cuda"))
    return (x * torch.rsqrt(x.square().mean(1, keepdim=True))).to(dtype)


def _zipf(n, V, g):
    """n token ids whose ranks follow p(rank) ~ 1 / rank, spread over the vocabulary."""
    rank = torch.exp(torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * math.log(V + 1.0)).long() - 1
    return (rank.clamp_(0, V - 1) * 7919 % V).to(torch.int32)


def _tokens(case, g):
    tok = _zipf(case["T"], case["V"], g)
    if case["pad"]:  # the batch's end
        tok[case["T"] - case["T"] // 50:] = -1
    return tok


def _adapter_rows(case, g):
    """int32 [T]: each row's adapter, -1 for none. A packed stream is four responses per adapter, one after another (one
    per adapter if it is short); of a decode step's requests one in n + 1 has none."""
    T, n = case["T"], case["n"]
    if case["packed"]:
        runs = 4 * n if T >= 4 * n else min(n, T)
        return (torch.arange(T, device="cuda") * runs // T % n).to(torch.int32)
    rows = (torch.arange(T, device="cuda") + 1) % (n + 1) - 1
    return rows[torch.randperm(T, generator=g, device="cuda")].to(torch.int32)


def _logit_gradients(T, N, dtype, g):
    """Gradients of sampled tokens' log-probs with respect to N logits: an advantage times one-hot less probability."""
    out = torch.empty((T, N), dtype=dtype, device="cuda")
    step = max(1, ELEMENTS // N)
    for r in range(0, T, step):
        z = 2.5 * torch.randn((min(step, T - r), N), generator=g, device="cuda")
        tok = torch.randint(0, N, (z.shape[0], 1), generator=g, device="cuda")
        z.scatter_add_(1, tok, torch.full(tok.shape, LIFT, device="cuda"))
        z = torch.exp(z - z.amax(1, keepdim=True))
        z = z / -z.sum(1, keepdim=True)
        z.scatter_add_(1, tok, torch.ones(tok.shape, device="cuda"))
        out[r:r + step] = (z * torch.randn((z.shape[0], 1), generator=g, device="cuda")).to(dtype)
    return out


def prepare(case, seed):
    kind, T, d = case["kind"], case["T"], case["d"]
    dtype = DTYPES[case["dtype"]]
    st = {"kind": kind}
    if kind in ("lookup", "scatter"):
        st["scale"], st["V"] = case["scale"], case["V"]
    if kind == "lookup":
        st["table"] = _normal(case["V"], d, dtype, TABLE_STD, _gen(seed, 0))
        st["tokens"] = _tokens(case, _gen(seed, 1))
        st["out"] = DTYPES[case["out"]]
        return st
    if kind == "scatter":
        st["grads"] = []
        for k in range(case["steps"]):
            size = torch.exp(torch.randn((T, 1), generator=_gen(seed, 4 + k), device="cuda"))
            g = _normal(T, d, torch.float32, 0.01, _gen(seed, 8 + k)) * size
            st["grads"].append((g.to(dtype), _tokens(case, _gen(seed, 12 + k))))
        if own:
            import paper_2605_14220_amd as tim

            st["total"] = torch.empty((case["V"], d), device="cuda")
            st["ws"] = torch.empty(tim.embedding_backward_workspace_size(T, case["V"], d), dtype=torch.uint8,
                                   device="cuda")
        return st
    n, r, N = case["n"], case["r"], case["N"]
    st["x"] = _hidden(T, d, dtype, _gen(seed, 0))
    st["a"] = _normal(n * r, d, dtype, (1.0 / d) ** 0.5, _gen(seed, 1)).view(n, r, d)
    st["b"] = _normal(n * N, r, dtype, B_STD, _gen(seed, 2)).view(n, N, r)
    st["scales"] = 2.0 ** torch.randint(-1, 3, (n,), generator=_gen(seed, 3), device="cuda").float()
    st["rows"] = _adapter_rows(case, _gen(seed, 4))
    out = DTYPES[case["out"]]
    if kind == "adapt":
        st["y"] = _normal(T, N, out, 2.5, _gen(seed, 5))
    else:
        st["g"] = _logit_gradients(T, N, out, _gen(seed, 5))
    if own:
        import paper_2605_14220_amd as tim

        st["adapters"] = tim.Adapters(st["a"], st["b"], st["scales"])
        size = tim.adapters_add_workspace_size if kind == "adapt" else tim.adapters_backward_workspace_size
        st["ws"] = torch.empty(size(T, d, N, n, r), dtype=torch.uint8, device="cuda")
        if kind == "train":
            st["grad_a"] = torch.empty((n, r, d), device="cuda")
            st["grad_b"] = torch.empty((n, N, r), device="cuda")
    return st


# ------------------------------------------------------------------ plain forms


def _plain_lookup(st):
    tok = st["tokens"]
    there = (tok >= 0) & (tok < st["V"])
    e = st["table"][torch.where(there, tok, 0).long()].float() * st["scale"]
    return torch.where(there[:, None], e, 0.0).to(st["out"])


def _plain_scatter(st):
    total = torch.zeros((st["V"], st["grads"][0][0].shape[1]), device="cuda")
    for g, tok in st["grads"]:
        there = (tok >= 0) & (tok < st["V"])
        g = torch.where(there[:, None], g.float() * st["scale"], 0.0)
        total.index_add_(0, torch.where(there, tok, 0).long(), g)
    return total


def _wide(st):
    """All adapters as one of rank n * r: (A fp32 [n * r, d], B fp32 [N, n * r], the scale of each row's own adapter and
    0 for the others' [T, n * r])."""
    n, r, d = st["a"].shape
    mine = st["rows"][:, None] == torch.arange(n, device="cuda")
    s = torch.where(mine, st["scales"], 0.0)[:, :, None].expand(-1, -1, r).reshape(-1, n * r)
    return st["a"].float().view(n * r, d), st["b"].float().transpose(0, 1).reshape(-1, n * r), s


def _plain_adapt(st):
    a, b, s = _wide(st)
    u = (st["x"].float() @ a.T) * s
    return (st["y"].float() + u @ b.T).to(st["y"].dtype)


def _plain_train(st):
    n, r, d = st["a"].shape
    a, b, s = _wide(st)
    x, g = st["x"].float(), st["g"].float()
    u = (x @ a.T) * s
    v = (g @ b) * s
    return {"grad_x": (v @ a).to(st["x"].dtype), "grad_a": (v.T @ x).view(n, r, d),
            "grad_b": (g.T @ u).view(-1, n, r).transpose(0, 1).contiguous()}


# ------------------------------------------------------------------ one pass


def run(st):
    kind = st["kind"]
    if not own:
        return {"lookup": _plain_lookup, "scatter": _plain_scatter, "adapt": _plain_adapt, "train": _plain_train}[kind](st)
    import paper_2605_14220_amd as tim

    if kind == "lookup":
        return tim.embedding(st["table"], st["tokens"], scale=st["scale"], dtype=st["out"])
    if kind == "scatter":
        for k, (g, tok) in enumerate(st["grads"]):
            tim.embedding_backward(g, tok, st["V"], scale=st["scale"], grad_table=st["total"], accumulate=k > 0,
                                   workspace=st["ws"])
        return st["total"]
    if kind == "adapt":
        return tim.adapters_add(st["y"], st["x"], st["rows"], st["adapters"], workspace=st["ws"])
    gx, ga, gb = tim.adapters_backward(st["g"], st["x"], st["rows"], st["adapters"], grad_a=st["grad_a"],
                                       grad_b=st["grad_b"], workspace=st["ws"])
    return {"grad_x": gx, "grad_a": ga, "grad_b": gb}


# ------------------------------------------------------------------ what a pass cannot do without


def _distinct(n, V):
    """Expected number of different tokens among n of _zipf's."""
    k = np.arange(1, V + 1, dtype=np.float64)
    p = np.log((k + 1) / k) / math.log(V + 1.0)
    return float(np.sum(-np.expm1(n * np.log1p(-p))))


def work(case):
    kind, T, d = case["kind"], case["T"], case["d"]
    size = SIZES[case["dtype"]]
    if kind in ("lookup", "scatter"):
        full = T - T // 50 if case["pad"] else T
        if kind == "lookup":
            return {"bytes": int(_distinct(full, case["V"]) * d * size) + T * d * SIZES[case["out"]] + 4 * T,
                    "flops": full * d}
        later = int(_distinct(full, case["V"]) * d * 8) * (case["steps"] - 1)  # rows added to: read and written
        return {"bytes": case["steps"] * (full * d * size + 4 * T) + case["V"] * d * 4 + later,
                "flops": 2 * case["steps"] * full * d}
    n, r, N, out = case["n"], case["r"], case["N"], SIZES[case["out"]]
    rows = T if case["packed"] else T - T // (n + 1)  # with an adapter
    weights = min(n, T) * r * (d + N) * size
    if kind == "adapt":
        return {"bytes": rows * d * size + weights + 2 * T * N * out + 4 * T, "flops": 2 * rows * r * (d + N)}
    return {"bytes": rows * (d * size + N * out) + T * d * size + weights + n * r * (d + N) * 4 + 4 * T,
            "flops": 2 * rows * r * (3 * d + 2 * N)}


# ------------------------------------------------------------------ from the definition, in 64 bits


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "lookup":
        out = torch.zeros((case["T"], case["d"]), dtype=torch.float64, device="cuda")
        rows = [t for t, v in enumerate(st["tokens"].tolist()) if 0 <= v < case["V"]]
        out[rows] = st["table"][st["tokens"][rows].long()].double().mul_(case["scale"])
        return out
    if kind == "scatter":
        total = torch.zeros((case["V"], case["d"]), dtype=torch.float64, device="cuda")
        for g, tok in st["grads"]:
            keep = [t for t, v in enumerate(tok.tolist()) if 0 <= v < case["V"]]
            total.index_put_((tok[keep].long(),), g[keep].double(), accumulate=True)
        return total.mul_(case["scale"])
    owner = st["rows"].tolist()
    groups = {a: [t for t, o in enumerate(owner) if o == a] for a in range(case["n"])}
    if kind == "adapt":
        y = st["y"].double()
        for a, rows in groups.items():
            if rows:
                u = torch.mm(st["x"][rows].double(), st["a"][a].double().t())
                y[rows] += float(st["scales"][a]) * torch.mm(u, st["b"][a].double().t())
        return y
    x, n, r, N = st["x"].double(), case["n"], case["r"], case["N"]
    gx = torch.zeros_like(x)
    ga = torch.zeros((n, r, case["d"]), dtype=torch.float64, device="cuda")
    gb = torch.zeros((n, N, r), dtype=torch.float64, device="cuda")
    for a, rows in groups.items():
        if rows:
            A, B, s, g = st["a"][a].double(), st["b"][a].double(), float(st["scales"][a]), st["g"][rows].double()
            v = torch.mm(g, B) * s
            gx[rows] = torch.mm(v, A)
            ga[a] = torch.mm(v.t().contiguous(), x[rows])
            gb[a] = torch.mm(g.t().contiguous(), torch.mm(x[rows], A.t()) * s)
    return {"grad_x": gx, "grad_a": ga, "grad_b": gb}
