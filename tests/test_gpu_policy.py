"""The 4-bit head and the changed logits together, as a rollout engine and a trainer use them: a decode loop whose
log-probs the trainer reproduces from the packed stream, the policy gradient through the changes, captured and
replayed steps, other streams, two calls at once."""

import math

import pytest
import torch

import paper_2605_14220_amd as tim
from tim_testutil import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def _head(V, d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (0.05 * torch.randn(V, d, device="cuda", generator=g)).to(torch.bfloat16)


def _grammar(V, n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    allowed = torch.rand((n, (V + 31) // 32 * 32), device="cuda", generator=g) < 0.7
    bits = (allowed.view(n, -1, 32).long() << torch.arange(32, device="cuda")).sum(2)
    return torch.where(bits >= 2 ** 31, bits - 2 ** 32, bits).to(torch.int32), allowed[:, :V]


def _rollout(W, hidden_of, prompts, steps, penalties, masks, state_of, tau, seed):
    """Decodes `steps` tokens for every prompt with the 4-bit head; returns the streams, the hidden rows and the
    reported log-probs, [requests, steps]."""
    n, V = len(prompts), W.codes.shape[0]
    room = max(len(p) for p in prompts) + steps
    streams = torch.zeros(n, room, dtype=torch.int32, device="cuda")
    for i, p in enumerate(prompts):
        streams[i, :len(p)] = p
    split = torch.tensor([i * room + len(p) for i, p in enumerate(prompts)], device="cuda")
    begin = torch.arange(n, device="cuda") * room
    g = torch.Generator(device="cuda").manual_seed(seed)
    hs, lps, states = [], [], []
    for k in range(steps):
        h = hidden_of(k)
        state = state_of(k)
        rules = tim.LogitRules(history=streams.view(-1), hist_begin=begin, hist_split=split, hist_end=split + k,
                               mask=masks, mask_rows=state, **{f: torch.full((n,), x, device="cuda")
                                                               for f, x in penalties.items()})
        z = tim.mxfp4_logits(tim.mxfp4_quantize(h), W)
        x = tim.logits_adjust(z, rules, tau)
        e = torch.empty_like(x).exponential_(generator=g)
        tok = torch.argmax(torch.softmax(x, 1) / e, 1).to(torch.int32)
        lp, _, _ = tim.logits_logprobs(z, tok, rules, tau)
        assert torch.isfinite(lp).all()
        streams.view(-1)[split + k] = tok
        hs.append(h)
        lps.append(lp)
        states.append(state)
    return streams, torch.stack(hs, 1), torch.stack(lps, 1), torch.stack(states, 1)


def test_trainer_reproduces_the_rollout_and_its_gradient():
    n, steps, V, d, tau = 3, 24, 1003, 256, 0.8
    W16 = _head(V, d, 1)
    W = tim.mxfp4_quantize(W16)
    g = torch.Generator(device="cuda").manual_seed(2)
    hidden = 2.0 * torch.randn(steps, n, d, device="cuda", generator=g).to(torch.bfloat16)
    prompts = [torch.randint(0, V, (k,), dtype=torch.int32, generator=torch.Generator().manual_seed(k)).cuda()
               for k in (5, 1, 9)]
    masks, allowed = _grammar(V, 4, 3)
    state_of = lambda k: torch.tensor([k % 4, -1, (k * 3) % 4], dtype=torch.int32, device="cuda")  # noqa: E731
    pen = {"repetition": 1.2, "frequency": 0.3, "presence": 0.1}
    streams, hs, lp_roll, states = _rollout(W, lambda k: hidden[k], prompts, steps, pen, masks, state_of, tau, 4)

    # the trainer: the packed responses, each row's history the part of its stream before it
    T, room = n * steps, streams.shape[1]
    begin = (torch.arange(n, device="cuda") * room).repeat_interleave(steps)
    split = begin + torch.tensor([len(p) for p in prompts], device="cuda").repeat_interleave(steps)
    end = split + torch.arange(steps, device="cuda").repeat(n)
    rules = tim.LogitRules(history=streams.view(-1), hist_begin=begin, hist_split=split, hist_end=end, mask=masks,
                           mask_rows=states.reshape(-1).contiguous(),
                           **{f: torch.full((T,), x, device="cuda") for f, x in pen.items()})
    tokens = streams.view(-1)[end].contiguous()
    h = hs.reshape(T, d)
    q = tim.mxfp4_quantize(h)
    # the same engine over the whole stream: the same bits as step by step
    lp_same, _, _ = tim.logits_logprobs(tim.mxfp4_logits(q, W), tokens, rules, tau)
    assert torch.equal(lp_same, lp_roll.reshape(-1))
    # the bf16 engine on the values the codes stand for: only the order of the sums differs
    hv, wv = tim.mxfp4_dequantize(q), tim.mxfp4_dequantize(W)
    z = tim.logits(hv, wv)
    lp, H, lse = tim.logits_logprobs(z, tokens, rules, tau, lse=True)
    _, k3, w = tim.mismatch(lp, lp_roll.reshape(-1))
    # each logit moves by at most 2 d 2^-23 sum |h w| < 2 * 256 * 2^-23 * 256 * (6 * 2) * (6 * 2^-5), a log-prob by twice that over tau
    assert (lp - lp_roll.reshape(-1)).abs().max().item() <= 2 / tau * 1.2 * 2 * 256 * 2.0 ** -23 * (
        hv.double().abs() @ wv.double().abs().T).max().item()
    assert (k3 < 1e-3).all() and (w > 0.9).all()
    # without the changes the two score another distribution
    assert (tim.logprobs(hv, wv, tokens, tau)[0] - lp).abs().max().item() > 0.05

    # the policy gradient down to the hidden rows, against autograd in 64 bits
    cu = torch.arange(n + 1, device="cuda") * steps
    adv = torch.randn(n, device="cuda", generator=g).repeat_interleave(steps)
    loss = tim.ppo_loss(lp, lp_roll.reshape(-1), adv, cu, weight=w)
    e = torch.full((T,), -0.01, device="cuda")
    dz = tim.logits_logprobs_backward(z, tokens, lse, loss["grad"], rules, tau, entropy=H, grad_entropy=e)
    dh = dz.double() @ wv.double()

    h64 = hv.double().requires_grad_()
    x = h64 @ wv.double().T
    pos = torch.arange(room * n, device="cuda")
    member = (pos >= begin[:, None]) & (pos < end[:, None])
    out = member & (pos >= split[:, None])
    toks = streams.view(-1).long()[None].expand(T, -1)
    seen = torch.zeros(T, V, device="cuda", dtype=torch.float64).scatter_add_(1, toks, member.double()) > 0
    count = torch.zeros(T, V, device="cuda", dtype=torch.float64).scatter_add_(1, toks, out.double())
    x = torch.where(seen, torch.where(x > 0, x / 1.2, x * 1.2), x)
    x = (x - 0.3 * count - 0.1 * (count > 0)) / tau
    st = states.reshape(-1).long()
    x = x.masked_fill(~allowed[st.clamp(min=0)] & (st >= 0)[:, None], -math.inf)
    logp = torch.log_softmax(x, 1)
    ent = -torch.where(torch.isinf(logp), 0.0, logp.exp() * torch.where(torch.isinf(logp), 0.0, logp)).sum(1)
    (logp.gather(1, tokens.long()[:, None])[:, 0] * loss["grad"].double() + ent * e.double()).sum().backward()
    scale = h64.grad.abs().max().item()
    # fp32 logits of magnitude below 32 carry 2^-19 each way into p; 1e-4 of the largest entry holds it with room
    assert (dh - h64.grad).abs().max().item() <= 1e-4 * scale


def _step_state(T=6, V=9001, d=256):
    g = torch.Generator(device="cuda").manual_seed(7)
    W = tim.mxfp4_quantize(_head(V, d, 8))
    masks, _ = _grammar(V, 3, 9)
    st = {"W": W, "h": torch.randn(T, d, device="cuda", generator=g).to(torch.bfloat16),
          "tok": torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=g),
          "q": tim.Mxfp4(torch.empty(T, d // 2, dtype=torch.uint8, device="cuda"),
                         torch.empty(T, d // 32, dtype=torch.uint8, device="cuda")),
          "z": torch.empty(T, V, device="cuda"), "x": torch.empty(T, V, device="cuda"),
          "ws": torch.empty(tim.logits_logprobs_workspace_size(T, V), dtype=torch.uint8, device="cuda"),
          "out": tuple(torch.empty(T, device="cuda") for _ in range(3)),
          "g": torch.randn(T, device="cuda", generator=g), "dz": torch.empty(T, V, device="cuda")}
    st["rules"] = tim.LogitRules(
        history=torch.randint(0, 50, (T * 40,), device="cuda", dtype=torch.int32, generator=g),
        hist_begin=torch.arange(T, device="cuda") * 40, hist_end=torch.arange(T, device="cuda") * 40 + 20,
        repetition=torch.full((T,), 1.3, device="cuda"), frequency=torch.full((T,), 0.2, device="cuda"),
        presence=torch.full((T,), 0.1, device="cuda"), mask=masks,
        mask_rows=torch.tensor([0, -1, 1, 2, 0, 1], dtype=torch.int32, device="cuda"),
        bias_ids=torch.tensor([3, 5], dtype=torch.int32, device="cuda"), bias_values=torch.tensor([1.0, -2.0]).cuda(),
        bias_begin=torch.zeros(T, dtype=torch.int64, device="cuda"),
        bias_end=torch.full((T,), 2, dtype=torch.int64, device="cuda"))
    return st


def _step(st):
    tim.mxfp4_quantize(st["h"], out=st["q"])
    tim.mxfp4_logits(st["q"], st["W"], 0.9, out=st["z"])
    tim.logits_adjust(st["z"], st["rules"], out=st["x"])
    tim.logits_logprobs(st["z"], st["tok"], st["rules"], workspace=st["ws"], out=st["out"])
    tim.logits_logprobs_backward(st["z"], st["tok"], st["out"][2], st["g"], st["rules"], out=st["dz"])


def _outputs(st):
    return [t.clone() for t in (*st["q"], st["z"], st["x"], *st["out"], st["dz"])]


def test_captured_steps_replay_with_new_inputs():
    """A captured step replayed over changing inputs, with eager work and synchronisations between, gives the eager bits."""
    st, eager = _step_state(), _step_state()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _step(st)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(st)
    for k in range(5):
        for x in (st, eager):
            x["h"].copy_((x["h"].float() * 1.25).to(torch.bfloat16).roll(k, 0))
            x["rules"].hist_end.add_(3)
            x["tok"].copy_((x["tok"] + 17 * k) % 9001)
        _step(eager)
        want = _outputs(eager)
        torch.cuda.synchronize()
        graph.replay()
        got = _outputs(st)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        torch.cuda.synchronize()


def test_two_streams_at_once():
    """Two steps with workspaces of their own on two streams: neither sees the other."""
    sts = [_step_state(), _step_state()]
    sts[1]["h"].mul_(-2.0)
    want = []
    for st in sts:
        _step(st)
        want.append(_outputs(st))
    for st in sts:
        for t in (st["z"], st["x"], st["dz"], *st["out"]):
            t.fill_(float("nan"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for st, s in zip(sts, streams):
            with torch.cuda.stream(s):
                _step(st)
    torch.cuda.synchronize()
    for st, w in zip(sts, want):
        assert all(torch.equal(a, b) for a, b in zip(_outputs(st), w))


def test_gradient_through_autograd():
    """The calls inside a torch autograd function, next to a captured backward of the same operators."""
    st = _step_state()
    _step(st)

    class Score(torch.autograd.Function):
        @staticmethod
        def forward(ctx, z):
            lp, H, lse = tim.logits_logprobs(z, st["tok"], st["rules"], lse=True)
            ctx.save_for_backward(z, H, lse)
            return lp, H

        @staticmethod
        def backward(ctx, g, e):
            z, H, lse = ctx.saved_tensors
            return tim.logits_logprobs_backward(z, st["tok"], lse, g.contiguous(), st["rules"], entropy=H,
                                                grad_entropy=e.contiguous())

    z = st["z"].clone().requires_grad_()
    lp, H = Score.apply(z)
    ok = torch.isfinite(lp)
    (torch.where(ok, lp, 0.0) * st["g"]).sum().backward()
    want = tim.logits_logprobs_backward(st["z"], st["tok"], st["out"][2], torch.where(ok, st["g"], 0.0), st["rules"],
                                        entropy=st["out"][1], grad_entropy=torch.zeros_like(st["g"]))
    assert torch.equal(z.grad, want)
