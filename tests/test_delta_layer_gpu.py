"""The decoder with the gated delta rule and the answer head, as they are used together: steps
continue prompts, ragged prompts equal their sequences alone, candidates and scores agree, and a
training step's gradients are those of the formulas chained."""
import math

import pytest
import torch

import delta_ref as R
from paper_2606_07317_gb300 import decoder, gbla

pytestmark = pytest.mark.gpu


def test_steps_continue_the_parallel_form():
    """bf16 storage between the operators: both forms round q, k, v, the gates, o and y at the same
    places; 2^-7 of the layer's own output, as for the decayed mixer."""
    assert decoder.main(B=3, N=200, new=9, mixer="delta") <= 2.0 ** -7


def test_ragged_prompts_and_their_steps():
    layer = decoder.DecoderLayer(128, 2, 64, 400, seed=3, mixer="delta")
    g = torch.Generator().manual_seed(4)
    lens = [130, 2, 0, 77]
    x = torch.randn((4, 130, 128), generator=g).to(torch.bfloat16).cuda()
    nxt = torch.randn((4, 2, 128), generator=g).to(torch.bfloat16).cuda()
    y, cache = layer.prompt(x, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    steps = [layer.step(nxt[:, i:i + 1], cache) for i in range(2)]
    for b, L in enumerate(lens):
        alone = torch.cat([x[b:b + 1, :L], nxt[b:b + 1]], 1).contiguous()
        want, _ = layer.prompt(alone)
        got = torch.cat([y[b:b + 1, :L]] + [s[b:b + 1] for s in steps], 1)
        scale = (want.float() - alone.float()).norm()
        assert (got.float() - want.float()).norm() <= 2.0 ** -7 * scale, b


def test_candidates_and_scores_agree():
    """A beam's step: the candidates' log probabilities are what scoring them gives, bit for bit
    (both are scale (x - max) - ln z of the same logits), and ruled-out items are none of them."""
    head = decoder.AnswerHead(128, 777, seed=1)
    y = torch.randn((4, 3, 128), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    best = head.candidates(y, 8)
    assert (best["top_logprob"][..., :-1] >= best["top_logprob"][..., 1:]).all()
    for i in range(8):
        got = head.score(y, best["top_token"][..., i].contiguous())
        assert torch.equal(got["logprob"], best["top_logprob"][..., i])
    out = torch.ones(777, dtype=torch.bool, device="cuda")
    out[[5, 99, 700]] = False
    few = head.candidates(y, 3, ruled_out=out)
    assert all(set(t) == {5, 99, 700} for t in few["top_token"].flatten(0, 1).tolist())
    assert torch.allclose(few["top_logprob"].exp().sum(-1), torch.ones((4, 3), device="cuda"), atol=1e-5)


def test_training_step_gradients():
    """Norm, delta rule and scores as torch functions, chained in fp32: the scores' gradient of
    the logits is the formula's, the delta rule's gradients are the recurrence's for the gradient
    that comes in (bounds of test_delta_gpu.py), and the norm's follow."""
    B, N, H, Hk, D, V = 2, 90, 4, 2, 64, 50
    g = torch.Generator().manual_seed(6)
    n = lambda *s: torch.randn(s, generator=g).cuda()  # noqa: E731
    lens = [90, 31]
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    leaf = dict(q=n(B, N, Hk, D), k=n(B, N, Hk, D), v=n(B, N, H, D), g=-n(B, N, H).abs(), b=n(B, N, H).sigmoid(),
                s0=n(B, H, D, D), w=n(V, H * D) * (H * D) ** -0.5)
    leaf = {m: t.requires_grad_() for m, t in leaf.items()}
    unit = torch.full((Hk, D), D ** -0.5, device="cuda")
    tok = torch.randint(-1, V, (B, N), generator=g).to(torch.int32).cuda()
    a, k = decoder.norm_rotate(leaf["q"], leaf["k"], unit, unit, None, None, sl)
    a.retain_grad(), k.retain_grad()
    o = decoder.delta_attention(a, k, leaf["v"], leaf["g"], leaf["b"], sl, leaf["s0"])
    logits = o.flatten(2) @ leaf["w"].t()
    o.retain_grad(), logits.retain_grad()
    got = decoder.token_logprobs(logits, tok, seq_lens=sl)
    (got["logprob"].sum() - 0.1 * got["entropy"].sum() + 0.01 * got["lse"].square().sum()).backward()
    past = (torch.arange(N)[None] >= torch.tensor(lens)[:, None]).cuda()
    live = (~past).double()
    ref = R.logprobs(logits.detach(), tok, 0, 1.0)
    want, mag = R.logprobs_backward(logits.detach(), tok, 1.0, live, -0.1 * live, 0.02 * ref["lse"] * live)
    assert (logits.grad[past] == 0).all()
    # test_logprob_gpu.py's bound: 96 u and 4 u of lse and logit, here below 32 in all; 2 ulp of dlse
    assert ((logits.grad.double() - want).abs() <= (96 + 4 * 32 + 4) * 2.0 ** -24 * mag + 2.0 ** -117).all()
    d = R.delta_backward(a.detach(), k.detach(), leaf["v"].detach(), leaf["g"].detach(), leaf["b"].detach(),
                         o.grad, lens, leaf["s0"].detach(), None, D ** -0.5)
    f = 2 * (4 * math.sqrt(N) + 2 * math.sqrt(D + 64) + 16) * 2.0 ** -24
    for name, t in (("dq", a), ("dk", k), ("dv", leaf["v"]), ("dbeta", leaf["b"]), ("dstate", leaf["s0"])):
        assert (t.grad.double() - d[name]).norm() <= f * d[name].norm(), name
    lengths = o.grad.double().norm(dim=-1) * o.detach().double().norm(dim=-1)
    lengths = lengths + d["dv"].norm(dim=-1) * leaf["v"].detach().double().norm(dim=-1)
    beside = torch.where(past[..., None], 0.0, lengths).norm()
    assert (leaf["g"].grad.double() - d["dlog_decay"]).norm() <= 8 * f * (d["dlog_decay"].norm() + beside)
    for m in ("q", "k"):
        assert (leaf[m].grad[past] == 0).all() and torch.isfinite(leaf[m].grad).all()


def test_gradients_against_differences():
    """The delta rule's gradients through the library alone: central differences of its own
    forward pass in fp32, along random directions.  With steps of 2^-6 the difference's own error
    is about 2^-12 of the third derivatives' size and the roundings' 2^-24 |loss| / 2^-6: 2^-8 of
    |gradient| |direction| holds both by far."""
    B, N, H, D = 1, 70, 2, 32
    g = torch.Generator().manual_seed(7)
    n = lambda *s: torch.randn(s, generator=g).cuda()  # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    x = dict(q=unit(n(B, N, H, D)), k=unit(n(B, N, H, D)) * 0.9, v=n(B, N, H, D), log_decay=-n(B, N, H).abs() - 0.1,
             beta=0.1 + 0.8 * n(B, N, H).sigmoid(), state=n(B, H, D, D))
    do, ds = n(B, N, H, D), n(B, H, D, D)
    args = ("q", "k", "v", "log_decay", "beta")

    def loss(x):
        o, S = gbla.delta_attention(*[x[a] for a in args], state=x["state"], return_state=True)
        return ((o.double() * do).sum() + (S.double() * ds).sum()).item()

    grads = gbla.delta_attention_backward(*[x[a] for a in args], do, state=x["state"], dstate=ds, return_dstate=True)
    for name, t in x.items():
        for _ in range(3):
            e = n(*t.shape)
            e = e / e.norm()
            h = 2.0 ** -6
            d = (loss({**x, name: t + h * e}) - loss({**x, name: t - h * e})) / (2 * h)
            got = (grads["d" + name].double() * e).sum().item()
            assert abs(d - got) <= 2.0 ** -8 * grads["d" + name].norm().item(), (name, d, got)


def test_gradients_that_come_as_slices():
    """Results of several batches in one flat tensor, each at an odd place of it: the gradients are
    those of the batches alone, bit for bit."""
    g = torch.Generator().manual_seed(8)
    n = lambda *s: torch.randn(s, generator=g).cuda()  # noqa: E731
    tok = torch.randint(0, 40, (2, 3), generator=g).to(torch.int32).cuda()
    weight = n(500)
    for apart in (True, False):
        g.manual_seed(9)
        logits = [n(2, 3, 40).requires_grad_() for _ in range(3)]
        results = [decoder.token_logprobs(x, tok) for x in logits]
        q, k, v = n(1, 5, 2, 32), n(1, 5, 2, 32) * 32 ** -0.5, n(1, 5, 2, 32).requires_grad_()
        o = decoder.delta_attention(q, k, v, -n(1, 5, 2).abs(), n(1, 5, 2).sigmoid())
        parts = [weight[:1]] + [r[m].flatten() for r in results for m in ("lse", "entropy", "logprob")] + [o.flatten()]
        if apart:
            split = torch.split(weight[:375], [p.numel() for p in parts])
            want = torch.autograd.grad(parts[1:], logits + [v], [w.clone() for w in split[1:]])
        else:
            (torch.cat(parts) * weight[:375]).sum().backward()
            got = [x.grad for x in logits] + [v.grad]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
