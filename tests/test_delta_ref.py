"""Pins of the 64-bit references of the gated delta rule and the token log probabilities (CPU):
closed forms, and gradients against central differences."""
import math

import pytest
import torch

import delta_ref as R

F64 = torch.float64


def _case(seed, B=2, N=6, H=4, Hk=2, D=8):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, dtype=F64)  # noqa: E731
    c = dict(q=n(B, N, Hk, D), k=n(B, N, Hk, D) / D ** 0.5, v=n(B, N, H, D), log_decay=-n(B, N, H).abs(),
             beta=n(B, N, H).sigmoid(), state=n(B, H, D, D))
    return c, n


def test_a_stored_value_is_read_back_and_replaced():
    """With unit keys, beta 1 and no decay the last value written under a key is what a query of
    that key reads; orthogonal keys do not touch it."""
    D = 8
    e = torch.eye(D, dtype=F64)
    k = torch.stack([e[0], e[1], e[0], e[2]])[None, :, None]
    g = torch.Generator().manual_seed(0)
    v = torch.randn((1, 4, 1, D), generator=g, dtype=F64)
    zero, one = torch.zeros((1, 4, 1), dtype=F64), torch.ones((1, 4, 1), dtype=F64)
    o, S = R.delta(k, k, v, zero, one, [4], None, 1.0)
    assert torch.allclose(o, v, atol=1e-12)  # each reads its own key after the write
    assert torch.allclose(S[0, 0, 0], v[0, 2, 0]) and torch.allclose(S[0, 0, 1], v[0, 1, 0])
    half, _ = R.delta(k, k, v, zero, one / 2, [4], None, 1.0)
    assert torch.allclose(half[0, 2, 0], (v[0, 2, 0] + v[0, 0, 0] / 2) / 2)


def test_without_overlap_it_is_the_decayed_sum():
    """Orthonormal keys never meet: the state is the decayed sum of the rank-one terms."""
    D = N = 8
    c, n = _case(1, B=1, N=N, H=2, Hk=1, D=D)
    k = torch.linalg.qr(n(D, D))[0][None, :, None]
    _, S = R.delta(c["q"], k, c["v"], c["log_decay"], c["beta"], [N], None, 1.0)
    G = c["log_decay"].cumsum(1)
    w = (G[:, -1:] - G).exp() * c["beta"]
    ref = torch.einsum("nd,bnh,bnhe->bhde", k[0, :, 0], w, c["v"])
    assert torch.allclose(S, ref, atol=1e-12)


def test_minus_infinity_ends_the_memory():
    c, _ = _case(2)
    c["log_decay"][:, 3] = -math.inf
    args = ("q", "k", "v", "log_decay", "beta")
    o, S = R.delta(*[c[a] for a in args], [6, 6], c["state"], 0.5)
    cut = {n: c[n][:, 3:] for n in args}
    o2, S2 = R.delta(*cut.values(), [3, 3], None, 0.5)
    assert torch.allclose(o[:, 3:], o2) and torch.allclose(S, S2)


def test_delta_gradients_against_differences():
    c, n = _case(3)
    lens, scale = [6, 4], -0.7
    do, ds = n(2, 6, 4, 8), n(2, 4, 8, 8)
    args = ("q", "k", "v", "log_decay", "beta")
    g = R.delta_backward(*[c[a] for a in args], do, lens, c["state"], ds, scale)

    def loss(x):
        o, S = R.delta(*[x[a] for a in args], lens, x["state"], scale)
        return (o * do).sum() + (S * ds).sum()

    for name in (*args, "state"):
        for _ in range(5):
            e = n(*c[name].shape)
            hi, lo = ({**c, name: c[name] + s * 1e-5 * e} for s in (1, -1))
            d = (loss(hi) - loss(lo)) / 2e-5
            assert abs(d - (g["d" + name] * e).sum()) <= 1e-7 * max(1.0, g["d" + name].norm() * e.norm()), name


@pytest.mark.parametrize("scale", [1.0, 0.3])
def test_logprobs_against_torch(scale):
    g = torch.Generator().manual_seed(4)
    x = torch.randn((2, 5, 37), generator=g, dtype=F64) * 3
    tok = torch.randint(-1, 38, (2, 5), generator=g)
    r = R.logprobs(x, tok, 4, scale)
    lp = torch.log_softmax(x * scale, -1)
    assert torch.allclose(r["lse"], torch.logsumexp(x * scale, -1))
    assert torch.allclose(r["entropy"], torch.distributions.Categorical(logits=x * scale).entropy())
    has = (tok >= 0) & (tok < 37)
    assert torch.allclose(r["logprob"][has], lp.gather(-1, tok.clamp(0, 36)[..., None])[..., 0][has])
    assert (r["logprob"][~has] == 0).all()
    assert torch.equal(r["top_token"].long(), lp.topk(4).indices) and torch.allclose(r["top_logprob"], lp.topk(4).values)


def test_logprob_gradients_against_autograd():
    g = torch.Generator().manual_seed(5)
    x = (torch.randn((2, 5, 37), generator=g, dtype=F64) * 2).requires_grad_()
    tok = torch.randint(-1, 37, (2, 5), generator=g)
    a, h, l = torch.randn((3, 2, 5), generator=g, dtype=F64)
    lp = torch.log_softmax(x * 0.6, -1)
    picked = torch.where(tok >= 0, lp.gather(-1, tok.clamp(min=0)[..., None])[..., 0], 0.0)
    loss = (a * picked).sum() + (h * -(lp.exp() * lp).sum(-1)).sum() + (l * torch.logsumexp(x * 0.6, -1)).sum()
    loss.backward()
    d, mag = R.logprobs_backward(x.detach(), tok, 0.6, a, h, l)
    assert torch.allclose(d, x.grad, atol=1e-12) and (mag >= d.abs() - 1e-12).all()


def test_empty_rows_and_ruled_out_tokens():
    x = torch.full((1, 3, 4), -math.inf, dtype=F64)
    x[0, 1, 2] = 5.0
    x[0, 2] = torch.tensor([1.0, -math.inf, 1.0, -math.inf])
    r = R.logprobs(x, torch.tensor([[0, 2, 1]]), 4, 1.0)
    assert r["lse"][0, 0] == -math.inf and r["logprob"][0].tolist() == [-math.inf, 0.0, -math.inf]
    assert r["entropy"][0].tolist()[:2] == [0.0, 0.0] and abs(r["entropy"][0, 2] - math.log(2)) < 1e-12
    assert r["top_token"][0].tolist() == [[0, 1, 2, 3], [2, 0, 1, 3], [0, 2, 1, 3]]
    d, _ = R.logprobs_backward(x, torch.tensor([[0, 2, 1]]), 1.0, *torch.ones((3, 1, 3), dtype=F64))
    assert torch.isfinite(d).all() and (d[0, 0] == 0).all()
