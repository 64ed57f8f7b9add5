"""Pins of the 64-bit decoder references (CPU): the recurrence against the
explicit sum over pairs of tokens, its gradients and those of the norm and
rotation against central differences, and the rotation's invariants."""
import itertools

import pytest
import torch

import decoder_ref as R

F64 = torch.float64


def _case(seed, B=2, N=7, H=4, Hk=2, D=32):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, dtype=F64)  # noqa: E731
    return dict(q=n(B, N, H, D), k=n(B, N, Hk, D), v=n(B, N, Hk, D),
                log_decay=-torch.rand(H, generator=g, dtype=F64), state=n(B, H, D, D)), n


def test_recurrence_equals_the_sum_over_pairs():
    c, _ = _case(0)
    lens, scale = [7, 4], -0.3
    o, S, om, Sm = R.decay(c["q"], c["k"], c["v"], c["log_decay"], lens, c["state"], scale)
    for b, h in itertools.product(range(2), range(4)):
        gam, q, k, v = c["log_decay"][h].exp(), c["q"][b, :, h], c["k"][b, :, h // 2], c["v"][b, :, h // 2]
        L = lens[b]
        t = torch.arange(L, dtype=F64)
        w = torch.where(t[:, None] >= t, gam ** (t[:, None] - t), torch.zeros((), dtype=F64))
        ref = scale * ((q[:L] @ k[:L].T * w) @ v[:L] + gam ** (t + 1)[:, None] * (q[:L] @ c["state"][b, h]))
        assert torch.allclose(o[b, :L, h], ref, atol=1e-11)
        assert (o[b, L:, h] == 0).all()
        fin = (k[:L] * (gam ** (L - 1 - t))[:, None]).T @ v[:L] + gam ** L * c["state"][b, h]
        assert torch.allclose(S[b, h], fin, atol=1e-11)
    assert (om >= o.abs() - 1e-12).all() and (Sm >= S.abs() - 1e-12).all()


def test_decay_gradients_against_differences():
    c, n = _case(1, N=4)
    lens, scale = [4, 2], 0.7
    do, ds = n(2, 4, 4, 32), n(2, 4, 32, 32)
    g, m = R.decay_backward(c["q"], c["k"], c["v"], c["log_decay"], do, lens, c["state"], ds, scale)

    def loss(x):
        o, S, _, _ = R.decay(x["q"], x["k"], x["v"], x["log_decay"], lens, x["state"], scale)
        return (o * do).sum() + (S * ds).sum()

    gen = torch.Generator().manual_seed(2)
    for name, key in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("state", "dstate")):
        for _ in range(6):  # random directions
            e = torch.randn(c[name].shape, generator=gen, dtype=F64)
            hi, lo = ({**c, name: c[name] + s * 1e-5 * e} for s in (1, -1))
            d = (loss(hi) - loss(lo)) / 2e-5
            assert abs(d - (g[key] * e).sum()) <= 1e-6 * (m[key] * e.abs()).sum(), name


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot_dims", [0, 16, 32])
def test_norm_rotate_gradients_against_differences(interleaved, rot_dims):
    g = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(s, generator=g, dtype=F64)  # noqa: E731
    x, w, dy = n(2, 5, 3, 32), n(3, 32), n(2, 5, 3, 32)
    a = n(9, rot_dims // 2)
    rot = torch.cat([a.cos(), a.sin()], 1)
    pos = torch.randint(0, 9, (2, 5), generator=g)
    lens, eps = [5, 3], 1e-2
    live = (torch.arange(5)[None] < torch.tensor(lens)[:, None])[:, :, None, None]
    dx, dxm, dw, dwm = R.norm_rotate_backward(x, w, rot, pos, rot_dims, interleaved, eps, dy, lens)

    def loss(x, w):
        y, _ = R.norm_rotate(x, w, rot, pos, rot_dims, interleaved, eps)
        return (y * dy * live).sum()

    for _ in range(6):
        e, f = n(*x.shape), n(*w.shape)
        d = (loss(x + 1e-5 * e, w) - loss(x - 1e-5 * e, w)) / 2e-5
        assert abs(d - (dx * e).sum()) <= 1e-6 * (dxm * e.abs()).sum()
        d = (loss(x, w + 1e-5 * f) - loss(x, w - 1e-5 * f)) / 2e-5
        assert abs(d - (dw * f).sum()) <= 1e-6 * (dwm * f.abs()).sum()


def test_rotation_keeps_lengths_and_relative_angles():
    g = torch.Generator().manual_seed(4)
    x, y = torch.randn((2, 1, 1, 1, 32), generator=g, dtype=F64)
    w = torch.ones((1, 32), dtype=F64)
    from paper_2606_07317_gb300.gbla import rotation_table
    rot = rotation_table(64, 32, device="cpu")
    assert rot.shape == (64, 32) and (rot[0, :16] == 1).all() and (rot[0, 16:] == 0).all()
    at = lambda v, p: R.norm_rotate(v, w, rot, torch.tensor([[p]]), 32, False, 1e-9)[0].flatten()  # noqa: E731
    assert torch.allclose(at(x, 0).norm(), at(x, 50).norm(), rtol=1e-6)
    assert torch.allclose(at(x, 10) @ at(y, 3), at(x, 47) @ at(y, 40), rtol=1e-5, atol=1e-5)
