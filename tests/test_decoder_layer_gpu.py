"""The decoder layer (projection, norm and rotation, decayed attention, single-token
steps) runs its operators together: steps continue prompts, ragged prompts equal
their sequences alone, and a training step's gradients are those of the formulas."""
import pytest
import torch

import decoder_ref as R
from paper_2606_07317_gb300 import decoder, gbla

pytestmark = pytest.mark.gpu


def test_steps_continue_the_parallel_form():
    """bf16 storage between the operators: both forms round q, k, v, o and y to 2^-9 at the
    same places, and o from tensor cores once more; 2^-7 of the layer's own output."""
    assert decoder.main(B=3, N=200, new=9) <= 2.0 ** -7


def test_ragged_prompts_and_their_steps():
    layer = decoder.DecoderLayer(128, 2, 64, 400, seed=3)
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
    assert cache["positions"].flatten().tolist() == [L + 2 for L in lens]


def test_training_step_gradients():
    """The two operators as torch functions, chained, against the 64-bit formulas chained
    (fp32: each stage adds its rounding, (D + 100) 2^-22 of the magnitudes' norm)."""
    B, N, H, Hk, D = 2, 60, 4, 2, 64
    g = torch.Generator().manual_seed(6)
    n = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    q, k, v, wq, wk = n(B, N, H, D), n(B, N, Hk, D), n(B, N, Hk, D), 1 + 0.1 * n(H, D), 1 + 0.1 * n(Hk, D)
    s0, do, ds = n(B, H, D, D), n(B, N, H, D), n(B, H, D, D)
    lens = [60, 23]
    ld = decoder.head_decays(H, 4, 64, device="cpu")
    rot = gbla.rotation_table(N, D, device="cpu")
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    leaf = {m: t.cuda().requires_grad_() for m, t in dict(q=q, k=k, v=v, wq=wq, wk=wk, s0=s0).items()}
    a, b = decoder.norm_rotate(leaf["q"], leaf["k"], leaf["wq"], leaf["wk"], rot.cuda(), None, sl)
    o, S = decoder.attention(a, b, leaf["v"], ld.cuda(), sl, leaf["s0"])
    ((o * do.cuda()).sum() + (S * ds.cuda()).sum()).backward()
    # the formulas, on the operator's own normed q and k
    ref, mag = R.decay_backward(a.detach().cpu(), b.detach().cpu(), v, ld, do, lens, s0, ds, D ** -0.5)
    bound = lambda m: (D + 100) * 2.0 ** -22 * m.norm()  # noqa: E731
    near = lambda got, want, m, what: (got.cpu().double() - want).norm() <= bound(m) or pytest.fail(what)  # noqa: E731
    near(leaf["v"].grad, ref["dv"], mag["dv"], "v")
    near(leaf["s0"].grad, ref["dstate"], mag["dstate"], "s0")
    for m, x, w, t in (("q", q, wq, "dq"), ("k", k, wk, "dk")):
        dx, dxm, dw, dwm = R.norm_rotate_backward(x, w, rot, None, D, False, 1e-6, ref[t], lens)
        _, big, _, bigw = R.norm_rotate_backward(x, w, rot, None, D, False, 1e-6, mag[t], lens)
        near(leaf[m].grad, dx, big, m)
        near(leaf["w" + m].grad, dw, bigw, "w" + m)
