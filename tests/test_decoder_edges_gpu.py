"""GPU tests of the decoder operators at the edges of their contract: launches behind one
another, infinite states, very weak decays, tiny eps, streams and autograd.  References
and bounds are those of decoder_ref.py and test_decoder_gpu.py where nothing else is said."""
import pytest
import torch

import decoder_ref as R
from paper_2606_07317_gb300 import decoder, gbla
from test_decoder_gpu import Case, _close, c32, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
def test_short_sequences_in_a_wide_batch(D):
    """Rows for 2600 tokens (several segments) that hold at most 60: every sequence lies in
    one segment, and the lengths are overwritten right behind the call."""
    lens = [60, 0, 1, 33]
    c = Case(500 + D, 4, 2600, 2, 1, D, "bf16", lens)
    q, k, v, do = c.tok(2), c.tok(1), c.tok(1), c.tok(2)
    ld = torch.tensor([-2.0 ** -9, -2.0 ** -6])
    s0, ds = (c.n(4, 2, D, D, to=torch.float32) for _ in range(2))
    args, sl = [dev(c.poison(x)) for x in (q, k, v)] + [dev(ld)], dev(c.seq_lens)
    o, S = gbla.decay_attention(*args, seq_lens=sl, state=dev(s0), return_state=True)
    sl.fill_(2600)
    sl.copy_(c.seq_lens)
    g = gbla.decay_attention_backward(*args, dev(c.poison(do)), seq_lens=sl, state=dev(s0), dstate=dev(ds),
                                      return_dstate=True)
    sl.fill_(2600)
    cut = [x[:, :60] for x in (q, k, v)]
    ref, Sr, om, Sm = R.decay(*cut, ld, lens, s0, D ** -0.5)
    on = ~c.past()[:, :60]
    _close(o.cpu()[:, :60][on], ref[on], om[on], 2.0 ** -8, "bf16", "o", 2.0 ** -7)
    c.N = 60
    _close(S, Sr, Sm, c32(c), "fp32", "state")
    ref, mag = R.decay_backward(*cut, ld, do[:, :60], lens, s0, ds, D ** -0.5)
    for n in ("dq", "dk", "dv"):
        got = g[n].cpu()
        assert (got[:, 60:] == 0).all(), n
        _close(got[:, :60], ref[n], mag[n], 2.0 ** -8, "bf16", n, 2.0 ** -7)
    _close(g["dstate"], ref["dstate"], mag["dstate"], c32(c), "fp32", "dstate")
    assert gbla.device_error() == 0


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_calls_on_a_given_stream(dtype, D):
    """`stream=side` while the current stream is busy writing to blocks of the results' sizes
    that it has just given back: the results are those of the current stream."""
    c = Case(520, 2, 700, 4, 2, D, dtype)
    q, k, v, do, dko = (dev(c.tok(h)) for h in (4, 2, 2, 4, 2))
    ld = torch.full((4,), -0.05, device="cuda")
    w, rot = torch.ones((4, D), device="cuda"), gbla.rotation_table(700, D)
    s0, ds = (dev(c.n(2, 4, D, D, to=torch.float32)) for _ in range(2))

    def work(**kw):
        state = s0.clone() if not kw else copies.pop()
        out = [*gbla.qk_norm_rotate(q, k, w, w[:2], rot, **kw),
               *gbla.qk_norm_rotate_backward(q, k, w, w[:2], rot, do, dko, **kw).values(),
               *gbla.decay_attention(q, k, v, ld, state=s0, return_state=True, **kw),
               *gbla.decay_attention_backward(q, k, v, ld, do, state=s0, dstate=ds, return_dstate=True, **kw).values(),
               gbla.decay_attention_step(q[:, :1], k[:, :1], v[:, :1], ld, state, **kw)]
        return out + [state]

    want = [t.clone() for t in work()]
    copies = [s0.clone() for _ in range(3)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        held = [torch.empty_like(t) for t in want]
        big = torch.randn((4096, 4096), device="cuda")
        for _ in range(8):
            big = big @ big * 1e-3
        for t in held:
            t.fill_(float("nan"))
        del held, t
        got = work(stream=side)
        side.synchronize()
        torch.cuda.current_stream().synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_steps_after_an_empty_prompt():
    """A sequence that starts with its first step follows the parallel form (2^-7 of the
    layer's own output, as the layer's own test)."""
    layer = decoder.DecoderLayer(128, 2, 64, 16, seed=3)
    x = torch.randn((3, 5, 128), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    y, cache = layer.prompt(x[:, :0].contiguous())
    assert y.shape == (3, 0, 128)
    got = torch.cat([layer.step(x[:, i:i + 1], cache) for i in range(5)], 1).float()
    want = layer.prompt(x)[0].float()
    assert (got - want).norm() <= 2.0 ** -7 * (want - x.float()).norm()


def test_second_derivatives_are_refused():
    """A gradient penalty through the operators is an error; the same loss without it trains."""
    c = Case(530, 2, 40, 2, 1, 64, "fp32")
    leaf = [t.cuda().requires_grad_() for t in (c.tok(2), c.tok(1), c.tok(1))]
    w = torch.ones((2, 64), device="cuda", requires_grad=True)
    ld, rot = torch.full((2,), -0.1, device="cuda"), gbla.rotation_table(40, 64)

    def loss():
        a, b = decoder.norm_rotate(leaf[0], leaf[1], w, w[:1], rot)
        return decoder.attention(a, b, leaf[2], ld)[0].sum()

    want = torch.autograd.grad(loss(), leaf)
    got = torch.autograd.grad(loss(), leaf, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(RuntimeError, match="differentiated once"):
        (loss() + sum(g.square().sum() for g in got)).backward()
    loss().backward()
    assert all(torch.equal(t.grad, b) for t, b in zip(leaf, want))


def test_a_state_stepped_after_it_was_saved():
    """A first state that a training forward keeps for its backward, and single-token steps
    then overwrite, is an error there."""
    c = Case(540, 2, 30, 2, 2, 64, "bf16")
    q, k, v = (dev(c.tok(2)).requires_grad_() for _ in range(3))
    ld, S = torch.full((2,), -0.1, device="cuda"), torch.zeros((2, 2, 64, 64), device="cuda")
    o, _ = decoder.attention(q, k, v, ld, state=S)
    with torch.no_grad():
        gbla.decay_attention_step(q[:, :1], k[:, :1], v[:, :1], ld, S)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()
