"""GPU tests of the decoder operators at the edges of their contract: launches behind one
another, infinite states, very weak decays, tiny eps, streams and autograd.  References
and bounds are those of decoder_ref.py and test_decoder_gpu.py where nothing else is said."""
import pytest
import torch

import decoder_ref as R
from paper_2606_07317_gb300 import decoder, gbla
from test_decoder_gpu import DEC, Case, _close, _decay_case, c32, dev

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


# ------------------------------------------------------------- infinite states
# D, dtype, N, lens: whole chunks, a chunk cut short, several segments
INF = [(32, "fp32", 70, None), (64, "fp32", 700, [700, 300]), (128, "fp32", 96, None), (32, "bf16", 129, None),
       (64, "bf16", 70, [70, 64]), (64, "bf16", 2500, [2500, 700]), (128, "bf16", 193, None),
       (128, "bf16", 2000, None), (64, "bf16", 10, [10, 0])]
INF_DECAYS = [-3.0, -0.05, -1e-3, 2e-4]  # the first fades to 0 in fp32 within a chunk


def _with_infinities(s):
    """s with an infinity of each sign in places that share no row and no column."""
    s = s.clone()
    s[:, :, 3, 5], s[:, :, 7, 11] = float("inf"), float("-inf")
    return s


@pytest.mark.parametrize("family", ["auto", "simt"])
@pytest.mark.parametrize("i", range(len(INF)))
def test_infinite_states_stay_infinite(i, family):
    """gamma S + k v^T of an infinite S is that infinity for every gamma > 0: its column of
    the results is infinite with the sign of the query's value, everything else as without."""
    D, dtype, N, lens = INF[i]
    c = Case(550 + i, 2, N, 4, 2, D, dtype, lens)
    q, k, v, do = (dev(c.tok(h)) for h in (4, 2, 2, 4))
    ld, algo = torch.tensor(INF_DECAYS, device="cuda"), {"auto": gbla.ALGO_AUTO, "simt": gbla.ALGO_SIMT}[family]
    s0, ds = (dev(c.n(2, 4, D, D, to=torch.float32)) for _ in range(2))
    kw = dict(seq_lens=dev(c.seq_lens), algo=algo)
    on = ~c.past().cuda()
    bad = torch.isinf(_with_infinities(s0))
    inf = float("inf")

    def check(got, plain, axis_of, name):
        """Rows or columns 5 and 11 (3 and 7) infinite by the other tensor's sign, the rest equal."""
        for at, sign in axis_of:
            assert torch.equal(got[..., at].float(), torch.sign(sign) * inf), (name, at)
        rest = [e for e in range(D) if e not in [at for at, _ in axis_of]]
        assert torch.equal(got[..., rest], plain[..., rest]), name

    zero = s0.masked_fill(bad, 0.0)
    o, S = gbla.decay_attention(q, k, v, ld, state=_with_infinities(s0), return_state=True, **kw)
    o2, S2 = gbla.decay_attention(q, k, v, ld, state=zero, return_state=True, **kw)
    check(o[on], o2[on], [(5, q[on][..., 3].float()), (11, -q[on][..., 7].float())], "o")
    assert torch.equal(S[bad], _with_infinities(s0)[bad]) and torch.equal(S[~bad], S2[~bad])
    g = gbla.decay_attention_backward(q, k, v, ld, do, state=_with_infinities(s0), **kw)
    g2 = gbla.decay_attention_backward(q, k, v, ld, do, state=zero, **kw)
    check(g["dq"][on], g2["dq"][on], [(3, do[on][..., 5].float()), (7, -do[on][..., 11].float())], "dq")
    assert torch.equal(g["dk"], g2["dk"]) and torch.equal(g["dv"], g2["dv"])
    # the gradient of the final state, with a head of keys for each of queries
    k, v = (dev(c.tok(4)) for _ in range(2))
    zero = ds.masked_fill(bad, 0.0)
    g = gbla.decay_attention_backward(q, k, v, ld, do, dstate=_with_infinities(ds), return_dstate=True, **kw)
    g2 = gbla.decay_attention_backward(q, k, v, ld, do, dstate=zero, return_dstate=True, **kw)
    check(g["dk"][on], g2["dk"][on], [(3, v[on][..., 5].float()), (7, -v[on][..., 11].float())], "dk")
    check(g["dv"][on], g2["dv"][on], [(5, k[on][..., 3].float()), (11, -k[on][..., 7].float())], "dv")
    assert torch.equal(g["dstate"][bad], _with_infinities(ds)[bad]) and torch.equal(g["dstate"][~bad], g2["dstate"][~bad])


@pytest.mark.parametrize("D,dtype", [(32, "fp32"), (64, "bf16"), (128, "bf16")])
def test_steps_on_infinite_states(D, dtype):
    c = Case(570, 2, 1, 4, 4, D, dtype)
    q, k, v = (dev(c.tok(4)) for _ in range(3))
    ld, s0 = torch.tensor(INF_DECAYS, device="cuda"), dev(c.n(2, 4, D, D, to=torch.float32))
    S, plain = _with_infinities(s0), s0.clone()
    bad = torch.isinf(S)
    o, o2 = (gbla.decay_attention_step(q, k, v, ld, s) for s in (S, plain))
    assert torch.equal(S[bad], _with_infinities(s0)[bad]) and torch.equal(S[~bad], plain[~bad])
    for at, sign in ((5, q[..., 3]), (11, -q[..., 7])):
        assert torch.equal(o[..., at].float(), torch.sign(sign.float()) * float("inf"))
    rest = [e for e in range(D) if e not in (5, 11)]
    assert torch.equal(o[..., rest], o2[..., rest])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_growing_state_overflows_to_infinity(dtype):
    """A state that grows past the largest float is infinite, not NaN (keys of zero)."""
    z = torch.zeros((1, 64, 2, 64), dtype=torch.float32 if dtype == "fp32" else torch.bfloat16, device="cuda")
    S = torch.full((1, 2, 64, 64), 2.0 ** 120, device="cuda")
    S[0, 1] = -S[0, 1]
    ld = torch.full((2,), 0.25, device="cuda")  # e^16 a call
    for _ in range(3):
        S = gbla.decay_attention(z, z, z, ld, state=S, return_state=True)[1]
    assert (S[0, 0] == float("inf")).all() and (S[0, 1] == float("-inf")).all()
    for _ in range(2):
        gbla.decay_attention_step(z[:, :1], z[:, :1], z[:, :1], ld, S)
    assert (S[0, 0] == float("inf")).all() and (S[0, 1] == float("-inf")).all()


@pytest.mark.parametrize("D,dtype,family", [(32, "fp32", "auto"), (128, "fp32", "auto"), (64, "bf16", "simt"),
                                            (64, "bf16", "auto"), (128, "bf16", "auto")])
def test_states_through_many_segments_do_not_drift(D, dtype, family):
    """A state (and the gradient of one) through 32768 tokens of zero keys at decays far
    weaker than a segment: at most 128 segments and 64 chunks each round once, at random,
    by up to 2^-24: 2 sqrt(192) 2^-24 of the norm.  A segment's factor rounded to one float
    is off by up to 2^-25 to the same side each time (128 of them: 3.8e-6 at these decays)."""
    N, H = 32768, 3
    algo = {"auto": gbla.ALGO_AUTO, "simt": gbla.ALGO_SIMT}[family]
    ld = torch.tensor([-9.536743e-07, -2.1909682e-06, -1.3283548e-05])
    z = torch.zeros((1, N, H, D), dtype=torch.float32 if dtype == "fp32" else torch.bfloat16, device="cuda")
    s0 = torch.randn((1, H, D, D), generator=torch.Generator().manual_seed(5))
    S = gbla.decay_attention(z, z, z, dev(ld), state=dev(s0), return_state=True, algo=algo)[1]
    g = gbla.decay_attention_backward(z, z, z, dev(ld), z, dstate=dev(s0), return_dstate=True, algo=algo)["dstate"]
    want = s0.double() * (N * ld.double()).exp()[None, :, None, None]
    off = [((t[0, h].cpu().double() - want[0, h]).norm() / want[0, h].norm()).item() for t in (S, g) for h in range(H)]
    assert max(off) <= 2 * 192 ** 0.5 * 2.0 ** -24, off


# ------------------------------------------------------------- norm and rotation

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1.17e-38, 1.2e-38, 1e-30])
def test_zero_heads_at_the_smallest_eps(eps, dtype):
    """Every positive eps that fp32 holds keeps zero heads at zero, and their gradients at
    g w / sqrt(eps); other heads are as with any eps below their mean square."""
    c = Case(580, 1, 6, 2, 2, 64, dtype)
    q, dqo, w = c.tok(2), c.tok(2), 1 + 0.3 * c.n(2, 64, to=torch.float32)
    q[0, [0, 3]] = 0
    dqo[0, [0, 3]] *= 2.0 ** -10  # (times 1 / sqrt(eps) within fp32)
    rot = gbla.rotation_table(6, 64, device="cpu")
    eps = torch.tensor(eps, dtype=torch.float32).item()
    o = gbla.qk_norm_rotate(dev(q), dev(q), dev(w), dev(w), dev(rot), eps=eps)[0]
    assert (o[0, [0, 3]] == 0).all()
    ref, mag = R.norm_rotate(q, w, rot, None, 64, False, eps)
    _close(o, ref, mag, 80 * 2.0 ** -24, dtype, "q")
    g = gbla.qk_norm_rotate_backward(dev(q), dev(q), dev(w), dev(w), dev(rot), dev(dqo), dev(dqo), eps=eps)
    dx, dxm, dw, dwm = R.norm_rotate_backward(q, w, rot, None, 64, False, eps, dqo, [6])
    _close(g["dq"], dx, dxm, 80 * 2.0 ** -23, dtype, "dq")
    _close(g["dnorm_q"], dw, dwm, 80 * 2.0 ** -23 + 6 * 2.0 ** -24, "fp32", "dnorm_q")


def test_heads_as_small_as_the_root_of_eps():
    """Heads about sqrt(eps) for a tiny eps: no product with three reciprocal roots overflows
    where the gradient (1e23) does not."""
    eps = torch.tensor(2e-37, dtype=torch.float32).item()
    c = Case(581, 1, 5, 2, 2, 64, "fp32")
    q, dqo, w = c.tok(2) * 3e-19, c.tok(2) * 2.0 ** 16, 1 + 0.3 * c.n(2, 64, to=torch.float32)
    rot = gbla.rotation_table(5, 64, device="cpu")
    g = gbla.qk_norm_rotate_backward(dev(q), dev(q), dev(w), dev(w), dev(rot), dev(dqo), dev(dqo), eps=eps)
    dx, dxm, dw, dwm = R.norm_rotate_backward(q, w, rot, None, 64, False, eps, dqo, [5])
    _close(g["dq"], dx, dxm, 80 * 2.0 ** -23, "fp32", "dq")
    _close(g["dnorm_q"], dw, dwm, 80 * 2.0 ** -23 + 5 * 2.0 ** -24, "fp32", "dnorm_q")


# ------------------------------------------------------------- differentiable forms

@pytest.mark.parametrize("dtype,D,algo", [("bf16", 64, gbla.ALGO_AUTO), ("bf16", 128, gbla.ALGO_AUTO),
                                          ("bf16", 64, gbla.ALGO_SIMT), ("fp32", 32, gbla.ALGO_AUTO)])
def test_differentiable_forms_give_the_operators_gradients(dtype, D, algo):
    """Options, packed inputs, an incoming gradient that is not contiguous and a final state
    that nothing uses: bit for bit the operators' own gradients."""
    c = Case(590, 2, 90, 4, 4, D, dtype, [90, 41])
    packed = dev(c.n(2, 90, 3, 4, D)).requires_grad_()
    q, k, v = packed.unbind(2)
    w = (1 + 0.1 * dev(c.n(4, D, to=torch.float32))).requires_grad_()
    ld, rot, sl = torch.full((4,), -0.05, device="cuda"), gbla.rotation_table(90, D), dev(c.seq_lens)
    do = dev(c.n(90, 2, 4, D)).transpose(0, 1)
    opt, att = dict(eps=1e-3, interleaved=True), dict(scale=0.3, algo=algo)
    a, b = decoder.norm_rotate(q, k, w, w, rot, None, sl, **opt)
    o, _ = decoder.attention(a, b, v, ld, sl, **att)
    dp, dw = torch.autograd.grad(o, [packed, w], do)
    with torch.no_grad():
        g = gbla.decay_attention_backward(a, b, v, ld, do.contiguous(), sl, **att)
        r = gbla.qk_norm_rotate_backward(q, k, w, w, rot, g["dq"], g["dk"], None, sl, **opt)
    assert torch.equal(dp, torch.stack([r["dq"], r["dk"], g["dv"]], 2))
    assert torch.equal(dw, r["dnorm_q"] + r["dnorm_k"])


# ------------------------------------------------------------- kernel families

@pytest.mark.parametrize("i", [i for i, c in enumerate(DEC) if c[5] == "bf16"])
def test_bf16_runs_on_tensor_cores(i):
    """The tensor-core family, asked for by name (an error where it does not cover a call),
    within its bounds, and what the automatic choice takes."""
    c, q, k, v, ld, s0 = _decay_case(i)
    do, ds = dev(c.tok(c.H)), dev(c.n(c.B, c.H, c.D, c.D, to=torch.float32))
    args, kw = [dev(x) for x in (q, k, v, ld)], dict(seq_lens=dev(c.seq_lens), state=dev(s0))
    out = [torch.zeros(q.shape, dtype=q.dtype, device="cuda") for _ in range(2)]
    (o, S), (o2, S2) = (gbla.decay_attention(*args, out=b, return_state=True, algo=a, **kw)
                        for a, b in ((gbla.ALGO_TC, out[0]), (gbla.ALGO_AUTO, out[1])))
    assert torch.equal(o, o2) and torch.equal(S, S2)
    on = ~c.past()
    ref, Sr, om, Sm = R.decay(q, k, v, ld, c.lens, s0, c.D ** -0.5)
    _close(o.cpu()[on], ref[on], om[on], 2.0 ** -8, "bf16", "o", 2.0 ** -7)
    _close(S, Sr, Sm, c32(c), "fp32", "state")
    g, g2 = (gbla.decay_attention_backward(*args, do, dstate=ds, return_dstate=True, algo=a, **kw)
             for a in (gbla.ALGO_TC, gbla.ALGO_AUTO))
    for n in g:
        assert torch.equal(g[n], g2[n]), n
    ref, mag = R.decay_backward(q, k, v, ld, do.cpu(), c.lens, s0, ds.cpu(), c.D ** -0.5)
    for n in ("dq", "dk", "dv"):
        _close(g[n], ref[n], mag[n], 2.0 ** -8, "bf16", n, 2.0 ** -7)
    _close(g["dstate"], ref["dstate"], mag["dstate"], c32(c), "fp32", "dstate")
    assert gbla.device_error() == 0
