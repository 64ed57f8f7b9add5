"""GPU parity of the decoder operators, through the C ABI, against the 64-bit
references of decoder_ref.py.

Bounds, with m the reference evaluated on magnitudes (every product and sum on
absolute values), so that a relative error e of the intermediates moves a
result by at most about e m, and half a bf16 ulp of the result for bf16 storage:

* norm and rotation: fp32 arithmetic, at most D + 16 roundings of 2^-24 on a
  path (the sum of squares, the reciprocal root, the products):
  (D + 16) 2^-24 m.  Weight gradients add one rounding a token at worst.
* decayed attention, fp32 arithmetic: sums of D, and of up to 64 tokens of a
  chunk, one product by a power of the decay a chunk of 32 tokens, the power's
  exponent rounded to 2^-24 of itself (a weight of gamma^n is off by n |ln gamma|
  2^-23, which times the weight stays below 2^-24):
  (N / 32 + D + 80) 2^-22 m.
* on tensor cores the weighted scores, or the state as it meets a query, are
  rounded once to bf16 (2^-9): 2^-8 m, and as these errors are independent,
  2^-7 of the tensor's norm.  The state itself stays in fp32 (the fp32 bound).
"""
import numpy as np
import pytest
import torch

import decoder_ref as R
from paper_2606_07317_gb300 import gbla

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
FAMILY = {"auto": gbla.ALGO_AUTO, "simt": gbla.ALGO_SIMT}


def _close(got, ref, mag, c, dtype, what, normwise=None):
    got = got.detach().cpu().double()
    assert torch.isfinite(got).all(), what
    bound = c * mag + (0.5 * R.ulp_bf16(ref) if dtype == "bf16" else 0) + 1e-30
    over = ((got - ref).abs() - bound).max().item() if ref.numel() else -1.0
    assert over <= 0, (what, over, ((got - ref).abs() / bound).max().item())
    if normwise is not None and ref.numel():
        assert (got - ref).norm() <= normwise * ref.norm() + 1e-30, (what, ((got - ref).norm() / ref.norm()).item())


class Case:
    """Seeded inputs on the host in their stored precision."""

    def __init__(self, seed, B, N, H, Hk, D, dtype, lens=None):
        self.g = torch.Generator().manual_seed(seed)
        self.B, self.N, self.H, self.Hk, self.D, self.dtype = B, N, H, Hk, D, dtype
        self.lens = list(lens) if lens is not None else [N] * B
        self.seq_lens = torch.tensor(self.lens, dtype=torch.int32) if lens is not None else None

    def n(self, *shape, to=None):
        return torch.randn(shape, generator=self.g).to(to or TYPES[self.dtype])

    def tok(self, heads):
        return self.n(self.B, self.N, heads, self.D)

    def past(self):
        """[B, N] truth values of the padding rows."""
        return torch.arange(self.N)[None] >= torch.tensor(self.lens)[:, None]

    def poison(self, x, value=float("nan")):
        x = x.clone()
        x[self.past()] = value
        return x


def dev(x):
    return x.cuda() if x is not None else None


# ------------------------------------------------------------ norm and rotation

ROT = [  # B, N, H, Hk, D, R, interleaved, dtype, lens, positions
    (1, 1, 1, 1, 32, 32, False, "fp32", None, "none"),
    (8, 1, 8, 8, 64, 64, False, "bf16", None, "random"),
    (2, 37, 6, 2, 64, 32, True, "fp32", [37, 11], "random"),
    (3, 50, 3, 1, 128, 128, False, "bf16", [50, 0, 1], "random"),
    (2, 33, 5, 5, 32, 16, False, "bf16", [7, 33], "none"),
    (2, 65, 4, 4, 128, 48, False, "fp32", None, "random"),
    (1, 19, 7, 7, 64, 0, False, "bf16", None, "none"),
    (2, 700, 8, 4, 64, 64, True, "bf16", [700, 333], "random"),
    (1, 2100, 16, 16, 128, 64, True, "fp32", None, "none"),
]


def _rotate_case(i):
    B, N, H, Hk, D, Rd, inter, dtype, lens, how = ROT[i]
    c = Case(100 + i, B, N, H, Hk, D, dtype, lens)
    P = max(N, 40)
    rot = gbla.rotation_table(P, Rd, device="cpu") if Rd else None
    pos = torch.randint(0, P, (B, N), generator=c.g).to(torch.int32) if how == "random" else None
    wq, wk = 1 + 0.3 * c.n(H, D, to=torch.float32), 1 + 0.3 * c.n(Hk, D, to=torch.float32)
    return c, c.tok(H), c.tok(Hk), wq, wk, rot, pos, Rd, inter


@pytest.mark.parametrize("i", range(len(ROT)))
def test_norm_rotate(i):
    c, q, k, wq, wk, rot, pos, Rd, inter = _rotate_case(i)
    eps = 1e-5
    out = (torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(k.shape, 7.0, dtype=q.dtype, device="cuda"))
    gbla.qk_norm_rotate(dev(c.poison(q)), dev(c.poison(k)), dev(wq), dev(wk), dev(rot), dev(pos), dev(c.seq_lens),
                        eps=eps, interleaved=inter, out=out)
    past = c.past()
    for x, w, o, name in ((q, wq, out[0], "q"), (k, wk, out[1], "k")):
        ref, mag = R.norm_rotate(x, w, rot, pos, Rd, inter, eps)
        o = o.cpu()
        assert (o[past] == 7.0).all(), "padding rows were written"
        _close(o[~past], ref[~past], mag[~past], (c.D + 16) * 2.0 ** -24, c.dtype, name)


@pytest.mark.parametrize("i", range(len(ROT)))
def test_norm_rotate_backward(i):
    c, q, k, wq, wk, rot, pos, Rd, inter = _rotate_case(i)
    eps, dqo, dko = 1e-5, c.tok(c.H), c.tok(c.Hk)
    args = (dev(c.poison(q)), dev(c.poison(k)), dev(wq), dev(wk), dev(rot), dev(c.poison(dqo)), dev(c.poison(dko)))
    kw = dict(positions=dev(pos), seq_lens=dev(c.seq_lens), eps=eps, interleaved=inter)
    g = gbla.qk_norm_rotate_backward(*args, **kw)
    again = gbla.qk_norm_rotate_backward(*args, **kw)
    for n in g:
        assert torch.equal(g[n], again[n]), n
    u = (c.D + 16) * 2.0 ** -23
    for x, w, dy, t in ((q, wq, dqo, "q"), (k, wk, dko, "k")):
        dx, dxm, dw, dwm = R.norm_rotate_backward(x, w, rot, pos, Rd, inter, eps, dy, c.lens)
        _close(g["d" + t], dx, dxm, u, c.dtype, "d" + t)
        assert (g["d" + t].cpu()[c.past()] == 0).all()
        _close(g["dnorm_" + t], dw, dwm, u + sum(c.lens) * 2.0 ** -24, "fp32", "dnorm_" + t)


def test_positions_are_clamped_to_the_table():
    c = Case(7, 1, 4, 2, 2, 64, "fp32")
    q, w, rot = dev(c.tok(2)), torch.ones((2, 64), device="cuda"), gbla.rotation_table(10, 64)
    at = lambda p: gbla.qk_norm_rotate(q, q, w, w, rot, torch.tensor([p], dtype=torch.int32, device="cuda"))[0]  # noqa: E731
    assert torch.equal(at([-5, 9, 10, 2 ** 31 - 1]), at([0, 9, 9, 9]))


def test_norm_rotate_zero_rows_and_large_values():
    """A zero head stays zero (eps holds the root up); heads of 1e18 do not overflow to NaN
    after the norm, as long as their squares' mean is finite."""
    w, rot = torch.ones((2, 64), device="cuda"), gbla.rotation_table(4, 64)
    x = torch.zeros((1, 4, 2, 64), device="cuda")
    x[0, 2] = 1e18
    o = gbla.qk_norm_rotate(x, x, w, w, rot)[0]
    assert (o[0, [0, 1, 3]] == 0).all() and torch.isfinite(o).all()
    assert abs(o[0, 2].square().mean().item() - 1) < 1e-4


# ------------------------------------------------------------ decayed attention

def c32(c):
    return (c.N / 32 + c.D + 80) * 2.0 ** -22


def _decays(H, kind, gen):
    if kind == "mixed":  # memoryless, strong, weak, none, growing
        return torch.tensor([float("-inf"), -3.0, -0.05, -1e-3, 0.0, 2e-4])[torch.arange(H) % 6]
    return -torch.exp2(-(3 + 6 * torch.rand(H, generator=gen)))


DEC = [  # B, N, H, Hk, D, dtype, lens, state, decays
    (1, 1, 1, 1, 32, "fp32", None, False, "some"),
    (2, 1, 6, 3, 64, "bf16", [1, 0], True, "mixed"),
    (3, 31, 6, 6, 64, "fp32", [31, 0, 1], True, "mixed"),
    (2, 33, 6, 2, 32, "bf16", [33, 32], True, "mixed"),
    (5, 65, 6, 6, 64, "bf16", [65, 64, 63, 0, 1], True, "mixed"),
    (4, 130, 2, 1, 64, "bf16", [127, 128, 129, 130], False, "some"),
    (5, 130, 2, 1, 128, "bf16", [127, 128, 129, 130, 0], True, "some"),
    (2, 193, 6, 3, 128, "bf16", None, True, "mixed"),
    (2, 97, 3, 3, 128, "fp32", [97, 40], False, "some"),
    (1, 2049, 2, 2, 64, "fp32", None, True, "some"),
    (1, 2301, 6, 2, 64, "bf16", None, True, "mixed"),
    (2, 1500, 3, 3, 128, "bf16", [1500, 700], True, "some"),
    (1, 1111, 3, 1, 32, "bf16", None, False, "some"),
    (40, 200, 6, 6, 64, "bf16", None, False, "some"),
]


def _decay_case(i):
    B, N, H, Hk, D, dtype, lens, state, kind = DEC[i]
    c = Case(200 + i, B, N, H, Hk, D, dtype, lens)
    ld = _decays(H, kind, c.g).float()
    s0 = c.n(B, H, D, D, to=torch.float32) if state else None
    return c, c.tok(H), c.tok(Hk), c.tok(Hk), ld, s0


def _tol(c, algo):
    """(elementwise, normwise) bounds of a result of the case."""
    tc = c.dtype == "bf16" and algo != gbla.ALGO_SIMT
    return (2.0 ** -8, 2.0 ** -7) if tc else (c32(c), None)


@pytest.mark.parametrize("family", FAMILY)
@pytest.mark.parametrize("i", range(len(DEC)))
def test_decay_attention(i, family):
    c, q, k, v, ld, s0 = _decay_case(i)
    algo = FAMILY[family]
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    args = [dev(c.poison(x)) for x in (q, k, v)] + [dev(ld), dev(c.seq_lens), dev(s0)]
    _, S = gbla.decay_attention(*args, out=out, return_state=True, algo=algo)
    ref, Sr, om, Sm = R.decay(q, k, v, ld, c.lens, s0, c.D ** -0.5)
    past, o = c.past(), out.cpu()
    assert (o[past] == 7.0).all(), "padding rows were written"
    el, nw = _tol(c, algo)
    _close(o[~past], ref[~past], om[~past], el, c.dtype, "o", nw)
    _close(S, Sr, Sm, c32(c), "fp32", "state")
    # the same without the state, and again: the same bits
    two = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    gbla.decay_attention(*args, out=two, algo=algo)
    three = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    _, S3 = gbla.decay_attention(*args, out=three, return_state=True, algo=algo)
    assert torch.equal(out, three) and torch.equal(S, S3)
    _close(two.cpu()[~past], ref[~past], om[~past], el, c.dtype, "o without state", nw)
    assert gbla.device_error() == 0


@pytest.mark.parametrize("family", FAMILY)
@pytest.mark.parametrize("i", range(len(DEC)))
def test_decay_attention_backward(i, family):
    c, q, k, v, ld, s0 = _decay_case(i)
    algo, scale = FAMILY[family], -0.2
    do = c.tok(c.H)
    ds = c.n(c.B, c.H, c.D, c.D, to=torch.float32) if s0 is not None else None
    args = [dev(c.poison(x)) for x in (q, k, v)] + [dev(ld), dev(c.poison(do))]
    kw = dict(seq_lens=dev(c.seq_lens), state=dev(s0), dstate=dev(ds), scale=scale, algo=algo)
    g = gbla.decay_attention_backward(*args, return_dstate=True, **kw)
    ref, mag = R.decay_backward(q, k, v, ld, do, c.lens, s0, ds, scale)
    el, nw = _tol(c, algo)
    for n in ("dq", "dk", "dv"):
        _close(g[n], ref[n], mag[n], el, c.dtype, n, nw)
        assert (g[n].cpu()[c.past()] == 0).all(), n
    _close(g["dstate"], ref["dstate"], mag["dstate"], c32(c), "fp32", "dstate")
    again = gbla.decay_attention_backward(*args, return_dstate=True, **kw)
    for n in g:
        assert torch.equal(g[n], again[n]), n
    assert gbla.device_error() == 0


@pytest.mark.parametrize("D,N,lens", [(64, 4100, [4100, 70]), (32, 4224, None), (128, 2600, [1, 2600])])
def test_many_segments_from_a_first_state(D, N, lens):
    """Few long sequences, which the tensor-core family cuts into many segments: states
    going in and out in both directions."""
    c = Case(300 + D, 2 if lens else 1, N, 2, 1, D, "bf16", lens)
    q, k, v, do = c.tok(2), c.tok(1), c.tok(1), c.tok(2)
    ld = torch.tensor([-2.0 ** -9, -2.0 ** -6])
    s0, ds = (c.n(c.B, 2, D, D, to=torch.float32) for _ in range(2))
    args, kw = [dev(c.poison(x)) for x in (q, k, v)] + [dev(ld)], dict(seq_lens=dev(c.seq_lens), state=dev(s0))
    o, S = gbla.decay_attention(*args, return_state=True, **kw)
    ref, Sr, om, Sm = R.decay(q, k, v, ld, c.lens, s0, D ** -0.5)
    on = ~c.past()
    _close(o.cpu()[on], ref[on], om[on], 2.0 ** -8, "bf16", "o", 2.0 ** -7)
    _close(S, Sr, Sm, c32(c), "fp32", "state")
    g = gbla.decay_attention_backward(*args, dev(c.poison(do)), dstate=dev(ds), return_dstate=True, **kw)
    ref, mag = R.decay_backward(q, k, v, ld, do, c.lens, s0, ds, D ** -0.5)
    for n in ("dq", "dk", "dv"):
        _close(g[n], ref[n], mag[n], 2.0 ** -8, "bf16", n, 2.0 ** -7)
    _close(g["dstate"], ref["dstate"], mag["dstate"], c32(c), "fp32", "dstate")
    assert gbla.device_error() == 0


@pytest.mark.parametrize("dtype,D", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_continued_prompt_and_steps_agree_with_one_call(dtype, D):
    """A prompt read in two calls and then token by token follows the one-call form."""
    c = Case(31, 2, 150, 4, 2, D, dtype)
    q, k, v = (dev(c.tok(h)) for h in (4, 2, 2))
    ld = dev(_decays(4, "some", c.g).float())
    whole, S = gbla.decay_attention(q, k, v, ld, return_state=True)
    a, S1 = gbla.decay_attention(q[:, :101], k[:, :101], v[:, :101], ld, return_state=True)
    b, S2 = gbla.decay_attention(q[:, 101:140], k[:, 101:140], v[:, 101:140], ld, state=S1, return_state=True)
    steps = []
    for t in range(140, 150):
        steps.append(gbla.decay_attention_step(q[:, t:t + 1], k[:, t:t + 1], v[:, t:t + 1], ld, S2))
    got = torch.cat([a, b] + steps, 1)
    ref, Sr, om, Sm = R.decay(q.cpu(), k.cpu(), v.cpu(), ld.cpu(), c.lens, None, D ** -0.5)
    el, nw = _tol(c, gbla.ALGO_AUTO)
    _close(got, ref, om, el, dtype, "o", nw)
    _close(whole, ref, om, el, dtype, "o", nw)
    _close(S2, Sr, Sm, c32(c), "fp32", "state")
    _close(S, Sr, Sm, c32(c), "fp32", "state")


@pytest.mark.parametrize("family", FAMILY)
@pytest.mark.parametrize("D,dtype", [(32, "fp32"), (64, "bf16"), (128, "bf16"), (128, "fp32")])
def test_packed_and_token_major_views(D, dtype, family):
    """Slices of a packed projection, and a [N, B, ...] layout, give the contiguous call's bits."""
    c = Case(41, 3, 77, 4, 4, D, dtype, [77, 30, 0])
    packed = dev(c.n(3, 77, 3, 4, D))
    ld, sl, algo = dev(_decays(4, "some", c.g).float()), dev(c.seq_lens), FAMILY[family]
    cut = [packed[:, :, i] for i in range(3)]
    turned = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in cut]
    whole = [x.contiguous() for x in cut]
    w, rot = torch.ones((4, D), device="cuda"), gbla.rotation_table(80, D)
    do = dev(c.tok(4))
    past = c.past()
    want = None
    for x in (whole, cut, turned):
        g = gbla.decay_attention_backward(*x, ld, do, sl, algo=algo)
        r = gbla.qk_norm_rotate_backward(x[0], x[1], w, w, rot, do, do, seq_lens=sl)
        got = [gbla.decay_attention(*x, ld, sl, algo=algo).cpu()[~past], *gbla.qk_norm_rotate(x[0], x[1], w, w, rot),
               *g.values(), *r.values()]
        assert want is None or all(torch.equal(a, b) for a, b in zip(want, got))
        want = got


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_offsets_past_32_bits(dtype, D):
    """Tokens 2^26 elements apart: byte and element offsets pass 2^32."""
    c = Case(51, 1, 70, 2, 2, D, dtype)
    x = [c.tok(2) for _ in range(3)]
    far = torch.empty(70 * 2 ** 26 // (2 if dtype == "fp32" else 1), dtype=TYPES[dtype], device="cuda")
    st = far.numel() // 70
    views = []
    for i, t in enumerate(x):
        view = far.as_strided((1, 70, 2, D), (far.numel(), st, D, 1), i * 2 * D)
        view.copy_(t)
        views.append(view)
    ld = dev(_decays(2, "some", c.g).float())
    near = [dev(t) for t in x]
    do, w, rot = dev(c.tok(2)), torch.ones((2, D), device="cuda"), gbla.rotation_table(70, D)
    assert torch.equal(gbla.decay_attention(*views, ld), gbla.decay_attention(*near, ld))
    a, b = (gbla.decay_attention_backward(*t, ld, do) for t in (views, near))
    assert all(torch.equal(a[n], b[n]) for n in a)
    a, b = (gbla.qk_norm_rotate(t[0], t[1], w, w, rot) for t in (views, near))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("B,H,Hk,D,dtype", [(1, 1, 1, 32, "fp32"), (3, 6, 2, 64, "bf16"), (2, 4, 4, 128, "fp32"),
                                            (5, 2, 1, 128, "bf16"), (4, 3, 3, 32, "bf16")])
def test_step(B, H, Hk, D, dtype):
    c = Case(61, B, 1, H, Hk, D, dtype)
    q, k, v = c.tok(H), c.tok(Hk), c.tok(Hk)
    ld = _decays(H, "mixed", c.g).float()
    pool = c.n(B + 4, H, D, D, to=torch.float32)
    slots = torch.randperm(B + 4, generator=c.g)[:B].to(torch.int32)
    ref, Sr, om, Sm = R.decay(q, k, v, ld, [1] * B, pool[slots.long()], 0.3)
    state = dev(pool)
    o = gbla.decay_attention_step(dev(q), dev(k), dev(v), dev(ld), state, dev(slots), scale=0.3)
    u = (D + 16) * 2.0 ** -23
    _close(o, ref, om, u, dtype, "o")
    _close(state.cpu()[slots.long()], Sr, Sm, u, "fp32", "state")
    rest = [i for i in range(B + 4) if i not in slots.tolist()]
    assert torch.equal(state.cpu()[rest], pool[rest]), "another sequence's state changed"
    # the identity pool
    state = dev(pool)
    ref, Sr, om, Sm = R.decay(q, k, v, ld, [1] * B, pool[:B], 0.3)
    o = gbla.decay_attention_step(dev(q), dev(k), dev(v), dev(ld), state, scale=0.3)
    _close(o, ref, om, u, dtype, "o")


def test_gradients_of_very_many_short_sequences():
    """More sequences than a third of a grid's 65535 rows, two tokens each."""
    g = torch.Generator().manual_seed(5)
    q, k, v, do = (torch.randn((22000, 2, 1, 32), generator=g) for _ in range(4))
    ld = torch.tensor([-0.25])
    got = gbla.decay_attention_backward(q.cuda(), k.cuda(), v.cuda(), ld.cuda(), do.cuda(), scale=0.5)
    q, k, v, do = (t.double()[:, :, 0] for t in (q, k, v, do))
    w = 0.5 * torch.exp(ld.double()) ** (torch.arange(2)[:, None] - torch.arange(2)).clamp(min=0) * torch.ones(2, 2).tril()

    def grads(q, k, v, do):
        dp, p = (do @ v.mT) * w, (q @ k.mT) * w
        return {"dq": dp @ k, "dk": dp.mT @ q, "dv": p.mT @ do}
    ref, mag = grads(q, k, v, do), grads(q.abs(), k.abs(), v.abs(), do.abs())
    for name in ref:
        err = (got[name].cpu().double()[:, :, 0] - ref[name]).abs()
        tol = (32 + 80) * 2.0 ** -22 * mag[name]
        assert bool((err <= tol).all()), (name, float((err / tol).max()))


def test_steps_do_not_drift():
    """A weak decay over 4096 steps (keys of zero) against the exact power: each step rounds
    once to 2^-24 at random, sqrt(n) 2^-24 of the norm (times 8); a decay held in one float
    would be off by up to n 2^-25."""
    n, ld = 4096, torch.tensor([-2.9e-4, -1.7e-4, -1e-3], device="cuda")
    S0 = torch.randn((1, 3, 64, 64), generator=torch.Generator().manual_seed(5))
    S, z = dev(S0), torch.zeros((1, 1, 3, 64), device="cuda")
    for _ in range(n):
        gbla.decay_attention_step(z, z, z, ld, S)
    want = S0.double() * (n * ld.cpu().double()).exp()[None, :, None, None]
    for h in range(3):
        got = S[0, h].cpu().double()
        assert (got - want[0, h]).norm() <= 8 * n ** 0.5 * 2.0 ** -24 * want[0, h].norm(), h


@pytest.mark.parametrize("D,dtype", [(32, "bf16"), (64, "bf16"), (128, "bf16"), (64, "fp32")])
def test_long_state_with_a_weak_decay(D, dtype):
    """The state after 32768 tokens at a horizon of 4096 against the explicit sum: fp32
    rounding at random, 32 x 2^-24 of the norm, no drift with the length."""
    c = Case(95, 1, 32768, 2, 2, D, dtype)
    q, k, v = (c.tok(2) for _ in range(3))
    ld = torch.log1p(-torch.exp2(torch.tensor([-12.0, -11.3])))
    _, S = gbla.decay_attention(dev(q), dev(k), dev(v), dev(ld), return_state=True)
    t = torch.arange(c.N, dtype=torch.float64)
    for h in range(2):
        w = ((c.N - 1 - t) * ld[h].double()).exp()[:, None]
        want = (k[0, :, h].double() * w).T @ v[0, :, h].double()
        assert (S[0, h].cpu().double() - want).norm() <= 32 * 2.0 ** -24 * want.norm(), h


def test_step_rows_without_a_sequence():
    c = Case(62, 4, 1, 2, 2, 64, "bf16")
    q = dev(c.tok(2))
    pool = dev(c.n(3, 2, 64, 64, to=torch.float32))
    before = pool.clone()
    out = torch.full_like(q, 7.0)
    slots = torch.tensor([-1, 3, 1, -2 ** 31], dtype=torch.int32, device="cuda")
    gbla.decay_attention_step(q, q, q, torch.zeros(2, device="cuda"), pool, slots, out=out)
    assert (out[[0, 1, 3]] == 7.0).all() and (out[2] != 7.0).any()
    assert torch.equal(pool[[0, 2]], before[[0, 2]]) and not torch.equal(pool[1], before[1])


def test_step_takes_rows_of_a_longer_buffer():
    c = Case(63, 3, 20, 4, 4, 64, "bf16")
    x = dev(c.n(3, 20, 3, 4, 64))
    cut = [x[:, 7:8, i] for i in range(3)]
    ld = torch.full((4,), -0.1, device="cuda")
    a, b = (torch.zeros((3, 4, 64, 64), device="cuda") for _ in range(2))
    o1 = gbla.decay_attention_step(*cut, ld, a)
    o2 = gbla.decay_attention_step(*[t.contiguous() for t in cut], ld, b)
    assert torch.equal(o1, o2) and torch.equal(a, b)


def test_empty_sequences_pass_the_state_on():
    s = torch.randn((2, 3, 64, 64), device="cuda")
    e = torch.empty((2, 0, 3, 64), dtype=torch.bfloat16, device="cuda")
    ld = torch.zeros(3, device="cuda")
    assert torch.equal(gbla.decay_attention(e, e, e, ld, state=s, return_state=True)[1], s)
    assert (gbla.decay_attention(e, e, e, ld, return_state=True)[1] == 0).all()
    g = gbla.decay_attention_backward(e, e, e, ld, e, dstate=s, return_dstate=True)
    assert torch.equal(g["dstate"], s)
    w, rot = torch.ones((3, 64), device="cuda"), gbla.rotation_table(4, 64)
    assert (gbla.qk_norm_rotate_backward(e, e, w, w, rot, e, e)["dnorm_q"] == 0).all()


def test_another_stream_orders_with_its_own_work():
    """Calls on a side stream see what that stream wrote before them."""
    c = Case(71, 2, 300, 4, 4, 64, "bf16")
    host = [c.tok(4) for _ in range(3)]
    ld = dev(_decays(4, "some", c.g).float())
    want = gbla.decay_attention(*[dev(x) for x in host], ld)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn((4096, 4096), device="cuda")
        for _ in range(4):
            big = big @ big * 1e-3
        x = [dev(t) for t in host]
        got = gbla.decay_attention(*x, ld)
        S = torch.zeros((2, 4, 64, 64), device="cuda")
        gbla.decay_attention_step(*[t[:, :1] for t in x], ld, S)
    side.synchronize()
    assert torch.equal(got, want)
    ref = R.decay(*[t[:, :1] for t in host], ld.cpu(), [1, 1], None, 1.0)
    _close(S, ref[1], ref[3], 80 * 2.0 ** -23, "fp32", "state")


def test_captured_in_a_graph():
    """The token path (norm and rotation, then the step) replays from a CUDA graph."""
    c = Case(81, 4, 1, 4, 4, 64, "bf16")
    q, k, v = (dev(c.tok(4)) for _ in range(3))
    w, rot = torch.ones((4, 64), device="cuda"), gbla.rotation_table(32, 64)
    pos = torch.zeros((4, 1), dtype=torch.int32, device="cuda")
    ld = torch.full((4,), -0.2, device="cuda")
    S, o = torch.zeros((4, 4, 64, 64), device="cuda"), torch.empty_like(q)
    buf = (torch.empty_like(q), torch.empty_like(k))

    def token():
        gbla.qk_norm_rotate(q, k, w, w, rot, pos, out=buf)
        gbla.decay_attention_step(buf[0], buf[1], v, ld, S, out=o)
        pos.add_(1)

    token()
    S.zero_()
    pos.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token()
    got = []
    for _ in range(5):
        graph.replay()
        got.append(o.clone())
    S.zero_()
    pos.zero_()
    for t in range(5):
        token()
        assert torch.equal(o, got[t]), t


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_prompt_and_gradients_in_a_graph(dtype, D):
    """Calls that cut the sequence (several launches, pool scratch) replay from a CUDA graph."""
    c = Case(82, 1, 1024, 2, 1, D, dtype)
    q, k, v, do = (dev(c.tok(h)) for h in (2, 1, 1, 2))
    ld, w = dev(_decays(2, "some", c.g).float()), torch.ones((2, D), device="cuda")
    rot = gbla.rotation_table(1024, D)

    def work():
        a, b = gbla.qk_norm_rotate(q, k, w, w[:1], rot)
        o, S = gbla.decay_attention(a, b, v, ld, return_state=True)
        return [o, S, *gbla.decay_attention_backward(a, b, v, ld, do).values()]

    want = [t.clone() for t in work()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for _ in range(2):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("D", [32, 64, 128])
def test_decay_attention_long_rows_sampled(D):
    """32768 tokens: sampled rows against explicit sums over pairs of tokens."""
    c = Case(91, 1, 32768, 2, 2, D, "bf16")
    q, k, v = (c.tok(2) for _ in range(3))
    ld = torch.tensor([-2.0 ** -6, -2.0 ** -12])
    o, S = gbla.decay_attention(dev(q), dev(k), dev(v), dev(ld), return_state=True)
    for h in range(2):
        kk, vv = k[0, :, h].double(), v[0, :, h].double()
        t = torch.arange(c.N, dtype=torch.float64)
        for r in (0, 63, 64, 4095, 4096, 20000, 32767):
            w = ((r - t[:r + 1]) * ld[h].double()).exp()
            s = (kk[:r + 1] @ q[0, r, h].double()) * w * D ** -0.5
            ref, mag = s @ vv[:r + 1], s.abs() @ vv[:r + 1].abs()
            _close(o[0, r, h], ref, mag, 2.0 ** -8, "bf16", (h, r))
        w = ((c.N - 1 - t) * ld[h].double()).exp()[:, None]
        _close(S[0, h], (kk * w).T @ vv, (kk.abs() * w).T @ vv.abs(), c32(c), "fp32", ("state", h))
    np.testing.assert_equal(gbla.device_error(), 0)
