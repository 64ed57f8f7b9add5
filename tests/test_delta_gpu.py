"""GPU parity of attention by the gated delta rule, against the 64-bit recurrence of
delta_ref.py.

Bounds, relative to a tensor's norm (no elementwise magnitudes: the recurrence evaluated on
absolute values grows without bound, while the recurrence itself, with beta |k|^2 <= 2, moves
no error of the state apart, so that rounding errors of tokens add up like independent ones):

* fp32 arithmetic: a token's step, or its share of a chunk, rounds an entry of the state a
  few times, 4 sqrt(N) together; a sum of D, or of the 64 tokens of a chunk, as many terms
  2 sqrt(D + 64); with the gates' exponentials:  (4 sqrt(N) + 2 sqrt(D + 64) + 16) 2^-24.
* bf16 results: one rounding, 2^-8 at most, and operands inside rounded to 2^-11 (the
  triangular products) or 2^-16 (the state) at most three times in a row:  2^-8 + 3 2^-11.
  The state itself: the fp32 bound, whatever the type.
* gradients: the same, with twice the products in a row; the log decays' are sums of up to 64
  shares of either sign, with errors that add like independent ones: 8 times what comes before
  the last rounding.  The shares may cancel (a first token without a state before it has none
  to fade, its gradient is exactly 0): as inner products they are off by that of their vectors'
  lengths, |do| |o| and |dv| |v|, which count beside the gradient.
Single elements: 24 times the bound times the tensor's root mean square, and half an ulp."""
import math

import pytest
import torch

import delta_ref as R
from paper_2606_07317_gb300 import gbla

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def bound(dtype, N, D):
    f = (4 * math.sqrt(N) + 2 * math.sqrt(D + 64) + 16) * 2.0 ** -24
    return f if dtype == "fp32" else 2.0 ** -8 + 3 * 2.0 ** -11 + f


def grad_bound(name, dtype, N, D):
    if name == "dstate":
        return 2 * bound("fp32", N, D)
    inner = 2 * (bound(dtype, N, D) - (2.0 ** -8 if dtype == "bf16" else 0))
    return (8 if name == "dlog_decay" else 1) * inner + (2.0 ** -8 if dtype == "bf16" else 0)


def shares(x, do, g, lens, state, scale):
    """Lengths of the vectors whose products a log decay's gradient consists of."""
    o, _ = R.delta(*x.values(), lens, state, scale)
    v, past = x["v"].double(), (o == 0).all(-1)
    got = do.double().norm(dim=-1) * o.norm(dim=-1) + g["dv"].norm(dim=-1) * v.norm(dim=-1)
    return torch.where(past, 0.0, got)


def close(got, ref, tol, what, beside=None):
    got, ref = got.detach().double(), ref.to(got.device)
    assert got.shape == ref.shape, what
    assert torch.isfinite(got).all(), what
    if not ref.numel():
        return
    d = got - ref
    size = ref.norm() + (0 if beside is None else beside.norm())
    assert d.norm() <= tol * size + 1e-30, (what, (d.norm() / size).item(), tol)
    rms = size / math.sqrt(ref.numel())
    over = (d.abs() - (24 * tol * rms + (2.0 ** -8 * ref.abs() if tol > 1e-3 else 0))).max()
    assert over <= 1e-30, (what, over.item(), rms.item())


class Case:
    """Seeded inputs on the GPU: unit keys and queries, gates as a model forms them."""

    def __init__(self, seed, B, N, H, Hk, D, dtype, lens=None, packed=False):
        self.g = torch.Generator().manual_seed(seed)
        self.B, self.N, self.H, self.Hk, self.D, self.dtype = B, N, H, Hk, D, dtype
        self.lens = list(lens) if lens is not None else [N] * B
        self.seq_lens = torch.tensor(self.lens, dtype=torch.int32).cuda() if lens is not None else None
        unit = lambda x: (x / x.norm(dim=-1, keepdim=True)).to(TYPES[dtype])  # noqa: E731
        horizon = 4.0 * 64.0 ** (torch.arange(H) / max(1, H - 1))
        g = -torch.nn.functional.softplus(self.n(B, N, H)) / horizon
        if packed:
            g[torch.rand((B, N, H), generator=self.g) < 0.05] = -math.inf
        x = dict(q=unit(self.n(B, N, Hk, D)), k=unit(self.n(B, N, Hk, D)), v=self.n(B, N, H, D), log_decay=g,
                 beta=self.n(B, N, H).sigmoid())
        self.x = {n: t.to(TYPES[dtype]).cuda() for n, t in x.items()}

    def n(self, *shape):
        return torch.randn(shape, generator=self.g)

    def state(self):
        return (0.5 * self.n(self.B, self.H, self.D, self.D)).cuda()

    def past(self):
        """[B, N] truth values of the padding rows."""
        return (torch.arange(self.N)[None] >= torch.tensor(self.lens)[:, None]).cuda()

    def poisoned(self):
        """The inputs with NaN in the padding rows."""
        past, got = self.past(), {}
        for n, t in self.x.items():
            got[n] = t.clone()
            got[n][past] = float("nan")
        return got


CASES = [  # B, N, H, Hk, D, dtype, lens, packed, state in
    (1, 1, 1, 1, 32, "fp32", None, False, False),
    (2, 1, 3, 1, 64, "bf16", None, False, True),
    (1, 2, 2, 2, 128, "bf16", None, False, True),
    (2, 63, 2, 1, 64, "fp32", None, True, True),
    (2, 64, 4, 4, 64, "bf16", [64, 64], False, False),
    (3, 65, 6, 3, 32, "bf16", [65, 0, 1], False, True),
    (2, 130, 2, 2, 128, "fp32", [130, 31], True, True),
    (2, 129, 2, 2, 128, "bf16", [97, 129], True, False),
    (4, 200, 5, 5, 32, "fp32", [200, 33, 64, 0], False, False),
    (2, 333, 8, 2, 64, "bf16", None, True, True),
    (1, 700, 3, 3, 64, "bf16", None, False, True),
    (1, 520, 2, 1, 32, "fp32", None, False, True),
    (17, 40, 9, 3, 64, "bf16", [40 - 2 * i for i in range(17)], True, True),
]


def _case(i):
    B, N, H, Hk, D, dtype, lens, packed, start = CASES[i]
    c = Case(300 + i, B, N, H, Hk, D, dtype, lens, packed)
    return c, c.state() if start else None


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward(i, keep):
    c, s0 = _case(i)
    out = torch.full_like(c.x["v"], 7.0)
    x = c.poisoned()
    got = gbla.delta_attention(*x.values(), seq_lens=c.seq_lens, state=s0, out=out, return_state=keep)
    o, S = R.delta(*c.x.values(), c.lens, s0, c.D ** -0.5)
    past = c.past()
    assert (out[past] == 7.0).all(), "padding rows were written"
    close(out[~past], o[~past], bound(c.dtype, c.N, c.D), "o")
    if keep:
        assert got[0] is out
        close(got[1], S, bound("fp32", c.N, c.D), "state")
    again = torch.full_like(out, 7.0)
    gbla.delta_attention(*c.x.values(), seq_lens=c.seq_lens, state=s0, out=again, return_state=keep)
    assert torch.equal(out, again)
    assert gbla.device_error() == 0


@pytest.mark.parametrize("ends", ["none", "dstate", "both"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_backward(i, ends):
    """ends: which of the last state's gradient (in) and the first one's (out) there are."""
    c, s0 = _case(i)
    do = c.n(*c.x["v"].shape).to(TYPES[c.dtype]).cuda()
    ds = c.n(c.B, c.H, c.D, c.D).cuda() if ends != "none" else None
    past = c.past()
    bad = do.clone()
    bad[past] = float("nan")
    kw = dict(seq_lens=c.seq_lens, state=s0, dstate=ds, return_dstate=ends == "both")
    got = gbla.delta_attention_backward(*c.poisoned().values(), bad, **kw)
    ref = R.delta_backward(*c.x.values(), do, c.lens, s0, ds, c.D ** -0.5)
    assert got.keys() == {"dq", "dk", "dv", "dlog_decay", "dbeta"} | ({"dstate"} if ends == "both" else set())
    for n, g in got.items():
        r = ref[n]
        if n == "dlog_decay":
            r = torch.where(c.x["log_decay"] == -math.inf, torch.zeros_like(r), r)
            assert (g[c.x["log_decay"] == -math.inf] == 0).all()
        if n != "dstate":
            assert (g[past] == 0).all(), (n, "padding rows are 0")
        beside = shares(c.x, do, ref, c.lens, s0, c.D ** -0.5) if n == "dlog_decay" else None
        close(g, r, grad_bound(n, c.dtype, c.N, c.D), n, beside)
    again = gbla.delta_attention_backward(*c.x.values(), do, **kw)
    for n in got:
        assert torch.equal(got[n], again[n]), n
    assert gbla.device_error() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_strides_and_scale(dtype, D):
    """Slices of packed projections, gates of any alignment among them."""
    c = Case(7, 2, 100, 6, 2, D, dtype, [100, 71])
    B, N, H, Hk = c.B, c.N, c.H, c.Hk
    pack = torch.cat([c.x["q"].flatten(2), c.x["k"].flatten(2), c.x["v"].flatten(2)], 2)
    gates = torch.cat([c.x["log_decay"], c.x["beta"], c.x["beta"][..., :1]], 2)
    q = pack[..., :Hk * D].unflatten(2, (Hk, D))
    k = pack[..., Hk * D:2 * Hk * D].unflatten(2, (Hk, D))
    v = pack[..., 2 * Hk * D:].unflatten(2, (H, D))
    g, b = gates[..., :H], gates[..., H:2 * H]
    assert not q.is_contiguous() and not g.is_contiguous()
    got, S = gbla.delta_attention(q, k, v, g, b, c.seq_lens, scale=-0.3, return_state=True)
    o, ref = R.delta(*c.x.values(), c.lens, None, -0.3)
    past = c.past()
    close(got[~past], o[~past], bound(dtype, N, D), "o")
    close(S, ref, bound("fp32", N, D), "state")
    do = c.n(B, N, H, D).to(TYPES[dtype]).cuda()
    grads = gbla.delta_attention_backward(q, k, v, g, b, do, c.seq_lens, scale=-0.3)
    want = R.delta_backward(*c.x.values(), do, c.lens, None, None, -0.3)
    for n, t in grads.items():
        beside = shares(c.x, do, want, c.lens, None, -0.3) if n == "dlog_decay" else None
        close(t, want[n], grad_bound(n, dtype, N, D), n, beside)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_chosen_splits_continue_one_another(dtype):
    """A sequence in pieces through states equals the sequence at once, whatever the cuts."""
    c = Case(8, 1, 300, 4, 4, 64, dtype)
    whole, S = gbla.delta_attention(*c.x.values(), return_state=True)
    for cuts in ([0, 1, 300], [0, 64, 128, 300], [0, 37, 38, 101, 300]):
        s, parts = None, []
        for a, b in zip(cuts, cuts[1:]):
            o, s = gbla.delta_attention(*[t[:, a:b] for t in c.x.values()], state=s, return_state=True)
            parts.append(o)
        close(torch.cat(parts, 1), whole.double(), 2 * bound(dtype, 300, 64), "o")
        close(s, S.double(), 2 * bound("fp32", 300, 64), "state")


@pytest.mark.parametrize("how", ["repeated", "opposite", "zero beta", "beta two", "zeros", "far"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_extreme_keys_and_gates(dtype, how):
    """The same key again and again, its opposite, nothing written, reflections, far fades."""
    c = Case(9, 1, 150, 2, 2, 64, dtype)
    x = c.x
    if how in ("repeated", "opposite"):
        x["k"] = x["k"][:, :1].expand_as(x["k"]).contiguous()
        x["beta"] = torch.ones_like(x["beta"])
        if how == "opposite":
            x["k"][:, ::2] *= -1
    elif how == "zero beta":
        x["beta"] = torch.zeros_like(x["beta"])
    elif how == "beta two":
        x["beta"] = torch.full_like(x["beta"], 1.99)
    elif how == "zeros":
        x["k"] = torch.zeros_like(x["k"])
    else:
        x["log_decay"] = torch.full_like(x["log_decay"], -60.0)
    s0 = c.state()
    o, S = R.delta(*x.values(), c.lens, s0, 0.125)
    got, fin = gbla.delta_attention(*x.values(), state=s0, return_state=True)
    # reflections keep the state's size while single values nearly cancel: 8 times the bound
    many = 8 if how == "beta two" else 1
    close(got, o, many * bound(dtype, 150, 64), "o")
    close(fin, S, many * bound("fp32", 150, 64), "state")
    do, ds = c.n(1, 150, 2, 64).to(TYPES[dtype]).cuda(), c.state()
    g = gbla.delta_attention_backward(*x.values(), do, state=s0, dstate=ds, scale=0.125, return_dstate=True)
    want = R.delta_backward(*x.values(), do, c.lens, s0, ds, 0.125)
    for n, t in g.items():
        beside = shares(x, do, want, c.lens, s0, 0.125) if n == "dlog_decay" else None
        close(t, want[n], many * grad_bound(n, dtype, 150, 64), n, beside)


def test_long_sequences():
    """Every D, 4000 tokens (weak fades among them), against the recurrence on the GPU."""
    for D, dtype in ((32, "bf16"), (64, "fp32"), (64, "bf16"), (128, "bf16"), (128, "fp32")):
        c = Case(10 + D, 1, 4001, 2, 1, D, dtype)
        c.x["log_decay"][..., 1] = -1e-4
        o, S = R.delta(*c.x.values(), c.lens, None, D ** -0.5)
        got, fin = gbla.delta_attention(*c.x.values(), return_state=True)
        close(got, o, bound(dtype, 4001, D), (D, dtype, "o"))
        close(fin, S, bound("fp32", 4001, D), (D, dtype, "state"))
        do = c.n(1, 4001, 2, D).to(TYPES[dtype]).cuda()
        g = gbla.delta_attention_backward(*c.x.values(), do)
        want = R.delta_backward(*c.x.values(), do, c.lens, None, None, D ** -0.5)
        for n, t in g.items():
            beside = shares(c.x, do, want, c.lens, None, D ** -0.5) if n == "dlog_decay" else None
            close(t, want[n], grad_bound(n, dtype, 4001, D), (D, dtype, n), beside)


@pytest.mark.parametrize("D,dtype", [(32, "bf16"), (64, "bf16"), (64, "fp32"), (128, "bf16"), (128, "fp32")])
def test_segments_of_ragged_sequences(D, dtype):
    """Long enough to be cut into segments: sequences that end in the first, in the middle of
    one, at a border, nowhere (empty), with states in and out and memories that end."""
    lens = [2600, 0, 1300, 64, 2599, 2560]
    c = Case(40 + D, 6, 2600, 2, 1, D, dtype, lens, packed=False)
    c.x["log_decay"][:, ::700] = -math.inf
    s0 = c.state()
    out = torch.full_like(c.x["v"], 7.0)
    x = c.poisoned()
    _, S = gbla.delta_attention(*x.values(), seq_lens=c.seq_lens, state=s0, out=out, return_state=True)
    o, ref = R.delta(*c.x.values(), c.lens, s0, D ** -0.5)
    past = c.past()
    assert (out[past] == 7.0).all()
    close(out[~past], o[~past], bound(dtype, 2600, D), "o")
    close(S, ref, bound("fp32", 2600, D), "state")
    alone = gbla.delta_attention(*x.values(), seq_lens=c.seq_lens, state=s0)
    close(alone[~past], o[~past], bound(dtype, 2600, D), "o without a state")
    do, ds = c.n(*o.shape).to(TYPES[dtype]).cuda(), c.state()
    want = R.delta_backward(*c.x.values(), do, c.lens, s0, ds, D ** -0.5)
    g = gbla.delta_attention_backward(*x.values(), do, seq_lens=c.seq_lens, state=s0, dstate=ds, return_dstate=True)
    for n, t in g.items():
        r = want[n]
        if n == "dlog_decay":
            r = torch.where(c.x["log_decay"] == -math.inf, 0.0, r)
        beside = shares(c.x, do, want, c.lens, s0, D ** -0.5) if n == "dlog_decay" else None
        close(t, r, grad_bound(n, dtype, 2600, D), n, beside)
    assert gbla.device_error() == 0


def test_far_offsets():
    """Rows of a batch more than 2^32 elements apart."""
    c = Case(50, 2, 70, 2, 2, 64, "bf16")
    far = torch.empty_strided((2, 70, 2, 64), ((1 << 32) + 64, 128, 64, 1), dtype=torch.bfloat16, device="cuda")
    far.copy_(c.x["v"])
    want = gbla.delta_attention(*c.x.values())
    x = {**c.x, "v": far}
    assert torch.equal(gbla.delta_attention(*x.values()), want)
    do = c.n(2, 70, 2, 64).to(torch.bfloat16).cuda()
    a, b = (gbla.delta_attention_backward(*t.values(), do) for t in (c.x, x))
    assert all(torch.equal(a[n], b[n]) for n in a)


STEPS = [(1, 1, 1, 32, "fp32"), (4, 8, 8, 64, "bf16"), (5, 6, 2, 128, "bf16"), (7, 4, 1, 64, "fp32"),
         (3, 3, 3, 128, "fp32"), (6, 8, 2, 32, "bf16")]


@pytest.mark.parametrize("B,H,Hk,D,dtype", STEPS)
def test_step(B, H, Hk, D, dtype):
    """On a pool, rows without a sequence and slots nobody names left alone; strided inputs."""
    c = Case(11, B, 3, H, Hk, D, dtype)
    one = {n: t[:, 1:2] for n, t in c.x.items()}  # strided
    n = B + 3
    pool = (0.5 * c.n(n, H, D, D)).cuda()
    before = pool.clone()
    slots = torch.randperm(n, generator=c.g)[:B].to(torch.int32)
    bad = [0] if B > 2 else []
    live = [b for b in range(B) if b not in bad]
    at = slots.clone()
    at[bad] = torch.tensor([-1], dtype=torch.int32) if bad else at[bad]
    out = torch.full((B, 1, H, D), 7.0, dtype=TYPES[dtype], device="cuda")
    gbla.delta_attention_step(*one.values(), pool, slots=at.cuda(), out=out)
    o, S = R.delta(*one.values(), [1] * B, before[slots.long().cuda()], D ** -0.5)
    close(out[live], o[live], bound(dtype, 1, D), "o")
    close(pool[slots[live].long().cuda()], S[live], bound("fp32", 1, D), "state")
    assert (out[bad] == 7.0).all()
    rest = [i for i in range(n) if i not in slots[live].tolist()]
    assert torch.equal(pool[rest], before[rest])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_steps_continue_a_prompt(dtype):
    c = Case(12, 3, 90, 4, 2, 64, dtype, packed=True)
    whole, S = gbla.delta_attention(*c.x.values(), return_state=True)
    _, state = gbla.delta_attention(*[t[:, :70] for t in c.x.values()], return_state=True)
    got = torch.cat([gbla.delta_attention_step(*[t[:, i:i + 1] for t in c.x.values()], state)
                     for i in range(70, 90)], 1)
    close(got, whole[:, 70:].double(), 2 * bound(dtype, 90, 64), "o")
    close(state, S.double(), 2 * bound("fp32", 90, 64), "state")


def test_nothing_to_do_and_empty_sequences():
    c = Case(13, 2, 5, 2, 2, 64, "bf16", [0, 0])
    s0 = c.state()
    out = torch.full_like(c.x["v"], 7.0)
    _, S = gbla.delta_attention(*c.x.values(), seq_lens=c.seq_lens, state=s0, out=out, return_state=True)
    assert torch.equal(S, s0) and (out == 7.0).all()
    none = {n: t[:, :0] for n, t in c.x.items()}
    o, S = gbla.delta_attention(*none.values(), state=s0, return_state=True)
    assert o.shape == (2, 0, 2, 64) and torch.equal(S, s0)
    _, S = gbla.delta_attention(*none.values(), return_state=True)
    assert (S == 0).all()
    for x in (c.x, none):  # no tokens: the state's gradient passes through
        g = gbla.delta_attention_backward(*x.values(), x["v"], dstate=s0, return_dstate=True,
                                          seq_lens=c.seq_lens)
        assert torch.equal(g["dstate"], s0) and all((g[n] == 0).all() for n in g if n != "dstate")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_another_stream_and_a_graph(dtype):
    c = Case(14, 2, 200, 4, 4, 64, dtype)
    ref, S = gbla.delta_attention(*c.x.values(), return_state=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, fin = gbla.delta_attention(*c.x.values(), return_state=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, ref) and torch.equal(fin, S)
    graphs = []
    do = c.n(*ref.shape).to(ref.dtype).cuda()
    dref = gbla.delta_attention_backward(*c.x.values(), do)
    for _ in range(2):  # two graphs of the same calls, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o, s = gbla.delta_attention(*c.x.values(), return_state=True)
            one = gbla.delta_attention_step(*[t[:, -1:] for t in c.x.values()], s)
            d = gbla.delta_attention_backward(*c.x.values(), do)
        graphs.append((graph, o, s, one, d))
    want = S.clone()
    last = gbla.delta_attention_step(*[t[:, -1:] for t in c.x.values()], want)
    for _ in range(3):
        for graph, o, s, one, d in graphs:
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(d[n], dref[n]) for n in d)
            assert torch.equal(o, ref) and torch.equal(s, want) and torch.equal(one, last)
