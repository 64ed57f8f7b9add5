"""GPU parity of the token log probabilities, against the 64-bit definitions of delta_ref.py.

Bounds, with u = 2^-24 and y = scale x: an exponent (x - m) scale log2 e carries three roundings
of itself and its exponential two ulp, so a probability is off by (3 |t| + 4) u of itself, where
terms with |t| > 24 weigh nothing: 80 u at most.  The normaliser's logarithm, summed over V terms
of one sign by threads (errors of the partial sums add like independent ones: at most
sqrt(V) u <= 512 u): |lse|, |log p| within 640 u + 4 u |value|; the entropy, whose terms are the
same times |t| <= 24 and sum up to ln V + ...: 24 times that.  Gradients: 96 u of the terms'
magnitudes (the exponent there is y - lse with |lse| u beside it: 4 (|lse| + |y|) u more), and
half a bf16 ulp.  Top tokens are equal."""
import math

import pytest
import torch

import delta_ref as R
from paper_2606_07317_gb300 import gbla

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def near(got, ref, room, what):
    got, ref = got.double(), ref.to(got.device)
    same = (got == ref) | (got.isnan() & ref.isnan())
    d = torch.where(same, torch.zeros_like(ref), (got - ref).abs())
    assert (d <= room).all(), (what, d.max().item())


def check(got, ref):
    for n, r in ref.items():
        if n == "top_token":
            assert got[n].dtype == torch.int32
            assert torch.equal(got[n].cpu(), r.cpu()), n
            continue
        room = 640 * U + 4 * U * torch.where(r.isfinite(), r.abs(), torch.zeros_like(r))
        near(got[n], r, room * (24 if n == "entropy" else 1), n)


def rows(seed, B, N, V, dtype, masked=0.0, std=3.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, N, V), generator=g) * std
    if masked:
        x[torch.rand((B, N, V), generator=g) < masked] = -math.inf
    tok = torch.randint(-2, V + 2, (B, N), generator=g).to(torch.int32)
    return x.to(TYPES[dtype]).cuda(), tok.cuda(), g


CASES = [  # B, N, V, dtype, top, masked, scale
    (1, 1, 1, "fp32", 1, 0, 1.0), (1, 3, 2, "bf16", 2, 0, 2.0), (2, 5, 7, "bf16", 7, 0.5, 1.0),
    (1, 2, 64, "fp32", 64, 0, 1.0), (3, 4, 63, "bf16", 33, 0.9, 0.5), (2, 3, 255, "fp32", 5, 0, 1.0),
    (2, 9, 1021, "bf16", 64, 0.97, 1.0), (1, 2, 2048, "bf16", 8, 0, 1.25), (1, 300, 513, "fp32", 0, 0.2, 1.0),
    (1, 4, 65536, "bf16", 8, 0, 1.0), (1, 2, 100003, "fp32", 64, 0.5, 0.7), (2, 700, 4097, "bf16", 32, 0, 1.0),
    (1, 1, 200001, "bf16", 1, 0, 1.0), (40, 1, 40000, "fp32", 64, 0.99, 1.0), (1, 3, 12289, "bf16", 0, 0, 1.0),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward(i):
    B, N, V, dtype, top, masked, scale = CASES[i]
    x, tok, _ = rows(i, B, N, V, dtype, masked)
    ref = R.logprobs(x, tok, top, scale)
    got = gbla.token_logprobs(x, tok, top=top, scale=scale)
    check(got, ref)
    again = gbla.token_logprobs(x, tok, top=top, scale=scale)
    for n in got:
        assert torch.equal(got[n], again[n]), n
    alone = gbla.token_logprobs(x, scale=scale)
    assert alone.keys() == {"lse", "entropy"} and torch.equal(alone["lse"], got["lse"])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_padding_strides_and_alignment(dtype):
    """Rows past the lengths are left alone and may hold NaN; rows begin at any place."""
    x, tok, _ = rows(20, 3, 6, 333, dtype)
    lens = torch.tensor([6, 0, 2], dtype=torch.int32).cuda()
    past = torch.arange(6).cuda()[None] >= lens[:, None]
    wide = torch.full((3, 7, 341), float("nan"), dtype=x.dtype, device="cuda")
    for off in range(9):
        view = wide[:, :6, off:off + 333]
        view.copy_(torch.where(past[..., None], torch.full_like(x, float("nan")), x))
        out = {"lse": torch.full((3, 6), 7.0).cuda(), "entropy": torch.full((3, 6), 7.0).cuda(),
               "logprob": torch.full((3, 6), 7.0).cuda(), "top_logprob": torch.full((3, 6, 5), 7.0).cuda(),
               "top_token": torch.full((3, 6, 5), 7, dtype=torch.int32).cuda()}
        got = gbla.token_logprobs(view, tok, top=5, seq_lens=lens, out=out)
        assert got is out
        check({n: t[~past] for n, t in out.items()},
              {n: t[~past] for n, t in R.logprobs(x, tok, 5, 1.0).items()})
        assert all((t[past] == 7).all() for t in out.values())
        d = gbla.token_logprobs_backward(view, out["lse"], out["entropy"], tok, dlogprob=torch.ones_like(out["lse"]),
                                         seq_lens=lens)
        assert (d[past] == 0).all() and torch.isfinite(d).all()
        ref, mag = R.logprobs_backward(x, tok, 1.0, torch.ones((3, 6)).cuda(), None, None)
        grads(d[~past], ref[~past], mag[~past], x[~past], dtype)


def grads(got, ref, mag, x, dtype, scale=1.0):
    y = torch.where(x.isfinite(), x.double() * scale, 0.0)
    room = (96 * U + 4 * U * (y.abs() + y.abs().amax(-1, keepdim=True) + 16)) * mag
    # a probability below 2^-126 is flushed to 0, with up to 2^-126 (|dlogprob| + |dlse| +
    # |dentropy| (|ln p| + entropy)) < 2^-126 * 4 (2 + 104 + 13) < 2^-117 of the gradient
    room = room + 2.0 ** -117
    if dtype == "bf16":
        room = room + 2.0 ** -8 * ref.abs()
    near(got, ref, room, "dlogits")


@pytest.mark.parametrize("which", ["all", "dlogprob", "dentropy", "dlse", "none"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_backward(i, which):
    B, N, V, dtype, _, masked, scale = CASES[i]
    x, tok, g = rows(50 + i, B, N, V, dtype, masked)
    names = ("dlogprob", "dentropy", "dlse")
    d = {n: torch.randn((B, N), generator=g).cuda() if which in ("all", n) else None for n in names}
    f = gbla.token_logprobs(x, tok, scale=scale)
    got = gbla.token_logprobs_backward(x, f["lse"], f["entropy"], tok, **d, scale=scale)
    ref, mag = R.logprobs_backward(x, tok, scale, *d.values())
    grads(got, ref, mag, x, dtype, scale)
    over = x.clone()
    same = gbla.token_logprobs_backward(over, f["lse"], f["entropy"], tok, **d, scale=scale, out=over)
    assert same is over and torch.equal(over, got)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [5, 300, 5000, 70000])
def test_masks_and_extremes(dtype, V):
    """Empty rows, rows of the type's lowest value, single survivors, equal logits, infinities, NaN."""
    low = torch.finfo(TYPES[dtype]).min
    x = torch.full((1, 9, V), -math.inf)
    x[0, 1] = low
    x[0, 2, V - 2] = -40.0
    x[0, 3] = 1.5
    x[0, 4] = torch.linspace(-80, 80, V)
    x[0, 5] = low
    x[0, 5, 3] = 2.0
    x[0, 6] = torch.randn(V, generator=torch.Generator().manual_seed(0)) + 3e4
    x[0, 7] = 0.0
    x[0, 7, 1] = math.nan
    x[0, 8] = 0.0
    x[0, 8, 2] = math.inf
    x = x.to(TYPES[dtype]).cuda()
    tok = torch.tensor([[0, 1, V - 2, 2, V - 1, 0, 4, 0, 2]], dtype=torch.int32).cuda()
    top = min(V, 6)
    got = gbla.token_logprobs(x, tok, top=top)
    ref = R.logprobs(x, tok, top, 1.0)
    check({n: t[:, :7] for n, t in got.items()}, {n: t[:, :7] for n, t in ref.items()})
    for n, t in got.items():
        if n == "top_token":
            assert ((t >= 0) & (t < V)).all()
            assert all(len(set(r)) == top for r in t[0].tolist())
        else:
            assert t[:, 7:].isnan().all(), n
    one = torch.ones((1, 9)).cuda()
    d = gbla.token_logprobs_backward(x, got["lse"], got["entropy"], tok, one, one, one)
    assert (d[0, :2] == 0).all() and torch.isfinite(d[0, :7]).all()
    ref, mag = R.logprobs_backward(x[:, 2:6], tok[:, 2:6], 1.0, *[one[:, 2:6]] * 3)
    grads(d[:, 2:6], ref, mag, torch.where(x[:, 2:6] < -1e30, -math.inf, x[:, 2:6].float()), dtype)
    assert d[0, 7:].isnan().any(-1).all()


@pytest.mark.parametrize("order", ["ascending", "descending", "one thread's", "ties"])
@pytest.mark.parametrize("V,top", [(70000, 64), (9000, 7), (100, 64)])
def test_top_in_unkind_orders(order, V, top):
    g = torch.Generator().manual_seed(3)
    x = torch.randn((1, 3, V), generator=g).sort(-1).values
    if order == "descending":
        x = x.flip(-1)
    elif order == "one thread's":  # large logits where a stride of vectors falls
        x = torch.randn((1, 3, V), generator=g)
        x[..., torch.arange(V) // 4 % 256 == 3] += 100
    elif order == "ties":
        x = torch.randint(0, 3, (1, 3, V), generator=g).float()
    x = x.cuda()
    check(gbla.token_logprobs(x, top=top), R.logprobs(x, None, top, 1.0))


@pytest.mark.parametrize("dtype,V,top,threads", [("fp32", 9000, 40, 128), ("bf16", 9001, 9, 128), ("fp32", 600, 16, 32)])
def test_top_where_one_thread_has_them(dtype, V, top, threads):
    """Many rows, so that a block (or a warp) has a row to itself: the largest logits all where
    the vectors of one thread fall, more of them than a block keeps as candidates."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn((2, 1300, V), generator=g).sort(-1).values
    vec = 4 if dtype == "fp32" else 8
    x[..., torch.arange(V) // vec % threads == 3] += 20
    x = x.to(TYPES[dtype]).cuda()
    check(gbla.token_logprobs(x, top=top), R.logprobs(x, None, top, 1.0))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [129, 300, 517, 641, 1000, 1024, 1025])
@pytest.mark.parametrize("top", [16, 17, 32, 33, 64])
def test_top_of_short_rows(dtype, V, top):
    """Rows that a warp takes: any order, ties, masks; the other results to the bit without them."""
    x, tok, g = rows(V, 1, 9, V, dtype)
    x[0, 1] = x[0, 1].sort(dim=-1).values
    x[0, 2] = x[0, 2].sort(dim=-1, descending=True).values
    x[0, 3] = torch.randint(0, 2, (V,), generator=g).to(x)
    x[0, 4, top + 1:] = -math.inf
    x[0, 5, :-3] = -math.inf
    x[0, 6] = -math.inf
    x[0, 7] = 1.5
    x[0, 8, ::3] = math.nan
    got = gbla.token_logprobs(x, tok, top=top)
    check({n: t[:, :8] for n, t in got.items()}, R.logprobs(x[:, :8], tok[:, :8], top, 1.0))
    last = got["top_token"][0, 8].tolist()
    assert all(0 <= i < V for i in last) and len(set(last)) == top
    alone = gbla.token_logprobs(x[:, :8], tok[:, :8])
    for n in alone:
        assert torch.equal(alone[n], got[n][:, :8]), n


def test_far_rows():
    """Offsets beyond 2^32 bytes."""
    B, V = 3, 4099
    x = torch.empty_strided((B, 2, V), ((1 << 30) + 3, V + 2, 1), dtype=torch.bfloat16, device="cuda")
    small, tok, g = rows(30, B, 2, V, "bf16")
    x.copy_(small)
    check(gbla.token_logprobs(x, tok, top=9), R.logprobs(small, tok, 9, 1.0))


def test_another_stream_and_graphs():
    x, tok, g = rows(31, 2, 5, 3000, "bf16")
    d = torch.randn((2, 5), generator=g).cuda()

    def call(stream=None):
        f = gbla.token_logprobs(x, tok, top=4, stream=stream)
        return f, gbla.token_logprobs_backward(x, f["lse"], f["entropy"], tok, d, stream=stream)

    ref, dref = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, dgot = call(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(dgot, dref) and all(torch.equal(got[n], ref[n]) for n in ref)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, *call()))
    for graph, f, df in graphs * 2:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(df, dref) and all(torch.equal(f[n], ref[n]) for n in ref)


def test_nothing_to_do():
    x = torch.zeros((2, 0, 5), device="cuda")
    got = gbla.token_logprobs(x, torch.zeros((2, 0), dtype=torch.int32, device="cuda"), top=2)
    assert got["lse"].shape == (2, 0) and got["top_token"].shape == (2, 0, 2)
