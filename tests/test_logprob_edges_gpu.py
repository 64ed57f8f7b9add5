"""Token log probabilities at the ends of what the types hold, and the launch shapes that few
sizes take.  Bounds: those of test_logprob_gpu.py."""
import math

import pytest
import torch

import delta_ref as R
from paper_2606_07317_gb300 import gbla
from test_logprob_gpu import TYPES, check, grads, rows

pytestmark = pytest.mark.gpu


def large(dtype, V, top):
    """Rows whose largest logit is `top`, at the first, a middle and the last place, beside
    ordinary logits, the type's lowest ones, -inf, and one half as large."""
    low = torch.finfo(TYPES[dtype]).min
    x = torch.randn((1, 8, V), generator=torch.Generator().manual_seed(V)) * 3
    x[0, 0, 0] = x[0, 1, V // 2] = x[0, 2, V - 1] = top
    x[0, 3] = low
    x[0, 3, V // 3] = top
    x[0, 4] = -math.inf
    x[0, 4, V // 3] = top
    x[0, 5, 1], x[0, 5, V - 2] = top, top / 2
    x[0, 6, ::2] = -top
    x[0, 6, 2] = top
    x[0, 7, 3] = top
    x[0, 7, 4:] = -math.inf
    tok = torch.tensor([[0, 1, V - 1, 0, 1, V - 2, 2, 0]], dtype=torch.int32)
    return x.to(TYPES[dtype]).cuda(), tok.cuda()


# the largest logit, the scale: their product passes fp32's range in the last two
SIZES = [(3.3e38, 1.0), (2.4e38, 1.0), (1.5e38, 2.0), (3e36, 100.0), (3e35, 1000.0), (3e38, 0.25), (1e30, 1e8),
         (3.3e38, 100.0), (3e38, 2.0 ** 20)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [8, 300, 5000, 70001])
@pytest.mark.parametrize("top,scale", SIZES)
def test_large_logits(dtype, V, top, scale):
    """Finite logits have finite entropies, whatever their size; what passes fp32's range is
    infinite."""
    x, tok = large(dtype, V, top)
    n = min(V, 5)
    got = gbla.token_logprobs(x, tok, top=n, scale=scale)
    ref = R.logprobs(x, tok, n, scale)
    check(got, {m: r if m == "top_token" else r.float().double() for m, r in ref.items()})
    assert torch.isfinite(got["entropy"]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_does_not_read_an_unused_entropy(dtype):
    x, tok, _ = rows(70, 2, 3, 900, dtype)
    f = gbla.token_logprobs(x, tok)
    one, nothing = torch.ones((2, 3)).cuda(), torch.zeros((2, 3)).cuda()
    bad = torch.full_like(one, math.nan)
    want = gbla.token_logprobs_backward(x, f["lse"], f["entropy"], tok, one)
    for h in (None, nothing):
        assert torch.equal(gbla.token_logprobs_backward(x, f["lse"], bad, tok, one, h), want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [8, 300, 5000, 70001])
@pytest.mark.parametrize("top,scale", SIZES)
def test_gradients_of_large_logits(dtype, V, top, scale):
    x, tok = large(dtype, V, top)
    f = gbla.token_logprobs(x, tok, scale=scale)
    g = torch.Generator().manual_seed(1)
    d = [torch.randn((1, 8), generator=g).cuda() for _ in range(3)]
    for which in ([0], [1], [2], [0, 1, 2]):
        args = [t if i in which else None for i, t in enumerate(d)]
        got = gbla.token_logprobs_backward(x, f["lse"], f["entropy"], tok, *args, scale=scale)
        want, mag = R.logprobs_backward(x, tok, scale, *args)
        assert torch.isfinite(got).all(), which
        # a probability is 0 or 1 here (the next logit is farther away than any exponent): no share
        # of lse and logit in the room
        on = [r for r in range(8) if r != 5 or top * scale < 3.4e38]  # two beyond the range
        grads(got[:, on], want[:, on], mag[:, on], torch.zeros_like(x[:, on]), dtype, scale)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [8, 5000])
def test_gradients_of_shared_largest_logits(dtype, V):
    """Three equal logits beyond fp32's range when scaled: a third of the probability each."""
    x = torch.zeros((1, 1, V), dtype=TYPES[dtype], device="cuda")
    x[0, 0, [1, 3, V - 2]] = 2e38
    tok = torch.tensor([[3]], dtype=torch.int32, device="cuda")
    f = gbla.token_logprobs(x, tok, scale=16.0)
    one = torch.ones((1, 1), device="cuda")
    got = gbla.token_logprobs_backward(x, f["lse"], f["entropy"], tok, one, 0.5 * one, 0.25 * one, scale=16.0)
    # p = 1/3, ln p + entropy = 0 (in closed form: 64 bits cannot hold ln 3 beside 3.2e39)
    want = torch.zeros((1, 1, V), dtype=torch.float64, device="cuda")
    want[0, 0, [1, 3, V - 2]] = 16 / 3 * (0.25 - 1)
    want[0, 0, 3] += 16
    # the probability by way of the entropy's bound, 24 times 640 u, in place of the exponent's;
    # magnitudes of the terms: at most 16 (1 + 1 + 0.5 * 3 + 0.25)
    room = (24 * 640 + 96) * 2.0 ** -24 * 60 + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0)
    assert ((got.double() - want).abs() <= room).all()
    assert (got[want == 0] == 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows_", [3, 400])
@pytest.mark.parametrize("V", [20, 300, 1021, 5000, 70000])
def test_top_tokens_beside_nan(dtype, rows_, V):
    """NaN counts as the least: what else a thread, a vector or a row holds keeps its order."""
    g = torch.Generator().manual_seed(V)
    x = torch.randn((1, rows_, V), generator=g)
    x[torch.rand(x.shape, generator=g) < 0.05] = -math.inf
    at = torch.randint(0, V, (rows_, 5), generator=g)
    for r in range(rows_):
        x[0, r, at[r, 0]] = 90.0 + r % 3            # the largest, then a NaN near it
        x[0, r, (at[r, 0] + 1) % V] = math.nan
        x[0, r, at[r, 1:3]] = math.nan
    x[0, 0, : V // 2] = math.nan
    x[0, 1] = math.nan
    x[0, 1, V - 3] = -math.inf
    x = x.to(TYPES[dtype]).cuda()
    top = min(V, 12)
    order = torch.where(x.isnan(), -math.inf, torch.where(x == -math.inf, -1e300, x.double()))
    want = order.sort(dim=-1, descending=True, stable=True).indices[..., :top]
    got = gbla.token_logprobs(x, top=top)
    assert torch.equal(got["top_token"].long(), want)
    bad = x.isnan().any(-1)
    assert got["lse"][bad].isnan().all() and got["entropy"][bad].isnan().all() and got["top_logprob"][bad].isnan().all()


@pytest.mark.parametrize("B,N,V,dtype,top", [(31, 10, 131087, "bf16", 0), (1, 306, 65603, "fp32", 9),
                                            (2, 160, 140003, "bf16", 64)])
def test_long_rows_with_a_block_each(B, N, V, dtype, top):
    x, tok, _ = rows(71, B, N, V, dtype, 0.1)
    got = gbla.token_logprobs(x, tok, top=top)
    check(got, R.logprobs(x, tok, top, 1.0))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [37, 900, 9001])
def test_far_rows_of_any_place(dtype, V):
    """Logits around 3e4 in rows of a wider tensor, at every place of a vector, ragged, and over
    the logits themselves: to the bit what contiguous ones give; and the definition's."""
    x, tok, g = rows(72, 2, 3, V, dtype)
    x = x + 3e4
    lens = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    d = [torch.randn((2, 3), generator=g).cuda() for _ in range(3)]
    f = gbla.token_logprobs(x, tok)
    want = gbla.token_logprobs_backward(x, f["lse"], f["entropy"], tok, *d, seq_lens=lens)
    ref, mag = R.logprobs_backward(x, tok, 1.0, *d)
    live = torch.arange(3, device="cuda")[None] < lens[:, None]
    grads(want[live], ref[live], mag[live], x[live], dtype)
    assert (want[~live] == 0).all()
    wide = torch.zeros((2, 4, V + 9), dtype=x.dtype, device="cuda")
    for off in range(9):
        view = wide[:, :3, off:off + V]
        view.copy_(x)
        got = gbla.token_logprobs_backward(view, f["lse"], f["entropy"], tok, *d, seq_lens=lens)
        assert torch.equal(got, want), off
    over = x.clone()
    assert torch.equal(gbla.token_logprobs_backward(over, f["lse"], f["entropy"], tok, *d, seq_lens=lens, out=over),
                       want)
