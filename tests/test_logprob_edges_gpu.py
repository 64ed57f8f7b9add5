"""Token log probabilities at the ends of what the types hold, and the launch shapes that few
sizes take.  Bounds: those of test_logprob_gpu.py."""
import math

import pytest
import torch

import delta_ref as R
from paper_2606_07317_gb300 import gbla
from test_logprob_gpu import TYPES, check, rows

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
