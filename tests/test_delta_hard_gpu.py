"""The gated delta rule where rounding inside counts: keys that are alike, opposite or have a
common part, with beta up to the end of its range, in every form (with and without states and
their gradients), whole and cut into segments; and sizes that take each branch of the launches.

Bounds: those of test_delta_gpu.py.  What is different here is the triangular inverse: for keys
that are alike and beta near 2 its entries, and those of the matrix it is the inverse of, are near
2 and of either sign.  A block of 32 x 32 of it is two products of 32 terms, of sizes 2 * 2 and of
what the first one is off by times 2, with errors that add like independent ones: off by
4 sqrt(32) * 2 sqrt(32) = 256 times what an operand is, 2^-22 in three terms (or 2^-24 in fp32, four
roundings).  What it makes of the 64 misses of a chunk, which the state makes nearly equal, is off
by sqrt(64) times that: 2^11 2^-22 = 2^-11 of the state, whatever the type.  Results are off by that
and by the products of scores and writes, sums of 64 terms of either sign whose sizes are twice the
state's: 2 sqrt(64) * 3 * 2^-16 < 2^-10 with operands of two bf16 numbers (2^-16 each, 2^-16 for the
product of the small parts).  Together 3 * 2^-11, the share of bound() beside the result's own
rounding, and twice it for gradients, with twice the products in a row."""
import pytest
import torch

import delta_ref as R
from paper_2606_07317_gb300 import gbla
from test_delta_gpu import TYPES, Case, bound, close, grad_bound, shares

pytestmark = pytest.mark.gpu
STATE = 2.0 ** -11


def hard(c, keys, beta):
    """Keys of unit length that are one key, its opposite in turn, or have that cosine with it."""
    x, k = c.x, c.x["k"].float()
    one = k[:, :1]
    if keys == "same":
        k = one.expand_as(k).clone()
    elif keys == "opposite":
        k = one.expand_as(k).clone()
        k[:, ::2] *= -1
    else:
        k = k - (k * one).sum(-1, keepdim=True) * one
        k = keys ** 0.5 * one + (1 - keys) ** 0.5 * k / k.norm(dim=-1, keepdim=True)
    x["k"] = (k / k.norm(dim=-1, keepdim=True)).to(TYPES[c.dtype]).contiguous()
    x["beta"] = torch.full_like(x["beta"], beta)
    x["log_decay"] = torch.full_like(x["log_decay"], -1e-4)
    x["log_decay"][:, :, 1::2] = 0


def close_state(got, ref, what):
    """Norm, and elements: with one key all along a state is k s^T, an element's error that of s_e
    times k_d, each the largest of 20000 normal ones, 4.3 of their root mean square; heads differ by
    2 (how long they remember: 64 tokens to the whole 260 of the case with many heads):
    4.3 * 4.3 * 2 < 40."""
    d, ref = got.double() - ref, ref.double()
    assert d.norm() <= STATE * ref.norm(), (what, (d.norm() / ref.norm()).item())
    assert d.abs().max() <= 40 * STATE * ref.norm() / ref.numel() ** 0.5, what


SHAPES = {"segments": (1, 1024, 2), "whole": (2, 260, 80), "odd": (3, 333, 6)}
KEYS = [("same", 1.0), ("same", 1.5), ("same", 1.99), ("opposite", 1.99), (0.9, 1.0), (0.9, 1.99), (0.5, 1.99)]
# every D with every shape, and with the hardest keys
HARD = [(s, *k, (32, 64, 128)[(i + j) % 3]) for i, s in enumerate(SHAPES) for j, k in enumerate(KEYS)]


@pytest.mark.parametrize("shape,keys,beta,D", HARD)
def test_forward(shape, keys, beta, D):
    c = Case(60, *SHAPES[shape], SHAPES[shape][2], D, "bf16")
    hard(c, keys, beta)
    o, S = R.delta(*c.x.values(), c.lens, None, D ** -0.5)
    alone = gbla.delta_attention(*c.x.values())
    got, fin = gbla.delta_attention(*c.x.values(), return_state=True)
    close(alone, o, bound("bf16", c.N, D), "o alone")
    close(got, o, bound("bf16", c.N, D), "o")
    close_state(fin, S, "state")


@pytest.mark.parametrize("shape,keys,beta,D", HARD)
def test_backward(shape, keys, beta, D):
    c = Case(61, *SHAPES[shape], SHAPES[shape][2], D, "bf16")
    hard(c, keys, beta)
    do, ds = c.n(*c.x["v"].shape).to(torch.bfloat16).cuda(), c.state()
    for ends in (False, True):
        want = R.delta_backward(*c.x.values(), do, c.lens, None, ds if ends else None, D ** -0.5)
        g = gbla.delta_attention_backward(*c.x.values(), do, dstate=ds if ends else None, return_dstate=ends)
        for n, t in g.items():
            beside = shares(c.x, do, want, c.lens, None, D ** -0.5) if n == "dlog_decay" else None
            if n == "dstate":
                close_state(t, want[n], n)
            else:
                close(t, want[n], grad_bound(n, "bf16", c.N, D), (n, ends), beside)


@pytest.mark.parametrize("keys,D", [("same", 64), ("opposite", 128), ("same", 32)])
def test_fp32(keys, D):
    """What the inverse is off by is all there is: 2^-11, and twice it for gradients."""
    c = Case(64, 3, 333, 6, 6, D, "fp32")
    hard(c, keys, 1.99)
    do, ds = c.n(*c.x["v"].shape).cuda(), c.state()
    o, S = R.delta(*c.x.values(), c.lens, None, D ** -0.5)
    got, fin = gbla.delta_attention(*c.x.values(), return_state=True)
    close(got, o, STATE, "o")
    close_state(fin, S, "state")
    want = R.delta_backward(*c.x.values(), do, c.lens, None, ds, D ** -0.5)
    for n, t in gbla.delta_attention_backward(*c.x.values(), do, dstate=ds, return_dstate=True).items():
        beside = shares(c.x, do, want, c.lens, None, D ** -0.5) if n == "dlog_decay" else None
        close(t, want[n], 2 * STATE, n, beside)


@pytest.mark.parametrize("keys,D", [("same", 64), (0.9, 128), (0.0, 64)])
def test_long(keys, D):
    """Where errors of the state would add up: 4096 tokens, reflections, hardly any fading."""
    c = Case(62, 1, 4096, 2, 1, D, "bf16")
    if keys:
        hard(c, keys, 1.99)
    else:
        c.x["beta"], c.x["log_decay"] = torch.full_like(c.x["beta"], 1.99), torch.full_like(c.x["beta"], -1e-4)
    do = c.n(*c.x["v"].shape).to(torch.bfloat16).cuda()
    o, _ = R.delta(*c.x.values(), c.lens, None, D ** -0.5)
    close(gbla.delta_attention(*c.x.values()), o, bound("bf16", 4096, D), "o")
    want = R.delta_backward(*c.x.values(), do, c.lens, None, None, D ** -0.5)
    for n, t in gbla.delta_attention_backward(*c.x.values(), do).items():
        beside = shares(c.x, do, want, c.lens, None, D ** -0.5) if n == "dlog_decay" else None
        close(t, want[n], grad_bound(n, "bf16", 4096, D), n, beside)


@pytest.mark.parametrize("B,N,H,D,dtype", [(40, 1000, 16, 32, "bf16"), (300, 70, 1, 64, "bf16"), (300, 70, 1, 32, "fp32")])
def test_large_ragged_batches(B, N, H, D, dtype):
    """Several chunks a block of the preparation (9728 chunks and more), and more sequences
    than are put in order of their lengths; empty ones among them."""
    g = torch.Generator().manual_seed(5)
    lens = torch.randint(0, N + 1, (B,), generator=g)
    lens[0], lens[1], lens[2] = N, 0, 1
    c = Case(63, B, N, H, H, D, dtype, lens.tolist())
    do, past = c.n(B, N, H, D).to(TYPES[dtype]).cuda(), c.past()
    out = torch.full_like(c.x["v"], 7.0)
    gbla.delta_attention(*c.poisoned().values(), seq_lens=c.seq_lens, out=out)
    o, _ = R.delta(*c.x.values(), c.lens, None, D ** -0.5)
    assert (out[past] == 7.0).all()
    close(out[~past], o[~past], bound(dtype, N, D), "o")
    want = R.delta_backward(*c.x.values(), do, c.lens, None, None, D ** -0.5)
    for n, t in gbla.delta_attention_backward(*c.poisoned().values(), do, seq_lens=c.seq_lens).items():
        assert (t[past] == 0).all(), n
        beside = shares(c.x, do, want, c.lens, None, D ** -0.5) if n == "dlog_decay" else None
        close(t, want[n], grad_bound(n, dtype, N, D), n, beside)
    assert gbla.device_error() == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("what", ["q", "k", "v", "log_decay", "beta"])
def test_nan_is_not_hidden(what, dtype):
    """A NaN in token 70 is in its result and, but for a query's, in all that follow; chunks before
    it have none."""
    c = Case(65, 1, 200, 2, 2, 64, dtype)
    c.x[what][0, 70] = float("nan")
    do = torch.ones_like(c.x["v"])
    for keep in (False, True):
        o = gbla.delta_attention(*c.x.values(), return_state=keep)
        o, S = o if keep else (o, None)
        assert torch.isfinite(o[0, :64]).all() and o[0, 70].isnan().all()
        assert what == "q" or (o[0, 71:].isnan().all() and (S is None or S.isnan().all()))
        g = gbla.delta_attention_backward(*c.x.values(), do, return_dstate=keep)
        # (results are linear in q and in v: their own gradients do not depend on them)
        assert g["dk" if what == "q" else "dq"][0, 70].isnan().all()
