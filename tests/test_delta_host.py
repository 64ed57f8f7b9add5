"""Argument checks of the gated delta rule and the token log probabilities (CPU: every call is
refused, or has nothing to do, before any GPU work)."""
import ctypes
import os

import pytest
import torch

from paper_2606_07317_gb300 import build, gbla

P = [0x10000 + i * 0x1000000 for i in range(24)]  # distinct aligned fake addresses
INV, UNS, OK = gbla.GBLA_ERR_INVALID_ARG, gbla.GBLA_ERR_UNSUPPORTED, gbla.GBLA_OK


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.LIB_PATH):
        build.build()
    return gbla.load()


DEL = dict(B=2, N=8, H=4, Hk=2, D=64, scale=0.125, dtype=1)
STEP = dict(B=2, H=4, Hk=2, D=64, n_slots=5, scale=0.125, dtype=1)
LOG = dict(B=2, N=8, V=100, top=4, scale=1.0, dtype=1)
LOGB = dict(B=2, N=8, V=100, scale=1.0, dtype=1)
OPS = {  # entry point, pointers in order, sizes, needed 16-byte aligned pointers, outputs
    "delta": ("gbla_delta_attention", "q k v log_decay beta seq_lens strides state_in o state_out", DEL, "q k v o",
              "o state_out"),
    "delta_backward": ("gbla_delta_attention_backward",
                       "q k v log_decay beta seq_lens strides state_in d_o dstate_out dq dk dv dlog_decay dbeta "
                       "dstate_in", DEL, "q k v d_o dq dk dv dlog_decay dbeta", "dq dk dv dlog_decay dbeta dstate_in"),
    "step": ("gbla_delta_attention_step", "q k v log_decay beta slots strides state o", STEP, "q k v state o", "o state"),
    "logprobs": ("gbla_token_logprobs", "logits tokens seq_lens strides lse entropy logprob top_logprob top_token", LOG,
                 "lse entropy", "lse entropy logprob top_logprob top_token"),
    "logprobs_backward": ("gbla_token_logprobs_backward",
                          "logits lse entropy tokens seq_lens strides dlogprob dentropy dlse dlogits", LOGB,
                          "lse entropy dlogits", "dlogits"),
}
DELTA = ["delta", "delta_backward", "step"]


def _run(lib, op, **kw):
    name, names, sizes, _, _ = OPS[op]
    names = names.split()
    vals = {n: P[i] for i, n in enumerate(names)}
    vals |= {"seq_lens": None, "strides": None, "slots": None} | sizes
    assert all(n in vals for n in kw), kw
    vals |= kw
    if vals["strides"] is not None:
        vals["strides"] = (ctypes.c_int64 * len(vals["strides"]))(*vals["strides"])
    return getattr(lib, name)(*[vals[n] for n in names], *[vals[n] for n in sizes], None)


@pytest.mark.parametrize("op", OPS)
def test_pointers(lib, op):
    names = OPS[op][1].split()
    for n in OPS[op][3].split():
        assert _run(lib, op, **{n: None}) == INV, n
        assert _run(lib, op, **{n: P[23] + 8}) == INV, n
    for n in ("state_in", "state_out", "dstate_in", "dstate_out", "logprob", "top_logprob", "top_token", "dlogprob",
              "dentropy", "dlse"):
        if n in names:
            assert _run(lib, op, **{n: P[23] + 4}) == INV, n
    for n in ("seq_lens", "slots", "tokens"):
        if n in names:
            assert _run(lib, op, **{n: P[23] + 2}) == INV, n
    for n in ("log_decay", "beta", "logits"):  # single values: their own alignment
        if n in names:
            assert _run(lib, op, **{n: None}) == INV and _run(lib, op, **{n: P[23] + 1}) == INV, n
            assert _run(lib, op, **{n: P[23] + 2, "dtype": 0}) == INV, n


@pytest.mark.parametrize("op", DELTA)
def test_sizes(lib, op):
    for bad in (dict(B=-1), dict(H=-4), dict(Hk=-1), dict(Hk=3), dict(Hk=0), dict(H=5), dict(B=70000), dict(H=0)):
        assert _run(lib, op, **bad) == INV, bad
    for bad in (dict(D=48), dict(D=0), dict(D=256), dict(dtype=5)):
        assert _run(lib, op, **bad) == UNS, bad
    for s in (0.0, float("nan"), float("inf"), 1e-40):
        assert _run(lib, op, scale=s) == INV, s
    if op != "step":
        assert _run(lib, op, N=-3) == INV


@pytest.mark.parametrize("op", ["logprobs", "logprobs_backward"])
def test_logit_sizes(lib, op):
    for bad in (dict(B=-1), dict(N=-1), dict(V=0), dict(V=-5), dict(V=(1 << 30) + 1), dict(B=1 << 16, N=1 << 15),
                dict(B=(1 << 15) + 1, N=1 << 15, V=1),
                dict(B=1 << 15, N=1 << 15, V=1 << 20), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(scale=1e-40)):
        assert _run(lib, op, **bad) == INV, bad
    assert _run(lib, op, dtype=7) == UNS


def test_top(lib):
    for bad in (dict(top=-1), dict(top=65), dict(V=3), dict(top=0), dict(top_token=None), dict(top_logprob=None),
                dict(logprob=None), dict(tokens=None)):
        assert _run(lib, "logprobs", **bad) == INV, bad
    assert _run(lib, "logprobs", top=0, top_token=None, top_logprob=P[20]) == INV


@pytest.mark.parametrize("op", OPS)
def test_outputs_overlap_nothing(lib, op):
    names = OPS[op][1].split()
    at = {n: P[i] for i, n in enumerate(names)}
    for o in OPS[op][4].split():
        for n in names:
            if n in ("strides", "seq_lens", "slots") or n == o:
                continue
            if (o, n) == ("dlogits", "logits"):
                continue  # over the logits themselves
            assert _run(lib, op, **{o: at[n]}) == INV, (o, n)
    for n in ("seq_lens", "slots"):
        if n in names:
            assert _run(lib, op, **{n: at[OPS[op][4].split()[0]]}) == INV
    if op == "logprobs_backward":  # but not over parts of them, nor over strided ones
        assert _run(lib, op, dlogits=at["logits"] + 16) == INV
        assert _run(lib, op, dlogits=at["logits"], strides=[1000, 101]) == INV


@pytest.mark.parametrize("op", ["delta", "delta_backward"])
def test_strides(lib, op):
    good = [8 * 128, 128] * 2 + [8 * 256, 256] + [32, 4] * 2
    for i in range(10):
        wide = 1 << (44 if i % 2 == 0 else 34)
        bads = (good[i] - 16, good[i] + 4, 0, -good[i], wide) if i < 6 else (3, 0, -4, wide)
        for bad in bads:
            if i % 2 == 0 and bad == good[i] - 16:
                continue  # overlapping batch rows are readable
            assert _run(lib, op, strides=good[:i] + [bad] + good[i + 1:]) == INV, (i, bad)
    # a strided input's whole span counts as the input
    out = OPS[op][4].split()[0]
    assert _run(lib, op, strides=[1 << 20] + good[1:], **{out: P[0] + (1 << 21) + 16}) == INV
    assert _run(lib, op, strides=good[:6] + [1 << 20] + good[7:], **{out: P[3] + (1 << 21) + 16}) == INV


def test_logit_strides(lib):
    for op in ("logprobs", "logprobs_backward"):
        for bad in ([800, 99], [99, 100], [800, -100], [1 << 44, 100], [800, 1 << 34]):
            assert _run(lib, op, strides=bad) == INV, bad


def test_step_pool(lib):
    assert _run(lib, "step", n_slots=1) == INV  # slot b of row 1 is missing
    assert _run(lib, "step", n_slots=-1) == INV
    assert _run(lib, "step", n_slots=0, slots=P[22]) == OK  # no row has a slot
    for s in ([112, 128, 256, 4, 4], [128, 132, 256, 4, 4], [128, 128, 240, 4, 4], [128, 128, 256, 3, 4],
              [128, 128, 256, 4, 1 << 44]):
        assert _run(lib, "step", strides=s) == INV, s


def test_nothing_to_do(lib):
    for op in OPS:
        none = {n: None for n in OPS[op][1].split()}
        assert _run(lib, op, **none, B=0, **({"top": 0} if op == "logprobs" else {})) == OK, op
        if op in DELTA:
            assert _run(lib, op, **none, H=0, Hk=0) == OK and _run(lib, op, **none, H=0, Hk=2) == INV, op
    none = {n: None for n in OPS["delta"][1].split()}
    assert _run(lib, "delta", **none, N=0) == OK
    assert _run(lib, "delta", **{**none, "state_out": P[3] + 8}, N=0) == INV
    assert _run(lib, "delta", **{**none, "state_out": P[3], "state_in": P[3] + 16}, N=0) == INV


def test_binding_refuses_before_the_call():
    q, v = torch.zeros((2, 5, 2, 64)), torch.zeros((2, 5, 4, 64))
    g, s, x = torch.zeros((2, 5, 4)), torch.zeros((2, 4, 64, 64)), torch.zeros((2, 5, 30))
    tok, f = torch.zeros((2, 5), dtype=torch.int32), torch.zeros((2, 5))
    base = dict(q=q, k=q, v=v, log_decay=g, beta=g)
    delta = lambda **a: gbla.delta_attention(**{**base, **a})  # noqa: E731
    back = lambda **a: gbla.delta_attention_backward(**{**base, "do": v, **a})  # noqa: E731
    one = {n: t[:, :1] for n, t in base.items()}
    step = lambda **a: gbla.delta_attention_step(**{**one, "state": s, **a})  # noqa: E731
    score = lambda **a: gbla.token_logprobs(**{**dict(logits=x, tokens=tok), **a})  # noqa: E731
    grad = lambda **a: gbla.token_logprobs_backward(**{**dict(logits=x, lse=f, entropy=f, tokens=tok), **a})  # noqa: E731
    for fn, a in [
        (delta, dict(q=q[0])), (delta, dict(v=v[0])), (delta, dict(k=q[:, :4])), (delta, dict(k=q.double())),
        (delta, dict(log_decay=g[:, :4])), (delta, dict(beta=g.double())), (delta, dict(beta=g[..., :2])),
        (delta, dict(log_decay=torch.zeros((2, 5, 8))[..., ::2])), (delta, dict(state=s[:1])),
        (delta, dict(state=s.transpose(2, 3))), (delta, dict(out=q)), (delta, dict(seq_lens=torch.zeros(2))),
        (back, dict(do=v.transpose(0, 1).contiguous().transpose(0, 1))), (back, dict(dstate=s.double())),
        (step, dict(q=q)), (step, dict(state=s[:, :2])), (step, dict(slots=torch.zeros(2))),
        (step, dict(out=torch.zeros((2, 1, 4, 32)))),
        (score, dict(logits=x[0])), (score, dict(logits=torch.zeros((2, 5, 60))[..., ::2])), (score, dict(tokens=f)),
        (score, dict(tokens=tok[:1])), (score, dict(seq_lens=torch.zeros(2))), (score, dict(out={"lse": f})),
        (score, dict(out={"lse": f, "entropy": f, "logprob": tok})), (grad, dict(lse=None)), (grad, dict(entropy=None)),
        (grad, dict(dlse=f.double())), (grad, dict(out=x[:, :4])), (grad, dict(out=x.transpose(0, 1).contiguous().transpose(0, 1))),
    ]:
        with pytest.raises(ValueError) as e:
            fn(**a)
        assert "CUDA device" not in str(e.value), (fn, a)
    for t in (q.half(), q.int()):
        with pytest.raises(TypeError):
            delta(q=t)
    for fn in (delta, back, step, score, grad):  # nothing else wrong: host tensors
        with pytest.raises(ValueError, match="CUDA device"):
            fn()


@pytest.mark.parametrize("op", ["logprobs", "logprobs_backward"])
def test_logit_scales(lib, op):
    """Scales whose products with log2 e, or with distances of logits, leave fp32's range."""
    none = {n: None for n in OPS[op][1].split()} | {"B": 0} | ({"top": 0} if op == "logprobs" else {})
    for s in (2.0 ** -101, 1.2e-38, 2.0 ** 101, 2.4e38, 3.4e38):
        assert _run(lib, op, scale=s) == INV, s
        assert _run(lib, op, **none, scale=s) == INV, s
    for s in (2.0 ** -100, 1.0, 2.0 ** 100):
        assert _run(lib, op, **none, scale=s) == OK, s
