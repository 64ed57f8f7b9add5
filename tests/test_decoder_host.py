"""Argument checks of the decoder operators (CPU: every call is refused, or has
nothing to do, before any GPU work)."""
import ctypes
import os

import pytest
import torch

from paper_2606_07317_gb300 import build, gbla

P = [0x10000 + i * 0x1000000 for i in range(20)]  # distinct aligned fake addresses
INV, UNS, OK = gbla.GBLA_ERR_INVALID_ARG, gbla.GBLA_ERR_UNSUPPORTED, gbla.GBLA_OK


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.LIB_PATH):
        build.build()
    return gbla.load()


def _call(fn, names, tail, defaults, **kw):
    """Calls fn with fake pointers by name; sizes and flags from defaults; keywords replace."""
    vals = {n: P[i] for i, n in enumerate(names)}
    vals.update(seq_lens=None, positions=None, strides=None, slots=None)
    vals.update(defaults)
    for n in kw:
        assert n in vals, n
    vals.update(kw)
    if vals["strides"] is not None:
        vals["strides"] = (ctypes.c_int64 * len(vals["strides"]))(*vals["strides"])
    return fn(*[vals[n] for n in names], *[vals[n] for n in tail], None)


ROT = dict(B=2, N=8, H=4, Hk=2, D=64, R=64, P=16, eps=1e-6, flags=0, dtype=1)
ROT_T = list(ROT)
DEC = dict(B=2, N=8, H=4, Hk=2, D=64, scale=0.125, dtype=1, algo=0)
DEC_T = list(DEC)
STEP = dict(B=2, H=4, Hk=2, D=64, n_slots=5, scale=0.125, dtype=1)
STEP_T = list(STEP)
OPS = {
    "rotate": ("gbla_qk_norm_rotate", "q k norm_q norm_k rot positions seq_lens strides qo ko".split(), ROT_T, ROT,
               "q k norm_q norm_k rot qo ko".split()),
    "rotate_backward": ("gbla_qk_norm_rotate_backward",
                        "q k norm_q norm_k rot positions seq_lens strides dqo dko dq dk dnorm_q dnorm_k".split(),
                        ROT_T, ROT, "q k norm_q norm_k rot dqo dko dq dk dnorm_q dnorm_k".split()),
    "decay": ("gbla_decay_attention", "q k v log_decay seq_lens strides state_in o state_out".split(), DEC_T, DEC,
              "q k v log_decay o".split()),
    "decay_backward": ("gbla_decay_attention_backward",
                       "q k v log_decay seq_lens strides state_in d_o dstate_out dq dk dv dstate_in".split(),
                       DEC_T, DEC, "q k v log_decay d_o dq dk dv".split()),
    "step": ("gbla_decay_attention_step", "q k v log_decay slots strides state o".split(), STEP_T, STEP,
             "q k v log_decay state o".split()),
}


def _run(lib, op, **kw):
    name, names, tail, defaults, _ = OPS[op]
    return _call(getattr(lib, name), names, tail, defaults, **kw)


@pytest.mark.parametrize("op", OPS)
def test_pointers(lib, op):
    for n in OPS[op][4]:
        assert _run(lib, op, **{n: None}) == INV, n
        assert _run(lib, op, **{n: P[19] + 8}) == INV, n
    for n in ("state_in", "state_out", "dstate_in", "dstate_out"):
        if n in OPS[op][1]:
            assert _run(lib, op, **{n: P[19] + 4}) == INV, n
    for n in ("seq_lens", "positions", "slots"):
        if n in OPS[op][1]:
            assert _run(lib, op, **{n: P[19] + 2}) == INV, n


@pytest.mark.parametrize("op", OPS)
def test_sizes(lib, op):
    for bad in (dict(B=-1), dict(H=-4), dict(Hk=-1), dict(Hk=3), dict(Hk=0), dict(H=5), dict(B=70000)):
        assert _run(lib, op, **bad) == INV, bad
    for bad in (dict(D=48), dict(D=0), dict(D=256), dict(dtype=5)):
        assert _run(lib, op, **bad) == UNS, bad
    if "N" in OPS[op][2]:
        assert _run(lib, op, N=-3) == INV


@pytest.mark.parametrize("op", ["rotate", "rotate_backward"])
def test_rotation_arguments(lib, op):
    for bad in (dict(R=8), dict(R=80), dict(R=-16), dict(P=0), dict(P=-1), dict(eps=0.0), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(flags=2)):
        assert _run(lib, op, **bad) == INV, bad


@pytest.mark.parametrize("op", ["decay", "decay_backward", "step"])
def test_scale(lib, op):
    for s in (0.0, float("nan"), float("inf"), float("-inf")):
        assert _run(lib, op, scale=s) == INV, s


@pytest.mark.parametrize("op", ["decay", "decay_backward", "step"])
def test_scale_without_a_reciprocal(lib, op):
    for s in (1e-40, -1e-45):
        assert _run(lib, op, scale=s) == INV, s


@pytest.mark.parametrize("op", ["decay", "decay_backward"])
def test_family(lib, op):
    assert _run(lib, op, algo=7) == UNS
    assert _run(lib, op, algo=gbla.ALGO_TC, dtype=gbla.GBLA_FP32) == UNS


@pytest.mark.parametrize("op,outs", [
    ("rotate", "qo ko"), ("rotate_backward", "dq dk dnorm_q dnorm_k"), ("decay", "o state_out"),
    ("decay_backward", "dq dk dv dstate_in"), ("step", "o state")])
def test_outputs_overlap_nothing(lib, op, outs):
    names = OPS[op][1]
    at = {n: P[i] for i, n in enumerate(names)}
    for o in outs.split():
        for n in names:
            if n in ("strides", "positions", "seq_lens", "slots") or n == o:
                continue
            assert _run(lib, op, **{o: at[n]}) == INV, (o, n)
    for n in ("positions", "seq_lens", "slots"):
        if n in names:
            assert _run(lib, op, **{n: at[outs.split()[0]]}) == INV


@pytest.mark.parametrize("op", ["rotate", "rotate_backward", "decay", "decay_backward"])
def test_strides(lib, op):
    n = 2 if op.startswith("rotate") else 3
    good = [8 * 256, 256] + [8 * 128, 128] * (n - 1)
    for i in range(2 * n):
        for bad in (good[i] - 16, good[i] + 4, 0, -good[i], 1 << (44 if i % 2 == 0 else 34)):
            s = list(good)
            s[i] = bad
            if i % 2 == 0 and bad == good[i] - 16:
                continue  # overlapping batch rows are readable
            assert _run(lib, op, strides=s) == INV, (i, bad)
    # a strided input's whole span counts as the input
    out = {"rotate": "qo", "rotate_backward": "dq", "decay": "o", "decay_backward": "dq"}[op]
    s = list(good)
    s[0] = 1 << 20
    assert _run(lib, op, strides=s, **{out: P[0] + (1 << 21) + 16}) == INV


def test_step_pool(lib):
    assert _run(lib, "step", n_slots=1) == INV  # slot b of row 1 is missing
    assert _run(lib, "step", n_slots=-1) == INV
    assert _run(lib, "step", n_slots=0, slots=P[18]) == OK  # no row has a slot
    for s in ([240, 128, 128], [256, 112, 128], [256, 128, 132], [1 << 44, 128, 128]):
        assert _run(lib, "step", strides=s) == INV, s


def test_nothing_to_do(lib):
    for op in OPS:
        none = {n: None for n in OPS[op][1]}
        assert _run(lib, op, **none, B=0) == (INV if op == "rotate_backward" else OK), op
        assert _run(lib, op, **none, H=0, Hk=0) == OK, op
    none = {n: None for n in OPS["decay"][1]}
    assert _run(lib, "decay", **none, N=0) == OK
    assert _run(lib, "rotate", **{n: None for n in OPS["rotate"][1]}, N=0) == OK
    assert _run(lib, "decay", **{**none, "state_out": P[3] + 8}, N=0) == INV
    assert _run(lib, "decay", **{**none, "state_out": P[3], "state_in": P[3] + 16}, N=0) == INV


def test_binding_refuses_before_the_call():
    q, k = torch.zeros((2, 5, 4, 64)), torch.zeros((2, 5, 2, 64))
    w4, w2, rot = torch.ones((4, 64)), torch.ones((2, 64)), torch.zeros((9, 64))
    ld, s = torch.zeros(4), torch.zeros((2, 4, 64, 64))
    rotate = lambda **a: gbla.qk_norm_rotate(**{**dict(q=q, k=k, norm_q=w4, norm_k=w2, rot=rot), **a})  # noqa: E731
    decay = lambda **a: gbla.decay_attention(**{**dict(q=q, k=k, v=k, log_decay=ld), **a})  # noqa: E731
    back = lambda **a: gbla.decay_attention_backward(**{**dict(q=q, k=k, v=k, log_decay=ld, do=q), **a})  # noqa: E731
    one = dict(q=q[:, :1], k=k[:, :1], v=k[:, :1], log_decay=ld, state=s)
    step = lambda **a: gbla.decay_attention_step(**{**one, **a})  # noqa: E731
    for f, a in [
        (rotate, dict(q=q[0])), (rotate, dict(k=k[:, :4])), (rotate, dict(k=k.double())),
        (rotate, dict(q=q.transpose(2, 3).contiguous().transpose(2, 3))), (rotate, dict(q=q[:, :, ::2], norm_q=w2)),
        (rotate, dict(norm_q=w2)), (rotate, dict(norm_k=w2.double())), (rotate, dict(rot=rot.t())),
        (rotate, dict(positions=torch.zeros((2, 5), dtype=torch.int64))),
        (rotate, dict(positions=torch.zeros((2, 4), dtype=torch.int32))),
        (rotate, dict(seq_lens=torch.zeros(3, dtype=torch.int32))), (rotate, dict(out=(q, k[:, :4]))),
        (decay, dict(v=q)), (decay, dict(log_decay=torch.zeros(2))), (decay, dict(state=s[:1])),
        (decay, dict(state=s.transpose(2, 3))), (decay, dict(out=q[:, :, :2])), (decay, dict(seq_lens=torch.zeros(2))),
        (back, dict(do=q.transpose(0, 1).contiguous().transpose(0, 1))), (back, dict(dstate=s.double())),
        (step, dict(q=q)), (step, dict(state=s[:, :2])), (step, dict(slots=torch.zeros(2))),
        (step, dict(out=torch.zeros((2, 1, 4, 32)))),
    ]:
        with pytest.raises(ValueError) as e:
            f(**a)
        assert "CUDA device" not in str(e.value), (f, a)
    for f in (rotate, decay, back, step):  # nothing else wrong: host tensors
        with pytest.raises(ValueError, match="CUDA device"):
            f()


@pytest.mark.parametrize("op", OPS)
def test_key_heads_without_query_heads(lib, op):
    """No query head leaves key heads that nothing would compute or write."""
    none = {n: None for n in OPS[op][1]}
    assert _run(lib, op, **none, H=0, Hk=2) == INV
    assert _run(lib, op, H=0, Hk=1) == INV
    assert _run(lib, op, **none, H=0, Hk=0) == OK
