"""The Python binding of the decoder operators and their differentiable forms, on the CPU:
the library is replaced by a stand-in that fills what it is given and reports success."""
import contextlib

import pytest
import torch

from paper_2606_07317_gb300 import gbla


class Library:
    """Takes every entry point's call; `calls` holds (name, arguments)."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return gbla.GBLA_OK
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(gbla, "_lib", lib)
    monkeypatch.setattr(gbla, "_raw_stream", lambda dev, stream: 0)
    return lib


def _inputs(B=2, N=5, H=4, Hk=2, D=64):
    n = lambda *s: torch.randn(s)  # noqa: E731
    return dict(q=n(B, N, H, D), k=n(B, N, Hk, D), v=n(B, N, Hk, D), wq=n(H, D), wk=n(Hk, D), rot=n(9, D),
                ld=-torch.rand(H), state=n(B, H, D, D), do=n(B, N, H, D), dko=n(B, N, Hk, D))


def _calls(x, **kw):
    """Every operator on the inputs x; {name: call}."""
    one = [x[m][:, :1] for m in ("q", "k", "v")]
    return {
        "rotate": lambda: gbla.qk_norm_rotate(x["q"], x["k"], x["wq"], x["wk"], x["rot"], **kw),
        "rotate_backward": lambda: gbla.qk_norm_rotate_backward(x["q"], x["k"], x["wq"], x["wk"], x["rot"], x["do"],
                                                               x["dko"], **kw),
        "decay": lambda: gbla.decay_attention(x["q"], x["k"], x["v"], x["ld"], state=x["state"], return_state=True,
                                              **kw),
        "decay_backward": lambda: gbla.decay_attention_backward(x["q"], x["k"], x["v"], x["ld"], x["do"],
                                                                state=x["state"], return_dstate=True, **kw),
        "step": lambda: gbla.decay_attention_step(*one, x["ld"], x["state"], **kw),
    }


@pytest.mark.parametrize("op", ["rotate", "rotate_backward", "decay", "decay_backward", "step"])
@pytest.mark.parametrize("packed", [False, True])
def test_results_belong_to_the_stream_of_the_call(lib, monkeypatch, op, packed):
    """Memory that the current stream's work may still use must not be written by a kernel
    on another stream, nor be handed out again while that kernel runs: with `stream`, every
    result is allocated on it."""
    current, made = [None], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def watch(name):
        make = getattr(torch, name)

        def wrapped(*args, **kw):
            t = make(*args, **kw)
            made.append((t.data_ptr(), current[-1]))
            return t
        monkeypatch.setattr(torch, name, wrapped)

    x = _inputs()
    if packed:
        x["q"], x["k"] = torch.randn((2, 5, 6, 4, 64))[:, :, 1], torch.randn((2, 5, 6, 2, 64))[:, :, 1]
    monkeypatch.setattr(torch.cuda, "stream", on)
    watch("empty"), watch("empty_like")
    side = object()
    for stream in (side, None):
        made.clear()
        got = _calls(x, stream=stream)[op]()
        got = list(got.values()) if isinstance(got, dict) else [got] if isinstance(got, torch.Tensor) else list(got)
        where = dict(made)
        assert [where[t.data_ptr()] for t in got] == [stream] * len(got)
        assert len(current) == 1
