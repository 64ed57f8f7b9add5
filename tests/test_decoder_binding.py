"""The Python binding of the decoder operators and their differentiable forms, on the CPU:
the library is replaced by a stand-in that fills what it is given and reports success."""
import contextlib

import pytest
import torch

from paper_2606_07317_gb300 import decoder, gbla


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


# ------------------------------------------------------------- the decoder layer

def _fakes(monkeypatch):
    """The library's operators as stand-ins of the right shapes on the CPU."""
    def project(x, conv_x, w_proj, H, D, seq_lens=None, out=None, stream=None):
        B, N, _ = x.shape
        return {n: x.new_zeros((B, N, H, D)) for n in ("q", "k", "v", "out_gate")} | {"gate": x.new_zeros((B, N, H))}

    def attention(q, k, v, log_decay, seq_lens=None, state=None, return_state=False, **kw):
        S = torch.zeros((q.shape[0], q.shape[2], q.shape[3], q.shape[3]))
        return (torch.zeros_like(q), S) if return_state else torch.zeros_like(q)

    monkeypatch.setattr(gbla, "project", project)
    monkeypatch.setattr(gbla, "qk_norm_rotate", lambda q, k, *a, **kw: (q, k))
    monkeypatch.setattr(gbla, "decay_attention", attention)
    monkeypatch.setattr(gbla, "decay_attention_step", lambda q, *a, **kw: torch.zeros_like(q))


@pytest.mark.parametrize("lens", [None, [0, 0, 0], [2, 0, 1]])
@pytest.mark.parametrize("N", [0, 1, 2, 3, 7])
def test_prompts_shorter_than_the_history(monkeypatch, N, lens):
    """The cache's window holds the last three inputs, zeros before the first; a prompt may
    be empty (on a GPU an index out of range would fault)."""
    _fakes(monkeypatch)
    layer = decoder.DecoderLayer(128, 2, 64, 16, device="cpu")
    x = torch.randn((3, N, 128)).to(torch.bfloat16)
    L = [N] * 3 if lens is None else [min(n, N) for n in lens]
    y, cache = layer.prompt(x, None if lens is None else torch.tensor(lens, dtype=torch.int32))
    assert y.shape == x.shape and cache["positions"].flatten().tolist() == L
    for b in range(3):
        past = torch.cat([torch.zeros((3, 128), dtype=x.dtype), x[b, :L[b]]])
        assert torch.equal(cache["window"][b], past[-3:])
    layer.step(x.new_ones((3, 1, 128)), cache)
    assert (cache["window"][:, -1] == 1).all() and cache["positions"].flatten().tolist() == [n + 1 for n in L]


# ------------------------------------------------------------- differentiable forms

def _grad_inputs():
    x = _inputs()
    return {n: t.requires_grad_() if n in ("q", "k", "v", "wq", "wk", "state") else t for n, t in x.items()}


def _forms(x):
    """{name: (differentiable form's results, its inputs)}"""
    return {
        "norm_rotate": (lambda **kw: decoder.norm_rotate(x["q"], x["k"], x["wq"], x["wk"], x["rot"], **kw),
                        [x["q"], x["k"], x["wq"], x["wk"]]),
        "attention": (lambda **kw: decoder.attention(x["q"], x["k"], x["v"], x["ld"], state=x["state"], **kw),
                      [x["q"], x["k"], x["v"], x["state"]]),
    }


@pytest.mark.parametrize("form", ["norm_rotate", "attention"])
def test_second_derivatives_are_refused(lib, form):
    """The gradients come from kernels that autograd does not see into: a derivative of them
    is an error, not zero."""
    call, leaves = _forms(_grad_inputs())[form]
    first = torch.autograd.grad(sum(t.sum() for t in call()), leaves, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiated once"):
        (first[0].square().sum() + leaves[1].square().sum()).backward()


@pytest.mark.parametrize("what", ["state", "out", "q out", "k out", "step out"])
def test_writes_are_seen_by_autograd(lib, what):
    """A tensor that a call writes through its address counts as changed in place: saved for
    a backward before, it raises there instead of giving another state's gradient."""
    x = _inputs()
    one = [x[m][:, :1] for m in ("q", "k", "v")]
    buf = {"state": x["state"], "out": torch.zeros_like(x["q"]), "q out": torch.zeros_like(x["q"]),
           "k out": torch.zeros_like(x["k"]), "step out": torch.zeros_like(one[0])}[what]
    factor = torch.ones(buf.shape, requires_grad=True)
    y = (factor * buf).sum()  # saves buf
    call = {"state": lambda: gbla.decay_attention_step(*one, x["ld"], buf),
            "out": lambda: gbla.decay_attention(x["q"], x["k"], x["v"], x["ld"], out=buf),
            "q out": lambda: gbla.qk_norm_rotate(x["q"], x["k"], x["wq"], x["wk"], x["rot"],
                                                 out=(buf, torch.zeros_like(x["k"]))),
            "k out": lambda: gbla.qk_norm_rotate(x["q"], x["k"], x["wq"], x["wk"], x["rot"],
                                                 out=(torch.zeros_like(x["q"]), buf)),
            "step out": lambda: gbla.decay_attention_step(*one, x["ld"], x["state"], out=buf)}[what]
    call()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_writes_to_tensors_of_inference_mode(lib):
    """Those have no version to count: the calls take them, inside the mode and after it."""
    x = _inputs()
    with torch.inference_mode():
        state, out = torch.zeros_like(x["state"]), torch.zeros_like(x["q"])[:, :1].contiguous()
        step = lambda: gbla.decay_attention_step(*[x[m][:, :1] for m in ("q", "k", "v")], x["ld"],  # noqa: E731
                                                 state, out=out)
        assert step() is out
    assert step() is out


def test_constants_that_ask_for_a_gradient_are_refused(lib):
    """Decays and the rotation's table have no gradient: asking for one is an error, not None."""
    x = _grad_inputs()
    x["ld"].requires_grad_()
    x["rot"].requires_grad_()
    with pytest.raises(ValueError, match="log_decay has no gradient"):
        decoder.attention(x["q"], x["k"], x["v"], x["ld"])
    with pytest.raises(ValueError, match="rot has no gradient"):
        decoder.norm_rotate(x["q"], x["k"], x["wq"], x["wk"], x["rot"])
    with torch.no_grad():
        decoder.attention(x["q"], x["k"], x["v"], x["ld"])
        decoder.norm_rotate(x["q"], x["k"], x["wq"], x["wk"], x["rot"])
    decoder.attention(x["q"], x["k"], x["v"], x["ld"].detach())


def test_options_reach_both_directions(lib):
    """eps and the pairs' layout, scale and the kernel family: the forward's and the backward's
    call get what the caller gave, or the operators' defaults."""
    x = _grad_inputs()
    sizes = (2, 5, 4, 2, 64)

    def tails(call):
        lib.calls.clear()
        sum(t.sum() for t in call()).backward()
        assert len(lib.calls) == 2
        return [args[-4:-2] for _, args in lib.calls]  # (then the dtype and the stream)

    rotate = lambda **kw: lambda: decoder.norm_rotate(x["q"], x["k"], x["wq"], x["wk"], x["rot"], **kw)  # noqa: E731
    assert tails(rotate()) == [(1e-6, 0)] * 2
    assert tails(rotate(eps=1e-3, interleaved=True)) == [(1e-3, gbla.ROTATE_INTERLEAVED)] * 2
    attend = lambda **kw: lambda: decoder.attention(x["q"], x["k"], x["v"], x["ld"], state=x["state"], **kw)  # noqa: E731
    one = lambda calls: [(args[-4], args[-2]) for _, args in calls]  # noqa: E731
    for kw, want in ((dict(), (64 ** -0.5, gbla.ALGO_AUTO)), (dict(scale=0.3, algo=gbla.ALGO_SIMT), (0.3, gbla.ALGO_SIMT))):
        lib.calls.clear()
        sum(t.sum() for t in attend(**kw)()).backward()
        assert one(lib.calls) == [want] * 2
        assert all(args[-9:-4] == sizes for _, args in lib.calls)


def test_the_layer_takes_a_kernel_family(monkeypatch):
    _fakes(monkeypatch)
    seen, attend = [], gbla.decay_attention

    def watch(*a, algo=gbla.ALGO_AUTO, **kw):
        seen.append(algo)
        return attend(*a, **kw)

    monkeypatch.setattr(gbla, "decay_attention", watch)
    x = torch.randn((1, 4, 128)).to(torch.bfloat16)
    for kw, want in ((dict(), gbla.ALGO_AUTO), (dict(algo=gbla.ALGO_SIMT), gbla.ALGO_SIMT)):
        decoder.DecoderLayer(128, 2, 64, 16, device="cpu", **kw).prompt(x)
        assert seen.pop() == want


def test_positions_past_the_table_are_refused(monkeypatch):
    """Where the host knows that a position has no row in the layer's table (a whole prompt, or
    as many steps), the call is refused instead of repeating the last angle."""
    _fakes(monkeypatch)
    layer = decoder.DecoderLayer(128, 2, 64, 6, device="cpu")
    x = torch.randn((2, 9, 128)).to(torch.bfloat16)
    with pytest.raises(ValueError, match="6 positions"):
        layer.prompt(x)
    _, cache = layer.prompt(x[:, :4].contiguous())
    for i in (4, 5):
        layer.step(x[:, i:i + 1], cache)
    before = {n: t.clone() for n, t in cache.items() if isinstance(t, torch.Tensor)}
    with pytest.raises(ValueError, match="6 positions"):
        layer.step(x[:, 6:7], cache)
    assert all(torch.equal(cache[n], t) for n, t in before.items())
    # lengths that only the device knows may lie within the table in a wider batch
    _, cache = layer.prompt(x, torch.tensor([5, 2], dtype=torch.int32))
    for i in range(6):
        layer.step(x[:, :1], cache)
    with pytest.raises(ValueError, match="6 positions"):
        layer.step(x[:, :1], cache)
