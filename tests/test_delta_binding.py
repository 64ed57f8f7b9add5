"""The Python binding of the gated delta rule and the token log probabilities, their
differentiable forms, and the decoder's mixer and answer head, on the CPU: the library is
replaced by a stand-in that reports success."""
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


def _inputs(B=2, N=5, H=4, Hk=2, D=64, V=30):
    n = lambda *s: torch.randn(s)  # noqa: E731
    return dict(q=n(B, N, Hk, D), k=n(B, N, Hk, D), v=n(B, N, H, D), g=-torch.rand((B, N, H)),
                beta=torch.rand((B, N, H)), state=n(B, H, D, D), do=n(B, N, H, D), x=n(B, N, V),
                tok=torch.zeros((B, N), dtype=torch.int32), f=n(B, N))


def _calls(x, **kw):
    five = [x[n] for n in ("q", "k", "v", "g", "beta")]
    one = [t[:, :1] for t in five]
    return {
        "delta": lambda: gbla.delta_attention(*five, state=x["state"], return_state=True, **kw),
        "delta_backward": lambda: gbla.delta_attention_backward(*five, x["do"], state=x["state"], return_dstate=True,
                                                                **kw),
        "step": lambda: gbla.delta_attention_step(*one, x["state"], **kw),
        "score": lambda: gbla.token_logprobs(x["x"], x["tok"], top=3, **kw),
        "score_backward": lambda: gbla.token_logprobs_backward(x["x"], x["f"], x["f"], x["tok"], x["f"], **kw),
    }


OPS = ["delta", "delta_backward", "step", "score", "score_backward"]


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("packed", [False, True])
def test_results_belong_to_the_stream_of_the_call(lib, monkeypatch, op, packed):
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
        x["v"], x["beta"], x["x"] = torch.randn((2, 5, 6, 4, 64))[:, :, 1], torch.rand((2, 5, 9))[..., 3:7], torch.randn((2, 5, 33))[..., 1:31]
    monkeypatch.setattr(torch.cuda, "stream", on)
    watch("empty"), watch("empty_like")
    for stream in (object(), None):
        made.clear()
        got = _calls(x, stream=stream)[op]()
        got = list(got.values()) if isinstance(got, dict) else [got] if isinstance(got, torch.Tensor) else list(got)
        where = dict(made)
        assert [where[t.data_ptr()] for t in got] == [stream] * len(got)
        assert all(t.is_contiguous() for t in got)


@pytest.mark.parametrize("what", ["out", "state", "step out", "score", "gradient", "logits"])
def test_writes_are_seen_by_autograd(lib, what):
    x = _inputs()
    five = [x[n] for n in ("q", "k", "v", "g", "beta")]
    one = [t[:, :1] for t in five]
    buf = {"out": torch.zeros_like(x["v"]), "state": x["state"], "step out": torch.zeros((2, 1, 4, 64)),
           "score": torch.zeros((2, 5)), "gradient": torch.zeros_like(x["x"]), "logits": x["x"]}[what]
    y = (torch.ones(buf.shape, requires_grad=True) * buf).sum()  # saves buf
    back = lambda out: gbla.token_logprobs_backward(x["x"], x["f"], x["f"], x["tok"], out=out)  # noqa: E731
    {"out": lambda: gbla.delta_attention(*five, out=buf), "state": lambda: gbla.delta_attention_step(*one, buf),
     "step out": lambda: gbla.delta_attention_step(*one, x["state"], out=buf),
     "score": lambda: gbla.token_logprobs(x["x"], out={"lse": buf, "entropy": torch.zeros((2, 5))}),
     "gradient": lambda: back(buf), "logits": lambda: back(buf)}[what]()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def _leaves(x):
    return {n: t.requires_grad_() if t.is_floating_point() and n not in ("do", "f") else t for n, t in x.items()}


def _forms(x):
    five = [x[n] for n in ("q", "k", "v", "g", "beta")]
    return {
        "delta": (lambda **kw: (decoder.delta_attention(*five, state=x["state"], **kw),), five + [x["state"]]),
        "delta state": (lambda **kw: decoder.delta_attention(*five, state=x["state"], return_state=True, **kw),
                        five + [x["state"]]),
        "score": (lambda **kw: tuple(decoder.token_logprobs(x["x"], x["tok"], **kw).values()), [x["x"]]),
    }


@pytest.mark.parametrize("form", ["delta", "delta state", "score"])
def test_second_derivatives_are_refused(lib, form):
    call, leaves = _forms(_leaves(_inputs()))[form]
    first = torch.autograd.grad(sum(t.sum() for t in call()), leaves, create_graph=True)
    assert all(g.shape == t.shape for g, t in zip(first, leaves))
    with pytest.raises(RuntimeError, match="differentiated once"):
        (first[0].square().sum() + leaves[-1].square().sum()).backward()


def test_options_reach_both_directions(lib):
    x = _leaves(_inputs())
    for form, kw, want in (("delta", {}, 64 ** -0.5), ("delta", {"scale": 0.3}, 0.3), ("score", {}, 1.0),
                           ("score", {"scale": 0.7}, 0.7)):
        lib.calls.clear()
        sum(t.sum() for t in _forms(x)[form][0](**kw)).backward()
        assert [args[-3] for _, args in lib.calls] == [want] * 2


def test_what_is_a_result_and_what_is_not(lib):
    """The state is formed where it is asked for; top alternatives are constants; without
    tokens there is no log probability."""
    x = _leaves(_inputs())
    five = [x[n] for n in ("q", "k", "v", "g", "beta")]
    assert decoder.delta_attention(*five).shape == x["v"].shape
    assert lib.calls[-1][1][9] is None  # state_out
    o, S = decoder.delta_attention(*five, return_state=True)
    assert lib.calls[-1][1][9] is not None and S.requires_grad
    (o.sum() + S.sum()).backward()
    assert lib.calls[-1][0] == "gbla_delta_attention_backward" and lib.calls[-1][1][15] is None  # dstate_in
    got = decoder.token_logprobs(x["x"], top=2)
    assert list(got) == ["lse", "entropy", "top_logprob", "top_token"]
    assert got["lse"].requires_grad and not got["top_logprob"].requires_grad and got["top_token"].dtype == torch.int32
    got["entropy"].sum().backward()
    assert x["x"].grad.shape == x["x"].shape
    assert list(decoder.token_logprobs(x["x"], x["tok"])) == ["lse", "entropy", "logprob"]


def _fakes(monkeypatch):
    def project(x, conv_x, w_proj, H, D, seq_lens=None, out=None, stream=None):
        B, N, _ = x.shape
        return {n: x.new_zeros((B, N, H, D)) for n in ("q", "k", "v", "out_gate")} | {"gate": x.new_zeros((B, N, H))}

    seen = []

    def delta(q, k, v, log_decay, beta, seq_lens=None, state=None, return_state=False, **kw):
        seen.append((log_decay, beta))
        return torch.zeros_like(v), torch.zeros((v.shape[0], v.shape[2], v.shape[3], v.shape[3]))

    def step(q, k, v, log_decay, beta, state, **kw):
        seen.append((log_decay, beta))
        return torch.zeros_like(v)

    monkeypatch.setattr(gbla, "project", project)
    monkeypatch.setattr(gbla, "qk_norm_rotate", lambda q, k, *a, **kw: (q, k))
    monkeypatch.setattr(gbla, "delta_attention", delta)
    monkeypatch.setattr(gbla, "delta_attention_step", step)
    return seen


@pytest.mark.parametrize("N", [0, 1, 3, 7])
def test_the_layer_with_the_delta_rule(monkeypatch, N):
    seen = _fakes(monkeypatch)
    layer = decoder.DecoderLayer(128, 2, 64, 16, device="cpu", mixer="delta")
    x = torch.randn((3, N, 128)).to(torch.bfloat16)
    y, cache = layer.prompt(x)
    assert y.shape == x.shape and cache["positions"].flatten().tolist() == [N] * 3
    layer.step(x.new_ones((3, 1, 128)), cache)
    for g, b in seen:
        assert g.shape == b.shape == (3, g.shape[1], 2) and g.dtype == b.dtype == torch.bfloat16
        assert (g <= 0).all() and ((b >= 0) & (b <= 1)).all()
    assert len(seen) == (2 if N else 1)


def test_the_layers_mixer_has_a_name():
    with pytest.raises(ValueError, match="mixer"):
        decoder.DecoderLayer(128, 2, 64, 16, device="cpu", mixer="other")


def test_mixers_share_the_other_weights():
    a, b = (decoder.DecoderLayer(128, 2, 64, 16, device="cpu", mixer=m) for m in ("decay", "delta"))
    assert torch.equal(a.w_proj, b.w_proj) and torch.equal(a.w_out, b.w_out)
    assert torch.allclose(a.norm_k * 64 ** -0.5, b.norm_k)


def test_answers(monkeypatch):
    seen = {}
    monkeypatch.setattr(gbla, "token_logprobs", lambda logits, **kw: seen.update(logits=logits, **kw) or seen)
    head = decoder.AnswerHead(16, 9, device="cpu")
    y = torch.randn((2, 3, 16)).to(torch.bfloat16)
    out = torch.zeros(9, dtype=torch.bool)
    out[4] = True
    head.candidates(y, 2, ruled_out=out, scale=0.5)
    assert seen["top"] == 2 and seen["scale"] == 0.5 and (seen["logits"][..., 4] == -torch.inf).all()
    assert torch.equal(seen["logits"][..., :4], head.logits(y)[..., :4])


@pytest.mark.parametrize("form,at", [("delta", (8,)), ("delta state", (8, 9)), ("score", (6, 7, 8))])
def test_incoming_gradients_of_any_place(lib, form, at):
    """Results that go into one flat tensor: their gradients are slices of its gradient, whole
    but at any address; the library gets them at those that it takes."""
    results = _forms(_leaves(_inputs()))[form][0]()
    flat = torch.cat([t for r in results for t in (r.new_zeros(1), r.flatten())])
    (flat * torch.arange(flat.numel())).sum().backward()
    name, args = lib.calls[-1]
    assert name.endswith("_backward")
    assert all(args[i] is not None and args[i] % 16 == 0 for i in at)
