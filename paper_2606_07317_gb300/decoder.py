"""A causal decoder layer on the library's decoder operators.

The layer that emits tokens next to the bidirectional encoder: the front end
(gbla_project: Conv1D on the input, stacked projections), the norm and rotation
of queries and keys, a mixer over the tokens, the SiLU output gate and an output
projection with a residual (a plain matrix product).  The mixer is the decayed
linear attention, whose decays are constants, or attention by the gated delta
rule, whose decays and writes are formed from the input.

* `DecoderLayer.prompt` reads whole, possibly ragged prompts in parallel and
  leaves a cache: the attention state of every head, the last three inputs (the
  Conv1D's history), the lengths and, on the host, the tokens it knows of.
* `DecoderLayer.step` takes one further input of every sequence and updates the
  cache in place: the library's projection (of the window with the new input: four
  rows, of which the last counts), norm with rotation and step, a kernel each, and
  PyTorch's operations for the window, the gate, the output product and the residual.
* `AnswerHead` turns a layer's outputs into logits over items and says what they say:
  the candidates of the next item with their log probabilities (a beam search's step), or
  the log probabilities of answers that are there (a training loss).
* `norm_rotate`, `attention`, `delta_attention` and `token_logprobs` are the operators as
  differentiable torch functions, for training (first derivatives; deriving their
  gradients is an error).

`python -m paper_2606_07317_gb300.decoder` reads a prompt with each mixer, continues it
token by token, compares the continuation with one parallel call over all tokens and
names the next item's candidates.
"""
from __future__ import annotations

import time

import torch

from . import gbla

HISTORY = gbla.CONV_WIDTH - 1  # inputs before the current one that the Conv1D sees


def _whole(t):
    """t contiguous, at an address that the library takes (what autograd hands on may be a slice
    of a larger gradient)."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _Gradients(torch.autograd.Function):
    """What `compute` makes of the tensors: gradients, whose own derivative is an error.  (As
    plain results of a backward they would pass for constants under create_graph, and
    once_differentiable only sees whether the incoming gradients have a graph.)"""

    @staticmethod
    def forward(ctx, compute, *tensors):
        return compute(*tensors)

    @staticmethod
    def backward(ctx, *unused):
        raise RuntimeError("the decoder operators can be differentiated once: their gradients "
                           "have no derivative")


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, options, q, k, norm_q, norm_k, rot, positions, seq_lens):
        ctx.options = options
        ctx.save_for_backward(q, k, norm_q, norm_k, rot, positions, seq_lens)
        out = (torch.zeros(q.shape, dtype=q.dtype, device=q.device),
               torch.zeros(k.shape, dtype=k.dtype, device=k.device))
        return gbla.qk_norm_rotate(q, k, norm_q, norm_k, rot, positions, seq_lens, out=out,
                                   **options)

    @staticmethod
    def backward(ctx, dqo, dko):
        *tensors, rot, positions, seq_lens = ctx.saved_tensors
        options = ctx.options

        def compute(q, k, norm_q, norm_k, dqo, dko):
            g = gbla.qk_norm_rotate_backward(q, k, norm_q, norm_k, rot, _whole(dqo),
                                             _whole(dko), positions, seq_lens, **options)
            return g["dq"], g["dk"], g["dnorm_q"], g["dnorm_k"]

        return None, *_Gradients.apply(compute, *tensors, dqo, dko), None, None, None


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, options, q, k, v, log_decay, seq_lens, state):
        ctx.options = options
        ctx.save_for_backward(q, k, v, log_decay, seq_lens, state)
        out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
        return gbla.decay_attention(q, k, v, log_decay, seq_lens, state, out=out,
                                    return_state=True, **options)

    @staticmethod
    def backward(ctx, do, dstate):
        *tensors, log_decay, seq_lens, state = ctx.saved_tensors
        options = ctx.options

        def compute(q, k, v, state, do, dstate):
            g = gbla.decay_attention_backward(q, k, v, log_decay, _whole(do), seq_lens, state,
                                              _whole(dstate),
                                              return_dstate=state is not None, **options)
            return g["dq"], g["dk"], g["dv"], g.get("dstate")

        dq, dk, dv, first = _Gradients.apply(compute, *tensors, state, do, dstate)
        return None, dq, dk, dv, None, None, first


class _DeltaAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, options, keep, q, k, v, log_decay, beta, seq_lens, state):
        ctx.options = options
        ctx.save_for_backward(q, k, v, log_decay, beta, seq_lens, state)
        out = torch.zeros(v.shape, dtype=v.dtype, device=v.device)
        return gbla.delta_attention(q, k, v, log_decay, beta, seq_lens, state, out=out,
                                    return_state=keep, **options)

    @staticmethod
    def backward(ctx, do, dstate=None):
        q, k, v, log_decay, beta, seq_lens, state = ctx.saved_tensors
        options = ctx.options

        def compute(q, k, v, log_decay, beta, state, do, dstate):
            g = gbla.delta_attention_backward(
                q, k, v, log_decay, beta, _whole(do), seq_lens, state,
                None if dstate is None else _whole(dstate), return_dstate=state is not None,
                **options)
            return (*(g["d" + n] for n in ("q", "k", "v", "log_decay", "beta")), g.get("dstate"))

        *grads, first = _Gradients.apply(compute, q, k, v, log_decay, beta, state, do, dstate)
        return None, None, *grads, None, first


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, scale, top, logits, tokens, seq_lens):
        ctx.scale, shape = scale, logits.shape[:2]
        f32 = dict(dtype=torch.float32, device=logits.device)
        out = {"lse": torch.zeros(shape, **f32), "entropy": torch.zeros(shape, **f32)}
        if tokens is not None:
            out["logprob"] = torch.zeros(shape, **f32)
        if top:
            out["top_logprob"] = torch.zeros((*shape, top), **f32)
            out["top_token"] = torch.zeros((*shape, top), dtype=torch.int32, device=logits.device)
            ctx.mark_non_differentiable(out["top_logprob"], out["top_token"])
        gbla.token_logprobs(logits, tokens, top=top, scale=scale, seq_lens=seq_lens, out=out)
        ctx.save_for_backward(logits, tokens, seq_lens, out["lse"], out["entropy"])
        return tuple(out.values())

    @staticmethod
    def backward(ctx, dlse, dentropy, *more):
        logits, tokens, seq_lens, lse, entropy = ctx.saved_tensors
        scale, dlogprob = ctx.scale, more[0] if tokens is not None else None

        def compute(logits, dlse, dentropy, dlogprob):
            g = [None if t is None else _whole(t) for t in (dlogprob, dentropy, dlse)]
            return (gbla.token_logprobs_backward(logits, lse, entropy, tokens, *g, scale=scale,
                                                 seq_lens=seq_lens),)

        return None, None, *_Gradients.apply(compute, logits, dlse, dentropy, dlogprob), None, None


def _constant(t, name):
    if t is not None and t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} has no gradient: it is a constant of the model (detach it)")


def norm_rotate(q, k, norm_q, norm_k, rot=None, positions=None, seq_lens=None,
                eps: float = 1e-6, interleaved: bool = False):
    """gbla.qk_norm_rotate with gradients for q, k and the weights; padding rows are 0.  The
    table is a constant (refused where it asks for a gradient)."""
    _constant(rot, "rot")
    return _NormRotate.apply(dict(eps=eps, interleaved=interleaved), q, k, norm_q, norm_k, rot,
                             positions, seq_lens)


def attention(q, k, v, log_decay, seq_lens=None, state=None, scale=None,
              algo: int = gbla.ALGO_AUTO):
    """gbla.decay_attention with gradients for q, k, v and the first state; returns (o, the
    state after each sequence), padding rows of o are 0.  The decays are constants (refused
    where they ask for a gradient).  `algo` is the kernel family of both directions: in bf16
    gbla.ALGO_SIMT keeps the scores and the state as queries meet it in 32 bits."""
    _constant(log_decay, "log_decay")
    return _Attention.apply(dict(scale=scale, algo=algo), q, k, v, log_decay, seq_lens, state)


def delta_attention(q, k, v, log_decay, beta, seq_lens=None, state=None, scale=None,
                    return_state: bool = False):
    """gbla.delta_attention with gradients for everything but the lengths; padding rows of o
    are 0.  Returns o, or with return_state (o, the state after each sequence)."""
    return _DeltaAttention.apply(dict(scale=scale), return_state, q, k, v, log_decay, beta,
                                 seq_lens, state)


def token_logprobs(logits, tokens=None, top: int = 0, scale: float = 1.0, seq_lens=None) -> dict:
    """gbla.token_logprobs with gradients of lse, entropy and logprob for the logits (the top
    alternatives are constants); padding rows are 0."""
    names = ["lse", "entropy"] + ["logprob"] * (tokens is not None)
    names += ["top_logprob", "top_token"] * bool(top)
    return dict(zip(names, _TokenLogprobs.apply(scale, top, logits, tokens, seq_lens)))


def head_decays(H: int, shortest: float = 32.0, longest: float = 4096.0, device="cuda"):
    """[H] fp32 ln of the decays whose horizons (tokens until a contribution has faded to
    1/e) run evenly in their logarithm from `shortest` to `longest`."""
    h = torch.arange(H, dtype=torch.float64) / max(1, H - 1)
    horizon = shortest * (longest / shortest) ** h
    return torch.log1p(-1.0 / horizon).to(torch.float32).to(device)


class DecoderLayer:
    """Random weights of a layer of width d with H heads of D (bf16; limits as gbla_project).
    `algo`: the kernel family of the prompts' decayed attention.  `mixer`: "decay" (decayed
    linear attention) or "delta" (the gated delta rule: keys of unit length, decays from a
    projection of the input, writes weighted by the layer's gate)."""

    def __init__(self, d: int, H: int, D: int, max_positions: int, seed: int = 0, device="cuda",
                 algo: int = gbla.ALGO_AUTO, mixer: str = "decay"):
        if mixer not in ("decay", "delta"):
            raise ValueError(f"mixer must be 'decay' or 'delta', not {mixer!r}")
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(shape, generator=g, device=device) * std

        self.d, self.H, self.D, self.algo = d, H, D, algo
        self.conv_x = normal(d, gbla.CONV_WIDTH, std=0.5)
        self.w_proj = normal(4 * H * D + H, d, std=d ** -0.5).to(torch.bfloat16)
        self.norm_q, self.norm_k = (1 + normal(H, D, std=0.02) for _ in range(2))
        self.w_out = normal(H * D, d, std=(H * D) ** -0.5).to(torch.bfloat16)
        self.log_decay = head_decays(H, device=device)
        self.rot = gbla.rotation_table(max_positions, D, device=device)
        self.mixer = mixer
        if mixer == "delta":
            self.norm_k = self.norm_k * D ** -0.5
            self.w_decay = normal(d, H, std=d ** -0.5).to(torch.bfloat16)

    def _gates(self, x, gate):
        """log_decay and beta [B, N, H] of inputs x and the projection's gate: a head fades by
        about its constant decay a token, by more or less as the input says."""
        more = torch.nn.functional.softplus((x @ self.w_decay).float()) / 0.6931471805599453
        return (more * self.log_decay).to(x.dtype), gate.sigmoid()

    def _out(self, x, o, out_gate):
        y = o * torch.nn.functional.silu(out_gate)
        return x + y.flatten(2) @ self.w_out

    def _within(self, tokens):
        """Refuses sequences that the host knows to be longer than the table."""
        if tokens > self.rot.shape[0]:
            raise ValueError(f"the layer's table has {self.rot.shape[0]} positions, not {tokens}")

    def prompt(self, x, seq_lens=None):
        """y [B, N, d] of the prompts x [B, N, d] bf16 (rows past seq_lens are undefined) and
        the cache that `step` continues from.  Lengths in seq_lens must lie within
        max_positions (positions past the table would take its last row)."""
        B, N, _ = x.shape
        tokens = N if seq_lens is None else 0  # of the longest sequence, at least
        self._within(tokens)
        if N == 0:  # nothing to project or index: the cache that the first step starts from
            zeros = lambda *s, to: torch.zeros(s, dtype=to, device=x.device)  # noqa: E731
            return x.clone(), {"state": zeros(B, self.H, self.D, self.D, to=torch.float32),
                               "window": zeros(B, HISTORY, self.d, to=x.dtype),
                               "positions": zeros(B, 1, to=torch.int32), "tokens": torch.tensor(0)}
        p = gbla.project(x, self.conv_x, self.w_proj, self.H, self.D, seq_lens)
        q, k = gbla.qk_norm_rotate(p["q"], p["k"], self.norm_q, self.norm_k, self.rot,
                                   seq_lens=seq_lens)
        if self.mixer == "delta":
            o, state = gbla.delta_attention(q, k, p["v"], *self._gates(x, p["gate"]), seq_lens,
                                            return_state=True)
        else:
            o, state = gbla.decay_attention(q, k, p["v"], self.log_decay, seq_lens,
                                            return_state=True, algo=self.algo)
        L = (torch.full((B,), N, dtype=torch.int32, device=x.device) if seq_lens is None
             else seq_lens.clamp(0, N))
        at = L[:, None].long() + torch.arange(-HISTORY, 0, device=x.device)  # the last inputs
        window = torch.gather(x, 1, at.clamp(min=0)[:, :, None].expand(-1, -1, self.d))
        window = torch.where(at[:, :, None] >= 0, window, torch.zeros_like(window))
        cache = {"state": state, "window": window, "positions": L[:, None].contiguous(),
                 "tokens": torch.tensor(tokens)}
        return self._out(x, o, p["out_gate"]), cache

    def step(self, x, cache):
        """y [B, 1, d] of the next input x [B, 1, d] of every sequence; updates the cache."""
        self._within(int(cache["tokens"]) + 1)
        wide = torch.cat([cache["window"], x], 1)
        p = gbla.project(wide, self.conv_x, self.w_proj, self.H, self.D)
        now = slice(HISTORY, HISTORY + 1)  # the one output whose history is whole
        q, k = gbla.qk_norm_rotate(p["q"][:, now], p["k"][:, now], self.norm_q, self.norm_k,
                                   self.rot, cache["positions"])
        if self.mixer == "delta":
            o = gbla.delta_attention_step(q, k, p["v"][:, now],
                                          *self._gates(x, p["gate"][:, now]), cache["state"])
        else:
            o = gbla.decay_attention_step(q, k, p["v"][:, now], self.log_decay, cache["state"])
        cache["window"].copy_(wide[:, 1:])
        cache["positions"].add_(1)
        cache["tokens"] += 1
        return self._out(x, o, p["out_gate"][:, now])


class AnswerHead:
    """Logits over V items from a layer's outputs y [B, N, d] (random weights, a plain matrix
    product), and what they say."""

    def __init__(self, d: int, V: int, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.w = (torch.randn((V, d), generator=g, device=device) * d ** -0.5).to(torch.bfloat16)

    def logits(self, y):
        return y @ self.w.t()

    def candidates(self, y, top: int, ruled_out=None, scale: float = 1.0) -> dict:
        """The `top` most probable items at every place, with their log probabilities and the
        entropy (gbla.token_logprobs); `ruled_out` (truth values that broadcast to [B, N, V])
        names items that cannot follow."""
        logits = self.logits(y)
        if ruled_out is not None:
            logits = logits.masked_fill(ruled_out, -torch.inf)
        return gbla.token_logprobs(logits, top=top, scale=scale)

    def score(self, y, items, seq_lens=None, scale: float = 1.0) -> dict:
        """Log probabilities of the items [B, N] int32 that are there, differentiable in y and
        the weights (token_logprobs)."""
        return token_logprobs(self.logits(y), items, scale=scale, seq_lens=seq_lens)


def main(B: int = 4, N: int = 2048, new: int = 64, d: int = 512, H: int = 8, D: int = 64,
         mixer: str = "decay", V: int = 4096):
    layer = DecoderLayer(d, H, D, N + new, mixer=mixer)
    x = torch.randn((B, N + new, d), generator=torch.Generator().manual_seed(1))
    x = x.to(torch.bfloat16).cuda()
    whole, _ = layer.prompt(x)
    _, cache = layer.prompt(x[:, :N].contiguous())
    torch.cuda.synchronize()
    t = time.perf_counter()
    steps = [layer.step(x[:, i:i + 1], cache) for i in range(N, N + new)]
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) / new * 1e3
    got = torch.cat(steps, 1).float()
    want = whole[:, N:].float()
    off = ((got - want).norm() / (want - x[:, N:].float()).norm()).item()
    print(f"{mixer}: {B} sequences: prompt of {N}, {new} steps at {ms:.3f} ms; the steps are "
          f"{off:.2e} of the layer's output off the parallel form")
    best = AnswerHead(d, V).candidates(steps[-1], 3)
    print(f"next items of the first sequence: {best['top_token'][0, 0].tolist()}, "
          f"log probabilities {[round(p, 3) for p in best['top_logprob'][0, 0].tolist()]}")
    return off


if __name__ == "__main__":
    main()
    main(mixer="delta")
