"""A causal decoder layer on the library's decoder operators.

The layer that emits tokens next to the bidirectional encoder: the front end
(gbla_project: Conv1D on the input, stacked projections), the norm and rotation
of queries and keys, the decayed linear attention, the SiLU output gate and an
output projection with a residual (a plain matrix product).

* `DecoderLayer.prompt` reads whole, possibly ragged prompts in parallel and
  leaves a cache: the attention state of every head, the last three inputs (the
  Conv1D's history), the lengths and, on the host, the tokens it knows of.
* `DecoderLayer.step` takes one further input of every sequence and updates the
  cache in place: the library's projection (of the window with the new input: four
  rows, of which the last counts), norm with rotation and step, a kernel each, and
  PyTorch's operations for the window, the gate, the output product and the residual.
* `norm_rotate` and `attention` are the two operators as differentiable torch
  functions, for training (first derivatives; deriving their gradients is an error).

`python -m paper_2606_07317_gb300.decoder` reads a prompt, continues it token by
token and compares the continuation with one parallel call over all tokens.
"""
from __future__ import annotations

import time

import torch

from . import gbla

HISTORY = gbla.CONV_WIDTH - 1  # inputs before the current one that the Conv1D sees


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
            g = gbla.qk_norm_rotate_backward(q, k, norm_q, norm_k, rot, dqo.contiguous(),
                                             dko.contiguous(), positions, seq_lens, **options)
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
            g = gbla.decay_attention_backward(q, k, v, log_decay, do.contiguous(), seq_lens, state,
                                              dstate.contiguous(),
                                              return_dstate=state is not None, **options)
            return g["dq"], g["dk"], g["dv"], g.get("dstate")

        dq, dk, dv, first = _Gradients.apply(compute, *tensors, state, do, dstate)
        return None, dq, dk, dv, None, None, first


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


def head_decays(H: int, shortest: float = 32.0, longest: float = 4096.0, device="cuda"):
    """[H] fp32 ln of the decays whose horizons (tokens until a contribution has faded to
    1/e) run evenly in their logarithm from `shortest` to `longest`."""
    h = torch.arange(H, dtype=torch.float64) / max(1, H - 1)
    horizon = shortest * (longest / shortest) ** h
    return torch.log1p(-1.0 / horizon).to(torch.float32).to(device)


class DecoderLayer:
    """Random weights of a layer of width d with H heads of D (bf16; limits as gbla_project).
    `algo`: the kernel family of the prompts' attention."""

    def __init__(self, d: int, H: int, D: int, max_positions: int, seed: int = 0, device="cuda",
                 algo: int = gbla.ALGO_AUTO):
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
        o, state = gbla.decay_attention(q, k, p["v"], self.log_decay, seq_lens, return_state=True,
                                        algo=self.algo)
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
        o = gbla.decay_attention_step(q, k, p["v"][:, now], self.log_decay, cache["state"])
        cache["window"].copy_(wide[:, 1:])
        cache["positions"].add_(1)
        cache["tokens"] += 1
        return self._out(x, o, p["out_gate"][:, now])


def main(B: int = 4, N: int = 2048, new: int = 64, d: int = 512, H: int = 8, D: int = 64):
    layer = DecoderLayer(d, H, D, N + new)
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
    print(f"{B} sequences: prompt of {N}, {new} steps at {ms:.3f} ms; the steps are {off:.2e} of "
          "the layer's output off the parallel form")
    return off


if __name__ == "__main__":
    main()
