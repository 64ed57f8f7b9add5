"""Plain 64-bit implementations of the decoder operators for the tests: the
definitions token by token, each also evaluated on magnitudes (every product
and sum on absolute values), the scale that rounding errors are measured by."""
from __future__ import annotations

import torch

F64 = torch.float64


def ulp_bf16(x: torch.Tensor) -> torch.Tensor:
    """Spacing of bf16 numbers at |x|."""
    ax = x.abs().clamp(min=torch.finfo(torch.float32).tiny)
    return torch.exp2(torch.floor(torch.log2(ax)) - 7)


def pairs(R, interleaved):
    i = torch.arange(R // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)


def turn(x, cos, sin, R, interleaved, magnitude=False):
    """Rotates the pairs of the last axis; magnitude: |a cos| + |b sin| and so on."""
    a, b = pairs(R, interleaved)
    y = x.clone()
    if magnitude:
        cos, sin = cos.abs(), sin.abs()
        y[..., a] = x[..., a] * cos + x[..., b] * sin
        y[..., b] = x[..., a] * sin + x[..., b] * cos
        return y
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def rot_rows(rot, positions, B, N, R):
    if R == 0:
        z = torch.zeros((B, N, 1, 0), dtype=F64)
        return z, z
    if positions is None:
        positions = torch.arange(N).expand(B, N)
    row = rot.to(F64)[positions.long().clamp(0, rot.shape[0] - 1)][:, :, None]
    return row[..., :R // 2], row[..., R // 2:]


def norm_rotate(x, w, rot, positions, R, interleaved, eps):
    """(result, magnitude) of one tensor [B, N, heads, D] in 64 bits."""
    B, N = x.shape[:2]
    cos, sin = rot_rows(rot, positions, B, N, R)
    x, w = x.to(F64), w.to(F64)
    y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w
    return turn(y, cos, sin, R, interleaved), turn(y.abs(), cos, sin, R, interleaved, True)


def norm_rotate_backward(x, w, rot, positions, R, interleaved, eps, dy, lens):
    """dx, |dx|, dw, |dw| for one tensor; rows past the lengths give zero."""
    B, N = x.shape[:2]
    cos, sin = rot_rows(rot, positions, B, N, R)
    live = (torch.arange(N)[None] < torch.as_tensor(lens)[:, None])[:, :, None, None].to(F64)
    x, w, dy = x.to(F64), w.to(F64), dy.to(F64)
    x, dy = torch.where(live > 0, x, torch.ones_like(x)), torch.where(live > 0, dy, torch.zeros_like(dy))
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    n = x * r
    g, gm = turn(dy, cos, -sin, R, interleaved), turn(dy.abs(), cos, sin, R, interleaved, True)
    u, um = g * w, gm * w.abs()
    dx = r * (u - n * (u * n).mean(-1, keepdim=True))
    dxm = r * (um + n.abs() * (um * n.abs()).mean(-1, keepdim=True))
    return dx * live, dxm * live, (g * n).sum((0, 1)), (gm * n.abs()).sum((0, 1))


def wide(x, H):
    """Each key / value head once for every query head that shares it."""
    return x.to(F64).repeat_interleave(H // x.shape[2], 2)


def decay(q, k, v, log_decay, lens, state, scale):
    """o, S, |o|, |S|: the recurrence, token after token."""
    B, N, H, D = q.shape
    gamma = log_decay.to(F64).exp()[:, None, None]
    lens = torch.as_tensor(lens)
    got = []
    for f in (lambda t: t.to(F64), lambda t: t.to(F64).abs()):
        qq, kk, vv = f(q), f(wide(k, H)), f(wide(v, H))
        S = f(state) if state is not None else torch.zeros((B, H, D, D), dtype=F64)
        S = S.clone()
        o = torch.zeros((B, N, H, D), dtype=F64)
        for t in range(N):
            on = lens > t
            S[on] = gamma * S[on] + kk[on, t, :, :, None] * vv[on, t, :, None, :]
            o[on, t] = (qq[on, t, :, None, :] @ S[on])[:, :, 0] * abs(scale)
        got += [o if scale > 0 or len(got) else -o, S]
    return tuple(got)


def decay_backward(q, k, v, log_decay, do, lens, state, dstate, scale):
    """dict of gradients and dict of their magnitudes; dq, dk, dv, dstate."""
    B, N, H, D = q.shape
    Hk = k.shape[2]
    gamma = log_decay.to(F64).exp()[:, None, None]
    lens = torch.as_tensor(lens)
    out = []
    for f, sc in ((lambda t: t.to(F64), scale), (lambda t: t.to(F64).abs(), abs(scale))):
        qq, kk, vv, dd = f(q), f(wide(k, H)), f(wide(v, H)), f(do) * sc
        S = f(state).clone() if state is not None else torch.zeros((B, H, D, D), dtype=F64)
        A = f(dstate).clone() if dstate is not None else torch.zeros((B, H, D, D), dtype=F64)
        dq, dk, dv = (torch.zeros((B, N, H, D), dtype=F64) for _ in range(3))
        for t in range(N):
            on = lens > t
            S[on] = gamma * S[on] + kk[on, t, :, :, None] * vv[on, t, :, None, :]
            dq[on, t] = (S[on] @ dd[on, t, :, :, None])[..., 0]
        for t in reversed(range(N)):
            on = lens > t
            A[on] = A[on] + qq[on, t, :, :, None] * dd[on, t, :, None, :]
            dk[on, t] = (A[on] @ vv[on, t, :, :, None])[..., 0]
            dv[on, t] = (kk[on, t, :, None, :] @ A[on])[:, :, 0]
            A[on] = gamma * A[on]
        fold = lambda x: x.view(B, N, Hk, H // Hk, D).sum(3)  # noqa: E731
        out.append({"dq": dq, "dk": fold(dk), "dv": fold(dv), "dstate": A})
    return out[0], out[1]
