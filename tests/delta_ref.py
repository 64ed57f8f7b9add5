"""Plain 64-bit implementations of attention by the gated delta rule (token by token) and of
the token log probabilities, for the tests.  They run where their inputs live."""
from __future__ import annotations

import torch

F64 = torch.float64


def _wide(x, H):
    """[B, N, Hk, D] in 64 bits, each query / key head once for every value head that reads it."""
    return x.to(F64).repeat_interleave(H // x.shape[2], 2)


def delta(q, k, v, log_decay, beta, lens, state, scale):
    """(o [B, N, H, D] with zeros past the lengths, S [B, H, D, D])."""
    B, N, H, D = v.shape
    q, k, v, gamma, beta = _wide(q, H), _wide(k, H), v.to(F64), log_decay.to(F64).exp(), beta.to(F64)
    lens = torch.as_tensor(lens, device=v.device)
    S = torch.zeros((B, H, D, D), dtype=F64, device=v.device) if state is None else state.to(F64).clone()
    o = torch.zeros_like(v)
    for t in range(N):
        on = lens > t
        kept = S[on] * gamma[on, t, :, None, None]
        miss = v[on, t] - (k[on, t, :, None] @ kept)[:, :, 0]
        S[on] = kept + k[on, t, :, :, None] * (beta[on, t, :, None] * miss)[:, :, None]
        o[on, t] = (q[on, t, :, None] @ S[on])[:, :, 0] * scale
    return o, S


def delta_backward(q, k, v, log_decay, beta, do, lens, state, dstate, scale):
    """dict of the gradients of sum(do o) + sum(dstate S)."""
    B, N, H, D = v.shape
    Hk = q.shape[2]
    q, k, v, do = _wide(q, H), _wide(k, H), v.to(F64), do.to(F64) * scale
    gamma, beta = log_decay.to(F64).exp(), beta.to(F64)
    lens = torch.as_tensor(lens, device=v.device)
    zero = torch.zeros((B, H, D, D), dtype=F64, device=v.device)
    S = zero.clone() if state is None else state.to(F64).clone()
    A = zero.clone() if dstate is None else dstate.to(F64).clone()
    dq, dk, dv = (torch.zeros_like(v) for _ in range(3))
    dg, db = torch.zeros_like(beta), torch.zeros_like(beta)
    kept, miss = [None] * N, [None] * N
    for t in range(N):
        on = lens > t
        kept[t] = S[on] * gamma[on, t, :, None, None]
        miss[t] = v[on, t] - (k[on, t, :, None] @ kept[t])[:, :, 0]
        S[on] = kept[t] + k[on, t, :, :, None] * (beta[on, t, :, None] * miss[t])[:, :, None]
        dq[on, t] = (S[on] @ do[on, t, :, :, None])[..., 0]
    for t in reversed(range(N)):
        on = lens > t
        b, kt = beta[on, t, :, None], k[on, t]
        now = A[on] + q[on, t, :, :, None] * do[on, t, :, None]
        du = (kt[:, :, None] @ now)[:, :, 0]
        db[on, t] = (du * miss[t]).sum(-1)
        dv[on, t] = b * du
        dk[on, t] = (now @ (b * miss[t])[..., None])[..., 0] - (kept[t] @ (b * du)[..., None])[..., 0]
        now = now - kt[..., None] * (b * du)[:, :, None]
        dg[on, t] = (now * kept[t]).sum((-1, -2))
        A[on] = now * gamma[on, t, :, None, None]
    fold = lambda x: x.view(B, N, Hk, H // Hk, D).sum(3)  # noqa: E731
    return {"dq": fold(dq), "dk": fold(dk), "dv": dv, "dlog_decay": dg, "dbeta": db, "dstate": A}


def logprobs(logits, tokens, top, scale):
    """dict as gbla.token_logprobs', over all rows.  Rows of -inf alone: -inf, entropy 0."""
    y = logits.to(F64) * scale
    m = y.amax(-1, keepdim=True)
    base = torch.where(m.isinf() & (m < 0), torch.zeros_like(m), m)
    e = (y - base).exp()
    z = e.sum(-1)
    none = z == 0
    lnz = z.log()
    lse = base[..., 0] + lnz
    p = e / z[..., None]
    lp = y - base - lnz[..., None]
    inner = torch.where(p > 0, lp, torch.zeros_like(lp))
    ent = -(p * inner).sum(-1)
    out = {"lse": lse, "entropy": torch.where(none, torch.zeros_like(ent), ent)}
    lp = torch.where(none[..., None] | (y == -torch.inf), torch.full_like(lp, -torch.inf), lp)
    if tokens is not None:
        V = logits.shape[-1]
        has = (tokens >= 0) & (tokens < V)
        got = lp.gather(-1, torch.where(has, tokens, 0).long()[..., None])[..., 0]
        out["logprob"] = torch.where(has, got, torch.zeros_like(got))
    if top:
        idx = logits.to(F64).sort(dim=-1, descending=True, stable=True).indices[..., :top]
        out["top_token"], out["top_logprob"] = idx.to(torch.int32), lp.gather(-1, idx)
    return out


def logprobs_backward(logits, tokens, scale, dlogprob, dentropy, dlse):
    """(gradient of the logits, its terms' magnitudes); rows of -inf alone give 0."""
    V = logits.shape[-1]
    y = logits.to(F64) * scale
    none = (y == -torch.inf).all(-1, keepdim=True)
    lp = torch.where(none, torch.zeros_like(y), y - torch.logsumexp(y, -1, keepdim=True))
    p = torch.where(none, torch.zeros_like(y), lp.exp())
    inner = torch.where(p > 0, lp, torch.zeros_like(lp))
    ent = -(p * inner).sum(-1, keepdim=True)
    zero = torch.zeros(logits.shape[:-1], dtype=F64, device=logits.device)
    a, h, l = (zero if t is None else t.to(F64) for t in (dlogprob, dentropy, dlse))
    if tokens is None:
        has = torch.zeros_like(zero, dtype=torch.bool)
        at = zero.long()
    else:
        has = (tokens >= 0) & (tokens < V)
        at = torch.where(has, tokens, 0).long()
    a = torch.where(has & ~none[..., 0], a, zero)[..., None]
    h, l = h[..., None], l[..., None]
    one = torch.zeros_like(p).scatter_(-1, at[..., None], a)
    d = one - p * a - h * p * (inner + ent) + l * p
    mag = one.abs() + p * a.abs() + h.abs() * p * (inner.abs() + ent) + l.abs() * p
    return d * scale, mag * abs(scale)
