"""Workloads of the decoder-side operators: per-head query / key norms with the
position rotation (forward and backward), decayed linear attention (prompt
form, its backward, and the single-token form on a pool of states).

Each case can be run in a plain form (elementary torch operations in 32 bits,
rounded once at the end) and through the library (`own`).  `exact` evaluates
the definitions in 64 bits, one token after the other.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}


def listed():
    return [
        # One new token of a small batch of running sequences: all latency.
        {"name": "rotate_token", "op": "rotate", "B": 8, "N": 1, "H": 8, "Hk": 8, "D": 64, "R": 64,
         "pairs": "half", "dtype": "bf16", "ragged": False, "reach": 32768},
        # q and k of the repository's headline workload.
        {"name": "rotate_long", "op": "rotate", "B": 2, "N": 32768, "H": 8, "Hk": 8, "D": 64, "R": 64,
         "pairs": "half", "dtype": "bf16", "ragged": False, "reach": 32768},
        # fp32, shared key heads, half of each head rotated, neighbouring pairs, ragged odd length.
        {"name": "rotate_shared_fp32", "op": "rotate", "B": 3, "N": 1037, "H": 6, "Hk": 2, "D": 128, "R": 64,
         "pairs": "next", "dtype": "fp32", "ragged": True, "reach": 4096},
        # A training step's gradients at the 8192-token workload.
        {"name": "rotate_back", "op": "rotate_back", "B": 4, "N": 8192, "H": 8, "Hk": 8, "D": 64, "R": 64,
         "pairs": "half", "dtype": "bf16", "ragged": False, "reach": 8192},
        # The repository's smallest configuration: one short fp32 prompt, its state kept for decoding.
        {"name": "decay_tiny_fp32", "op": "decay", "B": 1, "N": 256, "H": 2, "Hk": 2, "D": 32,
         "dtype": "fp32", "ragged": False, "start": False, "keep": True},
        # Prompts of a serving batch, states kept for the single-token form.
        {"name": "decay_prompt", "op": "decay", "B": 8, "N": 2048, "H": 8, "Hk": 8, "D": 64,
         "dtype": "bf16", "ragged": False, "start": False, "keep": True},
        # The headline shape: few long sequences, the sequence axis has to be split.
        {"name": "decay_long", "op": "decay", "B": 2, "N": 32768, "H": 8, "Hk": 8, "D": 64,
         "dtype": "bf16", "ragged": False, "start": False, "keep": False},
        # The repository's ragged batch (log-normal lengths), D = 128: the largest case.
        {"name": "decay_ragged", "op": "decay", "B": 32, "N": 32768, "H": 8, "Hk": 8, "D": 128,
         "dtype": "bf16", "ragged": True, "start": False, "keep": False},
        # A training step's gradients at the 8192-token workload.
        {"name": "decay_back", "op": "decay_back", "B": 4, "N": 8192, "H": 8, "Hk": 8, "D": 64,
         "dtype": "bf16", "ragged": False, "start": False},
        # fp32 gradients of a continued sequence: shared heads, ragged odd length, both state gradients.
        {"name": "decay_back_shared_fp32", "op": "decay_back", "B": 3, "N": 517, "H": 6, "Hk": 3, "D": 64,
         "dtype": "fp32", "ragged": True, "start": True},
        # One new token of four sequences: all latency.
        {"name": "step_few", "op": "step", "B": 4, "H": 8, "Hk": 8, "D": 64, "dtype": "bf16", "slots": 7},
        # One new token of a full serving batch out of a larger pool of states.
        {"name": "step_many", "op": "step", "B": 512, "H": 8, "Hk": 8, "D": 128, "dtype": "bf16", "slots": 600},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotate", "rotate_back", "decay", "decay", "decay_back", "decay_back", "step"])
    D = rng.choice([32, 64, 64, 128, 128])
    Hk = rng.choice([1, 2, 3, 4, 8])
    H = Hk * rng.choice([1, 1, 1, 2, 4])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "step":
        B = _log_int(rng, 1, 700)
        return {"op": op, "B": B, "H": H, "Hk": Hk, "D": D, "dtype": dtype, "slots": B + _log_int(rng, 1, 64)}
    B = _log_int(rng, 1, 32)
    # no more elements per tensor than the ragged listed case, far fewer where the plain form is slow
    most = (200_000_000 if dtype == "bf16" else 60_000_000) // (2 if op.endswith("back") else 1)
    N = _log_int(rng, 1, max(2, min(32768, most // (B * H * D))))
    c = {"op": op, "B": B, "N": N, "H": H, "Hk": Hk, "D": D, "dtype": dtype, "ragged": rng.random() < 0.5}
    if op.startswith("rotate"):
        c |= {"R": rng.choice([D, D, D // 2]), "pairs": rng.choice(["half", "next"]), "reach": N + _log_int(rng, 1, 16384)}
    else:
        c |= {"start": rng.random() < 0.5}
        if op == "decay":
            c |= {"keep": rng.random() < 0.5}
    return c


def _lengths(case):
    """Valid tokens of each sequence: log-normal about 4096 (the repository's ragged workload) or about
    half the longest for shorter batches, one sequence of full length, and an empty one in larger batches."""
    B, N = case["B"], case["N"]
    if not case["ragged"]:
        return [N] * B
    r = random.Random(B * 1000003 + N)
    L = [max(1, min(N, int(round(math.exp(r.gauss(math.log(min(4096, max(1, N // 2))), 1.0)))))) for _ in range(B)]
    if B > 4:
        L[B // 2] = 0
    if N <= 4096:
        L[0] = N
    return L


def _width(case):
    """Tokens a padded row holds: the longest sequence."""
    return max(_lengths(case))


def _decays(H, gen):
    """ln of the decay of each head: horizons from about 32 to about 4096 tokens, spread over the heads."""
    h = torch.arange(H, dtype=torch.float64) / max(1, H - 1)
    jitter = 1 + 0.02 * torch.rand(H, generator=gen, dtype=torch.float64)
    return torch.log1p(-torch.exp2(-(5 + 7 * h)) * jitter).to(torch.float32)


def _table(P, R):
    """[P, R]: cosines then sines of the angles position * 10000^(-2 i / R)."""
    f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device=DEV) / R)
    a = torch.arange(P, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt, op, B, H, Hk, D = TYPES[case["dtype"]], case["op"], case["B"], case["H"], case["Hk"], case["D"]

    def normal(*shape, std=1.0, to=dt):
        return (torch.randn(shape, generator=gen, device=DEV) * std).to(to)

    s = {"case": case}
    if op == "step":
        s |= {"q": normal(B, 1, H, D), "k": normal(B, 1, Hk, D), "v": normal(B, 1, Hk, D),
              "log_decay": _decays(H, host).to(DEV), "state": normal(case["slots"], H, D, D, std=4.0, to=torch.float32),
              "slots": torch.randperm(case["slots"], generator=host)[:B].to(torch.int32).to(DEV),
              "out": torch.zeros((B, 1, H, D), dtype=dt, device=DEV)}
        return s
    N = _width(case)
    s["seq_lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV) if case["ragged"] else None
    s |= {"q": normal(B, N, H, D), "k": normal(B, N, Hk, D)}
    if op.startswith("rotate"):
        reach = max(case["reach"], N)
        first = torch.randint(0, reach - N + 1, (B, 1), generator=host)
        s |= {"norm_q": 1 + normal(H, D, std=0.1, to=torch.float32), "norm_k": 1 + normal(Hk, D, std=0.1, to=torch.float32),
              "rot": _table(reach, case["R"]), "positions": (first + torch.arange(N)).to(torch.int32).to(DEV)}
        if op == "rotate_back":
            s |= {"dqo": normal(B, N, H, D), "dko": normal(B, N, Hk, D)}
        else:
            s |= {"qo": torch.zeros((B, N, H, D), dtype=dt, device=DEV), "ko": torch.zeros((B, N, Hk, D), dtype=dt, device=DEV)}
        return s
    s |= {"v": normal(B, N, Hk, D), "log_decay": _decays(H, host).to(DEV),
          "state": normal(B, H, D, D, std=4.0, to=torch.float32) if case["start"] else None}
    if op == "decay_back":
        s |= {"do": normal(B, N, H, D), "dstate": normal(B, H, D, D, to=torch.float32) if case["start"] else None}
    else:
        s["out"] = torch.zeros((B, N, H, D), dtype=dt, device=DEV)
    return s


# ---------------------------------------------------------------- the library

def _run_own(s):
    from paper_2606_07317_gb300 import gbla
    c = s["case"]
    if c["op"] == "rotate":
        return gbla.qk_norm_rotate(s["q"], s["k"], s["norm_q"], s["norm_k"], s["rot"], positions=s["positions"],
                                   seq_lens=s["seq_lens"], eps=EPS, interleaved=c["pairs"] == "next",
                                   out=(s["qo"], s["ko"]))
    if c["op"] == "rotate_back":
        return gbla.qk_norm_rotate_backward(s["q"], s["k"], s["norm_q"], s["norm_k"], s["rot"], s["dqo"], s["dko"],
                                            positions=s["positions"], seq_lens=s["seq_lens"], eps=EPS,
                                            interleaved=c["pairs"] == "next")
    if c["op"] == "decay":
        return gbla.decay_attention(s["q"], s["k"], s["v"], s["log_decay"], seq_lens=s["seq_lens"], state=s["state"],
                                    out=s["out"], return_state=c["keep"])
    if c["op"] == "decay_back":
        return gbla.decay_attention_backward(s["q"], s["k"], s["v"], s["log_decay"], s["do"], seq_lens=s["seq_lens"],
                                             state=s["state"], dstate=s["dstate"], return_dstate=c["start"])
    o = gbla.decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], slots=s["slots"], out=s["out"])
    return o, s["state"]


# ------------------------------------------------------------- the plain forms

def _valid(s, N):
    """[B, N, 1, 1] truth values: the token is before its sequence's end."""
    L = s["seq_lens"]
    if L is None:
        return None
    return (torch.arange(N, device=DEV) < L[:, None])[:, :, None, None]


def _cut(x, ok):
    return x if ok is None else torch.where(ok, x, torch.zeros((), dtype=x.dtype, device=x.device))


def _turn(x, cos, sin, R, pairs, back=False):
    """Rotates the first R values of each head by the pairs' angles (back: by the opposite angles)."""
    if back:
        sin = -sin
    if pairs == "half":
        a, b = x[..., :R // 2], x[..., R // 2:R]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., R:]], -1)
    a, b = x[..., 0:R:2], x[..., 1:R:2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., R:]], -1)


def _angles(s):
    R = s["case"]["R"]
    row = s["rot"][s["positions"].long()][:, :, None, :]
    return row[..., :R // 2], row[..., R // 2:]


def _norm_turn(s, x, w):
    c = s["case"]
    cos, sin = _angles(s)
    f = x.float()
    y = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS) * w
    return _cut(_turn(y, cos, sin, c["R"], c["pairs"]).to(x.dtype), _valid(s, x.shape[1]))


def _norm_turn_back(s, x, w, dy):
    c = s["case"]
    cos, sin = _angles(s)
    ok = _valid(s, x.shape[1])
    f = x.float()
    r = torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS)
    n = f * r
    g = _cut(_turn(dy.float(), cos, sin, c["R"], c["pairs"], back=True), ok)
    dw = (g * n).sum((0, 1))
    g = g * w
    return (r * (g - n * (g * n).mean(-1, keepdim=True))).to(x.dtype), dw


CHUNK = 128


def _decayed(x, y, z, ld, first):
    """out[b, t, h] = sum_{j <= t} decay^(t - j) (x_t . y_j) z_j + decay^(t + 1) x_t first: in chunks, all of
    them at once, whose sums meet through a triangular matrix of decays.  [B, N, H, D] fp32 in and out."""
    B, N, H, D = x.shape
    n = -(-N // CHUNK)
    C = CHUNK

    def cut(t):
        return torch.nn.functional.pad(t, (0, 0, 0, 0, 0, n * C - N)).view(B, n, C, H, D).permute(0, 3, 1, 2, 4)

    x, y, z = cut(x), cut(y), cut(z)
    i = torch.arange(C, device=x.device, dtype=torch.float32)
    gap = i[:, None] - i
    w = torch.where(gap >= 0, (gap.clamp(min=0) * ld[:, None, None]).exp(), torch.zeros((), device=x.device))
    out = (x @ y.transpose(-1, -2) * w[None, :, None]) @ z
    part = (y * ((C - 1 - i) * ld[:, None]).exp()[None, :, None, :, None]).transpose(-1, -2) @ z
    c = torch.arange(n, device=x.device, dtype=torch.float32)
    gap = c[:, None] - 1 - c
    w = torch.where(gap >= 0, (gap.clamp(min=0) * C * ld[:, None, None]).exp(), torch.zeros((), device=x.device))
    before = (w @ part.reshape(B, H, n, D * D)).view(B, H, n, D, D)
    if first is not None:
        before = before + (c * C * ld[:, None]).exp()[None, :, :, None, None] * first[:, :, None]
    out = out + ((i + 1) * ld[:, None]).exp()[None, :, None, :, None] * (x @ before)
    return out.permute(0, 2, 3, 1, 4).reshape(B, n * C, H, D)[:, :N]


def _spread(x, H):
    """Each key / value head once for every query head that shares it."""
    return x.float() if x.shape[2] == H else x.float().repeat_interleave(H // x.shape[2], 2)


def _left(s, N):
    """[B, N, H, 1]: decay^(tokens after this one)."""
    t = torch.arange(N, device=DEV, dtype=torch.float32)
    L = s["seq_lens"].float()[:, None] if s["seq_lens"] is not None else torch.full((1, 1), float(N), device=DEV)
    return ((L - 1 - t).clamp(min=0)[:, :, None] * s["log_decay"]).exp()[..., None]


def _whole(s, N):
    """[B, H, 1, 1]: decay^length."""
    L = s["seq_lens"].float()[:, None] if s["seq_lens"] is not None else torch.full((1, 1), float(N), device=DEV)
    return (L * s["log_decay"]).exp()[:, :, None, None]


def _outer_sum(a, b, w):
    return ((a * w).permute(0, 2, 3, 1)) @ b.permute(0, 2, 1, 3)


def _plain_decay(s):
    c, q = s["case"], s["q"]
    N, H, D = q.shape[1], c["H"], c["D"]
    ok, scale = _valid(s, N), c["D"] ** -0.5
    k, v = _cut(_spread(s["k"], H), ok), _cut(_spread(s["v"], H), ok)
    o = _cut((_decayed(q.float(), k, v, s["log_decay"], s["state"]) * scale).to(q.dtype), ok)
    if not c["keep"]:
        return o
    last = _outer_sum(k, v, _left(s, N))
    return o, last if s["state"] is None else last + _whole(s, N) * s["state"]


def _turned(s, x):
    """The valid tokens of each sequence in the opposite order, zeros after them."""
    if s["seq_lens"] is None:
        return x.flip(1)
    N = x.shape[1]
    at = (s["seq_lens"].long()[:, None] - 1 - torch.arange(N, device=DEV))
    x = torch.gather(x, 1, at.clamp(min=0)[:, :, None, None].expand_as(x))
    return _cut(x, _valid(s, N))


def _plain_decay_back(s):
    c = s["case"]
    N, H, Hk = s["q"].shape[1], c["H"], c["Hk"]
    ok, scale, ld = _valid(s, N), c["D"] ** -0.5, s["log_decay"]
    q, k, v, do = (_cut(_spread(s[n], H), ok) for n in ("q", "k", "v", "do"))
    do = do * scale
    s0, ds = s["state"], s["dstate"]
    dq = _decayed(do, v, k, ld, None if s0 is None else s0.transpose(-1, -2))
    rq, rk, rv, rdo = (_turned(s, x) for x in (q, k, v, do))
    dk, dv = _turned(s, _decayed(rv, rdo, rq, ld, None)), _turned(s, _decayed(rk, rq, rdo, ld, None))
    if ds is not None:
        w = _left(s, N)
        dk = dk + w * torch.einsum("bnhe,bhde->bnhd", v, ds)
        dv = dv + w * torch.einsum("bnhd,bhde->bnhe", k, ds)
    dk, dv = (_cut(x, ok).unflatten(2, (Hk, H // Hk)).sum(3) for x in (dk, dv))
    got = {"dq": _cut(dq, ok).to(s["q"].dtype), "dk": dk.to(s["k"].dtype), "dv": dv.to(s["v"].dtype)}
    if c["start"]:
        t = torch.arange(N, device=DEV, dtype=torch.float32)
        w = ((t + 1)[:, None] * ld).exp()[None, :, :, None]
        got["dstate"] = _outer_sum(q, do, w) + _whole(s, N) * ds
    return got


def _plain_step(s):
    c = s["case"]
    H, at = c["H"], s["slots"].long()
    q, k, v = (_spread(s[n], H)[:, 0] for n in ("q", "k", "v"))
    new = s["log_decay"].exp()[:, None, None] * s["state"][at] + k[..., :, None] * v[..., None, :]
    s["state"].index_copy_(0, at, new)
    o = (q[..., None, :] @ new)[..., 0, :] * c["D"] ** -0.5
    s["out"].copy_(o[:, None])
    return s["out"], s["state"]


def run(state):
    s = state
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op == "rotate":
        return _norm_turn(s, s["q"], s["norm_q"]), _norm_turn(s, s["k"], s["norm_k"])
    if op == "rotate_back":
        dq, dwq = _norm_turn_back(s, s["q"], s["norm_q"], s["dqo"])
        dk, dwk = _norm_turn_back(s, s["k"], s["norm_k"], s["dko"])
        return {"dq": dq, "dk": dk, "dnorm_q": dwq, "dnorm_k": dwk}
    if op == "decay":
        return _plain_decay(s)
    if op == "decay_back":
        return _plain_decay_back(s)
    return _plain_step(s)


# --------------------------------------------------------------------- floors

def work(case):
    op, B, H, Hk, D, e = case["op"], case["B"], case["H"], case["Hk"], case["D"], BYTES[case["dtype"]]
    if op == "step":
        return {"bytes": B * (2 * H * D * D * 4 + (2 * H + 2 * Hk) * D * e) + 4 * (B + H), "flops": B * H * D * D * 5}
    T = sum(_lengths(case))
    q, k = T * H * D * e, T * Hk * D * e
    if op.startswith("rotate"):
        # tables: the rows that are met, once; positions and lengths beside them
        table = min(T, max(case["reach"], _width(case))) * case["R"] * 4 + 4 * B * _width(case) + (4 * B if case["ragged"] else 0)
        w = (H + Hk) * D * 4
        if op == "rotate":
            return {"bytes": 2 * (q + k) + table + w, "flops": T * (H + Hk) * (4 * D + 3 * case["R"])}
        pad = (B * _width(case) - T) * (H + Hk) * D * e  # the padding rows of the gradients are written as zeros
        return {"bytes": 3 * (q + k) + pad + table + 2 * w, "flops": T * (H + Hk) * (9 * D + 3 * case["R"])}
    S = B * H * D * D * 4
    # the recurrent form's operations: one rank-one update and one product with the state a token
    if op == "decay":
        return {"bytes": 2 * q + 2 * k + S * (case["start"] + case["keep"]), "flops": T * H * D * D * 5}
    pad = (B * _width(case) - T) * (H + 2 * Hk) * D * e
    return {"bytes": 3 * q + 4 * k + pad + 3 * S * case["start"], "flops": T * H * D * D * 12}


# ------------------------------------------------------------ in 64 bits, token by token

def exact(case, seed):
    s = prepare(case, seed)
    op, H, D = case["op"], case["H"], case["D"]
    d = {n: x.double() for n, x in s.items() if isinstance(x, torch.Tensor) and x.is_floating_point()}
    if op.startswith("rotate"):
        return _exact_rotate(case, s, d)
    g = H // case["Hk"]
    gamma = d["log_decay"].exp()[None, :, None, None]
    scale = 1 / math.sqrt(D)
    wide = lambda x: x[:, :, torch.arange(H, device=DEV) // g]  # noqa: E731
    if op == "step":
        at = s["slots"].long()
        pool = d["state"].clone()
        k, v = wide(d["k"])[:, 0], wide(d["v"])[:, 0]
        new = pool[at] * gamma + torch.einsum("bhd,bhe->bhde", k, v)
        pool[at] = new
        return torch.einsum("bhd,bhde->bhe", d["q"][:, 0], new)[:, None] * scale, pool
    B, N = s["q"].shape[:2]
    if N * B * H * D * D > 1.6e11:
        return None
    L = s["seq_lens"].long().tolist() if s["seq_lens"] is not None else [N] * B
    on = torch.tensor(L, device=DEV)
    q, k, v = d["q"], d["k"], d["v"]
    S = d["state"].clone() if case["start"] else torch.zeros((B, H, D, D), dtype=torch.float64, device=DEV)
    if op == "decay":
        out = torch.zeros_like(q)
        for t in range(N):
            live = (t < on)[:, None, None, None]
            new = gamma * S + wide(k[:, t:t + 1])[:, 0, :, :, None] * wide(v[:, t:t + 1])[:, 0, :, None, :]
            S = torch.where(live, new, S)
            out[:, t] = torch.where(live[..., 0], (q[:, t, :, None, :] @ S)[:, :, 0] * scale, out[:, t])
        return (out, S) if case["keep"] else out
    do = d["do"] * scale
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    for t in range(N):
        live = (t < on)[:, None, None, None]
        S = gamma * S + wide(k[:, t:t + 1])[:, 0, :, :, None] * wide(v[:, t:t + 1])[:, 0, :, None, :]
        dq[:, t] = torch.where(live[..., 0], (S @ do[:, t, :, :, None])[..., 0], dq[:, t])
    A = d["dstate"].clone() if case["start"] else torch.zeros((B, H, D, D), dtype=torch.float64, device=DEV)
    for t in reversed(range(N)):
        live = (t < on)[:, None, None, None]
        new = A + q[:, t, :, :, None] * do[:, t, :, None, :]
        kt, vt = wide(k[:, t:t + 1])[:, 0], wide(v[:, t:t + 1])[:, 0]
        dk[:, t] = torch.where(live[..., 0], (new @ vt[..., None])[..., 0], dk[:, t])
        dv[:, t] = torch.where(live[..., 0], (kt[:, :, None, :] @ new)[:, :, 0], dv[:, t])
        A = torch.where(live, gamma * new, A)
    got = {"dq": dq, "dk": dk.view(B, N, case["Hk"], g, D).sum(3), "dv": dv.view(B, N, case["Hk"], g, D).sum(3)}
    if case["start"]:
        got["dstate"] = A
    return got


def _exact_rotate(case, s, d):
    R, B, N = case["R"], *s["q"].shape[:2]
    if case["pairs"] == "half":
        one, two = torch.arange(R // 2, device=DEV), torch.arange(R // 2, R, device=DEV)
    else:
        one, two = torch.arange(0, R, 2, device=DEV), torch.arange(1, R, 2, device=DEV)
    L = s["seq_lens"] if s["seq_lens"] is not None else torch.full((B,), N, device=DEV)
    live = (torch.arange(N, device=DEV)[None] < L[:, None]).double()[:, :, None, None]
    at = d["rot"][s["positions"].long()].unsqueeze(2)
    turn = torch.complex(at[..., :R // 2].contiguous(), at[..., R // 2:].contiguous())
    got = []
    for x, w, dy in ((d["q"], d["norm_q"], d.get("dqo")), (d["k"], d["norm_k"], d.get("dko"))):
        rms = (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
        if dy is None:
            y = x / rms * w
            p = torch.complex(y[..., one], y[..., two]) * turn
            y = y.clone()
            y[..., one], y[..., two] = p.real, p.imag
            got.append(y * live)
            continue
        p = torch.complex(dy[..., one], dy[..., two]) * turn.conj()
        u = dy.clone()
        u[..., one], u[..., two] = p.real, p.imag
        u = u * live
        dw = torch.einsum("bnhd,bnhd->hd", u, x / rms)
        u = u * w
        dx = u / rms - x * ((u * x).sum(-1, keepdim=True) / (x.shape[-1] * rms.pow(3)))
        got += [dx, dw]
    if len(got) == 2:
        return tuple(got)
    return {"dq": got[0], "dk": got[2], "dnorm_q": got[1], "dnorm_k": got[3]}
