"""Workloads of the operators that read and answer: attention by the gated delta
rule (prompt form, its backward, and the single-token form on a pool of
states), and the log probabilities of given tokens with entropy and top
alternatives (and their backward).

Each case can be run in a plain form (elementary torch operations in 32 bits,
rounded once at the end) and through the library (`own`).  `exact` evaluates
the definitions in 64 bits: the recurrence one token after the other, the
probabilities row by row.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}


def listed():
    return [
        # The repository's smallest configuration: one short fp32 prompt, its state kept for decoding.
        {"name": "delta_tiny_fp32", "op": "delta", "B": 1, "N": 256, "H": 2, "Hk": 2, "D": 32, "dtype": "fp32",
         "ragged": False, "packed": False, "start": False, "keep": True},
        # Prompts of a serving batch, several documents packed in each, states kept for the single-token form.
        {"name": "delta_prompt", "op": "delta", "B": 8, "N": 2048, "H": 8, "Hk": 8, "D": 64, "dtype": "bf16",
         "ragged": False, "packed": True, "start": False, "keep": True},
        # The repository's headline shape: few long sequences.
        {"name": "delta_long", "op": "delta", "B": 2, "N": 32768, "H": 8, "Hk": 8, "D": 64, "dtype": "bf16",
         "ragged": False, "packed": False, "start": False, "keep": False},
        # The repository's ragged batch (log-normal lengths), D = 128: the largest case.
        {"name": "delta_ragged", "op": "delta", "B": 32, "N": 32768, "H": 8, "Hk": 8, "D": 128, "dtype": "bf16",
         "ragged": True, "packed": False, "start": False, "keep": False},
        # A training step's gradients at the 8192-token workload.
        {"name": "delta_back", "op": "delta_back", "B": 4, "N": 8192, "H": 8, "Hk": 8, "D": 64, "dtype": "bf16",
         "ragged": False, "packed": False, "start": False},
        # fp32 gradients of a continued sequence: shared key heads, ragged odd length, both state gradients.
        {"name": "delta_back_shared_fp32", "op": "delta_back", "B": 3, "N": 517, "H": 6, "Hk": 3, "D": 64,
         "dtype": "fp32", "ragged": True, "packed": True, "start": True},
        # One new token of four sequences: all latency.
        {"name": "delta_step_few", "op": "delta_step", "B": 4, "H": 8, "Hk": 8, "D": 64, "dtype": "bf16", "slots": 7},
        # One new token of a full serving batch out of a larger pool of states.
        {"name": "delta_step_many", "op": "delta_step", "B": 512, "H": 8, "Hk": 8, "D": 128, "dtype": "bf16",
         "slots": 600},
        # The candidates of the next token of a few running sequences: all latency.
        {"name": "score_next", "op": "score", "B": 4, "N": 1, "V": 65536, "dtype": "bf16", "ragged": False,
         "masked": False, "top": 8, "tokens": False, "scale": 1.0},
        # A beam search's step over a codebook of items: fp32 logits, most items ruled out by a mask.
        {"name": "score_beams_fp32", "op": "score", "B": 64, "N": 32, "V": 8191, "dtype": "fp32", "ragged": False,
         "masked": True, "top": 32, "tokens": False, "scale": 1.25},
        # Scoring answers that are there: a ragged batch, a vocabulary of an odd size.
        {"name": "score_prompt", "op": "score", "B": 16, "N": 1024, "V": 50021, "dtype": "bf16", "ragged": True,
         "masked": False, "top": 0, "tokens": True, "scale": 1.0},
        # A training step's gradients of log probabilities, entropies and normalisers.
        {"name": "score_back", "op": "score_back", "B": 4, "N": 2048, "V": 32768, "dtype": "bf16", "ragged": False,
         "masked": False, "scale": 1.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["delta", "delta", "delta", "delta_back", "delta_back", "delta_step", "score", "score", "score_back"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op.startswith("score"):
        V = _log_int(rng, 5, 200000)
        # no more logits than the largest listed ones
        rows = _log_int(rng, 1, max(2, min(30000, (260_000_000 if dtype == "bf16" else 120_000_000) // V)))
        B = _log_int(rng, 1, min(64, rows))
        c = {"op": op, "B": B, "N": max(1, rows // B), "V": V, "dtype": dtype, "ragged": rng.random() < 0.5,
             "masked": rng.random() < 0.4, "scale": rng.choice([1.0, 1.0, 0.7, 1.25])}
        if op == "score":
            c |= {"top": min(V, rng.choice([0, 1, 5, 8, 32, 64])), "tokens": rng.random() < 0.6}
        return c
    D = rng.choice([32, 64, 64, 128, 128])
    Hk = rng.choice([1, 2, 3, 4, 8])
    H = Hk * rng.choice([1, 1, 1, 2, 4])
    if op == "delta_step":
        B = _log_int(rng, 1, 700)
        return {"op": op, "B": B, "H": H, "Hk": Hk, "D": D, "dtype": dtype, "slots": B + _log_int(rng, 1, 64)}
    B = _log_int(rng, 1, 32)
    # far fewer elements per tensor than the largest listed case: the plain form in 32 bits is slow
    most = (80_000_000 if dtype == "bf16" else 30_000_000) // (2 if op == "delta_back" else 1)
    N = _log_int(rng, 1, max(2, min(32768, most // (B * H * D))))
    c = {"op": op, "B": B, "N": N, "H": H, "Hk": Hk, "D": D, "dtype": dtype, "ragged": rng.random() < 0.5,
         "packed": rng.random() < 0.4, "start": rng.random() < 0.5}
    if op == "delta":
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


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt, op, B = TYPES[case["dtype"]], case["op"], case["B"]

    def normal(*shape, std=1.0, to=dt):
        return (torch.randn(shape, generator=gen, device=DEV) * std).to(to)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device=DEV)

    s = {"case": case}
    N = 1 if op == "delta_step" else _width(case)
    if op != "delta_step":
        s["seq_lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV) if case["ragged"] else None
    if op.startswith("score"):
        V = case["V"]
        s["logits"] = normal(B, N, V, std=3.0)
        if case["masked"]:  # ruled out: all but about a tenth of the tokens, the first one always allowed
            out = uniform(B, N, V) < 0.9
            out[..., 0] = False
            s["logits"].masked_fill_(out, -math.inf)
            del out
        tokens = (uniform(B, N).double() ** 2 * V).long().clamp(max=V - 1)
        if case["masked"]:  # an answer is a token that was allowed: the next one in order, or the first
            ok = s["logits"] > -math.inf
            at = torch.arange(V, device=DEV)
            nxt = torch.where(ok & (at >= tokens[..., None]), at, V).amin(-1)
            tokens = torch.where(nxt < V, nxt, 0)
            del ok, nxt
        s["tokens"] = tokens.to(torch.int32)
        s["tokens"][uniform(B, N) < 0.02] = -1  # positions without an answer
        f32 = dict(dtype=torch.float32, device=DEV)
        if op == "score":
            s["out"] = {"lse": torch.zeros((B, N), **f32), "entropy": torch.zeros((B, N), **f32)}
            if case["tokens"]:
                s["out"]["logprob"] = torch.zeros((B, N), **f32)
            else:
                s["tokens"] = None
            if case["top"]:
                s["out"]["top_logprob"] = torch.zeros((B, N, case["top"]), **f32)
                s["out"]["top_token"] = torch.zeros((B, N, case["top"]), dtype=torch.int32, device=DEV)
        else:
            # what the forward call left, and the gradients that come in
            lse, ent = _norms(s, torch.float64)
            s |= {"lse": lse.float(), "entropy": ent.float()}
            s |= {n: normal(B, N, to=torch.float32) for n in ("dlogprob", "dentropy", "dlse")}
        return s
    H, Hk, D = case["H"], case["Hk"], case["D"]
    # queries and keys as a norm of unit length leaves them; gates as a model forms them, horizons of the heads
    # from about 16 to about 4096 tokens
    unit = lambda x: (x / x.float().square().sum(-1, keepdim=True).sqrt()).to(dt)  # noqa: E731
    horizon = 16.0 * 256.0 ** (torch.arange(H, device=DEV) / max(1, H - 1))
    s |= {"q": unit(normal(B, N, Hk, D, to=torch.float32)), "k": unit(normal(B, N, Hk, D, to=torch.float32)),
          "v": normal(B, N, H, D),
          "log_decay": (-torch.nn.functional.softplus(normal(B, N, H, to=torch.float32)) / horizon).to(dt),
          "beta": normal(B, N, H, to=torch.float32).sigmoid().to(dt)}
    if op == "delta_step":
        s |= {"state": normal(case["slots"], H, D, D, std=0.5, to=torch.float32),
              "slots": torch.randperm(case["slots"], generator=gen, device=DEV)[:B].to(torch.int32),
              "out": torch.zeros((B, 1, H, D), dtype=dt, device=DEV)}
        return s
    if case["packed"]:  # a new document begins: the memory of the one before ends
        s["log_decay"][uniform(B, N) < 1 / 300] = -math.inf
    s["state"] = normal(B, H, D, D, std=0.5, to=torch.float32) if case["start"] else None
    if op == "delta_back":
        s |= {"do": normal(B, N, H, D), "dstate": normal(B, H, D, D, to=torch.float32) if case["start"] else None}
    else:
        s["out"] = torch.zeros((B, N, H, D), dtype=dt, device=DEV)
    return s


# ---------------------------------------------------------------- the library

def _run_own(s):
    from paper_2606_07317_gb300 import gbla
    c = s["case"]
    if c["op"] == "delta":
        return gbla.delta_attention(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], seq_lens=s["seq_lens"],
                                    state=s["state"], out=s["out"], return_state=c["keep"])
    if c["op"] == "delta_back":
        return gbla.delta_attention_backward(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["do"],
                                             seq_lens=s["seq_lens"], state=s["state"], dstate=s["dstate"],
                                             return_dstate=c["start"])
    if c["op"] == "delta_step":
        o = gbla.delta_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["state"],
                                      slots=s["slots"], out=s["out"])
        return o, s["state"]
    if c["op"] == "score":
        return gbla.token_logprobs(s["logits"], s["tokens"], top=c["top"], scale=c["scale"], seq_lens=s["seq_lens"],
                                   out=s["out"])
    return gbla.token_logprobs_backward(s["logits"], s["lse"], s["entropy"], s["tokens"], dlogprob=s["dlogprob"],
                                        dentropy=s["dentropy"], dlse=s["dlse"], scale=c["scale"],
                                        seq_lens=s["seq_lens"])


# ------------------------------------------------------------- the plain forms

def _cut(x, L):
    """x [B, N, ...] with zeros past the sequences' ends."""
    if L is None:
        return x
    ok = torch.arange(x.shape[1], device=DEV) < L[:, None]
    return torch.where(ok.view(*ok.shape, *[1] * (x.dim() - 2)), x, torch.zeros((), dtype=x.dtype, device=DEV))


CHUNK = 64


def _chunks(x, L, H):
    """[B, N, heads, ...] -> [B, H, chunks, CHUNK, ...], zeros past the ends, shared heads once for each user."""
    x = _cut(x, L)
    if x.shape[2] != H:
        x = x.repeat_interleave(H // x.shape[2], 2)
    n = -(-x.shape[1] // CHUNK)
    x = torch.cat([x, x.new_zeros((x.shape[0], n * CHUNK - x.shape[1], *x.shape[2:]))], 1)
    return x.unflatten(1, (n, CHUNK)).movedim(3, 1)


def _tokens(x, N):
    """The inverse of _chunks."""
    return x.movedim(1, 3).flatten(1, 2)[:, :N]


def _inverse(A):
    """(1 + A)^-1 for strictly lower triangular A [..., CHUNK, CHUNK]: the inverses of diagonal blocks of 1, 2, 4, ..."""
    T = torch.eye(CHUNK, device=DEV, dtype=A.dtype).expand(A.shape).contiguous()
    m = 1
    while m < CHUNK:
        t, a = (x.unflatten(-1, (-1, 2 * m)).unflatten(-3, (-1, 2 * m)).diagonal(dim1=-4, dim2=-2).movedim(-1, -3)
                for x in (T, A))
        t[..., m:, :m] = -(t[..., m:, m:] @ a[..., m:, :m] @ t[..., :m, :m])
        m *= 2
    return T


def _delta_parts(s):
    """What every chunk can form by itself."""
    c, L = s["case"], s["seq_lens"]
    H = c["H"]
    q, k, v, beta = (_chunks(s[n].float(), L, H) for n in ("q", "k", "v", "beta"))
    # sums of the log decays; -inf (which no weight survives) as a number that leaves sums exact
    G = _chunks(s["log_decay"].double().clamp(min=-1e3), L, H).cumsum(-1)
    i = torch.arange(CHUNK, device=DEV)
    gap = (G[..., :, None] - G[..., None, :]).float()
    dec = torch.where(i[:, None] >= i, gap, torch.full((), -math.inf, device=DEV)).exp()
    del gap
    X = (k @ k.transpose(-1, -2) * dec).tril_(-1)
    T = _inverse(beta[..., None] * X)
    up, down, whole = G.float().exp()[..., None], (G[..., -1:] - G).float().exp()[..., None], G[..., -1].float().exp()
    return {"q": q, "k": k, "v": v, "beta": beta[..., None], "dec": dec, "X": X, "T": T, "up": up, "down": down,
            "whole": whole[..., None, None], "P": q @ k.transpose(-1, -2) * dec,
            "w": T @ (beta[..., None] * up * k), "u0": T @ (beta[..., None] * v)}


def _states(s, p):
    """The states before the chunks, one after the other, and after the last; what the chunks' tokens add."""
    c, n = s["case"], p["q"].shape[2]
    S = s["state"] if c["start"] else torch.zeros((c["B"], c["H"], c["D"], c["D"]), device=DEV)
    before, u = [], []
    kd = (p["down"] * p["k"]).transpose(-1, -2)
    for j in range(n):  # the recurrence: each chunk needs the state that the one before leaves
        before.append(S)
        u.append(p["u0"][:, :, j] - p["w"][:, :, j] @ S)
        S = p["whole"][:, :, j] * S + kd[:, :, j] @ u[j]
    return torch.stack(before, 2), torch.stack(u, 2), S


def _plain_delta(s):
    c = s["case"]
    N, scale = s["q"].shape[1], c["D"] ** -0.5
    p = _delta_parts(s)
    S, u, last = _states(s, p)
    o = _tokens((p["up"] * (p["q"] @ S) + p["P"] @ u) * scale, N)
    o = _cut(o.to(s["q"].dtype), s["seq_lens"])
    return (o, last) if c["keep"] else o


def _plain_delta_back(s):
    c, L = s["case"], s["seq_lens"]
    N, H, Hk, scale = s["q"].shape[1], c["H"], c["Hk"], c["D"] ** -0.5
    p = _delta_parts(s)
    S, u, _ = _states(s, p)
    q, k, up, down, whole, dec = (p[n] for n in ("q", "k", "up", "down", "whole", "dec"))
    do = _chunks(s["do"].float(), L, H) * scale
    du0, wt = p["P"].transpose(-1, -2) @ do, p["w"].transpose(-1, -2)
    own_part = (up * q).transpose(-1, -2) @ do
    kd = down * k
    dS = s["dstate"] if c["start"] else torch.zeros((c["B"], H, c["D"], c["D"]), device=DEV)
    n = q.shape[2]
    after, du = [None] * n, [None] * n
    for j in reversed(range(n)):  # the recurrence of the gradients, from the last chunk on
        after[j] = dS
        du[j] = du0[:, :, j] + kd[:, :, j] @ dS
        dS = whole[:, :, j] * dS + own_part[:, :, j] - wt[:, :, j] @ du[j]
    D1, du = torch.stack(after, 2), torch.stack(du, 2)
    dr = p["T"].transpose(-1, -2) @ du
    dv = p["beta"] * dr
    miss = p["v"] - up * (k @ S) - p["X"] @ u
    dbeta = (dr * miss).sum(-1)
    St, kk = S.transpose(-1, -2), k @ k.transpose(-1, -2)
    dP = do @ u.transpose(-1, -2) * dec
    E = (-(dr @ u.transpose(-1, -2)) * dec * p["beta"]).tril_(-1)
    from_q, from_k, to_k = up * (do @ St), -up * (dv @ St), down * (u @ D1.transpose(-1, -2))
    dq = from_q + dP @ k
    dk = dP.transpose(-1, -2) @ q + E @ k + E.transpose(-1, -2) @ k + from_k + to_k
    M = dP * (q @ k.transpose(-1, -2)) + E * kk
    rows = M.double().sum(-1) - M.double().sum(-2)
    at_end = (to_k * k).double().sum(-1)
    dG = rows + (from_q * q + from_k * k).double().sum(-1) - at_end
    dG[..., -1] += at_end.sum(-1) + (whole * S * D1).double().sum((-1, -2))
    dg = dG.flip(-1).cumsum(-1).flip(-1)
    dg = torch.where(_chunks(s["log_decay"], L, H) == -math.inf, torch.zeros((), dtype=dg.dtype, device=DEV), dg)
    dt = s["q"].dtype

    def out(x, share=False):
        x = _tokens(x, N)
        x = x.unflatten(2, (Hk, H // Hk)).sum(3) if share else x
        return _cut(x.to(dt), L)

    got = {"dq": out(dq, True), "dk": out(dk, True), "dv": out(dv), "dlog_decay": out(dg), "dbeta": out(dbeta)}
    if c["start"]:
        got["dstate"] = dS
    return got


def _plain_delta_step(s):
    c = s["case"]
    H, at = c["H"], s["slots"].long()
    q, k = (s[n].float().repeat_interleave(H // c["Hk"], 2)[:, 0] for n in ("q", "k"))
    S = s["log_decay"].float()[:, 0, :, None, None].exp() * s["state"][at]
    miss = s["v"].float()[:, 0] - (k[..., None, :] @ S)[..., 0, :]
    S = S + k[..., :, None] * (s["beta"].float()[:, 0, :, None] * miss)[..., None, :]
    s["state"].index_copy_(0, at, S)
    o = (q[..., None, :] @ S)[..., 0, :] * c["D"] ** -0.5
    s["out"].copy_(o[:, None])
    return s["out"], s["state"]


def _norms(s, to):
    """(log of the sum of exponentials, entropy) of every row of the scaled logits."""
    y = s["logits"].to(to) * s["case"]["scale"]
    m = y.amax(-1, keepdim=True)
    e = (y - m).exp_()
    z = e.sum(-1)
    mean = (e * torch.where(e > 0, y - m, torch.zeros((), dtype=to, device=DEV))).sum(-1) / z
    return m[..., 0] + z.log(), z.log() - mean


def _plain_score(s):
    c, L = s["case"], s["seq_lens"]
    lse, ent = _norms(s, torch.float32)
    y = s["logits"].float() * c["scale"]
    got = {"lse": _cut(lse, L), "entropy": _cut(ent, L)}
    if c["tokens"]:
        has = (s["tokens"] >= 0) & (s["tokens"] < c["V"])
        at = torch.where(has, s["tokens"], 0).long()[..., None]
        got["logprob"] = _cut(torch.where(has, y.gather(-1, at)[..., 0] - lse, torch.zeros((), device=DEV)), L)
    if c["top"]:
        # the order of the logits themselves; equal ones in the tokens' order
        idx = s["logits"].float().sort(dim=-1, descending=True, stable=True).indices[..., :c["top"]]
        got["top_token"] = _cut(idx.int(), L)
        got["top_logprob"] = _cut(y.gather(-1, idx) - lse[..., None], L)
    return got


def _plain_score_back(s):
    c, L = s["case"], s["seq_lens"]
    logp = s["logits"].float() * c["scale"] - s["lse"][..., None]
    p = logp.exp()
    has = (s["tokens"] >= 0) & (s["tokens"] < c["V"])
    dlp = torch.where(has, s["dlogprob"], torch.zeros((), device=DEV))
    inner = torch.where(p > 0, logp, torch.zeros((), device=DEV)) + s["entropy"][..., None]
    d = p * ((s["dlse"] - dlp)[..., None] - s["dentropy"][..., None] * inner)
    d.scatter_add_(-1, torch.where(has, s["tokens"], 0).long()[..., None], dlp[..., None])
    return _cut((d * c["scale"]).to(s["logits"].dtype), L)


def run(state):
    s = state
    if own:
        return _run_own(s)
    return {"delta": _plain_delta, "delta_back": _plain_delta_back, "delta_step": _plain_delta_step,
            "score": _plain_score, "score_back": _plain_score_back}[s["case"]["op"]](s)


# --------------------------------------------------------------------- floors

def work(case):
    op, B, e = case["op"], case["B"], BYTES[case["dtype"]]
    if op.startswith("score"):
        T, V = sum(_lengths(case)), case["V"]
        lens = 4 * B if case["ragged"] else 0
        if op == "score":
            small = T * (8 + 8 * case["tokens"] + 8 * case["top"])
            return {"bytes": T * V * e + small + lens, "flops": T * V * 6}
        pad = (B * _width(case) - T) * V * e  # the padding rows of the gradient are written as zeros
        return {"bytes": 2 * T * V * e + pad + T * 24 + lens, "flops": T * V * 8}
    H, Hk, D = case["H"], case["Hk"], case["D"]
    if op == "delta_step":
        return {"bytes": B * (2 * H * D * D * 4 + (2 * H + 2 * Hk) * D * e + 2 * H * e + 4), "flops": B * H * D * D * 7}
    T = sum(_lengths(case))
    v, k, g = T * H * D * e, T * Hk * D * e, T * H * e
    S = B * H * D * D * 4
    lens = 4 * B if case["ragged"] else 0
    # the recurrent form's operations: decay, two products with the state and one rank-one update a token
    if op == "delta":
        return {"bytes": 2 * v + 2 * k + 2 * g + S * (case["start"] + case["keep"]) + lens, "flops": T * H * D * D * 7}
    pad = (B * _width(case) - T) * ((H + 2 * Hk) * D + 2 * H) * e
    return {"bytes": 3 * v + 4 * k + 4 * g + pad + 3 * S * case["start"] + lens, "flops": T * H * D * D * 18}


# ------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("score"):
        return _exact_score(case, s)
    op, H, D = case["op"], case["H"], case["D"]
    d = {n: x.double() for n, x in s.items() if isinstance(x, torch.Tensor) and x.is_floating_point()}
    wide = lambda x: x[:, torch.arange(H, device=DEV) // (H // case["Hk"])]  # noqa: E731
    scale = 1 / math.sqrt(D)

    def advance(S, t):
        """(decayed state, what the state misses of the value, state after the token)"""
        kept = S * d["log_decay"][:, t].exp()[..., None, None]
        k = wide(d["k"][:, t])
        miss = d["v"][:, t] - torch.einsum("bhd,bhde->bhe", k, kept)
        return kept, miss, kept + torch.einsum("bhd,bhe->bhde", k, d["beta"][:, t, :, None] * miss)

    if op == "delta_step":
        at, pool = s["slots"].long(), d["state"].clone()
        new = advance(pool[at], 0)[2]
        pool[at] = new
        return torch.einsum("bhd,bhde->bhe", wide(d["q"][:, 0]), new)[:, None] * scale, pool
    B, N = s["q"].shape[:2]
    if N * B * H * D * D > (1.6e11 if op == "delta" else 4e9):
        return None
    on = s["seq_lens"].long() if s["seq_lens"] is not None else torch.full((B,), N, device=DEV)
    S = d["state"].clone() if case["start"] else torch.zeros((B, H, D, D), dtype=torch.float64, device=DEV)
    d["v"], d["k"], d["q"] = (torch.nan_to_num(d[n]) for n in ("v", "k", "q"))
    if op == "delta":
        out = torch.zeros((B, N, H, D), dtype=torch.float64, device=DEV)
        for t in range(N):
            live = (t < on)[:, None, None, None]
            S = torch.where(live, advance(S, t)[2], S)
            out[:, t] = torch.einsum("bhd,bhde->bhe", wide(d["q"][:, t]), S) * scale * live[..., 0]
        return (out, S) if case["keep"] else out
    kept = torch.zeros((N, B, H, D, D), dtype=torch.float64, device=DEV)
    miss = torch.zeros((B, N, H, D), dtype=torch.float64, device=DEV)
    dq, dk, dv = (torch.zeros((B, N, H, D), dtype=torch.float64, device=DEV) for _ in range(3))
    dg, db = (torch.zeros((B, N, H), dtype=torch.float64, device=DEV) for _ in range(2))
    for t in range(N):
        live = (t < on)[:, None, None, None]
        kept[t], miss[:, t], new = advance(S, t)
        S = torch.where(live, new, S)
        dq[:, t] = torch.einsum("bhde,bhe->bhd", S, d["do"][:, t]) * scale * live[..., 0]
    A = d["dstate"].clone() if case["start"] else torch.zeros((B, H, D, D), dtype=torch.float64, device=DEV)
    for t in reversed(range(N)):
        live = (t < on)[:, None, None, None].double()
        k, beta = wide(d["k"][:, t]), d["beta"][:, t, :, None]
        now = A + torch.einsum("bhd,bhe->bhde", wide(d["q"][:, t]), d["do"][:, t]) * scale
        grad = torch.einsum("bhd,bhde->bhe", k, now)
        db[:, t] = (grad * miss[:, t]).sum(-1) * live[..., 0, 0]
        dv[:, t] = grad * beta * live[..., 0]
        dk[:, t] = torch.einsum("bhde,bhe->bhd", now, beta * miss[:, t]) - torch.einsum("bhde,bhe->bhd", kept[t], beta * grad)
        dk[:, t] *= live[..., 0]
        now = now - torch.einsum("bhd,bhe->bhde", k, beta * grad)
        dg[:, t] = (now * kept[t]).sum((-1, -2)) * live[..., 0, 0]
        A = torch.where(live > 0, now * d["log_decay"][:, t].exp()[..., None, None], A)
    shared = lambda x: x.view(B, N, case["Hk"], -1, D).sum(3)  # noqa: E731
    got = {"dq": shared(dq), "dk": shared(dk), "dv": dv, "dlog_decay": dg, "dbeta": db}
    if case["start"]:
        got["dstate"] = A
    return got


def _exact_score(case, s):
    """Some rows at a time: log softmax by its definition."""
    B, N, V = s["logits"].shape
    on = _lengths(case)
    step = max(1, 40_000_000 // V)
    flat, rows = s["logits"].view(B * N, V), {}
    valid = torch.tensor([t < on[b] for b in range(B) for t in range(N)], device=DEV)
    for r in range(0, B * N, step):
        y = flat[r:r + step].double() * case["scale"]
        lse = torch.logsumexp(y, -1)
        lp = y - lse[:, None]
        p = lp.exp()
        safe = torch.where(p > 0, lp, 0.0)
        ent = -(p * safe).sum(-1)
        ok = valid[r:r + step]
        tok = None if s["tokens"] is None else s["tokens"].view(-1)[r:r + step].long()
        if tok is not None:
            has = (tok >= 0) & (tok < V) & ok
            tok = torch.where(has, tok, 0)
        if case["op"] == "score":
            got = {"lse": lse, "entropy": ent}
            if tok is not None:
                got["logprob"] = torch.where(has, lp.gather(-1, tok[:, None])[:, 0], 0.0)
            if case["top"]:
                got["top_logprob"] = lp.topk(case["top"], -1).values
        else:
            one, two, three = (s[n].view(-1)[r:r + step, None].double() for n in ("dlogprob", "dentropy", "dlse"))
            one = torch.where(has[:, None], one, 0.0)
            g = -p * one - two * p * (safe + ent[:, None]) + three * p
            g[torch.arange(len(g), device=DEV), tok] += one[:, 0]
            got = {"d": g * case["scale"]}
            if case["dtype"] == "bf16":  # keeps the memory low; far finer than the type
                got["d"] = got["d"].float()
        for n, x in got.items():
            x = torch.where(ok.view(-1, *[1] * (x.dim() - 1)), x, 0.0)
            rows.setdefault(n, []).append(x)
    got = {n: torch.cat(x).unflatten(0, (B, N)) for n, x in rows.items()}
    return got["d"] if case["op"] == "score_back" else got
