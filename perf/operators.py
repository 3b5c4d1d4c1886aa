"""The operators that keep a user's history between requests, as cases to be measured.

Two ways of holding a history next to the rank-r factors of `lowrank_factor`:

  linear attention with a decay per head (`linear_attention_fwd`, `_bwd`, `_step`): the history is a d x d state
      S_t = g S_{t-1} + k_t v_t^T,  o_t = scale q_t S_t,  g = exp(log_decay[h])
  the history itself in 8 bits (`history_cache_append`, `history_cache_attention`): e4m3 rows [B,H,capacity,d] with a
      power-of-two scale for every block of 64 tokens and head, and softmax attention over them

`op` of a case says which calls make up a pass:

  forward   a whole history through linear attention, its last state out
  train     forward and backward of a padded batch, gradients of q, k, v and of the first state
  step      one new event per user: the state is updated in place
  serve     new tokens go into the cache, then queries attend over it (causal: the queries are the new tokens)
  attend    queries (candidates) over a cache that was filled earlier

Histories have the lengths of this repository's workloads (50 to 32768 positions, 16 to 4096 candidates, embeddings of
32, 64 and 128).
"""
import math

import torch

own = False

BLOCK = 64                                      # tokens that share a scale
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_E4M3 = torch.float8_e4m3fn


def _linear(name, op, dtype, B, T, H, d, ragged=False):
    return {"name": name, "op": op, "dtype": dtype, "B": B, "T": T, "H": H, "d": d, "ragged": ragged}


def _cache(name, op, dtype, B, N, new, M, Hq, H, d, ragged=False, causal=False):
    """N: capacity; new: tokens appended; M: queries per user; Hq query heads over H cached heads."""
    return {"name": name, "op": op, "dtype": dtype, "B": B, "N": N, "new": new, "M": M, "Hq": Hq, "H": H, "d": d,
            "ragged": ragged, "causal": causal}


def listed():
    return [
        # one request with a short history: launches and latency
        _linear("linear_short", "forward", "bf16", 1, 200, 4, 64),
        # the headline batch's histories
        _linear("linear_histories", "forward", "bf16", 16, 10240, 4, 64),
        # a training step on padded batches, both embedding widths
        _linear("linear_train", "train", "bf16", 8, 4096, 8, 64, True),
        _linear("linear_train_wide", "train", "bf16", 4, 2047, 8, 128),
        # the fp32 storage mode, a length and a head count that divide nothing
        _linear("linear_train_f32", "train", "f32", 3, 777, 5, 32, True),
        # one new event for every user of a serving batch, and for a single one
        _linear("linear_event_batch", "step", "bf16", 256, 1, 8, 64),
        _linear("linear_event_one", "step", "f32", 1, 1, 4, 128),
        # one event of one user: into the cache, then one query over 10,000 positions
        _cache("cache_event_one", "serve", "bf16", 1, 10240, 1, 1, 8, 2, 64),
        # the same for a serving batch of users with different lengths: bandwidth of the 8-bit rows
        _cache("cache_event_batch", "serve", "bf16", 64, 16384, 1, 1, 8, 2, 128, True),
        # new histories are taken in, each event attending over what came before it
        _cache("cache_prompt", "serve", "bf16", 4, 2048, 1950, 1950, 8, 2, 64, True, True),
        # the headline batch: 2048 candidates over 10240 positions
        _cache("cache_candidates", "attend", "bf16", 16, 10240, 0, 2048, 1, 1, 64),
        # the fp32 storage mode, few candidates
        _cache("cache_candidates_f32", "attend", "f32", 2, 5056, 0, 120, 1, 1, 32, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["forward", "forward", "train", "train", "step", "serve", "serve", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = rng.choice([32, 64, 64, 128])
    if op in ("forward", "train", "step"):
        H = _log(rng, 1, 16)
        T = 1 if op == "step" else _log(rng, 1, 10240 if op == "forward" else 4096)
        most = (1 << 25) // (T * H * d) if op != "step" else (1 << 23) // (H * d * d)
        if dtype == "f32":
            most //= 4
        return {k: v for k, v in _linear("", op, dtype, _log(rng, 1, max(1, min(256, most))), T, H, d,
                                         op == "train" and rng.random() < 0.5).items() if k != "name"}
    H = _log(rng, 1, 4)
    Hq = H * rng.choice([1, 2, 4])
    N = -(-_log(rng, 50, 32768) // BLOCK) * BLOCK
    if op == "serve":
        causal = rng.random() < 0.5
        new = _log(rng, 1, min(N, 2048)) if causal else rng.choice([1, 1, 2, 5])
        M = new if causal else 1
    else:
        causal, new, M = False, 0, _log(rng, 1, 4096)
    cost = N * d * H + M * N * Hq * d / (32 if dtype == "bf16" else 4)
    most = int((1 << 28) / cost)
    return {k: v for k, v in _cache("", op, dtype, _log(rng, 1, max(1, min(64, most))), N, new, M, Hq, H, d,
                                    rng.random() < 0.5, causal).items() if k != "name"}


# ---- inputs -------------------------------------------------------------------------------------
def _lengths(gen, B, lo, hi, ragged):
    if not ragged:
        return torch.full((B,), hi, dtype=torch.int32, device="cuda")
    return torch.randint(lo, hi + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 17)
    dt = _DTYPES[case["dtype"]]
    B, H, d = case["B"], case["H"], case["d"]

    def normal(*shape, dtype=dt):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)

    s = {"case": case, "scale": 1.0 / math.sqrt(d)}
    if case["op"] in ("forward", "train", "step"):
        T = case["T"]
        # memories from some ten events (the first head) to about a thousand (the last)
        s["log_decay"] = -torch.exp2(-3.0 - 7.0 * torch.arange(H, device="cuda", dtype=torch.float32) / max(1, H - 1))
        if case["op"] == "step":
            s.update(q=normal(B, H, d), k=normal(B, H, d), v=normal(B, H, d), state=normal(B, H, d, d, dtype=torch.float32))
            return s
        # q, k and v as a program has them: parts of one projection's output
        qkv = normal(B, T, 3, H, d)
        s.update(q=qkv[:, :, 0], k=qkv[:, :, 1], v=qkv[:, :, 2], state0=normal(B, H, d, d, dtype=torch.float32))
        s["lengths"] = _lengths(gen, B, T // 2, T, True) if case["ragged"] else None
        if case["op"] == "train":
            s.update(dO=normal(B, T, H, d), dstate=normal(B, H, d, d, dtype=torch.float32))
        return s

    N, new, M, Hq = case["N"], case["new"], case["M"], case["Hq"]
    s["q"] = normal(B, M, Hq, d)
    s["flags"] = case["causal"]
    held = _lengths(gen, B, (N - new) // 2, N - new, case["ragged"])        # tokens in the cache before the pass
    if case["causal"]:
        held = held % BLOCK if case["ragged"] and new + BLOCK <= N else held * 0
    # what earlier calls left: rows of differing size in 8 bits, the unused end of the cache never written
    for x in ("k", "v"):
        rows = torch.randn(B, H, N // BLOCK, BLOCK, d, generator=gen, device="cuda", dtype=torch.float32)
        rows *= torch.exp2(torch.randn(B, H, N // BLOCK, 1, 1, generator=gen, device="cuda"))
        e = _exponent(rows.abs().amax(dim=(3, 4)))
        s[x + "_scale"] = _two_to(e)
        s[x + "8"] = (rows * _two_to(-e)[..., None, None]).to(_E4M3).view(B, H, N, d)
        del rows
    s["start"] = held
    s["lengths"] = (held + new).to(torch.int32)
    if new:
        kv = normal(B, new, 2, H, d)
        s.update(k=kv[:, :, 0], v=kv[:, :, 1])
    return s


# ---- linear attention, plain ----------------------------------------------------------------------
def _powers(log_decay, n):
    """g^n for whole numbers n >= 0, [H, *n.shape]; 64-bit angles of far positions, rounded once."""
    return torch.exp(log_decay.double().view(-1, *[1] * n.dim()) * n.double()).float()


def _chunked(q, k, v, init, log_decay, off):
    """o_x = sum_{y <= x} g^(x-y) (q_x . k_y) v_y + g^(x+off) q_x . init, all [B,H,T,d] fp32."""
    B, H, T, d = q.shape
    C = BLOCK
    n = -(-T // C)
    q_, k_, v_ = (torch.nn.functional.pad(x, (0, 0, 0, n * C - T)).view(B, H, n, C, d) for x in (q, k, v))
    i = torch.arange(C, device=q.device)
    gap = i[:, None] - i[None, :]
    near = torch.where(gap >= 0, _powers(log_decay, gap.clamp(min=0)), torch.zeros((), device=q.device))
    o = ((q_ @ k_.transpose(-1, -2)) * near[:, None]) @ v_
    left = (k_ * _powers(log_decay, C - 1 - i)[:, None, :, None]).transpose(-1, -2) @ v_           # [B,H,n,d,d]
    c = torch.arange(n, device=q.device)
    far = c[:, None] - c[None, :] - 1
    carry = torch.where(far >= 0, _powers(log_decay, C * far.clamp(min=0)), torch.zeros((), device=q.device))
    before = (carry @ left.reshape(B, H, n, d * d)).view(B, H, n, d, d)
    o = o + (q_ @ before) * _powers(log_decay, i + 1)[:, None, :, None]
    o = o.reshape(B, H, n * C, d)[:, :, :T]
    return o + (q @ init) * _powers(log_decay, torch.arange(T, device=q.device) + off)[:, :, None]


def _sums(k, v, init, log_decay, lengths, off):
    """g^L init + sum_{x < L} g^(L-1-x+off) k_x v_x^T for every user's length L."""
    T = k.shape[2]
    x = torch.arange(T, device=k.device)
    n = lengths.long()[:, None] - 1 - x
    w = torch.where(n >= 0, _powers(log_decay, n.clamp(min=0) + off), torch.zeros((), device=k.device))      # [H,B,T]
    return (k * w.transpose(0, 1)[..., None]).transpose(-1, -2) @ v + init * _powers(log_decay, lengths.long()).t()[..., None, None]


def _heads(x, real):
    return torch.where(real, x.float().transpose(1, 2), torch.zeros((), device=x.device))


def _linear_plain(s):
    case, ld, scale = s["case"], s["log_decay"], s["scale"]
    B, T, H, d = s["q"].shape
    dt = s["q"].dtype
    x = torch.arange(T, device=ld.device)
    lengths = s["lengths"] if s["lengths"] is not None else torch.full((B,), T, dtype=torch.int32, device=ld.device)
    real = (x < lengths[:, None])[:, None, :, None]
    q, k, v = (_heads(s[n], real) for n in "qkv")
    out = lambda y: torch.where(real, y, torch.zeros((), device=ld.device)).transpose(1, 2).to(dt)  # noqa: E731
    O, state = out(scale * _chunked(q, k, v, s["state0"], ld, 1)), _sums(k, v, s["state0"], ld, lengths, 0)
    if case["op"] == "forward":
        return {"O": O, "state": state}
    do = _heads(s["dO"], real)
    dq = scale * _chunked(do, v, k, s["state0"].transpose(-1, -2), ld, 1)
    # reversed time within every user's length
    at = (lengths.long()[:, None] - 1 - x).clamp(min=0)[:, None, :, None].expand(B, H, T, d)
    back = lambda y: torch.where(real, y.gather(2, at), torch.zeros((), device=ld.device))  # noqa: E731
    rq, rk, rv, rdo = back(q) * scale, back(k), back(v), back(do)
    dk = back(_chunked(rv, rdo, rq, s["dstate"].transpose(-1, -2), ld, 0))
    dv = back(_chunked(rk, rq, rdo, s["dstate"], ld, 0))
    dstate0 = _sums(rq, rdo, s["dstate"], ld, lengths, 1)
    return {"O": O, "state": state, "dq": out(dq), "dk": out(dk), "dv": out(dv), "dstate0": dstate0}


def _step_plain(s):
    q, k, v = (s[n].float() for n in "qkv")
    g = torch.exp(s["log_decay"].double()).float()
    s["state"] = state = g[:, None, None] * s["state"] + k[..., :, None] * v[..., None, :]
    return {"O": (s["scale"] * (q[..., None, :] @ state)[..., 0, :]).to(s["q"].dtype), "state": state}


# ---- the 8-bit cache, plain -----------------------------------------------------------------------
def _exponent(amax):
    """Smallest whole e with amax <= 448 * 2^e, at least -100."""
    m, x = torch.frexp(amax)
    return torch.where(m <= 0.875, x - 9, x - 8).clamp(min=-100).masked_fill(amax == 0, -100)


def _two_to(e):
    """2^e exactly, for whole -126 <= e <= 127: a quotient by a scale must not move a tie."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _append_plain(s, x):
    rows, cache, scales, start = s[x], s[x + "8"], s[x + "_scale"], s["start"].long()
    B, new, H, d = rows.shape
    rows = rows.float().transpose(1, 2)
    pos = start[:, None] + torch.arange(new, device=rows.device)
    blk = (pos // BLOCK)[:, None, :].expand(B, H, new)
    amax = torch.zeros_like(scales).scatter_reduce(2, blk, rows.abs().amax(dim=3), "amax", include_self=True)
    touched = torch.zeros_like(scales).scatter(2, blk, 1.0) > 0
    n = torch.arange(scales.shape[2], device=rows.device)
    kept = (n == start[:, None] // BLOCK) & (start[:, None] % BLOCK > 0)                # blocks that hold older rows
    fresh = _exponent(amax)
    e = torch.where(kept[:, None, :], torch.maximum(fresh, torch.frexp(scales)[1] - 1), fresh)
    after = torch.where(touched, _two_to(e), scales)
    # the older rows of the block that the first new one falls into
    b, h = torch.arange(B, device=rows.device)[:, None, None], torch.arange(H, device=rows.device)[None, :, None]
    first = (start // BLOCK).clamp(max=scales.shape[2] - 1)
    old_at = first[:, None] * BLOCK + torch.arange(BLOCK, device=rows.device)
    older = (old_at < start[:, None])[:, None, :, None]
    old = cache.view(torch.uint8)[b, h, old_at[:, None, :]].view(_E4M3)
    shift = (scales.gather(2, first[:, None, None].expand(B, H, 1)) / after.gather(2, first[:, None, None].expand(B, H, 1)))
    moved = (old.float() * shift[..., None]).to(_E4M3)
    cache.view(torch.uint8)[b, h, old_at[:, None, :]] = torch.where(older, moved.view(torch.uint8), old.view(torch.uint8))
    cache.view(torch.uint8)[b, h, pos[:, None, :]] = (rows / after.gather(2, blk)[..., None]).to(_E4M3).view(torch.uint8)
    s[x + "_scale"] = after


def _attend_plain(s):
    B, M, Hq, d = s["q"].shape
    H, N = s["k8"].shape[1], s["k8"].shape[2]
    K, V = ((s[x + "8"].float().view(B, H, N // BLOCK, BLOCK, d) * s[x + "_scale"][..., None, None]).view(B, H, 1, N, d) for x in "kv")
    q = s["q"].float().view(B, M, H, Hq // H, d).permute(0, 2, 3, 1, 4)
    n = torch.arange(N, device=q.device)
    last = s["lengths"].long()[:, None] - 1 + (torch.arange(M, device=q.device) - (M - 1) if s["flags"] else torch.zeros(M, device=q.device, dtype=torch.long))
    seen = (n <= last[..., None])[:, None, None]                                                  # [B,1,1,M,N]
    p = (q @ K.transpose(-1, -2)) * s["scale"]
    p = torch.where(seen, p, torch.full((), -math.inf, device=q.device))
    top = p.amax(dim=-1, keepdim=True)
    p = torch.exp(p - torch.where(top > -math.inf, top, torch.zeros((), device=q.device)))
    held = (n < s["lengths"][:, None])[:, None, None, :, None]
    o = p @ torch.where(held, V, torch.zeros((), device=q.device))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.where(total > 0, o / total, torch.zeros((), device=q.device))
    return o.permute(0, 3, 1, 2, 4).reshape(B, M, Hq, d).to(s["q"].dtype)


# ---- one pass -------------------------------------------------------------------------------------
def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    if op == "step":
        return _step_plain(s)
    if op in ("forward", "train"):
        return _linear_plain(s)
    if op == "serve":
        _append_plain(s, "k")
        _append_plain(s, "v")
    O = _attend_plain(s)
    return {"O": O} if op == "attend" else {"O": O, "k8": s["k8"], "v8": s["v8"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _run_own(s, op):
    from paper_2603_02561_b200 import solar
    if op == "step":
        O = solar.linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["state"])
        return {"O": O, "state": s["state"]}
    if op in ("forward", "train"):
        O, last = solar.linear_attention_fwd(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], state0=s["state0"], lengths=s["lengths"])
        if op == "forward":
            return {"O": O, "state": last}
        dq, dk, dv, dstate0 = solar.linear_attention_bwd(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], s["dO"], state0=s["state0"],
                                                         dstate=s["dstate"], lengths=s["lengths"])
        return {"O": O, "state": last, "dq": dq, "dk": dk, "dv": dv, "dstate0": dstate0}
    cache = solar.HistoryCache(s["k8"], s["v8"], s["k_scale"], s["v_scale"])
    if op == "serve":
        solar.history_cache_append(s["k"], s["v"], cache, s["start"])
    O = solar.history_cache_attention(s["q"], cache, s["lengths"], s["scale"], flags=solar.FLAG_CAUSAL if s["flags"] else 0)
    return {"O": O} if op == "attend" else {"O": O, "k8": s["k8"], "v8": s["v8"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    B, H, d = case["B"], case["H"], case["d"]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("forward", "train", "step"):
        tokens = B * case["T"] * H
        state = B * H * d * d * 4
        if case["op"] == "train":          # q k v in, o out, then q k v do in, three gradients out; four states
            return {"bytes": 11 * tokens * d * e + 4 * state, "flops": 12 * tokens * d * d}
        return {"bytes": 4 * tokens * d * e + 2 * state, "flops": 4 * tokens * d * d}
    # ragged caches are three quarters full on average; a causal query sees half of what is held
    N, new, M = case["N"], case["new"], case["M"]
    held = (N - new) * (0.75 if case["ragged"] else 1.0)
    if case["causal"]:
        held = BLOCK / 2 if case["ragged"] and new + BLOCK <= N else 0
    seen = held + new / 2 if case["causal"] else held + new
    nbytes = 2 * B * H * (held + new) * (d + 4 / BLOCK) + 2 * B * M * case["Hq"] * d * e + 2 * B * new * H * d * e
    return {"bytes": nbytes, "flops": 4 * B * M * case["Hq"] * seen * d}


# ---- the definitions in 64 bits -----------------------------------------------------------------------
def _exact_linear(s):
    """The recurrences, one event after the other."""
    ld, scale, op = s["log_decay"].double(), s["scale"], s["case"]["op"]
    g = torch.exp(ld)[:, None, None]
    if op == "step":
        S = g * s["state"].double() + torch.einsum("bhi,bhj->bhij", s["k"].double(), s["v"].double())
        return {"O": scale * torch.einsum("bhi,bhij->bhj", s["q"].double(), S), "state": S}
    B, T, H, d = s["q"].shape
    lengths = s["lengths"].tolist() if s["lengths"] is not None else [T] * B
    q, k, v = (s[n].double() for n in "qkv")
    S = s["state0"].double().clone()
    O = torch.zeros(B, T, H, d, dtype=torch.float64, device=ld.device)
    train = op == "train"
    do = s["dO"].double() if train else None
    dq, dk, dv = (torch.zeros_like(O) for _ in range(3)) if train else (None, None, None)
    order = sorted(range(B), key=lambda b: -lengths[b])
    idx = torch.tensor(order, device=ld.device)
    q, k, v, S = q[idx], k[idx], v[idx], S[idx]
    do = do[idx] if train else None
    count = [sum(n > t for n in lengths) for t in range(T)]                 # the users that still have an event t
    for t in range(max(lengths)):
        a = count[t]
        S[:a] = g * S[:a] + k[:a, t, :, :, None] * v[:a, t, :, None, :]
        O[:a, t] = scale * (q[:a, t, :, None, :] @ S[:a])[..., 0, :]
        if train:
            dq[:a, t] = scale * (S[:a] @ do[:a, t, :, :, None])[..., 0]
    undo = torch.argsort(idx)
    out = {"O": O[undo], "state": S[undo]}
    if train:
        R = s["dstate"].double()[idx].clone()
        for t in range(max(lengths) - 1, -1, -1):
            a = count[t]
            R[:a] += scale * q[:a, t, :, :, None] * do[:a, t, :, None, :]
            dk[:a, t] = (R[:a] @ v[:a, t, :, :, None])[..., 0]
            dv[:a, t] = (k[:a, t, :, None, :] @ R[:a])[..., 0, :]
            R[:a] *= g
        out.update(dq=dq[undo], dk=dk[undo], dv=dv[undo], dstate0=R[undo])
    return out


def _exact_round8(x):
    """To the nearest e4m3 value, ties to even; |x| <= 448."""
    e = (torch.frexp(x)[1] - 1).clamp(min=-6)
    step = _two_to(e - 3).double()
    return torch.round(x / step) * step


def _exact_cache(s):
    case = s["case"]
    B, M, Hq, d = s["q"].shape
    H, N = case["H"], case["N"]
    out, small = {}, B * H * N * d <= 1 << 26
    O = torch.zeros(B, M, Hq, d, dtype=torch.float64, device=s["q"].device)
    held = {x: s[x + "8"].double() for x in "kv"} if small else None
    scales = {x: s[x + "_scale"].double() for x in "kv"}
    start, lengths = s["start"].tolist(), s["lengths"].tolist()
    for b in range(B):
        kv = {}
        for x in "kv":
            c = held[x][b] if small else s[x + "8"][b].double()
            sc = scales[x][b]
            if case["op"] == "serve":
                p0, p1 = start[b], lengths[b]
                for n in range(p0 // BLOCK, (p1 - 1) // BLOCK + 1):
                    lo, hi = max(p0, n * BLOCK), min(p1, (n + 1) * BLOCK)
                    new = s[x][b, lo - p0:hi - p0].double().transpose(0, 1)
                    top = new.abs().amax(dim=(1, 2))
                    grid = _two_to(torch.arange(-100, 121, device=top.device)).double()
                    at = torch.searchsorted(448 * grid, top)                     # the first e with top <= 448 * 2^e
                    if lo > n * BLOCK:
                        at = torch.maximum(at, torch.searchsorted(grid, sc[:, n].contiguous()))
                        old = c[:, n * BLOCK:lo]
                        c[:, n * BLOCK:lo] = _exact_round8(old * (sc[:, n] / grid[at])[:, None, None])
                    sc[:, n] = grid[at]
                    c[:, lo:hi] = _exact_round8(new / sc[:, n][:, None, None])
            kv[x] = c[:, :lengths[b]] * sc.repeat_interleave(BLOCK, dim=1)[:, :lengths[b], None]
        for m0 in range(0, M, 512):
            q = s["q"][b, m0:m0 + 512].double()
            at = lengths[b] - M + m0 + torch.arange(q.shape[0], device=q.device)
            for h in range(Hq):
                z = s["scale"] * q[:, h] @ kv["k"][h * H // Hq].T
                if case["causal"]:
                    z = z.masked_fill(torch.arange(lengths[b], device=q.device) > at[:, None], -math.inf)
                O[b, m0:m0 + 512, h] = torch.nan_to_num(torch.softmax(z, dim=-1)) @ kv["v"][h * H // Hq]
    out = {"O": O}
    if case["op"] == "serve":
        out.update(k8=held["k"] if small else None, v8=held["v"] if small else None, k_scale=scales["k"], v_scale=scales["v"])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("forward", "train", "step"):
        return _exact_linear(s)
    heavy = case["B"] * case["M"] * case["Hq"] * case["N"] * case["d"] > 1 << 37 or case["B"] * case["Hq"] * (case["M"] // 512 + 1) > 1 << 13
    return None if heavy else _exact_cache(s)
