"""The timed operators between the matrix products of a decoder layer whose activations and attention cache are held in 8 bits.

Every case is a plain dict:

    op     "norm"    root-mean-square norm of x (+ residual), int8 codes with one scale per row
           "gate"    silu(gate) * up, int8 codes with one scale per row
           "append"  keys and values into a paged 8-bit cache, keys and queries rotated on the way
           "attn"    attention of new rows over such a cache
    act    "f16" | "bf16": activations and results
    M, N   rows and columns ("norm", "gate"); residual: whether one is added ("norm")
    batch, rows, ctx   sequences, most new rows and most tokens already there, of one sequence; ragged: lengths are spread below
           these, drawn from the number `lens` (else all alike)
    qh, kvh, dim   query heads, key/value heads, size of a head
    kv     "i8" | "e4m3": what the cache holds
    rot, pairs   "append": rotated dimensions of a head, "halves" | "neighbours"
    causal, window   "attn": rows see keys up to their own place / the last `window` of those (0: all)

A cache block is 64 tokens of one head, with one scale for its keys and one for its values:

    keys    token 16 t + i, dimension 64 c + 16 b + e   at byte   (((t * dim/64 + c) * 4 + b) * 16 + i) * 16 + e
    values  token 16 t + 4 b + r, dimension 16 d + i    at byte   ((d * 4 + b) * 16 + i) * 16 + 4 t + r

int8 codes are stored plus 128.  8-bit results are returned as the values that they stand for.
"""
import math
import random

import torch

own = False

_DT = {"f16": torch.float16, "bf16": torch.bfloat16}
_QMAX = {"i8": 127.0, "e4m3": 448.0}
BLOCK = 64
EPS = 1e-5
TINY = 2.0 ** -40          # least scale
DEV = "cuda"


def _rows_case(name, op, M, N, act, residual=True):
    c = {"op": op, "M": M, "N": N, "act": act}
    if op == "norm":
        c["residual"] = residual
    return {"name": name, **c} if name else c


def _kv_case(name, op, batch, rows, ctx, qh, kvh, dim, act, kv, ragged=True, lens=1, rot=0, pairs="halves", causal=True, window=0):
    c = {"op": op, "batch": batch, "rows": rows, "ctx": ctx, "ragged": ragged, "lens": lens, "qh": qh, "kvh": kvh,
         "dim": dim, "act": act, "kv": kv}
    c.update({"rot": rot, "pairs": pairs} if op == "append" else {"causal": causal, "window": window})
    return {"name": name, **c} if name else c


def listed():
    return [
        # One token of one sequence, hidden size 4096: all latency.
        _rows_case("norm_one_row", "norm", 1, 4096, "f16"),
        # A large decode batch, ragged row count.
        _rows_case("norm_rows300", "norm", 300, 8192, "bf16"),
        # A prompt of 4096 tokens.
        _rows_case("norm_prompt", "norm", 4096, 8192, "bf16"),
        # The inner size of a layer for a decode batch ...
        _rows_case("gate_rows16", "gate", 16, 14336, "f16"),
        # ... and of a large one for a prompt of odd length.
        _rows_case("gate_prompt", "gate", 1000, 28672, "bf16"),
        # One decode step of sixteen sequences that are at different places.
        _kv_case("append_decode16", "append", 16, 1, 2000, 32, 8, 128, "f16", "e4m3", rot=128),
        # Prompts of four sequences, some with tokens in the cache already; part of the head is rotated.
        _kv_case("append_prompts", "append", 4, 1500, 500, 64, 8, 128, "bf16", "i8", rot=64, pairs="neighbours"),
        # One token of one sequence with a short history: latency.
        _kv_case("attn_one", "attn", 1, 1, 1000, 32, 8, 128, "f16", "i8", ragged=False),
        # Decode of a large batch with histories of all lengths: streaming the cache.
        _kv_case("attn_decode64", "attn", 64, 1, 8000, 64, 8, 128, "bf16", "i8"),
        # One sequence with a very long history: few rows, the history is all the parallelism there is.
        _kv_case("attn_long", "attn", 1, 1, 131070, 64, 8, 128, "bf16", "e4m3", ragged=False),
        # Chunks of prompts on top of histories, small heads.
        _kv_case("attn_chunks", "attn", 4, 600, 3500, 40, 8, 64, "f16", "e4m3", lens=3),
        # The largest: a prompt of 8192 tokens.
        _kv_case("attn_prompt", "attn", 1, 8192, 0, 64, 8, 128, "bf16", "i8", ragged=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "gate", "append", "attn", "attn"])
    act = rng.choice(["f16", "bf16"])
    if op in ("norm", "gate"):
        # any width that the int8 product takes
        N = 128 * _log(rng, 4, 64 if op == "norm" else 224)
        N += 128 * (N in (1536, 3072))            # widths that no layer here has
        M = _log(rng, 1, 4096 if op == "norm" else 28672000 // N)
        return _rows_case(None, op, M, N, act, rng.random() < 0.8)
    kvh = rng.choice([1, 2, 4, 8])
    qh = kvh * rng.choice([1, 2, 4, 5, 7, 8])
    dim = rng.choice([64, 128, 128])
    qh += kvh * ((qh + 2 * kvh) * dim == 3072)
    kv = rng.choice(["i8", "e4m3"])
    lens = rng.randrange(1 << 20)
    if op == "append":
        batch = _log(rng, 1, 128)
        rows = 1 if rng.random() < 0.4 else _log(rng, 2, max(2, 6000 // batch))
        return _kv_case(None, op, batch, rows, _log(rng, 1, 4000), qh, kvh, dim, act, kv, lens=lens,
                        rot=rng.choice([dim, dim // 2, 0]), pairs=rng.choice(["halves", "neighbours"]))
    if rng.random() < 0.5:                    # decode, up to a few tokens a sequence
        batch = _log(rng, 1, 64)
        rows, ctx = rng.choice([1, 1, 1, 2, 5]), _log(rng, 1, min(120000, 450000 // batch))
    else:                                     # (chunks of) prompts
        batch = _log(rng, 1, 8)
        rows = _log(rng, 8, 4096 // batch)
        ctx = _log(rng, 1, 8000 // batch)
    return _kv_case(None, op, batch, rows, ctx, qh, kvh, dim, act, kv, lens=lens, causal=rng.random() < 0.8,
                    window=rng.choice([0, 0, 0, _log(rng, 16, 4000)]))


def _lengths(c):
    """New rows and whole length (with them) of each sequence."""
    if not c["ragged"]:
        return [c["rows"]] * c["batch"], [c["ctx"] + c["rows"]] * c["batch"]
    r = random.Random(c["lens"])
    new = [r.randint((c["rows"] + 1) // 2, c["rows"]) for _ in range(c["batch"])]
    before = [r.randint(c["ctx"] // 8, c["ctx"]) for _ in range(c["batch"])]
    return new, [a + b for a, b in zip(new, before)]


def _pairs(c, new, length):
    """(visible pairs of row and key, keys that some row sees) of one sequence."""
    pairs, seen_from = 0, length
    for j in range(new):
        pos = length - new + j
        hi = pos + 1 if c["causal"] else length
        lo = max(0, pos - c["window"] + 1) if c["window"] else 0
        pairs += max(0, hi - lo)
        seen_from = min(seen_from, lo)
    return pairs, length - seen_from


def work(case):
    c = case
    if c["op"] == "norm":
        n = c["M"] * c["N"]
        return {"bytes": n * (2 + 1 + (4 if c["residual"] else 0)) + 4 * c["M"] + 2 * c["N"], "flops": 8 * n}
    if c["op"] == "gate":
        n = c["M"] * c["N"]
        return {"bytes": 5 * n + 4 * c["M"], "flops": 8 * n}
    new, length = _lengths(c)
    T, d = sum(new), c["dim"]
    if c["op"] == "append":
        return {"bytes": T * d * (4 * c["qh"] + 6 * c["kvh"]) + T * c["rot"] * 4, "flops": T * (3 * c["rot"] * (c["qh"] + c["kvh"]) + 4 * d * c["kvh"])}
    pk = [_pairs(c, a, b) for a, b in zip(new, length)]
    return {"bytes": 4 * T * c["qh"] * d + sum(k for _, k in pk) * c["kvh"] * (2 * d + 8 / BLOCK),
            "flops": 4 * d * c["qh"] * sum(p for p, _ in pk)}


# ---- inputs ---------------------------------------------------------------------------------

def _encode(x, scale, kv):
    """Codes (as bytes) of x / scale."""
    if kv == "i8":
        return (torch.round(x / scale).clamp_(-127, 127) + 128).to(torch.uint8)
    return (x / scale).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(DEV).manual_seed(int(seed))
    act = _DT[c["act"]]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=DEV) * std

    s = {"case": c}
    if c["op"] == "norm":
        # channels of very different size, as hidden states have them
        channel = torch.exp(0.7 * normal(c["N"]))
        s["x"] = (normal(c["M"], c["N"]) * channel).to(act)
        s["residual"] = (normal(c["M"], c["N"], std=3.0) * channel).to(act) if c["residual"] else None
        s["w"] = (1 + normal(c["N"], std=0.2)).to(act)
        return s
    if c["op"] == "gate":
        s["gu"] = normal(c["M"], 2 * c["N"], std=1.5).to(act)
        return s
    new, length = _lengths(c)
    B, H, D, T = c["batch"], c["kvh"], c["dim"], sum(new)
    width = -(-max(length) // BLOCK) + 1                      # a block more than is needed now, as a cache that grows has
    used = [-(-n // BLOCK) for n in length]
    blocks = sum(used) + 3
    order = torch.randperm(blocks, generator=g, device=DEV).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["row_start"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["kv_len"] = torch.tensor(length, dtype=torch.int32, device=DEV)
    s["table"], s["max_rows"], s["max_kv"] = table, max(new), max(length)
    # the cache's content: blocks of unlike magnitude, each with the scales that its largest values ask for
    for name in ("k", "v"):
        x = normal(blocks, H, BLOCK * D) * torch.exp(0.5 * normal(blocks, H, 1))
        scale = (x.abs().amax(-1, keepdim=True) / _QMAX[c["kv"]]).clamp_min(TINY)
        s[name + "_cache"], s[name + "_scale"] = _encode(x, scale, c["kv"]), scale[..., 0].contiguous()
        del x
    if c["op"] == "append":
        # rows as the product of a layer's q, k, v projection leaves them: side by side
        s["qkv"] = normal(T, (c["qh"] + 2 * H) * D, std=1.5).to(act)
        if c["rot"]:
            half = c["rot"] // 2
            angle = torch.arange(max(length), device=DEV, dtype=torch.float64)[:, None] * 500000.0 ** (
                -torch.arange(half, device=DEV, dtype=torch.float64) / half)
            s["cos"], s["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
        # the rows to look at afterwards: all tokens of the blocks that get new ones
        back = [n + (m - n) % BLOCK for n, m in zip(new, length)]
        starts = [0]
        for n in back:
            starts.append(starts[-1] + n)
        s["back_start"], s["back"], s["max_back"] = torch.tensor(starts, dtype=torch.int32, device=DEV), starts[-1], max(back)
    else:
        s["q"] = normal(T, c["qh"], D, std=2.0).to(act)
    if own:                                   # the handle that a program keeps beside its cache's tensors
        from paper_2504_12984_amd import binding as B_
        t = B_.WType(B_.QG_INT, 8) if c["kv"] == "i8" else B_.WType(B_.QG_FLOAT, 8, 4, 3)
        s["cache"] = B_.KvCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], t, D)
    return s


# ---- plain forms ----------------------------------------------------------------------------

def _scale_of(amax, qmax):
    return torch.where(torch.isfinite(amax), (amax / qmax).clamp_min(TINY), float("nan"))


def _row_codes(y):
    scale = _scale_of(y.abs().amax(-1, keepdim=True), 127.0)
    return torch.round(y * (1.0 / scale)).clamp(-127, 127), scale


def _norm_plain(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * s["w"].float()
    code, scale = _row_codes(y)
    out = {"values": (code * scale).to(s["x"].dtype), "scale": scale[:, 0]}
    if s["residual"] is not None:
        out["sum"] = h.to(s["x"].dtype)
    return out


def _gate_plain(s):
    gate, up = s["gu"].float().chunk(2, -1)
    code, scale = _row_codes(gate / (1 + torch.exp(-gate)) * up)
    return {"values": (code * scale).to(s["gu"].dtype), "scale": scale[:, 0]}


def _numbers(codes, kv):
    return codes.float() - 128.0 if kv == "i8" else codes.view(torch.float8_e4m3fn).float()


def _keys(codes, D):
    """[..., 64 * D] bytes of key blocks -> [..., 64 tokens, D]."""
    n = codes.dim() - 1
    x = codes.reshape(*codes.shape[:-1], 4, D // 64, 4, 16, 16)
    return x.permute(*range(n), n, n + 3, n + 1, n + 2, n + 4).reshape(*codes.shape[:-1], BLOCK, D)


def _keys_back(x, D):
    n = x.dim() - 2
    x = x.reshape(*x.shape[:-2], 4, 16, D // 64, 4, 16)
    return x.permute(*range(n), n, n + 2, n + 3, n + 1, n + 4).reshape(*x.shape[:n], BLOCK * D)


def _vals(codes, D):
    """[..., 64 * D] bytes of value blocks -> [..., 64 tokens, D]."""
    n = codes.dim() - 1
    x = codes.reshape(*codes.shape[:-1], D // 16, 4, 16, 4, 4)
    return x.permute(*range(n), n + 3, n + 1, n + 4, n, n + 2).reshape(*codes.shape[:-1], BLOCK, D)


def _vals_back(x, D):
    n = x.dim() - 2
    x = x.reshape(*x.shape[:-2], 4, 4, 4, D // 16, 16)
    return x.permute(*range(n), n + 3, n + 1, n + 4, n, n + 2).reshape(*x.shape[:n], BLOCK * D)


def _places(row_start, kv_len, T):
    """Sequence, row inside it and position of each of T rows."""
    row = torch.arange(T, device=DEV, dtype=torch.int32)
    b = torch.searchsorted(row_start[1:].contiguous(), row, right=True)
    j = row - row_start[b]
    new = row_start[1:] - row_start[:-1]
    return b, j.long(), (kv_len - new)[b].long() + j.long()


def _rotate(x, cos, sin, rot, pairs):
    """x [T, heads, D] in 32 bits; cos, sin [T, rot / 2]."""
    c, s = cos[:, None, :], sin[:, None, :]
    if pairs == "halves":
        x1, x2 = x[..., :rot // 2], x[..., rot // 2:rot]
        r = torch.cat((x1 * c - x2 * s, x2 * c + x1 * s), -1)
    else:
        x1, x2 = x[..., 0:rot:2], x[..., 1:rot:2]
        r = torch.stack((x1 * c - x2 * s, x2 * c + x1 * s), -1).flatten(-2)
    return torch.cat((r, x[..., rot:]), -1)


def _store_plain(s, name, x, b, slot, off, ids, there, old_upto):
    """Rows x [T, H, D] into the touched blocks ids [B, n]; the first block of each sequence keeps its first old_upto [B] tokens."""
    c = s["case"]
    kv, D = c["kv"], c["dim"]
    qmax = _QMAX[kv]
    B, n = ids.shape
    fresh = torch.zeros(B, n, BLOCK, c["kvh"], D, device=DEV)
    fresh[b, slot, off] = x
    is_new = torch.zeros(B, n, BLOCK, dtype=torch.bool, device=DEV)
    is_new[b, slot, off] = True
    token = torch.arange(BLOCK, device=DEV)
    is_old = (torch.arange(n, device=DEV)[None, :, None] == 0) & (token < old_upto[:, None, None])
    cache, scales = s[name + "_cache"], s[name + "_scale"]
    had = is_old.any(-1)[..., None]
    was = scales[ids]                                                     # [B, n, H]
    now = _scale_of(fresh.abs().amax((2, 4)), qmax)
    now = torch.where(had, torch.where(torch.isnan(now) | torch.isnan(was), float("nan"), torch.maximum(was, now)), now)
    inv = 1.0 / now
    codes = _numbers((_keys if name == "k" else _vals)(cache[ids], D), kv).transpose(2, 3)        # [B, n, 64, H, D]
    moved = codes * torch.where(now == was, 1.0, was * inv)[:, :, None, :, None]
    grown = fresh * inv[:, :, None, :, None]
    new = torch.where(is_new[..., None, None], grown, torch.where(is_old[..., None, None], moved, 0.0)).transpose(2, 3)
    new = _encode(torch.nan_to_num(new), 1.0, kv)
    new = (_keys_back if name == "k" else _vals_back)(new, D)
    cache[ids[there]] = new[there]
    scales[ids[there]] = now[there]


def _read_plain(s, name, row_start, T):
    """Values [T, H, D] of the last tokens of each sequence."""
    c = s["case"]
    b, _, pos = _places(row_start, s["kv_len"], T)
    ids = s["table"][b, pos // BLOCK].long()
    j, d = (pos % BLOCK)[:, None], torch.arange(c["dim"], device=DEV)[None, :]
    if name == "k":
        at = (((j // 16 * (c["dim"] // 64) + d // 64) * 4 + d % 64 // 16) * 16 + j % 16) * 16 + d % 16
    else:
        at = ((d // 16 * 4 + j % 16 // 4) * 16 + d % 16) * 16 + j // 16 * 4 + j % 4
    head = torch.arange(c["kvh"], device=DEV)
    codes = s[name + "_cache"][ids[:, None, None], head[None, :, None], at[:, None, :]]
    return (_numbers(codes, c["kv"]) * s[name + "_scale"][ids][..., None]).to(_DT[c["act"]])


def _split(s):
    c = s["case"]
    T, D = s["qkv"].shape[0], c["dim"]
    rows = s["qkv"].view(T, c["qh"] + 2 * c["kvh"], D)
    return rows[:, :c["qh"]], rows[:, c["qh"]:c["qh"] + c["kvh"]], rows[:, c["qh"] + c["kvh"]:]


def _append_plain(s):
    c = s["case"]
    q, k, v = (x.float() for x in _split(s))
    T = q.shape[0]
    new = s["row_start"][1:] - s["row_start"][:-1]
    b, _, pos = _places(s["row_start"], s["kv_len"], T)
    if c["rot"]:
        q, k = (_rotate(x, s["cos"][pos], s["sin"][pos], c["rot"], c["pairs"]) for x in (q, k))
    before = (s["kv_len"] - new).long()
    first = before // BLOCK
    n = (s["max_rows"] + BLOCK - 2) // BLOCK + 1                          # most blocks that so many rows touch
    at = first[:, None] + torch.arange(n, device=DEV)
    there = (at * BLOCK < s["kv_len"][:, None]) & (new[:, None] > 0)
    ids = torch.gather(s["table"], 1, at.clamp_max(s["table"].shape[1] - 1)).long()
    ids = torch.where(there, ids, 0)
    for name, x in (("k", k), ("v", v)):
        _store_plain(s, name, x, b, pos // BLOCK - first[b], pos % BLOCK, ids, there, before % BLOCK)
    return {"q": q.to(s["qkv"].dtype), "k": _read_plain(s, "k", s["back_start"], s["back"]),
            "v": _read_plain(s, "v", s["back_start"], s["back"])}


def _attn_plain(s):
    c = s["case"]
    B, H, D, R = c["batch"], c["kvh"], c["dim"], s["max_rows"]
    G, T = c["qh"] // c["kvh"], s["q"].shape[0]
    NB = -(-s["max_kv"] // BLOCK)
    L = NB * BLOCK
    new = s["row_start"][1:] - s["row_start"][:-1]
    j = torch.arange(R, device=DEV)
    row = (s["row_start"][:-1, None] + j).clamp_max(T - 1)
    q = s["q"][row].float().view(B, R, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * R, D)
    ids = s["table"][:, :NB].long().clamp_min(0)
    t = torch.arange(L, device=DEV)
    inside = t < s["kv_len"][:, None]                                     # [B, L]

    def whole(name, order):
        x = _numbers(order(s[name + "_cache"][ids], D), c["kv"])          # [B, NB, H, 64, D]
        x *= s[name + "_scale"][ids][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(B, H, L, D)

    p = torch.matmul(q, whole("k", _keys).transpose(-1, -2)).view(B, H, G, R, L)
    p *= D ** -0.5
    pos = (s["kv_len"] - new)[:, None] + j                                # [B, R]
    seen = (inside[:, None, :] & (j[None, :, None] < new[:, None, None])).expand(B, R, L)
    if c["causal"]:
        seen = seen & (t <= pos[..., None])
    if c["window"]:
        seen = seen & (t > pos[..., None] - c["window"])
    seen = seen[:, None, None]
    p = p.masked_fill_(~seen, float("-inf"))
    m = p.amax(-1, keepdim=True)
    p = (p - torch.where(torch.isfinite(m), m, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    v = whole("v", _vals).masked_fill_(~inside[:, None, :, None], 0.0)
    o = torch.matmul(p.view(B, H, G * R, L), v).view(B, H, G, R, D)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, R, c["qh"], D)
    b, at, _ = _places(s["row_start"], s["kv_len"], T)
    return o[b, at].to(s["q"].dtype)


# ---- one pass -------------------------------------------------------------------------------

def _values(code, scale, act):
    out = torch.empty(code.shape, dtype=act, device=code.device)
    return torch.mul(code, scale[:, None], out=out)


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"norm": _norm_plain, "gate": _gate_plain, "append": _append_plain, "attn": _attn_plain}[c["op"]](s)
    from paper_2504_12984_amd import binding as B
    if c["op"] == "norm":
        code, scale, total = B.qg_rmsnorm_a8(s["x"], s["w"], EPS, residual=s["residual"])
        out = {"values": _values(code, scale, s["x"].dtype), "scale": scale}
        if s["residual"] is not None:
            out["sum"] = total
        return out
    if c["op"] == "gate":
        code, scale = B.qg_silu_a8(s["gu"])
        return {"values": _values(code, scale, s["gu"].dtype), "scale": scale}
    if c["op"] == "append":
        q, k, v = _split(s)
        q = B.qg_kv_append(k, v, s["cache"], s["row_start"], s["kv_len"], s["table"], s["max_rows"], q=q, cos=s.get("cos"),
                           sin=s.get("sin"), neighbours=c["pairs"] == "neighbours")
        k, v = B.qg_kv_dequant(s["cache"], s["back_start"], s["kv_len"], s["table"], s["back"], _DT[c["act"]])
        return {"q": q, "k": k, "v": v}
    return B.qg_kv_attention(s["q"], s["cache"], s["row_start"], s["kv_len"], s["table"], c["dim"] ** -0.5, s["max_rows"],
                             s["max_kv"], causal=c["causal"], window=c["window"])


# ---- the definitions in 64 bits ---------------------------------------------------------------

def _code64(x, scale, kv):
    """The 8-bit number nearest to x / scale."""
    x = x / scale
    if kv == "i8":
        return x.round().clamp(-127, 127)
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -60))).clamp_min(-6)
    step = torch.exp2(e - 3)
    return ((x / step).round() * step).clamp(-448, 448)


def _quantised64(y):
    scale = (y.abs().amax(-1) / 127).clamp_min(TINY)
    return _code64(y, scale[:, None], "i8") * scale[:, None], scale


def _table64(kv):
    """The number of each byte."""
    got = []
    for u in range(256):
        if kv == "i8":
            got.append(float(u - 128))
            continue
        e, m = (u >> 3) & 15, u & 7
        x = math.ldexp(m / 8, -6) if e == 0 else math.ldexp(1 + m / 8, e - 7)
        got.append(-x if u >> 7 else x)
    return torch.tensor(got, dtype=torch.float64, device=DEV)


def _where64(name, D):
    """Byte of token j, dimension d inside a block, as a [64, D] table."""
    at = torch.empty(BLOCK, D, dtype=torch.int64)
    for j in range(BLOCK):
        for d in range(D):
            if name == "k":
                t, i, c, b, e = j // 16, j % 16, d // 64, d % 64 // 16, d % 16
                at[j, d] = (((t * (D // 64) + c) * 4 + b) * 16 + i) * 16 + e
            else:
                t, b, r, f, i = j // 16, j % 16 // 4, j % 4, d // 16, d % 16
                at[j, d] = ((f * 4 + b) * 16 + i) * 16 + 4 * t + r
    return at.to(DEV)


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    if c["op"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h = h + s["residual"].double()
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / c["N"] + EPS) * s["w"].double()
        values, scale = _quantised64(y)
        return {"values": values, "scale": scale, **({"sum": h} if s["residual"] is not None else {})}
    if c["op"] == "gate":
        g, u = s["gu"].double()[:, :c["N"]], s["gu"].double()[:, c["N"]:]
        values, scale = _quantised64(g * torch.sigmoid(g) * u)
        return {"values": values, "scale": scale}
    new, length = _lengths(c)
    D, H, kv = c["dim"], c["kvh"], c["kv"]
    number, place = _table64(kv), {n: _where64(n, D) for n in ("k", "v")}
    table = s["table"].cpu().tolist()

    def read(name, b, first, last):
        """Values [tokens, H, D] of the blocks first .. last - 1 of a sequence."""
        ids = torch.tensor(table[b][first:last], device=DEV)
        codes = s[name + "_cache"][ids][:, :, place[name]]                 # [n, H, 64, D]
        x = number[codes.long()] * s[name + "_scale"][ids].double()[..., None, None]
        return x.transpose(1, 2).reshape(-1, H, D)

    if c["op"] == "append":
        rows = s["qkv"].double().view(-1, c["qh"] + 2 * H, D)
        position = torch.cat([torch.arange(m - n, m, device=DEV) for n, m in zip(new, length)])
        if c["rot"]:
            both = rows[:, :c["qh"] + H]
            half = c["rot"] // 2
            cos, sin = s["cos"].double()[position][:, None], s["sin"].double()[position][:, None]
            first = torch.arange(half, device=DEV) if c["pairs"] == "halves" else 2 * torch.arange(half, device=DEV)
            second = first + (half if c["pairs"] == "halves" else 1)
            x, y = both[..., first], both[..., second]
            turned = both.clone()
            turned[..., first], turned[..., second] = x * cos - y * sin, y * cos + x * sin
            rows = torch.cat((turned, rows[:, c["qh"] + H:]), 1)
        got, at = {"k": [], "v": []}, 0
        for b, (n, m) in enumerate(zip(new, length)):
            for name, lo in (("k", c["qh"]), ("v", c["qh"] + H)):
                x = rows[at:at + n, lo:lo + H]                             # [n, H, D]
                before = m - n
                for blk in range(before // BLOCK, -(-m // BLOCK)):
                    lo_t, hi_t = max(before, blk * BLOCK), min(m, blk * BLOCK + BLOCK)
                    mine = x[lo_t - before:hi_t - before]
                    kept = read(name, b, blk, blk + 1)[:lo_t - blk * BLOCK]
                    scale = (mine.abs().amax((0, 2)) / _QMAX[kv]).clamp_min(TINY)
                    if kept.shape[0]:
                        was = s[name + "_scale"][table[b][blk]].double()
                        scale = torch.where(scale > was, scale, was)
                    every = torch.cat((kept, mine))
                    got[name].append(_code64(every, scale[None, :, None], kv) * scale[None, :, None])
            at += n
        return {"q": rows[:, :c["qh"]], "k": torch.cat(got["k"]), "v": torch.cat(got["v"])}
    out = torch.zeros(sum(new), c["qh"], D, dtype=torch.float64, device=DEV)
    G, at = c["qh"] // H, 0
    for b, (n, m) in enumerate(zip(new, length)):
        k, v = (read(name, b, 0, -(-m // BLOCK))[:m] for name in ("k", "v"))
        t = torch.arange(m, device=DEV)
        for lo in range(0, n, 2048):
            hi = min(n, lo + 2048)
            pos = (m - n + torch.arange(lo, hi, device=DEV))[:, None]
            hidden = torch.zeros(hi - lo, m, dtype=torch.bool, device=DEV)
            if c["causal"]:
                hidden |= t > pos
            if c["window"]:
                hidden |= t <= pos - c["window"]
            for h in range(c["qh"]):
                x = s["q"][at + lo:at + hi, h].double() @ k[:, h // G].t() / math.sqrt(D)
                x = torch.softmax(x.masked_fill_(hidden, float("-inf")), -1)
                out[at + lo:at + hi, h] = torch.nan_to_num(x, nan=0.0) @ v[:, h // G]
        at += n
    return out
