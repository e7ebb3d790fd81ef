"""The operators of the weighted, 8-bit side of the library as measurable cases.

Four operations, each through the public binding (``paper_2506_11498_b200.lrsa``):
  weights  the attention weight that every position has gathered from the queries that see it uncompressed
  select   of every lag window, the positions that gathered most
  append   a prompt enters a cache that keeps rows by that weight, in 8 bits with a scale per block of rows and head,
           and its kept rows are read back
  decode   one query token per sequence attends over such a cache and adds its weights to the recent rows'

``listed`` holds a fixed set of them; ``draw`` gives more of the same ranges.  With ``own`` false they are computed in
their plain form, by elementary tensor operations in 32 bits.
"""
import math

import torch

own = False

MOST = {"e4m3": 448.0, "int8": 127.0}   # largest magnitude of a code


def _case(name, op, heads, d, N, L, K, S, B=1, **kw):
    Hq, Hkv = heads
    case = {"name": name, "op": op, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "N": N, "L": L, "K": K, "S": S,
            "ndp": 1, "offset": False, "type": "e4m3", "block": 64, "keep": "weight", "piece": 0}
    case.update(kw)
    return case


def listed():
    return [
        # The smallest attention layer: 4K tokens, multi-head, d = 64.
        _case("weights_4k_mha_d64", "weights", (8, 8), 64, 4096, 512, 128, 16),
        # The 32K layer of a 7B-shaped model with outlier channels: the ordinary prompt.
        _case("weights_32k_gqa7", "weights", (28, 4), 128, 32768, 1024, 256, 4, offset=True),
        # Ragged: odd length and window, no sinks, the previous window compressed too.
        _case("weights_11k_l333_d64", "weights", (16, 2), 64, 11003, 333, 83, 0, B=2, ndp=0),
        # The selection for that prompt: launch and latency.
        _case("select_32k_gqa7", "select", (28, 4), 128, 32768, 1024, 256, 4),
        # The longest prompts, long windows.
        _case("select_128k_b2", "select", (32, 8), 128, 131072, 4096, 1024, 4, B=2),
        # The 32K prompt enters the cache in one call.
        _case("append_32k_gqa7_e4m3", "append", (28, 4), 128, 32768, 1024, 256, 4, offset=True),
        # A prompt of odd length arrives in pieces: windows leave the ring one by one.
        _case("append_9k_mha_int8", "append", (8, 8), 64, 9001, 512, 128, 16, B=2, type="int8", block=32, piece=2048),
        # One token on a short context of a small layer: the smallest call there is.
        _case("decode_4k_mha_d64_int8", "decode", (8, 8), 64, 3583, 512, 128, 16, type="int8"),
        # One token at 32K, interactive use.
        _case("decode_32k_gqa7_e4m3", "decode", (28, 4), 128, 31743, 1024, 256, 4, offset=True),
        # Sixteen sequences at once, rows kept by the lag score (no weights are gathered).
        _case("decode_32k_gqa7_b16_e4m3", "decode", (28, 4), 128, 31743, 1024, 256, 4, B=16, offset=True, keep="lag"),
        # Four sequences at 120K, half of every window kept: the largest cache.
        _case("decode_120k_b4_int8", "decode", (32, 8), 128, 126975, 4096, 2048, 4, B=4, type="int8", block=128),
        # Odd windows of which an odd number of rows is kept: blocks end inside a window's rows.
        _case("decode_20k_l333_e4m3", "decode", (16, 2), 64, 20011, 333, 83, 0, B=4, block=16),
    ]


def draw(rng):
    op = rng.choice(("weights", "weights", "select", "append", "append", "decode", "decode", "decode"))
    heads, d = rng.choice((((8, 8), 64), ((16, 2), 64), ((28, 4), 128), ((28, 4), 128), ((32, 8), 128)))
    lo, hi = {"weights": (300, 32768), "select": (1000, 131072), "append": (1500, 65536), "decode": (200, 131072)}[op]
    N = int(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    L = rng.choice([L for L in (128, 256, 333, 512, 1000, 1024, 2048, 4096) if L <= max(128, N // 3)])
    if op == "weights":
        L = min(L, 1024)
    K = max(1, L // rng.choice((2, 4, 4, 8, 16)))
    case = _case("", op, heads, d, N, L, K, rng.choice((0, 4, 16)), offset=rng.choice((False, True)))
    del case["name"]
    case["type"] = rng.choice(("e4m3", "e4m3", "int8"))
    case["block"] = rng.choice((16, 32, 64, 128))
    case["keep"] = rng.choice(("weight", "weight", "lag")) if op == "decode" else "weight"
    if op == "decode":
        case["B"] = min(max(1, (1 << 19) // N), rng.choice((1, 1, 2, 4, 8, 16)))
    elif op == "append":
        case["piece"] = rng.choice((0, 0, 512, 2048)) if N < 16384 else 0
        case["B"] = rng.choice((1, 1, 2, 4)) if N < 16384 else 1
    else:
        case["B"] = rng.choice((1, 1, 2)) if N < 16384 else 1
        case["ndp"] = rng.choice((1, 1, 0)) if op == "weights" else 1
    return case


# ---- geometry: sinks [0, S), window w = [S + wL, S + (w+1)L) ----
def _windows(c):
    W = (c["N"] - c["S"]) // c["L"] if c["N"] > c["S"] else 0
    return W, max(W - 1, 0)


def _chunks(c):
    """Number of query chunks, and of the windows that each of them sees compressed."""
    W, Wsel = _windows(c)
    C = -(-(c["N"] - c["S"]) // c["L"]) if c["N"] > c["S"] else 0
    return C, [min(max(i - c["ndp"], 0), Wsel) for i in range(C)]


def _compressed(c):
    """Windows in the list of a cache that holds N tokens."""
    return max((c["N"] - 1 - c["S"]) // c["L"] - 1, 0) if c["N"] > c["S"] else 0


def _pad(c):
    """List rows per window: a window starts a block of its own."""
    return -(-c["K"] // c["block"]) * c["block"]


# ---- inputs ----
def _rows(g, shape, offset):
    x = torch.randn(shape, generator=g, device="cuda")
    if offset:   # outlier channels
        x += 2.0 * torch.randn(shape[1:2] + (1,) + shape[3:], generator=g, device="cuda")
    return x.bfloat16()


def _round_up(x):
    """The least bfloat16 that is not below x (>= 0)."""
    return torch.where(x < math.inf, ((x.view(torch.int32) + 0xffff) & -65536).view(torch.float32), x)


def _quantize(x, kind, block):
    """Codes (as the numbers they are) and scales of rows [..., rows, d], rows a multiple of block."""
    b = x.float().unflatten(-2, (-1, block))
    most = b.abs().amax((-2, -1))
    limit = torch.full((), MOST[kind], device="cuda")   # (by a plain number torch multiplies with its rounded inverse)
    scale = torch.where(most > 0, _round_up(most / limit).clamp_min(2.0 ** -126), 1.0)
    y = b / scale[..., None, None]
    y = y.to(torch.float8_e4m3fn).float() if kind == "e4m3" else y.round()
    return y.flatten(-3, -2), scale


def _params(c):
    from paper_2506_11498_b200 import lrsa
    return lrsa.Params(c["B"], c["Hq"], c["Hkv"], c["N"], c["d"], c["L"], c["K"], c["S"], n_dense_prev=c["ndp"])


def _type(c):
    return torch.float8_e4m3fn if c["type"] == "e4m3" else torch.int8


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, Hq, Hkv, N, d, L, K, S = (c[k] for k in ("B", "Hq", "Hkv", "N", "d", "L", "K", "S"))
    s = {"case": c}
    if c["op"] == "weights":
        s["Q"] = _rows(g, (B, Hq, N, d), False)
        s["K"] = _rows(g, (B, Hkv, N, d), c["offset"])
        # the log-sum of a row of n keys whose scores are normal, as the forward gives it
        n = torch.arange(1, N + 1, device="cuda", dtype=torch.float32).clamp_max(2 * L + S + N / 4)
        k = s["K"][:, :, :: max(1, N // 64)].float()
        mean, var = k.mean(2), k.var(2)
        q = s["Q"].float().unflatten(1, (Hkv, Hq // Hkv)) / math.sqrt(d)
        lse = torch.log(n) + (q * mean[:, :, None, None]).sum(-1) + 0.5 * (q * q * var[:, :, None, None]).sum(-1)
        s["LSE"] = lse.flatten(1, 2).contiguous()
    elif c["op"] == "select":
        s["weight"] = torch.empty(B, Hkv, N, device="cuda").log_normal_(0, 2, generator=g)
    elif c["op"] == "append":
        s["K"], s["V"] = _rows(g, (B, Hkv, N, d), c["offset"]), _rows(g, (B, Hkv, N, d), False)
        s["weight"] = torch.empty(B, Hkv, N, device="cuda").log_normal_(0, 2, generator=g)
        step = c["piece"] or N
        s["pieces"] = [tuple(s[k][:, :, p:p + step].contiguous() for k in ("K", "V", "weight")) for p in range(0, N, step)]
    else:
        rows = _compressed(c) * _pad(c)
        used = torch.arange(rows, device="cuda") % _pad(c) < K
        s["q"] = _rows(g, (B, Hq, 1, d), False)[:, :, 0].contiguous()
        for k in "kv":
            x = _rows(g, (B, Hkv, rows, d), c["offset"] and k == "k") * used[:, None]
            s[k + "_list"], s[k + "_scale"] = _quantize(x, c["type"], c["block"])
            s[k + "_recent"] = _rows(g, (B, Hkv, S + 2 * L, d), c["offset"] and k == "k")
        s["weight"] = torch.rand(B, Hkv, 2 * L, generator=g, device="cuda")
    if own and c["op"] in ("append", "decode"):   # the cache that the program keeps
        from paper_2506_11498_b200 import lrsa
        s["cache"] = cache = lrsa.KVStore(_params(c), dtype=_type(c), block=c["block"], keep=c["keep"])
        if c["op"] == "decode":
            for k in ("k_list", "v_list", "k_scale", "v_scale"):
                at = getattr(cache, k)
                at[:, :, :s[k].shape[2]].copy_(s.pop(k).to(at.dtype))
            for k in ("k_recent", "v_recent"):
                getattr(cache, k).copy_(s.pop(k))
            cache.n_tokens = N
    elif own:
        s["params"] = _params(c)
    return s


# ---- the plain forms ----
def _weights(c, Q, K, LSE):
    B, Hq, Hkv, N, d, L, S = (c[k] for k in ("B", "Hq", "Hkv", "N", "d", "L", "S"))
    C, n = _chunks(c)
    first = S + L * torch.tensor(n, device="cuda")                        # first key of a chunk's contiguous range
    t = S + torch.arange(C * L, device="cuda").view(C, L)                  # queries
    j = first[:, None] + torch.arange(2 * L, device="cuda")                # keys
    sees = (j[:, None] <= t[:, :, None]) & (t < N)[:, :, None]
    t, at = t.clamp_max(N - 1), j.clamp_max(N - 1)
    q = Q.unflatten(1, (Hkv, Hq // Hkv))[:, :, :, t].float()               # [B, Hkv, G, C, L, d]
    k = K[:, :, at].float()                                                # [B, Hkv, C, 2L, d]
    x = q @ k[:, :, None].transpose(-1, -2)
    x *= 1 / math.sqrt(d)
    x -= LSE.unflatten(1, (Hkv, Hq // Hkv))[:, :, :, t][..., None]
    x.exp_()
    x *= sees
    w = torch.zeros(B, Hkv, N, device="cuda")
    return w.index_add_(2, at.flatten(), x.sum((2, 4)).flatten(2))


def _select(c, weight, n):
    """Positions of the K heaviest tokens of windows 0 .. n - 1, ascending; equal weights go to the lower position."""
    w = weight[:, :, c["S"]:c["S"] + n * c["L"]].unflatten(2, (n, c["L"]))
    top = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :c["K"]].sort(dim=-1).values
    return (top + c["S"] + c["L"] * torch.arange(n, device="cuda")[:, None]).int()


def _append(c, K, V, weight):
    n, N, L, S = _compressed(c), c["N"], c["L"], c["S"]
    out = {}
    idx = _select(c, weight, n) if n else weight.new_empty(c["B"], c["Hkv"], 0, c["K"]).int()
    p = torch.arange(max(S, N - 2 * L), N, device="cuda")                  # tokens that stay uncompressed in the ring
    for name, x in (("k", K), ("v", V)):
        kept = x.gather(2, idx.flatten(2).long()[..., None].expand(-1, -1, -1, c["d"])).unflatten(2, (n, c["K"]))
        kept = torch.nn.functional.pad(kept, (0, 0, 0, _pad(c) - c["K"])).flatten(2, 3)
        code, scale = _quantize(kept, c["type"], c["block"])
        rows = code * scale.repeat_interleave(c["block"], 2)[..., None]
        out[name] = rows.unflatten(2, (n, _pad(c)))[:, :, :, :c["K"]].flatten(2, 3)
        recent = x.new_zeros(c["B"], c["Hkv"], S + 2 * L, c["d"])
        recent[:, :, :min(S, N)] = x[:, :, :min(S, N)]
        recent[:, :, S + (p - S) % (2 * L)] = x[:, :, p]
        out[name + "_recent"] = recent
    out["idx"] = idx
    out["weight"] = weight.new_zeros(c["B"], c["Hkv"], 2 * L)
    out["weight"][:, :, (p - S) % (2 * L)] = weight[:, :, p]
    return out


def _recent_rows(c):
    """Rows of the recent buffer that the last token sees, in order of position (host numbers)."""
    S, L, t = c["S"], c["L"], c["N"] - 1
    if t < S:
        return 0, t + 1, 0
    n = _compressed(c)
    return n, S, t - (S + n * L) + 1


def _decode(s):
    c = s["case"]
    B, Hq, Hkv, d, L, S = (c[k] for k in ("B", "Hq", "Hkv", "d", "L", "S"))
    n, sinks, ring = _recent_rows(c)
    r = (n * L + torch.arange(ring, device="cuda")) % (2 * L)
    at = torch.cat([torch.arange(sinks, device="cuda"), S + r])
    rows = n * _pad(c)
    used = torch.arange(rows, device="cuda")
    used = used[used % _pad(c) < c["K"]]
    kv = []
    for k in "kv":
        x = s[k + "_list"] * s[k + "_scale"].repeat_interleave(c["block"], 2)[..., None]
        kv.append(torch.cat([x[:, :, used], s[k + "_recent"][:, :, at].float()], 2))
    q = s["q"].float().unflatten(1, (Hkv, Hq // Hkv))
    x = (q @ kv[0].transpose(-1, -2)) / math.sqrt(d)
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - lse[..., None])
    out = {"o": (p @ kv[1]).flatten(1, 2).bfloat16(), "lse": lse.flatten(1, 2)}
    if c["keep"] == "weight":
        out["weight"] = s["weight"].index_add(2, r, p[..., p.shape[-1] - ring:].sum(2))
    return out


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] == "weights":
            return _weights(c, s["Q"], s["K"], s["LSE"])
        if c["op"] == "select":
            return _select(c, s["weight"], _windows(c)[1])
        return _append(c, s["K"], s["V"], s["weight"]) if c["op"] == "append" else _decode(s)
    from paper_2506_11498_b200 import lrsa
    if c["op"] == "weights":
        return lrsa.lrsa_attn_weights(s["params"], s["Q"], s["K"], s["LSE"])
    if c["op"] == "select":
        return lrsa.lrsa_weight_select(s["params"], s["weight"])
    cache = s["cache"]
    if c["op"] == "append":
        cache.n_tokens = 0
        for k, v, w in s["pieces"]:
            cache.append(k, v, w)
        k, v = cache.rows()
        return {"k": k, "v": v, "k_recent": cache.k_recent, "v_recent": cache.v_recent,
                "idx": cache.idx[:, :, :_compressed(c)], "weight": cache.weight}
    if c["keep"] == "weight":
        cache.weight.copy_(s["weight"])
    o, lse = cache.decode(s["q"])
    return {"o": o, "lse": lse, "weight": cache.weight} if c["keep"] == "weight" else {"o": o, "lse": lse}


def work(case):
    c = case
    B, Hq, Hkv, N, d, L, K, S = (c[k] for k in ("B", "Hq", "Hkv", "N", "d", "L", "K", "S"))
    W, Wsel = _windows(c)
    if c["op"] == "weights":
        _, n = _chunks(c)
        pairs = sum(m * a + m * (m + 1) // 2 for m, a in
                    ((min(L, N - S - i * L), (i - n[i]) * L) for i in range(len(n))))
        return {"bytes": B * ((Hq + Hkv) * N * d * 2 + (Hq + Hkv) * N * 4), "flops": 2.0 * d * pairs * B * Hq}
    if c["op"] == "select":
        return {"bytes": 4 * B * Hkv * (Wsel * L + Wsel * K), "flops": 0}
    n, (_, sinks, ring) = _compressed(c), _recent_rows(c)
    scales = n * _pad(c) // c["block"] * 2 * 4
    if c["op"] == "append":
        kept, stay = n * K, min(N, S + 2 * L)
        # weights of all tokens; the kept rows in bf16 in, in 8 bits out and, read back, in 32 bits; the rows that stay
        per = 4 * N + kept * (2 * d * (2 + 1 + 1 + 4) + 4) + 2 * scales + stay * 2 * d * 4 + 4 * 2 * L
        return {"bytes": B * Hkv * per, "flops": 0}
    per = n * K * 2 * d + scales + (sinks + ring) * 2 * d * 2 + (2 * 4 * ring if c["keep"] == "weight" else 0)
    return {"bytes": B * (Hkv * per + Hq * (d * 4 + 4)), "flops": 4.0 * d * (n * K + sinks + ring) * B * Hq}


# ---- the definitions in 64 bits ----
def _held(x, kind):
    """What 8 bits hold of x (float64, magnitude at most MOST): the nearest code, ties to the even one."""
    if kind == "int8":
        return torch.round(x)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, Hq, Hkv, N, d, L, K, S = (c[k] for k in ("B", "Hq", "Hkv", "N", "d", "L", "K", "S"))
    G = Hq // Hkv
    if c["op"] == "weights":
        C, n = _chunks(c)
        w = torch.zeros(B, Hkv, N, dtype=torch.float64, device="cuda")
        for i in range(C):
            t0, t1, j0 = S + i * L, min(N, S + (i + 1) * L), S + n[i] * L
            k = s["K"][:, :, j0:t1].double()
            hide = torch.arange(j0, t1, device="cuda") > torch.arange(t0, t1, device="cuda")[:, None]
            for h in range(Hq):
                x = s["Q"][:, h, t0:t1].double() @ k[:, h // G].transpose(1, 2) / math.sqrt(d)
                p = torch.exp(x - s["LSE"][:, h, t0:t1, None].double()).masked_fill(hide, 0.0)
                w[:, h // G, j0:t1] += p.sum(1)
        return w
    if c["op"] == "select":
        return None
    if c["op"] == "append":
        n, out = _compressed(c), {"idx": None, "weight": None}
        w = s["weight"].double()
        order = [torch.argsort(w[:, :, S + i * L:S + (i + 1) * L], dim=2, descending=True, stable=True)[:, :, :K]
                 for i in range(n)]
        for name in "kv":
            x = s[name.upper()].double()
            rows = []
            for i in range(n):
                at = S + i * L + order[i].sort(dim=2).values
                kept = torch.take_along_dim(x, at[..., None], 2)
                for b in range(0, K, c["block"]):
                    part = kept[:, :, b:b + c["block"]]
                    most = part.abs().amax((2, 3), keepdim=True) / MOST[c["type"]]
                    e = torch.exp2(torch.floor(torch.log2(most)) - 7)          # spacing of 8-bit significands
                    scale = torch.ceil(most / e) * e
                    rows.append(_held(part / scale, c["type"]) * scale)
            out[name] = torch.cat(rows, 2) if rows else x[:, :, :0]
            out[name + "_recent"] = None
        return out
    n, sinks, ring = _recent_rows(c)
    keys = {}
    for k in "kv":
        x = s[k + "_list"].double().unflatten(2, (-1, c["block"])) * s[k + "_scale"].double()[..., None, None]
        x = x.flatten(2, 3).unflatten(2, (n, _pad(c)))[:, :, :, :K].flatten(2, 3) if n else x.flatten(2, 3)
        ordered = torch.roll(s[k + "_recent"][:, :, S:].double(), -(n * L) % (2 * L), 2)[:, :, :ring]
        keys[k] = torch.cat([x, s[k + "_recent"][:, :, :sinks].double(), ordered], 2)
    o, lse, gained = [], [], torch.zeros(B, Hkv, ring, dtype=torch.float64, device="cuda")
    for h in range(Hq):
        x = torch.einsum("bd,bnd->bn", s["q"][:, h].double(), keys["k"][:, h // G]) / math.sqrt(d)
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        total = e.sum(1, keepdim=True)
        lse.append((top + torch.log(total))[:, 0])
        o.append(torch.einsum("bn,bnd->bd", e / total, keys["v"][:, h // G]))
        gained[:, h // G] += (e / total)[:, x.shape[1] - ring:]
    out = {"o": torch.stack(o, 1), "lse": torch.stack(lse, 1)}
    if c["keep"] == "weight":
        w = s["weight"].double()
        at = (n * L + torch.arange(ring, device="cuda")) % (2 * L)
        w[:, :, at] += gained
        out["weight"] = w
    return out
