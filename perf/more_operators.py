"""The operators of the serving side as measurable cases: rotation, the paged cache, trees of drafted tokens.

Three operations, each through the public binding (``paper_2506_11498_b200.lrsa``):
  rotate  the position rotation of Q and K, and its gradient
  append  new tokens of many sequences enter a paged condensed cache, K rotated on the way; windows of tokens that are far
          enough back are cut to their highest-scoring rows
  attend  every sequence's next token, or a tree of drafted ones, attends over its pages and over its ancestors

``listed`` holds a fixed set of them; ``draw`` gives more of the same ranges.  With ``own`` false they are computed in
their plain form, by elementary tensor operations in 32 bits.
"""
import math
import random

import torch

own = False


def _case(name, op, heads, d, N, L, K, S, **kw):
    Hq, Hkv = heads
    case = {"name": name, "op": op, "Hq": Hq, "Hkv": Hkv, "d": d, "N": N, "L": L, "K": K, "S": S,
            "B": 1,             # sequences
            "least": N,         # the shortest sequence (lengths are spread from there to N)
            "rot": d, "interleaved": False, "inverse": False, "given": False,
            "page": 64, "new": 1, "mode": "token", "chain": False}
    case.update(kw)
    return case


def listed():
    return [
        # Rotation in front of the attention of the smallest layer: launch and latency.
        _case("rotate_4k_mha_d64", "rotate", (8, 8), 64, 4096, 512, 128, 16),
        # The gradient of the rotation of the 32K layer, three documents in a row (positions are given).
        _case("rotate_32k_gqa7_grad", "rotate", (28, 4), 128, 32768, 1024, 256, 4, inverse=True, given=True),
        # One token of sixteen sequences of different lengths: what every step of a server does.
        _case("append_token_b16", "append", (28, 4), 128, 32000, 1024, 256, 4, B=16, least=4000),
        # Accepted drafts of 64 sequences; some of them complete a window, and one leaves the recent pages.
        _case("append_drafts_b64_d64", "append", (16, 2), 64, 20000, 333, 83, 0, B=64, least=500, page=32, new=8, mode="drafts"),
        # Eight short prompts of odd lengths, small pages.
        _case("append_prompts_9k_d64", "append", (8, 8), 64, 9001, 512, 128, 16, B=8, least=700, page=16, mode="prompt"),
        # The 32K prompt enters the cache in one call.
        _case("append_prompt_32k", "append", (28, 4), 128, 32768, 1024, 256, 4, mode="prompt"),
        # One token on one short context: the smallest call there is.
        _case("attend_token_4k_mha_d64", "attend", (8, 8), 64, 3583, 512, 128, 16),
        # One token each for sixteen sequences of different lengths.
        _case("attend_token_32k_b16", "attend", (28, 4), 128, 32000, 1024, 256, 4, B=16, least=4000),
        # A tree of drafts at 32K, interactive use.
        _case("attend_tree48_32k", "attend", (28, 4), 128, 31743, 1024, 256, 4, new=48, mode="tree"),
        # Odd windows, rows that do not fill their pages, chains of drafts of different lengths.
        _case("attend_chain9_20k_b16_d64", "attend", (16, 2), 64, 20011, 333, 83, 0, B=16, least=60, page=16, new=9, mode="tree",
              chain=True),
        # Trees for sixteen sequences of different lengths: as much arithmetic as memory.
        _case("attend_tree32_32k_b16", "attend", (28, 4), 128, 32000, 1024, 256, 4, B=16, least=4000, new=32, mode="tree"),
        # Large trees over four sequences at 120K, half of every window kept.
        _case("attend_tree64_120k_b4", "attend", (32, 8), 128, 126975, 4096, 2048, 4, B=4, page=128, new=64, mode="tree"),
    ]


def draw(rng):
    op = rng.choice(("rotate", "append", "append", "append", "attend", "attend", "attend", "attend"))
    heads, d = rng.choice((((8, 8), 64), ((16, 2), 64), ((28, 4), 128), ((28, 4), 128), ((32, 8), 128)))
    N = int(math.exp(rng.uniform(math.log(100), math.log(32768 if op != "attend" else 131072))))
    L = rng.choice([L for L in (128, 256, 333, 512, 1000, 1024, 2048, 4096) if L <= max(128, N // 3)])
    K = max(1, L // rng.choice((2, 4, 4, 8, 16)))
    case = _case("", op, heads, d, N, L, K, rng.choice((0, 4, 16, 33)), page=rng.choice((16, 32, 64, 64, 128)))
    del case["name"]
    case["rot"] = rng.choice((d, d, d, d // 2))
    case["interleaved"] = rng.choice((False, False, True))
    if op == "rotate":
        case["inverse"], case["given"] = rng.choice((False, True)), rng.choice((False, True))
        return case
    case["least"] = max(1, N // rng.choice((1, 2, 8)))
    if op == "append":
        case["mode"] = rng.choice(("token", "drafts", "prompt"))
        most = 64 if case["mode"] != "prompt" else max(1, 40000 // N)
        case["new"] = rng.randint(2, 16) if case["mode"] == "drafts" else 1
    else:
        case["mode"] = rng.choice(("token", "tree", "tree"))
        case["chain"] = rng.choice((False, False, True))
        case["new"] = int(math.exp(rng.uniform(math.log(2), math.log(65)))) if case["mode"] == "tree" else 1
        most = max(1, min(64, 400000 // N))
    case["B"] = rng.randint(1, most) if most < 4 else int(math.exp(rng.uniform(0, math.log(most + 0.99))))
    return case


# ---- geometry: sinks [0, S), window w = [S + wL, S + (w+1)L) ----
def _cut(c, n):
    """Windows that a cache of n tokens holds by their kept rows, as its next token sees them."""
    return max((n - c["S"]) // c["L"] - 1, 0) if n >= c["S"] else 0


def _pages(c):
    """Pages of the sinks, of a recent window, of the kept rows of a window."""
    return tuple(-(-c[k] // c["page"]) for k in ("S", "L", "K"))


def _column(c, p):
    """Column of the page table, and row of that page, of the uncompressed token at position p (a tensor)."""
    sp, lp, _ = _pages(c)
    w, i = (p - c["S"]) // c["L"], (p - c["S"]) % c["L"]
    sink = p < c["S"]
    col = torch.where(sink, p // c["page"], sp + (w % 2) * lp + i // c["page"])
    return col, torch.where(sink, p % c["page"], i % c["page"])


def _lengths(c):
    """(tokens in the cache, new tokens) of every sequence: the same for every seed."""
    rng = random.Random(c["N"])
    out = []
    for s in range(c["B"]):
        n = c["N"] if s == 0 else int(math.exp(rng.uniform(math.log(c["least"]), math.log(c["N"] + 1))))
        n = min(max(n, c["least"]), c["N"])
        if c["mode"] == "prompt":
            out.append((0, n))
            continue
        m = c["new"] if s == 0 else rng.randint(min(1, c["new"]), c["new"])
        if c["op"] == "append" and c["mode"] == "drafts":
            full = c["S"] + (n - c["S"]) // c["L"] * c["L"] if n >= c["S"] else 0
            if s % 4 == 0 and full - m >= 0:      # these complete a window
                n = full - m
            else:                                 # these do not, and none starts one whose pages are still read
                room = c["L"] - (n - c["S"]) % c["L"] if n >= c["S"] else c["S"] - n
                m = max(0, min(m, room - 1))
        elif c["op"] == "append" and n >= c["S"] and (n + 1 - c["S"]) % c["L"] == 0 and s:
            n = max(n - 1, 0)
        out.append((n, m))
    return out


def _table(c, upto, seed):
    """Page table for sequences that grow to `upto` tokens: distinct pages where one is needed, -1 elsewhere."""
    sp, lp, kp = _pages(c)
    width = sp + 2 * lp + _cut(c, c["N"] + c["new"]) * kp
    need = torch.zeros(c["B"], max(width, 1), dtype=torch.bool)
    for s, n in enumerate(upto):
        need[s, :-(-min(n, c["S"]) // c["page"])] = True
        rest = max(n - c["S"], 0)
        for g in range(2):
            rows = min(max(rest - g * c["L"], 0), c["L"])
            need[s, sp + g * lp:sp + g * lp - (-rows // c["page"])] = True
        need[s, sp + 2 * lp:sp + 2 * lp + _cut(c, n) * kp] = True
    n_pages = int(need.sum()) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed + 1))
    table = torch.full(need.shape, -1, dtype=torch.int32)
    table[need] = order[:int(need.sum())].int()
    return table, n_pages


def _angles(c, n_pos):
    half = c["rot"] // 2
    f = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    a = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return a.cos().float(), a.sin().float()


def _rows(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").bfloat16()


def _salient(c, g, x, y, at):
    """Of every window at rows at[w] of x and y [Hkv, rows, d], K tokens a head that stand out: the kept ones."""
    for rows in at:
        pick = torch.rand(c["Hkv"], c["L"], generator=g, device="cuda").argsort(1)[:, :c["K"]]
        idx = rows[pick][..., None].expand(-1, -1, c["d"])
        for t in (x, y):
            t.scatter_(1, idx, 2.5 * t.gather(1, idx))


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    Hq, Hkv, d, N, L, S, P = (c[k] for k in ("Hq", "Hkv", "d", "N", "L", "S", "page"))
    s = {"case": c}
    if c["op"] == "rotate":
        s["Q"], s["K"] = _rows(g, 1, Hq, N, d), _rows(g, 1, Hkv, N, d)
        s["cos"], s["sin"] = _angles(c, N)
        if c["given"]:      # three documents in a row
            cuts = [0, N // 2, N - N // 7, N]
            s["positions"] = torch.cat([torch.arange(b - a, device="cuda") for a, b in zip(cuts, cuts[1:])]).int()
    else:
        lens = _lengths(c)
        s["lens"] = lens
        T = sum(m for _, m in lens)
        table, n_pages = _table(c, [n + m if c["op"] == "append" else n for n, m in lens], seed)
        s["table_host"], s["table"] = table, table.cuda()
        s["n_tokens"] = torch.tensor([n for n, _ in lens], dtype=torch.int32, device="cuda")
        cu = [0]
        for _, m in lens:
            cu.append(cu[-1] + m)
        s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
        s["cos"], s["sin"] = _angles(c, N + c["new"] + 1)
        k_pages, v_pages = _rows(g, n_pages, Hkv, P, d), _rows(g, n_pages, Hkv, P, d)
        # new tokens as a projection leaves them: token by token, heads side by side
        if c["op"] == "append":
            src = T if c["mode"] != "drafts" else 2 * T     # half of the drafts are accepted
            k, v = (_rows(g, src, Hkv, d).transpose(0, 1) for _ in "kv")
            if c["mode"] == "drafts":
                s["rows"] = (2 * torch.arange(T, device="cuda") + (torch.rand(T, generator=g, device="cuda") < 0.5)).int()
            for i, (n, m) in enumerate(lens):
                at = [cu[i] + S + w * L + torch.arange(L, device="cuda") for w in range(_cut(c, m))] if n == 0 else []
                _salient(c, g, k, v, at)
                for w in range(_cut(c, n), _cut(c, n + m)) if n else ():
                    col, row = _column(c, S + w * L + torch.arange(L, device="cuda"))
                    page = s["table"][i][col].long()
                    x, y = k_pages[page, :, row].transpose(0, 1), v_pages[page, :, row].transpose(0, 1)   # copies
                    _salient(c, g, x, y, [torch.arange(L, device="cuda")])
                    k_pages[page, :, row], v_pages[page, :, row] = x.transpose(0, 1), y.transpose(0, 1)
            s["kept"] = torch.zeros(c["B"], Hkv, _cut(c, N + c["new"]), c["K"], dtype=torch.int32, device="cuda")
        else:
            q = _rows(g, T, Hq, d).transpose(0, 1)
            k, v = (_rows(g, T, Hkv, d).transpose(0, 1) for _ in "kv")
            s["q"] = q
            if not c["chain"]:
                parent, rng = [], random.Random(seed)
                for _, m in lens:      # a root, and children mostly of the latest tokens
                    parent += [max(-1, i - 1 - min(int(rng.expovariate(0.4)), i - 1)) if i else -1 for i in range(m)]
                s["parent"] = torch.tensor(parent, dtype=torch.int32, device="cuda")
                s["parent_host"] = parent
        s["k"], s["v"], s["k_pages"], s["v_pages"] = k, v, k_pages, v_pages
    if own:
        from paper_2506_11498_b200 import lrsa
        params = lrsa.Params(1, Hq, Hkv, N + c["new"], d, L, c["K"], S)
        if c["op"] == "rotate":
            params = lrsa.Params(1, Hq, Hkv, N, d, L, c["K"], min(S, N))
        else:
            s["cache"] = cache = lrsa.PagedCache(params, s["k_pages"].shape[0], page=P)
            cache.k_pages, cache.v_pages = s.pop("k_pages"), s.pop("v_pages")
            assert cache.table_width == s["table"].shape[1] or s["table"].shape[1] == 1
        s["params"] = params
        s["rope"] = lrsa.Rope(s["cos"], s["sin"], interleaved=c["interleaved"])
    return s


# ---- the plain forms ----
def _turn(c, x, cos, sin, inverse=False):
    """x [..., tokens, d] in 32 bits with its leading channels rotated; cos, sin [tokens, rot / 2]."""
    x, r = x.float(), c["rot"]
    if inverse:
        sin = -sin
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _spread(c, x, ref):
    """Of the rows x [Hkv, L, d] of a window: standard deviation over the channels, in the range of the window behind."""
    lo, hi = ref.amin(1, keepdim=True), ref.amax(1, keepdim=True)
    width = hi - lo
    z = torch.where(width > 0, (x - lo) / width, 0.0)
    return torch.softmax(z.std(-1), -1)


def _append(s):
    c = s["case"]
    S, L, K, P, Hkv, d = (c[k] for k in ("S", "L", "K", "page", "Hkv", "d"))
    sp, lp, kp = _pages(c)
    k_pages, v_pages, kept_out = s["k_pages"], s["v_pages"], s["kept"]
    at = 0
    for i, (n, m) in enumerate(s["lens"]):
        if m == 0:
            continue
        new = torch.arange(at, at + m, device="cuda")
        at += m
        if "rows" in s:
            new = s["rows"][new].long()
        pos = torch.arange(n, n + m, device="cuda")
        k_new = _turn(c, s["k"][:, new], s["cos"][pos], s["sin"][pos]).bfloat16()
        v_new = s["v"][:, new]
        w0, w1 = _cut(c, n), _cut(c, n + m)
        if w1 > w0:
            # the tokens of windows w0 .. w1, from the pages and from the new ones
            p = torch.arange(S + w0 * L, min(S + (w1 + 1) * L, n + m), device="cuda")
            old = p[p < n]
            col, row = _column(c, old)
            page = s["table"][i][col].long()
            x = torch.cat([k_pages[page, :, row].transpose(0, 1), k_new[:, p[p >= n] - n]], 1).unflatten(1, (w1 - w0 + 1, L))
            y = torch.cat([v_pages[page, :, row].transpose(0, 1), v_new[:, p[p >= n] - n]], 1).unflatten(1, (w1 - w0 + 1, L))
            for w in range(w0, w1):
                j = w - w0
                score = sum(_spread(c, t[:, j].float(), t[:, j + 1].float()) for t in (x, y))
                top = torch.sort(score, dim=-1, descending=True, stable=True).indices[:, :K].sort(dim=-1).values
                kept_out[i, :, w] = (S + w * L + top).int()
                r = torch.arange(K, device="cuda")
                page = s["table"][i][sp + 2 * lp + w * kp + r // P].long()
                take = top[..., None].expand(-1, -1, d)
                k_pages[page, :, r % P] = x[:, j].gather(1, take).transpose(0, 1)
                v_pages[page, :, r % P] = y[:, j].gather(1, take).transpose(0, 1)
        stay = (pos < S) | (pos >= S + w1 * L)
        col, row = _column(c, pos[stay])
        page = s["table"][i][col].long()
        k_pages[page, :, row] = k_new[:, stay].transpose(0, 1)
        v_pages[page, :, row] = v_new[:, stay].transpose(0, 1)
    return {"k": k_pages, "v": v_pages, "kept": kept_out}


def _seen(c, n):
    """(column, row) of everything that a cache of n tokens shows its next token (tensors on the host)."""
    sp, lp, kp = _pages(c)
    w = _cut(c, n)
    p = torch.cat([torch.arange(min(n, c["S"])), torch.arange(min(n, c["S"] + w * c["L"]), n)]) if n > c["S"] else torch.arange(n)
    col, row = _column(c, p)
    r = torch.arange(w * c["K"])
    return torch.cat([col, sp + 2 * lp + r // c["K"] * kp + r % c["K"] // c["page"]]), torch.cat([row, r % c["K"] % c["page"]])


def _ancestors(s, i, m, at):
    """[m, m]: does token a of sequence i see drafted token b?  And the depth of every token (host)."""
    sees = torch.zeros(m, m, dtype=torch.bool)
    for a in range(m):
        parent = a - 1 if "parent" not in s else s["parent_host"][at + a]
        if parent >= 0:
            sees[a] = sees[parent]
        sees[a, a] = True
    return sees, sees.sum(1) - 1


def _attend(s):
    c = s["case"]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    out, lse_out, at = [], [], 0
    for i, (n, m) in enumerate(s["lens"]):
        col, row = _seen(c, n)
        page, row = s["table"][i][col.cuda()].long(), row.cuda()
        sees, depth = _ancestors(s, i, m, at)
        pos = (n + depth).cuda()
        q = _turn(c, s["q"][:, at:at + m], s["cos"][pos], s["sin"][pos])
        k = _turn(c, s["k"][:, at:at + m], s["cos"][pos], s["sin"][pos])
        k = torch.cat([s["k_pages"][page, :, row].transpose(0, 1).float(), k], 1)
        v = torch.cat([s["v_pages"][page, :, row].transpose(0, 1).float(), s["v"][:, at:at + m].float()], 1)
        x = (q.unflatten(0, (Hkv, Hq // Hkv)) @ k[:, None].transpose(-1, -2)) / math.sqrt(d)
        x[..., x.shape[-1] - m:].masked_fill_(~sees.cuda(), -math.inf)
        lse = torch.logsumexp(x, -1, keepdim=True)
        out.append((torch.exp(x - lse) @ v[:, None]).flatten(0, 1).bfloat16())
        lse_out.append(lse.squeeze(-1).flatten(0, 1))
        at += m
    return {"o": torch.cat(out, 1), "lse": torch.cat(lse_out, 1)}


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] == "rotate":
            pos = s["positions"].long() if c["given"] else torch.arange(c["N"], device="cuda")
            cos, sin = s["cos"][pos], s["sin"][pos]
            return {k: _turn(c, s[k], cos, sin, c["inverse"]).bfloat16() for k in "QK"}
        return _append(s) if c["op"] == "append" else _attend(s)
    from paper_2506_11498_b200 import lrsa
    if c["op"] == "rotate":
        q, k = lrsa.lrsa_rotate(s["params"], s["Q"], s["K"], s["rope"], positions=s.get("positions"), inverse=c["inverse"])
        return {"Q": q, "K": k}
    cache = s["cache"]
    if c["op"] == "append":
        cache.append(s["k"], s["v"], s["table"], s["n_tokens"], s["cu"], rows=s.get("rows"), rope=s["rope"], kept=s["kept"])
        return {"k": cache.k_pages, "v": cache.v_pages, "kept": s["kept"]}
    o, lse = cache.attend(s["q"], s["k"], s["v"], s["table"], s["n_tokens"], s["cu"], parent=s.get("parent"), rope=s["rope"],
                          max_new=c["new"])
    return {"o": o, "lse": lse}


def work(case):
    c = case
    Hq, Hkv, d, N, L, K, S = (c[k] for k in ("Hq", "Hkv", "d", "N", "L", "K", "S"))
    if c["op"] == "rotate":
        return {"bytes": (Hq + Hkv) * N * d * 4 + N * c["rot"] * 4, "flops": 3.0 * (Hq + Hkv) * N * c["rot"]}
    row, size, flops = 2 * d * 2 * Hkv, 0, 0.0     # K and V of a token
    for n, m in _lengths(c):
        if c["op"] == "append":
            w0, w1 = _cut(c, n), _cut(c, n + m)
            old = min((w1 - w0 + 1) * L, max(0, n - S - w0 * L)) if w1 > w0 else 0
            stay = m if w1 * L + S <= n else min(m, max(0, S - n) + n + m - S - w1 * L)
            size += row * (m + old + stay + (w1 - w0) * K) + m * c["rot"] * 4
            flops += 3.0 * m * c["rot"] * Hkv + 8.0 * (w1 - w0) * L * d * 2 * Hkv
        else:
            keys = len(_seen(c, n)[0])
            size += row * (keys + m) + m * Hq * (d * 4 + 4) + m * c["rot"] * 4
            flops += 4.0 * d * Hq * m * (keys + (m + 1) / 2)
    return {"bytes": size, "flops": flops}


# ---- the definitions in 64 bits ----
def _rotated(c, x, pos, s, sign=1.0):
    """Row by row as pairs of a complex number: x [heads, tokens, d] (float64) at positions pos."""
    half = c["rot"] // 2
    turn = torch.complex(s["cos"][pos].double(), sign * s["sin"][pos].double())
    i = torch.arange(half, device="cuda")
    first, second = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
    z = torch.complex(x[..., first], x[..., second]) * turn
    out = x.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = case
    Hq, Hkv, d, N, L, K, S, P = (c[k] for k in ("Hq", "Hkv", "d", "N", "L", "K", "S", "page"))
    if c["op"] == "rotate":
        pos = s["positions"].long() if c["given"] else torch.arange(N, device="cuda")
        return {k: _rotated(c, s[k].double(), pos, s, -1.0 if c["inverse"] else 1.0) for k in "QK"}
    sp, lp, kp = -(-S // P), -(-L // P), -(-K // P)
    table = s["table_host"].tolist()

    def place(i, p):
        """(page, row) of the uncompressed token at position p of sequence i."""
        if p < S:
            return table[i][p // P], p % P
        w, r = divmod(p - S, L)
        return table[i][sp + (w & 1) * lp + r // P], r % P

    def places(i, ps):
        both = [place(i, p) for p in ps]
        return [torch.tensor(x, dtype=torch.long, device="cuda") for x in (zip(*both) if both else ((), ()))]

    def cut(n):
        return max((n - S) // L - 1, 0) if n >= S else 0

    at = 0
    if c["op"] == "append":
        out = {"k": s["k_pages"].double(), "v": s["v_pages"].double(), "kept": None}
        for i, (n, m) in enumerate(s["lens"]):
            src = torch.arange(at, at + m, device="cuda")
            src = s["rows"].long()[src] if "rows" in s else src
            pos = torch.arange(n, n + m, device="cuda")
            new = {"k": _rotated(c, s["k"][:, src].double(), pos, s), "v": s["v"][:, src].double()}
            held = {"k": new["k"].to(torch.bfloat16).double(), "v": new["v"]}      # what is scored is what the cache holds
            at += m

            def window(name, w, of):
                ps = range(S + w * L, S + (w + 1) * L)
                page, row = places(i, [p for p in ps if p < n])
                old = s[name + "_pages"][page, :, row].double().transpose(0, 1)
                first = max(0, S + w * L - n)
                return torch.cat([old, of[name][:, first:first + L - old.shape[1]]], 1)

            for w in range(cut(n), cut(n + m)):
                score = 0
                for name in "kv":
                    x, ref = window(name, w, held), window(name, w + 1, held)
                    lo = ref.min(1, keepdim=True).values
                    wide = ref.max(1, keepdim=True).values - lo
                    z = torch.where(wide > 0, (x - lo) / wide.clamp_min(1e-300), torch.zeros_like(x))
                    e = torch.exp(torch.sqrt(((z - z.mean(2, keepdim=True)) ** 2).sum(2) / (d - 1)))
                    score = score + e / e.sum(1, keepdim=True)
                order = torch.argsort(score, dim=1, descending=True, stable=True)[:, :K].sort(dim=1).values
                for j in range(0, K, P):
                    page = table[i][sp + 2 * lp + w * kp + j // P]
                    for name in "kv":
                        part = torch.take_along_dim(window(name, w, new), order[:, j:j + P, None], 1)
                        out[name][page, :, :part.shape[1]] = part
            keep = [j for j in range(m) if n + j < S or n + j >= S + cut(n + m) * L]
            page, row = places(i, [n + j for j in keep])
            for name in "kv":
                out[name][page, :, row] = new[name][:, keep].transpose(0, 1)
        return out
    if sum(n * m for n, m in s["lens"]) * Hq > 1.2e9:
        return None
    o, lse = [], []
    for i, (n, m) in enumerate(s["lens"]):
        w = cut(n)
        page, row = places(i, list(range(min(n, S))) + list(range(S + w * L, n)))
        kept = [(table[i][sp + 2 * lp + j // K * kp + j % K // P], j % K % P) for j in range(w * K)]
        if kept:
            extra = torch.tensor(kept, dtype=torch.long, device="cuda")
            page, row = torch.cat([page, extra[:, 0]]), torch.cat([row, extra[:, 1]])
        lines, depth = [], []
        for a in range(m):
            line, b = [], a
            while b >= 0:
                line.append(b)
                b = b - 1 if "parent" not in s else s["parent_host"][at + b]
            lines.append(line)
            depth.append(len(line) - 1)
        hidden = torch.ones(m, m, dtype=torch.bool, device="cuda")
        for a, line in enumerate(lines):
            hidden[a, line] = False
        pos = torch.tensor(depth, dtype=torch.long, device="cuda") + n
        q = _rotated(c, s["q"][:, at:at + m].double(), pos, s)
        k = _rotated(c, s["k"][:, at:at + m].double(), pos, s)
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            keys = torch.cat([s["k_pages"][page, kv, row].double(), k[kv]])
            vals = torch.cat([s["v_pages"][page, kv, row].double(), s["v"][kv, at:at + m].double()])
            x = q[h] @ keys.T / math.sqrt(d)
            x[:, len(page):] = x[:, len(page):].masked_fill(hidden, -math.inf)
            top = x.max(1, keepdim=True).values
            e = torch.exp(x - top)
            total = e.sum(1, keepdim=True)
            o.append((e @ vals) / total)
            lse.append((top + torch.log(total))[:, 0])
        at += m
    Bh = [torch.stack(o[i * Hq:(i + 1) * Hq]) for i in range(c["B"])], [torch.stack(lse[i * Hq:(i + 1) * Hq]) for i in range(c["B"])]
    return {"o": torch.cat(Bh[0], 1), "lse": torch.cat(Bh[1], 1)}
