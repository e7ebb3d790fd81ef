"""Plain fp64 restatements of the weighted selection and of the 8-bit store, and the roundings their kernels may make."""
import math

import torch

MOST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
LOG2E = math.log2(math.e)


def n_hist(p, c):
    W = max(p.seq_len - p.n_sink, 0) // p.lag
    return min(max(c - p.n_dense_prev, 0), max(W - 1, 0))


def sees_uncompressed(p, N):
    """bool [N, N]: query t (row) sees position j >= S uncompressed.  `p` describes one sequence of N tokens."""
    S, L = min(p.n_sink, N), p.lag
    W = (N - S) // L
    t = torch.arange(N)
    first = torch.tensor([S + min(max((q - S) // L - p.n_dense_prev, 0), max(W - 1, 0)) * L if q >= S else N for q in range(N)],
                         dtype=torch.long)
    j = torch.arange(N)
    return (j[None] >= first[:, None]) & (j[None] <= t[:, None])


def weights(p, Q, K, LSE, cu=None):
    """(weight, what the arithmetic of the kernel may be off by), fp64 [B, Hkv, N].  A score's exponent (log2) is off by the
    roundings of a sum of d exact products (d / 8 steps of 2^-23 of the sum of their magnitudes, generously), of the scale
    and of LSE * log2(e); an exponential by 2^-21 relative; the sum of n terms by n 2^-24."""
    B, Hq, N, d = Q.shape
    Hkv = K.shape[1]
    scale = (p.softmax_scale or 1 / math.sqrt(d))
    w, tol = torch.zeros(B, Hkv, N, dtype=torch.float64), torch.zeros(B, Hkv, N, dtype=torch.float64)
    for lo, hi in zip((cu or (0, N))[:-1], (cu or (0, N))[1:]):
        see = sees_uncompressed(p, hi - lo)
        for b in range(B):
            for h in range(Hq):
                q, k = Q[b, h, lo:hi].double(), K[b, h // (Hq // Hkv), lo:hi].double()
                lse = LSE[b, h, lo:hi, None].double()
                P = torch.exp(q @ k.T * scale - lse).masked_fill(~see, 0.0)
                T = q.abs() @ k.abs().T * scale * LOG2E
                off = math.log(2) * 2.0 ** -23 * ((d / 8 + 2) * T + 3 * lse.abs() * LOG2E) + 2.0 ** -21
                w[b, h // (Hq // Hkv), lo:hi] += P.sum(0)
                tol[b, h // (Hq // Hkv), lo:hi] += (P * off).masked_fill(~see, 0.0).sum(0)
    return w, tol + w * (N * Hq // Hkv) * 2.0 ** -24


def select(p, weight, cu=None):
    """Per scored window the K heaviest positions, ascending, ties to the lower position, NaN last; int32 [B, Hkv, W_sel, K]."""
    B, Hkv, N = weight.shape
    out = []
    for lo, hi in zip((cu or (0, N))[:-1], (cu or (0, N))[1:]):
        S = min(p.n_sink, hi - lo)
        for w in range(max((hi - lo - S) // p.lag - 1, 0)):
            a = lo + S + w * p.lag
            x = weight[:, :, a:a + p.lag].double()
            x = torch.where(x.isnan(), torch.full_like(x, -math.inf), x)
            out.append(torch.sort(x, dim=2, descending=True, stable=True).indices[:, :, :p.top_k].sort(dim=2).values + a)
    return torch.stack(out, 2).int() if out else torch.zeros(B, Hkv, 0, p.top_k, dtype=torch.int32)


def held(x, dtype, block):
    """(what 8-bit blocks of the rows [..., rows, d] stand for, scales), fp64; rows are padded with zeros to whole blocks."""
    if dtype == torch.bfloat16:
        return x.double(), None
    rows = x.shape[-2]
    x = torch.nn.functional.pad(x.double(), (0, 0, 0, -rows % block)).unflatten(-2, (-1, block))
    most = x.abs().amax((-2, -1), keepdim=True) / MOST[dtype]
    e = torch.exp2(torch.floor(torch.log2(most.clamp_min(2.0 ** -140))) - 7)
    scale = torch.where(most > 0, (torch.ceil(most / e) * e).clamp_min(2.0 ** -126), torch.ones_like(most))
    y = x / scale
    if dtype == torch.int8:
        y = torch.round(y)
    else:
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
        y = torch.round(y / step) * step
    y = torch.where(torch.isfinite(most), y * scale, torch.full_like(y, math.nan))
    return y.flatten(-3, -2)[..., :rows, :], scale[..., 0, 0]


class Store:
    """A store in fp64: all tokens, their gathered weights, the kept positions and rows."""

    def __init__(self, p, dtype, block, keep):
        self.p, self.dtype, self.block, self.keep = p, dtype, block, keep
        shape = (p.batch, p.n_kv_heads)
        self.K = self.V = torch.zeros(*shape, 0, p.head_dim, dtype=torch.float64)
        self.w = torch.zeros(*shape, 0, dtype=torch.float64)
        self.idx = torch.zeros(*shape, 0, p.top_k, dtype=torch.long)
        self.k_rows = self.v_rows = self.K
        self.k_scale = self.v_scale = self.w           # of every kept row

    @property
    def n(self):
        return self.K.shape[2]

    def append(self, k, v, w=None, idx=None):
        """`idx`: the kept positions by the lag rule (the library's own selection)."""
        p = self.p
        self.K, self.V = torch.cat([self.K, k.double()], 2), torch.cat([self.V, v.double()], 2)
        self.w = torch.cat([self.w, torch.zeros(k.shape[:3], dtype=torch.float64) if w is None else w.double()], 2)
        while p.n_sink + (self.idx.shape[2] + 2) * p.lag < self.n:
            c = self.idx.shape[2]
            if self.keep == "weight":
                lo = p.n_sink + c * p.lag
                x = self.w[:, :, lo:lo + p.lag]
                at = torch.sort(x, dim=2, descending=True, stable=True).indices[:, :, :p.top_k].sort(dim=2).values + lo
            else:
                at = idx[:, :, c].long()
            self.idx = torch.cat([self.idx, at[:, :, None]], 2)
            for name, rows in (("k", self.K), ("v", self.V)):
                got, scale = held(rows.gather(2, at[..., None].expand(-1, -1, -1, p.head_dim)), self.dtype, self.block)
                setattr(self, name + "_rows", torch.cat([getattr(self, name + "_rows"), got], 2))
                if scale is not None:
                    scale = scale.repeat_interleave(self.block, 2)[:, :, :p.top_k]
                    setattr(self, name + "_scale", torch.cat([getattr(self, name + "_scale"), scale], 2))

    def decode(self, q):
        """(o, lse, weights of the ring's tokens) of the last token and what the kernel's roundings may add up to: the
        probabilities are rounded in front of the second product (2^-8 relative in front of bf16 rows, 2^-11 in front of
        8-bit rows), o is rounded to bf16, the exponents are off as in weights().  In front of 8-bit rows what is rounded to
        a half is p_j scale_j in units of 2^-7 of a running maximum of the same products (which the true one is not
        below): beside the relative error there is half of a half's smallest step, 2^-25 of that unit, for every code."""
        p, n = self.p, self.n
        B, Hq, d = q.shape
        G = Hq // p.n_kv_heads
        scale = (p.softmax_scale or 1 / math.sqrt(d))
        first = p.n_sink + self.idx.shape[2] * p.lag       # first ring position that is seen
        rows = [torch.cat([a, x[:, :, :min(p.n_sink, n)], x[:, :, first:]], 2)
                for a, x in ((self.k_rows, self.K), (self.v_rows, self.V))]
        m, ring = self.k_rows.shape[2], max(n - first, 0)
        k, v = (x.repeat_interleave(G, 1) for x in rows)
        s = torch.einsum("bhd,bhnd->bhn", q.double(), k) * scale
        T = torch.einsum("bhd,bhnd->bhn", q.double().abs(), k.abs()) * scale * LOG2E
        lse = torch.logsumexp(s, -1)
        P = torch.exp(s - lse[..., None])
        off = math.log(2) * 2.0 ** -23 * ((d / 8 + 4) * T + 3 * lse.abs()[..., None] * LOG2E) + 2.0 ** -20   # of an exponential
        lse_tol = (P * off).sum(-1) + 2.0 ** -22 * lse.abs() + 2.0 ** -20
        round_p = torch.full((P.shape[-1],), 2.0 ** -8, dtype=torch.float64)
        if self.dtype != torch.bfloat16:
            round_p[:m] = 2.0 ** -11
        o = torch.einsum("bhn,bhnd->bhd", P, v)
        o_tol = torch.einsum("bhn,bhnd->bhd", P * (round_p + off + lse_tol[..., None]), v.abs()) + 2.0 ** -8 * o.abs() + 2.0 ** -126
        if m and self.dtype != torch.bfloat16:
            sc = self.v_scale.repeat_interleave(G, 1)
            top = (P * torch.cat([sc, torch.ones(*sc.shape[:2], P.shape[-1] - m, dtype=torch.float64)], 2)).amax(-1)
            o_tol += 2.0 ** -32 * top[..., None] * (v[:, :, :m].abs() / sc[..., None]).sum(2)
        gained = P[..., P.shape[-1] - ring:].unflatten(1, (p.n_kv_heads, G)).sum(2)
        g_tol = (P * (off + lse_tol[..., None]))[..., P.shape[-1] - ring:].unflatten(1, (p.n_kv_heads, G)).sum(2)
        if self.keep == "weight" and ring:
            self.w[:, :, first:] += gained
        return (o, o_tol), (lse, lse_tol), (gained, g_tol)


def within(name, got, want, tol):
    err = (got.detach().double().cpu() - want).abs()
    bad = ~(err <= tol)
    worst = int((err - tol).nan_to_num(math.inf).argmax())
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {err.numel()} off, worst {err.flatten()[worst]:.3g} against "
                           f"{tol.flatten()[worst]:.3g} at {worst} (want {want.flatten()[worst]:.6g})")
