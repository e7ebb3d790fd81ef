"""Plain models of the rotation, the paged cache and the attention of drafted trees, in numpy on the CPU, and the roundings that the
kernels may differ by."""
import numpy as np
import torch

HALF_STEP = torch.finfo(torch.bfloat16).eps / 2      # 2^-8


def bf16(x):
    """float64 -> float32 -> bf16 -> float64, to nearest."""
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16().double().numpy()


def angles(n_pos, dim, base=10000.0):
    """cos, sin as float32 [n_pos, dim / 2]."""
    a = np.arange(n_pos)[:, None] * base ** (-np.arange(0, dim, 2) / dim)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def rotate(x, pos, cos, sin, interleaved=False, inverse=False, rounded=True):
    """x [..., tokens, d] (float64) at positions pos.  rounded: as a kernel does it (one product in 32 bits, one fused, then bf16);
    otherwise the formula in 64 bits."""
    half = cos.shape[1]
    first = np.arange(0, 2 * half, 2) if interleaved else np.arange(half)
    second = first + 1 if interleaved else first + half
    c, s = cos[pos].astype(np.float64), sin[pos].astype(np.float64)
    if inverse:
        s = -s
    a, b, out = x[..., first], x[..., second], np.array(x)
    if rounded:
        f32 = lambda v: v.astype(np.float32).astype(np.float64)
        out[..., first], out[..., second] = bf16(a * c + f32(b * -s)), bf16(b * c + f32(a * s))
    else:
        out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    return out


def cut(p, n):
    """Windows that a cache of n tokens holds by their kept rows."""
    return max((n - p.n_sink) // p.lag - 1, 0) if n >= p.n_sink else 0


def pages_of(p, page):
    return tuple(-(-x // page) for x in (p.n_sink, p.lag, p.top_k))


def place(p, page, pos):
    """(column of the table, row of the page) of the uncompressed token at `pos`."""
    if pos < p.n_sink:
        return pos // page, pos % page
    sinks, ring, _ = pages_of(p, page)
    w, i = divmod(pos - p.n_sink, p.lag)
    return sinks + w % 2 * ring + i // page, i % page


def kept_place(p, page, w, j):
    sinks, ring, kept = pages_of(p, page)
    return sinks + 2 * ring + w * kept + j // page, j % page


def ancestors(parent, m):
    """[m, m] bool: token i sees new token j."""
    sees = np.zeros((m, m), bool)
    for i in range(m):
        up = i - 1 if parent is None else parent[i]
        if up >= 0:
            sees[i] = sees[up]
        sees[i, i] = True
    return sees


def attend(q, k, v, sees, scale, rotated=False):
    """q [H, m, d], k, v [Hkv, n, d], sees [m, n] or [Hkv, m, n].  Returns o, lse, and bounds of what rounding may do to them: a probability
    is rounded to bf16 (half a step of each term), o to bf16; a score is a sum of d products in 32 bits (2^-24 of the terms' sum for
    each addition), and enters the exponent of p and the log-sum.  rotated: queries and new keys are sums of two bf16 (half a step of half a
    step, 2^-16, is lost of each, and their smaller parts' product)."""
    H, Hkv, d = q.shape[0], k.shape[0], q.shape[-1]
    o, lse, o_tol, lse_tol = [], [], [], []
    for h in range(H):
        kv = h * Hkv // H
        see = sees[kv] if sees.ndim == 3 else sees
        x = np.where(see, q[h] @ k[kv].T * scale, -np.inf)
        top = x.max(1, keepdims=True)
        e = np.exp(x - top)
        total = e.sum(1, keepdims=True)
        p = e / total
        o.append(p @ v[kv])
        lse.append((top + np.log(total))[:, 0])
        terms = p @ np.abs(v[kv])
        ds = ((d + 4) * 2.0 ** -24 + (3 * HALF_STEP ** 2 if rotated else 0)) * (np.where(see, np.abs(q[h]) @ np.abs(k[kv]).T, 0) * scale).max(1) + 2.0 ** -21
        o_tol.append((HALF_STEP + 2 * ds[:, None] + 2.0 ** -18) * terms + HALF_STEP * (np.abs(o[-1]) + HALF_STEP * terms))
        lse_tol.append(ds + 2.0 ** -21 + 2.0 ** -23 * np.abs(lse[-1]))
    return tuple(np.stack(t) for t in (o, lse, o_tol, lse_tol))
