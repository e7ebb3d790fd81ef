"""The paged cache on the GPU: pages to the bit and kept positions as lrsa_score_select keeps them, attention against 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2506_11498_b200 import lrsa
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu


def f64(t):
    return t.double().cpu().numpy()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Model:
    """What the cache of some sequences holds, by position, on the CPU; and the cache itself, its pages full of NaN at the start."""

    def __init__(self, p, page, n_seqs, dim=0, interleaved=False, seed=0):
        self.p, self.page, self.rng = p, page, np.random.default_rng(seed)
        self.gen = torch.Generator().manual_seed(seed)
        self.cache_width = lrsa.PagedCache(p, 1, page=page).table_width
        n_pages = n_seqs * self.cache_width + 2
        self.cache = lrsa.PagedCache(p, n_pages, page=page)
        self.cache.k_pages.fill_(float("nan"))
        self.cache.v_pages.fill_(float("nan"))
        self.table = np.full((n_seqs, self.cache_width), -1, np.int64)
        self.free = self.rng.permutation(n_pages).tolist()
        self.n = [0] * n_seqs
        empty = np.zeros((p.n_kv_heads, 0, p.head_dim))
        self.K, self.V = [empty] * n_seqs, [empty] * n_seqs        # rotated K (as bf16 holds it), V
        self.kept = torch.full((n_seqs, p.n_kv_heads, self.cache.w_cap, p.top_k), -1, dtype=torch.int32, device="cuda")
        self.rope, self.dim, self.interleaved = None, dim, interleaved
        if dim:
            self.cos, self.sin = ref.angles(p.seq_len, dim)
            self.rope = lrsa.Rope(torch.from_numpy(self.cos).cuda(), torch.from_numpy(self.sin).cuda(), interleaved)

    def rows(self, heads, n, token_major=True):
        x = torch.randn((n, heads, self.p.head_dim) if token_major else (heads, n, self.p.head_dim), generator=self.gen).bfloat16()
        return x.transpose(0, 1) if token_major else x

    def turned(self, x, pos, rounded=True):
        return ref.rotate(x, pos, self.cos, self.sin, self.interleaved, rounded=rounded) if self.dim else x

    def reach(self, s, n):
        """Pages for a sequence of n tokens."""
        for col in self.cache.columns(n):
            if self.table[s, col] < 0:
                self.table[s, col] = self.free.pop()

    def device(self, new):
        cu = np.concatenate([[0], np.cumsum(new)])
        return i32(self.table.tolist()), i32(self.n), i32(cu.tolist())

    def append(self, new, token_major=True, spare=0, pick=None):
        """new[s] tokens for every sequence.  spare: room behind them; pick: the new tokens are these rows of more."""
        p = self.p
        T = sum(new)
        src = T + spare if pick is None else int(max(pick, default=0)) + 3
        k, v = self.rows(p.n_kv_heads, src, token_major), self.rows(p.n_kv_heads, src, token_major)
        table, n_tokens, cu = self.device(new)      # what the step knew before it
        for s, m in enumerate(new):
            self.reach(s, self.n[s] + m)
        table = i32(self.table.tolist())
        self.cache.append(k.cuda() if not token_major else k.transpose(0, 1).contiguous().cuda().transpose(0, 1),
                          v.cuda() if not token_major else v.transpose(0, 1).contiguous().cuda().transpose(0, 1), table, n_tokens, cu,
                          rows=None if pick is None else i32(list(pick)), rope=self.rope, kept=self.kept)
        at = 0
        for s, m in enumerate(new):
            idx = np.arange(at, at + m) if pick is None else np.asarray(pick[at:at + m], int)
            pos = np.arange(self.n[s], self.n[s] + m)
            self.K[s] = np.concatenate([self.K[s], self.turned(f64(k)[:, idx], pos)], 1)
            self.V[s] = np.concatenate([self.V[s], f64(v)[:, idx]], 1)
            self.n[s] += m
            at += m
        assert self.cache.status() == 0

    def selected(self, s):
        """The kept positions of sequence s by lrsa_score_select over all its tokens: [Hkv, windows, top_k]."""
        p, n, w = self.p, self.n[s], ref.cut(self.p, self.n[s])
        if w == 0:
            return np.zeros((p.n_kv_heads, 0, p.top_k), int)
        q = lrsa.Params(1, p.n_q_heads, p.n_kv_heads, n, p.head_dim, p.lag, p.top_k, p.n_sink, std_ddof=p.std_ddof)
        K, V = (torch.from_numpy(x).bfloat16()[None].contiguous().cuda() for x in (self.K[s], self.V[s]))
        return lrsa.lrsa_score_select(q, K, V)[0][0, :, :w].cpu().numpy()

    def check_pages(self):
        """Every row that counts, to the bit; kept positions; and no other page of a sequence's touched."""
        p, page = self.p, self.page
        k_pages, v_pages = f64(self.cache.k_pages), f64(self.cache.v_pages)
        expect = np.full(k_pages.shape, np.nan), np.full(k_pages.shape, np.nan)
        for s, n in enumerate(self.n):
            w = ref.cut(p, n)
            idx = self.selected(s)
            assert np.array_equal(self.kept[s, :, :w].cpu().numpy(), idx), s
            for pos in list(range(min(n, p.n_sink))) + list(range(min(n, p.n_sink + w * p.lag), n)):
                col, row = ref.place(p, page, pos)
                for e, x in zip(expect, (self.K, self.V)):
                    e[self.table[s, col], :, row] = x[s][:, pos]
            for i in range(w):
                for j in range(p.top_k):
                    col, row = ref.kept_place(p, page, i, j)
                    for h in range(p.n_kv_heads):
                        for e, x in zip(expect, (self.K, self.V)):
                            e[self.table[s, col], h, row] = x[s][h, idx[h, i, j]]
        for got, want in zip((k_pages, v_pages), expect):
            there = ~np.isnan(want)
            assert np.array_equal(got[there], want[there])
            unused = [i for i in range(len(got)) if i not in set(self.table.ravel().tolist())]
            assert np.isnan(got[unused]).all()

    def attend(self, new, tree=True, max_new=None, token_major=True, given=True, **kw):
        """A random tree (or chain) of new[s] tokens for every sequence, against 64 bits."""
        p, T = self.p, sum(new)
        q, k, v = (self.rows(h, T, token_major) for h in (p.n_q_heads, p.n_kv_heads, p.n_kv_heads))
        parents = [[int(self.rng.integers(-1, i)) if i else -1 for i in range(m)] if tree else None for m in new]
        table, n_tokens, cu = self.device(new)
        on = lambda t: t.transpose(0, 1).contiguous().cuda().transpose(0, 1) if token_major else t.cuda()
        o, lse = self.cache.attend(on(q), on(k), on(v), table, n_tokens, cu, parent=i32(sum(parents, [])) if tree else None, rope=self.rope,
                                   max_new=(max(new) if given else None) if max_new is None else max_new, **kw)
        assert self.cache.status() == 0
        self.check_attend(new, parents, q, k, v, o, lse)
        return o, lse

    def check_attend(self, new, parents, q, k, v, o, lse):
        p, at = self.p, 0
        scale = p.softmax_scale or 1 / math.sqrt(p.head_dim)
        for s, m in enumerate(new):
            if m == 0:
                continue
            n, w = self.n[s], ref.cut(p, self.n[s])
            part = slice(at, at + m)
            at += m
            sees = ref.ancestors(parents[s], m)
            pos = n + sees.sum(1) - 1
            qs, ks, vs = self.turned(f64(q)[:, part], pos, False), self.turned(f64(k)[:, part], pos, False), f64(v)[:, part]
            idx = self.selected(s)
            keys, vals = [], []
            for h in range(p.n_kv_heads):
                seen = np.concatenate([np.arange(min(n, p.n_sink)), idx[h].ravel(), np.arange(min(n, p.n_sink + w * p.lag), n)]).astype(int)
                keys.append(np.concatenate([self.K[s][h, seen], ks[h]]))
                vals.append(np.concatenate([self.V[s][h, seen], vs[h]]))
            old = np.ones((m, keys[0].shape[0] - m), bool)
            want = ref.attend(qs, np.stack(keys), np.stack(vals), np.concatenate([old, sees], 1), scale, rotated=self.dim > 0)
            for name, got, x, tol in (("o", f64(o)[:, part], want[0], want[2]), ("lse", f64(lse)[:, part], want[1], want[3])):
                err = np.abs(got - x)
                assert (err <= tol).all(), (name, s, m, n, float((err / tol).max()))


P64 = dict(head_dim=64, lag=96, top_k=24, n_sink=5)
CASES = {   # params, page, rotated channels, interleaved
    "mha_d64": (lrsa.Params(1, 2, 2, 1500, 64, 96, 24, 5), 16, 64, False),
    "gqa7_d128": (lrsa.Params(1, 14, 2, 1500, 128, 128, 32, 4), 64, 128, False),
    "odd": (lrsa.Params(1, 6, 3, 1500, 64, 77, 19, 0), 32, 32, True),
    "whole_windows_kept": (lrsa.Params(1, 4, 1, 1500, 128, 50, 50, 130), 128, 48, False),
    "one_kept": (lrsa.Params(1, 3, 1, 1500, 64, 16, 1, 1), 16, 16, False),
    "no_rope": (lrsa.Params(1, 8, 2, 1500, 128, 200, 67, 3, std_ddof=0, softmax_scale=0.05), 64, 0, False),
}


def make(name, n_seqs, seed=0):
    p, page, dim, interleaved = CASES[name]
    return Model(p, page, n_seqs, dim, interleaved, seed)


@pytest.mark.parametrize("name", CASES)
def test_growth_by_steps_of_all_sizes(name):
    """Prompts of different lengths in one call, then tokens, drafts and pieces that cut none, one or several windows."""
    m = make(name, 4)
    L, S = m.p.lag, m.p.n_sink
    m.append([0, 1, S + 3 * L + 5, S + 2 * L])
    m.check_pages()
    m.append([1, 0, L, 1])
    m.append([S + 2 * L - 1, 3, 0, L - 1], token_major=False)
    m.check_pages()
    m.append([1, 1, 1, 1], spare=7)
    m.check_pages()
    m.append([2 * L + 3, S + 5 * L, L + 1, 4])
    m.check_pages()
    m.append([3, 0, 2, 5], pick=[0, 2, 3, 4, 6, 9, 10, 11, 12, 13])
    m.check_pages()


@pytest.mark.parametrize("name", CASES)
def test_token_by_token_is_the_prompt(name):
    """However the tokens came, the cache holds the same bits."""
    p, page, dim, interleaved = CASES[name]
    total = min(p.n_sink + 3 * p.lag + 2, 420)
    a, b = make(name, 1, seed=5), make(name, 1, seed=5)
    k, v = a.rows(p.n_kv_heads, total, False).cuda(), a.rows(p.n_kv_heads, total, False).cuda()
    for m in (a, b):
        m.reach(0, total)
    b.table = a.table
    table = i32(a.table.tolist())
    a.cache.append(k, v, table, i32([0]), i32([0, total]), rope=a.rope, kept=a.kept)
    n, one = i32([0]), i32([0, 1])
    for i in range(total):
        b.cache.append(k[:, i:i + 1], v[:, i:i + 1], table, n, one, rope=b.rope, kept=b.kept)
        n += 1
    w = ref.cut(p, total)
    assert torch.equal(a.kept[:, :, :w], b.kept[:, :, :w])
    for pos in list(range(min(total, p.n_sink))) + list(range(p.n_sink + w * p.lag, total)):
        col, row = ref.place(p, page, pos)
        for x, y in ((a.cache.k_pages, b.cache.k_pages), (a.cache.v_pages, b.cache.v_pages)):
            assert torch.equal(x[a.table[0, col], :, row], y[a.table[0, col], :, row]), pos
    for i in range(w):
        for j in range(p.top_k):
            col, row = ref.kept_place(p, page, i, j)
            assert torch.equal(a.cache.k_pages[a.table[0, col], :, row], b.cache.k_pages[a.table[0, col], :, row])
            assert torch.equal(a.cache.v_pages[a.table[0, col], :, row], b.cache.v_pages[a.table[0, col], :, row])


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("new", [[1, 1, 1, 1, 1], [0, 2, 1, 0, 2], [5, 1, 0, 4, 3], [33, 0, 7, 1, 64], [128, 3, 1, 0, 17]],
                         ids=["tokens", "pairs", "drafts", "trees", "full"])
def test_attend(name, new):
    m = make(name, 5, seed=1)
    L, S = m.p.lag, m.p.n_sink
    m.append([0, 1, S + L // 2, S + 2 * L, min(S + 6 * L + 3, 1300)])
    m.attend(new)
    m.attend(new, tree=False, token_major=False)
    m.append([1, S, L, L + 1, 2])
    m.attend(new, given=False)


def test_long_sequence_in_many_shares():
    p = lrsa.Params(1, 8, 2, 20000, 128, 512, 256, 4)
    m = Model(p, 64, 2, dim=128, seed=2)
    m.append([19000, 40])
    m.check_pages()
    for new in ([1, 1], [4, 2], [16, 16], [40, 1], [128, 128]):
        a, b = m.attend(new)
    again = m.cache   # results repeat bit by bit
    q, k, v = (m.rows(h, 50).cuda() for h in (8, 2, 2))
    args = m.device([40, 10])
    outs = [again.attend(q, k, v, *args, rope=m.rope, max_new=40) for _ in range(3)]
    assert all(torch.equal(x, y) for o in outs[1:] for x, y in zip(outs[0], o))


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("most", [1, 5, 20, 64])
def test_many_sequences_of_all_lengths(name, most):
    """More items than CTAs, empty caches and empty trees among them: a CTA works on several, one after the other."""
    n_seqs = 70 if most < 20 else 40
    m = make(name, n_seqs, seed=3)
    m.append([int(x) for x in m.rng.integers(0, 1400, n_seqs) * (m.rng.random(n_seqs) < 0.7)])
    for _ in range(2):
        m.attend([int(x) for x in m.rng.integers(0, most + 1, n_seqs)], max_new=most)
