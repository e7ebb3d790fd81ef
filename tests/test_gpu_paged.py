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


@pytest.mark.parametrize("name", CASES)
def test_more_cuts_than_run_at_once(name):
    """Prompts, and more tokens behind them, of so many windows that their cuts take turns on the SMs."""
    m = make(name, 40, seed=8)
    first = [int(x) for x in m.rng.integers(300, 900, 40)]
    m.append(first)
    m.check_pages()
    m.append([int(x) for x in m.rng.integers(200, 600, 40)])
    m.check_pages()


WIDE = {   # odd groups, windows longer than the scoring kernel's clusters take, tiny ones
    "g20": (lrsa.Params(1, 20, 1, 900, 64, 64, 16, 4), 16, 64, False),
    "g130": (lrsa.Params(1, 130, 1, 900, 128, 64, 16, 4), 32, 64, False),
    "g300": (lrsa.Params(1, 600, 2, 900, 64, 100, 7, 0), 64, 0, False),
    "mha24": (lrsa.Params(1, 24, 24, 900, 64, 33, 33, 2), 128, 32, True),
    "l1": (lrsa.Params(1, 4, 2, 300, 64, 1, 1, 0), 16, 16, False),
    "all_sinks": (lrsa.Params(1, 4, 2, 300, 128, 200, 3, 290), 64, 128, False),
}


@pytest.mark.parametrize("name", WIDE)
def test_wide_groups_and_odd_windows(name):
    p, page, dim, interleaved = WIDE[name]
    m = Model(p, page, 3, dim, interleaved, seed=4)
    m.append([p.seq_len // 3, 1, p.seq_len - 20])
    m.check_pages()
    m.attend([1, 1, 1])
    m.attend([3, 0, 7])
    m.append([5, 2, 12], pick=list(range(0, 38, 2)))
    m.check_pages()
    m.attend([2, 17, 1], tree=False)


@pytest.mark.parametrize("d, L", [(64, 9000), (128, 5001)])
def test_long_windows(d, L):
    p = lrsa.Params(1, 2, 1, 5 * L, d, L, L // 8, 3)
    m = Model(p, 128, 2, dim=d, seed=6)
    m.append([3 + 3 * L + 17, 3 + 2 * L - 1])
    m.append([1, 1])
    m.check_pages()
    m.attend([1, 30])


def test_a_thousand_sequences():
    p = lrsa.Params(1, 4, 2, 400, 64, 32, 8, 2)
    m = Model(p, 16, 1000, dim=64, seed=7)
    m.append([int(x) for x in m.rng.integers(0, 150, 1000)])
    m.append([int(x) for x in m.rng.integers(0, 3, 1000)])
    m.attend([1] * 1000)
    m.attend([int(x) for x in m.rng.integers(0, 12, 1000)], max_new=12)


def test_pages_far_into_a_large_pool():
    """More than 2^31 elements of K in front of the pages in use."""
    p = lrsa.Params(1, 8, 4, 900, 128, 128, 32, 4)
    m = Model(p, 64, 2, dim=128, seed=8)
    n_pages = (1 << 31) // (4 * 64 * 128) + 40
    small = m.cache
    m.cache = lrsa.PagedCache(p, 1, page=64)
    m.cache.n_pages, m.cache._shape = n_pages, torch.Size((n_pages, 4, 64, 128))
    m.cache.k_pages = torch.empty(m.cache._shape, dtype=torch.bfloat16, device="cuda")
    m.cache.v_pages = torch.empty_like(m.cache.k_pages)
    m.free = list(range(n_pages - 38, n_pages))
    m.append([700, 33])
    m.append([1, 300])
    used = sorted({int(x) for x in m.table.ravel() if x >= 0})
    assert min(used) * 4 * 64 * 128 >= 1 << 31
    for t, host in ((m.cache.k_pages, m.K), (m.cache.v_pages, m.V)):
        for s, n in enumerate(m.n):
            for pos in range(min(n, p.n_sink)):
                col, row = ref.place(p, 64, pos)
                assert np.array_equal(f64(t[m.table[s, col], :, row]), host[s][:, pos])
    m.attend([1, 1])
    m.attend([40, 3])
    del small


def test_infinities_and_nan_of_tokens_that_are_not_seen():
    """A row's result does not depend on drafts that it does not see, whatever they hold; a value that it sees does what it does in the formula."""
    for p, new in ((lrsa.Params(1, 4, 2, 600, 64, 64, 16, 4), 6), (lrsa.Params(1, 4, 2, 600, 128, 64, 16, 4), 3),
                   (lrsa.Params(1, 14, 2, 600, 128, 64, 16, 4), 30), (lrsa.Params(1, 8, 1, 600, 64, 64, 16, 4), 40)):
        m = Model(p, 16, 1, dim=64, seed=9)
        m.append([300])
        G = p.n_q_heads // p.n_kv_heads
        q, k, v = (m.rows(h, new, False).cuda() for h in (p.n_q_heads, p.n_kv_heads, p.n_kv_heads))
        parent = i32([-1] + [0 if i == 1 else -1 if i == 2 else i - 2 for i in range(1, new)])    # two chains: 0, 1, 3, 5 ... and 2, 4, 6 ...
        table, n_tokens, cu = m.device([new])
        args = (table, n_tokens, cu, parent, m.rope)
        want, want_lse = m.cache.attend(q, k, v, *args)
        k2, v2 = k.clone(), v.clone()
        k2[:, 2, 3], v2[:, 2, 5], v2[:, 2, 6], v2[:, 2, 7] = float("nan"), float("inf"), float("nan"), float("-inf")
        for bad_k in (k, k2):
            o, lse = m.cache.attend(q, bad_k, v2, *args)
            for i in [0, 1] + list(range(3, new, 2)):
                assert torch.equal(o[:, i], want[:, i]) and torch.equal(lse[:, i], want_lse[:, i])
            for i in range(2, new, 2):
                if bad_k is k:
                    assert torch.equal(lse[:, i], want_lse[:, i])
                    clean = [c for c in range(p.head_dim) if c not in (5, 6, 7)]
                    assert torch.equal(o[:, i, clean], want[:, i, clean])
                    assert (o[:, i, 5] == float("inf")).all() and torch.isnan(o[:, i, 6]).all() and (o[:, i, 7] == float("-inf")).all()
                else:
                    assert torch.isnan(o[:, i]).all() and torch.isnan(lse[:, i]).all()
        # both signs in one channel of two tokens of a line
        v3 = v.clone()
        v3[:, 0, 9], v3[:, 1, 9] = float("inf"), float("-inf")
        o, _ = m.cache.attend(q, k, v3, *args)
        assert (o[:, 0, 9] == float("inf")).all() and torch.isnan(o[:, 1, 9]).all() and torch.equal(o[:, 2::2], want[:, 2::2])
        # what is not finite in the cache is everybody's, in its channel
        col, row = ref.place(p, 16, 299)
        m.cache.v_pages[int(m.table[0, col]), :, row, 11] = float("inf")
        o, lse = m.cache.attend(q, k, v, *args)
        assert (o[:, :, 11] == float("inf")).all() and torch.equal(lse, want_lse)
        assert G >= 1


def test_scores_that_overflow_and_rows_of_zeros():
    p = lrsa.Params(1, 4, 2, 600, 64, 64, 16, 4)
    for new in (2, 20):
        m = Model(p, 32, 1, seed=10)
        m.append([200])
        q, k, v = (m.rows(h, new, False).cuda() for h in (4, 2, 2))
        table, n_tokens, cu = m.device([new])
        q[:, 0] = 0                                       # every key counts alike
        q[1, 1] *= 1e20
        o, lse = m.cache.attend(q, k, v, table, n_tokens, cu)
        w = ref.cut(p, 200)
        n = 4 + w * 16 + 200 - 4 - w * 64 + 1
        assert np.abs(f64(lse[:, 0]) - math.log(n)).max() < 1e-5
        assert torch.isfinite(o[[0, 2, 3]]).all() and torch.isfinite(lse[1, 1])      # one key has it all
        m.cache.k_pages.mul_(0)
        m.cache.v_pages.mul_(0)
        m.cache.k_pages.nan_to_num_()
        m.cache.v_pages.nan_to_num_()
        k0 = torch.full_like(k, -3e38)
        o, lse = m.cache.attend(torch.ones_like(q), k0, v, table, n_tokens, cu)      # the new tokens' scores are -infinity, the others' 0
        assert (o == 0).all() and np.abs(f64(lse) - math.log(n - 1)).max() < 1e-5


BAD = {   # what is wrong with which of three sequences
    "negative tokens": lambda a: a["n_tokens"].__setitem__(1, -1),
    "too many tokens": lambda a: a["n_tokens"].__setitem__(1, 2000),
    "counts go back": lambda a: a["cu_new"].__setitem__(2, a["cu_new"][1] - 1),
    "counts beyond the rows": lambda a: a["cu_new"].__setitem__(3, 1000),
    "a page that is not there": lambda a: a["table"].__setitem__((1, slice(None)), 1 << 30),
    "a negative page": lambda a: a["table"].__setitem__((1, slice(None)), -1),
}


@pytest.mark.parametrize("what", BAD)
@pytest.mark.parametrize("new", [1, 3, 20])
def test_counts_and_pages_that_cannot_be_used(what, new):
    p = lrsa.Params(1, 8, 2, 1500, 64, 64, 16, 4)
    m = Model(p, 16, 3, dim=64, seed=11)
    m.append([500, 300, 100])
    for s in range(3):
        m.reach(s, m.n[s] + new)
    table, n_tokens, cu = m.device([new] * 3)
    q, k, v = (m.rows(h, 3 * new).transpose(0, 1).contiguous().cuda().transpose(0, 1) for h in (8, 2, 2))
    good, _ = m.cache.attend(q, k, v, table, n_tokens, cu, rope=m.rope, max_new=new)
    assert m.cache.status() == 0
    args = dict(table=table.clone(), n_tokens=n_tokens.clone(), cu_new=cu.clone())
    BAD[what](args)
    o, _ = m.cache.attend(q, k, v, **args, rope=m.rope, max_new=new)
    assert m.cache.status() == 1
    if what != "counts beyond the rows":
        assert torch.equal(o[:, :new], good[:, :new])            # the first sequence is as it was
    pages = m.cache.k_pages.clone(), m.cache.v_pages.clone()
    m.cache.append(k, v, **args, rope=m.rope)
    assert m.cache.status() == 1
    # nothing is written but the pages of the other sequences
    fine = [0, 1] if what == "counts beyond the rows" else [0, 2]
    mine = sorted({int(x) for x in m.table[fine].ravel() if x >= 0})
    others = [i for i in range(m.cache.n_pages) if i not in mine]
    for x, y in zip(pages, (m.cache.k_pages, m.cache.v_pages)):
        assert torch.equal(x[others].view(torch.int16), y[others].view(torch.int16))
    m.cache.attend(q, k, v, table, n_tokens, cu, rope=m.rope, max_new=new)
    assert m.cache.status() == 0


def test_other_numbers_on_the_device_that_cannot_be_used():
    p = lrsa.Params(1, 8, 2, 400, 64, 64, 16, 4)
    m = Model(p, 16, 2, dim=64, seed=12)
    m.append([380, 100])
    for s in range(2):
        m.reach(s, 400 if s == 0 else 140)
    q, k, v = (m.rows(h, 40, False).cuda() for h in (8, 2, 2))
    table, n, cu = m.device([20, 20])
    for max_new in (20, 40):
        m.cache.attend(q, k, v, table, n, cu, rope=m.rope, max_new=max_new)
        assert m.cache.status() == 0
    m.cache.attend(q, k, v, table, n, cu, rope=m.rope, max_new=19)              # more of them than was said
    assert m.cache.status() == 1
    m.cache.attend(q, k, v, table, n, cu, max_new=20)                            # without a rope positions may go on
    m.cache.attend(q, k, v, table, n + 20, cu, max_new=20)
    assert m.cache.status() == 0
    m.cache.attend(q, k, v, table, i32([381, 100]), cu, rope=m.rope, max_new=20)  # the rope's last position
    assert m.cache.status() == 1
    for bad in (1, 20, -2):
        parent = i32(list(range(-1, 19)) * 2)
        parent[1] = bad
        m.cache.attend(q, k, v, table, n, cu, parent=parent, rope=m.rope, max_new=20)
        assert m.cache.status() == 1
    for bad in (40, -1):
        rows = torch.arange(40, dtype=torch.int32, device="cuda")
        rows[3] = bad
        m.cache.append(k, v, table, n, cu, rows=rows, rope=m.rope)
        assert m.cache.status() == 1
    m.cache.append(k, v, table, i32([381, 100]), cu, rope=m.rope)                 # beyond seq_len
    assert m.cache.status() == 1
    m.cache.append(k, v, table, n, cu, rope=m.rope)
    assert m.cache.status() == 0


def test_rows_behind_the_last_sequence_stay():
    p = lrsa.Params(1, 8, 2, 400, 64, 64, 16, 4)
    for new in (1, 20):
        m = Model(p, 16, 2, dim=64, seed=13)
        m.append([100, 50])
        q, k, v = (m.rows(h, 2 * new + 9, False).cuda() for h in (8, 2, 2))
        k[:, 2 * new:], v[:, 2 * new:] = float("nan"), float("nan")
        table, n, cu = m.device([new, new])
        o, lse = torch.full_like(q, 7.0), torch.full((8, 2 * new + 9), 7.0, device="cuda")
        m.cache.attend(q, k, v, table, n, cu, rope=m.rope, max_new=new, o=o, lse=lse)
        assert (o[:, 2 * new:] == 7).all() and (lse[:, 2 * new:] == 7).all() and torch.isfinite(o).all()


def step(m, q, k, v, table, n, cu, parent, rows, cu_kept, taken):
    """A step of a server: drafts are attended, some are accepted and enter the cache."""
    o, lse = m.cache.attend(q, k, v, table, n, cu, parent=parent, rope=m.rope, max_new=12)
    m.cache.append(k, v, table, n, cu_kept, rows=rows, rope=m.rope)
    n += taken
    return o, lse


@pytest.mark.parametrize("heads", [(4, 2), (14, 2)])
def test_a_captured_step_serves_the_later_ones(heads):
    """The counts are on the device: one graph, replayed while sequences of different lengths grow over windows' ends."""
    p = lrsa.Params(1, *heads, 1200, 64, 48, 12, 4)
    a, b = Model(p, 16, 3, dim=64, seed=14), Model(p, 16, 3, dim=64, seed=14)
    rng = np.random.default_rng(0)
    for m in (a, b):
        m.append([300, 40, 3])
        for s in range(3):
            m.reach(s, 1100)
    b.table = a.table
    b.cache.k_pages.copy_(a.cache.k_pages)
    b.cache.v_pages.copy_(a.cache.v_pages)
    table = i32(a.table.tolist())
    n_a, n_b = i32(a.n), i32(a.n)
    T = 24
    bufs = dict(q=a.rows(heads[0], T, False).cuda(), k=a.rows(heads[1], T, False).cuda(), v=a.rows(heads[1], T, False).cuda(),
                cu=i32([0, 8, 20, 24]), parent=i32([-1] * T), rows=i32([0] * T), cu_kept=i32([0, 1, 2, 3]), taken=i32([1, 1, 1]))
    n_warm = n_a.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.cache.attend(bufs["q"], bufs["k"], bufs["v"], table, n_warm, bufs["cu"], parent=bufs["parent"], rope=a.rope, max_new=12)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(a, bufs["q"], bufs["k"], bufs["v"], table, n_a, bufs["cu"], bufs["parent"], bufs["rows"], bufs["cu_kept"], bufs["taken"])
    for i in range(40):
        new = [int(x) for x in rng.integers(1, 9, 3)]
        cu = np.concatenate([[0], np.cumsum(new)])
        parent, rows, kept = [], [], []
        for s, x in enumerate(new):
            up = [int(rng.integers(-1, j)) if j else -1 for j in range(x)]
            line, j = [], x - 1
            while j >= 0:
                line.append(int(cu[s]) + j)
                j = up[j]
            parent += up
            rows += line[::-1]
            kept.append(len(line))
        for name, value in (("cu", cu), ("cu_kept", np.concatenate([[0], np.cumsum(kept)])), ("taken", kept)):
            bufs[name].copy_(i32([int(x) for x in value]))
        bufs["parent"].copy_(i32(parent + [0] * (T - len(parent))))
        bufs["rows"].copy_(i32(rows + [0] * (T - len(rows))))
        for name, h in (("q", heads[0]), ("k", heads[1]), ("v", heads[1])):
            bufs[name].copy_(a.rows(h, T, False))
        graph.replay()
        o, lse = step(b, bufs["q"], bufs["k"], bufs["v"], table, n_b, bufs["cu"], bufs["parent"], bufs["rows"], bufs["cu_kept"], bufs["taken"])
        used = int(cu[-1])
        assert torch.equal(n_a, n_b)
        assert torch.equal(out[0][:, :used], o[:, :used]) and torch.equal(out[1][:, :used], lse[:, :used]), i
        assert a.cache.status() == 0 and b.cache.status() == 0
    for x, y in ((a.cache.k_pages, b.cache.k_pages), (a.cache.v_pages, b.cache.v_pages)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_on_another_stream():
    p = lrsa.Params(1, 14, 2, 900, 128, 64, 16, 4)
    m = Model(p, 32, 2, dim=128, seed=15)
    m.append([400, 77])
    q, k, v = (m.rows(h, 20, False).cuda() for h in (14, 2, 2))
    table, n, cu = m.device([12, 8])
    want = m.cache.attend(q, k, v, table, n, cu, rope=m.rope)
    side = torch.cuda.Stream()
    for _ in range(5):
        side.wait_stream(torch.cuda.current_stream())
        got = m.cache.attend(q, k, v, table, n, cu, rope=m.rope, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_two_caches_at_once():
    """Layers share the table and the counts, nothing else."""
    p = lrsa.Params(1, 14, 2, 900, 128, 64, 16, 4)
    ms = [Model(p, 32, 2, dim=128, seed=16) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in ms]
    for m in ms:
        m.append([400, 77])
    calls = []
    for m in ms:
        q, k, v = (m.rows(h, 40, False).cuda() for h in (14, 2, 2))
        calls.append((q, k, v) + m.device([30, 10]))
    want = [m.cache.attend(*c, rope=m.rope) for m, c in zip(ms, calls)]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for m, c, st in zip(ms, calls, streams):
            with torch.cuda.stream(st):
                got.append(m.cache.attend(*c, rope=m.rope))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_from_a_prompt_to_tokens():
    """The operators as they are used together: rotation, selection and attention of a prompt, its rows into the cache, then token by
    token; each token's output against the row that lrsa_attn_fwd gives it when all of them are the prompt."""
    B, Hq, Hkv, d, L, K, S = 1, 8, 2, 128, 64, 16, 4
    N, prompt = 520, 300
    rope = lrsa.Rope.of_base(10000.0, d, N)
    gen = torch.Generator().manual_seed(17)
    Q, Kx, V = (torch.randn(B, h, N, d, generator=gen).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    whole = lrsa.Params(B, Hq, Hkv, N, d, L, K, S)
    Qr, Kr = lrsa.lrsa_rotate(whole, Q, Kx, rope)
    idx, _ = lrsa.lrsa_score_select(whole, Kr, V)
    O, LSE = lrsa.lrsa_attn_fwd(whole, Qr, Kr, V, idx)
    cache = lrsa.PagedCache(whole, 64, page=16)
    table = torch.full((1, cache.table_width), -1, dtype=torch.int32)
    cols = cache.columns(N)
    table[0, cols] = torch.randperm(64, generator=gen)[:len(cols)].int()
    table, n = table.cuda(), i32([0])
    cache.append(Kr[0, :, :prompt], V[0, :, :prompt], table, n, i32([0, prompt]))     # rotated already
    n += prompt
    t = prompt
    while t < N:
        m = min(1 if t % 3 else 7, N - t, L - (t - S) % L)        # a chain inside a chunk sees what the mask shows it
        part = slice(t, t + m)
        o, lse = cache.attend(Q[0, :, part], Kx[0, :, part], V[0, :, part], table, n, i32([0, m]), rope=rope, max_new=m)
        # bf16 probabilities and outputs on both sides (2^-8 each of terms of size 1 or less); the forward's queries are rounded
        assert (o.float() - O[0, :, part].float()).abs().max() < 2e-2 and (lse - LSE[0, :, part]).abs().max() < 5e-3, t
        cache.append(Kx[0, :, part], V[0, :, part], table, n, i32([0, m]), rope=rope)
        n += m
        t += m
        assert cache.status() == 0


def test_training_through_the_rotation():
    """Gradients of the unrotated queries and keys, against autograd in 64 bits through rotation and masked attention."""
    from oracle import lrsa_oracle as orc
    B, Hq, Hkv, N, d, L, K, S = 1, 4, 2, 200, 64, 32, 8, 4
    p = lrsa.Params(B, Hq, Hkv, N, d, L, K, S)
    cos, sin = ref.angles(N, d)
    rope = lrsa.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), True)
    gen = torch.Generator().manual_seed(18)
    Q, Kx, V, dO = (torch.randn(B, h, N, d, generator=gen).bfloat16() for h in (Hq, Hkv, Hkv, Hq))
    Qr, Kr = lrsa.lrsa_rotate(p, Q.cuda(), Kx.cuda(), rope)
    idx, _ = lrsa.lrsa_score_select(p, Kr, V.cuda())
    O, LSE = lrsa.lrsa_attn_fwd(p, Qr, Kr, V.cuda(), idx)
    dQr, dKr, dV = lrsa.lrsa_attn_bwd(p, Qr, Kr, V.cuda(), O, dO.cuda(), LSE, idx)
    dQ, dK = lrsa.lrsa_rotate(p, dQr, dKr, rope, inverse=True)
    op = orc.OracleParams(B, Hq, Hkv, N, d, L, K, S)
    hidx = idx.cpu().numpy()
    q, k, v = (x.double().requires_grad_() for x in (Q, Kx, V))
    c, s = torch.from_numpy(cos).double(), torch.from_numpy(sin).double()

    def turn(x):
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)

    x = turn(q) @ turn(k).repeat_interleave(Hq // Hkv, 1).transpose(-1, -2) / math.sqrt(d)
    vis = torch.stack([torch.from_numpy(np.stack([orc.visible_row(op, hidx, 0, h // (Hq // Hkv), t) for t in range(N)])) for h in range(Hq)])
    o = torch.softmax(x.masked_fill(~vis.bool(), -math.inf), -1) @ v.repeat_interleave(Hq // Hkv, 1)
    o.backward(dO.double())
    for name, got, want in (("dQ", dQ, q.grad), ("dK", dK, k.grad), ("dV", dV, v.grad)):
        err = (got.double().cpu() - want).norm() / want.norm()
        assert err < 1.5e-2, (name, float(err))     # the backward's bound on this norm, 1e-2, and one more rounding to bf16


def test_no_new_tokens():
    p = lrsa.Params(1, 14, 2, 400, 64, 64, 16, 4)
    m = Model(p, 16, 2, dim=64, seed=19)
    m.append([100, 50])
    before = m.cache.k_pages.clone()
    table, n, cu = m.device([0, 0])
    for T in (0, 5):                       # no rows at all, or room for some
        q, k, v = (m.rows(h, T, False).cuda() for h in (14, 2, 2))
        for max_new in (1, 20):
            o, lse = m.cache.attend(q, k, v, table, n, cu, rope=m.rope, max_new=max_new)
            assert o.shape == (14, T, 64) and lse.shape == (14, T) and m.cache.status() == 0
        m.cache.append(k, v, table, n, cu, rope=m.rope)
        assert m.cache.status() == 0 and torch.equal(before.view(torch.int16), m.cache.k_pages.view(torch.int16))


def test_launches_and_the_binding_without_its_module(monkeypatch):
    p = lrsa.Params(1, 14, 2, 900, 128, 64, 16, 4)
    m = Model(p, 32, 2, dim=128, seed=20)
    m.append([400, 77])
    assert lrsa.lrsa_last_launch_count() == 3
    for s in range(2):
        m.reach(s, m.n[s] + 12)
    q, k, v = (m.rows(h, 20, False).cuda() for h in (14, 2, 2))
    for new, launches in (([1, 1], 2), ([12, 8], 3)):
        args = m.device(new)
        with monkeypatch.context() as c:
            outs = []
            for call in (lrsa._calls(), lrsa._CtypesCalls(lrsa.lib())):
                c.setattr(lrsa, "_call", call)
                o, lse = m.cache.attend(q, k, v, *args, rope=m.rope, max_new=max(new))
                assert lrsa.lrsa_last_launch_count() == launches
                m.cache.append(k, v, *args, rope=m.rope)
                assert lrsa.lrsa_last_launch_count() == 1
                pages = m.cache.k_pages.clone()
                x, _ = lrsa.lrsa_rotate(lrsa.Params(1, 14, 2, 20, 128, 16, 4, 0), q[None], None, m.rope)
                outs.append((o[:, :sum(new)], lse[:, :sum(new)], pages.view(torch.int16), x))
        assert all(torch.equal(a, b) for a, b in zip(*outs))
