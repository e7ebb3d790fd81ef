"""The paged cache on the GPU where weights underflow, numbers on the device cannot be used, and steps are captured."""
import math

import numpy as np
import pytest
import torch

from paper_2506_11498_b200 import lrsa
from tests import paged_reference as ref
from tests.test_gpu_paged import Model, f64, i32

pytestmark = pytest.mark.gpu


def far_scores(m, new, n_seqs):
    """q, k, v of `new` tokens for every sequence, and pages, whose scores are 200 for every second window of tokens of the cache and 0 for the
    others and for the new tokens: in 32 bits those have no weight at all."""
    p = m.p
    q = torch.ones(p.n_q_heads, new * n_seqs, p.head_dim, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(p.n_kv_heads, new * n_seqs, p.head_dim, dtype=torch.bfloat16, device="cuda")
    v = torch.randn(k.shape, generator=m.gen).bfloat16().cuda()
    m.cache.k_pages.fill_(200 / p.head_dim ** 0.5)
    m.cache.v_pages.copy_(torch.randn(m.cache.v_pages.shape, generator=m.gen).bfloat16())
    return q, k, v


@pytest.mark.parametrize("heads, d, new", [((4, 2), 64, 3), ((8, 2), 128, 3), ((14, 2), 128, 9), ((8, 1), 64, 40)],
                         ids=["rows6", "rows12", "rows63", "rows320"])
@pytest.mark.parametrize("n_seqs, tokens", [(1, 2500), (2, 300), (200, 40)])
def test_an_infinity_that_is_seen_stays_one_however_little_it_weighs(heads, d, new, n_seqs, tokens):
    """Whether the item is one CTA's or divided: a sum with an infinity or NaN in it is not a finite number."""
    p = lrsa.Params(1, *heads, 2600, d, 1024, 16, 4)
    m = Model(p, 16, n_seqs, seed=1)
    m.append([tokens] * n_seqs)
    q, k, v = far_scores(m, new, n_seqs)
    args = m.device([new] * n_seqs)
    want, want_lse = m.cache.attend(q, k, v, *args, max_new=new)
    assert torch.isfinite(want).all()
    v[:, ::new, 5], v[:, ::new, 6], v[:, 1::new, 7] = float("inf"), float("nan"), float("-inf")   # the first token of each, and the second
    o, lse = m.cache.attend(q, k, v, *args, max_new=new)
    assert torch.equal(lse, want_lse)
    clean = [c for c in range(d) if c not in (5, 6, 7)]
    assert torch.equal(o[..., clean], want[..., clean])
    assert (o[..., 5] == float("inf")).all() and torch.isnan(o[..., 6]).all()
    assert (o[:, 1::new, 7] == float("-inf")).all() and torch.equal(o[:, ::new, 7], want[:, ::new, 7])


@pytest.mark.parametrize("heads, d, new", [((4, 2), 64, 3), ((8, 2), 128, 3), ((14, 2), 128, 9), ((8, 1), 64, 40)],
                         ids=["rows6", "rows12", "rows63", "rows320"])
@pytest.mark.parametrize("n_seqs, tokens", [(1, 2500), (2, 300), (200, 300)])
def test_an_infinity_in_the_pages_stays_one_however_little_it_weighs(heads, d, new, n_seqs, tokens):
    p = lrsa.Params(1, *heads, 2600, d, 1024, 16, 4)
    m = Model(p, 16, n_seqs, seed=2)
    m.append([tokens] * n_seqs)
    q, k, v = far_scores(m, new, n_seqs)
    args = m.device([new] * n_seqs)
    # the first tokens have score 0 too, whole key tiles of them, and one in the second such tile an infinite value
    for s in range(n_seqs):
        at = [ref.place(p, 16, pos) for pos in range(max(260, tokens // 2))]
        pages, rows = i32([int(m.table[s, col]) for col, _ in at]).long(), i32([row for _, row in at]).long()
        m.cache.k_pages[pages, :, rows] = 0
        m.cache.v_pages[pages[180], :, rows[180], 11] = float("inf")
    o, lse = m.cache.attend(q, k, v, *args, max_new=new)
    assert torch.isfinite(lse).all()
    assert not torch.isfinite(o[..., 11]).any()
    assert torch.isfinite(o[..., [c for c in range(d) if c != 11]]).all()


def twins(p, page, tokens, reach, **kw):
    """Two caches that hold the same in the same pages, and the table."""
    a, b = (Model(p, page, len(tokens), seed=3, **kw) for _ in "ab")
    for m in (a, b):
        m.append(tokens)
    for s, n in enumerate(reach):
        a.reach(s, n)
    b.table = a.table
    b.cache.k_pages.copy_(a.cache.k_pages)
    b.cache.v_pages.copy_(a.cache.v_pages)
    return a, b, i32(a.table.tolist())


def same_pages(a, b):
    return all(torch.equal(x.view(torch.int16), y.view(torch.int16))
               for x, y in ((a.cache.k_pages, b.cache.k_pages), (a.cache.v_pages, b.cache.v_pages)))


RANGES = {   # boundaries that go back
    "the first one only": [0, 30, 10, 20, 40],
    "first and last": [0, 10, 5, 30, 42],
    "all behind a large one": [0, 15, 90, 20, 40],
    "the second only": [-3, 4, 30, 22, 41],
}


def that_count(cu, room, most, apart=True):
    """(sequence, begin, end) of those that begin at or behind every boundary in front of them; not apart: of all whose own two can be used."""
    return [(s, cu[s], cu[s + 1]) for s in range(len(cu) - 1)
            if max([0] + (cu[:s] if apart else [])) <= cu[s] <= cu[s + 1] <= room and cu[s + 1] - cu[s] <= most]


@pytest.mark.parametrize("what", RANGES)
@pytest.mark.parametrize("times, rope", [(1, 64), (12, 64), (12, 0)], ids=["one_launch", "several_launches", "several_no_rope"])
def test_appends_whose_ranges_would_overlap(what, times, rope):
    """A sequence's keys are its own, rotated for its own positions.  Of prompts the later ones are left out; few tokens are each sequence's."""
    p = lrsa.Params(1, 8, 2, 1500, 64, 64, 16, 4)
    tokens = [0, 150, 30, 3]
    a, b, table = twins(p, 16, tokens, [n + 540 for n in tokens], dim=rope)
    cu = [x * times for x in RANGES[what]]
    T = 45 * times
    k, v = (a.rows(2, T, False).cuda() for _ in "kv")
    a.cache.append(k, v, table, i32(a.n), i32(cu), rope=a.rope)
    assert a.cache.status() == 1
    for s, begin, end in that_count(cu, T, T, apart=times > 1):     # one at a time
        one = [begin] * (s + 1) + [end] * (4 - s)
        b.cache.append(k, v, table, i32(b.n), i32(one), rope=b.rope)
        assert b.cache.status() == 0
    assert same_pages(a, b)


@pytest.mark.parametrize("what", RANGES)
@pytest.mark.parametrize("heads, most", [((2, 2), 6), ((4, 2), 6), ((8, 2), 30), ((14, 2), 30)], ids=["few", "few12", "tile", "tiles"])
def test_attends_whose_ranges_would_overlap(what, heads, most):
    p = lrsa.Params(1, *heads, 1500, 64, 64, 16, 4)
    m = Model(p, 16, 4, dim=64, seed=4)
    m.append([500, 0, 30, 150])
    cu = [x * most // 30 for x in RANGES[what]]
    T = 45 * most // 30
    q, k, v = (m.rows(h, T, False).cuda() for h in (heads[0], 2, 2))
    table = i32(m.table.tolist())
    o, lse = torch.full_like(q, 7.0), torch.full((heads[0], T), 7.0, device="cuda")
    m.cache.attend(q, k, v, table, i32(m.n), i32(cu), rope=m.rope, max_new=most, o=o, lse=lse)
    assert m.cache.status() == 1
    left = torch.ones(T, dtype=torch.bool)
    for s, begin, end in that_count(cu, T, most):
        one = [begin] * (s + 1) + [end] * (4 - s)
        want, want_lse = m.cache.attend(q, k, v, table, i32(m.n), i32(one), rope=m.rope, max_new=most)
        part = slice(begin, end)
        left[part] = False
        # (the items may be dealt out otherwise: on both sides a rounding of the probabilities and one of the sum, of values below 5)
        assert end > begin and (o[:, part].float() - want[:, part].float()).abs().max() <= 4 * 5 * ref.HALF_STEP
        assert torch.allclose(lse[:, part], want_lse[:, part], rtol=1e-5, atol=1e-5)
    assert (o[:, left] == 7).all() and (lse[:, left] == 7).all()


@pytest.mark.parametrize("n_seqs", [40, 300])
def test_many_sequences_behind_a_boundary_that_goes_back(n_seqs):
    """The boundaries in front are looked at by warps and blocks, 32 and 256 at a time."""
    p = lrsa.Params(1, 4, 2, 900, 64, 64, 16, 4)
    for at in (5, 33, n_seqs - 3):
        for new in (3, 80):
            tokens = [int(x) for x in np.random.default_rng(at).integers(0, 300, n_seqs)]
            a, b, table = twins(p, 16, tokens, [n + 4 * new for n in tokens], dim=64)
            k, v = (a.rows(2, new * n_seqs, False).cuda() for _ in "kv")
            cu = [new * s for s in range(n_seqs + 1)]
            cu[at] = new * (at - 3)
            a.cache.append(k, v, table, i32(a.n), i32(cu), rope=a.rope)
            few = lrsa.lrsa_last_launch_count() == 1
            assert a.cache.status() == 1 and few == (new == 3 and n_seqs == 40)
            # the one in front has its end before its beginning, the one behind begins too early: of prompts both are left out
            parts = [[new * min(s, at - 1) for s in range(n_seqs + 1)], [new * max(s, at + 1) for s in range(n_seqs + 1)]]
            if few:
                parts.append([cu[at]] * (at + 1) + [cu[at + 1]] * (n_seqs - at))
            for part in parts:
                b.cache.append(k, v, table, i32(b.n), i32(part), rope=b.rope)
                assert b.cache.status() == 0
            assert same_pages(a, b)
            if new == 3:
                q = a.rows(4, new * n_seqs, False).cuda()
                for heads_new in (3, 60):      # the kernel for few, the one for many
                    o, _ = a.cache.attend(q, k, v, table, i32(a.n), i32(cu), rope=a.rope, max_new=heads_new, o=torch.full_like(q, 7.0))
                    assert a.cache.status() == 1
                    out = torch.zeros(new * n_seqs, dtype=torch.bool)
                    out[new * (at - 1):new * (at + 1)] = True
                    assert (o[:, out] == 7).all() and not (o[:, ~out] == 7).all(-1).any()


BAD = {   # what is wrong with which of three sequences
    "negative tokens": lambda a: a["n_tokens"].__setitem__(1, -1),
    "too many tokens": lambda a: a["n_tokens"].__setitem__(1, 2000),
    "counts go back": lambda a: a["cu_new"].__setitem__(2, a["cu_new"][1] - 1),
    "counts beyond the rows": lambda a: a["cu_new"].__setitem__(3, 10000),
    "a page that is not there": lambda a: a["table"].__setitem__((1, slice(None)), 1 << 30),
    "a negative page": lambda a: a["table"].__setitem__((1, slice(None)), -1),
    "a row that is not there": lambda a: a["rows"].__setitem__(300, 750),
    "a negative row": lambda a: a["rows"].__setitem__(300, -1),
}


@pytest.mark.parametrize("what", BAD)
def test_prompts_with_numbers_that_cannot_be_used(what):
    """As the short calls: told by the status, nothing written but the pages of the other sequences, those to the bit."""
    p = lrsa.Params(1, 8, 2, 1500, 64, 64, 16, 4)
    a, b, table = twins(p, 16, [500, 300, 0], [750, 550, 250], dim=64)
    k, v = (a.rows(2, 750, False).cuda() for _ in "kv")
    fresh = lambda: dict(table=table.clone(), n_tokens=i32(a.n), cu_new=i32([0, 250, 500, 750]), rows=torch.arange(750, dtype=torch.int32, device="cuda"))
    args = fresh()
    BAD[what](args)
    a.cache.append(k, v, **args, rope=a.rope)
    assert lrsa.lrsa_last_launch_count() == 3 and a.cache.status() == 1
    b.cache.append(k, v, **{**fresh(), "cu_new": i32([0, 250, 250, 250])}, rope=b.rope)
    fine = {0} if what in ("counts go back", "counts beyond the rows") else {0, 2}
    if 2 in fine:
        b.cache.append(k, v, **{**fresh(), "cu_new": i32([500, 500, 500, 750])}, rope=b.rope)
    if what == "counts beyond the rows":
        b.cache.append(k, v, **{**fresh(), "cu_new": i32([250, 250, 500, 500])}, rope=b.rope)
        fine = {0, 1}
    others = [i for i in range(a.cache.n_pages) if i not in {int(x) for s in {0, 1, 2} - fine for x in a.table[s] if x >= 0}]
    if "row" not in what:
        others = list(range(a.cache.n_pages))      # (of a bad row another one is taken: its sequence's pages hold something)
    for x, y in ((a.cache.k_pages, b.cache.k_pages), (a.cache.v_pages, b.cache.v_pages)):
        assert torch.equal(x[others].view(torch.int16), y[others].view(torch.int16))
    a.cache.append(k, v, **fresh(), rope=a.rope)
    assert a.cache.status() == 0


def test_prompts_on_another_stream_and_captured():
    p = lrsa.Params(1, 8, 2, 1500, 64, 64, 16, 4)
    a, b, table = twins(p, 16, [0, 300], [900, 1200], dim=64)
    k, v = (a.rows(2, 800, False).cuda() for _ in "kv")
    n, cu = i32(a.n), i32([0, 400, 800])
    b.cache.append(k, v, table, n, cu, rope=b.rope)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.cache.append(k, v, table, n, cu, rope=a.rope, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert a.cache.status() == 0 and same_pages(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.cache.append(k, v, table, n, cu, rope=a.rope)
        n += cu.diff()
    for step in (400, 300):
        new = [step, 800 - step]
        k.copy_(a.rows(2, 800, False))
        v.copy_(a.rows(2, 800, False))
        cu.copy_(i32([0, step, 800]))
        n.copy_(i32([step, 500 - step]))
        b.cache.append(k, v, table, n, cu, rope=b.rope)
        graph.replay()
        assert a.cache.status() == 0 and same_pages(a, b), new
        assert n.tolist() == [step + new[0], 500 - step + new[1]]


def a_step(seed, heads=(8, 2)):
    p = lrsa.Params(1, *heads, 1500, 64, 64, 16, 4)
    m = Model(p, 16, 2, dim=64, seed=seed)
    m.append([300, 40])
    for s in range(2):
        m.reach(s, 1400)
    q, k, v = (m.rows(h, 40, False).cuda() for h in (heads[0], 2, 2))
    return m, q, k, v, i32(m.table.tolist()), i32(m.n), i32([0, 20, 40])


@pytest.mark.parametrize("most", [2, 20], ids=["few", "tile"])
def test_what_an_attend_found_is_told_behind_its_append(most):
    """A step is attend, then append: what only the attend can find, and an append that everything is right for."""
    m, q, k, v, table, n, _ = a_step(5)
    cu = i32([0, most, 2 * most])
    parent = i32(list(range(-1, most - 1)) * 2)
    wrong = parent.clone()
    wrong[1] = 1
    for bad in (dict(parent=wrong, max_new=most), dict(parent=parent, max_new=most - 1)):
        m.cache.attend(q, k, v, table, n, cu, rope=m.rope, **{**bad, "parent": torch.cat([bad["parent"], bad["parent"].new_zeros(40 - 2 * most)])})
        m.cache.append(k, v, table, n, cu, rope=m.rope)
        m.cache.attend(q, k, v, table, n, cu, rope=m.rope, max_new=most)
        assert lrsa.lrsa_workspace_status(m.cache.ws) == 0       # of the last call
        assert m.cache.status() == 1 and m.cache.status() == 0
    for _ in range(2):
        m.cache.attend(q, k, v, table, n, cu, rope=m.rope, max_new=most)
        m.cache.append(k, v, table, n, cu, rope=m.rope)
    assert m.cache.status() == 0


def test_what_a_captured_step_found_is_told_when_the_workspace_has_grown():
    m, q, k, v, table, n, cu = a_step(6)
    parent = i32(list(range(-1, 19)) * 2)
    step = lambda: (m.cache.attend(q, k, v, table, n, cu, parent=parent, rope=m.rope, max_new=20), m.cache.append(k, v, table, n, cu, rope=m.rope))
    step()
    assert m.cache.status() == 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    small = m.cache.ws
    big, big_cu = 500000, i32([0, 500000, 500000])          # (more tokens than a sequence may have: told, and nothing else done)
    x = torch.zeros(2, 1, 64, dtype=torch.bfloat16, device="cuda").expand(-1, big, -1)
    m.cache.append(x, x, table, n, big_cu, rope=m.rope)
    assert m.cache.ws is not small and m.cache.status() == 1 and m.cache.status() == 0
    graph.replay()
    assert m.cache.status() == 0
    parent[3] = 7
    graph.replay()
    parent[3] = 2
    for _ in range(3):
        graph.replay()                                      # ... and right again
        step()
    assert m.cache.status() == 1 and m.cache.status() == 0
    graph.replay()
    assert m.cache.status() == 0


def test_calls_of_two_threads_with_windows_of_different_lengths():
    """Kernels that take shared memory by the length of a window, called side by side: appends of two caches, selections, decodes."""
    import threading
    failed, work = [], []
    gate = threading.Barrier(2)
    for lag, group in ((9000, 32), (2100, 10)):
        p = lrsa.Params(1, 2 * group, 2, 4 * lag, 64, lag, lag // 4, 4)
        cache = lrsa.PagedCache(p, 2 * (-(-4 * lag // 128) + 8), page=128)
        table = torch.arange(cache.table_width, dtype=torch.int32, device="cuda")[None]
        k, v = (torch.randn(2, 3 * lag + 10, 64, generator=torch.Generator().manual_seed(lag)).bfloat16().cuda() for _ in "kv")
        some = lrsa.Params(1, 2 * group, 2, 1000, 64, 256, 64, 4)
        kv = lrsa.KVCache(some)
        x = k[None, :, :900].contiguous()
        kv.append(x, x)
        sel = lrsa.Params(1, 2 * group, 2, 3 * lag + 10, 64, lag, lag // 4, 4)
        q = torch.randn(1, 2 * group, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
        work.append((cache, k, v, table, i32([0]), i32([0, 3 * lag + 10]), kv, q, sel))

    def run(i):
        cache, k, v, table, n, cu, kv, q, sel = work[i]
        stream = torch.cuda.Stream()
        try:
            with torch.cuda.stream(stream):
                out = []
                gate.wait()
                for _ in range(200):
                    cache.append(k, v, table, n, cu)
                    idx, _ = lrsa.lrsa_score_select(sel, k[None], v[None])
                    out.append((idx, kv.decode(q)[0]))
            stream.synchronize()
            for idx, o in out[1:]:
                assert torch.equal(idx, out[0][0]) and torch.equal(o, out[0][1])
            assert cache.status(stream) == 0
        except Exception as e:
            failed.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed


@pytest.mark.parametrize("new", [2, 20])
def test_outputs_beside_the_inputs_in_one_buffer(new):
    """Rows that take turns with those of q, k and v, and o in other orders."""
    p = lrsa.Params(1, 8, 2, 900, 64, 64, 16, 4)
    m = Model(p, 16, 2, dim=64, seed=7)
    m.append([300, 40])
    table, n, cu = m.device([new, new])
    T = 2 * new
    q, k, v = (m.rows(h, T, False).cuda() for h in (8, 2, 2))
    want, _ = m.cache.attend(q, k, v, table, n, cu, rope=m.rope, max_new=new)
    fused = torch.zeros(T, 20 + 4, 64, dtype=torch.bfloat16, device="cuda")
    parts = [fused[:, a:b].transpose(0, 1) for a, b in ((0, 8), (8, 10), (10, 12), (12, 20))]
    for x, y in zip(parts, (q, k, v)):
        x.copy_(y)
    kept = fused.clone()
    o, _ = m.cache.attend(*parts[:3], table, n, cu, rope=m.rope, max_new=new, o=parts[3])
    assert torch.equal(o, want) and o.data_ptr() == parts[3].data_ptr()
    assert torch.equal(fused[:, :12], kept[:, :12]) and torch.equal(fused[:, 20:], kept[:, 20:])
    by_head = torch.zeros(8, T + 3, 3 * 64, dtype=torch.bfloat16, device="cuda")
    by_head[:, :T, 64:128] = q
    o, _ = m.cache.attend(by_head[:, :T, 64:128], k, v, table, n, cu, rope=m.rope, max_new=new, o=by_head[:, :T, 128:])
    assert torch.equal(o, want) and (by_head[:, T:] == 0).all() and (by_head[:, :, :64] == 0).all()
    back = torch.zeros(2 * T, 8, 64, dtype=torch.bfloat16, device="cuda")
    o, _ = m.cache.attend(q, k, v, table, n, cu, rope=m.rope, max_new=new, o=back[::2].transpose(0, 1))
    assert torch.equal(o, want) and (back[1::2] == 0).all()
    for bad in (q, by_head[:, :T, 64:128]):
        with pytest.raises(lrsa.LrsaError):
            m.cache.attend(bad, k, v, table, n, cu, rope=m.rope, max_new=new, o=bad)


def test_drafts_beyond_the_end_of_a_chunk_are_cut_on_the_device():
    """A captured step of drafts, of which as many are accepted as there is room for: tokens and pages are those of single steps."""
    p = lrsa.Params(1, 4, 2, 600, 64, 32, 8, 4)
    tokens, new = [4 + 2 * 32 - 3, 40], 7
    a, b, table = twins(p, 16, tokens, [500, 500], dim=64)
    q, k, v = (a.rows(h, 2 * new, False).cuda() for h in (4, 2, 2))
    n, nb, cu, slots = i32(tokens), i32(tokens), i32([0, new, 2 * new]), torch.arange(2 * new, dtype=torch.int32, device="cuda")
    a.cache.attend(q, k, v, table, n, cu, rope=a.rope, max_new=new)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = a.cache.attend(q, k, v, table, n, cu, rope=a.rope, max_new=new)
        taken = torch.minimum(cu.diff(), a.cache.room(n))
        cu_kept = torch.cat([taken.new_zeros(1), taken.cumsum(0, dtype=torch.int32)])
        s = (torch.searchsorted(cu_kept, slots, right=True) - 1).clamp(max=1)
        a.cache.append(k, v, table, n, cu_kept, rows=(cu[s] + slots - cu_kept[s]).clamp(max=2 * new - 1), rope=a.rope)
        n += taken
    capped = 0
    for i in range(14):
        for x, h in ((q, 4), (k, 2), (v, 2)):
            x.copy_(a.rows(h, 2 * new, False))
        graph.replay()
        most = taken.tolist()
        capped += sum(x < new for x in most)
        for j in range(max(most)):
            rows = [s * new + j for s in range(2) if j < most[s]]
            one = i32([0, 1 if j < most[0] else 0, len(rows)])
            args = [x[:, rows].contiguous() for x in (q, k, v)]
            want, want_lse = b.cache.attend(*args, table, nb, one, rope=b.rope, max_new=1)
            # A draft sees the drafts in front of it with keys of two bf16, a single token has them from the cache, rounded to one: half a step of
            # every channel, so at most 2^-8 |q| |k| / sqrt(d) of a score.  lse moves by no more than a score does, a probability by a factor of
            # exp(2 of that) at most.  And both sides round the probabilities and the sum, of values below 5.
            ds = ref.HALF_STEP * float(q.float().norm(dim=-1).max() * k.float().norm(dim=-1).max()) / 8
            assert (o[:, rows].float() - want.float()).abs().max() <= 4 * 5 * ref.HALF_STEP + 5 * (np.exp(2 * ds) - 1)
            assert (lse[:, rows] - want_lse).abs().max() <= ds + 1e-4, (i, j)
            b.cache.append(*args[1:], table, nb, one, rope=b.rope)
            nb += one.diff()
        assert torch.equal(n, nb) and a.cache.status() == 0 and b.cache.status() == 0
    assert capped > 3 and same_pages(a, b)


def test_layers_that_share_a_workspace():
    """The layers of a model, one step after the other, captured and not: each has what it has alone."""
    ps = [lrsa.Params(1, 8, 2, 900, 64, 64, 16, 4), lrsa.Params(1, 14, 2, 900, 128, 64, 16, 4), lrsa.Params(1, 8, 2, 900, 64, 64, 16, 4)]
    ms = [Model(p, 16, 2, dim=64, seed=8) for p in ps]
    shared = [lrsa.PagedCache(p, m.cache.n_pages, page=16, beside=None) for p, m in zip(ps[:1], ms)]
    shared += [lrsa.PagedCache(p, m.cache.n_pages, page=16, beside=shared[0]) for p, m in zip(ps[1:], ms[1:])]
    steps = []
    for m, cache in zip(ms, shared):
        m.append([400, 77])
        for s in range(2):
            m.reach(s, m.n[s] + 40)
        cache.k_pages, cache.v_pages = m.cache.k_pages.clone(), m.cache.v_pages.clone()
        p = m.p
        q, k, v = (m.rows(h, 40, False).cuda() for h in (p.n_q_heads, 2, 2))
        steps.append((q, k, v, i32(m.table.tolist()), i32(m.n), i32([0, 30, 40])))
    def run(caches):
        out = []
        for m, cache, (q, k, v, table, n, cu) in zip(ms, caches, steps):
            out.append(cache.attend(q, k, v, table, n, cu, rope=m.rope, max_new=30))
            cache.append(k, v, table, n, cu, rope=m.rope)
        return out
    want = run([m.cache for m in ms])
    got = run(shared)
    assert len({c.ws.data_ptr() for c in shared}) == 1
    for (o, lse), (x, y), m, cache in zip(want, got, ms, shared):
        assert torch.equal(o, x) and torch.equal(lse, y) and torch.equal(m.cache.k_pages.view(torch.int16), cache.k_pages.view(torch.int16))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = run(shared)
    for _ in range(3):
        graph.replay()
        assert all(torch.equal(x, z) and torch.equal(y, w) for (x, y), (z, w) in zip(got, again))
    steps[1][4].fill_(-1)
    graph.replay()
    assert [c.status() for c in shared] == [1, 0, 0]      # told once, by whichever is asked


@pytest.mark.parametrize("new, launches", [([1] * 16, 1), ([5] * 15 + [90], 1), ([300] + [1] * 15, 3), ([1] * 15 + [600], 3), ([0, 2] * 7 + [0, 250], 3)])
def test_prompts_beside_the_tokens_of_other_sequences(new, launches):
    """Where one sequence may have many windows to cut, they are cut side by side."""
    m = Model(lrsa.Params(1, 8, 2, 2500, 64, 64, 16, 4), 16, 16, dim=64, seed=9)
    m.append([int(x) for x in m.rng.integers(0, 500, 16)])
    m.append(new)
    for s in range(16):
        m.reach(s, m.n[s] + max(new))
    table, n, cu = m.device(new)
    k, v = (m.rows(2, sum(new), False).cuda() for _ in "kv")
    m.check_pages()
    m.cache.append(k, v, table, n, cu, rope=m.rope)
    assert lrsa.lrsa_last_launch_count() == launches and m.cache.status() == 0


@pytest.mark.parametrize("heads, d, new", [((8, 8), 64, 1), ((14, 2), 128, 1), ((8, 1), 64, 2), ((8, 2), 128, 4)], ids=["mha", "gqa7", "rows16", "drafts"])
@pytest.mark.parametrize("rope", [0, 64])
def test_up_to_sixteen_rows_lose_nothing_but_the_rounding_of_o(heads, d, new, rope):
    """Probabilities enter as sums of two bf16: what is left out of them, half a step of the second part (2^-7 of the first, so 2^-7 2^-8 of a
    term), the least that the second part is (2^-40), the scores' and the sums' rounding (the bounds that ref.attend gives for lse, which moves a
    probability by a factor), and one rounding of o."""
    p = lrsa.Params(1, *heads, 3000, d, 256, 64, 4)
    m = Model(p, 32, 3, dim=rope, seed=10)
    m.append([2500, 40, 700])
    sizes = [new] * 3
    q, k, v = (m.rows(h, 3 * new, False) for h in (heads[0], heads[1], heads[1]))
    table, n, cu = m.device(sizes)
    o, _ = m.cache.attend(q.cuda(), k.cuda(), v.cuda(), table, n, cu, rope=m.rope, max_new=new)
    for s in range(3):
        part = slice(s * new, (s + 1) * new)
        n_s, w = m.n[s], ref.cut(p, m.n[s])
        sees = ref.ancestors(None, new)
        pos = n_s + np.arange(new)
        qs, ks, vs = m.turned(f64(q)[:, part], pos, False), m.turned(f64(k)[:, part], pos, False), f64(v)[:, part]
        idx = m.selected(s)
        keys, vals = [], []
        for h in range(heads[1]):
            seen = np.concatenate([np.arange(min(n_s, p.n_sink)), idx[h].ravel(), np.arange(min(n_s, p.n_sink + w * p.lag), n_s)]).astype(int)
            keys.append(np.concatenate([m.K[s][h, seen], ks[h]]))
            vals.append(np.concatenate([m.V[s][h, seen], vs[h]]))
        sees = np.concatenate([np.ones((new, keys[0].shape[0] - new), bool), sees], 1)
        args = qs, np.stack(keys), sees, 1 / math.sqrt(d)
        want, _, _, lse_tol = ref.attend(args[0], args[1], np.stack(vals), *args[2:], rotated=rope > 0)
        terms = ref.attend(args[0], args[1], np.abs(np.stack(vals)), *args[2:], rotated=rope > 0)[0]
        tol = (2.0 ** -15 + 2.0 ** -39 + 2 * lse_tol[..., None] + 2.0 ** -18) * terms
        err = np.abs(f64(o)[:, part] - want)
        assert (err <= tol + ref.HALF_STEP * (np.abs(want) + tol)).all(), (s, float((err / (tol + ref.HALF_STEP * np.abs(want))).max()))
