"""The paged cache on the GPU where weights underflow, numbers on the device cannot be used, and steps are captured."""
import numpy as np
import pytest
import torch

from paper_2506_11498_b200 import lrsa
from tests import paged_reference as ref
from tests.test_gpu_paged import Model, i32

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
