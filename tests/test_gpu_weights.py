"""Accumulated attention weights of a prompt and the selection by them, against fp64."""
import pytest
import torch

from paper_2506_11498_b200 import lrsa
from tests import store_reference as ref

pytestmark = pytest.mark.gpu

P = lrsa.Params
#        batch Hq Hkv  N   d    L    K   S
CASES = [
    (P(1, 1, 1, 1, 64, 64, 16, 0), ()),                       # one token
    (P(1, 2, 1, 5, 128, 64, 16, 5), ()),                      # nothing but sinks
    (P(1, 2, 2, 130, 64, 64, 16, 129), ()),                   # one token behind many sinks
    (P(2, 4, 2, 100, 128, 128, 32, 4), ()),                   # shorter than a window
    (P(1, 7, 1, 4 + 3 * 128, 128, 128, 32, 4), ()),           # whole windows, tiles of 128 keys
    (P(2, 8, 8, 16 + 5 * 64 + 9, 64, 64, 16, 16), ()),        # windows shorter than a tile
    (P(1, 20, 1, 3 + 2 * 333 + 200, 128, 333, 83, 3), ()),    # odd windows, a large group
    (P(1, 4, 1, 900, 64, 100, 10, 0, n_dense_prev=0), ()),    # the previous window compressed too
    (P(1, 2, 1, 4 + 4 * 200, 128, 200, 50, 4, n_dense_prev=0), ()),
    (P(1, 4, 4, 1500, 64, 512, 128, 16, softmax_scale=0.3), ()),
    (P(1, 4, 2, 1000, 128, 128, 32, 4, cu_seqlens=(0, 1, 3, 400, 401, 1000)), (0, 1, 3, 400, 401, 1000)),
    (P(2, 2, 1, 800, 64, 64, 16, 7, cu_seqlens=tuple(range(0, 801, 40))), tuple(range(0, 801, 40))),   # 20 sequences: two launches
]


def inputs(p, seed=0, offset=2.0):
    g = torch.Generator().manual_seed(seed)
    Q = torch.randn(p.batch, p.n_q_heads, p.seq_len, p.head_dim, generator=g).bfloat16()
    K = (torch.randn(p.batch, p.n_kv_heads, p.seq_len, p.head_dim, generator=g)
         + offset * torch.randn(1, p.n_kv_heads, 1, p.head_dim, generator=g)).bfloat16()
    V = torch.randn(K.shape, generator=g).bfloat16()
    return Q, K, V


def forward_lse(p, Q, K, V):
    idx, _ = lrsa.lrsa_score_select(p, K, V)
    return lrsa.lrsa_attn_fwd(p, Q, K, V, idx)[1]


@pytest.mark.parametrize("p,cu", CASES, ids=lambda x: f"{x.n_q_heads}_{x.n_kv_heads}_d{x.head_dim}_{x.seq_len}_L{x.lag}" if isinstance(x, P) else "")
def test_weights(p, cu):
    Q, K, V = inputs(p)
    d = [x.cuda() for x in (Q, K, V)]
    lse = forward_lse(p, *d)
    ws = lrsa.new_workspace(256)
    out = torch.full((p.batch, p.n_kv_heads, p.seq_len), -7.0, device="cuda")
    got = lrsa.lrsa_attn_weights(p, d[0], d[1], lse, weight=out, workspace=ws)
    assert got is out and lrsa.lrsa_workspace_status(ws) == 0
    want, tol = ref.weights(p, Q, K, lse.cpu(), cu or None)
    ref.within("weight", got, want, tol)
    again = lrsa.lrsa_attn_weights(p, d[0], d[1], lse)
    assert torch.equal(got, again)          # no order of additions is left to chance


def test_weights_sum_to_the_queries():
    """Without compressed windows every query spends its whole weight on the positions: heads * queries in all (S = 0)."""
    p = P(1, 6, 2, 700, 128, 512, 64, 0)
    d = [x.cuda() for x in inputs(p)]
    w = lrsa.lrsa_attn_weights(p, d[0], d[1], forward_lse(p, *d))
    total = w.double().sum(-1).cpu()
    assert ((total - 3 * 700).abs() <= 3 * 700 * 1e-5).all()


def test_hidden_values_do_not_enter():
    """NaN and infinity in another sequence of the row, and in queries and keys that do not see one another."""
    cu = (0, 300, 500, 777)
    p = P(1, 4, 2, 777, 128, 64, 16, 4, cu_seqlens=cu)
    Q, K, V = inputs(p, 3)
    lse = forward_lse(p, *(x.cuda() for x in (Q, K, V))).cpu()
    want = lrsa.lrsa_attn_weights(p, Q.cuda(), K.cuda(), lse.cuda()).cpu()
    for bad in (float("nan"), float("inf")):
        q, k, e = Q.clone(), K.clone(), lse.clone()
        q[:, :, 300:500] = bad
        k[:, :, 300:500] = bad
        e[:, :, 300:500] = bad
        got = lrsa.lrsa_attn_weights(p, q.cuda(), k.cuda(), e.cuda()).cpu()
        assert torch.equal(got[:, :, :300], want[:, :, :300]) and torch.equal(got[:, :, 500:], want[:, :, 500:])
    q, k, e = Q.clone(), K.clone(), lse.clone()
    q[:, :, 100] = float("nan")       # spoils the positions that query 100 sees (its window is 1: windows 0 and 1 up to itself)
    e[:, :, 100] = float("nan")
    k[:, :, 260] = float("inf")       # spoils its own position only
    got = lrsa.lrsa_attn_weights(p, q.cuda(), k.cuda(), e.cuda()).cpu()
    same = torch.ones(777, dtype=torch.bool)
    same[4:101] = False
    same[260] = False
    assert torch.equal(got[:, :, same], want[:, :, same])
    assert got[:, :, 4:101].isnan().all()


def test_weights_on_a_stream_and_in_a_graph():
    p = P(1, 4, 2, 1200, 64, 256, 64, 4)
    first, second = ([x.cuda() for x in inputs(p, s)] for s in (1, 2))
    lses = [forward_lse(p, *x) for x in (first, second)]
    want = [lrsa.lrsa_weight_select(p, lrsa.lrsa_attn_weights(p, x[0], x[1], e)) for x, e in zip((first, second), lses)]
    q, k, e = first[0].clone(), first[1].clone(), lses[0].clone()
    w = torch.empty(1, 2, 1200, device="cuda")
    idx, ws = torch.empty_like(want[0]), lrsa.new_workspace(256)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        lrsa.lrsa_attn_weights(p, q, k, e, weight=w, workspace=ws)
        lrsa.lrsa_weight_select(p, w, idx=idx)
    s.synchronize()
    assert torch.equal(idx, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lrsa.lrsa_attn_weights(p, q, k, e, weight=w, workspace=ws)
        lrsa.lrsa_weight_select(p, w, idx=idx)
    for x, l, i in ((second, lses[1], want[1]), (first, lses[0], want[0])):
        q.copy_(x[0]); k.copy_(x[1]); e.copy_(l)
        idx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(idx, i)


@pytest.mark.parametrize("L,K,S,N,B,H", [(64, 16, 4, 1000, 2, 3), (1, 1, 0, 77, 1, 2), (64, 64, 3, 500, 1, 1), (333, 83, 0, 2000, 2, 1),
                                         (4096, 1024, 4, 13000, 1, 2), (20011, 3, 1, 60100, 1, 1), (32767, 16000, 0, 2 * 32767, 1, 1)])
def test_select(L, K, S, N, B, H):
    p = P(B, H, H, N, 64, L, K, S)
    g = torch.Generator().manual_seed(L)
    cases = [torch.empty(B, H, N).log_normal_(0, 3, generator=g), torch.randn(B, H, N, generator=g),
             torch.randint(0, 3, (B, H, N), generator=g).float(), torch.zeros(B, H, N),
             torch.rand(B, H, N, generator=g) * 2.0 ** -140,                       # subnormal
             (1 + torch.randint(0, 40, (B, H, N), generator=g) * 2.0 ** -23)]      # keys that differ in their last bits
    odd = torch.randn(B, H, N, generator=g)
    odd[torch.rand(odd.shape, generator=g) < 0.4] = float("nan")
    odd[torch.rand(odd.shape, generator=g) < 0.2] = float("inf")
    odd[torch.rand(odd.shape, generator=g) < 0.2] = -float("inf")
    odd[torch.rand(odd.shape, generator=g) < 0.2] = 0.0
    odd[torch.rand(odd.shape, generator=g) < 0.2] = -0.0
    for w in cases + [odd]:
        assert torch.equal(lrsa.lrsa_weight_select(p, w.cuda()).cpu(), ref.select(p, w))


def test_select_packed():
    cu = (0, 3, 400, 401, 1000) + tuple(range(1100, 3001, 100))
    p = P(2, 4, 2, 3000, 64, 30, 7, 5, cu_seqlens=cu)
    w = torch.rand(2, 2, 3000, generator=torch.Generator().manual_seed(1))
    assert torch.equal(lrsa.lrsa_weight_select(p, w.cuda()).cpu(), ref.select(p, w, cu))


def test_selection_by_weight_in_a_training_step():
    """Forward, weights, selection by them, forward and backward on that selection: finite, and the mask is the new one."""
    p = P(1, 4, 2, 4 + 6 * 128 + 50, 128, 128, 32, 4)
    Q, K, V = (x.cuda() for x in inputs(p, 5))
    idx, _ = lrsa.lrsa_score_select(p, K, V)
    w = lrsa.lrsa_attn_weights(p, Q, K, lrsa.lrsa_attn_fwd(p, Q, K, V, idx)[1])
    mine = lrsa.lrsa_weight_select(p, w)
    O, LSE = lrsa.lrsa_attn_fwd(p, Q, K, V, mine)
    grads = lrsa.lrsa_attn_bwd(p, Q, K, V, O, torch.randn_like(O), LSE, mine)
    assert all(torch.isfinite(x.float()).all() for x in (O, LSE) + grads)
    # the last query's log-sum over sinks, the kept rows of windows 0 .. 4 and the uncompressed positions
    at = torch.cat([torch.arange(4), mine[0, 0, :5].flatten().long().cpu(), torch.arange(4 + 5 * 128, p.seq_len)])
    s = (Q[0, 0, -1].double().cpu() @ K[0, 0].double().cpu()[at].T) / 128 ** 0.5
    assert abs(float(LSE[0, 0, -1]) - float(torch.logsumexp(s, 0))) <= 1e-4


def test_refusals():
    p = P(1, 4, 2, 1000, 128, 128, 32, 4)
    Q, K, V = (x.cuda() for x in inputs(p))
    lse, w = torch.zeros(1, 4, 1000, device="cuda"), torch.zeros(1, 2, 1000, device="cuda")
    for bad in ((Q.float(), K, lse), (Q[:, :, :999], K, lse), (Q, K.transpose(1, 2), lse), (Q, K, lse.half()), (Q.cpu(), K, lse),
                (Q, V[:, :1], lse), (Q.transpose(2, 3).contiguous().transpose(2, 3), K, lse)):
        with pytest.raises(lrsa.LrsaError) as e:
            lrsa.lrsa_attn_weights(p, *bad)
        assert e.value.status == 1
    with pytest.raises(lrsa.LrsaError) as e:
        lrsa.lrsa_attn_weights(p, Q, K, lse, workspace=torch.empty(128, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3
    for bad in (w.double(), w[:, :, 1:], w[0], w.cpu()):
        with pytest.raises(lrsa.LrsaError) as e:
            lrsa.lrsa_weight_select(p, bad)
        assert e.value.status == 1
    with pytest.raises(lrsa.LrsaError) as e:
        lrsa.lrsa_weight_select(p, w, idx=torch.zeros(1, 2, 3, 32, dtype=torch.int32, device="cuda"))
    assert e.value.status == 1


@pytest.mark.parametrize("L,K", [(8, 5), (64, 50), (333, 300), (4096, 4000)])
def test_nan_ranks_below_minus_infinity(L, K):
    """More rows are kept than there are numbers: first every -infinity, wherever it stands, then the NaN of lowest position."""
    p = P(1, 2, 2, 3 + 3 * L + 1, 64, L, K, 3)
    g = torch.Generator().manual_seed(L)
    w = torch.rand(1, 2, p.seq_len, generator=g)
    kind = torch.rand(w.shape, generator=g)
    w[kind < 0.6] = float("nan")
    w[kind < 0.3] = -float("inf")
    w[0, 0, 3:3 + L] = float("nan")                   # nothing but NaN; then one -infinity behind all of them
    w[0, 1, 3:3 + L] = float("nan")
    w[0, 1, 3 + L - 1] = -float("inf")
    w.view(torch.int32)[0, 0, 3 + L:3 + 2 * L:2] |= -2 ** 31     # NaN of either sign
    got = lrsa.lrsa_weight_select(p, w.cuda()).cpu()
    store = lrsa.KVStore(p, block=16)
    x = torch.zeros(1, 2, p.seq_len, 64, dtype=torch.bfloat16, device="cuda")
    store.append(x, x, w.cuda())
    for h in range(2):
        for i in range(2):
            a = 3 + i * L
            part = w[0, h, a:a + L].tolist()
            order = sorted(range(L), key=lambda j: (part[j] != part[j], -part[j] if part[j] == part[j] else 0.0, j))
            want = torch.tensor(sorted(a + j for j in order[:K]), dtype=torch.int32)
            assert torch.equal(got[0, h, i], want)
            assert torch.equal(store.idx[0, h, i].cpu(), want)
