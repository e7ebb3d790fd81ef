"""lrsa_rotate on the GPU against the formula: every bit of a rounded row, the formula in 64 bits, its gradient."""
import numpy as np
import pytest
import torch

from paper_2506_11498_b200 import lrsa
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu


def rows(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).bfloat16()


def f64(t):
    return t.double().cpu().numpy()


SHAPES = [   # B, Hq, Hkv, N, d, dim
    (1, 1, 1, 1, 64, 64), (1, 8, 8, 77, 64, 32), (2, 4, 2, 333, 64, 16), (1, 28, 4, 130, 128, 128), (3, 5, 1, 65, 128, 64),
    (1, 7, 7, 33, 128, 96), (1, 2, 2, 31, 128, 48), (1, 2, 1, 4097, 128, 16), (33, 3, 3, 5, 64, 48), (1, 140, 2, 9, 128, 112),
]


@pytest.mark.parametrize("B,Hq,Hkv,N,d,dim", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("inverse", [False, True], ids=["forward", "gradient"])
def test_every_bit_and_the_formula(B, Hq, Hkv, N, d, dim, interleaved, inverse):
    p = lrsa.Params(B, Hq, Hkv, N, d, 16, 4, 0)
    cos, sin = ref.angles(N + 3, dim)
    rope = lrsa.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), interleaved)
    Q, K = rows(1, B, Hq, N, d), rows(2, B, Hkv, N, d)
    got = lrsa.lrsa_rotate(p, Q.cuda(), K.cuda(), rope, inverse=inverse)
    for x, y in zip((Q, K), got):
        want = ref.rotate(f64(x), np.arange(N), cos, sin, interleaved, inverse)
        assert np.array_equal(f64(y), want)
        exact = ref.rotate(f64(x), np.arange(N), cos, sin, interleaved, inverse, rounded=False)
        # one rounding to bf16, two in 32 bits of terms that may cancel
        most = np.abs(f64(x)).max(-1, keepdims=True)
        assert (np.abs(f64(y) - exact) <= ref.HALF_STEP * np.abs(exact) + 2.0 ** -22 * most).all()
    only_k = lrsa.lrsa_rotate(p, None, K.cuda(), rope, inverse=inverse)
    assert only_k[0] is None and torch.equal(only_k[1], got[1])


@pytest.mark.parametrize("n_seqs", [1, 3, 700])
def test_positions_of_packed_rows_and_given_ones(n_seqs):
    rng = np.random.default_rng(3)
    N = 2100
    cuts = [0] + sorted(rng.choice(np.arange(1, N), n_seqs - 1, replace=False).tolist()) + [N]
    pos = np.concatenate([np.arange(b - a) for a, b in zip(cuts, cuts[1:])])
    cos, sin = ref.angles(int(pos.max()) + 1, 64)
    rope = lrsa.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    Q, K = rows(4, 1, 4, N, 64), rows(5, 1, 2, N, 64)
    packed = lrsa.Params(1, 4, 2, N, 64, 16, 4, 0, cu_seqlens=tuple(cuts))
    a = lrsa.lrsa_rotate(packed, Q.cuda(), K.cuda(), rope)
    b = lrsa.lrsa_rotate(lrsa.Params(1, 4, 2, N, 64, 16, 4, 0), Q.cuda(), K.cuda(), rope,
                         positions=torch.from_numpy(pos).int().cuda())
    for x, y, z in zip((Q, K), a, b):
        assert torch.equal(y, z)
        assert np.array_equal(f64(y), ref.rotate(f64(x), pos, cos, sin))


def test_in_place_and_back():
    p = lrsa.Params(1, 28, 4, 700, 128, 16, 4, 0)
    rope = lrsa.Rope.of_base(10000.0, 128, 700)
    Q, K = rows(6, 1, 28, 700, 128).cuda(), rows(7, 1, 4, 700, 128).cuda()
    q, k = lrsa.lrsa_rotate(p, Q, K, rope)
    x, y = Q.clone(), K.clone()
    assert lrsa.lrsa_rotate(p, x, y, rope, Q_out=x, K_out=y) == (x, y)
    assert torch.equal(x, q) and torch.equal(y, k)
    back, _ = lrsa.lrsa_rotate(p, q, None, rope, inverse=True)
    # two roundings of a pair, each at most half a step of a value that is at most the pair's length
    length = torch.hypot(*Q.double().chunk(2, -1)).repeat(1, 1, 1, 2)
    assert ((back.double() - Q.double()).abs() <= 2.9 * ref.HALF_STEP * length + 1e-30).all()


def test_gradient_by_differences():
    """<dy, R x'> - <dy, R x> along a direction equals <R^T dy, x' - x>: R^T is what inverse computes."""
    p = lrsa.Params(1, 2, 1, 50, 64, 16, 4, 0)
    cos, sin = ref.angles(50, 64)
    rope = lrsa.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), True)
    x, dy, step = rows(8, 1, 2, 50, 64), rows(9, 1, 2, 50, 64), rows(10, 1, 2, 50, 64)
    grad, _ = lrsa.lrsa_rotate(p, dy.cuda(), None, rope, inverse=True)
    turn = lambda t: ref.rotate(f64(t), np.arange(50), cos, sin, True, rounded=False)
    diff = (f64(dy) * (ref.rotate(f64(x) + f64(step), np.arange(50), cos, sin, True, rounded=False) - turn(x))).sum()
    mine = (f64(grad) * f64(step)).sum()
    # each element of the gradient is rounded once
    assert abs(diff - mine) <= (ref.HALF_STEP * np.abs(f64(grad) * f64(step))).sum() + 1e-4


def test_positions_out_of_range_are_nan_where_rotated():
    p = lrsa.Params(1, 2, 1, 4, 64, 16, 4, 0)
    rope = lrsa.Rope.of_base(10000.0, 32, 10)
    Q = rows(11, 1, 2, 4, 64).cuda()
    q, _ = lrsa.lrsa_rotate(p, Q, None, rope, positions=torch.tensor([0, -1, 10, 9], dtype=torch.int32, device="cuda"))
    assert torch.isnan(q[:, :, 1:3, :32]).all() and not torch.isnan(q[:, :, [0, 3]]).any()
    assert torch.equal(q[..., 32:], Q[..., 32:]) and torch.equal(q[:, :, 0], Q[:, :, 0])


def test_values_that_are_not_finite_stay_in_their_pair():
    p = lrsa.Params(1, 1, 1, 3, 64, 16, 4, 0)
    rope = lrsa.Rope.of_base(10000.0, 64, 3)
    Q = rows(12, 1, 1, 3, 64)
    Q[0, 0, 1, 5], Q[0, 0, 2, 40] = float("inf"), float("nan")
    q, _ = lrsa.lrsa_rotate(p, Q.cuda(), None, rope)
    bad = ~torch.isfinite(q.cpu())[0, 0]
    want = torch.zeros(3, 64, dtype=torch.bool)
    want[1, [5, 37]] = want[2, [8, 40]] = True
    assert torch.equal(bad, want)


def test_on_a_stream_and_captured():
    p = lrsa.Params(1, 8, 8, 300, 64, 16, 4, 0)
    rope = lrsa.Rope.of_base(10000.0, 64, 300)
    Q, K = rows(13, 1, 8, 300, 64).cuda(), rows(14, 1, 8, 300, 64).cuda()
    want = lrsa.lrsa_rotate(p, Q, K, rope)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lrsa.lrsa_rotate(p, Q, K, rope, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    x = Q.clone()
    with torch.cuda.graph(graph):
        y, _ = lrsa.lrsa_rotate(p, x, None, rope)
    x.copy_(Q * 2)
    graph.replay()
    assert torch.equal(y, lrsa.lrsa_rotate(p, Q * 2, None, rope)[0])
