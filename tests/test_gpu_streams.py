"""Calls with `stream=`: what they make for themselves and what they return is memory of that stream."""
import pytest
import torch

from paper_2506_11498_b200 import lrsa

pytestmark = pytest.mark.gpu

P = lrsa.Params(1, 4, 2, 1200, 128, 256, 64, 4)
BUSY = 100_000_000      # cycles that keep a stream at work while the host goes on: about 50 ms


def calls():
    """name -> a call on a stream that makes its own workspace and results."""
    g = torch.Generator().manual_seed(3)
    Q, dO = (torch.randn(1, 4, 1200, 128, generator=g).bfloat16().cuda() for _ in "ab")
    K, V = (torch.randn(1, 2, 1200, 128, generator=g).bfloat16().cuda() for _ in "kv")
    q = Q[:, :, -1].contiguous()
    idx, _ = lrsa.lrsa_score_select(P, K, V)
    O, LSE = lrsa.lrsa_attn_fwd(P, Q, K, V, idx)
    w = lrsa.lrsa_attn_weights(P, Q, K, LSE)
    cache, store = lrsa.KVCache(P), lrsa.KVStore(P, block=32)
    cache.append(K, V)
    store.append(K, V, w)

    return {
        "score_select": lambda s: lrsa.lrsa_score_select(P, K, V, want_score=True, stream=s),
        "attn_fwd": lambda s: lrsa.lrsa_attn_fwd(P, Q, K, V, idx, stream=s),
        "attn_bwd": lambda s: lrsa.lrsa_attn_bwd(P, Q, K, V, O, dO, LSE, idx, stream=s)[1:],   # (dQ is added up in no fixed order)
        "attn_weights": lambda s: (lrsa.lrsa_attn_weights(P, Q, K, LSE, stream=s),),
        "weight_select": lambda s: (lrsa.lrsa_weight_select(P, w, stream=s),),
        "cache_decode": lambda s: cache.decode(q, stream=s),
        "store_decode": lambda s: store.decode(q, stream=s),
        "store_rows": lambda s: store.rows(stream=s),
    }


NAMES = ("score_select", "attn_fwd", "attn_bwd", "attn_weights", "weight_select", "cache_decode", "store_decode", "store_rows")


@pytest.mark.parametrize("name", NAMES)
def test_a_call_ahead_of_its_stream(name):
    """The call waits on a busy stream while the current one asks for memory of the sizes that it may have dropped."""
    call = calls()[name]
    want = [x.clone() for x in call(None)]
    sizes = sorted({256, 512} | {lrsa.new_workspace(n).numel() for n in lrsa.lrsa_workspace_bytes(P)})
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BUSY)
    got = call(s)
    mine = [torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(8)]
    torch.cuda.synchronize()
    assert all((x == 0x5a).all() for x in mine)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("name", NAMES)
def test_a_call_beside_a_busy_current_stream(name):
    """Blocks that the current stream has dropped, but not yet written to, are not what the call on another stream returns."""
    call = calls()[name]
    want = [x.clone() for x in call(None)]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    blocks = [torch.empty_like(x) for x in want for _ in range(4)] + \
             [lrsa.new_workspace(n) for n in lrsa.lrsa_workspace_bytes(P) + (256,) for _ in range(4)]
    torch.cuda._sleep(BUSY)
    for x in blocks:
        x.fill_(7)
    del blocks, x
    got = [x.clone() for x in on(s, call)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def on(s, call):
    """The call's results, when the current stream has waited for `s`."""
    got = call(s)
    torch.cuda.current_stream().wait_stream(s)
    return got


@pytest.mark.parametrize("name", NAMES)
def test_results_that_are_dropped_early(name):
    """Results are read on the current stream and dropped; the next call on the side stream leaves them whole."""
    call = calls()[name]
    want = [x.clone() for x in call(None)]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = on(s, call)
    torch.cuda._sleep(BUSY)
    kept = [x.clone() for x in got]      # read when the current stream has slept
    shapes = [(x.shape, x.dtype) for x in got]
    del got
    with torch.cuda.stream(s):
        for _ in range(4):
            again = [torch.empty(shape, dtype=dtype, device="cuda").fill_(1) for shape, dtype in shapes]
    torch.cuda.synchronize()
    del again
    assert all(torch.equal(x, y) for x, y in zip(kept, want))


def test_streams_of_another_library():
    """Anything with a `cuda_stream` is a stream."""
    call = calls()["attn_weights"]
    want = call(None)[0]
    s = torch.cuda.Stream()
    other = type("S", (), {"cuda_stream": s.cuda_stream})
    torch.cuda.synchronize()
    got = call(other)[0]
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("name", NAMES)
def test_a_side_stream_in_a_graph(name):
    """Captured on a stream that joins the capture and leaves it again, replayed twice."""
    call = calls()[name]
    want = [x.clone() for x in call(None)]
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.wait_stream(torch.cuda.current_stream())
        got = on(s, call)
        kept = [x.clone() for x in got]
    for _ in range(2):
        for x in kept:
            x.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(kept, want))
