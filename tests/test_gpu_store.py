"""The store: rows kept by weight or by the lag score, in bf16 or 8 bits, and decode attention over them, against fp64."""
import math

import pytest
import torch

from paper_2506_11498_b200 import lrsa
from tests import store_reference as ref

pytestmark = pytest.mark.gpu

P = lrsa.Params
E4M3, INT8, BF16 = torch.float8_e4m3fn, torch.int8, torch.bfloat16


def tokens(p, seed, offset=2.0):
    g = torch.Generator().manual_seed(seed)
    K = (torch.randn(p.batch, p.n_kv_heads, p.seq_len, p.head_dim, generator=g)
         + offset * torch.randn(1, p.n_kv_heads, 1, p.head_dim, generator=g)).bfloat16()
    V = torch.randn(K.shape, generator=g).bfloat16()
    Q = torch.randn(p.batch, p.n_q_heads, p.seq_len, p.head_dim, generator=g).bfloat16()
    w = torch.empty(K.shape[:3]).log_normal_(0, 2, generator=g)
    return Q, K, V, w


def check_state(store, want):
    """Kept positions, kept rows and recent rows are exact."""
    p, c = store.params, want.idx.shape[2]
    assert store.windows_compressed() == c and store.status() == 0
    assert torch.equal(store.idx[:, :, :c].cpu().long(), want.idx)
    k, v = (x.double().cpu() for x in store.rows())
    for got, exact in ((k, want.k_rows), (v, want.v_rows)):
        assert torch.equal(got.nan_to_num(7e30), exact.nan_to_num(7e30))
    n, S, L = want.n, p.n_sink, p.lag
    at = torch.arange(min(S + c * L, n), n)
    for got, all_rows in ((store.k_recent, want.K), (store.v_recent, want.V)):
        got = got.double().cpu()
        assert torch.equal(got[:, :, :min(S, n)], all_rows[:, :, :min(S, n)])
        if len(at):
            assert torch.equal(got[:, :, S + (at - S) % (2 * L)], all_rows[:, :, at])
    return at


#        B Hq Hkv   N            d    L    K   S  type  block keep  steps
CASES = [
    (P(2, 4, 2, 4 + 5 * 128 + 77, 128, 128, 32, 4), E4M3, 16, "weight", (1, 1, 2, 37, 128, 300, 5, 1)),
    (P(1, 4, 4, 16 + 6 * 64, 64, 64, 16, 16), INT8, 16, "weight", (7, 64, 1, 129)),
    (P(1, 7, 1, 3 + 4 * 200 + 50, 128, 200, 50, 3), INT8, 64, "weight", (250, 1, 1, 199, 403)),       # K ends inside a block
    (P(1, 2, 2, 6 * 96, 64, 96, 24, 0), E4M3, 32, "lag", (96, 96, 1, 95, 200)),                      # no sinks
    (P(1, 4, 2, 4 + 7 * 128 + 3, 128, 128, 64, 4), E4M3, 64, "weight", (4 + 7 * 128 + 3,)),          # a prompt at once
    (P(1, 4, 2, 4 + 7 * 128 + 3, 128, 128, 77, 4), BF16, 32, "weight", (500, 300, 1)),
    (P(1, 20, 1, 4 + 3 * 128 + 50, 128, 128, 32, 4), INT8, 32, "weight", (200, 1, 150, 87)),         # more than 16 heads a group
    (P(2, 40, 1, 2 + 3 * 64 + 9, 64, 64, 16, 2), E4M3, 16, "weight", (100, 1, 1, 101)),
    (P(1, 9, 1, 2 + 5 * 40 + 9, 64, 40, 40, 2), BF16, 16, "lag", (33, 50, 1)),                       # every row kept
    (P(1, 16, 1, 5 + 5 * 33, 128, 33, 1, 5), E4M3, 128, "weight", (3, 31, 1)),                       # one row kept
    (P(1, 2, 1, 2 + 3 * 4608 + 100, 64, 4608, 100, 2), E4M3, 128, "lag", (5000, 4608, 1, 4000)),     # long windows
    (P(17, 2, 2, 4 + 4 * 64 + 9, 64, 64, 16, 4), INT8, 16, "weight", (1, 70, 64, 90)),               # many heads
]


@pytest.mark.parametrize("p,dtype,block,keep,steps", CASES, ids=[f"{i}_{str(c[1])[6:]}_{c[3]}" for i, c in enumerate(CASES)])
def test_growth_and_decode(p, dtype, block, keep, steps):
    Q, K, V, w = tokens(p, p.seq_len)
    dev = [x.cuda() for x in (Q, K, V, w)]
    store, want = lrsa.KVStore(p, dtype=dtype, block=block, keep=keep), ref.Store(p, dtype, block, keep)
    i = 0
    while store.n_tokens < p.seq_len:
        lo = store.n_tokens
        n = min(steps[i % len(steps)], p.seq_len - lo)
        i += 1
        enters = keep == "weight" and n > 1          # single tokens enter with no weight
        store.append(dev[1][:, :, lo:lo + n].contiguous(), dev[2][:, :, lo:lo + n].contiguous(),
                     dev[3][:, :, lo:lo + n].contiguous() if enters else None)
        if keep == "weight":
            # gathered weights are fp32 here and fp64 there: the reference selects by the same numbers, checked below
            c = store.windows_compressed()
            sel = store.idx[:, :, :c].cpu().long()
            for x in range(want.idx.shape[2], c):
                a = p.n_sink + x * p.lag
                if a + p.lag <= want.n:               # the window was in the ring: its weights were checked by the last decode
                    want.w[:, :, a:a + p.lag] = ring_weight(before, p, a, p.lag)
        want.append(K[:, :, lo:lo + n], V[:, :, lo:lo + n], w[:, :, lo:lo + n] if enters else None,
                    store.idx[:, :, :store.windows_compressed()].cpu())
        at = check_state(store, want)
        q = Q[:, :, lo + n - 1]
        if keep == "weight" and len(at):
            want.w[:, :, at] = ring_weight(store.weight, p, int(at[0]), len(at))
        o, lse = store.decode(q.cuda())
        assert store.status() == 0
        (eo, to), (el, tl), (eg, tg) = want.decode(q)
        ref.within(f"o at {lo + n}", o, eo, to)
        ref.within(f"lse at {lo + n}", lse, el, tl)
        if keep == "weight":
            if len(at):
                got = ring_weight(store.weight, p, int(at[0]), len(at))
                ref.within(f"weight at {lo + n}", got, want.w[:, :, at], tg + 2.0 ** -24 * want.w[:, :, at])
            before = store.weight.clone()
    if keep == "lag":
        idx, _ = lrsa.lrsa_score_select(p, dev[1], dev[2])
        c = store.windows_compressed()
        assert torch.equal(store.idx[:, :, :c], idx[:, :, :c])


def ring_weight(weight, p, first, n):
    """fp64 weights of positions first .. first + n - 1 out of a ring [B, Hkv, 2L]."""
    return weight.double().cpu()[:, :, (torch.arange(first, first + n) - p.n_sink) % (2 * p.lag)]


def test_a_prompt_and_its_answer():
    """The calls together, as they are used: forward of a prompt, weights, the prompt enters the store cut by them, then
    tokens are generated until two more windows have been cut by what decode gathered."""
    p = P(1, 8, 2, 4 + 7 * 128, 128, 128, 32, 4)
    n0 = 4 + 5 * 128 + 60
    Q, K, V, _ = tokens(p, 9)
    dev = [x.cuda() for x in (Q, K, V)]
    prompt = P(1, 8, 2, n0, 128, 128, 32, 4)
    q, k, v = (x[:, :, :n0].contiguous() for x in dev)
    idx, _ = lrsa.lrsa_score_select(prompt, k, v)
    w = lrsa.lrsa_attn_weights(prompt, q, k, lrsa.lrsa_attn_fwd(prompt, q, k, v, idx)[1])
    store, want = lrsa.KVStore(p, dtype=E4M3, block=32, keep="weight"), ref.Store(p, E4M3, 32, "weight")
    store.append(k, v, w)
    want.append(K[:, :, :n0], V[:, :, :n0], w.cpu())
    sel = lrsa.lrsa_weight_select(prompt, w)
    assert store.windows_compressed() == 4 and torch.equal(store.idx[:, :, :4], sel[:, :, :4])
    for t in range(n0, p.seq_len):
        cut = (t - 4) % 128 == 0
        if cut:                                        # the reference cuts by the weights that decode has gathered, in fp32
            lo = 4 + (want.idx.shape[2]) * 128
            want.w[:, :, lo:lo + 128] = ring_weight(store.weight, p, lo, 128)
        store.append(*(x[:, :, t:t + 1].contiguous() for x in dev[1:]))
        want.append(K[:, :, t:t + 1], V[:, :, t:t + 1])
        o, lse = store.decode(dev[0][:, :, t].contiguous())
        (eo, to), (el, tl), (_, tg) = want.decode(Q[:, :, t])
        if t % 17 == 0 or cut:
            ref.within(f"o at {t}", o, eo, to)
            ref.within(f"lse at {t}", lse, el, tl)
            first = 4 + want.idx.shape[2] * 128
            # every decode since adds its own roundings: none is larger than this one's bound by more than the number of them
            ref.within(f"weight at {t}", ring_weight(store.weight, p, first, t + 1 - first), want.w[:, :, first:],
                       256 * 2.0 ** -18 * want.w[:, :, first:].clamp_min(1.0))
    check_state(store, want)
    assert want.idx.shape[2] == 5


def fill(p, dtype, block, keep, n, seed, device="cuda"):
    """A store that holds n random tokens, made by writing its tensors, and its fp64 twin."""
    g = torch.Generator(device=device).manual_seed(seed)
    store, want = lrsa.KVStore(p, dtype=dtype, block=block, keep=keep), ref.Store(p, dtype, block, keep)
    c = max((n - 1 - p.n_sink) // p.lag - 1, 0) if n > p.n_sink else 0
    heads, kp = (p.batch, p.n_kv_heads), store.rows_per_window
    for name in "kv":
        x = torch.randn(*heads, c, p.top_k, p.head_dim, generator=g, device=device)
        if dtype != BF16:
            scale = torch.exp2(torch.randint(-9, -3, heads + (c, kp // block), generator=g, device=device).float())
            x = (x * 40).round().clamp(-127, 127) if dtype == INT8 else (x * 100).clamp(-448, 448).to(E4M3).float()
            getattr(store, name + "_scale")[:, :, :c * kp // block] = scale.flatten(2)
            setattr(want, name + "_scale", scale.repeat_interleave(block, 3)[:, :, :, :p.top_k].flatten(2).double().cpu())
            rows = x * scale.repeat_interleave(block, 3)[:, :, :, :p.top_k, None]
        else:
            rows = x = x.bfloat16().float()
        getattr(store, name + "_list")[:, :, :c * kp].unflatten(2, (c, kp))[:, :, :, :p.top_k] = x.to(dtype)
        recent = torch.randn(*heads, p.n_sink + 2 * p.lag, p.head_dim, generator=g, device=device).bfloat16()
        getattr(store, name + "_recent").copy_(recent)
        setattr(want, name + "_rows", rows.flatten(2, 3).double().cpu())
        full = torch.zeros(*heads, n, p.head_dim, dtype=torch.float64)
        at = torch.arange(min(p.n_sink + c * p.lag, n), n)
        full[:, :, :p.n_sink] = recent[:, :, :min(p.n_sink, n)].double().cpu()
        full[:, :, at] = recent.double().cpu()[:, :, p.n_sink + (at - p.n_sink) % (2 * p.lag)]
        setattr(want, name.upper(), full)
    want.idx = torch.zeros(*heads, c, p.top_k, dtype=torch.long)
    want.w = torch.zeros(*heads, n, dtype=torch.float64)
    store.n_tokens = n
    return store, want


@pytest.mark.parametrize("dtype", [E4M3, INT8, BF16], ids=["e4m3", "int8", "bf16"])
@pytest.mark.parametrize("B,Hq,Hkv,d,L,K,S,n,block", [
    (1, 4, 4, 64, 512, 128, 16, 1, 64), (1, 7, 1, 128, 64, 16, 4, 4, 16), (2, 8, 8, 64, 100, 17, 0, 100, 32),
    (1, 28, 4, 128, 1024, 256, 4, 31743, 64),           # clusters of many CTAs
    (1, 8, 1, 64, 4096, 4096, 4, 126975, 128),          # one head, a long list: several clusters and the merge
    (1, 16, 2, 128, 2048, 2048, 0, 80000, 16),          # the same with two head groups
    (1, 24, 1, 128, 1024, 1024, 4, 60000, 64),          # and with two passes over the heads
    (16, 28, 4, 128, 256, 64, 4, 5000, 64),             # small CTAs
    (3, 5, 1, 64, 333, 83, 7, 6000, 128),
])
def test_decode_of_large_and_odd_stores(dtype, B, Hq, Hkv, d, L, K, S, n, block):
    p = P(B, Hq, Hkv, n + 5 + S, d, L, K, S)
    store, want = fill(p, dtype, block, "weight", n, seed=n)
    q = torch.randn(B, Hq, d, generator=torch.Generator().manual_seed(n)).bfloat16()
    o, lse = store.decode(q.cuda())
    o2, lse2 = store.decode(q.cuda())
    assert store.status() == 0 and torch.equal(o, o2) and torch.equal(lse, lse2)
    (eo, to), (el, tl), (eg, tg) = want.decode(q)
    ref.within("o", o, eo, to)
    ref.within("lse", lse, el, tl)
    first = S + want.idx.shape[2] * L
    if n > first:
        got = ring_weight(store.weight, p, first, n - first)
        ref.within("weight", got, 2 * eg, 2 * tg + 2.0 ** -23 * eg)
    assert int((store.weight != 0).sum()) <= B * Hkv * max(n - first, 0)      # other tokens' weights stay
    plain = lrsa.KVStore(p, dtype=dtype, block=block, keep="lag")
    for name in ("k_list", "v_list", "k_scale", "v_scale", "k_recent", "v_recent"):
        setattr(plain, name, getattr(store, name))
    plain.n_tokens = n
    o3, lse3 = plain.decode(q.cuda())
    assert torch.equal(o, o3) and torch.equal(lse, lse3)


@pytest.mark.parametrize("dtype", [E4M3, INT8], ids=["e4m3", "int8"])
@pytest.mark.parametrize("what", ["v_scales", "k_small", "q_large", "q_small", "q_zero", "spread"])
def test_decode_over_the_range_of_scales(dtype, what):
    """Scales that differ by 2^40 between blocks, queries near the ends of bf16, scores that are far apart."""
    p = P(1, 4, 2, 2000, 128, 128, 64, 4)
    store, want = fill(p, dtype, 32, "weight", 1900, seed=5)
    q = torch.randn(1, 4, 128, generator=torch.Generator().manual_seed(5)).bfloat16()
    c = want.idx.shape[2]
    if what == "v_scales":
        f = torch.exp2(torch.arange(store.v_scale.shape[2]) % 5 * 10.0 - 20)
        store.v_scale *= f.cuda()
        f = f[:c * 2].repeat_interleave(32).double()
        want.v_rows *= f[:, None]
        want.v_scale *= f
    elif what == "k_small":
        store.k_scale *= 2.0 ** -100
        want.k_rows *= 2.0 ** -100
    elif what == "spread":
        store.k_scale *= 16.0
        want.k_rows *= 16.0
    else:
        q = q * {"q_large": 2.0 ** 60, "q_small": 2.0 ** -120, "q_zero": 0.0}[what]
        if what == "q_large":
            store.k_scale *= 2.0 ** -60
            want.k_rows *= 2.0 ** -60
            store.k_recent.zero_()
            want.K.zero_()
    o, lse = store.decode(q.cuda())
    (eo, to), (el, tl), _ = want.decode(q)
    ref.within("o", o, eo, to)
    ref.within("lse", lse, el, tl)


def test_values_that_are_not_finite():
    """A block with an infinity or a NaN stands for NaN; other heads, and blocks that a query does not see, are not touched."""
    p = P(1, 4, 2, 4 + 6 * 64, 64, 64, 32, 4)
    Q, K, V, w = tokens(p, 3)
    K[0, 0, 4 + 70, 5] = math.inf                 # window 1 of head 0
    V[0, 0, 4 + 2 * 64 + 3, 7] = math.nan         # window 2
    w[:, :, 4 + 70] = w[:, :, 4 + 2 * 64 + 3] = 1e9      # both kept
    n = 4 + 4 * 64 + 1                            # windows 0, 1, 2 compressed
    for dtype in (E4M3, INT8):
        store, want = lrsa.KVStore(p, dtype=dtype, block=16), ref.Store(p, dtype, 16, "weight")
        store.append(*(x[:, :, :n].cuda().contiguous() for x in (K, V, w)))
        want.append(K[:, :, :n], V[:, :, :n], w[:, :, :n])
        check_state(store, want)
        k, v = store.rows()
        assert int(k.isnan().sum()) == 16 * 64 and int(v.isnan().sum()) == 16 * 64 and not k[:, 1].isnan().any()
        o, lse = store.decode(Q[:, :, n - 1].cuda().contiguous())
        assert o[:, :2].isnan().all() and lse[:, :2].isnan().all()
        (eo, to), (el, tl), _ = want.decode(Q[:, :, n - 1])
        ref.within("o", o[:, 2:], eo[:, 2:], to[:, 2:])
        ref.within("lse", lse[:, 2:], el[:, 2:], tl[:, 2:])
    # a ring row that no query sees any more, and list rows of windows not compressed yet, may hold anything
    store, want = fill(p, E4M3, 16, "weight", n, seed=2)
    store.k_scale[:, :, 3 * 2:] = math.nan
    store.v_scale[:, :, 3 * 2:] = math.nan
    seen = 4 + (torch.arange(4 + 3 * 64, n) - 4) % 128
    hidden = torch.ones(store.k_recent.shape[2], dtype=torch.bool)
    hidden[:4] = hidden[seen] = False
    store.k_recent[:, :, hidden.cuda()] = math.nan
    store.v_recent[:, :, hidden.cuda()] = math.inf
    o, lse = store.decode(Q[:, :, 0].cuda().contiguous())
    (eo, to), (el, tl), _ = want.decode(Q[:, :, 0])
    ref.within("o", o, eo, to)
    ref.within("lse", lse, el, tl)


def test_quantization_edges():
    """Blocks of zeros, of one value, of subnormals, of values on the borders between codes."""
    p = P(1, 1, 1, 6 * 16 + 1, 64, 16, 16, 0)
    K = torch.zeros(1, 1, p.seq_len, 64)
    K[:, :, 16:32] = 448.0 * (1 - 2 * (torch.arange(64) % 2))
    K[:, :, 32:48] = 2.0 ** -130 * torch.arange(64)
    border = torch.arange(1, 64) + 0.5
    K[:, :, 48:64, 0] = 127.0
    K[:, :, 48:64, 1:] = border                       # ties of int8 at scale 1
    K[:, :, 64:80, 0] = 448.0
    K[:, :, 64:80, 1:] = (16 + torch.arange(63)) * 0.5     # ties of e4m3 at scale 1
    K = K.bfloat16()
    V = (K.flip(3) * -1).contiguous()
    for dtype in (E4M3, INT8):
        store, want = lrsa.KVStore(p, dtype=dtype, block=16), ref.Store(p, dtype, 16, "weight")
        store.append(K.cuda(), V.cuda(), torch.ones(1, 1, p.seq_len, device="cuda"))
        want.append(K, V, torch.ones(1, 1, p.seq_len))
        check_state(store, want)
        assert torch.equal(store.k_scale[0, 0].double().cpu(), ref.held(K[0, 0, :80], dtype, 16)[1][:5]) and store.k_scale[0, 0, 0] == 1


def test_offsets_beyond_32_bits():
    """A list of more than 2^31 elements: every key scores zero, only the last window of the last head holds values."""
    p = P(1, 8, 8, 2 + 570 * 4096, 128, 4096, 4096, 2)
    store = lrsa.KVStore(p, dtype=INT8, block=128)
    assert store.k_list.numel() > 2 ** 31
    n = 2 + 569 * 4096 + 5                         # windows 0 .. 567 compressed
    store.n_tokens = n
    store.k_scale.fill_(1.0)
    store.v_scale.fill_(0.5)
    store.v_list[0, 7, 567 * 4096:568 * 4096] = 64
    q = torch.randn(1, 8, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    o, lse = store.decode(q)
    keys = 568 * 4096 + 2 + 4096 + 5
    assert store.status() == 0 and float(o[:, :7].abs().max()) == 0.0
    assert ((o[0, 7].double() - 32.0 * 4096 / keys).abs() <= 2.0 ** -8 * 32.0 * 4096 / keys).all()
    assert ((lse.double() - math.log(keys)).abs() <= 1e-5).all()
    assert ((store.weight[:, :, :5].double() * keys - 1).abs() <= 1e-4).all()
    k = torch.randn(1, 8, 4096, 128, generator=torch.Generator().manual_seed(2)).bfloat16()
    w = torch.rand(1, 8, 4096, generator=torch.Generator().manual_seed(3))
    del store, o, lse
    wide = P(1, 8, 8, 2 + 571 * 4096, 128, 4096, 4096, 2)
    big = lrsa.KVStore(wide, dtype=INT8, block=128)
    big.n_tokens = 2 + 568 * 4096
    big.append(k.cuda(), (-k).cuda(), w.cuda())
    big.append(k.cuda(), (-k).cuda(), w.cuda())
    big.append(k[:, :, :1].cuda(), k[:, :, :1].cuda())     # window 568 is cut: its rows lie behind 2^31 elements
    assert big.windows_compressed() == 569
    for rows, scale, x in ((big.k_list, big.k_scale, k), (big.v_list, big.v_scale, -k)):
        got = rows[:, :, 568 * 4096:].double().cpu().unflatten(2, (-1, 128)) * scale[:, :, 568 * 32:].double().cpu()[..., None, None]
        assert torch.equal(got.flatten(2, 3)[:, :, :4096], ref.held(x, INT8, 128)[0])


@pytest.mark.parametrize("L,K", [(9729, 9729), (32767, 5000)])
def test_long_windows(L, K):
    """Windows whose weights take more shared memory than a kernel gets unasked, some of their tokens in the ring."""
    p = P(1, 2, 2, 3 + 5 * L, 64, L, K, 3)
    g = torch.Generator(device="cuda").manual_seed(L)
    n = 3 + 4 * L + 9
    k, v = (torch.randn(1, 2, n, 64, generator=g, device="cuda").bfloat16() for _ in "kv")
    w = torch.rand(1, 2, n, generator=g, device="cuda")
    store, at = lrsa.KVStore(p, dtype=E4M3, block=64), 3 + L + L // 2
    store.append(k[:, :, :at].contiguous(), v[:, :, :at].contiguous(), w[:, :, :at].contiguous())
    store.append(k[:, :, at:].contiguous(), v[:, :, at:].contiguous(), w[:, :, at:].contiguous())
    assert store.windows_compressed() == 3 and store.status() == 0
    sel = lrsa.lrsa_weight_select(P(1, 2, 2, n, 64, L, K, 3), w)
    assert torch.equal(store.idx, sel)
    for rows, x in zip(store.rows(), (k, v)):
        for i in range(3):
            kept = torch.gather(x, 2, sel[:, :, i, :, None].long().expand(-1, -1, -1, 64)).cpu()
            assert torch.equal(rows[:, :, i * K:(i + 1) * K].double().cpu(), ref.held(kept, E4M3, 64)[0])


def test_hundreds_of_heads_in_a_group():
    """More heads than the merge of several clusters has room for: one cluster, and no call that is refused half way."""
    p = P(1, 700, 1, 33010, 64, 512, 512, 2)
    store, want = fill(p, INT8, 64, "weight", 33000, seed=700)
    q = torch.randn(1, 700, 64, generator=torch.Generator().manual_seed(700)).bfloat16()
    o, lse = store.decode(q.cuda())
    (eo, to), (el, tl), (eg, tg) = want.decode(q)
    ref.within("o", o, eo, to)
    ref.within("lse", lse, el, tl)
    first = 2 + want.idx.shape[2] * 512
    ref.within("weight", ring_weight(store.weight, p, first, 33000 - first), eg, tg)


def test_a_selection_that_ran_out_of_time():
    """Long windows by the lag rule: a scoring kernel whose wait ends without an answer leaves no positions.  The status says so, the
    rows are copied from inside the store all the same, and the next selection is whole."""
    p = P(1, 2, 2, 2 + 6 * 4608, 64, 4608, 100, 2)
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn(1, 2, 2 + 5 * 4608 + 1, 64, generator=g, device="cuda").bfloat16() for _ in "kv")
    store, whole = (lrsa.KVStore(p, dtype=E4M3, block=32, keep="lag") for _ in "ab")
    at = 2 + 4 * 4608
    for s in (store, whole):
        s.append(k[:, :, :at].contiguous(), v[:, :, :at].contiguous())
    lrsa.lrsa_debug_set_wait_limit(-1)
    try:
        store.append(k[:, :, at:at + 1].contiguous(), v[:, :, at:at + 1].contiguous())      # window 2, out of the ring
        assert store.status() == 5
    finally:
        lrsa.lrsa_debug_set_wait_limit(0)
    whole.append(k[:, :, at:at + 1].contiguous(), v[:, :, at:at + 1].contiguous())
    for s in (store, whole):
        s.append(k[:, :, at + 1:].contiguous(), v[:, :, at + 1:].contiguous())
        assert s.status() == 0 and s.windows_compressed() == 4
    assert torch.equal(store.idx[:, :, [0, 1, 3]], whole.idx[:, :, [0, 1, 3]])
    a, b = store.rows(), whole.rows()
    for i in (0, 1, 3):
        assert all(torch.equal(x[:, :, 100 * i:100 * i + 100], y[:, :, 100 * i:100 * i + 100]) for x, y in zip(a, b))


def test_a_store_elsewhere_is_refused():
    p = P(1, 4, 2, 1000, 128, 128, 32, 4)
    store = lrsa.KVStore(p, device="cpu")
    k = torch.zeros(1, 2, 8, 128, dtype=BF16, device="cuda")
    with pytest.raises(lrsa.LrsaError) as e:
        store.append(k, k)
    assert e.value.status == 1 and store.n_tokens == 0
    store.n_tokens = 8
    with pytest.raises(lrsa.LrsaError) as e:
        store.decode(torch.zeros(1, 4, 128, dtype=BF16, device="cuda"))
    assert e.value.status == 1


def test_two_stores_on_two_streams_and_in_graphs():
    p = P(2, 8, 2, 3000, 128, 256, 64, 4)
    made = [fill(p, t, 64, "weight", 2800, seed=s) for t, s in ((E4M3, 1), (INT8, 2))]
    qs = [torch.randn(2, 8, 128, generator=torch.Generator().manual_seed(s)).bfloat16().cuda() for s in (1, 2)]
    want = []
    for (store, _), q in zip(made, qs):
        o, lse = store.decode(q)
        want.append((o.clone(), lse.clone(), store.weight.clone()))
        store.weight.zero_()
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):
        for (store, _), q, s in zip(made, qs, streams):
            with torch.cuda.stream(s):
                outs.append(store.decode(q))
    torch.cuda.synchronize()
    for i, (o, lse) in enumerate(outs):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])
    for (store, _), w in zip(made, want):
        assert (store.weight - 3 * w[2]).abs().max() <= 2.0 ** -22 * 3 * float(w[2].max())
        store.weight.zero_()
    torch.cuda.synchronize()
    graphs, res = [], []
    for (store, _), q in zip(made, qs):      # each store has a workspace of its own
        graph = torch.cuda.CUDAGraph()
        o, lse = torch.empty_like(q), torch.empty(2, 8, device="cuda")
        with torch.cuda.graph(graph):
            store.decode(q, o=o, lse=lse)
        graphs.append(graph)
        res.append((o, lse))
    for graph in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for (store, _), w, r in zip(made, want, res):
        assert torch.equal(r[0], w[0]) and torch.equal(r[1], w[1]) and torch.equal(store.weight, w[2])


def test_refusals():
    p = P(1, 4, 2, 1000, 128, 128, 32, 4)
    store = lrsa.KVStore(p)
    k = torch.zeros(1, 2, 8, 128, dtype=BF16, device="cuda")
    w = torch.zeros(1, 2, 8, device="cuda")
    q = torch.zeros(1, 4, 128, dtype=BF16, device="cuda")
    with pytest.raises(lrsa.LrsaError):            # nothing in it
        store.decode(q)
    for bad in ((k.float(), k, None), (k, k[:, :, :7], None), (k, k, w.double()), (k, k, w[:, :, :4]), (k.cpu(), k, None),
                (k[:, :, ::2], k[:, :, ::2], None), (k[0], k[0], None), (k[:, :1], k[:, :1], None), (k[:, :, :0], k[:, :, :0], None)):
        with pytest.raises(lrsa.LrsaError) as e:
            store.append(*bad)
        assert e.value.status == 1 and store.n_tokens == 0
    store.n_tokens = 996                           # beyond the capacity
    with pytest.raises(lrsa.LrsaError) as e:
        store.append(k, k)
    assert e.value.status == 1
    store.n_tokens = 500
    for bad in (q.float(), q[:, :2], q[None], q.cpu()):
        with pytest.raises(lrsa.LrsaError) as e:
            store.decode(bad)
        assert e.value.status == 1
    with pytest.raises(lrsa.LrsaError):
        store.decode(q, o=torch.empty(1, 4, 64, dtype=BF16, device="cuda"))
    store.n_tokens = 0
    prompt = torch.zeros(1, 2, 700, 128, dtype=BF16, device="cuda")
    with pytest.raises(lrsa.LrsaError) as e:       # cuts windows of its own tokens, by weights that nobody gave
        store.append(prompt, prompt)
    assert e.value.status == 1
    with pytest.raises(lrsa.LrsaError) as e:       # weights for a store that does not keep them
        lrsa.KVStore(p, keep="lag").append(k, k, w)
    assert e.value.status == 1


@pytest.mark.parametrize("keep", ["weight", "lag"])
def test_more_heads_than_a_grid_has_rows(keep):
    """65536 (batch, KV head) pairs: 64 different ones, repeated, against the small store that holds each once."""
    few, many = (P(b, 32, 32, 4 + 3 * 16 + 2, 64, 16, 5, 4) for b in (2, 2048))
    Q, K, V, w = tokens(few, 77)
    small, want = lrsa.KVStore(few, dtype=E4M3, block=16, keep=keep), ref.Store(few, E4M3, 16, keep)
    store = lrsa.KVStore(many, dtype=E4M3, block=16, keep=keep)
    for lo, n in ((0, 4 + 2 * 16), (4 + 2 * 16, 1), (4 + 2 * 16 + 1, few.seq_len - 4 - 2 * 16 - 1)):
        k, v, e = (x[:, :, lo:lo + n] for x in (K, V, w))
        e = e if keep == "weight" else None
        args = [x if x is None else x.cuda().contiguous() for x in (k, v, e)]
        small.append(*args)
        store.append(*(x if x is None else x.repeat((1024,) + (1,) * (x.dim() - 1)) for x in args))
        want.append(k, v, e, small.idx[:, :, :small.windows_compressed()].cpu())
    check_state(small, want)
    assert store.status() == 0 and store.windows_compressed() == 2
    for name in ("idx", "k_list", "v_list", "k_scale", "v_scale", "k_recent", "v_recent") + (("weight",) if keep == "weight" else ()):
        a, b = (getattr(s, name).view(torch.uint8) for s in (store, small))
        assert torch.equal(a.view(1024, *b.shape), b.expand(1024, *b.shape))
    for got, rows in zip(store.rows(), small.rows()):
        assert torch.equal(got.view(1024, *rows.shape), rows.expand(1024, *rows.shape))
    q = Q[:, :, -1].contiguous()
    o, lse = store.decode(q.cuda().repeat(1024, 1, 1))
    assert store.status() == 0
    (eo, to), (el, tl), (_, tg) = want.decode(q)
    ref.within("o", o, eo.repeat(1024, 1, 1), to.repeat(1024, 1, 1))
    ref.within("lse", lse, el.repeat(1024, 1), tl.repeat(1024, 1))
    if keep == "weight":
        first = 4 + 2 * 16
        got, all_w = ring_weight(store.weight, many, first, few.seq_len - first), want.w[:, :, first:]
        ref.within("weight", got, all_w.repeat(1024, 1, 1), (tg + 2.0 ** -24 * all_w).repeat(1024, 1, 1))


@pytest.mark.parametrize("given", [True, False], ids=["given", "zero"])
@pytest.mark.parametrize("p,steps", [
    (P(2, 4, 2, 5 + 9 * 48 + 7, 64, 48, 12, 5), (3, 1, 1, 40, 9, 48, 48, 96, 1, 30, 1)),     # sinks alone, then several turns of the ring
    (P(1, 3, 3, 7 * 64 + 2, 128, 64, 64, 0), (130, 64, 1, 63, 64, 2, 100)),                  # no sinks
    (P(1, 7, 1, 2 + 6 * 33, 64, 33, 8, 2), (2 + 33, 33, 34, 32, 17, 1)),
])
def test_weights_in_the_ring(p, steps, given):
    """What append leaves of the gathered weights, to the bit: the new tokens' are those that were given (zero without), the earlier
    tokens' are what they were, decode's additions among them."""
    Q, K, V, w = (x.cuda() for x in tokens(p, 31))
    store = lrsa.KVStore(p, dtype=INT8, block=16)
    store.weight.fill_(-5.0)                  # a row that is not written would show
    known, i = torch.zeros(p.batch, p.n_kv_heads, p.seq_len, device="cuda"), 0
    while store.n_tokens < p.seq_len:
        lo = store.n_tokens
        n = min(steps[i % len(steps)], p.seq_len - lo)
        i += 1
        c = max((lo + n - 1 - p.n_sink) // p.lag - 1, 0) if lo + n > p.n_sink else 0
        own = c > store.windows_compressed() and p.n_sink + c * p.lag > lo     # a window of the call's own tokens is cut
        e = w[:, :, lo:lo + n].contiguous() if given or own else None
        known[:, :, lo:lo + n] = 0.0 if e is None else e
        store.append(K[:, :, lo:lo + n].contiguous(), V[:, :, lo:lo + n].contiguous(), e)
        first = p.n_sink + c * p.lag
        if lo + n > first:
            at = torch.arange(first, lo + n, device="cuda")
            row = (at - p.n_sink) % (2 * p.lag)
            assert torch.equal(store.weight[:, :, row], known[:, :, at]), f"{lo} + {n}"
            rest = store.weight.clone()
            store.decode(Q[:, :, lo + n - 1].contiguous())
            known[:, :, at] = store.weight[:, :, row]
            assert (known[:, :, at] >= rest[:, :, row]).all() and (known[:, :, at] > rest[:, :, row]).any()
            hidden = torch.ones(2 * p.lag, dtype=torch.bool, device="cuda")
            hidden[row] = False
            assert torch.equal(store.weight[:, :, hidden], rest[:, :, hidden])
    assert store.status() == 0 and store.windows_compressed() >= 4


@pytest.mark.parametrize("d,L,n", [(128, 128, 4 + 5 * 128 + 3), (64, 48, 4 + 5 * 48 + 45), (64, 48, 4 + 2 * 48 + 1), (64, 100, 3), (128, 100, 54)])
@pytest.mark.parametrize("dtype", [E4M3, BF16], ids=["e4m3", "bf16"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_of_visible_rows_that_are_not_finite(dtype, d, L, n, bad):
    """An infinity in a value that the query sees is one channel's infinity, wherever the row stands in its tile: not a NaN, and
    nothing in the other channels."""
    p = P(1, 6, 2, n + 7, d, L, 16, 4)
    store, want = fill(p, dtype, 16, "weight", n, seed=n + d)
    q = torch.randn(1, 6, d, generator=torch.Generator().manual_seed(n)).bfloat16()
    (eo, to), (el, tl), _ = want.decode(q)
    first = min(n, 4 + want.idx.shape[2] * L)
    spots = [(store.v_recent, 0)] + [(store.v_recent, 4 + (t - 4) % (2 * L)) for t in {first, n - 1, (first + n) // 2} if t >= max(first, 4)]
    if dtype == BF16 and want.idx.shape[2]:
        spots += [(store.v_list, 0), (store.v_list, (want.idx.shape[2] - 1) * store.rows_per_window + 15)]
    for rows, at in spots:
        old = rows[0, 1, at, 9].clone()
        rows[0, 1, at, 9] = bad
        o, lse = store.decode(q.cuda())
        rows[0, 1, at, 9] = old
        ref.within("lse", lse, el, tl)
        o = o.cpu()
        hit = o[:, 3:, 9]
        assert torch.equal(hit.nan_to_num(7.0, 8.0, 9.0), torch.full_like(hit, bad).nan_to_num(7.0, 8.0, 9.0)), f"row {at}: {hit}"
        o[:, 3:, 9] = eo[:, 3:, 9].bfloat16()
        ref.within("o", o, eo, to)
