"""laq_paged_append and laq_paged_attention against the 64-bit oracle: pages of every kind, ragged
batches, chunks longer than their cache, strides, foreign streams."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import serving  # noqa: E402
from paper_2605_08755_gb300 import _lib  # noqa: E402

pytestmark = pytest.mark.gpu
D, SCALE = 128, 1 / math.sqrt(128)
F16, BF16 = torch.float16, torch.bfloat16
UNIT = {F16: 2.0 ** -11, BF16: 2.0 ** -8}   # unit roundoff


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2605_08755_gb300 import build
    build.build()


def batch(n, L, P, seed, spare=2, table_extra=1, wild=-1):
    """(table, q_start, kv_len): every request's pages scattered, unused entries ``wild``."""
    used = [max(0, -(-x // P)) for x in L]
    ids = np.random.default_rng(seed).permutation(sum(used) + spare).astype(np.int32)
    table = np.full((len(n), max(used + [0]) + table_extra), wild, np.int32)
    at = 0
    for b, x in enumerate(used):
        table[b, :x] = ids[at:at + x]
        at += x
    return table, np.concatenate([[0], np.cumsum(n)]).astype(np.int32), np.array(L, np.int32), \
        len(ids)


def f64(t):
    return t.double().cpu().numpy()


def make_cache(pages, Hkv, P, dtype, seed, order="head"):
    """k, v [pages, Hkv, P, D] views: dense, slots before heads, or halves of one buffer."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
    if order == "slot":
        return [r(pages, P, Hkv, D).transpose(1, 2) for _ in range(2)]
    if order == "joint":
        kv = r(pages, 2, Hkv, P, D)
        return [kv[:, 0], kv[:, 1]]
    return [r(pages, Hkv, P, D) for _ in range(2)]


def check_attention(out, q, k, v, table, q_start, kv_len, scale, dtype):
    """Output rounding u |out|; each probability rounded once, u A with A = sum P |v|; fp32 scores,
    exponentials and sums (and probabilities below fp16's normal range): 2^-14 A; half the smallest
    fp16 step."""
    ref, A = serving.paged_attention(f64(q), f64(k), f64(v), table, q_start, kv_len, scale)
    u = UNIT[dtype]
    err, tol = np.abs(f64(out) - ref), u * np.abs(ref) + (u + 2.0 ** -14) * A + 2.0 ** -25
    assert np.all(err <= tol), (err - tol).max()


ATTENTION = [
    # n, L, page, Hq, Hkv, type, cache order
    ([1], [1], 16, 4, 4, F16, "head"),
    ([1], [0], 16, 4, 2, F16, "head"),
    ([1, 1, 1], [17, 0, 2050], 16, 32, 8, F16, "head"),
    ([1] * 5, [127, 128, 129, 255, 257], 64, 8, 2, BF16, "slot"),
    ([1], [5000], 128, 8, 1, F16, "joint"),
    ([1], [20011], 32, 4, 1, BF16, "head"),
    ([1] * 33, list(range(1, 331, 10)), 8, 5, 1, F16, "head"),
    ([2, 0, 3, 1], [100, 50, 3, 1], 16, 8, 2, F16, "slot"),
    ([4] * 6, [300, 4, 64, 63, 1030, 129], 32, 16, 4, BF16, "head"),
    ([17, 1, 16], [17, 900, 500], 256, 14, 2, F16, "head"),
    ([128], [128], 16, 4, 1, F16, "head"),
    ([129], [129], 128, 4, 2, BF16, "joint"),
    ([200, 1, 77], [1000, 700, 77], 64, 7, 1, F16, "head"),
    ([300], [301], 1024, 6, 2, F16, "slot"),
    ([65], [2000], 8, 40, 2, BF16, "head"),
    ([3], [700], 16, 64, 1, F16, "head"),
    ([130], [9000], 32, 2, 2, F16, "head"),
    ([5, 300], [3, 100], 16, 8, 2, F16, "head"),       # more new tokens than cached ones
    ([1, 40], [-4, 1 << 30], 16, 4, 2, F16, "head"),    # lengths outside the table: clamped
]


@pytest.mark.parametrize("n,L,P,Hq,Hkv,dtype,order", ATTENTION)
def test_attention(n, L, P, Hq, Hkv, dtype, order):
    Lc = [max(0, x) if x < 1 << 20 else 3 * P for x in L]
    table, q_start, kv_len, pages = batch(n, Lc, P, seed=len(n) + sum(Lc),
                                          table_extra=0 if L != Lc else 1)
    Lc = [min(x, table.shape[1] * P) for x in Lc]
    k, v = make_cache(pages, Hkv, P, dtype, sum(n) + P, order)
    g = torch.Generator(device="cuda").manual_seed(5)
    q = (1.5 * torch.randn((sum(n), Hq, D), generator=g, device="cuda")).to(dtype)
    # a few dominant keys late in the requests, so that maxima move after much has been summed
    for b, x in enumerate(Lc):
        if x > 40:
            k[int(table[b, (x - 30) // P]), :, (x - 30) % P] *= 5
    # what lies past a request's last token must not matter
    for b, x in enumerate(Lc):
        if x % P:
            for c in (k, v):
                c[int(table[b, x // P]), :, x % P:] = float("nan")
    cache = _lib.PagedCache(k, v, torch.from_numpy(table).cuda(), torch.from_numpy(q_start).cuda(),
                            torch.tensor(L, dtype=torch.int32).cuda())
    ws = _lib.paged_attention_workspace(sum(n), len(n), max(n) + 100, Hq, Hkv, "cuda")
    out = torch.full((sum(n), Hq, D), float("nan"), dtype=dtype, device="cuda")
    for _ in range(2):   # the workspace serves again
        _lib.laq_paged_attention(q, cache, max(n), SCALE, ws, out=out)
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)) == 0
    check_attention(out, q, k, v, table, q_start, np.array(Lc), SCALE, dtype)
    first = out.clone()
    _lib.laq_paged_attention(q, cache, max(n) + 100 if sum(n) < 40 else max(n), SCALE, ws, out=out)
    if sum(n) >= 40:
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))   # bit for bit


def test_attention_strided_rows_and_foreign_pages():
    """q as the first part of wider rows; pages outside the cache read as zeros."""
    n, L, P, Hq, Hkv = [3, 150], [200, 150], 32, 8, 2
    table, q_start, kv_len, pages = batch(n, L, P, 3)
    k, v = make_cache(pages, Hkv, P, F16, 4)
    table[0, 2] = pages        # just outside
    table[1, 1] = -7
    rows = torch.randn((sum(n), Hq * D + 64), device="cuda").half()
    q = rows[:, :Hq * D].unflatten(1, (Hq, D))
    cache = _lib.PagedCache(k, v, torch.from_numpy(table).cuda(), torch.from_numpy(q_start).cuda(),
                            torch.from_numpy(kv_len).cuda())
    ws = _lib.paged_attention_workspace(sum(n), 2, 150, Hq, Hkv, "cuda")
    out = _lib.laq_paged_attention(q, cache, 150, SCALE, ws)
    check_attention(out, q, k, v, table, q_start, kv_len, SCALE, F16)


def test_attention_rows_of_no_request_and_past_max_q():
    n, L, P, Hq, Hkv = [4, 2], [50, 9], 16, 4, 2
    table, q_start, kv_len, pages = batch(n, L, P, 3)
    k, v = make_cache(pages, Hkv, P, F16, 4)
    T = sum(n) + 5
    q = torch.randn((T, Hq, D), device="cuda").half()
    cache = _lib.PagedCache(k, v, torch.from_numpy(table).cuda(), torch.from_numpy(q_start).cuda(),
                            torch.from_numpy(kv_len).cuda())
    ws = _lib.paged_attention_workspace(T, 2, 3, Hq, Hkv, "cuda")
    out = torch.full((T, Hq, D), 7.0, dtype=F16, device="cuda")
    _lib.laq_paged_attention(q, cache, 3, SCALE, ws, out=out)
    ref, _ = serving.paged_attention(f64(q[:6]), f64(k), f64(v), table, q_start, kv_len, SCALE)
    got = f64(out)
    assert np.allclose(got[:3], ref[:3], atol=4e-3) and np.allclose(got[4:6], ref[4:6], atol=4e-3)
    assert (got[3] == 7).all() and (got[6:] == 7).all()


@pytest.mark.parametrize("n,L", [([1], [3000]), ([40, 1], [3000, 100])])
def test_attention_on_another_stream_and_in_a_graph(n, L):
    P, Hq, Hkv = 64, 8, 2
    table, q_start, kv_len, pages = batch(n, L, P, 9)
    k, v = make_cache(pages, Hkv, P, F16, 2)
    q = torch.randn((sum(n), Hq, D), device="cuda").half()
    cache = _lib.PagedCache(k, v, torch.from_numpy(table).cuda(), torch.from_numpy(q_start).cuda(),
                            torch.from_numpy(kv_len).cuda())
    ws = _lib.paged_attention_workspace(sum(n), len(n), max(n), Hq, Hkv, "cuda")
    out = torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    _lib.laq_paged_attention(q, cache, max(n), SCALE, ws, out=out, stream=s)
    s.synchronize()
    check_attention(out, q, k, v, table, q_start, kv_len, SCALE, F16)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        _lib.laq_paged_attention(q, cache, max(n), SCALE, ws, out=out, stream=s)
    # the graph reads the tables anew: shorter requests at the same addresses
    q.normal_()
    kv_len = kv_len - 37
    cache.kv_len.copy_(torch.from_numpy(kv_len))
    g.replay()
    torch.cuda.synchronize()
    check_attention(out, q, k, v, table, q_start, kv_len, SCALE, F16)


def test_attention_offsets_past_32_bits():
    """The last pages of a cache of 5 GB a side: element offsets past 2^31, byte offsets past 2^32."""
    P, Hkv, Hq = 256, 8, 16
    pages = 10500
    k = torch.zeros((pages, Hkv, P, D), dtype=F16, device="cuda")
    v = torch.zeros_like(k)
    ids = [pages - 1, 0, pages - 2]
    for p in ids:
        k[p].normal_()
        v[p].normal_()
    for n, L in ((1, 700), (33, 650)):
        table = np.array([ids], np.int32)
        q_start, kv_len = np.array([0, n], np.int32), np.array([L], np.int32)
        q = torch.randn((n, Hq, D), device="cuda").half()
        cache = _lib.PagedCache(k, v, torch.from_numpy(table).cuda(),
                                torch.from_numpy(q_start).cuda(), torch.from_numpy(kv_len).cuda())
        ws = _lib.paged_attention_workspace(n, 1, n, Hq, Hkv, "cuda")
        out = _lib.laq_paged_attention(q, cache, n, SCALE, ws)
        small = [k[ids], v[ids]]
        check_attention(out, q, *small, np.array([[0, 1, 2]]), q_start, kv_len, SCALE, F16)
        qkv = torch.randn((n, (Hq + 2 * Hkv) * D), device="cuda").half()
        _lib.laq_paged_append(qkv, cache, Hq, 1e6, 1e-6)
        last = qkv[-1].view(-1, D)[Hq + Hkv:]
        assert torch.equal(v[ids[(L - 1) // P], :, (L - 1) % P], last)


@pytest.mark.parametrize("n,L,P,Hq,Hkv,dtype,order,normed", [
    ([1], [2048], 16, 32, 8, F16, "head", True),
    ([1, 1, 3, 0, 6], [9, 1, 3, 4, 1000], 8, 8, 2, BF16, "slot", True),
    ([37], [37], 32, 5, 1, F16, "joint", False),
    ([1] * 70, list(range(1, 71)), 16, 4, 4, BF16, "head", True),
    ([4, 9], [3, 100000], 1024, 16, 2, F16, "head", True),
])
def test_append(n, L, P, Hq, Hkv, dtype, order, normed):
    table, q_start, kv_len, pages = batch(n, L, P, sum(L))
    k, v = make_cache(pages, Hkv, P, dtype, 8, order)
    T = sum(n)
    wide = (2 * torch.randn((T, (Hq + 2 * Hkv) * D + 12), device="cuda")).to(dtype)
    qkv = wide[:, :(Hq + 2 * Hkv) * D]
    qw = (1 + 0.1 * torch.randn(D, device="cuda")).to(dtype) if normed else None
    kw = (1 + 0.1 * torch.randn(D, device="cuda")).to(dtype) if normed else None
    cache = _lib.PagedCache(k, v, torch.from_numpy(table).cuda(), torch.from_numpy(q_start).cuda(),
                            torch.from_numpy(kv_len).cuda())
    k0, v0 = f64(k), f64(v)
    q = _lib.laq_paged_append(qkv, cache, Hq, 1e6, 1e-6, q_norm_w=qw, k_norm_w=kw)
    ref, stored = serving.paged_append(f64(qkv), table, q_start, kv_len, Hq, Hkv, P,
                                       None if qw is None else f64(qw),
                                       None if kw is None else f64(kw), 1e6, 1e-6)
    u = UNIT[dtype]

    def close(a, r):
        # one rounding of the value; fp32 norm, cosine and products: 2^-20 of the pair's size
        pair = np.abs(r) + np.abs(np.roll(r, 64, -1))
        tol = u * np.abs(r) + 2.0 ** -20 * pair + 2.0 ** -25
        assert np.all(np.abs(a - r) <= tol)
    close(f64(q), ref)
    k1, v1 = f64(k), f64(v)
    for (page, g, s), (kr, vr) in stored.items():
        close(k1[page, g, s], kr)
        assert np.array_equal(v1[page, g, s], vr)
        k1[page, g, s], v1[page, g, s] = k0[page, g, s], v0[page, g, s]
    assert np.array_equal(k1, k0) and np.array_equal(v1, v0)   # nothing else was written


def test_append_page_outside_the_cache_and_rows_of_no_request():
    k, v = make_cache(4, 2, 16, F16, 1)
    cache = _lib.PagedCache(k, v, torch.tensor([[4, -1], [1, 2]], dtype=torch.int32, device="cuda"),
                            torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda"),
                            torch.tensor([17, 20], dtype=torch.int32, device="cuda"))
    before = k.clone()
    qkv = torch.randn((5, 6 * D), device="cuda").half()
    q = torch.full((5, 2, D), 9.0, dtype=F16, device="cuda")
    _lib.laq_paged_append(qkv, cache, 2, 1e4, 1e-6, q_out=q)
    torch.cuda.synchronize()
    before[2, :, 3] = k[2, :, 3]
    assert torch.equal(k, before) and (q[3:] == 9).all() and not (q[:3] == 9).all()


@pytest.mark.parametrize("n,L,Hkv", [([40], [1500], 1), ([200], [700], 2), ([2], [1500], 1)])
def test_attention_where_early_keys_score_minus_infinity(n, L, Hkv):
    """Keys of -inf in the first tiles (q positive): those tokens have weight 0 and leave a row without a
    maximum until its first finite score."""
    P, Hq = 16, 4 * Hkv
    table, q_start, kv_len, pages = batch(n, L, P, 21)
    k, v = make_cache(pages, Hkv, P, F16, 22)
    q = torch.rand((sum(n), Hq, D), device="cuda").half() + 0.01
    for t in range(400):
        k[int(table[0, t // P]), :, t % P] = float("-inf")
    cache = _lib.PagedCache(k, v, torch.from_numpy(table).cuda(), torch.from_numpy(q_start).cuda(),
                            torch.from_numpy(kv_len).cuda())
    ws = _lib.paged_attention_workspace(sum(n), 1, max(n), Hq, Hkv, "cuda")
    out = _lib.laq_paged_attention(q, cache, max(n), SCALE, ws)
    finite = k.clone()   # the same weights: far below every other key's
    finite[finite == float("-inf")] = -1000.0
    check_attention(out, q, finite, v, table, q_start, kv_len, SCALE, F16)


@pytest.mark.parametrize("n,L", [([33], [33]), ([150, 1], [2500, 90])])
def test_attention_of_scores_that_keep_growing(n, L):
    """Keys that grow along the request, so that the maximum moves in most tiles, in small steps and in
    large ones, up to scores of some hundreds."""
    P, Hq, Hkv = 32, 4, 1
    table, q_start, kv_len, pages = batch(n, L, P, 31)
    k, v = make_cache(pages, Hkv, P, BF16, 32)
    q = (2 * torch.randn((sum(n), Hq, D), device="cuda")).to(BF16)
    for b, x in enumerate(L):
        for t in range(x):
            k[int(table[b, t // P]), :, t % P] *= 0.05 + 12.0 * t / x
    cache = _lib.PagedCache(k, v, torch.from_numpy(table).cuda(), torch.from_numpy(q_start).cuda(),
                            torch.from_numpy(kv_len).cuda())
    ws = _lib.paged_attention_workspace(sum(n), len(n), max(n), Hq, Hkv, "cuda")
    out = _lib.laq_paged_attention(q, cache, max(n), SCALE, ws)
    # fp32 scores of a few hundred: 2^-24 of the products' sum, 128 of them, adds 2^-9 to a weight
    ref, A = serving.paged_attention(f64(q), f64(k), f64(v), table, q_start, kv_len, SCALE)
    u = UNIT[BF16]
    assert np.all(np.abs(f64(out) - ref) <= u * np.abs(ref) + (u + 2.0 ** -8) * A + 2.0 ** -25)
