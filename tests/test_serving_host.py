"""Host-side checks of the serving calls (no GPU): every refusal before anything touches a device,
empty work, the binding's checks, and the oracle's pins."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import serving  # noqa: E402
from paper_2605_08755_gb300 import _lib  # noqa: E402

A = 0x10000   # 16-byte aligned, never dereferenced: calls fail first
NULL, CONFIG, SHAPE, ALIGN, WS = 1, 9, 4, 5, 10


@pytest.fixture(scope="module")
def L():
    from paper_2605_08755_gb300 import build
    build.build()
    return _lib.lib()


def kv(**edit):
    f = dict(k=A, v=A, block_table=A, q_start=A, kv_len=A, pages=10, page_stride=8 * 16 * 128,
             head_stride=16 * 128, token_stride=128, batch=2, table_stride=4, max_pages=4,
             page_size=16, Hkv=8, D=128, dtype=0)
    f.update(edit)
    return ctypes.byref(_lib.PagedKv(**f))


BAD_KV = [(dict([(n, None)]), NULL) for n in ("k", "v", "block_table", "q_start", "kv_len")] + [
    (dict(D=64), SHAPE), (dict(Hkv=0), SHAPE), (dict(Hkv=5), SHAPE), (dict(page_size=24), SHAPE),
    (dict(page_size=4), SHAPE), (dict(page_size=2048), SHAPE), (dict(page_size=0), SHAPE),
    (dict(page_size=-16), SHAPE), (dict(pages=0), SHAPE), (dict(pages=1 << 31), SHAPE),
    (dict(batch=-1), SHAPE), (dict(batch=(1 << 24) + 1), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(max_pages=1 << 27, table_stride=1 << 27), SHAPE), (dict(table_stride=3), SHAPE),
    (dict(token_stride=64), SHAPE), (dict(token_stride=132), SHAPE), (dict(head_stride=0), SHAPE),
    (dict(page_stride=-128), SHAPE), (dict(page_stride=1 << 38), SHAPE), (dict(dtype=2), CONFIG),
    (dict(dtype=-1), CONFIG), (dict(k=A + 8), ALIGN), (dict(v=A + 2), ALIGN),
    (dict(block_table=A + 2), ALIGN), (dict(q_start=A + 1), ALIGN), (dict(kv_len=A + 2), ALIGN)]


@pytest.mark.parametrize("edit,status", BAD_KV)
def test_cache_refusals(L, edit, status):
    assert append(L, kv(**edit)) == status
    assert attend(L, kv(**edit)) == status


def append(L, c=None, qkv=A, stride=48 * 128, T=3, Hq=32, qw=A, kw=A, theta=1e6, eps=1e-6, out=A):
    return L.laq_paged_append(c or kv(), qkv, stride, T, Hq, qw, kw, theta, eps, out, None)


def attend(L, c=None, q=A, stride=32 * 128, T=3, max_q=2, Hq=32, scale=0.1, out=A, ws=A,
           ws_bytes=1 << 40):
    return L.laq_paged_attention(c or kv(), q, stride, T, max_q, Hq, scale, out, ws, ws_bytes, None)


def test_append_refusals(L):
    nan, inf = float("nan"), float("inf")
    assert L.laq_paged_append(None, A, 6144, 1, 32, A, A, 1e6, 0.0, A, None) == NULL
    for e in (dict(qkv=None), dict(out=None)):
        assert append(L, **e) == NULL
    for e in (dict(stride=48 * 128 - 4), dict(stride=48 * 128 + 2), dict(T=-1),
              dict(T=(1 << 24) + 1), dict(Hq=33), dict(Hq=0), dict(Hq=8 * 65), dict(theta=1.0),
              dict(theta=nan), dict(theta=inf), dict(eps=-1.0), dict(eps=nan)):
        assert append(L, **e) == SHAPE, e
    for e in (dict(qkv=A + 2), dict(out=A + 4), dict(qw=A + 2), dict(kw=A + 4)):
        assert append(L, **e) == ALIGN, e
    assert append(L, T=0) == 0 and append(L, kv(batch=0)) == 0     # nothing to do, no launch


def test_attention_refusals(L):
    nan, inf = float("nan"), float("inf")
    for e in (dict(q=None), dict(out=None), dict(ws=None)):
        assert attend(L, **e) == NULL
    for e in (dict(stride=32 * 128 - 8), dict(stride=32 * 128 + 4), dict(T=-1), dict(max_q=-1),
              dict(Hq=31), dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=inf)):
        assert attend(L, **e) == SHAPE, e
    for e in (dict(q=A + 8), dict(out=A + 8)):
        assert attend(L, **e) == ALIGN, e
    need = L.laq_paged_attention_workspace_bytes(3, 2, 2, 32, 8)
    assert need > 0
    assert attend(L, ws=A + 4) == WS and attend(L, ws_bytes=need - 1) == WS
    for sizes in ((-1, 2, 2, 32, 8), (3, -1, 2, 32, 8), (3, 2, -1, 32, 8), (3, 2, 2, 0, 8),
                  (3, 2, 2, 32, 0), (3, 2, 2, 32, 5), (1 << 30, 2, 2, 32, 8)):
        assert L.laq_paged_attention_workspace_bytes(*sizes) == 0
    assert attend(L, T=0) == 0 and attend(L, kv(batch=0)) == 0 and attend(L, max_q=0) == 0


def test_sample_refusals(L):
    def run(x=A, dt=0, M=2, V=100, stride=100, t=A, k=A, p=A, m=A, u=A, out=A, prob=A):
        return L.laq_sample(x, dt, M, V, stride, t, k, p, m, u, out, prob, None)
    assert run(dt=3) == CONFIG and run(dt=-1) == CONFIG
    for e in (dict(M=-1), dict(M=65536), dict(V=0), dict(V=(1 << 22) + 1, stride=1 << 23),
              dict(stride=99), dict(stride=0)):
        assert run(**e) == SHAPE, e
    for e in (dict(x=None), dict(u=None), dict(out=None)):
        assert run(**e) == NULL, e
    for e in (dict(x=A + 1), dict(x=A + 2, dt=2), dict(t=A + 2), dict(k=A + 1), dict(p=A + 2),
              dict(m=A + 2), dict(u=A + 2), dict(out=A + 2), dict(prob=A + 1)):
        assert run(**e) == ALIGN, e
    assert run(M=0, x=None) == 0


def test_binding_refuses_what_the_abi_cannot_see():
    k = torch.zeros((4, 2, 16, 128), dtype=torch.float16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    good = (k, k.clone(), i32(3, 2), i32(4), i32(3))
    c = _lib.PagedCache(*good)
    for at, bad in ((1, k.bfloat16()), (2, i32(3, 2).long()), (3, i32(3)), (4, i32(3).float()),
                    (2, i32(2, 2)), (3, i32(8)[::2]), (1, torch.zeros((4, 16, 2, 128)).half()
                                                       .transpose(1, 2)),
                    (2, i32(2, 3).t()), (0, k[..., ::2]), (1, k[:2])):
        args = list(good)
        args[at] = bad
        with pytest.raises((TypeError, ValueError)):
            _lib.PagedCache(*args)
    qkv = torch.zeros((3, 8 * 128), dtype=torch.float16)
    for bad in (qkv.bfloat16(), qkv[:, :-1], qkv.t()):
        with pytest.raises((TypeError, ValueError)):
            _lib.laq_paged_append(bad, c, 4, 1e6, 1e-6)
    with pytest.raises((TypeError, ValueError)):
        _lib.laq_paged_append(qkv, c, 4, 1e6, 1e-6, q_norm_w=torch.zeros(128))
    q = torch.zeros((3, 4, 128), dtype=torch.float16)
    for bad in (q.float(), q[..., :64], q.transpose(0, 1)):
        with pytest.raises((TypeError, ValueError)):
            _lib.laq_paged_attention(bad, c, 1, 0.1, torch.zeros(8))
    with pytest.raises(ValueError):
        _lib.laq_paged_attention(q, c, 1, 0.1, torch.zeros(8), out=q[:2].clone())
    x, u = torch.zeros((2, 50)), torch.zeros(2)
    for kw in (dict(logits=x.double()), dict(logits=x.t()), dict(u=u.double()), dict(u=u[:1]),
               dict(top_k=u), dict(temperature=u.half()), dict(top_p=torch.zeros(4)[::2]),
               dict(min_p=torch.zeros(3)), dict(out=u), dict(p_out=u.int())):
        args = dict(logits=x, u=u)
        args.update(kw)
        with pytest.raises((TypeError, ValueError)):
            _lib.laq_sample(**args)


def test_a_broadcast_tensor_is_refused_not_read_past_its_end(L):
    x = torch.zeros((1, 50)).expand(3, 50)
    with pytest.raises(_lib.LaqError):
        _lib.laq_sample(x, torch.zeros(3), stream=type("S", (), {"cuda_stream": 0}))


def test_oracle_attention_by_hand():
    """Two tokens, one head: P = (1, e^2) / (1 + e^2) for the second row; the first sees itself."""
    q = np.zeros((2, 1, 128))
    q[:, 0, 0] = 1.0
    k = np.zeros((3, 1, 1, 128))
    v = np.zeros((3, 1, 1, 128))
    k[2, 0, 0, 0], k[0, 0, 0, 0] = 1.0, 3.0      # tokens 0 and 1 in pages 2 and 0
    v[2, 0, 0, 5], v[0, 0, 0, 5] = 10.0, -20.0
    out, A_ = serving.paged_attention(q, k, v, [[2, 0]], [0, 2], [2], 1.0)
    w = np.exp(2) / (1 + np.exp(2))
    assert np.isclose(out[0, 0, 5], 10) and np.isclose(out[1, 0, 5], 10 * (1 - w) - 20 * w)
    assert np.isclose(A_[1, 0, 5], 10 * (1 - w) + 20 * w)
    out, _ = serving.paged_attention(q, k, v, [[2, 0]], [0, 2], [1], 1.0)   # the first row sees none
    assert not out[0].any() and np.isclose(out[1, 0, 5], 10)


def test_oracle_sampling_by_hand():
    x = np.log(np.array([1.0, 4.0, 4.0, np.e ** -50, 1.0]))
    at, lo, hi, share = serving.sample_bounds(x)
    assert list(at) == [0, 1, 2, 3, 4] and np.allclose(hi[:3], [0.1, 0.5, 0.9])
    at, lo, hi, _ = serving.sample_bounds(x, top_k=3)      # 1, 2, then the first of the ones
    assert list(at) == [0, 1, 2] and np.allclose(lo, [0, 1 / 9, 5 / 9])
    assert list(serving.sample_bounds(x, top_p=0.45)[0]) == [1, 2]
    assert list(serving.sample_bounds(x, top_k=2, top_p=0.45)[0]) == [1]   # of the two that are left
    assert list(serving.sample_bounds(x, min_p=0.2)[0]) == [0, 1, 2, 4]
    assert list(serving.sample_bounds(x, t=0.5, min_p=0.2)[0]) == [1, 2]
    assert list(serving.sample_bounds(x, t=0.0)[0]) == [1]
