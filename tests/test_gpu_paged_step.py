"""The serving step: against the decode step on the same weights and caches, chunks against whole
prompts, requests that wait, and pages handed on."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2605_08755_gb300.decode_step import DecodeStep  # noqa: E402
from paper_2605_08755_gb300.paged_step import PagedPool, PagedStep  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def weights():
    from paper_2605_08755_gb300 import build
    build.build()
    return DecodeStep(layers=2, M=3, context=200, vocab=4096)


def greedy(B):
    return dict(temperature=torch.zeros((B,), device="cuda")), torch.zeros((B,), device="cuda")


def close(a, b):
    """fp16 activations through two layers whose attention rounds its probabilities once: a few fp16
    steps of the logits' size."""
    a, b = a.double().cpu().numpy(), b.double().cpu().numpy()
    assert np.abs(a - b).max() <= 2e-2 * np.abs(b).max()


def test_single_tokens_match_the_decode_step(weights):
    ds = weights
    ds.run()
    torch.cuda.synchronize()
    st = PagedStep(ds, 3, 8, 8, pages=24, page_size=32)
    st.pool.extend([199, 199, 199])
    for l in range(2):
        c = st.caches[l]
        for b in range(3):
            for p in range(199):
                page = st.pool.held[b][p // 32]
                c.k[page, :, p % 32] = ds.kc[l][b, :, p]
                c.v[page, :, p % 32] = ds.vc[l][b, :, p]
    kw, u = greedy(3)
    nxt = st.run(ds.tokens, [1, 1, 1], u, **kw)
    close(st.logits, ds.logits)
    top = ds.logits.float().topk(2, 1).values
    for b in range(3):   # the same token wherever the first is clear of the second
        if top[b, 0] - top[b, 1] > 4e-2 * ds.logits.abs().max():
            assert int(nxt[b]) == int(ds.next[b])
    # the new keys and values lie where the tables say
    for b in range(3):
        page = st.pool.held[b][199 // 32]
        assert torch.equal(st.caches[0].v[page, :, 199 % 32], ds.vc[0][b, :, 199])


def test_chunks_match_a_whole_prompt(weights):
    ds = weights
    g = torch.Generator(device="cuda").manual_seed(3)
    prompt = torch.randint(0, ds.V, (2, 90), generator=g, device="cuda", dtype=torch.int32)
    kw, u = greedy(2)
    whole = PagedStep(ds, 2, 180, 90, pages=8, page_size=32)
    whole.run(prompt.reshape(-1), [90, 90], u, **kw)
    parts = PagedStep(ds, 2, 180, 90, pages=30, page_size=8)
    at = [0, 0]
    for counts in ([50, 1], [0, 70], [39, 18], [1, 1]):
        rows = torch.cat([prompt[b, at[b]:at[b] + n] for b, n in enumerate(counts)])
        parts.run(rows, counts, u, **kw)
        at = [a + n for a, n in zip(at, counts)]
    assert at == [90, 90]
    close(parts.logits, whole.logits)


def test_a_waiting_request_and_released_pages(weights):
    ds = weights
    kw, u = greedy(2)
    st = PagedStep(ds, 2, 40, 40, pages=2, page_size=32)
    prompt = torch.arange(30, dtype=torch.int32, device="cuda")
    st.run(prompt, [30, 0], u, **kw)
    first = st.logits[0].clone()
    st.pool.release(0)
    st.run(prompt, [0, 30], u, **kw)
    assert torch.equal(st.logits[1], first)      # the same sums on other rows and pages
    with pytest.raises(ValueError):
        st.run(prompt, [30, 1], u, **kw)


def test_pool_tables():
    p = PagedPool(2, 4, 16, 3, "cpu")
    p.extend([17, 0])
    assert p.table.tolist()[0][:2] == [0, 1] and p.table[0, 2] == -1 and p.kv_len.tolist() == [17, 0]
    assert p.q_start.tolist() == [0, 17, 17]
    p.extend([1, 16])
    assert p.held == [[0, 1], [2]] and p.kv_len.tolist() == [18, 16]
    with pytest.raises(ValueError):
        p.extend([0, 40])
