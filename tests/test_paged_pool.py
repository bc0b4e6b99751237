"""Page bookkeeping of the serving step (no GPU): random requests that grow and end."""
import random

import pytest

torch = pytest.importorskip("torch")
from paper_2605_08755_gb300.paged_step import PagedPool  # noqa: E402


@pytest.mark.parametrize("page_size,seed", [(8, 0), (16, 1), (64, 2)])
def test_pages_are_held_once_and_cover_the_tokens(page_size, seed):
    rng = random.Random(seed)
    requests, pages, most = 5, 23, 9
    pool = PagedPool(requests, pages, page_size, most, "cpu")
    length = [0] * requests
    for _ in range(200):
        if rng.random() < 0.15:
            b = rng.randrange(requests)
            pool.release(b)
            length[b] = 0
        counts = [rng.choice([0, 1, rng.randrange(3 * page_size)]) for _ in range(requests)]
        before = ([list(h) for h in pool.held], pool.table.clone(), list(pool.free))
        want = [-(-(n + c) // page_size) for n, c in zip(length, counts)]
        if max(want) > most or sum(want) > pages:  # refused, and nothing has changed
            with pytest.raises(ValueError):
                pool.extend(counts)
            assert (pool.held, pool.free) == (before[0], before[2])
            assert torch.equal(pool.table, before[1]) and pool.length == length
            continue
        pool.extend(counts)
        length = [n + c for n, c in zip(length, counts)]
        assert pool.kv_len.tolist() == length
        assert pool.q_start.tolist() == [sum(counts[:i]) for i in range(requests + 1)]
        held = []
        for b, n in enumerate(length):
            row = pool.table[b].tolist()
            used = -(-n // page_size)
            assert all(0 <= x < pages for x in row[:used]) and row[used:] == [-1] * (most - used)
            assert row[:len(before[0][b])] == before[1][b].tolist()[:len(before[0][b])]
            held += row[:used]
        assert len(set(held)) == len(held)
        assert sorted(held + pool.free) == list(range(pages))
