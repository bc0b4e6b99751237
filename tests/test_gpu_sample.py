"""laq_sample against its definition in 64 bits and, where the weights are exact, to the token."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import serving  # noqa: E402
from paper_2605_08755_gb300 import _lib  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# A weight's relative error: an argument of at most 40 in fp32 (2^-24 each of the difference and the
# quotient) and expf's two units: 44 * 2^-23; a share of a sum: twice that; u and top_p in steps
# of 2^-24.
EPS = 2 * 44 * 2.0 ** -23 + 2.0 ** -23


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2605_08755_gb300 import build
    build.build()


def sample(x, u, t=None, k=None, p=None, m=None, **kw):
    c = lambda a, d: None if a is None else torch.as_tensor(np.asarray(a, d)).cuda()
    prob = torch.full((x.shape[0],), -1.0, device="cuda")
    out = _lib.laq_sample(x, c(u, np.float32), temperature=c(t, np.float32), top_k=c(k, np.int32),
                          top_p=c(p, np.float32), min_p=c(m, np.float32), p_out=prob, **kw)
    return out.cpu().numpy(), prob.cpu().numpy()


def drawable(x, token, prob, u, t, k, p, m):
    """The token is one that the definition draws for a u within EPS of this one, under a top_p
    target and a min_p within EPS of these."""
    for slack in (0.0, EPS, -EPS):
        for f in (m, m * (1 + EPS), m * (1 - EPS)):
            at, lo, hi, share = serving.sample_bounds(x, t, k, p, f, slack)
            i = np.searchsorted(at, token)
            if i < len(at) and at[i] == token and lo[i] - EPS <= u <= hi[i] + EPS:
                assert abs(prob - share[i]) <= 2 * EPS * share[i] + EPS * 1e-3 or slack or f != m
                return True
    return False


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("M,V", [(1, 1), (3, 2), (5, 31), (4, 1000), (9, 4097), (2, 32003),
                                 (3, 151936), (1, 300001)])
def test_sample(dtype, M, V):
    rng = np.random.default_rng(M * V)
    x = rng.standard_normal((M, V)) * 2
    for r in range(M):
        x[r, rng.integers(0, V, 12)] += 8 + rng.random(12)
    x = torch.from_numpy(x).to(TYPES[dtype]).cuda()
    x64 = x.double().cpu().numpy()
    for settings in range(8):
        t = (0.5 + rng.random(M)).astype(np.float32)
        k = rng.integers(1, 60, M) if settings & 1 else np.zeros(M, int)
        p = (0.3 + 0.69 * rng.random(M)).astype(np.float32) if settings & 2 else np.ones(M, np.float32)
        m = (0.2 * rng.random(M)).astype(np.float32) if settings & 4 else np.zeros(M, np.float32)
        u = rng.random(M).astype(np.float32)
        tok, prob = sample(x, u, t, k, p, m)
        for r in range(M):
            assert drawable(x64[r], tok[r], prob[r], u[r], t[r], k[r], p[r], m[r]), (settings, r)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V", [7, 2048, 40000, 151936])
def test_equal_logits_are_cut_and_drawn_by_index(dtype, V):
    """Weights that are exact: every step to the token."""
    u = np.array([0.0, 0.25, 0.5, 1 - 2.0 ** -24, 0.7], np.float32)
    x = torch.full((5, V), -3.0, dtype=TYPES[dtype], device="cuda")
    u24 = np.floor(u.astype(np.float64) * 2 ** 24).astype(np.int64)

    def first(n):   # of n equal tokens: floor(u * n)
        return np.array([int(a) * n >> 24 for a in u24])
    tok, prob = sample(x, u)
    assert np.array_equal(tok, first(V)) and np.allclose(prob, 1 / V, rtol=1e-6)
    tok, _ = sample(x, u, k=[5] * 5)
    assert np.array_equal(tok, first(5))
    tok, prob = sample(x, u, p=[0.5] * 5)
    assert np.array_equal(tok, first(-(-V // 2)))
    tok, _ = sample(x, u, p=[0.0] * 5)
    assert np.array_equal(tok, np.zeros(5))
    tok, _ = sample(x, u, m=[1.0] * 5)
    assert np.array_equal(tok, first(V))
    tok, _ = sample(x, u, k=[6, 6, 6, 6, 6], p=[0.5] * 5, m=[0.5] * 5)
    assert np.array_equal(tok, first(3))
    # one above the rest, at the end: first in the order, last by the index
    x[:, V - 1] = 2.0
    tok, _ = sample(x, u, k=[1] * 5)
    assert np.array_equal(tok, np.full(5, V - 1))
    tok, _ = sample(x, [0.999] * 5, t=[1e6] * 5, k=[4] * 5)
    assert np.array_equal(tok, np.full(5, V - 1))
    tok, _ = sample(x, [0.0] * 5, t=[1e6] * 5, k=[4] * 5)
    assert np.array_equal(tok, np.zeros(5))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V", [5, 3000, 151936])
def test_greedy_masked_and_non_finite(dtype, V):
    nan, inf = float("nan"), float("inf")
    x = torch.randn((8, V), device="cuda").to(TYPES[dtype])
    x[0, 2] = 9
    x[0, 4] = 9
    x[1, :] = -inf
    x[1, 3] = -60000.0 if dtype != "bf16" else -3e38
    x[2, :] = nan
    x[2, 1] = 0.5
    x[3, :] = -inf
    x[4, :] = nan
    x[5, 3] = inf
    x[6, :] = torch.finfo(TYPES[dtype]).min
    x[6, 4] = -1.0
    x[7, :] = 0.0
    x[7, 1] = -0.0
    for t in (0.0, -1.0, nan):
        tok, prob = sample(x, [0.9] * 8, t=[t] * 8)
        assert list(tok[[0, 1, 2, 3, 4, 5, 6, 7]]) == [2, 3, 1, 0, 0, 3, 4, 0]
        assert list(prob) == [1, 1, 1, 0, 0, 1, 1, 1]
    for kw in (dict(), dict(k=[3] * 8), dict(p=[0.9] * 8), dict(m=[0.1] * 8)):
        tok, _ = sample(x, [0.5] * 8, **kw)
        assert list(tok[1:7]) == [3, 1, 0, 0, 3, 4]
    # the two zeros are one value: the first two by index
    tok, _ = sample(x[7:], [0.99], k=[2])
    assert tok[0] == 1


def test_settings_outside_their_ranges():
    x = torch.randn((6, 500), device="cuda")
    nan = float("nan")
    u = [0.3, 0.3, 0.3, 1.0, -1.0, nan]
    base, _ = sample(x, [0.3, 0.3, 0.3, 1 - 2.0 ** -24, 0.0, 0.0])
    got, _ = sample(x, u, k=[-1, 0, 1 << 30, 500, 501, 0], p=[1.0, 2.0, nan, 1.0, 1.0, 7.0],
                    m=[-1.0, nan, 0.0, 0.0, 0.0, 0.0])
    assert np.array_equal(base, got)


def test_strided_rows_and_another_batch():
    """A row's token does not depend on its place, its alignment or the rows beside it."""
    V = 20001
    x = (3 * torch.randn((40, V + 3), device="cuda")).half()
    u = np.random.default_rng(3).random(40).astype(np.float32)
    kw = dict(t=[0.8] * 40, k=[0, 50] * 20, p=[0.95, 0.9, 1.0, 0.8] * 10, m=[0.01] * 40)
    whole, prob = sample(x[:, 1:V + 1], u, **kw)
    dense, prob2 = sample(x[:, 1:V + 1].contiguous(), u, **kw)
    assert np.array_equal(whole, dense) and np.array_equal(prob, prob2)
    for r in (0, 7, 39):
        one, _ = sample(x[r:r + 1, 1:V + 1], u[r:r + 1], **{k: a[r:r + 1] for k, a in kw.items()})
        assert one[0] == whole[r]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    dev = torch.from_numpy(u).cuda()
    torch.cuda.synchronize()
    a = _lib.laq_sample(x[:, :V], dev, stream=s)
    s.synchronize()
    assert torch.equal(a, _lib.laq_sample(x[:, :V], dev))


def defined(x, u, t, k, p, m):
    """The definition in whole numbers, step by step, with the device's expf and division."""
    x = x.float()
    x = torch.where(torch.isnan(x), torch.full_like(x, float("-inf")), x)
    top = x.amax(1, keepdim=True)
    c = lambda a, d: torch.as_tensor(np.asarray(a, d)).cuda()[:, None]
    t, k, p, m, u = c(t, np.float32), c(k, np.int64), c(p, np.float32), c(m, np.float32), c(u, np.float32)
    w = (torch.where(x == top, 1.0, torch.exp((x - top) / t)) * 2.0 ** 40).long()
    by = torch.sort(x, dim=1, descending=True, stable=True).indices
    ws, rank = w.gather(1, by), torch.arange(x.shape[1], device="cuda")[None]

    def part(mass, f):
        f = (f * 2.0 ** 24).long()
        return (mass >> 24) * f + (((mass & 0xffffff) * f) >> 24)
    keep = (k <= 0) | (rank < k)
    ws = ws * keep
    cum = ws.cumsum(1)
    keep &= (p >= 1) | (rank == 0) | (cum - ws < part(cum[:, -1:], p))
    keep &= (ws >= (m * 2.0 ** 40).long()) | (rank == 0)
    w = w * torch.zeros_like(keep).scatter_(1, by, keep)
    cum = w.cumsum(1)
    tok = (cum <= part(cum[:, -1:], u)).sum(1)
    return tok.cpu().numpy(), (w.gather(1, tok[:, None]).float() / cum[:, -1:].float())[:, 0].cpu().numpy()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("M,V,stretch", [(70, 3001, 1.0), (40, 50000, 0.2), (12, 151936, 2.0),
                                         (3, 300001, 1.0), (2, 1 << 22, 1.0), (9, 100000, 1e-3)])
def test_every_step_is_exact(dtype, M, V, stretch):
    """To the token and the bit of its probability: rows whose cut lies deep in the body of the
    distribution, many logits of one value, cuts of thousands of tokens, nothing cut."""
    rng = np.random.default_rng(V)
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (stretch * torch.randn((M, V), generator=g, device="cuda")).to(TYPES[dtype])
    x[::3, :: 7] = float("-inf")
    x[1::3, 5] = stretch * 9
    for settings in range(8):
        t = np.exp(rng.uniform(-1.5, 1.5, M)).astype(np.float32)
        t[0] = (1e-30, 1e30, 1.0, 3e38, 1e-38, 2.0 ** -100, 2.0 ** 100, 0.99999994)[settings]
        k = rng.integers(2, [V + 5, 80][settings % 2], M) if settings & 1 or settings == 6 \
            else np.zeros(M, int)
        p = rng.random(M).astype(np.float32) if settings & 2 else np.ones(M, np.float32)
        m = (0.1 * rng.random(M) ** 4).astype(np.float32) if settings & 4 else np.zeros(M, np.float32)
        u = rng.random(M).astype(np.float32)
        u[-1] = 1 - 2.0 ** -24
        tok, prob = sample(x, u, t, k, p, m)
        want, share = defined(x, u, t, k, p, m)
        assert np.array_equal(tok, want), settings
        assert np.array_equal(prob, share), settings
