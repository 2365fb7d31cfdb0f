"""The draw of the next token against its definition in 64 bits and whole numbers, row by row, and what the call refuses.

Weights are multiples of 2^-bits, so all sums are exact and tokens have to be equal.  The two sides' exponentials differ by a few units
of 2^-53 of a weight at most, which moves a sum of 10^5 weights by less than 10^-12 of it: a draw differs with that
probability times the number of tokens per unit of probability at the place, 10^-7 at worst for a row.  The logarithm of a probability is that
of an exact share: fp32's rounding (2^-24 of it) and 10^-11 of the sum's.
"""
import math

import numpy as np
import pytest
import torch

from paper_2211_10280_b200 import binding as B
from paper_2211_10280_b200 import build as libbuild

gpu = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    libbuild.build()


def _sample(*args, **kw):
    from paper_2211_10280_b200 import sampling

    return sampling.sample(*args, **kw)


def _draw(x, u, T, k, p, min_p):
    """(token, logprob) of one row of float64 logits, by the definition."""
    V = len(x)
    x = np.where(np.isnan(x), -np.inf, x)
    largest = x.max()
    if largest == -np.inf:
        return -1, -INF
    if not T > 0:
        return int(np.argmax(x)), 0.0
    bits = min(46, 62 - int(V - 1).bit_length())
    gap = np.where(x == largest, 0.0, -np.inf) if largest == np.inf else x - largest
    order = np.argsort(-x, kind="stable")
    if 0 < k < V:
        order = order[:k]
    mass = np.rint(np.exp(gap[order] / T) * 2.0 ** bits).astype(np.int64)
    if p < 1:
        before = np.cumsum(mass) - mass
        front = before.astype(np.float64) < p * float(mass.sum())
        front[0] = True
        order, mass = order[front], mass[front]
    if min_p > 0:
        held = gap[order] >= min(0.0, T * math.log(min_p))
        order, mass = order[held], mass[held]
    at = np.argsort(order)
    running = np.cumsum(mass[at])
    total = int(running[-1])
    target = min(max(int(u * float(total)), 0), total - 1)
    token = int(order[at][np.searchsorted(running, target, side="right")])
    return token, gap[token] / T - math.log(total * 2.0 ** -bits)


def _check(logits, u, T=1.0, k=0, p=1.0, min_p=0.0):
    n = logits.shape[0]
    got, logprob = _sample(logits, u, T, k, p, min_p, logprobs=True)
    assert torch.equal(got, _sample(logits, u, T, k, p, min_p))

    def column(x):
        return x.double().cpu().numpy() if torch.is_tensor(x) else np.full(n, np.float32(x), np.float64)

    x, us = logits.double().cpu().numpy(), u.double().cpu().numpy()
    Ts, ks, ps, ms = column(T), column(k), column(p), column(min_p)
    want = [_draw(x[i], us[i], Ts[i], int(ks[i]), ps[i], ms[i]) for i in range(n)]
    tokens = np.array([w[0] for w in want])
    assert (got.cpu().numpy() == tokens).all(), np.nonzero(got.cpu().numpy() != tokens)[0][:5]
    lp = np.array([w[1] for w in want])
    have = logprob.double().cpu().numpy()
    none = tokens < 0
    assert (have[none] == -INF).all()
    assert (np.abs(have[~none] - lp[~none]) <= np.abs(lp[~none]) * 2.0 ** -24 + 1e-10).all()
    return got


def _logits(n, V, dtype=F32, std=2.5, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, V, generator=g) * std
    x.scatter_add_(1, torch.randint(0, V, (n, min(V, 8)), generator=g), torch.rand(n, min(V, 8), generator=g) * 8)
    return x.to(dtype).cuda()


def _uniform(n, seed=1):
    return torch.rand(n, generator=torch.Generator().manual_seed(seed)).cuda()


SETTINGS = [dict(), dict(T=0.7), dict(k=1), dict(k=40), dict(p=0.9), dict(min_p=0.05), dict(T=0.8, k=50, p=0.95), dict(T=1.5, k=300, p=0.6, min_p=0.01),
            dict(T=0.0), dict(p=0.0), dict(min_p=1.0), dict(T=30.0, p=0.99), dict(T=0.01, p=0.999)]
SIZES = [(3, 1), (5, 2), (4, 17), (7, 1000), (2, 4096), (3, 4099), (2, 50_000), (1, 100_003), (300, 2000), (40, 33_333)]


@gpu
@pytest.mark.parametrize("n,V", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_sample(n, V, dtype):
    logits = _logits(n, V, dtype, seed=V)
    for i, s in enumerate(SETTINGS):
        if i % 3 and n * V > 10 ** 6:
            continue
        _check(logits, _uniform(n, i), **s)


@gpu
@pytest.mark.parametrize("V", [30, 5000, 80_000])
def test_every_row_has_settings_of_its_own(V):
    n = 96
    r = np.random.default_rng(V)

    def pick(values, dtype):
        return torch.from_numpy(r.choice(values, n)).to(dtype).cuda()

    logits = _logits(n, V, seed=1)
    logits[:, r.random(V) < 0.3] = -INF
    _check(logits, _uniform(n), pick([0.0, 0.5, 1.0, 2.0, -1.0, math.nan], F32), pick([-3, 0, 1, 7, 60, 10 ** 6], torch.int32),
           pick([0.1, 0.5, 0.9, 0.999, 1.0, 3.0], F32), pick([0.0, -1.0, 0.01, 0.3, 1.0], F32))


@gpu
@pytest.mark.parametrize("dtype", [F32, F16])
def test_ties_go_to_the_lowest_ids(dtype):
    for V in (10, 3000, 70_001):
        n = 30
        logits = torch.randint(0, 4, (n, V), generator=torch.Generator().manual_seed(V)).to(dtype).cuda()       # thousands of ties
        for k in (1, 3, 100, 2000):
            _check(logits, _uniform(n, k), k=k)
            _check(logits, _uniform(n, k), k=k, p=0.5)
        for p in (0.01, 0.3, 0.77, 0.95):
            _check(logits, _uniform(n, 5), p=p)
        same = torch.full((2, V), -7.0, dtype=dtype, device="cuda")
        ends = torch.tensor([0.0, 1 - 2.0 ** -24], device="cuda")
        assert _check(same, ends).tolist() == [0, V - 1]
        assert _check(same, ends, k=5).tolist() == [0, 4]
        assert _check(same, ends, p=0.5).tolist() == [0, (V + 1) // 2 - 1]
        assert _check(same, ends, T=0.0).tolist() == [0, 0]
    zeros = torch.tensor([[-0.0, 0.0, -0.0, 0.0]], device="cuda")
    assert _check(zeros, torch.zeros(1, device="cuda"), k=1).tolist() == [0]


@gpu
@pytest.mark.parametrize("V", [40, 9000])
def test_masks_infinities_and_nan(V):
    n = 12
    x = _logits(n, V, seed=2)
    low = torch.finfo(F32).min
    x[0] = -INF                              # nothing is left
    x[1] = float("nan")
    x[2] = -INF
    x[2, V - 3] = -80.0                      # one token
    x[3, ::2] = low
    x[4] = low                               # masked by the lowest value throughout: as likely as one another
    x[5, 7], x[5, 9] = INF, INF              # only these have weight
    x[6, 3] = float("nan")
    x[7] *= 1e30
    x[8] *= 1e-30
    x[9] = torch.linspace(-3e38, 3e38, V)
    x[10, :V // 2] = -INF
    x[11] = x[11].abs() * -1e4
    for s in SETTINGS:
        got = _check(x, _uniform(n, 3), **s)
        assert got[0] == -1 and got[1] == -1 and got[2] == V - 3 and got[5].item() in (7, 9)
    half = x.clamp(-6e4, 6e4).half()
    half[x == -INF] = -INF
    for s in SETTINGS:
        _check(half, _uniform(n, 4), **s)


@gpu
def test_random_numbers_at_the_ends_and_outside():
    logits = _logits(8, 1000, seed=3)
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, INF, -INF, float("nan")], device="cuda")
    inside = torch.tensor([0.0, 1 - 2.0 ** -24, 1 - 2.0 ** -24, 1 - 2.0 ** -24, 0, 1 - 2.0 ** -24, 0, 0], device="cuda")
    a, b = _sample(logits, u, 0.9), _sample(logits, inside, 0.9)
    assert a[0] == b[0] and a[4] == b[4] and a[6:].tolist() == b[6:].tolist() and ((a >= 0) & (a < 1000)).all()


@gpu
def test_strided_rows_and_rows_between_two_vectors():
    wide = _logits(6, 5003, BF16, seed=4)
    u = _uniform(6)
    for off in (0, 1, 3, 8):
        x = wide[:, off:off + 4990]
        want = _check(x, u, 0.9, 200, 0.9)
        assert torch.equal(_sample(x.contiguous(), u, 0.9, 200, 0.9), want)
    by_token = wide.t().contiguous().t()
    assert torch.equal(_sample(by_token, u, 0.9, 0, 0.9), _sample(wide, u, 0.9, 0, 0.9))
    one = wide[:1].expand(6, 5003)
    assert torch.equal(_sample(one, u), _sample(one.contiguous(), u))
    out = torch.zeros(6, dtype=torch.int64, device="cuda")
    assert _sample(wide, u, out=out) is out and torch.equal(out, _sample(wide, u))
    assert _sample(wide[:0], u[:0]).shape == (0,)


@gpu
@pytest.mark.parametrize("V,dtype", [(2 ** 20, F32), (2 ** 20, BF16), (2 ** 20 - 5, F16)])
def test_the_largest_vocabularies(V, dtype):
    """Slices that do not fit into shared memory are read again."""
    logits = _logits(3, V, dtype, std=1.5, seed=5)
    for s in (dict(), dict(p=0.95), dict(k=1000, p=0.7), dict(T=0.0), dict(T=0.9, min_p=0.02)):
        _check(logits, _uniform(3, 7), **s)


@gpu
@pytest.mark.parametrize("n,V,dtype", [(3, 60_000, F32), (2, 40_000, BF16), (160, 20_000, F32), (150, 30_000, F16)])
def test_fronts_that_do_not_fit_into_one_block(n, V, dtype):
    """Flat rows, of which tens of thousands of tokens are kept: the border is looked for in the whole row, by a cluster or by a block."""
    x = _logits(n, V, dtype, std=0.4, seed=V)
    x[0, ::3] = -INF
    for s in (dict(p=0.93), dict(k=15_000), dict(k=15_000, p=0.8), dict(T=20.0, p=0.5, min_p=0.97), dict(k=9000, min_p=0.2)):
        _check(x, _uniform(n, 3), **s)


@gpu
@pytest.mark.parametrize("V", [8190, 8192, 8194, 4096, 4097, 16_400])
def test_sizes_at_which_the_search_changes_its_way(V):
    for dtype in (F32, BF16):
        x = _logits(3, V, dtype, std=0.3, seed=V)
        for s in (dict(p=0.999), dict(k=V - 1), dict(k=V), dict(k=V + 1, p=0.99), dict(k=4096), dict(k=8192, p=0.9999)):
            _check(x, _uniform(3, 5), **s)


@gpu
def test_rows_beyond_32_bits():
    V, n = 2 ** 20, 2100                    # 2.2 G logits
    logits = torch.full((n, V), -30.0, dtype=F16, device="cuda")
    logits[n - 1] = _logits(1, V, F16)[0]
    logits[5, 77] = 9.0
    u = _uniform(n)
    got = _sample(logits, u, 1.0, 3)
    assert got[5].item() == _draw(logits[5].double().cpu().numpy(), u[5].item(), 1.0, 3, 1.0, 0.0)[0]
    assert got[n - 1].item() == _draw(logits[n - 1].double().cpu().numpy(), u[n - 1].item(), 1.0, 3, 1.0, 0.0)[0]
    assert (got[6:n - 1] < 3).all()


@gpu
def test_draws_follow_the_probabilities():
    V, n = 6, 200_000
    x = torch.tensor([1.0, 0.0, -1.0, 2.0, -INF, 0.5], device="cuda")
    got = _sample(x.expand(n, V), _uniform(n, 9), 0.8)
    share = torch.softmax(x.double() / 0.8, 0).cpu().numpy()
    seen = np.bincount(got.cpu().numpy(), minlength=V) / n
    assert (np.abs(seen - share) <= 6 * np.sqrt(share * (1 - share) / n)).all()


@gpu
def test_draws_on_streams_and_captured():
    logits, u = _logits(20, 30_000, seed=6), _uniform(20)
    want = _sample(logits, u, 0.9, 100, 0.9)
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(_sample(logits, u, 0.9, 100, 0.9))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _sample(logits, u, 0.9, 100, 0.9)
    u.copy_(_uniform(20, 8))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, _sample(logits, u, 0.9, 100, 0.9))


@pytest.mark.parametrize("change,word", [
    (dict(n=2 ** 24 + 1), "n must"), (dict(uniform=None), "NULL"), (dict(token=None), "NULL"), (dict(uniform=4098), "aligned"), (dict(token=4100), "aligned"),
    (dict(logprob=4097), "aligned"), (dict(temperature=math.nan), "temperature"), (dict(temperature=INF), "temperature"), (dict(top_p=math.nan), "top_p"),
    (dict(min_p=math.nan), "min_p"), (dict(top_ks=4098), "setting"), (dict(temperatures=4098), "setting")])
def test_sample_refuses(change, word):
    h = B.Draw(uniform=4096, token=4096, n=3, temperature=1.0, top_p=1.0)
    for f, x in change.items():
        setattr(h, f, x)
    assert B.lib().tensair_sample(h, B.Rows(data=4096, stride=8, d=8, type=B.FLOAT32), None) == B.EINVAL
    assert word in B.lib().tensair_last_error(None).decode()


def test_sample_refuses_its_logits():
    h = B.Draw(uniform=4096, token=4096, n=3, temperature=1.0, top_p=1.0)
    for rows in (None, B.Rows(data=None, stride=8, d=8), B.Rows(data=4098, stride=8, d=8), B.Rows(data=4096, stride=7, d=8), B.Rows(data=4096, stride=8, d=0),
                 B.Rows(data=4096, stride=2 ** 21, d=2 ** 20 + 1), B.Rows(data=4096, stride=8, d=8, type=3)):
        assert B.lib().tensair_sample(h, rows, None) == B.EINVAL
        assert "logits" in B.lib().tensair_last_error(None).decode()
    assert B.lib().tensair_sample(None, B.Rows(data=4096, stride=8, d=8), None) == B.EINVAL
    h.n = 0
    assert B.lib().tensair_sample(h, B.Rows(data=None, stride=8, d=8), None) == B.OK


@gpu
def test_the_python_call_refuses():
    x, u = _logits(4, 50), _uniform(4)
    for i, call in enumerate([
            lambda: _sample(x.cpu(), u), lambda: _sample(x, u.cpu()), lambda: _sample(x[0], u), lambda: _sample(x.double(), u), lambda: _sample(x, u[:3]),
            lambda: _sample(x, u.double()), lambda: _sample(x, u, temperature=-1.0), lambda: _sample(x, u, temperature=math.nan), lambda: _sample(x, u, top_k=-1),
            lambda: _sample(x, u, top_p=math.nan), lambda: _sample(x, u, min_p=1.5), lambda: _sample(x, u, top_k=u), lambda: _sample(x, u, temperature=u[:2]),
            lambda: _sample(x, u, out=u), lambda: _sample(x[:, :0], u)]):
        with pytest.raises((ValueError, B.TensairError)):
            call()
            pytest.fail(f"call {i} was not refused")
