"""Layer norm, dropout and the gated linear recurrence against plain implementations in 64 bits, forwards and backwards, and what
their calls refuse.

Tolerances follow from fp32 arithmetic, u = 2^-24 the largest relative error of one rounding.  A sum of k terms by a tree of depth q is off
by at most q u times the sum of the magnitudes; expf is good to 2 u, 1 / (1 + e) by the fast quotient to 4 u, so 1 - f is good
to 8 u with the roundings between.  An output type with f fraction bits adds 2^-(f+1) of the value (half the smallest subnormal at least).
"""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2211_10280_b200 import binding as B
from paper_2211_10280_b200 import build as libbuild

gpu = pytest.mark.gpu
U = 2.0 ** -24
LAST = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25)}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _built():
    libbuild.build()


def _ops():
    from paper_2211_10280_b200 import layers

    return layers


def _rand(shape, dtype=F32, std=1.0, mean=0.0, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).cuda()


def _close(got, want, slack):
    """|got - want| <= slack + the output type's rounding"""
    rel, least = LAST[got.dtype]
    assert got.shape == want.shape
    assert not torch.isnan(got).any()
    excess = (got.double() - want).abs() - (slack + (want.abs() + slack) * rel + least)
    assert got.numel() == 0 or excess.max().item() <= 0, (excess.max().item(), (got.double() - want).abs().max().item())


# ---------------------------------------------------------------- layer norm
EPS = 1e-5


def _norm(x, w, b):
    """(y, its fp32 error, mean, 1 / sqrt, the normed rows c, the error of c)"""
    x, w = x.double(), w.double()
    d = x.shape[1]
    depth = 64 + d / 1024      # terms that a thread adds up, and the levels that join the threads
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    r = (var + EPS) ** -0.5
    c = (x - mean) * r
    off = (depth + 2) * U * x.abs().amax(1, keepdim=True)          # of x - mean
    rel = off * r + (depth / 2 + 4) * U                            # of 1 / sqrt, relative
    ec = off * r + c.abs() * (rel + 2 * U)
    b = torch.zeros_like(w) if b is None else b.double()
    y = c * w + b
    return y, ec * w.abs() + 2 * U * ((c * w).abs() + b.abs()) * 1.01, mean, r, c, ec, rel


SHAPES = [(1, 1), (3, 2), (1, 512), (5, 7), (70, 64), (33, 72), (9, 300), (1021, 301), (40, 1000), (17, 1024), (12, 2048), (5, 8192), (3, 8196), (3, 16_384), (4, 20_011), (2, 70_000)]


@gpu
@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("x_type,y_type,p_type", [(F32, F32, F32), (BF16, BF16, F32), (F16, F16, F16), (F32, BF16, BF16), (F32, F16, F32), (BF16, BF16, BF16)])
def test_layer_norm_and_its_gradient(n, d, x_type, y_type, p_type):
    L = _ops()
    x = _rand((n, d), x_type, 1.5, 0.4, seed=n + d)
    w, b = _rand((d,), p_type, 0.2, 1.0, seed=1), _rand((d,), p_type, 0.2, seed=2)
    bias = b if (n + d) % 3 else None
    y, mean, rstd = L.layer_norm(x, w, bias, eps=EPS, dtype=y_type, stats=True)
    want, slack, m, r, c, ec, rel = _norm(x, w, bias)
    assert y.dtype == y_type
    _close(y, want, slack)
    _close(mean, m[:, 0], (64 + d / 1024) * U * x.double().abs().amax(1))
    _close(rstd, r[:, 0], (r * rel)[:, 0])
    assert torch.equal(y, L.layer_norm(x, w, bias, eps=EPS, dtype=y_type))
    # backwards
    dy = _rand((n, d), y_type, 0.3, seed=3)
    dx, dw, db = L.layer_norm_gradient(dy, x, w, mean, rstd, bias=bias is not None)
    g = dy.double() * w.double()
    depth = 66 + d / 1024
    mg, mgc = g.mean(1, keepdim=True), (g * c).mean(1, keepdim=True)
    e_mg = depth * U * g.abs().mean(1, keepdim=True)
    e_mgc = depth * U * (g * c).abs().mean(1, keepdim=True) + (g.abs() * ec).mean(1, keepdim=True)
    want = r * (g - mg - c * mgc)
    slack = r * (4 * U * (g.abs() + mg.abs() + (c * mgc).abs()) + e_mg + c.abs() * e_mgc + ec * mgc.abs()) + want.abs() * rel
    assert dx.dtype == x_type
    _close(dx, want, slack * 1.01)
    rows = n + 64
    _close(dw, (dy.double() * c).sum(0), rows * U * (dy.double() * c).abs().sum(0) + (dy.double().abs() * ec).sum(0) * 1.01)
    if bias is None:
        assert db is None
    else:
        _close(db, dy.double().sum(0), rows * U * dy.double().abs().sum(0))
    again = L.layer_norm_gradient(dy, x, w, mean, rstd)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@gpu
@pytest.mark.parametrize("n", [8, 9, 2367, 2368, 2369, 9000])
@pytest.mark.parametrize("d", [24, 512])
def test_weight_gradient_where_the_rows_go_round(n, d):
    L = _ops()
    x, dy = _rand((n, d), BF16, seed=n), torch.randint(-3, 4, (n, d), device="cuda").to(BF16)
    w = _rand((d,), F32, seed=1)
    _, mean, rstd = L.layer_norm(x, w, stats=True)
    dx, dw, db = L.layer_norm_gradient(dy, x, w, mean, rstd)
    assert torch.equal(db.double(), dy.double().sum(0))          # whole numbers: exact in any order
    _, _, _, _, c, ec, _ = _norm(x, w, None)
    _close(dw, (dy.double() * c).sum(0), (n + 64) * U * (dy.double() * c).abs().sum(0) + (dy.double().abs() * ec).sum(0))


@gpu
def test_layer_norm_of_strided_rows_shapes_and_parts():
    L = _ops()
    wide = _rand((2, 30, 96), BF16)
    w = _rand((41,), F32, 0.1, 1.0)
    for off in (0, 1, 8):                 # rows that begin between two vectors
        x = wide[:, :, off:off + 41]
        want, slack, *_ = _norm(x.reshape(-1, 41), w, None)
        _close(L.layer_norm(x, w), want.view(2, 30, 41), slack.view(2, 30, 41))
        rows = wide[0, :, off:off + 41]
        out = torch.zeros(30, 64, dtype=BF16, device="cuda")
        L.layer_norm(rows, w, out=out[:, 3:44])
        assert torch.equal(out[:, 3:44], L.layer_norm(rows.contiguous(), w)) and not out[:, 44:].any() and not out[:, :3].any()
    big = torch.full((100,), 3.0, device="cuda")
    assert not L.layer_norm(big[None], torch.ones(100, device="cuda")).any()          # a row of one value
    x = _rand((4, 64))
    x[1, 5], x[2, 7] = float("nan"), float("inf")
    y = L.layer_norm(x, torch.ones(64, device="cuda"))
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).any() and torch.isfinite(y[[0, 3]]).all()
    assert L.layer_norm(x[:0], torch.ones(64, device="cuda")).shape == (0, 64)
    dx, dw, db = L.layer_norm_gradient(x[:0], x[:0], torch.ones(64, device="cuda"), x[:0, 0], x[:0, 0])
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    dx, dw, db = L.layer_norm_gradient(x, x, torch.ones(64, device="cuda"), x[:, 0].contiguous(), x[:, 0].contiguous(), params=False)
    assert dw is None and db is None


@gpu
def test_layer_norm_beyond_32_bits():
    n, d = 4_200_000, 512          # 2.15 G elements
    x = torch.zeros(n, d, dtype=BF16, device="cuda")
    x[-3:] = _rand((3, d), BF16)
    w = _rand((d,), F32, 0.1, 1.0)
    y, mean, rstd = _ops().layer_norm(x, w, stats=True)
    want, slack, *_ = _norm(x[-3:], w, None)
    _close(y[-3:], want, slack)
    assert not y[:1000].any()
    del y
    dy = torch.zeros_like(x)
    dy[-3:] = _rand((3, d), BF16, seed=1)
    dx, dw, db = _ops().layer_norm_gradient(dy, x, w, mean, rstd)
    _close(db, dy[-3:].double().sum(0), 8 * U * dy[-3:].double().abs().sum(0))
    tail = _ops().layer_norm_gradient(dy[-3:], x[-3:], w, mean[-3:].contiguous(), rstd[-3:].contiguous())
    assert torch.equal(tail[0], dx[-3:]) and not dx[:1000].any()


@gpu
def test_layer_norm_has_the_gradient_that_differences_give():
    L = _ops()
    x, w, b, dy = _rand((5, 12), seed=1), _rand((12,), seed=2), _rand((12,), seed=3), _rand((5, 12), seed=4)
    ins = [t.clone().requires_grad_() for t in (x, w, b)]
    got = torch.autograd.grad((L.layer_norm(*ins) * dy).sum(), ins)

    def value(x, w, b):
        x = x.double()
        c = x - x.mean(1, keepdim=True)
        return ((c / ((c ** 2).mean(1, keepdim=True) + 1e-5) ** 0.5 * w + b) * dy.double()).sum()

    for i, t in enumerate((x, w, b)):
        flat = got[i].reshape(-1)
        for j in range(0, t.numel(), 3):
            parts = [t.double() for t in (x, w, b)]
            step = torch.zeros(t.numel(), dtype=torch.float64, device="cuda")
            step[j] = 1e-5
            up, down = list(parts), list(parts)
            up[i], down[i] = parts[i] + step.view_as(t), parts[i] - step.view_as(t)
            slope = (value(*up) - value(*down)) / 2e-5
            assert abs(flat[j].item() - slope.item()) < 1e-4


# ---------------------------------------------------------------- dropout
def _philox(groups, call, seed, first=0):
    """Words of Philox4x32-10, (groups, 4), by the published definition."""
    at = np.arange(first, first + groups, dtype=np.uint64)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [at & low, at >> half, np.full(groups, call & 0xFFFFFFFF, np.uint64), np.full(groups, 6 << 24 | call >> 32, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        x, y = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(y >> half) ^ c[1] ^ np.uint64(k0), y & low, (x >> half) ^ c[3] ^ np.uint64(k1), x & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    return np.stack(c, 1)


def _kept(n, p, call, seed):
    words = _philox(-(-n // 4), call, seed).reshape(-1)[:n] if n else np.zeros(0, np.uint64)
    return torch.from_numpy(words >= np.uint64(int(np.floor(p * 2.0 ** 32)))).cuda()


@gpu
@pytest.mark.parametrize("n", [0, 1, 3, 4, 5, 7, 8, 9, 2047, 2048, 2049, 100_003])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_dropout(n, dtype):
    L = _ops()
    for off, p, call, seed in ((0, 0.1, 5, 7), (1, 0.5, 2 ** 40 + 3, 2 ** 63 + 11), (0, 0.0, 0, 0), (2, 1.0, 1, 1), (0, 0.999, 2 ** 56 - 1, 2 ** 64 - 1)):
        x, r = _rand((n + off,), dtype, seed=n)[off:], _rand((n + off,), dtype, seed=n + 1)[off:]
        kept = _kept(n, p, call, seed)
        scale = 1 / (1 - p) if p < 1 else 0.0
        want = torch.where(kept, x.double() * scale, 0.0)
        got = L.dropout(x, p, seed, call)
        _close(got, want, want.abs() * 2 * U)
        _close(L.dropout(x, p, seed, call, residual=r), want + r.double(), (want.abs() * 3 + r.double().abs()) * U)
        assert torch.equal(got == 0, ~kept | (x == 0))
        x[~kept] = float("nan")                     # what is dropped is not used
        assert not torch.isnan(L.dropout(x, p, seed, call)).any()
        same = r.clone()
        L.dropout(x, p, seed, call, residual=same, out=same)
        _close(same, want + r.double(), (want.abs() * 3 + r.double().abs()) * U)


@gpu
def test_dropout_in_autograd_and_with_a_number_on_the_device():
    L = _ops()
    x, r, dy = _rand((30, 41), seed=1).requires_grad_(), _rand((30, 41), seed=2).requires_grad_(), _rand((41, 30), seed=3).t()
    call = torch.tensor([11], device="cuda")
    y = L.dropout(x, 0.3, 9, call, residual=r)
    call += 1
    dx, dr = torch.autograd.grad(y, (x, r), dy)
    kept = _kept(30 * 41, 0.3, 11, 9).view(30, 41)
    assert torch.equal(dx != 0, kept) and torch.equal(dr, dy)
    _close(dx, torch.where(kept, dy.double() / 0.7, 0.0), dy.double().abs() * 3 * U)
    assert torch.equal(L.dropout(x.detach(), 0.3, 9, call), L.dropout(x.detach(), 0.3, 9, 12))
    # captured: a mask of its own for every replay
    graph, out, fixed = torch.cuda.CUDAGraph(), torch.empty_like(x.detach()), x.detach().clone()
    with torch.cuda.graph(graph):
        L.dropout(fixed, 0.3, 9, call, out=out)
        call += 1
    for number in (12, 13):
        graph.replay()
        assert torch.equal(out, L.dropout(fixed, 0.3, 9, number))
    with pytest.raises(B.TensairError), torch.cuda.graph(torch.cuda.CUDAGraph()):
        L.dropout(fixed, 0.3, 9, 5, out=out)


@gpu
def test_dropout_beyond_32_bits():
    n = 2 ** 34 // 4 + 9          # groups of four pass 2^30, offsets 2^32
    x = torch.ones(n, dtype=F16, device="cuda")
    y = _ops().dropout(x, 0.5, 3, 4)
    first = n // 4 - 5
    kept = torch.from_numpy(_philox(8, 4, 3, first).reshape(-1) >= np.uint64(2 ** 31)).cuda()[:n - first * 4]
    assert torch.equal(y[first * 4:] != 0, kept)
    assert abs((y[:10 ** 8] != 0).float().mean(dtype=torch.float64).item() - 0.5) < 6 * 0.5 / 10 ** 4


# ---------------------------------------------------------------- recurrence
def _run(gate, value, state, lengths, grad=None, grad_last=None):
    """The recurrence step by step in 64 bits, with bounds of its fp32 error: (out, last, bounds), and with grad (dgate, dvalue, dstate, bounds)."""
    B_, T, d = value.shape
    g, v = gate.double(), value.double()
    f, rest = torch.sigmoid(g), torch.sigmoid(-g)
    # 1 - f is off by 8 u of it.  Gates of 16 bits: exp(g) = 2^t with t the rounded product of g and the rounded log2(e), off by 1.5 u |t|
    # and so 2^t by 1.5 u |t| ln 2 <= 1.5 u |g| of it, which 1 / (1 + exp(g)) passes on at most whole: 1.5 |g| u more
    size = 8 + (1.5 * g.abs().clamp(max=90) if gate.dtype != torch.float32 else 0 * g)
    size = torch.where(torch.isfinite(g), size, 8.0)
    live = torch.ones(B_, T, 1, dtype=torch.bool, device=value.device)
    if lengths is not None:
        live = (torch.arange(T, device=value.device)[None] < lengths[:, None])[:, :, None]
    f, rest, v = torch.where(live, f, 1.0), torch.where(live, rest, 0.0), torch.where(live, v, 0.0)
    h = torch.zeros(B_, d, dtype=torch.float64, device=value.device) if state is None else state.double()
    e = torch.zeros_like(h)
    before, out, err, off = [], [], [], []
    for t in range(T):
        before.append(h)
        off.append(e)
        # per step: 1 - f is off by 8 u, two fused steps round, and the compositions that join stretches round as often again
        e = f[:, t] * e + U * (size[:, t] * rest[:, t] * (v[:, t].abs() + h.abs()) + 5 * (f[:, t] * h.abs() + rest[:, t] * v[:, t].abs()) * live[:, t])
        h = f[:, t] * h + rest[:, t] * v[:, t]
        out.append(h * live[:, t])
        err.append(e * live[:, t])
    empty = torch.zeros(B_, 0, d, dtype=torch.float64, device=value.device)

    def rows(xs):
        return torch.stack(xs, 1) if xs else empty

    joins = 1 + 3e-6
    first = U * 8 * (0 if state is None else state.double().abs())
    if grad is None:
        return rows(out), h, rows(err) * joins + first_bound(first, f, live), e * joins + first
    before, off = rows(before), rows(off)
    dh = torch.where(live, grad.double(), 0.0)
    c = torch.zeros(B_, d, dtype=torch.float64, device=value.device) if grad_last is None else grad_last.double()
    ec = U * 8 * c.abs()
    bulk = c.abs()
    dg, dv, eg, ev = [], [], [], []
    for t in range(T - 1, -1, -1):
        D = dh[:, t] + c
        big = dh[:, t].abs() + bulk
        eD = ec + 2 * U * big * live[:, t]
        dv.append(rest[:, t] * D)
        ev.append(rest[:, t] * (eD + (2 + size[:, t]) * U * D.abs()))
        gap = before[:, t] - v[:, t]
        slope = f[:, t] * rest[:, t] * live[:, t]
        dg.append(slope * gap * D)
        eg.append(slope * (gap.abs() * eD + (off[:, t] + (8 + 2 * size[:, t]) * U * (before[:, t].abs() + v[:, t].abs())) * big) + (8 + 2 * size[:, t]) * U * dg[-1].abs())
        ec = f[:, t] * eD + U * (size[:, t] * rest[:, t] + 5 * f[:, t]) * big * live[:, t]
        c, bulk = f[:, t] * D, f[:, t] * big
    back = [rows(x[::-1]) for x in (dg, dv, eg, ev)]
    return back[0], back[1], c, back[2] * 1.01, back[3] * 1.01, ec * 1.01


def first_bound(first, f, live):
    """What is off in the first state fades with it."""
    return torch.cumprod(f, 1) * first[:, None] * live if torch.is_tensor(first) else 0.0


CASES = [(1, 1, 1), (2, 1, 64), (3, 7, 5), (1, 8, 12), (2, 9, 16), (5, 16, 33), (2, 63, 300), (64, 65, 40), (3, 129, 301), (1, 257, 8),
         (2, 1000, 24), (1, 4097, 36), (1, 9000, 5), (7, 1025, 300), (300, 33, 64)]


@gpu
@pytest.mark.parametrize("shape", CASES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("ragged,given", [(False, False), (True, True), (False, True), (True, False)])
def test_recurrence_and_its_gradient(shape, dtype, ragged, given):
    L = _ops()
    B_, T, d = shape
    gate, value = _rand(shape, dtype, 2.0, 2.0, seed=T), _rand(shape, dtype, seed=d)
    state = _rand((B_, d), seed=3) if given else None
    grad, end = _rand(shape, dtype, seed=4), _rand((B_, d), seed=5) if given else None
    lengths = None
    if ragged:
        lengths = torch.from_numpy(np.random.default_rng(T).integers(0, T + 1, B_).astype(np.int32)).cuda()
        pad = torch.arange(T, device="cuda")[None] >= lengths[:, None]
        for x in (gate, value, grad):
            x[pad] = float("nan")                  # what is behind a sequence is not used
    want, h, slack, slack_h = _run(gate, value, state, lengths)
    out, last, marks = L.recurrence(gate, value, state, lengths, marks=True)
    _close(out, want, slack)
    _close(last, h, slack_h)
    again = L.recurrence(gate, value, state, lengths)
    assert torch.equal(out, again[0]) and torch.equal(last, again[1])
    if ragged:
        assert not out[pad].any()
    dg, dv, ds, eg, ev, es = _run(gate, value, state, lengths, grad, end)
    dgate, dvalue, dstate = L.recurrence_gradient(grad, gate, value, marks, lengths, grad_state=end)
    _close(dvalue, dv, ev)
    _close(dgate, dg, eg)
    _close(dstate, ds, es)


@gpu
def test_recurrence_follows_gates_near_one_and_resets():
    """A gate of 14 forgets 8e-7 of a state in a step: more of it than f = 1 - 2^-24 n could say.  A gate of minus infinity forgets all."""
    L = _ops()
    T = 20_000
    gate, value = torch.full((1, T, 4), 14.0, device="cuda"), _rand((1, T, 4))
    state = torch.full((1, 4), 1000.0, device="cuda")
    out, last = L.recurrence(gate, value, state)
    want, h, slack, slack_h = _run(gate, value, state, None)
    assert ((out.double() - want).abs() / want.abs()).max() < 2e-5      # T roundings, of which most cancel; f alone would be off by 4e-4
    _close(last, h, slack_h)
    gate[0, 5000] = float("-inf")
    gate[0, 7000] = float("inf")
    out, last = L.recurrence(gate, value, state)
    assert torch.equal(out[0, 5000], value[0, 5000])
    # step 7,000 = 875 * 8 is the first of a thread, which begins with a state that was composed; step 6,999 is the last of the thread before,
    # which got there by 8 steps of two roundings each from another composition (two roundings at each of three levels): (16 + 2 * 6) u
    assert ((out[0, 7000] - out[0, 6999]).abs() <= 28 * U * out[0, 6999].abs()).all()
    fresh, _ = L.recurrence(gate[:, 5001:], value[:, 5001:], value[:, 5000].contiguous())
    assert torch.allclose(out[:, 5001:], fresh, rtol=1e-4, atol=1e-6)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_recurrence_over_strided_halves_broadcast_and_one_value(dtype):
    L = _ops()
    B_, T, d = 3, 100, 48
    both = _rand((B_, T, 2 * d + 3), dtype)
    for off in (0, 1, 3):
        gate, value = both[..., off:off + d], both[..., off + d:off + 2 * d]
        out, last, marks = L.recurrence(gate, value, marks=True)
        same = L.recurrence(gate.contiguous(), value.contiguous())
        assert torch.equal(out, same[0]) and torch.equal(last, same[1])
        room = torch.zeros(B_, T, 2 * d + 5, dtype=dtype, device="cuda")
        L.recurrence_gradient(out, gate, value, marks, out=(room[..., off:off + d], room[..., off + d:off + 2 * d]))
        dgate, dvalue, _ = L.recurrence_gradient(out.contiguous(), gate.contiguous(), value.contiguous(), marks)
        assert torch.equal(room[..., off:off + d], dgate) and torch.equal(room[..., off + d:off + 2 * d], dvalue)
        assert not room[..., off + 2 * d:].any() and not room[..., :off].any()
    one = both[:1, :1, :d].expand(B_, T, d)                 # a gate for all steps and sequences
    want = L.recurrence(one.contiguous(), both[..., :d].contiguous())
    got = L.recurrence(one, both[..., :d])
    assert torch.equal(got[0], want[0])
    by_time = both[..., :d].transpose(0, 1).contiguous().transpose(0, 1)      # steps outermost
    assert torch.equal(L.recurrence(by_time, by_time)[0], L.recurrence(both[..., :d], both[..., :d])[0])


@gpu
def test_recurrence_of_nothing_and_lengths_out_of_range():
    L = _ops()
    state = _rand((2, 8))
    none = torch.zeros(2, 0, 8, device="cuda")
    out, last = L.recurrence(none, none, state)
    assert out.shape == (2, 0, 8) and torch.equal(last, state) and last.data_ptr() != state.data_ptr()
    assert not L.recurrence(none, none)[1].any()
    assert torch.equal(L.recurrence_gradient(none, none, none, torch.zeros(2, 0, 8, device="cuda"), grad_state=state)[2], state)
    nobody = torch.zeros(0, 5, 8, device="cuda")
    assert L.recurrence(nobody, nobody)[0].shape == (0, 5, 8)
    x = _rand((2, 30, 8))
    got = L.recurrence(x, x, state, torch.tensor([-5, 99], dtype=torch.int32, device="cuda"))
    want = L.recurrence(x, x, state, torch.tensor([0, 30], dtype=torch.int32, device="cuda"))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[1][0], state[0])


@gpu
@pytest.mark.parametrize("B_,d", [(1, 1), (64, 512), (3, 301), (5, 30), (130, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_recurrence_step_is_the_recurrence(B_, d, dtype):
    L = _ops()
    T = 11
    both, state = _rand((B_, T, 2 * d), dtype), _rand((B_, d), seed=2)
    gate, value = both[..., :d], both[..., d:]
    want, h, slack, slack_h = _run(gate, value, state, None)
    _, last = L.recurrence(gate, value, state)
    for t in range(T):
        out = L.recurrence_step(gate[:, t], value[:, t], state)
        _close(out, want[:, t], slack[:, t])
    _close(state, h, slack_h)
    assert torch.allclose(last, state, rtol=1e-5, atol=1e-6)


@gpu
def test_recurrence_has_the_gradient_that_differences_give():
    L = _ops()
    shape = (2, 11, 3)
    lengths = torch.tensor([11, 6], dtype=torch.int32, device="cuda")
    gate, value, state, dy, dl = _rand(shape, seed=1), _rand(shape, seed=2), _rand((2, 3), seed=3), _rand(shape, seed=4), _rand((2, 3), seed=5)
    ins = [t.clone().requires_grad_() for t in (gate, value, state)]
    out, last = L.recurrence(*ins, lengths)
    got = torch.autograd.grad((out * dy).sum() + (last * dl).sum(), ins)

    def weigh(parts):
        want, h, *_ = _run(*parts, lengths)
        return (want * dy.double()).sum() + (h * dl.double()).sum()

    parts = [t.double() for t in (gate, value, state)]
    for i, t in enumerate(parts):
        for j in range(t.numel()):
            step = torch.zeros(t.numel(), dtype=torch.float64, device="cuda")
            step[j] = 1e-5
            up, down = list(parts), list(parts)
            up[i], down[i] = t + step.view_as(t), t - step.view_as(t)
            slope = (weigh(up) - weigh(down)).item() / 2e-5
            assert abs(got[i].reshape(-1)[j].item() - slope) < 1e-4
    # a gradient of the last states alone, and one that is broadcast
    out, last = L.recurrence(*ins, lengths)
    a = torch.autograd.grad(last.sum(), ins, retain_graph=True)
    b = torch.autograd.grad(last, ins, torch.ones_like(last), retain_graph=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    a = torch.autograd.grad(out.sum(), ins, retain_graph=True)
    b = torch.autograd.grad(out, ins, torch.ones_like(out))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@gpu
def test_recurrence_beyond_32_bits():
    B_, T, d = 1, 4_300_000, 512          # 2.2 G elements
    x = torch.zeros(B_, T, d, dtype=BF16, device="cuda")
    x[:, -9:] = _rand((1, 9, d), BF16)
    out, last, marks = _ops().recurrence(x, x, marks=True)
    want, h, slack, slack_h = _run(x[:, -9:], x[:, -9:], None, None)
    _close(out[:, -9:], want, slack)
    _close(last, h, slack_h)
    assert not out[:, :1000].any()
    dg, dv, ds = _ops().recurrence_gradient(out, x, x, marks)
    small = _ops().recurrence(x[:, -16:], x[:, -16:], marks=True)
    tail = _ops().recurrence_gradient(out[:, -16:], x[:, -16:], x[:, -16:], small[2])
    assert torch.allclose(dg[:, -9:].float(), tail[0][:, -9:].float(), rtol=2 ** -7) and torch.allclose(dv[:, -9:].float(), tail[1][:, -9:].float(), rtol=2 ** -7)


# ---------------------------------------------------------------- streams and graphs
@gpu
def test_calls_on_two_streams_and_captured():
    L = _ops()
    x, w, dy = _rand((3000, 64), BF16), _rand((64,), F32, 0.1, 1.0), _rand((3000, 64), BF16, seed=1)
    gate, value, grad = (_rand((2, 1500, 64), BF16, seed=s) for s in (2, 3, 4))

    def all_of_it():
        y, mean, rstd = L.layer_norm(x, w, stats=True)
        out, last, marks = L.recurrence(gate, value, marks=True)
        return [y, *L.layer_norm_gradient(dy, x, w, mean, rstd), out, last, *L.recurrence_gradient(grad, gate, value, marks)]

    want = all_of_it()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(all_of_it())
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(all_of_it())
    for s, graph in zip(streams, graphs):          # replays beside one another
        with torch.cuda.stream(s):
            for _ in range(3):
                graph.replay()
    torch.cuda.synchronize()
    for g in outs:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


@gpu
def test_a_backward_pass_is_captured():
    L = _ops()
    x, w, b = _rand((64, 40), seed=1).requires_grad_(), _rand((40,), seed=2).requires_grad_(), _rand((40,), seed=3).requires_grad_()
    call = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step():
        y = L.layer_norm(x, w, b).view(2, 32, 40)
        h, _ = L.recurrence(y, y)
        return torch.autograd.grad((L.dropout(h, 0.2, 1, call, residual=y) ** 2).sum(), (x, w, b))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_calls_from_two_threads_at_once():
    import threading

    from paper_2211_10280_b200 import sampling

    L = _ops()

    def work(seed, out):
        with torch.cuda.stream(torch.cuda.Stream()):
            x, w, u = _rand((700, 96), BF16, seed=seed), _rand((96,), F32, 0.1, 1.0, seed=seed), torch.rand(5, generator=torch.Generator().manual_seed(seed)).cuda()
            logits, state = _rand((5, 4000), seed=seed), _rand((7, 96), seed=seed + 1)
            for _ in range(60):
                y, mean, rstd = L.layer_norm(x, w, stats=True)
                h, last = L.recurrence(y.view(7, 100, 96), y.view(7, 100, 96), state)
                out[seed] = [y, h, last, *L.layer_norm_gradient(y, x, w, mean, rstd), L.dropout(y, 0.3, seed, 4), sampling.sample(logits, u, 0.9, 30, 0.9)]
            torch.cuda.current_stream().synchronize()

    alone, together = {}, {}
    for seed in range(4):
        work(seed, alone)
    threads = [threading.Thread(target=work, args=(seed, together)) for seed in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for seed in range(4):
        assert all(torch.equal(a, b) for a, b in zip(alone[seed], together[seed]))


@gpu
def test_gradients_of_broadcast_inputs():
    L = _ops()
    gate, value, bias = _rand((1, 1, 24), seed=1).requires_grad_(), _rand((3, 50, 24), seed=2), _rand((24,), seed=3)
    full = gate.detach().expand(3, 50, 24).contiguous().requires_grad_()
    a, = torch.autograd.grad(L.recurrence(gate.expand(3, 50, 24), value)[0].square().sum(), gate)
    b, = torch.autograd.grad(L.recurrence(full, value)[0].square().sum(), full)
    assert torch.allclose(a, b.sum((0, 1), keepdim=True), rtol=1e-5, atol=1e-6)
    row = _rand((1, 24), seed=4).requires_grad_()
    many = row.detach().expand(70, 24).contiguous().requires_grad_()
    weigh = _rand((70, 24), seed=5)
    a, = torch.autograd.grad((L.layer_norm(row.expand(70, 24), bias) * weigh).sum(), row)
    b, = torch.autograd.grad((L.layer_norm(many, bias) * weigh).sum(), many)
    assert torch.allclose(a, b.sum(0, keepdim=True), rtol=1e-4, atol=1e-5)
    x = _rand((40, 30), seed=6)          # transposed: the mask goes by the element's place in the tensor, not in memory
    assert torch.equal(L.dropout(x.t(), 0.4, 1, 2), L.dropout(x.t().contiguous(), 0.4, 1, 2))


# ---------------------------------------------------------------- together
def _plain_block(model, x, w, kept, lengths):
    """The model's block and logits in 64 bits, elementary operations alone."""
    def norm(x, weight, bias):
        c = x - x.mean(-1, keepdim=True)
        return c / ((c * c).mean(-1, keepdim=True) + 1e-5) ** 0.5 * weight + bias

    n = norm(x, w["norm"], w["shift"])
    gate, value = (n @ w["gates"].t() + w["gate_bias"]).chunk(2, -1)
    f, h, out = torch.sigmoid(gate), torch.zeros_like(gate[:, 0]), []
    live = (torch.arange(x.shape[1], device="cuda")[None] < lengths[:, None])[:, :, None].double()
    for t in range(x.shape[1]):
        h = torch.where(live[:, t] > 0, f[:, t] * h + (1 - f[:, t]) * value[:, t], h)
        out.append(h * live[:, t])
    y = n + torch.where(kept, (torch.stack(out, 1) @ w["out"].t()) / (1 - model.drop), 0.0)
    return norm(y, w["last_norm"], w["last_shift"]) @ w["logits"].t() + w["bias"]


@gpu
def test_the_recurrent_model_has_the_gradients_of_its_formula():
    from paper_2211_10280_b200.next_token import RecurrentModel

    B_, T, V, d, hidden = 3, 41, 50, 24, 20
    model = RecurrentModel(V, d, hidden, dtype=F32, drop=0.25, seed=5)
    lengths = torch.tensor([41, 7, 30], dtype=torch.int32, device="cuda")
    x, weigh = _rand((B_, T, d), seed=1).requires_grad_(), _rand((B_, T, V), seed=2)
    w = model.weights()
    y, _ = model.block(x, w, call=3, lengths=lengths)
    logits = model.read(y, w)
    got = torch.autograd.grad((logits * weigh).sum(), [x] + list(w.values()))
    kept = _kept(B_ * T * d, 0.25, 3, 5).view(B_, T, d)
    x64, w64 = x.detach().double().requires_grad_(), {k: p.detach().double().requires_grad_() for k, p in w.items()}
    plain = _plain_block(model, x64, w64, kept, lengths)
    want = torch.autograd.grad((plain * weigh.double()).sum(), [x64] + list(w64.values()))
    # chains of some 300 roundings (T steps, products of 50 terms) of sums whose parts do not cancel by more than ten: 300 * 10 u
    assert (logits.double() - plain).norm() <= 3e3 * U * plain.norm()
    for a, b in zip(got, want):
        assert (a.double() - b).norm() <= 3e3 * U * b.norm(), (a.shape, ((a.double() - b).norm() / b.norm()).item())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_generation_goes_the_way_of_the_sequence(dtype):
    from paper_2211_10280_b200 import next_token, operators

    V, d, hidden, count = 300, 32, 24, 12
    model = next_token.RecurrentModel(V, d, hidden, dtype=dtype)
    table = _rand((V, d), seed=1)
    e = operators.Embedding(V, d, max_tokens=64, scale=d ** 0.5)
    first = torch.tensor([5, 17, 299], device="cuda")
    for temperature, top_k in ((0.0, 0), (0.8, 20)):
        got = next_token.generate(model, table, e, first, count, temperature=temperature, top_k=top_k, seed=4)
        assert got.shape == (3, count) and ((got >= 0) & (got < V)).all()
        assert torch.equal(got, next_token.generate(model, table, e, first, count, temperature=temperature, top_k=top_k, seed=4))
    # greedy: each token is the largest logit of the whole sequence's pass, or one that rounding (of 16 bits: a few 2^-8 of the logits) cannot tell from it
    got = next_token.generate(model, table, e, first, count, temperature=0.0)
    ids = torch.cat([first[:, None], got[:, :-1]], 1)
    with torch.no_grad():
        w = {k: model.half.get(k, p) for k, p in model.params.items()}
        y, _ = model.block(e.lookup(table, ids), w, call=0, drop=0.0)
        logits = model.read(y, w).float()
    chosen = logits.gather(2, got[:, :, None])[..., 0]
    size = logits.abs().amax()
    assert (logits.amax(2) - chosen <= (1e-5 if dtype == F32 else 0.05) * size).all()


@gpu
@pytest.mark.parametrize("state_bits", [8, 32])
def test_the_recurrent_example_runs(state_bits):
    from paper_2211_10280_b200 import next_token

    r = next_token.train_recurrent(steps=6, V=500, d=32, hidden=48, rows=16, window=20, state_bits=state_bits, report=3)
    assert len(r["losses"]) == 3 and all(np.isfinite(r["losses"]))
    assert all(torch.isfinite(p).all() for p in r["model"].params.values()) and torch.isfinite(r["table"]).all()
    out = next_token.generate(r["model"], r["table"], r["embedding"], torch.arange(4, device="cuda"), 5)
    assert out.shape == (4, 5) and ((out >= 0) & (out < 500)).all()


# ---------------------------------------------------------------- refusals
def _norm_call(gradient=False, **change):
    h = B.Norm(weight=4096, bias=4096, mean=4096, rstd=4096, n=10, param_type=B.FLOAT32, eps=1e-5)
    rows = {k: B.Rows(data=4096, stride=8, d=8, type=B.FLOAT32) for k in ("x", "y", "dx")}
    rest = dict(dweight=4096, dbias=4096, workspace=4096, bytes=1 << 30)
    for key, x in change.items():
        if key in rest:
            rest[key] = x
        elif key in rows:
            if x is None:
                rows[key] = None
            else:
                for f, v in x.items():
                    setattr(rows[key], f, v)
        elif key == "norm":
            h = None
        else:
            setattr(h, key, x)
    if gradient:
        return B.lib().tensair_layer_norm_gradient(h, rows["y"], rows["x"], rows["dx"], rest["dweight"], rest["dbias"], rest["workspace"],
                                                   rest["bytes"], None)
    return B.lib().tensair_layer_norm(h, rows["x"], rows["y"], None)


@pytest.mark.parametrize("change,word", [
    (dict(norm=None), "norm"), (dict(n=2 ** 30 + 1), "n must"), (dict(eps=float("nan")), "eps"), (dict(eps=-1.0), "eps"), (dict(param_type=3), "param_type"),
    (dict(weight=None), "weight"), (dict(weight=4098), "weight"), (dict(mean=None), "mean"), (dict(rstd=4097), "mean"), (dict(x=None), "x"),
    (dict(x=dict(d=0)), "d not in"), (dict(x=dict(d=2 ** 20 + 1)), "d not in"), (dict(x=dict(data=None)), "x"), (dict(x=dict(stride=7)), "x"), (dict(y=dict(data=None)), "NULL"),
    (dict(y=dict(d=4)), "width"), (dict(y=dict(stride=7)), "stride"), (dict(x=dict(type=B.BFLOAT16)), "types"), (dict(x=dict(type=3)), "x")])
def test_layer_norm_refuses(change, word):
    for gradient in (False, True):
        assert _norm_call(gradient, **change) == B.EINVAL
        assert word in B.lib().tensair_last_error(None).decode()


def test_layer_norm_gradient_refuses():
    for change, word in ((dict(dx=None), "dx"), (dict(dx=dict(type=B.BFLOAT16)), "dx"), (dict(mean=None, rstd=None), "mean"), (dict(dweight=4097), "dweight"),
                         (dict(dbias=4098), "dbias"), (dict(workspace=None), "workspace"), (dict(workspace=4100), "workspace")):
        assert _norm_call(True, **change) == B.EINVAL and word in B.lib().tensair_last_error(None).decode()
    assert _norm_call(True, bytes=100) == B.ENOMEM
    assert _norm_call(False, n=0) == B.OK and _norm_call(False, n=0, x=dict(data=None), y=dict(data=None)) == B.OK
    size = C.c_uint64()
    for bad in ((2 ** 30 + 1, 8), (5, 0), (5, 2 ** 20 + 1)):
        assert B.lib().tensair_norm_workspace_bytes(*bad, C.byref(size)) == B.EINVAL
    assert B.lib().tensair_norm_workspace_bytes(5, 8, None) == B.EINVAL


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(n=2 ** 40), "n must"), (dict(p=-0.1), "p must"), (dict(p=1.1), "p must"), (dict(p=float("nan")), "p must"),
    (dict(call=2 ** 56), "call"), (dict(call_at=4100), "call_at"), (dict(x=None), "NULL"), (dict(out=None), "NULL"), (dict(x=4098), "aligned"),
    (dict(residual=4097), "aligned")])
def test_dropout_refuses(change, word):
    h = B.DropoutCall(x=4096, out=4096, n=10, p=0.5, seed=1, call=1, type=B.FLOAT32)
    for f, x in change.items():
        setattr(h, f, x)
    assert B.lib().tensair_dropout(h, None) == B.EINVAL and word in B.lib().tensair_last_error(None).decode()
    assert B.lib().tensair_dropout(None, None) == B.EINVAL
    assert B.lib().tensair_dropout(B.DropoutCall(n=0, p=0.5), None) == B.OK


def _steps(**change):
    s = B.Steps(data=4096, batch=80, step=8)
    for f, x in change.items():
        setattr(s, f, x)
    return s


def _seq(gate=None, value=None, **change):
    q = B.Sequences(gate or _steps(), value or _steps(), None, 4, 10, 8, B.FLOAT32)
    for f, x in change.items():
        setattr(q, f, x)
    return q


@pytest.mark.parametrize("change,word", [
    (dict(d=0), "d must"), (dict(d=2 ** 20 + 1), "d must"), (dict(type=3), "type"), (dict(B=2 ** 31), "too large"), (dict(T=2 ** 31), "too large"),
    (dict(B=2 ** 29), "too large"), (dict(lengths=4098), "lengths"), (dict(gate=_steps(data=None)), "gate"), (dict(value=_steps(data=4097)), "gate or value"),
    (dict(gate=_steps(step=2 ** 40)), "gate"), (dict(value=_steps(batch=2 ** 40)), "gate or value")])
def test_recurrences_refuse(change, word):
    L, out = B.lib(), _steps()
    q = _seq(**change)
    assert L.tensair_recurrence(q, None, out, 4096, None, None) == B.EINVAL and word in L.tensair_last_error(None).decode()
    assert L.tensair_recurrence_gradient(q, out, None, 4096, out, out, 4096, None) == B.EINVAL and word in L.tensair_last_error(None).decode()
    q.T = 1 if "T" not in change else q.T
    assert L.tensair_recurrence_step(q, 4096, out, None) == B.EINVAL


def test_recurrences_refuse_their_other_arguments():
    L, ok = B.lib(), _steps()
    assert L.tensair_recurrence(None, None, ok, 4096, None, None) == B.EINVAL
    for bad in (None, _steps(data=None), _steps(data=4098), _steps(step=7), _steps(batch=7), _steps(step=2 ** 40)):
        assert L.tensair_recurrence(_seq(), None, bad, 4096, None, None) == B.EINVAL
        assert L.tensair_recurrence_gradient(_seq(), ok, None, 4096, bad, ok, None, None) == B.EINVAL
        assert L.tensair_recurrence_gradient(_seq(), ok, None, 4096, ok, bad, None, None) == B.EINVAL
        if bad is None or bad.data != 4096 or bad.batch == 7:
            assert L.tensair_recurrence_step(_seq(T=1), 4096, bad, None) == B.EINVAL
    for args in ((4098, 4096, None), (None, 4098, None), (None, 4096, 4098)):
        assert L.tensair_recurrence(_seq(), args[0], ok, args[1], args[2], None) == B.EINVAL
    assert L.tensair_recurrence_gradient(_seq(), ok, None, None, ok, ok, None, None) == B.EINVAL
    assert L.tensair_recurrence_gradient(_seq(), None, None, 4096, ok, ok, None, None) == B.EINVAL
    assert L.tensair_recurrence_gradient(_seq(), ok, 4096, 4096, ok, ok, 4096, None) == B.EINVAL
    assert L.tensair_recurrence_step(_seq(), 4096, ok, None) == B.EINVAL             # more than one step
    assert L.tensair_recurrence_step(_seq(T=1, lengths=4096), 4096, ok, None) == B.EINVAL
    assert L.tensair_recurrence_step(_seq(T=1), None, ok, None) == B.EINVAL
    assert L.tensair_recurrence_step(_seq(T=1, B=0), 4096, ok, None) == B.OK


def test_binding_structures_match_the_header(tmp_path):
    import subprocess

    names = {"tensair_norm": B.Norm, "tensair_dropout_call": B.DropoutCall, "tensair_steps": B.Steps, "tensair_sequences": B.Sequences,
             "tensair_draw": B.Draw}
    lines = []
    for name, s in names.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in s._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "tensair.h"\nint main(void) {' + "".join(lines) + "return 0;}")
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-I", str(libbuild.INCLUDE), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
    want = []
    for s in names.values():
        want += [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]
    assert got == want


def test_calls_on_cpu_tensors_are_refused():
    L, x = _ops(), torch.zeros(2, 3, 8)
    w, s = torch.ones(8), torch.zeros(2, 8)
    for call in (lambda: L.layer_norm(x, w), lambda: L.layer_norm_gradient(x, x, w, w, w), lambda: L.dropout(x, 0.5, 1, 1), lambda: L.recurrence(x, x),
                 lambda: L.recurrence_gradient(x, x, x, x), lambda: L.recurrence_step(s, s, s)):
        with pytest.raises(ValueError, match="no CUDA device"):
            call()


@gpu
def test_the_python_calls_refuse():
    L = _ops()
    x, w, s = _rand((2, 16, 8)), _rand((8,)), _rand((2, 8))
    marks = _rand((2, 2, 8))
    flat = x.view(32, 8)
    st = _rand((32,))
    n = torch.ones(2, dtype=torch.int32, device="cuda")
    grad = x.clone().requires_grad_()
    bad = [lambda: L.layer_norm(x, w[:7]), lambda: L.layer_norm(x, w.double()), lambda: L.layer_norm(x.double(), w), lambda: L.layer_norm(x, w.cpu()),
           lambda: L.layer_norm(x, w, w.half()), lambda: L.layer_norm(x, w, dtype=torch.float64), lambda: L.layer_norm(x.half(), w, dtype=F32),
           lambda: L.layer_norm(x, w, out=x[:1]), lambda: L.layer_norm(x, w, eps=-1.0), lambda: L.layer_norm(grad, w, stats=True), lambda: L.layer_norm(x, s),
           lambda: L.layer_norm_gradient(flat, x, w, st, st), lambda: L.layer_norm_gradient(x, x, w, st[:3], st), lambda: L.layer_norm_gradient(x.half(), x.bfloat16(), w, st, st),
           lambda: L.dropout(x, 1.5, 1, 1), lambda: L.dropout(x, 0.5, -1, 1), lambda: L.dropout(x, 0.5, 1, 2 ** 56), lambda: L.dropout(x, 0.5, 1, 1, residual=flat),
           lambda: L.dropout(x, 0.5, 1, n), lambda: L.dropout(x, 0.5, 1, 1, out=x.half()), lambda: L.dropout(x.double(), 0.5, 1, 1), lambda: L.dropout(x.int(), 0.5, 1, 1),
           lambda: L.recurrence(x, x.half()), lambda: L.recurrence(x[:1], x), lambda: L.recurrence(flat, flat), lambda: L.recurrence(x, x, s.half()),
           lambda: L.recurrence(x, x, s[:1]), lambda: L.recurrence(x, x, lengths=n.long()), lambda: L.recurrence(x, x, lengths=n[:1]), lambda: L.recurrence(x, x, lengths=n.cpu()),
           lambda: L.recurrence(x, x, out=x.transpose(1, 2)), lambda: L.recurrence(grad, x, marks=True), lambda: L.recurrence(x, x, out=x[:, :1].expand(2, 16, 8)),
           lambda: L.recurrence_gradient(x, x, x, marks[:, :1].contiguous()), lambda: L.recurrence_gradient(x.half(), x, x, marks),
           lambda: L.recurrence_gradient(x, x, x, marks, out=(x.half(), x)), lambda: L.recurrence_gradient(x, x, x, marks, grad_state=s.half()),
           lambda: L.recurrence_step(s, s, s.half()), lambda: L.recurrence_step(s, s[:1], s), lambda: L.recurrence_step(x, x, s), lambda: L.recurrence_step(s, s, None),
           lambda: L.recurrence_step(s.clone().requires_grad_(), s, s)]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, B.TensairError)):
            call()
            pytest.fail(f"call {i} was not refused")
