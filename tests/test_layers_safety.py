"""Calls of the recurrent model's operators that their documentation allows and that go wrong easily: results written over their inputs, states
that fall by many orders of magnitude, forward-mode derivatives, devices that hold no large clusters.

Bounds of the recurrence, u = 2^-24: 1 - f is off by S u of itself, and so is f where it is below 1/2 (S = 8: expf 2 u, the fast quotient 4 u and a
rounding each of 1 + e and the product; with gates of 16 bits 1.5 |gate| more for the rounded product with log2(e)).  Where f is 1/2 or
more it is taken from 1 - f and is off by S u (1 - f).  So f is off by S u min(f, 1 - f).  On top of that a step has two roundings, and the joining of
stretches of eight steps as often again or less; 8 u of the terms' sizes are allowed for all of these.  All of it is relative to
f |h| + (1 - f) |v|: nothing is left of a state that has been forgotten.
"""
import ctypes as C
import subprocess
import sys

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
    rel, least = LAST[got.dtype]
    assert got.shape == want.shape and not torch.isnan(got).any()
    excess = (got.double() - want).abs() - (slack + (want.abs() + slack) * rel + least)
    worst = excess.argmax()
    assert excess.max().item() <= 0, (got.flatten()[worst].item(), want.flatten()[worst].item(), slack.flatten()[worst].item())


def _ok(rc):
    assert rc == B.OK, B.lib().tensair_last_error(None)


# ---------------------------------------------------------------- results in the place of inputs
@gpu
@pytest.mark.parametrize("dtype,n,d", [(F32, 70, 64), (BF16, 33, 1000), (F16, 21, 301), (F32, 9, 4100), (BF16, 12, 8192), (F32, 5, 8192), (F32, 70, 8196), (BF16, 40, 16_384),
                                       (F16, 37, 8195), (F32, 40, 20_011), (BF16, 35, 70_000)])
def test_the_gradient_of_a_norm_in_the_place_of_the_incoming_one(dtype, n, d):
    """Rows that fit into a warp, into a block, and into none."""
    L = _ops()
    x, dy, w = _rand((n, d), dtype, seed=1), _rand((n, d), dtype, 0.5, 0.2, seed=2), _rand((d,), F32, 0.1, 1.0, seed=3)
    _, mean, rstd = L.layer_norm(x, w, stats=True)
    dx, dw, db = L.layer_norm_gradient(dy, x, w, mean, rstd)
    kind = {F32: B.FLOAT32, BF16: B.BFLOAT16, F16: B.FLOAT16}[dtype]
    size = C.c_uint64()
    _ok(B.lib().tensair_norm_workspace_bytes(n, d, C.byref(size)))
    workspace, sums = torch.empty(size.value, dtype=torch.uint8, device="cuda"), torch.empty(2, d, device="cuda")
    norm = B.Norm(w.data_ptr(), None, mean.data_ptr(), rstd.data_ptr(), n, B.FLOAT32, 0.0)
    place = B.Rows(dy.data_ptr(), d, d, kind)
    _ok(B.lib().tensair_layer_norm_gradient(norm, place, B.Rows(x.data_ptr(), d, d, kind), place, sums[0].data_ptr(), sums[1].data_ptr(), workspace.data_ptr(),
                                            size.value, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(dy, dx) and torch.equal(sums[0], dw) and torch.equal(sums[1], db)


@gpu
@pytest.mark.parametrize("n", [1, 7, 4096, 100_003])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_dropout_in_the_place_of_its_input(n, dtype):
    L = _ops()
    for off in (0, 1):
        x, r = _rand((n + off,), dtype, seed=n)[off:], _rand((n + off,), dtype, seed=n + 1)[off:]
        for residual in (None, r):
            want, same = L.dropout(x, 0.3, 5, 6, residual=residual), _rand((n + off,), dtype, seed=n)[off:]
            L.dropout(same, 0.3, 5, 6, residual=residual, out=same)
            assert torch.equal(same, want)


@gpu
@pytest.mark.parametrize("B_,T,d", [(3, 20, 30), (1, 9000, 64), (300, 2100, 64), (5, 3001, 301)])
def test_last_states_in_the_place_of_the_first(B_, T, d):
    """One group of channels to a cluster, and many of them one after the other."""
    L = _ops()
    gate, value, state = _rand((B_, T, d), BF16, 2.0, 2.0, seed=1), _rand((B_, T, d), BF16, seed=2), _rand((B_, d), seed=3)
    out, last = L.recurrence(gate, value, state)
    again = torch.empty_like(out)
    rows = [B.Steps(x.data_ptr(), T * d, d) for x in (gate, value, again)]
    q = B.Sequences(rows[0], rows[1], None, B_, T, d, B.BFLOAT16)
    _ok(B.lib().tensair_recurrence(q, state.data_ptr(), rows[2], state.data_ptr(), None, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(again, out) and torch.equal(state, last)


# ---------------------------------------------------------------- states that fall by orders of magnitude
def _run(gate, value, state, grad, end):
    """Everything in 64 bits, step by step, with the bounds of the head of this file: pairs (value, bound) of out, last, dgate, dvalue, dstate."""
    g, v = gate.double(), value.double()
    f, rest = torch.sigmoid(g), torch.sigmoid(-g)
    size = 8 + (1.5 * g.abs() if gate.dtype != F32 else 0 * g)
    off_f, off_rest = size * torch.minimum(f, rest) * U, size * rest * U
    h, H, e = state.double(), state.double().abs(), 0 * state.double()
    before, off, out, err = [], [], [], []
    for t in range(gate.shape[1]):
        before.append(h), off.append(e)
        new = f[:, t] * H + rest[:, t] * v[:, t].abs()
        e = f[:, t] * e + off_f[:, t] * H + off_rest[:, t] * v[:, t].abs() + 8 * U * new
        h, H = f[:, t] * h + rest[:, t] * v[:, t], new
        out.append(h), err.append(e)
    last = h, e * 1.001
    c, Z, e = end.double(), end.double().abs(), 0 * end.double()
    back = []
    for t in range(gate.shape[1] - 1, -1, -1):
        D, big = grad[:, t].double() + c, grad[:, t].double().abs() + Z
        e = e + 2 * U * big
        gap, e_gap = before[t] - v[:, t], off[t] + U * (before[t] - v[:, t]).abs()
        slope = f[:, t] * rest[:, t]
        dv, e_v = rest[:, t] * D, rest[:, t] * e + (off_rest[:, t] + 2 * U * rest[:, t]) * big
        dg, e_g = slope * gap * D, slope * (gap.abs() * e + e_gap * big + (2 * size[:, t] + 4) * U * gap.abs() * big)
        back.append((dg, e_g * 1.001, dv, e_v * 1.001))
        e = f[:, t] * e + off_f[:, t] * big + 8 * U * f[:, t] * big
        c, Z = f[:, t] * D, f[:, t] * big
    dg, eg, dv, ev = (torch.stack(x[::-1], 1) for x in zip(*back))
    return (torch.stack(out, 1), torch.stack(err, 1) * 1.001), last, (dg, eg), (dv, ev), (c, e * 1.001)


def _gates(kind, shape, seed):
    r = np.random.default_rng(seed)
    if kind == "two":                # each step keeps 0.88
        x = np.full(shape, 2.0)
    elif kind == "resets":           # two steps that keep next to nothing
        x = r.choice([0.0, 3.0, 8.0, 14.0], shape)
        x[:, 100:] = r.choice([8.0, 14.0], shape)[:, 100:]
        for t in (20, 70):
            x[:, t] = r.choice([-20.0, -17.0, -10.0, -5.0], (shape[0], shape[2]))
    elif kind == "slow":             # a stretch keeps nearly all, the sequence little: products cross 1/2 between stretches, blocks and turns
        x = r.uniform(5.5, 9.0, shape)
    else:                            # about 1/2
        x = r.uniform(-0.3, 0.3, shape)
    return torch.from_numpy(x)


@gpu
@pytest.mark.parametrize("kind,shape", [("two", (2, 7, 8)), ("two", (1, 128, 4)), ("two", (2, 192, 24)), ("two", (3, 300, 7)), ("half", (2, 90, 64)), ("half", (40, 33, 30)),
                                        ("resets", (2, 130, 24)), ("resets", (1, 1500, 5)), ("resets", (70, 200, 64)), ("slow", (1, 4000, 24)), ("slow", (2, 6000, 16)),
                                        ("slow", (60, 1100, 40))])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("small", [0.0, 1.0])
def test_a_state_and_a_gradient_that_are_forgotten_step_by_step(kind, shape, dtype, small):
    """A first state of 10^6 (16 bits' outputs: what they hold of it) over values of 0 or 1, and the gradient of the last states alone."""
    L = _ops()
    B_, T, d = shape
    gate, value = _gates(kind, shape, T).to(dtype).cuda(), (_rand(shape, F32, seed=T) * small).to(dtype)
    state = _rand((B_, d), seed=3) * (3e3 if dtype == F16 else 1e6)
    end, grad = _rand((B_, d), seed=5), torch.zeros(shape, dtype=dtype, device="cuda")
    out, last, marks = L.recurrence(gate, value, state, marks=True)
    dgate, dvalue, dstate = L.recurrence_gradient(grad, gate, value, marks, grad_state=end)
    want = _run(gate, value, state, grad, end)
    for got, (x, slack) in zip((out, last, dgate, dvalue, dstate), want):
        _close(got, x, slack)
    # and step by step, as it is served
    now = state.clone()
    for t in range(min(T, 100)):
        h = L.recurrence_step(gate[:, t], value[:, t], now)
        _close(h, want[0][0][:, t], want[0][1][:, t])


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T", [1, 5, 100, 5000])
def test_infinite_gates_keep_everything_or_nothing(dtype, T):
    L = _ops()
    B_, d = 2, 20
    value, state, grad, end = _rand((B_, T, d), dtype, 100.0), _rand((B_, d), seed=1), _rand((B_, T, d), dtype, seed=2), _rand((B_, d), seed=3)
    gate = torch.full((B_, T, d), float("inf"), dtype=dtype, device="cuda")
    out, last, marks = L.recurrence(gate, value, state, marks=True)
    assert torch.equal(last, state) and torch.equal(out, state.to(dtype)[:, None].expand_as(out))
    dgate, dvalue, dstate = L.recurrence_gradient(torch.zeros_like(grad), gate, value, marks, grad_state=end)
    assert torch.equal(dstate, end) and not dgate.any() and not dvalue.any()
    gate = -gate
    out, last, marks = L.recurrence(gate, value, state, marks=True)
    assert torch.equal(out, value) and torch.equal(last, value[:, -1].float())
    dgate, dvalue, dstate = L.recurrence_gradient(grad, gate, value, marks, grad_state=end)
    grad[:, -1] = (grad[:, -1].float() + end).to(dtype)
    assert torch.equal(dvalue, grad) and not dgate.any() and not dstate.any()
    step = state.clone()
    assert torch.equal(L.recurrence_step(gate[:, 0], value[:, 0], step), value[:, 0]) and torch.equal(step, value[:, 0].float())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_every_gate_has_the_factor_of_its_formula(dtype):
    """One step from 1 to 0 is f, one from 0 to 1 is 1 - f: all gates of 16 bits, a million of 32."""
    L = _ops()
    if dtype == F32:
        g = torch.cat([_rand((500_000,), std=30.0), _rand((500_000,), std=2.0, seed=1), _rand((50_000,), std=1e-3, seed=2)])
    else:
        g = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16).view(dtype).cuda()
        g = g[~torch.isnan(g)]
    g = g.view(-1, 50) if dtype == F32 else g[None]
    one, zero = torch.ones(g.shape, device="cuda"), torch.zeros(g.shape, device="cuda")
    keep, take = one.clone(), zero.clone()
    L.recurrence_step(g, zero.to(dtype), keep)
    L.recurrence_step(g, one.to(dtype), take)
    wide = g.double()
    f, rest = torch.sigmoid(wide), torch.sigmoid(-wide)
    size = (8 + (0 if dtype == F32 else 1.5 * wide.abs().clamp(max=100))) * torch.minimum(f, rest) * U
    for got, want in ((keep, f), (take, rest)):      # below 2^-126: zero, or what fp32 has of it
        assert ((got.double() - want).abs() <= size + want * U + 2.0 ** -126).all()


# ---------------------------------------------------------------- first calls
@gpu
def test_the_first_calls_of_a_process_may_be_captured():
    """What a device is asked once, and what kernels are told once, happens while the graph is being captured."""
    code = """
import torch
from paper_2211_10280_b200 import layers, sampling
x, u = torch.randn(1, 40_000, device="cuda"), torch.rand(1, device="cuda")
a, s = torch.randn(1, 5000, 64, device="cuda"), torch.randn(1, 64, device="cuda")
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    token = sampling.sample(x, u, 0.9, 50, 0.9)
    out, last, marks = layers.recurrence(a, a, s, marks=True)
    back = layers.recurrence_gradient(a, a, a, marks)
graph.replay()
torch.cuda.synchronize()
assert torch.equal(token, sampling.sample(x, u, 0.9, 50, 0.9))
again = layers.recurrence(a, a, s, marks=True)
assert all(torch.equal(p, q) for p, q in zip((out, last, marks), again))
assert all(torch.equal(p, q) for p, q in zip(back, layers.recurrence_gradient(a, a, a, marks)))
"""
    subprocess.run([sys.executable, "-c", code], check=True, timeout=300, cwd=libbuild.HERE.parent)


# ---------------------------------------------------------------- derivatives that are not there
def test_a_tangent_is_seen():
    import torch.autograd.forward_ad as fwd

    L, x = _ops(), torch.ones(3)
    assert not L._wants_gradient(x, None)
    with fwd.dual_level():
        dual = fwd.make_dual(x, torch.ones(3))
        assert L._wants_gradient(None, dual) and not L._wants_gradient(x, None)
        with torch.no_grad():              # which leaves forward mode on
            assert L._wants_gradient(dual)
        with torch.inference_mode():       # which does not
            assert not L._wants_gradient(x)
    assert not L._wants_gradient(x)


@gpu
def test_forward_mode_is_refused():
    import torch.autograd.forward_ad as fwd

    L = _ops()
    x, w, s = _rand((2, 16, 8)), _rand((8,)), _rand((2, 8))
    with fwd.dual_level():
        dx, dw, ds = (fwd.make_dual(t, torch.ones_like(t)) for t in (x, w, s))
        for i, call in enumerate([lambda: L.layer_norm(dx, w), lambda: L.layer_norm(x, dw), lambda: L.layer_norm(x, w, dw), lambda: L.dropout(dx, 0.1, 1, 1),
                                  lambda: L.dropout(x, 0.1, 1, 1, residual=dx), lambda: L.recurrence(dx, x), lambda: L.recurrence(x, dx), lambda: L.recurrence(x, x, ds),
                                  lambda: L.recurrence_step(ds, s, s.clone()), lambda: L.recurrence_step(s, s, ds), lambda: L.layer_norm(dx, w, stats=True)]):
            for mode in (torch.enable_grad, torch.no_grad):
                with pytest.raises((NotImplementedError, ValueError)), mode():
                    call()
                    pytest.fail(f"call {i} lost a tangent")
        assert L.layer_norm(x, w).shape == x.shape


# ---------------------------------------------------------------- devices that hold no large clusters
SIZES = [1, 2, 4, 8, 12, 16]
FULL = [296, 140, 71, 33, 20, 14]
WORK = [(T, total, e) for T in (1, 5, 8, 9, 300, 1021, 1024, 65_536, 2 ** 30) for total in (1, 75, 128, 4800, 8192, 2 ** 20, 2 ** 30) for e in (2, 4)]


def _compiled(tmp_path, header, body, lines):
    """What a program that includes `header` prints for each line of numbers."""
    src, exe = tmp_path / "cut.cpp", tmp_path / "cut"
    src.write_text(f'#include <cstdio>\n#include "{header}"\nusing namespace tensair;\nint main() {{ unsigned long long x[9]; {body} }}')
    subprocess.check_call(["g++", "-std=c++17", "-I", str(libbuild.CSRC), str(src), "-o", str(exe)])
    text = "\n".join(" ".join(map(str, line)) for line in lines)
    return [list(map(int, line.split())) for line in subprocess.check_output([str(exe)], input=text, text=True).splitlines()]


def test_the_recurrence_is_cut_for_the_clusters_that_there_are(tmp_path):
    rooms = [FULL, [296, 140, 71, 33, 0, 0], [296, 140, 71, 0, 0, 0], [296, 0, 0, 0, 0, 0], [20, 9, 0, 0, 1, 1], [2, 1, 1, 1, 1, 1], [0] * 6]
    body = """while (scanf("%llu %llu %llu %llu %llu %llu %llu %llu %llu", x, x + 1, x + 2, x + 3, x + 4, x + 5, x + 6, x + 7, x + 8) == 9) {
        const uint32_t room[recurrence::kSizes] = {(uint32_t)x[3], (uint32_t)x[4], (uint32_t)x[5], (uint32_t)x[6], (uint32_t)x[7], (uint32_t)x[8]};
        const recurrence::Plan p = recurrence::cut((uint32_t)x[0], (uint32_t)x[1], (uint32_t)x[2], room);
        printf("%u %u %u %u %u\\n", p.units, p.cluster, p.turns, p.groups, p.grid); }"""
    lines = [(*w, *room) for room in rooms for w in WORK]
    got = _compiled(tmp_path, "recurrence_cut.h", body, lines)
    assert len(got) == len(lines)
    for (T, total, e, *room), (units, cluster, turns, groups, grid) in zip(lines, got):
        held = room[SIZES.index(cluster)]
        assert held or cluster == 1                                              # none of a size that is not held
        assert units in (8, 16, 32, 64, 128, 256) and (cluster == 1 or units * e <= 64)
        span = cluster * (256 // units) * 8
        assert (turns - 1) * span < T <= turns * span and (groups - 1) * units < total <= groups * units
        assert grid == min(groups, max(held, 1)) * cluster
    # one long stream: the largest clusters of a whole device, or what there is
    long = WORK.index((65_536, 128, 4))
    assert [got[i * len(WORK) + long][1] for i in range(4)] == [12, 8, 4, 1]


def test_a_row_of_the_draw_is_shared_by_clusters_that_there_are(tmp_path):
    body = """while (scanf("%llu %llu %llu %llu", x, x + 1, x + 2, x + 3) == 4) printf("%u\\n", row_blocks((uint32_t)x[0], (uint32_t)x[1], (uint32_t)x[2], (uint32_t)x[3]));"""
    lines = [(n, V, sms, most) for n in (1, 2, 5, 9, 37, 74, 75, 148, 256, 2 ** 24) for V in (1, 8000, 8001, 16_001, 100_000, 2 ** 20) for sms in (18, 72, 148)
             for most in (1, 2, 4, 8, 16)]
    for (n, V, sms, most), (blocks,) in zip(lines, _compiled(tmp_path, "sample_cut.h", body, lines)):
        assert blocks in (1, 2, 4, 8, 16) and blocks <= most
        assert blocks == 1 or (n * blocks // 2 < sms and V > blocks // 2 * 8000)          # a half would not do
        assert blocks == most or n * blocks >= sms or V <= blocks * 8000                  # a double is not worth it


def test_the_lanes_that_exchange_compositions_are_those_that_are_there(tmp_path):
    """Blocks of a cluster have 16, 32 or 64 channels; the last part of each is a thread's, of the last ones of the block."""
    body = 'while (scanf("%llu %llu", x, x + 1) == 2) printf("%u\\n", recurrence::last_lanes((uint32_t)x[0], (uint32_t)x[1]));'
    lines = [(channels, thread) for channels in (16, 32, 64) for thread in range(256 - channels, 256)]
    for (channels, thread), (mask,) in zip(lines, _compiled(tmp_path, "recurrence_cut.h", body, lines)):
        first = thread // 32 * 32
        assert mask == sum(1 << lane for lane in range(32) if first + lane >= 256 - channels)
    assert "__activemask" not in (libbuild.CSRC / "recurrence.cu").read_text()


# ---------------------------------------------------------------- the example's command line
@pytest.mark.parametrize("args", [["--dense", "--recurrent"], ["--generate", "3"]])
def test_the_example_refuses_what_it_would_not_do(args, monkeypatch, capsys):
    from paper_2211_10280_b200 import next_token

    monkeypatch.setattr("sys.argv", ["next_token", *args])
    for name in ("train", "train_recurrent"):
        monkeypatch.setattr(next_token, name, lambda *a, **k: pytest.fail("it went on"))
    with pytest.raises(SystemExit):
        next_token.main()
    assert args[0] in capsys.readouterr().err
