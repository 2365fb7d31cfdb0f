"""The language-model operators against plain implementations in 64 bits: embedding lookup, its gradient by sorted tokens
(whole table, added, touched rows), the AdamW step of the touched rows, AdamW over many tensors with moments in 32 and
in 8 bits; and what the calls refuse.

Tolerances follow from fp32 arithmetic: u = 2^-24 is the largest relative error of one rounding, a sum of k
terms in any order is off by at most (k - 1) u (1 + small) times the sum of the magnitudes, and an output type with f fraction
bits adds 2^-(f+1) of the value (half the smallest subnormal at least).
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
    from paper_2211_10280_b200 import operators

    return operators


def _rand(shape, dtype=F32, std=1.0, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


def _ids(n, V, law, seed=0, padding=None, dtype=torch.int64):
    r = np.random.default_rng(seed)
    if law == "same":
        ids = np.full(n, V // 2)
    elif law == "distinct":
        ids = r.permutation(V)[:n]
    elif law == "zipf":
        ids = np.minimum(np.exp(r.random(n) * np.log(V + 1)) - 1, V - 1).astype(np.int64)
    elif law == "runs":       # tokens that come about 40 times each
        ids = r.integers(0, max(1, min(V, n // 40 + 1)), n)
    else:
        ids = r.integers(0, V, n)
    if padding is not None:
        ids = np.where(r.random(n) < 0.3, padding, ids)
    return torch.from_numpy(np.ascontiguousarray(ids)).to(dtype).cuda()


def _close(got, want, slack, dtype=F32):
    """|got - want| <= slack + the output type's rounding of want"""
    got, want, slack = got.double().cpu(), want.double().cpu(), slack.double().cpu() if torch.is_tensor(slack) else slack
    rel, least = LAST[dtype]
    excess = (got - want).abs() - (slack + (want.abs() + slack) * rel + least)
    assert not torch.isnan(got).any()
    assert excess.max().item() <= 0 if excess.numel() else True, (excess.max().item(), (got - want).abs().max().item())


# ---------------------------------------------------------------- lookup
@gpu
@pytest.mark.parametrize("d", [1, 2, 3, 8, 30, 64, 300, 301, 1030])
@pytest.mark.parametrize("table_type,out_type", [(F32, F32), (F32, BF16), (BF16, BF16), (F16, F32), (F16, F16), (BF16, F16)])
def test_lookup(d, table_type, out_type):
    V = 97
    table = _rand((V, d), table_type)
    for n, wide in ((0, True), (1, True), (5, False), (1000, False)):
        ids = _ids(n, V, "uniform", n, padding=-1, dtype=torch.int64 if wide else torch.int32)
        e = _ops().Embedding(V, d, max_tokens=n, scale=1.7, padding_id=-1)
        got = e.lookup(table, ids, dtype=out_type)
        want = table.double().cpu()[ids.long().cpu().clamp(min=0)] * np.float32(1.7).item()
        want[ids.cpu() < 0] = 0
        assert got.dtype == out_type and got.shape == (n, d)
        _close(got, want, want.abs() * U, out_type)
        e.check()


@gpu
def test_lookup_strides_shapes_and_rows_that_hold_nan():
    V, d = 50, 24
    wide = _rand((V, 40), BF16)
    table = wide[:, 8:32]
    ids = _ids(6, V, "uniform").view(2, 3)
    for off in (0, 1, 3):           # also tables and outputs that begin between two vectors
        t = wide.view(-1)[off:off + 40 * (V - 1) + d].as_strided((V, d), (40, 1))
        out = torch.zeros(6, 31, device="cuda")[:, 2:26]
        e = _ops().Embedding(V, d, max_tokens=6, scale=3.0)
        e.lookup(t, ids, out=out)
        _close(out, t.double()[ids.view(-1)] * 3, 0, F32)
    assert e.lookup(table, ids).shape == (2, 3, d)
    wide[~torch.isin(torch.arange(V, device="cuda"), ids)] = float("nan")
    assert not torch.isnan(e.lookup(table, ids)).any()
    wide[ids[0, 0]] = float("inf")
    assert torch.isinf(e.lookup(table, ids)[0, 0]).all()


@gpu
def test_ids_outside_the_vocabulary_read_as_no_token_and_are_reported():
    V, d = 20, 12
    table, grad = _rand((V, d)), _rand((5, d), seed=1)
    e = _ops().Embedding(V, d, max_tokens=5)
    for dtype, far in ((torch.int32, 2 ** 31 - 1), (torch.int64, 2 ** 40 + 3)):
        ids = torch.tensor([1, V, 3, -1, far], dtype=dtype, device="cuda")
        out = e.lookup(table, ids)
        assert torch.equal(out[[0, 2]], table[[1, 3]]) and not out[[1, 3, 4]].any()
        with pytest.raises(B.TensairError) as err:
            e.check()
        assert err.value.code == B.EBADTOKEN
        e.check()
        g = e.gradient(grad, ids)
        assert torch.equal(g[[1, 3]], grad[[0, 2]]) and not g[[x for x in range(V) if x not in (1, 3)]].any()
        with pytest.raises(B.TensairError):
            e.check()


# ---------------------------------------------------------------- gradient
def _sums(grad, ids, V, scale):
    """G, and per entry the bound of its fp32 error: (terms + 1) roundings of the sum of magnitudes."""
    ids, grad = ids.long().cpu(), grad.double().cpu()
    held = (ids >= 0) & (ids < V)
    total, size = (torch.zeros(V, grad.shape[1], dtype=torch.float64) for _ in range(2))
    total.index_add_(0, ids[held], grad[held])
    size.index_add_(0, ids[held], grad[held].abs())
    count = torch.bincount(ids[held], minlength=V)
    s = np.float32(scale).item()
    return total * s, size * s * ((count + 1) * U * 1.01)[:, None], count


LENGTHS = [0, 1, 2, 7, 8, 9, 17, 1000, 1024, 1025, 4097, 8191, 8192, 20_011, 40_000, 140_003]


@gpu
@pytest.mark.parametrize("n", LENGTHS)
@pytest.mark.parametrize("law", ["zipf", "same", "runs", "distinct"])
def test_gradient_of_the_whole_table(n, law):
    V, d, scale = 150_001 if law == "distinct" else 30_011, 20 if n > 20_000 else 36, 1.3
    ids = _ids(n, V, law, n, padding=-7, dtype=torch.int32 if n % 2 else torch.int64)
    grad = _rand((n, d), F32, seed=n)
    grad[ids < 0] = float("nan")                    # rows without a token are not read
    e = _ops().Embedding(V, d, max_tokens=max(n, 10_000), scale=scale, padding_id=-7)
    want, slack, count = _sums(grad, ids, V, scale)
    got = e.gradient(grad, ids)
    _close(got, want, slack)
    assert torch.equal(got, e.gradient(grad, ids))  # the same bits again
    # added to what is there: rows that do not occur keep their bits, NaN included
    old = _rand((V, d), F32, seed=3)
    old[count == 0] = float("nan")
    new = e.gradient(grad, ids, out=old.clone(), accumulate=True)
    assert torch.isnan(new[(count == 0).cuda()]).all()
    held = count > 0
    _close(new.cpu()[held], want[held] + old.double().cpu()[held], (slack + want.abs() * U)[held])
    # the touched rows alone
    row, rows, m = e.gradient_rows(grad, ids, out=(torch.full((n,), -5, dtype=torch.int32, device="cuda"),
                                                   torch.full((n, d), 9.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")))
    m = int(m)
    assert m == int(held.sum()) and torch.equal(row[:m].cpu().long(), held.nonzero()[:, 0])
    assert torch.equal(rows[:m], got[row[:m].long()])
    assert (row[m:] == -5).all() and (rows[m:] == 9).all()
    e.check()


@gpu
@pytest.mark.parametrize("d", [1, 2, 3, 8, 30, 64, 300, 301, 1030])
@pytest.mark.parametrize("grad_type,out_type", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F32, F16), (F16, BF16)])
def test_gradient_types_and_widths(d, grad_type, out_type):
    V, n = 500, 1500
    ids = _ids(n, V, "zipf", d)
    grad = _rand((n, d), grad_type, seed=d)
    e = _ops().Embedding(V, d, max_tokens=n, scale=0.5)
    want, slack, _ = _sums(grad, ids, V, 0.5)
    got = e.gradient(grad, ids, dtype=out_type)
    assert got.dtype == out_type
    _close(got, want, slack, out_type)
    old = _rand((V, d), out_type, seed=2)
    new = e.gradient(grad, ids, out=old.clone(), accumulate=True)
    _close(new, want + old.double().cpu(), slack + (want.abs() + old.double().cpu().abs()) * U, out_type)


@gpu
@pytest.mark.parametrize("V", [1, 2, 1023, 1024, 1 << 20, (1 << 20) + 5, 3_000_000])
def test_gradient_over_vocabularies_of_one_to_three_digits(V):
    for n in (100, 5000, 140_000):
        d = 4
        ids = _ids(n, V, "uniform", 5)
        grad = _rand((n, d), seed=n)
        e = _ops().Embedding(V, d, max_tokens=n)
        want, slack, count = _sums(grad, ids, V, 1.0)
        row, rows, m = e.gradient_rows(grad, ids)
        m = int(m)
        assert torch.equal(row[:m].cpu().long(), (count > 0).nonzero()[:, 0])
        _close(rows[:m], want[count > 0], slack[count > 0])


@gpu
@pytest.mark.parametrize("n", [63, 64, 65, 2047, 2048, 16_383, 16_384, 16_385, 65_536, 131_071, 131_072, 131_073])
def test_gradient_where_the_sort_changes_its_way(n):
    d = 3
    for V, law in ((1 << 30, "uniform"), (70_000, "zipf"), (5000, "runs")):
        ids = _ids(n, V, law, n, padding=-1, dtype=torch.int32)
        grad = _rand((n, d), seed=n)
        e = _ops().Embedding(V, d, max_tokens=n, padding_id=-1)
        row, rows, m = e.gradient_rows(grad, ids)
        m = int(m)
        held = ids >= 0
        want, index = torch.unique(ids[held].long(), return_inverse=True)
        assert m == want.numel() and torch.equal(row[:m].long(), want)
        total, size = (torch.zeros(m, d, dtype=torch.float64, device="cuda") for _ in range(2))
        total.index_add_(0, index, grad[held].double())
        size.index_add_(0, index, grad[held].double().abs())
        _close(rows[:m], total, size * (torch.bincount(index, minlength=m) + 1)[:, None] * U * 1.01)
        if V < 1 << 20:
            table = e.gradient(grad, ids)
            assert torch.equal(table[want], rows[:m]) and int((table != 0).any(1).sum()) == int((rows[:m] != 0).any(1).sum())


@gpu
def test_gradient_of_strided_and_broadcast_rows():
    V, d, n = 40, 24, 300
    ids = _ids(n, V, "zipf")
    e = _ops().Embedding(V, d, max_tokens=n, scale=2.0)
    wide = _rand((n, 50), BF16)
    out = torch.full((V, 33), 4.0, device="cuda")
    for off in (0, 1, 4):
        grad = wide[:, off:off + d]
        want, slack, _ = _sums(grad, ids, V, 2.0)
        e.gradient(grad, ids, out=out[:, 5:5 + d])
        _close(out[:, 5:5 + d], want, slack)
        assert (out[:, :5] == 4).all() and (out[:, 5 + d:] == 4).all()
    one = _rand((1, d))
    want, slack, _ = _sums(one.expand(n, d), ids, V, 2.0)
    _close(e.gradient(one.expand(n, d), ids), want, slack)
    columns = _rand((d, n)).t()
    want, slack, _ = _sums(columns, ids, V, 2.0)
    _close(e.gradient(columns, ids), want, slack)


@gpu
def test_lookup_has_the_gradient_that_differences_give():
    V, d, n = 11, 6, 40
    ids = _ids(n, V, "zipf", padding=-1).view(5, 8)
    table = _rand((V, d)).requires_grad_()
    weight = _rand((5, 8, d), seed=1)
    e = _ops().Embedding(V, d, max_tokens=n, scale=1.5, padding_id=-1)
    (e(table, ids) * weight).sum().backward()
    with torch.no_grad():
        for row, col in ((0, 0), (1, 5), (10, 2), (4, 3)):
            sides = []
            for h in (0.5, -0.5):      # the lookup is linear in the table, so a wide step is exact but for rounding
                t = table.detach().clone()
                t[row, col] += h
                sides.append((e.lookup(t, ids).double() * weight.double()).sum().item())
            bound = 2 * U * (e.lookup(table.detach().abs() + 0.5, ids).double() * weight.double().abs()).sum().item() * 4
            assert abs(table.grad[row, col].item() - (sides[0] - sides[1])) <= bound


@gpu
def test_tables_whose_offsets_pass_32_bits():
    V, d = 2_200_000, 1024            # 2.25e9 elements, 4.5 GB
    table = torch.zeros(V, d, dtype=BF16, device="cuda")
    ids = torch.tensor([V - 1, 0, 2_097_151, 2_097_152, V - 1], device="cuda")
    rows = _rand((5, d), BF16)
    rows[4] = rows[0]
    table[ids] = rows
    e = _ops().Embedding(V, d, max_tokens=5)
    assert torch.equal(e.lookup(table, ids), rows)
    table.zero_()
    e.gradient(rows, ids, out=table, accumulate=True)
    assert torch.equal(table[ids[1:4]], rows[1:4]) and torch.equal(table[-1], rows[0] + rows[4])
    assert int((table != 0).sum()) == int((table[ids[:4]] != 0).sum())


# ---------------------------------------------------------------- AdamW
HYPER = dict(lr=2e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)


def _adamw64(p, g, m, v, step, lr, betas, eps, weight_decay):
    """(p, m, v) in 64 bits, and the bounds of their fp32 errors (before the rounding of the stored type).

    m and v: three roundings of each of their two terms, and the float constants' own.  The update's
    quotient: the errors of m (which may cancel) over the denominator, and half of v's relative error plus five roundings."""
    b1, b2 = betas
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    em, ev = 5 * U * (b1 * m.abs() + (1 - b1) * g.abs()), 6 * U * v1
    low = (v1 / (1 - b2 ** step)).sqrt() + eps
    size = lr / (1 - b1 ** step)
    p1 = p * (1 - lr * weight_decay) - size * m1 / low
    return p1, m1, v1, 2 * U * p.abs() + size * (em + 10 * U * m1.abs()) / low + 2.0 ** -140, em + 2.0 ** -140, ev + 2.0 ** -140


def _check_rows_step(n, V, d, table_type, grad_type, law, scale=1.0, grad_scale=None, pad=0):
    ids = _ids(n, V, law, n, padding=-1)
    grad = _rand((n, d), grad_type, std=1e-2)
    table = _rand((V, d + pad), table_type, std=0.1, seed=1)[:, pad:]
    m, v = _rand((V, d), std=1e-3, seed=2), _rand((V, d), std=1e-3, seed=3).square()
    e = _ops().Embedding(V, d, max_tokens=n, scale=scale, padding_id=-1)
    want, slack, count = _sums(grad, ids, V, scale)
    if grad_scale is not None:
        want, slack = want * grad_scale.item(), slack * grad_scale.item()
    slack = slack + 2 * U * want.abs()
    p0, m0, v0 = table.clone(), m.clone(), v.clone()
    e.adamw(grad, ids, table, m, v, step=3, grad_scale=grad_scale, **HYPER)
    p1, m1, v1, ep, em, ev = _adamw64(p0.double().cpu(), want, m0.double().cpu(), v0.double().cpu(), 3, **HYPER)
    # the gradient's own error goes into m and v linearly, and through both into the update
    em2, ev2 = 0.1 * slack, 0.001 * 2 * want.abs() * slack
    root = (v1 / (1 - 0.999 ** 3)).sqrt() + 1e-8
    ep = ep + 2e-2 / (1 - 0.9 ** 3) * (em2 / root + m1.abs() / root * ev2 / v1.clamp(min=1e-300))
    held = count > 0
    _close(m.cpu()[held], m1[held], (em + em2)[held])
    _close(v.cpu()[held], v1[held], (ev + ev2)[held])
    _close(table.cpu()[held], p1[held], ep[held], table_type)
    for new, old in ((table, p0), (m, m0), (v, v0)):
        assert torch.equal(new.cpu()[~held], old.cpu()[~held])


@gpu
@pytest.mark.parametrize("n,V,d,law", [(1, 9, 1, "zipf"), (3, 5, 300, "same"), (500, 97, 33, "zipf"), (9000, 3000, 64, "zipf"),
                                       (20_000, 50, 24, "runs"), (5000, 20_000, 30, "distinct"), (10_000, 40, 20, "same")])
@pytest.mark.parametrize("table_type,grad_type", [(F32, F32), (F32, BF16), (BF16, BF16), (F16, F32)])
def test_adamw_of_the_touched_rows(n, V, d, law, table_type, grad_type):
    _check_rows_step(n, V, d, table_type, grad_type, law)


@gpu
def test_adamw_of_the_touched_rows_scaled_and_strided():
    _check_rows_step(700, 60, 32, F32, F32, "zipf", scale=1.5, grad_scale=torch.tensor(0.25, device="cuda"), pad=3)
    # a factor that is not finite leaves everything as it is
    V, d = 20, 8
    t, m, v = _rand((V, d)), _rand((V, d)), _rand((V, d)).square()
    before = [x.clone() for x in (t, m, v)]
    e = _ops().Embedding(V, d, max_tokens=64)
    for bad in (float("nan"), float("inf")):
        e.adamw(_rand((64, d)), _ids(64, V, "zipf"), t, m, v, step=1, grad_scale=torch.tensor(bad, device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip(before, (t, m, v)))
    # no tokens, or none that counts
    e.adamw(_rand((0, d)), _ids(0, V, "zipf"), t, m, v, step=1)
    e.adamw(_rand((3, d)), torch.full((3,), V, device="cuda"), t, m, v, step=1)
    assert all(torch.equal(x, y) for x, y in zip(before, (t, m, v)))


SIZES = [1, 3, 4, 255, 256, 257, 1000, 4096, 4097, 70_001]


def _flats(sizes, dtype, off, seed, std=1.0):
    """Tensors of the given sizes one behind the other in one buffer, from element `off` on."""
    flat = _rand(sum(sizes) + off, dtype, std, seed)
    at = np.cumsum([off] + sizes)
    return [flat[a:a + n] for a, n in zip(at, sizes)]


@gpu
@pytest.mark.parametrize("param_type,grad_type", [(F32, F32), (F32, BF16), (BF16, BF16), (F16, F16), (BF16, F32)])
@pytest.mark.parametrize("off", [0, 1, 2])
@pytest.mark.parametrize("copied", [None, BF16, F16])
def test_adamw_with_32_bit_moments(param_type, grad_type, off, copied):
    p, g = _flats(SIZES, param_type, off, 0), _flats(SIZES, grad_type, 0 if off == 2 else off, 1, 0.1)
    m, v = _flats(SIZES, F32, off, 2, 0.01), [x.square_() for x in _flats(SIZES, F32, off, 3, 0.1)]
    copies = _flats(SIZES, copied, off, 4) if copied else None
    lr_factors, decay_factors = [1 + i % 3 for i in range(len(SIZES))], [i % 2 for i in range(len(SIZES))]
    before = [[x.double().cpu() for x in xs] for xs in (p, m, v)]
    opt = _ops().AdamW(p, state_bits=32, copies=copies, state=dict(m=m, v=v), step=4, lr_factors=lr_factors,
                       decay_factors=decay_factors, **HYPER)
    opt.step(g, grad_scale=torch.tensor(0.5, device="cuda"))
    assert opt.step_count == 5
    for i in range(len(SIZES)):
        h = dict(HYPER, lr=HYPER["lr"] * lr_factors[i], weight_decay=HYPER["weight_decay"] * decay_factors[i])
        p1, m1, v1, ep, em, ev = _adamw64(before[0][i], g[i].double().cpu() * 0.5, before[1][i], before[2][i], 5, **h)
        _close(m[i], m1, em)
        _close(v[i], v1, ev)
        _close(p[i], p1, ep, param_type)
        if copied:
            _close(copies[i], p1, ep, copied)


@gpu
def test_adamw_follows_many_steps_and_leaves_out_what_has_no_gradient():
    sizes = [5, 300] * 200            # more tensors than one launch takes
    p = _flats(sizes, F32, 0, 0)
    want = [x.double().cpu() for x in p]
    m, v = ([torch.zeros_like(x) for x in want] for _ in range(2))
    opt = _ops().AdamW(p, state_bits=32, **HYPER)
    bound = [torch.zeros_like(x) for x in want]
    for t in range(1, 6):
        g = _flats(sizes, F32, 0, t)
        use = [None if i == 7 else x for i, x in enumerate(g)]
        opt.step(use)
        for i, x in enumerate(use):
            if x is not None:
                want[i], m[i], v[i], ep, em, ev = _adamw64(want[i], x.double().cpu(), m[i], v[i], t, **HYPER)
                # moments carry their errors on: at most t steps' worth, and so does p
                bound[i] = bound[i] + t * ep * 2 + want[i].abs() * U
    for i in range(len(sizes)):
        _close(p[i], want[i], bound[i])
    assert torch.equal(p[7], _flats(sizes, F32, 0, 0)[7])


@gpu
def test_adamw_keeps_nan_and_inf_where_they_are():
    for bits in (32, 8):
        p, g = _flats([1000], F32, 0, 0), _flats([1000], F32, 0, 1)
        clean = [x.clone() for x in p]
        a = _ops().AdamW(clean, state_bits=bits, **HYPER)
        a.step([g[0].clone()])
        g[0][300], g[0][301] = float("nan"), float("inf")
        b = _ops().AdamW(p, state_bits=bits, **HYPER)
        b.step(g)
        assert torch.isnan(p[0][300]) and not torch.isfinite(p[0][301])
        rest = torch.ones(1000, dtype=torch.bool, device="cuda")
        rest[300:302] = False
        assert torch.equal(p[0][rest], clean[0][rest])
        for x, y in zip(b.moments(0), a.moments(0)):
            assert not torch.isfinite(x[300:302]).any()
            top = y[256:512].abs().argmax().item() + 256
            if top not in (300, 301):      # the block's scale is that of its finite elements
                assert torch.equal(x[rest], y[rest])


def _philox(counter, key):
    c, k = [int(x) for x in counter], list(key)
    return B.tensair_philox4x32_10(c, k)


def _stored(x, largest, bits16, positive):
    """The e4m3 value that |x| / (largest / 448) is stored as, in 64 bits, and how near the choice was."""
    s = abs(x) / largest * 448 if largest > 0 else 0.0
    if positive and x > 0:
        s = max(s, 2.0 ** -9)
    if s < 2.0 ** -6:
        q = np.round(s * 512) / 512
        return q, abs(s * 512 - np.floor(s * 512) - 0.5)
    gap = 2.0 ** (np.floor(np.log2(s)) - 3)
    f = s / gap - np.floor(s / gap) + (bits16 + 0.5) / 65536
    return min(448.0, (np.floor(s / gap) + (f >= 1)) * gap), min(abs(f - 1), abs(f), abs(2 - f))


@gpu
@pytest.mark.parametrize("param_type,grad_type", [(F32, BF16), (BF16, BF16), (F32, F32), (F16, F16)])
@pytest.mark.parametrize("off", [0, 3])
def test_adamw_with_8_bit_moments(param_type, grad_type, off):
    sizes, seed = [700, 1, 256, 3000], (5 << 32) + 9
    p, g = _flats(sizes, param_type, off, 0), _flats(sizes, grad_type, off, 1, 0.1)
    g[3][::7] *= 1e-6                   # small elements beside large ones
    copies = _flats(sizes, BF16, off, 4)
    opt = _ops().AdamW(p, state_bits=8, copies=copies, seed=seed, **HYPER)
    opt.step(g)
    first = [opt.moments(i) for i in range(len(sizes))]
    before = [x.double().cpu() for x in p]
    scales = [(opt.m_scale[i].clone(), opt.v_scale[i].clone()) for i in range(len(sizes))]
    opt.step(g)
    block0 = 0
    for i, n in enumerate(sizes):
        # a second step from what the first one stored
        p1, m1, v1, ep, em, ev = _adamw64(before[i], g[i].double().cpu(), first[i][0].double().cpu(), first[i][1].double().cpu(), 2, **HYPER)
        # the kernel squares value * scale in fp32: two roundings more in v
        _close(p[i], p1, ep * 2, param_type)
        _close(copies[i], p1, ep * 2, BF16)
        for code, scale, x, positive in ((opt.m[i], opt.m_scale[i], m1, False), (opt.v[i], opt.v_scale[i], v1.sqrt(), True)):
            largest = torch.stack([x[a:a + 256].abs().max() for a in range(0, n, 256)])
            _close(scale, largest / 448, largest / 448 * 8 * U)
            code = code.double().cpu()
            for j in list(range(0, n, 37)) + [n - 1]:
                group = (block0 + j // 256) * 32 + j % 256 // 8
                words = _philox([group & 0xFFFFFFFF, group >> 32, 2, 5 << 24], [seed & 0xFFFFFFFF, seed >> 32])
                q, margin = _stored(x[j].item(), largest[j // 256].item(), words[j % 8 // 2] >> (16 * (j % 2)) & 0xFFFF, positive)
                if margin > 1e-4:      # not within fp32's error of the other neighbour
                    assert abs(code[j].item()) == q, (i, j)
                    assert q == 0 or np.sign(code[j].item()) == np.sign(x[j].item())
            if positive:
                assert (code[x > 0] > 0).all()
        block0 += -(-n // 256)
    del scales
    # the same steps give the same bits
    q = _flats(sizes, param_type, off, 0)
    again = _ops().AdamW(q, state_bits=8, seed=seed, **HYPER)
    again.step(g)
    again.step(g)
    assert all(torch.equal(x, y) for x, y in zip(p, q))
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(opt.v + opt.m, again.v + again.m))


@gpu
def test_8_bit_moments_are_those_of_separately_rounded_operations():
    """Every product, sum, root and quotient that leads to what is stored is one rounded fp32 operation: the scales have the bits
    that a program of separate operations gives, starting each step from what the step before stored."""
    n = 256 * 400
    g = _rand((n,), BF16, 1e-3)
    for beta1, beta2 in ((0.0, 0.0), (0.9, 0.999)):
        opt = _ops().AdamW([torch.zeros(n, device="cuda")], state_bits=8, betas=(beta1, beta2))
        m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        for _ in range(3):
            opt.step([g])
            x = g.float()
            m = m * beta1 + x * (1 - beta1)
            v = v * beta2 + (x * x) * (1 - beta2)
            for kept, scale in ((m, opt.m_scale[0]), (v.sqrt(), opt.v_scale[0])):
                assert torch.equal(scale, kept.abs().view(-1, 256).amax(1) * torch.tensor(1 / 448, dtype=torch.float32))
            # what the next step starts from
            m = (opt.m[0].float().view(-1, 256) * opt.m_scale[0][:, None]).view(-1)
            v = (opt.v[0].float().view(-1, 256) * opt.v_scale[0][:, None]).view(-1).square()


@gpu
def test_8_bit_second_moments_follow_a_gradient_that_changes():
    n = 256 * 64
    p = [torch.zeros(n, device="cuda")]
    g = torch.full((n,), 1e-2, device="cuda")
    g[::256] = 1.0                       # the element that sets every block's scale
    opt = _ops().AdamW(p, state_bits=8, lr=0.0, betas=(0.9, 0.99), weight_decay=0.0)
    exact = 0.0
    for size in (1e-2, 1e-3):
        g.masked_fill_(g < 0.5, size)
        for _ in range(700):
            opt.step([g])
            exact = 0.99 * exact + 0.01 * size ** 2
        v = opt.moments(0)[1][g < 0.5].double()
        # A step moves the root by a share s <= (1 - beta2) / 2 of itself, rounded to neighbours that are c <= 1/8 apart: up
        # or down by c with probability s / c, which adds at most s c = 6.3e-4 of v per step to its mean, 1 / (1 - beta2) =
        # 100 steps' worth in all: 6.3 % of v, 3.1 % of the root.  The mean over 16,320 elements wanders by under 1 %.
        assert abs(v.sqrt().mean().item() / exact ** 0.5 - 1) < 0.05
    assert (opt.moments(0)[1] > 0).all()


@gpu
def test_a_block_of_vanishing_moments_is_stored_as_zeros():
    p = [torch.ones(512, device="cuda")]
    opt = _ops().AdamW(p, state_bits=8, lr=0.1, weight_decay=0.0)
    g = torch.zeros(512, device="cuda")
    g[256:] = 1e-34
    opt.step([g])
    assert not opt.m[0].float().any() and not opt.m_scale[0].any() and torch.isfinite(p[0]).all()
    opt.step([torch.ones(512, device="cuda")])
    assert torch.isfinite(p[0]).all() and (opt.moments(0)[0] > 0).all()


# ---------------------------------------------------------------- streams, graphs
@gpu
def test_calls_of_two_streams_and_of_a_graph():
    V, d, n = 1000, 64, 3000
    table, grad, ids = _rand((V, d)), _rand((n, d), seed=1), _ids(n, V, "zipf")
    e = _ops().Embedding(V, d, max_tokens=n)
    want_rows, want = e.lookup(table, ids), e.gradient(grad, ids)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(5):                   # the workspace changes hands between the streams
        for s in (a, b):
            with torch.cuda.stream(s):
                outs.append(e.gradient(grad, ids))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in outs)
    p = [torch.ones(5000, device="cuda")]
    q = [torch.ones(5000, device="cuda")]
    g = [_rand((5000,))]
    out, rows = torch.empty_like(want), torch.empty_like(want_rows)
    graph = torch.cuda.CUDAGraph()
    opt = _ops().AdamW(p, state_bits=32)
    with torch.cuda.graph(graph):
        e.lookup(table, ids, out=rows)
        e.gradient(grad, ids, out=out)
        opt.step(g)
    out.fill_(3)
    rows.fill_(3)
    graph.replay()
    torch.cuda.synchronize()
    _ops().AdamW(q, state_bits=32).step(g)
    assert torch.equal(out, want) and torch.equal(rows, want_rows) and torch.equal(p[0], q[0])


# ---------------------------------------------------------------- the example
@gpu
@pytest.mark.parametrize("state_bits,dense", [(8, False), (32, False), (32, True)])
def test_next_token_model_learns_from_streamed_embeddings(state_bits, dense):
    from paper_2211_10280_b200 import next_token

    r = next_token.train(steps=60, V=1000, rows=512, state_bits=state_bits, dense=dense, report=30)
    # a uniform guess costs ln 1000 = 6.9; the stream's own entropy is under 0.3 * 6.9 + 0.7 = 2.8
    assert abs(r["losses"][0] - 6.9) < 1.5 and r["losses"][-1] < r["losses"][0] - 0.5
    unseen = ~r["seen"]
    if unseen.any():
        assert torch.equal(r["after"][unseen], r["before"][unseen])
    assert not torch.equal(r["after"][r["seen"]], r["before"][r["seen"]])


# ---------------------------------------------------------------- refusals
def _fake(**kw):
    """Arguments that pass every check, over addresses that nothing reads: a refused call enqueues nothing."""
    base = dict(tokens=B.Tokens(ids=4096, n=10, V=100, padding_id=-1, type=B.INT32),
                grad=B.Rows(data=4096, stride=8, d=8, type=B.FLOAT32), out=B.Rows(data=4096, stride=8, d=8, type=B.FLOAT32),
                m=B.Rows(data=4096, stride=8, d=8, type=B.FLOAT32), v=B.Rows(data=4096, stride=8, d=8, type=B.FLOAT32),
                adamw=B.Adamw(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1), workspace=4096, bytes=1 << 30)
    for key, fields in kw.items():
        if isinstance(fields, dict):
            for f, x in fields.items():
                setattr(base[key], f, x)
        else:
            base[key] = fields
    return base


def _calls(a):
    L = B.lib()
    return {
        "lookup": lambda: L.tensair_embedding_lookup(a["tokens"], a["out"], a["grad"], 1.0, None),
        "gradient": lambda: L.tensair_embedding_gradient(a["tokens"], a["grad"], a["out"], 1.0, 0, a["workspace"], a["bytes"], None),
        "rows": lambda: L.tensair_embedding_gradient_rows(a["tokens"], a["grad"], 1.0, 4096, a["out"], 4096, a["workspace"], a["bytes"], None),
        "adamw": lambda: L.tensair_embedding_adamw(a["tokens"], a["grad"], 1.0, a["out"], a["m"], a["v"], a["adamw"], a["workspace"],
                                                   a["bytes"], None)}


ALL = ("lookup", "gradient", "rows", "adamw")
SUMS = ("gradient", "rows", "adamw")
REFUSED = [
    (dict(tokens=None), ALL, "tokens"), (dict(tokens=dict(V=0)), ALL, "V must"), (dict(tokens=dict(V=2 ** 30 + 1)), ALL, "V must"),
    (dict(tokens=dict(n=2 ** 30 + 1)), ALL, "n must"), (dict(tokens=dict(type=B.FLOAT32)), ALL, "ids must"),
    (dict(tokens=dict(ids=None)), ALL, "ids are NULL"), (dict(tokens=dict(ids=4098)), ALL, "aligned"),
    (dict(tokens=dict(error=4097)), ALL, "error word"), (dict(out=None), ALL, ""), (dict(grad=None), ALL, ""),
    (dict(out=dict(data=None)), ALL, ""), (dict(grad=dict(data=None)), ALL, ""), (dict(out=dict(stride=7)), ALL, "stride"),
    (dict(grad=dict(stride=7)), ALL, "stride"), (dict(out=dict(stride=2 ** 31)), ALL, "stride"), (dict(out=dict(d=0)), ALL, "d not in"), (dict(grad=dict(d=4)), ALL, "width"),
    (dict(grad=dict(type=3)), ALL, "type"), (dict(out=dict(type=7)), ALL, ""), (dict(grad=dict(data=4098)), ALL, "alignment"),
    (dict(out=dict(type=B.BFLOAT16)), ("rows",), "must be TENSAIR_FLOAT32"), (dict(m=dict(type=B.FLOAT16)), ("adamw",), "m and v"),
    (dict(v=None), ("adamw",), "v: NULL"), (dict(m=dict(d=9)), ("adamw",), "m:"), (dict(adamw=None), ("adamw",), "adamw"),
    (dict(adamw=dict(step=0)), ("adamw",), "step"), (dict(adamw=dict(lr=float("nan"))), ("adamw",), "lr"),
    (dict(adamw=dict(beta1=1.0)), ("adamw",), "beta"), (dict(adamw=dict(eps=-1.0)), ("adamw",), "eps"),
    (dict(adamw=dict(grad_scale=4097)), ("adamw",), "grad_scale"), (dict(workspace=None), SUMS, "workspace"),
    (dict(workspace=4100), SUMS, "workspace"), (dict(bytes=100), SUMS, "workspace"),
]


@pytest.mark.parametrize("change,calls,word", REFUSED)
def test_embedding_calls_refuse(change, calls, word):
    for name in calls:
        rc = _calls(_fake(**change))[name]()
        assert rc == (B.ENOMEM if "bytes" in change else B.EINVAL), name
        assert word in B.lib().tensair_last_error(None).decode()


def test_workspace_sizes():
    size = C.c_uint64()

    def bytes_of(n, V=1000, d=64):
        assert B.lib().tensair_embedding_workspace_bytes(n, V, d, C.byref(size)) == B.OK
        return size.value

    lengths = sorted({x for p in range(0, 21) for x in (2 ** p - 1, 2 ** p, 2 ** p + 1)} | {131_072, 131_073, 2 ** 30})
    sizes = [bytes_of(n) for n in lengths]
    assert sizes == sorted(sizes)        # a workspace serves every smaller batch
    for bad in ((2 ** 30 + 1, 10, 8), (5, 0, 8), (5, 10, 0), (5, 10, 2 ** 20 + 1)):
        assert B.lib().tensair_embedding_workspace_bytes(*bad, C.byref(size)) == B.EINVAL
    assert B.lib().tensair_embedding_workspace_bytes(5, 10, 8, None) == B.EINVAL


@pytest.mark.parametrize("change,word", [
    (dict(param=None), "NULL"), (dict(grad=None), "NULL"), (dict(m=None), "NULL"), (dict(v=None), "NULL"), (dict(param=4098), "aligned"),
    (dict(m=4098), "aligned"), (dict(param_type=5), "param_type"), (dict(grad_type=3), "grad_type"),
    (dict(copy=4096, copy_type=B.FLOAT32), "copy"), (dict(lr_factor=-1.0), "lr_factor"), (dict(decay_factor=float("inf")), "decay_factor"),
    (dict(n=2 ** 40), "2^40")])
def test_adamw_step_refuses(change, word):
    t = (B.AdamwTensor * 1)(B.AdamwTensor(param=4096, grad=4096, m=4096, v=4096, n=10, lr_factor=1, decay_factor=1))
    for f, x in change.items():
        setattr(t[0], f, x)
    h = B.Adamw(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    assert B.lib().tensair_adamw_step(t, 1, 32, h, None) == B.EINVAL
    assert word in B.lib().tensair_last_error(None).decode()


def test_adamw_step_refuses_its_other_arguments():
    t = (B.AdamwTensor * 1)(B.AdamwTensor(param=4096, grad=4096, m=4096, v=4096, n=10, lr_factor=1, decay_factor=1))
    h = B.Adamw(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    L = B.lib()
    assert L.tensair_adamw_step(t, 1, 16, h, None) == B.EINVAL
    assert L.tensair_adamw_step(t, 1, 8, h, None) == B.EINVAL and "m_scale" in L.tensair_last_error(None).decode()
    assert L.tensair_adamw_step(None, 1, 32, h, None) == B.EINVAL
    assert L.tensair_adamw_step(t, 1, 32, None, None) == B.EINVAL
    assert L.tensair_adamw_step(None, 0, 32, h, None) == B.OK
    t[0].n, t[0].param = 0, None
    assert L.tensair_adamw_step(t, 1, 32, h, None) == B.OK      # nothing to do


def test_binding_structures_match_the_header(tmp_path):
    import subprocess

    names = {"tensair_tokens": B.Tokens, "tensair_rows": B.Rows, "tensair_adamw": B.Adamw, "tensair_adamw_tensor": B.AdamwTensor}
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


@gpu
def test_the_python_calls_refuse():
    o = _ops()
    e = o.Embedding(100, 8, max_tokens=10)
    table, ids, grad = _rand((100, 8)), _ids(10, 100, "zipf"), _rand((10, 8))
    bad = [lambda: e.lookup(table.cpu(), ids), lambda: e.lookup(table, ids.cpu()), lambda: e.lookup(table, ids.float()),
           lambda: e.lookup(table[:99], ids), lambda: e.lookup(table.double(), ids), lambda: e.lookup(table, torch.cat([ids, ids])),
           lambda: e.lookup(table.t().contiguous().t(), ids), lambda: e.gradient(grad[:9], ids),
           lambda: e.gradient(grad, ids, accumulate=True), lambda: e.gradient(grad, ids, out=table[:50]),
           lambda: e.gradient_rows(grad, ids, out=(ids.int()[:5], grad, ids.int()[:1])),
           lambda: e.adamw(grad, ids, table, table.half(), table, step=1), lambda: o.AdamW([]), lambda: o.AdamW([table.cpu()]),
           lambda: o.AdamW([table.t()]), lambda: o.AdamW([table], state_bits=4), lambda: o.AdamW([table], copies=[table]),
           lambda: o.AdamW([table], state=dict(m=[table])), lambda: o.AdamW([table]).step([grad]), lambda: o.AdamW([table]).step([]),
           lambda: e.adamw(grad, ids, table, table, table, step=1, grad_scale=torch.ones(2, device="cuda")),
           lambda: e.lookup(table, ids, dtype=torch.float64)]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, B.TensairError)):
            call()
            pytest.fail(f"call {i} was not refused")
