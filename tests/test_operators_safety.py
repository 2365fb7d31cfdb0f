"""The language-model operators where memory, order and lifetimes could go wrong: launches that begin before others end, other
streams, captured calls, tensors that change between calls.  Gradients are small whole numbers here, whose sums are exact in
fp32 in any order, so results are compared bit for bit.
"""
import numpy as np
import pytest
import torch

from paper_2211_10280_b200 import binding as B
from paper_2211_10280_b200 import build as libbuild

gpu = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    libbuild.build()


def _ops():
    from paper_2211_10280_b200 import operators

    return operators


def _batch(n, V, seed, d=4):
    """Zipf ids and whole-number gradients of a batch."""
    r = np.random.default_rng(seed)
    ids = np.minimum(np.exp(r.random(n) * np.log(V + 1)) - 1, V - 1).astype(np.int64)
    return torch.from_numpy(ids).cuda(), torch.from_numpy(r.integers(-4, 5, (n, d)).astype(np.float32)).cuda()


def _touched(ids, grad):
    row, index = torch.unique(ids, return_inverse=True)
    return row, torch.zeros(row.numel(), grad.shape[1], device=grad.device).index_add_(0, index, grad)


def _same_rows(got, ids, grad):
    row, rows, count = got
    want, sums = _touched(ids, grad)
    m = int(count)
    assert m == want.numel() and torch.equal(row[:m].long(), want) and torch.equal(rows[:m], sums)


# ---------------------------------------------------------------- launches that overlap
@gpu
@pytest.mark.parametrize("n,V", [(1025, 5000), (2048, 1 << 20), (4097, 100_000), (8192, 700), (16_384, 1 << 20)])
def test_sorts_in_a_cluster_whose_blocks_start_while_the_device_is_busy(n, V):
    """The blocks of a cluster write into one another's shared memory; whatever else occupies the multiprocessors when they
    start, no total may be lost."""
    e = _ops().Embedding(V, 4, max_tokens=n)
    batches = [_batch(n, V, s) for s in range(12)]
    a = torch.randn(2048, 2048, device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    side, outs = torch.cuda.Stream(), []
    for ids, grad in batches * 2:
        with torch.cuda.stream(side):
            a @ a
        outs.append(e.gradient_rows(grad, ids))
    torch.cuda.synchronize()
    for got, (ids, grad) in zip(outs, batches * 2):
        _same_rows(got, ids, grad)


@gpu
@pytest.mark.parametrize("V", [900, 300_000, (1 << 20) + 77])      # one, two and three digits
@pytest.mark.parametrize("n", [16_385, 40_000, 131_072])
def test_chained_launches_read_what_the_launch_before_them_wrote(n, V):
    """Digit counts and places are rewritten in every pass and every call, by launches that begin while the ones that read the old
    values still run: batches in a row without a pause, every one unlike the one before."""
    e = _ops().Embedding(V, 4, max_tokens=n)
    batches = [_batch(n, V, s) for s in range(4)]
    batches = [(torch.roll(ids, k * 777), torch.roll(grad, k * 777, 0)) for k in range(3) for ids, grad in batches]
    torch.cuda.synchronize()
    outs = [e.gradient_rows(grad, ids) for ids, grad in batches]
    tables = [e.gradient(grad, ids) for ids, grad in batches[:3]]
    torch.cuda.synchronize()
    for got, (ids, grad) in zip(outs, batches):
        _same_rows(got, ids, grad)
    for table, (ids, grad) in zip(tables, batches):
        assert torch.equal(table, torch.zeros(V, 4, device="cuda").index_add_(0, ids, grad))


# ---------------------------------------------------------------- parameters that change between steps
class _Recorder:
    """Stands in for the library: keeps what each AdamW step was asked to do."""

    def __init__(self):
        self.asked = []

    def tensair_adamw_step(self, tensors, count, bits, hyper, stream):
        self.asked.append([(t.param, t.param_type, t.grad, t.grad_type, t.m, t.v, t.copy, t.n) for t in tensors[:count]])
        self.skipped = [t.skip for t in tensors[:count]]
        return 0


@pytest.fixture
def recorder(monkeypatch):
    """operators on CPU tensors over a stand-in for the library."""
    ops, lib = _ops(), _Recorder()
    need = ops._need
    monkeypatch.setattr(ops, "_need", lambda cond, what: need(cond or "no CUDA device" in what, what))
    monkeypatch.setattr(ops, "_current_stream", lambda index: 0)
    monkeypatch.setattr(ops, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(ops, "_settle", lambda device: None)
    monkeypatch.setattr(ops.B, "lib", lambda: lib)
    return lib


def _with_grads(model, dtype=None):
    for p in model.parameters():
        p.grad = torch.ones_like(p, dtype=dtype)


def test_a_step_follows_parameters_that_were_converted(recorder):
    model = torch.nn.Linear(64, 64)
    opt = _ops().AdamW(model.parameters(), state_bits=32)
    for convert, kind in ((lambda: None, B.FLOAT32), (model.bfloat16, B.BFLOAT16), (model.half, B.FLOAT16), (model.float, B.FLOAT32)):
        convert()
        _with_grads(model)
        opt.step()
        for p, (place, param_type, _, grad_type, _, _, _, n) in zip(model.parameters(), recorder.asked[-1]):
            assert place == p.data_ptr() and param_type == kind and grad_type == kind and n == p.numel()
    # the same place with another type: as when the allocator hands a freed block out again
    for p in model.parameters():
        p.data = p.data.view(torch.int32).view(torch.float32)
    _with_grads(model)
    opt.step()
    model.half()
    flat = [p.data for p in model.parameters()]
    _with_grads(model)
    opt.step()
    for p, x in zip(model.parameters(), flat):
        p.data = x.view(torch.bfloat16)
    _with_grads(model)
    opt.step()
    assert [t[1] for t in recorder.asked[-1]] == [B.BFLOAT16] * 2 and [t[0] for t in recorder.asked[-1]] == [t[0] for t in recorder.asked[-2]]


@pytest.mark.parametrize("change", [lambda x: x[:5].clone(), lambda x: x.t().clone(), lambda x: x.double(), lambda x: torch.cat([x, x]),
                                    lambda x: x[:5], lambda x: x.t()])
def test_a_step_refuses_parameters_that_no_longer_fit(recorder, change):
    p = torch.nn.Parameter(torch.ones(8, 6))
    opt = _ops().AdamW([p], state_bits=32)
    grad = torch.ones(8, 6)
    opt.step([grad])
    old, p.data = p.data, change(p.data)
    for _ in range(2):
        if p.data_ptr() != old.data_ptr():
            with pytest.raises(ValueError):
                opt.step([grad])
        with pytest.raises(ValueError):           # in the same place the gradient says that the parameter is another one
            opt.step([torch.ones_like(p)])
    assert len(recorder.asked) == 1 and opt.step_count == 1
    p.data = old
    opt.step([grad])
    assert recorder.asked[0] == recorder.asked[1]


def test_a_gradient_of_another_shape_is_refused(recorder):
    p, q = torch.nn.Parameter(torch.ones(8, 6)), torch.ones(5)
    opt = _ops().AdamW([p, q])
    for bad in (torch.ones(6, 8), torch.ones(48, 1), torch.ones(2, 4, 6)):
        for _ in range(2):
            with pytest.raises(ValueError, match="shape"):
                opt.step([bad, torch.ones(5)])
    for good in (torch.ones(8, 6), torch.ones(48), torch.ones(8, 6), None):
        opt.step([good, torch.ones(5)])
    with pytest.raises(ValueError):
        opt.step([torch.ones(47), torch.ones(5)])
    p.data = torch.ones(6, 8)
    opt.step([torch.ones(6, 8), torch.ones(5)])
    assert len(recorder.asked) == 5


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_and_copies_cannot_be_replaced_unseen(recorder, bits):
    p = torch.ones(300)
    opt = _ops().AdamW([p], state_bits=bits, copies=[torch.empty(300, dtype=torch.bfloat16)])
    for name in ["m", "v", "copies"] + (["m_scale", "v_scale"] if bits == 8 else []):
        with pytest.raises(TypeError):
            getattr(opt, name)[0] = torch.ones(300)
        with pytest.raises(AttributeError):
            setattr(opt, name, [torch.ones(300)])
    place = opt.m[0].data_ptr()
    opt.m[0].data = torch.zeros(300)              # the memory that a step writes is held all the same
    opt.step([torch.ones(300)])
    assert recorder.asked[0][0][4] == place and place in [x.data_ptr() for x in opt._held]


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_converted_parameters_take_the_steps_of_their_type(bits):
    torch.manual_seed(0)
    model = torch.nn.Linear(300, 70).cuda()
    opt = _ops().AdamW(model.parameters(), state_bits=bits, seed=3)
    _with_grads(model)
    opt.step()
    state = {k: [x.clone() for x in xs] for k, xs in opt._state.items()}
    model.bfloat16()
    _with_grads(model)
    twin = [p.detach().clone() for p in model.parameters()]
    _ops().AdamW(twin, state_bits=bits, seed=3, state=state, step=1).step([p.grad for p in model.parameters()])
    opt.step()
    assert all(torch.equal(a, b) for a, b in zip(model.parameters(), twin))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for k in state for a, b in zip(opt._state[k], state[k]))


# ---------------------------------------------------------------- other streams
BUSY = 20_000_000          # clock cycles that a stream is kept busy for: some 10 ms


@gpu
@pytest.mark.parametrize("n", [700, 5000, 40_000])
def test_an_object_is_first_used_on_another_stream_than_it_was_made_on(n):
    """What is pending on the constructor's stream, a write to memory that the allocator hands on, or the error word's zero, is
    over before the first call uses that memory."""
    V = 3000
    ids, grad = _batch(n, V, 1)
    table, bad = torch.zeros(V, 4, device="cuda"), ids.clone()
    bad[5] = V
    size = _ops().Embedding(V, 4, max_tokens=n).workspace_bytes
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        left = torch.empty(size, dtype=torch.uint8, device="cuda")
        word = torch.empty(1, dtype=torch.int32, device="cuda")
        torch.cuda._sleep(BUSY)
        left.fill_(255)
        word.fill_(-1)
        del left, word
        e = _ops().Embedding(V, 4, max_tokens=n)
        with torch.cuda.stream(side):
            got = e.gradient_rows(grad, ids)
            e.lookup(table, bad)
        with pytest.raises(B.TensairError):
            e.check()
        e.check()
        _same_rows(got, ids, grad)


@gpu
def test_check_waits_for_calls_of_other_streams():
    V = 50
    e = _ops().Embedding(V, 4, max_tokens=8)
    table, bad = torch.zeros(V, 4, device="cuda"), torch.full((3,), V, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            torch.cuda._sleep(BUSY)
            e.lookup(table, bad)
        with pytest.raises(B.TensairError):
            e.check()


@gpu
@pytest.mark.parametrize("n", [5000, 40_000])
def test_memory_of_an_object_that_is_gone_is_not_reused_before_its_calls_are_done(n):
    V = 3000
    ids, grad = _batch(n, V, 2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        e = _ops().Embedding(V, 4, max_tokens=n)
        with torch.cuda.stream(side):
            torch.cuda._sleep(BUSY)
            got = e.gradient_rows(grad, ids)
        size = e.workspace_bytes
        del e
        held = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        _same_rows(got, ids, grad)
        del held


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_moments_that_the_optimizer_makes_are_zero_and_held_on_any_stream(bits):
    n = 100_000
    p, q, r = (torch.linspace(-1, 1, n, device="cuda") for _ in range(3))
    g = torch.linspace(0, 2, n, device="cuda")
    again = _ops().AdamW([q], state_bits=bits)
    again.step([g])
    r.copy_(q)
    again.step([g])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    left = [torch.empty(n * bits // 8, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda._sleep(BUSY)
    for x in left:
        x.fill_(66)
    del left, x
    opt = _ops().AdamW([p], state_bits=bits)
    with torch.cuda.stream(side):
        opt.step([g])
        first = p.clone()
        torch.cuda._sleep(BUSY)
        opt.step([g])
    del opt
    held = [torch.full((n * bits // 8,), 66, dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(first, r) and torch.equal(p, q) and len(held) == 3


@gpu
@pytest.mark.parametrize("n", [5000, 40_000])
def test_captured_calls_run_beside_others_of_the_same_object(n):
    V = 3000
    first, second = _batch(n, V, 3), _batch(n - 100, V, 4)
    e = _ops().Embedding(V, 4, max_tokens=n)
    side, outs = torch.cuda.Stream(), []
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = e.gradient_rows(first[1], first[0])
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(side):
            graph.replay()
        outs += [e.gradient_rows(second[1], second[0]) for _ in range(3)]
    torch.cuda.synchronize()
    _same_rows(captured, *first)
    for got in outs:
        _same_rows(got, *second)
    with torch.cuda.stream(side):          # the stream that captured, now without a graph
        got = e.gradient_rows(second[1], second[0])
    graph.replay()
    torch.cuda.synchronize()
    _same_rows(got, *second)
    _same_rows(captured, *first)


# ---------------------------------------------------------------- the example's clipping
BAD = {"inf": float("inf"), "minus inf": -float("inf"), "nan": float("nan"), "a square that overflows": 1e30}


def test_the_clip_factor_is_finite_only_where_the_norm_is():
    from paper_2211_10280_b200.next_token import clip_factor

    grads = [torch.full((3,), 2.0), torch.full((4,), 1.0, dtype=torch.bfloat16)]      # norm 4
    assert clip_factor(grads, 5.0).item() == 1.0
    assert abs(clip_factor(grads, 1.0).item() - 0.25) < 1e-6
    assert clip_factor([torch.zeros(5)], 1.0).item() == 1.0
    for bad in BAD.values():
        assert not torch.isfinite(clip_factor(grads + [torch.tensor([1.0, bad])], 1.0))


@gpu
@pytest.mark.parametrize("bad", BAD.values(), ids=BAD.keys())
def test_a_step_whose_gradient_norm_is_not_finite_is_left_out(bad):
    from paper_2211_10280_b200.next_token import clip_factor

    V, d, n = 50, 8, 300
    ids, _ = _batch(n, V, 1)
    layer, table, m, v = (torch.randn(x, d, device="cuda") for x in (70, V, V, V))
    v.square_()
    grads = [torch.randn(70, d, device="cuda"), torch.randn(n, d, device="cuda")]
    grads[1][7, 3] = bad
    clip = clip_factor(grads, 1.0)
    for bits in (32, 8):
        opt = _ops().AdamW([layer], state_bits=bits)
        opt.step([torch.ones_like(layer)])
        kept = [x.clone() for x in (layer, table, m, v, *opt.m, *opt.v)]
        opt.step(grads[:1], grad_scale=clip)
        _ops().Embedding(V, d, max_tokens=n).adamw(grads[1], ids, table, m, v, step=2, grad_scale=clip)
        for x, y in zip(kept, (layer, table, m, v, *opt.m, *opt.v)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@gpu
def test_the_table_has_the_same_norm_in_both_forms_of_the_example(n=700):
    """A token that occurs several times counts with the sum of its gradient rows, whichever form the gradient has."""
    from paper_2211_10280_b200 import next_token

    V, d = 90, 6
    e = _ops().Embedding(V, d, max_tokens=n, scale=2.0)
    slot = next_token.rows_slot(V, d)
    for k in (n, 3):                   # the second batch leaves rows of the first in the slot
        ids, grad = _batch(k, V, k, d)
        rows = next_token.touched_rows(e, grad, ids, slot)
        assert rows.square().sum().item() == e.gradient(grad, ids).square().sum().item()
        assert k < n or rows.square().sum().item() != (2 * grad).square().sum().item()


# ---------------------------------------------------------------- captured steps
@gpu
def test_a_captured_step_is_the_same_step_at_every_replay():
    V, d, n = 40, 8, 200
    ids, _ = _batch(n, V, 1)
    p, g, rows = (torch.randn(x, d, device="cuda") for x in (500, 500, n))
    state = [torch.randn(V, d, device="cuda") for _ in range(2)] + [torch.rand(V, d, device="cuda")]      # table, m, v
    q, twin = p.clone(), [x.clone() for x in state]
    e, opt = _ops().Embedding(V, d, max_tokens=n), _ops().AdamW([p], step=3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step([g])
        e.adamw(rows, ids, *state, step=4)
    assert opt.step_count == 4
    opt.lr = 100.0                     # the graph holds the values that it was captured with
    plain = _ops().AdamW([q], step=3)
    for _ in range(3):
        graph.replay()
        plain.step_count = 3
        plain.step([g])
        e.adamw(rows, ids, *twin, step=4)
        torch.cuda.synchronize()
        assert torch.equal(p, q) and all(torch.equal(x, y) for x, y in zip(state, twin))


@gpu
def test_a_step_with_8_bit_moments_is_not_captured():
    p, g = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    opt = _ops().AdamW([p], state_bits=8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.add_(1)
        with pytest.raises(B.TensairError, match="captured"):
            opt.step([g])
    assert opt.step_count == 0
    graph.replay()
    opt.step([g])
    torch.cuda.synchronize()
    assert (p < 1).all() and (g == 2).all()


# ---------------------------------------------------------------- autograd
def test_a_step_between_forward_and_backward_is_an_error(recorder):
    p, q = (torch.nn.Parameter(torch.ones(10)) for _ in range(2))
    copies = [torch.ones(10, dtype=torch.bfloat16) for _ in range(2)]
    opt = _ops().AdamW([p, q], copies=copies)
    leaves = [c.detach().requires_grad_() for c in copies]
    for x in (p, leaves[0]):
        loss = (x * x).sum()
        opt.step([torch.ones(10), None])
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    for x in (q, leaves[1]):           # what a step leaves alone can still be gone back through
        loss = (x * x).sum()
        opt.step([torch.ones(10), None])
        loss.backward()
    loss = (q * q).sum()
    opt.step([torch.ones(10)] * 2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    (p * p).sum().backward()


@gpu
def test_calls_of_an_embedding_tell_autograd_what_they_wrote():
    V, d, n = 20, 4, 30
    ids, grad = _batch(n, V, 1)
    table, m, v = (torch.ones(V, d, device="cuda") for _ in range(3))
    e = _ops().Embedding(V, d, max_tokens=n)
    leaf = table.detach().requires_grad_()
    for call in (lambda: e.adamw(grad, ids, table, m, v, step=1), lambda: e.gradient(grad, ids, out=table),
                 lambda: e.gradient(grad, ids, out=table, accumulate=True), lambda: e.lookup(m, ids[:V], out=table),
                 lambda: e.lookup(m, ids[:V].view(4, 5), out=table.view(4, 5, d)),
                 lambda: e.gradient_rows(grad, ids, out=(torch.empty(n, dtype=torch.int32, device="cuda"), table, torch.empty(1, dtype=torch.int32, device="cuda")))):
        loss = (leaf * leaf).sum()
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    loss = e(leaf, ids).sum()          # needs the ids alone
    e.adamw(grad, ids, table, m, v, step=2)
    loss.backward()
    with torch.inference_mode():       # tensors without a version
        t = torch.ones(V, d, device="cuda")
        e.adamw(grad, ids, t, t.clone(), t.clone(), step=1)
        _ops().AdamW([t]).step([torch.ones_like(t)])
    torch.cuda.synchronize()


# ---------------------------------------------------------------- parameters without a gradient
def test_parameters_without_a_gradient_keep_their_place(recorder):
    sizes = [300, 1, 7, 513]
    ps = [torch.ones(n) for n in sizes]
    opt = _ops().AdamW(ps)
    for left in ((), (1,), (0, 3), (), (2,)):
        opt.step([None if i in left else torch.ones(n) for i, n in enumerate(sizes)])
        assert recorder.skipped == [int(i in left) for i in range(4)] and [t[7] for t in recorder.asked[-1]] == sizes


def test_a_skipped_tensor_is_not_looked_at():
    t = (B.AdamwTensor * 2)(B.AdamwTensor(n=10, skip=1, lr_factor=float("nan"), param_type=9), B.AdamwTensor(n=0))
    h = B.Adamw(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    assert B.lib().tensair_adamw_step(t, 2, 8, h, None) == B.OK          # nothing to do
    t[0].n = 2 ** 40
    assert B.lib().tensair_adamw_step(t, 2, 8, h, None) == B.EINVAL


@gpu
def test_rounding_of_8_bit_moments_does_not_depend_on_the_gradients_that_others_have():
    sizes = [1000, 300, 0, 5000]
    gs = [torch.linspace(0.1, 1.7, n, device="cuda") for n in sizes]
    kept = []
    for use in (gs, [gs[0], None, gs[2], gs[3]], [None, None, None, gs[3]]):
        opt = _ops().AdamW([torch.ones(n, device="cuda") for n in sizes], state_bits=8, seed=5)
        opt.step(use)
        opt.step(use)
        assert use[1] is not None or not opt.m[1].float().any()
        kept.append((opt.m[3].view(torch.uint8), opt.v[3].view(torch.uint8), opt.params[3]))
    for other in kept[1:]:
        assert all(torch.equal(x, y) for x, y in zip(kept[0], other))


# ---------------------------------------------------------------- what 8-bit moments are made of, bit for bit
@gpu
def test_roots_of_second_moments_over_the_whole_range_of_exponents():
    """Blocks of one value each, from below 2^-96, where the kernel takes another way to its roots, to 2^127: a block's scale is its
    root, as torch.sqrt rounds it, over 448.  With beta2 = 0.3 the second moments are no squares."""
    gen = torch.Generator("cuda").manual_seed(0)
    size = torch.ldexp(torch.rand(60_000, device="cuda", generator=gen) + 1, torch.randint(-52, 63, (60_000,), device="cuda", generator=gen))
    ends = torch.ldexp(torch.linspace(0.99, 1.5, 2000, device="cuda"), torch.tensor(-48, device="cuda"))      # around 2^-96
    size = torch.cat([size, ends, torch.ldexp(torch.ones(114, device="cuda"), torch.arange(-51, 63, device="cuda"))])
    size = size * torch.where(torch.arange(size.numel(), device="cuda") % 2 > 0, -1.0, 1.0)
    opt = _ops().AdamW([torch.zeros(256 * size.numel(), device="cuda")], lr=0.0, betas=(0.9, 0.3), state_bits=8)
    opt.step([size.repeat_interleave(256)])
    v = (size * size) * torch.tensor(1 - 0.3, device="cuda")
    over = torch.tensor(1 / 448, device="cuda")
    assert (v < 2.0 ** -96).any() and (v > 2.0 ** 124).any() and torch.isfinite(v).all()
    assert torch.equal(opt.v_scale[0], v.sqrt() * over)
    assert torch.equal(opt.m_scale[0], (size * torch.tensor(1 - 0.9, device="cuda")).abs() * over)


def _bits16(groups, step, seed):
    """16 random bits for every element, from Philox4x32-10 over (group of 8 elements, step) with the seed as its key."""
    low = 0xFFFFFFFF
    at = torch.arange(groups, device="cuda")
    c, key = [at, torch.zeros_like(at), torch.full_like(at, step), torch.full_like(at, 5 << 24)], [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & low) ^ c[1] ^ key[0], b & low, ((a >> 32) & low) ^ c[3] ^ key[1], a & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    words = torch.stack(c, 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).view(-1).to(torch.int32)


@gpu
@pytest.mark.parametrize("spread", [0.0, 3.0, 12.0])
def test_every_code_of_8_bit_moments_is_that_of_separately_rounded_operations(spread):
    """Every element of both moments, from gradients of one size or of sizes over many orders of magnitude (codes in the format's
    subnormal range), step after step from what the step before stored."""
    n, seed = 256 * 500, (3 << 32) + 11
    gen = torch.Generator("cuda").manual_seed(1)
    opt = _ops().AdamW([torch.zeros(n, device="cuda")], state_bits=8, seed=seed)
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    c = [torch.tensor(x, device="cuda") for x in (0.9, 1 - 0.9, 0.999, 1 - 0.999)]
    for step in range(1, 5):
        g = torch.randn(n, device="cuda", generator=gen) * torch.exp(torch.randn(n, device="cuda", generator=gen) * spread) * 1e-3
        opt.step([g])
        m = m * c[0] + g * c[1]
        v = (v * v) * c[2] + (g * g) * c[3]                   # v: the stored root
        bits = _bits16(n // 8, step, seed)
        for x, code, scale in ((m, opt.m[0], opt.m_scale[0]), (v.sqrt(), opt.v[0], opt.v_scale[0])):
            finite = torch.isfinite(x)                        # a square that overflows is kept as NaN, and not in the block's scale
            top = torch.where(finite, x.abs(), 0.0).view(-1, 256).amax(1)
            assert torch.equal(scale, top * torch.tensor(1 / 448, device="cuda"))
            y = (x.abs().view(-1, 256) * ((1 / top) * 448)[:, None]).view(-1)
            if code is opt.v[0]:
                y = torch.where((x > 0) & (y < 2.0 ** -9), 2.0 ** -9, y)
            cut = ((y.view(torch.int32) + (bits << 4) + 8) & -0x100000).view(torch.float32).clamp(max=448.0)
            want = torch.copysign(torch.where(y < 2.0 ** -6, y, cut), x).to(torch.float8_e4m3fn)
            assert torch.equal(code.view(torch.uint8)[finite], want.view(torch.uint8)[finite]), step
            assert torch.isnan(code[~finite].float()).all() and finite.float().mean() > 0.99
        m = (opt.m[0].float().view(-1, 256) * opt.m_scale[0][:, None]).view(-1)
        v = (opt.v[0].float().view(-1, 256) * opt.v_scale[0][:, None]).view(-1)


# ---------------------------------------------------------------- ids
@gpu
def test_without_a_padding_id_every_id_outside_the_vocabulary_is_reported():
    V, d, low = 10, 4, -(1 << 63)
    table, grad = torch.ones(V, d, device="cuda"), torch.ones(3, d, device="cuda")
    for padding, bad in ((None, (low, -1, V)), (low, (low,)), (low + 1, (low, -1)), (-1, (low, V)), (3, (-1, low))):
        e = _ops().Embedding(V, d, max_tokens=3, padding_id=padding)
        for x in bad:
            ids = torch.tensor([1, x, 2], device="cuda")
            for call in (lambda: e.lookup(table, ids), lambda: e.gradient(grad, ids)):
                out = call()
                with pytest.raises(B.TensairError):
                    e.check()
                assert out.sum().item() == 2 * d
        if padding not in (None, low):
            ids = torch.tensor([1, padding, 2], device="cuda")
            assert e.lookup(table, ids).sum().item() == e.gradient(grad, ids).sum().item() == 2 * d
            e.check()


# ---------------------------------------------------------------- the checked build
@gpu
@pytest.mark.parametrize("n", [1, 200, 256, 257, 1024, 1025, 9000, 16_384, 16_385, 100_000, 131_073, 300_000])
def test_no_index_of_a_call_leaves_its_array(n):
    """With the checked build (TENSAIR_CHECKED=1) every index that is computed from data is compared with its bound; the error word
    stays clean over all lengths and forms, over vocabularies below and above the batch."""
    d = 5
    for V in (1, 300, 700_000):
        ids, grad = _batch(n, V, n, d)
        e = _ops().Embedding(V, d, max_tokens=n, padding_id=2)
        held = ids != 2
        _same_rows(e.gradient_rows(grad, ids), ids[held], grad[held])
        want = torch.zeros(V, d, device="cuda").index_add_(0, ids[held], grad[held])
        table = e.gradient(grad, ids)
        assert torch.equal(table, want)
        assert torch.equal(e.gradient(grad, ids, out=table, accumulate=True), 2 * want)
        e.adamw(grad, ids, table, torch.zeros_like(want), torch.zeros_like(want), step=1)
        e.lookup(table, ids)
        e.check()
