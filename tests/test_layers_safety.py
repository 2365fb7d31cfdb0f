"""Calls of the recurrent model's operators that their documentation allows and that go wrong easily: results written over their inputs.
"""
import ctypes as C

import pytest
import torch

from paper_2211_10280_b200 import binding as B
from paper_2211_10280_b200 import build as libbuild

gpu = pytest.mark.gpu
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
