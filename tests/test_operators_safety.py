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
