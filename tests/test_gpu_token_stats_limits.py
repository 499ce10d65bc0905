"""Token statistics at the values, orders and sizes where the kernels change their way: tolerances as
tests/test_gpu_token_stats.py derives them."""
import numpy as np
import pytest
import torch

from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.test_gpu_token_stats import DTYPES, check_stats, make, rows_of, run_stats
from tests.helpers import host_f64

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    B.build()
    H.load()
    H.device_error(clear=True)
    yield
    assert H.device_error(clear=True) == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k", [0, 6])
def test_rows_that_fill_a_stage_of_the_ring_in_part_and_whole(k, dtype):
    """A row's first and last 16 bytes are written to the ring by a thread where they are the row's in part, and by bulk
    copies in the next round of the ring: every call has the same bits, and they are right."""
    rows, V = 1400, 12301
    rng = np.random.default_rng(7)
    z, _ = rows_of(rng.normal(0, 3, (rows, V)), DTYPES[dtype], V + 2, 1)
    ids, values = rng.integers(0, V, rows), host_f64(z)
    first = run_stats(z, ids, None, rows, 1, k)
    check_stats(first, values, ids, None, rows, 1, k)
    for _ in range(20):
        again = run_stats(z, ids, None, rows, 1, k)
        assert all(torch.equal(first[name], again[name]) for name in first)


@pytest.mark.parametrize("k", [0, 5])
@pytest.mark.parametrize("rows", [1, 30, 70])
def test_clusters_whose_row_holds_no_token_end_at_once(rows, k):
    """The first CTA of a cluster waits for what the others send, which they do for a row that holds a token only: no
    wait may run out (the device error would say so), call after call."""
    V = 32000
    z, _ = rows_of(np.random.default_rng(rows).normal(0, 3, (rows, V)), torch.float32)
    ids, values = np.arange(rows), host_f64(z)
    for live in (np.zeros(rows, np.int64), np.ones(rows, np.int64), np.arange(rows) % 2):
        for _ in range(3):
            check_stats(run_stats(z, ids, live, rows, 1, k), values, ids, live, rows, 1, k)
            assert H.device_error() == 0


@pytest.mark.parametrize("rows,V", [(1300, 6000), (40, 20000), (400, 20000)])
@pytest.mark.parametrize("base", [2.0 ** 20, -(2.0 ** 20)])
def test_maximum_that_passes_2_to_the_20(rows, V, base):
    """A thread's terms are summed in another way from there on: nearly all of the row just below, later a
    little of it just above, more than the reference may trail. All values are multiples of 1/4, exact in fp32; what is
    below has 1 % to 10 % of the sum."""
    rng = np.random.default_rng(V + rows)
    z = base - rng.integers(28, 40, (rows, V)) / 4.0
    late = np.arange(V) >= V // 2
    z[:, late] = np.where(rng.random((rows, int(late.sum()))) < 0.01, base + rng.integers(0, 8, (rows, int(late.sum()))) / 4.0,
                          z[:, late])
    dev, _ = rows_of(z, torch.float32)
    values, ids = host_f64(dev), rng.integers(0, V, rows)
    assert np.array_equal(values, z)
    check_stats(run_stats(dev, ids, None, rows, 1, 0), values, ids, None, rows, 1, 0)
    if V == 20000:
        check_stats(run_stats(dev, ids, None, rows, 1, 5), values, ids, None, rows, 1, 5)


def slow_order(rows, V, dtype):
    """Rows whose 31 times 4 of 256 threads hold values that ascend in about the order in which a selection collects them:
    every bound of it is passed by the most values that there can be."""
    per = 4 if dtype is torch.float32 else 8
    slots = np.arange(V // per)
    stages = ((len(slots) + 1023) // 1024 + 7) // 8
    segment, summer, i = slots // (stages * 1024), slots % 256, slots % (stages * 1024) // 256
    high = (summer % 32 < 31) & (summer < 128)
    key = np.lexsort((i % 32, segment, summer // 32, summer % 32, i // 32))
    key = key[high[key]]
    z = np.zeros((len(slots), per))
    value = np.arange(len(key) * per, dtype=np.float64).reshape(-1, per)
    z[key] = 1 + value * (2.0 ** -20 if dtype is torch.float32 else 300.0 / value.size)
    dev, _ = rows_of(np.broadcast_to(z.reshape(1, V), (rows, V)).copy(), dtype)
    return dev


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V", [(1, 131072), (160, 131072), (1, 1 << 20), (160, 1 << 20)])
def test_selection_in_the_slowest_order_is_right(rows, V, dtype):
    k, z = 32, slow_order(rows, V, DTYPES[dtype])
    ids = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    H.hydra_token_logprobs_entropy(z, None, None, rows, 1, top_ids=ids, top_logp=torch.zeros(rows, k, device="cuda"))
    want = np.argsort(-host_f64(z[:1]), axis=1, kind="stable")[:, :k]
    assert np.array_equal(ids.cpu().numpy(), np.broadcast_to(want, (rows, k)))


@pytest.mark.parametrize("least", [0.0, -1e30])
@pytest.mark.parametrize("k", [1, 31, 32])
def test_selection_by_counting_with_ties_nan_and_infinities(k, least):
    """The slowest order with what a count of digits could get wrong at its top: equal values beyond k, zeros of
    both signs, negative values, +inf and NaN."""
    V = 131072
    base = host_f64(slow_order(1, V, torch.float32))[0]
    rng = np.random.default_rng(k)
    rows = []
    for n in range(8):
        z = base.copy()
        where = rng.choice(np.flatnonzero(base > 0), 40, replace=False)
        if n == 1:
            z[where] = base.max() + 1
        elif n == 2:
            z[where[:20]] = INF
        elif n == 3:
            z[where[:20]], z[where[20:]] = np.nan, INF
        elif n == 4:
            z = np.where(base > 0, base - base.max() - 1, -100.0)   # all negative
        elif n == 5:
            z = np.where(base > 0, base - base.max(), -100.0)       # up to a zero
            z[where] = np.where(np.arange(40) % 2 == 0, 0.0, -0.0)
        elif n == 6:
            z = np.where(base > 0, base * 1e-41, 0.0)               # subnormal
        elif n == 7:
            z = np.where(base > 0, base * 1e30, -1e38)
        rows.append(np.where(base > 0, z, np.minimum(z, least)))
    rows = np.stack(rows * 20)
    dev, _ = rows_of(rows, torch.float32)
    ids = torch.full((160, k), -7, dtype=torch.int32, device="cuda")
    H.hydra_token_logprobs_entropy(dev, None, None, 160, 1, top_ids=ids, top_logp=torch.zeros(160, k, device="cuda"))
    values = host_f64(dev[:8])
    order = np.lexsort((np.broadcast_to(np.arange(V), values.shape), -np.where(np.isnan(values), 0, values),
                        ~np.isnan(values)), axis=1)[:, :k]
    assert np.array_equal(ids.cpu().numpy(), np.tile(order, (20, 1)))


def test_selection_takes_a_time_that_grows_with_the_vocabulary():
    """Four times the logits in the slowest order: about four times the time, sixteen where it grows with the square.
    Eight lies between."""
    took = []
    for V in (1 << 17, 1 << 19):
        z = slow_order(160, V, torch.float32)
        ids, logp = torch.zeros(160, 32, dtype=torch.int32, device="cuda"), torch.zeros(160, 32, device="cuda")
        best = float("inf")
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            H.hydra_token_logprobs_entropy(z, None, None, 160, 1, top_ids=ids, top_logp=logp)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        took.append(best)
    assert took[1] < 8 * took[0], took


@pytest.mark.parametrize("dtype,V", [("f32", 6200), ("bf16", 8200)])
@pytest.mark.parametrize("S,L", [(1, 700), (127, 8), (128, 7), (129, 7), (700, 2)])
def test_ragged_batches_without_alternatives_that_go_through_the_ring(S, L, dtype, V):
    """Rows too long for a warp each, more of them than CTAs: up to 128 sequences have their live rows dealt by number, more
    of them by row. Full and empty sequences and those of one token, and a batch of none."""
    z, values, ids, lengths, _ = make(S + L, S, L, V, DTYPES[dtype], ld=V + 3, shift=1)
    lengths[1::4], lengths[2::7] = 0, 1
    check_stats(run_stats(z, ids, lengths, S, L, 0), values, ids, lengths, S, L, 0)
    lengths[:] = 0
    check_stats(run_stats(z, ids, lengths, S, L, 0), values, ids, lengths, S, L, 0)
