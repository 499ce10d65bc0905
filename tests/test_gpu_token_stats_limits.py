"""Token statistics at the values, orders and sizes where the kernels change their way: tolerances as
tests/test_gpu_token_stats.py derives them."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.test_gpu_token_stats import DTYPES, check_stats, rows_of, run_stats
from tests.helpers import host_f64

pytestmark = pytest.mark.gpu


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
