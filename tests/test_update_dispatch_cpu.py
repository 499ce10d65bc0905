"""Launches of the token statistics, their gradient and gradient clipping, without a GPU: the library linked to
the fake CUDA runtime of tests/test_dispatch_cpu.py, which dereferences no device pointer."""
import shutil

import numpy as np
import pytest

from paper_2309_00754_gb300 import hydra as H
from tests.test_dispatch_cpu import BIG, P, Fake, built  # noqa: F401 (a fixture)


@pytest.fixture()
def fake(built, tmp_path):  # noqa: F811
    f = Fake(shutil.copy(built, str(tmp_path / "lib.so")))
    f.device()
    return f


def stats(fake, rows, v, k, bf16=False, lengths=None, seqs=None):
    s = seqs or rows
    assert fake.lib.hydra_token_logprobs_entropy(P, 0 if bf16 else 1, s, rows // s, v, v, P, lengths, k, P, P, P, P, P, None) == 0
    (launch,) = fake.launches()
    return launch


def test_statistics_are_one_launch_of_a_kernel_by_type_and_selection(fake):
    names = [{stats(fake, rows, 32000, k, bf16)[0] for k in (0, 1, 32) for bf16 in (False, True)} for rows in (1, 1000)]
    compiled = {n for n in fake.lib.fake_kernels().decode().split() if "token_stats_kernel" in n}
    assert [len(n) for n in names] == [4, 4] and names[0] | names[1] == compiled  # of clusters, and of single CTAs
    assert not names[0] & names[1]


def test_few_long_rows_are_shared_by_clusters_that_fit(fake):
    """The fake device holds 76 clusters of two and 36 of four and eight at once."""
    for v, bf16 in ((32000, False), (128001, True)):
        for rows, cs in ((1, 8), (36, 8), (37, 2), (76, 2), (77, 1), (1000, 1)):
            name, x, y, z, cluster, _ = stats(fake, rows, v, 0, bf16)
            assert (cluster, x) == (cs, rows * cs if cs > 1 else min(rows, 4 * 152)), (v, rows)
    # selection: two, four and eight share rows of 120, 48 and 96 KB, and fewer CTAs are resident
    for rows, v, cs in ((20, 32000, 8), (20, 20000, 4), (40, 20000, 1), (40, 32000, 2), (40, 128001, 2), (400, 32000, 1)):
        name, x, *_, cluster, _ = stats(fake, rows, v, 5)
        assert (cluster, x) == (cs, rows * cs if cs > 1 else min(rows, 2 * 152))
    assert stats(fake, 1, 7900, 0)[4] == 1  # short rows are not shared
    assert stats(fake, 1, 8000, 0)[4] == 8 and stats(fake, 40, 8000, 0)[4] == 1


def test_short_rows_take_a_warp_each(fake):
    for rows, v, bf16, short in ((1, 1, False, True), (3, 1024, False, True), (3, 1025, False, False), (8, 2048, True, True),
                                 (1216, 6144, False, False), (1217, 6144, False, True), (1217, 6145, False, False),
                                 (20000, 8192, True, True), (20000, 8193, True, False)):
        name, x, *_ = stats(fake, rows, v, 0, bf16)
        assert ("token_stats_short_kernel" in name) == short, (rows, v, bf16)
        assert x == ((rows + 7) // 8 if short else min(rows, 608))
    assert "short" not in stats(fake, 3, 500, 1)[0]  # with alternatives


def test_a_device_without_clusters_takes_rows_one_by_one(fake):
    fake.device(device=1, pairs=0, quads=0)
    assert stats(fake, 1, 128001, 0)[4] == 1 and stats(fake, 1, 128001, 8)[4] == 1
    fake.device(device=2, error=1)
    assert stats(fake, 1, 128001, 0)[4] == 1
    fake.device(device=2)  # a failed query is not kept
    assert stats(fake, 1, 128001, 0)[4] == 8


def test_gradient_puts_few_tiles_on_many_multiprocessors(fake):
    def grad(rows, v, bf16=False):
        assert fake.lib.hydra_token_logprobs_entropy_grad(P, 1, rows, 1, v, v, P, None, P, P, P, P, 2 * P, 0 if bf16 else 1, v,
                                                          None) == 0
        (launch,) = fake.launches()
        return launch[1]
    assert grad(1, 32000) == 16            # 16 tiles of 2048, a warp and a CTA each
    assert grad(152, 2041) == 152          # one tile a row: 2048 with seven elements before the row
    assert grad(153, 2041) == 77           # two warps a CTA
    assert grad(4096, 32000) == 4096 * 16 // 8
    assert grad((1 << 31) - 1, 1) == 1 << 28


def clip(fake, sizes, fn="hydra_clip_grad_norm", dtype=1):
    at, list_ = 1 << 30, []
    for n in sizes:
        list_.append(H.GradTensorC(at, at, n, dtype))
        at += (4 * n + 511) // 512 * 512
    c = (H.GradTensorC * max(1, len(list_)))(*list_)
    assert getattr(fake.lib, fn)(c, len(list_), 1.0, P, P, BIG, None) == 0
    kind = lambda name: next(k for k in ("square", "scale", "norm") if f"grad_{k}_kernel" in name)  # noqa: E731
    return [(kind(name), x) for name, x, *_ in fake.launches()]


def test_clipping_is_two_launches_and_more_for_long_lists(fake):
    assert clip(fake, [100]) == [("square", 1), ("scale", 1)]
    assert clip(fake, [100], "hydra_grad_norm") == [("square", 1), ("norm", 1)]
    assert clip(fake, []) == [("norm", 1)] and clip(fake, [0, 0]) == [("norm", 1)]
    assert clip(fake, [4096] * 5 + [4097]) == [("square", 7), ("scale", 7)]  # chunks of 16 KB
    assert clip(fake, [1 << 28]) == [("square", 608), ("scale", 608)]        # as many CTAs as are resident
    assert clip(fake, [8] * 880) == [("square", 608), ("scale", 608)]
    # the first launch of several covers the partial sums of every other
    assert clip(fake, [8] * 881) == [("square", 608), ("square", 608), ("scale", 608), ("scale", 1)]
    assert clip(fake, [8] * 1761 + [0]) == [("square", 608)] * 3 + [("scale", 608), ("scale", 608), ("scale", 1)]


def test_every_compiled_table_is_taken_by_some_list(fake):
    taken = set()
    for n in (1, 32, 33, 224, 225, 880):
        at = 1 << 30
        c = (H.GradTensorC * n)(*[H.GradTensorC(at + 512 * i, at + 512 * i, 8, 1) for i in range(n)])
        assert fake.lib.hydra_clip_grad_norm(c, n, 1.0, P, P, BIG, None) == 0
        taken |= {v[0] for v in fake.launches()}
        assert fake.lib.hydra_grad_norm(c, n, 1.0, P, P, BIG, None) == 0
        taken |= {v[0] for v in fake.launches()}
    for n in (1, 225):  # large lists
        c = (H.GradTensorC * n)(*[H.GradTensorC((i + 1) << 40, (i + 1) << 40, 1 << 27, 0) for i in range(n)])
        assert fake.lib.hydra_clip_grad_norm(c, n, 1.0, P, P, BIG, None) == 0
        taken |= {v[0] for v in fake.launches()}
    assert taken == {n for n in fake.lib.fake_kernels().decode().split() if "grad_square" in n or "grad_scale" in n or
                     "grad_norm" in n}


def test_overlaps_are_found_in_lists_of_any_order(fake):
    """Against every pair of ranges: an output may overlap nothing but the gradient it replaces."""
    rng, seen = np.random.default_rng(5), set()
    for _ in range(400):
        n = int(rng.integers(1, 7))
        src, dst, numel = rng.integers(1, 60, n) * 16, rng.integers(1, 60, n) * 16, rng.integers(0, 13, n)
        inside = rng.random(n) < 0.5
        dst[inside] = src[inside]
        rows = [(int(a), int(b), int(m)) for a, b, m in zip(src, dst, numel) if m > 0]
        meet = lambda a, b, m, o: a < b + 4 * o and b < a + 4 * m  # noqa: E731
        clash = any(meet(b, a2, m, m2) and not (i == j and b == a2) or (i != j and meet(b, b2, m, m2))
                    for i, (a, b, m) in enumerate(rows) for j, (a2, b2, m2) in enumerate(rows))
        c = (H.GradTensorC * n)(*[H.GradTensorC(int(a), int(b), int(m), 1) for a, b, m in zip(src, dst, numel)])
        assert fake.lib.hydra_clip_grad_norm(c, n, 1.0, P, P, BIG, None) == (4 if clash else 0), rows
        fake.launches()
        seen.add(clash)
    assert seen == {True, False}
