"""Launches of the paged cache's operators and of verification, without a GPU: the library linked to the fake CUDA runtime
of tests/test_dispatch_cpu.py, which dereferences no device pointer."""
import ctypes
import shutil

import pytest

from paper_2309_00754_gb300 import hydra as H
from tests.test_dispatch_cpu import BIG, P, Fake, built  # noqa: F401 (a fixture)


@pytest.fixture()
def fake(built, tmp_path):  # noqa: F811
    f = Fake(shutil.copy(built, str(tmp_path / "lib.so")))
    f.device()
    return f


def cache(int4=True, kv=8, dh=128, page=16, pages=1 << 20):
    return ctypes.byref(H.KvCacheC(P, pages, page, kv, dh, int(int4)))


def append(fake, S, L, heads=32, kv=8, dh=128, int4=True):
    q = (P, heads, heads * dh) if heads else (None, 0, 0)
    assert fake.lib.hydra_kv_append(cache(int4, kv, dh), P, 64, 64, P, P, S, L, *q, P, P, kv * dh, P, 1024,
                                    P if heads else None, heads * dh, None) == 0
    return fake.launches()


def attend(fake, S, L, heads=32, kv=8, dh=128, int4=True, pages=64, page=16):
    assert fake.lib.hydra_paged_attention(cache(int4, kv, dh, page), P, pages, pages, P, P, S, L, P, heads, heads * dh, 0.1, P,
                                          heads * dh, P, BIG, None) == 0
    return fake.launches()


def verify(fake, S, D, V, bf16=False, greedy=False, draft=True):
    draft = P if draft and not greedy else None
    noise = (None, None) if greedy else (P, P)
    assert fake.lib.hydra_verify_drafts(P, draft, 0 if bf16 else 1, S, D, V, V, V, P, P, *noise, V, P, P, P, P, None) == 0
    ((name, x, y, z, cluster, _),) = fake.launches()
    assert "verify_kernel" in name and (y, z) == (1, 1)
    return x, cluster


def test_an_append_is_one_launch_of_a_kernel_by_head_size_and_kind(fake):
    names = {append(fake, 2, 3, dh=dh, int4=int4)[0][0] for dh in (64, 128) for int4 in (False, True)}
    assert len(names) == 4 and all("kv_append_kernel" in n for n in names)
    assert names == {n for n in fake.lib.fake_kernels().decode().split() if "kv_append_kernel" in n}


def test_appended_tokens_go_by_blocks_of_eight_positions(fake):
    """A block more than the tokens fill, as a sequence may begin anywhere in one; four warps a CTA."""
    def grid(*a, **k):
        ((_, x, y, _, _, _),) = append(fake, *a, **k)
        return x, y
    for L, blocks in ((1, 1), (2, 2), (9, 2), (10, 3), (512, 65)):
        assert grid(3, L, heads=0, kv=2)[0] == 3 * blocks
    assert grid(3, 2) == (6, 12)                    # 32 + 2 x 8 heads, a warp each
    assert grid(3, 1) == (3, 2)                     # single tokens: eight heads a warp, four of values: 4 + 1 + 2 warps
    assert grid(3, 1, heads=0, kv=1) == (3, 1)
    assert grid(64, 64, kv=32) == (64 * 9, 6)       # many: four heads a warp
    assert grid(2, 512, kv=32)[1] == 6 and grid(4, 128, kv=32)[1] == 24
    assert grid((1 << 31) - 1, 1, heads=4096, kv=4096)[1] == (4096 // 8 * 2 + 4096 // 4) // 4  # within a grid's limits


def test_reading_back(fake):
    def grid(S, L, kv):
        assert fake.lib.hydra_kv_read(cache(kv=kv), P, 64, 64, P, P, S, L, P, P, 1, kv * 128, None) == 0
        ((name, x, y, *_),) = fake.launches()
        assert "kv_read_kernel" in name
        return x, y
    assert grid(3, 9, 5) == (6, 3) and grid(1, 1, 4096) == (1, 2048) and grid((1 << 31) - 1, 1, 1) == ((1 << 31) - 1, 1)


def test_attention_of_short_tables_is_one_launch_else_two(fake):
    for int4, ctas in ((True, 304), (False, 152)):
        for S, L, pages, one in ((4, 1, 80, True), (4, 1, 81, False), (ctas // 8, 1, 80, True), (ctas // 8 + 1, 1, 80, False),
                                 (1, 2 * ctas // 8, 80, True), (1, 2 * ctas // 8 + 1, 80, False)):
            launches = attend(fake, S, L, int4=int4, pages=pages if pages == 80 or int4 else 2 * pages)
            items = S * 8 * -(-4 * L // 8)
            if one:
                ((name, x, *_),) = launches
                assert x == items and "paged_attention_kernel" in name, (S, L, pages)
            else:
                (_, x, *_), (name, jx, jy, *_) = launches
                assert x == jx == ctas and jy == min(8, 4 * L) and "join" in name, (S, L, pages)
    # twice the tokens for light tiles where a quarter of the CTAs have an item
    for dh, int4, S, pages, one in ((64, True, 9, 160, False), (64, True, 10, 160, True), (64, True, 10, 161, False), (64, False, 10, 160, True),
                                    (128, True, 20, 160, False), (128, False, 4, 160, False), (128, False, 5, 160, True)):
        assert len(attend(fake, S, 1, dh=dh, int4=int4, pages=pages)) == (1 if one else 2), (dh, int4, S, pages)
    # the workspace holds the parts of any device's grid
    fake.device(device=1, sms=1000)
    assert attend(fake, 900, 1)[0][1] == 320


def test_sequences_are_verified_by_clusters_that_fit(fake):
    """The fake device holds 76 clusters of two and 36 of four and eight at once."""
    for bf16 in (False, True):
        for greedy in (False, True):
            for S, cs in ((1, 8), (36, 8), (37, 2), (76, 2), (77, 1), (1 << 24, 1)):
                assert verify(fake, S, 4, 32000, bf16, greedy) == (S * cs, cs)
    for V, cs in ((1, 1), (1999, 1), (2000, 2), (4000, 4), (7999, 4), (8000, 8)):
        assert verify(fake, 1, 32, V, draft=False) == (cs, cs)


def test_a_device_without_clusters_verifies_all_the_same(fake):
    fake.device(device=1, pairs=0, quads=0)
    assert verify(fake, 1, 4, 32000) == (1, 1)
    fake.device(device=2, error=1)
    assert verify(fake, 1, 4, 32000) == (1, 1)
    fake.device(device=2)  # a failed query is not kept
    assert verify(fake, 1, 4, 32000) == (8, 8)
