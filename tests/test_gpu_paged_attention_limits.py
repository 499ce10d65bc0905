"""Attention over a paged cache at its limits: groups of channels of very different size, bad pages that only some rows of
an item read. Tolerances as tests/test_gpu_paged_attention.py derives them, with u = 2^-24 and e for a score's error, but for what
fp16's least step adds: a weight is off by 2^-25 at most where the largest product of probability and scale that the row has
met in that group of 64 channels is 2^6 or more. Relative to the row's largest product over all tokens it is off by 2^-31, times a
code of up to 15, and a scale is at most max |v| / 7.5 of its token and group, so over N tokens
    (2^-11 + 2 e + (N + 128) u) sum_j p_j |v_j| + N 2^-30 max_j (p_j max_group |v_j|),
and rounded to bf16. (In a bf16 cache less.)"""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.test_gpu_paged_attention import U, attend, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    B.build()
    H.load()
    H.device_error(clear=True)
    yield
    assert H.device_error(clear=True) == 0


def check_groups(c, got, rows=None):
    """Every channel against its own group's tolerance; `rows`: of the first so many new tokens of each sequence."""
    S, L, D, heads, kv = c["S"], c["L"], c["D"], c["heads"], c["kv"]
    got = got.double().cpu().numpy().reshape(S, L, heads, D)
    q = c["q"].double().numpy().reshape(S, L, heads, D)
    scale, by = D ** -0.5, heads // kv
    for s in range(S):
        n, at = int(c["lengths"][s] if rows is None else rows[s]), int(c["cached"][s])
        if n == 0:
            continue
        N = at + n
        k, v = (c[x][s, :N].astype(np.float64) for x in ("k", "v"))
        ref, size, reach = O.cached_attention(q[s, :n], k, v, at, scale)
        coarse = np.abs(q[s, :n]).max(-1) * np.abs(k).sum(-1).max(0).repeat(by)[None] * scale
        e = ((2 * (D + D // 16) + 16) * U * reach + 2.0 ** -28 * coarse)[..., None]
        largest = np.abs(v).reshape(N, kv, D // 64, 64).max(-1)  # of a token, head and group
        most = np.zeros((n, heads, D // 64))
        for t in range(n):
            for h in range(heads):
                z = k[:at + t + 1, h // by] @ q[s, t, h] * scale
                p = np.exp(z - z.max())
                most[t, h] = (p[:, None] / p.sum() * largest[:at + t + 1, h // by]).max(0)
        tol = (2.0 ** -11 + 2 * e + (N + 128) * U) * size + N * 2.0 ** -30 * most.repeat(64, -1)
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
        off = np.abs(got[s, :n] - ref)
        assert np.isfinite(got[s, :n]).all() and (off <= tol).all(), f"sequence {s}: {np.max(off / np.maximum(tol, 1e-300)):.3g}"


@pytest.mark.parametrize("cached", [[500, 37, 0], [5000, 900]])
@pytest.mark.parametrize("quiet", [0, 1])
@pytest.mark.parametrize("ratio", [1e-6, 1e-7, 1e-9, 1e-25, 0.0])
@pytest.mark.parametrize("int4", [True, False])
def test_groups_of_channels_of_different_size(int4, ratio, quiet, cached):
    def change(k, v):
        v[..., 64 * quiet:64 * quiet + 64] *= ratio
        v[:, :, 1:, 64 * quiet:64 * quiet + 64] *= 1e-3  # and from head to head

    c = make(60, 3, 8, 2, 128, 16, int4, cached, change=change)
    check_groups(c, attend(c))


@pytest.mark.parametrize("int4", [True, False])
@pytest.mark.parametrize("rising", [True, False])
def test_groups_that_grow_and_shrink_along_a_sequence(rising, int4):
    """One group's values shrink by 10^15 along the sequence, the other's grow, while scores rise to the end (or fall)."""
    def change(k, v):
        n = np.arange(v.shape[1])
        v[..., 64:] *= (10.0 ** (-n / 40))[:, None, None]
        v[..., :64] *= (10.0 ** (n / 60 - 10))[:, None, None]
        k *= (n / 100 if rising else (n.max() - n) / 100)[:, None, None]

    c = make(61, 2, 4, 2, 128, 32, int4, [600, 300], change=change)
    check_groups(c, attend(c))


@pytest.mark.parametrize("D", [64, 128])
def test_values_near_the_ends_of_bf16(D):
    """Values of up to 3e38 and down to 1e-33, alone and beside each other."""
    def change(k, v):
        v[0] *= 1e37 / np.abs(v[0]).max()
        v[1] *= 1e-33
        v[2] *= np.where(np.arange(v.shape[1]) % 2 == 0, 1e30, 1e-30)[:, None, None]

    c = make(62, 2, 4, 2, D, 16, True, [200] * 3, change=change)
    check_groups(c, attend(c))


@pytest.mark.parametrize("int4", [True, False])
@pytest.mark.parametrize("page,cached,L,bad", [(16, [12, 11, 2009], 8, 1), (32, [29, 1, 3101], 40, 1), (16, [0, 9, 33], 17, 0)])
def test_rows_that_end_before_a_bad_page_keep_theirs(page, cached, L, bad, int4):
    """The new tokens cross into a page that the table does not name (`bad` pages past the one that the first of them is in): those
    before it are what they should be, those behind it NaN. Sequences that are cut between CTAs among them."""
    c = make(63, L, 8, 2, 64, page, int4, cached)
    first = []
    for s in range(3):
        entry = cached[s] // page + bad
        c["table"][s, entry] = -1 if s % 2 else c["cache"].n_pages
        first.append(max(0, entry * page - cached[s]))
    got = attend(c)
    assert H.device_error(clear=True) == 0x203
    check_groups(c, got, first)
    got = got.cpu().view(3, L, -1)
    for s in range(3):
        assert torch.isnan(got[s, first[s]:]).all() and first[s] < L, s
