"""Attention over a paged cache at its limits: groups of channels of very different size, bad pages that only some rows of
an item read, infinite keys, scores of any size. Tolerances as tests/test_gpu_paged_attention.py derives them, with u = 2^-24 and e for a score's error, but for what
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

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    B.build()
    H.load()
    H.device_error(clear=True)
    yield
    assert H.device_error(clear=True) == 0


def check_one(q, k, v, cached, scale, got, what="", step=2.0 ** -28):
    """Rows [n, heads, D] of one sequence over held keys and values [cached + n, kv heads, D]: every channel against its own
    group's tolerance."""
    n, heads, D = q.shape
    N, kv = k.shape[:2]
    by = heads // kv
    ref, size, reach = O.cached_attention(q, k, v, cached, scale)
    coarse = np.abs(q).max(-1) * np.abs(k).sum(-1).max(0).repeat(by)[None] * scale
    e = ((2 * (D + D // 16) + 16) * U * reach + step * coarse)[..., None]
    largest = np.abs(v).reshape(N, kv, D // 64, 64).max(-1)  # of a token, head and group
    most = np.zeros((n, heads, D // 64))
    for t in range(n):
        for h in range(heads):
            z = k[:cached + t + 1, h // by] @ q[t, h] * scale
            p = np.exp(z - z.max())
            most[t, h] = (p[:, None] / p.sum() * largest[:cached + t + 1, h // by]).max(0)
    tol = (2.0 ** -11 + 2 * e + (N + 128) * U) * size + N * 2.0 ** -30 * most.repeat(64, -1)
    tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
    off = np.abs(got - ref)
    assert np.isfinite(got).all() and (off <= tol).all(), f"{what}: {np.max(off / np.maximum(tol, 1e-300)):.3g}"


def fp64(c, got):
    """(queries, output) [S, L, heads, D]"""
    return (x.double().cpu().numpy().reshape(c["S"], c["L"], c["heads"], c["D"]) for x in (c["q"], got))


def check_groups(c, got, rows=None):
    """`rows`: of the first so many new tokens of each sequence."""
    q, got = fp64(c, got)
    for s in range(c["S"]):
        n, at = int(c["lengths"][s] if rows is None else rows[s]), int(c["cached"][s])
        k, v = (c[x][s, :at + n].astype(np.float64) for x in ("k", "v"))
        if n > 0:
            check_one(q[s, :n], k, v, at, c["D"] ** -0.5, got[s, :n], f"sequence {s}")


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


@pytest.mark.parametrize("cached", [[1, 37, 200], [1, 3100, 37], [4, 12]])  # (a CTA an item, shared ones, few tiles)
@pytest.mark.parametrize("what", [INF, -INF])
@pytest.mark.parametrize("D", [64, 128])
def test_an_infinite_key_in_a_bf16_cache(D, what, cached):
    """Token 1 of each sequence has it in one channel: its score is +inf or -inf by the query's sign there, which makes the
    head NaN or drops the token."""
    def change(k, v):
        k[:, 1, :, 9] = what

    c = make(64, 2, 4, 2, D, 16, False, cached, change=change)
    q, got = fp64(c, attend(c))
    assert (q[..., 9] != 0).all()
    for s, at in enumerate(cached):
        k, v = (np.delete(c[x][s, :at + 2].astype(np.float64), 1, axis=0) for x in ("k", "v"))
        for h in range(4):
            for t in range(2):
                if np.sign(q[s, t, h, 9]) == np.sign(what):
                    assert np.isnan(got[s, t, h]).all(), (s, t, h)
                else:
                    check_one(q[s, t:t + 1, h:h + 1], k[:at + t, h // 2:h // 2 + 1], v[:at + t, h // 2:h // 2 + 1], at + t - 1, D ** -0.5,
                              got[s, t:t + 1, h:h + 1], f"{s}, {t}, {h}")


@pytest.mark.parametrize("cached", [[0, 37, 200], [0, 3100, 37], [500] * 40])
@pytest.mark.parametrize("what", [INF, -INF, NAN])
@pytest.mark.parametrize("int4", [True, False])
def test_keys_that_leave_a_query_nothing(int4, what, cached):
    """Every key has it: all scores are infinite or NaN, however the work is cut."""
    def change(k, v):
        k[..., 9] = what

    c = make(65, 2, 4, 2, 64, 16, int4, cached, change=change)
    assert torch.isnan(attend(c)).all()


@pytest.mark.parametrize("what", [INF, -INF, NAN])
@pytest.mark.parametrize("kind", ["int4", "bf16"])
def test_one_sick_key_and_the_queries_before_it(kind, what):
    """The last but one of four new tokens: queries before it are what they were; in 4 bits the others are NaN."""
    def change(k, v):
        k[:, -2, :, 9] = what

    c, calm = (make(66, 4, 4, 2, 64, 16, kind == "int4", [29, 29], change=f) for f in (change, None))
    got, ref = (attend(x).view(2, 4, -1) for x in (c, calm))
    assert torch.equal(got[:, :2], ref[:, :2])
    if kind == "int4" or what != what:
        assert torch.isnan(got[:, 2:]).all()


@pytest.mark.parametrize("cached", [[70, 0, 200], [3000, 37]])
@pytest.mark.parametrize("sign", [0, 1, -1])
@pytest.mark.parametrize("size", [1e4, 1e6, 1e9, 1e14, 1e33])
@pytest.mark.parametrize("int4", [True, False])
def test_scores_of_any_size(int4, size, sign, cached):
    """Scores of about +-size (of one sign, or both): where the largest leads by more than the others can be off, its value is the
    output. A score is off by e as above and by a product's rounding; then its weight is 1 of all but 2^-30, and enters the sum rounded
    (2^-11 and 16 u), as does its value to bf16."""
    def change(k, v):
        if sign:
            k[:] = np.abs(k)

    by = np.sqrt(size)
    c = make(67, 2, 4, 2, 128, 16, int4, cached, k_by=by, q_by=by, change=change)
    if sign:
        c["q"] = c["q"].abs() * sign
    q, got = fp64(c, attend(c))
    assert np.isfinite(got).all()
    led = 0
    for s, at in enumerate(cached):
        for t in range(2):
            for h in range(4):
                k, v = (c[x][s, :at + t + 1, h // 2].astype(np.float64) for x in ("k", "v"))
                z = k @ q[s, t, h] * 128 ** -0.5
                reach = (np.abs(k) @ np.abs(q[s, t, h])).max() * 128 ** -0.5
                coarse = np.abs(q[s, t, h]).max() * np.abs(k).sum(-1).max() * 128 ** -0.5
                e = (2 * (128 + 8) + 16) * U * reach + 2.0 ** -28 * coarse + 4 * U * np.abs(z).max()
                lead = np.partition(z, -2)[-2:] if len(z) > 1 else np.array([-np.inf, z[0]])
                if lead[1] - lead[0] <= 2 * e + np.log(len(z) * 2.0 ** 30):
                    continue
                led += 1
                one = v[z.argmax()]
                tol = (2.0 ** -11 + 16 * U) * np.abs(one) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(one) + 2.0 ** -30 * np.abs(v).max()
                assert (np.abs(got[s, t, h] - one) <= tol).all(), (s, t, h)
    assert led >= 8


@pytest.mark.parametrize("loud", [0, 1])
@pytest.mark.parametrize("D,channels", [(128, 64), (128, 16), (64, 16)])
@pytest.mark.parametrize("int4", [True, False])
def test_small_channels_of_a_query_that_meet_large_keys(int4, D, channels, loud):
    """The first (or last) channels have queries of 2^-26 and (where they are a group of their own) keys of 2^26 times the others'. A
    query is off by 2^-35 of its head's largest at most, as its largest is put at 2^14 or more and a sixteenth of it has
    steps of 2^-24 then; scores' other errors as above."""
    def change(k, v):
        if channels == 64:
            k[..., at:at + 64] *= 2.0 ** 26

    at = D - channels if loud else 0
    c = make(68, 2, 4, 2, D, 16, int4, [300, 0, 37], change=change)
    x = c["q"].view(-1, 4, D)
    x[..., at:at + channels] *= 2.0 ** -26
    q, got = fp64(c, attend(c))
    for s in range(3):
        n, old = 2, int(c["cached"][s])
        k, v = (c[y][s, :old + n].astype(np.float64) for y in ("k", "v"))
        check_one(q[s], k, v, old, D ** -0.5, got[s], f"sequence {s}", step=2.0 ** -35)


@pytest.mark.parametrize("k_by,q_by", [(1e33, 1e-33), (1e35, 1e-35), (1e-35, 1e35), (1e-30, 1e33), (1e20, 1e-20)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("int4", [True, False])
def test_large_keys_and_small_queries(int4, D, k_by, q_by):
    """And the other way round: what counts is that the score is a number."""
    c = make(69, 3, 4, 2, D, 16, int4, [200, 0, 37], k_by=k_by, q_by=q_by / (k_by * q_by if k_by * q_by > 1 else 1))
    check_groups(c, attend(c))
