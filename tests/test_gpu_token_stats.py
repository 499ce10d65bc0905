"""Token statistics (log-probability, entropy, top alternatives) and their gradient against the
fp64 oracle, at the sizes, strides and masks where they can go wrong.

Tolerances, with u = 2^-24 (half a step of fp32). A row's sum of exp(z - m) is added up in chains of
at most V / 128 + 32 terms and a tree; each term carries the rounding of z - m (relative error u of
the difference, so |z - m| u of the term, and p |log p| adds up to the entropy, at most log V <= 19),
of its product with log2 e (the same again) and of ex2 (2 ulp = 4 u): the sum is off by at most
    tol_s = (V / 128 + 32 + 2 * 19 + 8) u  relative,
    logp   (z_id - m) - c:  tol_s + 2 u (|z_id - m| + |c|) + u |logp|
    entropy c - w / s:      tol_s + (2 tol_s + 4 u) entropy + 2 u |c|; both may be sums relative to a number up to
        8 steps of 2 below m, which adds 8 times their own error (V / 1024 + 9 u: a quarter of a thread's V / 256
        terms in each of four chains), less than tol_s
    gradient, given norm and entropy rounded to fp32: p is off by e_p = u (4 |log p| + |c| + 8) relative,
        the weight g_logp + g_entropy (log p + H) by 4 u of the magnitudes in it; and the result is
        rounded to its type (half a step, eps / 2). ex2 flushes probabilities under 2^-126: 2e-38 of
        the weights."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.helpers import dev_f32, dev_i32, host_f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
INF = float("inf")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    B.build()
    H.load()
    H.device_error(clear=True)
    yield
    assert H.device_error(clear=True) == 0


def rows_of(values, dtype, ld=None, shift=0):
    """Device rows of `values` at stride ld, the first `shift` elements behind a 16-byte boundary; NaN around."""
    n, v = values.shape
    ld = ld or v
    buf = torch.full((n * ld + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    out = buf[shift:shift + n * ld].view(n, ld)
    out[:, :v] = torch.from_numpy(values).cuda().to(dtype)
    return out[:, :v], buf


def make(seed, S, L, V, dtype, mask=None, spread=3.0, ld=None, shift=0):
    """(device logits, the fp64 values they hold, ids, lengths): ragged, the first sequence whole, the last empty."""
    rng = np.random.default_rng(seed)
    z = rng.normal(0, spread, (S * L, V)) * 10 ** rng.uniform(-1, 0.5, (S * L, 1))
    if mask is not None:
        low = -INF if mask == "inf" else float(torch.finfo(dtype).min)
        z[rng.random((S * L, V)) < 0.7] = low
        z[::5] = np.where(np.arange(V) == V // 2, 1.5, low)  # one token left
        z[2::5] = low                                       # nothing left
    dev, buf = rows_of(z, dtype, ld, shift)
    lengths = rng.integers(0, L + 1, S)
    lengths[0], lengths[-1] = L, (0 if S > 1 else L)
    return dev, host_f64(dev), rng.integers(0, V, S * L), lengths, buf


def run_stats(z, ids, lengths, S, L, k):
    rows = S * L
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    o = {"logp": nan(rows), "entropy": nan(rows), "norm": nan(rows, 2)}
    if k:
        o["top_ids"] = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
        o["top_logp"] = nan(rows, k)
    H.hydra_token_logprobs_entropy(z, None if ids is None else dev_i32(ids), None if lengths is None else dev_i32(lengths),
                                   S, L, **o)
    return o


def close(got, want, tol, what):
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


def tol_sum(V):
    return (V / 128 + 32 + 2 * 19 + 8) * U


def check_stats(o, z, ids, lengths, S, L, k):
    V = z.shape[1]
    r = O.token_stats(z, ids, lengths, S, L, k)
    ts, c = tol_sum(V), np.abs(np.where(np.isfinite(r["norm"][:, 1]), r["norm"][:, 1], 0))
    shift = lambda lp: ts + 2 * U * (np.abs(np.where(np.isfinite(lp), lp, 0)) + 2 * c) + U * np.abs(np.where(np.isfinite(lp), lp, 0))  # noqa: E731
    norm = host_f64(o["norm"])
    assert np.array_equal(norm[:, 0], r["norm"][:, 0])
    close(norm[:, 1], r["norm"][:, 1], ts + 2 * U * c, "log-sum")
    if ids is not None:
        close(host_f64(o["logp"]), r["logp"], shift(r["logp"]), "logp")
    close(host_f64(o["entropy"]), r["entropy"], ts + (2 * ts + 4 * U) * r["entropy"] + 2 * U * c, "entropy")
    if k:
        assert np.array_equal(o["top_ids"].cpu().numpy(), r["top_ids"])
        close(host_f64(o["top_logp"]), r["top_logp"], ts + 3 * U * np.abs(np.where(np.isfinite(r["top_logp"]), r["top_logp"], 0))
              + 4 * U * c[:, None], "top_logp")


SIZES = [  # S, L, V, ld, shift, k
    (1, 1, 1, 1, 0, 1),
    (2, 3, 2, 5, 1, 2),
    (3, 2, 31, 31, 0, 31),
    (1, 4, 32, 33, 3, 32),
    (2, 2, 257, 257, 0, 32),
    (3, 5, 1000, 1000, 0, 20),
    (2, 3, 1001, 1003, 1, 8),
    (2, 2, 2048, 2048, 0, 1),
    (2, 2, 4095, 4097, 2, 32),
    (3, 3, 8191, 8192, 0, 5),
    (1, 1, 32000, 32000, 0, 20),
    (5, 3, 32000, 32008, 0, 0),
    (2, 5, 32001, 32001, 7, 32),
    (1, 2, 131071, 131073, 1, 20),
    (1, 1, 262147, 262147, 5, 32),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mask", [None, "inf", "lowest"])
@pytest.mark.parametrize("S,L,V,ld,shift,k", SIZES)
def test_stats_parity(S, L, V, ld, shift, k, mask, dtype):
    z, values, ids, lengths, _ = make(V + S, S, L, V, DTYPES[dtype], mask, ld=ld, shift=shift)
    check_stats(run_stats(z, ids, lengths, S, L, k), values, ids, lengths, S, L, k)


@pytest.mark.parametrize("rows", [1, 2, 9, 18, 19, 37, 38, 75, 76, 77, 150, 151, 152, 153, 303, 305, 700, 1300])
def test_stats_by_number_of_rows(rows):
    """However many CTAs share a row."""
    z, values, ids, _, _ = make(rows, rows, 1, 5003, torch.bfloat16)
    check_stats(run_stats(z, ids, None, rows, 1, 7), values, ids, None, rows, 1, 7)


@pytest.mark.parametrize("rows", [1, 40, 400])
def test_top_of_rows_with_ties_and_clusters(rows):
    """Equal values everywhere, ascending and descending rows, the best in one thread's slots only, more
    equal candidates than are ranked at once, zeros of both signs."""
    V, k = 40000, 32
    base = np.zeros((rows, V))
    i = np.arange(V)
    kinds = [np.zeros(V), i * 2.0 ** -10, -i * 2.0 ** -10, np.where(i % 2 == 0, 0.0, -0.0), np.where(i % 7 == 3, 1.0, 0.0),
             np.where((i // 8) % 256 == 17, 4.0, 0.0), np.where((i // 4) % 256 == 200, 4.0 + (i % 5), -1.0),
             np.where((i // 8) % 2048 < 40, 1.0 + (i % 3), 0.0), np.where(i >= V - 3, 9.0, 2.0),
             np.where((i // 4) % 512 < 33, 1.0 + i * 2.0 ** -12, 0.0)]
    for n in range(rows):
        base[n] = kinds[n % len(kinds)]
    for dtype in (torch.float32, torch.bfloat16):
        z, _ = rows_of(base, dtype, V + 3, 1)
        o = {"top_ids": torch.full((rows, k), -7, dtype=torch.int32, device="cuda"),
             "top_logp": torch.full((rows, k), float("nan"), device="cuda")}
        H.hydra_token_logprobs_entropy(z, None, None, rows, 1, **o)
        r = O.token_stats(host_f64(z), None, None, rows, 1, k)
        assert np.array_equal(o["top_ids"].cpu().numpy(), r["top_ids"])


@pytest.mark.parametrize("S,L,k", [(1, 700, 3), (5, 300, 0), (32, 41, 5), (127, 13, 0), (128, 11, 8), (129, 11, 8), (700, 2, 0),
                                   (900, 3, 2)])
def test_ragged_batches_of_more_rows_than_ctas(S, L, k):
    """Few sequences have their live rows dealt by number, many by row: empty ones, full ones and one token."""
    V = 600
    z, values, ids, lengths, _ = make(S + L, S, L, V, torch.bfloat16, ld=603, shift=1)
    lengths[1::4], lengths[2::7] = 0, 1
    check_stats(run_stats(z, ids, lengths, S, L, k), values, ids, lengths, S, L, k)
    lengths[:] = 0
    check_stats(run_stats(z, ids, lengths, S, L, k), values, ids, lengths, S, L, k)


@pytest.mark.parametrize("rows,V,k", [(20000, 37, 9), (5000, 1, 1), (3000, 300, 32)])
def test_many_short_rows(rows, V, k):
    z, values, ids, _, _ = make(V, rows, 1, V, torch.float32)
    check_stats(run_stats(z, ids, None, rows, 1, k), values, ids, None, rows, 1, k)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mask", [None, "inf", "lowest"])
@pytest.mark.parametrize("S,L,V,ld,shift", [(5, 3, 1, 1, 0), (700, 3, 33, 35, 1), (3, 7, 1000, 1003, 3), (7, 3, 2047, 2051, 5),
                                            (30, 60, 6100, 6101, 1), (9, 170, 9001, 9001, 7), (5, 300, 13001, 13003, 1)])
def test_stats_without_alternatives(S, L, V, ld, shift, mask, dtype):
    """A warp a row, up to where the rows are long or few, and beyond: ragged, with rows that start anywhere. Of 6100
    logits a lane adds 96 terms to each of its two sums, and six steps join them: with the terms' own 8 fewer
    than the 125 that the tolerance counts."""
    z, values, ids, lengths, _ = make(V + S, S, L, V, DTYPES[dtype], mask, ld=ld, shift=shift)
    check_stats(run_stats(z, ids, lengths, S, L, 0), values, ids, lengths, S, L, 0)
    only = torch.full((S * L,), float("nan"), device="cuda")
    H.hydra_token_logprobs_entropy(z, None, dev_i32(lengths), S, L, entropy=only)
    assert torch.equal(only, run_stats(z, ids, lengths, S, L, 0)["entropy"])


def test_short_rows_report_bad_ids_and_lengths():
    z, values, _, _, _ = make(3, 4, 3, 200, torch.float32)
    ids = np.full(12, 7)
    ids[5] = 200
    o = run_stats(z, ids, None, 4, 3, 0)
    assert H.device_error(clear=True) == 0x201 and torch.isnan(o["logp"][5]) and int(torch.isnan(o["logp"]).sum()) == 1
    for bad in (-1, 4):
        lengths = np.array([3, bad, 0, 2])
        o = run_stats(z, np.full(12, 7), lengths, 4, 3, 0)
        assert H.device_error(clear=True) == 0x202
        lengths[1] = 0 if bad < 0 else 3
        check_stats(o, values, np.full(12, 7), lengths, 4, 3, 0)


@pytest.mark.parametrize("rows", [2, 500])
def test_more_candidates_than_are_ranked_at_once(rows):
    """Values above the bound, equal to it and NaN, each in more places than fit: 32 lanes of a group share
    slots that hold them all."""
    V, k = 66000, 32
    i = np.arange(V)
    group = (i // 8) % 256 < 4  # four threads' slots of every 256
    kinds = [np.where(group, 1.0 + (i % 977) * 2.0 ** -6, 0.0),             # hundreds above any bound
             np.where(group, 2.0, np.where(i % 50 == 0, 1.0, 0.0)),         # thousands equal at the top
             np.where(i % 7 == 0, np.nan, 1.0),                             # thousands of NaN
             np.where(i > V - 400, 3.0, np.where(i % 9 == 0, 2.0, 1.0)),    # equal ones at the very end
             np.where(i < 10, 5.0, -np.inf)]                                # fewer than k, then -inf by index
    base = np.stack([kinds[n % len(kinds)] for n in range(rows)])
    z, _ = rows_of(base, torch.bfloat16, V + 1, 1)
    ids = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    logp = torch.zeros(rows, k, device="cuda")
    H.hydra_token_logprobs_entropy(z, None, None, rows, 1, top_ids=ids, top_logp=logp)
    values = np.where(np.isnan(base), np.inf, host_f64(z))  # NaN first, by index
    want = np.argsort(-values[:5], axis=1, kind="stable")[:, :k]
    got = ids.cpu().numpy()
    for n in range(rows):
        assert np.array_equal(got[n], want[n % 5]), n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V", [(1, 600000), (40, 262147), (4, 1 << 20)])
def test_large_logits_in_the_same_places_of_every_run(rows, V, dtype):
    """Ascending, descending and shuffled values that recur in a few slots of every 256, tens of thousands beyond
    any bound, with ties among the best."""
    k, t = 32, DTYPES[dtype]
    per = 4 if t is torch.float32 else 8
    rng = np.random.default_rng(V)
    i = np.arange(V)
    at = i[(i // per) % 256 < 12]
    z = np.zeros((rows, V))
    for n in range(rows):
        value = np.linspace(1, 200, len(at))
        z[n, at] = [value, value[::-1], rng.permutation(value), np.round(value / 16)][n % 4]
    dev, _ = rows_of(z, t, V + 3, 1)
    values = host_f64(dev)
    ids = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    H.hydra_token_logprobs_entropy(dev, None, None, rows, 1, top_ids=ids, top_logp=torch.zeros(rows, k, device="cuda"))
    want = np.argsort(-values, axis=1, kind="stable")[:, :k]
    assert np.array_equal(ids.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_stats_of_large_and_infinite_logits(dtype):
    """Large magnitudes cancel exactly; NaN and +inf make the row NaN and come first among the top."""
    V = 3001
    rng = np.random.default_rng(3)
    z = rng.normal(0, 1, (6, V))
    z[0] += 30000.0
    z[1] -= 30000.0
    z[2, 100], z[2, 2000] = 1e38, 1e38
    z[3] = -3e38
    z[4, 77] = INF
    z[5, 55], z[5, 99] = float("nan"), INF
    dev, _ = rows_of(z, DTYPES[dtype])
    values = host_f64(dev)
    ids = rng.integers(0, V, 6)
    o = run_stats(dev, ids, None, 6, 1, 4)
    top = {k: v[:4] for k, v in o.items()}
    check_stats(top, values[:4], ids[:4], None, 4, 1, 4)
    for key in ("logp", "entropy"):
        assert torch.isnan(o[key][4:]).all()
    assert torch.isnan(o["norm"][4:, 1]).all() and torch.isnan(o["top_logp"][4:]).all()
    assert o["top_ids"][4, 0] == 77 and o["top_ids"][5, :2].tolist() == [55, 99]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V", [(1, 32000), (40, 32001), (700, 4100)])
def test_masks_of_the_lowest_value_that_leave_few_tokens(rows, V, dtype):
    """None, one, fewer than k, just k or a few more tokens left, -inf beside the lowest value, all -inf but one and
    another row of the largest value: the statistics, the top and the gradient."""
    k, t = 20, DTYPES[dtype]
    rng = np.random.default_rng(V)
    low, high = float(torch.finfo(t).min), float(torch.finfo(t).max)
    z = np.full((rows, V), low)
    for n in range(rows):
        left = [0, 1, 7, 0, 20, 23, 300, 0][n % 8]
        at = rng.choice(V, left, replace=False)
        if n % 8 == 3:
            z[n, rng.random(V) < 0.5] = -INF  # equal weights on the rest
        elif n % 8 == 7:
            z[n] = high if n % 16 == 7 else -INF
            z[n, V // 3] = low if n % 16 == 15 else high
        z[n, at] = rng.normal(0, 3, left)
    dev, _ = rows_of(z, t)
    values, ids = host_f64(dev), rng.integers(0, V, rows)
    check_stats(run_stats(dev, ids, None, rows, 1, k), values, ids, None, rows, 1, k)
    gl, gh = (rng.normal(size=rows).astype(np.float32) for _ in range(2))
    r = O.token_stats(values, None, None, rows, 1)
    for t_out in DTYPES.values():
        d, _ = run_grad(dev, ids, None, rows, 1, r["norm"], r["entropy"], gl, gh, t_out)
        check_grad(d, values, ids, None, rows, 1, r, gl.astype(float), gh.astype(float))


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_nothing_but_positive_infinity(dtype):
    z, _ = rows_of(np.full((2, 5000), INF), DTYPES[dtype])
    o = run_stats(z, np.zeros(2, np.int64), None, 2, 1, 3)
    for key in ("logp", "entropy", "top_logp"):
        assert torch.isnan(o[key]).all(), key
    assert torch.isnan(o["norm"][:, 1]).all()
    assert o["top_ids"].tolist() == [[0, 1, 2]] * 2


def test_stats_outputs_one_by_one_and_dead_rows():
    """Each output alone equals it among all; rows behind a sequence's end are not read (NaN there)."""
    S, L, V, k = 3, 4, 5001, 6
    z, values, ids, lengths, _ = make(11, S, L, V, torch.float32)
    dead = np.arange(L)[None] >= lengths[:, None]
    z[torch.from_numpy(dead.reshape(-1)).cuda()] = float("nan")
    every = run_stats(z, ids, lengths, S, L, k)
    assert not np.isnan(host_f64(every["logp"])).any()
    for name in ("logp", "entropy", "norm"):
        one = torch.full_like(every[name], float("nan"))
        H.hydra_token_logprobs_entropy(z, dev_i32(ids) if name == "logp" else None, dev_i32(lengths), S, L, **{name: one})
        plain = run_stats(z, ids, lengths, S, L, 0)[name]
        assert torch.equal(one, plain)


def test_stats_bad_id_and_bad_length_are_reported():
    z, values, ids, _, _ = make(12, 2, 3, 2001, torch.bfloat16)
    for bad in (-1, 2001, 1 << 30):
        wrong = ids.copy()
        wrong[1] = bad
        o = run_stats(z, wrong, None, 2, 3, 2)
        assert H.device_error(clear=True) == 0x201
        assert np.isnan(host_f64(o["logp"])[1]) and not np.isnan(np.delete(host_f64(o["logp"]), 1)).any()
    for bad, rows in ((-1, 0), (4, 3)):
        o = run_stats(z, ids, np.array([3, bad]), 2, 3, 2)
        assert H.device_error(clear=True) == 0x202
        check_stats(o, values, ids, np.array([3, rows]), 2, 3, 2)


# ---------------------------------------------------------------- gradient


def run_grad(z, ids, lengths, S, L, norm, entropy, gl, gh, out_dtype, ld=None, shift=0, into=None):
    d, buf = (into, None) if into is not None else rows_of(np.full((S * L, z.shape[1]), 7.0), out_dtype, ld, shift)
    f = lambda a: None if a is None else dev_f32(a)  # noqa: E731
    H.hydra_token_logprobs_entropy_grad(z, None if ids is None else dev_i32(ids),
                                        None if lengths is None else dev_i32(lengths), S, L, f(norm), f(entropy), f(gl),
                                        f(gh), d)
    return d, buf


def check_grad(d, z, ids, lengths, S, L, r, gl, gh, extra=0.0):
    want = O.token_stats_grad(z, ids, lengths, S, L, gl, gh)
    got = host_f64(d)
    with np.errstate(invalid="ignore", over="ignore"):
        lp = np.where(r["norm"][:, :1] > -INF, z - r["norm"][:, :1], -INF) - r["norm"][:, 1:]
    p = np.exp(lp)
    a = np.minimum(np.abs(lp), 256.0)
    c, h = np.abs(r["norm"][:, 1:]), r["entropy"][:, None]
    weight = (0 if gl is None else np.abs(gl)[:, None]) + (0 if gh is None else np.abs(gh)[:, None] * (a + h + 1))
    half = torch.finfo(d.dtype).eps / 2
    tol = p * weight * (U * (4 * a + c + 12) + extra) + half * (1 + 2.0 ** -6) * np.abs(want) + 4e-38 * (weight + 1)
    if gl is not None:  # 1 - p of the drawn token moves as p does
        rows = np.arange(len(want))
        tol[rows, ids] += 4 * U * np.abs(gl)
    if d.dtype == torch.bfloat16:
        tol += 2.0 ** -133  # the smallest step
    close(got, want, tol, "gradient")


GRAD_SIZES = [  # S, L, V, ld, shift, ld_d, shift_d
    (1, 1, 1, 1, 0, 1, 0),
    (2, 3, 7, 9, 1, 9, 1),
    (2, 2, 8, 8, 0, 8, 0),
    (3, 7, 1001, 1001, 0, 1001, 0),
    (3, 2, 1001, 1001, 3, 1005, 3),
    (2, 2, 4096, 4096, 0, 4096, 0),
    (2, 2, 4097, 4099, 1, 4099, 2),   # the two rows start apart on the 16-byte grid
    (2, 3, 8195, 8200, 4, 8200, 4),
    (1, 2, 32000, 32000, 0, 32000, 0),
    (1, 1, 131073, 131073, 0, 131073, 5),
]


@pytest.mark.parametrize("types", ["f32/f32", "f32/bf16", "bf16/bf16", "bf16/f32"])
@pytest.mark.parametrize("mask", [None, "inf", "lowest"])
@pytest.mark.parametrize("S,L,V,ld,shift,ld_d,shift_d", GRAD_SIZES)
def test_grad_parity(S, L, V, ld, shift, ld_d, shift_d, mask, types):
    t_in, t_out = (DTYPES[x] for x in types.split("/"))
    z, values, ids, lengths, _ = make(V + 3 * S, S, L, V, t_in, mask, ld=ld, shift=shift)
    rng = np.random.default_rng(V)
    gl, gh = (rng.normal(size=S * L).astype(np.float32) for _ in range(2))
    r = O.token_stats(values, None, None, S, L)
    for a, b in ((gl, gh), (gl, None), (None, gh)):
        d, buf = run_grad(z, ids if a is not None else None, lengths, S, L, r["norm"], r["entropy"] if b is not None else None,
                          a, b, t_out, ld_d, shift_d)
        check_grad(d, values, ids, lengths, S, L, r, None if a is None else a.astype(float), None if b is None else b.astype(float))
        outside = buf.clone()
        outside[shift_d:shift_d + S * L * ld_d].view(S * L, ld_d)[:, :V] = float("nan")
        assert torch.isnan(outside).all()  # nothing beyond the columns was written


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ld,shift", [(5000, 0), (5003, 1)])
def test_grad_in_place_has_the_same_bits(dtype, ld, shift):
    S, L, V = 3, 4, 5000
    z, values, ids, lengths, _ = make(21, S, L, V, DTYPES[dtype], "inf", ld=ld, shift=shift)
    gl, gh = np.linspace(-1, 1, S * L), np.full(S * L, -0.01)
    r = O.token_stats(values, None, None, S, L)
    d, _ = run_grad(z, ids, lengths, S, L, r["norm"], r["entropy"], gl, gh, DTYPES[dtype], ld, shift)
    run_grad(z, ids, lengths, S, L, r["norm"], r["entropy"], gl, gh, None, into=z)
    assert torch.equal(z, d)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ld,shift", [(4100, 0), (4103, 3)])
def test_grad_in_place_where_the_lowest_value_masks(dtype, ld, shift):
    S, L, V = 3, 5, 4099
    z, values, ids, lengths, _ = make(22, S, L, V, DTYPES[dtype], "lowest", ld=ld, shift=shift)
    gl, gh = np.linspace(-1, 1, S * L), np.full(S * L, -0.01)
    r = O.token_stats(values, None, None, S, L)
    d, _ = run_grad(z, ids, lengths, S, L, r["norm"], r["entropy"], gl, gh, DTYPES[dtype], ld, shift)
    run_grad(z, ids, lengths, S, L, r["norm"], r["entropy"], gl, gh, None, into=z)
    assert torch.equal(z, d)


def test_grad_against_differences():
    """The kernel's gradient against central differences of the oracle's loss: with steps of 1e-4
    the differences are off by 1e-8 / 6 times a third derivative under 10, the kernel by fp32."""
    S, L, V = 2, 2, 23
    z, values, ids, _, _ = make(31, S, L, V, torch.float32, spread=1.0)
    gl, gh = np.array([0.5, -1.0, 2.0, 0.1]), np.array([0.3, 0.2, -0.7, 1.0])
    o = run_stats(z, ids, None, S, L, 0)
    d, _ = run_grad(z, ids, None, S, L, host_f64(o["norm"]), host_f64(o["entropy"]), gl, gh, torch.float32)

    def loss(y):
        r = O.token_stats(y, ids, None, S, L)
        return (gl * r["logp"] + gh * r["entropy"]).sum()

    for i in range(S * L):
        for v in range(V):
            up, down = values.copy(), values.copy()
            up[i, v] += 1e-4
            down[i, v] -= 1e-4
            assert abs((loss(up) - loss(down)) / 2e-4 - host_f64(d)[i, v]) <= 1e-6


def test_grad_bad_id_writes_nan_and_is_reported():
    z, values, ids, _, _ = make(12, 2, 3, 2001, torch.bfloat16)
    ids[1] = 2001
    r = O.token_stats(values, None, None, 2, 3)
    d, _ = run_grad(z, ids, None, 2, 3, r["norm"], r["entropy"], np.ones(6), None, torch.float32)
    assert H.device_error(clear=True) == 0x201
    assert torch.isnan(d[1]).all() and not torch.isnan(d[[0, 2, 3, 4, 5]]).any()


# ---------------------------------------------------------------- as they are used


def _update(z, ids, lengths, S, L, o, g):
    """Losses of the new log-probabilities and their gradient in the logits: the calls of one minibatch."""
    H.hydra_token_logprobs_entropy(z, ids, lengths, S, L, o["logp"], o["entropy"], o["norm"])
    H.hydra_ppo_loss(o["logp"].view(S, L), g["old"], g["adv"], g["ret"], g["val"], lengths, 0.2, False, o["gl"].view(S, L),
                     o["gv"], o["stats"], o["ws"])
    H.hydra_token_logprobs_entropy_grad(z, ids, lengths, S, L, o["norm"], o["entropy"], o["gl"], g["gh"], o["d"])


def _update_state(S, L, V, dtype, seed=41):
    z, values, ids, lengths, _ = make(seed, S, L, V, dtype)
    rng = np.random.default_rng(seed)
    f = lambda *s: dev_f32(rng.normal(size=s))  # noqa: E731
    old = O.token_stats(values, ids, None, S, L)["logp"].reshape(S, L) + rng.normal(0, 0.1, (S, L))
    g = {"old": dev_f32(old), "adv": f(S, L), "ret": f(S, L), "val": f(S, L), "gh": dev_f32(np.full(S * L, -0.01 / 30))}
    nan = lambda *s, dtype=torch.float32: torch.full(s, float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    o = {"logp": nan(S * L), "entropy": nan(S * L), "norm": nan(S * L, 2), "gl": nan(S * L), "gv": nan(S, L),
         "stats": nan(7, dtype=torch.float64), "d": nan(S * L, V, dtype=dtype),
         "ws": torch.empty(H.ppo_workspace_size(), dtype=torch.uint8, device="cuda")}
    return z, values, ids, lengths, o, g


def test_minibatch_from_logits_to_their_gradient():
    S, L, V = 4, 30, 4003
    z, values, ids, lengths, o, g = _update_state(S, L, V, torch.float32)
    _update(z, dev_i32(ids), dev_i32(lengths), S, L, o, g)
    gl, gh = host_f64(o["gl"]), host_f64(g["gh"])
    loss = O.ppo_loss(host_f64(o["logp"]).reshape(S, L), host_f64(g["old"]), host_f64(g["adv"]), host_f64(g["ret"]),
                      host_f64(g["val"]), lengths)
    np.testing.assert_allclose(gl.reshape(S, L), loss["grad_logp"], rtol=1e-5, atol=1e-6 * np.abs(loss["grad_logp"]).max())
    check_grad(o["d"], values, ids, lengths, S, L, O.token_stats(values, None, None, S, L), gl, gh, extra=8 * tol_sum(V))


def test_captured_graph_and_other_stream():
    """The same calls captured and replayed over new logits, and on another stream, give the same bits."""
    S, L, V = 3, 5, 33000
    z, values, ids, lengths, o, g = _update_state(S, L, V, torch.bfloat16)
    ids, lengths = dev_i32(ids), dev_i32(lengths)
    _update(z, ids, lengths, S, L, o, g)
    want = {k: o[k].clone() for k in ("logp", "entropy", "norm", "gl", "d")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _update(z, ids, lengths, S, L, o, g)
    keep = z.clone()
    z.zero_()
    graph.replay()
    z.copy_(keep)
    graph.replay()
    assert all(torch.equal(o[k], want[k]) for k in want)
    for k in want:
        o[k].fill_(float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _update(z, ids, lengths, S, L, o, g)
    side.synchronize()
    assert all(torch.equal(o[k], want[k]) for k in want)


def test_calls_on_two_streams_at_once():
    """Neither keeps anything that the other uses."""
    a, b = (_update_state(6, 40, 32000, torch.bfloat16, seed) for seed in (51, 52))
    want = []
    for z, _, ids, lengths, o, g in (a, b):
        _update(z, dev_i32(ids), dev_i32(lengths), 6, 40, o, g)
        want.append({k: o[k].clone() for k in ("logp", "entropy", "norm", "gl", "d")})
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    args = [(dev_i32(x[2]), dev_i32(x[3])) for x in (a, b)]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, (z, _, _, _, o, g), (ids, lengths) in zip(streams, (a, b), args):
            with torch.cuda.stream(st):
                _update(z, ids, lengths, 6, 40, o, g)
    torch.cuda.synchronize()
    for w, x in zip(want, (a, b)):
        assert all(torch.equal(x[4][k], w[k]) for k in w)


def test_update_from_logits_to_clipped_lora_gradients():
    """An update of the head's LoRA set as it would be made: statistics, losses, the gradient in the logits, the
    gradients of A and B (z = x W^T + (x A^T) B^T), and these clipped."""
    S, L, V, d, r = 4, 25, 2000, 64, 8
    g = torch.Generator(device="cuda").manual_seed(3)
    x, W, A, B = (torch.randn(*s, device="cuda", generator=g) * c for s, c in
                  (((S * L, d), 1.0), ((V, d), 0.2), ((r, d), 0.2), ((V, r), 0.2)))
    z = x @ W.T + (x @ A.T) @ B.T
    _, _, ids, lengths, o, gr = _update_state(S, L, V, torch.float32)
    values = host_f64(z)
    gr["old"] = dev_f32(O.token_stats(values, ids, None, S, L)["logp"].reshape(S, L) + 0.05)
    _update(z, dev_i32(ids), dev_i32(lengths), S, L, o, gr)
    dA, dB = (o["d"] @ B).T @ x, o["d"].T @ (x @ A.T)
    n2, ws = torch.zeros(2, device="cuda"), torch.empty(H.grad_norm_workspace_size(), dtype=torch.uint8, device="cuda")
    grads = [dA.contiguous(), dB.to(torch.bfloat16).contiguous()]
    before = [host_f64(t) for t in grads]
    H.hydra_clip_grad_norm(H.GradList(grads), 1e-3, n2, ws)
    norm, coef, want = O.clip_grad_norm(before, 1e-3)
    assert coef < 1 and abs(n2[0].item() - norm) <= 20 * U * norm
    for t, w in zip(grads, want):
        assert np.all(np.abs(host_f64(t) - w) <= (24 * U + torch.finfo(t.dtype).eps / 2 * 1.02) * np.abs(w) + 2.0 ** -133)
    # and the whole chain: the gradient of the fp64 loss in A, whose fp32 products are off by their sums of 100 and 2000
    lp = O.token_stats(values, ids, lengths, S, L)
    loss = O.ppo_loss(lp["logp"].reshape(S, L), host_f64(gr["old"]), host_f64(gr["adv"]), host_f64(gr["ret"]),
                      host_f64(gr["val"]), lengths)
    dz = O.token_stats_grad(values, ids, lengths, S, L, loss["grad_logp"].reshape(-1), host_f64(gr["gh"]))
    exact = (dz @ host_f64(B)).T @ host_f64(x)
    size = (np.abs(dz) @ np.abs(host_f64(B))).T @ np.abs(host_f64(x))
    assert np.all(np.abs(before[0] - exact) <= 1e-3 * size)  # TF32 products, if they are on, are off by 2^-11 a factor


def test_rows_far_into_a_large_buffer():
    """Offsets beyond 2^31 elements: the last of three rows 1.2e9 elements apart."""
    S, V, ld = 3, 1001, 1_200_000_001
    buf = torch.empty(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((S, V), (ld, 1))
    z.copy_(torch.randn(S, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)))
    ids = np.array([0, 500, 1000])
    o = run_stats(z, ids, None, S, 1, 5)
    values = host_f64(z)
    check_stats(o, values, ids, None, S, 1, 5)
    r = O.token_stats(values, None, None, S, 1)
    run_grad(z, ids, None, S, 1, r["norm"], r["entropy"], np.ones(S), np.ones(S), None, into=z)
    check_grad(z, values, ids, None, S, 1, r, np.ones(S), np.ones(S))
