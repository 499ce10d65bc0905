"""Attention over a paged cache against the fp64 oracle on the values that the cache holds.

Tolerances, with u = 2^-24. A score is a sum of D exact products in fp32. Sixteen at a time and the sum before are added
aligned to the largest, cut off below its last place: 17 D / 16 terms, each off by 2 u of the largest partial sum at most, so
2 (D + D / 16) u, with 16 u for scales and factors, of the sum of the products' magnitudes (`reach`); in 4 bits a query is
fp16, relative to its row's largest, between 2^7 and 2^8 then, a part of its elements divided by 16: below 2^-14 fp16 has
steps of 2^-24, so an element is off by 2^-21 at most, 2^-28 of the largest, and a score by that times sum_d |k_jd|
(`coarse`). So a weight is off by e = (2 (D + D / 16) + 16) u reach + 2^-28 coarse relative, and the quotient of two sums of
weights twice that. Weights enter the second product rounded to fp16 (half a step: 2^-11 relative) together with their
value's scale, the largest such product of a row at 2^6 or more: below 2^-14 fp16 has steps of 2^-24, so a weight is off by
2^-25 at most, 2^-31 of the largest product w sv. Times a code of up to 15, and sv <= max |v| / 7.5 (a scale is a fifteenth
of its range), that is N 2^-30 max |v| over N tokens. (Two bf16, 2^-16 relative, in a bf16 cache.) The sums themselves are
fp32 over N terms: at most N u, with 128 for the order and for logarithms of up to 128, rounded, by which parts are added up.
So an output is off by
    (2^-11 + 2 e + (N + 128) u) sum_j p_j |v_j| + N 2^-30 max |v|,
and rounded to bf16: half a step, 2^-8 of its value (and of what it is off by)."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.helpers import dev_i32
from tests.test_gpu_paged_cache import pages_for

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    B.build()
    H.load()
    H.device_error(clear=True)
    yield
    assert H.device_error(clear=True) == 0


def make(seed, L, heads, kv, D, page, int4, cached, lengths=None, k_by=1.0, v_by=1.0, q_by=1.0, change=None):
    """A cache with `cached` tokens of each sequence and new ones, all put in by hydra_kv_append without rotation, 0xFF
    (NaN in bf16) everywhere else."""
    rng = np.random.default_rng(seed)
    cached = np.asarray(cached)
    S = len(cached)
    lengths = np.full(S, L) if lengths is None else np.asarray(lengths)
    total = cached + lengths
    table, n_pages = pages_for(rng, total, page)
    cache = H.KvCache(H.HYDRA_KV_INT4 if int4 else H.HYDRA_KV_BF16, n_pages, page, kv, D)
    cache.data.fill_(0xFF)
    N = max(1, int(total.max()))
    loud = 10 ** rng.uniform(-0.5, 0.5, (1, 1, kv, D))
    k = rng.normal(0, 1, (S, N, kv, D)) * loud * k_by
    v = rng.normal(0, 1, (S, N, kv, D)) * 10 ** rng.uniform(-0.5, 0.5, (S, N, kv, 1)) * v_by
    if change is not None:
        change(k, v)
    k, v = (torch.from_numpy(x).bfloat16() for x in (k, v))
    t, full = dev_i32(table), dev_i32(total)
    H.hydra_kv_append(cache, t, None, full, S, N, None, k.reshape(S * N, -1).cuda(), v.reshape(S * N, -1).cuda())
    q = torch.from_numpy(rng.normal(0, q_by, (S * L, heads * D))).bfloat16()
    held = [O.kv_held(x.float().numpy(), int4) for x in (k, v)]
    return {"S": S, "L": L, "heads": heads, "kv": kv, "D": D, "cached": cached, "lengths": lengths, "table": table,
            "cache": cache, "q": q, "k": held[0], "v": held[1]}


def workspace(c):
    n = H.paged_attention_workspace_size(c["S"], c["L"], c["heads"], c["kv"], c["D"])
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")


def attend(c, scale=None, pad=0, ws=None, stream=None):
    rows, cols = c["S"] * c["L"], c["heads"] * c["D"]
    q = torch.full((rows, cols + pad), NAN, dtype=torch.bfloat16, device="cuda")
    q[:, :cols] = c["q"]
    out = torch.full((rows, cols + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    H.hydra_paged_attention(c["cache"], dev_i32(c["table"]), dev_i32(c["cached"]), dev_i32(c["lengths"]), c["S"], c["L"],
                            q[:, :cols], out[:, :cols], c["D"] ** -0.5 if scale is None else scale,
                            workspace(c) if ws is None else ws, stream=stream)
    assert (out[:, cols:] == 7.0).all()
    return out[:, :cols]


def check(c, got, scale=None, sick=None):
    S, L, D = c["S"], c["L"], c["D"]
    got = got.double().cpu().numpy().reshape(S, L, c["heads"], D)
    q = c["q"].double().numpy().reshape(S, L, c["heads"], D)
    scale = D ** -0.5 if scale is None else scale
    worst = 0.0
    for s in range(S):
        n = int(c["lengths"][s])
        assert (got[s, n:] == 0).all(), f"sequence {s}: empty slots"
        if n == 0:
            continue
        if sick is not None and s in sick:
            assert np.isnan(got[s, :n]).all()
            continue
        N = int(c["cached"][s]) + n
        ref, size, reach = O.cached_attention(q[s, :n], c["k"][s, :N], c["v"][s, :N], int(c["cached"][s]), scale)
        by = c["heads"] // c["kv"]
        coarse = np.abs(q[s, :n]).max(-1) * np.abs(c["k"][s, :N].astype(np.float64)).sum(-1).max(0).repeat(by)[None] * abs(scale)
        e = ((2 * (D + D // 16) + 16) * U * reach + 2.0 ** -28 * coarse)[..., None]
        tol = (2.0 ** -11 + 2 * e + (N + 128) * U) * size + N * 2.0 ** -30 * np.abs(c["v"][s, :N]).max()
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
        off = np.abs(got[s, :n] - ref)
        assert np.isfinite(got[s, :n]).all(), f"sequence {s}: not finite"
        assert (off <= tol).all(), f"sequence {s}: {np.max(off / tol):.3f} of the tolerance"
        worst = max(worst, float(np.max(off / np.maximum(tol, 1e-300))))
    return worst


CASES = [
    dict(L=1, heads=1, kv=1, D=128, page=16, cached=[0]),
    dict(L=1, heads=32, kv=32, D=128, page=16, cached=[299]),
    dict(L=1, heads=4, kv=4, D=64, page=16, cached=[0, 14, 15, 16, 31, 32, 33, 47]),
    dict(L=5, heads=8, kv=2, D=128, page=32, cached=[0, 1, 11, 12, 60], lengths=[5, 1, 0, 5, 3]),
    dict(L=7, heads=12, kv=4, D=64, page=64, cached=[500, 0, 129, 63], lengths=[7, 6, 5, 0]),
    dict(L=3, heads=7, kv=1, D=128, page=128, cached=[1000, 126]),
    dict(L=9, heads=16, kv=2, D=128, page=16, cached=[77, 0, 200]),        # 72 rows of a kv head
    dict(L=40, heads=2, kv=2, D=64, page=32, cached=[0, 33], lengths=[40, 17]),
    dict(L=1, heads=8, kv=8, D=128, page=64, cached=[4999, 0, 3, 2500]),
    dict(L=2, heads=5, kv=5, D=128, page=16, cached=list(range(0, 210, 3)), lengths=[2, 1] * 35),
    dict(L=1, heads=40, kv=1, D=64, page=16, cached=[700]),
    dict(L=4, heads=32, kv=1, D=128, page=32, cached=[90, 1]),             # 128 rows of one kv head
    dict(L=2, heads=4, kv=2, D=64, page=16, cached=[37 * i % 1700 for i in range(40)]),  # equal parts, more than 32 sequences
    dict(L=5, heads=32, kv=8, D=64, page=16, cached=[61 * i % 300 for i in range(16)], lengths=[5, 0, 1, 4] * 4),  # a row of units
    dict(L=1, heads=2, kv=2, D=64, page=16, cached=[7 * i % 90 for i in range(300)], lengths=[1, 0, 1] * 100),
    dict(L=2, heads=2, kv=2, D=64, page=16, cached=[40, 0, 7], lengths=[0, 0, 0]),
    dict(L=1, heads=3, kv=1, D=128, page=16, cached=[20000, 1281]),
    dict(L=300, heads=8, kv=2, D=64, page=64, cached=[0, 40], lengths=[300, 77]),  # prompts
]


@pytest.mark.parametrize("int4", [True, False])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_attention(i, int4):
    c = make(40 + i, int4=int4, **CASES[i])
    got = attend(c, pad=8 * (i % 3))
    check(c, got)
    assert torch.equal(got, attend(c))  # the same bits again, in another stride


@pytest.mark.parametrize("int4", [True, False])
@pytest.mark.parametrize("k_by,v_by,q_by", [(6.0, 1.0, 3.0), (1.0, 1e-30, 1.0), (1.0, 1e30, 1.0), (1e-30, 1.0, 1e30),
                                            (1e15, 1.0, 1e-15), (0.0, 1.0, 1.0), (1.0, 0.0, 1.0), (1.0, 1.0, 0.0)])
def test_ranges_of_values(int4, k_by, v_by, q_by):
    c = make(7, 3, 8, 2, 128, 16, int4, [100, 0, 33], k_by=k_by, v_by=v_by, q_by=q_by)
    check(c, attend(c))


@pytest.mark.parametrize("int4", [True, False])
def test_scales_that_change_along_a_sequence(int4):
    """Values that grow, shrink and jump by powers of ten along the sequence, keys whose scores rise to the end."""
    def change(k, v):
        n = np.arange(v.shape[1])
        v[0] *= (10.0 ** (n / 40 - 8))[:, None, None]
        v[1] *= (10.0 ** (8 - n / 40))[:, None, None]
        v[2] *= (10.0 ** np.where(n % 17 == 3, 6, 0))[:, None, None]
        k[3] *= (0.01 + n / 100)[:, None, None]

    c = make(8, 2, 4, 2, 128, 16, int4, [600] * 4, change=change)
    check(c, attend(c))


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
def test_scale(scale):
    c = make(9, 2, 4, 2, 64, 32, True, [50, 3], q_by=0.3)
    check(c, attend(c, scale=scale), scale=scale)


@pytest.mark.parametrize("int4", [True, False])
@pytest.mark.parametrize("what", [NAN, INF, -INF])
def test_what_a_query_must_not_see_does_not_change_it(int4, what):
    """The last of four new tokens has `what` in its value (and key, for the keys' NaN): earlier queries do not see it."""
    def change(k, v):
        v[:, -1, :, 5] = what
        if what != what:
            k[:, -1, :, 9] = what

    c = make(10, 4, 6, 2, 64, 16, int4, [29, 29], change=change)
    got = attend(c).double().cpu().numpy().reshape(2, 4, 6, 64)
    calm = make(10, 4, 6, 2, 64, 16, int4, [29, 29])
    ref = attend(calm).double().cpu().numpy().reshape(2, 4, 6, 64)
    np.testing.assert_array_equal(got[:, :3], ref[:, :3])
    dims = slice(None) if int4 or what != what else slice(5, 6)  # in 4 bits the whole group is NaN
    assert not np.isfinite(got[:, 3][..., dims]).any()
    if not int4 and what == what:
        assert (got[:, 3, :, 5] == what).all()
        assert np.isfinite(np.delete(got[:, 3], 5, axis=-1)).all()


def test_bad_pages_and_positions():
    c = make(11, 2, 4, 2, 128, 16, True, [40, 40, 40, 0, 40], lengths=[2, 2, 2, 0, 2])
    c["table"][1, 1] = -1
    c["table"][4, 2] = c["cache"].n_pages
    check(c, attend(c), sick={1, 4})
    assert H.device_error(clear=True) == 0x203
    c = make(12, 2, 4, 2, 128, 16, True, [40, 5, 40])
    c["cached"] = np.array([40, -3, 63])  # a table of four pages
    check(c, attend(c), sick={1, 2})
    assert H.device_error(clear=True) == 0x204


def test_shared_pages():
    """Two sequences with one prefix in the same pages."""
    c = make(13, 1, 4, 4, 64, 16, True, [64, 64])
    c["table"][1, :4] = c["table"][0, :4]
    c["k"][1, :64], c["v"][1, :64] = c["k"][0, :64], c["v"][0, :64]
    check(c, attend(c))


def test_streams_graphs_and_a_shared_workspace():
    a, b = (make(14 + i, int4=True, **CASES[i]) for i in (8, 6))
    want = [attend(a), attend(b)]
    s = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for c, st in ((a, s[0]), (b, s[1])):
        with torch.cuda.stream(st):
            got.append(attend(c))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))

    ws = max(workspace(a), workspace(b), key=len)
    graphs = []
    for c in (a, b):
        q, out = c["q"].cuda(), torch.empty(c["S"] * c["L"], c["heads"] * c["D"], dtype=torch.bfloat16, device="cuda")
        args = (dev_i32(c["table"]), dev_i32(c["cached"]), dev_i32(c["lengths"]))
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            H.hydra_paged_attention(c["cache"], *args, c["S"], c["L"], q, out, c["D"] ** -0.5, ws)
        graphs.append((g, out, q, args))
    for _ in range(3):
        for g, *_ in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x[1], y) for x, y in zip(graphs, want))
    # a replay takes the lengths that are there then
    short = dict(a, cached=np.array([17, 0, 3, 1]))
    graphs[0][3][1].copy_(dev_i32(short["cached"]))
    graphs[0][0].replay()
    torch.cuda.synchronize()
    assert torch.equal(graphs[0][1], attend(short))
