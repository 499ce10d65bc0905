"""Keys and values put into a paged cache and read back, against the oracle's roundings bit for bit: rotation, both
kinds of cache, pages in any order, ragged batches, what must stay as it was, and what the kernels refuse.

Every operation of the definition is a single rounding in fp32 (products, sums, the quotient, rint), so the oracle's
numpy and the kernel give equal bits; no tolerance."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.helpers import dev_i32

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


def rope_table(P, D):
    angle = np.arange(P)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
    return np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)


def pages_for(rng, totals, page, extra=2):
    """(table [S, width] with -1 where nothing is needed, number of pages): pages in random order."""
    need = [-(-int(n) // page) for n in totals]
    order = rng.permutation(sum(need) + extra)
    table = np.full((len(need), max(need) + 1), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, len(order)


def make(seed, S, L, heads, kv, D, page, int4, cached, lengths=None, values=None):
    rng = np.random.default_rng(seed)
    width = (heads + 2 * kv) * D
    x = rng.normal(0, 1, (S * L, width)) * 10 ** rng.uniform(-2, 1, (1, width))
    if values is not None:
        x = values(rng, x)
    x = torch.from_numpy(x).bfloat16()
    cached = np.asarray(cached)
    lengths = np.full(S, L) if lengths is None else np.asarray(lengths)
    table, n_pages = pages_for(rng, cached + lengths, page)
    kind = H.HYDRA_KV_INT4 if int4 else H.HYDRA_KV_BF16
    cache = H.KvCache(kind, n_pages, page, kv, D)
    cache.data.fill_(0xA5)
    return {"S": S, "L": L, "heads": heads, "kv": kv, "D": D, "cached": cached, "lengths": lengths, "table": table,
            "x": x, "cache": cache, "rope": rope_table(int((cached + lengths).max()) + 1, D), "int4": int4}


def parts(c, x):
    D, h, kv = c["D"], c["heads"], c["kv"]
    return x[:, :h * D], x[:, h * D:(h + kv) * D], x[:, (h + kv) * D:]


def append(c, rope=True, in_place=False, stream=None):
    x = c["x"].cuda()
    q, k, v = parts(c, x)
    q_out = q if in_place else torch.full((x.shape[0], q.shape[1] + 8), NAN, dtype=torch.bfloat16, device="cuda")[:, :q.shape[1]]
    H.hydra_kv_append(c["cache"], dev_i32(c["table"]), dev_i32(c["cached"]), dev_i32(c["lengths"]), c["S"], c["L"], q, k, v,
                      torch.from_numpy(c["rope"]).cuda() if rope else None, q_out, stream=stream)
    return q_out, x


def read(c, dtype=torch.float32):
    k, v = torch.full((2, c["S"] * c["L"], c["kv"] * c["D"]), NAN, dtype=dtype, device="cuda")
    H.hydra_kv_read(c["cache"], dev_i32(c["table"]), dev_i32(c["cached"]), dev_i32(c["lengths"]), c["S"], c["L"], k, v)
    return k, v


def want(c, rope=True):
    q, k, v = (y.float().numpy().reshape(c["S"], c["L"], -1, c["D"]) for y in parts(c, c["x"]))
    pos = np.minimum(c["cached"][:, None] + np.arange(c["L"])[None], len(c["rope"]) - 1)
    if rope:
        q, k = (O.rope_by_table(y, c["rope"][pos]) for y in (q, k))
    live = (np.arange(c["L"])[None] < c["lengths"][:, None])[..., None, None]
    flat = lambda y: np.where(live, y, 0).reshape(c["S"] * c["L"], -1).astype(np.float32)  # noqa: E731
    return flat(q), flat(O.kv_held(k, c["int4"])), flat(O.kv_held(v, c["int4"]))


def same(got, ref):
    np.testing.assert_array_equal(got.detach().float().cpu().numpy(), ref)


CASES = [
    dict(S=1, L=1, heads=1, kv=1, D=128, page=16, cached=[0]),
    dict(S=1, L=1, heads=32, kv=32, D=128, page=16, cached=[300]),
    dict(S=5, L=3, heads=6, kv=2, D=64, page=32, cached=[0, 31, 32, 95, 7], lengths=[3, 2, 0, 1, 3]),
    dict(S=3, L=70, heads=7, kv=7, D=128, page=64, cached=[0, 63, 129], lengths=[70, 1, 33]),
    dict(S=2, L=150, heads=40, kv=3, D=64, page=128, cached=[5, 250], lengths=[150, 149]),
    dict(S=9, L=2, heads=5, kv=1, D=128, page=16, cached=list(range(11, 20)), lengths=[2, 1, 0] * 3),
    # single tokens, a lane group a head: numbers of heads that fill no warp
    dict(S=23, L=1, heads=13, kv=6, D=128, page=16, cached=list(range(23)), lengths=[1, 1, 0, 1, 1] * 4 + [1] * 3),
    dict(S=4, L=1, heads=8, kv=9, D=64, page=32, cached=[31, 32, 7, 0]),
    # a warp has several heads
    dict(S=20, L=100, heads=50, kv=11, D=64, page=16, cached=list(range(0, 100, 5)), lengths=list(range(100, 0, -5))),
    dict(S=4, L=129, heads=33, kv=130, D=128, page=64, cached=[0, 1, 77, 64], lengths=[129, 3, 0, 8]),
]


@pytest.mark.parametrize("int4", [False, True])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_append_and_read(i, int4):
    c = make(10 + i, int4=int4, **CASES[i])
    q_out, x = append(c)
    k, v = read(c)
    q_ref, k_ref, v_ref = want(c)
    same(q_out, O.round_bf16(q_ref.astype(np.float64)).astype(np.float32))
    same(k, k_ref)
    same(v, v_ref)
    kb, vb = read(c, torch.bfloat16)
    same(kb, O.round_bf16(k_ref.astype(np.float64)).astype(np.float32))
    same(vb, O.round_bf16(v_ref.astype(np.float64)).astype(np.float32))
    assert torch.equal(x.cpu(), c["x"])  # inputs untouched


@pytest.mark.parametrize("int4", [False, True])
def test_in_place_without_rotation_and_without_queries(int4):
    c = make(31, int4=int4, **CASES[2])
    q_out, x = append(c, in_place=True)
    q_ref, k_ref, _ = want(c)
    same(q_out, O.round_bf16(q_ref.astype(np.float64)).astype(np.float32))
    assert torch.equal(x[:, c["heads"] * c["D"]:].cpu(), c["x"][:, c["heads"] * c["D"]:])
    append(c, rope=False)
    same(read(c)[0], want(c, rope=False)[1])
    c["cache"].data.fill_(0)
    _, k, v = parts(c, x)
    H.hydra_kv_append(c["cache"], dev_i32(c["table"]), dev_i32(c["cached"]), dev_i32(c["lengths"]), c["S"], c["L"], None, k, v,
                      torch.from_numpy(c["rope"]).cuda())
    same(read(c)[0], k_ref)


def test_rotation_is_hydra_ropes():
    """With hydra_rope_table's table the queries are hydra_rope's bit for bit, and a bf16 cache's keys too."""
    P, H_, D = 37, 3, 128
    c = make(5, 1, P, H_, H_, D, 16, False, [0])
    table = torch.empty(P, D // 2, 2, device="cuda")
    x = c["x"].cuda()
    ref = x.clone()
    H.hydra_rope(ref, H_ * D, D, P, 10000.0)
    H._check("t", H.load().hydra_rope_table(P, D, 10000.0, table.data_ptr(), H._stream(None)))
    q, k, v = parts(c, x)
    H.hydra_kv_append(c["cache"], dev_i32(c["table"]), None, None, 1, P, q, k, v, table, q)
    assert torch.equal(q, ref[:, :H_ * D])
    assert torch.equal(read(c, torch.bfloat16)[0], ref[:, H_ * D:2 * H_ * D])


def test_values_where_a_scale_goes_wrong():
    """Groups of zeros, of one value, of one sign, near the type's ends, with an infinity or NaN."""
    def odd(rng, x):
        x = x.reshape(-1, 64)
        x[0], x[1], x[2], x[3] = 0.0, 3.0, -np.abs(x[3]), np.abs(x[4])
        x[4] *= 3e38 / np.abs(x[4]).max()
        x[5] *= 1e-38
        x[6, :], x[6, 9] = 0.0, 1e-40
        x[7, 3], x[8, 5], x[9, 63] = np.nan, np.inf, -np.inf
        x[10, :], x[10, 1], x[10, 0] = 0.0, -3.38e38, 3.38e38
        return x.reshape(1, -1)

    c = make(8, 1, 1, 0, 11, 128, 16, True, [3], values=odd)
    x = c["x"].cuda()
    _, k, v = parts(c, x)
    H.hydra_kv_append(c["cache"], dev_i32(c["table"]), dev_i32(c["cached"]), None, 1, 1, None, k, v)
    _, k_ref, v_ref = want(c, rope=False)
    assert np.isnan(k_ref).sum() == 3 * 64
    same(read(c)[0], k_ref)
    same(read(c)[1], v_ref)


def test_quotients_half_way_between_codes():
    """Channels at whole and half codes of a scale of 1 (and 2^-20, 2^20): ties go to the even code, as rint has it."""
    def halves(rng, like):
        x = rng.integers(0, 31, like.size).reshape(-1, 64) / 2.0 - rng.integers(0, 16, (like.size // 64, 1))
        lo = rng.integers(0, 16, (len(x), 1)) * -1.0
        x = np.clip(x, lo, lo + 15)
        x[:, :1], x[:, 1:2] = lo, lo + 15
        return (x * rng.choice([1.0, 2.0 ** -20, 2.0 ** 20], (len(x), 1))).reshape(like.shape)

    c = make(9, 1, 18, 0, 40, 128, 16, True, [3], values=halves)
    _, k, v = parts(c, c["x"].cuda())
    H.hydra_kv_append(c["cache"], dev_i32(c["table"]), dev_i32(c["cached"]), None, 1, 18, None, k, v)
    _, k_ref, v_ref = want(c, rope=False)
    same(read(c)[0], k_ref)
    same(read(c)[1], v_ref)


@pytest.mark.parametrize("int4", [False, True])
def test_nothing_else_is_written(int4):
    c = make(77, int4=int4, **CASES[4])
    before = c["cache"].data.clone()
    append(c)
    same(read(c)[0], want(c)[1])
    # where other tokens and pages lie: read the neighbours before and after
    other = dict(c, cached=np.array([0, 0]), lengths=np.array([5, 250]), L=250)
    after = read(other)
    data, c["cache"].data[:] = c["cache"].data.clone(), before
    first = read(other)
    for a, b in zip(after, first):
        np.testing.assert_array_equal(a.cpu().numpy(), b.cpu().numpy())
    used = set(c["table"][c["table"] >= 0].tolist())
    for page in set(range(c["cache"].n_pages)) - used:
        assert torch.equal(data[page], before[page])


def test_appends_in_steps_are_one_append():
    for int4 in (False, True):
        a = make(3, 2, 40, 2, 2, 128, 16, int4, [9, 0])
        append(a)
        whole = read(a)
        bytes_whole = a["cache"].data.clone()
        a["cache"].data.fill_(0xA5)
        x = a["x"].cuda().view(2, 40, -1)
        for at in range(0, 40, 8):
            part = dict(a, L=8, x=x[:, at:at + 8].reshape(16, -1).cpu(), cached=a["cached"] + at, lengths=np.full(2, 8))
            append(part)
        assert torch.equal(a["cache"].data, bytes_whole)
        assert all(torch.equal(p, q) for p, q in zip(whole, read(a)))


def test_bad_pages_positions_and_lengths():
    c = make(4, 3, 4, 2, 2, 64, 16, True, [0, 15, 2], lengths=[4, 4, 4])
    c["table"][1, 1] = c["cache"].n_pages  # tokens 1..3 of the second sequence
    before = c["cache"].data.clone()
    q_out, _ = append(c)
    assert H.device_error(clear=True) == 0x203
    k, v = read(c)
    assert H.device_error(clear=True) == 0x203
    bad = np.zeros((3, 4), dtype=bool)
    bad[1, 1:] = True
    q_ref, k_ref, v_ref = want(c)
    k_ref[bad.reshape(-1)] = v_ref[bad.reshape(-1)] = NAN
    same(k, k_ref)
    same(v, v_ref)
    same(q_out, O.round_bf16(q_ref.astype(np.float64)).astype(np.float32))

    for cached, lengths, rope_rows in (([-1, 15, 2], [4, 1, 4], None), ([0, 60, 2], [4, 4, 4], None), ([0, 0, 0], [4, 4, 4], 2)):
        c["cache"].data[:] = before
        d = dict(c, cached=np.array(cached), lengths=np.array(lengths))
        d["table"] = np.arange(3 * 3, dtype=np.int32).reshape(3, 3) % c["cache"].n_pages
        d["rope"] = rope_table(rope_rows or 64, 64)
        q_out, _ = append(d)
        assert H.device_error(clear=True) == 0x204
        total = d["cached"] + d["lengths"]
        sick = (d["cached"] < 0) | (total > min(48, len(d["rope"])))
        assert np.array_equal(torch.isnan(q_out).all(1).view(3, 4)[:, 0].cpu().numpy(), sick)
        if sick.all():
            assert torch.equal(c["cache"].data, before)

    d = dict(c, cached=np.array([0, 0, 0]), lengths=np.array([9, -2, 4]), table=np.array([[0], [1], [2]], dtype=np.int32))
    append(d)
    assert H.device_error(clear=True) == 0x202
    read(d)
    assert H.device_error(clear=True) == 0x202


def test_two_streams_and_a_captured_call():
    cs = [make(20 + i, int4=bool(i), **CASES[3]) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for c, s in zip(cs, streams):
        with torch.cuda.stream(s):
            c["got"] = (append(c)[0], *read(c))
    torch.cuda.synchronize()
    for c in cs:
        _, k_ref, v_ref = want(c)
        same(c["got"][1], k_ref)
        same(c["got"][2], v_ref)

    c = cs[1]
    x, table, cached, lengths = c["x"].cuda(), dev_i32(c["table"]), dev_i32(c["cached"]), dev_i32(c["lengths"])
    rope, (q, k, v) = torch.from_numpy(c["rope"]).cuda(), parts(c, x)
    q_out, (ko, vo) = torch.empty_like(q.contiguous()), torch.empty(2, *k.shape, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H.hydra_kv_append(c["cache"], table, cached, lengths, c["S"], c["L"], q, k, v, rope, q_out)
        H.hydra_kv_read(c["cache"], table, cached, lengths, c["S"], c["L"], ko, vo)
    other = make(99, int4=True, **CASES[3])
    x.copy_(other["x"])
    c["cache"].data.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    c["x"] = other["x"]
    q_ref, k_ref, v_ref = want(c)
    same(ko, k_ref)
    same(vo, v_ref)
    same(q_out, O.round_bf16(q_ref.astype(np.float64)).astype(np.float32))


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GB, the token in its last page."""
    D, kv, page = 128, 8, 128
    size = H.kv_page_bytes(H.HYDRA_KV_BF16, page, kv, D)
    n_pages = (1 << 32) // size + 3
    c = make(1, 1, 3, 1, kv, D, page, False, [126])
    c["cache"] = H.KvCache(H.HYDRA_KV_BF16, n_pages, page, kv, D)
    c["table"] = np.array([[n_pages - 2, n_pages - 1]], dtype=np.int32)
    append(c)
    k, v = read(c)
    _, k_ref, v_ref = want(c)
    same(k, k_ref)
    same(v, v_ref)
