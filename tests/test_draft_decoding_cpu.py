"""The paged cache, attention over it and the verification of drafts without a GPU: the oracle against closed forms, and
what the entry points and the binding refuse on the host."""
import ctypes

import numpy as np
import pytest
import torch

import oracle as O
from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H

FAKE = 1 << 20  # aligned and non-null; never dereferenced on these paths
INF = float("inf")


@pytest.fixture(scope="module")
def lib():
    B.build()
    return H.load()


# ---------------------------------------------------------------- oracle


def test_oracle_quantisation_errs_by_half_a_scale():
    x = np.random.default_rng(0).normal(0, 3, (50, 128)).astype(np.float32)
    codes, scale, zero = O.kv_quantise(x)
    assert codes.min() >= 0 and codes.max() <= 15 and (zero == np.rint(zero)).all()
    held = O.kv_held(x, True).reshape(50, 2, 64)
    # a rounded scale may leave 15 steps short of the range by 15 eps, and the zero point's rounding half a step
    assert (np.abs(held - x.reshape(50, 2, 64)) <= scale * (1.0 + 15 * 2.0 ** -8)).all()
    inner = (codes > 0) & (codes < 15)
    assert (np.abs(held - x.reshape(50, 2, 64)) <= scale * (0.5 + 1e-5))[inner].all()
    assert (O.kv_held(np.zeros((1, 64)), True) == 0).all()
    one = O.kv_held(np.full((1, 64), 2.0), True)
    assert np.allclose(one, 2.0, rtol=2.0 ** -8)
    assert np.isnan(O.kv_held(np.array([[1.0] * 63 + [np.inf]]), True)).all()


def test_oracle_rotation_keeps_lengths_and_relative_positions():
    D = 64
    angle = np.arange(50)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
    table = np.stack([np.cos(angle), np.sin(angle)], -1)
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(2, 1, D))
    dot = [float(np.sum(O.rope_by_table(q, table[a]).astype(np.float64) * O.rope_by_table(k, table[b]))) for a, b in ((7, 3), (47, 43))]
    assert abs(dot[0] - dot[1]) <= 1e-4


def test_oracle_attention_of_equal_scores_is_a_mean():
    v = np.random.default_rng(2).normal(size=(5, 2, 64))
    out, size, reach = O.cached_attention(np.zeros((2, 4, 64)), np.ones((5, 2, 64)), v, 3, 0.1)
    np.testing.assert_allclose(out[0, 0], v[:4, 0].mean(0))
    np.testing.assert_allclose(out[1, 3], v[:5, 1].mean(0))
    assert (size >= np.abs(out) - 1e-12).all() and (reach == 0).all()


def test_oracle_verification_draws_from_the_target():
    """The exact distribution of the first token, over a grid of u and every draft: sum over drafts of q min(1, p/q)
    plus what refusals draw is p."""
    p, q = np.array([0.6, 0.3, 0.1]), np.array([0.2, 0.3, 0.5])
    z, w = np.log(p)[None].repeat(2, 0), np.log(q)[None]
    got = np.zeros(3)
    for x in range(3):
        a = O.verify_drafts(z, w, [[x]], None, [[0.0]], np.zeros((1, 3)), 1, 1)["accept"][0, 0]
        assert abs(a - min(1.0, p[x] / q[x])) < 1e-12
        rest = np.maximum(p - q, 0)
        got += q[x] * (a * np.eye(3)[x] + (1 - a) * rest / rest.sum())
        if a < 1:
            r = O.verify_drafts(z, w, [[x]], None, [[a]], np.zeros((1, 3)), 1, 1)
            assert r["accepted"][0] == 0 and r["tokens"][0].tolist() == [int(np.argmax(rest)), -1]
    np.testing.assert_allclose(got, p, atol=1e-12)


def test_oracle_verification_greedy_certain_and_empty():
    z = np.array([[0.0, 2.0, 2.0], [5.0, 0.0, 0.0], [0.0, 0.0, 1.0]])
    r = O.verify_drafts(z, None, [[1, 2]], None, None, None, 1, 2)
    assert r["tokens"].tolist() == [[1, 0, -1]] and r["accepted"][0] == 1 and r["accept"].tolist() == [[1.0, 0.0]]
    r = O.verify_drafts(z, None, [[1, 0]], None, [[0.99, 0.0]], np.zeros((1, 3)), 1, 2)
    assert r["tokens"].tolist() == [[2, -1, -1]]  # refused: row 0 without token 1
    r = O.verify_drafts(np.full((2, 3), -INF), np.zeros((1, 3)), [[1]], None, [[0.0]], np.zeros((1, 3)), 1, 1)
    assert r["tokens"].tolist() == [[0, -1]] and r["logp"][0, 0] == -INF


# ---------------------------------------------------------------- refusals


def test_page_bytes(lib):
    assert H.kv_page_bytes(H.HYDRA_KV_INT4, 16, 1, 128) == 2304 and H.kv_page_bytes(H.HYDRA_KV_BF16, 16, 1, 128) == 8192
    assert H.kv_page_bytes(H.HYDRA_KV_INT4, 128, 8, 64) == 128 * 8 * 72
    for bad in ((2, 16, 1, 128), (0, 8, 1, 128), (0, 48, 1, 128), (1, 256, 1, 128), (1, 16, 0, 128), (1, 16, 4097, 128), (1, 16, 1, 96)):
        assert H.kv_page_bytes(*bad) == 0


def _cache(**kw):
    a = dict(data=FAKE, n_pages=4, page=16, n_kv_heads=2, head_dim=128, kind=1)
    a.update(kw)
    return H.KvCacheC(*(a[k] for k in ("data", "n_pages", "page", "n_kv_heads", "head_dim", "kind")))


def _common(kw):
    cache = kw.pop("cache", None)
    a = dict(table=FAKE, ld_table=3, max_pages=3, cached=FAKE, lengths=FAKE, S=2, L=3)
    a.update({k: kw.pop(k) for k in list(kw) if k in a})
    return (cache if cache is not None else ctypes.byref(_cache()), a["table"], a["ld_table"], a["max_pages"], a["cached"],
            a["lengths"], a["S"], a["L"])


def _append(lib, **kw):
    head = _common(kw) if kw.pop("null_cache", None) is None else (None, *_common(kw)[1:])
    a = dict(q=FAKE, heads=4, ld_q=512, k=FAKE, v=FAKE, ld_kv=256, rope=FAKE, P=100, out=2 * FAKE, ld_o=512)
    a.update(kw)
    return lib.hydra_kv_append(*head, a["q"], a["heads"], a["ld_q"], a["k"], a["v"], a["ld_kv"], a["rope"], a["P"], a["out"],
                               a["ld_o"], None)


def _read(lib, **kw):
    head = _common(kw)
    a = dict(k=FAKE, v=FAKE, dt=0, ld=256)
    a.update(kw)
    return lib.hydra_kv_read(*head, a["k"], a["v"], a["dt"], a["ld"], None)


def _attend(lib, **kw):
    head = _common(kw)
    a = dict(q=FAKE, heads=4, ld_q=512, scale=0.1, out=2 * FAKE, ld_o=512, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return lib.hydra_paged_attention(*head, a["q"], a["heads"], a["ld_q"], a["scale"], a["out"], a["ld_o"], a["ws"], a["wsb"], None)


def test_what_all_calls_with_a_cache_refuse(lib):
    for f in (_append, _read, _attend):
        for bad in (dict(page=8), dict(head_dim=32), dict(kind=2)):
            assert f(lib, cache=ctypes.byref(_cache(**bad))) == 4
        for bad in (dict(n_pages=0), dict(n_pages=1 << 31), dict(n_kv_heads=0), dict(n_kv_heads=4097)):
            assert f(lib, cache=ctypes.byref(_cache(**bad))) in (2, 4)
        assert f(lib, cache=ctypes.byref(_cache(data=None))) == 1 and f(lib, cache=ctypes.byref(_cache(data=FAKE + 8))) == 3
        assert f(lib, S=-1) == 2 and f(lib, L=-1) == 2 and f(lib, S=1 << 16, L=1 << 15) == 2
        assert f(lib, max_pages=0) == 2 and f(lib, max_pages=4) == 2 and f(lib, max_pages=1 << 27, ld_table=1 << 27) == 2
        assert f(lib, table=None) == 1
        assert f(lib, S=0, table=None) == 0 and f(lib, L=0, table=None) == 0  # no rows


def test_append_argument_errors(lib):
    assert _append(lib, null_cache=True) == 1
    assert _append(lib, heads=-1) == 2 and _append(lib, heads=4097, ld_q=1 << 20) == 2
    assert _append(lib, P=0) == 2 and _append(lib, rope=FAKE + 8) == 3
    assert _append(lib, ld_kv=248) == 2 and _append(lib, ld_kv=260) == 3 and _append(lib, k=FAKE + 8) == 3 and _append(lib, v=FAKE + 2) == 3
    assert _append(lib, ld_q=504) == 2 and _append(lib, ld_q=516) == 3 and _append(lib, q=FAKE + 8) == 3
    assert _append(lib, ld_o=504) == 2 and _append(lib, ld_o=516) == 3 and _append(lib, out=FAKE + 8) == 3
    assert _append(lib, out=FAKE, ld_o=520) == 4  # in place with another stride
    for x in ("q", "k", "v", "out"):
        assert _append(lib, **{x: None}) == 1
    assert _append(lib, S=0, k=None) == 0 and _append(lib, L=0) == 0


def test_read_argument_errors(lib):
    assert _read(lib, dt=2) == 4 and _read(lib, ld=248) == 2 and _read(lib, ld=260) == 3 and _read(lib, k=FAKE + 8) == 3
    assert _read(lib, k=None, v=None) == 1
    assert _read(lib, S=0, k=None, v=None) == 0


def test_attention_argument_errors(lib):
    assert _attend(lib, heads=3, ld_q=384) == 2 and _attend(lib, heads=0) == 2  # not a multiple of two
    for bad in (INF, float("nan")):
        assert _attend(lib, scale=bad) == 4
    assert _attend(lib, ld_q=504) == 2 and _attend(lib, ld_q=516) == 3 and _attend(lib, out=FAKE + 8) == 3
    assert _attend(lib, q=None) == 1 and _attend(lib, out=None) == 1
    need = H.paged_attention_workspace_size(2, 3, 4, 2, 128)
    assert need >= 16 and H.paged_attention_workspace_size(2, 3, 3, 2, 128) == 0
    assert _attend(lib, ws=None) == 7 and _attend(lib, ws=FAKE + 8) == 7 and _attend(lib, wsb=need - 1) == 7
    assert _attend(lib, S=0, q=None) == 0


def _verify(lib, **kw):
    a = dict(z=FAKE, w=FAKE, dt=1, S=2, D=3, V=100, ld=100, ld_w=100, ids=FAKE, n=None, u=FAKE, g=FAKE, ld_g=100, tokens=FAKE,
             accepted=FAKE, logp=None, accept=None)
    a.update(kw)
    return lib.hydra_verify_drafts(*a.values(), None)


def test_verify_argument_errors(lib):
    assert _verify(lib, dt=2) == 4 and _verify(lib, D=33) == 4 and _verify(lib, D=-1) == 4
    assert _verify(lib, S=-1) == 2 and _verify(lib, S=(1 << 24) + 1) == 2 and _verify(lib, V=0) == 2
    assert _verify(lib, V=(1 << 30) + 1, ld=1 << 31, ld_w=1 << 31, ld_g=1 << 31) == 2
    assert _verify(lib, ld=99) == 2 and _verify(lib, ld_w=99) == 2 and _verify(lib, ld_g=99) == 2
    for x in ("z", "ids", "tokens", "accepted", "u", "g"):
        assert _verify(lib, **{x: None}) == 1, x
    assert _verify(lib, u=None, g=None) == 4  # greedy, with a draft distribution
    assert _verify(lib, z=FAKE + 2) == 3 and _verify(lib, w=FAKE + 1, dt=0) == 3
    assert _verify(lib, S=0, z=None) == 0


def test_binding_refuses_tensors_off_the_gpu_and_of_other_shapes(lib):
    with pytest.raises(ValueError):
        H.KvCache(H.HYDRA_KV_INT4, 3, 24, 2, 128, data=torch.zeros(1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        H.KvCache(H.HYDRA_KV_INT4, 3, 16, 2, 128, data=torch.zeros(3, 16 * 2 * 144, dtype=torch.uint8))
    with pytest.raises(ValueError):
        H._heads(torch.zeros(4, 256), 4, 128, torch.bfloat16, 0, "q")
    with pytest.raises(ValueError):
        H.hydra_verify_drafts(torch.zeros(4, 10), None, None, None, None, None, 1, 3, None, None)


def test_rows_that_are_one_row_repeated_are_refused(lib):
    """Keys and values (or outputs) expanded from a single row: their stride of 0 goes to the library as it is, which refuses it.
    As the stride of dense rows, rows past the first would lie outside the tensor."""
    class Two:
        n_kv_heads, head_dim = 2, 128
    bf16 = torch.bfloat16
    one, dense = torch.zeros(1, 256, dtype=bf16), torch.zeros(6, 256, dtype=bf16)
    for k, v in ((one.expand(6, 256),) * 2, (None, one.expand(6, 256)), (one.expand(6, 256), None)):
        *_, ld = H._kv_pair(k, v, 6, Two, bf16, -1, ("k", "v"))
        assert ld == 0
    assert _append(lib, ld_kv=0) == 2 and _read(lib, ld=0) == 2
    with pytest.raises(ValueError):
        H._kv_pair(one.expand(6, 256), dense, 6, Two, bf16, -1, ("k", "v"))
    assert H._kv_pair(dense, dense, 6, Two, bf16, -1, ("k", "v"))[2] == 256
    assert H._kv_pair(one, None, 1, Two, bf16, -1, ("k", "v"))[2] == 256
    assert H._kv_pair(dense[:0], dense[:0], 0, Two, bf16, -1, ("k", "v"))[2] == 256


def test_cache_struct_layout_is_the_headers():
    assert ctypes.sizeof(H.KvCacheC) == 48
    assert [getattr(H.KvCacheC, n).offset for n in ("data", "n_pages", "page", "n_kv_heads", "head_dim", "kind")] == [0, 8, 16, 24, 32, 40]
