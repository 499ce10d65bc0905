"""Token statistics, their gradient and gradient clipping without a GPU: the oracle's formulas
against differences and closed forms, and what the entry points refuse on the host."""
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


def test_oracle_of_a_uniform_row_and_of_a_certain_one():
    z = np.array([[2.0] * 8, [0.0] * 7 + [800.0], [-INF, 3.0, -INF, 3.0, -INF, -INF, -INF, -INF], [-INF] * 8])
    r = O.token_stats(z, [3, 7, 1, 0], None, 4, 1, k=3)
    np.testing.assert_allclose(r["logp"], [-np.log(8), 0.0, -np.log(2), -INF], atol=1e-15)
    np.testing.assert_allclose(r["entropy"], [np.log(8), 0.0, np.log(2), 0.0], atol=1e-15)
    assert r["norm"][3].tolist() == [-INF, 0.0] and r["norm"][1].tolist() == [800.0, 0.0]
    assert r["top_ids"].tolist() == [[0, 1, 2], [7, 0, 1], [1, 3, 0], [0, 1, 2]]
    np.testing.assert_allclose(r["top_logp"][2], [-np.log(2), -np.log(2), -INF])
    assert not O.token_stats_grad(z, [3, 7, 1, 0], None, 4, 1, np.ones(4), np.ones(4))[3].any()


def test_oracle_counts_the_lowest_value_as_a_number():
    low = float(np.finfo(np.float32).min)
    r = O.token_stats([[low] * 4, [low, 0.0, low, 0.0]], [1, 0], None, 1, 2, k=1)
    np.testing.assert_allclose(r["entropy"], [np.log(4), np.log(2)])
    assert r["logp"][0] == -np.log(4) and r["logp"][1] < -3e38


@pytest.mark.parametrize("masked", [False, True])
def test_oracle_gradient_against_differences(masked):
    """Central differences in 64 bits: (f(z + h) - f(z - h)) / 2h with h 1e-5 is off by
    h^2 / 6 times a third derivative of order 1 and by 1e-16 / h: under 1e-10."""
    rng = np.random.default_rng(5)
    S, L, V = 2, 3, 11
    z = rng.normal(0, 2, (S * L, V))
    if masked:
        z[:, ::3] = -INF
        z[4] = -INF
    ids, lengths = rng.integers(0, 3, S * L) * 3 + 1, np.array([3, 2])
    gl, gh = rng.normal(size=S * L), rng.normal(size=S * L)

    def loss(y):
        r = O.token_stats(y, ids, lengths, S, L)
        keep = np.isfinite(r["logp"])
        return (gl * np.where(keep, r["logp"], 0.0)).sum() + (gh * r["entropy"]).sum()

    d = O.token_stats_grad(z, ids, lengths, S, L, gl, gh)
    for i in range(S * L):
        for v in range(V):
            if np.isfinite(z[i, v]):
                up, down = z.copy(), z.copy()
                up[i, v] += 1e-5
                down[i, v] -= 1e-5
                assert abs((loss(up) - loss(down)) / 2e-5 - d[i, v]) <= 1e-9
    assert np.abs(d.sum(1)).max() <= 1e-14  # a shift of all logits changes nothing


def test_oracle_clip():
    g = [np.array([3.0, 0.0]), np.zeros(0), np.array([[4.0]])]
    norm, coef, out = O.clip_grad_norm(g, 1.0)
    assert norm == 5.0 and abs(coef - 0.2) < 1e-7 and abs(out[0][0] - 0.6) < 1e-6
    assert O.clip_grad_norm(g, 50.0)[1] == 1.0
    assert O.clip_grad_norm([np.array([INF])], 1.0)[:2] == (INF, 1.0)


# ---------------------------------------------------------------- refusals


def _stats(lib, **kw):
    a = dict(z=FAKE, dt=1, S=2, L=3, V=100, ld=100, ids=FAKE, lengths=None, k=0, logp=FAKE, ent=FAKE, norm=FAKE,
             top_ids=None, top_logp=None)
    a.update(kw)
    return lib.hydra_token_logprobs_entropy(a["z"], a["dt"], a["S"], a["L"], a["V"], a["ld"], a["ids"], a["lengths"],
                                            a["k"], a["logp"], a["ent"], a["norm"], a["top_ids"], a["top_logp"], None)


def test_token_stats_vocabulary_with_alternatives_is_bounded(lib):
    top = dict(top_ids=FAKE, top_logp=FAKE, k=5)
    assert _stats(lib, V=(1 << 20) + 1, ld=1 << 21, **top) == 2
    assert _stats(lib, V=1 << 20, ld=1 << 20, **top) not in (2, 4)
    assert _stats(lib, V=(1 << 20) + 1, ld=1 << 21) not in (2, 4)


def test_token_stats_argument_errors(lib):
    assert _stats(lib, dt=2) == 4
    assert _stats(lib, S=-1) == 2 and _stats(lib, L=-1) == 2 and _stats(lib, S=1 << 16, L=1 << 15) == 2
    assert _stats(lib, V=0, ld=0) == 2 and _stats(lib, ld=99) == 2
    assert _stats(lib, V=(1 << 30) + 1, ld=1 << 31) == 2
    top = dict(top_ids=FAKE, top_logp=FAKE)
    assert _stats(lib, k=33, **top) == 4 and _stats(lib, k=-1, **top) == 4 and _stats(lib, V=4, ld=4, k=5, **top) == 4
    assert _stats(lib, k=5) == 1 and _stats(lib, k=5, top_ids=FAKE) == 1
    assert _stats(lib, z=None) == 1 and _stats(lib, ids=None) == 1
    assert _stats(lib, logp=None, ent=None, norm=None) == 1
    assert _stats(lib, z=FAKE + 2) == 3 and _stats(lib, z=FAKE + 1, dt=0) == 3
    assert _stats(lib, S=0) == 0 and _stats(lib, L=0, z=None) == 0  # no rows


def _grad(lib, **kw):
    a = dict(z=FAKE, dt=1, S=2, L=3, V=100, ld=100, ids=FAKE, lengths=None, norm=FAKE, ent=FAKE, gl=FAKE, gh=FAKE,
             d=2 * FAKE, gdt=1, ld_d=100)
    a.update(kw)
    return lib.hydra_token_logprobs_entropy_grad(a["z"], a["dt"], a["S"], a["L"], a["V"], a["ld"], a["ids"], a["lengths"],
                                                 a["norm"], a["ent"], a["gl"], a["gh"], a["d"], a["gdt"], a["ld_d"], None)


def test_token_stats_grad_argument_errors(lib):
    assert _grad(lib, dt=2) == 4 and _grad(lib, gdt=5) == 4
    assert _grad(lib, S=-1) == 2 and _grad(lib, ld=99) == 2 and _grad(lib, ld_d=99) == 2
    assert _grad(lib, V=0, ld=0, ld_d=0) == 2
    assert _grad(lib, S=1 << 15, L=1 << 14, V=32000, ld=32000, ld_d=32000) == 2  # more than 2^32 tiles
    assert _grad(lib, z=None) == 1 and _grad(lib, norm=None) == 1 and _grad(lib, d=None) == 1
    assert _grad(lib, gl=None, gh=None) == 1
    assert _grad(lib, ids=None) == 1 and _grad(lib, ent=None) == 1
    assert _grad(lib, z=FAKE + 2) == 3 and _grad(lib, d=FAKE + 2) == 3 and _grad(lib, d=FAKE + 1, gdt=0) == 3
    assert _grad(lib, d=FAKE, gdt=0) == 4 and _grad(lib, d=FAKE, ld_d=104) == 4  # in place of another shape
    assert _grad(lib, L=0, z=None) == 0


def _clip(lib, tensors, fn="hydra_clip_grad_norm", **kw):
    a = dict(n=len(tensors), max_norm=1.0, out=FAKE, ws=FAKE, wsb=H.grad_norm_workspace_size())
    a.update(kw)
    c = (H.GradTensorC * max(1, len(tensors)))(*[H.GradTensorC(*t) for t in tensors])
    return getattr(lib, fn)(a.get("list", c), a["n"], a["max_norm"], a["out"], a["ws"], a["wsb"], None)


def test_grad_norm_argument_errors(lib):
    ok = (FAKE, FAKE, 100, 1)
    for fn in ("hydra_clip_grad_norm", "hydra_grad_norm"):
        assert _clip(lib, [ok], fn, n=-1) == 2 and _clip(lib, [ok], fn, n=1 << 31) == 2
        for bad in (0.0, -1.0, float("nan")):
            assert _clip(lib, [ok], fn, max_norm=bad) == 4
        assert _clip(lib, [ok], fn, out=None) == 1 and _clip(lib, [ok], fn, list=None) == 1
        assert _clip(lib, [ok], fn, out=FAKE + 2) == 3
        assert _clip(lib, [ok], fn, ws=None) == 7 and _clip(lib, [ok], fn, ws=FAKE + 8) == 7
        assert _clip(lib, [ok], fn, wsb=H.grad_norm_workspace_size() - 1) == 7
        assert _clip(lib, [(FAKE, FAKE, -1, 1)], fn) == 2 and _clip(lib, [(FAKE, FAKE, 1 << 40, 1)], fn) == 2
        assert _clip(lib, [(FAKE, FAKE, 4, 2)], fn) == 4
        assert _clip(lib, [(None, FAKE, 4, 1)], fn) == 1
        assert _clip(lib, [(FAKE + 2, FAKE, 4, 1)], fn) == 3 and _clip(lib, [(FAKE + 1, FAKE, 4, 0)], fn) == 3
    assert _clip(lib, [(FAKE, None, 4, 1)]) == 1 and _clip(lib, [(FAKE, FAKE + 2, 4, 1)]) == 3


def test_clip_refuses_ranges_that_overlap(lib):
    a, b, c = FAKE, 2 * FAKE, 3 * FAKE
    assert _clip(lib, [(a, a, 8, 1), (a, a, 8, 1)]) == 4             # the same tensor twice
    assert _clip(lib, [(a, a, 8, 1), (a + 28, a + 28, 8, 1)]) == 4   # the last element is the other's first
    assert _clip(lib, [(a + 28, a + 28, 8, 1), (a, a, 8, 1)]) == 4   # in either order
    assert _clip(lib, [(a, a + 4, 8, 1)]) == 4                       # onto itself, one element on
    assert _clip(lib, [(a, b, 8, 1), (c, b + 16, 8, 1)]) == 4        # two outputs
    assert _clip(lib, [(a, b, 8, 1), (b, c, 8, 1)]) == 4             # an output that is another's input
    assert _clip(lib, [(c, c, 1000, 1), (a, a, 8, 1), (c + 400, b, 8, 0)]) == 4  # inside a larger one


def test_binding_refuses_tensors_off_the_gpu_and_of_other_shapes():
    z = torch.zeros(6, 10)
    with pytest.raises(ValueError):
        H.hydra_token_logprobs_entropy(z, None, None, 2, 3, entropy=torch.zeros(6))
    with pytest.raises(ValueError):
        H.hydra_token_logprobs_entropy(z.half(), None, None, 2, 3, entropy=torch.zeros(6))
    with pytest.raises(ValueError):
        H.hydra_token_logprobs_entropy_grad(z, None, None, 2, 3, z, z, z, None, z)
    with pytest.raises(ValueError):
        H.GradList([torch.zeros(3)])
    with pytest.raises(ValueError):
        H.GradList([torch.zeros(3)], [])
    assert len(H.GradList([])) == 0


def test_list_entry_layout_is_the_headers():
    assert ctypes.sizeof(H.GradTensorC) == 32
    assert [getattr(H.GradTensorC, n).offset for n in ("grad", "out", "numel", "dtype")] == [0, 8, 16, 24]
