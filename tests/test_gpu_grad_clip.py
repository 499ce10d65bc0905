"""Global gradient norm and clipping against the fp64 oracle.

Tolerances, u = 2^-24: a thread adds at most 34 squares of a chunk in fp32 (relative error 35 u at
most, all terms positive) and the rest is fp64, so the norm is off by 18 u and its fp32 rounding by u;
the coefficient by the same and its own rounding; a clipped value by that, the product's rounding and
the rounding to its type (half a step, eps / 2)."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.helpers import host_f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
INF = float("inf")
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    B.build()
    H.load()
    H.device_error(clear=True)
    yield
    assert H.device_error(clear=True) == 0


def tensors(seed, sizes, types, scale=1.0, shifts=(0,)):
    """Tensors of the given sizes and types, each `shift` elements behind a 16-byte boundary."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        s, t = shifts[i % len(shifts)], types[i % len(types)]
        buf = torch.empty(n + s, dtype=t, device="cuda")
        buf[s:] = scale * torch.randn(n, device="cuda", generator=g)
        out.append(buf[s:])
    return out


def workspace():
    return torch.full((H.grad_norm_workspace_size(),), 0xFF, dtype=torch.uint8, device="cuda")


def check(grads, max_norm, in_place=False, out_shifts=(0,)):
    values = [host_f64(g) for g in grads]
    norm, coef, want = O.clip_grad_norm(values, max_norm)
    n2, ws = torch.full((2,), float("nan"), device="cuda"), workspace()
    H.hydra_grad_norm(H.GradList(grads), max_norm, n2, ws)
    got = n2.cpu().double().numpy().copy()
    assert abs(got[0] - norm) <= 20 * U * norm and abs(got[1] - coef) <= 22 * U * coef, (got, norm, coef)
    if in_place:
        outs = grads
    else:
        outs = []
        for i, g in enumerate(grads):
            s = out_shifts[i % len(out_shifts)]
            buf = torch.full((g.numel() + s + 3,), float("nan"), dtype=g.dtype, device="cuda")
            outs.append(buf[s:s + g.numel()])
    n3 = torch.full((2,), float("nan"), device="cuda")
    H.hydra_clip_grad_norm(H.GradList(grads, None if in_place else outs), max_norm, n3, ws)
    assert torch.equal(n2, n3)
    for o, w in zip(outs, want):
        half = torch.finfo(o.dtype).eps / 2
        tol = (24 * U + half * (1 + 2.0 ** -6)) * np.abs(w) + (2.0 ** -133 if o.dtype == BF16 else 2.0 ** -149)
        assert np.all(np.abs(host_f64(o) - w) <= tol)
    if not in_place:
        for g, v in zip(grads, values):
            assert np.array_equal(host_f64(g), v)  # the inputs stay
        for i, (o, g) in enumerate(zip(outs, grads)):
            s = out_shifts[i % len(out_shifts)]
            whole = o.as_strided((g.numel() + s + 3,), (1,), 0) if g.numel() else o
            assert torch.isnan(whole[:s]).all() and torch.isnan(whole[s + g.numel():]).all()
    return got


LISTS = [
    ([1], [F32]),
    ([1], [BF16]),
    ([0, 1, 0, 3, 0], [F32, BF16]),
    ([4096], [F32]),
    ([8192, 8193, 8191], [BF16]),
    ([4095, 4097, 1, 12289], [F32]),
    ([5, 70001, 33, 16384, 999], [BF16, F32]),
    ([3_000_017], [F32]),
    ([3_000_017, 5, 2_000_003], [BF16]),
    ([1000] * 150 + [100_003] * 20, [F32, BF16, F32]),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("shifts,out_shifts", [((0,), (0,)), ((1, 0, 3), (1, 0, 3)), ((1, 2, 5), (0, 7, 1))])
@pytest.mark.parametrize("sizes,types", LISTS)
def test_clip_parity(sizes, types, shifts, out_shifts, in_place):
    check(tensors(len(sizes) + sizes[0], sizes, types, shifts=shifts), 0.5, in_place, out_shifts)


@pytest.mark.parametrize("in_place", [False, True])
def test_norm_below_the_largest_leaves_every_bit(in_place):
    grads = tensors(3, [1000, 33333], [F32, BF16], 1e-3, (0, 1))
    before = [g.clone() for g in grads]
    got = check(grads, 10.0, in_place, (2, 1))
    assert got[1] == 1.0 and all(torch.equal(a, b) for a, b in zip(grads, before))


@pytest.mark.parametrize("scale", [1e-42, 1e-30, 1e-22, 1e-18, 1e12, 1e18, 1e30, 1e37])
def test_no_square_overflows_or_vanishes(scale):
    """Values down to subnormal ones and up to 1e38: the norm is right as long as it is an fp32 number."""
    check(tensors(5, [20011, 300], [F32]), 1.0)
    g = tensors(5, [20011, 300], [F32], scale)
    values = [host_f64(x) for x in g]
    norm, coef, want = O.clip_grad_norm(values, 1.0)
    n2 = torch.zeros(2, device="cuda")
    outs = [torch.empty_like(x) for x in g]
    H.hydra_clip_grad_norm(H.GradList(g, outs), 1.0, n2, workspace())
    got = n2.cpu().double().numpy()
    assert (abs(got[0] - norm) <= 20 * U * norm + 2.0 ** -149) if norm < 3.4e38 else got[0] == INF
    assert abs(got[1] - coef) <= 22 * U * coef + 2.0 ** -149
    for o, w in zip(outs, want):
        # a subnormal coefficient has few bits: half a step of 2^-149
        assert np.all(np.abs(host_f64(o) - w) <= 26 * U * np.abs(w) + 2.0 ** -149 * (1 + np.abs(w / max(coef, 1e-300))))


def test_one_large_value_among_zeros_and_small_ones():
    g = torch.zeros(100_000, device="cuda")
    g[77_777] = 1e25
    g[5] = 1e-30
    check([g, torch.zeros(50, dtype=BF16, device="cuda")], 1.0)
    check([torch.zeros(5000, device="cuda")], 1.0)


@pytest.mark.parametrize("bad", [INF, -INF, float("nan")])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_norm_that_is_not_finite_leaves_the_values(bad, in_place):
    grads = tensors(7, [9001, 513], [F32, BF16])
    grads[1][100] = bad
    before = [g.clone() for g in grads]
    outs = grads if in_place else [torch.zeros_like(g) for g in grads]
    n2 = torch.zeros(2, device="cuda")
    H.hydra_clip_grad_norm(H.GradList(grads, outs), 1.0, n2, workspace())
    assert not torch.isfinite(n2[0]) and torch.isnan(n2[0]).item() == (bad != bad) and n2[1] == 1.0
    for o, b in zip(outs, before):
        assert torch.equal(o.view(torch.int16), b.view(torch.int16))


def test_empty_lists_and_an_infinite_largest_norm():
    n2 = torch.full((2,), 5.0, device="cuda")
    for lst in (H.GradList([]), H.GradList([torch.empty(0, device="cuda")])):
        for fn in (H.hydra_grad_norm, H.hydra_clip_grad_norm):
            n2.fill_(5.0)
            fn(lst, 1.0, n2, workspace())
            assert n2.tolist() == [0.0, 1.0]
    assert check(tensors(8, [100], [F32]), INF)[1] == 1.0


@pytest.mark.parametrize("n", [959, 960, 961, 2500])
def test_more_tensors_than_one_launch_takes(n):
    check(tensors(9, [(i * 37) % 501 for i in range(n)], [F32, BF16], shifts=(0, 1, 2)), 0.25, True)


def test_large_tensors_and_equal_bits():
    """More than 2^31 bytes in one tensor; two calls and a list in other buffers agree in every bit."""
    g = torch.Generator(device="cuda").manual_seed(2)
    big = torch.randn(600_000_011, device="cuda", generator=g)
    small = torch.randn(1001, device="cuda", generator=g).to(BF16)
    n2, n3, ws = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda"), workspace()
    H.hydra_grad_norm(H.GradList([big, small]), 1.0, n2, ws)
    norm = float(torch.sqrt(sum(x.double().square().sum() for x in (*big.split(1 << 26), small))))
    assert abs(n2[0].item() - norm) <= 20 * U * norm
    tail = big[-1000:].double()
    H.hydra_clip_grad_norm(H.GradList([big, small]), 1.0, n3, ws)
    assert torch.equal(n2, n3)
    assert torch.allclose(big[-1000:].double(), tail * n2[1].double(), rtol=4 * U, atol=0)


def test_a_tensor_twice_is_counted_twice_and_not_clipped():
    (g,) = tensors(10, [777], [F32])
    n2, ws = torch.zeros(2, device="cuda"), workspace()
    H.hydra_grad_norm(H.GradList([g, g]), 1.0, n2, ws)
    want = np.sqrt(2 * (host_f64(g) ** 2).sum())
    assert abs(n2[0].item() - want) <= 20 * U * want
    before = g.clone()
    with pytest.raises(H.HydraError) as e:
        H.hydra_clip_grad_norm(H.GradList([g, g]), 1.0, n2, ws)
    assert e.value.status == 4 and torch.equal(g, before)


def test_two_captured_graphs_share_a_workspace():
    """Each replay stands by itself: new values in the same buffers, the other graph in between."""
    lists = [tensors(11, [30_011, 17], [F32, BF16]), tensors(12, [400] * 40, [BF16])]
    outs = [[torch.empty_like(g) for g in x] for x in lists]
    norms, ws = [torch.zeros(2, device="cuda") for _ in lists], workspace()
    plans = [H.GradList(g, o) for g, o in zip(lists, outs)]
    side, graphs = torch.cuda.Stream(), []
    for plan, n2 in zip(plans, norms):
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            H.hydra_clip_grad_norm(plan, 0.5, n2, ws)
        graphs.append(graph)
    for scale in (1.0, 3.0):
        for x in lists:
            for g in x:
                g.mul_(scale)
        for i in (0, 1, 0):
            graphs[i].replay()
        for x, o, n2 in zip(lists, outs, norms):
            norm, coef, want = O.clip_grad_norm([host_f64(g) for g in x], 0.5)
            assert abs(n2[0].item() - norm) <= 20 * U * norm
            for a, w in zip(o, want):
                half = torch.finfo(a.dtype).eps / 2
                assert np.all(np.abs(host_f64(a) - w) <= (24 * U + half * (1 + 2.0 ** -6)) * np.abs(w) + 2.0 ** -133)


def test_on_another_stream():
    side = torch.cuda.Stream()
    (g,) = tensors(13, [250_007], [F32])
    want, n2, n3 = torch.empty_like(g), torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    H.hydra_clip_grad_norm(H.GradList([g], [want]), 1.0, n2, workspace())
    ws = workspace()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        H.hydra_clip_grad_norm(H.GradList([g]), 1.0, n3, ws)
    side.synchronize()
    assert torch.equal(g, want) and torch.equal(n2, n3)
