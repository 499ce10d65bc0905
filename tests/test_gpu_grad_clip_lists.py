"""Gradient norm and clipping: the three operations behind the sum, and lists of every size that takes a way of its own.

u = 2^-24, half a step of fp32. A thread adds the squares of its elements of a chunk in fp32, one rounding each: of 32 KB (lists
of 120 MB on) up to 64 of bf16 and one or two at its ends, 66 roundings of sums that only grow, so 66 u relative; of 16 KB
34 u. These sums are added in pairs of fp32 numbers, whose own errors (2^-46 each, 2^11 in a row at most) vanish beside
that, and root and quotient are rounded once. So the norm is off by (66 / 2 + 1) u, the coefficient by 35 u, a clipped
value by 36 u with its product's rounding and by the rounding to its type (half a step, eps / 2)."""
import numpy as np
import pytest
import torch

from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.test_gpu_grad_clip import BF16, F32, U, workspace

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    B.build()
    H.load()
    H.device_error(clear=True)
    yield
    assert H.device_error(clear=True) == 0


def test_norm_and_coefficient_are_rounded_once():
    """Squares of whole numbers add up exactly, so nothing but root, sum and quotient can be off: half a step, and
    2^-40 for what the correction of each leaves out. Norms far below 1e-6 and in the range of the fp64 sums, too."""
    rng = np.random.default_rng(1)
    n2, ws = torch.zeros(2, device="cuda"), workspace()
    for _ in range(300):
        g = rng.integers(-999, 1000, rng.integers(1, 700)) * 2.0 ** rng.integers(-60, 50)
        max_norm = float(np.float32(np.sqrt((g * g).sum() + 1e-14) * 10 ** rng.uniform(-5, 1)))
        H.hydra_grad_norm(H.GradList([torch.from_numpy(g.astype(np.float32)).cuda()]), max_norm, n2, ws)
        norm = np.sqrt((g * g).sum())
        want = np.array([norm, min(1.0, max_norm / (norm + 1e-6))])
        got = n2.cpu().numpy()
        half = np.spacing(want.astype(np.float32)).astype(np.float64) / 2
        assert np.all(np.abs(got.astype(np.float64) - want) <= half + 2.0 ** -40 * want), (got, want, g)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("size,touched", [(1e38, True), (3e38, True), (INF, False)])
def test_the_coefficient_tells_whether_values_were_touched(size, touched, in_place):
    """A norm of +inf may be a finite one beyond fp32: then the coefficient is below 1 and every value clipped."""
    g = torch.full((100_000,), size, device="cuda")
    out, n2 = g if in_place else torch.zeros_like(g), torch.zeros(2, device="cuda")
    H.hydra_clip_grad_norm(H.GradList([g], [out]), 1.0, n2, workspace())
    norm, coef = n2.tolist()
    assert norm == INF and (coef < 1) == touched
    want = 1 / np.sqrt(1e5) if touched else size
    # a coefficient of about 1e-41 is a multiple of 2^-149: half a step of it
    tol = want * (2.0 ** -150 / coef + 4 * U) if touched else 0
    assert (out.double() == want).all() if not touched else ((out.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("fn", [H.hydra_grad_norm, H.hydra_clip_grad_norm])
def test_empty_lists_have_a_norm_of_zero(fn):
    n2 = torch.full((2,), 5.0, device="cuda")
    for max_norm, coef in ((1.0, 1.0), (1e-6, 1.0), (2.5e-7, 0.25), (INF, 1.0)):
        fn(H.GradList([]), max_norm, n2, workspace())
        assert n2[0] == 0 and abs(n2[1].item() - min(1.0, float(np.float32(max_norm)) / 1e-6)) <= U * coef


def test_a_list_keeps_the_memory_that_its_tensors_had():
    """Memory that a gradient has let go of is not given to another tensor while a list writes there."""
    n2, ws = torch.zeros(2, device="cuda"), workspace()
    g = torch.full((3_000_000,), 2.0, device="cuda")
    out = torch.zeros_like(g)
    plans = [H.GradList([g]), H.GradList([g], [out])]
    g.data, out.data = torch.ones(5, device="cuda"), torch.ones(5, device="cuda")
    others = [torch.full((3_000_000,), 7.0, device="cuda") for _ in range(4)]
    for plan in plans:
        H.hydra_clip_grad_norm(plan, 1.0, n2, ws)
    assert all((x == 7).all() for x in others)
    H.hydra_grad_norm(plans[0], 1.0, n2, ws)
    assert abs(n2[0].item() - 1) <= 1e-6


def filled(sizes, kinds, seed, shifts):
    """Tensors of the given sizes and types, `shift` elements behind a 16-byte boundary, each of a scale of its own."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        s, t = shifts[i % len(shifts)], kinds[i % len(kinds)]
        buf = torch.empty(n + s, dtype=t, device="cuda")
        buf[s:] = torch.randn(n, device="cuda", generator=g) * 10.0 ** (i % 5 - 2)
        out.append(buf[s:])
    return out


def check_all(grads, max_norm, out_shifts):
    """Every output against 64 bits, on the device; out_shifts None: in place. What lies around outputs stays."""
    norm = float(torch.stack([(x.double() ** 2).sum() for x in grads]).sum().sqrt())
    coef = min(1.0, max_norm / (norm + 1e-6))
    n2, n3, ws = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda"), workspace()
    H.hydra_grad_norm(H.GradList(grads), max_norm, n2, ws)
    assert abs(n2[0].item() - norm) <= 34 * U * norm and abs(n2[1].item() - coef) <= 35 * U * coef
    before = [x.clone() for x in grads]
    bufs, outs = [], grads
    if out_shifts is not None:
        for i, x in enumerate(grads):
            s = out_shifts[i % len(out_shifts)]
            bufs.append(torch.full((x.numel() + s + 9,), 7.0, dtype=x.dtype, device="cuda"))
        outs = [b[out_shifts[i % len(out_shifts)]:][:x.numel()] for i, (b, x) in enumerate(zip(bufs, grads))]
    H.hydra_clip_grad_norm(H.GradList(grads, outs), max_norm, n3, ws)
    assert torch.equal(n2, n3)
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for i, (x, o) in enumerate(zip(before, outs)):
        want = x.double() * coef
        half = torch.finfo(x.dtype).eps / 2
        tol = (36 * U + half * (1 + 2.0 ** -6)) * want.abs() + (2.0 ** -133 if x.dtype == BF16 else 2.0 ** -149)
        bad += ((o.double() - want).abs() > tol).sum()
        if out_shifts is not None:
            s, b = out_shifts[i % len(out_shifts)], bufs[i]
            bad += (b[:s] != 7).sum() + (b[s + x.numel():] != 7).sum() + (grads[i] != x).sum()
    assert int(bad) == 0


LARGE = {  # 32 KB chunks, in tables of 224 and 880 and several launches
    "few": ([20_000_003, 33_000_001, 5, 7_000_009, 8191, 16385, 1], [F32, BF16, F32, F32, BF16]),
    "bf16": ([60_000_007, 25_000_000, 333], [BF16]),
    "300": ([180_001 + 7 * i for i in range(300)], [F32, F32, BF16]),
    "1000": ([55_001 + 3 * i for i in range(1000)], [F32, BF16, F32]),
}


@pytest.mark.parametrize("shifts,out_shifts", [((0,), None), ((1, 0, 3), None), ((0, 1), (0, 1)), ((1, 2, 5), (0, 7, 1))])
@pytest.mark.parametrize("name", LARGE)
def test_large_lists(name, shifts, out_shifts):
    sizes, kinds = LARGE[name]
    grads = filled(sizes, kinds, len(sizes), shifts)
    assert sum(g.numel() * g.element_size() for g in grads) >= 160 << 20
    check_all(grads, 0.5, out_shifts)


@pytest.mark.parametrize("out_shifts", [None, (2, 0, 1)])
@pytest.mark.parametrize("n", [31, 32, 33, 223, 224, 225, 879, 880, 881, 1760, 1761])
def test_lists_around_the_sizes_of_the_tables(n, out_shifts):
    check_all(filled([(i * 37) % 501 + 1 for i in range(n)], [F32, BF16], n, (0, 1, 2)), 0.25, out_shifts)
    check_all(filled([(i * 1237) % 20011 + 1 for i in range(n)], [BF16, F32, F32], n, (0, 3)), 1e9, out_shifts)
