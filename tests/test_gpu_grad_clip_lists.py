"""Gradient norm and clipping: the three operations behind the sum, and lists of every size that takes a way of its own.

u = 2^-24, half a step of fp32."""
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
