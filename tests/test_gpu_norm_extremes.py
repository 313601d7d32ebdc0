"""GPU tests of the RMS norm at both ends of the 32-bit numbers, where a row's reciprocal root is none: without an eps the result
is a row's direction times the root of its width, whatever the row's size.  Tolerances are run_norm's."""
import pytest

from paper_2008_04567_amd import binding as B
from tests import parity as PT

pytestmark = pytest.mark.gpu

WIDTHS = [24, 700, 1500, 7000, 20000, 40000]      # rows of a wave, of four, of sixteen, and those that hold several pieces


@pytest.fixture(scope="module")
def A():
    PT.torch_dev()
    from tests import around_case
    return around_case


@pytest.mark.parametrize("scale", [1e-36, 1e-38, 2e-39, 1e-40, 1e-42, 1e-44])
@pytest.mark.parametrize("width", WIDTHS)
def test_rows_of_the_smallest_numbers(A, width, scale):
    A.run_norm(3, width, "f32", scale=scale, eps=0.0, q=True)
    A.run_norm(3, width, "f32", scale=scale, eps=0.0, residual=False, gain=False)


@pytest.mark.parametrize("scale", [2e-39, 1e-39])
def test_rows_of_the_smallest_numbers_in_bf16(A, scale):
    for width in (128, 2048):
        A.run_norm(3, width, "bf16", scale=scale, eps=0.0, q=True)


@pytest.mark.parametrize("width", WIDTHS + [65536])
def test_one_smallest_number_among_zeros(A, width):
    def edit(x, res, g):
        x.zero_()
        res.zero_()
        x[0, width // 2], x[1, 0], res[2, width - 1] = 2.0 ** -149, -2.0 ** -149, 2.0 ** -149
    A.run_norm(3, width, "f32", edit=edit, eps=0.0, q=True)


@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-30, 1e-5])
def test_small_rows_beside_an_eps(A, eps):
    # (the definition has the eps that the descriptor holds, 32 bits: 1e-44 is 7 2^-149 there, two parts of a hundred less)
    eps = B.make_rms_norm_desc(1, 1, eps=eps).eps
    for scale in (1e-12, 1e-20, 1e-39):
        A.run_norm(3, 1000, "f32", scale=scale, eps=eps)


@pytest.mark.parametrize("width", WIDTHS)
def test_rows_of_the_largest_numbers(A, width):
    def edit(x, res, g):
        x[:] = 3.4e38
        x[1, ::2] *= -1.0
        x[2] *= 0.5
        res.zero_()
    A.run_norm(3, width, "f32", edit=edit, eps=0.0, q=True)


def test_infinities_and_zeros_as_the_formula_has_them(A):
    """Over an infinite root numbers are zero and the infinity is none; zeros over zero are none."""
    def edit(x, res, g):
        x[0, 5] = float("inf")
        x[1], res[1] = 0.0, 0.0
    for width in (64, 3000):
        A.run_norm(3, width, "f32", edit=edit, eps=0.0)
