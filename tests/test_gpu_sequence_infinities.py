"""GPU tests of the scan over infinities, NaN and the largest numbers: what they leave is what the definition says, an
infinity of its sign where that has one, NaN where that has NaN, and all else as without them."""
import numpy as np
import pytest

from tests import parity as PT

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "f16", "f32"]
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def S():
    PT.torch_dev()
    from tests import sequence_case
    return sequence_case


@pytest.fixture(scope="module")
def kinds(S):
    """run_scan with finite values within the usual tolerances and all others of the same kind."""
    from tests import sequence_strict

    def close(got, ref, d, dtype, share, what):
        # (magnitudes are infinite where a value is; what has vanished against an infinity is compared as a kind only)
        with np.errstate(invalid="ignore"):
            d = np.where(np.isfinite(d), d, 0.0)
        sequence_strict.close(got, ref, d, dtype, share, what)
        mine, want = sequence_strict.kind(S.f64(got)), sequence_strict.kind(ref)
        assert np.array_equal(mine, want), "%s: %d infinities or NaN that are others" % (what, (mine != want).sum())

    def run(*args, **kw):
        with pytest.MonkeyPatch.context() as patch:
            patch.setattr(S, "close", close)
            S.run_scan(*args, **kw)
    return run


# (state_dim 1: y is one product, so its infinities are not sums of several)
SIZES = [(2, 32, 1, 1), (4, 20, 2, 36), (2, 64, 1, 64), (2, 72, 1, 128), (1, 16, 1, 200)]


def put(name, *where):
    def edit(i):
        for row, column, value in where:
            i[name][row, column] = value
    return edit


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,head_dim,groups,state_dim", SIZES)
@pytest.mark.parametrize("step", [False, True])
def test_infinite_inputs(kinds, dtype, heads, head_dim, groups, state_dim, step):
    lengths = [1] * 9 if step else [5, 70, 33, 130, 0, 64]
    last = sum(lengths) - 1
    edits = [put("x", (3, 7, INF), (last, 0, -INF), (last // 2, 9, NAN)), put("z", (2, 3, INF), (last, 1, -3.0)),
             put("b", (4, 0, -INF)), put("b", (last, 0, NAN)), put("c", (4, 0, INF), (last - 2, 0, -INF)), put("c", (1, 0, NAN))]
    for k, edit in enumerate(edits):
        kinds(lengths, heads, head_dim, groups, state_dim, dtype, step=step, edit=edit, pad=(0, 8, 3)[k % 3],
              offset=(0, 8, 1)[k % 3], in_place=k % 2 == 1, gate=k != 3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,head_dim,groups,state_dim", SIZES)
@pytest.mark.parametrize("step", [False, True])
def test_infinite_states_are_continued_from(kinds, dtype, heads, head_dim, groups, state_dim, step):
    def edit(i):
        i["pool"][2, 0, 3, 0], i["pool"][3, heads - 1, 5, state_dim - 1], i["pool"][4, 0, 0, 0] = INF, -INF, NAN
    lengths = [1] * 4 if step else [40, 65, 1, 130]
    for gate in (False, True):
        kinds(lengths, heads, head_dim, groups, state_dim, dtype, step=step, edit=edit, in_place=gate, gate=gate)


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_in_requests_that_are_cut(kinds, dtype):
    def edit(i):
        i["x"][40, 3], i["x"][700, 9], i["x"][1499, 20] = INF, -INF, INF
        i["c"][900, 0] = INF
        i["pool"][2, 1, 30, 0] = -INF
    for state_dim in (1, 64):
        kinds([1500], 2, 32, 1, state_dim, dtype, edit=edit)
        kinds([1500], 2, 32, 1, state_dim, dtype, edit=edit, pad=1, in_place=True)
        kinds([700, 3, 0, 1100], 2, 32, 2, state_dim, dtype, edit=edit, resume=[1, 0, 1, 1])


@pytest.mark.parametrize("step", [False, True])
def test_infinite_skip_and_steps(kinds, step):
    def edit(i):
        i["d"][1] = INF
        i["dt"][4, 0], i["dt"][6, 1] = INF, NAN
    for dtype in DTYPES:
        kinds([1] * 9 if step else [9, 70], 2, 20, 1, 16, dtype, step=step, edit=edit)


@pytest.mark.parametrize("step", [False, True])
def test_numbers_that_round_to_infinity_in_16_bits(kinds, step):
    # fp32 numbers beyond the largest bf16 number, in the state and in x
    def edit(i):
        i["pool"].mul_(1e-3)
        i["pool"][2, 0, 3, 0], i["pool"][3, 1, 5, 0] = 3.402e38, -3.4e38
        i["x"][2, 4] = 3.4e38
        for name in ("b", "c"):
            i[name].mul_(1e-3)
    kinds([1] * 4 if step else [40, 65], 2, 32, 1, 1, "f32", step=step, edit=edit, skip=False, gate=False)
    kinds([1] * 4 if step else [40, 65], 2, 32, 1, 64, "f32", step=step, edit=edit, skip=False, gate=False)
