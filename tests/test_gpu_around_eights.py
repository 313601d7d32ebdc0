"""GPU tests of 8-bit products whose neighbouring entries are far apart: one outlier beside small values, and outliers that cancel.

Into a y of 16 bits, the products of entries 8 i .. 8 i + 7 are added with 13 bits below the largest of them, so each of the other
seven may lose 2^-13 of it: a sum is off by at most 7 2^-13 M, M the largest magnitudes of its eights added up, and by what 32-bit
sums are, (k + 64) 2^-24 D (around_case.py).  Into a y of 32 bits the latter alone."""
import numpy as np
import pytest

from tests import parity as PT

pytestmark = pytest.mark.gpu

# rows, columns, reduction: both kernels for few rows, and tiles of 64, 128 and 256
SIZES = [(3, 300, 1160), (40, 500, 272), (130, 300, 1000), (2000, 3200, 4128), (4100, 4097, 1160)]
PATTERNS = ["outlier", "outlier of any sign", "outliers that cancel"]
DISTINCT_X, DISTINCT_W = 37, 41      # rows that there are of each; a matrix repeats them


@pytest.fixture(scope="module")
def A():
    PT.torch_dev()
    from tests import around_case
    return around_case


def in_range(r, lo, hi, shape):
    """Random e4m3 numbers, lo and hi powers of two: three bits of mantissa."""
    e = r.integers(int(np.log2(lo)), int(np.log2(hi)), shape)
    return (1.0 + r.integers(0, 8, shape) / 8.0) * 2.0 ** e


def operands(r, pattern, k):
    """Rows whose eights hold an outlier or two at the same places: products of some 2^15 beside such of some 2^1."""
    x, w = in_range(r, 0.25, 2.0, (DISTINCT_X, k)), in_range(r, 0.5, 4.0, (DISTINCT_W, k))
    big = np.zeros(k, bool)
    for i in range(0, k, 8):
        at = i + r.permutation(min(8, k - i))[:2]
        big[at[0]] = True
        if pattern == "outliers that cancel" and len(at) == 2:
            big[at[1]] = True
            x[:, at[1]] = x[:, at[0]] = in_range(r, 128.0, 256.0, DISTINCT_X)
            w[:, at[0]] = in_range(r, 64.0, 256.0, DISTINCT_W)
            w[:, at[1]] = -w[:, at[0]]
        else:
            x[:, at[0]], w[:, at[0]] = in_range(r, 128.0, 256.0, DISTINCT_X), in_range(r, 64.0, 256.0, DISTINCT_W)
    if pattern == "outlier of any sign":
        x *= r.choice([-1.0, 1.0], x.shape)
        w *= r.choice([-1.0, 1.0], w.shape)
    return x, w


def codes(A, v):
    """(rows in whole 16 bytes, NaN behind them) of e4m3 numbers."""
    import torch
    out = torch.full((len(v), -(-v.shape[1] // 16) * 16), 0x7f, device="cuda", dtype=torch.uint8)
    q = torch.from_numpy(v.astype(np.float32)).cuda().to(A.F8).view(torch.uint8)
    assert np.array_equal(A.numbers(q), v), "not e4m3 numbers"
    out[:, :v.shape[1]] = q
    return out


def reference(x, w, xs, ws):
    """(sums, magnitudes D, largest of eights M) of all pairs of distinct rows; xs, ws: scales of their blocks."""
    k = x.shape[1]
    x, w = x * np.repeat(xs, 128, axis=1)[:, :k], w * np.repeat(ws, 128)[:k]
    p = np.abs(x)[:, None, :] * np.abs(w)[None]
    p = np.pad(p, ((0, 0), (0, 0), (0, -k % 8)))
    return x @ w.T, p.sum(2), p.reshape(len(x), len(w), -1, 8).max(3).sum(2)


def allowed(d, most, k, dtype):
    return (k + 64) * 2.0 ** -24 * d + (0.0 if dtype == "f32" else 7 * 2.0 ** -13 * most)


def inputs(A, pattern, k, dtype):
    r = np.random.default_rng(k + PATTERNS.index(pattern))
    x, w = operands(r, pattern, k)
    # (f16 ends at 65504: sums of up to 516 eights of 2^16 are scaled below it)
    xs = r.uniform(0.5, 1.0, (DISTINCT_X, A.oa.blocks(k))).astype(np.float32) * np.float32(2.0 ** -11)
    ws = r.uniform(0.5, 1.0, A.oa.blocks(k)).astype(np.float32)
    return x, w, xs, ws, reference(x, w, xs.astype(np.float64), ws.astype(np.float64))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pattern", PATTERNS)
@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear_q8_keeps_the_stated_bound(A, m, n, k, pattern, dtype):
    import torch
    B, (code, ty) = A.B, A.TYPES[dtype][:2]
    x, w, xs, ws, (ref, d, most) = inputs(A, pattern, k, dtype)
    at_x, at_w = np.arange(m) % DISTINCT_X, np.arange(n) % DISTINCT_W
    xq, wq = codes(A, x)[torch.from_numpy(at_x).cuda()], codes(A, w)[torch.from_numpy(at_w).cuda()]
    x_scales = torch.from_numpy(xs[at_x]).cuda()
    w_scales = torch.from_numpy(ws).cuda().repeat(A.oa.blocks(n), 1)
    y = torch.empty((m, n), device="cuda", dtype=ty)
    desc = B.make_linear_q8_desc(m, n, k, dtype=code)
    B.linear_q8_fwd(desc, xq, x_scales, wq, w_scales, y, workspace=A.workspace(B.linear_q8_workspace(desc)))
    pairs = np.ix_(at_x, at_w)
    A.close(y, ref[pairs], allowed(d, most, k, dtype)[pairs], dtype, 1.0, "8-bit product, %s %s" % (pattern, (m, n, k, dtype)))


# rows of the experts, columns, reduction: the kernel for few rows, and tiles of 64, 128 and 256
GROUPED = [([5, 20, 0], 300, 1160), ([100, 0, 200], 3000, 1160), ([900, 300, 0, 1200], 3600, 1040), ([1500, 900, 0, 1700], 8200, 1040)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pattern", PATTERNS)
@pytest.mark.parametrize("lengths,n,k", GROUPED)
def test_products_by_expert_keep_the_stated_bound(A, lengths, n, k, pattern, dtype):
    import torch
    B, (code, ty) = A.B, A.TYPES[dtype][:2]
    groups, rows = len(lengths), sum(lengths)
    x, w, xs, ws, (ref, d, most) = inputs(A, pattern, k, dtype)
    expert = np.repeat(np.arange(groups), lengths)
    at_x = np.arange(rows) % DISTINCT_X
    at_w = (np.arange(n)[None] + 7 * np.arange(groups)[:, None]) % DISTINCT_W         # of every expert's columns
    xq, wq = codes(A, x)[torch.from_numpy(at_x).cuda()], codes(A, w)[torch.from_numpy(at_w).cuda()]
    x_scales = torch.from_numpy(xs[at_x]).cuda()
    w_scales = torch.from_numpy(ws).cuda().repeat(groups, A.oa.blocks(n), 1)
    y = torch.empty((rows, n), device="cuda", dtype=ty)
    desc = B.make_grouped_linear_desc(groups, rows, n, k, dtype=B.E4M3, y_dtype=code)
    B.grouped_linear_fwd(desc, xq, wq, A.i32([0] + np.cumsum(lengths).tolist()), y, x_scales=x_scales, w_scales=w_scales)
    pairs = at_x[:, None], at_w[expert]
    A.close(y, ref[pairs], allowed(d, most, k, dtype)[pairs], dtype, 1.0, "by expert, %s %s" % (pattern, (lengths, n, k, dtype)))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m", [2, 100])
def test_thirteen_bits_below_the_largest_are_kept(A, m, dtype):
    """2^14 - 2^14 + 2^1 within an eight is 2 in every type: what is 2^-13 of the largest is not lost.  In different eights,
    and in a y of 32 bits, far smaller terms are kept."""
    import torch
    B, (code, ty) = A.B, A.TYPES[dtype][:2]
    k, n = 128, 64
    for base in (0, 8, 56, 120):
        for order in range(8):
            x, w = np.zeros((m, k)), np.zeros((n, k))
            big, other, small = [base + (order + i) % 8 for i in (0, 3, 5)]
            x[:, big], x[:, other], x[:, small] = 128.0, 128.0, 2.0
            w[:, big], w[:, other], w[:, small] = 128.0, -128.0, 1.0
            x[:, (base + 64) % k], w[:, (base + 64) % k] = 0.125, 0.125
            y = torch.empty((m, n), device="cuda", dtype=ty)
            one = lambda *s: torch.ones(s, device="cuda")
            B.linear_q8_fwd(B.make_linear_q8_desc(m, n, k, dtype=code), codes(A, x), one(m, 1), codes(A, w), one(1, 1), y)
            assert bool((y == torch.tensor(2.0 + 2.0 ** -6, dtype=ty, device="cuda")).all()), (base, order, y[0, 0].item())
