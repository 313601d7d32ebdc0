"""GPU tests of the sequence layers' elementary functions, each value against 64 bits."""
from math import erfc

import numpy as np
import pytest

from tests import parity as PT

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "f16", "f32"]


@pytest.fixture(scope="module")
def S():
    PT.torch_dev()
    from tests import sequence_case
    return sequence_case


def half_spacing(v, dtype):
    """Half of the distance between neighbouring numbers of the type around v."""
    bits, least = {"bf16": (7, -126), "f16": (10, -14), "f32": (23, -126)}[dtype]
    return 0.5 * 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 1e-300))), least) - bits)


def of_every_value(S, values, dtype, act, y_f32, m):
    """act of every value, by a product with one entry of 1 in a row: [m][values] in 64 bits."""
    import torch
    B, (code, ty) = S.B, S.TYPES[dtype][:2]
    n, k = len(values), 8
    x, w = torch.zeros((m, k), device="cuda", dtype=ty), torch.zeros((n, k), device="cuda", dtype=ty)
    x[:, 3], w[:, 3] = 1.0, values.cuda()
    y = torch.empty((m, n), device="cuda", dtype=torch.float32 if y_f32 else ty)
    desc = B.make_linear_desc(m, n, k, dtype=code, y_dtype=B.F32 if y_f32 else code, act=S.ACTS[act])
    ws = torch.empty(max(16, B.linear_workspace(desc)), device="cuda", dtype=torch.uint8)
    B.linear_fwd(desc, x, w, y, workspace=ws)
    return S.f64(y)


@pytest.mark.parametrize("dtype,y_f32", [("bf16", False), ("f16", False), ("f32", False), ("f16", True)])
@pytest.mark.parametrize("m", [1, 70])
def test_gelu_holds_its_digits_below_zero(S, dtype, y_f32, m):
    # gelu(v) = v erfc(-v / sqrt 2) / 2, whose second factor goes to zero below zero.  Of that factor: in 16 bits 2^-17 from
    # the approximation, 2 v^2 2^-24 from the exponent v^2 / 2 (three roundings) and 32 2^-24 from the rest; in 32 bits
    # 1.3 (v^2 + 1) 2^-24 from the argument (rounded, times a rounded constant), 18 2^-24 from the rest.  Numbers below
    # 2^-120 may come out as zero.
    import torch
    if dtype == "f32":
        v = torch.from_numpy(np.concatenate([-np.geomspace(1e-6, 12.9, 9001), np.geomspace(1e-6, 30.0, 3001)]).astype(np.float32))
    else:
        v = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(S.TYPES[dtype][1])
        size = v.float().abs()
        v = v[torch.isfinite(v.float()) & (size < 30.0) & ((size > 2.0 ** -100) | (v == 0)) & (v.float() > -12.9)]
    ref = np.array([0.5 * t * erfc(-t * 0.5 ** 0.5) for t in S.f64(v)])
    got = of_every_value(S, v, dtype, "gelu", y_f32, m)
    out = "f32" if y_f32 else dtype
    square = S.f64(v) ** 2
    rel = 2.0 ** -17 + (2.0 * square + 32.0) * 2.0 ** -24 if out != "f32" else (1.3 * (square + 1.0) + 18.0) * 2.0 ** -24
    tol = half_spacing(ref * (1.0 + rel), out) + rel * np.abs(ref) + 2.0 ** -120
    worst = np.abs(got - ref) / tol
    at = np.unravel_index(np.argmax(worst), worst.shape)
    assert (worst <= 1.0).all(), "%d values beyond tolerance, worst %.3g times it at %r" % (
        (worst > 1.0).any(0).sum(), worst[at], float(S.f64(v)[at[1]]))


def test_gelu_of_infinities_and_nan(S):
    import torch
    for dtype in DTYPES:
        for m in (1, 70):
            x = torch.ones((m, 8), device="cuda", dtype=S.TYPES[dtype][1])
            w = torch.zeros((3, 8), device="cuda", dtype=x.dtype)
            w[0, 3], w[1, 3] = float("inf"), float("nan")
            y = torch.empty((m, 3), device="cuda", dtype=x.dtype)
            S.B.linear_fwd(S.B.make_linear_desc(m, 3, 8, dtype=S.TYPES[dtype][0], act=S.B.ACT_GELU), x, w, y)
            got = S.f64(y)
            assert np.isposinf(got[:, 0]).all() and np.isnan(got[:, 1]).all() and (got[:, 2] == 0.0).all(), (dtype, m)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("step", [False, True])
def test_softplus_holds_its_digits_for_all_sizes(S, dtype, step):
    # One token of x = 1 and B = 1 from no state leaves delta = log(1 + exp(v)) itself, v from dt_bias.  In units of 2^-24: the
    # exponential 3, its logarithm 3, the quotient that makes up for rounding 1 + e 6, the addition 1, the state (a sum of
    # three parts) 2: 15, and 20 are allowed.  Exponentials below 2^-125 may come out as zero.
    import torch
    B, (code, ty) = S.B, S.TYPES[dtype][:2]
    v = np.concatenate([-np.geomspace(1e-7, 100.0, 3000), np.geomspace(1e-7, 100.0, 1000), [0.0]]).astype(np.float32)
    heads = len(v)
    row = lambda n, value: torch.full((1, n), value, device="cuda", dtype=ty)
    x, dt, b, y = row(heads, 1.0), row(heads, 0.0), row(1, 1.0), row(heads, 0.0)
    a, out = torch.full((heads,), -1.0, device="cuda"), torch.empty((1, heads, 1, 1), device="cuda")
    desc = B.make_ssm_desc(1, 1, heads, 1, 1, 1, slots=1, dtype=code)
    call = B.ssm_scan_step if step else B.ssm_scan_fwd
    call(desc, x, dt, a, b, b, y, dt_bias=torch.from_numpy(v).cuda(), state_out=out)
    ref = np.logaddexp(0.0, v.astype(np.float64))
    err = np.abs(S.f64(out).reshape(-1) - ref) / (20.0 * 2.0 ** -24 * ref + 2.0 ** -125)
    at = int(np.argmax(err))
    assert (err <= 1.0).all(), "%d values beyond tolerance, worst %.3g times it at %r" % ((err > 1.0).sum(), err[at], v[at])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("step", [False, True])
def test_softplus_of_infinities_and_nan(S, dtype, step):
    import torch
    B, (code, ty) = S.B, S.TYPES[dtype][:2]
    v = torch.tensor([float("-inf"), float("nan"), -200.0, 200.0], device="cuda")
    row = lambda n, value: torch.full((1, n), value, device="cuda", dtype=ty)
    y, out = row(4, 0.0), torch.empty((1, 4, 1, 1), device="cuda")
    call = B.ssm_scan_step if step else B.ssm_scan_fwd
    call(B.make_ssm_desc(1, 1, 4, 1, 1, 1, slots=1, dtype=code), row(4, 1.0), row(4, 0.0), torch.full((4,), -1.0, device="cuda"),
         row(1, 1.0), row(1, 1.0), y, dt_bias=v, state_out=out)
    got = S.f64(out).reshape(-1)
    assert got[0] == 0.0 and np.isnan(got[1]) and got[2] == 0.0 and got[3] == 200.0


@pytest.mark.parametrize("dtype,y_f32", [("bf16", False), ("f16", False), ("f32", False), ("f16", True)])
@pytest.mark.parametrize("m", [1, 70])
def test_silu_holds_its_digits(S, dtype, y_f32, m):
    # v / (1 + exp(-v)): the exponent's error is (2 |v| + 1) 2^-24 of the exponential below zero in 16 bits (two roundings of
    # v log2(e) and of log2(e) itself), the rest 8 2^-24.  In 32 bits the exponential is good to four units whatever |v| is.
    # Below -88 results may be zero: 88 exp(-88) is 2^-120.
    import torch
    if dtype == "f32":
        v = torch.from_numpy(np.concatenate([-np.geomspace(1e-6, 100.0, 5001), np.geomspace(1e-6, 100.0, 3001)]).astype(np.float32))
    else:
        v = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(S.TYPES[dtype][1])
        size = v.float().abs()
        v = v[torch.isfinite(v.float()) & (size < 100.0) & ((size > 2.0 ** -100) | (v == 0))]
    x = S.f64(v)
    ref = x / (1.0 + np.exp(-x))
    got = of_every_value(S, v, dtype, "silu", y_f32, m)
    out = "f32" if y_f32 else dtype
    rel = ((0.0 if out == "f32" else 2.0 * np.abs(x)) + 8.0) * 2.0 ** -24
    tol = half_spacing(ref * (1.0 + rel), out) + rel * np.abs(ref) + 2.0 ** -119
    worst = np.abs(got - ref) / tol
    at = np.unravel_index(np.argmax(worst), worst.shape)
    assert (worst <= 1.0).all(), "%d values beyond tolerance, worst %.3g times it at %r" % (
        (worst > 1.0).any(0).sum(), worst[at], float(x[at[1]]))
