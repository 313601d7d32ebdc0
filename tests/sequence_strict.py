"""A comparison for the sequence layers' results that infinities and NaN do not pass: sequence_case.close compares sizes
of errors alone, and no error that is NaN is larger than a tolerance."""
import numpy as np

from tests.sequence_case import TYPES, f64


def kind(v):
    """0 where v is finite, 1 and -1 where it is an infinity, 2 where it is NaN."""
    with np.errstate(invalid="ignore"):
        return np.where(np.isnan(v), 2, np.where(np.isinf(v), np.sign(v), 0)).astype(int)


def close(got, ref, d, dtype, share, what):
    """`got` is finite exactly where `ref` is, and within the tolerance there."""
    u, tiny = TYPES[dtype][2:]
    got = f64(got)
    ok = np.isfinite(ref)
    stray = np.isfinite(got) != ok
    assert not stray.any(), "%s: %d of %d finite where they should not be, or not where they should" % (
        what, stray.sum(), stray.size)
    err = np.abs(got[ok] - ref[ok])
    tol = (u * np.abs(ref) + tiny + share * d)[ok]
    over = ~(err <= tol)
    assert not over.any(), "%s: %d of %d beyond tolerance, worst %.3g times it" % (
        what, over.sum(), over.size, (err / np.maximum(tol, 1e-300)).max())
