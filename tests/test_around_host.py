"""CPU tests of what stands around a mixer layer: refusals, descriptors and the 64-bit definitions themselves."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import around as oa
from paper_2008_04567_amd import binding as B
from tests.test_sequence_host import FAKE, ROOT, status


def test_descriptor_layouts_match_the_header(tmp_path):
    names = {"wpk_rms_norm_desc": B.RmsNormDesc, "wpk_quantize_desc": B.QuantizeDesc, "wpk_linear_q8_desc": B.LinearQ8Desc,
             "wpk_grouped_linear_desc": B.GroupedLinearDesc, "wpk_route_desc": B.RouteDesc}
    lines, want = [], []
    for c, py in names.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % c)
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (c, f[0]) for f in py._fields_]
        want += [ctypes.sizeof(py)] + [getattr(py, f[0]).offset for f in py._fields_]
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "wpk.h"\nint main(void){%s return 0;}' % "\n".join(lines))
    subprocess.check_call(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    assert [int(v) for v in subprocess.check_output([str(exe)]).split()] == want


NORM = dict(rows=4, width=256)
BIG = 1 << 30


def norm(desc, x=FAKE, gain=FAKE, **kw):
    return status(B.rms_norm_fwd, desc, x, gain, **dict(dict(y=FAKE, stream=0), **kw))


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), B.E_BAD_DESC), (dict(width=0), B.E_BAD_DESC), (dict(groups=0), B.E_BAD_DESC), (dict(groups=3), B.E_BAD_DESC),
    (dict(parts=0), B.E_BAD_DESC), (dict(x_rows=-1), B.E_BAD_DESC), (dict(eps=-1.0), B.E_BAD_DESC), (dict(eps=float("nan")), B.E_BAD_DESC),
    (dict(width=65537), B.E_UNSUPPORTED), (dict(parts=65), B.E_UNSUPPORTED), (dict(rows=BIG + 1, x_rows=BIG), B.E_UNSUPPORTED),
    (dict(dtype=B.E4M3), B.E_UNSUPPORTED), (dict(dtype=-1), B.E_UNSUPPORTED), (dict(x_rows=3), B.E_BAD_ARG), (dict(parts=2, x_rows=7), B.E_BAD_ARG),
    (dict(q_stride=264), B.E_UNSUPPORTED), (dict(rows=BIG, x_rows=BIG, groups=2), B.E_UNSUPPORTED)] +
    [(dict([(s, 255)]), B.E_BAD_DESC) for s in ("x_stride", "residual_stride", "h_stride", "y_stride", "q_stride")] +
    [(dict([(s, BIG)]), B.E_UNSUPPORTED) for s in ("x_stride", "residual_stride", "h_stride", "y_stride", "q_stride", "scale_stride")] +
    [(dict(scale_stride=1), B.E_BAD_DESC)])
def test_norm_refuses_descriptors(change, code):
    assert norm(B.make_rms_norm_desc(**dict(NORM, **change))) == code


def test_norm_refuses_pointers():
    d = B.make_rms_norm_desc(**NORM)
    assert norm(d, x=None) == B.E_NULL_PTR
    assert norm(d, y=None) == B.E_NULL_PTR
    assert norm(d, q=FAKE) == B.E_NULL_PTR                               # q without scales
    for name in ("x", "gain", "y", "residual", "h", "source", "weights"):
        assert norm(d, **{name: FAKE + 1}) == B.E_BAD_ARG, name
    assert norm(d, q=FAKE + 8, scales=FAKE) == B.E_BAD_ARG
    assert norm(d, q=FAKE, scales=FAKE + 2) == B.E_BAD_ARG
    assert norm(B.make_rms_norm_desc(4, 256, groups=4), q=FAKE, scales=FAKE) == B.E_UNSUPPORTED     # 64 columns a group
    assert norm(B.make_rms_norm_desc(4, 256, x_rows=0), source=FAKE) == B.E_BAD_ARG
    assert B.lib().wpk_rms_norm_fwd(None, *[FAKE] * 10) == B.E_NULL_PTR
    assert norm(B.make_rms_norm_desc(0, 256), x=None, y=None) == B.OK    # nothing to do


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), B.E_BAD_DESC), (dict(width=0), B.E_BAD_DESC), (dict(x_stride=255), B.E_BAD_DESC), (dict(q_stride=240), B.E_BAD_DESC),
    (dict(scale_stride=1), B.E_BAD_DESC), (dict(dtype=B.E4M3), B.E_UNSUPPORTED), (dict(q_stride=260), B.E_UNSUPPORTED),
    (dict(rows=BIG + 1), B.E_UNSUPPORTED), (dict(x_stride=BIG), B.E_UNSUPPORTED), (dict(q_stride=BIG), B.E_UNSUPPORTED),
    (dict(scale_stride=BIG), B.E_UNSUPPORTED)])
def test_quantize_refuses_descriptors(change, code):
    assert status(B.quantize_fwd, B.make_quantize_desc(**dict(dict(rows=4, width=256), **change)), FAKE, FAKE, FAKE) == code


def test_quantize_refuses_pointers():
    d = B.make_quantize_desc(4, 256)
    for i in range(3):
        assert status(B.quantize_fwd, d, *[None if j == i else FAKE for j in range(3)]) == B.E_NULL_PTR
    for p in ((FAKE + 1, FAKE, FAKE), (FAKE, FAKE + 8, FAKE), (FAKE, FAKE, FAKE + 2)):
        assert status(B.quantize_fwd, d, *p) == B.E_BAD_ARG
    d.reserved = 1
    assert status(B.quantize_fwd, d, FAKE, FAKE, FAKE) == B.E_UNSUPPORTED
    assert B.lib().wpk_quantize_fwd(None, *[FAKE] * 4) == B.E_NULL_PTR
    assert status(B.quantize_fwd, B.make_quantize_desc(0, 256), None, None, None) == B.OK


Q8 = dict(m=4, n=8, k=32)


@pytest.mark.parametrize("change,code", [
    (dict(m=-1), B.E_BAD_DESC), (dict(n=0), B.E_BAD_DESC), (dict(k=0), B.E_BAD_DESC), (dict(x_stride=16), B.E_BAD_DESC),
    (dict(w_stride=16), B.E_BAD_DESC), (dict(y_stride=7), B.E_BAD_DESC), (dict(residual_stride=7), B.E_BAD_DESC),
    (dict(k=129, x_scale_stride=1), B.E_BAD_DESC), (dict(k=129, w_scale_stride=1), B.E_BAD_DESC), (dict(dtype=B.E4M3), B.E_UNSUPPORTED),
    (dict(act=4), B.E_UNSUPPORTED), (dict(act=-1), B.E_UNSUPPORTED), (dict(x_stride=40), B.E_UNSUPPORTED), (dict(w_stride=40), B.E_UNSUPPORTED)] +
    [(dict([(s, 1 << 20)]), B.E_UNSUPPORTED) for s in ("x_stride", "w_stride", "y_stride", "residual_stride", "x_scale_stride", "w_scale_stride")])
def test_linear_q8_refuses_descriptors(change, code):
    d = B.make_linear_q8_desc(**dict(Q8, **change))
    assert status(B.linear_q8_workspace, d) == code
    assert status(B.linear_q8_fwd, d, *[FAKE] * 5, workspace=FAKE) == code


def test_linear_q8_refuses_pointers():
    d = B.make_linear_q8_desc(**Q8)
    for i in range(5):
        assert status(B.linear_q8_fwd, d, *[None if j == i else FAKE for j in range(5)], workspace=FAKE) == B.E_NULL_PTR
        off = 8 if i in (0, 2) else 2 if i < 4 else 1
        assert status(B.linear_q8_fwd, d, *[FAKE + off if j == i else FAKE for j in range(5)], workspace=FAKE) == B.E_BAD_ARG
    for name in ("bias", "residual", "workspace"):
        assert status(B.linear_q8_fwd, d, *[FAKE] * 5, **{name: FAKE + 1}) == B.E_BAD_ARG
    assert B.lib().wpk_linear_q8_fwd(None, *[FAKE] * 9) == B.E_NULL_PTR
    assert B.lib().wpk_linear_q8_workspace_bytes(None) == B.E_NULL_PTR
    assert status(B.linear_q8_fwd, B.make_linear_q8_desc(0, 8, 32), *[None] * 5) == B.OK
    long = B.make_linear_q8_desc(2, 16, 65536)                            # a reduction that is cut has to have room
    assert B.linear_q8_workspace(long) == 0 or status(B.linear_q8_fwd, long, *[FAKE] * 5) == B.E_NULL_PTR


GROUPED = dict(groups=3, rows=10, n=8, k=32)


@pytest.mark.parametrize("change,code", [
    (dict(groups=0), B.E_BAD_DESC), (dict(rows=-1), B.E_BAD_DESC), (dict(n=0), B.E_BAD_DESC), (dict(k=0), B.E_BAD_DESC),
    (dict(x_rows=-1), B.E_BAD_DESC), (dict(x_stride=31), B.E_BAD_DESC), (dict(w_stride=31), B.E_BAD_DESC), (dict(y_stride=7), B.E_BAD_DESC),
    (dict(w_group_stride=255), B.E_BAD_DESC), (dict(gated=True, w_group_stride=511), B.E_BAD_DESC), (dict(groups=4097), B.E_UNSUPPORTED),
    (dict(dtype=4), B.E_UNSUPPORTED), (dict(dtype=B.BF16, y_dtype=B.F16), B.E_UNSUPPORTED), (dict(dtype=B.E4M3, y_dtype=B.E4M3), B.E_UNSUPPORTED),
    (dict(act=4), B.E_UNSUPPORTED), (dict(x_stride=1 << 20), B.E_UNSUPPORTED), (dict(w_stride=1 << 20), B.E_UNSUPPORTED),
    (dict(y_stride=1 << 20), B.E_UNSUPPORTED), (dict(w_group_stride=1 << 40), B.E_UNSUPPORTED),
    (dict(dtype=B.E4M3, x_stride=40), B.E_UNSUPPORTED), (dict(dtype=B.E4M3, w_stride=40), B.E_UNSUPPORTED),
    (dict(dtype=B.E4M3, w_group_stride=264), B.E_UNSUPPORTED), (dict(dtype=B.E4M3, k=200, x_scale_stride=1), B.E_BAD_DESC),
    (dict(dtype=B.E4M3, k=200, w_scale_stride=1), B.E_BAD_DESC), (dict(dtype=B.E4M3, k=200, w_scale_group_stride=1), B.E_BAD_DESC),
    (dict(dtype=B.E4M3, gated=True, w_scale_group_stride=1), B.E_BAD_DESC)])
def test_grouped_refuses_descriptors(change, code):
    d = B.make_grouped_linear_desc(**dict(GROUPED, **change))
    assert status(B.grouped_linear_workspace, d) == code
    kw = dict(x_scales=FAKE, w_scales=FAKE) if d.dtype == B.E4M3 else {}
    assert status(B.grouped_linear_fwd, d, FAKE, FAKE, FAKE, FAKE, **kw) == code


def test_grouped_refuses_pointers():
    call = lambda d, x=FAKE, w=FAKE, starts=FAKE, y=FAKE, **kw: status(B.grouped_linear_fwd, d, x, w, starts, y, **kw)
    d, e = B.make_grouped_linear_desc(**GROUPED), B.make_grouped_linear_desc(dtype=B.E4M3, **GROUPED)
    for name in ("x", "w", "y"):
        assert call(d, **{name: None}) == B.E_NULL_PTR
        assert call(d, **{name: FAKE + 1}) == B.E_BAD_ARG
    assert call(d, starts=None) == B.E_BAD_ARG
    for kw in (dict(starts=FAKE + 2), dict(source=FAKE + 2), dict(workspace=FAKE + 8), dict(x_scales=FAKE), dict(w_scales=FAKE)):
        assert call(d, **kw) == B.E_BAD_ARG
    assert call(e) == B.E_NULL_PTR
    assert call(e, x_scales=FAKE) == B.E_NULL_PTR
    assert call(e, x=FAKE + 8, x_scales=FAKE, w_scales=FAKE) == B.E_BAD_ARG
    assert call(e, x_scales=FAKE + 2, w_scales=FAKE) == B.E_BAD_ARG
    assert call(B.make_grouped_linear_desc(**dict(GROUPED, x_rows=9))) == B.E_BAD_ARG          # fewer rows than y, none looked up
    assert call(B.make_grouped_linear_desc(**dict(GROUPED, x_rows=0)), source=FAKE) == B.E_BAD_ARG
    assert call(B.make_grouped_linear_desc(**dict(GROUPED, rows=0)), x=None, w=None, starts=None, y=None) == B.OK
    for name in ("gated", "reserved"):
        d = B.make_grouped_linear_desc(**GROUPED)
        setattr(d, name, 2)
        assert call(d) == B.E_UNSUPPORTED
    assert B.lib().wpk_grouped_linear_fwd(None, *[FAKE] * 9) == B.E_NULL_PTR
    assert B.lib().wpk_grouped_linear_workspace_bytes(None) == B.E_NULL_PTR


ROUTE = dict(tokens=4, experts=8, k=2)


@pytest.mark.parametrize("change,code", [
    (dict(tokens=-1), B.E_BAD_DESC), (dict(experts=0), B.E_BAD_DESC), (dict(k=0), B.E_BAD_DESC), (dict(k=9), B.E_BAD_DESC),
    (dict(logits_stride=7), B.E_BAD_DESC), (dict(experts=1025), B.E_UNSUPPORTED), (dict(experts=100, k=33), B.E_UNSUPPORTED),
    (dict(dtype=B.E4M3), B.E_UNSUPPORTED), (dict(tokens=BIG), B.E_UNSUPPORTED), (dict(logits_stride=BIG), B.E_UNSUPPORTED)])
def test_route_refuses_descriptors(change, code):
    d = B.make_route_desc(**dict(ROUTE, **change))
    assert status(B.route_workspace, d) == code
    assert status(B.route_fwd, d, *[FAKE] * 6, workspace=FAKE) == code


def test_route_refuses_pointers():
    d = B.make_route_desc(**ROUTE)
    for i in range(6):
        assert status(B.route_fwd, d, *[None if j == i else FAKE for j in range(6)], workspace=FAKE) == B.E_NULL_PTR
        assert status(B.route_fwd, d, *[FAKE + 1 if j == i else FAKE for j in range(6)], workspace=FAKE) == B.E_BAD_ARG
    assert status(B.route_fwd, d, *[FAKE] * 6, workspace=FAKE + 8) == B.E_BAD_ARG
    many = B.make_route_desc(5000, 8, 2)
    assert B.route_workspace(many) > 0
    assert status(B.route_fwd, many, *[FAKE] * 6) == B.E_NULL_PTR
    d.normalize = 2
    assert status(B.route_fwd, d, *[FAKE] * 6) == B.E_UNSUPPORTED
    assert status(B.route_fwd, B.make_route_desc(0, 8, 2), None, None, None) == B.OK
    assert B.lib().wpk_route_fwd(None, *[FAKE] * 8) == B.E_NULL_PTR
    assert B.lib().wpk_route_workspace_bytes(None) == B.E_NULL_PTR


# ---- the definitions ----------------------------------------------------------------------------------
def test_e4m3_rounding_is_nearest_and_even():
    v = np.sort(oa.e4m3_values()[np.isfinite(oa.e4m3_values())])
    v = np.unique(v)
    assert np.array_equal(oa.round_e4m3(v), v) and v.max() == 448.0
    mid = (v[1:] + v[:-1]) / 2
    got = oa.round_e4m3(mid)
    codes = {x: c for c, x in enumerate(oa.e4m3_values()[:127])}
    assert all(codes[abs(g)] % 2 == 0 for g in got)
    assert np.array_equal(oa.round_e4m3(mid * (1 + 1e-9)), np.where(mid > 0, v[1:], v[:-1]))
    import torch
    r = np.random.default_rng(1).standard_normal(20000).astype(np.float32) * np.exp(np.random.default_rng(2).uniform(-8, 5, 20000)).astype(np.float32)
    r = np.clip(r, -448, 448)
    assert np.array_equal(torch.from_numpy(r).to(torch.float8_e4m3fn).float().numpy(), oa.round_e4m3(r))


def test_quantize_definition():
    x = np.random.default_rng(1).standard_normal((5, 300)).astype(np.float32)
    q, s = oa.quantize(x)
    back = q * oa.spread(s, x.shape)
    assert np.abs(back - x).max() <= (2.0 ** -4 * np.abs(x) + 2.0 ** -10 * oa.spread(s, x.shape)).max()
    assert (np.abs(back - x) <= 2.0 ** -4 * np.abs(x) * (1 + 1e-6) + 2.0 ** -10 * oa.spread(s, x.shape)).all()
    q, s = oa.quantize(np.array([[np.nan, 1.0, np.inf, 2.0] + [0.0] * 124], np.float32))
    assert np.isinf(s[0, 0]) and np.isnan(q[0, 0]) and np.isnan(q[0, 2]) and q[0, 1] == 0
    q, s = oa.quantize(np.array([[np.nan, 1.0]], np.float32))
    assert np.isnan(q[0, 0]) and q[0, 1] == 448.0


def test_route_definition():
    l = np.array([[1.0, 3.0, 3.0, np.nan], [-np.inf] * 4, [0.0, -0.0, 1.0, 0.0]])
    ids, w, starts, source, place = oa.route(l, 3)
    assert ids.tolist() == [[1, 2, 0], [0, 1, 2], [2, 0, 1]]
    assert np.allclose(w[0].sum(), 1) and (w[1] == 0).all()
    assert starts.tolist() == [0, 3, 6, 9, 9]
    assert source.tolist() == [0, 1, 2, 0, 1, 2, 0, 1, 2]
    assert all(source[place[t, j]] == t and starts[ids[t, j]] <= place[t, j] < starts[ids[t, j] + 1] for t in range(3) for j in range(3))
    ids, w, _, _, _ = oa.route(np.array([[0.0, 1.0]]), 1, normalize=False, scale=2.0)
    assert np.allclose(w, 2 * np.exp(1) / (1 + np.exp(1)))
