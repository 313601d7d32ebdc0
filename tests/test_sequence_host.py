"""CPU tests of the sequence layers: refusals, descriptors and the 64-bit definitions themselves."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import sequence as osq
from paper_2008_04567_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20          # an aligned address that no refused call may touch


def status(fn, *a, **kw):
    try:
        fn(*a, **kw)
    except B.WpkError as e:
        return e.status
    return B.OK


def test_descriptor_layouts_match_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    names = {"wpk_linear_desc": B.LinearDesc, "wpk_causal_conv_desc": B.CausalConvDesc, "wpk_ssm_desc": B.SsmDesc}
    lines = []
    for c, py in names.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % c)
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (c, f[0]) for f in py._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "wpk.h"\nint main(void){%s return 0;}' % "\n".join(lines))
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    want = []
    for py in names.values():
        want.append(ctypes.sizeof(py))
        want += [getattr(py, f[0]).offset for f in py._fields_]
    assert got == want


LINEAR = dict(m=4, n=8, k=16)


@pytest.mark.parametrize("change,code", [
    (dict(m=-1), B.E_BAD_DESC), (dict(n=0), B.E_BAD_DESC), (dict(k=0), B.E_BAD_DESC), (dict(x_stride=15), B.E_BAD_DESC),
    (dict(w_stride=15), B.E_BAD_DESC), (dict(y_stride=7), B.E_BAD_DESC), (dict(residual_stride=7), B.E_BAD_DESC),
    (dict(dtype=3), B.E_UNSUPPORTED), (dict(dtype=B.BF16, y_dtype=B.F16), B.E_UNSUPPORTED), (dict(act=4), B.E_UNSUPPORTED),
    (dict(act=-1), B.E_UNSUPPORTED), (dict(x_stride=1 << 20), B.E_UNSUPPORTED)])
def test_linear_refuses_descriptors(change, code):
    desc = B.make_linear_desc(**dict(LINEAR, **change))
    assert status(B.linear_workspace, desc) == code
    assert status(B.linear_fwd, desc, FAKE, FAKE, FAKE, workspace=FAKE) == code


def test_linear_refuses_pointers():
    desc = B.make_linear_desc(**LINEAR)
    assert status(B.linear_fwd, desc, None, FAKE, FAKE) == B.E_NULL_PTR
    assert status(B.linear_fwd, desc, FAKE, None, FAKE) == B.E_NULL_PTR
    assert status(B.linear_fwd, desc, FAKE, FAKE, None) == B.E_NULL_PTR
    for k in range(3):
        p = [FAKE + (1 if i == k else 0) for i in range(3)]
        assert status(B.linear_fwd, desc, *p) == B.E_BAD_ARG
    assert status(B.linear_fwd, desc, FAKE, FAKE, FAKE, bias=FAKE + 1) == B.E_BAD_ARG
    assert status(B.linear_fwd, desc, FAKE, FAKE, FAKE, residual=FAKE + 1) == B.E_BAD_ARG
    assert B.lib().wpk_linear_fwd(None, *[FAKE] * 7) == B.E_NULL_PTR
    assert B.lib().wpk_linear_workspace_bytes(None) == B.E_NULL_PTR
    assert status(B.linear_fwd, B.make_linear_desc(0, 8, 16), None, None, None) == B.OK      # nothing to do


CONV = dict(sequences=2, tokens=10, channels=8, width=4, slots=4)


@pytest.mark.parametrize("change,code", [
    (dict(sequences=-1), B.E_BAD_DESC), (dict(tokens=-1), B.E_BAD_DESC), (dict(max_length=0), B.E_BAD_DESC),
    (dict(channels=0), B.E_BAD_DESC), (dict(width=1), B.E_BAD_DESC), (dict(width=9), B.E_UNSUPPORTED),
    (dict(slots=-1), B.E_BAD_DESC), (dict(x_stride=7), B.E_BAD_DESC), (dict(y_stride=7), B.E_BAD_DESC),
    (dict(dtype=7), B.E_UNSUPPORTED), (dict(act=B.ACT_GELU), B.E_UNSUPPORTED), (dict(max_length=4), B.E_BAD_ARG)])
def test_conv_refuses_descriptors(change, code):
    desc = B.make_causal_conv_desc(**dict(CONV, **change))
    assert status(B.causal_conv1d_fwd, desc, FAKE, FAKE, FAKE) == code


def test_conv_refuses_arguments():
    desc = B.make_causal_conv_desc(**CONV)
    assert status(B.causal_conv1d_fwd, desc, None, FAKE, FAKE) == B.E_NULL_PTR
    assert status(B.causal_conv1d_fwd, desc, FAKE, None, FAKE) == B.E_NULL_PTR
    assert status(B.causal_conv1d_fwd, desc, FAKE, FAKE, None) == B.E_NULL_PTR
    assert status(B.causal_conv1d_fwd, desc, FAKE + 1, FAKE, FAKE) == B.E_BAD_ARG
    assert status(B.causal_conv1d_fwd, desc, FAKE, FAKE, FAKE, starts=FAKE + 2) == B.E_BAD_ARG
    assert status(B.causal_conv1d_step, desc, FAKE, FAKE, FAKE) == B.E_BAD_ARG               # not one token a request
    few = B.make_causal_conv_desc(**dict(CONV, slots=1))
    assert status(B.causal_conv1d_fwd, few, FAKE, FAKE, FAKE, state_in=FAKE) == B.E_BAD_ARG   # two requests, one entry
    none = B.make_causal_conv_desc(**dict(CONV, slots=0))
    assert status(B.causal_conv1d_fwd, none, FAKE, FAKE, FAKE, slot_map=FAKE, state_out=FAKE) == B.E_BAD_ARG
    assert status(B.causal_conv1d_fwd, B.make_causal_conv_desc(0, 0, 8, 4), None, None, None) == B.OK


SSM = dict(sequences=2, tokens=10, heads=4, head_dim=8, groups=2, state_dim=16, slots=4)


@pytest.mark.parametrize("change,code", [
    (dict(sequences=-1), B.E_BAD_DESC), (dict(tokens=-1), B.E_BAD_DESC), (dict(max_length=0), B.E_BAD_DESC),
    (dict(heads=0), B.E_BAD_DESC), (dict(head_dim=0), B.E_BAD_DESC), (dict(groups=3), B.E_BAD_DESC),
    (dict(groups=0), B.E_BAD_DESC), (dict(state_dim=0), B.E_BAD_DESC), (dict(head_dim=257), B.E_UNSUPPORTED),
    (dict(state_dim=257), B.E_UNSUPPORTED), (dict(x_stride=31), B.E_BAD_DESC), (dict(z_stride=31), B.E_BAD_DESC),
    (dict(y_stride=31), B.E_BAD_DESC), (dict(b_stride=31), B.E_BAD_DESC), (dict(c_stride=31), B.E_BAD_DESC),
    (dict(dt_stride=3), B.E_BAD_DESC), (dict(dtype=-1), B.E_UNSUPPORTED), (dict(b_stride=1 << 22), B.E_UNSUPPORTED)])
def test_ssm_refuses_descriptors(change, code):
    desc = B.make_ssm_desc(**dict(SSM, **change))
    assert status(B.ssm_workspace, desc) == code
    assert status(B.ssm_scan_fwd, desc, *[FAKE] * 6, workspace=FAKE) == code


def test_ssm_refuses_arguments():
    desc = B.make_ssm_desc(**SSM)
    for k in range(6):
        p = [None if i == k else FAKE for i in range(6)]
        assert status(B.ssm_scan_fwd, desc, *p, workspace=FAKE) == B.E_NULL_PTR
        p = [FAKE + (1 if i == k else 0) for i in range(6)]
        assert status(B.ssm_scan_fwd, desc, *p, workspace=FAKE) == B.E_BAD_ARG
    for name in ("d", "z", "dt_bias", "starts", "slot_map", "resume", "state_in", "state_out"):
        assert status(B.ssm_scan_fwd, desc, *[FAKE] * 6, workspace=FAKE, **{name: FAKE + 1}) == B.E_BAD_ARG, name
    assert status(B.ssm_scan_step, desc, *[FAKE] * 6) == B.E_BAD_ARG
    odd = B.make_ssm_desc(**dict(SSM, max_length=7))
    assert status(B.ssm_scan_fwd, odd, *[FAKE] * 6, workspace=FAKE) == B.E_BAD_ARG
    desc.dt_softplus = 2
    assert status(B.ssm_workspace, desc) == B.E_UNSUPPORTED
    assert status(B.ssm_scan_fwd, B.make_ssm_desc(0, 0, 4, 8, 2, 16), *[None] * 6) == B.OK


def test_definitions_agree_with_closed_forms():
    # a convolution whose only tap is the present token, and one whose only tap is the one before
    rng = np.random.default_rng(0)
    x = rng.standard_normal((6, 3))
    w = np.zeros((3, 2))
    w[:, 1] = 1.0
    y, _, left = osq.causal_conv1d(x, w, None, [(0, 4), (4, 2)], [np.zeros((1, 3))] * 2, "none")
    assert np.array_equal(y, x) and np.array_equal(left[0], x[3:4])
    y, _, _ = osq.causal_conv1d(x, w[:, ::-1], None, [(0, 4), (4, 2)], [np.ones((1, 3))] * 2, "none")
    assert np.array_equal(y, np.concatenate([np.ones((1, 3)), x[:3], np.ones((1, 3)), x[4:5]]))
    # a scan that never forgets is a running sum; one that forgets at a constant rate is a geometric series
    ones = np.ones((5, 1, 1))
    y, _, left, _ = osq.ssm_scan(ones, np.ones((5, 1)), np.zeros(1), ones, ones, [(0, 5)], [np.zeros((1, 1, 1))], softplus=False)
    assert np.allclose(y[:, 0, 0], [1, 2, 3, 4, 5]) and np.allclose(left[0], 5)
    y, _, _, _ = osq.ssm_scan(ones, np.ones((5, 1)), np.log(np.full(1, 0.5)), ones, ones, [(0, 5)], [np.full((1, 1, 1), 8.0)],
                              softplus=False)
    assert np.allclose(y[:, 0, 0], [5, 3.5, 2.75, 2.375, 2.1875])


def test_more_rows_than_numbers_hold_are_refused():
    most = 1 << 30
    for change in (dict(m=most + 1), dict(n=most + 1)):
        desc = B.make_linear_desc(**dict(LINEAR, **change))
        assert status(B.linear_workspace, desc) == B.E_UNSUPPORTED
        assert status(B.linear_fwd, desc, FAKE, FAKE, FAKE) == B.E_UNSUPPORTED
    assert status(B.linear_workspace, B.make_linear_desc(**dict(LINEAR, m=most))) == B.OK
    desc = B.make_causal_conv_desc(**dict(CONV, tokens=most + 1))
    assert status(B.causal_conv1d_fwd, desc, FAKE, FAKE, FAKE, starts=FAKE) == B.E_UNSUPPORTED
    desc = B.make_ssm_desc(**dict(SSM, tokens=most + 1))
    assert status(B.ssm_workspace, desc) == B.E_UNSUPPORTED
    assert status(B.ssm_scan_fwd, desc, *[FAKE] * 6, starts=FAKE, workspace=FAKE) == B.E_UNSUPPORTED


def test_scan_workspace_follows_tokens_not_a_loose_bound_on_lengths():
    def room(**change):
        return B.ssm_workspace(B.make_ssm_desc(**dict(dict(SSM, sequences=2, tokens=4096, dtype=B.BF16), **change)))
    assert room(max_length=2 ** 31 - 1) == room(max_length=4096)
    assert room(max_length=2 ** 31 - 1, tokens=0) == 0
