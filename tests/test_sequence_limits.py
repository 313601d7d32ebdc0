"""CPU tests of the limits that include/wpk.h gives for the sequence layers' sizes."""
import pytest

from paper_2008_04567_amd import binding as B
from tests.test_sequence_host import CONV, FAKE, LINEAR, SSM, status


@pytest.mark.parametrize("name", ["x_stride", "w_stride", "y_stride", "residual_stride"])
def test_linear_strides(name):
    assert status(B.linear_workspace, B.make_linear_desc(**LINEAR, **{name: (1 << 20) - 1})) == B.OK
    for stride in (1 << 20, 1 << 33):
        desc = B.make_linear_desc(**LINEAR, **{name: stride})
        assert status(B.linear_workspace, desc) == B.E_UNSUPPORTED
        assert status(B.linear_fwd, desc, FAKE, FAKE, FAKE) == B.E_UNSUPPORTED


@pytest.mark.parametrize("name", ["x_stride", "y_stride"])
def test_conv_strides(name):
    desc = B.make_causal_conv_desc(**CONV, **{name: 1 << 40})
    assert status(B.causal_conv1d_fwd, desc, FAKE, FAKE, FAKE) == B.E_UNSUPPORTED
    desc = B.make_causal_conv_desc(**CONV, **{name: (1 << 40) - 1})
    assert status(B.causal_conv1d_fwd, desc, None, FAKE, FAKE) == B.E_NULL_PTR          # past the descriptor's checks


@pytest.mark.parametrize("name", ["x_stride", "z_stride", "y_stride", "b_stride", "c_stride", "dt_stride"])
def test_ssm_strides(name):
    assert status(B.ssm_workspace, B.make_ssm_desc(**SSM, **{name: (1 << 22) - 1})) == B.OK
    assert status(B.ssm_workspace, B.make_ssm_desc(**SSM, **{name: 1 << 22})) == B.E_UNSUPPORTED


def test_requests_and_heads():
    most = 65535
    for n, code in ((most, B.E_NULL_PTR), (most + 1, B.E_UNSUPPORTED)):
        desc = B.make_causal_conv_desc(**dict(CONV, sequences=n, tokens=n, max_length=1))
        assert status(B.causal_conv1d_fwd, desc, None, FAKE, FAKE) == code
        desc = B.make_ssm_desc(**dict(SSM, sequences=n, tokens=n, max_length=1))
        assert status(B.ssm_scan_step, desc, None, *[FAKE] * 5) == code
        desc = B.make_ssm_desc(**dict(SSM, heads=n, groups=1, head_dim=1))
        assert status(B.ssm_scan_fwd, desc, None, *[FAKE] * 5, starts=FAKE, workspace=FAKE) == code
