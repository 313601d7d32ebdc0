"""GPU tests of the mixer layer on hidden states that are slices of longer rows."""
import pytest

from tests import parity as PT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_hidden_states_may_be_slices(dtype):
    import torch
    PT.torch_dev()
    from paper_2008_04567_amd.mixer import Mixer
    from tests import sequence_case as S
    ty, lengths = S.TYPES[dtype][1], [9, 70, 3]
    rows = S.Rng(1).normal((3, 2, 96), dtype)          # [request][token][width]
    prompt, wide = S.Rng(2).normal((sum(lengths), 96), dtype), S.Rng(3).normal((sum(lengths), 200), dtype)
    wide[:, 8:104] = prompt
    out = []
    for far in (False, True):
        m = Mixer(96, 4, 16, 2, 32, slots=3, dtype=ty, seed=3)
        p, one = m.plan(3, sum(lengths), max(lengths)), m.plan(3, 3, 1)
        slots = S.i32([2, 0, 1])
        out.append([m.prompt(p, wide[:, 8:104] if far else prompt, S.i32(S.starts_of(lengths)), slots).clone(),
                    m.step(one, rows[:, -1] if far else rows[:, -1].contiguous(), slots).clone(), m.conv_state, m.scan_state])
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_requests_of_one_length_in_the_pool_s_order():
    import torch
    PT.torch_dev()
    from paper_2008_04567_amd.mixer import Mixer
    from tests import sequence_case as S
    h = S.Rng(4).normal((3, 20, 96), "bf16")
    out = []
    for plain in (False, True):
        m = Mixer(96, 4, 16, 2, 32, slots=3, seed=3)
        p = m.plan(3, 60, 20)
        if plain:
            y = m.prompt(p, h, None, None)
        else:
            y = m.prompt(p, h.view(60, 96), S.i32([0, 20, 40, 60]), S.i32([0, 1, 2]))
        out.append([y.clone(), m.conv_state, m.scan_state])
    assert all(torch.equal(a, b) for a, b in zip(*out))
