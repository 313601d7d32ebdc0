"""CPU tests of what the layer of experts refuses, and of its weights in 8 bits."""
import numpy as np
import pytest
import torch

from oracle import around as oa
from paper_2008_04567_amd.experts import Experts, weights_in_8
from paper_2008_04567_amd.mixer import Mixer


@pytest.fixture(scope="module")
def layer():
    m = Experts(32, 48, 4, 2, device="cpu")
    return m, m.plan(5)


@pytest.mark.parametrize("h", [torch.zeros((4, 32), dtype=torch.bfloat16), torch.zeros((5, 33), dtype=torch.bfloat16), torch.zeros((5, 32)),
                               torch.zeros(160, dtype=torch.bfloat16), torch.zeros((32, 5), dtype=torch.bfloat16).T,
                               torch.zeros((1, 32), dtype=torch.bfloat16).expand(5, 32)])
def test_run_refuses_rows(layer, h):
    with pytest.raises(ValueError, match="h"):
        layer[0].run(layer[1], h, stream=0)


def test_run_refuses_the_cpu_and_plans_of_others(layer):
    m, p = layer
    with pytest.raises(ValueError, match="GPU"):
        m.run(p, torch.zeros((5, 32), dtype=torch.bfloat16), stream=0)
    with pytest.raises(ValueError, match="plan"):
        Experts(32, 48, 4, 2, device="cpu").run(p, torch.zeros((5, 32), dtype=torch.bfloat16), stream=0)


def test_weights_in_8_are_off_by_half_a_step_at_most():
    w = torch.randn((2, 2, 150, 200), generator=torch.Generator().manual_seed(1))
    q, s = weights_in_8(w)
    assert q.shape == (2, 2, 150, 208) and s.shape == (2, 2, 2, 2) and not q[..., 200:].float().any()
    for e in range(2):
        for h in range(2):
            scale = oa.spread(s[e, h].double().numpy(), (150, 200), 128)
            v = w[e, h].double().numpy()
            err = np.abs(q[e, h, :, :200].double().numpy() * scale - v)
            assert (err <= 2.0 ** -4 * np.abs(v) * (1 + 1e-6) + 2.0 ** -10 * scale).all()


def test_a_mixer_without_norms_has_the_buffers_it_had():
    m = Mixer(32, 2, 8, 1, 16, slots=4, device="cpu")
    assert not m.norm and m.plan(3, 10, 6).normed is None
