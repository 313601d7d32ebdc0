"""GPU tests of the layer of experts, and of it between mixer layers with norms, as a program would run them."""
import numpy as np
import pytest

from tests import parity as PT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    PT.torch_dev()
    from tests import around_case
    return around_case


def spread_weight(A, q, s):
    """The numbers that 8-bit weights [experts][halves][n][k] stand for."""
    import torch
    v = A.oa.e4m3_values()[q.view(torch.uint8).cpu().numpy()]
    return np.stack([np.stack([v[e, h] * A.oa.spread(A.f64(s[e, h]), v.shape[2:], 128) for h in range(v.shape[1])])
                     for e in range(v.shape[0])])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens", [1, 9, 150])
def test_layer_is_its_formula(A, dtype, eight, tokens):
    from paper_2008_04567_amd.experts import Experts
    width, inner, k = 144, 80, 3
    m = Experts(width, inner, 10, k, eight=eight, dtype=A.TYPES[dtype][1], seed=2)
    p, h = m.plan(tokens), A.Rng(tokens).normal((tokens, width), dtype)
    out = A.f64(m.run(p, h))
    hv, x = A.f64(h), A.f64(p.x)
    up = spread_weight(A, m.w_up, m.s_up)[..., :width] if eight else A.f64(m.w_up)
    down = spread_weight(A, m.w_down, m.s_down)[..., :inner] if eight else A.f64(m.w_down)
    import torch
    x_in = A.numbers(p.x8.view(torch.uint8)) * A.oa.spread(A.f64(p.x_scales), p.x8.shape) if eight else x
    ids, weights = p.ids.cpu().numpy(), A.f64(p.weights)
    logits = x @ A.f64(m.w_route).T
    assert np.abs(A.f64(p.logits) - logits).max() <= 2.0 ** -18 * np.abs(x).max() * width ** 0.5
    assert np.array_equal(ids, A.oa.route(A.f64(p.logits), k)[0])
    want = hv.copy()
    for t in range(tokens):
        for j in range(k):
            g = up[ids[t, j]] @ x_in[t, :width]
            want[t] += weights[t, j] * (down[ids[t, j], 0] @ (A.osq.act(g[0], "silu") * g[1]))
    # each of three roundings (inner rows, outer rows, out) is off by half a step; 8 bits add 2^-4 of each inner value
    u = A.TYPES[dtype][2]
    err = np.linalg.norm(out - want) / np.linalg.norm(want)
    assert err <= 3 * u + (2.0 ** -4 if eight else 0.0) + 2.0 ** -18, err


@pytest.mark.parametrize("eight", [False, True])
def test_no_tokens(A, eight):
    """A batch that happens to be empty: no rows of any expert, and the next call is none the worse."""
    import torch
    from paper_2008_04567_amd.experts import Experts
    m = Experts(96, 64, 6, 2, eight=eight, seed=1)
    h = A.Rng(1).normal((3, 96), "bf16")
    p, none = m.plan(3), m.plan(0)
    first = m.run(p, h).clone()
    assert tuple(m.run(none, h[:0]).shape) == (0, 96) and none.starts.tolist() == [0] * 7
    assert torch.equal(first, m.run(p, h))


def test_another_current_device_is_refused(A, monkeypatch):
    import torch
    from paper_2008_04567_amd.experts import Experts
    m = Experts(96, 64, 6, 2, seed=1)
    p, h = m.plan(3), A.Rng(1).normal((3, 96), "bf16")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: h.device.index + 1)
    with pytest.raises(ValueError, match="current device"):
        m.run(p, h)


def test_rows_may_be_slices_and_calls_repeat(A):
    import torch
    from paper_2008_04567_amd.experts import Experts
    m = Experts(96, 64, 6, 2, seed=1)
    h, wide = A.Rng(1).normal((40, 96), "bf16"), A.Rng(2).normal((40, 200), "bf16")
    wide[:, 8:104] = h
    p = m.plan(40)
    first = m.run(p, h).clone()
    assert torch.equal(first, m.run(p, wide[:, 8:104])) and torch.equal(first, m.run(p, h))


@pytest.mark.parametrize("eight", [False, True])
def test_mixer_and_experts_prompts_then_tokens(A, eight):
    """Two layers of each kind: prompts at once, and the same tokens one after another through the forms for single tokens."""
    import torch
    from paper_2008_04567_amd.experts import Experts
    from paper_2008_04567_amd.mixer import Mixer
    width, requests, length = 128, 3, 12
    rows = A.Rng(5).normal((requests, length, width), "bf16")
    out = []
    for one_by_one in (False, True):
        mixers = [Mixer(width, 4, 32, 2, 16, slots=requests, seed=s, norm=True) for s in (1, 2)]
        experts = [Experts(width, 96, 8, 2, eight=eight, seed=s) for s in (3, 4)]
        slots = A.i32(list(range(requests)))
        if one_by_one:
            plans = [m.plan(requests, requests, 1) for m in mixers], [e.plan(requests) for e in experts]
            got = []
            for t in range(length):
                h = rows[:, t].contiguous()
                for m, e, pm, pe in zip(mixers, experts, *plans):
                    h = e.run(pe, m.step(pm, h, slots))
                got.append(h.clone())
            out.append(torch.stack(got, 1))
        else:
            plans = [m.plan(requests, requests * length, length) for m in mixers], [e.plan(requests * length) for e in experts]
            h = rows.reshape(-1, width).contiguous()
            for m, e, pm, pe in zip(mixers, experts, *plans):
                h = e.run(pe, m.prompt(pm, h, A.i32([i * length for i in range(requests + 1)]), slots))
            out.append(h.view(requests, length, width))
    a, b = [A.f64(t) for t in out]
    assert np.isfinite(a).all()
    # four layers, a few roundings of 2^-8 each, that a token's experts are rarely chosen otherwise by
    far = np.linalg.norm(a - b, axis=2) / np.linalg.norm(a, axis=2)
    assert np.median(far) <= 16 * 2.0 ** -8 and (far <= 0.25).mean() >= 0.9, far
