"""GPU tests of calls on another stream than the one that their inputs are made on: the helpers make everything first, then the
stream waits for it, then the call goes out; results are the definition's."""
import pytest

from tests import parity as PT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    PT.torch_dev()
    from tests import around_case
    return around_case


CALLS = [("rms_norm_fwd", lambda A, s: A.run_norm(70, 1500, "bf16", parts=3, source="random", weights="random", q=True, stream=s)),
         ("linear_q8_fwd", lambda A, s: A.run_linear_q8(100, 64, 4096, "bf16", stream=s)),            # (its reduction is cut)
         ("grouped_linear_fwd", lambda A, s: A.run_grouped([60, 0, 70], 200, 300, "e4m3", gated=True, act="silu", gather=True, stream=s)),
         ("grouped_linear_fwd", lambda A, s: A.run_grouped([60, 0, 70], 200, 300, "f32", stream=s)),
         ("route_fwd", lambda A, s: A.run_route(A.Rng(1).normal((3000, 60)), 6, "f32", stream=s))]


@pytest.mark.parametrize("entry,call", CALLS, ids=["norm", "linear_q8", "grouped_e4m3", "grouped_f32", "route"])
def test_calls_on_another_stream_wait_for_their_inputs(A, monkeypatch, entry, call):
    import torch
    log = []

    class Side(torch.cuda.Stream):
        def wait_stream(self, other):
            assert other == torch.cuda.current_stream()
            log.append("wait")
            super().wait_stream(other)

    def noted(name, fn):
        def run(*a, **kw):
            log.append(name)
            return fn(*a, **kw)
        return run

    monkeypatch.setattr(A, "workspace", noted("input", A.workspace))
    monkeypatch.setattr(A, "i32", noted("input", A.i32))
    monkeypatch.setattr(A.B, entry, noted("call", getattr(A.B, entry)))
    for _ in range(3):
        log.clear()
        call(A, Side())
        assert log[-2:] == ["wait", "call"] and log.count("call") == 1, log
