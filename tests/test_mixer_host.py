"""CPU tests of what the mixer layer refuses before it hands pointers to the library."""
import pytest
import torch

from paper_2008_04567_amd.mixer import Mixer

WIDTH, REQUESTS, TOKENS = 32, 3, 10


@pytest.fixture(scope="module")
def layer():
    m = Mixer(WIDTH, 2, 8, 1, 16, slots=4, dtype=torch.bfloat16, device="cpu")
    return m, m.plan(REQUESTS, TOKENS, 6), m.plan(REQUESTS, REQUESTS, 1)


def h(tokens=TOKENS, width=WIDTH, dtype=torch.bfloat16):
    return torch.zeros((tokens, width), dtype=dtype)


def i32(n):
    return torch.zeros(n, dtype=torch.int32)


@pytest.mark.parametrize("change,word", [
    (dict(h=h(TOKENS - 1)), "h"), (dict(h=h(TOKENS + 1)), "h"), (dict(h=h(width=WIDTH + 1)), "h"), (dict(h=h().view(-1)), "h"),
    (dict(h=h(dtype=torch.float32)), "h"), (dict(h=torch.zeros((WIDTH, TOKENS), dtype=torch.bfloat16).T), "h"),
    (dict(h=h(1).expand(TOKENS, WIDTH)), "h"),
    (dict(starts=i32(REQUESTS)), "starts"), (dict(starts=i32(REQUESTS + 1).long()), "starts"),
    (dict(starts=i32(2 * REQUESTS + 2)[::2]), "starts"), (dict(starts=[0, 1, 2, 3]), "starts"),
    (dict(slot_map=i32(REQUESTS).long()), "slot_map"), (dict(slot_map=i32(REQUESTS - 1)), "slot_map"),
    (dict(resume=i32(REQUESTS).bool()), "resume"), (dict(resume=i32((REQUESTS, 1))), "resume"),
    (dict(), "GPU"), (dict(starts=None, slot_map=None), "GPU")])
def test_prompt_refuses(layer, change, word):
    m, plan, _ = layer
    args = dict(dict(h=h(), starts=i32(REQUESTS + 1), slot_map=i32(REQUESTS), resume=i32(REQUESTS), stream=0), **change)
    with pytest.raises(ValueError, match=word):
        m.prompt(plan, **args)


@pytest.mark.parametrize("change,word", [
    (dict(h=h(REQUESTS + 1)), "h"), (dict(h=h(REQUESTS, dtype=torch.float16)), "h"), (dict(slot_map=i32(REQUESTS).long()), "slot_map"),
    (dict(), "GPU")])
def test_step_refuses(layer, change, word):
    m, _, one = layer
    with pytest.raises(ValueError, match=word):
        m.step(one, **dict(dict(h=h(REQUESTS), slot_map=i32(REQUESTS), stream=0), **change))


def test_calls_refuses_plans_of_others(layer):
    m, plan, one = layer
    with pytest.raises(ValueError, match="token"):
        m.step(plan, h(), i32(REQUESTS), stream=0)
    other = Mixer(WIDTH, 2, 8, 1, 16, slots=4, device="cpu", seed=1)
    with pytest.raises(ValueError, match="plan"):
        other.prompt(plan, h(), i32(REQUESTS + 1), i32(REQUESTS), stream=0)
