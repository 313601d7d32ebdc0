"""GPU tests of every kernel that the sequence layers' rules choose between, each with several whole steps and a rest, and
of which kernel a call runs."""
import pytest

from tests import parity as PT

pytestmark = pytest.mark.gpu

SIXTEEN = ["bf16", "f16"]


@pytest.fixture(scope="module")
def S():
    PT.torch_dev()
    from tests import sequence_case, sequence_strict
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(sequence_case, "close", sequence_strict.close)
        yield sequence_case


# (kernel, template arguments behind the type, types, m, n, k, rows' padding and offset in elements, whether the
# reduction is cut)
FORMS = [
    # few rows: columns by 16, 32 and 48, rows by 16, 32 and 64, the loads of U runs of 512 entries under way more than once
    ("rows", "1, 3, 4", SIXTEEN, 4, 9000, 8200, 0, False),
    ("rows", "1, 2, 4", SIXTEEN, 9, 5000, 4700, 0, False),
    ("rows", "1, 1, 4", SIXTEEN, 16, 2050, 4200, 1, False),
    ("rows", "1, 1, 4", SIXTEEN, 2, 300, 16500, 0, True),
    ("rows", "2, 3, 2", SIXTEEN, 32, 8512, 2048, 0, False),
    ("rows", "2, 3, 2", SIXTEEN, 24, 9000, 2100, 1, False),
    ("rows", "2, 2, 2", SIXTEEN, 17, 8000, 2300, 0, False),
    ("rows", "4, 3, 2", SIXTEEN, 64, 9000, 2500, 0, False),
    ("rows", "4, 1, 2", SIXTEEN, 50, 2000, 4100, 0, True),
    ("rows", "1, 3, 2", ["f32"], 4, 9000, 4200, 0, False),
    ("rows", "2, 2, 2", ["f32"], 32, 6000, 2300, 1, False),
    ("rows", "4, 3, 1", ["f32"], 64, 9000, 1300, 0, False),
    ("rows", "4, 1, 1", ["f32"], 40, 1500, 4300, 0, True),
    # tiles loaded straight to LDS: 256 wide, 128 wide in four and in two buffers, 64 wide
    ("direct", "256, 256, 2, 4, 64, 2", SIXTEEN, 4100, 4096, 456, 0, False),
    ("direct", "128, 128, 2, 4, 64, 4", SIXTEEN, 1777, 2304, 1544, 0, False),
    ("direct", "128, 128, 2, 4, 64, 2", SIXTEEN, 3000, 1500, 520, 0, False),
    ("direct", "64, 64, 2, 2, 64, 4", SIXTEEN, 500, 600, 936, 0, False),
    ("direct", "64, 64, 2, 2, 64, 4", SIXTEEN, 70, 300, 2056, 0, True),
    # tiles through registers: rows that are not aligned, and fp32
    ("tiles", "128, 128, 2, 2", SIXTEEN, 3000, 1500, 205, 0, False),
    ("tiles", "128, 128, 2, 2", SIXTEEN, 4100, 4097, 131, 1, False),
    ("tiles", "64, 64, 2, 2", SIXTEEN, 500, 600, 333, 1, False),
    ("tiles", "128, 128, 2, 2", ["f32"], 3000, 1500, 520, 0, False),
    ("tiles", "128, 128, 2, 2", ["f32"], 1500, 1500, 1100, 0, True),
    ("tiles", "64, 64, 2, 2", ["f32"], 777, 1000, 2048, 0, True),
    ("tiles", "64, 64, 2, 2", ["f32"], 300, 500, 700, 3, False),
]
CASES = [pytest.param(f, t, id="-".join([f[0], f[1].replace(", ", "x"), t, "x".join(str(v) for v in f[3:6])]))
         for f in FORMS for t in f[2]]


def kernels_of(call):
    """Names of the kernels that a call launches."""
    import torch
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    return [e.name for e in p.events() if "linear_" in e.name]


@pytest.mark.parametrize("form,dtype", CASES)
def test_linear_forms(S, form, dtype):
    kind, args, _, m, n, k, odd, cut = form
    S.run_linear(m, n, k, dtype, act="silu", pad=(odd, odd, odd), offset=odd)


@pytest.mark.parametrize("form,dtype", CASES)
def test_linear_form_is_the_one_meant(S, form, dtype):
    import torch
    kind, args, _, m, n, k, odd, cut = form
    B, (code, ty) = S.B, S.TYPES[dtype][:2]
    x, w = [S.sliced(torch.zeros((r, k), device="cuda", dtype=ty), k + odd, odd)[0] for r in (m, n)]
    y = torch.empty((m, n), device="cuda", dtype=ty)
    desc = B.make_linear_desc(m, n, k, dtype=code, x_stride=k + odd, w_stride=k + odd)
    ws = torch.empty(max(16, B.linear_workspace(desc)), device="cuda", dtype=torch.uint8)
    names = kernels_of(lambda: B.linear_fwd(desc, x, w, y, workspace=ws))
    if not names:
        pytest.skip("the profiler shows no kernels here")
    name, numbers = names[0], args.split(", ")
    assert "linear_%s_kernel" % kind in name, (form, names)
    # (some demanglers do not know the 16-bit types and lose the argument behind them)
    tail = "".join("Li%sE" % v for v in numbers) if name.startswith("_Z") else ", ".join(numbers[1:]) + ">"
    assert tail in name, (form, names)
    assert len(names) == (2 if cut else 1) and (not cut or "linear_join_kernel" in names[1]), names
    assert (B.linear_workspace(desc) > 0) == cut


def test_single_tokens_captured_in_a_graph(S):
    # a convolution's and a scan's step in place, as a serving program captures them: replayed over eager work between
    import torch
    B, (code, ty) = S.B, S.TYPES["bf16"][:2]
    n, H, P, N, W = 5, 4, 64, 128, 4
    channels, r = H * P + 2 * N, S.Rng(20)
    row, xbc, y = r.normal((n, channels), "bf16"), torch.empty((n, channels), device="cuda", dtype=ty), \
        torch.empty((n, H * P), device="cuda", dtype=ty)
    w, bias, dt, z = r.normal((channels, W), "bf16"), r.normal((channels,), "bf16"), r.normal((n, H), "bf16"), \
        r.normal((n, H * P), "bf16")
    a, conv_pool, pool = -r.normal((H,)).abs(), r.normal((8, W - 1, channels), "bf16"), r.normal((8, H, P, N))
    x, b, c = xbc[:, :H * P], xbc[:, H * P:H * P + N], xbc[:, H * P + N:]
    slot_map = S.i32([6, 0, 3, -1, 7])
    conv = B.make_causal_conv_desc(n, n, channels, W, slots=8, dtype=code)
    ssm = B.make_ssm_desc(n, n, H, P, 1, N, slots=8, dtype=code, x_stride=channels, b_stride=channels, c_stride=channels)

    def step():
        s = torch.cuda.current_stream()
        B.causal_conv1d_step(conv, row, w, xbc, bias=bias, slot_map=slot_map, state_in=conv_pool, state_out=conv_pool, stream=s)
        B.ssm_scan_step(ssm, x, dt, a, b, c, y, z=z, slot_map=slot_map, state_in=pool, state_out=pool, stream=s)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    for turn in range(4):
        row.copy_(S.Rng(70 + turn).normal((n, channels), "bf16"))
        before = conv_pool.clone(), pool.clone()
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, conv_pool, pool)]
        conv_pool.copy_(before[0])
        pool.copy_(before[1])
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, t) for g, t in zip(want, (y, conv_pool, pool))), "replay %d" % turn
