"""GPU tests of the sequence layers (product, short causal convolution, scan) against their definitions in 64 bits."""
import numpy as np
import pytest

from tests import parity as PT

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "f16", "f32"]


@pytest.fixture(scope="module")
def S():
    PT.torch_dev()
    from tests import sequence_case
    return sequence_case


# ---- product ------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 64), (1, 1000, 512), (2, 40, 2048), (5, 257, 96), (16, 512, 1024), (17, 130, 72),
                                   (33, 100, 1000), (64, 64, 4096), (65, 300, 40), (127, 129, 128), (200, 1000, 264),
                                   (255, 256, 320), (300, 511, 64), (513, 260, 200), (1030, 770, 136)])
def test_linear_sizes(S, dtype, m, n, k):
    S.run_linear(m, n, k, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k,y_f32", [(4097, 4100, 72, False), (4100, 4097, 200, True), (4096, 4352, 64, False), (8200, 2050, 136, False)])
def test_linear_many_large_tiles(S, dtype, m, n, k, y_f32):
    S.run_linear(m, n, k, dtype, act="silu", y_f32=y_f32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(2, 9000, 64), (20, 13000, 72), (50, 20000, 40), (64, 12290, 130), (3000, 1500, 24), (2000, 2300, 8)])
def test_linear_wide_outputs(S, dtype, m, n, k):
    S.run_linear(m, n, k, dtype, act="relu")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(3, 70, 37), (20, 33, 129), (130, 190, 201), (300, 290, 515)])
def test_linear_odd_reduction_and_unaligned_rows(S, dtype, m, n, k):
    S.run_linear(m, n, k, dtype, pad=(3, 1, 5), offset=1)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("bias,residual,y_f32", [(False, False, False), (True, False, True), (False, True, False)])
@pytest.mark.parametrize("m", [4, 150])
def test_linear_epilogues(S, act, bias, residual, y_f32, m):
    for dtype in DTYPES:
        S.run_linear(m, 200, 128, dtype, act=act, bias=bias, residual=residual, y_f32=y_f32, pad=(8, 16, 8))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 9, 40, 260])
def test_linear_long_reductions(S, dtype, m):
    S.run_linear(m, 72, 8192, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,k,pad", [(5, 96, 0), (70, 100, 4), (300, 520, 0), (300, 37, 3)])
def test_linear_values_beside_the_matrices_do_not_show(S, dtype, m, k, pad):
    # infinities and NaN in the rows' padding and in rows and columns beyond the matrices
    import torch
    B, (code, ty) = S.B, S.TYPES[dtype][:2]
    r, n = S.Rng(7), 130
    big_x = torch.full((m + 4, k + 8 + pad), float("nan"), device="cuda", dtype=ty)
    big_w = torch.full((n + 300, k + 8 + pad), float("inf"), device="cuda", dtype=ty)
    big_x[:m, :k], big_w[:n, :k] = r.normal((m, k), dtype), r.normal((n, k), dtype, k ** -0.5)
    y = torch.empty((m, n), device="cuda", dtype=ty)
    desc = B.make_linear_desc(m, n, k, dtype=code, x_stride=k + 8 + pad, w_stride=k + 8 + pad)
    ws = torch.full((max(16, B.linear_workspace(desc)),), 255, device="cuda", dtype=torch.uint8)
    B.linear_fwd(desc, big_x, big_w, y, workspace=ws)
    ref, d = S.osq.linear(S.f64(big_x[:m, :k]), S.f64(big_w[:n, :k]))
    S.close(y, ref, d, dtype, (k + 64) * 2.0 ** -24, "linear beside NaN")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [3, 40, 300])
def test_linear_infinities_and_nan_stay_in_their_rows_and_columns(S, dtype, m):
    import torch
    B, (code, ty) = S.B, S.TYPES[dtype][:2]
    r, n, k = S.Rng(8), 140, 72
    x, w = r.normal((m, k), dtype), r.normal((n, k), dtype)
    x[1, 5], w[7, 70] = float("nan"), float("inf")
    y = torch.empty((m, n), device="cuda", dtype=ty)
    desc = B.make_linear_desc(m, n, k, dtype=code)
    ws = torch.full((max(16, B.linear_workspace(desc)),), 255, device="cuda", dtype=torch.uint8)
    B.linear_fwd(desc, x, w, y, workspace=ws)
    got = S.f64(y)
    want = np.ones((m, n), bool)
    want[1], want[:, 7] = False, False
    assert np.array_equal(np.isfinite(got), want)


def test_linear_extremes_of_fp32(S):
    # operands near both ends of the type's range: products that fit, sums that fit
    import torch
    B, r = S.B, S.Rng(9)
    for scale_x, scale_w in ((2.0 ** 120, 2.0 ** -60), (2.0 ** -120, 2.0 ** 30), (2.0 ** 60, 2.0 ** 60)):
        for m in (3, 200):
            x, w = r.normal((m, 160)) * scale_x, r.normal((96, 160)) * scale_w
            y = torch.empty((m, 96), device="cuda")
            desc = B.make_linear_desc(m, 96, 160, dtype=B.F32)
            ws = torch.full((max(16, B.linear_workspace(desc)),), 255, device="cuda", dtype=torch.uint8)
            B.linear_fwd(desc, x, w, y, workspace=ws)
            ref, d = S.osq.linear(S.f64(x), S.f64(w))
            S.close(y, ref, d, "f32", (160 + 64) * 2.0 ** -24, "linear at 2^%d" % int(np.log2(scale_x)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(6, 200, 1024), (100, 64, 4096), (400, 300, 256)])
def test_linear_residual_in_place_other_stream_and_repeats(S, dtype, m, n, k):
    import torch
    B, (code, ty) = S.B, S.TYPES[dtype][:2]
    r = S.Rng(10)
    x, w, res = r.normal((m, k), dtype), r.normal((n, k), dtype, k ** -0.5), r.normal((m, n), dtype)
    desc = B.make_linear_desc(m, n, k, dtype=code)
    side, outs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        y = res.clone()
        side.wait_stream(torch.cuda.current_stream())
        ws = torch.full((max(16, B.linear_workspace(desc)),), 255, device="cuda", dtype=torch.uint8)
        side.wait_stream(torch.cuda.current_stream())
        B.linear_fwd(desc, x, w, y, residual=y, workspace=ws, stream=side)
        torch.cuda.synchronize()
        outs.append(y)
    ref, d = S.osq.linear(S.f64(x), S.f64(w), None, S.f64(res))
    S.close(outs[0], ref, d, dtype, (k + 64) * 2.0 ** -24, "linear in place")
    assert all(torch.equal(outs[0], o) for o in outs), "the same call gave different sums"


# ---- convolution ----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [2, 3, 4, 5, 8])
def test_conv_widths_and_lengths(S, dtype, width):
    lengths = [0, 1, 2, 3, 7, 15, 16, 17, 33, 100]
    S.run_conv(lengths, 40, width, dtype, resume=[1, 0, 1, 0, 1, 1, 0, 1, 0, 1])
    S.run_conv(lengths, 37, width, dtype, act="none", bias=False, in_place=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_conv_strides_and_alignment(S, dtype):
    for channels in (1, 8, 13, 64, 2056):
        S.run_conv([5, 40], channels, 4, dtype, pad=(3, 5), offset=1)
        S.run_conv([5, 40], channels, 4, dtype, pad=(8, 16), offset=8)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("channels", [4, 6, 9, 10, 42, 70, 2054])
def test_conv_channels_that_fill_no_lane(S, dtype, channels):
    lengths = [0, 1, 2, 33, 100]
    S.run_conv(lengths, channels, 4, dtype, resume=[1, 0, 1, 0, 1], in_place=True)
    S.run_conv(lengths, channels, 3, dtype, pad=(2, 6), offset=2)


@pytest.mark.parametrize("dtype", DTYPES)
def test_conv_requests(S, dtype):
    S.run_conv([20, 20, 20], 24, 4, dtype, uniform=True, in_place=True)
    S.run_conv([3, 90, 5], 24, 4, dtype, max_length=16, in_place=True)          # longer than the launch was shaped for
    S.run_conv([4, 0, 6, 2], 24, 4, dtype, slot_map=[-1, 2, 99, 0])             # entries that are none
    S.run_conv([4, 9], 24, 3, dtype, state=False)
    S.run_conv([1] * 300, 16, 4, dtype, in_place=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("channels", [9, 64])
def test_conv_step_continues_what_a_prompt_left(S, dtype, channels):
    import torch
    B, (code, ty) = S.B, S.TYPES[dtype][:2]
    r, width, n = S.Rng(11), 4, 7
    x, w, bb = r.normal((3 * n, channels), dtype), r.normal((channels, width), dtype), r.normal((channels,), dtype)
    whole, pool = torch.empty_like(x), r.normal((3, width - 1, channels), dtype)
    desc = B.make_causal_conv_desc(3, 3 * n, channels, width, slots=3, dtype=code)
    B.causal_conv1d_fwd(desc, x, w, whole, bias=bb, state_in=pool, state_out=torch.empty_like(pool))
    one = B.make_causal_conv_desc(3, 3, channels, width, slots=3, dtype=code)
    slot_map = S.i32([0, 1, 2])
    for t in range(n):
        xt = x.view(3, n, channels)[:, t].contiguous()
        y = torch.empty_like(xt)
        B.causal_conv1d_step(one, xt, w, y, bias=bb, slot_map=slot_map, state_in=pool, state_out=pool)
        assert torch.equal(y, whole.view(3, n, channels)[:, t])
    assert torch.equal(pool, x.view(3, n, channels)[:, n - width + 1:])


def test_conv_later_values_do_not_show_in_earlier_rows(S):
    import torch
    B, r = S.B, S.Rng(12)
    x = r.normal((50, 16), "bf16")
    x[20, 3], x[49, 5] = float("nan"), float("inf")
    y = torch.empty_like(x)
    B.causal_conv1d_fwd(B.make_causal_conv_desc(1, 50, 16, 4), x, r.normal((16, 4), "bf16"), y)
    bad = ~torch.isfinite(y)
    rows = torch.nonzero(bad).tolist()
    assert rows == [[t, 3] for t in range(20, 24)] + [[49, 5]]


# ---- scan -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,head_dim,groups,state_dim", [(1, 1, 1, 1), (4, 16, 2, 16), (3, 20, 1, 36), (2, 64, 1, 128), (2, 33, 2, 129),
                                                             (2, 128, 1, 64), (1, 200, 1, 250), (6, 48, 3, 72), (2, 64, 1, 256)])
def test_scan_sizes(S, dtype, heads, head_dim, groups, state_dim):
    S.run_scan([0, 1, 2, 31, 33, 63, 64, 65, 130], heads, head_dim, groups, state_dim, dtype,
               resume=[1, 0, 1, 1, 0, 1, 0, 1, 1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_scan_long_requests(S, dtype):
    # parallel along the tokens: parts of a request joined
    S.run_scan([1500], 2, 32, 1, 64, dtype)
    S.run_scan([700, 3, 0, 1100], 2, 64, 2, 32, dtype, resume=[1, 1, 1, 0], in_place=True)
    S.run_scan([900, 64], 1, 40, 1, 100, dtype, max_length=128, in_place=True)      # longer than the launch was shaped for


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,head_dim,groups,state_dim", [(4, 64, 1, 128), (5, 64, 1, 72), (12, 40, 2, 64), (14, 8, 2, 8), (4, 128, 1, 32),
                                                             (3, 136, 1, 40), (9, 24, 1, 120), (8, 200, 2, 16), (4, 64, 1, 130)])
def test_scan_many_heads_a_group(S, dtype, heads, head_dim, groups, state_dim):
    lengths = [0, 1, 2, 31, 33, 63, 64, 65, 130]
    S.run_scan(lengths, heads, head_dim, groups, state_dim, dtype, resume=[1, 0, 1, 1, 0, 1, 0, 1, 1], in_place=True)
    S.run_scan(lengths, heads, head_dim, groups, state_dim, dtype, gate=False, skip=False, bias=False, pad=8, offset=8)
    S.run_scan([700, 3, 0, 1100], heads, head_dim, groups, state_dim, dtype, resume=[1, 1, 1, 0], in_place=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_scan_many_heads_requests_values_and_alignment(S, dtype):
    S.run_scan([900, 64], 4, 40, 1, 64, dtype, max_length=128, in_place=True)       # longer than the launch was shaped for
    S.run_scan([4, 0, 70, 2], 6, 32, 1, 32, dtype, slot_map=[-1, 2, 99, 0])
    S.run_scan([90, 600], 4, 64, 1, 64, dtype, state=False)
    S.run_scan([70, 30], 4, 32, 1, 64, dtype, pad=4, offset=4)
    S.run_scan([70, 30], 4, 32, 1, 64, dtype, pad=3, offset=1)
    S.run_scan([40, 40, 40], 8, 32, 2, 32, dtype, uniform=True, in_place=True)

    def edit(i):
        i["x"][100, 5], i["x"][37, 70], i["x"][4, 250] = float("nan"), float("inf"), float("-inf")
        i["z"][20, 2], i["c"][50, 7], i["b"][300, 3] = float("nan"), float("nan"), float("nan")
        i["dt"][10::17] = 60.0
    S.run_scan([130, 140, 70], 4, 64, 1, 128, dtype, edit=edit)


def test_scan_many_requests_of_many_lengths(S):
    # more workgroups than run at once: the longest first, in parts
    r = np.random.default_rng(5)
    lengths = [int(v) for v in r.integers(0, 90, 150)]
    lengths[3], lengths[77], lengths[149] = 900, 0, 1500
    S.run_scan(lengths, 8, 16, 1, 16, "bf16", resume=[i % 3 == 0 for i in range(150)])
    S.run_scan(lengths, 8, 16, 1, 18, "bf16", in_place=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gate,skip,bias,softplus", [(False, False, False, True), (True, False, True, False), (False, True, False, False)])
def test_scan_terms(S, dtype, gate, skip, bias, softplus):
    S.run_scan([70, 30], 4, 32, 2, 64, dtype, gate=gate, skip=skip, bias=bias, softplus=softplus)


@pytest.mark.parametrize("dtype", DTYPES)
def test_scan_strides_requests_and_states(S, dtype):
    S.run_scan([50, 20], 2, 64, 1, 64, dtype, pad=3, offset=1)
    S.run_scan([50, 20], 2, 64, 1, 64, dtype, pad=8, offset=8)
    S.run_scan([40, 40, 40], 2, 32, 1, 32, dtype, uniform=True, in_place=True)
    S.run_scan([4, 0, 70, 2], 2, 32, 1, 32, dtype, slot_map=[-1, 2, 99, 0])
    S.run_scan([90], 2, 32, 1, 32, dtype, state=False)
    import torch
    S.run_scan([90, 300], 2, 32, 1, 64, dtype, stream=torch.cuda.Stream())


@pytest.mark.parametrize("dtype", DTYPES)
def test_scan_forgets_at_once_and_never(S, dtype):
    # steps so large that exp(delta a) is zero between steps that keep nearly everything
    def edit(i):
        i["dt"][10::17] = 60.0
        i["dt"][40:90] = -9.0
        i["dt_bias"].fill_(-2.0)
        i["a"][0] = -1000.0
    S.run_scan([200, 65], 2, 32, 1, 48, dtype, edit=edit)

    def still(i):
        i["a"].zero_()
        i["dt_bias"].fill_(-5.0)
    S.run_scan([300], 2, 32, 1, 48, dtype, edit=still)


@pytest.mark.parametrize("dtype", DTYPES)
def test_scan_infinities_and_nan_show_only_from_their_token_on(S, dtype):
    def edit(i):
        i["x"][100, 5] = float("nan")
        i["x"][37, 34] = float("inf")
        i["z"][20, 2] = float("nan")
        i["c"][50, 7] = float("nan")
        i["b"][300, 3] = float("nan")
    S.run_scan([130, 140, 70], 2, 32, 1, 64, dtype, edit=edit)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,head_dim,groups,state_dim", [(1, 1, 1, 1), (4, 16, 2, 16), (3, 20, 1, 36), (8, 64, 2, 128), (2, 33, 2, 129),
                                                             (2, 128, 1, 64), (1, 200, 1, 250), (2, 64, 1, 256)])
def test_scan_step(S, dtype, heads, head_dim, groups, state_dim):
    S.run_scan([1] * 5, heads, head_dim, groups, state_dim, dtype, step=True)
    S.run_scan([1] * 4, heads, head_dim, groups, state_dim, dtype, step=True, in_place=True, gate=False, skip=False, pad=3,
               offset=1, slot_map=[2, -1, 0, 5])


def test_step_and_prompt_captured_in_a_graph(S):
    import torch
    B = S.B
    lengths, H, P, N = [70, 200], 4, 64, 64
    i = S.ssm_inputs(lengths, H, P, 1, N, "bf16")
    desc = B.make_ssm_desc(2, 270, H, P, 1, N, max_length=200, slots=4, dtype=B.BF16)
    lin = B.make_linear_desc(270, 96, H * P, dtype=B.BF16)
    w = S.Rng(5).normal((96, H * P), "bf16", 0.1)
    y, o = torch.empty_like(i["x"]), torch.empty((270, 96), device="cuda", dtype=torch.bfloat16)
    out, starts = torch.zeros_like(i["pool"]), S.i32([0, 70, 270])
    ws = torch.empty(max(16, B.ssm_workspace(desc)), device="cuda", dtype=torch.uint8)
    wl = torch.empty(max(16, B.linear_workspace(lin)), device="cuda", dtype=torch.uint8)

    def call(stream):
        B.ssm_scan_fwd(desc, i["x"], i["dt"], i["a"], i["b"], i["c"], y, d=i["d"], z=i["z"], dt_bias=i["dt_bias"],
                       starts=starts, state_in=i["pool"], state_out=out, workspace=ws, stream=stream)
        B.linear_fwd(lin, y, w, o, workspace=wl, stream=stream)

    call(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(torch.cuda.current_stream())
    for turn in range(4):
        i["x"].copy_(S.Rng(50 + turn).normal(tuple(i["x"].shape), "bf16"))
        call(torch.cuda.current_stream())
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, o, out)]
        for t in (y, o, out):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, o, out))), "replay %d" % turn


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("state_dim", [16, 56, 128, 200])
def test_scan_rows_at_multiples_of_four_bytes(S, dtype, state_dim):
    for heads, head_dim, pad, offset in ((3, 24, 2, 2), (6, 72, 6, 0), (1, 8, 2, 4)):
        S.run_scan([1, 90, 0, 200], heads, head_dim, 1, state_dim, dtype, pad=pad, offset=offset, resume=[1, 0, 1, 1])
        S.run_scan([1] * 5, heads, head_dim, 1, state_dim, dtype, pad=pad, offset=offset, step=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_scan_more_workgroups_than_compute_units(S, dtype):
    for pad in (0, 2, 1):                                  # rows at multiples of 16 bytes, of four and of two
        S.run_scan([70, 200, 31], 160, 16, 2, 96, dtype, pad=pad, in_place=True)
        S.run_scan([33, 600], 4, 16, 1, 96, dtype, pad=pad)


@pytest.mark.parametrize("dtype", DTYPES)
def test_loose_bounds_on_lengths(S, dtype):
    for bound in (1000, 2 ** 31 - 1):
        S.run_conv([3, 90, 0, 1], 24, 4, dtype, max_length=bound, in_place=True)
        S.run_scan([3, 700, 0, 1], 4, 16, 2, 40, dtype, max_length=bound, in_place=True)


def test_offsets_beyond_32_bits(S):
    import torch
    B = S.B
    rows, stride, c = 1100, (1 << 22) - 8, 16          # 4.6e9 elements between the first row and the last
    buf = torch.empty(rows * stride, device="cuda", dtype=torch.bfloat16)
    x = buf.as_strided((rows, c), (stride, 1))
    r = S.Rng(13)
    small = r.normal((rows, c), "bf16")
    x.copy_(small)
    w, y1, y2 = r.normal((c, 4), "bf16"), torch.empty_like(small), torch.empty_like(small)
    B.causal_conv1d_fwd(B.make_causal_conv_desc(1, rows, c, 4, x_stride=stride), x, w, y1)
    B.causal_conv1d_fwd(B.make_causal_conv_desc(1, rows, c, 4), small, w, y2)
    torch.cuda.synchronize()
    assert torch.equal(y1, y2)
    i = S.ssm_inputs([rows], 1, 16, 1, 16, "bf16")
    i["x"].copy_(small)
    out = []
    for y in (x, torch.empty_like(small)):          # y in the far rows, then in dense ones
        desc = B.make_ssm_desc(1, rows, 1, 16, 1, 16, dtype=B.BF16, y_stride=y.stride(0))
        ws = torch.empty(max(16, B.ssm_workspace(desc)), device="cuda", dtype=torch.uint8)
        B.ssm_scan_fwd(desc, small, i["dt"], i["a"], i["b"], i["c"], y, workspace=ws)
        torch.cuda.synchronize()
        out.append(y.contiguous().clone())
    assert torch.equal(out[0], out[1])
    x.copy_(small)                                   # x in the far rows
    y = torch.empty_like(small)
    desc = B.make_ssm_desc(1, rows, 1, 16, 1, 16, dtype=B.BF16, x_stride=stride)
    B.ssm_scan_fwd(desc, x, i["dt"], i["a"], i["b"], i["c"], y, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(out[0], y)


# ---- all together ---------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
def test_mixer_prompts_then_steps_agree_with_whole_prompts(S, dtype):
    # A layer's prompts cut anywhere and continued token by token give what the whole prompts give, but for the order of
    # sums (few rows and many are multiplied by different kernels) and the roundings that come out of it: four in a row
    # (row, convolution, y, output), each of a unit of the type or of 2^-20 of sums of this length, and as much for what
    # they carry on.
    import torch
    from paper_2008_04567_amd.mixer import Mixer
    ty, u = S.TYPES[dtype][1], S.TYPES[dtype][2]
    whole, cut = [Mixer(96, 4, 32, 2, 48, slots=5, dtype=ty, seed=3) for _ in range(2)]
    lengths, first = [9, 70, 3, 141], [4, 66, 2, 100]
    slots = S.i32([4, 0, 2, 1])
    rows = [S.Rng(60 + i).normal((n, 96), dtype) for i, n in enumerate(lengths)]
    p = whole.plan(4, sum(lengths), max(lengths))
    want = whole.prompt(p, torch.cat(rows), S.i32(S.starts_of(lengths)), slots).clone()
    want = torch.split(want, lengths)
    part = cut.plan(4, sum(first), max(first))
    got = [list(torch.split(cut.prompt(part, torch.cat([r[:n] for r, n in zip(rows, first)]), S.i32(S.starts_of(first)),
                                       slots).clone(), first))]
    # the rest of the longest as a second prompt, the others token by token
    rest = [0, 0, 0, 30]
    second = cut.plan(4, 30, 30)
    more = cut.prompt(second, rows[3][100:130], S.i32(S.starts_of(rest)), slots, resume=S.i32([1, 1, 1, 1])).clone()
    at, outs = [4, 66, 2, 130], [[got[0][i]] for i in range(4)]
    outs[3].append(more)
    while any(at[i] < lengths[i] for i in range(4)):
        live = [i for i in range(4) if at[i] < lengths[i]]
        one = cut.plan(len(live), len(live), 1)
        h = torch.stack([rows[i][at[i]] for i in live])
        y = cut.step(one, h, slots[live].contiguous()).clone()
        for k, i in enumerate(live):
            outs[i].append(y[k:k + 1])
            at[i] += 1
    scale = max(float(w.float().abs().max()) for w in want)
    for i in range(4):
        err = (torch.cat(outs[i]).float() - want[i].float()).abs().max()
        assert float(err) <= 16 * max(u, 2.0 ** -20) * scale, "request %d differs by %.3g" % (i, float(err))
    for a, b in ((whole.conv_state, cut.conv_state), (whole.scan_state, cut.scan_state)):
        err = (a.float() - b.float()).abs().max() / a.float().abs().max()
        assert float(err) <= 16 * max(u, 2.0 ** -20)
