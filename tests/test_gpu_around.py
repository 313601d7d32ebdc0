"""GPU tests of what stands around a mixer layer (normalisation, 8-bit values and products, products by expert, the router)
against its definitions in 64 bits."""
import numpy as np
import pytest

from tests import parity as PT

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "f16", "f32"]
ALL = DTYPES + ["e4m3"]


@pytest.fixture(scope="module")
def A():
    PT.torch_dev()
    from tests import around_case
    return around_case


# ---- normalisation --------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 7), (5, 64), (2, 127), (7, 128), (3, 129), (4, 512), (9, 513), (6, 1000), (5, 1024),
                                        (4, 1025), (3, 2048), (2, 2056), (3, 4096), (2, 4100), (2, 8192), (1, 8193), (2, 16384),
                                        (1, 20000), (1, 32768), (1, 40001), (1, 65536)])
def test_norm_sizes(A, dtype, rows, width):
    A.run_norm(rows, width, dtype, q=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("y,q,h,residual,gain", [(True, False, False, False, True), (False, True, True, True, False),
                                                 (False, False, True, True, True), (True, False, True, False, False)])
def test_norm_outputs_and_inputs_left_out(A, dtype, y, q, h, residual, gain):
    for width in (128, 200):
        A.run_norm(5, width, dtype, y=y, q=q, h=h, residual=residual, gain=gain)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,width,groups,q", [(3, 96, 2, False), (4, 1024, 8, True), (2, 300, 3, False), (3, 4096, 2, True), (5, 10, 10, False)])
def test_norm_groups(A, dtype, rows, width, groups, q):
    A.run_norm(rows, width, dtype, groups=groups, q=q)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("parts", [1, 2, 3, 4, 5, 8, 12, 64])
@pytest.mark.parametrize("width", [136, 1500])
def test_norm_parts(A, dtype, parts, width):
    A.run_norm(5, width, dtype, parts=parts, source="random", weights="random", q=True)
    A.run_norm(3, width, dtype, parts=parts, weights="random", residual=False)
    A.run_norm(3, width, dtype, parts=parts, source="random", x_rows=7)


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_parts_that_are_not_there_add_nothing(A, dtype):
    # numbers of rows outside x, whatever row the kernel may read instead: it holds NaN
    def nan(x, res, g):
        x[0] = float("nan")
    source = np.array([[1, -1, 3], [8, 2, 1], [-2 ** 31, 2 ** 31 - 1, 7], [4, 4, 4]], dtype=np.int64)
    A.run_norm(4, 72, dtype, parts=3, x_rows=8, source=source, weights="random", edit=nan)
    A.run_norm(4, 72, dtype, parts=3, x_rows=8, source=source, edit=nan, residual=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width,pad,offset", [(40, 3, 1), (513, 5, 3), (2048, 1, 1), (2048, 8, 8), (5000, 7, 0)])
def test_norm_rows_at_any_address(A, dtype, width, pad, offset):
    A.run_norm(4, width, dtype, pad=pad, offset=offset, q=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_in_place(A, dtype):
    import torch
    for width in (100, 2048):
        r = A.run_norm(6, width, dtype, in_place="hy", seed=4)
        s = A.run_norm(6, width, dtype, seed=4)
        assert torch.equal(r["h"], s["h"]) and torch.equal(r["y"], s["y"])


def test_norm_infinities_and_nan_stay_in_their_rows(A):
    def edit(x, res, g):
        x[1, 3], x[2, 5] = float("nan"), float("inf")
    for width in (64, 3000):
        A.run_norm(4, width, "f32", edit=edit)


@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1e15, 1e25, 1e37])
def test_norm_small_and_large(A, scale):
    A.run_norm(3, 700, "f32", scale=scale, eps=0.0, q=True)
    A.run_norm(3, 7000, "f32", scale=scale, eps=0.0)
    A.run_norm(3, 700, "bf16", scale=scale, eps=1e-6)


def test_norm_rows_of_zeros(A):
    def zeros(x, res, g):
        x[1], res[1] = 0.0, 0.0
    for width in (64, 3000):
        r = A.run_norm(3, width, "f32", edit=zeros, q=True)
        assert not r["y"][1].any() and not A.numbers(r["q"])[1].any()
        A.run_norm(3, width, "f32", edit=zeros, eps=0.0)       # nothing over nothing


def test_norm_many_rows(A):
    A.run_norm(5000, 24, "bf16")
    A.run_norm(1000, 1024, "bf16", q=True)


# ---- 8-bit values -----------------------------------------------------------------------------------
def eight(A, x, pad=0, offset=0):
    import torch
    code = {torch.float32: A.B.F32, torch.bfloat16: A.B.BF16, torch.float16: A.B.F16}[x.dtype]
    rows, width = x.shape
    view, _ = A.sliced(x, width + pad, offset)
    q, qb = A.rows_of_8(rows, width, 16)
    s, sb = A.out_rows(rows, A.oa.blocks(width), A.oa.blocks(width) + 2, 0, torch.float32)
    desc = A.B.make_quantize_desc(rows, width, dtype=code, x_stride=width + pad, q_stride=q.stride(0), scale_stride=s.stride(0))
    A.B.quantize_fwd(desc, view, q, s)
    torch.cuda.synchronize()
    A.pattern_intact(q, qb)
    A.guard_intact(s, sb)
    ref, scales = A.oa.quantize(x.float().cpu().numpy())
    assert np.array_equal(s.cpu().numpy(), scales, equal_nan=True), "scales"
    assert np.array_equal(A.numbers(q), ref, equal_nan=True), "8-bit values"
    return q, s


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 15), (2, 16), (70, 100), (5, 128), (33, 129), (17, 256), (9, 300), (130, 512), (7, 640),
                                        (5, 1024), (3, 1100), (2, 2048), (4, 2050), (3, 5000), (1, 8192), (2, 9000), (1, 100000)])
def test_quantize_is_the_definition_bit_for_bit(A, dtype, rows, width):
    x = A.Rng(rows).normal((rows, width), dtype)
    eight(A, x)
    eight(A, x, pad=3, offset=1)


def test_quantize_every_kind_of_number(A):
    import torch
    inf, nan = float("inf"), float("nan")
    x = A.Rng(3).normal((8, 400))
    x[0] = 0.0
    x[1, :128] = 2.0 ** -140
    x[1, 130], x[2, 5], x[2, 6] = 1e-37, 3.4e38, -1e-45
    x[3, 7], x[3, 200] = nan, nan
    x[4, 9], x[4, 300] = inf, -inf
    x[5, :128], x[5, 128:256] = nan, -0.0
    x[6] = torch.linspace(-500, 500, 400)
    x[7] *= 1e30
    eight(A, x)
    for dtype in ("bf16", "f16"):
        eight(A, x.to(A.TYPES[dtype][1]))
    # every 16-bit number, beside one that sets the scale to one
    for dtype in ("bf16", "f16"):
        v = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(A.TYPES[dtype][1]).cuda()
        v = torch.where(v.float().abs() <= 448, v, torch.zeros_like(v)).view(-1, 64)
        one = torch.full((len(v), 64), 448.0, device="cuda", dtype=v.dtype)
        eight(A, torch.cat([v, one], 1))


# ---- 8-bit product ------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 64), (1, 1000, 512), (2, 40, 2048), (5, 257, 96), (16, 512, 1024), (17, 130, 72),
                                   (33, 100, 1000), (48, 64, 200), (64, 64, 4096), (65, 300, 40), (127, 129, 128), (128, 128, 129),
                                   (200, 1000, 264), (255, 256, 320), (300, 511, 64), (513, 260, 200), (1030, 770, 136)])
def test_linear_q8_sizes(A, dtype, m, n, k):
    A.run_linear_q8(m, n, k, dtype)


@pytest.mark.parametrize("m", [3, 40, 150])
@pytest.mark.parametrize("k", [3, 15, 17, 31, 100, 127, 130, 143, 255, 1999])
def test_linear_q8_odd_reductions_beside_nan(A, m, k):
    A.run_linear_q8(m, 100, k, "bf16", extra=32)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("m", [4, 150])
def test_linear_q8_epilogues(A, act, bias, residual, m):
    for dtype in DTYPES:
        A.run_linear_q8(m, 200, 256, dtype, act=act, bias=bias, residual=residual, pad=8)
        A.run_linear_q8(m, 203, 160, dtype, act=act, bias=bias, residual=residual, pad=3, offset=1)


@pytest.mark.parametrize("m", [1, 9, 40, 260])
def test_linear_q8_long_reductions(A, m):
    A.run_linear_q8(m, 72, 8192, "bf16")
    A.run_linear_q8(m, 200, 16500, "f32")


@pytest.mark.parametrize("m,n,k", [(2, 9000, 128), (20, 13000, 144), (64, 12290, 130), (3000, 1500, 256), (2000, 2300, 16), (4100, 4097, 384)])
def test_linear_q8_wide(A, m, n, k):
    A.run_linear_q8(m, n, k, "bf16", act="silu")


@pytest.mark.parametrize("m,n,k", [(6, 200, 1024), (100, 64, 4096), (400, 300, 256)])
def test_linear_q8_in_place_other_stream_and_repeats(A, m, n, k):
    import torch
    side, outs = torch.cuda.Stream(), []
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        outs.append(A.run_linear_q8(m, n, k, "bf16", in_place=True, stream=side))
    assert all(torch.equal(outs[0], o) for o in outs)


@pytest.mark.parametrize("m", [3, 150])
def test_linear_q8_nan_and_scales_stay_in_their_rows(A, m):
    import torch
    n, k, B = 140, 272, A.B
    x, xs, xv = A.in_8(A.Rng(8).normal((m, k)))
    w, ws, wv = A.weight_in_8(A.Rng(9).normal((n, k)))
    x[1, 5], w[7, 270] = 0x7f, 0xff
    xs[2, 1] = float("inf")
    y = torch.empty((m, n), device="cuda")
    desc = B.make_linear_q8_desc(m, n, k, dtype=B.F32)
    B.linear_q8_fwd(desc, x, xs, w, ws, y, workspace=A.workspace(B.linear_q8_workspace(desc)))
    want = np.ones((m, n), bool)
    want[1], want[2], want[:, 7] = False, False, False
    assert np.array_equal(np.isfinite(A.f64(y)), want)


def test_linear_q8_scales_in_longer_rows(A):
    import torch
    B = A.B
    for m in (5, 200):
        n, k = 300, 400
        x, xs, xv = A.in_8(A.Rng(1).normal((m, k)))
        w, ws, wv = A.weight_in_8(A.Rng(2).normal((n, k)))
        far_x, far_w = [torch.full((s.shape[0], s.shape[1] + 3), float("nan"), device="cuda") for s in (xs, ws)]
        far_x[:, 1:-2], far_w[:, 2:-1] = xs, ws
        out = []
        for a, b in ((xs, ws), (far_x[:, 1:-2], far_w[:, 2:-1])):
            y = torch.empty((m, n), device="cuda", dtype=torch.bfloat16)
            desc = B.make_linear_q8_desc(m, n, k, x_scale_stride=a.stride(0), w_scale_stride=b.stride(0))
            B.linear_q8_fwd(desc, x, a, w, b, y, workspace=A.workspace(B.linear_q8_workspace(desc)))
            out.append(y)
        assert torch.equal(*out)


# ---- products by expert ---------------------------------------------------------------------------------
LENGTHS = [[1], [5, 0, 1], [0, 0, 9], [3, 70, 0, 130, 1], [64, 64], [200, 1, 17], [2, 1, 0, 3, 1, 1, 0, 2], [16, 33, 48]]


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda l: "-".join(map(str, l)))
def test_grouped_lengths(A, dtype, gated, lengths):
    A.run_grouped(lengths, 72, 96, dtype, act="silu", gated=gated)
    A.run_grouped(lengths, 40, 200, dtype, gated=gated, gather=True, before=3, behind=2)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("n,k", [(1, 1), (16, 64), (17, 37), (130, 520), (257, 72), (64, 1000), (300, 129)])
@pytest.mark.parametrize("mean", [2, 40, 150])
def test_grouped_sizes(A, dtype, n, k, mean):
    lengths = [mean, 0, 2 * mean, mean // 2]
    A.run_grouped(lengths, n, k, dtype, act="gelu", gather=True)
    A.run_grouped(lengths, n, k, dtype, act="relu", gated=True)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("groups", [64, 65, 130, 300])
def test_grouped_many_experts(A, dtype, groups):
    lengths = np.random.default_rng(groups).integers(0, 5, groups).tolist()
    A.run_grouped(lengths, 24, 40, dtype, gather=True)
    lengths[groups - 2] = 150
    A.run_grouped(lengths, 24, 40, dtype, gated=True, act="silu")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mean", [2, 150])
def test_grouped_rows_and_weights_at_any_address(A, dtype, mean):
    A.run_grouped([mean, 3, mean], 75, 101, dtype, pad=3, offset=1, group_pad=1, gather=True)
    A.run_grouped([mean, 3, mean], 75, 104, dtype, pad=8, offset=8, group_pad=2, gated=True, act="gelu")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("mean", [2, 150])
def test_grouped_fp32_outputs(A, dtype, mean):
    A.run_grouped([mean, 0, mean], 100, 160, dtype, y_dtype="f32", act="silu")
    A.run_grouped([mean, 0, mean], 100, 160, dtype, y_dtype="f32", act="gelu", gated=True)


def test_grouped_e4m3_into_fp16_and_odd_reductions(A):
    for k in (15, 100, 130, 143):
        for mean in (2, 150):
            A.run_grouped([mean, 5, mean], 60, k, "e4m3", y_dtype="f16", gather=True, pad=1, group_pad=3)
            A.run_grouped([mean, 5, mean], 60, k, "e4m3", gated=True, act="silu", group_pad=3)


@pytest.mark.parametrize("dtype", ALL)
def test_grouped_numbers_out_of_range_are_clamped(A, dtype):
    source = np.array([0, -1, 9, 2 ** 31 - 1, -2 ** 31, 4, 8, 7, 1, 3])
    for lengths in ([4, 6], [10, 0]):
        A.run_grouped(lengths, 40, 64, dtype, x_rows=9, source=source, starts=[-5, lengths[0], 10 ** 6])
    # rows that starts leave out stay as they are, also where starts are in no order
    import torch
    B = A.B
    if dtype != "e4m3":
        y = torch.full((10, 40), A.GUARD, device="cuda", dtype=A.TYPES[dtype][1])
        x, w = A.Rng(1).normal((10, 64), dtype), A.Rng(2).normal((3, 40, 64), dtype)
        desc = B.make_grouped_linear_desc(3, 10, 40, 64, dtype=A.TYPES[dtype][0])
        B.grouped_linear_fwd(desc, x, w, A.i32([6, 2, 2, 1]), y)
        assert bool((y == A.GUARD).all())


@pytest.mark.parametrize("dtype", ALL)
def test_grouped_one_expert_is_a_product(A, dtype):
    for rows in (1, 30, 200):
        A.run_grouped([rows], 100, 136, dtype)
        A.run_grouped([rows], 100, 136, dtype, gated=True, act="silu", gather=True)


@pytest.mark.parametrize("dtype", ALL)
def test_grouped_larger(A, dtype):
    A.run_grouped([700, 0, 1, 300, 555], 520, 640, dtype, gated=True, act="silu", gather=True)
    A.run_grouped([900, 40, 256, 300], 1100, 256, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_grouped_infinities_and_nan_stay_in_their_rows_and_experts(A, dtype):
    import torch
    B, (code, ty) = A.B, A.TYPES[dtype][:2]
    for lengths in ([3, 4, 5], [90, 100, 110]):
        rows, n, k = sum(lengths), 50, 72
        x, w = A.Rng(1).normal((rows, k), dtype), A.Rng(2).normal((3, n, k), dtype)
        x[1, 5], w[2, 7, 70] = float("nan"), float("inf")
        y = torch.empty((rows, n), device="cuda", dtype=ty)
        desc = B.make_grouped_linear_desc(3, rows, n, k, dtype=code)
        B.grouped_linear_fwd(desc, x, w, A.i32([0] + np.cumsum(lengths).tolist()), y)
        want = np.ones((rows, n), bool)
        want[1], want[lengths[0] + lengths[1]:, 7] = False, False
        assert np.array_equal(np.isfinite(A.f64(y)), want)


def test_grouped_extremes_of_fp32(A):
    import torch
    B = A.B
    for sx, sw in ((2.0 ** 120, 2.0 ** -60), (2.0 ** -120, 2.0 ** 30), (2.0 ** 60, 2.0 ** 60)):
        for lengths in ([3, 2], [70, 130]):
            rows, n, k = sum(lengths), 96, 160
            x, w = A.Rng(1).normal((rows, k)) * sx, A.Rng(2).normal((2, n, k)) * sw
            y = torch.empty((rows, n), device="cuda")
            st = [0, lengths[0], rows]
            B.grouped_linear_fwd(B.make_grouped_linear_desc(2, rows, n, k, dtype=B.F32), x, w, A.i32(st), y)
            ref, d = A.oa.grouped(A.f64(x), A.f64(w), st)
            A.close(y, ref, d, "f32", (k + 64) * 2.0 ** -24, "grouped at 2^%d" % int(np.log2(sx)))


# ---- router ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k", [(1, 1), (2, 1), (5, 5), (8, 2), (16, 4), (63, 8), (64, 8), (65, 6), (128, 8), (200, 10), (256, 32),
                                 (500, 3), (512, 8), (700, 8), (1024, 32)])
def test_route_sizes(A, dtype, n, k):
    for tokens in (1, 7, 64, 65, 300):
        A.run_route(A.Rng(tokens).normal((tokens, n), "f32", 2.0), k, dtype, normalize=tokens % 2 == 0, pad=tokens % 3)


@pytest.mark.parametrize("tokens", [1, 63, 64, 65, 1000, 5000, 20000, 200000])
def test_route_tokens(A, tokens):
    A.run_route(A.Rng(tokens).normal((tokens, 60)), 6, "bf16", scale=2.5)


def test_route_ties_go_to_the_lowest(A):
    import torch
    for n, k in ((10, 4), (64, 8), (130, 8), (1000, 20)):
        for tokens in (9, 400):
            l = torch.from_numpy(np.random.default_rng(n).integers(-1, 2, (tokens, n)).astype(np.float32)).cuda()
            l[0] = 0.0
            l[1, ::2] = -0.0
            A.run_route(l, k, "f32")
            A.run_route(l, k, "f16", normalize=False)


def test_route_masks_infinities_and_nan(A):
    inf, nan = float("inf"), float("nan")
    for n in (12, 100):
        for tokens in (8, 200):
            l = A.Rng(n).normal((tokens, n))
            l[0] = -inf                                 # nothing left
            l[1, 2:] = -inf                             # fewer left than are chosen
            l[2] = nan
            l[3, 5], l[3, 7] = nan, -inf
            l[4, 3], l[4, 9] = inf, inf
            l[5] = -3.4028234663852886e38               # the lowest number is no mask
            l[6, 1:] = -3.4028234663852886e38
            A.run_route(l, 6, "f32")
            A.run_route(l, 6, "f32", normalize=False)


def test_route_choice_alone_one_expert_for_all_and_no_tokens(A):
    import torch
    A.run_route(A.Rng(1).normal((700, 40)), 4, "f32", order=False)
    l = torch.zeros((900, 30), device="cuda")
    l[:, 11] = 5.0
    A.run_route(l, 1, "bf16")
    B, starts = A.B, torch.full((6,), -7, dtype=torch.int32, device="cuda")
    B.route_fwd(B.make_route_desc(0, 5, 2), None, None, None, starts, None, None)
    assert starts.tolist() == [0] * 6


# ---- together ---------------------------------------------------------------------------------------------
def layer(A, dtype8, tokens, seed=3):
    """norm (8 bits or not) -> router -> experts -> combination with the residual and the next norm; (calls, outputs, check)."""
    import torch
    B, ty = A.B, torch.bfloat16
    width, inner, experts, k = 256, 192, 12, 3
    r, rows = A.Rng(seed), tokens * k
    empty = lambda *s, t=ty: torch.empty(s, device="cuda", dtype=t)
    h, gain, x = r.normal((tokens, width), "bf16"), r.normal((width,), "bf16"), empty(tokens, width)
    w_route = r.normal((experts, width), "bf16", width ** -0.5)
    logits, ids, weights = empty(tokens, experts, t=torch.float32), empty(tokens, k, t=torch.int32), empty(tokens, k, t=torch.float32)
    starts, source, place = empty(experts + 1, t=torch.int32), empty(rows, t=torch.int32), empty(tokens, k, t=torch.int32)
    up, down = r.normal((experts, 2 * inner, width), "f32", width ** -0.5), r.normal((experts, width, inner), "f32", inner ** -0.5)
    mid, out, h2, y2 = empty(rows, inner), empty(rows, width), empty(tokens, width), empty(tokens, width)
    norm = B.make_rms_norm_desc(tokens, width)
    lin = B.make_linear_desc(tokens, experts, width, y_dtype=B.F32)
    route = B.make_route_desc(tokens, experts, k, dtype=B.F32)
    after = B.make_rms_norm_desc(tokens, width, parts=k, x_rows=rows)
    ws = A.workspace(max(B.linear_workspace(lin), B.route_workspace(route), 16))
    if dtype8:
        parts = [A.weight_in_8(up[e, i * inner:(i + 1) * inner]) for e in range(experts) for i in range(2)]
        w1, s1 = torch.stack([p[0] for p in parts]).view(experts, 2 * inner, width).contiguous(), torch.stack([p[1] for p in parts])
        v1 = np.stack([p[2] for p in parts]).reshape(experts, 2 * inner, width)
        parts = [A.weight_in_8(down[e]) for e in range(experts)]
        w2, s2, v2 = torch.stack([p[0] for p in parts]).contiguous(), torch.stack([p[1] for p in parts]), np.stack([p[2] for p in parts])
        xq, xs = empty(tokens, width, t=torch.uint8), empty(tokens, B.scale_blocks(width), t=torch.float32)
        mq, ms = empty(rows, inner, t=torch.uint8), empty(rows, B.scale_blocks(inner), t=torch.float32)
        first = B.make_grouped_linear_desc(experts, rows, inner, width, dtype=B.E4M3, act=B.ACT_SILU, gated=True, x_rows=tokens)
        second = B.make_grouped_linear_desc(experts, rows, width, inner, dtype=B.E4M3)
        quant = B.make_quantize_desc(rows, inner)
    else:
        w1, w2 = up.to(ty), down.to(ty)
        v1, v2 = A.f64(w1), A.f64(w2)
        first = B.make_grouped_linear_desc(experts, rows, inner, width, act=B.ACT_SILU, gated=True, x_rows=tokens)
        second = B.make_grouped_linear_desc(experts, rows, width, inner)

    def calls(stream=None):
        s = stream or torch.cuda.current_stream()
        B.rms_norm_fwd(norm, h, gain, y=x, q=xq if dtype8 else None, scales=xs if dtype8 else None, stream=s)
        B.linear_fwd(lin, x, w_route, logits, workspace=ws, stream=s)
        B.route_fwd(route, logits, ids, weights, starts, source, place, workspace=ws, stream=s)
        if dtype8:
            B.grouped_linear_fwd(first, xq, w1, starts, mid, x_scales=xs, w_scales=s1, source=source, stream=s)
            B.quantize_fwd(quant, mid, mq, ms, stream=s)
            B.grouped_linear_fwd(second, mq, w2, starts, out, x_scales=ms, w_scales=s2, stream=s)
        else:
            B.grouped_linear_fwd(first, x, w1, starts, mid, source=source, stream=s)
            B.grouped_linear_fwd(second, mid, w2, starts, out, stream=s)
        B.rms_norm_fwd(after, out, gain, y=y2, residual=h, h=h2, source=place, weights=weights, stream=s)

    def check():
        # against the layer in 64 bits, token by token, with the experts that the router chose
        hv, xv = A.f64(h), A.f64(x)
        ref = hv / np.sqrt((hv ** 2).mean(1, keepdims=True) + 1e-5) * A.f64(gain)
        assert np.abs(xv - ref).max() <= 2.0 ** -7 * np.abs(ref).max()
        r5 = A.oa.route(A.f64(logits), k)
        assert np.array_equal(ids.cpu().numpy(), r5[0])
        x_in = A.numbers(xq) * A.oa.spread(A.f64(xs), ref.shape) if dtype8 else xv
        want = hv.copy()
        for t in range(tokens):
            for j in range(k):
                e = r5[0][t, j]
                g = v1[e] @ x_in[t]
                m = A.osq.act(g[:inner], "silu") * g[inner:]
                want[t] += r5[1][t, j] * (v2[e] @ m)
        # the inner rows are rounded to 16 bits (2^-8), in the other case then to 8 (2^-4, of every value alone: its square
        # root's share of a sum), the outer to 16
        err = np.linalg.norm(A.f64(h2) - want) / np.linalg.norm(want - hv)
        assert err <= (2.0 ** -4 if dtype8 else 2.0 ** -6), err
        g2 = want / np.sqrt((want ** 2).mean(1, keepdims=True) + 1e-5) * A.f64(gain)
        assert np.linalg.norm(A.f64(y2) - g2) <= (2.0 ** -4 if dtype8 else 2.0 ** -6) * np.linalg.norm(g2)

    return calls, [x, logits, ids, weights, starts, source, place, mid, out, h2, y2], check, h


@pytest.mark.parametrize("dtype8", [False, True])
@pytest.mark.parametrize("tokens", [1, 20, 400])
def test_expert_layer_from_norm_to_norm(A, dtype8, tokens):
    import torch
    calls, outs, check, _ = layer(A, dtype8, tokens)
    calls()
    torch.cuda.synchronize()
    check()


@pytest.mark.parametrize("dtype8", [False, True])
@pytest.mark.parametrize("tokens", [5, 300])
def test_expert_layer_captured_and_on_two_streams(A, dtype8, tokens):
    import torch
    first, second = [layer(A, dtype8, tokens, seed=s) for s in (3, 4)]
    for c in (first, second):
        c[0]()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        first[0]()
    side = torch.cuda.Stream()
    for turn in range(4):
        h = first[3]
        h.copy_(A.Rng(30 + turn).normal(tuple(h.shape), "bf16"))
        first[0]()
        second[0]()
        torch.cuda.synchronize()
        want = [[t.clone() for t in c[1]] for c in (first, second)]
        for c in (first, second):
            for t in c[1]:
                t.zero_()
        torch.cuda.synchronize()
        graph.replay()                                  # the one replayed while the other runs on another stream
        second[0](side)
        torch.cuda.synchronize()
        for c, w in zip((first, second), want):
            assert all(torch.equal(a, b) for a, b in zip(c[1], w)), "replay %d" % turn


# ---- every form that the rules choose between, with several whole steps and a rest ---------------------------
def kernels_of(call):
    """Names of the product kernels that a call launches."""
    import torch
    from torch.profiler import ProfilerActivity, profile
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    return [e.name for e in p.events() if "linear_" in e.name or "grouped_" in e.name]


def is_form(names, kernel, numbers):
    """Whether a call's first kernel is `kernel` with these leading numbers among its template arguments."""
    if not names:
        pytest.skip("the profiler shows no kernels here")
    # (some demanglers do not know the 16-bit types and lose the argument behind them)
    tail = "".join("Li%dE" % v for v in numbers) if names[0].startswith("_Z") else ", ".join(str(v) for v in numbers[1:])
    assert kernel in names[0] and tail in names[0], (kernel, numbers, names)


Q8_FORMS = [("linear_q8_rows_kernel", (1, 1), "bf16", 3, 300, 5000, True), ("linear_q8_rows_kernel", (1, 2), "f16", 9, 5000, 2700, False),
            ("linear_q8_rows_kernel", (1, 3), "f32", 16, 9000, 2200, False), ("linear_q8_rows_kernel", (2, 3), "bf16", 32, 8512, 2048, False),
            ("linear_q8_rows_kernel", (2, 2), "f32", 20, 7000, 2500, False), ("linear_q8_rows_kernel", (4, 1), "bf16", 50, 2000, 1300, False),
            ("linear_q8_rows_kernel", (4, 3), "f16", 64, 9000, 1500, False), ("linear_q8_kernel", (64, 128), "bf16", 70, 8512, 1111, False),
            ("linear_q8_kernel", (64, 128), "f16", 130, 1030, 4100, True), ("linear_q8_kernel", (64, 128), "f32", 200, 1000, 8200, True),
            ("linear_q8_kernel", (128, 128), "bf16", 2000, 3200, 4128, False), ("linear_q8_kernel", (128, 128), "f16", 1990, 3207, 4103, False),
            ("linear_q8_kernel", (256, 256), "bf16", 4100, 4097, 1160, False), ("linear_q8_kernel", (256, 256), "f16", 4096, 4096, 1283, False)]


@pytest.mark.parametrize("kernel,numbers,dtype,m,n,k,cut", Q8_FORMS)
def test_linear_q8_forms(A, kernel, numbers, dtype, m, n, k, cut):
    import torch
    B, (code, ty) = A.B, A.TYPES[dtype][:2]
    A.run_linear_q8(m, n, k, dtype, act="silu", pad=4)
    desc = B.make_linear_q8_desc(m, n, k, dtype=code)
    assert (B.linear_q8_workspace(desc) > 0) == cut
    row = desc.x_stride
    x, w = [torch.zeros((r, row), device="cuda", dtype=torch.uint8) for r in (m, n)]
    xs, ws = torch.ones((m, B.scale_blocks(k)), device="cuda"), torch.ones((B.scale_blocks(n), B.scale_blocks(k)), device="cuda")
    y, room = torch.empty((m, n), device="cuda", dtype=ty), A.workspace(B.linear_q8_workspace(desc))
    names = kernels_of(lambda: B.linear_q8_fwd(desc, x, xs, w, ws, y, workspace=room))
    is_form(names, kernel, numbers)
    assert len(names) == (2 if cut else 1)


GROUPED_FORMS = [("grouped_rows_kernel", (1, 2), "bf16", [1, 0, 3, 2], 200, 4200, True), ("grouped_rows_kernel", (1, 2), "f16", [5, 20, 0], 300, 2500, False),
                 ("grouped_direct_kernel", (64, 64, 2, 2), "bf16", [60, 1, 90, 80], 2000, 520, False),
                 ("grouped_direct_kernel", (64, 64, 2, 2), "f16", [60, 1, 90, 80], 1000, 456, True),
                 ("grouped_direct_kernel", (128, 128, 2, 4, 64, 4), "bf16", [200, 130, 1, 120], 600, 712, True),
                 ("grouped_direct_kernel", (128, 128, 2, 4, 64, 2), "f16", [200, 130, 1, 120], 6000, 264, False),
                 ("grouped_direct_kernel", (128, 128, 2, 4, 64, 2), "bf16", [200, 130, 1, 120], 3000, 392, True),
                 ("grouped_direct_kernel", (256, 256, 2, 4, 64, 2), "bf16", [900, 300, 0, 1200], 8000, 328, False),
                 ("grouped_direct_kernel", (256, 256, 2, 4, 64, 2), "f16", [900, 300, 0, 1200], 4000, 200, True),
                 ("grouped_rows_kernel", (1, 2), "f32", [3, 9, 0, 20], 500, 1300, True), ("grouped_rows_kernel", (1, 2), "f32", [60, 33, 1], 700, 700, False),
                 ("grouped_tiles_kernel", (64, 64, 2, 2), "f32", [90, 100, 0, 120], 3000, 140, False),
                 ("grouped_tiles_kernel", (64, 64, 2, 2), "bf16", [90, 100, 0, 120], 1500, 141, True),
                 ("grouped_tiles_kernel", (128, 128, 2, 2), "f32", [400, 300, 1, 500], 4000, 200, True),
                 ("grouped_tiles_kernel", (128, 128, 2, 2), "f16", [400, 300, 1, 500], 8000, 133, False),
                 ("linear_q8_rows_kernel", (1, 2), "e4m3", [1, 0, 17, 2], 300, 2900, True), ("linear_q8_rows_kernel", (1, 2), "e4m3", [5, 20, 0], 900, 5000, False),
                 ("linear_q8_kernel", (64, 128), "e4m3", [60, 1, 90, 80], 3000, 700, True), ("linear_q8_kernel", (64, 128), "e4m3", [100, 0, 200], 3000, 1100, False),
                 ("linear_q8_kernel", (128, 128), "e4m3", [900, 300, 0, 1200], 3600, 1040, False), ("linear_q8_kernel", (128, 128), "e4m3", [900, 300, 0, 1100], 1900, 1111, True),
                 ("linear_q8_kernel", (256, 256), "e4m3", [1500, 900, 0, 1700], 8200, 1036, False), ("linear_q8_kernel", (256, 256), "e4m3", [1500, 900, 0, 1700], 4400, 1040, True)]


@pytest.mark.parametrize("kernel,numbers,dtype,lengths,n,k,gated", GROUPED_FORMS)
def test_grouped_forms(A, kernel, numbers, dtype, lengths, n, k, gated):
    import torch
    B, rows, groups, halves = A.B, sum(lengths), len(lengths), 2 if gated else 1
    A.run_grouped(lengths, n, k, dtype, act="silu", gated=gated, gather=len(lengths) == 4)
    code = B.E4M3 if dtype == "e4m3" else A.TYPES[dtype][0]
    desc = B.make_grouped_linear_desc(groups, rows, n, k, dtype=code, gated=gated)
    ty = torch.uint8 if dtype == "e4m3" else A.TYPES[dtype][1]
    x, w = torch.zeros((rows, desc.x_stride), device="cuda", dtype=ty), torch.zeros((groups, halves * n, desc.w_stride), device="cuda", dtype=ty)
    y = torch.empty((rows, n), device="cuda", dtype=torch.bfloat16 if dtype == "e4m3" else ty)
    kw = dict(x_scales=torch.ones((rows, B.scale_blocks(k)), device="cuda"),
              w_scales=torch.ones((groups, halves, B.scale_blocks(n), B.scale_blocks(k)), device="cuda")) if dtype == "e4m3" else {}
    starts = A.i32([0] + np.cumsum(lengths).tolist())
    names = kernels_of(lambda: B.grouped_linear_fwd(desc, x, w, starts, y, **kw))
    is_form(names, kernel, numbers)
    assert len(names) == 1


# ---- passes over more bytes than the caches hold take another form -------------------------------------------
def test_norm_and_quantize_of_many_bytes(A):
    A.run_norm(4100, 2048, "f32", q=True)
    A.run_norm(4100, 2050, "f32", q=True, pad=1, offset=1)
    A.run_norm(2100, 1024, "bf16", parts=17, source="random", weights="random")
    eight(A, A.Rng(1).normal((8200, 2050)))
    eight(A, A.Rng(2).normal((270000, 130), "bf16"), pad=1, offset=1)


# ---- offsets that pass 32 bits: the last rows, experts and values of tensors of more than 2^32 bytes ------------
def test_norm_and_quantize_far_rows(A):
    import torch
    B, rows, width = A.B, 270000, 8192
    x, last = torch.zeros((rows, width), device="cuda", dtype=torch.bfloat16), A.Rng(1).normal((3, width), "bf16")
    x[-3:] = last
    gain = A.Rng(2).normal((width,), "bf16")
    out = []
    for t in (x, last):
        n = t.shape[0]
        y, q, s = torch.empty_like(t), torch.empty((n, width), device="cuda", dtype=torch.uint8), torch.empty((n, 64), device="cuda")
        B.rms_norm_fwd(B.make_rms_norm_desc(n, width), t, gain, y=y, q=q, scales=s)
        out.append([v[-3:].clone() for v in (y, q, s)])
        B.quantize_fwd(B.make_quantize_desc(n, width), t, q, s)
        out[-1] += [v[-3:].clone() for v in (q, s)]
    assert all(torch.equal(a, b) for a, b in zip(*out))
    # rows that are looked up
    source, y = A.i32([[rows - 1, rows - 3], [0, rows - 2]]), torch.empty((2, width), device="cuda", dtype=torch.bfloat16)
    B.rms_norm_fwd(B.make_rms_norm_desc(2, width, parts=2, x_rows=rows), x, None, h=y, source=source)
    assert torch.equal(y[0], (last[2].float() + last[0].float()).bfloat16()) and torch.equal(y[1], last[1])


def test_linear_q8_far_rows(A):
    import torch
    B, m, n, k = A.B, 270000, 72, 8192
    small, xs, xv = A.in_8(A.Rng(1).normal((5, k)))
    w, ws, wv = A.weight_in_8(A.Rng(2).normal((n, k), "f32", k ** -0.5))
    x, scales = torch.zeros((m, k), device="cuda", dtype=torch.uint8), torch.ones((m, 64), device="cuda")
    x[-5:], scales[-5:] = small, xs
    y = torch.full((m, n), A.GUARD, device="cuda", dtype=torch.bfloat16)
    desc = B.make_linear_q8_desc(m, n, k)
    B.linear_q8_fwd(desc, x, scales, w, ws, y, workspace=A.workspace(B.linear_q8_workspace(desc)))
    ref, d = A.osq.linear(xv, wv)
    A.close(y[-5:], ref, d, "bf16", (k + 64) * 2.0 ** -24 + 7 * 2.0 ** -13, "the last rows")
    assert not y[:-5].any()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [3, 150])
def test_grouped_far_experts_and_rows(A, dtype, rows):
    import torch
    B, E, n, k = A.B, 40 if dtype == "bf16" else 70, 4096, 8192
    far_rows = 270000 if dtype == "bf16" else 40000        # 8-bit rows that are looked up end at 2^31 bytes
    ty = torch.bfloat16 if dtype == "bf16" else torch.uint8
    w, x = torch.zeros((E, 2 * n, k), device="cuda", dtype=ty), torch.zeros((far_rows, k), device="cuda", dtype=ty)
    r, kw = A.Rng(rows), {}
    if dtype == "bf16":
        last, lw = r.normal((rows, k), dtype), r.normal((48, k), dtype, k ** -0.5)
        xv, wv = A.f64(last), A.f64(lw)
    else:
        last, xs, xv = A.in_8(r.normal((rows, k)))
        parts = [A.weight_in_8(r.normal((24, k), "f32", k ** -0.5)) for _ in range(2)]
        lw, wv = torch.cat([p[0] for p in parts]), np.concatenate([p[2] for p in parts])
        x_scales, w_scales = torch.ones((far_rows, 64), device="cuda"), torch.ones((E, 2, 32, 64), device="cuda")
        x_scales[-rows:], w_scales[-1, :, -1:] = xs, torch.stack([p[1] for p in parts])   # the last columns' block
        kw = dict(x_scales=x_scales, w_scales=w_scales)
    x[-rows:], w[-1, n - 24:n], w[-1, 2 * n - 24:] = last, lw[:24], lw[24:]
    y = torch.empty((rows, n), device="cuda", dtype=torch.bfloat16)
    desc = B.make_grouped_linear_desc(E, rows, n, k, dtype=B.BF16 if dtype == "bf16" else B.E4M3, act=B.ACT_SILU, gated=True, x_rows=far_rows)
    source = A.i32(list(range(far_rows - rows, far_rows)))
    B.grouped_linear_fwd(desc, x, w, A.i32([0] * E + [rows]), y, source=source, **kw)
    ref, d = A.oa.grouped(xv, wv[None], [0, rows], None, "silu", True)
    share = (k + 64) * 2.0 ** -24 + 2.0 ** -19 + (7 * 2.0 ** -13 if dtype == "e4m3" else 0.0)
    A.close(y[:, -24:], ref, d, "bf16", share, "the last expert's last columns")
    assert not y[:, :-24].any()
    if dtype == "e4m3":
        many = B.make_grouped_linear_desc(E, rows, n, k, dtype=B.E4M3, gated=True, x_rows=1 << 18)
        with pytest.raises(B.WpkError) as e:
            B.grouped_linear_fwd(many, x, w, A.i32([0] * E + [rows]), y, source=source, **kw)
        assert e.value.status == B.E_UNSUPPORTED


def test_two_graphs_that_share_a_workspace(A):
    import torch
    B, calls = A.B, []
    room = None
    for seed, (m, n, k) in enumerate(((3, 300, 5000), (130, 1030, 4096))):
        x, xs, _ = A.in_8(A.Rng(seed).normal((m, k)))
        w, ws, _ = A.weight_in_8(A.Rng(seed + 9).normal((n, k)))
        desc, y = B.make_linear_q8_desc(m, n, k), torch.empty((m, n), device="cuda", dtype=torch.bfloat16)
        assert B.linear_q8_workspace(desc) > 0
        calls.append((desc, x.contiguous() if x.stride(0) == desc.x_stride else x, xs, w, ws, y))
        calls[-1][0].x_stride, calls[-1][0].w_stride = x.stride(0), w.stride(0)
    room = A.workspace(max(B.linear_q8_workspace(c[0]) for c in calls))
    run = lambda c: B.linear_q8_fwd(*c, workspace=room, stream=torch.cuda.current_stream())
    graphs, want = [], []
    for c in calls:
        run(c)
        torch.cuda.synchronize()
        want.append(c[5].clone())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run(c)
    for turn in range(3):
        for c in calls:
            c[5].zero_()
        for g in graphs if turn % 2 else graphs[::-1]:
            g.replay()
        run(calls[turn % 2])
        torch.cuda.synchronize()
        assert all(torch.equal(c[5], t) for c, t in zip(calls, want)), "replay %d" % turn
