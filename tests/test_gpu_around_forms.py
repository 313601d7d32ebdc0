"""GPU tests of which kernel, with all of its template arguments, the rules choose for 8-bit products and products by expert."""
import numpy as np
import pytest

from tests import parity as PT
from tests.kernel_names import parse

pytestmark = pytest.mark.gpu

ROWS, TILES = "linear_q8_rows_kernel", "linear_q8_kernel"
T64, T128, T256 = (64, 128, 1, 4, 2), (128, 128, 2, 4, 2), (256, 256, 2, 4, 2)


@pytest.fixture(scope="module")
def A():
    PT.torch_dev()
    from tests import around_case
    return around_case


def forms_of(call):
    """(kernel, type, numbers) of every product kernel that a call launches."""
    from tests.test_gpu_around import kernels_of
    names = kernels_of(call)
    if not names:
        pytest.skip("the profiler shows no kernels here")
    read = [parse(n) for n in names]
    assert all(read), names
    return read


# rows, columns, reduction; whether the reduction is cut
Q8 = [(ROWS, (1, 1, 2), "bf16", 3, 300, 5000, True), (ROWS, (1, 2, 2), "f16", 9, 5000, 2700, False), (ROWS, (1, 3, 1), "f32", 16, 9000, 2200, False),
      (ROWS, (2, 3, 2), "bf16", 32, 8512, 2048, False), (ROWS, (2, 2, 1), "f32", 20, 7000, 2500, False), (ROWS, (4, 1, 1), "bf16", 50, 2000, 1300, False),
      (ROWS, (4, 3, 1), "f16", 64, 9000, 1500, False), (TILES, T64, "bf16", 65, 8512, 1111, False), (TILES, T64, "f16", 130, 1030, 4100, True),
      (TILES, T64, "f32", 200, 1000, 8200, True), (TILES, T64, "f32", 4096, 4096, 1283, False), (TILES, T128, "bf16", 2000, 3200, 4128, False),
      (TILES, T128, "f16", 1990, 3207, 4103, False), (TILES, T256, "bf16", 4100, 4097, 1160, False), (TILES, T256, "f16", 4096, 4096, 1283, False)]


@pytest.mark.parametrize("kernel,numbers,dtype,m,n,k,cut", Q8)
def test_linear_q8(A, kernel, numbers, dtype, m, n, k, cut):
    import torch
    B, (code, ty) = A.B, A.TYPES[dtype][:2]
    desc = B.make_linear_q8_desc(m, n, k, dtype=code)
    assert (B.linear_q8_workspace(desc) > 0) == cut
    x, w = [torch.zeros((r, desc.x_stride), device="cuda", dtype=torch.uint8) for r in (m, n)]
    xs, ws = torch.ones((m, B.scale_blocks(k)), device="cuda"), torch.ones((B.scale_blocks(n), B.scale_blocks(k)), device="cuda")
    y, room = torch.empty((m, n), device="cuda", dtype=ty), A.workspace(B.linear_q8_workspace(desc))
    got = forms_of(lambda: B.linear_q8_fwd(desc, x, xs, w, ws, y, workspace=room))
    assert got == [(kernel, dtype, numbers + (0, 0))] + [("linear_join_kernel", dtype, ())] * cut


# rows of the experts, columns, reduction; numbers without the two or one that say by expert and gated
R, D, T = "grouped_rows_kernel", "grouped_direct_kernel", "grouped_tiles_kernel"
GROUPED = [(R, (1, 2, 4), "bf16", [1, 0, 3, 2], 200, 4200, True), (R, (1, 2, 4), "f16", [5, 20, 0], 300, 2500, False),
           (D, (64, 64, 2, 2, 64, 4), "bf16", [60, 1, 90, 80], 2000, 520, False), (D, (64, 64, 2, 2, 64, 4), "f16", [60, 1, 90, 80], 1000, 456, True),
           (D, (128, 128, 2, 4, 64, 4), "bf16", [200, 130, 1, 120], 600, 712, True), (D, (128, 128, 2, 4, 64, 2), "f16", [200, 130, 1, 120], 6000, 264, False),
           (D, (128, 128, 2, 4, 64, 2), "bf16", [200, 130, 1, 120], 3000, 392, True), (D, (256, 256, 2, 4, 64, 2), "bf16", [900, 300, 0, 1200], 8000, 328, False),
           (D, (256, 256, 2, 4, 64, 2), "f16", [900, 300, 0, 1200], 4000, 200, True), (R, (1, 2, 2), "f32", [3, 9, 0, 20], 500, 1300, True),
           (R, (1, 2, 2), "f32", [60, 33, 1], 700, 700, False), (T, (64, 64, 2, 2), "f32", [90, 100, 0, 120], 3000, 140, False),
           (T, (64, 64, 2, 2), "bf16", [90, 100, 0, 120], 1500, 141, True), (T, (128, 128, 2, 2), "f32", [400, 300, 1, 500], 4000, 200, True),
           (T, (128, 128, 2, 2), "f16", [400, 300, 1, 500], 8000, 133, False), (ROWS, (1, 2, 2), "e4m3", [1, 0, 17, 2], 300, 2900, True),
           (ROWS, (1, 2, 2), "e4m3", [5, 20, 0], 900, 5000, False), (TILES, T64, "e4m3", [60, 1, 90, 80], 3000, 700, True),
           (TILES, T64, "e4m3", [100, 0, 200], 3000, 1100, False), (TILES, T128, "e4m3", [900, 300, 0, 1200], 3600, 1040, False),
           (TILES, T128, "e4m3", [900, 300, 0, 1100], 1900, 1111, True), (TILES, T256, "e4m3", [1500, 900, 0, 1700], 8200, 1036, False),
           (TILES, T256, "e4m3", [1500, 900, 0, 1700], 4400, 1040, True)]


@pytest.mark.parametrize("kernel,numbers,dtype,lengths,n,k,gated", GROUPED)
def test_grouped(A, kernel, numbers, dtype, lengths, n, k, gated):
    import torch
    B, rows, groups, halves, eight = A.B, sum(lengths), len(lengths), 2 if gated else 1, dtype == "e4m3"
    ty = torch.uint8 if eight else A.TYPES[dtype][1]
    desc = B.make_grouped_linear_desc(groups, rows, n, k, dtype=B.E4M3 if eight else A.TYPES[dtype][0], gated=gated)
    x, w = torch.zeros((rows, desc.x_stride), device="cuda", dtype=ty), torch.zeros((groups, halves * n, desc.w_stride), device="cuda", dtype=ty)
    y = torch.empty((rows, n), device="cuda", dtype=torch.bfloat16 if eight else ty)
    kw = dict(x_scales=torch.ones((rows, B.scale_blocks(k)), device="cuda"),
              w_scales=torch.ones((groups, halves, B.scale_blocks(n), B.scale_blocks(k)), device="cuda")) if eight else {}
    starts = A.i32([0] + np.cumsum(lengths).tolist())
    got = forms_of(lambda: B.grouped_linear_fwd(desc, x, w, starts, y, **kw))
    assert got == [(kernel, "bf16", numbers + (1, int(gated))) if eight else (kernel, dtype, numbers + (int(gated),))]
