"""A layer of experts as a serving program runs it between mixer layers, on the entry points around them.

    out = h + sum_j weight_j (silu(x G_e^T) * (x U_e^T)) D_e^T      x = RMS norm of h, e = the j-th expert of the token

``Experts`` owns the weights; ``run`` takes rows of any tokens.  The norm, the router, the products by expert and the
combination with the residual are the library's; nothing comes back to the host between them, so a call can be captured.  With
``eight`` the experts' weights and their inputs are 8-bit values with scales.  An example: its weights are random.

What a call returns is the plan's own buffer: it holds until the plan's next call.  A plan's calls share buffers and
workspace, so they belong on one stream, or in order.

``python -m paper_2008_04567_amd.experts`` takes a batch of tokens and single tokens of some requests through a layer, the latter
also captured in a HIP graph, and prints what they take.
"""
import argparse

import torch

from . import binding as B
from .mixer import _CODES


class Experts:
    def __init__(self, width, inner, experts, chosen, eight=False, dtype=torch.bfloat16, seed=0, device="cuda"):
        self.width, self.inner, self.experts, self.chosen, self.eight = width, inner, experts, chosen, eight
        self.dtype, self.code, self.device = dtype, _CODES[dtype], device
        g = torch.Generator(device=device).manual_seed(seed)
        rnd = lambda shape, scale: (torch.randn(shape, generator=g, device=device) * scale).to(dtype)
        self.gain = torch.ones(width, device=device, dtype=dtype)
        self.w_route = rnd((experts, width), width ** -0.5)
        up, down = rnd((experts, 2, inner, width), width ** -0.5), rnd((experts, 1, width, inner), inner ** -0.5)
        if eight:
            (self.w_up, self.s_up), (self.w_down, self.s_down) = weights_in_8(up), weights_in_8(down)
        else:
            self.w_up, self.w_down, self.s_up, self.s_down = up, down, None, None

    def plan(self, tokens):
        """Descriptors and room for calls of so many tokens; a program keeps one per number it serves."""
        return _Plan(self, tokens)

    def run(self, plan, h, stream=None):
        """h: [tokens][width], rows may be slices of longer ones.  Returns the plan's out."""
        if plan.m is not self:
            raise ValueError("the plan is another layer's")
        want = (plan.tokens, self.width)
        if tuple(h.shape) != want or h.dtype != self.dtype or h.device != self.w_route.device:
            raise ValueError("h is %s %s on %s, not %s %s on %s" % (tuple(h.shape), h.dtype, h.device, want, self.dtype,
                                                                    self.w_route.device))
        if h.stride(1) != 1 or (plan.tokens > 1 and h.stride(0) < self.width):
            raise ValueError("h: values of a row stand one after another, rows apart")
        if not h.is_cuda:
            raise ValueError("the layer is not on the GPU")
        if h.device.index != torch.cuda.current_device():      # (launches go to the current one)
            raise ValueError("the layer is on %s, the current device is %d" % (h.device, torch.cuda.current_device()))
        return plan.run(h, stream)


def weights_in_8(w):
    """(e4m3 values in rows of whole 16 bytes, scales) of weights [experts][halves][n][k]: one for each block of 128 x 128."""
    experts, halves, n, k = w.shape
    nb, kb, block = B.scale_blocks(n), B.scale_blocks(k), B.SCALE_BLOCK
    full = torch.nn.functional.pad(w.float(), (0, kb * block - k, 0, nb * block - n)).view(experts, halves, nb, block, kb, block)
    scales = torch.clamp_min(full.abs().amax((3, 5)) / 448.0, 2.0 ** -110)
    q = (full / scales[:, :, :, None, :, None]).view(experts, halves, nb * block, kb * block)[:, :, :n, :k]
    out = torch.zeros((experts, halves, n, (k + 15) // 16 * 16), device=w.device, dtype=torch.float8_e4m3fn)
    out[..., :k] = q.to(torch.float8_e4m3fn)
    return out, scales


class _Plan:
    def __init__(self, m, tokens):
        self.m, self.tokens = m, tokens
        rows, width, inner, experts, k = tokens * m.chosen, m.width, m.inner, m.experts, m.chosen
        empty = lambda *shape, dtype=m.dtype: torch.empty(shape, device=m.device, dtype=dtype)
        in_8 = lambda r, c: (empty(r, (c + 15) // 16 * 16, dtype=torch.float8_e4m3fn), empty(r, B.scale_blocks(c), dtype=torch.float32))
        self.x, self.mid, self.rows, self.out = empty(tokens, width), empty(rows, inner), empty(rows, width), empty(tokens, width)
        self.logits, self.weights = empty(tokens, experts, dtype=torch.float32), empty(tokens, k, dtype=torch.float32)
        self.ids, self.place = empty(tokens, k, dtype=torch.int32), empty(tokens, k, dtype=torch.int32)
        self.starts, self.source = empty(experts + 1, dtype=torch.int32), empty(rows, dtype=torch.int32)
        (self.x8, self.x_scales), (self.mid8, self.mid_scales) = (in_8(tokens, width), in_8(rows, inner)) if m.eight else ((None,) * 2,) * 2
        code = B.E4M3 if m.eight else m.code
        self.norm = B.make_rms_norm_desc(tokens, width, dtype=m.code)
        self.router = B.make_linear_desc(tokens, experts, width, dtype=m.code, y_dtype=B.F32)
        self.route = B.make_route_desc(tokens, experts, k, dtype=B.F32)
        self.up = B.make_grouped_linear_desc(experts, rows, inner, width, dtype=code, y_dtype=m.code, act=B.ACT_SILU, gated=True,
                                             x_rows=tokens)
        self.quantize = B.make_quantize_desc(rows, inner, dtype=m.code)
        self.down = B.make_grouped_linear_desc(experts, rows, width, inner, dtype=code, y_dtype=m.code)
        self.combine = B.make_rms_norm_desc(tokens, width, parts=k, x_rows=rows, dtype=m.code)
        need = max(B.linear_workspace(self.router), B.route_workspace(self.route), B.grouped_linear_workspace(self.up),
                   B.grouped_linear_workspace(self.down))
        self.workspace = torch.empty(max(16, need), device=m.device, dtype=torch.uint8)

    def run(self, h, stream):
        m, ws = self.m, self.workspace
        s = stream if stream is not None else torch.cuda.current_stream()
        self.norm.x_stride = self.combine.residual_stride = h.stride(0) if self.tokens > 1 else m.width
        B.rms_norm_fwd(self.norm, h, m.gain, y=self.x, q=self.x8, scales=self.x_scales, stream=s)
        B.linear_fwd(self.router, self.x, m.w_route, self.logits, workspace=ws, stream=s)
        B.route_fwd(self.route, self.logits, self.ids, self.weights, self.starts, self.source, self.place, workspace=ws, stream=s)
        x, mid = (self.x8, self.mid8) if m.eight else (self.x, self.mid)
        B.grouped_linear_fwd(self.up, x, m.w_up, self.starts, self.mid, x_scales=self.x_scales, w_scales=m.s_up, source=self.source,
                             workspace=ws, stream=s)
        if m.eight:
            B.quantize_fwd(self.quantize, self.mid, self.mid8, self.mid_scales, stream=s)
        B.grouped_linear_fwd(self.down, mid, m.w_down, self.starts, self.rows, x_scales=self.mid_scales, w_scales=m.s_down,
                             workspace=ws, stream=s)
        B.rms_norm_fwd(self.combine, self.rows, None, residual=h, h=self.out, source=self.place, weights=self.weights, stream=s)
        return self.out


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--inner", type=int, default=1024)
    ap.add_argument("--experts", type=int, default=64)
    ap.add_argument("--chosen", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=8192, help="of the batch")
    ap.add_argument("--requests", type=int, default=16, help="that get a single token")
    args = ap.parse_args()

    def timed(fn, n=20):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(n):
            fn()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / n * 1e3

    for eight in (False, True):
        m = Experts(args.width, args.inner, args.experts, args.chosen, eight=eight)
        many, one = m.plan(args.tokens), m.plan(args.requests)
        h, token = [torch.randn(n, args.width, device="cuda").to(m.dtype) for n in (args.tokens, args.requests)]
        m.run(many, h)
        m.run(one, token)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.run(one, token)
        print("experts in %s: %d tokens %.1f us a layer; a token of %d requests %.1f us, %.1f us replayed from a graph" % (
            "8 bits" if eight else "16 bits", args.tokens, timed(lambda: m.run(many, h)), args.requests,
            timed(lambda: m.run(one, token)), timed(graph.replay)))
        assert torch.isfinite(one.out.float()).all() and torch.isfinite(many.out.float()).all()


if __name__ == "__main__":
    main()
