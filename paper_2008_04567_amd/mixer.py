"""A state space mixer layer as a serving program runs it, on the sequence layers' entry points.

    out = h + (silu(z) * scan(silu(conv(x B C)), dt)) W_out^T        [z | x B C | dt] = h W_in^T

``Mixer`` owns the weights and a pool of states (one entry per request: the convolution's last inputs and the scan's
state); ``prompt`` takes the ragged prompts of some requests, ``step`` one token of each.  Tensors and streams are
PyTorch's; every operation is the library's.  An example: its weights are random.  Without ``norm`` it is the four calls alone; with
it h goes through an RMS norm before the first product, and the scan's rows through one of as many groups before the last.

What a call returns is the plan's own buffer: it holds until the plan's next call.  A plan's calls share buffers and
workspace, so they belong on one stream, or in order; so do calls of any plans that use the same entries of the pool.

``python -m paper_2008_04567_amd.mixer`` takes a batch of prompts through a layer, continues them token by token with the
step captured in a HIP graph, and prints what both take.
"""
import argparse
import math

import torch

from . import binding as B

_CODES = {torch.float32: B.F32, torch.bfloat16: B.BF16, torch.float16: B.F16}


class Mixer:
    def __init__(self, width, heads, head_dim, groups, state_dim, conv_width=4, slots=64, dtype=torch.bfloat16, seed=0,
                 device="cuda", norm=False):
        self.width, self.heads, self.head_dim = width, heads, head_dim
        self.groups, self.state_dim, self.conv_width, self.slots = groups, state_dim, conv_width, slots
        self.dtype, self.code, self.device = dtype, _CODES[dtype], device
        self.inner = heads * head_dim
        self.conv_channels = self.inner + 2 * groups * state_dim
        rows = self.inner + self.conv_channels + heads
        self.row = (rows + 7) // 8 * 8            # of the first product, its columns filled up to whole 16-byte pieces
        g = torch.Generator(device=device).manual_seed(seed)
        rnd = lambda shape, scale: (torch.randn(shape, generator=g, device=device) * scale).to(dtype)
        self.w_in = rnd((self.row, width), width ** -0.5)
        self.w_out = rnd((width, self.inner), self.inner ** -0.5)
        self.w_conv, self.b_conv = rnd((self.conv_channels, conv_width), conv_width ** -0.5), rnd((self.conv_channels,), 0.1)
        self.a = -(1.0 + 15.0 * torch.rand(heads, generator=g, device=device))
        d0 = torch.exp(math.log(1e-3) + math.log(100.0) * torch.rand(heads, generator=g, device=device))
        self.dt_bias = d0 + torch.log(-torch.expm1(-d0))
        self.d = torch.ones(heads, device=device)
        self.norm = norm
        self.gain_in, self.gain_out = torch.ones(width, device=device, dtype=dtype), torch.ones(self.inner, device=device, dtype=dtype)
        self.conv_state = torch.zeros((slots, conv_width - 1, self.conv_channels), device=device, dtype=dtype)
        self.scan_state = torch.zeros((slots, heads, head_dim, state_dim), device=device)

    def plan(self, sequences, tokens, max_length):
        """Descriptors and room for calls of this shape; a program keeps one per shape it serves."""
        return _Plan(self, sequences, tokens, max_length)

    def prompt(self, plan, h, starts, slot_map, resume=None, stream=None):
        """h: rows of the requests' tokens one after another, [tokens][width] (rows may be slices of longer ones).  starts
        [requests + 1], slot_map [requests] and resume [requests] are int32 on the GPU: without starts every request has the
        plan's max_length tokens, without slot_map request i has entry i, without resume all start afresh."""
        if resume is None:
            resume = plan.fresh
        h = self._check(plan, h, slot_map, starts=(starts, plan.sequences + 1), resume=(resume, plan.sequences))
        return plan.run(h, starts, slot_map, resume, False, stream)

    def step(self, plan, h, slot_map, stream=None):
        """One token of every request, row i that of request i."""
        if plan.tokens != plan.sequences or plan.max_length != 1:
            raise ValueError("the plan is not one of a token a request")
        h = self._check(plan, h, slot_map)
        return plan.run(h, None, slot_map, None, True, stream)

    def _check(self, plan, h, slot_map, **others):
        """What the library cannot see from addresses.  Returns the rows of h."""
        if plan.m is not self:
            raise ValueError("the plan is another layer's")
        want = (plan.tokens, self.width)
        if h.dim() != 2 and h.is_contiguous() and h.shape[-1] == self.width:
            h = h.view(-1, self.width)
        if tuple(h.shape) != want or h.dtype != self.dtype or h.device != self.w_in.device:
            raise ValueError("h is %s %s on %s, not %s %s on %s" % (tuple(h.shape), h.dtype, h.device, want, self.dtype,
                                                                    self.w_in.device))
        if h.stride(1) != 1 or (plan.tokens > 1 and h.stride(0) < self.width):
            raise ValueError("h: values of a row stand one after another, rows apart")
        for name, (t, n) in dict(others, slot_map=(slot_map, plan.sequences)).items():
            if t is not None and not (torch.is_tensor(t) and t.dtype == torch.int32 and tuple(t.shape) == (n,) and t.is_contiguous() and
                    t.device == h.device):
                raise ValueError("%s is not %d int32 numbers on %s" % (name, n, h.device))
        if not h.is_cuda:
            raise ValueError("the layer is not on the GPU")
        return h


class _Plan:
    def __init__(self, m, sequences, tokens, max_length):
        self.m, inner, gn = m, m.inner, m.groups * m.state_dim
        self.sequences, self.tokens, self.max_length = sequences, tokens, max_length
        empty = lambda *shape, dtype=m.dtype: torch.empty(shape, device=m.device, dtype=dtype)
        self.row, self.conv, self.y, self.out = (empty(tokens, m.row), empty(tokens, m.conv_channels), empty(tokens, inner),
                                                 empty(tokens, m.width))
        self.fresh = torch.zeros(sequences, device=m.device, dtype=torch.int32)
        self.z, self.xbc, self.dt = (self.row[:, :inner], self.row[:, inner:inner + m.conv_channels],
                                     self.row[:, inner + m.conv_channels:])
        self.x, self.b, self.c = self.conv[:, :inner], self.conv[:, inner:inner + gn], self.conv[:, inner + gn:]
        self.lin_in = B.make_linear_desc(tokens, m.row, m.width, dtype=m.code)
        self.lin_out = B.make_linear_desc(tokens, m.width, inner, dtype=m.code)
        self.conv_desc = B.make_causal_conv_desc(sequences, tokens, m.conv_channels, m.conv_width, max_length=max_length,
                                                 slots=m.slots, dtype=m.code, act=B.ACT_SILU, x_stride=m.row)
        self.ssm_desc = B.make_ssm_desc(sequences, tokens, m.heads, m.head_dim, m.groups, m.state_dim, max_length=max_length,
                                        slots=m.slots, dtype=m.code, dt_softplus=True, x_stride=m.conv_channels,
                                        b_stride=m.conv_channels, c_stride=m.conv_channels, z_stride=m.row, dt_stride=m.row)
        self.normed = empty(tokens, m.width) if m.norm else None
        self.norm_in = B.make_rms_norm_desc(tokens, m.width, dtype=m.code)
        self.norm_out = B.make_rms_norm_desc(tokens, inner, groups=m.groups, dtype=m.code)
        need = max(B.linear_workspace(self.lin_in), B.linear_workspace(self.lin_out), B.ssm_workspace(self.ssm_desc))
        self.workspace = torch.empty(max(16, need), device=m.device, dtype=torch.uint8)

    def run(self, h, starts, slot_map, resume, step, stream):
        m = self.m
        s = stream if stream is not None else torch.cuda.current_stream()
        row, x = h.stride(0) if self.tokens > 1 else m.width, h
        self.lin_in.x_stride = self.lin_out.residual_stride = self.norm_in.x_stride = row
        if m.norm:
            x = self.normed
            self.lin_in.x_stride = m.width
            B.rms_norm_fwd(self.norm_in, h, m.gain_in, y=x, stream=s)
        B.linear_fwd(self.lin_in, x, m.w_in, self.row, workspace=self.workspace, stream=s)
        conv = dict(bias=m.b_conv, slot_map=slot_map, state_in=m.conv_state, state_out=m.conv_state, stream=s)
        scan = dict(d=m.d, z=self.z, dt_bias=m.dt_bias, slot_map=slot_map, state_in=m.scan_state, state_out=m.scan_state,
                    stream=s)
        if step:
            B.causal_conv1d_step(self.conv_desc, self.xbc, m.w_conv, self.conv, **conv)
            B.ssm_scan_step(self.ssm_desc, self.x, self.dt, m.a, self.b, self.c, self.y, **scan)
        else:
            B.causal_conv1d_fwd(self.conv_desc, self.xbc, m.w_conv, self.conv, starts=starts, resume=resume, **conv)
            B.ssm_scan_fwd(self.ssm_desc, self.x, self.dt, m.a, self.b, self.c, self.y, starts=starts, resume=resume,
                           workspace=self.workspace, **scan)
        if m.norm:
            B.rms_norm_fwd(self.norm_out, self.y, m.gain_out, y=self.y, stream=s)
        B.linear_fwd(self.lin_out, self.y, m.w_out, self.out, residual=h, workspace=self.workspace, stream=s)
        return self.out


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--heads", type=int, default=64)
    ap.add_argument("--head-dim", type=int, default=64)
    ap.add_argument("--groups", type=int, default=1)
    ap.add_argument("--state-dim", type=int, default=128)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--length", type=int, default=512, help="of the longest prompt")
    ap.add_argument("--tokens", type=int, default=32, help="steps behind the prompts")
    args = ap.parse_args()

    m = Mixer(args.width, args.heads, args.head_dim, args.groups, args.state_dim, slots=args.requests)
    lengths = [max(1, args.length * (i + 1) // args.requests) for i in range(args.requests)]
    starts = torch.tensor([0] + torch.tensor(lengths).cumsum(0).tolist(), device="cuda", dtype=torch.int32)
    slots = torch.arange(args.requests, device="cuda", dtype=torch.int32)
    h = torch.randn(sum(lengths), args.width, device="cuda").to(m.dtype)
    plan = m.plan(args.requests, sum(lengths), max(lengths))
    one = m.plan(args.requests, args.requests, 1)
    token = torch.randn(args.requests, args.width, device="cuda").to(m.dtype)

    def timed(fn, n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(n):
            fn()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / n * 1e3

    m.prompt(plan, h, starts, slots)
    m.step(one, token, slots)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.step(one, token, slots)
    print("prompts: %d requests, %d tokens: %.1f us a layer" % (args.requests, sum(lengths),
                                                                timed(lambda: m.prompt(plan, h, starts, slots), 20)))
    print("step of %d requests: %.1f us a layer, %.1f us replayed from a graph" % (
        args.requests, timed(lambda: m.step(one, token, slots), args.tokens), timed(graph.replay, args.tokens)))
    assert torch.isfinite(one.out.float()).all() and torch.isfinite(plan.out.float()).all()


if __name__ == "__main__":
    main()
