"""Inputs, calls and tolerances that the GPU tests of what stands around a mixer layer share.

Tolerances, with u and D as in sequence_case.py (a rounding to the output's type; sums of magnitudes):

  norm      s: parts + 1 terms, each with a product: e = (parts + 2) 2^-24 D.  The root of the mean: a sum of squares with at
            most 64 additions a lane and 16 over lanes and waves, and s's own errors: relative (96 + (parts + 2) sum D |s| /
            sum s^2) 2^-24, half of it and 2^-22 for the reciprocal root.  v: both, and three roundings
  8 bits    a value is off by half a step, 2^-4 of itself or 2^-10 of its scale, and by what v is off; two roundings on the way
            to q, three on the way to the scale
  products  k terms in 32 bits in any order, in 8 bits a scale's product and a multiplication for each block:
            (k + 64) 2^-24 D; activations as in sequence_case.py; a gated product's two factors both.  Into 16 bits, 8-bit
            products of eight neighbouring entries are added with 13 bits below the largest: seven of them lose at most 2^-13
            of it, 7 2^-13 D
  router    exp of a difference that is rounded: 2^-20 and 2^-23 |difference| of a weight; numbers of rows are exact
"""
import numpy as np
import torch

from oracle import around as oa
from oracle import sequence as osq
from paper_2008_04567_amd import binding as B
from tests.sequence_case import ACTS, GUARD, TYPES, Rng, f64, guard_intact, i32, out_rows, sliced  # noqa: F401
from tests.sequence_strict import close

F8 = torch.float8_e4m3fn


def rows_of_8(rows, width, extra=0):
    """Room for 8-bit rows, filled with a pattern; (view, buffer)."""
    stride = -(-width // 16) * 16 + extra
    buf = torch.full((rows * stride + 64,), 0x55, device="cuda", dtype=torch.uint8)
    return buf[:rows * stride].view(rows, stride)[:, :width], buf


def numbers(q):
    """The numbers that codes stand for."""
    return oa.e4m3_values()[q.cpu().numpy()]


def pattern_intact(view, buf):
    keep = view.clone()
    view.fill_(0x55)
    assert bool((buf == 0x55).all()), "write outside the 8-bit rows"
    view.copy_(keep)


def check_8(q, scales, v, tol, what):
    """q and scales against rows v that are off by at most tol."""
    ref_scale = np.empty(scales.shape)
    room = np.empty(scales.shape)
    for b in range(scales.shape[1]):
        c = slice(b * 128, (b + 1) * 128)
        ref_scale[:, b] = np.maximum(np.abs(v[:, c]).max(1) / 448.0, 2.0 ** -110)
        room[:, b] = tol[:, c].max(1) / 448.0
    got = f64(scales)
    assert (np.abs(got - ref_scale) <= room + 2.0 ** -22 * ref_scale).all(), what + ": scales"
    s = oa.spread(got, v.shape)
    err = np.abs(numbers(q) * s - v)
    allowed = 2.0 ** -4 * np.abs(v) * (1 + 2.0 ** -20) + 2.0 ** -10 * s + 2 * tol
    assert (err <= allowed).all(), "%s: 8-bit values, worst %.3g times the tolerance" % (what, (err / allowed).max())


def after_inputs(stream):
    """Inputs, workspaces and what outputs hold before a call are made on the current stream: a call on another waits for them."""
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())


def run_norm(rows, width, dtype, groups=1, parts=1, residual=True, gain=True, y=True, q=False, h=True, source=None, weights=None,
             x_rows=None, pad=0, offset=0, eps=1e-5, seed=1, scale=1.0, edit=None, in_place=None, stream=None):
    r = Rng(seed)
    code, ty = TYPES[dtype][:2]
    x_rows = x_rows or rows * parts
    x, xb = sliced(r.normal((x_rows, width), dtype, scale), width + pad, offset)
    res, _ = sliced(r.normal((rows, width), dtype, 2.0 * scale), width + pad, offset) if residual else (None, None)
    g = (1.0 + r.normal((width,), "f32", 0.2)).to(ty) if gain else None
    if isinstance(source, str):
        source = np.random.default_rng(seed).permutation(x_rows)[:rows * parts].reshape(rows, parts) if x_rows >= rows * parts \
            else np.random.default_rng(seed).integers(0, x_rows, (rows, parts))
    if isinstance(weights, str):
        weights = np.random.default_rng(seed + 1).uniform(0.1, 1.0, (rows, parts)).astype(np.float32)
    if edit:
        edit(x, res, g)
    before = f64(x), f64(res)
    yo, yb = out_rows(rows, width, width + pad, offset, ty) if y else (None, None)
    ho, hb = out_rows(rows, width, width + pad, offset, ty) if h else (None, None)
    if in_place:
        yo, ho, yb, hb = (x if "y" in in_place else yo), (res if "h" in in_place else ho), None, None
    qo, qb = rows_of_8(rows, width, 32) if q else (None, None)
    nb = oa.blocks(width)
    so, sb = out_rows(rows, nb, nb + 1, 0, torch.float32) if q else (None, None)
    desc = B.make_rms_norm_desc(rows, width, groups=groups, parts=parts, x_rows=x_rows, dtype=code, eps=eps, x_stride=width + pad,
                                residual_stride=width + pad, h_stride=width + pad, y_stride=width + pad,
                                q_stride=-(-width // 16) * 16 + 32, scale_stride=nb + 1)
    on_device = dict(source=None if source is None else i32(source), weights=None if weights is None else torch.from_numpy(weights).cuda())
    after_inputs(stream)
    B.rms_norm_fwd(desc, x, g, y=yo, q=qo, scales=so, residual=res, h=ho, stream=stream, **on_device)
    torch.cuda.synchronize()
    s, d, v = oa.rms_norm(before[0], f64(g), eps, before[1], groups, parts, source, weights)
    e = (parts + 2) * 2.0 ** -24
    with np.errstate(invalid="ignore", divide="ignore"):
        by, db = s.reshape(rows, groups, -1), d.reshape(rows, groups, -1)
        square = (by ** 2).sum(2, keepdims=True)
        rel = 0.5 * (96 * 2.0 ** -24 + 2 * e * (db * np.abs(by)).sum(2, keepdims=True) / np.maximum(square, 1e-300)) + 2.0 ** -22
        root = np.sqrt(square / by.shape[2] + eps)
        gn = (np.ones(width) if g is None else np.abs(f64(g))).reshape(groups, -1)
        tol = ((e * db + np.abs(by) * (rel + 2.0 ** -22)) / root * gn).reshape(s.shape)
    what = "norm %s" % ((rows, width, dtype, groups, parts),)
    for name, out, ref, share, buf in (("h", ho, s, e * d, hb), ("y", yo, v, tol, yb)):
        if out is not None:
            if buf is not None:
                guard_intact(out, buf)
            with np.errstate(invalid="ignore"):
                close(out, ref, np.where(np.isfinite(share), share, 0.0), dtype, 1.0, what + " " + name)
    if q:
        pattern_intact(qo, qb)
        guard_intact(so, sb)
        check_8(qo, so, v, tol, what)
    return dict(x=x, res=res, g=g, y=yo, h=ho, q=qo, scales=so, s=s, v=v)


def in_8(values, extra=0):
    """(codes in rows with `extra` more behind them, scales, the numbers they stand for) of float32 rows, random codes behind."""
    q, s = oa.quantize(values.cpu().numpy())
    view, buf = rows_of_8(*q.shape, extra=extra)
    buf.copy_(torch.from_numpy(np.random.default_rng(5).integers(0, 256, buf.numel()).astype(np.uint8)).cuda())
    view.copy_(torch.from_numpy(q.astype(np.float32)).cuda().to(F8).view(torch.uint8))
    return view, torch.from_numpy(s).cuda(), q * oa.spread(s, q.shape)


def weight_in_8(values, extra=0):
    """The same of a weight [n][k], with blocks of 128 x 128."""
    v = values.cpu().numpy().astype(np.float32)
    n, k = v.shape
    s = np.empty((oa.blocks(n), oa.blocks(k)), np.float32)
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            s[i, j] = max(np.abs(v[i * 128:(i + 1) * 128, j * 128:(j + 1) * 128]).max() / 448.0, 2.0 ** -110)
    q = oa.round_e4m3(v / oa.spread(s, v.shape, 128))
    view, buf = rows_of_8(n, k, extra)
    buf.fill_(0x7f)                                       # NaN behind the rows
    view.copy_(torch.from_numpy(q.astype(np.float32)).cuda().to(F8).view(torch.uint8))
    return view, torch.from_numpy(s).cuda(), q * oa.spread(s, v.shape, 128)


def workspace(nbytes):
    return torch.full((max(16, nbytes),), 255, device="cuda", dtype=torch.uint8)


def run_linear_q8(m, n, k, dtype, act="none", bias=True, residual=True, extra=0, pad=0, offset=0, seed=1, in_place=False, stream=None):
    r = Rng(seed)
    code, ty = TYPES[dtype][:2]
    x, xs, xv = in_8(r.normal((m, k)), extra)
    w, ws, wv = weight_in_8(r.normal((n, k), "f32", k ** -0.5), extra)
    bb = r.normal((n,), dtype) if bias else None
    res, _ = sliced(r.normal((m, n), dtype), n + pad, offset) if residual else (None, None)
    before = f64(res)
    y, yb = out_rows(m, n, n + pad, offset, ty)
    if in_place:
        y, yb = res, None
    desc = B.make_linear_q8_desc(m, n, k, dtype=code, act=ACTS[act], x_stride=x.stride(0), w_stride=w.stride(0), y_stride=n + pad,
                                 residual_stride=n + pad)
    room = workspace(B.linear_q8_workspace(desc))
    after_inputs(stream)
    B.linear_q8_fwd(desc, x, xs, w, ws, y, bias=bb, residual=res, workspace=room, stream=stream)
    torch.cuda.synchronize()
    if yb is not None:
        guard_intact(y, yb)
    ref, d = osq.linear(xv, wv, f64(bb), before, act)
    close(y, ref, d, dtype, (k + 64) * 2.0 ** -24 + (2.0 ** -21 if dtype == "f32" else 2.0 ** -19 + 7 * 2.0 ** -13),
          "8-bit product %s" % ((m, n, k, dtype, act),))
    return y


def run_grouped(lengths, n, k, dtype, y_dtype=None, act="none", gated=False, gather=False, before=0, behind=0, pad=0, offset=0,
                group_pad=0, x_rows=None, source=None, starts=None, seed=1, stream=None, fresh=True):
    """lengths: rows of the experts; `before` and `behind`: rows of no expert."""
    r = Rng(seed)
    groups, halves, rows = len(lengths), 2 if gated else 1, before + sum(lengths) + behind
    st = [before] + (before + np.cumsum(lengths)).tolist()
    code = B.E4M3 if dtype == "e4m3" else TYPES[dtype][0]
    y_dtype = y_dtype or ("bf16" if dtype == "e4m3" else dtype)
    if gather and source is None:
        x_rows = x_rows or max(1, rows // 2)
        source = np.random.default_rng(seed).integers(0, x_rows, rows)
    x_rows = x_rows or rows
    kw = {}
    if dtype == "e4m3":
        x, xs, xv = in_8(r.normal((x_rows, k)), extra=pad * 16)
        ws, wv, stride = [], [], -(-k // 16) * 16 + 16
        buf = torch.full((groups, halves * n + group_pad, stride), 0x7f, device="cuda", dtype=torch.uint8)
        for g in range(groups):
            for half in range(halves):
                q, s, v = weight_in_8(r.normal((n, k), "f32", k ** -0.5))
                buf[g, half * n:(half + 1) * n, :k] = q
                ws.append(s)
                wv.append(v)
        w, w_scales = buf, torch.stack(ws).contiguous()
        wv = np.stack(wv).reshape(groups, halves * n, k)
        kw = dict(x_scales=xs, w_scales=w_scales)
        strides = dict(x_stride=x.stride(0), w_stride=stride, w_group_stride=buf.stride(0))
    else:
        ty = TYPES[dtype][1]
        x, _ = sliced(r.normal((x_rows, k), dtype), k + pad, offset)
        buf = torch.full((groups * (halves * n + group_pad) * (k + pad) + offset,), float("nan"), device="cuda", dtype=ty)
        w = buf[offset:].view(groups, halves * n + group_pad, k + pad)
        w[:, :halves * n, :k] = r.normal((groups, halves * n, k), dtype, k ** -0.5)
        xv, wv = f64(x), f64(w[:, :halves * n, :k])
        strides = dict(x_stride=k + pad, w_stride=k + pad, w_group_stride=w.stride(0))
    y, yb = out_rows(rows, n, n + pad, offset, TYPES[y_dtype][1])
    desc = B.make_grouped_linear_desc(groups, rows, n, k, dtype=code, y_dtype=TYPES[y_dtype][0], act=ACTS[act], gated=gated,
                                      x_rows=x_rows, y_stride=n + pad, **strides)
    first = i32(st if starts is None else starts) if groups > 1 or before or behind else None
    kw.update(source=None if source is None else i32(source), workspace=workspace(B.grouped_linear_workspace(desc)))
    after_inputs(stream)
    B.grouped_linear_fwd(desc, x, w, first, y, stream=stream, **kw)
    torch.cuda.synchronize()
    guard_intact(y, yb)
    mine = slice(before, before + sum(lengths))
    ref, d = oa.grouped(xv, wv, st, None if source is None else np.asarray(source), act, gated)
    what = "grouped %s" % ((lengths if groups < 9 else groups, n, k, dtype, act, gated),)
    share = (k + 64) * 2.0 ** -24 + (2.0 ** -21 if y_dtype == "f32" else 2.0 ** -19)
    share += 7 * 2.0 ** -13 if dtype == "e4m3" and y_dtype != "f32" else 0.0
    close(y[mine], ref[mine], d[mine], y_dtype, share, what)
    if fresh:
        assert bool((y[:before] == GUARD).all()) and bool((y[before + sum(lengths):] == GUARD).all()), what + ": rows of no expert"
    return y


def run_route(logits, k, dtype, normalize=True, scale=1.0, order=True, pad=0, stream=None):
    code, ty = TYPES[dtype][:2]
    tokens, n = logits.shape
    l, _ = sliced(logits.to(ty), n + pad, 0)
    dev = dict(device="cuda")
    experts, weights = torch.full((tokens, k), -7, dtype=torch.int32, **dev), torch.full((tokens, k), GUARD, **dev)
    starts, source = torch.full((n + 2,), -7, dtype=torch.int32, **dev), torch.full((tokens * k + 1,), -7, dtype=torch.int32, **dev)
    place = torch.full((tokens, k), -7, dtype=torch.int32, **dev)
    desc = B.make_route_desc(tokens, n, k, dtype=code, normalize=normalize, scale=scale, logits_stride=n + pad)
    room = workspace(B.route_workspace(desc))
    after_inputs(stream)
    B.route_fwd(desc, l, experts, weights, *((starts, source, place) if order else ()), workspace=room, stream=stream)
    torch.cuda.synchronize()
    ref = oa.route(f64(l), k, normalize, scale)
    assert np.array_equal(experts.cpu().numpy(), ref[0]), "experts"
    lv = np.where(np.isnan(f64(l)), -np.inf, f64(l))
    with np.errstate(invalid="ignore"):
        far = np.abs(np.take_along_axis(lv, ref[0], 1) - lv.max(1, keepdims=True))
    got, want = f64(weights), ref[1]
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), "weights"
    ok = np.isfinite(want)
    tol = np.abs(want) * (2.0 ** -20 + 2.0 ** -23 * np.where(np.isfinite(far), far, 0.0)) + 2.0 ** -126
    assert (np.abs(got - want)[ok] <= tol[ok]).all(), "weights"
    if order:
        assert np.array_equal(starts.cpu().numpy(), np.append(ref[2], -7)), "starts"
        assert np.array_equal(source.cpu().numpy(), np.append(ref[3], -7)), "source"
        assert np.array_equal(place.cpu().numpy(), ref[4]), "place"
    return experts, weights, starts, source, place
