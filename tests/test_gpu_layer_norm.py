"""co3_layer_norm and co3_layer_norm_backward against the definition in 64 bits, over widths (odd ones, one, beyond every
change of kernel), row strides, alignments, types, batches of clients, and the gradients against differences.

Tolerances, with u = 2^-24 and n the width.  Statistics are sums of n fp32 terms in a tree of depth at most d = 40
(up to 32 in a thread, 5 levels in a warp, 16 warps in order count as one each of 2^-24): |error of the mean| <=
d u mean(|x|), |error of rstd| <= d u rstd (1 + (mean(|x|) rstd)).  Results: x_hat is formed from x - mean, so that its
error is the statistics' times its own size and d u mean(|x|) rstd; the types' own rounding (2^-24, 2^-11, 2^-8
relative, 2^-25 absolute for the smallest fp16) is added.  Gradients of gain and bias: sums over R rows, at most
R + 64 additions deep: (R + 64) u sum|term|, the expected error being far below.
"""
import numpy as np
import pytest
import torch

import paper_2204_08211_b200 as co3

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
U, DEPTH, EPS = 2.0 ** -24, 40, 1e-5


def rows_of(t, type_, pad, shift, fill=0.0):
    """A copy of t on the GPU as a view of a padded buffer that starts `shift` elements after its base."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + shift + 3,), fill, dtype=TYPES[type_], device="cuda")
    view = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return buf, view


def outside_untouched(buf, view, fill):
    seen = torch.zeros(buf.numel(), dtype=torch.bool)
    seen.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(True)
    return (buf.cpu()[~seen] == fill).all()


def forward64(x, w, b, eps=EPS):
    x = x.double().cpu()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    xh = (x - mean) * rstd
    y = xh
    if w is not None:
        y = y * w.double().cpu()
    if b is not None:
        y = y + b.double().cpu()
    return y, mean, rstd, xh


def check_forward(x, w, b, y, mean, rstd, type_):
    want, m, r, xh = forward64(x, w, b)
    size = x.double().cpu().abs().mean(1, keepdim=True)
    assert ((mean.double().cpu()[:, None] - m).abs() <= DEPTH * U * size).all()
    assert ((rstd.double().cpu()[:, None] - r).abs() <= DEPTH * U * r * (1 + size * r)).all()
    wa = 1.0 if w is None else w.double().cpu().abs()
    err = wa * (DEPTH * U * (xh.abs() * (1 + size * r) + size * r)) + 4 * U * (want.abs() + wa * xh.abs())
    err = err + UNIT[type_] * want.abs() + (2.0 ** -25 if type_ == "f16" else 0.0)
    assert ((y.double().cpu() - want).abs() <= err).all()


def run_backward(dy, x, w, mean, rstd, dx, grads, clients, stride, cols, accumulate=False, want_w=True, want_b=True):
    rows = x.shape[0] // clients
    ws = torch.empty(co3.co3_layer_norm_workspace_bytes(rows, cols, clients), dtype=torch.uint8, device="cuda")
    ws.fill_(0xCD)
    st = co3.co3_layer_norm_backward(dy, x, w, mean, rstd, dx, grads[1:] if want_w else None,
                                     grads[1 + cols:] if want_b else None, clients, stride, ws, accumulate)
    assert st == co3.OK, co3.co3_status_string(st)
    torch.cuda.synchronize()


def backward64(dy, x, w, mean, rstd):
    dy, x, r = dy.double().cpu(), x.double().cpu(), rstd.double().cpu()[:, None]
    xh = (x - mean.double().cpu()[:, None]) * r
    g = dy if w is None else dy * w.double().cpu()
    c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    # size of what rounds on the way, per element
    size = g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True)
    return r * (g - c1 - xh * c2), dy * xh, dy, r * size


def check_backward(dy, x, w, mean, rstd, dx, grads, clients, stride, cols, type_, before=None):
    want, tw, tb, size = backward64(dy, x, w, mean, rstd)
    err = 2 * DEPTH * U * size + UNIT[type_] * want.abs() + (2.0 ** -25 if type_ == "f16" else 0.0)
    assert ((dx.double().cpu() - want).abs() <= err).all()
    rows = x.shape[0] // clients
    for k, terms in enumerate((tw, tb)):
        terms = terms.view(clients, rows, cols)
        sums, sizes = terms.sum(1), terms.abs().sum(1)
        for u in range(clients):
            at = 1 + u * stride + k * cols
            got = grads[at:at + cols].double().cpu()
            start = 0.0 if before is None else before[at:at + cols].double()
            assert ((got - start - sums[u]).abs() <= (rows + 64) * U * (sizes[u] + abs(start))).all()


def inputs(rows, cols, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen) * torch.exp(0.5 * torch.randn(cols, generator=gen)) + torch.randn(rows, 1, generator=gen)
    dy = torch.randn(rows, cols, generator=gen) * 0.1 + 0.02
    return x, dy, (1 + 0.3 * torch.randn(cols, generator=gen)).cuda(), torch.randn(cols, generator=gen).cuda()


WIDTHS = [1, 2, 3, 7, 8, 31, 64, 65, 129, 255, 256, 512, 513, 1000, 1023, 1024, 1025, 2048, 4095, 4096, 4104, 8192, 8200, 16383, 16384, 16400, 20001]


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("cols", WIDTHS)
def test_widths(cols, type_):
    """Dense rows (aligned whenever the width allows) and padded rows that start anywhere."""
    for rows, clients, pad, shift in ((6, 1, 0, 0), (10, 2, 3, 1)):
        x, dy, w, b = inputs(rows, cols, cols * 7 + rows)
        _, xv = rows_of(x, type_, pad, shift)
        ybuf, y = rows_of(torch.zeros(rows, cols), type_, pad, (shift * 5) % 8, 9.0)
        y.zero_()
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        assert co3.co3_layer_norm(xv, w, b, y, mean, rstd, EPS) == co3.OK
        torch.cuda.synchronize()
        check_forward(xv, w, b, y, mean, rstd, type_)
        assert outside_untouched(ybuf, y, 9.0)
        _, dv = rows_of(dy, type_, pad, (shift * 3) % 8)
        dbuf, dx = rows_of(torch.zeros(rows, cols), type_, pad, (shift * 2) % 8, 9.0)
        stride = 2 * cols + 5
        grads = torch.full((clients * stride + 1,), 5.0, device="cuda")
        run_backward(dv, xv, w, mean, rstd, dx, grads, clients, stride, cols)
        check_backward(dv, xv, w, mean, rstd, dx, grads, clients, stride, cols, type_)
        assert outside_untouched(dbuf, dx, 9.0)
        touched = torch.zeros(grads.numel(), dtype=torch.bool)
        for u in range(clients):
            touched[1 + u * stride:1 + u * stride + 2 * cols] = True
        assert (grads.cpu()[~touched] == 5.0).all()


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("clients,rows,cols,pad", [(1, 3000, 96, 0), (1, 2500, 515, 1), (7, 301, 1024, 0), (100, 13, 512, 0),
                                                   (3, 700, 2050, 6), (1, 1500, 4096, 0), (300, 1, 40, 0), (2, 90, 17000, 0)])
def test_many_rows_and_clients(clients, rows, cols, pad, type_):
    total = clients * rows
    x, dy, w, b = inputs(total, cols, total + cols)
    _, xv = rows_of(x, type_, pad, 0)
    _, dv = rows_of(dy, type_, pad, 0)
    _, y = rows_of(x, type_, pad, 0)
    _, dx = rows_of(x, type_, pad, 0)
    mean, rstd = torch.empty(total, device="cuda"), torch.empty(total, device="cuda")
    assert co3.co3_layer_norm(xv, w, b, y, mean, rstd, EPS) == co3.OK
    stride = 2 * cols + 1
    grads = torch.randn(clients * stride + 1, device="cuda")
    before = grads.cpu().clone()
    run_backward(dv, xv, w, mean, rstd, dx, grads, clients, stride, cols, accumulate=True)
    check_forward(xv, w, b, y, mean, rstd, type_)
    check_backward(dv, xv, w, mean, rstd, dx, grads, clients, stride, cols, type_, before)
    again, dx2 = before.cuda(), torch.empty_like(dx)
    run_backward(dv, xv, w, mean, rstd, dx2, again, clients, stride, cols, accumulate=True)
    assert torch.equal(again, grads) and torch.equal(dx2, dx)                     # the same call, the same bits


def test_optional_arguments_and_in_place():
    rows, cols = 40, 200
    x, dy, w, b = inputs(rows, cols, 3)
    x, dy = x.cuda(), dy.cuda()
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    for ww, bb in ((None, None), (w, None), (None, b)):
        y = torch.empty_like(x)
        assert co3.co3_layer_norm(x, ww, bb, y, mean, rstd, EPS) == co3.OK
        torch.cuda.synchronize()
        check_forward(x, ww, bb, y, mean, rstd, "f32")
        z = x.clone()
        assert co3.co3_layer_norm(z, ww, bb, z) == co3.OK                        # in place, statistics not wanted
        torch.cuda.synchronize()
        assert torch.equal(z, y)
    stride = 2 * cols
    want = torch.zeros(stride + 1, device="cuda")
    dx = torch.empty_like(x)
    run_backward(dy, x, None, mean, rstd, dx, want, 1, stride, cols)
    check_backward(dy, x, None, mean, rstd, dx, want, 1, stride, cols, "f32")
    for kw in (dict(want_w=False), dict(want_b=False), dict(want_w=False, want_b=False)):
        grads = torch.full((stride + 1,), 3.0, device="cuda")
        d = dy.clone()
        run_backward(d, x, None, mean, rstd, d, grads, 1, stride, cols, **kw)    # dx over dy
        assert torch.equal(d, dx)
        assert torch.equal(grads[1:1 + cols], want[1:1 + cols] if kw.get("want_w", True) else torch.full((cols,), 3.0, device="cuda"))
        assert torch.equal(grads[1 + cols:], want[1 + cols:] if kw.get("want_b", True) else torch.full((cols,), 3.0, device="cuda"))
    grads = torch.zeros(stride + 1, device="cuda")
    run_backward(dy, x, None, mean, rstd, None, grads, 1, stride, cols)          # no dx
    assert torch.equal(grads, want)


def test_constant_large_offset_and_nonfinite_rows():
    """A constant row gives the bias; an offset of 1000 deviations costs no more than the mean's rounding; a NaN or an
    infinity spoils its own row alone."""
    cols = 768
    x, _, w, b = inputs(6, cols, 9)
    x = x.cuda()
    x[1] = 3.25
    x[2] += 1000.0
    x[3, 5] = float("nan")
    x[4, 700] = float("inf")
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    assert co3.co3_layer_norm(x, w, b, y, mean, rstd, EPS) == co3.OK
    torch.cuda.synchronize()
    assert torch.equal(y[1], b) and mean[1] == 3.25
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).all()
    keep = [0, 1, 2, 5]
    check_forward(x[keep], w, b, y[keep], mean[keep], rstd[keep], "f32")


def test_no_rows_and_refusals():
    x = torch.zeros(0, 16, device="cuda")
    w = torch.ones(16, device="cuda")
    assert co3.co3_layer_norm(x, w, w, x.clone()) == co3.OK
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    st = torch.zeros(0, device="cuda")
    grads = torch.full((2, 32), 7.0, device="cuda")
    flat = grads.view(-1)
    assert co3.co3_layer_norm_backward(x, x, w, st, st, x.clone(), flat, flat[16:], 2, 32, ws, True) == co3.OK
    torch.cuda.synchronize()
    assert (grads == 7.0).all()
    assert co3.co3_layer_norm_backward(x, x, w, st, st, x.clone(), flat, flat[16:], 2, 32, ws) == co3.OK
    torch.cuda.synchronize()
    assert (grads == 0.0).all()                                                  # no rows: no gradient
    a = torch.randn(8, 64, device="cuda")
    y, m, r = torch.empty_like(a), torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    w = torch.ones(64, device="cuda")
    assert co3.co3_layer_norm(a, w, w, y, m, r, -1.0) == co3.ERR_INVALID_ARG
    assert co3.co3_layer_norm(a, w, w, y, m, r, float("nan")) == co3.ERR_INVALID_ARG
    for bad in (a.double(), a.t(), a[0]):
        with pytest.raises(ValueError):
            co3.co3_layer_norm(bad, w, w, torch.empty_like(bad))
    with pytest.raises(ValueError):
        co3.co3_layer_norm(a, w[:63], w, y)
    with pytest.raises(ValueError):
        co3.co3_layer_norm(a, w, w, y.half())
    g = torch.zeros(200, device="cuda")
    big = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    back = lambda n=1, stride=128, work=big: co3.co3_layer_norm_backward(a, a, w, m, r, y, g, g[64:], n, stride, work)
    assert back() == co3.OK
    assert back(work=big[:256]) == co3.ERR_CAPACITY
    assert back(work=big[16:]) == co3.ERR_INVALID_ARG
    assert back(n=2, stride=63) == co3.ERR_INVALID_ARG                           # clients' sums would overlap
    with pytest.raises(ValueError):
        back(n=3)                                                                # eight rows are no three batches
    with pytest.raises(ValueError):
        back(n=2, stride=128)                                                    # client 1 ends beyond the tensor
    torch.cuda.synchronize()


def test_gradients_against_differences():
    """Central differences of the 64-bit definition's sum(y * q) against the kernels' gradients.  The third derivative
    leaves about step^2, the gradients' own fp32 rounding 1e-5 of their size."""
    rows, cols, step = 3, 24, 1e-4
    x, q, w, b = inputs(rows, cols, 21)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    y, dx, grads = torch.empty(rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda"), torch.zeros(2 * cols + 1, device="cuda")
    assert co3.co3_layer_norm(x.cuda(), w, b, y, mean, rstd, EPS) == co3.OK
    run_backward(q.cuda(), x.cuda(), w, mean, rstd, dx, grads, 1, 2 * cols, cols)
    loss = lambda x_, w_, b_: (forward64(x_, w_, b_)[0] * q.double()).sum().item()
    x64, w64, b64 = x.double(), w.double().cpu(), b.double().cpu()
    for which, base, got in (("x", x64, dx.cpu()), ("w", w64, grads[1:1 + cols].cpu()), ("b", b64, grads[1 + cols:].cpu())):
        for idx in np.ndindex(*base.shape):
            up, down = base.clone(), base.clone()
            up[idx] += step
            down[idx] -= step
            args = {"x": x64, "w": w64, "b": b64}
            diff = (loss(*{**args, which: up}.values()) - loss(*{**args, which: down}.values())) / (2 * step)
            assert abs(got[idx].item() - diff) <= 1e-5 * (1 + abs(diff)) + 100 * step ** 2


def test_another_stream():
    x, _, w, b = inputs(500, 300, 2)
    x = x.cuda()
    want, got = torch.empty_like(x), torch.empty_like(x)
    assert co3.co3_layer_norm(x, w, b, want) == co3.OK
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert co3.co3_layer_norm(x, w, b, got, stream=side) == co3.OK
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(want, got)


def test_rows_beyond_32_bit_offsets():
    """Rows 2^31 elements apart: element and byte offsets that 32 bits do not hold."""
    step, cols = 2 ** 31 + 24, 1000
    x, dy, w, b = inputs(2, cols, 12)
    bufs = [torch.empty(step + cols, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    xs, ys = (t.as_strided((2, cols), (step, 1)) for t in bufs)
    xs.copy_(x)
    mean, rstd = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    assert co3.co3_layer_norm(xs, w, b, ys, mean, rstd) == co3.OK
    torch.cuda.synchronize()
    check_forward(xs, w, b, ys, mean, rstd, "bf16")
    ys.copy_(dy)
    d = ys.clone()
    grads = torch.full((1 + 2 * cols,), 7.0, device="cuda")
    run_backward(ys, xs, w, mean, rstd, ys, grads, 1, 2 * cols, cols)      # dx over dy, in place
    check_backward(d, xs, w, mean, rstd, ys, grads, 1, 2 * cols, cols, "bf16")
