"""co3_orthogonalize and co3_muon_update against the definition in 64 bits, over shapes, layouts, types and spectra.

Tolerance.  A singular value s of X_0 ends as f(s), f the composed polynomial; an error e in an iterate reaches the
result through divided differences of f, at most cond = max(|f'|, f(s)/s) on [0, s_max] times e.  Products and stored
iterates are good to u = 2^-22 of the iterate (pairs of fp16); five steps have about eight such roundings each, so that
    ||error||_F <= 40 u cond ||X_0||_F + (unit of the output type) ||result||_F,     ||X_0||_F = 1.
fp16 and bf16 results add their own rounding, 2^-11 and 2^-8 (half a unit in the last place, relative).  For bf16
results the library may take the products of the early steps with single fp16 values (u = 2^-11); what those errors
leave is held below another 2^-8.
"""
import numpy as np
import pytest
import torch

import paper_2204_08211_b200 as co3

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
OUT_UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8 + 2.0 ** -8}


def definition(g, coef=(COEF,) * 5, eps=1e-7):
    x = g.detach().double().cpu()
    if x.shape[0] > x.shape[1]:
        return definition(x.T, coef, eps).T
    n = torch.linalg.norm(x) + eps
    x = x / n if n > 0 else x
    for a, b, c in coef:
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return x


def bound(g, want, out_type, coef=(COEF,) * 5):
    """Allowed Frobenius norm of the error (see above)."""
    x = g.detach().double().cpu()
    n = torch.linalg.norm(x)
    if n == 0:
        return 0.0
    top = torch.linalg.matrix_norm(x / n, 2).item()
    s = np.linspace(top / 4096, top, 4096)
    f, d = s.copy(), np.ones_like(s)
    for a, b, c in coef:
        d = d * (a + 3 * b * f ** 2 + 5 * c * f ** 4)
        f = a * f + b * f ** 3 + c * f ** 5
    cond = max(np.abs(d).max(), np.abs(f / s).max(), float(np.prod([a for a, _, _ in coef])))
    return 40 * 2.0 ** -22 * cond + OUT_UNIT[out_type] * torch.linalg.norm(want).item()


def result():
    return torch.zeros(co3.RESULT_DTYPE.itemsize, dtype=torch.uint8, device="cuda")


def orthogonalize(inp, in_mats, out, out_mats=None, ns=None):
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(in_mats), dtype=torch.uint8, device="cuda")
    ws.fill_(0xAB)                                            # leftovers must not matter
    res = result()
    st = co3.co3_orthogonalize(inp, in_mats, out, out_mats, ws, res, ns)
    assert st == co3.OK, co3.co3_status_string(st)
    torch.cuda.synchronize()
    return co3.read_results(res, 1)[0]


def spectrum(kind, rows, cols, gen):
    g = torch.randn(rows, cols, generator=gen, dtype=torch.float64)
    if kind == "lowrank":
        r = min(3, rows, cols)
        g = torch.randn(rows, r, generator=gen, dtype=torch.float64) @ torch.randn(r, cols, generator=gen, dtype=torch.float64) + 1e-4 * g
    elif kind == "heavy":
        g = g ** 3 * torch.exp(2 * torch.randn(rows, 1, generator=gen, dtype=torch.float64))
    return g


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 300), (16, 16), (63, 65), (64, 147), (65, 64), (127, 129), (128, 128), (130, 70),
          (200, 513), (513, 200), (64, 1025), (700, 64), (10, 512), (129, 1000), (257, 255), (384, 640), (1000, 513)]


@pytest.mark.parametrize("kind", ["normal", "lowrank", "heavy"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_one_matrix_fp32(rows, cols, kind):
    gen = torch.Generator().manual_seed(rows * 1009 + cols)
    g = spectrum(kind, rows, cols, gen).float().cuda()
    out = torch.full_like(g, 7.0)
    r = orthogonalize(g, co3.make_mats([(0, rows, cols)]), out)
    want = definition(g)
    assert r["status"] == co3.OK and r["n_nonfinite"] == 0
    assert torch.linalg.norm(out.double().cpu() - want).item() <= bound(g, want, "f32")


@pytest.mark.parametrize("tin,tout", [("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("rows,cols", [(5, 3), (64, 147), (130, 70), (200, 513), (300, 300), (1000, 513)])
def test_types(rows, cols, tin, tout):
    gen = torch.Generator().manual_seed(rows + cols)
    g = spectrum("normal", rows, cols, gen).to(TYPES[tin]).cuda()
    out = torch.full((rows, cols), 7.0, dtype=TYPES[tout], device="cuda")
    r = orthogonalize(g, co3.make_mats([(0, rows, cols)]), out)
    want = definition(g)
    assert r["status"] == co3.OK
    assert torch.linalg.norm(out.double().cpu() - want).item() <= bound(g, want, tout)


def test_many_matrices_with_strides_offsets_and_scales():
    """More matrices than one batch of launches holds, padded rows, gaps, different layouts of input and output."""
    gen = torch.Generator().manual_seed(5)
    ins, outs, shapes, a, b = [], [], [], 3, 1
    for k in range(110):
        rows, cols = int(torch.randint(1, 150, (1,), generator=gen)), int(torch.randint(1, 150, (1,), generator=gen))
        if k == 17:
            rows, cols = 400, 900
        if k == 50:
            rows = 0                                          # nothing to do for this one
        pi, po, scale = k % 4, (k * 3) % 5, 0.5 + 0.1 * (k % 7)
        ins.append((a, rows, cols, cols + pi))
        outs.append((b, rows, cols, cols + po, scale, 0))
        shapes.append((rows, cols, scale))
        a += rows * (cols + pi) + k % 3
        b += rows * (cols + po) + 2
    g = torch.randn(a + 5, generator=gen).cuda()
    out = torch.full((b + 5,), 99.0, device="cuda")
    r = orthogonalize(g, co3.make_mats(ins), out, co3.make_mats(outs))
    assert r["status"] == co3.OK
    untouched = torch.ones(out.numel(), dtype=torch.bool)
    gh, oh = g.cpu(), out.cpu()
    for (off, rows, cols, st), (off2, _, _, st2, scale, _) in zip(ins, outs):
        if rows == 0:
            continue
        m = gh.as_strided((rows, cols), (st, 1), off)
        got = oh.as_strided((rows, cols), (st2, 1), off2).double()
        want = definition(m)
        assert torch.linalg.norm(got - scale * want).item() <= scale * bound(m, want, "f32")
        untouched.as_strided((rows, cols), (st2, 1), off2).fill_(False)
    assert (oh[untouched] == 99.0).all()


def test_in_place_and_repeated_calls_give_the_same_bits():
    gen = torch.Generator().manual_seed(8)
    g = torch.randn(3, 200, 333, generator=gen).cuda()
    mats = co3.make_mats([(k * 200 * 333, 200, 333) for k in range(3)])
    a, b, c = torch.empty_like(g), torch.empty_like(g), g.clone()
    orthogonalize(g, mats, a)
    orthogonalize(g, mats, b)
    orthogonalize(c, mats, c)
    assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("shapes", [[(700, 300)] * 3 + [(64, 576)] * 4 + [(130, 2000), (5, 9), (256, 1152)], [(513, 1000)], [(40, 900)], [(1100, 1200)]])
def test_many_calls_in_a_row(shapes):
    """Every wait inside a call ends by itself, call after call: no status, and the same bits each time."""
    mats, off = [], 0
    for rows, cols in shapes:
        mats.append((off, rows, cols))
        off += rows * cols
    mats = co3.make_mats(mats)
    g = torch.randn(off, generator=torch.Generator().manual_seed(6)).cuda()
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    want, out = torch.empty_like(g), torch.empty_like(g)
    res = torch.zeros(1000 * co3.RESULT_DTYPE.itemsize, dtype=torch.uint8, device="cuda")
    size = co3.RESULT_DTYPE.itemsize
    assert co3.co3_orthogonalize(g, mats, want, None, ws, res[:size]) == co3.OK
    for k in range(1, 1000):
        assert co3.co3_orthogonalize(g, mats, out, None, ws, res[k * size:(k + 1) * size]) == co3.OK
    torch.cuda.synchronize()
    assert (co3.read_results(res, 1000)["status"] == co3.OK).all()
    assert torch.equal(out, want)


@pytest.mark.parametrize("rows,cols", [(40, 60), (300, 200)])
def test_magnitudes(rows, cols):
    """The result does not depend on the input's scale, over nearly all of fp32's range."""
    gen = torch.Generator().manual_seed(3)
    g = torch.randn(rows, cols, generator=gen).cuda()
    for scale in (2.0 ** -100, 2.0 ** -40, 2.0 ** 100):
        x = g * scale
        out = torch.empty_like(x)
        r = orthogonalize(x, co3.make_mats([(0, rows, cols)]), out, ns=co3.make_ns(eps=0.0))
        want = definition(x, eps=0.0)
        assert r["status"] == co3.OK
        assert torch.linalg.norm(out.double().cpu() - want).item() <= bound(x, want, "f32")


def test_zero_matrix_and_nonfinite_matrices():
    rows, cols = 70, 90
    g = torch.randn(4, rows, cols, generator=torch.Generator().manual_seed(1)).cuda()
    g[0] = 0
    g[1, 3, 4] = float("nan")
    g[3, 69, 89] = float("inf")
    out = torch.empty_like(g)
    r = orthogonalize(g, co3.make_mats([(k * rows * cols, rows, cols) for k in range(4)]), out)
    assert r["status"] == co3.ERR_NONFINITE and r["n_nonfinite"] == 2 and r["first_bad_chunk"] == 1
    assert (out[0] == 0).all() and torch.isnan(out[1]).all() and torch.isnan(out[3]).all()
    want = definition(g[2])
    assert torch.linalg.norm(out[2].double().cpu() - want).item() <= bound(g[2], want, "f32")
    for eps in (0.0, 1e-7):
        r = orthogonalize(g[0], co3.make_mats([(0, rows, cols)]), out[0], ns=co3.make_ns(eps=eps))
        assert r["status"] == co3.OK and (out[0] == 0).all()


@pytest.mark.parametrize("coef", [[(1.5, -0.5, 0.0)] * 3, [(1.875, -1.25, 0.375)], [COEF] * 2 + [(1.875, -1.25, 0.375)] * 6])
@pytest.mark.parametrize("rows,cols", [(50, 40), (150, 400)])
def test_other_iterations(rows, cols, coef):
    """Coefficients per step: the cubic and quintic iterations of second and third order, and a mixture."""
    g = torch.randn(rows, cols, generator=torch.Generator().manual_seed(2)).cuda()
    out = torch.empty_like(g)
    coef32 = [tuple(float(np.float32(v)) for v in c) for c in coef]
    orthogonalize(g, co3.make_mats([(0, rows, cols)]), out, ns=co3.make_ns(coef, eps=0.0))
    want = definition(g, coef32, 0.0)
    assert torch.linalg.norm(out.double().cpu() - want).item() <= bound(g, want, "f32", coef32)


@pytest.mark.parametrize("steps", [1, 3, 5, 10])
@pytest.mark.parametrize("rows,cols", [(300, 520), (1100, 1030)])
def test_bf16_of_an_exactly_low_rank_matrix(rows, cols, steps):
    """What early steps round into directions that the matrix lacks must not have grown into the result."""
    gen = torch.Generator().manual_seed(steps)
    whole = lambda *s: torch.randint(-2, 3, s, generator=gen, dtype=torch.float64)
    g = (whole(rows, 8) @ whole(8, cols)).bfloat16().cuda()
    out = torch.empty_like(g)
    r = orthogonalize(g, co3.make_mats([(0, rows, cols)]), out, ns=co3.make_ns([COEF] * steps))
    want = definition(g, (COEF,) * steps)
    assert r["status"] == co3.OK
    assert torch.linalg.norm(out.double().cpu() - want).item() <= bound(g, want, "bf16", (COEF,) * steps)


def test_converges_to_the_polar_factor():
    """Second-order steps to convergence reach U V^T, whatever computes it."""
    g = torch.randn(96, 160, generator=torch.Generator().manual_seed(4)).cuda()
    out = torch.empty_like(g)
    orthogonalize(g, co3.make_mats([(0, 96, 160)]), out, ns=co3.make_ns([COEF] * 3 + [(1.875, -1.25, 0.375)] * 5))
    u, _, vh = torch.linalg.svd(g.double().cpu(), full_matrices=False)
    assert torch.linalg.norm(out.double().cpu() - u @ vh).item() <= 1e-3


# ------------------------------------------------------------------------------------------------ the server's step
@pytest.mark.parametrize("nesterov", [False, True])
def test_muon_update(nesterov):
    gen = torch.Generator().manual_seed(11)
    shapes = [(64, 147), (64, 0), (64, 576), (7, 0), (130, 70), (10, 512), (10, 0), (300, 300)]
    mats, off = [], 2
    for rows, cols in shapes:
        mats.append((off, rows, cols, cols, max(1.0, rows / cols) ** 0.5, 0) if cols else (off, 1, rows, rows, 1.0, co3.MAT_PLAIN))
        off += rows * max(cols, 1) + 1                        # one element between layers belongs to nobody
    n = off + 3
    mu, lr, wd = 0.9, 0.05, 0.1
    params, momentum = (torch.randn(n, generator=gen) * s for s in (0.1, 1e-3))
    p64, m64 = params.double(), momentum.double()
    p, m = params.cuda(), momentum.cuda()
    table = co3.make_mats(mats)
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(table), dtype=torch.uint8, device="cuda")
    res = result()
    f = lambda v: float(np.float32(v))
    slack = torch.zeros(n, dtype=torch.float64)
    for _ in range(3):
        g = torch.randn(n, generator=gen) * 1e-3
        assert co3.co3_muon_update(g.cuda(), m, p, table, mu, nesterov, lr, wd, ws, res) == co3.OK
        torch.cuda.synchronize()
        assert co3.read_results(res, 1)[0]["status"] == co3.OK
        for off, rows, cols, st, scale, flags in mats:
            s = slice(off, off + rows * cols)
            m64[s] = f(mu) * m64[s] + g[s].double()
            u = g[s].double() + f(mu) * m64[s] if nesterov else m64[s]
            step = u if flags else definition(u.view(rows, cols)).reshape(-1)
            p64[s] = (1 - f(lr) * f(wd)) * p64[s] - f(lr) * f(scale) * step
            # the step's own error, and four fp32 roundings of parameters and momentum
            err = 0.0 if flags else f(lr) * scale * bound(u.view(rows, cols), step, "f32")
            slack[s] = slack[s] + err + 2.0 ** -22 * (p64[s].abs() + f(lr) * scale * step.abs())
        assert ((m.double().cpu() - m64).abs() <= 2.0 ** -21 * (m64.abs() + 1e-2)).all()
        assert ((p.double().cpu() - p64).abs() <= slack).all()


def test_muon_update_nonfinite_layer_is_reported():
    n = 20 * 30
    g = torch.randn(2 * n).cuda()
    g[5] = float("inf")
    p, m = torch.zeros(2 * n, device="cuda"), torch.zeros(2 * n, device="cuda")
    table = co3.make_mats([(0, 20, 30), (n, 20, 30)])
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(table), dtype=torch.uint8, device="cuda")
    res = result()
    assert co3.co3_muon_update(g, m, p, table, 0.9, True, 0.1, 0.0, ws, res) == co3.OK
    torch.cuda.synchronize()
    r = co3.read_results(res, 1)[0]
    assert r["status"] == co3.ERR_NONFINITE and r["n_nonfinite"] == 1 and r["first_bad_chunk"] == 0
    assert torch.isnan(p[:n]).all() and torch.isfinite(p[n:]).all()


# ------------------------------------------------------------------------------------------------ refusals, streams
def test_refusals():
    g = torch.randn(64, 64, device="cuda")
    mats = co3.make_mats([(0, 64, 64)])
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    res, out = result(), torch.empty_like(g)
    call = lambda m=mats, w=ws, ns=None: co3.co3_orthogonalize(g, m, out, None, w, res, ns)
    assert call(w=ws[:-256]) == co3.ERR_CAPACITY
    assert call(w=ws[16:]) == co3.ERR_INVALID_ARG                                   # alignment
    assert call(m=co3.make_mats([(0, 64, 64, 63)])) == co3.ERR_INVALID_ARG          # rows overlap
    assert call(m=co3.make_mats([(0, 64, 64, 64, 1.0, 2)])) == co3.ERR_INVALID_ARG  # unknown flag
    assert call(m=co3.make_mats([(0, 64, 64, 64, 1.0, co3.MAT_PLAIN)])) == co3.ERR_INVALID_ARG
    assert call(ns=co3.make_ns(steps=0)) == co3.ERR_INVALID_ARG
    assert call(ns=co3.make_ns(steps=17)) == co3.ERR_INVALID_ARG
    assert call(ns=co3.make_ns(eps=-1.0)) == co3.ERR_INVALID_ARG
    assert call(ns=co3.make_ns((9.0, -4.0, 2.0))) == co3.ERR_INVALID_ARG            # diverges
    assert call(ns=co3.make_ns((float("nan"), 0.0, 0.0))) == co3.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        call(m=co3.make_mats([(1, 64, 64)]))                                        # ends beyond the tensor
    with pytest.raises(ValueError):
        co3.co3_orthogonalize(g.double(), mats, out, None, ws, res)
    with pytest.raises(ValueError):
        co3.co3_orthogonalize(g.t(), mats, out, None, ws, res)
    assert co3.co3_muon_update(g, g, out, mats, 1.5, True, 0.1, 0.0, ws, res) == co3.ERR_INVALID_ARG
    assert co3.co3_muon_update(g, g, out, mats, 0.9, True, float("nan"), 0.0, ws, res) == co3.ERR_INVALID_ARG
    assert call(m=co3.make_mats([])) == co3.OK and call() == co3.OK
    torch.cuda.synchronize()


def test_another_stream_and_a_graph():
    g = torch.randn(130, 257, device="cuda")
    mats = co3.make_mats([(0, 130, 257)])
    want = torch.empty_like(g)
    orthogonalize(g, mats, want)
    ws = torch.empty(co3.co3_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    res, out = result(), torch.empty_like(g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert co3.co3_orthogonalize(g, mats, out, None, ws, res, stream=side) == co3.OK
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert co3.co3_orthogonalize(g, mats, out, None, ws, res) == co3.OK
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("rows,cols", [(40, 60), (150, 90)])
def test_offsets_beyond_32_bits(rows, cols):
    """A matrix that starts 2^32 elements into its buffer, and one whose rows are far apart."""
    far = torch.empty(2 ** 32 + 5 + rows * (cols + 3), dtype=torch.float16, device="cuda")
    gen = torch.Generator().manual_seed(rows)
    g = torch.randn(rows, cols, generator=gen).half()
    step = 2 ** 32 // rows
    for offset, stride in ((2 ** 32 + 5, cols + 3), (1, step)):
        view = far.as_strided((rows, cols), (stride, 1), offset)
        view.copy_(g)
        table = co3.make_mats([(offset, rows, cols, stride)])
        r = orthogonalize(far, table, far)
        want = definition(g)
        assert r["status"] == co3.OK
        assert torch.linalg.norm(view.double().cpu() - want).item() <= bound(g, want, "f16")
