"""What is timed of the operators at the two ends of the compressed path: the clients' layer norms (forward, and
backward into the gradient vectors that are encoded) and the server's orthogonalised updates.

`run` computes a case in its plain form (elementary torch operations in 32 bits, rounded once at the end) or, with
`own` set, through the package's entry points.
"""
import math

import torch

own = False

NS_COEF = (3.4445, -4.7750, 2.0315)   # odd quintic whose iteration takes (0, 1] to about 1
NS_STEPS = 5
NS_EPS = 1e-7
LN_EPS = 1e-5
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of a decoding loop: only the latency of the call counts
        dict(name="ln_fwd_token", op="ln_fwd", type="bf16", rows=1, cols=1024, pad=0),
        # a ragged batch in a padded buffer, width no multiple of anything
        dict(name="ln_fwd_ragged", op="ln_fwd", type="f16", rows=3001, cols=1023, pad=17),
        # a training batch of a wide model: beyond the caches
        dict(name="ln_fwd_large", op="ln_fwd", type="bf16", rows=16384, cols=4096, pad=0),
        # a hundred clients' small local batches at the width of the residual network's head
        dict(name="ln_bwd_clients", op="ln_bwd", type="f32", clients=100, rows=64, cols=512, pad=0),
        # two clients, odd width, padded rows
        dict(name="ln_bwd_ragged", op="ln_bwd", type="f16", clients=2, rows=1501, cols=1023, pad=17),
        # a training batch of a wide model
        dict(name="ln_bwd_large", op="ln_bwd", type="bf16", clients=1, rows=16384, cols=4096, pad=0),
        # the residual network's first convolution, 64 filters of 3 x 7 x 7: latency
        dict(name="orth_stem", op="orth", type="f32", count=1, rows=64, cols=147),
        # a tall matrix of odd sizes (a classifier with 1000 classes)
        dict(name="orth_tall", op="orth", type="f16", count=1, rows=1000, cols=513),
        # the wide projections of a large model, update kept in bf16
        dict(name="orth_wide", op="orth", type="bf16", count=2, rows=2048, cols=8192),
        # a large square projection in full precision
        dict(name="orth_square", op="orth", type="f32", count=1, rows=4096, cols=4096),
        # the server's step on the 62 layers of the 18-layer residual network
        dict(name="muon_resnet18", op="muon", net="resnet18", width=64, layers=1, nesterov=True),
        # the server's step on two blocks of a transformer (four square matrices, two wide ones, norms)
        dict(name="muon_blocks", op="muon", net="blocks", width=1024, layers=2, nesterov=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "orth", "orth", "muon"])
    if op in ("ln_fwd", "ln_bwd"):
        cols = _log(rng, 16, 16384)
        rows = _log(rng, 1, max(2, min(65536, (1 << 26) // cols)))
        case = dict(op=op, type=rng.choice(list(DTYPES)), rows=rows, cols=cols, pad=rng.choice([0, 0, 1, 7, 64]))
        if op == "ln_bwd":
            case["clients"] = min(rows, _log(rng, 1, 100))
            case["rows"] = max(1, rows // case["clients"])
        return case
    if op == "orth":
        rows, cols = _log(rng, 8, 4096), _log(rng, 8, 8192)
        if rng.random() < 0.3:
            rows, cols = min(cols, 4096), rows
        m, n = min(rows, cols), max(rows, cols)
        count = rng.choice([1, 1, 2, 3, 6])
        while count > 1 and count * m * m * n > 4096 ** 3 // 4:
            count -= 1
        return dict(op=op, type=rng.choice(list(DTYPES)), count=count, rows=rows, cols=cols)
    net = rng.choice(["resnet18", "blocks"])
    if net == "resnet18":
        return dict(op=op, net=net, width=rng.randint(12, 80), layers=1, nesterov=rng.random() < 0.5)
    return dict(op=op, net=net, width=_log(rng, 48, 1400), layers=rng.randint(1, 2), nesterov=rng.random() < 0.5)


def shapes(case):
    """(rows, cols) of every layer in order; cols == 0: a vector of `rows` entries (updated without a matrix step)."""
    w = case["width"]
    if case["net"] == "resnet18":
        out, cin = [(w, 3 * 49), (w, 0), (w, 0)], w
        for stage in range(4):
            c = w << stage
            for block in range(2):
                out += [(c, cin * 9), (c, 0), (c, 0), (c, c * 9), (c, 0), (c, 0)]
                if cin != c:
                    out += [(c, cin), (c, 0), (c, 0)]
                cin = c
        return out + [(10, cin), (10, 0)]
    return [(w, 0), (w, 0), (w, w), (w, w), (w, w), (w, w), (w, 0), (w, 0), (4 * w, w), (w, 4 * w)] * case["layers"]


# ------------------------------------------------------------------------------------------------ inputs
def _normal(gen, *size):
    return torch.randn(*size, generator=gen, device="cuda")


def _gradient(gen, rows, cols):
    """A gradient as it comes from a batch: a few strong directions over a heavy-tailed remainder."""
    r = min(24, rows, cols)
    strong = (_normal(gen, rows, r) * torch.logspace(0, -2, r, device="cuda")) @ _normal(gen, r, cols)
    rest = _normal(gen, rows, cols)
    return 1e-3 * (strong + 0.3 * rest * rest.abs().sqrt())


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case}
    if case["op"] in ("ln_fwd", "ln_bwd"):
        t, clients, cols = DTYPES[case["type"]], case.get("clients", 1), case["cols"]
        rows = clients * case["rows"]

        def padded(fill):
            buf = torch.zeros(rows, cols + case["pad"], dtype=t, device="cuda")
            buf[:, :cols] = fill
            return buf[:, :cols]
        # activations: every channel has its own offset and spread
        x = _normal(gen, rows, cols) * torch.exp(0.5 * _normal(gen, cols)) + 0.5 * _normal(gen, cols) + 0.3 * _normal(gen, rows, 1)
        s["x"] = padded(x)
        s["weight"] = 1 + 0.2 * _normal(gen, cols)
        s["bias"] = 0.1 * _normal(gen, cols)
        if case["op"] == "ln_fwd":
            s["y"] = padded(0)
            s["mean"], s["rstd"] = (torch.zeros(rows, device="cuda") for _ in range(2))
        else:
            xf = s["x"].float()
            s["mean"] = xf.mean(1)
            s["rstd"] = torch.rsqrt((xf - s["mean"][:, None]).square().mean(1) + LN_EPS)
            s["dy"] = padded(1e-2 * _normal(gen, rows, cols) + 2e-3 * _normal(gen, cols))
            s["dx"] = padded(0)
            # the clients' gradient vectors: gain and bias are the first two layers of each
            s["stride"] = (2 * cols + 3) // 4 * 4
            s["grads"] = torch.zeros(clients * s["stride"], device="cuda")
    elif case["op"] == "orth":
        g = torch.stack([_gradient(gen, case["rows"], case["cols"]) for _ in range(case["count"])])
        s["g"] = g.to(DTYPES[case["type"]])
        s["out"] = torch.zeros_like(s["g"])
    else:
        parts, params = [], []
        for rows, cols in shapes(case):
            parts.append((_gradient(gen, rows, cols) if cols else 1e-3 * _normal(gen, rows)).reshape(-1))
            params.append((_normal(gen, rows, cols) / math.sqrt(cols) if cols else 1 + 0.1 * _normal(gen, rows)).reshape(-1))
        s["grad"] = torch.cat(parts)
        s["params"] = torch.cat(params)
        s["momentum"] = 0.5e-3 * _normal(gen, s["grad"].numel())
        s.update(mu=0.95, lr=0.02, wd=0.01)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _orth_plain(g):
    """[k, rows, cols] in 32 bits: every matrix divided by its norm, then the quintic steps."""
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2) if tall else g
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    a, b, c = NS_COEF
    for _ in range(NS_STEPS):
        p = x @ x.transpose(1, 2)
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.transpose(1, 2) if tall else x


def _gain(rows, cols):
    return max(1.0, rows / cols) ** 0.5


def _ln_fwd_plain(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = torch.rsqrt(xc.square().mean(1, keepdim=True) + LN_EPS)
    return (xc * rstd * s["weight"] + s["bias"]).to(s["x"].dtype), mean[:, 0], rstd[:, 0]


def _ln_bwd_plain(s):
    clients = s["case"]["clients"]
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    g = dy * s["weight"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    dw = (dy * xh).view(clients, -1, x.shape[1]).sum(1)
    db = dy.view(clients, -1, x.shape[1]).sum(1)
    return dx.to(s["x"].dtype), dw, db


def _muon_plain(s):
    """Layers of one shape are stepped together; parameters and momentum change in place."""
    if "groups" not in s:
        s["groups"] = _groups(s["case"])
    s["momentum"].mul_(s["mu"]).add_(s["grad"])
    u = s["grad"] + s["mu"] * s["momentum"] if s["case"]["nesterov"] else s["momentum"]
    s["params"].mul_(1 - s["lr"] * s["wd"])
    for (rows, cols), offs in s["groups"].items():
        if cols == 0:
            s["params"].index_add_(0, offs, u[offs], alpha=-s["lr"])
        else:
            o = _orth_plain(torch.stack([u[k:k + rows * cols].view(rows, cols) for k in offs]))
            for k, step in zip(offs, o):
                s["params"][k:k + rows * cols].sub_(step.reshape(-1), alpha=s["lr"] * _gain(rows, cols))
    return s["params"], s["momentum"]


def _groups(case):
    """{(rows, cols): offsets}; all vectors together under (0, 0) as one index."""
    groups, vectors, off = {}, [], 0
    for rows, cols in shapes(case):
        if cols:
            groups.setdefault((rows, cols), []).append(off)
        else:
            vectors.append(torch.arange(off, off + rows))
        off += rows * max(1, cols)
    groups[(0, 0)] = torch.cat(vectors).cuda()
    return groups


# ------------------------------------------------------------------------------------------------ the package's calls
def _run_own(s):
    import paper_2204_08211_b200 as co3
    case, op = s["case"], s["case"]["op"]
    if op == "ln_fwd":
        st = co3.co3_layer_norm(s["x"], s["weight"], s["bias"], s["y"], s["mean"], s["rstd"], LN_EPS)
        out = s["y"], s["mean"], s["rstd"]
    elif op == "ln_bwd":
        clients, cols = case["clients"], case["cols"]
        if "workspace" not in s:
            s["workspace"] = torch.empty(co3.co3_layer_norm_workspace_bytes(case["rows"], cols, clients), dtype=torch.uint8, device="cuda")
            s["dw"], s["db"] = s["grads"][:], s["grads"][cols:]
            s["views"] = tuple(s["grads"].view(clients, -1)[:, k * cols:(k + 1) * cols] for k in (0, 1))
        st = co3.co3_layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"],
                                         clients, s["stride"], s["workspace"])
        out = s["dx"], s["views"][0], s["views"][1]
    else:
        if "mats" not in s:
            if op == "orth":
                size = case["rows"] * case["cols"]
                s["mats"] = co3.make_mats([(k * size, case["rows"], case["cols"]) for k in range(case["count"])])
            else:
                rows, off = [], 0
                for r, c in shapes(case):
                    rows.append((off, r, c, c, _gain(r, c), 0) if c else (off, 1, r, r, 1.0, co3.MAT_PLAIN))
                    off += r * max(1, c)
                s["mats"] = co3.make_mats(rows)
            s["workspace"] = torch.empty(co3.co3_orthogonalize_workspace_bytes(s["mats"]), dtype=torch.uint8, device="cuda")
            s["res"] = torch.zeros(co3.RESULT_DTYPE.itemsize, dtype=torch.uint8, device="cuda")
        if op == "orth":
            st = co3.co3_orthogonalize(s["g"], s["mats"], s["out"], s["mats"], s["workspace"], s["res"])
            out = s["out"]
        else:
            st = co3.co3_muon_update(s["grad"], s["momentum"], s["params"], s["mats"], s["mu"], case["nesterov"], s["lr"],
                                     s["wd"], s["workspace"], s["res"])
            out = s["params"], s["momentum"]
    if st != co3.OK:
        raise RuntimeError(co3.co3_status_string(st))
    return out


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "ln_fwd":
        return _ln_fwd_plain(state)
    if op == "ln_bwd":
        return _ln_bwd_plain(state)
    if op == "orth":
        return _orth_plain(state["g"].float()).to(state["g"].dtype)
    return _muon_plain(state)


# ------------------------------------------------------------------------------------------------ work and exact values
def _orth_flops(rows, cols):
    m, n = min(rows, cols), max(rows, cols)
    return NS_STEPS * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)   # both m x m products are symmetric


def work(case):
    if case["op"] in ("ln_fwd", "ln_bwd"):
        clients, cols = case.get("clients", 1), case["cols"]
        rows, size = clients * case["rows"], 4 if case["type"] == "f32" else 2
        if case["op"] == "ln_fwd":
            return {"bytes": 2 * rows * cols * size + 8 * cols + 8 * rows, "flops": 8 * rows * cols}
        return {"bytes": 3 * rows * cols * size + 8 * rows + 4 * cols + 8 * clients * cols, "flops": 14 * rows * cols}
    if case["op"] == "orth":
        size = 4 if case["type"] == "f32" else 2
        return {"bytes": 2 * case["count"] * case["rows"] * case["cols"] * size,
                "flops": case["count"] * _orth_flops(case["rows"], case["cols"])}
    every = shapes(case)
    return {"bytes": 20 * sum(r * max(1, c) for r, c in every), "flops": sum(_orth_flops(r, c) for r, c in every if c)}


def _orth_exact(g):
    """From the definition in 64 bits, one matrix: X <- (a I + b A + c A^2) X with A = X X^T, small side first."""
    x = g.double()
    if x.shape[0] > x.shape[1]:
        return _orth_exact(x.T).T
    x = x / (torch.linalg.norm(x) + NS_EPS)
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for _ in range(NS_STEPS):
        gram = torch.mm(x, x.T)
        x = torch.mm(NS_COEF[0] * eye + torch.mm(gram, NS_COEF[1] * eye + NS_COEF[2] * gram), x)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "ln_fwd":
        x = s["x"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + LN_EPS)
        return torch.addcmul(s["bias"].double(), (x - mean[:, None]) * rstd[:, None], s["weight"].double()), mean, rstd
    if case["op"] == "ln_bwd":
        n, clients = case["cols"], case["clients"]
        dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
        xh = (s["x"].double() - s["mean"].double()[:, None]) * rstd
        g = dy * s["weight"].double()
        dx = (rstd / n) * (n * g - g.sum(1, keepdim=True) - xh * torch.einsum("rc,rc->r", g, xh)[:, None])
        dw = torch.einsum("urc,urc->uc", dy.reshape(clients, -1, n), xh.reshape(clients, -1, n))
        return dx, dw, dy.reshape(clients, -1, n).sum(1)
    if case["op"] == "orth":
        return torch.stack([_orth_exact(g) for g in s["g"]])
    momentum = s["mu"] * s["momentum"].double() + s["grad"].double()
    u = s["grad"].double() + s["mu"] * momentum if case["nesterov"] else momentum
    params, off = s["params"].double() * (1 - s["lr"] * s["wd"]), 0
    for rows, cols in shapes(case):
        end = off + rows * max(1, cols)
        step = _orth_exact(u[off:end].view(rows, cols)).reshape(-1) * math.sqrt(max(1.0, rows / cols)) if cols else u[off:end]
        params[off:end] -= s["lr"] * step
        off = end
    return params, momentum
