"""What is timed of the clients' linear layers on 8-bit activations: values held as e4m3 with a power of two for each
block of 128, products of them, and the backward pass that reads what the forward pass kept.

A block is 128 columns of a row (activations, gradients) or 128 x 128 entries (weights; what lies beyond the edge counts as
zero).  Its scale s is the smallest power of two with max|x| <= 448 s, its values are x / s rounded to e4m3, to nearest, ties
to even.  `run` computes a case in its plain form (elementary torch operations in 32 bits, rounded once at the end) or, with
`own` set, through the package's entry points.
"""
import math

import torch

own = False

BLOCK = 128
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = ["none", "relu", "gelu", "silu"]


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the activation between two layers of a small model, one client's batch: latency
        dict(name="act_small", op="act", act="relu", type="f32", rows=64, cols=512, pad=0),
        # the same of a wide model's training batch: beyond the caches
        dict(name="act_large", op="act", act="gelu", type="bf16", rows=16384, cols=8192, pad=0),
        # activations of a ragged batch in a padded buffer, kept and read again
        dict(name="store_ragged", op="store", kind="rows", type="f16", rows=3001, cols=1023, pad=17),
        # a large projection's weights, packed after each update of the model
        dict(name="store_weights", op="store", kind="square", type="f32", rows=4096, cols=4096, pad=0),
        # one token of a decoding loop
        dict(name="linear_token", op="linear", type="bf16", rows=1, ins=1024, outs=4096, bias=True, pad=0),
        # a ragged batch, odd widths
        dict(name="linear_ragged", op="linear", type="f16", rows=1501, ins=1023, outs=1001, bias=True, pad=17),
        # a training batch of a wide model
        dict(name="linear_large", op="linear", type="bf16", rows=16384, ins=4096, outs=4096, bias=False, pad=0),
        # a hundred clients' small local batches at the width of the residual network's head, towards the inputs
        dict(name="dinput_clients", op="dinput", type="f32", rows=6400, ins=512, outs=512, pad=0),
        # a training batch through a layer that widens fourfold
        dict(name="dinput_large", op="dinput", type="bf16", rows=16384, ins=2048, outs=8192, pad=0),
        # the hundred clients' gradients of that layer's weights and biases, each into the client's own vector
        dict(name="dweight_clients", op="dweight", type="f32", clients=100, rows=64, ins=512, outs=512, pad=0),
        # two clients, odd widths, padded rows
        dict(name="dweight_ragged", op="dweight", type="f16", clients=2, rows=1501, ins=1023, outs=1001, pad=17),
        # a training batch of a wide model
        dict(name="dweight_large", op="dweight", type="bf16", clients=1, rows=16384, ins=4096, outs=4096, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["act", "store", "linear", "linear", "dinput", "dweight", "dweight"])
    case = dict(op=op, type=rng.choice(list(DTYPES)), pad=rng.choice([0, 0, 1, 7, 64]))
    if op in ("act", "store"):
        case["cols"] = _log(rng, 16, 16384)
        case["rows"] = _log(rng, 1, max(2, min(65536, (1 << 26) // case["cols"])))
        if op == "act":
            case["act"] = rng.choice(ACTS)
        else:
            case["kind"] = rng.choice(["rows", "square"])
        return case
    case["ins"], case["outs"] = _log(rng, 16, 8192), _log(rng, 16, 8192)
    # at most a quarter of the largest listed case: the parts of a 32-bit gradient cost three times the products
    rows = _log(rng, 1, max(2, min(32768, (1 << 36) // (case["ins"] * case["outs"]))))
    if op == "linear":
        case["bias"] = rng.random() < 0.5
    if op == "dweight":
        # the gradients of all clients stay below 1 GB
        most = max(1, min(100, rows, (1 << 28) // (case["ins"] * case["outs"])))
        case["clients"] = _log(rng, 1, most)
        rows = max(1, rows // case["clients"])
    case["rows"] = rows
    return case


# ------------------------------------------------------------------------------------------------ inputs
def _normal(gen, *size):
    return torch.randn(*size, generator=gen, device="cuda")


def _padded(case, values):
    rows, cols = values.shape
    buf = torch.zeros(rows, cols + case["pad"], dtype=DTYPES[case["type"]], device="cuda")
    buf[:, :cols] = values
    return buf[:, :cols]


def _activations(gen, rows, cols):
    """Every channel has its own offset and spread, a few are far larger than the others, rows differ too."""
    spread = torch.exp(0.5 * _normal(gen, cols)) * torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 12.0, 1.0)
    return (_normal(gen, rows, cols) * spread + 0.3 * _normal(gen, cols)) * torch.exp(0.3 * _normal(gen, rows, 1))


def _gradients(gen, rows, cols):
    """Heavy tails, and rows (samples) of very different size."""
    g = _normal(gen, rows, cols)
    return 1e-3 * g * g.abs().sqrt() * torch.exp(_normal(gen, rows, 1))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, s = case["op"], {"case": case}
    if op in ("act", "store"):
        rows, cols = case["rows"], case["cols"]
        square = case.get("kind") == "square"
        s["x"] = _padded(case, _normal(gen, rows, cols) / math.sqrt(cols) if square else _activations(gen, rows, cols))
        s["y"] = _padded(case, torch.zeros(rows, cols, device="cuda"))
        if op == "act":
            s["dy"] = _padded(case, _gradients(gen, rows, cols))
            s["dx"] = _padded(case, torch.zeros(rows, cols, device="cuda"))
        if own:
            s["x8"] = _room(rows, cols, square)
        return s
    rows, ins, outs = case["rows"] * case.get("clients", 1), case["ins"], case["outs"]
    if op == "dweight":
        s["dy"] = _padded(case, _gradients(gen, rows, outs))
        x = _activations(gen, rows, ins)
        # the forward pass has kept the layer's inputs in 8 bits
        s["kept"] = _quantise(x)
        clients = case["clients"]
        s["stride"] = (outs * ins + outs + 3) // 4 * 4
        s["grads"] = torch.zeros(clients * s["stride"], device="cuda")
        if own:
            import paper_2204_08211_b200 as co3
            s["x8"] = _room(rows, ins, False)
            _ok(co3.co3_f8_pack(x, s["x8"]))
            s["workspace"] = torch.empty(co3.co3_f8_weight_gradient_workspace_bytes(case["rows"], outs, ins, clients),
                                         dtype=torch.uint8, device="cuda")
            del s["kept"]
        return s
    # the layer's weights are packed once for all calls until the next update of the model
    w = _normal(gen, outs, ins) / math.sqrt(ins)
    s["weights"] = _quantise(w, True)
    cols, width = (ins, outs) if op == "linear" else (outs, ins)
    s["x"] = _padded(case, _activations(gen, rows, cols) if op == "linear" else _gradients(gen, rows, cols))
    s["bias"] = 0.1 * _normal(gen, outs) if case.get("bias") else None
    s["y"] = _padded(case, torch.zeros(rows, width, device="cuda"))
    if own:
        import paper_2204_08211_b200 as co3
        s["x8"], s["w8"] = _room(rows, cols, False), _room(outs, ins, True)
        _ok(co3.co3_f8_pack(w, s["w8"], co3.F8_SQUARE))
        del s["weights"]
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _tiles(x, square):
    """x padded with zeros to whole blocks, [row blocks][rows][column blocks][columns]."""
    rows, cols = x.shape
    high = BLOCK if square else 1
    x = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK, 0, -rows % high))
    return x.view(x.shape[0] // high, high, x.shape[1] // BLOCK, BLOCK)


def _quantise(x, square=False):
    """(e4m3 values, scales) in blocks, and the shape."""
    t = _tiles(x, square)
    part, exponent = torch.frexp(t.abs().amax((1, 3), keepdim=True))
    exponent = (exponent - 9 + (part > 0.875).int()).clamp(-126, 120)     # 448 = 0.875 * 2^9
    scale = ((exponent + 127) << 23).view(torch.float32)
    return (t / scale).to(torch.float8_e4m3fn), scale, x.shape


def _values(packed):
    q, scale, (rows, cols) = packed
    t = q.float() * scale
    return t.reshape(t.shape[0] * t.shape[1], -1)[:rows, :cols]


def _act(act, x):
    if act == "relu":
        return x.clamp(min=0)
    if act == "gelu":
        return x * (0.5 * torch.erfc(x * -math.sqrt(0.5)))
    return x / (1 + torch.exp(-x)) if act == "silu" else x


def _act_grad(act, x):
    if act == "relu":
        return (x > 0).to(x.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(x * -math.sqrt(0.5)) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        p = 1 / (1 + torch.exp(-x))
        return p * (1 + x * (1 - p))
    return torch.ones_like(x)


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    t = DTYPES[case["type"]]
    if op == "act":
        kept = _quantise(s["x"])
        return _act(case["act"], s["x"].float()).to(t), (s["dy"].float() * _act_grad(case["act"], _values(kept))).to(t)
    if op == "store":
        return _values(_quantise(s["x"], case["kind"] == "square")).to(t)
    if op == "linear":
        y = _values(_quantise(s["x"])) @ _values(s["weights"]).T
        return (y if s["bias"] is None else y + s["bias"]).to(t)
    if op == "dinput":
        return (_values(_quantise(s["x"])) @ _values(s["weights"])).to(t)
    clients = case["clients"]
    dy, x = s["dy"].float().view(clients, -1, case["outs"]), _values(s["kept"]).view(clients, -1, case["ins"])
    return dy.transpose(1, 2) @ x, dy.sum(1)


# ------------------------------------------------------------------------------------------------ the package's calls
def _room(rows, cols, square):
    import paper_2204_08211_b200 as co3
    return torch.empty(co3.co3_f8_bytes(rows, cols, co3.F8_SQUARE if square else co3.F8_ROWS), dtype=torch.uint8, device="cuda")


def _ok(*statuses):
    import paper_2204_08211_b200 as co3
    for st in statuses:
        if st != co3.OK:
            raise RuntimeError(co3.co3_status_string(st))


def _run_own(s):
    import paper_2204_08211_b200 as co3
    case, op = s["case"], s["case"]["op"]
    if op == "act":
        act = ACTS.index(case["act"])
        _ok(co3.co3_f8_activation(s["x"], act, s["y"], None, s["x8"]),
            co3.co3_f8_activation_backward(s["dy"], s["x8"], act, s["dx"]))
        return s["y"], s["dx"]
    if op == "store":
        kind = co3.F8_SQUARE if case["kind"] == "square" else co3.F8_ROWS
        _ok(co3.co3_f8_pack(s["x"], s["x8"], kind), co3.co3_f8_unpack(s["x8"], s["y"], kind))
        return s["y"]
    if op in ("linear", "dinput"):
        _ok(co3.co3_f8_linear(s["x"], s["x8"], s["w8"], s["bias"], s["y"], op == "dinput"))
        return s["y"]
    clients, outs, ins = case["clients"], case["outs"], case["ins"]
    _ok(co3.co3_f8_weight_gradient(s["dy"], s["x8"], ins, s["grads"], s["grads"][outs * ins:], clients, s["stride"], s["workspace"]))
    vectors = s["grads"].view(clients, -1)
    return vectors[:, :outs * ins].view(clients, outs, ins), vectors[:, outs * ins:outs * ins + outs]


def run(state):
    if own:
        return _run_own(state)
    return _plain(state)


# ------------------------------------------------------------------------------------------------ work and exact values
def work(case):
    size, op = 4 if case["type"] == "f32" else 2, case["op"]
    if op in ("act", "store"):
        n = case["rows"] * case["cols"]
        per = (4 * size + 2, 30) if op == "act" else (2 * size + 2, 6)   # what is kept is written and read
        return {"bytes": per[0] * n, "flops": per[1] * n}
    rows, ins, outs = case["rows"] * case.get("clients", 1), case["ins"], case["outs"]
    flops = 2 * rows * ins * outs
    if op == "dweight":
        return {"bytes": rows * (outs * size + ins) + 4 * case["clients"] * outs * (ins + 1), "flops": flops}
    return {"bytes": rows * (ins + outs) * size + outs * ins, "flops": flops}


def _power64(k):
    return ((k.long() + 1023) << 52).view(torch.float64)


def _values64(x, square=False):
    """What the blocks stand for, from the definition in 64 bits."""
    rows, cols = x.shape
    high = BLOCK if square else 1
    full = torch.zeros(-(-rows // high) * high, -(-cols // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    full[:rows, :cols] = x.double()
    t = full.unfold(0, high, high).unfold(1, BLOCK, BLOCK)               # [block row][block column][rows][columns]
    most = t.abs().amax((2, 3), keepdim=True)
    k = torch.frexp(most)[1] - 11
    for _ in range(3):                                                   # the smallest power of two that holds the block
        k = torch.where(most > 448 * _power64(k), k + 1, k)
    s = _power64(k.clamp(min=-126))
    u = t / s
    step = _power64((torch.frexp(u)[1] - 1).clamp(min=-6) - 3)   # three bits behind the leading one; 2^-9 at least
    v = torch.round(u / step) * step * s
    return v.transpose(1, 2).reshape(full.shape)[:rows, :cols]


def _act64(act, x):
    """(act(x), its derivative)"""
    if act == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x)), torch.where(x > 0, 1.0, 0.0).double()
    if act == "gelu":
        below = torch.special.ndtr(x)
        return x * below, below + x * torch.exp(-x.square() / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        p = torch.sigmoid(x)
        return x * p, p + x * p * torch.sigmoid(-x)
    return x, torch.ones_like(x)


def exact(case, seed):
    op = case["op"]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    if op == "dweight":
        clients, outs, ins = case["clients"], case["outs"], case["ins"]
        dy = _padded(case, _gradients(gen, clients * case["rows"], outs)).double().view(clients, -1, outs)
        x = _values64(_activations(gen, clients * case["rows"], ins)).view(clients, -1, ins)
        return torch.stack([d.T @ v for d, v in zip(dy, x)]), dy.sum(1)
    if op in ("linear", "dinput"):
        w = _values64(_normal(gen, case["outs"], case["ins"]) / math.sqrt(case["ins"]), True)
        cols = case["ins"] if op == "linear" else case["outs"]
        x = _padded(case, (_activations if op == "linear" else _gradients)(gen, case["rows"], cols))
        bias = 0.1 * _normal(gen, case["outs"]) if case.get("bias") else None
        if op == "dinput":
            return _values64(x) @ w
        y = _values64(x) @ w.T
        return y if bias is None else y + bias.double()
    s = prepare(case, seed)
    if op == "store":
        return _values64(s["x"], case["kind"] == "square")
    y, _ = _act64(case["act"], s["x"].double())
    return y, s["dy"].double() * _act64(case["act"], _values64(s["x"]))[1]
