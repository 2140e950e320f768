"""8-bit blocks from their definition, in 64 bits, for the tests."""
import numpy as np
import torch

BLOCK = 128
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def blocks(x, square):
    """Exponents k of the scales 2^k, spread over the entries, and the values (both of x's shape)."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    high = BLOCK if square else 1
    exps, vals = np.zeros(x.shape, dtype=np.int64), np.zeros(x.shape)
    for r in range(0, rows, high):
        for c in range(0, cols, BLOCK):
            v = x[r:r + high, c:c + BLOCK]
            fine = np.abs(v[np.isfinite(v)])
            most = fine.max() if fine.size else 0.0
            k = max(-126, int(np.frexp(most)[1]) - 10) if most else -126
            while 448.0 * 2.0 ** k < most:
                k += 1
            exps[r:r + high, c:c + BLOCK] = k
            vals[r:r + high, c:c + BLOCK] = e4m3(v / 2.0 ** k, 240.0 if k == 120 else 448.0) * 2.0 ** k
    return exps, vals


def e4m3(u, most=448.0):
    """Nearest e4m3 values, ties to even; what is not finite is NaN."""
    u = np.where(np.isfinite(u), u, np.nan)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.maximum(np.floor(np.log2(np.abs(u))), -6.0)
    e = np.where(np.isfinite(e), e, -6.0)
    step = 2.0 ** (e - 3.0)
    return np.clip(np.round(u / step) * step, -most, most)


def values(x, square=False):
    return torch.from_numpy(blocks(x.double().cpu().numpy(), square)[1])


def padded(t, type_, pad, shift, fill=0.0):
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
