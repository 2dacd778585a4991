"""AdamW as include/tlc.h states it, operation by operation in fp32 on the CPU:
the states, weights and codes that tlc_adamw has to leave, bit for bit."""
import numpy as np
import torch

BLOCK = 256
f32 = np.float32


def factors(t, lr, beta1, beta2, eps, weight_decay, lr_scale=1.0):
    lr = lr * float(f32(lr_scale))
    with np.errstate(divide="ignore"):
        log1, log2 = np.log(beta1), np.log(beta2)
    return dict(rate=f32(lr / -np.expm1(t * log1)), root=f32(1.0 / np.sqrt(-np.expm1(t * log2))),
                decay=f32(lr * weight_decay), c1=f32(1.0 - beta1), c2=f32(1.0 - beta2),
                eps=f32(eps))


def fp32_step(p, g, m, v, coef, f):
    """p, g, m, v: float32 arrays.  Returns the new p (before its rounding), m, v."""
    with np.errstate(all="ignore"):
        g = f32(coef) * g
        m = m + (g - m) * f["c1"]
        v = v + (g * g - v) * f["c2"]
        new = p - (f["rate"] * (m / (np.sqrt(v) * f["root"] + f["eps"])) + f["decay"] * p)
    return new, m, v


def numpy_of(t):
    return t.detach().cpu().float().numpy().reshape(-1)


def rounded(x, dtype):
    return torch.from_numpy(x).to(dtype)


def decode(codes, dtype, scales, column):
    """float32 values of the codes (a torch tensor of `dtype` on the CPU)."""
    x = codes.view(dtype).float().numpy().reshape(-1)
    s = np.repeat(scales[:, column], BLOCK)[:x.size]
    with np.errstate(all="ignore"):
        return x * s


def dither(n, t):
    k = np.arange(n, dtype=np.uint64)
    h = k * np.uint64(0xC13FA9A9) + np.uint64(t) * np.uint64(0x91E10DA5)
    return h & np.uint64(0xffffffff)


def _codes(y, h, bits, mantissa, lowest, most):
    """y >= 0 (float32), h: dither as whole numbers of `bits` bits."""
    cut = 23 - mantissa
    assert cut == bits
    word = y.view(np.uint32).astype(np.int64)
    fine = ((word + h) >> cut) - ((126 + lowest) << mantissa)
    small = (np.floor(np.minimum(y.astype(np.float64), 2.0 ** lowest)
                      * 2.0 ** (mantissa - lowest + cut)).astype(np.int64) + h) >> cut
    return np.minimum(np.where(y < 2.0 ** lowest, small, fine), most)


def encode(m, v, t):
    """Codes (uint8) of m and v and the scales [blocks, 2]."""
    n = m.size
    nb = -(-n // BLOCK)
    h = dither(n, t).astype(np.int64)
    scales = np.zeros((nb, 2), f32)
    codes = []
    for c, (x, most) in enumerate(((m, 448), (v, 57344))):
        pad = np.zeros(nb * BLOCK, f32)
        pad[:n] = np.abs(x)
        big = pad.reshape(nb, BLOCK).max(1)  # NaN where there is one
        with np.errstate(all="ignore"):
            s = np.where(big == 0, f32(0), np.maximum(big * (f32(1) / f32(most)), f32(2.0 ** -126)))
        s = np.where(np.isfinite(big), s, f32(np.nan)).astype(f32)
        scales[:, c] = s
        each = np.repeat(s, BLOCK)[:n]
        ok = each > 0
        y = np.zeros(n, f32)
        y[ok] = np.abs(x[ok]) / each[ok]
        if c == 0:
            q = _codes(y, h >> 12, 20, 3, -6, 126) | (np.signbit(x).astype(np.int64) << 7)
        else:
            q = _codes(y, (h ^ 0x80000000) >> 11, 21, 2, -14, 123)
            q = np.where((q == 0) & (x > 0), 1, q)
        codes.append(np.where(np.isnan(each), 0, q).astype(np.uint8))
    return codes[0], codes[1], scales
