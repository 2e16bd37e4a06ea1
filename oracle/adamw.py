"""One AdamW step in 64 bits (Loshchilov & Hutter's decoupled decay; Kingma & Ba's bias corrections), with 8-bit moments.

An 8-bit moment is an e4m3 number (1 sign, 4 exponent bits of bias 7, 3 mantissa bits; no infinities, 0x7f NaN) times a power of two that
128 consecutive elements share.  It is rounded at random: up where the place between the two neighbours plus a 16-bit random
number / 2^16 reaches one.  The random bits are a 32-bit hash of (seed, step, tensor, element)."""
import numpy as np

GROUP = 128
M32 = np.uint64(0xFFFFFFFF)


def mix(x):
    """32-bit hash of uint64 arrays (or ints) below 2^32."""
    x = np.asarray(x, dtype=np.uint64)
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x9E3779B1)) & M32
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0xBB67AE85)) & M32
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, tensor, n, first=0):
    """uint32 hash of every element first .. first + n - 1 of a tensor, as uint64."""
    k = mix(((seed & 0xFFFFFFFF) + 0x9E3779B1 * (tensor + 1)) & 0xFFFFFFFF)
    k = mix(int(k) ^ (seed >> 32))
    k = mix((int(k) + step) & 0xFFFFFFFF)
    k = mix(int(k) ^ (step >> 32))
    e = np.arange(first, first + n, dtype=np.uint64)
    low = ((e & M32) + ((e >> np.uint64(32)) * np.uint64(0x9E3779B1) & M32)) & M32
    return mix(low ^ k)


def e4m3_values():
    """The 256 numbers by their byte."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    x = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * 2.0 ** (e - 7.0))
    x[(c & 127) == 127] = np.nan
    return np.where(c & 128, -x, x)


def unpack(code, byte):
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return e4m3_values()[code] * np.repeat(scale, GROUP)[:code.size]


def pack(x, dither, positive):
    """(values, bytes of the scales) of x: what the 8-bit numbers stand for without their scales."""
    x = np.asarray(x, dtype=np.float64)
    n = x.size
    rows = np.abs(np.concatenate([x, np.zeros(-n % GROUP)])).reshape(-1, GROUP)
    byte = np.zeros(len(rows), dtype=np.int64)
    val = np.zeros(rows.shape)
    d = np.concatenate([dither, np.zeros(-n % GROUP, dtype=np.uint64)]).reshape(-1, GROUP).astype(np.float64)
    for r, row in enumerate(rows):
        if not np.all(np.isfinite(row)):
            byte[r] = 255
            continue
        top = row.max()
        k = -127
        if top > 0:
            f, e = np.frexp(top)           # top = f * 2^e, f in [0.5, 1)
            k = max(int(e) - 9 + (1 if f > 0.875 else 0), -127)
        byte[r] = k + 127
        y = row * 2.0 ** -k
        step = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
        val[r] = np.floor(y / step + d[r] / 65536) * step
    val = val.reshape(-1)[:n]
    if positive:
        val = np.where((x > 0) & (val == 0) & np.isfinite(x), 2.0 ** -9, val)
    else:
        val = val * np.where(x < 0, -1.0, 1.0)
    return val, byte


def round_bf16_random(w, random16):
    w = np.asarray(w, dtype=np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(w), 2.0 ** -126))) - 7)
    return np.floor(np.abs(w) / step + random16.astype(np.float64) / 65536) * step * np.where(w < 0, -1.0, 1.0)


def step(w, m, v, grad_parts, *, lr, beta1, beta2, eps, t, decay, grad_scale=1.0):
    """(w, m, v) after step t; grad_parts [parts, n]."""
    g = np.asarray(grad_parts, dtype=np.float64).sum(axis=0) * grad_scale
    m = beta1 * np.asarray(m, dtype=np.float64) + (1 - beta1) * g
    v = beta2 * np.asarray(v, dtype=np.float64) + (1 - beta2) * g * g
    mh, vh = m / (1 - beta1 ** t), v / (1 - beta2 ** t)
    return w - lr * (mh / (np.sqrt(vh) + eps) + decay * np.asarray(w, dtype=np.float64)), m, v
