"""The 4-bit format from its definition, in 64 bits (numpy), for the tests of the kernels that write and read it."""
import numpy as np

GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6], np.float64)


def quantize(v):
    """f32 [..., blocks, 32] -> codes u8 (0 .. 15) of that shape, scale bytes u8 [..., blocks], values f64 (NaN where a block has Inf or NaN)."""
    v = np.asarray(v, np.float32).astype(np.float64)
    fine = np.isfinite(v).all(-1)
    safe = np.where(fine[..., None], v, 0.0)
    top = np.abs(safe).max(-1)
    e = np.frexp(top)[1].astype(np.int64) - 1  # floor(log2), for top > 0
    byte = np.where(top > 0, np.maximum(e - 2 + 127, 0), 0)
    a = np.abs(safe) * np.exp2(127.0 - byte)[..., None]
    code = np.zeros(v.shape, np.uint8)
    for c in range(7):  # past the midpoint between two codes, or on it where the upper one is even
        mid = (GRID[c] + GRID[c + 1]) / 2
        code += (a >= mid) if c % 2 else (a > mid)
    values = np.copysign(GRID[code], safe) * np.exp2(byte - 127.0)[..., None]
    code = code | (np.signbit(safe).astype(np.uint8) << 3)
    values[~fine] = np.nan
    code[~fine] = 0
    return code, np.where(fine, byte, 255).astype(np.uint8), values


def blocks_of(v):
    """[..., n] -> [..., ceil(n / 32), 32], filled up with zeros."""
    v = np.asarray(v)
    n = v.shape[-1]
    out = np.zeros(v.shape[:-1] + (-(-n // 32) * 32,), v.dtype)
    out[..., :n] = v
    return out.reshape(v.shape[:-1] + (-1, 32))


def pack(code):
    """codes [..., blocks, 32] -> bytes [..., blocks * 16], the even value in the low half."""
    c = code.reshape(code.shape[:-2] + (-1, 2))
    return c[..., 0] | (c[..., 1] << 4)


def message(d, layers):
    """One worker's message for a difference f32 [N]: codes, scales, C(d) f64 (0 where a block is absent), which elements are absent, err f64 [L]
    (Inf for a layer with an absent block)."""
    codes, scales, values, absent, err, at = [], [], [], [], [], 0
    for n in layers:
        part = d[at:at + n]
        code, byte, v = quantize(blocks_of(part))
        v = v.reshape(-1)[:n]
        gone = np.isnan(v)
        codes.append(pack(code).reshape(-1))
        scales.append(byte)
        values.append(np.where(gone, 0.0, v))
        absent.append(gone)
        err.append(np.inf if gone.any() else np.sum((part.astype(np.float64) - v) ** 2))
        at += n
    return np.concatenate(codes), np.concatenate(scales), np.concatenate(values), np.concatenate(absent), np.array(err)


def scale_tiles(byte):
    """[lines, blocks] -> [line tiles, block tiles, 512]: line r, block b of a tile of 128 by 4 at (r % 32) * 16 + r // 32 * 4 + b."""
    lines, nb = byte.shape
    lt, bt = -(-lines // 128), -(-nb // 4)
    out = np.zeros((lt, bt, 512), np.uint8)
    for r in range(lines):
        for b in range(nb):
            out[r // 128, b // 4, r % 32 * 16 + r % 128 // 32 * 4 + b % 4] = byte[r, b]
    return out


def operand(m):
    """f32 [lines, length] -> codes u8 [lines, 16 * blocks], scale tiles u8, values f64."""
    code, byte, v = quantize(blocks_of(m))
    return pack(code).reshape(len(m), -1), scale_tiles(byte), v.reshape(len(m), -1)[:, :m.shape[1]]


def hard_values(shape, rng):
    """Values where the format can go wrong: ties, the cut above 6 scales, zeros of both signs, subnormal and huge numbers, blocks of very different
    sizes, powers of two."""
    n = int(np.prod(shape))
    v = rng.standard_normal(n).astype(np.float32)
    kind = rng.integers(0, 8, -(-n // 32)).repeat(32)[:n]
    ties = (rng.integers(-32, 33, n) / 4).astype(np.float32)
    v = np.where(kind == 1, ties, v)
    v = np.where(kind == 2, v * np.exp2(rng.integers(-20, 20, n)).astype(np.float32), v)
    v = np.where(kind == 3, np.float32(0), v)
    v = np.where(kind == 4, v * np.float32(1e-40), v)
    v = np.where(kind == 5, np.clip(v, -2.9, 2.9) * np.float32(1e38), v)
    v = np.where(kind == 6, np.exp2(rng.integers(-4, 4, n)).astype(np.float32) * np.sign(v), v)
    v = np.where(rng.random(n) < 0.02, np.float32(-0.0), v)
    return v.astype(np.float32).reshape(shape)
