"""Microscaled 4-bit floating point (E2M1 elements, one power of two per 32 of K) in numpy float64: quantisation, the scale layout of the
expert products and the expert FFN on quantised operands (test infrastructure only)."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BORDER = (GRID[1:] + GRID[:-1]) / 2


def exponents(v):
    """v float64 [..., K], finite -> exponents [..., K / 32]: floor(log2(max)) - 2, clamped; 0 for a block of zeros."""
    top = np.abs(v.reshape(*v.shape[:-1], -1, 32)).max(axis=-1)
    _, ex = np.frexp(top)                      # top = m 2^ex, 0.5 <= m < 1
    return np.where(top == 0, 0, np.clip(ex - 3, -127, 125)).astype(np.int64)


def codes_of(v, ex):
    """E2M1 codes of v / 2^ex: nearest, ties to the even code, saturating."""
    m = np.ldexp(v.reshape(*v.shape[:-1], -1, 32), -ex[..., None])
    low = np.searchsorted(BORDER, np.abs(m), side="left")
    tie = (low < 7) & (np.abs(m) == BORDER[np.minimum(low, 6)])
    return (low + (tie & (low % 2 == 1)) + 8 * np.signbit(m)).astype(np.uint8).reshape(v.shape)


def values_of(codes, ex):
    """codes [..., K] one per byte -> float64."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return np.ldexp(v.reshape(*v.shape[:-1], -1, 32), ex[..., None]).reshape(v.shape)


def pack(codes):
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(packed):
    return np.stack((packed & 15, packed >> 4), axis=-1).reshape(*packed.shape[:-1], -1)


def quantize_rows(v):
    """float64 [R, K] -> (packed codes [R, K / 2], scale bytes [R, K / 32])."""
    ex = exponents(v)
    return pack(codes_of(v, ex)), (ex + 127).astype(np.uint8)


def dequantize_rows(packed, scale):
    return values_of(unpack(packed), scale.astype(np.int64) - 127)


def scale_place(n, kb, N, K, e=0):
    """Byte of the scale of block kb of column n of expert e."""
    return ((e * (-(-N // 128)) + n // 128) * 2 * (-(-K // 256)) + kb // 4) * 512 + (n % 32) * 16 + (n % 128) // 32 * 4 + kb % 4


def scale_bytes(E, K, N):
    return E * (-(-N // 128)) * (-(-K // 256)) * 1024


def tile_scales(scale):
    """[E, N, K / 32] -> the bytes that the expert products read (127 where no block is)."""
    E, N, KB = scale.shape
    out = np.full(scale_bytes(E, KB * 32, N), 127, dtype=np.uint8)
    e, n, kb = np.meshgrid(np.arange(E), np.arange(N), np.arange(KB), indexing="ij")
    out[scale_place(n, kb, N, KB * 32, e)] = scale
    return out


def quantize_weights(w):
    """float64 [E, K, N] -> (packed codes [E, N, K / 2], scale bytes [E, N, K / 32])."""
    v = np.ascontiguousarray(np.swapaxes(w, 1, 2))
    ex = exponents(v)
    return pack(codes_of(v, ex)), (ex + 127).astype(np.uint8)


def _near(v, ex, rel):
    """What the rounding of v to a code may be off by if v is known to `rel` only: the step across the border it lies next to, else 0."""
    m = np.abs(np.ldexp(v.reshape(*v.shape[:-1], -1, 32), -ex[..., None]))
    low = np.clip(np.searchsorted(BORDER, m), 0, 6)
    step = np.zeros_like(m)
    for i in (np.maximum(low - 1, 0), low):
        close = np.abs(m - BORDER[i]) <= rel(m)
        step = np.maximum(step, np.where(close, GRID[i + 1] - GRID[i], 0.0))
    return np.ldexp(step, ex[..., None]).reshape(v.shape)


def expert_ffn_fp4(xq, sx, lay, topk_w, w1, s1, w3, s3, w2, s2):
    """xq / sx: quantised dispatched rows; w* packed [E, N, K / 2] with row-major scales.  -> (o [P, d], allowance [P, d]): what the result
    may differ by when the accumulations are in fp32, h is rounded to codes from there, and o is not rounded."""
    E = w1.shape[0]
    off, rp, src = lay["expert_offsets"], lay["row_pair"], lay["row_src"]
    wf = None if topk_w is None else topk_w.reshape(-1).astype(np.float64)
    P, d, K1, K2 = rp.size, w2.shape[1], w1.shape[2] * 2, w2.shape[2] * 2
    x = dequantize_rows(xq, sx)
    o, tol = np.zeros((P, d)), np.zeros((P, d))
    eps1, eps2 = (K1 / 64 + 2) * 2.0 ** -22, (K2 / 64 + 2) * 2.0 ** -22   # one fp32 addition per 64 of K, truncation allowed
    for e in range(E):
        r = slice(off[e], off[e + 1])
        if off[e + 1] == off[e]:
            continue
        a, v1, v3, v2 = x[src[r]], dequantize_rows(w1[e], s1[e]), dequantize_rows(w3[e], s3[e]), dequantize_rows(w2[e], s2[e])
        a1, a3 = a @ v1.T, a @ v3.T
        d1, d3 = eps1 * (np.abs(a) @ np.abs(v1).T), eps1 * (np.abs(a) @ np.abs(v3).T)
        sl = a1 / (1 + np.exp(-a1))
        h = sl * a3
        # |silu'| <= 1.1, |silu(a)| <= |a|; exp, division and the products in fp32: 2^-20 of the result is ample for |a1| < 60
        dh = 1.1 * d1 * np.abs(a3) + np.abs(sl) * d3 + 1.1 * d1 * d3 + 2.0 ** -20 * np.abs(h)
        ex = exponents(h)
        hq = values_of(codes_of(h, ex), ex)
        unit = np.repeat(np.ldexp(1.0, ex), 32, axis=-1)
        near = _near(h, ex, lambda m: (dh / unit).reshape(m.shape))
        # the block's scale itself is in doubt where its largest value lies next to a power of two: any code may differ by a whole step then
        top = np.abs(h.reshape(*h.shape[:-1], -1, 32)).max(axis=-1)
        dtop = dh.reshape(*dh.shape[:-1], -1, 32).max(axis=-1)
        edge = np.repeat((np.ldexp(4.0, ex) > top - dtop) | (np.ldexp(8.0, ex) < top + dtop), 32, axis=-1)
        near = np.where(edge, 2 * unit, near)
        w = 1.0 if wf is None else wf[rp[r]][:, None]
        o[r] = w * (hq @ v2.T)
        tol[r] = np.abs(w) * (near @ np.abs(v2).T + eps2 * (np.abs(hq) @ np.abs(v2).T) + 2.0 ** -23 * np.abs(hq @ v2.T))
    return o, tol
