"""Block-scaled formats in plain numpy, 64 bits: what the kernels' results are compared with.

A block of 32 values shares 2^(s - 127), s = clamp(floor(log2 of the largest magnitude) - lead, -127, ..) + 127;
elements are the values over it, rounded to the nearest of the format's grid, the even code of two, cut at the
grid's end.  A block holding Inf or NaN has s = 255 and zero elements."""
import numpy as np

E2M1, E4M3 = 0, 1
LEAD = {E2M1: 2, E4M3: 8}
GRID = {E2M1: np.array([0, .5, 1, 1.5, 2, 3, 4, 6]),
        E4M3: np.array([m / 8 * 2.0 ** -6 for m in range(8)] +
                       [(1 + m / 8) * 2.0 ** (p - 7) for p in range(1, 16) for m in range(8)][:-1])}


def bf16_values(bits):
    return (np.asarray(bits, np.uint32) << 16).view(np.float32).astype(np.float64)


def quantize(x, fmt):
    """float64 [..., K] -> (codes uint8 [..., K] one per value, scale bytes [..., K / 32])."""
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    m = np.abs(b).max(-1)
    power = np.frexp(np.where(m > 0, m, 1.0))[1] - 1
    e = np.where(m > 0, np.clip(power - LEAD[fmt], -127, 127), -127)
    a = np.abs(b) / 2.0 ** e[..., None].astype(np.float64)
    grid = GRID[fmt]
    mid = (grid[1:] + grid[:-1]) / 2
    low, high = np.searchsorted(mid, a, side="left"), np.searchsorted(mid, a, side="right")
    code = np.where(low % 2 == 0, low, high)
    code = (code | np.where(np.signbit(b), 8 if fmt == E2M1 else 128, 0)).astype(np.uint8)
    code[bad] = 0
    scale = np.where(bad, 255, e + 127).astype(np.uint8)
    return code.reshape(x.shape), scale


def pack(codes, fmt):
    """One code per value -> the bytes of the elements."""
    return codes if fmt == E4M3 else (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(elements, fmt):
    if fmt == E4M3:
        return elements
    out = np.empty((*elements.shape[:-1], elements.shape[-1] * 2), np.uint8)
    out[..., 0::2], out[..., 1::2] = elements & 15, elements >> 4
    return out


def values(codes, scales, fmt):
    """float64 values of one code per value and scale bytes."""
    top = 8 if fmt == E2M1 else 128
    grid = np.concatenate([GRID[fmt], [np.nan]]) if fmt == E4M3 else GRID[fmt]
    v = np.where(codes & top, -1.0, 1.0) * grid[codes & (top - 1)]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v.reshape(*codes.shape[:-1], -1, 32) * s[..., None]).reshape(codes.shape)


def rounded(x, fmt):
    """x as the format holds it."""
    return values(*quantize(x, fmt), fmt)


def round_bf16(x):
    """float64 -> nearest bf16 value (ties to even), subnormals and overflow included."""
    x = np.asarray(x, np.float64)
    e = np.maximum(np.frexp(x)[1] - 1, -126)
    step = 2.0 ** (e - 7.0)
    with np.errstate(over="ignore", invalid="ignore"):
        r = np.rint(x / step) * step
        return np.where(np.isnan(x), np.nan, np.where(np.abs(r) >= 2.0 ** 128, np.copysign(np.inf, x), r))
