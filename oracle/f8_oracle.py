"""Plain numpy statement, in 64 bits, of the operators on 8-bit floats with block scales, root-mean-square norms and orthogonalised updates.

Test infrastructure only; shares nothing with the CUDA path.  Codes are one uint8 per element and scales one byte per block of 128 of a row; `pack` and `unpack`
go to and from the layout that the library keeps them in.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
NAN_SCALE = 255
_TYPES = {"e4m3": (3, 7, 448.0), "e5m2": (2, 15, 57344.0)}   # bits of mantissa, bias, largest value


def grid(kind: str) -> np.ndarray:
    """The values of the codes from 0 up, without sign, infinities and NaN."""
    mantissa, bias, most = _TYPES[kind]
    code = np.arange(128)
    e, m = code >> mantissa, (code & ((1 << mantissa) - 1)) / (1 << mantissa)
    v = np.where(e > 0, np.ldexp(1.0 + m, e - bias), np.ldexp(m, 1 - bias))
    return v[v <= most]


def _blocks(x: np.ndarray, square: bool) -> np.ndarray:
    """The largest size in each row's blocks; with `square` in blocks of 128 x 128, repeated."""
    rows, cols = x.shape
    nb = (cols + BLOCK - 1) // BLOCK
    most = np.zeros((rows, nb))
    for b in range(nb):
        most[:, b] = np.abs(x[:, b * BLOCK:(b + 1) * BLOCK]).max(1) if rows else 0
    if square:
        for r in range(0, rows, BLOCK):
            most[r:r + BLOCK] = most[r:r + BLOCK].max(0)
    return most


def encode(x: np.ndarray, kind: str, square: bool = False):
    """(codes, scales) of the rows of x (float64)."""
    rows, cols = x.shape
    values = grid(kind)
    most = _blocks(x, square)                                            # (a NaN stays one)
    bad = ~np.isfinite(most)
    limits = np.ldexp(values[-1], np.arange(-127, 128))
    e = np.searchsorted(limits, np.where(bad, 0.0, most)) - 127          # the least e with most <= the largest value times 2^e
    wide = np.repeat(e, BLOCK, 1)[:, :cols]
    gone = np.repeat(bad, BLOCK, 1)[:, :cols]
    y = np.ldexp(np.abs(np.where(gone, 0.0, x)), -wide)
    mid = (values[:-1] + values[1:]) / 2
    low = np.searchsorted(mid, y, side="left")                           # a tie goes to the code below ...
    tie = (low < mid.size) & (y == mid[np.minimum(low, mid.size - 1)])
    code = low + (tie & (low % 2 == 1)) + 128 * np.signbit(x)            # ... unless that one is odd
    return np.where(gone, 0, code).astype(np.uint8), np.where(bad, NAN_SCALE, e + 127).astype(np.uint8)


def decode(codes: np.ndarray, scales: np.ndarray, kind: str) -> np.ndarray:
    """The values, float64."""
    s = np.repeat(np.where(scales == NAN_SCALE, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127)), BLOCK, 1)[:, :codes.shape[1]]
    return np.where(codes & 128, -1.0, 1.0) * grid(kind)[codes & 127] * s


def _scale_at(rows: int, cols: int) -> np.ndarray:
    """Where the scale of every row's block lies."""
    r, b, tiles = np.arange(rows)[:, None], np.arange((cols + 127) // 128)[None, :], (cols + 511) // 512
    return ((r // 128) * tiles + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def pack(codes: np.ndarray, scales: np.ndarray):
    """The two flat byte arrays of a form."""
    rows, cols = codes.shape
    full = np.zeros((rows, (cols + 127) // 128 * 128), np.uint8)
    full[:, :cols] = codes
    out = np.zeros((rows + 127) // 128 * ((cols + 511) // 512) * 512, np.uint8)
    out[_scale_at(rows, cols)] = scales
    return full.reshape(-1), out


def unpack(code_bytes: np.ndarray, scale_bytes: np.ndarray, rows: int, cols: int):
    full = code_bytes.reshape(rows, (cols + 127) // 128 * 128)
    assert not full[:, cols:].any(), "codes past a row's end"
    at = _scale_at(rows, cols)
    rest = scale_bytes.copy()
    rest[at] = 0
    assert not rest.any(), "scales of rows or blocks that do not exist"
    return full[:, :cols].copy(), scale_bytes[at]


def rms_norm(h: np.ndarray, w: np.ndarray, eps: float):
    """(y, 1 / sqrt(mean h^2 + eps) as float32): y is formed with the root as it is stored."""
    with np.errstate(all="ignore"):
        r = (1.0 / np.sqrt((h * h).mean(1) + eps)).astype(np.float32)
        return h * r.astype(np.float64)[:, None] * w, r


def rms_norm_grad(dy: np.ndarray, h: np.ndarray, w: np.ndarray, r: np.ndarray):
    """(dx, dw), without what reaches h another way; r: the stored roots."""
    n = h * r.astype(np.float64)[:, None]
    g = dy * w
    return r.astype(np.float64)[:, None] * (g - n * (g * n).mean(1, keepdims=True)), (dy * n).sum(0)


def orthogonalise(x: np.ndarray, steps: int, coefficients, scale: float = 1.0) -> np.ndarray:
    """One matrix."""
    a, b, c = coefficients
    flip = x.shape[0] > x.shape[1]
    y = x.T if flip else x
    norm = np.sqrt((y * y).sum())
    y = y / norm if norm != 0 else y
    for _ in range(steps):
        g = y @ y.T
        y = a * y + (b * g + c * (g @ g)) @ y
    return scale * (y.T if flip else y)
