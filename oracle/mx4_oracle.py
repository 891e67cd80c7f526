"""Plain numpy statement, in 64 bits, of the operators on microscaled 4-bit floats and counter-based draws.

Test infrastructure only; shares nothing with the CUDA path.  Codes are one uint8 (0..15) per element and scales one byte per block of 32
of a row; `pack` and `unpack` go to and from the layout that the library keeps them in.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
DROPOUT, ROUNDING = 0, 1
NAN_SCALE = 255
_M = (1 << 64) - 1
_G = 0x9E3779B97F4A7C15


def _mix(z: int) -> int:
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & _M
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & _M
    return z ^ (z >> 31)


def stream(seed: int, worker: int, tensor: int, step: int) -> int:
    key = _mix((seed + worker + 1) & _M)
    return _mix((_mix((key + _G * (tensor + 1)) & _M) + _G * (step + 1)) & _M)


def numbers(seed: int, worker: int, tensor: int, step: int, rows: int, cols: int, which: int) -> np.ndarray:
    """The 16-bit number of every element of a rows x cols matrix."""
    s = stream(seed, worker, tensor, step)
    r, c = np.arange(rows, dtype=np.uint64)[:, None], np.arange(cols, dtype=np.uint64)[None, :]
    with np.errstate(over="ignore"):
        j = np.uint64(2) * (r * np.uint64((cols + 3) // 4) + c // np.uint64(4)) + np.uint64(which)
        z = np.uint64(s) + np.uint64(_G) * (j + np.uint64(1))
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    return ((z >> (np.uint64(16) * (c % np.uint64(4)))) & np.uint64(0xFFFF)).astype(np.int64)


def dropout(x: np.ndarray, p: float, u: np.ndarray) -> np.ndarray:
    """x (float64) behind a dropout, u the numbers of its elements."""
    f = int(np.rint(p * 65536))
    return np.where(u >= f, x * (65536.0 / max(1, 65536 - f)), 0.0)


def encode(x: np.ndarray, u=None):
    """(codes, scales) of the rows of x (float64); u: numbers of a stochastic rounding."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((rows, nb), np.uint8)
    limits = np.ldexp(6.0, np.arange(-127, 128))
    mid = (GRID[:-1] + GRID[1:]) / 2
    for b in range(nb):
        v = x[:, 32 * b:32 * b + 32]
        bad = ~np.isfinite(v).all(1)
        v = np.where(bad[:, None], 0.0, v)
        e = np.searchsorted(limits, np.abs(v).max(1)) - 127          # the least e with max <= 6 2^e
        y = np.ldexp(np.abs(v), -e[:, None])
        if u is None:
            low = np.searchsorted(mid, y, side="left")               # a tie goes to the code below ...
            tie = (low < 7) & (y == mid[np.minimum(low, 6)])
            c = low + (tie & (low % 2 == 1))                         # ... unless that one is odd
        else:
            low = np.minimum(np.searchsorted(GRID, y, side="right") - 1, 6)
            f = (y - GRID[low]) / (GRID[low + 1] - GRID[low])
            c = low + (np.floor(f * 65536 + 0.5) + u[:, 32 * b:32 * b + 32] >= 65536)
        c = c + 8 * np.signbit(v)
        codes[:, 32 * b:32 * b + 32] = np.where(bad[:, None], 0, c)
        scales[:, b] = np.where(bad, NAN_SCALE, e + 127)
    return codes, scales


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The values, float64."""
    s = np.repeat(np.where(scales == NAN_SCALE, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127)), 32, 1)[:, :codes.shape[1]]
    return np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7] * s


def pack(codes: np.ndarray, scales: np.ndarray):
    """The two flat byte arrays of a form."""
    rows, cols = codes.shape
    nb, tiles = (cols + 31) // 32, (cols + 127) // 128
    full = np.zeros((rows, nb * 32), np.uint8)
    full[:, :cols] = codes
    out = np.zeros((rows + 127) // 128 * tiles * 512, np.uint8)
    for r in range(rows):
        for b in range(nb):
            out[((r // 128) * tiles + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4] = scales[r, b]
    return (full[:, 0::2] | (full[:, 1::2] << 4)).reshape(-1), out


def unpack(code_bytes: np.ndarray, scale_bytes: np.ndarray, rows: int, cols: int):
    nb, tiles = (cols + 31) // 32, (cols + 127) // 128
    raw = code_bytes.reshape(rows, nb * 16)
    full = np.stack([raw & 15, raw >> 4], -1).reshape(rows, nb * 32)
    assert not full[:, cols:].any(), "codes past a row's end"
    s = np.empty((rows, nb), np.uint8)
    rest = scale_bytes.copy()
    for r in range(rows):
        at = ((r // 128) * tiles + np.arange(nb) // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + np.arange(nb) % 4
        s[r] = scale_bytes[at]
        rest[at] = 0
    assert not rest.any(), "scales of rows or blocks that do not exist"
    return full[:, :cols].copy(), s
