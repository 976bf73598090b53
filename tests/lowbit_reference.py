"""Plain 64-bit statements (numpy) of the microscaled 4-bit operators and of the 8-bit key/value cache, for the tests."""
from __future__ import annotations

import numpy as np

NVFP4, MXFP4 = 0, 1
INT8, E4M3 = 0, 1
E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])
_b = np.arange(256)
_e, _m = (_b >> 3) & 15, _b & 7
E4M3_VALUES = np.where(_b & 128, -1.0, 1.0) * np.where(_e > 0, (8 + _m) * 2.0 ** (_e - 10), _m * 2.0 ** -9)
E4M3_VALUES[[0x7F, 0xFF]] = np.nan


def block(fmt):
    return 16 if fmt == NVFP4 else 32


def round_steps(x, step):
    return np.rint(x / step) * step


def floor_log2(x):
    return np.frexp(x)[1] - 1


def to_e4m3(x):
    """Nearest e4m3 number, ties to even, at most 448."""
    x = np.asarray(x, np.float64)
    return np.clip(round_steps(x, 2.0 ** (np.maximum(floor_log2(np.maximum(np.abs(x), 2.0 ** -40)), -6) - 3)), -448, 448)


def to_e2m1(y):
    m = np.abs(y)
    return np.clip(round_steps(y, np.where(m < 2, .5, np.where(m < 4, 1.0, 2.0))), -6, 6)


def f32(x):
    return np.asarray(x, np.float32).astype(np.float64)


def mx4_quantize(x, fmt, g=1.0):
    """float64 [M, K] -> (values of the codes, block scales), the roundings of the definition in their places."""
    M, K = x.shape
    b = x.reshape(M, -1, block(fmt))
    a = np.abs(b).max(-1)
    if fmt == NVFP4:
        sc = to_e4m3(f32(f32(a / 6) / g))
        with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
            inv = np.where(sc > 0, f32(1.0 / f32(sc * g)), 0.0)
        y = f32(b * inv[..., None])
        y = np.where(np.abs(y) < 8, round_steps(y, 2.0 ** -19), y)
    else:
        e = np.where(a > 0, np.maximum(floor_log2(np.maximum(a, 1e-300)) - 2, -127), -127)
        sc = 2.0 ** e
        y = b / sc[..., None]
    return to_e2m1(y).reshape(M, K), sc


def scale_bytes_to_values(byte, fmt):
    return E4M3_VALUES[byte] if fmt == NVFP4 else 2.0 ** (byte.astype(np.float64) - 127)


def untile(raw, rows, nb):
    """Scale bytes of [rows][blocks] out of the stored tiles."""
    r, k = np.arange(rows)[:, None], np.arange(nb)[None, :]
    return raw.reshape(-1)[((r // 128) * -(-nb // 4) + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4]


def tile(byte, fill=0):
    rows, nb = byte.shape
    rt, kt = -(-rows // 128), -(-nb // 4)
    out = np.full(rt * kt * 512, fill, np.uint8)
    r, k = np.arange(rt * 128)[:, None], np.arange(kt * 4)[None, :]
    full = np.full((rt * 128, kt * 4), fill, np.uint8)
    full[:, nb:] = 0
    full[:rows, :nb] = byte
    out[((r // 128) * kt + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4] = full
    return out


def nibbles(codes):
    """uint8 [M, K/2] -> code numbers [M, K]."""
    return np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1)


def mx4_values(codes, byte, fmt, g=1.0):
    n = E2M1[nibbles(codes)]
    M, K = n.shape
    return (n.reshape(M, -1, block(fmt)) * scale_bytes_to_values(byte, fmt)[..., None]).reshape(M, K) * (g if fmt == NVFP4 else 1.0)
