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


# ------------------------------------------------------------------------------------------- 8-bit key/value cache

def kv_values(raw, kind):
    """Codes (uint8 bytes) -> numbers without their scale."""
    return raw.view(np.int8).astype(np.float64) if kind == INT8 else E4M3_VALUES[raw]


def kv_scale(amax, kind):
    """fp32 scale of a block, from the fp32 largest magnitude."""
    amax = np.float32(amax)
    if kind == INT8:
        s = np.float32(amax / np.float32(127))
        return s if s >= 2.0 ** -100 else np.float32(0)
    if not amax > 0:
        return np.float32(0)
    e = -100
    while float(amax) > 448 * 2.0 ** e:
        e += 1
    return np.float32(2.0 ** e)


def kv_round(y, kind):
    """fp32 quotients -> codes, as numbers."""
    y = np.asarray(y, np.float32).astype(np.float64)
    return np.clip(np.rint(y), -127, 127) if kind == INT8 else to_e4m3(y)


def inverse(scale):
    return np.float32(0) if scale == 0 else np.float32(1) / np.float32(scale)


def kv_append(codes, scales, table, lens, cu, rows, kind, P):
    """codes [pages, H, P, D] (numbers), scales [pages, H] fp32, rows [T, H, D] fp32: changed in place."""
    pages, H = scales.shape
    for b in range(len(lens)):
        n = cu[b + 1] - cu[b]
        start = lens[b] - n
        for j in range(table.shape[1]):
            lo, hi = j * P, (j + 1) * P
            t0, t1 = max(start, 0, lo), min(lens[b], hi)
            page = table[b, j]
            if t0 >= t1 or not 0 <= page < pages:
                continue
            for h in range(H):
                x = rows[cu[b] + t0 - start: cu[b] + t1 - start, h].astype(np.float32)
                before = scales[page, h] if t0 > max(lo, 0) else np.float32(0)
                s = max(before, kv_scale(np.abs(x).max(), kind))
                if t0 > lo and s > before:
                    codes[page, h, :t0 - lo] = kv_round(codes[page, h, :t0 - lo].astype(np.float32) * np.float32(before / s), kind)
                codes[page, h, t0 - lo:t1 - lo] = kv_round(x * inverse(s), kind)
                scales[page, h] = s


def kv_tokens(codes, scales, table_row, n, P):
    """Tokens 0 .. n-1 of a sequence [n, H, D] in 64 bits and whether each exists."""
    pages, H = scales.shape
    out, there = np.zeros((n, H, codes.shape[3])), np.zeros(n, bool)
    for t in range(n):
        page = table_row[t // P] if t // P < len(table_row) else -1
        if 0 <= page < pages:
            there[t] = True
            out[t] = codes[page, :, t % P] * scales[page].astype(np.float64)[:, None]
    return out, there


def attention(q, k, v, there, n_q, causal, scale):
    """q [n_q, Hq, D], k, v [len, H, D]: out [n_q, Hq, D], lse [n_q, Hq], and what the tolerances need: the largest sum
    of |q k| scale of a row, sum p |v|, max p vs-weighted."""
    G = q.shape[1] // k.shape[1]
    n = k.shape[0]
    kk, vv = np.repeat(k, G, 1), np.repeat(v, G, 1)
    s = np.einsum("ihd,thd->iht", q, kk) * scale
    mag = (np.einsum("ihd,thd->iht", np.abs(q), np.abs(kk)) * abs(scale)).max(-1) if n else np.zeros(q.shape[:2])
    seen = np.broadcast_to(there[None, :], (n_q, n)).copy()
    if causal:
        seen &= np.arange(n)[None, :] <= (n - n_q + np.arange(n_q))[:, None]
    s = np.where(seen[:, None, :], s, -np.inf)
    top = s.max(-1, initial=-np.inf)
    ref = np.where(np.isfinite(top), top, 0)
    p = np.exp(s - ref[..., None])
    total = p.sum(-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        p = np.where(total[..., None] > 0, p / np.where(total > 0, total, 1)[..., None], 0)
        lse = np.where(total > 0, ref + np.log(total), -np.inf)
    return np.einsum("iht,thd->ihd", p, vv), lse, mag, np.einsum("iht,thd->ihd", p, np.abs(vv)), p
