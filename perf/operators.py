"""Timed cases of the low-bit decoder operators: microscaled 4-bit floating point (quantizer and product), the paged
8-bit key/value cache with the attention that reads it, and the operations on the cache's pages.

Each case is one call (or the few calls) that a user's program makes. `run` computes it in elementary torch operations
where `own` is false and through the framework's binding where it is true; `exact` states the same result in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
NVFP4, MXFP4 = 0, 1          # microscaled formats: blocks of 16 with e4m3 scales / blocks of 32 with power-of-two scales
INT8, E4M3 = 0, 1            # what the cache holds
F16 = {"fp16": torch.float16, "bf16": torch.bfloat16}
TYPE = {"fp16": 0, "bf16": 1}


# --------------------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # the activations of 16 observations of 288 tokens before a projection
        dict(name="quantize 4608x4096", kind="quantize", format=NVFP4, dtype="fp16", M=4608, K=4096, pad=0),
        # a ragged handful of rows of the gated MLP's width, rows with a pitch of their own
        dict(name="quantize 37x11008", kind="quantize", format=MXFP4, dtype="bf16", M=37, K=11008, pad=64),
        # the fused QKV projection of one decode token: latency and the weight stream
        dict(name="linear 1x12288x4096", kind="linear", format=NVFP4, dtype="fp16", M=1, N=12288, K=4096),
        # the down projection of one observation after its visual tokens were pruned
        dict(name="linear 160x4096x11008", kind="linear", format=MXFP4, dtype="bf16", M=160, N=4096, K=11008),
        # the fused QKV projection of 16 observations: the large product
        dict(name="linear 4608x12288x4096", kind="linear", format=NVFP4, dtype="fp16", M=4608, N=12288, K=4096),
        # prompts of 16 observations enter an empty cache
        dict(name="append 16x288", kind="append", type=INT8, dtype="fp16", batch=16, heads=32, kv_heads=32, head_dim=128,
             page=64, new=288, old=0, ragged=0),
        # one decode step of 16 observations: the new token enters the cache, then attends to it
        dict(name="step 16x290", kind="step", type=INT8, dtype="fp16", batch=16, heads=32, kv_heads=32, head_dim=128,
             page=64, new=1, old=290, ragged=3),
        # a decode step over long, uneven histories with shared key/value heads
        dict(name="decode 32x16384", kind="attend", type=E4M3, dtype="bf16", batch=32, heads=32, kv_heads=8, head_dim=128,
             page=64, new=1, old=16384, ragged=5, causal=True),
        # the prompts of 16 observations
        dict(name="prompt 16x288", kind="attend", type=INT8, dtype="fp16", batch=16, heads=32, kv_heads=32, head_dim=128,
             page=64, new=288, old=0, ragged=0, causal=True),
        # long prompts that follow a cached prefix, shared heads, an odd length
        dict(name="prompt 2x4099+1000", kind="attend", type=E4M3, dtype="bf16", batch=2, heads=32, kv_heads=8, head_dim=128,
             page=32, new=4099, old=1000, ragged=0, causal=True),
        # eight action candidates are decoded from each of 16 observations
        dict(name="fork 16 to 128", kind="fork", type=INT8, dtype="fp16", batch=16, copies=8, kv_heads=32, head_dim=128,
             page=64, old=295, ragged=0),
        # the cache of a layer in front of the pruning is brought down to the tokens that were kept
        dict(name="compact 16x288 to 160", kind="compact", type=INT8, dtype="fp16", batch=16, kv_heads=32, head_dim=128,
             page=64, old=288, keep=160, ragged=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["fp16", "bf16"])
    kind = rng.choice(["quantize", "linear", "linear", "append", "step", "attend", "attend", "fork", "compact"])
    if kind in ("quantize", "linear"):
        K = 32 * _log(rng, 2, 512)
        c = dict(kind=kind, format=rng.choice([NVFP4, MXFP4]), dtype=dtype, M=_log(rng, 1, 4608), K=K)
        if kind == "quantize":
            c["M"] = min(c["M"], 4608 * 4096 // K)
            c["pad"] = rng.choice([0, 0, 8, 64])
        else:
            c["N"] = min(_log(rng, 17, 22016), max(17, 4608 * 12288 * 4096 // (c["M"] * K)))
        return c
    c = dict(kind=kind, type=rng.choice([INT8, E4M3]), dtype=dtype, page=rng.choice([16, 32, 64, 128]),
             head_dim=rng.choice([64, 128, 128, 256]))
    c["kv_heads"] = rng.choice([1, 2, 4, 8, 32])
    c["ragged"] = rng.randrange(1000)
    width = c["kv_heads"] * c["head_dim"]
    if kind in ("append", "step", "attend"):
        c["heads"] = c["kv_heads"] * rng.choice([1, 1, 2, 4, 7, 8])
    if kind == "append":
        c["batch"] = _log(rng, 1, 48)
        c["new"] = min(_log(rng, 1, 2000), max(1, 16 * 288 * 4096 // (c["batch"] * width)))
        c["old"] = rng.choice([0, _log(rng, 1, 600)])
    elif kind == "step":
        c["batch"], c["new"] = _log(rng, 1, 96), rng.choice([1, 1, 1, 2, 5])
        c["old"] = min(_log(rng, 1, 9000), max(1, 32 * 8192 * 1024 // (c["batch"] * width)))
    elif kind == "attend":
        c["batch"], c["causal"] = _log(rng, 1, 32), rng.random() < 0.7
        c["new"] = rng.choice([1, 1, 3, _log(rng, 8, 2500)])
        c["old"] = rng.choice([0, _log(rng, 1, 16000)])
        rows = 2 * 4099 * 3000 * 32 * 128
        c["new"] = max(1, min(c["new"], rows // (c["batch"] * c["heads"] * c["head_dim"] * 1200)))
        c["old"] = max(0, min(c["old"], rows // (c["batch"] * c["heads"] * c["head_dim"] * c["new"]), 32 * 8192 * 1024 // (c["batch"] * width)))
    elif kind == "fork":
        c["batch"], c["copies"], c["old"] = _log(rng, 1, 24), rng.choice([1, 2, 5, 8]), _log(rng, 1, 900)
    else:
        c["batch"], c["old"] = _log(rng, 1, 32), _log(rng, 2, 2000)
        c["old"] = max(2, min(c["old"], 16 * 288 * 4096 // (c["batch"] * width)))
        c["keep"] = rng.randint(1, c["old"])
    return c


def _lengths(case):
    """Tokens already in the cache, for each sequence: `old` for all of them, or spread below it."""
    if not case["ragged"]:
        return [case["old"]] * case["batch"]
    r = random.Random(case["ragged"])
    return [r.randint(case["old"] // 16, case["old"]) for _ in range(case["batch"])]


def work(case):
    kind = case["kind"]
    if kind in ("quantize", "linear"):
        M, K = case["M"], case["K"]
        blk = 16 if case["format"] == NVFP4 else 32
        packed = lambda rows: rows * K / 2 + rows * K / blk  # noqa: E731
        if kind == "quantize":   # 16-bit rows in; codes and scales, then the 16-bit values they stand for, out
            return {"bytes": 2 * M * K + packed(M) + 2 * M * K, "flops": 3 * M * K}
        return {"bytes": 2 * M * K + packed(case["N"]) + 2 * M * case["N"], "flops": 2.0 * M * case["N"] * K}
    D, H, P = case["head_dim"], case["kv_heads"], case["page"]
    if kind == "fork":     # one unfinished page of each copy is duplicated; its tokens are read back
        n, tail = case["batch"] * case["copies"], [x % P for x in _lengths(case)]
        back = sum(tail) * case["copies"] * H * D
        table = 4.0 * (len(tail) + n) * (max(_lengths(case)) // P + 1)
        return {"bytes": 2.0 * n * 2 * H * D * P * (sum(t > 0 for t in tail) / len(tail)) + 4.0 * back + table, "flops": 2.0 * back}
    if kind == "compact":
        n = case["batch"] * case["keep"] * H * D
        return {"bytes": 2.0 * n * 2 + 4.0 * n, "flops": 8.0 * n}
    new, lens = case["new"], _lengths(case)
    tokens = new * case["batch"]
    if kind == "append":   # keys and values in, codes out, the touched pages read back
        back = sum(x + new - x // P * P for x in lens) * H * D
        return {"bytes": 2 * (2.0 + 1.0) * tokens * H * D + 4.0 * back, "flops": 8.0 * tokens * H * D}
    Hq = case["heads"]
    held = sum(x + new for x in lens)
    pairs = sum(new * x + (new * (new + 1) // 2 if case.get("causal", True) else new * new) for x in lens)
    b = 2.0 * held * H * D + 2 * 2.0 * tokens * Hq * D + 4.0 * tokens * Hq
    if kind == "step":
        b += 2 * 2.0 * tokens * H * D
    return {"bytes": b, "flops": 4.0 * pairs * Hq * D}


# ------------------------------------------------------------------------------------------------------- the inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _table(lens, page, width, spare, g):
    """Pages of every sequence, in no order, and the number of pages in all; -1 behind a sequence's last page."""
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g, device=DEV)[: sum(need)].to(torch.int32)
    t = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    n = torch.tensor(need, device=DEV)
    t[torch.arange(width, device=DEV)[None, :] < n[:, None]] = order
    return t, pages


def _cache(pages, case, g):
    shape = (pages, case["kv_heads"], case["page"], case["head_dim"])
    c = {}
    for n in ("k", "v"):
        x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float16)
        u = torch.rand(shape[:2], generator=g, device=DEV)
        if case["type"] == INT8:
            c[n] = (x * 40).round_().clamp_(-127, 127).to(torch.int8)
            c[n + "s"] = (0.7 + 0.6 * u) / 40
        else:
            c[n] = (x * 100).clamp_(-448, 448).to(torch.float8_e4m3fn)
            c[n + "s"] = torch.where(u < 0.5, 2.0 ** -8, 2.0 ** -7)
    return c


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = {"case": case, "stream": torch.cuda.current_stream().cuda_stream}
    if kind in ("quantize", "linear"):
        M, K, f = case["M"], case["K"], case["format"]
        dt = F16[case["dtype"]]
        x = torch.randn(M, K + case.get("pad", 0), generator=g, device=DEV)
        x[:, torch.randint(0, K, (max(1, K // 100),), generator=g, device=DEV)] *= 20      # a few outlier channels
        s["x"] = x.to(dt)
        # scales of the tensors, as calibration finds them: the largest value meets the largest code and scale
        s["gx"] = (x.abs().amax() / (6 * 448)).reshape(1) if f == NVFP4 else torch.ones(1, device=DEV)
        nb = K // (16 if f == NVFP4 else 32)
        tiles = lambda rows: (-(-rows // 128), -(-nb // 4))  # noqa: E731
        s["codes"] = torch.empty(M, K // 2, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty(*tiles(M), 512, dtype=torch.uint8, device=DEV)
        N = case.get("N", 0)
        if kind == "linear":
            s["wc"] = torch.randint(0, 256, (N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
            lo, hi = (40, 72) if f == NVFP4 else (120, 125)       # e4m3 0.25 .. 4 / powers of two 2^-7 .. 2^-3
            e = torch.randint(lo, hi, (*tiles(N), 512), generator=g, device=DEV, dtype=torch.uint8)
            s["ws"] = _tile(_untile(e, N, nb), N, nb)             # zero behind the last row and block
            s["gw"] = torch.full((1,), 0.02, device=DEV)
        s["out"] = torch.empty(M, (max(N, K) + 7) // 8 * 8, dtype=dt, device=DEV)
        return s

    dt, D, H, P = F16[case["dtype"]], case["head_dim"], case["kv_heads"], case["page"]
    old, B = _lengths(case), case["batch"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    if kind in ("append", "step", "attend"):
        new, Hq = case["new"], case["heads"]
        lens = [n + new for n in old]
        width = -(-max(lens) // P)
        s["table"], pages = _table(lens, P, width, 5, g)
        s.update(_cache(pages, case, g))
        s["lens"], s["max_len"] = ints(lens), max(lens)
        s["cu"] = ints([new * i for i in range(B + 1)])
        first = [n // P * P for n in old]                        # the touched pages, read back
        s["first"], span = ints(first), [n - f for n, f in zip(lens, first)]
        s["back"] = ints([sum(span[:i]) for i in range(B + 1)])
        s["max_back"], rows = max(span), sum(span)
        qkv = torch.randn(B * new, (Hq + 2 * H) * D, generator=g, device=DEV).to(dt)
        s["q"], s["knew"], s["vnew"] = qkv[:, : Hq * D], qkv[:, Hq * D: (Hq + H) * D], qkv[:, (Hq + H) * D:]
        s["out"] = torch.empty(B * new, Hq * D, dtype=dt, device=DEV)
        s["lse"] = torch.empty(B * new, Hq, device=DEV)
    elif kind == "fork":
        C = case["copies"]
        lens = old + [0] * (B * C)
        width = -(-max(old) // P) + 1
        s["table"], pages = _table(lens, P, width, B * C + 3, g)
        s.update(_cache(pages, case, g))
        s["lens"] = ints(lens)
        s["src"], s["dst"] = ints([i // C for i in range(B * C)]), ints([B + i for i in range(B * C)])
        s["pairs"] = torch.empty(B * C, 2, dtype=torch.int32, device=DEV)
        tail = [old[i // C] % P for i in range(B * C)]
        s["first"] = ints([old[i // C] // P * P for i in range(B * C)])
        s["back"] = ints([sum(tail[:i]) for i in range(B * C + 1)])
        s["max_back"], rows = max(tail), sum(tail)
    else:
        keep = [min(case["keep"], n) for n in old]
        lens = old + [0] * B
        width = -(-max(old) // P)
        s["table"], pages = _table(lens, P, width, sum(-(-k // P) for k in keep) + 3, g)
        s.update(_cache(pages, case, g))
        s["lens"] = ints(lens)
        s["src"], s["dst"] = ints(list(range(B))), ints([B + i for i in range(B)])
        s["keep"] = ints(keep)
        key = torch.rand(B, max(old), generator=g, device=DEV)
        key[torch.arange(max(old), device=DEV)[None, :] >= s["lens"][:B, None]] = 2.0
        rank = key.argsort(1).argsort(1)                          # a token stays if it is among the first `keep` of a random order
        stay = rank < s["keep"][:, None]
        pos = torch.where(stay, torch.arange(max(old), device=DEV)[None, :], 1 << 30).sort(1).values
        s["kept"] = torch.where(pos < (1 << 30), pos, -1).to(torch.int32).contiguous()   # ascending, -1 behind the last
        s["first"] = torch.zeros(B, dtype=torch.int32, device=DEV)
        s["back"] = ints([sum(keep[:i]) for i in range(B + 1)])
        s["max_back"], rows = max(keep), sum(keep)
    if kind in ("fork", "compact"):
        s["refs"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
        s["refs"][s["table"][s["table"] >= 0].long()] = 1
    s["kback"], s["vback"] = (torch.empty(max(1, rows), H * D, dtype=dt, device=DEV) for _ in range(2))
    return s


# --------------------------------------------------------------------------- plain forms: microscaled 4-bit numbers

_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _untile(t, rows, nb):
    """Scale bytes as stored (tiles of 128 rows x 4 blocks: 32 x 4 x 4 bytes) -> [rows][blocks]."""
    rt, kt = t.shape[:2]
    return t.reshape(rt, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, kt * 4)[:rows, :nb]


def _tile(b, rows, nb):
    rt, kt = -(-rows // 128), -(-nb // 4)
    full = torch.zeros(rt * 128, kt * 4, dtype=torch.uint8, device=b.device)
    full[:rows, :nb] = b
    return full.reshape(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).reshape(rt, kt, 512).contiguous()


def _quantize(x, fmt, g):
    """Codes [M][K/2] (the even element in the low nibble) and scale bytes [M][blocks]."""
    M, K = x.shape
    b = x.float().reshape(M, -1, 16 if fmt == NVFP4 else 32)
    a = b.abs().amax(-1)
    if fmt == NVFP4:
        sc = ((a / torch.full((), 6.0, device=x.device)) / g).clamp(max=448.0).to(torch.float8_e4m3fn)
        d = sc.float() * g
        inv = torch.where(sc.float() > 0, 1.0 / d, 0.0)
        y = (b * inv[..., None]).abs()
        y = (y + 24.0) - 24.0                  # to a multiple of 2^-19: a quotient that is halfway between two codes stays there
        byte = sc.view(torch.uint8)
    else:
        e = (torch.frexp(a).exponent - 3).clamp(-127, 127)
        e = torch.where(a > 0, e, -127)
        y = (b * ((127 - e) << 23).view(torch.float32)[..., None]).abs()
        byte = (e + 127).to(torch.uint8)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    code = (code + 8 * (b < 0).to(torch.uint8)).reshape(M, K)
    return code[:, 0::2] + 16 * code[:, 1::2], byte


def _values(codes, byte, fmt, g):
    """The numbers, in 32 bits: value of the code x scale of its block x scale of the tensor."""
    M, K = codes.shape[0], 2 * codes.shape[1]
    v = torch.tensor(_VALUES + tuple(-x for x in _VALUES), device=codes.device)
    n = torch.stack((v[(codes & 15).long()], v[(codes >> 4).long()]), -1).reshape(M, -1, 16 if fmt == NVFP4 else 32)
    if fmt == NVFP4:
        sc = byte.contiguous().view(torch.float8_e4m3fn).float() * g
    else:
        sc = torch.where(byte > 0, (byte.int() << 23).view(torch.float32), 2.0 ** -127)
    return (n * sc[..., None]).reshape(M, K)


def _plain_mx(s):
    c = s["case"]
    K, f = c["K"], c["format"]
    nb = K // (16 if f == NVFP4 else 32)
    codes, byte = _quantize(s["x"][:, :K], f, s["gx"])
    x = _values(codes, byte, f, s["gx"])
    if c["kind"] == "quantize":
        return x.to(s["x"].dtype)
    w = _values(s["wc"], _untile(s["ws"], c["N"], nb), f, s["gw"])
    return (x @ w.t()).to(s["x"].dtype)


# ------------------------------------------------------------------------------------ plain forms: the 8-bit cache

def _scale_of(amax, kind):
    """The scale of a block whose largest value is amax: amax / 127, or the smallest power of two that holds it below 448."""
    if kind == INT8:
        return amax / torch.full((), 127.0, device=amax.device)
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-126)
    return torch.where(amax > 0, ((e + 127) << 23).view(torch.float32), 0.0)


def _codes_of(v, scale, kind):
    y = v * torch.where(scale > 0, 1.0 / scale, 0.0)
    return y.round().clamp(-127, 127).to(torch.int8) if kind == INT8 else y.clamp(-448, 448).to(torch.float8_e4m3fn)


def _held(s, a, at):
    """The cache's numbers at an index, without their scales, in 32 bits."""
    return s[a].view(torch.uint8)[at].view(s[a].dtype).float()


def _rows_of(first, cu, n, limit):
    """Sequence and position of n packed rows, where sequence i's rows cu[i] .. cu[i+1]-1 are positions first[i] on."""
    r = torch.arange(n, device=DEV)
    i = torch.searchsorted(cu[1:].long(), r, right=True).clamp(max=limit - 1)
    return i, first.long()[i] + r - cu.long()[i]


def _plain_read(s, table, n):
    P = s["case"]["page"]
    i, pos = _rows_of(s["first"], s["back"], n, table.shape[0])
    page = table[i, pos // P].long()
    return tuple((_held(s, a, (page, slice(None), pos % P)) * s[a + "s"][page][..., None]).reshape(n, s["kback"].shape[1]).to(s["kback"].dtype) for a in ("k", "v"))


def _plain_append(s):
    c = s["case"]
    P, H, D, kind, new = c["page"], c["kv_heads"], c["head_dim"], c["type"], c["new"]
    start = s["lens"].long() - new
    touched = (start + new - 1) // P - start // P + 1                    # pages that receive tokens, by sequence
    span = (new + P - 2) // P + 1
    j = start[:, None] // P + torch.arange(span, device=DEV)
    real = torch.arange(span, device=DEV)[None, :] < touched[:, None]
    page = s["table"].long().gather(1, j.clamp(max=s["table"].shape[1] - 1))[real]
    pos = (j[..., None] * P + torch.arange(P, device=DEV))[real]         # [touched pages][P] positions
    seq = torch.arange(c["batch"], device=DEV)[:, None].expand(-1, span)[real]
    fresh = (pos >= start[seq][:, None]) & (pos < start[seq][:, None] + new)
    row = (seq[:, None] * new + pos - start[seq][:, None]).clamp(0, c["batch"] * new - 1)
    kept = pos < start[seq][:, None]
    for a, src in (("k", s["knew"]), ("v", s["vnew"])):
        x = src.reshape(-1, H, D)[row].float().transpose(1, 2)           # [touched][H][P][D]
        x = torch.where(fresh[:, None, :, None], x, 0.0)
        had = kept.any(1)[:, None]
        before = torch.where(had, s[a + "s"][page], 0.0)
        scale = torch.maximum(before, _scale_of(x.abs().amax((2, 3)), kind))
        ratio = torch.where(scale > 0, before / scale, 0.0)
        again = _held(s, a, page) * ratio[..., None, None]
        again = again.round().to(torch.int8) if kind == INT8 else again.to(torch.float8_e4m3fn)
        code = torch.where(fresh[:, None, :, None], _codes_of(x, scale[..., None, None], kind).view(torch.uint8),
                           torch.where(kept[:, None, :, None], again.view(torch.uint8), s[a].view(torch.uint8)[page]))
        s[a].view(torch.uint8)[page] = code
        s[a + "s"][page] = scale
    return _plain_read(s, s["table"], s["kback"].shape[0])


def _plain_attend(s):
    c = s["case"]
    P, H, D, Hq, new, B = c["page"], c["kv_heads"], c["head_dim"], c["heads"], c["new"], c["batch"]
    G, W = Hq // H, s["table"].shape[1]
    page = s["table"].long().clamp(min=0)
    k, v = ((_held(s, a, page) * s[a + "s"][page][..., None, None]).transpose(1, 2).reshape(B, H, W * P, D) for a in ("k", "v"))
    q = s["q"].reshape(B, new, H, G, D).float().permute(0, 2, 3, 1, 4).reshape(B, H, G * new, D)
    t = torch.arange(W * P, device=DEV)
    lens = s["lens"].long()
    last = (lens[:, None] - new + torch.arange(new, device=DEV)) if c.get("causal", True) else (lens[:, None] - 1).expand(B, new)
    seen = (t[None, None, :] <= last[..., None])[:, None, None]          # [B][1][1][new][W*P]
    score = (q @ k.transpose(2, 3)).reshape(B, H, G, new, W * P) * (1.0 / math.sqrt(D))
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top)
    del score
    total = p.sum(-1, keepdim=True)
    v = torch.where((t[None, :] < lens[:, None])[:, None, :, None], v, 0.0)
    o = (p.reshape(B, H, G * new, W * P) @ v).reshape(B, H, G, new, D) / total
    lse = (top + torch.log(total)).reshape(B, H, G, new)
    return (o.permute(0, 3, 1, 2, 4).reshape(B * new, Hq * D).to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B * new, Hq))


# --------------------------------------------------------------------------------- plain forms: pages of the cache

def _plain_free(s, rows):
    t = s["table"][rows]
    used = t[t >= 0].long()
    s["refs"].index_add_(0, used, torch.full_like(used, -1, dtype=torch.int32))
    s["table"][rows] = -1
    s["lens"][rows] = 0


def _lowest_free(s, n):
    """The n lowest-numbered free pages, in order (the cases have enough of them)."""
    idle = s["refs"] == 0
    rank = torch.cumsum(idle, 0) - 1
    out = torch.empty(n + 1, dtype=torch.long, device=DEV)
    out[torch.where(idle & (rank < n), rank, n)] = torch.arange(idle.numel(), device=DEV)
    return out[:n]


def _plain_fork(s):
    P, n = s["case"]["page"], s["dst"].numel()
    src, dst = s["src"].long(), s["dst"].long()
    _plain_free(s, dst)
    lens, W = s["lens"].long()[src], s["table"].shape[1]
    full, tail = lens // P, lens % P > 0
    j = torch.arange(W, device=DEV)
    t = torch.where(j[None, :] < full[:, None], s["table"][src], -1)
    shared = t[t >= 0].long()
    order = torch.cumsum(tail, 0) - 1
    fresh = _lowest_free(s, n)[order.clamp(min=0)]
    s["refs"].index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    s["refs"].index_add_(0, fresh, tail.to(torch.int32))
    t = torch.where((j[None, :] == full[:, None]) & tail[:, None], fresh[:, None].to(torch.int32), t)
    s["table"][dst] = t
    s["lens"][dst] = s["lens"][src]
    a, b = s["table"][src, full.clamp(max=W - 1)].long()[tail], fresh[tail]
    for x in ("k", "v"):
        s[x].view(torch.uint8)[b] = s[x].view(torch.uint8)[a]
        s[x + "s"][b] = s[x + "s"][a]
    kb, vb = _plain_read(s, s["table"][dst], s["kback"].shape[0] if s["max_back"] else 0)
    return s["table"], s["lens"], s["refs"], kb, vb


def _plain_compact(s):
    c = s["case"]
    P, H, D = c["page"], c["kv_heads"], c["head_dim"]
    src, dst = s["src"].long(), s["dst"].long()
    _plain_free(s, dst)
    need = (s["keep"].long() + P - 1) // P
    W = s["table"].shape[1]
    j = torch.arange(W, device=DEV)
    mine = j[None, :] < need[:, None]
    order = (torch.cumsum(need, 0) - need)[:, None] + j[None, :]
    pages = _lowest_free(s, c["batch"] * W)[order.clamp(max=c["batch"] * W - 1)]
    t = torch.where(mine, pages, -1).to(torch.int32)
    s["refs"][pages[mine]] = 1
    s["table"][dst] = t
    s["lens"][dst] = s["keep"]
    # positions of the kept tokens, by page of the new row
    kept = torch.full((c["batch"], W * P), -1, dtype=torch.long, device=DEV)
    kept[:, : s["kept"].shape[1]] = s["kept"].long()[:, : W * P]
    kept = torch.where(torch.arange(W * P, device=DEV)[None, :] < s["keep"].long()[:, None], kept, -1).reshape(c["batch"], W, P)[mine]
    row = src[:, None].expand(-1, W)[mine]
    page = s["table"][row[:, None], kept.clamp(min=0) // P].long().clamp(min=0)
    for a in ("k", "v"):
        x = _held(s, a, (page, slice(None), kept.clamp(min=0) % P))      # [pages][P][H][D]
        x = torch.where((kept >= 0)[..., None, None], x * s[a + "s"][page][..., None], 0.0).transpose(1, 2)
        scale = _scale_of(x.abs().amax((2, 3)), c["type"])
        s[a].view(torch.uint8)[pages[mine]] = _codes_of(x, scale[..., None, None], c["type"]).view(torch.uint8)
        s[a + "s"][pages[mine]] = scale
    kb, vb = _plain_read(s, s["table"][dst], s["kback"].shape[0])
    return s["table"], s["lens"], s["refs"], kb, vb


# ------------------------------------------------------------------------------------------- the framework's calls

def _own_mx(s):
    from paper_2509_09090_b200 import binding as B
    c, x, st = s["case"], s["x"], s["stream"]
    M, K, f, dt = c["M"], c["K"], c["format"], TYPE[c["dtype"]]
    if c["kind"] == "quantize":
        B.sqap_mx4_quantize(x, dt, M, K, x.stride(0), None, f, s["gx"], s["codes"], s["scales"], st)
        B.sqap_mx4_dequantize(s["codes"], s["scales"], M, K, f, s["gx"], s["out"], s["out"].stride(0), dt, st)
        return s["out"][:, :K]
    if "work" not in s:
        s["work_bytes"] = B.sqap_mx4_workspace_bytes(M, c["N"], K, f)
        s["work"] = torch.empty(s["work_bytes"], dtype=torch.uint8, device=DEV)
    B.sqap_mx4_quantize_linear(x, dt, M, x.stride(0), None, s["gx"], s["wc"], s["ws"], s["gw"], c["N"], K, f,
                               s["out"], s["out"].stride(0), dt, s["work"], s["work_bytes"], st)
    return s["out"][:, : c["N"]]


def _own_cache(s):
    if "cache" not in s:
        from paper_2509_09090_b200 import binding as B
        c = s["case"]
        s["cache"] = B.KvCache(s["k"], s["v"], s["ks"], s["vs"], c["type"])
    return s["cache"]


def _own_read(B, s, cache, table, n):
    dt = TYPE[s["case"]["dtype"]]
    B.sqap_kv_read(cache, table, table.stride(0), n, s["first"], s["back"], s["max_back"], s["kback"], s["kback"].stride(0),
                   s["vback"], s["vback"].stride(0), dt, s["stream"])


def _own_attend(B, s, cache):
    c = s["case"]
    flags = B.SQAP_KV_CAUSAL if c.get("causal", True) else 0
    if "work" not in s:
        s["work_bytes"] = B.sqap_kv_attention_workspace_bytes(cache, c["batch"], c["new"], s["max_len"], c["heads"])
        s["work"] = torch.empty(max(1, s["work_bytes"]), dtype=torch.uint8, device=DEV)
    B.sqap_kv_attention(cache, s["table"], s["table"].stride(0), c["batch"], s["lens"], s["cu"], c["new"], s["max_len"],
                        s["q"], s["q"].stride(0), c["heads"], 1.0 / math.sqrt(c["head_dim"]), flags, s["out"], s["out"].stride(0),
                        s["lse"], TYPE[c["dtype"]], s["work"], s["work_bytes"], s["stream"])


def _own_kv(s):
    from paper_2509_09090_b200 import binding as B
    c, cache, st = s["case"], _own_cache(s), s["stream"]
    kind, table = c["kind"], s["table"]
    if kind in ("append", "step"):
        B.sqap_kv_append(cache, table, table.stride(0), c["batch"], s["lens"], s["cu"], c["new"], s["knew"], s["knew"].stride(0),
                         s["vnew"], s["vnew"].stride(0), TYPE[c["dtype"]], st)
    if kind in ("step", "attend"):
        _own_attend(B, s, cache)
    if kind == "attend":
        return s["out"], s["lse"]
    if kind in ("append", "step"):
        _own_read(B, s, cache, table, c["batch"])
        return (s["kback"], s["vback"]) if kind == "append" else (s["out"], s["lse"], s["kback"], s["vback"])
    rows, n = table.shape[0], s["dst"].numel()
    pool = (s["refs"], s["refs"].numel(), c["page"], table, table.stride(0), rows, s["lens"])
    B.sqap_kv_free(*pool, s["dst"], n, st)
    if kind == "fork":
        B.sqap_kv_fork(*pool, s["src"], s["dst"], n, s["pairs"], None, st)
        B.sqap_kv_copy_pages(cache, s["pairs"], n, st)
    else:
        B.sqap_kv_alloc(*pool, s["dst"], s["keep"], n, None, st)
        B.sqap_kv_compact(cache, table, table.stride(0), rows, s["lens"], s["src"], s["dst"], n, s["kept"], s["kept"].stride(0),
                          s["keep"], s["max_back"], st)
    if s["max_back"]:
        _own_read(B, s, cache, table[c["batch"]:], n)
    return table, s["lens"], s["refs"], s["kback"][: s["kback"].shape[0] if s["max_back"] else 0], s["vback"][: s["vback"].shape[0] if s["max_back"] else 0]


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own_mx(s) if kind in ("quantize", "linear") else _own_kv(s)
    if kind in ("quantize", "linear"):
        return _plain_mx(s)
    if kind == "append":
        return _plain_append(s)
    if kind == "attend":
        return _plain_attend(s)
    if kind == "step":
        k, v = _plain_append(s)
        return (*_plain_attend(s), k, v)
    return _plain_fork(s) if kind == "fork" else _plain_compact(s)


# ------------------------------------------------------------------------------------------------ the same in 64 bits

def _two_to(e):
    """2^e in 64 bits, for whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _floor_log2(x):
    return torch.frexp(x).exponent.long() - 1


def _round_e4m3(x):
    """Nearest number with 4 significant bits, exponents from -6 on, at most 448; ties to even."""
    step = _two_to(_floor_log2(x.abs().clamp(min=2.0 ** -30)).clamp(min=-6) - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_mx_values(x, fmt, g):
    M, K = x.shape
    b = x.double().reshape(M, -1, 16 if fmt == NVFP4 else 32)
    big = b.abs().amax(-1, keepdim=True)
    if fmt == NVFP4:
        d = _round_e4m3(big / 6 / g) * g
    else:
        d = _two_to((_floor_log2(big.clamp(min=1e-300)) - 2).clamp(-127, 127))
    y = torch.where(d > 0, b / torch.where(d > 0, d, 1.0), 0.0)
    m = y.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0)).double()
    return ((torch.round(y / step) * step).clamp(-6.0, 6.0) * d).reshape(M, K)


def _exact_mx(s):
    c = s["case"]
    K, f = c["K"], c["format"]
    x = _exact_mx_values(s["x"][:, :K], f, s["gx"].double())
    if c["kind"] == "quantize":
        return x
    N, nb = c["N"], K // (16 if f == NVFP4 else 32)
    n, k = torch.arange(N, device=DEV)[:, None], torch.arange(nb, device=DEV)[None, :]
    byte = s["ws"].reshape(-1)[(n // 128 * -(-nb // 4) + k // 4) * 512 + n % 32 * 16 + n % 128 // 32 * 4 + k % 4].long()
    if f == NVFP4:
        e, m = byte >> 3, (byte & 7).double()
        sc = torch.where(e > 0, (8 + m) * _two_to(e - 10), m * 2.0 ** -9) * s["gw"].double()
    else:
        sc = _two_to(byte - 127)
    nib = torch.stack((s["wc"] & 15, s["wc"] >> 4), -1).reshape(N, K).long()
    e, m = nib >> 1 & 3, (nib & 1).double()
    w = torch.where(e > 0, (1 + m / 2) * _two_to(e - 1), m / 2) * (1 - 2 * (nib >> 3)).double()
    return x @ (w.reshape(N, nb, -1) * sc[..., None]).reshape(N, K).t()


def _exact_held(s, a, table_row, n):
    """The first n tokens of a sequence, [n][heads][D], in 64 bits."""
    P = s["case"]["page"]
    p = torch.arange(n, device=DEV)
    page = table_row[p // P].long()
    return s[a].view(torch.uint8)[page, :, p % P].view(s[a].dtype).double() * s[a + "s"][page].double()[..., None]


def _exact_power(big):
    """The smallest power of two that holds `big` below 448; 0 for 0."""
    e = _floor_log2((big / 448).clamp(min=1e-300))
    e = torch.where(_two_to(e) * 448 < big, e + 1, e).clamp(min=-126)
    return torch.where(big > 0, _two_to(e), 0.0)


def _exact_block(x, floor, kind):
    """Values [n][heads][D] of one block -> what the cache makes of them, with scales of at least `floor` [heads]."""
    big = x.abs().amax((0, 2)) if x.shape[0] else torch.zeros_like(floor)
    if kind == INT8:
        d = torch.maximum(floor, big / 127)[None, :, None]
        return torch.where(d > 0, torch.round(x / torch.where(d > 0, d, 1.0)), 0.0) * d
    d = torch.maximum(floor, _exact_power(big))[None, :, None]
    return torch.where(d > 0, _round_e4m3(x / torch.where(d > 0, d, 1.0)), 0.0) * d


def _exact_appended(s, b, old):
    """Keys and values of sequence b after the new tokens have joined it."""
    c = s["case"]
    P, H, D, new = c["page"], c["kv_heads"], c["head_dim"], c["new"]
    got = []
    for a, src in (("k", s["knew"]), ("v", s["vnew"])):
        x = torch.cat((_exact_held(s, a, s["table"][b], old), src[b * new:(b + 1) * new].double().reshape(new, H, D)))
        for p in range(old // P, -(-(old + new) // P)):
            lo, hi = p * P, min((p + 1) * P, old + new)
            page = int(s["table"][b, p])
            had = old > lo
            floor = s[a + "s"][page].double() if had else torch.zeros(H, dtype=torch.float64, device=DEV)
            fresh = x[max(lo, old):hi]
            big = _exact_block(fresh, floor, c["type"])
            if had:
                d_old = floor
                amax = fresh.abs().amax((0, 2))
                d = torch.maximum(d_old, amax / 127 if c["type"] == INT8 else _exact_power(amax))[None, :, None]
                y = torch.where(d > 0, x[lo:old] / torch.where(d > 0, d, 1.0), 0.0)
                x[lo:old] = (torch.round(y) if c["type"] == INT8 else _round_e4m3(y)) * d
            x[max(lo, old):hi] = big
        got.append(x)
    return got


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("quantize", "linear"):
        return _exact_mx(s)
    old, H, D, P = _lengths(case), case["kv_heads"], case["head_dim"], case["page"]
    if kind in ("append", "step", "attend"):
        new, Hq = case["new"], case["heads"]
        outs, lses, ks, vs = [], [], [], []
        for b in range(case["batch"]):
            n = old[b] + new
            k, v = _exact_appended(s, b, old[b]) if kind != "attend" else (_exact_held(s, a, s["table"][b], n) for a in ("k", "v"))
            ks.append(k[old[b] // P * P:].reshape(-1, H * D))
            vs.append(v[old[b] // P * P:].reshape(-1, H * D))
            if kind == "append":
                continue
            q = s["q"][b * new:(b + 1) * new].double().reshape(new, Hq, D)
            head = torch.arange(Hq, device=DEV) // (Hq // H)
            o, l = torch.empty_like(q), torch.empty(new, Hq, dtype=torch.float64, device=DEV)
            for h0 in range(0, Hq, 8):
                h = head[h0:h0 + 8]
                sc = torch.einsum("qhd,thd->hqt", q[:, h0:h0 + 8], k[:, h]) / math.sqrt(D)
                if case.get("causal", True):
                    late = torch.arange(n, device=DEV)[None, :] > old[b] + torch.arange(new, device=DEV)[:, None]
                    sc = sc.masked_fill(late, -math.inf)
                l[:, h0:h0 + 8] = torch.logsumexp(sc, -1).t()
                o[:, h0:h0 + 8] = torch.einsum("hqt,thd->qhd", torch.softmax(sc, -1), v[:, h])
            outs.append(o.reshape(new, Hq * D))
            lses.append(l)
        if kind == "append":
            return torch.cat(ks), torch.cat(vs)
        r = (torch.cat(outs), torch.cat(lses))
        return r if kind == "attend" else (*r, torch.cat(ks), torch.cat(vs))
    got = {"k": [], "v": []}
    for a in ("k", "v"):
        for b in range(case["batch"]):
            x = _exact_held(s, a, s["table"][b], old[b])
            if kind == "fork":
                got[a] += [x[old[b] // P * P:].reshape(-1, H * D)] * case["copies"]
            else:
                x = x[s["kept"][b, : min(case["keep"], old[b])].long()]
                zero = torch.zeros(H, dtype=torch.float64, device=DEV)
                got[a] += [_exact_block(x[p:p + P], zero, case["type"]).reshape(-1, H * D) for p in range(0, x.shape[0], P)]
    return None, None, None, torch.cat(got["k"]), torch.cat(got["v"])
