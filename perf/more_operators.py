"""Timed cases of the operators around the paged key/value cache: rotary positions, attention over a sliding window, attention of
sequences that share a prefix, attention that accumulates the weights of the tokens, and eviction by those weights.

Each case is one call that a user's program makes. `run` computes it in elementary torch operations where `own` is false and
through the framework's binding where it is true; `exact` states the same result in 64 bits.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
INT8, E4M3 = 0, 1            # what the cache holds
F16 = {"fp16": torch.float16, "bf16": torch.bfloat16}
TYPE = {"fp16": 0, "bf16": 1}


# --------------------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # queries and keys of one new token of 16 observations, positions far into an episode
        dict(name="rotary 16 rows", kind="rotary", dtype="fp16", rows=16, heads=64, head_dim=128, rot=128, axes=1, neighbours=False,
             far=1000000, pad=4096),
        # the prompts of 16 observations: text and a grid of visual tokens with time, row and column
        dict(name="rotary 4608 rows", kind="rotary", dtype="bf16", rows=4608, heads=64, head_dim=128, rot=128, axes=3, neighbours=False,
             far=0, pad=4096),
        # one decode step of 16 observations that look at their instruction's start and the last 128 tokens
        dict(name="window step 16x290", kind="window", type=INT8, dtype="fp16", batch=16, heads=32, kv_heads=32, head_dim=128, page=64,
             new=1, old=290, ragged=3, window=128, sinks=4),
        # a decode step of long, uneven episodes
        dict(name="window step 32x16384", kind="window", type=E4M3, dtype="bf16", batch=32, heads=32, kv_heads=8, head_dim=128, page=64,
             new=1, old=16384, ragged=5, window=2048, sinks=16),
        # long prompts behind a cached prefix, an odd length and an odd window
        dict(name="window prompt 2x4099+1000", kind="window", type=E4M3, dtype="bf16", batch=2, heads=32, kv_heads=8, head_dim=128,
             page=32, new=4099, old=1000, ragged=0, window=1023, sinks=4),
        # eight action candidates of each of 16 observations, a few tokens into their answers
        dict(name="shared 16x8 256+40", kind="shared", type=INT8, dtype="fp16", groups=16, copies=8, heads=32, kv_heads=32, head_dim=128,
             page=64, prefix=256, own=40, new=1, ragged=0),
        # 64 requests behind one long instruction
        dict(name="shared 1x64 16384+300", kind="shared", type=E4M3, dtype="bf16", groups=1, copies=64, heads=32, kv_heads=8, head_dim=128,
             page=64, prefix=16384, own=300, new=1, ragged=7),
        # a decode step of 16 observations whose cache is to be evicted from
        dict(name="mass step 16x290", kind="mass", type=INT8, dtype="fp16", batch=16, heads=32, kv_heads=32, head_dim=128, page=64,
             new=1, old=290, ragged=3, last=1),
        # the same over long, uneven histories with shared key/value heads
        dict(name="mass step 32x16384", kind="mass", type=E4M3, dtype="bf16", batch=32, heads=32, kv_heads=8, head_dim=128, page=64,
             new=1, old=16384, ragged=5, last=1),
        # the prompts of 16 observations; their last 32 tokens say what is looked at
        dict(name="mass prompt 16x288", kind="mass", type=INT8, dtype="fp16", batch=16, heads=32, kv_heads=32, head_dim=128, page=64,
             new=288, old=0, ragged=0, last=32),
        # the observations' caches are brought down to 160 tokens
        dict(name="evict 16x288 to 160", kind="evict", n=16, old=288, ragged=0, keep=160, first=1, recent=32),
        # long episodes are brought down to a quarter
        dict(name="evict 32x16384 to 4096", kind="evict", n=32, old=16384, ragged=5, keep=4096, first=4, recent=256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["fp16", "bf16"])
    kind = rng.choice(["rotary", "window", "window", "shared", "shared", "mass", "mass", "evict"])
    if kind == "rotary":
        D, neighbours = rng.choice([64, 72, 80, 128, 128, 256]), rng.random() < 0.4
        heads = rng.choice([1, 3, 8, 12, 40, 64])
        return dict(kind=kind, dtype=dtype, rows=max(1, min(_log(rng, 1, 20000), 4608 * 64 * 128 // (heads * D))), heads=heads, head_dim=D,
                    rot=rng.choice([D, D, D // 16 * 8]), axes=rng.choice([1, 2, 3]), neighbours=neighbours,
                    far=rng.choice([0, 0, 30000, 1000000]), pad=rng.choice([0, 8, 1024]))
    if kind == "evict":
        n = _log(rng, 1, 64)
        old = min(_log(rng, 1, 40000), 32 * 16384 // n)
        return dict(kind=kind, n=n, old=old, ragged=rng.choice([0, rng.randrange(1, 1000)]), keep=rng.randint(1, old),
                    first=rng.choice([0, 1, 4, 64]), recent=rng.choice([0, 1, 32, 500]))
    c = dict(kind=kind, type=rng.choice([INT8, E4M3]), dtype=dtype, page=rng.choice([16, 32, 64, 128]),
             head_dim=rng.choice([64, 128, 128, 256]), kv_heads=rng.choice([1, 2, 4, 8, 32]), ragged=rng.randrange(1000))
    c["heads"] = c["kv_heads"] * rng.choice([1, 1, 2, 4, 7, 8])
    width, D = c["kv_heads"] * c["head_dim"], c["head_dim"]
    top = 31 * 7168 * 1024                                     # elements of the keys of a whole cache
    if kind == "shared":
        c["groups"], c["copies"], c["new"] = _log(rng, 1, 16), _log(rng, 1, 64), rng.choice([1, 1, 1, 2, 5])
        c["own"] = _log(rng, 1, 600)
        c["prefix"] = rng.choice([0, _log(rng, 1, 16384), _log(rng, 64, 16384)])
        c["copies"] = max(1, min(c["copies"], top // (c["groups"] * width * (c["prefix"] + c["own"]))))
        c["prefix"] = min(c["prefix"], top // (c["groups"] * c["copies"] * width))
        return c
    c["batch"] = _log(rng, 1, 32)
    c["new"] = rng.choice([1, 1, 1, 3, _log(rng, 8, 2500)])
    c["old"] = rng.choice([0, _log(rng, 1, 16000)])
    most = (2 if kind == "window" else 1.1) * 4099 * 1000 * 32 * 128     # query row, key and element products of a call
    c["new"] = max(1, min(c["new"], int(most) // (c["batch"] * c["heads"] * D * 1200)))
    c["old"] = max(0, min(c["old"], int(most) // (c["batch"] * c["heads"] * D * c["new"]), top // (c["batch"] * width)))
    if kind == "window":
        c["window"], c["sinks"] = _log(rng, 1, 4096), rng.choice([0, 1, 4, 100])
    else:
        c["last"] = rng.choice([c["new"], min(c["new"], 32), 1])
    return c


def _spread(seed, n, old):
    """Lengths of n histories: `old` for all of them, or spread below it."""
    if not seed:
        return [old] * n
    r = random.Random(seed)
    return [r.randint(old // 16, old) for _ in range(n)]


def _members(case):
    """Sequences of each group."""
    if not case["ragged"]:
        return [case["copies"]] * case["groups"]
    r = random.Random(case["ragged"])
    return [case["copies"]] + [r.randint(1, case["copies"]) for _ in range(case["groups"] - 1)]


def _owned(case):
    """Tokens of each sequence behind the shared ones, without the new."""
    return _spread(case["ragged"], sum(_members(case)), case["own"])


def work(case):
    kind = case["kind"]
    if kind == "rotary":
        n, r = case["rows"] * case["heads"], case["rows"] * case["axes"]
        return {"bytes": 4.0 * n * case["head_dim"] + 4.0 * r, "flops": 3.0 * n * case["rot"]}
    if kind == "evict":
        lens = _spread(case["ragged"], case["n"], case["old"])
        held = sum(min(x, case["keep"]) for x in lens)
        return {"bytes": 4.0 * sum(lens) + 8.0 * held + 16.0 * len(lens), "flops": float(sum(lens))}
    D, H, Hq, new = case["head_dim"], case["kv_heads"], case["heads"], case["new"]
    if kind == "shared":
        own_tokens = [x + new for x in _owned(case)]
        n = len(own_tokens)
        tokens = case["prefix"] * case["groups"] + sum(own_tokens)
        pairs = sum(new * (case["prefix"] + x - new) + new * (new + 1) // 2 for x in own_tokens)
        return {"bytes": 2.0 * tokens * H * D + 4.0 * n * new * Hq * D + 4.0 * n * new * Hq, "flops": 4.0 * pairs * Hq * D}
    old = _spread(case["ragged"], case["batch"], case["old"])
    rows = case["batch"] * new
    b = 4.0 * rows * Hq * D + 4.0 * rows * Hq
    if kind == "window":
        W, S = case["window"], case["sinks"]
        tokens = sum(x + new - max(0, min(x + 1 - W, x + new)) + min(S, max(0, x + 1 - W)) for x in old)
        pairs = sum(min(p + 1, W) + min(S, max(0, p + 1 - W)) for x in old for p in range(x, x + new))
        return {"bytes": b + 2.0 * tokens * H * D, "flops": 4.0 * pairs * Hq * D}
    tokens = sum(old) + rows
    pairs = sum(new * x + new * (new + 1) // 2 for x in old)
    again = 0 if new == 1 else sum(case["last"] * (x + new) for x in old)
    return {"bytes": b + 2.0 * tokens * H * D + 8.0 * tokens, "flops": (4.0 * pairs + 2.0 * again) * Hq * D}


# ------------------------------------------------------------------------------------------------------- the inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


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


def _axis_of(case):
    """The axis of each pair: runs of pairs for time, row and column, or one of each in turn."""
    half, axes = case["rot"] // 2, case["axes"]
    if case["neighbours"]:
        return [i % axes for i in range(half)]
    return [min(axes - 1, i * axes // half) for i in range(half)]


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    s = {"case": case, "stream": torch.cuda.current_stream().cuda_stream}
    if kind == "rotary":
        rows, H, D = case["rows"], case["heads"], case["head_dim"]
        # columns of a wider row, as a fused projection leaves them
        s["x"] = torch.randn(rows, H * D + case["pad"], generator=g, device=DEV).to(F16[case["dtype"]])
        pos = torch.arange(rows, device=DEV) % 288
        time = torch.where((pos > 0) & (pos <= 256), 1, pos)
        grid = torch.where((pos > 0) & (pos <= 256), (pos - 1) // 16 + 1, pos), torch.where((pos > 0) & (pos <= 256), (pos - 1) % 16 + 1, pos)
        far = torch.randint(0, case["far"] + 1, (rows,), generator=g, device=DEV)
        s["pos"] = torch.stack([(a + far).to(torch.int32) for a in (time, *grid)][: case["axes"]]).contiguous()
        s["axis_of"] = bytes(_axis_of(case))
        s["freq"] = torch.tensor([1e4 ** (-2 * i / case["rot"]) for i in range(case["rot"] // 2)], dtype=torch.float32, device=DEV)
        s["out"] = torch.empty(rows, H * D, dtype=F16[case["dtype"]], device=DEV)
        return s
    if kind == "evict":
        lens = _spread(case["ragged"], case["n"], case["old"])
        n, width = len(lens), (case["old"] + 7) // 8 * 8
        # weights that a few tokens share among them; many that were never looked at, many alike
        m = torch.exp(3 * torch.randn(2 * n, width, generator=g, device=DEV))
        u = torch.rand(2 * n, width, generator=g, device=DEV)
        s["mass"] = torch.where(u < 0.1, 0.0, torch.where(u < 0.3, (4 * m).round() / 4, m)).contiguous()
        s["lens"] = _ints(lens + [0] * n)
        s["src"], s["dst"] = _ints(list(range(n))), _ints(list(range(n, 2 * n)))
        s["keep"] = _ints([case["keep"]] * n)
        s["kept"] = torch.empty(n, case["keep"], dtype=torch.int32, device=DEV)
        s["n_kept"] = torch.empty(n, dtype=torch.int32, device=DEV)
        return s

    dt, D, H, P, Hq, new = F16[case["dtype"]], case["head_dim"], case["kv_heads"], case["page"], case["heads"], case["new"]
    if kind == "shared":
        members, owned, pre = _members(case), _owned(case), case["prefix"]
        B = len(owned)
        lens = [pre + x + new for x in owned]
        first = [sum(members[:i]) for i in range(len(members) + 1)]
        full = pre // P                                       # the pages that lie whole in the prefix are one group's; the rest each one's
        need = [-(-n // P) - full for n in lens]
        pages = full * len(members) + sum(need) + 5
        order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32).cpu().numpy()
        t, at = np.full((B, max(-(-n // P) for n in lens)), -1, np.int32), 0
        for i, m in enumerate(members):
            t[first[i]:first[i] + m, :full] = order[at:at + full]
            at += full
        for b, n in enumerate(need):
            t[b, full:full + n] = order[at:at + n]
            at += n
        s.update(_cache(pages, case, g))
        s["table"] = torch.from_numpy(t).to(DEV)
        if pre % P:                                           # the copies of the prefix's unfinished page hold the same tokens
            for i, m in enumerate(members):
                a, rest = int(t[first[i], full]), torch.from_numpy(t[first[i] + 1:first[i] + m, full].astype(np.int64)).to(DEV)
                for x in ("k", "v"):
                    s[x].view(torch.uint8)[rest, :, : pre % P] = s[x].view(torch.uint8)[a, :, : pre % P].clone()
                    s[x + "s"][rest] = s[x + "s"][a].clone()
        s["cu_group"], s["groups"], s["max_group"] = _ints(first), len(members), max(members)
        s["prefix"] = _ints([pre] * len(members))
    else:
        B = case["batch"]
        lens = [x + new for x in _spread(case["ragged"], B, case["old"])]
        need = [-(-n // P) for n in lens]
        pages = sum(need) + 5
        order = torch.randperm(pages, generator=g, device=DEV)[: sum(need)].to(torch.int32)
        s["table"] = torch.full((B, max(need)), -1, dtype=torch.int32, device=DEV)
        s["table"][torch.arange(max(need), device=DEV)[None, :] < _ints(need)[:, None]] = order
        s.update(_cache(pages, case, g))
    s["lens"], s["max_len"] = _ints(lens), max(lens)
    s["cu"] = _ints([new * i for i in range(B + 1)])
    s["q"] = torch.randn(B * new, (Hq + 2 * H) * D, generator=g, device=DEV).to(dt)[:, : Hq * D]
    s["out"] = torch.empty(B * new, Hq * D, dtype=dt, device=DEV)
    s["lse"] = torch.empty(B * new, Hq, device=DEV)
    if kind == "mass":
        width = (max(lens) + 7) // 8 * 8
        s["past"] = torch.rand(B, width, generator=g, device=DEV)
        s["mass"] = torch.zeros(B, width, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------------- plain forms

def _plain_rotary(s):
    c = s["case"]
    rows, H, D, rot = c["rows"], c["heads"], c["head_dim"], c["rot"]
    x = s["x"][:, : H * D].reshape(rows, H, D).float()
    axis = torch.tensor(list(s["axis_of"]), device=DEV)
    angle = s["pos"].double()[axis].t() * s["freq"].double()           # [rows][pairs]; far positions lose their angle in 32 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    y = x.clone()
    if c["neighbours"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        y[..., : rot // 2], y[..., rot // 2: rot] = a * cos - b * sin, b * cos + a * sin
    return y.reshape(rows, H * D).to(s["x"].dtype)


def _plain_attend(s, seen):
    """Attention over all places of the table's pages, of which query i of sequence b sees those where seen(position of the query
    [B][new][1], place [1][1][W * P]): rows, their log-sum-exp, the weights."""
    c = s["case"]
    P, H, D, Hq, new = c["page"], c["kv_heads"], c["head_dim"], c["heads"], c["new"]
    B, W, G = s["table"].shape[0], s["table"].shape[1], Hq // H
    page = s["table"].long().clamp(min=0)
    k, v = ((s[a].view(torch.uint8)[page].view(s[a].dtype).float() * s[a + "s"][page][..., None, None]).transpose(1, 2).reshape(B, H, W * P, D)
            for a in ("k", "v"))
    q = s["q"].reshape(B, new, H, G, D).float().permute(0, 2, 3, 1, 4).reshape(B, H, G * new, D)
    t = torch.arange(W * P, device=DEV)[None, None, :]
    lens = s["lens"].long()
    at = (lens[:, None] - new + torch.arange(new, device=DEV))[..., None]
    may = (seen(at, t) & (t <= at))[:, None, None]                       # [B][1][1][new][W * P]
    score = (q @ k.transpose(2, 3)).reshape(B, H, G, new, W * P) * (1.0 / math.sqrt(D))
    score = torch.where(may, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top)
    del score
    total = p.sum(-1, keepdim=True)
    v = torch.where((t[0] < lens[:, None])[:, None, :, None], v, 0.0)
    o = (p.reshape(B, H, G * new, W * P) @ v).reshape(B, H, G, new, D) / total
    lse = (top + torch.log(total)).reshape(B, H, G, new)
    return o.permute(0, 3, 1, 2, 4).reshape(B * new, Hq * D).to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B * new, Hq), p, total


def _plain_mass(s):
    c = s["case"]
    out, lse, p, total = _plain_attend(s, lambda at, t: t >= 0)
    w = (p[..., c["new"] - c["last"]:, :] / total[..., c["new"] - c["last"]:, :]).sum((1, 2, 3))     # [B][places]
    n = s["mass"].shape[1]
    w = torch.nn.functional.pad(w, (0, max(0, n - w.shape[1])))[:, :n]
    t, lens = torch.arange(n, device=DEV)[None, :], s["lens"].long()[:, None]
    w = w + torch.where(t < lens - c["new"], s["past"], 0.0)
    return out, lse, torch.where(t < lens, w, s["mass"])


def _plain_evict(s):
    c = s["case"]
    n, width = s["kept"].shape[0], s["mass"].shape[1]
    m = s["mass"][s["src"].long()]
    t, lens = torch.arange(width, device=DEV)[None, :], s["lens"].long()[s["src"].long()][:, None]
    keep = torch.minimum(s["keep"].long()[:, None], lens)
    recent = keep.clamp(max=c["recent"])
    first = torch.minimum((keep - recent).clamp(max=c["first"]), lens - recent)
    held = ((t >= lens - recent) & (t < lens)) | (t < first)
    key = torch.where(held, math.inf, torch.where(t < lens, m, -math.inf))
    rank = key.argsort(dim=1, descending=True, stable=True).argsort(dim=1)       # equal weights in the order of their tokens
    stay = (rank < keep) & (t < lens)
    pos = torch.where(stay, t, width).sort(1).values[:, : s["kept"].shape[1]]
    there = pos < width
    kept = torch.where(there, pos, -1).to(torch.int32)
    got = s["mass"].clone()
    k = kept.shape[1]
    got[s["dst"].long(), :k] = torch.where(there, m.gather(1, pos.clamp(max=width - 1)), got[s["dst"].long(), :k])
    return kept, keep[:, 0].to(torch.int32), got


# ------------------------------------------------------------------------------------------- the framework's calls

def _own(s):
    from paper_2509_09090_b200 import binding as B
    c, kind, st = s["case"], s["case"]["kind"], s["stream"]
    if kind == "rotary":
        x, out = s["x"], s["out"]
        B.sqap_rotary(x, x.stride(0), c["rows"], c["heads"], c["head_dim"], c["rot"], s["pos"], s["pos"].stride(0), c["axes"], s["axis_of"],
                      s["freq"], B.SQAP_ROTARY_NEIGHBOURS if c["neighbours"] else 0, out, out.stride(0), TYPE[c["dtype"]], st)
        return out
    if kind == "evict":
        m, kept = s["mass"], s["kept"]
        B.sqap_kv_evict(m, m.stride(0), m.shape[0], s["lens"], s["src"], s["dst"], kept.shape[0], s["keep"], c["first"], c["recent"],
                        c["old"], kept, kept.stride(0), s["n_kept"], st)
        return kept, s["n_kept"], m
    if "cache" not in s:
        s["cache"] = B.KvCache(s["k"], s["v"], s["ks"], s["vs"], c["type"])
        n, new, top, heads = s["table"].shape[0], c["new"], s["max_len"], c["heads"]
        if kind == "window":
            size = B.sqap_kv_attention_window_workspace_bytes(s["cache"], n, new, top, heads, c["window"], c["sinks"])
        elif kind == "shared":
            size = B.sqap_kv_attention_shared_workspace_bytes(s["cache"], n, new, top, s["groups"], s["max_group"], c["prefix"], heads)
        else:
            size = B.sqap_kv_attention_mass_workspace_bytes(s["cache"], n, new, top, heads, c["last"])
        s["work"], s["work_bytes"] = torch.empty(max(1, size), dtype=torch.uint8, device=DEV), size
    history = (s["cache"], s["table"], s["table"].stride(0), s["table"].shape[0], s["lens"], s["cu"], c["new"], s["max_len"])
    q = (s["q"], s["q"].stride(0), c["heads"], 1.0 / math.sqrt(c["head_dim"]))
    out = (s["out"], s["out"].stride(0), s["lse"])
    rest = (TYPE[c["dtype"]], s["work"], s["work_bytes"], st)
    if kind == "window":
        B.sqap_kv_attention_window(*history, *q, c["window"], c["sinks"], *out, *rest)
        return s["out"], s["lse"]
    if kind == "shared":
        B.sqap_kv_attention_shared(*history, s["cu_group"], s["groups"], s["max_group"], s["prefix"], c["prefix"], *q, B.SQAP_KV_CAUSAL,
                                   *out, *rest)
        return s["out"], s["lse"]
    B.sqap_kv_attention_mass(*history, *q, B.SQAP_KV_CAUSAL, c["last"], *out, s["past"], s["mass"], s["mass"].stride(0), *rest)
    return s["out"], s["lse"], s["mass"]


def run(s):
    if own:
        return _own(s)
    c = s["case"]
    kind = c["kind"]
    if kind == "rotary":
        return _plain_rotary(s)
    if kind == "evict":
        return _plain_evict(s)
    if kind == "mass":
        return _plain_mass(s)
    if kind == "window":
        return _plain_attend(s, lambda at, t: (t > at - c["window"]) | (t < c["sinks"]))[:2]
    return _plain_attend(s, lambda at, t: t >= 0)[:2]


# ------------------------------------------------------------------------------------------------ the same in 64 bits

def _exact_rotary(s):
    """The pair as a complex number, turned by e^(i angle)."""
    c = s["case"]
    rows, H, D, rot = c["rows"], c["heads"], c["head_dim"], c["rot"]
    x = s["x"][:, : H * D].double().reshape(rows, H, D)
    i = np.arange(rot // 2)
    lo, hi = (2 * i, 2 * i + 1) if c["neighbours"] else (i, i + rot // 2)
    angle = torch.stack([s["pos"][a].double() * f for a, f in zip(s["axis_of"], s["freq"].double())], 1)
    z = torch.complex(x[..., lo], x[..., hi]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    x[..., lo], x[..., hi] = z.real, z.imag
    return x.reshape(rows, H * D)


def _exact_attend(s, may):
    """One sequence after another; may(position, tokens) says which tokens a query sees."""
    c = s["case"]
    P, H, D, Hq, new = c["page"], c["kv_heads"], c["head_dim"], c["heads"], c["new"]
    head = torch.arange(Hq, device=DEV) // (Hq // H)
    outs, lses, weights = [], [], []
    for b in range(s["table"].shape[0]):
        n = int(s["lens"][b])
        at = torch.arange(n, device=DEV)
        page = s["table"][b][at // P].long()
        k, v = (s[a].view(torch.uint8)[page, :, at % P].view(s[a].dtype).double() * s[a + "s"][page].double()[..., None] for a in ("k", "v"))
        q = s["q"][b * new:(b + 1) * new].double().reshape(new, Hq, D)
        place = n - new + torch.arange(new, device=DEV)[:, None]
        hide = (at[None, :] > place) | ~may(place, at[None, :])
        o, lse, w = torch.empty_like(q), torch.empty(new, Hq, dtype=torch.float64, device=DEV), 0.0
        for h0 in range(0, Hq, 8):
            h = head[h0:h0 + 8]
            sc = torch.einsum("qhd,thd->hqt", q[:, h0:h0 + 8], k[:, h]) / math.sqrt(D)
            sc = sc.masked_fill(hide, -math.inf)
            p = torch.softmax(sc, -1)
            lse[:, h0:h0 + 8] = torch.logsumexp(sc, -1).t()
            o[:, h0:h0 + 8] = torch.einsum("hqt,thd->qhd", p, v[:, h])
            if c["kind"] == "mass":
                w = w + p[:, new - c["last"]:].sum((0, 1))
        outs.append(o.reshape(new, Hq * D))
        lses.append(lse)
        weights.append(w)
    return torch.cat(outs), torch.cat(lses), weights


def _exact_evict(s):
    c = s["case"]
    mass, lens = s["mass"].double().cpu().numpy(), s["lens"].tolist()
    kept, count, got = np.full(tuple(s["kept"].shape), -1, np.int32), [], mass.copy()
    for i, (a, b) in enumerate(zip(s["src"].tolist(), s["dst"].tolist())):
        n = lens[a]
        order = list(range(n - 1, max(n - c["recent"], 0) - 1, -1))                    # the last ones, the first ones, the heaviest
        order += [t for t in range(min(c["first"], n)) if t < n - c["recent"]]
        taken = np.zeros(n, bool)
        taken[order] = True
        rest = np.flatnonzero(~taken)
        order = np.concatenate([np.array(order, np.int64), rest[np.lexsort((rest, -mass[a, rest]))]])
        stay = np.sort(order[: min(c["keep"], n)])
        kept[i, : len(stay)], got[b, : len(stay)] = stay, mass[a, stay]
        count.append(len(stay))
    return torch.from_numpy(kept), torch.tensor(count, dtype=torch.int32), torch.from_numpy(got)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        return _exact_rotary(s)
    if kind == "evict":
        return _exact_evict(s)
    if kind == "window":
        return _exact_attend(s, lambda at, t: (at - t < case["window"]) | (t < case["sinks"]))[:2]
    out, lse, weights = _exact_attend(s, lambda at, t: t >= 0)
    if kind == "shared":
        return out, lse
    mass = s["mass"].double()
    for b, w in enumerate(weights):
        n = w.shape[0]
        mass[b, :n] = w
        mass[b, : n - case["new"]] += s["past"][b, : n - case["new"]].double()
    return out, lse, mass
