"""The paged 8-bit key/value cache (append, read back, attention, pages) against plain statements in 64 bits.

Codes and scales after an append or a compaction: equal (the reference makes the definition's fp32 roundings). Attention: with
p the softmax, per output element
  rounding of the output          |ref| eps / 2
  weights rounded to fp16         2^-11 sum p |v|     and 2^-25 of the largest weight where they are subnormal
  errors of the exponent          2 d sum p |v|,  d = 2^-19 (1 + max_t sum_d |q k| scale): fp32 sums of up to 256 products and the
                                  approximate exponential and logarithm (2^-22 each, relative to exponents of a few hundred at most)
and d for the log-sum-exp, plus its own rounding.
"""
import math

import numpy as np
import pytest

import lowbit_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B

DEV = "cuda:0"
T = {"fp16": torch.float16, "bf16": torch.bfloat16}
CODE = {"fp16": 0, "bf16": 1}


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def ints(a):
    return dev(np.asarray(a, np.int32))


class Setup:
    """A cache with random contents (numpy mirror: raw bytes, scales, table) and its device tensors."""

    def __init__(self, lens, H, D, P, kind, seed=0, spare=3, rows=None, spread=0.0, nan_behind=False):
        g = self.g = np.random.default_rng(seed)
        self.H, self.D, self.P, self.kind, self.lens = H, D, P, kind, list(lens)
        need = [-(-n // P) for n in lens]
        self.pages = sum(need) + spare
        self.width = max(need + [1]) + 1
        order = g.permutation(self.pages)[:sum(need)]
        rows = rows or len(lens)
        self.table = np.full((rows, self.width), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (self.pages, H, P, D)
        self.raw, self.scale = {}, {}
        for a in "kv":
            if kind == R.INT8:
                self.raw[a] = np.clip(np.rint(g.standard_normal(shape) * 40), -127, 127).astype(np.int8).view(np.uint8)
                self.scale[a] = ((0.7 + 0.6 * g.random(shape[:2])) / 40 * 2.0 ** (spread * g.standard_normal(shape[:2]))).astype(np.float32)
            else:
                # magnitudes over e4m3's range, subnormals among them
                x = g.integers(0, 0x7F, shape).astype(np.uint8) if spread else g.integers(0x28, 0x70, shape).astype(np.uint8)
                self.raw[a] = x | (g.integers(0, 2, shape) << 7).astype(np.uint8)
                self.scale[a] = (2.0 ** (g.integers(-8, -5, shape[:2]) + np.rint(spread * g.standard_normal(shape[:2])))).astype(np.float32)
        if nan_behind:      # places and pages that hold no token: not-a-numbers in e4m3, and in the scales of unused pages
            used = np.zeros((self.pages, P), bool)
            for b, n in enumerate(lens):
                for t in range(n):
                    used[self.table[b, t // P], t % P] = True
            for a in "kv":
                if kind == R.E4M3:
                    self.raw[a][np.broadcast_to(~used[:, None, :, None], shape)] = 0x7F
                self.scale[a][~used.any(1)] = np.nan
        self.to_device()

    def to_device(self):
        dt = torch.int8 if self.kind == R.INT8 else torch.float8_e4m3fn
        self.d = {a: dev(self.raw[a]).view(dt) for a in "kv"}
        self.ds = {a: dev(self.scale[a]) for a in "kv"}
        self.dtable = ints(self.table)
        self.cache = B.KvCache(self.d["k"], self.d["v"], self.ds["k"], self.ds["v"], self.kind)

    def codes(self, a):
        return R.kv_values(self.raw[a], self.kind)

    def device_codes(self, a):
        return R.kv_values(self.d[a].view(torch.uint8).cpu().numpy(), self.kind)


# ------------------------------------------------------------------------------------------------------- append, read

@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("dtype,H,D,P,old,new,gain", [
    ("fp16", 2, 64, 16, [0, 5, 16, 31], [1, 1, 1, 1], 1.0),
    ("bf16", 1, 128, 64, [0, 63, 64, 100], [1, 2, 0, 65], 5.0),
    ("fp16", 3, 256, 32, [0, 1], [97, 31], 0.01),
    ("bf16", 32, 128, 64, [0, 288], [288, 1], 3.0),
    ("fp16", 2, 64, 128, [0, 130, 7], [128, 127, 250], 1.5)])
def test_append(kind, dtype, H, D, P, old, new, gain):
    lens = [a + b for a, b in zip(old, new)]
    s = Setup(lens, H, D, P, kind, seed=sum(lens))
    T_rows = sum(new)
    x = s.g.standard_normal((T_rows + 2, (2 * H + 1) * D)) * gain
    if T_rows > 3:
        x[1, :2 * H * D] = 0
    x = dev(x, T[dtype])
    cu = np.concatenate([[0], np.cumsum(new)])
    B.sqap_kv_append(s.cache, s.dtable, s.width, len(old), ints(lens), ints(cu), max(new), x, x.stride(0), x[:, H * D:], x.stride(0), CODE[dtype])
    torch.cuda.synchronize()
    xn = x.float().cpu().numpy()
    for a, c0 in (("k", 0), ("v", H * D)):
        codes, scale = s.codes(a), s.scale[a].copy()
        R.kv_append(codes, scale, s.table, lens, cu, xn[:, c0:c0 + H * D].reshape(-1, H, D), kind, P)
        assert np.array_equal(s.ds[a].cpu().numpy(), scale)
        assert np.array_equal(s.device_codes(a), codes)


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
def test_append_token_by_token_then_read(kind):
    """A sequence grown one token at a time stays within one rounding per growth of a page's scale of what went in."""
    H, D, P, n = 2, 64, 16, 37
    s = Setup([n], H, D, P, kind, 1)
    x = s.g.standard_normal((n, H * D)) * np.exp(s.g.standard_normal((n, 1)))
    xd = dev(x, torch.float16)
    codes, scale = {a: s.codes(a) for a in "kv"}, {a: s.scale[a].copy() for a in "kv"}
    for i in range(n):
        B.sqap_kv_append(s.cache, s.dtable, s.width, 1, ints([i + 1]), ints([0, 1]), 1, xd[i:], H * D, xd[i:], H * D, 0)
        for a in "kv":
            R.kv_append(codes[a], scale[a], s.table, [i + 1], [0, 1], xd[i:i + 1].float().cpu().numpy().reshape(1, H, D), kind, P)
    k, v = (torch.full((n + 1, H * D + 8), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.sqap_kv_read(s.cache, s.dtable, s.width, 1, None, ints([0, n]), n, k, k.stride(0), v, v.stride(0), 1)
    torch.cuda.synchronize()
    for a, got in (("k", k), ("v", v)):
        assert np.array_equal(s.device_codes(a), codes[a]) and np.array_equal(s.ds[a].cpu().numpy(), scale[a])
        ref, _ = R.kv_tokens(codes[a], scale[a], s.table[0], n, P)
        g = got.double().cpu().numpy()
        assert (g[n] == 9).all() and (g[:, H * D:] == 9).all()
        assert (np.abs(g[:n, :H * D] - ref.reshape(n, -1)) <= np.abs(ref.reshape(n, -1)) * (2.0 ** -8 + 2.0 ** -23)).all()


def test_append_drops_what_has_no_page_and_positions_before_zero():
    for kind in (R.INT8, R.E4M3):
        s = Setup([40, 20, 8], 2, 64, 16, kind, 5)
        s.table[0, 1] = -1
        s.table[1, 0] = s.pages
        s.table[0, 3:] = 1 << 30
        s.to_device()
        new = [40, 5, 12]                       # the third has more rows than tokens: the first four are dropped
        cu = np.concatenate([[0], np.cumsum(new)])
        x = dev(s.g.standard_normal((sum(new), 128)), torch.float16)
        B.sqap_kv_append(s.cache, s.dtable, s.width, 3, ints(s.lens), ints(cu), 40, x, 128, x, 128, 0)
        torch.cuda.synchronize()
        for a in "kv":
            codes, scale = s.codes(a), s.scale[a].copy()
            R.kv_append(codes, scale, s.table, s.lens, cu, x.float().cpu().numpy().reshape(-1, 2, 64), kind, 16)
            assert np.array_equal(s.device_codes(a), codes) and np.array_equal(s.ds[a].cpu().numpy(), scale)
        # read: a missing page is zero, one output may be left out
        k = torch.full((40, 128), 9.0, dtype=torch.float16, device=DEV)
        B.sqap_kv_read(s.cache, s.dtable, s.width, 1, ints([8]), ints([0, 32]), 32, k, 128, None, 0, 0)
        torch.cuda.synchronize()
        g = k.double().cpu().numpy()
        assert (g[8:24] == 0).all() and (g[32:] == 9).all() and (g[:8] != 0).any()


# ------------------------------------------------------------------------------------------------------------ attention

def run_attention(s, q, new, heads, causal, dtype, max_len=None, scale=None, lens=None):
    """Returns out and lse as float64, with canaries around them checked. q: device rows (maybe a slice)."""
    lens = s.lens if lens is None else lens
    cu = np.concatenate([[2], 2 + np.cumsum(new)])       # two rows in front belong to nobody
    n = int(cu[-1])
    max_len = max(lens + [0]) if max_len is None else max_len
    out = torch.full((n + 2, heads * s.D + 8), 7.0, dtype=T[dtype], device=DEV)
    lse = torch.full((n + 2, heads), 7.0, device=DEV)
    mq = max(new)
    size = B.sqap_kv_attention_workspace_bytes(s.cache, len(lens), mq, max_len, heads)
    work = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    scale = 1 / math.sqrt(s.D) if scale is None else scale
    for _ in range(2):      # the second call finds the first one's workspace
        B.sqap_kv_attention(s.cache, s.dtable, s.width, len(lens), ints(lens), ints(cu), mq, max_len, q, q.stride(0), heads, scale,
                            B.SQAP_KV_CAUSAL if causal else 0, out, out.stride(0), lse, CODE[dtype], work, size)
    torch.cuda.synchronize()
    assert (work[size:] == 0xFF).all()
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert (o[:2] == 7).all() and (o[n:] == 7).all() and (o[:, heads * s.D:] == 7).all() and (l[:2] == 7).all() and (l[n:] == 7).all()
    return o[:n, :heads * s.D], l[:n], cu


def check_attention(s, new, heads, causal, dtype, seed=0, q_gain=1.0, lens=None, scale=None, max_len=None):
    lens = s.lens if lens is None else lens
    rows = 2 + sum(new)
    g = np.random.default_rng(seed)
    fused = dev(g.standard_normal((rows, heads * s.D + 64)) * q_gain, T[dtype])
    q = fused[:, 64:]
    o, l, cu = run_attention(s, q, new, heads, causal, dtype, lens=lens, scale=scale, max_len=max_len)
    qn = q.double().cpu().numpy().reshape(rows, heads, s.D)
    scale = 1 / math.sqrt(s.D) if scale is None else scale
    fi = torch.finfo(T[dtype])
    G = heads // s.H
    for b, n in enumerate(lens):
        if new[b] == 0:
            continue
        n = n if max_len is None else min(n, max_len)
        k, there = R.kv_tokens(s.codes("k"), s.scale["k"], s.table[b], n, s.P)
        v, _ = R.kv_tokens(s.codes("v"), s.scale["v"], s.table[b], n, s.P)
        ref, lse, mag, pv, p = R.attention(qn[cu[b]:cu[b + 1]], k, v, there, new[b], causal, scale)
        got = o[cu[b]:cu[b + 1]].reshape(ref.shape)
        d = 2.0 ** -19 * (1 + mag)
        # weights of the codes: p vs, rounded in fp16 relative to their largest
        vs = np.zeros((n, s.H))
        for t in range(n):
            if there[t]:
                vs[t] = s.scale["v"][s.table[b, t // s.P]]
        code = np.divide(np.abs(v), vs[..., None], out=np.zeros_like(v), where=vs[..., None] > 0)
        small = (p * np.repeat(vs, G, 1).T[None]).max(-1, initial=0.0)[..., None] * np.repeat(code.sum(0), G, 0)[None] * 2.0 ** -25
        tol = np.abs(ref) * fi.eps / 2 + pv * (2.0 ** -11 + 2 * d[..., None]) + small + float(fi.smallest_normal) * fi.eps
        bad = ~(np.abs(got - ref) <= tol)
        assert not bad.any(), f"sequence {b}: {bad.sum()} of {bad.size} off, worst {np.abs(got - ref).max()} at {np.argwhere(bad)[0]}"
        gl = l[cu[b]:cu[b + 1]]
        empty = ~np.isfinite(lse)
        assert (gl[empty] == -np.inf).all() and (got[empty] == 0).all()
        fine = ~empty
        assert (np.abs(gl[fine] - lse[fine]) <= (d + 2.0 ** -20)[fine] + np.abs(lse[fine]) * 2.0 ** -22).all()


# decode kernel: one row to 16 per key/value head; pieces of the history and none; odd lengths; every page size
@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("dtype,heads,H,D,P,lens,new", [
    ("fp16", 1, 1, 64, 16, [1], [1]),
    ("bf16", 4, 4, 128, 64, [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 291], [1] * 12),
    ("fp16", 8, 2, 128, 32, [33, 0, 700], [1, 1, 1]),
    ("bf16", 7, 1, 256, 128, [5, 300, 513], [1, 1, 1]),
    ("fp16", 16, 2, 64, 16, [40, 260, 2000], [1, 0, 1]),
    ("bf16", 6, 3, 128, 64, [10, 1500, 4], [5, 3, 4]),
    ("fp16", 5, 5, 256, 16, [100, 1, 3000], [3, 1, 2]),
    ("bf16", 16, 1, 128, 64, [9000], [1])])
def test_attention_of_single_tokens(dtype, heads, H, D, P, lens, new, kind):
    s = Setup(lens, H, D, P, kind, sum(lens), nan_behind=True)
    for causal in (True, False):
        check_attention(s, new, heads, causal, dtype, seed=len(lens))


# prompt kernel: odd sizes on both sides of its tiles, cached prefixes, more queries than tokens
@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("dtype,heads,H,D,P,lens,new", [
    ("fp16", 1, 1, 64, 16, [17], [17]),
    ("bf16", 2, 2, 128, 64, [288, 1, 65], [288, 1, 64]),
    ("fp16", 8, 2, 128, 32, [130, 400, 33], [130, 17, 0]),
    ("bf16", 7, 1, 64, 128, [300], [19]),
    ("fp16", 4, 4, 256, 64, [70, 129], [70, 33]),
    ("bf16", 12, 3, 128, 16, [40, 3], [45, 5]),
    ("fp16", 8, 1, 256, 16, [1100], [40]),
    ("bf16", 4, 1, 128, 64, [2500, 700], [30, 9])])
def test_attention_of_prompts(dtype, heads, H, D, P, lens, new, kind):
    s = Setup(lens, H, D, P, kind, sum(lens), nan_behind=True)
    for causal in (True, False):
        check_attention(s, new, heads, causal, dtype, seed=len(lens))


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("new", [[1, 1], [40, 24]])
def test_attention_with_scales_far_apart_and_zero_pages(kind, new):
    s = Setup([300, 1100], 2, 128, 32, kind, 7, spread=6.0)
    for a in "kv":                            # pages of zeros: zero codes and scale 0, as an append leaves them
        z = s.table[1, 2:5]
        s.raw[a][z] = 0
        s.scale[a][z] = 0
    z = s.table[0, :10]                       # a history whose values are all zero
    s.raw["v"][z] = 0
    s.scale["v"][z] = 0
    s.scale["k"] = np.minimum(s.scale["k"], np.float32(0.05))
    s.to_device()
    check_attention(s, new, 4, True, "bf16", q_gain=0.5)


@pytest.mark.parametrize("new", [[1, 1, 1], [20, 33, 4]])
def test_attention_around_missing_pages_and_beyond_max_len(new):
    for kind in (R.INT8, R.E4M3):
        s = Setup([200, 90, 64], 2, 64, 16, kind, 3)
        s.table[0, 3] = -1
        s.table[0, 7:9] = [s.pages, 1 << 30]
        s.table[1, :] = -5                    # nothing at all
        s.to_device()
        check_attention(s, new, 4, False, "fp16")
        check_attention(s, new, 4, True, "fp16")
        check_attention(s, new, 2, False, "fp16", max_len=130)


def test_attention_large_and_small_queries():
    for kind in (R.INT8, R.E4M3):
        s = Setup([77, 50], 2, 128, 16, kind, 9)
        for gain, scale in ((3e4, 1e-5), (1e-30, 1e28), (2.0, 0.0), (2.0, -0.3)):
            check_attention(s, [1, 1], 2, True, "bf16", q_gain=gain, scale=scale)
            check_attention(s, [30, 20], 2, True, "bf16", q_gain=gain, scale=scale)


def test_attention_without_lse_empty_batch_and_no_pages():
    s = Setup([20], 2, 64, 16, R.INT8, 1)
    q = torch.ones(1, 128, dtype=torch.float16, device=DEV)
    out = torch.full((1, 128), 7.0, dtype=torch.float16, device=DEV)
    args = (s.dtable, s.width, 1, ints([20]), ints([0, 1]), 1, 20, q, 128, 2, 0.1, 1, out, 128)
    B.sqap_kv_attention(s.cache, *args, None, 0, None, 0)
    assert (out != 7).any()
    B.sqap_kv_attention(s.cache, s.dtable, s.width, 0, None, None, 1, 20, None, 128, 2, 0.1, 1, None, 128, None, 0, None, 0)
    empty = B.KvCache(*(torch.empty(0, 2, 16, 64, dtype=torch.int8, device=DEV) for _ in range(2)),
                      *(torch.empty(0, 2, device=DEV) for _ in range(2)), 0)
    lse = torch.zeros(1, 2, device=DEV)
    B.sqap_kv_attention(empty, *args, lse, 0, None, 0)
    torch.cuda.synchronize()
    assert (out == 0).all() and (lse == -math.inf).all()
    out.fill_(7)
    B.sqap_kv_attention(s.cache, s.dtable, 0, 1, ints([20]), ints([0, 1]), 1, 20, q, 128, 2, 0.1, 1, out, 128, lse, 0, None, 0)
    torch.cuda.synchronize()
    assert (out == 0).all() and (lse == -math.inf).all()


def test_cache_beyond_32_bit_offsets():
    """Pages whose codes start behind 2^32 bytes (and 2^31 tokens' worth of elements)."""
    P, H, D = 128, 8, 128
    pages = 2 ** 32 // (P * H * D) + 40
    k = torch.zeros(pages, H, P, D, dtype=torch.int8, device=DEV)
    v = torch.zeros(pages, H, P, D, dtype=torch.int8, device=DEV)
    sc = torch.zeros(2, pages, H, device=DEV)
    cache = B.KvCache(k, v, sc[0], sc[1], 0)
    n = 300
    table = ints([[pages - 1, pages - 17, pages - 3]])
    x = torch.randn(n, 2 * H * D, device=DEV).half()
    B.sqap_kv_append(cache, table, 3, 1, ints([n]), ints([0, n]), n, x, 2 * H * D, x[:, H * D:], 2 * H * D, 0)
    kb, vb = (torch.empty(n, H * D, dtype=torch.float16, device=DEV) for _ in range(2))
    B.sqap_kv_read(cache, table, 3, 1, None, ints([0, n]), n, kb, H * D, vb, H * D, 0)
    for nq in (1, 64):
        q = torch.randn(nq, H * D, device=DEV).half()
        out, ref = torch.empty_like(q), torch.empty_like(q)
        w = B.sqap_kv_attention_workspace_bytes(cache, 1, nq, n, H)
        work = torch.empty(w + 16, dtype=torch.uint8, device=DEV)
        B.sqap_kv_attention(cache, table, 3, 1, ints([n]), ints([0, nq]), nq, n, q, H * D, H, 0.1, 1, out, H * D, None, 0, work, w)
        pages2 = [pages - 1, pages - 17, pages - 3]
        small = B.KvCache(k[pages2].contiguous(), v[pages2].contiguous(), sc[0, pages2].contiguous(), sc[1, pages2].contiguous(), 0)
        B.sqap_kv_attention(small, ints([[0, 1, 2]]), 3, 1, ints([n]), ints([0, nq]), nq, n, q, H * D, H, 0.1, 1, ref, H * D, None, 0, work, w)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
    assert (kb.float() - x[:, :H * D].float()).abs().max() < 0.03 and (vb.float() - x[:, H * D:].float()).abs().max() < 0.03


def test_step_in_a_graph_and_on_two_streams():
    """Append and attention captured and replayed, and two caches on two streams with a workspace each."""
    H, D, P = 4, 128, 64
    sets = []
    for i in range(2):
        s = Setup([1300, 200], H, D, P, R.INT8, 20 + i)
        x = dev(s.g.standard_normal((2, 3 * H * D)), torch.float16)
        n = B.sqap_kv_attention_workspace_bytes(s.cache, 2, 1, 1300, H)
        assert n > 0
        sets.append((s, x, ints(s.lens), ints([0, 1, 2]), torch.empty(2, H * D, dtype=torch.float16, device=DEV),
                     torch.empty(n, dtype=torch.uint8, device=DEV), n))

    def step(i, stream=None):
        s, x, lens, cu, out, work, n = sets[i]
        B.sqap_kv_append(s.cache, s.dtable, s.width, 2, lens, cu, 1, x[:, H * D:], 3 * H * D, x[:, 2 * H * D:], 3 * H * D, 0, stream)
        B.sqap_kv_attention(s.cache, s.dtable, s.width, 2, lens, cu, 1, 1300, x, 3 * H * D, H, 0.09, 1, out, H * D, None, 0, work, n, stream)

    ref = []
    for i in (0, 1):
        step(i)
        torch.cuda.synchronize()
        ref.append(sets[i][4].clone())
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(30):
        for i, st in enumerate(streams):
            step(i, st)
    torch.cuda.synchronize()
    assert all(torch.equal(sets[i][4], ref[i]) for i in (0, 1))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(0)
        step(1)
    for i in (0, 1):
        sets[i][4].zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(sets[i][4], ref[i]) for i in (0, 1))


# ---------------------------------------------------------------------------------------------------------------- pages

class Pool:
    """The book-keeping, stated plainly."""

    def __init__(self, pages, rows, width, P, refs=None):
        self.refs = np.zeros(pages, np.int32) if refs is None else refs
        self.table = np.full((rows, width), -1, np.int32)
        self.lens = np.zeros(rows, np.int32)
        self.P = P

    def need(self, n):
        return -(-int(n) // self.P)

    def alloc(self, rows, add):
        free, granted, seen = list(np.flatnonzero(self.refs == 0)), [], set()
        asked = 0
        for r, a in zip(rows, add):
            ok = 0 <= r < len(self.lens) and r not in seen and a >= 0
            if 0 <= r < len(self.lens):
                seen.add(r)
            if ok:
                have, want = self.need(self.lens[r]), self.need(int(self.lens[r]) + a)
                ok = want <= self.table.shape[1] and int(self.lens[r]) + a < 2 ** 31
                if ok and want > have:
                    asked += want - have
                    ok = asked <= len(free)
                    if ok:
                        mine = free[asked - (want - have):asked]
                        self.table[r, have:want] = mine
                        self.refs[mine] = 1
                if ok:
                    self.lens[r] += a
            granted.append(int(ok))
        return granted

    def fork(self, src, dst):
        free, pairs, seen = list(np.flatnonzero(self.refs == 0)), [], set()
        sources = {s for s in src}
        was, asked = self.lens.copy(), 0
        table = self.table.copy()
        for s, d in zip(src, dst):
            R_ = len(was)
            ok = 0 <= s < R_ and 0 <= d < R_ and d not in seen and d not in sources and was[d] == 0
            if 0 <= d < R_:
                seen.add(d)
            if not ok:
                pairs.append((-2, -2))
                continue
            full, tail = was[s] // self.P, was[s] % self.P
            if tail:
                asked += 1
                if asked > len(free):
                    pairs.append((-2, -2))
                    continue
            self.table[d] = -1
            self.table[d, :full] = table[s, :full]
            self.refs[table[s, :full]] += 1
            pairs.append((-1, -1))
            if tail:
                page = free[asked - 1]
                pairs[-1] = (table[s, full], page)
                self.table[d, full] = page
                self.refs[page] = 1
            self.lens[d] = was[s]
        return pairs

    def free(self, rows):
        for r in rows:
            if 0 <= r < len(self.lens):
                for j in range(min(self.need(self.lens[r]), self.table.shape[1])):
                    self.refs[self.table[r, j]] -= 1
                    self.table[r, j] = -1
                self.lens[r] = 0


@pytest.mark.parametrize("pages,rows,width,P", [(60, 12, 9, 16), (5000, 300, 40, 64), (9001, 40, 130, 32)])
def test_pool_against_a_plain_statement(pages, rows, width, P):
    g = np.random.default_rng(pages)
    ref = Pool(pages, rows, width, P)
    refs, table, lens = dev(ref.refs), dev(ref.table), dev(ref.lens)
    args = (refs, pages, P, table, width, rows, lens)
    for step in range(25):
        n = int(g.integers(1, rows + 3))
        who = g.permutation(rows)[:min(n, rows)].tolist() + [-1, rows, 0][:max(0, n - rows)]
        what = step % 4
        if what in (0, 2):
            add = g.integers(0, P * width // 3, len(who)).tolist()
            if step == 2:
                add[0] = -3
                who.append(who[0])
                add.append(5)
            granted = torch.full((len(who),), 9, dtype=torch.int32, device=DEV)
            B.sqap_kv_alloc(*args, ints(who), ints(add), len(who), granted)
            assert granted.cpu().tolist() == ref.alloc(who, add), step
        elif what == 1:
            empty = np.flatnonzero(ref.lens == 0).tolist() or [0]
            dst = (empty + [0, rows, -1, empty[0]])[:max(3, n)]
            src = g.integers(0, rows, len(dst)).tolist()
            if step == 5:
                src[-1] = rows + 7
            pairs = torch.full((len(dst), 2), 9, dtype=torch.int32, device=DEV)
            granted = torch.full((len(dst),), 9, dtype=torch.int32, device=DEV)
            B.sqap_kv_fork(*args, ints(src), ints(dst), len(dst), pairs, granted)
            want = ref.fork(src, dst)
            assert [tuple(p) for p in pairs.cpu().tolist()] == want, step
            assert granted.cpu().tolist() == [int(p != (-2, -2)) for p in want]
        else:
            who = who[:max(1, len(who) // 2)]
            who += [who[0], -4, rows]
            B.sqap_kv_free(*args, ints(who), len(who))
            ref.free(who)
        torch.cuda.synchronize()
        assert np.array_equal(refs.cpu().numpy(), ref.refs), step
        assert np.array_equal(lens.cpu().numpy(), ref.lens), step
        got = table.cpu().numpy()
        for r in range(rows):
            k = ref.need(ref.lens[r])
            assert np.array_equal(got[r, :k], ref.table[r, :k]) and (ref.refs[got[r, :k]] > 0).all(), (step, r)
    B.sqap_kv_free(*args, ints(range(rows)), rows)
    torch.cuda.synchronize()
    assert (refs == 0).all() and (lens == 0).all() and (table == -1).all()


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
def test_copy_pages(kind):
    s = Setup([64] * 6, 3, 64, 16, kind, 2, spare=5)
    pairs = [(0, s.pages - 1), (-1, -1), (s.pages, 1), (2, -2), (5, s.pages - 2), (7, 7)]
    B.sqap_kv_copy_pages(s.cache, ints(pairs), len(pairs))
    torch.cuda.synchronize()
    for a in "kv":
        raw, sc = s.raw[a].copy(), s.scale[a].copy()
        for x, y in ((0, s.pages - 1), (5, s.pages - 2)):
            raw[y], sc[y] = raw[x], sc[x]
        assert np.array_equal(s.d[a].view(torch.uint8).cpu().numpy(), raw) and np.array_equal(s.ds[a].cpu().numpy(), sc)


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("H,D,P,lens,keep", [(2, 64, 16, [50, 33], [20, 33]), (3, 128, 64, [288, 1, 70], [160, 1, 0]),
                                             (1, 256, 128, [300], [129]), (2, 128, 32, [90, 64], [64, 7])])
def test_compact(kind, H, D, P, lens, keep):
    n = len(lens)
    s = Setup(lens + keep, H, D, P, kind, sum(lens), spread=2.0)
    kept = np.full((n, max(keep) + 3), 1 << 29, np.int32)
    for i in range(n):
        kept[i, :keep[i]] = np.sort(s.g.permutation(lens[i])[:keep[i]])
    if keep[0] > 4:                              # out of order, twice, outside: allowed, the last two read as zero
        kept[0, :5] = [7, 7, 3, -1, lens[0]]
    all_lens = ints(lens + keep)
    B.sqap_kv_compact(s.cache, s.dtable, s.width, 2 * n, all_lens, ints(range(n)), ints(range(n, 2 * n)), n, ints(kept), kept.shape[1],
                      ints(keep), max(keep))
    torch.cuda.synchronize()
    for a in "kv":
        codes, scale = s.codes(a), s.scale[a].copy()
        src = codes.copy(), scale.copy()
        for i in range(n):
            for j in range(-(-keep[i] // P)):
                page = s.table[n + i, j]
                x = np.zeros((H, P, D), np.float32)
                for t in range(P):
                    if j * P + t < keep[i]:
                        pos = kept[i, j * P + t]
                        if 0 <= pos < lens[i]:
                            f = s.table[i, pos // P]
                            x[:, t] = src[0][f, :, pos % P].astype(np.float32) * src[1][f][:, None]
                for h in range(H):
                    scale[page, h] = R.kv_scale(np.abs(x[h]).max(), kind)
                    codes[page, h] = R.kv_round(x[h] * R.inverse(scale[page, h]), kind)
        assert np.array_equal(s.ds[a].cpu().numpy(), scale) and np.array_equal(s.device_codes(a), codes)
