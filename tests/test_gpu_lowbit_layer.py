"""The low-bit operators in the order in which a decoder layer uses them: 4-bit projections around the 8-bit cache, the cache
brought down to the tokens that pruning kept, forked for candidates, one decoded token each. All calls go to one stream with
nothing read back in between; every step is then compared with its plain statement in 64 bits on the inputs that it had.
Tolerances: those of the single operators (test_gpu_mx4.py, test_gpu_kv.py)."""
import math

import numpy as np
import pytest

import lowbit_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B
    from paper_2509_09090_b200 import workloads as wl
    from test_gpu_kv import Setup, check_attention, dev, ints
    from test_gpu_mx4 import check_product, product_case

DEV = "cuda:0"
BATCH, ROWS, HIDDEN, HEADS, KV_HEADS, D, P = 2, 40, 256, 4, 2, 64, 16
QKV = (HEADS + 2 * KV_HEADS) * D
TABLE_ROWS, WIDTH, PAGES = 2 * BATCH + 2 * BATCH, 6, 40
SCALE = 1 / math.sqrt(D)


class Weights:
    def __init__(self, g, N, K, fmt):
        self.N, self.K, self.fmt = N, K, fmt
        w = dev(g.standard_normal((N, K)) / math.sqrt(K), torch.float32)
        self.codes = torch.empty((N, K // 2), dtype=torch.uint8, device=DEV)
        self.scales = torch.empty(B.sqap_mx4_scale_bytes(N, K, fmt), dtype=torch.uint8, device=DEV)
        self.g = torch.tensor([2.0 ** -9], device=DEV) if fmt == R.NVFP4 else None
        B.sqap_mx4_quantize(w, B.SQAP_FP32, N, K, K, None, fmt, self.g, self.codes, self.scales)

    def __call__(self, x, row_index=None, M=None):
        M = x.shape[0] if M is None else M
        out = torch.empty((M, self.N), dtype=torch.float16, device=DEV)
        size = B.sqap_mx4_workspace_bytes(M, self.N, self.K, self.fmt)
        work = torch.empty(size, dtype=torch.uint8, device=DEV)
        B.sqap_mx4_quantize_linear(x, B.SQAP_FP16, M, x.stride(0), row_index, None, self.codes, self.scales, self.g, self.N, self.K,
                                   self.fmt, out, self.N, B.SQAP_FP16, work, size)
        return out

    def check(self, x, got):
        codes, scale = R.mx4_quantize(x.double().cpu().numpy(), self.fmt)
        xq = (codes.reshape(len(codes), -1, R.block(self.fmt)) * scale[..., None]).reshape(codes.shape)
        wv = torch.empty((self.N, self.K), device=DEV)
        B.sqap_mx4_dequantize(self.codes, self.scales, self.N, self.K, self.fmt, self.g, wv, self.K, B.SQAP_FP32)
        check_product(got.double().cpu().numpy(), xq, wv.double().cpu().numpy(), "fp16", self.K)


class Layer:
    def __init__(self, kind):
        dt = torch.int8 if kind == R.INT8 else torch.float8_e4m3fn
        self.kind = kind
        self.k, self.v = (torch.zeros((PAGES, KV_HEADS, P, D), dtype=torch.uint8, device=DEV).view(dt) for _ in range(2))
        self.ks, self.vs = (torch.full((PAGES, KV_HEADS), math.nan, device=DEV) for _ in range(2))
        self.cache = B.KvCache(self.k, self.v, self.ks, self.vs, kind)
        self.refs = torch.zeros(PAGES, dtype=torch.int32, device=DEV)
        self.table = torch.full((TABLE_ROWS, WIDTH), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(TABLE_ROWS, dtype=torch.int32, device=DEV)
        self.pool = (self.refs, PAGES, P, self.table, WIDTH, TABLE_ROWS, self.lens)

    def append(self, first, n, new, qkv):
        cu = ints(np.arange(n + 1) * new)
        k, v = qkv[:, HEADS * D:], qkv[:, (HEADS + KV_HEADS) * D:]
        B.sqap_kv_append(self.cache, self.table[first:], WIDTH, n, self.lens[first:], cu, new, k, QKV, v, QKV, B.SQAP_FP16)

    def attend(self, first, n, new, max_len, qkv):
        cu = ints(np.arange(n + 1) * new)
        out = torch.empty((n * new, HEADS * D), dtype=torch.float16, device=DEV)
        size = B.sqap_kv_attention_workspace_bytes(self.cache, n, new, max_len, HEADS)
        work = torch.empty(size + 16, dtype=torch.uint8, device=DEV)
        B.sqap_kv_attention(self.cache, self.table[first:], WIDTH, n, self.lens[first:], cu, new, max_len, qkv, QKV, HEADS, SCALE,
                            B.SQAP_KV_CAUSAL, out, HEADS * D, None, B.SQAP_FP16, work, size)
        return out

    def snapshot(self):
        return [t.clone() for t in (self.k.view(torch.uint8), self.v.view(torch.uint8), self.ks, self.vs, self.table, self.lens, self.refs)]

    def tokens(self, snap, row):
        """Keys and values of a row of the table in a snapshot, in 64 bits."""
        k, v, ks, vs, table, lens = (t.cpu().numpy() for t in snap[:6])
        return [R.kv_tokens(R.kv_values(c, self.kind), s, table[row], int(lens[row]), P)[0] for c, s in ((k, ks), (v, vs))]

    def check_append(self, before, after, first, n, new, qkv):
        x = qkv.float().cpu().numpy()
        table, lens = after[4].cpu().numpy()[first:first + n], after[5].cpu().numpy()[first:first + n]
        for i, c0 in ((0, HEADS * D), (1, (HEADS + KV_HEADS) * D)):
            codes, scale = R.kv_values(before[i].cpu().numpy(), self.kind), before[2 + i].cpu().numpy().copy()
            R.kv_append(codes, scale, table, lens, np.arange(n + 1) * new, x[:, c0:c0 + KV_HEADS * D].reshape(-1, KV_HEADS, D), self.kind, P)
            assert np.array_equal(R.kv_values(after[i].cpu().numpy(), self.kind), codes)
            assert np.array_equal(after[2 + i].cpu().numpy(), scale, equal_nan=True)

    def check_attend(self, snap, first, n, new, qkv, got):
        q = qkv[:, :HEADS * D].double().cpu().numpy().reshape(-1, HEADS, D)
        table, vs = snap[4].cpu().numpy(), snap[3].cpu().numpy().astype(np.float64)
        for b in range(n):
            k, v = self.tokens(snap, first + b)
            ref, _, mag, pv, p = R.attention(q[b * new:(b + 1) * new], k, v, np.ones(len(k), bool), new, True, SCALE)
            s = np.stack([vs[table[first + b, t // P]] for t in range(len(k))])
            code = np.divide(np.abs(v), s[..., None], out=np.zeros_like(v), where=s[..., None] > 0)
            G = HEADS // KV_HEADS
            small = (p * np.repeat(s, G, 1).T[None]).max(-1)[..., None] * np.repeat(code.sum(0), G, 0)[None] * 2.0 ** -25
            tol = np.abs(ref) * 2.0 ** -11 + pv * (2.0 ** -11 + 2.0 ** -18 * (1 + mag[..., None])) + small + 2.0 ** -24
            assert (np.abs(got[b * new:(b + 1) * new].double().cpu().numpy().reshape(ref.shape) - ref) <= tol).all()


@pytest.mark.parametrize("kind,fmt", [(R.INT8, R.NVFP4), (R.E4M3, R.MXFP4)])
def test_prompt_prune_fork_and_decode(kind, fmt):
    g = np.random.default_rng(7)
    wqkv, wo = Weights(g, QKV, HIDDEN, fmt), Weights(g, HIDDEN, HEADS * D, fmt)
    layer = Layer(kind)
    x = dev(g.standard_normal((BATCH * ROWS, HIDDEN)), torch.float16)
    rows = ints(range(BATCH))

    # the prompts
    qkv = wqkv(x)
    granted = torch.full((BATCH,), 9, dtype=torch.int32, device=DEV)
    B.sqap_kv_alloc(*layer.pool, rows, ints([ROWS] * BATCH), BATCH, granted)
    empty = layer.snapshot()
    layer.append(0, BATCH, ROWS, qkv)
    full = layer.snapshot()
    o = layer.attend(0, BATCH, ROWS, ROWS, qkv)
    y = wo(o)

    # 16 of 24 visual tokens are pruned; the cache is brought down to the kept ones, the next projection reads their rows alone
    params = wl.prune_params(BATCH, ROWS, 5, 24, 6, 4, 0, 3, 8)
    scores = dev(g.standard_normal((BATCH, 24)), torch.float32)
    kept_rows = ROWS - 24 + 8
    kept = torch.empty((BATCH, ROWS), dtype=torch.int32, device=DEV)
    n_kept = torch.empty(BATCH, dtype=torch.int32, device=DEV)
    row_index = torch.empty(BATCH * kept_rows, dtype=torch.int32, device=DEV)
    B.sqap_prune_select(params, scores, None, kept_rows, kept, n_kept, row_index)
    y2 = wqkv(y, row_index, BATCH * kept_rows)
    B.sqap_kv_alloc(*layer.pool, ints(range(BATCH, 2 * BATCH)), n_kept, BATCH)
    B.sqap_kv_compact(layer.cache, layer.table, WIDTH, TABLE_ROWS, layer.lens, rows, ints(range(BATCH, 2 * BATCH)), BATCH, kept, ROWS,
                      n_kept, kept_rows)
    B.sqap_kv_free(*layer.pool, rows, BATCH)
    small = layer.snapshot()

    # two candidates of each observation
    src, dst = ints([BATCH + b for b in range(BATCH) for _ in range(2)]), ints(range(2 * BATCH, 4 * BATCH))
    pairs = torch.empty((2 * BATCH, 2), dtype=torch.int32, device=DEV)
    B.sqap_kv_fork(*layer.pool, src, dst, 2 * BATCH, pairs)
    B.sqap_kv_copy_pages(layer.cache, pairs, 2 * BATCH)
    B.sqap_kv_alloc(*layer.pool, dst, ints([1] * (2 * BATCH)), 2 * BATCH)
    forked = layer.snapshot()
    x1 = dev(g.standard_normal((2 * BATCH, HIDDEN)), torch.float16)
    qkv1 = wqkv(x1)
    layer.append(2 * BATCH, 2 * BATCH, 1, qkv1)
    step = layer.snapshot()
    o1 = layer.attend(2 * BATCH, 2 * BATCH, 1, kept_rows + 1, qkv1)
    y1 = wo(o1)
    B.sqap_kv_free(*layer.pool, dst, 2 * BATCH)
    B.sqap_kv_free(*layer.pool, ints(range(BATCH, 2 * BATCH)), BATCH)
    torch.cuda.synchronize()

    assert granted.tolist() == [1] * BATCH and n_kept.tolist() == [kept_rows] * BATCH
    wqkv.check(x, qkv)
    layer.check_append(empty, full, 0, BATCH, ROWS, qkv)
    layer.check_attend(full, 0, BATCH, ROWS, qkv, o)
    wo.check(o, y)
    wqkv.check(y[row_index.long()], y2)
    k_of = kept.cpu().numpy()[:, :kept_rows]
    for b in range(BATCH):           # compaction: a code is off by half a step of the new scale, e4m3 by 2^-4 of the value
        before, after = layer.tokens(full, b), layer.tokens(small, BATCH + b)
        for i, (x0, x1_) in enumerate(zip(before, after)):
            table, sc = small[4].cpu().numpy()[BATCH + b], small[2 + i].cpu().numpy().astype(np.float64)
            s = np.stack([sc[table[t // P]] for t in range(kept_rows)])[..., None]
            want = x0[k_of[b]]
            half = s * 0.5 if kind == R.INT8 else np.maximum(np.abs(want) * 2.0 ** -4, s * 2.0 ** -10)
            assert (np.abs(x1_ - want) <= half * (1 + 2.0 ** -20) + np.abs(want) * 2.0 ** -21).all()
    for c in range(2 * BATCH):       # a candidate starts as its observation; the observation does not see the candidate's token
        for was, now, old in zip(layer.tokens(small, BATCH + c // 2), layer.tokens(forked, 2 * BATCH + c), layer.tokens(step, BATCH + c // 2)):
            assert np.array_equal(was, now[:kept_rows]) and np.array_equal(was, old)
    wqkv.check(x1, qkv1)
    layer.check_append(forked, step, 2 * BATCH, 2 * BATCH, 1, qkv1)
    layer.check_attend(step, 2 * BATCH, 2 * BATCH, 1, qkv1, o1)
    wo.check(o1, y1)
    assert (layer.refs == 0).all() and (layer.table == -1).all() and (layer.lens == 0).all()


# eight pieces of a history and more are joined by four warps to a row; uneven lengths leave some pieces empty
@pytest.mark.parametrize("dtype,heads,H,D_,lens,new", [("fp16", 4, 1, 64, [2300, 1, 0], [1, 1, 1]), ("bf16", 2, 2, 128, [5000, 1100], [1, 1]),
                                                       ("fp16", 2, 1, 256, [2500, 300], [1, 0]), ("bf16", 16, 1, 128, [10000], [20]), ("fp16", 2, 1, 256, [4200, 300], [20, 9]),
                                                       ("bf16", 4, 1, 64, [9000, 40, 0], [70, 40, 5])])
def test_attention_in_many_pieces(dtype, heads, H, D_, lens, new):
    s = Setup(lens, H, D_, 64, R.E4M3, sum(lens), nan_behind=True)
    check_attention(s, new, heads, True, dtype, seed=3)


# either side of the rules by which a product is given to a kernel: weight stream (one token; few elements and products), clusters
# (long K, few rows and tokens), pairs (one to three tiles of tokens)
@pytest.mark.parametrize("fmt", [R.NVFP4, R.MXFP4])
@pytest.mark.parametrize("M,N,K", [(4, 1000, 1024), (4, 136, 3104), (3, 4096, 4096), (3, 4104, 4096), (2, 40, 16384), (1, 17, 65536),
                                   (64, 1024, 4096), (65, 1024, 4096), (16, 1280, 1024), (256, 24, 16384), (257, 24, 16384),
                                   (5, 12288, 96), (70, 520, 1056), (193, 300, 608), (385, 264, 2080)])
def test_product_at_the_borders_of_the_rules(M, N, K, fmt):
    xc, xs, wc, ws, x, w = product_case(M, N, K, fmt, seed=M + N + K)
    xc, xs, wc, ws = (dev(a) for a in (xc, xs, wc, ws))
    ldo = (N + 7) // 8 * 8 + 8
    for dtype, code in (("fp32", B.SQAP_FP32), ("bf16", B.SQAP_BF16)):
        out = torch.full((M + 1, ldo), 7.0, dtype=torch.float32 if dtype == "fp32" else torch.bfloat16, device=DEV)
        B.sqap_mx4_linear(xc, xs, None, M, wc, ws, None, N, K, fmt, out, ldo, code)
        torch.cuda.synchronize()
        o = out.double().cpu().numpy()
        assert (o[M] == 7).all() and (o[:, N:] == 7).all()
        check_product(o[:M, :N], x, w, dtype, K)


def test_fork_of_a_row_whose_last_page_is_missing():
    """A number in the page table that is no page holds no tokens, whichever number it is: the full pages are shared all the same."""
    for hole in (-1, -2, -7, 50):
        layer = Layer(R.INT8)
        B.sqap_kv_alloc(*layer.pool, ints([0]), ints([2 * P + 3]), 1)
        layer.table[0, 2] = hole
        pairs = torch.empty((1, 2), dtype=torch.int32, device=DEV)
        granted = torch.empty(1, dtype=torch.int32, device=DEV)
        B.sqap_kv_fork(*layer.pool, ints([0]), ints([1]), 1, pairs, granted)
        B.sqap_kv_copy_pages(layer.cache, pairs, 1)
        torch.cuda.synchronize()
        assert granted.tolist() == [1] and pairs.tolist() == [[hole, 3]]
        assert layer.table[1].tolist() == [0, 1, 3, -1, -1, -1] and layer.lens[:2].tolist() == [2 * P + 3] * 2
        assert layer.refs[:5].tolist() == [2, 2, 1, 1, 0]
