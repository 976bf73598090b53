"""Attention over a window, of sequences that share a prefix, and with the weights that the tokens received, against plain statements in
64 bits. Tolerances of outputs and log-sum-exps: those of sqap_kv_attention (test_gpu_kv.py), whose arithmetic they share. A token's
received weight is a sum of softmax weights p, each off by the errors of its score and of its row's log-sum-exp,
  p (2 d + 2^-20 + |lse| 2^-21),  d = 2^-19 (1 + max_t sum_d |q k| scale)
and N positive terms added in fp32 add at most N 2^-24 of the sum; the past joins with one more rounding."""
import math

import numpy as np
import pytest

import cache_reference as C
import lowbit_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B
    from test_gpu_kv import CODE, DEV, Setup, T, dev, ints

GUARD = 3.0


def check_rows(s, got, lse_got, q, table_k, table_v, there, seen, dtype, scale):
    """Rows of one sequence against keys and values [n, H, D] of which it sees `seen`; returns the weights and what their errors need."""
    k, v, vs = table_k, table_v[0], table_v[1]
    seen = seen & there[None, :]
    ref, lse, mag, pv, p = C.attention(q, k, v, seen, scale)
    G = q.shape[1] // s.H
    fi = torch.finfo(T[dtype])
    d = 2.0 ** -19 * (1 + mag)
    code = np.divide(np.abs(v), vs[..., None], out=np.zeros_like(v), where=vs[..., None] > 0)
    small = (p * np.repeat(vs, G, 1).T[None]).max(-1, initial=0.0)[..., None] * np.repeat(code.sum(0), G, 0)[None] * 2.0 ** -25
    tol = np.abs(ref) * fi.eps / 2 + pv * (2.0 ** -11 + 2 * d[..., None]) + small + float(fi.smallest_normal) * fi.eps
    got = got.reshape(ref.shape)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - ref))} at {np.argwhere(bad)[0]}"
    empty = ~np.isfinite(lse)
    assert (lse_got[empty] == -np.inf).all() and (got[empty] == 0).all()
    fine = ~empty
    assert (np.abs(lse_got[fine] - lse[fine]) <= (d + 2.0 ** -20)[fine] + np.abs(lse[fine]) * 2.0 ** -22).all()
    return p, np.where(fine, 2 * d + 2.0 ** -20 + np.abs(np.where(fine, lse, 0)) * 2.0 ** -21, 0)


def tokens_of(s, row, n):
    """Keys, (values, value scale of each token) and whether each token exists, of a row of the table."""
    k, there = R.kv_tokens(s.codes("k"), s.scale["k"], row, n, s.P)
    v, _ = R.kv_tokens(s.codes("v"), s.scale["v"], row, n, s.P)
    vs = np.zeros((n, s.H))
    for t in range(n):
        if there[t]:
            vs[t] = s.scale["v"][row[t // s.P]]
    return k, (v, vs), there


class Queries:
    def __init__(self, s, new, heads, dtype, seed=0, gain=1.0, front=1, behind=2):
        g = np.random.default_rng(seed)
        self.cu = front + np.concatenate([[0], np.cumsum(new)])
        self.rows = int(self.cu[-1]) + behind
        self.fused = dev(g.standard_normal((self.rows, heads * s.D + 64)) * gain, T[dtype])
        self.q = self.fused[:, 64:]
        self.out = torch.full((self.rows, heads * s.D + 8), GUARD, dtype=T[dtype], device=DEV)
        self.lse = torch.full((self.rows, heads), GUARD, device=DEV)
        self.heads, self.dtype, self.dcu = heads, dtype, ints(self.cu)
        self.qn = self.q.double().cpu().numpy().reshape(self.rows, heads, s.D)

    def results(self, computed):
        """Outputs and log-sum-exps; rows that are not `computed` are as they were."""
        torch.cuda.synchronize()
        assert B.sqap_device_status() == B.SQAP_OK
        o, l = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        rest = np.ones(self.rows, bool)
        for a, b in computed:
            rest[a:b] = False
        assert (o[rest] == GUARD).all() and (l[rest] == GUARD).all() and (o[:, -8:] == GUARD).all()
        return o[:, :-8], l


def scratch(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------------------------------------------------ window

def run_window(s, qs, new, window, sinks, lens, max_q=None, max_len=None, table=None):
    max_q = max(new) if max_q is None else max_q
    max_len = max(lens) if max_len is None else max_len
    table = s.dtable if table is None else table
    n = B.sqap_kv_attention_window_workspace_bytes(s.cache, len(lens), max_q, max_len, qs.heads, window, sinks)
    B.sqap_kv_attention_window(s.cache, table, table.stride(0), len(lens), ints(lens), qs.dcu, max_q, max_len, qs.q, qs.q.stride(0), qs.heads,
                               1 / math.sqrt(s.D), window, sinks, qs.out, qs.out.stride(0), qs.lse, CODE[qs.dtype], scratch(n), n)


def check_window(s, new, heads, dtype, window, sinks, seed=0, lens=None):
    lens = s.lens if lens is None else lens
    qs = Queries(s, new, heads, dtype, seed)
    run_window(s, qs, new, window, sinks, lens)
    o, l = qs.results([(qs.cu[0], qs.cu[-1])])
    for b, n in enumerate(lens):
        r = slice(qs.cu[b], qs.cu[b + 1])
        if new[b]:
            check_rows(s, o[r], l[r], qs.qn[r], *tokens_of(s, s.table[b], n), C.in_window(n, new[b], window, sinks), dtype, 1 / math.sqrt(s.D))


WINDOWS = [(1, 0), (3, 1), (17, 5), (64, 64), (100, 0), (129, 40), (5000, 3), (1, 4000), (2 ** 31 - 1, 2 ** 31 - 1)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("kind,dtype,heads,H,D,P,lens,new", [
    (R.INT8, "fp16", 2, 2, 64, 16, [1, 0, 2, 63, 64, 65, 300], [1] * 7),
    (R.E4M3, "bf16", 8, 2, 128, 64, [5, 700, 1300], [1, 1, 1]),
    (R.E4M3, "fp16", 4, 1, 128, 32, [2, 400, 129], [4, 3, 4]),
    (R.INT8, "bf16", 7, 1, 256, 128, [9, 290, 513], [1, 1, 1])])
def test_window_of_single_tokens(kind, dtype, heads, H, D, P, lens, new, window, sinks):
    check_window(Setup(lens, H, D, P, kind, seed=len(lens) + D), new, heads, dtype, window, sinks)


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("kind,dtype,heads,H,D,P,lens,new", [
    (R.INT8, "fp16", 2, 2, 64, 16, [300, 20, 0, 64], [300, 20, 0, 30]),
    (R.E4M3, "bf16", 8, 2, 128, 64, [290, 700], [129, 67]),
    (R.INT8, "fp16", 3, 1, 128, 32, [600, 5], [40, 9]),
    (R.E4M3, "fp16", 2, 2, 256, 128, [290, 33], [150, 40])])
def test_window_of_prompts(kind, dtype, heads, H, D, P, lens, new, window, sinks):
    check_window(Setup(lens, H, D, P, kind, seed=len(lens) + D), new, heads, dtype, window, sinks)


def test_window_in_pieces():
    """Few long histories are cut into pieces, the sinks' tiles among them."""
    s = Setup([9000, 4100], 1, 128, 64, R.E4M3, seed=3)
    check_window(s, [1, 1], 4, "fp16", 3000, 200)
    check_window(s, [2, 1], 4, "bf16", 8000, 1)
    s = Setup([6000], 1, 128, 64, R.INT8, seed=4)
    check_window(s, [100], 2, "fp16", 3500, 70)
    s = Setup([5000], 1, 256, 64, R.INT8, seed=4)
    check_window(s, [60], 1, "fp16", 3500, 70)


@pytest.mark.parametrize("D,new", [(64, 1), (128, 2), (128, 40), (256, 30)])
def test_window_more_queries_than_tokens(D, new):
    """Queries at positions before the first token see nothing."""
    s = Setup([max(1, new - 1), 0, new + 200], 2, D, 16, R.INT8, seed=new)
    check_window(s, [new, new, new], 4, "fp16", 7, 2)


@pytest.mark.parametrize("D,new,P", [(64, 1, 16), (128, 1, 16), (128, 3, 64), (128, 70, 16), (64, 200, 32), (256, 1, 32), (256, 20, 16)])
@pytest.mark.parametrize("window,sinks", [(200, 20), (37, 0), (64, 16)])
def test_window_does_not_need_the_pages_outside(D, new, P, window, sinks):
    """Pages that hold neither the window's tokens nor the sinks' may have been given up: same bits, whatever their numbers are now,
    pages of not-a-numbers among them."""
    n = 1501
    s = Setup([n], 2, D, P, R.E4M3, seed=D + new, nan_behind=True)
    spare = next(i for i in range(s.pages) if i not in s.table)
    got = []
    for hole in (None, -1, s.pages + 5, spare):
        qs = Queries(s, [new], 4, "bf16")
        table = s.table.copy()
        if hole is not None:
            table[0, -(-sinks // P):(n - new + 1 - window) // P] = hole
        run_window(s, qs, [new], window, sinks, [n], table=ints(table))
        got.append(qs.results([(qs.cu[0], qs.cu[-1])]))
    for o, l in got[1:]:
        assert np.array_equal(o, got[0][0]) and np.array_equal(l, got[0][1])


@pytest.mark.parametrize("D,new,max_q", [(64, 5, 3), (128, 60, 41), (256, 30, 20)])
def test_window_queries_beyond_max_q_are_left_out(D, new, max_q):
    s = Setup([400], 1, D, 32, R.INT8, seed=9)
    qs = Queries(s, [new], 2, "fp16")
    run_window(s, qs, [new], 50, 3, [400], max_q=max_q)
    o, l = qs.results([(qs.cu[0], qs.cu[0] + max_q)])
    r = slice(qs.cu[0], qs.cu[0] + max_q)
    check_rows(s, o[r], l[r], qs.qn[r], *tokens_of(s, s.table[0], 400), C.in_window(400, new, 50, 3)[:max_q], "fp16", 1 / math.sqrt(D))


def test_window_without_lse_and_without_work():
    s = Setup([100], 2, 64, 16, R.INT8)
    qs = Queries(s, [1], 2, "fp16")
    run_window(s, qs, [1], 10, 1, [100])
    o, _ = qs.results([(qs.cu[0], qs.cu[-1])])
    again = Queries(s, [1], 2, "fp16")
    B.sqap_kv_attention_window(s.cache, s.dtable, s.width, 1, ints([100]), again.dcu, 1, 100, again.q, again.q.stride(0), 2, 1 / 8, 10, 1,
                               again.out, again.out.stride(0), None, 0, None, 0)
    torch.cuda.synchronize()
    assert np.array_equal(again.out.double().cpu().numpy()[:, :-8], o)
    B.sqap_kv_attention_window(s.cache, s.dtable, s.width, 0, ints([100]), again.dcu, 1, 100, again.q, again.q.stride(0), 2, 1 / 8, 10, 1,
                               again.out, again.out.stride(0), None, 0, None, 0)
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------------- shared prefix

class Group:
    """Sequences of groups (sizes, prefixes); own[b] tokens behind the prefix of sequence b. The pages of the prefix are missing from all
    rows of the table but the first of each group, and what the page in which a prefix ends holds of it is no number in theirs."""

    def __init__(self, sizes, prefixes, own, H, D, P, kind, seed=0, lens=None):
        self.first = np.concatenate([[0], np.cumsum(sizes)])
        self.prefix, self.sizes = list(prefixes), list(sizes)
        self.lens = [p + x for p, x in zip(np.repeat(prefixes, sizes), own)] if lens is None else list(lens)
        self.s = Setup([max(n, p) for n, p in zip(self.lens, np.repeat(prefixes, sizes))], H, D, P, kind, seed=seed)
        self.table = self.s.table.copy()
        for g, n in enumerate(sizes):
            self.table[self.first[g] + 1:self.first[g] + n, :prefixes[g] // P] = -1
            for b in range(self.first[g] + 1, self.first[g] + n):
                page = self.table[b, prefixes[g] // P]
                if page >= 0:
                    for a in "kv":
                        self.s.raw[a][page, :, :prefixes[g] % P] = 0x7F
        self.s.to_device()

    def tokens(self, b, max_prefix):
        """What sequence b is made of: the group's first tokens, then its own."""
        s = self.s
        g = int(np.searchsorted(self.first, b, side="right")) - 1
        n, pre = self.lens[b], max(0, min(self.prefix[g], max_prefix))
        k, (v, vs), there = tokens_of(s, s.table[b] if b == self.first[g] else self.table[b], n)
        k0, (v0, vs0), there0 = tokens_of(s, s.table[self.first[g]], min(n, pre))
        for own, shared in ((k, k0), (v, v0), (vs, vs0), (there, there0)):
            own[:len(shared)] = shared
        return k, (v, vs), there


def check_shared(gr, new, heads, dtype, causal=True, seed=0, max_prefix=None, max_group=None, cu_group=None, max_len=None):
    s, P = gr.s, gr.s.P
    max_prefix = max(gr.prefix) if max_prefix is None else max_prefix
    max_group = max(gr.sizes) if max_group is None else max_group
    cu_group = gr.first if cu_group is None else cu_group
    max_len = max(gr.lens) if max_len is None else max_len
    qs = Queries(s, new, heads, dtype, seed)
    table, batch, scale = ints(gr.table), len(gr.lens), 1 / math.sqrt(s.D)
    args = (batch, max(new), max_len, len(cu_group) - 1, max_group, max_prefix, heads)
    n = B.sqap_kv_attention_shared_workspace_bytes(s.cache, *args)
    B.sqap_kv_attention_shared(s.cache, table, table.stride(0), batch, ints(gr.lens), qs.dcu, max(new), max_len, ints(cu_group),
                               len(cu_group) - 1, max_group, ints(gr.prefix), max_prefix, qs.q, qs.q.stride(0), heads, scale,
                               B.SQAP_KV_CAUSAL if causal else 0, qs.out, qs.out.stride(0), qs.lse, CODE[dtype], scratch(n), n)
    members = [b for g in range(len(cu_group) - 1) for b in range(cu_group[g], min(cu_group[g + 1], cu_group[g] + max_group))]
    o, l = qs.results([(qs.cu[b], qs.cu[b + 1]) for b in members])
    for b in members:
        if not new[b]:
            continue
        r, n = slice(qs.cu[b], qs.cu[b + 1]), min(gr.lens[b], max_len)
        k, (v, vs), there = gr.tokens(b, max_prefix)
        seen = C.causal(gr.lens[b], new[b])[:, :n] if causal else np.ones((new[b], n), bool)
        check_rows(s, o[r], l[r], qs.qn[r], k[:n], (v[:n], vs[:n]), there[:n], seen, dtype, scale)


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("dtype,heads,H,D,P,sizes,prefixes,own,new", [
    ("fp16", 1, 1, 64, 16, [1], [1], [1], [1]),
    ("bf16", 4, 2, 128, 64, [3, 1, 2], [64, 0, 100], [1, 30, 64, 7, 2, 129], [1] * 6),
    ("fp16", 4, 1, 128, 32, [8, 5], [300, 33], [5] * 13, [1] * 13),                 # 32 rows over a prefix
    ("bf16", 8, 1, 128, 64, [40], [500], list(range(1, 41)), [1] * 40),             # 320: the tensor-core kernel
    ("fp16", 2, 1, 64, 16, [70, 2], [90, 17], [3] * 72, [1] * 72),
    ("bf16", 2, 1, 256, 16, [9, 20], [200, 65], [17] * 29, [1] * 29),
    ("fp16", 6, 3, 128, 64, [3, 4], [130, 128], [5, 6, 7, 300, 6, 5, 9], [5, 0, 3, 2, 4, 5, 1]),
    ("fp16", 128, 32, 64, 16, [20, 19], [120, 110], [1 + b % 13 for b in range(39)], [1 - b % 5 // 4 for b in range(39)]),   # tiles over own tokens
    ("bf16", 4, 2, 128, 16, [2, 3], [70, 300], [90, 60, 100, 40, 33], [90, 31, 64, 40, 1])])
def test_shared_prefix(dtype, heads, H, D, P, sizes, prefixes, own, new, kind):
    gr = Group(sizes, prefixes, own, H, D, P, kind, seed=len(own))
    check_shared(gr, new, heads, dtype)
    check_shared(gr, new, heads, dtype, causal=False, seed=1)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_shared_prefix_in_pieces(D):
    check_shared(Group([3, 2], [5000, 2100], [1500, 3, 40, 2500, 1], 1, D, 64, R.E4M3, seed=2), [1] * 5, 2, "fp16")
    check_shared(Group([20, 2], [3000, 2100], [1500, 3, 40, 2500, 1] + [9] * 17, 1, D, 64, R.INT8, seed=2), [2] * 22, 4, "bf16")


@pytest.mark.parametrize("D,heads", [(64, 2), (128, 2), (128, 16), (256, 2)])
def test_shared_queries_inside_the_prefix(D, heads):
    """Sequences that end within the prefix, and whose queries' positions lie in it or before the first token."""
    gr = Group([4, 3], [100, 50], None, 2, D, 32, R.INT8, seed=D, lens=[100, 40, 103, 0, 50, 1, 53])
    check_shared(gr, [5, 6, 7, 2, 3, 4, 1], heads, "fp16")
    check_shared(gr, [5, 6, 7, 2, 3, 4, 1], heads, "fp16", causal=False)
    check_shared(gr, [40, 30, 60, 0, 20, 40, 33], heads, "bf16")


@pytest.mark.parametrize("D,copies,heads", [(128, 3, 2), (128, 24, 2), (128, 24, 8), (256, 30, 2), (256, 40, 16)])
def test_shared_limits_drop_work_and_move_nothing(D, copies, heads):
    """More sequences than max_group, prefixes beyond max_prefix, sequences outside of all groups, tokens beyond max_len."""
    own = [7 + b for b in range(copies + 3)]
    gr = Group([1, copies, 2], [64, 130, 0], own, 1, D, 64, R.INT8, seed=5)
    new = [1] * (copies + 3)
    check_shared(gr, new, heads, "fp16", max_group=copies - 1)
    gr.table = gr.s.table.copy()
    shared = [gr.s.table[1, :2]]
    gr.table[2:copies + 1, :2] = shared[0]                  # beyond max_prefix every sequence reads its own entries
    for a in "kv":
        gr.s.raw[a][gr.s.raw[a] == 0x7F] = 0x31
    gr.s.to_device()
    check_shared(gr, new, heads, "fp16", max_prefix=100)
    check_shared(gr, new, heads, "fp16", max_prefix=0)
    gr.prefix = gr.prefix[1:2]
    some = np.array([1, copies + 1])
    gr.first, gr.sizes = np.array([0, 1, copies + 1, copies + 3]), [1, copies, 2]
    gr.prefix = [0, 130, 0]
    qs = Queries(gr.s, new, heads, "fp16")
    s, table = gr.s, ints(gr.table)
    n = B.sqap_kv_attention_shared_workspace_bytes(s.cache, copies + 3, 1, max(gr.lens), 1, copies, 130, heads)
    B.sqap_kv_attention_shared(s.cache, table, table.stride(0), copies + 3, ints(gr.lens), qs.dcu, 1, max(gr.lens), ints(some), 1, copies,
                               ints([130]), 130, qs.q, qs.q.stride(0), heads, 1 / math.sqrt(D), 1, qs.out, qs.out.stride(0), qs.lse, 0, scratch(n), n)
    o, l = qs.results([(qs.cu[1], qs.cu[copies + 1])])
    for b in range(1, copies + 1):
        r, n = slice(qs.cu[b], qs.cu[b + 1]), gr.lens[b]
        check_rows(s, o[r], l[r], qs.qn[r], *gr.tokens(b, 130), C.causal(n, 1), "fp16", 1 / math.sqrt(D))


def test_shared_groups_out_of_order_or_beyond_the_batch_touch_nothing():
    gr = Group([2, 2], [20, 20], [5, 6, 7, 8], 1, 128, 16, R.INT8)
    s = gr.s
    for cu_group in ([3, 1, 1], [-5, -1, 0], [4, 9, 12], [0, 0, 0]):
        qs = Queries(s, [1] * 4, 2, "fp16")
        n = B.sqap_kv_attention_shared_workspace_bytes(s.cache, 4, 1, 40, 2, 2, 20, 2)
        B.sqap_kv_attention_shared(s.cache, s.dtable, s.width, 4, ints(gr.lens), qs.dcu, 1, 40, ints(cu_group), 2, 2, ints([20, -3]), 20, qs.q,
                                   qs.q.stride(0), 2, 0.1, 1, qs.out, qs.out.stride(0), qs.lse, 0, scratch(n), n)
        qs.results([])


# ---------------------------------------------------------------------------------------------------- received weights

def check_mass(s, new, heads, dtype, last_q, causal=True, past="given", ldm=None, max_q=None, max_len=None, seed=0, spoil=None, lens=None):
    lens = s.lens if lens is None else lens
    batch, scale = len(lens), 1 / math.sqrt(s.D)
    max_q = max(new) if max_q is None else max_q
    max_len = max(lens) if max_len is None else max_len
    ldm = max(lens) + 3 if ldm is None else ldm
    qs = Queries(s, new, heads, dtype, seed)
    if spoil is not None:
        qs.q[qs.cu[0] + spoil, :s.D] = math.nan
        qs.qn = qs.q.double().cpu().numpy().reshape(qs.rows, heads, s.D)
    before = np.random.default_rng(seed).random((batch, ldm)).astype(np.float32)
    mass = dev(before.copy())
    old = {"given": dev(before * 2), "same": mass, "none": None}[past]
    n = B.sqap_kv_attention_mass_workspace_bytes(s.cache, batch, max_q, max_len, heads, last_q)
    B.sqap_kv_attention_mass(s.cache, s.dtable, s.width, batch, ints(lens), qs.dcu, max_q, max_len, qs.q, qs.q.stride(0), heads, scale,
                             B.SQAP_KV_CAUSAL if causal else 0, last_q, qs.out, qs.out.stride(0), qs.lse, old, mass, ldm, CODE[dtype], scratch(n), n)
    o, l = qs.results([(qs.cu[b], qs.cu[b] + min(new[b], max_q)) for b in range(batch)])
    got = mass.double().cpu().numpy()
    factor = {"given": 2.0, "same": 1.0, "none": 0.0}[past]
    for b, n in enumerate(lens):
        kept = min(new[b], max_q)
        r = slice(qs.cu[b], qs.cu[b] + kept)
        seen = (C.causal(n, new[b]) if causal else np.ones((new[b], n), bool))[:kept, :min(n, max_len)]
        n_seen = min(n, max_len)
        k, (v, vs), there = tokens_of(s, s.table[b], n_seen)
        q = qs.qn[r].copy()
        clean = np.isfinite(q).all(-1)
        q[~clean] = 0
        if clean.all():
            p, rel = check_rows(s, o[r], l[r], q, k, (v, vs), there, seen, dtype, scale)
        else:
            ref = C.attention(q, k, v, seen & there[None, :], scale)
            p, rel = ref[4], 2 * 2.0 ** -19 * (1 + ref[2]) + 2.0 ** -20 + np.abs(ref[1]) * 2.0 ** -21
            assert np.isnan(l[r][~clean]).all()
        p = p * clean[..., None]
        count = np.arange(kept) >= new[b] - last_q
        want, err = p[count].sum((0, 1)), (p * rel[..., None])[count].sum((0, 1))
        had = np.where(np.arange(n_seen) < n - new[b], before[b][:n_seen] * factor if n_seen <= ldm else np.resize(before[b] * factor, n_seen), 0)
        terms = max(1, int(count.sum()) * heads)
        m = min(n_seen, ldm)
        want = (want + had)[:m]
        bad = np.abs(got[b, :m] - want) > err[:m] + want * (terms + 2) * 2.0 ** -24 + 2.0 ** -100
        assert not bad.any(), f"sequence {b}: {bad.sum()} of {m} off, {got[b, :m][bad][:3]} for {want[bad][:3]}"
        assert np.array_equal(got[b, m:], before[b, m:])


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("dtype,heads,H,D,P,lens,new", [
    ("fp16", 1, 1, 64, 16, [1], [1]),
    ("bf16", 4, 4, 128, 64, [1, 2, 15, 16, 17, 0, 64, 65, 291], [1] * 9),
    ("fp16", 8, 2, 128, 32, [33, 0, 700], [1, 1, 1]),
    ("bf16", 7, 1, 256, 128, [5, 300, 513], [1, 1, 1]),
    ("bf16", 16, 1, 128, 64, [9000], [1]),
    ("fp16", 5, 5, 256, 16, [100, 1, 3000], [3, 1, 2]),
    ("fp16", 32, 32, 64, 16, [290, 100], [1, 1]),
    ("bf16", 6, 3, 128, 64, [300, 1500, 64], [290, 40, 64]),
    ("fp16", 2, 2, 256, 32, [200, 77], [100, 77])])
def test_mass(dtype, heads, H, D, P, lens, new, kind):
    s = Setup(lens, H, D, P, kind, seed=sum(lens))
    check_mass(s, new, heads, dtype, max(new))
    check_mass(s, new, heads, dtype, 1, past="none", seed=1)
    check_mass(s, new, heads, dtype, 32, past="same", causal=False, seed=2)


@pytest.mark.parametrize("D,heads,new", [(64, 4, 1), (128, 2, 1), (128, 4, 3), (128, 4, 50), (256, 2, 1), (256, 2, 30)])
def test_mass_limits(D, heads, new):
    s = Setup([400, new, 90 + new], 2, D, 16, R.E4M3, seed=new, nan_behind=True)
    check_mass(s, [new, new, new], heads, "fp16", 0)
    check_mass(s, [new, new, new], heads, "fp16", 2 ** 31 - 1, ldm=70)
    check_mass(s, [new, 0, new], heads, "bf16", new, past="same", max_len=410)
    if new > 2:
        check_mass(s, [new, new, new], heads, "bf16", new - 1, max_q=new - 1)
    check_mass(s, [new] * 3, heads, "fp16", new, spoil=new - 1)
    s.table[0, 3] = -1
    s.table[0, 5] = s.pages
    s.table[2, 0] = -7
    s.to_device()
    check_mass(s, [new] * 3, heads, "fp16", new)


def test_mass_of_tokens_before_the_first():
    """More queries than tokens: the first rows see nothing and give nothing."""
    s = Setup([3, 0, 40], 2, 128, 16, R.INT8)
    check_mass(s, [5, 4, 60], 4, "fp16", 60)
    check_mass(s, [5, 4, 6], 4, "fp16", 60)
