"""The operators around the cache in the order in which a decoder layer uses them over an episode: projection, rotary positions (rows and
columns of the visual tokens), the cache, attention with received weights, eviction and compaction, attention over a window, candidates
forked from each observation and attended to together. All calls go to one stream with nothing read back in between; every step is
then compared with its plain statement in 64 bits on the inputs that it had, and the same calls captured into a graph give the same bits.
Tolerances: those of the single operators."""
import math

import numpy as np
import pytest

import cache_reference as C
import lowbit_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B
    from test_gpu_kv import dev, ints
    from test_gpu_kv_views import check_rows
    from test_gpu_lowbit_layer import Weights

DEV = "cuda:0"
OBS, ROWS, HIDDEN, HEADS, KV, D, P, COPIES = 2, 40, 256, 4, 2, 64, 16, 3
QKV = (HEADS + 2 * KV) * D
TABLE, WIDTH, PAGES, LDM = 2 * OBS + OBS * COPIES, 6, 60, 64
KEEP, FIRST, RECENT, WINDOW, SINKS = 24, 1, 8, 9, 2
SCALE = 1 / math.sqrt(D)
AXES = [i // 4 % 3 for i in range(D // 2)]
FREQ = (1e4 ** (-2 * np.arange(D // 2) / D)).astype(np.float32)


class Episode:
    def __init__(self, kind):
        g = np.random.default_rng(3)
        self.kind = kind
        self.w = Weights(g, QKV, HIDDEN, R.NVFP4)
        dt = torch.int8 if kind == R.INT8 else torch.float8_e4m3fn
        self.k, self.v = (torch.zeros((PAGES, KV, P, D), dtype=torch.uint8, device=DEV).view(dt) for _ in range(2))
        self.ks, self.vs = (torch.zeros((PAGES, KV), device=DEV) for _ in range(2))
        self.cache = B.KvCache(self.k, self.v, self.ks, self.vs, kind)
        self.refs = torch.zeros(PAGES, dtype=torch.int32, device=DEV)
        self.table = torch.full((TABLE, WIDTH), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(TABLE, dtype=torch.int32, device=DEV)
        self.mass = torch.zeros((TABLE, LDM), device=DEV)
        self.kept = torch.zeros((OBS, KEEP), dtype=torch.int32, device=DEV)
        self.n_kept = torch.zeros(OBS, dtype=torch.int32, device=DEV)
        self.pool = (self.refs, PAGES, P, self.table, WIDTH, TABLE, self.lens)
        self.freq = dev(FREQ)
        self.work = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
        self.x = [dev(g.standard_normal((n, HIDDEN)), torch.float16) for n in (OBS * ROWS, OBS, OBS, OBS * COPIES)]
        prompt = np.stack([np.arange(ROWS) // 16, np.arange(ROWS) % 16 // 4, np.arange(ROWS) % 4])
        self.positions = [ints(np.tile(prompt, OBS))] + [ints(np.full((3, n), ROWS + i)) for i, n in enumerate((OBS, OBS, OBS * COPIES))]
        self.qkv = [torch.empty((x.shape[0], QKV), dtype=torch.float16, device=DEV) for x in self.x]
        self.raw = [torch.empty_like(q) for q in self.qkv]
        self.out = [torch.empty((x.shape[0], HEADS * D), dtype=torch.float16, device=DEV) for x in self.x]
        self.lse = [torch.empty((x.shape[0], HEADS), device=DEV) for x in self.x]
        self.all_rows, self.dst = ints(range(TABLE)), ints(range(OBS, 2 * OBS))
        self.pairs = torch.empty((OBS * COPIES, 2), dtype=torch.int32, device=DEV)
        self.fork_from, self.fork_to = ints([OBS + i // COPIES for i in range(OBS * COPIES)]), ints(range(2 * OBS, TABLE))
        self.prefix, self.groups = ints([KEEP // P * P] * OBS), ints(range(0, OBS * COPIES + 1, COPIES))
        self.ones, self.many, self.budget = ints([1] * TABLE), ints([ROWS] * OBS), ints([KEEP, KEEP - 3])
        self.cu = [ints(np.arange(n + 1) * m) for n, m in ((OBS, ROWS), (OBS, 1), (OBS, 1), (OBS * COPIES, 1))]
        self.size = [B.sqap_mx4_workspace_bytes(x.shape[0], QKV, HIDDEN, R.NVFP4) for x in self.x]

    def state(self):
        return [self.k.view(torch.uint8), self.v.view(torch.uint8), self.ks, self.vs, self.table, self.lens, self.refs, self.mass]

    def project(self, i, st):
        x, M = self.x[i], self.x[i].shape[0]
        B.sqap_mx4_quantize_linear(x, 0, M, HIDDEN, None, None, self.w.codes, self.w.scales, self.w.g, QKV, HIDDEN, R.NVFP4, self.qkv[i], QKV, 0,
                                   self.work, self.size[i], st)
        self.raw[i].copy_(self.qkv[i])
        B.sqap_rotary(self.qkv[i], QKV, M, HEADS + KV, D, D, self.positions[i], M, 3, bytes(AXES), self.freq, 0, self.qkv[i], QKV, 0, st)

    def append(self, i, first, n, new, rows, add, st):
        B.sqap_kv_alloc(*self.pool, rows, add, n, None, st)
        q = self.qkv[i]
        B.sqap_kv_append(self.cache, self.table[first:], WIDTH, n, self.lens[first:], self.cu[i], new, q[:, HEADS * D:], QKV,
                         q[:, (HEADS + KV) * D:], QKV, 0, st)

    def attend_mass(self, i, new, max_len, past, st):
        size = B.sqap_kv_attention_mass_workspace_bytes(self.cache, OBS, new, max_len, HEADS, 16)
        assert size <= self.work.numel()
        B.sqap_kv_attention_mass(self.cache, self.table, WIDTH, OBS, self.lens, self.cu[i], new, max_len, self.qkv[i], QKV, HEADS, SCALE, 1, 16,
                                 self.out[i], HEADS * D, self.lse[i], past, self.mass, LDM, 0, self.work, size, st)

    def run(self, snap):
        """All calls; `snap` is called after each step."""
        st = torch.cuda.current_stream()
        # the prompts, then a token
        self.project(0, st)
        self.append(0, 0, OBS, ROWS, self.all_rows, self.many, st)
        self.attend_mass(0, ROWS, ROWS, None, st)
        snap()
        self.project(1, st)
        self.append(1, 0, OBS, 1, self.all_rows, self.ones, st)
        self.attend_mass(1, 1, ROWS + 1, self.mass, st)
        snap()
        # evicted to other rows of the table, whose pages follow the counts
        B.sqap_kv_evict(self.mass, LDM, TABLE, self.lens, self.all_rows, self.dst, OBS, self.budget, FIRST, RECENT, ROWS + 1, self.kept, KEEP, self.n_kept, st)
        B.sqap_kv_alloc(*self.pool, self.dst, self.n_kept, OBS, None, st)
        B.sqap_kv_compact(self.cache, self.table, WIDTH, TABLE, self.lens, self.all_rows, self.dst, OBS, self.kept, KEEP, self.n_kept, KEEP, st)
        B.sqap_kv_free(*self.pool, self.all_rows, OBS, st)
        snap()
        # a token that looks at a window
        self.project(2, st)
        self.append(2, OBS, OBS, 1, self.dst, self.ones, st)
        size = B.sqap_kv_attention_window_workspace_bytes(self.cache, OBS, 1, KEEP + 1, HEADS, WINDOW, SINKS)
        B.sqap_kv_attention_window(self.cache, self.table[OBS:], WIDTH, OBS, self.lens[OBS:], self.cu[2], 1, KEEP + 1, self.qkv[2], QKV, HEADS, SCALE,
                                   WINDOW, SINKS, self.out[2], HEADS * D, self.lse[2], 0, self.work, size, st)
        snap()
        # candidates of each, a token of their own, attended to together
        n = OBS * COPIES
        B.sqap_kv_fork(*self.pool, self.fork_from, self.fork_to, n, self.pairs, None, st)
        B.sqap_kv_copy_pages(self.cache, self.pairs, n, st)
        self.project(3, st)
        self.append(3, 2 * OBS, n, 1, self.fork_to, self.ones, st)
        size = B.sqap_kv_attention_shared_workspace_bytes(self.cache, n, 1, KEEP + 2, OBS, COPIES, KEEP // P * P, HEADS)
        B.sqap_kv_attention_shared(self.cache, self.table[2 * OBS:], WIDTH, n, self.lens[2 * OBS:], self.cu[3], 1, KEEP + 2, self.groups, OBS, COPIES,
                                   self.prefix, KEEP // P * P, self.qkv[3], QKV, HEADS, SCALE, 1, self.out[3], HEADS * D, self.lse[3], 0, self.work,
                                   size, st)
        snap()


def tokens(snap, row, kind):
    k, v, ks, vs, table, lens = (t.cpu().numpy() for t in snap[:6])
    n = int(lens[row])
    got = [R.kv_tokens(R.kv_values(c, kind), s, table[row], n, P)[0] for c, s in ((k, ks), (v, vs))]
    scale = np.array([vs[table[row, t // P]] for t in range(n)]).reshape(n, KV).astype(np.float64)
    return got[0], (got[1], scale), np.ones(n, bool)


class Heads:
    H = KV


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
def test_episode(kind):
    e = Episode(kind)
    snaps = []
    e.run(lambda: snaps.append([t.clone() for t in e.state()]))
    torch.cuda.synchronize()
    assert B.sqap_device_status() == B.SQAP_OK
    outs = [o.double().cpu().numpy() for o in e.out]
    lses = [l.double().cpu().numpy() for l in e.lse]
    queries = [q.double().cpu().numpy()[:, :HEADS * D].reshape(-1, HEADS, D) for q in e.qkv]

    # rotary, in place over queries and keys; values as they were
    for raw, qkv, pos in zip(e.raw, e.qkv, e.positions):
        a, got = raw.double().cpu().numpy(), qkv.double().cpu().numpy()
        heads = a[:, :(HEADS + KV) * D].reshape(len(a), -1, D)
        ref = C.rotary(heads, pos.cpu().numpy(), AXES, FREQ, False).reshape(len(a), -1)
        half = np.abs(heads[..., :D // 2]) + np.abs(heads[..., D // 2:])
        size = np.concatenate([half, half], -1).reshape(ref.shape)
        assert (np.abs(got[:, :ref.shape[1]] - ref) <= np.abs(ref) * 2.0 ** -11 + size * 2.0 ** -20 + 2.0 ** -24).all()
        assert np.array_equal(got[:, ref.shape[1]:], a[:, ref.shape[1]:])

    # attention and received weights of the prompts and of the token behind them
    weight = np.zeros((OBS, LDM))
    slack = np.zeros((OBS, LDM))
    for i, new in ((0, ROWS), (1, 1)):
        for b in range(OBS):
            k, v, there = tokens(snaps[i], b, kind)
            r, n = slice(b * new, (b + 1) * new), len(k)
            p, rel = check_rows(Heads, outs[i][r], lses[i][r], queries[i][r], k, v, there, C.causal(n, new), "fp16", SCALE)
            count = np.arange(new) >= new - 16
            weight[b, :n] += p[count].sum((0, 1))
            slack[b, :n] += (p * rel[..., None])[count].sum((0, 1))
        got = snaps[i][7].double().cpu().numpy()[:OBS]
        assert (np.abs(got - weight) <= slack + weight * (16 * HEADS + 2) * 2.0 ** -24 * (i + 1)).all()

    # eviction by what the device summed, and the tokens that were kept
    mass = snaps[1][7].cpu().numpy()
    lens = snaps[1][5].tolist()
    want = C.evict(mass, lens, [0, 1], e.budget.tolist(), FIRST, RECENT, ROWS + 1, KEEP)
    for i, w in enumerate(want):
        assert e.kept[i].tolist() == w + [-1] * (KEEP - len(w)) and int(e.n_kept[i]) == len(w) == int(snaps[2][5][OBS + i])
        assert np.array_equal(snaps[2][7][OBS + i, :len(w)].cpu().numpy(), mass[i, w])
        before, after = tokens(snaps[1], i, kind), tokens(snaps[2], OBS + i, kind)
        for old, new in ((before[0], after[0]), (before[1][0], after[1][0])):
            step = np.abs(old[w]).max() * (1 / 254 if kind == R.INT8 else 2.0 ** -4) * 1.01
            assert np.abs(old[w] - new).max() <= step
    assert snaps[2][5].tolist()[:OBS] == [0] * OBS and (snaps[2][4][:OBS] == -1).all()

    # the window
    for i in range(OBS):
        k, v, there = tokens(snaps[3], OBS + i, kind)
        r = slice(i, i + 1)
        check_rows(Heads, outs[2][r], lses[2][r], queries[2][r], k, v, there, C.in_window(len(k), 1, WINDOW, SINKS), "fp16", SCALE)

    # the candidates
    for j in range(OBS * COPIES):
        k, v, there = tokens(snaps[4], 2 * OBS + j, kind)
        r = slice(j, j + 1)
        check_rows(Heads, outs[3][r], lses[3][r], queries[3][r], k, v, there, C.causal(len(k), 1), "fp16", SCALE)


def test_episode_in_a_graph():
    """The same calls captured and replayed, twice, from the same beginning: the bits of the calls one by one."""
    e = Episode(R.E4M3)
    start = [t.clone() for t in e.state()]

    def begin():
        for t, s in zip(e.state(), start):
            t.copy_(s)

    results = lambda: [t.clone() for t in e.state() + e.out + e.lse + [e.kept, e.n_kept]]  # noqa: E731
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        e.run(lambda: None)
        want = results()
        begin()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        graph.capture_begin()
        e.run(lambda: None)
        graph.capture_end()
        for _ in range(2):
            begin()
            for t in e.out + e.lse:
                t.fill_(7.0)
            graph.replay()
            got = results()
            stream.synchronize()
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(want, got))
    assert B.sqap_device_status() == B.SQAP_OK
