"""The operators around the cache where they can go wrong: queries that are not numbers, caches beyond 32-bit offsets, calls from two host
threads and on two streams at once, equal calls, histories without a token to see, what an empty call leaves alone. Tolerances: those of the
single operators (test_gpu_kv_views.py)."""
import math
import threading

import numpy as np
import pytest

import cache_reference as C
import lowbit_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B
    from test_gpu_kv import CODE, DEV, Setup, T, dev, ints
    from test_gpu_kv_views import Queries, check_rows, run_window, scratch, tokens_of


def run_shared(s, qs, new, sizes, prefix, lens, table=None, stream=None):
    cu = np.concatenate([[0], np.cumsum(sizes)])
    table = s.dtable if table is None else table
    args = (len(lens), max(new), max(lens), len(sizes), max(sizes), max(prefix), qs.heads)
    n = B.sqap_kv_attention_shared_workspace_bytes(s.cache, *args)
    B.sqap_kv_attention_shared(s.cache, table, table.stride(0), len(lens), ints(lens), qs.dcu, max(new), max(lens), ints(cu), len(sizes), max(sizes),
                               ints(prefix), max(prefix), qs.q, qs.q.stride(0), qs.heads, 1 / math.sqrt(s.D), 1, qs.out, qs.out.stride(0), qs.lse,
                               CODE[qs.dtype], scratch(n), n, stream)


def shared_setup(sizes, prefix, own, H, D, P, kind, seed=0):
    """Sequences whose tables name the same pages for the prefix (a multiple of the page)."""
    lens = [p + x for p, x in zip(np.repeat(prefix, sizes), own)]
    s = Setup(lens, H, D, P, kind, seed=seed)
    first = np.concatenate([[0], np.cumsum(sizes)])
    for g, n in enumerate(sizes):
        s.table[first[g]:first[g] + n, :prefix[g] // P] = s.table[first[g], :prefix[g] // P]
    s.to_device()
    return s, lens


def check_sequences(s, qs, o, l, lens, new, seen, skip=()):
    for b, n in enumerate(lens):
        if new[b] == 0:
            continue
        r = np.array([i for i in range(qs.cu[b], qs.cu[b + 1]) if i not in skip])
        if len(r):
            check_rows(s, o[r], l[r], qs.qn[r], *tokens_of(s, s.table[b], n), seen(n, new[b])[r - qs.cu[b]], qs.dtype, 1 / math.sqrt(s.D))


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("D,new", [(64, 1), (128, 3), (128, 40), (256, 1), (256, 20)])
def test_a_query_that_is_not_finite_spoils_its_own_row_alone(D, new, bad):
    s = Setup([300, 77], 2, D, 16, R.INT8, seed=D)
    qs = Queries(s, [new, new], 4, "fp16")
    at = qs.cu[0] + new - 1
    qs.q[at, :D] = bad
    run_window(s, qs, [new, new], 50, 3, [300, 77])
    o, l = qs.results([(qs.cu[0], qs.cu[-1])])
    if bad != bad:
        assert np.isnan(o[at, :D]).all() and np.isnan(l[at, 0])
    o[at, :D], l[at, 0] = 0, 0
    qs.qn[at] = np.where(np.isfinite(qs.qn[at]), qs.qn[at], 0)
    check_sequences(s, qs, o, l, [300, 77], [new, new], lambda n, m: C.in_window(n, m, 50, 3), skip=(at,))
    # the other heads of the row
    k, (v, vs), there = tokens_of(s, s.table[0], 300)
    ref = C.attention(qs.qn[at:at + 1], k, v, C.in_window(300, new, 50, 3)[-1:], 1 / math.sqrt(D))[0][0]
    assert np.abs(o[at].reshape(4, D)[1:] - ref[1:]).max() <= 2.0 ** -8

    s, lens = shared_setup([3, 2], [64, 48], [5, 9, 2, 30, 4], 2, D, 16, R.E4M3, seed=D)
    qs = Queries(s, [new] * 5, 4, "bf16")
    at = qs.cu[1] + new - 1
    qs.q[at, D:2 * D] = bad
    run_shared(s, qs, [new] * 5, [3, 2], [64, 48], lens)
    o, l = qs.results([(qs.cu[0], qs.cu[-1])])
    if bad != bad:
        assert np.isnan(o[at, D:2 * D]).all() and np.isnan(l[at, 1])
    check_sequences(s, qs, o, l, lens, [new] * 5, C.causal, skip=(at,))


def test_caches_beyond_32_bit_offsets():
    """Pages whose codes lie beyond 2^32 bytes, and received weights in rows far apart."""
    H, D, P, pages = 8, 128, 64, 70000
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    k, v = (torch.zeros((pages, H, P, D), dtype=torch.int8, device=DEV) for _ in range(2))
    ks, vs = (torch.full((pages, H), 1 / 40, device=DEV) for _ in range(2))
    g = np.random.default_rng(0)
    n, new = 200, 2
    table = np.array([[pages - 1, pages - 7, 65537, pages - 2], [pages - 1, pages - 3, pages - 4, pages - 5]], np.int32)
    raw = {}
    for a, t in (("k", k), ("v", v)):
        raw[a] = g.integers(-100, 101, (8, H, P, D)).astype(np.int8)
        for i, p in enumerate(table.reshape(-1)):
            if i != 4:
                t[int(p)] = dev(raw[a][i])
    cache = B.KvCache(k, v, ks, vs, R.INT8)

    class S:
        pass
    s = S()
    s.H, s.D, s.cache = H, D, cache
    q = Queries(s, [new, new], H, "fp16")
    dtable, lens = ints(table), ints([n, n])
    values = lambda a, b: np.concatenate([raw[a][0 if (b, i) == (1, 0) else 4 * b + i].transpose(1, 0, 2) for i in range(4)])[:n] / 40.0  # noqa: E731
    scale, ones = 1 / math.sqrt(D), np.ones(n, bool)

    def check(seen):
        o, l = q.results([(q.cu[0], q.cu[-1])])
        for b in range(2):
            r = slice(q.cu[b], q.cu[b + 1])
            yield check_rows(s, o[r], l[r], q.qn[r], values("k", b), (values("v", b), np.full((n, H), 1 / 40)), ones, seen, "fp16", scale)

    size = B.sqap_kv_attention_window_workspace_bytes(cache, 2, new, n, H, 70, 5)
    B.sqap_kv_attention_window(cache, dtable, 4, 2, lens, q.dcu, new, n, q.q, q.q.stride(0), H, scale, 70, 5, q.out, q.out.stride(0), q.lse, 0, scratch(size), size)
    list(check(C.in_window(n, new, 70, 5)))
    size = B.sqap_kv_attention_shared_workspace_bytes(cache, 2, new, n, 1, 2, 64, H)
    B.sqap_kv_attention_shared(cache, dtable, 4, 2, lens, q.dcu, new, n, ints([0, 2]), 1, 2, ints([64]), 64, q.q, q.q.stride(0), H, scale, 1, q.out,
                               q.out.stride(0), q.lse, 0, scratch(size), size)
    list(check(C.causal(n, new)))
    ldm = (1 << 30) + 8
    mass = torch.zeros(ldm + 256, device=DEV)
    size = B.sqap_kv_attention_mass_workspace_bytes(cache, 2, new, n, H, new)
    B.sqap_kv_attention_mass(cache, dtable, 4, 2, lens, q.dcu, new, n, q.q, q.q.stride(0), H, scale, 1, new, q.out, q.out.stride(0), q.lse, None, mass, ldm, 0,
                             scratch(size), size)
    for b, (p, rel) in enumerate(check(C.causal(n, new))):
        got = mass[b * ldm:b * ldm + n].double().cpu().numpy()
        want = p.sum((0, 1))
        assert (np.abs(got - want) <= (p * rel[..., None]).sum((0, 1)) + want * (new * H + 2) * 2.0 ** -24).all()
    # the row that lies behind 2^30 weights, evicted into the first
    kept, count = torch.empty((1, 50), dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
    m = mass[ldm:ldm + n].cpu().numpy()
    B.sqap_kv_evict(mass, ldm, 2, lens, ints([1]), ints([0]), 1, ints([50]), 2, 7, n, kept, 50, count)
    torch.cuda.synchronize()
    want = C.evict(m[None, :], [n], [0], [50], 2, 7, n, 50)[0]
    assert kept[0].tolist() == want and np.array_equal(mass[:50].cpu().numpy(), m[want])


def test_calls_from_two_host_threads_and_on_two_streams():
    """Each thread with a stream, outputs and a workspace of its own; the same bits as one call after the other."""
    s = Setup([900, 70, 301], 2, 128, 16, R.E4M3, seed=1)
    sh, lens = shared_setup([5, 3], [128, 64], [7] * 8, 2, 128, 16, R.INT8, seed=2)
    mass0 = dev(np.random.default_rng(4).random((6, 3000)).astype(np.float32))
    torch.cuda.synchronize()

    def once(i, stream):
        with torch.cuda.stream(stream):
            a, b = Queries(s, [1, 1, 1] if i % 2 else [30, 2, 9], 4, "bf16", seed=i), Queries(sh, [1] * 8, 4, "fp16", seed=i)
            stream.synchronize()
            run_window(s, a, [1, 1, 1] if i % 2 else [30, 2, 9], 100, 3, [900, 70, 301])
            run_shared(sh, b, [1] * 8, [5, 3], [128, 64], lens)
            m, kept, count = mass0.clone(), torch.empty((3, 700), dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
            B.sqap_kv_evict(m, 3000, 6, ints([3000, 1500, 17, 0, 0, 0]), ints([0, 1, 2]), ints([3, 4, 5]), 3, ints([700, 600, 5]), 1, 9, 3000, kept, 700, count)
            x = a.q.contiguous()
            y = torch.empty_like(x)
            B.sqap_rotary(x, x.stride(0), x.shape[0], 4, 128, 128, ints(np.arange(x.shape[0])[None]), x.shape[0], 1, None, mass0[0, :64], 0, y, y.stride(0), 1)
            stream.synchronize()
            return [t.clone() for t in (a.out, a.lse, b.out, b.lse, m, kept, count, y)]

    want = [once(i, torch.cuda.Stream()) for i in range(2)]
    got = [[], []]
    threads = [threading.Thread(target=lambda i=i: got[i].extend(once(i, torch.cuda.Stream()) for _ in range(8))) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert B.sqap_device_status() == B.SQAP_OK
    for i in range(2):
        assert len(got[i]) == 8
        for run in got[i]:
            assert all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(run, want[i]))


@pytest.mark.parametrize("D,new", [(64, 1), (128, 40), (256, 30)])
def test_nothing_to_see(D, new):
    """max_len 0, a cache without pages, a table without entries: rows are 0, their log-sum-exps -inf, weights only what they were."""
    s = Setup([100, 60], 2, D, 16, R.INT8)
    empty = B.KvCache(*(torch.empty((0, 2, 16, D), dtype=torch.int8, device=DEV) for _ in range(2)), *(torch.empty((0, 2), device=DEV) for _ in range(2)), R.INT8)
    for cache, ldt, max_len in ((s.cache, s.width, 0), (empty, s.width, 100), (s.cache, 0, 100)):
        for which in ("window", "shared", "mass"):
            qs = Queries(s, [new, new], 4, "fp16")
            mass = torch.full((2, 100), 5.0, device=DEV)
            tail = (qs.q, qs.q.stride(0), 4, 0.1)
            out = (qs.out, qs.out.stride(0), qs.lse)
            head = (cache, s.dtable, ldt, 2, ints([100, 60]), qs.dcu, new, max_len)
            work = scratch(1 << 20)
            if which == "window":
                B.sqap_kv_attention_window(*head, *tail, 9, 2, *out, 0, work, 1 << 20)
            elif which == "shared":
                B.sqap_kv_attention_shared(*head, ints([0, 2]), 1, 2, ints([32]), 32, *tail, 1, *out, 0, work, 1 << 20)
            else:
                B.sqap_kv_attention_mass(*head, *tail, 1, new, *out, None, mass, 100, 0, work, 1 << 20)
            o, l = qs.results([(qs.cu[0], qs.cu[-1])])
            r = slice(qs.cu[0], qs.cu[-1])
            assert (o[r] == 0).all() and (l[r] == -np.inf).all()
            if which == "mass":
                n = [min(x, max_len) for x in (100, 60)]
                assert all((mass[b, :n[b]] == 0).all() and (mass[b, n[b]:] == 5).all() for b in range(2))


@pytest.mark.parametrize("D,new", [(128, 1), (128, 50), (256, 9)])
def test_equal_calls_give_equal_bits(D, new):
    s, lens = shared_setup([4, 2], [512, 64], [700, 9, 20, 3, 1, 40], 2, D, 64, R.E4M3, seed=6)
    runs = []
    for _ in range(3):
        a, b, c = (Queries(s, [new] * 6, 8, "bf16") for _ in range(3))
        run_window(s, a, [new] * 6, 333, 5, lens)
        run_shared(s, b, [new] * 6, [4, 2], [512, 64], lens)
        mass = torch.zeros((6, max(lens)), device=DEV)
        n = B.sqap_kv_attention_mass_workspace_bytes(s.cache, 6, new, max(lens), 8, new)
        B.sqap_kv_attention_mass(s.cache, s.dtable, s.width, 6, ints(lens), c.dcu, new, max(lens), c.q, c.q.stride(0), 8, 0.1, 1, new, c.out, c.out.stride(0), c.lse,
                                 None, mass, max(lens), 1, scratch(n), n)
        torch.cuda.synchronize()
        runs.append([a.out, a.lse, b.out, b.lse, c.out, c.lse, mass])
    for r in runs[1:]:
        assert all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(r, runs[0]))
