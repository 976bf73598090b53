"""The 8-bit key/value cache at its corners, against plain statements in 64 bits. Tolerances: those of test_gpu_kv.py."""
import math

import numpy as np
import pytest

import lowbit_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B
    from test_gpu_kv import CODE, DEV, T, Setup, check_attention, dev, ints, run_attention


def unused_scales(s, value):
    """Page 0 belongs to no sequence (what it held moves to a spare page), and the scales of every page without a sequence are `value`."""
    used = set(s.table[s.table >= 0].tolist())
    if 0 in used:
        spare = min(set(range(s.pages)) - used)
        for a in "kv":
            s.raw[a][spare], s.scale[a][spare] = s.raw[a][0], s.scale[a][0]
        s.table[s.table == 0] = spare
        used = set(s.table[s.table >= 0].tolist())
    free = sorted(set(range(s.pages)) - used)
    assert free[0] == 0
    for a in "kv":
        s.scale[a][free] = value
    s.to_device()


# ------------------------------------------------------------------------------------------------- pages of no sequence

SMALLEST = float(np.array([1], np.int32).view(np.float32)[0])      # what an int32 left in recycled memory looks like


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("dtype,heads,H,D,P,lens,new,hole", [
    ("fp16", 1, 1, 64, 16, [1, 17, 40, 300], [1, 1, 1, 1], None),        # histories that end in the first half of a step of 32 keys
    ("fp16", 4, 2, 64, 32, [5000, 33], [1, 1], None),                    # ... cut into pieces
    ("bf16", 12, 1, 128, 64, [5, 290, 2000], [1, 1, 1], None),           # 9 to 16 rows
    ("fp16", 2, 2, 128, 16, [200, 60], [1, 1], 3),                       # a missing page inside
    ("bf16", 3, 1, 256, 32, [300], [2], 2),
    ("fp16", 2, 1, 128, 16, [200, 3], [40, 3], 3), ("bf16", 2, 1, 256, 16, [200], [40], 3)])
def test_attention_does_not_look_at_scales_of_pages_it_does_not_have(dtype, heads, H, D, P, lens, new, hole, kind):
    s = Setup(lens, H, D, P, kind, sum(lens))
    if hole is not None:
        s.table[0, hole] = -1
    for value in (SMALLEST, 1e-40, math.inf, math.nan):
        unused_scales(s, np.float32(value))
        check_attention(s, new, heads, True, dtype, seed=len(lens))


# ---------------------------------------------------------------------------------------------------------------- forks

@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("hole", [-1, -2, 1000])
def test_fork_of_a_row_without_its_last_page_is_a_copy(hole, kind):
    """What the source's missing page does not hold, its copy does not hold either, whoever had the free pages before."""
    P, H, D, n = 16, 2, 64, 2 * 16 + 3
    g = np.random.default_rng(3)
    pages, rows, width = 8, 3, 6
    k, v = (dev(g.integers(1, 0x70, (pages, H, P, D)).astype(np.uint8)).view(torch.int8 if kind == R.INT8 else torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (dev(np.exp(g.standard_normal((pages, H))).astype(np.float32)) for _ in range(2))
    cache = B.KvCache(k, v, ks, vs, kind)
    refs, lens = (torch.zeros(m, dtype=torch.int32, device=DEV) for m in (pages, rows))
    table = torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
    pool = (refs, pages, P, table, width, rows, lens)
    x = dev(g.standard_normal((n, 2 * H * D)), torch.float16)
    B.sqap_kv_alloc(*pool, ints([0]), ints([n]), 1)
    B.sqap_kv_append(cache, table, width, 1, lens, ints([0, n]), n, x, 2 * H * D, x[:, H * D:], 2 * H * D, 0)
    table[0, 2] = hole
    pairs, granted = torch.empty((1, 2), dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
    B.sqap_kv_fork(*pool, ints([0]), ints([1]), 1, pairs, granted)
    B.sqap_kv_copy_pages(cache, pairs, 1)
    assert granted.tolist() == [1] and pairs.tolist() == [[-1, -1]]
    assert table[1].tolist() == [0, 1, -1, -1, -1, -1] and refs.tolist() == [2, 2, 1, 0, 0, 0, 0, 0]
    for step in range(2):
        m = n + step
        assert lens[:2].tolist() == [m, m]
        back = torch.full((2 * m, H * D), 9.0, dtype=torch.float16, device=DEV)
        B.sqap_kv_read(cache, table, width, 2, None, ints([0, m, 2 * m]), m, None, 0, back, H * D, 0)
        q = x[:2, :H * D].contiguous()
        q[1] = q[0]
        out, lse = torch.empty_like(q), torch.empty((2, H), device=DEV)
        B.sqap_kv_attention(cache, table, width, 2, lens, ints([0, 1, 2]), 1, m, q, H * D, H, 0.125, 1, out, H * D, lse, 0, None, 0)
        torch.cuda.synchronize()
        assert torch.equal(back[:m], back[m:]) and (back[2 * P:m] == 0).all()
        assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1])
        # one more token for both: no page, so it is dropped for both
        B.sqap_kv_alloc(*pool, ints([0, 1]), ints([1, 1]), 2)
        B.sqap_kv_append(cache, table, width, 2, lens, ints([0, 1, 2]), 1, x, 2 * H * D, x[:, H * D:], 2 * H * D, 0)


def test_fork_of_a_row_without_its_last_page_needs_no_free_page():
    P, pages, rows, width = 16, 2, 3, 4
    refs, lens = (torch.zeros(m, dtype=torch.int32, device=DEV) for m in (pages, rows))
    table = torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
    pool = (refs, pages, P, table, width, rows, lens)
    B.sqap_kv_alloc(*pool, ints([0]), ints([P + 1]), 1)
    pairs, granted = torch.empty((2, 2), dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    B.sqap_kv_fork(*pool, ints([0]), ints([1]), 1, pairs, granted)                 # the pool is used up
    assert granted[0] == 0 and pairs[0].tolist() == [-2, -2]
    table[0, 1] = -1
    B.sqap_kv_fork(*pool, ints([0, 0]), ints([1, 2]), 2, pairs, granted)
    assert granted.tolist() == [1, 1] and pairs.tolist() == [[-1, -1]] * 2
    assert table[1:].tolist() == [[0, -1, -1, -1]] * 2 and lens.tolist() == [P + 1] * 3 and refs.tolist() == [3, 1]


# ---------------------------------------------------------------------------------------------------------- zero values

@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("exponent", [-40, -30, -16, 8])
@pytest.mark.parametrize("D,new", [(64, [1, 1]), (128, [1, 1]), (128, [40, 24]), (64, [30, 9]), (256, [1, 1]), (256, [40, 24])])
def test_a_page_of_zero_values_leaves_the_weights_of_the_others_their_bits(D, new, exponent, kind):
    s = Setup([300, 130], 2, D, 32, kind, 11)
    s.scale["v"] = (2.0 ** exponent * (1 + s.g.random(s.scale["v"].shape))).astype(np.float32)
    for z in (s.table[0, 4], s.table[1, 1]):
        s.raw["v"][z] = 0
        s.scale["v"][z] = 0
    s.to_device()
    for gain in (0.3, 2.0):
        check_attention(s, new, 4, True, "bf16", q_gain=gain)


# ---------------------------------------------------------------------------------------------------------- the maxima

@pytest.mark.parametrize("D,new", [(64, [4, 1, 3]), (128, [2, 4, 1]), (128, [40, 33, 7]), (64, [20, 70, 9]), (256, [3, 1, 2]), (256, [40, 30, 9])])
def test_causal_attention_beyond_max_len(D, new):
    """Places from max_len on are not seen; which of the places in front of it a query sees does not change."""
    lens, heads, H, P = [100, 90, 64], 4, 2, 16
    s = Setup(lens, H, D, P, R.INT8, 5)
    q = dev(np.random.default_rng(1).standard_normal((2 + sum(new), heads * D)), torch.bfloat16)
    for max_len in (50, 64, 95):
        o, l, cu = run_attention(s, q, new, heads, True, "bf16", max_len=max_len)
        qn = q.double().cpu().numpy().reshape(-1, heads, D)
        for b, n in enumerate(lens):
            k, there = R.kv_tokens(s.codes("k"), s.scale["k"], s.table[b], n, P)
            v, _ = R.kv_tokens(s.codes("v"), s.scale["v"], s.table[b], n, P)
            there[max_len:] = False
            ref, lse, mag, pv, _ = R.attention(qn[cu[b]:cu[b + 1]], k, v, there, new[b], True, 1 / math.sqrt(D))
            d = 2.0 ** -19 * (1 + mag)
            got = o[cu[b]:cu[b + 1]].reshape(ref.shape)
            # (the scales of a head lie within 2^3 of one another here: no weight that counts is subnormal in fp16)
            assert (np.abs(got - ref) <= np.abs(ref) * 2.0 ** -8 + pv * (2.0 ** -10 + 2 * d[..., None])).all()
            gl, seen = l[cu[b]:cu[b + 1]], np.isfinite(lse)
            assert (gl[~seen] == -np.inf).all() and (np.abs(gl - lse)[seen] <= (d + 2.0 ** -20)[seen] + np.abs(lse[seen]) * 2.0 ** -22).all()


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("max_new", [1, 5, 16, 39])
def test_append_of_more_rows_than_max_new(max_new, kind):
    """The rows that are read go where they would go without the limit; the places of the others stay as they are."""
    new, lens, H, D, P = [40, 3, 20], [50, 20, 12], 2, 64, 16
    s = Setup(lens, H, D, P, kind, 8)
    cu = np.concatenate([[0], np.cumsum(new)])
    x = dev(s.g.standard_normal((sum(new), 2 * H * D)), torch.float16)
    B.sqap_kv_append(s.cache, s.dtable, s.width, 3, ints(lens), ints(cu), max_new, x, 2 * H * D, x[:, H * D:], 2 * H * D, 0)
    torch.cuda.synchronize()
    xn = x.float().cpu().numpy()
    for a, c0 in (("k", 0), ("v", H * D)):
        codes, scale = s.codes(a), s.scale[a].copy()
        for b in range(3):
            m = min(new[b], max_new)
            end = lens[b] - new[b] + m
            if end > 0:
                R.kv_append(codes, scale, s.table[b:b + 1], [end], [0, m], xn[cu[b]:cu[b] + m, c0:c0 + H * D].reshape(-1, H, D), kind, P)
        assert np.array_equal(s.device_codes(a), codes) and np.array_equal(s.ds[a].cpu().numpy(), scale)


# ---------------------------------------------------------------------------------------------------------- not-a-numbers

@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("D,lens,new", [(64, [40, 9], [1, 1]), (128, [3000, 70], [1, 1]), (128, [40, 60], [33, 20]), (64, [4000, 50], [20, 20]),
                                        (256, [40, 9], [1, 1]), (256, [3000, 50], [40, 33])])
def test_a_query_that_is_not_finite_spoils_its_own_row_alone(D, lens, new, bad):
    """... and says so in the log-sum-exp as well, whether the history is cut into pieces or not: -inf means that nothing is seen."""
    heads, H = 4, 2
    s = Setup(lens, H, D, 16, R.INT8, 5)
    rows = 2 + sum(new)
    good = dev(np.random.default_rng(1).standard_normal((rows, heads * D)), torch.float16)
    q = good.clone()
    q[2, D + 5] = bad                     # the first sequence's first query, head 1
    o0, l0, _ = run_attention(s, good, new, heads, True, "fp16")
    o, l, _ = run_attention(s, q, new, heads, True, "fp16")
    o0, o = (a[2:].reshape(-1, heads, D) for a in (o0, o))
    assert np.isnan(l[2, 1]) and np.isnan(o[0, 1]).all()
    l0[2, 1] = l[2, 1] = 0
    o0[0, 1] = o[0, 1] = 0
    assert np.array_equal(l, l0) and np.array_equal(o, o0)


@pytest.mark.parametrize("kind", [R.INT8, R.E4M3])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("D,n", [(64, 3), (64, 60), (128, 4), (128, 200), (256, 3), (256, 60)])
def test_a_token_that_is_not_finite_does_not_reach_queries_that_do_not_see_its_page(D, n, bad, dtype, kind):
    H, P, old = 2, 16, 14                  # the new tokens begin two places in front of a page
    g = np.random.default_rng(2)
    got = []
    rows = dev(g.standard_normal((n, 3 * H * D)), T[dtype])
    for what in (0.5, bad):
        s = Setup([old + n], H, D, P, kind, 4)
        x = rows.clone()
        x[2, H * D + 3] = x[2, 2 * H * D + 7] = what              # key and value of the first token of the second page
        cu, lens = ints([0, n]), ints([old + n])
        B.sqap_kv_append(s.cache, s.dtable, s.width, 1, lens, cu, n, x[:, H * D:], 3 * H * D, x[:, 2 * H * D:], 3 * H * D, CODE[dtype])
        out, lse = torch.empty((n, H * D), dtype=T[dtype], device=DEV), torch.empty((n, H), device=DEV)
        size = B.sqap_kv_attention_workspace_bytes(s.cache, 1, n, old + n, H)
        work = torch.empty(size + 16, dtype=torch.uint8, device=DEV)
        B.sqap_kv_attention(s.cache, s.dtable, s.width, 1, lens, cu, n, old + n, x, 3 * H * D, H, 0.1, 1, out, H * D, lse, CODE[dtype], work, size)
        torch.cuda.synchronize()
        got.append((out[:2].clone(), lse[:2].clone()))
    assert torch.isfinite(got[0][0]).all() and torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


# ------------------------------------------------------------------------------------------------- many items, threads

# more items of 256 rows than CTAs; items without an upper half, and sequences without rows, in front of full ones
@pytest.mark.parametrize("kind,dtype", [(R.INT8, "fp16"), (R.E4M3, "bf16")])
@pytest.mark.parametrize("heads,H,D,P,old,new", [
    (32, 32, 128, 64, [0, 300, 7, 500, 200, 0], [288, 20, 150, 1, 129, 0]),
    (32, 32, 64, 16, [0, 300, 7, 0, 200, 100], [288, 20, 150, 1, 129, 300]),
    (32, 8, 128, 32, [0, 300, 64, 500, 1, 90], [250, 3, 390, 30, 129, 5])])
def test_prompts_of_several_items_to_a_cta(heads, H, D, P, old, new, kind, dtype):
    s = Setup([a + b for a, b in zip(old, new)], H, D, P, kind, 17, nan_behind=True)
    for causal in (True, False):
        check_attention(s, new, heads, causal, dtype, seed=3)
    q = dev(np.random.default_rng(0).standard_normal((2 + sum(new), heads * D)), T[dtype])
    a, b = (run_attention(s, q, new, heads, True, dtype)[:2] for _ in range(2))
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    assert B.sqap_device_status() == B.SQAP_OK


def test_calls_from_two_host_threads():
    import threading
    H, D, P = 4, 128, 64
    sets, ref = [], []
    for i in range(2):
        s = Setup([1300, 200], H, D, P, R.INT8, 20 + i)
        x = dev(s.g.standard_normal((2, 3 * H * D)), torch.float16)
        n = B.sqap_kv_attention_workspace_bytes(s.cache, 2, 1, 1300, H)
        sets.append((s, x, ints(s.lens), ints([0, 1, 2]), torch.empty(2, H * D, dtype=torch.float16, device=DEV),
                     torch.empty(n, dtype=torch.uint8, device=DEV), n, torch.cuda.Stream()))

    def step(i):
        s, x, lens, cu, out, work, n, stream = sets[i]
        B.sqap_kv_append(s.cache, s.dtable, s.width, 2, lens, cu, 1, x[:, H * D:], 3 * H * D, x[:, 2 * H * D:], 3 * H * D, 0, stream)
        B.sqap_kv_attention(s.cache, s.dtable, s.width, 2, lens, cu, 1, 1300, x, 3 * H * D, H, 0.09, 1, out, H * D, None, 0, work, n, stream)

    torch.cuda.synchronize()
    for i in (0, 1):
        step(i)
        torch.cuda.synchronize()
        ref.append(sets[i][4].clone())
        sets[i][4].zero_()
    torch.cuda.synchronize()
    failed = []

    def work(i):
        try:
            for _ in range(200):
                step(i)
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed and all(torch.equal(sets[i][4], ref[i]) for i in (0, 1))


# ------------------------------------------------------------------------------------------------- the ends of the sizes

@pytest.mark.parametrize("D,heads,H,new,max_q", [(64, 4, 2, [5, 2], 3), (128, 12, 2, [9, 1], 4), (128, 4, 2, [40, 20], 33), (256, 2, 2, [7, 3], 5), (256, 2, 2, [60, 9], 40)])
def test_queries_beyond_max_q_are_left_out(D, heads, H, new, max_q):
    lens = [200, 70]
    s = Setup(lens, H, D, 16, R.E4M3, 5)
    cu = np.concatenate([[0], np.cumsum(new)])
    q = dev(np.random.default_rng(1).standard_normal((sum(new), heads * D)), torch.float16)
    got = []
    for m in (max(new), max_q):
        out = torch.full((sum(new), heads * D), 7.0, dtype=torch.float16, device=DEV)
        lse = torch.full((sum(new), heads), 7.0, device=DEV)
        size = B.sqap_kv_attention_workspace_bytes(s.cache, 2, m, 200, heads)
        work = torch.empty(size + 16, dtype=torch.uint8, device=DEV)
        B.sqap_kv_attention(s.cache, s.dtable, s.width, 2, ints(lens), ints(cu), m, 200, q, heads * D, heads, 0.1, 1, out, heads * D, lse, 0, work, size)
        torch.cuda.synchronize()
        got.append((out.double().cpu().numpy(), lse.cpu().numpy()))
    for b in range(2):
        m = min(new[b], max_q)
        mine, rest = slice(cu[b], cu[b] + m), slice(cu[b] + m, cu[b + 1])
        # (another kernel may have taken the shorter call: two roundings of the weights and of the output apart)
        assert (np.abs(got[0][0][mine] - got[1][0][mine]) <= 2.0 ** -9 * np.abs(s.codes("v")).max() * s.scale["v"].max()).all()
        assert np.allclose(got[0][1][mine], got[1][1][mine], rtol=0, atol=1e-3)
        assert (got[1][0][rest] == 7).all() and (got[1][1][rest] == 7).all()


@pytest.mark.parametrize("pages,free_every", [(16385, 1), (40000, 3), (100003, 17)])
def test_pool_of_many_pages(pages, free_every):
    """More pages than one step of the reserving kernels looks at."""
    g = np.random.default_rng(pages)
    refs_n = np.ones(pages, np.int32)
    refs_n[::free_every] = 0
    free = np.flatnonzero(refs_n == 0)
    rows, width, P = 300, 40, 16
    refs, lens = dev(refs_n), torch.zeros(rows, dtype=torch.int32, device=DEV)
    table = torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
    args = (refs, pages, P, table, width, rows, lens)
    need = g.integers(1, width, rows)
    add = need * P - g.integers(0, P, rows)
    granted = torch.empty(rows, dtype=torch.int32, device=DEV)
    B.sqap_kv_alloc(*args, ints(range(rows)), ints(add), rows, granted)
    torch.cuda.synchronize()
    upto = np.cumsum(need)
    ok = upto <= len(free)
    assert granted.cpu().numpy().tolist() == ok.astype(int).tolist() and ok.any()
    t = table.cpu().numpy()
    for r in range(rows):
        want = free[upto[r] - need[r]:upto[r]].tolist() if ok[r] else []
        assert t[r].tolist() == want + [-1] * (width - len(want))
    refs_n[free[:upto[ok][-1]]] = 1
    assert np.array_equal(refs.cpu().numpy(), refs_n) and np.array_equal(lens.cpu().numpy(), np.where(ok, add, 0))


def test_pool_of_as_many_rows_as_there_may_be():
    rows, width, P, pages = 16384, 3, 16, 20000
    refs, lens = torch.zeros(pages, dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    table = torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
    args = (refs, pages, P, table, width, rows, lens)
    half = rows // 2
    granted = torch.empty(rows, dtype=torch.int32, device=DEV)
    B.sqap_kv_alloc(*args, ints(range(rows)), ints([17 if r < half else 0 for r in range(rows)]), rows, granted)
    assert (granted == 1).all() and (lens[:half] == 17).all() and (lens[half:] == 0).all()
    assert torch.equal(table[:half, :2].flatten().cpu(), torch.arange(rows, dtype=torch.int32)) and (refs[:rows] == 1).all() and (refs[rows:] == 0).all()
    pairs = torch.empty((half, 2), dtype=torch.int32, device=DEV)
    B.sqap_kv_fork(*args, ints(range(half)), ints(range(half, rows)), half, pairs, granted)
    ok = pages - rows                                       # so many last pages are left to be copied
    assert granted[:half].tolist() == [1] * ok + [0] * (half - ok)
    assert pairs[:ok].tolist() == [[2 * i + 1, rows + i] for i in range(ok)] and (pairs[ok:] == -2).all()
    assert table[half:half + ok].tolist() == [[2 * i, rows + i, -1] for i in range(ok)]
    B.sqap_kv_free(*args, ints(range(rows)), rows)
    torch.cuda.synchronize()
    assert (refs == 0).all() and (lens == 0).all() and (table == -1).all()
