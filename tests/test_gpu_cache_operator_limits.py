"""The operators around the cache at their limits: shares of a long sequence of which every token stays, more tokens than a launch was sized
for. Lists are whole numbers and equal the plain statement's; tolerances of outputs are those of the single operators
(test_gpu_kv_views.py)."""
import math

import numpy as np
import pytest

import cache_reference as C
import lowbit_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B
    from test_gpu_evict_rotary import check_evict, weights
    from test_gpu_kv import DEV, Setup, ints
    from test_gpu_kv_views import GUARD, Group, Queries, check_mass, check_rows, check_shared, run_window, scratch, tokens_of


@pytest.mark.parametrize("n,top,share", [(3, 8192, 4096), (5, 16384, 4096), (37, 14000, 4096), (2, 32768, 4096), (40, 33000, 16384), (20, 40000, 16384),
                                         (2, 131072, 16384), (41, 70000, 16384)])
def test_evict_where_all_of_a_share_stays(n, top, share):
    """Two, four and eight CTAs to a sequence, 4096 or 16384 tokens each and round: first or last tokens that fill a CTA's share, or leave it one token
    to choose from, beside sequences of which some CTAs have none."""
    g = np.random.default_rng(n + top)
    m = weights(g, n + 4, top + 3)
    lens = ([top, share + 1, 10, 2 * share - 5] + [0] * n)[:n] + [0] * 4
    lens[n - 1] = top - 1
    for first, recent in [(0, share - 1), (0, share), (0, share + 1), (share - 1, 0), (share, 0), (share + 1, 4), (4, share + 100), (share, share - 300),
                          (1, top - 700), (top - 700, 1)]:
        free = max(top - first - recent, 0)
        for keep in {first + recent + 1, first + recent + free // 3, top - 1}:
            check_evict(m, lens, list(range(n)), [keep] * n, first, recent, dst=[n, n + 1] + [-1] * (n - 3) + [n + 2] if n > 2 else [n, n + 2], max_len=top)


@pytest.mark.parametrize("max_len,window,sinks", [(1000, 100, 16), (1000, 100, 0), (1000, 2500, 5), (999, 1, 1200), (64, 7, 64), (1700, 300, 900)])
@pytest.mark.parametrize("kind,dtype,heads,H,D,P,lens,new", [
    (R.INT8, "fp16", 2, 2, 64, 16, [2600, 1000, 30, 1120], [1, 1, 1, 1]),
    (R.E4M3, "bf16", 8, 2, 128, 64, [2600, 1001, 1150], [1, 1, 1]),
    (R.E4M3, "fp16", 4, 1, 128, 32, [2600, 1040], [4, 3]),
    (R.INT8, "bf16", 3, 1, 256, 128, [2600, 1090, 999], [1, 2, 1]),
    (R.INT8, "fp16", 2, 2, 64, 16, [2600, 1030, 0], [300, 100, 30]),
    (R.E4M3, "bf16", 8, 2, 128, 64, [2600, 1100], [129, 200]),
    (R.E4M3, "fp16", 2, 2, 256, 128, [2600, 1033], [150, 40])])
def test_sinks_of_histories_beyond_max_len_stay_visible(kind, dtype, heads, H, D, P, lens, new, max_len, window, sinks):
    """A window that lies behind max_len holds no token that is looked at; the first tokens are seen all the same."""
    s = Setup(lens, H, D, P, kind, seed=max_len + D)
    qs = Queries(s, new, heads, dtype, seed=window)
    run_window(s, qs, new, window, sinks, lens, max_len=max_len)
    o, l = qs.results([(qs.cu[0], qs.cu[-1])])
    for b, n in enumerate(lens):
        r, held = slice(qs.cu[b], qs.cu[b + 1]), min(n, max_len)
        check_rows(s, o[r], l[r], qs.qn[r], *tokens_of(s, s.table[b], held), C.in_window(n, new[b], window, sinks)[:, :held], dtype, 1 / math.sqrt(D))


@pytest.mark.parametrize("dtype,heads,H,D,P,sizes,prefixes,own", [
    ("fp16", 2, 2, 64, 16, [8, 8], [2000, 0], [5] * 8 + [2005 - 70 * b for b in range(8)]),                  # one tile of rows to a group
    ("bf16", 4, 1, 128, 64, [6, 3, 1], [1600, 100, 0], [9, 1, 30, 4, 5, 6, 1500, 7, 800, 1601]),             # three
    ("fp16", 128, 32, 64, 16, [20, 19], [600, 0], [30] * 20 + [620 - 31 * b for b in range(19)]),            # prefix in a launch of its own, tiles of rows
    ("bf16", 8, 1, 128, 64, [40, 3], [1500, 0], [7] * 40 + [1507, 900, 1]),                                  # the same, a sequence to a CTA
    ("fp16", 2, 1, 256, 16, [7, 5], [900, 3], [4] * 7 + [850, 3, 777, 901, 90])])
def test_prefixes_of_very_uneven_lengths(dtype, heads, H, D, P, sizes, prefixes, own):
    """Own tokens behind a short prefix are as many as the longest prefix lets no group have."""
    check_shared(Group(sizes, prefixes, own, H, D, P, R.INT8, seed=sum(own)), [1] * len(own), heads, dtype)


@pytest.mark.parametrize("rows,heads,D,rot", [(2, 70_000_000, 8, 8), (1, 70_000_000, 24, 8)])
def test_rotary_of_very_many_heads(rows, heads, D, rot):
    """31 times the heads pass 31 bits. Tolerance: that of the other rotary tests (test_gpu_evict_rotary.py)."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    x = torch.randn((rows, heads * D), device=DEV, dtype=torch.float16)
    out = torch.full_like(x, 3.0)
    freq = torch.tensor([1.0, 0.1, 0.01, 0.001], device=DEV)
    at = torch.tensor([[5, 77]], device=DEV, dtype=torch.int32)
    B.sqap_rotary(x, heads * D, rows, heads, D, rot, at, 2, 1, None, freq, 0, out, heads * D, 0)
    torch.cuda.synchronize()
    for row in range(rows):
        angle = at[0, row].double() * freq.double()
        c, s = angle.cos(), angle.sin()
        for h in range(0, heads, 8_000_000):
            a, y = (t[row].view(heads, D)[h:h + 8_000_000] for t in (x, out))
            p, q = a[:, :4].double(), a[:, 4:8].double()
            size = 2.0 ** -20 * (p.abs() + q.abs()) + 2.0 ** -24
            for ref, got in ((p * c - q * s, y[:, :4]), (q * c + p * s, y[:, 4:8])):
                assert ((got.double() - ref).abs() <= ref.abs() * 2.0 ** -11 + size).all()
            assert torch.equal(a[:, 8:], y[:, 8:])


def test_rows_of_queries_beyond_32_bit_offsets():
    """2^24 + 16 heads of 128 on one key/value head: all but the last 16, which lie beyond 2^31 elements, see token 69 alone (the others' weights are
    below 2^-300). Its received weight is 2^24 and a sum of 16 weights: an addition at 2^22, where each of four lanes is by then, is off by 2^-2 at
    most, one of the three that join the lanes by 1."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    D, n, heads, more = 128, 70, (1 << 24) + 16, 16
    s = Setup([n], 1, D, 128, R.INT8, seed=7)
    page = s.table[0, 0]
    s.raw["k"][page, 0, :, :64] = np.int8(-100).view(np.uint8)
    s.raw["k"][page, 0, n - 1, :64] = 100
    s.scale["k"][:] = 1 / 40
    s.to_device()
    g = np.random.default_rng(1)
    last = np.concatenate([np.zeros((more, 64)), g.standard_normal((more, 64))], 1)
    q = torch.zeros((heads, D), device=DEV, dtype=torch.float16)
    q[:, :64] = 8.0
    q[-more:] = torch.from_numpy(last).to(DEV).half()
    out, lse = torch.full_like(q, GUARD), torch.full((heads,), GUARD, device=DEV)
    mass = torch.full((n,), GUARD, device=DEV)
    ld, scale = heads * D, 1 / math.sqrt(D)
    size = B.sqap_kv_attention_mass_workspace_bytes(s.cache, 1, 1, n, heads, 1)
    B.sqap_kv_attention_mass(s.cache, s.dtable, s.width, 1, ints([n]), ints([0, 1]), 1, n, q, ld, heads, scale, 1, 1, out, ld, lse, None, mass, n, 0,
                             scratch(size), size)
    torch.cuda.synchronize()
    assert B.sqap_device_status() == B.SQAP_OK
    k, (v, vs), there = tokens_of(s, s.table[0], n)
    seen = np.ones((1, n), bool)
    for at in (0, 12345678, heads - more - 40, heads - more):
        rows = slice(at, at + more)
        o, l, x = (t[rows].double().cpu().numpy() for t in (out, lse, q))
        p, need = check_rows(s, o[None], l[None], x[None], k, (v, vs), there, seen, "fp16", scale)
    m = mass.double().cpu().numpy()
    p, need = p[0], (p * need[..., None])[0]
    assert (np.abs(m - p.sum(0)) <= need.sum(0) + more * 2.0 ** -24 * p.sum(0) + 2.0 ** -126)[:-1].all()
    assert abs(m[-1] - (1 << 24) - p[:, -1].sum()) <= need[:, -1].sum() + more / 4 + 3


@pytest.mark.parametrize("dtype,heads,H,D,P,lens,new", [
    ("fp16", 9, 9, 64, 16, [60, 9, 290], [9, 9, 9]),                   # more than eight heads, 9 to 16 rows of each
    ("bf16", 20, 10, 128, 64, [33, 300], [5, 4]), ("fp16", 48, 12, 64, 16, [100, 3], [3, 2]), ("bf16", 126, 9, 64, 32, [70], [2]),
    ("fp16", 9, 9, 64, 32, [2049, 700], [9, 1]),                       # long histories
    ("bf16", 15, 1, 64, 16, [400, 30], [1, 1]), ("fp16", 12, 4, 128, 64, [290, 31], [4, 5]),      # eight heads or fewer
    ("fp16", 16, 1, 128, 16, [500, 40], [1, 1]), ("bf16", 4, 1, 64, 64, [2300, 100], [4, 3])])    # 16 rows
def test_received_weights_of_up_to_16_rows(dtype, heads, H, D, P, lens, new):
    """Either side of the rule by which scores are kept or computed again."""
    for kind in (R.INT8, R.E4M3):
        s = Setup(lens, H, D, P, kind, seed=heads + D)
        for last_q, past in ((max(new), "given"), (1, "same"), (2, "none")):
            check_mass(s, new, heads, dtype, last_q, past=past)
        check_mass(s, new, heads, dtype, max(new), causal=False, max_len=max(lens) - 7, ldm=max(lens) - 3)
        check_mass(s, new, heads, dtype, max(new), spoil=0)
