"""Eviction by received weight: the list equals the plain statement's. Rotary positions against 64 bits: with a, b the pair and y the
turned element, |y| eps / 2 for the output's rounding and 2^-20 (|a| + |b|) for the rest: two fp32 products and a sum (2^-24 each), the sine
and cosine (2^-22), and the angle, rounded in fp32 within a turn (2^-22.3) and in 64 bits before (2^31 radians: 2^-21.7)."""
import math

import numpy as np
import pytest

import cache_reference as C

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from paper_2509_09090_b200 import binding as B
    from test_gpu_kv import CODE, DEV, T, dev, ints


def check_evict(mass, lens, src, keep, first, recent, room=None, dst=None, max_len=None):
    rows, ldm = mass.shape
    room = max(max(keep), 1) if room is None else room
    max_len = max(list(lens) + [0]) if max_len is None else max_len
    d = dev(mass.copy())
    kept = torch.full((len(src) + 1, max(room, 1)), -9, dtype=torch.int32, device=DEV)
    count = torch.full((len(src) + 1,), -9, dtype=torch.int32, device=DEV)
    B.sqap_kv_evict(d, ldm, rows, ints(lens), ints(src), None if dst is None else ints(dst), len(src), ints(keep), first, recent, max_len, kept, room,
                    count)
    torch.cuda.synchronize()
    want = C.evict(mass, lens, src, keep, first, recent, max_len, room)
    k, c = kept.cpu().numpy(), count.cpu().numpy()
    assert (k[len(src):] == -9).all() and c[-1] == -9
    after = mass.copy()
    for i, w in enumerate(want):
        assert c[i] == len(w)
        if room:
            assert k[i, :len(w)].tolist() == w and (k[i, len(w):] == -1).all()
        if dst is not None and 0 <= dst[i] < rows:
            after[dst[i], :len(w)] = mass[src[i], w]
    assert np.array_equal(d.cpu().numpy(), after, equal_nan=True)


def weights(g, rows, width):
    m = np.exp(3 * g.standard_normal((rows, width)))
    u = g.random((rows, width))
    return np.where(u < 0.15, 0, np.where(u < 0.4, np.rint(2 * m) / 2, m)).astype(np.float32)


@pytest.mark.parametrize("n", [1, 2, 31, 255, 256, 257, 1023, 1024, 1025, 4095, 4096, 4097, 16384, 16385, 40000])
def test_evict_lengths(n):
    g = np.random.default_rng(n)
    lens = [n, n // 2, 0, max(1, n - 1), 0, 0, 0, 0]
    m = weights(g, 8, n + 5)
    for keep, first, recent in [(max(1, n // 3), 1, 4), (n, 0, 0), (1, 0, 0), (max(1, n - 1), 4, 300), (max(1, n // 2), 0, 0)]:
        check_evict(m, lens, [0, 1, 2, 3], [keep] * 4, first, recent, dst=[4, 5, 6, 7])


@pytest.mark.parametrize("n,top", [(20, 9000), (30, 20000), (37, 16384), (38, 16385), (64, 5000), (74, 20001), (75, 9000), (150, 33000)])
def test_evict_many_sequences(n, top):
    """As many CTAs to a sequence as the number of sequences leaves room for: eight, four, two, one; in one round and in several."""
    g = np.random.default_rng(n)
    m = weights(g, 2 * n, top)
    lens = [int(x) for x in g.integers(0, top + 1, n)] + [0] * n
    lens[0] = top
    check_evict(m, lens, list(range(n)), [int(x) for x in g.integers(0, top // 2, n)], 3, 70, dst=list(range(n, 2 * n)), max_len=top)


@pytest.mark.parametrize("keep,first,recent", [(0, 5, 5), (3, 5, 5), (7, 5, 5), (10, 5, 5), (11, 5, 5), (100, 0, 200), (100, 200, 0), (150, 3, 0), (2, 0, 0)])
def test_evict_what_is_always_kept(keep, first, recent):
    g = np.random.default_rng(keep)
    check_evict(weights(g, 3, 200), [150, 8, 200], [0, 1, 2], [keep] * 3, first, recent)


@pytest.mark.parametrize("fill", [0.0, 1.0, -1.0, math.inf, -math.inf, math.nan, 2.0 ** -140])
def test_evict_equal_weights_stay_in_their_order(fill):
    m = np.full((2, 700), fill, np.float32)
    check_evict(m, [700, 650], [0, 1], [123, 123], 2, 10)
    m[0, 300:400] = 2.0
    m[1, ::7] = -0.0
    check_evict(m, [700, 650], [0, 1], [123, 123], 2, 10)


def test_evict_every_kind_of_number():
    g = np.random.default_rng(0)
    m = g.integers(0, 2 ** 32, (4, 3000), dtype=np.uint32).view(np.float32).copy()
    m[1, ::3] = np.nan
    m[2, ::5], m[2, 1::5] = np.inf, -np.inf
    m[3] = np.float32(1) + np.arange(3000, dtype=np.float32)[::-1] * 2.0 ** -23      # neighbours
    with np.errstate(invalid="ignore"):
        for keep in (1, 100, 1500, 2999):
            check_evict(m, [3000, 2999, 2000, 3000], [0, 1, 2, 3], [keep] * 4, 0, 0)


def test_evict_rows_and_room():
    """Rows that do not exist, the same source twice, budgets of any sign, less room than the budget, lengths beyond the weights."""
    g = np.random.default_rng(1)
    m = weights(g, 6, 96)
    lens = [90, 96, 500, -4, 0, 0]
    check_evict(m, lens, [0, -1, 6, 0, 2, 3], [10, 10, 10, 20, 96, 5], 1, 2, dst=[4, 5, -1, 9, -1, -1])
    check_evict(m, lens, [0, 1], [50, -3], 1, 2, room=7, max_len=96)
    check_evict(m, lens, [0, 1], [50, 50], 1, 2, max_len=40)
    check_evict(m, lens, [0, 1], [50, 50], 1, 2, max_len=0)
    check_evict(m, lens, [0, 1], [50, 50], 1, 2, room=0, max_len=96)
    check_evict(m, lens, [1], [5], 2 ** 31 - 1, 2 ** 31 - 1, max_len=96)


# -------------------------------------------------------------------------------------------------------------- rotary

def check_rotary(dtype, rows, heads, D, rot, axes, axis_of, neighbours, positions, pad=16, in_place=False, seed=0):
    g = np.random.default_rng(seed)
    x = dev(g.standard_normal((rows + 1, heads * D + pad)) * 3, T[dtype])
    freq = (1e4 ** (-2 * np.arange(rot // 2) / rot)).astype(np.float32)
    pos = np.zeros((axes, rows + 3), np.int32)
    pos[:, :rows] = positions
    xin = x.clone()
    out = x if in_place else torch.full((rows + 1, heads * D + 24), 3.0, dtype=T[dtype], device=DEV)
    B.sqap_rotary(x, x.stride(0), rows, heads, D, rot, ints(pos), rows + 3, axes, None if axis_of is None else bytes(axis_of), dev(freq),
                  B.SQAP_ROTARY_NEIGHBOURS if neighbours else 0, out, out.stride(0), CODE[dtype])
    torch.cuda.synchronize()
    a = xin.double().cpu().numpy()[:rows, :heads * D].reshape(rows, heads, D)
    ref = C.rotary(a, pos[:, :rows], np.zeros(rot // 2, int) if axis_of is None else np.asarray(axis_of, int), freq, neighbours)
    got = out.double().cpu().numpy()
    i = np.arange(rot // 2)
    lo, hi = (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)
    size = np.zeros_like(a)
    size[..., lo] = size[..., hi] = np.abs(a[..., lo]) + np.abs(a[..., hi])
    fi = torch.finfo(T[dtype])
    tol = np.abs(ref) * fi.eps / 2 + 2.0 ** -20 * size + float(fi.smallest_normal) * fi.eps
    tol[..., rot:] = 0
    err = np.abs(got[:rows, :heads * D].reshape(ref.shape) - ref)
    assert (err <= tol).all(), (err / np.maximum(tol, 1e-30)).max()
    keep = xin.double().cpu().numpy() if in_place else np.full_like(got, 3.0)
    assert np.array_equal(got[rows:], keep[rows:]) and np.array_equal(got[:, heads * D:], keep[:, heads * D:])


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype,rows,heads,D,rot", [
    ("fp16", 1, 1, 64, 64), ("bf16", 16, 64, 128, 128), ("fp16", 300, 12, 72, 72), ("bf16", 77, 5, 80, 40), ("fp16", 33, 3, 256, 256),
    ("bf16", 500, 1, 128, 64), ("fp16", 9, 40, 128, 8), ("bf16", 2000, 8, 256, 248), ("fp16", 5, 2, 8, 8), ("bf16", 3000, 1, 16, 8),
    ("fp16", 1500, 64, 128, 128)])
def test_rotary(dtype, rows, heads, D, rot, neighbours):
    g = np.random.default_rng(rows)
    axis_of = [i % 3 for i in range(rot // 2)]
    pos = g.integers(0, 300, (3, rows))
    check_rotary(dtype, rows, heads, D, rot, 3, axis_of, neighbours, pos)
    check_rotary(dtype, rows, heads, D, rot, 1, None, neighbours, g.integers(-2000, 2000, (1, rows)), pad=0, in_place=True)


@pytest.mark.parametrize("top", [2 ** 20, 2 ** 31])
def test_rotary_far_positions(top):
    g = np.random.default_rng(1)
    pos = g.integers(-top, top, (8, 200))
    pos[:, 0], pos[:, 1], pos[:, 2] = 0, top - 1, -top
    check_rotary("fp16", 200, 4, 128, 128, 8, [i % 8 for i in range(64)], False, pos)


def test_rotary_is_undone_by_the_opposite_positions():
    x = torch.randn(50, 512, device=DEV).to(torch.bfloat16)
    freq = torch.tensor([100.0 ** (-i / 32) for i in range(32)], device=DEV)
    pos = torch.arange(50, dtype=torch.int32, device=DEV).reshape(1, 50) * 1001
    y, z = torch.empty_like(x), torch.empty_like(x)
    B.sqap_rotary(x, 512, 50, 8, 64, 64, pos, 50, 1, None, freq, 0, y, 512, 1)
    B.sqap_rotary(y, 512, 50, 8, 64, 64, -pos, 50, 1, None, freq, 0, z, 512, 1)
    torch.cuda.synchronize()
    size = x.abs().float()
    pair = (size.reshape(50, 8, 2, 32) ** 2).sum(2, keepdim=True).sqrt().expand(-1, -1, 2, -1).reshape(50, 512)
    # two roundings to bf16, the first of which (of either element of the pair, 2^-8 of its value) is turned back
    assert ((z.float() - x.float()).abs() <= pair * (2.0 ** -8 * math.sqrt(2) + 2.0 ** -8 + 2.0 ** -10)).all()


@pytest.mark.parametrize("width", [96, 4097, 16384, 40000])
def test_evict_into_the_source_itself(width):
    """An entry whose destination is its own source chooses its tokens, and moves no weights."""
    m = weights(np.random.default_rng(width), 2, width)
    keep = width // 3
    d, kept = dev(m.copy()), torch.zeros((2, keep), dtype=torch.int32, device=DEV)
    count = torch.zeros(2, dtype=torch.int32, device=DEV)
    B.sqap_kv_evict(d, width, 2, ints([width, width - 5]), ints([0, 1]), ints([0, 1]), 2, ints([keep, keep]), 4, 9, width, kept, keep, count)
    torch.cuda.synchronize()
    assert kept.tolist() == C.evict(m, [width, width - 5], [0, 1], [keep, keep], 4, 9, width, keep)
    assert count.tolist() == [keep, keep] and np.array_equal(d.cpu().numpy(), m)
