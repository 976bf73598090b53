"""What the microscaled 4-bit and key/value cache calls refuse, and the sizes they report. No kernel is launched."""
import numpy as np
import pytest

import lowbit_reference as R
from paper_2509_09090_b200 import binding as B


def test_mx4_scale_and_workspace_bytes():
    for rows, K in [(1, 32), (128, 64), (129, 64), (300, 11008), (1, 96)]:
        for fmt in (0, 1):
            nb = K // R.block(fmt)
            assert B.sqap_mx4_scale_bytes(rows, K, fmt) == -(-rows // 128) * -(-nb // 4) * 512
            n = B.sqap_mx4_workspace_bytes(rows, 64, K, fmt)
            assert n >= rows * K // 2 + B.sqap_mx4_scale_bytes(rows, K, fmt) and n % 256 == 0
    assert B.sqap_mx4_scale_bytes(0, 64, 0) == B.sqap_mx4_scale_bytes(4, 0, 0) == B.sqap_mx4_scale_bytes(4, 64, 2) == 0


def test_reference_scale_tiles_are_inverse():
    b = np.random.default_rng(0).integers(0, 256, (300, 11)).astype(np.uint8)
    assert np.array_equal(R.untile(R.tile(b), 300, 11), b)


INV, ALIGN, NOMEM, OK = B.SQAP_ERR_INVALID, B.SQAP_ERR_ALIGN, B.SQAP_ERR_NOMEM, B.SQAP_OK


@pytest.mark.parametrize("change,want", [
    (dict(M=0), OK), (dict(M=-1), INV), (dict(x=None), INV), (dict(codes=None), INV), (dict(scales=None), INV), (dict(K=0), INV),
    (dict(K=48), ALIGN), (dict(ldx=32), INV), (dict(ldx=68), ALIGN), (dict(x=8), ALIGN), (dict(codes=24), ALIGN),
    (dict(scales=8), ALIGN), (dict(dt=2), INV), (dict(dt=4), INV), (dict(fmt=2), INV), (dict(fmt=-1), INV)])
def test_mx4_quantize_refusals(change, want):
    a = dict(x=16, dt=0, M=4, K=64, ldx=64, ri=None, fmt=0, g=None, codes=16, scales=16, stream=None)
    a.update(change)
    assert B.lib().sqap_mx4_quantize(*a.values()) == want


@pytest.mark.parametrize("change,want", [
    (dict(M=0), OK), (dict(M=-1), INV), (dict(codes=None), INV), (dict(out=None), INV), (dict(K=40), ALIGN), (dict(ldo=32), INV),
    (dict(ldo=68), ALIGN), (dict(out=4), ALIGN), (dict(dt=2), INV), (dict(fmt=7), INV)])
def test_mx4_dequantize_refusals(change, want):
    a = dict(codes=16, scales=16, M=4, K=64, fmt=0, g=None, out=16, ldo=64, dt=1, stream=None)
    a.update(change)
    assert B.lib().sqap_mx4_dequantize(*a.values()) == want


@pytest.mark.parametrize("change,want", [
    (dict(M=0), OK), (dict(M=-1), INV), (dict(N=0), INV), (dict(K=0), INV), (dict(K=80), ALIGN), (dict(xc=None), INV),
    (dict(xs=None), INV), (dict(wc=None), INV), (dict(ws=None), INV), (dict(out=None), INV), (dict(xc=8), ALIGN), (dict(ws=4), ALIGN),
    (dict(ldo=64), INV), (dict(ldo=132), ALIGN), (dict(dt=2), INV), (dict(fmt=3), INV)])
def test_mx4_linear_refusals(change, want):
    a = dict(xc=16, xs=16, gx=None, M=4, wc=16, ws=16, gw=None, N=128, K=64, fmt=0, out=16, ldo=128, dt=0, stream=None)
    a.update(change)
    assert B.lib().sqap_mx4_linear(*a.values()) == want


@pytest.mark.parametrize("change,want", [
    (dict(M=0), OK), (dict(M=-1), INV), (dict(x=None), INV), (dict(xdt=2), INV), (dict(ldx=8), INV), (dict(ldx=65), ALIGN),
    (dict(work=None), INV), (dict(work=8), ALIGN), (dict(bytes=100), NOMEM), (dict(wc=None), INV), (dict(K=33), ALIGN)])
def test_mx4_quantize_linear_refusals(change, want):
    a = dict(x=16, xdt=0, M=4, ldx=64, ri=None, gx=None, wc=16, ws=16, gw=None, N=128, K=64, fmt=0, out=16, ldo=128, dt=0, work=16,
             bytes=1 << 20, stream=None)
    a.update(change)
    assert B.lib().sqap_mx4_quantize_linear(*a.values()) == want


# ------------------------------------------------------------------------------------------- 8-bit key/value cache
UNS = B.SQAP_ERR_UNSUPPORTED


def cache(**change):
    f = dict(k=16, v=16, k_scale=16, v_scale=16, pages=4, kv_heads=2, page_tokens=16, head_dim=64, type=0)
    f.update(change)
    return B._KvCacheStruct(**f)


BAD_CACHES = [(dict(k=None), INV), (dict(v_scale=None), INV), (dict(pages=-1), INV), (dict(kv_heads=0), INV), (dict(page_tokens=0), UNS),
              (dict(page_tokens=48), UNS), (dict(head_dim=0), INV), (dict(head_dim=96), UNS), (dict(type=2), INV), (dict(k=8), ALIGN),
              (dict(k_scale=6), ALIGN), (dict(kv_heads=65536), UNS)]


def call(name, c, a, change):
    a = dict(a)
    a.update(change)
    return getattr(B.lib(), name)(c, *a.values())


APPEND = dict(table=16, ldt=4, batch=2, lens=16, cu=16, max_new=3, k=16, ldk=128, v=16, ldv=128, dt=0, stream=None)
ATTEND = dict(table=16, ldt=4, batch=2, lens=16, cu=16, max_q=3, max_len=64, q=16, ldq=256, heads=4, scale=0.1, flags=1, out=16,
              ldo=256, lse=None, dt=0, work=None, bytes=0, stream=None)
READ = dict(table=16, ldt=4, batch=2, first=None, cu=16, max_rows=3, k=16, ldk=128, v=16, ldv=128, dt=0, stream=None)
COPY = dict(pairs=16, n=3, stream=None)
COMPACT = dict(table=16, ldt=4, rows=4, lens=16, src=16, dst=16, n=2, kept=16, ldkept=8, nk=16, mk=8, stream=None)


@pytest.mark.parametrize("name,args", [("sqap_kv_append", APPEND), ("sqap_kv_attention", ATTEND), ("sqap_kv_read", READ),
                                       ("sqap_kv_copy_pages", COPY), ("sqap_kv_compact", COMPACT)])
def test_kv_calls_refuse_bad_caches(name, args):
    for change, want in BAD_CACHES:
        assert call(name, cache(**change), args, {}) == want, change
    assert call(name, None, args, {}) == INV


@pytest.mark.parametrize("name,args,change,want", [
    ("sqap_kv_append", APPEND, dict(batch=0), OK), ("sqap_kv_append", APPEND, dict(max_new=0), OK),
    ("sqap_kv_append", APPEND, dict(batch=-1), INV), ("sqap_kv_append", APPEND, dict(table=None), INV),
    ("sqap_kv_append", APPEND, dict(lens=None), INV), ("sqap_kv_append", APPEND, dict(cu=None), INV),
    ("sqap_kv_append", APPEND, dict(k=None), INV), ("sqap_kv_append", APPEND, dict(v=8), ALIGN),
    ("sqap_kv_append", APPEND, dict(ldk=64), INV), ("sqap_kv_append", APPEND, dict(ldv=132), ALIGN),
    ("sqap_kv_append", APPEND, dict(dt=3), INV), ("sqap_kv_append", APPEND, dict(ldt=-1), INV),
    ("sqap_kv_append", APPEND, dict(ldt=1 << 40), INV), ("sqap_kv_append", APPEND, dict(batch=1 << 30, max_new=1 << 20), UNS),
    ("sqap_kv_attention", ATTEND, dict(batch=0), OK), ("sqap_kv_attention", ATTEND, dict(max_q=0), OK),
    ("sqap_kv_attention", ATTEND, dict(max_q=-1), INV), ("sqap_kv_attention", ATTEND, dict(max_len=-1), INV),
    ("sqap_kv_attention", ATTEND, dict(heads=3), INV), ("sqap_kv_attention", ATTEND, dict(heads=0), INV),
    ("sqap_kv_attention", ATTEND, dict(scale=float("nan")), INV), ("sqap_kv_attention", ATTEND, dict(scale=float("inf")), INV),
    ("sqap_kv_attention", ATTEND, dict(flags=2), INV), ("sqap_kv_attention", ATTEND, dict(q=None), INV),
    ("sqap_kv_attention", ATTEND, dict(out=8), ALIGN), ("sqap_kv_attention", ATTEND, dict(ldq=128), INV),
    ("sqap_kv_attention", ATTEND, dict(ldo=257), ALIGN), ("sqap_kv_attention", ATTEND, dict(lse=18), ALIGN),
    ("sqap_kv_attention", ATTEND, dict(dt=2), INV), ("sqap_kv_attention", ATTEND, dict(lens=None), INV),
    ("sqap_kv_attention", ATTEND, dict(max_len=4096), INV), ("sqap_kv_attention", ATTEND, dict(max_len=4096, work=16, bytes=64), NOMEM),
    ("sqap_kv_attention", ATTEND, dict(max_len=4096, work=8, bytes=1 << 30), ALIGN),
    ("sqap_kv_attention", ATTEND, dict(max_len=(1 << 30) + 1), UNS), ("sqap_kv_attention", ATTEND, dict(max_q=1 << 30), UNS),
    ("sqap_kv_read", READ, dict(batch=0), OK), ("sqap_kv_read", READ, dict(k=None, v=None), OK), ("sqap_kv_read", READ, dict(cu=None), INV),
    ("sqap_kv_read", READ, dict(ldk=100), INV), ("sqap_kv_read", READ, dict(ldv=129), ALIGN), ("sqap_kv_read", READ, dict(v=4), ALIGN),
    ("sqap_kv_read", READ, dict(max_rows=-1), INV), ("sqap_kv_read", READ, dict(dt=7), INV),
    ("sqap_kv_copy_pages", COPY, dict(n=0), OK), ("sqap_kv_copy_pages", COPY, dict(n=-1), INV),
    ("sqap_kv_copy_pages", COPY, dict(pairs=None), INV), ("sqap_kv_copy_pages", COPY, dict(pairs=12), ALIGN),
    ("sqap_kv_compact", COMPACT, dict(n=0), OK), ("sqap_kv_compact", COMPACT, dict(mk=0), OK), ("sqap_kv_compact", COMPACT, dict(ldkept=4), INV),
    ("sqap_kv_compact", COMPACT, dict(kept=None), INV), ("sqap_kv_compact", COMPACT, dict(rows=-1), INV),
    ("sqap_kv_compact", COMPACT, dict(n=1 << 30, mk=1 << 20, ldkept=1 << 20), UNS)])
def test_kv_refusals(name, args, change, want):
    assert call(name, cache(), args, change) == want


POOL = dict(refs=16, pages=8, P=16, table=16, ldt=4, rows=4, lens=16)


@pytest.mark.parametrize("name,rest", [("sqap_kv_alloc", dict(list=16, add=16, n=2, granted=None, stream=None)),
                                       ("sqap_kv_fork", dict(src=16, dst=16, n=2, pairs=16, granted=None, stream=None)),
                                       ("sqap_kv_free", dict(list=16, n=2, stream=None))])
def test_pool_refusals(name, rest):
    f = getattr(B.lib(), name)
    for change, want in [(dict(refs=None), INV), (dict(pages=-1), INV), (dict(P=24), UNS), (dict(table=None), INV), (dict(ldt=-1), INV),
                         (dict(rows=-1), INV), (dict(rows=16385), UNS), (dict(lens=None), INV), (dict(n=-1), INV), (dict(n=0), OK),
                         (dict(n=16385), UNS)]:
        a = {**POOL, **rest, **change}
        assert f(*a.values()) == want, change
    for key in ("list", "add", "src", "dst", "pairs"):
        if key in rest:
            assert f(*{**POOL, **rest, key: None}.values()) == INV
    if "pairs" in rest:
        assert f(*{**POOL, **rest, "pairs": 12}.values()) == ALIGN


def test_attention_workspace_bytes():
    n = B.lib().sqap_kv_attention_workspace_bytes
    assert n(cache(), 4, 1, 200, 2) == 0                      # short: not cut into pieces
    assert n(cache(), 1, 1, 16384, 2) % 16 == 0 and n(cache(), 1, 1, 16384, 2) > 0
    assert n(cache(), 0, 1, 4096, 2) == n(cache(), 1, 0, 4096, 2) == n(cache(), 1, 1, 4096, 3) == n(cache(type=5), 1, 1, 4096, 2) == 0
    assert n(cache(), 1, 1, 4096, 8) == 4 * n(cache(), 1, 1, 4096, 2)      # the pieces depend on the key/value heads alone


def test_kv_cache_wrapper_checks_its_tensors():
    torch = pytest.importorskip("torch")
    k = torch.zeros(3, 2, 16, 64, dtype=torch.int8)
    s = torch.zeros(3, 2)
    assert B.KvCache(k, k, s, s, 0).struct.pages == 3
    for bad in [(k, k[:2], s, s), (k, k, s[:, :1], s), (k.half(), k, s, s), (k, k, s.half(), s), (k, k.transpose(0, 1).contiguous().transpose(0, 1), s, s)]:
        with pytest.raises(ValueError):
            B.KvCache(*bad, 0)
