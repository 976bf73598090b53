"""Sizes whose products pass 64 bits are refused like all that are too large. No kernel is launched."""
import pytest

from paper_2509_09090_b200 import binding as B
from test_lowbit_host import APPEND, ATTEND, COMPACT, COPY, READ, cache, call

BIG = 1 << 30


# each product of sizes is a multiple of 2^64, or passes 2^63
@pytest.mark.parametrize("name,args,heads,change", [
    ("sqap_kv_append", APPEND, 32768, dict(batch=BIG, max_new=BIG)),
    ("sqap_kv_append", APPEND, 65535, dict(batch=2 * BIG - 1, max_new=2 * BIG - 1)),
    ("sqap_kv_read", READ, 32768, dict(batch=BIG, max_rows=2 * BIG - 15)),
    ("sqap_kv_read", READ, 65535, dict(batch=2 * BIG - 1, max_rows=2 * BIG - 1)),
    ("sqap_kv_copy_pages", COPY, 65535, dict(n=2 * BIG - 1)),
    ("sqap_kv_compact", COMPACT, 32768, dict(n=BIG, mk=BIG, ldkept=BIG)),
    ("sqap_kv_compact", COMPACT, 65535, dict(n=2 * BIG - 1, mk=2 * BIG - 1, ldkept=2 * BIG)),
    ("sqap_kv_attention", ATTEND, 32768, dict(batch=BIG, max_q=BIG, heads=32768)),
    ("sqap_kv_attention", ATTEND, 65535, dict(batch=2 * BIG - 1, max_q=BIG, heads=65535)),
    ("sqap_kv_attention", ATTEND, 1, dict(batch=2 * BIG - 1, max_q=1, max_len=BIG, heads=BIG)),
    ("sqap_kv_attention", ATTEND, 32768, dict(batch=BIG, max_q=1, max_len=BIG, heads=32768))])
def test_sizes_beyond_64_bits_are_refused(name, args, heads, change):
    wide = {k: heads * 256 for k in ("ldk", "ldv") if k in args}
    if "ldq" in args:
        wide = {k: change["heads"] * 64 for k in ("ldq", "ldo")}
    before = B.sqap_kernel_launch_count()
    assert call(name, cache(kv_heads=heads), {**args, **wide}, change) == B.SQAP_ERR_UNSUPPORTED
    assert B.sqap_kernel_launch_count() == before


def test_workspace_of_sizes_beyond_64_bits():
    n = B.lib().sqap_kv_attention_workspace_bytes
    assert n(cache(), 2 * BIG - 1, 2 * BIG - 1, 2 * BIG - 1, 2 * BIG - 2) == 0
    assert n(cache(kv_heads=65535), 2 * BIG - 1, 1, BIG, 65535) == 0
