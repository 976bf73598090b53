"""What the operators around the key/value cache refuse, and the sizes they report. No kernel is launched."""
import pytest

from paper_2509_09090_b200 import binding as B
from test_lowbit_host import ALIGN, ATTEND, BAD_CACHES, INV, NOMEM, OK, UNS, cache, call

BIG = 1 << 30
HISTORY = dict(table=16, ldt=4, batch=2, lens=16, cu=16, max_q=3, max_len=64)
Q = dict(q=16, ldq=256, heads=4, scale=0.1)
REST = dict(out=16, ldo=256, lse=None, dt=0, work=None, bytes=0, stream=None)
WINDOW = {**HISTORY, **Q, **dict(window=8, sinks=1), **REST}
SHARED = {**HISTORY, **dict(cu_group=16, groups=1, max_group=64, prefix=16, max_prefix=64), **Q, **dict(flags=1), **REST}
MASS = {**HISTORY, **Q, **dict(flags=1, last_q=1, out=16, ldo=256, lse=16, past=None, mass=16, ldm=64, dt=0, work=16, bytes=1 << 20, stream=None)}
SHARED_BYTES = 2 * 4 * 3 * 2 * (64 * 4 + 8)        # rows x pieces


@pytest.mark.parametrize("name,args", [("sqap_kv_attention_window", WINDOW), ("sqap_kv_attention_shared", SHARED), ("sqap_kv_attention_mass", MASS)])
def test_bad_caches(name, args):
    for change, want in BAD_CACHES:
        assert call(name, cache(**change), args, {}) == want, change
    assert call(name, None, args, {}) == INV


COMMON = [(dict(batch=0), OK), (dict(max_q=0), OK), (dict(max_q=-1), INV), (dict(max_len=-1), INV), (dict(heads=3), INV), (dict(heads=0), INV),
          (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV), (dict(q=None), INV), (dict(out=8), ALIGN), (dict(ldq=128), INV),
          (dict(ldo=257), ALIGN), (dict(dt=2), INV), (dict(lens=None), INV), (dict(cu=None), INV), (dict(table=None), INV), (dict(batch=-1), INV),
          (dict(ldt=-1), INV), (dict(ldt=1 << 40), INV), (dict(lse=18), ALIGN), (dict(max_len=BIG + 1), UNS), (dict(max_q=BIG), UNS)]


@pytest.mark.parametrize("change,want", COMMON + [
    (dict(window=0), INV), (dict(window=-4), INV), (dict(sinks=-1), INV), (dict(window=0, batch=0), INV), (dict(max_len=4096, window=4096), INV),
    (dict(max_len=4096, window=4096, work=16, bytes=64), NOMEM), (dict(max_len=4096, window=4096, work=8, bytes=BIG), ALIGN)])
def test_window_refusals(change, want):
    assert call("sqap_kv_attention_window", cache(), WINDOW, change) == want


@pytest.mark.parametrize("change,want", COMMON + [
    (dict(flags=2), INV), (dict(groups=0), OK), (dict(max_group=0), OK), (dict(groups=-1), INV), (dict(max_group=-1), INV),
    (dict(max_prefix=-1), INV), (dict(cu_group=None), INV), (dict(prefix=None), INV), (dict(cu_group=18), ALIGN), (dict(prefix=17), ALIGN),
    (dict(), INV), (dict(work=16, bytes=SHARED_BYTES - 1), NOMEM), (dict(work=8, bytes=BIG), ALIGN),
    (dict(max_group=BIG), UNS), (dict(groups=2 * BIG - 1, max_group=1 << 25), UNS), (dict(groups=2 * BIG - 1, max_group=2 * BIG - 1), UNS)])
def test_shared_refusals(change, want):
    assert call("sqap_kv_attention_shared", cache(), SHARED, change) == want


@pytest.mark.parametrize("change,want", COMMON + [
    (dict(flags=2), INV), (dict(last_q=-1), INV), (dict(ldm=-1), INV), (dict(lse=None), INV), (dict(mass=None), INV), (dict(mass=18), ALIGN),
    (dict(past=17), ALIGN), (dict(max_len=4096, work=None), INV), (dict(max_len=4096, bytes=64), NOMEM), (dict(max_len=4096, work=8, bytes=BIG), ALIGN)])
def test_mass_refusals(change, want):
    assert call("sqap_kv_attention_mass", cache(), MASS, change) == want


EVICT = dict(mass=16, ldm=64, rows=4, lens=16, src=16, dst=16, n=2, keep=16, first=1, recent=2, max_len=64, kept=16, ldkept=8, nk=16, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(n=0), OK), (dict(n=-1), INV), (dict(rows=-1), INV), (dict(first=-1), INV), (dict(recent=-1), INV), (dict(max_len=-1), INV),
    (dict(ldm=-1), INV), (dict(ldkept=-1), INV), (dict(mass=None), INV), (dict(lens=None), INV), (dict(src=None), INV), (dict(keep=None), INV),
    (dict(kept=None), INV), (dict(nk=None), INV), (dict(mass=18), ALIGN), (dict(dst=17), ALIGN), (dict(kept=19), ALIGN), (dict(nk=22), ALIGN),
    (dict(max_len=BIG + 1), UNS), (dict(ldkept=1 << 33), UNS)])
def test_evict_refusals(change, want):
    assert B.lib().sqap_kv_evict(*{**EVICT, **change}.values()) == want


ROTARY = dict(x=16, ldx=256, rows=4, heads=2, D=128, rot=64, pos=16, ldp=4, axes=2, axis=bytes(32), freq=16, flags=0, out=32, ldo=256, dt=0, stream=None)


@pytest.mark.parametrize("change,want", [
    (dict(rows=0), OK), (dict(rows=-1), INV), (dict(heads=0), INV), (dict(D=0), INV), (dict(rot=0), INV), (dict(rot=136), INV), (dict(rot=60), ALIGN),
    (dict(D=124), ALIGN), (dict(D=264, ldx=1024, ldo=1024), UNS), (dict(axes=0), INV), (dict(axes=9), UNS), (dict(axis=bytes([2] * 32)), INV),
    (dict(ldx=248), INV), (dict(ldo=248), INV), (dict(ldx=257), ALIGN), (dict(ldo=260), ALIGN), (dict(ldp=3), INV), (dict(flags=2), INV),
    (dict(dt=3), INV), (dict(x=None), INV), (dict(out=None), INV), (dict(pos=None), INV), (dict(freq=None), INV), (dict(x=8), ALIGN),
    (dict(out=24), ALIGN), (dict(pos=18), ALIGN), (dict(freq=17), ALIGN), (dict(out=16, ldo=264), INV),
    (dict(heads=1 << 30, ldx=1 << 38, ldo=1 << 38), UNS)])
def test_rotary_refusals(change, want):
    assert B.lib().sqap_rotary(*{**ROTARY, **change}.values()) == want


def test_workspace_bytes():
    L = B.lib()
    window, shared, mass = L.sqap_kv_attention_window_workspace_bytes, L.sqap_kv_attention_shared_workspace_bytes, L.sqap_kv_attention_mass_workspace_bytes
    assert window(cache(), 4, 1, 1 << 20, 2, 100, 4) == 0                       # a short window is not cut, however long the history
    assert window(cache(), 1, 1, 16384, 2, 16384, 0) > 0 and window(cache(), 1, 1, 16384, 2, 0, 0) == window(cache(), 1, 1, 16384, 2, 5, -1) == 0
    assert shared(cache(), 2, 3, 64, 1, 64, 64, 4) == SHARED_BYTES and shared(cache(), 2, 3, 64, 1, 2, 64, 4) == 0     # few rows: one launch, one piece
    assert shared(cache(), 2, 3, 64, 1, 64, 0, 4) == 0 == shared(cache(), 2, 3, 64, 0, 2, 32, 4) == shared(cache(), 2, 3, 64, 1, 2, -1, 4)
    assert mass(cache(), 0, 1, 64, 2, 1) == mass(cache(), 1, 1, 64, 3, 1) == mass(cache(), 1, 1, 64, 2, -1) == 0
    for f, args in ((window, (5, 5)), (mass, (1,))):
        assert f(cache(type=5), 1, 1, 64, 2, *args) == 0 and f(cache(), 2 * BIG - 1, 2 * BIG - 1, 2 * BIG - 1, 2 * BIG - 2, *args) == 0
    assert shared(cache(), 2 * BIG - 1, 2 * BIG - 1, 2 * BIG - 1, 2 * BIG - 1, 2 * BIG - 1, 2 * BIG - 1, 2 * BIG - 2) == 0


def test_attention_arguments_are_checked_in_one_manner():
    """The same refusals for the arguments that the attention calls share."""
    for change, want in COMMON:
        if "window" in change:
            continue
        assert call("sqap_kv_attention", cache(), ATTEND, change) == want, change


def test_long_tokens_of_a_group_are_not_taken_together():
    """Places in the own tokens of all sequences that a tile of rows meets are 32-bit numbers: where they pass 2^30, sequences go one by one, and each
    takes pieces for its prefix beside its own, unlike tiles of rows."""
    shared = B.lib().sqap_kv_attention_shared_workspace_bytes

    def workspace(max_len):
        return shared(cache(), 8, 1, max_len, 1, 8, 1024, 2)

    together, apart = workspace((1 << 27) - 2048), workspace((1 << 27) + 2048)      # eight times the own tokens: just below 2^30, just above
    assert together != apart == workspace(1 << 30)
