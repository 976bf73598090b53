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
