"""The operators around the cache at their limits: shares of a long sequence of which every token stays. Lists are whole numbers and equal
the plain statement's."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from test_gpu_evict_rotary import check_evict, weights


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
