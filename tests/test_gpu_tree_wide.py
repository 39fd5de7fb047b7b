"""Attention of drafted tokens where the row count or the place of a key picks
other code: more than 32 rows a head (both tiles), chunks' first keys."""
import numpy as np
import pytest

from serving import Batch

pytestmark = pytest.mark.gpu
ROWS = [(1, 4), (3, 7), (16, 3), (16, 7), (43, 7)]       # drafts, heads a KV head: 4, 21, 48, 112, 301 rows


@pytest.fixture(scope="module")
def ctx():
    from paper_2504_16083_amd import mmi
    return mmi.Ctx(0)


@pytest.mark.parametrize("T,g", ROWS)
@pytest.mark.parametrize("L", [20, 64, 300, 9000])
def test_infinities_in_cached_values(ctx, T, g, L):
    """Every row sees a cached token: an infinity in its V makes that channel infinite, wherever the token lies in
    its chunk, and both infinities in one channel a NaN. The other channels are as they were."""
    b = Batch("bf16", [L], [T], g, 1, 16, seed=L)
    for token, d, value in [(0, 5, np.inf), (19, 6, -np.inf), (L - 1, 7, np.inf), (L // 2, 8, np.inf), (0, 90, np.inf),
                            (L - 1, 90, -np.inf)] + [(c, d, -np.inf) for d, c in enumerate(range(128, min(L, 4000), 128), 20)]:
        s = int(b.slots[0][token])
        b.V[s, 0, d] = value
        b.cache.v[s // 16, 0, s % 16, d] = value
    with np.errstate(all="ignore"):
        b.check(*b.run(ctx), rows={(0, 0), (0, T - 1)})
