"""The cache within a budget at the ends of what its arrays may hold, against oracle/drafts.py."""
import numpy as np
import pytest

from test_gpu_evict import check_gather

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,Hkv,D", [(16, 2, 32), (64, 3, 64), (128, 1, 128)])
def test_gather_of_scales_of_minus_zero(page, Hkv, D):
    """A page whose scale is -0 holds zeros, as one with 0 does: it neither replaces other pages' scales nor stands above NaN."""
    def spoil(cache, table, keep, n, to):
        for side in (2, 3):
            cache[side][table[0, 0], :] = -0.0        # beside pages with scales
            cache[side][table[1, :], :] = -0.0        # nothing else
            cache[side][table[2, 0], :] = -0.0        # beside one that cannot be used
            cache[side][table[2, 1], :] = np.nan
            cache[side][table[3, 0], :] = -0.0        # beside 0
            cache[side][table[3, 1:], :] = 0.0
    d, to = check_gather([3 * page] * 4, [2 * page + 3] * 4, Hkv, D, page, spoil=spoil)
    for scales in d[2:]:
        s = scales.cpu().numpy()[to]
        assert not np.signbit(s[~np.isnan(s)]).any() and (s[0] > 0).all() and (s[1] == 0).all() and (s[3] == 0).all()
