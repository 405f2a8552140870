"""The forms that attention for trees of drafted tokens takes, by type, head size, page size and columns (drafts times query heads of
a key head); bounds as in tests/test_gpu_drafts.py."""
import pytest

from test_gpu_drafts import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("new,kv,Hq,Hkv,D,page,dtype,window", [
    # 17 to 96 columns of bf16 heads up to 128: tiles of 32 whose codes wait in LDS
    ([24, 7], [300, 90], 4, 4, 128, 32, "bf16", 0), ([20, 31, 1], [700, 40, 500], 4, 2, 96, 16, "bf16", 0),
    ([96], [2000], 2, 2, 128, 128, "bf16", 0), ([48, 13], [333, 64], 4, 2, 80, 256, "bf16", 100), ([17], [17], 3, 3, 112, 64, "bf16", 0),
    ([33, 65], [1000, 70], 2, 2, 16, 32, "bf16", 9),
    # up to 48 of larger heads and up to 64 of fp32: tiles of 16
    ([24, 9], [300, 600], 2, 2, 256, 64, "bf16", 0), ([48, 17], [200, 90], 3, 3, 192, 16, "bf16", 30), ([64, 5], [500, 33], 2, 2, 128, 64, "f32", 0),
    ([30, 32], [90, 1100], 4, 2, 256, 32, "f32", 0),
    # more: the prompts' tiles
    ([97, 20], [400, 64], 2, 2, 128, 64, "bf16", 0), ([49, 30], [300, 200], 2, 2, 256, 128, "bf16", 0), ([100], [900], 3, 3, 192, 32, "bf16", 70),
    ([65, 130], [300, 700], 2, 2, 128, 16, "f32", 0), ([70], [1200], 2, 1, 256, 64, "f32", 0), ([129, 64], [600, 64], 2, 1, 64, 32, "bf16", 0),
])
def test_forms(new, kv, Hq, Hkv, D, page, dtype, window, kind):
    check(new, kv, Hq, Hkv, D, page, dtype, window, kind=kind, seed=21)
