"""The 8-bit cache where its state or its numbers are out of the ordinary: sequences that became shorter, values and scales at the ends of their range."""
import numpy as np
import pytest

from tests.test_gpu_qcache import Rig

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ sequences that became shorter
@pytest.mark.parametrize("d,page,heads", [(64, 16, 2), (128, 16, 8), (128, 64, 3), (64, 256, 1)])
def test_bounds_are_those_of_the_rows_that_are_held_after_some_were_taken_back(d, page, heads):
    rig = Rig(3, 3 + 160 // page, heads, d, page, seed=100 + d + page)
    rig.append([page + 8, 9, 2 * page + 1], theta=1e4)
    rig.append([4, 5, 3], scale=4.0)                     # drafts, larger than the rest
    rig.check()
    for back, rows in (([3, 5, 2], [1, 1, 1]), ([1, 2, 3], [2, 1, 4]), ([2, 1, 1], [2, 1, 1])):
        rig.len = rig.len - np.array(back, np.int32)     # inside a page and over a page's border
        rig.append(rows, theta=1e4, scale=0.5)
        rig.check()


def test_a_selection_after_drafts_were_taken_back_goes_by_the_keys_that_are_held():
    rig = Rig(1, 60, 2, 64, 16, seed=110)
    n = 0
    for p in range(40):                                  # every page has had far larger rows that were taken back
        rig.append([10])
        rig.append([6], scale=float(1 + 7 * (p % 5)))
        rig.len = rig.len - 6
        rig.append([6], scale=0.5)
        n += 16
    rig.check()
    q, q64 = rig.draw(1, 8, 64)
    got = rig.gpu.select(rig.batch([1]), q, 9, 1, 1).cpu().numpy()[0]
    for h in range(2):
        assert got[h].tolist() == rig.ref.select(rig.table[0], h, q64[0, 4 * h:4 * h + 4], n, 9, 1, 1)
