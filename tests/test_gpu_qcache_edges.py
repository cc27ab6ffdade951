"""The 8-bit cache where its state or its numbers are out of the ordinary: sequences that became shorter, values and scales at the ends of their range."""
import numpy as np
import pytest

from tests.test_gpu_qcache import Rig, T, dev, f64

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


# ------------------------------------------------------------------------------------------------ selection at the ends of the range
def guarded(rig, batch, q, rows, keep, first, recent):
    """A selection into memory with other things on both sides of it."""
    n = rows * rig.heads * keep
    buf = T().full((n + 4096,), -77, dtype=T().int32, device="cuda")
    rig.gpu.select(batch, q, keep, first, recent, pages=buf[2048:2048 + n].view(rows, rig.heads, keep))
    got = buf.cpu().numpy()
    assert (got[:2048] == -77).all() and (got[2048 + n:] == -77).all()
    return got[2048:2048 + n].reshape(rows, rig.heads, keep)


@pytest.mark.parametrize("d,heads", [(64, 2), (128, 1)])
@pytest.mark.parametrize("pages", [100, 500])
def test_selection_by_queries_whose_sum_over_a_group_passes_fp32(d, heads, pages):
    rig = Rig(1, pages, heads, d, 16, seed=130)
    rig.append([pages * 16 - 3])
    q = np.sign(rig.rng.standard_normal((2, heads * 8, d))) * 3e38
    q = np.where(np.arange(d) % 2 == 0, np.abs(q), q)    # eight of one sign in half of the channels
    t = dev(q.astype(np.float32)).to(T().bfloat16)
    q64 = f64(t)
    for keep in (4, 40, 99):
        got = guarded(rig, rig.batch([2]), t, 2, keep, 1, 1)
        for i in range(2):
            for h in range(heads):
                assert got[i, h].tolist() == rig.ref.select(rig.table[0], h, q64[i, 8 * h:8 * h + 8], int(rig.len[0]) - 1 + i, keep, 1, 1), (keep, i, h)


@pytest.mark.parametrize("pages", [100, 500, 9000])
@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
def test_queries_that_are_no_numbers_still_give_lists_of_pages(pages, what):
    rig = Rig(1, pages, 1, 64, 16, seed=131)
    rig.append([pages * 16])
    q, q64 = rig.draw(3, 2, 64)
    bad = q.clone()
    bad[1, 0, 5] = what
    bad[2, :, :] = what
    for keep in (4, 60):
        got, want = guarded(rig, rig.batch([3]), bad, 3, keep, 2, 1), guarded(rig, rig.batch([3]), q, 3, keep, 2, 1)
        assert np.array_equal(got[0], want[0])           # another row's list
        for i in (1, 2):
            own = got[i, 0]
            assert (np.diff(own) > 0).all() and own[:2].tolist() == [0, 1] and own[-1] == pages - 1


@pytest.mark.parametrize("d,G", [(128, 4), (64, 1), (128, 1)])
def test_scores_that_differ_in_their_last_bits_are_in_the_order_of_fp64(d, G):
    """Nearly all of a score comes from channels of the first product that adds them up, at the largest code, and the order of the pages from what all the
    products behind it add: codes of 2^-9 and 2^-8 against 448.  Bounds and scales are written here as an append of such keys would leave them."""
    torch = T()
    rig = Rig(1, 400, 1, d, 16, seed=132)
    rig.len = np.array([400 * 16], np.int32)
    rng = np.random.default_rng(5)
    codes = rng.integers(0, 3, (402, 1, 2, d)).astype(np.uint8)      # 0, 2^-9, 2^-8
    codes[:, :, 1, :16] = 0x7e                           # high: 448 in all pages
    codes[:, :, 0, :16] = 0xfe                           # low: -448
    codes[:, :, 0, 16:] = 0
    rig.ref.bounds[:] = codes
    rig.ref.exps[:] = 0
    rig.bounds.view(torch.uint8).copy_(dev(codes))
    rig.scales.fill_(1.0)
    for n, small in enumerate((1.0, 2.0 ** -4, 2.0 ** -8)):
        q = np.abs(rig.rng.standard_normal((1, G, d))) * small + small
        q[:, :, :16] = np.sign(rig.rng.standard_normal((1, G, 16))) * (1 + np.arange(16) / 16)
        t = dev(q.astype(np.float32)).to(torch.bfloat16)
        q64 = f64(t)
        for keep in (3, 57, 200, 390):
            got = guarded(rig, rig.batch([1]), t, 1, keep, 0, 1)[0, 0].tolist()
            assert got == rig.ref.select(rig.table[0], 0, q64[0], 6400, keep, 0, 1), (n, keep)
