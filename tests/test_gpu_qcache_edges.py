"""The 8-bit cache where its state or its numbers are out of the ordinary: sequences that became shorter, values and scales at the ends of their range."""
import numpy as np
import pytest

from paper_2609_03494_b200 import binding as B
from tests.test_gpu_qcache import BF16, EPS, F32, Rig, T, check_attention, dev, f64

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


# ------------------------------------------------------------------------------------------------ scales of values far apart
def along(rig, logits):
    """Keys whose logit (base 2) for a query of ones in channel 0 is about what is given; queries like that."""
    k = np.zeros((len(logits), rig.heads, rig.d), np.float32)
    k[:, :, 0] = (np.asarray(logits, np.float64) * np.log(2) * np.sqrt(rig.d))[:, None]
    t = dev(k).to(T().bfloat16)
    return t, f64(t)


def values(rig, n, size):
    """About `size`, of one sign: 1 + 0.1 N(0, 1)."""
    t = dev(((1 + 0.1 * rig.rng.standard_normal((n, rig.heads, rig.d))) * size).astype(np.float32)).to(T().bfloat16)
    return t, f64(t)


def ones(rig, rows, G):
    q = np.zeros((rows, rig.heads * G, rig.d), np.float32)
    q[:, :, 0] = 1 + 0.01 * rig.rng.random((rows, rig.heads * G))
    t = dev(q).to(T().bfloat16)
    return t, f64(t)


def check_sharp(rig, rows, q64, out, out_dtype, pages=None):
    """Like check_attention, against a bound that a large value without weight does not widen.  With t_j = 448 * 2^e_j, e_j the exponent of the scale of token
    j's values, and w_j its weight:
      weights carry a relative error of 2 (d 2^-22 A + 2^-18), and for 16-bit results half a step of fp16 more, which is 2^-11 of a weight just above a power of
      two: that of the weighted sum of magnitudes;
      fp16 holds a weight down to 2^-25 where the largest is 2^7 at least, so a token may lose 2^-32 of the largest weight (few rows), or of the largest
      product of weight and scale (many rows, twice that as a scale's largest value is only known to a factor of two): counted as 2^-31 of both;
      sums are kept relative to the largest scale of the sequence, in numbers down to 2^-149."""
    got, at, G = f64(out), 0, q64.shape[1] // rig.heads
    for s, r in enumerate(rows):
        for i in range(r):
            n = int(rig.len[s]) - r + i + 1
            for h in range(rig.heads):
                k, v, ok = rig.ref.rows(rig.table[s], h, n)
                top = np.ldexp(448.0, rig.ref.exps[rig.table[s][np.arange(n) // rig.page], h, 1])
                most = np.ldexp(448.0, int(rig.ref.exps[rig.table[s][:-(-int(rig.len[s]) // rig.page)], h, 1].max()))
                if pages is not None:
                    ok &= np.isin(np.arange(n) // rig.page, pages[at, h])
                k, v, top = k[ok], v[ok], top[ok]
                for g in range(G):
                    x = k @ q64[at, h * G + g] / np.sqrt(rig.d)
                    w = np.exp(x - x.max())
                    w /= w.sum()
                    A = float((np.abs(k) @ np.abs(q64[at, h * G + g])).max()) / np.sqrt(rig.d)
                    ref, size = w @ v, w @ np.abs(v)
                    rel = 2 * (rig.d * 2.0 ** -22 * A + 2.0 ** -18) + (0 if out_dtype == F32 else 2.0 ** -11)
                    tol = rel * size + np.minimum(w, 2.0 ** -31 * w.max()) @ top + len(w) * 2.0 ** -31 * (w * top).max() + EPS[out_dtype] / 2 * np.abs(ref) + most * 2.0 ** -146
                    err = np.abs(got[at, h * G + g] - ref)
                    assert (err <= tol).all(), (s, i, h, g, float(err.max()), float(tol.min()), float(np.abs(ref).max()))
            at += 1


@pytest.mark.parametrize("d,G", [(128, 4), (64, 8)])
@pytest.mark.parametrize("rows", [1, 5, 40, 150])
def test_the_sum_of_weights_holds_when_far_smaller_values_come_first(d, G, rows):
    """Zeros first (the smallest scale there is), then values whose weights are 2^-110 of theirs, then values whose weights are equal to theirs: the zeros count for half."""
    rig = Rig(1, 30, 1, d, 16, seed=120)
    zero = dev(np.zeros((64, 1, d), np.float32)).to(T().bfloat16)
    rig.append([64], kv=(along(rig, [0] * 64), (zero, f64(zero))))
    rig.append([64], kv=(along(rig, [-110] * 64), values(rig, 64, 1.0)))
    rig.append([64], kv=(along(rig, [0] * 64), values(rig, 64, 1.0)))
    rig.append([rows], kv=(along(rig, [-110] * rows), values(rig, rows, 1.0)))
    q, q64 = ones(rig, rows, G)
    for out in (F32, BF16):
        check_sharp(rig, [rows], q64, rig.gpu.attention(rig.batch([rows]), q, out_dtype=getattr(T(), out)), out)


@pytest.mark.parametrize("d,G", [(128, 4), (64, 8)])
@pytest.mark.parametrize("rows", [5, 40, 150])
def test_far_larger_values_that_a_row_does_not_see_change_nothing_for_it(d, G, rows):
    rig = Rig(1, 40, 2, d, 16, seed=121)
    rig.append([301], kv=(rig.draw(301, 2, d), values(rig, 301, 1.0)))
    rig.append([rows - 2], kv=(rig.draw(rows - 2, 2, d), values(rig, rows - 2, 1e-3)))
    rig.append([2], kv=(rig.draw(2, 2, d), values(rig, 2, 1e36)))
    q, q64 = rig.draw(rows, 2 * G, d)
    for out in (F32, BF16):
        check_sharp(rig, [rows], q64, rig.gpu.attention(rig.batch([rows]), q, out_dtype=getattr(T(), out)), out)


@pytest.mark.parametrize("d,G", [(128, 4), (64, 8)])
@pytest.mark.parametrize("rows", [1, 5, 40, 150])
@pytest.mark.parametrize("logit", [-300, -140])
def test_far_larger_values_without_weight_leave_the_others_what_they_are(d, G, rows, logit):
    rig = Rig(1, 40, 1, d, 16, seed=122)
    rig.append([48], kv=(along(rig, [logit] * 48), values(rig, 48, 2.0 ** 110)))
    rig.append([200], kv=(along(rig, [0] * 200), values(rig, 200, 1.0)))
    rig.append([rows], kv=(along(rig, [0] * rows), values(rig, rows, 2.0 ** -10)))
    q, q64 = ones(rig, rows, G)
    for out in (F32, BF16):
        check_sharp(rig, [rows], q64, rig.gpu.attention(rig.batch([rows]), q, out_dtype=getattr(T(), out)), out)


# ------------------------------------------------------------------------------------------------ values at the upper end of the range
@pytest.mark.parametrize("d,G", [(128, 4), (64, 8)])
@pytest.mark.parametrize("rows", [1, 5, 40, 150])
@pytest.mark.parametrize("n", [1, 300, 9000])
@pytest.mark.parametrize("size", [2.0 ** 112, 2.0 ** 126, 2.0 ** -118])
def test_values_at_the_ends_of_the_range(d, G, rows, n, size):
    """Every held value is at most 448 * 2^119, and so is a weighted mean of them: sums on the way are not to pass what fp32 holds, in whole units and in
    those that blocks share (one KV head of 9000 tokens)."""
    rig = Rig(1, 600, 1, d, 16, seed=123)
    rig.append([n], kv=(rig.draw(n, 1, d), values(rig, n, size)))
    rig.append([rows], kv=(rig.draw(rows, 1, d), values(rig, rows, size)))
    q, q64 = rig.draw(rows, G, d)
    some = sorted({0, rows // 2, rows - 1})
    for out in (F32, BF16):
        got = rig.gpu.attention(rig.batch([rows]), q, out_dtype=getattr(T(), out))
        for i in some:
            one = Rig.__new__(Rig)
            one.__dict__.update(rig.__dict__)
            one.len = rig.len - (rows - 1 - i)
            check_sharp(one, [1], q64[i:i + 1], got[i:i + 1], out)


@pytest.mark.parametrize("size", [2.0 ** 112, 2.0 ** 126])
def test_values_at_the_upper_end_of_the_range_through_a_list(size):
    rig = Rig(1, 600, 1, 128, 16, seed=124)
    rig.append([9000], kv=(rig.draw(9000, 1, 128), values(rig, 9000, size)))
    q, q64 = rig.draw(1, 4, 128)
    pages = rig.gpu.select(rig.batch([1]), q, 500, 1, 1)
    for out in (F32, BF16):
        check_sharp(rig, [1], q64, rig.gpu.attention(rig.batch([1]), q, out_dtype=getattr(T(), out), pages=pages), out, pages.cpu().numpy())


# ------------------------------------------------------------------------------------------------ values that are no numbers
def check_with_nans(rig, s, rows, q64, got, out_dtype, some):
    """Rows `some` of a sequence's rows against the oracle: NaN where and only where a row sees one, the others within check_attention's bound."""
    G = q64.shape[1] // rig.heads
    for i in some:
        n = int(rig.len[s]) - rows + i + 1
        for h in range(rig.heads):
            k, v, _ = rig.ref.rows(rig.table[s], h, n)
            vmax = np.nanmax(np.abs(v))
            for g in range(G):
                q = q64[i, h * G + g]
                x = k @ q / np.sqrt(rig.d)
                w = np.exp(x - x.max())
                ref = (w @ np.nan_to_num(v)) / w.sum()
                ref[np.isnan(v).any(0)] = np.nan
                A = float((np.abs(k) @ np.abs(q)).max()) / np.sqrt(rig.d)
                o = got[i, h * G + g]
                assert np.array_equal(np.isnan(o), np.isnan(ref)), (s, i, h, g, np.flatnonzero(np.isnan(o) != np.isnan(ref)))
                if np.isnan(ref).all():
                    continue
                tol = 2 * vmax * (rig.d * 2.0 ** -22 * A + 2.0 ** -18) + (0 if out_dtype == F32 else vmax * 2.0 ** -11) + EPS[out_dtype] / 2 * np.abs(ref)
                ok = np.isnan(ref) | (np.abs(o - ref) <= tol)
                assert ok.all(), (s, i, h, g)


@pytest.mark.parametrize("d,G", [(128, 4), (64, 8), (64, 3)])
@pytest.mark.parametrize("rows,held", [(2, 300), (5, 12000), (6, 40), (40, 5000), (200, 7000), (260, 90)])
def test_values_that_are_no_numbers_reach_the_rows_that_see_them_and_no_others(d, G, rows, held):
    """In whole units and in those that blocks share (a long sequence with one KV head), in several channels, in rows before the first that is asked for."""
    rig = Rig(1, 800, 1, d, 16, seed=140 + rows)
    n = held + rows
    k, v = rig.draw(n, 1, d), rig.draw(n, 1, d)
    for back, channels in ((1, [2]), (rows // 2, [7, d - 1]), (rows - 1, [0]), (rows + 1, [9]), (rows + 30, [33])):
        for c in channels:
            v[0][n - 1 - back, 0, c] = float("nan" if c % 2 else "inf")
    rig.append([n], kv=((k[0], f64(k[0])), (v[0], f64(v[0]))))
    q, q64 = rig.draw(rows, G, d)
    some = sorted({0, 1, rows // 2 - 1, rows // 2, rows - 2, rows - 1, min(rows - 1, 63), min(rows - 1, 128)} & set(range(rows)))
    for out in (F32, BF16):
        got = f64(rig.gpu.attention(rig.batch([rows]), q, out_dtype=getattr(T(), out)))
        check_with_nans(rig, 0, rows, q64, got, out, some)


@pytest.mark.parametrize("d,G", [(128, 4), (64, 8)])
@pytest.mark.parametrize("rows", [4, 30])
def test_values_that_are_no_numbers_stay_in_their_sequence_and_head(d, G, rows):
    """Several units a block, those with such values among others."""
    seqs = 150
    rig = Rig(seqs, 12, 4, d, 16, seed=150 + rows)
    lens = [int(x) for x in rig.rng.integers(rows, 180, seqs)]
    k, v = rig.draw(sum(lens), 4, d), rig.draw(sum(lens), 4, d)
    at = np.concatenate([[0], np.cumsum(lens)])
    hit = {}
    for s in range(0, seqs, 7):
        h, c, back = s % 4, (5 * s) % d, 1 + s % (rows - 1)
        v[0][int(at[s + 1]) - 1 - back, h, c] = float("nan")
        hit[s] = (h, c, back)
    rig.append(lens, kv=((k[0], f64(k[0])), (v[0], f64(v[0]))))
    q, q64 = rig.draw(rows * seqs, 4 * G, d)
    got = f64(rig.gpu.attention(rig.batch([rows] * seqs), q, out_dtype=T().float32)).reshape(seqs, rows, 4, G, d)
    want = np.zeros(got.shape, bool)
    for s, (h, c, back) in hit.items():
        want[s, rows - 1 - back:, h, :, c] = True
    assert np.array_equal(np.isnan(got), want)
    for s in (0, 1, 7, 149):
        check_with_nans(rig, s, rows, q64[s * rows:(s + 1) * rows], got[s].reshape(rows, 4 * G, d), F32, [0, rows - 1])


# ------------------------------------------------------------------------------------------------ waits that run out
@pytest.mark.parametrize("d,G", [(128, 4), (64, 8)])
@pytest.mark.parametrize("what,rows,listed", [(1, 1, False), (1, 3, False), (1, 1, True), (2, 60, False), (2, 300, False)])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_as_before(d, G, what, rows, listed):
    """One hand-over is not made (never signalled, nothing faults): the waits of its thread block give up after 200 000 cycles, the block ends, the status word says so;
    blocks of other sequences are not affected."""
    torch = T()
    rig = Rig(6, 80, 2, d, 16, seed=160)
    rig.append([900, 30, 700, 400, 650, 880 - rows])
    rig.append([rows] * 6)
    q, q64 = rig.draw(6 * rows, 2 * G, d)
    b = rig.batch([rows] * 6)
    pages = rig.gpu.select(b, q, 20, 1, 1) if listed else None
    call = lambda: rig.gpu.attention(b, q, out=torch.full(q.shape, 9.0, device="cuda"), pages=pages)  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    assert int(rig.status.item()) == 0
    B.gp_qcache_test_withhold(what, 200000)
    try:
        got = call()
        torch.cuda.synchronize()
    finally:
        B.gp_qcache_test_withhold(0, 0)
    assert int(rig.status.item()) == 1
    assert torch.equal(got[-rows:], want[-rows:])
    rig.status.zero_()
    for _ in range(3):
        assert torch.equal(call(), want)
    assert int(rig.status.item()) == 0


# ------------------------------------------------------------------------------------------------ without the holder
def test_the_calls_of_the_c_interface_are_those_of_the_holder():
    torch = T()
    a, b = Rig(2, 30, 2, 64, 16, seed=180), Rig(2, 30, 2, 64, 16, seed=180)
    for rig in (a, b):
        rig.append([300, 41])
        rig.len = rig.len + 2
    batch, stream = a.batch([2, 2]), a.gpu.stream()
    q, k, v = (a.draw(4, n, 64)[0] for n in (8, 2, 2))
    want_q = a.gpu.append(batch, k, v, q=q, rope_theta=1e4)
    want_pages = a.gpu.select(batch, want_q, 5, 1, 1)
    want = a.gpu.attention(batch, want_q, pages=want_pages, out_dtype=torch.float32)
    batch = b.batch([2, 2])
    got_q, got_pages, got = torch.empty_like(want_q), torch.empty_like(want_pages), torch.empty_like(want)
    rows = B.gp_qrows(k=k.data_ptr(), v=v.data_ptr(), q=q.data_ptr(), q_out=got_q.data_ptr(), k_stride=128, v_stride=128, q_stride=512, q_out_stride=512,
                      rope_theta=1e4, n_q_heads=8, type=B.GP_TYPE_BF16)
    B.gp_qcache_append(b.gpu.desc, batch.desc, rows, stream)
    sizes = [B.gp_qcache_select_bytes(b.gpu.desc, batch.desc), B.gp_qcache_attention_bytes(b.gpu.desc, batch.desc, 8, 5)]
    work = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    B.gp_qcache_select(b.gpu.desc, batch.desc, got_q.data_ptr(), 512, 8, B.GP_TYPE_BF16, 5, 1, 1, got_pages.data_ptr(), work[0].data_ptr(), sizes[0], stream)
    B.gp_qcache_attention(b.gpu.desc, batch.desc, got_q.data_ptr(), 512, 8, B.GP_TYPE_BF16, got_pages.data_ptr(), 5, got.data_ptr(), B.GP_TYPE_F32,
                          work[1].data_ptr(), sizes[1], stream)
    assert torch.equal(got_q, want_q) and torch.equal(got_pages, want_pages) and torch.equal(got, want)
    assert torch.equal(a.codes.view(torch.uint8), b.codes.view(torch.uint8)) and torch.equal(a.bounds.view(torch.uint8), b.bounds.view(torch.uint8))


@pytest.mark.parametrize("d,page,dtype", [(64, 16, BF16), (128, 16, "float16"), (128, 64, BF16), (64, 128, "float16"), (128, 256, BF16)])
def test_a_cache_without_bounds(d, page, dtype):
    rig = Rig(3, 3 + 200 // page, 5, d, page, seed=190 + d, bounds=False)
    for rows, scale in (([page + 3, 0, 1], 1.0), ([1, 1, 1], 30.0), ([5, 2, 17], 0.1), ([page, page - 1, 0], 1e3), ([1, 1, 2], 1.0)):
        rig.append(rows, dtype=dtype, theta=1e4, norm=scale == 1.0, scale=scale, q_heads=10)
        rig.check()
    q, q64 = rig.draw(3, 10, d, dtype=dtype)
    check_attention(rig, [1, 1, 1], q, q64, rig.gpu.attention(rig.batch([1, 1, 1]), q, out_dtype=T().float32), F32)
    with pytest.raises(B.GpError):
        rig.gpu.select(rig.batch([1, 1, 1]), q, 3, 1, 1)


# ------------------------------------------------------------------------------------------------ a token that outweighs all others
@pytest.mark.parametrize("d,G,dtype", [(128, 4, BF16), (64, 8, "float16"), (64, 3, BF16)])
@pytest.mark.parametrize("rows", [1, 5, 100])
def test_a_row_that_goes_by_one_token_has_that_tokens_values(d, G, dtype, rows):
    """The first row of a prompt sees one token, later ones (here) one whose weight is 2^40 of the others' and more: 16-bit results are its held values exactly, fp32 ones up to
    the 2^-18 of weights and sums."""
    rig = Rig(2, 20, 1, d, 16, seed=200)
    n = rows + 30
    k = along(rig, [0.0 if i % 9 else 400.0 * 1.25 ** (i // 9) for i in range(n)])      # (e4m3 keeps numbers apart that differ by an eighth)
    v = rig.draw(n, 1, d, dtype=dtype)
    kd = (k[0].to(v[0].dtype), f64(k[0].to(v[0].dtype)))
    both = [(T().cat([x[0], x[0][:rows]]), np.concatenate([x[1], x[1][:rows]])) for x in (kd, v)]
    rig.append([n, rows], dtype=dtype, kv=both)
    q, q64 = ones(rig, 2 * rows, G)
    q = q.to(v[0].dtype)
    for out in (dtype, F32):
        got = f64(rig.gpu.attention(rig.batch([rows, rows]), q, out_dtype=getattr(T(), out)))
        for s in range(2):
            _, held, _ = rig.ref.rows(rig.table[s], 0, int(rig.len[s]))
            for i in range(rows):
                pos = int(rig.len[s]) - rows + i
                want = held[pos - pos % 9]
                err = np.abs(got[s * rows + i] - want)
                assert (err <= (0 if out != F32 else np.abs(want) * 2.0 ** -18)).all(), (s, i, out)
