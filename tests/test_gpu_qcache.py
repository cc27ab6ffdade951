"""The 8-bit cache through its public calls against the float64 oracle: what is put into the pages, the attention over them, the pages that
are chosen, and all of it in a run."""
import math

import numpy as np
import pytest

from paper_2609_03494_b200 import binding as B
from tests import qcache_oracle as O

pytestmark = pytest.mark.gpu
BF16, F16, F32 = "bfloat16", "float16", "float32"
EPS = {BF16: 2.0 ** -7, F16: 2.0 ** -10, F32: 2.0 ** -23}


def T():
    import torch
    return torch


def dev(a, dtype=None):
    t = T().from_numpy(np.ascontiguousarray(a)).cuda()
    return t.to(getattr(T(), dtype)) if dtype else t


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Rig:
    """A cache on the GPU and the oracle's, sequences on scattered pages."""

    def __init__(self, seqs, pages_each, heads, d, page, seed=0, bounds=True, spare=2):
        torch = T()
        self.rng = np.random.default_rng(seed)
        self.heads, self.d, self.page = heads, d, page
        n_pages = seqs * pages_each + spare
        self.table = self.rng.permutation(n_pages)[:seqs * pages_each].reshape(seqs, pages_each).astype(np.int32)
        self.ref = O.Cache(n_pages, heads, d, page)
        self.gpu = B.QCache.create(n_pages, heads, d, page, bounds=bounds)
        junk = self.rng.integers(0, 256, self.ref.codes.shape, dtype=np.uint8)      # what earlier owners left, NaNs among it
        self.ref.codes[:] = junk
        self.codes, self.scales, self.bounds, self.status = self.gpu.tensors
        self.codes.view(torch.uint8).copy_(dev(junk))
        self.len = np.zeros(seqs, np.int32)
        self.dtable = dev(self.table)

    def batch(self, rows, lens=None, max_rows=None, max_len=None, extra=0, gap=0):
        start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32) + gap
        lens = self.len if lens is None else lens
        return B.QBatch(dev(start), dev(np.asarray(lens, np.int32)), self.dtable, int(start[-1]) + extra, max(rows) if max_rows is None else max_rows,
                        max(int(max(lens)), 1) if max_len is None else max_len)

    def draw(self, *shape, dtype=BF16, scale=1.0):
        t = dev((self.rng.standard_normal(shape) * scale).astype(np.float32)).to(getattr(T(), dtype))
        return t, f64(t)

    def append(self, rows, dtype=BF16, theta=0.0, norm=False, shift=0, scale=1.0, q_heads=0, kv=None, extra=0):
        """Appends rows[s] new tokens to every sequence on both sides; returns (queries out, their exact value, their inputs)."""
        n = sum(rows) + extra
        k, k64 = kv[0] if kv else self.draw(n, self.heads, self.d, dtype=dtype, scale=scale)
        v, v64 = kv[1] if kv else self.draw(n, self.heads, self.d, dtype=dtype, scale=scale)
        old = self.len.copy()
        self.len = self.len + np.asarray(rows, np.int32)
        b = self.batch(rows, extra=extra)
        slots = np.concatenate([np.arange(o, o + r) for o, r in zip(old, rows)] + [np.zeros(extra, np.int64)]).astype(np.int64)
        pos = slots + shift
        w = (1 + 0.2 * self.rng.standard_normal((2, self.d))).astype(np.float32) if norm else None
        kw = dict(rope_theta=theta, k_weight=dev(w[0]) if norm else None, eps=1e-6, positions=dev(pos.astype(np.int32)) if shift else None)
        q_out = q_ref = None
        if q_heads:
            q, q64 = self.draw(n, q_heads, self.d, dtype=dtype)
            q_out = self.gpu.append(b, k, v, q=q, q_weight=dev(w[1]) if norm else None, **kw)
            q_ref = O.norm_rotate(q64, w[1].astype(np.float64) if norm else None, 1e-6, pos, theta)
        else:
            assert self.gpu.append(b, k, v, **kw) is None
        k_ref = O.norm_rotate(k64, w[0].astype(np.float64) if norm else None, 1e-6, pos, theta)
        at = 0
        for s, r in enumerate(rows):
            self.ref.append(self.table[s], int(old[s]), k_ref[at:at + r], v64[at:at + r])
            at += r
        return q_out, q_ref

    def check(self):
        """Codes, scales and bounds equal the oracle's.  (Keys are computed in fp64 on both sides; the one rounding to fp32 in front of the
        rounding to a code can move a key to the neighbouring code only within 2^-24 of a border: none is expected, one in 10^5 is let pass.)"""
        torch = T()
        got = self.codes.view(torch.uint8).cpu().numpy()
        exps = np.round(np.log2(f64(self.scales))).astype(np.int64)
        used = np.zeros(len(got), bool)
        for s, n in enumerate(self.len):
            used[self.table[s][:-(-int(n) // self.page)]] = True
        assert np.array_equal(exps[used], self.ref.exps[used])
        a, b = O.decode(got), O.decode(self.ref.codes)
        assert np.array_equal(np.isnan(a), np.isnan(b))
        assert np.array_equal(got[~used], self.ref.codes[~used])          # pages of nobody
        wrong = (np.nan_to_num(a) != np.nan_to_num(b))
        assert wrong.sum() <= wrong.size * 1e-5, wrong.sum()
        if self.bounds is not None:
            lo = O.decode(self.bounds.view(torch.uint8).cpu().numpy()[used])
            w2 = lo != O.decode(self.ref.bounds[used])
            assert w2.sum() <= max(w2.size * 1e-5, wrong.sum()), w2.sum()
        assert int(self.status.item()) == 0


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("d,page,heads,dtype", [(128, 16, 8, BF16), (64, 16, 2, F16), (128, 64, 3, BF16), (64, 32, 5, BF16), (128, 256, 1, F16), (64, 128, 2, BF16),
                                                (64, 256, 1, BF16), (128, 128, 2, BF16)])
@pytest.mark.parametrize("theta,norm,shift", [(0.0, False, 0), (1e6, True, 0), (1e4, False, 100000)])
def test_append(d, page, heads, dtype, theta, norm, shift):
    rig = Rig(4, 3 + 80 // page, heads, d, page, seed=d + page)
    for rows in ([page + 3, 0, 1, 2 * page], [1, 1, 1, 1], [5, 2, 0, 17], [0, page, page - 1, 0], [1, 1, 0, 1]):
        q, ref = rig.append(rows, dtype=dtype, theta=theta, norm=norm, shift=shift, q_heads=2 * heads)
        if q.shape[0]:
            # rounded once; before that fp32: a rotation of two elements after a sum of d squares, angles good to 2^-24 of a turn
            h = d // 2
            size = np.abs(ref[..., :h]) + np.abs(ref[..., h:])
            tol = EPS[dtype] / 2 * np.abs(ref) + np.concatenate([size, size], -1) * 2.0 ** -19 + (2.0 ** -25 if dtype == F16 else 0)
            assert (np.abs(f64(q) - ref) <= tol).all()
    rig.check()


def test_append_of_a_batch_of_single_tokens_and_one_prompt():
    rig = Rig(40, 40, 8, 128, 16, seed=3)
    for rows in ([1] * 39 + [601], [1] * 40, [0] * 20 + [3] * 20):
        rig.append(rows, theta=1e6, norm=True, q_heads=32)
    rig.check()


def test_a_scale_grows_and_the_codes_before_follow_it():
    rig = Rig(2, 3, 2, 128, 16, seed=5)
    for i, scale in enumerate([0.01, 0.02, 1.0, 0.5, 300.0, 1e-3, 70.0, 1e30, 1.0, 1e38]):
        rig.append([1 + i % 2, 2], scale=scale)
        rig.check()


def test_numbers_at_the_ends_of_the_range_and_no_numbers():
    torch = T()
    rig = Rig(1, 4, 1, 64, 16, seed=6)
    x = np.zeros((21, 1, 64), np.float32)
    x[0, 0, :8] = [3.38e38, -3.38e38, 1e-38, -1e-40, 0.0, -0.0, 448.0, 449.0]
    x[1] = 2.0 ** -126
    x[2, 0, 0], x[2, 0, 1], x[2, 0, 2] = np.nan, np.inf, -np.inf
    x[16:, 0] = 0.0                                      # a page that holds zeros, then something
    x[18, 0, 3] = 1.5
    x[20, 0, 4] = np.inf
    t = dev(x).to(torch.bfloat16)
    pair = (t, f64(t))
    rig.append([21], kv=(pair, pair))
    rig.check()
    rig.append([3], scale=1.0)
    rig.check()
    rig2 = Rig(1, 2, 1, 128, 16, seed=7)                 # a rotation whose result passes the largest fp32 number
    x = np.full((2, 1, 128), 3.38e38, np.float32)
    t = dev(x).to(torch.bfloat16)
    rig2.append([2], kv=((t, f64(t)), (t, f64(t))), theta=1e4, shift=1)
    rig2.check()


def test_rows_behind_the_batch_and_pages_of_others_stay():
    torch = T()
    rig = Rig(3, 4, 4, 64, 16, seed=8)
    rig.append([20, 3, 33], extra=5, theta=1e4, q_heads=8)
    rig.check()
    q = torch.full((6, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    out = torch.full((6, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    rig.len = rig.len + np.array([1, 0, 2], np.int32)
    k = torch.randn(6, 4, 64, device="cuda").to(torch.bfloat16)
    b = rig.batch([1, 0, 2], extra=2, gap=1)             # rows 1 .. 3 of six
    rig.gpu.append(b, k, k, q=q, q_out=out)
    assert (out[1:4] == 7).all() and (out[:1] == 3).all() and (out[4:] == 3).all()
    out.fill_(3.0)
    rig.gpu.attention(b, q, out=out)
    assert (out[:1] == 3).all() and (out[4:] == 3).all() and (out[1:4] != 3).any()
    pages = torch.full((6, 4, 2), -7, dtype=torch.int32, device="cuda")
    rig.gpu.select(b, q, 2, 0, 1, pages=pages)
    assert (pages[:1] == -7).all() and (pages[4:] == -7).all() and (pages[1:4] >= 0).all()


def test_slices_of_one_projection_and_queries_in_place():
    torch = T()
    a, b = Rig(2, 4, 2, 128, 16, seed=9), Rig(2, 4, 2, 128, 16, seed=9)
    qkv = torch.randn(30, (8 + 2 + 2) * 128 + 64, device="cuda").to(torch.bfloat16)
    part = lambda lo, n: qkv[:, lo * 128:(lo + n) * 128].view(30, n, 128)  # noqa: E731
    want = None
    for rig, inplace in ((a, False), (b, True)):
        rig.len = np.array([13, 17], np.int32)
        batch = rig.batch([13, 17])
        q, k, v = part(0, 8), part(8, 2), part(10, 2)
        if inplace:
            assert rig.gpu.append(batch, k, v, q=q, q_out=q, rope_theta=1e4) is q
            assert torch.equal(q, want)
        else:
            want = rig.gpu.append(batch, k.contiguous(), v.contiguous(), q=q, rope_theta=1e4)
    assert torch.equal(a.codes.view(torch.uint8), b.codes.view(torch.uint8)) and torch.equal(a.scales, b.scales)


# ------------------------------------------------------------------------------------------------ attention
def check_attention(rig, rows, q, q64, out, out_dtype, pages=None):
    """Against softmax in float64 over what the oracle holds.  Bound: a logit is a sum of d exact products, each addition of which
    is off by 2^-22 of the sum of magnitudes A at most (in whatever order and chain); weights carry that, 2^-20 of exp2f, fp32 sums and two-term
    fp16 together, so the output is off by 2 (d 2^-22 A + 2^-18) of the largest value, before its own rounding.  For 16-bit outputs the weights
    of the sum of values are rounded to fp16 once, half a step being 2^-11 / 2 of each: 2^-12 of the largest value more."""
    got, at, G, worst = f64(out), 0, q64.shape[1] // rig.heads, 0.0
    for s, r in enumerate(rows):
        for i in range(r):
            pos = int(rig.len[s]) - r + i
            for h in range(rig.heads):
                seen = np.arange(pos + 1)
                if pages is not None:
                    mine = set(int(p) for p in pages[at, h] if p >= 0)
                    seen = np.array([t for t in seen if t // rig.page in mine], np.int64)
                for g in range(G):
                    ref, A, vmax = rig.ref.attend(rig.table[s], h, q64[at, h * G + g], seen)
                    tol = 2 * vmax * (rig.d * 2.0 ** -22 * A + 2.0 ** -18) + (0 if out_dtype == F32 else vmax * 2.0 ** -12) + EPS[out_dtype] / 2 * np.abs(ref) + (2.0 ** -25 if out_dtype == F16 else 0)
                    err = np.abs(got[at, h * G + g] - ref)
                    assert (err <= tol).all(), (s, i, h, g, float(err.max()), float(tol.min()))
            at += 1


@pytest.mark.parametrize("d,page,heads,G,dtype,out", [(128, 16, 8, 4, BF16, BF16), (64, 16, 2, 8, F16, F32), (128, 64, 1, 1, BF16, F32), (64, 32, 3, 7, BF16, F16),
                                                      (128, 256, 2, 5, F16, F16), (128, 16, 1, 8, BF16, F32), (64, 128, 2, 2, F16, BF16)])
@pytest.mark.parametrize("rows", [[1, 1, 1, 1], [0, 1, 5, 2], [3, 7, 1, 40], [16, 33, 100, 2]])
def test_attention(d, page, heads, G, dtype, out, rows):
    rig = Rig(4, 3 + 300 // page, heads, d, page, seed=G + d)
    rig.append([max(rows[0], 1), 17, 130, 211])
    q, q64 = rig.draw(sum(rows), heads * G, d, dtype=dtype, scale=2.0)
    rows = [min(r, int(n)) for r, n in zip(rows, rig.len)]
    q, q64 = q[:sum(rows)], q64[:sum(rows)]
    got = rig.gpu.attention(rig.batch(rows), q, out_dtype=getattr(T(), out))
    check_attention(rig, rows, q, q64, got, out)
    assert int(rig.status.item()) == 0


def test_attention_over_a_long_cache_in_splits_with_far_weights():
    rig = Rig(2, 700, 1, 128, 16, seed=21)
    rig.append([11001, 5000], scale=1.0)
    rig.append([1, 1], scale=3.0)
    q, q64 = rig.draw(2, 4, 128, scale=3.0)
    for out in (F32, BF16):
        check_attention(rig, [1, 1], q, q64, rig.gpu.attention(rig.batch([1, 1]), q, out_dtype=getattr(T(), out)), out)


def test_pages_whose_values_differ_by_many_powers_of_two():
    rig = Rig(1, 8, 2, 64, 16, seed=22)
    for i, scale in enumerate([1.0, 1e-20, 1e4, 1e-3, 1e15]):
        rig.append([16], scale=scale if i != 2 else 1.0, kv=(rig.draw(16, 2, 64, scale=0.5), rig.draw(16, 2, 64, scale=scale)))
    q, q64 = rig.draw(1, 8, 64)
    check_attention(rig, [1], q, q64, rig.gpu.attention(rig.batch([1]), q, out_dtype=T().float32), F32)


@pytest.mark.parametrize("d,G,out", [(128, 4, BF16), (64, 8, F32)])
@pytest.mark.parametrize("rows", [1, 5, 40, 150])
def test_values_of_zero_and_of_all_sizes_before_many_rows(d, G, out, rows):
    """Pages of zeros have the smallest scale there is, others are 2^60 apart: the weights of all of them count alike."""
    rig = Rig(1, 30, 2, d, 16, seed=60 + rows)
    z = dev(np.zeros((48, 2, d), np.float32)).to(T().bfloat16)
    for scale in (0, 1.0, 0, 1e-18, 1e6, 0, 30.0):
        v = (z, f64(z)) if scale == 0 else rig.draw(48, 2, d, scale=scale)
        rig.append([48], kv=(rig.draw(48, 2, d), v))
    rig.append([64])
    q, q64 = rig.draw(rows, 2 * G, d)
    check_attention(rig, [rows], q, q64, rig.gpu.attention(rig.batch([rows]), q, out_dtype=getattr(T(), out)), out)
    zero = Rig(1, 30, 2, d, 16, seed=61)                 # nothing but zeros, then a page that is not
    zero.append([200], kv=(zero.draw(200, 2, d), (dev(np.zeros((200, 2, d), np.float32)).to(T().bfloat16), np.zeros((200, 2, d)))))
    zero.append([40], scale=2.0)
    check_attention(zero, [rows], q, q64, zero.gpu.attention(zero.batch([rows]), q, out_dtype=getattr(T(), out)), out)


@pytest.mark.parametrize("d,G", [(128, 4), (64, 8)])
def test_a_padded_batch_whose_sequences_have_fewer_rows_than_there_is_room_for(d, G):
    torch = T()
    rig = Rig(3, 20, 2, d, 16, seed=62)
    rig.append([250, 30, 111])
    q, q64 = rig.draw(300, 2 * G, d)
    for rows in ([1, 1, 1], [100, 1, 3], [0, 2, 100], [1, 0, 0]):
        out = torch.full((300, 2 * G, d), 5.0, dtype=torch.bfloat16, device="cuda")
        n = sum(rows)
        b = rig.batch(rows, max_rows=100, extra=300 - n)
        rig.gpu.attention(b, q, out=out)
        check_attention(rig, rows, q[:n], q64[:n], out[:n], BF16)
        assert (out[n:] == 5).all()
    one = Rig(1, 20, 2, d, 16, seed=63)
    one.append([250])
    out = torch.full((100, 2 * G, d), 5.0, dtype=torch.bfloat16, device="cuda")
    one.gpu.attention(one.batch([2], max_rows=100, extra=98), q[:100], out=out)
    check_attention(one, [2], q[:2], q64[:2], out[:2], BF16)
    assert (out[2:] == 5).all()


def test_many_rows_that_see_nothing():
    torch = T()
    for d, G in ((64, 2), (128, 8)):
        rig = Rig(2, 20, 2, d, 16, seed=64)
        rig.append([40, 300])
        rows, lens = [100, 120], np.array([30, 300], np.int32)      # sequence 0 claims fewer tokens than rows
        q, q64 = rig.draw(220, 2 * G, d)
        out = f64(rig.gpu.attention(rig.batch(rows, lens=lens), q, out_dtype=torch.float32))
        assert (out[:70] == 0).all()
        rig.len = lens
        check_attention(rig, [30, 0], q[70:100], q64[70:100], torch.from_numpy(out[70:100]), F32)
        check_attention(rig, [0, 120], q[100:], q64[100:], torch.from_numpy(out[100:]), F32)


def test_rows_that_see_nothing_and_lengths_beyond_the_bounds():
    torch = T()
    rig = Rig(3, 4, 2, 64, 16, seed=23)
    rig.append([30, 20, 5])
    q, q64 = rig.draw(6, 4, 64)
    # sequence 0 claims one token for three rows: the first two see nothing; sequence 1 holds none at all
    lens = np.array([1, 0, 5], np.int32)
    out = rig.gpu.attention(rig.batch([3, 2, 1], lens=lens), q, out_dtype=torch.float32)
    got = f64(out)
    assert (got[:2] == 0).all() and (got[3:5] == 0).all() and not (got[2] == 0).all()
    rig.len = lens
    check_attention(rig, [0, 0, 1], q[5:], q64[5:], out[5:], F32)
    rig.len = np.array([1, 0, 0], np.int32)
    check_attention(rig, [1, 0, 0], q[2:3], q64[2:3], out[2:3], F32)
    # tokens beyond max_len are not looked at, rows beyond max_rows are left
    rig.len = np.array([30, 20, 5], np.int32)
    out = torch.full((3, 4, 64), 9.0, dtype=torch.float32, device="cuda")
    rig.gpu.attention(rig.batch([1, 1, 1], max_len=18), q[:3], out=out)
    rig.len = np.array([18, 18, 5], np.int32)
    check_attention(rig, [1, 1, 1], q[:3], q64[:3], out, F32)
    out.fill_(9.0)
    rig.len = np.array([30, 20, 5], np.int32)
    rig.gpu.attention(rig.batch([3, 0, 0], max_rows=2), q[:3], out=out)
    assert (out[2] == 9).all() and not (out[:2] == 9).any()


def test_no_numbers_in_what_a_row_does_not_see():
    torch = T()
    for G, rows in ((4, 5), (1, 3), (8, 24)):
        rig = Rig(1, 6, 2, 64, 16, seed=24)
        n = 50
        k, v = rig.draw(n, 2, 64), rig.draw(n, 2, 64)
        bad = n - 2                                       # the last row but one
        v[0][bad, 1, 3] = float("nan")
        k[0][bad, 0, 7] = float("inf")
        kv = ((k[0], f64(k[0])), (v[0], f64(v[0])))
        rig.append([n], kv=kv)
        q, q64 = rig.draw(rows, 2 * G, 64)
        out = rig.gpu.attention(rig.batch([rows]), q, out_dtype=torch.float32)
        got = f64(out)
        rig.len = np.array([n - 2], np.int32)
        check_attention(rig, [rows - 2], q[:-2], q64[:-2], out[:-2], F32)
        assert np.isnan(got[-2:, :G]).all()               # a key that is no number: every weight of the head
        assert np.isnan(got[-2:, G:, 3]).all() and np.isfinite(np.delete(got[-2:, G:], 3, axis=2)).all()


def test_page_ids_that_are_none_of_the_caches():
    torch = T()
    rig = Rig(2, 4, 2, 64, 16, seed=25)
    rig.append([50, 40])
    rig.table[0, 1], rig.table[1, 0] = -1, 10 ** 6
    rig.dtable = dev(rig.table)
    q, q64 = rig.draw(2, 8, 64)
    out = rig.gpu.attention(rig.batch([1, 1]), q, out_dtype=torch.float32)
    check_attention(rig, [1, 1], q, q64, out, F32)
    assert int(rig.status.item()) == 4
    rig.status.zero_()
    before = rig.codes.view(torch.uint8).clone()
    k, _ = rig.draw(2, 2, 64)
    rig.table[:] = -5
    rig.dtable = dev(rig.table)
    rig.gpu.append(rig.batch([1, 1]), k, k)
    assert torch.equal(before, rig.codes.view(torch.uint8)) and int(rig.status.item()) == 4


def test_a_cache_whose_offsets_pass_32_bits():
    torch = T()
    rig = Rig(1, 2, 1, 128, 16, seed=26)
    n_pages = (1 << 32) // (8 * 2 * 256 * 128) + 40       # over 4 GB of codes
    big = B.QCache.create(n_pages, 8, 128, 256)
    ref = O.Cache(2, 8, 128, 256)
    table = np.array([[n_pages - 1, n_pages - 9]], np.int32)
    k, v = rig.draw(300, 8, 128), rig.draw(300, 8, 128)
    batch = B.QBatch(dev(np.array([0, 300], np.int32)), dev(np.array([300], np.int32)), dev(table), 300, 300, 300)
    big.append(batch, k[0], v[0])
    ref.append([0, 1], 0, k[1], v[1])
    got = big.tensors[0].view(torch.uint8)[[n_pages - 1, n_pages - 9]].cpu().numpy()
    assert np.array_equal(got[0], ref.codes[0]) and np.array_equal(got[1][:, :, :44], ref.codes[1][:, :, :44])
    rig.ref, rig.table, rig.heads, rig.page, rig.len = ref, np.array([[0, 1]]), 8, 256, np.array([300])
    q, q64 = rig.draw(300, 32, 128)
    one = B.QBatch(dev(np.array([0, 1], np.int32)), dev(np.array([300], np.int32)), dev(table), 1, 1, 300)
    check_attention(rig, [1], q[:1], q64[:1], big.attention(one, q[:1].contiguous(), out_dtype=torch.float32), F32)
    pages = big.select(one, q[:1].contiguous(), 2, 0, 1)
    assert pages.cpu().numpy().tolist() == [[[0, 1]] * 8]


# ------------------------------------------------------------------------------------------------ selection and lists
@pytest.mark.parametrize("d,page,heads,G,dtype", [(128, 16, 8, 4, BF16), (64, 32, 2, 8, F16), (128, 64, 3, 1, BF16), (64, 16, 1, 7, BF16)])
@pytest.mark.parametrize("keep,first,recent", [(1, 0, 1), (5, 1, 2), (9, 0, 1), (9, 4, 5), (40, 2, 3)])
def test_selection_and_attention_over_it(d, page, heads, G, dtype, keep, first, recent):
    rig = Rig(3, 45, heads, d, page, seed=keep + d)
    rig.append([45 * page - 5, 20 * page + 1, 3])
    rows = [2, 3, 1]
    q, q64 = rig.draw(6, heads * G, d, dtype=dtype, scale=2.0)
    b = rig.batch(rows)
    pages = rig.gpu.select(b, q, keep, first, recent)
    got, at = pages.cpu().numpy(), 0
    for s, r in enumerate(rows):
        for i in range(r):
            for h in range(heads):
                want = rig.ref.select(rig.table[s], h, q64[at, h * G:(h + 1) * G], int(rig.len[s]) - r + i + 1, keep, first, recent)
                assert got[at, h].tolist() == want, (s, i, h)
            at += 1
    out = rig.gpu.attention(b, q, out_dtype=T().float32, pages=pages)
    check_attention(rig, rows, q, q64, out, F32, pages=got)


def test_equal_scores_go_to_the_lower_pages_and_many_pages():
    torch = T()
    rig = Rig(1, 9001, 1, 64, 16, seed=31)               # more pages than the selection keeps on chip
    n = 9001 * 16 - 3
    k = rig.rng.standard_normal((n, 1, 64)).astype(np.float32)
    k[16 * 100:16 * 8000] = np.tile(k[:16], (7900, 1, 1))  # pages 100 .. 7999 all alike
    k[16 * 100:16 * 8000] *= 4.0
    t = dev(k).to(torch.bfloat16)
    rig.append([n], kv=((t, f64(t)), (t, f64(t))))
    q, q64 = rig.draw(1, 4, 64)
    for keep in (50, 1000, 8500):
        got = rig.gpu.select(rig.batch([1]), q, keep, 3, 2).cpu().numpy()[0, 0].tolist()
        assert got == rig.ref.select(rig.table[0], 0, q64[0], n, keep, 3, 2)


def test_lists_in_any_order_with_gaps_and_nonsense():
    rig = Rig(2, 6, 2, 128, 16, seed=32)
    rig.append([90, 35])
    q, q64 = rig.draw(2, 8, 128)
    lists = np.array([[[5, -1, 0, 2], [1, 3, 9, -4]], [[2, 1, -1, 4], [-1, -1, -1, -1]]], np.int32)     # 9: not in the table; 4: beyond its tokens
    out = rig.gpu.attention(rig.batch([1, 1]), q, out_dtype=T().float32, pages=dev(lists))
    lists[0, 1, 2] = lists[1, 0, 3] = -1
    check_attention(rig, [1, 1], q, q64, out, F32, pages=lists)
    assert (f64(out)[1, 4:] == 0).all() and int(rig.status.item()) == 0


# ------------------------------------------------------------------------------------------------ together
def test_a_serving_run_prompt_tokens_drafts_and_sparse_steps():
    rig = Rig(3, 40, 2, 128, 16, seed=41)
    for rows in ([100, 1, 37], [1, 1, 1], [1, 250, 5], [3, 3, 3], [0, 1, 1], [1, 1, 1]):
        q, ref = rig.append(rows, theta=1e6, norm=True, q_heads=8)
        q64 = f64(q)
        b = rig.batch(rows)
        check_attention(rig, rows, q, q64, rig.gpu.attention(b, q), BF16)
        pages = rig.gpu.select(b, q, 4, 1, 1)
        check_attention(rig, rows, q, q64, rig.gpu.attention(b, q, pages=pages, out_dtype=T().float32), F32, pages=pages.cpu().numpy())
    rig.check()


@pytest.mark.parametrize("d,page,G,out", [(128, 16, 4, BF16), (64, 32, 8, F32), (128, 64, 3, F16)])
def test_long_chunks_among_single_tokens_and_sequences_without_rows(d, page, G, out):
    n = 70
    rig = Rig(n, 6 + 400 // page, 2, d, page, seed=44 + d)
    first = [1 + (7 * i) % 60 for i in range(n)]
    rig.append(first)
    rows = [1] * n
    rows[3], rows[17], rows[18], rows[40], rows[69] = 333, 0, 170, 20, 9
    q, ref = rig.append(rows, theta=1e4, norm=True, q_heads=2 * G)
    rig.check()
    q64 = f64(q)
    check_attention(rig, rows, q, q64, rig.gpu.attention(rig.batch(rows), q, out_dtype=getattr(T(), out)), out)


def test_more_sequences_than_a_block_has_threads():
    n = 1100
    rig = Rig(n, 12, 1, 64, 16, seed=45)
    first = [(5 * i) % 23 for i in range(n)]
    first[700] = 60
    rig.append(first)
    rows = [i % 3 % 2 for i in range(n)]
    rows[0], rows[511], rows[700], rows[1099] = 1, 100, 2, 70
    q, _ = rig.append(rows, theta=1e4, q_heads=2)
    rig.check()
    check_attention(rig, rows, q, f64(q), rig.gpu.attention(rig.batch(rows), q, out_dtype=T().float32), F32)
    b = rig.batch(rows)
    pages = rig.gpu.select(b, q, 3, 1, 1)
    check_attention(rig, rows, q, f64(q), rig.gpu.attention(b, q, pages=pages, out_dtype=T().float32), F32, pages=pages.cpu().numpy())


@pytest.mark.parametrize("far", [1.0, 1e3, 1e9, 1e30])
def test_a_page_of_far_larger_keys_leaves_the_others_in_order(far):
    """The bound on the first scores' errors goes by the largest scale: with a page far above the others it leaves all of them open."""
    rig = Rig(1, 420, 2, 64, 16, seed=46)
    rig.append([200 * 16])
    rig.append([16], scale=far)
    rig.append([200 * 16 - 3])
    rig.append([1], scale=1e-20)
    q, q64 = rig.draw(2, 8, 64)
    for keep in (2, 5, 150, 399):
        got = rig.gpu.select(rig.batch([2]), q, keep, 0, 1).cpu().numpy()
        for i in range(2):
            for h in range(2):
                assert got[i, h].tolist() == rig.ref.select(rig.table[0], h, q64[i, h * 4:h * 4 + 4], int(rig.len[0]) - 1 + i, keep, 0, 1), (keep, i, h)


@pytest.mark.parametrize("absent", [3, 40, 58])
def test_selection_where_pages_are_none_of_the_caches(absent):
    rig = Rig(1, 60, 1, 128, 16, seed=47)
    rig.append([60 * 16])
    gone = rig.rng.permutation(np.arange(1, 59))[:absent]
    rig.table[0, gone] = -1
    rig.dtable = dev(rig.table)
    q, q64 = rig.draw(1, 4, 128)
    for keep in (4, 20, 45):
        got = rig.gpu.select(rig.batch([1]), q, keep, 1, 1).cpu().numpy()[0, 0].tolist()
        assert got == rig.ref.select(rig.table[0], 0, q64[0], 960, keep, 1, 1)
    assert int(rig.status.item()) == 4


def test_queries_of_zeros_choose_the_first_pages():
    torch = T()
    rig = Rig(1, 600, 1, 64, 16, seed=48)
    rig.append([600 * 16])
    q = torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda")
    assert rig.gpu.select(rig.batch([1]), q, 7, 2, 1).cpu().numpy()[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 599]


def test_a_captured_step_is_replayed_with_other_lengths_on_another_stream():
    torch = T()
    rig = Rig(3, 30, 2, 64, 16, seed=42)
    rig.append([100, 33, 70])
    k, v, q = (torch.empty(3, n, 64, dtype=torch.bfloat16, device="cuda") for n in (2, 2, 8))
    seq_len = dev(rig.len)
    b = B.QBatch(dev(np.arange(4, dtype=np.int32)), seq_len, rig.dtable, 3, 1, 480)
    stream = torch.cuda.Stream()
    def step():
        qo = rig.gpu.append(b, k, v, q=q, rope_theta=1e4)
        pages = rig.gpu.select(b, qo, 3, 1, 1)
        return qo, rig.gpu.attention(b, qo, out_dtype=torch.float32), pages, rig.gpu.attention(b, qo, pages=pages, out_dtype=torch.float32)
    with torch.cuda.stream(stream):
        step()                                           # (sequence lengths unchanged: the newest token's row is overwritten below)
    stream.synchronize()
    rig.codes.view(torch.uint8).copy_(dev(rig.ref.codes))
    rig.scales.copy_(dev(np.ldexp(1.0, rig.ref.exps).astype(np.float32)))
    rig.bounds.view(torch.uint8).copy_(dev(rig.ref.bounds))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = step()
    for n in range(20):
        kk, k64 = rig.draw(3, 2, 64)
        vv, v64 = rig.draw(3, 2, 64)
        qq, q64 = rig.draw(3, 8, 64)
        with torch.cuda.stream(stream):
            k.copy_(kk); v.copy_(vv); q.copy_(qq); seq_len.add_(1)
            graph.replay()
        stream.synchronize()
        kr = O.norm_rotate(k64, None, 0, rig.len, 1e4)
        for s in range(3):
            rig.ref.append(rig.table[s], int(rig.len[s]), kr[s:s + 1], v64[s:s + 1])
        rig.len = rig.len + 1
        qo, dense, pages, sparse = outs
        check_attention(rig, [1, 1, 1], qo, f64(qo), dense, F32)
        check_attention(rig, [1, 1, 1], qo, f64(qo), sparse, F32, pages=pages.cpu().numpy())
    rig.check()


def test_two_streams_at_once():
    torch = T()
    rig = Rig(4, 300, 2, 128, 16, seed=43)
    rig.append([4000, 4001, 3000, 17])
    q, _ = rig.draw(4, 16, 128)
    b = rig.batch([1, 1, 1, 1])
    want = rig.gpu.attention(b, q, out_dtype=torch.float32)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(3)], []
    for i in range(30):
        with torch.cuda.stream(streams[i % 3]):
            outs.append(rig.gpu.attention(b, q, out_dtype=torch.float32))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_the_holder_refuses_what_the_kernels_could_not_read():
    torch = T()
    rig = Rig(1, 2, 2, 64, 16)
    b = rig.batch([1], lens=[1])
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (q.float(), q.cpu(), q[:, :, :32], torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"), q.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            rig.gpu.attention(b, bad)
    for kw in (dict(k=k[:, :1]), dict(v=k.half()), dict(positions=torch.zeros(1, device="cuda")), dict(k_weight=torch.ones(32, device="cuda")), dict(q_out=q)):
        with pytest.raises(ValueError):
            rig.gpu.append(b, **{"k": k, "v": k, **kw})
    for kw in (dict(pages=torch.zeros(1, 2, 3, device="cuda")), dict(pages=torch.zeros(1, 1, 3, dtype=torch.int32, device="cuda")),
               dict(out=torch.zeros(1, 4, 64, dtype=torch.int16, device="cuda")), dict(out=torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            rig.gpu.attention(b, q, **kw)
    with pytest.raises(B.GpError):
        rig.gpu.select(b, q, 2, 2, 1)
    with pytest.raises(B.GpError):
        rig.gpu.attention(b, torch.zeros(1, 18, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        B.QBatch(torch.zeros(2, device="cuda"), rig.dtable[0], rig.dtable, 1, 1, 1)
    with pytest.raises(ValueError):
        B.QCache(rig.codes.view(torch.uint8), rig.scales)


@pytest.mark.parametrize("d,G,rows", [(128, 4, 6), (128, 4, 7), (128, 8, 3), (128, 8, 4), (64, 4, 16), (64, 4, 17), (64, 8, 8), (64, 8, 9)])
def test_attention_at_the_border_between_few_and_many_rows(d, G, rows):
    rig = Rig(3, 20, 2, d, 16, seed=70 + rows)
    rig.append([rows, 200, 97])
    q, q64 = rig.draw(3 * rows, 2 * G, d)
    for out in (BF16, F32):
        check_attention(rig, [rows] * 3, q, q64, rig.gpu.attention(rig.batch([rows] * 3), q, out_dtype=getattr(T(), out)), out)


@pytest.mark.parametrize("d,G,out", [(128, 4, BF16), (64, 8, F32)])
@pytest.mark.parametrize("rows", [30, 150])
def test_many_rows_where_pages_are_none_of_the_caches(d, G, out, rows):
    """A page that is not there counts as not seen, wherever in a step it lies; all of a step, too."""
    rig = Rig(2, 40, 1, d, 16, seed=80 + rows)
    rig.append([40 * 16 - 5, 300])
    gone = [[0, 5, 8, 9, 10, 11, 21, 30, 31, 39], [2, 18]]
    q, q64 = rig.draw(2 * rows, G, d)
    held = np.full((2 * rows, 1, 40), -1)
    for s in range(2):
        rig.table[s, gone[s]] = [-1, 1 << 30] * (len(gone[s]) // 2)
        held[s * rows:(s + 1) * rows, 0, :] = [-1 if p in gone[s] else p for p in range(40)]
    rig.dtable = dev(rig.table)
    got = rig.gpu.attention(rig.batch([rows] * 2), q, out_dtype=getattr(T(), out))
    check_attention(rig, [rows] * 2, q, q64, got, out, held)
    assert int(rig.status.item()) == 4


def test_many_rows_of_many_short_sequences_and_of_half_tiles():
    """Several pieces a block, most of them with nothing in the tile's second half, some of one step."""
    rig = Rig(60, 16, 8, 128, 16, seed=90)
    rng = np.random.default_rng(1)
    rig.append(list(rng.integers(40, 250, 60)))
    rows = [int(min(r, n)) for r, n in zip(rng.integers(7, 90, 60), rig.len)]
    q, q64 = rig.draw(sum(rows), 32, 128)
    got = f64(rig.gpu.attention(rig.batch(rows), q, out_dtype=T().float32))
    # some of the sequences
    at = np.concatenate([[0], np.cumsum(rows)])
    for s in (0, 17, 59):
        one = Rig.__new__(Rig)
        one.__dict__.update(rig.__dict__)
        one.table, one.dtable, one.len = rig.table[s:s + 1], dev(rig.table[s:s + 1]), rig.len[s:s + 1]
        part = slice(at[s], at[s + 1])
        check_attention(one, [rows[s]], q[part], q64[part], dev(got[part].astype(np.float32)), F32)
