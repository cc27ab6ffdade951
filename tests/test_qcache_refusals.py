"""What the calls of the 8-bit cache refuse, before anything is launched: no GPU is needed (the pointers are never followed)."""
import ctypes as C
import os
import re

import pytest

from paper_2609_03494_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20                                              # an aligned address


def _cache(**kw):
    c = B.gp_qcache(8, 128, 16, 0, 100, A, A, A, A)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _batch(**kw):
    b = B.gp_qbatch(A, A, A, 4, 10, 4, 1, 160, 0)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def _rows(**kw):
    r = B.gp_qrows(k=A, v=A, q=A, q_out=2 * A, k_stride=1024, v_stride=1024, q_stride=4096, q_out_stride=4096, positions=A, q_weight=A, k_weight=A,
                   eps=1e-6, rope_theta=1e4, n_q_heads=32, type=B.GP_TYPE_BF16)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def append(cache=None, batch=None, rows=None):
    return B.lib().gp_qcache_append(C.byref(cache or _cache()), C.byref(batch or _batch()), C.byref(rows or _rows()), None)


def attention(cache=None, batch=None, q=A, stride=4096, hq=32, type=0, pages=None, n_list=0, out=A, out_type=0, work=A, nbytes=1 << 40):
    return B.lib().gp_qcache_attention(C.byref(cache or _cache()), C.byref(batch or _batch()), q, stride, hq, type, pages, n_list, out, out_type, work,
                                       nbytes, None)


def select(cache=None, batch=None, q=A, stride=4096, hq=32, type=0, keep=4, first=1, recent=1, pages=A, work=A, nbytes=1 << 40):
    return B.lib().gp_qcache_select(C.byref(cache or _cache()), C.byref(batch or _batch()), q, stride, hq, type, keep, first, recent, pages, work,
                                    nbytes, None)


BAD_CACHE = [dict(n_kv_heads=0), dict(head_dim=96), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(n_pages=0), dict(device=-1),
             dict(codes=None), dict(scales=None), dict(codes=A + 8), dict(scales=A + 4), dict(bounds=A + 8), dict(status=A + 2)]
BAD_BATCH = [dict(n_seq=-1), dict(table_stride=0), dict(n_rows=-1), dict(max_rows=-1), dict(max_len=-1), dict(reserved=1), dict(row_start=None),
             dict(seq_len=None), dict(page_table=None), dict(page_table=A + 2)]


@pytest.mark.parametrize("call", [append, attention, select])
def test_bad_caches_and_batches(call):
    for kw in BAD_CACHE:
        assert call(cache=_cache(**kw)) == B.GP_ERR_INVALID, kw
    for kw in BAD_BATCH:
        assert call(batch=_batch(**kw)) == B.GP_ERR_INVALID, kw


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2), dict(k_stride=1016), dict(v_stride=1028), dict(type=2), dict(type=-1),
                                dict(positions=A + 1), dict(eps=-1.0), dict(eps=float("nan")), dict(rope_theta=-1.0), dict(rope_theta=float("inf")),
                                dict(q_out=None), dict(q=A + 8), dict(q_out=A + 8), dict(q_stride=4092), dict(q_out_stride=4088), dict(n_q_heads=0),
                                dict(n_q_heads=30), dict(n_q_heads=72), dict(q_out=A, q_out_stride=8192), dict(q_weight=A + 2), dict(k_weight=A + 1)])
def test_bad_rows(kw):
    assert append(rows=_rows(**kw)) == B.GP_ERR_INVALID


@pytest.mark.parametrize("kw", [dict(q=None), dict(q=A + 8), dict(stride=4095), dict(stride=4088), dict(hq=30), dict(hq=72), dict(hq=0), dict(type=2), dict(out=None),
                                dict(out=A + 8), dict(out_type=3), dict(pages=A, n_list=0), dict(pages=None, n_list=3), dict(pages=A + 2, n_list=4),
                                dict(pages=A, n_list=1 << 28)])
def test_bad_attention(kw):
    assert attention(**kw) == B.GP_ERR_INVALID


@pytest.mark.parametrize("kw", [dict(q=None), dict(stride=4094), dict(hq=12), dict(type=2), dict(keep=0), dict(first=-1), dict(recent=0), dict(keep=3, first=2, recent=2),
                                dict(pages=None), dict(pages=A + 2), dict(work=None), dict(work=A + 8), dict(nbytes=1), dict(cache=_cache(bounds=None))])
def test_bad_selections(kw):
    assert select(**kw) == B.GP_ERR_INVALID


def test_work_memory_that_is_too_small_is_refused():
    long = _batch(n_seq=1, n_rows=1, table_stride=8192, max_len=131072)
    need = B.gp_qcache_attention_bytes(_cache(), long, 32, 0)
    assert need > 0
    assert attention(batch=long, nbytes=need - 1) == B.GP_ERR_INVALID and attention(batch=long, work=None) == B.GP_ERR_INVALID


@pytest.mark.parametrize("kw", [dict(n_seq=0), dict(n_rows=0), dict(max_rows=0)])
def test_an_empty_batch_is_nothing_to_do(kw):
    b = _batch(**kw)
    if not kw.get("max_rows", 1):
        assert append(batch=b) == attention(batch=b) == select(batch=b) == B.GP_OK
        return
    b.row_start = b.seq_len = b.page_table = None
    assert append(batch=b, rows=_rows(k=None, v=None, q=None, q_out=None, positions=None)) == B.GP_OK
    assert attention(batch=b, q=None, out=None, work=None, nbytes=0) == B.GP_OK
    assert select(batch=b, q=None, pages=None, work=None, nbytes=0) == B.GP_OK


def test_structs_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "growpage.h")).read(), flags=re.S)
    for name in ("gp_qcache", "gp_qbatch", "gp_qrows"):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
        fields = [n.strip(" *") for decl in body.split(";") if decl.strip() for n in re.sub(r"^\s*(const\s+)?\w+", "", decl).split(",")]
        assert fields == [f[0] for f in getattr(B, name)._fields_], name


def test_withheld_hand_overs_are_numbered():
    for what, cycles in ((-1, 0), (4, 0), (1, -1)):
        assert B.lib().gp_qcache_test_withhold(what, cycles) == B.GP_ERR_INVALID
    assert B.lib().gp_qcache_test_withhold(0, 0) == B.GP_OK


@pytest.mark.parametrize("call", [append, attention, select])
def test_slots_that_would_pass_31_bits_are_refused(call):
    """A table of 2^31 tokens with a bound as large: indexes are added up in 32 bits."""
    assert call(cache=_cache(page_size=256), batch=_batch(table_stride=1 << 23, max_len=(1 << 31) - 1)) == B.GP_ERR_TOO_LARGE
    assert call(cache=_cache(page_size=256), batch=_batch(table_stride=1 << 24, max_len=(1 << 31) - (1 << 16) + 1)) == B.GP_ERR_TOO_LARGE


def test_lists_that_would_pass_31_bits_are_refused():
    c = _cache(page_size=256)
    assert attention(cache=c, pages=A, n_list=(1 << 23) - 255) == B.GP_ERR_INVALID
    assert B.gp_qcache_attention_bytes(c, _batch(), 32, (1 << 23) - 256) > 0
