"""What the paged-cache operators and the verification refuse, before anything is enqueued: runs without a GPU."""
import ctypes as C

import pytest

INVALID, SHAPE, CAPACITY = 1, 2, 3


@pytest.fixture(scope="module")
def b():
    from paper_2312_11462_b200 import build
    build.build()
    from paper_2312_11462_b200 import binding
    return binding


def pool(b, **kw):
    f = dict(kind=0, n_pages=8, page_size=16, n_kv_heads=2, d_head=128, k_dev=1 << 20, v_dev=1 << 21, k_exp_dev=None, v_exp_dev=None)
    f.update(kw)
    return b.KvPoolStruct(*f.values())


def batch(b, **kw):
    f = dict(n_seqs=2, max_pages=4, total_rows=4, max_rows=2, page_table_dev=4096, row_start_dev=4096, kv_len_dev=4096)
    f.update(kw)
    return b.PagedBatchStruct(*f.values())


BAD_POOLS = [(dict(kind=2), INVALID), (dict(n_pages=0), INVALID), (dict(page_size=24), SHAPE), (dict(page_size=8), SHAPE), (dict(page_size=256), SHAPE),
             (dict(page_size=0), SHAPE), (dict(n_kv_heads=0), INVALID), (dict(d_head=96), SHAPE), (dict(d_head=32), SHAPE), (dict(k_dev=None), INVALID),
             (dict(v_dev=None), INVALID), (dict(k_dev=(1 << 20) + 8), INVALID), (dict(kind=1), INVALID), (dict(kind=1, k_exp_dev=4096), INVALID),
             (dict(kind=1, k_exp_dev=4096, v_exp_dev=4104), INVALID),
             (dict(n_pages=1 << 26), SHAPE)]
BAD_BATCHES = [(dict(n_seqs=0), INVALID), (dict(n_seqs=1025), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=1 << 27), INVALID),
               (dict(total_rows=-1), INVALID), (dict(max_rows=0), INVALID), (dict(page_table_dev=None), INVALID), (dict(row_start_dev=None), INVALID),
               (dict(kv_len_dev=None), INVALID)]


def every_call(b, p, q, **kw):
    """Status of the three calls on a pool and a batch, with addresses that no kernel is meant to see."""
    L = b.lib
    p, q = C.byref(p) if p else None, C.byref(q) if q else None
    f = dict(rows=1 << 16, out=1 << 17, ld=256, type=0, heads=4, ldq=512, scale=0.1, tree=None, ws=1 << 18, ws_bytes=1 << 40)
    f.update(kw)
    return [L.csd_paged_append(p, q, f["rows"], f["out"], f["ld"], f["type"], None), L.csd_paged_read(p, q, f["rows"], f["out"], f["ld"], f["type"], None),
            L.csd_paged_attention(p, q, f["rows"], f["ldq"], f["heads"], f["type"], f["scale"], f["tree"], f["out"], f["ldq"], f["ws"], f["ws_bytes"], None)]


@pytest.mark.parametrize("kw,code", BAD_POOLS)
def test_pools(b, kw, code):
    assert every_call(b, pool(b, **kw), batch(b)) == [code] * 3
    assert b.lib.csd_paged_attention_workspace_bytes(C.byref(pool(b, **kw)), C.byref(batch(b)), 4, 0) == 0


@pytest.mark.parametrize("kw,code", BAD_BATCHES)
def test_batches(b, kw, code):
    assert every_call(b, pool(b), batch(b, **kw)) == [code] * 3
    assert b.lib.csd_paged_attention_workspace_bytes(C.byref(pool(b)), C.byref(batch(b, **kw)), 4, 0) == 0


def test_rows(b):
    assert every_call(b, None, batch(b)) == [INVALID] * 3
    assert every_call(b, pool(b), None) == [INVALID] * 3
    assert every_call(b, pool(b), batch(b), type=2) == [INVALID] * 3
    assert every_call(b, pool(b), batch(b), rows=None) == [INVALID] * 3
    assert every_call(b, pool(b), batch(b), out=None) == [INVALID] * 3
    assert every_call(b, pool(b), batch(b), rows=(1 << 16) + 4) == [INVALID] * 3
    assert every_call(b, pool(b), batch(b), ld=248, ldq=504) == [INVALID] * 3        # shorter than a row
    assert every_call(b, pool(b), batch(b), ld=260, ldq=516) == [INVALID] * 3        # rows off their boundary


def test_attention_alone(b):
    call = lambda **kw: every_call(b, pool(b), kw.pop("batch", batch(b)), **kw)[2]  # noqa: E731
    assert call(heads=3) == SHAPE                       # not a multiple of the pool's
    assert call(heads=0) == SHAPE
    assert call(heads=2 * 65, ldq=2 * 65 * 128) == SHAPE
    assert call(scale=float("nan")) == INVALID
    assert call(scale=float("inf")) == INVALID
    assert call(tree=4096, batch=batch(b, max_rows=65)) == INVALID
    assert call(ws=None) == INVALID
    assert call(ws=(1 << 18) + 16) == INVALID
    assert call(ws_bytes=16) == CAPACITY
    assert b.lib.csd_paged_attention_workspace_bytes(C.byref(pool(b)), C.byref(batch(b)), 3, 0) == 0
    assert b.lib.csd_paged_attention_workspace_bytes(C.byref(pool(b)), C.byref(batch(b)), 4, 2) == 0
    assert b.lib.csd_paged_attention_workspace_bytes(C.byref(pool(b)), C.byref(batch(b)), 4, 0) > 0


def test_sizes_that_pass_32_bits(b):
    """More (row, query head) pairs or key tiles than the division of the work counts."""
    big = batch(b, max_rows=1 << 29)
    assert every_call(b, pool(b), big, heads=8, ldq=1024)[2] == CAPACITY
    wide = pool(b, n_pages=1, n_kv_heads=1 << 16, page_size=16)
    assert every_call(b, wide, batch(b, max_pages=1 << 25), ld=128 << 16, heads=1 << 16, ldq=128 << 16)[2] == CAPACITY


def test_review_forward_paged(b):
    """Without a model, pools or a batch: nothing is looked at."""
    L, p, q = b.lib, C.byref(pool(b)), C.byref(batch(b))
    assert L.csd_review_forward_paged(None, p, q, 4096, None, 4096, 1 << 18, 1 << 40, None) == INVALID
    assert L.csd_review_forward_paged(1 << 20, None, q, 4096, None, 4096, 1 << 18, 1 << 40, None) == INVALID
    assert L.csd_review_forward_paged(1 << 20, p, None, 4096, None, 4096, 1 << 18, 1 << 40, None) == INVALID


def test_no_rows(b):
    """Nothing to do: no pointers are looked at."""
    assert every_call(b, pool(b), batch(b, total_rows=0), rows=None, out=None) == [0] * 3


def test_verify(b):
    L = b.lib

    def call(p=4096, ldp=64, q=4096, ldq=64, type=0, x=4096, n=4096, u=4096, rows=2, k=3, V=64, a=4096, out=4096):
        return L.csd_spec_verify(p, ldp, q, ldq, type, x, n, u, rows, k, V, a, out, None)
    assert call(rows=0) == 0
    for kw in (dict(rows=-1), dict(k=-1), dict(k=65), dict(V=0), dict(type=2), dict(type=-1), dict(p=None), dict(x=None), dict(u=None), dict(a=None), dict(out=None),
               dict(ldp=63), dict(ldq=63)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(V=(1 << 30) + 1, ldp=1 << 31, ldq=1 << 31), dict(p=4098), dict(q=4097, type=1)):      # too wide, laws between their entries' boundaries
        assert call(**kw) == INVALID, kw
    assert b.lib.csd_status_string(9) == b"page id outside the pool"


def test_struct_sizes(b):
    assert C.sizeof(b.KvPoolStruct) == 24 + 4 * 8 and C.sizeof(b.PagedBatchStruct) == 16 + 3 * 8
