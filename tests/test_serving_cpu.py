"""What the entry points for sequences of different lengths refuse, all on the
host before anything is enqueued: no GPU is needed."""
import ctypes

import pytest

INVALID = 1


@pytest.fixture(scope="module")
def T():
    import __graft_entry__ as g
    g.build()
    from paper_2609_37924_gb300 import tadm
    return tadm


P = 1 << 20          # stands for an aligned device pointer; no refused call follows it


def pool(T, **over):
    a = dict(k=P, v=P, k_scale=P, v_scale=P, layers=2, pages=8, n_kv_heads=4, head_dim=64)
    a.update(over)
    return T.tadm_page_pool(*a.values())


PACKED = dict(q=P, k=P, v=P, o=P, cu=P, batch=2, total=10, max_rows=8, heads=8, kv=4, hd=64, ldq=512, ldk=256, ldv=256,
              ldo=512, causal=1, window=0, dtype=1, stream=None)


@pytest.mark.parametrize("over", [
    dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(cu=None), dict(q=P + 8), dict(o=P + 2), dict(batch=-1),
    dict(total=-1), dict(max_rows=-1), dict(heads=0), dict(kv=0), dict(heads=6), dict(hd=32), dict(hd=96), dict(ldq=504),
    dict(ldk=255), dict(ldq=516), dict(ldv=260), dict(ldo=511), dict(causal=2), dict(window=-1), dict(dtype=2),
    dict(dtype=-1)])
def test_packed_attention_refuses(T, over):
    assert T.load_library().tadm_attention_packed(*{**PACKED, **over}.values()) == INVALID


@pytest.mark.parametrize("over", [dict(batch=0), dict(batch=0, cu=None), dict(total=0), dict(max_rows=0)])
def test_empty_calls_do_nothing(T, over):
    assert T.load_library().tadm_attention_packed(*{**PACKED, **over}.values()) == 0


ROWS = dict(layer=0, k=P, v=P, cu=P, start=P, batch=2, total=10, max_rows=8, ldk=256, ldv=256, table=P, ld_table=4, dtype=1,
            stream=None)
POOLS = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=P + 4), dict(v=P + 8),
         dict(k_scale=P + 2), dict(layers=0), dict(pages=-1), dict(pages=0), dict(n_kv_heads=0), dict(head_dim=32), dict(head_dim=256)]


@pytest.mark.parametrize("name", ["tadm_page_write", "tadm_page_read"])
@pytest.mark.parametrize("over", [
    dict(layer=-1), dict(layer=2), dict(k=None), dict(v=None), dict(cu=None), dict(start=None), dict(batch=-1),
    dict(total=-1), dict(max_rows=-1), dict(ldk=255), dict(ldv=252), dict(k=P + 8), dict(table=None), dict(ld_table=-1),
    dict(ld_table=(1 << 20) + 1), dict(dtype=3)])
def test_page_rows_refuse(T, name, over):
    f, c = getattr(T.load_library(), name), pool(T)
    assert f(ctypes.addressof(c), *{**ROWS, **over}.values()) == INVALID
    assert f(None, *ROWS.values()) == INVALID


@pytest.mark.parametrize("over", POOLS)
def test_pools_are_checked(T, over):
    lib, c = T.load_library(), pool(T, **over)
    assert lib.tadm_page_write(ctypes.addressof(c), *ROWS.values()) == INVALID
    assert lib.tadm_pages_copy(ctypes.addressof(c), P, P, 3, None) == INVALID
    assert lib.tadm_page_attention(P, ctypes.addressof(c), *ATTEND.values()) == INVALID


ATTEND = dict(layer=0, o=P, cu=P, lens=P, batch=2, total=10, max_rows=8, max_len=200, heads=8, ldq=512, ldo=512, table=P,
              ld_table=4, causal=0, window=0, dtype=1, scratch=P, scratch_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("over", [
    dict(layer=2), dict(layer=-1), dict(o=None), dict(cu=None), dict(lens=None), dict(batch=-1), dict(total=-1),
    dict(max_rows=-1), dict(max_len=-1), dict(max_len=257), dict(heads=0), dict(heads=6), dict(ldq=504), dict(ldo=516),
    dict(table=None), dict(ld_table=-1), dict(causal=-1), dict(window=-1), dict(dtype=2)])
def test_page_attention_refuses(T, over):
    c = pool(T)
    assert T.load_library().tadm_page_attention(P, ctypes.addressof(c), *{**ATTEND, **over}.values()) == INVALID


def test_page_attention_scratch(T):
    need = T.tadm_page_attention_scratch_size(2, 10, 8, 200, 8, 4, 64, 1)
    c = pool(T)
    if need:
        for over in (dict(scratch=None), dict(scratch=P + 8), dict(scratch_bytes=need - 1)):
            assert T.load_library().tadm_page_attention(P, ctypes.addressof(c), *{**ATTEND, **over}.values()) == INVALID
    n = ctypes.c_size_t()
    f = T.load_library().tadm_page_attention_scratch_size
    for bad in ((-1, 10, 8, 200, 8, 4, 64, 1), (2, 10, 8, 200, 6, 4, 64, 1), (2, 10, 8, 200, 8, 4, 65, 1), (2, 10, 8, 200, 8, 4, 64, 2)):
        assert f(*bad, ctypes.byref(n)) == INVALID
    assert f(2, 10, 8, 200, 8, 4, 64, 1, None) == INVALID


SEQS = dict(tables=P, lens=P, refs=P, pages=8, n_seqs=4, ld=4, list=P, n=2, tables_out=P, lens_out=P, refs_out=P, status=P,
            scratch=P, scratch_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("over", [
    dict(tables=None), dict(lens=None), dict(refs=None), dict(pages=-1), dict(n_seqs=-1), dict(ld=-1), dict(ld=(1 << 20) + 1),
    dict(list=None), dict(n=-1), dict(n=5), dict(tables_out=None), dict(lens_out=None), dict(refs_out=None), dict(status=None),
    dict(scratch=None), dict(scratch=P + 4), dict(scratch_bytes=100)])
def test_bookkeeping_refuses(T, over):
    lib, a, c = T.load_library(), {**SEQS, **over}, pool(T)
    assert lib.tadm_pages_free(*a.values()) == INVALID
    if "lens" not in over and "lens_out" not in over:
        assert lib.tadm_pages_reserve(a["tables"], a["refs"], a["pages"], a["n_seqs"], a["ld"], a["list"], P, a["n"],
                                      a["tables_out"], a["refs_out"], a["status"], a["scratch"], a["scratch_bytes"],
                                      None) == INVALID
    if "pages" not in over:
        assert lib.tadm_pages_fork(ctypes.addressof(c), a["tables"], a["lens"], a["refs"], a["n_seqs"], a["ld"], a["list"],
                                   P, a["n"], a["tables_out"], a["lens_out"], a["refs_out"], a["status"], a["scratch"],
                                   a["scratch_bytes"], None) == INVALID
    if not {"pages", "list", "n", "lens", "lens_out"} & set(over):
        assert lib.tadm_pages_compact(ctypes.addressof(c), a["tables"], a["refs"], a["n_seqs"], a["ld"], a["tables_out"],
                                      a["refs_out"], a["status"], a["scratch"], a["scratch_bytes"], None) == INVALID


def test_bookkeeping_needs_its_lists(T):
    lib, a, c = T.load_library(), SEQS, pool(T)
    assert lib.tadm_pages_reserve(P, P, 8, 4, 4, P, None, 2, P, P, P, P, 1 << 40, None) == INVALID
    assert lib.tadm_pages_fork(ctypes.addressof(c), P, P, P, 4, 4, P, None, 2, P, P, P, P, P, 1 << 40, None) == INVALID
    assert lib.tadm_pages_copy(ctypes.addressof(c), None, P, 1, None) == INVALID
    assert lib.tadm_pages_copy(ctypes.addressof(c), P, P, -1, None) == INVALID
    assert lib.tadm_pages_copy(None, P, P, 1, None) == INVALID
    assert lib.tadm_pages_scratch_size(-1, 4, ctypes.byref(ctypes.c_size_t())) == INVALID
    assert lib.tadm_pages_scratch_size(4, 4, None) == INVALID
    assert a["pages"] == c.pages


UNSUPPORTED = 2


def test_sizes_beyond_the_grids(T):
    """Well-formed calls that no kernel takes, and their neighbours in range that have nothing to do."""
    lib, c = T.load_library(), pool(T)
    many = dict(heads=4 * 129, ldq=4 * 129 * 64, ldo=4 * 129 * 64)
    assert lib.tadm_attention_packed(*{**PACKED, **many}.values()) == UNSUPPORTED
    assert lib.tadm_attention_packed(*{**PACKED, **many, "total": 0}.values()) == 0
    wide = dict(heads=16384, kv=16384, ldq=16384 * 64, ldk=16384 * 64, ldv=16384 * 64, ldo=16384 * 64, total=1 << 27, max_rows=1 << 27)
    assert lib.tadm_attention_packed(*{**PACKED, **wide}.values()) == UNSUPPORTED
    tall = dict(total=1 << 30, max_rows=1 << 30)              # 2 query heads per KV head: 2^31 rows of one
    assert lib.tadm_attention_packed(*{**PACKED, **tall, "dtype": 0}.values()) == UNSUPPORTED
    assert lib.tadm_page_attention(P, ctypes.addressof(c), *{**ATTEND, **tall}.values()) == UNSUPPORTED
    for f in (lib.tadm_page_write, lib.tadm_page_read):
        assert f(ctypes.addressof(c), *{**ROWS, "batch": 65536}.values()) == UNSUPPORTED
        assert f(ctypes.addressof(c), *{**ROWS, "batch": 65536, "max_rows": 0}.values()) == 0
