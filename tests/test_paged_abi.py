"""Host-side checks of the paged-cache and beam entry points: struct layouts and refusals, which fail before any
launch (no GPU is needed; the addresses below are never dereferenced)."""
import ctypes as C
import os

import pytest

from paper_2609_13804_gb300 import binding as b

INVALID, SHAPE, ALIGN, WORKSPACE = 1, 2, 3, 4
OK = 256  # an address


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(b.LIB_PATH):
        from paper_2609_13804_gb300 import build
        build.build()
    return b.lib()


def cache(**k):
    return b.sp_paged_kv(**dict(dict(kv=OK, n_pages=8, page_size=16, table=OK, max_pages=4, lens=OK), **k))


def append(**k):
    c = k.pop("cache", None) or cache()
    d = dict(B=2, T_cap=2, qkv=OK, ld=512, q_out=OK, ld_q=256, n_heads=4, n_kv_heads=2, head_dim=64, rope=OK, max_pos=9,
             pos=OK, cache=c)
    return b.sp_paged_append_io(**dict(d, **k))


def attend(**k):
    c = k.pop("cache", None) or cache()
    d = dict(B=2, T_cap=2, q=OK, ld_q=256, out=512, ld_out=256, n_heads=4, n_kv_heads=2, head_dim=64, cache=c)
    return b.sp_prefix_attention_io(**dict(d, **k))


def select(**k):
    d = dict(B=2, W=3, V=100, logits=OK, logits_f32=1, ld=100, cum=OK, n_out=3, score=OK, parent=OK, token=OK)
    return b.sp_beam_select_io(**dict(d, **k))


def reorder(**k):
    d = dict(B=2, W=3, n_layers=2, kv=OK, n_pages=9, page_size=16, row_elems=64, table=OK, own_table=512, max_pages=3,
             lens=OK, parent=OK, ld_parent=3)
    return b.sp_beam_reorder_io(**dict(d, **k))


def test_layouts():
    assert C.sizeof(b.sp_paged_kv) == 8 + 4 * 2 + 8 + 4 + 4 + 8
    assert C.sizeof(b.sp_paged_append_io) == 4 * 2 + 8 * 5 + 4 * 3 + 4 + 8 + 4 + 4 + 8 * 2 + 4 * 3 + 4 + 40 + 8
    assert C.sizeof(b.sp_prefix_attention_io) == 4 * 2 + 8 * 6 + 4 * 4 + 40 + 4 + 4 + 8 * 2 + 4 + 4 + 8 * 2
    assert C.sizeof(b.sp_beam_select_io) == 4 * 3 + 4 + 8 + 4 + 4 + 8 * 3 + 4 * 2 + 8 * 3
    assert C.sizeof(b.sp_beam_reorder_io) == 4 * 3 + 4 + 8 + 4 * 3 + 4 + 8 * 2 + 4 + 4 + 8 * 2 + 4 + 4 + 8


@pytest.mark.parametrize("want,change", [
    (SHAPE, dict(head_dim=96)), (SHAPE, dict(n_kv_heads=3)), (SHAPE, dict(n_kv_heads=0)), (SHAPE, dict(B=0)),
    (SHAPE, dict(B=257, T_cap=257)), (SHAPE, dict(T_cap=3)), (SHAPE, dict(T_cap=-1, cu_rows=OK)), (INVALID, dict(qkv=None)),
    (SHAPE, dict(ld=504)), (SHAPE, dict(ld=516)), (SHAPE, dict(ld_q=248)), (SHAPE, dict(ld_q=260)), (ALIGN, dict(qkv=264)),
    (ALIGN, dict(q_out=264)), (ALIGN, dict(rope=264)), (INVALID, dict(pos=None)), (INVALID, dict(pos3=OK)),
    (SHAPE, dict(max_pos=0)), (SHAPE, dict(pos=None, pos3=OK)),
    (SHAPE, dict(pos=None, pos3=OK, mrope_section=(C.c_int * 3)(11, 11, 10))),
    (SHAPE, dict(pos=None, pos3=OK, mrope_section=(C.c_int * 3)(16, 8, 10))),
    (SHAPE, dict(cache=cache(page_size=24))), (SHAPE, dict(cache=cache(page_size=8))), (SHAPE, dict(cache=cache(n_pages=0))),
    (SHAPE, dict(cache=cache(page_size=1024, n_pages=1 << 21))), (SHAPE, dict(cache=cache(max_pages=0))),
    (INVALID, dict(cache=cache(kv=None))), (INVALID, dict(cache=cache(table=None))), (ALIGN, dict(cache=cache(kv=264))),
])
def test_append_refusals(L, want, change):
    assert L.sp_paged_append(C.byref(append(**change)), None) == want


@pytest.mark.parametrize("want,change", [
    (SHAPE, dict(head_dim=256)), (SHAPE, dict(n_heads=5)), (SHAPE, dict(B=0)), (SHAPE, dict(T_cap=3)),
    (SHAPE, dict(n_groups=-1)), (SHAPE, dict(n_groups=257)), (SHAPE, dict(n_groups=1, prefix_max_pages=0)),
    (INVALID, dict(n_groups=1, prefix_max_pages=1)), (INVALID, dict(q=None)), (INVALID, dict(out=None)),
    (INVALID, dict(cache=cache(lens=None))), (SHAPE, dict(ld_q=248)), (SHAPE, dict(ld_out=260)), (ALIGN, dict(q=264)),
    (ALIGN, dict(out=264)), (INVALID, dict(scale=-1.0)), (INVALID, dict(scale=float("nan"))),
    (INVALID, dict(scale=float("inf"))), (SHAPE, dict(cache=cache(page_size=48))), (WORKSPACE, dict()),
])
def test_attention_refusals(L, want, change):
    assert L.sp_prefix_attention(C.byref(attend(**change)), OK, 64, None) == want
    assert L.sp_prefix_attention(C.byref(attend(**change)), None, 1 << 40, None) == want


@pytest.mark.parametrize("want,change", [
    (SHAPE, dict(B=0)), (SHAPE, dict(W=0)), (SHAPE, dict(W=17)), (SHAPE, dict(V=0)), (SHAPE, dict(n_out=0)),
    (SHAPE, dict(n_out=33)), (SHAPE, dict(ld=99)), (INVALID, dict(logits=None)), (INVALID, dict(cum=None)),
    (INVALID, dict(score=None)), (INVALID, dict(parent=None)), (INVALID, dict(token=None)),
    (INVALID, dict(done=OK, eos=100)), (INVALID, dict(done=OK, eos=-1)), (ALIGN, dict(logits=258)),
    (ALIGN, dict(logits=257, logits_f32=0)), (WORKSPACE, dict()),
])
def test_select_refusals(L, want, change):
    assert L.sp_beam_select(C.byref(select(**change)), OK, 64, None) == want
    assert L.sp_beam_select(C.byref(select(**change)), None, 1 << 40, None) == want


@pytest.mark.parametrize("want,change", [
    (SHAPE, dict(B=0)), (SHAPE, dict(W=17, ld_parent=17)), (SHAPE, dict(ld_parent=2)), (SHAPE, dict(n_layers=0)),
    (SHAPE, dict(n_layers=97)), (SHAPE, dict(row_elems=12)), (SHAPE, dict(row_elems=0)), (SHAPE, dict(page_size=17)),
    (SHAPE, dict(n_pages=0)), (SHAPE, dict(max_pages=0)), (INVALID, dict(kv=None)), (INVALID, dict(table=None)),
    (INVALID, dict(own_table=None)), (INVALID, dict(own_table=OK)), (INVALID, dict(lens=None)),
    (INVALID, dict(parent=None)), (ALIGN, dict(kv=264)),
])
def test_reorder_refusals(L, want, change):
    assert L.sp_beam_reorder(C.byref(reorder(**change)), None) == want


def test_decode_paged_layout_and_null(L):
    assert C.sizeof(b.sp_decode_paged_io) == 8 * 4 + 40 + 4 + 4 + 8 * 2 + 4 + 4 + 8 * 3
    assert L.sp_decode_paged(None, None, None, 0, None) == INVALID
    assert L.sp_prefill_paged(None, None, None, None, 0, None) == INVALID
    assert L.sp_decode_paged_workspace(None, 4, 0) == 0


def test_packed_arguments_are_the_structs(L):
    """The binding packs arguments with struct: the bytes are those of the ctypes structures."""
    io = reorder()
    packed = b._pack_reorder(2, 3, 2, OK, 9, 16, 64, OK, 512, 3, OK, OK, 3, 0)
    assert packed == bytes(io)
    io = attend(scale=0.5, n_groups=3, group_cu=OK, prefix_table=OK, prefix_max_pages=7, prefix_lens=OK)
    packed = b._pack_attention(2, 2, 0, OK, 256, 512, 256, 0, 4, 2, 64, 0.5, OK, 8, 16, OK, 4, OK, 3, OK, OK, 7, OK, 0)
    assert packed == bytes(io)
    io = append(mrope_section=(C.c_int * 3)(1, 2, 3))
    packed = b._pack_append(2, 2, 0, OK, 512, OK, 256, 4, 2, 64, OK, 9, OK, 0, 1, 2, 3, OK, 8, 16, OK, 4, OK, 0)
    assert packed == bytes(io)
    assert b._pack_select(2, 3, 100, OK, True, 100, OK, 0, 0, 3, OK, OK, OK) == bytes(select())


def test_no_rows_is_nothing_to_do(L):
    assert L.sp_paged_append(C.byref(append(T_cap=0, cu_rows=OK, qkv=None, q_out=None)), None) == 0
    assert L.sp_prefix_attention(C.byref(attend(T_cap=0, cu_rows=OK, q=None, out=None)), None, 0, None) == 0


def test_null_and_workspace_queries(L):
    assert L.sp_paged_append(None, None) == INVALID
    assert L.sp_prefix_attention(None, None, 0, None) == INVALID
    assert L.sp_beam_select(None, None, 0, None) == INVALID
    assert L.sp_beam_reorder(None, None) == INVALID
    assert L.sp_prefix_attention_workspace(4, 4, 1, 4, 3, 64) == 0
    assert L.sp_prefix_attention_workspace(4, 0, 1, 4, 2, 64) == 0
    assert L.sp_prefix_attention_workspace(0, 1, 0, 4, 2, 64) > 0
    assert L.sp_beam_select_workspace(1, 17, 10, 1) == 0
    assert L.sp_beam_select_workspace(1, 1, 10, 1) > 0


def test_group_arguments_count_with_groups_only(L):
    """Without groups their arguments are ignored, whatever they hold: the call goes on to its workspace."""
    for pages in (-1, 0, 1 << 30, (1 << 31) - 1):
        assert L.sp_prefix_attention(C.byref(attend(prefix_max_pages=pages)), OK, 64, None) == WORKSPACE
    assert L.sp_prefix_attention(C.byref(attend(n_groups=1, prefix_max_pages=1 << 27, group_cu=OK, prefix_table=OK,
                                                prefix_lens=OK)), OK, 64, None) == SHAPE


@pytest.mark.parametrize("sizes", [(-1, 4, 1, 4, 2, 64), (4, 257, 0, 4, 2, 64), (4, 4, 257, 4, 2, 64), (1 << 20, 4, 0, 512, 4, 64)])
def test_workspace_query_of_refused_sizes(L, sizes):
    """Sizes that the call refuses have no workspace, and the message says which."""
    L.sp_paged_append(None, None)  # (another message before)
    assert L.sp_prefix_attention_workspace(*sizes) == 0
    assert b"sp_prefix_attention_workspace" in L.sp_last_error() and b"n_groups" in L.sp_last_error()
