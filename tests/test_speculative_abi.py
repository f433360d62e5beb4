"""Host-side checks of the entry points for drafted tokens and pages: struct layouts and refusals, which fail before any
launch (no GPU is needed; the addresses below are never dereferenced)."""
import ctypes as C
import os
import re

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


def verify(**k):
    d = dict(B=2, V=100, T_cap=6, max_rows=4, cu_rows=OK, logits=OK, logits_f32=1, ld=100, draft=OK, draft_logits=OK, ld_draft=100,
             u=OK, noise=OK, ld_noise=100, temperature=OK, n_accept=OK, token=OK, logp=OK, err=OK)
    return b.sp_draft_verify_io(**dict(d, **k))


def pages(**k):
    d = dict(kv=OK, n_layers=2, n_pages=9, page_size=16, row_elems=64, S=3, table=OK, max_pages=4, lens=OK, refs=OK, err=OK)
    return b.sp_pages(**dict(d, **k))


def test_layouts():
    assert C.sizeof(b.sp_draft_verify_io) == 4 * 4 + 8 * 2 + 4 + 4 + 8 * 12 + 8
    assert C.sizeof(b.sp_pages) == 8 + 4 * 5 + 4 + 8 + 4 + 4 + 8 * 3


@pytest.mark.parametrize("want,change", [
    (SHAPE, dict(B=0)), (SHAPE, dict(B=257)), (SHAPE, dict(V=0)), (SHAPE, dict(V=(1 << 24) + 1)), (SHAPE, dict(T_cap=-1)),
    (SHAPE, dict(T_cap=(1 << 24) + 1)), (SHAPE, dict(max_rows=0)), (SHAPE, dict(max_rows=1025)), (SHAPE, dict(cu_rows=None)),
    (INVALID, dict(logits=None)), (INVALID, dict(draft=None)), (INVALID, dict(u=None)), (INVALID, dict(n_accept=None)),
    (INVALID, dict(token=None)), (SHAPE, dict(ld=99)), (SHAPE, dict(ld_draft=99)), (SHAPE, dict(ld_noise=99)),
    (ALIGN, dict(logits=258)), (ALIGN, dict(draft_logits=258)), (ALIGN, dict(noise=258)),
    (ALIGN, dict(logits=257, logits_f32=0)), (WORKSPACE, dict()),
    # what is not read is not asked for
    (WORKSPACE, dict(draft_logits=None, ld_draft=0)), (WORKSPACE, dict(noise=None, ld_noise=0, u=None, ld_draft=0)),
    (WORKSPACE, dict(max_rows=1, draft=None, u=None, draft_logits=None)), (WORKSPACE, dict(temperature=None, logp=None, err=None)),
    (WORKSPACE, dict(T_cap=2, max_rows=1, cu_rows=None)), (WORKSPACE, dict(T_cap=0, logits=None, draft=None, u=None)),
])
def test_verify_refusals(L, want, change):
    assert L.sp_draft_verify(C.byref(verify(**change)), OK, 64, None) == want
    assert L.sp_draft_verify(C.byref(verify(**change)), None, 1 << 40, None) == want


def test_workspaces(L):
    assert L.sp_draft_verify(None, OK, 64, None) == INVALID
    assert L.sp_draft_verify_workspace(6, 2, 100) > 0
    for bad in ((-1, 2, 100), (6, 0, 100), (6, 257, 100), (6, 2, 0), (6, 2, (1 << 24) + 1), ((1 << 24) + 1, 2, 100)):
        assert L.sp_draft_verify_workspace(*bad) == 0
    assert L.sp_pages_workspace(3, 4) > 0
    for bad in ((0, 4), (4097, 4), (3, 0), (4096, (1 << 18) + 1)):
        assert L.sp_pages_workspace(*bad) == 0


BOOKS = [
    (SHAPE, dict(S=0)), (SHAPE, dict(S=4097)), (SHAPE, dict(max_pages=0)), (SHAPE, dict(S=4096, max_pages=(1 << 18) + 1)),
    (SHAPE, dict(page_size=24)), (SHAPE, dict(page_size=8)), (SHAPE, dict(n_pages=0)), (SHAPE, dict(n_pages=1 << 28)),
    (SHAPE, dict(max_pages=1 << 27)), (INVALID, dict(table=None)), (INVALID, dict(lens=None)), (INVALID, dict(refs=None)),
    (ALIGN, dict(refs=264)),
]
MOVES = BOOKS + [
    (INVALID, dict(kv=None)), (SHAPE, dict(n_layers=0)), (SHAPE, dict(n_layers=97)), (SHAPE, dict(row_elems=0)),
    (SHAPE, dict(row_elems=12)), (ALIGN, dict(kv=264)), (WORKSPACE, dict()),
]


@pytest.mark.parametrize("want,change", BOOKS)
def test_trim_and_fork_refusals(L, want, change):
    p = pages(**dict(dict(kv=None, n_layers=0, row_elems=0), **change))  # (neither asks for the pool)
    assert L.sp_pages_trim(C.byref(p), None) == want
    assert L.sp_pages_fork(C.byref(p), OK, None) == want


@pytest.mark.parametrize("want,change", MOVES)
def test_reserve_and_compact_refusals(L, want, change):
    p = pages(**change)
    for ws, n in ((OK, 64), (None, 1 << 40)):
        assert L.sp_pages_reserve(C.byref(p), OK, ws, n, None) == want
        assert L.sp_pages_compact(C.byref(p), OK, 7, 7, OK, ws, n, None) == want


def test_pages_refusals_of_the_other_arguments(L):
    p = C.byref(pages())
    assert L.sp_pages_trim(None, None) == INVALID
    assert L.sp_pages_fork(p, None, None) == INVALID
    assert L.sp_pages_reserve(p, None, OK, 1 << 30, None) == INVALID
    for keep, ld, cap, count, want in ((None, 7, 7, OK, INVALID), (OK, 7, 7, None, INVALID), (OK, 6, 7, OK, SHAPE),
                                       (OK, 7, 0, OK, SHAPE), (OK, 1 << 30, 1 << 29, OK, SHAPE)):
        assert L.sp_pages_compact(p, keep, ld, cap, count, OK, 1 << 30, None) == want


def test_packed_arguments_are_the_structs(L):
    assert b._pack_pages(OK, 2, 9, 16, 64, 3, OK, 4, OK, OK, OK) == bytes(pages())
    assert b._pack_verify(2, 100, 6, 4, OK, OK, 1, 100, OK, OK, 100, OK, OK, 100, OK, OK, OK, OK, OK, 1) == bytes(verify(clear_err=1))


def _body(kernel):
    from test_kernel_sync import _kernel, _source
    return _kernel(_source("verify.cu"), kernel)


def test_the_end_kernel_reads_nothing_of_the_sums_before_its_wait():
    """It starts while the sums run: until its wait it may read what the caller gave, which no kernel of the call writes.  That
    was written before the sums' own wait, and they let it start only behind that."""
    sums, end = _body("verify_sums_kernel"), _body("verify_end_kernel")
    assert sums.index("pdl_wait()") < sums.index("pdl_trigger()")
    assert not re.search(r"\ba\.\w+\s*\[|__ldg|__ldcg|\bwork\.", sums[:sums.index("pdl_wait()")])
    before = end[:end.index("pdl_wait()")]
    assert "work" not in before and "pdl_trigger" not in before
    assert not re.search(r"\ba\.(n_accept|token|logp|err)\b", before)


@pytest.mark.parametrize("kernel", ["verify_end_kernel", "verify_sample_kernel"])
def test_every_cta_of_a_cluster_waits_before_it_ends(kernel):
    """A CTA that leaves early has taken part in the cluster's first barrier, and the others' memory is written behind it."""
    text = _body(kernel)
    assert text.index("cluster_arrive()") < text.index("cluster_wait()")
    assert text.rindex("cluster_wait()", 0, text.index("mapa_shared")) > text.index("cluster_arrive()")
    head = text[:text.index("mapa_shared")]
    for m in re.finditer(r"return;", head):
        assert "cluster_wait();" in head[max(0, m.start() - 60):m.start()], head[m.start() - 60:m.end()]
