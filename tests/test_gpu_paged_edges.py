"""Generation over a paged cache, where single cases of test_gpu_paged.py do not reach: NaN in every kernel of the
attention, one long sequence among short ones, rising scores, long items, equal beams, streams.

The bounds are test_gpu_paged.py's (its plain forms and its bound on attention are used here)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import test_gpu_paged as P  # noqa: E402
from test_gpu_paged import DEV, U, gen, ints, normal, starts, tables, widen  # noqa: E402


@pytest.fixture(autouse=True)
def single_precision():
    """Tensors without a type of their own are fp32, whatever another module has set."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_13804_gb300 import binding
    binding.lib()
    return binding


# ----------------------------------------------------------------------------- NaN

# Rows of each sequence and their own keys: prefix and own keys both by the tensor kernel (144 query vectors), own keys by
# the kernel for few vectors, and no own keys.  (With narrow tables all of them are one launch of the row kernel.)
MIXES = [([12, 12, 12], [40, 12, 200]), ([1] * 40, [5] * 40), ([1] * 40, [0] * 40)]


def shared_call(g, dh, rows, own, wide, prefix=300, page=16):
    """Arguments of a call whose sequences all share one prefix; kv rows are [0, prefix) of pages 0 .. for the prefix."""
    Hq, Hkv = 8, 2
    both, pages = tables(g, own + [prefix], page)
    table, ptable = both[:-1].contiguous(), both[-1:].contiguous()
    if wide:
        table, ptable = widen(table, page), widen(ptable, page)
    T = sum(rows)
    return dict(q=normal(g, T, Hq * dh), kv=normal(g, 2, pages, page, Hkv * dh), table=table, lens=ints(own),
                cu_rows=starts(rows) if max(rows) > 1 else None, n_heads=Hq, n_kv_heads=Hkv, head_dim=dh,
                prefix_table=ptable, prefix_lens=ints([prefix]), group_cu=ints([0, len(rows)]),
                lse=torch.zeros((T, Hq), device=DEV))


def put_nan_keys(a, table_row, first, last, page=16):
    for k in range(first, last):
        a["kv"][0, int(table_row[k // page]), k % page] = torch.nan


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("rows,own", MIXES)
@pytest.mark.parametrize("wide", [False, True])
def test_a_nan_query_gives_nan(sp, dh, rows, own, wide):
    """All scores of such a vector are NaN: so are its output and lse, and no other row's change."""
    a = shared_call(gen(dh + len(rows)), dh, rows, own, wide)
    ref, rl = sp.sp_prefix_attention(**a)["out"].clone(), a["lse"].clone()
    a["q"][7, 3 * dh + 5] = torch.nan
    got, gl = sp.sp_prefix_attention(**a)["out"], a["lse"]
    assert torch.isnan(got[7, 3 * dh:4 * dh]).all() and torch.isnan(gl[7, 3])
    got[7, 3 * dh:4 * dh] = ref[7, 3 * dh:4 * dh]
    gl[7, 3] = rl[7, 3]
    assert torch.equal(got, ref) and torch.equal(gl, rl)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("rows,own", MIXES)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("first,last", [(0, 300), (128, 256), (299, 300)])
def test_nan_keys_of_the_prefix_give_nan(sp, dh, rows, own, wide, first, last):
    """The whole prefix, a whole tile of it, its last key: every row sees them."""
    a = shared_call(gen(dh + len(rows) + first), dh, rows, own, wide)
    put_nan_keys(a, a["prefix_table"][0], first, last)
    r = sp.sp_prefix_attention(**a)
    assert torch.isnan(r["out"]).all() and torch.isnan(a["lse"]).all()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("wide", [False, True])
def test_a_nan_own_key_gives_nan_where_it_is_seen(sp, dh, wide):
    rows, own = MIXES[0]
    a = shared_call(gen(dh), dh, rows, own, wide)
    ref, rl = sp.sp_prefix_attention(**a)["out"].clone(), a["lse"].clone()
    put_nan_keys(a, a["table"][0], 33, 34)  # rows 5 .. 11 of the first sequence's 12 see keys up to 28 + row
    got, gl = sp.sp_prefix_attention(**a)["out"], a["lse"]
    assert torch.isnan(got[5:12]).all() and torch.isnan(gl[5:12]).all()
    keep = list(range(5)) + list(range(12, 36))
    assert torch.equal(got[keep], ref[keep]) and torch.equal(gl[keep], rl[keep])
