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


# ----------------------------------------------------------------------------- lengths

def test_one_long_sequence_among_255_short_ones(sp):
    """2,100 rows of 32 heads over 32,768 own keys (8.7 million tiles of 16 vectors by 16 keys) beside 255 single rows.
    A segment's sums take up to 2,048 tiles one after the other, a rounding (2^-23, the tensor core's may cut off) each: 2^-12
    of the weights' sum and of sum w |v| at most, beside P's bound for scores as small as these."""
    g = gen(41)
    Hq, dh, page, rows, keys = 32, 64, 256, 2100, 32768
    n = [rows] + [1] * 255
    lens = [keys] + [1 + (5 * i) % 60 for i in range(255)]
    kv = normal(g, 2, 64, page, Hq * dh)
    table = torch.randint(0, 64, (256, keys // page), device=DEV, generator=g, dtype=torch.int32)
    q = normal(g, sum(n), Hq * dh)
    lse = torch.zeros((sum(n), Hq), device=DEV)
    r = sp.sp_prefix_attention(q=q, kv=kv, table=table, lens=ints(lens), cu_rows=starts(n), n_heads=Hq, n_kv_heads=Hq,
                               head_dim=dh, lse=lse)
    assert int(r["err"].item()) == 0
    k = torch.arange(keys, device=DEV)
    for b, picked in [(0, [0, 1, 700, 1555, rows - 1])] + [(b, [0]) for b in range(1, 256)]:
        at = table[b, k[:lens[b]] // page].long(), k[:lens[b]] % page
        K, V = (x[at].double().view(-1, Hq, dh) for x in kv)
        for j in picked:
            row = j if b == 0 else rows + b - 1
            see = lens[b] - n[b] + j + 1
            z = torch.einsum("hd,khd->hk", q[row].double().view(Hq, dh), K[:see]) * dh ** -0.5
            w = torch.softmax(z, dim=-1)
            o, size = (torch.einsum("hk,khd->hd", w, x[:see]).reshape(-1) for x in (V, V.abs()))
            assert ((r["out"][row].double() - o).abs() <= U * o.abs() + (U + 2.0 ** -11) * size).all(), (b, j)
            assert ((lse[row].double() - torch.logsumexp(z, dim=-1)).abs() <= 2.0 ** -12).all()


# ----------------------------------------------------------------------------- equal beams

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [5, 700, 1001, 2049, 32003, 152063])
def test_equal_beams_tie_wherever_their_rows_begin(sp, V, dtype):
    """Rows of equal logits have equal sums, and a tie goes to the lower beam, although rows of V elements begin at
    different places within 16 bytes."""
    g = gen(V)
    x = (3 * torch.randn((2, 1, V), device=DEV, generator=g)).to(dtype).expand(2, 4, V).contiguous()
    P.select_case(sp, x, torch.zeros((2, 4), device=DEV), 8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("skip", [1, 2, 3, 5, 7])
def test_equal_beams_of_rows_apart_and_a_first_row_off_16_bytes(sp, skip, dtype):
    g = gen(skip)
    for V, ld in ((9000, 9001 + skip), (4095, 4103), (40, 47)):
        full = torch.full((1 + 3 * 5 * ld + ld,), torch.nan, device=DEV, dtype=dtype)
        x = full[skip:skip + 15 * ld].view(3, 5, ld)[..., :V]
        x.copy_((3 * torch.randn((3, 1, V), device=DEV, generator=g)).to(dtype))
        x[1, :, ::3] = torch.nan
        x[1, :, 1::7] = -torch.inf
        x[2, :, V // 2] = torch.inf
        cum = torch.full((3, 5), -1.5, device=DEV)
        P.select_case(sp, x, cum, 10)


# ----------------------------------------------------------------------------- rising scores, long items

def rising_call(sp, seed, heads, rows, own, prefix, *, top, page=64):
    """One call whose scores rise from 0 to about `top` along the prefix (each key of it a little above those before),
    compared with the plain form.  Scores stay within the 64 that the bound is derived for."""
    Hq, Hkv, dh = heads
    g = gen(seed)
    both, pages = tables(g, own + [prefix], page)
    kv = normal(g, 2, pages, page, Hkv * dh, std=0.3)
    u = torch.where(torch.rand(dh, device=DEV, generator=g) < 0.5, -1.0, 1.0)
    T = sum(rows)
    q = (2 * u.repeat(Hq) + 0.3 * torch.randn((T, Hq * dh), device=DEV, generator=g)).to(torch.bfloat16)
    k = torch.arange(prefix, device=DEV)
    at = both[-1, k // page].long(), k % page
    # 2 dh b / sqrt(dh) = top k / prefix
    rise = (top * k / prefix / (2 * dh ** 0.5))[:, None] * u.repeat(Hkv)
    kv[0][at] = (kv[0][at].float() + rise).to(torch.bfloat16)
    table, ptable = widen(both[:-1].contiguous(), page), widen(both[-1:].contiguous(), page)
    lse = torch.zeros((T, Hq), device=DEV)
    r = sp.sp_prefix_attention(q=q, kv=kv, table=table, lens=ints(own), cu_rows=starts(rows) if max(rows) > 1 else None,
                               n_heads=Hq, n_kv_heads=Hkv, head_dim=dh, prefix_table=ptable, prefix_lens=ints([prefix]),
                               group_cu=ints([0, len(rows)]), lse=lse)
    assert int(r["err"].item()) == 0
    ref, rl, size = P.plain_attention(q, kv, page, heads, rows, table, own, [0, len(rows)], ptable, [prefix], dh ** -0.5)
    assert rl.max() < 64
    bad = (r["out"].double() - ref).abs() - (U * ref.abs() + (U + 2.0 ** -12) * size)
    assert bad.max().item() <= 0, f"off by {bad.max().item()} over the bound"
    assert ((lse.double() - rl).abs() <= 2.0 ** -13).all()  # (what the bound grants a score)


@pytest.mark.parametrize("heads", [(8, 2, 64), (8, 2, 128), (32, 8, 128)])
@pytest.mark.parametrize("rows", [[1] * 40, [16] * 32])
def test_scores_that_rise_from_tile_to_tile(sp, heads, rows):
    """Key tiles of 128 whose largest scores are more than 8 (in powers of two) apart: the tensor kernel rescales what
    it has summed tile by tile, in segments of four tiles and of ten."""
    rising_call(sp, 51, heads, rows, [max(n, 20) for n in rows], 1024, top=50)


@pytest.mark.parametrize("heads", [(4, 2, 64), (4, 2, 128), (2, 2, 128)])
@pytest.mark.parametrize("rows,prefix", [([1], 15000), ([1] * 4, 4500), ([3, 1], 9001)])
@pytest.mark.parametrize("top", [0, 50])
def test_items_of_many_segments(sp, heads, rows, prefix, top):
    """Few rows over thousands of keys by plan and merge: far more than 32 segments of one item, whose maxima rise."""
    rising_call(sp, 52, heads, rows, [30 + n for n in rows], prefix, top=top)


@pytest.mark.parametrize("dtype,V", [(torch.float32, 4099), (torch.float32, 8191), (torch.bfloat16, 8195), (torch.bfloat16, 16391)])
def test_equal_beams_of_whole_tiles(sp, dtype, V):
    """One slice to a row of so many rows: its chunks fill whole tiles, and some are left behind the last."""
    g = gen(V)
    x = (3 * torch.randn((80, 1, V), device=DEV, generator=g)).to(dtype).expand(80, 4, V).contiguous()
    P.select_case(sp, x, torch.zeros((80, 4), device=DEV), 8)


# ----------------------------------------------------------------------------- infinite scores

@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("rows,own", MIXES)
@pytest.mark.parametrize("wide", [False, True])
def test_keys_with_a_score_of_minus_infinity_have_no_weight(sp, dh, rows, own, wide):
    """A prefix of such keys: rows with own keys see those alone (so its values do not matter), rows without see nothing."""
    a = shared_call(gen(dh + len(rows)), dh, rows, own, wide)
    a["q"].abs_()
    for k in range(300):
        a["kv"][0, int(a["prefix_table"][0, k // 16]), k % 16] = -torch.inf
    ref, rl = sp.sp_prefix_attention(**a)["out"].clone(), a["lse"].clone()
    alone = torch.zeros_like(rl)
    b = sp.sp_prefix_attention(**{**a, "lse": alone, "prefix_table": None})["out"]
    if own[0] == 0:
        assert (ref == 0).all() and torch.isinf(rl).all() and (rl < 0).all() and (b == 0).all()
        return
    # (cut into other segments: both within the bound, where the weights' sum of |v| is at most the largest |v|)
    most = a["kv"][1].abs().max().double()
    x, y = ref.double(), b.double()
    assert ((x - y).abs() <= 2 * (U * torch.maximum(x.abs(), y.abs()) + (U + 2.0 ** -12) * most)).all()
    assert ((rl - alone).abs() <= 2 * (1e-5 + 1e-6 * rl.abs())).all()
