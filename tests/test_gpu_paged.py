"""Generation over a paged cache with shared prefixes: sp_paged_append, sp_prefix_attention, sp_beam_select and
sp_beam_reorder against plain implementations in 64 bits.

Tolerances (u = 2^-8, half a bf16 step relative to the value; e = 2^-24, the same of fp32):
- append: y = x c - z s in fp32 (three roundings, c and s rounded: at most 5 e (|x c| + |z s|)), rounded once:
  |err| <= u |y| + 5 e (|x c| + |z s|); the bound used is u |y| + 1e-6 (|x| + |z|).
- attention: scores are fp32 sums of dh exact products (their error moves a weight by less than 2^-13 for scores
  up to 64), the weights are rounded to bf16 for the product with V (each by u relative, whatever the
  other side's scaling, and the sum of the weights is not), sums in fp32, the result rounded once:
  |err| <= u |o| + (u + 2^-12) sum_k w_k |v_k|.  lse: 1e-5 + 1e-6 |lse|.
- selection: beams and tokens equal; score: fp32 rounding plus a sum of exponentials good to 2^-20 relative:
  2^-24 |score| + 2^-20.
"""
import ctypes as C
import itertools

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -8
HEADS = [(32, 32, 128), (28, 4, 128), (16, 16, 64), (6, 2, 64), (40, 1, 128)]


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


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def starts(v):
    return ints([sum(v[:i]) for i in range(len(v) + 1)])


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, *shape, std=1.0):
    return (torch.randn(shape, device=DEV, generator=g) * std).to(torch.bfloat16)


def tables(g, lens, page, extra_pages=2, extra_columns=1):
    """Scattered pages for sequences of these lengths; unused entries hold -1."""
    need = [-(-n // page) for n in lens]
    width = max(need) + extra_columns
    ids = torch.randperm(sum(need) + extra_pages, device=DEV, generator=g).to(torch.int32)
    t = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = ids[at:at + n]
        at += n
    return t, sum(need) + extra_pages


def widen(t, page):
    """The same table with room for more than 16,384 keys: such calls are planned over the GPU, and many vectors of an entry
    go to the tensor kernel."""
    wide = torch.full((t.shape[0], max(t.shape[1], 16384 // page + 1)), -1, dtype=torch.int32, device=DEV)
    wide[:, :t.shape[1]] = t
    return wide


# ----------------------------------------------------------------------------- append

def plain_append(qkv, lens, rows, table, page, heads, theta, pos, section):
    """(q, k, v, slots) of every row in 64 bits: slots (page, row in page)."""
    Hq, Hkv, dh = heads
    T = qkv.shape[0]
    x = qkv.double().view(T, -1, dh)
    freq = theta ** (-torch.arange(0, dh, 2, dtype=torch.float64, device=DEV) / dh)
    if section is None:
        ang = pos.double()[:, None] * freq
    else:
        comp = torch.tensor(sum(([i] * n for i, n in enumerate(section)), []), device=DEV)
        ang = pos.double()[:, comp] * freq
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    a, b = x[:, :Hq + Hkv, :dh // 2], x[:, :Hq + Hkv, dh // 2:]
    y = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
    size = torch.cat((a.abs() + b.abs(),) * 2, dim=-1)
    slots = []
    for q, (n, L) in enumerate(zip(rows, lens)):
        for j in range(n):
            slots.append((int(table[q, (L + j) // page]), (L + j) % page))
    return y, size, x[:, Hq + Hkv:], slots


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page,mrope,strided", [(16, False, False), (64, True, True)])
def test_append_prompts_and_tokens(sp, heads, page, mrope, strided):
    Hq, Hkv, dh = heads
    g = gen(11)
    for rows, lens in (([1] * 5, [0, 15, 16, 63, 200]), ([7, 0, 1, 40, 17], [0, 3, 31, 16, 250])):
        T, width = sum(rows), (Hq + 2 * Hkv) * dh
        full = normal(g, T, width + (24 if strided else 0))
        qkv = full[:, :width]
        table, pages = tables(g, [a + b for a, b in zip(rows, lens)], page)
        kv = normal(g, 2, pages, page, Hkv * dh)
        before = kv.clone()
        section = ((dh // 4, dh // 8, dh // 8) if mrope else None)
        pos = torch.randint(0, 5000, (T, 4) if mrope else (T,), device=DEV, generator=g, dtype=torch.int32)
        rope = sp.rope_table(5000, dh, 1e6)
        cu = starts(rows) if max(rows) > 1 else None
        r = sp.sp_paged_append(qkv=qkv, kv=kv, table=table, lens=ints(lens), cu_rows=cu, n_heads=Hq, n_kv_heads=Hkv,
                               head_dim=dh, rope=rope, pos=None if mrope else pos, pos3=pos if mrope else None,
                               mrope_section=section)
        assert int(r["err"].item()) == 0
        y, size, v, slots = plain_append(qkv, lens, rows, table, page, heads, 1e6, pos, section)
        tol = U * y.abs() + 1e-6 * size
        assert ((r["q"].double().view(T, Hq, dh) - y[:, :Hq]).abs() <= tol[:, :Hq]).all()
        pg, at = (torch.tensor(z, device=DEV) for z in zip(*slots))
        got = kv[:, pg, at].double().view(2, T, Hkv, dh)
        assert ((got[0] - y[:, Hq:]).abs() <= tol[:, Hq:]).all()
        assert torch.equal(got[1], v)
        before[:, pg, at] = kv[:, pg, at]
        assert torch.equal(before, kv)  # nothing else was touched


def test_append_in_place_without_rotation_and_rows_behind_the_last(sp):
    g = gen(3)
    Hq, Hkv, dh, page = 4, 2, 128, 16
    qkv = normal(g, 9, (Hq + 2 * Hkv) * dh)
    table, pages = tables(g, [3, 4], page)
    kv = sp.paged_pool(pages, page, Hkv, dh)[0]
    rope = sp.rope_table(64, dh)
    pos = ints([5, 6, 7, 0, 1, 2, 3, 50, 51])
    plain = qkv.clone()
    ref = sp.sp_paged_append(qkv=plain, kv=kv.clone(), table=table, cu_rows=ints([0, 3, 7]), n_heads=Hq, n_kv_heads=Hkv,
                             head_dim=dh, rope=rope, pos=pos)["q"]
    r = sp.sp_paged_append(qkv=qkv, kv=kv, table=table, cu_rows=ints([0, 3, 7]), n_heads=Hq, n_kv_heads=Hkv,
                           head_dim=dh, rope=rope, pos=pos, q_out=qkv[:, :Hq * dh])
    assert int(r["err"].item()) == 0
    assert torch.equal(qkv[:7, :Hq * dh], ref[:7]) and torch.equal(qkv[7:], plain[7:])
    assert torch.equal(qkv[:, Hq * dh:], plain[:, Hq * dh:])
    kv2 = sp.paged_pool(pages, page, Hkv, dh)[0]
    sp.sp_paged_append(qkv=plain, kv=kv2, table=table, cu_rows=ints([0, 3, 7]), n_heads=Hq, n_kv_heads=Hkv,
                       head_dim=dh, keys_only=True)
    k = plain[:, Hq * dh:(Hq + Hkv) * dh]
    assert torch.equal(kv2[0, table[0, 0].item(), :3], k[:3]) and torch.equal(kv2[0, table[1, 0].item(), :4], k[3:7])


def test_append_past_the_table_and_the_rotary_range_are_skipped(sp):
    g = gen(4)
    Hq, Hkv, dh, page = 2, 1, 64, 16
    qkv = normal(g, 4, (Hq + 2 * Hkv) * dh)
    kv = normal(g, 2, 6, page, Hkv * dh)
    table = ints([[0, 1], [2, -1], [3, 99], [4, 5]])
    rope = sp.rope_table(32, dh)
    before = kv.clone()
    r = sp.sp_paged_append(qkv=qkv, kv=kv, table=table, lens=ints([32, 16, 17, -1]), n_heads=Hq, n_kv_heads=Hkv,
                           head_dim=dh, rope=rope, pos=ints([0, 0, 0, 0]))
    assert int(r["err"].item()) == 2 and torch.equal(kv, before)
    r = sp.sp_paged_append(qkv=qkv, kv=kv, table=table, lens=ints([0, 0, 0, 0]), n_heads=Hq, n_kv_heads=Hkv,
                           head_dim=dh, rope=rope, pos=ints([31, 32, -1, 3]))
    assert int(r["err"].item()) == 2
    assert torch.equal(kv[:, 2:4], before[:, 2:4]) and not torch.equal(kv[0, 4], before[0, 4])


# ----------------------------------------------------------------------------- attention

def plain_attention(q, kv, page, heads, rows, table, lens, group_cu, ptable, plens, scale):
    """Row by row in 64 bits; (out, lse, sum of weights times |v|)."""
    Hq, Hkv, dh = heads
    G = Hq // Hkv
    take = lambda t, n: kv[:, [int(t[k // page]) for k in range(n)], [k % page for k in range(n)]]  # noqa: E731
    outs, lses, sizes, at = [], [], [], 0
    for b, n in enumerate(rows):
        g = next((i for i in range(len(group_cu) - 1) if group_cu[i] <= b < group_cu[i + 1]), None)
        own = take(table[b], lens[b])
        pre = take(ptable[g], plens[g]) if g is not None else own[:, :0]
        x = torch.cat((pre, own), dim=1).double().view(2, -1, Hkv, dh)
        for j in range(n):
            see = pre.shape[1] + max(0, min(lens[b], lens[b] - n + j + 1))
            k, v = x[:, :see]
            qr = q[at].double().view(Hkv, G, dh)
            z = torch.einsum("hgd,khd->hgk", qr, k) * scale
            if see == 0:
                outs.append(torch.zeros(Hq * dh, dtype=torch.float64, device=DEV))
                sizes.append(torch.zeros_like(outs[-1]))
                lses.append(torch.full((Hq,), -torch.inf, dtype=torch.float64, device=DEV))
            else:
                w = torch.softmax(z, dim=-1)
                outs.append(torch.einsum("hgk,khd->hgd", w, v).reshape(-1))
                sizes.append(torch.einsum("hgk,khd->hgd", w, v.abs()).reshape(-1))
                lses.append(torch.logsumexp(z, dim=-1).reshape(-1))
            at += 1
    return torch.stack(outs), torch.stack(lses), torch.stack(sizes)


def attention_case(sp, seed, heads, page, rows, lens, groups, plens, **options):
    """Runs one call as each of the kernels takes it and compares it with the plain form."""
    for wide, offsets in ((False, False), (False, True), (True, True), (True, False)):
        attention_call(sp, seed, heads, page, rows, lens, groups, plens, wide=wide, offsets=offsets, **options)


def attention_call(sp, seed, heads, page, rows, lens, groups, plens, *, std=1.0, scale=None, strided=False, garbage=True,
                   graph=False, wide=False, offsets=False):
    """groups: sequences per group (the rest have no prefix)."""
    Hq, Hkv, dh = heads
    g = gen(seed)
    T = sum(rows)
    both, pages = tables(g, list(lens) + list(plens), page)
    table, ptable = both[:len(lens)].contiguous(), both[len(lens):].contiguous()
    kv = normal(g, 2, pages, page, Hkv * dh)
    if garbage:  # what lies in no sequence is NaN: unused pages and the rest of the last pages
        used = torch.zeros(pages, page, dtype=torch.bool, device=DEV)
        for t, n in zip(both, list(lens) + list(plens)):
            for k in range(0, n, page):
                used[int(t[k // page]), :min(page, n - k)] = True
        kv[:, ~used] = float("nan")
    extra = 3
    full = normal(g, T + extra, Hq * dh + (16 if strided else 0), std=std)
    q = full[:, :Hq * dh]
    one = all(n == 1 for n in rows)
    cu = None if one and not offsets else starts(rows)
    if cu is None:
        q = q[:T]
    out = torch.full((q.shape[0], Hq * dh + (8 if strided else 0)), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((q.shape[0], Hq), 7.0, device=DEV)
    group_cu = [sum(groups[:i]) for i in range(len(groups) + 1)]
    some = len(groups) > 0
    if wide:
        table, ptable = widen(table, page), widen(ptable, page)
    args = dict(q=q, kv=kv, table=table, lens=ints(lens), cu_rows=cu, n_heads=Hq, n_kv_heads=Hkv, head_dim=dh,
                prefix_table=ptable if some else None, prefix_lens=ints(plens) if some else None,
                group_cu=ints(group_cu) if some else None, scale=scale or 0.0, out=out[:, :Hq * dh], lse=lse)
    if graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        args["ws"] = sp.prefix_attention_workspace(T_cap=q.shape[0], B=len(lens), n_heads=Hq, n_kv_heads=Hkv,
                                                   head_dim=dh, n_groups=len(groups))
        args["ws"].fill_(255)
        args["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        cg = torch.cuda.CUDAGraph()
        with torch.cuda.graph(cg):
            r = sp.sp_prefix_attention(**args)
        for _ in range(2):
            cg.replay()
    else:
        r = sp.sp_prefix_attention(**args)
    assert int(r["err"].item()) == 0
    ref, rl, size = plain_attention(q, kv, page, heads, rows, table, lens, group_cu, ptable, plens, scale or dh ** -0.5)
    got = out[:T, :Hq * dh].double()
    bad = (got - ref).abs() - (U * ref.abs() + (U + 2.0 ** -12) * size)
    assert torch.isfinite(got).all() and bad.max().item() <= 0, f"off by {bad.max().item()} over the bound"
    empty = torch.isinf(rl)
    assert torch.equal(torch.isinf(lse[:T].double()), empty)
    assert ((lse[:T].double() - rl)[~empty].abs() <= 1e-5 + 1e-6 * rl[~empty].abs()).all()
    assert (out[T:] == 7).all() and (lse[T:] == 7).all() and (out[:, Hq * dh:] == 7).all()


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [16, 128])
def test_attention_single_tokens(sp, heads, page):
    attention_case(sp, 1, heads, page, [1] * 7, [1, 16, 17, 40, 0, 3, 129], [3, 0, 2, 1], [65, 9, 0, 200])


@pytest.mark.parametrize("heads", HEADS)
def test_attention_one_sequence_of_one_key(sp, heads):
    attention_case(sp, 2, heads, 16, [1], [1], [], [])
    attention_case(sp, 3, heads, 16, [1], [0], [1], [1])


def test_attention_rows_that_see_nothing(sp):
    attention_case(sp, 4, (4, 2, 64), 16, [1, 1, 1], [0, 5, 0], [2], [0])
    attention_case(sp, 5, (4, 2, 128), 16, [4, 2, 0, 3], [2, 2, 0, 0], [], [])


@pytest.mark.parametrize("heads", HEADS)
def test_attention_questions(sp, heads):
    attention_case(sp, 6, heads, 32, [5, 1, 0, 33, 12], [5, 4, 0, 50, 12], [3, 2], [300, 31], strided=True)


@pytest.mark.parametrize("heads,groups", [((28, 4, 128), [40]), ((16, 16, 64), [20, 30]), ((8, 1, 128), [33, 1, 7])])
def test_attention_many_sequences_of_a_prefix(sp, heads, groups):
    n = sum(groups)
    attention_case(sp, 7, heads, 16, [1] * n, [(7 * i) % 60 for i in range(n)], groups, [500 + 77 * i for i in range(len(groups))])


def test_attention_large_scores_and_a_scale(sp):
    attention_case(sp, 8, (8, 2, 128), 16, [1] * 6, [9, 30, 1, 2, 64, 100], [6], [333], std=4.0)
    attention_case(sp, 9, (8, 2, 64), 16, [3] * 4, [9, 30, 3, 4], [2, 2], [33, 64], scale=0.5)


def test_attention_full_batch(sp):
    attention_case(sp, 10, (4, 4, 64), 16, [1] * 256, [1 + i % 37 for i in range(256)], [1] * 256, [i % 50 for i in range(256)])


def test_attention_in_a_graph_on_a_dirty_workspace(sp):
    attention_case(sp, 12, (28, 4, 128), 64, [1] * 30, [1 + i for i in range(30)], [30], [700], graph=True)


def test_attention_reports_a_page_outside_the_pool(sp):
    kv = torch.zeros((2, 4, 16, 64), dtype=torch.bfloat16, device=DEV)
    kv[1] = 1.0
    q = torch.ones((2, 64), dtype=torch.bfloat16, device=DEV)
    r = sp.sp_prefix_attention(q=q, kv=kv, table=ints([[0], [9]]), lens=ints([16, 16]), n_heads=1, n_kv_heads=1, head_dim=64)
    assert int(r["err"].item()) == 2
    assert (r["out"][0] == 1).all() and (r["out"][1] == 0).all()
    r = sp.sp_prefix_attention(q=q, kv=kv, table=ints([[0], [1]]), lens=ints([17, 16]), n_heads=1, n_kv_heads=1, head_dim=64)
    assert int(r["err"].item()) == 2


@pytest.mark.parametrize("G,n", [(2, 3), (4, 64)])  # few query vectors per prefix, many
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("wide,offsets", [(False, False), (True, True), (True, False)])
def test_attention_counts_a_bad_page_as_zeros(sp, G, n, dh, page, wide, offsets):
    """Pages outside the pool inside a prefix and at its end: their keys and values are zeros, the error word says so."""
    g = gen(page + n)
    pages = -(-300 // page)
    kv = normal(g, 2, pages + 3, page, 2 * dh)
    q = normal(g, n, 2 * G * dh)
    ids = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
    good = torch.full((1, pages), pages, dtype=torch.int32, device=DEV)  # page `pages` of the pool: zeros
    kv[:, pages] = 0
    bad = good.clone()
    keep = [i for i in range(pages) if i not in (1, pages - 1)]
    for t in (good, bad):
        t[0, keep] = ids[keep]
    bad[0, 1 % pages], bad[0, pages - 1] = -1, pages + 3
    cu = starts([1] * n) if offsets else None
    if wide:
        good, bad = widen(good, page), widen(bad, page)
    args = dict(cu_rows=cu, q=q, kv=kv, lens=ints([0] * n), table=torch.full((n, 1), -1, dtype=torch.int32, device=DEV), n_heads=2 * G,
                n_kv_heads=2, head_dim=dh, prefix_lens=ints([300]), group_cu=ints([0, n]))
    a = sp.sp_prefix_attention(prefix_table=good, **args)
    b = sp.sp_prefix_attention(prefix_table=bad, **args)
    assert int(a["err"].item()) == 0 and int(b["err"].item()) == 2
    assert torch.equal(a["out"], b["out"])


@pytest.mark.parametrize("n", [3, 64])
@pytest.mark.parametrize("wide,offsets", [(False, False), (True, True), (True, False)])
def test_attention_nan_stays_in_its_row(sp, n, wide, offsets):
    g = gen(n)
    kv = normal(g, 2, 30, 16, 128)
    q = normal(g, n, 4 * 128)
    args = dict(kv=kv, lens=ints([5] * n), table=ints([[20]] * n), n_heads=4, n_kv_heads=1, head_dim=128,
                prefix_table=torch.arange(20, device=DEV, dtype=torch.int32)[None], prefix_lens=ints([311]), group_cu=ints([0, n]))
    if wide:
        args.update(prefix_table=widen(args["prefix_table"], 16))
    if offsets:
        args.update(cu_rows=starts([1] * n))
    ref = sp.sp_prefix_attention(q=q, **args)["out"].clone()
    q[1, 128:256] = torch.nan  # one head of one row
    got = sp.sp_prefix_attention(q=q, lse=(lse := torch.zeros((n, 4), device=DEV)), **args)["out"]
    assert torch.isnan(got[1, 128:256]).all() and torch.isnan(lse[1, 1])
    got[1, 128:256] = ref[1, 128:256]
    assert torch.equal(got, ref) and int(torch.isnan(lse).sum()) == 1
    kv[1, 3, 5, 7] = torch.nan  # a value that all rows see
    got = sp.sp_prefix_attention(q=ref.new_zeros(n, 512), **args)["out"].view(n, 4, 128)
    assert torch.isnan(got[..., 7]).all() and torch.isfinite(got[..., :7]).all() and torch.isfinite(got[..., 8:]).all()


@pytest.mark.parametrize("heads", [(32, 32, 128), (64, 32, 128), (48, 48, 64)])
def test_attention_rows_of_different_groups_together(sp, heads):
    """Up to eight query vectors share a CTA: rows of one prefix, of several, and of none."""
    for groups in ([8, 8], [3, 5, 1, 4], [1, 0, 2, 11]):
        lens = [(11 * i) % 30 for i in range(16)]
        attention_call(sp, 20, heads, 16, [1] * 16, lens, groups, [300, 17, 0, 290][:len(groups)])


@pytest.mark.parametrize("heads", [(4, 4, 128), (14, 2, 64), (40, 2, 128)])
@pytest.mark.parametrize("wide", [False, True])
def test_attention_rows_before_the_first_and_between_empty_sequences(sp, heads, wide):
    """Row offsets that begin behind row 0, sequences without rows, a group that begins with one: as the same rows from 0."""
    Hq, Hkv, dh = heads
    g = gen(22)
    kv = normal(g, 2, 12, 32, Hkv * dh)
    q = normal(g, 14, Hq * dh)
    table, prefix = ints([[0, 1], [2, 3], [4, 5], [6, 7]]), ints([[8, 9], [10, 11]])
    if wide:
        prefix = widen(prefix, 32)
    args = dict(kv=kv, table=table, lens=ints([9, 3, 40, 33]), n_heads=Hq, n_kv_heads=Hkv, head_dim=dh, prefix_table=prefix,
                prefix_lens=ints([50, 64]), group_cu=ints([0, 2, 4]))
    ref = sp.sp_prefix_attention(q=q[3:11].contiguous(), cu_rows=ints([0, 3, 3, 7, 8]), **args)["out"]
    out, lse = torch.full((14, Hq * dh), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((14, Hq), 7.0, device=DEV)
    r = sp.sp_prefix_attention(q=q, cu_rows=ints([3, 6, 6, 10, 11]), out=out, lse=lse, **args)
    assert int(r["err"].item()) == 0
    outside = [0, 1, 2, 11, 12, 13]
    assert (out[outside] == 7).all() and (lse[outside] == 7).all()
    # (cut into other tiles: both within attention_call's bound, where the weights' sum of |v| is at most the largest |v|)
    a, b, most = out[3:11].double(), ref.double(), kv[1].abs().max().double()
    assert ((a - b).abs() <= 2 * (U * torch.maximum(a.abs(), b.abs()) + (U + 2.0 ** -12) * most)).all()
    for bad in ([51, 65 if not wide else 1 << 20], [-1, 3]):
        r = sp.sp_prefix_attention(q=q, cu_rows=ints([3, 6, 6, 10, 11]), **dict(args, prefix_lens=ints(bad)))
        assert int(r["err"].item()) == 2


@pytest.mark.parametrize("heads", [(32, 32, 128), (64, 32, 128), (48, 48, 64)])
@pytest.mark.parametrize("wide", [False, True])
def test_attention_nan_in_own_keys_stays_in_its_row(sp, heads, wide):
    Hq, Hkv, dh = heads
    g = gen(21)
    n = 34 if wide else 16
    kv = normal(g, 2, 20 + 2 * n, 16, Hkv * dh)
    q = normal(g, n, Hq * dh)
    args = dict(q=q, kv=kv, lens=ints([5 + i for i in range(n)]), table=ints([[20 + 2 * i, 21 + 2 * i] for i in range(n)]),
                n_heads=Hq, n_kv_heads=Hkv, head_dim=dh, prefix_table=torch.arange(20, device=DEV, dtype=torch.int32)[None],
                prefix_lens=ints([311]), group_cu=ints([0, n]))
    args["lens"] = args["lens"].clamp(max=32)
    if wide:
        args["prefix_table"] = widen(args["prefix_table"], 16)
    ref = sp.sp_prefix_attention(**args)["out"].clone()
    kv[:, 20 + 2 * 5, 3] = torch.nan   # a key and value of row 5, a value of row 6, an infinite value of row 7
    kv[1, 20 + 2 * 6, 2] = torch.nan
    kv[1, 20 + 2 * 7, 1] = torch.inf
    got = sp.sp_prefix_attention(**args)["out"]
    keep = [i for i in range(n) if i not in (5, 6, 7)]
    assert torch.equal(got[keep], ref[keep]) and torch.isnan(got[5:7]).all() and torch.isinf(got[7]).all()


def test_attention_130_query_heads_of_one(sp):
    attention_case(sp, 15, (130, 1, 64), 16, [1, 2, 1], [9, 30, 1], [2, 1], [33, 64])
    attention_case(sp, 16, (48, 2, 128), 16, [1, 7], [9, 30], [2], [133])


def test_offsets_beyond_32_bits(sp):
    """A pool of more than 2^32 elements, pages at both ends of it: append, attention by both kernels, reordering."""
    g = gen(17)
    Hq, Hkv, dh, page = 32, 8, 128, 16
    pages = 140_000  # 2 x 140,000 x 16 x 1,024 elements
    kv = torch.empty((1, 2, pages, page, Hkv * dh), dtype=torch.bfloat16, device=DEV)
    table = ints([[0, pages - 1], [pages - 2, 1], [pages - 3, pages - 4]])
    kv[:, :, [0, 1, 2, pages - 1, pages - 2, pages - 3, pages - 4]] = normal(g, 1, 2, 7, page, Hkv * dh)
    qkv = normal(g, 3, (Hq + 2 * Hkv) * dh)
    sp.sp_paged_append(qkv=qkv, kv=kv[0], table=table, lens=ints([17, 15, 31]), n_heads=Hq, n_kv_heads=Hkv, head_dim=dh)
    for b, (p, r) in enumerate(((pages - 1, 1), (pages - 2, 15), (pages - 4, 15))):
        assert torch.equal(kv[0, :, p, r].reshape(-1), qkv[b, Hq * dh:])
    for n, wide, offsets in ((3, False, 0), (3, True, 1), (40, False, 1), (40, True, 1), (40, True, 0)):
        q = normal(g, n, Hq * dh)
        fit = lambda t: widen(t, page) if wide else t  # noqa: E731
        cu = starts([1] * n) if offsets else None
        r = sp.sp_prefix_attention(q=q, kv=kv[0], table=table[:1].expand(n, 2).contiguous(), lens=ints([18] * n), n_heads=Hq, n_kv_heads=Hkv,
                                   head_dim=dh, cu_rows=cu, prefix_table=fit(table[1:]), prefix_lens=ints([20, 32]), group_cu=ints([0, n - 1, n]))
        few = torch.cat((kv[0, :, [0, 1]], kv[0, :, pages - 4:]), dim=1)  # the same pages in a small pool
        at = lambda t: torch.where(t > 1, t - (pages - 4) + 2, t).to(torch.int32)  # noqa: E731
        s = sp.sp_prefix_attention(q=q, kv=few, table=at(table[:1]).expand(n, 2).contiguous(), lens=ints([18] * n), n_heads=Hq, n_kv_heads=Hkv,
                                   head_dim=dh, cu_rows=cu, prefix_table=fit(at(table[1:])), prefix_lens=ints([20, 32]), group_cu=ints([0, n - 1, n]))
        assert int(r["err"].item()) == 0 and torch.equal(r["out"], s["out"])
    own = ints([[0, pages - 1], [pages - 2, pages - 3]])
    t = own.clone()
    src = kv[0, :, pages - 1, :5].clone()
    err = sp.sp_beam_reorder(kv=kv, table=t, own_table=own, lens=ints([21, 21]), parent=ints([[0, 0]]))
    assert int(err.item()) == 0 and torch.equal(kv[0, :, pages - 3, :5], src)
    assert t.tolist() == [[0, pages - 1], [0, pages - 3]]


def test_calls_without_rows(sp):
    kv = sp.paged_pool(2, 16, 1, 64)[0]
    args = dict(kv=kv, table=ints([[0]]), lens=ints([3]), cu_rows=ints([0, 0]), n_heads=1, n_kv_heads=1, head_dim=64)
    q = torch.empty((0, 64), dtype=torch.bfloat16, device=DEV)
    assert sp.sp_prefix_attention(q=q, **args)["out"].shape == (0, 64)
    assert sp.sp_paged_append(qkv=torch.empty((0, 192), dtype=torch.bfloat16, device=DEV), **args)["q"].shape == (0, 64)


# ----------------------------------------------------------------------------- beam selection

def plain_select(logits, cum, n_out, done, eos):
    """Score, parent, token of every element, in 64 bits by sorting all candidates."""
    B, W, V = logits.shape
    x = logits.double().cpu().numpy()
    out = []
    for b in range(B):
        cand = []
        for w in range(W):
            c = float(cum[b, w])
            if not c > -np.inf:
                continue
            if done is not None and bool(done[b, w]):
                cand.append((c, w, eos, 0.0))
                continue
            r = x[b, w]
            r = np.where(np.isnan(r), -np.inf, r)
            m = r.max()
            if m == -np.inf:
                continue
            d = np.where(r == m, 0.0, r - m) if np.isinf(m) else r - m
            s = d - np.log(np.exp(d).sum())
            for v in np.lexsort((np.arange(V), -s))[:n_out]:
                if s[v] > -np.inf:
                    cand.append((c + s[v], w, int(v), float(r[v])))
        cand.sort(key=lambda t: (-t[0], t[1], t[2]))
        cand = cand[:n_out] + [(-np.inf, -1, -1, 0.0)] * (n_out - len(cand))
        out.append(cand[:n_out])
    return out


def select_case(sp, logits, cum, n_out, done=None, eos=0):
    ref = plain_select(logits, cum, n_out, done, eos)
    r = sp.sp_beam_select(logits=logits, cum=cum, n_out=n_out, done=done, eos=eos)
    s, p, t = (r[k].cpu().tolist() for k in ("score", "parent", "token"))
    for b, cand in enumerate(ref):
        assert [c[1] for c in cand] == p[b] and [c[2] for c in cand] == t[b], (b, cand, s[b], p[b], t[b])
        for (a, _, _, _), z in zip(cand, s[b]):
            assert a == z or abs(a - z) <= 2.0 ** -24 * abs(a) + 2.0 ** -20


@pytest.mark.parametrize("V", [1, 7, 31, 1000, 2049, 32003])
@pytest.mark.parametrize("W,n_out", [(1, 1), (4, 8), (5, 5), (16, 32)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_sizes(sp, V, W, n_out, dtype):
    g = gen(V + W)
    logits = (3 * torch.randn((3, W, V), device=DEV, generator=g)).to(dtype)
    cum = -5 * torch.rand((3, W), device=DEV, generator=g)
    select_case(sp, logits, cum, n_out)


def test_select_ties_go_to_the_lower_beam_and_token(sp):
    for dtype in (torch.float32, torch.bfloat16):
        logits = torch.zeros((2, 4, 5000), device=DEV, dtype=dtype)
        logits[1] = (torch.arange(5000, device=DEV) % 3).to(dtype)
        cum = torch.zeros((2, 4), device=DEV)
        select_case(sp, logits, cum, 8)
        r = sp.sp_beam_select(logits=logits, cum=cum, n_out=8)
        assert r["token"][0].tolist() == list(range(8)) and r["parent"][0].tolist() == [0] * 8


def test_select_descending_and_ascending_rows(sp):
    up = torch.linspace(-4, 4, 40000, device=DEV)[None, None]
    for x in (up, up.flip(-1), up.repeat(2, 3, 1)):
        select_case(sp, x.contiguous(), torch.zeros(x.shape[:2], device=DEV), 16)


def test_select_masks_infinities_and_nan(sp):
    g = gen(5)
    lowest = torch.finfo(torch.float32).min
    x = torch.randn((8, 2, 3001), device=DEV, generator=g)
    x[0, 0] = -torch.inf                      # a row that leaves nothing
    x[1] = -torch.inf                         # an element that leaves nothing
    x[2, 1, 5:] = -torch.inf                  # fewer tokens than asked for
    x[2, 0] = -torch.inf
    x[3, 0, ::2] = torch.nan
    x[4, 1] = torch.nan
    x[5, 0, [7, 2000]] = torch.inf            # the whole weight on two tokens
    x[6, 0, 100:] = lowest
    x[6, 1] = lowest                          # all equal and as low as the type goes
    cum = -torch.rand((8, 2), device=DEV, generator=g)
    cum[7, 0] = -torch.inf
    select_case(sp, x, cum, 8)
    x16 = x.to(torch.bfloat16)
    select_case(sp, x16, cum, 8)


def test_select_finished_beams_and_rows_apart(sp):
    g = gen(6)
    for V, ld in ((777, 800), (1023, 1025)):
        full = torch.randn((4, 3, ld), device=DEV, generator=g)
        done = torch.tensor([[0, 0, 0], [1, 0, 0], [1, 1, 1], [0, 1, 0]], dtype=torch.bool, device=DEV)
        full[done] = torch.nan  # not read
        cum = -3 * torch.rand((4, 3), device=DEV, generator=g)
        cum[3, 1] = -torch.inf
        select_case(sp, full[..., :V], cum, 6, done, eos=V - 1)
        select_case(sp, full.to(torch.bfloat16)[..., 1:V], cum, 6, done, eos=0)


@pytest.mark.parametrize("W,n_out", [(16, 32), (16, 5), (9, 8), (12, 17)])
def test_select_among_many_beams(sp, W, n_out):
    """Equal scores across all beams, far apart ones, and beams that offer one continuation or none."""
    g = gen(W + n_out)
    x = torch.randn((6, W, 700), device=DEV, generator=g)
    cum = torch.zeros((6, W), device=DEV)
    done = torch.zeros((6, W), dtype=torch.bool, device=DEV)
    x[0] = x[0, :1]                           # every score W times
    x[1] = 0
    cum[2] = -4 * torch.arange(W, device=DEV)[torch.randperm(W, generator=g, device=DEV)]
    cum[3, 1:] = -torch.inf                   # one beam left
    done[4, ::2] = True
    cum[4, 1::4] = -torch.inf
    done[5] = True                            # W candidates in all
    select_case(sp, x, cum, n_out, done, eos=3)
    # Rows of 1,400 bytes start at 0 or 8 bytes past a multiple of 16, and with that the sum of 700 terms is taken in
    # one order or another.  The sums of equal rows then differ by fp32's rounding of their additions (a thread adds no
    # more than 36 terms, 8 additions and 3 scalings join the threads: below 48 halves of an ulp, 48 x 2^-24 < 2^-18),
    # so such scores are equal within the bound and no more, and any of them may stand before another.
    x16 = x.to(torch.bfloat16)
    r = sp.sp_beam_select(logits=x16, cum=cum, n_out=n_out, done=done, eos=3)
    tol = 2.0 ** -18
    for b, cand in enumerate(plain_select(x16, cum, W * 700, done, 3)):
        of = {(w, v): a for a, w, v, _ in cand if w >= 0}
        best = (sorted(of.values(), reverse=True) + [-np.inf] * n_out)[:n_out]
        got = list(zip(*(r[k][b].cpu().tolist() for k in ("parent", "token", "score"))))
        named = [(w, v) for w, v, _ in got if w >= 0]
        assert len(set(named)) == len(named)
        for (w, v, s), a in zip(got, best):
            assert (w, v, s) == (-1, -1, -np.inf) if a == -np.inf else abs(s - a) <= tol and abs(s - of[w, v]) <= tol
        assert [s for _, _, s in got] == sorted((s for _, _, s in got), reverse=True)


# ----------------------------------------------------------------------------- reordering

@pytest.mark.parametrize("W", [1, 3, 4, 8, 16])
@pytest.mark.parametrize("page", [16, 64])
def test_reorder(sp, W, page):
    g = gen(W)
    for lens in ([0, 1], [page - 1, page], [3 * page + 5, 2 * page]):
        R = 2 * W
        own, pages = tables(g, [n + 1 for n in lens for _ in range(W)], page)
        table = own.clone()
        kv = normal(g, 3, 2, pages, page, 24)
        # a first order, then another: full pages are shared by then
        logical = None
        for step in range(2):
            parent = torch.randint(-1, W, (2, W + 1), device=DEV, generator=g, dtype=torch.int32)
            L = [n for n in lens for _ in range(W)]
            rows = lambda kv, t: [kv[:, :, [int(t[r, k // page]) for k in range(L[r])], [k % page for k in range(L[r])]].clone() for r in range(R)]  # noqa: E731
            before = rows(kv, table)
            if logical is not None:
                assert all(torch.equal(a, b) for a, b in zip(before, logical))
            src = [e * W + (int(parent[e, w]) if int(parent[e, w]) >= 0 else w) for e in range(2) for w in range(W)]
            err = sp.sp_beam_reorder(kv=kv, table=table, own_table=own, lens=ints(L), parent=parent[:, :W])
            assert int(err.item()) == 0
            after = rows(kv, table)
            assert all(torch.equal(after[r], before[src[r]]) for r in range(R))
            for r in range(R):
                assert torch.equal(table[r, L[r] // page:], own[r, L[r] // page:])
            logical = after


def test_reorder_refuses_bad_elements_on_the_device(sp):
    g = gen(1)
    W, page = 2, 16
    own, pages = tables(g, [20] * 8, page)
    table = own.clone()
    kv = normal(g, 2, 2, pages, page, 16)
    before, told = kv.clone(), table.clone()
    lens = ints([20, 19, 200, 200, -1, -1, 20, 20])
    err = sp.sp_beam_reorder(kv=kv, table=table, own_table=own, lens=lens, parent=ints([[1, 0]] * 3 + [[2, -2]]))
    assert int(err.item()) == 2
    assert torch.equal(kv, before) and torch.equal(table, told)


# ----------------------------------------------------------------------------- together, refusals

def test_generation_steps_of_beams_together(sp):
    """Five steps of beams over shared prefixes: append, attend, select, reorder, against a cache that every beam has
    for itself."""
    g = gen(21)
    Hq, Hkv, dh, page, W, E, V = 8, 2, 64, 16, 3, 2, 501
    R = E * W
    plens, steps = [40, 21], 20
    both, pages = tables(g, [steps] * R + plens, page)
    own, ptable = both[:R].contiguous(), both[R:].contiguous()
    table = own.clone()
    kv = normal(g, 1, 2, pages, page, Hkv * dh)
    rope = sp.rope_table(256, dh)
    lens = ints([0] * R)
    prefix = [[kv[0, :, [int(ptable[e, k // page]) for k in range(plens[e])], [k % page for k in range(plens[e])]]] for e in range(E)]
    hist = [prefix[e][0].clone() for e in range(E) for _ in range(W)]
    cum = torch.zeros((E, W), device=DEV)
    out_w = normal(g, Hq * dh, V, std=0.2)
    for step in range(steps):
        qkv = normal(g, R, (Hq + 2 * Hkv) * dh)
        pos = lens + ints([plens[e] for e in range(E) for _ in range(W)])
        a = sp.sp_paged_append(qkv=qkv, kv=kv[0], table=table, lens=lens, n_heads=Hq, n_kv_heads=Hkv, head_dim=dh,
                               rope=rope, pos=pos)
        lens += 1
        r = sp.sp_prefix_attention(q=a["q"], kv=kv[0], table=table, lens=lens, n_heads=Hq, n_kv_heads=Hkv, head_dim=dh,
                                   prefix_table=ptable, prefix_lens=ints(plens), group_cu=ints([0, W, 2 * W]))
        for b in range(R):
            k = int(lens[b]) - 1
            new = kv[0, :, int(table[b, k // page]), k % page]
            hist[b] = torch.cat((hist[b], new[:, None]), dim=1)
            x = hist[b].double().view(2, -1, Hkv, dh)
            z = torch.einsum("hgd,khd->hgk", a["q"][b].double().view(Hkv, Hq // Hkv, dh), x[0]) * dh ** -0.5
            w = torch.softmax(z, dim=-1)
            o, size = (torch.einsum("hgk,khd->hgd", w, v).reshape(-1) for v in (x[1], x[1].abs()))
            assert ((r["out"][b].double() - o).abs() <= U * o.abs() + (U + 2.0 ** -12) * size).all(), (step, b)
        logits = (r["out"] @ out_w).view(E, W, V)
        s = sp.sp_beam_select(logits=logits, cum=cum, n_out=W)
        cum = s["score"]
        err = sp.sp_beam_reorder(kv=kv, table=table, own_table=own, lens=lens, parent=s["parent"])
        assert int(err.item()) == 0 and int(a["err"].item()) == 0 and int(r["err"].item()) == 0
        hist = [hist[e * W + int(s["parent"][e, w])].clone() for e in range(E) for w in range(W)]


@pytest.mark.parametrize("wide,offsets", [(False, False), (True, True), (True, False)])
def test_calls_on_another_stream_and_two_at_once(sp, wide, offsets):
    """Two calls with workspaces of their own on two streams give what they give one after the other."""
    g = gen(31)
    Hq, Hkv, dh, page = 28, 4, 128, 16
    sets = []
    for _ in range(2):
        table, pages = tables(g, [100] * 20 + [900], page)
        sets.append(dict(q=normal(g, 20, Hq * dh), kv=normal(g, 2, pages, page, Hkv * dh), table=table[:20].contiguous(),
                         lens=ints([100] * 20), prefix_table=table[20:].contiguous(), prefix_lens=ints([900]),
                         group_cu=ints([0, 20]), n_heads=Hq, n_kv_heads=Hkv, head_dim=dh))
        if wide:
            sets[-1].update(prefix_table=widen(sets[-1]["prefix_table"], page))
        if offsets:
            sets[-1].update(cu_rows=starts([1] * 20))
    ref = [sp.sp_prefix_attention(**s)["out"].clone() for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for s, st in zip(sets, streams):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got.append(sp.sp_prefix_attention(**s))
    torch.cuda.synchronize()
    for a, b in zip(ref, got):
        assert torch.equal(a, b["out"])


def test_binding_refuses_wrong_tensors(sp):
    g = gen(2)
    kv = normal(g, 2, 4, 16, 64)
    q, t, n = normal(g, 2, 64), ints([[0], [1]]), ints([1, 1])
    call = lambda **k: sp.sp_prefix_attention(**dict(dict(q=q, kv=kv, table=t, lens=n, n_heads=1, n_kv_heads=1, head_dim=64), **k))  # noqa: E731
    call()
    for bad in (dict(q=q.float()), dict(q=q[:, :32]), dict(kv=kv.cpu()), dict(table=t.long()), dict(lens=ints([1])),
                dict(out=normal(g, 3, 64)), dict(lse=torch.zeros(2, 2, device=DEV)), dict(kv=kv.transpose(1, 2))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(head_dim=32, n_heads=2, n_kv_heads=2), dict(scale=-1.0), dict(ws=torch.empty(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(sp.SPError):
            call(**bad)


def test_attention_reports_offsets_that_do_not_ascend(sp):
    """Group and row offsets that run back: nothing outside the buffers is touched.  The workspace has room for
    floor(40 / 16) + 6 row tiles of prefixes and floor(40 / 16) + 4 of own keys, 14; the first offsets ask for
    3 x 3 + 2 x 3 = 15, which the error word reports, the second for 3 x 3 + 4 = 13, which fit.  (Short tables: no
    workspace is used.)"""
    g = gen(14)
    kv = normal(g, 2, 8, 16, 64)
    q = normal(g, 40, 64)
    ws = sp.prefix_attention_workspace(T_cap=40, B=4, n_heads=1, n_kv_heads=1, head_dim=64, n_groups=6)
    n = ws.numel()
    big = torch.full((n + (1 << 20),), 7, dtype=torch.uint8, device=DEV)
    groups = [0, 4, 0, 4, 0, 4, 0]
    for cu, err, wide in (([0, 40, 0, 40, 40], 2, True), ([0, 10, 20, 30, 40], 0, True), ([0, 40, 0, 40, 40], None, False),
                          ([0, 10, 20, 30, 40], 0, False)):
        prefix = ints([[4, 5]] * 6)
        out = torch.full((44, 64), 7.0, dtype=torch.bfloat16, device=DEV)
        r = sp.sp_prefix_attention(q=q, kv=kv, table=ints([[0], [1], [2], [3]]), lens=ints([16, 16, 16, 16]), n_heads=1,
                                   n_kv_heads=1, head_dim=64, cu_rows=ints(cu), prefix_table=widen(prefix, 16) if wide else prefix,
                                   prefix_lens=ints([32] * 6), group_cu=ints(groups), out=out[:40], ws=big[:n])
        assert err is None or int(r["err"].item()) == err
        assert (out[40:] == 7).all() and (big[n:] == 7).all()
