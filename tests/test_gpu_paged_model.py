"""The model over a paged cache: sp_prefill_paged and sp_decode_paged against sp_prefill and the oracle, and beams
generated with them, sp_beam_select and sp_beam_reorder.

sp_prefill_paged does the arithmetic of sp_prefill: equal bits.  sp_decode_paged does that of sp_decode up to the
attention, which weighs and adds in another order; both are inside the bounds of hidden_close, which hold a whole
layer's bf16 roundings."""
import numpy as np
import pytest

from oracle import core as O
from paper_2609_13804_gb300 import synth as S

import _parity as PT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(autouse=True)
def single_precision():
    """Tensors without a type of their own are fp32, whatever another module has set."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_13804_gb300 import binding
    binding.lib()
    return binding


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _model(B, seed, n_heads, n_kv, dh, n_layers=2, max_pos=256):
    w = S.tiny_workload(seed, [16], [4], D=128, D_text=256, h=128, d=256, n_heads=n_heads, n_kv_heads=n_kv, head_dim=dh,
                        ffn=256, n_layers=n_layers, k_max=8)
    layers = [S.make_layer_weights(w, l, norm_affine=True) for l in range(n_layers)]
    head = S.make_model_head(w, norm_affine=True)
    return w, layers, head, B.Model(w.model, layers, head, DEV, max_pos=max_pos)


def _prefill(B, w, model, lens, page, extra=0):
    """A prefill into scattered pages: the pools, the prefixes' tables and the tables of `extra` further rows."""
    m = w.model
    T = sum(lens)
    x = S.bf16_round(S.normal(w.seed, "packed", (T, m.d), 0.5))
    cu, pos = PT.lens_cu_pos(lens)
    need = max(-(-n // page) for n in lens) + 1
    g = torch.Generator(device=DEV).manual_seed(w.seed)
    ids = torch.randperm((len(lens) + extra) * need, device=DEV, generator=g).to(torch.int32)
    table = ids.view(len(lens) + extra, need).contiguous()
    kv = B.paged_pool(ids.numel(), page, m.n_kv_heads, m.head_dim, m.n_layers)
    args = dict(x=B.dev_bf16(x, DEV), cu_seqlens=ints(cu.tolist()), pos=ints(pos.tolist()), B=len(lens), T_cap=T,
                max_seqlen_cap=max(lens))
    out = B.sp_prefill_paged(model, kv=kv, table=table[:len(lens)].contiguous(), **args)
    assert int(out["err"].item()) == 0
    return x, cu, pos, kv, table, args, out


@pytest.mark.parametrize("heads", [(4, 2, 64), (2, 2, 128)])
@pytest.mark.parametrize("page", [16, 64])
def test_prefill_puts_the_same_rows_into_pages(B, heads, page):
    w, layers, head, model = _model(B, 11, *heads)
    lens = [37, 1, 64, 20]
    _, cu, _, kv, table, args, out = _prefill(B, w, model, lens, page)
    dense = B.kv_cache(model, len(lens), 80)
    ref = B.sp_prefill(model, kv=dense, **args)
    torch.cuda.synchronize()
    assert torch.equal(ref["hidden"], out["hidden"])
    used = torch.zeros(kv.shape[2], page, dtype=torch.bool, device=DEV)
    for b, n in enumerate(lens):
        for j in range(n):
            pg, r = int(table[b, j // page]), j % page
            used[pg, r] = True
            assert torch.equal(kv[:, :, pg, r], dense[:, :, b, j])
    assert (kv[:, :, ~used] == 0).all()
    with pytest.raises(B.SPError):  # one cache or the other
        io_kv = B.sp_prefill_io(1, 1, 1, 16, 16, 16, 16, None, None, 16, 1, None)
        pools = B.sp_paged_kv(16, 1, 16, 16, 1, None)
        B._check(B.lib().sp_prefill_paged(model.handle, B.C.byref(io_kv), B.C.byref(pools), None, 0, None), "sp_prefill_paged")
    model.close()


@pytest.mark.parametrize("heads", [(4, 2, 64), (2, 2, 128)])
def test_decode_steps_share_prefixes(B, heads):
    """Six sequences on two prefixes and one that has none of its own group's: steps against the oracle, which gives
    every sequence a cache of its own."""
    w, layers, head, model = _model(B, 12, *heads)
    m, page, steps = w.model, 16, 18
    lens, group_cu = [37, 20], [0, 4, 6]
    x, cu, pos, kv, table, _, _ = _prefill(B, w, model, lens, page, extra=6)
    rows = []
    O.prefill(x, layers, m, cu, pos, head["final_norm"], store="bf16", kv_out=rows)
    of_prefix = O.cache_from_prefill(rows, cu)
    group = [g for g in range(2) for _ in range(group_cu[g], group_cu[g + 1])]
    cache = [[lc[g] for g in group] for lc in of_prefix]
    own, prefix = table[2:].contiguous(), table[:2].contiguous()
    n, at = ints([0] * 6), ints([lens[g] for g in group])
    ws = None
    for step in range(steps):
        x_new = S.bf16_round(S.normal(w.seed, f"new{step}", (6, m.d), 0.5))
        o = B.sp_decode_paged(model, x=B.dev_bf16(x_new, DEV), lens=n, rope_pos=at, kv=kv, table=own, prefix_table=prefix,
                              prefix_lens=ints(lens), group_cu=ints(group_cu), ws=ws)
        ws = o["_ws"]
        assert int(o["err"].item()) == 0
        ref, cache = O.decode_step(x_new, layers, m, cache, head["final_norm"], store="bf16")
        PT.hidden_close(o["hidden"].cpu().numpy().astype(np.float64), ref, f"step {step}")
    assert n.tolist() == [steps] * 6 and at.tolist() == [lens[g] + steps for g in group]
    model.close()


def test_decode_without_prefixes_and_past_the_table(B):
    w, layers, head, model = _model(B, 13, 4, 2, 64)
    m, page = w.model, 16
    lens = [5, 16]
    x, cu, pos, kv, table, _, _ = _prefill(B, w, model, lens, page)
    rows = []
    O.prefill(x, layers, m, cu, pos, head["final_norm"], store="bf16", kv_out=rows)
    cache = O.cache_from_prefill(rows, cu)
    n, at = ints(lens), ints(lens)
    x_new = S.bf16_round(S.normal(w.seed, "new", (2, m.d), 0.5))
    o = B.sp_decode_paged(model, x=B.dev_bf16(x_new, DEV), lens=n, rope_pos=at, kv=kv, table=table[:2].contiguous())
    assert int(o["err"].item()) == 0
    ref, _ = O.decode_step(x_new, layers, m, cache, head["final_norm"], store="bf16")
    PT.hidden_close(o["hidden"].cpu().numpy().astype(np.float64), ref, "step")
    before = kv.clone()
    o = B.sp_decode_paged(model, x=B.dev_bf16(x_new, DEV), lens=ints([32, 32]), rope_pos=at, kv=kv, table=table[:2].contiguous())
    assert int(o["err"].item()) == 2 and torch.equal(kv, before)
    model.close()


def test_beam_generation_replays_in_a_graph(B):
    """A whole step of beam generation (decode, logits, selection, reordering) captured once and replayed gives the
    bits of the same steps issued one by one."""
    w, layers, head, model = _model(B, 14, 4, 2, 64)
    m, page, W, V, steps = w.model, 16, 3, 301, 19
    lens = [37, 20]
    R = 2 * W
    emb = (0.5 * torch.randn((V, m.d), device=DEV, generator=torch.Generator(device=DEV).manual_seed(5))).to(torch.bfloat16)
    runs = []
    for graph in (False, True):
        _, _, _, kv, table, _, _ = _prefill(B, w, model, lens, page, extra=R)
        prefix, own = table[:2].contiguous(), table[2:].contiguous()
        t = own.clone()
        n, at = ints([0] * R), ints([lens[g] for g in range(2) for _ in range(W)])
        cum = torch.tensor([[0.0] + [-torch.inf] * (W - 1)] * 2, device=DEV)
        x = emb[1][None].repeat(R, 1).contiguous()
        out = {k: torch.empty((2, W), dtype=d, device=DEV) for k, d in (("score", torch.float32), ("parent", torch.int32), ("token", torch.int32))}
        hid, err = torch.empty((R, m.d), device=DEV), ints([0])
        ws = torch.empty(B.lib().sp_decode_paged_workspace(model.handle, R, 2), dtype=torch.uint8, device=DEV)
        ws2 = B.beam_select_workspace(B=2, W=W, V=V, n_out=W)
        pl, gc = ints(lens), ints([0, W, R])

        def step():
            B.sp_decode_paged(model, x=x, lens=n, rope_pos=at, kv=kv, table=t, prefix_table=prefix, prefix_lens=pl, group_cu=gc,
                              hidden=hid, ws=ws, err=err)
            logits = (hid @ emb.float().T).view(2, W, V)
            B.sp_beam_select(logits=logits, cum=cum, n_out=W, ws=ws2, **out)
            B.sp_beam_reorder(kv=kv, table=t, own_table=own, lens=n, parent=out["parent"], err=err)
            cum.copy_(out["score"])
            x.copy_(emb[out["token"].view(-1).clamp(min=0).long()])

        seen = []
        if graph:
            state = [v.clone() for v in (kv, t, n, at, cum, x)]
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                step()  # (what the libraries allocate is allocated now)
            torch.cuda.current_stream().wait_stream(s)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            for v, o in zip((kv, t, n, at, cum, x), state):
                v.copy_(o)
        for _ in range(steps):
            g.replay() if graph else step()
            seen.append((out["token"].clone(), out["parent"].clone(), out["score"].clone(), hid.clone()))
        assert int(err.item()) == 0
        runs.append((seen, kv, t))
    for a, b in zip(runs[0][0], runs[1][0]):
        assert all(torch.equal(u, v) for u, v in zip(a, b))
    assert torch.equal(runs[0][1], runs[1][1]) and torch.equal(runs[0][2], runs[1][2])
    model.close()
