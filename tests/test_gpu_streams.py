"""Calls on a stream that is not torch's current one: what a call allocates and clears is ordered with its kernels."""
import numpy as np
import pytest

from paper_2609_13804_gb300 import synth as S

import _parity as PT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_paged_model import B, DEV, _model, ints, single_precision  # noqa: E402, F401


def behind(call, handle):
    """call(stream) while the current stream is busy for some 50 ms; its results when both streams are done."""
    st = torch.cuda.Stream()
    call(torch.cuda.current_stream())  # (what is made once is made now)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    got = call(st.cuda_stream if handle else st)
    assert st.cuda_stream != torch.cuda.current_stream().cuda_stream
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("handle", [False, True])
def test_an_error_word_is_cleared_before_the_call_sets_it(B, handle):
    kv = torch.zeros((1, 2, 4, 16, 64), dtype=torch.bfloat16, device=DEV)
    q, qkv = (torch.ones((2, n), dtype=torch.bfloat16, device=DEV) for n in (64, 192))
    bad, one = ints([[0], [9]]), ints([1, 1])
    heads = dict(n_heads=1, n_kv_heads=1, head_dim=64)
    own, table, parent = ints([[0], [1]]), ints([[0], [1]]), ints([[7, 0]])
    calls = {
        "append": lambda st: B.sp_paged_append(qkv=qkv, kv=kv[0], table=bad, lens=one, stream=st, **heads)["err"],
        "attention": lambda st: B.sp_prefix_attention(q=q, kv=kv[0], table=bad, lens=one, stream=st, **heads)["err"],
        "reorder": lambda st: B.sp_beam_reorder(kv=kv, table=table, own_table=own, lens=one, parent=parent, stream=st),
    }
    for name, call in calls.items():
        assert int(behind(call, handle).item()) == 2, name


@pytest.mark.parametrize("handle", [False, True])
def test_hidden_states_and_positions_are_cleared_before_they_are_written(B, handle):
    w, layers, head, model = _model(B, 18, 4, 2, 64)
    m, lens = w.model, [37, 1, 20]
    T = sum(lens)
    x = B.dev_bf16(S.bf16_round(S.normal(w.seed, "packed", (T, m.d), 0.5)), DEV)
    cu, pos = PT.lens_cu_pos(lens)
    args = dict(x=x, cu_seqlens=ints(cu.tolist()), pos=ints(pos.tolist()), B=3, T_cap=T, max_seqlen_cap=max(lens))
    pool, table = B.paged_pool(9, 16, m.n_kv_heads, m.head_dim, m.n_layers), ints([[0, 1, 2], [3, 4, 5], [6, 7, 8]])
    dense = B.kv_cache(model, 3, 80)
    B.sp_prefill(model, kv=dense, **args)
    ref = B.sp_prefill(model, **args)["hidden"].clone()
    calls = {
        "prefill": lambda st: B.sp_prefill(model, stream=st, **args)["hidden"],
        "prefill_paged": lambda st: B.sp_prefill_paged(model, kv=pool, table=table, stream=st, **args)["hidden"],
    }
    for name, call in calls.items():
        got = behind(call, handle)
        assert torch.equal(got, ref), name
    x1 = x[:3].contiguous()
    step = lambda st: B.sp_decode(model, x=x1, lens=ints(lens), kv=dense, max_len_cap=80, stream=st)  # noqa: E731
    ref = step(None)["hidden"].clone()
    n = ints(lens)  # (made before the current stream is busy)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    got = B.sp_decode(model, x=x1, lens=n, kv=dense, max_len_cap=80, stream=st.cuda_stream if handle else st)
    torch.cuda.synchronize()
    assert torch.equal(got["hidden"], ref) and int(got["err"].item()) == 0
    idx, count = ints([[0, 3, 5, 9]]), ints([4])
    mp = lambda st: B.sp_mrope_positions([12], [5], [4], idx=idx, count=count, k_cap=4, T_cap=9, stream=st)["pos3"]  # noqa: E731
    assert torch.equal(behind(mp, handle), mp(None))
    model.close()


@pytest.mark.parametrize("handle", [False, True])
def test_a_selection_clears_its_traces_before_it_writes_them(B, handle):
    w = S.tiny_workload(19, [40, 33], [4, 6], D=384, D_text=128, h=128, enc_head_dim=64)
    inp = S.make_inputs(w)
    sel = B.Selector(w.selector, S.make_selector_weights(w), DEV)
    a = dict(X=B.dev_bf16(inp["X"], DEV), E_text=B.dev_bf16(inp["E_text"], DEV), stop_bias=B.dev_f32(np.zeros(2), DEV), k_max=8)
    call = lambda st: B.sp_select(sel, w.n_vis, w.n_txt, stream=st, **a)  # noqa: E731
    ref, got = call(None), behind(call, handle)
    for k in ("idx", "count", "order", "ep_count", "rounds", "err"):
        assert torch.equal(ref[k], got[k]), k
    sel.close()
