"""The model over a paged cache, where test_gpu_paged_model.py does not reach: bits of the cached keys, wide tables."""
import numpy as np
import pytest

from oracle import core as O
from paper_2609_13804_gb300 import synth as S

import _parity as PT

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_paged_model import B, DEV, _model, _prefill, ints, single_precision  # noqa: E402, F401


@pytest.mark.parametrize("heads", [(4, 2, 64), (2, 2, 128)])
def test_the_step_caches_the_dense_steps_keys(B, heads):
    """The first layer's new keys and values are those of sp_decode to the bit: rotated before they are rounded."""
    w, layers, head, model = _model(B, 15, *heads, n_layers=1)
    m, page, lens = w.model, 16, [5, 16, 40]
    _, _, _, kv, table, args, _ = _prefill(B, w, model, lens, page)
    dense = B.kv_cache(model, 3, 80)
    B.sp_prefill(model, kv=dense, **args)
    x = B.dev_bf16(S.bf16_round(S.normal(w.seed, "new", (3, m.d), 0.5)), DEV)
    B.sp_decode(model, x=x, lens=ints(lens), kv=dense, max_len_cap=80)
    o = B.sp_decode_paged(model, x=x, lens=ints(lens), rope_pos=ints(lens), kv=kv, table=table)
    assert int(o["err"].item()) == 0
    for b, n in enumerate(lens):
        assert torch.equal(kv[:, :, int(table[b, n // page]), n % page], dense[:, :, b, n])
    model.close()


def test_a_rotary_position_outside_the_table_leaves_the_cache(B):
    w, layers, head, model = _model(B, 16, 4, 2, 64, max_pos=64)
    m, page, lens = w.model, 16, [5, 16, 9]
    _, _, _, kv, table, _, _ = _prefill(B, w, model, lens, page)
    before = kv.clone()
    x = B.dev_bf16(S.bf16_round(S.normal(w.seed, "new", (3, m.d), 0.5)), DEV)
    o = B.sp_decode_paged(model, x=x, lens=ints(lens), rope_pos=ints([64, 16, -1]), kv=kv, table=table)
    assert int(o["err"].item()) == 2
    changed = [(int(table[1, 1]), 0)]
    for pg, r in changed:
        assert not torch.equal(kv[:, :, pg, r], before[:, :, pg, r])
        before[:, :, pg, r] = kv[:, :, pg, r]
    assert torch.equal(kv, before)
    model.close()


@pytest.mark.parametrize("heads", [(4, 2, 64), (2, 2, 128)])
@pytest.mark.parametrize("groups", [[38, 2], [3, 3]])
def test_decode_steps_of_wide_tables(B, heads, groups):
    """The same steps with tables for more than 16,384 positions: planned attention, of many sequences by the tensor
    kernel, and the merge."""
    w, layers, head, model = _model(B, 17, *heads)
    m, page, R = w.model, 16, sum(groups)
    lens, group_cu = [37, 150], [0, groups[0], R]
    x, cu, pos, kv, table, _, _ = _prefill(B, w, model, lens, page, extra=R)
    rows = []
    O.prefill(x, layers, m, cu, pos, head["final_norm"], store="bf16", kv_out=rows)
    of_prefix = O.cache_from_prefill(rows, cu)
    group = [g for g in range(2) for _ in range(groups[g])]
    cache = [[lc[g] for g in group] for lc in of_prefix]
    wide = torch.full((2 + R, 1025), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    n, at, ws = ints([0] * R), ints([lens[g] for g in group]), None
    for step in range(3):
        x_new = S.bf16_round(S.normal(w.seed, f"new{step}", (R, m.d), 0.5))
        o = B.sp_decode_paged(model, x=B.dev_bf16(x_new, DEV), lens=n, rope_pos=at, kv=kv, table=wide[2:], prefix_table=wide[:2],
                              prefix_lens=ints(lens), group_cu=ints(group_cu), ws=ws)
        ws = o["_ws"]
        assert int(o["err"].item()) == 0
        ref, cache = O.decode_step(x_new, layers, m, cache, head["final_norm"], store="bf16")
        PT.hidden_close(o["hidden"].cpu().numpy().astype(np.float64), ref, f"step {step}")
    assert n.tolist() == [3] * R
    model.close()
