"""Verification of many rows that are cut into several slices, in order and not, and sampling from long rows by one CTA to eight."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"

from test_gpu_paged import single_precision  # noqa: E402, F401
from test_gpu_verify import compare, expect, problem  # noqa: E402

V = 60000  # two slices in calls of many waves


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_13804_gb300 import binding
    return binding


@pytest.mark.parametrize("dtype,model,counts", [
    (torch.bfloat16, True, [4 + b % 4 for b in range(240)] + [0, 1, 2, 3] * 4),
    (torch.bfloat16, False, [8 + b % 4 for b in range(240)] + [0, 1, 2, 3] * 4),
    (torch.float32, True, [4 + b % 2 for b in range(160)] + [0, 1, 2, 3]),
    (torch.float32, False, [6 + b % 3 for b in range(170)] + [0, 1, 2, 3]),
])
@pytest.mark.parametrize("pad", [0, 1])
def test_rows_in_order_of_several_slices(sp, dtype, model, counts, pad):
    """More rows than CTAs run at once, more than three to a sequence and more than 2^28 bytes; rows behind a sequence's end may
    hold anything."""
    rows = sum(2 * n - 1 if model and n else n for n in counts)
    assert rows > 608 and rows * V * (4 if dtype is torch.float32 else 2) > 2 ** 28
    s = problem(71 + pad, V, counts, dtype, model, pad, near=0.4)
    want = expect(s)
    got = sp.sp_draft_verify(**s)
    assert int(got["err"].item()) == 0
    compare(got, want, max(counts))
    at = [sum(counts[:b]) for b in range(len(counts))]
    late = [at[b] + j for b, (n, _, _, _) in enumerate(want) for j in range(n + 1, counts[b])]
    assert late
    s["logits"][late] = torch.nan
    if model:
        s["draft_logits"][late] = torch.nan
    again = sp.sp_draft_verify(**s)
    assert all(torch.equal(got[k], again[k]) for k in ("n_accept", "token", "logp"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("model", [True, False])
def test_many_rows_of_several_slices(sp, dtype, model):
    """Sequences of up to three rows: all of them are read."""
    s = problem(73, V, [3, 2, 3, 3] * 64, dtype, model, near=0.4)
    got = sp.sp_draft_verify(**s)
    assert int(got["err"].item()) == 0
    compare(got, expect(s), 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B", [256, 152, 101, 76, 50, 38])  # 1, 2, 3, 4, 6 and 8 CTAs to a row on 152 SMs
def test_sampling_from_long_rows(sp, dtype, B):
    s = problem(75 + B, V + 1, [1] * B, dtype, False, pad=B % 2)
    got = sp.sp_draft_verify(**dict(s, cu_rows=None, draft=None, u=None))
    assert int(got["err"].item()) == 0
    compare(got, expect(s), 1)
