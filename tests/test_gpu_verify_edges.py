"""Sampling and verification where a row's candidates have no weight next to its largest logit, drafts that are no token."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"

from test_gpu_paged import single_precision  # noqa: E402, F401
from test_gpu_verify import compare, expect, gen, ints, problem, rows  # noqa: E402


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_13804_gb300 import binding
    return binding


def as_rows_of_sequences(sp, s):
    """The same tokens by the kernels for drafts: sequences of one row in a call of up to two."""
    B = s["logits"].shape[0]
    r = sp.sp_draft_verify(**dict(s, cu_rows=torch.arange(B + 1, dtype=torch.int32, device=DEV), max_rows=2, draft=ints([0] * B),
                                  u=torch.zeros(B, device=DEV)))
    assert (r["token"][:, 1] == -1).all()
    return r["n_accept"], r["token"][:, 0], r["logp"][:, 0]


# One CTA to a sequence (256 of them), and several: a thread's later tokens lie 1,024 apart (fp32: pairs of such fours).
LATER = [1, 2, 3, 4, 1024, 2048, 4096, 8192]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,pad", [(256, 9000, 0), (256, 9001, 1), (256, 8997, 3), (3, 40000, 0), (3, 39999, 1)])
def test_noise_of_zero_where_the_weight_is_zero(sp, dtype, B, V, pad):
    """A token 900 temperatures below the largest logit has no weight in 64 bits either: its noise of 0 makes it no candidate,
    and takes nothing from the tokens behind it, in its row or beside it."""
    g = gen(51 + B + pad)
    x = torch.full((B, V), -80.0, device=DEV)
    noise = torch.empty((B, V), device=DEV).exponential_(generator=g)
    early = torch.randint(0, 800, (B,), device=DEV, generator=g)
    late = early + ints([LATER[b % len(LATER)] for b in range(B)]).long()
    late[:2] = ints([V - 1, 0]).long()  # beside the whole pieces
    at = torch.arange(B, device=DEV)
    noise[at, early] = 0.0
    early[1] = 5
    noise[1, 5] = 0.0
    x[at, late] = 10.0
    s = dict(logits=rows(x, pad, dtype), noise=noise, temperature=torch.full((B,), 0.1, device=DEV))
    got = sp.sp_draft_verify(**s)
    assert got["token"][:, 0].tolist() == late.tolist()
    assert (got["n_accept"] == 0).all() and (got["logp"] == 0.0).all()
    n, token, logp = as_rows_of_sequences(sp, s)
    assert torch.equal(token, got["token"][:, 0]) and torch.equal(logp, got["logp"][:, 0])
    # with some weight it wins
    x[at, early] = 9.0
    x[at, late] = 10.0
    s["logits"] = rows(x, pad, dtype)
    won = sp.sp_draft_verify(**s)["token"][:, 0]
    assert torch.equal(torch.where(early == late, late, early), won.long())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V", [(256, 9000), (5, 33000)])
def test_masked_tokens_with_noise_of_zero(sp, dtype, B, V):
    """Masks of the type's lowest value, and noise that a program has set to 0 at masked tokens."""
    s = problem(53 + B, V, [1] * B, dtype, False, temps=(1.0, 0.3, 0.05))
    g = gen(54)
    masked = torch.rand((B, V), device=DEV, generator=g) < 0.9
    s["logits"][masked] = torch.finfo(dtype).min
    s["noise"][masked & (torch.rand((B, V), device=DEV, generator=g) < 0.5)] = 0.0
    got = sp.sp_draft_verify(**s)
    compare(got, expect(s), 1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gap", [4, 1024, 2048, 4096, 8192])
@pytest.mark.parametrize("low,mid", [(-80.0, 9.0), (-4.0, 3.0)])
def test_what_a_token_without_weight_was_ahead_of(sp, dtype, gap, low, mid):
    """Token 5 has noise 0 and no weight, the largest logit's token is not to be drawn: token 6 is what is left.  (Next to token
    6 alone, 70 temperatures below it, token 5 would have some.)"""
    B, V = 256, 9000
    x = torch.full((B, V), -math.inf, device=DEV)
    noise = torch.ones((B, V), device=DEV)
    x[:, 5], x[:, 6], x[:, 5 + gap] = low, mid, 10.0
    noise[:, 5], noise[:, 5 + gap] = 0.0, math.nan
    s = dict(logits=x.to(dtype), noise=noise, temperature=torch.full((B,), 0.1, device=DEV))
    got = sp.sp_draft_verify(**s)
    assert (got["n_accept"] == 0).all() and (got["token"] == 6).all()
    n, token, logp = as_rows_of_sequences(sp, s)
    assert (token == 6).all() and torch.equal(logp, got["logp"][:, 0])


@pytest.mark.parametrize("draft", [2 ** 31 - 1, 700, -1, -2 ** 31])
def test_a_draft_that_is_no_token_behind_a_row_without_weight(sp, draft):
    """Greedy: such a row has no largest logit, and no draft is equal to that."""
    s = problem(57, 700, [3, 3, 3], temps=(0.0, 1.0, 0.0))
    s["logits"][[0, 3]] = math.nan
    s["logits"][6] = -math.inf
    s["draft"][[0, 3, 6]] = draft
    for noise in (s["noise"], None):
        got = sp.sp_draft_verify(**dict(s, noise=noise))
        assert int(got["err"].item()) == 2
        assert got["n_accept"].tolist() == [0, 0, 0]
        assert got["token"].tolist() == [[-1] * 3] * 3
        assert got["logp"].tolist() == [[-math.inf, 0.0, 0.0]] * 3


def test_a_workspace_for_the_largest_step_serves_smaller_ones(sp):
    for T, B, V in ((406, 64, 32000), (244, 64, 152064), (700, 256, 50001), (40, 8, 300000)):
        most = sp.draft_verify_workspace(T_cap=T, B=B, V=V).numel()
        for t in sorted(set(range(1, T + 1, 7)) | {T - 1, T // 2, 1}):
            for b in {1, B // 2, B}:
                for v in {1, 2049, V // 2, V - 1, V}:
                    assert sp.draft_verify_workspace(T_cap=t, B=b, V=v).numel() <= most, (t, b, v)
    s = problem(59, 32000, [7] * 15 + [6] * 50, torch.bfloat16, temps=(0.0,))  # 405 rows
    ws = sp.draft_verify_workspace(T_cap=406, B=65, V=32000)
    got = sp.sp_draft_verify(**dict(s, ws=ws))
    assert all(torch.equal(got[k], v) for k, v in sp.sp_draft_verify(**s).items() if k in ("n_accept", "token", "logp"))


def test_sequences_beside_wrong_offsets(sp):
    """Those that are right, and share no row with a wrong one, are what they are alone."""
    s = problem(61, 400, [3, 3, 3, 3])
    for cu, right in (([0, 4, 6, 9, 12], [1, 2, 3]), ([-1, 2, 5, 8, 13], [1, 2]), ([0, 3, 13, 9, 12], [0, 3]),
                      ([0, 3, 3, 7, 9], [0, 3])):
        got = sp.sp_draft_verify(**dict(s, cu_rows=ints(cu)))
        assert int(got["err"].item()) == 2
        for b in right:
            i, j = cu[b], cu[b + 1]
            one = {k: s[k][i:j] for k in ("logits", "draft_logits", "draft", "u")}
            one.update(noise=s["noise"][b:b + 1], temperature=s["temperature"][b:b + 1], cu_rows=ints([0, j - i]))
            want = expect(one)
            assert want[0][3]  # (clear)
            compare({k: got[k][b:b + 1] for k in ("n_accept", "token", "logp")}, want, 3)


# A decision compares u q(d) sum(p) with p(d) sum(q), sums and weights next to the rows' maxima.  In steps of 2^-24: log2 e / t
# is off by 1.5, x - m, its product and an exponential by 1, 1 and 4; so a weight of 2^-z is off by ln 2 * 3.5 z + 4 < 2.5 z + 4,
# and with the two of a decision, their three products and two sums of 2^-17.5 = 91 the whole by less than 5 z + 8 + 3 + 2 * 91.
def near(z):
    return (200 + 5 * z) * 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("model", [True, False])
def test_decisions_about_unlikely_tokens(sp, dtype, model):
    """Drafts down to 2^-110 of the likeliest token's probability, u a quarter more than the bound to either side of p / q."""
    g, V, B = gen(63), 32000, 240
    x = torch.randn((2 * B, V), device=DEV, generator=g) * 2
    y = x + 0.7 * torch.randn((2 * B, V), device=DEV, generator=g)
    t = torch.tensor([(1.0, 0.7, 1.5)[b % 3] for b in range(B)], device=DEV)
    d = torch.randint(0, V, (2 * B,), device=DEV, generator=g)
    first = torch.arange(0, 2 * B, 2, device=DEV)
    down = torch.linspace(0, 110, B, device=DEV)
    for v, z in ((x, down), (y, down[torch.randperm(B, device=DEV, generator=g)])):
        v[first, d[first]] = v[first].amax(dim=1) - z * math.log(2.0) * t
    x, y = x.to(dtype), y.to(dtype)
    lp = torch.log_softmax(x[first].double() / t.double()[:, None], dim=1).gather(1, d[first, None])[:, 0]
    lq = torch.log_softmax(y[first].double() / t.double()[:, None], dim=1).gather(1, d[first, None])[:, 0] if model else lp * 0
    z = -torch.minimum(lp, lq) / math.log(2.0)  # (no less than below the likeliest)
    side = torch.where(torch.arange(B, device=DEV) % 2 == 0, 1.0, -1.0).double()
    u = torch.ones(2 * B, device=DEV)
    u[first] = ((lp - lq).exp() * (1 + 1.25 * near(z) * side)).float()
    got = sp.sp_draft_verify(logits=x, draft_logits=y if model else None, draft=d.int(), u=u, max_rows=2, temperature=t,
                             noise=torch.ones((B, V), device=DEV), cu_rows=torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device=DEV))
    assert got["n_accept"].tolist() == (side < 0).int().tolist()
