"""Verification of drafted tokens against a plain computation in 64 bits, draft by draft."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"

from test_gpu_paged import single_precision  # noqa: E402, F401

# Sums are fp32.  exp((x - m) / t) is ex2 of z = (x - m) c with three roundings of 2^-24 in z (relative), 2^-22 of the
# approximation: a term is off by at most ln 2 * 3 * 2^-24 |z| + 2^-22 of itself.  Averaged with the terms as weights |z|
# is below log2 V + 2 < 20 for V < 2^18: 2^-18.6 + 2^-22 of the sum; adding up (some 2^10 terms a thread in pieces of 32,
# then pairs) less than 2^-19.  The sum is within 2^-17.5 of itself, and so is log p (absolutely); twice that decides
# between two probabilities or two scores, each a quotient of such sums: 2^-16.
SUM = 2.0 ** -17.5
CLEAR = 2.0 ** -16


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_13804_gb300 import binding
    return binding


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def weights(x):
    """Probabilities of a row's logits, NaN and -infinity without weight, +infinity with all of it."""
    x = np.where(np.isnan(x), -np.inf, x)
    m = x.max()
    if m == -np.inf:
        return np.zeros_like(x)
    e = (x == m).astype(np.float64) if m == np.inf else np.exp(x - m)
    return e / e.sum()


def reference(x, d, y, u, e, t):
    """(drafts that stay, next token, log-probabilities, whether everything is clear) of one sequence; x [n, V] in 64
    bits, d, u [n - 1], y [n - 1, V] or None, e [V] or None."""
    n, V = x.shape
    greedy = e is None or not t > 0
    temp = 1.0 if greedy else t
    out, logp, clear = [], [], True
    for j in range(n):
        p = weights(x[j] / temp)
        best = int(np.nanargmax(np.where(np.isnan(x[j]), -np.inf, x[j]))) if p.sum() > 0 else -1
        last = j == n - 1
        q = None
        if not last:
            there = 0 <= d[j] < V
            if greedy:
                stays = there and d[j] == best
            elif not there or math.isnan(u[j]):
                stays = False
            else:
                q = weights(y[j] / temp) if y is not None else None
                a, b = u[j] * (q[d[j]] if q is not None else 1.0), p[d[j]]
                stays = a < b
                clear &= abs(a - b) > CLEAR * max(a, b) or (a == 0 or b == 0)
            if stays:
                out.append(int(d[j]))
                logp.append(math.log(p[d[j]]))
                continue
        if greedy:
            nxt = best
        else:
            if y is not None and not last:
                q = weights(y[j] / temp)
                r = np.maximum(p - q, 0)
                off = (p + q) * SUM
            else:
                r, off = p.copy(), p * SUM
                if not last and 0 <= d[j] < V:
                    r[d[j]] = 0
            if not r.any():
                r, off = p, p * SUM
            with np.errstate(divide="ignore", invalid="ignore"):
                ok = (r > 0) & (e >= 0)
                score = np.where(ok, r / e, -1.0)
                least = np.where(ok, np.maximum(r - off, 0) / e * (1 - 2.0 ** -20), -1.0)
                most = np.where((p > 0) & (e >= 0), (r + off) / e * (1 + 2.0 ** -20), -1.0)
            nxt = int(score.argmax()) if ok.any() else -1
            if nxt >= 0 and score[nxt] < np.inf:
                rest = np.delete(most, nxt)
                clear &= rest.size == 0 or bool(rest.max() < least[nxt])
        out.append(nxt)
        logp.append(math.log(p[nxt]) if nxt >= 0 and p[nxt] > 0 else -math.inf)
        return len(out) - 1, out, logp, clear
    return -1, [], [], True


def compare(got, want, max_rows):
    """want: reference() of every sequence."""
    n_accept, token, logp = (got[k].cpu().numpy() for k in ("n_accept", "token", "logp"))
    clear = 0
    for b, (n, out, lp, sure) in enumerate(want):
        if not sure:
            continue
        clear += 1
        pad = max_rows - len(out)
        assert n_accept[b] == n and token[b].tolist() == out + [-1] * pad, (b, n_accept[b], n, token[b], out)
        for g, w in zip(logp[b], lp + [0.0] * pad):
            assert g == w if math.isinf(w) else abs(g - w) <= 2 * SUM + 2.0 ** -23 * abs(w), (b, g, w)
    assert clear >= len(want) * 0.9
    return clear


def rows(x, pad, dtype):
    y = torch.full((x.shape[0], x.shape[1] + pad), math.nan, dtype=dtype, device=DEV)
    y[:, :x.shape[1]] = x
    return y[:, :x.shape[1]]


def problem(seed, V, counts, dtype=torch.float32, model=True, pad=0, near=0.7, temps=(1.0, 0.7, 0.0, 1.5)):
    g = gen(seed)
    T, B = sum(counts), len(counts)
    x = torch.randn((T, V), device=DEV, generator=g) * 2
    x.scatter_(1, torch.randint(0, V, (T, 6), device=DEV, generator=g), 6.0)
    y = x + near * torch.randn((T, V), device=DEV, generator=g)
    race = torch.empty((T, V), device=DEV).exponential_(generator=g)
    d = (y - race.log()).argmax(dim=1).int()
    noise = torch.empty((B, V), device=DEV).exponential_(generator=g)
    cu = [sum(counts[:b]) for b in range(B + 1)]
    return dict(logits=rows(x, pad, dtype), draft_logits=rows(y, pad, dtype) if model else None, draft=d,
                u=torch.rand(T, device=DEV, generator=g), noise=noise, cu_rows=ints(cu),
                temperature=torch.tensor([temps[b % len(temps)] for b in range(B)], device=DEV), max_rows=max(max(counts), 1))


def expect(s):
    """reference() of every sequence of a problem."""
    host = lambda k: None if s.get(k) is None else s[k].double().cpu().numpy() if s[k].is_floating_point() else s[k].cpu().numpy()  # noqa: E731
    x, y, d, u, e, t = (host(k) for k in ("logits", "draft_logits", "draft", "u", "noise", "temperature"))
    B = s["cu_rows"].numel() - 1 if s.get("cu_rows") is not None else x.shape[0]
    cu = s["cu_rows"].tolist() if s.get("cu_rows") is not None else list(range(B + 1))
    out = []
    for b in range(B):
        i, j = cu[b], cu[b + 1]
        if j == i:
            out.append((-1, [], [], True))
            continue
        out.append(reference(x[i:j], None if d is None else d[i:j - 1], None if y is None else y[i:j - 1],
                             None if u is None else u[i:j - 1], None if e is None else e[b],
                             1.0 if t is None else float(t[b])))
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 31, 257, 5003, 32000, 50257])
@pytest.mark.parametrize("model,pad", [(True, 0), (True, 3), (False, 8), (False, 1)])
def test_drafts(sp, dtype, V, model, pad):
    s = problem(V + pad, V, [5, 1, 0, 3, 2, 5, 4, 1], dtype, model, pad)
    r = sp.sp_draft_verify(**s)
    assert int(r["err"].item()) == 0
    compare(r, expect(s), s["max_rows"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,B", [(1, 1), (9, 3), (1000, 256), (32000, 5), (152063, 2)])
def test_one_token_each(sp, dtype, V, B):
    s = problem(V, V, [1] * B, dtype, False)
    want = expect(s)
    for extra in (dict(), dict(cu_rows=None), dict(cu_rows=None, draft=None, u=None)):
        r = sp.sp_draft_verify(**dict(s, **extra))
        assert int(r["err"].item()) == 0
        compare(r, want, 1)


def test_many_drafts_and_wide_rows(sp):
    for V, counts in ((40, [33, 9, 8, 17]), (300001, [3, 2])):
        s = problem(3, V, counts, torch.bfloat16, near=0.1, temps=(1.0, 0.8))
        compare(sp.sp_draft_verify(**s), expect(s), s["max_rows"])


def test_the_largest(sp):
    """More than a thousand drafts of a sequence, and more than four million tokens."""
    s = problem(5, 33, [700, 1, 1024, 0], near=0.02, temps=(1.0, 0.9))
    s["u"][:] = 0.0
    s["u"][1720] = 1e9  # the last sequence ends at its row 1,019
    got = sp.sp_draft_verify(**s)
    compare(got, expect(s), 1024)
    assert got["n_accept"].tolist() == [699, 0, 1019, -1]
    with pytest.raises(sp.SPError):
        sp.sp_draft_verify(**dict(s, max_rows=1025))
    for counts in ([2, 1], [1, 1]):
        s = problem(7, (1 << 22) + 3, counts, torch.bfloat16, near=0.2, temps=(1.0, 0.0))
        compare(sp.sp_draft_verify(**s), expect(s), max(counts))


def test_a_graph_of_rows_in_order(sp):
    """Replayed, with other numbers in the same place."""
    s = problem(9, 50001, [6] * 128, near=0.4)
    u = s["u"].clone()
    ref = [sp.sp_draft_verify(**dict(s, u=v)) for v in (u, u * 0.0)]
    out = dict(ws=sp.draft_verify_workspace(T_cap=768, B=128, V=50001), err=ints([0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = sp.sp_draft_verify(**s, **out)
    for i in (1, 0, 1):
        s["u"].copy_(u * (1 - i))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], ref[i][k]) for k in ("n_accept", "token", "logp"))


def test_a_large_batch(sp):
    """More rows than CTAs that run at once."""
    s = problem(4, 9000, [1 + b % 6 for b in range(256)], torch.bfloat16)
    compare(sp.sp_draft_verify(**s), expect(s), 6)


def test_rows_in_order(sp):
    """Enough reading (more than 2^28 bytes of more rows than CTAs run at once) for rows behind a rejected draft to be passed
    over: 1,396 rows of 50,001 fp32 logits, some of NaN where nothing may look."""
    counts = [6] * 126 + [2, 4]
    s = problem(6, 50001, counts, near=0.4)
    want = expect(s)
    got = sp.sp_draft_verify(**s)
    assert int(got["err"].item()) == 0
    compare(got, want, 6)
    first = [6 * b for b in range(126)]
    late = [first[b] + n + 1 for b, (n, _, _, _) in enumerate(want[:126]) if n < 5]  # the row behind a sequence's end
    s["logits"][late] = torch.nan
    s["draft_logits"][late] = torch.nan
    again = sp.sp_draft_verify(**s)
    assert all(torch.equal(got[k], again[k]) for k in ("n_accept", "token", "logp"))
    s["cu_rows"][5], s["cu_rows"][9] = 20, 60  # rows that belong to two, or to none: nothing outside is touched
    r = sp.sp_draft_verify(**s)
    assert int(r["err"].item()) == 2
    assert ((r["token"] >= -1) & (r["token"] < 50001)).all()


@pytest.mark.parametrize("max_rows", [1, 3])
def test_a_padded_batch(sp, max_rows):
    """Sequences without rows and rows without a sequence, which are not read."""
    counts = [max_rows, 0, 1, 0]
    s = problem(8, 1001, counts)
    T = sum(counts)
    for k in ("logits", "draft_logits"):
        s[k] = torch.cat((s[k], torch.full((3, 1001), torch.nan, device=DEV)))
    s["draft"] = torch.cat((s["draft"], ints([1 << 30] * 3)))
    s["u"] = torch.cat((s["u"], torch.full((3,), torch.nan, device=DEV)))
    s["max_rows"] = max_rows
    got = sp.sp_draft_verify(**s)
    assert int(got["err"].item()) == 0
    compare(got, expect(s), max_rows)
    # as a program's graph has it: wide strides, an error word that is kept
    err = ints([8])
    wide = torch.zeros((4, 1203), device=DEV)
    wide[:, :1001] = s["noise"]
    again = sp.sp_draft_verify(**dict(s, noise=wide[:, :1001], err=err))
    assert int(err.item()) == 8 and all(torch.equal(got[k], again[k]) for k in ("n_accept", "token", "logp"))
    none = sp.sp_draft_verify(**dict(s, logits=s["logits"][:0], draft_logits=s["draft_logits"][:0], draft=s["draft"][:0], u=s["u"][:0],
                                     cu_rows=ints([0] * 5)))
    assert int(none["err"].item()) == 0 and (none["n_accept"] == -1).all() and (none["token"] == -1).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks_infinities_and_nan(sp, dtype):
    V = 777
    s = problem(11, V, [3] * 12, dtype, temps=(1.0, 0.5, 0.0))
    x, y = s["logits"], s["draft_logits"]
    low = torch.finfo(dtype).min
    x[0], x[1] = -math.inf, -math.inf                      # nothing left at all
    x[3, 100:] = -math.inf                                # a mask
    y[3, 50:] = -math.inf
    x[6, 5:] = low                                        # masked with the lowest value
    x[9, 7], x[9, 300] = math.inf, math.inf               # all the weight
    x[12, 3::2] = math.nan
    y[12, 1::3] = math.nan
    x[15] = math.nan                                      # nothing
    x[18] = low                                           # even
    y[21] = -math.inf                                     # a draft without weight: p > 0 stays
    x[24, :] = -math.inf
    x[24, 776] = 1.0                                      # one token left
    s["draft"][24] = 776
    s["u"][27] = math.nan
    y[30], y[31] = x[30], x[31]                           # the same distribution: drafts stay
    s["noise"][1, 3] = 0.0
    s["noise"][4, ::2] = math.inf
    s["noise"][7, ::2] = math.nan
    r = sp.sp_draft_verify(**s)
    want = expect(s)
    assert int(r["err"].item()) == 0
    compare(r, want, 3)
    assert want[0][:2] == (0, [-1]) and want[5][1][0] == -1


def test_equal_logits_and_equal_scores(sp):
    """The lowest token wins, wherever it lies in a slice."""
    V = 40003
    for pad in (0, 5):
        x = torch.zeros((8, V), device=DEV)
        at = [0, 3, 4, 1024, 4095, 20001, 39999, 40002]
        for b, v in enumerate(at):
            x[b, v] = 2.0
            x[b, -1] = 2.0
        for dtype in (torch.float32, torch.bfloat16):
            r = sp.sp_draft_verify(logits=rows(x, pad, dtype))
            assert r["token"].flatten().tolist() == at
            assert sp.sp_draft_verify(logits=rows(x * 0 - 5, pad, dtype))["token"].flatten().tolist() == [0] * 8
            # as scores: 2 and 2 for equal probabilities and noise
            e = torch.full((8, V), 4.0, device=DEV)
            for b, v in enumerate(at):
                e[b, v] = e[b, -1] = 0.5
            r = sp.sp_draft_verify(logits=rows(x * 0 - 5, pad, dtype), noise=e)
            assert r["token"].flatten().tolist() == at


@pytest.mark.parametrize("t", [1e-38, 1e-3, 30.0, 1e30, math.inf])
def test_temperatures(sp, t):
    s = problem(17, 5000, [4, 3, 2], temps=(t,))
    with np.errstate(invalid="ignore"):
        want = expect(s) if t < math.inf else expect(dict(s, temperature=torch.full((3,), 1e30, device=DEV)))
    got = sp.sp_draft_verify(**s)
    for b, (n, out, lp, sure) in enumerate(want):  # (nearly even rows have nearly equal scores only by chance)
        if sure:
            assert got["n_accept"][b] == n and got["token"][b].tolist() == out + [-1] * (4 - len(out))


def test_without_noise_everything_is_greedy(sp):
    s = problem(19, 3001, [4, 2, 5], near=0.0)
    s["draft"] = s["logits"].argmax(dim=1).int()
    s["draft"][2] = 5
    got = sp.sp_draft_verify(**dict(s, noise=None, u=None))
    compare(got, expect(dict(s, noise=None)), 5)
    assert got["n_accept"].tolist() == [2, 1, 4]
    zero = sp.sp_draft_verify(**dict(s, temperature=torch.zeros(3, device=DEV)))
    for k in ("n_accept", "token", "logp"):
        assert torch.equal(zero[k], got[k])


def test_temperatures_that_are_greedy(sp):
    s = problem(21, 700, [3, 2, 4, 1], near=0.1, temps=(-1.0, math.nan, -math.inf, 0.0))
    got = sp.sp_draft_verify(**s)
    compare(got, expect(s), 4)
    none = sp.sp_draft_verify(**dict(s, noise=None))
    assert all(torch.equal(got[k], none[k]) for k in ("n_accept", "token", "logp"))
    one = sp.sp_draft_verify(**dict(s, temperature=None))  # as 1
    compare(one, expect(dict(s, temperature=torch.ones(4, device=DEV))), 4)


def test_offsets_and_drafts_that_are_wrong(sp):
    s = problem(23, 400, [3, 3, 3, 3])
    s["draft"][0], s["draft"][3] = 400, -1
    got = sp.sp_draft_verify(**s)
    assert int(got["err"].item()) == 2
    compare(got, expect(s), 3)
    assert got["n_accept"][:2].tolist() == [0, 0]
    s = problem(23, 400, [3, 3, 3, 3])
    for cu, left in (([0, 4, 6, 9, 12], [1, 2, 3]), ([-1, 2, 6, 9, 13], []), ([0, 3, 2, 5, 12], [0, 2])):
        got = sp.sp_draft_verify(**dict(s, cu_rows=ints(cu)))
        assert int(got["err"].item()) == 2
        for b in range(4):
            i, j = cu[b], cu[b + 1]
            if not 0 <= j - i <= 3 or i < 0 or j > 12:
                assert got["n_accept"][b] == -1 and got["token"][b].tolist() == [-1] * 3 and got["logp"][b].tolist() == [0.0] * 3


def test_tokens_are_distributed_as_the_target(sp):
    """2^15 sequences of one draft: tokens at the first place follow p, whatever q is."""
    g, V, B = gen(29), 6, 256
    x = torch.tensor([1.0, 0.0, 2.0, -1.0, 0.5, -math.inf], device=DEV)
    y = torch.tensor([0.0, 2.0, 0.5, -1.0, -2.0, 1.0], device=DEV)
    p, q = torch.softmax(x, 0), torch.softmax(y, 0)
    for model in (True, False):
        seen = torch.zeros(V, device=DEV)
        for _ in range(128):
            d = torch.multinomial(q, 2 * B, replacement=True, generator=g).int()
            r = sp.sp_draft_verify(logits=x.expand(2 * B, V).contiguous(), draft=d, u=torch.rand(2 * B, device=DEV, generator=g),
                                   draft_logits=y.expand(2 * B, V).contiguous() if model else None, max_rows=2,
                                   noise=torch.empty((B, V), device=DEV).exponential_(generator=g),
                                   cu_rows=torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device=DEV))
            seen += torch.bincount(r["token"][:, 0].long(), minlength=V)
        n = seen.sum()
        assert n == 128 * B
        if model:
            assert ((seen / n - p).abs() <= 6 * (p * (1 - p) / n).sqrt()).all()
        else:  # a certain draft d: p(d) of it stays, the others fill the rest: p again, whatever drew d
            assert ((seen / n - p).abs() <= 6 * (p * (1 - p) / n).sqrt()).all()


def test_two_streams_a_graph_and_what_lies_beside(sp):
    sets = [problem(31 + i, 20001, [3, 5, 1, 2], torch.bfloat16) for i in range(2)]
    ref = [sp.sp_draft_verify(**s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [sp.sp_draft_verify(**s, stream=st) for s, st in zip(sets, streams)]
    torch.cuda.synchronize()
    for a, b in zip(ref, got):
        assert all(torch.equal(a[k], b[k]) for k in ("n_accept", "token", "logp"))
    s = sets[0]
    big = dict(n_accept=torch.full((6,), 7, dtype=torch.int32, device=DEV), token=torch.full((6, 5), 7, dtype=torch.int32, device=DEV),
               logp=torch.full((6, 5), 7.0, device=DEV))
    ws = sp.draft_verify_workspace(T_cap=11, B=4, V=20001)
    wide = torch.full((ws.numel() + 4096,), 7, dtype=torch.uint8, device=DEV)
    out = dict({k: v[1:5] for k, v in big.items()}, ws=wide[:ws.numel()], err=ints([0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.sp_draft_verify(**s, **out)
    for i in (1, 0):  # other inputs in the same place
        for k in ("logits", "draft_logits", "draft", "u", "noise"):
            s[k].copy_(problem(31 + i, 20001, [3, 5, 1, 2], torch.bfloat16)[k])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], ref[i][k]) for k in ("n_accept", "token", "logp"))
    for v in big.values():
        assert (v[0] == 7).all() and (v[5] == 7).all()
    assert (wide[ws.numel():] == 7).all()


def test_binding_refuses_wrong_tensors(sp):
    s = problem(37, 64, [2, 2])
    sp.sp_draft_verify(**s)
    for bad in (dict(logits=s["logits"].half()), dict(logits=s["logits"].t()), dict(draft_logits=s["draft_logits"].bfloat16()),
                dict(draft=s["draft"].long()), dict(u=s["u"][:3]), dict(noise=s["noise"].double()), dict(noise=s["noise"][:1]),
                dict(temperature=s["temperature"].cpu()), dict(token=ints([[0, 0]])), dict(cu_rows=s["cu_rows"].long()), dict(cu_rows=None)):
        with pytest.raises(ValueError):
            sp.sp_draft_verify(**dict(s, **bad))
    for bad in (dict(max_rows=0), dict(max_rows=1025), dict(u=None), dict(draft=None),
                dict(ws=torch.empty(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(sp.SPError):
            sp.sp_draft_verify(**dict(s, **bad))
