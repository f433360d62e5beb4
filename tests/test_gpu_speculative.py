"""Speculative generation over shared pages, its operators as a program uses them: samples fork a prompt or a pruned copy of
it, and every step reserves room, appends the last token and the drafts, attends, verifies and trims."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"

from test_gpu_paged import U, single_precision  # noqa: E402, F401
from test_gpu_verify import compare, gen, ints, reference  # noqa: E402

HQ, HKV, DH, PAGE, V, K = 8, 2, 64, 16, 303, 4


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_13804_gb300 import binding
    return binding


@pytest.mark.parametrize("pruned", [False, True])
def test_generation_with_drafts(sp, pruned):
    """Two prompts, three sequences of each (greedy ones among them); logits against attention in 64 bits, decisions against
    the rule, the cache against every sequence's own history, the prompts untouched, no page lost."""
    g = gen(41 + pruned)
    rand = lambda *s, std=1.0: (torch.randn(s, device=DEV, generator=g) * std).bfloat16()  # noqa: E731
    embed, wqkv, wout = rand(V, 128), rand(128, (HQ + 2 * HKV) * DH, std=0.15), rand(HQ * DH, V, std=0.25)
    bigram = rand(V, V, std=2.0)  # the draft model
    P, per = 2, 3
    S = P + P * per
    n0, mp = [37, 16], 8
    n_pages = S * mp
    kv = sp.paged_pool(n_pages, PAGE, HKV, DH)
    table = torch.full((S, mp), -1, dtype=torch.int32, device=DEV)
    lens, refs = ints([0] * S), ints([0] * n_pages)
    books = dict(table=table, lens=lens, refs=refs)
    rope = sp.rope_table(256, DH)
    heads = dict(n_heads=HQ, n_kv_heads=HKV, head_dim=DH)
    ws, err = sp.pages_workspace(S=S, max_pages=mp), ints([0])
    keys = lambda s: kv[0, :, [int(table[s, i // PAGE]) for i in range(int(lens[s]))], [i % PAGE for i in range(int(lens[s]))]]  # noqa: E731

    # the prompts
    sp.sp_pages_reserve(kv=kv, add=ints(n0 + [0] * (S - P)), ws=ws, err=err, **books)
    prompt = torch.randint(0, V, (sum(n0),), device=DEV, generator=g)
    cu = ints([0, n0[0]] + [sum(n0)] * (S - 1))
    pos = ints([i for n in n0 for i in range(n)])
    sp.sp_paged_append(qkv=embed[prompt] @ wqkv, kv=kv[0], table=table, lens=lens, cu_rows=cu, rope=rope, pos=pos, keys_only=True,
                       err=err, **heads)
    lens += ints(n0 + [0] * (S - P))
    parent = ints([-1] * P + [p for p in range(P) for _ in range(per)])
    sp.sp_pages_fork(page_size=PAGE, parent=parent, err=err, **books)
    hist = [keys(s).clone() for s in range(S)]
    if pruned:  # every sequence has positions of its own choice left
        kept = [None] * P + [sorted(torch.randperm(n0[p], device=DEV, generator=g)[:9 + s].tolist()) for p in range(P) for s in range(per)]
        keep = torch.zeros((S, 9 + per), dtype=torch.int32, device=DEV)
        for s, k in enumerate(kept):
            if k:
                keep[s, :len(k)] = ints(k)
                hist[s] = hist[s][:, k]
        sp.sp_pages_compact(kv=kv, keep=keep, count=ints([-1 if k is None else len(k) for k in kept]), ws=ws, err=err, **books)
    told = [keys(p).clone() for p in range(P)]
    at = ints([0] * P + [n0[p] for p in range(P) for _ in range(per)])  # the rotary position of a sequence's next token
    last = torch.randint(0, V, (S,), device=DEV, generator=g)
    live = torch.arange(S, device=DEV) >= P
    temperature = torch.tensor([1.0, 0.7, 0.0] * S, device=DEV)[:S].contiguous()
    emitted = 0
    for step in range(4):
        k = [0] * P + [(step + s) % (K + 1) for s in range(S - P)]  # drafts of each
        rows = [0] * P + [x + 1 for x in k[P:]]
        cu = ints([sum(rows[:s]) for s in range(S + 1)])
        T = sum(rows)
        sp.sp_pages_reserve(kv=kv, add=ints(rows), ws=ws, err=err, **books)
        # the draft model's tokens, each drawn from its logits
        tokens, logits_q, draft = [], torch.zeros((T, V), device=DEV, dtype=torch.bfloat16), torch.zeros(T, dtype=torch.int32, device=DEV)
        r = 0
        for s in range(S):
            t = last[s]
            for j in range(rows[s]):
                tokens.append(int(t))
                if j < k[s]:
                    logits_q[r] = bigram[t]
                    z = bigram[t].double() / max(float(temperature[s]), 1e-3)
                    t = torch.multinomial(torch.softmax(z, 0), 1, generator=g)[0]
                    draft[r] = int(t)
                r += 1
        x = embed[torch.tensor(tokens, device=DEV)]
        pos = torch.cat([at[s] + torch.arange(rows[s], device=DEV) for s in range(S)]).int()
        a = sp.sp_paged_append(qkv=x @ wqkv, kv=kv[0], table=table, lens=lens, cu_rows=cu, rope=rope, pos=pos, err=err, **heads)
        before = lens.clone()
        lens += ints(rows)
        o = sp.sp_prefix_attention(q=a["q"], kv=kv[0], table=table, lens=lens, cu_rows=cu, err=err, **heads)
        r = 0
        for s in range(P, S):
            hist[s] = torch.cat((hist[s], keys(s)[:, int(before[s]):]), dim=1)
            assert torch.equal(keys(s), hist[s])
            for j in range(rows[s]):
                n = int(before[s]) + j + 1
                h = hist[s][:, :n].double().view(2, n, HKV, DH)
                z = torch.einsum("hgd,khd->hgk", a["q"][r].double().view(HKV, HQ // HKV, DH), h[0]) * DH ** -0.5
                w = torch.softmax(z, dim=-1)
                want, size = (torch.einsum("hgk,khd->hgd", w, v).reshape(-1) for v in (h[1], h[1].abs()))
                assert ((o["out"][r].double() - want).abs() <= U * want.abs() + (U + 2.0 ** -12) * size).all(), (step, s, j)
                r += 1
        logits = o["out"] @ wout
        u = torch.rand(T, device=DEV, generator=g)
        u[::2] = 0.0  # these stay wherever the target gives them any weight
        noise = torch.empty((S, V), device=DEV).exponential_(generator=g)
        v = sp.sp_draft_verify(logits=logits, draft_logits=logits_q, draft=draft, u=u, noise=noise, temperature=temperature,
                               cu_rows=cu, max_rows=K + 1, err=err)
        want, r = [], 0
        X, Y, D, UU, E = (t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy() for t in (logits, logits_q, draft, u, noise))
        for s in range(S):
            n = rows[s]
            want.append(reference(X[r:r + n], D[r:r + n - 1], Y[r:r + n - 1], UU[r:r + n - 1], E[s], float(temperature[s])) if n else (-1, [], [], True))
            r += n
        compare(v, want, K + 1)
        got = v["n_accept"] + 1  # positions that stay: the last token's and the accepted drafts'
        assert got[:P].tolist() == [0] * P
        lens.copy_(before + got)
        at += got
        sp.sp_pages_trim(page_size=PAGE, err=err, **books)
        last = torch.where(live, v["token"].gather(1, v["n_accept"].clamp(min=0).long()[:, None])[:, 0].long(), last)
        for s in range(P, S):
            hist[s] = hist[s][:, :int(lens[s])]
        emitted += int(got.sum())
    assert int(err.item()) == 0
    assert emitted > 4 * (S - P)
    assert all(torch.equal(keys(p), told[p]) for p in range(P))  # the prompts are as they were
    named = torch.bincount(table[table >= 0].long(), minlength=n_pages)
    assert torch.equal(named.int(), refs)
    lens.zero_()
    sp.sp_pages_trim(page_size=PAGE, err=err, **books)
    assert int(refs.abs().sum()) == 0
