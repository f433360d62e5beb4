"""Operators of generation over shared, paged prefixes, as cases that can be timed and compared.

Several sequences that continue one pruned image prefix (questions about an image, samples, beams) share
its keys and values: the cache lies in pages, and a sequence has a table of its pages.  The operators, in
the order a generation step uses them:

  append   rows q | k | v of a QKV projection: queries rotated, rotated keys and values put into pages
  attend   every row attends to the prefix of its group and, causally, to its sequence's own keys
  select   the best continuations of every element's beams over the vocabulary
  reorder  the beams' page tables permuted and the rows of their partly filled pages copied

The pool of one layer is [2][pages][page_size][n_kv_heads * head_dim] bf16 (keys, values); page tables are
int32, and the pages of a sequence lie scattered over the pool, as an allocator leaves them.  Head counts
are those of the package's workloads (32 heads of 128; 28 query heads on 4 key / value heads; 16 heads of
64); page sizes, batch sizes and lengths are generic."""
import math

import torch

own = False
DEV = "cuda"

# (query heads, key / value heads, head dim)
HEADS = {"llava": (32, 32, 128), "qwen": (28, 4, 128), "small": (16, 16, 64)}
SECTIONS = (16, 24, 24)  # rotation pairs of the (t, h, w) position components
MAX_POS = 32768
EOS = 2


# ----------------------------------------------------------------------------- cases

def listed():
    return [
        # One token each of the four beams of one image: the smallest append, where latency counts.
        _append("append four beams", "llava", 16, seqs=4, n=1, ctx=200),
        # One token each of a full batch, grouped heads, three position components.
        _append("append large step mrope", "qwen", 64, seqs=256, n=1, ctx=300, ragged=True, mrope=True),
        # The prompts of a batch entering the cache: the largest append.
        _append("append prompts", "llava", 16, seqs=16, n=700, ctx=0, ragged=True),
        # The four beams of one pruned image: the smallest attention call.
        _attend("attend four beams", "llava", 16, groups=1, per=4, prefix=240, ctx=20),
        # Four beams of each image of a batch of pruned images, images and answers of uneven length.
        _attend("attend beams of images", "llava", 16, groups=16, per=4, prefix=300, ctx=64, ragged=True),
        # Sixty-four answers in progress about one unpruned multi-tile image.
        _attend("attend many answers", "qwen", 32, groups=1, per=64, prefix=2944, ctx=128, ragged=True),
        # Sixteen questions of up to 48 tokens about one such image, all their rows at once.
        _attend("attend questions", "qwen", 64, groups=1, per=16, prefix=2944, ctx=48, n=48, ragged=True),
        # 128 samples over a long video prefix, each with a long answer of its own: the largest.
        _attend("attend long prefix", "qwen", 64, groups=1, per=128, prefix=16384, ctx=1024, ragged=True),
        # One image's four beams: the smallest selection, 32-bit logits.
        _select("select one image", elems=1, beams=4, vocab=32000, n_out=4, f32=True),
        # A batch of 64 with twice the beams asked for, a large vocabulary, 16-bit logits, some beams done.
        _select("select batch", elems=64, beams=4, vocab=152064, n_out=8, f32=False, done=True),
        # One image's four beams after a step: 32 layers, a partly filled page each.
        _reorder("reorder one image", "llava", 16, elems=1, beams=4, layers=32, ctx=23),
        # The beams of a batch, 28 layers, grouped heads.
        _reorder("reorder batch", "qwen", 32, elems=16, beams=4, layers=28, ctx=90),
    ]


def _named(name, c):
    return dict(c, name=name) if name else c


def _append(name, heads, page, *, seqs, n, ctx, ragged=False, mrope=False):
    return _named(name, {"kind": "append", "heads": heads, "page": page, "seqs": seqs, "n": n, "ctx": ctx,
                         "ragged": ragged, "mrope": mrope})


def _attend(name, heads, page, *, groups, per, prefix, ctx, n=1, ragged=False):
    """ctx: a sequence's own keys, those of its n rows of this call among them (at least n)."""
    return _named(name, {"kind": "attend", "heads": heads, "page": page, "groups": groups, "per": per,
                         "prefix": prefix, "ctx": max(ctx, n), "n": n, "ragged": ragged})


def _select(name, *, elems, beams, vocab, n_out, f32, done=False):
    return _named(name, {"kind": "select", "elems": elems, "beams": beams, "vocab": vocab, "n_out": n_out,
                         "f32": f32, "done": done})


def _reorder(name, heads, page, *, elems, beams, layers, ctx):
    return _named(name, {"kind": "reorder", "heads": heads, "page": page, "elems": elems, "beams": beams,
                         "layers": layers, "ctx": ctx})


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Bytes, with 280 operations (a matrix unit's in the time memory moves a byte) counted as one."""
    w = work(case)
    return max(w["bytes"], w["flops"] / 280)


def draw(rng):
    most = max(map(_cost, listed()))
    while True:
        case = _any(rng)
        if _cost(case) <= most:
            return case


def _any(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "select", "select", "reorder"])
    heads, page, odd = rng.choice(list(HEADS)), rng.choice([16, 32, 64]), rng.random() < 0.6
    if kind == "append":
        if rng.random() < 0.5:
            return _append("", heads, page, seqs=_log(rng, 1, 256), n=1, ctx=_log(rng, 1, 900), ragged=odd,
                           mrope=heads == "qwen" and rng.random() < 0.7)
        seqs = _log(rng, 1, 64)
        return _append("", heads, page, seqs=seqs, n=_log(rng, 2, 8192 // seqs), ctx=rng.choice([0, 0, 77]),
                       ragged=odd, mrope=heads == "qwen" and rng.random() < 0.7)
    if kind == "attend":
        shape = rng.choice(["beams", "answers", "questions", "alone"])
        if shape == "beams":
            groups = _log(rng, 1, 48)
            return _attend("", heads, page, groups=groups, per=rng.randint(1, 5), prefix=_log(rng, 16, 700),
                           ctx=_log(rng, 1, 200), ragged=odd)
        if shape == "answers":
            groups = rng.choice([1, 1, 2])
            return _attend("", heads, page, groups=groups, per=_log(rng, 6, 100), prefix=_log(rng, 300, 8000),
                           ctx=_log(rng, 1, 500), ragged=odd)
        if shape == "questions":
            groups = rng.choice([1, 1, 3])
            return _attend("", heads, page, groups=groups, per=_log(rng, 1, 12), prefix=_log(rng, 100, 3300),
                           ctx=_log(rng, 3, 80), n=_log(rng, 2, 48), ragged=odd)
        # sequences with no prefix in common: one to a group, and the prefix may be empty
        return _attend("", heads, page, groups=_log(rng, 1, 64), per=1, prefix=rng.choice([0, 5, 100]),
                       ctx=_log(rng, 1, 1500), ragged=odd)
    if kind == "select":
        beams = rng.choice([1, 2, 3, 4, 5, 8, 16])
        return _select("", elems=_log(rng, 1, 256 // beams), beams=beams, vocab=_log(rng, 500, 152064),
                       n_out=min(32, rng.choice([1, 2]) * beams), f32=rng.random() < 0.5, done=odd)
    beams = rng.choice([2, 3, 4, 5, 8])
    return _reorder("", heads, page, elems=_log(rng, 1, 64 // beams), beams=beams, layers=_log(rng, 1, 32 if heads != "llava" else 16),
                    ctx=_log(rng, 1, 200))


# ----------------------------------------------------------------------------- sizes (from the case alone)

def _spread(n, count, ragged, low=0.35):
    """Lengths of the sequences: all n, or spread over low * n .. n."""
    if not ragged:
        return [n] * count
    return [max(min(n, 1), int(n * (low + (1 - low) * ((0.618034 * (i + 1)) % 1.0)))) for i in range(count)]


def _ctx(case):
    """Cached positions of each sequence (append: before the call; attend: with the call's own rows)."""
    if case["kind"] == "append":
        return _spread(case["ctx"], case["seqs"], case["ragged"], low=0.1)
    n = _rows(case)
    return [max(a, b) for a, b in zip(_spread(case["ctx"], len(n), case["ragged"], low=0.05), n)]


def _rows(case):
    count = case["seqs"] if case["kind"] == "append" else case["groups"] * case["per"]
    return _spread(case["n"], count, case["ragged"] and case["n"] > 1)


def _prefixes(case):
    return _spread(case["prefix"], case["groups"], case["ragged"] and case["groups"] > 1)


def _parents(case):
    """Parent beam of every beam: some stay, some are copied, some end."""
    W = case["beams"]
    return [[w if (b + w) % 3 == 0 else (7 * b + 5 * w + w * w) % W for w in range(W)] for b in range(case["elems"])]


def _beam_ctx(case):
    return _spread(case["ctx"], case["elems"], case["elems"] > 1, low=0.5)


def work(case):
    if case["kind"] == "select":
        n = case["elems"] * case["beams"]
        live = n - (sum(1 for i in range(n) if _is_done(i)) if case["done"] else 0)
        return {"bytes": live * case["vocab"] * (4 if case["f32"] else 2) + 8 * n + 12 * case["elems"] * case["n_out"],
                "flops": 4 * live * case["vocab"]}
    Hq, Hkv, dh = HEADS[case["heads"]]
    if case["kind"] == "append":
        T = sum(_rows(case))
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * dh * 2, "flops": 6 * T * (Hq + Hkv) * dh // 2}
    if case["kind"] == "attend":
        n, ctx, pre, per = _rows(case), _ctx(case), _prefixes(case), case["per"]
        seen = sum(n[b] * pre[b // per] + n[b] * (ctx[b] - n[b]) + n[b] * (n[b] + 1) // 2 for b in range(len(n)))
        return {"bytes": 2 * sum(n) * Hq * dh * 2 + 2 * (sum(pre) + sum(ctx)) * Hkv * dh * 2, "flops": 4 * dh * Hq * seen}
    rows = sum((c % case["page"]) * sum(p != w for w, p in enumerate(ps)) for c, ps in zip(_beam_ctx(case), _parents(case)))
    pages = case["elems"] * case["beams"] * (case["ctx"] // case["page"] + 2)
    return {"bytes": 2 * rows * 2 * case["layers"] * Hkv * dh * 2 + 2 * 4 * pages, "flops": 0}


# ----------------------------------------------------------------------------- inputs (from the seed alone)

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(v):
    return _ints([sum(v[:i]) for i in range(len(v) + 1)])


def _normal(gen, *shape, std=1.0):
    """bf16 normals, filled in parts (a pool is large)."""
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    return x.normal_(0.0, std, generator=gen)


def _tables(counts, width, gen, extra=3):
    """Page tables (rows of `width`, -1 behind a row's pages) with every row's pages scattered over the pool."""
    total = sum(counts)
    ids = torch.randperm(total + extra, device=DEV, generator=gen)[:total].to(torch.int32)
    t = torch.full((len(counts), max(width, 1)), -1, dtype=torch.int32, device=DEV)
    at = torch.arange(max(width, 1), device=DEV)[None] < _ints(counts)[:, None]
    t[at] = ids
    return t, total + extra


def _rope_table(dh):
    """(cos, sin) of every position and rotation pair: angles in 64 bits, stored in 32."""
    inv = 10000.0 ** (-torch.arange(0, dh, 2, dtype=torch.float64, device=DEV) / dh)
    a = torch.arange(MAX_POS, dtype=torch.float64, device=DEV)[:, None] * inv
    return torch.stack((a.cos(), a.sin()), dim=-1).to(torch.float32)


def _is_done(i):
    return i % 5 == 3


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "select":
        E, W, V = case["elems"], case["beams"], case["vocab"]
        # log-probabilities of a language model: a broad bulk and a few likely tokens
        x = torch.randn((E, W, V), device=DEV, generator=gen).mul_(2.0)
        top = torch.randint(0, V, (E, W, 12), device=DEV, generator=gen)
        x.scatter_add_(2, top, 4.0 + 3.0 * torch.randn((E, W, 12), device=DEV, generator=gen).abs())
        s["logits"] = x if case["f32"] else x.to(torch.bfloat16)
        s["cum"] = -20.0 * torch.rand((E, W), device=DEV, generator=gen)
        s["done"] = None
        if case["done"]:
            s["done"] = torch.tensor([[_is_done(e * W + w) for w in range(W)] for e in range(E)], device=DEV)
        return s
    Hq, Hkv, dh = HEADS[case["heads"]]
    page = case["page"]
    need = lambda n: -(-n // page)  # noqa: E731
    s.update(Hq=Hq, Hkv=Hkv, dh=dh, page=page)
    if kind == "append":
        n, ctx = _rows(case), _ctx(case)
        T = sum(n)
        s["table"], pages = _tables([need(a + b) for a, b in zip(ctx, n)], max(need(a + b) for a, b in zip(ctx, n)), gen)
        s["kv"] = _normal(gen, 2, pages, page, Hkv * dh)
        s["qkv"] = _normal(gen, T, (Hq + 2 * Hkv) * dh)
        s["lens"] = _ints(ctx)
        s["cu_rows"] = None if case["n"] == 1 else _starts(n)
        at = torch.arange(T, device=DEV, dtype=torch.int32)
        seq = torch.repeat_interleave(torch.arange(len(n), device=DEV), torch.tensor(n, device=DEV), output_size=T)
        pos = s["lens"][seq] + at - _starts(n)[seq]
        s["pos"] = s["pos3"] = None
        if case["mrope"]:
            grid = torch.randint(0, 40, (T, 4), device=DEV, generator=gen, dtype=torch.int32)
            s["pos3"] = (pos[:, None] + grid).contiguous()
        else:
            s["pos"] = pos.contiguous()
        s["rope"] = _rope_table(dh)
        s["q_out"] = torch.empty((T, Hq * dh), dtype=torch.bfloat16, device=DEV)
    elif kind == "attend":
        n, ctx, pre, per = _rows(case), _ctx(case), _prefixes(case), case["per"]
        T, width, pwidth = sum(n), max(map(need, ctx)), max(map(need, pre))
        both, pages = _tables([need(c) for c in ctx] + [need(p) for p in pre], max(width, pwidth), gen)
        s["table"] = both[:len(ctx), :max(width, 1)].contiguous()
        s["prefix_table"] = both[len(ctx):, :max(pwidth, 1)].contiguous()
        s["kv"] = _normal(gen, 2, pages, page, Hkv * dh)
        s["q"] = _normal(gen, T, Hq * dh, std=1.5)
        s["lens"], s["prefix_lens"] = _ints(ctx), _ints(pre)
        s["group_cu"] = _ints([g * per for g in range(case["groups"] + 1)])
        s["cu_rows"] = None if case["n"] == 1 else _starts(n)
        s.update(max_ctx=max(ctx), max_prefix=max(pre), max_n=max(n), max_group=max(sum(n[g * per:(g + 1) * per]) for g in range(case["groups"])))
        s["out"] = torch.empty((T, Hq * dh), dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=DEV)
    else:
        ctx, W = _beam_ctx(case), case["beams"]
        counts = [c // page + 1 for c in ctx for _ in range(W)]
        s["own_table"], pages = _tables(counts, max(counts), gen)
        s["table"] = s["own_table"].clone()
        s["kv"] = _normal(gen, case["layers"], 2, pages, page, Hkv * dh)
        s["lens"] = _ints([c for c in ctx for _ in range(W)])
        s["parent"] = _ints(_parents(case))
    s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


# ----------------------------------------------------------------------------- plain forms

def _plain_append(s):
    Hq, Hkv, dh, page = s["Hq"], s["Hkv"], s["dh"], s["page"]
    T, B = s["qkv"].shape[0], s["table"].shape[0]
    at = torch.arange(T, device=DEV)
    cu = torch.arange(B + 1, device=DEV, dtype=torch.int32) if s["cu_rows"] is None else s["cu_rows"]
    seq = torch.searchsorted(cu[1:], at, right=True)
    slot = s["lens"][seq] + at - cu[seq]
    row = (s["table"][seq, slot // page] * page + slot % page).long()
    pairs = torch.arange(dh // 2, device=DEV)
    if s["pos3"] is not None:
        comp = (pairs >= SECTIONS[0]).long() + (pairs >= SECTIONS[0] + SECTIONS[1]).long()
        cs = s["rope"][s["pos3"][:, comp].long(), pairs]
    else:
        cs = s["rope"][s["pos"].long()]
    c, d = cs[:, None, :, 0], cs[:, None, :, 1]
    x = s["qkv"].view(T, Hq + 2 * Hkv, dh)
    a, b = x[:, :Hq + Hkv].float().chunk(2, dim=-1)
    y = torch.cat((a * c - b * d, b * c + a * d), dim=-1).to(torch.bfloat16)
    flat = s["kv"].view(2, -1, Hkv, dh)
    flat[0, row] = y[:, Hq:]
    flat[1, row] = x[:, Hq + Hkv:]
    s["q_out"].copy_(y[:, :Hq].reshape(T, Hq * dh))
    return {"q": s["q_out"], "kv": s["kv"]}


def _paged(s, table, count):
    """Keys and values [rows, count, heads, dim] in 32 bits of the first `count` positions of every table row."""
    k = torch.arange(count, device=DEV)
    row = (table[:, k // s["page"]].clamp(min=0) * s["page"] + k % s["page"]).long()
    return (x.view(-1, s["Hkv"], s["dh"])[row].float() for x in s["kv"])


def _part(s, rows, table, count, visible):
    """Softmax statistics and weighted values (m, l, o) of the rows [entries, n] of q over the first `count`
    positions of each entry's pages; visible [entries, n, count]."""
    Hq, Hkv, dh = s["Hq"], s["Hkv"], s["dh"]
    K, V = _paged(s, table, count)
    q = s["q"].view(-1, Hkv, Hq // Hkv, dh)[rows].float()
    z = torch.einsum("enhgd,ekhd->ehngk", q, K) * (1.0 / math.sqrt(dh))
    z = z.masked_fill(~visible[:, None, :, None], -math.inf)
    m = z.amax(dim=-1)
    p = torch.exp(z - torch.where(m == -math.inf, 0.0, m)[..., None])
    o = torch.einsum("ehngk,ekhd->ehngd", p, V)
    return tuple(x.transpose(1, 2).flatten(2, 3) for x in (m, p.sum(dim=-1), o))


def _plain_attend(s):
    T, B = s["q"].shape[0], s["table"].shape[0]
    at = torch.arange(T, device=DEV)
    cu = torch.arange(B + 1, device=DEV, dtype=torch.int32) if s["cu_rows"] is None else s["cu_rows"]
    seq = torch.searchsorted(cu[1:], at, right=True)
    group = torch.searchsorted(s["group_cu"][1:], seq, right=True)
    parts = []
    if s["max_prefix"] > 0:
        start = cu[s["group_cu"][:-1].long()]
        rows = (start[:, None] + torch.arange(s["max_group"], device=DEV)).clamp(max=T - 1)
        visible = torch.arange(s["max_prefix"], device=DEV) < s["prefix_lens"][:, None, None]
        part = _part(s, rows, s["prefix_table"], s["max_prefix"], visible.expand(-1, rows.shape[1], -1))
        parts.append([x[group, at - start[group]] for x in part])
    j = torch.arange(s["max_n"], device=DEV)
    rows = (cu[:-1, None] + j).clamp(max=T - 1)
    last = (s["lens"] - (cu[1:] - cu[:-1]))[:, None] + j
    visible = torch.arange(s["max_ctx"], device=DEV) <= last[..., None]
    part = _part(s, rows, s["table"], s["max_ctx"], visible)
    parts.append([x[seq, at - cu[seq]] for x in part])
    m, l, o = (torch.stack(x) for x in zip(*parts))
    top = m.amax(dim=0)
    f = torch.exp(m - torch.where(top == -math.inf, 0.0, top))
    l = (f * l).sum(dim=0)
    o = (f[..., None] * o).sum(dim=0) / torch.where(l == 0, 1.0, l)[..., None]
    return {"out": o.reshape(T, -1).to(torch.bfloat16), "lse": top + torch.log(l)}


def _plain_select(s):
    """Scores in 64 bits: neighbours of different beams differ by less than 32 bits tell apart."""
    E, W, V = s["logits"].shape
    K = s["case"]["n_out"]
    score = s["cum"].double()[..., None] + torch.log_softmax(s["logits"].double(), dim=-1)
    if s["done"] is not None:
        kept = torch.where(torch.arange(V, device=DEV) == EOS, s["cum"].double()[..., None], -math.inf)
        score = torch.where(s["done"][..., None], kept, score)
    score = score.view(E, W * V)
    least = torch.topk(score, K, dim=-1).values[:, -1:]
    # the K best, of equal ones the first: those above the least in any place, then the least's first places
    at = torch.arange(W * V, device=DEV)
    place = torch.where(score > least, at, torch.where(score == least, at + W * V, 2 * W * V))
    place = torch.topk(place, K, dim=-1, largest=False).values % (W * V)
    place = place.sort(dim=-1).values
    best = score.gather(1, place)
    best, order = best.sort(dim=-1, descending=True, stable=True)
    place = place.gather(1, order)
    return {"score": best.float(), "parent": (place // V).int(), "token": (place % V).int()}


def _plain_reorder(s):
    W, page = s["case"]["beams"], s["page"]
    E = s["parent"].shape[0]
    old = (s["parent"] + torch.arange(0, E * W, W, device=DEV, dtype=torch.int32)[:, None]).view(-1).long()
    full = (s["lens"] // page).long()
    column = torch.arange(s["table"].shape[1], device=DEV)
    table = torch.where(column < full[:, None], s["table"][old], s["own_table"])
    mine = s["own_table"].gather(1, full[:, None])[:, 0].long()
    rows = torch.arange(page, device=DEV) < (s["lens"] % page)[:, None]
    there = s["kv"][:, :, mine[old]]
    here = s["kv"][:, :, mine]
    s["kv"][:, :, mine] = torch.where(rows[..., None], there, here)
    s["table"].copy_(table)
    return {"kv": s["kv"], "table": s["table"]}


_PLAIN = {"append": _plain_append, "attend": _plain_attend, "select": _plain_select, "reorder": _plain_reorder}


# ----------------------------------------------------------------------------- the framework's calls

def _own(s):
    from paper_2609_13804_gb300 import binding as sp
    kind = s["case"]["kind"]
    if kind == "append":
        sp.sp_paged_append(qkv=s["qkv"], kv=s["kv"], table=s["table"], lens=s["lens"], cu_rows=s["cu_rows"],
                           n_heads=s["Hq"], n_kv_heads=s["Hkv"], head_dim=s["dh"], rope=s["rope"], pos=s["pos"],
                           pos3=s["pos3"], mrope_section=SECTIONS if s["pos3"] is not None else None,
                           q_out=s["q_out"], err=s["err"])
        return {"q": s["q_out"], "kv": s["kv"]}
    if kind == "attend":
        if "ws" not in s:  # kept from call to call, as a program that generates keeps it
            s["ws"] = sp.prefix_attention_workspace(T_cap=s["q"].shape[0], B=s["table"].shape[0], n_heads=s["Hq"],
                                                    n_kv_heads=s["Hkv"], head_dim=s["dh"],
                                                    n_groups=s["prefix_table"].shape[0], device=DEV)
        r = sp.sp_prefix_attention(q=s["q"], kv=s["kv"], table=s["table"], lens=s["lens"], cu_rows=s["cu_rows"],
                                   prefix_table=s["prefix_table"], prefix_lens=s["prefix_lens"],
                                   group_cu=s["group_cu"], n_heads=s["Hq"], n_kv_heads=s["Hkv"], head_dim=s["dh"],
                                   out=s["out"], lse=s["lse"], ws=s["ws"], err=s["err"])
        return {"out": r["out"], "lse": r["lse"]}
    if kind == "select":
        if "ws" not in s:
            s["ws"] = sp.beam_select_workspace(B=s["logits"].shape[0], W=s["logits"].shape[1], V=s["logits"].shape[2],
                                               n_out=s["case"]["n_out"], device=DEV)
        r = sp.sp_beam_select(logits=s["logits"], cum=s["cum"], n_out=s["case"]["n_out"], done=s["done"], eos=EOS,
                              ws=s["ws"])
        return {"score": r["score"], "parent": r["parent"], "token": r["token"]}
    sp.sp_beam_reorder(kv=s["kv"], table=s["table"], own_table=s["own_table"], lens=s["lens"], parent=s["parent"],
                       err=s["err"])
    return {"kv": s["kv"], "table": s["table"]}


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["kind"]](state)


# ----------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_append(s):
    """Every row by itself: rotation by an angle as a complex product."""
    Hq, Hkv, dh, page = s["Hq"], s["Hkv"], s["dh"], s["page"]
    T, half = s["qkv"].shape[0], dh // 2
    n, ctx = _rows(s["case"]), _ctx(s["case"])
    freq = torch.exp(torch.arange(half, dtype=torch.float64, device=DEV) * (-2.0 * math.log(10000.0) / dh))
    if s["pos3"] is None:
        where = s["pos"].double()[:, None].expand(T, half)
    else:
        where = torch.cat([s["pos3"][:, c:c + 1].double().expand(T, k) for c, k in enumerate(SECTIONS)], dim=1)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), where * freq)[:, None]
    x = s["qkv"].double().view(T, -1, dh)
    z = torch.complex(x[..., :half], x[..., half:])[:, :Hq + Hkv] * turn
    rotated = torch.cat((z.real, z.imag), dim=-1)
    kv, r, table = s["kv"].double(), 0, s["table"].tolist()
    for b, (rows, before) in enumerate(zip(n, ctx)):
        done = 0
        while done < rows:  # the rows that share a page
            p = before + done
            take = min(rows - done, page - p % page)
            at, to = slice(r + done, r + done + take), slice(p % page, p % page + take)
            kv[0, table[b][p // page], to] = rotated[at, Hq:].reshape(take, -1)
            kv[1, table[b][p // page], to] = x[at, Hq + Hkv:].reshape(take, -1)
            done += take
        r += rows
    return {"q": rotated[:, :Hq].reshape(T, -1), "kv": kv}


def _exact_attend(s):
    """Sequence by sequence over the concatenated keys."""
    Hq, Hkv, dh, page = s["Hq"], s["Hkv"], s["dh"], s["page"]
    n, ctx, pre, per = _rows(s["case"]), _ctx(s["case"]), _prefixes(s["case"]), s["case"]["per"]
    out, lse, r = [], [], 0
    keys = lambda t, c: s["kv"][:, t[:-(-c // page)].long()].flatten(1, 2)[:, :c]  # noqa: E731
    for b in range(len(n)):
        g = b // per
        k, v = torch.cat((keys(s["prefix_table"][g], pre[g]), keys(s["table"][b], ctx[b])), dim=1).double().view(2, -1, Hkv, dh)
        q = s["q"][r:r + n[b]].double().view(n[b], Hkv, Hq // Hkv, dh)
        z = torch.matmul(q.permute(1, 2, 0, 3), k.permute(1, 2, 0)[:, None]) / math.sqrt(dh)
        late = torch.arange(k.shape[0], device=DEV)[None] > pre[g] + ctx[b] - n[b] + torch.arange(n[b], device=DEV)[:, None]
        z[:, :, late] = -math.inf
        w = torch.softmax(z, dim=-1)
        out.append(torch.matmul(w, v.permute(1, 0, 2)[:, None]).permute(2, 0, 1, 3).reshape(n[b], -1))
        lse.append(torch.logsumexp(z, dim=-1).permute(2, 0, 1).reshape(n[b], -1))
        r += n[b]
    return {"out": torch.cat(out), "lse": torch.cat(lse)}


def _exact_select(s):
    E, W, V = s["logits"].shape
    K, out = s["case"]["n_out"], []
    for e in range(E):
        x = s["logits"][e].double()
        p = s["cum"][e].double()[:, None] + x - torch.logsumexp(x, dim=1, keepdim=True)
        if s["done"] is not None:
            for w in s["done"][e].nonzero()[:, 0].tolist():
                p[w] = -math.inf
                p[w, EOS] = s["cum"][e, w].double()
        best, place = p.view(-1).sort(descending=True, stable=True)
        out.append((best[:K], place[:K]))
    score, place = (torch.stack(x) for x in zip(*out))
    return {"score": score, "parent": place // V, "token": place % V}


def exact(case, seed):
    if case["kind"] == "reorder":  # nothing is computed, only moved
        return None
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "select": _exact_select}[case["kind"]](s)
