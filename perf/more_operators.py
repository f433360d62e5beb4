"""Operators of speculative generation over a paged cache, as cases that can be timed and compared.

Sequences generate over pages of a pool that tables of theirs name.  A step puts drafted tokens behind a
sequence, the target model scores them all at once, and the operators here decide and keep the books:

  verify   which drafted tokens stay, and the token after them, from the target's and the draft's logits
           and given random numbers (without drafts: a token is sampled for every sequence)
  reserve  pages for the positions that a step will write; pages that others share are copied first
  trim     pages behind a sequence's end given back (a rejected draft's, an ended sequence's)
  fork     sequences that continue another one, sharing its pages
  compact  a sequence cut down to the positions that a selection keeps

The pool of all layers is [layers][2][pages][page_size][n_kv_heads * head_dim] bf16 (keys, values); a table
row names a sequence's pages (-1 behind them), and refs counts for every page the table entries that name it
(0: free).  Fresh pages are the free ones of the lowest numbers.  Head counts are those of the package's
workloads; page sizes, batch sizes, lengths and vocabularies are generic."""
import math

import torch

own = False
DEV = "cuda"

# width of a position's keys (or values): key / value heads times head dim
WIDTHS = {"llava": 32 * 128, "qwen": 4 * 128, "small": 16 * 64}


# ----------------------------------------------------------------------------- cases

def listed():
    return [
        # One question with four drafted tokens, 32-bit logits: the smallest step, where latency counts.
        _verify("verify one question", B=1, k=4, vocab=32000, f32=True),
        # No drafts: the next token of every sequence of a batch, sampled from its logits.
        _verify("verify no drafts", B=64, k=0, vocab=32000, f32=True),
        # A batch whose sequences have up to four drafts from a small model, large vocabulary, 16-bit logits.
        _verify("verify batch", B=64, k=4, vocab=152064, f32=False, ragged=True),
        # Drafts looked up in the prompt (no draft distribution), some sequences decoded greedily.
        _verify("verify looked up", B=32, k=7, vocab=152064, f32=False, model=False, greedy=True),
        # A full batch with five drafts each: the largest.
        _verify("verify large batch", B=256, k=5, vocab=152064, f32=False),
        # A speculative step of a batch: the last step's rejected pages go back, four drafts and a token get room.
        _reserve("reserve drafts", "qwen", 16, seqs=64, ctx=900, add=5, spare=1024),
        # Half of a batch's slots take in new prompts of up to 2,900 positions, in a large pool.
        _reserve("reserve prompts", "qwen", 16, seqs=256, ctx=1500, add=2944, spare=4096, admit=True),
        # Eight samples of one prompt: pages shared, the partly filled one copied on the first write.
        _fork("fork samples", "llava", 16, prompts=1, per=8, ctx=700, layers=32),
        # Four sequences of each prompt of a batch, uneven lengths, grouped heads.
        _fork("fork batch", "qwen", 32, prompts=32, per=4, ctx=600, layers=28, ragged=True),
        # One question keeps a tenth of an image's tokens and all of its text.
        _compact("compact one question", "llava", 16, prompts=1, per=1, vis=576, text=60, kept=58, layers=32),
        # Sixteen questions about one unpruned multi-tile image, each with tokens of its own choice.
        _compact("compact questions", "qwen", 32, prompts=1, per=16, vis=2880, text=64, kept=288, layers=28),
        # Eight questions about a long video prefix.
        _compact("compact video", "qwen", 64, prompts=1, per=8, vis=16384, text=100, kept=1638, layers=28),
    ]


def _named(name, c):
    return dict(c, name=name) if name else c


def _verify(name, *, B, k, vocab, f32, ragged=False, model=True, greedy=False, masked=False, pad=0):
    """k drafts at most; model: the drafts have a distribution; pad: elements between the rows."""
    return _named(name, {"kind": "verify", "B": B, "k": k, "vocab": vocab, "f32": f32, "ragged": ragged,
                         "model": model and k > 0, "greedy": greedy, "masked": masked, "pad": pad})


def _reserve(name, heads, page, *, seqs, ctx, add, spare, admit=False):
    """spare: free pages besides those that the call takes; admit: every other slot is empty and takes a prompt."""
    return _named(name, {"kind": "reserve", "heads": heads, "page": page, "seqs": seqs, "ctx": ctx, "add": add,
                         "spare": spare, "admit": admit})


def _fork(name, heads, page, *, prompts, per, ctx, layers, ragged=False):
    return _named(name, {"kind": "fork", "heads": heads, "page": page, "prompts": prompts, "per": per, "ctx": ctx,
                         "layers": layers, "ragged": ragged})


def _compact(name, heads, page, *, prompts, per, vis, text, kept, layers, ragged=False):
    """Sequences of vis visual and text positions behind them; kept of the visual ones and the text stay."""
    return _named(name, {"kind": "compact", "heads": heads, "page": page, "prompts": prompts, "per": per, "vis": vis,
                         "text": text, "kept": kept, "layers": layers, "ragged": ragged})


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    return work(case)["bytes"]


def _pool_bytes(case):
    if case["kind"] == "verify":
        return 0
    lens = _lens(case)
    pages = sum(-(-n // case["page"]) for n in lens) + _spare(case)
    return pages * case["page"] * WIDTHS[case["heads"]] * 4 * case.get("layers", 1)


def draw(rng):
    most = max(map(_cost, listed()))
    while True:
        case = _any(rng)
        if _cost(case) <= most and _pool_bytes(case) <= 4 << 30:
            return case


def _any(rng):
    kind = rng.choice(["verify"] * 4 + ["reserve", "fork", "compact", "compact"])
    heads, page, odd = rng.choice(list(WIDTHS)), rng.choice([16, 32, 64]), rng.random() < 0.6
    if kind == "verify":
        k = rng.choice([0, 1, 2, 3, 4, 5, 8])
        return _verify("", B=_log(rng, 1, 256), k=k, vocab=_log(rng, 500, 152064), f32=rng.random() < 0.4, ragged=odd,
                       model=rng.random() < 0.7, greedy=rng.random() < 0.4, masked=rng.random() < 0.3,
                       pad=rng.choice([0, 0, 1, 8, 36]))
    if kind == "reserve":
        admit = rng.random() < 0.4
        return _reserve("", "qwen", page, seqs=_log(rng, 1, 512), ctx=_log(rng, 1, 1500),
                        add=_log(rng, 20, 2000) if admit else rng.randint(1, 12), spare=_log(rng, 1, 8000), admit=admit)
    if kind == "fork":
        return _fork("", heads, page, prompts=_log(rng, 1, 48), per=rng.randint(1, 8), ctx=_log(rng, 1, 1500),
                     layers=_log(rng, 1, 32), ragged=odd)
    vis = _log(rng, 16, 6000)
    return _compact("", heads, page, prompts=_log(rng, 1, 4), per=_log(rng, 1, 16), vis=vis, text=_log(rng, 1, 120),
                    kept=_log(rng, 1, vis), layers=_log(rng, 1, 32), ragged=odd)


# ----------------------------------------------------------------------------- sizes (from the case alone)

def _spread(n, count, ragged, low=0.35):
    """Lengths of the sequences: all n, or spread over low * n .. n."""
    if not ragged:
        return [n] * count
    return [max(min(n, 1), int(n * (low + (1 - low) * ((0.618034 * (i + 1)) % 1.0)))) for i in range(count)]


def _drafts(case):
    """Drafted tokens of every sequence (with ragged ones some have none)."""
    if not case["ragged"]:
        return [case["k"]] * case["B"]
    return [(5 * b + b // 3 + 2) % (case["k"] + 1) for b in range(case["B"])]


def _lens(case):
    """Cached positions of every slot before the call (fork, compact: the prompts, then the empty children)."""
    if case["kind"] == "reserve":
        lens = _spread(case["ctx"], case["seqs"], True)
        return [0 if case["admit"] and b % 2 else n for b, n in enumerate(lens)]
    own_len = case["ctx"] if case["kind"] == "fork" else case["vis"] + case["text"]
    return _spread(own_len, case["prompts"], case["ragged"]) + [0] * (case["prompts"] * case["per"])


def _adds(case):
    if not case["admit"]:
        return [case["add"]] * case["seqs"]
    adds = _spread(case["add"], case["seqs"], True, low=0.1)
    return [n if b % 2 else 1 for b, n in enumerate(adds)]


def _spare(case):
    """Free pages of the pool before the call."""
    page = case["page"]
    if case["kind"] == "reserve":
        return case["spare"] + sum(-(-(n + a) // page) + 1 - n // page for n, a in zip(_lens(case), _adds(case)))
    n = case["prompts"] * case["per"]
    if case["kind"] == "fork":
        return 2 * n + 5
    return n * (-(-(case["kept"] + case["text"]) // page) + 1) + 5


def _kept(case, n):
    """How many of a prompt's n positions stay, and how many of those are its text."""
    text = min(case["text"], n)
    return min(case["kept"], n - text) + text, text


def work(case):
    if case["kind"] == "verify":
        drafts = _drafts(case)
        rows, sampled = sum(d + 1 for d in drafts), sum(1 for b in range(case["B"]) if not _is_greedy(case, b))
        scored = sum(d for b, d in enumerate(drafts) if not _is_greedy(case, b)) if case["model"] else 0
        logits = (rows + scored) * case["vocab"]
        return {"bytes": logits * (4 if case["f32"] else 2) + sampled * case["vocab"] * 4 + 20 * rows,
                "flops": 4 * logits + 6 * sampled * case["vocab"]}
    page, row = case["page"], WIDTHS[case["heads"]] * 2 * 2 * case.get("layers", 1)  # a position's keys and values
    lens = _lens(case)
    if case["kind"] == "reserve":
        taken = sum(-(-(n + a) // page) - -(-n // page) for n, a in zip(lens, _adds(case)))
        return {"bytes": 8 * len(lens) + 2 * taken * 16, "flops": 0}
    parents = lens[:case["prompts"]]
    if case["kind"] == "fork":
        shared = sum(-(-n // page) for n in parents) * case["per"]
        return {"bytes": 2 * row * case["per"] * sum(n % page for n in parents) + 24 * shared, "flops": 0}
    moved = sum(_kept(case, n)[0] for n in parents) * case["per"]
    return {"bytes": 2 * row * moved + 4 * moved + 24 * sum(-(-n // page) for n in parents) * case["per"], "flops": 0}


# ----------------------------------------------------------------------------- inputs (from the seed alone)

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _is_greedy(case, b):
    return case["greedy"] and b % 3 == 1


def _rows_of(x, pad):
    """The rows of x, `pad` elements between them."""
    if not pad:
        return x
    y = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=x.device)
    y[:, :x.shape[1]] = x
    return y[:, :x.shape[1]]


def _prepare_verify(case, gen, s):
    B, V, drafts = case["B"], case["vocab"], _drafts(case)
    T = sum(drafts) + B
    # log-probabilities of a language model: a broad bulk and a few likely tokens
    x = torch.randn((T, V), device=DEV, generator=gen).mul_(2.0)
    top = torch.randint(0, V, (T, 12), device=DEV, generator=gen)
    x.scatter_add_(1, top, 4.0 + 3.0 * torch.randn((T, 12), device=DEV, generator=gen).abs())
    if case["masked"]:  # a sampler's filter has left the likely tokens only
        x.masked_fill_(x < x.topk(min(60, V), dim=1).values[:, -1:], -math.inf)
    dtype = torch.float32 if case["f32"] else torch.bfloat16
    s["logits"] = _rows_of(x.to(dtype), case["pad"])
    s["cu_rows"] = None if case["k"] == 0 else _ints([sum(drafts[:b]) + b for b in range(B + 1)])
    s["draft"] = s["draft_logits"] = s["u"] = None
    if case["k"] > 0:
        if case["model"]:  # a smaller model's, close to the target's; it drew its tokens from them
            y = x.add(torch.randn((T, V), device=DEV, generator=gen), alpha=0.7)
            s["draft_logits"] = _rows_of(y.to(dtype), case["pad"])
            race = torch.empty((T, V), device=DEV).exponential_(generator=gen)
            s["draft"] = (y - race.log_()).argmax(dim=1).int()
            del y, race
        else:
            hit = torch.rand(T, device=DEV, generator=gen) < 0.6
            s["draft"] = torch.where(hit, x.argmax(dim=1), torch.randint(0, V, (T,), device=DEV, generator=gen)).int()
        s["u"] = torch.rand(T, device=DEV, generator=gen)
    s["noise"] = torch.empty((B, V), device=DEV).exponential_(generator=gen)
    s["temperature"] = torch.tensor([0.0 if _is_greedy(case, b) else (1.0, 0.7, 1.3)[b % 3] for b in range(B)], device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "verify":
        _prepare_verify(case, gen, s)
        return s
    page, lens = case["page"], _lens(case)
    S, spare = len(lens), _spare(case)
    held = [-(-n // page) for n in lens]
    if case["kind"] == "reserve":
        # pages that the last step's drafts took and lost (empty slots have none)
        want = [n + a for n, a in zip(lens, _adds(case))]
        held = [max(h, -(-(n + case["add"]) // page)) if n and not case["admit"] else h for h, n in zip(held, lens)]
    else:
        want = lens[:case["prompts"]] + [n + 1 for n in lens[:case["prompts"]] for _ in range(case["per"])]
    pages = sum(-(-n // page) for n in lens) + spare
    ids = torch.randperm(pages, device=DEV, generator=gen)[:sum(held)].to(torch.int32)
    width = max(max(-(-n // page) for n in want), max(held)) + 2
    s["table"] = torch.full((S, width), -1, dtype=torch.int32, device=DEV)
    s["table"][torch.arange(width, device=DEV) < _ints(held)[:, None]] = ids
    s["refs"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
    s["refs"][ids.long()] = 1
    s["lens"] = _ints(lens)
    s["kv"] = torch.empty((case.get("layers", 1), 2, pages, page, WIDTHS[case["heads"]]), dtype=torch.bfloat16, device=DEV)
    s["kv"].normal_(0.0, 1.0, generator=gen)
    P, per = case.get("prompts", 0), case.get("per", 0)
    s["parent"] = _ints([-1] * P + [p for p in range(P) for _ in range(per)])
    if case["kind"] == "reserve":
        s["add"] = _ints(_adds(case))
    elif case["kind"] == "fork":
        s["add"] = _ints([0] * P + [1] * (P * per))
    else:
        count = [_kept(case, n) for n in lens[:P] for _ in range(per)]
        most = max(c for c, _ in count)
        s["keep"] = torch.full((S, most), -1, dtype=torch.int32, device=DEV)
        for i, (c, text) in enumerate(count):  # in native order, the text behind the visual ones
            n = lens[i // per]
            vis = torch.randperm(n - text, device=DEV, generator=gen)[:c - text].sort().values
            s["keep"][P + i, :c] = torch.cat((vis, torch.arange(n - text, n, device=DEV))).int()
        s["count"] = _ints([-1] * P + [c for c, _ in count])
    s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


# ----------------------------------------------------------------------------- plain forms

def _first(x):
    """The place of each row's largest value, of equal ones the first."""
    at = torch.arange(x.shape[1], device=DEV)
    return torch.where(x == x.amax(dim=1, keepdim=True), at, x.shape[1]).amin(dim=1)


def _softmax(x, temperature):
    """Probabilities in 64 bits: accepting compares two of them, and where p and q are close their difference is
    what is left of them."""
    z = x.double() / temperature.double()[:, None]
    z = torch.exp(z - z.amax(dim=1, keepdim=True))
    return z / z.sum(dim=1, keepdim=True)


def _plain_verify(s):
    B, (T, V) = s["noise"].shape[0], s["logits"].shape
    cu = torch.arange(B + 1, device=DEV) if s["cu_rows"] is None else s["cu_rows"].long()
    most = s["case"]["k"] + 1
    row = torch.arange(T, device=DEV)
    seq = torch.searchsorted(cu[1:], row, right=True)
    greedy = s["temperature"] <= 0
    t = torch.where(greedy, 1.0, s["temperature"])[seq]
    p = _softmax(s["logits"], t)
    best = _first(s["logits"])
    last = row == cu[1:][seq] - 1
    q = None
    if s["draft"] is not None:
        d = s["draft"].long()
        pd = p.gather(1, d[:, None])[:, 0]
        if s["draft_logits"] is not None:
            q = _softmax(s["draft_logits"], t)
            accept = s["u"].double() * q.gather(1, d[:, None])[:, 0] < pd
        else:
            accept = s["u"].double() < pd
        accept = torch.where(greedy[seq], d == best, accept) & ~last
    else:
        accept = torch.zeros(T, dtype=torch.bool, device=DEV)
    # the first row of every sequence that accepts nothing (its last row at the latest)
    stop = torch.full((B,), T, device=DEV).scatter_reduce_(0, seq, torch.where(accept, T, row), "amin")
    n = stop - cu[:-1]
    r = p[stop]
    if q is not None:
        rest = (r - q[stop]).clamp_(min=0.0)
        r = torch.where((last[stop] | (rest.sum(dim=1) == 0))[:, None], r, rest)
    elif s["draft"] is not None:
        drafted = torch.arange(V, device=DEV) == d[stop][:, None]
        r = r.masked_fill(drafted & ~last[stop][:, None], 0.0)
    nxt = torch.where(greedy, best[stop], _first(r / s["noise"].double()))
    place = torch.arange(most, device=DEV)
    rows = (cu[:-1, None] + place).clamp(max=T - 1)
    token = nxt[:, None] if s["draft"] is None else torch.where(place == n[:, None], nxt[:, None], s["draft"].long()[rows])
    out = place <= n[:, None]
    token = torch.where(out, token, -1)
    logp = torch.log(p[rows, token.clamp(min=0)])
    return {"n_accept": n.int(), "token": token.int(), "logp": torch.where(out, logp, 0.0).float()}


def _plain_trim(s):
    behind = torch.arange(s["table"].shape[1], device=DEV) >= (s["lens"][:, None] + s["case"]["page"] - 1) // s["case"]["page"]
    drop = behind & (s["table"] >= 0)
    s["refs"].index_add_(0, s["table"][drop].long(), torch.full_like(s["table"][drop], -1))
    s["table"].masked_fill_(drop, -1)


def _plain_reserve(s):
    page, table, refs, lens, add = s["case"]["page"], s["table"], s["refs"], s["lens"][:, None], s["add"][:, None]
    place = torch.arange(table.shape[1], device=DEV)
    writes = (place >= lens // page) & (place < (lens + add + page - 1) // page) & (add > 0)
    shared = writes & (table >= 0) & (refs[table.clamp(min=0).long()] > 1)
    need = shared | (writes & (table < 0))
    free = (refs == 0).nonzero()[:, 0].int()
    need &= (need.sum(dim=1).cumsum(0) <= free.numel())[:, None]  # all of a sequence's pages or none
    shared &= need
    seq, at = need.nonzero(as_tuple=True)
    old = table[seq, at]
    new = free[:old.numel()]
    # the rows of a shared page that the sequence has written
    rows = s["lens"][seq] - at.int() * page
    move = (old >= 0) & (rows > 0)
    src, dst = old[move].long(), new[move].long()
    there = torch.arange(page, device=DEV) < rows[move][:, None]
    s["kv"][:, :, dst] = torch.where(there[..., None], s["kv"][:, :, src], s["kv"][:, :, dst])
    refs.index_add_(0, table[shared].long(), torch.full_like(table[shared], -1))
    refs.index_fill_(0, new.long(), 1)
    table[seq, at] = new


def _plain_fork(s):
    page, table, refs = s["case"]["page"], s["table"], s["refs"]
    child = s["parent"] >= 0
    src = s["parent"].clamp(min=0).long()
    lens = s["lens"][src]
    place = torch.arange(table.shape[1], device=DEV)
    new = torch.where(place < ((lens + page - 1) // page)[:, None], table[src], -1)
    new = torch.where(child[:, None], new, table)
    one = torch.ones_like(table)
    refs.index_add_(0, new[new >= 0].long(), one[new >= 0])
    refs.index_add_(0, table[table >= 0].long(), -one[table >= 0])
    table.copy_(new)
    s["lens"].copy_(torch.where(child, lens, s["lens"]))


def _plain_compact(s):
    page, table, refs = s["case"]["page"], s["table"], s["refs"]
    count, keep = s["count"], s["keep"]
    on = count >= 0
    place, at = torch.arange(table.shape[1], device=DEV), torch.arange(keep.shape[1], device=DEV)
    inside = at < count[:, None]
    first = torch.where(inside & (keep != at), at, count[:, None]).amin(dim=1)  # the first position that moves
    pages = (count + page - 1) // page
    stay = torch.where(first == count, pages, first // page)
    need = on[:, None] & (place >= stay[:, None]) & (place < pages[:, None])
    free = (refs == 0).nonzero()[:, 0].int()
    fits = need.sum(dim=1).cumsum(0) <= free.numel()
    on &= fits
    need &= on[:, None]
    seq, col = need.nonzero(as_tuple=True)
    new = torch.where((place < stay[:, None]) | ~on[:, None], table, -1)
    new[seq, col] = free[:seq.numel()]
    seq, col = (on[:, None] & inside & (at >= (stay * page)[:, None])).nonzero(as_tuple=True)
    old = keep[seq, col]
    src = table[seq, (old // page).long()].long() * page + old % page
    dst = new[seq, col // page].long() * page + col % page
    kv = s["kv"].view(s["kv"].shape[0], 2, -1, s["kv"].shape[-1])
    kv[:, :, dst] = kv[:, :, src]
    one = torch.ones_like(table)
    refs.index_add_(0, new[new >= 0].long(), one[new >= 0])
    refs.index_add_(0, table[table >= 0].long(), -one[table >= 0])
    table.copy_(new)
    s["lens"].copy_(torch.where(on, count, s["lens"]))


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "verify":
        return _plain_verify(s)
    if kind == "reserve":
        _plain_trim(s)
        _plain_reserve(s)
    else:
        _plain_fork(s)
        _plain_reserve(s) if kind == "fork" else _plain_compact(s)
    return _state(s)


def _state(s):
    """What the page operators change (reserving for sequences that share nothing moves no keys)."""
    out = {"table": s["table"], "refs": s["refs"], "lens": s["lens"]}
    return out if s["case"]["kind"] == "reserve" else dict(out, kv=s["kv"])


# ----------------------------------------------------------------------------- the framework's calls

def _own(s):
    from paper_2609_13804_gb300 import binding as sp
    kind = s["case"]["kind"]
    if kind == "verify":
        if "ws" not in s:  # kept from call to call, as a program that generates keeps it
            s["ws"] = sp.draft_verify_workspace(T_cap=s["logits"].shape[0], B=s["noise"].shape[0],
                                                V=s["logits"].shape[1], device=DEV)
        r = sp.sp_draft_verify(logits=s["logits"], cu_rows=s["cu_rows"], draft=s["draft"],
                               draft_logits=s["draft_logits"], u=s["u"], noise=s["noise"],
                               temperature=s["temperature"], max_rows=s["case"]["k"] + 1, ws=s["ws"])
        return {"n_accept": r["n_accept"], "token": r["token"], "logp": r["logp"]}
    if "ws" not in s:
        s["ws"] = sp.pages_workspace(S=s["table"].shape[0], max_pages=s["table"].shape[1], device=DEV)
    if kind == "reserve":
        sp.sp_pages_trim(table=s["table"], lens=s["lens"], refs=s["refs"], page_size=s["case"]["page"], err=s["err"])
    else:
        sp.sp_pages_fork(table=s["table"], lens=s["lens"], refs=s["refs"], page_size=s["case"]["page"],
                         parent=s["parent"], err=s["err"])
    if kind == "compact":
        sp.sp_pages_compact(kv=s["kv"], table=s["table"], lens=s["lens"], refs=s["refs"], keep=s["keep"],
                            count=s["count"], ws=s["ws"], err=s["err"])
    else:
        sp.sp_pages_reserve(kv=s["kv"], table=s["table"], lens=s["lens"], refs=s["refs"], add=s["add"], ws=s["ws"],
                            err=s["err"])
    return _state(s)


def run(state):
    return _own(state) if own else _plain(state)


# ----------------------------------------------------------------------------- the definitions, in 64 bits

def exact(case, seed):
    """Sequence by sequence and draft by draft, in logarithms."""
    if case["kind"] != "verify":  # nothing is computed, only moved
        return None
    s = prepare(case, seed)
    drafts, V = _drafts(case), case["vocab"]
    n_accept, token, logp = [], [], []
    r = 0
    for b, k in enumerate(drafts):
        t = float(s["temperature"][b])
        x = s["logits"][r:r + k + 1].double()
        lp = torch.log_softmax(x if t <= 0 else x / t, dim=1)
        lq = torch.log_softmax(s["draft_logits"][r:r + k].double() / t, dim=1) if case["model"] and k and t > 0 else None
        out = []
        for j in range(k):
            d = int(s["draft"][r + j])
            if t <= 0:
                ok = bool(x[j, d] == x[j].max()) and not bool((x[j, :d] == x[j, d]).any())
            else:
                ratio = lp[j, d] - (lq[j, d] if lq is not None else 0.0)
                ok = math.log(float(s["u"][r + j]) or 1e-300) < float(ratio)
            if not ok:
                break
            out.append(d)
        j = len(out)
        if t <= 0:
            score = x[j]
        else:
            left = lp[j].exp()
            if j < k and lq is not None:
                left = (left - lq[j].exp()).clamp(min=0.0)
                left = left if float(left.sum()) > 0 else lp[j].exp()
            elif j < k:
                left[int(s["draft"][r + j])] = 0.0
            score = torch.log(left) - torch.log(s["noise"][b].double())
        order = score.sort(descending=True, stable=True).indices
        out.append(int(order[0]))
        n_accept.append(j)
        logp.append([float(lp[i, v]) for i, v in enumerate(out)] + [0.0] * (case["k"] + 1 - len(out)))
        token.append(out + [-1] * (case["k"] + 1 - len(out)))
        r += k + 1
    return {"n_accept": torch.tensor(n_accept, device=DEV), "token": torch.tensor(token, device=DEV),
            "logp": torch.tensor(logp, dtype=torch.float64, device=DEV)}
