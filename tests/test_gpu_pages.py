"""The pages of a cache against books kept in Python: tables, counts and lengths to the entry, contents to the bit."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"

from test_gpu_paged import single_precision  # noqa: E402, F401


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2609_13804_gb300 import binding
    return binding


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Cache:
    """A cache on the GPU and the same on the host; every call is made on both and compared."""

    def __init__(self, sp, S, max_pages, n_pages, page, layers=2, width=16):
        self.sp, self.page, self.mp, self.S = sp, page, max_pages, S
        self.table = torch.full((S, max_pages), -1, dtype=torch.int32, device=DEV)
        self.lens, self.refs = ints([0] * S), ints([0] * n_pages)
        self.kv = torch.zeros((layers, 2, n_pages, page, width), dtype=torch.bfloat16, device=DEV)
        self.rows, self.n, self.count = [[-1] * max_pages for _ in range(S)], [0] * S, [0] * n_pages
        self.host = self.kv.cpu()
        self.ws = sp.pages_workspace(S=S, max_pages=max_pages)
        self.g = torch.Generator().manual_seed(S * max_pages + n_pages)
        self.args = dict(table=self.table, lens=self.lens, refs=self.refs)

    def check(self, err, want=0):
        assert int(err.item()) == want
        assert self.lens.tolist() == self.n
        assert self.table.tolist() == self.rows
        assert self.refs.tolist() == self.count
        assert torch.equal(self.kv.cpu(), self.host)
        named = [0] * len(self.count)
        for r in self.rows:
            for e in r:
                if 0 <= e < len(named):
                    named[e] += 1
        assert named == self.count

    def upload(self):
        self.table.copy_(torch.tensor(self.rows, dtype=torch.int32))
        self.lens.copy_(torch.tensor(self.n, dtype=torch.int32))
        self.refs.copy_(torch.tensor(self.count, dtype=torch.int32))
        self.kv.copy_(self.host)

    def pages(self, n):
        return -(-n // self.page)

    def _serve(self, need):
        """The fresh pages of every row, None from the first on that does not fit."""
        free = [p for p, c in enumerate(self.count) if c == 0]
        out, at, full = [], 0, False
        for k in need:
            full |= at + k > len(free)
            out.append(None if full else free[at:at + k])
            at += k
        return out, full

    def append(self, add):
        """New positions behind every row's, written as a program does it (rows that have the pages)."""
        for s, a in enumerate(add):
            for i in range(self.n[s], self.n[s] + a):
                e = self.rows[s][i // self.page]
                assert self.count[e] == 1
                self.host[:, :, e, i % self.page] = torch.randn(self.host.shape[0], 2, self.host.shape[-1], generator=self.g).bfloat16()
            self.n[s] += a
        self.upload()

    def logical(self, s):
        at = range(self.n[s])
        return self.host[:, :, [self.rows[s][i // self.page] for i in at], [i % self.page for i in at]]

    def trim(self):
        for s, r in enumerate(self.rows):
            for c in range(self.pages(self.n[s]), self.mp):
                if r[c] >= 0:
                    self.count[r[c]] -= 1
                    r[c] = -1
        self.check(self.sp.sp_pages_trim(page_size=self.page, **self.args))

    def fork(self, parent):
        old, n = [list(r) for r in self.rows], list(self.n)
        for s, p in enumerate(parent):
            if p < 0 or p == s:
                continue
            k = self.pages(n[p])
            new = old[p][:k] + [-1] * (self.mp - k)
            for e in new:
                self.count[e] += e >= 0
            for e in old[s]:
                self.count[e] -= e >= 0
            self.rows[s], self.n[s] = new, n[p]
        self.check(self.sp.sp_pages_fork(page_size=self.page, parent=ints(parent), **self.args))

    def reserve(self, add, want=0):
        take = []
        for s, a in enumerate(add):
            places = range(self.n[s] // self.page, self.pages(self.n[s] + a)) if a > 0 else ()
            take.append([c for c in places if self.rows[s][c] < 0 or self.count[self.rows[s][c]] > 1])
        fresh, full = self._serve([len(t) for t in take])
        before = self.host.clone()
        for s, (t, f) in enumerate(zip(take, fresh)):
            for c, e in zip(t, f or ()):
                old = self.rows[s][c]
                if old >= 0:
                    k = max(0, self.n[s] - c * self.page)
                    self.host[:, :, e, :k] = before[:, :, old, :k]
                    self.count[old] -= 1
                self.rows[s][c], self.count[e] = e, 1
        if full:
            want |= 4
        self.check(self.sp.sp_pages_reserve(kv=self.kv, add=ints(add), ws=self.ws, **self.args), want)
        return full

    def compact(self, keep, pad=0, extra=0):
        """keep: the positions of every row, None where it stays."""
        need, stay = [], []
        for s, k in enumerate(keep):
            if k is None:
                need.append(0)
                stay.append(0)
                continue
            first = next((i for i, x in enumerate(k) if x != i), len(k))
            stay.append(self.pages(len(k)) if first == len(k) else first // self.page)
            need.append(self.pages(len(k)) - stay[-1])
        fresh, full = self._serve(need)
        before = self.host.clone()
        for s, k in enumerate(keep):
            if k is None or fresh[s] is None:
                continue
            old = self.rows[s]
            new = old[:stay[s]] + fresh[s]
            for e in old[stay[s]:]:
                self.count[e] -= e >= 0
            for e in fresh[s]:
                self.count[e] = 1
            for i in range(stay[s] * self.page, len(k)):
                self.host[:, :, new[i // self.page], i % self.page] = before[:, :, old[k[i] // self.page], k[i] % self.page]
            self.rows[s], self.n[s] = new + [-1] * (self.mp - len(new)), len(k)
        width = max([len(k) for k in keep if k] + [1])
        t = torch.full((self.S, width + pad), 1 << 28, dtype=torch.int32, device=DEV)
        for s, k in enumerate(keep):
            if k:
                t[s, :len(k)] = ints(k)
        count = ints([-1 if k is None else len(k) for k in keep])
        self.check(self.sp.sp_pages_compact(kv=self.kv, keep=t[:, :width + extra], count=count, ws=self.ws, **self.args), 4 if full else 0)
        return full


@pytest.mark.parametrize("page,width,layers", [(16, 8, 1), (16, 24, 3), (32, 40, 1), (16, 264, 2), (32, 512, 2), (64, 64, 1), (128, 1024, 1),
                                               (16, 4104, 1)])
def test_a_prompt_its_samples_and_their_ends(sp, page, width, layers):
    c = Cache(sp, 5, 6, 24, page, layers, width)
    c.reserve([2 * page + 3, 0, 0, 0, 1])
    c.append([2 * page + 3, 0, 0, 0, 1])
    c.fork([-1, 0, 0, 0, -1])                       # three samples
    told = c.logical(0)
    c.reserve([0, 1, page, 2 * page, 0])            # the partly filled page becomes each one's own
    assert all(torch.equal(c.logical(s), told) for s in (1, 2, 3))
    c.append([0, 1, page, 5, 0])
    assert torch.equal(c.logical(0), told)
    c.trim()                                        # what the third did not use
    c.reserve([1, 0, 0, 0, 0])                      # nobody else writes there any more
    c.append([1, 0, 0, 0, 0])
    c.compact([None, list(range(0, 2 * page, 2)) + [2 * page + 3], list(range(page + 2)), [], list(range(1))])
    for s in range(5):
        c.n[s] = 0
    c.upload()
    c.trim()
    assert sum(c.count) == 0


@pytest.mark.parametrize("seed", range(6))
def test_random_calls(sp, seed):
    rng = random.Random(seed)
    page = rng.choice([16, 32])
    S, mp = rng.choice([(3, 5), (40, 7), (7, 40)])
    n_pages = rng.choice([S * mp, S * mp // 2 + 1, 4 * rng.randint(5, 12) + 3])
    c = Cache(sp, S, mp, n_pages, page, 1, 8)
    short = 0
    for _ in range(40):
        what = rng.choice(["reserve", "reserve", "append", "append", "trim", "fork", "compact", "end"])
        room = [mp * page - n for n in c.n]
        if what == "reserve":
            short += c.reserve([rng.choice([0, 0, 1, min(r, 5), rng.randint(0, r), min(r, page)]) if r else 0 for r in room])
        elif what == "append":
            def most(s):
                k = c.n[s]
                while k < mp * page and c.rows[s][k // page] >= 0 and c.count[c.rows[s][k // page]] == 1:
                    k += 1
                return k - c.n[s]
            c.append([rng.randint(0, most(s)) for s in range(S)])
        elif what == "trim":
            c.trim()
        elif what == "fork":
            c.fork([rng.choice([-1, -1, -1, s, rng.randrange(S)]) for s in range(S)])
        elif what == "compact":
            keep = []
            for s in range(S):
                n = c.n[s]
                lead = rng.randint(0, n)
                rest = sorted(rng.sample(range(lead, n), rng.randint(0, n - lead)))
                k = list(range(lead)) + rest
                if n and rng.random() < 0.2:
                    k = [rng.randrange(n) for _ in range(rng.randint(1, min(n + 3, mp * page)))]  # any order, positions twice
                keep.append(rng.choice([None, k, k]))
            pad = rng.choice([0, 3])
            short += c.compact(keep, pad, pad and rng.choice([0, 2]))
        else:
            for s in range(S):
                if rng.random() < 0.3:
                    c.n[s] = rng.randint(0, c.n[s])
            c.upload()


def test_pages_run_out(sp):
    c = Cache(sp, 4, 4, 6, 16)
    assert c.reserve([33, 20, 40, 0])               # 3 + 2 of 6; the third does not fit, the fourth wants none
    c.append([33, 20, 0, 0])
    assert c.reserve([0, 0, 33, 1])                 # neither does the fourth behind it
    assert not c.reserve([0, 0, 16, 0])
    c.append([0, 0, 16, 0])
    assert c.compact([list(range(1, 33)), list(range(5)), [0, 2], None])
    assert c.n == [33, 20, 16, 0]
    assert not c.compact([list(range(20)), list(range(5)), list(range(3)), None])  # what only gets shorter needs none
    assert not c.compact([[0, 2, 4], None, None, None])


def test_a_pool_of_one_page(sp):
    c = Cache(sp, 2, 1, 1, 1024, 1, 8)
    assert not c.reserve([1024, 0])
    c.append([1024, 0])
    assert c.reserve([0, 1])
    c.fork([-1, 0])
    assert c.compact([None, [1023]])                # the only page is shared
    c.fork([-1, -1])
    c.n[0] = 0
    c.upload()
    c.trim()
    assert c.count == [1]
    c.reserve([0, 0])


def test_a_page_shared_by_the_rows_that_write_it(sp):
    """Two rows share a partly filled page and nobody else has it: both copies are made and the page is free."""
    c = Cache(sp, 3, 3, 9, 16)
    c.reserve([20, 0, 0])
    c.append([20, 0, 0])
    c.fork([-1, 0, 0])
    c.n[0] = 0
    c.upload()
    c.trim()
    c.reserve([0, 1, 1])
    assert c.count.count(1) == 2 and c.count.count(2) == 1
    # entries behind the last position are shared too after a row was shortened: replaced, with nothing to copy
    c.fork([1, -1, -1])
    c.n[0] = c.n[1] = 3
    c.upload()
    c.reserve([30, 0, 0])


def test_bad_rows_stay_as_they_were(sp):
    c = Cache(sp, 6, 3, 20, 16)
    c.reserve([17, 5, 33, 1, 9, 2])
    c.append([17, 5, 33, 1, 9, 2])
    good = [list(c.n), [list(r) for r in c.rows]]
    # reserve: lengths and additions outside the table
    c.n[0], c.n[1] = 49, -1
    c.upload()
    for add in ([1, 1, 16, -1, 40, 2 ** 31 - 1], [0, 0, 16, 0, 48, 47]):
        before = [list(r) for r in c.rows]
        err = sp.sp_pages_reserve(kv=c.kv, add=ints(add), ws=c.ws, **c.args)
        assert int(err.item()) == 2
        assert c.table.tolist() == before
    assert int(sp.sp_pages_trim(page_size=16, **c.args).item()) == 2
    assert c.table.tolist() == c.rows and c.refs.tolist() == c.count
    # forks of rows that are not there, or have such lengths
    err = sp.sp_pages_fork(page_size=16, parent=ints([-1, -1, 6, -2, 0, 1]), **c.args)
    assert int(err.item()) == 2
    assert c.table.tolist() == c.rows and c.refs.tolist() == c.count and c.lens.tolist() == c.n
    # compact: counts outside keep, and a row with a bad length
    c.n = good[0]
    c.upload()
    keep = ints([[1, 2, 3]] * 6)
    err = sp.sp_pages_compact(kv=c.kv, keep=keep, count=ints([-2, 4, 2 ** 31 - 1, -1, -1, -2 ** 31]), ws=c.ws, **c.args)
    c.check(err, 2)


def test_bad_entries_and_positions_are_skipped(sp):
    c = Cache(sp, 3, 4, 12, 16)
    c.reserve([20, 20, 20])
    c.append([20, 20, 20])
    # positions that the row does not have: the others move
    want = c.logical(0)[:, :, [3, 19]]
    keep = ints([[3, 20, 19, -1]] * 3)
    err = sp.sp_pages_compact(kv=c.kv, keep=keep, count=ints([4, -1, -1]), ws=c.ws, **c.args)
    assert int(err.item()) == 2 and c.lens.tolist() == [4, 20, 20]
    p = int(c.table[0, 0])
    assert torch.equal(c.kv[:, :, p, [0, 2]].cpu(), want)
    # entries outside the pool count as none
    c.table[1, 0], c.table[1, 2] = 12, 2 ** 31 - 1
    refs = c.refs.clone()
    assert int(sp.sp_pages_trim(page_size=16, **c.args).item()) == 2
    assert c.table[1].tolist()[2:] == [-1, -1] and torch.equal(c.refs, refs)
    err = sp.sp_pages_fork(page_size=16, parent=ints([-1, -1, 1]), **c.args)
    assert int(err.item()) == 2 and int(c.table[2, 0]) == -1 and int(c.table[2, 1]) == int(c.table[1, 1])
    c.lens[1] = 0
    assert int(sp.sp_pages_reserve(kv=c.kv, add=ints([0, 1, 0]), ws=c.ws, **c.args).item()) == 2
    assert 0 <= int(c.table[1, 0]) < 12


def test_most_rows(sp):
    """As many rows as a table may have, and a pool whose free pages lie far apart."""
    S, page = 4096, 16
    c = Cache(sp, S, 2, 40000, page, 1, 8)
    for p in range(0, 40000):
        if p % 3:
            c.count[p] = 1
    busy = list(c.count)
    c.upload()
    for s, a in enumerate(add := [(s * 7) % 33 for s in range(S)]):
        assert a <= 2 * page
    err = sp.sp_pages_reserve(kv=c.kv, add=ints(add), ws=c.ws, **c.args)
    assert int(err.item()) == 0
    want, free = [], iter(range(0, 40000, 3))
    for a in add:
        k = -(-a // page)
        want.append([next(free) for _ in range(k)] + [-1] * (2 - k))
    assert c.table.tolist() == want
    c.lens.copy_(ints(add))
    c.kv.normal_()
    parent = [s - 1 if s % 2 else -1 for s in range(S)]
    assert int(sp.sp_pages_fork(page_size=page, parent=ints(parent), **c.args).item()) == 0
    want = [want[s - 1] if s % 2 else want[s] for s in range(S)]
    assert c.table.tolist() == want
    assert int(sp.sp_pages_compact(kv=c.kv, keep=ints([[1] if s % 5 == 0 and add[s - s % 2] > 1 else [0] for s in range(S)]),
                                   count=ints([1 if s % 5 == 0 and add[s - s % 2] > 1 else -1 for s in range(S)]), ws=c.ws,
                                   **c.args).item()) == 0
    for s in range(0, S, 5):
        if add[s - s % 2] > 1:
            assert torch.equal(c.kv[:, :, int(c.table[s, 0]), 0], c.kv[:, :, want[s][0], 1])
    c.lens.zero_()
    sp.sp_pages_trim(page_size=page, **c.args)
    assert c.refs.tolist() == busy and (c.table == -1).all()


def test_calls_in_a_graph_and_on_another_stream(sp):
    page = 16
    c = Cache(sp, 8, 6, 64, page, 2, 64)
    c.reserve([40] + [0] * 7)
    c.append([40] + [0] * 7)
    parent, add = ints([-1] + [0] * 7), ints([0] + [1] * 7)
    err, wide = ints([0]), torch.full((c.ws.numel() + 4096,), 7, dtype=torch.uint8, device=DEV)
    ws = wide[:c.ws.numel()]
    keep, count = ints([[0] * 3] + [[5, 17, 39]] * 7), ints([-1] + [3] * 7)

    def step(stream=None):
        sp.sp_pages_fork(page_size=page, parent=parent, err=err, stream=stream, **c.args)
        sp.sp_pages_reserve(kv=c.kv, add=add, ws=ws, err=err, stream=stream, **c.args)
        sp.sp_pages_compact(kv=c.kv, keep=keep, count=count, ws=ws, err=err, stream=stream, **c.args)
        sp.sp_pages_trim(page_size=page, err=err, stream=stream, **c.args)

    step()
    torch.cuda.synchronize()
    state = [t.clone() for t in (c.table, c.lens, c.refs, c.kv)]
    st = torch.cuda.Stream()
    step(st)
    torch.cuda.synchronize()
    assert c.lens.tolist() == [40] + [3] * 7
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert int(err.item()) == 0 and (wide[ws.numel():] == 7).all()
    assert c.lens.tolist() == state[1].tolist() and sorted(c.refs.tolist()) == sorted(state[2].tolist())
    told = state[3][:, :, [int(state[0][0, i // page]) for i in (5, 17, 39)], [i % page for i in (5, 17, 39)]]
    for s in range(1, 8):
        assert torch.equal(c.kv[:, :, int(c.table[s, 0]), :3], told)


def test_far_positions(sp):
    """A pool of more than 2^32 bytes and places behind 2^31 elements of a plane."""
    page, width, n_pages = 1024, 2048, 1100
    kv = torch.empty((1, 2, n_pages, page, width), dtype=torch.bfloat16, device=DEV)
    table, refs = torch.full((2, 1030), -1, dtype=torch.int32, device=DEV), torch.ones(n_pages, dtype=torch.int32, device=DEV)
    refs[[1090, 1098, 1099]] = 0
    args = dict(table=table, lens=ints([0, 0]), refs=refs)
    assert int(sp.sp_pages_reserve(kv=kv, add=ints([5, 0]), **args).item()) == 0
    assert table[0, 0] == 1090
    kv[:, :, 1090, :5].normal_()
    args["lens"][0] = 5
    assert int(sp.sp_pages_fork(page_size=page, parent=ints([-1, 0]), **{k: args[k] for k in args}).item()) == 0
    assert int(sp.sp_pages_reserve(kv=kv, add=ints([0, 1]), **args).item()) == 0
    assert table[1, 0] == 1098 and torch.equal(kv[:, :, 1098, :5], kv[:, :, 1090, :5])
    assert int(sp.sp_pages_compact(kv=kv, keep=ints([[4, 2]] * 2), count=ints([-1, 2]), **args).item()) == 0
    assert table[1, 0] == 1099 and torch.equal(kv[:, :, 1099, :2], kv[:, :, 1090, [4, 2]])
    assert refs[[1090, 1098, 1099]].tolist() == [1, 0, 1]


def test_binding_refuses_wrong_tensors(sp):
    c = Cache(sp, 3, 4, 12, 16)
    ok = dict(kv=c.kv, add=ints([1, 0, 0]), **c.args)
    sp.sp_pages_reserve(**ok)
    for bad in (dict(kv=c.kv[0]), dict(kv=c.kv.float()), dict(kv=c.kv[:, :, :11]), dict(table=c.table.long()), dict(lens=ints([0])),
                dict(refs=c.refs.cpu()), dict(add=ints([1, 0])), dict(table=c.table.t())):
        with pytest.raises(ValueError):
            sp.sp_pages_reserve(**dict(ok, **bad))
    with pytest.raises(ValueError):
        sp.sp_pages_fork(page_size=16, parent=ints([0]), **c.args)
    with pytest.raises(ValueError):
        sp.sp_pages_compact(kv=c.kv, keep=ints([[0]] * 3).long(), count=ints([-1] * 3), **c.args)
    for call in (lambda: sp.sp_pages_trim(page_size=24, **c.args),
                 lambda: sp.sp_pages_reserve(ws=torch.empty(256, dtype=torch.uint8, device=DEV), **ok)):
        with pytest.raises(sp.SPError):
            call()
