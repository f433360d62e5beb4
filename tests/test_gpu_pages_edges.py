"""Compacting to positions that a row does not have, where they are the ones that would stay in place."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_pages import DEV, Cache, ints, sp  # noqa: E402, F401


def _books(c):
    """The books hold for themselves: counts are what the tables name, and every position of a row has a page."""
    table, refs, lens = c.table.tolist(), c.refs.tolist(), c.lens.tolist()
    named = [0] * len(refs)
    for row, n in zip(table, lens):
        k = c.pages(n)
        assert all(0 <= e < len(refs) for e in row[:k]) and all(e == -1 for e in row[k:]), row
        for e in row[:k]:
            named[e] += 1
    assert named == refs


@pytest.mark.parametrize("length,keep", [
    (5, list(range(20))),                                # longer than the row, into a page that it does not have
    (5, list(range(6))),                                 # into the rest of its page
    (16, list(range(17))), (0, [0]), (0, list(range(40))), (31, list(range(33))), (32, list(range(33))),
    (20, list(range(24)) + [3]),                         # passes the end, then one that moves
    (20, list(range(32)) + [0]), (5, list(range(16)) + [3]), (20, list(range(40)) + [0]), (37, list(range(38)) + [2, 38]),
])
@pytest.mark.parametrize("shared", [False, True])
def test_identity_longer_than_the_row(sp, length, keep, shared):  # noqa: F811
    c = Cache(sp, 3, 4, 24, 16, 2, 24)
    c.reserve([length, 0, 33])
    c.append([length, 0, 33])
    if shared:
        c.fork([-1, 0, -1])
    told, other = c.logical(0), c.logical(2)
    t = torch.full((3, 64), 7, dtype=torch.int32, device=DEV)
    t[0, :len(keep)] = ints(keep)
    err = sp.sp_pages_compact(kv=c.kv, keep=t, count=ints([len(keep), -1, -1]), ws=c.ws, **c.args)
    assert int(err.item()) == 2
    assert c.lens.tolist() == [len(keep), length if shared else 0, 33]
    _books(c)
    host, table = c.kv.cpu(), c.table.tolist()

    def at(s, i):
        return host[:, :, table[s][i // 16], i % 16]

    for i, k in enumerate(keep):  # those that the row has are where they belong
        if k < length:
            assert torch.equal(at(0, i), told[:, :, k])
    if shared:
        assert all(torch.equal(at(1, i), told[:, :, i]) for i in range(length))
    assert all(torch.equal(at(2, i), other[:, :, i]) for i in range(33))


def test_identity_as_long_as_the_row(sp):  # noqa: F811
    """No longer: nothing moves, no error."""
    for length in (0, 1, 5, 16, 17, 33, 64):
        c = Cache(sp, 2, 4, 12, 16, 1, 8)
        c.reserve([length, 3])
        c.append([length, 3])
        table = c.table.tolist()
        c.compact([list(range(length)), None], pad=2, extra=1)
        assert c.table.tolist() == table
        c.compact([list(range(max(length - 1, 0))), None])


def test_identity_longer_than_a_row_in_a_full_pool(sp):  # noqa: F811
    """Such a row needs pages like any that moves; without them it stays as it was."""
    c = Cache(sp, 2, 4, 3, 16)
    c.reserve([20, 0])
    c.append([20, 0])
    before = [t.clone() for t in (c.table, c.lens, c.refs, c.kv)]
    err = sp.sp_pages_compact(kv=c.kv, keep=ints([list(range(40))] * 2), count=ints([40, -1]), ws=c.ws, **c.args)
    assert int(err.item()) & 4
    assert all(torch.equal(a, b) for a, b in zip(before, (c.table, c.lens, c.refs, c.kv)))
