"""Pages and slots on the GPU against the oracle's loops, value for value."""
import numpy as np
import pytest
import torch

from oracle import pages as PG
from paper_2504_06419_amd import spire

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Case:
    def __init__(self, seed, B, ps, hi, new_hi, slack=0, tokens=None, maxb=None, odd=False):
        r = np.random.default_rng(seed)
        self.ps = ps
        self.lens = [int(x) for x in r.integers(0, hi + 1, B)]
        self.new = [int(x) for x in r.integers(0, new_hi + 1, B)]
        if odd:  # values a caller should not give: all of them mean something
            for x in range(0, B, 5):
                self.new[x] = -3
            for x in range(1, B, 7):
                self.lens[x] = -2
        held = [-(-max(n, 0) // ps) for n in self.lens]
        want = [-(-(max(n, 0) + max(m, 0)) // ps) for n, m in zip(self.lens, self.new)]
        self.maxb = maxb or max(want + [1]) + 1
        pool = sum(want) + 5
        ids = [int(x) for x in r.permutation(pool)]
        self.table = [[ids.pop() if c < h else -1 for c in range(self.maxb)] for h in held]
        self.free = ids
        if odd and self.free:
            self.free[len(self.free) // 2] = -9
        self.n = len(self.free) - slack
        self.tokens = sum(max(m, 0) for m in self.new) + 3 if tokens is None else tokens
        self.B = B

    def gpu(self, in_place=False):
        d = dict(t=ints(self.table).view(self.B, self.maxb), lens=ints(self.lens), new=ints(self.new), free=ints(self.free),
                 n=ints([self.n]))
        slots = torch.full((self.tokens,), -77, dtype=torch.int64, device=DEV)
        pos = torch.full((self.tokens,), -77, dtype=torch.int32, device=DEV)
        cu = torch.full((self.B + 1,), -77, dtype=torch.int32, device=DEV)
        lo, no = (None, None) if in_place else (torch.full_like(d["lens"], -7), torch.full_like(d["n"], -7))
        spire.page_extend(d["t"], self.ps, d["lens"], d["new"], d["free"], d["n"], slots, pos, cu, lens_out=lo, n_free_out=no)
        torch.cuda.synchronize()
        assert d["free"].tolist() == self.free
        if not in_place:
            assert d["lens"].tolist() == self.lens and d["n"].tolist() == [self.n]
        return (d["t"].tolist(), slots.tolist(), pos.tolist(), cu.tolist(), (d["lens"] if in_place else lo).tolist(),
                int(d["n"] if in_place else no))

    def want(self):
        return PG.extend(self.table, self.ps, self.lens, self.new, self.free, self.n, self.tokens)


@pytest.mark.parametrize("B,ps,hi,new_hi", [(1, 16, 0, 1), (1, 1, 5, 40), (5, 16, 100, 5), (64, 64, 300, 900), (63, 7, 200, 9),
                                            (1023, 16, 90, 4), (1024, 16, 90, 4), (1025, 16, 90, 4), (8192, 2, 9, 3),
                                            (3, 128, 1, 20000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_extend(B, ps, hi, new_hi, in_place):
    c = Case(B + ps, B, ps, hi, new_hi)
    assert c.gpu(in_place) == tuple(c.want())


@pytest.mark.parametrize("B,ps,hi,new_hi", [(1000, 16, 90, 2), (1024, 4, 300, 1), (200, 1, 40, 18), (200, 8, 40, 30), (3, 16, 50, 600),
                                            (8192, 16, 90, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_extend_in_one_launch_and_two(B, ps, hi, new_hi, in_place):
    c = Case(7 * B + ps, B, ps, hi, new_hi)
    assert c.gpu(in_place) == tuple(c.want())


@pytest.mark.parametrize("slack,tokens,maxb", [(6, None, None), (40, None, None), (0, 20, None), (0, 0, None), (0, None, 6),
                                               (10**6, None, None), (-50, None, None)])
def test_extend_refuses(slack, tokens, maxb):
    """Too few pages, too few token places, short table rows, no free page at all, a count beyond the pool."""
    c = Case(9, 40, 4, 20, 9, slack, tokens, maxb) if maxb is None else None
    if c is None:
        c = Case(9, 40, 4, 20, 9)
        c.table = [r[:maxb] for r in c.table]
        c.lens = [min(n, maxb * 4) for n in c.lens]
        c.maxb = maxb
    assert c.gpu() == tuple(c.want())


def test_odd_values():
    """Negative lengths, counts and page ids."""
    c = Case(4, 50, 4, 30, 9, odd=True)
    assert c.gpu() == tuple(c.want())


def test_far_slots():
    """Slots beyond 32 bits."""
    t = ints([[2**31 - 1, -1]])
    slots, pos, cu = torch.empty(3, dtype=torch.int64, device=DEV), ints([0] * 3), ints([0, 0])
    spire.page_extend(t, 1 << 20, ints([5]), ints([3]), ints([]), ints([0]), slots, pos, cu)
    assert slots.tolist() == [(2**31 - 1) * 2**20 + p for p in (5, 6, 7)]


def test_nothing():
    """No sequences: only the padding and the counts are written."""
    slots, pos, cu, n = torch.zeros(5, dtype=torch.int64, device=DEV), ints([4] * 5), ints([9]), ints([2])
    spire.page_extend(torch.empty(0, 4, dtype=torch.int32, device=DEV), 16, ints([]), ints([]), ints([1, 2]), n, slots, pos, cu)
    assert slots.tolist() == [-1] * 5 and pos.tolist() == [0] * 5 and cu.tolist() == [0] and n.tolist() == [2]


@pytest.mark.parametrize("B,ps,hi,room", [(1, 16, 100, 99), (7, 1, 30, 400), (300, 16, 3000, 10**5), (1025, 4, 50, 10**5),
                                          (20, 4, 200, 30), (20, 4, 200, 0), (8192, 16, 40, 10**5)])
@pytest.mark.parametrize("in_place", [False, True])
def test_release(B, ps, hi, room, in_place):
    r = np.random.default_rng(B)
    lens = [int(x) for x in r.integers(0, hi + 1, B)]
    keep = [int(x) for x in r.integers(-2, hi + 10, B)]
    maxb = -(-hi // ps) + 1
    table = r.permutation(B * maxb).reshape(B, maxb)
    free = [-5] * 3 + [-6] * room
    t, l, k, f, n = ints(table), ints(lens), ints(keep), ints(free), ints([3])
    lo, no = (None, None) if in_place else (torch.empty_like(l), torch.empty_like(n))
    spire.page_release(t, ps, l, k, f, n, lens_out=lo, n_free_out=no)
    torch.cuda.synchronize()
    want = PG.release(table.tolist(), ps, lens, keep, free, 3)
    assert (f.tolist(), (l if in_place else lo).tolist(), int(n if in_place else no)) == tuple(want)
    assert np.array_equal(t.cpu().numpy(), table)


def test_rounds_in_a_graph():
    """Extend and release in place, captured, with the program's own work between replays."""
    B, ps, k = 33, 4, 4
    r = np.random.default_rng(5)
    lens, pool = [int(x) for x in r.integers(0, 20, B)], 600
    ids = [int(x) for x in r.permutation(pool)]
    table = [[ids.pop() if c < -(-n // ps) else -1 for c in range(40)] for n in lens]
    keeps = [[int(x) for x in r.integers(0, k + 2, B)] for _ in range(5)]
    t, l, f, n = ints(table), ints(lens), ints(ids + [-1] * (pool - len(ids))), ints([len(ids)])
    new, keep, before = ints([k + 1] * B), ints([0] * B), torch.empty(B, dtype=torch.int32, device=DEV)
    slots, pos, cu = torch.empty(B * (k + 1), dtype=torch.int64, device=DEV), torch.empty(B * (k + 1), dtype=torch.int32, device=DEV), ints([0] * (B + 1))
    ws = spire.workspace(spire.page_workspace_size(B))
    accepted = ints([0] * B)

    def step():
        before.copy_(l)
        spire.page_extend(t, ps, l, new, f, n, slots, pos, cu, ws=ws)
        torch.add(before, accepted, out=keep)
        spire.page_release(t, ps, l, keep, f, n, ws=ws)

    g = torch.cuda.CUDAGraph()
    state = [x.clone() for x in (t, l, f, n)]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step()
    for x, y in zip((t, l, f, n), state):
        x.copy_(y)
    free, count = f.tolist(), len(ids)
    for a in keeps:
        accepted.copy_(ints(a))
        g.replay()
        torch.cuda.synchronize()
        table, ws_, wp, _, grown, count = PG.extend(table, ps, lens, [k + 1] * B, free, count, B * (k + 1))
        free, lens, count = PG.release(table, ps, grown, [x + y for x, y in zip(lens, a)], free, count)
        assert slots.tolist() == ws_ and pos.tolist() == wp and t.tolist() == table
        assert l.tolist() == lens and int(n) == count and f.tolist() == free
