"""How the work of cross and shared-prefix attention is cut: the pieces that the planning workgroup leaves in the workspace have
to cover every row of every block once, their results must not overlap, and the outputs are the formula's in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2412_03213_amd as ck
from paged_ref import D, STEP

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
CUS, TILE, BLOCK, EXTRA = 256, 64, 256, 512              # rows of a tile; query rows of a block; pieces over all heads beyond blocks
PIECE = np.dtype([("t0", "<i4"), ("n_tok", "<i2"), ("flags", "<i2"), ("seq", "<i4"), ("lo", "<i4"), ("end", "<i4"),
                  ("row", "<i4"), ("n_tiles", "<i4"), ("result", "<i4")])
PATTERN = 0x55                                            # of a workspace that no plan was written to


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def attend64(q, K, V):
    """q [M, D], K, V [n, D] -> (out, tol), as paged_ref.attend for rows that all are seen, on the device."""
    q, K, V = q.double(), K.double(), V.double()
    if not K.shape[0]:
        return torch.zeros_like(q), torch.zeros_like(q)
    s = q @ K.T.contiguous() * D ** -0.5
    p = torch.softmax(s, dim=1)
    out, size = p @ V, p @ V.abs()
    ds = 2.0 ** -24 * (D * (q.abs() @ K.abs().T.contiguous()).amax(1) * D ** -0.5 + 4 * s.abs().amax(1) + 4)
    return out, (STEP[BF] * out.abs() * (1 + 2.0 ** -6) +
                 size * (2.0 ** -8 + 2 * ds[:, None] + (K.shape[0] + 8) * 2.0 ** -23) + 1e-30)


class Call:
    """Sequences whose pages are drawn from one pool, so that long ones fit: rows are only read here."""

    def __init__(self, lens, Hkv, G, page, width=0, groups=None, shares=None, pool=512, seed=0):
        self.lens, self.Hkv, self.G, self.page = lens, Hkv, G, page
        S = len(lens)
        g = torch.Generator().manual_seed(seed)
        self.K, self.V = ((torch.randn(pool, Hkv, page, D, generator=g) * f).to(BF).to(DEV) for f in (1.5, 1.0))
        need = -(-max(lens) // page)
        self.table = torch.randint(0, pool, (S, max(need, width, 1)), generator=g, dtype=torch.int32)
        if groups is not None:
            for a, b in zip(groups[:-1], groups[1:]):
                for s in range(a + 1, b):                 # what is shared is the first's, as far as that goes
                    n = max(0, min(shares[s], lens[s], shares[a], lens[a]))
                    self.table[s, :-(-n // page)] = self.table[a, :-(-n // page)]
        self.kv = ck.PagedKV(self.K, self.V, self.table.to(DEV))
        self.groups, self.shares, self.g = groups, shares, g
        self.sh = ck.Shape(S, Hkv * G, Hkv, 1, 1)

    def rows(self, pool, s, h):
        r = torch.arange(self.lens[s])
        return pool[self.table[s].long()[r // self.page].to(DEV), h, (r % self.page).to(DEV)]

    def run(self, news=None):
        """-> out, the workspace; news None: shared-prefix attention"""
        S = len(self.lens)
        self.news = [1] * S if news is None else news
        self.starts = [0] + np.cumsum(self.news).tolist()
        T = self.starts[-1]
        q = (torch.randn(T, self.Hkv * self.G, D, generator=self.g) * 1.5).to(BF).to(DEV)
        self.q, out = q, torch.full_like(q, float("nan"))
        make = (lambda: ck.shared_decode_workspace(self.sh, DEV)) if news is None else (lambda: ck.cross_workspace(self.sh, T, DEV))
        ws = make().fill_(PATTERN)
        if news is None:
            ck.ck_shared_decode_attn(self.sh, q, self.kv, i32(self.lens), i32(self.groups), i32(self.shares), out, workspace=ws)
        else:
            ck.ck_cross_attn(self.sh, q, i32(self.starts), self.kv, i32(self.lens), out, workspace=ws)
        torch.cuda.synchronize()
        return out, ws

    def check(self, out, only=None):
        for s in range(len(self.lens)) if only is None else only:
            a, b = self.starts[s], self.starts[s + 1]
            for h in range(self.Hkv if b > a else 0):
                want, tol = attend64(self.q[a:b, h * self.G:(h + 1) * self.G].reshape(-1, D), self.rows(self.K, s, h),
                                     self.rows(self.V, s, h))
                err = (out[a:b, h * self.G:(h + 1) * self.G].reshape(-1, D).double() - want).abs()
                assert bool((err <= tol).all()), (s, h, float((err - tol).max()))

    def units(self):
        """(first token, tokens, lo, end, group) of every run of rows with the queries that see them"""
        if self.groups is None:
            return [(self.starts[s], m, 0, self.lens[s], False) for s, m in enumerate(self.news)]
        shared = [max(0, min(n, m)) for n, m in zip(self.lens, self.shares)]
        units = [(a, b - a, 0, shared[a] if b > a else 0, True) for a, b in zip(self.groups[:-1], self.groups[1:])]
        first = {s: a for a, b in zip(self.groups[:-1], self.groups[1:]) for s in range(a, b)}
        return units + [(s, 1, min(shared[s], shared[first[s]]) if s in first else 0, n, False) for s, n in enumerate(self.lens)]

    def pieces(self, ws):
        """Pieces of every unit, checked; [numbers of pieces], of all blocks of a unit"""
        n, _ = ws[:8].cpu().numpy().view("<i4")
        p = ws[256:256 + 32 * int(n)].cpu().numpy().view(PIECE)
        left = {}
        for x in p:
            left.setdefault((int(x["t0"]), int(x["lo"]), int(x["end"]), bool(x["flags"] & 2)), []).append(x)
        T, counts, results = BLOCK // self.G, [], []
        for begin, tokens, lo, end, group in self.units():
            counts.append(0)
            for t0 in range(begin, begin + tokens, T):
                m = min(T, begin + tokens - t0)
                row, tiles = lo & ~7, -(-(end - (lo & ~7)) // TILE) if lo < end else 0
                mine = left.pop((t0, lo, end, group), [])
                if tiles == 0 and self.groups is not None:
                    assert not mine
                    continue
                assert mine, (t0, lo, end)
                for x in sorted(mine, key=lambda x: int(x["row"])):     # one behind the other, to the end
                    assert int(x["row"]) == row and int(x["n_tok"]) == m
                    row += TILE * int(x["n_tiles"])
                    if len(mine) > 1 or self.groups is not None:
                        assert int(x["n_tiles"]) > 0
                        results.append((int(x["result"]), m))
                    else:
                        assert int(x["result"]) == -1
                assert row == (lo & ~7) + TILE * tiles
                counts[-1] += len(mine)
        assert not left
        results.sort()
        assert all(a + m <= b for (a, m), (b, _) in zip(results, results[1:]))
        if results:                                       # each of them is in the workspace
            assert results[0][0] >= 0
            rows = (results[-1][0] + results[-1][1]) * self.Hkv * self.G
            assert 256 + 32 * int(n) + rows * (D + 4) * 4 <= ws.numel()
        return counts

    def blocks(self):
        return [-(-m // (BLOCK // self.G)) if lo < end or self.groups is None else 0
                for _, m, lo, end, _ in self.units()]

    def extra(self, counts):
        return sum(max(0, n - b) for n, b in zip(counts, self.blocks())) * self.Hkv


def planned(ws):
    return int(ws[:8].view(torch.int32)[0]) != int.from_bytes(bytes([PATTERN] * 4), "little")


@pytest.mark.parametrize("S,n,m,Hkv,G", [(144, 11759, 2, 2, 4), (18, 11759, 2, 16, 4), (152, 6732, 2, 2, 2)])
def test_blocks_just_above_the_compute_units_are_cut(S, n, m, Hkv, G):
    """One round and a few blocks more: three pieces each would be more pieces than there may be, two are not."""
    c = Call([n] * S, Hkv, G, 16)
    out, ws = c.run([m] * S)
    counts = c.pieces(ws)
    assert CUS < sum(c.blocks()) * Hkv < 2 * CUS
    assert all(k > b for k, b in zip(counts, c.blocks())) and c.extra(counts) <= EXTRA
    c.check(out, only=(0, 1, S // 2, S - 1))


def test_groups_just_above_the_compute_units_are_cut():
    S = 288
    c = Call([11759] * S, 2, 4, 16, groups=list(range(0, S + 1, 2)), shares=[11759] * S)
    out, ws = c.run()
    counts = c.pieces(ws)
    assert CUS < 144 * 2 < 2 * CUS and all(k > 1 for k in counts[:144]) and c.extra(counts) <= EXTRA
    c.check(out, only=(0, 1, 143, 286, 287))


@pytest.mark.parametrize("n,m,Hkv,G", [(3548, 405, 2, 8), (8579, 492, 1, 4), (2640, 357, 4, 1)])
def test_even_shares_fit_the_compute_units(n, m, Hkv, G):
    """Full blocks of 256 queries leave 20 us of results in every piece, more than the whole call should take: no cut that is
    tried fits, and shares are even."""
    c = Call([n] * (4 if Hkv == 4 else 1), Hkv, G, 16, width=4097 // 16 + 1)
    out, ws = c.run([m] * len(c.lens))
    counts = c.pieces(ws)
    even = -(-sum(c.blocks()) * -(-n // TILE) * Hkv // CUS)          # tiles of a share, before it is made longer
    assert 1 < counts[0] // c.blocks()[0] <= -(-n // TILE) // even + 1
    assert sum(counts) * Hkv <= CUS and c.extra(counts) <= EXTRA
    c.check(out)


@pytest.mark.parametrize("S,Hkv", [(4000, 2), (8000, 8), (30000, 1)])
def test_many_segments_are_planned(S, Hkv):
    """In one launch every workgroup walks over all segments to find its own: for so many the plan does it once."""
    lens = [(7 * s) % 97 for s in range(S)]
    c = Call(lens, Hkv, 2, 16)
    out, ws = c.run([(s % 3 > 0) + (s % 1000 == 7) for s in range(S)])
    assert planned(ws)
    c.pieces(ws)
    c.check(out, only=[*range(20), *range(1000, 1010), *range(S - 20, S)])


@pytest.mark.parametrize("S", [64, 500])
def test_segments_of_short_states_go_in_one_launch(S):
    c = Call([(7 * s) % 97 for s in range(S)], 2, 2, 16)
    out, ws = c.run([s % 3 for s in range(S)])
    assert not planned(ws)
    c.check(out, only=[0, 1, 2, S - 1])


@pytest.mark.parametrize("S,n,want", [(17, 3990, True), (17, 2500, False), (64, 3990, False)])
def test_a_round_and_a_few_blocks_of_long_states_are_planned(S, n, want):
    """272 workgroups of 8 heads: the last ones would walk over their rows alone.  512 fill two rounds."""
    c = Call([n - 37 * s % (n // 3) for s in range(S)], 8, 4, 16)
    out, ws = c.run([(100 if S == 17 else 16) - s % 30 * (S == 17) for s in range(S)])
    assert CUS < sum(c.blocks()) * 8
    assert planned(ws) == want
    c.check(out, only=(0, 1, S - 1))
    if want:
        c.pieces(ws)


def falling(n, S, least=1):
    """S lengths between a tenth of n and n."""
    return [max(least, int(n * (1 - 0.9 * ((s * 0.618) % 1)))) for s in range(S)]


def test_pieces_in_order_of_their_size_several_of_a_thread():
    """250 segments of one head, planned by 256 threads: some 500 pieces, put in order two at a time."""
    c = Call(falling(6000, 250), 1, 4, 16)
    out, ws = c.run([1] * 250)
    counts = c.pieces(ws)
    assert len(c.units()) <= 256 < sum(counts) and max(counts) > 1
    c.check(out)


def test_pieces_of_groups_in_order_of_their_size_several_of_a_thread():
    c = Call(falling(9000, 160, 64), 1, 4, 16, groups=list(range(0, 161, 2)), shares=[100] * 160)
    out, ws = c.run()
    counts = c.pieces(ws)
    assert len(c.units()) <= 256 < sum(counts) and max(counts) > 1
    c.check(out)


@pytest.mark.parametrize("even", [False, True])
def test_more_segments_than_threads_that_are_cut(even):
    """Long segments among the first 1024 units and behind them; with full blocks shares are even."""
    lens, news = [(7 * s) % 197 for s in range(1100)], [(3 * s) % 5 for s in range(1100)]
    for s in (0, 1, 1097, 1099):
        lens[s], news[s] = 9000, 3
    if even:
        lens, news = [(7 * s) % 40 for s in range(1100)], [s % 2 for s in range(1100)]
        lens[3], news[3], lens[1090], news[1090] = 9000, 3, 8579, 492
    c = Call(lens, 1, 4 if even else 2, 16)
    out, ws = c.run(news)
    counts = c.pieces(ws)
    cut = [i for i, (k, b) in enumerate(zip(counts, c.blocks())) if k > b]
    assert cut and cut[0] < 1024 <= cut[-1] and c.extra(counts) <= EXTRA
    c.check(out, only=[*cut, *range(4, 40), *range(1000, 1100)])


def test_more_groups_and_sequences_than_threads_that_are_cut():
    S = 900
    lens, shares = [100 + (s * 31) % 90 for s in range(S)], [90 if s % 2 == 0 else 71 for s in range(S)]
    for s in (0, 1):
        lens[s], shares[s] = 9100 + s, 9000
    lens[897] = lens[899] = 8000
    c = Call(lens, 1, 2, 16, width=161 * 10 ** 6 // (512 * S) // 16 + 1, groups=[*range(0, S, 2), S], shares=shares)
    out, ws = c.run()
    counts = c.pieces(ws)
    # groups 0 to 449, then the sequences
    assert counts[0] > 1 and counts[450 + 897] > 1 and 450 + 897 >= 1024 and c.extra(counts) <= EXTRA
    c.check(out, only=[*range(30), *range(880, S)])


def test_groups_of_full_blocks_in_even_shares():
    """Four groups of 256 query rows: as in the cross attention, no cut that is tried fits."""
    S, n = 256, 16900
    c = Call([n] * S, 1, 4, 16, groups=[0, 64, 128, 192, 256], shares=[n] * S)
    out, ws = c.run()
    counts = c.pieces(ws)
    even = -(-4 * -(-n // TILE) // CUS)
    assert counts[:4] == [counts[0]] * 4 and 1 < counts[0] <= -(-n // TILE) // even + 1 and sum(counts) <= CUS
    c.check(out, only=(0, 63, 64, 130, 255))


def test_cross_more_blocks_than_compute_units_and_a_long_segment():
    """280 workgroups without a cut, and a segment that is cut; longest first."""
    c = Call([150, 9000, 70, 3000], 8, 1, 16)
    out, ws = c.run([7000, 2, 900, 300])
    counts = c.pieces(ws)
    assert sum(c.blocks()) * 8 > CUS and counts[1] > 1
    c.check(out)
