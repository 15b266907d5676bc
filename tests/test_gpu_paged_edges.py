"""Calls on paged caches at the edge of what the header allows."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2412_03213_amd as ck
from paged_ref import D, STEP, Cache, attend, seen_rows
from test_gpu_paged import BF, DEV, F32, close, i32, shape

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_sink,window", [(0, -1), (3, 20)])
@pytest.mark.parametrize("lens,starts,n_rows", [
    ([10], [0, 10], 6), ([400, 90], [0, 300, 390], 350), ([400, 90], [0, 300, 390], 290), ([64, 700], [0, 64, 2 ** 30], 100),
    ([40, 300], [-7, 20, 320], 320), ([3000], [-2, 3], 1)])
def test_starts_beyond_the_rows_of_the_call(lens, starts, n_rows, n_sink, window):
    """Tokens in front of row 0 and from n_rows on are not there; the others keep the rows of the cache that starts
    and lengths give them, for the append and for the attention."""
    Hkv, G, page = 2, 2, 16
    S = len(lens)
    c = Cache(lens, Hkv, page, BF, 3, DEV)
    kv, sh = c.kv(), shape(S, Hkv, G)
    g = torch.Generator().manual_seed(1)
    q, v = (torch.randn(n_rows, h, D, generator=g).to(BF) for h in (Hkv * G, Hkv))
    rows = {}                                            # token row -> sequence, row of the cache
    for s in range(S):
        for t in range(max(0, starts[s]), min(n_rows, starts[s + 1])):
            rows[t] = (s, lens[s] - (starts[s + 1] - starts[s]) + t - starts[s])
    out = torch.full_like(q, 123.0, device=DEV)
    ck.ck_prompt_attn(sh, q.to(DEV), i32(starts), kv, i32(lens), out, n_sink=n_sink, window=window)
    for s in range(S):
        mine = [t for t in rows if rows[t][0] == s]
        seen = [seen_rows(lens[s], rows[t][1], n_sink, window) for t in mine]
        for h in range(Hkv if mine else 0):
            qs = q[mine, h * G:(h + 1) * G].reshape(-1, D)
            want, tol = attend(qs, c.rows_k[s][h], c.rows_v[s][h], np.stack(seen).repeat(G, 0), BF, p_step=2.0 ** -8)
            close(out[mine, h * G:(h + 1) * G].reshape(-1, D), want, tol, f"sequence {s} head {h}")
    assert (out[[t for t in range(n_rows) if t not in rows]] == 123.0).all()
    V = kv.V.clone()
    ck.ck_rope_append(sh, None, v.to(DEV), v.to(DEV), kv, i32(lens), torch.ones(64, device=DEV), None,
                      q_starts=i32(starts))
    for t, (s, r) in rows.items():
        if r >= 0:
            V[c.table[s, r // page], :, r % page] = v[t].to(DEV)
    assert torch.equal(kv.V.view(torch.int16), V.view(torch.int16))


def test_starts_beyond_the_rows_in_a_replayed_graph():
    c = Cache([500, 60], 2, 16, BF, 3, DEV)
    kv, sh = c.kv(), shape(2, 2, 4)
    q = torch.randn(100, 8, D, device=DEV).to(BF)
    starts, n, out, ws = i32([0, 60, 100]), i32([500, 60]), torch.empty_like(q), ck.prompt_workspace(sh, 100, DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ck.ck_prompt_attn(sh, q, starts, kv, n, out, workspace=ws)
    for at in ([0, 60, 100], [0, 450, 500], [0, 90, 150], [0, 60, 100]):
        starts.copy_(i32(at))
        graph.replay()
        torch.cuda.synchronize()
        # the same tokens, with rows for all of them
        whole = torch.zeros(at[-1], 8, D, dtype=BF, device=DEV)
        whole[:100] = q
        want = torch.empty_like(whole)
        ck.ck_prompt_attn(sh, whole, starts, kv, n, want)
        a, b = want[:100].float(), out.float()
        # cut into other pieces: probabilities of both sides rounded to bf16 relative to other maxima, and the outputs
        assert ((a - b).abs() <= 2 ** -7 * a.abs() + 2 * 2 ** -8 * 5.0).all()

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens", [[1], [3, 1, 40], [2100, 17], [9001]])
def test_decode_scores_of_any_finite_size(lens, dtype):
    """Equal scores near -2^110: every row has the same share, as where all scores are zero."""
    c = Cache(lens, 1, 16, dtype, 5, DEV)
    c.K.fill_(-2.0 ** 50)
    q = torch.full((len(lens), 2, D), 2.0 ** 56, dtype=dtype)
    out = torch.empty(len(lens), 2, D, dtype=dtype, device=DEV)
    ck.ck_paged_decode_attn(shape(len(lens), 1, 2, dtype), q.to(DEV), c.kv(), i32(lens), out)
    for s, n in enumerate(lens):
        want, tol = attend(q[s] * 0, c.rows_k[s][0], c.rows_v[s][0], np.ones((2, n)), dtype,
                           p_step=2.0 ** -15 if dtype is BF else 0.0)
        close(out[s], want, tol, f"sequence {s}")


@pytest.mark.parametrize("n,m", [(1, 1), (300, 300), (3000, 3), (9000, 40)])
def test_prompt_scores_of_any_finite_size(n, m):
    c = Cache([n], 1, 16, BF, 5, DEV)
    c.K.fill_(-2.0 ** 50)
    q = torch.full((m, 2, D), 2.0 ** 56, dtype=BF)
    out = torch.empty(m, 2, D, dtype=BF, device=DEV)
    ck.ck_prompt_attn(shape(1, 1, 2), q.to(DEV), i32([0, m]), c.kv(), i32([n]), out)
    seen = np.stack([seen_rows(n, n - m + i, 0, -1) for i in range(m)]).repeat(2, 0)
    want, tol = attend(q.reshape(2 * m, D) * 0, c.rows_k[0][0], c.rows_v[0][0], seen, BF, p_step=2.0 ** -8)
    close(out.reshape(2 * m, D), want, tol, "equal scores")


def overwritten(ws):
    """A workspace's words as a call has left them, with parts overwritten: what a smaller tensor writes that gets the
    memory after it was freed, and words that carry marks of their own."""
    left = ws.clone().view(torch.int16).view(-1, 4)
    for parts in ([0], [1], [3], [0, 1], [2, 3], [0, 3]):
        for value in (1, 2, 15, 0x3F80):
            w = left.clone()
            w[:, parts] = value
            yield w
    for byte in (0, 7):
        w = left.clone().view(torch.uint8).view(-1, 8)
        w[:, byte] = 1
        yield w
    for mark in (0x434B5061676E, 0x434B7469636B):
        for value in (1, 15, 0x3F80):
            yield torch.full_like(left.view(torch.int64), mark << 16 | value)


@pytest.mark.parametrize("lens,Hkv", [([2048], 1), ([2049], 1), ([9001, 300], 1), ([3000, 100, 700], 2)])
def test_decode_workspace_of_any_contents(lens, Hkv):
    """16 and 17 pieces of a head, joined in one stage and in two, and ragged ones."""
    c = Cache(lens, Hkv, 32, BF, 21, DEV)
    kv, sh, n = c.kv(), shape(len(lens), Hkv, 2), i32(lens)
    q = torch.randn(len(lens), 2 * Hkv, D, device=DEV).to(BF)
    ws, want, got = ck.paged_decode_workspace(sh, DEV), torch.empty_like(q), torch.empty_like(q)
    ck.ck_paged_decode_attn(sh, q, kv, n, want, workspace=ws)
    seen = np.ones((2, lens[0]))
    exact, tol = attend(q[0, :2].cpu(), c.rows_k[0][0], c.rows_v[0][0], seen, BF, p_step=2.0 ** -15)
    close(want[0, :2], exact, tol, "sequence 0")
    for i, words in enumerate(overwritten(ws)):
        for again in range(2):
            if again == 0:
                ws.copy_(words.view(torch.uint8).flatten())
            got.fill_(float("nan"))
            ck.ck_paged_decode_attn(sh, q, kv, n, got, workspace=ws)
            assert torch.equal(got, want), (i, again)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rope_angles_next_to_whole_turns(adjacent, dtype):
    """Positions that are close to multiples of pi: their sines show an error of the angle that is small beside a turn."""
    positions = [0, 22, 710, 103993, 833719, 4272943, 80143857, 411557987, 1068966896, 2137933792, 2 ** 31 - 1, -4272943]
    rates = [1.0, 0.5, float(np.float32(0.1))]
    pi = 4 * (4 * _atan_of_one_over(5) - _atan_of_one_over(239))
    n = len(positions)
    c = Cache([n], 1, 16, dtype, 0, DEV)
    kv = c.kv()
    k = torch.zeros(n, 1, D, dtype=dtype)
    first, second = (slice(0, D, 2), slice(1, D, 2)) if adjacent else (slice(0, D // 2), slice(D // 2, D))
    k[..., first] = 1.0
    freqs = torch.tensor(rates + [0.0] * (D // 2 - len(rates)), dtype=torch.float32, device=DEV)
    out = torch.empty(n, 1, D, dtype=dtype, device=DEV)
    ck.ck_rope_append(shape(1, 1, 1, dtype), k.to(DEV), k.to(DEV), k.to(DEV), kv, i32([n]), freqs, out,
                      q_starts=i32([0, n]), positions=i32(positions), interleaved=adjacent)
    rows = torch.stack([kv.K[c.table[0, r // 16], 0, r % 16] for r in range(n)])
    for got in (out[:, 0], rows):
        got = got.double().cpu()
        for i, p in enumerate(positions):
            for j, w in enumerate(rates):
                turns = p * Fraction(w) / (2 * pi)
                a = 2 * math.pi * float(turns - round(turns))
                # The reduced angle a is rounded to fp32 once: it is off by d <= 2^-24 |a|, a cosine by |sin a| d, a sine
                # by |cos a| d (near half a turn, where a sine is small and a is not, that is more than a rounding
                # of the sine).  Then 4 roundings of fp32 (function 2, factor, sum), and that of the type.
                d = abs(a) * 2.0 ** -24
                for want, slope, have in ((math.cos(a), math.sin(a), got[i, first][j]),
                                          (math.sin(a), math.cos(a), got[i, second][j])):
                    tol = 2 * math.pi * 2.0 ** -50 + abs(slope) * d + d * d + abs(want) * (4 * 2.0 ** -24 + STEP[dtype])
                    assert abs(float(have) - want) <= tol, (p, w, float(have), want)


def _atan_of_one_over(n):
    return sum(Fraction((-1) ** i, (2 * i + 1) * n ** (2 * i + 1)) for i in range(40))
