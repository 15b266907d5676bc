"""Operators on paged caches against their plain forms in 64 bits: one-token attention, prompt attention, rotary
append and row copies, at the sizes, masks and tables where they can go wrong."""
import math

import numpy as np
import pytest
import torch

import paper_2412_03213_amd as ck
from paged_ref import D, STEP, Cache, attend, seen_rows, turn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def shape(S, Hkv, G, dtype=BF):
    return ck.Shape(S, Hkv * G, Hkv, 1, 1, dtype=ck.CK_BF16 if dtype is BF else ck.CK_F32)


def close(got, want, tol, what):
    got = got.detach().double().cpu().numpy()
    assert np.isfinite(got).all(), f"{what}: not finite"
    worst = (np.abs(got - want) - tol).max()
    assert worst <= 0, f"{what}: off by {np.abs(got - want).max():.3g}, {worst:.3g} more than allowed"


# ---------------------------------------------------------------- one token
def run_decode(lens, Hkv, G, page, dtype, n_sink=0, window=-1, listed=None, cache=None, seed=0, lengths=None):
    S = len(lens)
    c = cache or Cache(lens, Hkv, page, dtype, seed, DEV)
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn(S, Hkv * G, D, generator=g) * 1.5).to(dtype)
    out = torch.full((S, Hkv * G, D), float("nan"), dtype=dtype, device=DEV)
    kw = {}
    if listed is not None:
        kw = dict(token_idx=i32(listed[0]), n_tokens=i32(listed[1]))
    ck.ck_paged_decode_attn(shape(S, Hkv, G, dtype), q.to(DEV), c.kv(), i32(lens if lengths is None else lengths), out,
                            n_sink=n_sink, window=window, **kw)
    torch.cuda.synchronize()
    for s, n in enumerate(lens):
        for h in range(Hkv):
            seen = seen_rows(n, n - 1, n_sink, window).astype(np.float64)
            if listed is not None:
                idx = listed[0][s][h][:max(0, min(listed[1][s][h], len(listed[0][s][h])))]
                for r in idx:
                    if 0 <= r < n:
                        seen[r] += 1
            if n:
                seen = seen * c.there(s)
            want, tol = attend(q[s, h * G:(h + 1) * G], c.rows_k[s][h], c.rows_v[s][h], np.tile(seen, (G, 1)), dtype,
                               p_step=2.0 ** -15 if dtype is BF else 0.0)
            close(out[s, h * G:(h + 1) * G], want, tol, f"sequence {s} head {h}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("lens,page", [([1], 1), ([0, 1, 2], 16), ([15, 16, 17, 63, 64, 65], 7), ([257, 0, 1000], 40),
                                       ([129, 128, 130], 64)])
def test_decode_whole(lens, page, G, dtype):
    run_decode(lens, 2, G, page, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n_sink,window", [(0, 0), (3, 0), (0, 1), (4, 1), (70, 33), (5, 64), (10, 10 ** 6), (1000, 7),
                                           (10 ** 9, 10 ** 9)])
def test_decode_window_and_sinks(n_sink, window, dtype):
    run_decode([0, 1, 5, 64, 100, 333], 2, 4, 24, dtype, n_sink, window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n_sink,window", [(0, 0), (4, 9)])
def test_decode_lists(n_sink, window, dtype):
    lens, Hkv, rng = [1, 40, 500, 1200], 2, np.random.default_rng(5)
    idx, n = [], []
    for length in lens:
        heads = []
        for _ in range(Hkv):
            v = rng.integers(0, length, 120)
            v[::7] = rng.choice([-1, length, 2 ** 31 - 1, -2 ** 31], v[::7].size)     # no rows of the sequence
            heads.append(v.tolist())
        idx.append(heads)
    n = [[0, 120], [-5, 1], [119, 2 ** 31 - 1], [64, 65]]
    run_decode(lens, Hkv, 4, 33, dtype, n_sink, window, (idx, n))


def test_decode_more_sequences_than_lanes():
    lens = [(7 * s) % 97 for s in range(131)]
    run_decode(lens, 1, 2, 16, BF)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decode_long_ragged(dtype):
    # pieces of several hundred rows, and sequences of one piece beside them
    run_decode([40003, 17, 9000, 0, 12345], 1, 4, 64, dtype)


def test_decode_ragged_batches_that_fit_with_longer_pieces():
    # at an even share the sequences would be cut into more pieces than run at once: longer ones are tried, for batches
    # of fewer and of more sequences than lanes
    run_decode([(s * 37) % 2000 + 1 for s in range(200)], 1, 2, 64, BF)
    run_decode([(s * 379) % 4000 + 1 for s in range(40)], 8, 1, 64, BF)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G", [1, 8])
@pytest.mark.parametrize("lens", [[2241], [2049, 64, 191], [9001], [33000]])
def test_decode_pieces_joined_in_stages(lens, G, dtype):
    """17, 16, 70 and 256 pieces of one head-problem, whose last may be longer or short; some hold an infinite value,
    and a workspace of any contents."""
    c = Cache(lens, 1, 32, dtype, 21, DEV)
    n = lens[0]
    for r in (3, n - 2):
        v = c.rows_v[0][0, r].clone()
        v[5] = math.inf
        c.write(0, 0, r, v=v)
    q = (torch.randn(len(lens), G, D, generator=torch.Generator().manual_seed(4)) * 0.2).to(dtype)
    out = torch.empty(len(lens), G, D, dtype=dtype, device=DEV)
    sh = shape(len(lens), 1, G, dtype)
    ws = ck.paged_decode_workspace(sh, DEV)
    ws.random_(0, 256)
    again = torch.empty_like(out)
    ck.ck_paged_decode_attn(sh, q.to(DEV), c.kv(), i32(lens), out, workspace=ws)
    ck.ck_paged_decode_attn(sh, q.to(DEV), c.kv(), i32(lens), again, workspace=ws)
    assert torch.equal(out, again)
    assert (out[0, :, 5] == math.inf).all()
    out[0, :, 5] = 0.0
    for s, m in enumerate(lens):
        v = c.rows_v[s][0].clone()
        v[torch.isinf(v)] = 0.0
        if s == 0:
            v[:, 5] = 0.0
        want, tol = attend(q[s], c.rows_k[s][0], v, np.ones((G, m)), dtype, p_step=2.0 ** -15 if dtype is BF else 0.0)
        close(out[s], want, tol, f"sequence {s}")


def test_decode_many_head_problems():
    # more head-problems than pieces
    run_decode([33] * 70, 8, 1, 32, BF)


def test_decode_pages_that_are_gone():
    c = Cache([300, 200], 2, 16, BF, 3, DEV)
    c.table[0, 2:9] = torch.tensor([-1, c.K.shape[0], -2 ** 31, 2 ** 31 - 1, -1, -1, -7])
    c.table[1, :] = -1                                   # nothing left at all
    run_decode([300, 200], 2, 4, 16, BF, cache=c)
    run_decode([300, 200], 2, 4, 16, BF, 20, 150, cache=c)
    run_decode([300, 200], 2, 4, 16, BF, 4, 50, cache=c, listed=([[[40, 2, 100, 299]] * 2] * 2, [[4, 3]] * 2))


def test_decode_pages_in_common_and_lengths_beyond_the_table():
    c = Cache([96, 80], 2, 16, BF, 4, DEV)
    c.table = c.table[:, :5].contiguous()                # sequence 0 ends at row 80 now
    c.lens[0] = 80
    c.rows_k[0], c.rows_v[0] = c.rows_k[0][:, :80], c.rows_v[0][:, :80]
    c.table[1, :3] = c.table[0, :3]                      # the first 48 rows are the same
    for rows in (c.rows_k, c.rows_v):
        rows[1][:, :48] = rows[0][:, :48]
    run_decode([80, 80], 2, 4, 16, BF, cache=c, lengths=[96, 2 ** 31 - 1])
    run_decode([0, 0], 2, 4, 16, BF, lengths=[-1, -2 ** 31])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decode_infinite_values_and_scores(dtype):
    """An infinite value reaches the channels of the queries that see it, as an infinity; what is not attended
    may hold anything."""
    c = Cache([200], 1, 16, dtype, 6, DEV)
    v = c.rows_v[0][0, 190].clone()
    v[3], v[5] = math.inf, -math.inf
    c.write(0, 0, 190, v=v)
    c.write(0, 0, 100, k=torch.full((D,), math.nan), v=torch.full((D,), math.inf))
    q = (torch.randn(1, 4, D, generator=torch.Generator().manual_seed(1)) * 0.2).to(dtype)
    out = torch.empty(1, 4, D, dtype=dtype, device=DEV)
    ck.ck_paged_decode_attn(shape(1, 1, 4, dtype), q.to(DEV), c.kv(), i32([200]), out, n_sink=16, window=50)
    o = out[0].float().cpu()
    assert (o[:, 3] == math.inf).all() and (o[:, 5] == -math.inf).all()
    keep = [j for j in range(D) if j not in (3, 5)]
    want, tol = attend(q[0], c.rows_k[0][0], torch.nan_to_num(c.rows_v[0][0], posinf=0, neginf=0),
                       np.tile(seen_rows(200, 199, 16, 50), (4, 1)), dtype, p_step=2.0 ** -15)
    close(out[0][:, keep], want[:, keep], tol[:, keep], "the other channels")


def test_decode_scores_far_apart():
    """One row outweighs all others by more than fp32 can hold, the row before it by e^30."""
    c = Cache([500], 1, 16, BF, 7, DEV)
    q = torch.ones(1, 1, D).to(BF)
    c.write(0, 0, 17, k=torch.full((D,), 100.0))
    c.write(0, 0, 400, k=torch.full((D,), 97.0))
    out = torch.empty(1, 1, D, dtype=BF, device=DEV)
    ck.ck_paged_decode_attn(shape(1, 1, 1), q.to(DEV), c.kv(), i32([500]), out)
    close(out[0], c.rows_v[0][0, 17].double().numpy()[None], 2 ** -8 * np.abs(c.rows_v[0][0, 17].double().numpy())[None]
          + 1e-12, "the heaviest row")


def test_decode_runs_twice_the_same_and_from_a_graph():
    """Bit-equal from run to run; a captured call replays with the lengths and tables of that time, eager calls on
    the same workspace between the replays."""
    lens, Hkv, G = [3000, 64, 1, 700], 2, 4
    c = Cache(lens, Hkv, 16, BF, 8, DEV)
    sh, kv = shape(4, Hkv, G), c.kv()
    q = torch.randn(4, Hkv * G, D, device=DEV).to(BF)
    n, out, ws = i32(lens), torch.empty_like(q), ck.paged_decode_workspace(sh, DEV)
    ws.random_(0, 256)                                   # whatever the memory held
    ck.ck_paged_decode_attn(sh, q, kv, n, out, workspace=ws)
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ck.ck_paged_decode_attn(sh, q, kv, n, out, workspace=ws)
    second, other = torch.cuda.CUDAGraph(), torch.empty_like(out)
    with torch.cuda.graph(second):
        ck.ck_paged_decode_attn(sh, q, kv, n, other, n_sink=4, window=100, workspace=ws)
    for new in (lens, [3000, 3, 0, 650], [17, 64, 1, 700], lens):
        n.copy_(i32(new))
        out.fill_(float("nan"))
        graph.replay()
        second.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(out)
        ck.ck_paged_decode_attn(sh, q, kv, n, want, workspace=ws)
        assert torch.equal(out, want)
        ck.ck_paged_decode_attn(sh, q, kv, n, want, n_sink=4, window=100)
        assert torch.equal(other, want)
    assert torch.equal(out, first)


def test_decode_on_another_stream():
    lens = [2000, 30]
    c = Cache(lens, 2, 16, BF, 9, DEV)
    sh, kv, q = shape(2, 2, 4), c.kv(), torch.randn(2, 8, D, device=DEV).to(BF)
    want, got, n = torch.empty_like(q), torch.empty_like(q), i32(lens)
    ck.ck_paged_decode_attn(sh, q, kv, n, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ck.ck_paged_decode_attn(sh, q, kv, n, got)
    side.synchronize()
    assert torch.equal(got, want)


def test_decode_equals_attention_over_the_contiguous_cache():
    """A contiguous cache is a cache of one page for each sequence: the same rows as ck_full_decode_attn."""
    S, Hkv, G, N = 2, 2, 4, 1500
    K, V = (torch.randn(S, Hkv, N, D, device=DEV).to(BF) for _ in range(2))
    q = torch.randn(S, Hkv * G, D, device=DEV).to(BF)
    full, got = torch.empty_like(q), torch.empty_like(q)
    ck.ck_full_decode_attn(ck.Shape(S, Hkv * G, Hkv, N, 1), q, K, V, 1400, full)
    ck.ck_paged_decode_attn(shape(S, Hkv, G), q, ck.PagedKV(K, V), i32([1400, 1400]), got)
    a, b = full.float(), got.float()
    assert ((a - b).abs() <= 2 ** -7 * a.abs() + 1e-5).all()          # one step of the type, and fp32 orders


# ---------------------------------------------------------------- prompts
def run_prompt(lens, news, Hkv, G, page, n_sink=0, window=-1, cache=None, seed=0, pad=0, before=0, qscale=1.5):
    S = len(lens)
    c = cache or Cache(lens, Hkv, page, BF, seed, DEV)
    starts = (before + np.concatenate([[0], np.cumsum(news)])).tolist()
    T = starts[-1] + pad
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn(max(T, 1), Hkv * G, D, generator=g) * qscale).to(BF)
    q[:before] = math.nan
    q[starts[-1]:] = math.nan
    out = torch.full((max(T, 1), Hkv * G, D), 123.0, dtype=BF, device=DEV)
    ck.ck_prompt_attn(shape(S, Hkv, G), q.to(DEV), i32(starts), c.kv(), i32(lens), out, n_sink=n_sink, window=window)
    torch.cuda.synchronize()
    assert (out[:before] == 123.0).all() and (out[starts[-1]:] == 123.0).all()
    for s, (n, m) in enumerate(zip(lens, news)):
        if not m:
            continue
        seen = np.stack([seen_rows(n, n - m + i, n_sink, window) for i in range(m)])
        if n:
            seen = seen & c.there(s)[None]
        for h in range(Hkv):
            qs = q[starts[s]:starts[s + 1], h * G:(h + 1) * G].reshape(m * G, D)
            want, tol = attend(qs, c.rows_k[s][h], c.rows_v[s][h], seen.repeat(G, 0), BF, p_step=2.0 ** -8)
            close(out[starts[s]:starts[s + 1], h * G:(h + 1) * G].reshape(m * G, D), want, tol,
                  f"sequence {s} head {h}")


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("lens,news,page", [([1], [1], 1), ([1, 2, 3], [1, 2, 3], 16), ([64], [64], 64),
                                            ([65, 63, 130], [65, 1, 130], 7), ([200, 0, 300], [17, 0, 33], 40),
                                            ([257], [129], 32), ([100, 90], [0, 90], 256)])
def test_prompt_whole(lens, news, page, G):
    run_prompt(lens, news, 2, G, page)


@pytest.mark.parametrize("n_sink,window", [(0, 0), (3, 0), (0, 1), (4, 1), (70, 33), (64, 64), (5, 64), (10, 10 ** 6),
                                           (1000, 7), (130, 65), (0, 129)])
def test_prompt_window_and_sinks(n_sink, window):
    run_prompt([5, 64, 333, 400], [5, 1, 333, 150], 2, 4, 24, n_sink, window)


@pytest.mark.parametrize("G,page,n_sink,window", [(1, 16, 0, 5), (1, 20, 0, 130), (2, 64, 0, 64), (1, 16, 70, 3),
                                                  (2, 9, 3, 200)])
def test_prompt_blocks_of_many_tokens_and_short_windows(G, page, n_sink, window):
    """Wavefronts of one workgroup see different tiles, some none of those at the begin, at the end or between."""
    run_prompt([900, 777], [700, 333], 1, G, page, n_sink, window)


@pytest.mark.parametrize("n_sink,window", [(0, 3), (2, 100), (0, -1), (5, 0)])
@pytest.mark.parametrize("G", [1, 8])
def test_prompt_masks_row_by_row(n_sink, window, G):
    """Equal scores and values that are one in a single channel: an output is the number of rows seen with that
    channel over the number of rows seen, so that a row too many or too few shows."""
    n, m = 300, 140
    c = Cache([n], 1, 20, BF, 0, DEV)
    for r in range(n):
        c.write(0, 0, r, v=torch.eye(D)[r % D])
    run_prompt([n], [m], 1, G, 20, n_sink, window, cache=c, qscale=0.0)


def test_prompt_rows_outside_the_sequences_are_left():
    run_prompt([70, 20], [70, 3], 2, 4, 16, pad=9, before=5)


def test_prompt_more_new_tokens_than_rows():
    """The first of them are before row 0 of the cache: they see nothing and give zeros."""
    run_prompt([3, 70], [10, 70], 1, 4, 16)


def test_prompt_more_sequences_than_lanes():
    lens = [1 + (7 * s) % 41 for s in range(131)]
    run_prompt(lens, [min(n, 1 + s % 5) for s, n in enumerate(lens)], 1, 2, 16)


def test_prompt_few_tokens_after_long_contexts():
    run_prompt([5000, 2100, 64], [3, 1, 5], 2, 4, 32)
    run_prompt([5000, 2100, 64], [3, 1, 5], 2, 4, 9, 16, 3000)


def test_prompt_pages_that_are_gone():
    c = Cache([300, 200], 2, 16, BF, 3, DEV)
    c.table[0, 2:9] = torch.tensor([-1, c.K.shape[0], -2 ** 31, 2 ** 31 - 1, -1, -1, -7])
    c.table[1, :] = -1
    run_prompt([300, 200], [300, 20], 2, 4, 16, cache=c)
    run_prompt([300, 200], [250, 20], 2, 4, 16, 20, 150, cache=c)


@pytest.mark.parametrize("window", [-1, 40])
def test_prompt_values_that_are_not_finite_reach_only_who_sees_them(window):
    n = 150
    c = Cache([n], 1, 16, BF, 6, DEV)
    for r, j, x in ((100, 3, math.inf), (30, 5, -math.inf), (70, 7, math.nan), (149, 9, math.inf)):
        v = c.rows_v[0][0, r].clone()
        v[j] = x
        c.write(0, 0, r, v=v)
    q = (torch.randn(n, 2, D, generator=torch.Generator().manual_seed(1)) * 0.2).to(BF)
    out = torch.empty(n, 2, D, dtype=BF, device=DEV)
    ck.ck_prompt_attn(shape(1, 1, 2), q.to(DEV), i32([0, n]), c.kv(), i32([n]), out, window=window)
    got = out.float().cpu()
    clean = torch.nan_to_num(c.rows_v[0][0], nan=0.0, posinf=0.0, neginf=0.0)
    seen = np.stack([seen_rows(n, p, 0, window) for p in range(n)])
    want, tol = attend(q.reshape(2 * n, D), c.rows_k[0][0], clean, seen.repeat(2, 0), BF, p_step=2.0 ** -8)
    ok = np.ones((n, D), dtype=bool)
    for r, j in ((100, 3), (30, 5), (70, 7), (149, 9)):
        ok[seen[:, r], j] = False
    ok = np.repeat(ok, 2, 0)
    flat = got.reshape(2 * n, D).double().numpy()
    assert np.isfinite(flat[ok]).all()
    assert (np.abs(flat - want) <= tol)[ok].all()
    for r, j, x in ((100, 3, math.inf), (30, 5, -math.inf), (149, 9, math.inf)):
        assert (flat[np.repeat(seen[:, r], 2), j] == x).all()
    assert np.isnan(flat[np.repeat(seen[:, 70], 2), 7]).all()


def test_prompt_keys_that_are_not_finite_in_masked_rows():
    n = 100
    c = Cache([n], 1, 16, BF, 6, DEV)
    c.write(0, 0, 99, k=torch.full((D,), math.nan))
    c.write(0, 0, 10, k=torch.full((D,), math.inf))
    q = torch.randn(n, 1, D, generator=torch.Generator().manual_seed(1)).to(BF)
    out = torch.empty(n, 1, D, dtype=BF, device=DEV)
    ck.ck_prompt_attn(shape(1, 1, 1), q.to(DEV), i32([0, n]), c.kv(), i32([n]), out, n_sink=0, window=20)
    sees_none = [p for p in range(n) if not (p >= 99 or 10 <= p < 30)]
    k = torch.nan_to_num(c.rows_k[0][0], nan=0.0, posinf=0.0)
    want, tol = attend(q[sees_none, 0], k, c.rows_v[0][0], np.stack([seen_rows(n, p, 0, 20) for p in sees_none]), BF,
                       p_step=2.0 ** -8)
    close(out[sees_none, 0], want, tol, "queries that do not see them")


@pytest.mark.parametrize("page,window", [(16, -1), (16, 2900), (12, -1), (12, 2900)])
@pytest.mark.parametrize("n,m", [(3000, 3), (1000, 40)])
def test_prompt_few_queries_and_values_that_are_not_finite(n, m, page, window):
    """Pieces of one block, most of whose wavefronts have no query but bring rows: infinite values that every query
    sees, that the last one sees, that none sees, and a page that is gone."""
    c = Cache([n], 1, page, BF, 11, DEV)
    last = n - 1                                        # only the last token sees it
    for r, j, x in ((n // 2, 3, math.inf), (last, 9, -math.inf), (n - m - 1, 5, math.inf), (0, 7, math.nan)):
        v = c.rows_v[0][0, r].clone()
        v[j] = x
        c.write(0, 0, r, v=v)
    hole = (n // 2 + 3 * page) // page                  # its rows: NaN in the pool, -1 in the table
    for r in range(hole * page, (hole + 1) * page):
        c.write(0, 0, r, k=torch.full((D,), math.nan), v=torch.full((D,), math.nan))
    c.table[0, hole] = -1
    G = 4
    q = (torch.randn(m, G, D, generator=torch.Generator().manual_seed(1)) * 0.2).to(BF)
    out = torch.empty(m, G, D, dtype=BF, device=DEV)
    ck.ck_prompt_attn(shape(1, 1, G), q.to(DEV), i32([0, m]), c.kv(), i32([n]), out, window=window)
    seen = np.stack([seen_rows(n, n - m + i, 0, window) for i in range(m)]) & c.there(0)[None]
    clean = [torch.nan_to_num(x[0][0], nan=0.0, posinf=0.0, neginf=0.0) for x in (c.rows_k, c.rows_v)]
    want, tol = attend(q.reshape(m * G, D), clean[0], clean[1], seen.repeat(G, 0), BF, p_step=2.0 ** -8)
    got = out.double().cpu().reshape(m * G, D).numpy()
    ok = np.ones((m, D), dtype=bool)
    for r, j in ((n // 2, 3), (last, 9), (n - m - 1, 5), (0, 7)):
        ok[seen[:, r], j] = False
    ok = ok.repeat(G, 0)
    assert np.isfinite(got[ok]).all() and (np.abs(got - want) <= tol)[ok].all()
    for r, j, x in ((n // 2, 3, math.inf), (last, 9, -math.inf), (n - m - 1, 5, math.inf)):
        assert (got[seen[:, r].repeat(G), j] == x).all()
    assert np.isnan(got[seen[:, 0].repeat(G), 7]).all()


def test_prompt_workspace_serves_fewer_rows():
    c = Cache([600], 1, 16, BF, 2, DEV)
    sh, kv = shape(1, 1, 2), c.kv()
    ws = ck.prompt_workspace(sh, 100000, DEV)
    for m in (1, 17, 600):
        q = torch.randn(m, 2, D, device=DEV).to(BF)
        a, b = torch.empty_like(q), torch.empty_like(q)
        ck.ck_prompt_attn(sh, q, i32([0, m]), kv, i32([600]), a, workspace=ws)
        ck.ck_prompt_attn(sh, q, i32([0, m]), kv, i32([600]), b)
        assert torch.equal(a, b)


def test_prompt_scores_far_apart_and_growing():
    """Maxima that grow from tile to tile, and one row that outweighs all."""
    n = 400
    c = Cache([n], 1, 16, BF, 7, DEV)
    for r in range(n):
        c.write(0, 0, r, k=torch.full((D,), 0.1 * r))
    q = torch.full((n, 1, D), 1.0).to(BF)
    out = torch.empty(n, 1, D, dtype=BF, device=DEV)
    ck.ck_prompt_attn(shape(1, 1, 1), q.to(DEV), i32([0, n]), c.kv(), i32([n]), out)
    seen = np.tril(np.ones((n, n)))
    want, tol = attend(q[:, 0], c.rows_k[0][0], c.rows_v[0][0], seen, BF, p_step=2.0 ** -8)
    close(out[:, 0], want, tol, "growing scores")
    ck.ck_prompt_attn(shape(1, 1, 1), (-q).to(DEV), i32([0, n]), c.kv(), i32([n]), out)
    want, tol = attend(-q[:, 0], c.rows_k[0][0], c.rows_v[0][0], seen, BF, p_step=2.0 ** -8)
    close(out[:, 0], want, tol, "falling scores")


@pytest.mark.parametrize("n_sink,window", [(0, -1), (0, 70), (3, 40)])
@pytest.mark.parametrize("level", [-50.0, 50.0])
def test_prompt_scores_far_from_zero(level, n_sink, window):
    """All scores near 565 or -565, and queries that see nothing of their first tiles."""
    n, m = 400, 300
    c = Cache([n], 1, 16, BF, 9, DEV)
    for r in range(n):
        c.write(0, 0, r, k=torch.full((D,), level * (1 + r % 3 / 64)))
    q = torch.ones(m, 1, D, dtype=BF)
    out = torch.empty(m, 1, D, dtype=BF, device=DEV)
    ck.ck_prompt_attn(shape(1, 1, 1), q.to(DEV), i32([0, m]), c.kv(), i32([n]), out, n_sink=n_sink, window=window)
    seen = np.stack([seen_rows(n, n - m + i, n_sink, window) for i in range(m)])
    want, tol = attend(q[:, 0], c.rows_k[0][0], c.rows_v[0][0], seen, BF, p_step=2.0 ** -8)
    close(out[:, 0], want, tol, "scores far from zero")


def test_prompt_long_runs_twice_the_same_and_from_a_graph():
    lens, news, Hkv, G = [1500, 700], [1500, 300], 2, 4
    c = Cache(lens, Hkv, 64, BF, 8, DEV)
    sh, kv = shape(2, Hkv, G), c.kv()
    q = torch.randn(1800, Hkv * G, D, device=DEV).to(BF)
    starts, n, out = i32([0, 1500, 1800]), i32(lens), torch.empty_like(q)
    ws = ck.prompt_workspace(sh, 1800, DEV)
    ws.random_(0, 256)
    ck.ck_prompt_attn(sh, q, starts, kv, n, out, workspace=ws)
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ck.ck_prompt_attn(sh, q, starts, kv, n, out, workspace=ws)
    for new, at in ((lens, [0, 1500, 1800]), ([1500, 9], [0, 1791, 1800]), ([64, 700], [0, 0, 700]),
                    (lens, [0, 1500, 1800])):
        n.copy_(i32(new))
        starts.copy_(i32(at))
        out.fill_(123.0)
        graph.replay()
        torch.cuda.synchronize()
        want = torch.full_like(out, 123.0)
        ck.ck_prompt_attn(sh, q, starts, kv, n, want)
        assert torch.equal(out, want)
    assert torch.equal(out, first)


def test_prompt_of_one_token_equals_decode():
    lens = [1, 64, 777]
    c = Cache(lens, 2, 16, BF, 5, DEV)
    q = torch.randn(3, 8, D, device=DEV).to(BF)
    a, b = torch.empty_like(q), torch.empty_like(q)
    for n_sink, window in ((0, -1), (4, 100)):
        ck.ck_prompt_attn(shape(3, 2, 4), q, i32([0, 1, 2, 3]), c.kv(), i32(lens), a, n_sink=n_sink, window=window)
        ck.ck_paged_decode_attn(shape(3, 2, 4), q, c.kv(), i32(lens), b, n_sink=n_sink, window=window)
        # probabilities rounded to bf16 on one side: 2^-8 of what they add up to
        assert ((a.float() - b.float()).abs() <= 2 ** -7 * b.float().abs() + 2 ** -8 * 3.0).all()


# ---------------------------------------------------------------- rotary append
def run_rope(lens, news, Hkv, G, page, dtype, rot=128, adjacent=False, factor=1.0, positions=None, pad=0, before=0,
             in_place=False, fused=True, with_q=True, cache=None):
    S = len(lens)
    c = cache or Cache(lens, Hkv, page, dtype, 3, DEV)
    kv = c.kv()
    K0, V0 = kv.K.clone(), kv.V.clone()
    starts = None
    T = S
    if news is not None:
        starts = (before + np.concatenate([[0], np.cumsum(news)])).tolist()
        T = max(1, starts[-1] + pad)
    Hq = Hkv * G
    g = torch.Generator().manual_seed(11)
    x = torch.randn(T, (Hq + 2 * Hkv) * D, generator=g).to(dtype)
    q, k, v = (t.unflatten(1, (-1, D)) for t in x.split([Hq * D, Hkv * D, Hkv * D], 1))
    if fused:
        dx = x.to(DEV)
        dq, dk, dv = (t.unflatten(1, (-1, D)) for t in dx.split([Hq * D, Hkv * D, Hkv * D], 1))
    else:
        dq, dk, dv = (t.contiguous().to(DEV) for t in (q, k, v))
    freqs = ck.ck_rope_frequencies(ck.CK_ROPE_PLAIN, rot)[0]
    out = dq if in_place else torch.full((T, Hq, D), 123.0, dtype=dtype, device=DEV)
    keep = out.clone()
    ck.ck_rope_append(shape(S, Hkv, G, dtype), dq if with_q else None, dk, dv, kv, i32(lens), freqs.to(DEV),
                      out if with_q else None, q_starts=None if starts is None else i32(starts),
                      positions=None if positions is None else i32(positions), attn_factor=factor,
                      interleaved=adjacent)
    torch.cuda.synchronize()
    K, V = K0.cpu(), V0.cpu()                            # what the pools have to be
    tolK = torch.zeros(K.shape, dtype=torch.float64)
    K = K.double()
    used = np.zeros(T, dtype=bool)
    for s in range(S):
        m = 1 if news is None else news[s]
        for i in range(m):
            t = s if news is None else starts[s] + i
            used[t] = True
            row = lens[s] - m + i
            pos = row if positions is None else positions[t]
            if with_q:
                want, tol = turn(q[t], pos, freqs, factor, adjacent)
                close(out[t], want, tol, f"query {t}")
            if 0 <= row < c.table.shape[1] * page:
                p = int(c.table[s, row // page])
                if 0 <= p < K.shape[0]:
                    want, tol = turn(k[t], pos, freqs, factor, adjacent)
                    K[p, :, row % page] = torch.from_numpy(want)
                    tolK[p, :, row % page] = torch.from_numpy(tol)
                    V[p, :, row % page] = v[t]
    gotK = kv.K.cpu().double()
    assert ((gotK - K).abs() <= tolK)[~torch.isnan(K)].all()
    assert (torch.isnan(gotK) == torch.isnan(K)).all()
    bits = torch.int16 if dtype is BF else torch.int32
    assert torch.equal(kv.V.cpu().view(bits), V.view(bits))
    if with_q:
        assert torch.equal(out[~used], keep[~used])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("rot", [2, 6, 16, 48, 64, 74, 96, 126, 128])
def test_rope_parts_of_a_head(rot, adjacent, dtype):
    run_rope([1, 40, 7], None, 2, 4, 16, dtype, rot, adjacent)
    run_rope([30, 9], [13, 9], 1, 2, 7, dtype, rot, adjacent, factor=1.25)


@pytest.mark.parametrize("G,Hkv", [(1, 1), (8, 1), (1, 3), (2, 5), (4, 8)])
@pytest.mark.parametrize("fused", [False, True])
def test_rope_heads_and_strides(G, Hkv, fused):
    run_rope([5, 64, 2], [5, 0, 1], Hkv, G, 32, BF, fused=fused)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("rot", [128, 64, 74])
def test_rope_in_place(rot, adjacent):
    run_rope([9, 3], [9, 2], 2, 4, 16, BF, rot, adjacent, in_place=True, fused=False)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rope_far_positions(dtype):
    run_rope([3, 4], [3, 4], 1, 2, 16, dtype, positions=[0, 1, 131071, 1000003, 2 ** 31 - 1, 16777217, 5])


def test_rope_rows_outside_the_sequences_are_left():
    run_rope([40, 9], [30, 4], 2, 2, 16, BF, pad=7, before=3)


def test_rope_without_queries():
    run_rope([4, 9], [4, 2], 2, 2, 16, BF, with_q=False)


def test_rope_rows_that_the_table_does_not_have():
    """More new tokens than rows, lengths behind the table, pages that are gone: nothing is stored there."""
    c = Cache([40, 40, 40], 1, 8, BF, 3, DEV)
    c.table = c.table[:, :5].contiguous()
    c.table[1, 4] = -1
    c.table[2, 4] = c.K.shape[0]
    run_rope([3, 40, 40], [9, 12, 4], 1, 2, 8, BF, cache=c)
    run_rope([43, 40, 2 ** 31 - 1], [9, 0, 4], 1, 2, 8, BF, cache=c)
    run_rope([0, -5, 41], None, 1, 2, 8, BF, cache=c)


def test_rope_more_sequences_than_lanes():
    lens = [1 + (5 * s) % 23 for s in range(300)]
    run_rope(lens, [s % 3 if s % 3 <= n else n for s, n in enumerate(lens)], 1, 1, 16, BF)
    run_rope(lens, None, 1, 1, 16, BF)


def test_rope_special_values_pass():
    """Channels that do not turn, and values, keep their bits: infinities, NaN of any kind, negative zero."""
    k = torch.zeros(1, 1, D, dtype=BF)
    k[..., 100:] = torch.tensor([math.inf, -math.inf, math.nan, -0.0]).repeat(7)
    k.view(torch.int16)[0, 0, 127] = 0x7F81              # a signalling NaN
    v = k.roll(37, -1).contiguous()
    for rot in (64, 74, 96):
        c = Cache([1], 1, 4, BF, 0, DEV)
        kv = c.kv()
        ck.ck_rope_append(shape(1, 1, 1), None, k.to(DEV), v.to(DEV), kv, i32([1]),
                          ck.ck_rope_frequencies(0, rot)[0].to(DEV), None, positions=i32([77]))
        p = int(c.table[0, 0])
        assert torch.equal(kv.K[p, 0, 0].cpu().view(torch.int16)[96:], k[0, 0].view(torch.int16)[96:])
        assert torch.equal(kv.V[p, 0, 0].cpu().view(torch.int16), v[0, 0].view(torch.int16))


def test_rope_from_a_graph():
    sh, c = shape(3, 2, 4), Cache([30, 31, 32], 2, 16, BF, 3, DEV)
    kv, freqs = c.kv(), ck.ck_rope_frequencies(0, 128)[0].to(DEV)
    q, k, v = (torch.randn(3, h, D, device=DEV).to(BF) for h in (8, 2, 2))
    n, out = i32([30, 31, 32]), torch.empty_like(q)
    ck.ck_rope_append(sh, q, k, v, kv, n, freqs, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ck.ck_rope_append(sh, q, k, v, kv, n, freqs, out)
    for new in ([1, 2, 3], [30, 7, 32], [16, 17, 15]):
        n.copy_(i32(new))
        graph.replay()
        torch.cuda.synchronize()
        other, want = c.kv(), torch.empty_like(out)
        ck.ck_rope_append(sh, q, k, v, other, n, freqs, want)
        assert torch.equal(out, want)
        for s, r in enumerate(new):
            p = int(c.table[s, (r - 1) // 16])
            assert torch.equal(kv.K[p, :, (r - 1) % 16], other.K[p, :, (r - 1) % 16])


# ---------------------------------------------------------------- row copies
def run_copy(src, dst, n_copy, most, kept=None, begin=None, seq=None, dtype=BF):
    """src, dst: Cache; checks the whole destination pool, bit by bit."""
    S, Hkv = dst.table.shape[0], dst.Hkv
    a, b = src.kv(), dst.kv()
    want = [t.clone().cpu() for t in (b.K, b.V)]
    ck.ck_copy_rows(shape(S, Hkv, 1, dtype), a, b, i32(n_copy), most, row_idx=None if kept is None else i32(kept),
                    begin=None if begin is None else i32(begin), src_seq=None if seq is None else i32(seq))
    torch.cuda.synchronize()

    def place(c, s, r):
        if not 0 <= s < c.table.shape[0] or not 0 <= r < c.table.shape[1] * c.page:
            return None
        p = int(c.table[s, r // c.page])
        return (p, r % c.page) if 0 <= p < c.K.shape[0] else None

    for s in range(S):
        for h in range(Hkv):
            for j in range(max(0, min(n_copy[s], most))):
                to = (0 if begin is None else begin[s]) + j
                at = place(src, s if seq is None else seq[s], to if kept is None else kept[s][h][j])
                to = place(dst, s, to)
                if at and to:
                    want[0][to[0], h, to[1]] = src.K[at[0], h, at[1]]
                    want[1][to[0], h, to[1]] = src.V[at[0], h, at[1]]
    bits = torch.int16 if dtype is BF else torch.int32
    assert torch.equal(b.K.cpu().view(bits), want[0].view(bits))
    assert torch.equal(b.V.cpu().view(bits), want[1].view(bits))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page,page2", [(16, 16), (7, 64), (64, 1), (33, 20)])
def test_copy_whole(page, page2, dtype):
    lens = [0, 1, 65, 130]
    run_copy(Cache(lens, 2, page, dtype, 1, DEV), Cache(lens, 2, page2, dtype, 2, DEV), lens, 130, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_copy_kept_rows(dtype):
    rng = np.random.default_rng(3)
    lens = [50, 300]
    kept = rng.integers(0, 50, (2, 3, 70))
    kept[1] = rng.integers(0, 300, (3, 70))
    kept[0, 0, :5] = [-1, 10 ** 9, 2 ** 31 - 1, -2 ** 31, 50]     # 50: a page that is none, or behind the table
    run_copy(Cache(lens, 3, 16, dtype, 1, DEV), Cache([64, 70], 3, 8, dtype, 2, DEV), [64, 70], 70, kept.tolist(),
             dtype=dtype)


def test_copy_forked_pages_and_counts_out_of_range():
    src = Cache([100, 40, 8], 2, 16, BF, 1, DEV)
    dst = Cache([100, 100, 48, 100], 2, 16, BF, 2, DEV)
    run_copy(src, dst, [4, 16, 99, -3], 16, begin=[96, 0, 32, 0], seq=[0, 1, 1, 0])
    run_copy(src, dst, [16, 16, 16, 16], 16, begin=[-8, 1000, 2 ** 31 - 1, -2 ** 31], seq=[0, 0, 0, 0])
    run_copy(src, dst, [16, 16, 16, 16], 16, begin=[0, 0, 0, 0], seq=[3, -1, 2 ** 31 - 1, 2])


def test_copy_within_one_pool():
    """A fork inside one pool: the new page of the second sequence gets the rows of the page it shared."""
    c = Cache([40, 0], 2, 16, BF, 1, DEV, spare=4)
    used = set(c.table[0, :3].tolist())
    fresh = [p for p in range(c.K.shape[0]) if p not in used][0]
    table = c.table.clone()
    table[1, :2], table[1, 2] = table[0, :2], fresh
    pool = c.kv()
    to = ck.PagedKV(pool.K, pool.V, table.to(DEV))
    ck.ck_copy_rows(shape(2, 2, 1), pool, to, i32([0, 8]), 16, begin=i32([0, 32]), src_seq=i32([0, 0]))
    old = int(c.table[0, 2])
    assert torch.equal(pool.K[fresh, :, :8], pool.K[old, :, :8]) and torch.equal(pool.V[fresh, :, :8], pool.V[old, :, :8])
    assert torch.isnan(pool.K[fresh, :, 8:]).all()


# ---------------------------------------------------------------- together
def test_pools_beyond_32_bit_offsets():
    """The same rows in a small pool and on the last pages of one of 5 GB: the same bits from every operator."""
    lens, Hkv, G, page = [200, 131], 2, 4, 64
    c = Cache(lens, Hkv, page, BF, 5, DEV, spare=0)
    small, sh = c.kv(), shape(2, Hkv, G)
    n_pages = 164000
    K = torch.empty(n_pages, Hkv, page, D, dtype=BF, device=DEV)
    assert K.numel() * 2 > 2 ** 32
    table = torch.where((c.table >= 0) & (c.table < c.K.shape[0]), c.table + n_pages - c.K.shape[0],
                        torch.tensor(-1, dtype=torch.int32)).to(DEV)
    big = ck.PagedKV(K, torch.empty_like(K), table)
    n = i32(lens)
    ck.ck_copy_rows(sh, small, big, n, 200)
    at = n_pages - c.K.shape[0]
    k = torch.randn(5, Hkv, D, device=DEV).to(BF)
    q = torch.randn(5, Hkv * G, D, device=DEV).to(BF)
    freqs = torch.ones(64, device=DEV) * 0.1
    for kv in (small, big):
        ck.ck_rope_append(sh, None, k, k, kv, n, freqs, None, q_starts=i32([0, 3, 5]))
    for s in range(2):
        for r in range(lens[s]):
            p = int(c.table[s, r // page])
            if r % 50 == 0 or r >= lens[s] - 3:
                assert torch.equal(big.K[at + p, :, r % page], small.K[p, :, r % page])
                assert torch.equal(big.V[at + p, :, r % page], small.V[p, :, r % page])
    outs = [[torch.empty_like(q), torch.empty_like(q[:2])] for _ in range(2)]
    for kv, (a, b) in zip((small, big), outs):
        ck.ck_prompt_attn(sh, q, i32([0, 3, 5]), kv, n, a)
        ck.ck_paged_decode_attn(sh, q[:2], kv, n, b)
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    back = ck.PagedKV(torch.zeros_like(small.K), torch.zeros_like(small.V), small.page_table)
    ck.ck_copy_rows(sh, big, back, n, 200)
    for s in range(2):
        p, r = int(c.table[s, (lens[s] - 1) // page]), (lens[s] - 1) % page
        assert torch.equal(back.V[p, :, :r + 1], small.V[p, :, :r + 1])


def test_tensors_on_another_device_are_refused(monkeypatch):
    """Host memory among device tensors, and a device that is not the current one, whose default stream has the
    same handle as the current one's."""
    c = Cache([20, 30], 2, 16, BF, 1, DEV)
    sh, kv, n = shape(2, 2, 4), c.kv(), i32([20, 30])
    x = torch.zeros(2, 8, D, dtype=BF, device=DEV)
    k, f, out = torch.zeros(2, 2, D, dtype=BF, device=DEV), torch.ones(64, device=DEV), torch.empty_like(x)
    host = ck.PagedKV(c.K, c.V, c.table)
    calls = [lambda **o: ck.ck_rope_append(sh, **{**dict(q=x, k=k, v=k, kv=kv, lengths=n, freqs=f, q_out=out), **o}),
             lambda **o: ck.ck_paged_decode_attn(sh, **{**dict(q=x, kv=kv, lengths=n, out=out), **o}),
             lambda **o: ck.ck_prompt_attn(sh, **{**dict(q=x, q_starts=i32([0, 1, 2]), kv=kv, lengths=n, out=out), **o})]
    for call in calls:
        for change in (dict(lengths=n.cpu()), dict(kv=host)):
            with pytest.raises(ValueError):
                call(**change)
    for change in (dict(freqs=f.cpu()), dict(v=k.cpu()), dict(q=x.cpu()), dict(q_out=out.cpu()),
                   dict(positions=n.cpu())):
        with pytest.raises(ValueError):
            calls[0](**change)
    for change in (dict(out=out.cpu()), dict(workspace=torch.zeros(1 << 21, dtype=torch.uint8))):
        for call in calls[1:]:
            with pytest.raises(ValueError):
                call(**change)
    with pytest.raises(ValueError):
        ck.ck_copy_rows(sh, kv, host, n, 4)
    with pytest.raises(ValueError):
        ck.ck_copy_rows(sh, kv, kv, n, 4, begin=n.cpu())
    with pytest.raises(ValueError):
        ck.PagedKV(c.K.to(DEV), c.V.to(DEV), c.table)
    monkeypatch.setattr(ck.binding, "_current_device", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        ck.ck_copy_rows(sh, kv, kv, n, 4)


def test_a_sequence_from_prompt_to_recalled_decode():
    """Prompts are turned and stored, attend, are moved to the contiguous form that clustering reads, and generated
    tokens recall their clusters from the pages: each step against the plain forms on what the steps before left."""
    S, Hkv, G, N, B, steps, page, C = 2, 2, 4, 400, 96, 3, 16, 8
    Hq, n_max = Hkv * G, 400 + 3
    c = Cache([n_max] * S, Hkv, page, BF, 21, DEV)
    kv, sh = c.kv(), shape(S, Hkv, G)
    kv.K.fill_(float("nan"))
    kv.V.fill_(float("nan"))
    freqs, af = ck.ck_rope_frequencies(ck.CK_ROPE_RAMP, 128, factor=4.0, trained_len=256.0, fast=32.0, slow=1.0)
    df = freqs.to(DEV)
    g = torch.Generator().manual_seed(2)
    x = torch.randn(S * N, (Hq + 2 * Hkv) * D, generator=g).to(BF)
    q, k, v = (t.unflatten(1, (-1, D)) for t in x.to(DEV).split([Hq * D, Hkv * D, Hkv * D], 1))
    starts, lengths = i32([0, N, 2 * N]), i32([N, N])
    qr, out = torch.empty(S * N, Hq, D, dtype=BF, device=DEV), torch.empty(S * N, Hq, D, dtype=BF, device=DEV)
    ck.ck_rope_append(sh, q, k, v, kv, lengths, df, qr, q_starts=starts, attn_factor=af)
    ck.ck_prompt_attn(sh, qr, starts, kv, lengths, out)

    # the contiguous form, clustering on it
    flat = ck.PagedKV(torch.zeros(S, Hkv, n_max, D, dtype=BF, device=DEV), torch.zeros(S, Hkv, n_max, D, dtype=BF, device=DEV))
    ck.ck_copy_rows(sh, kv, flat, lengths, N)
    csh = ck.Shape(S, Hq, Hkv, n_max, C)
    st = ck.ClusterState(csh, DEV, budget=B)
    init = torch.stack([torch.randperm(N - 4, generator=g)[:C] + 4 for _ in range(S * Hkv)])
    st.cluster(flat.K, init.view(S, Hkv, C).to(torch.int32).to(DEV), 4, N - 4, C, 5)
    K, V = flat.K.cpu(), flat.V.cpu()
    for s in range(S):
        qk = turn(k[s * N + 7].cpu(), 7, freqs, af, False)
        assert (np.abs(K[s, :, 7].double().numpy() - qk[0]) <= qk[1]).all()
        for h in range(Hkv):
            rows = [0, 1, 100, N - 1]
            qs = qr[s * N:(s + 1) * N].cpu()[rows, h * G:(h + 1) * G].reshape(-1, D)
            seen = np.stack([seen_rows(N, p, 0, -1) for p in rows]).repeat(G, 0)
            want, tol = attend(qs, K[s, h, :N], V[s, h, :N], seen, BF, p_step=2.0 ** -8)
            close(out[s * N:(s + 1) * N][rows, h * G:(h + 1) * G].reshape(-1, D), want, tol, f"prompt {s} {h}")

    for t in range(steps):
        x = torch.randn(S, (Hq + 2 * Hkv) * D, generator=g).to(BF).to(DEV)
        q, k, v = (y.unflatten(1, (-1, D)) for y in x.split([Hq * D, Hkv * D, Hkv * D], 1))
        lengths = i32([N + t + 1] * S)
        qt, o = torch.empty(S, Hq, D, dtype=BF, device=DEV), torch.empty(S, Hq, D, dtype=BF, device=DEV)
        ck.ck_rope_append(sh, q, k, v, kv, lengths, df, qt, attn_factor=af)
        ck.ck_select_clusters(csh, qt, st.centroids, st.sizes, C, B, 0, st.sel_clusters, st.n_sel_clusters,
                              st.n_sel_tokens, st.scores)
        ck.ck_gather_indices(csh, st.sel_clusters, st.n_sel_clusters, st.offsets, st.sorted_idx, B, 0, st.token_idx,
                             st.n_tokens)
        ck.ck_paged_decode_attn(sh, qt, kv, lengths, o, n_sink=4, window=t + 1, token_idx=st.token_idx,
                                n_tokens=st.n_tokens)
        # the same step over a contiguous copy of the cache
        ck.ck_copy_rows(sh, kv, flat, lengths, n_max)
        want = torch.empty_like(o)
        ck.ck_sparse_decode_attn(csh, qt, flat.K, flat.V, st.token_idx, st.n_tokens, B, want, n_sink=4, recent_begin=N,
                                 recent_end=N + t + 1)
        a, b = want.float(), o.float()
        assert torch.isfinite(b).all() and ((a - b).abs() <= 2 ** -7 * a.abs() + 1e-4).all()
