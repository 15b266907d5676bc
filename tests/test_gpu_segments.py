"""Attention over rows that a batch shares and cross attention, against their formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2412_03213_amd as ck
from paged_ref import D, Cache, attend

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
P_STEP = {BF: 2.0 ** -8, F32: 0.0}                       # a probability enters a product as bf16


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def shape(S, Hkv, G, dtype=BF):
    return ck.Shape(S, Hkv * G, Hkv, 1, 1, dtype=ck.CK_BF16 if dtype is BF else ck.CK_F32)


def close(got, want, tol, what):
    got = got.detach().double().cpu().numpy()
    assert np.isfinite(got).all(), f"{what}: not finite"
    worst = (np.abs(got - want) - tol).max()
    assert worst <= 0, f"{what}: off by {np.abs(got - want).max():.3g}, {worst:.3g} more than allowed"


# Tables with room for short sequences are served by one launch; for long ones the work is planned, cut and joined.
FORMS = ["short", "long"]


def width_of(form, page, S=1, Hkv=1):
    """Entries of a table: none more than needed, or room for 5000 rows and 160 MB of a batch."""
    return 0 if form == "short" else max(5000, int(161e6 / (512 * S * Hkv))) // page + 1


# ---------------------------------------------------------------- cross attention
def run_cross(lens, news, Hkv, G, page, cache=None, seed=0, pad=0, before=0, qscale=1.5, form="short"):
    S = len(lens)
    c = cache or Cache(lens, Hkv, page, BF, seed, DEV, width=width_of(form, page))
    starts = (before + np.concatenate([[0], np.cumsum(news)])).tolist()
    T = max(1, starts[-1] + pad)
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn(T, Hkv * G, D, generator=g) * qscale).to(BF)
    q[:before] = math.nan
    q[starts[-1]:] = math.nan
    out = torch.full((T, Hkv * G, D), 123.0, dtype=BF, device=DEV)
    ck.ck_cross_attn(shape(S, Hkv, G), q.to(DEV), i32(starts), c.kv(), i32(lens), out)
    torch.cuda.synchronize()
    assert (out[:before] == 123.0).all() and (out[starts[-1]:] == 123.0).all()
    for s, (n, m) in enumerate(zip(lens, news)):
        if not m:
            continue
        seen = c.there(s) if n else np.zeros(0)
        for h in range(Hkv):
            qs = q[starts[s]:starts[s + 1], h * G:(h + 1) * G].reshape(m * G, D)
            want, tol = attend(qs, c.rows_k[s][h], c.rows_v[s][h], np.tile(seen, (m * G, 1)), BF, p_step=P_STEP[BF])
            close(out[starts[s]:starts[s + 1], h * G:(h + 1) * G].reshape(m * G, D), want, tol, f"sequence {s} head {h}")
    return out


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("lens,news,page", [([1], [1], 1), ([0, 1, 2], [3, 1, 2], 16), ([64], [64], 64),
                                            ([65, 63, 130], [1, 65, 9], 7), ([200, 0, 300], [17, 5, 0], 40),
                                            ([129], [300], 32), ([7, 1000], [40, 3], 256), ([0, 0], [1, 2], 8)])
def test_cross(lens, news, page, G, form):
    run_cross(lens, news, 2, G, page, form=form)


@pytest.mark.parametrize("Hkv,G", [(1, 1), (3, 2), (8, 4), (16, 1)])
@pytest.mark.parametrize("page", [24, 9])
def test_cross_heads_and_pieces(Hkv, G, page):
    # several pieces of each, blocks that are not full, a sequence whose only block has one token
    run_cross([2500, 300, 1], [30, 1, 5], Hkv, G, page, form="long")


@pytest.mark.parametrize("form", FORMS)
def test_cross_rows_outside_the_sequences_are_left(form):
    run_cross([700, 30], [9, 4], 2, 4, 16, pad=5, before=3, form=form)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("S", [131, 300, 1100])
def test_cross_more_sequences_than_lanes_and_threads(S, form):
    run_cross([(7 * s) % 197 for s in range(S)], [(3 * s) % 5 for s in range(S)], 1, 2, 16, form=form)


def test_cross_more_blocks_than_fit_and_a_long_sequence():
    run_cross([150, 9000, 70], [700, 2, 900], 8, 1, 64)


def test_cross_many_pieces_of_many_tokens():
    # 200 tokens of 4 heads are four blocks, each in several pieces
    run_cross([8000, 40], [200, 3], 1, 4, 32)


@pytest.mark.parametrize("form", FORMS)
def test_cross_large_scores(form):
    run_cross([700], [20], 1, 4, 32, qscale=40.0, form=form)
    run_cross([3000], [3], 1, 4, 32, qscale=40.0, form=form)


@pytest.mark.parametrize("form", FORMS)
def test_cross_pages_that_are_missing(form):
    lens = [500, 260]
    c = Cache(lens, 2, 16, BF, 5, DEV, width=width_of(form, 16))
    c.table[0, 3:9] = -1
    c.table[1, :] = 10 ** 6                                # nothing is left of it
    run_cross(lens, [20, 20], 2, 2, 16, cache=c)


@pytest.mark.parametrize("form", FORMS)
def test_cross_infinite_values_reach_every_query_of_their_sequence_only(form):
    lens = [700, 300]
    c = Cache(lens, 1, 24, BF, 6, DEV, width=width_of(form, 24))
    for s, r, ch in ((0, 3, 5), (0, 699, 7), (1, 299, 9)):
        v = c.rows_v[s][0, r].clone()
        v[ch] = math.inf
        c.write(s, 0, r, v=v)
    starts = [0, 11, 17]
    q = (torch.randn(17, 2, D, generator=torch.Generator().manual_seed(1)) * 0.1).to(BF)
    out = torch.empty(17, 2, D, dtype=BF, device=DEV)
    ck.ck_cross_attn(shape(2, 1, 2), q.to(DEV), i32(starts), c.kv(), i32(lens), out)
    inf = torch.isinf(out).cpu()
    want = torch.zeros_like(inf)
    want[:11, :, 5] = want[:11, :, 7] = want[11:, :, 9] = True
    assert torch.equal(inf, want) and not torch.isnan(out).any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_cross_one_token_for_each_sequence(dtype):
    """Without starts: the attention of single tokens."""
    lens, Hkv, G = [0, 1, 300, 2000], 2, 4
    c = Cache(lens, Hkv, 24, dtype, 3, DEV)
    q = (torch.randn(4, Hkv * G, D, generator=torch.Generator().manual_seed(2)) * 1.5).to(dtype).to(DEV)
    out, want = torch.empty_like(q), torch.empty_like(q)
    sh = shape(4, Hkv, G, dtype)
    ck.ck_cross_attn(sh, q, None, c.kv(), i32(lens), out)
    ck.ck_paged_decode_attn(sh, q, c.kv(), i32(lens), want)
    assert torch.equal(out, want)
    if dtype is BF:                                       # with starts, the same but for the roundings
        ck.ck_cross_attn(sh, q, i32([0, 1, 2, 3, 4]), c.kv(), i32(lens), out)
        for s, n in enumerate(lens):
            for h in range(Hkv):
                ref, tol = attend(q[s, h * G:(h + 1) * G].cpu(), c.rows_k[s][h], c.rows_v[s][h], np.ones((G, n)), BF,
                                  p_step=P_STEP[BF])
                close(out[s, h * G:(h + 1) * G], ref, tol, f"sequence {s} head {h}")


@pytest.mark.parametrize("form", FORMS)
def test_cross_twice_the_same_and_from_a_graph(form):
    """Bit-equal from run to run; two captured calls on one workspace replay with the lengths of that time."""
    lens, Hkv, G = [3000 if form == "long" else 700, 64, 650], 2, 4
    c = Cache(lens, Hkv, 16, BF, 8, DEV, width=width_of(form, 16))
    sh, kv, T = shape(3, Hkv, G), c.kv(), 341
    q = torch.randn(T, Hkv * G, D, device=DEV).to(BF)
    starts, n, out = i32([0, 40, 340, 341]), i32(lens), torch.empty_like(q)
    ws = ck.cross_workspace(sh, T, DEV)
    ws.random_(0, 256)                                   # whatever the memory held
    ck.ck_cross_attn(sh, q, starts, kv, n, out, workspace=ws)
    first = out.clone()
    graph, second, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph(), torch.empty_like(out)
    with torch.cuda.graph(graph):
        ck.ck_cross_attn(sh, q, starts, kv, n, out, workspace=ws)
    with torch.cuda.graph(second):
        ck.ck_cross_attn(sh, q, starts, kv, n, other, softmax_scale=0.05, workspace=ws)
    for new in (lens, [lens[0], 0, 600], [17, 64, 1], lens):
        n.copy_(i32(new))
        out.fill_(float("nan"))
        graph.replay()
        second.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(out)
        ck.ck_cross_attn(sh, q, starts, kv, n, want, workspace=ws)
        assert torch.equal(out, want)
        ck.ck_cross_attn(sh, q, starts, kv, n, want, softmax_scale=0.05)
        assert torch.equal(other, want)
    assert torch.equal(out, first)


# ---------------------------------------------------------------- rows that a batch shares
def shared_cache(groups, lens, shares, Hkv, page, dtype=BF, seed=0, form="long"):
    """A cache whose sequences [groups[g], groups[g + 1]) begin with the first one's rows, in its pages where whole ones
    are shared, whose own copies hold NaN."""
    c = Cache(lens, Hkv, page, dtype, seed, DEV, width=width_of(form, page, len(lens), Hkv))
    for a, b in zip(groups[:-1], groups[1:]):
        for s in range(a + 1, b):
            n = max(0, min(shares[s], lens[s]))
            assert n <= max(0, min(shares[a], lens[a]))
            for r in range(n):
                for h in range(Hkv):
                    c.rows_k[s][h, r], c.rows_v[s][h, r] = c.rows_k[a][h, r], c.rows_v[a][h, r]
                p = c.table[s, r // page]
                if r < n // page * page:
                    c.K[p, :, r % page] = math.nan
                    c.V[p, :, r % page] = math.nan
                else:
                    c.K[p, :, r % page], c.V[p, :, r % page] = c.rows_k[a][:, r], c.rows_v[a][:, r]
            c.table[s, :n // page] = c.table[a, :n // page]
    return c


def run_shared(groups, lens, shares, Hkv, G, page, dtype=BF, cache=None, seed=0, qscale=1.5, form="long"):
    S = len(lens)
    c = cache or shared_cache(groups, lens, shares, Hkv, page, dtype, seed, form)
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn(S, Hkv * G, D, generator=g) * qscale).to(dtype)
    out = torch.full((S, Hkv * G, D), float("nan"), dtype=dtype, device=DEV)
    ck.ck_shared_decode_attn(shape(S, Hkv, G, dtype), q.to(DEV), c.kv(), i32(lens), i32(groups), i32(shares), out)
    torch.cuda.synchronize()
    for s, n in enumerate(lens):
        seen = c.there(s) if n else np.zeros(0)
        for h in range(Hkv):
            want, tol = attend(q[s, h * G:(h + 1) * G], c.rows_k[s][h], c.rows_v[s][h], np.tile(seen, (G, 1)), dtype,
                               p_step=P_STEP[dtype])
            close(out[s, h * G:(h + 1) * G], want, tol, f"sequence {s} head {h}")


CASES = [
    ([0, 2], [1, 1], [0, 0]),                             # a row each, none shared
    ([0, 3], [5, 5, 5], [5, 5, 5]),                       # nothing but what is shared
    ([0, 3], [64, 65, 70], [64, 64, 64]),
    ([0, 4], [300, 130, 200, 129], [128, 128, 100, 7]),   # as far as each goes
    ([0, 1, 4], [90, 400, 401, 700], [90, 333, 333, 333]),
    ([1, 3], [50, 200, 260, 30], [50, 190, 190, 30]),     # the first and the last in no group: they share nothing
    ([0, 2, 2, 5], [10, 0, 500, 0, 501], [10, 0, 490, 490, 490]),   # empty sequences and an empty group
    ([0, 3], [40, 20, 10], [10 ** 9, 25, -7]),            # numbers that are no lengths
]


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("page", [16, 7])
@pytest.mark.parametrize("case", CASES)
def test_shared(case, page, G):
    groups, lens, shares = case
    run_shared(groups, lens, shares, 2, G, page)


@pytest.mark.parametrize("case", CASES)
def test_shared_little(case):
    groups, lens, shares = case
    run_shared(groups, lens, shares, 2, 4, 16, form="short")


@pytest.mark.parametrize("case", CASES[2:5])
def test_shared_in_fp32(case):
    groups, lens, shares = case
    run_shared(groups, lens, shares, 2, 4, 16, F32)
    run_shared(groups, lens, shares, 2, 4, 16, F32, form="short")


@pytest.mark.parametrize("Hkv,G", [(1, 8), (3, 4), (8, 2)])
def test_shared_long_rows_in_pieces(Hkv, G):
    lens = [5000 + 37 * s for s in range(5)] + [300, 20]
    run_shared([0, 5, 7], lens, [5000, 5000, 4000, 5000, 130, 17, 17], Hkv, G, 40)


def test_shared_more_queries_than_a_block():
    # 40 sequences of 8 heads are two blocks of one group
    lens = [700 + 5 * s for s in range(40)] + [9]
    run_shared([0, 40, 41], lens, [700 - s for s in range(40)] + [9], 1, 8, 32)


def test_shared_few_queries_that_see_different_numbers_of_shared_rows():
    # two sequences of four heads: as many queries as would stream the rows, were they the same for all
    run_shared([0, 2], [900, 700], [890, 500], 2, 4, 16)
    run_shared([0, 2], [900, 890], [890, 890], 2, 4, 16)


@pytest.mark.parametrize("S", [150, 600, 900])
def test_shared_more_sequences_and_groups_than_lanes_and_threads(S):
    lens = [100 + (s * 31) % 90 for s in range(S)]
    groups = list(range(0, S, 2)) + [S]
    run_shared(groups, lens, [90 if s % 2 == 0 else 71 for s in range(S)], 1, 2, 16)


def test_shared_large_scores():
    run_shared([0, 4], [900, 910, 920, 930], [900] * 4, 1, 4, 64, qscale=40.0)


def test_shared_equals_attention_of_each_sequence():
    """The same rows as the attention of single tokens, but for roundings."""
    lens, groups, shares = [800, 1500, 900, 400], [0, 4], [800, 800, 800, 400]
    c = shared_cache(groups, lens, shares, 2, 24, form="long")
    q = torch.randn(4, 8, D, device=DEV).to(BF)
    a, b, sh = torch.empty_like(q), torch.empty_like(q), shape(4, 2, 4)
    ck.ck_shared_decode_attn(sh, q, c.kv(), i32(lens), i32(groups), i32(shares), a)
    ck.ck_paged_decode_attn(sh, q, c.kv(), i32(lens), b)
    size = max(v.abs().max().item() for v in c.rows_v)
    # each is within half a step of its output and of its probabilities of the formula
    assert ((a.float() - b.float()).abs() <= 2 ** -7 * b.float().abs() + 2 ** -8 * size * 1.01).all()


def test_shared_infinite_values_reach_those_who_see_them():
    lens, shares, groups = [300, 400, 350], [256, 200, 256], [0, 3]
    c = shared_cache(groups, lens, shares, 1, 16)
    for s, r, ch in ((0, 3, 5), (0, 230, 7), (1, 399, 9)):  # shared by all; by the first and third; own
        v = c.rows_v[s][0, r].clone()
        v[ch] = math.inf
        c.write(s, 0, r, v=v)
    q = (torch.randn(3, 4, D, generator=torch.Generator().manual_seed(1)) * 0.1).to(BF)
    out = torch.empty(3, 4, D, dtype=BF, device=DEV)
    ck.ck_shared_decode_attn(shape(3, 1, 4), q.to(DEV), c.kv(), i32(lens), i32(groups), i32(shares), out)
    inf = torch.isinf(out).cpu()
    want = torch.zeros_like(inf)
    want[:, :, 5] = want[0, :, 7] = want[2, :, 7] = want[1, :, 9] = True
    assert torch.equal(inf, want) and not torch.isnan(out).any()


def test_shared_twice_the_same_and_from_a_graph():
    lens, groups, shares, Hkv, G = [3000, 3064, 3001, 700], [0, 3, 4], [2990, 2990, 2990, 700], 2, 4
    c = shared_cache(groups, lens, shares, Hkv, 16)
    sh, kv = shape(4, Hkv, G), c.kv()
    q = torch.randn(4, Hkv * G, D, device=DEV).to(BF)
    n, g, r, out = i32(lens), i32(groups), i32(shares), torch.empty_like(q)
    ws = ck.shared_decode_workspace(sh, DEV)
    ws.random_(0, 256)
    ck.ck_shared_decode_attn(sh, q, kv, n, g, r, out, workspace=ws)
    first = out.clone()
    graph, second, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph(), torch.empty_like(out)
    with torch.cuda.graph(graph):
        ck.ck_shared_decode_attn(sh, q, kv, n, g, r, out, workspace=ws)
    with torch.cuda.graph(second):
        ck.ck_shared_decode_attn(sh, q, kv, n, g, r, other, softmax_scale=0.05, workspace=ws)
    for new, rows in ((lens, shares), ([3000, 0, 10, 650], shares), (lens, [0, 0, 0, 0]), (lens, shares)):
        n.copy_(i32(new))
        r.copy_(i32(rows))
        out.fill_(float("nan"))
        graph.replay()
        second.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(out)
        ck.ck_shared_decode_attn(sh, q, kv, n, g, r, want, workspace=ws)
        assert torch.equal(out, want)
        ck.ck_shared_decode_attn(sh, q, kv, n, g, r, want, softmax_scale=0.05)
        assert torch.equal(other, want)
    assert torch.equal(out, first)


def test_on_another_stream():
    lens, groups, shares = [2000, 1990], [0, 2], [1900, 1900]
    c = shared_cache(groups, lens, shares, 2, 16)
    sh, kv, q = shape(2, 2, 4), c.kv(), torch.randn(2, 8, D, device=DEV).to(BF)
    args = (i32(lens), i32(groups), i32(shares))
    starts = i32([0, 1, 2])
    want, got = [torch.empty_like(q) for _ in range(2)], [torch.empty_like(q) for _ in range(2)]
    ck.ck_shared_decode_attn(sh, q, kv, *args, want[0])
    ck.ck_cross_attn(sh, q, starts, kv, args[0], want[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ck.ck_shared_decode_attn(sh, q, kv, *args, got[0])
        ck.ck_cross_attn(sh, q, starts, kv, args[0], got[1])
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_pools_beyond_32_bit_offsets():
    """Elements of the pool beyond 2^32: 2^25 + some rows of 128 channels."""
    Hkv, page, rows = 1, 64, 300
    n_pages = 2 ** 25 // page + 8
    K = torch.empty(n_pages, Hkv, page, D, dtype=BF, device=DEV)
    V = torch.empty_like(K)
    table = torch.arange(n_pages - 8, n_pages, dtype=torch.int32, device=DEV)[None, :].expand(2, -1).contiguous()
    k, v = (torch.randn(rows, Hkv, D, device=DEV).to(BF) for _ in range(2))
    kv = ck.PagedKV(K, V, table)
    slots = (n_pages - 8) * page + torch.arange(rows, dtype=torch.int32, device=DEV)
    ck.ck_store_rows(shape(2, 1, 4), k, v, slots, kv)
    assert torch.equal(K[-8:, 0].reshape(-1, D)[:rows], k[:, 0]) and torch.equal(V[-8:, 0].reshape(-1, D)[:rows], v[:, 0])
    q = torch.randn(2, 4, D, device=DEV).to(BF)
    a, b = torch.empty_like(q), torch.empty_like(q)
    ck.ck_shared_decode_attn(shape(2, 1, 4), q, kv, i32([rows, rows]), i32([0, 2]), i32([290, 290]), a)
    ck.ck_cross_attn(shape(2, 1, 4), q, i32([0, 1, 2]), kv, i32([rows, rows]), b)
    for s in range(2):
        want, tol = attend(q[s].cpu(), k[:, 0].cpu(), v[:, 0].cpu(), np.ones((4, rows)), BF, p_step=P_STEP[BF])
        close(a[s], want, tol, f"shared {s}")
        close(b[s], want, tol, f"cross {s}")


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("lens,shares", [([64, 200, 130], [64, 90, 20]),      # the others share more than the first
                                         ([20, 200, 130], [100, 100, 100]),   # the first is shorter than its number
                                         ([0, 200, 7], [100, 100, 100])])     # ... and has no row at all
def test_shared_no_further_than_the_first_goes(lens, shares, form):
    """Rows that the first of a group does not share are read through each one's own table."""
    n = max(0, min(shares[0], lens[0]))
    groups, page = [0, 3], 16
    c = shared_cache(groups, lens, [min(x, n) for x in shares], 2, page, form=form)
    S, G = 3, 4
    q = (torch.randn(S, 2 * G, D, generator=torch.Generator().manual_seed(4)) * 1.5).to(BF)
    out = torch.full((S, 2 * G, D), float("nan"), dtype=BF, device=DEV)
    ck.ck_shared_decode_attn(shape(S, 2, G), q.to(DEV), c.kv(), i32(lens), i32(groups), i32(shares), out)
    for s, m in enumerate(lens):
        for h in range(2):
            want, tol = attend(q[s, h * G:(h + 1) * G], c.rows_k[s][h], c.rows_v[s][h], np.ones((G, m)), BF,
                               p_step=P_STEP[BF])
            close(out[s, h * G:(h + 1) * G], want, tol, f"sequence {s} head {h}")


@pytest.mark.parametrize("S", [9, 700])
def test_shared_groups_of_many_sizes_no_further_than_their_first(S):
    groups, s = [1], 1
    while s < S - 2:
        s = min(S - 2, s + 1 + len(groups) % 4)
        groups.append(s)
    lens = [40 + (s * 37) % 60 for s in range(S)]
    shares = [20 + (s * 13) % 70 for s in range(S)]
    real = list(shares)
    for a, b in zip(groups[:-1], groups[1:]):
        for s in range(a, b):
            real[s] = max(0, min(shares[s], shares[a], lens[a]))
    real[0] = real[-1] = real[-2] = 0
    c = shared_cache(groups, lens, real, 1, 16)
    run_shared(groups, lens, shares, 1, 2, 16, cache=c)


@pytest.mark.parametrize("S,page", [(40, 16), (64, 20)])
def test_cross_blocks_that_begin_in_the_order_of_their_lengths(S, page):
    # more than fit on the chip, in one launch; some of equal length, some empty, some without tokens, some of several blocks
    lens = [(s * 197) % 701 // 100 * 100 + s % 3 for s in range(S)]
    news = [0 if s % 11 == 5 else 1 + (5 * s) % 9 for s in range(S)]
    lens[3], news[2], news[3], lens[S - 1] = 0, 150, 4, 1300
    run_cross(lens, news, 8, 4, page)
