"""Page plans and rows into slots against plain loops, and the operators on caches in pages together."""
import numpy as np
import pytest
import torch

import paper_2412_03213_amd as ck
from paged_ref import D, attend, turn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INT_MIN = -2 ** 31


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def shape(S, Hkv=1, G=1, dtype=BF):
    return ck.Shape(S, Hkv * G, Hkv, 1, 1, dtype=ck.CK_BF16 if dtype is BF else ck.CK_F32)


class Batch:
    """Requests served one after the other, on lists."""

    def __init__(self, S, width, n_pages, size, held=()):
        self.size, self.width = size, width
        self.lengths, self.table = [0] * S, [[-1] * width for _ in range(S)]
        held = set(held)
        self.refs = [int(p in held) for p in range(n_pages)]

    def tensors(self):
        return i32(self.lengths), i32(self.table), i32(self.refs)

    def step(self, n_new, parent=None, shared=None, n_rows=0):
        size, width, pages = self.size, self.width, len(self.refs)
        before = list(self.lengths)
        for s, n in enumerate(n_new):
            if parent is None or n < 0 or before[s] > 0 or not 0 <= parent[s] < len(n_new):
                continue
            whole = min(max(0, min(shared[s], before[parent[s]])) // size, width)
            for e in range(whole):
                p = self.table[parent[s]][e]
                ok = 0 <= p < pages
                self.table[s][e] = p if ok else -1
                self.refs[p] += 1 if ok else 0
            self.lengths[s] = whole * size
        for s, n in enumerate(n_new):
            if n < 0:
                after = max(0, self.lengths[s] + n)
                for e in range(-(-after // size), min(width, -(-self.lengths[s] // size))):
                    p = self.table[s][e]
                    if 0 <= p < pages:
                        self.refs[p] -= 1
                    self.table[s][e] = -1
                self.lengths[s] = after
        free = [p for p in range(pages) if self.refs[p] == 0]
        starts, slots, lacking = [0], [], 0
        for s, n in enumerate(n_new):
            n = max(n, 0)
            for e in range(-(-self.lengths[s] // size), -(-(self.lengths[s] + n) // size)):
                if e >= width:
                    lacking += 1
                elif not free:
                    lacking += 1
                    self.table[s][e] = -1
                else:
                    self.table[s][e] = free.pop(0)
                    self.refs[self.table[s][e]] = 1
            for r in range(self.lengths[s], self.lengths[s] + n):
                p = self.table[s][r // size] if r // size < width else -1
                slots.append(p * size + r % size if 0 <= p < pages else -1)
            self.lengths[s] += n
            starts.append(starts[-1] + n)
        return starts, (slots + [-1] * n_rows)[:n_rows], lacking


class Steps:
    """The same requests on the device and in loops, compared after every step."""

    def __init__(self, S, width, n_pages, size, held=()):
        self.b, self.sh = Batch(S, width, n_pages, size, held), shape(S)
        self.lengths, self.table, self.refs = self.b.tensors()

    def step(self, n_new, parent=None, shared=None, n_rows=None):
        total = sum(max(n, 0) for n in n_new)
        n_rows = total if n_rows is None else n_rows
        starts = i32([77] * (len(n_new) + 1))
        slots = i32([77] * n_rows) if n_rows else None
        lacking = i32([77])
        ck.ck_plan_pages(self.sh, i32(n_new), self.lengths, self.table, self.refs, self.b.size, starts, lacking, slots=slots,
                         parent=None if parent is None else i32(parent),
                         shared_rows=None if shared is None else i32(shared))
        want = self.b.step(n_new, parent, shared, n_rows)
        assert starts.tolist() == want[0]
        assert int(lacking) == want[2]
        assert self.lengths.tolist() == self.b.lengths
        assert self.table.tolist() == self.b.table
        assert self.refs.tolist() == self.b.refs
        if n_rows:
            assert slots.tolist() == want[1]
        return want


@pytest.mark.parametrize("size", [1, 16, 7])
def test_plan_tokens_one_by_one(size):
    x = Steps(5, 40, 100, size, held=(0, 3, 4))
    x.step([1, 0, 20, 2, 0])
    for _ in range(18):
        x.step([1, 1, 1, 0, 1])


def test_plan_one_sequence_one_page():
    x = Steps(1, 1, 1, 64)
    x.step([64])
    x.step([0])
    assert x.step([1])[2] == 1                            # the table has no entry
    x.step([-1])
    x.step([INT_MIN])
    x.step([3])


def test_plan_takes_back_and_gives_out_the_same_pages():
    x = Steps(4, 30, 60, 8)
    x.step([100, 9, 0, 33])
    x.step([-4, -9, 50, -1])                              # pages of one go to another in the same call
    x.step([5, -1, -17, INT_MIN])
    x.step([-10 ** 9, 0, INT_MIN, 1])


def test_plan_without_enough_pages():
    x = Steps(3, 20, 10, 4, held=(1, 2))
    assert x.step([17, 9, 30])[2] == 8
    x.step([1, 1, 1])
    x.step([INT_MIN, 0, 0])
    x.step([0, 0, 9])                                     # rows that are there already stay on no page
    x = Steps(2, 3, 10, 4)
    assert x.step([20, 1])[2] == 2                        # five pages, three entries
    x.step([-8, 0])
    x.step([-1, 0])


def test_plan_parents():
    x = Steps(6, 20, 100, 8)
    x.step([50, 0, 0, 0, 0, 3])
    # children of the first: all of it, a part, more than there is; of one without rows; of themselves; of nobody
    x.step([1, 5, 0, 8, 2, 1], parent=[-1, 0, 0, 0, 4, 0], shared=[0, 50, 17, 1000, 9, 50])
    # grandchildren, next to a parent that ends: its pages are still theirs
    x.step([INT_MIN, INT_MIN, 0, 0, 0, INT_MIN], parent=[0] * 6, shared=[8] * 6)
    x.step([3, 3, 0, 0, 0, 2], parent=[3, 3, 3, 3, 3, 2 ** 31 - 1], shared=[48, 40, 1, 1, 1, 1])
    x.step([INT_MIN] * 6, parent=[-5] * 6, shared=[-5] * 6)
    assert sum(x.b.refs) == 0


def test_plan_parents_without_pages():
    x = Steps(3, 10, 3, 4)
    x.step([20, 0, 0])                                    # two of its pages are lacking
    x.step([0, 2, 1], parent=[-1, 0, 0], shared=[0, 20, 12])


def test_plan_rows_of_a_padded_batch():
    x = Steps(3, 10, 30, 4)
    x.step([5, 0, 3], n_rows=20)                          # -1 behind the last sequence
    x.step([5, 0, 3], n_rows=6)                           # fewer slots than rows
    x.step([2, 2, 2], n_rows=0)


@pytest.mark.parametrize("S", [64, 1023, 1025, 3000])
def test_plan_many_sequences(S):
    x = Steps(S, 6, 9 * S, 4, held=range(0, 9 * S, 5))
    rng = np.random.default_rng(S)
    x.step(rng.integers(0, 9, S).tolist())
    parent = rng.integers(-1, S, S).tolist()
    x.step(rng.integers(-6, 9, S).tolist(), parent=parent, shared=rng.integers(0, 20, S).tolist())
    x.step([1] * S)
    x.step(np.where(rng.random(S) < 0.3, INT_MIN, 1).tolist())


def test_plan_as_many_sequences_as_there_can_be():
    x = Steps(8192, 1, 9000, 4)
    x.step([1] * 8192)
    x.step([-1 if s % 2 else 2 for s in range(8192)])


def test_plan_long_prompts_and_pools():
    # more rows than the planning workgroup writes slots for, more pages than are looked at together
    n = 2 * 131072 + 77
    x = Steps(3, 5000, n, 3, held=range(0, n - 40000))
    x.step([9000, 1, 12345])
    x.step([1, 1, 1], n_rows=9001)
    x = Steps(2, 30000, 200, 3)
    x.step([8192, 0], n_rows=8192)
    x.step([0, 8193])


def test_plan_random_requests():
    for seed in range(30):
        rng = np.random.default_rng(seed)
        S, size = int(rng.integers(1, 40)), int(rng.integers(1, 20))
        x = Steps(S, int(rng.integers(1, 30)), int(rng.integers(1, 400)), size, held=rng.integers(0, 400, 50).tolist())
        for _ in range(6):
            n = rng.integers(0, 4 * size, S)
            n = np.where(rng.random(S) < 0.3, -rng.integers(0, 6 * size, S), n)
            n = np.where(rng.random(S) < 0.1, INT_MIN, n)
            parent, shared = rng.integers(-2, S + 2, S).tolist(), rng.integers(-3, 8 * size, S).tolist()
            # who takes over a page that the table names twice would make two sequences write to one page: plans only count
            x.step(n.tolist(), parent=parent, shared=shared)


def test_plan_from_a_graph():
    """Replayed with other requests, between eager work."""
    b = Batch(4, 20, 64, 8)
    sh = shape(4)
    lengths, table, refs = b.tensors()
    n_new, starts, slots, lacking = i32([0] * 4), i32([0] * 5), i32([0] * 16), i32([0])
    call = lambda: ck.ck_plan_pages(sh, n_new, lengths, table, refs, 8, starts, lacking, slots=slots)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in ([9, 1, 0, 2], [1, 1, 1, 1], [-3, INT_MIN, 8, 1], [1, 5, 1, 1], [INT_MIN] * 4):
        n_new.copy_(i32(n))
        graph.replay()
        torch.cuda.synchronize()
        want = b.step(n, n_rows=16)
        assert (starts.tolist(), slots.tolist(), int(lacking)) == want
        assert (lengths.tolist(), table.tolist(), refs.tolist()) == (b.lengths, b.table, b.refs)


# ---------------------------------------------------------------- rows into slots
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hkv,page", [(1, 1), (8, 16), (3, 7), (2, 64)])
def test_store(Hkv, page, dtype):
    g = torch.Generator().manual_seed(3)
    for n in (1, 2, 333):
        pages = n // page + 3
        qkv = torch.randn(n, (2 * Hkv + 1) * D, generator=g).to(dtype).to(DEV)
        k, v = (x.unflatten(1, (-1, D)) for x in (qkv[:, D:(Hkv + 1) * D], qkv[:, (Hkv + 1) * D:]))    # views
        slots = torch.randperm(pages * page, generator=g)[:n].to(torch.int32)
        slots[::5] = torch.tensor([-1, pages * page, 2 ** 31 - 1, INT_MIN])[torch.arange(len(slots[::5])) % 4].int()
        K = torch.randn(pages, Hkv, page, D, generator=g).to(dtype).to(DEV)
        V = torch.randn(pages, Hkv, page, D, generator=g).to(dtype).to(DEV)
        want_k, want_v = K.clone(), V.clone()
        for t, p in enumerate(slots.tolist()):
            if 0 <= p < pages * page:
                want_k[p // page, :, p % page], want_v[p // page, :, p % page] = k[t], v[t]
        ck.ck_store_rows(shape(1, Hkv, 1, dtype), k, v, slots.to(DEV), ck.PagedKV(K, V))
        assert torch.equal(K, want_k) and torch.equal(V, want_v)


def test_store_special_values_and_other_streams():
    k = torch.tensor([float("nan"), float("inf"), -0.0, 1e-40], device=DEV).repeat(32).view(1, 1, D)
    K, V = torch.zeros(2, 1, 4, D, device=DEV), torch.zeros(2, 1, 4, D, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ck.ck_store_rows(shape(1, dtype=F32), k, k, i32([5]), ck.PagedKV(K, V))
    side.synchronize()
    assert torch.equal(K[1, 0, 1].view(torch.int32), k[0, 0].view(torch.int32))
    assert K.view(torch.int32).count_nonzero() == k.view(torch.int32).count_nonzero()


# ---------------------------------------------------------------- together
def test_a_shared_prompt_and_an_encoder_from_requests_to_answers():
    """A prompt comes in; four answers begin with it and go on by themselves, planned, appended and attended to on the device;
    each also attends to the states of an encoder."""
    Hkv, G, size, n = 2, 4, 16, 150
    g = torch.Generator().manual_seed(11)
    S = 5                                                 # the prompt, then its answers
    sh, freqs = shape(S, Hkv, G), ck.ck_rope_frequencies(ck.CK_ROPE_PLAIN, D)[0]
    K = torch.full((80, Hkv, size, D), float("nan"), dtype=BF, device=DEV)
    kv = ck.PagedKV(K, K.clone(), torch.full((S, 20), -1, dtype=torch.int32, device=DEV))
    lengths, refs, starts, lacking = i32([0] * S), i32([0] * 80), i32([0] * (S + 1)), i32([0])
    rnd = lambda *s: torch.randn(*s, generator=g).to(BF).to(DEV)
    keys, values = [[] for _ in range(S)], [[] for _ in range(S)]

    def append(news, parent=None, shared=None):
        T = sum(news)
        ck.ck_plan_pages(sh, i32(news), lengths, kv.page_table, refs, size, starts, lacking, parent=parent, shared_rows=shared)
        q, k, v = rnd(T, Hkv * G, D), rnd(T, Hkv, D), rnd(T, Hkv, D)
        q_rot = torch.empty_like(q)
        ck.ck_rope_append(sh, q, k, v, kv, lengths, freqs.to(DEV), q_rot, q_starts=starts)
        t = 0
        for s, m in enumerate(news):
            for _ in range(m):
                keys[s].append(turn(k[t].cpu(), len(keys[s]), freqs.numpy(), 1.0, False)[0])
                values[s].append(v[t].double().cpu().numpy())
                t += 1
        return q_rot

    q = append([n, 0, 0, 0, 0])
    ck.ck_prompt_attn(sh, q, starts, kv, lengths, torch.empty_like(q))
    whole = n // size * size
    for s in range(1, S):                                 # rows of whole pages are taken over, the rest computed again
        keys[s], values[s] = keys[0][:whole], values[0][:whole]
    append([0, 3, 1, 9, 6], parent=i32([-1, 0, 0, 0, 0]), shared=i32([n] * S))
    groups, shared = i32([0, S]), i32([whole] * S)
    for step in range(3):
        q = append([1] * S)
        assert int(lacking) == 0
        out = torch.empty_like(q)
        ck.ck_shared_decode_attn(sh, q, kv, lengths, groups, shared, out)
        for s in range(S):
            # the rows as they stand in the cache: keys and values of each sequence
            k_rows = torch.from_numpy(np.stack(keys[s], 1)).to(BF)
            v_rows = torch.from_numpy(np.stack(values[s], 1)).to(BF)
            m = len(keys[s])
            assert m == int(lengths[s])
            r = torch.arange(m, device=DEV)
            page = kv.page_table[s].long()[r // size]
            got_k = kv.K[page, :, r % size].transpose(0, 1).cpu()
            # one rounding of the turned key, of which the plain form has one too
            assert ((got_k.double() - k_rows.double()).abs() <= 2 ** -7 * k_rows.double().abs() + 1e-5).all()
            assert torch.equal(kv.V[page, :, r % size].transpose(0, 1).cpu(), v_rows)
            for h in range(Hkv):
                want, tol = attend(q[s, h * G:(h + 1) * G].cpu(), got_k[h], v_rows[h], np.ones((G, m)), BF, p_step=2.0 ** -8)
                err = np.abs(out[s, h * G:(h + 1) * G].double().cpu().numpy() - want)
                assert (err <= tol).all(), (step, s, h)
    assert refs[kv.page_table[0, 0].long()] == S
    # an encoder's states, in pages of the same pool, planned with a table of their own
    states, table = [40, 70], torch.full((2, 8), -1, dtype=torch.int32, device=DEV)
    sh2, n2, starts2, slots = shape(2, Hkv, G), i32([0, 0]), i32([0] * 3), i32([0] * 110)
    ck.ck_plan_pages(sh2, i32(states), n2, table, refs, size, starts2, lacking, slots=slots)
    k, v = rnd(110, Hkv, D), rnd(110, Hkv, D)
    enc = ck.PagedKV(kv.K, kv.V, table)
    ck.ck_store_rows(sh2, k, v, slots, enc)
    q = rnd(S, Hkv * G, D)
    out = torch.empty_like(q)
    ck.ck_cross_attn(sh2, q, i32([0, 2, S]), enc, n2, out)
    for s in range(S):
        a, b = (0, 40) if s < 2 else (40, 110)
        for h in range(Hkv):
            want, tol = attend(q[s, h * G:(h + 1) * G].cpu(), k[a:b, h].cpu(), v[a:b, h].cpu(), np.ones((G, b - a)), BF, p_step=2.0 ** -8)
            err = np.abs(out[s, h * G:(h + 1) * G].double().cpu().numpy() - want)
            assert (err <= tol).all(), (s, h)
    ck.ck_plan_pages(sh, i32([INT_MIN] * S), lengths, kv.page_table, refs, size, starts, lacking)
    ck.ck_plan_pages(sh2, i32([INT_MIN] * 2), n2, table, refs, size, starts2, lacking)
    assert int(refs.abs().sum()) == 0


def test_calls_with_and_without_the_native_marshalling(monkeypatch):
    """The same results, and refusals of what the native form leaves to the general one."""
    g = torch.Generator().manual_seed(5)
    lib, sh = ck.load_library(), shape(2, 2, 4)
    rnd = lambda *s: torch.randn(*s, generator=g).to(BF).to(DEV)
    K, V, q, k = rnd(20, 2, 16, D), rnd(20, 2, 16, D), rnd(7, 8, D), rnd(7, 2, D)
    results = []
    for native in (True, False):
        if not native:
            for name in ("plan_pages", "store_rows", "shared_decode_attn", "cross_attn"):
                monkeypatch.setattr(lib, "host_" + name, lambda *args: None)
        kv = ck.PagedKV(K.clone(), V.clone(), torch.full((2, 8), -1, dtype=torch.int32, device=DEV))
        n, refs, starts, lacking, slots = i32([0, 0]), i32([0] * 20), i32([0] * 3), i32([0]), i32([0] * 7)
        ck.ck_plan_pages(sh, i32([40, 50]), n, kv.page_table, refs, 16, starts, lacking)
        ck.ck_plan_pages(sh, i32([3, 4]), n, kv.page_table, refs, 16, starts, lacking, slots=slots,
                         parent=i32([-1, -1]), shared_rows=i32([0, 0]))
        ck.ck_store_rows(sh, k, k, slots, kv)
        a, b, c = torch.empty_like(q), torch.empty_like(q[:2]), torch.empty_like(q[:2])
        ck.ck_cross_attn(sh, q, starts, kv, n, a)
        ck.ck_cross_attn(sh, q[:2], None, kv, n, b)
        ck.ck_shared_decode_attn(sh, q[:2], kv, n, i32([0, 2]), i32([0, 0]), c, softmax_scale=0.1)
        results.append((n, kv.page_table, refs, starts, lacking, slots, kv.K, kv.V, a, b, c))
        with pytest.raises(ck.ClusterKVError):
            ck.ck_cross_attn(sh, q, starts, kv, n, q)
        with pytest.raises(ck.ClusterKVError):
            ck.ck_shared_decode_attn(sh, q[:2], kv, n, i32([0, 1, 2, 2]), i32([0, 0]), c)
        with pytest.raises(ck.ClusterKVError):
            ck.ck_plan_pages(sh, n, n, kv.page_table, refs, 0, starts, lacking)
        with pytest.raises(ck.ClusterKVError):
            ck.ck_plan_pages(sh, n, n, kv.page_table, refs, 16, starts, lacking, parent=n)
        with pytest.raises(ValueError):
            ck.ck_store_rows(sh, k, k[:3], slots, kv)
        with pytest.raises(ValueError):
            ck.ck_plan_pages(sh, n, n, kv.page_table[:1], refs, 16, starts, lacking)
    assert all(torch.equal(x, y) for x, y in zip(*results))


def test_tensors_on_another_device_are_refused(monkeypatch):
    """A device that is not the current one."""
    from paper_2412_03213_amd import binding
    sh, n, starts, one = shape(1, 1, 4), i32([1]), i32([0, 1]), i32([0])
    kv = ck.PagedKV(torch.zeros(2, 1, 4, D, dtype=BF, device=DEV), torch.zeros(2, 1, 4, D, dtype=BF, device=DEV))
    q, k, refs = torch.zeros(1, 4, D, dtype=BF, device=DEV), torch.zeros(1, 1, D, dtype=BF, device=DEV), i32([0, 0])
    sh2 = ck.Shape(1, 4, 1, 4, 1)
    kv1 = ck.PagedKV(kv.K, kv.V, i32([[0]]))
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    for call in (lambda: ck.ck_plan_pages(sh, n, n, i32([[0]]), refs, 4, starts, one),
                 lambda: ck.ck_store_rows(sh, k, k, n, kv1), lambda: ck.ck_cross_attn(sh2, q, starts, kv1, n, q.clone()),
                 lambda: ck.ck_shared_decode_attn(sh2, q, kv1, n, starts, n, q.clone())):
        with pytest.raises(ValueError, match="current"):
            call()


@pytest.mark.parametrize("S,n_pages,width", [(130, 9003, 130), (130, 70001, 600), (1100, 40000, 20)])
def test_plan_many_pages_of_many_at_once(S, n_pages, width):
    """Enough entries for counts in LDS: pages at the end of what it holds and behind it, counted once for each of many."""
    rng = np.random.default_rng(S + width)
    far = n_pages * 15 // 16                              # free: a few pages before, all behind
    x = Steps(S, width, n_pages, 4, held=rng.choice(far, far - far // 200, replace=False).tolist())
    long = min(width - 4, 90) * 4 - 1
    x.step([long, long + 1, long] + [0] * (S - 3))
    x.step([0, 3, 0] + [int(v) for v in rng.integers(0, 9, S - 3)], parent=[s % 3 for s in range(S)], shared=[10 ** 6] * S)
    x.step([int(v) for v in rng.integers(-long, 5, S)])
    x.step([INT_MIN if s % 7 else 1 for s in range(S)], parent=[1] * S, shared=[long] * S)
    x.step([INT_MIN] * S)
    assert sum(x.b.refs) == far - far // 200


def test_plan_more_entries_than_counts_in_lds_hold():
    x = Steps(100, 400, 500, 1)
    x.step([390] + [0] * 99)
    x.step([0] * 100, parent=[0] * 100, shared=[380] * 100)   # 37620 entries of 380 pages
    assert x.b.refs[0] == 100
    x.step([INT_MIN] * 100)
    assert sum(x.b.refs) == 0
