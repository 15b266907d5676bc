"""Operators around caches in pages that a server needs between its requests and the attention, as
cases that can be timed one by one:

  plan    page tables, reference counts and the slot of every new token's row from the requests of a
          batch (ck_plan_pages): a pass gives tokens to sequences, then takes them back
  store   rows of keys and values into their slots (ck_store_rows)
  shared  attention of one new token of every sequence where sequences of a group begin with the same
          rows (ck_shared_decode_attn)
  cross   attention of several tokens of every sequence to all rows of an encoder's states
          (ck_cross_attn)

`run` computes them from elementary torch operations, or, where `own` is true, through the
package's entry points.  Sequences of a batch differ in length by a fixed pattern, pages lie
in the pool in random order, keys and queries follow the repository's mixture recipe.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
D = 128
ALL = 2 ** 31 - 1
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _plan(**kw):
    # S sequences that hold rows already get `draft` tokens, `fresh` new ones a prompt of up to `new`, of which
    # those with a parent take over its first pages; pool: pages there are; held: share of those that others hold
    return {**dict(op="plan", S=64, N=2048, spread=0.5, page=16, pool=16384, held=0.5, draft=1, fresh=0,
                   new=1, parents=False), **kw}


def _store(**kw):
    return {**dict(op="store", T=64, Hkv=8, G=4, page=64, pool=1024, lost=0.0, dtype="bf16"), **kw}


def _shared(**kw):
    # groups of up to `members` sequences; N shared rows, then up to `rest` of their own
    return {**dict(op="shared", groups=1, members=16, N=8192, rest=512, spread=0.5, Hkv=8, G=4, page=64,
                   dtype="bf16"), **kw}


def _cross(**kw):
    # new = 0: one token per sequence and no list of starts; every `gone`-th sequence has no rows (0: none)
    return {**dict(op="cross", S=8, N=1500, new=64, spread=0.5, gone=0, Hkv=8, G=1, page=64, dtype="bf16"), **kw}


def listed():
    return [
        # a token of 64 users: a launch and its latency
        _plan(name="plan_step"),
        # a large batch, half of it prompts that come in, most of them behind a prefix that is there already
        _plan(name="plan_prompts", S=128, N=4000, page=16, pool=131072, held=0.3, draft=5, fresh=128, new=700,
              parents=True),
        # a token of 64 users
        _store(name="store_step"),
        # states of an encoder for 16 inputs, pages of odd size
        _store(name="store_states", T=16 * 1500, page=20, pool=1500),
        # four answers to one short question: latency
        _shared(name="shared_few", members=4, N=2048, rest=100),
        # 64 users of one long system prompt
        _shared(name="shared_b64", members=64, N=32768, rest=2047),
        # several prompts, larger groups of heads, pages that end inside tiles, shared rows that end inside pages
        _shared(name="shared_groups", groups=5, members=7, N=7001, rest=1500, Hkv=4, G=8, page=40),
        # many answers about one book
        _shared(name="shared_128k", members=16, N=131072, rest=300),
        # four beams of 16 inputs, as many KV as query heads: nearly a decode step
        _cross(name="cross_beams", S=16, N=1500, new=4, spread=0.0, Hkv=16),
        # the first tokens of many outputs over states of different lengths, two of them empty
        _cross(name="cross_ragged", S=24, N=1500, new=220, gone=12, page=20, G=2),
        # a chunk of tokens over long states
        _cross(name="cross_chunk", S=1, N=30011, new=500, G=4, spread=0.0),
        # long outputs over long states: the rate of the matrix cores
        _cross(name="cross_8k", S=2, N=8192, new=6000, G=4, spread=0.3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "store", "shared", "shared", "cross", "cross"])
    page = rng.choice([16, 16, 32, 64, 64, 128, 256, rng.randint(1, 100)])
    spread = rng.choice([0.0, 0.3, 0.9])
    dtype = rng.choice(["bf16"] * 7 + ["f32"])
    while True:
        if op == "plan":
            c = _plan(S=_log(rng, 1, 512), N=_log(rng, 1, 20000), spread=spread, page=page,
                      held=rng.choice([0.1, 0.5]), draft=rng.choice([1, 1, rng.randint(1, 9)]),
                      fresh=rng.choice([0, _log(rng, 1, 256)]), new=_log(rng, 1, 4096),
                      parents=rng.choice([False, True]))
            # now and then the pool has fewer pages than are asked for
            need = sum(-(-n // page) for n in _plan_sizes(c)[0]) + c["fresh"] * (c["new"] // page + 1)
            c["pool"] = int(need * rng.choice([1.0 - 0.5 * c["held"], 1.3, 3.0])) + 8
            if c["pool"] <= 131072 and c["S"] * c["draft"] + c["fresh"] * c["new"] <= 90000:
                return c
            continue
        c = dict(Hkv=rng.choice([1, 2, 4, 8, 8]), G=rng.choice([1, 2, 4, 4, 8]), page=page, dtype=dtype)
        if op == "store":
            c["T"] = _log(rng, 1, 24000)
            c["pool"] = -(-c["T"] // page) * rng.choice([1, 2]) + 1
            if c["pool"] * page * c["Hkv"] <= 8 * 60000:
                return _store(**c, lost=rng.choice([0.0, 0.0, 0.1]))
        elif op == "shared":
            c.update(groups=_log(rng, 1, 12), members=_log(rng, 1, 64), N=_log(rng, 1, 131072),
                     rest=_log(rng, 1, 4096), spread=spread)
            if c["dtype"] == "f32":                       # check mode
                c["N"] = min(c["N"], 4096)
            # at most the rows, and the pairs of query and row, of the largest listed cases
            rows = c["groups"] * (c["N"] + c["members"] * c["rest"])
            pairs = c["groups"] * c["members"] * (c["N"] + c["rest"])
            if rows * c["Hkv"] <= 8 * 131072 and pairs * c["Hkv"] * c["G"] <= 32 * 64 * 33000:
                return _shared(**c)
        else:
            c.update(S=_log(rng, 1, 64), N=_log(rng, 1, 65536), spread=spread, gone=rng.choice([0, 0, 3]))
            c["new"] = rng.choice([_log(rng, 1, 8192), _log(rng, 1, 64), 0])
            c["dtype"] = dtype if c["new"] == 0 else "bf16"
            if (c["S"] * max(1, c["new"]) * c["N"] * c["Hkv"] * c["G"] <= 2 * 32 * 6000 * 8192
                    and c["S"] * c["N"] * c["Hkv"] <= 8 * 131072 and c["S"] * c["new"] <= 20000):
                return _cross(**c)
            page = rng.choice([16, 64, rng.randint(1, 100)])


# ---------------------------------------------------------------- sizes
def _ragged(n, count, spread, turn=0.6180339887):
    return [max(1, int(n * (1.0 - spread * ((i * turn) % 1.0)))) for i in range(count)]


def _plan_sizes(case):
    """Rows of every sequence before, tokens that it gets, its parent and how many rows it shares."""
    lens = _ragged(case["N"], case["S"], case["spread"]) + [0] * case["fresh"]
    news = [case["draft"]] * case["S"] + _ragged(case["new"], case["fresh"], case["spread"], 0.3819660113)
    parent, shared = [-1] * len(lens), [0] * len(lens)
    if case["parents"]:
        for i in range(case["fresh"]):
            if i % 4 != 3:                                # every fourth begins on its own
                p = i * 7 % case["S"]
                parent[case["S"] + i], shared[case["S"] + i] = p, lens[p] * (1 + i % 3) // 3
    return lens, news, parent, shared


def _shared_sizes(case):
    """First sequence of every group and the end; shared rows and all rows of every sequence."""
    starts, shared, lens = [0], [], []
    for m, n in zip(_ragged(case["members"], case["groups"], case["spread"], 0.3819660113),
                    _ragged(case["N"], case["groups"], case["spread"])):
        starts.append(starts[-1] + m)
        shared += [n] * m
        lens += [n + r for r in _ragged(case["rest"], m, case["spread"])]
    return starts, shared, lens


def _cross_sizes(case):
    lens = _ragged(case["N"], case["S"], case["spread"])
    if case["gone"]:
        lens = [0 if i % case["gone"] == case["gone"] - 1 else n for i, n in enumerate(lens)]
    news = _ragged(case["new"], case["S"], case["spread"], 0.3819660113) if case["new"] else [1] * case["S"]
    return lens, news


def work(case):
    op = case["op"]
    if op == "plan":
        lens, news, parent, shared = _plan_sizes(case)
        ps, S = case["page"], len(lens)
        taken = sum(s // ps for s in shared)
        given = sum(max(0, -(-(s // ps * ps + n + m) // ps) - -(-(s // ps * ps + n) // ps))
                    for n, m, s in zip(lens, news, shared))
        # counts of all pages once; every entry that changes, and its page's count, there and back; starts and slots
        return dict(bytes=4 * (case["pool"] + 2 * 4 * S + 2 * 2 * S + 4 * (taken + given) + 2 * S + sum(news)),
                    flops=0)
    size = 2 if case["dtype"] == "bf16" else 4
    row, Hkv, G = D * size, case["Hkv"], case["G"]
    if op == "store":
        return dict(bytes=4 * case["T"] * Hkv * row + 4 * case["T"], flops=0)
    if op == "shared":
        starts, shared, lens = _shared_sizes(case)
        rows = sum(shared[a] for a in starts[:-1]) + sum(lens) - sum(shared)
        T, pairs = len(lens), sum(lens)
    else:
        lens, news = _cross_sizes(case)
        T, rows, pairs = sum(news), sum(lens), sum(n * m for n, m in zip(lens, news))
    return dict(bytes=2 * T * Hkv * G * row + 2 * rows * Hkv * row, flops=4 * D * pairs * Hkv * G)


# ---------------------------------------------------------------- inputs
class _Inputs:
    def __init__(self, case, seed):
        self.c = case
        self.dtype = _TYPES[case.get("dtype", "bf16")]
        self.g = torch.Generator(device=DEV).manual_seed(int(seed))
        m = self.randn(case.get("Hkv", 1), 64, D)
        self.centers = m / m.norm(dim=-1, keepdim=True)

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g, device=DEV)

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device=DEV)

    def near_centers(self, *lead):
        """[*lead, Hkv, n, D] with n the last of lead: 3 * center + noise of 0.5 per channel."""
        *lead, n = lead
        Hkv = self.c["Hkv"]
        pick = torch.randint(0, 64, (*lead, Hkv, n), generator=self.g, device=DEV)
        x = self.centers[torch.arange(Hkv, device=DEV)[:, None], pick].mul_(3.0)
        return x.add_(self.randn(*x.shape), alpha=0.5).to(self.dtype)

    def queries(self, T):
        return self.near_centers(T, self.c["G"]).reshape(T, -1, D)

    def pool(self, n_pages):
        c = self.c
        K = torch.empty(n_pages, c["Hkv"], c["page"], D, dtype=self.dtype, device=DEV)
        V = torch.empty_like(K)
        part = max(1, (1 << 25) // (c["Hkv"] * c["page"] * D))
        for a in range(0, n_pages, part):                 # small temporaries
            n = min(part, n_pages - a)
            K[a:a + n] = self.near_centers(n, c["page"])
            V[a:a + n] = self.randn(n, c["Hkv"], c["page"], D).to(self.dtype)
        return K, V


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(news):
    return _ints([0] + list(np.cumsum(news)))


def prepare(case, seed):
    x = _Inputs(case, seed)
    s = dict(case=case)
    _PREPARE[case["op"]](s, case, x)
    if own:
        _handles(s)
    return s


def _prepare_plan(s, case, x):
    lens, news, parent, shared = _plan_sizes(case)
    ps, S, pool = case["page"], len(lens), case["pool"]
    width = max(-(-(k + n + m) // ps) for n, m, k in zip(lens, news, shared)) + 2
    order = x.perm(pool).to(torch.int32).cpu()
    table = torch.full((S, width), -1, dtype=torch.int32)
    refs = torch.zeros(pool, dtype=torch.int32)
    at = 0
    for i, n in enumerate(lens):
        mine = order[at:at + -(-n // ps)]                 # fewer where the pool is too small
        table[i, :mine.numel()] = mine
        refs[mine.long()] += 1
        at += mine.numel()
    rest = order[at:]
    refs[rest[:int(rest.numel() * case["held"])].long()] = 1
    s["table"], s["refs"], s["lengths"] = table.to(DEV), refs.to(DEV), _ints(lens)
    s["news"], s["n_rows"] = _ints(news), sum(news) + 3   # a batch that was rounded up
    s["back"] = _ints([-m if n else -ALL for n, m in zip(lens, news)])
    s["parent"], s["shared"] = (_ints(parent), _ints(shared)) if case["parents"] else (None, None)
    s["starts"], s["starts2"] = _ints([0] * (S + 1)), _ints([0] * (S + 1))
    s["slots"] = torch.zeros(s["n_rows"], dtype=torch.int32, device=DEV)
    s["lacking"], s["lacking2"] = _ints([0]), _ints([0])


def _prepare_store(s, case, x):
    T, Hkv, G = case["T"], case["Hkv"], case["G"]
    qkv = x.randn(T, Hkv * (G + 2) * D).to(x.dtype)       # the views of a projection's output
    s["k"], s["v"] = (a.unflatten(1, (-1, D)) for a in qkv.split([Hkv * G * D, Hkv * D, Hkv * D], dim=1)[1:])
    # whole pages in random order, as sequences of a batch hold them
    ps = case["page"]
    t = torch.arange(T, device=DEV)
    slots = x.perm(case["pool"])[t // ps] * ps + t % ps
    lost = torch.rand(T, generator=x.g, device=DEV) < case["lost"]
    s["slots"] = slots.masked_fill(lost, -1).to(torch.int32)
    s["K"] = torch.zeros(case["pool"], Hkv, ps, D, dtype=x.dtype, device=DEV)
    s["V"] = torch.zeros_like(s["K"])


def _prepare_shared(s, case, x):
    starts, shared, lens = _shared_sizes(case)
    ps, S = case["page"], len(lens)
    whole = [n // ps for n in shared]                     # a page that ends with rows of others is each one's own
    ends = [-(-n // ps) for n in lens]
    total = sum(whole[a] for a in starts[:-1]) + sum(ends) - sum(whole) + 3
    order = x.perm(total).to(torch.int32).cpu()
    table = torch.full((S, max(ends)), -1, dtype=torch.int32)
    at = 0
    for a, b in zip(starts[:-1], starts[1:]):
        table[a:b, :whole[a]] = order[at:at + whole[a]]
        at += whole[a]
        for i in range(a, b):
            n = ends[i] - whole[a]
            table[i, whole[a]:ends[i]] = order[at:at + n]
            at += n
    s["table"], s["lengths"], s["shared"], s["starts"] = table.to(DEV), _ints(lens), _ints(shared), _ints(starts)
    s["K"], s["V"] = x.pool(total)
    for a, b in zip(starts[:-1], starts[1:]):             # shared rows of such a page are the same in each
        r = shared[a] % ps
        pages = table[a:b, whole[a]].long().to(DEV) if r else []
        for p in pages[1:]:
            s["K"][p, :, :r], s["V"][p, :, :r] = s["K"][pages[0], :, :r], s["V"][pages[0], :, :r]
    s["q"] = x.queries(S)
    s["out"] = torch.empty_like(s["q"])
    s["lens"], s["shares"], s["bounds"] = lens, shared, starts


def _prepare_cross(s, case, x):
    lens, news = _cross_sizes(case)
    ps = case["page"]
    each = [-(-n // ps) for n in lens]
    total = sum(each) + 3
    order = x.perm(total).to(torch.int32).cpu()
    table = torch.full((len(lens), max(1, max(each))), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(each):
        table[i, :n] = order[at:at + n]
        at += n
    s["table"], s["lengths"], s["starts"] = table.to(DEV), _ints(lens), _starts(news)
    s["K"], s["V"] = x.pool(total)
    s["q"] = x.queries(sum(news))
    s["out"] = torch.empty_like(s["q"])
    s["lens"], s["news"] = lens, news


_PREPARE = dict(plan=_prepare_plan, store=_prepare_store, shared=_prepare_shared, cross=_prepare_cross)


def _handles(s):
    """The shape, caches and workspace that a program keeps beside its tensors."""
    import paper_2412_03213_amd as ck
    case, op = s["case"], s["case"]["op"]
    s["ck"] = ck
    dt = ck.CK_BF16 if case.get("dtype", "bf16") == "bf16" else ck.CK_F32
    if op == "plan":
        S = s["lengths"].shape[0]
        s["sh"] = ck.Shape(S, 1, 1, s["table"].shape[1] * case["page"], 1, dtype=dt)
        return
    S = 1 if op == "store" else s["lengths"].shape[0]
    s["sh"] = ck.Shape(S, case["Hkv"] * case["G"], case["Hkv"], case["page"], 1, dtype=dt)
    table = s["table"] if op != "store" else _ints([[0]])
    s["kv"] = ck.PagedKV(s["K"], s["V"], table)
    if op == "shared":
        s["ws"] = ck.shared_decode_workspace(s["sh"], DEV)
    if op == "cross":
        s["ws"] = ck.cross_workspace(s["sh"], s["q"].shape[0], DEV)


# ---------------------------------------------------------------- one pass
def run(s):
    return (_OWN if own else _RUN)[s["case"]["op"]](s)


def _own_plan(s):
    s["ck"].ck_plan_pages(s["sh"], s["news"], s["lengths"], s["table"], s["refs"], s["case"]["page"],
                          s["starts"], s["lacking"], slots=s["slots"], parent=s["parent"],
                          shared_rows=s["shared"])
    s["ck"].ck_plan_pages(s["sh"], s["back"], s["lengths"], s["table"], s["refs"], s["case"]["page"],
                          s["starts2"], s["lacking2"])
    return s["starts"], s["slots"], s["lacking"], s["lengths"], s["table"], s["refs"]


def _own_store(s):
    s["ck"].ck_store_rows(s["sh"], s["k"], s["v"], s["slots"], s["kv"])
    return s["K"], s["V"]


def _own_shared(s):
    s["ck"].ck_shared_decode_attn(s["sh"], s["q"], s["kv"], s["lengths"], s["starts"], s["shared"], s["out"],
                                  workspace=s["ws"])
    return s["out"]


def _own_cross(s):
    s["ck"].ck_cross_attn(s["sh"], s["q"], s["starts"] if s["case"]["new"] else None, s["kv"], s["lengths"],
                          s["out"], workspace=s["ws"])
    return s["out"]


_OWN = dict(plan=_own_plan, store=_own_store, shared=_own_shared, cross=_own_cross)


def _plan_call(case, news, lengths, table, refs, parent, shared, n_rows):
    """One call in whole-tensor steps; lengths, table and refs change in place.  -> starts, slots, lacking"""
    ps, (S, width), pool = case["page"], table.shape, refs.shape[0]
    news, old = news.long(), lengths.long()
    e = torch.arange(width, device=DEV)
    is_page = lambda p: (p >= 0) & (p < pool)
    one = torch.ones((), dtype=torch.int32, device=DEV)
    if parent is not None:
        p = parent.long()
        takes = (p >= 0) & (p < S) & (old == 0) & (news >= 0)
        p = p.clamp(0, S - 1)
        pages = torch.where(takes, torch.minimum(shared.long(), old[p]).clamp(min=0) // ps, 0).clamp(max=width)
        from_parent = table[p]
        took = (e < pages[:, None]) & is_page(from_parent)
        table.copy_(torch.where(e < pages[:, None], torch.where(took, from_parent, -1), table))
        refs.index_put_((from_parent[took].long(),), one, accumulate=True)
        old = old + pages * ps
    new = (old + news).clamp(0, ALL)
    first, last = -(-new // ps), -(-old // ps)
    gone = (news < 0)[:, None] & (e >= first[:, None]) & (e < last[:, None])
    pages = table[gone & is_page(table)].long()
    refs.index_put_((pages,), -one, accumulate=True)
    table.masked_fill_(gone, -1)
    s_, e_ = ((e >= last[:, None]) & (e < first[:, None])).nonzero(as_tuple=True)
    free = (refs == 0).nonzero()[:, 0]
    n = min(s_.shape[0], free.shape[0])
    table[s_[:n], e_[:n]] = free[:n].to(torch.int32)
    table[s_[n:], e_[n:]] = -1
    refs[free[:n]] = 1
    lacking = (first - torch.maximum(last, torch.full_like(last, width))).clamp(min=0).sum() + s_.shape[0] - n
    lengths.copy_(new)
    starts = torch.zeros(S + 1, dtype=torch.long, device=DEV)
    starts[1:] = news.clamp(min=0).cumsum(0)
    t = torch.arange(n_rows, device=DEV)
    seq = torch.bucketize(t, starts[1:], right=True).clamp(max=S - 1)
    r = old[seq] + t - starts[seq]
    page = table[seq, (r // ps).clamp(0, width - 1)].long()
    there = (t < starts[S]) & (r // ps < width) & is_page(page)
    slots = torch.where(there, page * ps + r % ps, -1)
    return starts.to(torch.int32), slots.to(torch.int32), lacking.to(torch.int32)[None]


def _run_plan(s):
    state = s["lengths"], s["table"], s["refs"]
    out = _plan_call(s["case"], s["news"], *state, s["parent"], s["shared"], s["n_rows"])
    _plan_call(s["case"], s["back"], *state, None, None, 0)
    return *out, *state


def _run_store(s):
    ps, slot = s["case"]["page"], s["slots"].long()
    t = (slot >= 0).nonzero()[:, 0]
    s["K"][slot[t] // ps, :, slot[t] % ps] = s["k"][t]
    s["V"][slot[t] // ps, :, slot[t] % ps] = s["v"][t]
    return s["K"], s["V"]


def _gathered(s, pool, table, lo, hi):
    """Rows lo..hi - 1 of every sequence of table in 32 bits, [S, Hkv, hi - lo, D]."""
    ps = s["case"]["page"]
    r = torch.arange(lo, hi, device=DEV)
    page = table.long()[:, (r // ps).clamp(max=table.shape[1] - 1)].clamp(min=0)
    return pool[page, :, r % ps].permute(0, 2, 1, 3).float()


def _weights(q, K):
    """q K^T / sqrt(d) in 32 bits."""
    return torch.matmul(q, K.transpose(-1, -2).contiguous()).mul_(D ** -0.5)


def _run_shared(s):
    case = s["case"]
    Hkv, G = case["Hkv"], case["G"]
    out = torch.empty_like(s["q"])
    for a, b in zip(s["bounds"][:-1], s["bounds"][1:]):
        m, n, end = b - a, s["shares"][a], max(s["lens"][a:b])
        q = s["q"][a:b].float().view(m, Hkv, G, D)
        # scores over the rows of all, [Hkv, m G, n], and over each one's own, [m, Hkv, G, end - n]
        K, V = (_gathered(s, x, s["table"][a:a + 1], 0, n)[0] for x in (s["K"], s["V"]))
        w = _weights(q.transpose(0, 1).reshape(Hkv, m * G, D), K).view(Hkv, m, G, n).transpose(0, 1)
        K2, V2 = (_gathered(s, x, s["table"][a:b], n, end) for x in (s["K"], s["V"]))
        w2 = _weights(q, K2)
        r = torch.arange(n, end, device=DEV)
        w2.masked_fill_((r >= s["lengths"].long()[a:b, None])[:, None, None], -math.inf)
        top = torch.maximum(w.amax(-1, keepdim=True), w2.amax(-1, keepdim=True))
        w, w2 = (w - top).exp_(), w2.sub_(top).exp_()
        total = w.sum(-1, keepdim=True) + w2.sum(-1, keepdim=True)
        o = torch.matmul(w.transpose(0, 1).reshape(Hkv, m * G, n), V).view(Hkv, m, G, D).transpose(0, 1)
        out[a:b] = ((o + torch.matmul(w2, V2)) / total).reshape(m, Hkv * G, D).to(out.dtype)
    return out


def _run_cross(s):
    case = s["case"]
    Hkv, G = case["Hkv"], case["G"]
    S, n, m = len(s["lens"]), max(1, max(s["lens"])), max(s["news"])
    K, V = (_gathered(s, x, s["table"], 0, n) for x in (s["K"], s["V"]))
    starts = s["starts"].long()
    t = torch.arange(s["q"].shape[0], device=DEV)
    seq = torch.bucketize(t, starts[1:], right=True)
    q = torch.zeros(S, m, Hkv, G, D, device=DEV)
    q[seq, t - starts[seq]] = s["q"].float().view(-1, Hkv, G, D)
    w = _weights(q.permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * m, D), K)
    unseen = torch.arange(n, device=DEV) >= s["lengths"].long()[:, None]
    w.masked_fill_(unseen[:, None, None], -math.inf)
    w = w.sub_(w.amax(-1, keepdim=True).clamp_(min=-1e30)).exp_()
    total = w.sum(-1, keepdim=True)
    V.masked_fill_(unseen[:, None, :, None], 0.0)
    o = torch.matmul(w, V) / torch.where(total > 0, total, 1.0)
    o = o.view(S, Hkv, G, m, D).permute(0, 3, 1, 2, 4)[seq, t - starts[seq]]
    return o.reshape(-1, Hkv * G, D).to(s["q"].dtype)


_RUN = dict(plan=_run_plan, store=_run_store, shared=_run_shared, cross=_run_cross)


# ---------------------------------------------------------------- from the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["op"]](s, case)


def _exact_plan(s, case):
    """One request after the other, in plain numbers."""
    ps, pool = case["page"], case["pool"]
    lens, table, refs = s["lengths"].tolist(), s["table"].cpu().numpy().astype(np.int64), s["refs"].tolist()
    news, back = s["news"].tolist(), s["back"].tolist()
    before, width = list(lens), table.shape[1]
    if s["parent"] is not None:
        for i, (p, n) in enumerate(zip(s["parent"].tolist(), s["shared"].tolist())):
            if p >= 0 and before[i] == 0:
                pages = min(n, before[p]) // ps
                for e in range(pages):
                    table[i, e] = table[p, e]
                    if table[p, e] >= 0:
                        refs[table[p, e]] += 1
                lens[i] = pages * ps
    free = iter([p for p in range(pool) if refs[p] == 0])
    starts, slots, lacking = [0], [], 0
    for i, m in enumerate(news):
        for e in range(-(-lens[i] // ps), -(-(lens[i] + m) // ps)):
            page = next(free, None) if e < width else None
            lacking += page is None
            if page is not None:
                table[i, e], refs[page] = page, 1
        for r in range(lens[i], lens[i] + m):
            page = table[i, r // ps] if r // ps < width else -1
            slots.append(int(page) * ps + r % ps if page >= 0 else -1)
        lens[i] += m
        starts.append(starts[-1] + m)
    slots += [-1] * (s["n_rows"] - len(slots))
    for i, m in enumerate(back):
        n = max(0, lens[i] + m)
        for e in range(-(-n // ps), min(width, -(-lens[i] // ps))):
            if table[i, e] >= 0:
                refs[table[i, e]] -= 1
            table[i, e] = -1
        lens[i] = n
    return _ints(starts), _ints(slots), _ints([lacking]), _ints(lens), torch.from_numpy(table).int().to(DEV), _ints(refs)


def _exact_store(s, case):
    ps = case["page"]
    K, V = s["K"].double().cpu(), s["V"].double().cpu()
    k, v = s["k"].double().cpu(), s["v"].double().cpu()
    for t, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            K[slot // ps, :, slot % ps], V[slot // ps, :, slot % ps] = k[t], v[t]
    return K.to(DEV), V.to(DEV)


def _mean64(s, i, n, q):
    """Softmax means over rows 0..n - 1 of sequence i: q [M, Hkv, G, D] -> the same; one head at a time."""
    out = torch.zeros_like(q)
    r = torch.arange(n, device=DEV)
    page, slot = s["table"][i].long()[r // s["case"]["page"]], r % s["case"]["page"]
    for h in range(q.shape[1] if n else 0):
        K, V = s["K"][page, h, slot].double(), s["V"][page, h, slot].double()
        for a in range(0, q.shape[0], 1024):
            x = q[a:a + 1024, h].reshape(-1, D)
            w = torch.softmax(x @ K.T / math.sqrt(D), dim=-1)
            out[a:a + 1024, h] = (w @ V).view(-1, q.shape[2], D)
    return out


def _exact_attention(s, case):
    news = [1] * len(s["lens"]) if case["op"] == "shared" else s["news"]
    q = s["q"].double().view(-1, case["Hkv"], case["G"], D)
    out, t = torch.zeros_like(q), 0
    for i, (n, m) in enumerate(zip(s["lens"], news)):
        out[t:t + m] = _mean64(s, i, n, q[t:t + m])
        t += m
    return out.view(-1, case["Hkv"] * case["G"], D)


_EXACT = dict(plan=_exact_plan, store=_exact_store, shared=_exact_attention, cross=_exact_attention)
