"""Operators around the clustered cache, as cases that can be timed one by one:

  rope     new tokens' queries and keys turned by their rotary positions, keys and values
           written to the cache (ck_rope_append)
  decode   attention of one new token of every sequence over a paged cache
           (ck_paged_decode_attn): whole, windowed with sinks, or over a recalled list
  prompt   causal attention of several new tokens of every sequence over a paged cache,
           whole or windowed with sinks (ck_prompt_attn)
  copy     rows of one cache into another: forks, compaction by kept lists, pages into the
           contiguous form that clustering reads (ck_copy_rows)

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
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(op, **kw):
    c = dict(op=op, S=1, Hkv=8, G=4, N=2048, spread=0.0, page=64, dtype="bf16")
    c.update(kw)
    return c


def _rope(**kw):
    # new = 0: one token per sequence and no list of starts; far: added to the positions
    return _case("rope", **{**dict(new=0, rot=128, pairs="half", scaling="none", far=0), **kw})


def _decode(**kw):
    # window -1: every row; recalled: tokens of a list per KV head
    return _case("decode", **{**dict(n_sink=0, window=-1, recalled=0, freed=False), **kw})


def _prompt(**kw):
    return _case("prompt", **{**dict(new=2048, n_sink=0, window=-1, freed=False), **kw})


def _copy(**kw):
    # kind: fork (the last page of other sequences), kept (a list per KV head), contiguous
    return _case("copy", **{**dict(kind="fork", rows=64), **kw})


def listed():
    return [
        # one token of one user: a launch and its latency
        _rope(name="rope_token", N=2048),
        # a token of 64 users; pairs lie next to each other and half of a head turns
        _rope(name="rope_b64", S=64, N=700, spread=0.9, page=16, rot=64, pairs="adjacent"),
        # ragged prompts at far positions with frequencies scaled for long contexts
        _rope(name="rope_prompts", S=4, N=2999, spread=0.4, new=2999, scaling="ramp", far=120000),
        # one user, a short context: latency
        _decode(name="decode_2k", N=2048, page=16),
        # 32 users some way into their conversations: ragged lengths
        _decode(name="decode_b32", S=32, N=8191, spread=0.9),
        # long contexts: the rate of the memory
        _decode(name="decode_128k_b4", S=4, N=131072),
        # a recalled list per head with sinks and the tokens generated since, pages of odd size
        _decode(name="decode_recalled", S=16, N=16384, page=40, n_sink=16, window=217,
                recalled=1024),
        # a few new tokens after long contexts: nearly a decode step
        _prompt(name="prompt_few", S=2, N=30011, spread=0.3, new=17),
        # one prompt from its beginning
        _prompt(name="prompt_8k", N=8192, new=8192),
        # chunks of ragged prompts with a window and sinks, larger groups, pages that end inside tiles
        _prompt(name="prompt_window", S=3, Hkv=4, G=8, N=7001, spread=0.5, page=20, new=4099,
                n_sink=16, window=1024, freed=True),
        # the last, shared page of forked sequences gets a copy of its own
        _copy(name="copy_fork", S=24, N=1500, spread=0.8, page=32, rows=32),
        # rows kept of every head's cache after eviction, into fresh pages
        _copy(name="copy_kept", S=8, N=8192, spread=0.5, kind="kept", rows=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "decode", "decode", "prompt", "prompt", "copy"])
    while True:
        c = dict(S=_log(rng, 1, 64), Hkv=rng.choice([1, 2, 4, 8, 8]), G=rng.choice([1, 2, 4, 4, 8]),
                 N=_log(rng, 1, 131072), spread=rng.choice([0.0, 0.3, 0.9]),
                 page=rng.choice([16, 16, 32, 64, 64, 128, 256, rng.randint(1, 100)]),
                 dtype=rng.choice(["bf16"] * 5 + ["f32"]))
        if c["S"] * c["Hkv"] * c["N"] > 4 * 8 * 131072 // (2 if c["dtype"] == "f32" else 1):
            continue
        masked = dict(n_sink=rng.choice([0, 4, 16, rng.randint(1, 200)]), window=_log(rng, 1, 4096),
                      freed=rng.choice([False, True]))
        if op == "rope":
            c["new"] = rng.choice([0, 0, c["N"], _log(rng, 1, c["N"])])
            if c["S"] * c["N"] > 16384:
                continue
            return _rope(**c, rot=rng.choice([128, 128, 64, 2 * rng.randint(1, 64)]),
                         pairs=rng.choice(["half", "adjacent"]),
                         scaling=rng.choice(["none", "linear", "base", "ramp", "bands"]),
                         far=rng.choice([0, 0, 100000, 1000000]))
        if op == "decode":
            form = rng.choice(["whole", "whole", "window", "recalled"])
            if form == "whole":
                return _decode(**c)
            if form == "window":
                return _decode(**c, **masked)
            if c["N"] < 64:
                continue
            return _decode(**c, n_sink=rng.choice([0, 16]), window=rng.randint(0, c["N"] // 4),
                           recalled=_log(rng, 1, min(4096, c["N"] // 2)))
        if op == "prompt":
            c["dtype"], c["N"] = "bf16", _log(rng, 16, 65536)
            c["new"] = rng.choice([c["N"], _log(rng, 1, c["N"]), _log(rng, 1, min(c["N"], 32))])
            # as many sequences as stay within the pairs, heads and rows of the largest listed case
            c["S"] = min(c["S"], 32 * 8192 * 8192 // 2 // (c["new"] * c["N"] * c["Hkv"] * c["G"]),
                         4 * 8 * 131072 // (c["Hkv"] * c["N"]))
            if c["S"] < 1:
                continue
            return _prompt(**c, **(masked if rng.random() < 0.5 else {}))
        kind = rng.choice(["fork", "kept", "contiguous"])
        if c["S"] * c["Hkv"] * c["N"] > 8 * 8 * 8192:
            continue
        return _copy(**c, kind=kind, rows={"fork": c["page"], "kept": rng.randint(1, c["N"]),
                                           "contiguous": c["N"]}[kind])


# ---------------------------------------------------------------- sizes
def _sizes(case):
    """Rows of every sequence after the call, and how many of them are new."""
    N, spread = case["N"], case["spread"]
    lens = [max(1, int(N * (1.0 - spread * ((s * 0.6180339887) % 1.0)))) for s in range(case["S"])]
    most = max(1, case.get("new", 1))
    news = [min(n, max(1, int(most * (1.0 - spread * ((s * 0.3819660113) % 1.0)))))
            for s, n in enumerate(lens)]
    return lens, news


def _rows_seen(case, lens, news):
    """Rows of K and V that some query sees, and the pairs of query and row, over all sequences."""
    rows = pairs = 0
    for n, m in zip(lens, news):
        p = np.arange(n - m, n, dtype=np.int64)
        sink, w = case["n_sink"], case["window"]
        if w < 0:
            rows, pairs = rows + n, pairs + int((p + 1).sum())
            continue
        lo = np.maximum(np.minimum(sink, p + 1), p - w + 1)
        pairs += int((np.minimum(sink, p + 1) + p + 1 - lo).sum())
        rows += min(sink, n) + n - max(min(sink, n), min(n, n - m - w + 1))
    return rows, pairs


def work(case):
    S, Hkv, G, op = case["S"], case["Hkv"], case["G"], case["op"]
    lens, news = _sizes(case)
    size = 2 if case["dtype"] == "bf16" else 4
    row = D * size
    T = sum(news)
    if op == "rope":
        return dict(bytes=2 * T * Hkv * (G + 2) * row, flops=3 * T * Hkv * (G + 1) * case["rot"])
    if op == "copy":
        rows = sum(_copied(case, lens))
        return dict(bytes=4 * rows * Hkv * row + (4 * rows * Hkv if case["kind"] == "kept" else 0),
                    flops=0)
    if case.get("recalled"):
        rows = pairs = sum(min(case["n_sink"], n) + _list_length(case, n) +
                           max(0, n - max(case["n_sink"], n - case["window"])) for n in lens)
    else:
        rows, pairs = _rows_seen(case, lens, news)
    return dict(bytes=2 * T * Hkv * G * row + 2 * rows * Hkv * row, flops=4 * D * pairs * Hkv * G)


def _copied(case, lens):
    if case["kind"] == "fork":                            # rows in the page that the last row is in
        return [(n - 1) % case["page"] + 1 for n in lens]
    return [min(n, case["rows"]) for n in lens]


def _list_length(case, n):
    return min(case["recalled"], max(0, n - case["n_sink"] - case["window"]))


# ---------------------------------------------------------------- inputs
class _Inputs:
    def __init__(self, case, seed):
        self.c = case
        self.dtype = _TYPES[case["dtype"]]
        self.g = torch.Generator(device=DEV).manual_seed(int(seed))
        m = self.randn(case["Hkv"], 64, D)
        self.centers = m / m.norm(dim=-1, keepdim=True)

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g, device=DEV)

    def keys(self, *lead):
        """[*lead, Hkv, n, D] with n the last of lead: 3 * center + noise of 0.5 per channel."""
        *lead, n = lead
        Hkv = self.c["Hkv"]
        pick = torch.randint(0, 64, (*lead, Hkv, n), generator=self.g, device=DEV)
        k = self.centers[torch.arange(Hkv, device=DEV)[:, None], pick].mul_(3.0)
        return k.add_(self.randn(*k.shape), alpha=0.5).to(self.dtype)

    def queries(self, T):
        """[T, Hq, D], each at a center of its KV head."""
        Hkv, G = self.c["Hkv"], self.c["G"]
        pick = torch.randint(0, 64, (T, Hkv, G), generator=self.g, device=DEV)
        q = self.centers[torch.arange(Hkv, device=DEV)[:, None], pick] * 3.0
        return q.add_(self.randn(*q.shape), alpha=0.5).reshape(T, Hkv * G, D).to(self.dtype)

    def table(self, lens, spare=3):
        """Page numbers [S, most pages], in random order, -1 behind the last; and the pool's size."""
        ps = self.c["page"]
        each = [(n + ps - 1) // ps for n in lens]
        total = sum(each) + spare
        perm = torch.randperm(total, generator=self.g, device=DEV).to(torch.int32).cpu()
        t = torch.full((len(lens), max(each)), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(each):
            t[s, :n] = perm[at:at + n]
            at += n
        return t.to(DEV), total

    def pool(self, n_pages):
        c = self.c
        K = torch.empty(n_pages, c["Hkv"], c["page"], D, dtype=self.dtype, device=DEV)
        V = torch.empty_like(K)
        part = max(1, (1 << 25) // (c["Hkv"] * c["page"] * D))
        for a in range(0, n_pages, part):                 # small temporaries
            n = min(part, n_pages - a)
            K[a:a + n] = self.keys(n, c["page"])
            V[a:a + n] = self.randn(n, c["Hkv"], c["page"], D).to(self.dtype)
        return K, V


def _frequencies(case):
    """Turning rates [rot / 2] and the factor on the cosines and sines."""
    rot, base, f, full = case["rot"], 10000.0, 8.0, 4096
    i = np.arange(0, rot, 2, dtype=np.float64)
    w = base ** (-i / rot)
    if case["scaling"] == "linear":
        return w / f, 1.0
    if case["scaling"] == "base":
        return (base * f ** (rot / max(1.0, rot - 2.0))) ** (-i / rot), 1.0
    if case["scaling"] == "ramp":                         # by turns over the trained length: 32 to 1
        dim = lambda turns: rot * math.log(full / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(0, math.floor(dim(32.0))), min(rot - 1, math.ceil(dim(1.0)))
        ramp = np.clip((i / 2 - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return w / f * ramp + w * (1.0 - ramp), 0.1 * math.log(f) + 1.0
    if case["scaling"] == "bands":                        # by wavelength against the trained length
        mix = np.clip((full * w / (2 * math.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return (1.0 - mix) * w / f + mix * w, 1.0
    return w, 1.0


def _free_pages(table, case, lens, news):
    """Entries of pages that no query sees any more become -1."""
    ps, t = case["page"], table.cpu()
    for s, (n, m) in enumerate(zip(lens, news)):
        lo, hi = -(-case["n_sink"] // ps), max(0, n - m - case["window"] + 1) // ps
        if hi > lo:
            t[s, lo:hi] = -1
    return t.to(DEV)


def prepare(case, seed):
    x = _Inputs(case, seed)
    S, Hkv, G, op = case["S"], case["Hkv"], case["G"], case["op"]
    lens, news = _sizes(case)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    starts = ints([0] + list(np.cumsum(news)))
    table, n_pages = x.table(lens)
    s = dict(case=case, lengths=ints(lens), starts=starts, news=news, lens=lens, table=table)
    s["K"], s["V"] = x.pool(n_pages)
    T = sum(news)
    if op == "rope":
        if not case["new"]:
            T = S
        # the views of one projection's output that a model has in hand
        qkv = x.randn(T, Hkv * (G + 2) * D).to(x.dtype)
        q, k, v = qkv.split([Hkv * G * D, Hkv * D, Hkv * D], dim=1)
        s["q"], s["k"], s["v"] = (a.unflatten(1, (-1, D)) for a in (q, k, v))
        w, s["factor"] = _frequencies(case)
        s["freq"] = torch.tensor(w, dtype=torch.float32, device=DEV)
        s["positions"] = None
        if case["far"]:
            s["positions"] = (_rows(s)[1] + case["far"]).to(torch.int32)
        s["out"] = torch.empty(T, Hkv * G, D, dtype=x.dtype, device=DEV)
    elif op == "copy":
        s["counts"] = ints(_copied(case, lens))
        s["src_seq"] = s["begin"] = s["kept"] = None
        if case["kind"] == "contiguous":
            s["table2"] = torch.arange(S, dtype=torch.int32, device=DEV)[:, None]
            s["K2"] = torch.zeros(S, Hkv, case["N"], D, dtype=x.dtype, device=DEV)
        else:
            s["table2"], n2 = x.table(lens)
            s["K2"] = torch.zeros(n2, Hkv, case["page"], D, dtype=x.dtype, device=DEV)
        s["V2"] = torch.zeros_like(s["K2"])
        if case["kind"] == "fork":
            s["begin"] = ints([(n - 1) // case["page"] * case["page"] for n in lens])
            # every sequence is copied from one that is at least as long
            order = sorted(range(S), key=lambda i: -lens[i])
            rank = {i: r for r, i in enumerate(order)}
            s["src_seq"] = ints([order[rank[i] // 2] for i in range(S)])
        if case["kind"] == "kept":
            rows = min(case["rows"], max(lens))
            score = torch.rand(S, Hkv, max(lens), generator=x.g, device=DEV)
            score[torch.arange(max(lens), device=DEV)[None] .expand(S, -1)[:, None].expand(-1, Hkv, -1)
                  >= s["lengths"].long()[:, None, None]] = 2.0
            kept = score.topk(rows, dim=-1, largest=False, sorted=True).indices
            order = torch.arange(rows, device=DEV) < s["counts"].long()[:, None, None]
            s["kept"] = torch.where(order, kept, kept.new_tensor(1 << 30)).sort(-1).values.to(torch.int32)
    else:
        s["q"] = x.queries(T if op == "prompt" else S)
        s["out"] = torch.empty_like(s["q"])
        if case["freed"]:
            s["table"] = _free_pages(table, case, lens, news if op == "prompt" else [1] * S)
        s["listed"] = s["counts"] = None
        if case.get("recalled"):
            # what is neither a sink nor in the window is recalled, in an order of its own
            r, n = case["recalled"], torch.arange(max(lens), device=DEV)
            score = torch.rand(S, Hkv, max(lens), generator=x.g, device=DEV)
            ln = s["lengths"].long()[:, None, None]
            score = score.masked_fill((n < case["n_sink"]) | (n >= ln - case["window"]), 2.0)
            s["listed"] = score.topk(r, dim=-1, largest=False).indices.to(torch.int32)
            s["counts"] = ints([_list_length(case, n) for n in lens])[:, None].expand(S, Hkv).contiguous()
    if own:
        _handles(s)
    return s


def _handles(s):
    """The shape, caches and workspace that a program keeps beside its tensors."""
    import paper_2412_03213_amd as ck
    case = s["case"]
    s["ck"] = ck
    dt = ck.CK_BF16 if case["dtype"] == "bf16" else ck.CK_F32
    n = s["table"].shape[1] * case["page"]
    s["sh"] = ck.Shape(case["S"], case["Hkv"] * case["G"], case["Hkv"], n, 1, dtype=dt)
    s["kv"] = ck.PagedKV(s["K"], s["V"], s["table"])
    if case["op"] == "copy":
        s["kv2"] = ck.PagedKV(s["K2"], s["V2"], s["table2"])
    if case["op"] == "decode":
        s["ws"] = ck.paged_decode_workspace(s["sh"], DEV)
    if case["op"] == "prompt":
        s["ws"] = ck.prompt_workspace(s["sh"], s["q"].shape[0], DEV)


# ---------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _RUN[s["case"]["op"]](s)


def _run_own(s):
    case, ck = s["case"], s["ck"]
    if case["op"] == "rope":
        ck.ck_rope_append(s["sh"], s["q"], s["k"], s["v"], s["kv"], s["lengths"], s["freq"], s["out"],
                          q_starts=s["starts"] if case["new"] else None, positions=s["positions"],
                          attn_factor=s["factor"], interleaved=case["pairs"] == "adjacent")
        return s["out"], s["K"], s["V"]
    if case["op"] == "decode":
        ck.ck_paged_decode_attn(s["sh"], s["q"], s["kv"], s["lengths"], s["out"],
                                n_sink=case["n_sink"], window=case["window"], token_idx=s["listed"],
                                n_tokens=s["counts"], workspace=s["ws"])
        return s["out"]
    if case["op"] == "prompt":
        ck.ck_prompt_attn(s["sh"], s["q"], s["starts"], s["kv"], s["lengths"], s["out"],
                          n_sink=case["n_sink"], window=case["window"], workspace=s["ws"])
        return s["out"]
    ck.ck_copy_rows(s["sh"], s["kv"], s["kv2"], s["counts"], case["rows"], row_idx=s["kept"],
                    begin=s["begin"], src_seq=s["src_seq"])
    return s["K2"], s["V2"]


def _rows(s):
    """Sequence and row in its cache of every new token, [T] each."""
    if not s["case"].get("new"):
        return torch.arange(s["case"]["S"], device=DEV), s["lengths"].long() - 1
    starts = s["starts"].long()
    t = torch.arange(sum(s["news"]), device=DEV)
    seq = torch.bucketize(t, starts[1:], right=True)
    return seq, s["lengths"].long()[seq] - starts[seq + 1] + t


def _turn(x, cos, sin, rot, adjacent):
    """The first rot channels of x [T, H, D] turned pair by pair; in 32 bits, rounded once."""
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if adjacent else (y[..., :rot // 2], y[..., rot // 2:rot])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((u, v), -1).flatten(-2) if adjacent else torch.cat((u, v), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(x.dtype)


def _run_rope(s):
    case, (seq, row) = s["case"], _rows(s)
    at = row if s["positions"] is None else s["positions"]
    angle = at.double()[:, None] * s["freq"].double()     # 32 bits would lose the angles of far positions
    angle = torch.remainder(angle, 2 * math.pi).float()[:, None]
    cos, sin = angle.cos() * s["factor"], angle.sin() * s["factor"]
    adjacent = case["pairs"] == "adjacent"
    page = s["table"].long()[seq, row // case["page"]]
    slot = row % case["page"]
    s["K"][page, :, slot] = _turn(s["k"], cos, sin, case["rot"], adjacent)
    s["V"][page, :, slot] = s["v"]
    return _turn(s["q"], cos, sin, case["rot"], adjacent), s["K"], s["V"]


def _gathered(pool, table, page, n):
    """Rows 0..n-1 of every sequence in 32 bits, [S, Hkv, n, D], and whether their page is there."""
    r = torch.arange(n, device=DEV)
    p = table.long()[:, r // page]
    rows = pool[p.clamp(min=0), :, r % page]               # [S, n, Hkv, D]
    return rows.permute(0, 2, 1, 3).float(), p >= 0


def _attend(q, K, V, seen):
    """softmax(q K^T / sqrt(d)) V over the rows seen: q [S, Hkv, M, D], K, V [S, Hkv, n, D], seen
    broadcast to [S, Hkv, M, n]; nothing seen gives zeros."""
    sc = torch.matmul(q, K.transpose(-1, -2).contiguous()).mul_(D ** -0.5)
    sc = sc.masked_fill_(~seen, -math.inf)
    top = sc.amax(-1, keepdim=True).clamp_(min=-1e30)
    p = sc.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, V) / torch.where(total > 0, total, 1.0)


def _run_decode(s):
    case = s["case"]
    S, Hkv, G, n = case["S"], case["Hkv"], case["G"], max(s["lens"])
    ln = s["lengths"].long()
    q = s["q"].float().view(S, Hkv, G, D)
    r = torch.arange(n, device=DEV)
    if case.get("recalled"):
        # the rows of sinks, list and window beside each other
        sink = torch.arange(case["n_sink"], device=DEV).expand(S, Hkv, -1)
        late = ln[:, None, None] - 1 - torch.arange(case["window"], device=DEV).expand(S, Hkv, -1)
        rows = torch.cat((sink, s["listed"].long(), late), -1)
        ok = torch.cat((sink < ln[:, None, None],
                        torch.arange(case["recalled"], device=DEV) < s["counts"].long()[..., None],
                        late >= case["n_sink"]), -1)
        rows = rows.clamp(0, n - 1)
        page = s["table"].long()[torch.arange(S, device=DEV)[:, None, None], rows // case["page"]]
        ok &= page >= 0
        h = torch.arange(Hkv, device=DEV)[:, None]
        at = (page.clamp(min=0), h, rows % case["page"])
        out = _attend(q, s["K"][at].float(), s["V"][at].float(), ok[:, :, None])
        return out.reshape(S, Hkv * G, D).to(s["q"].dtype)
    K, there = _gathered(s["K"], s["table"], case["page"], n)
    V, _ = _gathered(s["V"], s["table"], case["page"], n)
    seen = there & (r < ln[:, None])
    if case["window"] >= 0:
        seen &= (r < case["n_sink"]) | (r >= ln[:, None] - case["window"])
    return _attend(q, K, V, seen[:, None, None]).reshape(S, Hkv * G, D).to(s["q"].dtype)


def _run_prompt(s):
    case = s["case"]
    S, Hkv, G, n, m = case["S"], case["Hkv"], case["G"], max(s["lens"]), max(s["news"])
    K, there = _gathered(s["K"], s["table"], case["page"], n)
    V, _ = _gathered(s["V"], s["table"], case["page"], n)
    seq, row = _rows(s)
    t = torch.arange(seq.numel(), device=DEV) - s["starts"].long()[seq]
    q = torch.zeros(S, m, Hkv, G, D, device=DEV)
    q[seq, t] = s["q"].float().view(-1, Hkv, G, D)
    at = torch.full((S, m), -1, device=DEV)
    at[seq, t] = row                                      # -1: no query, sees nothing
    r = torch.arange(n, device=DEV)
    seen = (r <= at[..., None]) & there[:, None]
    if case["window"] >= 0:
        seen &= (r < case["n_sink"]) | (r > at[..., None] - case["window"])
    q = q.permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * m, D)
    out = _attend(q, K, V, seen[:, None].repeat(1, 1, G, 1))
    out = out.view(S, Hkv, G, m, D).permute(0, 3, 1, 2, 4)[seq, t]
    return out.reshape(-1, Hkv * G, D).to(s["q"].dtype)


def _run_copy(s):
    case = s["case"]
    S, Hkv, rows = case["S"], case["Hkv"], case["rows"]
    j = torch.arange(rows, device=DEV)
    seq = torch.arange(S, device=DEV)
    src_seq = seq if s["src_seq"] is None else s["src_seq"].long()
    dst = j + (0 if s["begin"] is None else s["begin"].long()[:, None])
    dst = dst.expand(S, rows)[:, None].expand(S, Hkv, rows)
    src = dst if s["kept"] is None else s["kept"].long()
    if src.shape[-1] < rows:
        src = torch.nn.functional.pad(src, (0, rows - src.shape[-1]))
    s_, h_, j_ = (j < s["counts"].long()[:, None])[:, None].expand(S, Hkv, rows).nonzero(as_tuple=True)
    a, b = src[s_, h_, j_], dst[s_, h_, j_]
    size2 = s["K2"].shape[2]
    page, page2 = s["table"].long()[src_seq[s_], a // case["page"]], s["table2"].long()[s_, b // size2]
    s["K2"][page2, h_, b % size2] = s["K"][page, h_, a % case["page"]]
    s["V2"][page2, h_, b % size2] = s["V"][page, h_, a % case["page"]]
    return s["K2"], s["V2"]


_RUN = dict(rope=_run_rope, decode=_run_decode, prompt=_run_prompt, copy=_run_copy)


# ---------------------------------------------------------------- from the definitions, in 64 bits
def _cache64(s, pool, seq, rows):
    """Rows of one sequence's cache [Hkv, n, D] and which of them are on a page."""
    ps = s["case"]["page"]
    page = s["table"][seq].long()[rows // ps]
    return pool[page.clamp(min=0), :, rows % ps].double().transpose(0, 1), page >= 0


def _softmax_mean64(q, K, V, seen):
    """q [M, D], K and V [n, D], seen [M, n] -> [M, D]; blocks of queries bound the memory."""
    out = torch.zeros_like(q)
    for a in range(0, q.shape[0], 2048):
        w = (q[a:a + 2048] @ K.T) / math.sqrt(D)
        w = torch.where(seen[a:a + 2048], w, -math.inf)
        w = torch.exp(w - w.max(-1, keepdim=True).values.nan_to_num(neginf=0.0))
        total = w.sum(-1, keepdim=True)
        out[a:a + 2048] = torch.where(total > 0, (w @ V) / total, 0.0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    Hkv, G = case["Hkv"], case["G"]
    if case["op"] == "copy":
        K, V = s["K2"].double(), s["V2"].double()
        for i, n in enumerate(_copied(case, s["lens"])):
            src = i if s["src_seq"] is None else int(s["src_seq"][i])
            first = 0 if s["begin"] is None else int(s["begin"][i])
            to = torch.arange(first, first + n, device=DEV)
            page2, slot2 = s["table2"][i].long()[to // K.shape[2]], to % K.shape[2]
            for h in range(Hkv):
                at = to if s["kept"] is None else s["kept"][i, h, :n].long()
                for old, new in ((s["K"], K), (s["V"], V)):
                    page = s["table"][src].long()[at // case["page"]]
                    new[page2, h, slot2] = old[page, h, at % case["page"]].double()
        return K, V
    if case["op"] == "rope":
        K, V = s["K"].double(), s["V"].double()
        rot, half = case["rot"], case["rot"] // 2
        i = torch.arange(half, device=DEV)
        first, second = (2 * i, 2 * i + 1) if case["pairs"] == "adjacent" else (i, i + half)
        q, k = s["q"].double().clone(), s["k"].double().clone()
        t = 0
        for b, (n, m) in enumerate(zip(s["lens"], s["news"] if case["new"] else [1] * case["S"])):
            row = torch.arange(n - m, n, device=DEV)
            z = torch.polar(torch.full((m, half), s["factor"], dtype=torch.float64, device=DEV),
                            (row + case["far"]).double()[:, None] * s["freq"].double())[:, None]
            for x in (q, k):
                part = x[t:t + m]
                c = torch.complex(part[..., first], part[..., second]) * z
                part[..., first], part[..., second] = c.real, c.imag
            page = s["table"][b].long()[row // case["page"]]
            K[page, :, row % case["page"]] = k[t:t + m]
            V[page, :, row % case["page"]] = s["v"][t:t + m].double()
            t += m
        return q, K, V
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    t = 0
    for b, (n, m) in enumerate(zip(s["lens"], s["news"] if case["op"] == "prompt" else [1] * case["S"])):
        every = torch.arange(n, device=DEV)
        K, there = _cache64(s, s["K"], b, every)
        V, _ = _cache64(s, s["V"], b, every)
        p = torch.arange(n - m, n, device=DEV)[:, None]
        seen = (every <= p) & there
        if case["window"] >= 0:
            near = (every < case["n_sink"]) | (every > p - case["window"])
            seen = seen & near
        for h in range(Hkv):
            vis = seen
            if case.get("recalled"):
                vis = seen.clone()
                vis[:, s["listed"][b, h, :int(s["counts"][b, h])].long()] = True
                vis &= there
            q = s["q"][t:t + m, h * G:(h + 1) * G].double()
            o = _softmax_mean64(q.reshape(m * G, D), K[h], V[h], vis.repeat_interleave(G, 0))
            out[t:t + m, h * G:(h + 1) * G] = o.view(m, G, D)
        t += m
    return out
