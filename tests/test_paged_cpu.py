"""Host side of the operators on paged caches: refusals before anything is enqueued, and the turning rates
of rotary positions."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2412_03213_amd as ck
from paper_2412_03213_amd import binding

A = 4096                                                # an aligned address that is never dereferenced
SH = ck.Shape(2, 8, 2, 64, 1)
EINVALID, EUNSUPPORTED, EWORKSPACE, EMISALIGNED = -1, -2, -3, -4


def kv(**k):
    v = dict(K=A, V=A, page_table=A, n_pages=8, page_size=16, n_seqs=2, pages_per_seq=4)
    v.update(k)
    return binding._CkPagedKV(**v)


BAD_CACHES = [(None, EINVALID), (dict(K=None), EINVALID), (dict(V=None), EINVALID),
              (dict(page_table=None), EINVALID), (dict(K=A + 8), EMISALIGNED), (dict(V=A + 2), EMISALIGNED),
              (dict(page_table=A + 4), EMISALIGNED), (dict(n_pages=0), EINVALID),
              (dict(page_size=0), EINVALID), (dict(page_size=-1), EINVALID), (dict(pages_per_seq=0), EINVALID),
              (dict(n_seqs=1), EINVALID), (dict(n_pages=2 ** 26, page_size=32), EUNSUPPORTED),
              (dict(page_size=2 ** 20, pages_per_seq=2 ** 11), EUNSUPPORTED)]

SHAPES = [(dict(Hq=6), EUNSUPPORTED), (dict(Hq=5), EINVALID), (dict(d=64), EUNSUPPORTED), (dict(S=0), EINVALID),
          (dict(dtype=2), EINVALID)]


def code(f, *args, **kw):
    with pytest.raises(ck.ClusterKVError) as e:
        f(*args, **kw)
    return e.value.code


def shape(**k):
    return ck.Shape(**{**dict(S=2, Hq=8, Hkv=2, N_cap=64, C_cap=1), **k})


def rope(sh=SH, n=2, q=A, k=A, v=A, q_out=A, qs=1024, ks=256, vs=256, starts=None, lengths=A, positions=None,
         freqs=A, rot=128, factor=1.0, flags=0, cache=kv()):
    s = sh.c()
    binding._check(binding.load_library().ck_rope_append(
        ctypes.byref(s), q, k, v, qs, ks, vs, n, starts, lengths, positions, freqs, rot, factor, flags, q_out,
        ctypes.byref(cache) if cache is not None else None, None))


def decode(sh=SH, q=A, cache=kv(), lengths=A, n_sink=0, window=-1, idx=None, n_tok=None, stride=0, most=0,
           scale=1.0, out=A, ws=A, size=1 << 30):
    s = sh.c()
    binding._check(binding.load_library().ck_paged_decode_attn(
        ctypes.byref(s), q, ctypes.byref(cache) if cache is not None else None, lengths, n_sink, window, idx, n_tok,
        stride, most, scale, out, ws, size, None))


def prompt(sh=SH, q=A, n=5, starts=A, cache=kv(), lengths=A, n_sink=0, window=-1, scale=1.0, out=2 * A, ws=A,
           size=1 << 40):
    s = sh.c()
    binding._check(binding.load_library().ck_prompt_attn(
        ctypes.byref(s), q, n, starts, ctypes.byref(cache) if cache is not None else None, lengths, n_sink, window,
        scale, out, ws, size, None))


def copy(sh=SH, src=kv(), dst=kv(), n=A, most=4, idx=None, stride=4, begin=None, seq=None):
    s = sh.c()
    binding._check(binding.load_library().ck_copy_rows(
        ctypes.byref(s), ctypes.byref(src) if src is not None else None,
        ctypes.byref(dst) if dst is not None else None, n, most, idx, stride, begin, seq, None))


@pytest.mark.parametrize("bad,want", BAD_CACHES)
def test_caches_that_are_refused(bad, want):
    c = kv(**bad) if bad is not None else None
    assert code(rope, cache=c) == want
    assert code(decode, cache=c) == want
    assert code(prompt, cache=c) == want
    assert code(copy, dst=c) == want
    if bad != dict(n_seqs=1):
        assert code(copy, src=c) == want
        assert code(copy, src=c, seq=A) == want


@pytest.mark.parametrize("bad,want", SHAPES)
def test_shapes_that_are_refused(bad, want):
    for f in (rope, decode, prompt, copy):
        assert code(f, sh=shape(**bad)) == want


@pytest.mark.parametrize("bad,want", [
    (dict(n=0), EINVALID), (dict(n=3), EINVALID), (dict(n=(1 << 24) + 1, starts=A), EUNSUPPORTED),
    (dict(rot=3), EINVALID), (dict(rot=0), EINVALID), (dict(rot=130), EINVALID), (dict(flags=2), EINVALID),
    (dict(factor=math.inf), EINVALID), (dict(factor=math.nan), EINVALID), (dict(q=None), EINVALID),
    (dict(q_out=None), EINVALID), (dict(k=None), EINVALID), (dict(v=None), EINVALID), (dict(lengths=None), EINVALID),
    (dict(freqs=None), EINVALID), (dict(q=A + 4), EMISALIGNED), (dict(k=A + 8), EMISALIGNED),
    (dict(positions=A + 4), EMISALIGNED), (dict(starts=A + 4), EMISALIGNED), (dict(lengths=A + 4), EMISALIGNED),
    (dict(qs=1016), EINVALID), (dict(qs=1028), EMISALIGNED), (dict(ks=255), EINVALID), (dict(vs=260), EMISALIGNED),
    (dict(qs=1032), EINVALID), (dict(ks=1 << 41), EUNSUPPORTED)])
def test_rope_append_refuses(bad, want):
    assert code(rope, **bad) == want


@pytest.mark.parametrize("bad,want", [
    (dict(q=None), EINVALID), (dict(out=None), EINVALID), (dict(lengths=None), EINVALID), (dict(n_sink=-1), EINVALID),
    (dict(scale=0.0), EINVALID), (dict(scale=math.nan), EINVALID), (dict(idx=A), EINVALID), (dict(n_tok=A), EINVALID),
    (dict(idx=A, n_tok=A, window=-1), EINVALID), (dict(idx=A, n_tok=A, window=4, most=5, stride=4), EINVALID),
    (dict(idx=A, n_tok=A, window=4, most=-1, stride=4), EINVALID), (dict(q=A + 2), EMISALIGNED),
    (dict(idx=A + 4, n_tok=A, window=4), EMISALIGNED), (dict(ws=None), EWORKSPACE), (dict(ws=A + 8), EMISALIGNED),
    (dict(size=1024), EWORKSPACE)])
def test_paged_decode_refuses(bad, want):
    assert code(decode, **bad) == want


@pytest.mark.parametrize("bad,want", [
    (dict(sh=shape(dtype=ck.CK_F32)), EUNSUPPORTED), (dict(n=0), EINVALID), (dict(n=1 << 25), EUNSUPPORTED),
    (dict(q=None), EINVALID), (dict(out=None), EINVALID), (dict(out=A), EINVALID), (dict(starts=None), EINVALID),
    (dict(lengths=None), EINVALID), (dict(n_sink=-1), EINVALID), (dict(scale=-1.0), EINVALID),
    (dict(q=A + 8), EMISALIGNED), (dict(ws=None), EWORKSPACE), (dict(size=1), EWORKSPACE)])
def test_prompt_attention_refuses(bad, want):
    assert code(prompt, **bad) == want


@pytest.mark.parametrize("bad,want", [
    (dict(n=None), EINVALID), (dict(most=0), EINVALID), (dict(most=(1 << 28) + 1), EUNSUPPORTED),
    (dict(idx=A, stride=3), EINVALID), (dict(idx=A + 4), EMISALIGNED), (dict(begin=A + 4), EMISALIGNED),
    (dict(seq=A + 4), EMISALIGNED)])
def test_copy_rows_refuses(bad, want):
    assert code(copy, **bad) == want


def test_tensors_of_other_shapes_and_types_are_refused():
    bf = torch.bfloat16
    K = torch.zeros(8, 2, 16, 128, dtype=bf)
    table = torch.zeros(2, 4, dtype=torch.int32)
    cache = ck.PagedKV(K, K.clone(), table)
    q, out = torch.zeros(2, 8, 128, dtype=bf), torch.zeros(2, 8, 128, dtype=bf)
    n = torch.ones(2, dtype=torch.int32)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError):
        ck.PagedKV(K, K.float(), table)
    with pytest.raises(ValueError):
        ck.PagedKV(K, K.clone(), table.long())
    with pytest.raises(ValueError):
        ck.PagedKV(K.transpose(0, 1), K.transpose(0, 1))
    for sh in (shape(Hkv=4), shape(dtype=ck.CK_F32)):
        with pytest.raises(ValueError):
            ck.ck_paged_decode_attn(sh, q, cache, n, out, workspace=ws)
    with pytest.raises(ValueError):
        ck.ck_paged_decode_attn(SH, q, cache, n.long(), out, workspace=ws)
    with pytest.raises(ValueError):
        ck.ck_paged_decode_attn(SH, q[:1], cache, n, out, workspace=ws)
    with pytest.raises(ValueError):
        ck.ck_prompt_attn(SH, q, n, cache, n, out, workspace=ws)           # q_starts has S + 1 entries
    k = torch.zeros(2, 2, 128, dtype=bf)
    f = torch.zeros(64)
    with pytest.raises(ValueError):
        ck.ck_rope_append(SH, q, k, k, cache, n, f.double(), out)
    with pytest.raises(ValueError):
        ck.ck_rope_append(SH, q[..., ::2], k, k, cache, n, f, out)
    with pytest.raises(ValueError):
        ck.ck_rope_append(SH, q, k, torch.zeros(3, 2, 128, dtype=bf), cache, n, f, out)
    with pytest.raises(ValueError):
        ck.ck_copy_rows(SH, cache, cache, n, 4, row_idx=torch.zeros(2, 4, dtype=torch.int32))


def test_workspaces():
    for S, Hq, Hkv in ((1, 8, 8), (64, 32, 8), (1000, 8, 1)):
        sh = shape(S=S, Hq=Hq, Hkv=Hkv)
        need = (S * Hkv * 8 + 255) // 256 * 256 + ((512 + S * Hkv) * (Hq // Hkv) * 130 * 4 + 255) // 256 * 256
        assert ck.ck_workspace_bytes(sh, binding.CK_WS_PAGED_ATTN, 0) >= need
        assert ck.ck_workspace_bytes(sh, binding.CK_WS_PROMPT_ATTN, 100) > 0
        assert ck.ck_workspace_bytes(sh, binding.CK_WS_PROMPT_ATTN, 0) == 0
        sizes = [ck.ck_workspace_bytes(sh, binding.CK_WS_PROMPT_ATTN, n) for n in (1, 17, 1000, 100000)]
        assert sizes == sorted(sizes)                     # enough for fewer rows too


def plain_rates(rot, base=10000.0):
    return base ** (-np.arange(0, rot, 2) / rot)


@pytest.mark.parametrize("rot", [2, 6, 64, 128])
def test_rates_plain_linear_base(rot):
    w = plain_rates(rot)
    f, a = ck.ck_rope_frequencies(ck.CK_ROPE_PLAIN, rot)
    assert a == 1.0 and np.allclose(f.numpy(), w, rtol=2 ** -23, atol=0)
    f, a = ck.ck_rope_frequencies(ck.CK_ROPE_LINEAR, rot, factor=4.0)
    assert a == 1.0 and np.allclose(f.numpy(), w / 4, rtol=2 ** -23, atol=0)
    if rot > 2:
        # the slowest pair turns `factor` times slower, the fastest as before
        f, a = ck.ck_rope_frequencies(ck.CK_ROPE_BASE, rot, factor=4.0)
        assert f[0] == 1.0 and np.isclose(f[-1].item(), w[-1] / 4, rtol=1e-6) and a == 1.0
        assert (np.diff(f.numpy()) < 0).all()


@pytest.mark.parametrize("kind", [ck.CK_ROPE_RAMP, ck.CK_ROPE_BANDS])
@pytest.mark.parametrize("rot", [64, 128])
def test_rates_by_turns_keep_the_fast_and_slow_the_slow(kind, rot):
    L, fast, slow, factor = 4096.0, 32.0, 1.0, 8.0
    w = plain_rates(rot)
    f, a = ck.ck_rope_frequencies(kind, rot, factor=factor, trained_len=L, fast=fast, slow=slow)
    f = f.numpy().astype(np.float64)
    turns = L * w / (2 * math.pi)
    # the ramp over j may begin and end one pair off the exact ones: its ends are whole pairs
    off = 1.4 if kind == ck.CK_ROPE_RAMP else 1.0
    keep, slowed = turns > fast * off, turns < slow / off
    assert keep.any() and slowed.any()
    assert np.allclose(f[keep], w[keep], rtol=1e-6) and np.allclose(f[slowed], w[slowed] / factor, rtol=1e-6)
    assert ((f <= w * (1 + 1e-6)) & (f >= w / factor * (1 - 1e-6))).all()
    assert a == (pytest.approx(0.1 * math.log(factor) + 1) if kind == ck.CK_ROPE_RAMP else 1.0)
    f1, a1 = ck.ck_rope_frequencies(kind, rot, factor=1.0, trained_len=L, fast=fast, slow=slow)
    assert np.allclose(f1.numpy(), w, rtol=1e-6) and a1 == 1.0


@pytest.mark.parametrize("bad", [
    dict(kind=5), dict(kind=-1), dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=130), dict(base=1.0),
    dict(base=math.nan), dict(kind=1, factor=0.5), dict(kind=2, factor=2.0, rot_dim=2),
    dict(kind=3, trained_len=0.0), dict(kind=3, fast=1.0, slow=1.0), dict(kind=4, slow=0.0),
    dict(kind=4, factor=math.inf)])
def test_rates_refuse(bad):
    with pytest.raises(ck.ClusterKVError) as e:
        ck.ck_rope_frequencies(**{**dict(kind=0, rot_dim=128, trained_len=4096.0, fast=32.0, slow=1.0, factor=2.0),
                                  **bad})
    assert e.value.code == EINVALID


def _either_way(call, name):
    """What a call raises with the native marshalling and without it."""
    lib = ck.load_library()
    seen = []
    real = getattr(lib, name)
    for form in (real, lambda *args: None):
        setattr(lib, name, form)
        try:
            with pytest.raises((ck.ClusterKVError, ValueError, ctypes.ArgumentError)) as e:
                call()
        finally:
            setattr(lib, name, real)
        seen.append((type(e.value), str(e.value)))
    return seen


_ROPE_CHANGES = {
    "refused by the library": {}, "strided heads": {"q": lambda a: a["q"].transpose(0, 1)},
    "channels apart": {"k": lambda a: torch.zeros(3, 2, 256, dtype=torch.bfloat16)[..., ::2]},
    "other type": {"v": lambda a: a["v"].float()}, "no values": {"v": lambda a: None},
    "address": {"k": lambda a: 4096}, "no queries": {"q": lambda a: None, "q_out": lambda a: None},
    "queries without an output": {"q_out": lambda a: None}, "one output row short": {"q_out": lambda a: a["q_out"][:2]},
    "wide lengths": {"lengths": lambda a: a["lengths"].long()}, "no lengths": {"lengths": lambda a: None},
    "half rates": {"freqs": lambda a: a["freqs"].bfloat16()}, "table of rates": {"freqs": lambda a: a["freqs"][None]},
    "starts": {"q_starts": lambda a: torch.zeros(3, dtype=torch.int32)},
    "positions": {"positions": lambda a: torch.zeros(2, dtype=torch.int32)},
    "whole factor": {"attn_factor": lambda a: 0}, "other heads": {"kv": lambda a: _cpu_cache(Hkv=1)},
    "other cache type": {"kv": lambda a: _cpu_cache(dtype=torch.float32)}, "no cache": {"kv": lambda a: None},
}


def _cpu_cache(Hkv=2, dtype=torch.bfloat16):
    K = torch.zeros(4, Hkv, 8, 128, dtype=dtype)
    return ck.PagedKV(K, torch.zeros_like(K), torch.zeros(3, 1, dtype=torch.int32))


@pytest.mark.parametrize("what", _ROPE_CHANGES)
def test_rope_append_refuses_the_same_calls_on_either_way(what):
    bf = dict(dtype=torch.bfloat16)
    a = dict(q=torch.zeros(3, 4, 128, **bf), k=torch.zeros(3, 2, 128, **bf), v=torch.zeros(3, 2, 128, **bf),
             kv=_cpu_cache(), lengths=torch.zeros(3, dtype=torch.int32), freqs=torch.zeros(64),
             q_out=torch.zeros(3, 4, 128, **bf), attn_factor=float("inf"))    # refused where all else is right
    for k, change in _ROPE_CHANGES[what].items():
        a[k] = change(a)
    native, general = _either_way(lambda: ck.ck_rope_append(ck.Shape(3, 4, 2, 8, 1), **a), "host_rope_append")
    assert native == general


_DECODE_CHANGES = {
    "refused by the library": {}, "strided": {"q": lambda a: a["q"].transpose(0, 1)},
    "other type": {"out": lambda a: a["out"].float()}, "no output": {"out": lambda a: None},
    "address": {"q": lambda a: 4096}, "wide lengths": {"lengths": lambda a: a["lengths"].long()},
    "list": {"token_idx": lambda a: torch.zeros(3, 2, 5, dtype=torch.int32)},
    "list of one head": {"token_idx": lambda a: torch.zeros(3, 1, 5, dtype=torch.int32)},
    "flat list": {"token_idx": lambda a: torch.zeros(30, dtype=torch.int32)},
    "counts": {"n_tokens": lambda a: torch.zeros(3, 2, dtype=torch.int32)},
    "flat counts": {"n_tokens": lambda a: torch.zeros(6, dtype=torch.int32)},
    "small workspace": {"workspace": lambda a: a["workspace"][:8], "n_sink": lambda a: 0},
    "workspace of words": {"workspace": lambda a: torch.zeros(2, dtype=torch.int32), "n_sink": lambda a: 0},
    "most": {"max_tokens": lambda a: 2.5}, "whole scale": {"softmax_scale": lambda a: 1},
    "other heads": {"kv": lambda a: _cpu_cache(Hkv=1)}, "no cache": {"kv": lambda a: None},
    "sinks": {"n_sink": lambda a: 1.0}, "wide window": {"window": lambda a: 1 << 70},
}


@pytest.mark.parametrize("what", _DECODE_CHANGES)
def test_paged_decode_refuses_the_same_calls_on_either_way(what):
    bf = dict(dtype=torch.bfloat16)
    a = dict(q=torch.zeros(3, 4, 128, **bf), kv=_cpu_cache(), lengths=torch.zeros(3, dtype=torch.int32),
             out=torch.zeros(3, 4, 128, **bf), n_sink=-1, workspace=torch.zeros(1 << 21, dtype=torch.uint8))
    for k, change in _DECODE_CHANGES[what].items():
        a[k] = change(a)
    native, general = _either_way(lambda: ck.ck_paged_decode_attn(ck.Shape(3, 4, 2, 8, 1), **a),
                                  "host_paged_decode_attn")
    assert native == general


_PROMPT_CHANGES = {
    "refused by the library": {}, "strided": {"q": lambda a: a["q"].transpose(0, 1)}, "address": {"q": lambda a: 4096},
    "other type": {"out": lambda a: a["out"].float()}, "one output row short": {"out": lambda a: a["out"][:4]},
    "starts": {"q_starts": lambda a: a["lengths"]}, "no starts": {"q_starts": lambda a: None},
    "wide lengths": {"lengths": lambda a: a["lengths"].long()}, "no cache": {"kv": lambda a: None},
    "small workspace": {"workspace": lambda a: a["workspace"][:8], "n_sink": lambda a: 0},
    "whole scale": {"softmax_scale": lambda a: 1}, "sinks": {"n_sink": lambda a: 1.0},
    "no rows": {"q": lambda a: a["q"][:0], "out": lambda a: a["out"][:0]},
}


@pytest.mark.parametrize("what", _PROMPT_CHANGES)
def test_prompt_attn_refuses_the_same_calls_on_either_way(what):
    bf, i32 = dict(dtype=torch.bfloat16), dict(dtype=torch.int32)
    a = dict(q=torch.zeros(5, 4, 128, **bf), q_starts=torch.zeros(4, **i32), kv=_cpu_cache(),
             lengths=torch.zeros(3, **i32), out=torch.zeros(5, 4, 128, **bf), n_sink=-1,
             workspace=torch.zeros(1 << 26, dtype=torch.uint8))
    for k, change in _PROMPT_CHANGES[what].items():
        a[k] = change(a)
    native, general = _either_way(lambda: ck.ck_prompt_attn(ck.Shape(3, 4, 2, 8, 1), **a), "host_prompt_attn")
    assert native == general


_COPY_CHANGES = {
    "refused by the library": {}, "wide counts": {"n_copy": lambda a: a["n_copy"].long()},
    "no counts": {"n_copy": lambda a: None}, "most": {"max_rows": lambda a: 2.5},
    "many": {"max_rows": lambda a: (1 << 32) + 1}, "short list": {"max_rows": lambda a: 8, "row_idx": lambda a: a["row_idx"][..., :4]},
    "narrow list": {"max_rows": lambda a: 8, "row_idx": lambda a: a["row_idx"][..., :4].contiguous()},
    "flat list": {"row_idx": lambda a: a["row_idx"].flatten()}, "begin": {"begin": lambda a: a["begin"][:2]},
    "source": {"src_seq": lambda a: a["begin"].float()}, "no source": {"src": lambda a: None},
    "other heads": {"dst": lambda a: _cpu_cache(Hkv=1)}, "other type": {"src": lambda a: _cpu_cache(dtype=torch.float32)},
}


@pytest.mark.parametrize("what", _COPY_CHANGES)
def test_copy_rows_refuses_the_same_calls_on_either_way(what):
    i32 = dict(dtype=torch.int32)
    a = dict(src=_cpu_cache(), dst=_cpu_cache(), n_copy=torch.zeros(3, **i32), max_rows=0,
             row_idx=torch.zeros(3, 2, 16, **i32), begin=torch.zeros(3, **i32))     # no row at most
    for k, change in _COPY_CHANGES[what].items():
        a[k] = change(a)
    native, general = _either_way(lambda: ck.ck_copy_rows(ck.Shape(3, 4, 2, 8, 1), **a), "host_copy_rows")
    assert native == general


def test_the_native_way_takes_the_plain_calls():
    """Not None: the general way would be right too, and slower."""
    lib, bf, i32 = ck.load_library(), dict(dtype=torch.bfloat16), dict(dtype=torch.int32)
    pytest.importorskip("paper_2412_03213_amd._ckhost")
    sh, kv, n = ck.Shape(3, 4, 2, 8, 1), _cpu_cache(), torch.zeros(3, **i32)
    qkv = torch.zeros(3, 8 * 128, **bf)
    q, k, v = (x.unflatten(1, (-1, 128)) for x in qkv.split([512, 256, 256], dim=1))
    out = torch.zeros(3, 4, 128, **bf)
    inf = float("inf")
    assert lib.host_rope_append(lib.rope_append_entry, sh, kv, q, k, v, out, n, torch.zeros(64), None, None,
                                inf, 0, 0) == -1
    assert lib.host_rope_append(lib.rope_append_entry, sh, kv, None, k, v, None, n, torch.zeros(64),
                                torch.zeros(4, **i32), n, inf, 1, 0) == -1
    ws = torch.zeros(1 << 21, dtype=torch.uint8)
    assert lib.host_paged_decode_attn(lib.paged_decode_attn_entry, sh, kv, out, n, out, None, None, ws, -1, -1,
                                      None, 0.1, 0) == -1
    assert lib.host_paged_decode_attn(lib.paged_decode_attn_entry, sh, kv, out, n, out, torch.zeros(3, 2, 7, **i32),
                                      torch.zeros(3, 2, **i32), ws, -1, 2, 5, 0.1, 0) == -1
    assert lib.host_copy_rows(lib.copy_rows_entry, sh, kv, _cpu_cache(), n, 0, torch.zeros(3, 2, 7, **i32), n, n, 0) == -1
    assert lib.host_copy_rows(lib.copy_rows_entry, sh, kv, kv, n, 0, None, None, None, 0) == -1
    assert lib.host_prompt_attn(lib.prompt_attn_entry, sh, kv, out, torch.zeros(4, **i32), n, out, ws, -1, -1, 0.1, 0) == -1
