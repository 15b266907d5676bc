"""Host side of page plans, rows into slots, shared-prefix and cross attention: refusals before anything is
enqueued, and workspaces."""
import ctypes
import math

import pytest
import torch

import paper_2412_03213_amd as ck
from paper_2412_03213_amd import binding

A = 4096                                                # an aligned address that is never dereferenced
EINVALID, EUNSUPPORTED, EWORKSPACE, EMISALIGNED = -1, -2, -3, -4


def shape(**k):
    return ck.Shape(**{**dict(S=2, Hq=8, Hkv=2, N_cap=64, C_cap=1), **k})


SH, F32 = shape(), shape(dtype=ck.CK_F32)


def kv(**k):
    return binding._CkPagedKV(**{**dict(K=A, V=A, page_table=A, n_pages=8, page_size=16, n_seqs=2, pages_per_seq=4), **k})


def code(f, **kw):
    with pytest.raises(ck.ClusterKVError) as e:
        f(**kw)
    return e.value.code


def ref(c):
    return ctypes.byref(c) if c is not None else None


def plan(sh=SH, n_new=A, lengths=A, table=A, width=4, refs=A, pages=8, size=16, parent=None, rows=None, starts=A,
         slots=A, n=5, lacking=A):
    binding._check(binding.load_library().ck_plan_pages(
        ref(sh.c()), n_new, lengths, table, width, refs, pages, size, parent, rows, starts, slots, n, lacking, None))


def store(sh=SH, k=A, v=A, ks=256, vs=256, n=3, slots=A, cache=kv()):
    binding._check(binding.load_library().ck_store_rows(ref(sh.c()), k, v, ks, vs, n, slots, ref(cache), None))


def shared(sh=SH, q=A, cache=kv(), lengths=A, groups=1, starts=A, rows=A, scale=1.0, out=2 * A, ws=A, size=1 << 40):
    binding._check(binding.load_library().ck_shared_decode_attn(
        ref(sh.c()), q, ref(cache), lengths, groups, starts, rows, scale, out, ws, size, None))


def cross(sh=SH, q=A, n=5, starts=A, cache=kv(), lengths=A, scale=1.0, out=2 * A, ws=A, size=1 << 40):
    binding._check(binding.load_library().ck_cross_attn(
        ref(sh.c()), q, n, starts, ref(cache), lengths, scale, out, ws, size, None))


@pytest.mark.parametrize("bad,want", [
    (None, EINVALID), (dict(K=None), EINVALID), (dict(V=None), EINVALID), (dict(page_table=None), EINVALID),
    (dict(K=A + 8), EMISALIGNED), (dict(V=A + 2), EMISALIGNED), (dict(page_table=A + 4), EMISALIGNED),
    (dict(n_pages=0), EINVALID), (dict(page_size=0), EINVALID), (dict(pages_per_seq=0), EINVALID),
    (dict(n_seqs=1), EINVALID), (dict(n_pages=2 ** 26, page_size=32), EUNSUPPORTED),
    (dict(page_size=2 ** 20, pages_per_seq=2 ** 11), EUNSUPPORTED)])
def test_caches_that_are_refused(bad, want):
    c = kv(**bad) if bad is not None else None
    assert code(shared, cache=c) == want
    assert code(cross, cache=c) == want
    if bad != dict(n_seqs=1):                             # its table is not read
        assert code(store, cache=c) == want


@pytest.mark.parametrize("bad,want", [(dict(Hq=6), EUNSUPPORTED), (dict(Hq=5), EINVALID), (dict(d=64), EUNSUPPORTED),
                                      (dict(S=0), EINVALID), (dict(dtype=2), EINVALID)])
def test_shapes_that_are_refused(bad, want):
    for f in (plan, store, shared, cross):
        assert code(f, sh=shape(**bad)) == want


@pytest.mark.parametrize("bad,want", [
    (dict(n_new=None), EINVALID), (dict(lengths=None), EINVALID), (dict(table=None), EINVALID),
    (dict(refs=None), EINVALID), (dict(starts=None), EINVALID), (dict(lacking=None), EINVALID),
    (dict(n_new=A + 4), EMISALIGNED), (dict(refs=A + 4), EMISALIGNED), (dict(slots=A + 4), EMISALIGNED),
    (dict(parent=A), EINVALID), (dict(rows=A), EINVALID), (dict(parent=A, rows=A + 4), EMISALIGNED),
    (dict(slots=None), EINVALID), (dict(n=0), EINVALID), (dict(n=-1), EINVALID), (dict(n=(1 << 24) + 1), EUNSUPPORTED),
    (dict(width=0), EINVALID), (dict(pages=0), EINVALID), (dict(size=0), EINVALID), (dict(size=-3), EINVALID),
    (dict(size=2 ** 20, width=2 ** 11), EUNSUPPORTED), (dict(pages=2 ** 28), EUNSUPPORTED),
    (dict(pages=2 ** 30 + 1, size=1), EUNSUPPORTED), (dict(sh=shape(S=8193)), EUNSUPPORTED), (dict(sh=shape(S=8192), size=1, width=2 ** 18), EUNSUPPORTED)])
def test_plan_refuses(bad, want):
    assert code(plan, **bad) == want


@pytest.mark.parametrize("bad,want", [
    (dict(k=None), EINVALID), (dict(v=None), EINVALID), (dict(slots=None), EINVALID), (dict(k=A + 8), EMISALIGNED),
    (dict(slots=A + 4), EMISALIGNED), (dict(ks=255), EINVALID), (dict(vs=260), EMISALIGNED), (dict(n=0), EINVALID),
    (dict(ks=1 << 41), EUNSUPPORTED), (dict(n=(1 << 24) + 1), EUNSUPPORTED),
    (dict(sh=shape(S=1, Hq=64, Hkv=64), n=(1 << 20) + 1, ks=8192, vs=8192), EUNSUPPORTED)])
def test_store_refuses(bad, want):
    assert code(store, **bad) == want


@pytest.mark.parametrize("bad,want", [
    (dict(q=None), EINVALID), (dict(out=None), EINVALID), (dict(lengths=None), EINVALID), (dict(starts=None), EINVALID),
    (dict(rows=None), EINVALID), (dict(out=A), EINVALID), (dict(groups=0), EINVALID), (dict(groups=3), EINVALID),
    (dict(scale=0.0), EINVALID), (dict(scale=math.nan), EINVALID), (dict(q=A + 2), EMISALIGNED),
    (dict(starts=A + 4), EMISALIGNED), (dict(rows=A + 8), EMISALIGNED), (dict(ws=None), EWORKSPACE),
    (dict(ws=A + 8), EMISALIGNED), (dict(size=1024), EWORKSPACE), (dict(sh=F32, size=1024), EWORKSPACE)])
def test_shared_attention_refuses(bad, want):
    assert code(shared, **bad) == want


@pytest.mark.parametrize("bad,want", [
    (dict(q=None), EINVALID), (dict(out=None), EINVALID), (dict(lengths=None), EINVALID), (dict(out=A), EINVALID),
    (dict(n=0), EINVALID), (dict(n=1 << 25), EUNSUPPORTED), (dict(starts=None), EINVALID),
    (dict(sh=F32), EUNSUPPORTED), (dict(scale=-1.0), EINVALID), (dict(q=A + 8), EMISALIGNED),
    (dict(starts=A + 4), EMISALIGNED), (dict(ws=None), EWORKSPACE), (dict(size=1), EWORKSPACE),
    (dict(starts=None, n=2, size=1), EWORKSPACE)])
def test_cross_attention_refuses(bad, want):
    assert code(cross, **bad) == want


def test_workspaces():
    for S, Hq, Hkv in ((1, 8, 8), (64, 32, 8), (1000, 8, 1)):
        for dtype in (ck.CK_BF16, ck.CK_F32):
            sh = shape(S=S, Hq=Hq, Hkv=Hkv, dtype=dtype)
            single = ck.ck_workspace_bytes(sh, binding.CK_WS_PAGED_ATTN, 0)
            assert ck.ck_workspace_bytes(sh, binding.CK_WS_SHARED_ATTN, 0) >= single
            sizes = [ck.ck_workspace_bytes(sh, binding.CK_WS_CROSS_ATTN, n) for n in (1, 17, 1000, 100000)]
            assert sizes == sorted(sizes) and sizes[0] >= single      # enough for fewer rows too
        assert ck.ck_workspace_bytes(sh, binding.CK_WS_CROSS_ATTN, 0) == 0


NATIVE = ("plan_pages", "store_rows", "shared_decode_attn", "cross_attn")


@pytest.mark.parametrize("native", [True, False])
def test_host_tensors_are_refused(native, monkeypatch):
    if not native:
        for name in NATIVE:
            monkeypatch.setattr(ck.load_library(), "host_" + name, lambda *args: None)
    bf = torch.bfloat16
    K = torch.zeros(8, 2, 16, 128, dtype=bf)
    table = torch.zeros(2, 4, dtype=torch.int32)
    cache = ck.PagedKV(K, K.clone(), table)
    q, out, n = torch.zeros(2, 8, 128, dtype=bf), torch.zeros(2, 8, 128, dtype=bf), torch.ones(2, dtype=torch.int32)
    starts, ws, k = torch.zeros(3, dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(2, 2, 128, dtype=bf)
    refs, one = torch.zeros(8, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: ck.ck_shared_decode_attn(SH, q, cache, n, starts[:2], n, out, workspace=ws),   # on the host
                 lambda: ck.ck_cross_attn(SH, q, starts, cache, n, out, workspace=ws),
                 lambda: ck.ck_store_rows(SH, k, k, n, cache),
                 lambda: ck.ck_plan_pages(SH, n, n, table, refs, 16, starts, one)):
        with pytest.raises(ValueError, match="host"):
            call()


@pytest.fixture
def as_device_tensors(monkeypatch):
    """Host tensors pass for those of the current device, so that the other checks are reached."""
    monkeypatch.setattr(binding, "_device", lambda t: -1)
    monkeypatch.setattr(binding, "_elsewhere", lambda d, dev: False)
    monkeypatch.setattr(binding, "_check", lambda rc: pytest.fail("reached the library"))


def test_shapes_and_types_of_tensors(as_device_tensors):
    bf = torch.bfloat16
    K = torch.zeros(8, 2, 16, 128, dtype=bf)
    table = torch.zeros(2, 4, dtype=torch.int32)
    cache = ck.PagedKV(K, K.clone(), table)
    q, out, n = torch.zeros(2, 8, 128, dtype=bf), torch.zeros(2, 8, 128, dtype=bf), torch.ones(2, dtype=torch.int32)
    starts, ws, k = torch.zeros(3, dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(2, 2, 128, dtype=bf)
    refs, one = torch.zeros(8, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for args in ((q[:1], cache, n, starts, n, out), (q, cache, n.long(), starts, n, out), (q, cache, n, starts, n[:1], out),
                 (q, cache, n, starts.float(), n, out), (q.float(), cache, n, starts, n, out),
                 (q, cache, n, starts, n, out[..., ::2])):
        with pytest.raises(ValueError):
            ck.ck_shared_decode_attn(SH, *args, workspace=ws)
    for args in ((q, n, cache, n, out), (q, starts, cache, n.long(), out), (q, starts, cache, n, out[:1])):
        with pytest.raises(ValueError):
            ck.ck_cross_attn(SH, *args, workspace=ws)
    for sh in (shape(Hkv=4), F32):
        with pytest.raises(ValueError):
            ck.ck_cross_attn(sh, q, starts, cache, n, out, workspace=ws)
    for args in ((k, k[:1], n, cache), (k, k.float(), n, cache), (k, k, n.long(), cache), (k, k, starts, cache),
                 (k.transpose(0, 1), k, n, cache)):
        with pytest.raises(ValueError):
            ck.ck_store_rows(SH, *args)
    for args in ((n, n, table[:1], refs, 16, starts, one), (n.long(), n, table, refs, 16, starts, one),
                 (n, n, table, refs[::2], 16, starts, one), (n, n, table.t(), refs, 16, starts, one),
                 (n, n, table, refs, 16, n, one), (n, n, table, refs, 16, starts, n), (n, n, refs, refs, 16, starts, one)):
        with pytest.raises(ValueError):
            ck.ck_plan_pages(SH, *args)
    with pytest.raises(ValueError):
        ck.ck_plan_pages(SH, n, n, table, refs, 16, starts, one, parent=n, shared_rows=one)
