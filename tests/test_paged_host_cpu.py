"""Host tensors are refused by the calls on paged caches, also where all tensors of a call are on the host."""
import pytest
import torch

import paper_2412_03213_amd as ck
import test_paged_cpu as plain
from paper_2412_03213_amd import binding

I32, BF = dict(dtype=torch.int32), dict(dtype=torch.bfloat16)
SH = ck.Shape(3, 4, 2, 8, 1)


def calls():
    kv, n, q = plain._cpu_cache(), torch.zeros(3, **I32), torch.zeros(3, 4, 128, **BF)
    k, ws = torch.zeros(3, 2, 128, **BF), torch.zeros(1 << 26, dtype=torch.uint8)
    return {
        "append": lambda: ck.ck_rope_append(SH, q, k, k, kv, n, torch.zeros(64), q),
        "append without queries": lambda: ck.ck_rope_append(SH, None, k, k, kv, n, torch.zeros(64), None),
        "decode": lambda: ck.ck_paged_decode_attn(SH, q, kv, n, q.clone(), workspace=ws),
        "decode with its own workspace": lambda: ck.ck_paged_decode_attn(SH, q, kv, n, q.clone()),
        "prompt": lambda: ck.ck_prompt_attn(SH, q, torch.zeros(4, **I32), kv, n, q.clone(), workspace=ws),
        "copy": lambda: ck.ck_copy_rows(SH, kv, plain._cpu_cache(), n, 4),
    }


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("what", calls())
def test_calls_of_host_tensors_alone(what, native, monkeypatch):
    lib = ck.load_library()
    if not native:
        for name in ("rope_append", "paged_decode_attn", "prompt_attn", "copy_rows"):
            monkeypatch.setattr(lib, "host_" + name, lambda *args: None)
    with pytest.raises(ValueError, match="host"):
        calls()[what]()


def test_host_tensors_beside_addresses():
    kv, n, q, ws = plain._cpu_cache(), torch.zeros(3, **I32), torch.zeros(3, 4, 128, **BF), 4096
    raw = binding._CkPagedKV(4096, 4096, 4096, 4, 8, 3, 1)
    starts = torch.zeros(4, **I32)
    for call in (lambda: ck.ck_paged_decode_attn(SH, 4096, raw, n, 4096, workspace=ws),
                 lambda: ck.ck_paged_decode_attn(SH, 4096, kv, 4096, 4096, workspace=ws),
                 lambda: ck.ck_paged_decode_attn(SH, 4096, raw, 4096, q, workspace=ws),
                 lambda: ck.ck_prompt_attn(SH, 4096, starts, raw, 4096, 8192, workspace=ws),
                 lambda: ck.ck_prompt_attn(SH, 4096, 4096, raw, 4096, 8192, workspace=torch.zeros(9, dtype=torch.uint8)),
                 lambda: ck.ck_rope_append(SH, None, 4096, 4096, raw, 4096, torch.zeros(64), None),
                 lambda: ck.ck_copy_rows(SH, raw, kv, 4096, 4),
                 lambda: ck.ck_copy_rows(SH, raw, raw, 4096, 4, begin=n)):
        with pytest.raises(ValueError, match="another device"):
            call()


@pytest.fixture
def no_device_is_asked_for(monkeypatch):
    monkeypatch.setattr(binding, "_device", lambda t: t.get_device() if isinstance(t, torch.Tensor) else None)


# What the calls refuse apart from that: the comparison of both ways needs tensors, and there is no device here.
@pytest.mark.parametrize("what", plain._ROPE_CHANGES)
def test_rope_append_both_ways(what, no_device_is_asked_for):
    plain.test_rope_append_refuses_the_same_calls_on_either_way(what)


@pytest.mark.parametrize("what", plain._DECODE_CHANGES)
def test_paged_decode_both_ways(what, no_device_is_asked_for):
    plain.test_paged_decode_refuses_the_same_calls_on_either_way(what)


@pytest.mark.parametrize("what", plain._PROMPT_CHANGES)
def test_prompt_attn_both_ways(what, no_device_is_asked_for):
    plain.test_prompt_attn_refuses_the_same_calls_on_either_way(what)


@pytest.mark.parametrize("what", plain._COPY_CHANGES)
def test_copy_rows_both_ways(what, no_device_is_asked_for):
    plain.test_copy_rows_refuses_the_same_calls_on_either_way(what)


def test_shapes_and_types_without_a_device(no_device_is_asked_for):
    plain.test_tensors_of_other_shapes_and_types_are_refused()
