"""Which shapes a page plan takes: its header promises 8192 sequences of any model that the library serves."""
import pytest
import torch

import paper_2412_03213_amd as ck
from test_gpu_plan import Steps
from test_segments_cpu import A, EINVALID, EUNSUPPORTED, code, cross, kv, plan, shape, shared


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (64, 8), (8, 8), (64, 64), (1, 1)])
def test_plan_takes_as_many_sequences_of_every_model(Hq, Hkv):
    # what is refused is the missing list, so the shape has passed
    assert code(plan, sh=shape(S=8192, Hq=Hq, Hkv=Hkv), n_new=None) == EINVALID
    assert code(plan, sh=shape(S=8193, Hq=Hq, Hkv=Hkv), n_new=None) == EUNSUPPORTED


def test_attention_of_as_many_heads_is_refused_as_before():
    sh = shape(S=8192, Hq=64, Hkv=8)
    cache = kv(n_seqs=8192)
    assert code(shared, sh=sh, cache=cache) == EUNSUPPORTED
    assert code(cross, sh=sh, cache=cache, starts=A) == EUNSUPPORTED
    assert ck.ck_workspace_bytes(sh, 5, 0) == 0 and ck.ck_workspace_bytes(sh, 6, 100) == 0


@pytest.mark.gpu
def test_plan_of_a_model_with_eight_kv_heads():
    x = Steps(8192, 2, 9000, 4)
    x.sh = ck.Shape(8192, 32, 8, 8, 1)
    x.step([1] * 8192)
    x.step([-1 if s % 2 else 3 for s in range(8192)])
