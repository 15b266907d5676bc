"""The merge of the decode step in workspaces of any contents, words of earlier calls that were partly overwritten
among them."""
import pytest
import torch

import paper_2412_03213_amd as ck
from test_gpu_merge import DEV, make
from test_gpu_paged_edges import overwritten

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S,Hq,Hkv,N,n_max,dtype", [
    (1, 32, 8, 8192, 1024, ck.CK_BF16), (1, 4, 1, 16384, 9000, ck.CK_BF16), (2, 4, 4, 2048, 500, ck.CK_F32)])
def test_merge_in_a_workspace_of_any_contents(S, Hq, Hkv, N, n_max, dtype):
    tdt = torch.bfloat16 if dtype == ck.CK_BF16 else torch.float32
    g, K, V, idx = make(S, Hq, Hkv, N, n_max, seed=n_max, dtype=tdt)
    sh = ck.Shape(S, Hq, Hkv, N, 8, dtype=dtype)
    q = torch.randn(S, Hq, 128, generator=g, device=DEV).to(tdt)
    n_tok = torch.full((S, Hkv), n_max, dtype=torch.int32, device=DEV)
    want, got = torch.empty_like(q), torch.empty_like(q)
    ck.ck_sparse_decode_attn(sh, q, K, V, idx, n_tok, n_max, want, two_pass=True)
    ws = torch.empty(ck.ck_workspace_bytes(sh, 1, n_max), dtype=torch.uint8, device=DEV)
    ck.ck_sparse_decode_attn(sh, q, K, V, idx, n_tok, n_max, got, workspace=ws)
    assert torch.equal(got, want)
    for i, words in enumerate(overwritten(ws)):
        ws.copy_(words.view(torch.uint8).flatten())
        for again in range(2):
            got.fill_(float("nan"))
            ck.ck_sparse_decode_attn(sh, q, K, V, idx, n_tok, n_max, got, workspace=ws)
            assert torch.equal(got, want), (i, again)
    full, other = torch.empty_like(q), torch.empty_like(q)
    ws = torch.empty(ck.ck_workspace_bytes(sh, 1, N), dtype=torch.uint8, device=DEV)
    ck.ck_full_decode_attn(sh, q, K, V, N, full, workspace=ws)
    for i, words in enumerate(overwritten(ws)):
        ws.copy_(words.view(torch.uint8).flatten())
        ck.ck_full_decode_attn(sh, q, K, V, N, other, workspace=ws)
        assert torch.equal(other, full), i
