"""Which rows of logits the verification reads: a draft model's rows begin with a request's second."""
import numpy as np
import pytest
import torch

from oracle import kvpr_paged_oracle as po
from paged_testlib import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


@pytest.mark.parametrize("vocab", [65, 5000, 50272])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_draft_logits_without_the_first_row(k, vocab, dtype):
    """One request whose draft logits are an array of m - 1 rows: the call is given the address one row in front of it.  No row lies there."""
    m = 5
    g = torch.Generator(device="cuda").manual_seed(vocab)
    target = (torch.randn((m, vocab), generator=g, device="cuda") * 2).to(dtype)
    draft = (target[:-1].float() + 0.3 * torch.randn((m - 1, vocab), generator=g, device="cuda")).to(dtype).contiguous()
    tokens = torch.cat([torch.zeros(1, device="cuda"), draft.float().argmax(-1)]).int()
    ua, us = torch.full((m,), 0.4, device="cuda"), torch.tensor([0.6], device="cuda")
    full = np.concatenate([np.zeros((1, vocab)), draft.double().cpu().numpy()])
    for t in (1.0, 0.0):
        temperature = torch.tensor([t], device="cuda")
        want, kept = po.verify(target.double().cpu().numpy(), full, tokens.cpu().numpy(), [0, m], [t], ua.cpu().numpy(), us.cpu().numpy(), m)
        out, got = i32([-7] * m), i32([-7])
        ws = torch.full((k.kvpr_verify_workspace_bytes(1, m, vocab),), 0xFF, dtype=torch.uint8, device="cuda")
        k.kvpr_verify_drafts(target, draft.data_ptr() - vocab * draft.element_size(), k.KVPR_F16 if dtype == torch.float16 else k.KVPR_F32, vocab, vocab, vocab,
                             tokens, i32([0, m]), 1, m, temperature, ua, us, None, None, got, out, ws, ws.numel())
        torch.cuda.synchronize()
        assert got.tolist() == kept and out.tolist() == want
