"""Lists of batches that leave them empty, into buffers of the size that they may have."""
import pytest
import torch

import paper_2010_10458_amd as tk
from gpu_common import announce, need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [4, 300, 20000])
def test_no_tokens_into_empty_buffers(rows):
    announce(f"lists of no tokens, a plan of {rows}")
    dev = need_gpu()
    plan = tk.EmbedPlan(rows, 300, 17, dtype=torch.float32, check=True)
    tok, dout = torch.zeros(0, dtype=torch.int32, device=dev), torch.zeros(0, 17, device=dev)
    assert plan.most(0) == 0
    idx, val = torch.zeros(0, dtype=torch.int32, device=dev), torch.zeros(0, device=dev)
    nnz = torch.full((1,), 9, dtype=torch.int32, device=dev)
    assert plan.lists(tok, dout, idx_out=idx, val_out=val, nnz_out=nnz) == (idx, val, nnz)
    assert int(nnz.item()) == 0
    idx, val = tk.embed_lists(tok, dout, 300)
    assert idx.numel() == 0 and val.numel() == 0
