"""Decode steps whose requests are of very different lengths, with as many items as CTAs."""
import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.attn_helpers import Problem, run_decode
from tests.gpu_helpers import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv_heads,group,d,dtype", [(8, 4, 128, "bf16"), (4, 2, 64, "fp16")])
def test_one_long_request_beside_short_ones(kv_heads, group, d, dtype):
    """Its keys are shared out over CTAs (there is a workspace), and every request is answered."""
    dev = device()
    batch = torch.cuda.get_device_properties(dev).multi_processor_count * 2 // kv_heads
    kv_len = [(13 * b) % 101 for b in range(batch)]
    kv_len[5] = 9000
    p = Problem(51, kv_heads * group, kv_heads, d, 16, dtype, kv_len, batch)
    p.table = torch.cat((p.table, torch.full((batch, 300), -1, dtype=torch.int32)), dim=1)
    bound = p.table.shape[1] * 16
    assert hs.hs_attn_decode_workspace_bytes(p.shape(batch), bound) > 0
    run_decode(p, kv_len, bound, dev, shared=False).check(p.decode_rows(kv_len))
    run_decode(p, kv_len, 9000, dev, shared=False, unsplit=True).check(p.decode_rows(kv_len))
