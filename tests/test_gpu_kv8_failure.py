"""Failure detection of the decode step over the 8-bit cache without a GPU fault: a wait that runs out ends the kernel
through its abort path with a status that the host reads (hs_test_kv8_stalled, include/hs_test.h)."""
import time

import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.gpu_helpers import device
from tests.kv8_helpers import DT, filled, shape_of
from tests.test_gpu_kv8 import decoded, near, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,d,dtype,lens,unsplit", [
    (8, 2, 128, "bf16", [3000, 10, 0], False), (16, 1, 64, "fp16", [2000], False), (8, 2, 64, "bf16", [300] * 400, True),
    (16, 1, 128, "fp16", [900, 5], True), (4, 4, 128, "bf16", [20] * 3, False)])
def test_a_wait_that_runs_out_reports_timeout_and_leaves_the_context_usable(heads, kv_heads, d, dtype, lens, unsplit):
    dev = device()
    lens = lens[:384]
    c, table = filled(30, lens, kv_heads, 16, d)
    q = rows_of(31, len(lens), heads * d, 0, DT[dtype], dev)
    shape = shape_of(len(lens), heads, kv_heads, d, 16, c.blocks, table.shape[1], dtype, unsplit=unsplit)
    bound = max(lens)
    size = hs.hs_kv8_decode_workspace_bytes(shape, bound)
    ws = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device=dev)
    o = torch.full((len(lens) + 1, heads * d), 7.0, dtype=DT[dtype], device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    args = [x.to(dev) for x in (q, c.image(), table, torch.tensor(lens, dtype=torch.int32))]
    t0 = time.perf_counter()
    hs.hs_test_kv8_stalled(shape, *args, bound, o, None, ws, size, err)
    torch.cuda.synchronize()
    waited = time.perf_counter() - t0
    assert err.item() == hs.HS_DEVERR_TIMEOUT
    assert 0.9 < waited < 30.0                       # the 1 s bound, not a hang
    assert (ws[size:] == 0xFF).all() and (o[-1] == 7.0).all()
    o, z, code = decoded(dev, c, table, q, heads, dtype, lens, bound, unsplit=unsplit)
    assert code == 0
    near(c, table, q, heads, dtype, lens, o, z, d ** -0.5, only={0, 1, len(lens) - 1})
