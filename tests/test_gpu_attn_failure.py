"""Failure detection of the attention kernel without a GPU fault: every wait is bounded, and one that
runs out ends the kernel through its abort path with a status that the host reads
(hs_test_attn_stalled, include/hs_test.h)."""
import time

import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.attn_helpers import Outputs, Problem, run_prefill, workspace
from tests.gpu_helpers import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [20, 200])      # one and two tiles of rows to a CTA
def test_a_wait_that_runs_out_reports_timeout_and_leaves_the_context_usable(n):
    dev = device()
    p = Problem(20, 2, 1, 128, 16, "bf16", [n], n)
    out = Outputs(p, dev)
    shape = p.shape(1, unsplit=True)
    t0 = time.perf_counter()
    hs.hs_test_attn_stalled(shape, p.q.to(dev), p.cache.to(dev), p.table.to(dev), out.o, out.lse, [0], [n],
                            [0, n], workspace(0, dev), 0, out.err)
    torch.cuda.synchronize()
    waited = time.perf_counter() - t0
    assert out.err.item() == hs.HS_DEVERR_TIMEOUT
    assert 0.9 < waited < 30.0                       # the 1 s bound, not a hang
    assert torch.isnan(out.o).all() and torch.isnan(out.lse).all()
    # the same context, the normal call
    run_prefill(p, [0], [n], dev).check(p.prefill_rows([0], [n], [0, n]))


@pytest.mark.parametrize("n", [20, 200, 1500])
def test_a_wait_that_runs_out_with_heads_of_64(n):
    """The groups of 64-wide heads do not wait for one another: what the second one has finished may be
    written, and it is right."""
    dev = device()
    p = Problem(21, 2, 1, 64, 16, "fp16", [n], n)
    out = Outputs(p, dev)
    shape = p.shape(1, unsplit=True)
    t0 = time.perf_counter()
    hs.hs_test_attn_stalled(shape, p.q.to(dev), p.cache.to(dev), p.table.to(dev), out.o, out.lse, [0], [n],
                            [0, n], workspace(0, dev), 0, out.err)
    torch.cuda.synchronize()
    assert out.err.item() == hs.HS_DEVERR_TIMEOUT
    assert 0.9 < time.perf_counter() - t0 < 30.0
    o = out.o.cpu()
    rows = [x for x in p.prefill_rows([0], [n], [0, n]) if not torch.isnan(o[x[0], :2 * 64]).any()]
    for r, want, _, bound, _ in rows:
        assert ((o[r, :2 * 64].double().reshape(2, 64) - want).abs() <= bound).all()
    run_prefill(p, [0], [n], dev).check(p.prefill_rows([0], [n], [0, n]))


@pytest.mark.parametrize("d", [64, 128])
def test_a_wait_that_runs_out_in_a_call_with_a_join(d):
    """The join runs all the same: the status says that the outputs mean nothing, and nothing else is touched."""
    dev = device()
    p = Problem(22, 4, 2, d, 16, "bf16", [3000], 20)
    out = Outputs(p, dev)
    shape = p.shape(1)
    size = hs.hs_attn_prefill_workspace_bytes(shape, [2980], [20])
    assert size > 0
    ws = workspace(size, dev)
    hs.hs_test_attn_stalled(shape, p.q.to(dev), p.cache.to(dev), p.table.to(dev), out.o, out.lse, [2980], [20],
                            [0, 20], ws, size, out.err)
    torch.cuda.synchronize()
    assert out.err.item() == hs.HS_DEVERR_TIMEOUT
    assert (ws[size:] == 0xFF).all()
    assert torch.isnan(out.o[20:]).all() and torch.isnan(out.lse[20:]).all()
    run_prefill(p, [2980], [20], dev).check(p.prefill_rows([2980], [20], [0, 20]))
