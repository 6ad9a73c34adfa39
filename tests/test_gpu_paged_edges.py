"""GPU tests of the paged calls at their edges, against the float64 oracle: batches whose sequences need different forms of
a kernel, scores at the ends of their range, values that are not numbers."""
import numpy as np
import pytest
import torch

import paged_utils as U
from oracle import paged_oracle as PO

pytestmark = pytest.mark.gpu


def _want_selected(s, sink, tail, topk):
    *want, pages = PO.block_attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q,
                                      np.nan_to_num(U.f64(s.bounds)), sink, tail, topk)
    return want, pages


# ---------------------------------------------------------------------------------------------- page selection
def test_one_very_long_sequence_among_shorter_ones_that_select_too():
    # tokens with more pages than a selecting CTA keeps in shared memory (40,960), tokens of the same chunk with just as
    # many, and two shorter sequences
    s = U.make_step(2, 1, 64, 16, "bf16", [(20, 16 * 40964 - 6), (2, 16 * 700 + 5), (1, 16 * 5000)], seed=100, with_bounds=True)
    y, lse, idx = U.gpu_block_attention(s, 1, 2, 50)
    want, pages = _want_selected(s, 1, 2, 50)
    assert (idx == pages).all()
    U.check_attention("bf16", 64, y, lse, *want, n_keys=53 * 16)


def test_a_selection_captured_for_very_many_pages_is_replayed_for_fewer():
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    s = U.make_step(2, 1, 64, 16, "bf16", [(1, 16 * 42000 + 3)], seed=101, with_bounds=True)
    kv, sel = U.to_device(s), T.PageSelection(1, 2, 50)
    q = s.q.to(dev)
    y, lse = torch.empty_like(q), torch.empty(1, 2, device=dev)
    idx = torch.empty(1, 1, sel.n_pages, dtype=torch.int32, device=dev)
    ws = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_BLOCK_ATTENTION, sel), dtype=torch.uint8, device=dev)

    def run():
        T.paged_block_attention(kv, sel, q, y, lse, idx, None, ws)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for n in (16 * 800 + 1, 16 * 42000 + 3, 16 * 30000):
        kv.kv_lens_dev.copy_(torch.tensor([n]))
        graph.replay()
        torch.cuda.synchronize()
        assert kv.device_status() == 0
        short = U.Step(s.k, s.v, s.table, np.array([n], np.int64), s.cu_q, 2, s.q, s.bounds)
        want, pages = _want_selected(short, 1, 2, 50)
        assert (idx.cpu().numpy() == pages).all()
        U.check_attention("bf16", 64, U.f64(y), U.f64(lse), *want, n_keys=53 * 16)
