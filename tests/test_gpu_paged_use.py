"""GPU tests of the paged calls as a program uses them: together with each other and with the library's other calls, in
CUDA graphs, on several streams, with shared and with bad pages, far offsets, and buffers that must stay as they are."""
import numpy as np
import pytest
import torch

import paged_utils as U
from oracle import paged_oracle as PO
from oracle import tkphi_oracle as O

pytestmark = pytest.mark.gpu


def _want(s, causal=True, scale=None):
    return PO.attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q, causal, scale)


# ---------------------------------------------------------------------------------------------- numerics of long rows
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("q_len", [4, 30, 90])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("direction", [1, -1])
def test_scores_that_rise_and_fall_along_the_keys(d, q_len, dtype, direction):
    # the reference of a row's exponentials is set by its first tile: later tiles are far above (or below) it
    s = U.make_step(8, 2, d, 32, dtype, [(q_len, 1300), (1, 700)], seed=30)
    u = torch.randn(d, generator=torch.Generator().manual_seed(31))
    s.q = (u + 0.1 * s.q.float()).to(s.q.dtype)
    for b, n in enumerate(s.kv_lens):
        for t in range(int(n)):
            x = t / float(n) if direction == 1 else 1 - t / float(n)
            s.k[s.table[b, t // 32], :, t % 32] = (u * (24 * x - 4)).to(s.k.dtype)
    y, lse = U.gpu_attention(s)
    U.check_attention(dtype, d, y, lse, *_want(s), n_keys=1300)


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (3, 1, 128), (5, 1, 64), (9, 1, 128), (12, 1, 64), (16, 1, 128), (7, 1, 128)])
def test_chunks_cut_over_the_keys_for_every_group(hq, hkv, d):
    s = U.make_step(hq, hkv, d, 64, "bf16", [(45, 7001), (70, 300)], seed=32)
    y, lse = U.gpu_attention(s)
    U.check_attention("bf16", d, y, lse, *_want(s), n_keys=7001)


def test_results_over_disjoint_keys_join():
    # a shared prefix, attended in full, and the rest, attended causally
    import paper_2604_05438_b200 as T
    whole = U.make_step(6, 2, 128, 16, "bf16", [(20, 20 + 320), (1, 1 + 320)], seed=33)
    prefix = U.Step(whole.k, whole.v, whole.table, np.array([320, 320], np.int64), whole.cu_q, 6, whole.q)
    rest = U.Step(whole.k, whole.v, np.ascontiguousarray(whole.table[:, 20:]), np.array([20, 1], np.int64), whole.cu_q, 6, whole.q)
    ya, la = U.gpu_attention(prefix, causal=False)
    yb, lb = U.gpu_attention(rest)
    w = np.exp(np.stack([la, lb]) - np.logaddexp(la, lb))[..., None]
    y, lse, A, _ = _want(whole)
    assert (np.abs(w[0] * ya + w[1] * yb - y) <= 2 * (2.0 ** -7 * A + 1e-3)).all()
    np.testing.assert_allclose(np.logaddexp(la, lb), lse, atol=2e-3)


# ---------------------------------------------------------------------------------------------- one step of a model layer
@pytest.mark.parametrize("tokens_first", [False, True])
def test_a_prompt_then_decoding_with_every_call(tokens_first):
    """Chunks of two prompts are appended and attended, then tokens are decoded with exact attention, with selected pages
    and, on the same memory, with the library's summary build and Top-K+phi decode step."""
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    g = torch.Generator().manual_seed(40)
    hq, hkv, d, ps = 8, 2, 64, 16
    lens = [7 * ps, 11 * ps]                                 # after the last token
    n_pages = sum(lens) // ps
    # contiguous sequences are paged ones: page = row / page_size, in order
    total = sum(lens)
    store = torch.full((2, total, hkv, d) if tokens_first else (2, hkv, total, d), float("nan"), dtype=torch.bfloat16, device=dev)
    heads = store.transpose(1, 2) if tokens_first else store                   # [k/v, head, row, dim]
    k, v = (heads[i].unflatten(1, (n_pages, ps)).transpose(0, 1) for i in (0, 1))
    table = np.full((2, 11), -1, np.int32)
    table[0, :7], table[1] = np.arange(7), np.arange(7, 18)
    bounds = torch.full((n_pages, hkv, 2, d), float("nan"), dtype=torch.bfloat16, device=dev)
    inv = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float()
    rot = T.RotaryMap(inv.to(dev))
    tokens = [torch.randn(n, hq + 2 * hkv, d, generator=g).bfloat16() for n in lens]

    ref_k = np.full((n_pages, hkv, ps, d), np.nan)
    ref_v = ref_k.copy()
    done = [0, 0]
    for step in ([50, 33], [lens[0] - 51, 0], [0, lens[1] - 34], [1, 1]):
        qkv = torch.cat([tokens[b][done[b]:done[b] + m] for b, m in enumerate(step)]).to(dev)
        done = [x + m for x, m in zip(done, step)]
        cu = np.array([0, step[0], sum(step)], np.int64)
        kv = T.PagedKVCache(k, v, torch.from_numpy(table).to(dev), done, cu, hq, bounds)
        q = torch.empty(sum(step), hq, d, dtype=torch.bfloat16, device=dev)
        T.paged_append(kv, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], rot, qkv[:, :hq], q)
        s = U.Step(k.cpu(), v.cpu(), table, np.array(done, np.int64), cu, hq, q.cpu())
        y, lse = U.gpu_attention(s, kv=kv)
        want_k, want_v = PO.append(ref_k, ref_v, table, done, cu, U.f64(qkv[:, hq:hq + hkv]), U.f64(qkv[:, hq + hkv:]), inv.double().numpy())
        got_k = U.f64(k)
        live = ~np.isnan(want_k)
        np.testing.assert_array_equal(np.isnan(got_k), ~live)
        assert (np.abs(got_k - want_k)[live] <= 2.0 ** -8 * np.abs(want_k[live]) + 2.0 ** -18).all()
        ref_k, ref_v = got_k, want_v
        np.testing.assert_array_equal(U.f64(v)[live], want_v[live])
        want = PO.attention(U.f64(q), ref_k, ref_v, table, done, cu)
        U.check_attention("bf16", d, y, lse, *want, n_keys=max(done))

    # the last token of both again, over selected pages
    y, lse, idx = U.gpu_block_attention(s, 1, 1, 3, kv=kv)
    *want, pages = PO.block_attention(U.f64(q), ref_k, ref_v, table, done, cu, U.f64(bounds), 1, 1, 3)
    assert (idx == pages).all()
    U.check_attention("bf16", d, y, lse, *want, n_keys=80)

    # and over the contiguous view of the same memory: Top-K with all of the mid-region retrieved is plain attention
    cu_seq = np.array([0, lens[0], total], np.int64)
    ckv = T.KVCache(heads[0], heads[1], cu_seq, hq, 64, 4, 16)
    topk = np.array([n - 20 for n in lens], np.int32)
    ws = torch.empty(T.workspace_bytes(ckv, topk, int(topk.max()), T.WS_TOPK_DECODE), dtype=torch.uint8, device=dev)
    y_top = torch.empty(2, hq, d, device=dev)
    T.topk_decode(ckv, q, topk, torch.from_numpy(topk).to(dev), int(topk.max()), None, y_top, ws)
    torch.cuda.synchronize()
    full = PO.attention(U.f64(q), ref_k, ref_v, table, done, cu)[0]
    assert np.abs(U.f64(y_top) - full).max() <= 2e-3 * np.abs(full).max()
    w = torch.randn(hkv, 64, d, generator=g) / 8
    phi = T.PhiMaps(*(t.to(dev) for t in (torch.randn(hq, 64, d, generator=g) / 8, torch.zeros(hq, 64), w, torch.zeros(hkv, 64))), 0.1, 0.1)
    S, u = torch.empty(2, hkv, d, 64, device=dev), torch.empty(2, hkv, 64, device=dev)
    T.build_summaries(ckv, phi, S, u, torch.empty(T.workspace_bytes(ckv, None, 0, T.WS_BUILD), dtype=torch.uint8, device=dev))
    for h in range(hkv):
        K, V = PO.rows(ref_k, table[1], lens[1])[h], PO.rows(ref_v, table[1], lens[1])[h]
        S0, _ = O.build_summaries(K, V, w[h].double().numpy(), np.zeros(64), 0.1, 4, 16)
        assert np.abs(U.f64(S)[1, h] - S0).max() <= 1e-3 * np.abs(S0).max()


@pytest.mark.parametrize("topk", [2, 30])
def test_selected_pages_right_behind_an_append(topk):
    # (with 30 the selection takes every page and has no bounds to compute: its first grid is another one)
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    s = U.make_step(8, 2, 128, 16, "bf16", [(9, 200), (1, 333), (30, 30)] * 8, seed=43, with_bounds=True)
    g = torch.Generator().manual_seed(44)
    kv = U.to_device(s)
    sel = T.PageSelection(1, 1, topk)
    ws = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_BLOCK_ATTENTION, sel), dtype=torch.uint8, device=dev)
    for _ in range(20):
        qkv = torch.randn(s.total_q, 12, 128, generator=g).bfloat16().to(dev)
        got = []
        for wait in (False, True):
            kv.key_bounds.zero_()
            q, y, lse = torch.zeros_like(s.q, device=dev), torch.zeros_like(s.q, device=dev), torch.zeros(s.total_q, 8, device=dev)
            T.paged_append(kv, qkv[:, 8:10], qkv[:, 10:], None, qkv[:, :8], q)
            if wait:
                torch.cuda.synchronize()
            T.paged_block_attention(kv, sel, q, y, lse, None, None, ws)
            got.append((y, lse))
        torch.cuda.synchronize()
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_bounds_are_right_after_a_rollback_of_drafted_tokens():
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    s = U.make_step(8, 2, 64, 16, "bf16", [(5, 37)], seed=41, with_bounds=True)
    kv = U.to_device(s)
    new = torch.randn(5, 2, 64, generator=torch.Generator().manual_seed(42)).bfloat16().to(dev)
    T.paged_append(kv, 100 * new, new)                                # five drafted tokens, far out
    again = T.PagedKVCache(kv.k, kv.v, kv.page_table, [35], [0, 3], 8, kv.key_bounds)
    T.paged_append(again, new[:3].contiguous(), new[:3].contiguous())  # three of them, with other values
    torch.cuda.synchronize()
    for page, (lo, hi) in PO.page_bounds(U.f64(kv.k), s.table, [35]).items():
        if page != s.table[0, 0]:
            np.testing.assert_array_equal(U.f64(kv.key_bounds)[page, :, 0], lo)
            np.testing.assert_array_equal(U.f64(kv.key_bounds)[page, :, 1], hi)


# ---------------------------------------------------------------------------------------------- graphs, streams, buffers
def _calls(T, kv, q, k_new, v_new, dev):
    """The three calls on one descriptor, each with a workspace and outputs of its own: (run, outputs)."""
    sel = T.PageSelection(1, 2, 4)
    out = {n: torch.zeros_like(q) for n in ("q", "y", "yb")}
    out["lse"] = torch.zeros(q.shape[:2], device=dev)
    out["lse_b"] = torch.zeros(q.shape[:2], device=dev)
    out["idx"] = torch.zeros(q.shape[0], kv.k.shape[1], sel.n_pages, dtype=torch.int32, device=dev)
    wa = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_ATTENTION), dtype=torch.uint8, device=dev)
    wb = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_BLOCK_ATTENTION, sel), dtype=torch.uint8, device=dev)
    rot = T.RotaryMap((10000.0 ** (-torch.arange(0, q.shape[2], 2) / q.shape[2])).float().to(dev))

    def run(stream=None):
        T.paged_append(kv, k_new, v_new, rot, q, out["q"], stream=stream)
        T.paged_attention(kv, out["q"], out["y"], out["lse"], None, 0, wa, stream=stream)
        T.paged_block_attention(kv, sel, out["q"], out["yb"], out["lse_b"], out["idx"], None, wb, stream=stream)
    return run, out


@pytest.mark.parametrize("lens,shorter", [([(1, 300), (1, 17), (1, 2000)], [(1, 288), (1, 1), (1, 33)]),
                                          ([(40, 900), (1, 5000), (7, 64)], [(40, 41), (1, 650), (7, 60)])])
def test_captured_calls_follow_shorter_device_lengths(lens, shorter):
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    long = U.make_step(8, 2, 64, 16, "bf16", lens, seed=50, with_bounds=True)
    g = torch.Generator().manual_seed(51)
    new = torch.randn(2, long.total_q, 2, 64, generator=g).bfloat16().to(dev)
    q = long.q.to(dev)
    kv = U.to_device(long)
    k0, v0, b0 = kv.k.clone(), kv.v.clone(), kv.key_bounds.clone()
    run, out = _calls(T, kv, q, new[0], new[1], dev)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for which in (shorter, lens, shorter):
        kv.kv_lens_dev.copy_(torch.tensor([n for _, n in which]))
        for t, t0 in ((kv.k, k0), (kv.v, v0), (kv.key_bounds, b0)):
            t.copy_(t0)
        for t in out.values():
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in out.items()}
        # the same step, called with these lengths
        eager = T.PagedKVCache(k0.clone(), v0.clone(), kv.page_table, [n for _, n in which], long.cu_q, 8, b0.clone())
        run2, want = _calls(T, eager, q, new[0], new[1], dev)
        run2()
        torch.cuda.synchronize()
        assert torch.equal(eager.k.nan_to_num(), kv.k.nan_to_num()) and torch.equal(eager.key_bounds.nan_to_num(), kv.key_bounds.nan_to_num())
        assert torch.equal(got["q"], want["q"]) and torch.equal(got["idx"], want["idx"])
        for n in ("y", "yb"):      # the split over CTAs may differ: equal up to its roundings
            assert (got[n].float() - want[n].float()).abs().max() <= 2.0 ** -6 * want[n].float().abs().max()
        for n in ("lse", "lse_b"):
            assert (got[n] - want[n]).abs().max() <= 1e-4
        assert kv.device_status() == 0 and eager.device_status() == 0


def test_two_streams_at_once_and_repeated_calls_are_bit_identical():
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    steps = [U.make_step(8, 2, 64, 32, "bf16", lens, seed=60 + i, with_bounds=True)
             for i, lens in enumerate(([(1, 3000), (50, 700), (1, 9)], [(90, 2000), (1, 20000), (3, 400)]))]
    runs = []
    for i, s in enumerate(steps):
        new = torch.randn(2, s.total_q, 2, 64, generator=torch.Generator().manual_seed(70 + i)).bfloat16().to(dev)
        runs.append(_calls(T, U.to_device(s), s.q.to(dev), new[0], new[1], dev))
    for run, _ in runs:
        run()
    torch.cuda.synchronize()
    first = [{n: t.clone() for n, t in out.items()} for _, out in runs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for st, (run, _) in zip(streams, runs):
            run(stream=st)
    torch.cuda.synchronize()
    for want, (_, out) in zip(first, runs):
        for n in want:
            assert torch.equal(want[n], out[n]), n


def test_rows_behind_the_last_sequence_stay_as_they_are():
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    s = U.make_step(6, 2, 128, 16, "fp16", [(1, 100), (60, 200), (0, 30)], seed=80, with_bounds=True)
    kv = U.to_device(s)
    n = s.total_q

    def guarded(shape, dtype):
        big = torch.full((shape[0] + 9,) + shape[1:], 7, dtype=dtype, device=dev)
        return big, big[:shape[0]]
    (qb, q), (yb, y), (lb, lse) = guarded((n, 6, 128), torch.float16), guarded((n, 6, 128), torch.float16), guarded((n, 6), torch.float32)
    ib, idx = guarded((n, 2, 7), torch.int32)
    new = torch.randn(n, 2, 128, device=dev).half()
    sel = T.PageSelection(1, 2, 4)
    T.paged_append(kv, new, new, None, s.q.to(dev), q)
    ws = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_ATTENTION) + 512, dtype=torch.uint8, device=dev).fill_(7)
    T.paged_attention(kv, q, y, lse, None, 0, ws[:-512])
    wb = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_BLOCK_ATTENTION, sel) + 512, dtype=torch.uint8, device=dev).fill_(7)
    T.paged_block_attention(kv, sel, q, y, lse, idx, None, wb[:-512])
    torch.cuda.synchronize()
    for big in (qb, yb, lb, ib):
        assert (big[n:] == 7).all()
    assert (ws[-512:] == 7).all() and (wb[-512:] == 7).all()
    # optional outputs left out
    T.paged_attention(kv, q, y, None, 0.3, 0, ws)
    T.paged_block_attention(kv, sel, q, y, None, None, 0.3, wb)
    torch.cuda.synchronize()
    assert kv.device_status() == 0


# ---------------------------------------------------------------------------------------------- pages
def test_pages_shared_by_two_sequences_are_read_by_both():
    s = U.make_step(8, 2, 64, 16, "bf16", [(1, 170), (40, 200)], seed=90, with_bounds=True)
    s.table[1, :9] = s.table[0, :9]                         # a common prefix of 144 tokens
    y, lse = U.gpu_attention(s)
    U.check_attention("bf16", 64, y, lse, *_want(s), n_keys=200)
    y, lse, idx = U.gpu_block_attention(s, 1, 1, 3)
    *want, pages = PO.block_attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q, np.nan_to_num(U.f64(s.bounds)), 1, 1, 3)
    assert (idx == pages).all()
    U.check_attention("bf16", 64, y, lse, *want, n_keys=200)


@pytest.mark.parametrize("bad", [-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31])
def test_bad_pages_are_reported_and_touch_only_their_sequence(bad):
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    lens = [(1, 300), (40, 200), (1, 128), (20, 64)]
    s = U.make_step(8, 2, 64, 16, "bf16", lens, seed=91, with_bounds=True)
    n_pages = s.k.shape[0]
    new = torch.randn(2, s.total_q, 2, 64, generator=torch.Generator().manual_seed(92)).bfloat16().to(dev)
    good = U.to_device(s)
    run, want = _calls(T, good, s.q.to(dev), new[0], new[1], dev)
    run()
    torch.cuda.synchronize()
    assert good.device_status() == 0
    s.table[0, 18] = bad if bad != 10 ** 6 else n_pages       # the page of a decoding sequence's last token
    s.table[1, 11] = bad if bad != 10 ** 6 else n_pages       # a page in the middle of a chunk
    kv = U.to_device(s)
    k0 = kv.k.clone()
    run, out = _calls(T, kv, s.q.to(dev), new[0], new[1], dev)
    run()
    torch.cuda.synchronize()
    assert kv.device_status() == -1
    rows = slice(int(s.cu_q[2]), None)                        # the other two sequences
    for n in want:
        assert torch.equal(want[n][rows], out[n][rows]), n
    # pages that belong to nobody's new rows are untouched
    touched = {int(s.table[b, p]) for b, (m, n) in enumerate(lens) for p in range((n - m) // 16, (n - 1) // 16 + 1)}
    for page in range(n_pages):
        if page not in touched:
            assert torch.equal(kv.k[page].nan_to_num(), k0[page].nan_to_num())


def test_offsets_beyond_32_bits():
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    hq, hkv, d, ps = 24, 8, 128, 64
    n_pages = 36000                                          # 4.7 GB of keys: 2.36e9 elements
    k = torch.empty(n_pages, hkv, ps, d, dtype=torch.bfloat16, device=dev)
    v = torch.empty_like(k)
    bounds = torch.empty(n_pages, hkv, 2, d, dtype=torch.bfloat16, device=dev)
    s = U.make_step(hq, hkv, d, ps, "bf16", [(1, 500), (30, 200)], seed=93, with_bounds=True, spare=0)
    small = U.to_device(s)
    far = n_pages - 1 - torch.arange(s.k.shape[0], device=dev)     # the same pages at the far end
    k[far], v[far], bounds[far] = small.k, small.v, small.key_bounds
    table = torch.where(torch.from_numpy(s.table).to(dev) < 0, -1, n_pages - 1 - torch.from_numpy(s.table).to(dev)).int()
    big = T.PagedKVCache(k, v, table, s.kv_lens, s.cu_q, hq, bounds)
    new = torch.randn(2, s.total_q, hkv, d, device=dev).bfloat16()
    outs = []
    for kv in (small, big):
        run, out = _calls(T, kv, s.q.to(dev), new[0], new[1], dev)
        run()
        torch.cuda.synchronize()
        assert kv.device_status() == 0
        outs.append(out)
    for n in outs[0]:
        assert torch.equal(outs[0][n], outs[1][n]), n
    assert torch.equal(k[far].nan_to_num(), small.k.nan_to_num()) and torch.equal(bounds[far].nan_to_num(), small.key_bounds.nan_to_num())


def test_the_largest_batch():
    import paper_2604_05438_b200 as T
    rng = np.random.RandomState(94)
    lens = [(int(rng.randint(0, 3)), int(rng.randint(2, 60))) for _ in range(1024)]
    s = U.make_step(4, 2, 64, 16, "bf16", lens, seed=95)
    y, lse = U.gpu_attention(s)
    U.check_attention("bf16", 64, y, lse, *_want(s), n_keys=60)


def test_a_step_without_tokens_leaves_everything():
    import paper_2604_05438_b200 as T
    s = U.make_step(8, 2, 64, 16, "bf16", [(0, 40), (0, 0)], seed=96, with_bounds=True)
    y, lse = U.gpu_attention(s)
    assert y.shape == (0, 8, 64) and lse.shape == (0, 8)
    U.gpu_block_attention(s, 1, 1, 2)
