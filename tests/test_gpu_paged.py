"""GPU parity of the paged-cache calls with the float64 oracle: small cases where the kernels can go wrong (lengths
around tiles and pages, every page size, head layout, type and storage order, masks that leave a row empty, unused slots
full of NaN)."""
import numpy as np
import pytest
import torch

import paged_utils as U
from oracle import paged_oracle as PO

pytestmark = pytest.mark.gpu

GEOMETRIES = [(8, 2, 64), (24, 8, 128), (6, 6, 128), (32, 8, 64), (16, 1, 128), (5, 1, 64), (24, 3, 64)]


def _check(s, dtype, causal=True, scale=None, tokens_first=False):
    y, lse = U.gpu_attention(s, causal, scale, tokens_first)
    want = PO.attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q, causal, scale)
    U.check_attention(dtype, s.q.shape[2], y, lse, *want, n_keys=int(s.kv_lens.max()))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
def test_decode_lengths_around_tiles_and_pages(hq, hkv, d, dtype):
    lens = [(1, n) for n in (1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200)]
    _check(U.make_step(hq, hkv, d, 16, dtype, lens, seed=1), dtype)


@pytest.mark.parametrize("tokens_first", [False, True])
@pytest.mark.parametrize("ps", [16, 32, 64, 128])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (6, 2, 128)])
def test_page_sizes_and_storage_orders(hq, hkv, d, ps, tokens_first):
    lens = [(1, 700), (3, 131), (0, 50), (1, 1), (5, 5), (2, 513)]
    _check(U.make_step(hq, hkv, d, ps, "bf16", lens, seed=2), "bf16", tokens_first=tokens_first)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (6, 2, 128), (3, 3, 128), (32, 2, 64)])
def test_chunks_of_every_length(hq, hkv, d, dtype):
    lens = [(1, 300), (130, 130), (17, 400), (256, 300), (85, 90), (0, 10), (33, 33), (129, 385)]
    _check(U.make_step(hq, hkv, d, 32, dtype, lens, seed=3), dtype)


@pytest.mark.parametrize("lens", [[(1, 0), (3, 2), (1, 129), (40, 7), (2, 200)], [(70, 0), (300, 5)]])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (6, 2, 128)])
def test_full_context_with_empty_and_short_caches(hq, hkv, d, lens):
    _check(U.make_step(hq, hkv, d, 16, "bf16", lens, seed=4), "bf16", causal=False)


@pytest.mark.parametrize("scale", [0.01, 1.0])
def test_scale(scale):
    _check(U.make_step(8, 2, 64, 32, "bf16", [(1, 333), (60, 150)], seed=5), "bf16", scale=scale)


@pytest.mark.parametrize("key_scale", [30.0, 1e-3])
def test_peaked_and_flat_scores(key_scale):
    _check(U.make_step(6, 2, 128, 32, "bf16", [(1, 2000), (90, 400)], seed=6, key_scale=key_scale), "bf16")


def test_one_sequence_is_cut_over_many_ctas():
    _check(U.make_step(4, 1, 64, 64, "fp16", [(1, 20011)], seed=7), "fp16")


def test_many_sequences():
    _check(U.make_step(4, 2, 64, 16, "bf16", [(i % 3, 1 + 7 * i % 90 + i % 3) for i in range(301)], seed=8), "bf16")


# ---------------------------------------------------------------------------------------------- page-selected form
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("sink,tail,topk", [(0, 1, 3), (1, 2, 5), (2, 1, 0), (0, 1, 100), (3, 4, 1)])
@pytest.mark.parametrize("hq,hkv,d,ps", [(8, 2, 64, 16), (6, 2, 128, 32), (16, 1, 128, 16), (3, 3, 64, 64), (6, 2, 64, 128)])
def test_block_attention(hq, hkv, d, ps, sink, tail, topk, dtype):
    lens = [(1, 700), (3, 131), (0, 50), (1, 1), (5, 5), (2, 1025)]
    s = U.make_step(hq, hkv, d, ps, dtype, lens, seed=9, with_bounds=True)
    y, lse, idx = U.gpu_block_attention(s, sink, tail, topk, tokens_first=ps == 32)
    *want, pages = PO.block_attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q,
                                      np.nan_to_num(U.f64(s.bounds)), sink, tail, topk)
    assert (idx == pages).all()
    U.check_attention(dtype, d, y, lse, *want, n_keys=1100)


def test_block_attention_equal_bounds_go_to_the_lower_page():
    s = U.make_step(8, 2, 64, 16, "bf16", [(1, 900), (2, 650)], seed=10, with_bounds=True)
    # pages 3 .. 40 of both sequences share one pair of bounds; page 20 and 21 a larger one
    for b in range(2):
        n = int(s.kv_lens[b]) // 16
        for p in range(3, min(41, n)):
            s.bounds[s.table[b, p]] = s.bounds[s.table[b, 3]]
        for p in (20, 21):
            s.bounds[s.table[b, p], :, 0], s.bounds[s.table[b, p], :, 1] = -9.0, 9.0
    y, lse, idx = U.gpu_block_attention(s, 1, 1, 9)
    *want, pages = PO.block_attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q,
                                      np.nan_to_num(U.f64(s.bounds)), 1, 1, 9)
    assert (idx == pages).all()
    U.check_attention("bf16", 64, y, lse, *want, n_keys=900)


def test_block_attention_long_list_of_pages():
    # more candidate pages than the selecting threads hold in registers, zeros and both signs among the bounds
    s = U.make_step(2, 1, 64, 16, "bf16", [(1, 16 * 9000 + 3)], seed=11, with_bounds=True)
    s.bounds[::7] = 0.0
    s.bounds[::11] = -s.bounds[::11].abs()
    s.bounds[:, :, 0] = torch.minimum(s.bounds[:, :, 0], s.bounds[:, :, 1])
    y, lse, idx = U.gpu_block_attention(s, 2, 3, 777)
    *want, pages = PO.block_attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q,
                                      np.nan_to_num(U.f64(s.bounds)), 2, 3, 777)
    assert (idx == pages).all()
    U.check_attention("bf16", 64, y, lse, *want, n_keys=783 * 16)


def _check_selected(s, dtype, sink, tail, topk):
    y, lse, idx = U.gpu_block_attention(s, sink, tail, topk)
    *want, pages = PO.block_attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q,
                                      np.nan_to_num(U.f64(s.bounds)), sink, tail, topk)
    assert (idx == pages).all()
    U.check_attention(dtype, s.q.shape[2], y, lse, *want, n_keys=(sink + tail + topk) * s.k.shape[2])


@pytest.mark.parametrize("pages,topk", [(1500, 700), (1500, 20), (700, 650), (5000, 1000), (5000, 3)])
def test_block_attention_hundreds_of_equal_bounds(pages, topk):
    # more pages tie at the threshold than are ranked directly; a few are above and below
    s = U.make_step(4, 1, 64, 16, "bf16", [(2, 16 * pages + 5)], seed=12, with_bounds=True)
    s.bounds[:, :, 0], s.bounds[:, :, 1] = -1.0, 1.0
    for p in (pages // 2, pages // 3):
        s.bounds[s.table[0, p], :, 1] = 1.5
    for p in (4, 5, 6):
        s.bounds[s.table[0, p], :, 1] = 0.5
    _check_selected(s, "bf16", 1, 2, topk)


@pytest.mark.parametrize("topk", [30, 600])
def test_block_attention_bounds_that_32_bits_do_not_tell_apart(topk):
    # pages whose bounds differ by one unit of a small element beside large ones: their order is in the last bits
    s = U.make_step(2, 1, 128, 16, "bf16", [(1, 16 * 1200 + 9)], seed=13, with_bounds=True)
    g = torch.Generator().manual_seed(14)
    s.bounds[:, :, 0], s.bounds[:, :, 1] = -1.0, 8.0
    n = int(s.table.max()) + 1
    s.bounds[:n, :, 1, 64:] = (2.0 ** -12 * (1 + torch.randint(0, 64, (n, 1, 64), generator=g) / 128)).bfloat16()
    _check_selected(s, "bf16", 2, 1, topk)


def test_block_attention_scores_too_large_for_32_bits():
    s = U.make_step(2, 1, 64, 16, "bf16", [(1, 16 * 100 + 9)], seed=15, with_bounds=True)
    s.bounds *= 2.0 ** 100
    s.q *= 2.0 ** 30
    s.k *= 2.0 ** -30
    _check_selected(s, "bf16", 1, 1, 9)


@pytest.mark.parametrize("pages,topk", [(9000, 20), (42000, 50)])
def test_block_attention_over_very_many_pages(pages, topk):
    s = U.make_step(2, 1, 64, 16, "fp16", [(1, 16 * pages + 3)], seed=16, with_bounds=True)
    _check_selected(s, "fp16", 1, 2, topk)


# ---------------------------------------------------------------------------------------------- append
def _append_inputs(s, seed, packed):
    g = torch.Generator().manual_seed(seed)
    hkv, d = s.k.shape[1], s.k.shape[3]
    qkv = torch.randn(s.total_q, s.hq + 2 * hkv, d, generator=g).to(s.k.dtype)
    parts = qkv[:, :s.hq], qkv[:, s.hq:s.hq + hkv], qkv[:, s.hq + hkv:]
    return parts if packed else tuple(x.contiguous() for x in parts)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rot,pairs", [(0, False), (1, False), (1, True), (2, False), (2, True)])
@pytest.mark.parametrize("hq,hkv,d,ps,tokens_first", [(8, 2, 64, 16, False), (24, 8, 128, 64, True), (6, 6, 128, 128, False),
                                                      (16, 1, 64, 32, True)])
def test_append(hq, hkv, d, ps, tokens_first, rot, pairs, dtype):
    import paper_2604_05438_b200 as T
    rot = rot * d // 2
    lens = [(1, 1), (1, 64), (1, 65), (3, 140), (0, 20), (200, 200), (130, 333), (16, 16), (17, 17)]
    s = U.make_step(hq, hkv, d, ps, dtype, lens, seed=20, with_bounds=True)
    q, k_new, v_new = (x.cuda() for x in _append_inputs(s, 21, packed=True))
    inv = None if rot == 0 else (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float()
    kv = U.to_device(s, tokens_first)
    kv.key_bounds.fill_(7.0)                       # whatever was there must not matter
    q_out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    T.paged_append(kv, k_new, v_new, None if inv is None else T.RotaryMap(inv.cuda(), pairs), q, q_out)
    torch.cuda.synchronize()
    assert kv.device_status() == 0
    inv64 = None if inv is None else inv.double().numpy()
    k64, v64 = U.f64(s.k), U.f64(s.v)
    want_k, want_v = PO.append(k64, v64, s.table, s.kv_lens, s.cu_q, U.f64(k_new), U.f64(v_new), inv64, pairs)
    got_k, got_v = U.f64(kv.k), U.f64(kv.v)
    np.testing.assert_array_equal(got_v, want_v)
    # a rotated element: one rounding to 16 bits, and fp32 products and sums of magnitudes up to |a| + |c| with sines
    # off by 2^-23 or so: 2^-21 of them
    u = torch.finfo(U.DT[dtype]).eps / 2
    most = float(max(k_new.abs().max(), q.abs().max()))
    np.testing.assert_array_equal(np.isnan(got_k), np.isnan(want_k))
    live = ~np.isnan(want_k)
    assert (np.abs(got_k - want_k)[live] <= (u * np.abs(want_k) + 2.0 ** -20 * most)[live]).all()
    touched = np.zeros(got_k.shape[:3], bool)
    for b, (m, n) in enumerate(lens):
        for t in range(n - m, n):
            touched[s.table[b, t // ps], :, t % ps] = True
    np.testing.assert_array_equal(got_k[~touched], k64[~touched])          # nothing else moved (NaN included)
    pos = np.concatenate([np.arange(n - m, n) for m, n in lens])
    want_q = np.stack([PO.rotate(U.f64(q[i]), pos[i], inv64, pairs) for i in range(s.total_q)])
    got_q = U.f64(q_out)
    assert (np.abs(got_q - want_q) <= u * np.abs(want_q) + 2.0 ** -20 * most).all()
    # bounds: exactly those of the rows that are there now, for the touched pages; the others as they were
    bounds = PO.page_bounds(got_k, s.table, s.kv_lens)
    got_b = U.f64(kv.key_bounds)
    changed = {int(s.table[b, p]) for b, (m, n) in enumerate(lens) if m for p in range((n - m) // ps, (n - 1) // ps + 1)}
    for page in range(len(got_b)):
        if page in changed:
            np.testing.assert_array_equal(got_b[page, :, 0], bounds[page][0])
            np.testing.assert_array_equal(got_b[page, :, 1], bounds[page][1])
        else:
            assert (got_b[page] == 7.0).all()


def test_append_far_positions_and_in_place_queries():
    import paper_2604_05438_b200 as T
    lens = [(5, 40), (2, 2)]
    s = U.make_step(8, 2, 128, 16, "bf16", lens, seed=22)
    q, k_new, v_new = (x.cuda() for x in _append_inputs(s, 23, packed=False))
    inv = (500000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).float()
    positions = torch.tensor([0, 1, 1_048_575, 123_456_789, 2 ** 31, 7, 2 ** 40 + 1], dtype=torch.int64)
    kv = U.to_device(s)
    q_in = U.f64(q)
    T.paged_append(kv, k_new, v_new, T.RotaryMap(inv.cuda()), q, q, positions.cuda())
    torch.cuda.synchronize()
    want_k, _ = PO.append(U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q, U.f64(k_new), U.f64(v_new),
                          inv.double().numpy(), False, positions.numpy())
    # the oracle's own angle carries position * 2^-53 of rounding (2^-13 at 2^40): the two agree to bf16 all the same
    live = ~np.isnan(want_k)
    assert (np.abs(U.f64(kv.k) - want_k)[live] <= 2.0 ** -8 * np.abs(want_k[live]) + 2.0 ** -9).all()
    want_q = np.stack([PO.rotate(q_in[i], int(positions[i]), inv.double().numpy(), False) for i in range(7)])
    assert (np.abs(U.f64(q) - want_q) <= 2.0 ** -8 * np.abs(want_q) + 2.0 ** -9).all()
