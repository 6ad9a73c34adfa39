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


# ---------------------------------------------------------------------------------------------- range of the scores
def _one_high_key(d, dtype, high, at, q_len, kv_len, group=1):
    """A sequence per entry of `high`: all keys score about 0 but the one at position at[i], which scores high[i] (scale 1)."""
    s = U.make_step(group, 1, d, 32, dtype, [(q_len, kv_len)] * len(high), seed=110)
    s.q = (0.25 * s.q.float()).to(s.q.dtype)
    s.q[:, :, 0] = 16.0
    s.k[:, :, :, 0] = torch.where(s.k[:, :, :, 0].isnan(), s.k[:, :, :, 0], 0.0)
    for b, (x, t) in enumerate(zip(high, at)):
        s.k[s.table[b, t // 32], 0, t % 32] = 0.0
        s.k[s.table[b, t // 32], 0, t % 32, 0] = x / 16
    return s


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap", [80, 92, 150, 200, 300, 500])
def test_one_key_far_above_the_first_tile_at_every_offset_of_a_tile(d, dtype, gap):
    s = _one_high_key(d, dtype, [gap] * 128, [128 + o for o in range(128)], 17, 530)
    y, lse = U.gpu_attention(s, scale=1.0)
    want = PO.attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q, True, 1.0)
    U.check_attention(dtype, d, y, lse, *want, n_keys=530)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_scores_of_a_wide_random_spread(d, dtype):
    s = U.make_step(8, 2, d, 32, dtype, [(40, 2100), (3, 900)], seed=111, key_scale=8.0)
    s.q = (12 * s.q.float()).to(s.q.dtype)
    y, lse = U.gpu_attention(s)
    want = PO.attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q)
    U.check_attention(dtype, d, y, lse, *want, n_keys=2100)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,low", [("bf16", -118.0), ("fp16", -28.0)])
def test_the_exponential_over_its_range(d, dtype, low):
    # a sequence per exponent x: the keys of the first tile score 0, one behind it x (in powers of two), and only that one has
    # a value in dim 0, so that y[0] = 2^x / (sum): down to the smallest x whose power the products' type holds.  fp16: scaled
    # by 2^7 there (x >= -21 is a normal number)
    x = torch.linspace(low, 126.0, 245).bfloat16().double().tolist()
    at = [128 + (37 * i) % 128 for i in range(len(x))]
    s = U.make_step(1, 1, d, 32, dtype, [(17, 300)] * len(x), seed=112)
    for t in (s.q, s.k, s.v):
        t[~t.isnan()] = 0.0
    s.q[:, :, 0] = 1.0
    for b in range(len(x)):
        s.k[s.table[b, at[b] // 32], 0, at[b] % 32, 0] = x[b]
        s.v[s.table[b, :9], :, :, 1] = 1.0
        s.v[s.table[b, at[b] // 32], 0, at[b] % 32, :2] = torch.tensor([1.0, 0.0]).to(s.v.dtype)
    y, lse = U.gpu_attention(s, scale=float(np.log(2.0)))
    want, want_lse, A, C = PO.attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q, True, float(np.log(2.0)))
    # fp16: a product below 2^-14 is off by up to 2^-25, 2^-32 of the reference key's weight, so 300 keys by 300 2^-32
    more = 300 * 2.0 ** -32 if dtype == "fp16" else 0.0
    U.check_attention(dtype, d, y - np.clip(y - want, -more, more), lse, want, want_lse, A, C, n_keys=300)
    # relative where check_attention is absolute: two roundings to 16 bits, the score's error (one product: 2^-23 of it
    # twice), the polynomial's and the sum's
    u = torch.finfo(U.DT[dtype]).eps / 2
    X = np.repeat(np.abs(np.array(x)), 17)
    tol = (2 * u + X * 2.0 ** -22 + 2.0 ** -20 + 300 * 2.0 ** -24) * want[:, 0, 0]
    if dtype == "fp16":
        tol = tol + 2.0 ** -25 + more
    assert (np.abs(y[:, 0, 0] - want[:, 0, 0]) <= tol).all()


@pytest.mark.parametrize("dtype,high", [("fp16", 2.0 ** 15), ("bf16", 2.0 ** 15), ("bf16", 2.0 ** 24)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_len,n", [(1, 900), (3, 1200), (1, 20000), (30, 700), (60, 7001)])
def test_scores_of_very_large_size(q_len, n, d, dtype, high):
    # exact products up to 2^30 (2^48), no two of them closer than 2^15: the largest key takes all
    s = U.make_step(2, 1, d, 32, dtype, [(q_len, n)], seed=113)
    g = torch.Generator().manual_seed(114)
    s.q[:] = 0.0
    s.q[:, :, 0] = high
    s.k[~s.k.isnan()] = 0.0
    unit = 128.0 if dtype == "fp16" else high / 256                    # 256 different keys, the largest one from each of them on
    best, at = -1, []
    for t in range(n):
        x = int(torch.randint(0, 4 + 252 * t // n, (1,), generator=g))
        while x == best:                                               # (one key is the largest of those before it)
            x = int(torch.randint(0, 4 + 252 * t // n, (1,), generator=g))
        if x > best:
            best, top = x, t
        at.append(top)
        s.k[s.table[0, t // 32], 0, t % 32, 0] = x * unit
    y, lse = U.gpu_attention(s, scale=1.0)
    v, k = U.f64(s.v), U.f64(s.k)
    u = torch.finfo(U.DT[dtype]).eps / 2
    for i in range(q_len):
        t = at[n - q_len + i]
        row = v[s.table[0, t // 32], 0, t % 32]
        assert (np.abs(y[i] - row) <= 2 * u * np.abs(row) + 2.0 ** -24).all(), i      # (the weight 1 and the output rounded)
        want = high * k[s.table[0, t // 32], 0, t % 32, 0]
        assert (np.abs(lse[i] - want) <= 2.0 ** -21 * want).all()      # product by log2 e, the sum's logarithm, and back


# ---------------------------------------------------------------------------------------------- values that are no numbers
def _check_rows(dtype, d, y, lse, want, n_keys):
    """Rows whose sum is no number: y and lse are NaN.  The others as ever (C without the keys whose score is -inf)."""
    w, want_lse, A, C = (x.reshape(-1, *x.shape[2:]) for x in want)
    y, lse = y.reshape(w.shape), lse.reshape(want_lse.shape)
    none = np.isnan(want_lse)
    np.testing.assert_array_equal(np.isnan(lse), none)
    assert np.isnan(y[none]).all()
    C = np.where(np.isfinite(C), C, 60.0)
    U.check_attention(dtype, d, y[~none], lse[~none], w[~none], want_lse[~none], A[~none], C[~none], n_keys)
    return none


# steps that reach every form: clusters, the line with its join, many rows with and without cuts over the keys
WAYS = [([(1, 500)] * 4, 4, 2), ([(1, 20011)], 4, 1), ([(3, 1500), (1, 900), (2, 65)], 4, 2), ([(45, 7001)], 4, 1),
        ([(60, 700), (33, 33), (1, 300)], 6, 2), ([(300, 300)], 3, 1)]


def _step_of(way, d, dtype, seed):
    lens, hq, hkv = WAYS[way]
    return U.make_step(hq, hkv, d, 32, dtype, lens, seed=seed, with_bounds=True)


def _attend_both(s):
    y, lse = U.gpu_attention(s)
    with np.errstate(all="ignore"):
        return y, lse, PO.attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_a_query_that_is_no_number_makes_its_row_none(way, d, dtype):
    s = _step_of(way, d, dtype, 120)
    T, hq = s.q.shape[:2]
    s.q[T // 2, hq - 1, 3] = float("nan")
    none = _check_rows(dtype, d, *_attend_both(s), int(s.kv_lens.max()))
    assert none.sum() == 1


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["nan", "inf"])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_a_key_that_is_no_number_makes_the_rows_that_see_it_none(way, what, d, dtype):
    # (an infinite one: rows whose score is -inf are without it; +inf is no number in the softmax)
    s = _step_of(way, d, dtype, 121)
    n = int(s.kv_lens[0])
    for t in {n // 3, n - 1, min(n - 1, 136)}:
        s.k[s.table[0, t // 32], 0, t % 32, 5] = float(what)
    none = _check_rows(dtype, d, *_attend_both(s), int(s.kv_lens.max()))
    assert what == "inf" or none.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("o", [0, 1, 2, 7, 64, 120])
def test_one_key_that_is_no_number_at_any_offset_of_a_tile(o, d, dtype):
    s = U.make_step(4, 1, d, 32, dtype, [(20, 600), (40, 300)], seed=124)
    s.k[s.table[0, (256 + o) // 32], 0, (256 + o) % 32, 9] = float("nan")
    none = _check_rows(dtype, d, *_attend_both(s), 600)
    assert none.sum() == 80


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(1, 20011), (1, 300)], [(1, 4000), (1, 300)], [(45, 7001), (20, 300)]])
def test_pieces_of_a_row_whose_keys_are_all_no_numbers(lens, d, dtype):
    # whole warps, tiles and chunks without a single number
    s = U.make_step(4, 1, d, 32, dtype, lens, seed=122)
    for p in range(64, 96):
        s.k[s.table[0, p]] = float("nan")
    none = _check_rows(dtype, d, *_attend_both(s), int(s.kv_lens.max()))
    assert none.any() and not none.all()


# ---------------------------------------------------------------------------------------------- page bounds at their edges
@pytest.mark.parametrize("pages,topk", [(700, 300), (700, 20), (1020, 600), (2500, 900)])
def test_bounds_that_differ_in_the_last_of_64_bits(pages, topk):
    # more than 512 pages too close for 32 bits, of both signs: 1 + k 2^-50, the larger ones behind the smaller ones
    s = U.make_step(2, 1, 64, 16, "bf16", [(1, 16 * pages + 9)], seed=140, with_bounds=True)
    s.q[:] = 0.0
    s.q[:, :, 0], s.q[:, :, 1] = 1.0, 2.0 ** -25
    s.bounds[:] = 0.0
    s.bounds[:, :, 1, 0] = 1.0
    g = torch.Generator().manual_seed(141)
    for p in range(pages + 1):
        s.bounds[s.table[0, p], :, 1, 1] = (1 + int(torch.randint(0, 1 + 254 * p // pages, (1,), generator=g))) * 2.0 ** -25
    for p in (5, 77, 300):
        s.bounds[s.table[0, p], :, :, 0] = -1.0
    y, lse, idx = U.gpu_block_attention(s, 1, 1, topk)
    want, got = _want_selected(s, 1, 1, topk)
    assert (idx == got).all()
    U.check_attention("bf16", 64, y, lse, *want, n_keys=(topk + 2) * 16)


# ---------------------------------------------------------------------------------------------- small probabilities
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[(1, 500)], [(1, 20000)], [(4, 300)], [(30, 300)]])
def test_many_keys_far_below_a_few(lens, d, dtype):
    # one key in 16 has e^18 = 2^26 times the weight of each other one, and value 0: y is made of the others alone
    s = U.make_step(4, 1, d, 32, dtype, lens * 3, seed=130)
    s.q[:] = 0.0
    s.q[:, :, 0] = 8.0
    s.k[~s.k.isnan()] = 0.0
    s.k[:, :, ::16, 0] = torch.where(s.k[:, :, ::16, 0].isnan(), s.k[:, :, ::16, 0], 2.25)
    s.v = torch.where(s.v.isnan(), s.v, 16384.0 + 4096.0 * s.v.float().clamp(-3, 3)).to(s.v.dtype)
    s.v[:, :, ::16] = torch.where(s.v[:, :, ::16].isnan(), s.v[:, :, ::16], 0.0)
    y, lse = U.gpu_attention(s, scale=1.0)
    want, want_lse, A, C = PO.attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q, True, 1.0)
    n = int(s.kv_lens.max())
    # Many rows of fp16: a probability is rounded once as 2^7 p, here 2^-19, by up to 2^-25 absolute.  That is 2^-32 of the
    # weight of one of the keys on top, for 15 keys of values up to 28672 per key on top.  (In range of the type otherwise.)
    more = 15 * 2.0 ** -32 * 28672 if dtype == "fp16" and lens[0][0] == 30 else 0.0
    y = y - np.clip(y - want, -more, more)
    U.check_attention(dtype, d, y, lse, want, want_lse, A, C, n_keys=n)
    # That tolerance counts two roundings to 16 bits; with few rows the probabilities are pairs: the output's alone, and
    # the error of an exponent's argument of 26 (2^-22 of it), of exp2 (2^-21), of a pair (2^-16) and of the sums.
    if lens[0][0] < 30:
        u = torch.finfo(U.DT[dtype]).eps / 2
        tol = (u + 26 * 2.0 ** -22 + 2.0 ** -20 + 2.0 ** -16 + 2 * n * 2.0 ** -24) * np.abs(want)
        assert (np.abs(y - want) <= tol).all(), float((np.abs(y - want) / tol).max())


# ---------------------------------------------------------------------------------------------- infinite bounds
@pytest.mark.parametrize("pages,topk", [(60, 7), (700, 30), (1500, 20), (5000, 600)])
@pytest.mark.parametrize("share", [0.02, 0.6, 1.0])
@pytest.mark.parametrize("counts", [False, True])
def test_infinite_bounds(pages, topk, share, counts):
    # one infinite element in some pages: which side of it counts goes by the query's sign.  Without `counts` it is always the
    # one that does not, so that every bound is finite
    s = U.make_step(1, 1, 64, 16, "fp16", [(1, 16 * pages + 9)], seed=142, with_bounds=True)
    g = torch.Generator().manual_seed(143)
    for p in range(pages + 1):
        if float(torch.rand(1, generator=g)) < share:
            c, side = int(torch.randint(0, 64, (1,), generator=g)), p % 2
            if not counts:
                side = 0 if float(s.q[0, 0, c]) > 0 else 1
            s.bounds[s.table[0, p], 0, side, c] = float("inf") if side else -float("inf")
    s.q[:, :, 11] = 0.0
    s.bounds[:, :, :, 11] = s.bounds[:, :, :, 11].nan_to_num(0.0, 0.0, 0.0)
    y, lse, idx = U.gpu_block_attention(s, 1, 2, topk)
    *want, got = PO.block_attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), s.table, s.kv_lens, s.cu_q,
                                    np.nan_to_num(U.f64(s.bounds), nan=0.0, posinf=np.inf, neginf=-np.inf), 1, 2, topk)
    assert (idx == got).all()
    U.check_attention("fp16", 64, y, lse, *want, n_keys=(topk + 3) * 16)


def test_an_infinite_bound_beside_a_zero_of_the_query():
    # 0 * inf counts as 0: a page with an infinite key element that the query does not look at is no better than without
    s = U.make_step(1, 1, 64, 16, "fp16", [(1, 16 * 300 + 9)], seed=144, with_bounds=True)
    s.q[:, :, 11] = 0.0
    plain = U.Step(s.k, s.v, s.table, s.kv_lens, s.cu_q, s.hq, s.q, s.bounds.clone())
    plain.bounds[:, :, :, 11] = 0.0
    s.bounds[:, :, 0, 11], s.bounds[:, :, 1, 11] = -1.0, float("inf")
    _, _, idx = U.gpu_block_attention(s, 1, 2, 20)
    assert (idx == _want_selected(plain, 1, 2, 20)[1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_selection_for_a_query_that_is_no_number(what, dtype):
    # whatever it selects, its page list is whole, its output is no number, and the tokens beside it are as ever
    s = U.make_step(8, 2, 64, 16, dtype, [(5, 16 * 700), (1, 900)], seed=145, with_bounds=True)
    s.q[2, :, 3] = what
    y, lse, idx = U.gpu_block_attention(s, 1, 1, 9)
    with np.errstate(all="ignore"):
        (want, want_lse, A, C), pages = _want_selected(s, 1, 1, 9)
    rest = [0, 1, 3, 4, 5]
    assert (idx[rest] == pages[rest]).all()
    U.check_attention(dtype, 64, y[rest], lse[rest], want[rest], want_lse[rest], A[rest], C[rest], n_keys=11 * 16)
    assert (np.diff(idx[2], axis=-1) > 0).all() and (idx[2] >= 0).all() and (idx[2] < 700).all()
    if what != what:
        assert np.isnan(y[2]).all() and np.isnan(lse[2]).all()


# ---------------------------------------------------------------------------------------------- values that some rows do not see
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,lens", [(8, 2, [(4, 300), (2, 77), (3, 3)]), (16, 2, [(2, 500)]), (2, 2, [(16, 40), (9, 200)]),
                                         (8, 2, [(70, 500), (130, 130), (4, 200)]), (3, 1, [(300, 301)]), (1, 1, [(256, 400), (33, 1000)]),
                                         (16, 1, [(50, 333)]), (4, 1, [(45, 7001)])])
def test_values_that_are_no_numbers_stay_out_of_the_rows_that_do_not_see_them(hq, hkv, lens, d, dtype, what):
    s = U.make_step(hq, hkv, d, 32, dtype, lens, seed=123, with_bounds=True)
    for b, (m, n) in enumerate(lens):
        for t, c in ((n - 1, 7), (n - (m + 1) // 2, 60), (n - m + 1, 0)):         # keys of new tokens
            s.v[s.table[b, t // 32], :, t % 32, c:c + 2] = what
    for form in ("all", "selected"):
        if form == "all":
            y, lse, (want, want_lse, A, C) = _attend_both(s)
        else:
            y, lse, idx = U.gpu_block_attention(s, 1, 1, 5)
            with np.errstate(all="ignore"):
                (want, want_lse, A, C), pages = _want_selected(s, 1, 1, 5)
            assert (idx == pages).all()
        out = ~np.isfinite(want)
        assert out.any() and not out.all()
        np.testing.assert_array_equal(~np.isfinite(y), out)
        y, want, A = (np.where(out, 0.0, x) for x in (y, want, A))
        U.check_attention(dtype, d, y, lse, want, want_lse, A, C, n_keys=int(s.kv_lens.max()))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_and_missing_values_of_one_dim_add_up(d, dtype):
    # per token: inf alone stays inf (many rows), inf and -inf or NaN give NaN, in the dims that have them and from the first
    # token on that sees them
    s = U.make_step(2, 1, d, 16, dtype, [(200, 450)], seed=125)
    for t, c, x in ((300, 1, "inf"), (310, 2, "-inf"), (320, 2, "inf"), (330, 3, "nan"), (260, 3, "inf"), (449, 4, "inf"), (260, 40, "-inf")):
        s.v[s.table[0, t // 16], 0, t % 16, c] = float(x)
    y, lse, (want, want_lse, A, C) = _attend_both(s)
    np.testing.assert_array_equal(np.isnan(y), np.isnan(want))
    np.testing.assert_array_equal(np.isinf(y) * np.sign(np.nan_to_num(y)), np.isinf(want) * np.sign(np.nan_to_num(want)))
    out = ~np.isfinite(want)
    y, want, A = (np.where(out, 0.0, x) for x in (y, want, A))
    U.check_attention(dtype, d, y, lse, want, want_lse, A, C, n_keys=450)


# ---------------------------------------------------------------------------------------------- thread blocks without work
@pytest.mark.parametrize("d", [64, 128])
def test_replays_with_shorter_lengths_between_other_calls(d):
    # the graph's grid is that of the captured lengths: with shorter ones some thread blocks have nothing to do, and their
    # shared memory holds what other calls left there
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    lens, short = [(40, 900), (90, 9000), (7, 64)], [(40, 41), (90, 95), (7, 60)]
    s = U.make_step(8, 2, d, 16, "bf16", lens, seed=160)
    kv, q = U.to_device(s), s.q.to(dev)
    y, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=dev)
    ws = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_ATTENTION), dtype=torch.uint8, device=dev)
    T.paged_attention(kv, q, y, lse, None, 0, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        T.paged_attention(kv, q, y, lse, None, 0, ws)
    others = [U.make_step(8, 2, dd, 32, "bf16", [(300, 5000), (64, 700)], seed=161) for dd in (64, 128)]
    others = [(U.to_device(o), o.q.to(dev), torch.empty_like(o.q, device=dev), torch.empty(1 << 28, dtype=torch.uint8, device=dev)) for o in others]
    kv.kv_lens_dev.copy_(torch.tensor([n for _, n in short]))
    step = U.Step(s.k, s.v, s.table, np.array([n for _, n in short], np.int64), s.cu_q, 8, s.q)
    want = PO.attention(U.f64(s.q), U.f64(s.k), U.f64(s.v), step.table, step.kv_lens, s.cu_q)
    for i in range(12):
        o = others[i % 2]
        T.paged_attention(o[0], o[1], o[2], None, None, i % 2 * T.FLAG_FULL_CONTEXT, o[3])
        y.fill_(7)
        graph.replay()
        assert kv.device_status() == 0
        U.check_attention("bf16", d, U.f64(y), U.f64(lse), *want, n_keys=95)
# ---------------------------------------------------------------------------------------------- streams
def _one_call(s, kv, stream):
    import paper_2604_05438_b200 as T
    q = s.q.cuda()
    out = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda:0")
    ws = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_ATTENTION), dtype=torch.uint8, device="cuda:0")
    torch.cuda.current_stream().synchronize()
    T.paged_attention(kv, q, *out, None, 0, ws, stream=stream)
    return out + (q, ws)


def test_a_call_on_another_stream_waits_for_the_status_word_that_the_cache_made():
    import paper_2604_05438_b200 as T
    s = U.make_step(4, 2, 64, 16, "bf16", [(1, 100)], seed=150)
    s.table[0, 2] = -1                                      # a page that is reported
    k, v, table = s.k.cuda(), s.v.cuda(), torch.from_numpy(s.table).cuda()
    lens, cu, q = torch.tensor(s.kv_lens).cuda(), torch.tensor(s.cu_q).cuda(), s.q.cuda()
    y, lse, ws = torch.empty_like(q), torch.empty(1, 4, device="cuda:0"), torch.empty(1 << 24, dtype=torch.uint8, device="cuda:0")
    side, maker = torch.cuda.Stream(), torch.cuda.Stream()
    # (a first call loads the kernels, which may wait for the device)
    T.paged_attention(T.PagedKVCache(k, v, table, s.kv_lens, s.cu_q, 4), q, y, lse, None, 0, ws)
    torch.cuda.synchronize()
    with torch.cuda.stream(maker):
        torch.cuda._sleep(100_000_000)                      # the zero of the status word comes behind this
        kv = T.PagedKVCache(k, v, table, s.kv_lens, s.cu_q, 4, kv_lens_dev=lens, cu_q_dev=cu)
    T.paged_attention(kv, q, y, lse, None, 0, ws, stream=side)
    torch.cuda.synchronize()
    assert kv.device_status() == -1


@pytest.mark.parametrize("given", [False, True])
def test_memory_that_the_cache_made_is_kept_until_a_call_on_another_stream_is_complete(given):
    import paper_2604_05438_b200 as T
    s = U.make_step(4, 2, 64, 16, "bf16", [(1, 100)], seed=151)
    k, v, table = s.k.cuda(), s.v.cuda(), torch.from_numpy(s.table).cuda()
    more = dict(kv_lens_dev=torch.tensor(s.kv_lens).cuda(), cu_q_dev=torch.tensor(s.cu_q).cuda()) if given else {}
    side = torch.cuda.Stream()
    for use in ("argument", "current"):
        kv = T.PagedKVCache(k, v, table, s.kv_lens, s.cu_q, 4, **more)
        made = {t.untyped_storage().data_ptr() for t in ([kv.status] if given else [kv.status, kv.kv_lens_dev, kv.cu_q_dev])}
        size = max(t.untyped_storage().nbytes() for t in (kv.status, kv.kv_lens_dev, kv.cu_q_dev))
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        if use == "argument":
            keep = _one_call(s, kv, side)
        else:
            with torch.cuda.stream(side):
                q = s.q.cuda(non_blocking=True)
                ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda:0")
                keep = torch.empty_like(q), q, ws
                T.paged_attention(kv, q, keep[0], None, None, 0, ws)
        busy = not side.query()
        del kv
        fresh = [torch.empty(size, dtype=torch.uint8, device="cuda:0") for _ in range(8)]
        taken = {t.data_ptr() for t in fresh} & made
        torch.cuda.synchronize()
        assert busy and not taken, use
        del keep, fresh


def test_the_same_results_on_another_stream_than_the_cache_was_made_on():
    import paper_2604_05438_b200 as T
    s = U.make_step(4, 2, 64, 16, "bf16", [(1, 100), (40, 90)], seed=152)
    want, want_lse = U.gpu_attention(s)
    side = torch.cuda.Stream()
    for _ in range(3):
        kv = U.to_device(s)
        y, lse, *keep = _one_call(s, kv, side)
        del kv
        junk = [torch.full((4096,), 255, dtype=torch.uint8, device="cuda:0") for _ in range(4)]
        torch.cuda.synchronize()
        np.testing.assert_array_equal(U.f64(y), want)
        np.testing.assert_array_equal(U.f64(lse), want_lse)


def test_device_status_waits_for_calls_on_every_stream():
    import paper_2604_05438_b200 as T
    s = U.make_step(4, 2, 64, 16, "bf16", [(1, 100)], seed=153)
    s.table[0, 2] = -1
    kv, q = U.to_device(s), s.q.cuda()
    y, ws = torch.empty_like(q), torch.empty(1 << 24, dtype=torch.uint8, device="cuda:0")
    T.paged_attention(U.to_device(s), q, y, None, None, 0, ws)         # (loads the kernels)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    T.paged_attention(kv, q, y, None, None, 0, ws, stream=side)
    assert kv.device_status() == -1


@pytest.mark.parametrize("use", ["argument", "current"])
def test_memory_that_a_contiguous_cache_made_is_kept_for_other_streams_too(use):
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    k = torch.randn(2, 300, 64, device=dev).bfloat16()
    q, y = torch.randn(1, 4, 64, device=dev).bfloat16(), torch.empty(1, 4, 64, device=dev)
    topk = np.array([20], np.int32)
    topk_dev, side = torch.from_numpy(topk).to(dev), torch.cuda.Stream()
    kv = T.KVCache(k, k, np.array([0, 300]), 4, 64, 4, 16, n_tail_seq=[12])
    ws = torch.empty(T.workspace_bytes(kv, topk, 20, T.WS_TOPK_DECODE), dtype=torch.uint8, device=dev)
    T.topk_decode(kv, q, topk, topk_dev, 20, None, y, ws)              # (loads the kernels)
    torch.cuda.synchronize()
    want = y.clone()
    made = {kv.cu_seqlens_dev.untyped_storage().data_ptr(), kv.n_tail_seq_dev.untyped_storage().data_ptr()}
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    if use == "argument":
        T.topk_decode(kv, q, topk, topk_dev, 20, None, y, ws, stream=side)
    else:
        with torch.cuda.stream(side):
            T.topk_decode(kv, q, topk, topk_dev, 20, None, y, ws)
    busy = not side.query()
    del kv
    fresh = [torch.empty(16, dtype=torch.uint8, device=dev) for _ in range(8)]
    taken = {t.data_ptr() for t in fresh} & made
    torch.cuda.synchronize()
    assert busy and not taken
    assert torch.equal(y, want)


def test_two_captured_steps_replayed_side_by_side():
    # each with outputs, status word and workspaces of its own
    import paper_2604_05438_b200 as T
    dev = torch.device("cuda:0")
    jobs = []
    for i, lens in enumerate(([(1, 3000), (50, 700), (1, 9)], [(90, 2000), (1, 20000), (3, 400)])):
        s = U.make_step(8, 2, 64, 32, "bf16", lens, seed=170 + i, with_bounds=True)
        kv, q, sel = U.to_device(s), s.q.to(dev), T.PageSelection(1, 2, 4)
        out = torch.zeros_like(q), torch.zeros(q.shape[:2], device=dev), torch.zeros_like(q)
        idx = torch.zeros(q.shape[0], 2, sel.n_pages, dtype=torch.int32, device=dev)
        wa = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_ATTENTION), dtype=torch.uint8, device=dev)
        wb = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_BLOCK_ATTENTION, sel), dtype=torch.uint8, device=dev)

        def run(kv=kv, q=q, sel=sel, out=out, idx=idx, wa=wa, wb=wb):
            T.paged_attention(kv, q, out[0], out[1], None, 0, wa)
            T.paged_block_attention(kv, sel, q, out[2], None, idx, None, wb)
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in out + (idx,)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        jobs.append((graph, out + (idx,), want, kv, run))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(6):
        for job in jobs:
            for t in job[1]:
                t.fill_(7)
        torch.cuda.synchronize()
        for st, job in zip(streams, jobs):
            with torch.cuda.stream(st):
                for _ in range(3):
                    job[0].replay()
        torch.cuda.synchronize()
        for _, got, want, kv, _ in jobs:
            assert kv.device_status() == 0
            for a, b in zip(got, want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", range(len(WAYS)))
def test_outputs_in_the_place_of_the_queries(way, d):
    import paper_2604_05438_b200 as T
    s = _step_of(way, d, "bf16", 180)
    kv, sel = U.to_device(s), T.PageSelection(1, 1, 5)
    ws = [torch.empty(T.paged_workspace_bytes(kv, w, sel), dtype=torch.uint8, device="cuda:0") for w in (T.WS_PAGED_ATTENTION, T.WS_PAGED_BLOCK_ATTENTION)]
    q = s.q.cuda()
    apart = torch.empty_like(q), torch.empty_like(q)
    T.paged_attention(kv, q, apart[0], None, None, 0, ws[0])
    T.paged_block_attention(kv, sel, q, apart[1], None, None, None, ws[1])
    for _ in range(3):
        a, b = q.clone(), q.clone()
        T.paged_attention(kv, a, a, None, None, 0, ws[0])
        T.paged_block_attention(kv, sel, b, b, None, None, None, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(a, apart[0]) and torch.equal(b, apart[1])

