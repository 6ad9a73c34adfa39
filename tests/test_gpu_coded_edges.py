"""GPU tests of the calls over an 8-bit cache where they can go wrong: values that are no numbers, scales far apart, strides,
graphs replayed with other lengths, other streams, bad and far pages, rows that must stay as they are, and a run of the calls
together with the library's summary build and decode step."""
import math

import numpy as np
import pytest
import torch

from oracle import paged8_oracle as P8
from oracle import paged_oracle as PO
from paged8_utils import E8, F8, bounds_of, device_cache, gpu_attention8, gpu_block_attention8, make_step8, to_device8
from paged_utils import DT, check_attention, f64

pytestmark = pytest.mark.gpu

# few rows (one row tile of 8, of 16, several), many rows
WAYS = {"one": (1, 4), "tile": (4, 4), "tiles": (9, 4), "many": (40, 4)}       # way: (q_len, group)


def T():
    import paper_2604_05438_b200
    return paper_2604_05438_b200


def oracle8(s, causal=True, scale=None):
    return PO.attention(f64(s.q), *s.values(), s.table, s.kv_lens, s.cu_q, causal, scale)


def compare8(s, causal=True, scale=None, **kw):
    got = gpu_attention8(s, causal, scale, **kw)
    check_attention(s.dtype, s.k.shape[3], *got, *oracle8(s, causal, scale), int(s.kv_lens.max()))
    return got


def at(s, b, t):
    """Index of position t of sequence b in the cache's arrays, all heads."""
    ps = s.k.shape[2]
    return s.table[b, t // ps], slice(None), t % ps


# ---------------------------------------------------------------------------------------------- numbers
@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 1), (7, 1), (9, 1), (16, 1), (24, 3)])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "fp16")])
def test_every_group(d, dtype, hq, hkv):
    compare8(make_step8(hq, hkv, d, 64, dtype, [(1, 1500), (3, 77), (6, 400), (20, 2100)], seed=20))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1), (9, 1), (12, 1), (16, 1), (32, 2)])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (64, "fp16"), (128, "fp16")])
@pytest.mark.parametrize("lens", [[(1, 1500), (3, 77), (6, 400)],                 # few units: clusters
                                  [(40, 3000)] + [(1, 900 + 64 * i) for i in range(90)]])     # many: pieces of a line
def test_every_group_over_selected_pages(lens, d, dtype, hq, hkv):
    sink, tail, topk, ps = 1, 2, 4, 64
    s = make_step8(hq, hkv, d, ps, dtype, lens, seed=35, with_bounds=True)
    y, lse, idx = gpu_block_attention8(s, sink, tail, topk)
    k, v = s.values()
    wy, wl, A, C, pages = PO.block_attention(f64(s.q), k, v, s.table, s.kv_lens, s.cu_q, f64(s.bounds), sink, tail, topk)
    assert (idx == pages).all()
    check_attention(dtype, d, y, lse, wy, wl, A, C, (sink + tail + topk) * ps)


def test_a_very_long_sequence():
    compare8(make_step8(8, 2, 64, 128, "bf16", [(1, 90001), (2, 40), (1, 1)], seed=21))


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("fp16", 128)])
def test_scores_that_rise_and_fall_along_the_keys(dtype, d, way):
    q_len, g = WAYS[way]
    for sign in (1, -1):
        s = make_step8(2 * g, 2, d, 32, dtype, [(q_len, 1300), (1, 700)], seed=22, spread=0.0)
        u = np.random.default_rng(1).standard_normal(d)
        s.q = (torch.from_numpy(u) + 0.1 * s.q.double()).to(s.q.dtype)
        for b, n in enumerate(s.kv_lens):
            for t in range(int(n)):
                x = t / float(n) if sign == 1 else 1 - t / float(n)
                held, e = P8.hold(np.tile(u * (24 * x - 4), (2, 1)))
                s.ks[at(s, b, t)] = e
                s.k[at(s, b, t)] = torch.from_numpy(held / P8.power(e)[:, None]).to(F8).view(torch.uint8).numpy()
        compare8(s)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_row_sizes_far_apart(dtype, way):
    """Rows' sizes spread over 2^-20 .. 2^20; the values of a row count relative to the largest: 2^-39 of it (few rows) or the
    type's own range (many) are lost, which the tolerance's absolute part has to know."""
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 16, dtype, [(q_len, 333), (1, 50)], seed=23, spread=0.0)
    r = np.random.default_rng(2)
    shape = s.vs.shape
    keep = s.vs != 255
    s.vs[keep] = (s.vs.astype(int) + r.integers(-20, 6, shape))[keep].astype(np.uint8)
    s.ks[keep] = (s.ks.astype(int) + r.integers(-12, 3, shape))[keep].astype(np.uint8)
    y, lse = gpu_attention8(s)
    wy, wl, A, C = oracle8(s)
    _, v = s.values()
    check = np.nanmax(np.abs(v)) * 2.0 ** -24                # one rounding of a subnormal fp16 value, and what is below 2^-39
    big = np.abs(y - wy)
    u = torch.finfo(DT[dtype]).eps / 2
    e = (64 * 2.0 ** -22 * C + 2.0 ** -21)[..., None]
    assert (big <= u * np.abs(wy) + (u + 2 * e + 2 * 333 * 2.0 ** -24) * A + check).all()
    assert np.abs(lse - wl).max() <= e.max() + 1e-4


@pytest.mark.parametrize("way", ["one", "tile", "tiles"])
def test_one_value_far_above_the_others(way):
    """A value 2^30 times the others whose key nothing attends to: the others keep their accuracy to 2^-39 of it."""
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 64, "bf16", [(q_len, 300)], seed=24, spread=0.0)
    s.q = torch.ones_like(s.q)
    s.k[at(s, 0, 100)] = 0xfe                                # -448 in every dim: far below
    s.ks[at(s, 0, 100)] = 127
    s.vs[at(s, 0, 100)] += 30
    y, _ = gpu_attention8(s)
    wy, _, A, _ = oracle8(s)
    big = np.abs(P8.values(s.v, s.vs)[at(s, 0, 100)]).max()
    assert (np.abs(y - wy) <= 2.0 ** -7 * A + 300 * 2.0 ** -39 * big).all()


@pytest.mark.parametrize("way", ["one", "tile", "tiles"])
@pytest.mark.parametrize("power", [-60, -14, 20, 90])
def test_queries_and_keys_of_any_size(power, way):
    """bf16 queries times 2^power, keys times 2^-power: the same scores."""
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 128, 32, "bf16", [(q_len, 500), (1, 33)], seed=25)
    s.q = (s.q.double() * 2.0 ** power).to(s.q.dtype)
    keep = s.ks != 255
    s.ks[keep] = (s.ks.astype(int) - power)[keep].astype(np.uint8)
    compare8(s)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("power", [-112, -90, 105])
def test_queries_and_keys_near_the_ends_of_the_range(power, way):
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 32, "bf16", [(q_len, 500), (1, 33)], seed=31, spread=0.0)
    s.q = (s.q.double() * 2.0 ** power).to(s.q.dtype)
    keep = s.ks != 255
    s.ks[keep] = (s.ks.astype(int) - power)[keep].astype(np.uint8)
    compare8(s)


@pytest.mark.parametrize("way", WAYS)
def test_keys_beyond_2_to_the_115(way):
    """Scores of 2^115 and more, finite: the largest takes all."""
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 32, "bf16", [(q_len, 300)], seed=32, spread=0.0)
    s.ks[s.ks != 255] += 115
    y, lse = gpu_attention8(s)
    k, v = s.values()
    for tok in range(q_len):
        for h in range(2 * g):
            n = 300 - q_len + tok + 1
            score = PO.rows(k, s.table[0], n)[h // g] @ f64(s.q)[tok, h] / 8
            want = PO.rows(v, s.table[0], n)[h // g][score.argmax()]
            first, second = np.sort(score)[-1], np.sort(score)[-2]
            assert first - second > 2.0 ** -18 * first         # (told apart in 32 bits)
            assert (np.abs(y[tok, h] - want) <= 2.0 ** -8 * np.abs(want)).all()
            assert abs(lse[tok, h] - first) <= 2.0 ** -17 * first


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("scale,power", [(1e-20, None), (2.0 ** -100, None), (2.0 ** 100, 60), (2.0 ** 60, -60)])
def test_scales_of_any_size(scale, power, way):
    """Queries of zeros with a very small scale: every key counts the same.  Others with a very large one: finite scores are
    told apart, or (their product with the scale is of usual size) as ever."""
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 32, "bf16", [(q_len, 300), (1, 5)], seed=34, spread=0.0)
    s.q = torch.zeros_like(s.q) if power is None else (s.q.double() * 2.0 ** power).to(s.q.dtype)
    if power == 60:
        s.k[:] = 0                                           # scores of 0 times 2^100
    compare8(s, scale=scale)


@pytest.mark.parametrize("way", WAYS)
def test_values_beyond_2_to_the_110(way):
    """Their mean over 300 keys stays in range, and so does every sum on the way: below 300 * 2^4 * 2^110."""
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 32, "bf16", [(q_len, 300)], seed=33, spread=0.0)
    y0, lse0 = gpu_attention8(s)
    s.vs[s.vs != 255] += 110
    y, lse = gpu_attention8(s)
    assert (y == y0 * 2.0 ** 110).all() and (lse == lse0).all()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "fp16")])
def test_scores_of_very_large_size(d, dtype, way):
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, d, 16, dtype, [(q_len, 200)], seed=26, spread=0.0)
    y, lse = gpu_attention8(s, scale=1e6)
    # the largest score takes all: its value row
    k, v = s.values()
    for tok in range(q_len):
        for h in range(2 * g):
            n = 200 - q_len + tok + 1
            keys = PO.rows(k, s.table[0], n)[h // g]
            score = keys @ f64(s.q)[tok, h] * 1e6
            best = score.argmax()
            if np.sort(score)[-1] - np.sort(score)[-2] < 1e3:
                continue                                     # (as near as 32 bits tell these apart)
            want = PO.rows(v, s.table[0], n)[h // g][best]
            assert (np.abs(y[tok, h] - want) <= 2.0 ** -7 * np.abs(want) + 1e-6).all()
            assert abs(lse[tok, h] - score[best]) <= 2.0 ** -20 * np.abs(keys[best] * f64(s.q)[tok, h]).sum() * 1e6


# ---------------------------------------------------------------------------------------------- no numbers
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("what", ["key", "key scale", "value scale", "query"])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "fp16")])
def test_no_numbers_reach_the_rows_that_see_them_only(d, dtype, what, way):
    q_len, g = WAYS[way]
    lens = [(q_len, 300), (q_len, 300), (1, 90)]
    s = make_step8(2 * g, 2, d, 16, dtype, lens, seed=27)
    clean = gpu_attention8(s)
    pos = 300 - max(q_len // 2, 1)                           # of a token in the middle of the new ones of sequence 0
    tok = pos - (300 - q_len)
    if what == "query":
        s.q[tok, 1, 5] = math.nan
    elif what == "key":
        s.k[s.table[0, pos // 16], 0, pos % 16, 3] = 0xff
    else:
        (s.ks if what == "key scale" else s.vs)[s.table[0, pos // 16], 0, pos % 16] = 255
    y, lse = gpu_attention8(s)
    hit = np.zeros((s.total_q, 2 * g), bool)
    if what == "query":
        hit[tok, 1] = True
    else:
        hit[tok:q_len, :g] = True                            # KV head 0, the tokens from that position on
    assert np.isnan(y[hit]).all() and np.isnan(lse[hit]).all() == (what != "value scale")
    if what == "value scale":
        assert (lse == clean[1]).all()
    # (not bit by bit: a tile that has such values is worked on in another way)
    assert (np.abs(y[~hit] - clean[0][~hit]) <= 2.0 ** -6 * np.abs(clean[0][~hit]).max()).all()
    assert np.abs(lse[~hit] - clean[1][~hit]).max() <= 1e-4


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "bf16")])
def test_a_nan_code_of_a_value_reaches_its_dim_only(d, dtype, way):
    q_len, g = WAYS[way]
    for pos in (0, 130, 300 - max(q_len // 2, 1)):
        s = make_step8(2 * g, 2, d, 32, dtype, [(q_len, 300), (2, 100)], seed=28)
        for i, c in ((5, 0x7f), (d - 1, 0xff)):
            s.v[s.table[0, pos // 32], 1, pos % 32, i] = c
        y, lse = gpu_attention8(s)
        first = max(pos - (300 - q_len), 0)
        hit = np.zeros(y.shape, bool)
        hit[first:q_len, g:, [5, d - 1]] = True
        assert (np.isnan(y) == hit).all() and np.isfinite(lse).all()
        s.v[s.table[0, pos // 32], 1, pos % 32, [5, d - 1]] = 0
        wy, _, A, _ = oracle8(s)
        tol = 2.0 ** (-7 if dtype == "bf16" else -9) * A + 1e-3
        assert (np.abs(y - wy)[~hit] <= tol[~hit]).all()


@pytest.mark.parametrize("way", WAYS)
def test_a_sequence_of_nothing_but_no_numbers(way):
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 16, "bf16", [(q_len, 200), (1, 60)], seed=29)
    for p in s.table[0][:13]:
        s.ks[p] = 255
    y, lse = gpu_attention8(s)
    assert np.isnan(y[:q_len]).all() and np.isnan(lse[:q_len]).all() and np.isfinite(y[q_len:]).all()


# ---------------------------------------------------------------------------------------------- the calls as a program makes them
def make_calls(kv, q, new, dtype, graph_ws=None):
    """(run, outputs): append, read, attention and selected pages of one step."""
    dev = q.device
    hkv, d = kv.k.shape[1], kv.k.shape[3]
    n, hq = q.shape[0], q.shape[1]
    sel = T().PageSelection(1, 1, 3)
    out = {"q": torch.full_like(q, 7), "y": torch.full_like(q, 7), "lse": torch.full((n, hq), 7.0, device=dev), "yb": torch.full_like(q, 7),
           "lse_b": torch.full((n, hq), 7.0, device=dev), "idx": torch.full((n, hkv, 5), 7, dtype=torch.int32, device=dev)}
    total = int(kv.kv_lens.sum())
    out["k16"] = torch.full((total, hkv, d), 7, dtype=DT[dtype], device=dev)
    rows = T().CacheRows(np.concatenate([[0], np.cumsum(kv.kv_lens)]), device=dev)
    ws = [torch.empty(T().paged_workspace_bytes(kv, w, s), dtype=torch.uint8, device=dev) for w, s in
          ((T().WS_PAGED_ATTENTION, None), (T().WS_PAGED_BLOCK_ATTENTION, sel))]
    inv = (10000.0 ** (-torch.arange(16, dtype=torch.float64) / 16)).float().to(dev)
    w = torch.linspace(0.5, 1.5, d, device=dev)
    rotary, norms = T().RotaryMap(inv), T().HeadNorms(w, w, 1e-6)

    def run(stream=None):
        T().paged_append(kv, new[0], new[1], rotary, q, out["q"], norms=norms, stream=stream)
        T().paged_attention(kv, out["q"], out["y"], out["lse"], None, 0, ws[0], stream=stream)
        T().paged_block_attention(kv, sel, out["q"], out["yb"], out["lse_b"], out["idx"], None, ws[1], stream=stream)
        T().paged_read(kv, rows, out["k16"], None, stream=stream)
    run.keep = (ws, rows, rotary, norms)
    return run, out


def new_rows(s, hkv, d, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(2, s.total_q, hkv, d, generator=g).to(DT[s.dtype]).cuda()


@pytest.mark.parametrize("lens,shorter", [([(1, 300), (1, 17), (1, 2000)], [(1, 288), (1, 1), (1, 33)]),
                                          ([(40, 900), (1, 5000), (7, 64)], [(40, 41), (1, 650), (7, 60)]),
                                          ([(20, 1500), (17, 400)], [(20, 128), (17, 17)])])
def test_captured_calls_follow_shorter_device_lengths(lens, shorter):
    s = make_step8(8, 2, 64, 16, "bf16", lens, seed=50, with_bounds=True)
    new, q = new_rows(s, 2, 64, 51), s.q.cuda()
    kv = to_device8(s)
    state = [kv.k, kv.v, kv.k_scales, kv.v_scales, kv.key_bounds]
    kept = [t.clone() for t in state]
    run, out = make_calls(kv, q, new, "bf16")
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for which in (shorter, lens, shorter):
        kv.kv_lens_dev.copy_(torch.tensor([n for _, n in which]))
        for t, t0 in zip(state, kept):
            t.copy_(t0)
        for t in out.values():
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in out.items()}
        # the same step, called with these lengths
        eager = T().PagedKVCache8(*(t.clone() for t in kept[:4]), kv.page_table, [n for _, n in which], s.cu_q, 8, torch.bfloat16, kept[4].clone())
        run2, want = make_calls(eager, q, new, "bf16")
        run2()
        torch.cuda.synchronize()
        for a, b in zip(state, (eager.k, eager.v, eager.k_scales, eager.v_scales, eager.key_bounds)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert torch.equal(got["q"], want["q"]) and torch.equal(got["idx"], want["idx"])
        for n in ("y", "yb"):      # the split over CTAs may differ: equal up to its roundings
            assert (got[n].float() - want[n].float()).abs().max() <= 2.0 ** -6 * want[n].float().abs().max()
        for n in ("lse", "lse_b"):
            assert (got[n] - want[n]).abs().max() <= 1e-4
        # rows read: those below the device lengths, the others as they were
        at_g = at_w = 0
        for (_, n), (_, most) in zip(which, lens):
            assert torch.equal(got["k16"][at_g:at_g + n], want["k16"][at_w:at_w + n])
            assert (got["k16"][at_g + n:at_g + most] == 7).all()
            at_g, at_w = at_g + most, at_w + n
        assert kv.device_status() == 0 and eager.device_status() == 0


def test_two_streams_at_once_and_repeated_calls_are_bit_identical():
    steps = [make_step8(8, 2, 64, 32, "bf16", lens, seed=60 + i, with_bounds=True)
             for i, lens in enumerate(([(1, 3000), (50, 700), (1, 9)], [(90, 2000), (1, 20000), (3, 400)]))]
    runs = [make_calls(to_device8(s), s.q.cuda(), new_rows(s, 2, 64, 70 + i), "bf16") for i, s in enumerate(steps)]
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


def test_rows_made_on_one_stream_and_read_on_another():
    s = make_step8(4, 2, 64, 16, "bf16", [(0, 200), (0, 33)], seed=61)
    side = torch.cuda.Stream()
    kv = to_device8(s)
    out = torch.zeros(233, 2, 64, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        rows = T().CacheRows([0, 200, 233], [0, 0], device="cuda")
        with torch.cuda.stream(side):
            T().paged_read(kv, rows, out, None)
        del rows
        torch.full((64,), 99, dtype=torch.int64, device="cuda")       # would land in the rows' memory
    torch.cuda.synchronize()
    want, _ = s.values()
    got = f64(out)
    for t in range(200):
        assert (got[t] == want[s.table[0, t // 16], :, t % 16]).all()
    assert kv.device_status() == 0


@pytest.mark.parametrize("bad", [-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31])
def test_bad_pages_are_reported_and_touch_only_their_sequence(bad):
    lens = [(1, 300), (40, 200), (1, 128), (20, 64)]
    s = make_step8(8, 2, 64, 16, "bf16", lens, seed=91, with_bounds=True)
    n_pages = s.k.shape[0]
    new = new_rows(s, 2, 64, 92)
    good = to_device8(s)
    run, want = make_calls(good, s.q.cuda(), new, "bf16")
    run()
    torch.cuda.synchronize()
    assert good.device_status() == 0
    s.table[0, 18] = bad if bad != 10 ** 6 else n_pages       # the page of a decoding sequence's last token
    s.table[1, 11] = bad if bad != 10 ** 6 else n_pages       # a page in the middle of a chunk
    kv = to_device8(s)
    k0 = kv.k.clone().view(torch.uint8)
    run, out = make_calls(kv, s.q.cuda(), new, "bf16")
    run()
    torch.cuda.synchronize()
    assert kv.device_status() == -1
    rows = slice(int(s.cu_q[2]), None)                        # the other two sequences
    for n in want:
        if n != "k16":
            assert torch.equal(want[n][rows], out[n][rows]), n
    assert torch.equal(want["k16"][500:], out["k16"][500:])
    assert (out["k16"][288:300] == 7).all()                   # rows of the bad page
    touched = {int(s.table[b, p]) for b, (m, n) in enumerate(lens) for p in range((n - m) // 16, (n - 1) // 16 + 1)}
    for page in range(n_pages):
        if page not in touched:
            assert torch.equal(kv.k.view(torch.uint8)[page], k0[page])


def test_offsets_beyond_32_bits():
    hq, hkv, d, ps = 24, 8, 128, 64
    n_pages = 72000                                          # 4.7 GB of key codes
    k, v = (torch.empty(n_pages, hkv, ps, d, dtype=torch.uint8, device="cuda").view(F8) for _ in range(2))
    ks, vs = (torch.empty(n_pages, hkv, ps, dtype=torch.uint8, device="cuda").view(E8) for _ in range(2))
    bounds = torch.empty(n_pages, hkv, 2, d, dtype=torch.bfloat16, device="cuda")
    s = make_step8(hq, hkv, d, ps, "bf16", [(1, 500), (30, 200)], seed=93, with_bounds=True, spare=0)
    small = to_device8(s)
    far = n_pages - 1 - torch.arange(s.k.shape[0], device="cuda")     # the same pages at the far end
    for x, y in ((k, small.k), (v, small.v), (ks, small.k_scales), (vs, small.v_scales)):
        x.view(torch.uint8)[far] = y.view(torch.uint8)
    bounds[far] = small.key_bounds
    table = torch.from_numpy(s.table).cuda()
    table = torch.where(table < 0, -1, n_pages - 1 - table).int()
    big = T().PagedKVCache8(k, v, ks, vs, table, s.kv_lens, s.cu_q, hq, torch.bfloat16, bounds)
    new = new_rows(s, hkv, d, 94)
    outs = []
    for kv in (small, big):
        run, out = make_calls(kv, s.q.cuda(), new, "bf16")
        run()
        torch.cuda.synchronize()
        assert kv.device_status() == 0
        outs.append(out)
    for n in outs[0]:
        assert torch.equal(outs[0][n], outs[1][n]), n
    assert torch.equal(k.view(torch.uint8)[far], small.k.view(torch.uint8)) and torch.equal(bounds[far].nan_to_num(), small.key_bounds.nan_to_num())
    assert torch.equal(ks.view(torch.uint8)[far], small.k_scales.view(torch.uint8))


def test_the_largest_batch():
    r = np.random.default_rng(5)
    lens = [(int(r.integers(0, 3)), int(r.integers(3, 200))) for _ in range(1024)]
    s = make_step8(4, 2, 64, 16, "bf16", lens, seed=95, with_bounds=True)
    kv = to_device8(s)
    run, out = make_calls(kv, s.q.cuda(), new_rows(s, 2, 64, 96), "bf16")
    run()
    torch.cuda.synchronize()
    assert kv.device_status() == 0
    after = make_step8(4, 2, 64, 16, "bf16", lens, seed=95)
    for a, t in ((after.k, kv.k), (after.v, kv.v), (after.ks, kv.k_scales), (after.vs, kv.v_scales)):
        a[:] = t.view(torch.uint8).cpu().numpy()
    after.q = out["q"].cpu()
    check_attention("bf16", 64, f64(out["y"]), f64(out["lse"]), *oracle8(after), 200)
    assert torch.equal(kv.key_bounds.cpu().nan_to_num(), bounds_of(after).nan_to_num())


def test_rows_behind_the_last_sequence_and_workspace_ends_stay_as_they_are():
    s = make_step8(6, 2, 128, 16, "fp16", [(1, 100), (60, 200), (0, 30)], seed=80, with_bounds=True)
    kv, n = to_device8(s), s.total_q

    def guarded(shape, dtype):
        big = torch.full((shape[0] + 9,) + shape[1:], 7, dtype=dtype, device="cuda")
        return big, big[:shape[0]]
    sel = T().PageSelection(1, 1, 3)
    bigs = {k: guarded(sh, dt) for k, sh, dt in (("q", (n, 6, 128), torch.float16), ("y", (n, 6, 128), torch.float16), ("lse", (n, 6), torch.float32),
                                                 ("idx", (n, 2, 5), torch.int32), ("k", (330, 2, 128), torch.float16))}
    sizes = [T().paged_workspace_bytes(kv, T().WS_PAGED_ATTENTION), T().paged_workspace_bytes(kv, T().WS_PAGED_BLOCK_ATTENTION, sel)]
    ws = [torch.full((b + 4096,), 0x5a, dtype=torch.uint8, device="cuda") for b in sizes]
    new = new_rows(s, 2, 128, 81)
    T().paged_append(kv, new[0], new[1], None, s.q.cuda(), bigs["q"][1])
    T().paged_attention(kv, bigs["q"][1], bigs["y"][1], bigs["lse"][1], None, 0, ws[0][:sizes[0]])
    T().paged_block_attention(kv, sel, bigs["q"][1], bigs["y"][1], bigs["lse"][1], bigs["idx"][1], None, ws[1][:sizes[1]])
    T().paged_read(kv, T().CacheRows([0, 100, 300, 330], device="cuda"), bigs["k"][1], None)
    torch.cuda.synchronize()
    assert kv.device_status() == 0
    for k, (big, part) in bigs.items():
        assert (big[part.shape[0]:] == 7).all(), k
    for w, b in zip(ws, sizes):
        assert (w[b:] == 0x5a).all()
    with pytest.raises(T().TkphiError) as e:
        T().paged_attention(kv, bigs["q"][1], bigs["y"][1], None, None, 0, ws[0][:sizes[0] - 256])
    assert e.value.status == -3


def test_outputs_of_read_at_any_stride():
    """Rows whose pieces are aligned to 16 bytes but not to 32, and heads between rows."""
    s = make_step8(4, 2, 64, 16, "bf16", [(0, 77)], seed=62)
    kv = to_device8(s)
    want = torch.empty(77, 2, 64, dtype=torch.bfloat16, device="cuda")
    T().paged_read(kv, T().CacheRows([0, 77], device="cuda"), want, None)
    for shape in ((80, 2, 72), (80, 3, 64), (80, 2, 136)):
        for off in (0, 8):
            store = torch.full(shape, 5, dtype=torch.bfloat16, device="cuda")
            view = store[1:78, :2, off:off + 64] if shape[2] >= 64 + off else None
            if view is None:
                continue
            T().paged_read(kv, T().CacheRows([0, 77], device="cuda"), view, None)
            assert torch.equal(view, want)
            view.fill_(5)
            assert (store == 5).all()
    heads = torch.full((2, 90, 64), 5, dtype=torch.bfloat16, device="cuda")
    T().paged_read(kv, T().CacheRows([0, 77], device="cuda"), heads[:, 3:80].transpose(0, 1), heads[:, 3:80].transpose(0, 1).clone())
    assert torch.equal(heads[:, 3:80].transpose(0, 1), want) and (heads[:, 80:] == 5).all() and (heads[:, :3] == 5).all()


def test_positions_of_the_callers_own_and_queries_in_place():
    s = make_step8(4, 2, 64, 16, "bf16", [(3, 40), (1, 7)], seed=63)
    new = new_rows(s, 2, 64, 64)
    inv = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).float()
    pos = torch.tensor([1000003, 5, 77, 123456])
    kv, q = to_device8(s), s.q.cuda()
    T().paged_append(kv, new[0], new[1], T().RotaryMap(inv.cuda()), q, q, positions=pos.cuda())
    got = f64(q)
    for tok in range(4):
        want = PO.rotate(f64(s.q)[tok], int(pos[tok]), inv.double().numpy(), False)
        assert (np.abs(got[tok] - want) <= 2.0 ** -8 * np.abs(want) + 24 * 2.0 ** -24 * np.abs(want).max(-1, keepdims=True)).all()


def test_a_step_without_tokens_leaves_everything():
    s = make_step8(4, 2, 64, 16, "bf16", [(0, 100), (0, 0)], seed=97, with_bounds=True)
    kv = to_device8(s)
    before = [t.clone() for t in (kv.k, kv.v, kv.k_scales, kv.v_scales, kv.key_bounds)]
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(T().paged_workspace_bytes(kv, T().WS_PAGED_ATTENTION), dtype=torch.uint8, device="cuda")
    T().paged_append(kv, none, none, None, q, q)
    T().paged_attention(kv, q, q, None, None, 0, ws)
    T().paged_read(kv, T().CacheRows([0, 0, 0], device="cuda"), none, none)
    torch.cuda.synchronize()
    assert kv.device_status() == 0
    for t, t0 in zip((kv.k, kv.v, kv.k_scales, kv.v_scales, kv.key_bounds), before):
        assert torch.equal(t.view(torch.uint8), t0.view(torch.uint8))


@pytest.mark.parametrize("way", ["one", "tiles", "many"])
def test_outputs_in_the_place_of_the_queries(way):
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 16, "bf16", [(q_len, 300), (1, 50)], seed=98)
    want, _ = gpu_attention8(s)
    kv, q = to_device8(s), s.q.cuda()
    ws = torch.empty(T().paged_workspace_bytes(kv, T().WS_PAGED_ATTENTION), dtype=torch.uint8, device="cuda")
    T().paged_attention(kv, q, q, None, None, 0, ws)
    assert (f64(q) == want).all()


# ---------------------------------------------------------------------------------------------- one step of a model layer
def test_a_prompt_in_8_bits_then_the_summary_build_and_decoding():
    """Chunks of two prompts go into an 8-bit cache and are attended; the prompts are read back into a contiguous 16-bit cache,
    on which summaries are built and Top-K+phi decoding runs; tokens are decoded over the 8-bit cache, with all and with
    selected pages, which with every page selected is the same."""
    hq, hkv, d, ps = 8, 2, 64, 16
    lens = [130, 200]
    g = torch.Generator().manual_seed(40)
    n_pages = sum((n + 4 + ps - 1) // ps for n in lens)
    table = torch.full((2, 13), -1, dtype=torch.int32)
    order, at_page = torch.randperm(n_pages, generator=g).int(), 0
    for b, n in enumerate(lens):
        need = (n + 4 + ps - 1) // ps
        table[b, :need] = order[at_page:at_page + need]
        at_page += need
    table = table.cuda()
    k, v = (torch.zeros(n_pages, hkv, ps, d, dtype=torch.uint8, device="cuda").view(F8) for _ in range(2))
    ks, vs = (torch.zeros(n_pages, hkv, ps, dtype=torch.uint8, device="cuda").view(E8) for _ in range(2))
    bounds = torch.zeros(n_pages, hkv, 2, d, dtype=torch.bfloat16, device="cuda")
    inv = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).float().cuda()
    w = (1 + 0.1 * torch.randn(d, generator=g)).cuda()
    norms, rotary = T().HeadNorms(w, w), T().RotaryMap(inv)

    def step(q_lens, kv_lens):
        cu = np.concatenate([[0], np.cumsum(q_lens)])
        kv = T().PagedKVCache8(k, v, ks, vs, table, kv_lens, cu, hq, torch.bfloat16, bounds)
        qkv = torch.randn(int(cu[-1]), hq + 2 * hkv, d, generator=g).bfloat16().cuda()
        q = torch.empty(int(cu[-1]), hq, d, dtype=torch.bfloat16, device="cuda")
        T().paged_append(kv, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], rotary, qkv[:, :hq], q, norms=norms)
        y, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        ws = torch.empty(T().paged_workspace_bytes(kv, T().WS_PAGED_ATTENTION), dtype=torch.uint8, device="cuda")
        T().paged_attention(kv, q, y, lse, None, 0, ws)
        torch.cuda.synchronize()
        assert kv.device_status() == 0
        raw = [x.view(torch.uint8).cpu().numpy() for x in (k, v, ks, vs)]
        K, V = P8.values(raw[0], raw[2]), P8.values(raw[1], raw[3])
        want = PO.attention(f64(q), K, V, table.cpu().numpy(), kv_lens, cu)
        check_attention("bf16", d, f64(y), f64(lse), *want, max(kv_lens))
        return kv, q, y

    step([70, 1], [70, 1])
    step([60, 199], lens)
    kv, q, y = step([1, 1], [131, 201])
    # the pages that promise most: with as many as there are, plain attention
    sel = T().PageSelection(1, 1, 20)
    yb, idx = torch.empty_like(y), torch.empty(2, hkv, 22, dtype=torch.int32, device="cuda")
    ws = torch.empty(T().paged_workspace_bytes(kv, T().WS_PAGED_BLOCK_ATTENTION, sel), dtype=torch.uint8, device="cuda")
    T().paged_block_attention(kv, sel, q, yb, None, idx, None, ws)
    assert (yb.float() - y.float()).abs().max() <= 2.0 ** -7 * y.float().abs().max()
    # the caches handed to the summary build, head-major
    total = 131 + 201
    flat = torch.empty(2, hkv, total, d, dtype=torch.bfloat16, device="cuda")
    T().paged_read(kv, T().CacheRows([0, 131, total], device="cuda"), flat[0].transpose(0, 1), flat[1].transpose(0, 1))
    whole = T().KVCache(flat[0], flat[1], np.array([0, 131, total]), hq, 64, 4, 16)
    gen = torch.Generator().manual_seed(41)
    phi = T().PhiMaps(*((0.1 * torch.randn(*sh, generator=gen)).cuda() for sh in ((hq, 64, d), (hq, 64), (hkv, 64, d), (hkv, 64))), 0.02, 0.02)
    S, u = torch.empty(2, hkv, d, 64, device="cuda"), torch.empty(2, hkv, 64, device="cuda")
    wb = torch.empty(T().workspace_bytes(whole, None, 0, T().WS_BUILD), dtype=torch.uint8, device="cuda")
    T().build_summaries(whole, phi, S, u, wb)
    topk = np.array([111, 181], np.int32)                    # every mid-region key: plain attention again
    wd = torch.empty(T().workspace_bytes(whole, topk, 181, T().WS_TOPK_DECODE), dtype=torch.uint8, device="cuda")
    yt = torch.empty(2, hq, d, device="cuda")
    T().topk_decode(whole, q, topk, torch.from_numpy(topk).cuda(), 181, None, yt, wd)
    torch.cuda.synchronize()
    assert T().device_status(wd) == 0 and T().device_status(wb) == 0 and torch.isfinite(S).all()
    assert (yt - y.float()).abs().max() <= 2.0 ** -7 * y.float().abs().max()
