"""The 8-bit paged cache on the GPU against the float64 oracle: append (with and without head norms), read, attention,
attention over selected pages; and the head norms of the 16-bit append."""
import math

import numpy as np
import pytest
import torch

from oracle import paged8_oracle as P8
from oracle import paged_oracle as PO
from paged8_utils import (E8, F8, bounds_of, device_cache, gpu_attention8, gpu_block_attention8, make_step8, to_device8)
from paged_utils import DT, check_attention, f64, make_step, to_device

pytestmark = pytest.mark.gpu

GEOMETRIES = [(8, 2, 64), (6, 2, 128), (4, 4, 64), (16, 1, 128)]


def T():
    import paper_2604_05438_b200
    return paper_2604_05438_b200


def raw(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def angles(n, seed=1):
    return (10000.0 ** (-torch.arange(n, dtype=torch.float64) / max(n, 1))).float()


def new_tokens(s, seed, hkv, d, dtype):
    """k_new, v_new, q as slices of one fused projection, on the host."""
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(s.total_q, s.hq + 2 * hkv, d, generator=g).to(DT[dtype])
    return qkv[:, s.hq:s.hq + hkv], qkv[:, s.hq + hkv:], qkv[:, :s.hq]


def places(s, ps):
    """(token row, page, slot) of every new token."""
    for b in range(len(s.kv_lens)):
        m = int(s.cu_q[b + 1] - s.cu_q[b])
        for i in range(m):
            t = int(s.kv_lens[b]) - m + i
            yield int(s.cu_q[b]) + i, int(s.table[b, t // ps]), t % ps, t


def u_of(dtype):
    return torch.finfo(DT[dtype]).eps / 2


def expected_heads(x, weight, eps, position, inv, pairs):
    """Norm and rotation of one token's heads in 64 bits."""
    return PO.rotate(P8.norm(x.double().numpy(), weight, eps), position, inv, pairs)


# an fp32 head after norm and rotation is off by at most this part of its largest magnitude: the sum of squares n 2^-24,
# rsqrt 2^-22, a few products 2^-24 each, sine and cosine 2^-22 with their argument's rounding 2^-22
def slack(d):
    return (d / 2 + 4 + 4 + 8 + 8) * 2.0 ** -24


# ---------------------------------------------------------------------------------------------- append
LENS = [[(1, 1)], [(1, 37), (1, 64), (1, 130)], [(5, 5), (0, 20), (70, 90), (33, 200), (3, 66)]]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("dtype,ps", [("bf16", 16), ("fp16", 64), ("bf16", 128), ("fp16", 32)])
def test_rows_without_arithmetic_are_held_exactly_as_defined(dtype, ps, hq, hkv, d, lens):
    s = make_step8(hq, hkv, d, ps, dtype, lens, seed=3)
    k_new, v_new, q = new_tokens(s, 4, hkv, d, dtype)
    kv = to_device8(s, tokens_first=ps == 32)
    T().paged_append(kv, k_new.cuda(), v_new.cuda())
    assert kv.device_status() == 0
    got = [raw(x) for x in (kv.k, kv.v, kv.k_scales, kv.v_scales)]
    want = [s.k.copy(), s.v.copy(), s.ks.copy(), s.vs.copy()]
    for tok, page, slot, _ in places(s, ps):
        for i, x in ((0, k_new), (1, v_new)):
            held, e = P8.hold(x[tok].double().numpy())
            assert (got[2 + i][page, :, slot] == e).all()
            assert (P8.values(got[i][page, :, slot], got[2 + i][page, :, slot]) == held).all()
            want[i][page, :, slot], want[2 + i][page, :, slot] = got[i][page, :, slot], got[2 + i][page, :, slot]
    for g, w in zip(got, want):
        assert (g == w).all()                              # and nothing else was touched


@pytest.mark.parametrize("rot,pairs,per_head,bounds", [("all", False, False, True), ("half", True, True, True), (None, False, False, False),
                                                       ("half", False, True, False), ("all", True, False, True)])
@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("dtype,ps", [("bf16", 16), ("fp16", 64), ("bf16", 128)])
def test_append_with_norms_and_rotation(dtype, ps, hq, hkv, d, rot, pairs, per_head, bounds):
    lens = [(1, 1), (1, 77), (9, 40), (70, 150), (0, 3)]
    s = make_step8(hq, hkv, d, ps, dtype, lens, seed=5, with_bounds=bounds)
    k_new, v_new, q = new_tokens(s, 6, hkv, d, dtype)
    g = torch.Generator().manual_seed(7)
    wq = 1 + 0.3 * torch.randn(*((hq, d) if per_head else (d,)), generator=g)
    wk = 1 + 0.3 * torch.randn(*((hkv, d) if per_head else (d,)), generator=g)
    n = {"all": d // 2, "half": d // 4, None: 0}[rot]
    inv = angles(n) if n else None
    kv = to_device8(s)
    q_dev, q_out = q.cuda(), torch.full((s.total_q, hq, d), float("nan"), dtype=DT[dtype], device="cuda")
    T().paged_append(kv, k_new.cuda(), v_new.cuda(), T().RotaryMap(inv.cuda(), pairs) if n else None, q_dev, q_out,
                     norms=T().HeadNorms(wq.cuda(), wk.cuda(), 1e-5))
    assert kv.device_status() == 0
    gk, gks = raw(kv.k), raw(kv.k_scales)
    inv64 = None if inv is None else inv.double().numpy()
    q_got = f64(q_out)
    for tok, page, slot, t in places(s, ps):
        x = expected_heads(k_new[tok], wk.double().numpy(), 1e-5, t, inv64, pairs)
        most = np.abs(x).max(-1, keepdims=True)
        got = P8.values(gk[page, :, slot], gks[page, :, slot])
        e = gks[page, :, slot].astype(np.int64)
        # the scale is the defined one, or its neighbour where the largest magnitude is that near to the border
        border = np.abs(most[:, 0] / (448 * 2.0 ** (P8.scale_byte(x) - 127)) - 1) < slack(d)
        assert ((e == P8.scale_byte(x)) | border | (e == P8.scale_byte(x * (1 + slack(d)))) | (e == P8.scale_byte(x * (1 - slack(d))))).all()
        tol = 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * P8.power(e)[:, None] + 1.1 * slack(d) * most
        assert (np.abs(got - x) <= tol).all()
        assert (P8.values(raw(kv.v)[page, :, slot], raw(kv.v_scales)[page, :, slot]) == P8.hold(v_new[tok].double().numpy())[0]).all()
        y = expected_heads(q[tok], wq.double().numpy(), 1e-5, t, inv64, pairs)
        assert (np.abs(q_got[tok] - y) <= u_of(dtype) * np.abs(y) + 1.1 * slack(d) * np.abs(y).max(-1, keepdims=True) + 2.0 ** -25).all()
    if bounds:
        s.k, s.ks = gk, gks
        want = bounds_of(s)
        touched = sorted({page for _, page, _, _ in places(s, ps)})
        assert torch.equal(kv.key_bounds.cpu()[touched], want[touched])
        rest = [i for i in range(len(want)) if i not in touched]
        assert torch.equal(kv.key_bounds.cpu()[rest], s.bounds[rest])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rows_at_the_ends_of_the_range(dtype):
    """Zeros, subnormals, the largest numbers, powers at which the scale changes, infinities and NaN."""
    d, ps, hkv = 64, 16, 2
    fi = torch.finfo(DT[dtype])
    rows = [torch.zeros(d), torch.full((d,), -0.0), torch.full((d,), fi.max), torch.full((d,), fi.tiny), torch.full((d,), fi.smallest_normal * 2 ** -3)]
    for top in (1.75, 1.75 * (1 + fi.eps), 448.0, 448.0 * (1 + fi.eps), 1.0, 2.0):
        r = torch.linspace(-1, 1, d)
        r[5] = top
        rows.append(r)
    for bad in (math.inf, -math.inf, math.nan):
        r = torch.linspace(-1, 1, d)
        r[63] = bad
        rows.append(r)
    x = torch.stack(rows)[:, None].expand(-1, hkv, -1).contiguous().to(DT[dtype])
    n = len(rows)
    s = make_step8(4, hkv, d, ps, dtype, [(n, n)], seed=1)
    kv = to_device8(s)
    T().paged_append(kv, x.cuda(), x.flip(0).contiguous().cuda())
    assert kv.device_status() == 0
    for codes, scales, y in ((kv.k, kv.k_scales, x), (kv.v, kv.v_scales, x.flip(0))):
        c, e = raw(codes), raw(scales)
        for tok, page, slot, _ in places(s, ps):
            held, want = P8.hold(y[tok].double().numpy())
            assert (e[page, :, slot] == want).all(), tok
            assert np.array_equal(P8.values(c[page, :, slot], e[page, :, slot]), held, equal_nan=True), tok


@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("dtype,ps,rot,pairs,sides", [("bf16", 16, 1, False, "both"), ("fp16", 64, 2, True, "both"), ("bf16", 128, 0, False, "k"),
                                                      ("fp16", 32, 1, False, "q")])
def test_norms_of_the_16_bit_append(dtype, ps, rot, pairs, sides, hq, hkv, d):
    lens = [(1, 1), (1, 77), (9, 40), (70, 150), (0, 3)]
    s = make_step(hq, hkv, d, ps, dtype, lens, seed=8, with_bounds=True)
    k_new, v_new, q = new_tokens(s, 9, hkv, d, dtype)
    k_new = k_new * torch.exp2(torch.arange(s.total_q) % 9 - 4.0)[:, None, None].to(DT[dtype])
    g = torch.Generator().manual_seed(10)
    wq = 1 + 0.3 * torch.randn(d, generator=g) if sides != "k" else None
    wk = 1 + 0.3 * torch.randn(hkv, d, generator=g) if sides != "q" else None
    n = d // 2 // rot if rot else 0
    inv = angles(n) if n else None
    kv = to_device(s, tokens_first=ps == 32)
    k0, v0 = kv.k.clone(), kv.v.clone()
    q_dev = q.contiguous().cuda()
    T().paged_append(kv, k_new.cuda(), v_new.cuda(), T().RotaryMap(inv.cuda(), pairs) if n else None, q_dev, q_dev,   # in place
                     norms=T().HeadNorms(*(None if w is None else w.cuda() for w in (wq, wk)), 1e-6))
    assert kv.device_status() == 0
    inv64 = None if inv is None else inv.double().numpy()
    gk, gq, expect_k, expect_v = f64(kv.k), f64(q_dev), k0.clone(), v0.clone()
    for tok, page, slot, t in places(s, ps):
        for got, x, w in ((gk[page, :, slot], k_new[tok], wk), (gq[tok], q[tok], wq)):
            y = expected_heads(x, None if w is None else w.double().numpy(), 1e-6, t, inv64, pairs)
            assert (np.abs(got - y) <= u_of(dtype) * np.abs(y) + 1.1 * slack(d) * np.abs(y).max(-1, keepdims=True) + 2.0 ** -25).all()
        expect_k[page, :, slot] = kv.k[page, :, slot]
        expect_v[page, :, slot] = v_new[tok].cuda()
    bits = lambda t: t.contiguous().view(torch.int16)  # noqa: E731
    assert torch.equal(bits(expect_k), bits(kv.k)) and torch.equal(bits(expect_v), bits(kv.v))
    want = PO.page_bounds(gk, s.table, s.kv_lens)
    for page in {page for _, page, _, _ in places(s, ps)}:
        assert (f64(kv.key_bounds)[page, :, 0] == want[page][0]).all() and (f64(kv.key_bounds)[page, :, 1] == want[page][1]).all()


def test_norms_of_heads_of_zeros_and_of_no_numbers():
    """A zero head stays zero (eps > 0); a head with NaN is NaN and leaves its neighbours alone."""
    d, ps, hq, hkv = 128, 16, 4, 2
    s = make_step8(hq, hkv, d, ps, "bf16", [(3, 3)], seed=2)
    k_new, v_new, q = (x.clone() for x in new_tokens(s, 3, hkv, d, "bf16"))
    q[0, 1] = 0
    q[1, 2, 7] = math.nan
    k_new[2, 0] = 0
    kv, out = to_device8(s), torch.empty_like(q).contiguous().cuda()
    w = torch.ones(d).cuda()
    T().paged_append(kv, k_new.cuda(), v_new.cuda(), None, q.cuda(), out, norms=T().HeadNorms(w, w, 1e-6))
    got = f64(out)
    assert (got[0, 1] == 0).all() and np.isnan(got[1, 2]).all()
    got[1, 2] = 0
    assert np.isfinite(got).all()
    page = int(s.table[0, 0])
    assert (raw(kv.k)[page, 0, 2] & 127 == 0).all() and raw(kv.k_scales)[page, 0, 2] == 1


# ---------------------------------------------------------------------------------------------- read
@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("dtype,ps,head_major", [("bf16", 16, True), ("fp16", 64, False), ("bf16", 128, False), ("fp16", 32, True)])
def test_rows_read_back(dtype, ps, head_major, hq, hkv, d):
    lens = [(0, 5), (1, 130), (0, 0), (2, 64), (0, 333)]
    s = make_step8(hq, hkv, d, ps, dtype, lens, seed=11, spread=3.0)
    first, count = np.array([2, 0, 0, 60, 17]), np.array([3, 130, 0, 1, 300])
    cu = np.concatenate([[0], np.cumsum(count)])
    kv = to_device8(s, tokens_first=ps == 32)
    n = int(cu[-1])
    shape = (hkv, n + 2, d) if head_major else (n + 2, hkv, d)
    outs = [torch.full(shape, 7.0, dtype=DT[dtype], device="cuda") for _ in range(2)]
    views = [(o.transpose(0, 1) if head_major else o)[:n] for o in outs]
    T().paged_read(kv, T().CacheRows(cu, first, device="cuda"), *views)
    assert kv.device_status() == 0
    for view, full, codes, scales in ((views[0], outs[0], s.k, s.ks), (views[1], outs[1], s.v, s.vs)):
        x = P8.values(codes, scales)
        for b in range(len(lens)):
            for i in range(count[b]):
                t = first[b] + i
                want = torch.from_numpy(x[s.table[b, t // ps], :, t % ps]).to(DT[dtype])
                assert torch.equal(view[cu[b] + i].cpu(), want), (b, i)
        tail = full.transpose(0, 1)[n:] if head_major else full[n:]
        assert (tail == 7).all()
    only = torch.zeros_like(views[1]).contiguous()
    T().paged_read(kv, T().CacheRows(cu, first, device="cuda"), None, only)
    assert torch.equal(only, views[1].contiguous())


def test_every_code_and_every_scale_reads_as_what_it_stands_for():
    d, ps = 64, 128
    s = make_step8(1, 1, d, ps, "bf16", [(0, 1024)], seed=0)
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(4, 64), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8), 4)
    for t in range(1024):
        p = s.table[0, t // ps]
        s.k[p, 0, t % ps], s.ks[p, 0, t % ps] = codes[t], scales[t]
    kv = to_device8(s)
    out = torch.empty(1024, 1, d, dtype=torch.bfloat16, device="cuda")
    T().paged_read(kv, T().CacheRows([0, 1024], device="cuda"), out, None)
    # 64 bits to bf16 by way of 32, which hold all of these numbers that bf16 does not round to 0 or to infinity
    want = torch.from_numpy(P8.values(codes, scales)).float().bfloat16()
    assert torch.equal(out[:, 0].cpu().nan_to_num(3.0), want.nan_to_num(3.0)) and torch.equal(out[:, 0].cpu().isnan(), want.isnan())


# ---------------------------------------------------------------------------------------------- attention
def oracle8(s, causal=True, scale=None):
    k, v = s.values()
    return PO.attention(f64(s.q), k, v, s.table, s.kv_lens, s.cu_q, causal, scale)


def compare8(s, causal=True, scale=None, tokens_first=False):
    got = gpu_attention8(s, causal, scale, tokens_first)
    check_attention(s.dtype, s.k.shape[3], *got, *oracle8(s, causal, scale), int(s.kv_lens.max()))


@pytest.mark.parametrize("lens", [[(1, 1)], [(1, 4096)], [(1, 40), (1, 333), (0, 9), (1, 128), (1, 129), (1, 1000)], [(2, 700), (1, 2), (1, 1537)]])
@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("dtype,ps", [("bf16", 16), ("fp16", 64), ("bf16", 128), ("fp16", 32)])
def test_decode_attention8(dtype, ps, hq, hkv, d, lens):
    compare8(make_step8(hq, hkv, d, ps, dtype, lens, seed=12), tokens_first=ps == 32)


@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("dtype,ps,batch", [("bf16", 64, 40), ("fp16", 16, 24)])
def test_a_line_of_ragged_sequences(dtype, ps, batch, hq, hkv, d):
    r = np.random.default_rng(3)
    lens = [(1, int(n)) for n in r.integers(1, 3000, batch)]
    lens[4] = (0, 700)
    lens[5] = (1, 9000)
    compare8(make_step8(hq, hkv, d, ps, dtype, lens, seed=13))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("dtype,ps", [("bf16", 16), ("fp16", 64), ("bf16", 128)])
def test_chunks8(dtype, ps, hq, hkv, d, causal):
    lens = [(17, 17), (1, 50), (130, 500), (65, 65), (0, 10), (33, 1000), (300, 300)]
    compare8(make_step8(hq, hkv, d, ps, dtype, lens, seed=14), causal)


def test_full_context_of_short_and_empty_sequences8():
    lens = [(3, 0), (40, 3), (1, 0), (2, 1), (30, 0)]
    compare8(make_step8(8, 2, 64, 16, "bf16", lens, seed=15), causal=False)


@pytest.mark.parametrize("scale", [0.01, 1.0])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("fp16", 128)])
def test_scales_of_the_softmax8(dtype, d, scale):
    compare8(make_step8(8, 2, d, 32, dtype, [(1, 900), (40, 300)], seed=16), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (6, 2, 128)])
def test_block_attention8(dtype, hq, hkv, d):
    for ps, sink, tail, topk, lens in ((16, 1, 2, 5, [(1, 400), (3, 333), (0, 8), (1, 20)]), (128, 0, 1, 3, [(1, 2000), (2, 129), (1, 128)]),
                                       (64, 2, 1, 0, [(1, 700)]), (32, 1, 1, 40, [(1, 5000), (5, 900)])):
        s = make_step8(hq, hkv, d, ps, dtype, lens, seed=17, with_bounds=True)
        y, lse, idx = gpu_block_attention8(s, sink, tail, topk, tokens_first=ps == 32)
        k, v = s.values()
        wy, wl, A, C, pages = PO.block_attention(f64(s.q), k, v, s.table, s.kv_lens, s.cu_q, f64(s.bounds), sink, tail, topk)
        assert (idx == pages).all()
        check_attention(dtype, d, y, lse, wy, wl, A, C, (sink + tail + topk) * ps)
