"""GPU tests of the calls over an 8-bit cache, and of the head norms, with numbers far apart or near the ends of their range,
against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import paged8_oracle as P8
from oracle import paged_oracle as PO
from paged8_utils import F8, gpu_attention8, gpu_block_attention8, make_step8, to_device8
from paged_utils import DT, check_attention, f64, make_step, to_device

pytestmark = pytest.mark.gpu

# few rows (one row tile of 8, of 16, several), many rows
WAYS = {"one": (1, 4), "tile": (4, 4), "tiles": (9, 4), "many": (40, 4)}       # way: (q_len, group)
FEW = ["one", "tile", "tiles"]


def T():
    import paper_2604_05438_b200
    return paper_2604_05438_b200


def oracle8(s):
    return PO.attention(f64(s.q), *s.values(), s.table, s.kv_lens, s.cu_q)


def at(s, b, t):
    """Index of position t of sequence b in the cache's arrays, all heads."""
    ps = s.k.shape[2]
    return s.table[b, t // ps], slice(None), t % ps


def code(x):
    return int(torch.tensor(float(x)).to(F8).view(torch.uint8))


def attended(s, d):
    """compare with the oracle by check_attention's bound, after a look that this bound would not let zeros pass."""
    y, lse = gpu_attention8(s)
    wy, wl, A, C = oracle8(s)
    u = torch.finfo(DT[s.dtype]).eps / 2
    assert (np.abs(wy) > u * np.abs(wy) + (u + 2 * (d * 2.0 ** -22 * C[..., None] + 2.0 ** -21) + 2 * s.kv_lens.max() * 2.0 ** -24) * A + 2.0 ** -24).mean() > 0.5
    check_attention(s.dtype, d, y, lse, wy, wl, A, C, int(s.kv_lens.max()))
    return y, lse


# ---------------------------------------------------------------------------------------------- values far apart
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("power", [8, 12, 20, 30, 40, 100])
def test_a_large_value_whose_key_gets_nothing(power, way):
    """One key's score is 224 below the others', its values 2^power times theirs: e^-224 = 2^-323 of them reaches no output."""
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 64, "bf16", [(q_len, 300)], seed=70, spread=0.0)
    s.q = torch.ones_like(s.q)
    s.k[at(s, 0, 100)], s.ks[at(s, 0, 100)] = code(-28), 127
    s.vs[at(s, 0, 100)] += power
    attended(s, 64)


@pytest.mark.parametrize("way", FEW)
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("fp16", 128)])
def test_one_key_takes_all_and_its_values_are_small(dtype, d, first, way):
    """The key with all the probability has values 2^-45 of everybody's else's, whose probabilities are e^-72 and less: the
    products of probability and value are largest at that key all the same."""
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, d, 32, dtype, [(q_len, 400), (1, 3)], seed=71, spread=0.0)
    s.q = torch.full_like(s.q, 9 * d ** -0.5)                    # scores of 9 times a key's elements
    best = 3 if first else 390 - q_len
    for t in range(400):
        s.k[at(s, 0, t)], s.ks[at(s, 0, t)] = code(4 if t == best else -4), 127
    s.vs[at(s, 0, best)] -= 4
    for t in range(400):
        if t != best:
            s.vs[at(s, 0, t)] += 41
    attended(s, d)


def falling_products(s, order, top, seed):
    """Keys of scores 0 .. -56 below the best, in the given order, with values that make up for it: all products count."""
    r = np.random.default_rng(seed)
    n = int(s.kv_lens[0])
    below = np.linspace(0, 7, n)
    below = np.where(below < 4, np.round(below * 4) / 4, np.round(below * 2) / 2)             # e4m3 numbers
    if order == "rising":
        below = below[::-1]
    elif order == "mixed":
        below = r.permutation(below)
    s.q = torch.ones_like(s.q)
    for t in range(n):
        s.k[at(s, 0, t)], s.ks[at(s, 0, t)] = code(-below[t]), 127
        gain = int(np.round(8 * below[t] / np.log(2))) + r.integers(-3, 4)
        s.vs[at(s, 0, t)] = np.clip(s.vs[at(s, 0, t)].astype(int) + top + gain, 1, 254)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("order", ["falling", "rising", "mixed"])
def test_values_that_make_up_for_small_probabilities(order, way):
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 32, "bf16", [(q_len, 900), (q_len, 70)], seed=72, spread=0.0)
    falling_products(s, order, 0, 5)
    attended(s, 64)


@pytest.mark.parametrize("hq", [4, 16])
@pytest.mark.parametrize("order", ["falling", "rising", "mixed"])
def test_values_that_make_up_for_small_probabilities_on_selected_pages(order, hq):
    s = make_step8(hq, 1, 64, 64, "fp16", [(1, 400)] + [(1, 70)] * 3, seed=73, spread=0.0, with_bounds=True)
    falling_products(s, order, -85, 6)
    y, lse, idx = gpu_block_attention8(s, 1, 2, 9)               # (every page)
    wy, wl, A, C = oracle8(s)
    assert (idx[0, 0, :7] == np.arange(7)).all()
    check_attention("fp16", 64, y[:1], lse[:1], wy[:1], wl[:1], A[:1], C[:1], 400)


@pytest.mark.parametrize("lens", [[(1, 5000)], [(1, 3000 + 64 * i) for i in range(40)]])        # a cluster, a line
def test_values_far_apart_in_pieces_of_long_sequences(lens):
    s = make_step8(8, 2, 64, 64, "bf16", lens, seed=74, spread=0.0)
    falling_products(s, "mixed", 0, 7)
    y, lse = gpu_attention8(s)
    one = make_step8(8, 2, 64, 64, "bf16", lens, seed=74, spread=0.0)
    one.q, one.k, one.ks, one.v, one.vs = s.q[:1], s.k, s.ks, s.v, s.vs
    one.kv_lens, one.cu_q, one.table = s.kv_lens[:1], s.cu_q[:2], s.table[:1]
    wy, wl, A, C = oracle8(one)
    check_attention("bf16", 64, y[:1], lse[:1], wy, wl, A, C, int(s.kv_lens[0]))


@pytest.mark.parametrize("way", ["tile", "tiles", "many"])
@pytest.mark.parametrize("power", [9, 28, 40, 100])
@pytest.mark.parametrize("kv_len", [40, 300])
def test_a_later_tokens_values_do_not_reach_the_tokens_before_it(kv_len, power, way):
    q_len, g = WAYS[way]
    s = make_step8(2 * g, 2, 64, 32, "bf16", [(q_len, kv_len), (1, 20)], seed=75, spread=2.0)
    clean = gpu_attention8(s)
    s.vs[at(s, 0, kv_len - 1)] += power
    y, lse = gpu_attention8(s)
    assert (y[:q_len - 1] == clean[0][:q_len - 1]).all() and (lse == clean[1]).all()
    assert (y[q_len:] == clean[0][q_len:]).all()
    check_attention("bf16", 64, y, lse, *oracle8(s), kv_len)


# ---------------------------------------------------------------------------------------------- head norms
# a norm's error relative to the head's largest element: the sum of squares d/2 2^-24, the root 2^-22, four products
def norm_slack(d):
    return (d / 2 + 4 + 4) * 2.0 ** -24


@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-30, 1e-6])
@pytest.mark.parametrize("d,held", [(64, True), (128, False)])
def test_norms_of_heads_of_any_size(d, held, eps):
    """bf16 heads of 2^-130 to 2^120, some elements far below the others; eps 0, below and above their squares."""
    powers = [-130, -126, -120, -100, -76, -75, -64, -63, -50, -40, -30, -10, 0, 40, 60, 62, 63, 64, 90, 120]
    hq, hkv, ps, n = 4, 2, 16, len(powers)
    g = torch.Generator().manual_seed(90)
    x = torch.randn(n, hq + 2 * hkv, d, generator=g, dtype=torch.float64)
    x[:, :, ::7] *= 2.0 ** -20
    x = (x * torch.exp2(torch.tensor(powers, dtype=torch.float64))[:, None, None]).to(torch.bfloat16)
    k_new, v_new, q = x[:, hq:hq + hkv], x[:, hq + hkv:], x[:, :hq]
    w = 1 + 0.3 * torch.randn(d, generator=g)
    if held:
        s = make_step8(hq, hkv, d, ps, "bf16", [(n, n)], seed=91)
        kv = to_device8(s)
    else:
        s = make_step(hq, hkv, d, ps, "bf16", [(n, n)], seed=91)
        kv = to_device(s)
    out = torch.full((n, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    T().paged_append(kv, k_new.cuda(), v_new.cuda(), None, q.cuda(), out, norms=T().HeadNorms(w.cuda(), w.cuda(), eps))
    assert kv.device_status() == 0
    eps32 = float(np.float32(eps))
    qy, ky = (P8.norm(t.double().numpy(), w.double().numpy(), eps32) for t in (q, k_new))
    u, tiny = torch.finfo(torch.bfloat16).eps / 2, 2.0 ** -134      # half a step of bf16 (8 bits: 2^-8), half of its smallest number
    most = np.abs(qy).max(-1, keepdims=True)
    assert (np.abs(f64(out) - qy) <= u * np.abs(qy) + norm_slack(d) * most + tiny).all()
    for t in range(n):
        page, slot = s.table[0, t // ps], t % ps
        most = np.abs(ky[t]).max(-1, keepdims=True)
        if held:
            c, e = kv.k.view(torch.uint8).cpu().numpy()[page, :, slot], kv.k_scales.view(torch.uint8).cpu().numpy()[page, :, slot]
            got, tol = P8.values(c, e), 2.0 ** -4 * np.abs(ky[t]) + 2.0 ** -10 * P8.power(e)[:, None]
        else:
            got, tol = f64(kv.k)[page, :, slot], u * np.abs(ky[t])
        assert (np.abs(got - ky[t]) <= tol + 1.1 * norm_slack(d) * most + tiny).all(), powers[t]


def test_norms_of_heads_without_a_size():
    """eps 0: a head of zeros is 0 / 0, as is an infinite element; the others of that head are 0.  Neighbours are as ever."""
    d, ps = 64, 16
    s = make_step(2, 1, d, ps, "bf16", [(3, 3)], seed=92)
    q = torch.ones(3, 2, d)
    q[0, 0] = 0
    q[1, 1, 3] = float("inf")
    q[2, 0, 5] = float("nan")
    q, out = q.bfloat16().cuda(), torch.empty(3, 2, d, dtype=torch.bfloat16, device="cuda")
    kv, w = to_device(s), torch.ones(d).cuda()
    T().paged_append(kv, torch.ones(3, 1, d).bfloat16().cuda(), torch.ones(3, 1, d).bfloat16().cuda(), None, q, out, norms=T().HeadNorms(w, None, 0.0))
    got = f64(out)
    want = np.ones((3, 2, d))
    want[0, 0], want[2, 0], want[1, 1], want[1, 1, 3] = np.nan, np.nan, 0, np.nan
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("held,ps,d,pairs", [(True, 16, 128, False), (True, 128, 64, True), (False, 32, 64, False), (False, 128, 128, True)])
def test_heads_of_any_size_beside_others(held, ps, d, pairs):
    """Some heads of some tokens are very small or large: rotated, queries in place, weights of each head, bounds of pages that hold
    rows of earlier calls, a group of more than four heads."""
    hq, hkv, lens = 12, 2, [(5, 90), (1, 33), (150, 200), (0, 4)]
    if held:
        s = make_step8(hq, hkv, d, ps, "bf16", lens, seed=99, with_bounds=True)
        kv = to_device8(s)
    else:
        s = make_step(hq, hkv, d, ps, "bf16", lens, seed=99, with_bounds=True)
        kv = to_device(s)
    n = s.total_q
    g = torch.Generator().manual_seed(100)
    x = torch.randn(n, hq + 2 * hkv, d, generator=g, dtype=torch.float64)
    power = torch.tensor([0, -100, 0, 0, 80, 0, -70, 0], dtype=torch.float64)[torch.randint(0, 8, (n, hq + 2 * hkv), generator=g)]
    power[:, hq + hkv:] = 0                                  # values are not normed
    x = (x * torch.exp2(power)[..., None]).bfloat16()
    k_new, v_new, q = x[:, hq:hq + hkv], x[:, hq + hkv:], x[:, :hq].contiguous()
    wq, wk = (1 + 0.3 * torch.randn(m, d, generator=g) for m in (hq, hkv))
    inv = 0.5 ** torch.arange(d // 4, dtype=torch.float32)
    q_dev = q.cuda()
    T().paged_append(kv, k_new.cuda(), v_new.cuda(), T().RotaryMap(inv.cuda(), pairs), q_dev, q_dev, norms=T().HeadNorms(wq.cuda(), wk.cuda(), 0.0))
    assert kv.device_status() == 0
    u, slack = torch.finfo(torch.bfloat16).eps / 2, norm_slack(d) + 16 * 2.0 ** -24        # (sine and cosine: 2^-22 each, their angle 2^-22)
    got_k = P8.values(kv.k.view(torch.uint8).cpu().numpy(), kv.k_scales.view(torch.uint8).cpu().numpy()) if held else f64(kv.k)
    for b, (m, length) in enumerate(lens):
        for i in range(m):
            tok, t = int(s.cu_q[b]) + i, length - m + i
            y = PO.rotate(P8.norm(q[tok].double().numpy(), wq.double().numpy(), 0.0), t, inv.double().numpy(), pairs)
            assert (np.abs(f64(q_dev)[tok] - y) <= u * np.abs(y) + 1.1 * slack * np.abs(y).max(-1, keepdims=True)).all()
            y = PO.rotate(P8.norm(k_new[tok].double().numpy(), wk.double().numpy(), 0.0), t, inv.double().numpy(), pairs)
            got = got_k[s.table[b, t // ps], :, t % ps]
            tol = 2.0 ** -4 * np.abs(y) + 2.0 ** -10 * P8.power(P8.scale_byte(got))[:, None] if held else u * np.abs(y)
            assert (np.abs(got - y) <= tol + 1.1 * slack * np.abs(y).max(-1, keepdims=True)).all()
    want = PO.page_bounds(got_k, s.table, s.kv_lens)
    for b, (m, length) in enumerate(lens):
        for p in range((length - m) // ps, (length + ps - 1) // ps if m else 0):
            page = int(s.table[b, p])
            lo, hi = (torch.from_numpy(w).bfloat16().double().numpy() for w in want[page])
            assert (f64(kv.key_bounds)[page, :, 0] == lo).all() and (f64(kv.key_bounds)[page, :, 1] == hi).all()


# ---------------------------------------------------------------------------------------------- fp16 near the end of its range
def big_rows(s, hkv, d, seed):
    """New tokens with elements up to the largest fp16 number; those from 63488 on are held as 65536."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(s.total_q, hkv, d, generator=g)
    for t in range(s.total_q):
        x[t, :, (3 * t) % d] = [65504, -65504, 63488, -63520, 60000, 65504][t % 6]
    return x.half()


@pytest.mark.parametrize("d", [64, 128])
def test_fp16_rows_at_the_end_of_the_range_stay_finite(d):
    hkv, ps, n = 2, 16, 70
    s = make_step8(4, hkv, d, ps, "fp16", [(n, n)], seed=95, with_bounds=True)
    x = big_rows(s, hkv, d, 96)
    kv = to_device8(s)
    T().paged_append(kv, x.cuda(), x.flip(0).contiguous().cuda())
    out = [torch.empty(n, hkv, d, dtype=torch.float16, device="cuda") for _ in range(2)]
    T().paged_read(kv, T().CacheRows([0, n], device="cuda"), *out)
    assert kv.device_status() == 0
    for got, rows in ((f64(out[0]), f64(x)), (f64(out[1]), f64(x.flip(0)))):
        held = P8.hold(rows)[0]
        assert np.abs(held).max() == 65536                   # (it is what this test is about)
        # (2^-14: the smallest normal number; elements beside one of 65504 are held to 2^-10 * 2^8)
        want = np.clip(held, -65504, 65504)
        assert (got == want).all()
        assert (np.abs(got - rows) <= 2.0 ** -4 * np.abs(rows) + 2.0 ** -2).all()
    for p in range((n + ps - 1) // ps):
        have = f64(out[0])[p * ps:(p + 1) * ps]
        b = f64(kv.key_bounds)[s.table[0, p]]
        assert (b[:, 0] == have.min(0)).all() and (b[:, 1] == have.max(0)).all()


def test_fp16_rows_beyond_the_range_read_as_its_ends():
    """Every scale byte from that of 65504 on; NaN codes and byte 255 stay NaN."""
    d, ps = 64, 128
    s = make_step8(1, 1, d, ps, "fp16", [(0, 1024)], seed=97)
    codes = np.tile(np.arange(256, dtype=np.uint8).reshape(4, 64), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8), 4)
    for t in range(1024):
        p = s.table[0, t // ps]
        s.v[p, 0, t % ps], s.vs[p, 0, t % ps] = codes[t], scales[t]
    out = torch.empty(1024, 1, d, dtype=torch.float16, device="cuda")
    T().paged_read(to_device8(s), T().CacheRows([0, 1024], device="cuda"), None, out)
    x = P8.values(codes, scales)
    want = torch.from_numpy(np.clip(x, -65504, 65504)).half()
    assert np.array_equal(f64(out[:, 0]), f64(want), equal_nan=True)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("side", ["values", "keys"])
def test_attention_over_fp16_rows_at_the_end_of_the_range(side, way):
    """Values held as 65536 count as that or as 65504, 2^-11 less; so do keys, here in a dim in which the queries are 0.  Outputs
    are finite."""
    q_len, g = WAYS[way]
    n = 200
    s = make_step8(2 * g, 2, 64, 32, "fp16", [(q_len, n), (1, 40)], seed=98, spread=0.0)
    codes, scales = (s.v, s.vs) if side == "values" else (s.k, s.ks)
    if side == "values":
        for t in range(n):                                   # all of them: the output is 65504 or what lies near
            codes[at(s, 0, t)], scales[at(s, 0, t)] = code(256), 127 + 8
            s.v[s.table[0, t // 32], :, t % 32, ::2] = code(-256)
    else:
        s.q[:, :, 5] = 0
        for t in range(0, n, 3):
            codes[at(s, 0, t)], scales[at(s, 0, t)] = 0, 127 + 8
            s.k[s.table[0, t // 32], :, t % 32, 5] = code(256)
    y, lse = gpu_attention8(s)
    wy, wl, A, C = oracle8(s)
    assert np.isfinite(y).all() and np.isfinite(lse).all()
    u = 2.0 ** -11
    C = C if side == "values" else np.minimum(C, 40.0)       # (products with 0 are exact)
    e = (64 * 2.0 ** -22 * C + 2.0 ** -21)[..., None]
    assert (np.abs(y - np.clip(wy, -65504, 65504)) <= u * np.abs(wy) + (2 * u + 2 * e + 2 * n * 2.0 ** -24) * A + 2.0 ** -24).all()
    assert np.abs(lse - wl).max() <= e.max() + n * 2.0 ** -24 + 2.0 ** -18
    assert (np.abs(y[:q_len]) >= 65000).all() or side == "keys"


# ---------------------------------------------------------------------------------------------- angles
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("held,norm", [(True, False), (True, True), (False, True)])
def test_frequencies_that_are_no_numbers(held, norm, pairs):
    """Pairs with an infinite or NaN frequency become NaN, as in the append without norms, and a row of an 8-bit cache with them."""
    hq, hkv, d, ps, n = 4, 2, 64, 16, 5
    g = torch.Generator().manual_seed(93)
    x = torch.randn(n, hq + 2 * hkv, d, generator=g).bfloat16()
    k_new, v_new, q = x[:, hq:hq + hkv], x[:, hq + hkv:], x[:, :hq]
    inv = 0.5 ** torch.arange(16, dtype=torch.float32)
    bad = [2, 7, 15]
    for i, b in zip(bad, (float("inf"), float("nan"), -float("inf"))):
        inv[i] = b
    if held:
        s = make_step8(hq, hkv, d, ps, "bf16", [(n, n)], seed=94)
        kv = to_device8(s)
    else:
        s = make_step(hq, hkv, d, ps, "bf16", [(n, n)], seed=94)
        kv = to_device(s)
    out = torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(d).cuda()
    T().paged_append(kv, k_new.cuda(), v_new.cuda(), T().RotaryMap(inv.cuda(), pairs), q.cuda(), out, norms=T().HeadNorms(w, w, 1e-6) if norm else None)
    assert kv.device_status() == 0
    none = np.zeros(d, bool)
    for i in bad:
        none[[2 * i, 2 * i + 1] if pairs else [i, i + 16]] = True
    assert np.array_equal(np.isnan(f64(out)), np.broadcast_to(none, (n, hq, d)))
    page = int(s.table[0, 0])
    if held:
        assert (kv.k_scales.view(torch.uint8).cpu().numpy()[page, :, :n] == 255).all()
    else:
        assert np.array_equal(np.isnan(f64(kv.k)[page, :, :n]), np.broadcast_to(none, (hkv, n, d)))
    clean = inv.double().numpy()
    clean[bad] = 0
    for t in range(n):
        y = PO.rotate(P8.norm(q[t].double().numpy(), np.ones(d) if norm else None, 1e-6), t, clean, pairs)
        assert (np.abs(f64(out)[t] - y)[:, ~none] <= 2.0 ** -8 * np.abs(y)[:, ~none] + 2.0 ** -14).all()
