"""GPU tests of the calls over an 8-bit cache, and of the head norms, with numbers far apart or near the ends of their range,
against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import paged8_oracle as P8
from oracle import paged_oracle as PO
from paged8_utils import F8, gpu_attention8, gpu_block_attention8, make_step8
from paged_utils import DT, check_attention, f64

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
