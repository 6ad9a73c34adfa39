"""Shared helpers of the 8-bit cache's tests: random steps, the library's calls on them."""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

from oracle import paged8_oracle as P8
from paged_utils import DT, f64

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


@dataclass
class Step8:
    """An 8-bit paged cache and one step's inputs on the host; every slot without a row holds NaN codes and the NaN scale."""
    k: np.ndarray              # codes [n_pages, hkv, ps, d]
    v: np.ndarray
    ks: np.ndarray             # scale bytes [n_pages, hkv, ps]
    vs: np.ndarray
    table: np.ndarray
    kv_lens: np.ndarray
    cu_q: np.ndarray
    hq: int
    dtype: str
    q: torch.Tensor
    bounds: Optional[torch.Tensor] = None

    @property
    def total_q(self) -> int:
        return int(self.cu_q[-1])

    def values(self):
        """What the cache stands for, in 64 bits (NaN where there is no row)."""
        return P8.values(self.k, self.ks), P8.values(self.v, self.vs)


def bounds_of(s: Step8) -> torch.Tensor:
    k, ps = P8.values(s.k, s.ks), s.k.shape[2]
    out = torch.zeros(k.shape[0], k.shape[1], 2, k.shape[3], dtype=DT[s.dtype])
    for b, n in enumerate(s.kv_lens):
        for p in range((n + ps - 1) // ps):
            have = k[s.table[b, p], :, :min(ps, n - p * ps)]
            out[s.table[b, p], :, 0] = torch.from_numpy(have.min(1)).to(DT[s.dtype])
            out[s.table[b, p], :, 1] = torch.from_numpy(have.max(1)).to(DT[s.dtype])
    return out


def make_step8(hq, hkv, d, ps, dtype, lens, seed=0, spare=2, with_bounds=False, key_scale=1.0, spread=1.0) -> Step8:
    """lens: (q_len, kv_len) of each sequence.  Rows' sizes differ by powers of two of standard deviation `spread`."""
    g = np.random.default_rng(seed)
    n_seq = [(n + ps - 1) // ps for _, n in lens]
    n_pages = sum(n_seq) + spare
    shape = (n_pages, hkv, ps, d)
    codes, scales = [], []
    for size in (key_scale, 1.0):
        x = size * g.standard_normal(shape) * np.exp2(np.round(spread * g.standard_normal(shape[:3])))[..., None]
        e = np.frexp(np.abs(x).max(-1))[1] - 9 + 127 + 1          # (a power that fits; now and then not the smallest)
        codes.append(torch.from_numpy(x / P8.power(e)[..., None]).to(F8).view(torch.uint8).numpy())
        scales.append(e.astype(np.uint8))
    k, v, ks, vs = codes[0], codes[1], scales[0], scales[1]
    order = g.permutation(n_pages).tolist()
    table = np.full((len(lens), max(max(n_seq), 1)), -1, np.int32)
    empty = np.ones(shape[:3], bool)
    for b, (_, n) in enumerate(lens):
        for p in range(n_seq[b]):
            table[b, p] = order.pop()
            empty[table[b, p], :, :min(ps, n - p * ps)] = False
    for c, e in ((k, ks), (v, vs)):
        c[empty] = 0x7f
        e[empty] = 255
    cu_q = np.concatenate([[0], np.cumsum([m for m, _ in lens])]).astype(np.int64)
    q = torch.from_numpy(g.standard_normal((int(cu_q[-1]), hq, d))).to(DT[dtype])
    s = Step8(k, v, ks, vs, table, np.array([n for _, n in lens], np.int64), cu_q, hq, dtype, q)
    if with_bounds:
        s.bounds = bounds_of(s)
    return s


def device_cache(s: Step8, tokens_first=False, dev="cuda:0"):
    """(k, v, k_scales, v_scales) on the device; storage [page][head][slot] or [page][slot][head]."""
    k, v = (torch.from_numpy(x.copy()).to(dev).view(F8) for x in (s.k, s.v))
    if tokens_first:
        k, v = (x.view(torch.uint8).transpose(1, 2).contiguous().view(F8).transpose(1, 2) for x in (k, v))
    return k, v, *(torch.from_numpy(x.copy()).to(dev).view(E8) for x in (s.ks, s.vs))


def to_device8(s: Step8, tokens_first=False, bounds=None, dev="cuda:0"):
    import paper_2604_05438_b200 as T
    b = s.bounds if bounds is None else bounds
    return T.PagedKVCache8(*device_cache(s, tokens_first, dev), torch.from_numpy(s.table).to(dev), s.kv_lens, s.cu_q, s.hq,
                           DT[s.dtype], None if b is None else b.to(dev))


def gpu_attention8(s: Step8, causal=True, scale=None, tokens_first=False, kv=None):
    import paper_2604_05438_b200 as T
    kv = to_device8(s, tokens_first) if kv is None else kv
    q = s.q.to(kv.k.device)
    y = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), device=q.device)
    ws = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_ATTENTION), dtype=torch.uint8, device=q.device).fill_(0xFF)
    T.paged_attention(kv, q, y, lse, scale, T.FLAG_NONE if causal else T.FLAG_FULL_CONTEXT, ws)
    torch.cuda.synchronize()
    assert kv.device_status() == 0
    return f64(y), f64(lse)


def gpu_block_attention8(s: Step8, sink, tail, topk, scale=None, tokens_first=False):
    import paper_2604_05438_b200 as T
    kv = to_device8(s, tokens_first)
    sel = T.PageSelection(sink, tail, topk)
    q = s.q.to(kv.k.device)
    y = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), device=q.device)
    idx = torch.full((s.total_q, s.k.shape[1], sel.n_pages), -7, dtype=torch.int32, device=q.device)
    ws = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_BLOCK_ATTENTION, sel), dtype=torch.uint8, device=q.device).fill_(0xFF)
    T.paged_block_attention(kv, sel, q, y, lse, idx, scale, ws)
    torch.cuda.synchronize()
    assert kv.device_status() == 0
    return f64(y), f64(lse), idx.cpu().numpy()
