"""Shared helpers of the paged-cache tests: random steps, the library's calls on them, comparisons."""
from __future__ import annotations

import math
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

from oracle import paged_oracle as PO

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@dataclass
class Step:
    """A paged cache and one step's inputs on the host; every slot without a row holds NaN."""
    k: torch.Tensor            # [n_pages, hkv, ps, d]
    v: torch.Tensor
    table: np.ndarray
    kv_lens: np.ndarray
    cu_q: np.ndarray
    hq: int
    q: torch.Tensor
    bounds: Optional[torch.Tensor] = None

    @property
    def total_q(self) -> int:
        return int(self.cu_q[-1])


def make_step(hq, hkv, d, ps, dtype, lens, seed=0, spare=2, with_bounds=False, key_scale=1.0) -> Step:
    """lens: (q_len, kv_len) of each sequence.  Pages are dealt out in random order; table entries behind a sequence's
    last page are -1."""
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    n_seq = [(n + ps - 1) // ps for _, n in lens]
    n_pages = sum(n_seq) + spare
    k = torch.full((n_pages, hkv, ps, d), float("nan"), dtype=dt)
    v = torch.full_like(k, float("nan"))
    order = torch.randperm(n_pages, generator=g).tolist()
    table = np.full((len(lens), max(max(n_seq), 1)), -1, np.int32)
    for b, (_, n) in enumerate(lens):
        for p in range(n_seq[b]):
            page = order.pop()
            table[b, p] = page
            m = min(ps, n - p * ps)
            k[page, :, :m] = (key_scale * torch.randn(hkv, m, d, generator=g)).to(dt)
            v[page, :, :m] = torch.randn(hkv, m, d, generator=g).to(dt)
    cu_q = np.concatenate([[0], np.cumsum([m for m, _ in lens])]).astype(np.int64)
    q = torch.randn(int(cu_q[-1]), hq, d, generator=g).to(dt)
    s = Step(k, v, table, np.array([n for _, n in lens], np.int64), cu_q, hq, q)
    if with_bounds:
        s.bounds = torch.full((n_pages, hkv, 2, d), float("nan"), dtype=dt)
        for page, (lo, hi) in PO.page_bounds(f64(k), table, s.kv_lens).items():
            s.bounds[page, :, 0], s.bounds[page, :, 1] = torch.from_numpy(lo).to(dt), torch.from_numpy(hi).to(dt)
    return s


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().double().numpy()


def to_device(s: Step, tokens_first=False, bounds=None, dev="cuda:0"):
    """The binding's descriptor over a copy of the step's cache; storage [page][head][slot] or [page][slot][head]."""
    import paper_2604_05438_b200 as T
    k, v = s.k.to(dev), s.v.to(dev)
    if tokens_first:
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    b = s.bounds if bounds is None else bounds
    return T.PagedKVCache(k, v, torch.from_numpy(s.table).to(dev), s.kv_lens, s.cu_q, s.hq, None if b is None else b.to(dev))


def gpu_attention(s: Step, causal=True, scale=None, tokens_first=False, kv=None):
    import paper_2604_05438_b200 as T
    kv = to_device(s, tokens_first) if kv is None else kv
    q = s.q.to(kv.k.device)
    y = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), device=q.device)
    ws = torch.empty(T.paged_workspace_bytes(kv, T.WS_PAGED_ATTENTION), dtype=torch.uint8, device=q.device).fill_(0xFF)
    T.paged_attention(kv, q, y, lse, scale, T.FLAG_NONE if causal else T.FLAG_FULL_CONTEXT, ws)
    torch.cuda.synchronize()
    assert kv.device_status() == 0
    return f64(y), f64(lse)


def gpu_block_attention(s: Step, sink, tail, topk, scale=None, tokens_first=False, kv=None):
    import paper_2604_05438_b200 as T
    kv = to_device(s, tokens_first) if kv is None else kv
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


def check_attention(dtype, d, got_y, got_lse, y, lse, A, C, n_keys):
    """Error bounds from arithmetic, with u = eps / 2 of the 16-bit type:
      - a score's error is at most d 2^-22 C (an fp32 sum of d exact products, each addition off by 2^-23 of the running
        sum at worst, tensor-core truncation included; doubled for the scaling and the exponent's argument), exp2 adds
        2^-21, and both multiply a probability;
      - a probability enters the second product rounded to 16 bits: u, relative;
      - a sum of n fp32 terms is off by n 2^-24, relative to the sum of magnitudes (A per value dim);
      - the output is rounded once more: u |y| (fp16 below its normal range: 2^-25 absolute)."""
    u = torch.finfo(DT[dtype]).eps / 2
    e = (d * 2.0 ** -22 * C + 2.0 ** -21)[..., None]
    n = n_keys * 2.0 ** -24
    tol = u * np.abs(y) + (u + 2 * e + 2 * n) * A + 2.0 ** -24
    bad = np.abs(got_y - y) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float((np.abs(got_y - y) / tol).max()))
    none = ~np.isfinite(lse)
    assert (got_lse[none] == -math.inf).all()
    if not none.all():
        import parity_utils as PU
        tol_l = e[..., 0][~none] + n + np.abs(lse[~none]) * 2.0 ** -22 + 2.0 ** -20
        err_l = np.abs(got_lse[~none] - lse[~none])
        assert (err_l <= tol_l).all(), float((err_l / tol_l).max())
        PU.note("paged_y_err_over_tol", float((np.abs(got_y - y) / tol).max()))
        PU.note("paged_lse_err_over_tol", float((err_l / tol_l).max()))
