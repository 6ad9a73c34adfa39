"""Host-side behaviour of the paged calls: argument validation, workspace sizing, refusals of the binding.  No kernel is
launched; runs without a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2604_05438_b200 as T
from paper_2604_05438_b200 import binding as B
from paper_2604_05438_b200.build import build_library


@pytest.fixture(scope="module")
def lib():
    build_library()
    return T.load_library()


class Desc:
    """A descriptor over made-up device addresses; host arrays are kept alive beside it."""

    def __init__(self, lens=((1, 100), (3, 64)), hq=8, hkv=2, d=64, dtype=0, ps=16, n_pages=64, max_pages=32, k=0x1000,
                 v=0x2000, strides=None, table=0x3000, kv_dev=0x4000, cu_dev=0x5000, bounds=0x6000, status=0x7000,
                 cu=None, kv=None):
        self.kv = np.array([n for _, n in lens] if kv is None else kv, np.int64)
        self.cu = np.concatenate([[0], np.cumsum([m for m, _ in lens])]).astype(np.int64) if cu is None else np.array(cu, np.int64)
        sp, sh, st = strides or (hkv * ps * d, ps * d, d)
        self.c = B._PagedDesc(len(self.kv), hq, hkv, d, dtype, ps, n_pages, max_pages, k, v, sp, sh, st, table,
                              self.kv.ctypes.data, kv_dev, self.cu.ctypes.data, cu_dev, bounds, status)

    @property
    def ref(self):
        return C.byref(self.c)


def _attend(lib, d, q=0x10000, y=0x20000, lse=0x30000, scale=0.0, flags=0, ws=0x100000, ws_bytes=1 << 40):
    return lib.tkphi_paged_attention(d.ref, q, y, lse, scale, flags, ws, ws_bytes, None)


def _block(lib, d, sel=(1, 1, 4), q=0x10000, y=0x20000, lse=0x30000, idx=0x40000, scale=0.0, ws=0x100000, ws_bytes=1 << 40):
    s = B._PageSelection(*sel)
    return lib.tkphi_paged_block_attention(d.ref, C.byref(s), q, y, lse, idx, scale, ws, ws_bytes, None)


def _append(lib, d, **kw):
    a = dict(k_new=0x10000, k_stride_token=128, k_stride_head=64, v_new=0x20000, v_stride_token=128, v_stride_head=64, q=0x30000,
             q_stride_token=512, q_stride_head=64, q_out=0x40000, o_stride_token=512, o_stride_head=64, inv_freq=0x50000,
             rot_dim=64, pairs=0, positions=None)
    a.update(kw)
    s = B._AppendDesc(**a)
    return lib.tkphi_paged_append(d.ref, C.byref(s), None)


ALL = (_attend, _block, _append)


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("bad,status", [
    (dict(d=96), -2), (dict(d=32), -2), (dict(dtype=2), -2), (dict(hq=7), -1), (dict(hkv=0), -1), (dict(hq=34, hkv=2), -2),
    (dict(ps=8), -2), (dict(ps=48), -2), (dict(ps=256), -2), (dict(n_pages=0), -1), (dict(max_pages=0), -1),
    (dict(k=0), -1), (dict(v=0x2008), -1), (dict(table=0), -1), (dict(kv_dev=0), -1), (dict(cu_dev=0), -1), (dict(status=0), -1),
    (dict(strides=(2048, 1024, 60)), -1), (dict(strides=(2048, 1024, 56)), -1), (dict(strides=(2048, 1024, -64)), -1),
    (dict(strides=(2048, 960, 64)), -1), (dict(strides=(2000, 1024, 64)), -1), (dict(strides=(0, 1024, 64)), -1),
    (dict(table=0x3002), -1), (dict(kv_dev=0x4004), -1), (dict(cu_dev=0x5004), -1), (dict(status=0x7001), -1),
    (dict(bounds=0x6008), -1), (dict(cu=[0, 2, 1]), -1), (dict(cu=[1, 2, 3]), -1), (dict(kv=[-1, 64]), -1),
    (dict(kv=[100, 513]), -1), (dict(kv=[100, 2]), -1), (dict(kv=[1 << 40, 64]), -1), (dict(cu=[0, 1 << 40, 1 << 41]), -1),
])
def test_bad_descriptors_are_refused(lib, call, bad, status):
    assert call(lib, Desc(**bad)) == status, lib.tkphi_last_error()
    assert lib.tkphi_last_error()


def test_batch_limits(lib):
    assert _attend(lib, Desc(lens=((1, 5),) * 1025)) == -1 and b"batch" in lib.tkphi_last_error()
    d = Desc()
    d.c.batch = 0
    assert _attend(lib, d) == -1
    assert lib.tkphi_paged_attention(None, 1, 1, 1, 0.0, 0, 1, 1, None) == -1


def test_bad_arguments_of_the_attention_calls(lib):
    d = Desc()
    for call in (_attend, _block):
        assert call(lib, d, q=0) == -1
        assert call(lib, d, q=0x10008) == -1
        assert call(lib, d, y=0) == -1
        assert call(lib, d, lse=0x30002) == -1
        for scale in (-1.0, float("nan"), float("inf")):
            assert call(lib, d, scale=scale) == -1
        assert call(lib, d, ws=0) == -3
        assert call(lib, d, ws=0x100010) == -3
    assert _attend(lib, d, flags=1) == -1 and b"flag" in lib.tkphi_last_error()
    assert _attend(lib, d, flags=4) == -1
    assert _block(lib, Desc(bounds=0)) == -1 and b"key_bounds" in lib.tkphi_last_error()
    assert _block(lib, d, idx=0x40002) == -1
    for sel in ((-1, 1, 1), (0, 0, 1), (0, 1, -1)):
        assert _block(lib, d, sel=sel) == -1
    assert _block(lib, d, sel=(1 << 20, 1 << 20, 5)) == -2
    assert lib.tkphi_paged_block_attention(d.ref, None, 1 << 16, 1 << 17, 0, 0, 0.0, 1 << 20, 1 << 40, None) == -1
    long = Desc(lens=((1, 131073 * 16),), max_pages=131073, n_pages=131073)
    assert _block(lib, long) == -2 and b"pages" in lib.tkphi_last_error()


def test_bad_arguments_of_append(lib):
    d = Desc()
    assert lib.tkphi_paged_append(d.ref, None, None) == -1
    for bad in (dict(k_new=0), dict(v_new=0x20008), dict(q=0), dict(q_out=0), dict(q=0x30008), dict(q_out=0x40004),
                dict(inv_freq=0), dict(inv_freq=0x50002), dict(pairs=2), dict(positions=0x60004), dict(k_stride_token=60), dict(v_stride_head=-64),
                dict(o_stride_head=0), dict(o_stride_token=448), dict(q_out=0x30000, o_stride_token=520)):
        assert _append(lib, d, **bad) == -1, bad
    for rot in (8, 24, 80, -16):
        assert _append(lib, d, rot_dim=rot) == -2


def test_full_context_lifts_the_length_rule_for_attention_only(lib):
    d = Desc(kv=[100, 2])
    assert _attend(lib, d) == -1 and b"new tokens" in lib.tkphi_last_error()
    assert _attend(lib, d, flags=2, ws=0) == -3          # past the length checks


def test_a_step_without_tokens_does_nothing(lib):
    d = Desc(lens=((0, 100), (0, 0)))
    assert _attend(lib, d, q=0, y=0) == 0
    assert _block(lib, d, q=0, y=0) == 0
    assert _append(lib, d, k_new=0) == 0


def test_workspace_sizes(lib):
    def size(d, which, sel=None):
        s = None if sel is None else C.byref(B._PageSelection(*sel))
        return lib.tkphi_paged_workspace_bytes(d.ref, s, which)

    assert size(Desc(), T.WS_PAGED_ATTENTION) >= 256
    assert size(Desc(), 0) == 0 and b"kind" in lib.tkphi_last_error()
    assert size(Desc(), T.WS_PAGED_BLOCK_ATTENTION) == 0
    assert size(Desc(d=96), T.WS_PAGED_ATTENTION) == 0
    # no device pointer is needed to ask
    assert size(Desc(k=0, v=0, table=0, status=0), T.WS_PAGED_ATTENTION) > 0
    # the largest steps stay within what a device has
    for which, sel in ((T.WS_PAGED_ATTENTION, None), (T.WS_PAGED_BLOCK_ATTENTION, (1, 2, 20))):
        for n in (400, 10000, 100000):
            assert 0 < size(Desc(lens=[(m, n) for m in (1, 40, 7, 300)], max_pages=8192, n_pages=40000), which, sel) < 1 << 30
    # a call with a smaller workspace is refused before anything is enqueued
    d = Desc(lens=((1, 400), (1, 9000)), max_pages=1024, n_pages=4096)
    n = size(d, T.WS_PAGED_ATTENTION)
    assert _attend(lib, d, ws_bytes=n - 1) == -3 and b"needed" in lib.tkphi_last_error()
    n = size(d, T.WS_PAGED_BLOCK_ATTENTION, (1, 1, 4))
    assert _block(lib, d, ws_bytes=n - 1) == -3


def test_the_binding_keeps_its_own_lengths():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    lens, cu = np.array([20]), np.array([0, 1])
    kv = T.PagedKVCache(k, k.clone(), torch.zeros(1, 4, dtype=torch.int32), lens, cu, 4)
    lens[0], cu[1] = 10 ** 9, 10 ** 6
    assert kv.kv_lens[0] == 20 and kv.total_q == 1
    with pytest.raises(ValueError):
        kv.cu_q[1] = 5


def test_the_binding_refuses_tensors_of_another_device_type_or_shape(lib):
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    kv = T.PagedKVCache(k, k.clone(), torch.zeros(1, 4, dtype=torch.int32), [20], [0, 1], 4)
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    ws = torch.zeros(1024, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device"):
        T.paged_attention(kv, q, q.clone(), None, None, 0, ws)          # the cache is not on a GPU
    with pytest.raises(ValueError, match="type"):
        T.paged_attention(kv, q.float(), q.clone(), None, None, 0, ws)
    with pytest.raises(ValueError, match="tensor"):
        T.paged_append(kv, None, q)
    for bad in (dict(k=k.float()), dict(v=k[:2]), dict(page_table=torch.zeros(1, 4)), dict(page_table=torch.zeros(2, 4, dtype=torch.int32)),
                dict(cu_q=[0, 1, 2]), dict(key_bounds=torch.zeros(4, 2, 64, dtype=torch.bfloat16))):
        a = dict(k=k, v=k, page_table=torch.zeros(1, 4, dtype=torch.int32), kv_lens=[20], cu_q=[0, 1], n_q_heads=4)
        a.update(bad)
        with pytest.raises(AssertionError):
            T.PagedKVCache(**a)
