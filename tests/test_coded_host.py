"""Host-side behaviour of the calls over an 8-bit cache and of the head norms: the oracle against torch's types, refusals of
the library and of the binding.  No kernel is launched; runs without a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2604_05438_b200 as T
from oracle import paged8_oracle as P8
from paper_2604_05438_b200 import binding as B
from paper_2604_05438_b200.build import build_library
from test_paged_host import Desc


@pytest.fixture(scope="module")
def lib():
    build_library()
    return T.load_library()


# ---------------------------------------------------------------------------------------------- oracle
def test_codes_and_scales_of_the_oracle_are_those_of_the_types():
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    for table, kind in ((P8.CODES, torch.float8_e4m3fn), (P8.power(np.arange(256)), torch.float8_e8m0fnu)):
        assert np.array_equal(table, every.view(kind).double().numpy(), equal_nan=True)


def test_the_nearest_code_of_the_oracle():
    x = np.concatenate([np.linspace(-448, 448, 20011), np.exp2(np.linspace(-14, 8.8, 5001)), P8.CODES[:127], -P8.CODES[:127],
                        (P8.CODES[:126] + P8.CODES[1:127]) / 2])                       # (ties)
    x = x.astype(np.float32).astype(np.float64)                                        # (torch rounds from 32 bits)
    assert (P8.nearest(x) == torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()).all()


@pytest.mark.parametrize("top,byte", [(448.0, 127), (448.0000001, 128), (1.75, 119), (1.7500001, 120), (0.0, 1), (2.0 ** -130, 1), (np.inf, 255),
                                      (np.nan, 255), (3e38, 247)])
def test_scale_bytes_of_the_oracle(top, byte):
    assert P8.scale_byte(np.array([[0.0, top, -0.0]]))[0] == byte


# ---------------------------------------------------------------------------------------------- the library's refusals
class Coded:
    def __init__(self, ks=0x8000, vs=0x9000, **kw):
        d = kw.get("d", 64)
        self.step = Desc(**kw)
        self.c = B._CodedDesc(self.step.c, ks, vs)

    @property
    def ref(self):
        return C.byref(self.c)


def _attend(lib, d, ws=0x100000, ws_bytes=1 << 50, **kw):
    a = dict(q=0x10000, y=0x20000, lse=0x30000, scale=0.0, flags=0)
    a.update(kw)
    return lib.tkphi_coded_attention(d.ref, a["q"], a["y"], a["lse"], a["scale"], a["flags"], ws, ws_bytes, None)


def _block(lib, d, ws=0x100000, ws_bytes=1 << 50, **kw):
    a = dict(q=0x10000, y=0x20000, lse=0x30000, scale=0.0, idx=0x40000)
    a.update(kw)
    s = B._PageSelection(1, 1, 4)
    return lib.tkphi_coded_block_attention(d.ref, C.byref(s), a["q"], a["y"], a["lse"], a["idx"], a["scale"], ws, ws_bytes, None)


def _step(**kw):
    a = dict(k_new=0x10000, k_stride_token=128, k_stride_head=64, v_new=0x20000, v_stride_token=128, v_stride_head=64, q=0x30000,
             q_stride_token=512, q_stride_head=64, q_out=0x40000, o_stride_token=512, o_stride_head=64, inv_freq=0x50000,
             rot_dim=64, pairs=0, positions=None)
    a.update(kw)
    return B._AppendDesc(**a)


def _norm(**kw):
    a = dict(q_weight=0x60000, q_stride_head=0, k_weight=0x70000, k_stride_head=64, eps=1e-6)
    a.update(kw)
    return B._NormDesc(**a)


def _append(lib, d, norm=None, **kw):
    s = _step(**kw)
    return lib.tkphi_coded_append(d.ref, C.byref(s), None if norm is None else C.byref(norm), None)


def _read(lib, d, cu=(0, 100, 164), first=None, **kw):
    cu = np.array(cu, np.int64)
    f = None if first is None else np.array(first, np.int64)
    a = dict(cu_rows_host=cu.ctypes.data, cu_rows_dev=0xA000, first_host=None if f is None else f.ctypes.data,
             first_dev=None if f is None else 0xB000, k_out=0x100000, k_stride_row=128, k_stride_head=64, v_out=0x200000,
             v_stride_row=64, v_stride_head=64 * 164)
    a.update(kw)
    r = B._ReadDesc(**a)
    return lib.tkphi_coded_read(d.ref, C.byref(r), None)


ALL = (_attend, _block, _append, _read)


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("bad,status", [
    (dict(ks=0), -1), (dict(vs=0), -1), (dict(ks=0x8008), -1), (dict(vs=0x9004), -1), (dict(d=96), -2), (dict(dtype=2), -2), (dict(hq=7), -1),
    (dict(ps=48), -2), (dict(k=0), -1), (dict(v=0x2008), -1), (dict(table=0), -1), (dict(kv_dev=0), -1), (dict(status=0), -1),
    (dict(strides=(2048, 1024, 72)), -1), (dict(strides=(2056, 1024, 64)), -1), (dict(strides=(2048, 1024, -64)), -1),
    (dict(strides=(2048, 960, 64)), -1), (dict(strides=(0, 1024, 64)), -1), (dict(kv=[100, 513]), -1), (dict(kv=[1 << 40, 64]), -1),
])
def test_bad_descriptors_are_refused(lib, call, bad, status):
    assert call(lib, Coded(**bad)) == status, lib.tkphi_last_error()
    assert lib.tkphi_last_error()


def test_missing_descriptors(lib):
    sel, norm, step = B._PageSelection(1, 1, 4), _norm(), _step()
    assert lib.tkphi_coded_attention(None, 1, 1, 1, 0.0, 0, 1, 1, None) == -1
    assert lib.tkphi_coded_block_attention(None, C.byref(sel), 1, 1, 1, 1, 0.0, 1, 1, None) == -1
    assert lib.tkphi_coded_block_attention(Coded().ref, None, 1 << 16, 1 << 17, 0, 0, 0.0, 1 << 20, 1 << 40, None) == -1
    assert lib.tkphi_coded_append(None, C.byref(step), None, None) == -1
    assert lib.tkphi_coded_append(Coded().ref, None, None, None) == -1
    assert lib.tkphi_coded_read(None, None, None) == -1
    assert lib.tkphi_coded_read(Coded().ref, None, None) == -1
    assert lib.tkphi_coded_workspace_bytes(None, None, T.WS_PAGED_ATTENTION) == 0
    assert lib.tkphi_paged_append_norm(None, C.byref(step), C.byref(norm), None) == -1
    assert lib.tkphi_paged_append_norm(Desc().ref, None, C.byref(norm), None) == -1
    assert lib.tkphi_paged_append_norm(Desc().ref, C.byref(step), None, None) == -1 and b"norm" in lib.tkphi_last_error()


def test_bad_arguments_of_the_attention_calls(lib):
    for call in (_attend, _block):
        for bad in (dict(q=0), dict(q=0x10008), dict(y=0), dict(lse=0x30002), dict(scale=-1.0), dict(scale=float("nan"))):
            assert call(lib, Coded(), **bad) == -1
        assert call(lib, Coded(), ws=0) == -3 and call(lib, Coded(), ws=0x100010) == -3 and call(lib, Coded(), ws_bytes=64) == -3
    assert _attend(lib, Coded(), flags=1) == -1
    assert _block(lib, Coded(bounds=0)) == -1 and b"key_bounds" in lib.tkphi_last_error()
    assert _block(lib, Coded(), idx=0x40002) == -1


@pytest.mark.parametrize("bad", [dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(q_weight=0x60008), dict(k_weight=0x70004),
                                 dict(q_stride_head=32), dict(k_stride_head=66), dict(k_stride_head=-64), dict(q_stride_head=1 << 40)])
def test_bad_norms_are_refused(lib, bad):
    norm, step = _norm(**bad), _step()
    assert _append(lib, Coded(), norm) == -1 and lib.tkphi_last_error()
    assert lib.tkphi_paged_append_norm(Desc().ref, C.byref(step), C.byref(norm), None) == -1 and lib.tkphi_last_error()


def test_bad_arguments_of_append(lib):
    for bad in (dict(k_new=0), dict(v_new=0x20008), dict(q=0), dict(q_out=0x40004), dict(inv_freq=0), dict(pairs=2), dict(rot_dim=24),
                dict(k_stride_token=60), dict(o_stride_head=0), dict(positions=0x60004), dict(q_out=0x30000, o_stride_token=520)):
        assert _append(lib, Coded(), **bad) in (-1, -2), bad
        assert _append(lib, Coded(), _norm(), **bad) in (-1, -2), bad


@pytest.mark.parametrize("bad", [
    dict(cu=(1, 100, 164)), dict(cu=(0, 100, 99)), dict(cu=(0, 101, 164)), dict(cu=(0, 100, 165)), dict(cu=(0, 100, 1 << 32)),
    dict(first=(-1, 0)), dict(first=(1, 0)), dict(first=(0, 65), cu=(0, 1, 1)), dict(first=(1 << 62, 0), cu=(0, 1, 1)),
    dict(cu_rows_host=None), dict(cu_rows_dev=None), dict(cu_rows_dev=0xA004), dict(first_dev=0xB000), dict(first=(0, 0), first_dev=None),
    dict(first=(0, 0), first_dev=0xB004), dict(k_out=None, v_out=None), dict(k_out=0x100008), dict(v_out=0x200004), dict(k_stride_row=100),
    dict(k_stride_head=-64), dict(v_stride_head=64), dict(k_stride_row=64), dict(v_stride_row=1 << 40)])
def test_bad_rows_are_refused(lib, bad):
    assert _read(lib, Coded(), **bad) == -1, bad
    assert lib.tkphi_last_error()


def test_nothing_to_do_is_done_without_a_device(lib):
    none = Coded(lens=((0, 100), (0, 64)))
    assert _attend(lib, none) == 0 and _append(lib, none) == 0 and _append(lib, none, _norm()) == 0 and _block(lib, none) == 0
    assert _read(lib, Coded(), cu=(0, 0, 0)) == 0
    assert _read(lib, Coded(), cu=(0, 0, 0), first=(100, 64)) == 0


def test_workspace_sizes(lib):
    ask = lambda d: lib.tkphi_coded_workspace_bytes(d.ref, None, T.WS_PAGED_ATTENTION)  # noqa: E731
    # 32 tokens x group 4 = 128 query rows: the cache is expanded to 16 bits there, 128 rows x 2 heads x 64 dims x 4 bytes a page
    few, many = ask(Coded(lens=((16, 100), (3, 64)))), ask(Coded(lens=((32, 100), (3, 64))))
    assert few > 0 and many >= 128 * 2 * 64 * 4
    assert ask(Coded(lens=((32, 300), (32, 64)))) >= 4 * 128 * 2 * 64 * 4
    assert ask(Coded(d=96)) == 0 and lib.tkphi_coded_workspace_bytes(Coded().ref, None, 17) == 0
    sel = B._PageSelection(1, 1, 4)
    assert lib.tkphi_coded_workspace_bytes(Coded().ref, C.byref(sel), T.WS_PAGED_BLOCK_ATTENTION) > 0
    # a batch of sequences that share pages may name more rows than any memory holds
    huge = Coded(lens=((64, 1 << 30),) * 200, max_pages=1 << 26)
    assert ask(huge) == 0 and b"too many" in lib.tkphi_last_error()


# ---------------------------------------------------------------------------------------------- the binding's refusals
F8, E8, BF = torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.bfloat16


def cache(**kw):
    a = dict(k=torch.zeros(4, 2, 16, 64, dtype=F8), v=torch.zeros(4, 2, 16, 64, dtype=F8), k_scales=torch.zeros(4, 2, 16, dtype=torch.uint8).view(E8),
             v_scales=torch.zeros(4, 2, 16, dtype=torch.uint8).view(E8), page_table=torch.zeros(1, 4, dtype=torch.int32), kv_lens=[20], cu_q=[0, 1],
             n_q_heads=4, dtype=BF)
    a.update(kw)
    return T.PagedKVCache8(**a)


@pytest.mark.parametrize("bad", [dict(k=torch.zeros(4, 2, 16, 64, dtype=BF)), dict(v=torch.zeros(4, 2, 16, 64, dtype=torch.uint8)), dict(dtype=torch.float32),
                                 dict(dtype=F8), dict(k_scales=torch.zeros(4, 2, 16)), dict(v_scales=torch.zeros(4, 2, 32, dtype=torch.uint8).view(E8)),
                                 dict(k_scales=torch.zeros(4, 16, 2, dtype=torch.uint8).view(E8).transpose(1, 2)),
                                 dict(key_bounds=torch.zeros(4, 2, 2, 64)), dict(k=torch.zeros(4, 16, 2, 64, dtype=F8).transpose(1, 2)),
                                 dict(cu_q=[0, 1, 2]), dict(page_table=torch.zeros(1, 4, dtype=torch.int64))])
def test_caches_that_are_none(lib, bad):
    with pytest.raises(AssertionError):
        cache(**bad)


def test_calls_that_the_binding_refuses(lib):
    kv, ws = cache(), torch.zeros(1 << 20, dtype=torch.uint8)
    k16 = torch.zeros(4, 2, 16, 64, dtype=BF)
    kv16 = T.PagedKVCache(k16, k16.clone(), torch.zeros(1, 4, dtype=torch.int32), [20], [0, 1], 4)
    kn, q = torch.zeros(1, 2, 64, dtype=BF), torch.zeros(1, 4, 64, dtype=BF)
    rows = T.CacheRows([0, 20])
    out = torch.zeros(20, 2, 64, dtype=BF)
    with pytest.raises(ValueError, match="8 bits"):
        T.paged_read(kv16, rows, out, out)
    with pytest.raises(ValueError, match="number of sequences"):
        T.paged_read(kv, T.CacheRows([0, 1, 2]), out, out)
    with pytest.raises(ValueError, match="k_out"):
        T.paged_read(kv, rows, out.half(), out)
    with pytest.raises(ValueError, match="device"):                    # the next check: these tensors are on the CPU
        T.paged_read(kv, rows, out, out)
    with pytest.raises(ValueError, match="type"):
        T.paged_append(kv, kn.half(), kn)
    with pytest.raises(ValueError, match="scale"):
        T.paged_attention(kv, q, q.clone(), None, -1.0, T.FLAG_NONE, ws)
    for bad in (torch.zeros(64, dtype=torch.float64), torch.zeros(3, 2, 64)):
        with pytest.raises(AssertionError):
            T.HeadNorms(bad, None)
    with pytest.raises(AssertionError):
        T.CacheRows([0])
    with pytest.raises(AssertionError):
        T.CacheRows([0, 1], [0, 0])
    with pytest.raises(AssertionError):
        T.CacheRows([0, 1], None, first_dev=torch.zeros(1, dtype=torch.int64))


def test_the_build_takes_every_kernel_source():
    import os

    from paper_2604_05438_b200 import build

    assert sorted(f for f in os.listdir(build.CSRC) if f.endswith(".cu")) == sorted(build.SOURCES)
    assert sorted(f for f in os.listdir(build.CSRC) if f.endswith(".cuh")) == sorted(os.path.basename(h) for h in build.HEADERS
                                                                                      if h.endswith(".cuh"))
