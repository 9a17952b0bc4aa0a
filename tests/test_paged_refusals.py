"""Paged caches without a GPU: what the entry points refuse before any CUDA call, and the layout of the descriptor."""
import ctypes as C

import pytest

import paper_2607_19456_b200 as moa
from paper_2607_19456_b200 import build as moa_build


@pytest.fixture(scope="module", autouse=True)
def built():
    moa_build.build()


def cache(**kw):
    a = dict(format=moa.KV_BF16, k=256, v=256, num_pages=4, page_size=16, h_kv=2, d=128)
    a.update(kw)
    return moa.PagedCache(**a)


INT4 = dict(format=moa.KV_INT4, k_params=256, v_params=256)
BAD_CACHES = [
    (dict(k=None), moa.ERR_INVALID), (dict(v=None), moa.ERR_INVALID), (dict(format=4), moa.ERR_INVALID),
    (dict(format=-1), moa.ERR_INVALID), (dict(num_pages=0), moa.ERR_INVALID), (dict(page_size=0), moa.ERR_INVALID),
    (dict(h_kv=0), moa.ERR_INVALID), (dict(d=96), moa.ERR_UNSUPPORTED), (dict(d=256), moa.ERR_UNSUPPORTED),
    (dict(k=264), moa.ERR_ALIGN), (dict(v=258), moa.ERR_ALIGN),
    (dict(k_strides=(4096, 2048, 64)), moa.ERR_INVALID), (dict(k_strides=(-4096, 2048, 128)), moa.ERR_INVALID),
    (dict(v_strides=(1 << 41, 2048, 128)), moa.ERR_INVALID), (dict(v_strides=(4096, 2048, 132)), moa.ERR_ALIGN),
    (dict(INT4, k_params=None), moa.ERR_INVALID), (dict(INT4, v_params=258), moa.ERR_ALIGN),
    (dict(INT4, v_strides=(4096, 2048, 144)), moa.ERR_ALIGN),
]


def attend(c, q=256, out=256, dtype=moa.BF16, q_stride=0, batch=2, h_q=4, lens=256, table=256, max_pages=3, scale=1.0, ws=256,
           ws_bytes=1 << 30):
    return moa.lib().moa_paged_decode_attn(c, q, out, dtype, q_stride, batch, h_q, lens, table, max_pages, scale, ws, ws_bytes, None)


def append(c, q=256, k=256, v=256, q_out=256, dtype=moa.BF16, strides=None, tokens=2, h_q=4, batch=2, start=None, lens=256,
           table=256, max_pages=3, cos_sin=256, rows=10, rot=128, style=0):
    st = None if strides is None else (C.c_longlong * 4)(*strides)
    return moa.lib().moa_paged_append(c, q, k, v, q_out, dtype, st, tokens, h_q, batch, start, lens, table, max_pages,
                                      cos_sin, rows, rot, style, None)


def gather(c, k_out=256, v_out=256, dtype=moa.F32, batch=2, n_out=5, start=None, lens=256, table=256, max_pages=3):
    return moa.lib().moa_paged_gather(c, k_out, v_out, dtype, batch, n_out, start, lens, table, max_pages, None)


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_descriptor(change, code):
    c = cache(**change)
    dtype = moa.BF16
    assert attend(c, dtype=dtype) == code
    assert append(c, dtype=dtype) == code
    assert gather(c) == code


def test_null_descriptor():
    assert attend(None) == append(None) == gather(None) == moa.ERR_INVALID


@pytest.mark.parametrize("change,code", [
    (dict(q=None), 1), (dict(out=None), 1), (dict(lens=None), 1), (dict(table=None), 1), (dict(batch=0), 1), (dict(h_q=3), 1),
    (dict(h_q=0), 1), (dict(max_pages=0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(dtype=3), 1),
    (dict(dtype=moa.F16), moa.ERR_UNSUPPORTED), (dict(q_stride=-8), 1), (dict(q_stride=513), moa.ERR_ALIGN),
    (dict(q=258), moa.ERR_ALIGN), (dict(out=264), moa.ERR_ALIGN), (dict(lens=257), moa.ERR_ALIGN), (dict(table=258), moa.ERR_ALIGN),
    (dict(ws=None), moa.ERR_WORKSPACE), (dict(ws=128), moa.ERR_ALIGN), (dict(batch=1 << 30), moa.ERR_CAPACITY),
])
def test_attend(change, code):
    assert attend(cache(), **change) == code


def test_dtype_of_a_4_bit_cache():
    for call in (attend, append):
        assert call(cache(**INT4), dtype=moa.F32) == moa.ERR_UNSUPPORTED
    assert attend(cache(format=moa.KV_F32), dtype=moa.BF16) == moa.ERR_UNSUPPORTED


@pytest.mark.parametrize("change,code", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(q=None), 1), (dict(q_out=None), 1), (dict(lens=None), 1), (dict(table=None), 1),
    (dict(tokens=0), 1), (dict(tokens=3), 1), (dict(h_q=-2), 1), (dict(h_q=3), 1), (dict(batch=0), 1), (dict(max_pages=0), 1),
    (dict(rot=-2), 1), (dict(rot=130), 1), (dict(rot=63), 1), (dict(cos_sin=None), 1), (dict(rows=0), 1), (dict(style=2), 1),
    (dict(dtype=5), 1), (dict(dtype=moa.F16), moa.ERR_UNSUPPORTED), (dict(cos_sin=260), moa.ERR_ALIGN), (dict(k=264), moa.ERR_ALIGN),
    (dict(q_out=264), moa.ERR_ALIGN), (dict(start=258), moa.ERR_ALIGN), (dict(strides=(1024, 1024, 1024, 511)), 1),
    (dict(strides=(1024, -8, 1024, 512)), 1), (dict(strides=(512, 1028, 1024, 512)), moa.ERR_ALIGN),
    (dict(strides=(1024, 1024, 1024, 512)), 1),                        # q_out is q, with another stride
])
def test_append(change, code):
    assert append(cache(), **change) == code


def test_a_pool_that_is_written_has_no_zero_strides():
    for st in ((0, 2048, 128), (4096, 0, 128)):
        assert append(cache(k_strides=st)) == moa.ERR_INVALID
        assert append(cache(v_strides=st)) == moa.ERR_INVALID


@pytest.mark.parametrize("change,code", [
    (dict(k_out=None), 1), (dict(v_out=None), 1), (dict(dtype=3), 1), (dict(batch=0), 1), (dict(n_out=0), 1), (dict(lens=None), 1),
    (dict(table=None), 1), (dict(max_pages=0), 1), (dict(k_out=260), moa.ERR_ALIGN), (dict(start=257), moa.ERR_ALIGN),
    (dict(n_out=(1 << 31) - 1, batch=1 << 20), moa.ERR_CAPACITY),
])
def test_gather(change, code):
    assert gather(cache(), **change) == code


def test_workspace_size():
    assert moa.moa_paged_workspace_bytes(4, 32, 8, 128) > 0
    for bad in ((0, 32, 8, 128), (4, 30, 8, 128), (4, 32, 0, 128), (4, 32, 8, 80)):
        assert moa.moa_paged_workspace_bytes(*bad) == 0


def test_without_a_gpu_the_calls_fail_loudly():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    c = cache()
    assert attend(c) == append(c) == gather(c) == moa.ERR_CUDA


def test_bindings_raise():
    with pytest.raises(moa.MoaError) as e:
        moa.moa_paged_gather(cache(d=80), 256, 256, moa.F32, 1, 1, None, 256, 256, 1, stream=0)
    assert e.value.code == moa.ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        moa.moa_paged_append(cache(), 256, 256, 256, 256, moa.BF16, (1, 2), 1, 4, 1, None, 256, 256, 1, None, 0, 0, 0, stream=0)
    with pytest.raises(ValueError):
        cache(k_strides=(1, 2))
