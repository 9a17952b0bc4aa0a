"""Attention of many new tokens and positions with several axes, without a GPU: what the entry points refuse before any CUDA call."""
import ctypes as C

import pytest

import paper_2607_19456_b200 as moa
from paper_2607_19456_b200 import build as moa_build
from test_paged_refusals import BAD_CACHES, INT4, cache


@pytest.fixture(scope="module", autouse=True)
def built():
    moa_build.build()


def strides(st):
    return None if st is None else (C.c_longlong * 4)(*st)


def prompt(q=256, k=256, v=256, out=256, dtype=moa.BF16, st=None, tokens=10, h_q=4, h_kv=2, d=128, batch=2, start=256, causal=1, scale=1.0, ws=256,
           ws_bytes=1 << 40):
    return moa.lib().moa_prompt_attn(q, k, v, out, dtype, strides(st), tokens, h_q, h_kv, d, batch, start, causal, scale, ws, ws_bytes, None)


def chunk(c, q=256, out=256, dtype=moa.BF16, q_stride=0, tokens=10, h_q=4, batch=2, start=256, lens=256, table=256, max_pages=3, scale=1.0, ws=256,
          ws_bytes=1 << 40):
    return moa.lib().moa_paged_chunk_attn(c, q, out, dtype, q_stride, tokens, h_q, batch, start, lens, table, max_pages, scale, ws, ws_bytes, None)


def rotate(q=256, k=256, q_out=512, k_out=512, dtype=moa.BF16, st=None, tokens=10, h_q=4, h_kv=2, d=128, pos=256, axes=3, amap=bytes(64), cos_sin=256, rows=10,
           rot=128, style=0):
    return moa.lib().moa_rotate_axes(q, k, q_out, k_out, dtype, strides(st), tokens, h_q, h_kv, d, pos, axes, amap, cos_sin, rows, rot, style, None)


def append(c, pos=256, axes=3, amap=bytes(64), rot=128, h_q=4, cos_sin=256):
    return moa.lib().moa_paged_append_axes(c, 256, 256, 256, 256, moa.BF16, None, 2, h_q, 2, None, 256, 256, 3, pos, axes, amap, cos_sin, 10, rot, 0, None)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(out=None), 1), (dict(tokens=0), 1), (dict(h_q=0), 1), (dict(h_q=3), 1), (dict(h_kv=0), 1),
    (dict(batch=0), 1), (dict(start=None), 1), (dict(causal=2), 1), (dict(causal=-1), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(scale=3e38), 1), (dict(d=0), 1), (dict(d=96), moa.ERR_UNSUPPORTED), (dict(d=256), moa.ERR_UNSUPPORTED),
    (dict(st=(-8, 256, 256, 512)), 1), (dict(st=(512, 1 << 41, 256, 512)), 1), (dict(st=(512, 256, 256, 504)), 1), (dict(st=(516, 256, 256, 512)), moa.ERR_ALIGN),
    (dict(q=264), moa.ERR_ALIGN), (dict(k=258), moa.ERR_ALIGN), (dict(v=264), moa.ERR_ALIGN), (dict(out=8), moa.ERR_ALIGN), (dict(start=258), moa.ERR_ALIGN),
    (dict(tokens=1 << 30), moa.ERR_CAPACITY), (dict(tokens=1 << 24, h_q=64, h_kv=64), moa.ERR_CAPACITY), (dict(batch=1 << 20), moa.ERR_CAPACITY),
    (dict(ws=None), moa.ERR_WORKSPACE), (dict(ws=128), moa.ERR_ALIGN),
])
def test_prompt(change, code):
    assert prompt(**change) == code


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_descriptor(change, code):
    assert chunk(cache(**change)) == code
    assert append(cache(**change)) == code


@pytest.mark.parametrize("change,code", [
    (dict(q=None), 1), (dict(out=None), 1), (dict(lens=None), 1), (dict(table=None), 1), (dict(tokens=0), 1), (dict(batch=0), 1), (dict(h_q=0), 1), (dict(h_q=3), 1),
    (dict(max_pages=0), 1), (dict(start=None), 1), (dict(dtype=3), 1), (dict(dtype=moa.F16), moa.ERR_UNSUPPORTED), (dict(dtype=moa.F32), moa.ERR_UNSUPPORTED),
    (dict(q_stride=-8), 1), (dict(q_stride=1 << 41), 1), (dict(q_stride=513), moa.ERR_ALIGN), (dict(q=258), moa.ERR_ALIGN), (dict(out=264), moa.ERR_ALIGN),
    (dict(lens=257), moa.ERR_ALIGN), (dict(table=258), moa.ERR_ALIGN), (dict(start=258), moa.ERR_ALIGN), (dict(scale=float("nan")), 1),
    (dict(tokens=1 << 30), moa.ERR_CAPACITY), (dict(ws=None), moa.ERR_WORKSPACE), (dict(ws=64), moa.ERR_ALIGN),
])
def test_chunk(change, code):
    assert chunk(cache(), **change) == code
    assert chunk(None) == moa.ERR_INVALID
    assert chunk(cache(**INT4), dtype=moa.F32) == moa.ERR_UNSUPPORTED


@pytest.mark.parametrize("change,code", [
    (dict(q=None), 1), (dict(k=None), 1), (dict(q_out=None), 1), (dict(k_out=None), 1), (dict(tokens=0), 1), (dict(h_q=-1), 1), (dict(h_q=0, h_kv=0), 1),
    (dict(d=32), moa.ERR_UNSUPPORTED), (dict(dtype=3), 1), (dict(pos=None), 1), (dict(amap=None), 1), (dict(axes=0), 1), (dict(axes=5), 1),
    (dict(amap=bytes([0] * 63 + [3])), 1), (dict(rot=0), 1), (dict(rot=130), 1), (dict(rot=63), 1), (dict(cos_sin=None), 1), (dict(rows=0), 1), (dict(style=2), 1),
    (dict(q_out=256, st=(512, 256, 1024, 256)), 1), (dict(st=(512, 256, 504, 256)), 1), (dict(st=(-8, 256, 512, 256)), 1), (dict(st=(516, 256, 512, 256)), moa.ERR_ALIGN),
    (dict(q=258), moa.ERR_ALIGN), (dict(k_out=264), moa.ERR_ALIGN), (dict(cos_sin=260), moa.ERR_ALIGN), (dict(pos=258), moa.ERR_ALIGN),
])
def test_rotate(change, code):
    assert rotate(**change) == code


@pytest.mark.parametrize("change,code", [
    (dict(pos=None), 1), (dict(amap=None), 1), (dict(axes=0), 1), (dict(axes=5), 1), (dict(axes=2, amap=bytes([2] * 64)), 1), (dict(rot=0), 1), (dict(rot=63), 1),
    (dict(cos_sin=None), 1), (dict(pos=257), moa.ERR_ALIGN), (dict(cos_sin=264), moa.ERR_ALIGN),
])
def test_append(change, code):
    assert append(cache(), **change) == code


def test_workspace_bytes():
    assert moa.moa_prompt_workspace_bytes(0, 4, 2, 128, 1) == moa.moa_prompt_workspace_bytes(10, 3, 2, 128, 1) == 0
    assert moa.moa_prompt_workspace_bytes(10, 4, 2, 96, 1) == moa.moa_prompt_workspace_bytes(10, 4, 2, 128, 0) == 0
    small, large = moa.moa_prompt_workspace_bytes(4, 4, 2, 64, 1), moa.moa_prompt_workspace_bytes(4000, 4, 2, 128, 1)
    assert 0 < small < large == moa.moa_prompt_workspace_bytes(1 << 20, 4, 2, 128, 9) and small % 256 == 0


def test_binding_checks_what_c_cannot():
    with pytest.raises(ValueError):
        moa.moa_rotate_axes(None, None, None, None, 0, None, 1, 1, 0, 64, None, 3, bytes(31), None, 1, 64, 0, stream=0)
    with pytest.raises(ValueError):
        moa.moa_prompt_attn(256, 256, 256, 256, 1, (1, 2, 3), 1, 1, 1, 64, 1, None, True, 1.0, None, 0, stream=0)
    with pytest.raises(moa.MoaError):
        moa.moa_prompt_attn(None, 256, 256, 256, 1, None, 1, 1, 1, 64, 1, None, True, 1.0, None, 0, stream=0)
