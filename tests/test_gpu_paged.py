"""Attention over paged caches in fp32, bf16, fp16 and 4 bits against the definition in 64 bits."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, attend, attend64, dtype_of, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

FORMATS = [moa.KV_F32, moa.KV_BF16, moa.KV_F16, moa.KV_INT4]


def queries(rng, batch, h_q, d, dtype):
    return torch.from_numpy(rng.standard_normal((batch, h_q, d)).astype(np.float32)).cuda().to(TYPES[dtype])


def check(p, q, out, scale, lens=None, skip=()):
    want, bound = attend64(q.double().cpu().numpy(), p, scale, lens)
    got = out.double().cpu().numpy()
    if p.fmt == moa.KV_F32:
        bound = np.maximum(bound, 5e-6)                                     # the library's bar
    tol = bound + np.abs(want) * torch.finfo(out.dtype).eps / 2 + 2.0 ** -25
    for b in range(len(want)):
        if b not in skip:
            known = ~np.isnan(want[b])                                      # (infinite queries: NaN by the definition too)
            assert np.array_equal(known, ~np.isnan(got[b])), b
            off, tol_b = np.abs(got[b] - want[b])[known], tol[b][known]
            assert np.all(off <= tol_b), (b, float(off.max()), float((off / tol_b).max()))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (4, 4), (8, 2), (7, 1), (8, 1), (18, 2), (16, 1), (33, 1)])
def test_lengths_and_groups(fmt, d, h_q, h_kv):
    rng = np.random.default_rng(100 * h_q + 10 * h_kv + fmt + d)
    lens = [1, 0, 15, 16, 17, 300, 2, 129]
    p = Paged(rng, fmt, lens, h_kv, d, 16)
    dtype = dtype_of(fmt, moa.F16 if h_q % 2 else moa.BF16)
    q = queries(rng, len(lens), h_q, d, dtype)
    out = attend(p, q, dtype, d ** -0.5)
    torch.cuda.synchronize()
    assert moa.moa_device_status() == 0 and moa.moa_last_path() == moa.PATH_PAGED
    assert bool((out[1] == 0).all())
    check(p, q, out, d ** -0.5)


@pytest.mark.parametrize("page", [1, 5, 8, 20, 24, 64, 100])
@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_page_sizes_and_layouts(fmt, page):
    rng = np.random.default_rng(page + 1000 * fmt)
    for heads_inner, d in ((False, 128), (True, 64), (True, 128)):
        lens = [203, 1, 64, 37]
        p = Paged(rng, fmt, lens, 3, d, page, heads_inner=heads_inner)
        dtype = dtype_of(fmt)
        q = queries(rng, 4, 6, d, dtype)
        check(p, q, attend(p, q, dtype, 0.1), 0.1)
    assert moa.moa_device_status() == 0


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
@pytest.mark.parametrize("lens,h_q,h_kv", [([20011], 8, 1), ([9000, 3], 32, 2), ([1700] * 9, 12, 3), ([33] * 150, 4, 2)])
def test_units_cut_between_warps_and_ctas(fmt, lens, h_q, h_kv):
    rng = np.random.default_rng(len(lens) + fmt)
    p = Paged(rng, fmt, lens, h_kv, 128, 32)
    dtype = dtype_of(fmt, moa.F16)
    q = queries(rng, len(lens), h_q, 128, dtype)
    ws = workspace(len(lens), h_q, h_kv, 128)
    first = attend(p, q, dtype, 0.08, ws=ws)
    check(p, q, first, 0.08)
    assert torch.equal(first, attend(p, q, dtype, 0.08, ws=ws))             # the same bits again, on a used workspace
    for ctas in (1, 5, 300):
        moa.moa_set_option(moa.OPT_NUM_CTAS, ctas)
        try:
            check(p, q, attend(p, q, dtype, 0.08), 0.08)
        finally:
            moa.moa_set_option(moa.OPT_NUM_CTAS, 0)
    assert moa.moa_device_status() == 0


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_many_sequences(fmt):
    rng = np.random.default_rng(7 + fmt)
    lens = rng.integers(0, 40, 1300).tolist()                               # several sequences to a thread of the length scan
    p = Paged(rng, fmt, lens, 1, 64, 16)
    dtype = dtype_of(fmt)
    q = queries(rng, len(lens), 2, 64, dtype)
    out = attend(p, q, dtype, 0.125)
    check(p, q, out, 0.125)
    assert bool((out[torch.tensor(lens, device="cuda") == 0] == 0).all()) and moa.moa_device_status() == 0


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_weight_on_few_rows(fmt):
    """Scores far apart, rising and falling through the sequence, so that the reference maximum moves often."""
    rng = np.random.default_rng(17 + fmt)
    d, n = 128, 1500
    dtype = dtype_of(fmt, moa.F16)
    q = rng.standard_normal((4, 4, d)).astype(np.float32)
    q[:, 1:] = q[:, :1]
    unit = q[:, 0] / (q[:, 0] ** 2).sum(-1, keepdims=True)                  # a row t * unit scores t
    ramps = [np.linspace(-40, 4, n), np.linspace(4, -40, n), np.where(np.arange(n) == 777, 5.0, -30.0), np.linspace(-3000, 0, n)]
    k = [(r[:, None] * unit[b][None] / 0.1)[None] for b, r in enumerate(ramps)]
    p = Paged(rng, fmt, [n] * 4, 1, d, 16, k=k)
    qd = torch.from_numpy(q).cuda().to(TYPES[dtype])
    check(p, qd, attend(p, qd, dtype, 0.1), 0.1)


def test_value_rows_of_very_different_size():
    """4 bits: the scales of V span 2^-20..2^8 inside a sequence, small ones first, large ones first, and with the weight on a small one."""
    rng = np.random.default_rng(23)
    d, n = 128, 700
    grow = 2.0 ** np.linspace(-20, 8, n)
    v = [rng.standard_normal((1, n, d)) * grow[:, None], rng.standard_normal((1, n, d)) * grow[::-1, None],
         rng.standard_normal((1, n, d)) * np.where(np.arange(n) == 5, 2.0 ** -6, 1.0)[:, None]]
    k = [rng.standard_normal((1, n, d)) for _ in v]
    q = rng.standard_normal((3, 8, d)).astype(np.float32)
    q[2] = q[2, :1]
    k[2][0, 5] = 400 * q[2, 0] / (q[2, 0] ** 2).sum()
    p = Paged(rng, moa.KV_INT4, [n] * 3, 1, d, 16, k=k, v=v)
    for dtype in (moa.BF16, moa.F16):
        qd = torch.from_numpy(q).cuda().to(TYPES[dtype])
        check(p, qd, attend(p, qd, dtype, 0.05), 0.05)


@pytest.mark.parametrize("size", [1e-30, 1e-6, 3e4, 1e30])
def test_query_sizes_on_a_4_bit_cache(size):
    rng = np.random.default_rng(31)
    p = Paged(rng, moa.KV_INT4, [90, 5], 1, 128, 16)
    dtype = moa.BF16 if size in (1e-30, 1e30) else moa.F16
    q = (torch.from_numpy(rng.standard_normal((2, 3, 128)).astype(np.float32)) * size).cuda().to(TYPES[dtype])
    if size == 1e-6:
        q[0, 0] = 0
    scale = 0.1 / size
    check(p, q, attend(p, q, dtype, scale), scale)


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_strided_queries_negative_and_zero_scale(fmt):
    rng = np.random.default_rng(41 + fmt)
    p = Paged(rng, fmt, [100, 257], 2, 64, 16)
    dtype = dtype_of(fmt)
    wide = queries(rng, 2, 9, 64, dtype)
    q = wide[:, 2:6]
    for scale in (-0.2, 0.0):
        check(p, q, attend(p, q, dtype, scale, q_stride=9 * 64), scale)


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_values_that_are_no_numbers(fmt):
    """A NaN among a sequence's own rows spoils that sequence's head only; infinite values in a row do too."""
    rng = np.random.default_rng(43 + fmt)
    v = [rng.standard_normal((2, 50, 64)) for _ in range(3)]
    v[1][1, 20, 3] = np.nan
    p = Paged(rng, fmt, [50] * 3, 2, 64, 16, v=v)
    dtype = dtype_of(fmt)
    q = queries(rng, 3, 4, 64, dtype)
    out = attend(p, q, dtype, 0.1)
    assert bool(out[1, 2:, 3].isnan().all()) and not bool(out[1, :2].isnan().any())
    check(p, q, out, 0.1, skip=(1,))


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_lengths_and_pages_out_of_range(fmt):
    rng = np.random.default_rng(47 + fmt)
    p = Paged(rng, fmt, [70, 40, 200, 33, 64], 2, 128, 16)
    dtype = dtype_of(fmt)
    q = queries(rng, 5, 4, 128, dtype)
    lens = p.lens_dev.clone()
    lens[0], lens[3] = -1, p.max_pages * 16 + 1
    out = attend(p, q, dtype, 0.1, lens=lens)
    assert moa.moa_device_status() == moa.STATUS_SEQLEN_RANGE
    assert bool((out[0] == -3).all()) and bool((out[3] == -3).all())
    check(p, q, out, 0.1, skip=(0, 3))
    for bad in (p.num_pages, -1, 1 << 30, -(1 << 31)):
        p.table[2, 3] = bad
        out = attend(p, q, dtype, 0.1)
        assert moa.moa_device_status() == moa.STATUS_PAGE_RANGE
        assert bool(out[2].isnan().all())
        check(p, q, out, 0.1, skip=(2,))


def test_a_shared_page_and_a_smaller_workspace():
    rng = np.random.default_rng(53)
    p = Paged(rng, moa.KV_BF16, [64, 64], 2, 128, 32)
    p.table[1, 0] = p.table[0, 0]
    p.table_host[1, 0] = p.table_host[0, 0]
    q = queries(rng, 2, 4, 128, moa.BF16)
    check(p, q, attend(p, q, moa.BF16, 0.1), 0.1)
    ws, n = workspace(2, 4, 2, 128)
    with pytest.raises(moa.MoaError) as e:
        attend(p, q, moa.BF16, 0.1, ws=(ws, n // 2))
    assert e.value.code == moa.ERR_WORKSPACE


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_captured_calls_on_one_workspace_and_two_streams(fmt):
    rng = np.random.default_rng(59 + fmt)
    dtype = dtype_of(fmt)
    caches = [Paged(rng, fmt, [900, 31], 2, 128, 16), Paged(rng, fmt, [3, 2500], 2, 128, 16)]
    qs = [queries(rng, 2, 8, 128, dtype) for _ in caches]
    ws = workspace(2, 8, 2, 128)
    outs = [torch.zeros_like(q) for q in qs]
    for p, q, o in zip(caches, qs, outs):
        attend(p, q, dtype, 0.1, out=o, ws=ws)
    torch.cuda.synchronize()
    graphs = []
    for p, q, o in zip(caches, qs, outs):                                   # two graphs that share a workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            attend(p, q, dtype, 0.1, out=o, ws=ws)
        graphs.append(graph)
    lens = [[500, 31], [3, 1]]
    for p, n in zip(caches, lens):
        p.lens_dev.copy_(torch.tensor(n, dtype=torch.int32))                # lengths are read at replay
    for k in (0, 1, 0, 1, 1, 0):
        outs[k].zero_()
        graphs[k].replay()
        torch.cuda.synchronize()
        check(caches[k], qs[k], outs[k], 0.1, lens=lens[k])
    streams = [torch.cuda.Stream() for _ in caches]
    for _ in range(5):                                                      # two streams, a workspace each
        spaces = [workspace(2, 8, 2, 128) for _ in caches]
        torch.cuda.synchronize()
        for st, p, q, o, w in zip(streams, caches, qs, outs, spaces):
            with torch.cuda.stream(st):
                attend(p, q, dtype, 0.1, out=o, ws=w)
        torch.cuda.synchronize()
        for k in (0, 1):
            check(caches[k], qs[k], outs[k], 0.1, lens=lens[k])
    assert moa.moa_device_status() == 0
