"""Attention of chunks of new tokens over paged caches against the definition in 64 bits."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, dtype_of
from paged_util import attend as attend_one
from prompt_util import check_chunk, chunk, close, attend_new64, starts_of, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

FORMATS = [moa.KV_F32, moa.KV_BF16, moa.KV_F16, moa.KV_INT4]


def queries(rng, tokens, h_q, d, dtype):
    return torch.from_numpy(rng.standard_normal((tokens, h_q, d)).astype(np.float32)).cuda().to(TYPES[dtype])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (8, 2), (7, 1), (18, 2), (33, 1)])
def test_chunks_and_groups(fmt, d, h_q, h_kv):
    rng = np.random.default_rng(100 * h_q + h_kv + fmt + d)
    new, past = [1, 0, 5, 130, 17, 64, 1, 3], [0, 40, 300, 7, 0, 65, 511, 127]
    p = Paged(rng, fmt, [a + b for a, b in zip(new, past)], h_kv, d, 16)
    dtype = dtype_of(fmt, moa.F16 if h_q % 2 else moa.BF16)
    q = queries(rng, sum(new), h_q, d, dtype)
    out = chunk(p, q, new, dtype, d ** -0.5)
    torch.cuda.synchronize()
    assert moa.moa_device_status() == 0 and moa.moa_last_path() == moa.PATH_PROMPT
    check_chunk(out, p, q, new, dtype, d ** -0.5)


@pytest.mark.parametrize("page", [1, 5, 8, 16, 20, 48, 64, 100])
@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_page_sizes_and_layouts(fmt, page):
    rng = np.random.default_rng(page + 1000 * fmt)
    for heads_inner, d in ((False, 128), (True, 64), (True, 128)):
        new, past = [70, 2, 9], [133, 0, 290]
        p = Paged(rng, fmt, [a + b for a, b in zip(new, past)], 3, d, page, heads_inner=heads_inner)
        dtype = dtype_of(fmt)
        q = queries(rng, sum(new), 6, d, dtype)
        check_chunk(chunk(p, q, new, dtype, 0.1), p, q, new, dtype, 0.1)
    assert moa.moa_device_status() == 0


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
@pytest.mark.parametrize("new,past,h_q,h_kv", [([4], [9001], 8, 1), ([300], [2500], 8, 2), ([2, 1], [4000, 10], 16, 2), ([3] * 60, [90] * 60, 4, 2)])
def test_pieces(fmt, new, past, h_q, h_kv):
    """Few rows over many keys: cut into pieces, the same bits on a used workspace, any number of CTAs."""
    rng = np.random.default_rng(len(new) + fmt)
    p = Paged(rng, fmt, [a + b for a, b in zip(new, past)], h_kv, 128, 32)
    dtype = dtype_of(fmt, moa.F16)
    q = queries(rng, sum(new), h_q, 128, dtype)
    ws = workspace(sum(new), h_q, h_kv, 128, len(new))
    first = chunk(p, q, new, dtype, 0.08, ws=ws)
    check_chunk(first, p, q, new, dtype, 0.08)
    assert torch.equal(first, chunk(p, q, new, dtype, 0.08, ws=ws))
    try:
        for ctas in (1, 5, 300):
            moa.moa_set_option(moa.OPT_NUM_CTAS, ctas)
            check_chunk(chunk(p, q, new, dtype, 0.08), p, q, new, dtype, 0.08)
    finally:
        moa.moa_set_option(moa.OPT_NUM_CTAS, 0)
    assert moa.moa_device_status() == 0


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_single_tokens(fmt):
    """One token each, with and without starts, lengths of 0 among them, beside the single-query call."""
    rng = np.random.default_rng(7 + fmt)
    lens = [40, 0, 1, 333, 128, 0]
    p = Paged(rng, fmt, lens, 2, 64, 16)
    dtype = dtype_of(fmt)
    q = queries(rng, 6, 8, 64, dtype)
    out = chunk(p, q, [1] * 6, dtype, 0.125, uniform=True)
    one = attend_one(p, q, dtype, 0.125)
    assert bool((out[[1, 5]] == 0).all()) and bool((one[[1, 5]] == 0).all()) and moa.moa_device_status() == 0
    for b in (0, 2, 3, 4):
        new = [1 if i == b else 0 for i in range(6)]
        check_chunk(out[b:b + 1], p, q[b:b + 1], new, dtype, 0.125)
    with_starts = chunk(p, q, [1] * 6, dtype, 0.125)        # a token in a sequence without rows
    assert moa.moa_device_status() == moa.STATUS_SEQLEN_RANGE
    assert bool((with_starts[[1, 5]] == -3).all()) and torch.equal(with_starts[[0, 2, 3, 4]], out[[0, 2, 3, 4]])


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_many_sequences(fmt):
    rng = np.random.default_rng(9 + fmt)                    # several sequences to a thread of the plan
    new = rng.integers(0, 3, 1300).tolist()
    lens = [n + int(x) if n else int(x) for n, x in zip(new, rng.integers(0, 40, 1300))]
    p = Paged(rng, fmt, lens, 1, 64, 16)
    dtype = dtype_of(fmt)
    q = queries(rng, sum(new), 2, 64, dtype)
    out = chunk(p, q, new, dtype, 0.125)
    check_chunk(out, p, q, new, dtype, 0.125)
    assert moa.moa_device_status() == 0


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_refused_lengths_and_pages(fmt):
    rng = np.random.default_rng(13 + fmt)
    new, past = [20, 30, 25, 5], [100, 50, 0, 400]
    p = Paged(rng, fmt, [a + b for a, b in zip(new, past)], 2, 128, 16)
    dtype = dtype_of(fmt)
    q = queries(rng, sum(new), 4, 128, dtype)
    for wrong in (29, -5, p.max_pages * 16 + 1):
        lens = p.lens_dev.clone()
        lens[1] = wrong
        out = chunk(p, q, new, dtype, 0.1, lens=lens)
        assert moa.moa_device_status() == moa.STATUS_SEQLEN_RANGE
        assert bool((out[20:50] == -3).all())
        check_chunk(out, p, q, new, dtype, 0.1, skip=(1,))
    # a page that does not exist: rows 96..111 of sequence 0 (tokens of it at rows 100..119)
    for wrong in (-1, p.num_pages, 1 << 30):
        kept = int(p.table[0, 6])
        p.table[0, 6] = wrong
        out = chunk(p, q, new, dtype, 0.1)
        assert moa.moa_device_status() == moa.STATUS_PAGE_RANGE
        assert bool(torch.isnan(out[:20]).all())
        check_chunk(out, p, q, new, dtype, 0.1, skip=(0,))
        p.table[0, 6] = kept
        # only the last tokens see the last page
        kept = int(p.table[0, 7])
        p.table[0, 7] = wrong
        out = chunk(p, q, new, dtype, 0.1)
        assert moa.moa_device_status() == moa.STATUS_PAGE_RANGE
        assert bool(torch.isnan(out[12:20]).all()) and bool(torch.isfinite(out[:12]).all())
        p.table[0, 7] = kept


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_what_is_not_seen_does_not_touch(fmt):
    """Values that are not finite in rows behind a token's own."""
    rng = np.random.default_rng(19 + fmt)
    new, past, d = [60], [150], 128
    p = Paged(rng, fmt, [210], 2, d, 16)
    dtype = dtype_of(fmt)
    q = queries(rng, 60, 4, d, dtype)
    clean = chunk(p, q, new, dtype, 0.1)
    row = 150 + 33
    page = int(p.table_host[0, row // 16])
    if fmt == moa.KV_INT4:
        p.params["v"][page, 0, row % 16, 0] = float("nan")
        p.params["k"][page, 1, row % 16, 1] = float("nan")
    else:
        p.pools["v"][page, 0, row % 16, 11] = float("inf")
        p.pools["k"][page, 1, row % 16, 3] = float("nan")
    got = chunk(p, q, new, dtype, 0.1)
    assert torch.equal(got[:33], clean[:33])
    assert not bool(torch.isfinite(got[33:, :2, 11]).any()) and not bool(torch.isfinite(got[33:, 2:]).any())
    if fmt != moa.KV_INT4:
        others = [f for f in range(d) if f != 11]
        assert torch.equal(got[33:, :2][..., others], clean[33:, :2][..., others])


def test_value_rows_of_very_different_size():
    """4 bits: the scales of V span 2^-20..2^8 inside a sequence, small ones first, large ones first."""
    rng = np.random.default_rng(29)
    d, n = 128, 700
    grow = 2.0 ** np.linspace(-20, 8, n)
    v = [rng.standard_normal((1, n, d)) * grow[:, None], rng.standard_normal((1, n, d)) * grow[::-1, None]]
    k = [rng.standard_normal((1, n, d)) for _ in v]
    p = Paged(rng, moa.KV_INT4, [n] * 2, 1, d, 16, k=k, v=v)
    for dtype in (moa.BF16, moa.F16):
        q = queries(rng, 9, 8, d, dtype)
        check_chunk(chunk(p, q, [5, 4], dtype, 0.1), p, q, [5, 4], dtype, 0.1)


def test_pools_beyond_4_gib():
    """Pages whose offset passes 2^32 bytes, by tiled copies and row by row (an odd page size)."""
    for page in (32, 20):
        d, h_kv = 128, 8
        pages = (1 << 32) // (h_kv * page * d * 2) + 100
        pool = torch.zeros((pages, h_kv, page, d), dtype=torch.bfloat16, device="cuda")
        rng = np.random.default_rng(3)
        last = torch.arange(pages - 9, pages, dtype=torch.int32)
        pool[-9:] = torch.from_numpy(rng.standard_normal((9, h_kv, page, d)).astype(np.float32)).cuda().bfloat16()
        n = 9 * page - 3
        q = queries(rng, 7, 8, d, moa.BF16)
        cache = moa.PagedCache(moa.KV_BF16, pool, pool, pages, page, h_kv, d)
        out = torch.empty_like(q)
        ws = workspace(7, 8, h_kv, d, 1)
        moa.moa_paged_chunk_attn(cache, q, out, moa.BF16, 0, 7, 8, 1, starts_of([7]), torch.tensor([n], dtype=torch.int32).cuda(),
                                 last[None].contiguous().cuda(), 9, 0.1, *ws)
        rows = pool[-9:].double().cpu().numpy().transpose(1, 0, 2, 3).reshape(h_kv, -1, d)[:, :n]
        want, tol = attend_new64(q.double().cpu().numpy(), rows, rows, 0.1, moa.BF16)
        close(out, want, tol)
        assert moa.moa_device_status() == 0
        del pool, cache


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_graph_with_lengths_that_advance(fmt):
    rng = np.random.default_rng(37 + fmt)
    p = Paged(rng, fmt, [400, 300], 2, 64, 16)
    dtype = dtype_of(fmt)
    q = queries(rng, 8, 4, 64, dtype)
    wide = torch.zeros((8, 4 * 64 + 64), dtype=TYPES[dtype], device="cuda")      # queries with a stride between tokens
    wide[:, :256] = q.flatten(1)
    lens, ws = p.lens_dev.clone(), workspace(8, 4, 2, 64, 2)
    out = chunk(p, q, [4, 4], dtype, 0.1, lens=lens, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    starts = starts_of([4, 4])
    with torch.cuda.graph(g):
        moa.moa_paged_chunk_attn(p.cache, wide, out, dtype, 320, 8, 4, 2, starts, lens, p.table, p.max_pages, 0.1, *ws)
    for at in ([4, 4], [100, 5], [399, 300]):
        lens.copy_(torch.tensor(at, dtype=torch.int32))
        out.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        kept, p.lens = p.lens, at
        check_chunk(out, p, q, [4, 4], dtype, 0.1)
        p.lens = kept
    assert moa.moa_device_status() == 0
