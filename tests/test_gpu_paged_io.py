"""Appending to paged caches with the rotation on the way, reading rows back, and the operators together."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, attend, attend64, dtype_of, pack4, rope_table, rotate32, unpack4

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

FORMATS = [moa.KV_F32, moa.KV_BF16, moa.KV_F16, moa.KV_INT4]


def raw(x):
    return x.contiguous().view(-1).view(torch.uint8).cpu().numpy() if x.numel() else np.zeros(0, np.uint8)


def tensors(rng, tokens, h_q, h_kv, d, dtype):
    """q, k, v as slices of one [tokens, (h_q + 2 h_kv) * d] tensor, and their fp32 values."""
    wide = torch.from_numpy(rng.standard_normal((tokens, (h_q + 2 * h_kv) * d)).astype(np.float32)).cuda().to(TYPES[dtype])
    parts = [x.unflatten(-1, (-1, d)) if x.shape[-1] else x.reshape(tokens, 0, d) for x in wide.split([h_q * d, h_kv * d, h_kv * d], -1)]
    return wide, parts, [x.float().cpu().numpy() for x in parts]


def place(p, new):
    """(sequence, position) of every token of ragged `new` counts; lens are lengths with the new rows."""
    return [(b, p.lens[b] - n + i) for b, n in enumerate(new) for i in range(n)]


def expected(p, where, kf, vf, q32, cos_sin, rot, pairs, dtype):
    """Bytes of the pools (and the params) and of q_out after the append."""
    pos = np.array([x[1] for x in where])
    k, v = rotate32(kf, pos, cos_sin, rot, pairs), vf
    pools, params = {}, {}
    for name, x in (("k", k), ("v", v)):
        pool = p.pools[name].clone()
        par = p.params[name].clone() if p.fmt == moa.KV_INT4 else None
        pages = torch.tensor([int(p.table_host[b, i // p.page]) for b, i in where], device="cuda")
        offs = torch.tensor([i % p.page for _, i in where], device="cuda")
        if p.fmt == moa.KV_INT4:
            codes, pr = pack4(x)
            pool[pages, :, offs] = torch.from_numpy(codes).cuda()
            par[pages, :, offs] = torch.from_numpy(pr).cuda()
        else:
            pool[pages, :, offs] = torch.from_numpy(x).cuda().to(pool.dtype)
        pools[name], params[name] = pool, par
    q_out = torch.from_numpy(rotate32(q32, pos, cos_sin, rot, pairs)).cuda().to(TYPES[dtype])
    return pools, params, q_out


@pytest.mark.parametrize("rot,pairs", [(None, 0), (None, 1), (32, 0), (24, 0), (24, 1), (2, 0), (0, 0)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_append_bit_for_bit(fmt, d, rot, pairs):
    rot = d if rot is None else rot
    rng = np.random.default_rng(1000 * fmt + d + rot + pairs)
    for dtype in ([moa.BF16, moa.F16] if fmt == moa.KV_INT4 else [fmt]):
        for heads_inner, page, (h_q, h_kv) in ((False, 16, (6, 3)), (True, 7, (4, 1))):
            new = [1, 0, 40, 17, 5]
            p = Paged(rng, fmt, [a + b for a, b in zip(new, [0, 9, 30, 100, 3])], h_kv, d, page, heads_inner=heads_inner)
            tokens, pad = sum(new), 3                                        # rows behind the last sequence: left as they are
            wide, (q, k, v), (qf, kf, vf) = tensors(rng, tokens + pad, h_q, h_kv, d, dtype)
            table = rope_table(200, rot)
            where = place(p, new)
            pools, params, want_q = expected(p, where, kf[:tokens], vf[:tokens], qf[:tokens], table, rot, pairs, dtype)
            q_out = torch.full((tokens + pad, h_q, d), 9.0, dtype=TYPES[dtype], device="cuda")
            starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
            st = wide.shape[1]
            moa.moa_paged_append(p.cache, q, k, v, q_out, dtype, (st, st, st, h_q * d), tokens + pad, h_q, len(new), starts,
                                 p.lens_dev, p.table, p.max_pages, torch.from_numpy(table).cuda() if rot else None, 200, rot, pairs)
            torch.cuda.synchronize()
            assert moa.moa_device_status() == 0
            assert np.array_equal(raw(q_out[:tokens]), raw(want_q)) and bool((q_out[tokens:] == 9).all())
            for n in "kv":
                assert np.array_equal(raw(p.pools[n]), raw(pools[n])), n
                if fmt == moa.KV_INT4:
                    assert np.array_equal(raw(p.params[n]), raw(params[n])), n


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
@pytest.mark.parametrize("in_place", [False, True])
def test_one_token_each_without_starts_and_in_place(fmt, in_place):
    rng = np.random.default_rng(5 + fmt)
    for rot in (64, 20):
        p = Paged(rng, fmt, [5, 1, 33, 16], 2, 64, 16)
        dtype = dtype_of(fmt)
        wide, (q, k, v), (qf, kf, vf) = tensors(rng, 4, 4, 2, 64, dtype)
        table = rope_table(64, rot)
        pools, params, want_q = expected(p, place(p, [1] * 4), kf, vf, qf, table, rot, 0, dtype)
        st = wide.shape[1]
        q_out = q if in_place else torch.empty((4, 4, 64), dtype=TYPES[dtype], device="cuda")
        moa.moa_paged_append(p.cache, q, k, v, q_out, dtype, (st, st, st, st if in_place else 256), 4, 4, 4, None, p.lens_dev, p.table,
                             p.max_pages, torch.from_numpy(table).cuda(), 64, rot, moa.ROPE_HALVES)
        assert np.array_equal(raw(q_out), raw(want_q))
        assert all(np.array_equal(raw(p.pools[n]), raw(pools[n])) for n in "kv") and moa.moa_device_status() == 0


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_a_padded_batch_of_single_tokens(fmt):
    """Length 0 and no token starts: that token is left alone, without a status, and the attention gives zeros for it."""
    rng = np.random.default_rng(67 + fmt)
    p = Paged(rng, fmt, [9, 0, 40], 1, 128, 16)
    dtype = dtype_of(fmt)
    wide, (q, k, v), (qf, kf, vf) = tensors(rng, 3, 2, 1, 128, dtype)
    table = rope_table(64, 128)
    live = [0, 2]
    pools, params, want_q = expected(p, [(0, 8), (2, 39)], kf[live], vf[live], qf[live], table, 128, 0, dtype)
    q_out = torch.full((3, 2, 128), 9.0, dtype=TYPES[dtype], device="cuda")
    st = wide.shape[1]
    moa.moa_paged_append(p.cache, q, k, v, q_out, dtype, (st, st, st, 256), 3, 2, 3, None, p.lens_dev, p.table, p.max_pages,
                         torch.from_numpy(table).cuda(), 64, 128, 0)
    assert np.array_equal(raw(q_out[live]), raw(want_q)) and bool((q_out[1] == 9).all())
    assert all(np.array_equal(raw(p.pools[n]), raw(pools[n])) for n in "kv")
    assert bool((attend(p, q_out, dtype, 0.1)[1] == 0).all()) and moa.moa_device_status() == 0


def test_many_tokens_and_no_queries():
    rng = np.random.default_rng(11)
    for fmt in FORMATS:
        dtype = dtype_of(fmt, moa.F16)
        p = Paged(rng, fmt, [2500, 1300], 4, 128, 64)
        for h_q in (12, 0):
            wide, (q, k, v), (qf, kf, vf) = tensors(rng, 3800, h_q, 4, 128, dtype)
            table = rope_table(2500, 128)
            pools, params, want_q = expected(p, place(p, [2500, 1300]), kf, vf, qf, table, 128, 0, dtype)
            q_out = torch.zeros((3800, h_q, 128), dtype=TYPES[dtype], device="cuda")
            st = wide.shape[1]
            moa.moa_paged_append(p.cache, q if h_q else None, k, v, q_out if h_q else None, dtype, (st, st, st, h_q * 128), 3800, h_q, 2,
                                 torch.tensor([0, 2500, 3800], dtype=torch.int32, device="cuda"), p.lens_dev, p.table, p.max_pages,
                                 torch.from_numpy(table).cuda(), 2500, 128, 0)
            assert np.array_equal(raw(q_out), raw(want_q))
            assert all(np.array_equal(raw(p.pools[n]), raw(pools[n])) for n in "kv") and moa.moa_device_status() == 0


def test_rows_that_4_bits_hold_badly():
    """Equal values, tiny and huge ranges, values beyond fp16, NaN and infinities: the formulas, and NaN where a row has no number."""
    rng = np.random.default_rng(13)
    rows = rng.standard_normal((12, 1, 64)).astype(np.float32)
    rows[0] = 3.25
    rows[1] = 0
    rows[2] *= 1e-9
    rows[3] *= 1e-4
    rows[4] *= 3e4
    rows[5] = 1e30 * rows[5]
    rows[6, 0, 5] = np.nan
    rows[7, 0, 63] = np.inf
    rows[8, 0, 0] = -np.inf
    rows[9] = 1000 + 1e-3 * rows[9]
    rows[10, 0, 1:] = 0
    x = torch.from_numpy(rows).cuda().bfloat16()
    vals = x.float().cpu().numpy()
    p = Paged(rng, moa.KV_INT4, [12], 1, 64, 8)
    moa.moa_paged_append(p.cache, None, x, x, None, moa.BF16, None, 12, 0, 1, torch.tensor([0, 12], dtype=torch.int32, device="cuda"),
                         p.lens_dev, p.table, p.max_pages, None, 0, 0, 0)
    codes, params = pack4(vals)
    k = torch.full((1, 1, 12, 64), 7.0, device="cuda")
    v = k.clone()
    moa.moa_paged_gather(p.cache, k, v, moa.F32, 1, 12, None, p.lens_dev, p.table, p.max_pages)
    want = unpack4(codes, params)[:, 0]
    got = k[0, 0].double().cpu().numpy()
    assert np.array_equal(np.isnan(got).all(-1), [i in (6, 7, 8) for i in range(12)])
    fine = ~np.isnan(want)
    assert np.all(np.abs(got - want)[fine] <= np.abs(want)[fine] * 2.0 ** -24 + 1e-45) and torch.equal(k.nan_to_num(), v.nan_to_num())
    # inside fp16's range: half a step, and fp16's rounding of the pair (row 4 reaches 7.3e4 in size, beyond it)
    ok = [i for i in (0, 1, 3, 4, 9, 11) if np.abs(vals[i]).max() <= 65504]
    step = (vals.max(-1) - vals.min(-1)) / 15
    off = np.abs(got - vals[:, 0])
    # half a code, scale's rounding on 15 codes (and 2^-25), least's rounding where it lies above the smallest value
    tol = step * (0.5 + 15 * 2.0 ** -11) + np.abs(vals[:, 0]).max(-1, keepdims=True) * 2.0 ** -11 + 16 * 2.0 ** -25
    assert np.all(off[ok] <= tol[ok])


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_tokens_that_cannot_be_placed(fmt):
    rng = np.random.default_rng(17 + fmt)
    p = Paged(rng, fmt, [20, 30, 40, 5], 1, 64, 16)
    dtype = dtype_of(fmt)
    wide, (q, k, v), (qf, kf, vf) = tensors(rng, 8, 2, 1, 64, dtype)
    st = wide.shape[1]
    table = torch.from_numpy(rope_table(39, 64)).cuda()                      # no row for position 39

    def call(lens, tab, starts=(0, 2, 4, 6, 8)):
        q_out = torch.full((8, 2, 64), 9.0, dtype=TYPES[dtype], device="cuda")
        moa.moa_paged_append(p.cache, q, k, v, q_out, dtype, (st, st, st, 128), 8, 2, 4, torch.tensor(starts, dtype=torch.int32, device="cuda"),
                             torch.tensor(lens, dtype=torch.int32, device="cuda"), tab, p.max_pages, table, 39, 64, 0)
        return (q_out == 9).all(-1).all(-1).cpu().tolist()

    assert call([20, 30, 40, 5], p.table) == [False] * 5 + [True] + [False] * 2
    assert moa.moa_device_status() == moa.STATUS_APPEND_RANGE
    assert call([1, p.max_pages * 16 + 1, -5, 2], p.table) == [True, False, True, True, True, True, False, False]
    assert moa.moa_device_status() == moa.STATUS_APPEND_RANGE
    bad = p.table.clone()
    bad[0, 1], bad[1, 1] = p.num_pages, -1
    assert call([20, 30, 38, 5], bad) == [True] * 4 + [False] * 4
    assert moa.moa_device_status() == moa.STATUS_PAGE_RANGE
    assert call([20, 30, 38, 5], p.table, starts=(0, 0, 0, 0, 0)) == [True] * 8 and moa.moa_device_status() == 0


@pytest.mark.parametrize("dtype", [moa.F32, moa.BF16, moa.F16])
@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_gather(fmt, dtype):
    rng = np.random.default_rng(19 + fmt + dtype)
    lens, first = [100, 1, 0, 47, 64], [30, 0, 0, 47, 63]
    for d, heads_inner, page in ((128, False, 16), (64, True, 12)):
        p = Paged(rng, fmt, lens, 3, d, page, heads_inner=heads_inner)
        for start in (None, first):
            n_out = 100 if start is None else 70
            k = torch.full((5, 3, n_out, d), 9.0, dtype=TYPES[dtype], device="cuda")
            v = k.clone()
            moa.moa_paged_gather(p.cache, k, v, dtype, 5, n_out, None if start is None else torch.tensor(start, dtype=torch.int32, device="cuda"),
                                 p.lens_dev, p.table, p.max_pages)
            torch.cuda.synchronize()
            assert moa.moa_device_status() == 0
            for b in range(5):
                lo = 0 if start is None else start[b]
                for name, got in (("k", k), ("v", v)):
                    n = lens[b] - lo
                    want = torch.from_numpy(p.rows(name, b)[:, lo:].astype(np.float32)).cuda().to(TYPES[dtype])
                    assert torch.equal(got[b, :, :n], want), (b, name)
                    assert bool((got[b, :, n:] == 9).all())


def test_gather_out_of_range():
    rng = np.random.default_rng(29)
    p = Paged(rng, moa.KV_F16, [40, 40, 40, 40], 1, 64, 16)
    k = torch.full((4, 1, 40, 64), 9.0, device="cuda")
    v = k.clone()
    start = torch.tensor([-1, 0, 41, 0], dtype=torch.int32, device="cuda")
    lens = torch.tensor([40, 41, 40, 40], dtype=torch.int32, device="cuda")
    moa.moa_paged_gather(p.cache, k, v, moa.F32, 4, 40, start, lens, p.table, p.max_pages)
    assert moa.moa_device_status() == moa.STATUS_SEQLEN_RANGE
    assert bool((k[:3] == 9).all()) and not bool((k[3] == 9).all(-1).any())
    p.table[3, 1] = p.num_pages
    k.fill_(9)
    moa.moa_paged_gather(p.cache, k, v, moa.F32, 4, 40, None, p.lens_dev, p.table, p.max_pages)
    assert moa.moa_device_status() == moa.STATUS_PAGE_RANGE
    assert bool((k[3, 0, 16:32] == 9).all()) and not bool((k[3, 0, :16] == 9).all(-1).any())


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_prompt_then_tokens(fmt):
    """As a serving program uses them: prompts appended, then steps of append and attention in a captured graph, the lengths
    advanced on the device; every step's output against the definition on the rows as the cache holds them."""
    rng = np.random.default_rng(37 + fmt)
    h_q, h_kv, d, page, steps = 8, 2, 128, 16, 5
    prompts = [33, 1, 80]
    p = Paged(rng, fmt, [n + steps for n in prompts], h_kv, d, page)
    for n in "kv":
        p.pools[n].fill_(0 if fmt == moa.KV_INT4 else float("nan"))
    dtype = dtype_of(fmt)
    rows = torch.from_numpy(rope_table(128, d)).cuda()
    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 33, 34, 114], dtype=torch.int32, device="cuda")
    wide, (q, k, v), (qf, kf, vf) = tensors(rng, 114, h_q, h_kv, d, dtype)
    st = wide.shape[1]
    q_out = torch.empty((114, h_q, d), dtype=TYPES[dtype], device="cuda")
    moa.moa_paged_append(p.cache, q, k, v, q_out, dtype, (st, st, st, h_q * d), 114, h_q, 3, starts, lens, p.table, p.max_pages, rows, 128, d, 0)
    step_in = [tensors(rng, 3, h_q, h_kv, d, dtype) for _ in range(steps)]
    wide1 = torch.empty_like(step_in[0][0])
    q1, k1, v1 = (x.unflatten(-1, (-1, d)) for x in wide1.split([h_q * d, h_kv * d, h_kv * d], -1))
    turned = torch.empty((3, h_q, d), dtype=TYPES[dtype], device="cuda")
    out = torch.empty_like(turned)
    n_ws = moa.moa_paged_workspace_bytes(3, h_q, h_kv, d)
    ws = torch.empty(n_ws, dtype=torch.uint8, device="cuda")

    def step():
        moa.moa_lens_add(lens, 3, 1)
        moa.moa_paged_append(p.cache, q1, k1, v1, turned, dtype, (st, st, st, h_q * d), 3, h_q, 3, None, lens, p.table, p.max_pages, rows, 128, d, 0)
        moa.moa_paged_decode_attn(p.cache, turned, out, dtype, 0, 3, h_q, lens, p.table, p.max_pages, d ** -0.5, ws, n_ws)

    saved = {n: p.pools[n].clone() for n in "kv"}
    wide1.copy_(step_in[0][0])
    step()
    lens.copy_(torch.tensor(prompts, dtype=torch.int32))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in "kv":
        p.pools[n].copy_(saved[n])
    rope = rows.cpu().numpy()
    full = {name: [rotate32(x[a:b], np.arange(b - a), rope, d if name == "k" else 0, 0) for a, b in ((0, 33), (33, 34), (34, 114))]
            for name, x in (("k", kf), ("v", vf))}
    for i in range(steps):
        wide1.copy_(step_in[i][0])
        graph.replay()
        torch.cuda.synchronize()
        assert moa.moa_device_status() == 0
        now = [n + i + 1 for n in prompts]
        assert lens.cpu().tolist() == now
        for b in range(3):
            for name, x, rot in (("k", step_in[i][2][1], d), ("v", step_in[i][2][2], 0)):
                full[name][b] = np.concatenate([full[name][b], rotate32(x[b:b + 1], np.array([now[b] - 1]), rope, rot, 0)])

        class Held:                                                          # the rows as the cache holds them
            pass
        held = Held()
        held.fmt, held.h_kv, held.lens = fmt, h_kv, now

        def rows64(name, b, n):
            x = full[name][b].transpose(1, 0, 2)
            return unpack4(*pack4(x)) if fmt == moa.KV_INT4 else torch.from_numpy(x).to(TYPES[fmt]).double().numpy()
        held.rows = rows64
        want, bound = attend64(turned.double().cpu().numpy(), held, d ** -0.5)
        if fmt == moa.KV_F32:
            bound = np.maximum(bound, 5e-6)
        off = np.abs(out.double().cpu().numpy() - want)
        assert np.all(off <= bound + np.abs(want) * torch.finfo(out.dtype).eps / 2 + 2.0 ** -25), (i, float(off.max()))


@pytest.mark.parametrize("h_q,h_kv,d", [(8, 2, 128), (16, 2, 64), (4, 4, 128)])
def test_the_dense_calls_take_what_is_read_back(h_q, h_kv, d):
    """moa_paged_gather in fp32 gives the cache of moa_decode_attn_varlen; both attentions agree on it."""
    rng = np.random.default_rng(61 + d)
    lens = [700, 33, 1]
    for fmt in FORMATS:
        p = Paged(rng, fmt, lens, h_kv, d, 16)
        dtype = dtype_of(fmt, moa.F16)
        q = torch.from_numpy(rng.standard_normal((3, h_q, d)).astype(np.float32)).cuda().to(TYPES[dtype])
        K = torch.zeros((3, h_kv, 700, d), device="cuda")
        V = torch.zeros_like(K)
        moa.moa_paged_gather(p.cache, K, V, moa.F32, 3, 700, None, p.lens_dev, p.table, p.max_pages)
        dense = torch.empty((3, h_q, d), device="cuda")
        n = moa.moa_workspace_bytes(3, h_q, h_kv, 700, d, d)
        moa.moa_decode_attn_varlen(q.float(), K, V, dense, 3, h_q, h_kv, p.lens_dev, 700, d, d, 0.1, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
        paged = attend(p, q, dtype, 0.1)
        want, bound = attend64(q.double().cpu().numpy(), p, 0.1)
        off = (paged.double() - dense.double()).abs().cpu().numpy()
        assert np.all(off <= np.maximum(bound, 5e-6) + 5e-6 + np.abs(want) * torch.finfo(paged.dtype).eps / 2 + 2.0 ** -25)
