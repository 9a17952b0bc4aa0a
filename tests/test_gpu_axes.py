"""Positions with several axes: queries and keys turned bit for bit, into tensors and into caches, and a run of the calls together."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, attend, dtype_of, rope_table
from paged_util import workspace as decode_workspace
from prompt_util import attend_new64, check_chunk, check_prompt, chunk, prompt, starts_of

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

FORMATS = [moa.KV_F32, moa.KV_BF16, moa.KV_F16, moa.KV_INT4]


def turned(x, positions, axis_map, cos_sin, rot, pairs):
    """x fp32 [tokens, heads, d], every operation rounded to fp32; pair i by positions[axis_map[i]]."""
    y = x.astype(np.float32).copy()
    for i in range(rot // 2):
        at = positions[axis_map[i]]
        c, s = cos_sin[at, i][:, None], cos_sin[at, rot // 2 + i][:, None]
        lo, hi = (2 * i, 2 * i + 1) if pairs else (i, rot // 2 + i)
        a, b = y[..., lo].copy(), y[..., hi].copy()
        y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    return y


def axis_map(rng, axes, pairs, kind):
    if kind == "runs":
        return np.sort(rng.integers(0, axes, pairs)).astype(np.uint8)
    return (np.arange(pairs) % axes).astype(np.uint8) if kind == "turns" else rng.integers(0, axes, pairs).astype(np.uint8)


@pytest.mark.parametrize("rot,pairs", [(None, 0), (None, 1), (32, 0), (24, 0), (24, 1), (2, 0)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [moa.F32, moa.BF16, moa.F16], ids=["f32", "bf16", "f16"])
def test_rotate_bit_for_bit(dtype, d, rot, pairs):
    rot = d if rot is None else rot
    rng = np.random.default_rng(dtype + d + rot + pairs)
    for axes, kind, tokens, h_q, h_kv in ((1, "runs", 5, 3, 1), (3, "runs", 700, 8, 8), (3, "turns", 37, 7, 2), (4, "any", 1, 2, 0), (2, "any", 9000, 0, 3)):
        table = rope_table(300, rot)
        amap, pos = axis_map(rng, axes, rot // 2, kind), rng.integers(0, 300, (axes, tokens)).astype(np.int32)
        wide = torch.from_numpy(rng.standard_normal((tokens, (h_q + h_kv + 1) * d)).astype(np.float32)).cuda().to(TYPES[dtype])
        parts = [x.unflatten(-1, (-1, d)) if x.shape[-1] else None for x in wide.split([h_q * d, h_kv * d, d], -1)[:2]]
        outs = [None if x is None else torch.full_like(x.contiguous(), 9.0) for x in parts]
        w = wide.shape[1]
        args = (dtype, (w, w, h_q * d, h_kv * d), tokens, h_q, h_kv, d, torch.from_numpy(pos).cuda(), axes, amap.tobytes(), torch.from_numpy(table).cuda(), 300,
                rot, moa.ROPE_PAIRS if pairs else moa.ROPE_HALVES)
        moa.moa_rotate_axes(parts[0], parts[1], outs[0], outs[1], *args)
        for x, y in zip(parts, outs):
            if x is not None:
                want = torch.from_numpy(turned(x.float().cpu().numpy(), pos, amap, table, rot, pairs)).cuda().to(TYPES[dtype])
                assert torch.equal(y, want), (axes, kind)
        # in place
        moa.moa_rotate_axes(parts[0], parts[1], parts[0], parts[1], dtype, (w, w, w, w), *args[2:])
        for x, y in zip(parts, outs):
            assert x is None or torch.equal(x, y)
    assert moa.moa_device_status() == 0


@pytest.mark.parametrize("style", [moa.ROPE_HALVES, moa.ROPE_PAIRS])
@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_append_is_the_append_of_turned_rows(fmt, style):
    """The pools after moa_paged_append_axes hold, bit for bit, what an append without rotation of rows turned beforehand in fp32 holds;
    with every axis at the row's number, what moa_paged_append stores."""
    rng = np.random.default_rng(fmt + 10 * style)
    new, past, h_q, h_kv, d, rot = [1, 0, 30, 6], [5, 9, 70, 0], 4, 2, 64, 48
    tokens = sum(new)
    for dtype in ([moa.BF16, moa.F16] if fmt == moa.KV_INT4 else [fmt]):
        rows = np.concatenate([np.arange(a, a + n) for n, a in zip(new, past)]).astype(np.int32)
        table = torch.from_numpy(rope_table(200, rot)).cuda()
        q, k, v = (torch.from_numpy(rng.standard_normal((tokens, h, d)).astype(np.float32)).cuda().to(TYPES[dtype]) for h in (h_q, h_kv, h_kv))

        def appended(positions, amap):
            p = Paged(np.random.default_rng(1), fmt, [a + b for a, b in zip(new, past)], h_kv, d, 16)
            q_out = torch.full_like(q, 5.0)
            common = (None, tokens, h_q, 4, starts_of(new), p.lens_dev, p.table, p.max_pages)
            if positions is None:
                moa.moa_paged_append(p.cache, q, k, v, q_out, dtype, *common, table, 200, rot, style)
            else:
                moa.moa_paged_append_axes(p.cache, q, k, v, q_out, dtype, *common, torch.from_numpy(positions).cuda(), len(positions), amap, table, 200, rot, style)
            torch.cuda.synchronize()
            assert moa.moa_device_status() == 0
            return p, [q_out] + [x.contiguous().view(torch.uint8) for x in (*p.pools.values(), *p.params.values())]

        _, plain = appended(None, None)
        _, same = appended(np.stack([rows] * 3), bytes(i % 3 for i in range(rot // 2)))
        for a, b in zip(plain, same):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        pos, amap = rng.integers(0, 200, (3, tokens)).astype(np.int32), axis_map(rng, 3, rot // 2, "any")
        p, got = appended(pos, amap.tobytes())
        want_q = torch.from_numpy(turned(q.float().cpu().numpy(), pos, amap, rope_table(200, rot), rot, style == moa.ROPE_PAIRS)).cuda().to(TYPES[dtype])
        assert torch.equal(got[0], want_q)
        if fmt != moa.KV_INT4:
            want_k = torch.from_numpy(turned(k.float().cpu().numpy(), pos, amap, rope_table(200, rot), rot, style == moa.ROPE_PAIRS)).cuda().to(TYPES[dtype])
            at = 0
            for b, n in enumerate(new):
                for i in range(n):
                    page, off = int(p.table_host[b, (past[b] + i) // 16]), (past[b] + i) % 16
                    assert torch.equal(p.pools["k"][page, :, off], want_k[at]) and torch.equal(p.pools["v"][page, :, off], v[at])
                    at += 1


def test_positions_out_of_range():
    """The token is left as it was, in whichever axis the position lies outside; its neighbours are not touched."""
    rng = np.random.default_rng(3)
    tokens, d = 40, 64
    table = torch.from_numpy(rope_table(50, d)).cuda()
    q = torch.from_numpy(rng.standard_normal((tokens, 2, d)).astype(np.float32)).cuda()
    pos = rng.integers(0, 50, (3, tokens)).astype(np.int32)
    amap = bytes(i % 3 for i in range(d // 2))
    want, out = torch.empty_like(q), torch.full_like(q, 4.0)
    moa.moa_rotate_axes(q, None, want, None, moa.F32, None, tokens, 2, 0, d, torch.from_numpy(pos).cuda(), 3, amap, table, 50, d, 0)
    assert moa.moa_device_status() == 0
    pos[1, 7], pos[2, 30], pos[0, 39] = 50, -1, 1 << 30
    moa.moa_rotate_axes(q, None, out, None, moa.F32, None, tokens, 2, 0, d, torch.from_numpy(pos).cuda(), 3, amap, table, 50, d, 0)
    assert moa.moa_device_status() == moa.STATUS_APPEND_RANGE
    left = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    left[[7, 30, 39]] = True
    assert bool((out[left] == 4).all()) and torch.equal(out[~left], want[~left])


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_prompt_then_pieces_then_a_token(fmt):
    """A prompt turned and attended to without a cache; then the same tokens appended to a cache in two pieces with attention after each, and one
    token more by the single-query call: each against the definition on what the cache holds, without a wait in between."""
    rng = np.random.default_rng(51 + fmt)
    h_q, h_kv, d, page = 8, 2, 64, 16
    dtype = dtype_of(fmt)
    sizes = ([90, 41], [60, 7], [1, 1])                     # a first piece, a second, a token
    total = [sum(x) for x in zip(*sizes)]
    p = Paged(rng, fmt, total, h_kv, d, page)
    table = torch.from_numpy(rope_table(400, d)).cuda()
    amap = bytes([0] * 16 + [1] * 8 + [2] * 8)
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = []
    for new in sizes:
        tokens = sum(new)
        q, k, v = (torch.from_numpy(rng.standard_normal((tokens, h, d)).astype(np.float32)).cuda().to(TYPES[dtype]) for h in (h_q, h_kv, h_kv))
        pos = torch.from_numpy(rng.integers(0, 400, (3, tokens)).astype(np.int32)).cuda()
        lens += torch.tensor(new, dtype=torch.int32, device="cuda")
        turned_q = torch.empty_like(q)
        moa.moa_paged_append_axes(p.cache, q, k, v, turned_q, dtype, None, tokens, h_q, 2, starts_of(new), lens, p.table, p.max_pages, pos, 3, amap, table, 400, d,
                                  moa.ROPE_HALVES)
        out = attend(p, turned_q, dtype, 0.2, lens=lens) if new == [1, 1] else chunk(p, turned_q, new, dtype, 0.2, lens=lens)
        kept.append((new, lens.tolist(), turned_q, out, (q, k, v, pos)))
    assert moa.moa_device_status() == 0
    # what the cache holds now, read back
    n = max(total)
    back = [torch.zeros((2, h_kv, n, d), device="cuda") for _ in "kv"]
    moa.moa_paged_gather(p.cache, back[0], back[1], moa.F32, 2, n, None, lens, p.table, p.max_pages)
    rows = [x.double().cpu().numpy() for x in back]
    for new, at, q, out, _ in kept:
        x, got, t = q.double().cpu().numpy(), out.double().cpu().numpy(), 0
        for b, m in enumerate(new):
            k, v = rows[0][b, :, :at[b]], rows[1][b, :, :at[b]]
            steps = (v.max(-1) - v.min(-1)) / 15 if fmt == moa.KV_INT4 else None
            want, tol = attend_new64(x[t:t + m], k, v, 0.2, dtype, steps4=steps)
            if fmt == moa.KV_INT4:                          # (the single-query call rounds weights to fp16)
                tol = tol + 2.0 ** -11 * np.abs(v).max()
            assert np.all(np.abs(got[t:t + m] - want) <= tol), (new, b)
            t += m
    # the first piece without a cache
    if fmt != moa.KV_INT4:
        new, _, turned_q, out, (q, k, v, pos) = kept[0]
        qkv = torch.cat([q, k, v], 1).flatten(1)
        wide = qkv.shape[1]
        qs, ks, _ = (y.unflatten(-1, (-1, d)) for y in qkv.split([h_q * d, h_kv * d, h_kv * d], -1))
        moa.moa_rotate_axes(qs, ks, qs, ks, dtype, (wide, wide, wide, wide), sum(new), h_q, h_kv, d, pos, 3, amap, table, 400, d, moa.ROPE_HALVES)
        assert torch.equal(qs, turned_q)
        dense = prompt(qkv, h_q, h_kv, d, new, dtype, True, 0.2)
        check_prompt(dense, qkv, h_q, h_kv, d, new, dtype, True, 0.2)
