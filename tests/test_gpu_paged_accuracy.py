"""Attention over paged caches where the sums are hard.

Scores here come from one feature of q (the others are 0), so that they carry a few fp32 roundings and no more, and the
bounds are those of the weights and sums alone."""
import contextlib

import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, attend, attend64, dtype_of, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@contextlib.contextmanager
def one_cta():
    moa.moa_set_option(moa.OPT_NUM_CTAS, 1)
    try:
        yield
    finally:
        moa.moa_set_option(moa.OPT_NUM_CTAS, 0)


def one_feature(batch, h_q, d, dtype, size=1.0):
    q = torch.zeros((batch, h_q, d), dtype=TYPES[dtype], device="cuda")
    q[:, :, 0] = size
    return q


@pytest.mark.parametrize("nats", [12.0, 15.0, 17.5])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt,dtype", [(f, dtype_of(f, t)) for f, t in ((0, 0), (1, 1), (2, 2), (3, moa.BF16), (3, moa.F16))],
                         ids=["f32", "bf16", "f16", "int4-bf16", "int4-f16"])
def test_many_light_rows_beside_a_heavy_one(fmt, dtype, d, nats):
    """One row carries nearly all weight and holds zeros; what is left is the sum of 4096 rows `nats` lower."""
    rng = np.random.default_rng(3)
    n, batch = 4097, 16
    k = [np.zeros((1, n, d), np.float32) for _ in range(batch)]
    v = [rng.uniform(1, 2, (1, n, d)).astype(np.float32) for _ in range(batch)]
    for b in range(batch):
        heavy = [0, n - 1, 2000][b % 3]
        k[b][0, :, 0], k[b][0, heavy, 0] = -nats, 0
        v[b][0, heavy] = 0
    p = Paged(rng, fmt, [n] * batch, 1, d, 16, k=k, v=v)
    q = one_feature(batch, 3, d, dtype)
    with one_cta():
        out = attend(p, q, dtype, 1.0)
    assert moa.moa_device_status() == 0
    want, _ = attend64(q.double().cpu().numpy(), p, 1.0)
    # Relative: the sum of a lane's 512 probabilities 2^-15, the sum over 256 stages 2^-16, two-term weights 2^-17, scores of
    # 25 (log2) with three roundings and exp2 2^-17: below 2^-14 together; one-term fp16 weights of 4-bit rows 2^-12 of what
    # the rows span, which is less than they are.  Weights in fp16 end at 2^-25 of 2^11 times a row's: 2^-36 and less lost of
    # each (V at most 2; 4 bits: of 8 steps, the scale's power of two 2^-3).  The output's rounding, 2^-25 among fp16's subnormals.
    rel = 2.0 ** -14 + (2.0 ** -12 if fmt == moa.KV_INT4 else 0)
    tol = want * (rel + torch.finfo(out.dtype).eps / 2) + n * 2.0 ** -35 + 2.0 ** -25
    off = np.abs(out.double().cpu().numpy() - want)
    assert np.all(off <= tol), (float(off.max()), float((off / tol).max()))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", [moa.KV_F32, moa.KV_BF16, moa.KV_F16, moa.KV_INT4], ids=lambda f: NAMES[f])
def test_long_sums_of_one_sign(fmt, d):
    """131072 rows of positive values and nearly even weights in one warp's sums: no bias but that of fp32 additions.
    All sequences name the same few pages again and again."""
    rng = np.random.default_rng(5)
    n, page, pages, batch = 131072, 64, 3, 12
    dtype = dtype_of(fmt, moa.F16)
    k = rng.uniform(-1, 1, (1, page * pages, d)).astype(np.float32)
    v = rng.uniform(1, 2, (1, page * pages, d)).astype(np.float32)
    p = Paged(rng, fmt, [page * pages], 1, d, page, k=[k], v=[v])
    own = p.table_host[0, :pages]
    order = own[rng.integers(0, pages, (batch, n // page))].astype(np.int32)
    lens = torch.full((batch,), n, dtype=torch.int32, device="cuda")
    q = one_feature(batch, 2, d, dtype)
    out = torch.empty((batch, 2, d), dtype=TYPES[dtype], device="cuda")
    ws, size = workspace(batch, 2, 1, d)
    with one_cta():
        moa.moa_paged_decode_attn(p.cache, q, out, dtype, 0, batch, 2, lens, torch.from_numpy(order).cuda(), n // page, 0.5, ws, size)
    assert moa.moa_device_status() == 0
    got = out.double().cpu().numpy()
    for b in range(batch):
        w = np.exp(0.5 * p.values["k"][order[b], 0, :, 0].reshape(-1))
        want = (w / w.sum()) @ p.values["v"][order[b], 0].reshape(-1, d)
        # The rows repeat, so the roundings of a sum's additions may repeat too and all have one sign: N additions of equal parts, each
        # off by half a unit in the last place of the sum so far, are off by N * 2^-25 of the whole sum.  N is the stages of 16 rows
        # (32 for rows of 64 in 16 bits and for 4 bits): 2^13 in the weighted sum and as many in the sum of probabilities, 2^-11
        # in all, 2^-12 for stages of 32; in 4 bits the sum of probabilities goes row by row (2^14 additions in a lane, 2^-11) and
        # the weights have one rounding (2^-12 of either sign, 192 different rows of a span of less than 1: 2^-14).  Products and sums within a stage 2^-16.
        stage = 32 if fmt == moa.KV_INT4 or (d == 64 and fmt in (moa.KV_BF16, moa.KV_F16)) else 16
        rel = (2 if fmt != moa.KV_INT4 else 5) * (n // stage) * 2.0 ** -25 + 2.0 ** -16 + (2.0 ** -14 if fmt == moa.KV_INT4 else 0)
        tol = np.abs(want) * (torch.finfo(out.dtype).eps / 2 + rel)
        off = np.abs(got[b] - want)
        assert np.all(off <= tol), (b, float((off / want).max()), float((off / tol).max()))


def rowwise64(p, b, q0, scale, terms):
    """Definition and bound of sequence b (one kv head, one-feature queries of size q0) on a 4-bit cache: weights in fp16 in `terms` terms,
    relative to each row's own span, and what fp16's least positive value takes off each of them."""
    k, v = p.rows("k", b)[0], p.rows("v", b)[0]
    s = scale * q0 * k[:, 0]
    w = np.exp(s - s.max())
    w /= w.sum()
    span, top = v.max(-1) - v.min(-1), np.abs(v).max(-1)
    # scores: four roundings of parts below 2^5 in log2, twice 2^-17; probabilities and their sums 2^-16; a stage's codes in the
    # MMA's accumulation 2^-18 of eight steps each
    bound = (w * (top * 2.0 ** -15 + span * (2.0 ** -12 if terms == 1 else 2.0 ** -18))).sum() + len(w) * 2.0 ** -32 * span.max() / 15
    return w @ v, bound


@pytest.mark.parametrize("n", [2, 3, 7, 40])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("h_q", [4, 16])
def test_few_rows_in_4_bits(n, d, h_q):
    """fp16 outputs of a 4-bit cache are rounded once: the weights of a few heavy rows do not add a rounding of their own."""
    rng = np.random.default_rng(n + d)
    batch = 24
    v = [rng.standard_normal((1, n, d)) for _ in range(batch)]
    k = [np.clip(rng.standard_normal((1, n, d)), -2, 2) for _ in range(batch)]
    p = Paged(rng, moa.KV_INT4, [n] * batch, 1, d, 16, k=k, v=v)
    q = one_feature(batch, h_q, d, moa.F16)
    out = attend(p, q, moa.F16, 0.7).double().cpu().numpy()
    for b in range(batch):
        want, bound = rowwise64(p, b, 1.0, 0.7, 2)
        tol = bound + np.abs(want) * 2.0 ** -11 + 2.0 ** -25
        off = np.abs(out[b] - want)
        assert np.all(off <= tol), (b, float(off.max()), float((off / tol).max()))


@pytest.mark.parametrize("size", [1e-38, 2.0 ** 115, 2.0 ** 116, 1e36, 3.3e38])
def test_queries_at_the_ends_of_bf16(size):
    """4 bits: a query's largest value is brought to 2^13 whatever it is; the product of queries and scale is an ordinary one."""
    rng = np.random.default_rng(31)
    d = 128
    p = Paged(rng, moa.KV_INT4, [90, 5, 300], 1, d, 16)
    q = rng.uniform(-1, 1, (3, 3, d))
    q[:, :, 7] = [1, -1, 0.9]
    qd = (torch.from_numpy(q) * size).cuda().bfloat16()
    scale = float(np.float32(0.25 / size))
    out = attend(p, qd, moa.BF16, scale)
    want, bound = attend64(qd.double().cpu().numpy(), p, scale)
    # scale * log2(e) among fp32's subnormals (below 2^-126) has a rounding of 2^-150 of its own: twice that, relative to the scale, of scores of
    # 300 at most, acting on weights
    extra = 300 * 2.0 ** -149 / scale * np.abs(p.values["v"][np.isfinite(p.values["v"])]).max()
    off = np.abs(out.double().cpu().numpy() - want)
    tol = bound + extra + np.abs(want) * 2.0 ** -8 + 2.0 ** -25
    assert np.all(off <= tol), (float(off.max()), float((off / tol).max()))


@pytest.mark.parametrize("dtype", [moa.BF16, moa.F16])
@pytest.mark.parametrize("ratio", [2.0 ** 8, 2.0 ** 14])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_a_light_row_of_large_scale_in_4_bits(where, ratio, dtype):
    """A row `ratio` times as large as the others, with a weight of e^-60: before, among and after them, it takes nothing from the others'."""
    rng = np.random.default_rng(11)
    d, n, batch = 128, 700, 6
    at = {"first": 0, "middle": 333, "last": n - 1}[where]
    k, v = [], []
    for b in range(batch):
        kb = np.clip(rng.standard_normal((1, n, d)), -2, 2)
        vb = rng.standard_normal((1, n, d)) * 2.0 ** -6
        kb[0, at, 0] = -60
        vb[0, at] *= ratio
        k.append(kb)
        v.append(vb)
    p = Paged(rng, moa.KV_INT4, [n] * batch, 1, d, 16, k=k, v=v)
    q = one_feature(batch, 5, d, dtype)
    with one_cta():
        out = attend(p, q, dtype, 1.0)
    got = out.double().cpu().numpy()
    for b in range(batch):
        want, bound = rowwise64(p, b, 1.0, 1.0, 1)
        tol = bound + np.abs(want) * torch.finfo(out.dtype).eps / 2 + 2.0 ** -25
        off = np.abs(got[b] - want)
        assert np.all(off <= tol), (b, float(off.max()), float((off / tol).max()))


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("fmt", range(4), ids=lambda f: NAMES[f])
def test_values_that_are_not_finite_stay_where_they_are(fmt, value):
    """In V: the feature they stand in (the row, in 4 bits) of the heads of that K/V head is not finite; everything else of the sequence, and
    the other sequences, are what the definition gives."""
    rng = np.random.default_rng(43 + fmt)
    v = [rng.standard_normal((2, 50, 64)) for _ in range(3)]
    v[1][1, 20, 3] = value
    p = Paged(rng, fmt, [50] * 3, 2, 64, 16, v=v)
    dtype = dtype_of(fmt)
    q = torch.from_numpy(rng.standard_normal((3, 4, 64)).astype(np.float32)).cuda().to(TYPES[dtype])
    out = attend(p, q, dtype, 0.1).double().cpu().numpy()
    hit = np.zeros(out.shape, bool)
    hit[1, 2:, 3] = True
    if fmt == moa.KV_INT4:
        hit[1, 2:] = True
    assert not np.isfinite(out[hit]).any() and np.isfinite(out[~hit]).all()
    for name in "kv":                                       # (the definition elsewhere: that value counts as 0)
        p.values[name] = np.where(np.isfinite(p.values[name]), p.values[name], 0)
    want, bound = attend64(q.double().cpu().numpy(), p, 0.1)
    if fmt == moa.KV_F32:
        bound = np.maximum(bound, 5e-6)
    off = np.abs(out - want)
    tol = bound + np.abs(want) * torch.finfo(TYPES[dtype]).eps / 2 + 2.0 ** -25
    assert np.all((off <= tol)[~hit])


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("fmt", range(4), ids=lambda f: NAMES[f])
def test_keys_that_are_not_finite_stay_where_they_are(fmt, value):
    """In K: NaN in the heads of that K/V head that the definition makes NaN; a score of -inf is a weight of 0 in 16 bits and may be NaN
    elsewhere.  The other head and the other sequences are what the definition gives."""
    rng = np.random.default_rng(47 + fmt)
    k = [rng.standard_normal((2, 50, 64)) for _ in range(3)]
    k[1][1, 20, 3] = value
    p = Paged(rng, fmt, [50] * 3, 2, 64, 16, k=k)
    dtype = dtype_of(fmt)
    q = torch.from_numpy(rng.standard_normal((3, 4, 64)).astype(np.float32)).cuda().to(TYPES[dtype])
    q[1, 2, 3], q[1, 3, 3] = 0.5, -0.5
    out = attend(p, q, dtype, 0.1).double().cpu().numpy()
    nan = [fmt == moa.KV_INT4 or np.isnan(value) or s * value > 0 for s in (0.5, -0.5)]       # of heads 2 and 3
    check = np.ones(out.shape, bool)
    for i in (0, 1):
        if nan[i]:
            assert np.isnan(out[1, 2 + i]).all()
        if nan[i] or fmt == moa.KV_F32:
            check[1, 2 + i] = False
    if not check[1, 2:].any():                              # (the definition elsewhere: that value counts as 0)
        p.values["k"] = np.where(np.isfinite(p.values["k"]), p.values["k"], 0)
    with np.errstate(invalid="ignore"):
        want, bound = attend64(q.double().cpu().numpy(), p, 0.1)
    if check[1, 2:].any():                                  # a weight of 0 for row 20: the bound is that of the other rows
        b = p.table_host[1, 1]
        p.values["k"][b, 1, 4] = 0
        bound[1, 2:] = attend64(q.double().cpu().numpy(), p, 0.1)[1][1, 2:]
    if fmt == moa.KV_F32:
        bound = np.maximum(bound, 5e-6)
    tol = bound + np.abs(want) * torch.finfo(TYPES[dtype]).eps / 2 + 2.0 ** -25
    assert np.all((np.abs(out - want) <= tol)[check])
