"""Paged caches whose pools pass 2^32 bytes (and 2^32 elements in 16 and 4 bits): rows on pages at both ends and on either side of
the boundary, appended, read back and attended to; their neighbours stay as they were."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, attend64, dtype_of, pack4, rotate32, rope_table, unpack4, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fmt,pages", [(moa.KV_F32, 300_000), (moa.KV_BF16, 600_000), (moa.KV_F16, 600_000), (moa.KV_INT4, 1_300_000)],
                         ids=lambda v: NAMES.get(v, str(v)) if isinstance(v, int) and v < 4 else str(v))
def test_pools_beyond_2_to_the_32(fmt, pages):
    rng = np.random.default_rng(71 + fmt)
    h_q, h_kv, d, page = 4, 2, 128, 32
    width, dtype = (d // 2 if fmt == moa.KV_INT4 else d), dtype_of(fmt)
    kind = torch.uint8 if fmt == moa.KV_INT4 else TYPES[fmt]
    row_bytes = width * (1 if fmt == moa.KV_INT4 else torch.empty(0, dtype=kind).element_size())
    per_page = h_kv * page * row_bytes
    assert pages * per_page > 2 ** 32
    pools = [torch.zeros((pages, h_kv, page, width), dtype=kind, device="cuda") for _ in "kv"]
    params = [torch.zeros((pages, h_kv, page, 2), dtype=torch.float16, device="cuda") for _ in "kv"] if fmt == moa.KV_INT4 else [None, None]
    cache = moa.PagedCache(fmt, pools[0], pools[1], pages, page, h_kv, d, None, None, params[0], params[1])
    edge = 2 ** 32 // per_page                              # its bytes pass 2^32
    picked = [0, pages - 1, edge - 1, edge, edge + 1, 2 ** 31 // per_page, pages // 2 + 7]
    lens = [32 * 4 + 9, 32 + 3]
    table = np.array([[picked[1], picked[3], picked[0], picked[5], picked[4]], [picked[2], picked[6], 0, 0, 0]], np.int32)
    new = sum(lens)
    x = [rng.standard_normal((new, h, d)).astype(np.float32) for h in (h_q, h_kv, h_kv)]
    q, k, v = (torch.from_numpy(y).cuda().to(TYPES[dtype]) for y in x)
    xf = [y.float().cpu().numpy() for y in (q, k, v)]
    q_out = torch.empty_like(q)
    rope = rope_table(256, d)
    starts, lens_d, table_d = (torch.tensor(y, dtype=torch.int32, device="cuda") for y in ([0, lens[0], new], lens, table.tolist()))
    moa.moa_paged_append(cache, q, k, v, q_out, dtype, None, new, h_q, 2, starts, lens_d, table_d, 5, torch.from_numpy(rope).cuda(), 256, d, 0)
    assert moa.moa_device_status() == 0
    pos = np.concatenate([np.arange(n) for n in lens])

    class Held:
        pass
    held = Held()
    held.fmt, held.h_kv, held.lens = fmt, h_kv, lens
    rows = {"k": rotate32(xf[1], pos, rope, d, 0), "v": xf[2]}

    def rows64(name, b, n):
        y = rows[name][:lens[0]] if b == 0 else rows[name][lens[0]:]
        y = y.transpose(1, 0, 2)
        return unpack4(*pack4(y)) if fmt == moa.KV_INT4 else torch.from_numpy(y.copy()).to(TYPES[fmt]).double().numpy()
    held.rows = rows64

    kb = torch.full((2, h_kv, lens[0], d), 9.0, device="cuda")
    vb = kb.clone()
    moa.moa_paged_gather(cache, kb, vb, moa.F32, 2, lens[0], None, lens_d, table_d, 5)
    for b, n in enumerate(lens):
        for name, got in (("k", kb), ("v", vb)):
            assert np.array_equal(got[b, :, :n].cpu().numpy(), rows64(name, b, n).astype(np.float32)), (b, name)
    last = torch.stack([q_out[lens[0] - 1], q_out[new - 1]])
    out = torch.empty_like(last)
    ws, n_ws = workspace(2, h_q, h_kv, d)
    moa.moa_paged_decode_attn(cache, last, out, dtype, 0, 2, h_q, lens_d, table_d, 5, d ** -0.5, ws, n_ws)
    assert moa.moa_device_status() == 0
    want, bound = attend64(last.double().cpu().numpy(), held, d ** -0.5)
    if fmt == moa.KV_F32:
        bound = np.maximum(bound, 5e-6)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound + np.abs(want) * torch.finfo(out.dtype).eps / 2 + 2.0 ** -25)
    for p in picked:                                       # the pages beside those that were written are still zero
        for n in (p - 1, p + 1):
            if 0 <= n < pages and n not in picked:
                assert not bool(pools[0][n].any()) and not bool(pools[1][n].any())
