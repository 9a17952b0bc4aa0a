"""Keys turned by positions of several axes on their way into a 4-bit cache: the codes and parameters of the turned rows, bit for bit."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import TYPES, Paged, pack4, rope_table
from prompt_util import starts_of
from test_gpu_axes import axis_map, turned

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("rot,style,kind", [(128, moa.ROPE_HALVES, "runs"), (128, moa.ROPE_HALVES, "turns"), (128, moa.ROPE_PAIRS, "any"), (48, moa.ROPE_HALVES, "any"),
                                            (48, moa.ROPE_PAIRS, "turns"), (32, moa.ROPE_HALVES, "runs")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [moa.BF16, moa.F16], ids=["bf16", "f16"])
def test_keys_of_a_four_bit_cache(dtype, d, rot, style, kind):
    rot = min(rot, d)
    rng = np.random.default_rng(d + rot + style)
    new, past, h_q, h_kv = [1, 0, 30, 6], [5, 9, 70, 0], 4, 2
    tokens, table = sum(new), rope_table(200, rot)
    q, k, v = (torch.from_numpy(rng.standard_normal((tokens, h, d)).astype(np.float32)).cuda().to(TYPES[dtype]) for h in (h_q, h_kv, h_kv))
    pos, amap = rng.integers(0, 200, (3, tokens)).astype(np.int32), axis_map(rng, 3, rot // 2, kind)
    p = Paged(rng, moa.KV_INT4, [a + b for a, b in zip(new, past)], h_kv, d, 16)
    q_out = torch.empty_like(q)
    moa.moa_paged_append_axes(p.cache, q, k, v, q_out, dtype, None, tokens, h_q, 4, starts_of(new), p.lens_dev, p.table, p.max_pages,
                              torch.from_numpy(pos).cuda(), 3, amap.tobytes(), torch.from_numpy(table).cuda(), 200, rot, style)
    assert moa.moa_device_status() == 0
    want = {"k": pack4(turned(k.float().cpu().numpy(), pos, amap, table, rot, style == moa.ROPE_PAIRS)), "v": pack4(v.float().cpu().numpy())}
    for name in "kv":
        codes, params = p.pools[name].cpu().numpy(), p.params[name].cpu().numpy()
        at = 0
        for b, n in enumerate(new):
            for i in range(n):
                page, off = int(p.table_host[b, (past[b] + i) // 16]), (past[b] + i) % 16
                assert np.array_equal(codes[page, :, off], want[name][0][at]) and np.array_equal(params[page, :, off], want[name][1][at]), (name, b, i)
                at += 1
