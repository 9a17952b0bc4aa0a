"""Steps of a serving program enqueued without a wait between them (every kernel is launched while the one before it runs), against the
same steps with a wait after every call: the same bits."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, dtype_of, rope_table, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("batch", [3, 70, 200])
@pytest.mark.parametrize("fmt", range(4), ids=lambda f: NAMES[f])
def test_steps_without_a_wait(fmt, batch):
    """Lengths advance, a row is appended, attended to and read back, 25 times over pages of 8 rows: lengths and rows are always those of
    the kernel just before."""
    h_q, h_kv, d, page, steps = 4, 2, 64, 8, 25
    dtype = dtype_of(fmt)
    results = []
    for wait in (True, False):
        rng = np.random.default_rng(83 + batch)
        start = rng.integers(0, 30, batch)
        p = Paged(rng, fmt, (start + steps).tolist(), h_kv, d, page)
        lens = torch.from_numpy(start.astype(np.int32)).cuda()
        starts = torch.arange(batch + 1, dtype=torch.int32, device="cuda")
        rope = torch.from_numpy(rope_table(64, d)).cuda()
        new = [[torch.from_numpy(rng.standard_normal((batch, h, d)).astype(np.float32)).cuda().to(TYPES[dtype]) for h in (h_q, h_kv, h_kv)]
               for _ in range(steps)]
        turned = torch.empty((batch, h_q, d), dtype=TYPES[dtype], device="cuda")
        outs = torch.zeros((steps, batch, h_q, d), dtype=TYPES[dtype], device="cuda")
        back = torch.zeros((steps, 2, batch, h_kv, 64, d), device="cuda")
        ws, size = workspace(batch, h_q, h_kv, d)
        torch.cuda.synchronize()
        for i, (q, k, v) in enumerate(new):
            calls = [lambda: moa.moa_lens_add(lens, batch, 1),
                     lambda: moa.moa_paged_append(p.cache, q, k, v, turned, dtype, None, batch, h_q, batch, starts if i % 2 else None, lens,
                                                  p.table, p.max_pages, rope, 64, d, moa.ROPE_HALVES),
                     lambda: moa.moa_paged_decode_attn(p.cache, turned, outs[i], dtype, 0, batch, h_q, lens, p.table, p.max_pages, 0.2, ws, size),
                     lambda: moa.moa_paged_gather(p.cache, back[i, 0], back[i, 1], moa.F32, batch, 64, None, lens, p.table, p.max_pages)]
            for call in calls:
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert moa.moa_device_status() == 0 and torch.equal(lens.cpu(), torch.from_numpy((start + steps).astype(np.int32)))
        results.append((outs, back))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1].nan_to_num(7), results[1][1].nan_to_num(7))
    assert bool(results[0][0].isfinite().all())
