"""Calls that overlap on streams with workspaces of their own, in every type: the bits that they give alone."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, dtype_of
from paged_util import attend as attend_one
from prompt_util import chunk, prompt, starts_of, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", [moa.KV_F32, moa.KV_BF16, moa.KV_F16, moa.KV_INT4], ids=lambda f: NAMES[f])
def test_calls_that_overlap(fmt, d):
    rng = np.random.default_rng(71 + fmt)
    dtype = dtype_of(fmt, moa.F16)

    def tensors(*shape):
        return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda().to(TYPES[dtype])

    x = tensors(900, 12 * d)
    p = Paged(rng, fmt, [800, 650, 30], 2, d, 16)
    q, one, new = tensors(60, 8, d), tensors(3, 8, d), [20, 30, 10]
    starts = starts_of([500, 1, 399]), starts_of(new)
    alone = (prompt(x, 8, 2, d, [0] * 3, dtype, True, 0.1, starts=starts[0]), chunk(p, q, new, dtype, 0.1, starts=starts[1]), attend_one(p, one, dtype, 0.1))
    streams = [torch.cuda.Stream() for _ in range(4)]
    wss = [workspace(900, 8, 2, d, 3) for _ in streams]
    outs = [[torch.empty_like(a) for a in alone[:2]] for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, ws, out in zip(streams, wss, outs):
            prompt(x, 8, 2, d, [0] * 3, dtype, True, 0.1, out=out[0], ws=ws, starts=starts[0], stream=s)
            chunk(p, q, [0] * 3, dtype, 0.1, out=out[1], ws=ws, starts=starts[1], stream=s)
        again = attend_one(p, one, dtype, 0.1)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for out in outs for a, b in zip(alone, out)) and torch.equal(again, alone[2])
    assert moa.moa_device_status() == 0
