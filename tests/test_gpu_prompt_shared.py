"""Two captured graphs on one workspace, calls that overlap on streams of their own, and a call between others of the library."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import TYPES, Paged
from paged_util import attend as attend_one
from prompt_util import check_chunk, check_prompt, chunk, prompt, starts_of, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def tensors(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda().to(TYPES[dtype])


@pytest.mark.parametrize("dtype", [moa.F32, moa.BF16, moa.F16], ids=["f32", "bf16", "f16"])
def test_two_graphs_on_one_workspace(dtype):
    rng = np.random.default_rng(61 + dtype)
    x = tensors(rng, (1500, 3 * 128), dtype)                # one K/V head: cut into pieces
    p = Paged(rng, dtype, [3000, 77], 2, 128, 16)
    q = tensors(rng, (9, 8, 128), dtype)
    new = [5, 4]
    starts = [starts_of([1500]), starts_of(new)]
    sizes = moa.moa_prompt_workspace_bytes(1500, 1, 1, 128, 1), moa.moa_prompt_workspace_bytes(9, 8, 2, 128, 2)
    ws = torch.full((max(sizes),), 0x5A, dtype=torch.uint8, device="cuda")
    calls = [lambda out: prompt(x, 1, 1, 128, [1500], dtype, True, 0.1, out=out, ws=(ws, sizes[0]), starts=starts[0]),
             lambda out: chunk(p, q, new, dtype, 0.1, out=out, ws=(ws, sizes[1]), starts=starts[1])]
    outs = [call(None) for call in calls]
    want = [o.clone() for o in outs]
    torch.cuda.synchronize()
    graphs = []
    for call, out in zip(calls, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(out)
    for order in ((0, 1), (1, 0), (0, 0), (1, 1), (0, 1)):
        for o in outs:
            o.fill_(-3.0)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in set(order):
            assert torch.equal(outs[i], want[i]), order
    check_prompt(want[0], x, 1, 1, 128, [1500], dtype, True, 0.1)
    check_chunk(want[1], p, q, new, dtype, 0.1)
    assert moa.moa_device_status() == 0


def test_calls_that_overlap():
    """Calls on four streams with workspaces of their own, beside single-query calls, give the bits that they give alone."""
    rng = np.random.default_rng(71)
    dtype = moa.BF16
    x = tensors(rng, (900, 12 * 64), dtype)
    p = Paged(rng, dtype, [800, 650, 30], 2, 64, 16)
    q, one = tensors(rng, (60, 8, 64), dtype), tensors(rng, (3, 8, 64), dtype)
    new = [20, 30, 10]
    streams = [torch.cuda.Stream() for _ in range(4)]
    wss = [workspace(900, 8, 2, 64, 3) for _ in streams]
    alone = prompt(x, 8, 2, 64, [500, 1, 399], dtype, True, 0.1), chunk(p, q, new, dtype, 0.1), attend_one(p, one, dtype, 0.1)
    outs = [[torch.empty_like(a) for a in alone[:2]] for _ in streams]
    starts = starts_of([500, 1, 399]), starts_of(new)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, ws, out in zip(streams, wss, outs):
            prompt(x, 8, 2, 64, [0] * 3, dtype, True, 0.1, out=out[0], ws=ws, starts=starts[0], stream=s)
            chunk(p, q, [0] * 3, dtype, 0.1, out=out[1], ws=ws, starts=starts[1], stream=s)
        again = attend_one(p, one, dtype, 0.1)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for out in outs for a, b in zip(alone, out)) and torch.equal(again, alone[2])
    assert moa.moa_device_status() == 0
