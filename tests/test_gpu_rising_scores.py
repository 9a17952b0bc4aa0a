"""Scores that rise a little after the first rows: the reference moves once and the weights are made once, not twice for the rest."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES
from prompt_util import attend_new64, close, prompt, starts_of, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [moa.BF16, moa.F16], ids=lambda t: NAMES[t])
def test_scores_a_few_powers_of_two_above_the_first(dtype):
    rng = np.random.default_rng(5)
    n, heads, d = 4096, 16, 128
    times = {}
    for rise in (0.0, 5.0):                                # log2 of the weights, row 64 on against the first ones
        x = rng.standard_normal((n, heads, 3 * d)).astype(np.float32)
        u = rng.standard_normal(d).astype(np.float32)
        x[..., :d] = u
        x[..., d:2 * d] *= 0.01
        x[64:, :, d:2 * d] += rise * np.log(2) * u / (u ** 2).sum()
        q, k, v = (torch.from_numpy(np.ascontiguousarray(y)).cuda().to(TYPES[dtype]) for y in np.split(x, 3, -1))
        qkv = torch.cat([y.flatten(1) for y in (q, k, v)], 1)
        ws, out, starts = workspace(n, heads, heads, d, 1), torch.empty_like(q), starts_of([n])
        each = []
        for _ in range(25):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            prompt(qkv, heads, heads, d, [n], dtype, False, 1.0, out=out, ws=ws, starts=starts)
            b.record()
            b.synchronize()
            each.append(a.elapsed_time(b))
        times[rise] = float(np.median(each[5:]))
        m = 3
        want, tol = attend_new64(q[:m, :1].double().cpu().numpy(), k[None, :, 0].double().cpu().numpy(), v[None, :, 0].double().cpu().numpy(), 1.0, dtype, causal=False)
        close(out[:m, :1], want, tol)
    print(times)
    assert times[5.0] < 1.3 * times[0.0], times            # (made twice: 1.48 times)
