"""4-bit rows whose scale is infinite, NaN or far larger than the others': tokens that do not see the row give the bits that they give
without it, and the ones that see it what the definition gives."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import TYPES, Paged
from prompt_util import attend_new64, chunk, close

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("odd", [float("inf"), float("nan"), 2.0 ** 15, 2.0 ** 11], ids=["inf", "nan", "2^15", "2^11"])
@pytest.mark.parametrize("new,past,h_q,d", [(60, 150, 4, 128), (60, 150, 4, 64), (300, 20, 2, 128), (9, 3000, 8, 128), (200, 0, 8, 64)])
@pytest.mark.parametrize("dtype", [moa.F16, moa.BF16], ids=["f16", "bf16"])
def test_a_scale_that_some_do_not_see(dtype, new, past, h_q, d, odd):
    rng = np.random.default_rng(new + past + d)
    n, h_kv = new + past, 2
    p = Paged(rng, moa.KV_INT4, [n], h_kv, d, 16)
    q = torch.from_numpy(rng.standard_normal((new, h_q, d)).astype(np.float32)).cuda().to(TYPES[dtype])
    clean = chunk(p, q, [new], dtype, 0.1)
    # two rows, the first one seen from the middle of the new tokens on
    for row, head in ((past + new // 2, 0), (n - 2, 1)):
        p.params["v"][int(p.table_host[0, row // 16]), head, row % 16, 0] = odd
    got = chunk(p, q, [new], dtype, 0.1)
    half = h_q // h_kv
    for first, heads in ((new // 2, slice(0, half)), (new - 2, slice(half, h_q))):
        assert torch.equal(got[:first, heads], clean[:first, heads])
        if not np.isfinite(odd):
            assert not bool(torch.isfinite(got[first:, heads]).any())
    if np.isfinite(odd):
        codes = p.pools["v"].cpu().numpy()
        par = p.params["v"].double().cpu().numpy()
        c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
        pages = p.table_host[0, :-(-n // 16)]

        def rows(x):
            return x[pages].transpose(1, 0, 2, 3).reshape(h_kv, -1, x.shape[-1])[:, :n]

        v, steps = rows(par[..., :1] * c + par[..., 1:]), rows(par[..., :1])[..., 0]
        want, tol = attend_new64(q.double().cpu().numpy(), p.rows("k", 0), v, 0.1, dtype, steps4=steps)
        if np.abs(want).max() < 65504:                      # (fp16 outputs)
            close(got, want, tol)
    assert moa.moa_device_status() == 0
