"""One CTA that works through units of several tiles and of one tile by turns: both slots, one, or (a padded token) none has a tile."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, dtype_of
from prompt_util import check_chunk, chunk

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", [moa.KV_BF16, moa.KV_F16, moa.KV_INT4], ids=lambda f: NAMES[f])
def test_units_of_several_tiles_and_of_one_by_turns(fmt, d):
    rng = np.random.default_rng(fmt + d)
    lens = [300, 40, 0, 700, 3, 129, 128, 0, 385, 1] * 4
    p = Paged(rng, fmt, lens, 2, d, 16)
    for dtype in [moa.BF16, moa.F16] if fmt == moa.KV_INT4 else [dtype_of(fmt)]:
        q = torch.from_numpy(rng.standard_normal((len(lens), 8, d)).astype(np.float32)).cuda().to(TYPES[dtype])
        first = None
        try:
            for ctas in (1, 1, 1, 2, 0):
                moa.moa_set_option(moa.OPT_NUM_CTAS, ctas)
                out = chunk(p, q, [1] * len(lens), dtype, d ** -0.5, uniform=True)
                assert ctas != 1 or first is None or torch.equal(out, first)
                if ctas != 1 or first is None:
                    for b, n in enumerate(lens):
                        if n == 0:
                            assert bool((out[b] == 0).all())
                        else:
                            check_chunk(out[b:b + 1], p, q[b:b + 1], [1 if i == b else 0 for i in range(len(lens))], dtype, d ** -0.5)
                first = out if ctas == 1 else first
        finally:
            moa.moa_set_option(moa.OPT_NUM_CTAS, 0)
    assert moa.moa_device_status() == 0
