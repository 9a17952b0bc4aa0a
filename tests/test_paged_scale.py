"""Scales that a paged attention call refuses: what the kernels work with is scale * log2(e) in fp32."""
import pytest

import paper_2607_19456_b200 as moa
from paper_2607_19456_b200 import build as moa_build


@pytest.mark.parametrize("format", range(4))
@pytest.mark.parametrize("scale", [2.5e38, -2.5e38, 3.4e38])
def test_a_scale_that_overflows_is_refused(format, scale):
    moa_build.build()
    cache = moa.PagedCache(format, 256, 256, 4, 16, 2, 128, None, None, 256, 256)
    dtype = moa.BF16 if format == moa.KV_INT4 else format
    code = moa.lib().moa_paged_decode_attn(cache, 256, 256, dtype, 0, 2, 4, 256, 256, 3, scale, 256, 1 << 30, None)
    assert code == moa.ERR_INVALID
