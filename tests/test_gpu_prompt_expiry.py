"""A wait of the prompt kernel that runs out, without faulting the GPU: one CTA, one tile of K that is announced and never copied (nothing is in
flight for it), and a limit of a few hundred polls.  The call returns, its status says so, and the next call is right."""
import time

import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, dtype_of
from prompt_util import check_chunk, check_prompt, chunk, prompt, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("tile", [0, 1, 3])
@pytest.mark.parametrize("dtype,d", [(moa.BF16, 128), (moa.F16, 64)], ids=["bf16-128", "f16-64"])
@pytest.mark.parametrize("paged", [False, True], ids=["tensors", "pools"])
def test_an_expired_wait_is_reported_and_the_workspace_stays_usable(dtype, d, tile, paged):
    rng = np.random.default_rng(tile + d)
    new = [40, 600]
    if paged:
        p = Paged(rng, dtype, [500, 700], 1, d, 32)
        x = torch.from_numpy(rng.standard_normal((640, 1, d)).astype(np.float32)).cuda().to(TYPES[dtype])
    else:
        x = torch.from_numpy(rng.standard_normal((640, 3 * d)).astype(np.float32)).cuda().to(TYPES[dtype])
    ws = workspace(640, 1, 1, d, 2)

    def call():
        return chunk(p, x, new, dtype, 0.1, ws=ws) if paged else prompt(x, 1, 1, d, new, dtype, True, 0.1, ws=ws)

    call()
    torch.cuda.synchronize()
    moa.moa_set_option(moa.OPT_NUM_CTAS, 1)
    moa.moa_set_option(moa.OPT_WAIT_LIMIT, 300)
    moa.moa_set_option(moa.OPT_TEST_SKIP_COPY, tile)
    try:
        began = time.time()
        call()
        torch.cuda.synchronize()
        assert moa.moa_device_status() & moa.STATUS_WAIT_TIMEOUT
        assert time.time() - began < 5
    finally:
        moa.moa_set_option(moa.OPT_TEST_SKIP_COPY, -1)
        moa.moa_set_option(moa.OPT_WAIT_LIMIT, 0)
        moa.moa_set_option(moa.OPT_NUM_CTAS, 0)
    assert moa.moa_device_status() == 0                     # reading the status cleared it
    out = call()                                            # on the workspace that the call left as it was
    torch.cuda.synchronize()
    assert moa.moa_device_status() == 0
    if paged:
        check_chunk(out, p, x, new, dtype, 0.1)
    else:
        check_prompt(out, x, 1, 1, d, new, dtype, True, 0.1)
