"""fp32: how keys are cut into pieces follows from the sequences' lengths, not from how many pages a table could name."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import Paged
from prompt_util import check_chunk, chunk

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("new,past,h_q,h_kv,d", [([5], [300], 8, 1, 128), ([3, 40], [1700, 0], 4, 2, 64), ([1], [0], 1, 1, 128), ([4, 0, 2], [4000, 9, 255], 8, 2, 128),
                                                 ([130], [2500], 2, 1, 64)])
def test_a_wider_page_table_changes_nothing(new, past, h_q, h_kv, d):
    rng = np.random.default_rng(sum(new) + d)
    p = Paged(rng, moa.KV_F32, [a + b for a, b in zip(new, past)], h_kv, d, 16, extra_pages=0)
    q = torch.from_numpy(rng.standard_normal((sum(new), h_q, d)).astype(np.float32)).cuda()
    first = chunk(p, q, new, moa.F32, 0.1)
    check_chunk(first, p, q, new, moa.F32, 0.1)
    for pages in (p.max_pages + 1, 400, 40000):
        wide = torch.full((len(new), pages), -7, dtype=torch.int32, device="cuda")
        wide[:, :p.table.shape[1]] = p.table
        kept = p.table, p.max_pages
        p.table, p.max_pages = wide, pages
        assert torch.equal(chunk(p, q, new, moa.F32, 0.1), first), pages
        p.table, p.max_pages = kept
    assert moa.moa_device_status() == 0
