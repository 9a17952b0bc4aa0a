"""Paged caches in random mixtures of format, heads, pages, lengths and layouts, two kinds of calls on one stream without a wait
between them, and a batch at every size around the borders of the length scan."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, attend, attend64, dtype_of, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def close(p, q, out, scale):
    want, bound = attend64(q.double().cpu().numpy(), p, scale)
    if p.fmt == moa.KV_F32:
        bound = np.maximum(bound, 5e-6)
    off = np.abs(out.double().cpu().numpy() - want)
    tol = bound + np.abs(want) * torch.finfo(out.dtype).eps / 2 + 2.0 ** -25
    assert np.all(off <= tol), float((off / tol).max())


@pytest.mark.parametrize("seed", range(24))
def test_random_mixture(seed):
    rng = np.random.default_rng(9000 + seed)
    fmt = int(rng.integers(4))
    d = int(rng.choice([64, 128]))
    h_kv = int(rng.integers(1, 6))
    h_q = h_kv * int(rng.choice([1, 2, 3, 5, 8, 9, 13, 16, 17, 24, 40]))
    page = int(rng.choice([1, 3, 8, 16, 20, 32, 48, 64, 256]))
    lens = rng.integers(0, int(rng.choice([3, 40, 700])), int(rng.integers(1, 40))).tolist()
    p = Paged(rng, fmt, lens, h_kv, d, page, heads_inner=bool(rng.integers(2)))
    dtype = dtype_of(fmt, int(rng.choice([moa.BF16, moa.F16])))
    q = torch.from_numpy(rng.standard_normal((len(lens), h_q, d)).astype(np.float32)).cuda().to(TYPES[dtype])
    moa.moa_set_option(moa.OPT_NUM_CTAS, int(rng.choice([0, 0, 2, 37])))
    try:
        out = attend(p, q, dtype, 0.09)
    finally:
        moa.moa_set_option(moa.OPT_NUM_CTAS, 0)
    assert moa.moa_device_status() == 0
    close(p, q, out, 0.09)


@pytest.mark.parametrize("batch", [31, 32, 33, 127, 128, 129, 148, 149, 192, 256, 257, 385])
def test_batches_around_the_borders_of_the_scan(batch):
    rng = np.random.default_rng(batch)
    for fmt in (moa.KV_BF16, moa.KV_INT4):
        lens = rng.integers(0, 20, batch).tolist()
        lens[-1] = 130
        p = Paged(rng, fmt, lens, 1, 64, 16)
        q = torch.from_numpy(rng.standard_normal((batch, 2, 64)).astype(np.float32)).cuda().bfloat16()
        close(p, q, attend(p, q, moa.BF16, 0.125), 0.125)
    assert moa.moa_device_status() == 0


def test_calls_of_different_kinds_back_to_back():
    """Formats and the dense calls in turn on one stream, one workspace for all that is paged: no call waits on the host."""
    rng = np.random.default_rng(5)
    caches = [Paged(rng, fmt, [1500, 40, 0, 3000], 2, d, 16) for fmt in (0, 1, 2, 3) for d in (64, 128)]
    qs = [torch.from_numpy(rng.standard_normal((4, 12, p.d)).astype(np.float32)).cuda().to(TYPES[dtype_of(p.fmt)]) for p in caches]
    n = max(moa.moa_paged_workspace_bytes(4, 12, 2, d) for d in (64, 128))
    ws = (torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    dense = [torch.randn(2, 8, 128, device="cuda"), torch.randn(2, 2, 900, 128, device="cuda"), torch.randn(2, 2, 900, 128, device="cuda")]
    got = torch.empty(2, 8, 128, device="cuda")
    for _ in range(4):
        outs = []
        for p, q in zip(caches, qs):
            outs.append(attend(p, q, dtype_of(p.fmt), 0.1, ws=ws))
            moa.moa_decode_attn(dense[0], dense[1], dense[2], got, 2, 8, 2, 900, 128, 128, 0.1)
        torch.cuda.synchronize()
        for p, q, o in zip(caches, qs, outs):
            close(p, q, o, 0.1)
    assert moa.moa_device_status() == 0


@pytest.mark.parametrize("batch", [1, 5, 200])
@pytest.mark.parametrize("fmt", range(4), ids=lambda f: NAMES[f])
def test_nothing_but_empty_sequences(fmt, batch):
    p = Paged(np.random.default_rng(batch), fmt, [0] * batch, 2, 64, 16)
    dtype = dtype_of(fmt)
    out = attend(p, torch.ones((batch, 4, 64), dtype=TYPES[dtype], device="cuda"), dtype, 0.1)
    assert bool((out == 0).all()) and moa.moa_device_status() == 0


@pytest.mark.parametrize("fmt", range(4), ids=lambda f: NAMES[f])
def test_one_kv_head_for_128_query_heads(fmt):
    rng = np.random.default_rng(97 + fmt)
    p = Paged(rng, fmt, [1000, 7], 1, 128, 16)
    dtype = dtype_of(fmt, moa.F16)
    q = torch.from_numpy(rng.standard_normal((2, 128, 128)).astype(np.float32)).cuda().to(TYPES[dtype])
    close(p, q, attend(p, q, dtype, 0.09), 0.09)
    assert moa.moa_device_status() == 0
