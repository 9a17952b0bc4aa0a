"""Attention over paged caches where the sums are hard.

Scores here come from one feature of q (the others are 0), so that they carry a few fp32 roundings and no more, and the
bounds are those of the weights and sums alone."""
import contextlib

import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, attend, attend64, dtype_of

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@contextlib.contextmanager
def one_cta():
    moa.moa_set_option(moa.OPT_NUM_CTAS, 1)
    try:
        yield
    finally:
        moa.moa_set_option(moa.OPT_NUM_CTAS, 0)


def one_feature(batch, h_q, d, dtype, size=1.0):
    q = torch.zeros((batch, h_q, d), dtype=TYPES[dtype], device="cuda")
    q[:, :, 0] = size
    return q


@pytest.mark.parametrize("nats", [12.0, 15.0, 17.5])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt,dtype", [(f, dtype_of(f, t)) for f, t in ((0, 0), (1, 1), (2, 2), (3, moa.BF16), (3, moa.F16))],
                         ids=["f32", "bf16", "f16", "int4-bf16", "int4-f16"])
def test_many_light_rows_beside_a_heavy_one(fmt, dtype, d, nats):
    """One row carries nearly all weight and holds zeros; what is left is the sum of 4096 rows `nats` lower."""
    rng = np.random.default_rng(3)
    n, batch = 4097, 16
    k = [np.zeros((1, n, d), np.float32) for _ in range(batch)]
    v = [rng.uniform(1, 2, (1, n, d)).astype(np.float32) for _ in range(batch)]
    for b in range(batch):
        heavy = [0, n - 1, 2000][b % 3]
        k[b][0, :, 0], k[b][0, heavy, 0] = -nats, 0
        v[b][0, heavy] = 0
    p = Paged(rng, fmt, [n] * batch, 1, d, 16, k=k, v=v)
    q = one_feature(batch, 3, d, dtype)
    with one_cta():
        out = attend(p, q, dtype, 1.0)
    assert moa.moa_device_status() == 0
    want, _ = attend64(q.double().cpu().numpy(), p, 1.0)
    # Relative: the sum of a lane's 512 probabilities 2^-15, the sum over 256 stages 2^-16, two-term weights 2^-17, scores of
    # 25 (log2) with three roundings and exp2 2^-17: below 2^-14 together; one-term fp16 weights of 4-bit rows 2^-12 of what
    # the rows span, which is less than they are.  Weights in fp16 end at 2^-25 of 2^11 times a row's: 2^-36 and less lost of
    # each (V at most 2; 4 bits: of 8 steps, the scale's power of two 2^-3).  The output's rounding, 2^-25 among fp16's subnormals.
    rel = 2.0 ** -14 + (2.0 ** -12 if fmt == moa.KV_INT4 else 0)
    tol = want * (rel + torch.finfo(out.dtype).eps / 2) + n * 2.0 ** -35 + 2.0 ** -25
    off = np.abs(out.double().cpu().numpy() - want)
    assert np.all(off <= tol), (float(off.max()), float((off / tol).max()))
