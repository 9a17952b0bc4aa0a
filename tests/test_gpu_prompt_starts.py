"""Entries of token_start that do not ascend: a sequence that starts below an earlier entry is left out, in every type, and the others are
what they are alone."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import NAMES, TYPES, Paged, dtype_of
from prompt_util import check_chunk, check_prompt, chunk, prompt
from test_prompt_starts import taken

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

FORMATS = [moa.KV_F32, moa.KV_BF16, moa.KV_F16, moa.KV_INT4]


def check_starts(out, x, h_q, h_kv, d, starts, dtype):
    """Every token of `out` [tokens, h_q, d] that was -3: its sequence's, or as it was."""
    tokens, left = x.shape[0], np.ones(x.shape[0], bool)
    for b, ok in enumerate(taken(tokens, starts)):
        if ok:
            at = slice(starts[b], starts[b + 1])
            left[at] = False
            check_prompt(out[at], x[at], h_q, h_kv, d, [starts[b + 1] - starts[b]], dtype, True, 0.1)
    assert bool((out[torch.from_numpy(left).cuda()] == -3).all())


@pytest.mark.parametrize("starts", [[0, 200, 100, 256], [0, 256, 0, 256], [0, 256] * 40 + [0], [100, 40, 130, 256, 256], [0, 50, -7, 60, 1 << 30, 60, 256],
                                    [256, 0, 0, 0]], ids=lambda s: str(s[:6]))
@pytest.mark.parametrize("dtype", [moa.F32, moa.BF16, moa.F16], ids=lambda t: NAMES[t])
def test_starts_that_descend(dtype, starts):
    rng = np.random.default_rng(len(starts) + dtype)
    for h_q, h_kv in ((4, 2), (1, 1)):
        x = torch.from_numpy(rng.standard_normal((256, (h_q + 2 * h_kv) * 64)).astype(np.float32)).cuda().to(TYPES[dtype])
        out = prompt(x, h_q, h_kv, 64, [0] * (len(starts) - 1), dtype, True, 0.1, starts=torch.tensor(starts, dtype=torch.int32).cuda())
        assert moa.moa_device_status() == moa.STATUS_SEQLEN_RANGE
        check_starts(out, x, h_q, h_kv, 64, starts, dtype)


@pytest.mark.parametrize("dtype", [moa.F32, moa.BF16, moa.F16], ids=lambda t: NAMES[t])
def test_many_sequences_some_of_them_out_of_order(dtype):
    """More sequences than threads, and (fp32) more units than CTAs."""
    rng = np.random.default_rng(3 + dtype)
    new = rng.integers(0, 9, 1500)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    tokens = int(starts[-1])
    x = torch.from_numpy(rng.standard_normal((tokens, 4 * 64)).astype(np.float32)).cuda().to(TYPES[dtype])
    good = prompt(x, 2, 1, 64, new.tolist(), dtype, True, 0.1)
    assert moa.moa_device_status() == 0
    check_prompt(good, x, 2, 1, 64, new.tolist(), dtype, True, 0.1)
    for at, value in ((700, int(starts[900])), (40, 3), (1200, -1), (1499, tokens + 1)):
        wrong = starts.copy()
        wrong[at] = value
        out = prompt(x, 2, 1, 64, new.tolist(), dtype, True, 0.1, starts=torch.from_numpy(wrong).cuda())
        assert moa.moa_device_status() == moa.STATUS_SEQLEN_RANGE
        check_starts(out, x, 2, 1, 64, wrong.tolist(), dtype)


@pytest.mark.parametrize("fmt", FORMATS, ids=lambda f: NAMES[f])
def test_chunks_whose_starts_descend(fmt):
    rng = np.random.default_rng(17 + fmt)
    new, past = [20, 30, 25, 5], [100, 50, 0, 400]
    p = Paged(rng, fmt, [a + b for a, b in zip(new, past)], 2, 128, 16)
    dtype = dtype_of(fmt)
    q = torch.from_numpy(rng.standard_normal((80, 4, 128)).astype(np.float32)).cuda().to(TYPES[dtype])
    out = chunk(p, q, new, dtype, 0.1, starts=torch.tensor([0, 50, 20, 75, 80], dtype=torch.int32).cuda())      # 50, -30, 55 and 5 tokens
    assert moa.moa_device_status() == moa.STATUS_SEQLEN_RANGE
    check_chunk(out[75:], p, q[75:], [0, 0, 0, 5], dtype, 0.1)
    kept, p.lens = p.lens, [120]                            # the first sequence's length says 120: 50 new tokens behind 70
    check_chunk(out[:50], p, q[:50], [50], dtype, 0.1)
    p.lens = kept
    assert bool((out[50:75] == -3).all())


@pytest.mark.parametrize("batch", [128, 129, 511, 512, 513, 20000])
def test_fp32_by_number_of_sequences(batch):
    """Where the search takes another round, and where a CTA starts to take several units; the last sequence is out of order."""
    rng = np.random.default_rng(batch)
    new = rng.integers(0, 5, batch)
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    tokens = int(starts[-1])
    x = torch.from_numpy(rng.standard_normal((tokens, 5 * 64)).astype(np.float32)).cuda()
    out = prompt(x, 3, 1, 64, new.tolist(), moa.F32, True, 0.1)
    assert moa.moa_device_status() == 0
    check_prompt(out, x, 3, 1, 64, new.tolist(), moa.F32, True, 0.1)
    starts[-2] = tokens - 1 if starts[-2] != tokens - 1 else tokens       # one sequence longer or shorter than the one behind it
    starts[-1] = starts[-2] - 1
    again = prompt(x, 3, 1, 64, new.tolist(), moa.F32, True, 0.1, starts=torch.from_numpy(starts).cuda())
    assert moa.moa_device_status() == moa.STATUS_SEQLEN_RANGE
    same = int(starts[-3])
    assert torch.equal(again[:same], out[:same])
