"""Attention over packed prompts against the definition in 64 bits."""
import numpy as np
import pytest

import paper_2607_19456_b200 as moa
from paged_util import TYPES
from prompt_util import attend_new64, check_prompt, close, prompt, starts_of, workspace

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

NAMES = {moa.F32: "f32", moa.BF16: "bf16", moa.F16: "f16"}
DTYPES = [moa.F32, moa.BF16, moa.F16]


def made(rng, tokens, h_q, h_kv, d, dtype):
    x = rng.standard_normal((tokens, (h_q + 2 * h_kv) * d)).astype(np.float32)
    x[:, h_q * d:(h_q + h_kv) * d] += rng.standard_normal(h_kv * d).astype(np.float32)
    return torch.from_numpy(x).cuda().to(TYPES[dtype])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES, ids=lambda t: NAMES[t])
@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (4, 4), (8, 2), (7, 1), (18, 2)])
def test_lengths_and_groups(dtype, d, h_q, h_kv, causal):
    rng = np.random.default_rng(100 * h_q + h_kv + dtype + d)
    new = [1, 0, 15, 128, 17, 300, 2, 129, 0]
    x = made(rng, sum(new), h_q, h_kv, d, dtype)
    out = prompt(x, h_q, h_kv, d, new, dtype, causal, d ** -0.5)
    torch.cuda.synchronize()
    assert moa.moa_device_status() == 0 and moa.moa_last_path() == moa.PATH_PROMPT
    check_prompt(out, x, h_q, h_kv, d, new, dtype, causal, d ** -0.5)


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda t: NAMES[t])
@pytest.mark.parametrize("new,h_q,h_kv,d,causal", [([1537], 8, 2, 128, True), ([1100], 4, 4, 64, False), ([257] * 40, 4, 1, 64, True), ([1] * 700, 2, 1, 128, True)])
def test_long_and_many(dtype, new, h_q, h_kv, d, causal):
    rng = np.random.default_rng(len(new) + dtype)
    x = made(rng, sum(new), h_q, h_kv, d, dtype)
    out = prompt(x, h_q, h_kv, d, new, dtype, causal, 0.11)
    assert moa.moa_device_status() == 0
    check_prompt(out, x, h_q, h_kv, d, new, dtype, causal, 0.11)
    assert torch.equal(out, prompt(x, h_q, h_kv, d, new, dtype, causal, 0.11))          # the same bits again


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda t: NAMES[t])
def test_few_units_are_cut(dtype):
    """One K/V head over 2600 keys: pieces, joined in order, whatever the number of CTAs."""
    rng = np.random.default_rng(5 + dtype)
    new, h_q, d = [40, 2600], 1, 128
    x = made(rng, sum(new), h_q, 1, d, dtype)
    try:
        for ctas in (0, 1, 7, 300):
            moa.moa_set_option(moa.OPT_NUM_CTAS, ctas)
            check_prompt(prompt(x, h_q, 1, d, new, dtype, False, 0.1), x, h_q, 1, d, new, dtype, False, 0.1)
    finally:
        moa.moa_set_option(moa.OPT_NUM_CTAS, 0)
    assert moa.moa_device_status() == 0


@pytest.mark.parametrize("scale", [-0.09, 0.0, 1e-30, 1.5])
@pytest.mark.parametrize("dtype", DTYPES, ids=lambda t: NAMES[t])
def test_scales(dtype, scale):
    rng = np.random.default_rng(11)
    x = made(rng, 333, 4, 2, 64, dtype)
    check_prompt(prompt(x, 4, 2, 64, [333], dtype, True, scale), x, 4, 2, 64, [333], dtype, True, scale)


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda t: NAMES[t])
def test_weight_on_few_rows(dtype):
    """Scores far apart, rising and falling through the sequence, so that the reference moves often; and one row of all the weight
    beside 1500 rows 17 nats below it, which fp16 must not lose."""
    rng = np.random.default_rng(17 + dtype)
    d, n = 128, 1500
    for ramp in (np.linspace(-40, 4, n), np.linspace(4, -40, n), np.where(np.arange(n) == 777, 5.0, -12.0), np.linspace(-3000, 0, n)):
        x = rng.standard_normal((n, 3 * d)).astype(np.float32)
        x[:, :d] = x[:1, :d]
        x[:, d:2 * d] = ramp[:, None] * (x[0, :d] / (x[0, :d] ** 2).sum())[None] / 0.1
        x[:, 2 * d:] = np.abs(x[:, 2 * d:])
        xd = torch.from_numpy(x).cuda().to(TYPES[dtype])
        check_prompt(prompt(xd, 1, 1, d, [n], dtype, True, 0.1), xd, 1, 1, d, [n], dtype, True, 0.1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES, ids=lambda t: NAMES[t])
def test_what_is_not_seen_does_not_touch(dtype, d):
    """NaN and infinities in keys, values and queries reach the rows that see them and no other, across sequences too."""
    rng = np.random.default_rng(23)
    new, h_q, h_kv = [200, 333, 150], 4, 2
    x = made(rng, sum(new), h_q, h_kv, d, dtype)
    clean = prompt(x, h_q, h_kv, d, new, dtype, True, 0.1)
    at = 200 + 170                                          # token 170 of the second sequence
    bad = x.clone()
    bad[at, (h_q + h_kv) * d + 5] = float("nan")            # V, head 0, feature 5
    bad[at + 3, (h_q + h_kv + 1) * d + 7] = float("inf")    # V, head 1, feature 7
    bad[at + 40, h_q * d + 9] = float("nan")                # K, head 0
    bad[200 + 20, 3 * d + 1] = float("nan")                 # q, head 3
    got = prompt(bad, h_q, h_kv, d, new, dtype, True, 0.1)
    odd = torch.zeros_like(got, dtype=torch.bool)
    odd[at:533, :2, 5] = True
    odd[at + 3:533, 2:, 7] = True
    odd[at + 40:533, :2] = True
    odd[220, 3] = True
    assert bool((~torch.isfinite(got))[odd].all())
    assert torch.equal(got[~odd], clean[~odd])
    assert moa.moa_device_status() == 0


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda t: NAMES[t])
def test_padding_strides_and_refused_sequences(dtype):
    rng = np.random.default_rng(31)
    h_q, h_kv, d, new = 4, 2, 128, [50, 140, 66]
    x = made(rng, 300, h_q, h_kv, d, dtype)
    x[256:] = float("nan")                                  # tokens behind the last sequence
    wide = torch.full((300, h_q + 3, d), 7.0, dtype=TYPES[dtype], device="cuda")
    q, k, v = (y.unflatten(-1, (-1, d)) for y in x.split([h_q * d, h_kv * d, h_kv * d], -1))
    w = x.shape[1]
    ws = workspace(300, h_q, h_kv, d, 3)
    moa.moa_prompt_attn(q, k, v, wide, dtype, (w, w, w, (h_q + 3) * d), 300, h_q, h_kv, d, 3, starts_of(new), True, 0.1, *ws)
    check_prompt(wide[:256, :h_q], x[:256], h_q, h_kv, d, new, dtype, True, 0.1)
    assert bool((wide[256:] == 7).all()) and bool((wide[:, h_q:] == 7).all()) and moa.moa_device_status() == 0
    # a start behind the end, and one before the start before it: those sequences are left out
    out = prompt(x, h_q, h_kv, d, new, dtype, True, 0.1, starts=torch.tensor([0, 50, 190, 400], dtype=torch.int32).cuda())
    check_prompt(out[:190], x[:190], h_q, h_kv, d, new[:2], dtype, True, 0.1)
    assert bool((out[190:] == -3).all()) and moa.moa_device_status() == moa.STATUS_SEQLEN_RANGE
    # no starts: one sequence
    ws = workspace(256, h_q, h_kv, d, 1)
    out = torch.full((256, h_q, d), -3.0, dtype=TYPES[dtype], device="cuda")
    moa.moa_prompt_attn(q, k, v, out, dtype, (w, w, w, h_q * d), 256, h_q, h_kv, d, 1, None, True, 0.1, *ws)
    check_prompt(out, x[:256], h_q, h_kv, d, [256], dtype, True, 0.1)


@pytest.mark.parametrize("dtype", DTYPES, ids=lambda t: NAMES[t])
def test_graph_streams_and_one_workspace(dtype):
    """Captured and replayed with other starts and inputs, and calls of different sizes in turn on one workspace and another stream."""
    rng = np.random.default_rng(41)
    h_q, h_kv, d = 4, 1, 64
    x = made(rng, 640, h_q, h_kv, d, dtype)
    starts = starts_of([300, 340])
    ws = workspace(640, h_q, h_kv, d, 2)
    out = prompt(x, h_q, h_kv, d, [0, 0], dtype, True, 0.1, starts=starts, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        prompt(x, h_q, h_kv, d, [0, 0], dtype, True, 0.1, starts=starts, ws=ws, out=out)
    for new in ([300, 340], [1, 639], [640, 0], [7, 5]):
        starts.copy_(starts_of(new))
        x.copy_(made(rng, 640, h_q, h_kv, d, dtype))
        out.fill_(-3.0)
        g.replay()
        check_prompt(out[:sum(new)], x[:sum(new)], h_q, h_kv, d, new, dtype, True, 0.1)
        assert bool((out[sum(new):] == -3).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [prompt(x[:n], h_q, h_kv, d, [n], dtype, True, 0.1, ws=ws, stream=side) for n in (640, 3, 200)]
    side.synchronize()
    for n, o in zip((640, 3, 200), outs):
        check_prompt(o, x[:n], h_q, h_kv, d, [n], dtype, True, 0.1)
    assert moa.moa_device_status() == 0


def test_positive_values_over_many_rows():
    """What the tensor core cuts off its sums grows with the rows; 40000 positive values keep within the tolerance."""
    rng = np.random.default_rng(47)
    n, d, m = 40000, 64, 5
    x = np.abs(rng.standard_normal((n, 3 * d))).astype(np.float32)
    x[:, :2 * d] *= 0.05
    xd = torch.from_numpy(x).cuda().half()
    out = prompt(xd, 1, 1, d, [n], moa.F16, False, 0.1)
    h = xd.double().cpu().numpy()
    want, tol = attend_new64(h[:m, None, :d], h[None, :, d:2 * d], h[None, :, 2 * d:], 0.1, moa.F16, causal=False)
    close(out[:m], want, tol)
