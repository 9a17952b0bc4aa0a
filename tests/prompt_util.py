"""Attention of many new tokens for the tests: the definition in 64 bits with a bound of what the kernels may be off, and the calls."""
import numpy as np
import torch

import paper_2607_19456_b200 as moa
from paged_util import TYPES


def bound64(out, weight, v, size, n, dtype, steps4=None):
    """How far an output row may be off, before anything else is known.

    Scores: 2^-19 of scale * sum|q||k| (fp32 sums of d products, cut off instead of rounded), a weight is off by twice that,
    relatively.  Weights of 16 bits are rounded to eps/2 of them on the way into the sum (their own sum is of the unrounded
    ones), made to 2^-13 (bf16: a polynomial of degree 3 for some of them) or 2^-18; fp16 drops what is below 2^-33 of the
    heaviest.  The tensor core's sums are cut off at 2^-23 for every 16 rows.  fp32: two terms of 11 bits each, 2^-20.
    4 bits: what is rounded is weight * scale, and stands for at most 8 steps of the row."""
    top = np.abs(v).max() if v.size else 0.0
    eps = torch.finfo(TYPES[dtype]).eps
    if dtype == moa.F32:
        return top * (2.0 ** -18 * size + 2.0 ** -19 + n * 2.0 ** -27)
    rounded = weight @ (np.abs(v) if steps4 is None else np.broadcast_to(8 * steps4[:, None], v.shape))
    made = 2.0 ** -13 if dtype == moa.BF16 else 2.0 ** -18 + n * 2.0 ** -33
    return eps / 2 * rounded + top * (2.0 ** -18 * size + 2 * made + 2.0 ** -17 + n / 16 * 2.0 ** -23)


def attend_new64(q, k, v, scale, dtype, causal=True, steps4=None):
    """q [m, h_q, d], k, v [h_kv, n, d] in float64; token i of the m sees rows up to n - m + i.  -> (out, tolerance)"""
    m, h_q, d = q.shape
    h_kv, n, _ = k.shape
    out, tol = np.zeros_like(q), np.zeros_like(q)
    eps = torch.finfo(TYPES[dtype]).eps
    for h in range(h_q):
        kk, vv = k[h // (h_q // h_kv)], v[h // (h_q // h_kv)]
        s = scale * (q[:, h] @ kk.T)
        if causal:
            s = np.where(np.arange(n)[None] > (n - m + np.arange(m))[:, None], -np.inf, s)
        with np.errstate(invalid="ignore"):
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
        out[:, h] = w @ vv
        size = (abs(scale) * (np.abs(q[:, h]) @ np.abs(kk).T)).max(-1, keepdims=True)
        if steps4 is not None:                              # the score is a sum of two parts, each up to the range of the row
            size = abs(scale) * np.abs(q[:, h]).sum(-1, keepdims=True) * 2 * np.abs(kk).max()
        tol[:, h] = bound64(out[:, h], w, vv, size, n, dtype, None if steps4 is None else steps4[h // (h_q // h_kv)])
    return out, tol + eps / 2 * np.abs(out) + 2.0 ** -25


def close(got, want, tol, what=None):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    off = np.abs(got - want)
    assert np.all(off <= tol), (what, float(off.max()), float((off / tol).max()))


def workspace(tokens, h_q, h_kv, d, batch, fill=0xA5):
    n = moa.moa_prompt_workspace_bytes(tokens, h_q, h_kv, d, batch)
    return torch.full((n,), fill, dtype=torch.uint8, device="cuda"), n


def starts_of(new, device="cuda"):
    return torch.tensor(np.concatenate([[0], np.cumsum(new)]).astype(np.int32), device=device)


def prompt(qkv, h_q, h_kv, d, new, dtype, causal, scale, out=None, ws=None, starts=None, stream=None):
    """The call on slices of one projection's output [tokens, (h_q + 2 h_kv) d]."""
    tokens, wide = qkv.shape
    q, k, v = (x.unflatten(-1, (-1, d)) for x in qkv.split([h_q * d, h_kv * d, h_kv * d], -1))
    out = torch.full((tokens, h_q, d), -3.0, dtype=TYPES[dtype], device="cuda") if out is None else out
    ws = workspace(tokens, h_q, h_kv, d, len(new)) if ws is None else ws
    moa.moa_prompt_attn(q, k, v, out, dtype, (wide, wide, wide, h_q * d), tokens, h_q, h_kv, d, len(new),
                        starts_of(new) if starts is None else starts, causal, scale, ws[0], ws[1], stream)
    return out


def check_prompt(out, qkv, h_q, h_kv, d, new, dtype, causal, scale, skip=()):
    x = qkv.double().cpu().numpy()
    at = 0
    for b, n in enumerate(new):
        if n and b not in skip:
            q, k, v = np.split(x[at:at + n], [h_q * d, (h_q + h_kv) * d], -1)
            q, k, v = (y.reshape(n, -1, d) for y in (q, k, v))
            want, tol = attend_new64(q, k.transpose(1, 0, 2), v.transpose(1, 0, 2), scale, dtype, causal)
            close(out[at:at + n], want, tol, b)
        at += n


def chunk(p, q, new, dtype, scale, lens=None, starts=None, out=None, ws=None, q_stride=0, stream=None, uniform=False):
    tokens, h_q, d = q.shape
    batch = len(new)
    out = torch.full((tokens, h_q, d), -3.0, dtype=TYPES[dtype], device="cuda") if out is None else out
    ws = workspace(tokens, h_q, p.h_kv, d, batch) if ws is None else ws
    starts = None if uniform else starts_of(new) if starts is None else starts
    moa.moa_paged_chunk_attn(p.cache, q, out, dtype, q_stride, tokens, h_q, batch, starts, p.lens_dev if lens is None else lens, p.table,
                             p.max_pages, scale, ws[0], ws[1], stream)
    return out


def check_chunk(out, p, q, new, dtype, scale, skip=()):
    x = q.double().cpu().numpy()
    at = 0
    for b, m in enumerate(new):
        if m and b not in skip:
            k, v = p.rows("k", b), p.rows("v", b)
            steps = None
            if p.fmt == moa.KV_INT4:
                pages = p.table_host[b, :-(-p.lens[b] // p.page)]
                par = p.params["v"].double().cpu().numpy()[pages][..., 0]
                steps = par.transpose(1, 0, 2).reshape(p.h_kv, -1)[:, :p.lens[b]]
            want, tol = attend_new64(x[at:at + m], k, v, scale, dtype, steps4=steps)
            close(out[at:at + m], want, tol, b)
        at += m
