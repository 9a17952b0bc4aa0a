"""Paged caches for the tests: pools with NaN in every place that no call may read, and the plain
64-bit form of what the operators compute."""
import numpy as np
import torch

import paper_2607_19456_b200 as moa

TYPES = {moa.F32: torch.float32, moa.BF16: torch.bfloat16, moa.F16: torch.float16}
NAMES = {moa.KV_F32: "f32", moa.KV_BF16: "bf16", moa.KV_F16: "f16", moa.KV_INT4: "int4"}


def dtype_of(fmt, dtype=None):
    return (moa.BF16 if dtype is None else dtype) if fmt == moa.KV_INT4 else fmt


def pack4(x):
    """Rows (numpy fp32) in 4 bits, every operation in fp32: codes uint8 [..., d/2], (scale, least) fp16 [..., 2]."""
    x = x.astype(np.float32)
    mn, mx = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        s = np.minimum((mx - mn) * np.float32(1.0 / 15.0), np.float32(65504)).astype(np.float16)
        m = np.clip(mn, -65504, 65504).astype(np.float16)
        c = np.rint((x - m.astype(np.float32)) / s.astype(np.float32))
        odd = ~np.isfinite(x).all(-1, keepdims=True)
        c = np.where((s > 0) & ~odd, np.clip(np.nan_to_num(c, nan=0.0, posinf=15.0, neginf=0.0), 0, 15), 0).astype(np.uint8)
    p = np.concatenate([s, m], -1)
    p[np.broadcast_to(odd, p.shape)] = np.nan
    return c[..., 0::2] | (c[..., 1::2] << 4), p


def unpack4(codes, params):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    return params[..., :1].astype(np.float64) * c + params[..., 1:].astype(np.float64)


class Paged:
    """A cache of `batch` sequences of `lens` rows on `device`, its pages in random order.  Unused rows and pages
    hold NaN, unused table entries hold numbers that no pool has.  heads_inner: [page, row, head, d] pools."""

    def __init__(self, rng, fmt, lens, h_kv, d, page, heads_inner=False, spare=3, extra_pages=1, k=None, v=None, device="cuda"):
        self.fmt, self.lens, self.h_kv, self.d, self.page = fmt, list(lens), h_kv, d, page
        batch = len(self.lens)
        need = [-(-n // page) for n in self.lens]
        self.max_pages = max(1, max(need) + extra_pages)
        self.num_pages = sum(need) + spare
        order = rng.permutation(self.num_pages).astype(np.int32)
        self.table_host = np.full((batch, self.max_pages), -7, np.int32)
        self.table_host[:, 1::2] = 1 << 30
        self.values = {}
        shape = (self.num_pages, h_kv, page, d)
        host = {"k": np.full(shape, np.nan, np.float32), "v": np.full(shape, np.nan, np.float32)}
        at = 0
        for b, n in enumerate(self.lens):
            mine = order[at:at + need[b]]
            at += need[b]
            self.table_host[b, :need[b]] = mine
            for name, given in (("k", k), ("v", v)):
                x = rng.standard_normal((h_kv, n, d)).astype(np.float32) if given is None else given[b].astype(np.float32)
                if name == "k" and given is None:
                    x += rng.standard_normal((h_kv, 1, d)).astype(np.float32)
                for i in range(need[b]):
                    rows = x[:, i * page:(i + 1) * page]
                    host[name][mine[i], :, :rows.shape[1]] = rows
        self.pools, self.params = {}, {}
        for name in "kv":
            if fmt == moa.KV_INT4:
                codes, params = pack4(host[name])
                pool = torch.from_numpy(codes).to(device)
                self.params[name] = torch.from_numpy(params).to(device)
                self.values[name] = unpack4(codes, params)
            else:
                pool = torch.from_numpy(host[name]).to(device).to(TYPES[fmt])
                self.values[name] = pool.double().cpu().numpy()
            self.pools[name] = pool.transpose(1, 2).contiguous().transpose(1, 2) if heads_inner else pool
        width = d // 2 if fmt == moa.KV_INT4 else d
        per = d // width
        strides = {n: tuple(int(s) * per for s in self.pools[n].stride()[:3]) for n in "kv"}
        self.table = torch.from_numpy(self.table_host).to(device)
        self.lens_dev = torch.tensor(self.lens, dtype=torch.int32, device=device)
        self.cache = moa.PagedCache(fmt, self.pools["k"], self.pools["v"], self.num_pages, page, h_kv, d, strides["k"],
                                    strides["v"], self.params.get("k"), self.params.get("v"))

    def rows(self, name, b, n=None):
        """Rows of sequence b in 64 bits, [h_kv, n, d]."""
        n = self.lens[b] if n is None else n
        pages = self.table_host[b, :-(-n // self.page)]
        x = self.values[name][pages].transpose(1, 0, 2, 3).reshape(self.h_kv, -1, self.d)
        return x[:, :n]


def attend64(q, p, scale, lens=None):
    """The definition: q float64 [batch, h_q, d] -> (out, bound), the bound without the rounding of the output.

    Per head: a score's error is at most 2^-19 of scale * sum|q||k| (fp32 sums of d products, 2^-22 or less for each of
    the d/16 accumulations); a weight's error is twice that, relatively; 2^-16 covers the two-term probabilities (2^-17), exp2
    and the sums.  4 bits: weights are rounded to fp16 (2^-12 of scale*15), or flushed below 2^-25 of their range."""
    batch, h_q, d = q.shape
    out, bound = np.zeros_like(q), np.zeros_like(q)
    g = h_q // p.h_kv
    for b in range(batch):
        n = p.lens[b] if lens is None else lens[b]
        if n <= 0:
            continue
        k, v = p.rows("k", b, n), p.rows("v", b, n)
        for h in range(h_q):
            with np.errstate(invalid="ignore"):            # (infinite queries)
                s = scale * (k[h // g] @ q[b, h])
            w = np.exp(s - s.max())
            out[b, h] = (w / w.sum()) @ v[h // g]
            size = abs(scale) * (np.abs(k[h // g]) @ np.abs(q[b, h])).max()
            if p.fmt == moa.KV_INT4:        # the score is a sum of two parts, each up to the range of the row
                size = abs(scale) * np.abs(q[b, h]).sum() * 2 * np.abs(k[h // g]).max()
            top = np.abs(v[h // g]).max()
            bound[b, h] = top * (2.0 ** -18 * size + 2.0 ** -16)
            if p.fmt == moa.KV_INT4:
                span = (v[h // g].max(-1) - v[h // g].min(-1)).max() + 1e-30
                bound[b, h] += span * (2.0 ** -12 + n * 2.0 ** -31)
    return out, bound


def workspace(batch, h_q, h_kv, d, fill=0xA5):
    n = moa.moa_paged_workspace_bytes(batch, h_q, h_kv, d)
    return torch.full((n,), fill, dtype=torch.uint8, device="cuda"), n


def attend(p, q, dtype, scale, lens=None, out=None, ws=None, q_stride=0, stream=None):
    """The call, on device tensors; q [batch, h_q, d] (or with a stride between sequences)."""
    batch, h_q, d = q.shape
    out = torch.full((batch, h_q, d), -3.0, dtype=TYPES[dtype], device="cuda") if out is None else out
    ws = workspace(batch, h_q, p.h_kv, d) if ws is None else ws
    moa.moa_paged_decode_attn(p.cache, q, out, dtype, q_stride, batch, h_q, p.lens_dev if lens is None else lens, p.table,
                              p.max_pages, scale, ws[0], ws[1], stream)
    return out


def rotate32(x, pos, cos_sin, rot, pairs):
    """x fp32 [tokens, heads, d] turned by its positions, every operation rounded to fp32."""
    y = x.astype(np.float32).copy()
    if rot == 0:
        return y
    c, s = cos_sin[pos][:, None, :rot // 2], cos_sin[pos][:, None, rot // 2:]
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = y[..., lo].copy(), y[..., hi].copy()
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    return y


def rope_table(rows, rot):
    angle = np.arange(rows, dtype=np.float64)[:, None] * 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / max(rot, 1))
    return np.concatenate([np.cos(angle), np.sin(angle)], -1).astype(np.float32)
