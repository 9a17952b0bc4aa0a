"""The operators on a paged key/value cache, as cases: appending keys and values with the position
rotation on the way, single-query attention over caches held in 32, 16 and 4 bits, and reading rows back.

`run` computes them in plain torch operations, or, where `own` is true, with the calls of the package.
A cache is a pool of pages; row `i` of sequence `b` is row `i % page_size` of page
`page_table[b, i // page_size]`.  A row held in 4 bits is `d` codes from 0 to 15 (two to a byte, the even
feature in the low half) and a pair (scale, least value) in fp16; it stands for `scale * code + least`.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FORMATS = {"f32": 0, "bf16": 1, "f16": 2, "int4": 3}      # of a cache; the first three also name the types of tensors


def listed():
    return [
        # one sequence in a chat: the smallest calls, bound by their latency
        dict(name="attend_f16_one", op="attend", dtype="f16", fmt="f16", batch=1, h_q=8, h_kv=1, d=128, lo=257, hi=257, page=16),
        # a decode step of a batch whose sequences are of different ages (the library's multi-step workload, in bf16)
        dict(name="attend_bf16_batch", op="attend", dtype="bf16", fmt="bf16", batch=32, h_q=32, h_kv=8, d=128, lo=512, hi=2048, page=16),
        # rows of 64 features, groups of six heads, pages of an odd size, one sequence without rows
        dict(name="attend_f16_odd", op="attend", dtype="f16", fmt="f16", batch=47, h_q=24, h_kv=4, d=64, lo=0, hi=4999, page=20),
        # long documents, the largest cache in 16 bits
        dict(name="attend_bf16_long", op="attend", dtype="bf16", fmt="bf16", batch=4, h_q=64, h_kv=8, d=128, lo=100003, hi=131072, page=64),
        # the library's own type
        dict(name="attend_f32_batch", op="attend", dtype="f32", fmt="f32", batch=16, h_q=32, h_kv=8, d=128, lo=1000, hi=4096, page=32),
        # the 4-bit cache: one sequence, a serving batch, one K/V head for 16 query heads over long sequences
        dict(name="attend_int4_one", op="attend", dtype="bf16", fmt="int4", batch=1, h_q=32, h_kv=8, d=128, lo=901, hi=901, page=16),
        dict(name="attend_int4_batch", op="attend", dtype="bf16", fmt="int4", batch=64, h_q=32, h_kv=8, d=128, lo=1024, hi=8192, page=16),
        dict(name="attend_int4_long", op="attend", dtype="f16", fmt="int4", batch=8, h_q=16, h_kv=1, d=128, lo=60001, hi=131072, page=64),
        # the prompts of seven requests, and one token for each of 64 sequences
        dict(name="append_bf16_prompts", op="append", dtype="bf16", fmt="bf16", batch=7, h_q=32, h_kv=8, d=128, lo=301, hi=2047, past=100, page=16, rot=128, style="halves"),
        dict(name="append_bf16_step", op="append", dtype="bf16", fmt="bf16", batch=64, h_q=32, h_kv=8, d=128, lo=1, hi=1, past=255, page=16, rot=128, style="halves"),
        # the same into a 4-bit cache, and the new rows read back
        dict(name="append_int4_prompts", op="append", dtype="f16", fmt="int4", batch=5, h_q=32, h_kv=8, d=128, lo=33, hi=1900, past=77, page=32, rot=64, style="pairs"),
        dict(name="append_int4_step", op="append", dtype="bf16", fmt="int4", batch=96, h_q=16, h_kv=4, d=64, lo=1, hi=1, past=200, page=16, rot=64, style="halves"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["attend", "attend", "append"])
    fmt = rng.choice(["bf16", "f16", "int4", "int4", "f32"])
    dtype = rng.choice(["bf16", "f16"]) if fmt == "int4" else fmt
    d = rng.choice([64, 128, 128])
    h_kv = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 3, 4, 6, 7, 8, 12, 16])
    page = rng.choice([8, 16, 16, 20, 32, 64])
    batch = spread(1, 64)
    if op == "attend":
        rows = spread(64, 2_000_000 // h_kv)               # rows of all sequences
        hi = max(1, min(131072, rows // batch))
        lo = rng.randint(0, hi)
        return dict(op=op, dtype=dtype, fmt=fmt, batch=batch, h_q=group * h_kv, h_kv=h_kv, d=d, lo=lo, hi=hi, page=page)
    hi = max(1, spread(64, 8000) // batch)
    if rng.random() < 0.3:
        hi = 1
    lo = rng.randint(1, hi)
    h_q = min(group * h_kv, 32 // h_kv * h_kv)
    return dict(op=op, dtype=dtype, fmt=fmt, batch=batch, h_q=h_q, h_kv=h_kv, d=d, lo=lo, hi=hi, past=rng.randint(0, 300), page=page,
                rot=rng.choice([d, d, d // 2, 24]), style=rng.choice(["halves", "halves", "pairs"]))


def _sizes(case):
    """Rows of each sequence: spread over lo..hi; the first is the shortest, the last the longest."""
    n, lo, hi = case["batch"], case["lo"], case["hi"]
    return [hi if b == n - 1 else lo if b == 0 else lo + int((hi - lo) * ((b * 0.6180339887498949) % 1.0)) for b in range(n)]


def _past(case):
    return [int(case["past"] * (((b + 1) * 0.7548776662466927) % 1.0)) for b in range(case["batch"])]


def _pack(x):
    """Rows in 4 bits: codes two to a byte, and (scale, least value) in fp16."""
    least, most = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((most - least) * torch.tensor(1.0 / 15.0, dtype=torch.float32, device=x.device)).half()
    least = least.half()
    codes = torch.where(scale > 0, ((x - least.float()) / scale.float()).round().clamp(0, 15), torch.zeros_like(x)).to(torch.uint8)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), torch.cat([scale, least], -1)


def _unpack(packed, params, dtype):
    codes = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).to(dtype)
    return params[..., :1].to(dtype) * codes + params[..., 1:].to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    batch, h_q, h_kv, d, page = (case[k] for k in ("batch", "h_q", "h_kv", "d", "page"))
    dtype, fmt, new = DTYPES[case["dtype"]], case["fmt"], _sizes(case)
    past = _past(case) if case["op"] == "append" else [0] * batch
    lens = [a + b for a, b in zip(past, new)]
    need = [-(-n // page) for n in lens]
    pages, per_seq = sum(need) + 3, max(1, max(need))
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    at = torch.arange(per_seq, device="cuda")[None]
    need_t = torch.tensor(need, device="cuda")[:, None]
    start = need_t.cumsum(0) - need_t
    table = torch.where(at < need_t, order[(start + at).clamp(max=pages - 1)], torch.full((), -1, dtype=torch.int32, device="cuda")).contiguous()
    s = dict(case=case, table=table, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), per_seq=per_seq, pages=pages, scale=d ** -0.5)

    for name in ("k", "v"):
        drift = normal(h_kv, 1, d) if name == "k" else torch.zeros((), device="cuda")    # keys have features with an offset of their own
        pool = torch.empty((pages, h_kv, page, d // 2), dtype=torch.uint8, device="cuda") if fmt == "int4" else torch.empty((pages, h_kv, page, d), dtype=dtype, device="cuda")
        params = torch.zeros((pages, h_kv, page, 2), dtype=torch.float16, device="cuda")
        step = max(1, (1 << 26) // (h_kv * page * d))
        for i in range(0, pages, step):
            x = normal(min(step, pages - i), h_kv, page, d) + drift
            if case["op"] == "append":
                x = torch.zeros_like(x)
            if fmt == "int4":
                pool[i : i + step], params[i : i + step] = _pack(x)
            else:
                pool[i : i + step] = x
        s[name + "_pool"], s[name + "_params"] = pool, params

    if case["op"] == "attend":
        s["q"] = normal(batch, h_q, d).to(dtype)
        s["out"] = torch.empty_like(s["q"])
    else:
        tokens = sum(new)
        s["tokens"], s["longest"] = tokens, max(new)
        qkv = normal(tokens, (h_q + 2 * h_kv) * d).to(dtype)      # as one projection gives them
        s["q"], s["k"], s["v"] = (x.unflatten(-1, (-1, d)) for x in qkv.split([h_q * d, h_kv * d, h_kv * d], -1))
        s["q_out"] = torch.empty((tokens, h_q, d), dtype=dtype, device="cuda")
        s["starts"] = torch.tensor([sum(new[:b]) for b in range(batch + 1)], dtype=torch.int32, device="cuda")
        s["first"] = torch.tensor(past, dtype=torch.int32, device="cuda")
        rows, rot = 512 + case["past"] + max(new), case["rot"]
        angle = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
        s["cos_sin"], s["rope_rows"] = torch.cat([angle.cos(), angle.sin()], -1).float(), rows
        if fmt == "int4":
            s["k_back"], s["v_back"] = (torch.zeros((batch, h_kv, s["longest"], d), dtype=dtype, device="cuda") for _ in "kv")
    if own:
        import paper_2607_19456_b200 as moa

        more = dict(k_params=s["k_params"], v_params=s["v_params"]) if fmt == "int4" else {}
        s["cache"] = moa.PagedCache(FORMATS[fmt], s["k_pool"], s["v_pool"], pages, page, h_kv, d, **more)
        s["ws_bytes"] = moa.moa_paged_workspace_bytes(batch, h_q, h_kv, d)
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms ------------------------------------------------------------------


def _where(s):
    """Of each new token: its sequence, its place in it, and its row's page and place there."""
    t = torch.arange(s["tokens"], device="cuda")
    b = torch.searchsorted(s["starts"][1:].long(), t, right=True)
    i = t - s["starts"].long()[b]
    pos = s["first"].long()[b] + i
    page = s["case"]["page"]
    return b, i, pos, s["table"].long()[b, pos // page], pos % page


def _rotate(x, cos, sin, rot, style):
    x = x.float()
    if style == "pairs":
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2 : rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_append(s):
    case = s["case"]
    b, i, pos, page, row = _where(s)
    cos, sin = s["cos_sin"][pos][:, None].chunk(2, -1)
    s["q_out"].copy_(_rotate(s["q"], cos, sin, case["rot"], case["style"]))
    k, v = _rotate(s["k"], cos, sin, case["rot"], case["style"]), s["v"].float()
    at = (page[:, None], torch.arange(case["h_kv"], device="cuda")[None], row[:, None])
    if case["fmt"] != "int4":
        s["k_pool"][at], s["v_pool"][at] = k.to(s["k_pool"].dtype), v.to(s["v_pool"].dtype)
        return s["q_out"], s["k_pool"], s["v_pool"]
    (s["k_pool"][at], s["k_params"][at]), (s["v_pool"][at], s["v_params"][at]) = _pack(k), _pack(v)
    back = (b[:, None], at[1], i[:, None])
    s["k_back"][back] = _unpack(s["k_pool"][at], s["k_params"][at], torch.float32).to(s["k_back"].dtype)
    s["v_back"][back] = _unpack(s["v_pool"][at], s["v_params"][at], torch.float32).to(s["v_back"].dtype)
    return s["q_out"], s["k_back"], s["v_back"]


def _rows(s, name, dtype):
    """The rows of every sequence, [batch, h_kv, pages of a sequence * page, d]."""
    at = s["table"].long().clamp(min=0)
    x = s[name + "_pool"][at]
    x = _unpack(x, s[name + "_params"][at], dtype) if s["case"]["fmt"] == "int4" else x.to(dtype)
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    case = s["case"]
    q = s["q"].float().unflatten(1, (case["h_kv"], -1))
    scores = q @ _rows(s, "k", torch.float32).transpose(-1, -2) * s["scale"]
    seen = torch.arange(scores.shape[-1], device="cuda") < s["lens"][:, None, None, None]
    scores = scores.masked_fill(~seen, -math.inf)
    most = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = (scores - most).exp()
    total = p.sum(-1, keepdim=True)
    out = (p @ _rows(s, "v", torch.float32)) / total.masked_fill(total == 0, 1.0)
    return out.flatten(1, 2).to(s["q"].dtype)


def run(s):
    case = s["case"]
    if not own:
        return _plain_attend(s) if case["op"] == "attend" else _plain_append(s)
    import paper_2607_19456_b200 as moa

    dtype = FORMATS[case["dtype"]]
    if case["op"] == "attend":
        moa.moa_paged_decode_attn(s["cache"], s["q"], s["out"], dtype, case["h_q"] * case["d"], case["batch"], case["h_q"], s["lens"], s["table"],
                                  s["per_seq"], s["scale"], s["ws"], s["ws_bytes"])
        return s["out"]
    wide = (case["h_q"] + 2 * case["h_kv"]) * case["d"]
    moa.moa_paged_append(s["cache"], s["q"], s["k"], s["v"], s["q_out"], dtype, (wide, wide, wide, case["h_q"] * case["d"]), s["tokens"], case["h_q"],
                         case["batch"], s["starts"], s["lens"], s["table"], s["per_seq"], s["cos_sin"], s["rope_rows"], case["rot"],
                         moa.ROPE_PAIRS if case["style"] == "pairs" else moa.ROPE_HALVES)
    if case["fmt"] != "int4":
        return s["q_out"], s["k_pool"], s["v_pool"]
    moa.moa_paged_gather(s["cache"], s["k_back"], s["v_back"], dtype, case["batch"], s["longest"], s["first"], s["lens"], s["table"], s["per_seq"])
    return s["q_out"], s["k_back"], s["v_back"]


# ---- what a pass cannot do without -----------------------------------------------------


def work(case):
    size = DTYPES[case["dtype"]].itemsize
    row = case["d"] // 2 + 4 if case["fmt"] == "int4" else case["d"] * size
    rows, page, d = sum(_sizes(case)), case["page"], case["d"]
    if case["op"] == "attend":
        pages = sum(-(-n // page) for n in _sizes(case))
        return {"bytes": 2 * rows * case["h_kv"] * row + 2 * case["batch"] * case["h_q"] * d * size + 4 * pages + 4 * case["batch"],
                "flops": 4 * rows * case["h_q"] * d}
    heads = case["h_q"] + 2 * case["h_kv"]
    moved = rows * (heads * d * size + case["h_q"] * d * size + 2 * case["h_kv"] * row) + 4 * case["rot"] * min(rows, case["past"] + case["hi"])
    if case["fmt"] == "int4":                     # read back
        moved += rows * 2 * case["h_kv"] * (row + d * size)
    return {"bytes": moved, "flops": rows * (3 * case["rot"] * (case["h_q"] + case["h_kv"]) + (8 * d * case["h_kv"] if case["fmt"] == "int4" else 0))}


# ---- the definition in 64 bits ---------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    page, h_kv, d = case["page"], case["h_kv"], case["d"]
    lens, table = s["lens"].tolist(), s["table"].long()

    def stored(name, pages):
        rows = s[name + "_pool"][pages].transpose(0, 1).flatten(1, 2)
        if case["fmt"] != "int4":
            return rows.double()
        scale, least = s[name + "_params"][pages].transpose(0, 1).flatten(1, 2).double().unbind(-1)
        full = torch.empty((*rows.shape[:-1], d), dtype=torch.float64, device="cuda")
        full[..., 0::2], full[..., 1::2] = rows.bitwise_and(15).double(), rows.bitwise_right_shift(4).double()
        return full * scale[..., None] + least[..., None]

    if case["op"] == "attend":
        out = torch.zeros((case["batch"], case["h_q"], d), dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            if n == 0:
                continue
            pages = table[b, : -(-n // page)]
            keys, values = stored("k", pages)[:, :n], stored("v", pages)[:, :n]
            q = s["q"][b].double().reshape(h_kv, -1, d)
            weight = torch.softmax(torch.einsum("hgd,hnd->hgn", q, keys) * s["scale"], -1)
            out[b] = torch.einsum("hgn,hnd->hgd", weight, values).reshape(-1, d)
        return out

    starts, rot = s["starts"].tolist(), case["rot"]
    low = (torch.arange(0, rot, 2) if case["style"] == "pairs" else torch.arange(rot // 2)).cuda()
    high = low + (1 if case["style"] == "pairs" else rot // 2)

    def turn(x, at):
        x = x.double()
        c, z = s["cos_sin"][at].double()[:, None].tensor_split(2, -1)
        y = x.clone()
        y[..., low], y[..., high] = x[..., low] * c - x[..., high] * z, x[..., low] * z + x[..., high] * c
        return y

    def held(x):
        small, large = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
        step, floor = ((large - small) / 15).half().double(), small.half().double()
        return floor + step * torch.nan_to_num((x - floor) / step, nan=0.0, posinf=0.0, neginf=0.0).round().clamp(0, 15)

    q_out = torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")
    k_out, v_out = (torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in (("k_back", "v_back") if case["fmt"] == "int4" else ("k_pool", "v_pool")))
    for b, n in enumerate(lens):
        mine, at = slice(starts[b], starts[b + 1]), torch.arange(n - (starts[b + 1] - starts[b]), n, device="cuda")
        q_out[mine] = turn(s["q"][mine], at)
        k, v = turn(s["k"][mine], at), s["v"][mine].double()
        if case["fmt"] == "int4":
            k_out[b, :, : len(at)], v_out[b, :, : len(at)] = held(k).transpose(0, 1), held(v).transpose(0, 1)
        else:
            k_out[table[b, at // page], :, at % page], v_out[table[b, at // page], :, at % page] = k, v
    return q_out, k_out, v_out
