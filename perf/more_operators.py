"""Attention of many new tokens at once, and rotary positions with several axes, as cases: whole prompts packed one
behind the other, chunks of new tokens over a paged cache, and queries and keys turned by positions of up
to four axes, for themselves or on their way into a paged cache.

`run` computes them in plain torch operations, or, where `own` is true, with the calls of the package.
A cache is a pool of pages; row `i` of sequence `b` is row `i % page_size` of page
`page_table[b, i // page_size]`.  A row held in 4 bits is `d` codes from 0 to 15 (two to a byte, the even
feature in the low half) and a pair (scale, least value) in fp16; it stands for `scale * code + least`.
The tokens of all sequences lie one behind the other, as one projection gives them; `starts` says where each begins.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FORMATS = {"f32": 0, "bf16": 1, "f16": 2, "int4": 3}      # of a cache; the first three also name the types of tensors


def listed():
    return [
        # prompt: q, k, v of every token of a batch of prompts, lo..hi tokens each
        # one short question, one K/V head: the smallest call, bound by its latency
        dict(name="prompt_bf16_one", op="prompt", dtype="bf16", batch=1, h_q=8, h_kv=1, d=128, lo=77, hi=77, causal=True),
        # the prompts of seven requests
        dict(name="prompt_bf16_packed", op="prompt", dtype="bf16", batch=7, h_q=32, h_kv=8, d=128, lo=301, hi=2047, causal=True),
        # two long documents: the largest
        dict(name="prompt_bf16_long", op="prompt", dtype="bf16", batch=2, h_q=32, h_kv=8, d=128, lo=7001, hi=8192, causal=True),
        # an encoder: every token sees every token of its sequence; rows of 64, as many K/V heads as query heads, one sequence without tokens
        dict(name="prompt_f16_whole", op="prompt", dtype="f16", batch=23, h_q=16, h_kv=16, d=64, lo=0, hi=1500, causal=False),
        # the library's own type
        dict(name="prompt_f32_packed", op="prompt", dtype="f32", batch=4, h_q=32, h_kv=8, d=128, lo=99, hi=700, causal=True),
        # chunk: lo..hi new tokens behind some of `past` rows each, all in the cache already
        # draft tokens of one chat checked at once, and those of a batch (four each, sequences of different ages)
        dict(name="chunk_f16_one", op="chunk", dtype="f16", fmt="f16", batch=1, h_q=8, h_kv=1, d=128, lo=5, hi=5, past=300, page=16),
        dict(name="chunk_bf16_drafts", op="chunk", dtype="bf16", fmt="bf16", batch=64, h_q=32, h_kv=8, d=128, lo=4, hi=4, past=8192, page=16),
        # a long document's next piece
        dict(name="chunk_bf16_long", op="chunk", dtype="bf16", fmt="bf16", batch=1, h_q=32, h_kv=8, d=128, lo=2048, hi=2048, past=60000, page=64),
        # pages of an odd size, groups of six heads, pieces of very different length
        dict(name="chunk_f16_odd", op="chunk", dtype="f16", fmt="f16", batch=13, h_q=24, h_kv=4, d=64, lo=1, hi=700, past=4999, page=20),
        # the 4-bit cache: pieces of prompts beside single tokens
        dict(name="chunk_int4_mixed", op="chunk", dtype="bf16", fmt="int4", batch=16, h_q=32, h_kv=8, d=128, lo=1, hi=512, past=8192, page=16),
        # axes: queries and keys of 9k image patches turned by (time, height, width) ...
        dict(name="axes_bf16_patches", op="axes", dtype="bf16", fmt="none", batch=6, h_q=16, h_kv=16, d=64, lo=700, hi=2301, axes=3, order="runs", rot=64, style="halves"),
        # ... and on the way into a cache, one token for each of 64 sequences
        dict(name="axes_bf16_step", op="axes", dtype="bf16", fmt="bf16", batch=64, h_q=32, h_kv=8, d=128, lo=1, hi=1, past=255, page=16, axes=3, order="turns", rot=128, style="halves"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["prompt", "prompt", "chunk", "chunk", "axes"])
    d = rng.choice([64, 128, 128])
    h_kv = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 3, 4, 4, 6, 7, 8])
    h_q = min(group * h_kv, 32 // h_kv * h_kv)
    case = dict(op=op, d=d, h_q=h_q, h_kv=h_kv)
    if op == "prompt":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        hi = spread(16, 2048 if dtype == "f32" else 8192)
        batch = min(64, spread(1, max(1, 16384 // hi)))
        while batch * h_q * hi * hi > 3.0e9:
            hi = hi * 3 // 4
        return dict(case, dtype=dtype, batch=batch, lo=rng.randint(0, hi), hi=hi, causal=rng.random() < 0.7)
    page = rng.choice([8, 16, 16, 20, 32, 64])
    if op == "chunk":
        fmt = rng.choice(["bf16", "f16", "int4", "f32"])
        dtype = rng.choice(["bf16", "f16"]) if fmt == "int4" else fmt
        hi = spread(1, 1024 if fmt in ("bf16", "f16") else 300)
        batch = spread(1, 32)
        past = spread(16, 32000)
        while batch * h_q * hi * (hi + past) > 2.0e9 or batch * h_kv * (hi + past) > 1_000_000:
            batch, hi, past = max(1, batch * 3 // 4), max(1, hi * 3 // 4), past * 3 // 4
        return dict(case, dtype=dtype, fmt=fmt, batch=batch, lo=rng.randint(1, hi), hi=hi, past=past, page=page)
    fmt = rng.choice(["none", "none", "bf16", "f16", "f32"])
    batch = spread(1, 32)
    hi = max(1, spread(64, 9000) // batch)
    if fmt != "none" and rng.random() < 0.3:
        hi = 1
    return dict(case, dtype=rng.choice(["bf16", "f16", "f32"]) if fmt == "none" else fmt, fmt=fmt, batch=batch, lo=rng.randint(1, hi), hi=hi, past=rng.randint(0, 300), page=page,
                axes=rng.choice([2, 3, 3, 4]), order=rng.choice(["runs", "turns"]), rot=rng.choice([d, d, d // 2, 24]), style=rng.choice(["halves", "halves", "pairs"]))


def _sizes(case):
    """New tokens of each sequence: spread over lo..hi; the first is the shortest, the last the longest."""
    n, lo, hi = case["batch"], case["lo"], case["hi"]
    return [hi if b == n - 1 else lo if b == 0 else lo + int((hi - lo) * ((b * 0.6180339887498949) % 1.0)) for b in range(n)]


def _past(case):
    """Rows that each sequence has before them: an eighth of `past` to all of it; none in a prompt."""
    past = case.get("past", 0)
    return [past if case["batch"] == 1 else past // 8 + int(past * 7 / 8 * (((b + 1) * 0.7548776662466927) % 1.0)) for b in range(case["batch"])]


def _pack(x):
    """Rows in 4 bits: codes two to a byte, and (scale, least value) in fp16."""
    least, most = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((most - least) * torch.tensor(1.0 / 15.0, dtype=torch.float32, device=x.device)).half()
    least = least.half()
    codes = torch.where(scale > 0, ((x - least.float()) / scale.float()).round().clamp(0, 15), torch.zeros_like(x)).to(torch.uint8)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), torch.cat([scale, least], -1)


def _axis_of_pair(case):
    """Which axis turns each pair: runs of neighbouring pairs (the first axis the longest), or the axes by turns."""
    pairs, axes = case["rot"] // 2, case["axes"]
    if case["order"] == "turns":
        return [i % axes for i in range(pairs)]
    each = pairs // (axes + 1)
    return [max(0, axes - 1 - (pairs - 1 - i) // each) if each else 0 for i in range(pairs)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    op, batch, h_q, h_kv, d = (case[k] for k in ("op", "batch", "h_q", "h_kv", "d"))
    dtype, fmt, new, past = DTYPES[case["dtype"]], case.get("fmt", "none"), _sizes(case), _past(case)
    lens = [a + b for a, b in zip(past, new)]
    tokens = sum(new)
    s = dict(case=case, tokens=tokens, longest=max(new), scale=d ** -0.5, past=torch.tensor(past, dtype=torch.int32, device="cuda"),
             starts=torch.tensor([sum(new[:b]) for b in range(batch + 1)], dtype=torch.int32, device="cuda"),
             lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))

    if fmt != "none":
        page = case["page"]
        need = [-(-n // page) for n in lens]
        pages, per_seq = sum(need) + 3, max(1, max(need))
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        at = torch.arange(per_seq, device="cuda")[None]
        need_t = torch.tensor(need, device="cuda")[:, None]
        start = need_t.cumsum(0) - need_t
        s["table"] = torch.where(at < need_t, order[(start + at).clamp(max=pages - 1)], torch.full((), -1, dtype=torch.int32, device="cuda")).contiguous()
        s["pages"], s["per_seq"] = pages, per_seq
        for name in ("k", "v"):
            drift = normal(h_kv, 1, d) if name == "k" else torch.zeros((), device="cuda")    # keys have features with an offset of their own
            pool = torch.empty((pages, h_kv, page, d // 2), dtype=torch.uint8, device="cuda") if fmt == "int4" else torch.zeros((pages, h_kv, page, d), dtype=dtype, device="cuda")
            params = torch.zeros((pages, h_kv, page, 2), dtype=torch.float16, device="cuda")
            step = max(1, (1 << 26) // (h_kv * page * d))
            for i in range(0, pages if op == "chunk" else 0, step):
                x = normal(min(step, pages - i), h_kv, page, d) + drift
                if fmt == "int4":
                    pool[i : i + step], params[i : i + step] = _pack(x)
                else:
                    pool[i : i + step] = x
            s[name + "_pool"], s[name + "_params"] = pool, params

    if op == "chunk":
        s["q"] = normal(tokens, h_q, d).to(dtype)
    else:
        qkv = normal(tokens, (h_q + 2 * h_kv) * d)
        qkv[:, h_q * d : (h_q + h_kv) * d] += normal(h_kv * d)
        s["q"], s["k"], s["v"] = (x.unflatten(-1, (-1, d)) for x in qkv.to(dtype).split([h_q * d, h_kv * d, h_kv * d], -1))
    if op == "axes":
        rot, axes = case["rot"], case["axes"]
        # the first axis counts frames, the others lie inside them; a cache's next tokens are at positions of their own too
        rows = 600 + max(lens)
        s["positions"] = torch.randint(0, rows, (axes, tokens), generator=gen, device="cuda", dtype=torch.int32)
        angle = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
        s["cos_sin"], s["rope_rows"] = torch.cat([angle.cos(), angle.sin()], -1).float(), rows
        s["axis_of_pair"] = torch.tensor(_axis_of_pair(case), device="cuda")
        s["q_out"] = torch.empty((tokens, h_q, d), dtype=dtype, device="cuda")
        s["k_out"] = torch.empty((tokens, h_kv, d), dtype=dtype, device="cuda")
    else:
        s["out"] = torch.empty((tokens, h_q, d), dtype=dtype, device="cuda")

    if own:
        import paper_2607_19456_b200 as moa

        if fmt != "none":
            more = dict(k_params=s["k_params"], v_params=s["v_params"]) if fmt == "int4" else {}
            s["cache"] = moa.PagedCache(FORMATS[fmt], s["k_pool"], s["v_pool"], pages, page, h_kv, d, **more)
        if op == "axes":
            s["map"] = bytes(_axis_of_pair(case))
        else:
            s["ws_bytes"] = moa.moa_prompt_workspace_bytes(tokens, h_q, h_kv, d, batch)
            s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms ------------------------------------------------------------------


def _where(s):
    """Of each new token: its sequence, its place among the new ones, and its row in the sequence."""
    t = torch.arange(s["tokens"], device="cuda")
    b = torch.searchsorted(s["starts"][1:].long(), t, right=True)
    i = t - s["starts"].long()[b]
    return b, i, s["past"].long()[b] + i


def _unpack(packed, params):
    codes = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).float()
    return params[..., :1].float() * codes + params[..., 1:].float()


def _rows(s, name):
    """The rows of every sequence, [batch, h_kv, rows, d]."""
    case = s["case"]
    if case["op"] == "prompt":
        b, i, _ = _where(s)
        x = torch.zeros((case["batch"], s["longest"], case["h_kv"], case["d"]), device="cuda")
        x[b, i] = s[name].float()
        return x.transpose(1, 2)
    at = s["table"].long().clamp(min=0)
    x = s[name + "_pool"][at]
    x = _unpack(x, s[name + "_params"][at]) if case["fmt"] == "int4" else x.float()
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    case = s["case"]
    b, i, row = _where(s)
    g = case["h_q"] // case["h_kv"]
    q = torch.zeros((case["batch"], s["longest"], case["h_q"], case["d"]), device="cuda")
    q[b, i] = s["q"].float()
    q = q.unflatten(2, (case["h_kv"], g)).permute(0, 2, 3, 1, 4).flatten(2, 3)                   # [batch, h_kv, g * tokens, d]
    scores = q @ _rows(s, "k").transpose(-1, -2)
    scores = scores.mul_(s["scale"]).unflatten(2, (g, s["longest"]))
    key = torch.arange(scores.shape[-1], device="cuda")
    last = s["past"].long()[:, None] + torch.arange(s["longest"], device="cuda")                  # [batch, tokens]
    if not case.get("causal", True):
        last = (s["lens"].long()[:, None] - 1).expand_as(last)
    hidden = (key > last[..., None]) | (key >= s["lens"][:, None, None])
    scores.masked_fill_(hidden[:, None, None], -math.inf)
    scores.sub_(scores.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = (scores.flatten(2, 3) @ _rows(s, "v")).unflatten(2, (g, s["longest"])) / total.masked_fill(total == 0, 1.0)
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)                                                # [batch, tokens, h_q, d]
    s["out"].copy_(out[b, i])
    return s["out"]


def _rotate(x, cos, sin, rot, style):
    x = x.float()
    if style == "pairs":
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2 : rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_axes(s):
    case = s["case"]
    rot = case["rot"]
    at = s["positions"].long()[s["axis_of_pair"]].T                                               # [tokens, pairs]
    pair = torch.arange(rot // 2, device="cuda")
    cos, sin = s["cos_sin"][at, pair][:, None], s["cos_sin"][at, rot // 2 + pair][:, None]
    s["q_out"].copy_(_rotate(s["q"], cos, sin, rot, case["style"]))
    k = _rotate(s["k"], cos, sin, rot, case["style"])
    if case["fmt"] == "none":
        s["k_out"].copy_(k)
        return s["q_out"], s["k_out"]
    b, i, row = _where(s)
    page = case["page"]
    place = (s["table"].long()[b, row // page][:, None], torch.arange(case["h_kv"], device="cuda")[None], (row % page)[:, None])
    s["k_pool"][place], s["v_pool"][place] = k.to(s["k_pool"].dtype), s["v"].to(s["v_pool"].dtype)
    return s["q_out"], s["k_pool"], s["v_pool"]


def run(s):
    case = s["case"]
    if not own:
        return _plain_axes(s) if case["op"] == "axes" else _plain_attend(s)
    import paper_2607_19456_b200 as moa

    dtype, h_q, h_kv, d = FORMATS[case["dtype"]], case["h_q"], case["h_kv"], case["d"]
    wide = (h_q + 2 * h_kv) * d
    if case["op"] == "prompt":
        moa.moa_prompt_attn(s["q"], s["k"], s["v"], s["out"], dtype, (wide, wide, wide, h_q * d), s["tokens"], h_q, h_kv, d, case["batch"], s["starts"],
                            case["causal"], s["scale"], s["ws"], s["ws_bytes"])
        return s["out"]
    if case["op"] == "chunk":
        moa.moa_paged_chunk_attn(s["cache"], s["q"], s["out"], dtype, h_q * d, s["tokens"], h_q, case["batch"], s["starts"], s["lens"], s["table"], s["per_seq"],
                                 s["scale"], s["ws"], s["ws_bytes"])
        return s["out"]
    style = moa.ROPE_PAIRS if case["style"] == "pairs" else moa.ROPE_HALVES
    if case["fmt"] == "none":
        moa.moa_rotate_axes(s["q"], s["k"], s["q_out"], s["k_out"], dtype, (wide, wide, h_q * d, h_kv * d), s["tokens"], h_q, h_kv, d, s["positions"], case["axes"],
                            s["map"], s["cos_sin"], s["rope_rows"], case["rot"], style)
        return s["q_out"], s["k_out"]
    moa.moa_paged_append_axes(s["cache"], s["q"], s["k"], s["v"], s["q_out"], dtype, (wide, wide, wide, h_q * d), s["tokens"], h_q, case["batch"], s["starts"], s["lens"],
                              s["table"], s["per_seq"], s["positions"], case["axes"], s["map"], s["cos_sin"], s["rope_rows"], case["rot"], style)
    return s["q_out"], s["k_pool"], s["v_pool"]


# ---- what a pass cannot do without -----------------------------------------------------


def work(case):
    size = DTYPES[case["dtype"]].itemsize
    new, past, h_q, h_kv, d = _sizes(case), _past(case), case["h_q"], case["h_kv"], case["d"]
    tokens = sum(new)
    if case["op"] == "axes":
        moved = 2 * tokens * (h_q + (h_kv if case["fmt"] == "none" else 2 * h_kv)) * d * size
        return {"bytes": moved + 4 * tokens * case["axes"] + 4 * case["rot"] * min(tokens, 600), "flops": 3 * case["rot"] * tokens * (h_q + h_kv)}
    row = d // 2 + 4 if case.get("fmt") == "int4" else d * size
    rows = sum(new) + sum(past)
    seen = sum(n * p + (n * (n + 1) // 2 if case.get("causal", True) else n * n) for n, p in zip(new, past))
    table = 4 * sum(-(-(n + p) // case["page"]) for n, p in zip(new, past)) if case["op"] == "chunk" else 0
    return {"bytes": 2 * rows * h_kv * row + 2 * tokens * h_q * d * size + table + 8 * case["batch"], "flops": 4 * seen * h_q * d}


# ---- the definition in 64 bits ---------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    h_kv, d = case["h_kv"], case["d"]
    starts, lens = s["starts"].tolist(), s["lens"].tolist()

    def stored(name, b, n):
        """Rows of a sequence, [h_kv, n, d]."""
        if case["op"] == "prompt":
            return s[name][starts[b] : starts[b + 1]].double().transpose(0, 1)
        pages = s["table"][b, : -(-n // case["page"])].long()
        rows = s[name + "_pool"][pages].transpose(0, 1).flatten(1, 2)[:, :n]
        if case["fmt"] != "int4":
            return rows.double()
        scale, least = s[name + "_params"][pages].transpose(0, 1).flatten(1, 2)[:, :n].double().unbind(-1)
        full = torch.empty((h_kv, n, d), dtype=torch.float64, device="cuda")
        full[..., 0::2], full[..., 1::2] = rows.bitwise_and(15).double(), rows.bitwise_right_shift(4).double()
        return full * scale[..., None] + least[..., None]

    if case["op"] != "axes":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            m = starts[b + 1] - starts[b]
            if m == 0:
                continue
            keys, values = stored("k", b, n), stored("v", b, n)
            q = s["q"][starts[b] : starts[b + 1]].double().reshape(m, h_kv, -1, d)
            step = max(1, 200_000_000 // (n * case["h_q"]))
            for i in range(0, m, step):
                logit = torch.einsum("mhgd,hnd->hgmn", q[i : i + step], keys) * s["scale"]
                if case.get("causal", True):
                    logit = logit + torch.full((m, n), -math.inf, dtype=torch.float64, device="cuda").triu(n - m + 1)[i : i + step]
                weight = torch.softmax(logit, -1)
                out[starts[b] + i : starts[b] + min(m, i + step)] = torch.einsum("hgmn,hnd->mhgd", weight, values).flatten(1, 2)
        return out

    rot = case["rot"]
    low = (torch.arange(0, rot, 2) if case["style"] == "pairs" else torch.arange(rot // 2)).cuda()
    high = low + (1 if case["style"] == "pairs" else rot // 2)

    def turn(x):
        x = x.double()
        y = x.clone()
        for i, axis in enumerate(_axis_of_pair(case)):
            turned_by = s["cos_sin"][s["positions"][axis].long()].double()
            c, z = turned_by[:, i, None], turned_by[:, rot // 2 + i, None]
            y[..., low[i]], y[..., high[i]] = x[..., low[i]] * c - x[..., high[i]] * z, x[..., low[i]] * z + x[..., high[i]] * c
        return y

    q_out, k = turn(s["q"]), turn(s["k"])
    if case["fmt"] == "none":
        return q_out, k
    k_pool, v_pool = (torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("k_pool", "v_pool"))
    for b, n in enumerate(lens):
        mine = slice(starts[b], starts[b + 1])
        at = torch.arange(n - (starts[b + 1] - starts[b]), n, device="cuda")
        pages = s["table"][b].long()[at // case["page"]]
        k_pool[pages, :, at % case["page"]], v_pool[pages, :, at % case["page"]] = k[mine], s["v"][mine].double()
    return q_out, k_pool, v_pool
