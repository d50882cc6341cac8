"""What the language side does with the embedding rows that an encode worker sends it, as measurable cases.

Four operators: attention over whole packed prompts (causal, grouped heads), the append of new keys and
values to a cache held in 8 bits with a scale for each page of tokens and head, that cache's rows read
back, and the attention of new tokens over it.  The prompts are what the encoders produce rows for: 577
rows of an image of the CLIP encoder, some hundreds to thousands of a variable-resolution image, 2,048 of a
video clip, 1,500 of an audio clip, each with a little text.  Head layouts: 28 heads of 128 over 4 (the width
3,584 of the connector's rows), 32 over 8, 16 of 64 over 16 or 4, 20 of 64 over 20.

A cache page holds `page` tokens of every key / value head: keys [pages, heads, page, dim], values
[pages, heads, dim, page], scales [pages, heads].  A block (a page's tokens of one head) is held as
code * 2^e, with e the smallest exponent under which its values fit (127 in int8, 448 in e4m3).

The plain forms pad a packed batch to its longest member, as torch operations need.
"""
import math

import torch

own = False

HEADS = ((28, 4, 128), (32, 8, 128), (16, 16, 64), (16, 4, 64), (20, 20, 64), (40, 8, 128), (32, 1, 128))
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
FORMATS = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}


def listed():
    return [
        # a short text turn on an idle worker: the latency of one call
        {"name": "prompt_short", "op": "prompt", "dtype": "bf16", "heads": 28, "kv_heads": 4, "dim": 128,
         "new": "37", "held": "0", "causal": True},
        # eight requests with images of several sizes and a little text, packed: an ordinary micro-batch
        {"name": "prompt_images_8", "op": "prompt", "dtype": "bf16", "heads": 28, "kv_heads": 4, "dim": 128,
         "new": "620,1201,97,2309,577,1764,333,915", "held": "0", "causal": True},
        # chunks of four long prompts, each over the rows that its earlier chunks left
        {"name": "prompt_chunks_4", "op": "prompt", "dtype": "fp16", "heads": 16, "kv_heads": 4, "dim": 64,
         "new": "1024,1024,700,1024", "held": "4096,2048,9216,511", "causal": True},
        # one request with eight video clips: a single long prompt, the largest attention work
        {"name": "prompt_video", "op": "prompt", "dtype": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "new": "16484", "held": "0", "causal": True},
        # a decoding step's new token of 16 requests
        {"name": "append_token_16", "op": "append", "dtype": "bf16", "format": "int8", "page": 64, "kv_heads": 4,
         "dim": 128, "new": ",".join(["1"] * 16), "held": "620,1201,97,2309,577,1764,333,915,64,1500,2048,63,8191,4000,12,0"},
        # two long prompts, one of them behind a cached prefix, into e4m3
        {"name": "append_prompts", "op": "append", "dtype": "fp16", "format": "e4m3", "page": 32, "kv_heads": 8,
         "dim": 128, "new": "16484,12111", "held": "0,1000"},
        # the cached prefixes of four requests, taken back for their next chunks
        {"name": "rows_prefix_4", "op": "rows", "dtype": "bf16", "format": "e4m3", "page": 16, "kv_heads": 16,
         "dim": 64, "held": "1500,577,2048,1201"},
        # sixteen long histories, moved to rows
        {"name": "rows_long_16", "op": "rows", "dtype": "bf16", "format": "int8", "page": 64, "kv_heads": 8,
         "dim": 128, "held": ",".join(["8192"] * 15 + ["8001"])},
        # the next token of one short request
        {"name": "decode_short", "op": "decode", "dtype": "bf16", "format": "int8", "page": 64, "heads": 28,
         "kv_heads": 4, "dim": 128, "new": "1", "held": "300"},
        # the next tokens of 32 requests of mixed lengths: an ordinary decoding step
        {"name": "decode_mixed_32", "op": "decode", "dtype": "bf16", "format": "int8", "page": 64, "heads": 28,
         "kv_heads": 4, "dim": 128, "new": ",".join(["1"] * 32),
         "held": "620,1201,97,2309,577,1764,333,915,64,1500,2048,63,8191,4000,12,1,"
                 "5000,777,1024,6001,2600,450,7300,130,999,3500,255,257,4600,1800,2222,8192"},
        # a few guessed tokens of eight requests, checked in one step
        {"name": "decode_guess_8", "op": "decode", "dtype": "fp16", "format": "e4m3", "page": 16, "heads": 16,
         "kv_heads": 4, "dim": 64, "new": "5,5,5,5,5,5,5,5", "held": "1200,577,9000,2048,4100,333,1500,7007"},
        # the next tokens of 16 requests with hours of video behind them: the largest cache
        {"name": "decode_long_16", "op": "decode", "dtype": "bf16", "format": "e4m3", "page": 64, "heads": 32,
         "kv_heads": 8, "dim": 128, "new": ",".join(["1"] * 16), "held": ",".join(["32768"] * 15 + ["30001"])},
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "append", "rows", "decode", "decode"])
    heads, kv_heads, dim = rng.choice(HEADS)
    case = {"op": op, "dtype": rng.choice(["bf16", "fp16"]), "kv_heads": kv_heads, "dim": dim}
    if op == "prompt":
        n = _log_int(rng, 1, 16)
        causal = rng.random() < 0.8
        new = [_log_int(rng, 1, (10000 if causal else 7000) // n) for _ in range(n)]
        held = [_log_int(rng, 1, 3000 // n) if rng.random() < 0.3 else 0 for _ in range(n)]
        return dict(case, heads=heads, causal=causal, new=",".join(map(str, new)),
                    held=",".join(map(str, held)))
    case.update(format=rng.choice(["int8", "e4m3"]), page=rng.choice([16, 32, 64, 128]))
    if op == "append":
        n = _log_int(rng, 1, 64)
        one = rng.random() < 0.4
        new = [1 if one else _log_int(rng, 1, 20000 // n) for _ in range(n)]
        held = [rng.choice([0, _log_int(rng, 1, 4000)]) for _ in range(n)]
        return dict(case, new=",".join(map(str, new)), held=",".join(map(str, held)))
    if op == "rows":
        n = _log_int(rng, 1, 32)
        return dict(case, held=",".join(str(_log_int(rng, 1, 60000 // n)) for _ in range(n)))
    n = _log_int(rng, 1, 64)
    new = 1 if rng.random() < 0.7 else rng.randint(2, 9)
    return dict(case, heads=heads, new=",".join([str(new)] * n),
                held=",".join(str(_log_int(rng, 1, 262144 // n)) for _ in range(n)))


def _ints(text):
    return [int(t) for t in text.split(",")]


def _lengths(case):
    """New tokens and tokens held before, of each request."""
    held = _ints(case["held"])
    new = _ints(case["new"]) if "new" in case else [0] * len(held)
    return new, held * len(new) if len(held) == 1 else held


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) % (1 << 62))
    return g


def _vectors(g, rows, heads, dim, dtype, spread=0.0):
    """Unit vectors' worth of noise; with `spread`, channels of unequal size, as keys have."""
    x = torch.randn((rows, heads, dim), generator=g, device="cuda")
    if spread:
        x *= torch.exp(spread * torch.randn((1, heads, dim), generator=g, device="cuda"))
    return x.to(dtype)


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _device_ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- the blocks' scales and codes (plain form) ------------------------------

def _needed(top, most):
    """The power of two under which values of up to `top` fit into [-most, most]; 0 where top is 0."""
    m, e = torch.frexp(top)                     # top = m 2^e, m in [0.5, 1)
    limit, bits = math.frexp(most)
    e = (e - bits + (m > limit)).clamp(min=-126)
    return torch.where(top > 0, ((e + 127) << 23).to(torch.int32).view(torch.float32), torch.zeros_like(top))


def _codes(x, scale, form):
    kind, most = FORMATS[form]
    inverse = (0x7F000000 - scale.view(torch.int32)).view(torch.float32)      # of a power of two, exactly
    y = x * torch.where(scale > 0, inverse, 0.0)
    y = torch.nan_to_num(y, nan=0.0, posinf=most, neginf=-most)
    return (torch.round(y) if kind == torch.int8 else y).to(kind)


def _magnitude(x):
    return torch.where(torch.isfinite(x), x.abs(), 0.0)


# ---- inputs -----------------------------------------------------------------

def _cache(case, g, held, total):
    """A cache with `held` tokens of each request in it and pages for `total`, its page table, shuffled."""
    page, h, d, form = case["page"], case["kv_heads"], case["dim"], case["format"]
    need = [-(-t // page) for t in total]
    order = torch.randperm(sum(need) + 1, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(total), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    pages = at + 1
    kind, most = FORMATS[form]
    gain = torch.exp(0.5 * torch.randn((1, h, 1, d), generator=g, device="cuda"))
    # which of a page's places hold tokens: the others keep code 0
    full = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    for r, n in enumerate(held):
        spots = torch.arange(n, device="cuda")
        full[table[r, spots // page].long(), spots % page] = True

    def blocks(scaled):
        codes = torch.zeros((pages, h, page, d), dtype=kind, device="cuda")
        scales = torch.zeros((pages, h), device="cuda")
        step = max(1, (1 << 26) // (h * page * d))
        for i in range(0, pages, step):
            x = torch.randn((min(step, pages - i), h, page, d), generator=g, device="cuda")
            x = (x * gain if scaled else x) * full[i:i + step, None, :, None]
            s = _needed(x.abs().amax((2, 3)), most)
            scales[i:i + step] = s
            codes[i:i + step] = _codes(x, s[..., None, None], form)
        return codes, scales

    k, ks = blocks(True)
    v, vs = blocks(False)
    v = v.view(torch.uint8).transpose(2, 3).contiguous().view(kind)
    return k, v, ks, vs, table


def prepare(case, seed):
    g, dtype = _generator(seed), DTYPES[case["dtype"]]
    new, held = _lengths(case)
    total = [a + b for a, b in zip(new, held)]
    h, d = case["kv_heads"], case["dim"]
    s = {"case": case, "n": len(new), "most_new": max(new), "most": max(total)}
    if case["op"] == "prompt":
        s.update(q=_vectors(g, sum(new), case["heads"], d, dtype), k=_vectors(g, sum(total), h, d, dtype, 0.5),
                 v=_vectors(g, sum(total), h, d, dtype), cu_q=_cu(new), cu_k=_cu(total))
        s.update(_places(new, "q"), **_places(total, "k"))
        return s
    k, v, ks, vs, table = _cache(case, g, held, total)
    s.update(k_codes=k, v_codes=v, k_scale=ks, v_scale=vs, pages=table, held=_device_ints(held),
             lens=_device_ints(total), cu_new=_device_ints(_cu(new)), same=len(set(new)) == 1)
    if case["op"] == "append":
        s.update(k=_vectors(g, sum(new), h, d, dtype, 0.5), v=_vectors(g, sum(new), h, d, dtype))
        # what is read back: from the start of the first page that gets a token
        first = [n // case["page"] * case["page"] for n in held]
        back = [t - f for t, f in zip(total, first)]
        s.update(first=_device_ints(first), cu_rows=_device_ints(_cu(back)), rows=sum(back), most_rows=max(back))
        s.update(_places(back, "r"))
    elif case["op"] == "rows":
        s.update(first=None, cu_rows=_device_ints(_cu(held)), rows=sum(held), most_rows=max(held))
        s.update(_places(held, "r"))
    else:
        s.update(q=_vectors(g, sum(new), case["heads"], d, dtype))
        s.update(_places(new, "q"))
    return s


def _places(lens, name):
    """Of each row of a packed batch: its request, and its place there."""
    n = torch.tensor(lens, device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), n)
    start = torch.cumsum(n, 0) - n
    return {name + "_seq": seq, name + "_at": torch.arange(sum(lens), device="cuda") - start[seq], name + "_len": n}


# ---- the operators ----------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _own(state)
    if case["op"] == "prompt":
        return _plain_prompt(state)
    if case["op"] == "decode":
        return _plain_decode(state)
    if case["op"] == "append":
        _plain_append(state)
    out = _plain_rows(state)
    if case["op"] == "append":
        out.update(k_scale=state["k_scale"], v_scale=state["v_scale"])
    return out


def _own(state):
    from paper_2609_31551_amd import attention
    case, dtype = state["case"], DTYPES[state["case"]["dtype"]]
    if case["op"] == "prompt":
        out, lse = attention.prompt_attention(state["q"], state["k"], state["v"], state["cu_q"], state["cu_k"],
                                              causal=case["causal"], with_lse=True)
        return {"out": out, "lse": lse}
    cache = attention.Kv8Cache(state["k_codes"], state["v_codes"], state["k_scale"], state["v_scale"])
    if case["op"] == "decode":
        out, lse = cache.attention(state["q"], state["lens"], state["pages"],
                                   cu_q=None if state["same"] else state["cu_new"], max_q=state["most_new"],
                                   max_len=state["most"], with_lse=True)
        return {"out": out, "lse": lse}
    if case["op"] == "append":
        cache.append(state["k"], state["v"], state["held"], state["pages"],
                     cu_new=None if state["same"] else state["cu_new"], max_new=state["most_new"])
    k, v = cache.rows(state["pages"], state["cu_rows"], state["rows"], first=state["first"],
                      max_len=state["most_rows"], dtype=dtype)
    out = {"k": k, "v": v}
    if case["op"] == "append":
        out.update(k_scale=state["k_scale"], v_scale=state["v_scale"])
    return out


def _padded(x, seq, at, n, longest):
    """[rows, heads, dim] -> [n, heads, longest, dim] in 32 bits."""
    y = torch.zeros((n, longest) + x.shape[1:], device=x.device)
    y[seq, at] = x.float()
    return y.transpose(1, 2).contiguous()


def _attend(q, k, v, q_len, k_len, causal):
    """q [n, heads, queries, dim] over k, v [n, kv_heads, keys, dim]; q_len, k_len: how many are real."""
    n, heads, nq, d = q.shape
    h, nk = k.shape[1], k.shape[2]
    s = q.reshape(n, h, heads // h * nq, d) @ k.transpose(2, 3).contiguous()
    s = s.mul_(d ** -0.5).view(n, h, heads // h, nq, nk)
    i = torch.arange(nq, device=q.device)[None, :, None]
    j = torch.arange(nk, device=q.device)[None, None, :]
    hidden = j >= k_len[:, None, None]
    if causal:
        hidden = hidden | (j > i + (k_len - q_len)[:, None, None])
    s.masked_fill_(hidden[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = s.sum(-1, keepdim=True)
    o = s.view(n, h, -1, nk) @ v
    o = o.view(n, h, heads // h, nq, d) / torch.where(total > 0, total, 1.0)
    return o.reshape(n, heads, nq, d), (top + total.log()).reshape(n, heads, nq)


def _plain_prompt(s):
    case, n = s["case"], s["n"]
    q = _padded(s["q"], s["q_seq"], s["q_at"], n, s["most_new"])
    k = _padded(s["k"], s["k_seq"], s["k_at"], n, s["most"])
    v = _padded(s["v"], s["k_seq"], s["k_at"], n, s["most"])
    o, lse = _attend(q, k, v, s["q_len"], s["k_len"], case["causal"])
    return {"out": o[s["q_seq"], :, s["q_at"]].to(s["q"].dtype), "lse": lse[s["q_seq"], :, s["q_at"]].contiguous()}


def _values(s):
    """The cache's values in 32 bits, by request: [n, kv_heads, tokens, dim] each; absent pages hold zeros."""
    table = s["pages"].long().clamp(min=0)

    def of(codes, scale):
        x = codes[table].float() * scale[table][..., None, None]
        return x * (s["pages"] >= 0)[:, :, None, None, None]

    def order(x):   # [n, pages, heads, page, dim]
        return x.transpose(1, 2).reshape(x.shape[0], x.shape[2], -1, x.shape[4])

    return order(of(s["k_codes"], s["k_scale"])), order(of(s["v_codes"], s["v_scale"]).transpose(3, 4))


def _plain_decode(s):
    k, v = _values(s)
    q = _padded(s["q"], s["q_seq"], s["q_at"], s["n"], s["most_new"])
    o, lse = _attend(q, k, v, s["q_len"], s["lens"].long(), True)
    return {"out": o[s["q_seq"], :, s["q_at"]].to(s["q"].dtype), "lse": lse[s["q_seq"], :, s["q_at"]].contiguous()}


def _plain_append(s):
    """Every page that gets tokens, [pages touched, heads, page, dim], with its earlier tokens' values."""
    case = s["case"]
    page, form, n = case["page"], case["format"], s["n"]
    most = FORMATS[form][1]
    at = torch.arange(s["pages"].shape[1] * page, device="cuda").view(1, -1, page)
    held, lens = s["held"].long()[:, None, None], s["lens"].long()[:, None, None]
    fresh, old = (at >= held) & (at < lens), at < held                        # [n, pages, page]
    seq, slot = torch.nonzero(fresh.any(-1), as_tuple=True)
    fresh, old, where = fresh[seq, slot][:, None, :, None], old[seq, slot][:, None, :, None], s["pages"][seq, slot].long()
    row = s["cu_new"].long()[seq, None] + at[0, slot] - s["held"].long()[seq, None]
    row = row.clamp(0, s["k"].shape[0] - 1)

    def one(codes, scale, x, turned):
        x = x[row].float().transpose(1, 2)                                    # [touched, heads, page, dim]
        x = torch.where(fresh, x, 0.0)
        was = codes[where]
        was = was.view(torch.uint8).transpose(2, 3).contiguous().view(codes.dtype) if turned else was
        before = torch.where(old.any(2)[..., 0], scale[where], 0.0)           # a new page's scale says nothing
        after = torch.maximum(before, _needed(_magnitude(x).amax((2, 3)), most))
        value = torch.where(fresh, x, was.float() * before[..., None, None])
        new = _codes(value, after[..., None, None], form)
        new = torch.where((fresh | old), new.view(torch.uint8), was.view(torch.uint8))
        new = new.transpose(2, 3).contiguous() if turned else new
        codes.view(torch.uint8)[where] = new
        scale[where] = after

    one(s["k_codes"], s["k_scale"], s["k"], False)
    one(s["v_codes"], s["v_scale"], s["v"], True)


def _plain_rows(s):
    case = s["case"]
    page, dtype = case["page"], DTYPES[case["dtype"]]
    at = s["r_at"] if s["first"] is None else s["r_at"] + s["first"].long()[s["r_seq"]]
    where = s["pages"].long()[s["r_seq"], at // page]
    k = s["k_codes"].view(torch.uint8)[where, :, at % page].view(s["k_codes"].dtype).float()
    v = s["v_codes"].view(torch.uint8)[where, :, :, at % page].view(s["v_codes"].dtype).float()
    return {"k": (k * s["k_scale"][where][..., None]).to(dtype), "v": (v * s["v_scale"][where][..., None]).to(dtype)}


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    new, held = _lengths(case)
    total = [a + b for a, b in zip(new, held)]
    h, d = case["kv_heads"], case["dim"]
    if case["op"] in ("prompt", "decode"):
        causal = case.get("causal", True)
        pairs = sum(a * b + a * (a + 1) // 2 if causal else a * (a + b) for a, b in zip(new, held))
        q = 2 * 2 * sum(new) * case["heads"] * d + 4 * sum(new) * case["heads"]
        each = 2 if case["op"] == "prompt" else 1
        return {"bytes": q + 2 * each * sum(total) * h * d, "flops": 4 * case["heads"] * d * pairs}
    if case["op"] == "rows":
        return {"bytes": (2 + 4) * sum(held) * h * d, "flops": 0}
    back = sum(t - n // case["page"] * case["page"] for t, n in zip(total, held))
    return {"bytes": (4 + 2) * sum(new) * h * d + 4 * back * h * d, "flops": 0}


# ---- the same results in 64 bits --------------------------------------------

def _exact_head(q, k, v, before, causal):
    """One head: q [queries, dim] over k, v [keys, dim], the first query behind `before` keys."""
    outs, sums = [], []
    for i in range(0, q.shape[0], 4096):
        s = q[i:i + 4096] @ k.t().contiguous() / math.sqrt(q.shape[1])
        if causal:
            last = torch.arange(i, i + s.shape[0], device=q.device) + before
            s = s.masked_fill(torch.arange(k.shape[0], device=q.device)[None] > last[:, None], -math.inf)
        lse = torch.logsumexp(s, 1)
        outs.append(torch.exp(s - torch.where(torch.isfinite(lse), lse, 0.0)[:, None]) @ v)
        sums.append(lse)
    return torch.cat(outs), torch.cat(sums)


def _exact_attention(q, k, v, new, total, causal):
    """Packed rows, request by request and head by head."""
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    group = q.shape[1] // k[0].shape[1]
    at = 0
    for r, (a, b) in enumerate(zip(new, total)):
        for h in range(q.shape[1]):
            kk, vv = k[r][:, h // group].double().contiguous(), v[r][:, h // group].double().contiguous()
            out[at:at + a, h], lse[at:at + a, h] = _exact_head(q[at:at + a, h].double().contiguous(), kk, vv, b - a, causal)
        at += a
    return {"out": out, "lse": lse}


def _exact_tokens(s, codes, scale, turned, r, length):
    """Request r's first `length` tokens as the cache holds them, [tokens, heads, dim]."""
    page = s["case"]["page"]
    where = s["pages"][r, :-(-length // page)].long()
    x = codes[where].double() * scale[where].double()[..., None, None]
    x = x.transpose(2, 3) if turned else x
    return x.transpose(1, 2).reshape(-1, x.shape[1], x.shape[3])[:length]


def _power(e):
    """2^e for whole e in 64 bits, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_blocks(s, codes, scale, turned, new, r, held):
    """Request r's tokens after the append of `new` [tokens, heads, dim], from its first touched page on, and
    those pages with their scales."""
    case = s["case"]
    page, (kind, most) = case["page"], FORMATS[case["format"]]
    first = held // page
    old = _exact_tokens(s, codes, scale, turned, r, held)[first * page:] if held else new[:0].double()
    every = torch.cat([old, new.double()])
    out, scales, pages = [], [], []
    for i in range(0, every.shape[0], page):
        x = every[i:i + page]
        where = int(s["pages"][r, first + i // page])
        earlier = max(0, old.shape[0] - i)                       # tokens of this page that were there before
        fresh = x[earlier:]
        top = fresh.abs().amax((0, 2))
        # smallest power of two with top / scale <= most
        e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / most))
        e = torch.where(top <= most * _power(e - 1), e - 1, torch.where(top > most * _power(e), e + 1, e)).clamp(min=-126)
        want = torch.where(top > 0, _power(e), 0.0)
        if earlier:
            want = torch.maximum(want, scale[where].double())
        y = x / torch.where(want > 0, want, 1.0)[None, :, None]
        # the last steps of a code: whole numbers, or 3 bits behind the leading one, at least 2^-9
        step = 1.0 if kind == torch.int8 else _power(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        out.append(torch.round(y / step) * step * want[None, :, None])
        scales.append(want)
        pages.append(where)
    return torch.cat(out), scales, pages


def exact(case, seed):
    s = prepare(case, seed)
    new, held = _lengths(case)
    total = [a + b for a, b in zip(new, held)]
    if case["op"] == "prompt":
        k = [s["k"][a:b] for a, b in zip(s["cu_k"], s["cu_k"][1:])]
        v = [s["v"][a:b] for a, b in zip(s["cu_k"], s["cu_k"][1:])]
        return _exact_attention(s["q"], k, v, new, total, case["causal"])
    sides = (("k", s["k_codes"], s["k_scale"], False), ("v", s["v_codes"], s["v_scale"], True))
    if case["op"] in ("rows", "decode"):
        back = {name: [_exact_tokens(s, codes, scale, turned, r, n) for r, n in enumerate(total)]
                for name, codes, scale, turned in sides}
        if case["op"] == "decode":
            return _exact_attention(s["q"], back["k"], back["v"], new, total, True)
        return {name: torch.cat(x) for name, x in back.items()}
    out, cu = {}, _cu(new)
    for name, codes, scale, turned in sides:
        rows, scales = [], scale.double().clone()
        for r in range(len(new)):
            x, sc, pages = _exact_blocks(s, codes, scale, turned, s[name][cu[r]:cu[r + 1]], r, held[r])
            rows.append(x)
            scales[torch.tensor(pages, device="cuda")] = torch.stack(sc)
        out[name], out[name + "_scale"] = torch.cat(rows), scales
    return out
