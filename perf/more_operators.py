"""What a prefill and a decoding worker do with prompts of images and video in pieces, as measurable cases.

Three operators: rotary positions with several axes (time, height, width) over the heads' rows, the append of
new keys and values to a paged 16-bit cache with that rotation on the way (the queries are rotated in the same
call), and the attention of a request's new tokens -- one, a few, or a chunk of its prompt -- over that cache.
Head layouts: 28 heads of 128 over 4 (the width 3,584 of the connector's rows), 32 or 40 over 8, 16 of 64 over
16 or 4, 20 of 64 over 20.  Prompts are the rows that the encoders produce (577 of an image, 2,048 of a video
clip, 1,500 of an audio clip) with a little text.

A cache page holds `page` tokens of every key / value head: keys and values [pages, heads, page, dim].
Positions are [axes, rows]; pair i of a head turns by position[axis of i] * theta ** (-i / pairs), or, with
`per_axis`, by theta ** (-j / n) as the axis's pair j of n.  A pair is (i, i + pairs) or, `adjacent`, (2 i, 2 i + 1).

The plain forms pad a packed batch to its longest member, as torch operations need.
"""
import functools
import math

import torch

own = False

HEADS = ((28, 4, 128), (32, 8, 128), (16, 16, 64), (16, 4, 64), (20, 20, 64), (40, 8, 128), (32, 1, 128))
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
# pairs of each axis, by the dimensions of a head: text alone, images and video, parts of a head
SECTIONS = {128: ("64", "16,24,24", "0,32,32", "32", "8,16,16", "24,20,20"), 64: ("32", "8,12,12", "0,16,16", "16", "4,2,2")}
MIXED = "620,1201,97,2309,577,1764,333,915,64,1500,2048,63,8191,4000,12,1," \
        "5000,777,1024,6001,2600,450,7300,130,999,3500,255,257,4600,1800,2222,8192"


def listed():
    wide = {"dtype": "bf16", "heads": 28, "kv_heads": 4, "dim": 128}
    video = {"sections": "16,24,24", "theta": 1e6, "per_axis": False, "adjacent": False}
    return [
        # the new tokens of 16 requests, before an attention that takes rotated rows: the latency of one call
        dict(wide, name="rotary_tokens_16", op="rotary", **video, new=",".join(["1"] * 16), held="4000", inverse=False),
        # eight requests with images of several sizes, half of each head rotated, as adjacent pairs
        {"name": "rotary_images_8", "op": "rotary", "dtype": "fp16", "heads": 16, "kv_heads": 4, "dim": 64,
         "sections": "4,6,6", "theta": 10000.0, "per_axis": True, "adjacent": True,
         "new": "620,1201,97,2309,577,1764,333,915", "held": "0", "inverse": False},
        # the gradient of a long prompt's rotation: eight video clips
        {"name": "rotary_video_back", "op": "rotary", "dtype": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, **video,
         "new": "16484", "held": "0", "inverse": True},
        # a decoding step's new token of 32 requests into the cache
        dict(wide, name="append_tokens_32", op="append", **video, page=64, new=",".join(["1"] * 32), held=MIXED),
        # chunks of four long prompts behind what their earlier chunks left
        {"name": "append_chunks_4", "op": "append", "dtype": "fp16", "heads": 16, "kv_heads": 4, "dim": 64,
         "sections": "8,12,12", "theta": 1e6, "per_axis": False, "adjacent": True, "page": 16,
         "new": "1024,1024,700,1024", "held": "4096,2048,9217,511"},
        # two long prompts with many video clips at once
        {"name": "append_prompts_2", "op": "append", "dtype": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, **video,
         "page": 32, "new": "16484,12111", "held": "0,1000"},
        # the next token of one short request
        dict(wide, name="token_short", op="attention", page=64, new="1", held="299"),
        # the next tokens of 32 requests of mixed lengths: an ordinary decoding step
        dict(wide, name="tokens_mixed_32", op="attention", page=64, new=",".join(["1"] * 32), held=MIXED),
        # the next tokens of 16 requests with hours of video behind them: the largest cache
        {"name": "tokens_long_16", "op": "attention", "dtype": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, "page": 64,
         "new": ",".join(["1"] * 16), "held": ",".join(["32768"] * 15 + ["30001"])},
        # a few guessed tokens of eight requests, checked in one step
        {"name": "guesses_8", "op": "attention", "dtype": "fp16", "heads": 16, "kv_heads": 4, "dim": 64, "page": 16,
         "new": "5,5,5,5,5,5,5,5", "held": "1200,577,9000,2048,4100,333,1500,7007"},
        # one step of a worker that mixes both: chunks of three prompts beside five requests' next tokens
        dict(wide, name="chunks_mixed_8", op="attention", page=32, new="1024,1,777,1,1,512,1,1",
             held="2048,1201,0,4000,333,6001,915,2309"),
        # a chunk of one long video prompt: the largest attention work
        dict(wide, name="chunk_long", op="attention", page=64, new="4096", held="32768"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["rotary", "append", "append", "attention", "attention", "attention"])
    heads, kv_heads, dim = rng.choice(HEADS)
    case = {"op": op, "dtype": rng.choice(["bf16", "fp16"]), "heads": heads, "kv_heads": kv_heads, "dim": dim}
    n = _log_int(rng, 1, 64)
    if op != "rotary":
        case["page"] = rng.choice([16, 32, 64, 128])
    if op == "attention":
        kind = rng.choice(["token", "token", "guess", "chunk", "chunk", "mixed"])
        if kind in ("token", "guess"):
            each = 1 if kind == "token" else rng.randint(2, 9)
            return dict(case, new=",".join([str(each)] * n),
                        held=",".join(str(_log_int(rng, 1, 262144 // n)) for _ in range(n)))
        new = [1 if kind == "mixed" and rng.random() < 0.5 else _log_int(rng, 1, 4096 // n) for _ in range(n)]
        held = [rng.choice([0, _log_int(rng, 1, 16384 // n)]) for _ in range(n)]
        return dict(case, new=",".join(map(str, new)), held=",".join(map(str, held)))
    case.update(sections=rng.choice(SECTIONS[dim]), theta=rng.choice([10000.0, 1e6, 5e5]), per_axis=rng.random() < 0.3,
                adjacent=rng.random() < 0.4)
    one = rng.random() < 0.4
    new = [1 if one else _log_int(rng, 1, 16000 // n) for _ in range(n)]
    held = [rng.choice([0, _log_int(rng, 1, 4000)]) for _ in range(n)]
    case.update(new=",".join(map(str, new)), held=",".join(map(str, held)))
    return dict(case, inverse=rng.random() < 0.3) if op == "rotary" else case


def _ints(text):
    return [int(t) for t in text.split(",")]


def _lengths(case):
    """New tokens and tokens held before, of each request."""
    new, held = _ints(case["new"]), _ints(case["held"])
    return new, held * len(new) if len(held) == 1 else held


def _pairs(case):
    """Of each rotated pair of a head: the axis that turns it, and its turn for one position, in radians."""
    sections = _ints(case["sections"])
    n = sum(sections)
    axis = [a for a, s in enumerate(sections) for _ in range(s)]
    place = [(j, s) for s in sections for j in range(s)] if case["per_axis"] else [(i, n) for i in range(n)]
    return axis, [case["theta"] ** (-j / s) for j, s in place]


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


# ---- inputs -----------------------------------------------------------------

def _positions(s, axes):
    """[axes, rows]: an eighth of each request's new tokens is text, in which all axes count on, the others are frames
    of 24 by 32 places."""
    text = s["q_len"][s["q_seq"]] // 8 + 1
    first = s["held"].long()[s["q_seq"]]
    j = (s["q_at"] - text).clamp(min=0)
    grid = torch.stack((j // 768, j // 32 % 24, j % 32, j // 768))[:axes]
    at = torch.where(s["q_at"] < text, s["q_at"], text + grid)
    return (first + at).to(torch.int32).contiguous()


def _cache(case, g, total):
    """Pages for `total` tokens of each request, filled, and the requests' page table, shuffled."""
    page, h, d, dtype = case["page"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
    need = torch.tensor([-(-t // page) for t in total], device="cuda")
    pages = int(need.sum()) + 1
    slot = torch.arange(int(need.max()), device="cuda")[None]
    place = (torch.cumsum(need, 0) - need)[:, None] + slot
    order = torch.randperm(pages, generator=g, device="cuda")
    table = torch.where(slot < need[:, None], order[place.clamp(max=pages - 1)], -1).to(torch.int32)
    gain = torch.exp(0.5 * torch.randn((1, h, 1, d), generator=g, device="cuda"))
    k = torch.empty((pages, h, page, d), dtype=dtype, device="cuda")
    v = torch.empty_like(k)
    step = max(1, (1 << 27) // (h * page * d))
    for i in range(0, pages, step):
        shape = (min(step, pages - i), h, page, d)
        k[i:i + step] = (torch.randn(shape, generator=g, device="cuda") * gain).to(dtype)
        v[i:i + step] = torch.randn(shape, generator=g, device="cuda").to(dtype)
    return k, v, table


def _places(lens):
    """Of each new row: its request, and its place among the new ones."""
    n = torch.tensor(lens, device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), n)
    start = torch.cumsum(n, 0) - n
    return {"q_seq": seq, "q_at": torch.arange(sum(lens), device="cuda") - start[seq], "q_len": n}


def prepare(case, seed):
    g, dtype = _generator(seed), DTYPES[case["dtype"]]
    new, held = _lengths(case)
    total = [a + b for a, b in zip(new, held)]
    heads, h, d, rows = case["heads"], case["kv_heads"], case["dim"], sum(new)
    s = {"case": case, "n": len(new), "most_new": max(new), "most": max(total), "same": len(set(new)) == 1,
         "held": _device_ints(held), "lens": _device_ints(total), "cu_new": _device_ints(_cu(new)),
         "q": _vectors(g, rows, heads, d, dtype)}
    s.update(_places(new))
    if case["op"] != "attention":
        s["k"] = _vectors(g, rows, h, d, dtype, 0.5)
        s["positions"] = _positions(s, len(_ints(case["sections"])))
    if case["op"] == "append":
        s["v"] = _vectors(g, rows, h, d, dtype)
    if case["op"] != "rotary":
        s["k_pages"], s["v_pages"], s["pages"] = _cache(case, g, total)
    return s


# ---- the operators ----------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _own(state)
    if case["op"] == "rotary":
        turn = _turns(state, -1.0 if case["inverse"] else 1.0)
        return {"q": _rotated(state["q"], case, *turn), "k": _rotated(state["k"], case, *turn)}
    if case["op"] == "append":
        return _plain_append(state)
    return _plain_attention(state)


@functools.lru_cache(maxsize=32)
def _rotary(sections, theta, per_axis, adjacent):
    """The plan of one model's positions, which its program keeps."""
    from paper_2609_31551_amd import paged
    return paged.Rotary.sections(_ints(sections), theta, per_axis=per_axis, adjacent=adjacent)


def _own(s):
    from paper_2609_31551_amd import paged
    case = s["case"]
    if case["op"] != "attention":
        rotary = _rotary(case["sections"], case["theta"], case["per_axis"], case["adjacent"])
    if case["op"] == "rotary":
        q, k = rotary.rows(s["q"], s["positions"], s["k"], inverse=case["inverse"])
        return {"q": q, "k": k}
    cache = paged.Kv16Cache(s["k_pages"], s["v_pages"])
    cu = None if s["same"] else s["cu_new"]
    if case["op"] == "append":
        q = cache.append(s["k"], s["v"], s["held"], s["pages"], cu_new=cu, max_new=s["most_new"], rotary=rotary,
                         positions=s["positions"], q=s["q"])
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    out, lse = cache.attention(s["q"], s["lens"], s["pages"], cu_q=cu, max_q=s["most_new"], max_len=s["most"],
                               with_lse=True)
    return {"out": out, "lse": lse}


def _turns(s, sign):
    """Cosine and sine of each row's pairs, [rows, 1, pairs]; the angles in 64 bits, as positions are far."""
    axis, freqs = _pairs(s["case"])
    angle = s["positions"].double()[axis].t() * torch.tensor(freqs, dtype=torch.float64, device="cuda") * sign
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _rotated(x, case, cos, sin):
    n, y = cos.shape[-1], x.float()
    if case["adjacent"]:
        a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        both = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = y[..., :n], y[..., n:2 * n]
        both = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((both, y[..., 2 * n:]), -1).to(x.dtype)


def _plain_append(s):
    case = s["case"]
    turn = _turns(s, 1.0)
    place = s["held"].long()[s["q_seq"]] + s["q_at"]
    page, slot = s["pages"].long()[s["q_seq"], place // case["page"]], place % case["page"]
    s["k_pages"][page, :, slot] = _rotated(s["k"], case, *turn)
    s["v_pages"][page, :, slot] = s["v"]
    return {"q": _rotated(s["q"], case, *turn), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attention(s):
    """Every request's tokens gathered from its pages, [requests, kv_heads, tokens, dim], and one masked softmax."""
    case, n, nq = s["case"], s["n"], s["most_new"]
    heads, h, d = case["heads"], case["kv_heads"], case["dim"]
    table = s["pages"].long().clamp(min=0)
    k = s["k_pages"][table].transpose(1, 2).reshape(n, h, -1, d).float()
    v = s["v_pages"][table].transpose(1, 2).reshape(n, h, -1, d).float()
    nk = k.shape[2]
    q = torch.zeros((n, nq, heads, d), device="cuda")
    q[s["q_seq"], s["q_at"]] = s["q"].float()
    q = q.transpose(1, 2).reshape(n, h, heads // h * nq, d)
    x = (q @ k.transpose(2, 3).contiguous()).mul_(d ** -0.5).view(n, h, heads // h, nq, nk)
    first = (s["lens"].long() - s["q_len"])[:, None, None]
    i, j = torch.arange(nq, device="cuda")[None, :, None], torch.arange(nk, device="cuda")[None, None]
    x.masked_fill_((j > i + first)[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.view(n, h, -1, nk) @ v).view(n, h, heads // h, nq, d) / total
    lse = (top + total.log()).view(n, heads, nq)
    return {"out": o.view(n, heads, nq, d)[s["q_seq"], :, s["q_at"]].to(s["q"].dtype),
            "lse": lse[s["q_seq"], :, s["q_at"]].contiguous()}


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    new, held = _lengths(case)
    heads, h, d, rows = case["heads"], case["kv_heads"], case["dim"], sum(new)
    if case["op"] == "attention":
        pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(new, held))
        return {"bytes": 4 * rows * heads * d + 4 * rows * heads + 4 * (rows + sum(held)) * h * d,
                "flops": 4 * heads * d * pairs}
    sections = _ints(case["sections"])
    turned = heads + h
    moved = turned + (h if case["op"] == "append" else 0)
    return {"bytes": 4 * rows * moved * d + 4 * rows * len(sections), "flops": 6 * rows * turned * sum(sections)}


# ---- the same results in 64 bits --------------------------------------------

def _exact_rotated(x, s, sign):
    """Each pair a complex number, times e^(i angle)."""
    case, d = s["case"], x.shape[2]
    axis, freqs = _pairs(case)
    n = len(axis)
    order = torch.arange(d, device="cuda")
    if not case["adjacent"]:
        order[:2 * n] = torch.stack((torch.arange(n), torch.arange(n, 2 * n)), 1).reshape(-1).cuda()
    y = x.double()[..., order].contiguous()
    pairs = torch.view_as_complex(y[..., :2 * n].reshape(x.shape[0], x.shape[1], n, 2).contiguous())
    angle = torch.stack([s["positions"][a].double() * (f * sign) for a, f in zip(axis, freqs)], 1)
    turned = pairs * torch.polar(torch.ones_like(angle), angle)[:, None]
    y[..., :2 * n] = torch.view_as_real(turned).flatten(-2)
    out = torch.empty_like(y)
    out[..., order] = y
    return out


def _exact_attention(s, new, total):
    q, page = s["q"], s["case"]["page"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    group = q.shape[1] // s["case"]["kv_heads"]
    at = 0
    for r, (a, b) in enumerate(zip(new, total)):
        where = s["pages"][r, :-(-b // page)].long()
        for h in range(q.shape[1]):
            kk = s["k_pages"][where, h // group].reshape(-1, q.shape[2])[:b].double()
            vv = s["v_pages"][where, h // group].reshape(-1, q.shape[2])[:b].double()
            for i in range(0, a, 2048):
                rows = slice(at + i, at + min(a, i + 2048))
                x = q[rows, h].double() @ kk.t().contiguous() / math.sqrt(q.shape[2])
                last = torch.arange(i, i + x.shape[0], device="cuda") + (b - a)
                x = x.masked_fill(torch.arange(b, device="cuda")[None] > last[:, None], -math.inf)
                lse[rows, h] = torch.logsumexp(x, 1)
                out[rows, h] = torch.softmax(x, 1) @ vv
        at += a
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    new, held = _lengths(case)
    if case["op"] == "rotary":
        sign = -1 if case["inverse"] else 1
        return {"q": _exact_rotated(s["q"], s, sign), "k": _exact_rotated(s["k"], s, sign)}
    if case["op"] == "attention":
        return _exact_attention(s, new, [a + b for a, b in zip(new, held)])
    k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
    k, at = _exact_rotated(s["k"], s, 1), 0
    for r, (a, b) in enumerate(zip(new, held)):
        places = torch.arange(b, a + b, device="cuda")
        page, slot = s["pages"][r].long()[places // case["page"]], places % case["page"]
        k_pages[page, :, slot] = k[at:at + a]
        v_pages[page, :, slot] = s["v"][at:at + a].double()
        at += a
    return {"q": _exact_rotated(s["q"], s, 1), "k_pages": k_pages, "v_pages": v_pages}
