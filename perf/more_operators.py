"""Operators of a paged cache held in 4 bits, as cases that can be timed and compared.

A case is a dict of plain values.  `op` says which operators it goes through:

  append      cs_paged_fp4_append, cs_paged_fp4_read: new key and value rows are quantised into the pages of their
              streams, and what the pages then hold of them is read back
  read        cs_paged_fp4_read: the keys and values of whole streams, as a program takes them that moves a stream to
              another cache
  attention   cs_paged_fp4_attention: a chunk of new rows per stream attends to the pages of its stream

An element is one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a sign (code 0 to 7, 8 for the sign), two to a byte, the even one
in the low half.  32 elements of a head's row share a scale s, a power of two held as its exponent + 127: the smallest
one with max|x| <= 7 s.  An element becomes the nearest code of x / s, ties to the even one.  A cache of one layer is
two pools of codes, `pages` pages with `page` tokens each, head-major or token-major, two pools of scales in which the
tokens of a page lie side by side, and a table that names the pages of every stream in order.  Pages are handed out in
random order, as they are in a server that has run for a while, and the table holds -1 behind a stream's last page.

Streams have between a quarter and all of `cached` tokens (`even`: all have it), and `rows` says how many new rows
each brings: "all" the same number, "ragged" down to a quarter of it, "mixed" the first stream a block of a prompt and
every other one token.  `pad` rows of the batch lie behind the last stream and belong to nobody.

Queries, keys and values are normal; queries of attention cases have a spread of 2, which makes attention about as
peaked as a trained model's.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 32


def listed():
    return [
        # ---- quantising as it is written, and reading back ----------------------------------------------
        # the rows of one verify step of eight streams: launches are what it costs
        dict(name="append_step", op="append", batch=8, rows="all", most=11, cached=18431, even=True, pad=0, kv_heads=8, hd=128, page=64,
             order="head", type="bf16"),
        # eight ragged prompts at once into small pages, token-major pools
        dict(name="append_prompts", op="append", batch=8, rows="ragged", most=2047, cached=0, even=True, pad=13, kv_heads=8, hd=128, page=32,
             order="token", type="bf16"),
        # float32 rows of a small model
        dict(name="append_f32", op="append", batch=5, rows="ragged", most=301, cached=700, even=False, pad=0, kv_heads=4, hd=64, page=32,
             order="head", type="f32"),
        # a stream of the tiny float32 configuration goes to another cache
        dict(name="read_tiny_f32", op="read", batch=1, cached=565, even=True, pad=0, kv_heads=4, hd=64, page=32, order="head", type="f32"),
        # twelve streams of up to 18431 tokens go to a cache of 16 bits
        dict(name="read_streams", op="read", batch=12, cached=18431, even=False, pad=7, kv_heads=8, hd=128, page=64, order="head", type="bf16"),
        # ---- attention over the pages -------------------------------------------------------------------
        # the tiny float32 configuration: one stream, one block of copied tokens, a short context
        dict(name="attn_tiny_f32", op="attention", batch=1, rows="all", most=11, cached=565, even=True, pad=0, heads=4, kv_heads=4, hd=64,
             page=32, order="head", type="f32", window=0),
        # single tokens: 64 streams in the middle of their answers
        dict(name="attn_decode", op="attention", batch=64, rows="all", most=1, cached=8191, even=False, pad=0, heads=32, kv_heads=8, hd=128,
             page=32, order="token", type="bf16", window=0),
        # the verify step of the benchmark's shape: eight streams, pending token and ten copied ones
        dict(name="attn_step", op="attention", batch=8, rows="all", most=11, cached=18431, even=True, pad=0, heads=32, kv_heads=8, hd=128,
             page=64, order="head", type="bf16", window=0),
        # long copy blocks behind a long context, seven query heads per KV head
        dict(name="attn_long_blocks", op="attention", batch=16, rows="all", most=33, cached=65535, even=True, pad=0, heads=28, kv_heads=4,
             hd=128, page=128, order="head", type="bf16", window=0),
        # one stream's prompt block rides along with fifteen streams that decode
        dict(name="attn_mixed", op="attention", batch=16, rows="mixed", most=2048, cached=16384, even=False, pad=3, heads=32, kv_heads=8,
             hd=128, page=32, order="head", type="bf16", window=0),
        # the first block of a prompt: what it sees it has just written
        dict(name="attn_prompt", op="attention", batch=1, rows="all", most=4096, cached=0, even=True, pad=0, heads=32, kv_heads=8, hd=128,
             page=64, order="token", type="bf16", window=0),
        # float32 prompt blocks
        dict(name="attn_f32_blocks", op="attention", batch=2, rows="ragged", most=700, cached=3001, even=False, pad=0, heads=8, kv_heads=2,
             hd=128, page=32, order="token", type="f32", window=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "read", "attention", "attention", "attention", "attention"])
    kind = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads, kv_heads = rng.choice([(4, 4), (32, 8), (32, 8), (28, 4), (64, 8), (16, 16), (8, 1)])
    hd = rng.choice([64, 96, 128, 128, 128, 256])
    case = dict(op=op, batch=_log_int(rng, 1, 64), even=rng.random() < 0.3, pad=rng.choice([0, 0, 5]), kv_heads=kv_heads, hd=hd,
                page=rng.choice([32, 32, 64, 128, 256]), order=rng.choice(["head", "token"]), type=kind)
    if op == "read":
        case["cached"] = _log_int(rng, 1, max(1, (1 << 27) // (case["batch"] * kv_heads * hd)))
        return case
    case["rows"] = rng.choice(["all", "all", "ragged", "mixed"])
    if op == "append":
        case["most"] = _log_int(rng, 1, max(1, min(4096, (1 << 24) // (case["batch"] * kv_heads * hd))))
        case["cached"] = rng.choice([0, _log_int(rng, 1, max(1, (1 << 26) // (case["batch"] * kv_heads * hd)))])
        return case
    kind_of = rng.choice(["token", "block", "prompt"])
    case["most"] = 1 if kind_of == "token" else _log_int(rng, 2, 48) if kind_of == "block" else _log_int(rng, 49, 4096)
    if kind == "f32":
        case["most"] = min(case["most"], 512)
    case["cached"] = _log_int(rng, 16, min(131072, (1 << 29) // (case["batch"] * kv_heads * hd)))
    if kind_of == "prompt" and rng.random() < 0.4:
        case["cached"] = 0
    if case["rows"] == "mixed" and case["most"] == 1:
        case["rows"] = "all"
    case.update(heads=heads, window=rng.choice([0, 0, 0, 1024]))
    top = 4e11 if kind == "bf16" else 4e10
    while work(case)["flops"] > top:               # no dearer than the largest listed one of the type
        if case["most"] > 1:
            case["most"] = max(1, case["most"] // 2)
        else:
            case["cached"] //= 2
    return case


# ---------------------------------------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------------------------------------

def _lengths(c):
    """Tokens that every stream has in the cache before the call."""
    B, n = c["batch"], c["cached"]
    return [n if c["even"] else n - (n * 3 * b) // (4 * B) for b in range(B)]


def _rows(c):
    """Rows that every stream brings, or that are read of it."""
    if c["op"] == "read":
        return _lengths(c)
    B, n = c["batch"], c["most"]
    if c["rows"] == "all":
        return [n] * B
    if c["rows"] == "mixed":
        return [n] + [1] * (B - 1)
    return [max(1, n - (n * 3 * b) // (4 * B)) for b in range(B)]


def _held(c):
    """Tokens that every stream has pages for."""
    return [n + (0 if c["op"] == "read" else r) for n, r in zip(_lengths(c), _rows(c))]


def _seen(c):
    """(query row, token) pairs, and tokens that somebody sees."""
    pairs = tokens = 0
    for length, rows in zip(_lengths(c), _rows(c)):
        w = c["window"]
        for i in range(rows):
            pairs += min(length + i + 1, w) if w else length + i + 1
        tokens += min(length + rows, w + rows - 1) if w else length + rows
    return pairs, tokens


def work(c):
    size = 2 if c["type"] == "bf16" else 4
    live = sum(_rows(c))
    n = 2 * live * c["kv_heads"] * c["hd"]                      # elements of the rows' keys and values
    if c["op"] == "append":                                     # rows in, codes and scales out, values out
        return {"bytes": 2 * n * size + n * 17 // 32, "flops": 3 * n}
    if c["op"] == "read":
        return {"bytes": n * size + n * 17 // 32, "flops": n}
    pairs, tokens = _seen(c)
    return {"bytes": 2 * tokens * c["kv_heads"] * c["hd"] * 17 // 32 + 2 * live * c["heads"] * c["hd"] * size,
            "flops": 4 * pairs * c["heads"] * c["hd"]}


# ---------------------------------------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------------------------------------

def _normal(shape, gen, dtype, spread=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * spread).to(dtype)


def _quantise(x):
    """float32 [..., hd] -> codes uint8 [..., hd/2], scales uint8 [..., hd/32]"""
    y = x.unflatten(-1, (-1, GROUP))
    top = y.abs().amax(-1)
    # the exponent of max|x|, one more where its mantissa exceeds 7/4, less that of 4
    held = (((top.view(torch.int32) + 0x1fffff) >> 23) - 2).clamp(min=2)
    a = y.abs() / (held << 23).view(torch.float32).unsqueeze(-1)
    code = (a > 0.25).to(torch.uint8)
    for border, even in ((0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)):
        code += (a > border) if even else (a >= border)
    code = (code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], held.to(torch.uint8)


def _values(codes, scales):
    """What codes uint8 [..., hd/2] and scales uint8 [..., hd/32] stand for, float32 [..., hd]"""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    at = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()
    s = (scales.to(torch.int32) << 23).view(torch.float32)
    return (table[at].unflatten(-1, (-1, GROUP)) * s.unsqueeze(-1)).flatten(-2)


def _pools(c, gen, total):
    """Codes [pages][kv_heads][page][hd/2] (token-major: [pages][page][kv_heads][hd/2]) and scales [pages][kv_heads][hd/32][page]
    of normal rows, made in pieces."""
    KVH, P, hd = c["kv_heads"], c["page"], c["hd"]
    head = c["order"] == "head"
    codes = torch.empty((total, KVH, P, hd // 2) if head else (total, P, KVH, hd // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((total, KVH, hd // GROUP, P), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 26) // (KVH * P * hd))
    for a in range(0, total, step):
        n = min(step, total - a)
        x, s = _quantise(torch.randn((n, KVH, P, hd), generator=gen, device=DEV))
        codes[a:a + n] = x if head else x.transpose(1, 2)
        scales[a:a + n] = s.transpose(2, 3)
    return codes, scales


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 1000003 + 29)
    dtype, hd, P = TYPES[c["type"]], c["hd"], c["page"]
    rows, held = _rows(c), _held(c)
    need = [-(-n // P) for n in held]
    total = sum(need) + 3
    s = {"case": c}
    s["k"], s["k_scale"] = _pools(c, gen, total)
    s["v"], s["v_scale"] = _pools(c, gen, total)
    names = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    s["table"] = torch.full((c["batch"], max(need) + 1), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        s["table"][b, :n] = names[at:at + n]
        at += n
    s["len"] = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    ends = [0]
    for r in rows:
        ends.append(ends[-1] + r)
    s["R"] = R = ends[-1] + c["pad"]
    # a batch of equal rows needs no offsets
    s["row0"] = None if len(set(rows)) == 1 and not c["pad"] else torch.tensor(ends, dtype=torch.int32, device=DEV)
    if c["op"] == "attention":
        s["q"] = _normal((R, c["heads"], hd), gen, dtype, 2.0)
        s["out"] = torch.zeros((R, c["heads"], hd), dtype=dtype, device=DEV)
    else:
        if c["op"] == "append":
            s["k_rows"] = _normal((R, c["kv_heads"], hd), gen, dtype)
            s["v_rows"] = _normal((R, c["kv_heads"], hd), gen, dtype)
        s["first"] = s["len"] if c["op"] == "append" else torch.zeros_like(s["len"])
        s["k_out"] = torch.zeros((R, c["kv_heads"], hd), dtype=dtype, device=DEV)
        s["v_out"] = torch.zeros((R, c["kv_heads"], hd), dtype=dtype, device=DEV)
    if own:
        from paper_2502_08923_amd import binding as cs
        view = (lambda t: t) if c["order"] == "head" else (lambda t: t.transpose(1, 2))
        s["handle"] = cs.PagesFP4(view(s["k"]), view(s["v"]), s["k_scale"], s["v_scale"], s["table"], s["len"])
    return s


# ---------------------------------------------------------------------------------------------------------
# the operators
# ---------------------------------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    return {"append": _plain_append, "read": _plain_read, "attention": _plain_attention}[c["op"]](state, c)


def _run_own(s, c):
    from paper_2502_08923_amd import binding as cs
    if c["op"] == "attention":
        return cs.cs_paged_fp4_attention(s["handle"], s["q"], row0=s["row0"], window=c["window"], max_rows=c["most"],
                                         max_len=c["cached"] + c["most"], out=s["out"])
    if c["op"] == "append":
        cs.cs_paged_fp4_append(s["handle"], s["k_rows"], s["v_rows"], row0=s["row0"])
    return cs.cs_paged_fp4_read(s["handle"], s["first"], row0=s["row0"], out=(s["k_out"], s["v_out"]))


def _places(s, c):
    """Page and slot of every row of the streams."""
    live, P = sum(_rows(c)), c["page"]
    r = torch.arange(live, device=DEV)
    if s["row0"] is None:
        b = r // _rows(c)[0]
        i = r - b * _rows(c)[0]
    else:
        b = torch.searchsorted(s["row0"][1:].long(), r, right=True)
        i = r - s["row0"].long()[b]
    pos = s["first"].long()[b] + i
    return live, s["table"].long()[b, pos // P], pos % P


def _at(c, pool, page, slot):
    """Rows [rows][kv_heads][hd/2] of a pool of codes."""
    return pool[page, :, slot] if c["order"] == "head" else pool[page, slot]


def _plain_read(s, c):
    live, page, slot = _places(s, c)
    for out, codes, scales in ((s["k_out"], s["k"], s["k_scale"]), (s["v_out"], s["v"], s["v_scale"])):
        step = max(1, (1 << 28) // (c["kv_heads"] * c["hd"]))
        for a in range(0, live, step):
            p, t = page[a:a + step], slot[a:a + step]
            out[a:min(live, a + step)] = _values(_at(c, codes, p, t), scales[p, :, :, t]).to(out.dtype)
    return s["k_out"], s["v_out"]


def _plain_append(s, c):
    live, page, slot = _places(s, c)
    for x, codes, scales in ((s["k_rows"], s["k"], s["k_scale"]), (s["v_rows"], s["v"], s["v_scale"])):
        code, scale = _quantise(x[:live].float())
        if c["order"] == "head":
            codes[page, :, slot] = code
        else:
            codes[page, slot] = code
        scales[page, :, :, slot] = scale
    return _plain_read(s, c)


def _plain_attention(s, c):
    H, KVH, hd, P, w = c["heads"], c["kv_heads"], c["hd"], c["page"], c["window"]
    G = H // KVH
    rows, lengths = _rows(c), _lengths(c)
    start = [0]
    for r in rows:
        start.append(start[-1] + r)
    out = s["out"]
    b = 0
    while b < c["batch"]:
        # streams with the same number of rows go together, as many as 4 GB of float32 keys or scores hold
        e, n = b, 0
        while e < c["batch"] and rows[e] == rows[b]:
            n = max(n, lengths[e] + rows[e])
            if e > b and (e + 1 - b) * n * max(KVH * hd, H * rows[b]) > 1 << 30:
                n = max(lengths[j] + rows[j] for j in range(b, e))
                break
            e += 1
        S, m = e - b, rows[b]
        pages = s["table"][b:e, :-(-n // P)].long().clamp(min=0)

        def tokens(codes, scales):
            t = codes[pages]                                             # [S][pages][KVH][P][hd/2] or [S][pages][P][KVH][hd/2]
            t = t.transpose(1, 2) if c["order"] == "head" else t.permute(0, 3, 1, 2, 4)
            f = scales[pages].permute(0, 2, 1, 4, 3)
            return _values(t.reshape(S, KVH, -1, hd // 2)[:, :, :n], f.reshape(S, KVH, -1, hd // GROUP)[:, :, :n])

        q = s["q"][start[b]:start[e]].view(S, m, KVH, G, hd).permute(0, 2, 1, 3, 4).reshape(S, KVH, m * G, hd).float()
        x = torch.matmul(q, tokens(s["k"], s["k_scale"]).transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(hd))
        last = s["len"][b:e].long()[:, None] + torch.arange(m, device=DEV)[None, :].repeat_interleave(G, 1)
        t = torch.arange(n, device=DEV)
        hidden = t[None, None, :] > last[:, :, None]
        if w:
            hidden = hidden | (t[None, None, :] <= last[:, :, None] - w)
        x.masked_fill_(hidden[:, None], -math.inf)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        y = torch.matmul(x, tokens(s["v"], s["v_scale"])) / x.sum(-1, keepdim=True)
        out[start[b]:start[e]] = y.view(S, KVH, m, G, hd).permute(0, 2, 1, 3, 4).reshape(S * m, H, hd).to(out.dtype)
        b = e
    return out


# ---------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------

def _power(n):
    """2^n in float64, exactly"""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _rounded(x):
    """float64 [..., hd] -> the values that its codes stand for: steps of 1/2 up to 2, of 1 up to 4, of 2 beyond."""
    y = x.unflatten(-1, (-1, GROUP))
    mantissa, power = torch.frexp(y.abs().amax(-1, keepdim=True))                        # mantissa in [1/2, 1)
    s = _power(torch.where(mantissa > 7 / 8, power - 2, power - 3).clamp(min=-125))
    a = y / s
    step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0))
    return ((torch.round(a / step) * step).clamp(-6, 6) * s).flatten(-2)


def _decoded(codes, scales):
    """Codes uint8 [..., hd/2], scales uint8 [..., hd/32] -> float64 [..., hd], by sign, exponent and mantissa"""
    both = torch.stack([codes.long() % 16, codes.long() // 16], dim=-1).flatten(-2)
    sign, power, half = 1.0 - 2.0 * (both // 8), both % 8 // 2, both % 2
    size = torch.where(power == 0, 0.5 * half, (1.0 + 0.5 * half) * _power(power - 1))
    return sign * size * torch.repeat_interleave(_power(scales.long() - 127), GROUP, dim=-1)


def exact(case, seed):
    c = case
    if c["op"] == "attention" and work(c)["flops"] > 3e12:
        return None
    s = prepare(case, seed)
    rows, lengths, P, KVH = _rows(c), _lengths(c), c["page"], c["kv_heads"]
    hd, table = c["hd"], s["table"].cpu()
    by_token = (lambda t: t.transpose(1, 2)) if c["order"] == "head" else (lambda t: t)      # [pages][P][KVH][hd/2]
    if c["op"] != "attention":
        out = []
        for side in ("k", "v"):
            y = torch.zeros(s[side + "_out"].shape, dtype=torch.float64, device=DEV)
            at = 0
            for b in range(c["batch"]):
                if c["op"] == "append":
                    y[at:at + rows[b]] = _rounded(s[side + "_rows"][at:at + rows[b]].double())
                else:
                    names = table[b][:-(-lengths[b] // P)].long().to(DEV)
                    y[at:at + rows[b]] = _decoded(by_token(s[side])[names].flatten(0, 1)[:rows[b]],
                                                  s[side + "_scale"].permute(0, 3, 1, 2)[names].flatten(0, 1)[:rows[b]])
                at += rows[b]
            out.append(y)
        return tuple(out)
    H = c["heads"]
    G = H // KVH
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for b in range(c["batch"]):
        n = lengths[b] + rows[b]
        names = table[b][:-(-n // P)].long().to(DEV)
        for g in range(KVH):
            k, v = (_decoded(by_token(s[side])[names, :, g].reshape(-1, hd // 2)[:n],
                             s[side + "_scale"][names, g].transpose(1, 2).reshape(-1, hd // GROUP)[:n]) for side in ("k", "v"))
            for r0 in range(0, rows[b], 512):
                r1 = min(rows[b], r0 + 512)
                q = s["q"][at + r0:at + r1, g * G:(g + 1) * G].double()
                x = torch.tensordot(q, k, dims=([2], [1])) / math.sqrt(hd)               # [rows][G][tokens]
                back = torch.arange(lengths[b] + r0, lengths[b] + r1, device=DEV)[:, None] - torch.arange(n, device=DEV)
                sees = (back >= 0) & ((back < c["window"]) if c["window"] else torch.ones_like(back, dtype=torch.bool))
                p = torch.softmax(torch.where(sees[:, None, :], x, torch.full_like(x, -math.inf)), dim=-1)
                out[at + r0:at + r1, g * G:(g + 1) * G] = torch.tensordot(p, v, dims=([2], [0]))
        at += rows[b]
    return out
