"""Operators of serving over a paged cache, as cases that can be timed and compared.

A case is a dict of plain values.  `op` says which operator it goes through:

  norm_rope   cs_op_qk_norm_rope: RMSNorm of every query and key head and the rotary embedding, in one pass
  append      cs_paged_append: new key and value rows into the pages of a cache, keys rotated on the way
  attention   cs_paged_attention: a chunk of new rows per stream attends to the pages of its stream

A paged cache of one layer is two pools of `pages` pages with `page` tokens each, and a table that names the pages of
every stream in order.  Pages are handed out in random order, as they are in a server that has run for a while, and the
table holds -1 behind a stream's last page.  Streams have between a quarter and all of `cached` tokens (`even`: all have
it), and `rows` says how many new rows each brings: "all" the same number, "ragged" down to a quarter of it, "mixed" the
first stream a block of a prompt and every other one token.  `pad` rows of the batch lie behind the last stream and
belong to nobody.

Queries and keys have unit variance per element; queries of attention cases have twice that spread, which makes
attention about as peaked as a trained model's.
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # ---- head norms and rotation ------------------------------------------------------------------
        # one verify step of eight streams at the 8B shape: 88 rows, where a launch is what it costs
        dict(name="norm_rope_step", op="norm_rope", rows=88, heads=32, kv_heads=8, hd=128, rot=128, type="bf16", far=18442, norm=True),
        # a prompt block of the same shape: a stream of memory
        dict(name="norm_rope_prompt", op="norm_rope", rows=4096, heads=32, kv_heads=8, hd=128, rot=128, type="bf16", far=16384, norm=True),
        # float32 rows (what the projections hand out), an odd number of them, seven query heads per KV head
        dict(name="norm_rope_f32", op="norm_rope", rows=1531, heads=28, kv_heads=4, hd=128, rot=128, type="f32", far=131072, norm=True),
        # ---- appending to the pages -------------------------------------------------------------------
        # the rows of one verify step of eight streams
        dict(name="append_step", op="append", batch=8, rows="all", most=11, cached=18431, even=True, pad=0, kv_heads=8, hd=128, page=64,
             order="head", type="bf16"),
        # eight ragged prompts at once into small pages, token-major pools
        dict(name="append_prompts", op="append", batch=8, rows="ragged", most=2047, cached=0, even=True, pad=13, kv_heads=8, hd=128, page=16,
             order="token", type="bf16"),
        # float32 cache of a small model
        dict(name="append_f32", op="append", batch=5, rows="ragged", most=301, cached=700, even=False, pad=0, kv_heads=4, hd=64, page=32,
             order="head", type="f32"),
        # ---- attention over the pages -----------------------------------------------------------------
        # the tiny float32 configuration: one stream, one block of copied tokens, a short context
        dict(name="attn_tiny_f32", op="attention", batch=1, rows="all", most=11, cached=565, even=True, pad=0, heads=4, kv_heads=4, hd=64,
             page=16, order="head", type="f32", window=0),
        # single tokens: 64 streams in the middle of their answers
        dict(name="attn_decode", op="attention", batch=64, rows="all", most=1, cached=8191, even=False, pad=0, heads=32, kv_heads=8, hd=128,
             page=16, order="token", type="bf16", window=0),
        # the verify step of the benchmark's shape: eight streams, pending token and ten copied ones
        dict(name="attn_step", op="attention", batch=8, rows="all", most=11, cached=18431, even=True, pad=0, heads=32, kv_heads=8, hd=128,
             page=64, order="head", type="bf16", window=0),
        # long copy blocks behind a long context, seven query heads per KV head
        dict(name="attn_long_blocks", op="attention", batch=16, rows="all", most=33, cached=65535, even=True, pad=0, heads=28, kv_heads=4,
             hd=128, page=128, order="head", type="bf16", window=0),
        # one stream's prompt block rides along with fifteen streams that decode
        dict(name="attn_mixed", op="attention", batch=16, rows="mixed", most=2048, cached=16384, even=False, pad=3, heads=32, kv_heads=8,
             hd=128, page=32, order="head", type="bf16", window=0),
        # float32 prompt blocks
        dict(name="attn_f32_blocks", op="attention", batch=2, rows="ragged", most=700, cached=3001, even=False, pad=0, heads=8, kv_heads=2,
             hd=128, page=32, order="token", type="f32", window=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rope", "append", "attention", "attention", "attention"])
    kind = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads, kv_heads = rng.choice([(4, 4), (32, 8), (32, 8), (28, 4), (64, 8), (16, 16), (8, 1)])
    hd = rng.choice([64, 128, 128, 128, 256])
    if op == "norm_rope":
        rows = _log_int(rng, 1, max(1, min(8192, (1 << 26) // ((heads + kv_heads) * hd))))
        return dict(op=op, rows=rows, heads=heads, kv_heads=kv_heads, hd=hd, rot=rng.choice([hd, hd, hd // 2]), type=kind,
                    far=_log_int(rng, 16, 1 << 20), norm=rng.random() < 0.75)
    case = dict(op=op, batch=_log_int(rng, 1, 64), rows=rng.choice(["all", "all", "ragged", "mixed"]), even=rng.random() < 0.3,
                pad=rng.choice([0, 0, 5]), kv_heads=kv_heads, hd=hd, page=rng.choice([16, 16, 32, 64, 128, 256]),
                order=rng.choice(["head", "token"]), type=kind)
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
    """New rows of every stream."""
    B, n = c["batch"], c["most"]
    if c["rows"] == "all":
        return [n] * B
    if c["rows"] == "mixed":
        return [n] + [1] * (B - 1)
    return [max(1, n - (n * 3 * b) // (4 * B)) for b in range(B)]


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
    if c["op"] == "norm_rope":
        n = c["rows"] * (c["heads"] + c["kv_heads"]) * c["hd"]
        return {"bytes": 2 * n * size + 4 * c["rows"], "flops": 8 * n}
    live = sum(_rows(c))
    if c["op"] == "append":
        n = 2 * live * c["kv_heads"] * c["hd"]
        return {"bytes": 2 * n * size, "flops": 3 * n // 2}
    pairs, tokens = _seen(c)
    moved = 2 * tokens * c["kv_heads"] * c["hd"] + 2 * live * c["heads"] * c["hd"]
    return {"bytes": moved * size, "flops": 4 * pairs * c["heads"] * c["hd"]}


# ---------------------------------------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------------------------------------

def _normal(shape, gen, dtype, spread=1.0):
    """Normal values, drawn in pieces so that a large pool needs no float32 copy of itself."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 28):
        piece = flat[a:a + (1 << 28)]
        piece.copy_(torch.randn(piece.numel(), generator=gen, device=DEV) * spread)
    return out


def _inv_freq(rot, theta=500000.0):
    return torch.tensor([theta ** (-2.0 * j / rot) for j in range(rot // 2)], dtype=torch.float64, device=DEV)


def _pages(c, gen):
    """Pools and table: logical shape [pages][kv_heads][page][hd], in memory head-major or token-major."""
    dtype, P = TYPES[c["type"]], c["page"]
    need = [-(-(n + r) // P) for n, r in zip(_lengths(c), _rows(c))]
    total = sum(need) + 3
    shape = (total, c["kv_heads"], P, c["hd"]) if c["order"] == "head" else (total, P, c["kv_heads"], c["hd"])
    k, v = _normal(shape, gen, dtype), _normal(shape, gen, dtype)
    names = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((c["batch"], max(need) + 1), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = names[at:at + n]
        at += n
    return k, v, table


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 1000003 + 17)
    dtype, hd = TYPES[c["type"]], c["hd"]
    s = {"case": c}
    if c["op"] == "norm_rope":
        H, KVH, R = c["heads"], c["kv_heads"], c["rows"]
        s["qkv"] = _normal((R, H + 2 * KVH, hd), gen, dtype)             # the packed output of a q/k/v projection
        s["q"], s["k"] = s["qkv"][:, :H], s["qkv"][:, H:H + KVH]
        s["pos"] = torch.randint(0, c["far"], (R,), generator=gen, device=DEV, dtype=torch.int32)
        s["inv_freq"] = _inv_freq(c["rot"])
        s["q_gain"] = s["k_gain"] = None
        if c["norm"]:
            s["q_gain"] = 1 + 0.1 * torch.randn(hd, generator=gen, device=DEV)
            s["k_gain"] = 1 + 0.1 * torch.randn(hd, generator=gen, device=DEV)
        return s
    rows, lengths = _rows(c), _lengths(c)
    R = sum(rows) + c["pad"]
    s["k_pool"], s["v_pool"], s["table"] = _pages(c, gen)
    s["len"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    ends = [0]
    for r in rows:
        ends.append(ends[-1] + r)
    # a batch of equal rows needs no offsets
    s["row0"] = None if c["rows"] == "all" and not c["pad"] else torch.tensor(ends, dtype=torch.int32, device=DEV)
    if c["op"] == "append":
        s["k"] = _normal((R, c["kv_heads"], hd), gen, dtype)
        s["v"] = _normal((R, c["kv_heads"], hd), gen, dtype)
        s["inv_freq"] = _inv_freq(hd)
    else:
        s["q"] = _normal((R, c["heads"], hd), gen, dtype, 2.0)
        s["out"] = torch.zeros((R, c["heads"], hd), dtype=dtype, device=DEV)
    if own:
        from paper_2502_08923_amd import binding as cs
        view = (lambda t: t) if c["order"] == "head" else (lambda t: t.transpose(1, 2))
        s["handle"] = cs.Pages(view(s["k_pool"]), view(s["v_pool"]), s["table"], s["len"])
    return s


# ---------------------------------------------------------------------------------------------------------
# the operators
# ---------------------------------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    return {"norm_rope": _plain_norm_rope, "append": _plain_append, "attention": _plain_attention}[c["op"]](state, c)


def _run_own(s, c):
    from paper_2502_08923_amd import binding as cs
    if c["op"] == "norm_rope":
        return cs.cs_op_qk_norm_rope(s["q"], s["k"], s["pos"], s["inv_freq"], s["q_gain"], s["k_gain"], 1e-6)
    if c["op"] == "append":
        cs.cs_paged_append(s["handle"], s["k"], s["v"], row0=s["row0"], inv_freq=s["inv_freq"])
        return s["k_pool"], s["v_pool"]
    return cs.cs_paged_attention(s["handle"], s["q"], row0=s["row0"], window=c["window"], max_rows=c["most"],
                                 max_len=c["cached"] + c["most"], out=s["out"])


def _angles(pos, inv_freq):
    a = pos.double()[:, None] * inv_freq[None, :]
    return torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]


def _rotate(x, cos, sin):
    half = cos.shape[-1]
    a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], dim=-1)


def _plain_norm_rope(s, c):
    cos, sin = _angles(s["pos"], s["inv_freq"])
    out = []
    for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
        y = x.float()
        if gain is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * gain
        out.append(_rotate(y, cos, sin).to(x.dtype))
    return tuple(out)


def _plain_append(s, c):
    rows, P = _rows(c), c["page"]
    live = sum(rows)
    r = torch.arange(live, device=DEV)
    if s["row0"] is None:
        b = r // rows[0]
        i = r - b * rows[0]
    else:
        b = torch.searchsorted(s["row0"][1:].long(), r, right=True)
        i = r - s["row0"].long()[b]
    pos = s["len"].long()[b] + i
    page = s["table"].long()[b, pos // P]
    slot = pos % P
    cos, sin = _angles(pos, s["inv_freq"])
    k = _rotate(s["k"][:live].float(), cos, sin).to(s["k"].dtype)
    for pool, x in ((s["k_pool"], k), (s["v_pool"], s["v"][:live])):
        if c["order"] == "head":
            pool[page, :, slot] = x
        else:
            pool[page, slot] = x
    return s["k_pool"], s["v_pool"]


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

        def tokens(pool):
            t = pool[pages]                                              # [S][pages][KVH][P][hd] or [S][pages][P][KVH][hd]
            t = t.transpose(1, 2) if c["order"] == "head" else t.permute(0, 3, 1, 2, 4)
            return t.reshape(S, KVH, -1, hd)[:, :, :n].float()

        q = s["q"][start[b]:start[e]].view(S, m, KVH, G, hd).permute(0, 2, 1, 3, 4).reshape(S, KVH, m * G, hd).float()
        x = torch.matmul(q, tokens(s["k_pool"]).transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(hd))
        last = s["len"][b:e].long()[:, None] + torch.arange(m, device=DEV)[None, :].repeat_interleave(G, 1)
        t = torch.arange(n, device=DEV)
        hidden = t[None, None, :] > last[:, :, None]
        if w:
            hidden = hidden | (t[None, None, :] <= last[:, :, None] - w)
        x.masked_fill_(hidden[:, None], -math.inf)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        y = torch.matmul(x, tokens(s["v_pool"])) / x.sum(-1, keepdim=True)
        out[start[b]:start[e]] = y.view(S, KVH, m, G, hd).permute(0, 2, 1, 3, 4).reshape(S * m, H, hd).to(out.dtype)
        b = e
    return out


# ---------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------

def _turn(x, pos, inv_freq):
    """Pairs (j, j + rot/2) as complex numbers, turned by pos * inv_freq[j]."""
    half = inv_freq.numel()
    z = torch.complex(x[..., :half], x[..., half:2 * half])
    theta = torch.outer(pos.double(), inv_freq)
    z = z * torch.polar(torch.ones_like(theta), theta).unsqueeze(1)
    y = x.clone()
    y[..., :half] = z.real
    y[..., half:2 * half] = z.imag
    return y


def exact(case, seed):
    c = case
    if c["op"] == "attention" and work(c)["flops"] > 3e12:
        return None
    s = prepare(case, seed)
    if c["op"] == "norm_rope":
        out = []
        for x, gain in ((s["q"].double(), s["q_gain"]), (s["k"].double(), s["k_gain"])):
            if gain is not None:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["hd"] + 1e-6) * gain.double()
            out.append(_turn(x, s["pos"], s["inv_freq"]))
        return tuple(out)
    rows, lengths, P, KVH = _rows(c), _lengths(c), c["page"], c["kv_heads"]
    table = s["table"].cpu()
    by_token = (lambda t: t.transpose(1, 2)) if c["order"] == "head" else (lambda t: t)      # [pages][P][KVH][hd]
    if c["op"] == "append":
        kp, vp = s["k_pool"].double(), s["v_pool"].double()
        at = 0
        for b in range(c["batch"]):
            pos = torch.arange(lengths[b], lengths[b] + rows[b])
            page, slot = table[b][pos // P].long().to(DEV), (pos % P).to(DEV)
            by_token(kp)[page, slot] = _turn(s["k"][at:at + rows[b]].double(), pos.to(DEV), s["inv_freq"])
            by_token(vp)[page, slot] = s["v"][at:at + rows[b]].double()
            at += rows[b]
        return kp, vp
    H, hd = c["heads"], c["hd"]
    G = H // KVH
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for b in range(c["batch"]):
        n = lengths[b] + rows[b]
        names = table[b][:-(-n // P)].long().to(DEV)
        for g in range(KVH):
            k = by_token(s["k_pool"])[names, :, g].reshape(-1, hd)[:n].double()
            v = by_token(s["v_pool"])[names, :, g].reshape(-1, hd)[:n].double()
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
