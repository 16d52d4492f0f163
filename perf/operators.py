"""Performance cases of the operators that stand between the q, k, v and the o projections of a layer:
rotary positions, the paged 4-bit KV cache's append, and attention over that cache.

A case is one call of one operator, as a serving (or training) program makes it for one layer; the append is followed by the
read of the same rows, which gives what the cache then holds as values.

Fields of a case
  op           "rotate", "append" or "attend"
  dtype        element type of q, k, v and the outputs: bf16, fp16 or fp32
  heads, kv_heads, head_dim   query heads, key / value heads (rotate: kv_heads is not used)
  rot, pairs   channels of a head that are rotated (0: none; attend: q arrives rotated), and whether a pair is
               (j, j + rot/2), "half", or (2j, 2j+1), "interleaved"
  inverse      rotate: by the negative angle, the gradient of the rotation
  page         tokens of a page of the cache
  seqs         sequences of the batch
  new_lo, new_hi   tokens of a sequence in this call (its last ones)
  ctx_lo, ctx_hi   tokens of a sequence that are in the cache before this call (rotate: the first position)
  causal, window   attend: which keys a token sees: up to its own position, and only the last `window` (0: all)

The cache of a layer: pages of `page` tokens for all kv heads; of a page, head after head,
  keys' codes    page x head_dim/2 bytes: the code of channel d of token t is nibble d % 2 (low first) of byte t*head_dim/2 + d/2
  values' codes  page x head_dim/2 bytes: per 32 tokens head_dim/64 x 4 x 16 x 4 words [j][g][r][i] of 8 codes; nibble n
                 belongs to token 16*(n/4) + 4*g + n%4 and channel (r/4)*(head_dim/4) + (4*j + i)*4 + r%4
  keys' (scale, min), values' (scale, min)   page x two bf16 each, scale first
and a code c of 0 .. 15 stands for min + scale * c.
"""
import math
import random

import torch

own = False
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ELT = {"bf16": 2, "fp16": 2, "fp32": 4}
WORKSPACE = 64 << 20  # bytes that a program keeps for attention that is split along the keys
TINY = 2.0 ** -100  # a scale below this is none: all 16 codes stand for the row's min


def _case(name=None, **kw):
    c = dict(op="attend", dtype="bf16", heads=32, kv_heads=8, head_dim=128, rot=128, pairs="half", inverse=False, page=64,
             seqs=1, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=0, causal=True, window=0)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one interactive user, one token: nothing but latency
        _case("rotate_1tok", op="rotate", ctx_lo=777, ctx_hi=777),
        # the queries of some 30 prompts of a 13B-shaped layer
        _case("rotate_prompts_5k_fp16", op="rotate", dtype="fp16", heads=40, seqs=32, new_lo=64, new_hi=256, pairs="interleaved"),
        # a training step's gradient back through the rotation of part of an 80-wide head, ragged, fp32
        _case("rotate_gradient_fp32", op="rotate", dtype="fp32", heads=20, head_dim=80, rot=32, inverse=True, seqs=5, new_lo=301,
              new_hi=901),
        # a decode step of 256 users with grouped heads: one new token each, anywhere in a page
        _case("append_decode_256", op="append", seqs=256, ctx_lo=64, ctx_hi=4000),
        # a batch of prompts of a 7B-shaped layer with a head of its own per query
        _case("append_prompts_5k", op="append", kv_heads=32, seqs=32, new_lo=64, new_hi=256),
        # chunks of long documents behind ragged contexts: narrow heads, part of them rotated, fp32
        _case("append_chunks_fp32", op="append", dtype="fp32", kv_heads=12, head_dim=64, rot=32, pairs="interleaved", page=32, seqs=7,
              new_lo=777, new_hi=2049, ctx_lo=1, ctx_hi=1000),
        # one interactive user, one token over a short conversation
        _case("attend_1tok_777", ctx_lo=776, ctx_hi=776),
        # the usual decode step: 256 users, grouped heads, conversations of all lengths
        _case("attend_decode_256", seqs=256, ctx_lo=64, ctx_hi=4095),
        # a fp32 model with narrow heads and a window of 1000 keys: 24 users, q rotated ahead of the call
        _case("attend_window_fp32", dtype="fp32", heads=12, kv_heads=12, head_dim=64, rot=0, page=32, seqs=24, ctx_lo=100, ctx_hi=3000,
              window=1000),
        # two users with very long documents: few rows, all work along the keys
        _case("attend_decode_128k", seqs=2, ctx_lo=131071, ctx_hi=131071, page=256),
        # a batch of prompts of a 7B-shaped layer with a head of its own per query
        _case("attend_prompts_5k", kv_heads=32, seqs=32, new_lo=64, new_hi=256),
        # a chunk of 2048 tokens of one long document, fp16, behind 30000 tokens that are in the cache
        _case("attend_chunk_2k_over_30k_fp16", dtype="fp16", new_lo=2048, new_hi=2048, ctx_lo=30000, ctx_hi=30000, page=128),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["rotate", "append", "attend", "attend"])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp16", "fp32"])
        head_dim = rng.choice([64, 128, 128, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 8, 8, 12, 32, 40])
        heads = kv_heads * rng.choice([1, 1, 2, 4, 5, 8])
        if op == "rotate":
            heads = _spread(rng, 1, 64)
            head_dim = rng.choice([64, 80, 96, 128, 128, 256])
        rot = rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4])
        if op != "rotate" and rng.random() < 0.15:
            rot = 0
        c = _case(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, rot=rot, pairs=rng.choice(["half", "interleaved"]),
                  inverse=op == "rotate" and rng.random() < 0.3, page=rng.choice([32, 64, 128, 256]), seqs=_spread(rng, 1, 256))
        if rng.random() < 0.4:  # prompts and chunks; else one token a sequence
            c["new_lo"] = _spread(rng, 1, 1024)
            c["new_hi"] = c["new_lo"] * rng.choice([1, 2, 4])
        c["ctx_lo"] = _spread(rng, 1, 65536) - 1
        c["ctx_hi"] = c["ctx_lo"] * rng.choice([1, 2, 4]) + rng.choice([0, 33])
        if op == "attend":
            c["causal"] = rng.random() < 0.85
            c["window"] = _spread(rng, 16, 8192) if c["causal"] and rng.random() < 0.2 else 0
        if _fits(c):
            return c


def _fits(c):
    """Whether the plain form of a drawn case costs no more than that of the listed ones."""
    most = [_cost(l) for l in listed() if l["op"] == c["op"]]
    mine = _cost(c)
    return all(m <= max(o[k] for o in most) for k, m in enumerate(mine))


def _cost(c):
    new, length = _lengths(c)
    elt = c["head_dim"]
    if c["op"] != "attend":
        return (sum(new) * (c["heads"] if c["op"] == "rotate" else c["kv_heads"]) * elt * ELT[c["dtype"]], max(length))
    w = work(c)
    return (w["bytes"], w["flops"], len(new) * max(length) * c["kv_heads"] * elt, len(new) * max(new) * c["heads"] * max(length), max(length))


def _lengths(c):
    """(tokens of each sequence in this call, tokens of each sequence with them): they belong to the case, not to the seed."""
    rng = random.Random(repr([(k, c[k]) for k in sorted(c) if k != "name"]))
    new = [rng.randint(c["new_lo"], c["new_hi"]) for _ in range(c["seqs"])]
    return new, [n + rng.randint(c["ctx_lo"], c["ctx_hi"]) for n in new]


def _pairs_seen(c):
    """Keys seen, summed over the tokens of the call."""
    total = 0
    for n, length in zip(*_lengths(c)):
        if not c["causal"]:
            total += n * length
            continue
        first = length - n + 1  # keys up to the first token's own
        if c["window"]:
            total += sum(min(c["window"], k) for k in range(first, length + 1))
        else:
            total += n * (first + length) // 2
    return total


def _keys_read(c):
    """Cache rows that some token of the call sees."""
    total = 0
    for n, length in zip(*_lengths(c)):
        total += min(length, c["window"] + n - 1) if c["window"] else length
    return total


def work(case):
    """q (or x, or k and v) read once, the result written once, every cache row that is seen read or written once, the
    rotation's rows read once."""
    c = case
    new, _ = _lengths(c)
    tokens, d, elt = sum(new), c["head_dim"], ELT[c["dtype"]]
    angles = tokens * c["rot"] * 4
    if c["op"] == "rotate":
        return {"bytes": 2 * tokens * c["heads"] * d * elt + angles, "flops": 3 * tokens * c["heads"] * c["rot"]}
    rows = tokens * c["kv_heads"]
    if c["op"] == "append":  # k and v in, both forms of the rows out and in, values out
        return {"bytes": 2 * rows * d * elt * 2 + 2 * rows * (d + 8) + angles, "flops": rows * (3 * c["rot"] + 2 * 10 * d)}
    return {"bytes": _keys_read(c) * c["kv_heads"] * (d + 8) + 2 * tokens * c["heads"] * d * elt + angles,
            "flops": 4 * d * c["heads"] * _pairs_seen(c)}


# ---- inputs -------------------------------------------------------------------------------------------

def _gen(seed, k):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + k) & 0x7FFFFFFFFFFF)
    return g


def _randn(seed, k, *shape):
    return torch.randn(*shape, generator=_gen(seed, k), device=DEV)


def _angle_table(positions, rot):
    """cos and sin of position * 10000^(-2j/rot): [positions][rot/2][2] in 32 bits."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    a = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _keys(seed, rows, heads, d):
    """Keys as projections give them: a few channels of every head carry much more than the others, and an offset."""
    loud = 1 + 3 * (torch.rand(heads, d, generator=_gen(seed, 3), device=DEV) < 0.05)
    return _randn(seed, 1, rows, heads, d) * loud + 0.5 * _randn(seed, 4, heads, d)


def _quantised(x):
    """4-bit form of rows of x: (codes as numbers, scale, min); a row with a value that is not finite has neither."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s = ((hi - lo) / torch.full_like(hi, 15.0)).bfloat16().float()
    m = lo.bfloat16().float()
    s = torch.where(s < TINY, 0.0, s)
    c = torch.where(s > 0, (x - m) / s, 0.0).round().clamp(0, 15)
    fine = torch.isfinite(s) & torch.isfinite(m)
    nan = float("nan")
    return torch.where(fine, c, 0.0), torch.where(fine, s, nan), torch.where(fine, m, nan)


def _packed_pages(c, seed, n_pages, written):
    """A cache of random rows; written[page][token] says which rows are: the others hold what no row stands for."""
    p, h, d = c["page"], c["kv_heads"], c["head_dim"]
    pages = torch.empty(n_pages, h, p * (d + 8), device=DEV, dtype=torch.uint8)
    at = max(1, (1 << 28) // (p * h * d))
    for a in range(0, n_pages, at):
        b = min(n_pages, a + at)
        par = []
        for which in (0, 1):
            x = (_keys(seed + a * 7, (b - a) * p, h, d) if which == 0 else _randn(seed, 100 + a, (b - a) * p, h, d)).view(b - a, p, h, d)
            q, s, m = _quantised(x)
            q = q.to(torch.uint8).transpose(1, 2)  # page, head, token, channel
            if which == 0:
                pages[a:b, :, :p * d // 2] = (q[..., 0::2] | q[..., 1::2] << 4).reshape(b - a, h, p * d // 2)
            else:
                q = q.reshape(b - a, h, p // 32, 2, 4, 4, 4, d // 64, 4, 4)  # block, n/4, g, n%4, r/4, j, i, r%4
                q = q.permute(0, 1, 2, 7, 4, 6, 9, 8, 3, 5).reshape(b - a, h, p * d // 2, 2)
                pages[a:b, :, p * d // 2:p * d] = q[..., 0] | q[..., 1] << 4
            w = torch.cat([s, m], -1).transpose(1, 2)  # page, head, token, 2
            w = torch.where(written[a:b, None, :, None], w, float("nan")).bfloat16().contiguous()
            par.append(w.view(torch.uint8).reshape(b - a, h, p * 4))
        pages[a:b, :, p * d:] = torch.cat(par, -1)
    return pages.view(n_pages, h * p * (d + 8))


def prepare(case, seed):
    c = case
    new, length = _lengths(c)
    tokens, d, dt = sum(new), c["head_dim"], DTYPES[c["dtype"]]
    s = {"case": c, "tokens": tokens, "max_new": max(new), "max_len": max(length)}
    i32 = dict(dtype=torch.int32, device=DEV)
    s["tok_start"] = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], **i32)
    s["kv_len"] = torch.tensor(length, **i32)
    s["positions"] = torch.cat([torch.arange(l - n, l, **i32) for n, l in zip(new, length)])
    s["angles"] = _angle_table(max(length), c["rot"]) if c["rot"] else None
    if c["op"] == "rotate":
        s["x"] = _randn(seed, 0, tokens, c["heads"], d).to(dt)
        s["out"] = torch.empty_like(s["x"])
        return s
    # sequences own pages that lie anywhere in the pool
    p = c["page"]
    need = [-(-l // p) for l in length]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=_gen(seed, 9), device=DEV).to(torch.int32)
    at = torch.tensor([sum(need[:i]) for i in range(len(need))], **i32)
    col = torch.arange(max(need), **i32)
    has = col[None, :] * p < s["kv_len"][:, None]
    s["table"] = torch.where(has, order[torch.where(has, at[:, None] + col[None, :], 0)], -1).contiguous()
    if c["op"] == "append":
        s["pages"] = torch.randint(0, 256, (n_pages, c["kv_heads"] * p * (d + 8)), generator=_gen(seed, 5), device=DEV, dtype=torch.uint8)
        s["k"] = _keys(seed, tokens, c["kv_heads"], d).to(dt)
        s["v"] = _randn(seed, 2, tokens, c["kv_heads"], d).to(dt)
        s["k_out"], s["v_out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        return s
    left = torch.where(has, (s["kv_len"][:, None] - col[None, :] * p).clamp(max=p), 0)
    rows = torch.zeros(n_pages, **i32)
    rows[s["table"][has].long()] = left[has]
    s["pages"] = _packed_pages(c, seed, n_pages, torch.arange(p, device=DEV)[None, :] < rows[:, None])
    s["q"] = (1.5 * _randn(seed, 0, tokens, c["heads"], d)).to(dt)
    s["out"] = torch.empty_like(s["q"])
    s["workspace"] = torch.empty(WORKSPACE, device=DEV, dtype=torch.uint8)
    return s


# ---- one pass -----------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if own:
        return _library(s, c)
    if c["op"] == "rotate":
        return {"out": _rotated(s, s["x"].float(), c["inverse"]).to(s["x"].dtype)}
    if c["op"] == "append":
        k = s["k"].float()
        k = _rotated(s, k, False) if c["rot"] else k
        got = {}
        for name, x in (("k", k), ("v", s["v"].float())):
            q, sc, mn = _quantised(x)
            got[name] = (mn + sc * q).to(s["k"].dtype)
        return got
    return {"out": _attended(s, c)}


def _library(s, c):
    import paper_2512_20210_amd as plora
    if "handles" not in s:
        h = s["handles"] = {"rotary": plora.Rotary(s["angles"], c["rot"], c["pairs"] == "interleaved") if c["rot"] else None}
        if c["op"] != "rotate":
            dtype = {"bf16": plora.PLORA_BF16, "fp16": plora.PLORA_F16, "fp32": plora.PLORA_F32}[c["dtype"]]
            h["cache"] = plora.PagedKvCache(dtype, c["kv_heads"], c["head_dim"], c["page"], s["pages"])
            h["batch"] = plora.KvBatch(s["tok_start"], s["kv_len"], s["table"], s["tokens"], s["max_new"], s["max_len"], s["positions"])
    h = s["handles"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "rotate":
        h["rotary"].rotate(s["positions"], s["x"], s["out"], c["inverse"], stream)
        return {"out": s["out"]}
    if c["op"] == "append":
        h["cache"].append(h["batch"], s["k"], s["v"], h["rotary"], stream)
        h["cache"].read(h["batch"], s["k_out"], s["v_out"], stream)
        return {"k": s["k_out"], "v": s["v_out"]}
    h["cache"].attend(h["batch"], s["q"], s["out"], c["head_dim"] ** -0.5, s["workspace"], c["causal"], c["window"], h["rotary"], stream)
    return {"out": s["out"]}


# ---- plain forms --------------------------------------------------------------------------------------

def _rotated(s, x, inverse):
    rot, half = s["case"]["rot"], s["case"]["pairs"] == "half"
    cs = s["angles"][s["positions"].long()][:, None]
    cos, sin = cs[..., 0], -cs[..., 1] if inverse else cs[..., 1]
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if half else (x[..., 0:rot:2], x[..., 1:rot:2])
    u, w = a * cos - b * sin, b * cos + a * sin
    y = torch.cat([u, w], -1) if half else torch.stack([u, w], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _unpacked(s, c):
    """(keys, values) of every sequence in 32 bits: [sequence][kv head][token][channel]."""
    p, h, d = c["page"], c["kv_heads"], c["head_dim"]
    raw = s["pages"][s["table"].clamp(min=0).long()].view(*s["table"].shape, h, p * (d + 8))
    n_seq, n_col = s["table"].shape
    kq, vq, par = raw[..., :p * d // 2], raw[..., p * d // 2:p * d], raw[..., p * d:].contiguous().view(torch.bfloat16)
    par = par.view(n_seq, n_col, h, 2, p, 2).transpose(1, 2).float()  # sequence, head, page, k or v, token, (scale, min)
    kq = torch.stack([kq & 15, kq >> 4], -1).view(n_seq, n_col, h, p, d)
    vq = torch.stack([vq & 15, vq >> 4], -1).view(n_seq, n_col, h, p // 32, d // 64, 4, 4, 4, 4, 2, 4)  # block, j, g, r/4, r%4, i, n/4, n%4
    vq = vq.permute(0, 1, 2, 3, 9, 5, 10, 6, 4, 8, 7).reshape(n_seq, n_col, h, p, d)
    k = par[..., 0, :, 1:] + par[..., 0, :, :1] * kq.transpose(1, 2)
    v = par[..., 1, :, 1:] + par[..., 1, :, :1] * vq.transpose(1, 2)
    return k.reshape(n_seq, h, n_col * p, d), v.reshape(n_seq, h, n_col * p, d)


def _attended(s, c):
    q = s["q"].float()
    q = _rotated(s, q, False) if c["rot"] else q
    k, v = _unpacked(s, c)
    n_seq, h, n_key, d = k.shape
    rep, most = c["heads"] // h, s["max_new"]
    key = torch.arange(n_key, device=k.device)
    live = key < s["kv_len"][:, None]  # sequence, key
    v = torch.where(live[:, None, :, None], v, 0.0)
    n_new = s["tok_start"][1:] - s["tok_start"][:-1]
    row = torch.arange(most, device=k.device)
    mine = row < n_new[:, None]  # sequence, row
    at = torch.where(mine, s["tok_start"][:-1, None] + row, 0).long()
    qs = q[at].view(n_seq, most, h, rep, d).permute(0, 2, 1, 3, 4).reshape(n_seq, h, most * rep, d)
    t = torch.matmul(qs, k.transpose(-1, -2).contiguous()).mul_(d ** -0.5).view(n_seq, h, most, rep, n_key)
    sees = live[:, None, :].expand(n_seq, most, n_key)
    if c["causal"]:
        pos = s["kv_len"][:, None] - n_new[:, None] + row
        sees = sees & (key <= pos[..., None])
        if c["window"]:
            sees = sees & (key > pos[..., None] - c["window"])
    t = torch.where(sees[:, None, :, None, :], t, float("-inf"))
    top = t.amax(-1, keepdim=True)
    t = t.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = t.sum(-1, keepdim=True)
    o = torch.matmul(t.view(n_seq, h, most * rep, n_key), v).view(n_seq, h, most, rep, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(n_seq, most, h * rep, d)
    return o[mine].to(s["q"].dtype)


# ---- what is right ------------------------------------------------------------------------------------

def _turned64(c, s, x):
    """Rotation as a complex product, in 64 bits."""
    rot = c["rot"]
    if not rot:
        return x
    z = torch.view_as_complex(s["angles"].double())[s["positions"].long()][:, None, :]
    z = z.conj() if c["inverse"] else z
    y = x.clone()
    if c["pairs"] == "half":
        w = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * z
        y[..., :rot // 2], y[..., rot // 2:rot] = w.real, w.imag
    else:
        w = torch.complex(x[..., 0:rot:2].contiguous(), x[..., 1:rot:2].contiguous()) * z
        y[..., 0:rot:2], y[..., 1:rot:2] = w.real, w.imag
    return y


def _nearest16(x):
    lo = torch.aminmax(x, dim=-1, keepdim=True)
    s = ((lo.max - lo.min) / 15).to(torch.bfloat16).double()
    m = lo.min.to(torch.bfloat16).double()
    steps = torch.round((x - m) / torch.where(s >= TINY, s, 1.0)).clamp(0, 15)
    return torch.where(s >= TINY, m + s * steps, m)


def _row_values64(c, s, seq, head, n_key):
    """Keys and values of one sequence and head, looked up byte by byte."""
    p, d = c["page"], c["head_dim"]
    t, ch = torch.arange(n_key, device=DEV)[:, None], torch.arange(d, device=DEV)[None, :]
    raw = s["pages"].view(-1)
    base = s["table"][seq].long()[t // p] * s["pages"].shape[1] + head * p * (d + 8)
    t = t % p
    byte = raw[base + t * (d // 2) + ch // 2]
    k = torch.where(ch % 2 == 1, byte >> 4, byte & 15).double()
    quarter, rest = ch // (d // 4), ch % (d // 4)
    tile, r = rest // 4, quarter * 4 + rest % 4
    u = t % 32
    g, nib = u % 16 // 4, u % 4 + u // 16 * 4
    word = t // 32 * (4 * d) + ((tile // 4 * 4 + g) * 16 + r) * 4 + tile % 4
    byte = raw[base + p * d // 2 + 4 * word + nib // 2]
    v = torch.where(nib % 2 == 1, byte >> 4, byte & 15).double()
    par = raw[base + p * d + t * 4 + torch.arange(4, device=DEV)].contiguous().view(torch.bfloat16).double()
    k = par[:, :1] * k + par[:, 1:]
    par = raw[base + p * d + (p + t) * 4 + torch.arange(4, device=DEV)].contiguous().view(torch.bfloat16).double()
    return k, par[:, :1] * v + par[:, 1:]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rotate":
        return {"out": _turned64(c, s, s["x"].double())}
    if c["op"] == "append":
        return {"k": _nearest16(_turned64(c, s, s["k"].double())), "v": _nearest16(s["v"].double())}
    q = _turned64(c, s, s["q"].double())
    out = torch.zeros_like(q)
    rep = c["heads"] // c["kv_heads"]
    start = s["tok_start"].tolist()
    for i, length in enumerate(s["kv_len"].tolist()):
        rows = slice(start[i], start[i + 1])
        n = start[i + 1] - start[i]
        ahead = torch.arange(length, device=DEV)[None, :] - torch.arange(length - n, length, device=DEV)[:, None]
        hidden = torch.zeros(n, length, device=DEV, dtype=torch.bool)
        if c["causal"]:
            hidden = ahead > 0
            if c["window"]:
                hidden = hidden | (ahead <= -c["window"])
        for h in range(c["kv_heads"]):
            k, v = _row_values64(c, s, i, h, length)
            for j in range(h * rep, (h + 1) * rep):
                t = (q[rows, j] @ k.t() / math.sqrt(c["head_dim"])).masked_fill(hidden, -math.inf)
                out[rows, j] = torch.softmax(t, -1).nan_to_num(0.0) @ v
    return {"out": out}
