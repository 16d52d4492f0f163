"""Performance cases of the operators around the adapters of a layer whose base weights are held in 8 bits: the norm between two
blocks, activations in 8 bits, the base products, the routing of tokens to experts and the experts' products.

A case is one call of one operator, as a serving program makes it for one layer.

8-bit rows: a row of k values is held as e4m3 codes, and for each block of 128 of them (the last one may be short) one scale in
32 bits,  scale = amax / 448,  code = e4m3(x * (448 / amax)), both quotients rounded to 32 bits; a block with amax < 2^-100 has scale 0 and
codes 0. Scales lie block after block: [blocks][rows]. Weights [n][k] have a scale for each 128 x 128 block: [blocks of n][blocks of k].

Fields of a case
  op       "norm", "quantise", "matmul", "grouped" or "route"
  dtype    element type of the tensors that are not in 8 bits: bf16, fp16 or fp32
  tokens   rows of the batch
  k, n     norm: k channels; quantise: k values a row; matmul, grouped: rows of k values times weights [n][k]
  experts, top_k  grouped: experts, and how many of them a token goes to (its row is read once for each: rows are gathered);
           route: the same; norm: top_k > 0 means that the block's output is the weighted sum of top_k rows of the experts' products
  gathered grouped: whether rows are gathered (the first product of an expert) or lie sorted already (the second one)
  act      quantise: "none", or "silu" / "gelu" of the first k of 2k values a row times the other k
  eight    norm: whether the result is in 8 bits (codes and scales) or of the type
  residual, post, gate, center, scale   norm: parts of hidden = residual + scale * gate * post(block), result = pre(hidden)
  padded   route: share of the tokens that are padding (their logits are all -inf)
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ELT = {"bf16": 2, "fp16": 2, "fp32": 4}
BLOCK = 128
TOP = 448.0  # the largest e4m3 value
TINY = 2.0 ** -100
EPS = 1e-5


def _case(name=None, **kw):
    c = dict(op="norm", dtype="bf16", tokens=1, k=4096, n=0, experts=0, top_k=0, gathered=False, act="none", eight=False, residual=True,
             post=False, gate=False, center=False, scale=1.0, padded=0.0)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one interactive user, one token: residual, norm, 8 bits; nothing but latency
        _case("norm_1tok", eight=True),
        # prompts of some 30 users of a 13B-shaped layer, norms on both sides of the block, a gate for each channel and token
        _case("norm_prompts_5k", tokens=5093, k=5120, eight=True, post=True, gate=True, scale=0.5),
        # behind the experts: every token takes the weighted sum of four rows, then residual and norm
        _case("norm_experts_2k_fp16", dtype="fp16", tokens=2049, top_k=4),
        # between the two products of a gated block of a 13B-shaped layer, a decode step
        _case("quantise_gated_64tok", op="quantise", tokens=64, k=13824, act="silu"),
        # rows of prompts ahead of the o projection
        _case("quantise_prompts_5k_fp16", op="quantise", dtype="fp16", tokens=5093),
        # one interactive user, one token, a square projection of a 7B-shaped layer: the weights have to be read
        _case("matmul_1tok", op="matmul", n=4096),
        # the usual decode step, up projection of a 13B-shaped layer
        _case("matmul_decode_256_fp16", op="matmul", dtype="fp16", tokens=256, k=5120, n=13824),
        # prefill of 16k tokens, down projection of a 13B-shaped layer
        _case("matmul_prompts_16k", op="matmul", tokens=16384, k=13824, n=5120),
        # a decode step over many small experts: a few rows for each, all weights have to be read
        _case("grouped_decode_64tok", op="grouped", tokens=64, k=2048, n=2816, experts=64, top_k=6, gathered=True),
        # prompts over eight large experts, groups of ragged sizes
        _case("grouped_prompts_5k_fp16", op="grouped", dtype="fp16", tokens=5093, k=4096, n=7168, experts=8, top_k=2, gathered=True),
        # a decode step's routing, a quarter of it padding
        _case("route_decode_256", op="route", tokens=256, experts=64, top_k=6, padded=0.25),
        # routing of a batch of long prompts over many experts
        _case("route_prompts_16k_fp32", op="route", dtype="fp32", tokens=16384, experts=256, top_k=8),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["norm", "norm", "quantise", "matmul", "matmul", "grouped", "grouped", "route"])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp16", "fp32"])
        c = _case(op=op, dtype=dtype, tokens=_spread(rng, 1, 16384))
        if op == "norm":
            c["k"] = 8 * _spread(rng, 8, 2048)
            c.update(eight=rng.random() < 0.5, residual=rng.random() < 0.8, post=rng.random() < 0.4, gate=rng.random() < 0.4,
                     center=rng.random() < 0.3, scale=rng.choice([1.0, 0.25]), top_k=rng.choice([0, 0, 1, 2, 4, 8]))
        elif op == "quantise":
            c["k"] = 16 * _spread(rng, 4, 1024)
            c["act"] = rng.choice(["none", "silu", "gelu"])
        elif op == "route":
            c["experts"] = _spread(rng, 4, 512)
            c["top_k"] = rng.choice([j for j in (1, 2, 4, 6, 8) if j <= c["experts"]])
            c["padded"] = rng.choice([0.0, 0.0, 0.3])
        else:
            c["k"], c["n"] = 16 * _spread(rng, 8, 864), 8 * _spread(rng, 8, 1728)
            if op == "grouped":
                c["experts"] = _spread(rng, 2, 128)
                c["top_k"] = rng.choice([j for j in (1, 2, 4, 6, 8) if j <= c["experts"]])
                c["gathered"] = rng.random() < 0.6
        if all(m <= max(_cost(l)[i] for l in listed() if l["op"] == op) for i, m in enumerate(_cost(c))):
            return c


def _cost(c):
    """What the plain form of a case costs: passes over memory, products, and the padded products of ragged groups."""
    w = work(c)
    if c["op"] != "grouped":
        return (w["bytes"], w["flops"])
    most = max(_counts(c))
    return (w["bytes"], c["experts"] * most * c["k"] * c["n"], c["experts"] * (most * (c["k"] + c["n"]) + c["k"] * c["n"]))


def _choice(c):
    """Which experts the tokens of a case go to, [tokens][top_k], some experts liked more: they belong to the case, not to the seed."""
    rs = np.random.RandomState(random.Random(repr([(k, c[k]) for k in sorted(c) if k != "name"])).randrange(1 << 31))
    score = rs.gumbel(size=(c["tokens"], c["experts"])) + 0.5 * rs.normal(size=c["experts"])
    return np.sort(np.argsort(-score, axis=1, kind="stable")[:, :c["top_k"]], axis=1)


def _counts(c):
    return np.bincount(_choice(c).reshape(-1), minlength=c["experts"]).tolist()


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    """Inputs read once (of weights: those of the experts that have rows), results written once."""
    c = case
    t, k, n, elt = c["tokens"], c["k"], c["n"], ELT[c["dtype"]]
    eight = t * k + 4 * t * _blocks(k)  # rows in 8 bits
    if c["op"] == "norm":
        rows = max(1, c["top_k"]) + c["residual"] * 1 + c["gate"] + 1  # the last one: hidden
        b = rows * t * k * elt + (eight if c["eight"] else t * k * elt) + 8 * t * c["top_k"] + (1 + c["center"]) * (1 + c["post"]) * k * elt
        return {"bytes": b, "flops": t * k * (6 + 2 * c["top_k"] + 5 * c["post"] + 4 * c["eight"])}
    if c["op"] == "quantise":
        wide = 1 if c["act"] == "none" else 2
        return {"bytes": wide * t * k * elt + eight, "flops": t * k * (4 if wide == 1 else 12)}
    if c["op"] == "route":
        e, j = c["experts"], c["top_k"]
        return {"bytes": t * e * elt + t * j * 16 + 4 * (e + 1), "flops": t * e * (4 + j)}
    weights = n * k + 4 * _blocks(n) * _blocks(k)
    if c["op"] == "matmul":
        return {"bytes": eight + weights + t * n * elt, "flops": 2 * t * n * k}
    rows = t * c["top_k"]
    read = t if c["gathered"] else rows
    return {"bytes": read * (k + 4 * _blocks(k)) + sum(m > 0 for m in _counts(c)) * weights + rows * n * elt + 4 * rows * c["gathered"],
            "flops": 2 * rows * n * k}


# ---- inputs -------------------------------------------------------------------------------------------

def _gen(seed, k):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + k) & 0x7FFFFFFFFFFF)
    return g


def _randn(seed, k, *shape):
    return torch.randn(*shape, generator=_gen(seed, k), device=DEV)


def _hidden(seed, at, rows, k):
    """Rows as the residual stream of a model has them: a few channels much louder than the others, rows of different size."""
    loud = 1 + 15 * (torch.rand(k, generator=_gen(seed, at + 1), device=DEV) < 0.01)
    return _randn(seed, at, rows, k) * loud * torch.exp(0.5 * _randn(seed, at + 2, rows, 1))


def _weights8(seed, at, *shape):
    """Codes and scales of weights: a block's largest value has the largest code."""
    codes = (_randn(seed, at, *shape) * (TOP / 4.3)).clamp(-TOP, TOP).to(torch.float8_e4m3fn)
    scales = torch.exp(0.2 * _randn(seed, at + 1, *shape[:-2], _blocks(shape[-2]), _blocks(shape[-1]))) * (4.3 / TOP * shape[-1] ** -0.5)
    return codes, scales.contiguous()


def prepare(case, seed):
    c = case
    t, k, n, dt = c["tokens"], c["k"], c["n"], DTYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "norm":
        j = c["top_k"]
        s["block"] = _hidden(seed, 0, t * max(1, j), k).to(dt)
        if j:  # rows of the experts' products lie sorted by expert: a token's are anywhere
            s["places"] = torch.randperm(t * j, generator=_gen(seed, 9), device=DEV).to(torch.int32).view(t, j)
            w = torch.rand(t, j, generator=_gen(seed, 10), device=DEV) + 0.05
            s["place_weights"] = w / w.sum(-1, keepdim=True)
        s["residual"] = (4 * _hidden(seed, 20, t, k)).to(dt) if c["residual"] else None
        s["gate"] = (0.5 + 0.3 * _randn(seed, 30, t, k)).to(dt) if c["gate"] else None
        for i, name in enumerate(("pre", "post")):
            if name == "pre" or c["post"]:
                s[name + "_weight"] = (1 + 0.2 * _randn(seed, 40 + i, k)).to(dt)
                s[name + "_bias"] = (0.1 * _randn(seed, 50 + i, k)).to(dt) if c["center"] else None
        s["hidden"] = torch.empty(t, k, device=DEV, dtype=dt)
    elif c["op"] == "quantise":
        s["x"] = _hidden(seed, 0, t, k if c["act"] == "none" else 2 * k).to(dt)
    elif c["op"] == "route":
        x = _randn(seed, 0, t, c["experts"]) * 1.5 + 0.7 * _randn(seed, 1, c["experts"])
        x[torch.rand(t, generator=_gen(seed, 2), device=DEV) < c["padded"]] = -math.inf
        j = c["top_k"]
        i32 = dict(device=DEV, dtype=torch.int32)
        s.update(logits=x.to(dt), experts=torch.empty(t, j, **i32), weights=torch.empty(t, j, device=DEV), rows=torch.empty(t * j, **i32),
                 places=torch.empty(t, j, **i32), offsets=torch.empty(c["experts"] + 1, **i32), workspace=torch.empty(1 << 22, device=DEV, dtype=torch.uint8))
        return s
    else:
        rows = t
        if c["op"] == "grouped":
            choice = torch.from_numpy(_choice(c)).to(DEV)
            flat = choice.reshape(-1)
            order = torch.sort(flat, stable=True)[1]
            counts = torch.bincount(flat, minlength=c["experts"])
            s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
            s["rows"] = (order // c["top_k"]).to(torch.int32) if c["gathered"] else None
            s["most"] = max(_counts(c))
            rows = t if c["gathered"] else t * c["top_k"]
            s["w"], s["ws"] = _weights8(seed, 60, c["experts"], n, k)
        else:
            s["w"], s["ws"] = _weights8(seed, 60, n, k)
        s["x"], s["xs"] = _quantised(_hidden(seed, 0, rows, k))
        s["out"] = torch.empty(t * max(1, c["top_k"]), n, device=DEV, dtype=dt)
        return s
    if c["op"] == "quantise" or c["eight"]:
        s["codes"], s["scales"] = torch.empty(t, k, device=DEV, dtype=torch.float8_e4m3fn), torch.empty(_blocks(k), t, device=DEV)
    else:
        s["out"] = torch.empty(t, k, device=DEV, dtype=dt)
    return s


# ---- one pass -----------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if own:
        return _library(s, c)
    if c["op"] == "norm":
        return _normed(s, c)
    if c["op"] == "quantise":
        x = s["x"].float()
        if c["act"] != "none":
            a, b = x[:, :c["k"]], x[:, c["k"]:]
            x = (a / (1 + torch.exp(-a)) if c["act"] == "silu" else 0.5 * a * (1 + torch.tanh(math.sqrt(2 / math.pi) * (a + 0.044715 * a * a * a)))) * b
        codes, scales = _quantised(x)
        return {"codes": codes, "scales": scales}
    if c["op"] == "route":
        return _routed(s, c)
    x = s["x"].float() * _wide(s["xs"].t(), c["k"])
    w = s["w"].float() * _wide(s["ws"].repeat_interleave(BLOCK, -2)[..., :c["n"], :], c["k"])
    if c["op"] == "matmul":
        return {"out": (x @ w.t()).to(s["out"].dtype)}
    # groups padded to the largest one
    at = s["offsets"][:-1, None] + torch.arange(s["most"], device=DEV)
    has = at < s["offsets"][1:, None]
    row = torch.where(has, at, 0).long()
    y = torch.bmm(x[s["rows"][row].long() if c["gathered"] else row], w.transpose(1, 2).contiguous())
    return {"out": y[has].to(s["out"].dtype)}


def _library(s, c):
    import paper_2512_20210_amd as plora
    h = s.get("handles")
    if h is None:
        h = s["handles"] = {}
        if "codes" in s:
            h["out8"] = plora.Fp8Rows(s["codes"], s["scales"])
        if c["op"] == "norm":
            of = lambda p: plora.NormWeights(s[p + "_weight"], s[p + "_bias"], EPS, c["center"])  # noqa: E731
            h["norm"] = plora.BlockNorm(of("pre"), of("post") if c["post"] else None, c["scale"])
        elif c["op"] == "quantise":
            h["act"] = {"none": plora.PLORA_ACT_NONE, "silu": plora.PLORA_ACT_SILU, "gelu": plora.PLORA_ACT_GELU}[c["act"]]
        elif c["op"] == "route":
            h["routing"] = plora.Routing(s["experts"], s["weights"], s["offsets"], s["rows"], s["places"], s["workspace"])
        else:
            h["x"], h["w"] = plora.Fp8Rows(s["x"], s["xs"]), plora.Fp8Weights(s["w"], s["ws"])
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "norm":
        h["norm"].run(s["block"], s["residual"], s["hidden"], s.get("out"), h.get("out8"), s["gate"], s.get("places"), s.get("place_weights"), stream)
        return {"hidden": s["hidden"], "codes": s["codes"], "scales": s["scales"]} if c["eight"] else {"hidden": s["hidden"], "out": s["out"]}
    if c["op"] == "quantise":
        h["out8"].quantise(s["x"], h["act"], stream)
        return {"codes": s["codes"], "scales": s["scales"]}
    if c["op"] == "route":
        h["routing"].route(s["logits"], True, 1.0, stream)
        return {name: s[name] for name in ("experts", "weights", "offsets", "rows", "places")}
    if c["op"] == "matmul":
        h["w"].matmul(h["x"], s["out"], stream)
    else:
        h["w"].grouped(h["x"], s["offsets"], s["out"], s["rows"], stream)
    return {"out": s["out"]}


# ---- plain forms --------------------------------------------------------------------------------------

def _wide(scales, k):
    """A scale for each block of 128 channels as one for each channel."""
    return scales.repeat_interleave(BLOCK, -1)[..., :k]


def _quantised(x):
    """Rows of x in 8 bits: (codes [rows][k], scales [blocks][rows])."""
    rows, k = x.shape
    pad = torch.nn.functional.pad(x, (0, -k % BLOCK)).view(rows, -1, BLOCK)
    amax = pad.abs().amax(-1, keepdim=True)
    none = amax < TINY
    top = torch.full_like(amax, TOP)
    scale = torch.where(none, 0.0, amax / top)
    inverse = torch.where(none, 0.0, top / amax)
    codes = (pad * inverse).to(torch.float8_e4m3fn).view(rows, -1)[:, :k]
    return codes.contiguous(), scale[..., 0].t().contiguous()


def _norm_of(x, weight, bias):
    x = x - x.mean(-1, keepdim=True) if bias is not None else x
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    return y if bias is None else y + bias.float()


def _normed(s, c):
    u = s["block"].float()
    if c["top_k"]:
        u = (u[s["places"].long()] * s["place_weights"][..., None]).sum(1)
    if c["post"]:
        u = _norm_of(u, s["post_weight"], s["post_bias"])
    u = c["scale"] * u
    u = u * s["gate"].float() if c["gate"] else u
    hidden = u + s["residual"].float() if c["residual"] else u
    y = _norm_of(hidden, s["pre_weight"], s["pre_bias"])
    dt = s["block"].dtype
    if not c["eight"]:
        return {"hidden": hidden.to(dt), "out": y.to(dt)}
    codes, scales = _quantised(y)
    return {"hidden": hidden.to(dt), "codes": codes, "scales": scales}


def _routed(s, c):
    x, e, j = s["logits"].float(), c["experts"], c["top_k"]
    value, index = torch.sort(x, dim=-1, descending=True, stable=True)  # ties: the lowest index first
    value, index = value[:, :j], index[:, :j]
    some = value > -math.inf
    experts = torch.where(some, index, -1)
    w = torch.exp(value - torch.where(some[:, :1], value[:, :1], 0.0))
    w = torch.where(some, w / torch.where(some[:, :1], w.sum(-1, keepdim=True), 1.0), 0.0)
    flat = torch.where(some, index, e).reshape(-1)
    order = torch.sort(flat, stable=True)[1]
    at = torch.empty_like(order)
    at[order] = torch.arange(order.numel(), device=DEV)
    places = torch.where(some, at.view(-1, j), -1)
    counts = torch.bincount(flat, minlength=e + 1)[:e]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    rows = torch.where(flat[order] < e, order // j, -1)
    i32 = torch.int32
    return {"experts": experts.to(i32), "weights": w, "offsets": offsets.to(i32), "rows": rows.to(i32), "places": places.to(i32)}


# ---- definitions in 64 bits ---------------------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "norm":
        return _exact_norm(c, s)
    if c["op"] == "quantise":
        x = s["x"].double()
        if c["act"] != "none":
            gate = x[:, :c["k"]]
            inner = math.sqrt(2 / math.pi) * (gate + 0.044715 * gate ** 3)
            x = x[:, c["k"]:] * gate * (torch.sigmoid(gate) if c["act"] == "silu" else torch.sigmoid(2 * inner))
        return _exact_eight(x)
    if c["op"] == "route":
        p = torch.softmax(s["logits"].double(), -1).nan_to_num(0.0).cpu().numpy()
        best = -np.sort(-p, axis=1)[:, :c["top_k"]]
        total = best.sum(1, keepdims=True)
        return {"experts": None, "weights": best / np.where(total > 0, total, 1.0), "offsets": None, "rows": None, "places": None}
    k, n = c["k"], c["n"]
    channel, unit = torch.arange(k, device=DEV) // BLOCK, torch.arange(n, device=DEV) // BLOCK
    x = s["x"].double() * s["xs"].double()[channel].t()
    if c["op"] == "matmul":
        return {"out": torch.mm(x, (s["w"].double() * s["ws"].double()[unit][:, channel]).t())}
    out, edge = torch.empty(s["out"].shape, device=DEV, dtype=torch.float64), s["offsets"].tolist()
    for e in range(c["experts"]):
        a, b = edge[e], edge[e + 1]
        if a < b:
            part = x[s["rows"][a:b].long()] if c["gathered"] else x[a:b]
            out[a:b] = torch.mm(part, (s["w"][e].double() * s["ws"][e].double()[unit][:, channel]).t())
    return {"out": out}


def _exact_eight(x):
    """Codes and scales from their definition: a value's step is 2^-3 of its power of two, and 2^-9 below 2^-6."""
    rows, k = x.shape
    block = torch.arange(k, device=DEV) // BLOCK
    amax = torch.zeros(rows, _blocks(k), device=DEV, dtype=torch.float64).scatter_reduce_(1, block.expand(rows, k), x.abs(), "amax")
    amax = torch.where(amax < TINY, 0.0, amax)
    v = torch.where(amax[:, block] > 0, x * TOP / amax[:, block], 0.0)
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return {"codes": torch.round(v / step) * step, "scales": (amax / TOP).t().contiguous()}


def _exact_norm(c, s):
    get = lambda name: None if s.get(name) is None else s[name].double()  # noqa: E731

    def unit(v, name):
        if c["center"]:
            v = v - v.mean(1, keepdim=True)
        v = v / torch.sqrt(v.square().mean(1, keepdim=True) + EPS) * get(name + "_weight")
        return v + get(name + "_bias") if c["center"] else v

    block = get("block")
    if c["top_k"]:
        total = torch.zeros(c["tokens"], c["k"], device=DEV, dtype=torch.float64)
        for j in range(c["top_k"]):
            total += block[s["places"][:, j].long()] * s["place_weights"][:, j:j + 1].double()
        block = total
    if c["post"]:
        block = unit(block, "post")
    hidden = c["scale"] * block * (get("gate") if c["gate"] else 1.0)
    if c["residual"]:
        hidden = hidden + get("residual")
    y = unit(hidden, "pre")
    return {"hidden": hidden, **(_exact_eight(y) if c["eight"] else {"out": y})}
