"""What lies around attention in a model that answers questions about frames and regions: norms, products and the choice of a token.

Three kinds of call, over tokens of regions (49 each) and of clips (32 frames of 20 x 20), single answer tokens and short texts:

  norm     the residual's sum and its root-mean-square norm, in the states' type or in 8 bits (E4M3, one power of two for each 32 values),
           and what those 8 bits hold
  product  rows times the weights of a layer with bias, activation (or the product of two halves, one of them activated) and residual,
           in the states' type or from 8 bits
  sample   one token of each row of logits: temperature, top-k, top-p, min-p and a given random number

`run` is one pass; with `own` it goes through the package's public calls, otherwise through the plain form: elementary
torch operations in 32 bits (the sums of a distribution in 64: the token is where a sum passes a border).
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6
# a drawn case costs no more than this: the largest listed pass by traffic and by arithmetic
MOST_BYTES, MOST_FLOPS = 1.1e9, 2.6e12


def listed():
    return [
        # the states of sixteen running answers on their way into a layer of 8 bits: latency
        dict(name="norm_token", kind="norm", dtype="bf16", tokens=16, width=4096, res=True, out="mx8"),
        # tokens of 300 regions, 7 x 7 each
        dict(name="norm_regions_f32", kind="norm", dtype="f32", tokens=14700, width=256, res=True, out="plain"),
        # a clip of 32 frames of 20 x 20 tokens on its way into a layer of 8 bits
        dict(name="norm_clip", kind="norm", dtype="bf16", tokens=12800, width=4096, res=True, out="mx8"),
        # one answer token through an output layer: latency
        dict(name="product_token", kind="product", dtype="bf16", rows="plain", tokens=1, k=4096, cols=4096, act="none", gated=False, bias=True, res=True, out="plain"),
        # sixteen answer tokens through the two halves of a gated layer, everything in 8 bits
        dict(name="gate_token_mx8", kind="product", dtype="bf16", rows="mx8", tokens=16, k=4096, cols=12288, act="silu", gated=True, bias=False, res=False, out="mx8"),
        # logits of sixteen answer tokens
        dict(name="logits_token", kind="product", dtype="bf16", rows="plain", tokens=16, k=4096, cols=131072, act="none", gated=False, bias=False, res=False, out="f32"),
        # four short questions of 77 tokens, widths that are no multiples of a tile
        dict(name="product_text_f16", kind="product", dtype="f16", rows="plain", tokens=308, k=1160, cols=1100, act="gelu", gated=False, bias=True, res=True, out="plain"),
        # a clip of 32 frames of 20 x 20 tokens through an output layer
        dict(name="product_clip", kind="product", dtype="bf16", rows="plain", tokens=12800, k=4096, cols=4096, act="none", gated=False, bias=False, res=True, out="plain"),
        # the same through the two halves of a gated layer of 8 bits
        dict(name="gate_clip_mx8", kind="product", dtype="bf16", rows="mx8", tokens=12800, k=4096, cols=12288, act="silu", gated=True, bias=False, res=False, out="plain"),
        # the next token of one answer: latency
        dict(name="sample_token", kind="sample", dtype="bf16", rows=1, vocab=32768, settings="topk"),
        # the next tokens of 48 answers, each with settings of its own
        dict(name="sample_batch_f32", kind="sample", dtype="f32", rows=48, vocab=131072, settings="mixed"),
        # many answers at once, an odd number of words, all cut by probability
        dict(name="sample_many", kind="sample", dtype="bf16", rows=512, vocab=100003, settings="topp"),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _drawn(rng):
    kind = rng.choice(["norm", "product", "product", "sample"])
    if kind == "norm":
        out = rng.choice(["plain", "mx8"])
        width = _spread(rng, 32, 16384)
        return dict(kind=kind, dtype=rng.choice(["bf16", "f16", "f32"]), tokens=_spread(rng, 1, 51200), width=(width + 31) // 32 * 32 if out == "mx8" else width, res=rng.random() < 0.7, out=out)
    if kind == "sample":
        return dict(kind=kind, dtype=rng.choice(["bf16", "f16", "f32"]), rows=_spread(rng, 1, 512), vocab=_spread(rng, 1000, 262144), settings=rng.choice(["topk", "topp", "minp", "mixed", "none"]))
    rows = rng.choice(["plain", "mx8"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f16", "f32"]) if rows == "plain" else rng.choice(["bf16", "f16"])
    unit = 32 if rows == "mx8" else 8
    out = rng.choice(["plain", "plain", "f32", "mx8"] if dtype != "f32" else ["plain"])
    cols = _spread(rng, 64, 32768)
    return dict(kind=kind, dtype=dtype, rows=rows, tokens=_spread(rng, 1, 12800), k=_spread(rng, 64, 16384) // unit * unit, cols=(cols + 31) // 32 * 32 if out == "mx8" else cols,
                act=rng.choice(["none", "relu", "silu", "gelu"]), gated=rng.random() < 0.3, bias=rng.random() < 0.5, res=out != "mx8" and rng.random() < 0.5, out=out)


def draw(rng):
    while True:
        c = _drawn(rng)
        w = work(c)
        if w["bytes"] <= MOST_BYTES and w["flops"] * (16 if c["dtype"] == "f32" else 1) <= MOST_FLOPS:
            return c


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _to_mx8(x):
    """Codes (uint8, E4M3) and exponent bytes of x [rows][width], fp32: groups of 32, the smallest power of two that keeps them within 448."""
    u = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(u.abs().amax(-1, keepdim=True))
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-126, 127)
    return torch.ldexp(u, -e).to(torch.float8_e4m3fn).flatten(-2).view(torch.uint8), (e[..., 0] + 127).to(torch.uint8)


def _of_mx8(codes, exps):
    return (codes.view(torch.float8_e4m3fn).float().unflatten(-1, (-1, 32)) * torch.exp2(exps.float() - 127)[..., None]).flatten(-2)


def _states(g, rows, width):
    """Values as they run through a model: normal, some channels several times larger than the others."""
    x = torch.randn(rows, width, generator=g, device="cuda")
    return x.mul_(1.0 + 5.0 * (torch.rand(width, generator=g, device="cuda") < 0.04))


def _settings(g, c):
    """temperature, top_k, top_p, min_p of the rows as a running batch has them; 0, 0, 1 and 0 stand for none."""
    n, kind = c["rows"], c["settings"]
    some = lambda share: torch.rand(n, generator=g, device="cuda") < share  # noqa: E731
    one = lambda: torch.rand(n, generator=g, device="cuda")  # noqa: E731
    mixed = kind == "mixed"
    temperature = 0.3 + 1.2 * one()
    top_k = torch.randint(1, 200, (n,), generator=g, device="cuda", dtype=torch.int32)
    top_p, min_p = 0.5 + 0.49 * one(), 0.01 + 0.2 * one()
    if mixed:
        temperature = torch.where(some(0.15), 0.0, temperature)
    top_k = torch.where(some(0.4 if mixed else 1.0 if kind == "topk" else 0.0), top_k, 0)
    top_p = torch.where(some(0.5 if mixed else 1.0 if kind == "topp" else 0.0), top_p, 1.0)
    min_p = torch.where(some(0.3 if mixed else 1.0 if kind == "minp" else 0.0), min_p, 0.0)
    return dict(temperature=temperature.float(), top_k=top_k.to(torch.int32), top_p=top_p.float(), min_p=min_p.float())


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[c["dtype"]]
    s = dict(case=c)
    shown = torch.bfloat16 if c["dtype"] == "f32" else t   # what 8 bits hold is exact in bf16
    if c["kind"] == "norm":
        n, w = c["tokens"], c["width"]
        s.update(x=_states(g, n, w).to(t), res=_states(g, n, w).mul_(3.0).to(t) if c["res"] else None, weight=1.0 + 0.2 * torch.randn(w, generator=g, device="cuda"),
                 sum=torch.empty(n, w, dtype=t, device="cuda") if c["res"] else None, y=torch.empty(n, w, dtype=shown if c["out"] == "mx8" else t, device="cuda"))
        if c["out"] == "mx8":
            s["held"] = (torch.empty(n, w, dtype=torch.uint8, device="cuda"), torch.empty(n, w // 32, dtype=torch.uint8, device="cuda"))
        return s
    if c["kind"] == "sample":
        n, v = c["rows"], c["vocab"]
        logits = torch.randn(n, v, generator=g, device="cuda").mul_(2.0)
        # a few words stand out in every row; one in a hundred is not allowed, and of many rows one has none left
        likely = torch.randint(0, v, (n, 24), generator=g, device="cuda")
        logits.scatter_add_(1, likely, 4.0 + 6.0 * torch.rand(n, 24, generator=g, device="cuda"))
        logits.masked_fill_(torch.rand(v, generator=g, device="cuda") < 0.01, -math.inf)
        if n > 40:
            logits[n // 2] = -math.inf
        s.update(logits=logits.to(t), u=torch.rand(n, generator=g, device="cuda"), token=torch.empty(n, dtype=torch.int32, device="cuda"), kept=torch.empty(n, dtype=torch.int32, device="cuda"),
                 logprob=torch.empty(n, dtype=torch.float32, device="cuda"), **_settings(g, c))
        return s
    n, k, cols = c["tokens"], c["k"], c["cols"]
    wide = cols * (2 if c["gated"] else 1)
    x = _states(g, n, k)
    w = torch.randn(wide, k, generator=g, device="cuda").mul_(1.0 / math.sqrt(k))
    out = torch.float32 if c["out"] == "f32" else t
    s.update(x=_to_mx8(x) if c["rows"] == "mx8" else x.to(t), w=_to_mx8(w) if c["rows"] == "mx8" else w.to(t), bias=torch.randn(wide, generator=g, device="cuda") if c["bias"] else None,
             res=_states(g, n, cols).to(out) if c["res"] else None, y=torch.empty(n, cols, dtype=out, device="cuda"))
    if c["out"] == "mx8":
        s["held"] = (torch.empty(n, cols, dtype=torch.uint8, device="cuda"), torch.empty(n, cols // 32, dtype=torch.uint8, device="cuda"))
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------

def _act(name, x):
    if name == "relu":
        return torch.clamp(x, min=0.0)
    if name == "silu":
        return x / (1.0 + torch.exp(-x))
    if name == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    return x


def _plain_norm(s):
    c, t = s["case"], s["x"].dtype
    u = s["x"].float()
    if s["res"] is not None:
        u = u + s["res"].float()
    y = u * torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS) * s["weight"]
    out = {"y": (_of_mx8(*_to_mx8(y)) if c["out"] == "mx8" else y).to(s["y"].dtype)}
    if s["res"] is not None:
        out["sum"] = u.to(t)
    return out


def _plain_product(s):
    c = s["case"]
    x, w = (_of_mx8(*s["x"]), _of_mx8(*s["w"])) if c["rows"] == "mx8" else (s["x"].float(), s["w"].float())
    y = x @ w.T
    if s["bias"] is not None:
        y = y + s["bias"]
    if c["gated"]:
        y = _act(c["act"], y[:, :c["cols"]]) * y[:, c["cols"]:]
    else:
        y = _act(c["act"], y)
    if s["res"] is not None:
        y = y + s["res"].float()
    return {"y": (_of_mx8(*_to_mx8(y)) if c["out"] == "mx8" else y).to(s["y"].dtype)}


def _plain_sample(s):
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    v, order = torch.sort(x, descending=True, stable=True)
    there = v > -math.inf
    some = there.any(-1)
    greedy = ~(s["temperature"] > 0)
    scale = torch.where(greedy, 1.0, s["temperature"]).double()[:, None]
    top = torch.where(some, v[:, 0], 0.0).double()[:, None]
    w = torch.where(there, torch.exp((v.double() - top) / scale), 0.0)
    rank = torch.arange(v.shape[1], device=v.device)
    limit = torch.where(s["top_k"] > 0, s["top_k"], v.shape[1])
    limit = torch.where(greedy, 1, limit)[:, None]
    keep = there & (rank < limit)
    w = torch.where(keep, w, 0.0)
    up_to = torch.cumsum(w, -1)
    cut = (s["top_p"] < 1.0)[:, None] & (up_to - w >= s["top_p"].double()[:, None] * up_to[:, -1:])
    keep = keep & ~(cut & (rank > 0)) & ((w >= s["min_p"].double()[:, None]) | (rank == 0))
    w = torch.where(keep, w, 0.0)
    by_index = torch.zeros_like(w).scatter_(1, order, w)
    up_to = torch.cumsum(by_index, -1)
    total = up_to[:, -1:]
    token = (up_to > s["u"].double()[:, None] * total).to(torch.int8).argmax(-1)
    prob = by_index.gather(1, token[:, None])[:, 0] / torch.where(some, total[:, 0], 1.0)
    return {"token": torch.where(some, token, -1).to(torch.int32), "kept": keep.sum(-1).to(torch.int32), "logprob": torch.log(prob).float()}


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2502_01277_amd import binding
        if c["kind"] == "norm":
            y = binding.Mx8(*s["held"]) if c["out"] == "mx8" else s["y"]
            binding.op_norm(s["x"], y, s["weight"], res=s["res"], total=s["sum"], eps=EPS)
            if c["out"] == "mx8":
                binding.op_mx8_load(y, s["y"])
            return {"y": s["y"], "sum": s["sum"]} if c["res"] else {"y": s["y"]}
        if c["kind"] == "sample":
            binding.op_sample(s["logits"], s["u"], s["token"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], logprob=s["logprob"], kept=s["kept"])
            return {"token": s["token"], "kept": s["kept"], "logprob": s["logprob"]}
        x, w = (binding.Mx8(*s["x"]), binding.Mx8(*s["w"])) if c["rows"] == "mx8" else (s["x"], s["w"])
        y = binding.Mx8(*s["held"]) if c["out"] == "mx8" else s["y"]
        binding.op_product(x, w, y, bias=s["bias"], act=c["act"], gated=c["gated"], res=s["res"])
        if c["out"] == "mx8":
            binding.op_mx8_load(y, s["y"])
        return {"y": s["y"]}
    if c["kind"] == "norm":
        return _plain_norm(s)
    if c["kind"] == "sample":
        return _plain_sample(s)
    return _plain_product(s)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    c = case
    es = BYTES[c["dtype"]]
    if c["kind"] == "norm":
        values = c["tokens"] * c["width"]
        # 8 bits are written, read again and given out as values
        out = 2 + 2 * 33 / 32 if c["out"] == "mx8" else es
        return {"bytes": values * ((3 if c["res"] else 1) * es + out) + 4 * c["width"], "flops": 5 * values}
    if c["kind"] == "sample":
        return {"bytes": c["rows"] * (c["vocab"] * es + 32), "flops": 4 * c["rows"] * c["vocab"]}
    wide = c["cols"] * (2 if c["gated"] else 1)
    value = 33 / 32 if c["rows"] == "mx8" else es
    y = 4 if c["out"] == "f32" else es
    out = y + 2 * 33 / 32 if c["out"] == "mx8" else y * (2 if c["res"] else 1)
    return {"bytes": (c["tokens"] + wide) * c["k"] * value + c["tokens"] * c["cols"] * out + (4 * wide if c["bias"] else 0), "flops": 2 * c["tokens"] * wide * c["k"]}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def _exact_held(x):
    """The values of E4M3 nearest to x / 2^e, times 2^e: multiples of 2^(p - 3) between 2^p and 2^(p + 1), of 2^-9 below 2^-6; ties to even."""
    u = x.reshape(x.shape[0], -1, 32)
    most = u.abs().amax(-1, keepdim=True)
    e = torch.where(most > 0, torch.ceil(torch.log2(most / 448)), torch.full_like(most, -126))
    e = torch.where(most <= 448 * torch.exp2(e - 1), e - 1, torch.where(most > 448 * torch.exp2(e), e + 1, e)).clamp(-126, 127)
    r = u / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(r.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(r / step) * step * torch.exp2(e)).reshape(x.shape)


def _exact_values(held):
    """Values of E4M3 codes from their bits, times the power of two of their group."""
    codes, exps = held
    code, out = torch.arange(256, device=codes.device), None
    power, fraction = (code >> 3 & 15).double(), (code & 7).double()
    value = torch.where(power > 0, torch.exp2(power - 7) * (1 + fraction / 8), fraction * 2.0 ** -9) * torch.where(code >= 128, -1.0, 1.0)
    out = value[codes.long()]
    return out * torch.exp2(exps.double() - 127).repeat_interleave(32, 1)


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "norm":
        y, total = [], []
        for rows in torch.arange(c["tokens"], device="cuda").split(4096):
            u = s["x"][rows].double()
            if c["res"]:
                u = u + s["res"][rows].double()
                total.append(u)
            v = u / (u.pow(2).sum(-1, keepdim=True) / c["width"] + EPS).sqrt() * s["weight"].double()
            y.append(_exact_held(v) if c["out"] == "mx8" else v)
        return {"y": torch.cat(y), "sum": torch.cat(total)} if c["res"] else {"y": torch.cat(y)}
    if c["kind"] == "product":
        if c["rows"] == "mx8":
            x, w = _exact_values(s["x"]), _exact_values(s["w"])
        else:
            x, w = s["x"].double(), s["w"].double()
        y = torch.empty(c["tokens"], c["cols"], dtype=torch.float64, device="cuda")

        def half(rows, first):
            z = x[rows] @ w[first:first + c["cols"]].T
            return z if s["bias"] is None else z.add_(s["bias"][first:first + c["cols"]].double())

        for rows in torch.arange(c["tokens"], device="cuda").split(1024):
            z = half(rows, 0)
            if c["act"] == "relu":
                z = z * (z > 0)
            elif c["act"] == "silu":
                z = z * torch.sigmoid(z)
            elif c["act"] == "gelu":
                z = z * (0.5 * torch.special.erfc(z * -math.sqrt(0.5)))
            if c["gated"]:
                z = z * half(rows, c["cols"])
            if s["res"] is not None:
                z = z + s["res"][rows].double()
            y[rows] = _exact_held(z) if c["out"] == "mx8" else z
        return {"y": y}
    logprob = torch.full((c["rows"],), -math.inf, dtype=torch.float64, device="cuda")
    settings = [s[name].tolist() for name in ("temperature", "top_k", "top_p", "min_p", "u")]
    for r, (temperature, top_k, top_p, min_p, u) in enumerate(zip(*settings)):
        x = s["logits"][r].double()
        words = torch.nonzero(x > -math.inf)[:, 0]
        if not len(words):
            continue
        if temperature <= 0:
            logprob[r] = 0.0
            continue
        words = words[torch.sort(-x[words], stable=True)[1]]
        if top_k > 0:
            words = words[:top_k]
        share = torch.softmax(x[words] / temperature, 0)
        count = len(words)
        if top_p < 1:
            count = min(count, max(1, int((torch.cumsum(share, 0) < top_p).sum()) + 1))
        words, share = words[:count], share[:count]
        near = share >= min_p * share[0]
        near[0] = True
        words, share = words[near], share[near]
        words, back = torch.sort(words)
        share = share[back] / share.sum()
        at = min(len(words) - 1, int((torch.cumsum(share, 0) <= u).sum()))
        logprob[r] = torch.log(share[at])
    return {"token": None, "kept": None, "logprob": logprob}
