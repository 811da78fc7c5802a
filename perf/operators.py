"""Operators of a serving step around the compensated layers, as cases that can be timed and compared.

A decoder block of a served model runs  q|k|v projection -> per-head norm and position rotation, new keys and values into
a paged cache -> attention over that cache -> o projection -> gate|up, down.  The compensated layers are the projections;
these cases are what stands between and beside them:

  adapters   low-rank adapters of many requests at once, beside a projection that the requests share:
             y[i] = base[i] + s_j (x[i] . A_j) . B_j   with j = ids[i]   (base[i] where the token has no adapter)
  rotate     norms of queries and keys for each head, rotation by the token's position, and the new keys and values put
             into a paged cache, in one pass
  attend     attention of one new token per sequence over a paged cache

`own` false: the plain form in elementary torch operations; true: the library's entry points.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    lora = {"op": "adapters", "ranks": "equal", "none": 0, "runs": 0, "x": "f16", "y": "f16"}
    rot = {"op": "rotate", "heads": 32, "kv": 8, "dim": 128, "rot": 128, "pairs": "half", "norm": True, "fused": False, "page": 16, "padded": 0, "x": "bf16", "far": 8192}
    att = {"op": "attend", "heads": 32, "kv": 8, "dim": 128, "page": 16, "layout": "hnd", "x": "bf16", "window": 0}
    return [
        # the smallest call there is: one request decoding, a small adapter beside the key projection of an 8B model
        {**lora, "name": "adapters, 1 token", "d_in": 4096, "d_out": 1024, "rank": 16, "adapters": 8, "m": 1},
        # a decode batch of requests that nearly all have a task of their own, adapters of several ranks in one bank
        {**lora, "name": "adapters, 32 requests", "d_in": 4096, "d_out": 4096, "rank": 64, "ranks": "mixed", "adapters": 48, "m": 32, "none": 2, "x": "bf16", "y": "bf16"},
        # an odd batch beside an up projection, the sum kept in 32 bits for what follows
        {**lora, "name": "adapters, 61 tokens, f32 out", "d_in": 4096, "d_out": 14336, "rank": 128, "adapters": 5, "m": 61, "none": 3, "y": "f32"},
        # prompts of nine requests in one batch beside the down projection
        {**lora, "name": "adapters, prompts, 2048 tokens", "d_in": 14336, "d_out": 4096, "rank": 64, "adapters": 16, "m": 2048, "runs": 9, "none": 131, "x": "bf16", "y": "bf16"},
        # one token of an 8B model that has no norms of heads: rotation and cache only
        {**rot, "name": "rotate, 1 token", "norm": False, "m": 1, "x": "f16"},
        # a decode batch padded to the size of its captured graph, q|k|v the columns of one product, neighbouring pairs
        {**rot, "name": "rotate, 48 tokens, padded", "heads": 16, "kv": 2, "pairs": "adjacent", "fused": True, "m": 48, "padded": 5, "far": 131072},
        # a prompt of odd length with wide heads of which only the first channels rotate
        {**rot, "name": "rotate, 333 tokens, partly", "heads": 8, "kv": 1, "dim": 256, "rot": 64, "page": 64, "m": 333, "x": "f16"},
        # the prompts of a batch, prefilled in one pass
        {**rot, "name": "rotate, 8192 tokens", "m": 8192, "page": 64},
        # one short conversation of an 8B model
        {**att, "name": "attend, 1 x 1000", "batch": 1, "short": 1000, "long": 1000, "x": "f16"},
        # a few requests with narrow heads in groups of seven that look back over a window only, small pages
        {**att, "name": "attend, 13, window", "heads": 14, "kv": 2, "dim": 64, "batch": 13, "short": 0, "long": 9001, "window": 4096},
        # a serving batch of ragged lengths, cache with the heads of a token side by side
        {**att, "name": "attend, 64 x 512-8192", "batch": 64, "short": 512, "long": 8192, "layout": "nhd", "page": 64},
        # one very long document
        {**att, "name": "attend, 1 x 131072", "batch": 1, "short": 131072, "long": 131072, "page": 64},
    ]


# ------------------------------------------------------------------------------------------------------- the sizes
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _mult(v, q):
    return max(q, int(round(v / q)) * q)


def draw(rng):
    op = rng.choice(["adapters", "rotate", "attend"])
    most = max((work(c) for c in listed() if c["op"] == op), key=lambda w: w["bytes"])
    while True:
        c = {"adapters": _draw_adapters, "rotate": _draw_rotate, "attend": _draw_attend}[op](rng)
        w = work(c)
        held = 4 * sum(_lengths(c)) * c["kv"] * c["dim"] if op == "attend" else 0      # a window leaves the rest of the cache where it is
        if max(w["bytes"], held) <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


def _draw_adapters(rng):
    x = rng.choice(["f16", "bf16"])
    m = _log_int(rng, 1, 2048)
    n = _log_int(rng, 1, 64)
    return {"op": "adapters", "ranks": rng.choice(["equal", "mixed"]), "x": x, "y": rng.choice([x, x, "f32"]), "rank": rng.choice([8, 16, 32, 64, 128, 8 * rng.randint(1, 16)]),
            "d_in": _mult(_log_int(rng, 512, 14336), 128), "d_out": _mult(_log_int(rng, 512, 14336), 32), "adapters": n, "m": m,
            "runs": rng.randint(1, 12) if m > 64 else 0, "none": rng.choice([0, 0, m // 10])}


def _draw_rotate(rng):
    dim = rng.choice([64, 96, 128, 128, 256])
    kv = rng.choice([1, 2, 4, 8])
    m = _log_int(rng, 1, 8192)
    return {"op": "rotate", "heads": kv * rng.choice([1, 2, 4, 5, 7, 8]), "kv": kv, "dim": dim, "rot": rng.choice([dim, dim, dim // 2]), "pairs": rng.choice(["half", "adjacent"]),
            "norm": rng.random() < 0.7, "fused": rng.random() < 0.5, "page": rng.choice([16, 32, 64, 128]), "padded": rng.choice([0, 0, m // 8]), "x": rng.choice(["f16", "bf16"]),
            "far": _log_int(rng, 8192, 131072), "m": m}


def _draw_attend(rng):
    kv = rng.choice([1, 2, 4, 8])
    long = _log_int(rng, 1, 131072)
    return {"op": "attend", "heads": kv * rng.choice([1, 2, 4, 5, 7, 8, 12, 16]), "kv": kv, "dim": rng.choice([64, 96, 128, 128, 256]), "page": rng.choice([16, 32, 64, 128]),
            "layout": rng.choice(["hnd", "nhd"]), "x": rng.choice(["f16", "bf16"]), "window": rng.choice([0, 0, 0, _log_int(rng, 128, 8192)]),
            "batch": _log_int(rng, 1, 256), "short": rng.choice([long, long // 2, long // 16, 0]), "long": long}


def _spread(i, lo, hi):
    """Values over [lo, hi] that are the same for every seed, so that a case's work is; the largest comes first."""
    return hi - int((i * 0.6180339887498949) % 1.0 * (hi - lo) + 0.5)


def _lengths(c):
    return [_spread(i, c["short"], c["long"]) for i in range(c["batch"])]


def _seen(c):
    return [min(n, c["window"]) if c["window"] else n for n in _lengths(c)]


def _rank(c, j):
    return c["rank"] if c["ranks"] == "equal" else max(4, c["rank"] >> (j % 3))


def _ids(c):
    """The adapter of every token, before a seed puts them in order: one list per run of tokens that stay together."""
    with_one = c["m"] - c["none"]
    if not c["runs"]:
        return [[i % c["adapters"]] for i in range(with_one)] + [[-1] for _ in range(c["none"])]
    share = [1 + 3 * ((j * 0.6180339887498949) % 1.0) for j in range(c["runs"])]
    cut = [int(with_one * sum(share[:j]) / sum(share)) for j in range(c["runs"])] + [with_one]
    return [[j % c["adapters"]] * (cut[j + 1] - cut[j]) for j in range(c["runs"])] + [[-1] * c["none"]]


# -------------------------------------------------------------------------------------------------------- the inputs
class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0, dtype=torch.float16):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=self.g)

    def perm(self, n):
        return torch.randperm(n, device=DEV, generator=self.g)


def prepare(case, seed):
    c, g = case, _Gen(seed)
    s = {"c": c, "plan": None}
    {"adapters": _prepare_adapters, "rotate": _prepare_rotate, "attend": _prepare_attend}[c["op"]](s, c, g)
    if own:
        s["plan"] = {"adapters": _plan_adapters, "rotate": _plan_rotate, "attend": _plan_attend}[c["op"]](s, c)
    return s


def _prepare_adapters(s, c, g):
    t, n, r = TORCH[c["x"]], c["adapters"], c["rank"]
    s["a"] = g.normal(n, c["d_in"], r, std=0.02, dtype=t)      # columns behind an adapter's rank: what a wider one left there
    s["b"] = g.normal(n, r, c["d_out"], std=0.02, dtype=t)
    s["ranks"] = torch.tensor([_rank(c, j) for j in range(n)], dtype=torch.int32, device=DEV)
    s["scales"] = 0.5 + torch.rand(n, device=DEV, generator=g.g)
    runs = _ids(c)
    s["ids"] = torch.tensor([i for k in g.perm(len(runs)).tolist() for i in runs[k]], dtype=torch.int32, device=DEV)
    s["x"] = g.normal(c["m"], c["d_in"], dtype=t)
    s["base"] = g.normal(c["m"], c["d_out"], dtype=TORCH[c["y"]])
    s["y"] = torch.empty_like(s["base"])


def _cache(g, c, pages):
    """Keys and values of a cache of `pages` pages; viewed as [page, head, token, channel] whatever the order in memory."""
    shape = (pages, c["kv"], c["page"], c["dim"]) if c.get("layout", "hnd") == "hnd" else (pages, c["page"], c["kv"], c["dim"])
    return g.normal(*shape, dtype=TORCH[c["x"]]), g.normal(*shape, dtype=TORCH[c["x"]])


def _by_head(cache, c):
    return cache if c.get("layout", "hnd") == "hnd" else cache.transpose(1, 2)


def _prepare_rotate(s, c, g):
    t, m, d = TORCH[c["x"]], c["m"], c["dim"]
    if c["fused"]:
        both = g.normal(m, (c["heads"] + 2 * c["kv"]) * d, dtype=t)
        s["q"], s["k"], s["v"] = both.split([c["heads"] * d, c["kv"] * d, c["kv"] * d], dim=1)
    else:
        s["q"], s["k"], s["v"] = (g.normal(m, h * d, dtype=t) for h in (c["heads"], c["kv"], c["kv"]))
    s["qw"], s["kw"] = ((1 + 0.1 * g.normal(d, dtype=torch.float32)).to(t) if c["norm"] else None for _ in range(2))
    pos = torch.randint(0, c["far"], (m,), device=DEV, generator=g.g)
    s["positions"] = pos.to(torch.int32)
    angle = torch.arange(c["far"], device=DEV, dtype=torch.float64)[:, None] * (500000.0 ** -(torch.arange(0, c["rot"], 2, device=DEV, dtype=torch.float64) / c["rot"]))
    s["table"] = torch.cat([angle.cos(), angle.sin()], 1).to(torch.float32)
    pages = -(-m // c["page"]) + 2
    s["kc"], s["vc"] = _cache(g, c, pages)
    slots = g.perm(pages * c["page"])[:m].to(torch.int32)
    if c["padded"]:
        slots[m - c["padded"]:] = -1                           # tokens behind the batch: rotated, kept nowhere
    s["slots"] = slots
    s["qo"] = torch.empty((m, c["heads"] * d), dtype=t, device=DEV)


def _prepare_attend(s, c, g):
    lengths = torch.tensor(_lengths(c), device=DEV)[g.perm(c["batch"])]
    need = -(-lengths // c["page"])
    per = max(1, -(-c["long"] // c["page"]))
    pages = int(sum(-(-n // c["page"]) for n in _lengths(c))) + 3
    s["kc"], s["vc"] = _cache(g, c, pages)
    start = torch.cumsum(need, 0) - need
    at = torch.arange(per, device=DEV)
    table = g.perm(pages)[(start[:, None] + at).clamp_(max=pages - 1)]
    s["pages"] = torch.where(at < need[:, None], table, 0).to(torch.int32).contiguous()
    s["lengths"] = lengths.to(torch.int32)
    s["q"] = g.normal(c["batch"], c["heads"] * c["dim"], std=2.0, dtype=TORCH[c["x"]])       # scores with a deviation of two
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((c["batch"], c["heads"]), dtype=torch.float32, device=DEV)


# ---------------------------------------------------------------------------------------------- the library's calls
def _plan_adapters(s, c):
    import paper_2410_21271_b200 as E
    return E.AdapterBank(s["a"], s["b"], ranks=s["ranks"], scales=s["scales"], y_dtype=c["y"])


def _plan_rotate(s, c):
    import paper_2410_21271_b200 as E
    cache = E.PagedCache(s["kc"], s["vc"], layout="hnd")
    return cache, E.QKNormRope(c["heads"], c["kv"], c["dim"], s["table"], q_weight=s["qw"], k_weight=s["kw"], eps=1e-6, pairs=c["pairs"], dtype=c["x"])


def _plan_attend(s, c):
    import paper_2410_21271_b200 as E
    cache = E.PagedCache(s["kc"], s["vc"], layout=c["layout"])
    return cache, E.PagedAttention(c["heads"], c["kv"], c["dim"], page_size=c["page"], max_batch=c["batch"], max_pages=s["pages"].shape[1], dtype=c["x"], window=c["window"])


def run(s):
    return {"adapters": _run_adapters, "rotate": _run_rotate, "attend": _run_attend}[s["c"]["op"]](s, s["c"])


def _run_adapters(s, c):
    if own:
        return s["plan"].forward(s["x"], s["ids"], base=s["base"], y=s["y"])
    n, k, r = s["a"].shape
    # every token against every adapter, then only its own one's columns
    t = (s["x"].float() @ s["a"].float().transpose(0, 1).reshape(k, n * r)).view(-1, n, r)
    mine = s["ids"][:, None] == torch.arange(n, device=DEV)
    there = torch.arange(r, device=DEV) < s["ranks"][:, None]
    t = torch.where(mine[:, :, None] & there, t * s["scales"][:, None], 0.0)
    b = torch.where(there[:, :, None], s["b"].float(), 0.0)
    return (s["base"].float() + t.view(-1, n * r) @ b.view(n * r, -1)).to(s["base"].dtype)


def _run_rotate(s, c):
    if own:
        cache, rope = s["plan"]
        q, _ = rope.forward(s["q"], s["k"], s["v"], s["positions"], slots=s["slots"], cache=cache, q_out=s["qo"])
        return q, s["kc"], s["vc"]
    m, d, half = c["m"], c["dim"], c["rot"] // 2
    cos, sin = s["table"][s["positions"].long()].view(m, 1, 2, half).unbind(2)

    def one(x, w):
        x = x.reshape(m, -1, d).float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        turn, rest = x[..., :2 * half], x[..., 2 * half:]
        if c["pairs"] == "half":
            u, v = turn[..., :half], turn[..., half:]
            turn = torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
        else:
            u, v = turn[..., 0::2], turn[..., 1::2]
            turn = torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)
        return torch.cat([turn, rest], -1).to(s["q"].dtype)

    keep = s["slots"] >= 0
    page, row = s["slots"][keep].long() // c["page"], s["slots"][keep].long() % c["page"]
    _by_head(s["kc"], c)[page, :, row] = one(s["k"], s["kw"])[keep]
    _by_head(s["vc"], c)[page, :, row] = s["v"].reshape(m, -1, d)[keep]
    return one(s["q"], s["qw"]).view(m, -1), s["kc"], s["vc"]


def _run_attend(s, c):
    if own:
        cache, attn = s["plan"]
        return attn.forward(s["q"], cache, s["pages"], s["lengths"], out=s["out"], lse=s["lse"]), s["lse"]
    b, h, d = c["batch"], c["kv"], c["dim"]
    k, v = (_by_head(x, c)[s["pages"].long()].transpose(1, 2).reshape(b, h, -1, d).float() for x in (s["kc"], s["vc"]))
    at = torch.arange(k.shape[2], device=DEV)
    last = s["lengths"][:, None].long()
    seen = at < last
    if c["window"]:
        seen &= at >= last - c["window"]
    score = (s["q"].float().view(b, h, -1, d) / math.sqrt(d)) @ k.transpose(2, 3)
    score = score.masked_fill(~seen[:, None, None, :], -math.inf)
    top = score.amax(-1, keepdim=True).clamp_min(-1e30)          # a sequence without tokens: nothing to subtract
    e = torch.exp(score - top)
    total = e.sum(-1, keepdim=True)
    out = (e @ v.masked_fill(~seen[:, None, :, None], 0.0)) / total.clamp_min(1e-30)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    return out.reshape(b, -1).to(s["q"].dtype), lse.reshape(b, -1)


# ------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"adapters": _exact_adapters, "rotate": _exact_rotate, "attend": _exact_attend}[case["op"]](s, case)


def _exact_adapters(s, c):
    y = s["base"].double()
    for j in set(s["ids"].tolist()) - {-1}:
        rows = (s["ids"] == j).nonzero()[:, 0]
        r = int(s["ranks"][j])
        y[rows] += float(s["scales"][j]) * ((s["x"][rows].double() @ s["a"][j, :, :r].double()) @ s["b"][j, :r].double())
    return y


def _exact_rotate(s, c):
    m, d, half = c["m"], c["dim"], c["rot"] // 2
    at = s["positions"].long()
    turn = torch.complex(s["table"][at, :half].double(), s["table"][at, half:].double())[:, None]

    def one(x, w):
        x = x.double().reshape(m, -1, d).clone()
        if w is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / d + 1e-6) * w.double()
        first, second = (slice(0, half), slice(half, 2 * half)) if c["pairs"] == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    kc, vc, k = s["kc"].double(), s["vc"].double(), one(s["k"], s["kw"])
    for i, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            kc[slot // c["page"], :, slot % c["page"]] = k[i]
            vc[slot // c["page"], :, slot % c["page"]] = s["v"][i].double().view(-1, d)
    return one(s["q"], s["qw"]).reshape(m, -1), kc, vc


def _exact_attend(s, c):
    out = torch.zeros((c["batch"], c["heads"], c["dim"]), dtype=torch.float64, device=DEV)
    lse = torch.full((c["batch"], c["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    for i, n in enumerate(s["lengths"].tolist()):
        if n == 0:
            continue
        tokens = torch.arange(max(0, n - c["window"]) if c["window"] else 0, n, device=DEV)
        page, row = s["pages"][i, tokens // c["page"]].long(), tokens % c["page"]
        for h in range(c["kv"]):
            mine = slice(h * (c["heads"] // c["kv"]), (h + 1) * (c["heads"] // c["kv"]))
            k, v = _by_head(s["kc"], c)[page, h, row].double(), _by_head(s["vc"], c)[page, h, row].double()
            score = s["q"][i].double().view(c["heads"], -1)[mine] @ k.t() / c["dim"] ** 0.5
            lse[i, mine] = torch.logsumexp(score, 1)
            out[i, mine] = torch.softmax(score, 1) @ v
    return out.view(c["batch"], -1), lse


# ------------------------------------------------------------------------------------------------------- accounting
def work(case):
    c = case
    if c["op"] == "adapters":
        ids = [j for run in _ids(c) for j in run]
        yb, width = 4 if c["y"] == "f32" else 2, c["d_in"] + c["d_out"]
        read = sum(2 * _rank(c, j) * width for j in set(ids) - {-1}) + 2 * c["d_in"] * (c["m"] - c["none"])
        return {"bytes": read + 2 * yb * c["m"] * c["d_out"] + 4 * c["m"], "flops": sum(2 * _rank(c, j) * width for j in ids if j >= 0)}
    if c["op"] == "rotate":
        kept = c["m"] - c["padded"]
        moved = 2 * c["dim"] * (c["m"] * (2 * c["heads"] + c["kv"]) + kept * c["kv"] + 2 * kept * c["kv"])
        return {"bytes": moved + c["m"] * (4 * c["rot"] + 8), "flops": c["m"] * (c["heads"] + c["kv"]) * (3 * c["rot"] + (4 * c["dim"] if c["norm"] else 0))}
    tokens = sum(_seen(c))
    pages = sum(-(-n // c["page"]) for n in _seen(c))
    q = c["batch"] * c["heads"] * c["dim"]
    return {"bytes": 4 * tokens * c["kv"] * c["dim"] + 4 * q + 4 * c["batch"] * c["heads"] + 4 * pages + 4 * c["batch"], "flops": 4 * tokens * c["heads"] * c["dim"]}
