"""What a request brings of its own and gets back, around the shared quantized layers, for timing.

Each case is one call that a serving loop makes: rotary positions on the queries and keys of a step
or a prompt, alone or on the way into a paged cache; the low-rank adapters of many requests beside a
shared projection; and, behind the last layer, the log probabilities of given tokens with the
entropy and the top alternatives of every row. Sizes are those of this repository's 7B-class layers
(4096, 11008, 32 heads of 128) and generic ones around them. Inputs are synthetic, drawn on the GPU
from the seed: N(0, 1) activations with 0.1 % of the entries 20 times larger, adapter weights that
change a projection's output by a fraction of itself, logits of standard deviation 2.5 with a few
likely tokens in every row and, where a case masks, -infinity for the others' half.

Where ``own`` is false, ``run`` is plain torch in 32 bits (64 for the angles of far positions).
``exact`` is the definition in 64 bits.
"""
import math

import torch

own = False

_DT = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32, "f8": torch.float8_e4m3fn}
_FLOOR = 2.0 ** -100
_BASE = 10000.0


def listed():
    return [
        # one new token of one stream: the smallest call, latency counts
        dict(name="rotary_1token", op="rotary", tokens=1, heads=32, kv=8, dim=128, rot=128, layout="half", dtype="bf16",
             factor=1.0, inverse=False, far=4096),
        # a long prompt at far positions, frequencies scaled for a long context
        dict(name="rotary_8192tokens", op="rotary", tokens=8192, heads=32, kv=8, dim=128, rot=128, layout="half",
             dtype="bf16", factor=8.0, inverse=False, far=1000000),
        # neighbours turned in the first part of heads of 80, backwards (the gradient's direction)
        dict(name="rotary_part", op="rotary", tokens=777, heads=20, kv=20, dim=80, rot=32, layout="interleaved",
             dtype="fp16", factor=1.0, inverse=True, far=2048),
        # the new tokens of 64 streams turned and written to an 8-bit cache
        dict(name="rotary_append_f8", op="append", tokens=64, heads=32, kv=8, dim=128, rot=128, layout="half", dtype="bf16",
             cache="f8", order="head", page=64, pages=256, factor=4.0, far=32768),
        # a prompt of 2048 tokens turned and written to a 16-bit cache
        dict(name="rotary_append_2048", op="append", tokens=2048, heads=32, kv=32, dim=128, rot=128, layout="half",
             dtype="bf16", cache="same", order="slot", page=16, pages=512, factor=1.0, far=4096),
        # a single stream with its adapter beside a square projection
        dict(name="adapters_1row", op="adapters", rows=1, n=8, rank=16, mixed=False, d_in=4096, d_out=4096, dtype="bf16",
             out="bf16", none=0.0, spans=False),
        # a decode step of 32 streams, an adapter each of mixed ranks, beside an up projection
        dict(name="adapters_32rows", op="adapters", rows=32, n=64, rank=64, mixed=True, d_in=4096, d_out=11008, dtype="bf16",
             out="bf16", none=0.1, spans=False),
        # odd sizes: a ragged batch of streams, sums in 32 bits
        dict(name="adapters_odd", op="adapters", rows=117, n=9, rank=20, mixed=False, d_in=2305, d_out=4099, dtype="fp16",
             out="fp32", none=0.2, spans=False),
        # prompts of a few requests, one behind the other, through a square projection
        dict(name="adapters_8192rows", op="adapters", rows=8192, n=8, rank=32, mixed=False, d_in=4096, d_out=4096,
             dtype="bf16", out="bf16", none=0.1, spans=True),
        # the next token of one stream, with alternatives
        dict(name="log_probs_1row", op="log_probs", rows=1, vocab=32000, top=5, targets=1, dtype="bf16", scale=1.0,
             masked=False),
        # 16 streams over a large vocabulary, at a temperature, half of it ruled out by a grammar
        dict(name="log_probs_16rows", op="log_probs", rows=16, vocab=131072, top=20, targets=2, dtype="fp32", scale=1.25,
             masked=True),
        # the tokens of a text scored (odd vocabulary, unaligned rows), no alternatives
        dict(name="log_probs_text", op="log_probs", rows=2600, vocab=50001, top=0, targets=1, dtype="bf16", scale=1.0,
             masked=False),
    ]


_MOST = 260000000          # bytes of a drawn case


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["rotary", "rotary", "append", "append", "adapters", "adapters", "adapters", "log_probs", "log_probs",
                     "log_probs"])
    dtype = rng.choice(["bf16", "fp16"])
    if op in ("rotary", "append"):
        kv = rng.choice([1, 2, 4, 8, 8, 20, 32])
        heads = kv * rng.choice([1, 2, 4, 4, 7] if kv < 20 else [1, 1, 2])
        dim = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
        rot = rng.choice([dim, dim, dim, dim // 2, dim // 4, 2 * rng.randint(1, dim // 2)])
        layout, factor = rng.choice(["half", "half", "interleaved"]), rng.choice([1.0, 1.0, 4.0, 8.0, 32.0])
        far = _log(rng, 1, 1000000)
        most = _MOST // (4 * dim * (heads + 2 * kv))
        if op == "rotary":
            return dict(op=op, tokens=_log(rng, 1, min(8192, most)), heads=heads, kv=kv, dim=dim, rot=rot, layout=layout,
                        dtype=dtype, factor=factor, inverse=rng.random() < 0.25, far=far)
        page = rng.choice([8, 16, 16, 32, 64, 128, 20, 1])
        pages = max(2, min(1024, 32000000 // (kv * dim * page)))
        return dict(op=op, tokens=_log(rng, 1, min(4096, most, pages * page)), heads=heads, kv=kv, dim=dim, rot=rot,
                    layout=layout, dtype=dtype, cache=rng.choice(["same", "f8"]), order=rng.choice(["head", "slot"]),
                    page=page, pages=pages, factor=factor, far=far)
    if op == "adapters":
        d_in, d_out = (_log(rng, 256, 11008) for _ in range(2))
        if rng.random() < 0.7:
            d_in, d_out = d_in // 8 * 8, d_out // 8 * 8
        rank, n = rng.choice([4, 8, 16, 16, 20, 32, 64, 128]), _log(rng, 1, 64)
        n = max(1, min(n, 60000000 // (rank * (d_in + d_out))))
        out = rng.choice([dtype, dtype, dtype, "fp32"])
        rows = _log(rng, 1, min(8192, _MOST // (2 * d_in + (8 if out == "fp32" else 4) * d_out)))
        return dict(op=op, rows=rows, n=n, rank=rank, mixed=rng.random() < 0.4, d_in=d_in, d_out=d_out, dtype=dtype, out=out,
                    none=rng.choice([0.0, 0.1, 0.5]), spans=rows > 64 and rng.random() < 0.7)
    vocab, dtype = _log(rng, 1000, 200000), rng.choice(["bf16", "fp16", "fp32"])
    if rng.random() < 0.6:
        vocab = vocab // 8 * 8
    rows = _log(rng, 1, min(4096, _MOST // (vocab * (4 if dtype == "fp32" else 2))))
    return dict(op=op, rows=rows, vocab=vocab, top=rng.choice([0, 0, 1, 5, 10, 20, 32]), targets=rng.choice([1, 1, 1, 4]),
                dtype=dtype, scale=rng.choice([1.0, 1.0, 0.7, 1.25]), masked=rng.random() < 0.3)


# ---------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _acts(g, rows, cols, dt):
    x = _normal(g, rows, cols)
    big = torch.rand((rows, cols), generator=g, device="cuda") < 0.001
    return torch.where(big, 20.0 * x, x).to(dt)


def _int(g, hi, *shape):
    return torch.randint(0, hi, shape, generator=g, device="cuda")


def _frequencies(c):
    """Radians per position of every pair; a context `factor` times longer by a larger base."""
    base = _BASE * c["factor"] ** (c["rot"] / (c["rot"] - 2)) if c["factor"] != 1.0 and c["rot"] > 2 else _BASE
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
    return base ** (-2.0 * i / c["rot"])


def _rotary_inputs(g, c, dt):
    n, heads, kv, dim = c["tokens"], c["heads"], c["kv"], c["dim"]
    qkv = _acts(g, n, (heads + 2 * kv) * dim, dt).view(n, heads + 2 * kv, dim)      # one projection's rows
    start = _int(g, c["far"], 1)
    positions = start + torch.arange(n, device="cuda") if n > 64 else _int(g, c["far"], n)
    s = dict(q=qkv[:, :heads], k=qkv[:, heads:heads + kv], v=qkv[:, heads + kv:], positions=positions, freq=_frequencies(c))
    s["q_out"] = torch.empty((n, heads, dim), dtype=dt, device="cuda")
    s["k_out"] = torch.empty((n, kv, dim), dtype=dt, device="cuda")
    if own:
        import paper_2606_12876_amd as aq
        s["rotary"] = aq.Rotary(s["freq"], layout=c["layout"])
    return s


def _adapter_index(g, c):
    """The adapter of every row, -1 for none; `spans`: whole prompts, one behind the other."""
    rows, n = c["rows"], c["n"]
    if c["spans"]:
        parts = min(rows, 2 * n)
        which = torch.where(torch.rand((parts,), generator=g, device="cuda") < c["none"], -1, _int(g, n, parts))
        ends = torch.sort(_int(g, rows, parts - 1)).values if parts > 1 else torch.empty((0,), dtype=torch.int64, device="cuda")
        return which[torch.bucketize(torch.arange(rows, device="cuda"), ends, right=True)].to(torch.int32)
    index = torch.randperm(max(n, rows), generator=g, device="cuda")[:rows] % n
    return torch.where(torch.rand((rows,), generator=g, device="cuda") < c["none"], -1, index).to(torch.int32)


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    op, dt = c["op"], _DT[c["dtype"]]
    s = dict(c=c, op=op, dt=dt)
    if op in ("rotary", "append"):
        s.update(_rotary_inputs(g, c, dt))
    if op == "append":
        a, b = (c["kv"], c["page"]) if c["order"] == "head" else (c["page"], c["kv"])
        f8 = c["cache"] == "f8"
        for name in "kv":
            x = torch.randn((c["pages"], a, b, c["dim"]), generator=g, device="cuda", dtype=dt)
            s["c" + name] = (x * 100).clamp(-448.0, 448.0).to(_DT["f8"]) if f8 else x
            if f8:
                s["c" + name + "s"] = 0.01 * (0.5 + torch.rand((c["pages"], a, b), generator=g, device="cuda"))
        s["slots"] = torch.randperm(c["pages"] * c["page"], generator=g, device="cuda")[:c["tokens"]]
        if own:
            import paper_2606_12876_amd as aq
            s["cache"] = aq.KVCache(s["ck"], s["cv"], s.get("cks"), s.get("cvs"), layout=c["order"])
    if op == "adapters":
        n, r, rows = c["n"], c["rank"], c["rows"]
        s["a"] = (c["d_in"] ** -0.5 * torch.randn((n, r, c["d_in"]), generator=g, device="cuda")).to(dt)
        s["b"] = (0.3 * r ** -0.5 * torch.randn((n, c["d_out"], r), generator=g, device="cuda")).to(dt)
        s["scales"] = 0.5 + torch.rand((n,), generator=g, device="cuda")
        s["ranks"] = (1 + _int(g, r, n)).to(torch.int32) if c["mixed"] else None
        s["index"] = _adapter_index(g, c)
        s["x"] = _acts(g, rows, c["d_in"], dt)
        s["base"] = _normal(g, rows, c["d_out"]).to(_DT[c["out"]])
        s["y"] = torch.empty_like(s["base"])
        if own:
            import paper_2606_12876_amd as aq
            s["adapters"] = aq.Adapters(s["a"], s["b"], s["scales"], s["ranks"])
    if op == "log_probs":
        rows, vocab = c["rows"], c["vocab"]
        z = torch.randn((rows, vocab), generator=g, device="cuda", dtype=dt) * 2.5
        likely = _int(g, vocab, rows, 6)
        z.scatter_add_(1, likely, 8.0 * torch.rand((rows, 6), generator=g, device="cuda").to(dt))
        s["targets"] = _int(g, vocab, rows, c["targets"])
        if c["masked"]:
            out = torch.rand((rows, vocab), generator=g, device="cuda") < 0.5
            out.scatter_(1, s["targets"], False)
            z.masked_fill_(out, -math.inf)
        s["z"] = z
        s["lp"] = torch.empty((rows, c["targets"]), dtype=torch.float32, device="cuda")
        s["lse"], s["entropy"] = (torch.empty((rows,), dtype=torch.float32, device="cuda") for _ in range(2))
        s["ids"] = torch.empty((rows, c["top"]), dtype=torch.int64, device="cuda") if c["top"] else None
        s["tops"] = torch.empty((rows, c["top"]), dtype=torch.float32, device="cuda") if c["top"] else None
    return s


# ------------------------------------------------------------------------------ plain forms
def _angles(s, c):
    """(cos, sin) of every token and pair, [tokens][1][rot / 2]."""
    angle = (s["positions"].double()[:, None] * s["freq"])[:, None]
    sin = torch.sin(angle).float()
    return torch.cos(angle).float(), -sin if c.get("inverse") else sin


def _turn(x, cos, sin, c):
    x, rot = x.float(), c["rot"]
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., rot:]), -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned, x[..., rot:]), -1)


def _write(s, c, name, new):
    page, at = s["slots"] // c["page"], s["slots"] % c["page"]
    where = (page, slice(None), at) if c["order"] == "head" else (page, at)
    if c["cache"] != "f8":
        s["c" + name][where] = new.to(s["dt"])
        return
    x = new.float()
    a = x.abs().amax(-1).clamp_min(_FLOOR)
    s["c" + name].view(torch.uint8)[where] = (x * (448.0 / a)[..., None]).to(_DT["f8"]).view(torch.uint8)
    s["c" + name + "s"][where] = a / 448.0


def _cached(s):
    return {name: s[name] for name in ("ck", "cv", "cks", "cvs") if name in s}


def _adapt(s, c):
    """The adapters' part of every row in 32 bits: gathered for few rows, all adapters' products for many."""
    x, index = s["x"].float(), s["index"].long()
    rows, n, r = c["rows"], c["n"], c["rank"]
    at = index.clamp_min(0)
    factor = torch.where(index < 0, 0.0, s["scales"][at])[:, None]
    if s["ranks"] is not None:
        factor = factor * (torch.arange(r, device="cuda")[None, :] < s["ranks"][at][:, None])
    if rows <= 32:
        t = torch.matmul(s["a"][at].float(), x[..., None])[..., 0] * factor
        return torch.matmul(s["b"][at].float(), t[..., None])[..., 0]
    mine = torch.arange(n, device="cuda")[None, :, None] == index[:, None, None]
    t = torch.matmul(x, s["a"].float().view(n * r, -1).t()).view(rows, n, r)
    t = torch.where(mine, t * factor[:, None], 0.0)
    return torch.matmul(t.view(rows, n * r), s["b"].float().transpose(1, 2).reshape(n * r, -1))


def _order(z):
    """A whole number for every value, larger for a larger value, and among equals for a lower index."""
    bits = (z.float() + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    return bits * 2 ** 32 - torch.arange(z.shape[1], device="cuda")[None, :]


def _plain(s, c):
    op = s["op"]
    if op == "rotary":
        cos, sin = _angles(s, c)
        return {"q": _turn(s["q"], cos, sin, c).to(s["dt"]), "k": _turn(s["k"], cos, sin, c).to(s["dt"])}
    if op == "append":
        cos, sin = _angles(s, c)
        _write(s, c, "k", _turn(s["k"], cos, sin, c))
        _write(s, c, "v", s["v"])
        return dict(_cached(s), q=_turn(s["q"], cos, sin, c).to(s["dt"]))
    if op == "adapters":
        return {"y": (s["base"].float() + _adapt(s, c)).to(s["base"].dtype)}
    z = s["z"].float() * c["scale"]
    top = z.amax(1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(1, keepdim=True)
    lse = top + torch.log(total)
    entropy = torch.log(total) - torch.where(p > 0, p * (z - top), 0.0).sum(1, keepdim=True) / total
    got = {"logprobs": z.gather(1, s["targets"]) - lse, "lse": lse[:, 0], "entropy": entropy[:, 0]}
    if c["top"]:
        got["ids"] = torch.topk(_order(s["z"]), c["top"], dim=1).indices
        got["tops"] = z.gather(1, got["ids"]) - lse
    return got


# ---------------------------------------------------------------------- the framework's calls
def _framework(s, c):
    import paper_2606_12876_amd as aq
    op = s["op"]
    if op == "rotary":
        s["rotary"].apply(s["q"], s["positions"], s["q_out"], k=s["k"], k_out=s["k_out"], inverse=c["inverse"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "append":
        s["cache"].rotary_append(s["rotary"], s["q"], s["k"], s["v"], s["positions"], s["slots"], s["q_out"])
        return dict(_cached(s), q=s["q_out"])
    if op == "adapters":
        s["adapters"].add(s["x"], s["index"], s["base"], s["y"])
        return {"y": s["y"]}
    aq.log_probs(s["z"], s["targets"], s["lp"], lse=s["lse"], entropy=s["entropy"], top_ids=s["ids"], top_logprobs=s["tops"],
                 scale=c["scale"])
    got = {"logprobs": s["lp"], "lse": s["lse"], "entropy": s["entropy"]}
    if c["top"]:
        got.update(ids=s["ids"], tops=s["tops"])
    return got


def run(state):
    return (_framework if own else _plain)(state, state["c"])


# -------------------------------------------------------------------------------------- work
def work(case):
    c = case
    if c["op"] in ("rotary", "append"):
        n = c["tokens"]
        turned = n * (c["heads"] + c["kv"]) * c["rot"]
        if c["op"] == "rotary":
            return {"bytes": 4 * n * (c["heads"] + c["kv"]) * c["dim"] + 8 * n + 4 * c["rot"], "flops": 3 * turned}
        each = c["dim"] + 4 if c["cache"] == "f8" else 2 * c["dim"]
        return {"bytes": n * (4 * c["heads"] * c["dim"] + 2 * c["kv"] * (2 * c["dim"] + each) + 16) + 4 * c["rot"],
                "flops": 3 * turned + (4 * n * c["kv"] * c["dim"] if c["cache"] == "f8" else 0)}
    if c["op"] == "adapters":
        with_one = c["rows"] * (1.0 - c["none"])
        rank = (1 + c["rank"]) / 2 if c["mixed"] else c["rank"]
        parts = min(c["rows"], 2 * c["n"]) * (1.0 - c["none"]) if c["spans"] else with_one
        # spans draw their adapters; rows without spans take as many different ones as there are
        used = c["n"] * (1.0 - (1.0 - 1.0 / c["n"]) ** parts) if c["spans"] else min(c["n"], parts)
        size = 4 if c["out"] == "fp32" else 2
        return {"bytes": int(2 * used * rank * (c["d_in"] + c["d_out"]) + 2 * with_one * c["d_in"]
                             + 2 * size * c["rows"] * c["d_out"] + 4 * c["rows"]),
                "flops": int(2 * with_one * rank * (c["d_in"] + c["d_out"]))}
    size = 4 if c["dtype"] == "fp32" else 2
    return {"bytes": c["rows"] * (size * c["vocab"] + 12 * c["targets"] + 8 + 12 * c["top"]), "flops": 6 * c["rows"] * c["vocab"]}


# ------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The operators' definitions in 64 bits, a token, row or span at a time where that is shorter to say. A value held in
    8 bits is the one it is rounded from: the rounding itself jumps."""
    s = prepare(case, seed)
    c, op = s["c"], s["op"]
    d = torch.float64

    def turned(x):
        """Every pair as a complex number, times the unit number of its angle."""
        at = torch.outer(s["positions"].to(d), s["freq"])
        unit = torch.polar(torch.ones_like(at), -at if c.get("inverse") else at)[:, None, :]
        x = x.to(d).clone()
        half = c["rot"] // 2
        first, second = ((slice(0, half), slice(half, c["rot"])) if c["layout"] == "half"
                         else (slice(0, c["rot"], 2), slice(1, c["rot"], 2)))
        z = torch.complex(x[..., first].clone(), x[..., second].clone()) * unit
        x[..., first], x[..., second] = z.real, z.imag
        return x

    if op == "rotary":
        return {"q": turned(s["q"]), "k": turned(s["k"])}
    if op == "append":
        f8 = c["cache"] == "f8"
        got = {n: s[n].to(torch.float32).to(d) if f8 else s[n].to(d) for n in ("ck", "cv")}
        if f8:
            got.update(cks=s["cks"].to(d), cvs=s["cvs"].to(d))
        new = {"ck": turned(s["k"]), "cv": s["v"].to(d)}
        page, at = torch.div(s["slots"], c["page"], rounding_mode="floor"), s["slots"].remainder(c["page"])
        heads = torch.arange(c["kv"], device="cuda")[None, :]
        where = (page[:, None], heads, at[:, None]) if c["order"] == "head" else (page[:, None], at[:, None], heads)
        for n, x in new.items():
            if f8:
                a = x.abs().amax(-1).clamp_min(_FLOOR)
                got[n][where], got[n + "s"][where] = x / a[..., None] * 448.0, a / 448.0
            else:
                got[n][where] = x
        return dict(got, q=turned(s["q"]))
    if op == "adapters":
        y = s["base"].to(d)
        for i in range(c["n"]):
            rows = torch.nonzero(s["index"] == i)[:, 0]
            if rows.numel():
                r = c["rank"] if s["ranks"] is None else int(s["ranks"][i])
                t = s["x"][rows].to(d) @ s["a"][i, :r].to(d).t()
                y[rows] += (t @ s["b"][i, :, :r].to(d).t()) * s["scales"][i].to(d)
        return {"y": y}
    parts = []
    for z, t in zip(s["z"].split(256), s["targets"].split(256)):
        w = z.to(d) * c["scale"]
        lp = torch.log_softmax(w, 1)
        one = {"logprobs": lp.gather(1, t), "lse": torch.logsumexp(w, 1),
               "entropy": -torch.where(lp == -math.inf, 0.0, lp.exp() * lp).sum(1)}
        if c["top"]:
            one["ids"] = torch.sort(z.to(d), dim=1, descending=True, stable=True).indices[:, :c["top"]].contiguous()
            one["tops"] = lp.gather(1, one["ids"])
        parts.append(one)
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
