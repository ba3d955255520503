"""The operators of a decode step around the quantized linear layers, for timing.

Each case is one call (or the two calls that always go together) that a serving loop makes between
its linear layers: the root-mean-square norm with the residual's addition, 16-bit or 8-bit output;
the product with 4-bit weights of the layers that are not additively coded; attention of one new
token per sequence over a paged cache; and the cache's upkeep (writing new tokens, copying pages).
Sizes are those of this repository's 7B-class layers (4096, 11008, 32 heads of 128) and generic
ones around them. Inputs are synthetic, drawn on the GPU from the seed: N(0, 1) activations with
0.1 % of the entries 20 times larger, weights of standard deviation about 0.02, N(0, 1) keys and
values with NaN in every cache slot that no sequence holds (memory that is never cleared).

Where ``own`` is false, ``run`` is plain torch in 32 bits. ``exact`` is the definition in 64 bits.
"""
import math

import torch

own = False

_DT = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32, "f8": torch.float8_e4m3fn,
       "i8": torch.int8}
_TOP = {"f8": 448.0, "i8": 127.0}
_FLOOR = 2.0 ** -100


def listed():
    return [
        # one token of one stream between two layers: the smallest call, latency counts
        dict(name="norm_1row", op="norm", rows=1, cols=4096, dtype="bf16", out="same", group=0, residual=True, w0=0.0),
        # a long prompt's rows ahead of an 8-bit product, a scale for every 128 inputs
        dict(name="norm_q8_8192rows", op="norm", rows=8192, cols=4096, dtype="bf16", out="f8", group=128,
             residual=True, w0=0.0),
        # rows of an odd length (unaligned), no residual, weights stored as offsets from one
        dict(name="norm_odd", op="norm", rows=517, cols=2305, dtype="fp16", out="same", group=0, residual=False, w0=1.0),
        # single-stream decoding through a square 4-bit projection
        dict(name="w4_1row", op="w4", d_out=4096, d_in=4096, group=128, zeros=False, batch=1, x="fp16"),
        # batched decoding through an up projection with zero points, an odd number of streams
        dict(name="w4_up_11rows", op="w4", d_out=11008, d_in=4096, group=64, zeros=True, batch=11, x="bf16"),
        # norm to int8 with scales, then the 4-bit product that takes them: 16 streams, a down projection's sizes
        dict(name="norm_w4_int8", op="norm_w4", d_out=4096, d_in=11008, group=128, zeros=False, batch=16, x="bf16",
             q="i8", q_group=128),
        # attention of a single stream, one key-value head for every head
        dict(name="attn_1seq", op="attn", seqs=1, length=1000, heads=32, kv=32, dim=128, page=16, dtype="bf16",
             cache="same", layout="head", window=0),
        # a batch of ragged streams, four heads to a key-value head
        dict(name="attn_16seqs", op="attn", seqs=16, length=4096, heads=32, kv=8, dim=128, page=64, dtype="fp16",
             cache="same", layout="slot", window=0),
        # one very long context: few rows, so the length has to be split
        dict(name="attn_long", op="attn", seqs=1, length=131072, heads=32, kv=8, dim=128, page=256, dtype="bf16",
             cache="same", layout="head", window=0),
        # many ragged streams on an 8-bit cache
        dict(name="attn_f8_64seqs", op="attn", seqs=64, length=8192, heads=32, kv=8, dim=128, page=128, dtype="bf16",
             cache="f8", layout="head", window=0),
        # the new tokens of 16 streams written to an 8-bit cache
        dict(name="kv_append_f8", op="append", tokens=16, kv=8, dim=128, page=64, pages=256, dtype="bf16", cache="f8",
             layout="head"),
        # streams forked with their last pages copied, four layers' caches at once
        dict(name="kv_copy", op="copy", pairs=200, caches=4, kv=8, dim=128, page=64, pages=512, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "w4", "w4", "norm_w4", "attn", "attn", "attn", "append", "copy"])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "norm":
        cols = _log(rng, 64, 16384)
        if rng.random() < 0.6:
            cols = max(64, cols // 8 * 8)
        out = rng.choice(["same", "same", "f8", "fp32"])
        return dict(op="norm", rows=_log(rng, 1, min(16384, 33000000 // cols)), cols=cols, dtype=dtype, out=out,
                    group=rng.choice([0, 32, 64, 128]) if out == "f8" else 0, residual=rng.random() < 0.7,
                    w0=rng.choice([0.0, 0.0, 1.0]))
    if op in ("w4", "norm_w4"):
        group = rng.choice([32, 64, 128, 128])
        more = dict(q=rng.choice(["i8", "f8"]), q_group=rng.choice([0, group, group])) if op == "norm_w4" else {}
        return dict(op=op, d_out=_log(rng, 500, 14336), d_in=_log(rng, 500, 11008), group=group,
                    zeros=rng.random() < 0.5, batch=rng.choice([1, 1, 2, rng.randint(3, 16), rng.randint(3, 16)]), x=dtype,
                    **more)
    if op == "attn":
        kv = rng.choice([1, 2, 4, 8, 8, 32])
        heads = kv * rng.choice([1, 2, 4, 4, 7, 8, 16] if kv < 32 else [1, 2])
        dim = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
        seqs = _log(rng, 1, 64)
        length = _log(rng, 1, min(65536, 100000000 // (kv * dim * seqs)))
        return dict(op="attn", seqs=seqs, length=length, heads=heads, kv=kv, dim=dim,
                    page=rng.choice([8, 16, 16, 32, 48, 64, 128, 256, 1, 20]), dtype=dtype,
                    cache=rng.choice(["same", "same", "f8"]), layout=rng.choice(["head", "slot"]),
                    window=rng.choice([0, 0, 0, _log(rng, 1, 4096)]))
    kv, dim = rng.choice([1, 2, 8, 8, 32]), rng.choice([64, 80, 96, 128, 128, 256])
    page = rng.choice([8, 16, 32, 64, 128, 20])
    room = 32000000 // (kv * dim * page)
    if op == "append":
        pages = max(2, min(room, 1024))
        return dict(op="append", tokens=_log(rng, 1, min(4096, pages * page)), kv=kv, dim=dim, page=page, pages=pages,
                    dtype=dtype, cache=rng.choice(["same", "f8"]), layout=rng.choice(["head", "slot"]))
    caches = rng.randint(1, 8)
    pages = max(4, min(2 * room // caches, 1024))
    return dict(op="copy", pairs=_log(rng, 1, pages // 2), caches=caches, kv=kv, dim=dim, page=page, pages=pages,
                dtype=dtype)


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


def _norm_inputs(g, c, rows, cols, dt):
    x = _acts(g, rows, cols, dt)
    w = (1.0 - c.get("w0", 0.0) + 0.1 * _normal(g, cols)).to(dt)
    r = _acts(g, rows, cols, dt) if c.get("residual", True) else None
    return dict(x=x, w=w, r=r, eps=1e-5, w0=c.get("w0", 0.0))


def _w4_inputs(g, c):
    d_out, d_in, groups = c["d_out"], c["d_in"], -(-c["d_in"] // c["group"])
    weights = _int(g, 256, d_out, (d_in + 1) // 2).to(torch.uint8)
    scales = (0.004 * (0.5 + torch.rand((d_out, groups), generator=g, device="cuda"))).to(torch.float16)
    zeros = _int(g, 16, d_out, groups).to(torch.uint8) if c["zeros"] else None
    s = dict(weights=weights, scales=scales, zeros=zeros, d_in=d_in)
    if own:
        import paper_2606_12876_amd as aq
        s["layer"] = aq.W4Linear(weights, scales, zeros, d_in=d_in, group_size=c["group"])
    return s


def _page_shape(c):
    return (c["kv"], c["page"]) if c.get("layout", "head") == "head" else (c["page"], c["kv"])


def _cache(c, k, v, ks=None, vs=None):
    import paper_2606_12876_amd as aq
    return aq.KVCache(k, v, ks, vs, layout=c.get("layout", "head"))


def _stored(g, c, n_pages):
    """A full cache of n_pages pages: keys, values and, for 8 bits, a scale for every token and head."""
    a, b = _page_shape(c)
    dt, f8 = _DT[c["dtype"]], c.get("cache") == "f8"
    made = {}
    for name in "kv":
        x = torch.randn((n_pages, a, b, c["dim"]), generator=g, device="cuda", dtype=dt)
        if f8:
            made[name] = (x * 100).clamp(-448.0, 448.0).to(_DT["f8"])
            made[name + "s"] = 0.01 * (0.5 + torch.rand((n_pages, a, b), generator=g, device="cuda"))
        else:
            made[name] = x
    return made


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    op, dt = c["op"], _DT[c.get("dtype", c.get("x"))]
    s = dict(c=c, op=op, dt=dt)
    if op == "norm":
        rows, cols = c["rows"], c["cols"]
        s.update(_norm_inputs(g, c, rows, cols, dt))
        out = dt if c["out"] == "same" else _DT[c["out"]]
        s["y"] = torch.empty((rows, cols), dtype=out, device="cuda")
        s["r2"] = torch.empty_like(s["x"]) if c["residual"] else None
        s["ys"] = (torch.empty((rows, -(-cols // (c["group"] or cols))), dtype=torch.float32, device="cuda")
                   if c["out"] == "f8" else None)
    elif op in ("w4", "norm_w4"):
        s.update(_w4_inputs(g, c))
        s["y"] = torch.empty((c["batch"], c["d_out"]), dtype=dt, device="cuda")
        if op == "w4":
            s["x"] = _acts(g, c["batch"], c["d_in"], dt)
        else:
            s.update(_norm_inputs(g, c, c["batch"], c["d_in"], dt))
            s["r2"] = torch.empty_like(s["x"])
            s["xq"] = torch.empty((c["batch"], c["d_in"]), dtype=_DT[c["q"]], device="cuda")
            s["xs"] = torch.empty((c["batch"], -(-c["d_in"] // (c["q_group"] or c["d_in"]))), dtype=torch.float32, device="cuda")
    elif op == "attn":
        n, page = c["seqs"], c["page"]
        lens = _int(g, c["length"] + 1, n)
        lens[0] = c["length"]                      # one stream of full length; others from zero up
        per = -(-c["length"] // page)
        used = -(-lens // page)
        n_pages = int(used.sum()) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda")
        inside = torch.arange(per, device="cuda")[None, :] < used[:, None]
        table = torch.full((n, per), -1, dtype=torch.int32, device="cuda")
        table[inside] = order[:int(used.sum())].to(torch.int32)
        made = _stored(g, c, n_pages)
        # slots that no sequence holds: never written, NaN in places
        held = torch.zeros((n_pages, page), dtype=torch.bool, device="cuda")
        at = torch.arange(per * page, device="cuda")[None, :] < lens[:, None]
        held[table[inside].long()] = at.view(n, per, page)[inside]
        free = ~(held[:, None, :] if c["layout"] == "head" else held[:, :, None])
        for name in "kv":
            if c["cache"] == "f8":
                made[name + "s"].masked_fill_(free, math.nan)
            else:
                made[name].masked_fill_(free[..., None], math.nan)
        s.update(made)
        s.update(q=(2.0 * _normal(g, n, c["heads"], c["dim"])).to(dt), table=table, lens=lens.to(torch.int32),
                 scale=c["dim"] ** -0.5)
        s["y"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((n, c["heads"]), dtype=torch.float32, device="cuda")
    elif op == "append":
        s.update(_stored(g, c, c["pages"]))
        s["new_k"] = _acts(g, c["tokens"], c["kv"] * c["dim"], dt).view(c["tokens"], c["kv"], c["dim"])
        s["new_v"] = _acts(g, c["tokens"], c["kv"] * c["dim"], dt).view(c["tokens"], c["kv"], c["dim"])
        s["slots"] = torch.randperm(c["pages"] * c["page"], generator=g, device="cuda")[:c["tokens"]]
    else:
        for name in "kv":
            s[name] = torch.randn((c["caches"], c["pages"], c["kv"], c["page"], c["dim"]), generator=g, device="cuda",
                                  dtype=dt)
        order = torch.randperm(c["pages"], generator=g, device="cuda")
        s["dst"] = order[:c["pairs"]].to(torch.int32)
        s["src"] = order[c["pairs"]:][_int(g, c["pages"] - c["pairs"], c["pairs"])].to(torch.int32)
    if own and op in ("attn", "append"):
        s["cache"] = _cache(c, s["k"], s["v"], s.get("ks"), s.get("vs"))
    if own and op == "copy":
        s["caches"] = [_cache(c, s["k"][i], s["v"][i]) for i in range(c["caches"])]
    return s


# ------------------------------------------------------------------------------ plain forms
def _norm_plain(s):
    h = s["x"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    return h, h * torch.rsqrt((h * h).mean(-1, keepdim=True) + s["eps"]) * (s["w"].float() + s["w0"])


def _grouped(y, group):
    """y [rows][cols] as [rows][groups][group], zeros after the end."""
    rows, cols = y.shape
    group = group or cols
    n = -(-cols // group)
    return torch.nn.functional.pad(y, (0, n * group - cols)).view(rows, n, group)


def _quantized(y, group, top):
    """(values on the 8-bit grid before rounding [rows][cols], scales [rows][groups])."""
    yg = _grouped(y, group)
    a = yg.abs().amax(-1).clamp_min(_FLOOR)
    return (yg * (top / a)[..., None]).view(y.shape[0], -1)[:, :y.shape[1]], a / top


def _nibbles(s):
    w = s["weights"]
    return torch.stack((w & 15, w >> 4), -1).view(w.shape[0], -1)[:, :s["d_in"]]


def _dequantized(s, group):
    per = torch.arange(s["d_in"], device="cuda") // group
    z = s["zeros"].float()[:, per] if s["zeros"] is not None else 8.0
    return (_nibbles(s).float() - z) * s["scales"].float()[:, per]


def _gathered(s, c, name):
    """Keys or values of every sequence in order, [seqs][kv][positions][dim] in 32 bits, zeros past the end."""
    n, per = s["table"].shape
    idx = s["table"].clamp_min(0).long().view(-1)
    x = s[name].view(torch.uint8)[idx].view(_DT["f8"]).float() if c["cache"] == "f8" else s[name][idx].float()
    if c["cache"] == "f8":
        x = x * s[name + "s"][idx][..., None]
    if c["layout"] == "head":
        x = x.view(n, per, c["kv"], c["page"], c["dim"]).transpose(1, 2)
    else:
        x = x.view(n, per * c["page"], c["kv"], c["dim"]).transpose(1, 2)
    x = x.reshape(n, c["kv"], per * c["page"], c["dim"])
    return x.masked_fill(~s["seen"][:, None, :, None], 0.0)


def _attend_plain(s, c):
    n, per = s["table"].shape
    at = torch.arange(per * c["page"], device="cuda")[None, :]
    seen = at < s["lens"][:, None]
    if c["window"]:
        seen = seen & (at >= s["lens"][:, None] - c["window"])
    s = dict(s, seen=seen)
    k, v = _gathered(s, c, "k"), _gathered(s, c, "v")
    q = s["q"].float().view(n, c["kv"], c["heads"] // c["kv"], c["dim"])
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    scores = scores.masked_fill(~seen[:, None, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    lse = top + torch.log(total)
    return o.view(n, c["heads"], c["dim"]).to(s["dt"]), lse.view(n, c["heads"])


def _write_plain(s, c, name, new):
    page, at = s["slots"] // c["page"], s["slots"] % c["page"]
    where = (page, slice(None), at) if c["layout"] == "head" else (page, at)
    if c["cache"] != "f8":
        s[name][where] = new
        return
    x = new.float()
    a = x.abs().amax(-1).clamp_min(_FLOOR)
    s[name].view(torch.uint8)[where] = (x * (448.0 / a)[..., None]).to(_DT["f8"]).view(torch.uint8)
    s[name + "s"][where] = a / 448.0


def _plain(s, c):
    op = s["op"]
    if op == "norm":
        h, y = _norm_plain(s)
        got = {}
        if c["out"] == "f8":
            y, got["scales"] = _quantized(y, c["group"], 448.0)
        got["y"] = y.to(s["y"].dtype)
        if c["residual"]:
            got["residual"] = h.to(s["dt"])
        return got
    if op == "w4":
        return {"y": torch.matmul(s["x"].float(), _dequantized(s, c["group"]).t()).to(s["dt"])}
    if op == "norm_w4":
        h, y = _norm_plain(s)
        q, xs = _quantized(y, c["q_group"], _TOP[c["q"]])
        per = torch.arange(c["d_in"], device="cuda") // (c["q_group"] or c["d_in"])
        q = q.round().clamp(-127.0, 127.0) if c["q"] == "i8" else q.to(_DT["f8"]).float()
        x = q * xs[:, per]
        return {"residual": h.to(s["dt"]), "scales": xs,
                "y": torch.matmul(x, _dequantized(s, c["group"]).t()).to(s["dt"])}
    if op == "attn":
        o, lse = _attend_plain(s, c)
        return {"o": o, "lse": lse}
    if op == "append":
        _write_plain(s, c, "k", s["new_k"])
        _write_plain(s, c, "v", s["new_v"])
        return {name: s[name] for name in ("k", "v", "ks", "vs") if name in s}
    src, dst = s["src"].long(), s["dst"].long()
    s["k"][:, dst] = s["k"][:, src]
    s["v"][:, dst] = s["v"][:, src]
    return {"k": s["k"], "v": s["v"]}


# ---------------------------------------------------------------------- the framework's calls
def _framework(s, c):
    import paper_2606_12876_amd as aq
    op = s["op"]
    if op == "norm":
        aq.rms_norm(s["x"], s["w"], s["y"], eps=s["eps"], weight_offset=s["w0"], residual=s["r"], residual_out=s["r2"],
                    scales=s["ys"], scale_group=c["group"])
        got = {"y": s["y"]}
        if s["ys"] is not None:
            got["scales"] = s["ys"]
        if c["residual"]:
            got["residual"] = s["r2"]
        return got
    if op == "w4":
        s["layer"].gemv(s["x"], s["y"])
        return {"y": s["y"]}
    if op == "norm_w4":
        aq.rms_norm(s["x"], s["w"], s["xq"], eps=s["eps"], residual=s["r"], residual_out=s["r2"], scales=s["xs"],
                    scale_group=c["q_group"])
        s["layer"].gemv(s["xq"], s["y"], x_scales=s["xs"])
        return {"residual": s["r2"], "scales": s["xs"], "y": s["y"]}
    if op == "attn":
        s["cache"].attention(s["q"], s["table"], s["lens"], s["y"], max_length=c["length"], scale=s["scale"],
                             window=c["window"], lse=s["lse"])
        return {"o": s["y"], "lse": s["lse"]}
    if op == "append":
        s["cache"].append(s["new_k"], s["new_v"], s["slots"])
        return {name: s[name] for name in ("k", "v", "ks", "vs") if name in s}
    aq.kv_copy_pages(s["caches"], s["src"], s["dst"])
    return {"k": s["k"], "v": s["v"]}


def run(state):
    return (_framework if own else _plain)(state, state["c"])


# -------------------------------------------------------------------------------------- work
def work(case):
    c = case
    if c["op"] == "norm":
        n, groups = c["rows"] * c["cols"], -(-c["cols"] // (c["group"] or c["cols"]))
        out = {"same": 2, "f8": 1, "fp32": 4}[c["out"]]
        return {"bytes": n * (2 + out + (4 if c["residual"] else 0)) + 2 * c["cols"]
                + (4 * c["rows"] * groups if c["out"] == "f8" else 0), "flops": 5 * n}
    if c["op"] in ("w4", "norm_w4"):
        groups = -(-c["d_in"] // c["group"])
        w = c["d_out"] * ((c["d_in"] + 1) // 2 + groups * (3 if c["zeros"] else 2))
        x = c["batch"] * c["d_in"]
        more = 6 * x + 2 * c["d_in"] + 4 * c["batch"] * -(-c["d_in"] // (c["q_group"] or c["d_in"])) if c["op"] == "norm_w4" else 2 * x
        return {"bytes": w + more + 2 * c["batch"] * c["d_out"], "flops": 2 * c["batch"] * c["d_out"] * c["d_in"]}
    if c["op"] == "attn":
        # lengths are uniform over 0..length except the first, which is the length
        seen = [c["length"]] + [c["length"] / 2] * (c["seqs"] - 1)
        tokens = sum(min(t, c["window"]) if c["window"] else t for t in seen)
        each = c["dim"] + 4 if c["cache"] == "f8" else 2 * c["dim"]
        return {"bytes": 2 * tokens * c["kv"] * each + 4 * c["seqs"] * c["heads"] * (c["dim"] + 1),
                "flops": 4 * tokens * c["heads"] * c["dim"]}
    if c["op"] == "append":
        n = 2 * c["tokens"] * c["kv"]
        return {"bytes": n * (2 * c["dim"] + (c["dim"] + 4 if c["cache"] == "f8" else 2 * c["dim"])),
                "flops": 3 * n * c["dim"] if c["cache"] == "f8" else 0}
    # a page that is the source of several copies is read once
    others = c["pages"] - c["pairs"]
    sources = others * (1.0 - (1.0 - 1.0 / others) ** c["pairs"])
    return {"bytes": 2 * c["caches"] * (c["pairs"] + sources) * c["kv"] * c["page"] * c["dim"] * 2, "flops": 0}


# ------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The operators' definitions in 64 bits, a row, sequence, token or page at a time where that is shorter to say.
    A value held in 8 bits is the one it is rounded from: the rounding itself jumps."""
    s = prepare(case, seed)
    c, op = s["c"], s["op"]
    d = torch.float64

    def normed():
        h = s["x"].to(d) if s["r"] is None else s["x"].to(d) + s["r"].to(d)
        rms = torch.sqrt(torch.linalg.vector_norm(h, dim=1) ** 2 / h.shape[1] + s["eps"])
        return h, (h / rms[:, None]) * (s["w"].to(d) + s["w0"])

    def on_grid(y, group, top):
        parts = torch.split(y, group or y.shape[1], dim=1)
        largest = torch.stack([p.abs().amax(1).clamp_min(_FLOOR) for p in parts], 1)
        return torch.cat([p / largest[:, i:i + 1] * top for i, p in enumerate(parts)], 1), largest / top

    def product(x):
        total = torch.zeros((x.shape[0], c["d_out"]), dtype=d, device="cuda")
        codes = _nibbles(s)
        for i, a in enumerate(range(0, c["d_in"], c["group"])):
            xs, q = x[:, a:a + c["group"]], codes[:, a:a + c["group"]].to(d)
            z = 8.0 if s["zeros"] is None else s["zeros"][:, i].to(d)
            total += (xs @ q.t() - z * xs.sum(1, keepdim=True)) * s["scales"][:, i].to(d)
        return total

    if op == "norm":
        h, y = normed()
        got = {}
        if c["out"] == "f8":
            y, got["scales"] = on_grid(y, c["group"], 448.0)
        got["y"] = y
        if c["residual"]:
            got["residual"] = h
        return got
    if op == "w4":
        return {"y": product(s["x"].to(d))}
    if op == "norm_w4":
        h, y = normed()
        q, xs = on_grid(y, c["q_group"], _TOP[c["q"]])
        q = q.round() if c["q"] == "i8" else q.to(_DT["f8"]).to(d)
        x = q * xs.repeat_interleave(c["q_group"] or c["d_in"], 1)[:, :c["d_in"]]
        return {"residual": h, "scales": xs, "y": product(x)}
    if op == "attn":
        o = torch.zeros((c["seqs"], c["heads"], c["dim"]), dtype=d, device="cuda")
        lse = torch.full((c["seqs"], c["heads"]), -math.inf, dtype=d, device="cuda")
        for i, length in enumerate(s["lens"].tolist()):
            lo = max(0, length - c["window"]) if c["window"] else 0
            if length == 0:
                continue
            pos = torch.arange(lo, length, device="cuda")
            page, at = s["table"][i, pos // c["page"]].long(), pos % c["page"]
            where = (page, slice(None), at) if c["layout"] == "head" else (page, at)
            if c["cache"] == "f8":
                k, v = (s[n].view(torch.uint8)[where].view(_DT["f8"]).to(d) * s[n + "s"][where].to(d)[..., None]
                        for n in "kv")
            else:
                k, v = s["k"][where].to(d), s["v"][where].to(d)
            for j in range(c["kv"]):
                a, b = j * (c["heads"] // c["kv"]), (j + 1) * (c["heads"] // c["kv"])
                score = s["q"][i, a:b].to(d) @ k[:, j].t() * s["scale"]
                lse[i, a:b] = torch.logsumexp(score, 1)
                o[i, a:b] = torch.softmax(score, 1) @ v[:, j]
        return {"o": o, "lse": lse}
    if op == "append":
        f8 = c["cache"] == "f8"
        got = {n: s[n].to(torch.float32).to(d) if f8 else s[n].to(d) for n in ("k", "v")}
        if f8:
            got.update(ks=s["ks"].to(d), vs=s["vs"].to(d))
        for i, slot in enumerate(s["slots"].tolist()):
            page, at = divmod(slot, c["page"])
            where = (page, slice(None), at) if c["layout"] == "head" else (page, at)
            for n in "kv":
                x = s["new_" + n][i].to(d)
                if f8:
                    a = x.abs().amax(-1).clamp_min(_FLOOR)
                    got[n][where], got[n + "s"][where] = x / a[:, None] * 448.0, a / 448.0
                else:
                    got[n][where] = x
        return got
    k, v = s["k"].clone(), s["v"].clone()
    for i, j in zip(s["src"].tolist(), s["dst"].tolist()):
        k[:, j].copy_(s["k"][:, i])
        v[:, j].copy_(s["v"][:, i])
    return {"k": k, "v": v}
