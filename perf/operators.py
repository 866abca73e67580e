"""What the window, decode, norm and 4-bit operators are timed on: the calls a serving program makes of them, and
the same results from elementary torch operations.

A case describes a batch by plain numbers.  `q_heads`, `kv_heads`, `dim` (head_dim), `page` and `pairing` (0: half-split
rotary pairs, 1: interleaved) are the model's; `batch` requests have lengths between `least` and `most`, drawn from `layout`,
which also draws which positions are queries: lengths and positions belong to the case, page numbers and tensor contents
come from the seed given to prepare().  `op` names the call of one pass:
  prefill   partial_prefill_attn of a plan with a window: each of `rows` scattered positions a request sees the first `sinks`
            tokens and the last `window` up to itself
  write     extend_write_norm: whole fresh prompts; q and k normalised per head, rotated, k and v written to their pages
  step      Decode.write: the same for the one new token of every request
  decode    Decode.attn: one query token a request over its 16-bit pages (`window` 0: all of them)
  decode4   Decode.attn_kv4: the same over 4-bit pages
  tier4     kv_retain_kv4, then kv_compose_from_kv4: cached units go to the 4-bit store and come back into prompts at other
            positions, keys rotated by what they moved

A 4-bit pool is [pages][kv_heads][page * (dim / 2 + 8)] bytes: of a page and KV head first the codes of all tokens, dim / 2
bytes each (byte i: element i in the low, element i + dim / 2 in the high four bits), then for every token four bf16 numbers,
scale and least value of the first half of the head and of the second.  A code c stands for scale * c + least.
"""
import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda"
THETA, EPS = 500000.0, 1e-6

SHAPE_8B = dict(q_heads=32, kv_heads=8, dim=128, page=64, pairing=0)
SHAPE_70B = dict(q_heads=64, kv_heads=8, dim=128, page=64, pairing=0)
SHAPE_GROUP5 = dict(q_heads=40, kv_heads=8, dim=128, page=16, pairing=0)
SHAPE_TINY = dict(q_heads=4, kv_heads=2, dim=64, page=16, pairing=0)


def listed():
    return [
        # the smallest prefill: one short prompt on a small model, window shorter than it
        dict(name="prefill-tiny", op="prefill", **SHAPE_TINY, batch=1, least=304, most=304, rows=64, window=96, sinks=4, layout=1),
        # questions over retrieved passages, recomputed tokens scattered over all of them
        dict(name="prefill-rag", op="prefill", **SHAPE_8B, batch=8, least=2100, most=5312, rows=352, window=1024, sinks=16, layout=2),
        # prompts of 33 thousand tokens
        dict(name="prefill-long", op="prefill", **SHAPE_8B, batch=2, least=32001, most=33024, rows=1152, window=4096, sinks=64, layout=3),
        # a decode step's keys and queries of eight conversations: all latency
        dict(name="write-step", op="step", **SHAPE_8B, batch=8, least=100, most=33024, layout=4),
        # whole prompts of a 70B model
        dict(name="write-prompts", op="write", **SHAPE_70B, batch=5, least=2048, most=16384, layout=5),
        # one conversation's next token
        dict(name="decode-one", op="decode", **SHAPE_8B, batch=1, least=5312, most=5312, window=0, sinks=0, layout=6),
        # a full batch of ragged conversations
        dict(name="decode-many", op="decode", **SHAPE_8B, batch=64, least=200, most=16384, window=0, sinks=0, layout=7),
        # long conversations through a window, groups of five heads, 16-token pages
        dict(name="decode-window", op="decode", **SHAPE_GROUP5, batch=48, least=1000, most=33024, window=4096, sinks=64, layout=8),
        # one conversation's next token, over 4-bit pages
        dict(name="decode4-one", op="decode4", **SHAPE_8B, batch=1, least=5312, most=5312, window=0, sinks=0, layout=9),
        # a full batch over 4-bit pages
        dict(name="decode4-many", op="decode4", **SHAPE_8B, batch=64, least=200, most=16384, window=0, sinks=0, layout=10),
        # a few snippets into the 4-bit store and back, small model
        dict(name="tier4-tiny", op="tier4", **SHAPE_TINY, batch=4, least=37, most=64, layout=11),
        # a batch's passages into the 4-bit store and back
        dict(name="tier4-many", op="tier4", **SHAPE_8B, batch=128, least=128, most=1024, layout=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prefill", "write", "step", "decode", "decode", "decode4", "decode4", "tier4"])
    dim, kv_heads = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 5, 7, 8, 16]) if op != "prefill" else rng.choice([1, 2, 4, 5, 7, 8])
    c = dict(op=op, q_heads=group * kv_heads, kv_heads=kv_heads, dim=dim, page=rng.choice([8, 16, 32, 64, 128]),
             pairing=rng.choice([0, 0, 1]), layout=rng.randrange(1 << 30))
    if op == "prefill":
        batch, most = _log(rng, 1, 8), _log(rng, 16, 33024)
        rows = min(most // 2, _log(rng, 1, 1152))
        while batch * rows * most * c["q_heads"] > 2 * 1152 * 33024 * 32:       # the largest listed one's scores
            batch, rows = max(1, batch // 2), max(1, rows // 2) if batch == 1 else rows
        return dict(c, batch=batch, least=max(rows, most // 2, 1), most=most, rows=max(1, rows), window=_log(rng, 1, 8192), sinks=rng.choice([0, 1, 4, 64, 200]))
    if op == "step":
        return dict(c, batch=_log(rng, 1, 256), least=1, most=_log(rng, 8, 33024))
    if op == "write":
        return dict(c, batch=_log(rng, 1, 8), least=1, most=_log(rng, 8, 5000))
    if op == "tier4":
        return dict(c, batch=_log(rng, 1, 128), least=1, most=_log(rng, 8, 1024))
    batch, most = _log(rng, 1, 64), _log(rng, 8, 33024)
    while batch * most * kv_heads > 64 * 16384 * 8 or batch * most * c["q_heads"] > 64 * 16384 * 32:
        most = max(1, most // 2)
    window = rng.choice([0, 0, _log(rng, 1, 8192)])
    return dict(c, batch=batch, least=1, most=most, window=window, sinks=rng.choice([0, 4, 64]) if window else 0)


# ---- what belongs to the case: lengths, positions of queries

def _lengths(c):
    r = random.Random(c["layout"])
    lens = [r.randint(c["least"], c["most"]) for _ in range(c["batch"])]
    lens[0] = c["most"]
    return np.array(lens, np.int64)


def _positions(c, lens):
    """[batch][rows] ascending positions, the last token always among them."""
    r = np.random.default_rng(c["layout"] + 1)
    return np.stack([np.sort(np.append(r.choice(int(t) - 1, c["rows"] - 1, replace=False), t - 1)) for t in lens]).astype(np.int64)


def _visible(c, pos):
    """Keys a query at position pos sees."""
    if not c.get("window"):
        return pos + 1
    return np.minimum(pos + 1, c["window"]) + np.minimum(np.maximum(pos + 1 - c["window"], 0), c["sinks"])


def work(c):
    lens = _lengths(c)
    hq, h, d = c["q_heads"], c["kv_heads"], c["dim"]
    if c["op"] == "prefill":
        pos, keys = _positions(c, lens), 0
        for t, p in zip(lens, pos):             # keys that some query of the request sees
            seen = np.zeros(int(t) + 1, np.int64)
            np.add.at(seen, np.maximum(p + 1 - c["window"], 0), 1)
            np.add.at(seen, p + 1, -1)
            hit = np.cumsum(seen)[:-1] > 0
            hit[: min(c["sinks"], int(p[-1]) + 1)] = True
            keys += int(hit.sum())
        pairs = int(_visible(c, pos).sum())
        return {"bytes": keys * h * d * 4 + pos.size * hq * (d * 4 + 4), "flops": 4 * d * hq * pairs}
    if c["op"] in ("write", "step"):
        n = int(lens.sum()) if c["op"] == "write" else c["batch"]
        return {"bytes": n * (hq + 2 * h) * d * 4, "flops": n * (hq + h) * d * 8}
    if c["op"] in ("decode", "decode4"):
        keys = int(_visible(c, lens - 1).sum())
        row = d * 4 if c["op"] == "decode" else d + 16
        return {"bytes": keys * h * row + c["batch"] * hq * (d * 4 + 4), "flops": 4 * d * hq * keys}
    n = int(lens.sum())
    return {"bytes": n * h * 2 * (2 * d + 2 * (d // 2 + 8) + 2 * d), "flops": n * h * d * 10}


# ---- inputs

def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, *dims):
    return torch.randn(*dims, generator=g, device=DEVICE, dtype=torch.bfloat16)


def _tables(c, lens, g, spare=3):
    """Pages in a random order: (pool pages, [batch][widest] page ids, 0 past a request's last page)."""
    per = -(-lens // c["page"])
    total = int(per.sum()) + spare
    perm = torch.randperm(total, generator=g, device=DEVICE, dtype=torch.int32)
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(per)[:-1]])).to(DEVICE)
    col = torch.arange(int(per.max()), device=DEVICE)
    at = off[:, None] + col
    there = col < torch.from_numpy(per).to(DEVICE)[:, None]
    return total, torch.where(there, perm[torch.where(there, at, 0)], 0).to(torch.int32).contiguous()


def _store4(x):
    """[pages][page][heads][dim] -> the 4-bit pool that stands for it."""
    pages, page, h, d = x.shape
    rec = torch.empty(pages, h, page * (d // 2 + 8), dtype=torch.uint8, device=x.device)
    for p0 in range(0, pages, 2048):
        y = x[p0:p0 + 2048].float().permute(0, 2, 1, 3).reshape(-1, h, page, 2, d // 2)
        scale, least, code = _codes(y)
        rec[p0:p0 + 2048, :, : page * (d // 2)] = (code[..., 0, :] + 16 * code[..., 1, :]).to(torch.uint8).reshape(-1, h, page * (d // 2))
        four = torch.stack([scale[..., 0, 0], least[..., 0, 0], scale[..., 1, 0], least[..., 1, 0]], -1).to(torch.bfloat16)
        rec[p0:p0 + 2048, :, page * (d // 2):] = four.view(torch.uint8).reshape(-1, h, page * 8)
    return rec


def _codes(y):
    """The last axis in 32 bits -> scale, least value (both bf16 numbers) and codes 0..15."""
    least, top = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    scale = ((top - least) / torch.full_like(top, 15.0)).to(torch.bfloat16).float()
    code = torch.where(scale > 0, (y - least) / torch.where(scale > 0, scale, 1.0), 0.0).round().clamp(0, 15)
    return scale, least, code


def _model(c):
    from paper_2609_32999_b200 import workloads as wl
    return wl.ModelShape(c["q_heads"], c["kv_heads"], c["dim"], c["page"], THETA, rope_pairing=c["pairing"])


def _i32(x):
    return np.ascontiguousarray(np.asarray(x), dtype=np.int32)


def _plan(c, lens, units, pages, pool_pages, recompute=None, sources=0, cached_pos=None, targets=None, **more):
    """A plan whose request r is one unit (units: its source pages, None: not cached), `pages` its destination pages."""
    from paper_2609_32999_b200 import binding as tb
    from paper_2609_32999_b200 import workloads as wl
    n = len(lens)
    per = -(-lens // c["page"])
    cached = units is not None
    rec = recompute if recompute is not None else [np.arange(0 if cached else t) for t in lens]
    w = wl.Workload("case", _model(c), _i32(lens), _i32(np.arange(n + 1)), _i32(lens), _i32(np.zeros(n) if cached_pos is None else cached_pos),
                    _i32(np.ones(n)), _i32(np.zeros(n)), _i32(np.concatenate([[0], np.cumsum(per)]) if cached else np.zeros(n + 1)),
                    _i32(units if cached else []), _i32(np.concatenate([[0], np.cumsum([len(x) for x in rec])])),
                    _i32(np.concatenate(rec)), _i32(pages), pool_pages, num_source_pages=sources)
    return tb.Plan(w, **more)


def prepare(case, seed):
    c, g, lens = case, _gen(seed), _lengths(case)
    hq, h, d, page = c["q_heads"], c["kv_heads"], c["dim"], c["page"]
    s = {"case": c, "lens": lens}
    per = -(-lens // page)
    if c["op"] == "tier4":
        return _prepare_tier(c, s, g, lens, per)
    total, s["table"] = _tables(c, lens, g)
    s["pages"] = total
    flat = np.concatenate([t[:n] for t, n in zip(s["table"].cpu().numpy(), per)])
    s["lens_dev"] = torch.from_numpy(lens).to(DEVICE, torch.int32)
    if c["op"] == "prefill":
        pos = _positions(c, lens)
        n = pos.size
        s["pos"] = torch.from_numpy(pos).to(DEVICE)
        s["k"], s["v"], s["q"] = _normal(g, total, page, h, d), _normal(g, total, page, h, d), _normal(g, n, hq, d)
        s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(n, hq, device=DEVICE)
        if own:
            s["plan"] = _plan(c, lens, np.arange(per.sum()), flat, total, list(pos), int(per.sum()), window=c["window"], n_sink=c["sinks"])
        return s
    if c["op"] in ("write", "step"):
        n = int(lens.sum()) if c["op"] == "write" else c["batch"]
        s["k"], s["v"] = torch.zeros(total, page, h, d, dtype=torch.bfloat16, device=DEVICE), torch.zeros(total, page, h, d, dtype=torch.bfloat16, device=DEVICE)
        # projections have a size of their own in every head, which is what the norms take away
        s["q"], s["k_new"], s["v_new"] = 3 * _normal(g, n, hq, d), 0.5 * _normal(g, n, h, d), _normal(g, n, h, d)
        s["q_weight"], s["k_weight"] = (1 + 0.25 * _normal(g, d)), (1 + 0.25 * _normal(g, d))
        s["q_out"] = torch.zeros_like(s["q"])
        p = np.concatenate([np.arange(t) for t in lens]) if c["op"] == "write" else lens - 1
        r = np.repeat(np.arange(c["batch"]), lens if c["op"] == "write" else 1)
        s["pos"] = torch.from_numpy(p).to(DEVICE)
        s["slot"] = s["table"][torch.from_numpy(r).to(DEVICE), s["pos"] // page].long() * page + s["pos"] % page
        if own and c["op"] == "write":
            s["plan"] = _plan(c, lens, None, flat, total)
    else:
        s["q"] = _normal(g, c["batch"], hq, d)
        s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(c["batch"], hq, device=DEVICE)
        # keys whose channels differ in size and lie off zero, as those of trained models do
        size, off = torch.exp(0.5 * _normal(g, h, d).float()).to(torch.bfloat16), _normal(g, h, d)
        s["k"], s["v"] = _normal(g, total, page, h, d), _normal(g, total, page, h, d)
        if c["op"] == "decode4":
            s["k"], s["v"] = _store4(s["k"].mul_(size).add_(off)), _store4(s["v"])
    if own and c["op"] != "write":
        from paper_2609_32999_b200 import binding as tb
        s["decode"] = tb.Decode(_model(c), s["table"], s["lens_dev"], total, window=c.get("window", 0), n_sink=c.get("sinks", 0))
    return s


def _prepare_tier(c, s, g, lens, per):
    n, page, h, d = c["batch"], c["page"], c["kv_heads"], c["dim"]
    r = np.random.default_rng(c["layout"] + 2)
    moved = r.integers(-2000, 30000, n)                  # how far a unit moves from where it was cached
    s["k_src"], s["v_src"] = _normal(g, int(per.sum()), page, h, d), _normal(g, int(per.sum()), page, h, d)
    perms = [torch.randperm(int(per.sum()), generator=g, device=DEVICE).cpu().numpy() for _ in range(3)]
    s["k"], s["v"] = torch.zeros_like(s["k_src"]), torch.zeros_like(s["v_src"])
    unit, i = np.repeat(np.arange(n), lens), np.concatenate([np.arange(t) for t in lens])
    at = (np.cumsum(per) - per)[unit] + i // page
    s["src"], s["dst"] = (torch.from_numpy(p[at] * page + i % page).to(DEVICE) for p in (perms[0], perms[2]))
    s["moved"] = torch.from_numpy(moved[unit]).to(DEVICE)
    if own:
        size = (int(per.sum()), h, page * (d // 2 + 8))
        s["k4"], s["v4"] = torch.zeros(size, dtype=torch.uint8, device=DEVICE), torch.zeros(size, dtype=torch.uint8, device=DEVICE)
        s["store"] = _plan(c, lens, perms[0], perms[1], int(per.sum()), sources=int(per.sum()))
        s["load"] = _plan(c, lens, perms[1], perms[2], int(per.sum()), sources=int(per.sum()), cached_pos=-moved)
    return s


# ---- one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return _calls(s, op)
    if op == "prefill":
        return _prefill(s)
    if op in ("write", "step"):
        return _write(s)
    if op == "tier4":
        return _tier(s)
    return _decode(s)


def _calls(s, op):
    if op == "prefill":
        s["plan"].partial_prefill_attn(s["k"], s["v"], s["q"], None, None, s["out"], s["lse"])
        return s["out"], s["lse"]
    if op == "write":
        s["plan"].extend_write_norm(s["k"], s["v"], s["q"], s["q_out"], s["k_new"], s["v_new"], s["q_weight"], s["k_weight"], EPS)
        return s["q_out"], s["k"], s["v"]
    if op == "step":
        s["decode"].write(s["k"], s["v"], s["q"], s["q_out"], s["k_new"], s["v_new"], s["q_weight"], s["k_weight"], EPS)
        return s["q_out"], s["k"], s["v"]
    if op == "decode":
        s["decode"].attn(s["k"], s["v"], s["q"], s["out"], s["lse"])
        return s["out"], s["lse"]
    if op == "decode4":
        s["decode"].attn_kv4(s["k"], s["v"], s["q"], s["out"], s["lse"])
        return s["out"], s["lse"]
    s["store"].kv_retain_kv4(s["k_src"], s["v_src"], s["k4"], s["v4"], fuse_rope=False)
    s["load"].kv_compose_from_kv4(s["k4"], s["v4"], s["k"], s["v"])
    return s["k"], s["v"]


def _softmax_sum(score, seen, v, product):
    """exp-normalised `score` where `seen`, times v by `product`; and the log of the sums."""
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    return torch.einsum(product, score, v), total, (top + total.log()).squeeze(-1)


def _prefill(s):
    c = s["case"]
    b, n, h, g, d = c["batch"], c["rows"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    k = s["k"][s["table"].long()].float().reshape(b, -1, h, d)
    v = s["v"][s["table"].long()].float().reshape(b, -1, h, d)
    q = s["q"].float().reshape(b, n, h, g, d) * (1.0 / math.sqrt(d))
    pos, key = s["pos"][..., None], torch.arange(k.shape[1], device=k.device)
    seen = (key <= pos) & ((key < c["sinks"]) | (key > pos - c["window"]))
    o, total, lse = _softmax_sum(torch.einsum("bnhgd,bthd->bhgnt", q, k), seen[:, None, None], v, "bhgnt,bthd->bhgnd")
    return (o / total).permute(0, 3, 1, 2, 4).reshape(b * n, h * g, d).to(torch.bfloat16), lse.permute(0, 3, 1, 2).reshape(b * n, h * g).contiguous()


def _seen_positions(c, lens):
    """[batch][n] the positions a decoded token sees, and which of them there are."""
    n = c["most"] if not c["window"] else min(c["most"], c["window"] + c["sinks"])
    j = torch.arange(n, device=lens.device)
    t = lens.long()[:, None]
    if not c["window"]:
        return torch.minimum(j, t - 1), j < t
    first = (t - c["window"]).clamp(min=0)              # of the window; the first tokens before it come first
    sinks = first.clamp(max=c["sinks"])
    at = torch.where(j < sinks, j, first + j - sinks)
    return torch.minimum(at, t - 1), at < t


def _decode(s):
    c, page = s["case"], s["case"]["page"]
    b, h, g, d = c["batch"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    at, seen = _seen_positions(c, s["lens_dev"])
    where, slot = s["table"].gather(1, at // page).long(), at % page
    read = _read16 if c["op"] == "decode" else _read4
    q = s["q"].float().reshape(b, h, g, d) * (1.0 / math.sqrt(d))
    score = torch.einsum("bhgd,bthd->bhgt", q, read(c, s["k"], where, slot))
    o, total, lse = _softmax_sum(score, seen[:, None, None], read(c, s["v"], where, slot), "bhgt,bthd->bhgd")
    return (o / total).reshape(b, h * g, d).to(torch.bfloat16), lse.reshape(b, h * g)


def _read16(c, pool, where, slot):
    return pool[where, slot].float()


def _read4(c, pool, where, slot):
    page, d, h = c["page"], c["dim"], c["kv_heads"]
    code = pool[:, :, : page * (d // 2)].view(-1, h, page, d // 2)[where, :, slot]
    four = pool[:, :, page * (d // 2):].view(-1, h, page, 8)[where, :, slot].view(torch.bfloat16).float()
    return torch.cat([(code & 15).float() * four[..., 0:1] + four[..., 1:2], (code >> 4).float() * four[..., 2:3] + four[..., 3:4]], -1)


def _turn(c, x, pos):
    """Rotates [n][heads][dim] for the positions [n]: angles in 64 bits."""
    d = c["dim"]
    angle = pos.double()[:, None] * THETA ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = (x[..., : d // 2], x[..., d // 2:]) if c["pairing"] == 0 else (x[..., 0::2], x[..., 1::2])
    turned = (a * cos - b * sin, b * cos + a * sin)
    return torch.cat(turned, -1) if c["pairing"] == 0 else torch.stack(turned, -1).reshape(x.shape)


def _write(s):
    c = s["case"]
    h, d = c["kv_heads"], c["dim"]
    q, k = s["q"].float(), s["k_new"].float()
    q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + EPS) * s["q_weight"].float()
    k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * s["k_weight"].float()
    s["q_out"].copy_(_turn(c, q, s["pos"]))
    s["k"].view(-1, h, d)[s["slot"]] = _turn(c, k, s["pos"]).to(torch.bfloat16)
    s["v"].view(-1, h, d)[s["slot"]] = s["v_new"]
    return s["q_out"], s["k"], s["v"]


def _tier(s):
    c = s["case"]
    h, d = c["kv_heads"], c["dim"]

    def back(pool):
        scale, least, code = _codes(pool.view(-1, h, d)[s["src"]].float().reshape(-1, h, 2, d // 2))
        return (code * scale + least).reshape(-1, h, d)

    s["k"].view(-1, h, d)[s["dst"]] = _turn(c, back(s["k_src"]), s["moved"]).to(torch.bfloat16)
    s["v"].view(-1, h, d)[s["dst"]] = back(s["v_src"]).to(torch.bfloat16)
    return s["k"], s["v"]


# ---- the definitions in 64 bits, request by request and head by head

def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] in ("write", "step"):
        return _exact_write(c, s)
    if c["op"] == "tier4":
        return _exact_tier(c, s)
    page, h, d, b = c["page"], c["kv_heads"], c["dim"], c["batch"]
    g = c["q_heads"] // h
    pos = _positions(c, s["lens"]) if c["op"] == "prefill" else (s["lens"] - 1)[:, None]
    outs, lses = [], []
    for r in range(b):
        t, n = int(s["lens"][r]), pos.shape[1]
        ids = s["table"][r, : -(-t // page)].long()
        q = s["q"][r * n:(r + 1) * n].double()
        p, key = torch.from_numpy(pos[r]).to(DEVICE)[:, None], torch.arange(t, device=DEVICE)[None]
        hidden = key > p
        if c["window"]:
            hidden = hidden | ((key >= c["sinks"]) & (key + c["window"] <= p))
        o, l = torch.empty(n, h * g, d, dtype=torch.float64, device=DEVICE), torch.empty(n, h * g, dtype=torch.float64, device=DEVICE)
        for head in range(h):
            k, v = (_exact_rows(c, s[x], ids, head)[:t] for x in ("k", "v"))
            for x in range(head * g, (head + 1) * g):
                logit = (q[:, x] @ k.T) / math.sqrt(d)
                logit[hidden] = -math.inf
                l[:, x] = torch.logsumexp(logit, -1)
                o[:, x] = torch.exp(logit - l[:, x:x + 1]) @ v
        outs.append(o)
        lses.append(l)
    return torch.cat(outs), torch.cat(lses)


def _exact_rows(c, pool, ids, head):
    page, d = c["page"], c["dim"]
    if c["op"] != "decode4":
        return pool[ids, :, head].double().reshape(-1, d)
    rec = pool[ids, head]
    byte = rec[:, : page * d // 2].reshape(-1, d // 2)
    par = rec[:, page * d // 2:].contiguous().view(torch.bfloat16).double().reshape(-1, 4)
    low, high = byte.remainder(16).double(), byte.div(16, rounding_mode="floor").double()
    return torch.cat([par[:, :1] * low + par[:, 1:2], par[:, 2:3] * high + par[:, 3:]], 1)


def _exact_turn(c, x, pos):
    d = c["dim"]
    out = torch.empty_like(x)
    for m in range(d // 2):
        i, j = (m, m + d // 2) if c["pairing"] == 0 else (2 * m, 2 * m + 1)
        a = (pos.double() * math.exp(-2.0 * m / d * math.log(THETA)))[:, None]
        out[:, :, i] = x[:, :, i] * torch.cos(a) - x[:, :, j] * torch.sin(a)
        out[:, :, j] = x[:, :, i] * torch.sin(a) + x[:, :, j] * torch.cos(a)
    return out


def _exact_write(c, s):
    def normed(x, weight):
        x = x.double()
        return x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["dim"] + EPS) * weight.double()

    k, v = s["k"].double(), s["v"].double()
    k.view(-1, c["kv_heads"], c["dim"])[s["slot"]] = _exact_turn(c, normed(s["k_new"], s["k_weight"]), s["pos"])
    v.view(-1, c["kv_heads"], c["dim"])[s["slot"]] = s["v_new"].double()
    return _exact_turn(c, normed(s["q"], s["q_weight"]), s["pos"]), k, v


def _exact_tier(c, s):
    h, d = c["kv_heads"], c["dim"]
    rows = {}
    for name in ("k", "v"):
        x = s[name + "_src"].view(-1, h, d)[s["src"]].double()
        halves = []
        for y in (x[..., : d // 2], x[..., d // 2:]):
            least = y.min(-1, keepdim=True).values
            # the scale is a bf16 number: a fifteenth of the range, to the nearest
            scale = ((y.max(-1, keepdim=True).values - least) / 15).to(torch.bfloat16).double()
            code = torch.where(scale > 0, torch.round((y - least) / torch.where(scale > 0, scale, 1.0)), 0.0).clamp(0, 15)
            halves.append(code * scale + least)
        rows[name] = torch.cat(halves, -1)
    k, v = s["k"].double(), s["v"].double()
    k.view(-1, h, d)[s["dst"]] = _exact_turn(c, rows["k"], s["moved"])
    v.view(-1, h, d)[s["dst"]] = rows["v"]
    return k, v
