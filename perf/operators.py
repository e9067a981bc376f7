"""Cases of the operators around the paged cache: rotary positions fused with the append, attention of drafted trees,
moving accepted entries, reading the cache back.

A case is one call of one operator ("op") for a batch of sequences over a paged cache (16-token pages, K tiles
[dim chunk][slot][chunk], V tiles [dim][slot]).  `run` computes it in plain torch operations, or (`own`) through the
framework's entry points.  Lengths and trees come from the case's own `lengths` seed, so a case is the same batch
whatever the inputs' seed; values are normal, page tables random permutations of the pool.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_CACHE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
_SIZE = {"f32": 4, "bf16": 2, "fp8": 1}
_TINY, _GQA4, _GQA4S, _GQA5, _GQA8 = (4, 1, 64), (32, 8, 128), (32, 8, 64), (40, 8, 128), (64, 8, 128)


def _case(name, op, heads, dtype, cache, lengths=1, **more):
    c = {"op": op, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": heads[2], "dtype": dtype, "cache": cache,
         "lengths": lengths}
    c.update(more)
    return dict(c, name=name) if name else c


def _rope(name, heads, dtype, cache, rows=0, ctx=(1, 1), chunks=0, chunk=(1, 1), prefix=(0, 0), rot=None, layout="half",
          scaling="none", drafts=False, packed=False, **kw):
    """rows of one new token at the end of a context in ctx, then `chunks` chunks over a cached prefix.  drafts: the chunks
    are trees of drafted tokens, whose positions go by depth.  packed: q, k and v are slices of one projection's output."""
    return _case(name, "rope", heads, dtype, cache, rows=rows, ctx_lo=ctx[0], ctx_hi=ctx[1], chunks=chunks,
                 chunk_lo=chunk[0], chunk_hi=chunk[1], prefix_lo=prefix[0], prefix_hi=prefix[1],
                 rot=rot or heads[2], layout=layout, scaling=scaling, drafts=drafts, packed=packed, **kw)


def _tree(name, heads, dtype, cache, seqs, nodes, prefix, chain=False, **kw):
    """seqs trees of nodes[0]..nodes[1] drafted tokens over a cached prefix; chain: every node follows the one before."""
    return _case(name, "tree", heads, dtype, cache, seqs=seqs, nodes_lo=nodes[0], nodes_hi=nodes[1], prefix_lo=prefix[0],
                 prefix_hi=prefix[1], chain=chain, **kw)


def _move(name, heads, dtype, cache, seqs, depth, nodes, prefix, **kw):
    """seqs accepted paths of depth[0]..depth[1] tokens out of trees of `nodes` tokens over a cached prefix."""
    return _case(name, "move", heads, dtype, cache, seqs=seqs, depth_lo=depth[0], depth_hi=depth[1], nodes=nodes,
                 prefix_lo=prefix[0], prefix_hi=prefix[1], **kw)


def _read(name, heads, dtype, cache, seqs, length, start=(0, 0), **kw):
    """length[0]..length[1] tokens of each of seqs sequences from a position in start on."""
    return _case(name, "read", heads, dtype, cache, seqs=seqs, len_lo=length[0], len_hi=length[1], start_lo=start[0],
                 start_hi=start[1], **kw)


def listed():
    return [
        # A decoder at low load: one new token of a handful of sequences, q, k and v slices of the projection's output.
        _rope("rope_decode_few_bf16", _GQA4, "bf16", "bf16", 8, (500, 2500), packed=True),
        # Part of the head rotated, interleaved pairs, full precision, odd sizes (reference runs, precision studies).
        _rope("rope_partial_f32", _TINY, "f32", "f32", 5, (1, 300), chunks=3, chunk=(17, 61), prefix=(0, 47), rot=24,
              layout="interleaved"),
        # Drafted trees of a loaded decoder, far into contexts that were stretched past the trained length.
        _rope("rope_drafts_fp8", _GQA8, "bf16", "fp8", chunks=48, chunk=(24, 64), prefix=(1000, 120000), scaling="yarn",
              drafts=True),
        # The largest append: a decode batch and 32 Ki prompt tokens.
        _rope("rope_burst_bf16", _GQA8, "bf16", "bf16", 256, (256, 32768), chunks=16, chunk=(1024, 3000), prefix=(0, 4096),
              scaling="wavelength", packed=True),
        # The smallest tree in full precision.
        _tree("tree_small_f32", _TINY, "f32", "f32", 3, (1, 13), (0, 150)),
        # A decoder at low load verifying small trees.
        _tree("tree_few_bf16", _GQA4, "bf16", "bf16", 4, (7, 26), (500, 2500)),
        # The largest: a loaded decoder verifying trees of up to 64 nodes.
        _tree("tree_batch_bf16", _GQA8, "bf16", "bf16", 32, (32, 64), (1024, 8192)),
        # Few requests with very long contexts, e4m3 cache, short chains.
        _tree("tree_long_fp8", _GQA8, "bf16", "fp8", 2, (5, 16), (30000, 131072)),
        # Accepted paths of a small and of a full decode batch.
        _move("move_few_bf16", _GQA4, "bf16", "bf16", 4, (1, 6), 26, (500, 2500)),
        _move("move_batch_fp8", _GQA8, "bf16", "fp8", 256, (1, 9), 64, (256, 8192)),
        # K/V of finished prompts leaving for another instance, and one long prompt of an e4m3 cache from its middle on.
        _read("read_prompts_bf16", _GQA4, "bf16", "bf16", 12, (100, 4000)),
        _read("read_long_fp8", _GQA8, "bf16", "fp8", 2, (20000, 90000), (1, 30000)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A call of the same ranges: operators, types and geometries as listed, sizes over the whole range."""
    while True:
        op = rng.choice(["rope", "rope", "tree", "tree", "tree", "move", "read"])
        dtype, cache = rng.choice([("bf16", "bf16")] * 3 + [("bf16", "fp8")] * 3 + [("f32", "f32")])
        full = dtype == "f32"
        heads = rng.choice([_TINY, _GQA4S, _GQA4] if full else [_GQA4, _GQA4, _GQA5, _GQA8, _GQA4S])
        lengths = rng.randrange(1 << 16)
        if op == "rope":
            drafts = rng.random() < 0.4
            hi = _log(rng, 2, 64 if drafts else 4096)
            pre = rng.choice([0, _log(rng, 16, 120000)])
            dim = heads[2]
            c = _rope("", heads, dtype, cache, 0 if drafts else _log(rng, 1, 512), (1, _log(rng, 2, 32768)),
                      _log(rng, 1, 64 if drafts else 16), (max(1, int(hi * rng.uniform(0.1, 1.0))), hi),
                      (int(pre * rng.uniform(0.0, 1.0)), pre), rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)]),
                      rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "ntk", "yarn", "wavelength"]),
                      drafts, rng.random() < 0.5, lengths=lengths)
        elif op == "tree":
            hi, pre = _log(rng, 1, 128), _log(rng, 1, 131072)
            c = _tree("", heads, dtype, cache, _log(rng, 1, 64), (max(1, int(hi * rng.uniform(0.2, 1.0))), hi),
                      (int(pre * rng.uniform(0.0, 1.0)), pre), rng.random() < 0.25, lengths=lengths)
        elif op == "move":
            nodes, pre = _log(rng, 2, 128), _log(rng, 1, 16384)
            hi = max(1, min(_log(rng, 1, 16), nodes // 2))
            c = _move("", heads, dtype, cache, _log(rng, 1, 256), (rng.randint(1, hi), hi), nodes,
                      (int(pre * rng.uniform(0.0, 1.0)), pre), lengths=lengths)
        else:
            hi, start = _log(rng, 1, 100000), rng.choice([0, _log(rng, 1, 30000)])
            c = _read("", heads, dtype, cache, _log(rng, 1, 64), (max(1, int(hi * rng.uniform(0.1, 1.0))), hi),
                      (int(start * rng.uniform(0.0, 1.0)), start), lengths=lengths)
        w, b = work(c), _batch(c)
        most = {"rope": 1.5e9, "tree": 1.2e9, "move": 2e7, "read": 1.0e9}[op]
        padded = len(b["q"]) * int((b["prefix"] + b["q"]).max())         # what the plain form of the trees computes over
        if w["bytes"] <= most and w["flops"] <= 2.5e11 and b["pool"] * 2 * PAGE * heads[1] * heads[2] * _SIZE[cache] <= 3 << 30:
            if op != "tree" or padded * heads[0] * int(b["q"].max()) <= 2 << 30:
                return c


def _batch(c):
    """Lengths of a case: q (tokens that the call deals with), prefix (tokens in front of them), pages of the pool, trees."""
    rng = np.random.default_rng(c["lengths"])
    between = lambda lo, hi, n: rng.integers(lo, hi + 1, n).astype(np.int64)  # noqa: E731
    b = {"parents": None, "path": None}
    if c["op"] == "rope":
        ctx = between(c["ctx_lo"], c["ctx_hi"], c["rows"])
        b["q"] = np.concatenate([np.ones(c["rows"], np.int64), between(c["chunk_lo"], c["chunk_hi"], c["chunks"])])
        b["prefix"] = np.concatenate([ctx - 1, between(c["prefix_lo"], c["prefix_hi"], c["chunks"])])
    elif c["op"] == "tree":
        b["q"] = between(c["nodes_lo"], c["nodes_hi"], c["seqs"])
        b["prefix"] = between(c["prefix_lo"], c["prefix_hi"], c["seqs"])
    elif c["op"] == "move":
        b["q"] = np.full(c["seqs"], c["nodes"], np.int64)
        b["prefix"] = between(c["prefix_lo"], c["prefix_hi"], c["seqs"])
        # the root, then one node of each level, all of them behind the places that the path goes to
        b["path"] = [np.concatenate([[0], np.sort(rng.choice(np.arange(d, c["nodes"]), d - 1, replace=False))]).astype(np.int64)
                     for d in between(c["depth_lo"], c["depth_hi"], c["seqs"])]
    else:
        b["q"] = between(c["len_lo"], c["len_hi"], c["seqs"])
        b["prefix"] = between(c["start_lo"], c["start_hi"], c["seqs"])
    if c["op"] == "tree" or c.get("drafts"):
        b["parents"] = []
        for s, n in enumerate(b["q"]):                              # a node's parent: one of the few nodes before it
            i = np.arange(1, n)
            p = i - 1 if c.get("chain") else np.maximum(0, i - 1 - rng.integers(0, 8, max(0, n - 1)))
            b["parents"].append(np.concatenate([[-1], p]).astype(np.int32))
    pages = (b["prefix"] + b["q"] + PAGE - 1) // PAGE
    # the append and the move touch no earlier token: their sequences share the pages of their prefixes
    b["shared"] = b["prefix"] // PAGE if c["op"] in ("rope", "move") else np.zeros_like(pages)
    b["pages"], b["pool"] = pages, int((pages - b["shared"]).sum() + b["shared"].max()) + 7
    return b


def _masks(parents):
    """Per node the set of nodes it sees (its ancestors and itself), as rows of truth values, and its depth."""
    n = len(parents)
    see, depth = np.eye(n, dtype=bool), np.zeros(n, np.int64)
    for i in range(1, n):
        see[i] |= see[parents[i]]
        depth[i] = depth[parents[i]] + 1
    return see, depth


_SCALING = {"none": {}, "linear": {"factor": 4.0}, "ntk": {"factor": 4.0},
            "yarn": {"factor": 16.0, "original_length": 8192},
            "wavelength": {"factor": 8.0, "original_length": 8192, "low": 1.0, "high": 4.0}}
_BASE = 500000.0


def _frequencies(rot, scaling):
    """Angle per position of every pair, and the factor of both functions, in 64 bits."""
    i, s = np.arange(0, rot, 2) / rot, _SCALING[scaling]
    f, m = _BASE ** -i, 1.0
    if scaling == "linear":
        f = f / s["factor"]
    elif scaling == "ntk" and rot > 2:
        f = (_BASE * s["factor"] ** (rot / (rot - 2))) ** -i
    elif scaling == "yarn":
        # pairs that turn more than 32 times within the original length keep their angle, those that turn less than once
        # get it divided, with a ramp over the pairs between
        dim = lambda turns: rot * math.log(s["original_length"] / (turns * 2 * math.pi)) / (2 * math.log(_BASE))  # noqa: E731
        lo, hi = max(math.floor(dim(32.0)), 0), min(math.ceil(dim(1.0)), rot - 1)
        ramp = np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 0.001), 0, 1)
        f = f / s["factor"] * ramp + f * (1 - ramp)
        m = 0.1 * math.log(s["factor"]) + 1
    elif scaling == "wavelength":
        turns = s["original_length"] * f / (2 * math.pi)
        keep = np.clip((turns - s["low"]) / (s["high"] - s["low"]), 0, 1)
        f = f * keep + f / s["factor"] * (1 - keep)
    return f, m


def _randn(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=_TORCH[dtype])


def _fill(gen, elems, kind):
    """A cache of normal values, as its bytes; an e4m3 cache holds them over a scale of about 4.5 / 448."""
    if kind != "fp8":
        return _randn(gen, elems, kind).view(torch.uint8)
    out = torch.empty(elems, dtype=torch.uint8, device="cuda")
    for at in range(0, elems, 1 << 27):
        part = out[at:at + (1 << 27)]
        x = _randn(gen, part.numel(), "f32") * (448 / 4.5)
        part.copy_(x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    return out


def prepare(case, seed):
    b = _batch(case)
    hq, hkv, dim, dtype, kind = case["q_heads"], case["kv_heads"], case["head_dim"], case["dtype"], case["cache"]
    q_lens, total = b["q"].astype(np.int32), int(b["q"].sum())
    ctx_lens = (b["prefix"] + b["q"]).astype(np.int32)
    width = int(b["pages"].max())
    perm = np.random.default_rng(seed).permutation(b["pool"]).astype(np.int32)
    table = np.full((len(q_lens), width), -1, np.int32)
    at = int(b["shared"].max())
    for s, n in enumerate(b["pages"]):
        k = int(b["shared"][s])
        table[s, :k] = perm[:k]
        table[s, k:n] = perm[at:at + int(n) - k]
        at += int(n) - k
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    elems = b["pool"] * hkv * PAGE * dim
    s = {"case": case, "k_cache": _fill(gen, elems, kind), "v_cache": _fill(gen, elems, kind), "k_scale": None, "v_scale": None,
         "table": torch.from_numpy(table).cuda(), "q_lens": q_lens, "ctx_lens": ctx_lens}
    if kind == "fp8":
        s["k_scale"], s["v_scale"] = ((4.0 + torch.rand(hkv, generator=gen, device="cuda")) / 448.0 for _ in range(2))
    seq = np.repeat(np.arange(len(q_lens)), q_lens)
    place = np.arange(total) - np.repeat(np.cumsum(q_lens) - q_lens, q_lens)     # token's number within its sequence
    pos = b["prefix"][seq] + place
    if case["op"] in ("rope", "read"):
        s["page"] = s["table"][torch.from_numpy(seq).cuda(), torch.from_numpy(pos // PAGE).cuda()].long()
        s["slot"] = torch.from_numpy(pos % PAGE).cuda()
    if case["op"] == "rope":
        heads = hq + 2 * hkv
        if case["packed"]:
            x = _randn(gen, (total, heads, dim), dtype)
            s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        else:
            s["q"], s["k"], s["v"] = (_randn(gen, (total, h, dim), dtype) for h in (hq, hkv, hkv))
        s["q_out"] = torch.empty((total, hq, dim), dtype=_TORCH[dtype], device="cuda")
        s["positions"] = None
        if case["drafts"]:
            pos = b["prefix"][seq] + np.concatenate([_masks(p)[1] for p in b["parents"]])
            s["positions"] = torch.from_numpy(pos.astype(np.int32)).cuda()
        f, s["factor"] = _frequencies(case["rot"], case["scaling"])
        s["freq"], s["pos"] = torch.from_numpy(f).cuda(), torch.from_numpy(pos).cuda()
    elif case["op"] == "tree":
        s["q"], most = _randn(gen, (total, hq, dim), dtype), int(q_lens.max())
        s["out"] = torch.empty_like(s["q"])
        see = [_masks(p)[0] for p in b["parents"]]
        words = (most + 63) // 64
        bits = np.zeros((total, words), np.uint64)
        pad = np.zeros((len(q_lens), most, most), bool)
        for i, m in enumerate(see):
            pad[i, :len(m), :len(m)] = m
            rows = bits[seq == i]
            for j in range(len(m)):
                rows[:, j // 64] |= m[:, j].astype(np.uint64) << np.uint64(j % 64)
            bits[seq == i] = rows
        s["mask"] = None if case["chain"] else torch.from_numpy(bits.view(np.int64)).cuda()
        s["see"], s["seq"], s["place"] = torch.from_numpy(pad).cuda(), torch.from_numpy(seq).cuda(), torch.from_numpy(place).cuda()
        s["prefix"] = torch.from_numpy(b["prefix"]).cuda()
    elif case["op"] == "move":
        n = np.array([len(p) for p in b["path"]])
        seq = np.repeat(np.arange(len(n)), n)
        src = b["prefix"][seq] + np.concatenate(b["path"])
        dst = b["prefix"][seq] + np.arange(len(seq)) - np.repeat(np.cumsum(n) - n, n)
        s["n"], s["src"], s["dst"] = n.astype(np.int32), *(torch.from_numpy(a.astype(np.int32)).cuda() for a in (src, dst))
        s["seq"] = torch.from_numpy(seq).cuda()
    else:
        s["starts"] = b["prefix"].astype(np.int32)
        s["k_out"], s["v_out"] = (torch.empty((total, hkv, dim), dtype=_TORCH[dtype], device="cuda") for _ in range(2))
    if own:
        import paper_2512_03416_amd as ts
        ctx = s["ctx"] = ts.Context(ts.Desc.make(hq, hkv, dim, dtype, kind, b["pool"], width))
        if case["op"] == "rope":
            ctx.set_rope(case["rot"], base=_BASE, layout=case["layout"], scaling=case["scaling"], **_SCALING[case["scaling"]])
        if case["op"] == "tree":
            ctx.reserve_tree()
    return s


def _tiles(s, which):
    """The cache's tiles with page and slot in front: [page, slot, head, chunk, element] for K, [page, slot, head, dim] for
    V, as a view; an e4m3 cache as its bytes."""
    c = s["case"]
    kind, hkv, dim = c["cache"], c["kv_heads"], c["head_dim"]
    x = 16 // _SIZE[kind]
    t = s[which] if kind == "fp8" else s[which].view(_CACHE[kind])
    if which == "k_cache":
        return t.view(-1, hkv, dim // x, PAGE, x).permute(0, 3, 1, 2, 4)
    return t.view(-1, hkv, dim, PAGE).permute(0, 3, 1, 2)


def _values(s, t, which):
    """Cache elements as the numbers they stand for, in 32 bits."""
    if s["case"]["cache"] != "fp8":
        return t.float()
    return t.view(torch.float8_e4m3fn).float() * s[which[0] + "_scale"].view(1, -1, 1)


def _caches(s):
    return {w: s[w].view(_CACHE[s["case"]["cache"]]) for w in ("k_cache", "v_cache")}


def _rotated(x, cos, sin, rot, layout):
    x = x.float()
    r = x[..., :rot]
    a, b = (r[..., :rot // 2], r[..., rot // 2:]) if layout == "half" else (r[..., 0::2], r[..., 1::2])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.cat(y, -1) if layout == "half" else torch.stack(y, -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _rope_plain(s):
    c = s["case"]
    angle = s["pos"].double()[:, None] * s["freq"]
    cos, sin = ((f(angle) * s["factor"]).float()[:, None, :] for f in (torch.cos, torch.sin))
    s["q_out"].copy_(_rotated(s["q"], cos, sin, c["rot"], c["layout"]))
    k = _rotated(s["k"], cos, sin, c["rot"], c["layout"])
    for which, x in (("k_cache", k), ("v_cache", s["v"])):
        if c["cache"] == "fp8":
            x = (x.float() / s[which[0] + "_scale"].view(1, -1, 1)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        t = _tiles(s, which)
        t[s["page"], s["slot"]] = x.to(t.dtype).view(len(x), *t.shape[2:])
    return {"q_out": s["q_out"], **_caches(s)}


def _tree_plain(s):
    c = s["case"]
    hq, hkv, dim = c["q_heads"], c["kv_heads"], c["head_dim"]
    n_seq, most = len(s["q_lens"]), s["see"].shape[1]
    pages = s["table"].clamp(min=0).long()
    keys = pages.shape[1] * PAGE
    k, v = (_values(s, _tiles(s, w)[pages].reshape(-1, hkv, dim), w).view(n_seq, keys, hkv, dim).transpose(1, 2).contiguous()
            for w in ("k_cache", "v_cache"))
    q = torch.zeros((n_seq, most, hq, dim), device="cuda")
    q[s["seq"], s["place"]] = s["q"].float()
    q = q.view(n_seq, most, hkv, hq // hkv, dim).permute(0, 2, 3, 1, 4).reshape(n_seq, hkv, -1, dim)
    w = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(dim)
    at = torch.arange(keys, device="cuda")[None] - s["prefix"][:, None]          # key's number among the nodes
    see = torch.gather(s["see"], 2, at.clamp(0, most - 1)[:, None, :].expand(-1, most, -1))
    see = (see & (at < torch.from_numpy(s["q_lens"]).cuda()[:, None])[:, None]) | (at < 0)[:, None]
    w = w.view(n_seq, hkv, hq // hkv, most, keys).masked_fill(~see[:, None, None], -math.inf)
    w = torch.exp(w - w.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(n_seq, hkv, -1, keys), v).view(n_seq, hkv, hq // hkv, most, dim)
    return o.permute(0, 3, 1, 2, 4).reshape(n_seq, most, hq, dim)[s["seq"], s["place"]].to(_TORCH[c["dtype"]])


def _move_plain(s):
    for which in ("k_cache", "v_cache"):
        t = _tiles(s, which)
        page = lambda p: s["table"][s["seq"], p // PAGE].long()  # noqa: E731
        t[page(s["dst"]), (s["dst"] % PAGE).long()] = t[page(s["src"]), (s["src"] % PAGE).long()]
    return _caches(s)


def _read_plain(s):
    c = s["case"]
    for which, out in (("k_cache", s["k_out"]), ("v_cache", s["v_out"])):
        out.copy_(_values(s, _tiles(s, which)[s["page"], s["slot"]].reshape(out.shape), which))
    return {"k_out": s["k_out"], "v_out": s["v_out"]}


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"rope": _rope_plain, "tree": _tree_plain, "move": _move_plain, "read": _read_plain}[op](s)
    ctx, cache = s["ctx"], (s["k_cache"], s["v_cache"])
    scales = (s["k_scale"], s["v_scale"])
    if op == "rope":
        ctx.rope_kv_append(s["q"], s["k"], s["v"], s["q_out"], *cache, *scales, s["table"], s["q_lens"], s["ctx_lens"],
                           positions=s["positions"])
        return {"q_out": s["q_out"], **_caches(s)}
    if op == "tree":
        ctx.tree_attention(s["q"], *cache, *scales, s["table"], s["mask"], s["q_lens"], s["ctx_lens"], 0.0, s["out"])
        return s["out"]
    if op == "move":
        ctx.kv_move(*cache, s["table"], s["src"], s["dst"], s["n"], s["ctx_lens"])
        return _caches(s)
    ctx.kv_read(*cache, *scales, s["table"], s["starts"], s["q_lens"], s["k_out"], s["v_out"])
    return {"k_out": s["k_out"], "v_out": s["v_out"]}


def work(case):
    """Bytes: every input that the call needs read once, every output written once; flops: two products over every key
    that a row sees, or the rotation."""
    b = _batch(case)
    row, kv = case["q_heads"] * case["head_dim"], 2 * case["kv_heads"] * case["head_dim"]
    es, cs, total = _SIZE[case["dtype"]], _SIZE[case["cache"]], int(b["q"].sum())
    if case["op"] == "rope":
        rotated = total * case["rot"] * (case["q_heads"] + case["kv_heads"])
        return {"bytes": total * (2 * row * es + kv * (es + cs)), "flops": 3 * rotated}
    if case["op"] == "tree":
        seen = sum(int(p) * len(t) + int(_masks(t)[0].sum()) for p, t in zip(b["prefix"], b["parents"]))
        return {"bytes": int((b["prefix"] + b["q"]).sum()) * kv * cs + 2 * total * row * es, "flops": 4 * row * seen}
    if case["op"] == "move":
        return {"bytes": sum(len(p) for p in b["path"]) * (2 * kv * cs + 8), "flops": 0}
    return {"bytes": total * kv * (es + cs), "flops": 0}


# ---- the definition in 64 bits, token by token or sequence by sequence, from the same inputs ----------------------------

def _index(c, table, seq, pos):
    """Element numbers of tokens in a flat cache buffer: (K, V), each [token, head, dim]."""
    hkv, dim = c["kv_heads"], c["head_dim"]
    x = 16 // _SIZE[c["cache"]]
    d = np.arange(dim)
    tile = (table[seq, pos // PAGE].astype(np.int64)[:, None] * hkv + np.arange(hkv)[None])[:, :, None] * (PAGE * dim)
    slot = (pos % PAGE)[:, None, None]
    return tile + (d // x) * (PAGE * x) + slot * x + d % x, tile + d * PAGE + slot


def _numbers(s, which):
    return s[which].view(_CACHE[s["case"]["cache"]]).double()


def exact(case, seed):
    s, b, c = prepare(case, seed), _batch(case), case
    table = s["table"].cpu().numpy()
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    scale = {w: s[w[0] + "_scale"].double().view(1, -1, 1) if c["cache"] == "fp8" else 1.0 for w in ("k_cache", "v_cache")}
    seq = np.repeat(np.arange(len(b["q"])), b["q"])
    pos = np.concatenate([np.arange(p, p + n) for p, n in zip(b["prefix"], b["q"])])
    if c["op"] == "rope":
        at = pos if not c["drafts"] else s["pos"].cpu().numpy()
        f, m = _frequencies(c["rot"], c["scaling"])
        phase = torch.polar(torch.tensor(m, dtype=torch.float64, device="cuda"), dev(at[:, None] * f))[:, None]

        def turn(x):
            x = x.double().clone()
            pair = torch.arange(c["rot"], device="cuda").view(2, -1) if c["layout"] == "half" else \
                torch.arange(c["rot"], device="cuda").view(-1, 2).T
            z = torch.complex(x[..., pair[0]], x[..., pair[1]]) * phase
            x[..., pair[0]], x[..., pair[1]] = z.real, z.imag
            return x

        got, where = {"q_out": turn(s["q"])}, _index(c, table, seq, pos)
        for which, at, x in (("k_cache", where[0], turn(s["k"])), ("v_cache", where[1], s["v"].double())):
            got[which] = _numbers(s, which)
            x = x / scale[which]
            got[which][dev(at)] = x.clamp(-448, 448) if c["cache"] == "fp8" else x
        return got
    if c["op"] == "read":
        where = _index(c, table, seq, pos)
        return {o: s[w].view(_CACHE[c["cache"]])[dev(at)].double() * scale[w] if c["cache"] != "fp8" else
                s[w][dev(at)].view(torch.float8_e4m3fn).double() * scale[w]
                for o, w, at in (("k_out", "k_cache", where[0]), ("v_out", "v_cache", where[1]))}
    if c["op"] == "move":
        seq = s["seq"].cpu().numpy()
        src, dst = (_index(c, table, seq, s[w].cpu().numpy().astype(np.int64)) for w in ("src", "dst"))
        got = {}
        for i, which in enumerate(("k_cache", "v_cache")):
            got[which] = _numbers(s, which)
            got[which][dev(dst[i])] = got[which][dev(src[i])].clone()
        return got
    out, first = [], 0
    group = c["q_heads"] // c["kv_heads"]
    for i, (p, n) in enumerate(zip(b["prefix"], b["q"])):
        p, n = int(p), int(n)
        where = _index(c, table, np.full(p + n, i), np.arange(p + n))
        q = s["q"][first:first + n].double()
        first += n
        see = torch.ones((n, p + n), dtype=torch.bool, device="cuda")
        see[:, p:] = dev(_masks(b["parents"][i])[0])
        head = []
        for g in range(c["kv_heads"]):
            k, v = ((s[w][dev(a[:, g])].view(torch.float8_e4m3fn).double() * scale[w][0, g] if c["cache"] == "fp8" else
                     s[w].view(_CACHE[c["cache"]])[dev(a[:, g])].double())
                    for w, a in (("k_cache", where[0]), ("v_cache", where[1])))
            x = q[:, g * group:(g + 1) * group].transpose(0, 1).reshape(group * n, -1) @ k.T.contiguous()
            x = (x / math.sqrt(c["head_dim"])).masked_fill(~see.repeat(group, 1), -math.inf)
            head.append((torch.softmax(x, -1) @ v).view(group, n, -1))
        out.append(torch.cat(head).transpose(0, 1))
    return torch.cat(out)
