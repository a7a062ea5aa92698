"""The target's cache in 8 bits, as measurable cases.

A cache of e4m3 values with a power-of-two scale (e8m0) for every block of
``scale_block`` consecutive slots of a page and KV head:

``append``     per-head norms of queries and keys, their position rotation, and
               the append of keys and values in 8 bits (``pctree_kv8_append``).
``attention``  attention of new rows over that cache (``pctree_kv8_attention``):
               single tokens, chains of drafted tokens, packed trees, prompts.
``compact``    the accepted path's rows moved behind the verified prefix, in
               all layers (``pctree_kv8_compact``).

With ``own`` false ``run`` computes them in plain torch operations in 32 bits
(rotation angles in 64); with ``own`` true it makes the library's calls.  Inputs
are drawn on the GPU from the seed.  Caches and scales come back in their own
8-bit floating types: a byte's value is what it stands for.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
EPS = 1e-6
MAX_CODE, MIN_EXP, MAX_EXP = 448.0, -15, 7      # of a code, and of the scales


def _append(name, batch, rows, prefix_max, Hq, Hkv, page, block, D=128, rotary=128,
            interleaved=False, norm=True, dtype="bf16", tree=False):
    return {"name": name, "kind": "append", "batch": batch, "rows": rows,
            "prefix_max": prefix_max, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "block": block,
            "rotary": rotary, "interleaved": interleaved, "norm": norm, "dtype": dtype,
            "tree": tree}


def _attention(name, batch, rows, prefix_max, Hq, Hkv, page, block, D=128, dtype="bf16",
               tree=False):
    return {"name": name, "kind": "attention", "batch": batch, "rows": rows,
            "prefix_max": prefix_max, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "block": block,
            "dtype": dtype, "tree": tree}


def _compact(name, batch, B, N, layers, prefix_max, Hkv, page, block, D=128):
    return {"name": name, "kind": "compact", "batch": batch, "rows": N, "B": B, "layers": layers,
            "prefix_max": prefix_max, "Hkv": Hkv, "D": D, "page": page, "block": block,
            "tree": True}


def listed():
    """``page`` 0 is a contiguous cache (one page a request)."""
    return [
        # one new token of one request, 4B-shaped: the smallest call, latency
        _append("append8_4b_token", 1, 1, 2048, 32, 8, 16, 1),
        # chains of 7 drafted tokens behind their roots, in blocks that hold
        # earlier slots whose scale they may raise
        _append("append8_8b_chains", 16, 8, 1024, 32, 8, 32, 32),
        # the drafted trees of a 14B-shaped serving batch, contiguous caches
        _append("append8_14b_trees", 32, 128, 1024, 40, 8, 0, 1, tree=True),
        # prompts of another family: fp16, no norms, half of a head rotated,
        # interleaved pairs, odd lengths
        _append("append8_prompts_f16", 7, 2741, 333, 16, 16, 64, 16, rotary=64, interleaved=True,
                norm=False, dtype="f16"),
        # decoding: one request, and a serving batch with long contexts
        _attention("attention8_4b_token", 1, 1, 2048, 32, 8, 16, 1),
        _attention("attention8_14b_tokens", 32, 1, 8192, 40, 8, 64, 1),
        # chains of 7 drafted tokens behind their roots
        _attention("attention8_8b_chains", 16, 8, 1024, 32, 8, 32, 32),
        # the drafted trees of a 14B-shaped batch, contiguous caches
        _attention("attention8_14b_trees", 32, 128, 1024, 40, 8, 0, 1, tree=True),
        # prompts without a prefix
        _attention("attention8_14b_prompts", 4, 4096, 0, 40, 8, 16, 16),
        # odd chunks behind long prefixes, 64-dim heads, fp16, odd pages
        _attention("attention8_chunks_f16", 2, 777, 6001, 10, 2, 48, 4, D=64, dtype="f16"),
        # one request's accepted path in all layers
        _compact("compact8_4b", 1, 16, 64, 36, 2048, 8, 16, 1),
        # a 14B-shaped batch's, in blocks of 16 slots
        _compact("compact8_14b_blocks", 32, 16, 128, 40, 512, 8, 0, 16),
    ]


def _log(rng, lo, hi):
    """An integer, uniform in the logarithm over [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(32, 8), (40, 8), (16, 8), (16, 16), (10, 2), (64, 8), (5, 5), (24, 1)]
PAGES = [0, 8, 16, 32, 64, 128, 48, 200]
BLOCKS = [1, 1, 2, 8, 16, 32, 128]


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "compact"])
    Hq, Hkv = rng.choice(HEADS)
    page, block = rng.choice(PAGES), rng.choice(BLOCKS)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    D = rng.choice([64, 128, 128])
    if kind == "append":
        batch = _log(rng, 1, 64)
        tree = rng.random() < 0.3
        rows = _log(rng, 1, min(256 if tree else 4096, 20000 // batch))
        c = _append("", batch, rows, _log(rng, 1, 4096), Hq, Hkv, page, block, D=D,
                    rotary=rng.choice([D, D, D // 2, 16, 0]), interleaved=rng.random() < 0.3,
                    norm=rng.random() < 0.6, dtype=dtype, tree=tree)
    elif kind == "attention":
        form = rng.choice(["token", "chain", "tree", "chunk"])
        if form == "chunk":
            batch, rows = _log(rng, 1, 4), _log(rng, 17, 4096)
            # no more products than the largest listed case
            prefix = _log(rng, 1, max(16, min(8192, 15000000 // (batch * rows) - rows)))
        else:
            batch = _log(rng, 1, 64)
            rows = {"token": 1, "chain": rng.randint(2, 16), "tree": _log(rng, 8, 128)}[form]
            prefix = _log(rng, 1, min(16384, 1200000 // (batch * Hkv)))
            if form == "tree":
                prefix = min(prefix, max(16, 8000000 // (batch * rows) - rows))
        c = _attention("", batch, rows, prefix, Hq, Hkv, page, block, D=D, dtype=dtype,
                       tree=form == "tree")
    else:
        batch, layers = _log(rng, 1, 32), _log(rng, 4, 64)
        prefix = _log(rng, 1, max(16, min(4096, 900000 // (batch * layers))))
        c = _compact("", batch, rng.choice([5, 7, 16]), _log(rng, 8, 128), layers, prefix, Hkv,
                     page, block, D=D)
    del c["name"]
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _dev(a, dtype=torch.int32):
    return torch.tensor(a, dtype=dtype, device="cuda")


def _sizes(c):
    """Rows and prefix of each request, by the case alone: request 0 has the
    most of both."""
    rng = random.Random(c["batch"] + 100 * c["rows"] + 1000000 * c["prefix_max"])
    rows = [c["rows"]] + [rng.randint((c["rows"] + 1) // 2, c["rows"])
                          for _ in range(c["batch"] - 1)]
    prefix = [c["prefix_max"]] + [rng.randint(c["prefix_max"] // 2, c["prefix_max"])
                                  for _ in range(c["batch"] - 1)]
    return rows, prefix


def _accepted(c):
    """Drafted tokens that each request's walk accepts, by the case alone."""
    rng = random.Random(7 * c["batch"] + c["rows"])
    rows, _ = _sizes(c)
    return [min(rng.randint(c["B"] // 3, c["B"]), n - 1) for n in rows]


def _pages(c, rows, prefix, rng):
    """Page size, number of pages and page table [batch][max_pages].  A
    contiguous cache is one page a request; paged requests have theirs in
    random order, with some pages free."""
    if c["page"] == 0:
        return c["prefix_max"] + c["rows"], c["batch"], [[r] for r in range(c["batch"])]
    size = c["page"]
    need = [-(-(p + n) // size) for p, n in zip(prefix, rows)]
    order = list(range(sum(need) + 3))
    rng.shuffle(order)
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [0] * (max(need) - n))
        at += n
    return size, len(order), table


def _tree(n, rng):
    """Parents of a packed tree, breadth first: parent[i] < i, not falling."""
    parent = [-1]
    for i in range(1, n):
        parent.append(max(parent[-1], rng.randint(i // 4, max(i // 4, i // 2)), 0))
    return parent


def _ancestors(parents, N):
    """The packed trees' ancestor masks [batch][N][N], as a draft gives them."""
    mask = torch.zeros(len(parents), N, N, dtype=torch.uint8)
    for m, p in zip(mask, parents):
        for i, a in enumerate(p):
            if a >= 0:
                m[i] = m[a]
            m[i, i] = 1
    return mask.cuda()


def _cache(c, n_pages, size, g, *lead):
    """A cache's codes and scales: codes of normal numbers, as a normalised
    head's elements are, and scales of some binades around one."""
    shape = (*lead, n_pages, size, c["Hkv"], c["D"])
    code = torch.empty(shape, dtype=E4M3, device="cuda")
    flat = code.view(-1)
    step = 1 << 27
    for i in range(0, flat.numel(), step):
        part = flat[i:i + step]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda").mul_(96.0)
                   .clamp_(-MAX_CODE, MAX_CODE))
    exp = torch.randint(-8, -4, (*lead, n_pages, -(-size // c["block"]), c["Hkv"]), generator=g,
                        device="cuda")
    return code, (exp + 127).to(torch.uint8).view(E8M0)


def prepare(case, seed):
    c = case
    rows, prefix = _sizes(c)
    rng, g = random.Random(int(seed)), _gen(seed, 1)
    tree = c["tree"]                             # [batch][N] rows, as the tree tensors
    start = [r * c["rows"] for r in range(c["batch"])] if tree else \
        [sum(rows[:r]) for r in range(c["batch"])]
    total = c["batch"] * c["rows"] if tree else sum(rows)
    size, n_pages, table = _pages(c, rows, prefix, rng)
    dt = DTYPES[c.get("dtype", "bf16")]
    parents = [_tree(n, rng) for n in rows] if tree else None
    s = {"kind": c["kind"], "total": total, "max_rows": max(rows), "block": c["block"],
         "max_keys": max(p + n for p, n in zip(prefix, rows)), "page_size": size,
         "n_pages": n_pages, "Hq": c.get("Hq", 0), "Hkv": c["Hkv"], "D": c["D"], "dtype": dt,
         "row_start": _dev(start), "n_rows": _dev(rows), "prefix_len": _dev(prefix),
         "page_table": _dev(table), "contiguous": c["page"] == 0,
         "status": torch.zeros(1, dtype=torch.int32, device="cuda"), "parent": None}
    lead = (c["layers"],) if c["kind"] == "compact" else ()
    s["k_cache"], s["k_scale"] = _cache(c, n_pages, size, g, *lead)
    s["v_cache"], s["v_scale"] = _cache(c, n_pages, size, g, *lead)
    if c["kind"] == "compact":
        idx = []
        for p, n in zip(parents, _accepted(c)):
            path = [len(p) - 1]
            while path[0] > 0:
                path.insert(0, p[path[0]])
            # as many of the rows behind the root, in order, as were accepted
            path = sorted(set(path) | set(rng.sample(range(len(p)), min(len(p), n + 1))))
            path = [0] + sorted(rng.sample(path[1:], n))
            idx.append(path + [-1] * (c["B"] - n))
        s["B"], s["N"], s["layers"] = c["B"], c["rows"], c["layers"]
        s["accepted_idx"], s["accepted_len"] = _dev(idx), _dev(_accepted(c))
        return s
    rnd = dict(generator=g, dtype=dt, device="cuda")
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["kind"] == "attention":
        if tree:
            N = c["rows"]
            s["parent"] = _dev([p + [-1] * (N - len(p)) for p in parents])
            s["mask"] = _ancestors(parents, N)
        s["q"] = torch.randn(total, Hq, D, **rnd).mul_(1.5)
        s["out"] = torch.zeros(total, Hq, D, dtype=dt, device="cuda")
        return s
    # q, k and v as the slices of one projection's output
    qkv = torch.randn(total, (Hq + 2 * Hkv) * D, **rnd)
    s["q"] = qkv[:, :Hq * D].unflatten(1, (Hq, D))
    s["k"] = qkv[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D))
    s["v"] = qkv[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
    s["q_weight"] = torch.rand(D, **rnd).add_(0.5) if c["norm"] else None
    s["k_weight"] = torch.rand(D, **rnd).add_(0.5) if c["norm"] else None
    s["rotary"], s["interleaved"] = c["rotary"], c["interleaved"]
    s["inv_freq"] = 1e6 ** (-torch.arange(0, c["rotary"], 2, dtype=torch.float64, device="cuda")
                            / max(c["rotary"], 1))
    s["positions"] = None
    if tree:                                     # depth + prefix, siblings share one
        depth = [[0] * c["rows"] for _ in range(c["batch"])]
        for d, p in zip(depth, parents):
            for i, a in enumerate(p[1:], 1):
                d[i] = d[a] + 1
        s["positions"] = (_dev(depth) + s["prefix_len"][:, None]).reshape(-1)
    s["q_out"] = torch.zeros(total, Hq, D, dtype=dt, device="cuda")
    return s


# --------------------------------------------------------------------------
# one pass, in plain operations
# --------------------------------------------------------------------------

def _exponent(x):
    """Exponents of a scale tensor."""
    return x.view(torch.uint8).int() - 127


def _value(code, exp):
    return code.float() * torch.exp2(exp.float())


def _least_exp(top):
    """The smallest exponent whose largest code reaches `top`."""
    m, e = torch.frexp(top)                      # top = m 2^e, m in [0.5, 1)
    e = e - 9 + (m > MAX_CODE / 512.0)           # 448 = 0.875 * 2^9
    return torch.where(top > 0, e, MIN_EXP).clamp(MIN_EXP, MAX_EXP)


def _places(s, slot):
    """Places of slots [batch][n] in the flat cache, and of their scales."""
    page = torch.gather(s["page_table"], 1, slot // s["page_size"]).long()
    off = slot % s["page_size"]
    blocks = -(-s["page_size"] // s["block"])
    return page * s["page_size"] + off, page * blocks + off // s["block"]


def _norm_rotate(x, w, cos, sin, rotary, interleaved):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    if rotary == 0:
        return x
    r, rest = x[..., :rotary], x[..., rotary:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else r.chunk(2, -1)
    y, z = a * cos - b * sin, b * cos + a * sin
    r = torch.stack((y, z), -1).flatten(-2) if interleaved else torch.cat((y, z), -1)
    return torch.cat((r, rest), -1)


def _quantised(s, cache, scale, place, at, value, new):
    """Values [n][Hkv][D] at flat places into cache and scale, where those of
    `new` are what is appended and the others the slots that share a block with
    them.  `at` is the scale each belongs to."""
    top = value.abs().amax(-1)                                            # [n][Hkv]
    flat = scale.view(torch.uint8).view(-1, s["Hkv"])
    old = _exponent(scale).view(-1, s["Hkv"])
    want = torch.where(new[:, None], _least_exp(top), old[at])
    exp = torch.full_like(old, -128).scatter_reduce_(
        0, at[:, None].expand_as(want), want.int(), "amax")
    flat.copy_(torch.where(exp > -128, exp + 127, old + 127).to(torch.uint8))
    code = (value * torch.exp2(-exp[at].float())[..., None]).clamp(-MAX_CODE, MAX_CODE)
    cache.view(-1, s["Hkv"], s["D"])[place] = code.to(E4M3)


def _plain_append(s):
    j = torch.arange(s["max_rows"], device="cuda")
    row = s["row_start"][:, None] + j                                     # [batch][max_rows]
    real = j < s["n_rows"][:, None]
    rows = row[real]
    slot = s["prefix_len"][:, None] + j
    pos = slot[real] if s["positions"] is None else s["positions"][rows]
    angle = pos.double()[:, None, None] * s["inv_freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    how = (cos, sin, s["rotary"], s["interleaved"])
    s["q_out"][rows] = _norm_rotate(s["q"][rows], s["q_weight"], *how).to(s["dtype"])
    # earlier slots of a block that new rows begin inside: they share its scale
    back = torch.arange(-s["block"], 0, device="cuda")
    first = s["prefix_len"][:, None]
    in_block = (first % s["page_size"]) % s["block"]
    old_slot = first + back
    old = (old_slot >= first - in_block) & (s["n_rows"][:, None] > 0)
    last = s["page_table"].shape[1] * s["page_size"] - 1
    place, at = _places(s, torch.cat((old_slot, slot), 1).clamp(0, last).long())
    use = torch.cat((old, real), 1)
    place, at = place[use], at[use]
    new = torch.cat((torch.zeros_like(old), real), 1)[use]
    for cache, scale, x in ((s["k_cache"], s["k_scale"],
                             _norm_rotate(s["k"][rows], s["k_weight"], *how)),
                            (s["v_cache"], s["v_scale"], s["v"][rows].float())):
        value = _value(cache.view(-1, s["Hkv"], s["D"])[place],
                       _exponent(scale).view(-1, s["Hkv"])[at][..., None])
        value[new] = x
        _quantised(s, cache, scale, place, at, value, new)
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"],
            "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_attention(s):
    Hkv, D, G = s["Hkv"], s["D"], s["Hq"] // s["Hkv"]
    B = s["row_start"].numel()
    j = torch.arange(s["max_rows"], device="cuda")
    row = s["row_start"][:, None] + j                                     # [B][R]
    real = j < s["n_rows"][:, None]
    q = s["q"][row.clamp(max=s["total"] - 1)].float()                     # [B][R][Hq][D]
    q = q.view(B, -1, Hkv, G, D).permute(0, 2, 3, 1, 4)                   # [B][Hkv][G][R][D]
    slot = torch.arange(s["max_keys"], device="cuda")
    place, at = _places(s, slot.expand(B, -1))                            # [B][S]
    k, v = (_value(s[n + "_cache"].view(-1, Hkv, D)[place],
                   _exponent(s[n + "_scale"]).view(-1, Hkv)[at][..., None])
            for n in ("k", "v"))
    x = torch.matmul(q.flatten(2, 3), k.permute(0, 2, 3, 1)).mul_(D ** -0.5)
    x = x.view(B, Hkv, G, -1, slot.numel())
    node = slot - s["prefix_len"][:, None]                                # [B][S]
    if s["parent"] is None:
        seen = node[:, None] <= j[:, None]                                # [B][R][S]
    else:
        N = s["mask"].shape[1]
        path = torch.gather(s["mask"][:, :s["max_rows"]], 2,
                            node.clamp(0, N - 1)[:, None].expand(-1, s["max_rows"], -1))
        seen = (node < 0)[:, None] | ((path != 0) & (node < N)[:, None])
    x.masked_fill_(~seen[:, None, None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.flatten(2, 3), v.transpose(1, 2)).view(B, Hkv, G, -1, D) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(B, -1, s["Hq"], D)
    s["out"][row[real]] = o[real].to(s["dtype"])
    return {"out": s["out"]}


def _plain_compact(s):
    L, Hkv, D = s["layers"], s["Hkv"], s["D"]
    T = s["prefix_len"][:, None]
    # the final slots of the blocks that the accepted rows go to, and where
    # their rows come from
    j = torch.arange(-s["block"], s["B"] + 1, device="cuda")
    slot = T + j
    final = (j <= s["accepted_len"][:, None]) & (
        (j >= 0) | (slot >= T - (T % s["page_size"]) % s["block"]))
    src = T + torch.where(j >= 0, s["accepted_idx"][:, j.clamp(min=0)], j)
    last = s["page_table"].shape[1] * s["page_size"] - 1
    to, to_scale = (x[final] for x in _places(s, slot.clamp(0, last).long()))
    of, of_scale = (x[final] for x in _places(s, src.clamp(0, last).long()))
    for cache, scale in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])):
        flat, byte = cache.view(L, -1, Hkv, D), scale.view(torch.uint8).view(L, -1, Hkv)
        code, old = flat[:, of], byte[:, of_scale].int()                  # [L][n][Hkv](D)
        best = torch.zeros(byte.shape, dtype=torch.int32, device="cuda").scatter_reduce_(
            1, to_scale[:, None].expand_as(old), old, "amax")
        exp = best[:, to_scale]
        flat[:, to] = (code.float() * torch.exp2((old - exp).float())[..., None]).to(E4M3)
        byte[:, to_scale] = exp.to(torch.uint8)
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"],
            "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


# --------------------------------------------------------------------------
# one pass, by the library
# --------------------------------------------------------------------------

def _own_run(s):
    from paper_2608_02123_gb300 import pctree as P
    cfg = s.get("cfg")
    table = None if s["contiguous"] else s["page_table"]
    pages = (s["page_size"], s["n_pages"], s["page_table"].shape[1])
    caches = (s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    named = dict(zip(("k_cache", "v_cache", "k_scale", "v_scale"), caches))
    if s["kind"] == "compact":
        if cfg is None:
            cfg = s["cfg"] = P.kv8_compact_config(
                s["n_rows"].numel(), s["B"], s["N"], s["layers"], s["Hkv"], s["D"], *pages,
                scale_block=s["block"])
        P.pctree_kv8_compact(cfg, s["accepted_idx"], s["accepted_len"], s["prefix_len"], *caches,
                             page_table=table, status=s["status"])
        return named
    if s["kind"] == "append":
        if cfg is None:
            cfg = s["cfg"] = P.kv8_append_config(
                s["n_rows"].numel(), s["total"], s["Hq"], s["Hkv"], s["D"], *pages,
                scale_block=s["block"], dtype=s["dtype"], rotary_dim=s["rotary"],
                interleaved=s["interleaved"], q_stride=s["q"].stride(0),
                k_stride=s["k"].stride(0), v_stride=s["v"].stride(0), eps=EPS)
        P.pctree_kv8_append(cfg, s["q"], s["k"], s["v"], *caches, s["q_out"], s["row_start"],
                            s["n_rows"], s["prefix_len"], page_table=table,
                            positions=s["positions"], inv_freq=s["inv_freq"],
                            q_weight=s["q_weight"], k_weight=s["k_weight"], status=s["status"])
        return {"q": s["q_out"], **named}
    if cfg is None:
        cfg = s["cfg"] = P.kv8_attn_config(
            s["n_rows"].numel(), s["total"], s["Hq"], s["Hkv"], s["D"], *pages,
            scale_block=s["block"], dtype=s["dtype"])
        s["ws"] = torch.empty(P.pctree_kv8_attention_workspace_bytes(cfg), dtype=torch.uint8,
                              device="cuda")
    P.pctree_kv8_attention(cfg, s["q"], *caches, s["row_start"], s["n_rows"], s["prefix_len"],
                           s["out"], s["ws"], page_table=table, parent=s["parent"],
                           status=s["status"])
    return {"out": s["out"]}


def run(s):
    if own:
        return _own_run(s)
    if s["kind"] == "append":
        return _plain_append(s)
    if s["kind"] == "attention":
        return _plain_attention(s)
    return _plain_compact(s)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    c = case
    rows, prefix = _sizes(c)
    Hkv, D = c["Hkv"], c["D"]
    if c["kind"] == "compact":
        # the accepted rows of both planes behind the root, read and written
        moved = 2.0 * c["layers"] * sum(_accepted(c)) * Hkv
        return {"bytes": 2.0 * moved * D, "flops": moved * D}
    if c["kind"] == "append":
        n = float(sum(rows))
        return {"bytes": n * D * (4.0 * c["Hq"] + 6.0 * Hkv) + 2.0 * n * Hkv / c["block"],
                "flops": 8.0 * n * (c["Hq"] + 2 * Hkv) * D}
    keys = sum(prefix) + sum(rows)
    if c["tree"]:                                # the prefix and the row itself, at least
        pairs = sum(n * (T + 1.0) for n, T in zip(rows, prefix))
    else:
        pairs = sum(n * T + n * (n + 1) / 2 for n, T in zip(rows, prefix))
    return {"bytes": 4.0 * D * sum(rows) * c["Hq"] + 2.0 * keys * Hkv * (D + 1.0 / c["block"]),
            "flops": 4.0 * D * c["Hq"] * pairs}


# --------------------------------------------------------------------------
# the same results in 64 bits
# --------------------------------------------------------------------------

def _spots(s, r, n):
    """Places of the first n slots of request r, and of their scales."""
    slot = torch.arange(n, device="cuda")
    page, off = s["page_table"][r].long()[slot // s["page_size"]], slot % s["page_size"]
    per = (s["page_size"] + s["block"] - 1) // s["block"]
    return page * s["page_size"] + off, page * per + off // s["block"]


def _powers(scale):
    """The scales' values: their types know them."""
    return scale.float().double()


def _turned(x, w, pos, s):
    """Norm and rotation as a product with e^(i angle)."""
    x = x.double()
    if w is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / s["D"] + EPS).sqrt() * w.double()
    R = s["rotary"]
    if R:
        half = x[..., :R].unflatten(-1, (R // 2, 2)) if s["interleaved"] else \
            x[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           pos.double()[:, None] * s["inv_freq"])
        y = torch.view_as_real(torch.view_as_complex(half.contiguous()) * turn[:, None])
        y = y.flatten(-2) if s["interleaved"] else y.transpose(-1, -2).flatten(-2)
        x = torch.cat((y, x[..., R:]), -1)
    return x


def _exact_append(s):
    q = s["q_out"].double()
    out = {n: s[n].float().double() for n in ("k_cache", "v_cache")}
    out |= {n: _powers(s[n]) for n in ("k_scale", "v_scale")}
    ladder = 2.0 ** torch.arange(MIN_EXP, MAX_EXP + 1, dtype=torch.float64, device="cuda")
    for r in range(s["n_rows"].numel()):
        a, n, T = (int(s[f][r]) for f in ("row_start", "n_rows", "prefix_len"))
        place, at = _spots(s, r, T + n)
        pos = torch.arange(T, T + n, device="cuda") if s["positions"] is None else \
            s["positions"][a:a + n]
        q[a:a + n] = _turned(s["q"][a:a + n], s["q_weight"], pos, s)
        new = {"k": _turned(s["k"][a:a + n], s["k_weight"], pos, s), "v": s["v"][a:a + n].double()}
        touched, which = torch.unique(at[T:], return_inverse=True)
        for name, x in new.items():
            code = out[name + "_cache"].view(-1, s["Hkv"], s["D"])
            power = out[name + "_scale"].view(-1, s["Hkv"])
            top = torch.zeros(touched.numel(), s["Hkv"], dtype=torch.float64, device="cuda")
            top.index_reduce_(0, which, x.abs().amax(-1), "amax")
            # the first power of the ladder whose largest code is no smaller
            rung = torch.searchsorted(ladder * MAX_CODE, top).clamp(max=ladder.numel() - 1)
            scale = ladder[rung]
            before = torch.isin(at[:T], touched).nonzero()[:, 0]
            if before.numel():                   # (all in the first block touched)
                b = int(at[before[0]])
                i = int((touched == b).nonzero())
                was = power[b].clone()
                scale[i] = torch.maximum(scale[i], was)
                code[place[before]] *= (was / scale[i])[:, None]
            power[touched] = scale
            code[place[T:]] = x / scale[which][..., None]
    return {"q": q, **out}


def _exact_attention(s):
    out = s["out"].double()
    G = s["Hq"] // s["Hkv"]
    parent = None if s["parent"] is None else s["parent"].cpu().numpy()
    for r in range(s["n_rows"].numel()):
        a, n, T = (int(s[f][r]) for f in ("row_start", "n_rows", "prefix_len"))
        place, at = _spots(s, r, T + n)
        hide = torch.ones(n, T + n, dtype=torch.bool).triu(T + 1)
        if parent is not None:
            hide[:, T:] = True
            for i in range(n):
                at_node = i
                while at_node >= 0:
                    hide[i, T + at_node] = False
                    at_node = int(parent[r][at_node])
        hide = hide.cuda()
        for h in range(s["Hkv"]):
            K, W = (s[m + "_cache"].view(-1, s["Hkv"], s["D"])[place, h].float().double() *
                    _powers(s[m + "_scale"]).view(-1, s["Hkv"])[at, h][:, None] for m in "kv")
            for g in range(h * G, h * G + G):
                x = s["q"][a:a + n, g].double() @ K.T / math.sqrt(s["D"])
                out[a:a + n, g] = torch.softmax(x.masked_fill_(hide, -math.inf), -1) @ W
    return {"out": out}


def _exact_compact(s):
    """Block by block, in place, from the first slot that moves on."""
    out = {n: s[n].float().double() for n in ("k_cache", "v_cache")}
    out |= {n: _powers(s[n]) for n in ("k_scale", "v_scale")}
    L, Hkv, D = s["layers"], s["Hkv"], s["D"]
    for r in range(s["n_rows"].numel()):
        T, n = int(s["prefix_len"][r]), int(s["accepted_len"][r]) + 1
        path = s["accepted_idx"][r, :n].tolist()
        place, at = _spots(s, r, T + max(s["N"] if s["contiguous"] else 0, max(path) + 1))
        begin = T - T % s["page_size"] % s["block"]
        final = list(range(begin, T + n))
        src = [f if f < T else T + path[f - T] for f in final]
        for m in "kv":
            code, power = out[m + "_cache"].view(L, -1, Hkv, D), out[m + "_scale"].view(L, -1, Hkv)
            rows, was = code[:, place[src]], power[:, at[src]]            # copies
            blocks, which = torch.unique(at[final], return_inverse=True)
            scale = torch.zeros(L, blocks.numel(), Hkv, dtype=torch.float64, device="cuda")
            scale.index_reduce_(1, which, was, "amax")
            code[:, place[final]] = rows * (was / scale[:, which])[..., None]
            power[:, blocks] = scale
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    return _exact_attention(s) if case["kind"] == "attention" else _exact_compact(s)
