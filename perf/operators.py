"""The operators around a drafting round, as measurable cases.

``append``     per-head norms of queries and keys, their position rotation, and
               the append of keys and values to the cache
               (``pctree_kv_append``): what precedes every attention layer.
``attention``  causal attention of new rows over a paged or contiguous cache
               (``pctree_paged_attention``): single tokens, chains of drafted
               tokens, prompts.
``sample``     the target's tokens from its logits and given random numbers,
               with temperature, top-k, top-p and min-p (``pctree_sample``):
               what precedes the acceptance walk.

With ``own`` false ``run`` computes them in plain torch operations in 32 bits
(64 where 32 lose what matters: rotation angles, cumulative probabilities);
with ``own`` true it makes the library's calls.  Inputs are drawn on the GPU
from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
V_QWEN3 = 151936
EPS = 1e-6


def _append(name, batch, rows, prefix_max, Hq, Hkv, page, D=128, rotary=128, interleaved=False,
            norm=True, dtype="bf16", tree=False):
    return {"name": name, "kind": "append", "batch": batch, "rows": rows,
            "prefix_max": prefix_max, "Hq": Hq, "Hkv": Hkv, "D": D, "rotary": rotary,
            "interleaved": interleaved, "norm": norm, "page": page, "dtype": dtype, "tree": tree}


def _attention(name, batch, rows, prefix_max, Hq, Hkv, page, D=128, dtype="bf16"):
    return {"name": name, "kind": "attention", "batch": batch, "rows": rows,
            "prefix_max": prefix_max, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "dtype": dtype}


def _sample(name, batch, group, V, dtype, temperature, top_k, top_p, min_p):
    return {"name": name, "kind": "sample", "batch": batch, "group": group, "V": V,
            "dtype": dtype, "temperature": temperature, "top_k": top_k, "top_p": top_p,
            "min_p": min_p}


def listed():
    """``page`` 0 is a contiguous cache (one page a request)."""
    return [
        # one new token of one request, 4B-shaped: the smallest call, latency
        _append("append_4b_token", 1, 1, 2048, 32, 8, 16),
        # the drafted trees of a 14B-shaped serving batch, contiguous caches
        _append("append_14b_trees", 32, 128, 1024, 40, 8, 0, tree=True),
        # prompts of another family: fp16, no norms, half of a head rotated,
        # interleaved pairs, odd lengths
        _append("append_prompts_f16", 7, 2741, 333, 16, 16, 64, rotary=64, interleaved=True,
                norm=False, dtype="f16"),
        # decoding: one request, and a serving batch with long contexts
        _attention("attention_4b_token", 1, 1, 2048, 32, 8, 16),
        _attention("attention_14b_tokens", 32, 1, 8192, 40, 8, 64),
        # chains of 7 drafted tokens behind their roots, contiguous caches
        _attention("attention_8b_chains", 16, 8, 1024, 32, 8, 0),
        # prompts without a prefix
        _attention("attention_14b_prompts", 4, 4096, 0, 40, 8, 16),
        # odd chunks behind long prefixes, 64-dim heads, fp16
        _attention("attention_chunks_f16", 2, 777, 6001, 10, 2, 32, D=64, dtype="f16"),
        # the next token of one request
        _sample("sample_token", 1, 1, V_QWEN3, "f32", "one", 0, 0.95, 0.0),
        # a serving batch, no filter
        _sample("sample_batch_plain", 32, 1, V_QWEN3, "f32", "mixed", 0, 1.0, 0.0),
        # a small vocabulary, ragged, fp16, top-k and min-p
        _sample("sample_small_vocab_f16", 61, 1, 32003, "f16", "mixed", 40, 1.0, 0.05),
        # every node of a 14B-shaped batch of trees, parameters per request:
        # the largest logits
        _sample("sample_14b_trees", 32, 128, V_QWEN3, "bf16", "mixed", -1, -1.0, -1.0),
    ]


def _log(rng, lo, hi):
    """An integer, uniform in the logarithm over [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(32, 8), (40, 8), (16, 8), (16, 16), (10, 2), (64, 8), (5, 5), (24, 1)]
PAGES = [0, 8, 16, 32, 64, 128, 48, 200]


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "sample"])
    Hq, Hkv = rng.choice(HEADS)
    page = rng.choice(PAGES)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "append":
        batch = _log(rng, 1, 64)
        D = rng.choice([64, 128, 128, 256])
        tree = rng.random() < 0.3
        rows = _log(rng, 1, min(256 if tree else 4096, 20000 // batch))
        c = _append("", batch, rows, _log(rng, 1, 4096), Hq, Hkv, page, D=D,
                    rotary=rng.choice([D, D, D // 2, 16, 0]), interleaved=rng.random() < 0.3,
                    norm=rng.random() < 0.6, dtype=dtype, tree=tree)
    elif kind == "attention":
        D = rng.choice([64, 128, 128])
        form = rng.choice(["token", "chain", "chunk"])
        if form == "chunk":
            batch, rows = _log(rng, 1, 4), _log(rng, 17, 4096)
            # no more products than the largest listed case
            prefix = _log(rng, 1, max(16, min(8192, 15000000 // (batch * rows) - rows)))
        else:
            batch = _log(rng, 1, 64)
            rows = 1 if form == "token" else rng.randint(2, 16)
            prefix = _log(rng, 1, min(16384, 1200000 // (batch * Hkv)))
        c = _attention("", batch, rows, prefix, Hq, Hkv, page, D=D, dtype=dtype)
    else:
        batch = _log(rng, 1, 32)
        group = 1 if rng.random() < 0.6 else _log(rng, 2, 64)
        c = _sample("", batch, group, _log(rng, 500, V_QWEN3), rng.choice(["f32", "bf16", "f16"]),
                    rng.choice(["one", "mixed"]), rng.choice([0, 1, 20, 50, 1000, -1]),
                    rng.choice([1.0, 0.95, 0.5, -1.0]), rng.choice([0.0, 0.0, 0.05, -1.0]))
    del c["name"]
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _dev(a, dtype):
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


def _pages(c, rows, prefix, rng):
    """Page size, number of pages and page table [batch][max_pages].  A
    contiguous cache is one page a request; paged requests have theirs in
    random order, with some pages free."""
    if c["page"] == 0:
        size = c["prefix_max"] + c["rows"]
        return size, c["batch"], [[r] for r in range(c["batch"])]
    size = c["page"]
    need = [-(-(p + n) // size) for p, n in zip(prefix, rows)]
    n_pages = sum(need) + 3
    order = list(range(n_pages))
    rng.shuffle(order)
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [0] * (max(need) - n))
        at += n
    return size, n_pages, table


def _paged_state(c, seed):
    rows, prefix = _sizes(c)
    rng = random.Random(int(seed))
    padded = c.get("tree", False)                # [batch][N] rows, as the tree tensors
    start = [r * c["rows"] for r in range(c["batch"])] if padded else \
        [int(x) for x in np.cumsum([0] + rows[:-1])]
    total = c["batch"] * c["rows"] if padded else sum(rows)
    size, n_pages, table = _pages(c, rows, prefix, rng)
    g = _gen(seed, 1)
    dt = DTYPES[c["dtype"]]
    cache = [torch.randn(n_pages, size, c["Hkv"], c["D"], generator=g, dtype=dt, device="cuda")
             for _ in range(2)]
    i32 = torch.int32
    return {"kind": c["kind"], "total": total, "max_rows": max(rows), "rng": rng, "g": g,
            "max_keys": max(p + n for p, n in zip(prefix, rows)), "page_size": size,
            "n_pages": n_pages, "Hq": c["Hq"], "Hkv": c["Hkv"], "D": c["D"], "dtype": dt,
            "row_start": _dev(start, i32), "n_rows": _dev(rows, i32),
            "prefix_len": _dev(prefix, i32), "page_table": _dev(table, i32),
            "contiguous": c["page"] == 0, "k_cache": cache[0], "v_cache": cache[1]}


def prepare(case, seed):
    c = case
    if c["kind"] == "sample":
        g = _gen(seed, 2)
        f32 = dict(dtype=torch.float32, device="cuda")
        R, V = c["batch"] * c["group"], c["V"]
        L = torch.randn(R, V, generator=g, **f32).mul_(3.0)
        rank = torch.rand(R, V, generator=g, **f32).mul_(V).floor_().add_(1.0)
        L.sub_(rank.log_().mul_(1.1))            # Zipf(1.1) log-rank boost
        del rank
        rng = random.Random(int(seed))
        B, many = c["batch"], c["group"] > 1
        # -1: every request has its own, some of them switched off
        temp = [1.0] * B if c["temperature"] == "one" else \
            [rng.choice([0.0, 0.6, 0.7, 1.0, rng.uniform(0.3, 1.5)]) for _ in range(B)]
        top_k = [c["top_k"] if c["top_k"] >= 0 else rng.choice([0, 20, 50, 200]) for _ in range(B)]
        top_p = [c["top_p"] if c["top_p"] >= 0 else rng.choice([1.0, 0.8, 0.95]) for _ in range(B)]
        min_p = [c["min_p"] if c["min_p"] >= 0 else rng.choice([0.0, 0.0, 0.02, 0.1])
                 for _ in range(B)]
        # requests of several rows (trees) use some of them
        n_rows = [c["group"]] + [rng.randint((c["group"] + 1) // 2, c["group"])
                                 for _ in range(B - 1)]
        s = {"kind": "sample", "rows": R, "V": V, "group": c["group"],
             "logits": L.to(DTYPES[c["dtype"]]),
             "uniform": torch.rand(R, generator=g, **f32),
             "temperature": _dev(temp, torch.float32), "top_k": _dev(top_k, torch.int32),
             "top_p": _dev(top_p, torch.float32), "min_p": _dev(min_p, torch.float32),
             "n_rows": _dev(n_rows, torch.int32) if many else None,
             "tokens": torch.full((R,), -1, dtype=torch.int32, device="cuda"),
             "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
        return s
    s = _paged_state(c, seed)
    rng, g = s.pop("rng"), s.pop("g")
    total, Hq, Hkv, D, dt = s["total"], c["Hq"], c["Hkv"], c["D"], s["dtype"]
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    rnd = dict(generator=g, dtype=dt, device="cuda")
    if c["kind"] == "attention":
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
    if c["tree"]:                                # depth + prefix, siblings share one
        depth = [[min(i, rng.randint(i // 8, i // 4 + 1)) for i in range(c["rows"])]
                 for _ in range(c["batch"])]
        s["positions"] = (_dev(depth, torch.int32) + s["prefix_len"][:, None]).reshape(-1)
    s["q_out"] = torch.zeros(total, Hq, D, dtype=dt, device="cuda")
    return s


# --------------------------------------------------------------------------
# one pass, in plain operations
# --------------------------------------------------------------------------

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


def _plain_append(s):
    i = torch.arange(s["total"], device="cuda")[:, None]
    mine = (i >= s["row_start"]) & (i < s["row_start"] + s["n_rows"])      # [total][batch]
    rows = mine.any(1).nonzero()[:, 0]
    req = mine[rows].int().argmax(1)
    slot = s["prefix_len"][req] + rows - s["row_start"][req]
    page = s["page_table"][req, slot // s["page_size"]]
    at = page.long() * s["page_size"] + slot % s["page_size"]
    pos = slot if s["positions"] is None else s["positions"][rows]
    angle = pos.double()[:, None, None] * s["inv_freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    how = (cos, sin, s["rotary"], s["interleaved"])
    dt = s["dtype"]
    s["q_out"][rows] = _norm_rotate(s["q"][rows], s["q_weight"], *how).to(dt)
    s["k_cache"].view(-1, s["Hkv"], s["D"])[at] = \
        _norm_rotate(s["k"][rows], s["k_weight"], *how).to(dt)
    s["v_cache"].view(-1, s["Hkv"], s["D"])[at] = s["v"][rows]
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    Hkv, D, G = s["Hkv"], s["D"], s["Hq"] // s["Hkv"]
    B = s["row_start"].numel()
    j = torch.arange(s["max_rows"], device="cuda")
    row = s["row_start"][:, None] + j                                     # [B][R]
    real = j < s["n_rows"][:, None]
    q = s["q"][row.clamp(max=s["total"] - 1)].float()                     # [B][R][Hq][D]
    q = q.view(B, -1, Hkv, G, D).permute(0, 2, 3, 1, 4)                   # [B][Hkv][G][R][D]
    slot = torch.arange(s["max_keys"], device="cuda")
    page = s["page_table"][:, slot // s["page_size"]]
    at = page.long() * s["page_size"] + slot % s["page_size"]             # [B][S]
    k = s["k_cache"].view(-1, Hkv, D)[at].float().permute(0, 2, 3, 1)     # [B][Hkv][D][S]
    v = s["v_cache"].view(-1, Hkv, D)[at].float().transpose(1, 2)         # [B][Hkv][S][D]
    x = torch.matmul(q.flatten(2, 3), k).mul_(D ** -0.5).view(B, Hkv, G, -1, slot.numel())
    seen = slot <= (s["prefix_len"][:, None] + j)[..., None]              # [B][R][S]
    x.masked_fill_(~seen[:, None, None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.flatten(2, 3), v).view(B, Hkv, G, -1, D) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(B, -1, s["Hq"], D)
    s["out"][row[real]] = o[real].to(s["dtype"])
    return {"out": s["out"]}


def _per_row(s, name):
    return s[name].repeat_interleave(s["group"])[:, None]


def _plain_sample(s):
    z = s["logits"].float()
    T = _per_row(s, "temperature").double()
    order = z.sort(dim=1, descending=True, stable=True)
    top = order.values[:, :1].double()
    warm = torch.where(T > 0, T, torch.ones_like(T))
    w = ((order.values.double() - top) / warm).exp_()                     # best first
    rank = torch.arange(s["V"], device="cuda")
    k = _per_row(s, "top_k")
    keep = (rank < k) | (k <= 0)
    w.masked_fill_(~keep, 0.0)
    cum = w.cumsum(1)
    p = _per_row(s, "top_p").double()
    keep &= (cum - w < p * cum[:, -1:]) | (p >= 1.0)
    keep &= w >= _per_row(s, "min_p").double()
    w.masked_fill_(~keep, 0.0)
    w = torch.zeros_like(w).scatter_(1, order.indices, w).cumsum_(1)      # ascending index
    t = s["uniform"].double()[:, None] * w[:, -1:]
    token = (w <= t).sum(1)
    token = torch.where(T[:, 0] > 0, token, order.indices[:, 0]).int()
    if s["n_rows"] is None:
        return {"tokens": token}
    used = torch.arange(s["group"], device="cuda") < s["n_rows"][:, None]
    return {"tokens": torch.where(used.reshape(-1), token, -1)}


# --------------------------------------------------------------------------
# one pass, by the library
# --------------------------------------------------------------------------

def _own_run(s):
    from paper_2608_02123_gb300 import pctree as P
    cfg = s.get("cfg")
    if s["kind"] == "sample":
        if cfg is None:
            cfg = s["cfg"] = P.sample_config(s["rows"], s["V"], group=s["group"],
                                             dtype=s["logits"].dtype)
        P.pctree_sample(cfg, s["logits"], s["uniform"], s["tokens"],
                        temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                        min_p=s["min_p"], n_rows=s["n_rows"], status=s["status"])
        return {"tokens": s["tokens"]}
    table = None if s["contiguous"] else s["page_table"]
    if s["kind"] == "append":
        if cfg is None:
            cfg = s["cfg"] = P.append_config(
                s["n_rows"].numel(), s["total"], s["Hq"], s["Hkv"], s["D"], s["page_size"],
                s["n_pages"], s["page_table"].shape[1], dtype=s["dtype"], rotary_dim=s["rotary"],
                interleaved=s["interleaved"], q_stride=s["q"].stride(0),
                k_stride=s["k"].stride(0), v_stride=s["v"].stride(0), eps=EPS)
        P.pctree_kv_append(cfg, s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["q_out"],
                           s["row_start"], s["n_rows"], s["prefix_len"], page_table=table,
                           positions=s["positions"], inv_freq=s["inv_freq"],
                           q_weight=s["q_weight"], k_weight=s["k_weight"], status=s["status"])
        return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if cfg is None:
        cfg = s["cfg"] = P.paged_attn_config(
            s["n_rows"].numel(), s["total"], s["Hq"], s["Hkv"], s["D"], s["page_size"],
            s["n_pages"], s["page_table"].shape[1], dtype=s["dtype"])
        s["ws"] = torch.empty(P.pctree_paged_attention_workspace_bytes(cfg), dtype=torch.uint8,
                              device="cuda")
    P.pctree_paged_attention(cfg, s["q"], s["k_cache"], s["v_cache"], s["row_start"],
                             s["n_rows"], s["prefix_len"], s["out"], s["ws"], page_table=table,
                             status=s["status"])
    return {"out": s["out"]}


def run(s):
    if own:
        return _own_run(s)
    if s["kind"] == "append":
        return _plain_append(s)
    if s["kind"] == "attention":
        return _plain_attention(s)
    return _plain_sample(s)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    c = case
    el = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "sample":
        # the rows in use vary with the seed: their expectation
        rows = c["group"] * (1 + (c["batch"] - 1) * 0.75) if c["group"] > 1 else c["batch"]
        return {"bytes": rows * (c["V"] * el + 8.0), "flops": 3.0 * rows * c["V"]}
    rows, prefix = _sizes(c)
    if c["kind"] == "append":
        elements = float(sum(rows)) * (c["Hq"] + 2 * c["Hkv"]) * c["D"]
        return {"bytes": 2.0 * el * elements, "flops": 8.0 * elements}
    keys = sum(prefix) + sum(rows)
    pairs = sum(n * T + n * (n + 1) / 2 for n, T in zip(rows, prefix))
    return {"bytes": 2.0 * el * c["D"] * (sum(rows) * c["Hq"] + keys * c["Hkv"]),
            "flops": 4.0 * c["D"] * c["Hq"] * pairs}


# --------------------------------------------------------------------------
# the same results in 64 bits
# --------------------------------------------------------------------------

def _slots(s, r):
    """Rows of request r, and where its slots 0 .. prefix + rows - 1 lie."""
    a, n, T = (int(s[f][r]) for f in ("row_start", "n_rows", "prefix_len"))
    slot = torch.arange(T + n, device="cuda")
    at = s["page_table"][r].long()[slot // s["page_size"]] * s["page_size"] + slot % s["page_size"]
    return a, n, T, at


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
    k, v = (s[n].double() for n in ("k_cache", "v_cache"))
    for r in range(s["n_rows"].numel()):
        a, n, T, at = _slots(s, r)
        pos = torch.arange(T, T + n, device="cuda") if s["positions"] is None else \
            s["positions"][a:a + n]
        q[a:a + n] = _turned(s["q"][a:a + n], s["q_weight"], pos, s)
        k.view(-1, s["Hkv"], s["D"])[at[T:]] = _turned(s["k"][a:a + n], s["k_weight"], pos, s)
        v.view(-1, s["Hkv"], s["D"])[at[T:]] = s["v"][a:a + n].double()
    return {"q": q, "k_cache": k, "v_cache": v}


def _exact_attention(s):
    out = s["out"].double()
    G = s["Hq"] // s["Hkv"]
    for r in range(s["n_rows"].numel()):
        a, n, T, at = _slots(s, r)
        hide = torch.ones(n, T + n, dtype=torch.bool, device="cuda").triu(T + 1)
        for h in range(s["Hkv"]):
            K = s["k_cache"].view(-1, s["Hkv"], s["D"])[at, h].double()
            W = s["v_cache"].view(-1, s["Hkv"], s["D"])[at, h].double()
            for g in range(h * G, h * G + G):
                x = s["q"][a:a + n, g].double() @ K.T / math.sqrt(s["D"])
                out[a:a + n, g] = torch.softmax(x.masked_fill_(hide, -math.inf), -1) @ W
    return {"out": out}


def _exact_sample(s):
    """Row by row, from the sets' definitions."""
    L = s["logits"].double().cpu().numpy()
    par = {n: s[n].double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p")}
    u = s["uniform"].double().cpu().numpy()
    used = None if s["n_rows"] is None else s["n_rows"].cpu().numpy()
    tokens = np.full(s["rows"], -1, np.int32)
    for i in range(s["rows"]):
        b = i // s["group"]
        if used is not None and i % s["group"] >= used[b]:
            continue
        best = np.lexsort((np.arange(s["V"]), -L[i]))
        T = par["temperature"][b]
        if T == 0:
            tokens[i] = best[0]
            continue
        if par["top_k"][b] > 0:
            best = best[:int(par["top_k"][b])]
        w = np.exp((L[i][best] - L[i][best[0]]) / T)
        if par["top_p"][b] < 1:
            cum = np.cumsum(w)
            m = 1 + int(np.searchsorted(cum, par["top_p"][b] * cum[-1], side="left"))
            best, w = best[:m], w[:m]
        some = w >= par["min_p"][b]
        best, w = best[some], w[some]
        by = np.argsort(best)
        cum = np.cumsum(w[by])
        tokens[i] = best[by][np.searchsorted(cum, u[i] * cum[-1], side="right")]
    return {"tokens": torch.from_numpy(tokens)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    if case["kind"] == "attention":
        return _exact_attention(s)
    return _exact_sample(s) if s["rows"] <= 512 else None
