"""The operators over a cache in 8 bits together, as a serving loop runs them over
paged caches of two layers: prompts are appended and attended to, a tree is
drafted, appended and verified, its sampled acceptance compacted in all layers,
and one more token decoded -- every step against the oracles, with no host
synchronisation in between, and the whole round replayed from a graph."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8
from oracle import kv_oracle as KO
from oracle import pctree_oracle as PO
from tests import gpu_util as G
from tests.kv8_util import host
from tests.kv_util import f64, half_step
from workloads import WORKLOADS, draw_round

pytestmark = pytest.mark.gpu

HQ, HKV, D = 8, 2, 128
N, PAGE, BLOCK, LAYERS = 16, 16, 4, 2
U = half_step(torch.bfloat16)


class Cache:
    """All layers' codes and scales, and the pages of two requests."""

    def __init__(self, slots):
        self.max_pages = -(-slots // PAGE)
        self.n_pages = 2 * self.max_pages + 1
        self.table = np.random.default_rng(1).permutation(self.n_pages)[:2 * self.max_pages] \
            .reshape(2, -1).astype(np.int32)
        self.dev_table = torch.from_numpy(self.table).cuda()
        shape = (LAYERS, self.n_pages)
        u8 = dict(dtype=torch.uint8, device="cuda")
        # (what is not written yet may be anything)
        self.codes = [torch.full((*shape, PAGE, HKV, D), 0x7f, **u8) for _ in range(2)]
        self.scales = [torch.full((*shape, PAGE // BLOCK, HKV), 255, **u8) for _ in range(2)]

    def layer(self, i):
        return [t[i] for t in (*self.codes, *self.scales)]

    def bytes(self):
        """[plane][layer] codes [places][HKV][D] and scales [blocks][HKV]."""
        return [[(host(c[i]).reshape(-1, HKV, D).copy(), host(s[i]).reshape(-1, HKV).copy())
                 for i in range(LAYERS)] for c, s in zip(self.codes, self.scales)]


def values(pair, used):
    """A plane's values, those of unused places 0."""
    codes, scales = pair
    with np.errstate(over="ignore", invalid="ignore"):
        v = O8.values(codes, scales, PAGE, BLOCK)
    v[~used] = 0.0
    return v


def close(got, want, size):
    """test_gpu_kv8_attention.py's tolerance."""
    assert (np.abs(got - want) <= (2.0 ** -11 + 5e-4) * size + U * np.abs(want) + 1e-6).all()


def test_prompt_round_and_token():
    from paper_2608_02123_gb300 import pctree as P
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    i32 = dict(dtype=torch.int32, device="cuda")
    bf = dict(dtype=torch.bfloat16, device="cuda")
    rnd = lambda *s: torch.randn(*s, generator=g, **bf)
    wl = WORKLOADS["4b_b16"].with_(V=1500, H=64, B=4, k=4, N=N, batch=2, head_scale_e=1.0,
                                   head_scale_w=0.25, seed=3)
    inp = draw_round(wl)
    R, V = wl.batch, wl.V
    C = Cache(200)
    qw, kw = rnd(D), rnd(D)
    freq = 1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    status = torch.zeros(1, **i32)
    pages = (PAGE, C.n_pages, C.max_pages, BLOCK)

    def append(layer, qkv, q_out, start, n, prefix, positions=None):
        q, k, v = (t.unflatten(1, (h, D)) for t, h in
                   zip(qkv.split([HQ * D, HKV * D, HKV * D], 1), (HQ, HKV, HKV)))
        st = qkv.stride(0)
        cfg = P.kv8_append_config(R, qkv.shape[0], HQ, HKV, D, *pages, q_stride=st, k_stride=st,
                                  v_stride=st)
        P.pctree_kv8_append(cfg, q, k, v, *C.layer(layer), q_out, start, n, prefix, C.dev_table,
                            positions, freq, qw, kw, status)

    def attend(layer, q, out, ws, start, n, prefix, parent=None):
        cfg = P.kv8_attn_config(R, q.shape[0], HQ, HKV, D, *pages)
        P.pctree_kv8_attention(cfg, q, *C.layer(layer), start, n, prefix, out, ws, C.dev_table,
                               parent, status)

    # ---- prompts of 150 and 37 tokens, packed ----
    prompt = [150, 37]
    total = sum(prompt)
    qkv = [rnd(total, (HQ + 2 * HKV) * D) for _ in range(LAYERS)]
    q = [torch.zeros(total, HQ, D, **bf) for _ in range(LAYERS)]
    out = [torch.zeros(total, HQ, D, **bf) for _ in range(LAYERS)]
    start, rows = torch.tensor([0, 150], **i32), torch.tensor(prompt, **i32)
    zero = torch.zeros(R, **i32)
    nb = P.pctree_kv8_attention_workspace_bytes(P.kv8_attn_config(R, total, HQ, HKV, D, *pages))
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    for i in range(LAYERS):
        append(i, qkv[i], q[i], start, rows, zero)
        attend(i, q[i], out[i], ws, start, rows, zero)
    after_prompt = C.bytes()

    # ---- a round: draft, append the trees, verify, accept, compact ----
    Ld, E, W, root = G.device_inputs(inp)
    dr = P.Drafter(P.make_config(V, wl.H, wl.B, wl.k, N, R))
    tree = dr.draft(Ld, E, W, root)
    prefix = rows.clone()
    tree_qkv = [rnd(R * N, (HQ + 2 * HKV) * D) for _ in range(LAYERS)]
    tree_q = [torch.zeros(R * N, HQ, D, **bf) for _ in range(LAYERS)]
    tree_out = [torch.zeros(R, N, HQ, D, **bf) for _ in range(LAYERS)]
    tree_start = torch.arange(R, **i32) * N
    head = torch.randn(HQ * D, V, generator=g, device="cuda") * 0.2
    u = torch.rand(R, N, generator=g, device="cuda")
    temp = torch.tensor([0.8, 1.0], device="cuda")
    logits = torch.empty(R, N, V, device="cuda")
    favour = torch.zeros(R, N, V, device="cuda")
    tree_host = tree.to_host()
    for r in range(R):
        for i in range(1, int(tree_host["n_nodes"][r])):
            favour[r, int(tree_host["parent"][r, i]), int(tree_host["tokens"][r, i])] += 9.0
    cc = P.kv8_compact_config(R, wl.B, N, LAYERS, HKV, D, *pages)

    def verify():
        positions = (tree.depth + prefix[:, None]).reshape(-1)
        for i in range(LAYERS):
            append(i, tree_qkv[i], tree_q[i], tree_start, tree.n_nodes, prefix, positions)
            attend(i, tree_q[i], tree_out[i], ws, tree_start, tree.n_nodes, prefix, tree.parent)
        torch.matmul(tree_out[-1].float().view(R, N, HQ * D), head, out=logits)
        logits.add_(favour)
        dr.sample_accept(logits, u, temp)

    def compact():
        P.pctree_kv8_compact(cc, dr.accepted_idx, dr.accepted_len, prefix, *C.codes, *C.scales,
                             C.dev_table, status)

    verify()
    with_tree = C.bytes()
    compact()
    compacted = C.bytes()

    # ---- one more token ----
    grown = prefix + dr.accepted_len + 1
    one, at = torch.ones(R, **i32), torch.arange(R, **i32)
    tok_qkv = rnd(R, (HQ + 2 * HKV) * D)
    tok_q, tok_out = torch.zeros(R, HQ, D, **bf), torch.zeros(R, HQ, D, **bf)
    append(0, tok_qkv, tok_q, at, one, grown)
    attend(0, tok_q, tok_out, ws, at, one, grown)
    torch.cuda.synchronize()
    dr.check_status()
    assert int(status.item()) == 0
    last = C.bytes()

    # ---- every step against its oracle ----
    place = lambda r, s: KO.place_of(s, r, PAGE, C.table)
    places = C.n_pages * PAGE

    def used_to(ends):
        m = np.zeros(places, bool)
        for r, e in enumerate(ends):
            m[[place(r, s) for s in range(e)]] = True
        return m

    n_nodes, parent = tree_host["n_nodes"], tree_host["parent"].reshape(-1)
    scale = D ** -0.5
    for i in range(LAYERS):
        used = used_to(prompt)
        K, W_ = (values(after_prompt[p][i], used) for p in range(2))
        # keys are the rotated rows, to half a step of their codes
        x, size = O8.rotated_rows(f64(qkv[i])[:, HQ * D:(HQ + HKV) * D].reshape(-1, HKV, D),
                                  f64(kw), np.r_[0:150, 0:37], f64(freq), False, 1e-6)
        codes, scales = np.zeros((places, HKV, D), np.uint8), np.zeros(
            (C.n_pages * PAGE // BLOCK, HKV), np.uint8)
        O8.append_plane(codes, scales, x, [0, 150], prompt, [0, 0], PAGE, BLOCK, C.table)
        for r, T in enumerate(prompt):
            for s in range(T):
                p, row = place(r, s), (0, 150)[r] + s
                b = O8.block_of(s, r, PAGE, BLOCK, C.table)
                assert (after_prompt[0][i][1][b] == scales[b]).all()
                e2 = 2.0 ** (scales[b].astype(float) - O8.BIAS)[:, None]
                off = 2e-6 * size[row]
                step = O8.half_step(np.abs(x[row] / e2) + off / e2) * e2
                assert (np.abs(K[p] - x[row]) <= step + off).all()
        want, size = O8.attention(f64(q[i]), K, W_, [0, 150], prompt, [0, 0], PAGE, C.table,
                                  scale)
        close(f64(out[i]), want, size)
        used = used_to([T + int(n) for T, n in zip(prompt, n_nodes)])
        K, W_ = (values(with_tree[p][i], used) for p in range(2))
        want, size = O8.attention(f64(tree_q[i]), K, W_, [0, N], n_nodes, prompt, PAGE, C.table,
                                  scale, parent)
        got = f64(tree_out[i]).reshape(R * N, HQ, D)
        for r in range(R):
            rows_r = slice(r * N, r * N + int(n_nodes[r]))
            close(got[rows_r], want[rows_r], size[rows_r])
    z = f64(logits)
    target = np.full((R, N), -1, np.int32)
    for r in range(R):
        for i in range(int(n_nodes[r])):
            target[r, i] = KO.sample_row(z[r, i], float(u[r, i]), float(temp[r]))
    lengths, paths = [], []
    for r in range(R):
        t = PO.Tree(**{f.name: tree_host[f.name][r] for f in dataclasses.fields(PO.Tree)
                       if f.name in tree_host})
        idx, length, bonus = PO.accept(t, target[r], wl.B)
        np.testing.assert_array_equal(dr.accepted_idx[r].cpu().numpy(), idx)
        assert int(dr.accepted_len[r]) == length and int(dr.bonus[r]) == bonus
        lengths.append(length)
        paths.append(idx)
    assert max(lengths) > 0
    for p in range(2):
        for i in range(LAYERS):
            codes, scales = (x.copy() for x in with_tree[p][i])
            defined = O8.compact_plane(codes, scales, np.array(paths), lengths, prompt, PAGE,
                                       BLOCK, C.table)
            defined &= used_to([T + n + 1 for T, n in zip(prompt, lengths)])
            assert (compacted[p][i][0][defined] == codes[defined]).all()
            assert (compacted[p][i][1] == scales).all()
    after = [T + n + 1 for T, n in zip(prompt, lengths)]
    used = used_to([T + 1 for T in after])
    K, W_ = (values(last[p][0], used) for p in range(2))
    want, size = O8.attention(f64(tok_q), K, W_, [0, 1], [1, 1], after, PAGE, C.table, scale)
    close(f64(tok_out), want, size)

    # ---- the round as a graph, replayed on the caches as they were before it ----
    def restore():
        for c, s, b in zip(C.codes, C.scales, after_prompt):
            c.copy_(torch.from_numpy(np.stack([x[0] for x in b])).view_as(c))
            s.copy_(torch.from_numpy(np.stack([x[1] for x in b])).view_as(s))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        verify()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        verify()
        compact()
    for _ in range(2):
        restore()
        for t in (*tree_out, dr.accepted_idx, dr.accepted_len):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = C.bytes()
        used = used_to(after)
        for p in range(2):
            for i in range(LAYERS):
                assert (replayed[p][i][0][used] == compacted[p][i][0][used]).all()
                assert (replayed[p][i][1] == compacted[p][i][1]).all()
    assert int(status.item()) == 0
