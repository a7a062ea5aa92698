"""The operators around a round together, as a serving loop runs them: a prompt
is appended and attended to, a tree is drafted, appended and verified, tokens
are sampled from logits, accepted and compacted, and one more token is decoded
over the compacted cache -- against the float64 oracles at every step, with no
host synchronisation in between, and the verification replayed from a graph.
"""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import attention_oracle as AO
from oracle import kv_oracle as KO
from oracle import pctree_oracle as PO
from tests import gpu_util as G
from tests.kv_util import f64, half_step
from workloads import WORKLOADS, draw_round

pytestmark = pytest.mark.gpu

HQ, HKV, D = 8, 2, 128
N, SLOTS = 16, 240
U = half_step(torch.bfloat16)


@dataclasses.dataclass
class Layer:
    """One attention layer's state: contiguous caches and weights."""
    kc: torch.Tensor
    vc: torch.Tensor
    qw: torch.Tensor
    kw: torch.Tensor
    freq: torch.Tensor


def rnd(g, *shape):
    return torch.randn(*shape, generator=g, dtype=torch.bfloat16, device="cuda")


def append(P, L, qkv, q_out, start, n, prefix, positions=None):
    q, k, v = (t.unflatten(1, (h, D)) for t, h in
               zip(qkv.split([HQ * D, HKV * D, HKV * D], 1), (HQ, HKV, HKV)))
    batch = n.numel()
    cfg = P.append_config(batch, qkv.shape[0], HQ, HKV, D, SLOTS, batch, q_stride=qkv.stride(0),
                          k_stride=qkv.stride(0), v_stride=qkv.stride(0))
    P.pctree_kv_append(cfg, q, k, v, L.kc, L.vc, q_out, start, n, prefix, positions=positions,
                       inv_freq=L.freq, q_weight=L.qw, k_weight=L.kw)


def check_rotated(L, qkv, q_out, slot_k, row, pos):
    """q_out and one slot's key against norm and rotation in float64."""
    x = f64(qkv[row])
    freq = f64(L.freq)
    for got, raw, w in ((f64(q_out[row]), x[:HQ * D].reshape(HQ, D), f64(L.qw)),
                        (f64(slot_k), x[HQ * D:(HQ + HKV) * D].reshape(HKV, D), f64(L.kw))):
        for h in range(len(raw)):
            want, size = KO.norm_rotate(raw[h], w, pos, freq, False, 1e-6)
            assert (np.abs(got[h] - want) <= U * np.abs(want) + 3e-6 * size).all()


def close(got, want, size):
    """The attention tests' tolerance: probabilities and output rounded to
    bfloat16, 5e-4 for float32 scores and exponentials."""
    assert (np.abs(got - want) <= (U + 5e-4) * size + U * np.abs(want)).all()


def test_prompt_round_and_token():
    from paper_2608_02123_gb300 import pctree as P
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    i32 = dict(dtype=torch.int32, device="cuda")
    wl = WORKLOADS["4b_b16"].with_(V=1500, H=64, B=4, k=4, N=N, batch=2, head_scale_e=1.0,
                                   head_scale_w=0.25, seed=3)
    inp = draw_round(wl)
    R, V = wl.batch, wl.V
    L = Layer(torch.full((R, SLOTS, HKV, D), float("nan"), dtype=torch.bfloat16, device="cuda"),
              torch.full((R, SLOTS, HKV, D), float("nan"), dtype=torch.bfloat16, device="cuda"),
              rnd(g, D), rnd(g, D),
              1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D))

    # ---- prompts of 150 and 37 tokens, packed ----
    prompt = [150, 37]
    total = sum(prompt)
    qkv = rnd(g, total, (HQ + 2 * HKV) * D)
    q = torch.zeros(total, HQ, D, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    start, rows = torch.tensor([0, 150], **i32), torch.tensor(prompt, **i32)
    zero = torch.zeros(R, **i32)
    append(P, L, qkv, q, start, rows, zero)
    pc = P.paged_attn_config(R, total, HQ, HKV, D, SLOTS, R)
    ws = torch.empty(P.pctree_paged_attention_workspace_bytes(pc), dtype=torch.uint8,
                     device="cuda")
    P.pctree_paged_attention(pc, q, L.kc, L.vc, start, rows, zero, out, ws)

    # ---- a round: draft, append the trees, verify ----
    Ld, E, W, root = G.device_inputs(inp)
    dr = P.Drafter(P.make_config(V, wl.H, wl.B, wl.k, N, R))
    tree = dr.draft(Ld, E, W, root)
    prefix = rows.clone()
    tree_qkv = rnd(g, R * N, (HQ + 2 * HKV) * D)
    tree_q = torch.zeros(R * N, HQ, D, dtype=torch.bfloat16, device="cuda")
    tree_out = torch.zeros(R, N, HQ, D, dtype=torch.bfloat16, device="cuda")
    tree_start = torch.arange(R, **i32) * N
    ac = P.attn_config(R, N, HQ, HKV, SLOTS)
    nb = P.pctree_tree_attention_workspace_bytes(ac)
    tree_ws = torch.empty(max(nb, 256), dtype=torch.uint8, device="cuda")
    head = torch.randn(HQ * D, V, generator=g, device="cuda") * 0.2
    u = torch.rand(R, N, generator=g, device="cuda")
    temp = torch.tensor([0.8, 1.0], device="cuda")
    top_k = torch.tensor([40, 0], **i32)
    top_p = torch.tensor([1.0, 0.9], device="cuda")
    # logits that favour the drafted children, so that paths are accepted
    logits = torch.empty(R, N, V, device="cuda")
    favour = torch.zeros(R, N, V, device="cuda")
    host = tree.to_host()
    for r in range(R):
        for i in range(1, int(host["n_nodes"][r])):
            favour[r, int(host["parent"][r, i]), int(host["tokens"][r, i])] += 9.0

    def verify():
        positions = (tree.depth + prefix[:, None]).reshape(-1)
        append(P, L, tree_qkv, tree_q, tree_start, tree.n_nodes, prefix, positions)
        P.pctree_tree_attention(ac, tree_q, L.kc, L.vc, prefix, tree.n_nodes, tree.parent,
                                tree_out, tree_ws if nb else None)
        torch.matmul(tree_out.float().view(R, N, HQ * D), head, out=logits)
        logits.add_(favour)
        return dr.sample_accept(logits, u, temp, top_k, top_p)

    verify()
    first = [t.clone() for t in (tree_out, dr.target, dr.accepted_idx, dr.accepted_len, dr.bonus)]
    kc_tree, vc_tree = L.kc.clone(), L.vc.clone()

    # ---- compaction, and one more token ----
    lay = P.compact_layout(R, wl.B, N, 1, 1, SLOTS, HKV * D * 2)
    for cache in (L.kc, L.vc):
        P.pctree_compact(lay, dr.accepted_idx, dr.accepted_len, prefix, cache)
    grown = prefix + dr.accepted_len + 1
    one = torch.ones(R, **i32)
    tok_qkv = rnd(g, R, (HQ + 2 * HKV) * D)
    tok_q = torch.zeros(R, HQ, D, dtype=torch.bfloat16, device="cuda")
    tok_out = torch.zeros_like(tok_q)
    append(P, L, tok_qkv, tok_q, torch.arange(R, **i32), one, grown)
    tc = P.paged_attn_config(R, R, HQ, HKV, D, SLOTS, R)
    P.pctree_paged_attention(tc, tok_q, L.kc, L.vc, torch.arange(R, **i32), one, grown, tok_out,
                             ws)
    torch.cuda.synchronize()
    dr.check_status()

    # ---- every step against its oracle ----
    n_nodes, parent = host["n_nodes"], host["parent"]
    k, v = f64(kc_tree), f64(vc_tree)
    for r, T in enumerate(prompt):
        check_rotated(L, qkv, q, kc_tree[r, T - 1], int(start[r]) + T - 1, T - 1)
        for i in (0, int(n_nodes[r]) - 1):
            check_rotated(L, tree_qkv, tree_q, kc_tree[r, T + i], r * N + i,
                          T + int(host["depth"][r, i]))
        assert np.isnan(k[r, T + int(n_nodes[r]):]).all()        # nothing written past the tree
    k, v = np.nan_to_num(k), np.nan_to_num(v)
    flat = lambda x: x.reshape(R * SLOTS, HKV, D)
    want, size = KO.paged_attention(f64(q), flat(k), flat(v), [0, 150], prompt, [0, 0], SLOTS,
                                    None, D ** -0.5)
    close(f64(out), want, size)
    tq = f64(tree_q).reshape(R, N, HQ, D)
    want = AO.tree_attention(tq, k, v, prompt, n_nodes, parent, D ** -0.5)
    size = AO.tree_attention(tq, k, np.abs(v), prompt, n_nodes, parent, D ** -0.5)
    close(f64(first[0]), want, size)
    z = f64(logits)
    target = np.full((R, N), -1, np.int32)
    for r in range(R):
        for i in range(int(n_nodes[r])):
            target[r, i] = KO.sample_row(z[r, i], float(u[r, i]), float(temp[r]), int(top_k[r]),
                                         float(top_p[r]))
    np.testing.assert_array_equal(first[1].cpu().numpy(), target)
    lengths = []
    for r in range(R):
        t = PO.Tree(**{f.name: host[f.name][r] for f in dataclasses.fields(PO.Tree)
                       if f.name in host})
        idx, length, bonus = PO.accept(t, target[r], wl.B)
        np.testing.assert_array_equal(first[2][r].cpu().numpy(), idx)
        assert int(first[3][r]) == length and int(first[4][r]) == bonus
        lengths.append(length)
        # the accepted path's rows follow the prefix in the caches
        for j in range(length + 1):
            k[r, prompt[r] + j] = f64(kc_tree[r, prompt[r] + int(idx[j])])
            v[r, prompt[r] + j] = f64(vc_tree[r, prompt[r] + int(idx[j])])
    assert max(lengths) > 0
    after = [T + n + 1 for T, n in zip(prompt, lengths)]
    for r, T in enumerate(after):
        check_rotated(L, tok_qkv, tok_q, L.kc[r, T], r, T)
        k[r, T], v[r, T] = f64(L.kc[r, T]), f64(L.vc[r, T])
    want, size = KO.paged_attention(f64(tok_q), flat(k), flat(v), [0, 1], [1, 1], after, SLOTS,
                                    None, D ** -0.5)
    close(f64(tok_out), want, size)

    # ---- the verification step as a graph, replayed ----
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        verify()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        verify()
    for t in (tree_out, dr.target, dr.accepted_idx, dr.accepted_len, dr.bonus):
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for t, ref in zip((tree_out, dr.target, dr.accepted_idx, dr.accepted_len, dr.bonus), first):
        assert torch.equal(t, ref)


def test_sample_accept_with_temperature_zero_is_the_greedy_rule():
    from paper_2608_02123_gb300 import pctree as P
    wl = WORKLOADS["4b_b16"].with_(V=3000, H=64, B=5, k=4, N=20, batch=3, head_scale_e=1.0,
                                   head_scale_w=0.25, seed=9)
    inp = draw_round(wl)
    Ld, E, W, root = G.device_inputs(inp)
    dr = P.Drafter(P.make_config(wl.V, wl.H, wl.B, wl.k, wl.N, wl.batch))
    dr.draft(Ld, E, W, root)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    logits = torch.randn(wl.batch, wl.N, wl.V, generator=g, device="cuda").to(torch.bfloat16)
    u = torch.rand(wl.batch, wl.N, generator=g, device="cuda")
    got = [t.clone() for t in dr.sample_accept(logits, u, torch.zeros(3, device="cuda"))]
    # lowest index among equal maxima, as the library ranks
    best = (logits == logits.amax(-1, keepdim=True)).int().argmax(-1).int()
    want = dr.accept(best)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
