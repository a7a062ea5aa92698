"""Pieces of work that take longer than the limit of the kernel's waits."""
import pytest
import torch

from tests.kv_util import half_step

pytestmark = pytest.mark.gpu


def test_a_piece_of_more_than_a_second(slots=1_500_000):
    """One token over pages of one slot, a block of keys each: a KV head is a unit
    of 1.5 million blocks, about as many heads as SMs.  Queries of zero: every
    weight is 1 and sums of small whole numbers are exact, so the output is the
    mean of the values, rounded by the reciprocal, the product and the type."""
    from paper_2608_02123_gb300 import pctree as P
    heads, D, pages = 152, 64, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    i32 = dict(dtype=torch.int32, device="cuda")
    v = torch.randint(0, 4, (pages, 1, heads, D), generator=g, device="cuda")
    table = torch.randint(0, pages, (1, slots), generator=g, **i32)
    cfg = P.paged_attn_config(1, 1, heads, heads, D, 1, pages, slots)
    ws = torch.empty(P.pctree_paged_attention_workspace_bytes(cfg), dtype=torch.uint8,
                     device="cuda")
    q = torch.zeros(1, heads, D, dtype=torch.bfloat16, device="cuda")
    k = torch.randn(pages, 1, heads, D, generator=g, device="cuda").to(torch.bfloat16)
    out = torch.full_like(q, 9.0)
    status = torch.zeros(1, **i32)
    P.pctree_paged_attention(cfg, q, k, v.to(torch.bfloat16), torch.zeros(1, **i32),
                             torch.ones(1, **i32), torch.full((1,), slots - 1, **i32), out, ws,
                             page_table=table, status=status)
    assert int(status.item()) == 0
    times = torch.bincount(table[0], minlength=pages).double()
    want = (times[:, None, None] * v[:, 0].double()).sum(0) / slots
    tol = (half_step(torch.bfloat16) + 2.0 ** -22) * want.abs()
    assert bool(((out[0].double() - want).abs() <= tol).all())
