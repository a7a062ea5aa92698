"""Drafter.sample_accept: what goes wrong in sampling is seen by check_status,
and padded vocabularies are sampled as they lie."""
import pytest
import torch

from tests import gpu_util as G
from workloads import WORKLOADS, draw_round

pytestmark = pytest.mark.gpu


@pytest.fixture()
def drafted():
    from paper_2608_02123_gb300 import pctree as P
    wl = WORKLOADS["4b_b16"].with_(V=3000, H=64, B=5, k=4, N=20, batch=3, head_scale_e=1.0,
                                   head_scale_w=0.25, seed=9)
    Ld, E, W, root = G.device_inputs(draw_round(wl))
    dr = P.Drafter(P.make_config(wl.V, wl.H, wl.B, wl.k, wl.N, wl.batch))
    dr.draft(Ld, E, W, root)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    logits = torch.randn(wl.batch, wl.N, wl.V, generator=g, device="cuda").to(torch.bfloat16)
    u = torch.rand(wl.batch, wl.N, generator=g, device="cuda")
    return P, dr, logits, u


def test_a_bad_row_is_reported(drafted):
    """NaN in the logits of one tree's root: no token, and an error."""
    P, dr, logits, u = drafted
    dr.sample_accept(logits, u)
    dr.check_status()
    logits[1, 0, 77] = float("nan")
    dr.sample_accept(logits, u)
    torch.cuda.synchronize()
    assert int(dr.bonus[1]) == -1
    with pytest.raises(P.PctreeError):
        dr.check_status()


def test_a_bad_parameter_is_reported(drafted):
    P, dr, logits, u = drafted
    dr.sample_accept(logits, u, temperature=torch.tensor([1.0, -1.0, 1.0], device="cuda"))
    with pytest.raises(P.PctreeError):
        dr.check_status()


def test_a_status_of_the_callers_takes_the_error(drafted):
    P, dr, logits, u = drafted
    own = torch.zeros(1, dtype=torch.int32, device="cuda")
    logits[1, 0, 77] = float("nan")
    dr.sample_accept(logits, u, status=own)
    assert int(own.item()) == -5
    dr.check_status()


def test_padded_vocabularies(drafted):
    """logits[..., :V] of a wider tensor: the same tokens, padding never drawn."""
    P, dr, logits, u = drafted
    want = [t.clone() for t in dr.sample_accept(logits, u)] + [dr.target.clone()]
    R, N, V = logits.shape
    wide = torch.full((R, N, V + 72), 50.0, dtype=logits.dtype, device="cuda")
    wide[..., :V] = logits
    for padded in (wide[..., :V], wide.view(R * N, V + 72)[:, :V]):
        dr.target.fill_(-7)
        got = [*dr.sample_accept(padded, u), dr.target]
        dr.check_status()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
