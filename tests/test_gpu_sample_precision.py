"""pctree_sample where the random number lies close to a border between tokens.

A relative error of at most d of the weights moves a border at F (of the total)
by at most 2 d F (1 - F) <= d / 2.  Rows of two tokens have fine weights, good to
2^-39.5 (half a dozen float roundings of terms below 2^-17, and rounding to units
of 2^-45): tokens are the formula's while the random number is further than 2^-40
from the border.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

L = np.longdouble


@pytest.fixture(scope="module")
def P():
    from paper_2608_02123_gb300 import pctree
    return pctree


def sample(P, z, u, **params):
    n, V = z.shape
    cfg = P.sample_config(n, V, dtype=z.dtype)
    tokens = torch.empty(n, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dev = {k: torch.from_numpy(v).cuda() for k, v in params.items()}
    P.pctree_sample(cfg, z, torch.from_numpy(u).cuda(), tokens, status=status, **dev)
    assert int(status.item()) == 0
    return tokens.cpu().numpy()


def near(F, lo, hi):
    """Random numbers next to the borders F whose distance is in [lo, hi), and
    where they are."""
    u = F.astype(np.float32)
    d = np.abs(F - u.astype(L))
    at = np.flatnonzero((d >= lo) & (d < hi) & (u < 1))
    return u[at], at


@pytest.mark.parametrize("form", ["plain", "streamed", "top_k", "min_p"])
def test_two_tokens(P, form):
    rng = np.random.default_rng(5)
    n = 1 << 20
    z = rng.uniform(-6, 6, (n, 2)).astype(np.float32)
    T = rng.uniform(0.5, 3, n).astype(np.float32)
    F = 1 / (1 + np.exp((z[:, 1].astype(L) - z[:, 0]) / T))
    u, at = near(F, 2.0 ** -40, 2.0 ** -36)
    assert len(u) > 200
    z, T, want = z[at], T[at], (u.astype(L) >= F[at]).astype(np.int32)
    params = dict(temperature=T)
    if form == "streamed":                       # rows of whole vectors
        z = np.concatenate([z, np.full((len(u), 6), -np.inf, np.float32)], 1)
    elif form == "top_k":
        z = np.concatenate([z, np.full((len(u), 40), -1e4, np.float32)], 1)
        params["top_k"] = np.full(len(u), 2, np.int32)
    elif form == "min_p":
        params["min_p"] = np.full(len(u), 1e-12, np.float32)
    np.testing.assert_array_equal(sample(P, torch.from_numpy(z).cuda(), u, **params), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("streamed", [False, True])
def test_thousands_of_equal_tokens(P, dtype, streamed):
    """Rows of two values, all of them light: weights good to 2^-29.4, the same
    error for equal logits, so a border moves by up to 2^-30.4."""
    V = 16384 if streamed else 16383
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    rng = np.random.default_rng(7)
    n = 1 << 17
    z = torch.from_numpy(rng.uniform(-1, 1, (n, 2)).astype(np.float32)).to(dt).float().numpy()
    T = rng.uniform(0.8, 3, n).astype(np.float32)
    first = rng.integers(6000, V - 6000, n)      # tokens of the first value
    w = np.exp((z[:, 1].astype(L) - z[:, 0]) / T)
    F = first / (first + (V - first) * w)
    u, at = near(F, 2.0 ** -30.3, 2.0 ** -28.5)
    u, at = u[:400], at[:400]
    assert len(u) == 400
    rows = torch.from_numpy(z[at]).cuda().to(dt)
    low = torch.arange(V, device="cuda") < torch.from_numpy(first[at]).cuda()[:, None]
    rows = torch.where(low, rows[:, :1], rows[:, 1:])
    want = first[at] - (u.astype(L) < F[at])
    np.testing.assert_array_equal(sample(P, rows, u, temperature=T[at]), want)
