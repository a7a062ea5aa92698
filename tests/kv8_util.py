"""Caches in 8 bits on the GPU, for the tests of the operators over them."""
import numpy as np
import torch

from oracle import kv8_oracle as O8

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def host(t):
    """The bytes of a tensor of codes or scales."""
    return t.view(torch.uint8).cpu().numpy()


def scale_blocks(b, block):
    return b.n_pages * -(-b.page_size // block)


class Plane:
    """One plane (K or V) of a cache of `layers` layers: random codes and scales
    with a margin of a fixed pattern at both ends."""

    def __init__(self, b, Hkv, D, block, seed, layers=1, exps=(-10, -7), as_bytes=False):
        rng = np.random.default_rng(seed)
        places, blocks = b.n_pages * b.page_size, scale_blocks(b, block)
        x = np.clip(rng.standard_normal((layers, places, Hkv, D)) * 96.0, -448, 448)
        self.codes = torch.full(((layers * places + 2) * Hkv * D,), 0x55, dtype=torch.uint8)
        self.codes[Hkv * D:-Hkv * D] = torch.from_numpy(O8.encode(x).reshape(-1))
        e = rng.integers(exps[0], exps[1] + 1, (layers, blocks, Hkv)) + O8.BIAS
        self.scales = torch.full((layers * blocks * Hkv + 32,), 0x33, dtype=torch.uint8)
        self.scales[16:-16] = torch.from_numpy(e.astype(np.uint8).reshape(-1))
        self.codes, self.scales = self.codes.cuda(), self.scales.cuda()
        self.b, self.shape, self.as_bytes = b, (layers, places, blocks, Hkv, D), as_bytes

    @property
    def cache(self):
        layers, places, _, Hkv, D = self.shape
        t = self.codes[Hkv * D:-Hkv * D].view(layers * self.b.n_pages, self.b.page_size, Hkv, D)
        return t if self.as_bytes else t.view(E4M3)

    @property
    def scale(self):
        layers, _, blocks, Hkv, _ = self.shape
        t = self.scales[16:-16].view(layers * self.b.n_pages, blocks // self.b.n_pages, Hkv)
        return t if self.as_bytes else t.view(E8M0)

    def bytes(self):
        """Codes [layers][places][Hkv][D] and scales [layers][blocks][Hkv]."""
        layers, places, blocks, Hkv, D = self.shape
        return (host(self.cache).reshape(layers, places, Hkv, D).copy(),
                host(self.scale).reshape(layers, blocks, Hkv).copy())

    def margins_hold(self):
        Hkv, D = self.shape[3:]
        c, s = self.codes, self.scales
        return bool((c[:Hkv * D] == 0x55).all() and (c[-Hkv * D:] == 0x55).all()
                    and (s[:16] == 0x33).all() and (s[-16:] == 0x33).all())
