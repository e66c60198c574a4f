"""Shapes and device plumbing shared by the e4m3 pool's tests."""
import numpy as np

from synth import gen
from synth.configs import LayerShape

PAGE = 16


def shape(n_q, n_kv, hd, hidden=None, ffn=256):
    return LayerShape(hidden or n_q * hd, n_q, n_kv, hd, ffn, 1e-5, 500000.0, "bf16")


def bf16(rng, shp, std=1.0):
    """bf16 storage bits of N(0, std^2) draws."""
    return gen.to_storage(rng.standard_normal(shp).astype(np.float32) * np.float32(std), "bf16")


def wide(bits):
    return gen.widen(bits, "bf16")
