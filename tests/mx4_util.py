"""Inputs and error bounds shared by the GPU tests of the 4-bit operators."""
import numpy as np
import torch

import oracle
import synth

EPS32 = 2.0 ** -24   # half a step of fp32, relative
EPSB = 2.0 ** -8     # of bf16


def bf16_normal(g, *shape, scale=1.0):
    """bf16 bits of normal values."""
    return synth.f32_to_bf16_bits(g.standard_normal(shape, dtype=np.float32) * np.float32(scale))


def f64(bits):
    return synth.bf16_bits_to_f32(bits).astype(np.float64)


def host_f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def random_cache(g, Hkv, cap, D):
    """(codes, scales) of a cache of normal rows (numpy)."""
    return oracle.mx4.quantize(f64(bf16_normal(g, 2, Hkv, cap, D)))


def cache_rows(codes, scales, P):
    """K and V values [P][Hkv][D] of a cache's first P rows."""
    v = oracle.mx4.values(codes[:, :, :P], scales[:, :, :P])
    return v[0].transpose(1, 0, 2), v[1].transpose(1, 0, 2)


def attention_bounds(ref_o, mean_abs_v, ref_lse, q, k, D, n_keys):
    """Bounds on o and lse against the 64-bit result.

    Scores are sums of D exact products in fp32: each is off by at most D EPS32 sum|q k| <= D EPS32
    |q| |k|, times the scale: e (and its exponent's base-2 form by as much again).  A probability is then
    off by 2 e and by half a bf16 step for the second product, relative; the row sum adds up to n_keys
    fp32 terms.  So o, a mean of V weighted by them, is off by (EPSB + 4 e + 2 n_keys EPS32) times the mean
    of |V|, and the output's own rounding adds EPSB |o|; lse by 2 e + n_keys EPS32 and a few steps of its own
    value (at least 1)."""
    scale = D ** -0.5
    e = 2 * D * EPS32 * scale * np.linalg.norm(q, axis=-1).max() * np.linalg.norm(k, axis=-1).max()
    o = EPSB * np.abs(ref_o) + (EPSB + 4 * e + 2 * n_keys * EPS32) * mean_abs_v + 1e-30
    lse = 2 * e + n_keys * EPS32 + 8 * EPS32 * np.maximum(1.0, np.abs(ref_lse))
    return o * 1.01, lse


def lmhead_bounds(hidden, W, lse):
    """Bounds on a logit, lse and (relative) conf: fp32 sums of exact products, d / 32 MFMA steps of 32
    products each (at most d / 32 + 32 additions follow one another), and a sum of exponentials by lanes of
    16, then merges of at most 64 deep, each exponential off by 4 steps."""
    d = hidden.shape[1]
    z = (d / 32 + 32) * EPS32 * np.linalg.norm(hidden, axis=1) * np.linalg.norm(W, axis=1).max()
    s = 100 * EPS32
    return z, z + s + 4 * EPS32 * np.abs(lse), 2 * z + s + 8 * EPS32 * np.abs(lse)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()
