"""mx4_quantize, mx4_dequantize and kv4_store on the GPU against the oracle.  Codes, scales and values
are exact: every comparison is for equality."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_08411_amd as al
from gpu_util import dev_bf16
from mx4_util import bf16_normal, dev, f64, host_f64, random_cache

pytestmark = pytest.mark.gpu


def _all_bf16():
    """Every bf16 pattern as the largest of a block and as a smaller element, 2^16 blocks x 2."""
    x = np.zeros((2 << 16, 32), np.uint16)
    p = np.arange(1 << 16, dtype=np.uint16)
    x[:1 << 16, :] = p[:, None]                      # all 32 alike: the sign, subnormals, inf, NaN
    g = np.random.default_rng(1)
    x[1 << 16:, :31] = g.integers(0, 0x7F80, (1 << 16, 31)).astype(np.uint16)
    x[1 << 16:, 31] = p
    return x


def _quantize(bits):
    c, s = al.mx4_quantize(dev_bf16(bits))
    torch.cuda.synchronize()
    return c.cpu().numpy(), s.cpu().numpy()


def test_quantize_every_pattern():
    x = _all_bf16()
    c, s = _quantize(x)
    with np.errstate(invalid="ignore"):
        rc, rs = oracle.mx4.quantize(f64(x))
    assert np.array_equal(s, rs)
    assert np.array_equal(c, rc)


@pytest.mark.parametrize("shape", [(1, 32), (3, 96), (33, 160), (128, 4096), (1, 32 * 1001), (2, 3, 5, 64), (1025, 32)])
def test_quantize_shapes(shape):
    g = np.random.default_rng(list(shape))
    x = bf16_normal(g, *shape)
    x[..., :1] = 0x4200   # (32.0 in each row's first block)
    c, s = _quantize(x)
    rc, rs = oracle.mx4.quantize(f64(x))
    assert c.shape == rc.shape and np.array_equal(c, rc) and np.array_equal(s, rs)


def test_quantize_nothing():
    c, s = al.mx4_quantize(torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"))
    assert c.shape == (0, 32) and s.shape == (0, 2)
    assert al.mx4_dequantize(c, s).shape == (0, 64)


def test_dequantize_every_code_and_scale():
    c = np.tile(np.arange(256, dtype=np.uint8).reshape(16, 16), (256, 1))
    s = np.repeat(np.arange(256, dtype=np.uint8), 16).reshape(-1, 1)
    y = al.mx4_dequantize(dev(c), dev(s))
    torch.cuda.synchronize()
    ref = oracle.mx4.values(c, s)
    ref = np.where(np.abs(ref) >= 2.0 ** 128, np.copysign(np.inf, ref), ref)   # past bf16's range
    got = host_f64(y)
    assert np.array_equal(got, ref, equal_nan=True)
    fin = np.isfinite(ref)
    assert np.array_equal(np.signbit(got[fin]), np.signbit(ref[fin]))


def test_large_and_outputs_given():
    """A tensor of more segments than one pass of the grid's threads, into given outputs with guards."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn(4099, 4128, generator=g, device="cuda").bfloat16()
    n = x.numel()
    c = torch.full((n // 2 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((n // 32 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    al.mx4_quantize(x, codes=c[:n // 2].view(4099, -1), scales=s[:n // 32].view(4099, -1))
    assert bool((c[n // 2:] == 0xA5).all()) and bool((s[n // 32:] == 0xA5).all())
    rows = [0, 1, 2048, 4098]
    rc, rs = oracle.mx4.quantize(host_f64(x[rows]))
    assert np.array_equal(c[:n // 2].view(4099, -1)[rows].cpu().numpy(), rc)
    assert np.array_equal(s[:n // 32].view(4099, -1)[rows].cpu().numpy(), rs)
    y = al.mx4_dequantize(c[:n // 2].view(4099, -1), s[:n // 32].view(4099, -1))
    assert np.array_equal(host_f64(y[rows]), oracle.mx4.values(rc, rs))
    # nearest: never further off than half a step of the largest magnitude, 1 of 6 scales
    assert bool(((y.float() - x.float()).abs().view(-1, 32).amax(1) <= x.float().abs().view(-1, 32).amax(1) / 4).all())


@pytest.mark.parametrize("T,cap,Hkv,D", [(1, 1, 1, 64), (1, 100, 4, 128), (32, 544, 8, 128), (77, 80, 3, 64),
                                         (513, 700, 2, 128)])
@pytest.mark.parametrize("indexed", [True, False])
def test_store(T, cap, Hkv, D, indexed):
    g = np.random.default_rng([T, cap, Hkv, D])
    codes, scales = random_cache(g, Hkv, cap, D)
    k, v = bf16_normal(g, T, Hkv, D), bf16_normal(g, T, Hkv, D, scale=9.0)
    start = cap - T
    rows = g.choice(cap, T, replace=False).astype(np.int32) if indexed else np.arange(start, start + T)
    c, s = dev(codes), dev(scales)
    al.kv4_store(dev_bf16(k), dev_bf16(v), c, s, row_idx=dev(rows) if indexed else None, start=start)
    torch.cuda.synchronize()
    for plane, x in enumerate((k, v)):
        rc, rs = oracle.mx4.quantize(f64(x))
        codes[plane][:, rows], scales[plane][:, rows] = rc.transpose(1, 0, 2), rs.transpose(1, 0, 2)
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales)
    assert np.array_equal(host_f64(al.mx4_dequantize(c, s)), oracle.mx4.values(codes, scales))


def test_store_leaves_out_rows_outside():
    g = np.random.default_rng(8)
    T, cap, Hkv, D = 6, 20, 2, 64
    codes, scales = random_cache(g, Hkv, cap, D)
    k, v = bf16_normal(g, T, Hkv, D), bf16_normal(g, T, Hkv, D)
    rows = np.array([3, -1, 20, 19, 2 ** 31 - 1, -2 ** 31], np.int32)
    # guards on both sides of the cache
    cb = torch.full((codes.size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    sb = torch.full((scales.size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    c, s = cb[2048:2048 + codes.size].view(codes.shape), sb[2048:2048 + scales.size].view(scales.shape)
    c.copy_(dev(codes)), s.copy_(dev(scales))
    al.kv4_store(dev_bf16(k), dev_bf16(v), c, s, row_idx=dev(rows))
    torch.cuda.synchronize()
    for plane, x in enumerate((k, v)):
        rc, rs = oracle.mx4.quantize(f64(x))
        for r in (0, 3):
            codes[plane][:, rows[r]], scales[plane][:, rows[r]] = rc[r], rs[r]
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales)
    for b, n in ((cb, codes.size), (sb, scales.size)):
        assert bool((b[:2048] == 0x5A).all()) and bool((b[2048 + n:] == 0x5A).all())
    al.kv4_store(dev_bf16(k[:0]), dev_bf16(v[:0]), c, s)
    assert np.array_equal(c.cpu().numpy(), codes)


def test_strided_rows_are_refused():
    x = torch.zeros(8, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(al.AsyncLaneError, match="contiguous"):
        al.mx4_quantize(x[:, :64])
