"""The 4-bit calls on the GPU at the ends of their ranges."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_08411_amd as al
from gpu_util import dev_bf16
from mx4_util import EPS32, EPSB, bf16_normal, f64, host_f64
import synth

pytestmark = pytest.mark.gpu


def _room(nbytes):
    """Skips where the card has not that much memory left."""
    torch.cuda.empty_cache()
    free, _ = torch.cuda.mem_get_info()
    if free < nbytes:
        pytest.skip(f"needs {nbytes / 1e9:.0f} GB, {free / 1e9:.0f} are free")


def test_the_longest_prefix():
    """One token over INT32_MAX rows: zeros, then a few that take about half of the weight.

    What is off: a score by e (mx4_util.attention_bounds); the sums of the zero keys are whole numbers below
    2^24 in each wavefront (2^31 keys on 64 splits x 16 wavefronts), so exact, and the joins add at most 16 + 64
    + 40 roundings; P and the output are rounded to bf16."""
    P, D, Hq, T = 2 ** 31 - 1, 64, 4, 40
    _room(2 * P * (D // 2 + D // 32) + (8 << 30))
    codes = torch.zeros((2, 1, P, D // 2), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((2, 1, P, D // 32), dtype=torch.uint8, device="cuda")
    g = np.random.default_rng(2)
    q = bf16_normal(g, 1, Hq, D)
    k, v = bf16_normal(g, T, 1, D), bf16_normal(g, T, 1, D)
    along = f64(q)[0] * (21.5 * D ** 0.5 / (f64(q)[0] ** 2).sum(1, keepdims=True))   # a key along each query, score ~21.5
    k[-Hq:, 0] = synth.f32_to_bf16_bits(along.astype(np.float32))
    al.kv4_store(dev_bf16(k), dev_bf16(v), codes, scales, start=P - T)
    o, lse, _, _ = al.lane_attn_forward_kv4(dev_bf16(q), dev_bf16(k[:1]), dev_bf16(v[:1]), codes, scales, P, [-1], 1)
    got_o, got_lse = host_f64(o)[0], host_f64(lse)[0]
    del codes, scales
    torch.cuda.empty_cache()
    kk = np.concatenate([oracle.mx4.rounded(f64(k)), f64(k[:1])])[:, 0]
    vv = np.concatenate([oracle.mx4.rounded(f64(v)), f64(v[:1])])[:, 0]
    for h in range(Hq):
        qh = f64(q)[0, h]
        z = kk @ qh / D ** 0.5
        total = (P - T) + np.exp(z).sum()
        e = 2 * D * EPS32 * D ** -0.5 * np.linalg.norm(qh) * np.linalg.norm(kk, axis=1).max()
        assert 0.05 < np.exp(z).sum() / total < 0.999
        ref = np.exp(z) @ vv / total
        mean_abs = np.exp(z) @ np.abs(vv) / total
        assert (np.abs(got_o[h] - ref) <= 1.01 * (EPSB * np.abs(ref) + (EPSB + 4 * e + 240 * EPS32) * mean_abs)).all()
        assert abs(got_lse[h] - np.log(total)) <= 2 * e + 120 * EPS32 + 8 * EPS32 * np.log(total)


@pytest.mark.parametrize("n", [2 ** 32, -2 ** 32, 2 ** 31])
def test_numbers_past_32_bits_are_refused(n):
    """In the calls themselves; nothing is written."""
    codes = torch.full((2, 2, 8, 32), 0x5A, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, 2, 8, 2), 0x5A, dtype=torch.uint8, device="cuda")
    rows = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(al.AsyncLaneError, match="kv4_store: .*32-bit"):
        al.kv4_store(rows, rows, codes, scales, start=n)
    assert bool((codes == 0x5A).all()) and bool((scales == 0x5A).all())
    h = torch.ones(3, 64, dtype=torch.bfloat16, device="cuda")
    W = al.lmhead_pack_weight_mx4(*al.mx4_quantize(torch.ones(100, 64, dtype=torch.bfloat16, device="cuda")))
    conf = torch.full((3,), 7.0, device="cuda")
    with pytest.raises(al.AsyncLaneError, match="lmhead_confidence_mx4: .*32-bit"):
        al.lmhead_confidence_mx4(h, W, 100, eos_id=n, conf=conf)
    assert bool((conf == 7).all())


# Sizes past one pass of the kernels' threads (2^20 workgroups of 256 threads; four 8-element segments a thread in the
# quantiser and its inverse, one in the store): the same rows in calls that take one pass are the reference.
def _normal_rows(R, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    x = torch.empty(R, n, dtype=torch.bfloat16, device="cuda")
    for r in range(0, R, 1 << 17):
        x[r:r + (1 << 17)].normal_(generator=g)
    return x


def test_quantize_and_read_back_in_two_passes():
    R, n, step = (1 << 21) + 5, 4096, 1 << 18
    assert R * n // 8 > (1 << 20) * 256 * 4 >= step * n // 8
    _room(int(2.2 * R * n * 2.6))
    x = _normal_rows(R, n)
    codes, scales = al.mx4_quantize(x)
    for r in range(0, R, step):
        c, s = al.mx4_quantize(x[r:r + step])
        assert torch.equal(codes[r:r + step], c) and torch.equal(scales[r:r + step], s)
    rc, rs = oracle.mx4.quantize(host_f64(x[-7:]))
    assert np.array_equal(codes[-7:].cpu().numpy(), rc) and np.array_equal(scales[-7:].cpu().numpy(), rs)
    del x
    y = al.mx4_dequantize(codes, scales)
    for r in range(0, R, step):
        assert torch.equal(y[r:r + step], al.mx4_dequantize(codes[r:r + step], scales[r:r + step]))
    assert np.array_equal(host_f64(y[-7:]), oracle.mx4.values(rc, rs))


def test_store_in_two_passes():
    T, Hkv, D = (1 << 21) + 3, 8, 128
    assert T * Hkv * D // 8 > (1 << 20) * 256
    _room(16 * T * Hkv * D)
    k, v = _normal_rows(T * Hkv, D).view(T, Hkv, D), _normal_rows(T * Hkv, D).view(T, Hkv, D).neg()
    codes = torch.full((2, Hkv, T + 2, D // 2), 0x5A, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, Hkv, T + 2, D // 32), 0x5A, dtype=torch.uint8, device="cuda")
    al.kv4_store(k, v, codes, scales, start=1)
    for plane, x in enumerate((k, v)):
        c, s = al.mx4_quantize(x)
        assert torch.equal(codes[plane, :, 1:-1], c.transpose(0, 1))
        assert torch.equal(scales[plane, :, 1:-1], s.transpose(0, 1))
    for t in (codes, scales):
        assert bool((t[:, :, 0] == 0x5A).all()) and bool((t[:, :, -1] == 0x5A).all())


@pytest.mark.parametrize("rows", [1 << 15, (1 << 15) + 3])
def test_read_back_of_large_tensors(rows):
    """At 2^25 elements and past them, where the values are stored past the caches: every value."""
    n = 1024
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    codes = torch.randint(0, 256, (rows, n // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(2, 250, (rows, n // 32), generator=g, device="cuda", dtype=torch.uint8)
    y = al.mx4_dequantize(codes, scales)
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    code = torch.stack([codes & 15, codes >> 4], -1).view(rows, n // 32, 32).int()
    power = (scales.int() << 23).view(torch.float32)   # 2^(s - 127), exactly (torch.ldexp's powf is off by a step for some)
    want = (table[code] * power[..., None]).view(rows, n)
    assert torch.equal(y.float(), want)
