"""lmhead_confidence_mx4 on the GPU against the fp64 oracle on the weight's 4-bit values, within the
bounds derived in mx4_util.lmhead_bounds.  argmax is compared where the two largest logits are further
apart than twice a logit's bound."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_08411_amd as al
from gpu_util import dev_bf16
from mx4_util import bf16_normal, dev, f64, lmhead_bounds

pytestmark = pytest.mark.gpu


def _inputs(N, n_rows, d, V):
    g = np.random.default_rng([N, d, V])
    H = bf16_normal(g, n_rows, d)
    codes, scales = oracle.mx4.quantize(f64(bf16_normal(g, V, d, scale=d ** -0.5)))
    target = g.integers(0, V, n_rows)
    lean = g.uniform(0, 9, n_rows)
    Hf = (f64(H) + lean[:, None] * oracle.mx4.values(codes[target], scales[target])) * g.uniform(0.5, 3, n_rows)[:, None]
    import synth
    H = synth.f32_to_bf16_bits(Hf.astype(np.float32))
    rows = g.choice(n_rows, N, replace=False).astype(np.int32)
    return H, codes, scales, rows, (g.random(N) < 0.5).astype(np.uint8)


def _check(H, codes, scales, rows, sup, eos, out):
    conf, arg, lse = (t.cpu().numpy() for t in out)
    W = oracle.mx4.values(codes, scales)
    h = f64(H)
    ref = oracle.lmhead.lmhead_confidence_full(h, rows, W, sup, eos)
    bz, bl, bc = lmhead_bounds(h[rows], W, ref["lse"])
    ok = ref["gap"] > 2 * bz
    assert ok.mean() > 0.8
    assert np.array_equal(arg[ok], ref["argmax"][ok])
    assert (np.abs(lse - ref["lse"]) <= bl).all()
    assert (np.abs(conf - ref["conf"]) <= bc * ref["conf"]).all()


SWEEP = [  # N, n_rows, d, V, eos
    (1, 1, 32, 1, -1), (1, 3, 32, 2, 1), (1, 1, 4096, 700, 5), (5, 9, 64, 7, 3), (16, 16, 96, 64, -1),
    (17, 20, 128, 65, 64), (32, 64, 256, 1024, 2), (33, 40, 160, 1000, 2), (48, 48, 288, 513, 0),
    (64, 70, 384, 4097, 9), (77, 80, 416, 3000, 2), (81, 90, 640, 1111, 4), (96, 96, 544, 2049, 700),
    (97, 100, 224, 640, 3), (128, 130, 1024, 1500, -1), (129, 150, 352, 777, 5), (160, 200, 512, 900, 1),
    (161, 161, 256, 1300, 2), (208, 210, 320, 2048, 7), (209, 230, 192, 300, 9), (300, 310, 64, 513, 2),
    (614, 640, 128, 2000, 4), (77, 80, 64, 70000, 3), (8, 8, 32, 140000, 2),
]


@pytest.mark.parametrize("case", SWEEP, ids=[str(c) for c in SWEEP])
def test_against_the_oracle(case):
    N, n_rows, d, V, eos = case
    H, codes, scales, rows, sup = _inputs(N, n_rows, d, V)
    if V == 1:
        sup[:] = 0
    W = al.lmhead_pack_weight_mx4(dev(codes), dev(scales))
    out = al.lmhead_confidence_mx4(dev_bf16(H), W, V, row_idx=dev(rows), suppress_eos=dev(sup) if V > 1 else None,
                                   eos_id=eos)
    torch.cuda.synchronize()
    _check(H, codes, scales, rows, sup, eos, out)
    if eos >= 0 and V > 1:
        assert not (out[1].cpu().numpy()[sup == 1] == eos).any()


@pytest.mark.parametrize("d,V", [(32, 1), (160, 65), (4096, 200)])
def test_packed_layout(d, V):
    """Byte by byte the layout that the header states."""
    g = np.random.default_rng([d, V])
    codes = g.integers(0, 256, (V, d // 2)).astype(np.uint8)
    scales = g.integers(0, 256, (V, d // 32)).astype(np.uint8)
    U, C = 4 * ((V + 63) // 64), (d + 127) // 128
    want = np.zeros(C * U * 1088, np.uint8)
    for v in range(V):
        u, r = divmod(v, 16)
        for blk in range(d // 32):
            c, b = divmod(blk, 4)
            at = ((c * U + u) * 64 + 16 * b + r) * 16
            want[at:at + 16] = codes[v, 16 * blk:16 * blk + 16]
            want[C * U * 1024 + ((c * (U // 4) + u // 4) * 64 + 16 * b + r) * 4 + u % 4] = scales[v, blk]
    out = torch.full((want.size + 64,), 0xEE, dtype=torch.uint8, device="cuda")
    al.lmhead_pack_weight_mx4(dev(codes), dev(scales), out=out)
    got = out.cpu().numpy()
    assert np.array_equal(got[:want.size], want) and (got[want.size:] == 0xEE).all()
    assert al.lmhead_packed_weight_mx4_size(d, V) == want.size


def test_zero_weight_ties_and_duplicates():
    """W = 0: conf = 1 / |C|, the lowest allowed id; of equal largest rows the lower id."""
    N, d, V = 40, 64, 3001
    g = np.random.default_rng(5)
    H = bf16_normal(g, N, d)
    sup = np.zeros(N, np.uint8)
    sup[::2] = 1
    z = torch.zeros(V, d // 2, dtype=torch.uint8, device="cuda"), torch.full((V, d // 32), 127, dtype=torch.uint8, device="cuda")
    conf, arg, lse = al.lmhead_confidence_mx4(dev_bf16(H), al.lmhead_pack_weight_mx4(*z), V, suppress_eos=dev(sup), eos_id=0)
    assert np.array_equal(arg.cpu().numpy(), np.where(sup == 1, 1, 0))
    assert np.array_equal(conf.cpu().numpy(), (np.float32(1) / np.where(sup == 1, V - 1, V).astype(np.float32)))
    Wf = g.standard_normal((V, d)) * 0.05
    Hn = np.zeros((N, d), np.float32)
    for n in range(N):
        Hn[n, n % d] = 1.0
        for v in (100 + 7 * n, 2000 - 11 * n):
            Wf[v] = 0
            Wf[v, n % d] = 4.0
    import synth
    codes, scales = oracle.mx4.quantize(Wf)
    W = al.lmhead_pack_weight_mx4(dev(codes), dev(scales))
    _, arg, _ = al.lmhead_confidence_mx4(dev_bf16(synth.f32_to_bf16_bits(Hn)), W, V)
    assert np.array_equal(arg.cpu().numpy(), 100 + 7 * np.arange(N))


def test_agrees_with_the_bf16_head():
    """The 4-bit values as a bf16 weight: the same logits, sums in another order."""
    N, n_rows, d, V = 77, 90, 4096, 9000
    H, codes, scales, rows, sup = _inputs(N, n_rows, d, V)
    h, r, s = dev_bf16(H), dev(rows), dev(sup)
    c, sc = dev(codes), dev(scales)
    a = al.lmhead_confidence(h, al.mx4_dequantize(c, sc), row_idx=r, suppress_eos=s, eos_id=2)
    b = al.lmhead_confidence_mx4(h, al.lmhead_pack_weight_mx4(c, sc), V, row_idx=r, suppress_eos=s, eos_id=2)
    W, hr = oracle.mx4.values(codes, scales), f64(H)[rows]
    bz, bl, bc = lmhead_bounds(hr, W, b[2].cpu().numpy().astype(np.float64))
    assert (np.abs(a[2].cpu().numpy() - b[2].cpu().numpy()) <= 2 * bl).all()
    assert (np.abs(a[0].cpu().numpy() - b[0].cpu().numpy()) <= 2 * bc * b[0].cpu().numpy()).all()
    assert (a[1] == b[1]).float().mean() > 0.95


@pytest.mark.parametrize("case", [(77, 80, 416, 3000, 2), (300, 310, 64, 513, 2), (1, 3, 1024, 20000, 1)], ids=str)
def test_repeatable_workspace_and_guards(case):
    """The same bits again, on a workspace of the exact size, outputs longer than N left alone behind it."""
    N, n_rows, d, V, eos = case
    H, codes, scales, rows, sup = _inputs(N, n_rows, d, V)
    W = al.lmhead_pack_weight_mx4(dev(codes), dev(scales))
    h, r, s = dev_bf16(H), dev(rows), dev(sup)
    want = al.lmhead_confidence_mx4(h, W, V, row_idx=r, suppress_eos=s, eos_id=eos)
    need = al.lmhead_confidence_mx4_workspace_size(N, d, V)
    for fill in (0xFF, 0x00):
        ws = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
        conf, arg, lse = (torch.full((N + 8,), 3, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.float32))
        al.lmhead_confidence_mx4(h, W, V, row_idx=r, suppress_eos=s, eos_id=eos, conf=conf, argmax=arg, lse=lse,
                                 workspace=ws[:need])
        assert bool((ws[need:] == fill).all())
        for x, y in zip((conf, arg, lse), want):
            assert torch.equal(x[:N], y) and bool((x[N:] == 3).all())


def test_no_rows():
    codes, scales = torch.zeros(100, 32, dtype=torch.uint8, device="cuda"), torch.zeros(100, 2, dtype=torch.uint8, device="cuda")
    W = al.lmhead_pack_weight_mx4(codes, scales)
    conf, arg, lse = al.lmhead_confidence_mx4(torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda"), W, 100,
                                              row_idx=torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert conf.shape == arg.shape == lse.shape == (0,)
