"""Every kernel instance of the 4-bit head and every plan of the 4-bit attention (test_mx4_plans_host.py
checks that the cases reach them all), against torch in 64 bits, within the bounds of mx4_util."""
import numpy as np
import pytest
import torch

import paper_2606_08411_amd as al
from mx4_util import EPS32, EPSB

pytestmark = pytest.mark.gpu

LM_CASES = [  # N, d, V
    (1, 32, 1), (1, 128, 1), (17, 512, 1), (1, 960, 1), (1, 1024, 1), (19, 2944, 1), (17, 32, 1), (18, 128, 1),
    (38, 256, 1), (18, 800, 1), (17, 896, 1), (40, 896, 1), (33, 32, 1), (34, 128, 1), (162, 128, 32972),
    (173, 960, 3017), (50, 1792, 17618), (166, 1152, 3385), (69, 32, 36294), (72, 128, 54835), (221, 128, 16403),
    (788, 1696, 1), (79, 1792, 15245), (390, 1280, 10), (87, 32, 40994), (85, 128, 66503), (249, 128, 16991),
    (906, 2016, 1), (85, 1920, 28057), (954, 2304, 1), (65, 32, 1), (75, 128, 1), (171, 128, 1), (131, 32, 1),
    (134, 128, 1), (259, 128, 1), (387, 32, 1), (176, 128, 22444), (389, 128, 1),
    (1417, 32, 516), (21, 128, 34189), (20, 1152, 1), (38, 1280, 1), (42, 128, 34714), (99, 2720, 9429), (57, 2944, 17378),
    (109, 3200, 9577), (75, 1216, 27701), (71, 1280, 31131), (129, 1536, 13628), (244, 2720, 9002), (89, 3456, 22568),
    (176, 3584, 13161), (828, 128, 2416), (134, 32, 22397), (131, 128, 25307), (200, 32, 23592), (207, 256, 22710),
    (403, 128, 15153),
    # several rounds of workgroups, units shared out unevenly, K groups of every remainder
    (16, 1024, 140001), (40, 1152, 17000), (77, 1408, 70000), (100, 1056, 100003), (150, 640, 66000), (420, 384, 40000),
    (12, 4224, 9000), (30, 4128, 9001), (8, 8192, 777), (300, 2080, 12345),
]


@pytest.mark.parametrize("case", LM_CASES, ids=[str(c) for c in LM_CASES])
def test_lmhead_instance(case):
    N, d, V = case
    g = torch.Generator(device="cuda")
    g.manual_seed(N * 1000003 + d * 1009 + V)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    codes, scales = al.mx4_quantize((rnd(V, d) / d ** 0.5).bfloat16())
    H = (rnd(N + 3, d) * (1 + 2 * torch.rand((N + 3, 1), generator=g, device="cuda"))).bfloat16()
    rows = torch.randperm(N + 3, generator=g, device="cuda")[:N].to(torch.int32)
    sup = (torch.rand(N, generator=g, device="cuda") < 0.5).to(torch.uint8)
    eos = V // 3 if V > 1 else -1
    conf, arg, lse = al.lmhead_confidence_mx4(H, al.lmhead_pack_weight_mx4(codes, scales), V, row_idx=rows,
                                              suppress_eos=sup, eos_id=eos)
    h = H[rows.long()].double()
    W = al.mx4_dequantize(codes, scales)
    z = torch.cat([torch.mm(h, w.double().t().contiguous()) for w in W.split(16384)], 1)
    if eos >= 0:
        z[sup.bool(), eos] = -np.inf
    top = z.topk(min(2, V), dim=1).values
    ref = torch.logsumexp(z, 1)
    bz = (d / 32 + 32) * EPS32 * h.norm(dim=1) * W.float().norm(dim=1).max().double()
    bl = bz + 100 * EPS32 + 4 * EPS32 * ref.abs()
    assert bool(((lse.double() - ref).abs() <= bl).all())
    want = torch.exp(top[:, 0] - ref)
    assert bool(((conf.double() - want).abs() <= (bz + bl + 8 * EPS32 * ref.abs()) * want).all())
    clear = top[:, 0] - top[:, 1] > 2 * bz if V > 1 else torch.ones(N, dtype=torch.bool, device="cuda")
    assert bool((arg.long() == z.argmax(1))[clear].all())
    assert bool((z.gather(1, arg.long()[:, None])[:, 0] >= top[:, 0] - 2 * bz).all())   # an id that is nearly the largest


ATTN_CASES = [  # L, B, P, Hq, Hkv, D, refreshed rows
    (1, 1, 1, 1, 1, 64, 0), (1, 1, 3104, 1, 1, 64, 0), (1, 1, 4058, 1, 1, 64, 0), (1, 1, 11147, 1, 1, 64, 0),
    (1, 1, 18164, 1, 1, 64, 0), (1, 3, 1, 7, 1, 64, 0), (33, 1, 944, 1, 1, 64, 0), (5, 1, 2850, 4, 1, 64, 1),
    (5, 1, 6241, 4, 1, 64, 0), (1, 32, 8341, 1, 1, 64, 0), (1, 32, 17124, 1, 1, 64, 0), (16, 3, 2, 224, 32, 64, 0),
    (33, 32, 140, 8, 2, 64, 0), (5, 16, 1, 512, 32, 64, 1), (33, 64, 325, 4, 4, 64, 0), (5, 64, 2500, 32, 32, 64, 0),
    (1, 1, 1, 1, 1, 128, 0), (1, 1, 3424, 2, 2, 128, 0), (1, 1, 5188, 1, 1, 128, 0), (1, 1, 9527, 1, 1, 128, 0),
    (1, 1, 18919, 1, 1, 128, 0), (1, 3, 1, 7, 1, 128, 0), (5, 1, 997, 4, 1, 128, 1), (5, 1, 2112, 4, 1, 128, 0),
    (5, 1, 4185, 4, 1, 128, 0), (1, 3, 9168, 7, 1, 128, 0), (5, 1, 16917, 4, 1, 128, 1), (16, 3, 2, 224, 32, 128, 0),
    (33, 16, 404, 16, 4, 128, 0), (5, 16, 2, 512, 32, 128, 0), (33, 16, 3299, 16, 4, 128, 0), (33, 16, 5865, 32, 32, 128, 1),
    (0, 1, 1299, 7, 1, 64, 1299), (0, 1, 2061, 8, 8, 64, 2061), (0, 1, 1108, 8, 2, 128, 1108), (0, 1, 1098, 8, 8, 128, 1098),
    (33, 16, 5326, 32, 2, 64, 0), (33, 64, 6960, 8, 2, 64, 1), (33, 16, 8968, 32, 8, 128, 0), (33, 100, 7597, 7, 1, 128, 1),
    (2, 100, 20675, 56, 8, 128, 0), (5, 64, 23356, 32, 32, 64, 0), (33, 16, 18507, 16, 4, 64, 0), (33, 64, 16255, 4, 4, 128, 0),
    (1, 1, 1800, 1, 1, 64, 0), (1, 1, 1810, 28, 4, 128, 0), (1, 1, 33001, 2, 2, 64, 0), (1, 32, 33005, 1, 1, 128, 0),
    (1, 3, 33003, 8, 2, 64, 0),
]


def _reference(q, k, v, visible):
    """softmax(q k^T / sqrt(D)) v in 64 bits, with |v| too; k, v [S][Hkv][D]."""
    Hq, g, scale = q.shape[1], q.shape[1] // k.shape[1], q.shape[2] ** -0.5
    o, a = (torch.empty(q.shape, dtype=torch.float64, device="cuda") for _ in "oa")
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device="cuda")
    for h in range(Hq):
        z = torch.mm(q[:, h].double().contiguous(), k[:, h // g].t().contiguous()) * scale
        if visible is not None:
            z.masked_fill_(~visible, -np.inf)
        lse[:, h] = torch.logsumexp(z, 1)
        p = torch.exp(z - lse[:, h:h + 1])
        o[:, h], a[:, h] = torch.mm(p, v[:, h // g].contiguous()), torch.mm(p, v[:, h // g].abs().contiguous())
    return o, a, lse


def _close(o, lse, ref, q, k):
    ro, ra, rl = ref
    D, n = q.shape[2], k.shape[0]
    e = 2 * D * EPS32 * D ** -0.5 * float(q.float().norm(dim=2).max()) * float(k.norm(dim=2).max())
    assert bool(((o.double() - ro).abs() <= 1.01 * (EPSB * ro.abs() + (EPSB + 4 * e + 2 * n * EPS32) * ra)).all())
    assert bool(((lse.double() - rl).abs() <= 2 * e + n * EPS32 + 8 * EPS32 * rl.abs().clamp(min=1)).all())


@pytest.mark.parametrize("case", ATTN_CASES, ids=[str(c) for c in ATTN_CASES])
def test_attention_plan(case):
    L, B, P, Hq, Hkv, D, n_ref = case
    g = torch.Generator(device="cuda")
    g.manual_seed(L * 7 + B * 31 + P * 1009 + Hq)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    codes, scales = al.mx4_quantize(rnd(2, Hkv, P + 3, D))
    scales[:, :, P:] = 255   # (NaN: never read)
    rng = np.random.default_rng(P)
    parent = [-1] + [int(rng.integers(-1, i)) for i in range(1, L)] if L else []
    q, kl, vl = (rnd(L * B, Hq, D), rnd(L * B, Hkv, D), rnd(L * B, Hkv, D)) if L else (None,) * 3
    ref = {}
    if n_ref:
        idx = torch.randperm(P, generator=g, device="cuda")[:n_ref].to(torch.int32)
        ref = dict(refresh_idx=idx, q_ref=rnd(n_ref, Hq, D), k_ref=rnd(n_ref, Hkv, D), v_ref=rnd(n_ref, Hkv, D))
    o, lse, o_ref, lse_ref = al.lane_attn_forward_kv4(q, kl, vl, codes, scales, P, parent, B, **ref)
    kv = al.mx4_dequantize(codes, scales)[:, :, :P].double()
    if n_ref:   # (the rows that the call quantised are those that the quantiser gives)
        for plane, x in enumerate((ref["k_ref"], ref["v_ref"])):
            assert torch.equal(kv[plane][:, idx.long()].transpose(0, 1), al.mx4_dequantize(*al.mx4_quantize(x)).double())
    k, v = kv[0].transpose(0, 1), kv[1].transpose(0, 1)
    if L:
        see = torch.eye(L, dtype=torch.bool)
        for i, j in enumerate(parent):
            if j >= 0:
                see[i] |= see[j]
        lanes = see.repeat_interleave(B, 0).repeat_interleave(B, 1).cuda()
        visible = torch.cat([torch.ones((L * B, P), dtype=torch.bool, device="cuda"), lanes], 1)
        ka, va = torch.cat([k, kl.double()]), torch.cat([v, vl.double()])
        _close(o, lse, _reference(q, ka, va, visible), q, ka)
    if n_ref:
        _close(o_ref, lse_ref, _reference(ref["q_ref"], k, v, None), ref["q_ref"], k)
