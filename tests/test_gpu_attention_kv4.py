"""lane_attn_forward_kv4 on the GPU against the fp64 oracle on the cache's values, within the bounds
derived in mx4_util.attention_bounds."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_08411_amd as al
import synth
from gpu_util import dev_bf16
from mx4_util import attention_bounds, bf16_normal, cache_rows, dev, f64, host_f64, random_cache

pytestmark = pytest.mark.gpu


def _step(case, seed=0):
    L, B, P, Hq, Hkv, D, tree, n_ref = case
    g = np.random.default_rng([seed, L, B, P, Hq, D, n_ref])
    cap = P + int(g.integers(0, 70))
    codes, scales = random_cache(g, Hkv, max(cap, 1), D)
    codes[:, :, P:], scales[:, :, P:] = 0x77, 255           # rows past the prefix: NaN, never read
    s = dict(q=bf16_normal(g, L * B, Hq, D), k=bf16_normal(g, L * B, Hkv, D), v=bf16_normal(g, L * B, Hkv, D),
             codes=codes, scales=scales, parent=synth.lane_tree(tree, L, seed, 4) if L else np.zeros(0, np.int32))
    if n_ref:
        s.update(idx=np.sort(g.choice(P, n_ref, replace=False)).astype(np.int32), q_ref=bf16_normal(g, n_ref, Hq, D),
                 k_ref=bf16_normal(g, n_ref, Hkv, D), v_ref=bf16_normal(g, n_ref, Hkv, D))
    return s


def _run(s, case, **more):
    L, B, P, _, _, _, _, n_ref = case
    c, sc = dev(s["codes"]), dev(s["scales"])
    lanes = [dev_bf16(s[x]) for x in "qkv"] if L else [None] * 3
    ref = dict(refresh_idx=dev(s["idx"]), q_ref=dev_bf16(s["q_ref"]), k_ref=dev_bf16(s["k_ref"]),
               v_ref=dev_bf16(s["v_ref"])) if n_ref else {}
    out = al.lane_attn_forward_kv4(*lanes, c, sc, P, list(s["parent"]), B, **ref, **more)
    torch.cuda.synchronize()
    return out, c, sc


def _check(s, case):
    L, B, P, Hq, Hkv, D, _, n_ref = case
    (o, lse, o_ref, lse_ref), c, sc = _run(s, case)
    codes, scales = s["codes"].copy(), s["scales"].copy()
    if n_ref:
        for plane, x in enumerate((s["k_ref"], s["v_ref"])):
            rc, rs = oracle.mx4.quantize(f64(x))
            codes[plane][:, s["idx"]], scales[plane][:, s["idx"]] = rc.transpose(1, 0, 2), rs.transpose(1, 0, 2)
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(sc.cpu().numpy(), scales)
    kp, vp = cache_rows(codes, scales, P)
    if L:
        q, k, v = f64(s["q"]), f64(s["k"]), f64(s["v"])
        ro, rl = oracle.attention.lane_attention_concat(q, k, v, kp, vp, s["parent"], B)
        ra, _ = oracle.attention.lane_attention_concat(q, k, np.abs(v), kp, np.abs(vp), s["parent"], B)
        bo, bl = attention_bounds(ro, ra, rl, q, np.concatenate([kp, k]), D, P + L * B)
        assert (np.abs(host_f64(o) - ro) <= bo).all()
        assert (np.abs(host_f64(lse) - rl) <= bl).all()
    if n_ref:
        q = f64(s["q_ref"])
        ro, rl = oracle.attention.refresh_attention(q, kp, vp)
        ra, _ = oracle.attention.refresh_attention(q, kp, np.abs(vp))
        bo, bl = attention_bounds(ro, ra, rl, q, kp, D, P)
        assert (np.abs(host_f64(o_ref) - ro) <= bo).all()
        assert (np.abs(host_f64(lse_ref) - rl) <= bl).all()


CASES = [  # L, B, P, Hq, Hkv, D, tree, refreshed rows
    # one token; a prefix of nothing, of one row, to both sides of a key tile
    (1, 1, 0, 1, 1, 64, "linear", 0), (1, 1, 1, 1, 1, 128, "linear", 0), (1, 1, 63, 4, 2, 64, "linear", 0),
    (1, 1, 64, 4, 4, 128, "linear", 0), (1, 1, 65, 7, 1, 128, "linear", 0), (1, 1, 700, 28, 4, 128, "linear", 0),
    (1, 1, 5000, 8, 8, 64, "linear", 0), (1, 1, 4097, 32, 1, 128, "linear", 0), (1, 1, 300, 128, 1, 64, "linear", 0),
    # single-token lanes: one key tile holds many blocks, one query tile many lanes
    (64, 1, 100, 4, 4, 64, "random", 0), (64, 1, 100, 6, 2, 128, "linear", 0), (33, 1, 0, 1, 1, 64, "random", 0),
    (64, 1, 2000, 8, 1, 128, "random", 3),
    # odd blocks; blocks that straddle tiles; blocks of several tiles
    (3, 5, 33, 4, 2, 64, "random", 0), (13, 7, 129, 6, 6, 128, "random", 0), (5, 48, 200, 28, 4, 128, "random", 20),
    (7, 33, 64, 4, 4, 64, "forest", 0), (2, 130, 10, 2, 1, 128, "fork", 1), (1, 1024, 70, 2, 2, 64, "linear", 0),
    (4, 32, 512, 8, 8, 128, "linear", 0), (8, 32, 320, 14, 2, 128, "random", 32), (64, 16, 65, 4, 4, 64, "random", 0),
    (32, 64, 128, 2, 2, 128, "random", 12), (60, 17, 333, 6, 2, 64, "linear", 0),
    # key splits: few rows over long prefixes, some starting inside the lane tiles
    (2, 32, 4097, 4, 4, 64, "fork", 0), (9, 16, 3000, 4, 1, 128, "random", 0), (40, 16, 100, 2, 1, 64, "random", 7),
    # refresh only: one row, odd counts, every row
    (0, 1, 1, 4, 4, 64, "linear", 1), (0, 1, 333, 14, 2, 128, "linear", 5), (0, 1, 257, 8, 8, 64, "linear", 257),
    (0, 1, 1000, 8, 2, 128, "linear", 999),
]


@pytest.mark.parametrize("case", CASES, ids=[str(c) for c in CASES])
def test_against_the_oracle(case):
    _check(_step(case), case)


@pytest.mark.parametrize("scale", [0.25, 3.0])
def test_scale(scale):
    case = (3, 16, 100, 4, 2, 64, "random", 0)
    s = _step(case)
    (o, lse, _, _), _, _ = _run(s, case, scale=scale)
    kp, vp = cache_rows(s["codes"], s["scales"], 100)
    q, k, v = f64(s["q"]), f64(s["k"]), f64(s["v"])
    ro, rl = oracle.attention.lane_attention_concat(q, k, v, kp, vp, s["parent"], 16, scale=scale)
    ra, _ = oracle.attention.lane_attention_concat(q, k, np.abs(v), kp, np.abs(vp), s["parent"], 16, scale=scale)
    bo, bl = attention_bounds(ro, ra, rl, q * scale * 8, np.concatenate([kp, k]), 64, 148)   # (the bound's scale: 1/8)
    assert (np.abs(host_f64(o) - ro) <= bo).all() and (np.abs(host_f64(lse) - rl) <= bl).all()


def test_scores_of_unlike_size():
    """The running maximum moves far up and down along the keys; one key takes nearly all."""
    case = (1, 4, 400, 2, 2, 64, "linear", 0)
    s = _step(case)
    k = f64(bf16_normal(np.random.default_rng(4), 2, 2, 400, 64))
    k[0] *= np.exp(np.linspace(-3, 3, 400))[None, :, None] * np.where(np.arange(400) % 7 == 0, 5.0, 0.2)[None, :, None]
    s["codes"][:, :, :400], s["scales"][:, :, :400] = oracle.mx4.quantize(k)
    _check(s, case)


def test_long_cache_offsets_past_32_bits():
    """The last rows of a cache of more than 2^32 bytes of codes."""
    Hkv, cap, D = 8, 5_000_000, 128      # 8 heads x 5e6 rows x 64 bytes = 2.56e9 a plane
    codes = torch.zeros((2, Hkv, cap, D // 2), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((2, Hkv, cap, D // 32), dtype=torch.uint8, device="cuda")
    assert codes.numel() > 2 ** 32
    g = np.random.default_rng(2)
    T = 40
    k, v = bf16_normal(g, T, Hkv, D), bf16_normal(g, T, Hkv, D)
    al.kv4_store(dev_bf16(k), dev_bf16(v), codes, scales, start=cap - T)
    q = bf16_normal(g, 1, Hkv, D)
    o, lse, _, _ = al.lane_attn_forward_kv4(dev_bf16(q), dev_bf16(k[:1]), dev_bf16(v[:1]), codes, scales, cap, [-1], 1)
    torch.cuda.synchronize()
    for plane, x in enumerate((k, v)):
        rc, rs = oracle.mx4.quantize(f64(x))
        assert np.array_equal(codes[plane, :, cap - T:].cpu().numpy(), rc.transpose(1, 0, 2))
        assert np.array_equal(scales[plane, :, cap - T:].cpu().numpy(), rs.transpose(1, 0, 2))
    # cap - T zero keys (scale byte 0: values 0), the stored rows, the lane's own
    kk = np.concatenate([oracle.mx4.rounded(f64(k)), f64(k[:1])])
    vv = np.concatenate([oracle.mx4.rounded(f64(v)), f64(v[:1])])
    for h in range(Hkv):
        z = kk[:, h] @ f64(q)[0, h] / D ** 0.5
        total = (cap - T) + np.exp(z).sum()
        ref = (np.exp(z)[:, None] * vv[:, h]).sum(0) / total
        # about 1e-5, all of it from 41 keys: relative to the sum of their weights
        bound = 3 * 2.0 ** -8 * (np.exp(z)[:, None] * np.abs(vv[:, h])).sum(0) / total
        assert (np.abs(host_f64(o)[0, h] - ref) <= bound).all()
        assert abs(float(lse[0, h]) - np.log(total)) < 1e-3


@pytest.mark.parametrize("case", [(4, 32, 512, 8, 8, 128, "linear", 40), (1, 1, 4097, 28, 4, 128, "linear", 0)], ids=str)
def test_repeatable_and_workspace(case):
    """The same bits again, on a workspace of the exact size full of NaN."""
    L, B, P, Hq, Hkv, D, _, n_ref = case
    s = _step(case)
    need = al.lane_attn_kv4_workspace_size(L, B, P, Hq, Hkv, D, n_ref)
    a, _, _ = _run(s, case)
    for fill in (0xFF, 0x00):
        ws = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
        b, _, _ = _run(s, case, **(dict(workspace=ws[:need]) if need else {}))
        assert bool((ws[need:] == fill).all())
        for x, y in zip(a, b):
            assert x is None and y is None or torch.equal(x, y)


def test_outputs_given_and_guards():
    case = (3, 5, 70, 6, 2, 64, "random", 0)
    s = _step(case)
    want, _, _ = _run(s, case)
    n = 15 * 6 * 64
    ob = torch.full((n + 256,), 7.0, dtype=torch.bfloat16, device="cuda")
    lb = torch.full((90 + 64,), 7.0, device="cuda")
    got, _, _ = _run(s, case, o=ob[128:128 + n].view(15, 6, 64), lse=lb[32:122].view(15, 6))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert bool((ob[:128] == 7).all()) and bool((ob[128 + n:] == 7).all())
    assert bool((lb[:32] == 7).all()) and bool((lb[122:] == 7).all())
    none, _, _ = _run(s, case, want_lse=False)
    assert none[1] is None and torch.equal(none[0], want[0])


def test_refresh_index_outside_the_prefix_is_left_out():
    case = (1, 4, 100, 2, 2, 64, "linear", 4)
    s = _step(case)
    s["idx"] = np.array([5, -1, 100, 99], np.int32)
    _, c, sc = _run(s, case)
    codes, scales = s["codes"].copy(), s["scales"].copy()
    for plane, x in enumerate((s["k_ref"], s["v_ref"])):
        rc, rs = oracle.mx4.quantize(f64(x))
        for r in (0, 3):
            codes[plane][:, s["idx"][r]], scales[plane][:, s["idx"][r]] = rc[r], rs[r]
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(sc.cpu().numpy(), scales)
