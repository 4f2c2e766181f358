"""The 4-bit operators on the host: the oracle's format against loops and printed values, workspace
sizes, and the refusals of the C ABI and of the binding (nothing here launches a kernel)."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2606_08411_amd as al
from paper_2606_08411_amd import AsyncLaneError

bf16, u8, i32 = torch.bfloat16, torch.uint8, torch.int32


# ------------------------------------------------------------------- format
def test_codes_stand_for_their_values():
    codes = np.array([[0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE] + [0] * 8], np.uint8)
    want = [0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6] + [0.] * 16
    got = oracle.mx4.values(codes, np.array([[127]], np.uint8))[0]
    assert got.tolist() == want and np.signbit(got[8])
    assert oracle.mx4.values(codes, np.array([[130]], np.uint8))[0, 7] == 48.0
    assert oracle.mx4.values(codes, np.array([[0]], np.uint8))[0, 1] == 2.0 ** -128
    assert np.isnan(oracle.mx4.values(codes, np.array([[255]], np.uint8))).all()


@pytest.mark.parametrize("x,code", [(0.25, 0), (0.26, 1), (0.75, 2), (0.74, 1), (1.25, 2), (1.75, 4),
                                    (2.5, 4), (2.51, 5), (3.5, 6), (5.0, 6), (5.01, 7), (7.9, 7)])
def test_rounding_by_hand(x, code):
    """Ties go to the even code; what lies above 6 scales becomes 6 (top 7.9: scale 1)."""
    b = np.zeros(32)
    b[0], b[1], b[2] = 7.9, x, -x
    codes, scales = oracle.mx4.quantize(b)
    assert scales.tolist() == [127]
    assert codes[0] >> 4 == code and codes[1] & 15 == code + 8


@pytest.mark.parametrize("top,s", [(4.0, 127), (7.99, 127), (8.0, 128), (3.99, 126), (2.0 ** -125, 0),
                                   (2.0 ** -126, 0), (2.0 ** -133, 0), (0.0, 0), (2.0 ** 127, 252),
                                   (np.inf, 255), (np.nan, 255)])
def test_scale_bytes(top, s):
    b = np.zeros(32)
    b[31] = -top
    codes, scales = oracle.mx4.quantize(b)
    assert scales.tolist() == [s]
    if s == 255:
        assert not codes.any()


def test_oracle_against_loops():
    g = np.random.default_rng(3)
    x = g.standard_normal((7, 96)) * np.exp(4 * g.standard_normal((7, 1)))
    got = oracle.mx4.rounded(x)
    for r in range(7):
        for b in range(3):
            blk = x[r, 32 * b:32 * b + 32]
            e = 2.0 ** (int(np.floor(np.log2(np.abs(blk).max()))) - 2)
            for i, v in enumerate(blk):
                best = min(oracle.mx4.MAGNITUDES, key=lambda m: abs(abs(v) / e - m))
                assert got[r, 32 * b + i] == np.sign(v) * best * e


# -------------------------------------------------------------- ABI refusals
FAKE = 1 << 20            # aligned non-null address, never dereferenced
ODD = FAKE + 8


def test_workspace_and_packed_sizes():
    assert al.lane_attn_kv4_workspace_size(4, 32, 512, 32, 32, 128) >= 0
    assert al.lane_attn_kv4_workspace_size(1, 1, 32769, 28, 4, 128) > 0
    assert al.lane_attn_kv4_workspace_size(1, 1, 100, 28, 5, 128) == 0       # Hq % Hkv
    assert al.lmhead_packed_weight_mx4_size(96, 70) == 1 * 2 * 4352
    assert al.lmhead_packed_weight_mx4_size(100, 70) == 0                    # d % 32
    assert al.lmhead_confidence_mx4_workspace_size(77, 4096, 126464) > 0
    assert al.lmhead_confidence_mx4_workspace_size(0, 4096, 126464) == 0
    assert al.lmhead_confidence_mx4_workspace_size(4, 40, 100) == 0


def test_abi_quantize_refuses():
    lib = al.library()
    for f, a in ((lib.mx4_quantize, lambda x, c, s, R=4, n=64: (x, R, n, c, s, None)),
                 (lib.mx4_dequantize, lambda x, c, s, R=4, n=64: (c, s, R, n, x, None))):
        assert f(*a(FAKE, FAKE, FAKE, n=48)) == -2
        assert f(*a(FAKE, FAKE, FAKE, n=0)) == -2
        assert f(*a(FAKE, FAKE, FAKE, R=-1)) == -2
        assert f(*a(FAKE, FAKE, FAKE, R=1 << 62)) == -2
        for bad in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None)):
            assert f(*a(*bad)) == -1
        for bad in ((ODD, FAKE, FAKE), (FAKE, ODD, FAKE), (FAKE, FAKE, ODD)):
            assert f(*a(*bad)) == -5
        assert f(*a(None, None, None, R=0)) == 0


def test_abi_store_refuses():
    lib = al.library()

    def f(k=FAKE, v=FAKE, idx=None, start=0, T=4, cap=16, Hkv=2, D=64, c=FAKE, s=FAKE):
        return lib.kv4_store(k, v, idx, start, T, cap, Hkv, D, c, s, None)
    for bad in (dict(T=-1), dict(cap=0), dict(Hkv=0), dict(Hkv=2000), dict(D=96), dict(start=-1),
                dict(start=13), dict(start=(1 << 31) - 1)):
        assert f(**bad) == -2, bad
    for key in ("k", "v", "c", "s"):
        assert f(**{key: None}) == -1
        assert f(**{key: ODD}) == -5
    assert f(idx=FAKE + 2) == -5
    assert f(T=0) == 0


def test_abi_attention_refuses():
    lib = al.library()

    def f(parent=(-1, 0), L=2, B=3, P=64, cap=64, Hq=4, Hkv=2, D=64, q=FAKE, kl=FAKE, c=FAKE, s=FAKE, o=FAKE,
          lse=None, scale=0.0, n_ref=0, idx=None, ref=FAKE, ws=None, wsb=0):
        par = np.asarray(parent, np.int32)
        return lib.lane_attn_forward_kv4(q, kl, kl, c, s, cap, par.ctypes.data_as(ctypes.c_void_p) if L else None,
                                         L, B, P, Hq, Hkv, D, scale, idx, n_ref, ref, ref, ref, ref, None, o, lse,
                                         ws, wsb, None)
    for bad in (dict(B=0), dict(B=1025), dict(P=-1), dict(cap=63), dict(D=32), dict(Hq=5), dict(Hq=0),
                dict(Hq=258), dict(L=65), dict(L=-1), dict(L=0), dict(n_ref=65, idx=FAKE), dict(n_ref=-1),
                dict(scale=float("nan")), dict(scale=float("inf"))):
        assert f(**bad) == -2, bad
    for key in ("q", "kl", "c", "s", "o"):
        assert f(**{key: None}) == -1, key
        assert f(**{key: ODD}) == -5, key
    assert f(lse=FAKE + 2) == -5
    assert f(n_ref=2, idx=None) == -1
    assert f(n_ref=2, idx=FAKE, ref=None) == -1
    assert f(n_ref=2, idx=FAKE + 2) == -5
    assert f(parent=(-1, 1)) == -3 and f(parent=(-2, 0)) == -3
    need = al.lane_attn_kv4_workspace_size(1, 1, 4096, 4, 2, 64)
    assert need > 0
    long = dict(parent=(-1,), L=1, B=1, P=4096, cap=4096)
    assert f(**long) == -1
    assert f(**long, ws=FAKE, wsb=need - 1) == -4
    assert f(**long, ws=ODD, wsb=need) == -5


def test_abi_lmhead_refuses():
    lib = al.library()

    def f(h=FAKE, n_rows=8, idx=None, N=8, W=FAKE, d=64, V=100, sup=None, eos=-1, conf=FAKE, arg=FAKE, lse=None,
          ws=FAKE, wsb=1 << 30):
        return lib.lmhead_confidence_mx4(h, n_rows, idx, N, W, d, V, sup, eos, conf, arg, lse, ws, wsb, None)
    for bad in (dict(d=40), dict(d=0), dict(V=0), dict(N=9), dict(n_rows=-1), dict(eos=100), dict(eos=-2),
                dict(V=1, eos=0, sup=FAKE)):
        assert f(**bad) == -2, bad
    for key in ("h", "W", "conf", "arg", "ws"):
        assert f(**{key: None}) == -1, key
    for key in ("h", "W", "ws"):
        assert f(**{key: ODD}) == -5, key
    assert f(wsb=al.lmhead_confidence_mx4_workspace_size(8, 64, 100) - 1) == -4
    assert f(N=0) == 0
    p = lambda c=FAKE, s=FAKE, d=64, V=100, o=FAKE, n=1 << 30: lib.lmhead_pack_weight_mx4(c, s, d, V, o, n, None)
    assert p(d=40) == -2 and p(V=0) == -2 and p(c=None) == -1 and p(s=None) == -1 and p(o=None) == -1
    assert p(c=ODD) == -5 and p(o=ODD) == -5 and p(n=al.lmhead_packed_weight_mx4_size(64, 100) - 1) == -4


# ---------------------------------------------------------- binding refusals
def _cache(Hkv=2, cap=64, D=64):
    return torch.zeros(2, Hkv, cap, D // 2, dtype=u8), torch.zeros(2, Hkv, cap, D // 32, dtype=u8)


def _attn_args(L=2, B=5, P=32, Hq=4, Hkv=2, D=64):
    c, s = _cache(Hkv, 64, D)
    return dict(q=torch.zeros(L * B, Hq, D, dtype=bf16), k_lane=torch.zeros(L * B, Hkv, D, dtype=bf16),
                v_lane=torch.zeros(L * B, Hkv, D, dtype=bf16), kv_codes=c, kv_scales=s, P=P, parent=[-1, 0], B=B)


@pytest.mark.parametrize("key,bad,msg", [
    ("q", torch.zeros(10, 4, 64), "q: dtype"), ("q", torch.zeros(9, 4, 64, dtype=bf16), "q:"),
    ("q", None, "q: a tensor"), ("k_lane", torch.zeros(10, 4, 64, dtype=bf16), "k_lane: shape"),
    ("v_lane", torch.zeros(10, 2, 64, dtype=torch.float16), "v_lane: dtype"),
    ("kv_codes", torch.zeros(2, 2, 64, 32, dtype=torch.int8), "kv_codes: dtype"),
    ("kv_codes", torch.zeros(2, 64, 32, dtype=u8), "kv_codes:"),
    ("kv_codes", torch.zeros(3, 2, 64, 32, dtype=u8), "kv_codes:"),
    ("kv_scales", torch.zeros(2, 2, 63, 2, dtype=u8), "kv_scales: shape"),
    ("P", 65, "P:"), ("P", -1, "P:"), ("o", torch.zeros(10, 4, 64), "o: dtype"),
    ("lse", torch.zeros(10, 3), "lse: shape"), ("workspace", "no tensor", "workspace|device tensor"),
])
def test_attention_rejects(key, bad, msg):
    a = _attn_args()
    a[key] = bad
    with pytest.raises(AsyncLaneError, match=msg):
        al.lane_attn_forward_kv4(**a)


def test_attention_refresh_rejects():
    ref = dict(refresh_idx=torch.zeros(3, dtype=torch.int64), q_ref=torch.zeros(3, 4, 64, dtype=bf16),
               k_ref=torch.zeros(3, 2, 64, dtype=bf16), v_ref=torch.zeros(3, 2, 64, dtype=bf16))
    with pytest.raises(AsyncLaneError, match="refresh_idx: dtype"):
        al.lane_attn_forward_kv4(**_attn_args(), **ref)
    ref["refresh_idx"] = torch.zeros(3, dtype=i32)
    with pytest.raises(AsyncLaneError, match="device tensor expected"):
        al.lane_attn_forward_kv4(**_attn_args(), **ref)
    ref["k_ref"] = torch.zeros(3, 4, 64, dtype=bf16)
    with pytest.raises(AsyncLaneError, match="k_ref: shape"):
        al.lane_attn_forward_kv4(**_attn_args(), **ref)
    with pytest.raises(AsyncLaneError, match="no lanes"):
        c, s = _cache()
        al.lane_attn_forward_kv4(None, None, None, c, s, 3, [], 1)


@pytest.mark.parametrize("x", [torch.zeros(4, 64), torch.zeros(4, 48, dtype=bf16), torch.zeros(4, 0, dtype=bf16),
                               torch.tensor(1.0, dtype=bf16), torch.zeros(4, 64, dtype=bf16)])
def test_quantize_rejects(x):
    """(The last is well-formed but on the host.)"""
    with pytest.raises(AsyncLaneError):
        al.mx4_quantize(x)


@pytest.mark.parametrize("c,s", [(torch.zeros(4, 32, dtype=u8), torch.zeros(4, 1, dtype=u8)),
                                 (torch.zeros(4, 24, dtype=u8), torch.zeros(4, 1, dtype=u8)),
                                 (torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 2, dtype=u8)),
                                 (torch.zeros(4, 32, dtype=u8), torch.zeros(4, 2, dtype=bf16)),
                                 (torch.zeros(4, 32, dtype=u8), torch.zeros(4, 2, dtype=u8))])
def test_dequantize_rejects(c, s):
    with pytest.raises(AsyncLaneError):
        al.mx4_dequantize(c, s)
    with pytest.raises(AsyncLaneError):
        al.lmhead_pack_weight_mx4(c, s)


@pytest.mark.parametrize("key,bad", [("k", torch.zeros(3, 4, 64, dtype=bf16)), ("k", torch.zeros(3, 2, 64)),
                                     ("v", torch.zeros(4, 2, 64, dtype=bf16)), ("row_idx", torch.zeros(3)),
                                     ("row_idx", torch.zeros(2, dtype=i32)), ("kv_codes", torch.zeros(3)),
                                     ("kv_scales", torch.zeros(2, 2, 64, 4, dtype=u8)), (None, None)])
def test_store_rejects(key, bad):
    c, s = _cache()
    a = dict(k=torch.zeros(3, 2, 64, dtype=bf16), v=torch.zeros(3, 2, 64, dtype=bf16), kv_codes=c, kv_scales=s,
             row_idx=torch.zeros(3, dtype=i32))
    if key:
        a[key] = bad
    with pytest.raises(AsyncLaneError):
        al.kv4_store(**a)


@pytest.mark.parametrize("key,bad,msg", [
    ("hidden", torch.zeros(8, 64), "hidden: dtype"), ("hidden", torch.zeros(8, 40, dtype=bf16), "no packed layout"),
    ("W_mx4", torch.zeros(8703, dtype=u8), "W_mx4:"), ("W_mx4", torch.zeros(8704, dtype=bf16), "W_mx4: dtype"),
    ("row_idx", torch.zeros(8, dtype=torch.int64), "row_idx: dtype"), ("conf", torch.zeros(7), "conf:"),
    ("suppress_eos", torch.zeros(8, dtype=torch.bool), "suppress_eos: dtype"), ("V", 0, "no packed layout"),
    (None, None, "device tensor expected")])
def test_lmhead_rejects(key, bad, msg):
    a = dict(hidden=torch.zeros(8, 64, dtype=bf16), W_mx4=torch.zeros(8704, dtype=u8), V=100)
    if key:
        a[key] = bad
    with pytest.raises(AsyncLaneError, match=msg):
        al.lmhead_confidence_mx4(**a)
