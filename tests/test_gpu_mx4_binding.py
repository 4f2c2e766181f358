"""Native marshalling of the 4-bit calls against the Python checks: accepted forms give the same
results both ways, what one refuses the other refuses with the same message."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_08411_amd as al
from gpu_util import dev_bf16
from mx4_util import bf16_normal, dev, random_cache
from test_gpu_fast_call import _both, _same, _Subclass

pytestmark = pytest.mark.gpu
u8, i32 = torch.uint8, torch.int32


def _attn_args(n_ref=0):
    g = np.random.default_rng(6)
    L, B, P, cap, Hq, Hkv, D = 3, 5, 70, 80, 6, 2, 64
    c, s = random_cache(g, Hkv, cap, D)
    mk = lambda *shape: dev_bf16(bf16_normal(g, *shape))
    a = dict(q=mk(L * B, Hq, D), k_lane=mk(L * B, Hkv, D), v_lane=mk(L * B, Hkv, D), kv_codes=dev(c), kv_scales=dev(s),
             P=P, parent=np.array([-1, 0, 0], np.int32), B=B)
    if n_ref:
        a.update(refresh_idx=torch.arange(n_ref, dtype=i32, device="cuda") * 3, q_ref=mk(n_ref, Hq, D),
                 k_ref=mk(n_ref, Hkv, D), v_ref=mk(n_ref, Hkv, D))
    return a


ATTN = {   # form: (change, what the native module makes of it)
    "plain": (lambda a: a, "native"),
    "list": (lambda a: dict(a, parent=[-1, 0, 0]), "native"),
    "int64": (lambda a: dict(a, parent=a["parent"].astype(np.int64)), "declined"),
    "numpy P": (lambda a: dict(a, P=np.int64(70)), "declined"),
    "no prefix": (lambda a: dict(a, P=0) if "q_ref" not in a else a, "native"),
    "no lse": (lambda a: dict(a, want_lse=False), "native"),
    "outputs": (lambda a: dict(a, o=torch.empty_like(a["q"])), "native"),
    "subclass": (lambda a: dict(a, q=a["q"].as_subclass(_Subclass)), "declined"),
    "workspace": (lambda a: dict(a, workspace=torch.empty(1 << 20, dtype=u8, device="cuda")), "native"),
    "bad tree": (lambda a: dict(a, parent=[0, 0, 0]), "raised"),
    "long prefix": (lambda a: dict(a, P=81), "declined"),
    "negative prefix": (lambda a: dict(a, P=-1), "declined"),
    "dtype": (lambda a: dict(a, kv_codes=a["kv_codes"].int()), "declined"),
    "scales": (lambda a: dict(a, kv_scales=a["kv_scales"][:, :, :79]), "declined"),
    "layout": (lambda a: dict(a, kv_codes=a["kv_codes"].transpose(0, 1).contiguous().transpose(0, 1)), "declined"),
    "cpu": (lambda a: dict(a, v_lane=a["v_lane"].cpu()), "declined"),
    "missing": (lambda a: dict(a, v_lane=None), "declined"),
    "shape": (lambda a: dict(a, k_lane=a["k_lane"][:-1]), "declined"),
}


@pytest.mark.parametrize("form", ATTN)
@pytest.mark.parametrize("n_ref", [0, 7])
def test_attention_forms(form, n_ref, monkeypatch):
    change, how = ATTN[form]
    a = change(_attn_args(n_ref))
    _same(_both(monkeypatch, lambda: al.lane_attn_forward_kv4(**a), how))


def test_refresh_only(monkeypatch):
    a = dict(_attn_args(7), q=None, k_lane=None, v_lane=None, parent=[])
    _same(_both(monkeypatch, lambda: al.lane_attn_forward_kv4(**a)))


def _lm_args():
    g = np.random.default_rng(4)
    c, s = oracle.mx4.quantize(bf16_normal(g, 300, 96).astype(np.float64) / 1e4)
    return dict(hidden=dev_bf16(bf16_normal(g, 9, 96)), W_mx4=al.lmhead_pack_weight_mx4(dev(c), dev(s)), V=300,
                row_idx=torch.tensor([4, 0, 8], dtype=i32, device="cuda"), eos_id=2,
                suppress_eos=torch.tensor([1, 0, 1], dtype=u8, device="cuda"))


LM = {
    "plain": (lambda a: a, "native"),
    "all rows": (lambda a: dict(a, row_idx=None, suppress_eos=None), "native"),
    "outputs": (lambda a: dict(a, conf=torch.empty(5, device="cuda"), want_lse=False), "native"),
    "no rows": (lambda a: dict(a, row_idx=a["row_idx"][:0]), "declined"),
    "numpy V": (lambda a: dict(a, V=np.int64(300)), "declined"),
    "bf16 weight": (lambda a: dict(a, W_mx4=a["W_mx4"].view(torch.bfloat16)), "declined"),
    "short weight": (lambda a: dict(a, W_mx4=a["W_mx4"][:-1]), "declined"),
    "eos": (lambda a: dict(a, eos_id=300), "raised"),
    "width": (lambda a: dict(a, hidden=a["hidden"][:, :72].contiguous()), "declined"),
    "small workspace": (lambda a: dict(a, workspace=torch.empty(16, dtype=u8, device="cuda")), "raised"),
}


@pytest.mark.parametrize("form", LM)
def test_lmhead_forms(form, monkeypatch):
    change, how = LM[form]
    a = change(_lm_args())
    got = _both(monkeypatch, lambda: [x if x is None else x[:len(a["row_idx"]) if a["row_idx"] is not None else 9]
                                      for x in al.lmhead_confidence_mx4(**a)], how)
    _same(got)


@pytest.mark.parametrize("form,how", [("plain", "native"), ("empty", "native"), ("outputs", "native"), ("one row", "native"),
                                      ("dtype", "declined"), ("width", "declined"), ("strided", "declined"),
                                      ("outputs' shape", "declined"), ("cpu", "declined")])
def test_quantizer_forms(form, how, monkeypatch):
    g = np.random.default_rng(2)
    x = dev_bf16(bf16_normal(g, 3, 5, 128))
    a = dict(x=x)
    if form == "empty":
        a["x"] = x[:0]
    elif form == "outputs":
        a.update(codes=torch.empty(3, 5, 64, dtype=u8, device="cuda"), scales=torch.empty(3, 5, 4, dtype=u8, device="cuda"))
    elif form == "one row":
        a["x"] = x[0, 0]
    elif form == "dtype":
        a["x"] = x.float()
    elif form == "width":
        a["x"] = x[..., :48].contiguous()
    elif form == "strided":
        a["x"] = x[..., :64]
    elif form == "outputs' shape":
        a["codes"] = torch.empty(15, 64, dtype=u8, device="cuda")
    elif form == "cpu":
        a["x"] = x.cpu()
    _same(_both(monkeypatch, lambda: al.mx4_quantize(**a), how))
    if how == "native":
        c, s = al.mx4_quantize(a["x"])
        _same(_both(monkeypatch, lambda: [al.mx4_dequantize(c, s)]))
        _same(_both(monkeypatch, lambda: [al.mx4_dequantize(c, s[..., :-1])], "declined"))


@pytest.mark.parametrize("form,how", [("rows", "native"), ("start", "native"), ("none", "native"), ("past the end", "raised"),
                                      ("index dtype", "declined"), ("heads", "declined"), ("numpy start", "declined")])
def test_store_forms(form, how, monkeypatch):
    g = np.random.default_rng(2)
    c, s = random_cache(g, 2, 40, 64)
    k, v = dev_bf16(bf16_normal(g, 6, 2, 64)), dev_bf16(bf16_normal(g, 6, 2, 64))
    a = dict(k=k, v=v, start=3)
    if form in ("rows", "index dtype"):
        a["row_idx"] = torch.tensor([5, 0, 39, -1, 40, 7], dtype=i32 if form == "rows" else torch.int64, device="cuda")
    elif form == "none":
        a.update(k=k[:0], v=v[:0])
    elif form == "past the end":
        a["start"] = 35
    elif form == "heads":
        a["v"] = v[:, :1].contiguous()
    elif form == "numpy start":
        a["start"] = np.int32(3)

    def call():
        codes, scales = dev(c), dev(s)
        al.kv4_store(kv_codes=codes, kv_scales=scales, **a)
        return [codes, scales]
    _same(_both(monkeypatch, call, how))


def test_a_capture_needs_a_workspace():
    a = _lm_args()
    graph = torch.cuda.CUDAGraph()
    al.lmhead_confidence_mx4(**a)
    torch.cuda.synchronize()
    with pytest.raises(al.AsyncLaneError, match="pass workspace="):
        with torch.cuda.graph(graph):
            al.lmhead_confidence_mx4(**a)


def test_outputs_are_ordinary_tensors():
    """New outputs: of the caching allocator, on the input's device, inference tensors where inputs would be;
    also beside an input whose storage has no allocator."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn((3, 64, 256), generator=g, device="cuda").bfloat16()
    codes, scales = al.mx4_quantize(x)
    before = torch.cuda.memory_allocated()
    c, s = al.mx4_quantize(x)
    y = al.mx4_dequantize(c, s)
    assert torch.cuda.memory_allocated() - before >= c.nbytes + s.nbytes + y.nbytes
    for t, shape, dtype in ((c, (3, 64, 128), torch.uint8), (s, (3, 64, 8), torch.uint8), (y, (3, 64, 256), torch.bfloat16)):
        assert t.shape == shape and t.dtype == dtype and t.device == x.device
        assert t.is_contiguous() and t.is_leaf and not t.requires_grad and not t.is_inference()
    y.requires_grad_()
    (y.float() ** 2).sum().backward()
    assert torch.equal(y.grad, (2 * y.detach().float()).bfloat16())
    with torch.inference_mode():
        assert all(t.is_inference() for t in al.mx4_quantize(x))
    shared = torch.utils.dlpack.from_dlpack(torch.utils.dlpack.to_dlpack(x))
    for t, want in zip(al.mx4_quantize(shared), (codes, scales)):
        assert torch.equal(t, want)
    W = al.lmhead_pack_weight_mx4(*al.mx4_quantize(x[0]))
    conf, arg, lse = al.lmhead_confidence_mx4(x[1], W, 64)
    assert conf.dtype == lse.dtype == torch.float32 and arg.dtype == torch.int32
    assert conf.shape == arg.shape == lse.shape == (64,)
    del c, s, y
    torch.cuda.synchronize()
