"""New outputs of natively marshalled calls beside torch's modes: what watches torch's allocations sees them."""
import numpy as np
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

import oracle
import paper_2606_08411_amd as al
from gpu_util import dev_bf16
from mx4_util import bf16_normal, dev, random_cache

pytestmark = pytest.mark.gpu


class _Made(TorchDispatchMode):
    """Shapes and types of what empty.memory_format makes."""

    def __init__(self):
        super().__init__()
        self.made = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if func is torch.ops.aten.empty.memory_format:
            self.made.append((tuple(out.shape), out.dtype))
        return out


def _calls():
    """name: (call, its outputs' shapes and types)"""
    g = np.random.default_rng(3)
    h, W = dev_bf16(bf16_normal(g, 9, 96)), dev_bf16(bf16_normal(g, 300, 96))
    W4 = al.lmhead_pack_weight_mx4(*al.mx4_quantize(W))
    Wp = al.lmhead_pack_weight(W)
    head = [((9,), torch.float32), ((9,), torch.int32), ((9,), torch.float32)]
    c, s = (dev(x) for x in random_cache(g, 2, 70, 64))
    q, k, v = (dev_bf16(bf16_normal(g, 15, n, 64)) for n in (6, 2, 2))
    ref = dict(refresh_idx=torch.tensor([3, 1], dtype=torch.int32, device="cuda"), q_ref=q[:2], k_ref=k[:2], v_ref=v[:2])
    attn = [((15, 6, 64), torch.bfloat16), ((15, 6), torch.float32), ((2, 6, 64), torch.bfloat16), ((2, 6), torch.float32)]
    codes, scales = al.mx4_quantize(W)
    u8 = torch.uint8
    return {
        "lmhead": (lambda: al.lmhead_confidence(h, W), head),
        "lmhead_packed": (lambda: al.lmhead_confidence_packed(h, Wp, 300), head),
        "lmhead_mx4": (lambda: al.lmhead_confidence_mx4(h, W4, 300), head),
        "attn_kv4": (lambda: al.lane_attn_forward_kv4(q, k, v, c, s, 70, [-1, 0, 0], 5, **ref), attn),
        "quantize": (lambda: al.mx4_quantize(W), [((300, 48), u8), ((300, 3), u8)]),
        "dequantize": (lambda: [al.mx4_dequantize(codes, scales)], [((300, 96), torch.bfloat16)]),
    }


@pytest.mark.parametrize("name", ["lmhead", "lmhead_packed", "lmhead_mx4", "attn_kv4", "quantize", "dequantize"])
def test_dispatch_modes_see_new_outputs(name):
    call, outputs = _calls()[name]
    want = call()   # (workspaces are made here)
    with _Made() as mode:
        got = call()
    assert mode.made == outputs
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", ["lmhead", "lmhead_packed", "lmhead_mx4", "attn_kv4", "quantize", "dequantize"])
def test_deterministic_mode(name):
    """Uninitialised memory is filled first; the results are the same."""
    call, _ = _calls()[name]
    want = call()
    before = torch.are_deterministic_algorithms_enabled()
    try:
        torch.use_deterministic_algorithms(True)
        assert torch.utils.deterministic.fill_uninitialized_memory
        got = call()
    finally:
        torch.use_deterministic_algorithms(before)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
