"""Calls of several host threads on one stream, with the binding's default workspaces: each call's partials
are joined by its own second kernel, so every result is the serial one, bit for bit."""
import threading

import numpy as np
import pytest
import torch

import oracle
import paper_2606_08411_amd as al
import synth
from gpu_util import dev_bf16
from mx4_util import bf16_normal, dev, random_cache

pytestmark = pytest.mark.gpu
THREADS, ROUNDS = 4, 40


def _attn_kv4(seed, python):
    """(B: 1, a token whose keys are split.)"""
    g = np.random.default_rng(seed)
    P, Hq, Hkv, D = 4000, 8, 2, 64
    assert al.lane_attn_kv4_workspace_size(1, 1, P, Hq, Hkv, D) > 0
    c, s = (dev(x) for x in random_cache(g, Hkv, P, D))
    q, k, v = (dev_bf16(bf16_normal(g, 1, h, D)) for h in (Hq, Hkv, Hkv))
    parent = np.array([-1], np.int64 if python else np.int32)   # (int64: marshalled in Python)
    return lambda: al.lane_attn_forward_kv4(q, k, v, c, s, P, parent, 1)[:2]


def _lmhead_mx4(seed, python):
    g = np.random.default_rng(seed)
    V, d, N = 5000, 128, 9
    W = al.lmhead_pack_weight_mx4(*(dev(x) for x in oracle.mx4.quantize(g.standard_normal((V, d)))))
    h = dev_bf16(bf16_normal(g, N, d))
    return lambda: al.lmhead_confidence_mx4(h, W, np.int64(V) if python else V)


def _attn(seed, python):
    s = synth.make_step("long", seed, with_weight=False)
    assert al.lane_attn_workspace_size(s.L, s.B, s.P, s.Hq, s.Hkv, s.D, 0) > 0
    a = [dev_bf16(x) for x in (s.q, s.k_lane, s.v_lane, s.k_pre, s.v_pre)]
    parent = np.asarray(s.parent, np.int64 if python else np.int32)
    return lambda: al.lane_attn_forward(*a, parent, s.B)[:2]


def _lmhead(seed, python):
    g = np.random.default_rng(seed)
    h, W = dev_bf16(bf16_normal(g, 9, 128)), dev_bf16(bf16_normal(g, 5000, 128))
    return lambda: al.lmhead_confidence(h, W, eos_id=np.int64(-1) if python else -1)


@pytest.mark.parametrize("python", [False, True], ids=["native", "python"])
@pytest.mark.parametrize("make", [_attn_kv4, _lmhead_mx4, _attn, _lmhead], ids=lambda f: f.__name__[1:])
def test_threads_on_one_stream(make, python):
    calls = [make(10 + i, python) for i in range(THREADS)]
    want = [[x.clone() for x in c()] for c in calls]
    torch.cuda.synchronize()
    start, got = threading.Barrier(THREADS), [None] * THREADS

    def work(i):
        start.wait()
        got[i] = [calls[i]() for _ in range(ROUNDS)]
    threads = [threading.Thread(target=work, args=(i,)) for i in range(THREADS)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(THREADS):
        assert got[i] is not None and len(got[i]) == ROUNDS
        for out in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
