"""A decode step in 4 bits, as a program runs it: the head's weight quantised and packed once, a prompt
stored in a 4-bit cache, then steps of attention over it, the head and the selection, and the block
that a lane finishes appended to the cache.  Against the fp64 oracle, captured in a graph, and on
two streams at once."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_08411_amd as al
import synth
from gpu_util import dev, dev_bf16
from mx4_util import attention_bounds, cache_rows, f64, host_f64, lmhead_bounds

pytestmark = pytest.mark.gpu


class Step:
    """Inputs, kept weights and cache, outputs and workspaces of one prefix group."""

    def __init__(self, name, seed, cap_more=70, **over):
        s = self.s = synth.make_step(name, seed, **over)
        self.W = dev_bf16(s.W)
        codes, scales = al.mx4_quantize(self.W)
        self.W_mx4 = al.lmhead_pack_weight_mx4(codes, scales)
        self.cap = s.P + cap_more
        self.codes = torch.zeros((2, s.Hkv, self.cap, s.D // 2), dtype=torch.uint8, device="cuda")
        self.scales = torch.zeros((2, s.Hkv, self.cap, s.D // 32), dtype=torch.uint8, device="cuda")
        al.kv4_store(dev_bf16(s.k_pre), dev_bf16(s.v_pre), self.codes, self.scales)
        self.q, self.k, self.v = dev_bf16(s.q), dev_bf16(s.k_lane), dev_bf16(s.v_lane)
        self.ref = {}
        if s.n_ref:
            self.ref = dict(refresh_idx=dev(s.refresh_idx), q_ref=dev_bf16(s.q_ref), k_ref=dev_bf16(s.k_ref),
                            v_ref=dev_bf16(s.v_ref), o_ref=torch.empty_like(dev_bf16(s.q_ref)),
                            lse_ref=torch.empty((s.n_ref, s.Hq), device="cuda"))
        self.hidden, self.rows, self.sup = dev_bf16(s.hidden), dev(s.row_pos), dev(s.suppress_eos)
        self.tokens, self.masked = dev(s.tokens), dev(s.is_masked)
        self.ws_a = torch.empty(max(16, al.lane_attn_kv4_workspace_size(s.L, s.B, s.P, s.Hq, s.Hkv, s.D, s.n_ref)),
                                dtype=torch.uint8, device="cuda")
        self.ws_l = torch.empty(al.lmhead_confidence_mx4_workspace_size(s.N, s.d, s.V), dtype=torch.uint8, device="cuda")
        f = dict(device="cuda")
        self.o, self.lse = torch.empty_like(self.q), torch.empty((s.L * s.B, s.Hq), **f)
        self.conf, self.lm_lse = torch.empty(s.N, **f), torch.empty(s.N, **f)
        self.arg = torch.empty(s.N, dtype=torch.int32, **f)

    def run(self, own_workspaces=True):
        s = self.s
        a, b = (dict(workspace=self.ws_a), dict(workspace=self.ws_l)) if own_workspaces else ({}, {})
        al.lane_attn_forward_kv4(self.q, self.k, self.v, self.codes, self.scales, s.P, s.parent, s.B, o=self.o,
                                 lse=self.lse, **self.ref, **a)
        al.lmhead_confidence_mx4(self.hidden, self.W_mx4, s.V, row_idx=self.rows, suppress_eos=self.sup,
                                 eos_id=s.eos_id, conf=self.conf, argmax=self.arg, lse=self.lm_lse, **b)
        self.sel = al.select_unmask(self.conf, self.arg, self.rows, self.tokens, self.masked, s.L, s.B, s.role, s.b_len,
                                    s.t_lane, al.MODE_THRESHOLD, s.tau, 1, out=getattr(self, "sel", None))

    def outputs(self):
        r = [self.o, self.lse, self.conf, self.arg, self.lm_lse, self.tokens, self.masked, self.sel["lane_stats"],
             self.codes, self.scales]
        return [x.clone() for x in r + ([self.ref["o_ref"], self.ref["lse_ref"]] if self.ref else [])]

    def reset(self):
        self.tokens.copy_(dev(self.s.tokens)), self.masked.copy_(dev(self.s.is_masked))


@pytest.mark.parametrize("refresh", [0.0, 0.1])
def test_step_against_the_oracle(refresh):
    t = Step("tiny", 3, P=150, refresh_frac=refresh, Hq=8, Hkv=2, L=3, tree="random", depth_max=2)
    s = t.s
    t.run()
    torch.cuda.synchronize()
    codes, scales = (np.stack(x) for x in zip(*(oracle.mx4.quantize(f64(x)) for x in (s.k_pre, s.v_pre))))
    codes, scales = codes.transpose(0, 2, 1, 3).copy(), scales.transpose(0, 2, 1, 3).copy()
    if s.n_ref:
        for plane, x in enumerate((s.k_ref, s.v_ref)):
            rc, rs = oracle.mx4.quantize(f64(x))
            codes[plane][:, s.refresh_idx], scales[plane][:, s.refresh_idx] = rc.transpose(1, 0, 2), rs.transpose(1, 0, 2)
    assert np.array_equal(t.codes[:, :, :s.P].cpu().numpy(), codes) and not bool(t.codes[:, :, s.P:].any())
    kp, vp = cache_rows(codes, scales, s.P)
    q, k, v = f64(s.q), f64(s.k_lane), f64(s.v_lane)
    ro, rl = oracle.attention.lane_attention_concat(q, k, v, kp, vp, s.parent, s.B)
    ra, _ = oracle.attention.lane_attention_concat(q, k, np.abs(v), kp, np.abs(vp), s.parent, s.B)
    bo, bl = attention_bounds(ro, ra, rl, q, np.concatenate([kp, k]), s.D, s.P + s.L * s.B)
    assert (np.abs(host_f64(t.o) - ro) <= bo).all() and (np.abs(host_f64(t.lse) - rl) <= bl).all()
    W = oracle.mx4.rounded(f64(s.W))
    h = f64(s.hidden)
    ref = oracle.lmhead.lmhead_confidence_full(h, s.row_pos, W, s.suppress_eos, s.eos_id)
    bz, bl, bc = lmhead_bounds(h[s.row_pos], W, ref["lse"])
    conf, arg = t.conf.cpu().numpy(), t.arg.cpu().numpy()
    ok = ref["gap"] > 2 * bz
    assert np.array_equal(arg[ok], ref["argmax"][ok]) and ok.mean() > 0.8
    assert (np.abs(conf - ref["conf"]) <= bc * ref["conf"]).all()
    # the selection on these confidences, exactly
    r = oracle.select.select_unmask(conf, arg, s.row_pos, s.tokens, s.is_masked, s.B, s.role, s.b_len, s.t_lane, 0, s.tau, 1)
    assert np.array_equal(t.tokens.cpu().numpy(), r["tokens"])
    assert np.array_equal(t.sel["lane_stats"].cpu().numpy(), r["lane_stats"])


def test_finished_block_joins_the_prefix():
    """A finished root lane's rows appended to the cache: its child then sees the same keys, in 4 bits."""
    s = synth.make_step("tiny", 5, with_weight=False, L=1, B=20, P=75, tree="linear", V=64, d=64)
    t = Step("tiny", 5, L=1, B=20, P=75, tree="linear")
    al.kv4_store(t.k, t.v, t.codes, t.scales, start=s.P)
    g = np.random.default_rng(1)
    q, k, v = (synth.f32_to_bf16_bits(g.standard_normal((1, h, s.D), dtype=np.float32)) for h in (s.Hq, s.Hkv, s.Hkv))
    o, lse, _, _ = al.lane_attn_forward_kv4(dev_bf16(q), dev_bf16(k), dev_bf16(v), t.codes, t.scales, s.P + 20, [-1], 1)
    rnd = lambda a, b: np.concatenate([oracle.mx4.rounded(f64(x)) for x in (a, b)])
    kp, vp = rnd(s.k_pre, s.k_lane), rnd(s.v_pre, s.v_lane)
    ro, rl = oracle.attention.lane_attention_concat(f64(q), f64(k), f64(v), kp, vp, [-1], 1)
    ra, _ = oracle.attention.lane_attention_concat(f64(q), f64(k), np.abs(f64(v)), kp, np.abs(vp), [-1], 1)
    bo, bl = attention_bounds(ro, ra, rl, f64(q), np.concatenate([kp, f64(k)]), s.D, 96)
    assert (np.abs(host_f64(o) - ro) <= bo).all() and (np.abs(host_f64(lse) - rl) <= bl).all()


@pytest.mark.parametrize("over", [dict(P=150, refresh_frac=0.1), dict(P=6000, L=1, B=1, tree="linear", d=4096)], ids=["refresh", "splits"])
def test_graph_replays(over):
    """Captured and replayed, with eager steps of another group between the replays."""
    t, other = Step("tiny", 3, **over), Step("tiny", 4, **over)
    t.run()
    other.run()
    torch.cuda.synchronize()
    want, want_other = t.outputs(), other.outputs()
    graph = torch.cuda.CUDAGraph()
    t.reset()
    with torch.cuda.graph(graph):
        t.run()
    for rep in range(4):
        t.reset()
        for x in (t.o, t.conf, t.arg, t.lse):
            x.zero_()
        graph.replay()
        other.reset()
        other.run(own_workspaces=False)
        torch.cuda.synchronize()
        for x, y in zip(t.outputs() + other.outputs(), want + want_other):
            assert torch.equal(x, y), rep


def test_two_streams():
    """Two groups on two streams at once, on the binding's workspaces."""
    over = dict(P=6000, L=2, B=3, tree="fork", d=2048, V=3000)
    steps = [Step("tiny", i, **over) for i in (1, 2)]
    assert al.lane_attn_kv4_workspace_size(2, 3, 6000, 4, 4, 64) > 0
    for t in steps:
        t.run(own_workspaces=False)
    torch.cuda.synchronize()
    want = [t.outputs() for t in steps]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(6):
        for t in steps:
            t.reset()
            for x in (t.o, t.conf, t.arg):
                x.zero_()
        torch.cuda.synchronize()
        for st, t in zip(streams, steps):
            with torch.cuda.stream(st):
                t.run(own_workspaces=False)
        torch.cuda.synchronize()
        for t, w in zip(steps, want):
            for x, y in zip(t.outputs(), w):
                assert torch.equal(x, y), rep
