"""What the 4-bit operators are timed on: a decode step in microscaled 4-bit floating point.

The format (MXFP4): e2m1 codes, two to a byte, and one power-of-two scale byte for every 32
consecutive elements.  The operators are the row quantiser and its inverse (mx4_quantize,
mx4_dequantize), the store of K/V rows into a 4-bit prefix cache (kv4_store), lane attention over
that cache (lane_attn_forward_kv4) and the fused LM head with confidence on a 4-bit weight
(lmhead_confidence_mx4).  Shapes are those of the synthetic workloads "tiny", "llada", "dream" and
"wide"; draw() gives other sizes of the same ranges.
"""
import math

import numpy as np
import torch

own = False   # True: the framework's calls; False: the plain forms

EOS_ID = 2


# ------------------------------------------------------------------- cases
def _quant(name, R, n):
    return dict(name=name, kind="quant", R=R, n=n)


def _store(name, T, cap, Hkv, D):
    return dict(name=name, kind="store", T=T, cap=cap, Hkv=Hkv, D=D)


def _attn(name, L, B, P, cap, Hq, Hkv, D, tree, depth, n_ref=0):
    return dict(name=name, kind="attn", L=L, B=B, P=P, cap=cap, Hq=Hq, Hkv=Hkv, D=D, tree=tree,
                depth=depth, n_ref=n_ref)


def _lm(name, N, n_rows, d, V):
    return dict(name=name, kind="lmhead", N=N, n_rows=n_rows, d=d, V=V)


def listed():
    return [
        # The hidden rows of one decode step: latency and launches.
        _quant("quant_rows", 128, 4096),
        # The LLaDA-8B head's weight, quantised once at load time: the largest.
        _quant("quant_head", 126464, 4096),
        # One lane's block stored behind a prompt of 512 rows (32 heads of 128).
        _store("store_lane", 32, 544, 32, 128),
        # A prompt of odd length stored at prefill.
        _store("store_prompt", 2563, 2816, 32, 128),
        # The smallest step: two lanes, four heads of 64.
        _attn("attn_tiny", 2, 32, 128, 128, 4, 4, 64, "random", 1),
        # A single token over a long cache with grouped queries (28 heads on 4).
        _attn("attn_token", 1, 1, 32769, 33000, 28, 4, 128, "linear", 0),
        # One layer of a Dream-7B decode step: 8 lanes, grouped queries.
        _attn("attn_dream", 8, 32, 1024, 1280, 28, 4, 128, "random", 3),
        # Many lanes, long prefix, and a tenth of the prefix refreshed in the same call.
        _attn("attn_wide", 32, 64, 4096, 4352, 32, 32, 128, "random", 8, 410),
        # A small head as small models and tests have it: latency and launches.
        _lm("lm_tiny", 32, 64, 256, 1024),
        # LLaDA-8B head for a single token.
        _lm("lm_token", 1, 1, 4096, 126464),
        # LLaDA-8B head, 77 masked rows: the usual decode step.
        _lm("lm_llada", 77, 128, 4096, 126464),
        # LLaDA-8B head, 614 masked rows: many lanes of one batch.
        _lm("lm_wide", 614, 2048, 4096, 126464),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {c["name"]: work(c) for c in listed()}
    while True:
        kind = rng.choice(["quant", "store", "attn", "attn", "attn", "lmhead", "lmhead", "lmhead"])
        if kind == "quant":
            c = dict(kind="quant", R=_log_int(rng, 1, 126464), n=32 * _log_int(rng, 1, 256))
            if work(c)["bytes"] <= most["quant_head"]["bytes"]:
                return c
        elif kind == "store":
            T, D = _log_int(rng, 1, 2563), rng.choice([64, 128])
            Hkv = rng.choice([1, 4, 8, 32])
            return dict(kind="store", T=T, cap=T + rng.randint(0, 512), Hkv=Hkv, D=D)
        elif kind == "attn":
            Hkv, g = rng.choice([(4, 1), (8, 1), (32, 1), (8, 4), (4, 7)])
            P = _log_int(rng, 33, 32769)
            c = dict(kind="attn", L=_log_int(rng, 1, 32), B=rng.choice([1, 1, 5, 16, 32, 32, 48, 64]),
                     P=P, cap=P + rng.randint(0, 300), Hq=Hkv * g, Hkv=Hkv, D=rng.choice([64, 128, 128]),
                     tree=rng.choice(["linear", "random", "random"]), depth=rng.randint(1, 8),
                     n_ref=rng.choice([0, 0, 0, P // 10]))
            if work(c)["flops"] <= most["attn_wide"]["flops"]:
                return c
        else:
            N = _log_int(rng, 1, 614)
            d, V = rng.choice([(4096, 126464), (3584, 152064), (4096, _log_int(rng, 1000, 126464)),
                               (32 * _log_int(rng, 2, 128), _log_int(rng, 1000, 126464))])
            c = dict(kind="lmhead", N=N, n_rows=N + rng.randint(0, 2 * N), d=d, V=V)
            if work(c)["flops"] <= most["lm_wide"]["flops"]:
                return c


# ------------------------------------------------------------------ inputs
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + stream)
    return g


def _normal(seed, stream, shape, std=1.0):
    n = math.prod(shape)
    out = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    g = _gen(seed, stream)
    for i in range(0, n, 1 << 26):   # in pieces: the fp32 draws of a whole weight would be 2 GB
        m = min(1 << 26, n - i)
        out[i:i + m] = torch.randn(m, generator=g, device="cuda") * std
    return out.view(shape)


def _tree(case):
    """Lane tree, parent[i] in [-1, i): a chain, or random forks up to a depth (one tree a case:
    what the call has to do depends on it)."""
    L = case["L"]
    rng = np.random.default_rng([L, case["depth"], 71])
    parent = np.full(L, -1, np.int32)
    depth = np.zeros(L, np.int64)
    for i in range(1, L):
        j = i - 1 if case["tree"] == "linear" else int(
            rng.choice(np.nonzero(depth[:i] < max(1, case["depth"]))[0]))
        parent[i] = j
        depth[i] = depth[j] + 1
    return parent


def _see(parent):
    """[L][L] truth values: lane j is lane i or one of its ancestors."""
    see = np.eye(len(parent), dtype=bool)
    for i, p in enumerate(parent):
        if p >= 0:
            see[i] |= see[p]
    return torch.from_numpy(see).cuda()


def _pack_weight(codes, scales, V, d):
    """The weight as a program keeps it for the head, laid out once: K stages of 128 elements,
    in each the 16-row units, in each 64 lanes of 16 bytes (lane 16 b + r: row r, scale block b);
    behind them the scales, four units to a dword.  Rows past V and elements past d are zero."""
    U, C = 4 * ((V + 63) // 64), (d + 127) // 128
    c = torch.zeros((16 * U, 64 * C), dtype=torch.uint8, device="cuda")
    s = torch.zeros((16 * U, 4 * C), dtype=torch.uint8, device="cuda")
    c[:V, :d // 2] = codes
    s[:V, :d // 32] = scales
    c = c.view(U, 16, C, 4, 16).permute(2, 0, 3, 1, 4).reshape(-1)
    s = s.view(U // 4, 4, 16, C, 4).permute(3, 0, 4, 2, 1).reshape(-1)
    return torch.cat([c, s])


def prepare(case, seed):
    rng = np.random.default_rng([int(seed), 77])
    if case["kind"] == "quant":
        # Weights and activations have rows of unlike size.
        std = torch.exp(torch.randn((case["R"], 1), generator=_gen(seed, 2), device="cuda"))
        x = _normal(seed, 1, (case["R"], case["n"]))
        for i in range(0, case["R"], 16384):
            x[i:i + 16384] = x[i:i + 16384].float() * std[i:i + 16384]
        return dict(case=case, x=x)
    if case["kind"] == "store":
        T, cap, Hkv, D = (case[k] for k in ("T", "cap", "Hkv", "D"))
        codes, scales = _quantize(_normal(seed, 3, (2, Hkv, cap, D)))   # what the cache held before
        rows = rng.choice(cap, T, replace=False).astype(np.int32)
        return dict(case=case, k=_normal(seed, 1, (T, Hkv, D)), v=_normal(seed, 2, (T, Hkv, D)),
                    rows=torch.from_numpy(rows).cuda(), codes=codes, scales=scales)
    if case["kind"] == "attn":
        L, B, P, cap, Hq, Hkv, D, n_ref = (case[k] for k in ("L", "B", "P", "cap", "Hq", "Hkv", "D", "n_ref"))
        R = L * B
        codes, scales = _quantize(_normal(seed, 1, (2, Hkv, cap, D)))
        parent = _tree(case)
        s = dict(case=case, codes=codes, scales=scales, parent=parent, see=_see(parent),
                 q=_normal(seed, 3, (R, Hq, D)), k_lane=_normal(seed, 4, (R, Hkv, D)),
                 v_lane=_normal(seed, 5, (R, Hkv, D)), ref={})
        if n_ref:
            idx = np.sort(rng.choice(P, n_ref, replace=False)).astype(np.int32)
            s["ref"] = dict(refresh_idx=torch.from_numpy(idx).cuda(), q_ref=_normal(seed, 6, (n_ref, Hq, D)),
                            k_ref=_normal(seed, 7, (n_ref, Hkv, D)), v_ref=_normal(seed, 8, (n_ref, Hkv, D)))
        return s
    N, n_rows, d, V = (case[k] for k in ("N", "n_rows", "d", "V"))
    W = _normal(seed, 10, (V, d), 1.0 / math.sqrt(d))
    codes, scales = _quantize(W)
    # Masked rows of a trained model: each leans to one token, with logits of unlike size, so that
    # confidences range from a few percent to near 1.
    target = torch.from_numpy(rng.integers(3, V, n_rows)).cuda()
    lean = 7.0 + 5.0 * torch.rand((n_rows, 1), generator=_gen(seed, 11), device="cuda")
    scale = 1.0 + 2.0 * torch.rand((n_rows, 1), generator=_gen(seed, 12), device="cuda")
    hidden = ((_normal(seed, 9, (n_rows, d)).float() + lean * W[target].float()) * scale).to(torch.bfloat16)
    rows = np.sort(rng.choice(n_rows, N, replace=False)).astype(np.int32)
    return dict(case=case, hidden=hidden, row_idx=torch.from_numpy(rows).cuda(),
                sup=torch.from_numpy(rng.integers(0, 2, N).astype(np.uint8)).cuda(),
                codes=codes, scales=scales, W_mx4=_pack_weight(codes, scales, V, d))


# ------------------------------------------------------------- plain forms
def _pow2(e):
    """2^e in 64 bits, exactly (exp2 and ldexp are rounded on the GPU)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantize(x):
    """codes [..., n/2] and scales [..., n/32] of x [..., n]: the scale's exponent is that of the
    block's largest magnitude less 2; codes are rounded to nearest, ties to even, saturated at 6."""
    codes = torch.empty(x.shape[:-1] + (x.shape[-1] // 2,), dtype=torch.uint8, device=x.device)
    scales = torch.empty(x.shape[:-1] + (x.shape[-1] // 32,), dtype=torch.uint8, device=x.device)
    xf, cf, sf = x.reshape(-1, 32), codes.view(-1, 16), scales.view(-1)
    for i in range(0, xf.shape[0], 1 << 21):
        b = xf[i:i + (1 << 21)].float()
        top = b.abs().amax(dim=1, keepdim=True)
        e = torch.clamp(torch.frexp(top)[1] - 3, -127, 127)   # frexp: top = m 2^k, m in [0.5, 1)
        e = torch.where(top > 0, e, -127)
        a = b.abs().double() * _pow2(-e)
        m = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
        m = m + 8 * torch.signbit(b)
        cf[i:i + (1 << 21)] = (m[:, 0::2] + 16 * m[:, 1::2]).to(torch.uint8)
        sf[i:i + (1 << 21)] = (e + 127).view(-1).to(torch.uint8)
    return codes, scales


def _values(codes, scales):
    """fp32 values [..., n] of codes [..., n/2] and scales [..., n/32]."""
    e2m1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    e2m1 = torch.cat([e2m1, -e2m1])
    pair = torch.stack([e2m1.repeat(16), e2m1.repeat_interleave(16)], dim=1)   # of a byte
    v = pair[codes.reshape(-1).int()].view(scales.numel(), 32)
    return (v * _pow2(scales.reshape(-1, 1).int() - 127).float()).view(codes.shape[:-1] + (2 * codes.shape[-1],))


def _store_rows(codes, scales, k, v, rows):
    for plane, x in enumerate((k, v)):
        c, s = _quantize(x)
        codes[plane][:, rows.long()] = c.transpose(0, 1)
        scales[plane][:, rows.long()] = s.transpose(0, 1)


def _attend(q, k, v, visible):
    """softmax(q k^T / sqrt(D)) v; q [R][Hq][D], k and v [Hkv][S][D], visible [R][S] or None."""
    R, Hq, D = q.shape
    Hkv = k.shape[0]
    g = Hq // Hkv
    qh = q.float().view(R, Hkv, g, D).permute(1, 2, 0, 3).reshape(Hkv, g * R, D)
    z = torch.bmm(qh, k.transpose(1, 2).contiguous()) / math.sqrt(D)
    if visible is not None:
        z.view(Hkv, g, R, -1).masked_fill_(~visible, -math.inf)
    top = z.amax(dim=2, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=2, keepdim=True)
    o = torch.bmm(e, v) / total
    lse = (top + torch.log(total)).view(Hkv, g, R).permute(2, 0, 1).reshape(R, Hq)
    o = o.view(Hkv, g, R, D).permute(2, 0, 1, 3).reshape(R, Hq, D)
    return o.to(torch.bfloat16), lse


def _plain(s):
    case = s["case"]
    if case["kind"] == "quant":
        return dict(y=_values(*_quantize(s["x"])).to(torch.bfloat16))
    if case["kind"] == "store":
        _store_rows(s["codes"], s["scales"], s["k"], s["v"], s["rows"])
        return dict(cache=_values(s["codes"], s["scales"]).to(torch.bfloat16))
    if case["kind"] == "attn":
        B, P, ref = case["B"], case["P"], s["ref"]
        if ref:
            _store_rows(s["codes"], s["scales"], ref["k_ref"], ref["v_ref"], ref["refresh_idx"])
        kv = _values(s["codes"], s["scales"])
        k, v = kv[0, :, :P], kv[1, :, :P]
        lanes = s["see"].repeat_interleave(B, 0).repeat_interleave(B, 1)
        visible = torch.cat([torch.ones((lanes.shape[0], P), dtype=torch.bool, device="cuda"), lanes], 1)
        o, lse = _attend(s["q"], torch.cat([k, s["k_lane"].float().transpose(0, 1)], 1),
                         torch.cat([v, s["v_lane"].float().transpose(0, 1)], 1), visible)
        out = dict(o=o, lse=lse)
        if ref:
            out["o_ref"], out["lse_ref"] = _attend(ref["q_ref"], k.contiguous(), v.contiguous(), None)
            out["cache"] = kv.to(torch.bfloat16)
        return out
    h = s["hidden"][s["row_idx"].long()].float()
    z = torch.mm(h, _values(s["codes"], s["scales"]).t())
    z[s["sup"].bool(), EOS_ID] = -math.inf
    top = z.amax(dim=1, keepdim=True)
    ids = torch.arange(z.shape[1], dtype=torch.int32, device="cuda")
    arg = torch.where(z == top, ids, z.shape[1]).amin(dim=1).to(torch.int32)
    total = torch.exp(z - top).sum(dim=1, dtype=torch.float64)
    return dict(conf=(1.0 / total).float(), argmax=arg, lse=(top[:, 0].double() + torch.log(total)).float())


# -------------------------------------------------------------------- runs
def run(state):
    if not own:
        return _plain(state)
    import paper_2606_08411_amd as al
    s, case = state, state["case"]
    if case["kind"] == "quant":
        # The weight (or rows) in 4 bits, and the values that stand in its place.
        return dict(y=al.mx4_dequantize(*al.mx4_quantize(s["x"])))
    if case["kind"] == "store":
        # Rows into the cache, and the whole cache read back.
        al.kv4_store(s["k"], s["v"], s["codes"], s["scales"], row_idx=s["rows"])
        return dict(cache=al.mx4_dequantize(s["codes"], s["scales"]))
    if case["kind"] == "attn":
        o, lse, o_ref, lse_ref = al.lane_attn_forward_kv4(
            s["q"], s["k_lane"], s["v_lane"], s["codes"], s["scales"], case["P"], s["parent"],
            case["B"], **s["ref"])
        out = dict(o=o, lse=lse)
        if s["ref"]:
            out.update(o_ref=o_ref, lse_ref=lse_ref, cache=al.mx4_dequantize(s["codes"], s["scales"]))
        return out
    conf, arg, lse = al.lmhead_confidence_mx4(s["hidden"], s["W_mx4"], case["V"], row_idx=s["row_idx"],
                                              suppress_eos=s["sup"], eos_id=EOS_ID)
    return dict(conf=conf, argmax=arg, lse=lse)


# --------------------------------------------------------- work and 64 bits
MX4 = 0.5 + 1.0 / 32.0   # bytes of an element


def work(case):
    if case["kind"] == "quant":   # in bf16, into 4 bits and out of them, out in bf16
        return dict(bytes=case["R"] * case["n"] * (4.0 + 2.0 * MX4), flops=0)
    if case["kind"] == "store":
        e = 2.0 * case["Hkv"] * case["D"]
        return dict(bytes=case["T"] * (e * (2.0 + MX4) + 4.0) + case["cap"] * e * (2.0 + MX4), flops=0)
    if case["kind"] == "attn":
        L, B, P, cap, Hq, Hkv, D, n_ref = (case[k] for k in ("L", "B", "P", "cap", "Hq", "Hkv", "D", "n_ref"))
        sees = np.ones(L, np.int64)   # lanes that a lane sees: itself and its ancestors
        for i, p in enumerate(_tree(case)):
            if p >= 0:
                sees[i] += sees[p]
        keys = float(sum(B * (P + B * int(n)) for n in sees)) + float(n_ref) * P
        rows, e = L * B + n_ref, 2.0 * Hkv * D
        move = rows * Hq * (4.0 * D + 4.0) + e * (MX4 * P + 2.0 * L * B)
        if n_ref:
            move += n_ref * e * 2.0 + cap * e * (2.0 + MX4)   # (the whole cache read back)
        return dict(bytes=move, flops=4.0 * Hq * D * keys)
    N, d, V = case["N"], case["d"], case["V"]
    return dict(bytes=MX4 * V * d + 2.0 * N * d + 17.0 * N, flops=2.0 * N * V * d)


def _exact_values(x):
    """The values that x [..., n] is held as, in 64 bits: to the nearest multiple of the step that
    e2m1 has at a magnitude (half, one or two scales), ties to the even one."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    src, dst = x.reshape(-1, 32), out.view(-1, 32)
    for i in range(0, src.shape[0], 1 << 20):
        b = src[i:i + (1 << 20)].double()
        top = b.abs().amax(dim=1, keepdim=True)
        # 2^floor(log2 top): its exponent's bits alone (log2 may miss a power of two)
        scale = torch.clamp((top.view(torch.int64) & (0x7FF << 52)).view(torch.float64) / 4.0, min=2.0 ** -127)
        a = b.abs() / scale
        step = torch.where(a >= 4.0, 2.0, torch.where(a >= 2.0, 1.0, 0.5)).double()
        dst[i:i + (1 << 20)] = torch.sign(b) * torch.clamp(torch.round(a / step) * step, max=6.0) * scale
    return out


def _exact_cache(codes, scales):
    """The values of a cache as it was before the call."""
    c = codes.cpu().numpy()
    n = np.stack([c & 15, c >> 4], axis=-1).reshape(c.shape[:-1] + (2 * c.shape[-1],))
    m, x = (n & 1).astype(np.float64), (n >> 1) & 3
    mag = np.where(x == 0, 0.5 * m, (1.0 + 0.5 * m) * 2.0 ** (x.astype(np.float64) - 1.0))
    e = np.repeat(scales.cpu().numpy().astype(np.float64) - 127.0, 32, axis=-1)
    return torch.from_numpy(np.where(n & 8, -mag, mag) * 2.0 ** e).cuda()


def _exact_attention(q, k, v, visible):
    """Head by head; k and v [S][Hkv][D] in 64 bits, visible [rows][keys] or None."""
    Hq, g = q.shape[1], q.shape[1] // k.shape[1]
    o = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    for h in range(Hq):
        kh, vh = k[:, h // g].contiguous(), v[:, h // g].contiguous()
        z = torch.mm(q[:, h].double().contiguous(), kh.t().contiguous()) * (q.shape[2] ** -0.5)
        if visible is not None:
            z.masked_fill_(~visible, -math.inf)
        lse[:, h] = torch.logsumexp(z, dim=1)
        o[:, h] = torch.mm(torch.exp(z - lse[:, h:h + 1]), vh)
    return o, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quant":
        return dict(y=_exact_values(s["x"]))
    if case["kind"] == "store":
        cache = _exact_cache(s["codes"], s["scales"])
        for plane, x in enumerate((s["k"], s["v"])):
            cache[plane][:, s["rows"].long()] = _exact_values(x).transpose(0, 1)
        return dict(cache=cache)
    if case["kind"] == "attn":
        B, P, ref = case["B"], case["P"], s["ref"]
        cache = _exact_cache(s["codes"], s["scales"])
        if ref:
            for plane, x in enumerate((ref["k_ref"], ref["v_ref"])):
                cache[plane][:, ref["refresh_idx"].long()] = _exact_values(x).transpose(0, 1)
        k, v = (cache[i, :, :P].transpose(0, 1) for i in (0, 1))
        out = {}
        lane = s["see"].repeat_interleave(B, 0).repeat_interleave(B, 1)
        visible = torch.nn.functional.pad(lane, (P, 0), value=True)
        out["o"], out["lse"] = _exact_attention(s["q"], torch.cat([k, s["k_lane"].double()]),
                                                torch.cat([v, s["v_lane"].double()]), visible)
        if ref:
            out["o_ref"], out["lse_ref"] = _exact_attention(ref["q_ref"], k, v, None)
            out["cache"] = cache
        return out
    h = s["hidden"][s["row_idx"].long()].double()
    z = torch.cat([torch.mm(h, _exact_cache(c, e).t().contiguous())
                   for c, e in zip(s["codes"].split(16384), s["scales"].split(16384))], dim=1)
    z[s["sup"].bool(), EOS_ID] = -math.inf
    top, arg = z.max(dim=1)
    lse = torch.logsumexp(z, dim=1)
    return dict(conf=torch.exp(top - lse), argmax=arg.to(torch.int32), lse=lse)
