// Shared-prefix lane-batched bidirectional attention over a prefix cache held
// in MXFP4 (mx4.h); lane blocks are bf16.  The visible keys and the softmax are
// those of lane_attn.hip.
//
// Query rows.  The g query heads of a K/V head and the rows of all lanes form
// one list of "pairs" (row-major, the g heads of a row adjacent), cut into tiles
// of 32.  Every pair sees the whole prefix, so a tile may hold rows of several
// lanes, and single-token lanes of a grouped-query model fill tiles; which lane
// blocks a pair sees is a mask of its own lane of the wavefront (S^T = K Q^T
// leaves a pair's scores to the wavefront lanes l and l ^ 32).
//
// Keys.  Tiles of 64: first the prefix, then the rows of all lane blocks as one
// list.  A prefix tile is read as codes (a 16-byte load per 32 elements), converted
// to bf16 (exact) and written to LDS once per workgroup, K and V row-major with
// their 16-byte segments permuted; a lane tile is copied.  Both products are the
// 32x32x16 bf16 MFMA with fp32 accumulation, transposed as in lane_attn.hip:
//     S^T = K Q^T,   O^T = V^T P^T  (V^T by LDS transpose reads).
// P is rounded to bf16 for the second product; the row sum adds the unrounded
// fp32 values, so the log-sum-exp keeps fp32 accuracy (adding the rounded ones
// would move it by up to 2^-9).
//
// Keys are split over blockIdx.z where there are few query tiles; the splits'
// partials are kept in fp32 and combined by kv4_merge_kernel.
#include <math.h>

#include "common.h"
#include "launch.h"
#include "mx4.h"

namespace al {

constexpr int K4_KT = 64;            // keys per tile
constexpr int K4_WAVES = 8;          // query tiles per workgroup
constexpr int K4_THREADS = K4_WAVES * kWave;
constexpr float K4_LN2 = 0.6931471805599453f;

struct Kv4Params {
  const uint16_t* q;        // [n_rows][Hq][D]
  const uint16_t* k_lane;   // [R][Hkv][D]
  const uint16_t* v_lane;
  const uint8_t* codes;     // [2][Hkv][cap][D / 2]
  const uint8_t* scales;    // [2][Hkv][cap][D / 32]
  uint16_t* o;              // [n_rows][Hq][D]
  float* lse;               // [n_rows][Hq] or null
  float* part_o;            // [n_split][n_rows * Hq][D] unnormalised, when n_split > 1
  float* part_ml;           // [n_split][n_rows * Hq][2]
  int n_rows, R, B, P, cap, Hq, Hkv, g;
  int n_pairs;              // n_rows * g
  int n_pre, n_tiles, n_split;   // prefix tiles, all key tiles
  float scale_log2;
  unsigned long long vis[64];    // bit j: lane block j visible to lane i
};

// Bits of the 64 lane rows from `row` on that a pair with visibility v sees.
__device__ __forceinline__ unsigned long long key_mask(unsigned long long v, int row, int B, int R) {
  unsigned long long m = 0;
  const int end = min(row + K4_KT, R);
  for (int j = row / B; j * B < end; ++j) {   // (uniform)
    const int a = max(j * B - row, 0), b = min((j + 1) * B, end) - row;
    const unsigned long long bits = (b >= 64 ? ~0ull : (1ull << b) - 1) & ~((1ull << a) - 1);
    m |= (v >> j) & 1 ? bits : 0ull;
  }
  return m;
}

template <int D>
__global__ __launch_bounds__(K4_THREADS) void lane_attn_kv4_kernel(Kv4Params p) {
  constexpr int KS = D / 16;        // MFMA k-steps of S^T = K Q^T
  constexpr int DT = D / 32;        // 32-row tiles of O^T; scale blocks of a row
  constexpr int ROWB = 2 * D;       // bytes of a K or V row in LDS
  constexpr int TB = K4_KT * ROWB;
  constexpr int SEGS = D / 8;       // 16-byte segments of a row
  constexpr int NL = 2 * K4_KT * SEGS / K4_THREADS;   // bf16 segments per thread of a lane tile
  __shared__ __attribute__((aligned(1024))) char lds[4 * TB];   // two buffers of K then V

  const int hk = blockIdx.y, split = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, hh = lane >> 5, lgrp = lane >> 4, lg = lane & 15;
  const int x0 = blockIdx.x * 32 * K4_WAVES;
  const int x = x0 + w * 32 + r32;
  const bool ok = x < p.n_pairs;
  const int row = ok ? x / p.g : 0;
  const int hq = hk * p.g + (ok ? x - row * p.g : 0);
  unsigned long long my_vis = 0, wg_vis = 0;
  if (p.R > 0) {
    if (ok) my_vis = p.vis[row / p.B];
    const int l1 = (min(x0 + 32 * K4_WAVES, p.n_pairs) - 1) / p.g / p.B;
    for (int l = x0 / p.g / p.B; l <= l1; ++l) wg_vis |= p.vis[l];
  }

  bf16x8 qf[KS];
  {
    const uint16_t* qrow = p.q + ((size_t)row * p.Hq + hq) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = ok ? load_bf16x8(qrow + ks * 16 + hh * 8) : zero_bf16x8();
  }
  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[dt][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  // The key tiles of this split that some pair of the workgroup sees.
  const int t_end = (int)((long long)(split + 1) * p.n_tiles / p.n_split);
  auto next_visible = [&](int t) {
    for (; t < t_end && t >= p.n_pre; ++t) {
      const int row0 = (t - p.n_pre) * K4_KT;
      const int j0 = row0 / p.B, j1 = (min(row0 + K4_KT, p.R) - 1) / p.B;
      const unsigned long long upto = j1 >= 63 ? ~0ull : (1ull << (j1 + 1)) - 1;
      if (wg_vis & upto & ~((1ull << j0) - 1)) break;
    }
    return t;
  };

  // Staging.  Row r's 16-byte segment s sits in slot s ^ f(r): f_K puts the 16 rows
  // that one LDS cycle of the K reads serves into different banks, f_V the rows of
  // a transpose read.
  auto fk = [](int r) { return D == 128 ? r & 15 : (r >> 1) & 7; };
  auto fv = [](int r) {
    return D == 128 ? (4 * (r & 3)) ^ (2 * ((r >> 2) & 1)) : (4 * ((r >> 1) & 1)) ^ (2 * ((r >> 2) & 1));
  };
  struct Stage {
    i32x4 x[NL];      // lane tile: segments; prefix tile: x[0] the codes of 32 elements
    unsigned s;
  };
  constexpr int NP = 2 * K4_KT * DT;   // 16-byte pieces of codes of a tile (at D = 64 half the threads have none)
  const int prow = (tid & (NP / 2 - 1)) / DT, pblk = tid & (DT - 1), pv = tid / (NP / 2);
  auto load_tile = [&](Stage& g, int t) {
    if (t < p.n_pre) {
      const int r = t * K4_KT + prow;
      g.x[0] = i32x4{0, 0, 0, 0};
      g.s = 0;
      if (tid < NP && r < p.P) {
        const size_t at = (((size_t)pv * p.Hkv + hk) * p.cap + r) * DT + pblk;
        g.x[0] = reinterpret_cast<const i32x4*>(p.codes)[at];
        g.s = p.scales[at];
      }
    } else {
      const int r0 = (t - p.n_pre) * K4_KT;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int seg = tid + i * K4_THREADS;           // K rows, then V rows
        const int sr = (seg / SEGS) % K4_KT, sv = seg / (SEGS * K4_KT);
        const uint16_t* base = sv ? p.v_lane : p.k_lane;
        g.x[i] = i32x4{0, 0, 0, 0};
        if (r0 + sr < p.R)
          g.x[i] = *reinterpret_cast<const i32x4*>(base + ((size_t)(r0 + sr) * p.Hkv + hk) * D + (seg % SEGS) * 8);
      }
    }
  };
  auto store_tile = [&](const Stage& g, int t, int buf) {
    char* b = lds + buf * 2 * TB;
    if (t < p.n_pre) {
      if (tid < NP) {
        const float sc = mx4_scale(g.s);
        char* dst = b + pv * TB + prow * ROWB;
        const int f = pv ? fv(prow) : fk(prow);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *reinterpret_cast<bf16x8*>(dst + ((4 * pblk + j) ^ f) * 16) = mx4_bf16x8((unsigned)g.x[0][j], sc);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int seg = tid + i * K4_THREADS;
        const int sr = (seg / SEGS) % K4_KT, sv = seg / (SEGS * K4_KT);
        *reinterpret_cast<i32x4*>(b + sv * TB + sr * ROWB + ((seg % SEGS) ^ (sv ? fv(sr) : fk(sr))) * 16) = g.x[i];
      }
    }
  };
  const int ka = r32 * ROWB + ((hh ^ fk(r32)) * 16);   // K fragment (row r32, segment 2 ks + hh) at ka ^ 32 ks
  const int vr = 4 * hh + (lg >> 2);
  const int va = vr * ROWB + (((2 * (lgrp & 1) + ((lg & 3) >> 1)) ^ fv(vr)) * 16) + (lg & 1) * 8;

  auto compute = [&](int t, int buf) {
    const char* kt = lds + buf * 2 * TB;
    unsigned long long km = ~0ull;
    bool all = true;
    if (t >= p.n_pre) {
      km = key_mask(my_vis, (t - p.n_pre) * K4_KT, p.B, p.R);
      if (!__ballot(km != 0)) return;
      all = false;
    } else if (p.P - t * K4_KT < K4_KT) {
      km = (1ull << (p.P - t * K4_KT)) - 1;
      all = false;
    }
    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i) {
      const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kt + (ka ^ (32 * (i >> 1))) + (i & 1) * 32 * ROWB);
      s[i & 1] = mfma32x32x16(kf, qf[i >> 1], s[i & 1]);
    }
    if (!all) {
      const unsigned mw[2] = {(unsigned)km >> (4 * hh), (unsigned)(km >> 32) >> (4 * hh)};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kb][r] = mw[kb] & (1u << (8 * (r >> 2) + (r & 3))) ? s[kb][r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
    // (A pair that has seen no key yet keeps m_run = -inf, all of its P 0.)
    const float m_new = fmaxf(m_run, pair_max32(mx) * p.scale_log2);
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = exp2_fast(m_run - m_use);
    m_run = m_new;
    bf16x8 pk[4];
    float rs = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float pe = exp2_fast(fmaf(s[q >> 1][8 * (q & 1) + e], p.scale_log2, -m_use));
        rs += pe;
        pk[q][e] = (__bf16)pe;
      }
    l_run = l_run * alpha + pair_sum32(rs);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint16_t* a = reinterpret_cast<const uint16_t*>(kt + TB + (va ^ (64 * dt)) + 16 * q * ROWB);
        oacc[dt] = mfma32x32x16(cat_bf16x4(lds_read_tr16(a), lds_read_tr16(a + 8 * D)), pk[q], oacc[dt]);
      }
  };

  int t = next_visible((int)((long long)split * p.n_tiles / p.n_split));
  Stage g;
  if (t < t_end) {
    load_tile(g, t);
    store_tile(g, t, 0);
  }
  int tn = next_visible(t + 1);
  if (tn < t_end) load_tile(g, tn);
  __syncthreads();
  for (int buf = 0; t < t_end; buf ^= 1) {
    if (tn < t_end) store_tile(g, tn, buf ^ 1);
    const int t2 = next_visible(tn + 1);
    if (t2 < t_end) load_tile(g, t2);
    compute(t, buf);
    __syncthreads();
    t = tn;
    tn = t2;
  }

  if (!ok) return;
  const size_t orow = (size_t)row * p.Hq + hq;
  if (p.n_split == 1) {
    const float inv_l = 1.0f / l_run;
    uint16_t* op = p.o + orow * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        bf16x4 v4;
#pragma unroll
        for (int e = 0; e < 4; ++e) v4[e] = (__bf16)(oacc[dt][rg * 4 + e] * inv_l);
        *reinterpret_cast<bf16x4*>(op + dt * 32 + 8 * rg + 4 * hh) = v4;
      }
    if (p.lse && hh == 0) p.lse[orow] = (m_run + log2f(l_run)) * K4_LN2;
  } else {
    const size_t prow2 = (size_t)split * p.n_rows * p.Hq + orow;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        f32x4 v4;
#pragma unroll
        for (int e = 0; e < 4; ++e) v4[e] = oacc[dt][rg * 4 + e];
        *reinterpret_cast<f32x4*>(p.part_o + prow2 * D + dt * 32 + 8 * rg + 4 * hh) = v4;
      }
    if (hh == 0) {
      p.part_ml[prow2 * 2] = m_run;
      p.part_ml[prow2 * 2 + 1] = l_run;
    }
  }
}

// Combines the key splits of each (row, head): D / 4 lanes each, 4 elements a lane,
// in ascending order of the splits.
template <int D>
__global__ __launch_bounds__(256) void kv4_merge_kernel(const float* part_o, const float* part_ml, int n_rowheads,
                                                        int n_split, uint16_t* o, float* lse) {
  constexpr int LPR = D / 4;
  const int rh = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, sl = threadIdx.x % LPR;
  if (rh >= n_rowheads) return;
  float M = -INFINITY;
  for (int s = 0; s < n_split; ++s) M = fmaxf(M, part_ml[((size_t)s * n_rowheads + rh) * 2]);
  float L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < n_split; ++s) {
    const float2 ml = *reinterpret_cast<const float2*>(part_ml + ((size_t)s * n_rowheads + rh) * 2);
    const float wgt = exp2_fast(ml.x - M);   // (0 where the split saw no key)
    L += ml.y * wgt;
    const f32x4 v = *reinterpret_cast<const f32x4*>(part_o + ((size_t)s * n_rowheads + rh) * D + sl * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += v[e] * wgt;
  }
  const float inv = 1.0f / L;
  bf16x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (__bf16)(acc[e] * inv);
  *reinterpret_cast<bf16x4*>(o + (size_t)rh * D + sl * 4) = out;
  if (lse && sl == 0) lse[rh] = (M + log2f(L)) * K4_LN2;
}

// ------------------------------------------------------------------ host
struct Kv4Pass {
  int n_rows, n_pairs, q_wgs, n_pre, n_tiles, n_split;
  size_t ws;
};

// R: rows of all lane blocks (0: refreshed rows, which see the prefix alone).
static Kv4Pass kv4_pass(int n_rows, int R, int P, int Hq, int Hkv, int D) {
  Kv4Pass s{};
  s.n_rows = n_rows;
  s.n_pairs = n_rows * (Hq / Hkv);
  s.q_wgs = (s.n_pairs + 32 * K4_WAVES - 1) / (32 * K4_WAVES);
  s.n_pre = (P + K4_KT - 1) / K4_KT;
  s.n_tiles = s.n_pre + (R + K4_KT - 1) / K4_KT;
  s.n_split = 1;
  while (s.n_split < 64 && (long long)s.q_wgs * Hkv * s.n_split < 256 && s.n_tiles >= 4 * s.n_split) s.n_split *= 2;
  s.ws = s.n_split > 1 ? (size_t)s.n_split * n_rows * Hq * (D + 2) * sizeof(float) : 0;
  return s;
}

size_t kv4_workspace_bytes(int L, int B, int P, int Hq, int Hkv, int D, int n_refresh) {
  const size_t a = L > 0 ? kv4_pass(L * B, L * B, P, Hq, Hkv, D).ws : 0;
  const size_t b = n_refresh > 0 ? kv4_pass(n_refresh, 0, P, Hq, Hkv, D).ws : 0;
  return a > b ? a : b;
}

template <int D>
static hipError_t run_kv4_pass(Kv4Params p, const Kv4Pass& s, void* ws, hipStream_t stream) {
  p.n_rows = s.n_rows;
  p.n_pairs = s.n_pairs;
  p.n_pre = s.n_pre;
  p.n_tiles = s.n_tiles;
  p.n_split = s.n_split;
  p.part_o = static_cast<float*>(ws);
  p.part_ml = p.part_o + (size_t)s.n_split * s.n_rows * p.Hq * D;
  hipLaunchKernelGGL(lane_attn_kv4_kernel<D>, dim3(s.q_wgs, p.Hkv, s.n_split), dim3(K4_THREADS), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || s.n_split == 1) return e;
  const int nrh = s.n_rows * p.Hq, per = 256 / (D / 4);
  hipLaunchKernelGGL(kv4_merge_kernel<D>, dim3((nrh + per - 1) / per), dim3(256), 0, stream, p.part_o, p.part_ml, nrh,
                     s.n_split, p.o, p.lse);
  return hipGetLastError();
}

hipError_t launch_lane_attn_kv4(const uint16_t* q, const uint16_t* k_lane, const uint16_t* v_lane, uint8_t* codes,
                                uint8_t* scales, int cap, const unsigned long long* vis, int L, int B, int P, int Hq,
                                int Hkv, int D, float scale, const int32_t* refresh_idx, int n_refresh,
                                const uint16_t* q_ref, const uint16_t* k_ref, const uint16_t* v_ref, uint16_t* o_ref,
                                float* lse_ref, uint16_t* o, float* lse, void* ws, hipStream_t stream) {
  if (n_refresh > 0) {
    const hipError_t e = launch_kv4_store(k_ref, v_ref, refresh_idx, 0, n_refresh, P, cap, Hkv, D, codes, scales, stream);
    if (e != hipSuccess) return e;
  }
  Kv4Params p{};
  p.codes = codes;
  p.scales = scales;
  p.P = P;
  p.cap = cap;
  p.Hq = Hq;
  p.Hkv = Hkv;
  p.g = Hq / Hkv;
  p.scale_log2 = scale * 1.4426950408889634f;
  if (L > 0) {
    p.q = q;
    p.k_lane = k_lane;
    p.v_lane = v_lane;
    p.o = o;
    p.lse = lse;
    p.R = L * B;
    p.B = B;
    for (int i = 0; i < L; ++i) p.vis[i] = vis[i];
    const Kv4Pass s = kv4_pass(L * B, L * B, P, Hq, Hkv, D);
    const hipError_t e = D == 64 ? run_kv4_pass<64>(p, s, ws, stream) : run_kv4_pass<128>(p, s, ws, stream);
    if (e != hipSuccess) return e;
  }
  if (n_refresh > 0) {   // refreshed rows, over the updated prefix alone
    p.q = q_ref;
    p.k_lane = p.v_lane = nullptr;
    p.o = o_ref;
    p.lse = lse_ref;
    p.R = 0;
    p.B = 1;
    const Kv4Pass s = kv4_pass(n_refresh, 0, P, Hq, Hkv, D);
    return D == 64 ? run_kv4_pass<64>(p, s, ws, stream) : run_kv4_pass<128>(p, s, ws, stream);
  }
  return hipSuccess;
}

}  // namespace al
