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
// Keys.  First the prefix, then the rows of all lane blocks as one list, in tiles of
// 64 (the tile kernel: many query tiles, which share the converted keys of a
// workgroup) or units of 32 (the unit kernel: few query tiles, a wavefront to a unit;
// the token kernel: at most 16 pairs to a K/V head).  Prefix rows are read as codes (a
// 16-byte load per 32 elements) and converted to bf16, which is exact.  Both products
// are bf16 MFMAs with fp32 accumulation, transposed as in lane_attn.hip:
//     S^T = K Q^T,   O^T = V^T P^T  (V^T by LDS transpose reads).
// P is rounded to bf16 for the second product; the row sum adds the unrounded
// fp32 values, so the log-sum-exp keeps fp32 accuracy (adding the rounded ones
// would move it by up to 2^-9).
//
// Keys are split over blockIdx.z where there are few query tiles; the splits'
// partials are kept in fp32 and combined by kv4_merge_kernel.
//
// Per call (MI355X; keys x K/V heads, query heads, rows): the tile kernel 172 us for
// 2048 rows x 32 heads over 4096 keys and their lane blocks (about 0.85 PFLOP/s),
// the unit kernel 11.1 us for 128 rows x 32 heads over 512, 13.6 for 256 rows x 28 over
// 1024 x 4, the token kernel with its merge 11 us for a row of 28 over 32769 x 4 (17.8 MB).
#include <math.h>

#include "common.h"
#include "launch.h"
#include "mx4.h"

namespace al {

constexpr int K4_KT = 64;            // keys per tile of the tile kernel
constexpr int K4_UT = 32;            // keys per unit of the unit kernel
constexpr int K4_WAVES = 8;
constexpr int K4_THREADS = K4_WAVES * kWave;
constexpr float K4_LN2 = 0.6931471805599453f;
// A pair's reference maximum moves only when a tile's scores exceed it by more than
// this many powers of two, so O is rescaled in few tiles.
constexpr float K4_RESCALE_LOG2 = 8.0f;

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
  int n_pre, n_tiles, n_split;   // prefix tiles (units), all key tiles (units)
  float scale_log2;
  unsigned long long vis[64];    // bit j: lane block j visible to lane i
  // The lanes in the order in which their rows are listed as pairs (depth first, so
  // that neighbours share most of their ancestors), four to a word.
  unsigned order[16];
};
__device__ __forceinline__ int lane_at(const Kv4Params& p, int pos) { return (p.order[pos >> 2] >> (8 * (pos & 3))) & 255; }

// Bits of the KT lane rows from `row` on that a pair with visibility v sees.
template <int KT>
__device__ __forceinline__ unsigned long long key_mask(unsigned long long v, int row, int B, int R) {
  unsigned long long m = 0;
  const int end = min(row + KT, R);
  for (int j = row / B; j * B < end; ++j) {   // (uniform)
    const int a = max(j * B - row, 0), b = min((j + 1) * B, end) - row;
    const unsigned long long bits = (b >= 64 ? ~0ull : (1ull << b) - 1) & ~((1ull << a) - 1);
    m |= (v >> j) & 1 ? bits : 0ull;
  }
  return m;
}

// The query tile of 32 pairs from x0 + r32: this lane's pair.
struct Pair {
  bool ok;
  int row, hq;
  unsigned long long vis;
};
__device__ __forceinline__ Pair pair_at(const Kv4Params& p, int hk, int x) {
  Pair q;
  q.ok = x < p.n_pairs;
  const int r = q.ok ? x / p.g : 0;
  q.hq = hk * p.g + (q.ok ? x - r * p.g : 0);
  q.row = r;
  q.vis = 0;
  if (p.R > 0) {
    const int pos = r / p.B, l = lane_at(p, pos);
    q.row = l * p.B + r - pos * p.B;
    if (q.ok) q.vis = p.vis[l];
  }
  return q;
}
// Lane blocks that some pair of [x0, x1) sees.
__device__ __forceinline__ unsigned long long blocks_seen(const Kv4Params& p, int x0, int x1) {
  unsigned long long v = 0;
  if (p.R > 0 && x0 < p.n_pairs) {
    const int l1 = (min(x1, p.n_pairs) - 1) / p.g / p.B;
    for (int l = x0 / p.g / p.B; l <= l1; ++l) v |= p.vis[lane_at(p, l)];
  }
  return v;
}
// The first key tile at or after t, before t_end, that a workgroup with wg_vis sees.
template <int KT>
__device__ __forceinline__ int next_visible(const Kv4Params& p, unsigned long long wg_vis, int t, int t_end) {
  for (; t < t_end && t >= p.n_pre; ++t) {
    const int row0 = (t - p.n_pre) * KT;
    const int j0 = row0 / p.B, j1 = (min(row0 + KT, p.R) - 1) / p.B;
    const unsigned long long upto = j1 >= 63 ? ~0ull : (1ull << (j1 + 1)) - 1;
    if (wg_vis & upto & ~((1ull << j0) - 1)) break;
  }
  return t;
}

// ---------------------------------------------------------------- tile kernel
// Many query tiles: eight (or four) of them, a wavefront each, share the key tiles
// of a workgroup.  While prefix tile i is worked on, tile i + 1 is complete in LDS,
// tile i + 2 goes there from registers and tile i + 3 is loaded: each wavefront
// multiplies K of tile i + 1 while the softmax of tile i runs between the MFMAs, then
// V of tile i, with the conversion of tile i + 2 between the last of them.  Three
// buffers, one barrier a tile.
//
// Eight query tiles (TPW): every wavefront computes and stages an eighth of each
// tile.  Four: wavefronts 0 .. 3 compute, 4 .. 7 stage.  (Window of 2563 refreshed
// rows x 32 heads, its store included: 203 us with the computing wavefronts staging,
// 174 with the idle ones.)
//
// What bounds it: matrix (38% of the cycles) and vector work (conversion, exponentials;
// 40%) of a tile, which partly take turns, and the waits at its barrier; a lane tile
// does not overlap its two products with the next tile's and takes ~3.4 us, a prefix
// tile 1.9.  At D = 128 the first lane tile's rows, loaded before the last prefix tile's
// softmax, spill registers there (78 with eight query tiles, 46 with four), once a
// workgroup; neither loop spills.
template <int D, int TPW>
__global__ __launch_bounds__(K4_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2)))
void lane_attn_kv4_kernel(Kv4Params p) {
  constexpr int KS = D / 16;        // MFMA k-steps of S^T = K Q^T
  constexpr int DT = D / 32;        // 32-row tiles of O^T; scale blocks of a row
  constexpr int ROWB = 2 * D;       // bytes of a K or V row in LDS
  constexpr int TB = K4_KT * ROWB;
  constexpr int SEGS = D / 8;       // 16-byte segments of a row
  constexpr int ST = TPW == K4_WAVES ? K4_THREADS : K4_THREADS / 2;   // staging threads
  constexpr int NL = 2 * K4_KT * SEGS / ST;           // bf16 segments per staging thread of a lane tile
  constexpr int AHEAD = 4;          // K fragments read ahead
  // Fragments of q kept in LDS: at D = 128 the registers hold all but the last few (with all
  // of them the compiler spills some, and their reloads wait for every load in flight).
  constexpr int QL = D == 64 ? 0 : TPW == K4_WAVES ? 3 : 2, QR = KS - QL;
  __shared__ __attribute__((aligned(1024))) char lds[6 * TB + QL * K4_WAVES * 1024];   // three buffers of K then V, q

  const int hk = blockIdx.y, split = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, hh = lane >> 5, lgrp = lane >> 4, lg = lane & 15;
  const int x0 = blockIdx.x * 32 * TPW;
  const bool computing = w < TPW && x0 + w * 32 < p.n_pairs;
  constexpr bool staging = TPW == K4_WAVES;   // (of the loops below; with four query tiles wavefronts 4 .. 7 have their own)
  const Pair pr = pair_at(p, hk, w < TPW ? x0 + w * 32 + r32 : p.n_pairs);
  const unsigned long long wg_vis = blocks_seen(p, x0, x0 + 32 * TPW);

  bf16x8 qr[QR];
  bf16x8* const ql = reinterpret_cast<bf16x8*>(lds + 6 * TB) + w * kWave + lane;   // (this lane's own)
  {
    const uint16_t* qrow = p.q + ((size_t)pr.row * p.Hq + pr.hq) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 v = pr.ok ? load_bf16x8(qrow + ks * 16 + hh * 8) : zero_bf16x8();
      if (ks < QR) qr[ks] = v;
      else ql[(ks - QR) * K4_THREADS] = v;
    }
  }
  auto qf = [&](int ks) -> bf16x8 { return ks < QR ? qr[ks < QR ? ks : 0] : ql[(ks - QR) * K4_THREADS]; };
  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[dt][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  // Staging.  Row r's 16-byte segment s sits in slot s ^ f(r): f_K puts the 16 rows
  // that one LDS cycle of the K reads serves into different banks, f_V the rows of
  // a transpose read; f_V's low bit parts the neighbouring rows of a store.
  auto fk = [](int r) { return D == 128 ? r & 15 : (r >> 1) & 7; };
  auto fv = [](int r) {
    return D == 128 ? (4 * (r & 3)) ^ (2 * ((r >> 2) & 1)) ^ (r & 1) : (5 * ((r >> 1) & 1)) ^ (2 * ((r >> 2) & 1));
  };
  struct Codes {      // of a prefix tile: 32 elements
    i32x4 x;
    unsigned s;
  };
  // (At D = 64 and eight query tiles there are 256 pieces: threads 256 .. 511 do those
  // of 0 .. 255 again.  A row past the prefix repeats the last one; its P is 0.  No
  // branches: where two paths meet the compiler waits for LDS as if the longer one
  // had been taken.)
  constexpr int NP = 2 * K4_KT * DT;   // 16-byte pieces of codes of a tile
  constexpr int NC = NP > ST ? NP / ST : 1;   // per staging thread: 1, or 2 (K and V)
  const int pidx = tid & (NP / 2 - 1), prow = pidx / DT, pblk = pidx & (DT - 1);
  const int pv = NC == 2 ? 0 : (w / (NP / 2 / kWave)) & 1;   // K or V, the same for a whole wavefront
  auto load_codes = [&](Codes (&g)[NC], int t) {
    const unsigned off = min(prow, p.P - 1 - t * K4_KT) * DT + pblk;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const size_t at = (((size_t)(pv + c) * p.Hkv + hk) * p.cap + (size_t)t * K4_KT) * DT;   // (uniform)
      g[c].x = reinterpret_cast<const i32x4*>(p.codes)[at + off];
      g[c].s = p.scales[at + off];
    }
  };
  const int pdst = pv * TB + prow * ROWB, pf = pv ? fv(prow) : fk(prow);
  auto store_piece = [&](const Codes& g, int dst, int f, int buf, int j) {   // j = 0..3
    *reinterpret_cast<bf16x8*>(lds + buf * 2 * TB + dst + ((4 * pblk + j) ^ f) * 16) =
        mx4_bf16x8((unsigned)g.x[j], mx4_scale(g.s));
  };
  auto store_codes = [&](const Codes (&g)[NC], int buf) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) store_piece(g[c], pdst + c * TB, c ? fv(prow) : pf, buf, j);
  };
  const int sid = tid & (ST - 1);
  auto load_rows = [&](i32x4 (&x)[NL], int t) {   // of lane tile t: K rows, then V rows
    const int r0 = (t - p.n_pre) * K4_KT;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int seg = sid + i * ST;
      const int sr = (seg / SEGS) % K4_KT, sv = seg / (SEGS * K4_KT);
      const uint16_t* base = sv ? p.v_lane : p.k_lane;
      // (A row past the last repeats it; nobody sees it.)
      x[i] = *reinterpret_cast<const i32x4*>(base + ((size_t)min(r0 + sr, p.R - 1) * p.Hkv + hk) * D + (seg % SEGS) * 8);
    }
  };
  auto store_rows = [&](const i32x4 (&x)[NL], int buf) {
    char* b = lds + buf * 2 * TB;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int seg = sid + i * ST;
      const int sr = (seg / SEGS) % K4_KT, sv = seg / (SEGS * K4_KT);
      *reinterpret_cast<i32x4*>(b + sv * TB + sr * ROWB + ((seg % SEGS) ^ (sv ? fv(sr) : fk(sr))) * 16) = x[i];
    }
  };
  const int ka = r32 * ROWB + ((hh ^ fk(r32)) * 16);   // K fragment (row r32, segment 2 ks + hh) at ka ^ 32 ks
  const int vr = 4 * hh + (lg >> 2);
  const int va = vr * ROWB + (((2 * (lgrp & 1) + ((lg & 3) >> 1)) ^ fv(vr)) * 16) + (lg & 1) * 8;

  struct Scores {
    f32x16 s[2];   // the two 32-key halves
  };
  auto kread = [&](int buf, int i) {
    return *reinterpret_cast<const bf16x8*>(lds + buf * 2 * TB + (ka ^ (32 * (i >> 1))) + (i & 1) * 32 * ROWB);
  };
  auto vfrag = [&](int buf, int ks2, int dt, int half = 0) {
    const uint16_t* a = reinterpret_cast<const uint16_t*>(lds + buf * 2 * TB + TB + (va ^ (64 * dt)) +
                                                          (16 * ks2 + 32 * half) * ROWB);
    return cat_bf16x4(lds_read_tr16(a), lds_read_tr16(a + 8 * D));
  };
  const f32x16 zero16 = {};
  auto qk = [&](Scores& sc, int buf) {
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i)
      sc.s[i & 1] = mfma32x32x16(kread(buf, i), qf(i >> 1), i < 2 ? zero16 : sc.s[i & 1]);
  };
  auto qk_half = [&](Scores& sc, int buf, int half) {   // keys 32 half .. 32 half + 31, into s[0]
    const char* kt = lds + buf * 2 * TB + half * 32 * ROWB;
    f32x16 s1 = zero16;   // (two chains)
    sc.s[0] = zero16;
#pragma unroll
    for (int i = 0; i < KS; i += 2) {
      sc.s[0] = mfma32x32x16(*reinterpret_cast<const bf16x8*>(kt + (ka ^ (32 * i))), qf(i), sc.s[0]);
      s1 = mfma32x32x16(*reinterpret_cast<const bf16x8*>(kt + (ka ^ (32 * (i + 1)))), qf(i + 1), s1);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) sc.s[0][r] += s1[r];
  };
  auto mask = [&](auto nh_tag, Scores& sc, unsigned long long km) {   // (of NH = 1 or 2 halves)
    const unsigned mw[2] = {(unsigned)km >> (4 * hh), (unsigned)(km >> 32) >> (4 * hh)};
#pragma unroll
    for (int kb = 0; kb < decltype(nh_tag)::value; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc.s[kb][r] = mw[kb] & (1u << (8 * (r >> 2) + (r & 3))) ? sc.s[kb][r] : -INFINITY;
  };
  auto max_piece = [&](float mx, const Scores& sc, int q) {   // q = 0..3: 8 scores
#pragma unroll
    for (int r = 0; r < 8; ++r) mx = fmaxf(mx, sc.s[q >> 1][8 * (q & 1) + r]);
    return mx;
  };
  // Returns the factor on O.  (A pair that has seen no key yet keeps m_run = -inf; its
  // exponents are then taken from 0, all of its P are 0.)
  auto new_max = [&](float mx, float& m_use) {
    const float m_tile = pair_max32(mx) * p.scale_log2;
    const float m_new = m_tile > m_run + K4_RESCALE_LOG2 ? m_tile : m_run;
    m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = exp2_fast(m_run - m_use);
    m_run = m_new;
    return alpha;
  };
  auto exp_pair = [&](const Scores& sc, bf16x8* pk, float m_use, float& rs, int q) {   // q = 0..15
    const int ks2 = q >> 2, e = 2 * (q & 3), r = 8 * (ks2 & 1) + e;
    const float p0 = exp2_fast(fmaf(sc.s[ks2 >> 1][r], p.scale_log2, -m_use));
    const float p1 = exp2_fast(fmaf(sc.s[ks2 >> 1][r + 1], p.scale_log2, -m_use));
    pk[ks2][e] = (__bf16)p0;
    pk[ks2][e + 1] = (__bf16)p1;
    rs += p0 + p1;
  };
  auto rescale = [&](float alpha) {   // (O only when some pair's reference has moved; otherwise alpha is 1)
    if (__builtin_amdgcn_read_exec() & __ballot(alpha != 1.0f)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
    }
  };
  // O^T += V^T P^T, the second half of P's exponentials between the MFMAs of the
  // first two steps and, where a prefix tile is to be stored, its pieces between
  // those of the last two.  vf[0] holds the first step's fragments.
  // (NH = 1: the 32 keys of one half alone, their exponentials done.)
  auto pv_product = [&](auto nh_tag, auto store_tag, const Scores& sc, bf16x8* pk, bf16x8 (*vf)[DT], float m_use,
                        float alpha, float rs, int buf, int half, const Codes (&g)[NC], int sbuf) {
    constexpr int NH = decltype(nh_tag)::value;
#pragma unroll
    for (int ks2 = 0; ks2 < 2 * NH; ++ks2) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        if (ks2 < 2 * NH - 1) vf[(ks2 + 1) & 1][dt] = vfrag(buf, ks2 + 1, dt, half);
        oacc[dt] = mfma32x32x16(vf[ks2 & 1][dt], pk[ks2], oacc[dt]);
        if (NH == 2 && ks2 < 2) {
#pragma unroll
          for (int q = 0; q < 4 / DT; ++q) exp_pair(sc, pk, m_use, rs, 8 + ks2 * 4 + dt * (4 / DT) + q);
        } else if (decltype(store_tag)::value && (dt & (DT / 2 - 1)) == 0) {
          store_piece(g[0], pdst, pf, sbuf, 2 * (ks2 - 2) + dt / (DT / 2));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    l_run = l_run * alpha + pair_sum32(rs);
  };
  // Q K^T of the tile in buffer bq into nxt, with the max and the first half of the
  // exponentials of cur between its MFMAs; then cur's P V.
  auto hot_tile = [&](const Scores& cur, Scores& nxt, int bq, int bv, const Codes (&g)[NC], int sbuf) {
    bf16x8 kf[2 * KS], pk[4], vf[2][DT];
    float mx = -INFINITY, m_use = 0.f, alpha = 1.f, rs = 0.f;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) kf[i] = kread(bq, i);
    __builtin_amdgcn_sched_barrier(0);
    constexpr int MX = KS / 2;                 // MFMAs with a piece of the max
    constexpr int EX = 2 * KS - MX;            // and with exponentials
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i) {
      if (i + AHEAD < 2 * KS) kf[i + AHEAD] = kread(bq, i + AHEAD);
      else if (i + DT >= 2 * KS) vf[0][i + DT - 2 * KS] = vfrag(bv, 0, i + DT - 2 * KS);
      nxt.s[i & 1] = mfma32x32x16(kf[i], qf(i >> 1), i < 2 ? zero16 : nxt.s[i & 1]);
      if (i < MX) {
#pragma unroll
        for (int q = 0; q < 4 / MX; ++q) mx = max_piece(mx, cur, i * (4 / MX) + q);
        if (i == MX - 1) alpha = new_max(mx, m_use);
      } else {
        const int j = i - MX;
#pragma unroll
        for (int q = 8 * j / EX; q < 8 * (j + 1) / EX; ++q) {
          exp_pair(cur, pk, m_use, rs, q);
          // (Left alone, the compiler sinks these past the branch below to their use.)
          const i32x4 pq = __builtin_bit_cast(i32x4, pk[q >> 2]);
          asm volatile("" ::"v"(pq[q & 3]), "v"(rs));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    rescale(alpha);
    pv_product(IntTag<2>{}, IntTag<TPW == K4_WAVES>{}, cur, pk, vf, m_use, alpha, rs, bv, 0, g, sbuf);
  };
  auto cold_tile = [&](auto nh_tag, const Scores& cur, int bv, int half) {   // softmax and P V alone
    constexpr int NH = decltype(nh_tag)::value;
    bf16x8 pk[4], vf[2][DT];
    float mx = -INFINITY, m_use, rs = 0.f;
#pragma unroll
    for (int q = 0; q < 2 * NH; ++q) mx = max_piece(mx, cur, q);
    const float alpha = new_max(mx, m_use);
#pragma unroll
    for (int q = 0; q < 8; ++q) exp_pair(cur, pk, m_use, rs, q);
    rescale(alpha);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) vf[0][dt] = vfrag(bv, 0, dt, half);
    __builtin_amdgcn_sched_barrier(0);
    const Codes none[NC] = {};
    pv_product(nh_tag, IntTag<0>{}, cur, pk, vf, m_use, alpha, rs, bv, half, none, 0);
  };

  // This split's tiles: prefix tiles [t0, pe), then the lane tiles that some pair of
  // the workgroup sees.
  const int t0 = (int)((long long)split * p.n_tiles / p.n_split);
  const int t_end = (int)((long long)(split + 1) * p.n_tiles / p.n_split);
  const int pe = min(t_end, p.n_pre);
  i32x4 rows[NL];
  const int lt0 = next_visible<K4_KT>(p, wg_vis, max(p.n_pre, t0), t_end);   // first lane tile
  if (TPW < K4_WAVES && w >= TPW) {   // stages only: the barriers of the loops below
    if (t0 < pe) {
      Codes g[NC];
      load_codes(g, t0);
      store_codes(g, 0);
      load_codes(g, min(t0 + 1, pe - 1));
      store_codes(g, 1);
      load_codes(g, min(t0 + 2, pe - 1));
      __syncthreads();
      int sbuf = 2;
      for (int t = t0; t + 1 < pe; ++t) {
        store_codes(g, sbuf);
        load_codes(g, min(t + 3, pe - 1));
        sbuf = sbuf == 2 ? 0 : sbuf + 1;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      }
      if (lt0 < t_end) load_rows(rows, lt0);
      __syncthreads();
    } else if (lt0 < t_end) {
      load_rows(rows, lt0);
    }
    if (lt0 < t_end) store_rows(rows, 0);
    __syncthreads();
    for (int t = lt0, buf = 0; t < t_end; buf ^= 1) {
      t = next_visible<K4_KT>(p, wg_vis, t + 1, t_end);
      if (t < t_end) {
        load_rows(rows, t);
        store_rows(rows, buf ^ 1);
      }
      __syncthreads();
    }
    return;
  }
  if (t0 < pe) {
    auto third = [](int x) { return x >= 3 ? x - 3 : x; };
    Codes g[NC];
    if (staging) {
      load_codes(g, t0);
      store_codes(g, 0);
      load_codes(g, min(t0 + 1, pe - 1));
      store_codes(g, 1);
      load_codes(g, min(t0 + 2, pe - 1));
    }
    __syncthreads();
    Scores sa, sb;
    if (computing) qk(sa, 0);
    int t = t0, buf = 0;
    auto step = [&](Scores& cur, Scores& nxt) {   // t + 1 < pe
      // (Past the last tile its codes are stored once more, in a buffer that nobody reads.)
      const int sbuf = third(buf + 2);
      if (computing) hot_tile(cur, nxt, third(buf + 1), buf, g, sbuf);
      else if (staging) store_codes(g, sbuf);
      if (staging) load_codes(g, min(t + 3, pe - 1));
      // (__syncthreads would wait for the loads too)
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      ++t;
      buf = third(buf + 1);
    };
    auto last = [&](Scores& cur) {
      if (computing) {
        if (p.P - t * K4_KT < K4_KT) mask(IntTag<2>{}, cur, (1ull << (p.P - t * K4_KT)) - 1);
        cold_tile(IntTag<2>{}, cur, buf, 0);
      }
    };
    while (t + 2 < pe) {   // (two at a time: the scores keep their registers)
      step(sa, sb);
      step(sb, sa);
    }
    if (t + 1 < pe) {
      step(sa, sb);
      if (staging && lt0 < t_end) load_rows(rows, lt0);
      last(sb);
    } else {
      if (staging && lt0 < t_end) load_rows(rows, lt0);
      last(sa);
    }
    __syncthreads();
  } else if (staging && lt0 < t_end) {
    load_rows(rows, lt0);
  }
  // Lane tiles, one after another in two buffers.
  if (staging && lt0 < t_end) store_rows(rows, 0);
  __syncthreads();
  for (int t = lt0, buf = 0; t < t_end; buf ^= 1) {
    const int tn = next_visible<K4_KT>(p, wg_vis, t + 1, t_end);
    if (staging && tn < t_end) load_rows(rows, tn);
    if (computing) {
      const unsigned long long km = key_mask<K4_KT>(pr.vis, (t - p.n_pre) * K4_KT, p.B, p.R);
      // A half that no pair of the wavefront sees is left out.
      const bool lo = __ballot((unsigned)km != 0) != 0, hi = __ballot((unsigned)(km >> 32) != 0) != 0;
      Scores sc;
      if (lo && hi) {
        qk(sc, buf);
        if (__ballot(km != ~0ull)) mask(IntTag<2>{}, sc, km);
        cold_tile(IntTag<2>{}, sc, buf, 0);
      } else if (lo || hi) {
        qk_half(sc, buf, hi);
        const unsigned kh = (unsigned)(hi ? km >> 32 : km);
        if (__ballot(kh != ~0u)) mask(IntTag<1>{}, sc, kh);
        cold_tile(IntTag<1>{}, sc, buf, hi);
      }
    }
    if (staging && tn < t_end) store_rows(rows, buf ^ 1);
    __syncthreads();
    t = tn;
  }

  if (!computing || !pr.ok) return;
  const size_t orow = (size_t)pr.row * p.Hq + pr.hq;
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

// ---------------------------------------------------------------- unit kernel
// Few query tiles: a workgroup serves one, and its eight wavefronts share out the
// keys in units of 32, each with a softmax state of its own (combined in LDS at the
// end), so the loop has no barrier.  K needs no LDS: lane (key, half) of a wavefront
// takes the 16 bytes of a scale block, converts them and has its operand of four
// MFMA steps (q's fragments follow the same order of d).  V is converted into an LDS
// region of the wavefront's own for the transpose reads.
//
// What bounds it: latency.  A call with one unit to a wavefront takes 6 us (launch, q,
// one unit, the combination), every further round of units ~1.2 with an idle chip, 1.7
// with a workgroup on nearly every compute unit (256 rows x 28 heads over 1024 keys).
// Codes two or three units ahead do not help.
template <int D>
__global__ __launch_bounds__(K4_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2)))
void lane_attn_kv4_unit_kernel(Kv4Params p) {
  constexpr int KS = D / 16, DT = D / 32, DC = D / 64;
  constexpr int VROW = D + 32;              // elements of a V row in LDS
  constexpr int WBUF = K4_UT * VROW;        // of a wavefront
  constexpr int OSTR = D + 4;               // fp32 per row of the merge area
  constexpr int LDSB = K4_WAVES * 32 * (OSTR + 2) * 4 > K4_WAVES * WBUF * 2 ? K4_WAVES * 32 * (OSTR + 2) * 4
                                                                           : K4_WAVES * WBUF * 2;
  __shared__ __attribute__((aligned(16))) char lds[LDSB];

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, hh = lane >> 5, lgrp = lane >> 4, lg = lane & 15;
  const int hk = blockIdx.x % p.Hkv, x0 = (int)(blockIdx.x / p.Hkv) * 32, split = blockIdx.z;
  uint16_t* v_s = reinterpret_cast<uint16_t*>(lds) + w * WBUF;
  const Pair pr = pair_at(p, hk, x0 + r32);
  const unsigned long long wg_vis = blocks_seen(p, x0, x0 + 32);

  // q's fragment c, j: elements 64 c + 32 hh + 8 j + (0..7).
  bf16x8 qf[KS];
  {
    const uint16_t* qrow = p.q + ((size_t)pr.row * p.Hq + pr.hq) * D + 32 * hh;
#pragma unroll
    for (int i = 0; i < KS; ++i) qf[i] = pr.ok ? load_bf16x8(qrow + 64 * (i >> 2) + 8 * (i & 3)) : zero_bf16x8();
  }
  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[dt][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  struct Codes {
    i32x4 x[2 * DC];   // of K, then of V: block 2 c + hh of the key's row
    unsigned ks, vs;   // scale bytes of the rows
  };
  const size_t vplane = (size_t)p.Hkv * p.cap;
  auto load_codes = [&](Codes& g, int u) {
    const int key = min(u * K4_UT + r32, p.P - 1);   // (a key past the prefix repeats the last one, with P = 0)
    const size_t row = (size_t)hk * p.cap + key;
    const i32x4* kc = reinterpret_cast<const i32x4*>(p.codes) + row * DT + hh;
    const i32x4* vc = kc + vplane * DT;
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      g.x[c] = kc[2 * c];
      g.x[DC + c] = vc[2 * c];
    }
    if (DT == 4) {
      g.ks = reinterpret_cast<const unsigned*>(p.scales)[row];
      g.vs = reinterpret_cast<const unsigned*>(p.scales)[vplane + row];
    } else {
      g.ks = reinterpret_cast<const uint16_t*>(p.scales)[row];
      g.vs = reinterpret_cast<const uint16_t*>(p.scales)[vplane + row];
    }
  };
  // V's row of this lane's key, piece c, j.  (The 16-byte segments of rows 4 .. 7 of
  // every eight change places in pairs: rows r and r + 4 start in the same bank.)
  auto put_v = [&](int c, int j, bf16x8 v) {
    *reinterpret_cast<bf16x8*>(&v_s[r32 * VROW + 64 * c + 32 * hh + 8 * (j ^ ((r32 >> 2) & 1))]) = v;
  };
  // (The region is this wavefront's own: its LDS operations complete in issue order;
  // the fences order the compiler alone.)
  auto fence = []() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  // A unit's scores are there and V is in LDS; km: the keys that the pair sees.
  auto update = [&](f32x16 s, unsigned km) {
    if (__ballot(km != ~0u)) {
      const unsigned mw = km >> (4 * hh);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = mw & (1u << (8 * (r >> 2) + (r & 3))) ? s[r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
    const float m_tile = pair_max32(mx) * p.scale_log2;
    const float m_new = m_tile > m_run + K4_RESCALE_LOG2 ? m_tile : m_run;
    const float m_use = m_new == -INFINITY ? 0.f : m_new;   // (no key seen yet: all P are 0)
    const float alpha = exp2_fast(m_run - m_use);
    m_run = m_new;
    float rs = 0.f;
    bf16x8 pk[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float pe = exp2_fast(fmaf(s[r], p.scale_log2, -m_use));
      rs += pe;
      pk[r >> 3][r & 7] = (__bf16)pe;
    }
    l_run = l_run * alpha + pair_sum32(rs);
    if (__ballot(alpha != 1.0f)) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
    }
#pragma unroll
    for (int ks2 = 0; ks2 < 2; ++ks2)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const uint16_t* va = &v_s[(16 * ks2 + 4 * hh + (lg >> 2)) * VROW + dt * 32 + 16 * (lgrp & 1) + 4 * ((lg & 3) ^ (2 * hh))];
        oacc[dt] = mfma32x32x16(cat_bf16x4(lds_read_tr16(va), lds_read_tr16(va + 8 * VROW)), pk[ks2], oacc[dt]);
      }
  };

  // Wavefront w takes every eighth unit of the split's share, the next prefix unit's
  // loads in flight.
  const int u0 = (int)((long long)split * p.n_tiles / p.n_split);
  const int u_end = (int)((long long)(split + 1) * p.n_tiles / p.n_split);
  auto seen = [&](int u) {   // this unit or a later one of the wavefront that the tile sees
    for (; u < u_end && u >= p.n_pre; u += K4_WAVES) {
      const int row0 = (u - p.n_pre) * K4_UT;
      const int j0 = row0 / p.B, j1 = (min(row0 + K4_UT, p.R) - 1) / p.B;
      const unsigned long long upto = j1 >= 63 ? ~0ull : (1ull << (j1 + 1)) - 1;
      if (wg_vis & upto & ~((1ull << j0) - 1)) break;
    }
    return u;
  };
  // The lane units come first: their rows arrive while q does.
  const int pe = min(u_end, p.n_pre);
  int u = u0 + w;
  Codes g;
  if (u < pe) load_codes(g, u);
  for (int v = seen(u < p.n_pre ? u + (p.n_pre - u + K4_WAVES - 1) / K4_WAVES * K4_WAVES : u); v < u_end; v = seen(v + K4_WAVES)) {
    const int r = min((v - p.n_pre) * K4_UT + r32, p.R - 1);
    const size_t at = ((size_t)r * p.Hkv + hk) * D + 32 * hh;
    bf16x8 kf[KS], vf[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      kf[i] = load_bf16x8(p.k_lane + at + 64 * (i >> 2) + 8 * (i & 3));
      vf[i] = load_bf16x8(p.v_lane + at + 64 * (i >> 2) + 8 * (i & 3));
    }
    const unsigned km = (unsigned)key_mask<K4_UT>(pr.vis, (v - p.n_pre) * K4_UT, p.B, p.R);
    fence();
    f32x16 s = {};
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      put_v(i >> 2, i & 3, vf[i]);
      s = mfma32x32x16(kf[i], qf[i], s);
    }
    fence();
    update(s, km);
  }
  while (u < pe) {
    fence();
    f32x16 s = {};
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      const float ksc = mx4_scale((g.ks >> (16 * c + 8 * hh)) & 255), vsc = mx4_scale((g.vs >> (16 * c + 8 * hh)) & 255);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        put_v(c, j, mx4_bf16x8((unsigned)g.x[DC + c][j], vsc));
        s = mfma32x32x16(mx4_bf16x8((unsigned)g.x[c][j], ksc), qf[4 * c + j], s);
      }
    }
    fence();
    const int left = p.P - u * K4_UT;
    u += K4_WAVES;
    if (u < pe) load_codes(g, u);
    update(s, left < K4_UT ? (1u << left) - 1 : ~0u);
  }

  // Combine the wavefronts' states, in ascending order.
  __syncthreads();
  float* o_s = reinterpret_cast<float*>(lds);
  float* ml_s = o_s + K4_WAVES * 32 * OSTR;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg)
      *reinterpret_cast<float4*>(&o_s[(w * 32 + r32) * OSTR + dt * 32 + 8 * rg + 4 * hh]) =
          make_float4(oacc[dt][rg * 4 + 0], oacc[dt][rg * 4 + 1], oacc[dt][rg * 4 + 2], oacc[dt][rg * 4 + 3]);
  if (hh == 0) {
    ml_s[(w * 32 + r32) * 2 + 0] = m_run;
    ml_s[(w * 32 + r32) * 2 + 1] = l_run;
  }
  __syncthreads();
  constexpr int TPR = D / 8;                  // threads per pair
  constexpr int RPP = K4_THREADS / TPR;       // pairs per pass
  const int d0 = (tid % TPR) * 8;
  for (int r = tid / TPR; r < 32 && x0 + r < p.n_pairs; r += RPP) {
    float mw[K4_WAVES], M = -INFINITY;
#pragma unroll
    for (int i = 0; i < K4_WAVES; ++i) {
      mw[i] = ml_s[(i * 32 + r) * 2];
      M = fmaxf(M, mw[i]);
    }
    float L = 0.f, acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
    for (int i = 0; i < K4_WAVES; ++i) {
      const float wgt = mw[i] == -INFINITY ? 0.f : exp2_fast(mw[i] - M);
      L += ml_s[(i * 32 + r) * 2 + 1] * wgt;
      const f32x4 a = *reinterpret_cast<const f32x4*>(&o_s[(i * 32 + r) * OSTR + d0]);
      const f32x4 b = *reinterpret_cast<const f32x4*>(&o_s[(i * 32 + r) * OSTR + d0 + 4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[e] += a[e] * wgt;
        acc[4 + e] += b[e] * wgt;
      }
    }
    const Pair out_pair = pair_at(p, hk, x0 + r);
    const size_t orow = (size_t)out_pair.row * p.Hq + out_pair.hq;
    if (p.n_split == 1) {
      const float inv = 1.0f / L;
      bf16x8 out;
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] = (__bf16)(acc[e] * inv);
      *reinterpret_cast<bf16x8*>(p.o + orow * D + d0) = out;
      if (p.lse && d0 == 0) p.lse[orow] = (M + log2f(L)) * K4_LN2;
    } else {
      const size_t at = (size_t)split * p.n_rows * p.Hq + orow;
      *reinterpret_cast<f32x4*>(p.part_o + at * D + d0) = f32x4{acc[0], acc[1], acc[2], acc[3]};
      *reinterpret_cast<f32x4*>(p.part_o + at * D + d0 + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
      if (d0 == 0) {
        p.part_ml[at * 2] = M;
        p.part_ml[at * 2 + 1] = L;
      }
    }
  }
}

// ---------------------------------------------------------------- token kernel
// At most 16 pairs to a K/V head (a single token of a grouped-query model, a few
// tokens of another): the unit kernel on 16x16x32 MFMAs, whose scores and sums take
// half the registers and vector work, with sixteen wavefronts to a workgroup.  Lane
// (key r, quarter b) takes D/4 elements of a key's row: 16 bytes of codes at D = 128,
// 1 KB a wavefront; q's fragments follow that order of d.  The scores
//     S^T = K Q^T: lane (pair, b) has keys 16 t + 4 b + (0..3) of the unit's halves t
// are the second product's operand as they stand, and V's comes from two transpose
// reads of those keys' rows.  (A row of 28 heads over 32769 keys: 8.5 us, 2.1 TB/s, of
// which ~6 are the chain of one unit; over 131072 keys 18.7 with the merge, 3.8 TB/s.)
constexpr int K4_TW = 16;   // wavefronts
template <int D>
__global__ __launch_bounds__(K4_TW * kWave) void lane_attn_kv4_token_kernel(Kv4Params p) {
  constexpr int EL = D / 4, KS = EL / 8, DT = D / 32, OT = D / 16;
  constexpr int VROWB = 2 * D + 32;         // bytes of a V row in LDS (4 rows of a transpose read in different banks)
  constexpr int OSTR = D + 4;               // fp32 per pair of the merge area
  constexpr int WB = K4_UT * VROWB;
  constexpr int MB = K4_TW * 16 * (OSTR + 2) * 4;
  __shared__ __attribute__((aligned(16))) char lds[MB > K4_TW * WB ? MB : K4_TW * WB];

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kb = lane >> 4;
  const int hk = blockIdx.x, split = blockIdx.z;
  char* const v_s = lds + w * WB;
  const Pair pr = pair_at(p, hk, r16);
  const unsigned long long wg_vis = blocks_seen(p, 0, 16);

  bf16x8 qf[KS];
  {
    const uint16_t* qrow = p.q + ((size_t)pr.row * p.Hq + pr.hq) * D + kb * EL;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = pr.ok ? load_bf16x8(qrow + 8 * s) : zero_bf16x8();
  }
  f32x4 oacc[OT];
#pragma unroll
  for (int d = 0; d < OT; ++d) oacc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;

  struct Codes {
    unsigned k[2][KS], v[2][KS], ks[2], vs[2];   // of the unit's two 16-key halves
  };
  const size_t vplane = (size_t)p.Hkv * p.cap;
  auto load_codes = [&](Codes& g, int u) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = min(u * K4_UT + 16 * t + r16, p.P - 1);   // (a key past the prefix repeats the last one, with P = 0)
      const size_t row = (size_t)hk * p.cap + key;
      const uint8_t* kc = p.codes + row * (D / 2) + kb * (EL / 2);
      __builtin_memcpy(g.k[t], __builtin_assume_aligned(kc, EL / 2), EL / 2);
      __builtin_memcpy(g.v[t], __builtin_assume_aligned(kc + vplane * (D / 2), EL / 2), EL / 2);
      const uint8_t* sc = p.scales + row * DT + kb * EL / 32;
      g.ks[t] = sc[0];
      g.vs[t] = sc[vplane * DT];
    }
  };
  f32x4 s[2];
  auto put_v = [&](int t, int j, bf16x8 v) {
    *reinterpret_cast<bf16x8*>(v_s + (16 * t + r16) * VROWB + (kb * EL + 8 * j) * 2) = v;
  };
  // (The region is this wavefront's own: its LDS operations complete in issue order;
  // the fences order the compiler alone.)
  auto fence = []() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  // The scores s are there and V is in LDS; km: the keys of the unit that the pair sees.
  auto update = [&](unsigned km) {
    if (__ballot(km != ~0u)) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[t][r] = (km >> (16 * t + 4 * kb + r)) & 1 ? s[t][r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[t][r]);
    const float m_tile = quad_max(mx) * p.scale_log2;
    const float m_new = m_tile > m_run + K4_RESCALE_LOG2 ? m_tile : m_run;
    const float m_use = m_new == -INFINITY ? 0.f : m_new;   // (no key seen yet: all P are 0)
    const float alpha = exp2_fast(m_run - m_use);
    m_run = m_new;
    float rs = 0.f;
    bf16x8 pk;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float pe = exp2_fast(fmaf(s[t][r], p.scale_log2, -m_use));
        rs += pe;
        pk[4 * t + r] = (__bf16)pe;
      }
    l_run = l_run * alpha + quad_sum(rs);
    if (__ballot(alpha != 1.0f)) {
#pragma unroll
      for (int d = 0; d < OT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) oacc[d][r] *= alpha;
    }
#pragma unroll
    for (int d = 0; d < OT; ++d) {
      const uint16_t* va = reinterpret_cast<const uint16_t*>(v_s + (4 * kb + (r16 >> 2)) * VROWB + (16 * d + 4 * (r16 & 3)) * 2);
      oacc[d] = mfma16x16x32(cat_bf16x4(lds_read_tr16(va), lds_read_tr16(va + 16 * VROWB / 2)), pk, oacc[d]);
    }
  };

  const int u0 = (int)((long long)split * p.n_tiles / p.n_split);
  const int u_end = (int)((long long)(split + 1) * p.n_tiles / p.n_split);
  const int pe = min(u_end, p.n_pre);
  int u = u0 + w;
  {
    Codes g;
    if (u < pe) load_codes(g, u);
    while (u < pe) {
      fence();
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        const float ksc = mx4_scale(g.ks[t]), vsc = mx4_scale(g.vs[t]);
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          put_v(t, j, mx4_bf16x8(g.v[t][j], vsc));
          s[t] = mfma16x16x32(mx4_bf16x8(g.k[t][j], ksc), qf[j], s[t]);
        }
      }
      fence();
      const int left = p.P - u * K4_UT;
      u += K4_TW;
      if (u < pe) load_codes(g, u);
      update(left < K4_UT ? (1u << left) - 1 : ~0u);
    }
  }
  // Lane units.
  for (; u < u_end; u += K4_TW) {
    const int row0 = (u - p.n_pre) * K4_UT;
    const int j0 = row0 / p.B, j1 = (min(row0 + K4_UT, p.R) - 1) / p.B;
    const unsigned long long upto = j1 >= 63 ? ~0ull : (1ull << (j1 + 1)) - 1;
    if (!(wg_vis & upto & ~((1ull << j0) - 1))) continue;
    fence();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const size_t at = ((size_t)min(row0 + 16 * t + r16, p.R - 1) * p.Hkv + hk) * D + kb * EL;
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        put_v(t, j, load_bf16x8(p.v_lane + at + 8 * j));
        s[t] = mfma16x16x32(load_bf16x8(p.k_lane + at + 8 * j), qf[j], s[t]);
      }
    }
    fence();
    update((unsigned)key_mask<K4_UT>(pr.vis, row0, p.B, p.R));
  }

  // Combine the wavefronts' states, in ascending order.
  __syncthreads();
  float* o_s = reinterpret_cast<float*>(lds);
  float* ml_s = o_s + K4_TW * 16 * OSTR;
#pragma unroll
  for (int d = 0; d < OT; ++d)
    *reinterpret_cast<f32x4*>(&o_s[(w * 16 + r16) * OSTR + 16 * d + 4 * kb]) = oacc[d];
  if (kb == 0) {
    ml_s[(w * 16 + r16) * 2 + 0] = m_run;
    ml_s[(w * 16 + r16) * 2 + 1] = l_run;
  }
  __syncthreads();
  constexpr int TPR = D / 4;   // threads per pair: all 16 pairs at once (half the threads at D = 64)
  const int r = tid / TPR, d0 = (tid % TPR) * 4;
  if (r >= min(16, p.n_pairs)) return;
  float mw[K4_TW], M = -INFINITY;
#pragma unroll
  for (int i = 0; i < K4_TW; ++i) {
    mw[i] = ml_s[(i * 16 + r) * 2];
    M = fmaxf(M, mw[i]);
  }
  float L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < K4_TW; ++i) {
    const float wgt = mw[i] == -INFINITY ? 0.f : exp2_fast(mw[i] - M);
    L += ml_s[(i * 16 + r) * 2 + 1] * wgt;
    const f32x4 a = *reinterpret_cast<const f32x4*>(&o_s[(i * 16 + r) * OSTR + d0]);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += a[e] * wgt;
  }
  const Pair out_pair = pair_at(p, hk, r);
  const size_t orow = (size_t)out_pair.row * p.Hq + out_pair.hq;
  if (p.n_split == 1) {
    const float inv = 1.0f / L;
    bf16x4 out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (__bf16)(acc[e] * inv);
    *reinterpret_cast<bf16x4*>(p.o + orow * D + d0) = out;
    if (p.lse && d0 == 0) p.lse[orow] = (M + log2f(L)) * K4_LN2;
  } else {
    const size_t at = (size_t)split * p.n_rows * p.Hq + orow;
    *reinterpret_cast<f32x4*>(p.part_o + at * D + d0) = acc;
    if (d0 == 0) {
      p.part_ml[at * 2] = M;
      p.part_ml[at * 2 + 1] = L;
    }
  }
}

// Combines the NS key splits of each (row, head): D / 4 lanes to a run of K4_RUN
// splits, 4 elements a lane, all loads of a run issued at once; then the runs through
// LDS.  Both sums go in ascending order.  (All splits in one run: 32 of them fill the
// registers; a call over 8192 rows 16.4 us, 14.7 with runs of 8.)
constexpr int K4_RUN = 8;
template <int D, int NS>
__global__ __launch_bounds__(256) void kv4_merge_kernel(const float* part_o, const float* part_ml, int n_rowheads,
                                                        uint16_t* o, float* lse) {
  constexpr int LPR = D / 4, N = NS < K4_RUN ? NS : K4_RUN, RUNS = NS / N, PER = 256 / LPR / RUNS;
  static_assert(PER >= 1, "a row's runs are one workgroup's");
  const int sl = threadIdx.x % LPR, run = threadIdx.x / LPR % RUNS;
  const int rh = blockIdx.x * PER + threadIdx.x / (LPR * RUNS), rc = min(rh, n_rowheads - 1);
  float m[N], l[N];
  f32x4 v[N];
#pragma unroll
  for (int s = 0; s < N; ++s) {
    const size_t at = (size_t)(run * N + s) * n_rowheads + rc;
    const float2 ml = *reinterpret_cast<const float2*>(part_ml + at * 2);
    m[s] = ml.x;
    l[s] = ml.y;
    v[s] = *reinterpret_cast<const f32x4*>(part_o + at * D + sl * 4);
  }
  float M = -INFINITY, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < N; ++s) M = fmaxf(M, m[s]);
  {
    const float ref = M == -INFINITY ? 0.f : M;   // (no split of the run saw a key: weights 0)
#pragma unroll
    for (int s = 0; s < N; ++s) {
      const float wgt = exp2_fast(m[s] - ref);
      L += l[s] * wgt;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += v[s][e] * wgt;
    }
  }
  if constexpr (RUNS > 1) {
    __shared__ f32x4 acc_s[256];
    __shared__ float2 ml_s[256];
    acc_s[threadIdx.x] = acc;
    ml_s[threadIdx.x] = float2{M, L};
    __syncthreads();
    if (run) return;
#pragma unroll
    for (int s = 1; s < RUNS; ++s) M = fmaxf(M, ml_s[threadIdx.x + s * LPR].x);   // (some run saw a key: finite)
    L = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < RUNS; ++s) {
      const float2 ml = ml_s[threadIdx.x + s * LPR];
      const f32x4 a = acc_s[threadIdx.x + s * LPR];
      const float wgt = exp2_fast(ml.x - M);
      L += ml.y * wgt;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += a[e] * wgt;
    }
  }
  if (rh >= n_rowheads) return;
  const float inv = 1.0f / L;
  bf16x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (__bf16)(acc[e] * inv);
  *reinterpret_cast<bf16x4*>(o + (size_t)rh * D + sl * 4) = out;
  if (lse && sl == 0) lse[rh] = (M + log2f(L)) * K4_LN2;
}

template <int D, int NS>
static void launch_kv4_merge(const float* part_o, const float* part_ml, int n, uint16_t* o, float* lse, hipStream_t stream) {
  constexpr int runs = NS < K4_RUN ? 1 : NS / K4_RUN, per = 256 / (D / 4) / runs;
  hipLaunchKernelGGL((kv4_merge_kernel<D, NS>), dim3((n + per - 1) / per), dim3(256), 0, stream, part_o, part_ml, n, o, lse);
}

// ------------------------------------------------------------------ host
constexpr int K4_MAX_SPLIT = 64;
struct Kv4Pass {
  bool token, units;   // token kernel, unit kernel (else the tile kernel)
  int n_rows, n_pairs, n_pre, n_tiles, n_split, tpw;
  size_t ws;
};

// Tiles of kt keys that n rows make (n up to INT32_MAX: n + kt - 1 would not do).
static int kv4_tiles(int n, int kt) { return n / kt + (n % kt != 0); }

// R: rows of all lane blocks (0: refreshed rows, which see the prefix alone).
static Kv4Pass kv4_pass(int n_rows, int R, int P, int Hq, int Hkv, int D) {
  Kv4Pass s{};
  s.n_rows = n_rows;
  s.n_pairs = n_rows * (Hq / Hkv);
  const long long q_tiles = (s.n_pairs + 31) / 32;
  const int units = kv4_tiles(P, K4_UT) + kv4_tiles(R, K4_UT);
  s.n_split = 1;
  s.token = s.n_pairs <= 16;
  // Up to a workgroup of the unit kernel per compute unit.  It converts the keys for every query
  // tile, the tile kernel once for 8 or 4 of them, so the limit also depends a little on the
  // length.  Unit and tile kernel (MI355X, us, D = 128; at D = 64 the ratios are the same) over
  // 512, 4096, 16384 and 32768 keys: 128 rows x 32 heads (128 query tiles) 10.7 17.7, 20.8 28.2, 48.6
  // 51.4, 86.9 86.9; 256 rows x 28 heads on 4 (224) 11.2 19.7, 26.3 33.1, 78.9 79.9, 149 133; 384 rows
  // (336, past the limit) 19.4 21.1, 49.8 50.4, 154 126, 295 223; at 1024 keys 23.6 28.0.
  s.units = q_tiles * Hkv <= 256;
  if (s.token) {
    s.n_pre = kv4_tiles(P, K4_UT);
    s.n_tiles = units;
    // One token, 28 heads on 4: 1024 rows 9.7 us unsplit, 11.3 with two splits; 2048 rows 12.7 and
    // 11.4, 3000 rows 15.9 and 11.3 with four (MI355X).  64 splits against 32 (half of the
    // compute units): 32769 rows 14 -> 11.5, 131072 rows 23.8 -> 18.7.
    if (units > 3 * K4_TW)
      while (s.n_split < K4_MAX_SPLIT && Hkv * s.n_split * 2 <= 256 && units >= 2 * K4_TW * s.n_split) s.n_split *= 2;
  } else if (s.units) {
    s.n_pre = kv4_tiles(P, K4_UT);
    s.n_tiles = units;
    while (s.n_split < K4_MAX_SPLIT && q_tiles * Hkv * s.n_split * 2 <= 256 && units >= 4 * K4_WAVES * s.n_split) s.n_split *= 2;
  } else {
    s.n_pre = kv4_tiles(P, K4_KT);
    s.n_tiles = s.n_pre + kv4_tiles(R, K4_KT);
    // The cheapest of 8 or 4 query tiles a workgroup and 1 to 16 splits, in us
    // (MI355X): a key tile costs 1.9 with 8, 1.1 with 4 (two thirds of it at D = 64), a
    // round of one workgroup per compute unit 5, a split its partials and a merge.
    double best = 1e30;
    for (int t = K4_WAVES; t >= 4; t /= 2)
      for (int ns = 1; ns <= 16 && (ns == 1 || s.n_tiles >= 3 * ns); ns *= 2) {
        const long long wgs = (q_tiles + t - 1) / t * Hkv * ns;
        const double tile = (t == K4_WAVES ? 1.9 : 1.1) * (D == 64 ? 0.68 : 1.0);
        const double cost = (double)((wgs + 255) / 256) * ((s.n_tiles + ns - 1) / ns * tile + 5.0) +
                            (ns > 1 ? 5.0 + 1.7e-6 * ns * n_rows * (double)Hq * D : 0.0);
        if (cost < best) {
          best = cost;
          s.tpw = t;
          s.n_split = ns;
        }
      }
  }
  s.ws = s.n_split > 1 ? (size_t)s.n_split * n_rows * Hq * (D + 2) * sizeof(float) : 0;
  return s;
}

size_t kv4_workspace_bytes(int L, int B, int P, int Hq, int Hkv, int D, int n_refresh) {
  const size_t a = L > 0 ? kv4_pass(L * B, L * B, P, Hq, Hkv, D).ws : 0;
  const size_t b = n_refresh > 0 ? kv4_pass(n_refresh, 0, P, Hq, Hkv, D).ws : 0;
  return a > b ? a : b;
}

int al_internal_kv4_plan(int L, int B, int P, int Hq, int Hkv, int D, int n_refresh, int32_t* out) {
  for (int i = 0; i < 2; ++i) {
    out[2 * i] = out[2 * i + 1] = -1;
    if (i ? n_refresh <= 0 : L <= 0) continue;
    const Kv4Pass s = i ? kv4_pass(n_refresh, 0, P, Hq, Hkv, D) : kv4_pass(L * B, L * B, P, Hq, Hkv, D);
    out[2 * i] = s.token ? 0 : s.units ? 1 : s.tpw;
    out[2 * i + 1] = s.n_split;
  }
  return 0;
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
  const int q_tiles = (s.n_pairs + 31) / 32;
  if (s.token)
    hipLaunchKernelGGL(lane_attn_kv4_token_kernel<D>, dim3(p.Hkv, 1, s.n_split), dim3(K4_TW * kWave), 0, stream, p);
  else if (s.units)
    hipLaunchKernelGGL(lane_attn_kv4_unit_kernel<D>, dim3((unsigned)(q_tiles * p.Hkv), 1, s.n_split), dim3(K4_THREADS), 0,
                       stream, p);
  else {
    const dim3 grid((q_tiles + s.tpw - 1) / s.tpw, p.Hkv, s.n_split);
    if (s.tpw == K4_WAVES) hipLaunchKernelGGL((lane_attn_kv4_kernel<D, 8>), grid, dim3(K4_THREADS), 0, stream, p);
    else hipLaunchKernelGGL((lane_attn_kv4_kernel<D, 4>), grid, dim3(K4_THREADS), 0, stream, p);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || s.n_split == 1) return e;
  const int nrh = s.n_rows * p.Hq;
#define AL_K4_MERGE(NS) \
  case NS: launch_kv4_merge<D, NS>(p.part_o, p.part_ml, nrh, p.o, p.lse, stream); break;
  switch (s.n_split) {
    AL_K4_MERGE(2) AL_K4_MERGE(4) AL_K4_MERGE(8) AL_K4_MERGE(16) AL_K4_MERGE(32) AL_K4_MERGE(64)
    default: return hipErrorInvalidValue;
  }
#undef AL_K4_MERGE
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
    attn_dfs_order(vis, L, p.order);
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
