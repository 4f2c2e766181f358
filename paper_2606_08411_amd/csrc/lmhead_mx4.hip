// Fused LM head + confidence on a weight in MXFP4 (mx4.h): the computation of
// lmhead.hip, z[v] = <H[row_idx[n]], W[v]> with W's values the 4-bit ones.  Codes
// are converted to bf16 in registers (exact) and multiplied by the 16x16x32
// bf16 MFMA with fp32 accumulation, so the hidden rows keep all their bits.
//
// A workgroup is WR x WC wavefronts: wavefront row i owns 64 vocabulary rows
// (a "unit" of the packed weight, four 16-row MFMA tiles), and the WC columns of
// wavefronts share out 16 CBT scored rows.  K goes in stages of 128 elements:
// lane 16 b + r of a wavefront takes the 16 bytes of row r, scale block b, so one
// dwordx4 load per 16 rows and stage, one scale per lane and four MFMA steps of 8
// elements a lane (a contraction may walk its index in any order, as long as both
// operands do).  W goes straight to registers, two or three stages ahead: no wavefront
// of the same column needs another's, and LDS carries only the hidden rows.  A
// stage's loads are issued one to each group of MFMAs: all at its start they keep the
// wavefronts from the matrix cores while the address unit takes them (8 wavefronts x up
// to 12 KB at 64 bytes a cycle; 614 rows of the 126464 x 4096 head 500 us, 470 spread).
//
// What bounds it: with few columns the W stream (17/32 byte an element, against
// 2 in bf16), with many the matrix cores.  A stage of a wavefront is 64
// conversions (4 cycles each, beside the MFMAs) against 16 x 16 cycles of MFMA per 16
// columns.  126464 x 4096: 1 row 43 us (275 MB at 6.4 TB/s; a bare read of them 40.5),
// 77 rows 66-72 (1.1-1.2 PFLOP/s), 614 rows 465-480 (1.33-1.37 PFLOP/s; an 8192 cubed
// library product 1.25 on the same card), then the merge, 4-5 us.  The power limit holds
// the clock at 1.9-2.2 GHz: with a weight or hidden rows of zeros 77 rows take 58 us, 614
// take 406.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "launch.h"
#include "lmhead.h"
#include "mx4.h"

namespace al {

constexpr int LM_MX4_WAVES = 8;

struct LmMx4Params {
  const uint16_t* hidden;
  const int32_t* row_idx;
  const uint8_t* codes;    // [n_st][4 n_u][64][16]
  const uint8_t* scales;   // [n_st][n_u][64][4]
  const uint8_t* sup;
  LmPartial* part;         // [n_nt][16 CBT][n_vt]
  int N, d, V, eos_id;
  int n_u, n_st;           // 64-row units, 128-element stages
  int n_vt, n_nt;          // workgroups over the units (n_u units shared out evenly) and the columns
};

// Row c of a hidden stage is 256 bytes in LDS, segment s (16 bytes) in slot s ^
// lm_slot(c): the 16 lanes that one LDS cycle serves (0-3, 12-15, 20-23, 24-27 and
// so on) then touch every bank once.
__device__ __forceinline__ int lm_slot(int c) { return (c & 3) | ((c & 8) ? 12 : 0); }

template <int CBT, int WC, int KS, int DEPTH, bool RAGGED, bool NT>
__global__ __launch_bounds__(512) void lmhead_mx4_kernel(LmMx4Params p) {
  constexpr int COLS = 16 * CBT;
  constexpr int CB0 = (CBT + WC - 1) / WC, CB1 = CBT - (WC - 1) * CB0;   // column tiles of the first, last column
  static_assert(WC == 1 || (WC == 2 && KS == 1), "at most two columns of wavefronts");
  constexpr int WR = LM_MX4_WAVES / (WC * KS), TH = LM_MX4_WAVES * kWave;
  constexpr int HB = COLS * 256;             // bytes of the hidden rows of a stage
  constexpr int LH = (KS * COLS / 4 + LM_MX4_WAVES - 1) / LM_MX4_WAVES;   // direct loads of a group per wavefront
  __shared__ __attribute__((aligned(1024))) char ring[3 * KS * HB];

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wc = WC == 1 ? 0 : w & 1, ks = w % KS, wr = w / (WC * KS);
  const int l16 = lane & 15, kb = lane >> 4;
  const int nt = blockIdx.x % p.n_nt, vt = blockIdx.x / p.n_nt;
  const int u_begin = (int)((long long)vt * p.n_u / p.n_vt), u_end = (int)((long long)(vt + 1) * p.n_u / p.n_vt);
  const int u = u_begin + wr;
  const bool active = u < u_end;   // (a wavefront past the tile's units loads hidden rows only)

  // Hidden rows go straight to LDS, in pieces of 1 KB (4 rows of a stage): pieces w + 8
  // i of a group of KS stages by wavefront w (an earlier one with the same rows mod 16
  // again where there are none left, so that every wavefront has LH loads a group).
  // Past d, where the packed W is zero, a segment of the same row is read again.
  // (Stages past the last load from the first: the loads of a group are always the
  // same number and need no branch, so every wait counts them exactly.)
  const unsigned ring0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)ring;
  unsigned hoff[LH];   // bytes (n_rows * d < 2^31)
  auto piece = [&](int i) {
    const int q = w + LM_MX4_WAVES * i;
    return q < KS * COLS / 4 ? q : q - (i ? LM_MX4_WAVES : 4);
  };
  const int hseg = l16 ^ lm_slot((4 * w + kb) & 15);   // this lane's segment of a stage, in every piece
#pragma unroll
  for (int i = 0; i < LH; ++i) {
    const int c = 4 * (piece(i) % (COLS / 4)) + kb;
    const int n = min(nt * COLS + c, p.N - 1);
    hoff[i] = 2 * (unsigned)(p.row_idx ? p.row_idx[n] : n) * (unsigned)p.d + hseg * 16;
  }
  auto load_hidden1 = [&](int group, int slot, int i) {
    const int st = group * KS + piece(i) / (COLS / 4);
    const char* src = reinterpret_cast<const char*>(p.hidden) + (size_t)(st < p.n_st ? st : 0) * 256;
    const unsigned lds_at = ring0 + slot + piece(i) * 1024;
    unsigned off = hoff[i];
    if (RAGGED) off -= st * 128 + 8 * hseg < p.d ? 0 : 16 * hseg;
    load_to_lds16<0, 0, false>(uniform_ptr(src), off, lds_at);
  };
  auto load_hidden = [&](int group, int slot) {
#pragma unroll
    for (int i = 0; i < LH; ++i) load_hidden1(group, slot, i);
  };
  struct Stage {
    i32x4 c[4];
    unsigned s;
  };
  auto load_w1 = [&](Stage& g, int st, int i) {   // i = 0..3: codes, 4: scales
    const int in = st < p.n_st;
    const size_t at = (size_t)(in ? st : 0) * p.n_u + (in ? u : 0);
    const i32x4* src = reinterpret_cast<const i32x4*>(p.codes) + at * 256 + lane;
    if (i < 4) g.c[i] = NT ? __builtin_nontemporal_load(src + i * 64) : src[i * 64];
    else g.s = reinterpret_cast<const unsigned*>(p.scales)[at * 64 + lane];
  };
  auto load_w = [&](Stage& g, int st) {
#pragma unroll
    for (int i = 0; i < 5; ++i) load_w1(g, st, i);
  };

  auto body = [&](auto nc_tag) {
    constexpr int NC = decltype(nc_tag)::value;
    f32x4 acc[4][NC];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NC; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Step s (8 elements a lane) of a stage: 4 NC MFMAs, in groups of a row tile
    // i.  While a group runs, the next group's codes are converted and a quarter of
    // the next step's hidden fragments are read (ROLL: read in the step's last group,
    // each into the register that its last product has freed).
    constexpr bool ROLL = CBT > 10;
    constexpr int RPG = (NC + 3) / 4, NB = ROLL ? 1 : 2;
    const int brow = (wc * CB0 * 16 + l16) * 256;
    bf16x8 b[NB][NC], a[2];
    auto read_b = [&](int slot, int s, int j) {
      b[s % NB][j] = *reinterpret_cast<const bf16x8*>(ring + slot + brow + j * 4096 + (((4 * kb + s) ^ lm_slot(l16)) * 16));
    };
    auto convert = [&](const Stage& g, int q) {   // group q = 4 s + i
      a[q & 1] = mx4_bf16x8((unsigned)g.c[q & 3][q >> 2], mx4_scale((g.s >> (8 * (q & 3))) & 255));
    };
    // (The next stage's first fragments come with this one's last step: its hidden rows
    // are in LDS already, and the matrix cores need not wait for them behind the barrier.)
    auto compute = [&](const Stage& g, int slot, const Stage& gn, int slot_n, auto load) {
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int s = q >> 2, i = q & 3;
        load(q);
        if (!ROLL) {
#pragma unroll
          for (int j = i * RPG; j < (i + 1) * RPG; ++j)
            if (j < NC) read_b(s < 3 ? slot : slot_n, (s + 1) & 3, j);
        }
        if (q < 15) convert(g, q + 1);
        else convert(gn, 0);
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          acc[i][j] = mfma16x16x32(a[q & 1], b[s % NB][j], acc[i][j]);
          if (ROLL && i == 3) read_b(s < 3 ? slot : slot_n, (s + 1) & 3, j);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // Group i is stages KS i .. KS i + KS - 1, of which this wavefront multiplies stage
    // KS i + ks.  At the barrier on its top the hidden rows of groups i and i + 1 have
    // arrived (all but the five loads of W issued after them), everyone is done with
    // group i - 1, and its buffer takes the hidden rows of group i + 2.
    const int n_group = (p.n_st + KS - 1) / KS;
    int slot = 0;   // byte of the ring
    auto next_slot = [&](int x, int by) {
      x += by * KS * HB;
      return x >= 3 * KS * HB ? x - 3 * KS * HB : x;
    };
    if (!active) {
      load_hidden(0, 0);
      load_hidden(1, KS * HB);
      wait_loads_and_barrier<0>();
      for (int i = 0; i < n_group; ++i) {
        if (i) wait_loads_and_barrier<0>();
        load_hidden(i + 2, next_slot(slot, 2));
        slot = next_slot(slot, 1);
      }
    } else {
      Stage g[DEPTH];
#pragma unroll
      for (int q = 0; q < DEPTH - 1; ++q) {
        load_w(g[q], q * KS + ks);
        asm volatile("" ::: "memory");   // (in this order, which the waits in the loop assume)
      }
      load_hidden(0, 0);
      load_hidden(1, KS * HB);
      wait_loads_and_barrier<0>();
#pragma unroll
      for (int j = 0; j < NC; ++j) read_b(ks * HB, 0, j);
      convert(g[0], 0);
      // (One group inside the other's condition: no path leaves one out and takes a
      // later one, so the compiler's waits for W stay exact too.)
      auto step = [&](auto self, auto q_tag, int i0) -> void {
        constexpr int q = decltype(q_tag)::value;
        const int i = i0 + q;
        if (i < n_group) {
          if (q > 0 || i0 > 0) wait_loads_and_barrier<5>();
          const int slot2 = next_slot(slot, 2);
          auto load = [&](int t) {
            if (t < LH) load_hidden1(i + 2, slot2, t);
            else if (t < LH + 5) load_w1(g[(q + DEPTH - 1) % DEPTH], (i + DEPTH - 1) * KS + ks, t - LH);
          };
          if (KS == 1 || i * KS + ks < p.n_st) compute(g[q], slot + ks * HB, g[(q + 1) % DEPTH], next_slot(slot, 1) + ks * HB, load);
          slot = next_slot(slot, 1);
          if constexpr (q + 1 < DEPTH) self(self, IntTag<q + 1>{}, i0);
        }
      };
      for (int i0 = 0; i0 < n_group; i0 += DEPTH) step(step, IntTag<0>{}, i0);
    }
    wait_loads_and_barrier<0>();   // (the last loads land in the ring too)
    // The KS partial sums of a tile, in ascending order of ks.
    if (KS > 1) {
      f32x4* sum = reinterpret_cast<f32x4*>(ring) + (size_t)wr * (KS - 1) * 4 * NC * 64 + lane;
      if (active && ks > 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < NC; ++j) sum[((ks - 1) * 4 * NC + i * NC + j) * 64] = acc[i][j];
      }
      __syncthreads();
      if (active && ks == 0) {
        for (int k = 0; k < KS - 1; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < NC; ++j) {
              const f32x4 v = sum[(k * 4 * NC + i * NC + j) * 64];
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j][e] += v[e];
            }
      }
      __syncthreads();
    }
    // Lane (l16, kb) holds vocabulary rows 64 u + 16 i + 4 kb + r of column 16 j + l16.
    float* red_m = reinterpret_cast<float*>(ring);
    float* red_s = red_m + WR * COLS;
    int* red_i = reinterpret_cast<int*>(red_s + WR * COLS);
    if (active && ks == 0) {
      const int ve = min(p.V, (u + 1) * 64);
      const bool eos_here = p.sup && p.eos_id >= u * 64 && p.eos_id < ve;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int col = wc * CB0 * 16 + 16 * j + l16;
        int excl = -1;
        if (eos_here) {
          const int n = nt * COLS + col;
          excl = (n < p.N && p.sup[n]) ? p.eos_id : -1;
        }
        // The column's maximum over the four lanes that hold it, the first id that has
        // it, and the sum of exponentials against it: no branches, no LDS.
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int v = u * 64 + 16 * i + 4 * kb + r;
            acc[i][j][r] = (v < ve && v != excl) ? acc[i][j][r] : -INFINITY;
            m = fmaxf(m, acc[i][j][r]);
          }
        m = quad_max(m);
        const float m0 = (m == -INFINITY) ? 0.f : m;
        float s = 0.f;
        int idx = 0x7fffffff;
#pragma unroll
        for (int i = 3; i >= 0; --i)
#pragma unroll
          for (int r = 3; r >= 0; --r) {
            idx = acc[i][j][r] == m ? u * 64 + 16 * i + 4 * kb + r : idx;
            s += exp2_fast((acc[i][j][r] - m0) * LM_LOG2E);
          }
        s = quad_sum(s);
        idx = quad_min(idx);
        if (kb == 0) {
          red_m[wr * COLS + col] = m;
          red_s[wr * COLS + col] = s;
          red_i[wr * COLS + col] = idx;
        }
      }
    }
    __syncthreads();
    for (int col = tid; col < COLS; col += TH) {
      const int n = u_end - u_begin;
      float mu[WR], m = -INFINITY, s = 0.f;
      int idx = 0x7fffffff;
#pragma unroll
      for (int i = 0; i < WR; ++i) {
        mu[i] = i < n ? red_m[i * COLS + col] : -INFINITY;
        m = fmaxf(m, mu[i]);
      }
#pragma unroll
      for (int i = WR - 1; i >= 0; --i) {
        const bool some = mu[i] != -INFINITY;   // (a unit whose only row is a suppressed EOS has none)
        s += some ? red_s[i * COLS + col] * exp2_fast((mu[i] - m) * LM_LOG2E) : 0.f;
        idx = some && mu[i] == m ? red_i[i * COLS + col] : idx;
      }
      LmPartial q;
      q.m = m;
      q.s = s;
      q.idx = idx;
      q.pad = 0;
      p.part[((size_t)nt * COLS + col) * p.n_vt + vt] = q;
    }
  };
  if (WC == 1 || wc == 0) body(IntTag<CB0>{});
  else body(IntTag<CB1>{});
}

// ------------------------------------------------------------------ pack
// One 16-byte segment of codes per thread (lane 16 b + r of unit-quarter uq, stage
// c: row 16 uq + r, bytes 64 c + 16 b), then one dword of scales (the four quarters).
// A wavefront reads 64 bytes of each of 16 rows and writes 1 KB.  Once at load time, bound by those
// short reads: 126464 x 4096 in 166 us, 3.3 TB/s read and written (a copy 5.1), 152064 x 3584 in 188.
__global__ __launch_bounds__(256) void lmhead_pack_mx4_kernel(const uint8_t* codes, const uint8_t* scales, int d, int V,
                                                              int n_u, int n_st, uint8_t* out) {
  const long long n_seg = (long long)n_st * n_u * 256, n_sc = (long long)n_st * n_u * 64;
  for (long long o = (long long)blockIdx.x * 256 + threadIdx.x; o < n_seg + n_sc; o += (long long)gridDim.x * 256) {
    if (o < n_seg) {
      const int l = (int)(o & 63);
      const long long b = o >> 6;
      const int uq = (int)(b % (4 * n_u)), c = (int)(b / (4 * n_u));
      const long long v = 16ll * uq + (l & 15);
      const int blk = 4 * c + (l >> 4);   // 32-element block of the row
      i32x4 x = {0, 0, 0, 0};
      if (v < V && 32 * blk < d) x = *reinterpret_cast<const i32x4*>(codes + v * (d / 2) + 16ll * blk);
      reinterpret_cast<i32x4*>(out)[o] = x;
    } else {
      const long long q = o - n_seg;
      const int l = (int)(q & 63);
      const long long b = q >> 6;
      const int u = (int)(b % n_u), c = (int)(b / n_u);
      const int blk = 4 * c + (l >> 4);
      unsigned x = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long v = 64ll * u + 16 * i + (l & 15);
        if (v < V && 32 * blk < d) x |= (unsigned)scales[v * (d / 32) + blk] << (8 * i);
      }
      reinterpret_cast<unsigned*>(out + n_seg * 16)[q] = x;
    }
  }
}

// ------------------------------------------------------------------ host
static int mx4_units(int V) { return (V + 63) / 64; }
static int mx4_stages(int d) { return (d + 127) / 128; }

size_t lmhead_packed_mx4_bytes(int d, int V) { return (size_t)mx4_stages(d) * mx4_units(V) * (4096 + 256); }

hipError_t launch_lmhead_pack_mx4(const uint8_t* codes, const uint8_t* scales, int d, int V, uint8_t* out,
                                  hipStream_t stream) {
  hipLaunchKernelGGL(lmhead_pack_mx4_kernel, dim3(8192), dim3(256), 0, stream, codes, scales, d, V, mx4_units(V),
                     mx4_stages(d), out);
  return hipGetLastError();
}

// The instances built, X(CBT, WC, KS, DEPTH): 16 CBT columns, WC columns of
// wavefronts, K split over KS wavefronts, W loaded DEPTH - 1 stages ahead.  One
// unit row of wavefronts is 8 / (WC KS) units.  A wavefront's 16 CBT / WC fp32 sums, DEPTH
// x 17 registers of W and the fragments have to fit 256 registers, three groups of
// hidden rows (12 KS CBT KB) the LDS.
#define AL_LM_MX4_INSTANCES(X) \
  X(1, 1, 1, 4) X(2, 1, 1, 4) X(4, 1, 1, 4) X(5, 1, 1, 3) X(6, 1, 1, 3) X(8, 2, 1, 3) X(10, 2, 1, 3) X(13, 2, 1, 3) \
  X(1, 1, 8, 4) X(2, 1, 4, 4) X(4, 1, 2, 4) X(5, 1, 2, 3) X(6, 1, 2, 3)

struct LmMx4Layout {
  int cbt, wc, ks, n_vt, n_nt;
};

// Most workgroups over the vocabulary that a layout may have, and the bytes of the
// partials under it (column tiles pad N to at most 12 fragments more): grows with N,
// so that a workspace made for N rows serves every smaller call.
static int lm_mx4_most_vt(int V) {
  const int n_u = mx4_units(V);
  return std::max(std::min(n_u, lm_cu_count()), (n_u + 3) / 4);
}
size_t lmhead_mx4_workspace_bytes(int N, int d, int V) {
  (void)d;
  if (N <= 0 || V <= 0) return 0;
  return sizeof(LmPartial) * 16 * (size_t)((N + 15) / 16 + 12) * lm_mx4_most_vt(V);
}

// The cheapest instance under a cost model: n_nt column tiles, and either whole rounds of
// workgroups of as many units as there are unit rows, or one round with the units
// shared out over all compute units.  In us (MI355X): a stage takes 0.33 (two columns of
// wavefronts: 0.27) + 0.16 a column fragment for each wavefront on a SIMD, 0.67 at least, a
// K split 3.4 a round more and 4% for every further column tile.  Fitted to every instance
// at 17 pairs of d and V from 256 x 1024 to 2048 x 250000, 1 to 1024 rows: the choice takes
// 0.7% more than the fastest on average, 10% at most.  Both sides: d = 3584, V =
// 152064, 512 rows 450 with six fragments unsplit, 481 with thirteen in two columns, 128
// rows 137 with eight in two columns, 144 with four; d = 4096, V = 32000, 32 rows 21 with
// K split in four, 25 without; d = 2048, V = 2000, 320 rows 14 unsplit, 16 split in two.
static LmMx4Layout lm_mx4_layout(int N, int d, int V) {
  const int frags = (N + 15) / 16, n_u = mx4_units(V), n_st = mx4_stages(d), cus = lm_cu_count();
  const int most = lm_mx4_most_vt(V);
  LmMx4Layout best{};
  double best_t = 1e30;
#define AL_LM_MX4_TRY(CBT, WC, KS, DEPTH)                                                          \
  {                                                                                                \
    const int wr = LM_MX4_WAVES / (WC * KS), n_nt = (frags + CBT - 1) / CBT;                       \
    const int n_vt = std::max((n_u + wr - 1) / wr, std::min(n_u, std::max(1, cus / n_nt)));        \
    const int upw = (n_u + n_vt - 1) / n_vt;                                                       \
    const double waves = (upw * WC * KS + 3) / 4;                                                  \
    const double stage = std::max(0.67, waves * ((WC > 1 ? 0.27 : 0.33) + 0.16 * ((CBT + WC - 1) / WC))); \
    const double rounds = (double)(((long long)n_vt * n_nt + cus - 1) / cus);                      \
    const double t = rounds * (((n_st + KS - 1) / KS) * stage + (KS > 1 ? 3.4 : 0.0)) *            \
                     (KS > 1 ? 1 + 0.04 * (n_nt - 1) : 1.0);                                       \
    if (n_vt <= most && t < best_t) {                                                              \
      best_t = t;                                                                                  \
      best = LmMx4Layout{CBT, WC, KS, n_vt, n_nt};                                                 \
    }                                                                                              \
  }
#define AL_LM_MX4_X(CBT, WC, KS, DEPTH) AL_LM_MX4_TRY(CBT, WC, KS, DEPTH)
  AL_LM_MX4_INSTANCES(AL_LM_MX4_X)
#undef AL_LM_MX4_X
#undef AL_LM_MX4_TRY
  return best;
}

int al_internal_lmhead_mx4_plan(int N, int d, int V, int32_t* out) {
  const LmMx4Layout L = lm_mx4_layout(N, d, V);
  const int32_t v[6] = {L.cbt, L.wc, L.ks, L.n_vt, L.n_nt, d % 128 ? 0 : L.n_nt == 1 ? 1 : 2};
  std::copy(v, v + 6, out);
  return 0;
}

int al_internal_lmhead_mx4_instances(int32_t* out, int most) {
  int n = 0;
#define AL_LM_MX4_X(CBT, WC, KS, DEPTH)                \
  if (n < most) {                                      \
    const int32_t v[3] = {CBT, WC, KS};                \
    std::copy(v, v + 3, out + 3 * n++);                \
  }
  AL_LM_MX4_INSTANCES(AL_LM_MX4_X)
#undef AL_LM_MX4_X
  return n;
}

template <int CBT, int WC, int KS, int DEPTH>
static void launch_mx4_tile(const LmMx4Params& p, bool nt, hipStream_t stream) {
  const dim3 grid((unsigned)p.n_vt * p.n_nt), block(LM_MX4_WAVES * kWave);
  if (p.d % 128)
    hipLaunchKernelGGL((lmhead_mx4_kernel<CBT, WC, KS, DEPTH, true, false>), grid, block, 0, stream, p);
  else if (nt)
    hipLaunchKernelGGL((lmhead_mx4_kernel<CBT, WC, KS, DEPTH, false, true>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((lmhead_mx4_kernel<CBT, WC, KS, DEPTH, false, false>), grid, block, 0, stream, p);
}

hipError_t launch_lmhead_mx4(const uint16_t* hidden, const int32_t* row_idx, int N, const uint8_t* W, int d, int V,
                             const uint8_t* sup, int eos_id, float* conf, int32_t* argmax, float* lse, void* ws,
                             hipStream_t stream) {
  if (N <= 0) return hipSuccess;
  const LmMx4Layout L = lm_mx4_layout(N, d, V);
  LmMx4Params p{};
  p.hidden = hidden;
  p.row_idx = row_idx;
  p.n_u = mx4_units(V);
  p.n_st = mx4_stages(d);
  p.codes = W;
  p.scales = W + (size_t)p.n_st * p.n_u * 4096;
  p.sup = sup;
  p.part = static_cast<LmPartial*>(ws);
  p.N = N;
  p.d = d;
  p.V = V;
  p.eos_id = eos_id;
  p.n_vt = L.n_vt;
  p.n_nt = L.n_nt;
  const bool nt = L.n_nt == 1;
  switch (L.cbt * 64 + L.wc * 16 + L.ks) {
#define AL_LM_MX4_X(CBT, WC, KS, DEPTH) \
  case CBT * 64 + WC * 16 + KS: launch_mx4_tile<CBT, WC, KS, DEPTH>(p, nt, stream); break;
    AL_LM_MX4_INSTANCES(AL_LM_MX4_X)
#undef AL_LM_MX4_X
    default: return hipErrorInvalidValue;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_lmhead_merge(p.part, N, L.n_vt, 16 * L.cbt, conf, argmax, lse, stream);
}

}  // namespace al
