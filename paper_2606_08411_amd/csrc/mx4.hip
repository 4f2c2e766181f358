// The MXFP4 row quantiser, its inverse and the store of K/V rows into a 4-bit
// prefix cache (format and rounding: mx4.h).
//
// All three are bound by memory: the quantiser reads 2 bytes and writes 17/32 of
// a byte per element, the inverse the other way round.  A lane takes 16 bytes of
// bf16 (8 elements); the four lanes of a block agree on its scale by two DPP
// moves, so nothing passes through LDS and every access of a wavefront is one
// contiguous run.  126464 x 4096: quantised in 193 us (6.8 TB/s), read back in 200 (6.6);
// 128 x 4096: 2.5 and 2.2 us, the length of a short launch; 2563 rows of K and V of 32
// heads stored in 11.6 us (4.6 TB/s).
#include "common.h"
#include "launch.h"
#include "mx4.h"

namespace al {

constexpr int MX_THREADS = 256;
constexpr int MX_SEGS = 4;   // 8-element segments in flight per lane
constexpr long long MX_MAX_BLOCKS = 1ll << 20;

__device__ __forceinline__ void put_segment(unsigned* codes, uint8_t* scales, long long seg, i32x4 x) {
  unsigned s;
  const unsigned c = mx4_quantize8(x, s);
  codes[seg] = c;
  if ((threadIdx.x & 3) == 0) scales[seg >> 2] = (uint8_t)s;
}

__global__ __launch_bounds__(MX_THREADS) void mx4_quantize_kernel(const i32x4* x, long long n_seg,
                                                                  unsigned* codes, uint8_t* scales) {
  const long long step = (long long)gridDim.x * MX_THREADS * MX_SEGS;
  for (long long base = (long long)blockIdx.x * MX_THREADS * MX_SEGS + threadIdx.x; base < n_seg; base += step) {
    i32x4 v[MX_SEGS];
#pragma unroll
    for (int i = 0; i < MX_SEGS; ++i)   // n_seg is a multiple of 4: the lanes of a block stay together
      if (base + i * MX_THREADS < n_seg) v[i] = __builtin_nontemporal_load(x + base + i * MX_THREADS);
#pragma unroll
    for (int i = 0; i < MX_SEGS; ++i)
      if (base + i * MX_THREADS < n_seg) put_segment(codes, scales, base + i * MX_THREADS, v[i]);
  }
}

template <bool NT>
__global__ __launch_bounds__(MX_THREADS) void mx4_dequantize_kernel(const unsigned* codes, const uint8_t* scales,
                                                                    long long n_seg, i32x4* y) {
  const long long step = (long long)gridDim.x * MX_THREADS * MX_SEGS;
  for (long long base = (long long)blockIdx.x * MX_THREADS * MX_SEGS + threadIdx.x; base < n_seg; base += step) {
    unsigned c[MX_SEGS], s[MX_SEGS];
#pragma unroll
    for (int i = 0; i < MX_SEGS; ++i) {
      const long long seg = base + i * MX_THREADS;
      if (seg < n_seg) {
        c[i] = codes[seg];
        s[i] = scales[seg >> 2];
      }
    }
#pragma unroll
    for (int i = 0; i < MX_SEGS; ++i)
      if (base + i * MX_THREADS < n_seg) {
        const i32x4 v = __builtin_bit_cast(i32x4, mx4_bf16x8(c[i], mx4_scale(s[i])));
        if (NT) __builtin_nontemporal_store(v, y + base + i * MX_THREADS);
        else y[base + i * MX_THREADS] = v;
      }
  }
}

// Row r of K (blockIdx.y 0) and V (1) to cache row idx[r] (or start + r): the
// cache is head-major, [2][Hkv][cap][D], so that a head's rows stream.  A row
// whose index lies outside [0, limit) is left out.
__global__ __launch_bounds__(MX_THREADS) void kv4_store_kernel(const i32x4* k, const i32x4* v, const int32_t* idx,
                                                               int start, int T, int limit, int cap, int Hkv, int row_segs,
                                                               unsigned* codes, uint8_t* scales) {
  const i32x4* x = blockIdx.y ? v : k;
  const long long n_seg = (long long)T * Hkv * row_segs;
  const long long step = (long long)gridDim.x * MX_THREADS;
  for (long long seg = (long long)blockIdx.x * MX_THREADS + threadIdx.x; seg < n_seg; seg += step) {
    const long long rh = seg / row_segs;
    const int part = (int)(seg - rh * row_segs);
    const int r = (int)(rh / Hkv), h = (int)(rh - (long long)r * Hkv);
    const int row = idx ? idx[r] : start + r;
    const i32x4 xv = x[seg];
    if ((unsigned)row < (unsigned)limit)
      put_segment(codes, scales, (((long long)blockIdx.y * Hkv + h) * cap + row) * row_segs + part, xv);
  }
}

static unsigned mx_blocks(long long n_seg, int per_block) {
  const long long b = (n_seg + per_block - 1) / per_block;
  return (unsigned)(b < MX_MAX_BLOCKS ? b : MX_MAX_BLOCKS);
}

hipError_t launch_mx4_quantize(const uint16_t* x, long long n, uint8_t* codes, uint8_t* scales, hipStream_t stream) {
  hipLaunchKernelGGL(mx4_quantize_kernel, dim3(mx_blocks(n / 8, MX_THREADS * MX_SEGS)), dim3(MX_THREADS), 0, stream,
                     reinterpret_cast<const i32x4*>(x), n / 8, reinterpret_cast<unsigned*>(codes), scales);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, long long n, uint16_t* y,
                                 hipStream_t stream) {
  // Values past 64 MB, more than the L2s hold, are stored non-temporally (and the
  // quantiser's input, read once, is loaded so): 126464 x 4096 quantised and read back
  // 472 us with neither, 471 and 467 with one, 406 with both; 46 MB of a cache 21.9 and
  // 21.4 (MI355X).
  const dim3 grid(mx_blocks(n / 8, MX_THREADS * MX_SEGS)), block(MX_THREADS);
  const unsigned* c = reinterpret_cast<const unsigned*>(codes);
  if (n > (32ll << 20)) hipLaunchKernelGGL(mx4_dequantize_kernel<true>, grid, block, 0, stream, c, scales, n / 8, reinterpret_cast<i32x4*>(y));
  else hipLaunchKernelGGL(mx4_dequantize_kernel<false>, grid, block, 0, stream, c, scales, n / 8, reinterpret_cast<i32x4*>(y));
  return hipGetLastError();
}

hipError_t launch_kv4_store(const uint16_t* k, const uint16_t* v, const int32_t* row_idx, int start, int T, int limit,
                            int cap, int Hkv, int D, uint8_t* codes, uint8_t* scales, hipStream_t stream) {
  const dim3 grid(mx_blocks((long long)T * Hkv * (D / 8), MX_THREADS), 2);
  hipLaunchKernelGGL(kv4_store_kernel, grid, dim3(MX_THREADS), 0, stream, reinterpret_cast<const i32x4*>(k),
                     reinterpret_cast<const i32x4*>(v), row_idx, start, T, limit, cap, Hkv, D / 8,
                     reinterpret_cast<unsigned*>(codes), scales);
  return hipGetLastError();
}

}  // namespace al
