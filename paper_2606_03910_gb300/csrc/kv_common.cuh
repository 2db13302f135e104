// Definitions shared by the kernels on 8-bit KV blocks and the attention that reads them.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>

#include "netkv_internal.cuh"

constexpr uint32_t kBlockTokens = NETKV_BLOCK_TOKENS;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A softmax scale: the exponentials are powers of two, so its product with log2(e) has to be finite
// too (an infinite one would make NaN of a score of 0).
inline bool scale_ok(float scale) { return scale > 0.f && scale * kLog2e <= 3.4028235e38f; }

// The pages by value, and the sizes of one page's part for one head.
struct KvArgs {
  unsigned char* k;
  unsigned char* v;
  float* k_scale;
  float* v_scale;
  uint32_t n_pages, heads;
};

inline bool kv_pages_ok(const netkv_kv_pages* p) {
  return p && p->d_k && p->d_v && p->d_k_scale && p->d_v_scale && aligned_to(p->d_k, 16) &&
         aligned_to(p->d_v, 16) && aligned_to(p->d_k_scale, 4) && aligned_to(p->d_v_scale, 4) &&
         p->n_pages >= 1 && p->n_pages < (1u << 31) && p->kv_heads >= 1 && p->kv_heads <= 1024 &&
         (p->head_dim == 64 || p->head_dim == 128) &&
         (p->format == NETKV_KV_INT8 || p->format == NETKV_KV_E4M3);
}

inline KvArgs kv_args(const netkv_kv_pages* p) {
  return {(unsigned char*)p->d_k, (unsigned char*)p->d_v, p->d_k_scale, p->d_v_scale, p->n_pages,
          p->kv_heads};
}

// Allows a kernel its dynamic shared memory, once for each device (0.8 us a time).
template <auto kKernel>
inline cudaError_t allow_shared(int bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// Registers a thread of a kernel's launches; 0 where the runtime does not say, as for want of memory to
// load the kernel, which a later call asks again.
template <auto kKernel>
inline int launch_registers() {
  static std::atomic<int> known{0};
  int n = known.load(std::memory_order_relaxed);
  if (n) return n;
  cudaFuncAttributes has;
  if (cudaFuncGetAttributes(&has, kKernel) == cudaSuccess)
    known.store(n = has.numRegs, std::memory_order_relaxed);
  else
    cudaGetLastError();  // or the next call's launch would be taken for the one that failed
  return n;
}

// Rows of heads * dim 16-bit values: 16-byte aligned, strides in values.
inline bool rows_ok(const void* p, uint64_t stride, uint64_t width) {
  return p && aligned_to(p, 16) && stride % 8 == 0 && stride >= width && stride < (1ull << 40);
}

// The rows [first, first + count) of sequence i by offsets that must not decrease or pass
// `rows`; a pair that does has no rows.
struct RowRange {
  uint64_t first, count;
  bool bad;
};
__device__ __forceinline__ RowRange row_range(const uint64_t* off, uint32_t i, uint64_t rows) {
  const uint64_t a = off[i], b = off[i + 1];
  const bool bad = b < a || b > rows;
  return {bad ? 0 : a, bad ? 0 : b - a, bad};
}

// Finds the sequence that holds unit `unit` when sequence i has count(i) units, one sequence's
// units after another's.  Called by whole warps; lane l counts sequences 4 l .. 4 l + 3 of 128,
// so batches of up to 128 sequences take one round trip to memory.  seq = n: past the end.
struct Found {
  uint32_t seq, unit;  // the sequence, and the unit's number within it
};
template <class Count>
__device__ __forceinline__ Found find_unit(uint32_t n, uint32_t unit, Count count) {
  const uint32_t lane = threadIdx.x & 31;
  for (uint32_t base = 0; base < n; base += 128) {
    uint32_t c[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t i = base + lane * 4 + j;
      c[j] = i < n ? count(i) : 0;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += c[j];
    uint32_t upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t x = __shfl_up_sync(~0u, upto, d);
      if (lane >= (uint32_t)d) upto += x;
    }
    const uint32_t hit = __ballot_sync(~0u, unit < upto);
    if (hit) {
      const int at = __ffs(hit) - 1;
      uint32_t left = unit - (upto - sum), j = 0;
#pragma unroll
      for (int q = 0; q < 3; ++q)
        if (j == (uint32_t)q && left >= c[q]) {
          left -= c[q];
          ++j;
        }
      return {__shfl_sync(~0u, base + lane * 4 + j, at), __shfl_sync(~0u, left, at)};
    }
    unit -= __shfl_sync(~0u, upto, 31);
  }
  return {n, 0};
}

template <bool kBf16>
__device__ __forceinline__ float2 unpack16(uint32_t x) {
  if (kBf16) return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x));
  return __half22float2(*reinterpret_cast<const __half2*>(&x));
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if (kBf16) {
    const __nv_bfloat162 y = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&y);
  }
  const __half2 y = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&y);
}

// Four codes to two pairs of fp16.  int8: u = code + 128 behind fp16's exponent of 1024 is
// 1024 + u, from which 1152 leaves the code, all exact.
template <bool kE4m3>
__device__ __forceinline__ void widen(uint32_t w, uint32_t* lo, uint32_t* hi) {
  if (kE4m3) {
    const __half2_raw x = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xffff), __NV_E4M3);
    const __half2_raw y = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3);
    *lo = (uint32_t)x.x | (uint32_t)x.y << 16;
    *hi = (uint32_t)y.x | (uint32_t)y.y << 16;
  } else {
    const uint32_t u = w ^ 0x80808080u, p = __byte_perm(u, 0x64646464u, 0x4140),
                   q = __byte_perm(u, 0x64646464u, 0x4342);
    const uint32_t k1152 = 0x64806480u;
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&p),
                              *reinterpret_cast<const __half2*>(&k1152));
    const __half2 y = __hsub2(*reinterpret_cast<const __half2*>(&q),
                              *reinterpret_cast<const __half2*>(&k1152));
    *lo = *reinterpret_cast<const uint32_t*>(&x);
    *hi = *reinterpret_cast<const uint32_t*>(&y);
  }
}

// Four codes times a factor.
template <bool kE4m3>
__device__ __forceinline__ void decode4(uint32_t w, float by, float* x) {
  uint32_t lo, hi;
  widen<kE4m3>(w, &lo, &hi);
  const float2 a = unpack16<false>(lo), b = unpack16<false>(hi);
  x[0] = a.x * by, x[1] = a.y * by, x[2] = b.x * by, x[3] = b.y * by;
}

// Four values over their scale, which are not above the format's largest by more than rounding,
// to codes.  int8: 1.5 * 2^23 + x has rn(x) in its low bits, two's complement.
template <bool kE4m3>
__device__ __forceinline__ uint32_t encode4(const float* x) {
  if constexpr (kE4m3)
    return __nv_cvt_float2_to_fp8x2(make_float2(x[0], x[1]), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x[2], x[3]), __NV_SATFINITE, __NV_E4M3)
               << 16;
  uint32_t c[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = __float_as_uint(__fadd_rn(x[i], 12582912.f));
  return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
}
