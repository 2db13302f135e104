// New rows into the 8-bit KV blocks: what netkv_kv_store and netkv_kv_append share.
#pragma once

#include "rotary.cuh"

constexpr float kSmallest = 7.8886091e-31f;  // 2^-100: blocks below are held as zeros, so that
                                             // 1 / s stays finite

// A unit is one block of one KV head, its keys or its values, taken by one warp: 16 rows of
// kDim 16-bit values.  A lane has 8 neighbouring values of a row, kDim / 8 lanes a row.
// Up to kSearched sequences a warp finds its block by counting (find_unit), 128 sequences a step, so
// that ragged batches spread evenly.  Of more, a sequence has `parts` warps for a head's keys, as many
// as an average one has blocks, which take its blocks in turn: with each warp counting, a call's time
// would grow with the square of its sequences.  Ragged rows of 2 heads stored: 300 sequences 47 us by
// counting and 61 in turn, 600 125 and 100, 4,096 2,860 and 590; a token each: 300 8.6 and 7.1, 4,096
// 248 and 17, 262,144 407 ms by counting.
constexpr uint32_t kSearched = 512;
struct Units {
  uint32_t seq, block, step, end;  // blocks block, block + step, ... below end
  uint32_t head;
  bool values;
};

struct StoreArgs {
  KvArgs kv;
  const unsigned char* k;
  const unsigned char* v;
  uint64_t k_stride, v_stride, rows;
  const uint64_t* off;
  const uint32_t* start;
  const int32_t* table;
  uint32_t n_seqs, width;
  uint32_t parts;  // kMany: warps of a sequence for a head's keys
  int* status;
};

// Blocks that sequence i's new rows touch, cut to its table.
__device__ __forceinline__ uint32_t touched(const StoreArgs& a, uint32_t i) {
  const uint64_t n = row_range(a.off, i, a.rows).count, s = a.start ? a.start[i] : 0;
  if (n == 0) return 0;
  const uint64_t end = min((s + n + kBlockTokens - 1) / kBlockTokens, (uint64_t)a.width);
  return end > s / kBlockTokens ? (uint32_t)(end - s / kBlockTokens) : 0;
}

// Bad offsets or a table that is too short, said once a sequence.
__device__ __forceinline__ void check_ranges(const StoreArgs& a) {
  for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < a.n_seqs;
       i += (uint64_t)gridDim.x * blockDim.x) {
    const RowRange r = row_range(a.off, (uint32_t)i, a.rows);
    const uint64_t s = a.start ? a.start[i] : 0;
    if (r.bad || (r.count && s + r.count > (uint64_t)a.width * kBlockTokens))
      flag_status(a.status, NETKV_DEV_ERANGE);
  }
}

// Block `at` of those that u's sequence touches, for one head.  kTurn: the rows are turned by their
// positions on the way, and what goes by their 16-bit values elsewhere goes by the turned fp32 ones.
template <int kDim, bool kBf16, bool kE4m3, bool kTurn = false>
__device__ __forceinline__ void store_block(const StoreArgs& a, const Units& u, uint32_t at,
                                            const Turns* turns = nullptr) {
  constexpr int kLanes = kDim / 8, kRows = 32 / kLanes, kSteps = kBlockTokens / kRows;
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t start = a.start ? a.start[u.seq] : 0;
  const RowRange r = row_range(a.off, u.seq, a.rows);
  const uint64_t block = start / kBlockTokens + at;
  const int32_t page = a.table[(uint64_t)u.seq * a.width + block];
  if (page < 0 || (uint32_t)page >= a.kv.n_pages) {
    if (lane == 0) flag_status(a.status, NETKV_DEV_ERANGE);
    return;
  }
  const unsigned char* src = u.values ? a.v : a.k;
  const uint64_t stride = u.values ? a.v_stride : a.k_stride;
  const uint64_t part = (uint64_t)page * a.kv.heads + u.head;
  unsigned char* codes = (u.values ? a.kv.v : a.kv.k) + part * (kBlockTokens * kDim);
  float* scale = (u.values ? a.kv.v_scale : a.kv.k_scale) + part;

  const uint32_t col = (lane % kLanes) * 8, row0 = lane / kLanes;
  const uint64_t pos0 = block * kBlockTokens;
  // rows [lo, hi) of the block are new, those before lo are from earlier calls
  const uint32_t lo = start > pos0 ? (uint32_t)(start - pos0) : 0;
  const uint32_t hi = (uint32_t)min((uint64_t)kBlockTokens, start + r.count - pos0);
  const bool all = hi - lo == kBlockTokens;
  // all loads at once: where a row is not a new one, the nearest that is, for nothing
  const unsigned char* from =
      src + ((r.first + (pos0 + lo - start)) * stride + (uint64_t)u.head * kDim + col) * 2;
  uint4 x[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const uint32_t row = min(max(row0 + i * kRows, lo), hi - 1);
    x[i] = __ldcs(reinterpret_cast<const uint4*>(from + (row - lo) * stride * 2));
  }
  if (!all) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const uint32_t row = row0 + i * kRows;
      if (row < lo || row >= hi) x[i] = make_uint4(0, 0, 0, 0);
    }
  }
  const float was = lo ? *scale : 0.f;
  float largest;
  // The turned rows are made twice, for their largest and for their codes: kept, they would take 64
  // registers a thread and half of the SM's warps.
  auto turned = [&](int i, float* y) {
    const uint32_t row = row0 + i * kRows;
    const bool fresh = all || (row >= lo && row < hi);  // others have no angles
    turn8<kBf16>(*turns, row, lane % kLanes, x[i], y);
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // infinities and NaN have no code: they are held as zeros
      const bool fine = fabsf(y[j]) <= 3.4028235e38f;
      odd |= fresh && !fine;
      y[j] = fresh && fine ? y[j] : 0.f;
    }
    return odd;
  };
  if constexpr (kTurn) {
    largest = 0.f;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      float y[8];
      odd |= turned(i, y);
#pragma unroll
      for (int j = 0; j < 8; ++j) largest = fmaxf(largest, fabsf(y[j]));
    }
    if (__any_sync(~0u, odd) && lane == 0) flag_status(a.status, NETKV_DEV_EDOMAIN);
    largest = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(largest)));
#pragma unroll
    for (int i = 0; i < kSteps; ++i)  // not to be kept after all
      asm volatile("" : "+r"(x[i].x), "+r"(x[i].y), "+r"(x[i].z), "+r"(x[i].w));
  } else {
    // Magnitudes are in the order of their bits, two values a word.
    constexpr uint32_t kInf = kBf16 ? 0x7f80 : 0x7c00;
    auto top_bits = [&]() {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        m = __vimax3_u16x2(m, x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu);
        m = __vimax3_u16x2(m, x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu);
      }
      return __reduce_max_sync(~0u, max(m & 0xffffu, m >> 16));
    };
    uint32_t top = top_bits();
    if (top >= kInf) {  // infinities and NaN have no code: they are held as zeros
      if (lane == 0) flag_status(a.status, NETKV_DEV_EDOMAIN);
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&x[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if ((w[j] & 0x7fffu) >= kInf) w[j] &= 0xffff0000u;
          if ((w[j] >> 16 & 0x7fffu) >= kInf) w[j] &= 0x0000ffffu;
        }
      }
      top = top_bits();
    }
    largest = unpack16<kBf16>(top).x;
  }
  const float fresh = largest < kSmallest ? 0.f : largest / (kE4m3 ? 448.f : 127.f);
  const float now = fmaxf(was, fresh);
  const float inv = now > 0.f ? 1.f / now : 0.f;
  unsigned char* to = codes + row0 * kDim + col;
  const bool grows = lo && now > was;
  const float ratio = grows ? was / now : 0.f;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const uint32_t row = row0 + i * kRows;
    uint2* at = reinterpret_cast<uint2*>(to + i * kRows * kDim);
    float y[8];
    if constexpr (kTurn) turned(i, y);  // (a whole warp's work)
    if (all || (row >= lo && row < hi)) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 z = kTurn ? make_float2(y[2 * j], y[2 * j + 1]) : unpack16<kBf16>(w[j]);
        y[2 * j] = z.x * inv;
        y[2 * j + 1] = z.y * inv;
      }
      *at = make_uint2(encode4<kE4m3>(y), encode4<kE4m3>(y + 4));
    } else if (grows && row < lo) {
      // the block's scale grew: its earlier codes follow
      const uint2 old = *at;
      decode4<kE4m3>(old.x, ratio, y);
      decode4<kE4m3>(old.y, ratio, y + 4);
      *at = make_uint2(encode4<kE4m3>(y), encode4<kE4m3>(y + 4));
    }
  }
  if (lane == 0) *scale = now;
}
