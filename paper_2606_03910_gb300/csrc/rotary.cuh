// Rotary positions: the rotation of a head's channel pairs by angles that grow with the token's
// position, (x, y) -> (x cos a - y sin a, y cos a + x sin a), a = position * frequency.
//
// An angle is needed only up to whole turns, and a 64-bit product wraps exactly there: a pair's
// frequency is held as the part of a turn that one position is, times 2^64, and position * step
// mod 2^64 is the angle.  A step is off by 2^-52 of itself at most (2 pi and the division, in doubles), so
// the angle of position t at frequency f by t * f * 2^-52 of a radian, and by 2^-23 more where its upper
// half becomes fp32 for sincospif: 2^-21 at the last of 2^31 positions for frequencies up to 1.  (An fp32
// product of a position near 2^20 would be 2^-4 off.)
#pragma once

#include "kv_common.cuh"

inline bool rotary_ok(const netkv_rotary* r, uint32_t head_dim) {
  if (!r || r->pairs < 8 || r->pairs % 8 || r->pairs * 2 > head_dim || r->axes < 1 || r->axes > 4 ||
      r->interleaved > 1 || r->reserved)
    return false;
  for (uint32_t p = 0; p < r->pairs; ++p)
    if (r->axis[p] >= r->axes) return false;
  return true;
}

// Cosines and sines of 16 tokens in shared memory, shared by all heads: a row's pairs in the order
// (p / 4 % 2, p / 8, p % 4), so that neighbouring lanes, 8 pairs each, read neighbouring 16 bytes.
struct Turns {
  const float* cos;  // [16][pairs]
  const float* sin;
  uint32_t pairs;
  bool interleaved;
};

__device__ __forceinline__ uint32_t turn_place(uint32_t pairs, uint32_t p) {
  return p / 4 % 2 * (pairs / 2) + p / 8 * 4 + p % 4;
}

// Rows [lo, hi) of the table, by the block's threads: row r is of the token with position
// first + r (pos NULL) or pos[axis * rows + at + r].
__device__ __forceinline__ void make_turns(const netkv_rotary& rot, float* cos, float* sin,
                                           const int32_t* pos, uint64_t rows, int64_t at,
                                           int64_t first, uint32_t lo, uint32_t hi) {
  for (uint32_t i = threadIdx.x; i < (hi - lo) * rot.pairs; i += blockDim.x) {
    const uint32_t r = lo + i / rot.pairs, p = i % rot.pairs;
    const int64_t t = pos ? pos[rot.axis[p] * rows + (at + r)] : first + r;
    const int32_t part = (int32_t)(((uint64_t)t * rot.step[p]) >> 32);
    float s, c;
    sincospif((float)part * 4.656612873077393e-10f, &s, &c);  // 2^-31: in half turns
    const uint32_t to = r * rot.pairs + turn_place(rot.pairs, p);
    cos[to] = c;
    sin[to] = s;
  }
}

// The 8 channels of a lane, chunk `j` of row `row`, turned.  Called by whole warps: lanes of a row
// are neighbours, so a pair's other channel is pairs / 8 lanes away.
template <bool kBf16>
__device__ __forceinline__ void turn8(const Turns& t, uint32_t row, uint32_t j, const uint4& x,
                                      float* y) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w}, apart = t.pairs / 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 z = unpack16<kBf16>(w[i]);
    y[2 * i] = z.x;
    y[2 * i + 1] = z.y;
  }
  const float* cos = t.cos + row * t.pairs;
  const float* sin = t.sin + row * t.pairs;
  if (t.interleaved) {
    if (j >= 2 * apart) return;
    const uint32_t at = turn_place(t.pairs, 4 * j);
    const float4 c = *reinterpret_cast<const float4*>(cos + at);
    const float4 s = *reinterpret_cast<const float4*>(sin + at);
    const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = y[2 * i], b = y[2 * i + 1];
      y[2 * i] = fmaf(a, cs[i], -(b * sn[i]));
      y[2 * i + 1] = fmaf(b, cs[i], a * sn[i]);
    }
    return;
  }
  const bool first = j < apart, in = j < 2 * apart;
  const uint32_t lane = threadIdx.x & 31, from = in ? first ? lane + apart : lane - apart : lane;
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = __shfl_sync(~0u, w[i], from);
  if (!in) return;
  const uint32_t at = (first ? j : j - apart) * 4;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const float4 c = *reinterpret_cast<const float4*>(cos + q * (t.pairs / 2) + at);
    const float4 s = *reinterpret_cast<const float4*>(sin + q * (t.pairs / 2) + at);
    const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 z = unpack16<kBf16>(o[q * 2 + i / 2]);
      const float other = i % 2 ? z.y : z.x;
      y[q * 4 + i] = fmaf(y[q * 4 + i], cs[i], first ? -(other * sn[i]) : other * sn[i]);
    }
  }
}
