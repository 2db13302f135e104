// Rows turned by their positions, and new tokens into the 8-bit KV blocks with the rotation on the
// way.
//
// Bound: HBM.  A block of threads has 16 tokens (of a sequence's block, where rows go into blocks):
// it makes the cosines and sines of all their pairs once, in shared memory, and its warps take the
// tokens' heads one by one, 4 loads of 16 bytes a lane under way at a time: 32,768 rows of 72 heads of
// 128 in 215 us, 5.6 TB/s (all 8 loads of 16 rows under way, and half the warps: 314).  New tokens of
// 8 KV and 64 query heads: 70,319 of them in 595 us, 4.6 TB/s; the keys' warps set the pace, which
// turn their rows twice, for the scale and for the codes.
#include <math.h>

#include "kv_store.cuh"

namespace {

constexpr uint32_t kWarps = 8;
constexpr uint32_t kResident = 4;  // blocks an SM: bytes under way
// Heads that a warp takes of 16 tokens: the more, the less the cosines and sines cost; fewer where
// tokens are few.  Always two against always ten, in us: 72 heads of 64 rows 10.4 and 22.9, 2,048 rows 25.7
// and 31.0, 9,728 85 and 72, 16,384 130 and 119, 19,456 152 and 131, 32,768 243 and 216; appended, 64 and 8
// heads, 64 rows 12.7 and 24.8, 2,048 29 and 39, 8,192 85 and 98, 9,728 99 and 101, 19,456 187 and 172,
// 32,768 309 and 282.  From 4,096 rows on ten are the better for rows without blocks.
constexpr uint32_t kFewBlocks = 1216, kPerWarp[2] = {2, 10};

struct RotateArgs {
  const unsigned char* x;
  unsigned char* out;
  uint64_t x_stride, out_stride, rows;
  const int32_t* pos;
  uint32_t heads;
  netkv_rotary rot;
};

// Rows [lo, hi) of a head, of up to 16 that start at `x`, turned into `out`.
template <int kDim, bool kBf16>
__device__ __forceinline__ void turn_rows(const Turns& t, const unsigned char* x, uint64_t x_stride,
                                          unsigned char* out, uint64_t out_stride, uint32_t lo,
                                          uint32_t hi) {
  constexpr int kLanes = kDim / 8, kRows = 32 / kLanes, kSteps = kBlockTokens / kRows;
  constexpr int kPart = kSteps < 4 ? kSteps : 4;  // loads under way at a time
  const uint32_t lane = threadIdx.x & 31, col = (lane % kLanes) * 8, row0 = lane / kLanes;
#pragma unroll 1
  for (int from = 0; from < kSteps; from += kPart) {
    if (row0 + from * kRows - lane / kLanes >= hi) break;
    uint4 v[kPart];
#pragma unroll
    for (int i = 0; i < kPart; ++i) {
      const uint32_t row = row0 + (from + i) * kRows;
      v[i] = make_uint4(0, 0, 0, 0);
      if (row >= lo && row < hi)
        v[i] = __ldcs(reinterpret_cast<const uint4*>(x + ((int64_t)(row * x_stride) + col) * 2));
    }
#pragma unroll
    for (int i = 0; i < kPart; ++i) {
      const uint32_t row = row0 + (from + i) * kRows;
      float y[8];
      turn8<kBf16>(t, row, lane % kLanes, v[i], y);
      if (row >= lo && row < hi)
        __stcs(reinterpret_cast<uint4*>(out + (row * out_stride + col) * 2),
               make_uint4(pack16<kBf16>(y[0], y[1]), pack16<kBf16>(y[2], y[3]),
                          pack16<kBf16>(y[4], y[5]), pack16<kBf16>(y[6], y[7])));
    }
  }
}

struct Table {
  alignas(16) float cos[kBlockTokens * 64], sin[kBlockTokens * 64];
};

template <int kDim, bool kBf16>
__global__ void __launch_bounds__(kWarps * 32, kResident) rotate_kernel(const __grid_constant__ RotateArgs a) {
  __shared__ Table table;
  const uint64_t first = (uint64_t)blockIdx.x * kBlockTokens;
  const uint32_t n = (uint32_t)min((uint64_t)kBlockTokens, a.rows - first);
  make_turns(a.rot, table.cos, table.sin, a.pos, a.rows, (int64_t)first, 0, 0, n);
  __syncthreads();
  const Turns t = {table.cos, table.sin, a.rot.pairs, a.rot.interleaved != 0};
  for (uint32_t h = blockIdx.y * kWarps + threadIdx.x / 32; h < a.heads; h += gridDim.y * kWarps)
    turn_rows<kDim, kBf16>(t, a.x + (first * a.x_stride + (uint64_t)h * kDim) * 2, a.x_stride,
                           a.out + (first * a.out_stride + (uint64_t)h * kDim) * 2, a.out_stride, 0,
                           n);
}

struct AppendArgs {
  StoreArgs s;
  const unsigned char* q;
  unsigned char* q_out;
  uint64_t q_stride, q_out_stride;
  const int32_t* pos;
  uint32_t heads;  // of queries; 0: none
  netkv_rotary rot;
};

// Blocks that sequence i's new rows touch, in its table or past it.
__device__ __forceinline__ uint32_t reached(const StoreArgs& a, uint32_t i) {
  const uint64_t n = row_range(a.off, i, a.rows).count, s = a.start ? a.start[i] : 0;
  return n ? (uint32_t)((s + n + kBlockTokens - 1) / kBlockTokens - s / kBlockTokens) : 0;
}

// The block `at` of those that a sequence's new rows touch: its keys and values, and its queries.
template <int kDim, bool kBf16, bool kE4m3>
__device__ __forceinline__ void append_block(const AppendArgs& a, Table& table, uint32_t seq,
                                             uint32_t at) {
  const RowRange r = row_range(a.s.off, seq, a.s.rows);
  const uint64_t start = a.s.start ? a.s.start[seq] : 0, block = start / kBlockTokens + at;
  const uint64_t pos0 = block * kBlockTokens;
  const uint32_t lo = start > pos0 ? (uint32_t)(start - pos0) : 0;
  const uint32_t hi = (uint32_t)min((uint64_t)kBlockTokens, start + r.count - pos0);
  const int64_t row0 = (int64_t)(r.first + pos0 - start);  // of the block's row 0
  make_turns(a.rot, table.cos, table.sin, a.pos, a.s.rows, row0, (int64_t)pos0, lo, hi);
  __syncthreads();
  const Turns t = {table.cos, table.sin, a.rot.pairs, a.rot.interleaved != 0};
  const uint32_t kv = a.s.kv.heads, units = 2 * kv + a.heads;
  for (uint32_t u = blockIdx.y * kWarps + threadIdx.x / 32; u < units; u += gridDim.y * kWarps) {
    if (u < 2 * kv) {
      if (block >= a.s.width) continue;
      const Units x = {seq, at, 1, at + 1, u / 2, (u & 1) != 0};
      if (u & 1) store_block<kDim, kBf16, kE4m3>(a.s, x, at);
      else store_block<kDim, kBf16, kE4m3, true>(a.s, x, at, &t);
    } else {
      const int64_t head = (int64_t)(u - 2 * kv) * kDim;
      turn_rows<kDim, kBf16>(t, a.q + (row0 * (int64_t)a.q_stride + head) * 2, a.q_stride,
                             a.q_out + (row0 * (int64_t)a.q_out_stride + head) * 2, a.q_out_stride,
                             lo, hi);
    }
  }
}

template <int kDim, bool kBf16, bool kE4m3, bool kMany>
__global__ void __launch_bounds__(kWarps * 32, kResident - 1) append_kernel(const __grid_constant__ AppendArgs a) {
  __shared__ Table table;
  if (blockIdx.y == 0) check_ranges(a.s);
  if constexpr (kMany) {
    const uint32_t seq = blockIdx.x / a.s.parts;
    if (seq >= a.s.n_seqs) return;
    const uint32_t end = reached(a.s, seq);
    for (uint32_t at = blockIdx.x % a.s.parts; at < end; at += a.s.parts) {
      append_block<kDim, kBf16, kE4m3>(a, table, seq, at);
      __syncthreads();
    }
  } else {
    const Found f =
        find_unit(a.s.n_seqs, blockIdx.x, [&](uint32_t i) { return reached(a.s, i); });
    if (f.seq < a.s.n_seqs) append_block<kDim, kBf16, kE4m3>(a, table, f.seq, f.unit);
  }
}

// Blocks of threads that share 16 tokens' heads.
uint32_t shares(uint32_t units, uint64_t blocks) {
  const uint32_t per = kWarps * kPerWarp[blocks >= kFewBlocks];
  return min((units + per - 1) / per, 65535u);
}

}  // namespace

extern "C" netkv_status netkv_rotary_set(netkv_rotary* rot, uint32_t pairs, const double* frequency,
                                         uint32_t axes, const uint32_t* sections,
                                         uint32_t interleaved) {
  if (!rot || !frequency || pairs < 8 || pairs > 64 || pairs % 8 || axes < 1 || axes > 4 ||
      (!sections && axes > 1) || interleaved > 1)
    return NETKV_EINVAL;
  netkv_rotary r = {};
  r.pairs = pairs;
  r.axes = axes;
  r.interleaved = interleaved;
  uint64_t at = 0;
  for (uint32_t i = 0; i < axes; ++i) {
    const uint64_t n = sections ? sections[i] : pairs;
    if (at + n > pairs) return NETKV_EINVAL;
    for (uint64_t p = at; p < at + n; ++p) r.axis[p] = (uint8_t)i;
    at += n;
  }
  if (at != pairs) return NETKV_EINVAL;
  const double kTurn = 6.283185307179586476925;
  for (uint32_t p = 0; p < pairs; ++p) {
    if (!(frequency[p] >= 0.0) || !(frequency[p] < kTurn)) return NETKV_EINVAL;
    // to 2^-52 of itself by 2 pi and the division, and to 2^-64; what rounds to a whole turn is none
    const double part = frequency[p] / kTurn;
    r.step[p] = part < 1.0 ? (uint64_t)ldexp(part, 64) : 0;
  }
  *rot = r;
  return NETKV_OK;
}

extern "C" netkv_status netkv_rotate(const netkv_rotary* rot, uint32_t dtype, const void* d_x,
                                     uint64_t x_stride, uint32_t heads, uint32_t head_dim,
                                     uint64_t rows, const int32_t* d_pos, void* d_out,
                                     uint64_t out_stride, netkv_stream_t stream) {
  if (dtype > NETKV_BF16 || (head_dim != 64 && head_dim != 128) || heads == 0 || heads > 65535 ||
      !rotary_ok(rot, head_dim) || rows >> 31)
    return NETKV_EINVAL;
  if (rows == 0) return NETKV_OK;
  const uint64_t row = (uint64_t)heads * head_dim;
  if (!rows_ok(d_x, x_stride, row) || !rows_ok(d_out, out_stride, row) || !d_pos ||
      !aligned_to(d_pos, 4) || (d_x == d_out && x_stride != out_stride))
    return NETKV_EINVAL;
  const RotateArgs a = {(const unsigned char*)d_x, (unsigned char*)d_out, x_stride, out_stride, rows,
                        d_pos, heads, *rot};
  const uint64_t blocks = (rows + kBlockTokens - 1) / kBlockTokens;
  const dim3 grid((unsigned)blocks, shares(heads, blocks));
  const bool bf = dtype == NETKV_BF16;
  auto go = [&](auto kernel) { kernel<<<grid, kWarps * 32, 0, (cudaStream_t)stream>>>(a); };
  if (head_dim == 64) go(bf ? rotate_kernel<64, true> : rotate_kernel<64, false>);
  else go(bf ? rotate_kernel<128, true> : rotate_kernel<128, false>);
  return netkv_launch_status();
}

extern "C" netkv_status netkv_kv_append(const netkv_kv_pages* pages, const netkv_rotary* rot,
                                        uint32_t dtype, const void* d_k, uint64_t k_stride,
                                        const void* d_v, uint64_t v_stride, uint32_t n_seqs,
                                        const uint64_t* d_off, uint64_t rows,
                                        const uint32_t* d_start, const int32_t* d_table,
                                        uint32_t width, const int32_t* d_pos, uint32_t heads,
                                        const void* d_q, uint64_t q_stride, void* d_q_out,
                                        uint64_t q_out_stride, int* d_status,
                                        netkv_stream_t stream) {
  if (!kv_pages_ok(pages) || dtype > NETKV_BF16 || !rotary_ok(rot, pages->head_dim) ||
      (!d_pos && rot->axes > 1) || (d_q && (heads == 0 || heads > 65535)))
    return NETKV_EINVAL;
  if (n_seqs == 0 || rows == 0) return NETKV_OK;
  const uint64_t row = (uint64_t)pages->kv_heads * pages->head_dim,
                 q_row = (uint64_t)heads * pages->head_dim;
  if (!rows_ok(d_k, k_stride, row) || !rows_ok(d_v, v_stride, row) || !d_off || !d_table ||
      !aligned_to(d_off, 8) || !aligned_to(d_table, 4) || !aligned_to(d_start, 4) ||
      !aligned_to(d_pos, 4) || !aligned_to(d_status, 4) || width == 0 || width >= (1u << 28) ||
      rows >> 31 || n_seqs >> 24 ||
      (d_q && (!rows_ok(d_q, q_stride, q_row) || !rows_ok(d_q_out, q_out_stride, q_row) ||
               (d_q == d_q_out && q_stride != q_out_stride))))
    return NETKV_EINVAL;
  const uint32_t parts =
      n_seqs > kSearched ? (uint32_t)(rows / ((uint64_t)kBlockTokens * n_seqs)) + 1 : 0;
  // a sequence touches at most one block more than its rows fill at either end
  const uint64_t blocks =
      parts ? (uint64_t)parts * n_seqs : rows / kBlockTokens + 2ull * n_seqs;
  if (blocks >> 31) return NETKV_EINVAL;
  const AppendArgs a = {{kv_args(pages), (const unsigned char*)d_k, (const unsigned char*)d_v,
                         k_stride, v_stride, rows, d_off, d_start, d_table, n_seqs, width, parts,
                         d_status},
                        (const unsigned char*)d_q, (unsigned char*)d_q_out, q_stride, q_out_stride,
                        d_pos, d_q ? heads : 0, *rot};
  const dim3 grid((unsigned)blocks, shares(2 * pages->kv_heads + a.heads, blocks));
  const bool bf = dtype == NETKV_BF16, e4 = pages->format == NETKV_KV_E4M3;
  auto go = [&](auto kernel) { kernel<<<grid, kWarps * 32, 0, (cudaStream_t)stream>>>(a); };
  auto pick = [&](auto dim, auto many) {
    constexpr int kDim = decltype(dim)::value;
    constexpr bool kMany = decltype(many)::value;
    if (bf && e4) go(append_kernel<kDim, true, true, kMany>);
    else if (bf) go(append_kernel<kDim, true, false, kMany>);
    else if (e4) go(append_kernel<kDim, false, true, kMany>);
    else go(append_kernel<kDim, false, false, kMany>);
  };
  auto widths = [&](auto many) {
    if (pages->head_dim == 64) pick(std::integral_constant<int, 64>(), many);
    else pick(std::integral_constant<int, 128>(), many);
  };
  if (parts) widths(std::true_type());
  else widths(std::false_type());
  return netkv_launch_status();
}
