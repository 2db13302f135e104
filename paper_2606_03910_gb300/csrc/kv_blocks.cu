// The 8-bit KV blocks: new keys and values into blocks, blocks back into rows, and the
// eviction of blocks by the attention weight that they have drawn.
//
// A block is 16 tokens of one KV head (Sec. III-B's B_tok) with one scale s = max|x| / c,
// c = 127 (int8) or 448 (e4m3): code = rn(x * (1 / s)), value = code * s.  Dividing once a
// block and multiplying an element costs one more rounding than x / s, 2^-24 of a value that
// is kept to 2^-8 or 2^-4.
//
// Storing and loading are bound by HBM: 223,000 rows of 8 heads of 128 in 235 us (5.8 TB/s) and
// back in 207 (6.6 TB/s), one warp a block and head with all of its loads under way at once.
// With the loads behind a branch each, the way back took 277 us; with conversions one value at a
// time, the way there 476.
#include "kv_store.cuh"

namespace {

constexpr uint32_t kWarps = 8;            // warps of a store or load block, one unit each

template <bool kMany>
__device__ __forceinline__ Units units_of(const StoreArgs& a) {
  const uint32_t w = blockIdx.x * kWarps + threadIdx.x / 32, per = 2 * a.kv.heads;
  const uint32_t head = (w % per) / 2, n = w / per;
  const bool values = (w & 1) != 0;
  if (kMany) {
    const uint32_t seq = n / a.parts;
    return {seq, n % a.parts, a.parts, seq < a.n_seqs ? touched(a, seq) : 0, head, values};
  }
  const Found f = find_unit(a.n_seqs, n, [&](uint32_t i) { return touched(a, i); });
  return {f.seq, f.unit, 1, f.unit + 1, head, values};
}

template <int kDim, bool kBf16, bool kE4m3, bool kMany>
__global__ void __launch_bounds__(kWarps * 32) store_kernel(const __grid_constant__ StoreArgs a) {
  check_ranges(a);
  const Units u = units_of<kMany>(a);
  if (u.seq >= a.n_seqs) return;
  if constexpr (kMany) {
    for (uint32_t at = u.block; at < u.end; at += u.step) store_block<kDim, kBf16, kE4m3>(a, u, at);
  } else {
    store_block<kDim, kBf16, kE4m3>(a, u, u.block);
  }
}

// Rows from blocks: the reverse walk, its output rows through StoreArgs' k and v.
template <int kDim, bool kBf16, bool kE4m3>
__device__ __forceinline__ void load_block(const StoreArgs& a, const Units& u, uint32_t at) {
  constexpr int kLanes = kDim / 8, kRows = 32 / kLanes, kSteps = kBlockTokens / kRows;
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t start = a.start ? a.start[u.seq] : 0;
  const RowRange r = row_range(a.off, u.seq, a.rows);
  const uint64_t block = start / kBlockTokens + at;
  const int32_t page = a.table[(uint64_t)u.seq * a.width + block];
  const bool there = page >= 0 && (uint32_t)page < a.kv.n_pages;
  if (!there && lane == 0) flag_status(a.status, NETKV_DEV_ERANGE);
  unsigned char* dst = const_cast<unsigned char*>(u.values ? a.v : a.k);
  const uint64_t stride = u.values ? a.v_stride : a.k_stride;
  const uint64_t part = (uint64_t)(there ? page : 0) * a.kv.heads + u.head;
  const unsigned char* codes = (u.values ? a.kv.v : a.kv.k) + part * (kBlockTokens * kDim);
  // an absent page's rows are zeros; page 0 is read in its place
  const float s = there ? (u.values ? a.kv.v_scale : a.kv.k_scale)[part] : 0.f;
  const uint32_t col = (lane % kLanes) * 8, row0 = lane / kLanes;
  const uint64_t pos0 = block * kBlockTokens;
  const uint32_t lo = start > pos0 ? (uint32_t)(start - pos0) : 0;
  const uint32_t hi = (uint32_t)min((uint64_t)kBlockTokens, start + r.count - pos0);
  const bool all = hi - lo == kBlockTokens;
  uint2 x[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const uint32_t row = row0 + i * kRows;
    x[i] = __ldcs(reinterpret_cast<const uint2*>(codes + row * kDim + col));
  }
  unsigned char* to =
      dst + ((int64_t)(r.first + pos0 - start + row0) * (int64_t)stride +
             (int64_t)u.head * kDim + col) * 2;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const uint32_t row = row0 + i * kRows;
    if (all || (row >= lo && row < hi)) {
      float y[8];
      decode4<kE4m3>(there ? x[i].x : 0u, s, y);
      decode4<kE4m3>(there ? x[i].y : 0u, s, y + 4);
      *reinterpret_cast<uint4*>(to) =
          make_uint4(pack16<kBf16>(y[0], y[1]), pack16<kBf16>(y[2], y[3]),
                     pack16<kBf16>(y[4], y[5]), pack16<kBf16>(y[6], y[7]));
    }
    to += kRows * stride * 2;
  }
}

template <int kDim, bool kBf16, bool kE4m3, bool kMany>
__global__ void __launch_bounds__(kWarps * 32) load_kernel(const __grid_constant__ StoreArgs a) {
  check_ranges(a);
  const Units u = units_of<kMany>(a);
  if (u.seq >= a.n_seqs) return;
  if constexpr (kMany) {
    for (uint32_t at = u.block; at < u.end; at += u.step) load_block<kDim, kBf16, kE4m3>(a, u, at);
  } else {
    load_block<kDim, kBf16, kE4m3>(a, u, u.block);
  }
}

// Units of a call: at most one block a sequence more than its rows fill, at either end; of many
// sequences, the average's blocks and one for each.
template <bool kStore>
netkv_status blocks_call(const netkv_kv_pages* pages, uint32_t dtype, const void* d_k,
                         uint64_t k_stride, const void* d_v, uint64_t v_stride, uint32_t n_seqs,
                         const uint64_t* d_off, uint64_t rows, const uint32_t* d_start,
                         const int32_t* d_table, uint32_t width, int* d_status,
                         netkv_stream_t stream) {
  if (!kv_pages_ok(pages) || dtype > NETKV_BF16) return NETKV_EINVAL;
  if (n_seqs == 0 || rows == 0) return NETKV_OK;
  const uint64_t row = (uint64_t)pages->kv_heads * pages->head_dim;
  if (!rows_ok(d_k, k_stride, row) || !rows_ok(d_v, v_stride, row) || !d_off || !d_table ||
      !aligned_to(d_off, 8) || !aligned_to(d_table, 4) || !aligned_to(d_start, 4) ||
      !aligned_to(d_status, 4) || width == 0 || width >= (1u << 28) || rows >> 31 ||
      n_seqs >> 24)
    return NETKV_EINVAL;
  const uint32_t parts =
      n_seqs > kSearched ? (uint32_t)(rows / ((uint64_t)kBlockTokens * n_seqs)) + 1 : 0;
  const uint64_t units =
      (parts ? (uint64_t)parts * n_seqs : rows / kBlockTokens + 2ull * n_seqs) * 2 * pages->kv_heads;
  const uint64_t grid = (units + kWarps - 1) / kWarps;
  if (units >> 32 || grid >> 31) return NETKV_EINVAL;
  const StoreArgs a = {kv_args(pages), (const unsigned char*)d_k, (const unsigned char*)d_v,
                       k_stride, v_stride, rows, d_off, d_start, d_table, n_seqs, width, parts,
                       d_status};
  const bool bf = dtype == NETKV_BF16, e4 = pages->format == NETKV_KV_E4M3;
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)grid, kWarps * 32, 0, (cudaStream_t)stream>>>(a);
  };
  auto pick = [&](auto dim, auto many) {
    constexpr int kDim = decltype(dim)::value;
    constexpr bool kMany = decltype(many)::value;
    if (bf && e4)
      go(kStore ? store_kernel<kDim, true, true, kMany> : load_kernel<kDim, true, true, kMany>);
    else if (bf)
      go(kStore ? store_kernel<kDim, true, false, kMany> : load_kernel<kDim, true, false, kMany>);
    else if (e4)
      go(kStore ? store_kernel<kDim, false, true, kMany> : load_kernel<kDim, false, true, kMany>);
    else
      go(kStore ? store_kernel<kDim, false, false, kMany> : load_kernel<kDim, false, false, kMany>);
  };
  auto widths = [&](auto many) {
    if (pages->head_dim == 64) pick(std::integral_constant<int, 64>(), many);
    else pick(std::integral_constant<int, 128>(), many);
  };
  if (parts) widths(std::true_type());
  else widths(std::false_type());
  return netkv_launch_status();
}

// ------------------------------------------------------------------ eviction
// One block of threads a sequence, a thread per eight neighbouring entries, 1,024 at most.
constexpr uint32_t kEvictPer = 8, kEvictMost = 1024;

// Weights in the order of unsigned keys; NaN above every number, the two zeros alike.
__device__ __forceinline__ uint32_t weight_key(float x) {
  if (x != x) return ~0u;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct EvictArgs {
  const int32_t* table;
  const uint32_t* len;
  const float* mass;
  const uint32_t* budget;
  uint32_t width, sink, recent;
  int32_t* table_out;
  uint32_t* len_out;
  float* mass_out;
  int32_t* freed;
  uint32_t* n_freed;
  int* status;
};

// Exclusive sums over the block of two counts; every thread gets its own and the totals.
__device__ __forceinline__ uint2 block_scan(uint2 x, uint2* total, uint2* scratch) {
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32, warps = blockDim.x / 32;
  uint2 y = x;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint32_t p = __shfl_up_sync(~0u, y.x, d), q = __shfl_up_sync(~0u, y.y, d);
    if (lane >= (uint32_t)d) y.x += p, y.y += q;
  }
  __syncthreads();  // scratch of an earlier call has been read
  if (lane == 31) scratch[warp] = y;
  __syncthreads();
  const uint2 z = lane < warps ? scratch[lane] : make_uint2(0, 0);
  const uint2 before = make_uint2(__reduce_add_sync(~0u, lane < warp ? z.x : 0),
                                  __reduce_add_sync(~0u, lane < warp ? z.y : 0));
  *total = make_uint2(__reduce_add_sync(~0u, z.x), __reduce_add_sync(~0u, z.y));
  return make_uint2(before.x + y.x - x.x, before.y + y.y - x.y);
}

// One pass of the selection: 11 bits of the keys as 64 groups of 32 bins.
struct Bins {
  uint32_t group[64], bin[2048];
};

// The bin in which the left-th key lies, and how many of its keys are up to that one; found by
// each warp for itself.
__device__ __forceinline__ uint2 find_bin(const Bins& h, uint32_t left) {
  const uint32_t lane = threadIdx.x & 31;
  const uint32_t x = h.group[2 * lane], y = h.group[2 * lane + 1];
  uint32_t upto = x + y;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint32_t z = __shfl_up_sync(~0u, upto, d);
    if (lane >= (uint32_t)d) upto += z;
  }
  const int at = __ffs(__ballot_sync(~0u, left <= upto)) - 1;  // there is one
  const uint32_t before = __shfl_sync(~0u, upto - x - y, at), first = __shfl_sync(~0u, x, at);
  const bool second = left - before > first;
  left -= before + (second ? first : 0);
  const uint32_t group = 2 * at + second, mine = h.bin[group * 32 + lane];
  upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint32_t z = __shfl_up_sync(~0u, upto, d);
    if (lane >= (uint32_t)d) upto += z;
  }
  const int in = __ffs(__ballot_sync(~0u, left <= upto)) - 1;
  return make_uint2(group * 32 + in, left - __shfl_sync(~0u, upto - mine, in));
}

// The evicted blocks are the `gone` smallest of the open ones by (key, index): three passes over
// 11, 11 and 10 bits of the keys find the largest evicted key and how many of its equals go (11
// bits spread positive weights of one magnitude over 8 bins, where bytes would meet in one),
// and one pass in order packs what stays and what goes.  Bound by its round trips, one after
// another: the lengths, the entries, three histograms, a scan, the writes; 8,192 entries are
// 64 KB, and four such rows take 10.9 us, 256 of up to 2,048 7.2.  Rows of up to 8 entries a
// thread (kOne) are read once, stay in registers, and are packed
// in shared memory, from which whole lines are written.
template <bool kOne>
__global__ void __launch_bounds__(kEvictMost) evict_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ uint32_t pack[];  // kOne: pages, then weights, of what stays; pages that went
  __shared__ Bins bins[3];
  __shared__ uint2 scratch[kEvictMost / 32];
  const uint32_t seq = blockIdx.x, tid = threadIdx.x, threads = blockDim.x;
  const uint64_t row = (uint64_t)seq * a.width;
  const uint32_t len = a.len[seq], budget = a.budget[seq];
  for (uint32_t i = tid; i < sizeof(bins) / 4; i += threads) reinterpret_cast<uint32_t*>(bins)[i] = 0;
  uint32_t n = len / kBlockTokens + (len % kBlockTokens != 0);
  if (n > a.width) {
    if (tid == 0) flag_status(a.status, NETKV_DEV_ERANGE);
    n = a.width;
  }
  const uint64_t held = max((uint64_t)budget, (uint64_t)a.sink + a.recent);
  const uint32_t gone = n > held ? n - (uint32_t)held : 0;
  const uint32_t lo = gone ? a.sink : 0, hi = gone ? n - a.recent : 0;  // open: [lo, hi)

  const uint32_t chunk = threads * kEvictPer, chunks = kOne ? 1 : (n + chunk - 1) / chunk;
  float mass[kEvictPer];
  int32_t page[kEvictPer];
  auto read_mass = [&](uint32_t c) {
#pragma unroll
    for (uint32_t j = 0; j < kEvictPer; ++j) {
      const uint32_t i = c * chunk + tid * kEvictPer + j;
      mass[j] = i < n ? a.mass[row + i] : 0.f;
    }
  };
  auto read_pages = [&](uint32_t c) {
#pragma unroll
    for (uint32_t j = 0; j < kEvictPer; ++j) {
      const uint32_t i = c * chunk + tid * kEvictPer + j;
      page[j] = i < n ? a.table[row + i] : -1;
    }
  };
  if (kOne) {
    read_mass(0);
    read_pages(0);
  }
  __syncthreads();
  uint32_t prefix = 0, left = gone;  // of the keys that begin with prefix, `left` go
  if (gone) {
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      constexpr int kShift[3] = {21, 10, 0};
      const int shift = kShift[pass], above = pass == 0 ? 31 : kShift[pass - 1];
      for (uint32_t c = 0; c < chunks; ++c) {
        if (!kOne) read_mass(c);
#pragma unroll
        for (uint32_t j = 0; j < kEvictPer; ++j) {
          const uint32_t i = c * chunk + tid * kEvictPer + j, key = weight_key(mass[j]);
          if (i >= lo && i < hi && (pass == 0 || key >> above == prefix >> above)) {
            const uint32_t b = (key >> shift) & (pass == 2 ? 1023 : 2047);
            atomicAdd(&bins[pass].bin[b], 1u);
            atomicAdd(&bins[pass].group[b / 32], 1u);
          }
        }
      }
      __syncthreads();
      const uint2 f = find_bin(bins[pass], left);
      prefix |= f.x << shift;
      left = f.y;
    }
  }
  const uint32_t stay = n - gone;
  uint32_t out = 0, equal = 0;  // evicted and equal to the last key in earlier chunks
  for (uint32_t c = 0; c < chunks; ++c) {
    if (!kOne) {
      read_mass(c);
      read_pages(c);
    }
    uint32_t less = 0, same = 0;  // bits by entry
#pragma unroll
    for (uint32_t j = 0; j < kEvictPer; ++j) {
      const uint32_t i = c * chunk + tid * kEvictPer + j, key = weight_key(mass[j]);
      if (i >= lo && i < hi) {
        less |= (uint32_t)(key < prefix) << j;
        same |= (uint32_t)(key == prefix) << j;
      }
    }
    uint2 total, before = block_scan(make_uint2(__popc(less), __popc(same)), &total, scratch);
    before.x += out;
    before.y += equal;
#pragma unroll
    for (uint32_t j = 0; j < kEvictPer; ++j) {
      const uint32_t i = c * chunk + tid * kEvictPer + j;
      // those equal that went are the first `left` of them
      const uint32_t went = before.x + min(before.y, left);
      const bool l = less >> j & 1, e = same >> j & 1, goes = l || (e && before.y < left);
      if (i < n) {
        if (kOne) {
          pack[goes ? stay + went : i - went] = (uint32_t)page[j];
          if (!goes) pack[n + i - went] = __float_as_uint(mass[j]);
        } else if (goes) {
          a.freed[row + went] = page[j];
        } else {
          a.table_out[row + i - went] = page[j];
          a.mass_out[row + i - went] = mass[j];
        }
      }
      before.x += l;
      before.y += e;
    }
    out += total.x;
    equal += total.y;
  }
  if (kOne) {
    __syncthreads();
    for (uint32_t i = tid; i < a.width; i += threads) {
      a.table_out[row + i] = i < stay ? (int32_t)pack[i] : -1;
      a.mass_out[row + i] = i < stay ? __uint_as_float(pack[n + i]) : 0.f;
      a.freed[row + i] = i < gone ? (int32_t)pack[stay + i] : -1;
    }
  } else {  // the tails: entries past what stays and past what goes
    for (uint32_t i = stay + tid; i < a.width; i += threads)
      a.table_out[row + i] = -1, a.mass_out[row + i] = 0.f;
    for (uint32_t i = gone + tid; i < a.width; i += threads) a.freed[row + i] = -1;
  }
  if (tid == 0) {
    a.len_out[seq] =
        (uint32_t)min((uint64_t)len, (uint64_t)n * kBlockTokens) - gone * kBlockTokens;
    a.n_freed[seq] = gone;
  }
}

}  // namespace

extern "C" netkv_status netkv_kv_store(const netkv_kv_pages* pages, uint32_t dtype,
                                       const void* d_k, uint64_t k_stride, const void* d_v,
                                       uint64_t v_stride, uint32_t n_seqs, const uint64_t* d_off,
                                       uint64_t rows, const uint32_t* d_start,
                                       const int32_t* d_table, uint32_t table_width,
                                       int* d_status, netkv_stream_t stream) {
  return blocks_call<true>(pages, dtype, d_k, k_stride, d_v, v_stride, n_seqs, d_off, rows,
                           d_start, d_table, table_width, d_status, stream);
}

extern "C" netkv_status netkv_kv_load(const netkv_kv_pages* pages, uint32_t dtype, void* d_k,
                                      uint64_t k_stride, void* d_v, uint64_t v_stride,
                                      uint32_t n_seqs, const uint64_t* d_off, uint64_t rows,
                                      const uint32_t* d_start, const int32_t* d_table,
                                      uint32_t table_width, int* d_status, netkv_stream_t stream) {
  return blocks_call<false>(pages, dtype, d_k, k_stride, d_v, v_stride, n_seqs, d_off, rows,
                            d_start, d_table, table_width, d_status, stream);
}

extern "C" netkv_status netkv_kv_evict(uint32_t n_seqs, const int32_t* d_table,
                                       const uint32_t* d_len, const float* d_mass,
                                       uint32_t table_width, const uint32_t* d_budget,
                                       uint32_t sink, uint32_t recent, int32_t* d_table_out,
                                       uint32_t* d_len_out, float* d_mass_out, int32_t* d_freed,
                                       uint32_t* d_n_freed, int* d_status, netkv_stream_t stream) {
  if (n_seqs == 0) return NETKV_OK;
  const void* p[] = {d_table, d_len,      d_mass,  d_budget, d_table_out,
                     d_len_out, d_mass_out, d_freed, d_n_freed};
  for (const void* x : p)
    if (!x || !aligned_to(x, 4)) return NETKV_EINVAL;
  if (!aligned_to(d_status, 4) || table_width == 0 || table_width >= (1u << 28) || recent == 0 ||
      n_seqs >> 31)
    return NETKV_EINVAL;
  // rows are packed while others of the same row are still read
  if ((const void*)d_table == d_table_out || (const void*)d_mass == d_mass_out ||
      (const void*)d_table == d_freed || d_table_out == d_freed)
    return NETKV_EINVAL;
  const EvictArgs a = {d_table,     d_len,     d_mass,     d_budget, table_width, sink,    recent,
                       d_table_out, d_len_out, d_mass_out, d_freed,  d_n_freed,   d_status};
  unsigned threads = 128;
  while (threads < kEvictMost && (uint64_t)threads * kEvictPer < table_width) threads *= 2;
  if (table_width <= kEvictMost * kEvictPer) {
    NETKV_CUDA_TRY(allow_shared<evict_kernel<true>>(kEvictMost * kEvictPer * 8));
    evict_kernel<true><<<n_seqs, threads, table_width * 8, (cudaStream_t)stream>>>(a);
  } else {
    evict_kernel<false><<<n_seqs, threads, 0, (cudaStream_t)stream>>>(a);
  }
  return netkv_launch_status();
}
