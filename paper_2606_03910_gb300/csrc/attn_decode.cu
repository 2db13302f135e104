// Attention of one query row a sequence over its 8-bit KV blocks, and the weight that each
// block has drawn.
#include "kv_common.cuh"

namespace {

struct DecodeArgs {
  KvArgs kv;
  const unsigned char* q;
  unsigned char* out;
  uint64_t q_stride, out_stride;
  uint32_t heads, n_seqs, width;
  const uint32_t* len;
  const int32_t* table;
  float scale;
  float* lse;
  const float* mass_in;
  float* mass_out;
  float* ws_lse;  // [n_seqs][heads]
  int* status;
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int d = 16; d; d /= 2) x += __shfl_xor_sync(~0u, x, d);
  return x;
}

__device__ __forceinline__ uint32_t tokens_of(const DecodeArgs& a, uint32_t seq) {
  return (uint32_t)min((uint64_t)a.len[seq], (uint64_t)a.width * kBlockTokens);
}

// scale * q . k of one token, a lane's kDim / 32 values at a time; every lane gets the sum.
template <int kDim, bool kE4m3>
__device__ __forceinline__ float score(const DecodeArgs& a, const float* q, uint64_t part,
                                       uint32_t row) {
  const uint32_t lane = threadIdx.x & 31;
  const unsigned char* k = a.kv.k + (part * kBlockTokens + row) * kDim + lane * (kDim / 32);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kDim / 32; i += 2) {
    const float2 x = decode2<kE4m3>(*reinterpret_cast<const uint16_t*>(k + i));
    s += x.x * q[i] + x.y * q[i + 1];
  }
  return warp_sum(s) * a.kv.k_scale[part] * a.scale;
}

// One warp a (sequence, head): its tokens one after another with a running maximum and sum.
template <int kDim, bool kBf16, bool kE4m3>
__global__ void __launch_bounds__(32) decode_kernel(const __grid_constant__ DecodeArgs a) {
  const uint32_t seq = blockIdx.x, head = blockIdx.y, lane = threadIdx.x;
  const uint32_t kv_head = head / (a.heads / a.kv.heads), n = tokens_of(a, seq);
  if (lane == 0 && n != a.len[seq]) flag_status(a.status, NETKV_DEV_ERANGE);
  constexpr int kPer = kDim / 32;
  float q[kPer], o[kPer] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) {
    const float2 x = unpack16<kBf16>(*reinterpret_cast<const uint32_t*>(
        a.q + (seq * a.q_stride + (uint64_t)head * kDim + lane * kPer + i) * 2));
    q[i] = x.x, q[i + 1] = x.y;
  }
  for (uint32_t t = 0; t < n; ++t) {
    const int32_t page = a.table[(uint64_t)seq * a.width + t / kBlockTokens];
    if (page < 0 || (uint32_t)page >= a.kv.n_pages) {
      if (lane == 0) flag_status(a.status, NETKV_DEV_ERANGE);
      continue;
    }
    const uint64_t part = (uint64_t)page * a.kv.heads + kv_head;
    const uint32_t row = t % kBlockTokens;
    const float s = score<kDim, kE4m3>(a, q, part, row);
    const float next = fmaxf(m, s), keep = __expf(m - next), p = __expf(s - next);
    m = next;
    l = l * keep + p;
    const unsigned char* v = a.kv.v + (part * kBlockTokens + row) * kDim + lane * kPer;
    const float w = p * a.kv.v_scale[part];
#pragma unroll
    for (int i = 0; i < kPer; i += 2) {
      const float2 x = decode2<kE4m3>(*reinterpret_cast<const uint16_t*>(v + i));
      o[i] = o[i] * keep + w * x.x;
      o[i + 1] = o[i + 1] * keep + w * x.y;
    }
  }
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
#pragma unroll
  for (int i = 0; i < kPer; i += 2)
    *reinterpret_cast<uint32_t*>(
        a.out + (seq * a.out_stride + (uint64_t)head * kDim + lane * kPer + i) * 2) =
        pack16<kBf16>(o[i] * inv, o[i + 1] * inv);
  if (lane == 0) {
    const float lse = l == 0.f ? -INFINITY : m + logf(l);
    if (a.lse) a.lse[(uint64_t)seq * a.heads + head] = lse;
    if (a.mass_out) a.ws_lse[(uint64_t)seq * a.heads + head] = lse;
  }
}

// One warp a block: the weights of its tokens over all heads, from the heads' lse.
template <int kDim, bool kBf16, bool kE4m3>
__global__ void __launch_bounds__(32) mass_kernel(const __grid_constant__ DecodeArgs a) {
  const uint32_t seq = blockIdx.y, block = blockIdx.x, lane = threadIdx.x;
  const uint32_t n = tokens_of(a, seq);
  if ((uint64_t)block * kBlockTokens >= n) return;
  const uint64_t at = (uint64_t)seq * a.width + block;
  const int32_t page = a.table[at];
  float sum = 0.f;
  constexpr int kPer = kDim / 32;
  if (page >= 0 && (uint32_t)page < a.kv.n_pages)
    for (uint32_t head = 0; head < a.heads; ++head) {
      float q[kPer];
#pragma unroll
      for (int i = 0; i < kPer; i += 2) {
        const float2 x = unpack16<kBf16>(*reinterpret_cast<const uint32_t*>(
            a.q + (seq * a.q_stride + (uint64_t)head * kDim + lane * kPer + i) * 2));
        q[i] = x.x, q[i + 1] = x.y;
      }
      const float lse = a.ws_lse[(uint64_t)seq * a.heads + head];
      const uint64_t part = (uint64_t)page * a.kv.heads + head / (a.heads / a.kv.heads);
      for (uint32_t row = 0; row < kBlockTokens && block * kBlockTokens + row < n; ++row)
        sum += __expf(score<kDim, kE4m3>(a, q, part, row) - lse);
    }
  if (lane == 0) a.mass_out[at] = (a.mass_in ? a.mass_in[at] : 0.f) + sum;
}

bool sizes_ok(const netkv_kv_pages* pages, uint32_t n_seqs, uint32_t heads, uint32_t width) {
  return kv_pages_ok(pages) && heads >= 1 && heads <= 65535 && heads % pages->kv_heads == 0 &&
         !(n_seqs >> 24) && width >= 1 && width < (1u << 28);
}

}  // namespace

extern "C" size_t netkv_attn_decode_workspace_size(const netkv_kv_pages* pages, uint32_t n_seqs,
                                                   uint32_t heads, uint32_t table_width,
                                                   int with_mass) {
  if (!sizes_ok(pages, n_seqs, heads, table_width)) return 0;
  return ((size_t)n_seqs * heads * 4 + 15) / 16 * 16 + 16;
}

extern "C" netkv_status netkv_attn_decode(const netkv_kv_pages* pages, uint32_t dtype,
                                          const void* d_q, uint64_t q_stride, uint32_t heads,
                                          uint32_t n_seqs, const uint32_t* d_len,
                                          const int32_t* d_table, uint32_t table_width,
                                          float scale, void* d_out, uint64_t out_stride,
                                          float* d_lse, const float* d_mass_in, float* d_mass_out,
                                          void* d_ws, size_t ws_bytes, int* d_status,
                                          netkv_stream_t stream) {
  if (!sizes_ok(pages, n_seqs, heads, table_width) || dtype > NETKV_BF16) return NETKV_EINVAL;
  if (n_seqs == 0) return NETKV_OK;
  const uint64_t row = (uint64_t)heads * pages->head_dim;
  if (!rows_ok(d_q, q_stride, row) || !rows_ok(d_out, out_stride, row) || !d_len || !d_table ||
      !d_ws || !aligned_to(d_len, 4) || !aligned_to(d_table, 4) || !aligned_to(d_lse, 4) ||
      !aligned_to(d_mass_in, 4) || !aligned_to(d_mass_out, 4) || !aligned_to(d_ws, 16) ||
      !aligned_to(d_status, 4) || (d_mass_in && !d_mass_out) || !(scale > 0.f) ||
      !(scale <= 3.4e38f) ||
      ws_bytes < netkv_attn_decode_workspace_size(pages, n_seqs, heads, table_width,
                                                  d_mass_out != nullptr))
    return NETKV_EINVAL;
  const DecodeArgs a = {kv_args(pages), (const unsigned char*)d_q, (unsigned char*)d_out, q_stride,
                        out_stride, heads, n_seqs, table_width, d_len, d_table, scale, d_lse,
                        d_mass_in, d_mass_out, (float*)d_ws, d_status};
  auto go = [&](auto dim, auto bf, auto e4) {
    constexpr int kDim = decltype(dim)::value;
    constexpr bool kB = decltype(bf)::value, kE = decltype(e4)::value;
    decode_kernel<kDim, kB, kE><<<dim3(n_seqs, heads), 32, 0, (cudaStream_t)stream>>>(a);
    if (d_mass_out)
      mass_kernel<kDim, kB, kE><<<dim3(table_width, n_seqs), 32, 0, (cudaStream_t)stream>>>(a);
  };
  auto types = [&](auto dim) {
    const bool bf = dtype == NETKV_BF16, e4 = pages->format == NETKV_KV_E4M3;
    if (bf && e4) go(dim, std::true_type(), std::true_type());
    else if (bf) go(dim, std::true_type(), std::false_type());
    else if (e4) go(dim, std::false_type(), std::true_type());
    else go(dim, std::false_type(), std::false_type());
  };
  if (pages->head_dim == 64) types(std::integral_constant<int, 64>());
  else types(std::integral_constant<int, 128>());
  return netkv_launch_status();
}
