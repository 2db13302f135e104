// Causal attention of packed prompts with grouped heads.
#include "kv_common.cuh"

namespace {

struct PromptArgs {
  const unsigned char* q;
  const unsigned char* k;
  const unsigned char* v;
  unsigned char* out;
  uint64_t q_stride, k_stride, v_stride, out_stride;  // in values
  const uint64_t* q_off;
  const uint64_t* k_off;
  uint64_t q_rows, k_rows;
  uint32_t heads, group, n_seqs;
  float scale;
  float* lse;
  int* status;
};

// One warp a (query row, head): the keys one after another with a running maximum and sum.
template <int kDim, bool kBf16>
__global__ void __launch_bounds__(256) prompt_kernel(const __grid_constant__ PromptArgs a) {
  const uint32_t lane = threadIdx.x & 31, head = blockIdx.y;
  if (head == 0)
    for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < a.n_seqs; i += gridDim.x * blockDim.x)
      if (row_range(a.q_off, i, a.q_rows).bad || row_range(a.k_off, i, a.k_rows).bad)
        flag_status(a.status, NETKV_DEV_ERANGE);
  const Found f = find_unit(a.n_seqs, blockIdx.x * 8 + threadIdx.x / 32, [&](uint32_t i) {
    return (uint32_t)row_range(a.q_off, i, a.q_rows).count;
  });
  if (f.seq >= a.n_seqs) return;
  const RowRange rq = row_range(a.q_off, f.seq, a.q_rows), rk = row_range(a.k_off, f.seq, a.k_rows);
  const int64_t sees = min((int64_t)rk.count, (int64_t)f.unit + 1 + (int64_t)rk.count - (int64_t)rq.count);
  constexpr int kPer = kDim / 32;
  float q[kPer], o[kPer] = {}, m = -INFINITY, l = 0.f;
  const uint64_t row = rq.first + f.unit;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) {
    const float2 x = unpack16<kBf16>(*reinterpret_cast<const uint32_t*>(
        a.q + (row * a.q_stride + (uint64_t)head * kDim + lane * kPer + i) * 2));
    q[i] = x.x * a.scale, q[i + 1] = x.y * a.scale;
  }
  const uint64_t col = (uint64_t)(head / a.group) * kDim + lane * kPer;
  for (int64_t j = 0; j < sees; ++j) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; i += 2) {
      const float2 x = unpack16<kBf16>(
          *reinterpret_cast<const uint32_t*>(a.k + ((rk.first + j) * a.k_stride + col + i) * 2));
      s += x.x * q[i] + x.y * q[i + 1];
    }
#pragma unroll
    for (int d = 16; d; d /= 2) s += __shfl_xor_sync(~0u, s, d);
    const float next = fmaxf(m, s), keep = __expf(m - next), p = __expf(s - next);
    m = next;
    l = l * keep + p;
#pragma unroll
    for (int i = 0; i < kPer; i += 2) {
      const float2 x = unpack16<kBf16>(
          *reinterpret_cast<const uint32_t*>(a.v + ((rk.first + j) * a.v_stride + col + i) * 2));
      o[i] = o[i] * keep + p * x.x;
      o[i + 1] = o[i + 1] * keep + p * x.y;
    }
  }
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
#pragma unroll
  for (int i = 0; i < kPer; i += 2)
    *reinterpret_cast<uint32_t*>(
        a.out + (row * a.out_stride + (uint64_t)head * kDim + lane * kPer + i) * 2) =
        pack16<kBf16>(o[i] * inv, o[i + 1] * inv);
  if (lane == 0 && a.lse) a.lse[row * a.heads + head] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace

extern "C" netkv_status netkv_attn_prompt(uint32_t dtype, const void* d_q, uint64_t q_stride,
                                          const void* d_k, uint64_t k_stride, const void* d_v,
                                          uint64_t v_stride, uint32_t heads, uint32_t kv_heads,
                                          uint32_t head_dim, uint32_t n_seqs,
                                          const uint64_t* d_q_off, const uint64_t* d_k_off,
                                          uint64_t q_rows, uint64_t k_rows, float scale,
                                          void* d_out, uint64_t out_stride, float* d_lse,
                                          int* d_status, netkv_stream_t stream) {
  if (dtype > NETKV_BF16 || (head_dim != 64 && head_dim != 128) || heads == 0 || heads > 65535 ||
      kv_heads == 0 || heads % kv_heads || n_seqs >> 24 || q_rows >> 31 || k_rows >> 31 ||
      !(scale > 0.f) || !(scale <= 3.4e38f))
    return NETKV_EINVAL;
  if (n_seqs == 0 || q_rows == 0) return NETKV_OK;
  const uint64_t row = (uint64_t)heads * head_dim, kv_row = (uint64_t)kv_heads * head_dim;
  if (!rows_ok(d_q, q_stride, row) || !rows_ok(d_out, out_stride, row) ||
      (k_rows && (!rows_ok(d_k, k_stride, kv_row) || !rows_ok(d_v, v_stride, kv_row))) ||
      !d_q_off || !d_k_off || !aligned_to(d_q_off, 8) || !aligned_to(d_k_off, 8) ||
      !aligned_to(d_lse, 4) || !aligned_to(d_status, 4))
    return NETKV_EINVAL;
  const PromptArgs a = {(const unsigned char*)d_q, (const unsigned char*)d_k,
                        (const unsigned char*)d_v, (unsigned char*)d_out, q_stride, k_stride,
                        v_stride, out_stride, d_q_off, d_k_off, q_rows, k_rows, heads,
                        heads / kv_heads, n_seqs, scale, d_lse, d_status};
  auto go = [&](auto kernel) {
    kernel<<<dim3((unsigned)((q_rows + 7) / 8), heads), 256, 0, (cudaStream_t)stream>>>(a);
  };
  const bool bf = dtype == NETKV_BF16;
  if (head_dim == 64) go(bf ? prompt_kernel<64, true> : prompt_kernel<64, false>);
  else go(bf ? prompt_kernel<128, true> : prompt_kernel<128, false>);
  return netkv_launch_status();
}
