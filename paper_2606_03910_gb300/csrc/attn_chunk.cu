// Causal attention of each sequence's new tokens over its 8-bit KV blocks, in its simplest kernel: a
// warp has a row and head, and goes through the tokens that the row sees one by one.
#include "kv_common.cuh"

namespace {

constexpr uint32_t kWarps = 8, kParts = 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct ChunkArgs {
  KvArgs kv;
  const unsigned char* q;
  unsigned char* out;
  uint64_t q_stride, out_stride, rows;
  const uint64_t* off;
  const uint32_t* len;
  const int32_t* table;
  uint32_t heads, group, n_seqs, width;
  float scale;
  float* lse;
  int* status;
};

template <int kDim, bool kBf16, bool kE4m3>
__global__ void __launch_bounds__(kWarps * 32) chunk_kernel(const __grid_constant__ ChunkArgs a) {
  constexpr int kPer = kDim / 32;  // values of a lane
  const uint32_t lane = threadIdx.x & 31;
  for (uint32_t seq = blockIdx.x; seq < a.n_seqs; seq += gridDim.x) {
    const RowRange r = row_range(a.off, seq, a.rows);
    const uint64_t most = (uint64_t)a.width * kBlockTokens;
    const uint64_t tokens = min((uint64_t)a.len[seq], most);
    if (threadIdx.x == 0 && blockIdx.y == 0 && (r.bad || a.len[seq] > most))
      flag_status(a.status, NETKV_DEV_ERANGE);
    for (uint64_t u = blockIdx.y * kWarps + threadIdx.x / 32; u < r.count * a.heads;
         u += gridDim.y * kWarps) {
      const uint64_t row = u / a.heads;
      const uint32_t head = (uint32_t)(u % a.heads), kv_head = head / a.group;
      const int64_t sees = min((int64_t)tokens, (int64_t)(row + 1 + tokens) - (int64_t)r.count);
      float q[kPer], o[kPer] = {}, m = -INFINITY, l = 0.f;
      const uint16_t* from = reinterpret_cast<const uint16_t*>(a.q) +
                             (r.first + row) * a.q_stride + (uint64_t)head * kDim + lane * kPer;
      for (int i = 0; i < kPer; ++i) q[i] = unpack16<kBf16>(from[i]).x;
      for (int64_t t = 0; t < sees; ++t) {
        const int32_t page = a.table[(uint64_t)seq * a.width + t / kBlockTokens];
        if (page < 0 || (uint32_t)page >= a.kv.n_pages) {
          flag_status(a.status, NETKV_DEV_ERANGE);
          continue;
        }
        const uint64_t part = (uint64_t)page * a.kv.heads + kv_head;
        const uint64_t at = (part * kBlockTokens + t % kBlockTokens) * kDim + lane * kPer;
        float k[4], v[4], s = 0.f;
        const uint32_t wk = kPer == 4 ? *reinterpret_cast<const uint32_t*>(a.kv.k + at)
                                      : *reinterpret_cast<const uint16_t*>(a.kv.k + at);
        const uint32_t wv = kPer == 4 ? *reinterpret_cast<const uint32_t*>(a.kv.v + at)
                                      : *reinterpret_cast<const uint16_t*>(a.kv.v + at);
        decode4<kE4m3>(wk, a.kv.k_scale[part], k);
        decode4<kE4m3>(wv, a.kv.v_scale[part], v);
        for (int i = 0; i < kPer; ++i) s += q[i] * k[i];
        for (int d = 16; d; d /= 2) s += __shfl_xor_sync(~0u, s, d);
        s *= a.scale;
        const float top = fmaxf(m, s), to = m == -INFINITY ? 0.f : exp2f((m - top) * kLog2e);
        const float p = exp2f((s - top) * kLog2e);
        l = l * to + p;
        for (int i = 0; i < kPer; ++i) o[i] = o[i] * to + p * v[i];
        m = top;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      uint16_t* to = reinterpret_cast<uint16_t*>(a.out) + (r.first + row) * a.out_stride +
                     (uint64_t)head * kDim + lane * kPer;
      for (int i = 0; i < kPer; ++i) to[i] = (uint16_t)pack16<kBf16>(o[i] * inv, 0.f);
      if (a.lse && lane == 0)
        a.lse[(r.first + row) * a.heads + head] = l == 0.f ? -INFINITY : m + log2f(l) * kLn2;
    }
  }
}

bool sizes_ok(const netkv_kv_pages* pages, uint64_t rows, uint32_t n_seqs, uint32_t heads) {
  return kv_pages_ok(pages) && heads >= 1 && heads <= 65535 && heads % pages->kv_heads == 0 &&
         !(n_seqs >> 24) && !(rows >> 31);
}

}  // namespace

extern "C" size_t netkv_attn_chunk_workspace_size(const netkv_kv_pages* pages, uint64_t rows,
                                                  uint32_t n_seqs, uint32_t heads) {
  return sizes_ok(pages, rows, n_seqs, heads) ? 128 : 0;
}

extern "C" netkv_status netkv_attn_chunk(const netkv_kv_pages* pages, uint32_t dtype,
                                         const void* d_q, uint64_t q_stride, uint32_t heads,
                                         uint32_t n_seqs, const uint64_t* d_off, uint64_t rows,
                                         const uint32_t* d_len, const int32_t* d_table,
                                         uint32_t table_width, float scale, void* d_out,
                                         uint64_t out_stride, float* d_lse, void* d_ws,
                                         size_t ws_bytes, int* d_status, netkv_stream_t stream) {
  if (!sizes_ok(pages, rows, n_seqs, heads) || dtype > NETKV_BF16 || table_width == 0 ||
      table_width >= (1u << 28) || !(scale > 0.f) || !(scale <= 3.4e38f))
    return NETKV_EINVAL;
  if (n_seqs == 0 || rows == 0) return NETKV_OK;
  const uint64_t row = (uint64_t)heads * pages->head_dim;
  if (!rows_ok(d_q, q_stride, row) || !rows_ok(d_out, out_stride, row) || !d_off || !d_len ||
      !d_table || !d_ws || !aligned_to(d_off, 8) || !aligned_to(d_len, 4) ||
      !aligned_to(d_table, 4) || !aligned_to(d_lse, 4) || !aligned_to(d_ws, 16) ||
      !aligned_to(d_status, 4) ||
      ws_bytes < netkv_attn_chunk_workspace_size(pages, rows, n_seqs, heads))
    return NETKV_EINVAL;
  const ChunkArgs a = {kv_args(pages), (const unsigned char*)d_q, (unsigned char*)d_out, q_stride,
                       out_stride, rows, d_off, d_len, d_table, heads, heads / pages->kv_heads,
                       n_seqs, table_width, scale, d_lse, d_status};
  const dim3 grid(min(n_seqs, 1u << 20), kParts);
  const bool bf = dtype == NETKV_BF16, e4 = pages->format == NETKV_KV_E4M3;
  auto go = [&](auto kernel) { kernel<<<grid, kWarps * 32, 0, (cudaStream_t)stream>>>(a); };
  auto types = [&](auto dim) {
    constexpr int kDim = decltype(dim)::value;
    if (bf && e4) go(chunk_kernel<kDim, true, true>);
    else if (bf) go(chunk_kernel<kDim, true, false>);
    else if (e4) go(chunk_kernel<kDim, false, true>);
    else go(chunk_kernel<kDim, false, false>);
  };
  if (pages->head_dim == 64) types(std::integral_constant<int, 64>());
  else types(std::integral_constant<int, 128>());
  return netkv_launch_status();
}
