// Attention of one query row a sequence over its 8-bit KV blocks, and the weight that each
// block has drawn.
//
// Bound: the codes are read once, 2 kDim bytes a token and KV head, and everything else is
// small, so the kernel streams pages and its arithmetic has to fit in their shadow.
//
// Split: the work is the list of all pages, (sequence, KV head, block) in order, and every block
// of the grid takes an equal run of it, so ragged batches and single long sequences spread over
// the card alike.  A run holds whole (sequence, head) segments, which are finished at once, and
// at most two that other blocks share, whose sums go to the workspace for the join.  Within a
// segment the four warps take every fourth page; each has a ring of pages in flight, filled by
// bulk copies (a page's part for a head is 16 kDim contiguous bytes) and refilled for the next
// segment before the present one is summed up.
//
// Arithmetic: a page is 16 tokens and a KV head serves a group of query heads, so S^T = K q^T
// and O^T = V^T P^T are products of 16 x 16 by 16 x 8: m16n8k16, with up to 8 (kTiles = 1) or
// 16 heads (2) side by side.  A tcgen05 product would be 128 rows high, of which the group
// fills 8.  Both code types are exact in fp16, so codes go into the products as they are and
// the scales are applied to scores and weights in fp32.  A row of queries is brought to [1, 2)
// by a power of two, which loses nothing of bf16's 8 bits.  The order of the inner dimension is
// free in a product: a thread's operands are the bytes that lie together, 16 at a load.
#include "kv_common.cuh"

namespace {

constexpr uint32_t kWarps = 4;
// Blocks of the grid: three an SM on 152 SMs, two where the sums of two tiles leave no room for
// a third; and pages in flight a warp, 12 KB or 16 KB of them.
template <int kTiles>
constexpr uint32_t kCtas = kTiles == 1 ? 456 : 304;
constexpr uint32_t kMostCtas = 456;
template <int kDim, int kTiles>
constexpr uint32_t kStages = (kTiles == 1 ? 3 : 4) * (128 / kDim);
constexpr uint32_t kMinPages = 8;   // a block's run at least: two pages a warp
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The running maximum follows the scores once one is above it by this (in powers of two):
// weights up to 2^8 are as exact in fp16 as those up to 1, and sums are fp32.
constexpr float kLag = 8.f;

struct DecodeArgs {
  KvArgs kv;
  const unsigned char* q;
  unsigned char* out;
  uint64_t q_stride, out_stride;
  uint32_t heads, group, chunks, n_seqs, width;  // chunks of kTiles * 8 heads of a group
  const uint32_t* len;
  const int32_t* table;
  float scale2;  // scale * log2(e)
  float* lse;
  const float* mass_in;
  float* mass_out;
  float* part_o;    // [ctas][2][kTiles * 8][kDim]
  float* part_ml;   // [ctas][2][kTiles * 8][2]
  float* lse2;      // [n_seqs][heads], in powers of two; with mass only
  float* block2;    // [n_seqs][width][heads]: log2 of a block's weight; with mass only
  uint32_t ctas;
  int* status;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A kernel that follows another of the same call starts while that one ends: what it reads of
// the call's own it reads after follow().
__device__ __forceinline__ void follow() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_follow() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ uint32_t pages_of(const DecodeArgs& a, uint32_t seq) {
  const uint32_t n = a.len[seq];
  return min(n / kBlockTokens + (n % kBlockTokens != 0), a.width);
}
__device__ __forceinline__ uint32_t tokens_of(const DecodeArgs& a, uint32_t seq) {
  return (uint32_t)min((uint64_t)a.len[seq], (uint64_t)a.width * kBlockTokens);
}

// The runs: `total` pages over `ctas` blocks.
struct Runs {
  uint64_t total;
  uint32_t ctas;
  __device__ __forceinline__ uint64_t start(uint32_t c) const { return total * c / ctas; }
};

__device__ __forceinline__ Runs runs_of(const DecodeArgs& a, uint32_t units) {
  const uint32_t lane = threadIdx.x & 31;
  uint64_t sum = 0;
  for (uint32_t i = lane; i < a.n_seqs; i += 32) sum += pages_of(a, i);
#pragma unroll
  for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
  Runs r;
  r.total = sum * units;
  r.ctas = (uint32_t)min((uint64_t)a.ctas, max((uint64_t)1, r.total / kMinPages));
  return r;
}

// A segment: pages [first, first + count) of one (sequence, unit); a unit is a KV head and a
// chunk of its query heads.
struct Segment {
  uint32_t seq, unit, first, count, pages;
};

__device__ __forceinline__ Segment segment_at(const DecodeArgs& a, uint32_t units, uint64_t item) {
  const uint32_t lane = threadIdx.x & 31;
  for (uint32_t base = 0; base < a.n_seqs; base += 32) {
    const uint32_t i = base + lane, n = i < a.n_seqs ? pages_of(a, i) : 0;
    const uint64_t mine = (uint64_t)n * units;
    uint64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint64_t x = __shfl_up_sync(~0u, upto, d);
      if (lane >= (uint32_t)d) upto += x;
    }
    const uint32_t hit = __ballot_sync(~0u, item < upto);
    if (hit) {
      const int at = __ffs(hit) - 1;
      const uint64_t rest = __shfl_sync(~0u, item - (upto - mine), at);
      const uint32_t pages = __shfl_sync(~0u, n, at);
      return {base + at, (uint32_t)(rest / pages), (uint32_t)(rest % pages), 0, pages};
    }
    item -= __shfl_sync(~0u, upto, 31);
  }
  return {a.n_seqs, 0, 0, 0, 0};
}

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}

// Waits for a phase of a barrier, a second at most (a hundredth once that has run out).
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, bool late) {
  if (try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!try_wait(bar, parity))
    if (clock64() - t0 > (late ? 20000000ll : 2000000000ll)) return false;
  return true;
}

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                    uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
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

template <int kDim, int kTiles>
struct Shared {
  static constexpr int kHeads = kTiles * 8;
  static constexpr uint32_t kRing = kStages<kDim, kTiles>;
  static constexpr int kGroupFloats = 16 * kHeads + 8;  // of 16 dims; the 8 spread the banks
  alignas(128) unsigned char ring[kWarps][kRing][2][kBlockTokens * kDim];
  float o[kWarps][kDim / 16 * kGroupFloats];
  float m[kWarps][kHeads], l[kWarps][kHeads];
  alignas(8) uint64_t full[kWarps][kRing];
};

template <int kDim, int kTiles, bool kBf16, bool kE4m3, bool kMass>
__global__ void __launch_bounds__(kWarps * 32, kTiles == 1 ? 3 : 2)
    decode_kernel(const __grid_constant__ DecodeArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  using Sh = Shared<kDim, kTiles>;
  Sh& sh = *reinterpret_cast<Sh*>(smem);
  constexpr int kHeads = kTiles * 8, kSteps = kDim / 16, kPart = kBlockTokens * kDim;
  constexpr uint32_t kRing = Sh::kRing;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32, r = lane / 4, c = lane % 4;
  const uint32_t units = a.kv.heads * a.chunks;
  let_follow();

  if (lane < kRing)
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_addr(&sh.full[warp][lane]))
                 : "memory");
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();

  // rows of sequences without tokens, and lengths past the table
  for (uint32_t i = blockIdx.x; i < a.n_seqs; i += gridDim.x) {
    const uint32_t n = a.len[i];
    if (tid == 0 && n > (uint64_t)a.width * kBlockTokens) flag_status(a.status, NETKV_DEV_ERANGE);
    if (n) continue;
    for (uint32_t x = tid; x < a.heads * kDim / 8; x += kWarps * 32)
      reinterpret_cast<uint4*>(a.out + i * a.out_stride * 2)[x] = make_uint4(0, 0, 0, 0);
    for (uint32_t h = tid; h < a.heads && a.lse; h += kWarps * 32)
      a.lse[(uint64_t)i * a.heads + h] = -INFINITY;
  }

  const Runs runs = runs_of(a, units);
  if (blockIdx.x >= runs.ctas) return;
  uint64_t left = runs.start(blockIdx.x + 1) - runs.start(blockIdx.x);
  if (left == 0) return;
  Segment next = segment_at(a, units, runs.start(blockIdx.x));
  next.count = (uint32_t)min((uint64_t)(next.pages - next.first), left);

  // A warp's pages of a segment are numbered k = 0, 1, ...: block first + warp + 4 k.  Lane j
  // keeps the page numbers of k = j, 32 + j and 64 + j past the present 32 and the scales of
  // the first two, so that neither is waited for in a long segment.
  uint32_t issued = 0, taken = 0;  // pages of all segments
  uint32_t mine = 0, kv_head = 0, head0 = 0, batch = 0;
  int32_t page0 = -1, page1 = -1, page2 = -1;
  float ks0 = 0.f, vs0 = 0.f, ks1 = 0.f, vs1 = 0.f;
  Segment seg = next;
  auto page_at = [&](uint32_t k) -> int32_t {
    if (k >= mine) return -1;
    const int32_t p = a.table[(uint64_t)seg.seq * a.width + seg.first + warp + kWarps * k];
    if (p >= 0 && (uint32_t)p < a.kv.n_pages) return p;
    flag_status(a.status, NETKV_DEV_ERANGE);
    return -1;
  };
  auto scales = [&](int32_t p, float* ks, float* vs) {
    const uint64_t at = (uint64_t)(p < 0 ? 0 : p) * a.kv.heads + kv_head;
    *ks = a.kv.k_scale[at];
    *vs = a.kv.v_scale[at];
  };
  auto issue = [&](uint32_t k) {  // the k-th page of the segment into the ring
    const int32_t p = __shfl_sync(~0u, k / 32 == batch ? page0 : page1, k % 32);
    if (lane == 0) {
      const uint32_t st = issued % kRing, bar = smem_addr(&sh.full[warp][st]);
      if (p >= 0) {
        const uint64_t at = ((uint64_t)p * a.kv.heads + kv_head) * kPart;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar),
                     "r"(2 * kPart)
                     : "memory");
        asm volatile(
            "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, "
            "[%3];" ::"r"(smem_addr(sh.ring[warp][st][0])),
            "l"(a.kv.k + at), "r"(kPart), "r"(bar)
            : "memory");
        asm volatile(
            "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, "
            "[%3];" ::"r"(smem_addr(sh.ring[warp][st][1])),
            "l"(a.kv.v + at), "r"(kPart), "r"(bar)
            : "memory");
      } else {  // an absent page keeps its place in the ring
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
      }
    }
    ++issued;
  };
  auto begin = [&](const Segment& s) {
    seg = s;
    mine = s.count > warp ? (s.count - warp + kWarps - 1) / kWarps : 0;
    kv_head = s.unit / a.chunks;
    head0 = s.unit % a.chunks * kHeads;
    batch = 0;
    page0 = page_at(lane);
    page1 = page_at(32 + lane);
    page2 = page_at(64 + lane);
    scales(page0, &ks0, &vs0);
    scales(page1, &ks1, &vs1);
    for (uint32_t k = 0; k < mine && k < kRing; ++k) issue(k);
  };

  begin(next);
  bool first_segment = true, late = false;
  while (true) {
    // ---- queries of the segment: thread (r, c) has head r of each tile, dims by 16 bytes of
    // codes: 64 h + 16 c + 4 i + 0..3 in step 4 h + i
    uint32_t q[kTiles][kSteps][2];
    float f[kTiles][2];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const uint32_t h = head0 + t * 8 + r;
      const bool real = h < a.group;
      uint4 raw[kDim / 32];
      const uint4* src = reinterpret_cast<const uint4*>(
          a.q + (seg.seq * a.q_stride + ((uint64_t)kv_head * a.group + (real ? h : 0)) * kDim) * 2);
#pragma unroll
      for (int i = 0; i < kDim / 32; ++i)
        raw[i] = real ? src[(i / 2) * 8 + c * 2 + i % 2] : make_uint4(0, 0, 0, 0);
      const uint32_t* w = reinterpret_cast<const uint32_t*>(raw);
      float largest = 0.f;
#pragma unroll
      for (int i = 0; i < kDim / 8; ++i) {
        const float2 x = unpack16<kBf16>(w[i]);
        largest = fmaxf(largest, fmaxf(fabsf(x.x), fabsf(x.y)));
      }
      largest = fmaxf(largest, __shfl_xor_sync(~0u, largest, 1));
      largest = fmaxf(largest, __shfl_xor_sync(~0u, largest, 2));
      uint32_t e = __float_as_uint(largest) >> 23;
      if (e < 2 || e > 252) e = 127;
      const float inv = __uint_as_float((254 - e) << 23);
      const float up = __uint_as_float(e << 23) * a.scale2;
      f[t][0] = __shfl_sync(~0u, up, 8 * c);
      f[t][1] = __shfl_sync(~0u, up, 8 * c + 4);
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 x = unpack16<kBf16>(w[i * 2 + j]);
          q[t][i][j] = pack16<false>(x.x * inv, x.y * inv);
        }
    }
    float o[kTiles][kDim / 16][4] = {}, m[kTiles][2], l[kTiles][2] = {};
#pragma unroll
    for (int t = 0; t < kTiles; ++t) m[t][0] = m[t][1] = -INFINITY;
    float v_unit = 0.f, v_inv = 0.f;  // a power of two that the value scales are taken by
    const uint32_t tokens = tokens_of(a, seg.seq);

    for (uint32_t k = 0; k < mine; ++k) {
      if (k / 32 != batch) {
        batch = k / 32;
        page0 = page1, page1 = page2;
        ks0 = ks1, vs0 = vs1;
        scales(page1, &ks1, &vs1);
        page2 = page_at((batch + 2) * 32 + lane);
      }
      const uint32_t st = taken % kRing, bar = smem_addr(&sh.full[warp][st]);
      if (!wait(bar, (taken / kRing) & 1, late)) late = true;
      ++taken;
      const int32_t page = __shfl_sync(~0u, page0, k % 32);
      if (page >= 0) {
        const float ks = __shfl_sync(~0u, ks0, k % 32), vs = __shfl_sync(~0u, vs0, k % 32);
        const uint32_t block = seg.first + warp + kWarps * k, t0 = block * kBlockTokens;
        const uint32_t valid = min(tokens - t0, kBlockTokens);
        const unsigned char* kp = sh.ring[warp][st][0];
        const unsigned char* vp = sh.ring[warp][st][1];

        float s[kTiles][4] = {};
#pragma unroll
        for (int h = 0; h < kDim / 64; ++h) {
          const uint4 x = *reinterpret_cast<const uint4*>(kp + r * kDim + h * 64 + c * 16);
          const uint4 y = *reinterpret_cast<const uint4*>(kp + (r + 8) * kDim + h * 64 + c * 16);
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t a0, a1, a2, a3;
            widen<kE4m3>(xs[i], &a0, &a2);
            widen<kE4m3>(ys[i], &a1, &a3);
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
              mma(s[t], a0, a1, a2, a3, q[t][h * 4 + i][0], q[t][h * 4 + i][1]);
          }
        }
        // s: tokens r and r + 8, heads 2 c and 2 c + 1 of each tile
        bool above = false;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[t][i] *= ks * f[t][i & 1];
            if (valid < kBlockTokens && r + (i / 2) * 8 >= valid) s[t][i] = -INFINITY;
            above |= s[t][i] > m[t][i & 1] + kLag;
          }
        if (__any_sync(~0u, above)) {
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            float to[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float x = fmaxf(m[t][j], fmaxf(s[t][j], s[t][j + 2]));
#pragma unroll
              for (int d = 4; d < 32; d *= 2) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
              to[j] = m[t][j] == -INFINITY ? 0.f : ex2(m[t][j] - x);
              m[t][j] = x;
              l[t][j] *= to[j];
            }
#pragma unroll
            for (int j = 0; j < kDim / 16; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[t][j][i] *= to[i & 1];
          }
        }
        if (vs > v_unit) {  // the whole warp; values of other blocks stay within fp16's range
          const uint32_t e = min(max(__float_as_uint(vs) >> 23, 2u), 252u);
          const float unit = __uint_as_float((e + 1) << 23), shrink = v_unit / unit;
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int j = 0; j < kDim / 16; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[t][j][i] *= shrink;
          v_unit = unit;
          v_inv = __uint_as_float((253 - e) << 23);
        }
        const float w = vs * v_inv;
        uint32_t p[kTiles][2];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = ex2(s[t][i] - m[t][i & 1]);
#pragma unroll
          for (int j = 0; j < 2; ++j) l[t][j] += x[j] + x[j + 2];
          if (kMass) {  // over the tokens: odd threads r take head 2 c + 1, even ones 2 c
            const float sum0 = x[0] + x[2], sum1 = x[1] + x[3];
            float sum = r & 1 ? sum1 : sum0;
            sum += __shfl_xor_sync(~0u, r & 1 ? sum0 : sum1, 4);
            sum += __shfl_xor_sync(~0u, sum, 8);
            sum += __shfl_xor_sync(~0u, sum, 16);
            const uint32_t h = head0 + t * 8 + 2 * c + r;
            if (r < 2 && h < a.group)
              a.block2[((uint64_t)seg.seq * a.width + block) * a.heads + kv_head * a.group + h] =
                  (r & 1 ? m[t][1] : m[t][0]) + lg2(sum);
          }
          p[t][0] = transpose8x8(pack16<false>(x[0] * w, x[1] * w));
          p[t][1] = transpose8x8(pack16<false>(x[2] * w, x[3] * w));
        }
        // values: tokens 2 c, 2 c + 1, 2 c + 8 and 2 c + 9, dims r * kDim / 8 on; zeros past
        // the last token, whose codes may stand for anything
        constexpr int kWords = kDim / 32;
        uint32_t v[4][kWords];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t row = 2 * c + (i & 1) + (i / 2) * 8;
          const uint32_t* src = reinterpret_cast<const uint32_t*>(vp + row * kDim + r * (kDim / 8));
          if (kWords == 4) *reinterpret_cast<uint4*>(v[i]) = *reinterpret_cast<const uint4*>(src);
          else *reinterpret_cast<uint2*>(v[i]) = *reinterpret_cast<const uint2*>(src);
          if (valid < kBlockTokens && row >= valid) {
#pragma unroll
            for (int j = 0; j < kWords; ++j) v[i][j] = 0;
          }
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {  // tile 2 i + j: dims 4 i + 2 j and the next of the run
            const uint32_t sel = j ? 0x7362 : 0x5140;
            uint32_t a0, a1, a2, a3;
            widen<kE4m3>(__byte_perm(v[0][i], v[1][i], sel), &a0, &a1);
            widen<kE4m3>(__byte_perm(v[2][i], v[3][i], sel), &a2, &a3);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) mma(o[t][2 * i + j], a0, a1, a2, a3, p[t][0], p[t][1]);
          }
      } else if (kMass && r == 0) {
        const uint32_t block = seg.first + warp + kWarps * k;
#pragma unroll
        for (int i = 0; i < kHeads / 4; ++i) {
          const uint32_t h = head0 + c + i * 4;
          if (h < a.group)
            a.block2[((uint64_t)seg.seq * a.width + block) * a.heads + kv_head * a.group + h] =
                -INFINITY;
        }
      }
      __syncwarp();
      if (k + kRing < mine) issue(k + kRing);
    }

    // ---- the warps' sums
    const Segment done = seg;
    const uint32_t done_kv = kv_head, done_head0 = head0;
    const bool whole = done.count == done.pages;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[t][j] += __shfl_xor_sync(~0u, l[t][j], d);
        if (r == 0) {
          sh.m[warp][t * 8 + 2 * c + j] = m[t][j];
          sh.l[warp][t * 8 + 2 * c + j] = l[t][j];
        }
#pragma unroll
        for (int x = 0; x < kDim / 16; ++x)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t dim = r * (kDim / 8) + 2 * x + i;
            sh.o[warp][dim / 16 * Sh::kGroupFloats + dim % 16 * kHeads + t * 8 + 2 * c + j] =
                o[t][x][2 * i + j] * v_unit;
          }
      }
    left -= done.count;
    if (left) {  // the next segment's pages are on their way while this one is summed up
      next = {done.seq, done.unit + 1, 0, 0, done.pages};
      if (next.unit == units) {
        next.unit = 0;
        do {
          ++next.seq;
          next.pages = next.seq < a.n_seqs ? pages_of(a, next.seq) : 1;
        } while (next.pages == 0);
        if (next.seq >= a.n_seqs) left = 0;  // lengths that changed under the call
      }
    }
    if (left) {
      next.count = (uint32_t)min((uint64_t)next.pages, left);
      begin(next);
    }
    __syncthreads();
    for (uint32_t x = tid; x < kHeads * kDim; x += kWarps * 32) {
      const uint32_t h = x / kDim, dim = x % kDim;
      if (done_head0 + h >= a.group) break;
      float top = sh.m[0][h];
#pragma unroll
      for (uint32_t w = 1; w < kWarps; ++w) top = fmaxf(top, sh.m[w][h]);
      float sum = 0.f, all = 0.f;
#pragma unroll
      for (uint32_t w = 0; w < kWarps; ++w) {
        const float y = sh.m[w][h] == -INFINITY ? 0.f : ex2(sh.m[w][h] - top);
        sum += y * sh.l[w][h];
        all += y * sh.o[w][dim / 16 * Sh::kGroupFloats + dim % 16 * kHeads + h];
      }
      const uint32_t head = done_kv * a.group + done_head0 + h;
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const uint32_t y = pack16<kBf16>(all * inv, 0.f);
        reinterpret_cast<uint16_t*>(a.out)[done.seq * a.out_stride + (uint64_t)head * kDim + dim] =
            (uint16_t)y;
        if (dim == 0) {
          const float z = sum == 0.f ? -INFINITY : top + log2f(sum);
          if (a.lse) a.lse[(uint64_t)done.seq * a.heads + head] = z * kLn2;
          if (kMass) a.lse2[(uint64_t)done.seq * a.heads + head] = z;
        }
      } else {
        const uint32_t slot = blockIdx.x * 2 + (first_segment ? 0 : 1);
        a.part_o[((uint64_t)slot * kHeads + h) * kDim + dim] = all;
        if (dim == 0) {
          a.part_ml[(slot * kHeads + h) * 2] = top;
          a.part_ml[(slot * kHeads + h) * 2 + 1] = sum;
        }
      }
    }
    if (!left) break;
    first_segment = false;
    __syncthreads();
  }
  if (late && lane == 0) flag_status(a.status, NETKV_DEV_ETIMEOUT);
}

// Joins the segments that runs share: one block a (boundary between runs, head of the unit),
// where the boundary is the first inside its segment.  The parts' weights first, then eight
// groups of threads (a thread has four dims) over every eighth part: a long sequence alone on
// the card has a part from each run, 456 for one unit.
constexpr uint32_t kJoin = 256;
template <int kDim, int kTiles, bool kBf16, bool kMass>
__global__ void __launch_bounds__(kJoin) join_kernel(const __grid_constant__ DecodeArgs a) {
  constexpr int kHeads = kTiles * 8, kLanes = kDim / 4, kGroups = kJoin / kLanes;
  __shared__ float weight[kCtas<kTiles>], reduce[kJoin / 32][2];
  __shared__ float4 sums[kGroups][kLanes];
  const uint32_t units = a.kv.heads * a.chunks, tid = threadIdx.x, h = blockIdx.y;
  let_follow();
  const Runs runs = runs_of(a, units);
  const uint32_t cut = blockIdx.x + 1;
  if (cut >= runs.ctas) return;
  const Segment s = segment_at(a, units, runs.start(cut));
  const uint64_t at = runs.start(cut) - s.first;  // the segment's first page
  if (s.first == 0 || (cut > 1 && runs.start(cut - 1) > at)) return;
  const uint32_t head0 = s.unit % a.chunks * kHeads;
  if (head0 + h >= a.group) return;
  const uint64_t end = at + s.pages;
  // runs that start before the end, less those before cut - 1
  const uint32_t parts =
      (uint32_t)min((uint64_t)runs.ctas, (end * runs.ctas + runs.total - 1) / runs.total) - (cut - 1);
  const uint32_t second = runs.start(cut - 1) < at;  // the segment is that run's last one
  auto slot = [&](uint32_t i) {
    return ((uint64_t)(cut - 1 + i) * 2 + (i == 0 ? second : 0)) * kHeads + h;
  };
  follow();
  float top = -INFINITY, sum = 0.f;
  for (uint32_t i = tid; i < parts; i += kJoin) top = fmaxf(top, a.part_ml[slot(i) * 2]);
#pragma unroll
  for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
  if (tid % 32 == 0) reduce[tid / 32][0] = top;
  __syncthreads();
  top = reduce[0][0];
#pragma unroll
  for (int w = 1; w < (int)kJoin / 32; ++w) top = fmaxf(top, reduce[w][0]);
  for (uint32_t i = tid; i < parts; i += kJoin) {
    const float m = a.part_ml[slot(i) * 2], l = a.part_ml[slot(i) * 2 + 1];
    const float w = m == -INFINITY ? 0.f : ex2(m - top);
    weight[i] = w;
    // a part of NaN scores has no maximum, but its sum says so
    sum += m == -INFINITY && l == l ? 0.f : w * l;
  }
#pragma unroll
  for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
  if (tid % 32 == 0) reduce[tid / 32][1] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < (int)kJoin / 32; ++w) sum += reduce[w][1];
  const uint32_t lane = tid % kLanes, group = tid / kLanes;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (uint32_t i = group; i < parts; i += kGroups) {
    const float4 x = reinterpret_cast<const float4*>(a.part_o + slot(i) * kDim)[lane];
    const float w = weight[i];
    o.x += w * x.x, o.y += w * x.y, o.z += w * x.z, o.w += w * x.w;
  }
  sums[group][lane] = o;
  __syncthreads();
  if (group) return;
#pragma unroll
  for (int g = 1; g < kGroups; ++g) {
    const float4 x = sums[g][lane];
    o.x += x.x, o.y += x.y, o.z += x.z, o.w += x.w;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const uint32_t head = s.unit / a.chunks * a.group + head0 + h;
  reinterpret_cast<uint2*>(a.out + (s.seq * a.out_stride + (uint64_t)head * kDim) * 2)[lane] =
      make_uint2(pack16<kBf16>(o.x * inv, o.y * inv), pack16<kBf16>(o.z * inv, o.w * inv));
  if (lane == 0) {
    const float z = sum == 0.f ? -INFINITY : top + log2f(sum);
    if (a.lse) a.lse[(uint64_t)s.seq * a.heads + head] = z * kLn2;
    if (kMass) a.lse2[(uint64_t)s.seq * a.heads + head] = z;
  }
}

// A block's weight over all heads, in the heads' order: one thread a block.
__global__ void __launch_bounds__(128) mass_kernel(const __grid_constant__ DecodeArgs a) {
  const uint32_t seq = blockIdx.x, pages = pages_of(a, seq);
  follow();
  for (uint32_t block = blockIdx.y * 128 + threadIdx.x; block < pages; block += gridDim.y * 128) {
    const uint64_t at = (uint64_t)seq * a.width + block;
    float sum = 0.f;
    for (uint32_t h = 0; h < a.heads; ++h) {
      const float b = a.block2[at * a.heads + h];
      if (b != -INFINITY) sum += ex2(b - a.lse2[(uint64_t)seq * a.heads + h]);
    }
    a.mass_out[at] = (a.mass_in ? a.mass_in[at] : 0.f) + sum;
  }
}

template <class Kernel>
cudaError_t launch_following(Kernel kernel, dim3 grid, unsigned threads, cudaStream_t s,
                             const DecodeArgs& a) {
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = grid;
  c.blockDim = dim3(threads);
  c.stream = s;
  c.attrs = &early;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, a);
}

bool sizes_ok(const netkv_kv_pages* pages, uint32_t n_seqs, uint32_t heads, uint32_t width) {
  return kv_pages_ok(pages) && heads >= 1 && heads <= 65535 && heads % pages->kv_heads == 0 &&
         !(n_seqs >> 24) && width >= 1 && width < (1u << 28);
}

// Groups of up to 8 query heads take one tile of them, larger ones two: a second tile costs
// registers and products, and a second chunk reads the pages again.
int tiles_of(uint32_t group) { return group <= 8 ? 1 : 2; }

struct Workspace {
  size_t part_ml, lse2, block2, total;  // part_o is at 0
};
Workspace workspace(const netkv_kv_pages* p, uint32_t n_seqs, uint32_t heads, uint32_t width,
                    bool mass) {
  auto up = [](size_t x) { return (x + 127) / 128 * 128; };
  const size_t rows = (size_t)kMostCtas * 2 * tiles_of(heads / p->kv_heads) * 8;
  Workspace w;
  w.part_ml = up(rows * p->head_dim * 4);
  w.lse2 = w.part_ml + up(rows * 8);
  w.block2 = w.lse2 + (mass ? up((size_t)n_seqs * heads * 4) : 0);
  w.total = w.block2 + (mass ? (size_t)n_seqs * width * heads * 4 : 0);
  return w;
}

}  // namespace

extern "C" size_t netkv_attn_decode_workspace_size(const netkv_kv_pages* pages, uint32_t n_seqs,
                                                   uint32_t heads, uint32_t table_width,
                                                   int with_mass) {
  if (!sizes_ok(pages, n_seqs, heads, table_width)) return 0;
  return workspace(pages, n_seqs, heads, table_width, with_mass != 0).total;
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
      !(scale <= 3.4e38f))
    return NETKV_EINVAL;
  const Workspace ws = workspace(pages, n_seqs, heads, table_width, d_mass_out != nullptr);
  if (ws_bytes < ws.total) return NETKV_EINVAL;
  const uint32_t group = heads / pages->kv_heads, per = tiles_of(group) * 8;
  unsigned char* w = (unsigned char*)d_ws;
  const DecodeArgs a = {kv_args(pages),
                        (const unsigned char*)d_q,
                        (unsigned char*)d_out,
                        q_stride,
                        out_stride,
                        heads,
                        group,
                        (group + per - 1) / per,
                        n_seqs,
                        table_width,
                        d_len,
                        d_table,
                        scale * kLog2e,
                        d_lse,
                        d_mass_in,
                        d_mass_out,
                        (float*)w,
                        (float*)(w + ws.part_ml),
                        (float*)(w + ws.lse2),
                        (float*)(w + ws.block2),
                        per == 8 ? kCtas<1> : kCtas<2>,
                        d_status};
  const cudaStream_t s = (cudaStream_t)stream;
  auto go = [&](auto dim, auto tiles, auto bf, auto e4, auto mass) -> netkv_status {
    constexpr int kDim = decltype(dim)::value, kTiles = decltype(tiles)::value;
    constexpr bool kB = decltype(bf)::value, kE = decltype(e4)::value, kM = decltype(mass)::value;
    auto kernel = decode_kernel<kDim, kTiles, kB, kE, kM>;
    constexpr int bytes = (int)sizeof(Shared<kDim, kTiles>);
    NETKV_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    kernel<<<kCtas<kTiles>, kWarps * 32, bytes, s>>>(a);
    if (netkv_launch_status() != NETKV_OK) return NETKV_ECUDA;
    NETKV_CUDA_TRY(launch_following(join_kernel<kDim, kTiles, kB, kM>,
                                    dim3(kCtas<kTiles> - 1, min(group, per)), kJoin, s, a));
    return NETKV_OK;
  };
  auto with_mass = [&](auto dim, auto tiles, auto bf, auto e4) {
    return d_mass_out ? go(dim, tiles, bf, e4, std::true_type())
                      : go(dim, tiles, bf, e4, std::false_type());
  };
  auto types = [&](auto dim, auto tiles) {
    const bool bf = dtype == NETKV_BF16, e4 = pages->format == NETKV_KV_E4M3;
    if (bf && e4) return with_mass(dim, tiles, std::true_type(), std::true_type());
    if (bf) return with_mass(dim, tiles, std::true_type(), std::false_type());
    if (e4) return with_mass(dim, tiles, std::false_type(), std::true_type());
    return with_mass(dim, tiles, std::false_type(), std::false_type());
  };
  auto widths = [&](auto tiles) {
    return pages->head_dim == 64 ? types(std::integral_constant<int, 64>(), tiles)
                                 : types(std::integral_constant<int, 128>(), tiles);
  };
  const netkv_status st = per == 8 ? widths(std::integral_constant<int, 1>())
                                   : widths(std::integral_constant<int, 2>());
  if (st != NETKV_OK) return st;
  if (d_mass_out)
    NETKV_CUDA_TRY(launch_following(mass_kernel, dim3(n_seqs, min((table_width + 127) / 128, 1024u)),
                                    128, s, a));
  return netkv_launch_status();
}
