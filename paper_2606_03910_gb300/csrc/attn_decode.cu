// Attention of one query row a sequence over its 8-bit KV blocks, and the weight that each
// block has drawn.
//
// Bound: the codes are read once, 2 kDim bytes a token and KV head, and everything else is
// small, so the kernel streams pages and its arithmetic has to fit in their shadow: about 330
// instructions a warp and page of 4 KB, which take 45 % of the issue slots.  160 sequences of
// 5,500 tokens with 64 query heads on 8 KV heads of 128, int8: 291 us, 6.2 TB/s (bf16 queries 298);
// 64 of 13,000 with 16 on 2 and block weights: 90 us, 4.8 TB/s; two of 131,072, e4m3: 40 us, 3.4 TB/s
// (of which 20 are the bytes and 10 the join and both ends); one of 512: 10 us.
//
// Split: the work is the list of all pages, (sequence, KV head, block) in order, cut into equal
// runs, so that ragged batches and single long sequences spread over the card alike.  A run is
// a block's (four warps take a segment's pairs of pages in turn) or, where there are segments for
// every warp, a warp's.  It holds whole (sequence, head) segments, which are finished at once,
// and at most two that other runs share, whose sums go to the workspace for the join.  A warp of
// its own fills rings of pages by bulk copies (a page's part for a head is 16 kDim contiguous
// bytes) over the ends of segments and ahead of their queries: with the copies issued by the
// warps that use them, 160 sequences took 372 us.  Two pages a step make two chains of products
// to interleave; three blocks an SM hide what is left (two: 363 us).
//
// Arithmetic: a page is 16 tokens and a KV head serves a group of query heads, so S^T = K q^T
// and O^T = V^T P^T are products of 16 x 16 by 16 x 8: m16n8k16, with up to 8 (kTiles = 1) or
// 16 heads (2) side by side.  A tcgen05 product would be 128 rows high, of which the group
// fills 8.  Both code types are exact in fp16, so codes go into the products as they are and
// the scales are applied to scores and weights in fp32.  A row of bf16 queries is brought to
// [2^14, 2^15) by a power of two, the top of fp16's range that sums of fp32 leave room for: channels
// down to 2^-31 of the largest keep all of bf16's 8 bits.  The order of the inner dimension is free
// in a product: a thread's operands are the bytes that lie together, 16 at a load.
#include "kv_common.cuh"

namespace {

constexpr uint32_t kWarps = 4;
constexpr uint32_t kThreads = kWarps * 32 + 32;  // and a warp for the loads
// Blocks of the grid: three an SM on 152 SMs, two where a second tile of heads takes the registers.
template <int kTiles>
constexpr uint32_t kCtas = kTiles == 1 ? 456 : 304;
constexpr uint32_t kUncutBlocks = 32;  // see uncut_runs
template <int kDim>
constexpr uint32_t kStages = 256 / kDim;  // pairs of pages in flight a warp: 16 KB
constexpr uint32_t kEdge = 8;       // see Runs; at 0 runs of short segments end last (338 us for 308)
constexpr uint32_t kMinPages = 16;  // places of a run at least: a pair of pages for each of a block's
                                    // warps and an edge; a warp's own then cuts few short segments
// The running maximum follows the scores once one is above it by this (in powers of two):
// weights up to 2^8 are as exact in fp16 as those up to 1, and sums are fp32.
constexpr float kLag = 8.f;
// Weights go into the second product times their value scale over a unit that is above all value
// scales so far (at most twice the largest), and times 2^kUp: up to 2^(kLag + kUp), below fp16's
// 2^16.  They are exact to 2^-11 down to 2^-20 of the largest one, 0 below 2^-31; without the
// factor, keys 2^-24 below a sink of small values would leave the output and not its sum.
constexpr uint32_t kUp = 7;

struct Cut;

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
  float* part_o;    // [runs][2][kTiles * 8][kDim]
  float* part_ml;   // [runs][2][kTiles * 8][2]
  Cut* cuts;        // [runs - 1]
  float* lse2;      // [n_seqs][heads], in powers of two; with mass only
  float* block2;    // [n_seqs][width][heads]: log2 of a block's weight; with mass only
  uint32_t most_runs;
  uint32_t uncut;   // 1: a segment is all its first run's
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

__device__ __forceinline__ uint64_t div_floor(uint64_t x, uint64_t y) {
  return (x | y) >> 32 ? x / y : (uint32_t)x / (uint32_t)y;
}

// The runs: equal parts of a line on which every segment (a sequence and a unit: a KV head and a
// chunk of its query heads) takes kEdge places, what it costs to begin and end one in pages, and
// one for each page.
struct Runs {
  uint64_t total, base;
  uint32_t count, rest;
  __device__ __forceinline__ uint64_t start(uint32_t c) const { return base * c + min(c, rest); }
  // the first run that starts at `end` (up to total) or after it
  __device__ __forceinline__ uint32_t until(uint64_t end) const {
    const uint64_t longer = (base + 1) * rest;
    return end <= longer ? (uint32_t)div_floor(end + base, base + 1)
                         : rest + (uint32_t)div_floor(end - longer + base - 1, base);
  }
};

__device__ __forceinline__ uint64_t places(uint32_t pages) { return pages ? pages + kEdge : 0; }

// The sequences in chunks of 128, lane l's 4 l .. 4 l + 3 of one: the pages of the first chunk,
// and of chunk c (of the first 32) its places, in lane c.  Read once a warp.
struct Lens {
  uint32_t n[4];
  uint64_t chunk, total;
  static __device__ __forceinline__ uint64_t read(const DecodeArgs& a, uint32_t from, uint32_t* n) {
    const uint32_t i = from + (threadIdx.x & 31) * 4;
    uint64_t sum = 0;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      n[j] = i + j < a.n_seqs ? pages_of(a, i + j) : 0;
      sum += places(n[j]);
    }
    return sum;
  }
  static __device__ __forceinline__ uint64_t all(uint64_t x) {
#pragma unroll
    for (int d = 16; d; d /= 2) x += __shfl_xor_sync(~0u, x, d);
    return x;
  }
  __device__ __forceinline__ explicit Lens(const DecodeArgs& a) {
    const uint32_t lane = threadIdx.x & 31;
    total = all(read(a, 0, n));
    chunk = lane == 0 ? total : 0;
#pragma unroll 4
    for (uint32_t c = 1; c < min((a.n_seqs + 127) / 128, 32u); ++c) {
      uint32_t m[4];
      const uint64_t sum = all(read(a, c * 128, m));
      if (lane == c) chunk = sum;
      total += sum;
    }
    for (uint32_t from = 32 * 128; from < a.n_seqs; from += 128) {
      uint32_t m[4];
      total += all(read(a, from, m));
    }
  }
};

__device__ __forceinline__ Runs runs_of(const DecodeArgs& a, const Lens& lens, uint32_t units) {
  Runs r;
  r.total = lens.total * units;
  r.count = (uint32_t)min((uint64_t)a.most_runs, max((uint64_t)1, r.total / kMinPages));
  r.base = div_floor(r.total, r.count);
  r.rest = (uint32_t)(r.total - r.base * r.count);
  return r;
}

// A segment and a run's part of it: pages [first, first + count) of a sequence's `pages`.
struct Segment {
  uint32_t seq, unit, first, count, pages;
};

// The segment at a place of the line, and how far into it the place is.
__device__ __forceinline__ Segment segment_at(const DecodeArgs& a, const Lens& lens, uint32_t units,
                                              uint64_t at, uint64_t* into) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t from = 0;
  if (a.n_seqs > 128) {  // the chunk first
    uint64_t upto = lens.chunk * units;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint64_t x = __shfl_up_sync(~0u, upto, d);
      if (lane >= (uint32_t)d) upto += x;
    }
    const uint32_t hit = __ballot_sync(~0u, at < upto);
    const uint32_t c = hit ? __ffs(hit) - 1 : 32;
    const uint64_t before = __shfl_sync(~0u, upto, c ? c - 1 : 0);
    at -= c ? before : 0;
    from = c * 128;
  }
  for (; from < a.n_seqs; from += 128) {
    uint32_t n[4];
    uint64_t mine = 0;
    if (from == 0) {
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) n[j] = lens.n[j];
    } else {
      Lens::read(a, from, n);
    }
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) mine += places(n[j]) * units;
    uint64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint64_t x = __shfl_up_sync(~0u, upto, d);
      if (lane >= (uint32_t)d) upto += x;
    }
    const uint32_t hit = __ballot_sync(~0u, at < upto);
    if (hit) {
      const int who = __ffs(hit) - 1;
      uint64_t rest = at - (upto - mine);
      uint32_t j = 0, pages = n[0];
#pragma unroll
      for (uint32_t q = 0; q < 3; ++q)
        if (j == q && rest >= places(n[q]) * units) {
          rest -= places(n[q]) * units;
          j = q + 1;
          pages = n[q + 1];
        }
      rest = __shfl_sync(~0u, rest, who);
      pages = __shfl_sync(~0u, pages, who);
      const uint32_t seq = __shfl_sync(~0u, from + lane * 4 + j, who);
      const uint64_t unit = div_floor(rest, places(pages));
      *into = rest - unit * places(pages);
      return {seq, (uint32_t)unit, 0, 0, pages};
    }
    at -= __shfl_sync(~0u, upto, 31);
  }
  *into = 0;
  return {a.n_seqs, 0, 0, 0, 0};
}

// A boundary before a run, for the join: where it is inside a segment (parts > 0), that segment
// has parts from the runs run0, run0 + 1, ...; of the first of them it is the second or a later
// one (`second`) or the first; and `order` numbers the segment's boundaries.
struct Cut {
  uint32_t seq, unit, parts, run0, order, second;
};

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

// Waits for a phase of a barrier, a second at most.  Once that has run out for a thread of the
// block, which says so, nobody waits any longer and the block runs to its end.
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, volatile int* late,
                                     int* status) {
  if (try_wait(bar, parity)) return;
  const long long t0 = clock64();
  while (!try_wait(bar, parity)) {
    if (*late) return;
    if (clock64() - t0 > 2000000000ll) {
      *late = 1;
      flag_status(status, NETKV_DEV_ETIMEOUT);
      return;
    }
  }
}
// Before a warp ends: after a wait has run out, what is still in flight gets a moment to land.
__device__ __forceinline__ void settle(volatile int* late) {
  if (!*late) return;
  const long long t0 = clock64();
  while (clock64() - t0 < 20000000ll) {
  }
}
__device__ __forceinline__ void sync_warps() {  // all but the loading one
  asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
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

template <int kDim, int kTiles>
struct Shared {
  static constexpr int kHeads = kTiles * 8;
  static constexpr uint32_t kRing = kStages<kDim>;
  static constexpr int kGroupFloats = 16 * kHeads + 8;  // of 16 dims; the 8 spread the banks
  alignas(128) unsigned char ring[kWarps][kRing][2][2][kBlockTokens * kDim];
  float o[kWarps / 2][kDim / 16 * kGroupFloats];
  float m[kWarps][kHeads], l[kWarps][kHeads];
  float by[kHeads];  // what a head's sums are multiplied by
  alignas(16) float2 scale[kWarps][kRing][2];  // of keys and values
  uint2 tokens[kWarps][kRing];                 // of each page; 0 where it is absent
  alignas(8) uint64_t full[kWarps][kRing], empty[kWarps][kRing];
  int late;
};

// The segments of one run, in order.
struct Walk {
  Segment s;
  uint64_t left;  // places from s on
  __device__ __forceinline__ void take(const DecodeArgs& a, uint64_t into) {
    if (a.uncut) {
      left -= min(left, places(s.pages));
      s.first = 0;
      s.count = s.pages;
      return;
    }
    const uint64_t end = min(into + left, places(s.pages));
    left -= end - into;
    s.first = into > kEdge ? (uint32_t)(into - kEdge) : 0;
    s.count = end > kEdge ? (uint32_t)(end - kEdge) - s.first : 0;
  }
  // s.count = 0: no (more) segments
  __device__ __forceinline__ void start(const DecodeArgs& a, const Lens& lens, uint32_t units,
                                        const Runs& runs, uint32_t run, Cut* cut) {
    s.count = 0;
    left = 0;
    cut->parts = 0;
    if (run >= runs.count) return;
    const uint64_t first = runs.start(run);
    left = runs.start(run + 1) - first;
    if (left == 0) return;
    uint64_t into;
    s = segment_at(a, lens, units, first, &into);
    if (run && into > kEdge) {
      const uint64_t begin = first - into;
      cut->seq = s.seq;
      cut->unit = s.unit;
      cut->run0 = runs.until(begin + kEdge + 1) - 1;
      cut->parts = runs.until(begin + places(s.pages)) - cut->run0;
      cut->order = run - cut->run0 - 1;
      cut->second = runs.start(cut->run0) < begin;
    }
    if (a.uncut && into) {  // the segment is an earlier run's
      cut->parts = 0;
      left -= min(left, places(s.pages) - into);
      next(a, units);
      return;
    }
    take(a, into);
  }
  __device__ __forceinline__ void next(const DecodeArgs& a, uint32_t units) {
    s.count = 0;
    if (left == 0) return;
    if (++s.unit == units) {
      s.unit = 0;
      do {
        if (++s.seq >= a.n_seqs) return;  // lengths that changed under the call
        s.pages = pages_of(a, s.seq);
      } while (s.pages == 0);
    }
    take(a, 0);
  }
};

// The run of a block's warp: the block's, or (kOwn) the warp's own.
template <bool kOwn>
__device__ __forceinline__ uint32_t run_of(uint32_t warp) {
  return kOwn ? warp * gridDim.x + blockIdx.x : blockIdx.x;
}

// Pages on their way into the ring, a lane each: 32 of the block's segment, or (kOwn) 8 of each
// warp's.
struct Batch {
  uint32_t count;  // pages; 0: none left
  uint32_t kv_head, tokens;
  int32_t page;
  float2 scale;
};

// The loading warp: pairs of neighbouring pages.  Of a block's run they go to the four warps in
// turn; of the warps' own runs (kOwn), eight lanes serve a warp each.  The table's entries are
// read two batches ahead and the scales one, over the ends of segments too, so that a ring's
// place is filled as soon as it is free.
template <int kDim, int kTiles, bool kOwn>
__device__ __forceinline__ void load_pages(const DecodeArgs& a, Shared<kDim, kTiles>& sh,
                                           const Lens& lens, uint32_t units, const Runs& runs) {
  constexpr uint32_t kRing = kStages<kDim>, kPart = kBlockTokens * kDim;
  constexpr uint32_t kLanes = kOwn ? 32 / kWarps : 32;  // of a batch
  const uint32_t lane = threadIdx.x & 31, in = lane % kLanes;
  volatile int* late = &sh.late;
  Walk walk;
  Cut unused;
#pragma unroll
  for (uint32_t w = 0; w < (kOwn ? kWarps : 1); ++w) {
    Walk x;
    x.start(a, lens, units, runs, run_of<kOwn>(w), &unused);
    if (w == lane / kLanes) walk = x;
  }
  uint32_t at = 0;  // pages of the present segment that batches have
  auto take = [&]() {
    Batch b = {0, 0, 0, -1, make_float2(0.f, 0.f)};
    if (walk.s.count && at == walk.s.count) {
      walk.next(a, units);
      at = 0;
    }
    if (walk.s.count == 0) return b;
    b.count = min(walk.s.count - at, kLanes);
    b.kv_head = walk.s.unit / a.chunks;
    if (in < b.count) {
      const uint32_t block = walk.s.first + at + in;
      b.page = a.table[(uint64_t)walk.s.seq * a.width + block];
      b.tokens = min(tokens_of(a, walk.s.seq) - block * kBlockTokens, kBlockTokens);
    }
    at += b.count;
    return b;
  };
  auto scales = [&](Batch& b) {
    if (in >= b.count) return;
    if (b.page < 0 || (uint32_t)b.page >= a.kv.n_pages) {
      flag_status(a.status, NETKV_DEV_ERANGE);
      b.page = -1;
      b.tokens = 0;
      return;
    }
    const uint64_t part = (uint64_t)b.page * a.kv.heads + b.kv_head;
    b.scale = make_float2(a.kv.k_scale[part], a.kv.v_scale[part]);
  };
  // the warp that a lane's pages go to, and the pairs that it was given
  const uint32_t w = kOwn ? lane / kLanes : lane / 2 % kWarps, step = kOwn ? 1 : kWarps;
  const uint32_t turn = in / 2 / step;  // of the batch's pairs for that warp
  uint32_t given = 0;
  Batch b0 = take(), b1 = take();
  scales(b0);
  scales(b1);
  while (__any_sync(~0u, b0.count && !*late)) {
    const Batch b2 = take();
    const uint32_t pairs = (b0.count + 1) / 2, n = given + turn;
    for (uint32_t q = 0; q < 32 / (2 * kWarps); ++q) {  // a pair for each warp
      if (turn == q && in / 2 < pairs) {
        const uint32_t st = n % kRing, bar = smem_addr(&sh.full[w][st]);
        if (n >= kRing) wait(smem_addr(&sh.empty[w][st]), (n / kRing - 1) & 1, late, a.status);
        if (!*late) {
          if (b0.page >= 0) {
            const uint64_t from = ((uint64_t)b0.page * a.kv.heads + b0.kv_head) * kPart;
            asm volatile(
                "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, "
                "[%3];" ::"r"(smem_addr(sh.ring[w][st][lane & 1][0])),
                "l"(a.kv.k + from), "r"(kPart), "r"(bar)
                : "memory");
            asm volatile(
                "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, "
                "[%3];" ::"r"(smem_addr(sh.ring[w][st][lane & 1][1])),
                "l"(a.kv.v + from), "r"(kPart), "r"(bar)
                : "memory");
          }
          sh.scale[w][st][lane & 1] = b0.scale;
          (&sh.tokens[w][st].x)[lane & 1] = b0.tokens;
          asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar),
                       "r"(b0.page >= 0 ? 2 * kPart : 0)
                       : "memory");
        }
      }
      __syncwarp();
    }
    given += kOwn ? pairs : (pairs + kWarps - 1 - w) / kWarps;
    b0 = b1;
    b1 = b2;
    scales(b1);
  }
}

template <int kDim, int kTiles, bool kBf16, bool kE4m3, bool kMass, bool kOwn>
__global__ void __launch_bounds__(kThreads, kTiles == 1 ? 3 : 2)
    decode_kernel(const __grid_constant__ DecodeArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  using Sh = Shared<kDim, kTiles>;
  Sh& sh = *reinterpret_cast<Sh*>(smem);
  constexpr int kHeads = kTiles * 8, kSteps = kDim / 16, kPart = kBlockTokens * kDim;
  constexpr uint32_t kRing = Sh::kRing;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32, r = lane / 4, c = lane % 4;
  const uint32_t units = a.kv.heads * a.chunks;
  let_follow();

  if (warp < kWarps && lane < kRing) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 2;" ::"r"(smem_addr(&sh.full[warp][lane]))
                 : "memory");
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_addr(&sh.empty[warp][lane]))
                 : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 0) sh.late = 0;
  const Lens lens(a);
  const Runs runs = runs_of(a, lens, units);
  __syncthreads();
  volatile int* late = &sh.late;
  if (warp == kWarps) {
    load_pages<kDim, kTiles, kOwn>(a, sh, lens, units, runs);
    settle(late);
    return;
  }
  Walk walk;
  Cut cut;
  const uint32_t run = run_of<kOwn>(warp);
  walk.start(a, lens, units, runs, run, &cut);
  if (run && (kOwn ? lane : tid) == 0) a.cuts[run - 1] = cut;

  // Queries of a segment: thread (r, c) has head r of each tile, dims by 16 bytes of codes:
  // 64 h + 16 c + 4 i + 0..3 in step 4 h + i.  Read ahead of their segment.
  uint4 raw[kTiles][kDim / 32];
  auto load_queries = [&]() {
    const uint32_t kv_head = walk.s.unit / a.chunks, head0 = walk.s.unit % a.chunks * kHeads;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const uint32_t h = head0 + t * 8 + r;
      const uint4* src = reinterpret_cast<const uint4*>(
          a.q + (walk.s.seq * a.q_stride +
                 ((uint64_t)kv_head * a.group + min(h, a.group - 1)) * kDim) * 2);
#pragma unroll
      for (int i = 0; i < kDim / 32; ++i)
        raw[t][i] = h < a.group ? src[(i / 2) * 8 + c * 2 + i % 2] : make_uint4(0, 0, 0, 0);
    }
  };
  if (walk.s.count) load_queries();
  uint32_t taken = 0;  // pairs of all segments
  bool first_segment = true;
  while (walk.s.count) {
    const Segment seg = walk.s;
    const uint32_t kv_head = seg.unit / a.chunks, head0 = seg.unit % a.chunks * kHeads;
    const uint32_t all_pairs = (seg.count + 1) / 2;
    const uint32_t pairs =
        kOwn ? all_pairs : all_pairs > warp ? (all_pairs - warp + kWarps - 1) / kWarps : 0;
    uint32_t q[kTiles][kSteps][2];
    float f[kTiles][2];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(raw[t]);
      if constexpr (kBf16) {
        float largest = 0.f;
#pragma unroll
        for (int i = 0; i < kDim / 8; ++i) {
          const float2 x = unpack16<kBf16>(w[i]);
          largest = fmaxf(largest, fmaxf(fabsf(x.x), fabsf(x.y)));
        }
        largest = fmaxf(largest, __shfl_xor_sync(~0u, largest, 1));
        largest = fmaxf(largest, __shfl_xor_sync(~0u, largest, 2));
        // 2^14 over the largest value's power of two, and the reverse; both are normal numbers
        const uint32_t e = max(__float_as_uint(largest) >> 23, 15u);
        const float inv = __uint_as_float((254 + 14 - e) << 23);
        const float up = __uint_as_float((e - 14) << 23) * a.scale2;
        f[t][0] = __shfl_sync(~0u, up, 8 * c);
        f[t][1] = __shfl_sync(~0u, up, 8 * c + 4);
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 x = unpack16<kBf16>(w[i * 2 + j]);
            q[t][i][j] = pack16<false>(x.x * inv, x.y * inv);
          }
      } else {
        f[t][0] = f[t][1] = a.scale2;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) q[t][i][j] = w[i * 2 + j];
      }
    }
    float o[kTiles][kDim / 16][4] = {}, m[kTiles][2], l[kTiles][2] = {};
#pragma unroll
    for (int t = 0; t < kTiles; ++t) m[t][0] = m[t][1] = -INFINITY;
    float v_unit = 0.f, v_inv = 0.f;  // a power of two that the sums are in, 1 over it

    for (uint32_t i = 0; i < pairs; ++i) {
      const uint32_t st = taken % kRing;
      wait(smem_addr(&sh.full[warp][st]), (taken / kRing) & 1, late, a.status);
      ++taken;
      const uint32_t at = 2 * (kOwn ? i : warp + kWarps * i), block = seg.first + at;
      const uint2 nn = sh.tokens[warp][st];
      const uint32_t n[2] = {nn.x, nn.y};
      const bool full = n[0] + n[1] == 2 * kBlockTokens;
      if (n[0] + n[1]) {
        const float4 sc = *reinterpret_cast<const float4*>(sh.scale[warp][st]);
        const float ks[2] = {sc.x, sc.z}, vs[2] = {sc.y, sc.w};
        const unsigned char(*pg)[2][kPart] = sh.ring[warp][st];

        float s[2][kTiles][4] = {};
#pragma unroll
        for (int h = 0; h < kDim / 64; ++h)
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const unsigned char* kp = pg[g][0] + h * 64 + c * 16;
            const uint4 x = *reinterpret_cast<const uint4*>(kp + r * kDim);
            const uint4 y = *reinterpret_cast<const uint4*>(kp + (r + 8) * kDim);
            const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              uint32_t a0, a1, a2, a3;
              widen<kE4m3>(xs[z], &a0, &a2);
              widen<kE4m3>(ys[z], &a1, &a3);
#pragma unroll
              for (int t = 0; t < kTiles; ++t)
                mma(s[g][t], a0, a1, a2, a3, q[t][h * 4 + z][0], q[t][h * 4 + z][1]);
            }
          }
        // s: tokens r and r + 8 of a page, heads 2 c and 2 c + 1 of each tile
        bool above = false;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              s[g][t][z] *= ks[g] * f[t][z & 1];
              if (!full && r + (z / 2) * 8 >= n[g]) s[g][t][z] = -INFINITY;
              above |= s[g][t][z] > m[t][z & 1] + kLag;
            }
        if (__any_sync(~0u, above)) {
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            float to[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float x = m[t][j];
#pragma unroll
              for (int g = 0; g < 2; ++g) x = fmaxf(x, fmaxf(s[g][t][j], s[g][t][j + 2]));
#pragma unroll
              for (int d = 4; d < 32; d *= 2) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
              to[j] = m[t][j] == -INFINITY ? 0.f : ex2(m[t][j] - x);
              m[t][j] = x;
              l[t][j] *= to[j];
            }
#pragma unroll
            for (int j = 0; j < kDim / 16; ++j)
#pragma unroll
              for (int z = 0; z < 4; ++z) o[t][j][z] *= to[z & 1];
          }
        }
        if (fmaxf(vs[0], vs[1]) > v_unit * (1 << kUp)) {  // the whole warp
          const uint32_t e = min(max(__float_as_uint(fmaxf(vs[0], vs[1])) >> 23, kUp + 2), 254u);
          const float unit = __uint_as_float((e + 1 - kUp) << 23), shrink = v_unit / unit;
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int j = 0; j < kDim / 16; ++j)
#pragma unroll
              for (int z = 0; z < 4; ++z) o[t][j][z] *= shrink;
          v_unit = unit;
          v_inv = __uint_as_float((253 + kUp - e) << 23);
        }
        uint32_t p[2][kTiles][2];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          float sums[2][2];  // of a page's tokens r and r + 8
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const float w = vs[g] * v_inv;
            float x[4];
#pragma unroll
            for (int z = 0; z < 4; ++z) x[z] = ex2(s[g][t][z] - m[t][z & 1]);
#pragma unroll
            for (int j = 0; j < 2; ++j) l[t][j] += sums[g][j] = x[j] + x[j + 2];
            p[g][t][0] = transpose8x8(pack16<false>(x[0] * w, x[1] * w));
            p[g][t][1] = transpose8x8(pack16<false>(x[2] * w, x[3] * w));
          }
          if (kMass) {  // over the tokens: a quarter of the threads r for each page and head
            const bool page1 = r & 1, head1 = r & 2;
            float y[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
              y[j] = (page1 ? sums[1][j] : sums[0][j]) +
                     __shfl_xor_sync(~0u, page1 ? sums[0][j] : sums[1][j], 4);
            float sum = (head1 ? y[1] : y[0]) + __shfl_xor_sync(~0u, head1 ? y[0] : y[1], 8);
            sum += __shfl_xor_sync(~0u, sum, 16);
            const uint32_t h = head0 + t * 8 + 2 * c + (r >> 1), g = r & 1;
            if (r < 4 && h < a.group && at + g < seg.count)
              a.block2[((uint64_t)seg.seq * a.width + block + g) * a.heads + kv_head * a.group + h] =
                  (head1 ? m[t][1] : m[t][0]) + lg2(sum);
          }
        }
        // values: tokens 2 c, 2 c + 1, 2 c + 8 and 2 c + 9, dims r * kDim / 8 on; zeros past
        // the last token, whose codes may stand for anything
        constexpr int kWords = kDim / 32;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          uint32_t v[4][kWords];
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const uint32_t row = 2 * c + (z & 1) + (z / 2) * 8;
            const unsigned char* src = pg[g][1] + row * kDim + r * (kDim / 8);
            if (kWords == 4) {
              const uint4 y = *reinterpret_cast<const uint4*>(src);
              v[z][0] = y.x, v[z][1] = y.y, v[z][kWords - 2] = y.z, v[z][kWords - 1] = y.w;
            } else {
              const uint2 y = *reinterpret_cast<const uint2*>(src);
              v[z][0] = y.x, v[z][1] = y.y;
            }
            if (!full && row >= n[g]) {
#pragma unroll
              for (int j = 0; j < kWords; ++j) v[z][j] = 0;
            }
          }
#pragma unroll
          for (int z = 0; z < kWords; ++z)
#pragma unroll
            for (int j = 0; j < 2; ++j) {  // tile 2 z + j: dims 4 z + 2 j and the next of the run
              const uint32_t sel = j ? 0x7362 : 0x5140;
              uint32_t a0, a1, a2, a3;
              widen<kE4m3>(__byte_perm(v[0][z], v[1][z], sel), &a0, &a1);
              widen<kE4m3>(__byte_perm(v[2][z], v[3][z], sel), &a2, &a3);
#pragma unroll
              for (int t = 0; t < kTiles; ++t)
                mma(o[t][2 * z + j], a0, a1, a2, a3, p[g][t][0], p[g][t][1]);
            }
        }
      } else if (kMass && r < 2) {
#pragma unroll
        for (int z = 0; z < kHeads / 4; ++z) {
          const uint32_t h = head0 + c + z * 4;
          if (h < a.group && at + r < seg.count)
            a.block2[((uint64_t)seg.seq * a.width + block + r) * a.heads + kv_head * a.group + h] =
                -INFINITY;
        }
      }
      __syncwarp();
      if (lane == 0)
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(&sh.empty[warp][st]))
                     : "memory");
    }

    // ---- the warps' sums
    const bool whole = seg.count == seg.pages;
    walk.next(a, units);
    if (walk.s.count) load_queries();
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[t][j] += __shfl_xor_sync(~0u, l[t][j], d);
    const uint32_t slot = run * 2 + (first_segment ? 0 : 1);
    first_segment = false;
    if constexpr (kOwn) {  // a thread has kDim / 8 neighbouring dims of each of its heads
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t h = t * 8 + 2 * c + j;
          if (head0 + h >= a.group) continue;
          const uint32_t head = kv_head * a.group + head0 + h;
          const float sum = l[t][j], top = m[t][j];
          const float by = !whole ? v_unit : sum == 0.f ? 0.f : v_unit / sum;
          float x[kDim / 8];
#pragma unroll
          for (int i = 0; i < kDim / 8; ++i) x[i] = o[t][i / 2][2 * (i & 1) + j] * by;
          if (whole) {
            uint4* to = reinterpret_cast<uint4*>(
                a.out + (seg.seq * a.out_stride + (uint64_t)head * kDim + r * (kDim / 8)) * 2);
#pragma unroll
            for (int i = 0; i < kDim / 64; ++i)
              to[i] = make_uint4(pack16<kBf16>(x[i * 8], x[i * 8 + 1]),
                                 pack16<kBf16>(x[i * 8 + 2], x[i * 8 + 3]),
                                 pack16<kBf16>(x[i * 8 + 4], x[i * 8 + 5]),
                                 pack16<kBf16>(x[i * 8 + 6], x[i * 8 + 7]));
            if (r == 0) {
              const float z = sum == 0.f ? -INFINITY : top + log2f(sum);
              if (a.lse) a.lse[(uint64_t)seg.seq * a.heads + head] = z * kLn2;
              if (kMass) a.lse2[(uint64_t)seg.seq * a.heads + head] = z;
            }
          } else {
            float4* to = reinterpret_cast<float4*>(a.part_o + ((uint64_t)slot * kHeads + h) * kDim +
                                                   r * (kDim / 8));
#pragma unroll
            for (int i = 0; i < kDim / 32; ++i)
              to[i] = make_float4(x[i * 4], x[i * 4 + 1], x[i * 4 + 2], x[i * 4 + 3]);
            if (r == 0) {
              a.part_ml[(slot * kHeads + h) * 2] = top;
              a.part_ml[(slot * kHeads + h) * 2 + 1] = sum;
            }
          }
        }
      continue;
    }
    if (r == 0) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          sh.m[warp][t * 8 + 2 * c + j] = m[t][j];
          sh.l[warp][t * 8 + 2 * c + j] = l[t][j];
        }
    }
    sync_warps();
    if (tid < kHeads) {
      float top = sh.m[0][tid], sum = 0.f;
#pragma unroll
      for (uint32_t w = 1; w < kWarps; ++w) top = fmaxf(top, sh.m[w][tid]);
#pragma unroll
      for (uint32_t w = 0; w < kWarps; ++w)
        sum += (sh.m[w][tid] == -INFINITY ? 0.f : ex2(sh.m[w][tid] - top)) * sh.l[w][tid];
      sh.by[tid] = !whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
      if (head0 + tid < a.group) {
        const uint64_t at = (uint64_t)seg.seq * a.heads + kv_head * a.group + head0 + tid;
        const float z = sum == 0.f ? -INFINITY : top + log2f(sum);
        if (whole && a.lse) a.lse[at] = z * kLn2;
        if (whole && kMass) a.lse2[at] = z;
        if (!whole)
          reinterpret_cast<float2*>(a.part_ml)[slot * kHeads + tid] = make_float2(top, sum);
      }
    }
    // to one maximum; then two warps' sums through shared memory onto the other two's
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int h = t * 8 + 2 * c + j;
        float top = sh.m[0][h];
#pragma unroll
        for (uint32_t w = 1; w < kWarps; ++w) top = fmaxf(top, sh.m[w][h]);
        const float by = m[t][j] == -INFINITY ? 0.f : ex2(m[t][j] - top) * v_unit;
#pragma unroll
        for (int x = 0; x < kDim / 16; ++x)
#pragma unroll
          for (int i = 0; i < 2; ++i) o[t][x][2 * i + j] *= by;
      }
    auto place = [&](int t, int j, int x, int i) -> float& {
      const uint32_t dim = r * (kDim / 8) + 2 * x + i;
      return sh.o[warp % 2][dim / 16 * Sh::kGroupFloats + dim % 16 * kHeads + t * 8 + 2 * c + j];
    };
#pragma unroll
    for (int half = 1; half >= 0; --half) {
      if (warp / 2 == half) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int x = 0; x < kDim / 16; ++x)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                float& z = place(t, j, x, i);
                z = half ? o[t][x][2 * i + j] : z + o[t][x][2 * i + j];
              }
      }
      sync_warps();
    }
#pragma unroll
    for (uint32_t i = 0; i < kHeads * kDim / 2 / (kWarps * 32); ++i) {  // two dims a thread
      const uint32_t x = 2 * (i * kWarps * 32 + tid), h = x / kDim, dim = x % kDim;
      const uint32_t at = dim / 16 * Sh::kGroupFloats + dim % 16 * kHeads + h;
      const float by = sh.by[h];
      const float y0 = (sh.o[0][at] + sh.o[1][at]) * by;
      const float y1 = (sh.o[0][at + kHeads] + sh.o[1][at + kHeads]) * by;
      if (head0 + h >= a.group) continue;
      const uint32_t head = kv_head * a.group + head0 + h;
      if (whole)
        *reinterpret_cast<uint32_t*>(
            a.out + (seg.seq * a.out_stride + (uint64_t)head * kDim + dim) * 2) = pack16<kBf16>(y0, y1);
      else
        *reinterpret_cast<float2*>(a.part_o + ((uint64_t)slot * kHeads + h) * kDim + dim) =
            make_float2(y0, y1);
    }
    sync_warps();
  }

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
  settle(late);
}

// Joins the segments that runs share: one block of threads a boundary.  The boundaries of a
// segment share its heads; a head's parts are spread over the block's warps that have it (all 8
// for one head: a long sequence alone on the card has 456 parts; one for each of eight heads where
// a segment is cut once), a lane has kDim / 32 dims, and their sums are added in the warps' order.
// A warp reads kBatch parts at a time: 8 where segments are few and long; 2 with a run for each
// warp, whose boundaries are many and need the SMs' registers for other blocks (at 8, 300
// sequences of 1,000 tokens at 64 query heads took 148 us instead of 134).
template <int kTiles>
constexpr uint32_t kJoin = kTiles == 1 ? 256 : 512;  // a warp for each head of a tile, at least
template <int kDim, int kTiles, bool kBf16, bool kMass, bool kOwn>
__global__ void __launch_bounds__(kJoin<kTiles>) join_kernel(const __grid_constant__ DecodeArgs a) {
  constexpr int kBatch = kOwn ? 2 : 8;
  constexpr uint32_t kHeads = kTiles * 8, kJoinWarps = kJoin<kTiles> / 32, kPer = kDim / 32;
  __shared__ float sums[kJoinWarps][kDim];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  let_follow();
  follow();
  const Cut s = a.cuts[blockIdx.x];
  const uint32_t joiners = min(s.parts - 1, kHeads);
  if (s.parts == 0 || s.order >= joiners) return;
  const uint32_t heads = (kHeads - s.order + joiners - 1) / joiners;  // of this block
  uint32_t spread = 1;
  while (spread < heads) spread *= 2;
  const uint32_t each = kJoinWarps / spread;  // warps of a head
  const uint32_t h = s.order + warp % spread * joiners, head0 = s.unit % a.chunks * kHeads;
  const bool real = h < kHeads && head0 + h < a.group;
  auto slot = [&](uint32_t i) {
    return ((uint64_t)(s.run0 + i) * 2 + (i == 0 ? s.second : 0)) * kHeads + h;
  };
  float top = -INFINITY, sum = 0.f, o[kPer] = {};
  if (real) {
    // loads of several parts are under way at a time, the first sums before the maxima they
    // wait for: each is a round trip to L2
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
    float m[kBatch], x[kBatch][kPer];
    auto read = [&](uint32_t i) {
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t at = i + j * each;
        const bool in = at < s.parts;
        m[j] = in ? ml[slot(at)].x : -INFINITY;
#pragma unroll
        for (uint32_t q = 0; q < kPer; ++q) x[j][q] = 0.f;
        if (in) {
          const float* from = a.part_o + slot(at) * kDim + lane * kPer;
          if constexpr (kPer == 4) {
            const float4 y = *reinterpret_cast<const float4*>(from);
            x[j][0] = y.x, x[j][1] = y.y, x[j][2] = y.z, x[j][3] = y.w;
          } else {
            const float2 y = *reinterpret_cast<const float2*>(from);
            x[j][0] = y.x, x[j][1] = y.y;
          }
        }
      }
    };
    uint32_t next = warp / spread;
    read(next);
    for (uint32_t i = 0; i < s.parts; i += 128) {
      float2 z[4];
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        const uint32_t at = i + j * 32 + lane;
        z[j] = at < s.parts ? ml[slot(at)] : make_float2(-INFINITY, 0.f);
      }
      float to = fmaxf(fmaxf(fmaxf(z[0].x, z[1].x), fmaxf(z[2].x, z[3].x)), top);
#pragma unroll
      for (int d = 16; d; d /= 2) to = fmaxf(to, __shfl_xor_sync(~0u, to, d));
      sum = top == -INFINITY ? sum : sum * ex2(top - to);
      // a part of NaN scores has no maximum, but its sum says so
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
        sum += z[j].x == -INFINITY ? 0.f * z[j].y : ex2(z[j].x - to) * z[j].y;
      top = to;
    }
#pragma unroll
    for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
    while (true) {
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const float w = m[j] == -INFINITY ? 0.f : ex2(m[j] - top);
#pragma unroll
        for (uint32_t q = 0; q < kPer; ++q) o[q] += w * x[j][q];
      }
      next += kBatch * each;
      if (next >= s.parts) break;
      read(next);
    }
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) sums[warp][lane * kPer + i] = o[i];
  }
  __syncthreads();
  if (warp >= spread || !real) return;
  for (uint32_t w = 1; w < each; ++w)
#pragma unroll
    for (uint32_t i = 0; i < kPer; ++i) o[i] += sums[warp + w * spread][lane * kPer + i];
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const uint32_t head = s.unit / a.chunks * a.group + head0 + h;
  uint32_t* to =
      reinterpret_cast<uint32_t*>(a.out + (s.seq * a.out_stride + (uint64_t)head * kDim) * 2);
#pragma unroll
  for (uint32_t i = 0; i < kPer; i += 2)
    to[lane * (kPer / 2) + i / 2] = pack16<kBf16>(o[i] * inv, o[i + 1] * inv);
  if (lane == 0) {
    const float z = sum == 0.f ? -INFINITY : top + log2f(sum);
    if (a.lse) a.lse[(uint64_t)s.seq * a.heads + head] = z * kLn2;
    if (kMass) a.lse2[(uint64_t)s.seq * a.heads + head] = z;
  }
}

// A block's weight over all heads: its heads' parts are neighbours, a lane each (two or more
// lanes' worth above 32 heads, several blocks a warp up to 16), added in one order.
constexpr uint32_t kMassWarps = 8, kMassSteps = 8;
__global__ void __launch_bounds__(kMassWarps * 32) mass_kernel(const __grid_constant__ DecodeArgs a) {
  const uint32_t seq = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const uint32_t pages = pages_of(a, seq);
  uint32_t lanes = 32;  // of a block
  while (lanes / 2 >= a.heads) lanes /= 2;
  const uint32_t per = 32 / lanes, head = lane % lanes;
  // a sequence's first block waits without work too: were all blocks done before the kernels ahead,
  // so would be the call
  if (blockIdx.y && blockIdx.y * kMassWarps * kMassSteps * per >= pages) return;
  follow();
  for (uint32_t from = blockIdx.y * kMassWarps * kMassSteps * per; from < pages;
       from += gridDim.y * kMassWarps * kMassSteps * per) {
    const uint32_t first = from + warp * per + lane / lanes;
    float sum[kMassSteps] = {}, before[kMassSteps] = {};
    if (a.mass_in && head == 0)
#pragma unroll
      for (uint32_t q = 0; q < kMassSteps; ++q) {
        const uint32_t block = first + q * kMassWarps * per;
        if (block < pages) before[q] = a.mass_in[(uint64_t)seq * a.width + block];
      }
    for (uint32_t h = head; h < a.heads; h += lanes) {
      const float z = a.lse2[(uint64_t)seq * a.heads + h];
      float b[kMassSteps];  // loaded together: each is a round trip to memory
#pragma unroll
      for (uint32_t q = 0; q < kMassSteps; ++q) {
        const uint32_t block = first + q * kMassWarps * per;
        b[q] = -INFINITY;
        if (block < pages) b[q] = a.block2[((uint64_t)seq * a.width + block) * a.heads + h];
      }
#pragma unroll
      for (uint32_t q = 0; q < kMassSteps; ++q) sum[q] += b[q] == -INFINITY ? 0.f : ex2(b[q] - z);
    }
#pragma unroll
    for (uint32_t q = 0; q < kMassSteps; ++q) {
      for (uint32_t d = lanes / 2; d; d /= 2) sum[q] += __shfl_xor_sync(~0u, sum[q], d);
      const uint32_t block = first + q * kMassWarps * per;
      if (head == 0 && block < pages)
        a.mass_out[(uint64_t)seq * a.width + block] = before[q] + sum[q];
    }
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

// Batches with a segment for every warp of the grid give each warp a run of its own: segments
// then begin and end without the other warps (1,000 sequences of about 100 tokens at 64 query
// heads 153 -> 86 us).  With fewer, four warps are through a segment sooner than one.
bool own_runs(const netkv_kv_pages* p, uint32_t n_seqs, uint32_t heads) {
  const uint32_t group = heads / p->kv_heads;
  const int tiles = tiles_of(group);
  return (uint64_t)n_seqs * p->kv_heads * ((group + tiles * 8 - 1) / (tiles * 8)) >=
         (tiles == 1 ? kCtas<1> : kCtas<2>) * kWarps;
}

// Tables of up to 32 blocks: no segment is worth a join, whose launch and round trips take 5 us
// (64 sequences of 500 tokens 18.8 -> 14.8 us).  At 64 blocks one of 1,000 tokens alone would
// take 16.7 us instead of 14.7, and 300 of them 66 instead of 57, as runs get uneven.
bool uncut_runs(uint32_t width) { return width <= kUncutBlocks; }

struct Workspace {
  uint32_t runs;
  size_t part_ml, cuts, lse2, block2, total;  // part_o is at 0
};
Workspace workspace(const netkv_kv_pages* p, uint32_t n_seqs, uint32_t heads, uint32_t width,
                    bool mass) {
  auto up = [](size_t x) { return (x + 127) / 128 * 128; };
  const int tiles = tiles_of(heads / p->kv_heads);
  Workspace w;
  w.runs = (tiles == 1 ? kCtas<1> : kCtas<2>) * (own_runs(p, n_seqs, heads) ? kWarps : 1);
  const size_t rows = (size_t)w.runs * 2 * tiles * 8;
  w.part_ml = up(rows * p->head_dim * 4);
  w.cuts = w.part_ml + up(rows * 8);
  w.lse2 = w.cuts + up(w.runs * sizeof(Cut));
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
      !aligned_to(d_status, 4) || (d_mass_in && !d_mass_out) || !scale_ok(scale))
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
                        (Cut*)(w + ws.cuts),
                        (float*)(w + ws.lse2),
                        (float*)(w + ws.block2),
                        ws.runs,
                        uncut_runs(table_width),
                        d_status};
  const cudaStream_t s = (cudaStream_t)stream;
  const bool own = own_runs(pages, n_seqs, heads);
  auto go = [&](auto dim, auto tiles, auto bf, auto e4, auto mass) -> netkv_status {
    constexpr int kDim = decltype(dim)::value, kTiles = decltype(tiles)::value;
    constexpr bool kB = decltype(bf)::value, kE = decltype(e4)::value, kM = decltype(mass)::value;
    constexpr auto shared = decode_kernel<kDim, kTiles, kB, kE, kM, false>;
    constexpr auto owned = decode_kernel<kDim, kTiles, kB, kE, kM, true>;
    constexpr int bytes = (int)sizeof(Shared<kDim, kTiles>);
    NETKV_CUDA_TRY(own ? allow_shared<owned>(bytes) : allow_shared<shared>(bytes));
    (own ? owned : shared)<<<kCtas<kTiles>, kThreads, bytes, s>>>(a);
    if (netkv_launch_status() != NETKV_OK) return NETKV_ECUDA;
    if (!uncut_runs(table_width))
      NETKV_CUDA_TRY(launch_following(own ? join_kernel<kDim, kTiles, kB, kM, true>
                                          : join_kernel<kDim, kTiles, kB, kM, false>,
                                      ws.runs - 1, kJoin<kTiles>, s, a));
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
    NETKV_CUDA_TRY(launch_following(
        mass_kernel, dim3(n_seqs, min((table_width - 1) / (kMassWarps * kMassSteps) + 1, 1024u)),
        kMassWarps * 32, s, a));
  return netkv_launch_status();
}
