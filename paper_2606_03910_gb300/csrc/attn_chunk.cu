// Causal attention of each sequence's new tokens over its 8-bit KV blocks.
//
// A KV head serves `group` query heads, so a sequence's new tokens are tokens * group rows for it,
// token by token, and a row block is 256 of them: two tiles of 128 rows that read the same keys.  Where
// a row block has 128 rows or fewer, both tiles are the same rows, and take the even and the odd key
// tiles.  Keys come 128 at a time: eight blocks of 16 tokens.
//
// Bound: with 256 rows shared memory, which a key tile at 128 wide takes for 2,500 clocks (320 KB: the
// products read 192, widening moves 128), where the tensor cores take 2,048; with 128 or fewer the
// widening, where HBM would take 1,400 (32 KB of codes, an SM's share).  2,048 tokens of 16 heads on 2
// behind 65,536: 800 to 816 us, 1,370 to 1,400 TFLOP/s; 512 behind 7,680: 54 us; two parts of 900 tokens
// among 24 decoded ones: 217 us; 64 sequences of 9,400 tokens with 5 drafted ones each, e4m3: 133 us, 2.3
// TB/s.
//
// Split: a line on which every row block has places for the keys that it sees and for its beginning
// and end is cut into equal runs, one a block of threads, so that single long sequences, ragged
// batches and long chunks spread over the card alike.  Row blocks that runs share are joined by a
// second kernel from fp32 sums in the workspace.
//
// Roles of a block's warps: one plans (the run's items), one reads table entries and scales ahead and
// copies the keys' codes to shared memory, one the values', four widen them into fp16 tiles, one issues
// the products, and eight take the softmax.
//
// Arithmetic: both code types are exact in fp16, so codes go into the products as they are, and the
// blocks' scales are applied to scores and weights in fp32.  A row of bf16 queries is brought to
// [2^14, 2^15) by a power of two.  S = Q K^T and O += P V are tcgen05 products with fp32 sums in TMEM;
// P takes S's place as fp16.  One pass over the keys carries a row's maximum and sum (Milakov and
// Gimelshein, 2018).
#include "tensor.cuh"

namespace {

constexpr uint32_t kRows = 128, kKeys = 128;  // of a tile
constexpr uint32_t kTileBlocks = kKeys / kBlockTokens;
constexpr uint32_t kCtas = 152;  // blocks of the grid, one an SM: they hold all of TMEM
// The running maximum follows the scores once one is above it by this (in powers of two).
constexpr float kLag = 8.f;
// Weights go into the second product times their value scale over the largest one that the row has seen
// so far, and times 2^kUp: up to 2^(kLag + kUp), below fp16's 2^16.  They are exact to 2^-11 down to
// 2^-21 of the largest one, 0 below 2^-32; that of the only token of a row, or of the largest of a block
// alone, is exact.
constexpr float kUp = 7.f;
constexpr float kLeastScale = 1e-37f;  // value scales below are 0: 1 over them has to be finite
// Places on the line: a key of a row block with two tiles of rows, of one with one tile, and the
// beginning and end of a row block.  (An end at 1,536: two parts among 24 decoded tokens 232 us instead
// of 221, 512 behind 7,680 55.5 instead of 53.4; one-tile keys at 5: four drafted tokens 19.0 for 17.9.)
constexpr uint64_t kPairKey = 8, kOneKey = 6, kEdge = 4096;
constexpr uint64_t kLeast = 1280;  // places of a run at least (at 4,096 four drafted tokens: 29.6 us)
// Scores that may be above this (in powers of two) are rounded before the maximum is taken from them,
// as where some are hidden: a product that is not is off the rounded maximum by 2^-24 of itself.
constexpr float kFar = 1048576.f;
// Limits of waits in clocks: two seconds for what is at most a few steps away; what may be a whole
// item away has ten times what the steps of the longest one take.
constexpr long long kPatience = 4000000000, kStepClocks = 20000;
constexpr long long kItemPatience = kPatience + ((1ll << 32) / kKeys) * kStepClocks;
constexpr uint32_t kSoftmaxWarps = 8, kWidenWarps = 4;
constexpr uint32_t kThreads = (kSoftmaxWarps + kWidenWarps + 4) * 32;
constexpr uint32_t kProducts = 12, kPlan = 13, kPages = 14, kValues = 15;  // warps with one role each
// Registers: the launch has kThreads * kLaunchRegs, which the warps share out.
constexpr int kLaunchRegs = 128, kSoftmaxRegs = 200, kWidenRegs = 56, kOtherRegs = 56;
static_assert(256 * kSoftmaxRegs + 128 * kWidenRegs + 128 * kOtherRegs <= kThreads * kLaunchRegs,
              "register split");
template <int kDim>
constexpr uint32_t kStages = kDim == 128 ? 3 : 6;  // fp16 tiles in the ring, 32 or 16 KB each
// Key tiles whose codes are on their way or there, 32 or 16 KB each.
template <int kDim>
constexpr uint32_t kDeep = kDim == 128 ? 2 : 4;
constexpr uint32_t kBatchTiles = 4, kBatches = 3;  // table entries and scales read ahead
constexpr uint32_t kItems = 4;                     // items planned ahead

struct Cut;

struct ChunkArgs {
  KvArgs kv;
  const unsigned char* q;
  unsigned char* out;
  uint64_t q_stride, out_stride, rows;
  const uint64_t* off;
  const uint32_t* len;
  const int32_t* table;
  uint32_t heads, group, n_seqs, width;
  uint32_t slope;  // of the line, see Shape
  float scale2;    // scale * log2(e)
  float* lse;
  float* part_o;   // [kCtas][2][kDim / 4][slot_rows][4], over a power of two, see over_power
  float2* part_ml; // [kCtas][2][slot_rows]: a row's maximum and sum
  Cut* cuts;       // [kCtas]
  uint32_t slot_rows;
  int* status;
};

// A wait of a limited time; once one has run out for a thread of the block, nobody waits any longer
// and the block runs to its end.
template <long long kLimit = kPatience>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* late) {
  if (try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!try_wait(bar, parity)) {
    if (*late) return false;
    if (clock64() - t0 > kLimit) {
      *late = 1;
      return false;
    }
  }
  return true;
}
// Whether a thread of the block has given up, by the whole warp: its threads go the same way.
__device__ __forceinline__ bool given_up(volatile int* late) { return __any_sync(~0u, *late); }

// ---- the line
// A sequence of the call: its rows and tokens.
struct Seq {
  uint64_t first, new_tokens;
  uint32_t tokens;
};
__device__ __forceinline__ Seq seq_of(const ChunkArgs& a, uint32_t i) {
  const RowRange r = row_range(a.off, i, a.rows);
  return {r.first, r.count,
          (uint32_t)min((uint64_t)a.len[i], (uint64_t)a.width * kBlockTokens)};
}
// x / y for y below 2^16, a digit of 16 bits at a time (a 64-bit division is a hundred instructions).
__device__ __forceinline__ uint64_t divide(uint64_t x, uint32_t y) {
  if (!(x >> 32)) return (uint32_t)x / y;
  uint64_t q = 0;
  uint32_t r = 0;
#pragma unroll 1
  for (int i = 48; i >= 0; i -= 16) {
    const uint32_t d = r << 16 | (uint32_t)(x >> i & 0xffff);
    q = q << 16 | d / y;
    r = d % y;
  }
  return q;
}
// Row blocks of a sequence and KV head, and the places that they take: block b has kEdge and about the
// keys that its last row sees, the last one all the sequence's keys.  Any rising line would do: a
// run's ends are found in it the same way from both sides.
struct Shape {
  uint32_t blocks, one;  // whether the last row block has one tile of rows
  uint64_t before;       // places of the keys before the new tokens
  uint64_t slope, last;  // places that a row block has more than the one before, times 32; of the last
  __device__ __forceinline__ Shape(const Seq& s, const ChunkArgs& a) {
    const uint64_t rows = s.new_tokens * a.group;
    blocks = (uint32_t)((rows + 2 * kRows - 1) / (2 * kRows));
    before = s.tokens > s.new_tokens ? (s.tokens - s.new_tokens) * kPairKey : 0;
    slope = a.slope;
    one = blocks && rows - (uint64_t)(blocks - 1) * (2 * kRows) <= kRows;
    last = blocks ? kEdge + s.tokens * (one ? kOneKey : kPairKey) : 0;
  }
  // places before block b < blocks
  __device__ __forceinline__ uint64_t upto(uint32_t b) const {
    return b * (kEdge + before) + (slope * ((uint64_t)b * (b + 1)) >> 5);
  }
  __device__ __forceinline__ uint64_t all() const { return blocks ? upto(blocks - 1) + last : 0; }
  __device__ __forceinline__ uint64_t of(uint32_t b) const {
    return b + 1 == blocks ? last : upto(b + 1) - upto(b);
  }
};

// Equal parts of the line.
struct Runs {
  uint64_t total, base;
  uint32_t count, rest;
  __device__ __forceinline__ explicit Runs(uint64_t t) {
    total = t;
    count = (uint32_t)max((uint64_t)1, min((uint64_t)kCtas, t / kLeast));
    base = divide(t, count);
    rest = (uint32_t)(t - base * count);
  }
  __device__ __forceinline__ uint64_t start(uint32_t c) const { return base * c + min(c, rest); }
  // the run that has place p < total
  __device__ __forceinline__ uint32_t at(uint64_t p) const {
    uint32_t lo = 0, hi = count;
#pragma unroll 1
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (start(mid) <= p) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

// What a block works on: key tiles [first, first + steps) of a row block.
struct Item {
  uint64_t row;       // of queries: the row block's first token
  int64_t sees;       // tokens that the first token sees; each later one sees one more
  uint32_t seq, kv_head;
  uint32_t lead;      // heads of the first token that are another row block's
  uint32_t rows;      // 1 .. 256
  uint32_t tokens;    // of the sequence
  uint32_t first, steps;  // of an item that is sent on, steps >= 1
  int32_t slot;       // of the workspace; -1: the row block is all this item's
  int32_t valid;      // 0: no more items
};

// A run's beginning inside a row block, for the join: it has parts of the runs run0, run0 + 1, ...; of
// run0 it is the first row block (second = 0) or a later one; `order` numbers its cuts.
struct Cut {
  uint64_t row;
  uint32_t kv_head, lead, rows;
  uint32_t parts, run0, second, order;
};

// Pages and scales of a batch of key tiles' blocks.
struct Batch {
  int32_t page[kBatchTiles * kTileBlocks];  // -1: absent
  alignas(16) float k_scale[kBatchTiles * kTileBlocks], v_scale[kBatchTiles * kTileBlocks];
  uint32_t absent;  // blocks without a page, or past the sequence's end; a bit each
};

template <int kDim>
struct Shared {
  alignas(1024) unsigned char q[2][kRows * kDim * 2];
  alignas(1024) unsigned char kv[kStages<kDim>][kKeys * kDim * 2];
  alignas(1024) unsigned char codes[2 * kDeep<kDim>][kKeys * kDim];  // keys', values'
  alignas(16) Batch batch[kBatches];
  alignas(8) uint64_t q_full[2], kv_full[kStages<kDim>], kv_empty[kStages<kDim>];
  uint64_t codes_full[2 * kDeep<kDim>], codes_empty[2 * kDeep<kDim>];
  uint64_t s_full[2], p_full[2][2], o_full[2];  // p: the two halves of the keys
  uint64_t item_full[kItems], item_empty[kItems], batch_full[kBatches], batch_empty[kBatches], met;
  Item item[kItems];
  uint64_t sums[kThreads / 32];
  uint32_t tmem;
  int late;
};

// Places in shared memory, from the address of its beginning in a register: an address taken anew
// costs three instructions.
#define AT(x) (sb + (uint32_t)(reinterpret_cast<const char*>(&(sh.x)) - reinterpret_cast<const char*>(&sh)))

// The items of a block, as its warps read them: places that the planning warp fills.
struct Items {
  uint32_t n = 0;
  template <class Sh>
  __device__ __forceinline__ Item next(Sh& sh, uint32_t sb, volatile int* late) {
    const uint32_t at = n % kItems;
    wait<kItemPatience>(AT(item_full[at]), n / kItems & 1, late);
    Item x = sh.item[at];
    ++n;
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(AT(item_empty[at]));
    if (given_up(late)) x.valid = 0;
    return x;
  }
  // The item where it is, kept until done(); null: no more.
  template <class Sh>
  __device__ __forceinline__ const Item* see(Sh& sh, uint32_t sb, volatile int* late) {
    wait<kItemPatience>(AT(item_full[n % kItems]), n / kItems & 1, late);
    const Item* x = &sh.item[n % kItems];
    return __any_sync(~0u, !x->valid) || given_up(late) ? nullptr : x;
  }
  template <class Sh>
  __device__ __forceinline__ void done(Sh& sh, uint32_t sb) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(AT(item_empty[n % kItems]));
    ++n;
  }
};

// A warp's view of the batches: those it has seen filled, and those it has given back.
struct Batches {
  uint32_t seen = 0, given = 0, base = 0;
  template <class Sh>
  __device__ __forceinline__ void see(Sh& sh, uint32_t sb, uint32_t upto, volatile int* late) {
    for (; seen < upto; ++seen)
      wait(AT(batch_full[seen % kBatches]), seen / kBatches & 1, late);
  }
  template <class Sh>
  __device__ __forceinline__ const Batch& get(Sh& sh, uint32_t sb, uint32_t tile, volatile int* late) {
    see(sh, sb, base + tile / kBatchTiles + 1, late);
    return sh.batch[(base + tile / kBatchTiles) % kBatches];
  }
  // back to the pages' warp: what comes before tile `next` of n
  template <class Sh>
  __device__ __forceinline__ void give(Sh& sh, uint32_t sb, uint32_t next, uint32_t n, volatile int* late) {
    const uint32_t upto = base + (next < n ? next / kBatchTiles : (n + kBatchTiles - 1) / kBatchTiles);
    if (given == upto) return;
    see(sh, sb, upto, late);
    __syncwarp();
    for (; given < upto; ++given)
      if ((threadIdx.x & 31) == 0) bar_arrive(AT(batch_empty[given % kBatches]));
  }
  __device__ __forceinline__ void end(uint32_t n) { base += (n + kBatchTiles - 1) / kBatchTiles; }
};

__device__ __forceinline__ uint64_t shfl64(uint64_t x, int from) {
  return (uint64_t)__shfl_sync(~0u, (uint32_t)(x >> 32), from) << 32 |
         __shfl_sync(~0u, (uint32_t)x, from);
}

// Sequences that a warp adds up the places of: whole windows of 32.
__device__ __forceinline__ uint32_t share_of(uint32_t n_seqs) {
  constexpr uint32_t kWarps = kThreads / 32;
  return (n_seqs + kWarps * 32 - 1) / (kWarps * 32) * 32;
}

// Rows that see no key, or a run's part of a row block without any: 0 and -inf.  Such items go no
// further: the warps that look ahead wait for items with keys only, of which kItems are enough.
template <int kDim>
__device__ __forceinline__ void nothing_seen(const ChunkArgs& a, const Item& x) {
#pragma unroll 1
  for (uint32_t r = threadIdx.x & 31; r < x.rows; r += 32) {
    if (x.slot >= 0) {
      a.part_ml[(uint64_t)x.slot * a.slot_rows + r] = make_float2(-INFINITY, 0.f);
      continue;
    }
    const uint64_t row = x.row + (x.lead + r) / a.group;
    const uint32_t head = x.kv_head * a.group + (x.lead + r) % a.group;
    uint4* to = reinterpret_cast<uint4*>(a.out + (row * a.out_stride + (uint64_t)head * kDim) * 2);
#pragma unroll 1
    for (uint32_t i = 0; i < kDim / 8; ++i) to[i] = make_uint4(0, 0, 0, 0);
    if (a.lse) a.lse[row * a.heads + head] = -INFINITY;
  }
}

// ---- the planning warp: the run's items one after another
template <int kDim, class Sh>
__device__ __forceinline__ void plan(const ChunkArgs& a, Sh& sh, uint32_t sb, volatile int* late) {
  const uint32_t lane = threadIdx.x & 31;
  uint64_t total = 0;
  for (uint32_t w = 0; w < kThreads / 32; ++w) total += sh.sums[w];
  const Runs runs(total);
  const uint32_t run = blockIdx.x;
  uint64_t at = total ? runs.start(min(run, runs.count)) : 0;
  const uint64_t end = total && run < runs.count ? runs.start(run + 1) : at;
  if (lane == 0) a.cuts[run].parts = 0;
  // a window of 32 sequences, a lane each
  uint32_t base = 0, seq = 0;
  Seq mine = {0, 0, 0};
  auto window = [&](uint32_t from) {
    base = from;
    mine = from + lane < a.n_seqs ? seq_of(a, from + lane) : Seq{0, 0, 0};
  };
  auto pick = [&](uint32_t i) -> Seq {
    const int j = (int)(i - base);
    return {shfl64(mine.first, j), shfl64(mine.new_tokens, j), __shfl_sync(~0u, mine.tokens, j)};
  };
  uint32_t n = 0;
  auto publish = [&](const Item& x) {
    const bool ok = n < kItems ||
                    wait<kItemPatience>(AT(item_empty[n % kItems]), (n / kItems - 1) & 1, late);
    if (!__all_sync(~0u, ok)) return;  // the item there may be in use; nobody asks for another
    if (lane == 0) {
      sh.item[n % kItems] = x;
      bar_arrive(AT(item_full[n % kItems]));
    }
    __syncwarp();
    ++n;
  };
  Item x = {};
  // the sequence that has place `at`
  uint64_t before = 0, into = 0;
  bool found = false;
  if (at < end) {
    uint32_t share = 0;  // the warp that has counted it
    while (share + 1 < kThreads / 32 && at >= before + sh.sums[share]) before += sh.sums[share++];
    for (uint32_t from = share * share_of(a.n_seqs); from < a.n_seqs; from += 32) {
      window(from);
      const uint64_t c = Shape(mine, a).all() * a.kv.heads;
      uint64_t upto = c;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const uint64_t y = (uint64_t)__shfl_up_sync(~0u, (uint32_t)(upto >> 32), d) << 32 |
                           __shfl_up_sync(~0u, (uint32_t)upto, d);
        if (lane >= (uint32_t)d) upto += y;
      }
      const uint32_t hit = __ballot_sync(~0u, at < before + upto);
      if (hit) {
        const int who = __ffs(hit) - 1;
        seq = from + who;
        into = at - before - shfl64(upto - c, who);
        found = true;
        break;
      }
      before += shfl64(upto, 31);
    }
  }
  if (found) {  // (not with lengths that change under the call)
    Seq s = pick(seq);
    Shape shape(s, a);
    uint32_t kv_head = 0;
    uint32_t b = 0;
    {
      const uint64_t all = shape.all();
      uint32_t to = a.kv.heads;
#pragma unroll 1
      while (to - kv_head > 1) {
        const uint32_t mid = (kv_head + to) / 2;
        if (mid * all <= into) kv_head = mid;
        else to = mid;
      }
      into -= kv_head * all;
      b = shape.blocks - 1;
      if (into < shape.upto(b)) {
        uint32_t lo = 0, hi = b;  // upto(lo) <= into < upto(hi)
#pragma unroll 1
        while (hi - lo > 1) {
          const uint32_t mid = (lo + hi) / 2;
          if (shape.upto(mid) <= into) lo = mid;
          else hi = mid;
        }
        b = lo;
      }
      into -= shape.upto(b);
    }
    bool first = true;
    while (at < end && !given_up(late)) {
      const uint64_t places = shape.of(b), upto = min(places, into + (end - at));
      const uint64_t row0 = (uint64_t)b * (2 * kRows);
      x.rows = (uint32_t)min((uint64_t)(2 * kRows), s.new_tokens * a.group - row0);
      const uint64_t token = divide(row0, a.group);
      x.lead = (uint32_t)(row0 - token * a.group);
      x.row = s.first + token;
      x.sees = (int64_t)s.tokens - (int64_t)s.new_tokens + (int64_t)token + 1;
      x.seq = seq;
      x.kv_head = kv_head;
      x.tokens = s.tokens;
      const int64_t most = x.sees + (x.lead + x.rows - 1) / a.group;  // of the last row
      const uint64_t tiles = most > 0 ? ((uint64_t)most + kKeys - 1) / kKeys : 0;
      const bool one = shape.one && b + 1 == shape.blocks;
      auto step = [&](uint64_t p) -> uint64_t {
        if (p == places) return tiles;
        return p <= kEdge ? 0 : min(tiles, one ? (p - kEdge) / (kOneKey * kKeys) : (p - kEdge) / (kPairKey * kKeys));
      };
      x.first = (uint32_t)step(into);
      x.steps = (uint32_t)step(upto) - x.first;
      const bool whole = into == 0 && upto == places;
      x.slot = whole ? -1 : (int32_t)(run * 2 + (first ? 0 : 1));
      x.valid = 1;
      if (into && lane == 0) {
        const uint64_t begin = at - into;
        const uint32_t run0 = runs.at(begin);
        a.cuts[run] = {x.row, kv_head, x.lead, x.rows, runs.at(begin + places - 1) - run0 + 1, run0,
                       runs.start(run0) < begin, run - run0 - 1};
      }
      if (x.steps) publish(x);
      else nothing_seen<kDim>(a, x);
      first = false;
      at += upto - into;
      into = 0;
      if (++b < shape.blocks) continue;
      b = 0;
      if (++kv_head < a.kv.heads) continue;
      kv_head = 0;
      // the next sequence with rows, a window at a time: of a pool's slots few may have some.  (One by
      // one, and by runs that had ended too, four tokens of two of 4,096 sequences took 311 us; now 47,
      // and 21 where they are neighbours.)
      if (at >= end) break;
      uint32_t later = seq + 1 - base < 32 ? ~0u << (seq + 1 - base) : 0u, hit;
      while (!(hit = __ballot_sync(~0u, mine.new_tokens != 0) & later) && base + 32 < a.n_seqs) {
        window(base + 32);
        later = ~0u;
      }
      if (!hit) break;
      seq = base + __ffs(hit) - 1;
      s = pick(seq);
      shape = Shape(s, a);
    }
  }
  x.valid = 0;
  publish(x);
}

__device__ __forceinline__ uint4 load_shared(uint32_t at) {
  uint4 x;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
               : "r"(at)
               : "memory");
  return x;
}
__device__ __forceinline__ void store_shared(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}

// A key tile's codes, keys' (z = 0) or values', into their place once the widening warps have left it:
// a copy each block, by 8 lanes, and zeros for blocks without a page.  A copy takes its warp 80 clocks
// to issue, so keys and values have a warp each.
template <int kDim, uint32_t z, class Sh>
__device__ __forceinline__ bool copy_tile(const ChunkArgs& a, Sh& sh, uint32_t sb, uint32_t tile, bool mine,
                                          int32_t page, uint32_t kv_head, volatile int* late) {
  constexpr uint32_t kPart = kBlockTokens * kDim, kRing = kDeep<kDim>;
  const uint32_t lane = threadIdx.x & 31, st = tile % kRing + z * kRing, bar = AT(codes_full[st]);
  const bool ok = tile < kRing || wait(AT(codes_empty[st]), (tile / kRing - 1) & 1, late);
  if (!__all_sync(~0u, ok)) return false;
  const uint32_t at = AT(codes[st]) + lane % kTileBlocks * kPart;
  const uint32_t bytes = __popc(__ballot_sync(~0u, mine && page >= 0)) * kPart;
  if (bytes < kTileBlocks * kPart) {
    if (mine && page < 0)
      for (uint32_t i = 0; i < kPart; i += 16) store_shared(at + i, 0, 0, 0, 0);
    __syncwarp();
  }
  if (lane == 0) bar_expect(bar, bytes);
  __syncwarp();
  if (mine && page >= 0)
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, "
        "[%3];" ::"r"(at),
        "l"((z ? a.kv.v : a.kv.k) + ((uint64_t)page * a.kv.heads + kv_head) * kPart), "r"(kPart), "r"(bar)
        : "memory");
  __syncwarp();
  return true;
}

// ---- the pages' warp: table entries and scales, a batch of key tiles at a time, a lane each block, and
// the keys' codes.  Entries are read two batches ahead and scales one, over the ends of items too.
template <int kDim, class Sh>
__device__ __forceinline__ void read_pages(const ChunkArgs& a, Sh& sh, uint32_t sb, volatile int* late) {
  const uint32_t lane = threadIdx.x & 31;
  struct Next {
    uint32_t tiles, kv_head;  // key tiles of the batch, 0: no more
    int32_t page;
    bool in;
    float2 scale;
  };
  Items items;
  Item x = {};
  uint32_t at = 0;  // key tiles of the item that batches have
  bool over = false;
  auto take = [&]() -> Next {
    while (!over && at >= x.steps) {
      x = items.next(sh, sb, late);
      over = !x.valid;
      at = 0;
    }
    Next b = {0, x.kv_head, -1, false, make_float2(0.f, 0.f)};
    if (over) return b;
    b.tiles = min(kBatchTiles, x.steps - at);
    const uint32_t block = (x.first + at) * kTileBlocks + lane;
    b.in = lane < b.tiles * kTileBlocks && (uint64_t)block * kBlockTokens < x.tokens;
    if (b.in) b.page = a.table[(uint64_t)x.seq * a.width + block];
    at += b.tiles;
    return b;
  };
  bool begun = false;
  auto scales = [&](Next& b) {
    if (!b.in) return;
    if (b.page < 0 || (uint32_t)b.page >= a.kv.n_pages) {
      flag_status(a.status, NETKV_DEV_ERANGE);
      b.page = -1;
      return;
    }
    const uint64_t part = (uint64_t)b.page * a.kv.heads + b.kv_head;
    b.scale = make_float2(a.kv.k_scale[part], a.kv.v_scale[part]);
    if (!begun) return;  // the first are copied at once
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.kv.k + part * (kBlockTokens * kDim)),
                 "n"(kBlockTokens * kDim)
                 : "memory");
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.kv.v + part * (kBlockTokens * kDim)),
                 "n"(kBlockTokens * kDim)
                 : "memory");
  };
  uint32_t tile = 0;
  Next b0 = take(), b1 = take();
  scales(b0);
  begun = true;
  for (uint32_t n = 0; b0.tiles; ++n) {
    Next b2 = {};
    if (n) {
      scales(b1);
      b2 = take();
    }
    Batch& to = sh.batch[n % kBatches];
    if (n >= kBatches) wait(AT(batch_empty[n % kBatches]), (n / kBatches - 1) & 1, late);
    to.page[lane] = b0.page;
    to.k_scale[lane] = b0.scale.x;
    to.v_scale[lane] = b0.scale.y;
    const uint32_t absent = __ballot_sync(~0u, b0.page < 0);
    if (lane == 0) to.absent = absent;
    __syncwarp();
    if (lane == 0) bar_arrive(AT(batch_full[n % kBatches]));
    for (uint32_t q = 0; q < b0.tiles; ++q) {
      if (!copy_tile<kDim, 0>(a, sh, sb, tile++, lane / kTileBlocks == q, b0.page, b0.kv_head, late))
        return;
      if (n == 0 && q + 1 == min(b0.tiles, kDeep<kDim>)) {  // the first batch before all else
        scales(b1);
        b2 = take();
      }
    }
    b0 = b1;
    b1 = b2;
  }
}

// ---- the values' warp: their codes
template <int kDim, class Sh>
__device__ __forceinline__ void copy_values(const ChunkArgs& a, Sh& sh, uint32_t sb, volatile int* late) {
  const uint32_t lane = threadIdx.x & 31;
  Items items;
  Batches batches;
  uint32_t count = 0;
  while (true) {
    const Item x = items.next(sh, sb, late);
    if (!x.valid) break;
    for (uint32_t from = 0; from < x.steps; from += kBatchTiles) {
      const int32_t page = batches.get(sh, sb, from, late).page[lane];
      if (given_up(late)) return;  // it may not be a page
      batches.give(sh, sb, from + kBatchTiles, x.steps, late);
      for (uint32_t q = 0; q < min(kBatchTiles, x.steps - from); ++q)
        if (!copy_tile<kDim, 1>(a, sh, sb, count++, lane / kTileBlocks == q, page, x.kv_head, late))
          return;
    }
    batches.end(x.steps);
  }
}

// ---- the widening warps: codes of two of a key tile's blocks each, to fp16 in the ring.  A lane has
// 16 codes of a row at a time; 8 lanes have the halves of two rows such that their loads and their
// stores of 16 bytes are in all banks.
template <int kDim, bool kE4m3, class Sh>
__device__ __forceinline__ void widen_tiles(Sh& sh, uint32_t sb, volatile int* late) {
  constexpr uint32_t kRing = kStages<kDim>, kLoads = 2 * kDim / 32, kBox = kKeys * 128;
  constexpr uint32_t kCodes = kDeep<kDim>, kTile = kKeys * kDim * 2;
  const uint32_t lane = threadIdx.x & 31, w = threadIdx.x / 32 - kSoftmaxWarps;
  // A lane's load i: row 8 * (i / 2) + row0 of the warp's 32, half (i + odd) % 2 (of 64: row 8 i + row0)
  const uint32_t row0 = kDim == 128 ? lane / 8 * 2 + lane / 4 % 2 : lane / 4;
  const uint32_t odd = kDim == 128 ? lane / 4 % 2 : 0;
  const uint32_t src0 = AT(codes[0]) + (w * 32 + row0) * kDim + lane % 4 * 16;
  const uint32_t dst0 = AT(kv[0]) + (w * 32 + row0) * 128;
  const uint32_t at0 = ((lane % 4 * 2) ^ (row0 & 7)) * 16, at1 = at0 ^ 16;
  Items items;
  uint32_t n = 0, tiles = 0;  // tiles of the ring; key tiles of the items before
  while (true) {
    const Item* item = items.see(sh, sb, late);
    if (!item) break;
    const uint32_t steps = item->steps, first = item->first, tokens = item->tokens;
    // in the order in which the products want them: of two tiles of rows K 0, V 0, K 1, V 1, ...; of
    // one K 0, K 1, V 0, K 2, V 1, ...
    const uint32_t ahead = item->rows <= kRows ? 2 : 1;
    items.done(sh, sb);
#pragma unroll 1
    for (uint32_t p = 0; p < 2 * (steps + ahead); ++p) {
      const uint32_t z = p & 1 ? 0 : 1;  // values of an earlier tile, then keys
      const uint32_t tile = p / 2 - (z ? ahead : 0);
      if (tile >= steps) continue;
      const uint32_t cs = (tiles + tile) % kCodes + z * kCodes, st = n % kRing;
      wait(AT(codes_full[cs]), (tiles + tile) / kCodes & 1, late);
      const uint32_t src = src0 + cs * (kKeys * kDim);
      uint4 c[kLoads];
#pragma unroll
      for (uint32_t i = 0; i < kLoads; ++i)
        c[i] = load_shared(kDim == 128 ? src + (i % 2 ? 64 - odd * 64 : odd * 64) + i / 2 * 8 * kDim
                                       : src + i * 8 * kDim);
      // past the sequence's end are others' codes, and weights of 0 would not hide a NaN
      if (tile + 1 == steps) {
        const uint32_t key0 = (first + tile) * kKeys + w * 32;
        const uint32_t own = key0 < tokens ? tokens - key0 : 0;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i)
          if (row0 + (kDim == 128 ? i / 2 : i) * 8 >= own) c[i] = make_uint4(0, 0, 0, 0);
      }
      bool ok = n < kRing || wait(AT(kv_empty[st]), (n / kRing - 1) & 1, late);
      ++n;
      if (!__all_sync(~0u, ok)) break;
      const uint32_t dst = dst0 + st * kTile, dst_even = dst + odd * kBox, dst_odd = dst + (kBox - odd * kBox);
#pragma unroll
      for (uint32_t i = 0; i < kLoads; ++i) {
        const uint32_t to = kDim == 128 ? (i % 2 ? dst_odd : dst_even) + i / 2 * 1024 : dst + i * 1024;
        uint32_t h[8];
        widen<kE4m3>(c[i].x, &h[0], &h[1]);
        widen<kE4m3>(c[i].y, &h[2], &h[3]);
        widen<kE4m3>(c[i].z, &h[4], &h[5]);
        widen<kE4m3>(c[i].w, &h[6], &h[7]);
        store_shared(to + at0, h[0], h[1], h[2], h[3]);
        store_shared(to + at1, h[4], h[5], h[6], h[7]);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        bar_arrive(AT(kv_full[st]));
        bar_arrive(AT(codes_empty[cs]));
      }
    }
    tiles += steps;
  }
}

// ---- the products
template <int kDim, class Sh>
__device__ __forceinline__ void multiply(Sh& sh, uint32_t sb, volatile int* late) {
  constexpr uint32_t kRing = kStages<kDim>, kBox = 128 * 128, kS = 0, kO = 256;
  constexpr uint32_t kScores = product(false, false, kKeys), kSums = product(false, true, kDim);
  constexpr uint32_t kTile = kRows * kDim * 2 >> 4;  // of operands' addresses
  const bool leader = elect();
  const uint64_t q0 = operand(AT(q[0]), 16), k0 = operand(AT(kv[0]), 16),
                 v0 = operand(AT(kv[0]), kBox);
  auto scores = [&](uint32_t t, uint32_t st) {  // S_t from the ring's place st
    if (leader) {
#pragma unroll
      for (int x = 0; x < kDim / 16; ++x) {
        const uint32_t off = (x / 4 * kBox + x % 4 * 32) >> 4;
        mma_smem(kS + t * 128, q0 + t * kTile + off, k0 + st * kTile + off, kScores, x > 0);
      }
      commit(AT(s_full[t]));
    }
    __syncwarp();
  };
  auto signal = [&](uint32_t bar) {
    if (leader) commit(bar);
    __syncwarp();
  };
  uint32_t i = 0, with_q = 0, done0 = 0, done1 = 0;  // tiles of the ring, items, steps
  auto arrived = [&](uint32_t n) {
    wait(AT(kv_full[n % kRing]), (n / kRing) & 1, late);
    after_sync();
  };
  Items items;
  while (true) {
    const Item x = items.next(sh, sb, late);
    if (!x.valid) break;
    // Of two tiles of rows each key tile is both tiles' (a turn each), of one it is the even or the odd
    // one's.  The ring has K 0, V 0, K 1, V 1, ... or K 0, K 1, V 0, K 2, V 1, ...
    const uint32_t n = x.steps, turns = x.rows <= kRows ? n : 2 * n;
    const bool one = x.rows <= kRows;
    wait(AT(q_full[0]), with_q & 1, late);
    wait(AT(q_full[1]), with_q & 1, late);
    ++with_q;
#pragma unroll 1
    for (uint32_t u = 0; u < min(2u, turns) + turns; ++u) {
      const bool first = u < min(2u, turns);  // the first scores of each tile; then P V and the next scores
      const uint32_t w = first ? u : u - min(2u, turns), t = w & 1;
      const bool last = one || t;  // the turn after which key tiles are left
      const uint32_t v = i + (one ? w + min(w + 2, n) : w | 1);
      const uint32_t k = i + (first ? (one ? w : 0) : one ? 2 * w + 3 : (w | 1) + 1);
      const bool more = first || w + 2 < turns;
      if (!first) {
        if (one || t == 0) arrived(v);
        const uint32_t parity = (t ? done1++ : done0++) & 1;
#pragma unroll
        for (uint32_t half = 0; half < 2; ++half) {
          wait(AT(p_full[t][half]), parity, late);
          after_sync();
          if (leader) {
#pragma unroll
            for (uint32_t x = 0; x < kKeys / 32; ++x)
              mma_tmem(kO + t * kDim, kS + t * 128 + half * 32 + x * 8,
                       v0 + v % kRing * kTile + (half * (kKeys / 32) + x) * (2048 >> 4), kSums,
                       w >= 2 || half || x);
          }
          __syncwarp();
        }
        if (!more) signal(AT(o_full[t]));
        if (last) signal(AT(kv_empty[v % kRing]));
      }
      if (more) {
        if (one || t == 0) arrived(k);
        scores(t, k % kRing);
        if (last) signal(AT(kv_empty[k % kRing]));
      }
    }
    i += 2 * n;
  }
  // the last signals have to reach a block that is still there
  if (i >= 1) wait(smem_addr(&sh.kv_empty[(i - 1) % kRing]), ((i - 1) / kRing) & 1, late);
  if (i >= 2) wait(smem_addr(&sh.kv_empty[(i - 2) % kRing]), ((i - 2) / kRing) & 1, late);
}

// A part's sums go to the workspace over a power of two, the one above the sum of its weights: that sum
// is up to 2^15 times the row's tokens, and its product with a large value may pass fp32's range where
// their quotient does not.  The powers leave the bits of whatever is a normal number as they are.
__device__ __forceinline__ uint32_t power_of(float sum) {
  return min(max(__float_as_uint(sum) >> 23, 1u), 252u);
}
__device__ __forceinline__ float over_power(float sum) { return __uint_as_float((253 - power_of(sum)) << 23); }
__device__ __forceinline__ float times_power(float sum) { return __uint_as_float((power_of(sum) + 1) << 23); }

// ---- softmax: a thread has a row of its tile
template <int kDim, bool kBf16, bool kE4m3, class Sh>
__device__ __forceinline__ void softmax(const ChunkArgs& a, Sh& sh, uint32_t sb, volatile int* late) {
  constexpr uint32_t kS = 0, kO = 256, kBox = 128 * 128;
  constexpr float kTop = kE4m3 ? 448.f : 128.f;  // of the codes
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(~0u, tid / 32, 0);
  const uint32_t t = warp / 4, row = tid % kRows, lanes = (warp % 4) * 32 << 16;
  const uint32_t s_at = kS + t * 128 + lanes, o_at = kO + t * kDim + lanes;
  Items items;
  Batches batches;
  uint32_t taken = 0, finished = 0, meetings = 0;  // of the tile: steps, items with any; meetings
  auto meet = [&]() {
    __syncwarp();
    if (lane == 0) bar_arrive(AT(met));
    wait(AT(met), meetings++ & 1, late);
    __syncwarp();
  };
  while (true) {
    const Item* item = items.see(sh, sb, late);
    if (!item) break;
    const Item& x = *item;  // read where it is used: registers are for scores
    const bool one = x.rows <= kRows;
    const uint32_t mine = (one ? 0 : t * kRows) + row;  // the thread's row of the row block
    const bool real = mine < x.rows;
    const bool busy = __any_sync(~0u, real);
    float by = 0.f;  // what brings a sum of products to a score in powers of two, but for the scales
    float reach = 0.f;  // no score is above this times the scales
    // the row's queries as fp16, 16 bytes of row r in place (c ^ r) of 8
    if (busy) {
      const uint32_t token = (x.lead + mine) / a.group;
      const uint32_t head = x.kv_head * a.group + (x.lead + mine) % a.group;
      const uint4* from = reinterpret_cast<const uint4*>(
          a.q + ((x.row + token) * a.q_stride + (uint64_t)head * kDim) * 2);
      uint4 v[kDim / 8];
#pragma unroll
      for (int i = 0; i < kDim / 8; ++i) v[i] = real ? __ldcs(from + i) : make_uint4(0, 0, 0, 0);
      by = a.scale2;
      // magnitudes are in the order of their bits, two values a word
      uint32_t bits = 0;
#pragma unroll
      for (int i = 0; i < kDim / 8; ++i) {
        bits = __vimax3_u16x2(bits, v[i].x & 0x7fff7fffu, v[i].y & 0x7fff7fffu);
        bits = __vimax3_u16x2(bits, v[i].z & 0x7fff7fffu, v[i].w & 0x7fff7fffu);
      }
      const float largest = unpack16<kBf16>(max(bits & 0xffffu, bits >> 16)).x;
      // (rows of infinities are not others' concern)
      reach = largest <= 3.4028235e38f ? largest * by * (kDim * kTop) : 0.f;
      if constexpr (kBf16) {
        // 2^14 over the largest value's power of two, and the reverse; both are normal numbers
        const uint32_t e = max(__float_as_uint(largest) >> 23, 15u);
        const float inv = __uint_as_float((254 + 14 - e) << 23);
        by *= __uint_as_float((e - 14) << 23);
#pragma unroll
        for (int i = 0; i < kDim / 8; ++i) {
          uint32_t* w = reinterpret_cast<uint32_t*>(&v[i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 y = unpack16<true>(w[j]);
            w[j] = pack16<false>(y.x * inv, y.y * inv);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kDim / 8; ++i)
        *reinterpret_cast<uint4*>(sh.q[t] + i / 8 * kBox + row * 128 + ((i % 8) ^ (row & 7)) * 16) = v[i];
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    bar_arrive(AT(q_full[t]));
    // tokens that this row sees: of its key tiles all of the first `full`, and `rest` of the next
    const int64_t sees = (real ? x.sees + (x.lead + mine) / a.group : (int64_t)x.tokens) -
                         (int64_t)x.first * kKeys;
    const uint32_t full = sees < (int)kKeys ? 0 : (uint32_t)(sees / kKeys);
    const int rest = (int)max((int64_t)0, sees - (int64_t)full * kKeys);
    const uint32_t stride = one ? 2 : 1, own0 = one ? t : 0, steps = x.steps;
    float m = -INFINITY, l = 0.f;
    float unit = 0.f, over = 0.f;  // the largest value scale seen so far, and 1 over it
    bool any = false;
    for (uint32_t j = own0; j < steps; j += stride) {
      wait(AT(s_full[t]), taken++ & 1, late);
      after_sync();
      if (busy) {
        float s[kKeys];
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_load(s_at + i * 32, s + i * 32);
        const Batch& batch = batches.get(sh, sb, j, late);
        const uint32_t b0 = j % kBatchTiles * kTileBlocks;
        float k[kTileBlocks];
        *reinterpret_cast<float4*>(k) = *reinterpret_cast<const float4*>(batch.k_scale + b0);
        *reinterpret_cast<float4*>(k + 4) = *reinterpret_cast<const float4*>(batch.k_scale + b0 + 4);
        const float4* v = reinterpret_cast<const float4*>(batch.v_scale + b0);
        const uint32_t absent = batch.absent >> b0 & 0xff;
        const int seen = j < full ? kKeys : j == full ? rest : 0;
        float most = max3(max3(v[0].x, v[0].y, v[0].z), max3(v[0].w, v[1].x, v[1].y),
                          fmaxf(v[1].z, v[1].w));
        const float most_k = max3(max3(k[0], k[1], k[2]), max3(k[3], k[4], k[5]), fmaxf(k[6], k[7]));
        const bool masked = __any_sync(~0u, seen < (int)kKeys || reach * most_k > kFar) || absent;
#pragma unroll
        for (uint32_t b = 0; b < kTileBlocks; ++b) k[b] *= by;
        tmem_loaded();
        if (masked) {
#pragma unroll
          for (int i = 0; i < (int)kKeys; ++i)
            s[i] = i < seen && !(absent >> (i / 16) & 1) ? s[i] * k[i / 16] : -INFINITY;
#pragma unroll
          for (uint32_t b = 0; b < kTileBlocks; ++b) k[b] = 1.f;
          // of the blocks that the row sees: a later token's scale takes no bits from its weights
          if (seen < (int)kKeys) {
            const float* each = reinterpret_cast<const float*>(v);
            most = 0.f;
#pragma unroll
            for (int b = 0; b < (int)kTileBlocks; ++b) most = b * 16 < seen ? fmaxf(most, each[b]) : most;
          }
        }
        float top = m;
#pragma unroll
        for (uint32_t b = 0; b < kTileBlocks; ++b) {
          const float* y = s + b * 16;
          float u = max3(y[0], y[1], y[2]), w = max3(y[3], y[4], y[5]);
#pragma unroll
          for (int i = 6; i + 3 < 16; i += 4) {
            u = max3(u, y[i], y[i + 1]);
            w = max3(w, y[i + 2], y[i + 3]);
          }
          u = max3(u, y[14], y[15]);
          top = fmaxf(top, fmaxf(u, w) * k[b]);
        }
        const bool grown = most > unit;
        const bool follow = top - m > kLag;  // also the first maximum
        if (__any_sync(~0u, grown || follow)) {
          float to = 1.f;
          if (follow) {
            to = m == -INFINITY ? 0.f : ex2(m - top);
            m = top;
          }
          __syncwarp();
          l *= to;
          if (grown) {
            to *= any ? unit / most : 0.f;
            unit = most;
            over = most >= kLeastScale ? 1.f / most : 0.f;
          }
          if (any) {  // S_t is complete, and so is P_t V before it
#pragma unroll 1
            for (int i = 0; i < kDim / 16; ++i) {
              float o[16];
              tmem_load16(o_at + i * 16, o);
              tmem_loaded();
#pragma unroll
              for (int z = 0; z < 16; ++z) o[z] *= to;
              tmem_store16(o_at + i * 16, reinterpret_cast<const uint32_t*>(o));
            }
          }
        }
        any = true;
        const float base = m == -INFINITY ? 0.f : kUp - m;
        const uint64_t base_2 = pair(base, base);
        uint64_t sums_2[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t p[32];
          const float4 four = v[h];
          const float scale[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            // (at most 1, but of blocks that are not seen, whose weights of 0 should meet no infinity)
            const float g = __saturatef(scale[b] * over), f = k[h * 4 + b];
            const uint64_t f_2 = pair(f, f), g_2 = pair(g, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float* y = s + h * 64 + b * 16 + 2 * i;
              float u, w;
              split(fma2(pair(y[0], y[1]), f_2, base_2), &u, &w);
              const uint64_t e = pair(ex2(u), ex2(w));
              sums_2[i & 1] = add2(sums_2[i & 1], e);
              split(mul2(e, g_2), &u, &w);
              p[b * 8 + i] = pack16<false>(u, w);
            }
          }
          tmem_store(s_at + h * 32, p);
          tmem_stored();
          before_sync();
          bar_arrive(AT(p_full[t][h]));
        }
        float u, w;
        split(add2(sums_2[0], sums_2[1]), &u, &w);
        l += u + w;
      } else {
        before_sync();
        bar_arrive(AT(p_full[t][0]));
        bar_arrive(AT(p_full[t][1]));
      }
      batches.give(sh, sb, j + stride, steps, late);
    }
    batches.give(sh, sb, steps, steps, late);
    batches.end(steps);

    // ---- the row's output, or its part
    float w0 = 1.f, w1 = 0.f;  // what the two tiles' sums are multiplied by
    if (one) {
      if (steps > t) wait(AT(o_full[t]), finished++ & 1, late);
      // what a row's two threads have goes through their lane of TMEM, where the scores were
      float own[4] = {m, l, unit, 0.f}, other[4];
      after_sync();
      tmem_store4(s_at, reinterpret_cast<const uint32_t*>(own));
      tmem_stored();
      before_sync();
      meet();
      after_sync();
      tmem_load4(kS + (1 - t) * 128 + lanes, other);
      tmem_loaded();
      const float m0 = t ? other[0] : m, m1 = t ? m : other[0];
      m = fmaxf(m0, m1);
      w0 = m0 == -INFINITY ? 0.f : ex2(m0 - m);
      w1 = m1 == -INFINITY ? 0.f : ex2(m1 - m);
      // (a tile of NaN scores has no maximum, but its sum says so)
      l = w0 * (t ? other[1] : l) + w1 * (t ? l : other[1]);
      w0 *= t ? other[2] : unit;
      w1 *= t ? unit : other[2];
    } else {
      wait(AT(o_full[t]), finished++ & 1, late);
      after_sync();
      w0 = unit;
    }
    if (busy) {
      const uint32_t token = (x.lead + mine) / a.group;
      const uint32_t head = x.kv_head * a.group + (x.lead + mine) % a.group;
      const float inv = x.slot >= 0 ? over_power(l) : l == 0.f ? 1.f : 1.f / l;
      const bool none = l == 0.f;  // NaN is not
      w0 *= inv;
      w1 *= inv;
      // of one tile of rows each tile's warps write half the columns
      constexpr int kCols = 16;
      const uint32_t c0 = one ? t * (kDim / 2) : 0, c1 = one ? c0 + kDim / 2 : kDim;
#pragma unroll 1
      for (uint32_t c = c0; c < c1; c += kCols) {
        float o[kCols], y[kCols];
        tmem_load16(kO + lanes + (one ? 0 : t * kDim) + c, o);
        if (one && x.steps > 1) tmem_load16(kO + lanes + kDim + c, y);
        tmem_loaded();
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          o[i] = none ? 0.f : o[i] * w0;
          if (one && x.steps > 1) o[i] += none ? 0.f : y[i] * w1;
        }
        if (!real) {
        } else if (x.slot >= 0) {
          float4* to = reinterpret_cast<float4*>(a.part_o) +
                       ((uint64_t)x.slot * (kDim / 4) + c / 4) * a.slot_rows + mine;
#pragma unroll
          for (int i = 0; i < kCols / 4; ++i)
            to[i * a.slot_rows] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        } else {
          uint4* to = reinterpret_cast<uint4*>(
              a.out + ((x.row + token) * a.out_stride + (uint64_t)head * kDim + c) * 2);
#pragma unroll
          for (int i = 0; i < kCols / 8; ++i)
            to[i] = make_uint4(pack16<kBf16>(o[8 * i], o[8 * i + 1]), pack16<kBf16>(o[8 * i + 2], o[8 * i + 3]),
                               pack16<kBf16>(o[8 * i + 4], o[8 * i + 5]),
                               pack16<kBf16>(o[8 * i + 6], o[8 * i + 7]));
        }
        __syncwarp();
      }
      if (real && !(one && t)) {
        if (x.slot >= 0)
          a.part_ml[(uint64_t)x.slot * a.slot_rows + mine] = make_float2(m, l);
        else if (a.lse)
          a.lse[(x.row + token) * a.heads + head] = none ? -INFINITY : (m - kUp) * kLn2 + logf(l);
      }
      __syncwarp();
    }
    before_sync();
    if (one) meet();  // both tiles' sums have been read
    items.done(sh, sb);
  }
}

template <int kDim, bool kBf16, bool kE4m3>
__global__ void __launch_bounds__(kThreads, 1) chunk_kernel(const __grid_constant__ ChunkArgs a) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Shared<kDim>& sh = *reinterpret_cast<Shared<kDim>*>(smem);
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(~0u, tid / 32, 0);
  volatile int* late = &sh.late;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (warp == 0) {
    if (lane == 0) {
      sh.late = 0;
      for (uint32_t i = 0; i < kStages<kDim>; ++i) {
        bar_init(smem_addr(&sh.kv_full[i]), kWidenWarps);
        bar_init(smem_addr(&sh.kv_empty[i]), 1);
      }
      for (uint32_t i = 0; i < 2 * kDeep<kDim>; ++i) {
        bar_init(smem_addr(&sh.codes_full[i]), 1);
        bar_init(smem_addr(&sh.codes_empty[i]), kWidenWarps);
      }
      for (uint32_t i = 0; i < kBatches; ++i) {
        bar_init(smem_addr(&sh.batch_full[i]), 1);
        bar_init(smem_addr(&sh.batch_empty[i]), kSoftmaxWarps + 1);
      }
      for (uint32_t i = 0; i < kItems; ++i) {
        bar_init(smem_addr(&sh.item_full[i]), 1);
        bar_init(smem_addr(&sh.item_empty[i]), kSoftmaxWarps + kWidenWarps + 3);
      }
      for (int t = 0; t < 2; ++t) {
        bar_init(smem_addr(&sh.q_full[t]), kRows);
        bar_init(smem_addr(&sh.s_full[t]), 1);
        bar_init(smem_addr(&sh.p_full[t][0]), kRows);
        bar_init(smem_addr(&sh.p_full[t][1]), kRows);
        bar_init(smem_addr(&sh.o_full[t]), 1);
      }
      bar_init(smem_addr(&sh.met), kSoftmaxWarps);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
                     smem_addr(&sh.tmem))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    before_sync();
  }
  // the line's length, and what is wrong with the sequences, said by the first block
  // (a warp has neighbouring sequences, so that the plan finds its own among those of one warp)
  uint64_t sum = 0;
  const uint32_t each = share_of(a.n_seqs);
  for (uint32_t i = warp * each + lane; i < min(a.n_seqs, (warp + 1) * each); i += 32) {
    sum += Shape(seq_of(a, i), a).all();
    if (blockIdx.x == 0 && (row_range(a.off, i, a.rows).bad ||
                            a.len[i] > (uint64_t)a.width * kBlockTokens))
      flag_status(a.status, NETKV_DEV_ERANGE);
  }
  sum *= a.kv.heads;
#pragma unroll
  for (int d = 16; d; d /= 2)
    sum += (uint64_t)__shfl_xor_sync(~0u, (uint32_t)(sum >> 32), d) << 32 |
           __shfl_xor_sync(~0u, (uint32_t)sum, d);
  if (lane == 0) sh.sums[warp] = sum;
  __syncthreads();
  after_sync();
  uint32_t sb;
  asm volatile("mov.u32 %0, %1;" : "=r"(sb) : "r"(smem_addr(&sh)));
  if (warp >= kProducts) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kProducts) multiply<kDim>(sh, sb, late);
    else if (warp == kPlan) plan<kDim>(a, sh, sb, late);
    else if (warp == kPages) read_pages<kDim>(a, sh, sb, late);
    else if (warp == kValues) copy_values<kDim>(a, sh, sb, late);
  } else if (warp >= kSoftmaxWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kWidenRegs));
    widen_tiles<kDim, kE4m3>(sh, sb, late);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    softmax<kDim, kBf16, kE4m3>(a, sh, sb, late);
  }
  __syncthreads();
  if (warp == 0) {
    if (*late) {  // what is still in flight gets a moment to end
      const long long t0 = clock64();
      while (clock64() - t0 < 20000000ll) {
      }
    }
    __syncwarp();
    after_sync();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sh.tmem) : "memory");
    if (lane == 0 && *late) flag_status(a.status, NETKV_DEV_ETIMEOUT);
  }
}

// Joins the row blocks that runs share: a run's beginning inside one has blocks of threads for a share
// of its rows, a thread each row and 4 columns.
constexpr uint32_t kJoinThreads = 256, kJoinShares = 8;
static_assert(kCtas <= 256, "parts of a row block");
template <int kDim, bool kBf16>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ ChunkArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Cut c = a.cuts[blockIdx.x + 1];
  if (c.parts == 0) return;
  const uint32_t shares = (c.parts - 1) * kJoinShares;
  auto slot = [&](uint32_t i) { return (c.run0 + i) * 2 + (i == 0 ? c.second : 0); };
  for (uint32_t u = (c.order * kJoinShares + blockIdx.y) * kJoinThreads + threadIdx.x;
       u < c.rows * (kDim / 4); u += shares * kJoinThreads) {
    const uint32_t row = u % c.rows, col = u / c.rows;
    float top = -INFINITY, most = 0.f;
    for (uint32_t i = 0; i < c.parts; ++i) {
      const float2 ml = a.part_ml[(uint64_t)slot(i) * a.slot_rows + row];
      top = fmaxf(top, ml.x);
      most = fmaxf(most, ml.y);
    }
    // all parts over one power of two, 2^8 (they are fewer) above that of the largest
    const float over = over_power(most) * 0x1p-8f;
    float sum = 0.f, o[4] = {};
    for (uint32_t i = 0; i < c.parts; ++i) {
      const float2 ml = a.part_ml[(uint64_t)slot(i) * a.slot_rows + row];
      const float w = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
      sum += w * ml.y;
      if (ml.y == 0.f) continue;
      const float4 y = reinterpret_cast<const float4*>(
          a.part_o)[((uint64_t)slot(i) * (kDim / 4) + col) * a.slot_rows + row];
      const float by = w * (times_power(ml.y) * over);
      o[0] += by * y.x;
      o[1] += by * y.y;
      o[2] += by * y.z;
      o[3] += by * y.w;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum * (times_power(most) * 0x1p8f);
    const uint64_t to = c.row + (c.lead + row) / a.group;
    const uint32_t head = c.kv_head * a.group + (c.lead + row) % a.group;
    *reinterpret_cast<uint2*>(a.out + (to * a.out_stride + (uint64_t)head * kDim + col * 4) * 2) =
        make_uint2(pack16<kBf16>(o[0] * inv, o[1] * inv), pack16<kBf16>(o[2] * inv, o[3] * inv));
    if (col == 0 && a.lse)
      a.lse[to * a.heads + head] = sum == 0.f ? -INFINITY : (top - kUp) * kLn2 + logf(sum);
  }
}

bool sizes_ok(const netkv_kv_pages* pages, uint64_t rows, uint32_t n_seqs, uint32_t heads) {
  return kv_pages_ok(pages) && heads >= 1 && heads <= 65535 && heads % pages->kv_heads == 0 &&
         !(n_seqs >> 24) && !(rows >> 31);
}

struct Workspace {
  uint32_t slot_rows;
  size_t part_ml, cuts, total;  // part_o is at 0
};
Workspace workspace(const netkv_kv_pages* p, uint64_t rows, uint32_t heads) {
  auto up = [](size_t x) { return (x + 127) / 128 * 128; };
  Workspace w;
  // rows of a row block at most, in whole lines
  w.slot_rows = (uint32_t)up(min((uint64_t)(2 * kRows), max((uint64_t)1, rows * (heads / p->kv_heads))) * 16) / 16;
  w.part_ml = up((size_t)kCtas * 2 * w.slot_rows * p->head_dim * 4);
  w.cuts = w.part_ml + up((size_t)kCtas * 2 * w.slot_rows * sizeof(float2));
  w.total = w.cuts + up(kCtas * sizeof(Cut));
  return w;
}

}  // namespace

extern "C" size_t netkv_attn_chunk_workspace_size(const netkv_kv_pages* pages, uint64_t rows,
                                                  uint32_t n_seqs, uint32_t heads) {
  return sizes_ok(pages, rows, n_seqs, heads) ? workspace(pages, rows, heads).total : 0;
}

extern "C" netkv_status netkv_attn_chunk(const netkv_kv_pages* pages, uint32_t dtype,
                                         const void* d_q, uint64_t q_stride, uint32_t heads,
                                         uint32_t n_seqs, const uint64_t* d_off, uint64_t rows,
                                         const uint32_t* d_len, const int32_t* d_table,
                                         uint32_t table_width, float scale, void* d_out,
                                         uint64_t out_stride, float* d_lse, void* d_ws,
                                         size_t ws_bytes, int* d_status, netkv_stream_t stream) {
  if (!sizes_ok(pages, rows, n_seqs, heads) || dtype > NETKV_BF16 || table_width == 0 ||
      table_width >= (1u << 28) || !scale_ok(scale))
    return NETKV_EINVAL;
  if (n_seqs == 0 || rows == 0) return NETKV_OK;
  const uint64_t row = (uint64_t)heads * pages->head_dim;
  if (!rows_ok(d_q, q_stride, row) || !rows_ok(d_out, out_stride, row) || !d_off || !d_len ||
      !d_table || !d_ws || !aligned_to(d_off, 8) || !aligned_to(d_len, 4) ||
      !aligned_to(d_table, 4) || !aligned_to(d_lse, 4) || !aligned_to(d_ws, 16) ||
      !aligned_to(d_status, 4))
    return NETKV_EINVAL;
  const Workspace ws = workspace(pages, rows, heads);
  if (ws_bytes < ws.total) return NETKV_EINVAL;
  unsigned char* w = (unsigned char*)d_ws;
  const ChunkArgs a = {kv_args(pages),
                       (const unsigned char*)d_q,
                       (unsigned char*)d_out,
                       q_stride,
                       out_stride,
                       rows,
                       d_off,
                       d_len,
                       d_table,
                       heads,
                       heads / pages->kv_heads,
                       n_seqs,
                       table_width,
                       (uint32_t)(kPairKey * 2 * kRows * 16 / (heads / pages->kv_heads)),
                       scale * kLog2e,
                       d_lse,
                       (float*)w,
                       (float2*)(w + ws.part_ml),
                       (Cut*)(w + ws.cuts),
                       ws.slot_rows,
                       d_status};
  auto go = [&](auto dim, auto bf, auto e4) -> netkv_status {
    constexpr int kDim = decltype(dim)::value;
    constexpr bool kB = decltype(bf)::value, kE = decltype(e4)::value;
    constexpr auto kernel = chunk_kernel<kDim, kB, kE>;
    constexpr size_t bytes = sizeof(Shared<kDim>);
    static_assert(bytes <= 227 * 1024, "shared memory");
    // a launch with fewer registers than the warps share out would never end
    if (launch_registers<kernel>() < kLaunchRegs) return NETKV_ECUDA;
    NETKV_CUDA_TRY(allow_shared<kernel>((int)bytes));
    kernel<<<kCtas, kThreads, bytes, (cudaStream_t)stream>>>(a);
    if (netkv_launch_status() != NETKV_OK) return NETKV_ECUDA;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(kCtas - 1, kJoinShares);
    c.blockDim = dim3(kJoinThreads);
    c.stream = (cudaStream_t)stream;
    c.attrs = &early;
    c.numAttrs = 1;
    NETKV_CUDA_TRY(cudaLaunchKernelEx(&c, join_kernel<kDim, kB>, a));
    return netkv_launch_status();
  };
  auto types = [&](auto dim) {
    const bool bf = dtype == NETKV_BF16, e4 = pages->format == NETKV_KV_E4M3;
    if (bf && e4) return go(dim, std::true_type(), std::true_type());
    if (bf) return go(dim, std::true_type(), std::false_type());
    if (e4) return go(dim, std::false_type(), std::true_type());
    return go(dim, std::false_type(), std::false_type());
  };
  return pages->head_dim == 64 ? types(std::integral_constant<int, 64>())
                               : types(std::integral_constant<int, 128>());
}
