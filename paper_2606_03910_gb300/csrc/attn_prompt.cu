// Causal attention of packed prompts with grouped heads.
//
// Bound: 4 kDim flops a visible (query, key) pair on the tensor cores, 1,024 clocks for 128 x 128
// pairs at 128 wide; the exponentials, 512 clocks at 32 a clock and SM, come next and bind at 64
// wide.  One prompt of 32,768 tokens, 16 heads of 128: 2.57 ms, 1,710 TFLOP/s; ten ragged ones of
// 10,740 tokens in all: 68 us, 1,010; six behind cached prefixes, 8 heads of 64: 41 us, 590 (the
// longest row block's 41 key tiles are 21 steps in a row); one of 512: 10 us on the device.
//
// A block takes two tiles of 128 query rows that read the same keys: two heads of a group where
// the group is even, else two neighbouring row blocks of one head.  Where items are few it takes
// one row block twice, with the even and the odd key tiles, and adds the two up in shared memory:
// half the steps in a row (six behind prefixes 54 -> 40 us), at twice the reads of keys.
// Keys and values come in tiles of 128 rows by TMA, through a ring that serves both.  One thread
// issues the products,
//     S_t = Q_t K^T (fp32, in TMEM)   O_t += P_t V (P_t from TMEM, in S_t's place)
// so that one tile's products run while four warps take the other tile's softmax: a thread has
// a row, reads its 128 scores, and writes the weights back as 16-bit values, half of them first,
// on which their product can begin.  The products of one issuing thread complete in order, so S_t
// of the next keys may follow P_t V at once.  The issuing warp stays together and elects that
// thread: operands of a divergent thread go through vector registers, 70 clocks a product.
// One pass over the keys carries a row's maximum and sum (Milakov and Gimelshein, 2018).  The maximum
// is left behind until a score passes it by 2^8 (kLag): weights of up to 2^8 are as exact, and the
// output is then rescaled only a few times a row.
// Loads, products and softmax run on from one item to the next.  The grid has a block for each
// item; a running block takes over items of blocks that have not started (cluster launch control),
// one ahead, so that they end together (ten ragged prompts 82 -> 65 us with the order by steps).
#include <cuda.h>

#include "kv_common.cuh"

namespace {

constexpr int kRows = 128, kKeys = 128;  // of a tile
// Items an SM, in halves, up to which a row block's key tiles go to two tiles: at 3 a prompt of
// 4,096 tokens takes 58 us, 67 without; at 6 ten ragged ones would take 89 instead of 67.
constexpr uint32_t kFewItems = 6;
// Sequences up to which an item's row block is found by counting through them; above, a sequence and
// column has indices of the grid of its own, as many as the average has row blocks, which take its
// row blocks in turn: with each item counting, a call's time grows with the square of the sequences.
// 7 heads on 1 of 128: ragged prompts, 600 1,000 us by counting and 1,260 in turn, 1,024 1,460 and
// 1,550, 4,096 8,130 and 6,530; up to 200 rows each, 1,024 372 and 289, 4,096 2,730 and 1,130.
constexpr uint32_t kSearched = 1024;
constexpr float kLag = 8.f;              // in powers of two
// Where the weight of the running maximum stands, in powers of two.  fp16 ends at 2^16, so weights
// up to 2^kLag have room for 2^7, and are exact to 2^-11 down to 2^-21 of the largest one, 0 below
// 2^-32; at 1, keys 2^-25 below a sink of small values would leave the output and not its sum.
template <bool kBf16>
constexpr float kUp = kBf16 ? 0.f : 7.f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Limits of waits in clocks: two seconds for what is at most a few steps away.  What may be a whole
// item away (the next item, or a tile's scores where it has no rows in the item before) has ten times
// what the steps of the longest one take; that others wait for the steps of that item ends it too.
constexpr long long kPatience = 4000000000, kStepClocks = 20000;
constexpr long long kItemPatience = kPatience + ((1ll << 31) / kKeys) * kStepClocks;
constexpr int kSoftmaxWarps = 8;
constexpr int kThreads = (kSoftmaxWarps + 4) * 32;  // and a warp for the loads, one for the products
// Registers: the launch has kThreads * kLaunchRegs, of which the softmax warps, that hold a row
// of scores each thread, take more than the others.
constexpr int kLaunchRegs = 168, kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(256 * kSoftmaxRegs + 128 * kOtherRegs <= kThreads * kLaunchRegs, "register split");

// Two neighbouring row blocks of a head; two heads of a group; the even and the odd key tiles of
// one row block.
enum Mode : uint32_t { kRowPairs = 0, kHeadPairs = 1, kKeyHalves = 2 };

struct PromptArgs {
  unsigned char* out;
  uint64_t out_stride;  // in values
  const uint64_t* q_off;
  const uint64_t* k_off;
  uint64_t q_rows, k_rows;
  uint32_t heads, group, n_seqs;
  uint32_t mode;        // what a block's two tiles are
  uint32_t tiles;       // row blocks that the grid has
  uint32_t ordered;     // 1: row blocks by their key tiles, the most first
  uint32_t parts;       // many sequences: indices of the grid for each one and column; else 0
  float scale2;         // scale * log2(e)
  float* lse;
  int* status;
};

// (kept in order: the first half of a row's weights is wanted first)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two fp32 values in one operation
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ void split(uint64_t x, float* a, float* b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(x));
}
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(x), "l"(y), "l"(z));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(x), "l"(y));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
               : "memory");
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
// Waits for a phase, kPatience clocks at most; once one thread of the block has given up, nobody
// waits any longer and the block runs to its end.
template <long long kLimit = kPatience>
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, volatile int* late) {
  if (try_wait(bar, parity)) return;
  const long long t0 = clock64();
  while (!try_wait(bar, parity)) {
    if (*late) return;
    if (clock64() - t0 > kLimit) {
      *late = 1;
      return;
    }
  }
}

// Whether a thread of the block has, by the whole warp: its threads go the same way.  (The warp that
// issues products ends its item without asking, a vote a step cost 1 % of ten ragged prompts: its waits
// are over at once, and each of its signals is a phase's only one.)
__device__ __forceinline__ bool given_up(volatile int* late) {
  return __any_sync(~0u, *late);
}

__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, int z,
                                         uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], "
      "[%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

// Operands of 128-byte swizzled rows of 64 values.  Queries and keys (the inner dimension
// along a row): groups of 8 rows 1024 bytes apart.  Values (the inner dimension across rows):
// the same groups along the inner dimension, and 64 columns every 128 rows.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t columns_every) {
  return (uint64_t)((at & 0x3ffff) >> 4) | (uint64_t)(columns_every >> 4) << 16 |
         (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// fp32 sums of 128 rows by n columns
__device__ __forceinline__ constexpr uint32_t product(bool bf16, bool b_across, uint32_t n) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (b_across ? 1u << 16 : 0u) | (n >> 3) << 17 |
         (128u >> 4) << 24;
}
// Products and commits are issued by one thread (`leader`) of a warp whose threads stay together,
// so that operands are the warp's, not a thread's.
__device__ __forceinline__ bool elect() {
  uint32_t yes;
  asm volatile(
      "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(yes));
  return yes != 0;
}
__device__ __forceinline__ void mma_smem(uint32_t d, uint64_t a, uint64_t b, uint32_t what,
                                         bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(what), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t what,
                                         bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(what), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                   bar)
               : "memory");
}
__device__ __forceinline__ void after_sync() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void before_sync() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t at, float* x) {  // 32 columns of the warp's lanes
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, "
      "%8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, "
      "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]),
        "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, "
      "%8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, "
      "%24, %25, %26, %27, %28, %29, %30, %31};"
      :
      : "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
        "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]),
        "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t at, float* x) {
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, "
      "%8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]),
        "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at));
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, "
      "%8, %9, %10, %11, %12, %13, %14, %15};"
      :
      : "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
        "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_loaded() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_stored() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Tiles in the ring: 32 KB each at 128 wide, with 64 KB of queries and 32 KB for outputs.
template <int kDim>
constexpr int kStages = kDim == 128 ? 4 : 8;

// What a block works on: a row block of one sequence for a column (a pair of heads, or a head).
struct Item {
  uint64_t q_first, k_first;  // the sequence's rows
  uint32_t q_count, k_count;
  uint32_t row;     // the block's first row within the sequence
  uint32_t column;
  uint32_t steps[2];  // key tiles of each of the two tiles
  int32_t valid;      // 0: nothing to do; -1: no more items
};

template <int kDim>
struct Shared {
  alignas(1024) unsigned char q[2][kRows * kDim * 2];
  alignas(1024) unsigned char kv[kStages<kDim>][kKeys * kDim * 2];
  alignas(128) unsigned char out[kSoftmaxWarps][32 * 128];
  alignas(8) uint64_t q_full, q_empty, kv_full[kStages<kDim>], kv_empty[kStages<kDim>], landed;
  uint64_t s_full[2], p_full[2][2], o_full[2];  // p: the two halves of the keys
  uint64_t item_full[2], item_empty[2], begun, claimed, met;
  alignas(16) uint4 claim;
  Item item[2];
  float half_m[kRows], half_l[kRows];  // kKeyHalves: the odd key tiles' maxima and sums
  uint32_t tmem;
  int late;
};

// One of a block's two tiles: 128 rows of one head.
struct Tile {
  uint32_t head, rows;  // 0 .. 128 rows
  int32_t row;          // the first, within the sequence
};
__device__ __forceinline__ Tile tile_of(const PromptArgs& a, const Item& x, uint32_t t) {
  Tile y;
  y.head = a.mode == kHeadPairs ? x.column * 2 + t : x.column;
  y.row = (int32_t)(x.row + (a.mode == kRowPairs ? t * kRows : 0));
  y.rows = (uint32_t)min(kRows, max(0, (int32_t)x.q_count - y.row));
  return y;
}

// The n-th row block of all sequences: (sequence, block), sequence n_seqs where there is none.
// In the plain order the last blocks of a sequence, which see the most keys, come first.  In the
// ordered one the blocks come by their key tiles over all sequences, so that blocks of the grid
// that take one item after another end together: the number of row blocks with at least s key
// tiles is known for each sequence, and a search over s finds where the n-th stands.
__device__ __forceinline__ Found row_block(const PromptArgs& a, uint32_t n, uint32_t block_rows) {
  if (!a.ordered)
    return find_unit(a.n_seqs, a.tiles - 1 - n, [&](uint32_t i) {
      return (uint32_t)((row_range(a.q_off, i, a.q_rows).count + block_rows - 1) / block_rows);
    });
  const uint32_t lane = threadIdx.x & 31;
  uint32_t q[4], k[4], most = 0, all = 0;  // lane l has sequences 4 l .. 4 l + 3 of up to 128
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t i = lane * 4 + j;
    q[j] = i < a.n_seqs ? (uint32_t)row_range(a.q_off, i, a.q_rows).count : 0;
    k[j] = i < a.n_seqs ? (uint32_t)row_range(a.k_off, i, a.k_rows).count : 0;
    if (q[j]) most = max(most, (k[j] + kKeys - 1) / kKeys);
    all += (q[j] + block_rows - 1) / block_rows;
  }
  // row blocks of q rows and k keys with at least s key tiles
  auto least = [&](uint32_t q, uint32_t k, uint32_t s) -> uint32_t {
    const uint32_t blocks = (q + block_rows - 1) / block_rows;
    if (s == 0) return blocks;
    // rows up to a block's end that make it see key 128 (s - 1)
    const int64_t rows = (int64_t)(s - 1) * kKeys + 1 - k + q;
    if (rows > (int64_t)q) return 0;
    return rows <= 0 ? blocks : blocks + 1 - (uint32_t)((rows + block_rows - 1) / block_rows);
  };
  most = __reduce_max_sync(~0u, most);
  all = __reduce_add_sync(~0u, all);
  if (n >= all) return {a.n_seqs, 0};
  uint32_t lo = 0, hi = most + 1;  // more than n blocks have lo key tiles, not so hi
  while (hi - lo > 1) {
    const uint32_t s = (lo + hi) / 2;
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) c += least(q[j], k[j], s);
    if (__reduce_add_sync(~0u, c) > n) lo = s;
    else hi = s;
  }
  uint32_t above[4], sum = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) sum += above[j] = least(q[j], k[j], hi);
  n -= __reduce_add_sync(~0u, sum);
  const Found f = find_unit(a.n_seqs, n, [&](uint32_t i) {
    const uint32_t j = i % 4;  // the lane's own sequences
    const uint32_t qi = j == 0 ? q[0] : j == 1 ? q[1] : j == 2 ? q[2] : q[3];
    const uint32_t ki = j == 0 ? k[0] : j == 1 ? k[1] : j == 2 ? k[2] : k[3];
    return least(qi, ki, lo) - least(qi, ki, hi);
  });
  if (f.seq >= a.n_seqs) return f;
  const uint32_t at = f.seq % 4, from = f.seq / 4;
  const uint32_t qs = __shfl_sync(~0u, at == 0 ? q[0] : at == 1 ? q[1] : at == 2 ? q[2] : q[3], from);
  const uint32_t ks =
      __shfl_sync(~0u, at == 0 ? above[0] : at == 1 ? above[1] : at == 2 ? above[2] : above[3], from);
  return {f.seq, (qs + block_rows - 1) / block_rows - 1 - ks - f.unit};
}

// The grid's n-th item.  Of many sequences (a.parts) an index of the grid has every parts-th row block
// of a sequence, the last ones first: the one of turn `turn`, and whether there is another.
__device__ __forceinline__ Item item_at(const PromptArgs& a, uint32_t n, uint32_t turn, bool* more) {
  const uint32_t columns = a.mode == kHeadPairs ? a.heads / 2 : a.heads;
  const uint32_t block_rows = a.mode == kRowPairs ? 2 * kRows : kRows;
  Found f = {a.n_seqs, 0};
  *more = false;
  if (a.parts) {
    const uint32_t seq = n / columns / a.parts, unit = n / columns % a.parts + turn * a.parts;
    const uint32_t blocks =
        (uint32_t)((row_range(a.q_off, seq, a.q_rows).count + block_rows - 1) / block_rows);
    if (unit < blocks) f = {seq, blocks - 1 - unit};
    *more = unit + a.parts < blocks;
  } else {
    f = row_block(a, n / columns, block_rows);
  }
  Item x = {};
  if (f.seq >= a.n_seqs) return x;
  const RowRange q = row_range(a.q_off, f.seq, a.q_rows), k = row_range(a.k_off, f.seq, a.k_rows);
  x.q_first = q.first;
  x.k_first = k.first;
  x.q_count = (uint32_t)q.count;
  x.k_count = (uint32_t)k.count;
  x.row = f.unit * block_rows;
  x.column = n % columns;
  x.valid = 1;
#pragma unroll
  for (uint32_t t = 0; t < 2; ++t) {
    const Tile y = tile_of(a, x, t);
    // keys that the tile's last row sees
    const int64_t last = min((int64_t)x.k_count, (int64_t)x.k_count - x.q_count + y.row + y.rows);
    x.steps[t] = y.rows && last > 0 ? (uint32_t)((last + kKeys - 1) / kKeys) : 0;
  }
  if (a.mode == kKeyHalves) {
    x.steps[1] = x.steps[0] / 2;
    x.steps[0] -= x.steps[1];
  }
  return x;
}

// The items of a block, as its warps read them: two places, filled by the planning warp.
struct Items {
  uint32_t n = 0;
  template <class Sh>
  __device__ __forceinline__ Item next(Sh& sh, volatile int* late) {
    const uint32_t at = n % 2;
    wait<kItemPatience>(smem_addr(&sh.item_full[at]), n / 2 & 1, late);
    const Item x = sh.item[at];
    ++n;
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(smem_addr(&sh.item_empty[at]));
    if (given_up(late)) return Item{0, 0, 0, 0, 0, 0, {0, 0}, -1};
    return x;
  }
};

template <int kDim, bool kBf16>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ CUtensorMap map_q,
                  const __grid_constant__ CUtensorMap map_k,
                  const __grid_constant__ CUtensorMap map_v) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Shared<kDim>& sh = *reinterpret_cast<Shared<kDim>*>(smem);
  constexpr uint32_t kRing = kStages<kDim>;
  constexpr int kHalves = kDim / 64;
  constexpr uint32_t kBox = 128 * 128;  // bytes of 128 rows of 64 values
  // the whole of TMEM, from column 0: S of the two tiles, then their O
  constexpr uint32_t kS = 0, kO = 256;
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(~0u, tid / 32, 0);
  volatile int* late = &sh.late;

  if (warp == 0) {
    if (lane == 0) {
      sh.late = 0;
      bar_init(smem_addr(&sh.q_full), 1);
      bar_init(smem_addr(&sh.q_empty), 1);
      bar_init(smem_addr(&sh.landed), 1);
      bar_init(smem_addr(&sh.claimed), 1);
      bar_init(smem_addr(&sh.begun), 1);
      bar_init(smem_addr(&sh.met), kSoftmaxWarps);
      for (uint32_t i = 0; i < kRing; ++i) {
        bar_init(smem_addr(&sh.kv_full[i]), 1);
        bar_init(smem_addr(&sh.kv_empty[i]), 1);
      }
      for (int t = 0; t < 2; ++t) {
        bar_init(smem_addr(&sh.s_full[t]), 1);
        bar_init(smem_addr(&sh.p_full[t][0]), 128);
        bar_init(smem_addr(&sh.p_full[t][1]), 128);
        bar_init(smem_addr(&sh.o_full[t]), 1);
        bar_init(smem_addr(&sh.item_full[t]), 1);
        bar_init(smem_addr(&sh.item_empty[t]), kSoftmaxWarps + 2);
      }
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
                     smem_addr(&sh.tmem))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    before_sync();
  }
  __syncthreads();
  after_sync();
  Items items;

  if (warp >= kSoftmaxWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kSoftmaxWarps) {
      // ---- loads: of each item the queries, then K 0, V 0, K 1, V 1, ...
      uint32_t i = 0, cleared = 0, with_q = 0;
      while (true) {
        const Item x = items.next(sh, late);
        if (x.valid < 0) break;
        const uint32_t steps = max(x.steps[0], x.steps[1]);
        if (steps == 0) continue;
        const uint32_t kv_head = (a.mode == kHeadPairs ? x.column * 2 : x.column) / a.group;
        const uint32_t tiles = a.mode == kKeyHalves ? 1 : 2;  // of queries
        if (with_q) wait(smem_addr(&sh.q_empty), (with_q - 1) & 1, late);
        ++with_q;
        bool gone = given_up(late);  // no copy into a place that may be in use
        if (lane == 0 && !gone) {
          bar_expect(smem_addr(&sh.q_full), tiles * kRows * kDim * 2);
          for (uint32_t t = 0; t < tiles; ++t) {
            const Tile y = tile_of(a, x, t);
            for (int h = 0; h < kHalves; ++h)
              load_box(smem_addr(sh.q[t]) + h * kBox, &map_q, h * 64, y.head,
                       (int)(x.q_first + y.row), smem_addr(&sh.q_full));
          }
        }
        auto load = [&](uint32_t tile, bool values) {  // a key tile's keys or values
          const uint32_t st = i % kRing, full = smem_addr(&sh.kv_full[st]);
          if (i >= kRing) wait(smem_addr(&sh.kv_empty[st]), (i / kRing - 1) & 1, late);
          gone = given_up(late);
          if (gone) return;
          ++i;
          const uint32_t key = tile * kKeys;
          // values past the sequence's end are another's and meet weights of 0: an infinity or a
          // NaN among them would not vanish, so the rows are cleared before they are handed on
          const uint32_t own = x.k_count - key;
          const bool clear = values && own < kKeys;
          const uint32_t bar = clear ? smem_addr(&sh.landed) : full;
          if (lane == 0) {
            bar_expect(bar, kKeys * kDim * 2);
            for (int h = 0; h < kHalves; ++h)
              load_box(smem_addr(sh.kv[st]) + h * kBox, values ? &map_v : &map_k, h * 64, kv_head,
                       (int)(x.k_first + key), bar);
          }
          if (clear) {  // a sequence's last tile only
            wait(bar, cleared++ & 1, late);
            for (int h = 0; h < kHalves; ++h)
              for (uint32_t z = own * 8 + lane; z < kKeys * 8; z += 32)
                reinterpret_cast<uint4*>(sh.kv[st] + h * kBox)[z] = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(full);
          }
          __syncwarp();
        };
        // in the order in which the products want them
        if (a.mode == kKeyHalves) {
          const uint32_t all = x.steps[0] + x.steps[1];
          load(0, false);
          if (all > 1) load(1, false);
          for (uint32_t j = 0; j < all && !gone; ++j) {
            load(j, true);
            if (j + 2 < all) load(j + 2, false);
          }
        } else {
          for (uint32_t j = 0; j < steps && !gone; ++j) {
            load(j, false);
            load(j, true);
          }
        }
      }
    } else if (warp == kSoftmaxWarps + 1) {
      // ---- products
      constexpr uint32_t kScores = product(kBf16, false, kKeys), kSums = product(kBf16, true, kDim);
      const bool leader = elect();
      const uint64_t q0 = operand(smem_addr(sh.q[0]), 16), k0 = operand(smem_addr(sh.kv[0]), 16),
                     v0 = operand(smem_addr(sh.kv[0]), kBox);
      constexpr uint32_t kTile = kRows * kDim * 2 >> 4;  // of operands' addresses
      auto scores = [&](uint32_t t, uint32_t st, uint32_t tq) {  // S_t from the ring's place st
        if (leader) {
#pragma unroll
          for (int x = 0; x < kDim / 16; ++x) {
            const uint32_t off = (x / 4 * kBox + x % 4 * 32) >> 4;
            mma_smem(kS + t * 128, q0 + tq * kTile + off, k0 + st * kTile + off, kScores, x > 0);
          }
          commit(smem_addr(&sh.s_full[t]));
        }
        __syncwarp();
      };
      auto sums = [&](uint32_t t, uint32_t st, uint32_t half, bool add) {
        if (leader) {
#pragma unroll
          for (uint32_t x = 0; x < kKeys / 32; ++x) {
            const uint32_t step = half * (kKeys / 32) + x;
            mma_tmem(kO + t * kDim, kS + t * 128 + step * 8, v0 + st * kTile + step * (2048 >> 4),
                     kSums, add || step > 0);
          }
        }
        __syncwarp();
      };
      auto signal = [&](uint64_t* bar) {
        if (leader) commit(smem_addr(bar));
        __syncwarp();
      };
      auto arrived = [&](uint32_t i) {
        wait(smem_addr(&sh.kv_full[i % kRing]), (i / kRing) & 1, late);
      };
      uint32_t i = 0, with_q = 0, done0 = 0, done1 = 0;  // tiles of the ring, items, steps
      while (true) {
        const Item x = items.next(sh, late);
        if (x.valid < 0) break;
        if (leader) bar_arrive(smem_addr(&sh.begun));
        __syncwarp();
        const uint32_t n0 = x.steps[0], n1 = x.steps[1], steps = max(n0, n1);
        if (steps == 0) continue;
        wait(smem_addr(&sh.q_full), with_q++ & 1, late);
        arrived(i);
        after_sync();
        auto take = [&](uint32_t t, uint32_t v, bool add) {  // P_t V from the ring's place v
          const uint32_t parity = (t ? done1++ : done0++) & 1;
          wait(smem_addr(&sh.p_full[t][0]), parity, late);
          after_sync();
          sums(t, v, 0, add);
          wait(smem_addr(&sh.p_full[t][1]), parity, late);
          after_sync();
          sums(t, v, 1, true);
        };
        if (a.mode == kKeyHalves) {
          const uint32_t all = n0 + n1;
          scores(0, i % kRing, 0);
          signal(&sh.kv_empty[i++ % kRing]);
          if (all > 1) {
            arrived(i);
            after_sync();
            scores(1, i % kRing, 0);
            signal(&sh.kv_empty[i++ % kRing]);
          }
          for (uint32_t j = 0; j < all; j += 2) {
#pragma unroll
            for (uint32_t t = 0; t < 2; ++t) {
              if (j + t >= all) continue;
              arrived(i);
              take(t, i % kRing, j > 0);
              const bool more = j + t + 2 < all;
              if (!more) signal(&sh.o_full[t]);
              signal(&sh.kv_empty[i++ % kRing]);
              if (more) {
                arrived(i);
                after_sync();
                scores(t, i % kRing, 0);
                signal(&sh.kv_empty[i++ % kRing]);
              }
            }
          }
          signal(&sh.q_empty);
          continue;
        }
        if (n0) scores(0, i % kRing, 0);
        if (n1) scores(1, i % kRing, 1);
        signal(&sh.kv_empty[i % kRing]);
        if (steps == 1) signal(&sh.q_empty);
        for (uint32_t j = 0; j < steps; ++j) {
          const uint32_t v = (i + 1) % kRing, k = (i + 2) % kRing;
          const bool more = j + 1 < steps;
          arrived(i + 1);
          if (more) arrived(i + 2);
#pragma unroll
          for (uint32_t t = 0; t < 2; ++t) {
            const uint32_t n = t ? n1 : n0;
            if (j < n) {
              take(t, v, j > 0);
              if (j + 1 < n) scores(t, k, t);
              else signal(&sh.o_full[t]);
            }
          }
          signal(&sh.kv_empty[v]);
          if (more) signal(&sh.kv_empty[k]);
          if (j + 2 == steps) signal(&sh.q_empty);
          i += 2;
        }
      }
      // the last signals have to reach a block that is still there
      if (with_q) wait(smem_addr(&sh.q_empty), (with_q - 1) & 1, late);
      if (i >= 1) wait(smem_addr(&sh.kv_empty[(i - 1) % kRing]), ((i - 1) / kRing) & 1, late);
    } else if (warp == kSoftmaxWarps + 2) {
      // ---- plan: the block's own item, then those of blocks that have not started, which it
      // takes over one by one
      // An item is claimed once the products of the one before begin, not earlier: what a block
      // holds in advance, another that is ready cannot take.
      uint32_t n = blockIdx.x, claims = 0, turn = 0;
      bool more = false;
      for (uint32_t i = 0;; ++i) {
        if (i) wait<kItemPatience>(smem_addr(&sh.begun), (i - 1) & 1, late);
        turn = more ? turn + 1 : 0;
        if (more) {
          if (given_up(late)) n = ~0u;
        } else if (i) {
          if (lane == 0) {
            bar_expect(smem_addr(&sh.claimed), 16);
            asm volatile(
                "clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes."
                "b128 [%0], [%1];" ::"r"(smem_addr(&sh.claim)),
                "r"(smem_addr(&sh.claimed))
                : "memory");
          }
          wait(smem_addr(&sh.claimed), claims++ & 1, late);
          uint32_t got, first;
          asm volatile(
              "{\n\t.reg .b128 c;\n\t.reg .pred p;\n\t.reg .b32 y, z, w;\n\t"
              "ld.shared.b128 c, [%2];\n\t"
              "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, c;\n\t"
              "selp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
              "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, w}, c;"
              "\n\t}"
              : "=r"(got), "=r"(first)
              : "r"(smem_addr(&sh.claim))
              : "memory");
          const bool gone = given_up(late);
          n = got && !gone ? first : ~0u;
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        // Every index of the grid is some block's to check offsets for, its own or one taken over:
        // blocks whose items others take never start.
        if (n != ~0u && turn == 0)
          for (uint64_t j = (uint64_t)n * 32 + lane; j < a.n_seqs; j += (uint64_t)gridDim.x * 32)
            if (row_range(a.q_off, (uint32_t)j, a.q_rows).bad ||
                row_range(a.k_off, (uint32_t)j, a.k_rows).bad)
              flag_status(a.status, NETKV_DEV_ERANGE);
        Item x = {};
        x.valid = -1;
        if (n != ~0u) x = item_at(a, n, turn, &more);
        if (i >= 2) wait(smem_addr(&sh.item_empty[i % 2]), (i / 2 - 1) & 1, late);
        if (lane == 0) {
          sh.item[i % 2] = x;
          bar_arrive(smem_addr(&sh.item_full[i % 2]));
        }
        if (n == ~0u) break;
      }
    }
  } else {
    // ---- softmax: a thread has a row of its tile
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const uint32_t t = warp / 4, row = tid % 128, lanes = (warp % 4) * 32 << 16;
    const uint32_t s_at = kS + t * 128 + lanes, o_at = kO + t * kDim + lanes;
    uint32_t taken = 0, finished = 0;  // steps, and items with any
    // kKeyHalves: the two tiles' warps meet inside an item.  The wait ends like every other: after
    // one has run out, some may have taken the item and some been told that there is none.
    uint32_t meetings = 0;
    auto meet = [&]() {
      __syncwarp();
      if (lane == 0) bar_arrive(smem_addr(&sh.met));
      wait(smem_addr(&sh.met), meetings++ & 1, late);
      __syncwarp();
    };
    while (true) {
      const Item x = items.next(sh, late);
      if (x.valid < 0) break;
      if (x.valid == 0) continue;
      const Tile y = tile_of(a, x, t);
      const uint32_t steps = t ? x.steps[1] : x.steps[0];
      // keys of this row
      const int visible =
          (int)min((int64_t)x.k_count, (int64_t)x.k_count - x.q_count + y.row + row + 1);
      float m = -INFINITY, l = 0.f;
      for (uint32_t j = 0; j < steps; ++j, ++taken) {
        float s[kKeys];
        wait<kItemPatience>(smem_addr(&sh.s_full[t]), taken & 1, late);
        after_sync();
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_load(s_at + i * 32, s + i * 32);
        tmem_loaded();
        const int seen = visible - (int)((a.mode == kKeyHalves ? 2 * j + t : j) * kKeys);
        if (__any_sync(~0u, seen < kKeys)) {
#pragma unroll
          for (int i = 0; i < kKeys; ++i)
            if (i >= seen) s[i] = -INFINITY;
        }
        float tops[4] = {m, s[0], s[1], s[2]};
#pragma unroll
        for (int i = 3; i + 1 < kKeys; i += 2)
          tops[i / 2 % 4] = max3(tops[i / 2 % 4], s[i], s[i + 1]);
        const float top =
            fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], fmaxf(tops[3], s[kKeys - 1])));
        const bool follow = (top - m) * a.scale2 > kLag;  // also the first maximum
        if (__any_sync(~0u, follow)) {
          float to = 1.f;
          if (follow) {
            to = m == -INFINITY ? 0.f : ex2((m - top) * a.scale2);
            m = top;
          }
          __syncwarp();
          l *= to;
          if (j) {  // S_t is complete, and so is P_t V before it
#pragma unroll
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
        const float base = m == -INFINITY ? 0.f : fmaf(-m, a.scale2, kUp<kBf16>);
        const uint64_t scale_2 = pair(a.scale2, a.scale2), base_2 = pair(base, base);
        uint64_t sums_2[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t p[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float u, w;
            split(fma2(pair(s[h * 64 + 2 * i], s[h * 64 + 2 * i + 1]), scale_2, base_2), &u, &w);
            u = ex2(u);
            w = ex2(w);
            sums_2[i & 1] = add2(sums_2[i & 1], pair(u, w));
            p[i] = pack16<kBf16>(u, w);
          }
          tmem_store(s_at + h * 32, p);
          tmem_stored();
          before_sync();
          bar_arrive(smem_addr(&sh.p_full[t][h]));
        }
        float u, w;
        split(add2(sums_2[0], sums_2[1]), &u, &w);
        l += u + w;
      }
      // ---- the rows' outputs, through shared memory so that whole lines are written: 64
      // values of a warp's 32 rows at a time, 16 bytes of row r in place (c ^ r) of 8
      if (steps) {
        wait(smem_addr(&sh.o_full[t]), finished++ & 1, late);
        after_sync();
      }
      uint4* stage = reinterpret_cast<uint4*>(sh.out[warp]);
      const uint32_t row0 = (warp % 4) * 32;
      unsigned char* dst =
          a.out + ((x.q_first + y.row + row0) * a.out_stride + (uint64_t)y.head * kDim) * 2;
      const bool halves = a.mode == kKeyHalves;
      float own = 1.f, other = 0.f;  // kKeyHalves: what brings the two sums to one maximum
      float* part = reinterpret_cast<float*>(sh.out);  // and the odd tiles' sums, [64][kRows]
      if (halves) {
        if (t) {
          sh.half_m[row] = m;
          sh.half_l[row] = l;
        }
        meet();
        const float m1 = sh.half_m[row], l1 = sh.half_l[row];
        if (t == 0 && l1 != 0.f) {  // NaN too
          const float top = fmaxf(m, m1);
          own = ex2((m - top) * a.scale2);
          other = m1 == -INFINITY ? l1 : ex2((m1 - top) * a.scale2);
          l = l * own + l1 * other;
          m = top;
        }
      }
      const bool any = steps && l != 0.f;
      const float inv = any ? 1.f / l : 0.f;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        if (halves) {
          if (h) meet();  // the half before has left shared memory
          if (t && steps) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float o[32];
              tmem_load(o_at + h * 64 + i * 32, o);
              tmem_loaded();
#pragma unroll
              for (int z = 0; z < 32; ++z) part[(i * 32 + z) * kRows + row] = o[z];
            }
          }
          meet();
        }
        uint4 packed[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float o[32];
          if (steps) {
            tmem_load(o_at + h * 64 + i * 32, o);
            tmem_loaded();
          }
          if (halves && t == 0 && x.steps[1]) {
#pragma unroll
            for (int z = 0; z < 32; ++z) o[z] = o[z] * own + part[(i * 32 + z) * kRows + row] * other;
          }
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            uint32_t w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
              w[q] = any ? pack16<kBf16>(o[z * 8 + q * 2] * inv, o[z * 8 + q * 2 + 1] * inv) : 0u;
            packed[i * 4 + z] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
        if (halves) meet();  // the odd tiles' sums have been read
        if (halves && t) continue;
#pragma unroll
        for (int z = 0; z < 8; ++z) stage[lane * 8 + (z ^ (lane & 7))] = packed[z];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t r = i * 4 + lane / 8, c = lane % 8;
          if (row0 + r < y.rows)
            *reinterpret_cast<uint4*>(dst + (r * a.out_stride + h * 64 + c * 8) * 2) =
                stage[r * 8 + (c ^ (r & 7))];
        }
        __syncwarp();
      }
      if (halves) {
        meet();
        if (t) continue;
      }
      if (row < y.rows && a.lse)
        a.lse[(x.q_first + y.row + row) * a.heads + y.head] =
            l == 0.f ? -INFINITY : logf(l) - fmaf(-m, a.scale2, kUp<kBf16>) * kLn2;
      __syncwarp();
      before_sync();
    }
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

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                            const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                            CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                            CUtensorMapFloatOOBfill);

Encode encoder() {
  static const Encode found = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess)
      p = nullptr;
    return (Encode)p;
  }();
  return found;
}

// Rows of heads * dim values as boxes of 128 rows by 64 values of one head.
bool row_map(CUtensorMap* map, bool bf16, const void* p, uint64_t stride, uint32_t heads,
             uint32_t dim, uint64_t rows) {
  const cuuint64_t dims[3] = {dim, heads, rows ? rows : 1};
  const cuuint64_t strides[2] = {dim * 2ull, stride * 2};
  const cuuint32_t box[3] = {64, 1, 128}, step[3] = {1, 1, 1};
  return encoder()(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                   const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
  PromptArgs a = {};
  a.out = (unsigned char*)d_out;
  a.out_stride = out_stride;
  a.q_off = d_q_off;
  a.k_off = d_k_off;
  a.q_rows = q_rows;
  a.k_rows = k_rows;
  a.heads = heads;
  a.group = heads / kv_heads;
  a.n_seqs = n_seqs;
  a.scale2 = scale * kLog2e;
  a.lse = d_lse;
  a.status = d_status;
  int dev = 0, sms = 0;
  NETKV_CUDA_TRY(cudaGetDevice(&dev));
  NETKV_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  // A sequence ends at most one row block that it does not fill.
  a.mode = a.group % 2 == 0 ? kHeadPairs : kRowPairs;
  uint64_t block_rows = a.mode == kHeadPairs ? kRows : 2 * kRows;
  uint64_t tiles = q_rows / block_rows + n_seqs, columns = a.mode == kHeadPairs ? heads / 2 : heads;
  if (tiles * columns <= (uint64_t)sms * kFewItems / 2) {
    a.mode = kKeyHalves;
    block_rows = kRows;
    tiles = q_rows / block_rows + n_seqs;
    columns = heads;
  }
  if (n_seqs > kSearched) {
    a.parts = (uint32_t)(q_rows / (block_rows * n_seqs)) + 1;
    tiles = (uint64_t)n_seqs * a.parts;
  }
  const uint64_t grid = tiles * columns;
  if (grid >> 31) return NETKV_EINVAL;
  a.tiles = (uint32_t)tiles;
  // One sequence alone is in order as it is, and where every item has an SM the order does not
  // matter; more than 128 sequences would take the search longer than their blocks last.
  a.ordered = n_seqs > 1 && n_seqs <= 128 && grid > (uint64_t)sms;
  if (!encoder()) return NETKV_ECUDA;
  const bool bf = dtype == NETKV_BF16;
  CUtensorMap q, k, v;
  if (!row_map(&q, bf, d_q, q_stride, heads, head_dim, q_rows) ||
      !row_map(&k, bf, k_rows ? d_k : d_q, k_rows ? k_stride : q_stride, k_rows ? kv_heads : 1,
               head_dim, k_rows) ||
      !row_map(&v, bf, k_rows ? d_v : d_q, k_rows ? v_stride : q_stride, k_rows ? kv_heads : 1,
               head_dim, k_rows))
    return NETKV_EINVAL;
  auto go = [&](auto dim, auto b) -> netkv_status {
    constexpr auto kernel = prompt_kernel<decltype(dim)::value, decltype(b)::value>;
    constexpr size_t bytes = sizeof(Shared<decltype(dim)::value>);
    // a launch with fewer registers than the warps share out would never end
    static const int regs = [] {
      cudaFuncAttributes has;
      return cudaFuncGetAttributes(&has, kernel) == cudaSuccess ? has.numRegs : 0;
    }();
    if (regs < kLaunchRegs) return NETKV_ECUDA;
    NETKV_CUDA_TRY(allow_shared<kernel>((int)bytes));
    kernel<<<(unsigned)grid, kThreads, bytes, (cudaStream_t)stream>>>(a, q, k, v);
    return netkv_launch_status();
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (head_dim == 64) return bf ? go(D64(), std::true_type()) : go(D64(), std::false_type());
  return bf ? go(D128(), std::true_type()) : go(D128(), std::false_type());
}
