// Attention of a few tokens of every path over the prefix that its prompt shares and over the path's own tokens.
//
//   o = sum_j exp(scale q.k_j - m) v_j / sum_j exp(scale q.k_j - m),   m = max_j scale q.k_j
//
// Rows that read the same K and V are multiplied together: for the prefix of a prompt all paths * tokens * (query heads per K/V head), so its
// bytes are read once a prompt and not once a path; for a path's own tokens that path's rows.  Both are the same work item (rows, one head of K and
// V, a run of keys), cut along the keys into tiles of 128, and all tiles of a launch, laid end to end, are dealt out in runs of equal length to 148
// CTAs: long prefixes are split, short tails are not, whatever the lengths (they are read on the device).  Every run of an item leaves its rows'
// unnormalised sums, maxima and weights' totals in the workspace; attend_join_kernel puts an output row's parts together.
//
// A CTA (one per SM): products on the tensor cores, 128 rows by 128 keys, with accumulators in tensor memory: two tiles of products and two sums.  All
// softmax warps (0-7, two threads a row) work on one tile of products while the next is made behind the sums of the one before.  An item with more
// than 128 rows has a sum for each half of them, both over the same tiles of K and V.  Warp 8 fetches tiles (TMA), warp 9 asks for the products, warp
// 10 (8-bit caches: 10-17, which turn 8 bits into 16) sees to what lies behind the last key, one more deals the segments.
//
// Weights are rounded to the query's 16 bits for the second product, which takes no others; their total is not.  Outputs are 0.0019 to 0.0023 from 64 bits (rms,
// relative) in bfloat16 and 0.00029 in fp16, where rounding the output alone leaves 0.0017 and 0.00021.
//
// What bounds it (head 128; back to back, and called one by one where that differs): 64 x 5 tokens behind 65536 keys, 370 to 425 us (927 to 805 TFLOP/s, by the power
// limit): the chain of one tile, 2100 cycles in the softmax warps of which 1160 are exponentials; the products' 1026 hide behind it.  16 x 1 behind 32768, 46 us: K and V
// of a tile in 2500 cycles, which is the memory's rate, and 15 us in front of the first tile and behind the last.  32 x 16 x 1 in 16 bits, 216 us (5.6 TB/s), 247 one
// by one.  8-bit caches, the conversion and the steps of few rows: 16 x 9, 76 us; 32 x 16 x 1, 381.  The smallest, 10.5 us: its chain of lengths, segment, Q and K,
// products, join.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "attend_plan.h"
#include "decode_dev.cuh"

namespace sdms {

namespace {

constexpr int kTile = 128;               // keys of a tile, rows of a product
constexpr int kBlock = 64 * kTile * 2;   // a tile's 64 columns: 128 rows of 128 bytes, swizzled
// A row's reference may lag behind its maximum by 2^lazy before its sums are scaled anew, and the largest weight is 2^lift or so.  bfloat16 has weights of any
// size.  fp16 has none below 2^-25, so many small ones would be lost that the total counts, and none from 2^16 on: with 6 and 6 those from 2^-31 of the
// largest are there, and 2^4 are left above for the rounding of references, which products of 2^25 need.
template <bool BF16> struct Weights {
  static constexpr float kLazy = BF16 ? 8.f : 6.f, kLift = BF16 ? 0.f : 6.f;
};
constexpr int kUnit = 64;                // keys of a tile that one softmax thread has
constexpr uint32_t kColS = 0, kColO = 256;   // tensor memory: two tiles of products, the weights over the first half of each; two sums behind them
constexpr int kTensorColumns = 512;

// x / d and the rest for 0 <= x < 2^31: the estimate is at most one too small.
__device__ __forceinline__ int divide(int x, Divisor d, int* rest) {
  uint32_t q = __umulhi((uint32_t)x, d.m);
  if ((uint32_t)x - q * d.d >= d.d) ++q;
  *rest = x - (int)(q * d.d);
  return (int)q;
}

// ---- what all roles agree on -------------------------------------------------------------------------------------------------------

// What work costs, in units of about 450 cycles: a tile with up to 16 rows, up to 128, more; to begin an item and to leave its sums.  8-bit tiles of one
// product each are held up by their conversion.  (Counted by tiles alone, CTAs with prefixes took a third longer than the others for 32 x 16 x 1
// tokens, those with the most items for 64 x 5.)
constexpr int kFewRows = 16, kFew = 4, kOne = 5, kTwo = 10, kBegin = 12;
__host__ __device__ inline int few_cost(bool quant) { return kFew + quant; }
__host__ __device__ inline int one_cost(bool quant) { return kOne + quant; }
// of a tile of one head, with all of an entry's rows
__host__ __device__ inline int tile_cost(int rows, bool quant) {
  const int rest = rows % 256;
  return rows / 256 * kTwo + (rest == 0 ? 0 : rest > 128 ? kTwo : rest > kFewRows ? one_cost(quant) : few_cost(quant));
}

struct Plan {
  int pre_rows, pre_tiles_m, own_rows, own_tiles_m;        // rows of an item's source, items per head
  int pre_plain, own_plain, pre_cost, own_cost;            // products of a tile of one head of such an entry; its cost
  int pre_slot, own_slot;                                  // rows of a slot of partial results
  int pre_items, own_items;
  size_t range_bytes, o_bytes;
};

__host__ __device__ inline int slot_rows(int rows) { return rows < 2 * kTile ? rows : 2 * kTile; }

__host__ __device__ inline long long part_rows(const Plan& p) {
  return (long long)(p.pre_items + kCtas) * p.pre_slot + (long long)(p.own_items + kCtas) * p.own_slot;
}
__host__ __device__ inline Plan plan_of(const AttendDev& a) {
  Plan p;
  p.pre_rows = a.N * a.T * a.group;
  p.own_rows = a.T * a.group;
  p.pre_tiles_m = (p.pre_rows + 2 * kTile - 1) / (2 * kTile);
  p.own_tiles_m = (p.own_rows + 2 * kTile - 1) / (2 * kTile);
  p.pre_plain = (p.pre_rows + kTile - 1) / kTile;
  p.own_plain = (p.own_rows + kTile - 1) / kTile;
  const bool quant = a.pk_scale || a.k_scale;
  p.pre_cost = tile_cost(p.pre_rows, quant);
  p.own_cost = tile_cost(p.own_rows, quant);
  p.pre_slot = slot_rows(p.pre_rows);
  p.own_slot = slot_rows(p.own_rows);
  p.pre_items = a.G * a.Hkv * p.pre_tiles_m;
  p.own_items = a.P * a.Hkv * p.own_tiles_m;
  p.range_bytes = ((size_t)(p.pre_items + p.own_items) * sizeof(int2) + 255) / 256 * 256;
  p.o_bytes = ((size_t)part_rows(p) * a.d * 4 + 255) / 256 * 256;
  return p;
}

// The workspace: first and last CTA of every item, partial sums, their maxima and totals.
struct Parts { int2* range; float* o; float2* ml; };
__host__ __device__ inline Parts parts_of(const AttendDev& a, const Plan& p) {
  unsigned char* w = static_cast<unsigned char*>(a.workspace);
  return Parts{reinterpret_cast<int2*>(w), reinterpret_cast<float*>(w + p.range_bytes), reinterpret_cast<float2*>(w + p.range_bytes + p.o_bytes)};
}
// First row of what CTA c leaves of an item.  (Numbers of item and CTA: from one of a CTA's items to the next, or from one of an item's CTAs to the
// next, one of the two goes up, so their sum names the pair.)
__host__ __device__ inline long long part_row(const Plan& p, bool prefix, int item, int c) {
  return prefix ? (long long)(item + c) * p.pre_slot : (long long)(p.pre_items + kCtas) * p.pre_slot + (long long)(item + c) * p.own_slot;
}

// An entry is a prompt's prefix (0 .. G-1) or a path's own tokens (G .. G+P-1): tokens that its rows see, whole.
__device__ __forceinline__ int queries_of(const AttendDev& a, int p) { return a.count ? min(max(a.count[p], 0), a.T) : a.T; }
__device__ __forceinline__ int keys_of(const AttendDev& a, int e) {
  // (both loads under way together, whichever of the two kinds a lane's entry is)
  const bool own = e >= a.G;
  if (own ? !a.path_cap : !a.prefix_cap) return 0;
  const int len = max(own ? a.len[e - a.G] : a.prefix_len[e], 0), n = own ? queries_of(a, e - a.G) : 1;
  return own ? (n ? (int)min((long long)len + n, (long long)a.path_cap) : 0) : min(len, a.prefix_cap);
}
__device__ __forceinline__ int tiles_of(int keys) { return (keys + kTile - 1) / kTile; }
// An entry's cost by products alone, for calls of a few tiles a CTA, and as above.
struct Cost { uint32_t plain, full; };
__device__ __forceinline__ Cost cost_of(const AttendDev& a, const Plan& p, int e, int keys) {
  const uint32_t n = tiles_of(keys) * a.Hkv;
  if (e < a.G) return Cost{n * p.pre_plain, n ? n * p.pre_cost + kBegin * a.Hkv * p.pre_tiles_m : 0u};
  return Cost{n * p.own_plain, n ? n * p.own_cost + kBegin * a.Hkv * p.own_tiles_m : 0u};
}

// A CTA's run of units, item by item.
struct Segment {
  int n, j0;                             // tiles j0 .. j0 + n - 1 (n = 0: no more)
  int entry, row, head;                  // row of the cache
  int keys, whole, queries;              // keys; how many of them all rows see; new tokens behind those
  int rows, row0;                        // rows of the item: row0 .. row0 + rows - 1 of its source's
  int item;
  int place;                             // of its `unfinite`
  bool prefix, dual;                     // dual: more than 128 rows, two sums
  bool first, last;                      // whether the item begins, ends here
};

// ---- instructions ------------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t* bar, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
  return ok;
}
// False after some two seconds (2^32 cycles), or once another warp of the CTA has given up.
__device__ __forceinline__ bool bar_wait_long(uint64_t* bar, uint32_t parity, volatile int* dead) {
  const long long begin = clock64();
  for (long long i = 0; i < 1LL << 32; ++i) {
    if (bar_try(bar, parity)) return true;
    if (*dead) return false;
    if ((i & 255) == 255 && clock64() - begin > 1LL << 32) break;
  }
  *dead = 1;
  return false;
}
__device__ __forceinline__ bool bar_wait(uint64_t* bar, uint32_t parity, volatile int* dead) {
  return bar_try(bar, parity) || bar_wait_long(bar, parity, dead);
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ void load_tile(void* to, const CUtensorMap* map, int x, int token, int head, int row, uint64_t* bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(smem_addr(to)), "l"(map), "r"(x), "r"(token), "r"(head), "r"(row), "r"(smem_addr(bar)) : "memory");
}

// Shared-memory operands: rows of 128 bytes in groups of eight (1024 bytes), swizzled.  The lower word says where and, for elements that run along
// M or N, how far blocks of 64 of them lie apart; the upper one is always the same.
constexpr uint32_t kOperandHigh = 1024 >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t operand_low(uint32_t addr, uint32_t lead) { return (addr & 0x3ffff) >> 4 | lead >> 4 << 16; }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t what, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 x, {%1, %4};\n\tmov.b64 y, {%2, %4};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b), "r"(what), "r"(kOperandHigh), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t what, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 y, {%2, %4};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b), "r"(what), "r"(kOperandHigh), "r"((uint32_t)add) : "memory");
}
// One lane of a warp that runs as one.  (Products are asked for in such code: with operands that the compiler knows to be the same in all lanes an
// instruction takes a few cycles; from a branch of one thread's own it took 64 to 130.)
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(~0u, x, 0); }
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tensor_load(uint32_t at, float (&x)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tensor_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// (what was loaded is used behind the wait only, and the compiler is told so)
__device__ __forceinline__ void behind_wait(float (&x)[32]) {
  asm volatile("" : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]), "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]),
               "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]), "+f"(x[16]), "+f"(x[17]), "+f"(x[18]), "+f"(x[19]), "+f"(x[20]), "+f"(x[21]), "+f"(x[22]),
               "+f"(x[23]), "+f"(x[24]), "+f"(x[25]), "+f"(x[26]), "+f"(x[27]), "+f"(x[28]), "+f"(x[29]), "+f"(x[30]), "+f"(x[31]));
}
__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tensor_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 16 rows, 64 columns: column 8 k + 2 (lane % 4) + j of row lane / 4 (+ 8) is element 4 k + j (+ 2).
__device__ __forceinline__ void tensor_load_16(uint32_t at, float (&x)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tensor_store_16(uint32_t at, const float (&x)[32]) {
  uint32_t r[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(x[i]);
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// The weights of a unit, two to a column: column 4 k + lane % 4 of row lane / 4 (+ 8) is element 2 k (+ 1).
__device__ __forceinline__ void tensor_store_16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// Which keys of a unit a row sees.  b: its first key, from the end of what all rows see; last: keys that there are from it on; bits: those behind
// that end.
__device__ __forceinline__ uint64_t seen(int b, int last, uint64_t bits) {
  uint64_t s = b <= -64 ? ~0ull : b < 0 ? bits << -b | ((1ull << -b) - 1) : b < 64 ? bits >> b : 0;
  if (last < 64) s &= last > 0 ? (1ull << last) - 1 : 0;
  return s;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float x, float y, float z) {
  float m;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(x), "f"(y), "f"(z));
  return m;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  if (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// ---- shared memory -----------------------------------------------------------------------------------------------------------------

// D: head; QUANT: 8-bit caches.  Q has two places: a segment of both streams' rows takes both, others one after the other.
template <int D, bool QUANT>
struct Shape {
  static constexpr int kHalves = D / 64;
  static constexpr int kOperand = kHalves * kBlock;                 // one tile of Q, K or V in 16 bits
  static constexpr int kRaw = QUANT ? kTile * D : 0;                // one in 8 bits
  static constexpr int kStages = QUANT ? (D == 64 ? 6 : 4) : D == 64 ? 10 : 5;
  static constexpr int kRawStages = QUANT ? (D == 64 ? 6 : 2) : 0;
  static constexpr int kBytes = 2 * kOperand + kStages * kOperand + kRawStages * kRaw;
  // 8-bit caches: eight warps more, and registers moved from them to the softmax warps (640 * 96 = 256 * 144 + 384 * 64).
  static constexpr int kThreads = QUANT ? 640 : 384;
  static constexpr int kConverters = QUANT ? 8 : 0;                 // warps
};
constexpr int kSegments = 4;             // segments that are dealt out ahead
constexpr int kPlaces = 8;
template <class S>
struct Bars {
  uint64_t full[S::kStages], empty[S::kStages], landed[S::kStages];
  uint64_t raw_full[S::kRawStages + 1], raw_empty[S::kRawStages + 1];
  uint64_t q_full[2], q_empty[2], s_ready[2], p_ready[2], o_ready[2], o_free[2], pair[4], o_step, drain;
  uint64_t seg_full[kSegments], seg_empty[kSegments];
};
// What all warps share beside the tiles, behind them.
template <class S>
struct Shared {
  Bars<S> bars;
  Segment segment[kSegments];
  float half[2][2][kTile];               // what the two threads of a row tell each other
  // New tokens whose V has an infinity or NaN: a bit each, a segment's place each.  (A dealt segment is at most five behind one that is worked on.)
  unsigned long long unfinite[kPlaces];
  uint32_t tensor;
  volatile int dead;
};
struct Maps { CUtensorMap pre_k, pre_v, own_k, own_v; };

// The order in which tiles of K and V are used, which those that fetch and convert them follow.  Two halves of rows: K0, V0, K1, V1, ...; one: K0, K1,
// V0, K2, V1, ...
template <class F>
__device__ __forceinline__ bool each_tile(const Segment& s, F use) {
  for (int e = 0; e < 2 * s.n; ++e) {
    bool v;
    int i;
    if (s.dual) { v = e & 1; i = e >> 1; }
    else if (e & 1) { v = (e + 1) / 2 >= s.n; i = v ? s.n - 1 : (e + 1) / 2; }
    else { v = e > 0; i = v ? e / 2 - 1 : 0; }
    if (!use(v, s.j0 + i)) return false;
  }
  return true;
}

template <int D, bool QUANT, bool BF16>
__global__ void __launch_bounds__(Shape<D, QUANT>::kThreads, 1)
attend_kernel(const __grid_constant__ Maps maps, const AttendDev a) {
  using S = Shape<D, QUANT>;
  // (no static shared memory: the tiles start where the CTA's does, on a multiple of 1024 bytes)
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* sm_q = smem;
  unsigned char* sm_kv = sm_q + 2 * S::kOperand;
  unsigned char* sm_raw = sm_kv + S::kStages * S::kOperand;
  Shared<S>& sh = *reinterpret_cast<Shared<S>*>(smem + S::kBytes);
  Bars<S>& bars = sh.bars;
  volatile int& dead = sh.dead;
  constexpr int kDealer = QUANT ? 10 + S::kConverters : 11, kTakers = QUANT ? 10 + S::kConverters : 11;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh.tensor)), "r"(kTensorColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    fence_before();
  } else if (warp == 0) {
    // (a lane per barrier: arrivals that end a phase)
    if (lane < S::kStages) { bar_init(&bars.full[lane], QUANT ? S::kConverters : 1); bar_init(&bars.empty[lane], 1); bar_init(&bars.landed[lane], 1); }
    else if (lane < S::kStages + S::kRawStages) { bar_init(&bars.raw_full[lane - S::kStages], 1); bar_init(&bars.raw_empty[lane - S::kStages], S::kConverters); }
    else if (lane == 16 || lane == 17) {
      const int i = lane - 16;
      bar_init(&bars.q_full[i], 256); bar_init(&bars.q_empty[i], 1); bar_init(&bars.s_ready[i], 1); bar_init(&bars.p_ready[i], 256);
      bar_init(&bars.o_ready[i], 1); bar_init(&bars.o_free[i], 256);
    } else if (lane >= 18 && lane < 18 + kSegments) { bar_init(&bars.seg_full[lane - 18], 1); bar_init(&bars.seg_empty[lane - 18], kTakers); }
    else if (lane >= 24 && lane < 28) bar_init(&bars.pair[lane - 24], 64);
    else if (lane == 30) { bar_init(&bars.o_step, 1); bar_init(&bars.drain, 1); dead = 0; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  } else if (warp == 8 && lane < 4) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &maps.pre_k : lane == 1 ? &maps.pre_v : lane == 2 ? &maps.own_k : &maps.own_v) : "memory");
  }
  static_assert(S::kStages + S::kRawStages <= 16, "a lane per barrier");
  __syncthreads();
  fence_after();
  grid_wait();
  grid_release();
  const Plan plan = plan_of(a);
  const Parts parts = parts_of(a, plan);
  // Units of every 32 entries, for the warp that deals them out (in the place of what the softmax warps tell each other later).  With 32 entries
  // or fewer it needs none: half a microsecond and more that every small call would wait.
  const int entries = a.G + a.P, chunks = (entries + 31) / 32;
  uint2* chunk_cost = reinterpret_cast<uint2*>(sh.half);
  constexpr int kMostChunks = sizeof(sh.half) / 8;
  auto cost_of_chunk = [&](int i) {
    const int e = i * 32 + lane;
    const Cost x = e < entries ? cost_of(a, plan, e, keys_of(a, e)) : Cost{0u, 0u};
    return make_uint2(__reduce_add_sync(~0u, x.plain), __reduce_add_sync(~0u, x.full));
  };
  if (chunks > 1) {
    for (int i = warp; i < min(chunks, kMostChunks); i += S::kThreads / 32) {
      const uint2 x = cost_of_chunk(i);
      if (lane == 0) chunk_cost[i] = x;
    }
    __syncthreads();
  }
  const uint32_t tensor = sh.tensor;
  // Segments come from one warp, a few ahead; every other warp takes them in turn.
  int seg_next = 0;
  auto take = [&](Segment& s) -> bool {
    const int i = seg_next % kSegments;
    if (!__all_sync(~0u, bar_wait(&bars.seg_full[i], seg_next / kSegments & 1, &dead))) { s.n = 0; return false; }
    s = sh.segment[i];
    __syncwarp();
    if (lane == 0) bar_arrive(&bars.seg_empty[i]);
    ++seg_next;
    return s.n > 0;
  };
  // whether a query may not see what another of its path does
  auto doubtful = [&](const Segment& s) { return !s.prefix && (s.queries > 1 || a.mask); };
  Segment seg;
  if (QUANT) {
    if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
  }

  if (warp < 8) {
    // ---- softmax: two threads per row, 64 of a tile's 128 keys each; all eight warps on one tile of products while the next is made ----
    const int half = warp >> 2, r = tid & 127;
    const uint32_t at_lanes = tensor + ((uint32_t)(warp & 3) << 21);            // 32 * (warp % 4) in the upper half of an address
    const float c = a.scale * 1.4426950408889634f;
    constexpr float kLazy = Weights<BF16>::kLazy, kLift = Weights<BF16>::kLift;
    int step = 0;                                                   // tiles of products so far
    uint32_t phase_o = 0;                                           // a bit per sum
    int o_place = 0, q_place = 0, q_uses = 0, q_said = 0;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(~0u, bar_wait(bar, parity, &dead)); };
    // the two warps of the same rows meet
    uint32_t phase_pair = 0;
    auto both = [&]() -> bool {
      bar_arrive(&bars.pair[warp & 3]);
      const bool met = wait(&bars.pair[warp & 3], phase_pair);
      phase_pair ^= 1;
      return met;
    };
    // Q of a segment: asked for once the products that read what was there are through, in place once they say so
    auto ask_q = [&](const Segment& g) -> bool {
      for (int t = 0; t <= (g.dual ? 1 : 0); ++t) {
        const int place = q_place;
        if (q_uses > 1 && !wait(&bars.q_empty[place], (q_uses >> 1) + 1 & 1)) return false;
        q_place ^= 1;
        ++q_uses;
        const int row = t * kTile + r;
        if (row < g.rows) {
          int rest, j;
          const int n = divide(g.row0 + row, a.per_path, &rest), token = divide(rest, a.per_token, &j);
          const uint16_t* from = a.q + (long long)(g.prefix ? g.entry * a.N + n : g.row) * a.q_path + (long long)token * a.q_token +
                                 (long long)(g.head * a.group + j) * a.q_head + half * (D / 2);
          const uint32_t to = smem_addr(sm_q) + place * S::kOperand + r * 128 + (D == 128 ? half * kBlock : 0);
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                         ::"r"(to + (((i + (D == 64 ? half * 4 : 0)) ^ (r & 7)) << 4)), "l"(from + i * 8) : "memory");
        }
      }
      return true;
    };
    auto say_q = [&](const Segment& g) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_async();
      for (int t = 0; t <= (g.dual ? 1 : 0); ++t) { bar_arrive(&bars.q_full[q_said]); q_said ^= 1; }
    };
    Segment next;
    bool going = take(seg);
    if (going) {
      going = ask_q(seg);
      if (going) say_q(seg);
    }
    while (going) {
      const bool more = take(next);
      // (with a place for each, the next segment's Q comes in while this one is worked on)
      bool asked = more && !seg.dual && !next.dual;
      if (asked && !ask_q(next)) break;
      const int halves = seg.dual ? 2 : 1, whole = seg.whole;
      // 16 rows at most: lanes 4 i .. 4 i + 3 have rows i and i + 8, a quarter of the columns each, so that a warp has 16 x 64 weights to compute
      // and not 32 x 64 of which half and more are nobody's
      const bool few = seg.rows <= kFewRows, more_than_8 = seg.rows > 8;
      // what a row sees: tokens in front of `whole`, and of the 64 behind it those of its bits
      uint64_t bits0 = 0, bits1 = 0;
      auto bits_of = [&](int row) -> uint64_t {
        int j;
        const int token = divide(seg.row0 + min(row, seg.rows - 1), a.per_token, &j);
        const uint64_t x = a.mask ? a.mask[(size_t)seg.row * a.T + token] : ~0ull >> (63 - token);
        return seg.queries < 64 ? x & ((1ull << seg.queries) - 1) : x;
      };
      if (!seg.prefix) {
        bits0 = bits_of(few ? lane >> 2 : r);
        if (few || seg.dual) bits1 = bits_of(few ? (lane >> 2) + 8 : kTile + r);
      }
      // Reference (of the products as they come) and the weights' total, of this thread's keys; of rows r and 128 + r, or of the two of `few`
      float m0 = -INFINITY, l0 = 0.f, m1 = -INFINITY, l1 = 0.f;
      bool ok = true;
      for (int i = 0; i < seg.n && ok; ++i) {
        const int key0 = (seg.j0 + i) * kTile + half * kUnit;
        const int b = key0 - whole, last = seg.keys - key0;         // the first key, from the end of what all see; keys left
#pragma unroll 1
        for (int t = 0; t < halves; ++t) {
          const int buffer = step & 1, place = seg.dual ? t : o_place;
          const uint32_t at = at_lanes + kColS + buffer * kTile, at_o = at_lanes + kColO + place * D + half * (D / 2);
          ok = wait(&bars.s_ready[buffer], step >> 1 & 1);
          if (!ok) break;
          fence_after();
          // (the sums of the step before have to be in before they are scaled anew; those of the one before that are, or these products would not be)
          // (of two sums, the other one's step came last)
          auto summed = [&] {
            const bool in = seg.dual || wait(&bars.o_step, step + 1 & 1);
            fence_after();
            return in;
          };
          const bool there = (seg.dual ? t * kTile : 0) + (r & ~31) < seg.rows;        // (the same in all lanes and in both warps of a row)
          if (there && !few) {
            float x[2][32];
            tensor_load(at + half * kUnit, x[0]);
            tensor_load(at + half * kUnit + 32, x[1]);
            tensor_load_wait();
            behind_wait(x[0]);
            behind_wait(x[1]);
            if (b + kUnit > 0) {
              const uint64_t sees = seen(b, last, t ? bits1 : bits0);
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                x[0][j] = (uint32_t)sees >> j & 1u ? x[0][j] : -INFINITY;
                x[1][j] = (uint32_t)(sees >> 32) >> j & 1u ? x[1][j] : -INFINITY;
              }
            }
            float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              most[j >> 1 & 1] = max3(most[j >> 1 & 1], x[0][j], x[0][j + 1]);
              most[2 + (j >> 1 & 1)] = max3(most[2 + (j >> 1 & 1)], x[1][j], x[1][j + 1]);
            }
            float mx = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
            // (also: both have read their products, which the weights are written over)
            sh.half[buffer][half][r] = mx;
            ok = both();
            mx = fmaxf(mx, sh.half[buffer][half ^ 1][r]);
            float m = t ? m1 : m0, f = 1.f;
            if (i == 0) m = mx;
            const bool lags = mx * c > m * c + kLazy;
            if (__any_sync(~0u, lags)) {
              if (lags) { f = exp2_fast((m - mx) * c); m = mx; }
              ok = ok && summed();
#pragma unroll 1
              for (int k = 0; k < D / 64; ++k) {
                float o[32];
                uint32_t w[32];
                tensor_load(at_o + k * 32, o);
                tensor_load_wait();
                behind_wait(o);
#pragma unroll
                for (int j = 0; j < 32; ++j) w[j] = __float_as_uint(o[j] * f);
                tensor_store(at_o + k * 32, w);
              }
            }
            const float ref = m == -INFINITY ? 0.f : m * c - kLift;
            // (All 64 on the special function unit: sixteen of them by a polynomial instead, 6.5 instructions each, took 480 us where this takes 405,
            // 64 x 5 tokens behind 65536.)
            const Pair scale = Pair::of(c, c), minus_ref = Pair::of(-ref, -ref);
            Pair sum[2] = {Pair::of(0.f, 0.f), Pair::of(0.f, 0.f)};
            uint32_t w[32];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                float u, v;
                fma(Pair::of(x[k][j], x[k][j + 1]), scale, minus_ref).split(&u, &v);
                u = exp2_fast(u); v = exp2_fast(v);
                sum[k] = add(sum[k], Pair::of(u, v));
                w[k * 16 + j / 2] = pack<BF16>(u, v);
              }
            tensor_store(at + half * 32, w);
            float s0, s1;
            add(sum[0], sum[1]).split(&s0, &s1);
            const float l = fmaf(t ? l1 : l0, f, s0 + s1);
            if (t) { m1 = m; l1 = l; } else { m0 = m; l0 = l; }
            tensor_store_wait();
          } else if (there && (warp & 3) == 0) {
            float x[32];                                            // 8 columns at a time: two of row i, two of row i + 8
            tensor_load_16(at + half * kUnit, x);
            tensor_load_wait();
            behind_wait(x);
            const int col = (lane & 3) * 2, row = lane >> 2;
            if (b + kUnit > 0) {
              const uint64_t sees = seen(b, last, bits0) >> col, sees1 = seen(b, last, bits1) >> col;
#pragma unroll
              for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                  x[4 * k + j] = sees >> (8 * k + j) & 1u ? x[4 * k + j] : -INFINITY;
                  x[4 * k + 2 + j] = sees1 >> (8 * k + j) & 1u ? x[4 * k + 2 + j] : -INFINITY;
                }
            }
            float mx = -INFINITY, mx1 = -INFINITY;
#pragma unroll
            for (int k = 0; k < 8; ++k) { mx = fmaxf(mx, fmaxf(x[4 * k], x[4 * k + 1])); mx1 = fmaxf(mx1, fmaxf(x[4 * k + 2], x[4 * k + 3])); }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) { mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, o)); mx1 = fmaxf(mx1, __shfl_xor_sync(~0u, mx1, o)); }
            if ((lane & 3) == 0) { sh.half[buffer][half][row] = mx; sh.half[buffer][half][row + 8] = mx1; }
            ok = both();
            mx = fmaxf(mx, sh.half[buffer][half ^ 1][row]);
            mx1 = fmaxf(mx1, sh.half[buffer][half ^ 1][row + 8]);
            if (i == 0) { m0 = mx; m1 = mx1; }
            const bool lags = mx * c > m0 * c + kLazy, lags1 = more_than_8 && mx1 * c > m1 * c + kLazy;
            if (__any_sync(~0u, lags || lags1)) {
              const float f = lags ? exp2_fast((m0 - mx) * c) : 1.f, f1 = lags1 ? exp2_fast((m1 - mx1) * c) : 1.f;
              if (lags) m0 = mx;
              if (lags1) m1 = mx1;
              l0 *= f; l1 *= f1;
              ok = ok && summed();
              if (D == 128) {
                float o[32];
                tensor_load_16(at_o, o);
                tensor_load_wait();
                behind_wait(o);
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] *= j & 2 ? f1 : f;
                tensor_store_16(at_o, o);
              } else {                                              // 32 columns a half: the thread-per-row form, factors from the lanes that have them
                const int from = (lane & 7) * 4;
                const float fa = __shfl_sync(~0u, f, from), fb = __shfl_sync(~0u, f1, from), fr = lane < 8 ? fa : lane < 16 ? fb : 1.f;
                float o[32];
                uint32_t w[32];
                tensor_load(at_o, o);
                tensor_load_wait();
                behind_wait(o);
#pragma unroll
                for (int j = 0; j < 32; ++j) w[j] = __float_as_uint(o[j] * fr);
                tensor_store(at_o, w);
              }
            }
            const float ref = m0 == -INFINITY ? 0.f : m0 * c - kLift, ref1 = m1 == -INFINITY ? 0.f : m1 * c - kLift;
            uint32_t w[16];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float u = exp2_fast(fmaf(x[4 * k], c, -ref)), v = exp2_fast(fmaf(x[4 * k + 1], c, -ref));
              l0 += u + v;
              w[2 * k] = pack<BF16>(u, v);
            }
            if (more_than_8) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float u = exp2_fast(fmaf(x[4 * k + 2], c, -ref1)), v = exp2_fast(fmaf(x[4 * k + 3], c, -ref1));
                l1 += u + v;
                w[2 * k + 1] = pack<BF16>(u, v);
              }
            } else {
#pragma unroll
              for (int k = 0; k < 8; ++k) w[2 * k + 1] = 0u;
            }
            tensor_store_16(at + half * 32, w);
            tensor_store_wait();
          }
          fence_before();
          bar_arrive(&bars.p_ready[buffer]);
          ++step;
          if (asked) { say_q(next); asked = false; }
          if (!ok) break;
        }
      }
      if (!ok) break;
      if (!asked && more && (seg.dual || next.dual)) {
        if (!ask_q(next)) break;
        say_q(next);
      }
      // ---- what the segment leaves: sums, the reference in powers of two, the weights' total ----
      if (few) {                                                    // back to a thread per row
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) { l0 += __shfl_xor_sync(~0u, l0, o); l1 += __shfl_xor_sync(~0u, l1, o); }
        const int from = (lane & 7) * 4;
        const float ma = __shfl_sync(~0u, m0, from), mb = __shfl_sync(~0u, m1, from), la = __shfl_sync(~0u, l0, from), lb = __shfl_sync(~0u, l1, from);
        m0 = lane < 8 ? ma : mb;
        l0 = lane < 8 ? la : lb;
      }
      // The place of the maxima two steps ago, which both have read: they met in the last step.  Not so where the second of two halves of rows has none for
      // these warps, which pass its steps without meeting.
      if (seg.dual) ok = both() && ok;
      auto other = [&](float x) {
        sh.half[step & 1][half][r] = x;
        ok = both() && ok;
        const float y = sh.half[step & 1][half ^ 1][r];
        ok = both() && ok;
        return y;
      };
      const float total0 = l0 + other(l0), total1 = seg.dual ? l1 + other(l1) : 0.f;
      const long long at = part_row(plan, seg.prefix, seg.item, blockIdx.x);
      for (int t = 0; t < halves && ok; ++t) {
        const int place = seg.dual ? t : o_place, row = t * kTile + r;
        ok = wait(&bars.o_ready[place], phase_o >> place & 1);
        if (!ok) break;
        phase_o ^= 1u << place;
        fence_after();
        if (t * kTile + (r & ~31) < seg.rows) {
#pragma unroll 1
          for (int k = 0; k < D / 64; ++k) {
            float o[32];
            tensor_load(at_lanes + kColO + place * D + half * (D / 2) + k * 32, o);
            tensor_load_wait();
            behind_wait(o);
            if (row < seg.rows) {
              float4* to = reinterpret_cast<float4*>(parts.o + (at + row) * D + half * (D / 2) + k * 32);
#pragma unroll
              for (int j = 0; j < 8; ++j) to[j] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
            }
          }
          if (row < seg.rows && half == 0) {
            const float m = t ? m1 : m0;
            float total = t ? total1 : total0;
            const uint64_t unfinite = *(volatile unsigned long long*)&sh.unfinite[seg.place];
            if (unfinite && unfinite & bits_of(row)) total = NAN;
            parts.ml[at + row] = make_float2(m == -INFINITY ? -INFINITY : m * c - kLift, total);
          }
        }
        fence_before();
        bar_arrive(&bars.o_free[place]);
      }
      if (!ok) break;
      if (!seg.dual) o_place ^= 1;
      if (tid == 0) {
        int* range = reinterpret_cast<int*>(parts.range + (seg.prefix ? 0 : plan.pre_items) + seg.item);
        if (seg.first) range[0] = blockIdx.x;
        if (seg.last) range[1] = blockIdx.x;
      }
      seg = next;
      going = more;
    }
  } else if (warp == 8) {
    // ---- fetches ----
    int slot = 0;
    uint32_t phase = 1;
    constexpr int kRing = QUANT ? S::kRawStages : S::kStages;
    bool ok = true;
    while (ok && take(seg))
      ok = each_tile(seg, [&](bool v, int j) {
        if (!__all_sync(~0u, bar_wait(QUANT ? &bars.raw_empty[slot] : &bars.empty[slot], phase, &dead))) return false;
        if (lane == 0) {
          const CUtensorMap* map = seg.prefix ? (v ? &maps.pre_v : &maps.pre_k) : (v ? &maps.own_v : &maps.own_k);
          // (V of tiles with new tokens, and of the last one: see warp 10)
          uint64_t* bar = QUANT ? &bars.raw_full[slot] : v && (j + 1) * kTile > seg.whole ? &bars.landed[slot] : &bars.full[slot];
          if (QUANT) {
            bar_expect(bar, S::kRaw);
            load_tile(sm_raw + slot * S::kRaw, map, 0, j * kTile, seg.head, seg.row, bar);
          } else {
            bar_expect(bar, S::kOperand);
#pragma unroll
            for (int h = 0; h < S::kHalves; ++h)
              load_tile(sm_kv + slot * S::kOperand + h * kBlock, map, h * 64, j * kTile, seg.head, seg.row, bar);
          }
        }
        __syncwarp();
        if (++slot == kRing) { slot = 0; phase ^= 1; }
        return true;
      });
  } else if (warp == 9) {
    // ---- products ----
    int slot = 0;
    uint32_t phase = 0;
    uint32_t phase_q = 0, phase_free = 0, used = 0;                  // a bit per place of Q, per sum
    int q_place = 0, o_place = 0;
    uint32_t made = 0, taken = 0;                                    // tiles: products asked for, weights used
    // sums in 32 bits; both operands of one 16-bit type; 128 rows; K: its rows are the columns of S; V: its rows run along the sum
    constexpr uint32_t type = BF16 ? 1u : 0u;
    constexpr uint32_t kind = 1u << 4 | type << 7 | type << 10 | (uint32_t)(kTile / 16) << 24;
    constexpr uint32_t what_s = kind | (uint32_t)(kTile / 8) << 17, what_o = kind | (uint32_t)(D / 8) << 17 | 1u << 16;
    const uint32_t tensor_u = uniform(tensor);
    const uint32_t q_low = operand_low(smem_addr(sm_q), 16), k_low = operand_low(smem_addr(sm_kv), 16), v_low = operand_low(smem_addr(sm_kv), kBlock);
    // the next tile of K or V: its place
    auto next_tile = [&]() -> int {
      if (!__all_sync(~0u, bar_wait(&bars.full[slot], phase, &dead))) return -1;
      const int at = slot;
      if (++slot == S::kStages) { slot = 0; phase ^= 1; }
      return at;
    };
    bool ok = true;
    while (ok && take(seg)) {
      const bool dual = uniform(seg.dual);
      const int n = uniform(seg.n), keys = uniform(seg.keys - seg.j0 * kTile), halves = dual ? 2 : 1;
      const int q_first = q_place, q_second = dual ? q_place ^ 1 : q_place;
      ok = bar_wait(&bars.q_full[q_first], phase_q >> q_first & 1, &dead);
      phase_q ^= 1u << q_first;
      if (dual) { ok = ok && bar_wait(&bars.q_full[q_second], phase_q >> q_second & 1, &dead); phase_q ^= 1u << q_second; }
      if (!dual) q_place ^= 1;
      ok = __all_sync(~0u, ok);
      if (!ok) break;
      // Tile i = -ahead .. n - 1: its sums and, behind each half's, the products that take the weights' place, of the tile `ahead` further on
      const int ahead = dual ? 1 : 2;
      for (int i = -ahead; i < n && ok; ++i) {
        const int ik = i + ahead;
        const int v = i >= 0 ? next_tile() : 0, k = ik < n ? next_tile() : -2;
        if (v < 0 || k == -1) { ok = false; break; }
#pragma unroll 1
        for (int t = 0; t < halves; ++t) {
          const int place = dual ? t : o_place;
          if (i >= 0) {
            // weights times V, once they are there and (the first of a segment) what the sum's place held before has been read
            const int buffer = taken & 1;
            ok = bar_wait(&bars.p_ready[buffer], taken >> 1 & 1, &dead);
            if (i == 0 && (used >> place & 1)) {
              ok = ok && bar_wait(&bars.o_free[place], phase_free >> place & 1, &dead);
              phase_free ^= 1u << place;
            }
            ok = __all_sync(~0u, ok);
            if (!ok) break;
            ++taken;
            fence_after();
            const uint32_t d = tensor_u + kColO + place * D, w = tensor_u + kColS + buffer * kTile, y = v_low + v * (S::kOperand >> 4);
            const int left = keys - i * kTile;
            if (elect_one()) {
              if (left >= kTile) {
#pragma unroll
                for (int x = 0; x < kTile / 16; ++x) mma_ts(d, w + x * 8, y + x * (2048 >> 4), what_o, i > 0 || x > 0);
              } else {
#pragma unroll 1
                for (int x = 0; x * 16 < left; ++x) mma_ts(d, w + x * 8, y + x * (2048 >> 4), what_o, i > 0 || x > 0);
              }
              mma_commit(&bars.o_step);
              if (i == n - 1) mma_commit(&bars.o_ready[place]);
            }
            __syncwarp();
          } else {
            fence_after();
          }
          if (k >= 0) {
            const int buffer = made & 1;
            ++made;
            const uint32_t d = tensor_u + kColS + buffer * kTile, x = q_low + (t ? q_second : q_first) * (S::kOperand >> 4), y = k_low + k * (S::kOperand >> 4);
            if (elect_one()) {
#pragma unroll
              for (int z = 0; z < D / 16; ++z) {
                const uint32_t at = ((z >> 2) * kBlock + (z & 3) * 32) >> 4;
                mma_ss(d, x + at, y + at, what_s, z > 0);
              }
              mma_commit(&bars.s_ready[buffer]);
            }
            __syncwarp();
          }
        }
        if (!ok) break;
        if (elect_one()) {
          if (i >= 0) mma_commit(&bars.empty[v]);
          if (k >= 0) mma_commit(&bars.empty[k]);
          if (ik == n - 1) { mma_commit(&bars.q_empty[q_first]); if (dual) mma_commit(&bars.q_empty[q_second]); }
        }
        __syncwarp();
      }
      used |= dual ? 3u : 1u << o_place;
      if (!dual) o_place ^= 1;
    }
    // (given up: what is under way ends before the tensor memory is given back)
    if (!ok) {
      if (elect_one()) mma_commit(&bars.drain);
      __syncwarp();
      for (int i = 0; i < (1 << 20) && !bar_try(&bars.drain, 0); ++i) {}
    }
    __syncwarp();
  } else if (!QUANT) {
    if (warp == 10) {
    // ---- what lies behind the last key in V's last tile becomes zero: the weights there are, but 0 * NaN is not.  So does an infinity or NaN in V of a
    // new token, which some queries see and others do not; those that see it get a total of NaN instead ----
    int slot = 0;
    uint32_t phases = 0;
    bool ok = true;
    while (ok && take(seg))
      ok = each_tile(seg, [&](bool v, int j) {
        if (v && (j + 1) * kTile > seg.whole) {
          if (!__all_sync(~0u, bar_wait(&bars.landed[slot], phases >> slot & 1, &dead))) return false;
          phases ^= 1u << slot;
          const int from = min(seg.keys - j * kTile, kTile), to = (from + 15) & ~15;          // (the products stop there)
          for (int x = lane; x < (to - from) * (D / 8); x += 32) {
            const int row = from + x / (D / 8), piece = x % (D / 8);
            *reinterpret_cast<uint4*>(sm_kv + slot * S::kOperand + (piece >> 3) * kBlock + row * 128 + (piece & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          if (doubtful(seg)) {
            const int fresh = max(seg.whole - j * kTile, 0);
            for (int x = lane; x < (from - fresh) * (D / 8); x += 32) {
              // (a token's pieces, in whatever order the swizzle has them)
              const int row = fresh + x / (D / 8), piece = x % (D / 8);
              uint4* at = reinterpret_cast<uint4*>(sm_kv + slot * S::kOperand + (piece >> 3) * kBlock + row * 128 + (piece & 7) * 16);
              const uint4 w = *at;
              constexpr uint32_t top = BF16 ? 0x7f80u : 0x7c00u;
              auto bad = [&](uint32_t y) { return (y & top) == top || (y >> 16 & top) == top; };
              if (bad(w.x) || bad(w.y) || bad(w.z) || bad(w.w)) {
                *at = make_uint4(0u, 0u, 0u, 0u);
                atomicOr(&sh.unfinite[seg.place], 1ull << (j * kTile + row - seg.whole));
              }
            }
          }
          fence_async();
          __syncwarp();
          if (lane == 0) bar_arrive(&bars.full[slot]);
        }
        if (++slot == S::kStages) slot = 0;
        return true;
      });
    }
  } else if (warp < 10 + S::kConverters) {
    // ---- 8 bits to 16 ----
    // A code's seven bits of exponent and mantissa are a bfloat16's but for the exponent's offset: code << 4 reads as value * 2^-120, subnormal codes
    // included, and one multiplication by a power of two sets that right and applies the token's scale.  Exact, but for values that a
    // bfloat16 does not hold, and for the two codes that are not numbers, which are looked for on the way and put right behind it (16 x 9 tokens: 75.5 us
    // for 73.5 without a look).  A warp has 16 tokens of a tile.
    constexpr int kTokens = kTile / (S::kConverters ? S::kConverters : 1), kPieces = D / 16;
    const int token0 = (warp - 10) * kTokens;
    int slot = 0, raw = 0;
    uint32_t phase = 1, phase_raw = 0;
    // Which 16 bytes a lane takes of every four (D = 64: eight) tokens: such that eight lanes in a row read 128 bytes from different banks and write
    // to different banks, halves of two tokens that the swizzle sends to even and odd places
    const int quarter = lane >> 3, pair = lane >> 2 & 1;
    const int my_token = D == 128 ? 2 * (quarter & 1) + pair : lane >> 2;
    const int my_piece = D == 128 ? 4 * ((quarter >> 1) ^ pair) + (lane & 3) : lane & 3;
    constexpr int kStep = 32 / kPieces;                             // tokens at a time
    bool ok = true;
    while (ok && take(seg)) {
      const uint8_t* ks = seg.prefix ? a.pk_scale : a.k_scale;
      const uint8_t* vs = seg.prefix ? a.pv_scale : a.v_scale;
      const size_t base = ((size_t)seg.row * a.Hkv + seg.head) * (seg.prefix ? a.prefix_cap : a.path_cap);
      ok = each_tile(seg, [&](bool v, int j) {
        // scales of the warp's tokens, a lane each; 2^(s - 127 + 120), in two factors where that is more than a bfloat16 holds; 0 behind the last key
        const int key = j * kTile + token0 + (lane & (kTokens - 1));
        const int sc = key < seg.keys ? (v ? vs : ks)[base + key] : 0, e = min(sc + 120, 254);
        // (V of a new token that reads as NaN: nothing, and a total of NaN for those that see it)
        const bool noted = v && sc == 255 && key >= seg.whole && key < seg.keys && doubtful(seg);
        if (noted) atomicOr(&sh.unfinite[seg.place], 1ull << (key - seg.whole));
        const uint32_t first = (key >= seg.keys || noted ? 0u : sc == 255 ? 0x7fc0u : (uint32_t)e << 7) * 0x10001u, second = (uint32_t)(sc + 120 - e + 127) * 0x800080u;
        const bool large = __any_sync(~0u, sc > 134 && sc < 255);
        if (!__all_sync(~0u, bar_wait(&bars.raw_full[raw], phase_raw, &dead) && bar_wait(&bars.empty[slot], phase, &dead))) return false;
        const unsigned char* from = sm_raw + raw * S::kRaw + (token0 + my_token) * D + my_piece * 16;
        unsigned char* to = sm_kv + slot * S::kOperand + (my_piece >> 2) * kBlock + (token0 + my_token) * 128;
        uint32_t most = 0;                                          // of the codes without their signs, one in each half
#pragma unroll
        for (int x = 0; x < kTokens; x += kStep) {
          const uint4 w = *reinterpret_cast<const uint4*>(from + x * D);
          const uint32_t g1 = __shfl_sync(~0u, first, x + my_token);
          const uint32_t in[4] = {w.x, w.y, w.z, w.w};
          uint32_t out[8], before = 0;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint32_t t = __byte_perm(in[k >> 1], 0u, k & 1 ? 0x3322 : 0x1100);
            const uint32_t size = t << 4 & 0x07f007f0u, b = (t & 0x80008000u) | size;
            if (k & 1) most = __vimax3_u16x2(most, size, before);
            before = size;
            const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&b), *reinterpret_cast<const __nv_bfloat162*>(&g1));
            out[k] = *reinterpret_cast<const uint32_t*>(&y);
          }
          if (large) {
            const uint32_t g2 = __shfl_sync(~0u, second, x + my_token);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&out[k]), *reinterpret_cast<const __nv_bfloat162*>(&g2));
              out[k] = *reinterpret_cast<const uint32_t*>(&y);
            }
          }
          unsigned char* at = to + x * 128;
          const int c0 = (my_piece & 3) * 2, r = (my_token + x) & 7;                // (token0 is a multiple of eight)
          *reinterpret_cast<uint4*>(at + ((c0 ^ r) << 4)) = make_uint4(out[0], out[1], out[2], out[3]);
          *reinterpret_cast<uint4*>(at + (((c0 + 1) ^ r) << 4)) = make_uint4(out[4], out[5], out[6], out[7]);
        }
        // 256 * 2^120, which the largest bfloat16 is stored as, is none itself: what has become infinite is the largest number.  (NaN stays.  A loop of its own:
        // in the one above the largest and smallest of two cost 1.5 us of 75 where no scale is large.)
        if (large) {
#pragma unroll 1
          for (int x = 0; x < kTokens; x += kStep)
#pragma unroll 1
            for (int k = 0; k < 8; ++k) {
              uint32_t* at = reinterpret_cast<uint32_t*>(to + x * 128 + ((((my_piece & 3) * 2 + (k >> 2)) ^ ((my_token + x) & 7)) << 4)) + (k & 3);
              uint32_t y = *at;
              if ((y & 0x7fffu) == 0x7f80u) y -= 1u;
              if ((y & 0x7fff0000u) == 0x7f800000u) y -= 0x10000u;
              *at = y;
            }
        }
        // The code that is not a number, 0x7f, read as 480 above.  (Hardly ever there.)
        if ((most + 0x00100010u) & 0x08000800u) {
#pragma unroll 1
          for (int i = 0; i < kTokens / kStep * 16; ++i) {
            const int x = (i >> 4) * kStep, k = i & 15, t = token0 + my_token + x, key2 = j * kTile + t;
            if ((from[x * D + k] & 0x7f) != 0x7f || key2 >= seg.keys) continue;
            const bool note = v && key2 >= seg.whole && doubtful(seg);
            *reinterpret_cast<uint16_t*>(to + x * 128 + ((((my_piece & 3) * 2 + (k >> 3)) ^ (t & 7)) << 4) + (k & 7) * 2) = note ? 0 : 0x7fc0;
            if (note) atomicOr(&sh.unfinite[seg.place], 1ull << (key2 - seg.whole));
          }
        }
        fence_async();
        __syncwarp();
        if (lane == 0) { bar_arrive(&bars.raw_empty[raw]); bar_arrive(&bars.full[slot]); }
        if (++slot == S::kStages) { slot = 0; phase ^= 1; }
        if (++raw == S::kRawStages) { raw = 0; phase_raw ^= 1; }
        return true;
      });
    }
  }
  if (warp == kDealer) {
    // ---- segments: CTA c has units [total * c / ctas, total * (c + 1) / ctas) ----
    // 32 entries, one a lane
    struct Entry { int keys, whole, queries; Cost cost; };
    auto entry_of = [&](int e) {
      Entry x{0, 0, 0, Cost{0u, 0u}};
      if (e >= entries) return x;
      x.keys = x.whole = keys_of(a, e);
      x.cost = cost_of(a, plan, e, x.keys);
      if (e >= a.G && x.keys) {
        x.whole = min(max(a.len[e - a.G], 0), a.path_cap);
        x.queries = queries_of(a, e - a.G);
      }
      return x;
    };
    Entry mine = entry_of(lane);
    uint32_t plain = mine.cost.plain, full = mine.cost.full;
    if (chunks > 1) {
      plain = full = 0;
      for (int i = lane; i < min(chunks, kMostChunks); i += 32) { plain += chunk_cost[i].x; full += chunk_cost[i].y; }
    }
    plain = __reduce_add_sync(~0u, plain);
    full = __reduce_add_sync(~0u, full);
    for (int i = kMostChunks; i < chunks; ++i) {                    // (thousands of paths)
      const uint2 x = cost_of_chunk(i);
      plain += x.x; full += x.y;
    }
    // Full costs where every CTA has several tiles.  Each has at least as many units as lie between the beginnings of two tiles of an item, so that
    // every CTA between an item's first and last has a tile of it (a tile is the CTA's that has its first unit).
    const bool many = plain >= 8 * kCtas;
    const uint32_t begin = many ? kBegin : 0, of_few = many ? few_cost(QUANT) : 1, of_one = many ? one_cost(QUANT) : 1, of_two = many ? kTwo : 2;
    const uint32_t total = many ? full : plain;
    const uint32_t least = many ? begin + of_two : plan.pre_plain > 1 || plan.own_plain > 1 ? 2 : 1;
    static_assert(8 * kFew >= kBegin + kTwo, "with full costs there is work for all CTAs");
    const uint32_t block = blockIdx.x, ctas = total ? max(1u, min((uint32_t)kCtas, total / least)) : 0;
    uint32_t u = block < ctas ? (uint32_t)((uint64_t)total * block / ctas) : total;
    const uint32_t end = block < ctas ? (uint32_t)((uint64_t)total * (block + 1) / ctas) : total;
    int dealt = 0;
    bool ok = true;
    auto deal = [&](const Segment& s) {
      const int i = dealt % kSegments;
      ok = dealt < kSegments || __all_sync(~0u, bar_wait(&bars.seg_empty[i], dealt / kSegments + 1 & 1, &dead));
      if (ok && lane == 0) {
        sh.segment[i] = s;
        sh.segment[i].place = dealt % kPlaces;
        sh.unfinite[dealt % kPlaces] = 0;
        bar_arrive(&bars.seg_full[i]);
      }
      __syncwarp();
      ++dealt;
    };
    // the 32 entries that its first unit is in
    uint32_t before = 0;
    int chunk = 0;
    for (; chunks > 1 && chunk < chunks && u < end; chunk += 32) {
      const uint2 x = chunk + lane < min(chunks, kMostChunks) ? chunk_cost[chunk + lane] : make_uint2(0u, 0u);
      uint32_t upto = many ? x.y : x.x;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t other = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += other;
      }
      upto += before;
      const uint32_t in = __ballot_sync(~0u, upto > u);
      if (in || chunk + 32 >= kMostChunks) {
        const int src = in ? __ffs(in) - 1 : 31;                    // (beyond what is noted: one chunk after the other, below)
        if (src > 0) before = __shfl_sync(~0u, upto, src - 1);
        chunk += src;
        break;
      }
      before = __shfl_sync(~0u, upto, 31);
    }
    for (int e0 = chunk * 32; e0 < entries && u < end && ok; e0 += 32) {
      if (e0 > 0) mine = entry_of(e0 + lane);
      const int keys = mine.keys, whole = mine.whole, queries = mine.queries;
      const uint32_t units = many ? mine.cost.full : mine.cost.plain;
      uint32_t upto = units;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t other = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += other;
      }
      upto += before;
      const uint32_t chunk_end = __shfl_sync(~0u, upto, 31);
      while (u < end && u < chunk_end && ok) {
        const int src = __ffs(__ballot_sync(~0u, upto > u)) - 1;
        Segment s;
        s.entry = e0 + src;
        s.keys = __shfl_sync(~0u, keys, src);
        s.whole = __shfl_sync(~0u, whole, src);
        s.queries = __shfl_sync(~0u, queries, src);
        s.prefix = s.entry < a.G;
        const uint32_t tiles = (uint32_t)tiles_of(s.keys), m_tiles = s.prefix ? plan.pre_tiles_m : plan.own_tiles_m;
        const uint32_t weight = many ? (s.prefix ? plan.pre_cost : plan.own_cost) : (s.prefix ? plan.pre_plain : plan.own_plain);
        uint32_t unit = u - __shfl_sync(~0u, upto - units, src);
        const uint32_t per_head = tiles * weight + begin * m_tiles, per_item = of_two * tiles + begin;       // (an item but the last of a head)
        s.head = (int)(unit / per_head);
        unit -= s.head * per_head;
        const uint32_t mt = m_tiles == 1 ? 0 : min(unit / per_item, m_tiles - 1);
        unit -= mt * per_item;
        s.row0 = (int)mt * 2 * kTile;
        s.rows = min(2 * kTile, (s.prefix ? plan.pre_rows : plan.own_rows) - s.row0);
        const uint32_t each = s.rows > kTile ? of_two : s.rows > kFewRows ? of_one : of_few, some = min(tiles * each + begin - unit, end - u);
        // the first tile that does not begin in front of unit x of the item
        auto tile_from = [&](uint32_t x) { return x == 0 ? 0u : max(1u, x > begin ? (x - begin + each - 1) / each : 0u); };
        s.j0 = (int)min(tile_from(unit), tiles);
        s.n = (int)min(tile_from(unit + some), tiles) - s.j0;
        const uint32_t item = s.head * m_tiles + mt;
        s.dual = s.rows > kTile;
        s.row = s.prefix ? s.entry : s.entry - a.G;
        s.item = s.row * a.Hkv * (int)m_tiles + (int)item;
        s.first = s.j0 == 0;
        s.last = s.j0 + s.n == (int)tiles;
        u += some;
        if (s.n > 0) deal(s);
      }
      before = chunk_end;
    }
    if (ok) {
      Segment s{};
      deal(s);
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  // Given up, whichever warp it was: tiles and products that are under way, asked for by warps that came to their own end, arrive before memory is given back, or a
  // millisecond has passed.  (Nobody asks for any behind the barrier.)
  if (dead)
    for (const long long begin = clock64(); clock64() - begin < 2000000;) {}
  if (warp == 9) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tensor), "r"(kTensorColumns) : "memory");
  }
  if (tid == 0 && dead && a.status) atomicOr(a.status, SDMS_STATUS_TIMEOUT);
}

// ---- the parts of an output row put together: a warp per row -----------------------------------------------------------------------

constexpr int kJoinThreads = 128;

template <int D, bool BF16>
__global__ void __launch_bounds__(kJoinThreads) attend_join_kernel(const AttendDev a) {
  grid_wait();
  grid_release();
  const int id = blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (id >= a.P * a.T * a.Hq) return;
  int hq, t;
  const int pt = divide(id, a.per_row, &hq), p = divide(pt, a.per_query, &t), g = a.G == 1 ? 0 : p / a.N;
  const Plan plan = plan_of(a);
  const Parts parts = parts_of(a, plan);
  int j;
  const int h = divide(hq, a.per_token, &j);
  // the row's parts in the prefix and among the path's own: from a first row on, one every slot
  const int r_pre = ((p - g * a.N) * a.T + t) * a.group + j, r_own = t * a.group + j;
  const int i_pre = (g * a.Hkv + h) * plan.pre_tiles_m + r_pre / (2 * kTile), i_own = (p * a.Hkv + h) * plan.own_tiles_m + r_own / (2 * kTile);
  const int2 c_pre = parts.range[i_pre], c_own = parts.range[plan.pre_items + i_own];
  const int keys_pre = keys_of(a, g), keys_own = keys_of(a, a.G + p);
  if (t >= queries_of(a, p)) return;
  const PartRun pre = part_run(c_pre.x, c_pre.y), own = part_run(c_own.x, c_own.y);
  const int n_pre = keys_pre ? pre.count : 0, n_own = keys_own ? own.count : 0, parts_n = n_pre + n_own;
  const long long first_pre = part_row(plan, true, i_pre, pre.first) + r_pre % (2 * kTile);
  const long long first_own = part_row(plan, false, i_own, own.first) + r_own % (2 * kTile);
  auto row_of = [&](int i) { return i < n_pre ? first_pre + (long long)i * plan.pre_slot : first_own + (long long)(i - n_pre) * plan.own_slot; };
  // Eight parts at a time, sums, references and totals under way together (18 parts a row: 7.3 us; four at a time, behind their references, 10.7;
  // sixteen 6.7, but 11.5 for 9.0 where rows have two or three).
  constexpr int W = D / 32, kAtOnce = 8;
  float acc[W];
#pragma unroll
  for (int i = 0; i < W; ++i) acc[i] = 0.f;
  float most = -INFINITY, l = 0.f;
  for (int i0 = 0; i0 < parts_n; i0 += kAtOnce) {
    const bool mine = lane < kAtOnce && i0 + lane < parts_n;
    const float2 ml = mine ? parts.ml[row_of(i0 + lane)] : make_float2(-INFINITY, 0.f);
    float x[kAtOnce][W];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (i0 + k >= parts_n) continue;                 // (the same in all lanes)
      const float* from = parts.o + row_of(i0 + k) * D + lane * W;
      if (W == 4) {
        const float4 v = *reinterpret_cast<const float4*>(from);
        x[k][0] = v.x; x[k][1] = v.y; x[k][W - 2] = v.z; x[k][W - 1] = v.w;
      } else {
        const float2 v = *reinterpret_cast<const float2*>(from);
        x[k][0] = v.x; x[k][1] = v.y;
      }
    }
    float top = ml.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    top = fmaxf(top, most);
    const float ref = top == -INFINITY ? 0.f : top, old = exp2_fast(most - ref);
    most = top;
    const bool use = mine && !(ml.y == 0.f);           // (rows that saw nothing: what lies there may be anything; not NaN)
    const float w = use ? exp2_fast((ml.x == -INFINITY ? 0.f : ml.x) - ref) : 0.f;
    float part = w * ml.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(~0u, part, o);
    l = fmaf(l, old, part);
    const uint32_t used = __ballot_sync(~0u, use);
#pragma unroll
    for (int i = 0; i < W; ++i) acc[i] *= old;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const float f = __shfl_sync(~0u, w, k);
      if (used >> k & 1)
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] = fmaf(f, x[k][i], acc[i]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t* out = a.out + p * a.o_path + t * a.o_token + hq * a.o_head + lane * W;
  if (W == 4) *reinterpret_cast<uint2*>(out) = make_uint2(pack<BF16>(acc[0] * inv, acc[1] * inv), pack<BF16>(acc[W - 2] * inv, acc[W - 1] * inv));
  else *reinterpret_cast<uint32_t*>(out) = pack<BF16>(acc[0] * inv, acc[1] * inv);
}

// ---- host --------------------------------------------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

// Tiles of 128 tokens of one head of one row: 64 elements of 16 bits wide, swizzled as the products read them, or all of a head's 8 bits.
bool encode(CUtensorMap* map, const KvDev& kv, void* base, bool bf16) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const int b = kv.bytes_per_element;
  const cuuint64_t dims[4] = {(cuuint64_t)kv.head_dim, (cuuint64_t)kv.capacity, (cuuint64_t)kv.heads, (cuuint64_t)kv.rows};
  const cuuint64_t strides[3] = {(cuuint64_t)kv.stride_token * b, (cuuint64_t)kv.stride_head * b, (cuuint64_t)kv.stride_row * b};
  const cuuint32_t box[4] = {(cuuint32_t)(b == 1 ? kv.head_dim : 64), (cuuint32_t)kTile, 1, 1}, step[4] = {1, 1, 1, 1};
  return f(map, b == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dims, strides,
           box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, b == 1 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool QUANT, bool BF16>
cudaError_t launch_d(const Maps& maps, const AttendDev& a, cudaStream_t stream) {
  using S = Shape<D, QUANT>;
  const auto kernel = attend_kernel<D, QUANT, BF16>;
  const size_t smem = S::kBytes + sizeof(Shared<S>);
  static_assert(S::kBytes + sizeof(Shared<S>) <= 227 * 1024, "what a CTA can have");
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_shared(kernel, smem, &allowed);
  if (e != cudaSuccess) return e;
  e = launch_overlapped(kernel, dim3(kCtas), dim3(S::kThreads), smem, stream, maps, a);
  if (e != cudaSuccess) return e;
  const long long rows = (long long)a.P * a.T * a.Hq;
  return launch_overlapped(attend_join_kernel<D, BF16>, dim3((unsigned)((rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32))), dim3(kJoinThreads), 0, stream,
                           a);
}

}  // namespace

size_t attend_bytes(const AttendDev& a) {
  const Plan p = plan_of(a);
  return p.range_bytes + p.o_bytes + (size_t)part_rows(p) * sizeof(float2);
}

cudaError_t launch_attend(const AttendDev& a, const KvDev* prefix, const KvDev* paths, cudaStream_t stream) {
  Maps maps{};
  if (prefix && (!encode(&maps.pre_k, *prefix, prefix->k, a.bf16) || !encode(&maps.pre_v, *prefix, prefix->v, a.bf16))) return cudaErrorInvalidValue;
  if (paths && (!encode(&maps.own_k, *paths, paths->k, a.bf16) || !encode(&maps.own_v, *paths, paths->v, a.bf16))) return cudaErrorInvalidValue;
  const bool quant = a.pk_scale || a.k_scale;
  if (quant) return a.d == 64 ? launch_d<64, true, true>(maps, a, stream) : launch_d<128, true, true>(maps, a, stream);
  if (a.bf16) return a.d == 64 ? launch_d<64, false, true>(maps, a, stream) : launch_d<128, false, true>(maps, a, stream);
  return a.d == 64 ? launch_d<64, false, false>(maps, a, stream) : launch_d<128, false, false>(maps, a, stream);
}

}  // namespace sdms
