// K/V caches: tokens written at the ends of the rows (quantised where the cache is), rows that follow other rows.
//
// sdms_kv_append   scale of a token and head: the smallest power of two 2^b with max |x| <= 448 * 2^b.  A power of two loses
//                  nothing that 8 bits with an exponent would keep (x / 2^b has x's own mantissa), costs one byte, and makes what attention
//                  reads back, code * 2^b, exact in bfloat16: the products see it without a second rounding.  (But for 256 * 2^120, which numbers
//                  next to the largest bfloat16 round to.)
//                  32 x 4096 tokens of 8 heads of 128: 16 bits 163 us, 6.6 TB/s, the memory's rate; 8 bits 167 us, 4.85 TB/s, bounded by instructions (74 %
//                  of issue slots, DRAM 44 %).  512 x 9: 6.2 and 7.7 us, a launch and four to five waves of CTAs of one item a thread.
// sdms_kv_reorder  copies of rows, bounded by bytes: 278 to 296 us for 2.0 GB read and written (what was read twice comes from the L2), 7.6 for 16 rows of
//                  1024 (8.5 called one by one).
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include "decode_internal.h"

namespace sdms {

namespace {

constexpr int kKvThreads = 256;

// Eight elements of a token's head a thread: 16 lanes for a head of 128, 8 for one of 64, both groups of lanes of one warp.
// `items` = tokens * heads * lanes of a row; K and V are blockIdx.z.  (Ordinary loads: what comes in may be what the kernel before
// this one writes, which this one is resident with.)
// ROUNDS > 1: a CTA has that many times four items a thread, and writes the scales, a byte a token and head that lie a whole row apart from token to
// token where they are computed, from shared memory head by head (32 x 4096 tokens: 193 to 166 us).
template <bool QUANT, int UNROLL, int ROUNDS>
__global__ void __launch_bounds__(kKvThreads) kv_append_kernel(KvDev kv, const uint4* k_new, const uint4* v_new, int tokens, const int32_t* len,
                                                               const int32_t* count, int items, int blocks_per_row) {
  constexpr bool kStaged = QUANT && ROUNDS > 1;
  constexpr int kVectors = kKvThreads * UNROLL * ROUNDS / 8;        // at most, of a CTA
  __shared__ uint8_t scales[kStaged ? kVectors : 1];
  grid_wait();
  grid_release();
  const int row = blockIdx.x / blocks_per_row;
  const int start = (blockIdx.x - row * blocks_per_row) * (kKvThreads * UNROLL * ROUNDS);
  const int at0 = max(len[row], 0);
  int n = count ? min(max(count[row], 0), tokens) : tokens;
  n = min(n, max(kv.capacity - at0, 0));
  const uint4* src = (blockIdx.z ? v_new : k_new) + (size_t)row * items;
  const int shift = kv.head_dim == 128 ? 4 : 3, lanes = 1 << shift;
  const int live = n * (kv.heads << shift);            // items of tokens that are there (a token's lanes are there or not together)
  if (start >= live) return;
  uint8_t* to_scale = QUANT ? (blockIdx.z ? kv.v_scale : kv.k_scale) + (size_t)row * kv.heads * kv.capacity + at0 : nullptr;
#pragma unroll 1
  for (int round = 0; round < ROUNDS; ++round) {
    const int first = start + round * (kKvThreads * UNROLL) + threadIdx.x;
    uint4 x[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int i = first + u * kKvThreads;
      x[u] = i < live ? src[i] : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int i = first + u * kKvThreads;
      const int vector = i >> shift, lane = i & (lanes - 1), t = vector / kv.heads, head = vector - t * kv.heads;
      const size_t at = (size_t)row * kv.stride_row + (size_t)(at0 + t) * kv.stride_token + (size_t)head * kv.stride_head + lane * 8;
      if (!QUANT) {
        if (i < live) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(blockIdx.z ? kv.v : kv.k) + at) = x[u];
        continue;
      }
      // largest magnitude of the vector: the bit patterns of magnitudes are ordered as the magnitudes are, infinities and NaN above all
      uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) most = max(most, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1)
        if (o < lanes) most = max(most, __shfl_xor_sync(~0u, most, o));
      if (i >= live) continue;
      // amax = 1.m * 2^(e - 127) in bfloat16 (7 bits of m); 448 = 1.75 * 2^8, so b = e - 127 - 8, one more above a mantissa of 1.75 (0x60)
      const int e = most >> 7, m = most & 0x7f;
      int s = e - 8 + (m > 0x60 ? 1 : 0);              // b + 127
      s = most >= 0x7f80u ? 255 : max(s, 0);
      // 2^-b: exact, as are the products down to where the 8 bits have long become 0
      const float inv = s == 255 ? 0.f : __uint_as_float((uint32_t)(254 - s) << 23);
      uint32_t out[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float f[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t h = (w[2 * j + (c >> 1)] >> ((c & 1) * 16)) << 16;
          f[c] = s == 255 ? 0.f : __uint_as_float(h) * inv;
        }
        const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[0], f[1]), __NV_SATFINITE, __NV_E4M3);
        const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[2], f[3]), __NV_SATFINITE, __NV_E4M3);
        out[j] = (uint32_t)lo | (uint32_t)hi << 16;
      }
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(blockIdx.z ? kv.v : kv.k) + at) = make_uint2(out[0], out[1]);
      if (lane == 0) {
        if (kStaged) scales[vector - (start >> shift)] = (uint8_t)s;
        else to_scale[(size_t)head * kv.capacity + t] = (uint8_t)s;
      }
    }
  }
  if (!kStaged) return;
  __syncthreads();
  // head by head, a token a lane: vectors first .. last - 1 are (token, head) in that order
  const int first = start >> shift, last = min(first + (kKvThreads * UNROLL * ROUNDS >> shift), live >> shift);
  const int t0 = first / kv.heads, t1 = (last - 1) / kv.heads + 1, width = t1 - t0;
  for (int i = threadIdx.x; i < width * kv.heads; i += kKvThreads) {
    const int head = i / width, t = t0 + i - head * width, vector = t * kv.heads + head;
    if (vector >= first && vector < last) to_scale[(size_t)head * kv.capacity + t] = scales[vector - first];
  }
}

// Row p = blockIdx.y takes a run of tokens over from its parent; K and V are blockIdx.z.
__global__ void __launch_bounds__(kKvThreads) kv_reorder_kernel(KvDev kv, const int32_t* parent, const int32_t* len, int paths_per_group, int chunk) {
  grid_wait();
  grid_release();
  const int p = blockIdx.y, q = parent[p];
  if (q == p || q < 0 || q >= kv.rows || q / paths_per_group != p / paths_per_group || parent[q] != q) return;
  const int n = min(max(len[q], 0), kv.capacity);
  const int t0 = blockIdx.x * chunk, t1 = min(t0 + chunk, n);
  if (t0 >= t1) return;
  const int bytes = kv.bytes_per_element, pieces = kv.head_dim * bytes / 16, per_token = kv.heads * pieces;
  char* base = static_cast<char*>(blockIdx.z ? kv.v : kv.k);
  const char* from = base + (size_t)q * kv.stride_row * bytes;
  char* to = base + (size_t)p * kv.stride_row * bytes;
  const int total = (t1 - t0) * per_token;
  constexpr int kUnroll = 8;
  for (int i0 = threadIdx.x; i0 < total; i0 += kKvThreads * kUnroll) {
    uint4 x[kUnroll];
    size_t at[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int i = i0 + u * kKvThreads;
      const int t = i / per_token, rest = i - t * per_token, head = rest / pieces, piece = rest - head * pieces;
      at[u] = ((size_t)(t0 + t) * kv.stride_token + (size_t)head * kv.stride_head) * bytes + (size_t)piece * 16;
      if (i < total) x[u] = *reinterpret_cast<const uint4*>(from + at[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i0 + u * kKvThreads < total) *reinterpret_cast<uint4*>(to + at[u]) = x[u];
  }
  uint8_t* scale = blockIdx.z ? kv.v_scale : kv.k_scale;
  if (scale)
    for (int i = threadIdx.x; i < kv.heads * (t1 - t0); i += kKvThreads) {
      const int head = i / (t1 - t0), t = t0 + i - head * (t1 - t0);
      scale[((size_t)p * kv.heads + head) * kv.capacity + t] = scale[((size_t)q * kv.heads + head) * kv.capacity + t];
    }
}

}  // namespace

cudaError_t launch_kv_append(const KvDev& kv, const void* k_new, const void* v_new, int tokens, const int32_t* len, const int32_t* count,
                             cudaStream_t stream) {
  const int items = tokens * kv.heads * (kv.head_dim / 8);
  const bool many = (long long)items * kv.rows * 2 >= 148LL * 2048 * 16;
  const int per_cta = kKvThreads * (many ? 16 : 1), blocks = (items + per_cta - 1) / per_cta;
  const auto kernel = kv.k_scale ? (many ? kv_append_kernel<true, 4, 4> : kv_append_kernel<true, 1, 1>)
                                 : (many ? kv_append_kernel<false, 4, 4> : kv_append_kernel<false, 1, 1>);
  return launch_overlapped(kernel, dim3((unsigned)(kv.rows * blocks), 1, 2), dim3(kKvThreads), 0, stream, kv, static_cast<const uint4*>(k_new),
                           static_cast<const uint4*>(v_new), tokens, len, count, items, blocks);
}

cudaError_t launch_kv_reorder(const KvDev& kv, const int32_t* parent, const int32_t* len, int paths_per_group, cudaStream_t stream) {
  const int per_token = kv.heads * kv.head_dim * kv.bytes_per_element / 16;
  // a CTA's part: four rounds of its loads; one where there are too few CTAs for every SM otherwise (16 rows of 1024 tokens, 6 of them copied: 11.4 us with four, 7.8)
  const int rounds = (long long)kv.rows * kv.capacity * per_token >= 1LL << 25 ? 4 : 1;
  const int chunk = (rounds * 8 * kKvThreads + per_token - 1) / per_token;
  return launch_overlapped(kv_reorder_kernel, dim3((unsigned)((kv.capacity + chunk - 1) / chunk), (unsigned)kv.rows, 2), dim3(kKvThreads), 0, stream, kv,
                           parent, len, paths_per_group, chunk);
}

}  // namespace sdms
