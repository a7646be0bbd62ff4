// Beam search's selection: the N best of a prompt's N * V continuations, and where they go.
//
// Candidate (path r, token v) is worth s_r + x_rv - lse_r, lse_r = log sum_v exp x_rv.  Inside a path the order is that of the logits, so one
// pass over them (beam_rows_kernel, a CTA per chunk of a row, held in registers) finds both the chunk's share of the sum and its N best
// tokens; only across paths do the sums matter (beam_merge_kernel, a CTA per prompt).
//
// Two candidates of different paths can lie as near to each other as their sums are exact, so the sums are: exp in 32 bits (1 ulp each, of
// either sign), added without rounding error to speak of (Sum, exp_neg), chunks joined and candidates compared in 64 bits.
//
// The N best of a chunk, without sorting it: split its threads into N groups or more; N different elements at least are no less than the smallest
// of the groups' largest elements.  What is no less than that bound (N * H(N) elements of random data: 54 for N = 16) is listed and sorted.
// The merge does the same with the chunks' best for elements.
//
// Where a row's chunks do not all run at once, later ones know how good the N best of an earlier one are (a word a row, which only goes up): what lies
// below is not listed.  Which chunk knew of which changes what is listed, never what is selected.
//
// What bounds it: 32 x 16 rows of 151936 in 16 bits take 96 us, of which the bytes are 21.  Neither the memory (16 % busy) nor the issue slots (69 % used) are
// full: a CTA waits for its chunk, and the loads overlap with the three other CTAs of its SM only.  By leaving parts out: loads, maximum and bound 50, sums 20, the
// rest listing and sorting (39 where no chunk knows of another: 108 us).  1 x 16 of 128256: 14 to 15, 1 x 4 of 32000: 8.1 in a graph, 11 by a call, the two launches'
// chain of latencies.  Prompts of many paths, the merge's one CTA and the rows' lists: 1 x 256 of 32000 222 us, of 151936 303; 1 x 64 of 128256 77.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include "decode_dev.cuh"

namespace sdms {

namespace {

constexpr int kRowThreads = 256;
constexpr int kRowList = 2048, kList = 2048;   // candidates listed by a CTA of the one kernel and the other
static_assert((kRowList & (kRowList - 1)) == 0 && (kList & (kList - 1)) == 0, "sorting fills a list up to a power of two");
static_assert(kList >= 2 * SDMS_MAX_BEAM_PATHS && kRowList >= SDMS_MAX_BEAM_PATHS, "the N best and another list's");
static_assert((SDMS_MAX_BEAM_PATHS & (SDMS_MAX_BEAM_PATHS - 1)) == 0 && SDMS_MAX_BEAM_PATHS <= kRowThreads, "a group is a thread at least");
constexpr int kMergeThreads = 512;
constexpr int kRanked = 384;              // candidates up to which ranks are counted instead of sorting (1024: 1 x 128 rows of 151936 183 for 126 us)
constexpr int kKnownFrom = 4 * 148 * 4;

struct ChunkHead { double sum; unsigned long long best; float most; int32_t unused; };      // sum of exp(x - most); best = 0: not one token

size_t align256(size_t x) { return (x + 255) / 256 * 256; }
// (elements of a row that a CTA holds: fewer where there would not be a CTA for every SM)
int chunk_of(int rows, int vocab) {
  if ((long long)rows * ((vocab + 8191) / 8192) >= 240) return 8192;
  return (long long)rows * ((vocab + 4095) / 4096) >= 240 ? 4096 : 2048;
}
int chunks_of(int rows, int vocab) {
  const int c = chunk_of(rows, vocab);
  return (vocab + c - 1) / c;
}

// Larger value first, then smaller token; 0 = no candidate.  (Floats as integers in the order of their values; -0 has become +0.)
__device__ __forceinline__ unsigned long long key_of(float x, int token) {
  const uint32_t b = __float_as_uint(x);
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (unsigned long long)o << 32 | (uint32_t)~token;
}
__device__ __forceinline__ float value_of(unsigned long long key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int token_of(unsigned long long key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ unsigned long long order_of(double x) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(x);
  return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double worth_of(unsigned long long o) { return __longlong_as_double((long long)(o >> 63 ? o & ~(1ull << 63) : ~o)); }

// Sums of up to 16 pairs of numbers in [0, 1]: each number is split into a multiple of 2^-13 and the rest, so that the upper parts add without
// rounding and the rounding of the lower ones stays below 2^-33.
struct Sum {
  Pair hi = Pair::of(0.f, 0.f), lo = Pair::of(0.f, 0.f);
  __device__ __forceinline__ void add(Pair x) {
    const Pair c = Pair::of(1536.f, 1536.f), minus_c = Pair::of(-1536.f, -1536.f), minus_1 = Pair::of(-1.f, -1.f);       // 1.5 * 2^10: its last place is 2^-13
    const Pair h = sdms::add(sdms::add(x, c), minus_c);
    hi = sdms::add(hi, h);
    lo = sdms::add(lo, sdms::fma(h, minus_1, x));
  }
  __device__ __forceinline__ double value() const {
    float a, b, c, d;
    hi.split(&a, &b); lo.split(&c, &d);
    return ((double)a + (double)b) + ((double)c + (double)d);
  }
};

// exp(d), -250 < d <= 0: 2^(d log2 e) with the product in two parts, a + b, 2^a as the hardware has it (2^-22.5 at most) and 2^b = 1 + b ln 2, which
// is below 2^-22 of 1 from it.
__device__ __forceinline__ Pair exp_neg(Pair d) {
  constexpr double log2e = 1.4426950408889634074;
  constexpr float high = (float)log2e, low = (float)(log2e - (double)high), ln2 = 0.69314718055994531f;
  const Pair h = Pair::of(high, high), a = mul(d, h), minus_a = mul(a, Pair::of(-1.f, -1.f));
  const Pair b = fma(d, Pair::of(low, low), fma(d, h, minus_a));
  float x, y;
  a.split(&x, &y);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(y));
  const Pair e = Pair::of(x, y);
  return fma(e, mul(b, Pair::of(ln2, ln2)), e);
}

template <class T> struct Vec;
template <> struct Vec<float> {
  static constexpr int kSize = 4;
  static constexpr uint32_t kNone = 0xff800000u;       // -infinity
  static __device__ __forceinline__ float top() { return 3.402823466e38f; }
  static __device__ __forceinline__ void unpack(uint4 w, float* x) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ float most(uint4 w) {
    return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
  }
  static __device__ __forceinline__ float one(float x) { return x; }
  static __device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x); }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int kSize = 8;
  static constexpr uint32_t kNone = 0xff80ff80u;
  static __device__ __forceinline__ float top() { return __uint_as_float(0x7f7f0000u); }
  static __device__ __forceinline__ void unpack(uint4 w, float* x) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(v[j] << 16); x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u); }
  }
  static __device__ __forceinline__ float most(uint4 w) {
    const __nv_bfloat162* v = reinterpret_cast<const __nv_bfloat162*>(&w);
    const __nv_bfloat162 m = __hmax2(__hmax2(v[0], v[1]), __hmax2(v[2], v[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x) >> 16; }
};
template <> struct Vec<__half> {
  static constexpr int kSize = 8;
  static constexpr uint32_t kNone = 0xfc00fc00u;
  static __device__ __forceinline__ float top() { return 65504.f; }
  static __device__ __forceinline__ void unpack(uint4 w, float* x) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v[j]));
      x[2 * j] = f.x; x[2 * j + 1] = f.y;
    }
  }
  static __device__ __forceinline__ float most(uint4 w) {
    const __half2* v = reinterpret_cast<const __half2*>(&w);
    const __half2 m = __hmax2(__hmax2(v[0], v[1]), __hmax2(v[2], v[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ float one(__half x) { return __half2float(x); }
  static __device__ __forceinline__ uint32_t bits(float x) { return __half_as_ushort(__float2half_rn(x)); }
};
// A logit that is not a number is not there; +infinity counts as the largest.
template <class T>
__device__ __forceinline__ float cleaned(float x) { return x == x ? fminf(x, Vec<T>::top()) : -INFINITY; }
template <class T>
__device__ __forceinline__ uint4 packed(const float* x) {
  if constexpr (Vec<T>::kSize == 4) return make_uint4(Vec<T>::bits(x[0]), Vec<T>::bits(x[1]), Vec<T>::bits(x[2]), Vec<T>::bits(x[3]));
  else {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = Vec<T>::bits(x[2 * j]) | Vec<T>::bits(x[2 * j + 1]) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// W elements from `skew` elements into a on; b is the aligned vector behind a.  (One of W uniform cases, so that no word is picked by a
// variable index.)
template <int SHIFT>
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b) {
  const uint32_t w[9] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, 0u};
  constexpr int i = SHIFT / 4, bits = SHIFT % 4 * 8;
  return make_uint4(__funnelshift_r(w[i], w[i + 1], bits), __funnelshift_r(w[i + 1], w[i + 2], bits), __funnelshift_r(w[i + 2], w[i + 3], bits),
                    __funnelshift_r(w[i + 3], w[i + 4], bits));
}
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, int bytes) {
  switch (bytes) {
    case 2: return shifted<2>(a, b);
    case 4: return shifted<4>(a, b);
    case 6: return shifted<6>(a, b);
    case 8: return shifted<8>(a, b);
    case 10: return shifted<10>(a, b);
    case 12: return shifted<12>(a, b);
    case 14: return shifted<14>(a, b);
    default: return a;
  }
}

// Sorts list[0, count) downwards (count <= kList); all threads of the CTA take part.  Short lists: every element's rank is counted.
template <int THREADS, class Less, class E>
__device__ void sort_down(E* list, int count, Less less) {
  if (count <= THREADS && count <= 256) {
    E mine{};
    int rank = 0;
    if ((int)threadIdx.x < count) {
      mine = list[threadIdx.x];
      for (int j = 0; j < count; ++j) rank += less(mine, list[j]);
    }
    __syncthreads();
    if ((int)threadIdx.x < count) list[rank] = mine;
    __syncthreads();
    return;
  }
  int size = 512;
  while (size < count) size <<= 1;
  for (int i = count + threadIdx.x; i < size; i += THREADS) list[i] = E{};
  __syncthreads();
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int x = threadIdx.x; x < size / 2; x += THREADS) {
        const int a = ((x & ~(j - 1)) << 1) | (x & (j - 1)), b = a | j;
        const E u = list[a], v = list[b];
        if (less(u, v) == ((a & k) == 0)) { list[a] = v; list[b] = u; }
      }
      __syncthreads();
    }
}

// (The unpacked values of one use are not kept for the next: they would take twice the registers.)
template <int N>
__device__ __forceinline__ void as_new(uint4 (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(w[i].x), "+r"(w[i].y), "+r"(w[i].z), "+r"(w[i].w));
}

// One chunk of one row, E elements a thread, kept as they came.
template <class T, int E>
__global__ void __launch_bounds__(kRowThreads, 4)
beam_rows_kernel(int paths, int vocab, int chunks, int rows, const T* logits, int64_t row_stride, const float* scores, const int32_t* done, ChunkHead* heads,
                 unsigned long long* lists, uint32_t* known) {
  constexpr int W = Vec<T>::kSize, VECS = E / W;
  __shared__ unsigned long long list[kRowList];
  __shared__ float sh_most[kRowThreads / 32], sh_low[kRowThreads / 32];
  __shared__ double sh_sum[kRowThreads / 32];
  __shared__ int sh_count, sh_n;
  __shared__ float sh_known;
  grid_wait();
  grid_release();
  // (all rows' first chunks before their second ones: those know of the first ones' N best)
  const int chunk = blockIdx.x / rows, row = blockIdx.x - chunk * rows;
  const float score = scores[row];
  const int gone = done ? done[row] : 0;
  const T* x0 = logits + (size_t)row * row_stride;
  // Which thread holds which token does not depend on where the row lies in memory: rows that are alike have sums that are alike to the last
  // bit, and ties between them stay ties.  A row that starts inside an aligned vector is read as pairs of aligned ones.
  const int skew = (int)((reinterpret_cast<uintptr_t>(x0) & 15) / sizeof(T));
  const int base = chunk * (kRowThreads * E);
  auto token_of_vec = [&](int v) { return base + (v * kRowThreads + (int)threadIdx.x) * W; };
  if (!(score > -INFINITY) || gone) return;                         // the merge does not ask
  uint4 raw[VECS];
#pragma unroll
  for (int v = 0; v < VECS; ++v) {
    const int t = token_of_vec(v);
    raw[v] = make_uint4(Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone);
    if (skew == 0) {
      if (t + W <= vocab) raw[v] = *reinterpret_cast<const uint4*>(x0 + t);
    } else if (t >= skew && t - skew + 2 * W <= vocab) {
      const uint4* a = reinterpret_cast<const uint4*>(x0 + t - skew);
      raw[v] = shifted(a[0], a[1], skew * (int)sizeof(T));
    }
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    const uint32_t k = known ? *(volatile uint32_t*)&known[row] : 0u;
    sh_count = 0;
    sh_known = k ? value_of((unsigned long long)k << 32) : -INFINITY;
  }
#pragma unroll
  for (int v = 0; v < VECS; ++v) {                                  // the row's ends
    const int t = token_of_vec(v);
    const bool whole = skew == 0 ? t + W <= vocab : t >= skew && t - skew + 2 * W <= vocab;
    if (!whole && t < vocab) {
      float x[W];
#pragma unroll
      for (int e = 0; e < W; ++e) x[e] = t + e < vocab ? Vec<T>::one(x0[t + e]) : -INFINITY;
      raw[v] = packed<T>(x);
    }
  }
  // groups of threads: the smallest power of two from N, 16 at least
  int groups = 16;
  while (groups < paths) groups <<= 1;
  const int lanes = kRowThreads / groups;                           // 16 .. 1
  float most, least;
  double total;
  for (int pass = 0;; ++pass) {
    most = -INFINITY;
#pragma unroll
    for (int v = 0; v < VECS; ++v) most = fmaxf(most, Vec<T>::most(raw[v]));
    float top = most;
    for (int o = lanes >> 1; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    float low = top;
    most = top;
    for (int o = 16; o >= lanes && o > 0; o >>= 1) {
      low = fminf(low, __shfl_xor_sync(~0u, low, o));
      most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    }
    if (lane == 0) { sh_most[warp] = most; sh_low[warp] = low; }
    __syncthreads();
    most = sh_most[0];
    least = sh_low[0];
#pragma unroll
    for (int w = 1; w < kRowThreads / 32; ++w) { most = fmaxf(most, sh_most[w]); least = fminf(least, sh_low[w]); }
    if (!(most > -INFINITY)) {                                      // no token in this chunk
      if (threadIdx.x == 0) { ChunkHead* h = heads + (size_t)row * chunks + chunk; h->sum = 0.0; h->best = 0; h->most = -INFINITY; }
      return;
    }
    least = fmaxf(least, sh_known);                                 // (one value for all threads)
    as_new(raw);
    Sum sum;
    const Pair minus = Pair::of(-most, -most);
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
      float x[W];
      Vec<T>::unpack(raw[v], x);
#pragma unroll
      for (int e = 0; e < W; e += 2) {
        float c, d;
        add(Pair::of(x[e], x[e + 1]), minus).split(&c, &d);
        sum.add(exp_neg(Pair::of(fmaxf(c, -200.f), fmaxf(d, -200.f))));       // (nothing is left of -200; nor of what is not a number)
      }
    }
    double s = sum.value();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    if (lane == 0) sh_sum[warp] = s;
    __syncthreads();
    total = 0.0;
#pragma unroll
    for (int w = 0; w < kRowThreads / 32; ++w) total += sh_sum[w];
    if (most < INFINITY || pass == 1) break;
    // infinities among the logits count as the largest number: once more
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
      float x[W];
      Vec<T>::unpack(raw[v], x);
#pragma unroll
      for (int e = 0; e < W; ++e) x[e] = cleaned<T>(x[e]);
      raw[v] = packed<T>(x);
    }
    __syncthreads();
  }
  // List what is no less than the bound (few vectors have any).
  auto each = [&](auto use) {
    as_new(raw);
#pragma unroll
    for (int v = 0; v < VECS; ++v)
      if (const float m = Vec<T>::most(raw[v]); m >= least && m > -INFINITY) {
        float x[W];
        Vec<T>::unpack(raw[v], x);
#pragma unroll
        for (int e = 0; e < W; ++e)
          if (x[e] >= least && x[e] > -INFINITY) use(key_of(x[e] + 0.f, token_of_vec(v) + e));               // -0 becomes +0
      }
  };
  each([&](unsigned long long k) {
    const int at = atomicAdd(&sh_count, 1);
    if (at < kRowList) list[at] = k;
  });
  __syncthreads();
  int count = sh_count;
  if (count > kRowList) {
    // Many that are alike, or groups without a candidate, which leave no bound (long runs that are masked): halve the range of keys until the count
    // fits.  Keys are all different, so some threshold has exactly N above it.
    unsigned long long lo = least > -INFINITY ? key_of(least + 0.f, base + kRowThreads * E - 1) : 1ull, hi = key_of(most + 0.f, base) + 1, bound = 0;
    for (int round = 0; round < 64 && (count > kRowList || count < paths); ++round) {      // (64 bits: it ends sooner)
      const unsigned long long mid = lo + (hi - lo) / 2;
      int c = 0;
      as_new(raw);
#pragma unroll
      for (int v = 0; v < VECS; ++v) {
        float x[W];
        Vec<T>::unpack(raw[v], x);
#pragma unroll
        for (int e = 0; e < W; ++e) c += x[e] > -INFINITY && key_of(x[e] + 0.f, token_of_vec(v) + e) >= mid;
      }
      if (threadIdx.x == 0) sh_n = 0;
      __syncthreads();
      c = __reduce_add_sync(~0u, c);
      if (lane == 0) atomicAdd(&sh_n, c);
      __syncthreads();
      count = sh_n;
      if (count > kRowList) lo = mid; else if (count < paths) hi = mid; else bound = mid;
      __syncthreads();
    }
    if (threadIdx.x == 0) sh_count = 0;
    __syncthreads();
    each([&](unsigned long long k) {
      if (k >= bound)
        if (const int at = atomicAdd(&sh_count, 1); at < kRowList) list[at] = k;
    });
    __syncthreads();
    count = min(sh_count, kRowList);
  }
  sort_down<kRowThreads>(list, count, [](unsigned long long a, unsigned long long b) { return a < b; });
  unsigned long long* out = lists + ((size_t)row * chunks + chunk) * paths;
  for (int i = threadIdx.x; i < paths; i += kRowThreads) out[i] = i < count ? list[i] : 0ull;
  if (threadIdx.x == 0) {
    ChunkHead* h = heads + (size_t)row * chunks + chunk;
    // (nothing listed: the best one is known by its value alone, which is what the merge's bound goes by)
    h->sum = total; h->best = count ? list[0] : key_of(most + 0.f, base + kRowThreads * E - 1); h->most = most;
    // N tokens of this row are no less than the last of N here: other chunks need list nothing below it
    if (known && count >= paths)
      if (const uint32_t k = (uint32_t)(list[paths - 1] >> 32); value_of((unsigned long long)k << 32) > sh_known) atomicMax(&known[row], k);
  }
}

// (Worth is compared first.  Where two are equal in 64 bits the lower path comes first, and in a path what its own order says: the larger logit,
// which only a sum that swallows the difference makes equal, then the lower token.)
struct Candidate {
  unsigned long long worth;              // order_of; 0 = none
  unsigned long long key;                // key_of; a path that is done: 0
  int32_t row, unused;
};
struct CandidateLess {
  __device__ __forceinline__ bool operator()(const Candidate& a, const Candidate& b) const {
    return a.worth < b.worth || (a.worth == b.worth && (a.row > b.row || (a.row == b.row && a.key < b.key)));
  }
};

__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(int paths, int chunks, const float* scores, const int32_t* done, int done_token,
                                                                   const ChunkHead* heads, const unsigned long long* lists, int32_t* token_out,
                                                                   int32_t* parent_out, float* score_out) {
  extern __shared__ __align__(16) unsigned char smem[];
  Candidate* list = reinterpret_cast<Candidate*>(smem);                              // [kList]
  double* lift = reinterpret_cast<double*>(list + kList);                            // [paths] s - lse
  unsigned long long* group = reinterpret_cast<unsigned long long*>(lift + paths);   // [paths]
  float* top = reinterpret_cast<float*>(group + paths);                              // [paths] largest logit
  int32_t* live = reinterpret_cast<int32_t*>(top + paths);                           // [paths] rows that offer their tokens
  int32_t* child = live + paths;                                                     // [paths] by rank: parent row
  int32_t* taken = child + paths;                                                    // [paths]
  int32_t* queue = taken + paths;                                                    // [paths * chunks]
  __shared__ int sh_live, sh_count, sh_queue, sh_end;
  const int g = blockIdx.x, p0 = g * paths, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) { sh_live = 0; sh_count = 0; sh_queue = 0; sh_end = kList; }
  for (int r = tid; r < paths; r += kMergeThreads) { group[r] = 0; taken[r] = 0; }
  grid_wait();
  grid_release();
  __syncthreads();
  for (int r = warp; r < paths; r += kMergeThreads / 32) {
    const ChunkHead* h = heads + (size_t)(p0 + r) * chunks;
    // (what a row without offers has for heads is old, and not used)
    const float score = scores[p0 + r];
    const int gone = done ? done[p0 + r] : 0;
    const float most_of_first = lane < chunks ? h[lane].most : -INFINITY;
    const double sum_of_first = lane < chunks ? h[lane].sum : 0.0;
    if (!(score > -INFINITY)) continue;
    if (gone) {
      if (lane == 0) {
        const int at = atomicAdd(&sh_count, 1);                     // (N of them at most, in front of all others)
        list[at].worth = order_of((double)score);
        list[at].key = 0;
        list[at].row = r;
      }
      continue;
    }
    float most = most_of_first;
    for (int c = lane + 32; c < chunks; c += 32) most = fmaxf(most, h[c].most);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    if (!(most > -INFINITY)) continue;                              // not one token
    double sum = most_of_first > -INFINITY ? sum_of_first * exp((double)most_of_first - (double)most) : 0.0;
    for (int c = lane + 32; c < chunks; c += 32)
      if (h[c].most > -INFINITY) sum += h[c].sum * exp((double)h[c].most - (double)most);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane == 0) {
      lift[r] = (double)score - log(sum);                           // worth of token v: lift + (x_v - most)
      top[r] = most;
      live[atomicAdd(&sh_live, 1)] = r;
    }
  }
  __syncthreads();
  const int done_count = sh_count, entries = sh_live * chunks;
  auto worth = [&](int r, unsigned long long key) { return order_of(lift[r] + ((double)value_of(key) - (double)top[r])); };
  // bound: as many groups as there are paths, over the chunks' best and the paths that are done
  auto best_of = [&](int i, int* r, int* c) -> unsigned long long {
    const int x = i / chunks;
    *r = live[x];
    *c = i - x * chunks;
    const unsigned long long key = heads[(size_t)(p0 + *r) * chunks + *c].best;
    return key ? worth(*r, key) : 0ull;
  };
  int r0 = 0, c0 = 0;
  const unsigned long long first = tid < entries ? best_of(tid, &r0, &c0) : 0ull;     // kept: mostly there is one a thread at most
  if (first) atomicMax(&group[tid % paths], first);
  for (int i = tid + kMergeThreads; i < entries; i += kMergeThreads) {
    int r, c;
    if (const unsigned long long w = best_of(i, &r, &c)) atomicMax(&group[i % paths], w);
  }
  for (int i = tid; i < done_count; i += kMergeThreads) atomicMax(&group[(entries + i) % paths], list[i].worth);
  __syncthreads();
  unsigned long long bound = ~0ull;
  for (int i = lane; i < paths; i += 32) bound = group[i] < bound ? group[i] : bound;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned long long other = __shfl_xor_sync(~0u, bound, o);
    bound = other < bound ? other : bound;
  }
  if (first && first >= bound) queue[atomicAdd(&sh_queue, 1)] = r0 << 16 | c0;
  for (int i = tid + kMergeThreads; i < entries; i += kMergeThreads) {
    int r, c;
    const unsigned long long w = best_of(i, &r, &c);
    if (w && w >= bound) queue[atomicAdd(&sh_queue, 1)] = r << 16 | c;
  }
  __syncthreads();
  const int queued = sh_queue;
  auto put = [&](int r, unsigned long long key, unsigned long long w) {
    const int at = atomicAdd(&sh_count, 1);
    list[at].worth = w; list[at].key = key; list[at].row = r;
  };
  if (done_count + queued * paths <= kList) {
    // all of the lists' elements fit: one a thread, all at once
    for (int i = tid; i < queued * paths; i += kMergeThreads) {
      const int l = i / paths, r = queue[l] >> 16, c = queue[l] & 0xffff;
      const unsigned long long key = lists[((size_t)(p0 + r) * chunks + c) * paths + i - l * paths];
      const unsigned long long w = key ? worth(r, key) : 0ull;
      if (key && w >= bound) put(r, key, w);
    }
    __syncthreads();
  } else {
    // A warp per list, 32 of its elements at a time while there is room; then only the N best so far matter, and every warp goes on where it was.  (Each
    // has room for its next 32 after that: N + 16 * 32 <= kList.  The count only goes up, so all that is in lies in front of
    // the first place that was given in vain.)
    static_assert(SDMS_MAX_BEAM_PATHS + kMergeThreads <= kList && kList - 32 >= SDMS_MAX_BEAM_PATHS, "every round gets on; a full list has N");
    int l = warp, i0 = 0;
    for (;;) {
      while (l < queued) {
        const int r = queue[l] >> 16, c = queue[l] & 0xffff;
        const unsigned long long key = i0 + lane < paths ? lists[((size_t)(p0 + r) * chunks + c) * paths + i0 + lane] : 0ull;
        const unsigned long long w = key ? worth(r, key) : 0ull;
        const bool good = key && w >= bound;
        const uint32_t all = __ballot_sync(~0u, good);
        const int n = __popc(all);
        int at = 0;
        if (lane == 0 && n > 0) at = atomicAdd(&sh_count, n);
        at = __shfl_sync(~0u, at, 0);
        if (n > 0 && at + n > kList) {
          if (lane == 0) atomicMin(&sh_end, at);
          break;
        }
        if (good) {
          Candidate* to = list + at + __popc(all & ((1u << lane) - 1));
          to->worth = w; to->key = key; to->row = r;
        }
        i0 += 32;
        if (n < 32 || i0 >= paths) { i0 = 0; l += kMergeThreads / 32; }       // (downwards sorted: nothing behind it either)
      }
      if (!__syncthreads_or(l < queued)) break;
      const int full = min(sh_count, sh_end);
      sort_down<kMergeThreads>(list, full, CandidateLess());
      bound = list[paths - 1].worth > bound ? list[paths - 1].worth : bound;
      if (tid == 0) { sh_count = paths; sh_end = kList; }
      __syncthreads();
    }
  }
  const int count = sh_count, found = min(count, paths);
  __syncthreads();
  // the N best in order
  int32_t* order = queue;
  if (count <= kRanked) {
    // ranks counted, a warp per candidate
    for (int i = warp; i < count; i += kMergeThreads / 32) {
      const Candidate mine = list[i];
      int n = 0;
      for (int j = lane; j < count; j += 32) {
        const unsigned long long w = list[j].worth;
        n += w > mine.worth || (w == mine.worth && CandidateLess()(mine, list[j]));
      }
      n = __reduce_add_sync(~0u, n);
      if (lane == 0 && n < paths) order[n] = i;
    }
  } else {
    sort_down<kMergeThreads>(list, count, CandidateLess());
    for (int i = tid; i < found; i += kMergeThreads) order[i] = i;
  }
  __syncthreads();
  auto write = [&](int at, int k) {
    const Candidate c = list[order[k]];
    token_out[p0 + at] = c.key == 0 ? done_token : token_of(c.key);
    parent_out[p0 + at] = p0 + c.row;
    score_out[p0 + at] = (float)worth_of(c.worth);
  };
  auto write_none = [&](int at) { token_out[p0 + at] = -1; parent_out[p0 + at] = p0 + at; score_out[p0 + at] = -INFINITY; };
  // Places: the best child of a path stays in it, the others take the free ones in order, the rest stays empty.  (Scores may be read and written in
  // one place: all of them have been read.)
  if (paths <= 32) {
    if (warp > 0) return;
    const int r = lane < found ? list[order[lane]].row : -1 - lane;        // a lane per rank
    const uint32_t alike = __match_any_sync(~0u, r);                // (by all lanes, whether they have a rank or not)
    const bool eldest = lane < found && __ffs(alike) - 1 == lane;
    const uint32_t full = __reduce_or_sync(~0u, eldest ? 1u << r : 0u), below = (1u << lane) - 1;
    const uint32_t rest = __ballot_sync(~0u, lane < found && !eldest);
    if (lane < paths && !(full >> lane & 1)) live[__popc(~full & below)] = lane;      // free places
    __syncwarp();
    if (lane < found) write(eldest ? r : live[__popc(rest & below)], lane);
    const int n = __popc(rest), empty = paths - __popc(full);
    if (n + lane < empty) write_none(live[n + lane]);
    return;
  }
  for (int k = tid; k < found; k += kMergeThreads) child[k] = list[order[k]].row;
  __syncthreads();
  int32_t* place = live;
  for (int k = tid; k < found; k += kMergeThreads) {
    bool eldest = true;
    for (int j = 0; j < k; ++j) eldest = eldest && child[j] != child[k];
    place[k] = eldest ? child[k] : -1;
    if (eldest) taken[child[k]] = 1;
  }
  if (tid == 0) sh_live = 0;
  __syncthreads();
  int32_t *free_places = reinterpret_cast<int32_t*>(group), *extra = free_places + paths;
  for (int k = tid; k < paths; k += kMergeThreads) {
    if (k < found && place[k] < 0) {                                // k as a rank: how many without a place lie in front of it
      int n = 0;
      for (int j = 0; j < k; ++j) n += place[j] < 0;
      extra[k] = n;
      atomicAdd(&sh_live, 1);
    }
    if (!taken[k]) {                                                // k as a place
      int n = 0;
      for (int j = 0; j < k; ++j) n += !taken[j];
      free_places[n] = k;
    }
  }
  __syncthreads();
  for (int k = tid; k < found; k += kMergeThreads) write(place[k] >= 0 ? place[k] : free_places[extra[k]], k);
  for (int k = found + tid; k < paths; k += kMergeThreads) write_none(free_places[sh_live + k - found]);
}

size_t merge_smem(int paths, int chunks) {
  return (size_t)kList * sizeof(Candidate) + (size_t)paths * 16 + (size_t)paths * 16 + (size_t)paths * chunks * 4;
}

template <class T>
cudaError_t launch_rows(int groups, int paths, int vocab, const void* logits, int64_t row_stride, const float* scores, const int32_t* done,
                        ChunkHead* heads, unsigned long long* lists, uint32_t* known, cudaStream_t stream) {
  const int rows = groups * paths, chunk = chunk_of(rows, vocab), chunks = chunks_of(rows, vocab);
  // What chunks know of one another, where there are at least four CTAs for every place on the GPU: one of a row begins when others have ended, mostly,
  // and clearing it (a launch more) costs little.  (Without and with: 2400 to 2600 CTAs alike; 64 x 16 rows of 32000, 4096 CTAs, 69.5 and 66.5 us; 4 x 64
  // of 151936, 4864, 222 and 159.)
  if ((long long)rows * chunks < kKnownFrom) known = nullptr;
  if (known)
    if (const cudaError_t e = cudaMemsetAsync(known, 0, (size_t)rows * 4, stream); e != cudaSuccess) return e;
  const auto kernel = chunk == 8192 ? beam_rows_kernel<T, 32> : chunk == 4096 ? beam_rows_kernel<T, 16> : beam_rows_kernel<T, 8>;
  return launch_overlapped(kernel, dim3((unsigned)(rows * chunks)), dim3(kRowThreads), 0, stream, paths, vocab, chunks, rows, static_cast<const T*>(logits),
                           row_stride, scores, done, heads, lists, known);
}

}  // namespace

size_t beam_select_bytes(int groups, int paths, int vocab) {
  const size_t rows = (size_t)groups * paths, entries = rows * chunks_of((int)rows, vocab);
  return align256(entries * sizeof(ChunkHead)) + align256(entries * paths * 8) + align256(rows * 4);
}

cudaError_t launch_beam_select(int groups, int paths, int vocab, const void* logits, int dtype, int64_t row_stride, const float* scores,
                               const int32_t* done, int32_t done_token, int32_t* token, int32_t* parent, float* score, void* workspace,
                               cudaStream_t stream) {
  const int rows = groups * paths, chunks = chunks_of(rows, vocab);
  ChunkHead* heads = static_cast<ChunkHead*>(workspace);
  unsigned long long* lists =
      reinterpret_cast<unsigned long long*>(static_cast<unsigned char*>(workspace) + align256((size_t)rows * chunks * sizeof(ChunkHead)));
  uint32_t* known = reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(lists) + align256((size_t)rows * chunks * paths * 8));
  cudaError_t e = dtype == SDMS_TYPE_FP32   ? launch_rows<float>(groups, paths, vocab, logits, row_stride, scores, done, heads, lists, known, stream)
                  : dtype == SDMS_TYPE_BF16 ? launch_rows<__nv_bfloat16>(groups, paths, vocab, logits, row_stride, scores, done, heads, lists, known, stream)
                                            : launch_rows<__half>(groups, paths, vocab, logits, row_stride, scores, done, heads, lists, known, stream);
  if (e != cudaSuccess) return e;
  const size_t smem = merge_smem(paths, chunks);
  static std::atomic<uint64_t> allowed{0};
  e = allow_shared(beam_merge_kernel, merge_smem(SDMS_MAX_BEAM_PATHS, SDMS_MAX_BEAM_VOCAB / 8192), &allowed);
  if (e != cudaSuccess) return e;
  return launch_overlapped(beam_merge_kernel, dim3((unsigned)groups), dim3(kMergeThreads), smem, stream, paths, chunks, scores, done, done_token, heads,
                           lists, token, parent, score);
}

}  // namespace sdms
