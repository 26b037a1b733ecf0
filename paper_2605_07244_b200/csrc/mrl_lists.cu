// Top tokens and learning from them: mrl_top_logprobs and mrl_distill_loss_fwd_bwd.
//
// Both read rows of logits against a running (m, s): m the largest of z c, c = log2(e) / T, and s = sum_v 2^(z_v c - m).  m starts at the
// lowest float, not at -inf, so that -inf - m stays -inf and a NaN always reaches the sum.  s = 0: nothing but -inf, or logits so low that z c
// leaves float32 (rows masked throughout with the type's lowest value): those are summed again against their largest logit itself.
#include <float.h>

#include <type_traits>

#include "mrl_common.cuh"

namespace {

using namespace mrl;

constexpr int kTopThreads = 256, kTopCtas = 5;          // threads, and CTAs an SM, of the top tokens
constexpr int kThreads = 512, kWarps = kThreads / 32;  // two CTAs an SM
constexpr int kTop = MRL_MAX_TOP;
constexpr int kMaxParts = 8;                            // CTAs that share a row

template <typename T>
__device__ __forceinline__ float load_f(const T* p);
template <>
__device__ __forceinline__ float load_f<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_f<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_f(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// 32 bytes of a row: eight floats, or sixteen bf16
constexpr int kVecBytes = 32;
template <typename T>
constexpr int kVecElems = kVecBytes / (int)sizeof(T);
struct Vec {
  uint32_t w[8];
};
__device__ __forceinline__ Vec load_vec(const void* p) {
  Vec v;
  asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]), "=r"(v.w[7])
               : "l"(p));
  return v;
}
template <typename T>
__device__ __forceinline__ Vec no_vec() {  // -inf throughout
  Vec v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v.w[j] = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
  return v;
}
template <typename T>
__device__ __forceinline__ float vec_max(const Vec& v) {  // passes over NaN
  if constexpr (sizeof(T) == 2) {
    uint32_t m = v.w[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.w[j]));
    return fmaxf(bf16lo_to_f32(m), bf16hi_to_f32(m));
  } else {
    float m = __uint_as_float(v.w[0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) m = fmaxf(m, __uint_as_float(v.w[j]));
    return m;
  }
}

// A CTA's part of a row: `head` elements up to the first address that is a multiple of 32 bytes, `vecs` vectors, `tail` elements.  So rows
// of any address and stride are read with the same wide loads.
template <typename T>
struct Part {
  const T* z;
  int first, n, head, vecs, tail;  // `first`: index in the row of the part's first element
  __device__ Part(const T* row, int V, int parts, int rank) {
    const int step = ((V + parts - 1) / parts + 15) & ~15;  // (V <= 2^31 - 1 where parts = 1: no addition passes it)
    first = parts == 1 ? 0 : min(V, rank * step);
    n = parts == 1 ? V : min(V - first, step);
    z = row + first;
    head = min(n, (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(z)) & (kVecBytes - 1)) / (int)sizeof(T));
    vecs = (n - head) / kVecElems<T>;
    tail = n - head - vecs * kVecElems<T>;
  }
  __device__ __forceinline__ const char* body() const { return reinterpret_cast<const char*>(z + head); }
};

// How many CTAs share a row: as many as there is room for on 148 SMs, with 16 KB of it at least.
int parts_of(long long N, long long row_bytes, int ctas_per_sm) {
  int parts = 1;
  while (parts < kMaxParts && N * parts * 2 <= ctas_per_sm * 148 && row_bytes / (parts * 2) >= 16 * 1024) parts *= 2;
  return parts;
}

template <typename... Params>
int launch_rows(void (*kernel)(Params...), long long N, int parts, int threads, size_t smem, bool behind, cudaStream_t st, const Params&... args) {
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)parts;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(N * parts));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = behind ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// `p` of this CTA's shared memory, in CTA `rank` of the cluster
template <typename U>
__device__ __forceinline__ U* in_cta(U* p, int rank) {
  U* q;
  asm("mapa.u64 %0, %1, %2;" : "=l"(q) : "l"(p), "r"(rank));
  return q;
}

struct Sums {
  float m, s, u;  // u = sum_v 2^(t_v) t_v, t_v = z_v c - m
};
__device__ __forceinline__ Sums sums_empty() { return Sums{-FLT_MAX, 0.f, 0.f}; }
// s and u over a higher maximum: u' = sum 2^(t + d) (t + d) with d = m - m'
__device__ __forceinline__ Sums sums_raise(Sums a, float m) {
  const float d = a.m - m, f = ex2_approx(d);                       // (NaN for two infinities)
  return Sums{m, a.s * f, fmaf(a.s, fmaxf(d, -1000.f), a.u) * f};  // 2^-1000 = 0, and no 0 * inf
}
__device__ __forceinline__ Sums sums_merge(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  a = sums_raise(a, m);
  b = sums_raise(b, m);
  return Sums{m, a.s + b.s, a.u + b.u};
}
// kGuard: right for z = -inf too, where 2^t t is 0
template <bool kEnt, bool kGuard>
__device__ __forceinline__ void sums_term(float z, float c, float m, float& s, float& u) {
  const float t = fmaf(z, c, -m), e = ex2_approx(t);
  s += e;
  if (kEnt) u = fmaf(e, kGuard ? fmaxf(t, -1000.f) : t, u);
}
// The sums of vectors in pairs: even and odd elements
struct Sums2 {
  f2 s, u;
};
// adds the elements of a vector, none of which is above m; c2 = (c, c), m2 = (-m, -m)
template <typename T, bool kEnt, bool kGuard>
__device__ __forceinline__ void sums_add(Sums2& a, const Vec& v, f2 c2, f2 m2) {
#pragma unroll
  for (int j = 0; j < 8; j += sizeof(T) == 2 ? 1 : 2) {
    const f2 z = sizeof(T) == 2 ? bf16x2_to_f2(v.w[j]) : make_f2(__uint_as_float(v.w[j]), __uint_as_float(v.w[(j + 1) & 7]));
    f2 t = fma_f2(z, c2, m2);
    float2 x = split_f2(t);
    const f2 e = make_f2(ex2_approx(x.x), ex2_approx(x.y));
    a.s = add_f2(a.s, e);
    if (kEnt && kGuard) t = make_f2(fmaxf(x.x, -1000.f), fmaxf(x.y, -1000.f));
    if (kEnt) a.u = fma_f2(e, t, a.u);
  }
}
__device__ __forceinline__ void sums_add(Sums& a, float z, float c) {
  const float m = fmaxf(a.m, z * c);
  if (m > a.m) a = sums_raise(a, m);
  sums_term<true, true>(z, c, a.m, a.s, a.u);
}
// Over the block, in a fixed order; every thread gets the result.  The maximum first, so that each thread rescales once.
template <int kT>
__device__ __forceinline__ Sums block_sums(Sums a, Sums* red) {
  constexpr int kWarps = kT / 32;
  float m = a.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) red[warp].m = m;
  __syncthreads();
  m = lane < kWarps ? red[lane].m : -FLT_MAX;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  a = sums_raise(a, m);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.u += __shfl_xor_sync(0xffffffffu, a.u, o);
  }
  if (lane == 0) red[warp].s = a.s, red[warp].u = a.u;
  __syncthreads();
  a.s = lane < kWarps ? red[lane].s : 0.f;
  a.u = lane < kWarps ? red[lane].u : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.u += __shfl_xor_sync(0xffffffffu, a.u, o);
  }
  return a;
}

// A row's sums against their offset x0 = m, in float64: x = z c, ln p = (x - x0) nat - ln s, nat = 1 / (c T).
struct Totals {
  double x0;
  float s, u;
};
// The sums of a row whose s above is 0, against its largest logit: 2^((z - zm) c).  `keep` says which elements count.  Called by the block;
// slow, and hardly ever needed.
template <typename T, int kT, typename Keep>
__device__ __noinline__ Totals low_sums(const T* z, int V, float c, Sums* red, Keep keep) {
  float zm = -FLT_MAX;
  for (int v = threadIdx.x; v < V; v += kT)
    if (keep(v)) zm = fmaxf(zm, load_f<T>(z + v));
  Sums a{zm, 0.f, 0.f};
  __syncthreads();
  zm = block_sums<kT>(a, red).m;
  a = Sums{0.f, 0.f, 0.f};
  for (int v = threadIdx.x; v < V; v += kT)
    if (keep(v)) sums_term<true, true>(load_f<T>(z + v) - zm, c, 0.f, a.s, a.u);
  __syncthreads();
  a = block_sums<kT>(a, red);
  return Totals{(double)zm * (double)c, a.s, a.u};
}

// Whole numbers in the order of floats; 0: NaN.  -0 and +0 are one value.
__device__ __forceinline__ uint32_t ordinal(float z) {
  if (z != z) return 0u;
  const uint32_t b = __float_as_uint(z + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordinal(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o); }

struct TopArgs {
  const void* logits;
  long long ld;
  int V;
  const int32_t* ids;
  const uint8_t* mask;
  float temperature, c;
  int top;
  float *logp, *lse, *entropy, *top_logp;
  int32_t *top_ids, *status;
};

// ------------------------------------------------------------------------------------------ top tokens
// A token's key: its logit's ordinal above its reversed index, so that larger keys come first in a list, and no two are alike.
typedef unsigned long long Key;
__device__ __forceinline__ Key key_of(float z, int index) { return ((Key)ordinal(z) << 32) | (uint32_t)(0x7fffffff - index); }

constexpr int kUnroll = 3;       // vectors of a thread and group
constexpr int kSecondFloor = 3;  // the group behind which the floor is set again
constexpr int kTopWarps = kTopThreads / 32;
constexpr int kNoted = 2048, kCap = 1024;  // vectors noted, and candidates, of a CTA
constexpr int kFew = 256;        // keys that are put in order by counting
struct TopShared {
  Key cand[kCap];                // candidates of this CTA
  Key list[kFew];                // what is left of them, or (CTA 0) of the pool
  Sums part[kMaxParts], red[kTopWarps];
  int vec[kNoted];               // vectors noted
  uint32_t hist[256], pick[4], pick2[2 * kTopWarps], n_vec, n_cand, n_list, n_pool;
};
// (CTA 0 of a row that several share) what is left of the candidates of all
constexpr int kPool = kMaxParts * kFew;

// The largest digit d (of 256) such that at least `want` counts lie at or above it; `want` becomes what is wanted of d itself.
__device__ __forceinline__ int pick_digit(TopShared& sh, uint32_t& want) {
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t above = 0;
    int d = 255;
    for (; d > 0 && above + sh.hist[d] < want; --d) above += sh.hist[d];
    sh.pick[0] = (uint32_t)d;
    sh.pick[1] = want - above;
  }
  __syncthreads();
  want = sh.pick[1];
  return (int)sh.pick[0];
}
__device__ __forceinline__ void count_digit(uint32_t* hist, bool on, uint32_t digit) {
  const unsigned who = __ballot_sync(0xffffffffu, on);
  if (who == 0) return;
  int same;
  const uint32_t d = __shfl_sync(0xffffffffu, digit, __ffs(who) - 1);
  same = __all_sync(0xffffffffu, !on || digit == d);  // (long runs of one value: one addition a warp)
  if (same) {
    if ((threadIdx.x & 31) == __ffs(who) - 1) atomicAdd(&hist[d], (uint32_t)__popc(who));
  } else if (on) {
    atomicAdd(&hist[digit], 1u);
  }
}

// Calls f(z, index in the part) for every element of a part, with all threads of a warp together; z is NaN where a thread has none.
template <typename T, typename F>
__device__ __forceinline__ void each_element(const Part<T>& part, F f) {
  const int tid = threadIdx.x;
  f(tid < part.head ? load_f<T>(part.z + tid) : NAN, tid);
  f(tid < part.tail ? load_f<T>(part.z + part.n - part.tail + tid) : NAN, part.n - part.tail + tid);
#pragma unroll 1
  for (int r = 0; r < part.vecs; r += kTopThreads) {
    const bool on = r + tid < part.vecs;
    const int at = part.head + (r + tid) * kVecElems<T>;
    const Vec v = on ? load_vec(part.z + at) : no_vec<T>();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (sizeof(T) == 2) {
        f(on ? bf16lo_to_f32(v.w[j]) : NAN, at + 2 * j);
        f(on ? bf16hi_to_f32(v.w[j]) : NAN, at + 2 * j + 1);
      } else {
        f(on ? __uint_as_float(v.w[j]) : NAN, at + j);
      }
    }
  }
}

// The `top` largest keys of a part by 256-way counting: a pass for each eight bits of the last one's value, then of its index up to which tokens of that
// value are listed, and one that collects.  For rows with more than kCap tokens that are not below the last floor: long runs of one value at the top.  Reads
// the row six (bf16) to eight times.
template <typename T>
__device__ void select_top(const Part<T> part, int top, TopShared& sh) {
  Key last = 0;
  uint32_t want = (uint32_t)top;
#pragma unroll 1
  for (int shift = 56; shift >= 0; shift -= 8) {
    if (sizeof(T) == 2 && (shift == 40 || shift == 32)) {  // a bf16's ordinal ends in sixteen zeros, or ones
      if (!(last >> 63)) last |= (Key)0xff << shift;
      continue;
    }
    for (int i = threadIdx.x; i < 256; i += kTopThreads) sh.hist[i] = 0;
    __syncthreads();
    each_element<T>(part, [&](float z, int i) {
      const Key key = key_of(z, part.first + i);
      count_digit(sh.hist, (key >> 32) != 0 && (shift == 56 || (key >> (shift + 8)) == (last >> (shift + 8))), (uint32_t)(key >> shift) & 255u);
    });
    last |= (Key)pick_digit(sh, want) << shift;
  }
  if (threadIdx.x == 0) sh.n_cand = 0;
  __syncthreads();
  each_element<T>(part, [&](float z, int i) {
    const Key key = key_of(z, part.first + i);
    if (key >= last) sh.cand[min(atomicAdd(&sh.n_cand, 1u), (uint32_t)(kCap - 1))] = key;
  });
  __syncthreads();
}

// Adds the first `want` tokens of -inf of a part to its candidates (all others are there).
template <typename T>
__device__ __noinline__ void add_masked(const Part<T> part, int want, TopShared& sh) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll 1
  for (int r = 0; r < part.n && want > 0; r += kTopThreads) {
    const int i = r + threadIdx.x;
    const bool masked = i < part.n && load_f<T>(part.z + i) == -INFINITY;
    const unsigned who = __ballot_sync(0xffffffffu, masked);
    if (lane == 0) sh.hist[warp] = (uint32_t)__popc(who);
    __syncthreads();
    int before = __popc(who & ((1u << lane) - 1)), all = 0;
    for (int w = 0; w < kTopWarps; ++w) {
      before += w < warp ? (int)sh.hist[w] : 0;
      all += (int)sh.hist[w];
    }
    if (masked && before < want) sh.cand[atomicAdd(&sh.n_cand, 1u)] = key_of(-INFINITY, part.first + i);
    want -= all;
    __syncthreads();
  }
}

// Copies the keys that can be among the `top` largest of `from` to `to` (of CTA `rank`, behind what its counter says is there): at most kFew,
// and all of the `top` largest among them.  Bits are settled from above until few enough are left.
template <int kMost>
__device__ __noinline__ void keep_largest(const Key* from, int n, int top, Key* to, uint32_t* n_to) {
  constexpr int kEach = kMost / kTopThreads;
  Key mine[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) mine[i] = i * kTopThreads + threadIdx.x < n ? from[i * kTopThreads + threadIdx.x] : 0;
  Key least = 1;
  if (n > kFew) {
    least = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const Key next = least | ((Key)1 << bit);
      int total = __syncthreads_count(mine[0] >= next);
      if (n > kTopThreads) {
#pragma unroll
        for (int i = 1; i < kEach; ++i) total += __syncthreads_count(mine[i] >= next);
      }
      if (total >= top) least = next;
      if (total >= top && total <= kFew) break;
    }
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (mine[i] >= least) to[atomicAdd(n_to, 1u)] = mine[i];
}

constexpr uint32_t kLowest = 0x00800000u;  // the ordinal above that of -inf
// An ordinal, kLowest at least, that `want` threads at least do not fall below with theirs, and `more` + 2 others if that can be.  Bits are settled from above, from
// the first that the threads differ in.
template <typename T>
__device__ __forceinline__ uint32_t kth_ordinal(uint32_t mine, int want, int more, uint32_t* red) {
  uint32_t high = __reduce_max_sync(0xffffffffu, mine), low = __reduce_min_sync(0xffffffffu, mine);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) red[warp] = high, red[kTopWarps + warp] = low;
  __syncthreads();
  high = __reduce_max_sync(0xffffffffu, red[lane % kTopWarps]);
  low = __reduce_min_sync(0xffffffffu, red[kTopWarps + lane % kTopWarps]);
  if (high == low) {
    __syncthreads();  // (`red` may be used again)
    return max(low, kLowest);
  }
  const int first = 31 - __clz(high ^ low);
  uint32_t found = high & ~(first == 31 ? ~0u : (2u << first) - 1);
  for (int bit = first; bit >= (sizeof(T) == 2 ? 16 : 0); --bit) {
    const uint32_t next = found | (1u << bit);
    const int n = __syncthreads_count(mine >= next);
    if (n >= want) found = next;
    if (n >= want && n <= want + more + 2) break;
  }
  return max(found, kLowest);
}
// bits 0 .. 7 to the even places
__device__ __forceinline__ uint32_t spread_bits(uint32_t b) {
  b = (b | b << 4) & 0x0f0fu;
  b = (b | b << 2) & 0x3333u;
  return (b | b << 1) & 0x5555u;
}
// The least T whose ordinal is not below `o`.  (A bf16 has the ordinal of the float it is: sixteen zeros below, or ones if negative.)
template <typename T>
__device__ __forceinline__ float floor_of(uint32_t o) {
  const float z = from_ordinal(o);
  return sizeof(T) == 2 ? __uint_as_float(__float_as_uint(z) & 0xffff0000u) : z;
}
// Bit e: element e of the vector is not below `floor`, a T
template <typename T>
__device__ __forceinline__ uint32_t not_below(const Vec& v, float floor) {
  uint32_t bits = 0;
  if constexpr (sizeof(T) == 2) {
    const uint32_t f = __float_as_uint(floor) >> 16 | (__float_as_uint(floor) & 0xffff0000u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t m;
      asm("set.ge.u32.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(v.w[j]), "r"(f));
      bits |= m & (0x10001u << j);
    }
    bits = spread_bits(bits & 0xffu) | spread_bits(bits >> 16) << 1;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) bits |= __uint_as_float(v.w[j]) >= floor ? 1u << j : 0u;
  }
  return bits;
}

template <typename T, bool kEnt>
__global__ void __launch_bounds__(kTopThreads, kTopCtas) top_kernel(const TopArgs p) {
  __shared__ TopShared sh;
  const int tid = threadIdx.x;
  int parts, rank;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const long long row = blockIdx.x / (unsigned)parts;
  const T* zrow = static_cast<const T*>(p.logits) + row * p.ld;
  const int id = p.ids != nullptr ? p.ids[row] : 0;
  const bool on = p.mask == nullptr || p.mask[row] != 0, good = id >= 0 && id < p.V;
  if (!on || !good) {  // (all CTAs of the row)
    if (rank != 0) return;
    if (tid == 0) {
      if (on && p.status != nullptr) atomicOr(p.status, MRL_DEV_BAD_TOKEN_ID);
      if (p.logp != nullptr) p.logp[row] = 0.f;
      if (p.lse != nullptr) p.lse[row] = 0.f;
      if (kEnt) p.entropy[row] = 0.f;
    }
    if (tid < p.top) {
      p.top_ids[row * p.top + tid] = -1;
      p.top_logp[row * p.top + tid] = 0.f;
    }
    return;
  }
  if (tid == 0) sh.n_vec = sh.n_cand = sh.n_list = sh.n_pool = 0;
  __syncthreads();
  extern __shared__ Key pool[];  // [kPool] where parts > 1
  if (parts > 1) cluster_arrive();  // "my counters are set"
  const Part<T> part(zrow, p.V, parts, rank);
  const char* body = part.body() + (size_t)tid * kVecBytes;
  const float z_head = tid < part.head ? load_f<T>(part.z + tid) : -INFINITY;
  const float z_tail = tid < part.tail ? load_f<T>(part.z + part.n - part.tail + tid) : -INFINITY;
  Sums a = sums_empty();
  if (tid < part.head) sums_add(a, z_head, p.c);
  if (tid < part.tail) sums_add(a, z_tail, p.c);
  // Vectors that can hold a listed token are noted, by their place: those with an element that is not below a floor, which the first group sets
  // so that `top` threads at least have an element there, each at least one.  The largest element of each thread sets the last floor behind the last
  // group in the same way, a tight one, and what is not below it is read again from the vectors noted.
  float best = z_head, floor = floor_of<T>(kLowest);
  const int groups = max(1, (part.vecs + kTopThreads * kUnroll - 1) / (kTopThreads * kUnroll));
#pragma unroll 1
  for (int g = 0; g < groups; ++g) {
    const int v0 = g * kTopThreads * kUnroll + tid;
    Vec v[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) v[i] = v0 + i * kTopThreads < part.vecs ? load_vec(body + (size_t)(v0 - tid + i * kTopThreads) * kVecBytes) : no_vec<T>();
    float high[kUnroll], most = best;
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      high[i] = vec_max<T>(v[i]);
      most = fmaxf(most, high[i]);
    }
    best = most;
    const float m = fmaxf(a.m, most * p.c);
    if (m > a.m) a = sums_raise(a, m);
    const f2 c2 = make_f2(p.c, p.c), m2 = make_f2(-a.m, -a.m);
    Sums2 more{0, 0};
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (v0 + i * kTopThreads < part.vecs) sums_add<T, kEnt, false>(more, v[i], c2, m2);
    float2 s = split_f2(more.s), u = split_f2(more.u);
    if (kEnt && !(u.x + u.y == u.x + u.y)) {  // 0 * inf: masked logits among them (or NaN, which it stays)
      more = Sums2{0, 0};
#pragma unroll
      for (int i = 0; i < kUnroll; ++i) sums_add<T, kEnt, true>(more, v[i], c2, m2);
      u = split_f2(more.u);
    }
    a.s += s.x + s.y;
    a.u += u.x + u.y;
    if (p.top == 0) continue;
    if (g == 0 || (g == kSecondFloor && g + 1 < groups)) floor = floor_of<T>(kth_ordinal<T>(ordinal(best), p.top, p.top / 4, sh.pick2));
#pragma unroll
    for (int i = 0; i < kUnroll; ++i)
      if (high[i] >= floor) {
        const uint32_t at = atomicAdd(&sh.n_vec, 1u);
        if (at < kNoted) sh.vec[at] = v0 + i * kTopThreads;
      }
  }
  int n = 0;
  if (p.top > 0) {
    best = fmaxf(best, z_tail);
    floor = floor_of<T>(kth_ordinal<T>(ordinal(best), p.top, p.top / 4, sh.pick2));  // (barriers: the vectors are noted)
    auto push = [&](float z, int index) {
      if (z >= floor) {
        const uint32_t at = atomicAdd(&sh.n_cand, 1u);
        if (at < kCap) sh.cand[at] = key_of(z, part.first + index);
      }
    };
    if (tid < part.head) push(z_head, tid);
    if (tid < part.tail) push(z_tail, part.n - part.tail + tid);
    // (too many noted -- a row that rises: all vectors, once more)
    const bool all = sh.n_vec > kNoted;
    const int noted = all ? part.vecs : (int)sh.n_vec;
    for (int k = tid; k < noted; k += kTopThreads) {
      const int at = all ? k : sh.vec[k];
      const Vec v = load_vec(part.body() + (size_t)at * kVecBytes);
      uint32_t bits = not_below<T>(v, floor);
#pragma unroll 1
      for (; bits != 0; bits &= bits - 1) {
        const int index = part.head + at * kVecElems<T> + __ffs(bits) - 1;
        push(load_f<T>(part.z + index), index);
      }
    }
  }
  a = block_sums<kTopThreads>(a, sh.red);  // (a barrier: the candidates are there)
  if (p.top > 0) {
    const int found = (int)sh.n_cand;
    if (found > kCap) select_top<T>(part, p.top, sh);
    if (found < min(p.top, part.n)) {
      __syncthreads();  // (all have read the number)
      add_masked<T>(part, p.top - found, sh);
    }
    n = (int)sh.n_cand;
  }
  if (parts > 1) {
    cluster_wait();
    if (tid == 0) *in_cta(&sh.part[rank], 0) = a;
    if (n > 0) keep_largest<kCap>(sh.cand, n, p.top, in_cta(pool, 0), in_cta(&sh.n_pool, 0));
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
    a = sh.part[0];
    for (int k = 1; k < parts; ++k) a = sums_merge(a, sh.part[k]);
    n = (int)sh.n_pool;
    if (n > 0) keep_largest<kPool>(pool, n, p.top, sh.list, &sh.n_list);
  } else if (n > 0) {
    keep_largest<kCap>(sh.cand, n, p.top, sh.list, &sh.n_list);
  }
  __syncthreads();
  n = (int)sh.n_list;
  const Key* keys = sh.list;
  Totals t{(double)a.m, a.s, a.u};
  if (t.s == 0.f) t = low_sums<T, kTopThreads>(zrow, p.V, p.c, sh.red, [](int) { return true; });
  const double nat = 1.0 / ((double)p.c * (double)p.temperature), ln_s = t.s == 0.f ? NAN : log((double)t.s);
  auto ln_p = [&](float z) { return (float)(((double)z * (double)p.c - t.x0) * nat - ln_s); };
  if (tid == 0) {
    if (p.lse != nullptr) p.lse[row] = (float)(t.x0 * nat + ln_s);
    if (p.logp != nullptr) p.logp[row] = ln_p(load_f<T>(zrow + id));
    if (kEnt) p.entropy[row] = (float)(ln_s - (double)t.u / (double)t.s * nat);
  }
  // in order: a key's place is the number of larger ones, counted by four threads a key
  for (int k0 = 0; k0 < n; k0 += kTopThreads / 4) {
    const int k = k0 + (tid >> 2);
    const Key key = k < n ? keys[k] : 0;
    int at = 0;
#pragma unroll 4
    for (int j = tid & 3; j < n; j += 4) at += keys[j] > key;
    at += __shfl_xor_sync(0xffffffffu, at, 1);
    at += __shfl_xor_sync(0xffffffffu, at, 2);
    if (k < n && at < p.top && (tid & 3) == 0) {
      p.top_ids[row * p.top + at] = 0x7fffffff - (int32_t)(uint32_t)key;
      p.top_logp[row * p.top + at] = ln_p(from_ordinal((uint32_t)(key >> 32)));
    }
  }
  for (int k = n + tid; k < p.top; k += kTopThreads) {
    p.top_ids[row * p.top + k] = -1;
    p.top_logp[row * p.top + k] = -INFINITY;
  }
}

// ------------------------------------------------------------------------------------------ distillation
constexpr int kRowOff = 0, kRowValid = 1, kRowRefused = 2;
constexpr int kListThreads = 1024, kListRows = 64;  // rows of a CTA of the list check

struct DistillArgs {
  const void* logits;
  void* dlogits;
  long long ld, ld_out, N;
  int V, top;
  const int32_t* top_ids;
  const float* top_logp;
  const uint8_t* mask;
  const float* weight;
  mrl_distill_params dp;
  float c;
  float *row_kl, *loss;
  long long* stats;
  int32_t* status;
  uint8_t* rowstat;     // [N] kRow*
  int2* counts;         // [n_counts] valid and refused rows
  int n_counts;         // of `counts` as the row kernel reads them: sums of up to 32 CTAs of the check each
  double* term;         // [N] weight_t KL_t
  int bit_words, park_slots;  // shared memory of the row kernel
};

// A warp per row: is its list one to learn from?  The entries stay in registers, four a lane; a token twice shows when every entry
// is compared with those of the other places, carried round the warp.
__global__ void __launch_bounds__(kListThreads) list_check_kernel(const DistillArgs p) {
  __shared__ int2 part[kListThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  let_next_start();
  int2 n{0, 0};
  for (int r = warp; r < kListRows; r += kListThreads / 32) {
    const long long row = (long long)blockIdx.x * kListRows + r;
    if (row >= p.N) break;
    if (p.mask != nullptr && p.mask[row] == 0) {
      if (lane == 0) p.rowstat[row] = kRowOff;
      continue;
    }
    int id[kTop / 32];
    int bad = 0;
    bool any = false;
#pragma unroll
    for (int q = 0; q < kTop / 32; ++q) {
      const int k = q * 32 + lane;
      id[q] = k < p.top ? p.top_ids[row * p.top + k] : -1;
      const float l = k < p.top && id[q] >= 0 ? p.top_logp[row * p.top + k] : -INFINITY;
      if (!(l < INFINITY)) bad |= MRL_DEV_BAD_LIST;  // (NaN too)
      if (l == -INFINITY) id[q] = -1;
      if (id[q] >= p.V) bad |= MRL_DEV_BAD_TOKEN_ID;
      any |= id[q] >= 0;
    }
    const int used = (p.top + 31) / 32;
#pragma unroll 1
    for (int o = 0; o < 32; ++o) {
#pragma unroll
      for (int q = 0; q < kTop / 32; ++q) {
        if (q >= used) break;
        const int other = __shfl_sync(0xffffffffu, id[q], (lane + o) & 31);
#pragma unroll
        for (int j = 0; j < kTop / 32; ++j)
          if (other >= 0 && other == id[j] && !(o == 0 && j == q)) bad |= MRL_DEV_BAD_LIST;
      }
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
    any = __any_sync(0xffffffffu, any);
    const int stat = bad != 0 ? kRowRefused : any ? kRowValid : kRowOff;
    n.x += stat == kRowValid;
    n.y += stat == kRowRefused;
    if (lane == 0) {
      p.rowstat[row] = (uint8_t)stat;
      if (bad != 0 && p.status != nullptr) atomicOr(p.status, bad);
    }
  }
  if (lane == 0) part[warp] = n;
  __syncthreads();
  if (warp == 0) {
    n = part[lane];
    n.x = __reduce_add_sync(0xffffffffu, n.x);
    n.y = __reduce_add_sync(0xffffffffu, n.y);
    if (lane == 0) p.counts[blockIdx.x] = n;
  }
}

// Valid and refused rows of the call
__device__ __forceinline__ int2 sum_counts(const int2* counts, int n, int2* red) {
  int2 a{0, 0};
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    a.x += counts[i].x;
    a.y += counts[i].y;
  }
  a.x = __reduce_add_sync(0xffffffffu, a.x);
  a.y = __reduce_add_sync(0xffffffffu, a.y);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = a;
  __syncthreads();
  a = red[0];
  for (int k = 1; k < (int)(blockDim.x >> 5); ++k) {
    a.x += red[k].x;
    a.y += red[k].y;
  }
  return a;
}

// The counts of kListRows rows each added up to kCounts at most, so that the CTAs of the rows have few to read
constexpr int kCounts = 32;
__global__ void __launch_bounds__(1024) counts_kernel(const int2* __restrict__ from, int n, int each, int2* __restrict__ to) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  let_next_start();
  wait_for_previous();
  int2 a{0, 0};
  for (int i = warp * each + lane; i < min(n, (warp + 1) * each); i += 32) {
    a.x += from[i].x;
    a.y += from[i].y;
  }
  a.x = __reduce_add_sync(0xffffffffu, a.x);
  a.y = __reduce_add_sync(0xffffffffu, a.y);
  if (lane == 0) to[warp] = a;
}

// Sum over the block in a fixed order.
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
  for (int k = 1; k < (int)(blockDim.x >> 5); ++k) v += red[k];
  return v;
}

// Listed tokens and rest of a row are told apart by a bit for each element in shared memory: a vector's bits are one word, hardly ever other than 0.  Pass 1
// sums the rest (the listed tokens' logits are at hand from the start), thread k < 128 then works on place k of the list in float64, and pass 2 writes
// of_rest * 2^(z c - m) everywhere but at the listed tokens, which come last.  As in the policy loss's kernel the row is read from HBM once: pass 1 walks it from
// its end, the group read last stays in registers, the first ones are parked in shared memory, the rest comes from L2.
constexpr int kDistillUnroll = 4;
// Shared memory of a CTA: bits, parked vectors, staging of outputs that start off 16 bytes from their inputs.  What it leaves is L1, which holds the
// loads in flight.
constexpr size_t kDistillSmem = 68 * 1024;
constexpr uint32_t kStageRow = kVecBytes * 32, kStageBytes = kWarps * kStageRow;
constexpr double kNoRest = -700.0;  // ln p_r below which the learner gives the rest nothing: masks, of -inf or of the type's lowest value

struct DistillShared {
  Sums part[kMaxParts], red[kWarps];
  double sum[3][2][kTop / 32];
  float high[2][kTop / 32];
  float of_rest, m;
  int low;
  uint32_t head_bits, tail_bits;
  int ids[kTop];
};

// Two sums over the 128 threads of a list, in a fixed order
__device__ __forceinline__ void list_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ void list_sums(double& a, double& b, double (*red)[kTop / 32]) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b += __shfl_xor_sync(0xffffffffu, b, o);
  }
  if ((threadIdx.x & 31) == 0) red[0][threadIdx.x >> 5] = a, red[1][threadIdx.x >> 5] = b;
  list_barrier();
  a = (red[0][0] + red[0][1]) + (red[0][2] + red[0][3]);
  b = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
}

struct RowResult {
  double kl, at;    // KL_t; T dKL/dz of this thread's listed token
  double of_rest;   // T dKL/dz_v = of_rest * softmax over the rest (v)
};

// A row's KL and gradient factors from its list (thread k < 128 holds place k) and the sums over the rest, in float64
__device__ RowResult distill_row(bool used, float z, float l, Totals rest, float c, const mrl_distill_params& dp, DistillShared& sh) {
  const double nat = 1.0 / ((double)c * (double)dp.temperature);
  float zs = used ? fmaxf(z, -FLT_MAX) : -FLT_MAX, ls = used ? l : -FLT_MAX;
  if (used && z != z) zs = INFINITY;  // (NaN: inf - inf below)
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    zs = fmaxf(zs, __shfl_xor_sync(0xffffffffu, zs, o));
    ls = fmaxf(ls, __shfl_xor_sync(0xffffffffu, ls, o));
  }
  if ((threadIdx.x & 31) == 0) sh.high[0][threadIdx.x >> 5] = zs, sh.high[1][threadIdx.x >> 5] = ls;
  list_barrier();
#pragma unroll
  for (int k = 0; k < kTop / 32; ++k) {
    zs = fmaxf(zs, sh.high[0][k]);
    ls = fmaxf(ls, sh.high[1][k]);
  }
  const bool event = dp.rest == MRL_REST_EVENT, any_rest = rest.s != 0.f;
  double m = (double)zs * (double)c;  // (+inf stays what it is)
  if (any_rest) m = fmax(m, rest.x0);
  const double x = used ? ((double)z * (double)c - m) * nat : 0.0;
  const double in_rest = any_rest ? (double)rest.s * exp((rest.x0 - m) * nat) : 0.0;
  const double d = event ? (double)l : (double)l - (double)ls;  // (without a rest any logits will do: from the largest)
  double q = used ? exp(d) : 0.0, total = used ? exp(x) : 0.0, mass = q;
  list_sums(total, mass, sh.sum[0]);
  total += in_rest;
  const double ln_total = total > 0.0 ? log(total) : NAN;
  const double ln_p = x - ln_total, p = used ? exp(ln_p) : 0.0;
  const double ln_p_rest = any_rest ? log((double)rest.s) + (rest.x0 - m) * nat - ln_total : -INFINITY;
  const bool has_rest = !(ln_p_rest < kNoRest);
  const double p_rest = has_rest ? exp(ln_p_rest) : 0.0;
  double term = 0.0, none = 0.0, q_rest = 0.0, ratio = 0.0;
  if (!event) {
    const double ln_q = d - log(mass);
    q = used ? exp(ln_q) : 0.0;
    term = q > 0.0 ? q * (ln_q - ln_p) : 0.0;
  } else {
    q_rest = has_rest ? fmax(1.0 - mass, (double)dp.rest_floor) : 0.0;
    ratio = ln_p - (double)l;
    if (dp.direction == MRL_DISTILL_FORWARD) term = q > 0.0 ? -q * ratio : 0.0;
    else term = used && p != 0.0 ? p * ratio : 0.0;
  }
  list_sums(term, none, sh.sum[1]);
  RowResult r;
  r.kl = term;
  if (!event) {
    r.at = p - q;
    r.of_rest = p_rest;
  } else if (dp.direction == MRL_DISTILL_FORWARD) {
    r.kl += q_rest > 0.0 ? q_rest * (log(q_rest) - ln_p_rest) : 0.0;
    r.at = (mass + q_rest) * p - q;
    r.of_rest = has_rest ? (mass + q_rest) * p_rest - q_rest : 0.0;
  } else {
    const double ratio_rest = has_rest ? ln_p_rest - log(q_rest) : 0.0;
    r.kl += p_rest != 0.0 ? p_rest * ratio_rest : 0.0;
    r.at = p != 0.0 ? p * (ratio - r.kl) : 0.0;
    r.of_rest = p_rest != 0.0 ? p_rest * (ratio_rest - r.kl) : 0.0;
  }
  return r;
}

// a vector that pass 2 wants again, if L2 can keep it
__device__ __forceinline__ Vec load_vec_keep(const void* p) {
  Vec v;
  asm volatile("ld.global.L1::no_allocate.L2::evict_last.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]), "=r"(v.w[7])
               : "l"(p));
  return v;
}
__device__ __forceinline__ void store_vec(void* p, const Vec& v) {  // 32 bytes on 32
  asm volatile("st.global.L2::evict_first.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v.w[0]), "r"(v.w[1]), "r"(v.w[2]),
               "r"(v.w[3]), "r"(v.w[4]), "r"(v.w[5]), "r"(v.w[6]), "r"(v.w[7])
               : "memory");
}
// A thread's own vectors in shared memory, as two planes of 16-byte halves
__device__ __forceinline__ void park(uint4* planes, int slots, int slot, const Vec& v) {
  planes[slot] = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
  planes[slots + slot] = make_uint4(v.w[4], v.w[5], v.w[6], v.w[7]);
}
__device__ __forceinline__ Vec parked(const uint4* planes, int slots, int slot) {
  const uint4 a = planes[slot], b = planes[slots + slot];
  return Vec{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
// -inf in place of the elements whose bits are set
template <typename T>
__device__ __forceinline__ void strike_out(Vec& v, uint32_t bits) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (sizeof(T) == 2) {
      if (bits & (1u << (2 * j))) v.w[j] = (v.w[j] & 0xffff0000u) | 0xff80u;
      if (bits & (2u << (2 * j))) v.w[j] = (v.w[j] & 0xffffu) | 0xff800000u;
    } else {
      if (bits & (1u << j)) v.w[j] = 0xff800000u;
    }
  }
}

// The 32 vectors of a warp -- `count` of them -- to an address that is a multiple of the element only: through shared memory, in words as they lie in the output
template <typename T>
__device__ __forceinline__ void store_shifted(char* out, const Vec& v, int count, uint32_t* stage) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  uint4* mine = reinterpret_cast<uint4*>(stage) + 2 * lane;
  mine[0] = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
  mine[1] = make_uint4(v.w[4], v.w[5], v.w[6], v.w[7]);
  __syncwarp();
  const int words = count * 8;
  if (sizeof(T) == 4 || (reinterpret_cast<uintptr_t>(out) & 3) == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i * 32 + lane < words) __stcs(reinterpret_cast<uint32_t*>(out) + i * 32 + lane, stage[i * 32 + lane]);
  } else {  // odd elements of bf16: word i of the output is the upper half of word i and the lower one of word i + 1
    uint32_t* odd = reinterpret_cast<uint32_t*>(out + 2);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = i * 32 + lane;
      if (at + 1 < words) __stcs(odd + at, __funnelshift_r(stage[at], stage[at + 1], 16));
    }
    if (lane == 0 && words > 0) {
      reinterpret_cast<uint16_t*>(out)[0] = (uint16_t)stage[0];
      reinterpret_cast<uint16_t*>(out)[2 * words - 1] = (uint16_t)(stage[words - 1] >> 16);
    }
  }
}

template <typename T>
__device__ void zero_part(T* out, int n) {
  const int head = min(n, (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(out)) & 15) / (int)sizeof(T));
  const int pieces = (n - head) / (16 / (int)sizeof(T)), tail0 = head + pieces * (16 / (int)sizeof(T));
  for (int i = threadIdx.x; i < pieces; i += kThreads) __stcs(reinterpret_cast<uint4*>(out + head) + i, make_uint4(0, 0, 0, 0));
  if ((int)threadIdx.x < head) store_f(out + threadIdx.x, 0.f);
  if (tail0 + (int)threadIdx.x < n) store_f(out + tail0 + threadIdx.x, 0.f);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) distill_kernel(const DistillArgs p) {
  extern __shared__ uint4 dyn[];
  __shared__ DistillShared sh;
  const int tid = threadIdx.x;
  int parts, rank;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const long long row = blockIdx.x / (unsigned)parts;
  const T* zrow = static_cast<const T*>(p.logits) + row * p.ld;
  const Part<T> part(zrow, p.V, parts, rank);
  T* out = p.dlogits != nullptr ? static_cast<T*>(p.dlogits) + row * p.ld_out + part.first : nullptr;
  let_next_start();
  wait_for_previous();
  if (p.rowstat[row] != kRowValid) {  // (all CTAs of the row)
    if (out != nullptr) zero_part(out, part.n);
    if (tid == 0 && rank == 0) {
      p.term[row] = 0.0;
      if (p.row_kl != nullptr) p.row_kl[row] = 0.f;
    }
    return;
  }
  // shared memory: bits of the body's vectors | parked vectors | staging
  using Bits = typename std::conditional<sizeof(T) == 2, uint16_t, uint8_t>::type;
  Bits* bits = reinterpret_cast<Bits*>(dyn);
  uint4* planes = dyn + p.bit_words / 4;
  uint32_t* stage = reinterpret_cast<uint32_t*>(planes + 2 * p.park_slots) + (tid >> 5) * (kStageRow / 4);
  for (int i = tid; i < p.bit_words / 4; i += kThreads) dyn[i] = make_uint4(0, 0, 0, 0);
  if (tid == 0) sh.head_bits = sh.tail_bits = 0;
  int id = tid < p.top ? p.top_ids[row * p.top + tid] : -1;
  const float l = id >= 0 ? p.top_logp[row * p.top + tid] : -INFINITY;
  if (l == -INFINITY) id = -1;
  const float mine = id >= 0 ? load_f<T>(zrow + id) : 0.f;
  const float z_head = tid < part.head ? load_f<T>(part.z + tid) : -INFINITY;
  const float z_tail = tid < part.tail ? load_f<T>(part.z + part.n - part.tail + tid) : -INFINITY;
  if (tid < kTop) sh.ids[tid] = id;
  __syncthreads();
  if (parts > 1) cluster_arrive();  // "here": its shared memory may be written to
  const int rel = id - part.first;  // the listed token in this part
  const bool owner = id >= 0 && rel >= 0 && rel < part.n;
  if (owner) {
    const int at = rel - part.head;
    if (at < 0) atomicOr(&sh.head_bits, 1u << rel);
    else if (at >= part.vecs * kVecElems<T>) atomicOr(&sh.tail_bits, 1u << (at - part.vecs * kVecElems<T>));
    else atomicOr(reinterpret_cast<uint32_t*>(dyn) + (at >> 5), 1u << (at & 31));
  }
  __syncthreads();
  const bool head_on = tid < part.head && !((sh.head_bits >> tid) & 1u), tail_on = tid < part.tail && !((sh.tail_bits >> tid) & 1u);
  Sums a = sums_empty();
  if (head_on) sums_add(a, z_head, p.c);
  if (tail_on) sums_add(a, z_tail, p.c);

  // ---- pass 1, from the last group (the ragged one) to the first, which is a full one wherever there are two
  constexpr int kGroup = kThreads * kDistillUnroll;
  const char* in = part.body() + (size_t)tid * kVecBytes;
  const int last = part.vecs > 0 ? (part.vecs - 1) / kGroup * kGroup : -kGroup;
  Vec v[kDistillUnroll];
#pragma unroll 1
  for (int base = last; base >= 0; base -= kGroup) {
    const int slot0 = (last - base) / kDistillUnroll;  // of the parked vectors: kThreads a step of the unrolled loop
#pragma unroll
    for (int i = 0; i < kDistillUnroll; ++i) {
      const int at = base + i * kThreads;
      v[i] = at + tid < part.vecs ? load_vec_keep(in + (size_t)at * kVecBytes) : no_vec<T>();
    }
#pragma unroll
    for (int i = 0; i < kDistillUnroll; ++i) {
      const int at = base + i * kThreads + tid;
      if (at < part.vecs) {
        const uint32_t some = bits[at];
        if (some != 0) strike_out<T>(v[i], some);
        const int slot = slot0 * kDistillUnroll + i * kThreads + tid;
        if (slot < p.park_slots) park(planes, p.park_slots, slot, v[i]);
      }
    }
    float high = vec_max<T>(v[0]);
#pragma unroll
    for (int i = 1; i < kDistillUnroll; ++i) high = fmaxf(high, vec_max<T>(v[i]));
    const float m = fmaxf(a.m, high * p.c);
    if (m > a.m) a = sums_raise(a, m);
    const f2 c2 = make_f2(p.c, p.c), m2 = make_f2(-a.m, -a.m);
    Sums2 more{0, 0};
#pragma unroll
    for (int i = 0; i < kDistillUnroll; ++i)
      if (base + i * kThreads + tid < part.vecs) sums_add<T, false, false>(more, v[i], c2, m2);
    const float2 s = split_f2(more.s);
    a.s += s.x + s.y;
  }
  a = block_sums<kThreads>(a, sh.red);
  if (parts > 1) {
    cluster_wait();
    if (tid < parts) *in_cta(&sh.part[rank], tid) = a;
    cluster_arrive();
    cluster_wait();
    a = sh.part[0];
    for (int k = 1; k < parts; ++k) a = sums_merge(a, sh.part[k]);
  }
  Totals rest{(double)a.m, a.s, 0.f};
  const bool low = a.s == 0.f;
  if (low) {
    rest = low_sums<T, kThreads>(zrow, p.V, p.c, sh.red, [&](int v) {
      bool keep = true;
      for (int k = 0; k < p.top; ++k) keep &= sh.ids[k] != v;
      return keep;
    });
  }

  // ---- the list
  double scale = 0.0, at_listed = 0.0;
  if (tid < kTop) {
    const RowResult r = distill_row(id >= 0, mine, l, rest, p.c, p.dp, sh);
    const float w = p.weight != nullptr ? p.weight[row] : 1.f;
    double denominator = p.dp.denominator;
    if (!(denominator > 0.0)) {
      int n = 0;
      for (int i = tid & 31; i < p.n_counts; i += 32) n += p.counts[i].x;
      denominator = (double)__reduce_add_sync(0xffffffffu, n);
    }
    scale = (double)p.dp.coeff * w / (denominator * p.dp.temperature);
    at_listed = scale != 0.0 ? r.at * scale : 0.0;
    if (tid == 0) {
      sh.of_rest = scale != 0.0 && rest.s != 0.f ? (float)(r.of_rest * scale / rest.s) : 0.f;
      if (rank == 0) {
        p.term[row] = w != 0.f ? (double)w * r.kl : 0.0;
        if (p.row_kl != nullptr) p.row_kl[row] = (float)r.kl;
      }
    }
  }
  if (out == nullptr) return;
  __syncthreads();
  const float of_rest = sh.of_rest;
  if (of_rest == 0.f) {
    zero_part(out, part.n);
  } else if (low) {
    for (int i = tid; i < part.n; i += kThreads)
      store_f(out + i, ex2_approx((float)((double)load_f<T>(part.z + i) * (double)p.c - rest.x0)) * of_rest);
  } else {
    // ---- pass 2: the first group from registers, the others as pass 1 read them last to first
    const float m = -a.m;
    char* body_out = reinterpret_cast<char*>(out + part.head);
    const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(body_out) & (kVecBytes - 1);
#pragma unroll 1
    for (int base = 0; base <= last; base += kGroup) {
      if (base != 0) {
        const int slot0 = (last - base) / kDistillUnroll;
#pragma unroll
        for (int i = 0; i < kDistillUnroll; ++i) {
          const int at = base + i * kThreads, slot = slot0 * kDistillUnroll + i * kThreads + tid;
          v[i] = at + tid >= part.vecs ? no_vec<T>() : slot < p.park_slots ? parked(planes, p.park_slots, slot) : load_vec(in + (size_t)at * kVecBytes);
        }
      }
#pragma unroll
      for (int i = 0; i < kDistillUnroll; ++i) {
        Vec r;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if constexpr (sizeof(T) == 2)
            r.w[j] = pack_bf16x2(ex2_approx(fmaf(bf16lo_to_f32(v[i].w[j]), p.c, m)) * of_rest, ex2_approx(fmaf(bf16hi_to_f32(v[i].w[j]), p.c, m)) * of_rest);
          else
            r.w[j] = __float_as_uint(ex2_approx(fmaf(__uint_as_float(v[i].w[j]), p.c, m)) * of_rest);
        }
        const int at = base + i * kThreads + tid;
        char* dst = body_out + (size_t)at * kVecBytes;
        if (off == 0) {
          if (at < part.vecs) store_vec(dst, r);
        } else if (off == 16) {
          if (at < part.vecs) {
            __stcs(reinterpret_cast<uint4*>(dst), make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]));
            __stcs(reinterpret_cast<uint4*>(dst) + 1, make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]));
          }
        } else {
          const int count = max(0, min(32, part.vecs - (at - (tid & 31))));
          store_shifted<T>(dst - (size_t)(tid & 31) * kVecBytes, r, count, stage);
        }
      }
    }
    if (tid < part.head) store_f(out + tid, ex2_approx(fmaf(z_head, p.c, m)) * of_rest);
    if (tid < part.tail) store_f(out + part.n - part.tail + tid, ex2_approx(fmaf(z_tail, p.c, m)) * of_rest);
  }
  __syncthreads();  // the listed tokens over what stands in their places
  if (owner) store_f(out + rel, (float)at_listed);
}

// Sums of the rows' terms and counts, one CTA, in a fixed order.
__global__ void __launch_bounds__(1024) distill_finish_kernel(const DistillArgs p) {
  __shared__ double red[32];
  __shared__ int2 redc[32];
  wait_for_previous();
  double v = 0.0;
  for (long long i = threadIdx.x; i < p.N; i += 1024) v += p.term[i];
  v = block_sum(v, red);
  const int2 n = sum_counts(p.counts, p.n_counts, redc);
  if (threadIdx.x == 0) {
    const bool more = (p.dp.flags & MRL_FLAG_ACCUMULATE_LOSS) != 0;
    const double d = p.dp.denominator > 0.0 ? p.dp.denominator : (double)n.x;
    const double loss = d > 0.0 && p.dp.coeff != 0.f ? v * (double)p.dp.coeff / d : 0.0;
    p.loss[0] = (float)((more ? (double)p.loss[0] : 0.0) + loss);
    if (p.stats != nullptr) {
      p.stats[0] = (more ? p.stats[0] : 0) + n.x;
      p.stats[1] = (more ? p.stats[1] : 0) + n.y;
    }
  }
}

struct DistillWs {
  uint8_t* rowstat;
  int2 *counts, *sums;
  double* term;
  size_t bytes;
};
DistillWs carve(void* ws, long long N) {
  MrlCarver c(ws);
  DistillWs w;
  w.term = c.take<double>((size_t)N);
  w.counts = c.take<int2>((size_t)((N + kListRows - 1) / kListRows));
  w.sums = c.take<int2>(kCounts);
  w.rowstat = c.take<uint8_t>((size_t)N);
  w.bytes = c.off;
  return w;
}

bool row_type_ok(int32_t dtype) { return dtype == MRL_BF16 || dtype == MRL_F32; }
bool on_element(const void* p, int elem) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(elem - 1)) == 0; }
bool temperature_ok(float t) { return t >= 1e-6f && t <= 1e6f; }
float scale_of(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }

}  // namespace

size_t mrl_distill_workspace_bytes(long long N) { return N > 0 ? carve(nullptr, N).bytes : 0; }

extern "C" int mrl_top_logprobs(const void* logits, int32_t dtype, int64_t N, int32_t V, int64_t ld, const int32_t* ids,
                                const uint8_t* mask, float temperature, int32_t top, float* logp, float* lse, float* entropy,
                                int32_t* top_ids, float* top_logp, int32_t* status, void* stream) {
  if (!row_type_ok(dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
  if (N < 0 || V < 1 || ld < V || !temperature_ok(temperature) || top < 0 || top > V) return MRL_ERR_INVALID_ARG;
  if (top > kTop || N > 0x7fffffffll || V > (1 << 30)) return MRL_ERR_UNSUPPORTED_SHAPE;
  if (N == 0) return MRL_OK;
  if (top > 0 && (top_ids == nullptr || top_logp == nullptr)) return MRL_ERR_INVALID_ARG;
  if (top == 0) top_ids = nullptr, top_logp = nullptr;
  if (logp == nullptr && lse == nullptr && entropy == nullptr && top == 0) return MRL_ERR_INVALID_ARG;
  if (logits == nullptr || (ids == nullptr && logp != nullptr)) return MRL_ERR_INVALID_ARG;
  const void* outs[5] = {logp, lse, entropy, top_ids, top_logp};
  for (int i = 0; i < 5; ++i) {
    if (outs[i] == nullptr) continue;
    if (!on_element(outs[i], 4) || outs[i] == logits || outs[i] == ids || outs[i] == mask) return MRL_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (outs[i] == outs[j]) return MRL_ERR_INVALID_ARG;
  }
  if (!on_element(logits, dtype == MRL_BF16 ? 2 : 4) || !on_element(ids, 4) || !on_element(status, 4)) return MRL_ERR_INVALID_ARG;
  const TopArgs a{logits, ld, V, ids, mask, temperature, scale_of(temperature), top, logp, lse, entropy, top_logp, top_ids, status};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool bf16 = dtype == MRL_BF16, ent = entropy != nullptr;
  const int parts = parts_of(N, (long long)V * (bf16 ? 2 : 4), kTopCtas);
  mrl_profile_before(st, "top_kernel");
  const int rc = launch_rows(bf16 ? (ent ? top_kernel<__nv_bfloat16, true> : top_kernel<__nv_bfloat16, false>)
                                  : (ent ? top_kernel<float, true> : top_kernel<float, false>), N, parts, kTopThreads,
                             parts > 1 ? kPool * sizeof(Key) : 0, false, st, a);
  mrl_profile_after(st);
  return rc;
}

extern "C" int mrl_distill_loss_fwd_bwd(const void* logits, int32_t dtype, int64_t N, int32_t V, int64_t ld, const int32_t* top_ids,
                                        const float* top_logp, int32_t top, const uint8_t* mask, const float* row_weight,
                                        const mrl_distill_params* dp, void* dlogits, int64_t ld_out, float* row_kl, float* loss,
                                        int64_t* stats, int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
  if (!row_type_ok(dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
  if (dp == nullptr || N < 0 || V < 1 || ld < V || top < 1 || top > V || (dlogits != nullptr && ld_out < V)) return MRL_ERR_INVALID_ARG;
  if (top > kTop || V > (1 << 20) || N > 0x3fffffffll) return MRL_ERR_UNSUPPORTED_SHAPE;
  const bool forward = dp->direction == MRL_DISTILL_FORWARD, event = dp->rest == MRL_REST_EVENT;
  if (!temperature_ok(dp->temperature) || !(dp->coeff - dp->coeff == 0.f) || !(dp->denominator - dp->denominator == 0.0) ||
      (!forward && dp->direction != MRL_DISTILL_REVERSE) || (!event && dp->rest != MRL_REST_NONE) || (!forward && !event) ||
      !(dp->rest_floor >= (forward ? 0.f : FLT_MIN)) || dp->rest_floor >= 1.f || (dp->flags & ~MRL_FLAG_ACCUMULATE_LOSS) != 0)
    return MRL_ERR_INVALID_ARG;
  if (loss == nullptr || !on_element(loss, 4) || !on_element(stats, 8)) return MRL_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (N == 0) {
    if ((dp->flags & MRL_FLAG_ACCUMULATE_LOSS) == 0) {
      MRL_CUDA_OK(cudaMemsetAsync(loss, 0, 4, st));
      if (stats != nullptr) MRL_CUDA_OK(cudaMemsetAsync(stats, 0, 16, st));
    }
    return MRL_OK;
  }
  if (logits == nullptr || top_ids == nullptr || top_logp == nullptr) return MRL_ERR_INVALID_ARG;
  const int elem = dtype == MRL_BF16 ? 2 : 4;
  if (!on_element(logits, elem) || !on_element(dlogits, elem) || !on_element(top_ids, 4) || !on_element(top_logp, 4) ||
      !on_element(row_weight, 4) || !on_element(row_kl, 4) || !on_element(status, 4))
    return MRL_ERR_INVALID_ARG;
  if (dlogits == logits && ld_out != ld && N > 1) return MRL_ERR_INVALID_ARG;
  if (row_kl != nullptr && (row_kl == loss || row_kl == row_weight || row_kl == top_logp)) return MRL_ERR_INVALID_ARG;
  if (workspace == nullptr || workspace_bytes < mrl_distill_workspace_bytes(N)) return MRL_ERR_WORKSPACE_TOO_SMALL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MRL_ERR_INVALID_ARG;
  const DistillWs w = carve(workspace, N);
  const int blocks = (int)((N + kListRows - 1) / kListRows);
  DistillArgs a{logits, dlogits, ld, ld_out, N, V, top, top_ids, top_logp, mask, row_weight, *dp, scale_of(dp->temperature), row_kl,
                loss, reinterpret_cast<long long*>(stats), status, w.rowstat, w.counts, blocks, w.term, 0, 0};
  list_check_kernel<<<blocks, kListThreads, 0, st>>>(a);
  MRL_CUDA_OK(cudaGetLastError());
  if (blocks > kCounts) {
    MRL_CUDA_OK(mrl_launch_behind(counts_kernel, 1, 1024, st, w.counts, blocks, (blocks + kCounts - 1) / kCounts, w.sums));
    a.counts = w.sums;
    a.n_counts = kCounts;
  }
  // Rows of 512 KB or more are shared by two CTAs, so that the rows in flight still fit L2 between the passes.
  int parts = parts_of(N, (long long)V * elem, 2);
  if (parts == 1 && (long long)V * elem >= 512 * 1024) parts = 2;
  const long long off = static_cast<const char*>(dlogits) - static_cast<const char*>(logits);
  const bool shifted = dlogits != nullptr && (off % 16 != 0 || (N > 1 && (ld_out - ld) * elem % 16 != 0));
  a.bit_words = (int)mrl_align_up((size_t)((V + parts - 1) / parts + 16 + 31) / 32, 4);
  const size_t fixed = (size_t)a.bit_words * 4 + (shifted ? kStageBytes : 0);
  if (dlogits != nullptr && fixed < kDistillSmem) a.park_slots = (int)((kDistillSmem - fixed) / (kThreads * kVecBytes)) * kThreads;
  const size_t smem = fixed + (size_t)a.park_slots * kVecBytes;
  using Kernel = void (*)(const DistillArgs);
  const Kernel kernel = dtype == MRL_BF16 ? distill_kernel<__nv_bfloat16> : distill_kernel<float>;
  static std::atomic<uint64_t> attr_done;
  int rc = mrl_once_per_device(attr_done, [] {
    // the carve-out that two CTAs an SM need, as a percentage of the 228 KB it can give: the rest stays L1
    constexpr int kCarve = (int)((2 * (kDistillSmem + 4096) * 100 + 228 * 1024 - 1) / (228 * 1024));
    for (const Kernel k : {static_cast<Kernel>(distill_kernel<__nv_bfloat16>), static_cast<Kernel>(distill_kernel<float>)}) {
      cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout, kCarve);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  });
  if (rc != MRL_OK) return rc;
  mrl_profile_before(st, "distill_kernel");
  rc = launch_rows(kernel, N, parts, kThreads, smem, true, st, a);
  mrl_profile_after(st);
  if (rc != MRL_OK) return rc;
  MRL_CUDA_OK(mrl_launch_behind(distill_finish_kernel, 1, 1024, st, a));
  return MRL_OK;
}
