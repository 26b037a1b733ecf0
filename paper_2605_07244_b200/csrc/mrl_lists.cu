// Top tokens and learning from them: mrl_top_logprobs and mrl_distill_loss_fwd_bwd.
//
// Both read rows of logits against a running (m, s): m the largest of z c, c = log2(e) / T, and s = sum_v 2^(z_v c - m), each exponent one multiply-add.
// m is rounded and z c there is not, so the largest exponent is the product's rounding error: 64 at most where |z c| < 2^31, but thousands and up beyond (a mask
// of -1e10: 440), where 2^t is infinite or 0.  So m starts at -2^31: what lies below (masks of -1e10, -1e30, of the type's lowest value, -inf) adds 0, and a NaN
// always reaches the sum.  A row whose s is 0 is summed again against its largest logit itself: one with nothing above -2^31, and one with z c of
// 2^31 or more, whose s is made 0.
#include <float.h>

#include <type_traits>

#include "mrl_common.cuh"

namespace {

using namespace mrl;

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

template <typename T>
__device__ __forceinline__ float element(const Vec& v, int e) {
  const int j = sizeof(T) == 2 ? e >> 1 : e;
  const uint32_t a = j & 1 ? v.w[1] : v.w[0], b = j & 1 ? v.w[3] : v.w[2], c = j & 1 ? v.w[5] : v.w[4], d = j & 1 ? v.w[7] : v.w[6];
  const uint32_t w = j & 4 ? (j & 2 ? d : c) : (j & 2 ? b : a);
  return sizeof(T) == 4 ? __uint_as_float(w) : e & 1 ? bf16hi_to_f32(w) : bf16lo_to_f32(w);
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
  // (CTAs of a launch with a cluster's attribute, be the cluster one CTA, start at half the rate: 47,360 rows of 2,722 bf16 260 us instead of 143)
  cfg.attrs = parts > 1 ? attr : attr + 1;
  cfg.numAttrs = (behind ? 1 : 0) + (parts > 1 ? 1 : 0);
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
constexpr float kFar = 2147483648.f;  // 2^31
__device__ __forceinline__ Sums sums_empty() { return Sums{-kFar, 0.f, 0.f}; }
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
// Over the block, in a fixed order; every thread gets the result.  The maximum first, so that each thread rescales once.  (kRaw: whatever the maximum; otherwise
// s = 0 where it is kFar or more.)
template <int kT, bool kRaw = false>
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
  a = !kRaw && m >= kFar ? Sums{FLT_MAX, 0.f, 0.f} : sums_raise(a, m);
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
// The sums of a row whose s above is 0, against its largest logit: 2^((z - zm) c); without the `n` tokens of `ids`.  Called by the block; slow: two reads by
// single elements, and each token is compared with each of `ids` (distillation of 8,192 x 128,256 bf16 whose unlisted tokens are all masked: 779 -> 1,940 to 2,410 us).  (Plain arguments: what a lambda takes by reference is copied to every thread's stack before the kernel begins, 250 MB for 1,480 rows.)
template <typename T, int kT>
__device__ __noinline__ Totals low_sums(const T* z, int V, float c, Sums* red, const int* ids, int n) {
  auto listed = [&](int v) {
    bool found = false;
    for (int k = 0; k < n; ++k) found |= ids[k] == v;
    return found;
  };
  float zm = -FLT_MAX;
  for (int v = threadIdx.x; v < V; v += kT)
    if (!listed(v)) zm = fmaxf(zm, load_f<T>(z + v));
  Sums a{zm, 0.f, 0.f};
  __syncthreads();
  zm = block_sums<kT, true>(a, red).m;
  a = Sums{0.f, 0.f, 0.f};
  for (int v = threadIdx.x; v < V; v += kT)
    if (!listed(v)) sums_term<true, true>(load_f<T>(z + v) - zm, c, 0.f, a.s, a.u);
  __syncthreads();
  a = block_sums<kT, true>(a, red);
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
  float c;
  double nat;  // 1 / (c T)
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
// What a CTA of kT threads holds.  256 threads take any rows, and those that several CTAs share; 128 and 64 shorter ones.
template <int kT>
struct TopSize {
  static constexpr bool kAny = kT == 256;
  static constexpr int kCtas = kAny ? 5 : 1280 / kT;        // an SM
  static constexpr int kWarps = kT / 32;
  static constexpr int kNoted = kT >= 128 ? 2048 : 384;     // vectors noted
  static constexpr int kHeld = kAny ? 320 : kT;             // those of them whose elements are held
  static constexpr int kCap = kAny ? 1024 : 512;            // candidates
  static constexpr int kFew = kT;                           // keys that are put in order by counting
};
template <int kT>
struct TopShared {
  using Size = TopSize<kT>;
  Key cand[Size::kCap];                // candidates of this CTA
  Key list[Size::kFew];                // what is left of them, or (CTA 0) of the pool
  Sums part[Size::kAny ? kMaxParts : 1], red[Size::kWarps];
  uint4 held[2 * Size::kHeld];         // the first vectors noted
  alignas(16) int vec[Size::kNoted];   // vectors noted; then what puts the list in order
  uint32_t pick2[2 * Size::kWarps], n_vec, n_cand, n_list, n_pool;
};
// (CTA 0 of a row that several share) what is left of the candidates of all
constexpr int kPool = kMaxParts * TopSize<256>::kFew;

// Adds the first `want` tokens of a part whose logits are `z` to its candidates.
template <typename T, int kT>
__device__ __noinline__ void add_equal(const T* part, int n, int first, float z, int want, TopShared<kT>& sh) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll 1
  for (int r = 0; r < n && want > 0; r += kT) {
    const int i = r + threadIdx.x;
    const bool equal = i < n && load_f<T>(part + i) == z;
    const unsigned who = __ballot_sync(0xffffffffu, equal);
    if (lane == 0) sh.pick2[warp] = (uint32_t)__popc(who);
    __syncthreads();
    int before = __popc(who & ((1u << lane) - 1)), all = 0;
    for (int w = 0; w < kT / 32; ++w) {
      before += w < warp ? (int)sh.pick2[w] : 0;
      all += (int)sh.pick2[w];
    }
    if (equal && before < want) sh.cand[atomicAdd(&sh.n_cand, 1u)] = key_of(z, first + i);
    want -= all;
    __syncthreads();
  }
}

// The ordinal of the `want`th largest of a full list of candidates.
template <int kT>
__device__ __forceinline__ uint32_t nth_ordinal(const Key* cand, int want) {
  constexpr int kEach = TopSize<kT>::kCap / kT;
  uint32_t mine[kEach], found = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) mine[i] = (uint32_t)(cand[i * kT + threadIdx.x] >> 32);
#pragma unroll 1
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t next = found | (1u << bit);
    int total = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) total += __syncthreads_count(mine[i] >= next);
    if (total >= want) found = next;
  }
  return found;
}

// Copies the keys that can be among the `top` largest of `from` to `to` (of CTA `rank`, behind what its counter says is there): at most kFew,
// and all of the `top` largest among them.  Bits are settled from above until few enough are left.
template <int kMost, int kT>
__device__ __noinline__ void keep_largest(const Key* from, int n, int top, Key* to, uint32_t* n_to) {
  constexpr int kEach = kMost / kT, kFew = TopSize<kT>::kFew;
  Key mine[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) mine[i] = i * kT + threadIdx.x < n ? from[i * kT + threadIdx.x] : 0;
  Key least = 1;
  if (n > kFew) {
    least = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const Key next = least | ((Key)1 << bit);
      int total = __syncthreads_count(mine[0] >= next);
      if (n > kT) {
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
template <typename T, int kT>
__device__ __forceinline__ uint32_t kth_ordinal(uint32_t mine, int want, int more, uint32_t* red) {
  constexpr int kWarps = kT / 32;
  uint32_t high = __reduce_max_sync(0xffffffffu, mine), low = __reduce_min_sync(0xffffffffu, mine);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) red[warp] = high, red[kWarps + warp] = low;
  __syncthreads();
  high = __reduce_max_sync(0xffffffffu, red[lane % kWarps]);
  low = __reduce_min_sync(0xffffffffu, red[kWarps + lane % kWarps]);
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

// Candidates: what is not below `least_z`.  Behind kCap of them each takes an earlier one's place, by a hash of its index.  The vectors that were noted are
// read; where too many were (a row that rises) all are, once more.  At 16 kCap it is clear that the floor has to rise, and the rest is left (a row of one
// value, 2,048 x 151,936 bf16, top 20: 841 -> 307 us; random values 130).
template <typename T, int kT>
__device__ __forceinline__ void collect(const Part<T>& part, float z_head, float z_tail, float least_z, TopShared<kT>& sh) {
  constexpr int kCap = TopSize<kT>::kCap, kNoted = TopSize<kT>::kNoted, kHeld = TopSize<kT>::kHeld;
  const int tid = threadIdx.x;
  auto put = [&](uint32_t at, float z, int index) {
    if (at < kCap) sh.cand[at] = key_of(z, part.first + index);
    else atomicExch(&sh.cand[((uint32_t)index * 2654435769u) / (0xffffffffu / kCap + 1)], key_of(z, part.first + index));
  };
  if (tid < part.head && z_head >= least_z) put(atomicAdd(&sh.n_cand, 1u), z_head, tid);
  if (tid < part.tail && z_tail >= least_z) put(atomicAdd(&sh.n_cand, 1u), z_tail, part.n - part.tail + tid);
  const bool all = sh.n_vec > kNoted;
  const int noted = all ? part.vecs : (int)sh.n_vec;
  for (int k = tid; k < noted && *(volatile uint32_t*)&sh.n_cand < 16 * kCap; k += kT) {
    const int at = all ? k : sh.vec[k];
    Vec v;
    if (!all && k < kHeld) {
      const uint4 a = sh.held[k], b = sh.held[kHeld + k];
      v = Vec{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
    } else {
      v = load_vec(part.body() + (size_t)at * kVecBytes);
    }
    uint32_t bits = not_below<T>(v, least_z);
    uint32_t place = bits != 0 ? atomicAdd(&sh.n_cand, (uint32_t)__popc(bits)) : 0;
#pragma unroll 1
    for (; bits != 0; bits &= bits - 1) {
      const int e = __ffs(bits) - 1;
      put(place++, element<T>(v, e), part.head + at * kVecElems<T> + e);
    }
  }
}

// As kth_ordinal, of the largest elements of the quarters of each thread's vector: where a row has hardly more vectors than its list has places.
// (Those of whole vectors would be no floor, and all tokens candidates: 8,192 rows of 1,000 bf16, top 64: 141 us, this way 68.)
template <typename T, int kT>
__device__ __noinline__ uint32_t kth_of_quarters(const Vec v, int want) {
  uint32_t mine[4], found = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float high;
    if constexpr (sizeof(T) == 2)
      high = fmaxf(fmaxf(bf16lo_to_f32(v.w[2 * q]), bf16hi_to_f32(v.w[2 * q])), fmaxf(bf16lo_to_f32(v.w[2 * q + 1]), bf16hi_to_f32(v.w[2 * q + 1])));
    else
      high = fmaxf(__uint_as_float(v.w[2 * q]), __uint_as_float(v.w[2 * q + 1]));
    mine[q] = ordinal(high);
  }
  for (int bit = 31; bit >= (sizeof(T) == 2 ? 16 : 0); --bit) {
    const uint32_t next = found | (1u << bit);
    int n = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) n += __syncthreads_count(mine[q] >= next);
    if (n >= want) found = next;
    if (n >= want && n <= want + want / 4 + 2) break;
  }
  return max(found, kLowest);
}

template <typename T, bool kEnt, int kT>
__global__ void __launch_bounds__(kT, TopSize<kT>::kCtas) top_kernel(const TopArgs p) {
  using Size = TopSize<kT>;
  __shared__ TopShared<kT> sh;
  const int tid = threadIdx.x;
  int parts = 1, rank = 0;
  if (Size::kAny) {
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  }
  const long long row = blockIdx.x / (unsigned)parts;
  const T* zrow = static_cast<const T*>(p.logits) + row * p.ld;
  const int id = p.ids != nullptr ? p.ids[row] : 0;
  auto none = [&](bool bad_id) {
    if (tid == 0) {
      if (bad_id && p.status != nullptr) atomicOr(p.status, MRL_DEV_BAD_TOKEN_ID);
      if (p.logp != nullptr) p.logp[row] = 0.f;
      if (p.lse != nullptr) p.lse[row] = 0.f;
      if (kEnt) p.entropy[row] = 0.f;
    }
    if (tid < p.top) {
      p.top_ids[row * p.top + tid] = -1;
      p.top_logp[row * p.top + tid] = 0.f;
    }
  };
  if (p.mask != nullptr && p.mask[row] == 0) {  // (all CTAs of the row)
    if (rank == 0) none(false);
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
  // group in the same way, a tight one, and what is not below it is taken from the vectors noted: the first are held in shared memory, others read again.
  float best = z_head, floor = floor_of<T>(kLowest);
  const int groups = max(1, (part.vecs + kT * kUnroll - 1) / (kT * kUnroll));
#pragma unroll 1
  for (int g = 0; g < groups; ++g) {
    const int v0 = g * kT * kUnroll + tid;
    Vec v[kUnroll];
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) v[i] = v0 + i * kT < part.vecs ? load_vec(body + (size_t)(v0 - tid + i * kT) * kVecBytes) : no_vec<T>();
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
      if (v0 + i * kT < part.vecs) sums_add<T, kEnt, false>(more, v[i], c2, m2);
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
    if (part.vecs <= kT && 2 * p.top > part.vecs) floor = floor_of<T>(kth_of_quarters<T, kT>(v[0], p.top));
    else if (g == 0 || (g == kSecondFloor && g + 1 < groups)) floor = floor_of<T>(kth_ordinal<T, kT>(ordinal(best), p.top, p.top / 4, sh.pick2));
    int hits = 0;
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) hits += high[i] >= floor;
    if (hits != 0) {
      uint32_t at = atomicAdd(&sh.n_vec, (uint32_t)hits);
#pragma unroll
      for (int i = 0; i < kUnroll; ++i)
        if (high[i] >= floor) {
          if (at < Size::kNoted) sh.vec[at] = v0 + i * kT;
          if (at < Size::kHeld) {
            sh.held[at] = make_uint4(v[i].w[0], v[i].w[1], v[i].w[2], v[i].w[3]);
            sh.held[Size::kHeld + at] = make_uint4(v[i].w[4], v[i].w[5], v[i].w[6], v[i].w[7]);
          }
          ++at;
        }
    }
  }
  a = block_sums<kT>(a, sh.red);
  int n = 0;
  if (p.top > 0) {
    // (barriers: the vectors are noted; with one group the floor is the last one already)
    uint32_t least = groups == 1 ? max(ordinal(floor), kLowest) : kth_ordinal<T, kT>(ordinal(fmaxf(best, z_tail)), p.top, p.top / 16, sh.pick2);
    float crowd = -INFINITY;
    // More candidates than there is room for: the `top`th value of the kCap that were kept is the next floor, or what is above it, where that is the floor
    // already and so is what crowds the list.  Two rounds drop kCap - top of them at least.
#pragma unroll 1
    for (;;) {
      collect<T, kT>(part, z_head, z_tail, floor_of<T>(least), sh);
      __syncthreads();
      n = (int)sh.n_cand;
      if (n <= Size::kCap) break;
      const uint32_t higher = nth_ordinal<kT>(sh.cand, p.top);
      if (floor_of<T>(higher) > floor_of<T>(least)) {
        least = higher;
      } else {
        crowd = floor_of<T>(least);
        least = sizeof(T) == 2 ? ((ordinal(crowd) >> 16) + 1) << 16 : ordinal(crowd) + 1;
      }
      __syncthreads();  // (all have read the number)
      if (tid == 0) sh.n_cand = 0;
      __syncthreads();
    }
    // Masked tokens, or those of the value that crowds, from the front.
    if (n < min(p.top, part.n)) {
      __syncthreads();
      add_equal<T, kT>(part.z, part.n, part.first, crowd, p.top - n, sh);
      n = (int)sh.n_cand;
    }
  }
  if (parts > 1) {
    cluster_wait();
    if (tid == 0) *in_cta(&sh.part[rank], 0) = a;
    if (n > 0) keep_largest<Size::kCap, kT>(sh.cand, n, p.top, in_cta(pool, 0), in_cta(&sh.n_pool, 0));
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
    a = sh.part[0];
    for (int k = 1; k < parts; ++k) a = sums_merge(a, sh.part[k]);
    n = (int)sh.n_pool;
    if (n > 0) keep_largest<kPool, kT>(pool, n, p.top, sh.list, &sh.n_list);
  } else if (n > Size::kFew) {
    keep_largest<Size::kCap, kT>(sh.cand, n, p.top, sh.list, &sh.n_list);
  }
  const bool few = parts == 1 && n <= Size::kFew;  // the candidates are the list
  if (id < 0 || id >= p.V) {  // (asked here, so that the row's loads do not wait for the id's)
    none(true);
    return;
  }
  if (!few) {
    __syncthreads();
    n = (int)sh.n_list;
  }
  Totals t{(double)a.m, a.s, a.u};
  const bool low = t.s == 0.f;
  if (low) t = low_sums<T, kT>(zrow, p.V, p.c, sh.red, nullptr, 0);
  const float ln_s = t.s == 0.f ? NAN : logf(t.s), nat = (float)p.nat;
  // In order: a key's place is the number of larger ordinals, and of lower indices among those that share that place.  (64-bit keys compared as they are, four
  // threads a key: 2,051 x 50,021 float32, top 128, 123 us against 110.)
  uint32_t* ordinals = reinterpret_cast<uint32_t*>(sh.vec);
  uint32_t *shared_by = ordinals + kT, *low_half = shared_by + kT;
  const Key key = tid < n ? (few ? sh.cand : sh.list)[tid] : 0;
  const uint32_t mine = (uint32_t)(key >> 32);
  ordinals[tid] = mine;
  shared_by[tid] = 0;
  __syncthreads();
  int at = 0;
  if (tid < n) {
    const uint4* all = reinterpret_cast<const uint4*>(ordinals);
#pragma unroll 4
    for (int j = 0; j < (n + 3) / 4; ++j) {
      const uint4 o = all[j];
      at += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
    }
    low_half[at + atomicAdd(&shared_by[at], 1u)] = (uint32_t)key;
  }
  __syncthreads();
  if (tid < n) {
    const int first = at, others = (int)shared_by[at];
    for (int j = 0; others > 1 && j < others; ++j) at += low_half[first + j] > (uint32_t)key;
    if (at < p.top) {
      const float z = from_ordinal(mine);
      const float x = fmaf(z, p.c, -a.m);
      p.top_ids[row * p.top + at] = 0x7fffffff - (int32_t)(uint32_t)key;
      // (float64 where z c leaves float32)
      p.top_logp[row * p.top + at] = low || x < -FLT_MAX ? (float)(((double)z * (double)p.c - t.x0) * p.nat - (double)ln_s) : fmaf(x, nat, -ln_s);
    }
  }
  if (tid == kT - 32) {  // (a warp that has hardly any keys)
    const double ln_s64 = t.s == 0.f ? NAN : log((double)t.s);
    if (p.lse != nullptr) p.lse[row] = (float)(t.x0 * p.nat + ln_s64);
    if (p.logp != nullptr) p.logp[row] = (float)(((double)load_f<T>(zrow + id) * (double)p.c - t.x0) * p.nat - ln_s64);
    if (kEnt) p.entropy[row] = (float)(ln_s64 - (double)t.u / (double)t.s * p.nat);
  }
  for (int k = n + tid; k < p.top; k += kT) {
    p.top_ids[row * p.top + k] = -1;
    p.top_logp[row * p.top + k] = -INFINITY;
  }
}

// ------------------------------------------------------------------------------------------ distillation
// Three kernels.  list_kernel: which rows count, and what a row's list gives by itself.  distill_kernel: the rows of logits, the bulk of the work.  finish_kernel: the
// gradient of the listed tokens, and the loss.
constexpr int kRowOff = 0, kRowValid = 1, kRowRefused = 2;
constexpr int kListThreads = 256, kListRows = kListThreads / 32;  // of a CTA of list_kernel: a warp per row
constexpr int kPlaces = kTop / 32;                 // places of a lane

// Of a row's list.  With x_k = z_k / T, xs the largest of them, e_k = exp(x_k - xs), q_k the teacher's probabilities:
struct ListRecord {
  double xs;      // in units of z c
  double sum_e;   // sum e_k
  double mass;    // sum q_k
  double mixed;   // forward: sum q_k (ln q_k - (x_k - xs)); reverse: sum e_k ((x_k - xs) - ln q_k)
  double q_rest, ln_q_rest;
  double ln_one;  // ln q_k = top_logp_k - ln_one
  // what the gradient of the rest needs, in float32, so that it is there soon
  float zs;              // the largest listed logit
  float sum_e_f, mass_f, q_rest_f;
  float against, against_lo;  // reverse: ln q_rest + mixed / sum_e, in two floats
  float weight;
  int stat;       // kRow*
};
// Of a row, for its listed tokens: p_k = p_of_e e_k, ln p_k = (x_k - xs) + shift
struct RowFactors {
  double shift, kl;
  double mass;    // forward: sum q_k + q_rest
  double scale;   // coeff weight / (D T)
  float p_of_e, of_rest;  // T dKL/dz_v = of_rest * softmax over the rest (v); rest_factor gives it sooner
};

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
  double nat;            // 1 / (c T)
  float *row_kl, *loss;
  long long* stats;
  int32_t* status;
  ListRecord* records;   // [N]
  float* z;              // [N, top] the listed tokens' logits (the gradient may be written over them)
  RowFactors* factors;   // [N]
  double* term;          // [N] weight_t KL_t
  int2* counts;          // valid and refused rows: of kListRows rows each, or sums of those, kCounts at most
  int n_counts;
  int bit_words, park_slots;  // shared memory of distill_kernel
};

__device__ __forceinline__ double warp_sum(double a) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
  return a;
}

// A row's list: is it one to learn from, and its sums?  The entries stay in registers, kPlaces a lane; a token twice shows when every entry is compared
// with those of the other places, carried round the warp.
template <typename T>
__global__ void __launch_bounds__(kListThreads) list_kernel(const DistillArgs p) {
  __shared__ int2 part[kListThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  let_next_start();
  int2 n{0, 0};
  for (int r = warp; r < kListRows; r += kListThreads / 32) {
    const long long row = (long long)blockIdx.x * kListRows + r;
    if (row >= p.N) break;
    if (p.mask != nullptr && p.mask[row] == 0) {
      if (lane == 0) p.records[row].stat = kRowOff;
      continue;
    }
    int id[kPlaces];
    float l[kPlaces], z[kPlaces];
    int bad = 0;
    bool any = false;
#pragma unroll
    for (int q = 0; q < kPlaces; ++q) {
      const int k = q * 32 + lane;
      id[q] = k < p.top ? p.top_ids[row * p.top + k] : -1;
      l[q] = k < p.top ? p.top_logp[row * p.top + k] : -INFINITY;
    }
#pragma unroll
    for (int q = 0; q < kPlaces; ++q) {
      if (id[q] < 0) l[q] = -INFINITY;
      if (!(l[q] < INFINITY)) bad |= MRL_DEV_BAD_LIST;  // (NaN too)
      if (l[q] == -INFINITY) id[q] = -1;
      if (id[q] >= p.V) bad |= MRL_DEV_BAD_TOKEN_ID;
      any |= id[q] >= 0;
      z[q] = id[q] >= 0 && id[q] < p.V ? load_f<T>(static_cast<const T*>(p.logits) + row * p.ld + id[q]) : 0.f;
    }
    const int used = (p.top + 31) / 32;
#pragma unroll 1
    for (int o = 0; o <= 16; ++o) {  // (of two lanes one is at most 16 ahead of the other)
#pragma unroll
      for (int q = 0; q < kPlaces; ++q) {
        if (q >= used) break;
        const int other = __shfl_sync(0xffffffffu, id[q], (lane + o) & 31);
#pragma unroll
        for (int j = 0; j < kPlaces; ++j) {
          if (j >= used) break;
          if (other >= 0 && other == id[j] && !(o == 0 && j == q)) bad |= MRL_DEV_BAD_LIST;
        }
      }
    }
    bad = __reduce_or_sync(0xffffffffu, bad);
    any = __any_sync(0xffffffffu, any);
    const int stat = bad != 0 ? kRowRefused : any ? kRowValid : kRowOff;
    n.x += stat == kRowValid;
    n.y += stat == kRowRefused;
    if (stat != kRowValid) {
      if (lane == 0) {
        p.records[row].stat = stat;
        if (bad != 0 && p.status != nullptr) atomicOr(p.status, bad);
      }
      continue;
    }
    float zs = -FLT_MAX, ls = -FLT_MAX;
#pragma unroll
    for (int q = 0; q < kPlaces; ++q)
      if (id[q] >= 0) {
        zs = z[q] == z[q] ? fmaxf(zs, z[q]) : INFINITY;  // (NaN: inf - inf below)
        ls = fmaxf(ls, l[q]);
      }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      zs = fmaxf(zs, __shfl_xor_sync(0xffffffffu, zs, o));
      ls = fmaxf(ls, __shfl_xor_sync(0xffffffffu, ls, o));
    }
    const bool event = p.dp.rest == MRL_REST_EVENT, forward = p.dp.direction == MRL_DISTILL_FORWARD;
    ListRecord rec{};
    rec.xs = (double)zs * (double)p.c;
    double x[kPlaces], e[kPlaces], q[kPlaces];
#pragma unroll
    for (int i = 0; i < kPlaces; ++i) {
      x[i] = e[i] = q[i] = 0.0;
      if (id[i] >= 0) {
        x[i] = ((double)z[i] * (double)p.c - rec.xs) * p.nat;
        e[i] = exp(x[i]);
        q[i] = exp(event ? (double)l[i] : (double)l[i] - (double)ls);  // (without a rest any logits will do: from the largest)
      }
      rec.sum_e += e[i];
      rec.mass += q[i];
      if (i * 32 + lane < p.top) p.z[row * p.top + i * 32 + lane] = z[i];
    }
    rec.sum_e = warp_sum(rec.sum_e);
    rec.mass = warp_sum(rec.mass);
    rec.ln_one = event ? 0.0 : (double)ls + log(rec.mass);  // (scaled to 1)
    const double to_one = event ? 1.0 : 1.0 / rec.mass;
#pragma unroll
    for (int i = 0; i < kPlaces; ++i) {
      const double ratio = x[i] - ((double)l[i] - rec.ln_one);
      if (id[i] >= 0 && forward && q[i] > 0.0) rec.mixed -= q[i] * to_one * ratio;
      if (id[i] >= 0 && !forward && e[i] != 0.0) rec.mixed += e[i] * ratio;
    }
    rec.mixed = warp_sum(rec.mixed);
    if (event) {
      rec.q_rest = fmax(1.0 - rec.mass, (double)p.dp.rest_floor);
      rec.ln_q_rest = rec.q_rest > 0.0 ? log(rec.q_rest) : 0.0;
    } else {
      rec.mass = 1.0;
    }
    rec.zs = zs;
    rec.sum_e_f = (float)rec.sum_e;
    rec.mass_f = (float)rec.mass;
    rec.q_rest_f = (float)rec.q_rest;
    const double against = rec.ln_q_rest + rec.mixed / rec.sum_e;
    rec.against = (float)against;
    rec.against_lo = (float)(against - (double)rec.against);
    rec.weight = p.weight != nullptr ? p.weight[row] : 1.f;
    rec.stat = kRowValid;
    if (lane == 0) p.records[row] = rec;
  }
  if (lane == 0) part[warp] = n;
  __syncthreads();
  if (warp == 0) {
    n = lane < kListThreads / 32 ? part[lane] : int2{0, 0};
    n.x = __reduce_add_sync(0xffffffffu, n.x);
    n.y = __reduce_add_sync(0xffffffffu, n.y);
    if (lane == 0) p.counts[blockIdx.x] = n;
  }
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

// Listed tokens and rest of a row are told apart by a bit for each element in shared memory: a vector's bits are one word, hardly ever other than 0.  Pass 1
// sums the rest, a few steps join it with the list's record, and pass 2 writes of_rest * 2^(z c - m), and 0 for the listed tokens, whose gradient comes behind
// the last row.  As in the policy loss's kernel the row is read from HBM once: pass 1 walks it from its end, the group read last stays in registers, the first ones
// are parked in shared memory, the rest comes from L2.  (A small load takes some 3 us while all others stream: what a row needs besides its logits is asked for
// together with its first vectors.)
constexpr int kDistillUnroll = 4;
// CTAs of kT threads: 512 for rows of any length, and those that several CTAs share; 128 for short ones.
constexpr uint32_t kStageRow = kVecBytes * 32;
template <int kT>
struct DistillSize {
  static constexpr bool kAny = kT == 512;
  static constexpr int kCtas = 1024 / kT;   // an SM
  static constexpr int kStream = kT - 32;   // threads that work on the logits; the last warp works on the list (in float64: with vectors in its registers too it would spill)
  // Shared memory of a CTA: bits, parked vectors, staging of outputs that start off 16 bytes from their inputs.  What it leaves is L1, which holds the
  // loads in flight.
  static constexpr size_t kSmem = kT * 136;
  static constexpr uint32_t kStageBytes = kT / 32 * kStageRow;
};
// Bytes of a row up to which 128 threads work on it, where rows are more than CTAs of 512 fit: loads, sums and barriers of more rows overlap (20,000 rows of 1,000
// float32 302 -> 110 us, 2,000 of 32,003 bf16 93 -> 75; of 20,000 float32, 80 KB, 77 and 78; of 32,768 105 and 122).
constexpr long long kShortRow = 64 * 1024;
// A rest whose largest logit (x0 in units of z c) is a mask, kMask or less, and which the learner leaves nothing, is no event.  What else has a small p_r is one,
// however small: at T = 0.01 logits 8 apart make ln p_r = -800.  (A power of two, so that it is exact times c.)
constexpr double kNoRest = -700.0, kMask = -67108864.0;
__device__ __forceinline__ bool masked_away(double ln_p_rest, double x0, float c) { return ln_p_rest < kNoRest && x0 <= kMask * (double)c; }

template <int kT>
struct DistillShared {
  Sums part[DistillSize<kT>::kAny ? kMaxParts : 1], red[kT / 32];
  float of_rest;
  uint32_t head_bits, tail_bits;
  int ids[kTop];
};

// exp(d), d <= 0 in units of z c (so 2^d but for the rounding of c), and ln of a float, their arguments split so that float32 functions are off by some
// 1e-7 of the first and 3e-8 in the second, whatever the size: as exact as the sums that they are applied to, at a fraction of float64's latency.
__device__ __forceinline__ float exp_of(double d, double nat) {
  if (!(d > -1000.0)) return d == d && d < 0.0 ? 0.f : NAN;
  const int whole = (int)rint(d);
  return ldexpf(expf((float)((d - (double)whole) * nat)), max(whole, -200));
}
__device__ __forceinline__ double ln_of(float v) {  // v > 0 and normal, or +inf, NaN
  if (!(v <= FLT_MAX)) return (double)v;
  int whole = (int)(__float_as_uint(v) >> 23) - 127;
  float part = __uint_as_float((__float_as_uint(v) & 0x007fffffu) | 0x3f800000u);
  if (part > 1.41421356f) part *= 0.5f, ++whole;
  return (double)whole * 0.69314718055994530942 + (double)logf(part);
}

// The rest's gradient from a list's record and the sums over the rest: T dKL/dz_v = rest_factor * softmax over the rest (v).  In float32, for all other warps
// wait for it (float64 took 4,000 cycles here).  With p_r and P the learner's mass on the rest and on the list:
//   forward  (sum q_k + q_r) p_r - q_r;   no rest in the teacher  p_r
//   reverse  p_r (ln p_r - ln q_r - KL) = p_r P (ln s - d - (ln q_r + mixed / sum_e)), where the difference is taken in two floats a term
__device__ __forceinline__ float rest_factor(const ListRecord& list, Sums a, float c, float nat_hi, float nat_lo, const mrl_distill_params& dp) {
  const float d = fmaf(list.zs, c, -a.m);  // from the largest of the rest to the largest of the list, in units of z c
  const float of_list = d < 0.f ? exp2f(d) : 1.f, of_rest = d < 0.f ? 1.f : exp2f(-d);
  const float in_list = list.sum_e_f * of_list, in_rest = a.s * of_rest, total = in_list + in_rest;
  const float p_rest = in_rest / total;
  if (dp.rest != MRL_REST_EVENT) return p_rest;
  if (!(p_rest >= 1e-30f) && p_rest == p_rest) {  // is there a rest?
    const double ln_p_rest = (double)logf(a.s / total) - (d > 0.f ? (double)d * (double)nat_hi : 0.0);
    if (masked_away(ln_p_rest, (double)a.m, c)) return 0.f;
  }
  if (dp.direction == MRL_DISTILL_FORWARD) return fmaf(list.mass_f + list.q_rest_f, p_rest, -list.q_rest_f);
  if (in_list == 0.f || p_rest == 0.f) return 0.f;  // (a list masked away, or one logit far above all: d may be infinite)
  int whole = (int)(__float_as_uint(a.s) >> 23) - 127;  // ln s = whole ln 2 + ln part
  float part = __uint_as_float((__float_as_uint(a.s) & 0x007fffffu) | 0x3f800000u);
  if (part > 1.41421356f) part *= 0.5f, ++whole;
  constexpr float kLn2Hi = 0.693145751953125f, kLn2Lo = 1.42860677e-6f;  // ln 2; products of the first and of small whole numbers are exact
  const float u = (float)whole * kLn2Hi, w = d * nat_hi, v = u - w, v_err = (u - v) - w;
  const float x = v - list.against, x_err = (v - x) - list.against;
  const float rest = (logf(part) + (float)whole * kLn2Lo) - fmaf(d, nat_lo, fmaf(d, nat_hi, -w)) - list.against_lo;
  return p_rest * (in_list / total) * (x + (x_err + v_err + rest));
}

// A row's KL, and what its listed tokens' gradient takes
__device__ __forceinline__ RowFactors distill_row(const ListRecord& list, Totals rest, float c, double nat, const mrl_distill_params& dp) {
  const bool event = dp.rest == MRL_REST_EVENT, any_rest = rest.s != 0.f;
  const double m = any_rest ? fmax(list.xs, rest.x0) : list.xs, below = list.xs - m, below_rest = rest.x0 - m;
  const float of_list = exp_of(below, nat), in_rest = any_rest ? rest.s * exp_of(below_rest, nat) : 0.f;
  const float total = fmaf((float)list.sum_e, of_list, in_rest);
  const double ln_total = total > 0.f ? ln_of(total) : NAN;
  RowFactors r;
  r.shift = below * nat - ln_total;
  r.p_of_e = of_list / total;
  const double ln_p_rest = any_rest ? ln_of(rest.s) + below_rest * nat - ln_total : -INFINITY;
  const bool has_rest = any_rest && !masked_away(ln_p_rest, rest.x0, c);
  r.mass = list.mass;
  const float p_rest = has_rest ? in_rest / total : 0.f;
  r.of_rest = p_rest;
  if (!event || dp.direction == MRL_DISTILL_FORWARD) {
    r.kl = list.mixed - list.mass * r.shift;
    if (event && has_rest) {
      r.mass += list.q_rest;
      if (list.q_rest > 0.0) r.kl += list.q_rest * (list.ln_q_rest - ln_p_rest);
      r.of_rest = (float)(r.mass * (double)p_rest - list.q_rest);
    }
  } else {
    r.kl = r.p_of_e != 0.f ? (double)r.p_of_e * (list.mixed + r.shift * list.sum_e) : 0.0;
    if (p_rest != 0.f) {
      r.kl += (double)p_rest * (ln_p_rest - list.ln_q_rest);
      r.of_rest = (float)((double)p_rest * (ln_p_rest - list.ln_q_rest - r.kl));
    }
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
// asks L2 for `bytes` (a multiple of 16) from `p` (on 16 bytes)
__device__ __forceinline__ void prefetch_l2(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
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

template <typename T, int kStream>
__device__ void zero_part(T* out, int n) {
  const int head = min(n, (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(out)) & 15) / (int)sizeof(T));
  const int pieces = (n - head) / (16 / (int)sizeof(T)), tail0 = head + pieces * (16 / (int)sizeof(T));
  for (int i = threadIdx.x; i < pieces; i += kStream) __stcs(reinterpret_cast<uint4*>(out + head) + i, make_uint4(0, 0, 0, 0));
  if ((int)threadIdx.x < head) store_f(out + threadIdx.x, 0.f);
  if (tail0 + (int)threadIdx.x < n) store_f(out + tail0 + threadIdx.x, 0.f);
}

// The sums over the rest of a row from those of this thread, over all CTAs of the row; `low`: their offset is not a.m.  Called by all threads.
template <typename T, int kT>
__device__ __forceinline__ Totals rest_of_row(Sums& a, bool& low, const DistillArgs& p, const T* zrow, int parts, int rank, DistillShared<kT>& sh) {
  a = block_sums<kT>(a, sh.red);
  if (parts > 1) {
    cluster_wait();
    if ((int)threadIdx.x < parts) *in_cta(&sh.part[rank], threadIdx.x) = a;
    cluster_arrive();
    cluster_wait();
    a = sh.part[0];
    for (int k = 1; k < parts; ++k) a = sums_merge(a, sh.part[k]);
  }
  low = a.s == 0.f;
  if (!low) return Totals{(double)a.m, a.s, 0.f};
  const Totals t = low_sums<T, kT>(zrow, p.V, p.c, sh.red, sh.ids, p.top);
  if (parts > 1) {  // (the whole row was read: no CTA may write its gradient over it before all have)
    cluster_arrive();
    cluster_wait();
  }
  return t;
}

// kShifted: outputs need not start on the same bytes of 32 as their inputs.  (A kernel of its own: code that a row runs through once comes from far, some 30 cycles
// an instruction, if the loops leave no room for it near the SM.)
template <typename T, bool kShifted, int kT>
__global__ void __launch_bounds__(kT, DistillSize<kT>::kCtas) distill_kernel(const DistillArgs p) {
  constexpr int kStream = DistillSize<kT>::kStream;
  extern __shared__ uint4 dyn[];
  __shared__ DistillShared<kT> sh;
  const int tid = threadIdx.x, lane = tid & 31;
  int parts = 1, rank = 0;
  if (DistillSize<kT>::kAny) {
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(parts));
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  }
  const long long row = blockIdx.x / (unsigned)parts;
  const T* zrow = static_cast<const T*>(p.logits) + row * p.ld;
  const Part<T> part(zrow, p.V, parts, rank);
  T* out = p.dlogits != nullptr ? static_cast<T*>(p.dlogits) + row * p.ld_out + part.first : nullptr;
  // shared memory: bits of the body's vectors | parked vectors | staging
  using Bits = typename std::conditional<sizeof(T) == 2, uint16_t, uint8_t>::type;
  Bits* bits = reinterpret_cast<Bits*>(dyn);

  if (tid >= kStream) {
    // ---- the last warp: the list
    int id[kPlaces];
    float l[kPlaces];
#pragma unroll
    for (int i = 0; i < kPlaces; ++i) {
      const int k = lane + 32 * i;
      id[i] = k < p.top ? p.top_ids[row * p.top + k] : -1;
      l[i] = k < p.top ? p.top_logp[row * p.top + k] : -INFINITY;
    }
    wait_for_previous();
    let_next_start();  // (behind the wait: what list_kernel wrote is there when finish_kernel starts)
    // (a word of the record a lane, and the counts: they come together)
    constexpr int kRecordWords = (int)sizeof(ListRecord) / 4;
    const int stat = p.records[row].stat, word = reinterpret_cast<const int*>(p.records + row)[lane % kRecordWords];
    int valid = lane < p.n_counts ? p.counts[lane].x : 0;
    if (stat != kRowValid) {
      if (lane == 0 && rank == 0) {
        p.term[row] = 0.0;
        if (p.row_kl != nullptr) p.row_kl[row] = 0.f;
      }
      return;
    }
    __syncthreads();  // the bits are zero
    if (parts > 1) cluster_arrive();  // "here": its shared memory may be written to
#pragma unroll
    for (int i = 0; i < kPlaces; ++i) {
      if (l[i] == -INFINITY) id[i] = -1;
      sh.ids[lane + 32 * i] = id[i];
      const int rel = id[i] - part.first, at = rel - part.head;  // the listed token in this part
      if (id[i] < 0 || rel < 0 || rel >= part.n) continue;
      if (at < 0) atomicOr(&sh.head_bits, 1u << rel);
      else if (at >= part.vecs * kVecElems<T>) atomicOr(&sh.tail_bits, 1u << (at - part.vecs * kVecElems<T>));
      else atomicOr(reinterpret_cast<uint32_t*>(dyn) + (at >> 5), 1u << (at & 31));
    }
    __syncthreads();  // the bits are set
    union {
      ListRecord list;
      int words[kRecordWords];
    } rec;
#pragma unroll
    for (int k = 0; k < kRecordWords; ++k) rec.words[k] = __shfl_sync(0xffffffffu, word, k);
    const double denominator = p.dp.denominator > 0.0 ? p.dp.denominator : (double)__reduce_add_sync(0xffffffffu, valid);
    const double scale = (double)p.dp.coeff * rec.list.weight / (denominator * p.dp.temperature);
    const float scale_f = (float)scale, nat_hi = (float)p.nat, nat_lo = (float)(p.nat - (double)nat_hi);
    Sums a = sums_empty();
    bool low;
    const Totals rest = rest_of_row<T, kT>(a, low, p, zrow, parts, rank, sh);
    if (lane == 0) {
      float f = 0.f;
      if (scale != 0.0 && rest.s != 0.f)
        f = (low ? distill_row(rec.list, rest, p.c, p.nat, p.dp).of_rest : rest_factor(rec.list, a, p.c, nat_hi, nat_lo, p.dp)) / rest.s * scale_f;
      sh.of_rest = f;
    }
    __syncwarp();
    if (out != nullptr) asm volatile("bar.arrive 1, %0;" ::"n"(kT) : "memory");
    RowFactors r = distill_row(rec.list, rest, p.c, p.nat, p.dp);
    r.scale = scale;
    if (lane == 0 && rank == 0) {
      p.factors[row] = r;
      p.term[row] = rec.list.weight != 0.f ? (double)rec.list.weight * r.kl : 0.0;
      if (p.row_kl != nullptr) p.row_kl[row] = (float)r.kl;
    }
    return;
  }

  // ---- the other warps: the logits.  The first loads wait for nothing: the logits were there before list_kernel began.  (A row that is not valid reads
  // them in vain.)
  constexpr int kGroup = kStream * kDistillUnroll;
  const char* in = part.body() + (size_t)tid * kVecBytes;
  const int last = part.vecs > 0 ? (part.vecs - 1) / kGroup * kGroup : -kGroup;
  Vec v[kDistillUnroll];
  auto load_group = [&](int base) {
#pragma unroll
    for (int i = 0; i < kDistillUnroll; ++i) {
      const int at = base + i * kStream;
      v[i] = at + tid < part.vecs ? load_vec_keep(in + (size_t)at * kVecBytes) : no_vec<T>();
    }
  };
  load_group(max(last, 0));
  const float z_head = tid < part.head ? load_f<T>(part.z + tid) : -INFINITY;
  const float z_tail = tid < part.tail ? load_f<T>(part.z + part.n - part.tail + tid) : -INFINITY;
  wait_for_previous();
  let_next_start();
  const int stat = p.records[row].stat;
  uint4* planes = dyn + p.bit_words / 4;
  for (int i = tid; i < p.bit_words / 4; i += kStream) dyn[i] = make_uint4(0, 0, 0, 0);
  if (tid == 0) sh.head_bits = sh.tail_bits = 0;
  if (stat != kRowValid) {  // (all CTAs of the row)
    if (out != nullptr) zero_part<T, kStream>(out, part.n);
    return;
  }
  __syncthreads();
  if (parts > 1) cluster_arrive();
  __syncthreads();
  Sums a = sums_empty();
  if (tid < part.head && !((sh.head_bits >> tid) & 1u)) sums_add(a, z_head, p.c);
  if (tid < part.tail && !((sh.tail_bits >> tid) & 1u)) sums_add(a, z_tail, p.c);

  // pass 1, from the last group (the ragged one) to the first, which is a full one wherever there are two
#pragma unroll 1
  for (int base = last; base >= 0; base -= kGroup) {
    if (base != last) load_group(base);
    if (tid == 0 && base > 0) prefetch_l2(part.body() + (size_t)(base - kGroup) * kVecBytes, kGroup * kVecBytes);
#pragma unroll
    for (int i = 0; i < kDistillUnroll; ++i) {
      const int at = base + i * kStream + tid;
      if (at < part.vecs) {
        const uint32_t some = bits[at];
        if (some != 0) strike_out<T>(v[i], some);
        const int slot = last - base + i * kStream + tid;
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
      if (base + i * kStream + tid < part.vecs) sums_add<T, false, false>(more, v[i], c2, m2);
    const float2 s = split_f2(more.s);
    a.s += s.x + s.y;
  }
  bool low;
  const double x0 = rest_of_row<T, kT>(a, low, p, zrow, parts, rank, sh).x0;
  if (out == nullptr) return;
  asm volatile("bar.sync 1, %0;" ::"n"(kT) : "memory");  // the list warp has the factor
  const float of_rest = sh.of_rest;
  if (of_rest == 0.f) {
    zero_part<T, kStream>(out, part.n);
    return;
  }
  if (low) {
    for (int i = tid; i < part.n; i += kStream) store_f(out + i, ex2_approx((float)((double)load_f<T>(part.z + i) * (double)p.c - x0)) * of_rest);
    return;
  }

  // pass 2: the first group from registers, the others as pass 1 read them last to first
  const float m = -a.m;
  char* body_out = reinterpret_cast<char*>(out + part.head);
  const bool aligned = (reinterpret_cast<uintptr_t>(body_out) & (kVecBytes - 1)) == 0;
  uint32_t* stage = reinterpret_cast<uint32_t*>(planes + 2 * p.park_slots) + (tid >> 5) * (kStageRow / 4);
#pragma unroll 1
  for (int base = 0; base <= last; base += kGroup) {
    if (base != 0) {
#pragma unroll
      for (int i = 0; i < kDistillUnroll; ++i) {
        const int at = base + i * kStream, slot = last - base + i * kStream + tid;
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
      const int at = base + i * kStream + tid;
      char* dst = body_out + (size_t)at * kVecBytes;
      if (!kShifted || aligned) {
        if (at < part.vecs) store_vec(dst, r);
      } else {
        const int count = max(0, min(32, part.vecs - (at - lane)));
        store_shifted<T>(dst - (size_t)lane * kVecBytes, r, count, stage);
      }
    }
  }
  if (tid < part.head) store_f(out + tid, ex2_approx(fmaf(z_head, p.c, m)) * of_rest);
  if (tid < part.tail) store_f(out + part.n - part.tail + tid, ex2_approx(fmaf(z_tail, p.c, m)) * of_rest);
}

// The gradient of the listed tokens, a warp per row, over what stands in their places; the first CTA sums the rows' terms and counts in a fixed order.
template <typename T>
__global__ void __launch_bounds__(1024) finish_kernel(const DistillArgs p) {
  __shared__ double red[32];
  __shared__ int2 redc[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x > 0) {
    const long long row = (long long)(blockIdx.x - 1) * 32 + warp;
    // what is known before the rows are done: list_kernel's results (from L2: it ended before distill_kernel's CTAs let this kernel start)
    const bool valid = row < p.N && __ldcg(&p.records[row].stat) == kRowValid;
    int id[kPlaces];
    double x[kPlaces], ln_q[kPlaces], e[kPlaces];
    if (valid) {
      const double xs = __ldcg(&p.records[row].xs), ln_one = __ldcg(&p.records[row].ln_one);
#pragma unroll
      for (int i = 0; i < kPlaces; ++i) {
        const int k = i * 32 + lane;
        id[i] = -1;
        if (k >= p.top) continue;
        id[i] = p.top_ids[row * p.top + k];
        const float l = p.top_logp[row * p.top + k];
        if (l == -INFINITY) id[i] = -1;
        x[i] = ((double)__ldcg(p.z + row * p.top + k) * (double)p.c - xs) * p.nat;
        ln_q[i] = (double)l - ln_one;
      }
#pragma unroll
      for (int i = 0; i < kPlaces; ++i)
        if (id[i] >= 0) {
          e[i] = exp(x[i]);
          if (p.dp.direction == MRL_DISTILL_FORWARD) ln_q[i] = exp(ln_q[i]);  // (q itself)
        }
    }
    wait_for_previous();
    if (!valid) return;
    const RowFactors r = p.factors[row];
    T* out = static_cast<T*>(p.dlogits) + row * p.ld_out;
#pragma unroll
    for (int i = 0; i < kPlaces; ++i) {
      if (id[i] < 0) continue;
      const double pk = e[i] * (double)r.p_of_e;
      double g;
      if (p.dp.direction == MRL_DISTILL_REVERSE) g = pk != 0.0 ? pk * (x[i] - ln_q[i] + r.shift - r.kl) : 0.0;
      else g = r.mass * pk - ln_q[i];
      store_f(out + id[i], r.scale != 0.0 ? (float)(g * r.scale) : 0.f);
    }
    return;
  }
  wait_for_previous();
  double v = 0.0;
  for (long long i = threadIdx.x; i < p.N; i += 1024) v += p.term[i];
  v = warp_sum(v);
  int2 n{0, 0};
  for (int i = threadIdx.x; i < p.n_counts; i += 1024) {
    n.x += p.counts[i].x;
    n.y += p.counts[i].y;
  }
  n.x = __reduce_add_sync(0xffffffffu, n.x);
  n.y = __reduce_add_sync(0xffffffffu, n.y);
  if (lane == 0) red[warp] = v, redc[warp] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < 32; ++k) {
      v += red[k];
      n.x += redc[k].x;
      n.y += redc[k].y;
    }
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
  ListRecord* records;
  RowFactors* factors;
  float* z;
  double* term;
  int2 *counts, *sums;
  size_t bytes;
};
DistillWs carve(void* ws, long long N, int top) {
  MrlCarver c(ws);
  DistillWs w;
  w.records = c.take<ListRecord>((size_t)N);
  w.factors = c.take<RowFactors>((size_t)N);
  w.z = c.take<float>((size_t)N * top);
  w.term = c.take<double>((size_t)N);
  w.counts = c.take<int2>((size_t)((N + kListRows - 1) / kListRows));
  w.sums = c.take<int2>(kCounts);
  w.bytes = c.off;
  return w;
}

bool row_type_ok(int32_t dtype) { return dtype == MRL_BF16 || dtype == MRL_F32; }
bool on_element(const void* p, int elem) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(elem - 1)) == 0; }
bool temperature_ok(float t) { return t >= 1e-6f && t <= 1e6f; }
float scale_of(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }

}  // namespace

size_t mrl_distill_workspace_bytes(long long N, int top) {
  if (N <= 0 || top > kTop) return 0;
  return carve(nullptr, N, top > 0 ? top : kTop).bytes;
}

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
  const float c = scale_of(temperature);
  const TopArgs a{logits, ld, V, ids, mask, c, 1.0 / ((double)c * (double)temperature), top, logp, lse, entropy, top_logp, top_ids, status};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool bf16 = dtype == MRL_BF16, ent = entropy != nullptr;
  const long long row_bytes = (long long)V * (bf16 ? 2 : 4);
  const int parts = parts_of(N, row_bytes, TopSize<256>::kCtas);
  // More rows than CTAs of 256 threads fit at a time: of fewer threads for shorter rows, so that a row's loads and those of more others are under way during
  // its selection, if half of the threads can be above a floor.  (6,000 rows of 30,000 bf16, top 20: 114 us with 256 threads, 98 with 128; 2,051 of 50,021 float32 88 and
  // 97.  4,756 rows of 2,722 bf16, top 4: 60 with 256, 35 with 64; 2,790 of 6,301 float32 35 with 128.)
  const int threads = N <= TopSize<256>::kCtas * 148 || row_bytes > 128 * 1024 || top > 64 ? 256 : row_bytes > 12 * 1024 || top > 32 ? 128 : 64;
  using Kernel = void (*)(TopArgs);
  const Kernel kernels[3][4] = {
      {top_kernel<float, false, 256>, top_kernel<float, true, 256>, top_kernel<__nv_bfloat16, false, 256>, top_kernel<__nv_bfloat16, true, 256>},
      {top_kernel<float, false, 128>, top_kernel<float, true, 128>, top_kernel<__nv_bfloat16, false, 128>, top_kernel<__nv_bfloat16, true, 128>},
      {top_kernel<float, false, 64>, top_kernel<float, true, 64>, top_kernel<__nv_bfloat16, false, 64>, top_kernel<__nv_bfloat16, true, 64>}};
  mrl_profile_before(st, "top_kernel");
  const int rc = launch_rows(kernels[threads == 256 ? 0 : threads == 128 ? 1 : 2][2 * bf16 + ent], N, parts, threads,
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
  if (workspace == nullptr || workspace_bytes < mrl_distill_workspace_bytes(N, top)) return MRL_ERR_WORKSPACE_TOO_SMALL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MRL_ERR_INVALID_ARG;
  const DistillWs w = carve(workspace, N, top);
  const int blocks = (int)((N + kListRows - 1) / kListRows);
  const bool bf16 = dtype == MRL_BF16;
  DistillArgs a{logits, dlogits, ld, ld_out, N, V, top, top_ids, top_logp, mask, row_weight, *dp, scale_of(dp->temperature), 0.0, row_kl,
                loss, reinterpret_cast<long long*>(stats), status, w.records, w.z, w.factors, w.term, w.counts, blocks, 0, 0};
  a.nat = 1.0 / ((double)a.c * (double)dp->temperature);
  if (bf16)
    list_kernel<__nv_bfloat16><<<blocks, kListThreads, 0, st>>>(a);
  else
    list_kernel<float><<<blocks, kListThreads, 0, st>>>(a);
  MRL_CUDA_OK(cudaGetLastError());
  if (blocks > kCounts) {
    MRL_CUDA_OK(mrl_launch_behind(counts_kernel, 1, 1024, st, w.counts, blocks, (blocks + kCounts - 1) / kCounts, w.sums));
    a.counts = w.sums;
    a.n_counts = kCounts;
  }
  const long long row_bytes = (long long)V * elem;
  const int threads = N > DistillSize<512>::kCtas * 148 && row_bytes <= kShortRow ? 128 : 512;
  // Rows of 512 KB or more are shared by two CTAs, so that the rows in flight still fit L2 between the passes.
  int parts = parts_of(N, row_bytes, DistillSize<512>::kCtas);
  if (parts == 1 && row_bytes >= 512 * 1024) parts = 2;
  const long long off = static_cast<const char*>(dlogits) - static_cast<const char*>(logits);
  const bool shifted = dlogits != nullptr && (off % kVecBytes != 0 || (N > 1 && (ld_out - ld) * elem % kVecBytes != 0));
  a.bit_words = (int)mrl_align_up((size_t)((V + parts - 1) / parts + 16 + 31) / 32, 4);
  const size_t stage = threads == 128 ? DistillSize<128>::kStageBytes : DistillSize<512>::kStageBytes, room = threads == 128 ? DistillSize<128>::kSmem : DistillSize<512>::kSmem;
  const size_t fixed = (size_t)a.bit_words * 4 + (shifted ? stage : 0);
  const int movers = threads - 32;
  if (dlogits != nullptr && fixed < room) a.park_slots = (int)((room - fixed) / (movers * kVecBytes)) * movers;
  const size_t smem = fixed + (size_t)a.park_slots * kVecBytes;
  using Kernel = void (*)(const DistillArgs);
  const Kernel kernels[2][4] = {{distill_kernel<__nv_bfloat16, false, 512>, distill_kernel<__nv_bfloat16, true, 512>, distill_kernel<float, false, 512>,
                                 distill_kernel<float, true, 512>},
                                {distill_kernel<__nv_bfloat16, false, 128>, distill_kernel<__nv_bfloat16, true, 128>, distill_kernel<float, false, 128>,
                                 distill_kernel<float, true, 128>}};
  static std::atomic<uint64_t> attr_done;
  int rc = mrl_once_per_device(attr_done, [&] {
    // the carve-out that an SM's CTAs need, as a percentage of the 228 KB it can give: the rest stays L1
    auto carve_out = [](size_t ctas, size_t bytes) { return (int)((ctas * bytes * 100 + 228 * 1024 - 1) / (228 * 1024)); };
    for (int i = 0; i < 8; ++i) {
      const Kernel k = kernels[i >> 2][i & 3];
      cudaError_t e = i < 4 ? cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) : cudaSuccess;
      if (e == cudaSuccess)
        e = cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout,
                                 i < 4 ? carve_out(DistillSize<512>::kCtas, DistillSize<512>::kSmem + 4096) : carve_out(DistillSize<128>::kCtas, DistillSize<128>::kSmem + 2048));
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  });
  if (rc != MRL_OK) return rc;
  mrl_profile_before(st, "distill_kernel");
  rc = launch_rows(kernels[threads == 128][(bf16 ? 0 : 2) + shifted], N, parts, threads, smem, true, st, a);
  mrl_profile_after(st);
  if (rc != MRL_OK) return rc;
  const unsigned ctas = dlogits != nullptr ? 1 + (unsigned)((N + 31) / 32) : 1;
  MRL_CUDA_OK(mrl_launch_behind(bf16 ? finish_kernel<__nv_bfloat16> : finish_kernel<float>, ctas, 1024, st, a));
  return MRL_OK;
}
