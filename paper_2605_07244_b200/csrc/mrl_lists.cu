// Top tokens and learning from them: mrl_top_logprobs and mrl_distill_loss_fwd_bwd.
//
// Both read rows of logits against a running (zm, s): zm the largest logit, s = sum_v 2^((z_v - zm) c) with c = log2(e) / T.  The
// difference is taken before the product, so that rows of the type's lowest value keep their softmax; zm starts at the lowest
// float, not at -inf, so that -inf - zm stays -inf and a NaN always reaches the sum.  s = 0: nothing but -inf.
#include <float.h>

#include "mrl_common.cuh"

namespace {

using namespace mrl;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kTop = MRL_MAX_TOP;

template <typename T>
__device__ __forceinline__ float load_f(const T* p);
template <>
__device__ __forceinline__ float load_f<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_f<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_f(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

struct Sums {
  float zm, s, u;  // u = sum_v 2^(t_v) t_v, t_v = (z_v - zm) c
};
__device__ __forceinline__ Sums sums_empty() { return Sums{-FLT_MAX, 0.f, 0.f}; }
// s and u over a higher maximum: u' = sum 2^(t + d) (t + d) with d = (zm - zm') c
__device__ __forceinline__ Sums sums_raise(Sums a, float zm, float c) {
  if (zm == a.zm) return a;
  const float d = fmaxf((a.zm - zm) * c, -1000.f);  // 2^-1000 = 0, and no 0 * inf
  const float f = ex2_approx((a.zm - zm) * c);      // (NaN for two infinities)
  return Sums{zm, a.s * f, fmaf(a.s, d, a.u) * f};
}
__device__ __forceinline__ Sums sums_merge(Sums a, Sums b, float c) {
  const float zm = fmaxf(a.zm, b.zm);
  a = sums_raise(a, zm, c);
  b = sums_raise(b, zm, c);
  return Sums{zm, a.s + b.s, a.u + b.u};
}
__device__ __forceinline__ void sums_add(Sums& a, float z, float c) {
  if (z > a.zm) a = sums_raise(a, z, c);
  const float t = (z - a.zm) * c, e = ex2_approx(t);
  a.s += e;
  a.u = fmaf(e, fmaxf(t, -1000.f), a.u);
}
// over the block, in a fixed order; every thread gets the result
__device__ __forceinline__ Sums block_sums(Sums a, float c, Sums* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Sums b;
    b.zm = __shfl_xor_sync(0xffffffffu, a.zm, o);
    b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
    b.u = __shfl_xor_sync(0xffffffffu, a.u, o);
    a = (threadIdx.x & o) ? sums_merge(b, a, c) : sums_merge(a, b, c);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = a;
  __syncthreads();
  a = red[0];
  for (int k = 1; k < (int)(blockDim.x >> 5); ++k) a = sums_merge(a, red[k], c);
  return a;
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

// The largest digit d (of 256) such that at least `want` counts lie at or above it; `want` becomes what is wanted of d itself.
// Called by all threads; counts in shared memory.
__device__ __forceinline__ int pick_digit(const uint32_t* hist, uint32_t& want, uint32_t* out) {
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t above = 0;
    int d = 255;
    for (; d > 0 && above + hist[d] < want; --d) above += hist[d];
    out[0] = (uint32_t)d;
    out[1] = want - above;
  }
  __syncthreads();
  want = out[1];
  return (int)out[0];
}

// The `top` likeliest tokens of a row by 256-way counting: four passes find the value of the last of them, up to four more the index up
// to which tokens of that value are listed, one collects.  Right for every row; the row is read nine times.  Returns their number.
template <typename T>
__device__ int select_top(const T* z, int V, int top, uint32_t* hist, uint32_t* pick, unsigned long long* keys) {
  uint32_t value = 0, want = (uint32_t)top;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += blockDim.x) hist[i] = 0;
    __syncthreads();
    for (int v = threadIdx.x; v < V; v += blockDim.x) {
      const uint32_t o = ordinal(load_f<T>(z + v));
      if (o != 0 && (shift == 24 || (o >> (shift + 8)) == (value >> (shift + 8)))) atomicAdd(&hist[(o >> shift) & 255u], 1u);
    }
    if (shift == 24) {  // (fewer numbers than places: all of them)
      __syncthreads();
      if (threadIdx.x == 0) {
        uint32_t n = 0;
        for (int i = 0; i < 256; ++i) n += hist[i];
        pick[2] = n;
      }
      __syncthreads();
      want = min(want, pick[2]);
      if (want == 0) return 0;
    }
    value |= (uint32_t)pick_digit(hist, want, pick) << shift;
  }
  const int listed = (int)min((uint32_t)top, pick[2]);
  // of the tokens of this value the first `want`: the largest bound that keeps that many of the reversed indices
  uint32_t rev = 0;  // 2^31 - 1 - index
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += blockDim.x) hist[i] = 0;
    __syncthreads();
    for (int v = threadIdx.x; v < V; v += blockDim.x) {
      const uint32_t r = 0x7fffffffu - (uint32_t)v;
      if (ordinal(load_f<T>(z + v)) == value && (shift == 24 || (r >> (shift + 8)) == (rev >> (shift + 8))))
        atomicAdd(&hist[(r >> shift) & 255u], 1u);
    }
    rev |= (uint32_t)pick_digit(hist, want, pick) << shift;
  }
  const unsigned long long last = ((unsigned long long)value << 32) | rev;
  if (threadIdx.x == 0) pick[3] = 0;
  __syncthreads();
  for (int v = threadIdx.x; v < V; v += blockDim.x) {
    const unsigned long long key = ((unsigned long long)ordinal(load_f<T>(z + v)) << 32) | (0x7fffffffu - (uint32_t)v);
    if (key >= last) keys[min(atomicAdd(&pick[3], 1u), (uint32_t)(kTop - 1))] = key;
  }
  __syncthreads();
  return listed;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) top_kernel(const TopArgs p) {
  __shared__ Sums red[kWarps];
  __shared__ uint32_t hist[256], pick[4];
  __shared__ unsigned long long keys[kTop];
  const long long row = blockIdx.x;
  const T* z = static_cast<const T*>(p.logits) + row * p.ld;
  const int id = p.ids != nullptr ? p.ids[row] : 0;
  const bool on = p.mask == nullptr || p.mask[row] != 0, good = id >= 0 && id < p.V;
  if (!on || !good) {
    if (threadIdx.x == 0) {
      if (on && p.status != nullptr) atomicOr(p.status, MRL_DEV_BAD_TOKEN_ID);
      if (p.logp != nullptr) p.logp[row] = 0.f;
      if (p.lse != nullptr) p.lse[row] = 0.f;
      if (p.entropy != nullptr) p.entropy[row] = 0.f;
    }
    for (int k = threadIdx.x; k < p.top; k += kThreads) {
      p.top_ids[row * p.top + k] = -1;
      p.top_logp[row * p.top + k] = 0.f;
    }
    return;
  }
  Sums a = sums_empty();
  for (int v = threadIdx.x; v < p.V; v += kThreads) sums_add(a, load_f<T>(z + v), p.c);
  a = block_sums(a, p.c, red);
  const float ln_s = a.s == 0.f ? NAN : logf(a.s);
  if (threadIdx.x == 0) {
    if (p.lse != nullptr) p.lse[row] = a.zm / p.temperature + ln_s;
    if (p.logp != nullptr) p.logp[row] = (load_f<T>(z + id) - a.zm) / p.temperature - ln_s;
    if (p.entropy != nullptr) p.entropy[row] = ln_s - a.u / a.s * MRL_NAT_HI;
  }
  if (p.top == 0) return;
  const int n = select_top<T>(z, p.V, p.top, hist, pick, keys);
  for (int k = threadIdx.x; k < p.top; k += kThreads) {
    if (k < n) {  // its place is the number of larger keys
      const unsigned long long key = keys[k];
      int at = 0;
      for (int j = 0; j < n; ++j) at += keys[j] > key;
      p.top_ids[row * p.top + at] = (int32_t)(0x7fffffffu - (uint32_t)key);
      p.top_logp[row * p.top + at] = (from_ordinal((uint32_t)(key >> 32)) - a.zm) / p.temperature - ln_s;
    } else {
      p.top_ids[row * p.top + k] = -1;
      p.top_logp[row * p.top + k] = -INFINITY;
    }
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
  int n_counts;
  double* term;         // [N] weight_t KL_t
};

// A warp per row: is its list one to learn from?  The entries stay in registers, four a lane; a token twice shows when every entry
// is compared with those of the other places, carried round the warp.
__global__ void __launch_bounds__(kListThreads) list_check_kernel(const DistillArgs p) {
  __shared__ int2 part[kListThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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

// Valid rows of the call, for the denominator: the counts of all CTAs of the check, summed by a block (or one count, summed before).
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

constexpr double kNoRest = -700.0;  // ln p_r below which the learner gives the rest nothing: masks, of -inf or of the type's lowest value

struct RowResult {
  double kl, at;    // KL_t; T dKL/dz of this thread's listed token
  double of_rest;   // T dKL/dz_v = of_rest * softmax over the rest (v)
};

// A row's KL and gradient factors from its list (thread k holds place k) and the sums over the rest, in float64.  Called by the block.
__device__ RowResult distill_row(bool used, float z, float l, Sums rest, const mrl_distill_params& dp, double* red) {
  const double T = dp.temperature;
  float zs = used ? fmaxf(z, -FLT_MAX) : -FLT_MAX;
  if (used && z != z) zs = INFINITY;  // (NaN: inf - inf below)
  __shared__ float zred[32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) zs = fmaxf(zs, __shfl_xor_sync(0xffffffffu, zs, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) zred[threadIdx.x >> 5] = zs;
  __syncthreads();
  const bool any_rest = rest.s != 0.f;
  float m = any_rest ? rest.zm : -FLT_MAX;
  for (int k = 0; k < (int)(blockDim.x >> 5); ++k) m = fmaxf(m, zred[k]);
  const double x = used ? ((double)z - (double)m) / T : 0.0;
  const double in_rest = any_rest ? (double)rest.s * exp(((double)rest.zm - (double)m) / T) : 0.0;
  const double total = block_sum(used ? exp(x) : 0.0, red) + in_rest;
  const double ln_total = total > 0.0 ? log(total) : NAN;
  const double ln_p = x - ln_total, p = used ? exp(ln_p) : 0.0;
  const double ln_p_rest = any_rest ? log((double)rest.s) + ((double)rest.zm - (double)m) / T - ln_total : -INFINITY;
  const bool has_rest = !(ln_p_rest < kNoRest);
  const double p_rest = has_rest ? exp(ln_p_rest) : 0.0;
  RowResult r;
  if (dp.rest == MRL_REST_EVENT) {
    const double q = used ? exp((double)l) : 0.0, mass = block_sum(q, red);
    const double q_rest = has_rest ? fmax(1.0 - mass, (double)dp.rest_floor) : 0.0;
    if (dp.direction == MRL_DISTILL_FORWARD) {
      r.kl = block_sum(q > 0.0 ? q * ((double)l - ln_p) : 0.0, red) + (q_rest > 0.0 ? q_rest * (log(q_rest) - ln_p_rest) : 0.0);
      r.at = (mass + q_rest) * p - q;
      r.of_rest = has_rest ? (mass + q_rest) * p_rest - q_rest : 0.0;
    } else {
      const double ratio = ln_p - (double)l, ratio_rest = has_rest ? ln_p_rest - log(q_rest) : 0.0;
      r.kl = block_sum(used && p != 0.0 ? p * ratio : 0.0, red) + (p_rest != 0.0 ? p_rest * ratio_rest : 0.0);
      r.at = p != 0.0 ? p * (ratio - r.kl) : 0.0;
      r.of_rest = p_rest != 0.0 ? p_rest * (ratio_rest - r.kl) : 0.0;
    }
  } else {
    __syncthreads();
    float lm = used ? l : -FLT_MAX;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) lm = fmaxf(lm, __shfl_xor_sync(0xffffffffu, lm, o));
    if ((threadIdx.x & 31) == 0) zred[threadIdx.x >> 5] = lm;
    __syncthreads();
    for (int k = 0; k < (int)(blockDim.x >> 5); ++k) lm = fmaxf(lm, zred[k]);
    const double d = (double)l - (double)lm, mass = block_sum(used ? exp(d) : 0.0, red);
    const double ln_q = d - log(mass), q = used ? exp(ln_q) : 0.0;
    r.kl = block_sum(q > 0.0 ? q * (ln_q - ln_p) : 0.0, red);
    r.at = p - q;
    r.of_rest = p_rest;
  }
  return r;
}

// One CTA per row; a bit for each listed token in shared memory.
template <typename T>
__global__ void __launch_bounds__(kThreads) distill_kernel(const DistillArgs p) {
  extern __shared__ uint32_t listed[];
  __shared__ Sums red[kWarps];
  __shared__ double red64[kWarps];
  __shared__ int2 redc[kWarps];
  const long long row = blockIdx.x;
  const T* z = static_cast<const T*>(p.logits) + row * p.ld;
  T* dz = p.dlogits != nullptr ? static_cast<T*>(p.dlogits) + row * p.ld_out : nullptr;
  const int valid = p.dp.denominator > 0.0 ? 1 : sum_counts(p.counts, p.n_counts, redc).x;
  if (p.rowstat[row] != kRowValid) {
    if (dz != nullptr)
      for (int v = threadIdx.x; v < p.V; v += kThreads) store_f(dz + v, 0.f);
    if (threadIdx.x == 0) {
      p.term[row] = 0.0;
      if (p.row_kl != nullptr) p.row_kl[row] = 0.f;
    }
    return;
  }
  for (int i = threadIdx.x; i < (p.V + 31) / 32; i += kThreads) listed[i] = 0;
  __syncthreads();
  const int k = threadIdx.x;
  int id = k < p.top ? p.top_ids[row * p.top + k] : -1;
  const float l = id >= 0 ? p.top_logp[row * p.top + k] : -INFINITY;
  if (l == -INFINITY) id = -1;
  const float mine = id >= 0 ? load_f<T>(z + id) : 0.f;
  if (id >= 0) atomicOr(&listed[id >> 5], 1u << (id & 31));
  __syncthreads();
  Sums rest = sums_empty();
  for (int v = threadIdx.x; v < p.V; v += kThreads)
    if (!((listed[v >> 5] >> (v & 31)) & 1u)) sums_add(rest, load_f<T>(z + v), p.c);
  rest = block_sums(rest, p.c, red);
  const RowResult r = distill_row(id >= 0, mine, l, rest, p.dp, red64);
  const float w = p.weight != nullptr ? p.weight[row] : 1.f;
  if (threadIdx.x == 0) {
    p.term[row] = w != 0.f ? (double)w * r.kl : 0.0;
    if (p.row_kl != nullptr) p.row_kl[row] = (float)r.kl;
  }
  if (dz == nullptr) return;
  const double denominator = p.dp.denominator > 0.0 ? p.dp.denominator : (double)valid;
  const double scale = (double)p.dp.coeff * w / (denominator * p.dp.temperature);
  const float of_rest = scale != 0.0 && rest.s != 0.f ? (float)(r.of_rest * scale / rest.s) : 0.f;
  for (int v = threadIdx.x; v < p.V; v += kThreads)
    if (!((listed[v >> 5] >> (v & 31)) & 1u))
      store_f(dz + v, scale != 0.0 ? ex2_approx((load_f<T>(z + v) - rest.zm) * p.c) * of_rest : 0.f);
  if (id >= 0) store_f(dz + id, scale != 0.0 ? (float)(r.at * scale) : 0.f);
}

// Sums of the rows' terms and counts, one CTA, in a fixed order.
__global__ void __launch_bounds__(1024) distill_finish_kernel(const DistillArgs p) {
  __shared__ double red[32];
  __shared__ int2 redc[32];
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
  int2* counts;
  double* term;
  size_t bytes;
};
DistillWs carve(void* ws, long long N) {
  MrlCarver c(ws);
  DistillWs w;
  w.term = c.take<double>((size_t)N);
  w.counts = c.take<int2>((size_t)((N + kListRows - 1) / kListRows));
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
  if (top > kTop || N > 0x7fffffffll) return MRL_ERR_UNSUPPORTED_SHAPE;
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
  mrl_profile_before(st, "top_kernel");
  if (dtype == MRL_BF16)
    top_kernel<__nv_bfloat16><<<(unsigned)N, kThreads, 0, st>>>(a);
  else
    top_kernel<float><<<(unsigned)N, kThreads, 0, st>>>(a);
  mrl_profile_after(st);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
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
                loss, reinterpret_cast<long long*>(stats), status, w.rowstat, w.counts, blocks, w.term};
  list_check_kernel<<<blocks, kListThreads, 0, st>>>(a);
  MRL_CUDA_OK(cudaGetLastError());
  const size_t smem = (size_t)(V + 31) / 32 * 4;
  static std::atomic<uint64_t> attr_done;
  const int rc = mrl_once_per_device(attr_done, [] {
    const cudaError_t e = cudaFuncSetAttribute(distill_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, 1 << 17);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(distill_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, 1 << 17);
  });
  if (rc != MRL_OK) return rc;
  mrl_profile_before(st, "distill_kernel");
  if (dtype == MRL_BF16)
    distill_kernel<__nv_bfloat16><<<(unsigned)N, kThreads, smem, st>>>(a);
  else
    distill_kernel<float><<<(unsigned)N, kThreads, smem, st>>>(a);
  mrl_profile_after(st);
  MRL_CUDA_OK(cudaGetLastError());
  distill_finish_kernel<<<1, 1024, 0, st>>>(a);
  MRL_CUDA_OK(cudaGetLastError());
  return MRL_OK;
}
