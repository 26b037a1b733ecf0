// The end of an optimisation step over many tensors at once: the gradients' 2-norm with the factor that clips it
// (mrl_grad_norm) and the AdamW update (mrl_adamw_step), App. A.
//
// Both read the tensors' addresses from a table that is passed by value with the launch, so nothing has to be kept on the
// device and a call can be captured.  The tensors are cut into chunks; a CTA finds its chunk's tensor by bisection in
// the table.  A few operations per element against 2 to 28 bytes: bound by HBM.
#include <type_traits>

#include "mrl_common.cuh"

namespace {

using namespace mrl;

constexpr int kThreads = 256;
constexpr int kChunk = 8 * MRL_STATE_BLOCK;   // elements of a CTA at least: a state block per warp
constexpr int kSlotsFew = 16, kSlots = 352;   // tensors per launch: the tables stay below the 32,764 bytes of kernel arguments
constexpr int kSms = 148;
constexpr int kNormCtas = kSms * 8;
constexpr int kAdamwCtas = 4;                 // per SM

struct Slot {
  const void* grad;
  void* param;
  float* master;
  void *m, *v;
  float *m_scale, *v_scale;
  long long numel;
  unsigned long long rng_first;
  float decay;
  uint8_t kind;     // kind_of()
  uint8_t aligned;  // groups of eight elements may be read and written at once
  uint8_t pad[2];
};

// What changes from step to step.
struct Hyper {
  float lr, lr_c1, root_c2;  // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  int skip;
  unsigned long long key;   // of the step's random words
};

template <int kN>
struct Table {
  int n, chunk;            // tensors; elements of a chunk
  uint32_t first[kN + 1];  // first chunk of each tensor, and the number of chunks
  Slot slot[kN];
};
static_assert(sizeof(Table<kSlots>) + 256 <= 32764, "kernel arguments");

// The tensor that holds a chunk: the last one whose first chunk is not behind it.
template <int kN>
__device__ __forceinline__ int slot_of(const Table<kN>& t, uint32_t chunk) {
  int lo = 0, hi = t.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.first[mid] <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ float sqrt_approx(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  double r = 0.0;
  for (int k = 0; k < kThreads / 32; ++k) r += red[k];
  return r;
}

__global__ void __launch_bounds__(kThreads) grad_norm_finish_kernel(const double* __restrict__ partial, int n, float max_norm,
                                                                    float* norm, float* coef) {
  __shared__ double red[kThreads / 32];
  double sum = 0.0;
  for (int k = threadIdx.x; k < n; k += kThreads) sum += partial[k];
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) {
    const double root = sqrt(sum);
    if (norm != nullptr) *norm = (float)root;
    if (coef != nullptr) {
      const float c = max_norm > 0.f ? (float)((double)max_norm / fmax(root, (double)max_norm)) : 1.f;
      *coef = root < INFINITY ? c : NAN;
    }
  }
}

// Reads the step's device-resident inputs (learning rate, step counter), once per call.
__global__ void adamw_prepare_kernel(Hyper h, double lr, double beta1, double beta2, const float* lr_dev, int64_t* step_dev,
                                     int64_t step, unsigned long long seed, const float* grad_scale, Hyper* out) {
  const float gs = grad_scale != nullptr ? *grad_scale : 1.f;
  h.skip = !(fabsf(gs) < INFINITY);
  if (step_dev != nullptr) {
    step = *step_dev + 1;
    if (!h.skip) *step_dev = step;
  }
  if (lr_dev != nullptr) lr = (double)*lr_dev;
  h.lr = (float)lr;
  h.lr_c1 = (float)(lr / (1.0 - pow(beta1, (double)step)));
  h.root_c2 = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
  h.key = splitmix64(splitmix64(seed) + (unsigned long long)step);
  *out = h;
}

struct AdamwArgs {
  Hyper hyper;
  const Hyper* hyper_dev;  // in place of hyper where given
  const float* grad_scale;
  int32_t* status;
  float beta1, one_beta1, beta2, one_beta2, eps;
  bool seeded;
};

// ---- eight adjacent elements of a lane; a warp works on the 256 that share the scales of an 8-bit state

// kN = 8 elements: whole (one or two wide accesses) where `vec`, else one by one below n.
template <typename T>
__device__ __forceinline__ void load8(const void* base, long long i, int n, bool vec, float (&x)[8]) {
  const T* p = static_cast<const T*>(base) + i;
  if (vec) {
    if constexpr (sizeof(T) == 4) {
      uint32_t w[8];
      asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                   : "l"(p));
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(w[j]);
    } else {
      uint32_t w[4];
      asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = bf16lo_to_f32(w[j]);
        x[2 * j + 1] = bf16hi_to_f32(w[j]);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = 0.f;
      if (j < n) {
        if constexpr (sizeof(T) == 4) x[j] = p[j]; else x[j] = __bfloat162float(p[j]);
      }
    }
  }
}
__device__ __forceinline__ void store8(float* base, long long i, int n, bool vec, const float (&x)[8]) {
  float* p = base + i;
  if (vec) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(__float_as_uint(x[0])),
                 "r"(__float_as_uint(x[1])), "r"(__float_as_uint(x[2])), "r"(__float_as_uint(x[3])), "r"(__float_as_uint(x[4])),
                 "r"(__float_as_uint(x[5])), "r"(__float_as_uint(x[6])), "r"(__float_as_uint(x[7]))
                 : "memory");
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = x[j];
  }
}
// words of two bf16 each
__device__ __forceinline__ void store8(__nv_bfloat16* base, long long i, int n, bool vec, const uint32_t (&w)[4]) {
  uint16_t* p = reinterpret_cast<uint16_t*>(base) + i;
  if (vec) {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
  }
}
__device__ __forceinline__ uint2 load_codes(const void* base, long long i, int n, bool vec) {
  const uint8_t* p = static_cast<const uint8_t*>(base) + i;
  if (vec) return *reinterpret_cast<const uint2*>(p);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) w[j >> 2] |= (uint32_t)p[j] << (8 * (j & 3));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_codes(void* base, long long i, int n, bool vec, const uint32_t (&w)[2]) {
  uint8_t* p = static_cast<uint8_t*>(base) + i;
  if (vec) {
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
  }
}
__device__ __forceinline__ void decode(uint2 codes, float scale, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 u = unpack_e4m3x2((uint16_t)((j < 2 ? codes.x : codes.y) >> (16 * (j & 1))));
    x[2 * j] = __fmul_rn(u.x, scale);
    x[2 * j + 1] = __fmul_rn(u.y, scale);
  }
}

// |y| (at most about 448) with the part below an e4m3 step rounded up with probability remainder / step: the 16 bits are
// added below the last kept bit and the rest is cut.  Below 2^-6 the codes are 2^-9 apart, as they are from 2^-6 to 2^-5: the
// value is moved there and back.  y that is not finite comes back as it is.
__device__ __forceinline__ float e4m3_dither(float y, uint32_t bits16) {
  const float a = fabsf(y);
  const bool small = a < 0.015625f;
  const float up = small ? 0.015625f : 0.f;
  const float z = __uint_as_float((__float_as_uint(a + up) + (bits16 << 4)) & 0xfff00000u) - up;
  return a < INFINITY ? copysignf(z, y) : y;
}
// Codes of eight values at most 448 / inv in magnitude.  kFloor: what is above zero stays above zero.
template <bool kFloor>
__device__ __forceinline__ void encode(const float (&x)[8], float inv, bool seeded, const uint32_t (&bits)[8], int shift, uint32_t (&codes)[2]) {
  codes[0] = codes[1] = 0;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    float a = __fmul_rn(x[j], inv), b = __fmul_rn(x[j + 1], inv);
    if (seeded) {
      a = e4m3_dither(a, (bits[j] >> shift) & 0xffffu);
      b = e4m3_dither(b, (bits[j + 1] >> shift) & 0xffffu);
    }
    uint32_t c = pack_e4m3x2(a, b);
    if (kFloor) {
      if ((c & 0xffu) == 0 && x[j] > 0.f) c |= 1u;
      if ((c & 0xff00u) == 0 && x[j + 1] > 0.f) c |= 0x100u;
    }
    codes[j >> 2] |= c << (8 * (j & 3));
  }
}

// Sum of squares of a chunk's elements by this thread: runs of 32 in float32, added up in float64.  A run whose sum is near
// either end of float32's range (or 0) is squared again in float64.
template <typename G>
__device__ __forceinline__ double chunk_squares(const Slot& s, long long lo, long long hi) {
  double sum = 0.0;
  for (long long base = lo; base < hi; base += kChunk * 4) {
    float x[4][8];
    float run = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long i = base + k * kChunk + threadIdx.x * 8;
      const int n = (int)(hi - i < 8 ? (hi > i ? hi - i : 0) : 8);
      load8<G>(s.grad, i, n, s.aligned && n == 8, x[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) run = fmaf(x[k][j], x[k][j], run);
    if (run >= 1e-30f && run <= 1e38f) {
      sum += (double)run;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fma((double)x[k][j], (double)x[k][j], sum);
    }
  }
  return sum;
}

// One partial sum per CTA; a later launch of the same call adds to it.
template <int kN>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ Table<kN> t, double* __restrict__ partial,
                                                             bool first_launch) {
  __shared__ double red[kThreads / 32];
  double sum = 0.0;
  for (uint32_t chunk = blockIdx.x; chunk < t.first[t.n]; chunk += gridDim.x) {
    const int k = slot_of(t, chunk);
    const Slot& s = t.slot[k];
    const long long lo = (long long)(chunk - t.first[k]) * t.chunk, hi = min(lo + t.chunk, s.numel);
    sum += (s.kind & 4) ? chunk_squares<__nv_bfloat16>(s, lo, hi) : chunk_squares<float>(s, lo, hi);
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) partial[blockIdx.x] = first_launch ? sum : partial[blockIdx.x] + sum;
}

// One block of MRL_STATE_BLOCK elements by a warp.  The moments are rounded operation by operation as the formula stands
// (no fused multiply-add) and the 8-bit states take the IEEE root and quotients: the codes, which feed the next step, are
// then the same for every evaluation of the formula in float32, and a value on the border between two codes does not
// depend on how an expression was contracted.
template <bool kParamBf16, bool kMaster, bool kGradBf16, bool kCodes>
__device__ __forceinline__ void adamw_block(const Slot& s, const AdamwArgs& a, const Hyper& hy, float gs, long long base) {
  using G = typename std::conditional<kGradBf16, __nv_bfloat16, float>::type;
  using P = typename std::conditional<kParamBf16, __nv_bfloat16, float>::type;
  const long long i = base + (threadIdx.x & 31) * 8;
  const int n = (int)(s.numel - i < 8 ? (s.numel > i ? s.numel - i : 0) : 8);
  const bool vec = s.aligned && n == 8;
  float g[8], m[8], v[8], p[8];
  load8<G>(s.grad, i, n, vec, g);
  uint2 cm, cv;
  float sm = 0.f, sv = 0.f;
  if constexpr (kCodes) {
    cm = load_codes(s.m, i, n, vec);
    cv = load_codes(s.v, i, n, vec);
    sm = s.m_scale[base / MRL_STATE_BLOCK];
    sv = s.v_scale[base / MRL_STATE_BLOCK];
  } else {
    load8<float>(s.m, i, n, vec, m);
    load8<float>(s.v, i, n, vec, v);
  }
  if constexpr (kMaster)
    load8<float>(s.master, i, n, vec, p);
  else
    load8<P>(s.param, i, n, vec, p);
  if constexpr (kCodes) {
    decode(cm, sm, m);
    decode(cv, sv, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], v[j]);
  }
  float root[8];
  const float decay = hy.lr * s.decay;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float gj = __fmul_rn(g[j], gs);
    m[j] = __fadd_rn(__fmul_rn(a.beta1, m[j]), __fmul_rn(a.one_beta1, gj));
    v[j] = __fadd_rn(__fmul_rn(a.beta2, v[j]), __fmul_rn(a.one_beta2, __fmul_rn(gj, gj)));
    if constexpr (kCodes) root[j] = __fsqrt_rn(v[j]); else root[j] = sqrt_approx(v[j]);
    p[j] -= fmaf(decay, p[j], __fdividef(hy.lr_c1 * m[j], fmaf(root[j], hy.root_c2, a.eps)));
  }
  uint32_t bits[8];  // of each element: 16 for m, 16 for v above them
  if (a.seeded && (kCodes || (kParamBf16 && !kMaster))) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned long long w = splitmix64(hy.key + s.rng_first + (unsigned long long)(i / 2 + j));
      bits[2 * j] = (uint32_t)w;
      bits[2 * j + 1] = (uint32_t)(w >> 32);
    }
  }
  if constexpr (kMaster) store8(s.master, i, n, vec, p);
  if constexpr (kParamBf16) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = pack_bf16x2(p[2 * j], p[2 * j + 1]);
      if (!kMaster && a.seeded) {  // the 16 bits that are cut decide against m's in reverse order
        const uint32_t lo = __float_as_uint(p[2 * j]) + (__brev(bits[2 * j]) >> 16);
        const uint32_t hi = __float_as_uint(p[2 * j + 1]) + (__brev(bits[2 * j + 1]) >> 16);
        if (fabsf(p[2 * j]) < INFINITY && fabsf(p[2 * j + 1]) < INFINITY) {
          w[j] = __byte_perm(lo, hi, 0x7632);
        } else {  // not finite: as it is
          if (fabsf(p[2 * j]) < INFINITY) w[j] = (w[j] & 0xffff0000u) | lo >> 16;
          if (fabsf(p[2 * j + 1]) < INFINITY) w[j] = (w[j] & 0xffffu) | (hi & 0xffff0000u);
        }
      }
    }
    store8(static_cast<__nv_bfloat16*>(s.param), i, n, vec, w);
  } else {
    store8(static_cast<float*>(s.param), i, n, vec, p);
  }
  if constexpr (kCodes) {
    uint32_t am = 0, av = 0;  // magnitudes as ordered integers
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      am = max(am, __float_as_uint(m[j]) & 0x7fffffffu);
      av = max(av, __float_as_uint(root[j]) & 0x7fffffffu);
    }
    sm = e4m3_scale(__uint_as_float(__reduce_max_sync(0xffffffffu, am)));
    sv = e4m3_scale(__uint_as_float(__reduce_max_sync(0xffffffffu, av)));
    if ((threadIdx.x & 31) == 0) {
      s.m_scale[base / MRL_STATE_BLOCK] = sm;
      s.v_scale[base / MRL_STATE_BLOCK] = sv;
    }
    uint32_t codes[2];
    encode<false>(m, __frcp_rn(sm), a.seeded, bits, 0, codes);
    store_codes(s.m, i, n, vec, codes);
    encode<true>(root, __frcp_rn(sv), a.seeded, bits, 16, codes);
    store_codes(s.v, i, n, vec, codes);
  } else {
    store8(static_cast<float*>(s.m), i, n, vec, m);
    store8(static_cast<float*>(s.v), i, n, vec, v);
  }
}

// The tensors of one kind (types of gradient, parameter and states), which share the launch and its registers.
template <int kKind, int kN>
__global__ void __launch_bounds__(kThreads, kAdamwCtas) adamw_kernel(const __grid_constant__ Table<kN> t, const __grid_constant__ AdamwArgs a) {
  const float gs = a.grad_scale != nullptr ? *a.grad_scale : 1.f;
  if (!(fabsf(gs) < INFINITY)) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.status != nullptr) atomicOr(a.status, MRL_DEV_NONFINITE_GRAD);
    return;
  }
  const Hyper hy = a.hyper_dev != nullptr ? *a.hyper_dev : a.hyper;
  const int k = slot_of(t, blockIdx.x);
  const Slot& s = t.slot[k];
  const long long lo = (long long)(blockIdx.x - t.first[k]) * t.chunk, hi = min(lo + t.chunk, s.numel);
  for (long long base = lo + (threadIdx.x >> 5) * MRL_STATE_BLOCK; base < hi; base += kThreads / 32 * MRL_STATE_BLOCK)
    adamw_block<(kKind & 1) != 0, (kKind & 2) != 0, (kKind & 4) != 0, (kKind & 8) != 0>(s, a, hy, gs, base);
}

bool grad_type_ok(int32_t dtype) { return dtype == MRL_BF16 || dtype == MRL_F32; }

bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Groups of eight elements: 32 bytes of float32, 16 of bf16, 8 of codes.
bool grad_aligned(const mrl_tensor_slot& s) { return aligned_to(s.grad, s.grad_dtype == MRL_BF16 ? 16 : 32); }
bool all_aligned(const mrl_tensor_slot& s) {
  const uintptr_t state = s.state_dtype == MRL_E4M3 ? 8 : 32;
  return grad_aligned(s) && aligned_to(s.param, s.param_dtype == MRL_BF16 ? 16 : 32) && aligned_to(s.master, 32) &&
         aligned_to(s.m, state) && aligned_to(s.v, state);
}

// 1: bf16 parameter, 2: master weights, 4: bf16 gradient, 8: 8-bit states
int kind_of(const mrl_tensor_slot& s) {
  return (s.param_dtype == MRL_BF16 ? 1 : 0) | (s.master != nullptr ? 2 : 0) | (s.grad_dtype == MRL_BF16 ? 4 : 0) |
         (s.state_dtype == MRL_E4M3 ? 8 : 0);
}

// Fills the table with tensors from slots[at] on, as many as it holds, and returns the index of the first one left out.
// only: those of one kind, for the update; -1: all, for their gradients.
template <int kN>
int fill_table(const mrl_tensor_slot* slots, int n, int at, int chunk, int only, Table<kN>* t) {
  uint32_t chunks = 0;
  t->n = 0;
  t->chunk = chunk;
  for (; at < n && t->n < kN; ++at) {
    const mrl_tensor_slot& s = slots[at];
    if (s.numel == 0 || (only >= 0 && kind_of(s) != only)) continue;
    const long long need = (s.numel + chunk - 1) / chunk;
    if (chunks + need > 0x7fffffffll) break;
    t->slot[t->n] = Slot{s.grad, s.param, s.master, s.m, s.v, s.m_scale, s.v_scale, s.numel, s.rng_first, s.weight_decay,
                         (uint8_t)kind_of(s), (uint8_t)(only < 0 ? grad_aligned(s) : all_aligned(s)), {0, 0}};
    t->first[t->n++] = chunks;
    chunks += (uint32_t)need;
  }
  t->first[t->n] = chunks;
  return at;
}

// Elements of a chunk: small ones while there are few, for the sake of parallel CTAs.
int chunk_of(const mrl_tensor_slot* slots, int n) {
  long long total = 0;
  for (int k = 0; k < n; ++k) total += slots[k].numel;
  return total <= (long long)kSms * 8 * 4 * kChunk ? kChunk : 4 * kChunk;
}

template <int kN>
int launch_grad_norm(const mrl_tensor_slot* slots, int n, double* partial, int* ctas, cudaStream_t st) {
  Table<kN> t;
  const int chunk = chunk_of(slots, n);
  for (int at = 0; at < n;) {
    at = fill_table(slots, n, at, chunk, -1, &t);
    if (t.n == 0) break;
    // (the first launch decides how many partials there are)
    const bool first = *ctas == 0;
    if (first) *ctas = at < n || t.first[t.n] > (uint32_t)kNormCtas ? kNormCtas : (int)t.first[t.n];
    mrl_profile_before(st, "grad_norm_kernel");
    grad_norm_kernel<kN><<<*ctas, kThreads, 0, st>>>(t, partial, first);
    mrl_profile_after(st);
    MRL_CUDA_OK(cudaGetLastError());
  }
  return MRL_OK;
}

template <int kKind, int kN>
int launch_adamw_kind(const mrl_tensor_slot* slots, int n, int chunk, const AdamwArgs& a, cudaStream_t st) {
  Table<kN> t;
  for (int at = 0; at < n;) {
    at = fill_table(slots, n, at, chunk, kKind, &t);
    if (t.n == 0) break;
    mrl_profile_before(st, "adamw_kernel");
    adamw_kernel<kKind, kN><<<t.first[t.n], kThreads, 0, st>>>(t, a);
    mrl_profile_after(st);
    MRL_CUDA_OK(cudaGetLastError());
  }
  return MRL_OK;
}
template <int kKind>
int launch_adamw(const mrl_tensor_slot* slots, int n, int count, int chunk, const AdamwArgs& a, cudaStream_t st) {
  if (count == 0) return MRL_OK;
  return count <= kSlotsFew ? launch_adamw_kind<kKind, kSlotsFew>(slots, n, chunk, a, st)
                            : launch_adamw_kind<kKind, kSlots>(slots, n, chunk, a, st);
}

constexpr long long kMaxNumel = 0x7fffffffll * kChunk;

}  // namespace

size_t mrl_grad_norm_workspace_bytes() { return mrl_align_up(kNormCtas * sizeof(double), 256); }
size_t mrl_adamw_workspace_bytes() { return 256; }

extern "C" int mrl_grad_norm(const mrl_tensor_slot* slots, int32_t n_slots, float max_norm, float* norm, float* coef,
                             void* workspace, size_t workspace_bytes, void* stream) {
  if (n_slots < 0 || (n_slots > 0 && slots == nullptr) || max_norm != max_norm || (norm == nullptr && coef == nullptr))
    return MRL_ERR_INVALID_ARG;
  for (int k = 0; k < n_slots; ++k) {
    if (!grad_type_ok(slots[k].grad_dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
    if (slots[k].numel < 0 || slots[k].numel > kMaxNumel || (slots[k].numel > 0 && slots[k].grad == nullptr))
      return MRL_ERR_INVALID_ARG;
  }
  if (workspace == nullptr || workspace_bytes < mrl_grad_norm_workspace_bytes()) return MRL_ERR_WORKSPACE_TOO_SMALL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MRL_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  double* partial = static_cast<double*>(workspace);
  int grid = 0;
  const int rc = n_slots <= kSlotsFew ? launch_grad_norm<kSlotsFew>(slots, n_slots, partial, &grid, st)
                                      : launch_grad_norm<kSlots>(slots, n_slots, partial, &grid, st);
  if (rc != MRL_OK) return rc;
  grad_norm_finish_kernel<<<1, kThreads, 0, st>>>(partial, grid, max_norm, norm, coef);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
}

extern "C" int mrl_adamw_step(const mrl_tensor_slot* slots, int32_t n_slots, const mrl_adamw_params* ap,
                              const float* grad_scale, int32_t* status, void* workspace, size_t workspace_bytes,
                              void* stream) {
  if (ap == nullptr || n_slots < 0 || (n_slots > 0 && slots == nullptr)) return MRL_ERR_INVALID_ARG;
  if (!(ap->beta1 >= 0.0 && ap->beta1 < 1.0) || !(ap->beta2 >= 0.0 && ap->beta2 < 1.0) || !(ap->eps > 0.0) ||
      (float)ap->eps == 0.f || !(ap->eps < 3.4e38) || !(ap->lr - ap->lr == 0.0) || ap->flags != 0 ||
      (ap->step_dev == nullptr && ap->step < 1) || (ap->rounding != MRL_ROUND_NEAREST && ap->rounding != MRL_ROUND_SEEDED))
    return MRL_ERR_INVALID_ARG;
  for (int k = 0; k < n_slots; ++k) {
    const mrl_tensor_slot& s = slots[k];
    if (!grad_type_ok(s.grad_dtype) || !grad_type_ok(s.param_dtype) || (s.state_dtype != MRL_F32 && s.state_dtype != MRL_E4M3))
      return MRL_ERR_UNSUPPORTED_DTYPE;
    if (s.numel < 0 || s.numel > kMaxNumel || !(s.weight_decay - s.weight_decay == 0.f)) return MRL_ERR_INVALID_ARG;
    if (s.numel == 0) continue;
    if (s.grad == nullptr || s.param == nullptr || s.m == nullptr || s.v == nullptr) return MRL_ERR_INVALID_ARG;
    if (s.master != nullptr && s.param_dtype != MRL_BF16) return MRL_ERR_INVALID_ARG;
    if (s.state_dtype == MRL_E4M3 && (s.m_scale == nullptr || s.v_scale == nullptr)) return MRL_ERR_INVALID_ARG;
  }
  const bool on_device = ap->lr_dev != nullptr || ap->step_dev != nullptr;
  if (on_device) {
    if (workspace == nullptr || workspace_bytes < mrl_adamw_workspace_bytes()) return MRL_ERR_WORKSPACE_TOO_SMALL;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MRL_ERR_INVALID_ARG;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  AdamwArgs a{};
  a.hyper_dev = on_device ? static_cast<const Hyper*>(workspace) : nullptr;
  a.grad_scale = grad_scale;
  a.status = status;
  a.beta1 = (float)ap->beta1;
  a.one_beta1 = (float)(1.0 - ap->beta1);
  a.beta2 = (float)ap->beta2;
  a.one_beta2 = (float)(1.0 - ap->beta2);
  a.eps = (float)ap->eps;
  a.seeded = ap->rounding == MRL_ROUND_SEEDED;
  if (on_device) {
    adamw_prepare_kernel<<<1, 1, 0, st>>>(Hyper{}, ap->lr, ap->beta1, ap->beta2, ap->lr_dev, ap->step_dev, ap->step, ap->seed,
                                          grad_scale, static_cast<Hyper*>(workspace));
    MRL_CUDA_OK(cudaGetLastError());
  } else {
    a.hyper.lr = (float)ap->lr;
    a.hyper.lr_c1 = (float)(ap->lr / (1.0 - pow(ap->beta1, (double)ap->step)));
    a.hyper.root_c2 = (float)(1.0 / sqrt(1.0 - pow(ap->beta2, (double)ap->step)));
    a.hyper.key = splitmix64(splitmix64(ap->seed) + (uint64_t)ap->step);
  }
  int count[16] = {0};
  for (int k = 0; k < n_slots; ++k) count[kind_of(slots[k])] += slots[k].numel > 0;
  const int chunk = chunk_of(slots, n_slots);
  int rc = MRL_OK;
  const auto run = [&](auto kind) {
    constexpr int kKind = decltype(kind)::value;
    if (rc == MRL_OK) rc = launch_adamw<kKind>(slots, n_slots, count[kKind], chunk, a, st);
  };
  run(std::integral_constant<int, 0>{}), run(std::integral_constant<int, 1>{}), run(std::integral_constant<int, 3>{});
  run(std::integral_constant<int, 4>{}), run(std::integral_constant<int, 5>{}), run(std::integral_constant<int, 7>{});
  run(std::integral_constant<int, 8>{}), run(std::integral_constant<int, 9>{}), run(std::integral_constant<int, 11>{});
  run(std::integral_constant<int, 12>{}), run(std::integral_constant<int, 13>{}), run(std::integral_constant<int, 15>{});
  return rc;
}
