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
constexpr int kSlotsFew = 16, kSlots = 160;   // tensors per launch: the tables stay below the 32,764 bytes of kernel arguments
constexpr int kSms = 148;
constexpr int kNormCtas = kSms * 5;           // as many as are resident (48 registers)
constexpr uint32_t kSmallChunks = 16;
constexpr int kCluster = 8;                   // CTAs of the gradient norm of few elements
// The update's threads and CTAs per SM (8: the kind's bit for 8-bit states), and the blocks of a warp in a large call.
// 8-bit states, 525 M elements, compared before the arithmetic's last steps (1,194 us with them): 24 warps of 80 registers in 6
// CTAs 1,231 us, in 3 CTAs 1,343; 28 of 72 registers 1,279, 32 of 64 slower still; 8, 16, 32 and 128 blocks a warp 1,252, 1,249, 1,255
// and 1,276.  That is the kind with bf16 weights and gradients and no master weights, which has no spills; the other 8-bit kinds spill
// 40 to 64 bytes at 80 registers and were not compared.  float32 states, 622 M: 4 blocks 2,583, 8 2,624.
__host__ __device__ constexpr int step_threads(int kind) { return kind & 8 ? 128 : 256; }
__host__ __device__ constexpr int step_ctas(int kind) { return kind & 8 ? 6 : 4; }
__host__ __device__ constexpr int step_blocks(int kind) { return kind & 8 ? 16 : 4; }

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
  float lr, lr_c1, root_c2;  // lr, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
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

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// a + b of two products: a packed sum of packed products is compiled to a fused multiply-add, a single one is not.
__device__ __forceinline__ f2 add_apart(f2 a, f2 b) {
  const float2 u = split_f2(a), v = split_f2(b);
  return make_f2(__fadd_rn(u.x, v.x), __fadd_rn(u.y, v.y));
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

__device__ __forceinline__ void write_norm(double sum, float max_norm, float* norm, float* coef) {
  const double root = sqrt(sum);
  if (norm != nullptr) *norm = (float)root;
  if (coef != nullptr) {
    const float c = max_norm > 0.f && max_norm < INFINITY ? (float)((double)max_norm / fmax(root, (double)max_norm)) : 1.f;
    *coef = root < INFINITY ? c : NAN;
  }
}

__global__ void __launch_bounds__(kThreads) grad_norm_finish_kernel(const double* partial, int n, float max_norm, float* norm, float* coef) {
  __shared__ double red[kThreads / 32];
  wait_for_previous();
  double sum = 0.0;
  for (int k = threadIdx.x; k < n; k += kThreads) sum += partial[k];
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) write_norm(sum, max_norm, norm, coef);
}

// Reads the step's device-resident inputs (learning rate, step counter), once per call; out is null where there are none and the
// call has no elements whose kernels would set the status.
__global__ void adamw_prepare_kernel(Hyper h, double lr, double beta1, double beta2, const float* lr_dev, int64_t* step_dev,
                                     int64_t step, unsigned long long seed, const float* grad_scale, int32_t* status, Hyper* out) {
  const float gs = grad_scale != nullptr ? *grad_scale : 1.f;
  if (!(fabsf(gs) < INFINITY) && status != nullptr) atomicOr(status, MRL_DEV_NONFINITE_GRAD);
  if (out == nullptr) return;
  if (step_dev != nullptr) {
    step = *step_dev + 1;
    if (fabsf(gs) < INFINITY) *step_dev = step;  // (the step is skipped otherwise)
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

// ---- eight adjacent elements of a lane, as four pairs; a warp works on the 256 that share the scales of an 8-bit state

// As they lie in memory: eight words of float32, four of two bf16.  Whole (one wide access) where `vec`, else one by one below n
// and 0 from there.
template <typename T>
struct Raw8 {
  static constexpr int kWords = (int)sizeof(T) * 2;
  uint32_t w[kWords];

  __device__ __forceinline__ void load(const void* at, int n, bool vec) {
    const T* p = static_cast<const T*>(at);
    if (vec) {
      if constexpr (sizeof(T) == 4)
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                     : "l"(p));
      else
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    } else {
#pragma unroll
      for (int k = 0; k < kWords; ++k) w[k] = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) {
          if constexpr (sizeof(T) == 4) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
          else w[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
        }
    }
  }
  __device__ __forceinline__ f2 pair(int j) const {
    if constexpr (sizeof(T) == 4)
      return make_f2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
    else
      return bf16x2_to_f2(w[j]);
  }
};
__device__ __forceinline__ void store8(void* at, int n, bool vec, const f2 (&x)[4]) {
  float* p = static_cast<float*>(at);
  if (vec) {
    asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p), "l"(x[0]), "l"(x[1]), "l"(x[2]), "l"(x[3]) : "memory");
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 u = split_f2(x[j]);
      if (2 * j < n) p[2 * j] = u.x;
      if (2 * j + 1 < n) p[2 * j + 1] = u.y;
    }
  }
}
// words of two bf16 each
__device__ __forceinline__ void store8_bf16(void* at, int n, bool vec, const uint32_t (&w)[4]) {
  uint16_t* p = static_cast<uint16_t*>(at);
  if (vec) {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
  }
}
__device__ __forceinline__ uint2 load_codes(const void* at, int n, bool vec) {
  const uint8_t* p = static_cast<const uint8_t*>(at);
  if (vec) return *reinterpret_cast<const uint2*>(p);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) w[j >> 2] |= (uint32_t)p[j] << (8 * (j & 3));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_codes(void* at, int n, bool vec, const uint32_t (&w)[2]) {
  uint8_t* p = static_cast<uint8_t*>(at);
  if (vec) {
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
  }
}
__device__ __forceinline__ void decode(uint2 codes, float scale, f2 (&x)[4]) {
  const f2 s2 = make_f2(scale, scale);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 u = unpack_e4m3x2((uint16_t)((j < 2 ? codes.x : codes.y) >> (16 * (j & 1))));
    x[j] = mul_f2(make_f2(u.x, u.y), s2);
  }
}

// IEEE square roots of eight values whose smallest and largest are given.  Values near zero, where newton_root's residual would
// leave float32, and infinities go through sqrtf.
__device__ __forceinline__ void root8(const f2 (&v)[4], uint32_t least, uint32_t most, f2 (&root)[4]) {
  if (least >= __float_as_uint(kRootMin) && most <= __float_as_uint(kRootMax)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) root[j] = newton_root(v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 u = split_f2(v[j]);
      root[j] = make_f2(__fsqrt_rn(u.x), __fsqrt_rn(u.y));
    }
  }
}
// of magnitudes; a NaN among them is passed over by the minimum and is the maximum
__device__ __forceinline__ float min3(float a, float b, float c) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
  return r;
}
// The smallest and the largest magnitude of eight values as ordered integers; NaN lies above infinity.
__device__ __forceinline__ void bounds8(const f2 (&x)[4], uint32_t* least, uint32_t* most) {
  const float2 a = split_f2(x[0]), b = split_f2(x[1]), c = split_f2(x[2]), d = split_f2(x[3]);
  *least = __float_as_uint(min3(min3(a.x, a.y, b.x), min3(b.y, c.x, c.y), fminf(fabsf(d.x), fabsf(d.y))));
  *most = __float_as_uint(max3(max3(max3(a.x, a.y, b.x), b.y, c.x), max3(c.y, d.x, d.y), 0.f));
}
// |y| (at most about 448, not NaN) with the part below an e4m3 step rounded up with probability remainder / step: the 16
// bits are added below the last kept bit and the rest is cut.  Below 2^-6 the codes are 2^-9 apart, as they are from 2^-6
// to 2^-5: the value is moved there and back.
__device__ __forceinline__ float e4m3_dither(float y, uint32_t bits16) {
  const float up = fabsf(y) < 0.015625f ? 0.015625f : 0.f;
  return copysignf(__uint_as_float((__float_as_uint(fabsf(y) + up) + (bits16 << 4)) & 0xfff00000u) - up, y);
}
// the same from 2^-6 on
__device__ __forceinline__ float e4m3_dither_normal(float y, uint32_t bits16) {
  return __uint_as_float((__float_as_uint(y) + (bits16 << 4)) & 0xfff00000u);
}
// Codes of x / scale, |x| at most 448 scale.  bits: 16 of each element, the lower ones for the first moment, the upper ones
// for the (root of the) second, of which a value above zero keeps a code above zero.
template <bool kSecond>
__device__ __forceinline__ void encode(const f2 (&x)[4], float least, float inv, bool seeded, const uint32_t (&bits)[8], uint32_t (&codes)[2]) {
  const f2 inv2 = make_f2(inv, inv);
  least *= inv;
  const auto bits16 = [&](int j) { return kSecond ? bits[j] >> 16 : bits[j] & 0xffffu; };
  codes[0] = codes[1] = 0;
  if (seeded && least >= 0.015625f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 u = split_f2(mul_f2(x[j], inv2));
      codes[j >> 1] |= pack_e4m3x2(e4m3_dither_normal(u.x, bits16(2 * j)), e4m3_dither_normal(u.y, bits16(2 * j + 1))) << (16 * (j & 1));
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 u = split_f2(mul_f2(x[j], inv2));
    const float a = seeded ? e4m3_dither(u.x, bits16(2 * j)) : u.x, b = seeded ? e4m3_dither(u.y, bits16(2 * j + 1)) : u.y;
    codes[j >> 1] |= pack_e4m3x2(a, b) << (16 * (j & 1));
  }
  if (kSecond && least < 0.001953125f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 u = split_f2(x[j >> 1]);
      if (((codes[j >> 2] >> (8 * (j & 3))) & 0xffu) == 0 && (j & 1 ? u.y : u.x) > 0.f) codes[j >> 2] |= 1u << (8 * (j & 3));
    }
  }
}

// One block of MRL_STATE_BLOCK elements by a warp.  The moments are rounded operation by operation as the formula stands
// (no fused multiply-add) and the 8-bit states take the IEEE root and reciprocal: the codes, which feed the next step, are
// then the same for every evaluation of the formula in float32, and a value on the border between two codes does not
// depend on how an expression was contracted.
// kKind: kind_of().
template <int kKind>
struct AdamwBlock {
  static constexpr bool kParamBf16 = (kKind & 1) != 0, kMaster = (kKind & 2) != 0, kCodes = (kKind & 8) != 0;
  using G = typename std::conditional<(kKind & 4) != 0, __nv_bfloat16, float>::type;
  using P = typename std::conditional<kParamBf16 && !kMaster, __nv_bfloat16, float>::type;
  Raw8<G> g;
  Raw8<P> p;
  Raw8<float> m, v;  // float32 states
  uint2 cm, cv;      // or codes
  float sm, sv;

  // Where a lane's eight elements are; moved from block to block.
  struct Cursor {
    const G* g;
    P* p;               // what the step is taken on: the master weights where there are any
    __nv_bfloat16* low; // and the parameter then
    char *m, *v;
    float *ms, *vs;
    unsigned long long word;  // position in the stream of random words
    int left;           // elements from the block's start to the end of the chunk
    bool aligned;

    __device__ __forceinline__ Cursor(const Slot& s, long long base, long long end, unsigned long long key) {
      const long long i = base + (threadIdx.x & 31) * 8;
      constexpr int kState = kCodes ? 1 : 4;
      g = static_cast<const G*>(s.grad) + i;
      p = static_cast<P*>(kMaster ? (void*)s.master : s.param) + i;
      low = static_cast<__nv_bfloat16*>(s.param) + i;
      m = static_cast<char*>(s.m) + i * kState;
      v = static_cast<char*>(s.v) + i * kState;
      ms = s.m_scale + base / MRL_STATE_BLOCK;
      vs = s.v_scale + base / MRL_STATE_BLOCK;
      word = key + s.rng_first + (unsigned long long)(i / 2);
      left = (int)(end - base);
      aligned = s.aligned;
    }
    __device__ __forceinline__ void advance(int blocks) {
      constexpr int kState = kCodes ? 1 : 4;
      const int e = blocks * MRL_STATE_BLOCK;
      g += e, p += e, m += e * kState, v += e * kState, word += e / 2, left -= e;
      if constexpr (kMaster) low += e;
      if constexpr (kCodes) ms += blocks, vs += blocks;
    }
    // elements of the lane in the block `ahead` elements on; whether the block is whole and aligned (the same for the warp)
    template <bool kWhole>
    __device__ __forceinline__ int count(int ahead) const { return kWhole ? 8 : min(8, max(0, left - ahead - (int)(threadIdx.x & 31) * 8)); }
    template <bool kWhole>
    __device__ __forceinline__ bool vec(int ahead) const { return kWhole || (aligned && left - ahead >= MRL_STATE_BLOCK); }
  };

  // `ahead` blocks behind the cursor
  template <bool kWhole>
  __device__ __forceinline__ void load(const Cursor& c, int ahead) {
    constexpr int kState = kCodes ? 1 : 4;
    const int e = ahead * MRL_STATE_BLOCK, n = c.template count<kWhole>(e);
    const bool vec = c.template vec<kWhole>(e);
    g.load(c.g + e, n, vec);
    if constexpr (kCodes) {
      cm = load_codes(c.m + e, n, vec);
      cv = load_codes(c.v + e, n, vec);
      sm = c.ms[ahead];
      sv = c.vs[ahead];
    } else {
      m.load(c.m + e * kState, n, vec);
      v.load(c.v + e * kState, n, vec);
    }
    p.load(c.p + e, n, vec);
  }
};

// `in` is the block; where `next` blocks on there is another one, its loads take the registers once they are free.
template <int kKind, bool kWhole>
__device__ __forceinline__ void adamw_block(const AdamwArgs& a, const Hyper& hy, float gs, float decay, const typename AdamwBlock<kKind>::Cursor& c,
                                            AdamwBlock<kKind>& in, bool more, int next) {
  using In = AdamwBlock<kKind>;
  constexpr bool kParamBf16 = In::kParamBf16, kMaster = In::kMaster, kCodes = In::kCodes;
  const int n = c.template count<kWhole>(0);
  const bool vec = c.template vec<kWhole>(0);
  f2 m[4], v[4], p[4];
  if constexpr (kCodes) {
    decode(in.cm, in.sm, m);
    decode(in.cv, in.sv, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = mul_f2(v[j], v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = in.m.pair(j);
      v[j] = in.v.pair(j);
    }
  }
  f2 root[4], g[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) g[j] = in.g.pair(j);
  const Raw8<typename In::P> raw = in.p;
  if (kCodes && more) in.template load<kWhole>(c, next);
  const f2 gs2 = make_f2(gs, gs), b1 = make_f2(a.beta1, a.beta1), o1 = make_f2(a.one_beta1, a.one_beta1);
  const f2 b2 = make_f2(a.beta2, a.beta2), o2 = make_f2(a.one_beta2, a.one_beta2);
  const f2 rc2 = make_f2(hy.root_c2, hy.root_c2), eps2 = make_f2(a.eps, a.eps), lr2 = make_f2(-hy.lr_c1, -hy.lr_c1);
  const f2 keep2 = make_f2(-hy.lr * decay, -hy.lr * decay);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f2 gj = mul_f2(g[j], gs2);
    p[j] = raw.pair(j);
    m[j] = add_apart(mul_f2(b1, m[j]), mul_f2(o1, gj));
    v[j] = add_apart(mul_f2(b2, v[j]), mul_f2(o2, mul_f2(gj, gj)));
  }
  uint32_t least_m = 0, most_m = 0, least_v = 0, most_v = 0;
  if constexpr (kCodes) {
    bounds8(m, &least_m, &most_m);
    bounds8(v, &least_v, &most_v);
    root8(v, least_v, most_v, root);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (!kCodes) {
      const float2 u = split_f2(v[j]);
      root[j] = make_f2(sqrt_approx(u.x), sqrt_approx(u.y));
    }
    const float2 den = split_f2(fma_f2(root[j], rc2, eps2));
    const f2 quot = mul_f2(mul_f2(m[j], lr2), make_f2(rcp_approx(den.x), rcp_approx(den.y)));
    p[j] = add_f2(p[j], fma_f2(keep2, p[j], quot));
  }
  uint32_t bits[8];  // of each element: 16 for m, 16 for v above them
  if (a.seeded && (kCodes || (kParamBf16 && !kMaster))) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned long long w = splitmix64(c.word + j);
      bits[2 * j] = (uint32_t)w;
      bits[2 * j + 1] = (uint32_t)(w >> 32);
    }
  }
  if constexpr (kMaster) store8(c.p, n, vec, p);
  if constexpr (kParamBf16) {
    uint32_t w[4];
    const bool cut = !kMaster && a.seeded;
    if (cut) {  // the 16 bits that are cut decide against m's in reverse order
      f2 nothing = 0ull;  // 0, or NaN where a value is not finite
#pragma unroll
      for (int j = 0; j < 4; ++j) nothing = fma_f2(p[j], 0ull, nothing);
      const float2 none = split_f2(nothing);
      if (none.x + none.y == 0.f) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 u = split_f2(p[j]);
          w[j] = __byte_perm(__float_as_uint(u.x) + (__brev(bits[2 * j]) >> 16), __float_as_uint(u.y) + (__brev(bits[2 * j + 1]) >> 16), 0x7632);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 u = split_f2(p[j]);
          const uint32_t lo = __float_as_uint(u.x) + (__brev(bits[2 * j]) >> 16), hi = __float_as_uint(u.y) + (__brev(bits[2 * j + 1]) >> 16);
          w[j] = f2_to_bf16x2(p[j]);
          if (fabsf(u.x) < INFINITY) w[j] = (w[j] & 0xffff0000u) | lo >> 16;
          if (fabsf(u.y) < INFINITY) w[j] = (w[j] & 0xffffu) | (hi & 0xffff0000u);
        }
      }
    }
    if (!cut) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = f2_to_bf16x2(p[j]);
    }
    store8_bf16(kMaster ? (void*)c.low : (void*)c.p, n, vec, w);
  } else {
    store8(c.p, n, vec, p);
  }
  if constexpr (kCodes) {
    most_m = __reduce_max_sync(0xffffffffu, most_m);
    most_v = __reduce_max_sync(0xffffffffu, most_v);
    const float sm = e4m3_scale(__uint_as_float(most_m));
    const float sv = e4m3_scale(__fsqrt_rn(__uint_as_float(most_v)));  // (the largest root is the root of the largest)
    if ((threadIdx.x & 31) == 0) {
      *c.ms = sm;
      *c.vs = sv;
    }
    uint32_t codes[2];
    const bool seeded = a.seeded && most_m < 0x7f800000u && most_v < 0x7f800000u;  // (the dither's arithmetic on bits is for numbers)
    encode<false>(m, __uint_as_float(least_m), __frcp_rn(sm), seeded, bits, codes);
    store_codes(c.m, n, vec, codes);
    encode<true>(root, sqrt_approx(__uint_as_float(least_v)) * 0.9999f, __frcp_rn(sv), seeded, bits, codes);
    store_codes(c.v, n, vec, codes);
  } else {
    store8(c.m, n, vec, m);
    store8(c.v, n, vec, v);
  }
}

// Sum of squares of a chunk's elements by this thread: runs of 32 in float32, added up in float64.  A run whose sum is near
// either end of float32's range (or 0) is squared again in float64.  Bound by HBM: 622 M bf16 elements in 179 us, 7.0 TB/s.
template <typename G>
__device__ __forceinline__ double chunk_squares(const Slot& s, long long lo, long long hi) {
  double sum = 0.0;
  for (long long base = lo; base < hi; base += kChunk * 4) {
    Raw8<G> x[4];
    f2 run2[2] = {0ull, 0ull};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long i = base + k * kChunk + threadIdx.x * 8;
      const int n = (int)(hi - i < 8 ? (hi > i ? hi - i : 0) : 8);
      x[k].load(static_cast<const G*>(s.grad) + i, n, s.aligned && n == 8);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) run2[j & 1] = fma_f2(x[k].pair(j), x[k].pair(j), run2[j & 1]);
    const float2 part = split_f2(add_f2(run2[0], run2[1]));
    const float run = part.x + part.y;
    if (run >= 1e-30f && run <= 1e38f) {
      sum += (double)run;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 u = split_f2(x[k].pair(j));
          sum = fma((double)u.x, (double)u.x, fma((double)u.y, (double)u.y, sum));
        }
    }
  }
  return sum;
}

// The chunks blockIdx.x, + gridDim.x, ... of the table; every thread gets the CTA's sum.
template <int kN>
__device__ __forceinline__ double table_squares(const Table<kN>& t, double* red) {
  double sum = 0.0;
  for (uint32_t chunk = blockIdx.x; chunk < t.first[t.n]; chunk += gridDim.x) {
    const int k = slot_of(t, chunk);
    const Slot& s = t.slot[k];
    const long long lo = (long long)(chunk - t.first[k]) * t.chunk, hi = min(lo + t.chunk, s.numel);
    sum += (s.kind & 4) ? chunk_squares<__nv_bfloat16>(s, lo, hi) : chunk_squares<float>(s, lo, hi);
  }
  return block_sum(sum, red);
}

// One partial sum per CTA; a later launch of the same call adds to it.
template <int kN>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ Table<kN> t, double* partial, bool first_launch) {
  __shared__ double red[kThreads / 32];
  let_next_start();
  const double sum = table_squares(t, red);
  if (threadIdx.x == 0) partial[blockIdx.x] = first_launch ? sum : partial[blockIdx.x] + sum;
}

// Few elements: one cluster, whose CTAs' sums meet in the first one's shared memory.  One launch.
template <int kN>
__global__ void __cluster_dims__(kCluster) __launch_bounds__(kThreads) grad_norm_small_kernel(const __grid_constant__ Table<kN> t, float max_norm,
                                                                                             float* norm, float* coef) {
  __shared__ double red[kThreads / 32], all[kCluster];
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const double sum = table_squares(t, red);
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // all CTAs run: their shared memory may be written
  if (threadIdx.x == 0) {
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(&all[blockIdx.x])));
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(sum) : "memory");
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    double total = 0.0;
    for (int k = 0; k < kCluster; ++k) total += all[k];
    write_norm(total, max_norm, norm, coef);
  }
}

// A chunk by its CTA.  kWhole: blocks of 256 aligned elements throughout, without tests.
template <int kKind, bool kWhole>
__device__ __forceinline__ void adamw_chunk(const AdamwArgs& a, const Hyper& hy, float gs, const Slot& s, long long lo, long long hi) {
  constexpr int kNext = step_threads(kKind) / 32;
  typename AdamwBlock<kKind>::Cursor c(s, lo + (threadIdx.x >> 5) * MRL_STATE_BLOCK, hi, hy.key);
  if (c.left <= 0) return;
  const float decay = s.decay;
  AdamwBlock<kKind> in;
  in.template load<kWhole>(c, 0);
#pragma unroll 1
  for (;;) {
    const bool more = c.left > kNext * MRL_STATE_BLOCK;
    adamw_block<kKind, kWhole>(a, hy, gs, decay, c, in, more, kNext);
    if (!more) break;
    c.advance(kNext);
    if (!AdamwBlock<kKind>::kCodes) in.template load<kWhole>(c, 0);
  }
}

// The tensors of one kind (types of gradient, parameter and states), which share the launch and its registers.
// With float32 states bound by HBM: 622 M elements (28 bytes each) in 2,585 us, 6.7 TB/s.  With 8-bit states and seeded
// rounding bound by the instructions' issue: a warp's 256 elements take 480 of them (two 64-bit multiplications for
// every two elements' random words, an IEEE root, codes both ways), 525 M elements (10 bytes each) 1,194 us, 4.4 TB/s.  The
// next block's loads are under way meanwhile, into the registers that this block's have left.
template <int kKind, int kN>
__global__ void __launch_bounds__(step_threads(kKind), step_ctas(kKind)) adamw_kernel(const __grid_constant__ Table<kN> t, const __grid_constant__ AdamwArgs a) {
  const float gs = a.grad_scale != nullptr ? *a.grad_scale : 1.f;
  if (!(fabsf(gs) < INFINITY)) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.status != nullptr) atomicOr(a.status, MRL_DEV_NONFINITE_GRAD);
    return;
  }
  const Hyper hy = a.hyper_dev != nullptr ? *a.hyper_dev : a.hyper;
  const int k = slot_of(t, blockIdx.x);
  const Slot& s = t.slot[k];
  const long long lo = (long long)(blockIdx.x - t.first[k]) * t.chunk, hi = min(lo + t.chunk, s.numel);
  if (s.aligned && ((hi - lo) & (MRL_STATE_BLOCK - 1)) == 0)
    adamw_chunk<kKind, true>(a, hy, gs, s, lo, hi);
  else
    adamw_chunk<kKind, false>(a, hy, gs, s, lo, hi);
}

bool grad_type_ok(int32_t dtype) { return dtype == MRL_BF16 || dtype == MRL_F32; }

bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Every pointer has to be a multiple of its element: a kernel's access anywhere else loses the context.  (Codes are bytes.)
int elem_bytes(int32_t dtype) { return dtype == MRL_BF16 ? 2 : 4; }
// (This and apart() avoid branches: for 154 tensors they take 0.1 and 0.3 us of an update's 8.)
uintptr_t bits_of(const void* p) { return reinterpret_cast<uintptr_t>(p); }
bool on_elements(const mrl_tensor_slot& s) {
  const bool codes = s.state_dtype == MRL_E4M3;
  const uintptr_t floats = bits_of(s.master) | bits_of(codes ? s.m_scale : s.m) | bits_of(codes ? s.v_scale : s.v);
  const uintptr_t halves = bits_of(s.grad) | bits_of(s.param);
  if (((floats & 3) | (halves & 1)) != 0) return false;
  return (halves & 2) == 0 || (aligned_to(s.grad, elem_bytes(s.grad_dtype)) && aligned_to(s.param, elem_bytes(s.param_dtype)));
}

// One buffer may not stand for two of a tensor's.
bool apart(const mrl_tensor_slot& s) {
  const void *g = s.grad, *p = s.param, *c = s.master;  // (the master alone may be null)
  return !((g == p) | (g == s.m) | (g == s.v) | (g == c) | (p == s.m) | (p == s.v) | (p == c) | (s.m == s.v) | (s.m == c) | (s.v == c) |
           ((s.state_dtype == MRL_E4M3) & (s.m_scale == s.v_scale)));
}

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

// Elements of a chunk: small ones while there are few in all, for the sake of parallel CTAs; `most` times as many otherwise.
int chunk_of(long long total, int threads, int most) {
  return threads * 8 * (total <= (long long)kSms * 8 * 4 * kChunk ? 1 : most);
}

template <int kN>
int launch_grad_norm(const mrl_tensor_slot* slots, int n, long long total, float max_norm, float* norm, float* coef, double* partial, cudaStream_t st) {
  Table<kN> t;
  const int chunk = chunk_of(total, kThreads, 8);
  int ctas = 0;
  for (int at = 0; at < n || ctas == 0;) {
    at = fill_table(slots, n, at, chunk, -1, &t);
    // Few chunks: one launch of a cluster (2.3 us for 2 chunks, 3.5 for 17, 6.9 for 65) in place of two of the whole GPU (3.2 us
    // up to 160, and 2 us more of the host's time); tables of nothing go there too.
    if (ctas == 0 && at == n && t.first[t.n] <= kSmallChunks) {
      mrl_profile_before(st, "grad_norm_small_kernel");
      grad_norm_small_kernel<kN><<<kCluster, kThreads, 0, st>>>(t, max_norm, norm, coef);
      mrl_profile_after(st);
      return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
    }
    if (t.n == 0) break;
    // (the first launch decides how many partials there are)
    const bool first = ctas == 0;
    if (first) ctas = at < n || t.first[t.n] > (uint32_t)kNormCtas ? kNormCtas : (int)t.first[t.n];
    mrl_profile_before(st, "grad_norm_kernel");
    grad_norm_kernel<kN><<<ctas, kThreads, 0, st>>>(t, partial, first);
    mrl_profile_after(st);
    MRL_CUDA_OK(cudaGetLastError());
  }
  MRL_CUDA_OK(mrl_launch_behind(grad_norm_finish_kernel, 1u, (unsigned)kThreads, st, partial, ctas, max_norm, norm, coef));
  return MRL_OK;
}

template <int kKind, int kN>
int launch_adamw_kind(const mrl_tensor_slot* slots, int n, int chunk, const AdamwArgs& a, cudaStream_t st) {
  Table<kN> t;
  for (int at = 0; at < n;) {
    at = fill_table(slots, n, at, chunk, kKind, &t);
    if (t.n == 0) break;
    mrl_profile_before(st, "adamw_kernel");
    adamw_kernel<kKind, kN><<<t.first[t.n], step_threads(kKind), 0, st>>>(t, a);
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
  if (n_slots < 0 || (n_slots > 0 && slots == nullptr) || max_norm != max_norm || (norm == nullptr && coef == nullptr) ||
      !aligned_to(norm, 4) || !aligned_to(coef, 4))
    return MRL_ERR_INVALID_ARG;
  long long total = 0;
  for (int k = 0; k < n_slots; ++k) {
    if (!grad_type_ok(slots[k].grad_dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
    if (slots[k].numel < 0 || slots[k].numel > kMaxNumel ||
        (slots[k].numel > 0 && (slots[k].grad == nullptr || !aligned_to(slots[k].grad, elem_bytes(slots[k].grad_dtype)))))
      return MRL_ERR_INVALID_ARG;
    total += slots[k].numel;
  }
  if (workspace == nullptr || workspace_bytes < mrl_grad_norm_workspace_bytes()) return MRL_ERR_WORKSPACE_TOO_SMALL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MRL_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  double* partial = static_cast<double*>(workspace);
  return n_slots <= kSlotsFew ? launch_grad_norm<kSlotsFew>(slots, n_slots, total, max_norm, norm, coef, partial, st)
                              : launch_grad_norm<kSlots>(slots, n_slots, total, max_norm, norm, coef, partial, st);
}

extern "C" int mrl_adamw_step(const mrl_tensor_slot* slots, int32_t n_slots, const mrl_adamw_params* ap,
                              const float* grad_scale, int32_t* status, void* workspace, size_t workspace_bytes,
                              void* stream) {
  if (ap == nullptr || n_slots < 0 || (n_slots > 0 && slots == nullptr)) return MRL_ERR_INVALID_ARG;
  if (!(ap->beta1 >= 0.0 && ap->beta1 < 1.0) || !(ap->beta2 >= 0.0 && ap->beta2 < 1.0) || !(ap->eps > 0.0) ||
      (float)ap->eps < 1.17549435e-38f || !(ap->eps < 3.4e38) || !(ap->lr - ap->lr == 0.0) || ap->flags != 0 ||
      (ap->step_dev == nullptr && ap->step < 1) || (ap->rounding != MRL_ROUND_NEAREST && ap->rounding != MRL_ROUND_SEEDED))
    return MRL_ERR_INVALID_ARG;
  // (one pass for all that the host needs of the tensors)
  bool all_apart = true;
  int count[16] = {0}, tensors = 0;
  long long total = 0;
  for (int k = 0; k < n_slots; ++k) {
    const mrl_tensor_slot& s = slots[k];
    if (!grad_type_ok(s.grad_dtype) || !grad_type_ok(s.param_dtype) || (s.state_dtype != MRL_F32 && s.state_dtype != MRL_E4M3))
      return MRL_ERR_UNSUPPORTED_DTYPE;
    if (s.numel < 0 || s.numel > kMaxNumel || !(s.weight_decay - s.weight_decay == 0.f)) return MRL_ERR_INVALID_ARG;
    if (s.numel == 0) continue;
    if (s.grad == nullptr || s.param == nullptr || s.m == nullptr || s.v == nullptr) return MRL_ERR_INVALID_ARG;
    if (s.master != nullptr && s.param_dtype != MRL_BF16) return MRL_ERR_INVALID_ARG;
    if (s.state_dtype == MRL_E4M3 && (s.m_scale == nullptr || s.v_scale == nullptr)) return MRL_ERR_INVALID_ARG;
    if (!on_elements(s)) return MRL_ERR_INVALID_ARG;
    all_apart &= apart(s);
    total += s.numel;
    ++count[kind_of(s)], ++tensors;
  }
  if (!aligned_to(grad_scale, 4) || !aligned_to(status, 4) || !aligned_to(ap->lr_dev, 4) || !aligned_to(ap->step_dev, 8))
    return MRL_ERR_INVALID_ARG;
  const bool on_device = ap->lr_dev != nullptr || ap->step_dev != nullptr;
  if (on_device) {
    if (workspace == nullptr || workspace_bytes < mrl_adamw_workspace_bytes()) return MRL_ERR_WORKSPACE_TOO_SMALL;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MRL_ERR_INVALID_ARG;
  }
  if (!all_apart) return MRL_ERR_INVALID_ARG;
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
  if (on_device || (tensors == 0 && grad_scale != nullptr && status != nullptr)) {
    adamw_prepare_kernel<<<1, 1, 0, st>>>(Hyper{}, ap->lr, ap->beta1, ap->beta2, ap->lr_dev, ap->step_dev, ap->step, ap->seed,
                                          grad_scale, status, on_device ? static_cast<Hyper*>(workspace) : nullptr);
    MRL_CUDA_OK(cudaGetLastError());
  }
  if (!on_device) {
    a.hyper.lr = (float)ap->lr;
    a.hyper.lr_c1 = (float)(ap->lr / (1.0 - pow(ap->beta1, (double)ap->step)));
    a.hyper.root_c2 = (float)(1.0 / sqrt(1.0 - pow(ap->beta2, (double)ap->step)));
    a.hyper.key = splitmix64(splitmix64(ap->seed) + (uint64_t)ap->step);
  }
  const int chunk[2] = {chunk_of(total, step_threads(0), step_blocks(0)), chunk_of(total, step_threads(8), step_blocks(8))};
  int rc = MRL_OK;
  const auto run = [&](auto kind) {
    constexpr int kKind = decltype(kind)::value;
    if (rc == MRL_OK) rc = launch_adamw<kKind>(slots, n_slots, count[kKind], chunk[kKind >> 3], a, st);
  };
  run(std::integral_constant<int, 0>{}), run(std::integral_constant<int, 1>{}), run(std::integral_constant<int, 3>{});
  run(std::integral_constant<int, 4>{}), run(std::integral_constant<int, 5>{}), run(std::integral_constant<int, 7>{});
  run(std::integral_constant<int, 8>{}), run(std::integral_constant<int, 9>{}), run(std::integral_constant<int, 11>{});
  run(std::integral_constant<int, 12>{}), run(std::integral_constant<int, 13>{}), run(std::integral_constant<int, 15>{});
  return rc;
}
