// The end of an optimisation step over many tensors at once: the gradients' 2-norm with the factor that clips it
// (mrl_grad_norm) and the AdamW update (mrl_adamw_step), App. A.
//
// Both read the tensors' addresses from a table that is passed by value with the launch, so nothing has to be kept on the
// device and a call can be captured.  The tensors are cut into chunks; a CTA finds its chunk's tensor by bisection in
// the table.  A few operations per element against 2 to 28 bytes: bound by HBM.
#include "mrl_common.cuh"

namespace {

using namespace mrl;

constexpr int kThreads = 256;
constexpr int kChunk = 2048;      // elements; a multiple of MRL_STATE_BLOCK
constexpr int kSlots = 352;       // tensors per launch: the table stays below the 32,764 bytes of kernel arguments
constexpr int kNormCtas = 148 * 8;

struct Slot {
  const void* grad;
  void* param;
  float* master;
  void *m, *v;
  float *m_scale, *v_scale;
  long long numel;
  unsigned long long rng_first;
  float decay;
  uint8_t grad_bf16, param_bf16, state_e4m3, pad;
};

// What changes from step to step.
struct Hyper {
  float lr, lr_c1, inv_c2;  // lr / (1 - beta1^t), 1 / (1 - beta2^t)
  int skip;
  unsigned long long key;   // of the step's random words
};

struct Table {
  Slot slot[kSlots];
  uint32_t first[kSlots + 1];  // first chunk of each tensor, and the number of chunks
  int n;
};
static_assert(sizeof(Table) + 256 <= 32764, "kernel arguments");

// The tensor that holds a chunk: the last one whose first chunk is not behind it.
__device__ __forceinline__ int slot_of(const Table& t, uint32_t chunk) {
  int lo = 0, hi = t.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.first[mid] <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ float grad_at(const Slot& s, long long i) {
  return s.grad_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(s.grad)[i]) : static_cast<const float*>(s.grad)[i];
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

// One partial sum of squares per CTA; a later launch of the same call adds to it.
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ Table t, double* __restrict__ partial,
                                                             bool first_launch) {
  __shared__ double red[kThreads / 32];
  double sum = 0.0;
  for (uint32_t chunk = blockIdx.x; chunk < t.first[t.n]; chunk += gridDim.x) {
    const int k = slot_of(t, chunk);
    const Slot& s = t.slot[k];
    const long long lo = (long long)(chunk - t.first[k]) * kChunk, hi = min(lo + kChunk, s.numel);
    for (long long i = lo + threadIdx.x; i < hi; i += kThreads) {
      const double g = grad_at(s, i);
      sum += g * g;
    }
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) partial[blockIdx.x] = first_launch ? sum : partial[blockIdx.x] + sum;
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
  h.inv_c2 = (float)(1.0 / (1.0 - pow(beta2, (double)step)));
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

// y (magnitude at most about 448) with the part below an e4m3 step rounded up with probability remainder / step: the
// 16 bits are added below the last kept bit and the rest is cut.  Below 2^-6 the codes are 2^-9 apart, as they are from
// 2^-6 to 2^-5: the value is moved there and back.
__device__ __forceinline__ float e4m3_dither(float y, uint32_t bits) {
  const float a = fabsf(y);
  if (!(a <= 1e30f)) return y;
  const bool small = a < 0.015625f;
  float z = small ? a + 0.015625f : a;
  z = __uint_as_float((__float_as_uint(z) + (bits << 4)) & 0xfff00000u);
  return copysignf(small ? z - 0.015625f : z, y);
}

__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table t, const __grid_constant__ AdamwArgs a) {
  __shared__ float red[2][kThreads / 32];
  const float gs = a.grad_scale != nullptr ? *a.grad_scale : 1.f;
  if (!(fabsf(gs) < INFINITY)) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.status != nullptr) atomicOr(a.status, MRL_DEV_NONFINITE_GRAD);
    return;
  }
  const Hyper hy = a.hyper_dev != nullptr ? *a.hyper_dev : a.hyper;
  const int k = slot_of(t, blockIdx.x);
  const Slot& s = t.slot[k];
  const long long lo = (long long)(blockIdx.x - t.first[k]) * kChunk;
  for (long long base = lo; base < min(lo + kChunk, s.numel); base += kThreads) {  // one state block per step
    const long long i = base + threadIdx.x;
    const bool in = i < s.numel;
    const long long blk = base / MRL_STATE_BLOCK;
    float m = 0.f, v = 0.f, p = 0.f;
    uint32_t rm = 0, rv = 0;
    if (in) {
      const float g = grad_at(s, i) * gs;
      if (s.state_e4m3) {
        m = unpack_e4m3x2(static_cast<const uint8_t*>(s.m)[i]).x * s.m_scale[blk];
        const float q = unpack_e4m3x2(static_cast<const uint8_t*>(s.v)[i]).x * s.v_scale[blk];
        v = q * q;
      } else {
        m = static_cast<const float*>(s.m)[i];
        v = static_cast<const float*>(s.v)[i];
      }
      m = fmaf(a.beta1, m, a.one_beta1 * g);
      v = fmaf(a.beta2, v, a.one_beta2 * g * g);
      p = s.master != nullptr ? s.master[i]
                              : (s.param_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(s.param)[i])
                                              : static_cast<const float*>(s.param)[i]);
      p -= fmaf(hy.lr * s.decay, p, hy.lr_c1 * m / (sqrtf(v * hy.inv_c2) + a.eps));
      if (a.seeded) {
        const unsigned long long w = splitmix64(hy.key + s.rng_first + (unsigned long long)(i >> 1)) >> (32 * (i & 1));
        rm = (uint32_t)w & 0xffffu;
        rv = (uint32_t)(w >> 16) & 0xffffu;
      }
      if (s.master != nullptr) s.master[i] = p;
      if (!s.param_bf16)
        static_cast<float*>(s.param)[i] = p;
      else if (a.seeded && s.master == nullptr && fabsf(p) < INFINITY)
        static_cast<uint16_t*>(s.param)[i] = (uint16_t)((__float_as_uint(p) + (__brev(rm) >> 16)) >> 16);
      else
        static_cast<__nv_bfloat16*>(s.param)[i] = __float2bfloat16_rn(p);
      if (!s.state_e4m3) {
        static_cast<float*>(s.m)[i] = m;
        static_cast<float*>(s.v)[i] = v;
      }
    }
    if (s.state_e4m3) {  // the branch is the same for the whole CTA
      const float root = sqrtf(v);
      float am = fabsf(m), av = root;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, o));
        av = fmaxf(av, __shfl_xor_sync(0xffffffffu, av, o));
      }
      __syncthreads();
      if ((threadIdx.x & 31) == 0) {
        red[0][threadIdx.x >> 5] = am;
        red[1][threadIdx.x >> 5] = av;
      }
      __syncthreads();
      for (int w = 0; w < kThreads / 32; ++w) {
        am = fmaxf(am, red[0][w]);
        av = fmaxf(av, red[1][w]);
      }
      const float sm = e4m3_scale(am), sv = e4m3_scale(av);
      if (threadIdx.x == 0) {
        s.m_scale[blk] = sm;
        s.v_scale[blk] = sv;
      }
      if (in) {
        float ym = m * (1.f / sm), yv = root * (1.f / sv);
        if (a.seeded) {
          ym = e4m3_dither(ym, rm);
          yv = e4m3_dither(yv, rv);
        }
        uint32_t cv = pack_e4m3x2(yv, 0.f) & 0xffu;
        if (cv == 0 && v > 0.f) cv = 1;
        static_cast<uint8_t*>(s.m)[i] = (uint8_t)pack_e4m3x2(ym, 0.f);
        static_cast<uint8_t*>(s.v)[i] = (uint8_t)cv;
      }
    }
  }
}
static_assert(kThreads == MRL_STATE_BLOCK, "one state block per step of a CTA");

bool grad_type_ok(int32_t dtype) { return dtype == MRL_BF16 || dtype == MRL_F32; }

// Fills the table with tensors from slots[at] on, as many as it holds, and returns the index of the first one left out.
int fill_table(const mrl_tensor_slot* slots, int n, int at, Table* t) {
  uint32_t chunks = 0;
  t->n = 0;
  for (; at < n && t->n < kSlots; ++at) {
    const mrl_tensor_slot& s = slots[at];
    if (s.numel == 0) continue;
    const long long need = (s.numel + kChunk - 1) / kChunk;
    if (chunks + need > 0x7fffffffll) break;
    t->slot[t->n] = Slot{s.grad, s.param, s.master, s.m, s.v, s.m_scale, s.v_scale, s.numel, s.rng_first, s.weight_decay,
                         (uint8_t)(s.grad_dtype == MRL_BF16), (uint8_t)(s.param_dtype == MRL_BF16),
                         (uint8_t)(s.state_dtype == MRL_E4M3), 0};
    t->first[t->n++] = chunks;
    chunks += (uint32_t)need;
  }
  t->first[t->n] = chunks;
  return at;
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
  Table t;
  int at = 0, grid = 0;
  while (at < n_slots) {
    at = fill_table(slots, n_slots, at, &t);
    if (t.n == 0) break;
    // (every launch but the last holds a full table; the first decides how many partials there are)
    const bool first = grid == 0;
    if (first) grid = at < n_slots || t.first[t.n] > (uint32_t)kNormCtas ? kNormCtas : (int)t.first[t.n];
    mrl_profile_before(st, "grad_norm_kernel");
    grad_norm_kernel<<<grid, kThreads, 0, st>>>(t, partial, first);
    mrl_profile_after(st);
    MRL_CUDA_OK(cudaGetLastError());
  }
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
    a.hyper.inv_c2 = (float)(1.0 / (1.0 - pow(ap->beta2, (double)ap->step)));
    a.hyper.key = splitmix64(splitmix64(ap->seed) + (uint64_t)ap->step);
  }
  Table t;
  for (int at = 0; at < n_slots;) {
    at = fill_table(slots, n_slots, at, &t);
    if (t.n == 0) break;
    mrl_profile_before(st, "adamw_kernel");
    adamw_kernel<<<t.first[t.n], kThreads, 0, st>>>(t, a);
    mrl_profile_after(st);
    MRL_CUDA_OK(cudaGetLastError());
  }
  return MRL_OK;
}
