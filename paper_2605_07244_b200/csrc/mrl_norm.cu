// Root-mean-square norm with the residual's addition (mrl_rmsnorm_residual_fwd / _bwd): the rows that enter the fused LM
// head, and the way back for its dHidden.
//
// Forward: h = x + r, rstd = 1 / sqrt(mean h^2 + eps), y = h rstd (w + o), optionally as e4m3 codes with a scale per group.
// Backward: with g = (w + o) dy and xhat = h rstd, dx = dh + rstd (g - xhat mean(g xhat)), dw = sum over rows of dy xhat.
// A few operations per element against 6 to 9 bytes: bound by HBM.
#include "mrl_common.cuh"

namespace {

using namespace mrl;

constexpr int kSms = 148;
constexpr int kLoopThreads = 512;
constexpr int kRowCols = 16;                       // columns a thread holds in registers
constexpr int kRowMax = kRowCols * 1024;           // the widest row that one CTA holds

template <typename T>
__device__ __forceinline__ float load_f(const T* p);
template <>
__device__ __forceinline__ float load_f<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_f<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_f(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float weight_at(const void* w, bool w_bf16, int i) {
  return w_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(w)[i]) : static_cast<const float*>(w)[i];
}

// Sum / maximum over the block in a fixed order; every thread gets the result.  `red` holds 32 floats.
template <bool kMax>
__device__ __forceinline__ float block_reduce(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, v, o);
    v = kMax ? fmaxf(v, u) : v + u;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float r = red[0];
  for (int k = 1; k < (int)(blockDim.x >> 5); ++k) r = kMax ? fmaxf(r, red[k]) : r + red[k];
  return r;
}

struct NormFwdArgs {
  const void *x, *res, *w;
  void *h_out, *y;
  uint8_t* y8;
  float *scales, *rstd;
  long long ld_x, ld_res, ld_h, ld_y, ld_y8, N;
  int H, group;
  bool w_bf16;
  float eps, offset, inv_h;
};

struct NormBwdArgs {
  const void *dy, *dh, *h, *w;
  const float* rstd;
  void* dx;
  float* partial;  // [gridDim.x, H], null: no dweight
  long long ld_dy, ld_dh, ld_h, ld_dx, N;
  int H;
  bool w_bf16;
  float offset, inv_h;
};

// Rows of any length and alignment, one element per thread and step; the inputs are read again in each pass.
template <typename T>
__global__ void __launch_bounds__(kLoopThreads) rmsnorm_fwd_loop_kernel(NormFwdArgs a) {
  __shared__ float red[32];
  const int tid = threadIdx.x, nt = blockDim.x;
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    const T* r = a.res != nullptr ? static_cast<const T*>(a.res) + row * a.ld_res : nullptr;
    const auto h_at = [&](int i) { return r != nullptr ? load_f(x + i) + load_f(r + i) : load_f(x + i); };
    float ss = 0.f;
    for (int i = tid; i < a.H; i += nt) {
      const float h = h_at(i);
      ss = fmaf(h, h, ss);
    }
    ss = block_reduce<false>(ss, red);
    float rstd = rsqrtf(fmaf(ss, a.inv_h, a.eps));
    if (ss == INFINITY) {  // the squares may have left float32 although the row has not
      float m = 0.f;
      for (int i = tid; i < a.H; i += nt) m = fmaxf(m, fabsf(h_at(i)));
      m = block_reduce<true>(m, red);
      if (m < INFINITY) {
        const float s = scalbnf(1.f, -ilogbf(m));
        float q = 0.f;
        for (int i = tid; i < a.H; i += nt) {
          const float h = h_at(i) * s;
          q = fmaf(h, h, q);
        }
        q = block_reduce<false>(q, red);
        rstd = s * rsqrtf(fmaf(q, a.inv_h, a.eps * s * s));
      }
    }
    if (tid == 0 && a.rstd != nullptr) a.rstd[row] = rstd;
    if (a.y8 != nullptr) {
      const int group = a.group > 0 ? a.group : a.H, groups = (a.H + group - 1) / group;
      for (int k = 0; k < groups; ++k) {
        const int lo = k * group, hi = min(a.H, lo + group);
        float m = 0.f;
        for (int i = lo + tid; i < hi; i += nt) m = fmaxf(m, fabsf(h_at(i) * rstd * (weight_at(a.w, a.w_bf16, i) + a.offset)));
        m = block_reduce<true>(m, red);
        const float scale = e4m3_scale(m);
        if (tid == 0) a.scales[row * groups + k] = scale;
        const float inv = 1.f / scale;
        for (int i = lo + tid; i < hi; i += nt)
          a.y8[row * a.ld_y8 + i] = (uint8_t)pack_e4m3x2(h_at(i) * rstd * (weight_at(a.w, a.w_bf16, i) + a.offset) * inv, 0.f);
      }
    }
    if (a.y != nullptr || a.h_out != nullptr) {
      // last, since either may lie over an input; each element is written by the thread that has just read it
      for (int i = tid; i < a.H; i += nt) {
        const float h = h_at(i);
        if (a.h_out != nullptr) store_f(static_cast<T*>(a.h_out) + row * a.ld_h + i, h);
        if (a.y != nullptr) store_f(static_cast<T*>(a.y) + row * a.ld_y + i, h * rstd * (weight_at(a.w, a.w_bf16, i) + a.offset));
      }
    }
  }
}

// Backward, any length and alignment.  Each CTA keeps its own row of dweight partials (written by the thread that owns the
// column: no atomics).
template <typename T>
__global__ void __launch_bounds__(kLoopThreads) rmsnorm_bwd_loop_kernel(NormBwdArgs a) {
  __shared__ float red[32];
  const int tid = threadIdx.x, nt = blockDim.x;
  float* part = a.partial != nullptr ? a.partial + (size_t)blockIdx.x * a.H : nullptr;
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x) {
    const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
    const T* hr = static_cast<const T*>(a.h) + row * a.ld_h;
    const float rstd = a.rstd[row];
    float c = 0.f;
    for (int i = tid; i < a.H; i += nt) {
      const float d = load_f(dy + i), xhat = load_f(hr + i) * rstd;
      c = fmaf(d * (weight_at(a.w, a.w_bf16, i) + a.offset), xhat, c);
      if (part != nullptr) part[i] = row == blockIdx.x ? d * xhat : fmaf(d, xhat, part[i]);
    }
    c = block_reduce<false>(c, red) * a.inv_h;
    for (int i = tid; i < a.H; i += nt) {
      const float g = load_f(dy + i) * (weight_at(a.w, a.w_bf16, i) + a.offset), xhat = load_f(hr + i) * rstd;
      float v = (g - xhat * c) * rstd;
      if (a.dh != nullptr) v += load_f(static_cast<const T*>(a.dh) + row * a.ld_dh + i);
      store_f(static_cast<T*>(a.dx) + row * a.ld_dx + i, v);
    }
  }
}

// kE adjacent elements of a row as 32-bit words: one load or store of 32, 16, 4 or 2 bytes.
template <typename T, int kE>
struct RowVec {
  static constexpr int kBytes = kE * (int)sizeof(T);
  static constexpr int kWords = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[kWords];

  // (not the read-only path: outputs may lie over inputs)
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes == 32)
      asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                   : "l"(p));
    else if constexpr (kBytes == 16)
      asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    else if constexpr (kBytes == 4)
      asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
    else {
      uint16_t h;
      asm volatile("ld.global.b16 %0, [%1];" : "=h"(h) : "l"(p));
      w[0] = h;
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kBytes == 32)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                   "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                   : "memory");
    else if constexpr (kBytes == 16)
      asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    else if constexpr (kBytes == 4)
      asm volatile("st.global.b32 [%0], %1;" ::"l"(p), "r"(w[0]) : "memory");
    else
      asm volatile("st.global.b16 [%0], %1;" ::"l"(p), "h"((uint16_t)w[0]) : "memory");
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < kWords; ++k) w[k] = 0;
  }
  __device__ __forceinline__ float at(int j) const {
    if constexpr (sizeof(T) == 4)
      return __uint_as_float(w[j]);
    else
      return (j & 1) ? bf16hi_to_f32(w[j >> 1]) : bf16lo_to_f32(w[j >> 1]);
  }
  __device__ __forceinline__ void set(const float* v) {
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      if constexpr (sizeof(T) == 4)
        w[k] = __float_as_uint(v[k]);
      else
        w[k] = pack_bf16x2(v[2 * k], kE > 1 ? v[2 * k + 1] : 0.f);
    }
  }
};

// kE gains from column c on (weight + offset); the weight stays in L1.
template <int kE>
__device__ __forceinline__ void load_gain(const void* w, bool w_bf16, float offset, int c, float* g) {
  if constexpr (kE == 1) {
    g[0] = weight_at(w, w_bf16, c) + offset;
  } else if (w_bf16) {
    const uint2* p = reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(w) + c);
#pragma unroll
    for (int k = 0; k < kE / 4; ++k) {
      const uint2 u = __ldg(p + k);
      g[4 * k] = bf16lo_to_f32(u.x) + offset;
      g[4 * k + 1] = bf16hi_to_f32(u.x) + offset;
      g[4 * k + 2] = bf16lo_to_f32(u.y) + offset;
      g[4 * k + 3] = bf16hi_to_f32(u.y) + offset;
    }
  } else {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(w) + c);
#pragma unroll
    for (int k = 0; k < kE / 4; ++k) {
      const float4 u = __ldg(p + k);
      g[4 * k] = u.x + offset;
      g[4 * k + 1] = u.y + offset;
      g[4 * k + 2] = u.z + offset;
      g[4 * k + 3] = u.w + offset;
    }
  }
}

// As block_reduce, for a kernel that never reuses `red` before another barrier: one barrier, none for a single warp.
template <bool kMax>
__device__ __forceinline__ float row_reduce(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, v, o);
    v = kMax ? fmaxf(v, u) : v + u;
  }
  const int warps = blockDim.x >> 5;
  if (warps == 1) {
    __syncwarp();
    return v;
  }
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float r = red[0];
  for (int k = 1; k < warps; ++k) r = kMax ? fmaxf(r, red[k]) : r + red[k];
  return r;
}

// One CTA per row, the row in registers between its one read and its writes: kV vectors of kE columns per thread, vector v
// of thread t at column (v * blockDim.x + t) * kE.
template <typename T, int kE, int kV, int kMaxThreads, int kMinCtas>
__global__ void __launch_bounds__(kMaxThreads, kMinCtas) rmsnorm_fwd_row_kernel(const __grid_constant__ NormFwdArgs a) {
  using Vec = RowVec<T, kE>;
  __shared__ float red[4][32];
  __shared__ uint32_t peak[kRowMax / 32];
  const int tid = threadIdx.x, nt = blockDim.x;
  const int group = a.group > 0 ? a.group : a.H, groups = (a.H + group - 1) / group;
  // lanes whose columns share a scale sit side by side; more than a warp of them meet in shared memory
  const bool meet = a.y8 != nullptr && a.group > 32 * kE;
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x) {
    float h[kV][kE];
    {
      Vec x[kV], r[kV];
#pragma unroll
      for (int v = 0; v < kV; ++v) {
        const int c = (v * nt + tid) * kE;
        x[v].zero();
        if (c < a.H) x[v].load(static_cast<const T*>(a.x) + row * a.ld_x + c);
      }
      if (a.res != nullptr) {
#pragma unroll
        for (int v = 0; v < kV; ++v) {
          const int c = (v * nt + tid) * kE;
          r[v].zero();
          if (c < a.H) r[v].load(static_cast<const T*>(a.res) + row * a.ld_res + c);
        }
      }
#pragma unroll
      for (int v = 0; v < kV; ++v)
#pragma unroll
        for (int j = 0; j < kE; ++j) h[v][j] = a.res != nullptr ? x[v].at(j) + r[v].at(j) : x[v].at(j);
    }
    if (meet)
      for (int k = tid; k < groups; k += nt) peak[k] = 0;
    float ss = 0.f;
#pragma unroll
    for (int v = 0; v < kV; ++v)
#pragma unroll
      for (int j = 0; j < kE; ++j) ss = fmaf(h[v][j], h[v][j], ss);
    ss = row_reduce<false>(ss, red[0]);
    float rstd = rsqrtf(fmaf(ss, a.inv_h, a.eps));
    if (ss == INFINITY) {  // the squares may have left float32 although the row has not
      float m = 0.f;
#pragma unroll
      for (int v = 0; v < kV; ++v)
#pragma unroll
        for (int j = 0; j < kE; ++j) m = fmaxf(m, fabsf(h[v][j]));
      m = row_reduce<true>(m, red[1]);
      if (m < INFINITY) {
        const float s = scalbnf(1.f, -ilogbf(m));
        float q = 0.f;
#pragma unroll
        for (int v = 0; v < kV; ++v)
#pragma unroll
          for (int j = 0; j < kE; ++j) q = fmaf(h[v][j] * s, h[v][j] * s, q);
        q = row_reduce<false>(q, red[2]);
        rstd = s * rsqrtf(fmaf(q, a.inv_h, a.eps * s * s));
      }
    }
    if (tid == 0 && a.rstd != nullptr) a.rstd[row] = rstd;
    if (a.h_out != nullptr) {
#pragma unroll
      for (int v = 0; v < kV; ++v) {
        const int c = (v * nt + tid) * kE;
        Vec o;
        o.set(h[v]);
        if (c < a.H) o.store(static_cast<T*>(a.h_out) + row * a.ld_h + c);
      }
    }
    float top = 0.f;  // of the row (one scale for all columns)
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int c = (v * nt + tid) * kE;
      float g[kE];
      if (c < a.H) {
        load_gain<kE>(a.w, a.w_bf16, a.offset, c, g);
#pragma unroll
        for (int j = 0; j < kE; ++j) h[v][j] = h[v][j] * rstd * g[j];
      }  // (columns behind the row hold 0)
      if (a.y != nullptr) {
        Vec o;
        o.set(h[v]);
        if (c < a.H) o.store(static_cast<T*>(a.y) + row * a.ld_y + c);
      }
    }
    if (a.y8 == nullptr) {
      if (row + gridDim.x < a.N) __syncthreads();
      continue;
    }
    float inv[kV];
    if (a.group == 0) {
#pragma unroll
      for (int v = 0; v < kV; ++v)
#pragma unroll
        for (int j = 0; j < kE; ++j) top = fmaxf(top, fabsf(h[v][j]));
      top = row_reduce<true>(top, red[3]);
      const float scale = e4m3_scale(top);
      if (tid == 0) a.scales[row] = scale;
#pragma unroll
      for (int v = 0; v < kV; ++v) inv[v] = 1.f / scale;
    } else {
      const int lanes = min(32, group / kE);
#pragma unroll
      for (int v = 0; v < kV; ++v) {
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < kE; ++j) m = fmaxf(m, fabsf(h[v][j]));
        for (int o = lanes >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const int c = (v * nt + tid) * kE;
        if (meet) {
          if ((tid & 31) == 0 && c < a.H) atomicMax(&peak[c / group], __float_as_uint(m));
        } else {
          const float scale = e4m3_scale(m);
          if (c < a.H && c % group == 0) a.scales[row * groups + c / group] = scale;
          inv[v] = 1.f / scale;
        }
      }
      if (meet) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < kV; ++v) {
          const int c = (v * nt + tid) * kE;
          if (c < a.H) {
            const float scale = e4m3_scale(__uint_as_float(peak[c / group]));
            if (c % group == 0) a.scales[row * groups + c / group] = scale;
            inv[v] = 1.f / scale;
          }
        }
      }
    }
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int c = (v * nt + tid) * kE;
      if (c >= a.H) continue;
      uint8_t* q = a.y8 + row * a.ld_y8 + c;
      if constexpr (kE == 1) {
        *q = (uint8_t)pack_e4m3x2(h[v][0] * inv[v], 0.f);
      } else {
        uint32_t o[kE / 4];
#pragma unroll
        for (int k = 0; k < kE / 4; ++k)
          o[k] = pack_e4m3x2(h[v][4 * k] * inv[v], h[v][4 * k + 1] * inv[v]) |
                 pack_e4m3x2(h[v][4 * k + 2] * inv[v], h[v][4 * k + 3] * inv[v]) << 16;
        if constexpr (kE == 16)
          *reinterpret_cast<uint4*>(q) = make_uint4(o[0], o[1], o[2], o[3]);
        else if constexpr (kE == 8)
          *reinterpret_cast<uint2*>(q) = make_uint2(o[0], o[1]);
        else
          *reinterpret_cast<uint32_t*>(q) = o[0];
      }
    }
    if (row + gridDim.x < a.N) __syncthreads();
  }
}

// Backward of rows held in registers.  A CTA walks rows blockIdx.x, + gridDim.x, ...; each thread keeps the dweight sums of
// its columns in registers over all of them and writes them once.
template <typename T, int kE, int kV, int kMaxThreads, int kMinCtas>
__global__ void __launch_bounds__(kMaxThreads, kMinCtas) rmsnorm_bwd_row_kernel(const __grid_constant__ NormBwdArgs a) {
  using Vec = RowVec<T, kE>;
  __shared__ float red[2][32];
  const int tid = threadIdx.x, nt = blockDim.x;
  float dw[kV][kE];
#pragma unroll
  for (int v = 0; v < kV; ++v)
#pragma unroll
    for (int j = 0; j < kE; ++j) dw[v][j] = 0.f;
  int turn = 0;  // the reduction's scratch alternates: one barrier per row
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x, turn ^= 1) {
    Vec dy[kV], h[kV], dh[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int c = (v * nt + tid) * kE;
      dy[v].zero();
      h[v].zero();
      dh[v].zero();
      if (c < a.H) {
        dy[v].load(static_cast<const T*>(a.dy) + row * a.ld_dy + c);
        h[v].load(static_cast<const T*>(a.h) + row * a.ld_h + c);
        if (a.dh != nullptr) dh[v].load(static_cast<const T*>(a.dh) + row * a.ld_dh + c);
      }
    }
    const float rstd = a.rstd[row];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int c = (v * nt + tid) * kE;
      if (c < a.H) {
        float g[kE];
        load_gain<kE>(a.w, a.w_bf16, a.offset, c, g);
#pragma unroll
        for (int j = 0; j < kE; ++j) {
          const float d = dy[v].at(j), xhat = h[v].at(j) * rstd;
          sum = fmaf(d * g[j], xhat, sum);
          dw[v][j] = fmaf(d, xhat, dw[v][j]);
        }
      }
    }
    const float mean = row_reduce<false>(sum, red[turn]) * a.inv_h;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int c = (v * nt + tid) * kE;
      if (c < a.H) {
        float g[kE];
        load_gain<kE>(a.w, a.w_bf16, a.offset, c, g);
#pragma unroll
        for (int j = 0; j < kE; ++j) g[j] = fmaf(dy[v].at(j) * g[j] - h[v].at(j) * rstd * mean, rstd, dh[v].at(j));
        Vec o;
        o.set(g);
        o.store(static_cast<T*>(a.dx) + row * a.ld_dx + c);
      }
    }
  }
  if (a.partial != nullptr) {
    float* part = a.partial + (size_t)blockIdx.x * a.H;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const int c = (v * nt + tid) * kE;
      if (c < a.H) {
#pragma unroll
        for (int j = 0; j < kE; ++j) part[c + j] = dw[v][j];
      }
    }
  }
}

// dweight[i] = sum over the CTAs' partials, in their order within each of 8 lanes and then over the lanes.
__global__ void __launch_bounds__(256) rmsnorm_dw_kernel(const float* __restrict__ partial, int rows, int H,
                                                         float* __restrict__ dw, bool accumulate) {
  __shared__ float red[8][33];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
  float s = 0.f;
  if (col < H)
    for (int k = lane; k < rows; k += 8) s += partial[(size_t)k * H + col];
  red[lane][threadIdx.x & 31] = s;
  __syncthreads();
  if (lane == 0 && col < H) {
    for (int k = 1; k < 8; ++k) s += red[k][threadIdx.x];
    dw[col] = accumulate ? dw[col] + s : s;
  }
}

int row_threads(int H) { return (H + kRowCols * 32 - 1) / (kRowCols * 32) * 32; }

// CTAs of the backward kernels, and rows of dweight partials: as many as are resident together.
int bwd_ctas(long long N, int H) {
  int per_sm = 2;
  if (H <= kRowMax) {
    per_sm = 768 / row_threads(H);
    per_sm = per_sm < 1 ? 1 : (per_sm > 16 ? 16 : per_sm);
  }
  return (int)(N < (long long)kSms * per_sm ? N : (long long)kSms * per_sm);
}

bool aligned(const void* p, long long ld, int bytes, int elem) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0 && (ld * elem) % bytes == 0);
}

// Bytes of the widest vector that every row of the call allows: 32, 16, or one element.
int fwd_vector(const NormFwdArgs& a, int elem) {
  for (int bytes = 32; bytes >= 16; bytes >>= 1) {
    const int e = bytes / elem;
    if (a.H % e == 0 && aligned(a.x, a.ld_x, bytes, elem) && aligned(a.res, a.ld_res, bytes, elem) &&
        aligned(a.h_out, a.ld_h, bytes, elem) && aligned(a.y, a.ld_y, bytes, elem) && aligned(a.y8, a.ld_y8, e, 1) &&
        aligned(a.w, 0, 16, 1))
      return bytes;
  }
  return elem;
}
int bwd_vector(const NormBwdArgs& a, int elem) {
  for (int bytes = 32; bytes >= 16; bytes >>= 1)
    if (a.H % (bytes / elem) == 0 && aligned(a.dy, a.ld_dy, bytes, elem) && aligned(a.dh, a.ld_dh, bytes, elem) &&
        aligned(a.h, a.ld_h, bytes, elem) && aligned(a.dx, a.ld_dx, bytes, elem) && aligned(a.w, 0, 16, 1))
      return bytes;
  return elem;
}

template <typename T, int kE>
void launch_fwd_rows(const NormFwdArgs& a, unsigned grid, cudaStream_t st) {
  const int nt = row_threads(a.H);
  if (nt <= 256)
    rmsnorm_fwd_row_kernel<T, kE, kRowCols / kE, 256, 5><<<grid, nt, 0, st>>>(a);
  else
    rmsnorm_fwd_row_kernel<T, kE, kRowCols / kE, 1024, 1><<<grid, nt, 0, st>>>(a);
}
template <typename T, int kE>
void launch_bwd_rows(const NormBwdArgs& a, int grid, cudaStream_t st) {
  const int nt = row_threads(a.H);
  if (nt <= 256)
    rmsnorm_bwd_row_kernel<T, kE, kRowCols / kE, 256, 3><<<grid, nt, 0, st>>>(a);
  else
    rmsnorm_bwd_row_kernel<T, kE, kRowCols / kE, 1024, 1><<<grid, nt, 0, st>>>(a);
}

bool row_type_ok(int32_t dtype) { return dtype == MRL_BF16 || dtype == MRL_F32; }

}  // namespace

size_t mrl_rmsnorm_bwd_workspace_bytes(long long N, int H) {
  if (N <= 0 || H <= 0) return 0;
  return mrl_align_up((size_t)bwd_ctas(N, H) * (size_t)H * 4, 256);
}

extern "C" int mrl_rmsnorm_residual_fwd(const void* x, int64_t ld_x, const void* residual, int64_t ld_res, int32_t dtype,
                                        const void* weight, int32_t w_dtype, int64_t N, int32_t H,
                                        const mrl_norm_params* np, void* h_out, int64_t ld_h, void* y, int64_t ld_y,
                                        void* y8, int64_t ld_y8, float* scales, float* rstd, void* stream) {
  if (!row_type_ok(dtype) || !row_type_ok(w_dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
  if (np == nullptr || N < 0 || H < 1) return MRL_ERR_INVALID_ARG;
  if (!(np->eps > 0.f) || np->eps > 3.4e38f || !(np->weight_offset - np->weight_offset == 0.f)) return MRL_ERR_INVALID_ARG;
  if (np->group != 0 && np->group != 32 && np->group != 64 && np->group != 128 && np->group != 256) return MRL_ERR_INVALID_ARG;
  if (N == 0) return MRL_OK;
  if (h_out == nullptr && y == nullptr && y8 == nullptr && rstd == nullptr) return MRL_ERR_INVALID_ARG;
  if (ld_x < H || (residual != nullptr && ld_res < H) || (h_out != nullptr && ld_h < H) || (y != nullptr && ld_y < H) ||
      (y8 != nullptr && (ld_y8 < H || scales == nullptr)))
    return MRL_ERR_INVALID_ARG;
  if (h_out != nullptr && h_out == y) return MRL_ERR_INVALID_ARG;
  if (x == nullptr || weight == nullptr) return MRL_ERR_INVALID_ARG;
  NormFwdArgs a{x, residual, weight, h_out, y, static_cast<uint8_t*>(y8), scales, rstd, ld_x, ld_res, ld_h, ld_y, ld_y8, N,
                H, np->group, w_dtype == MRL_BF16, np->eps, np->weight_offset, 1.0f / (float)H};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const unsigned grid = (unsigned)(N < 0x7fffffffll ? N : 0x7fffffffll);
  const bool bf16 = dtype == MRL_BF16;
  if (H <= kRowMax) {
    const int bytes = fwd_vector(a, bf16 ? 2 : 4);
    mrl_profile_before(st, "rmsnorm_fwd_row_kernel");
    if (bf16 && bytes == 32) launch_fwd_rows<__nv_bfloat16, 16>(a, grid, st);
    else if (bf16 && bytes == 16) launch_fwd_rows<__nv_bfloat16, 8>(a, grid, st);
    else if (bf16) launch_fwd_rows<__nv_bfloat16, 1>(a, grid, st);
    else if (bytes == 32) launch_fwd_rows<float, 8>(a, grid, st);
    else if (bytes == 16) launch_fwd_rows<float, 4>(a, grid, st);
    else launch_fwd_rows<float, 1>(a, grid, st);
  } else {
    mrl_profile_before(st, "rmsnorm_fwd_loop_kernel");
    if (bf16)
      rmsnorm_fwd_loop_kernel<__nv_bfloat16><<<grid, kLoopThreads, 0, st>>>(a);
    else
      rmsnorm_fwd_loop_kernel<float><<<grid, kLoopThreads, 0, st>>>(a);
  }
  mrl_profile_after(st);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
}

extern "C" int mrl_rmsnorm_residual_bwd(const void* dy, int64_t ld_dy, const void* dh, int64_t ld_dh, const void* h,
                                        int64_t ld_h, int32_t dtype, const void* weight, int32_t w_dtype,
                                        const float* rstd, int64_t N, int32_t H, const mrl_norm_params* np, void* dx,
                                        int64_t ld_dx, float* dweight, void* workspace, size_t workspace_bytes,
                                        void* stream) {
  if (!row_type_ok(dtype) || !row_type_ok(w_dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
  if (np == nullptr || N < 0 || H < 1 || (np->flags & ~MRL_FLAG_ACCUMULATE_DW) != 0) return MRL_ERR_INVALID_ARG;
  if (!(np->weight_offset - np->weight_offset == 0.f)) return MRL_ERR_INVALID_ARG;
  if (ld_dy < H || ld_h < H || ld_dx < H || (dh != nullptr && ld_dh < H)) return MRL_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool accumulate = (np->flags & MRL_FLAG_ACCUMULATE_DW) != 0;
  if (N == 0) {
    if (dweight != nullptr && !accumulate) MRL_CUDA_OK(cudaMemsetAsync(dweight, 0, (size_t)H * 4, st));
    return MRL_OK;
  }
  if (dy == nullptr || h == nullptr || weight == nullptr || rstd == nullptr || dx == nullptr) return MRL_ERR_INVALID_ARG;
  if (dweight != nullptr) {
    if (workspace == nullptr || workspace_bytes < mrl_rmsnorm_bwd_workspace_bytes(N, H)) return MRL_ERR_WORKSPACE_TOO_SMALL;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MRL_ERR_INVALID_ARG;
  }
  const int grid = bwd_ctas(N, H);
  NormBwdArgs a{dy, dh, h, weight, rstd, dx, dweight != nullptr ? static_cast<float*>(workspace) : nullptr, ld_dy, ld_dh,
                ld_h, ld_dx, N, H, w_dtype == MRL_BF16, np->weight_offset, 1.0f / (float)H};
  const bool bf16 = dtype == MRL_BF16;
  if (H <= kRowMax) {
    const int bytes = bwd_vector(a, bf16 ? 2 : 4);
    mrl_profile_before(st, "rmsnorm_bwd_row_kernel");
    if (bf16 && bytes == 32) launch_bwd_rows<__nv_bfloat16, 16>(a, grid, st);
    else if (bf16 && bytes == 16) launch_bwd_rows<__nv_bfloat16, 8>(a, grid, st);
    else if (bf16) launch_bwd_rows<__nv_bfloat16, 1>(a, grid, st);
    else if (bytes == 32) launch_bwd_rows<float, 8>(a, grid, st);
    else if (bytes == 16) launch_bwd_rows<float, 4>(a, grid, st);
    else launch_bwd_rows<float, 1>(a, grid, st);
  } else {
    mrl_profile_before(st, "rmsnorm_bwd_loop_kernel");
    if (bf16)
      rmsnorm_bwd_loop_kernel<__nv_bfloat16><<<grid, kLoopThreads, 0, st>>>(a);
    else
      rmsnorm_bwd_loop_kernel<float><<<grid, kLoopThreads, 0, st>>>(a);
  }
  mrl_profile_after(st);
  MRL_CUDA_OK(cudaGetLastError());
  if (dweight != nullptr) {
    rmsnorm_dw_kernel<<<(H + 31) / 32, 256, 0, st>>>(a.partial, grid, H, dweight, accumulate);
    MRL_CUDA_OK(cudaGetLastError());
  }
  return MRL_OK;
}
