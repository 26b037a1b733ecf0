// Root-mean-square norm with the residual's addition (mrl_rmsnorm_residual_fwd / _bwd): the rows that enter the fused LM
// head, and the way back for its dHidden.
//
// Forward: h = x + r, rstd = 1 / sqrt(mean h^2 + eps), y = h rstd (w + o), optionally as e4m3 codes with a scale per group.
// Backward: with g = (w + o) dy and xhat = h rstd, dx = dh + rstd (g - xhat mean(g xhat)), dw = sum over rows of dy xhat.
// A few operations per element against 6 to 9 bytes: bound by HBM.
#include "mrl_common.cuh"

namespace {

using namespace mrl;

constexpr int kLoopThreads = 512;
constexpr int kBwdCtas = 296;   // CTAs of the backward kernel at most: rows of the dweight partials

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

int bwd_ctas(long long N) { return (int)(N < kBwdCtas ? N : kBwdCtas); }

bool row_type_ok(int32_t dtype) { return dtype == MRL_BF16 || dtype == MRL_F32; }

}  // namespace

size_t mrl_rmsnorm_bwd_workspace_bytes(long long N, int H) {
  if (N <= 0 || H <= 0) return 0;
  return mrl_align_up((size_t)bwd_ctas(N) * (size_t)H * 4, 256);
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
  mrl_profile_before(st, "rmsnorm_fwd_loop_kernel");
  if (dtype == MRL_BF16)
    rmsnorm_fwd_loop_kernel<__nv_bfloat16><<<grid, kLoopThreads, 0, st>>>(a);
  else
    rmsnorm_fwd_loop_kernel<float><<<grid, kLoopThreads, 0, st>>>(a);
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
  const int grid = bwd_ctas(N);
  NormBwdArgs a{dy, dh, h, weight, rstd, dx, dweight != nullptr ? static_cast<float*>(workspace) : nullptr, ld_dy, ld_dh,
                ld_h, ld_dx, N, H, w_dtype == MRL_BF16, np->weight_offset, 1.0f / (float)H};
  mrl_profile_before(st, "rmsnorm_bwd_loop_kernel");
  if (dtype == MRL_BF16)
    rmsnorm_bwd_loop_kernel<__nv_bfloat16><<<grid, kLoopThreads, 0, st>>>(a);
  else
    rmsnorm_bwd_loop_kernel<float><<<grid, kLoopThreads, 0, st>>>(a);
  mrl_profile_after(st);
  MRL_CUDA_OK(cudaGetLastError());
  if (dweight != nullptr) {
    rmsnorm_dw_kernel<<<(H + 31) / 32, 256, 0, st>>>(a.partial, grid, H, dweight, accumulate);
    MRL_CUDA_OK(cudaGetLastError());
  }
  return MRL_OK;
}
