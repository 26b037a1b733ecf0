// Scoring in 8 bits: mrl_e4m3_quantize and mrl_e4m3_product.
#include "mrl_common.cuh"

namespace {

using namespace mrl;

constexpr int kBlock = MRL_SCALE_BLOCK;

template <typename T>
__device__ __forceinline__ float load_f(const T* p);
template <>
__device__ __forceinline__ float load_f<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_f<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_f(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// One CTA per block of `rows` x 128 elements.
template <typename T>
__global__ void __launch_bounds__(256) quantize_kernel(const T* __restrict__ x, long long ld_x, long long N, int H, int rows,
                                                       uint8_t* __restrict__ codes, long long ld_codes, float* __restrict__ scales) {
  __shared__ float red[8];
  const long long row0 = (long long)blockIdx.x * rows;
  const int col = (int)blockIdx.y * kBlock + (threadIdx.x & 127), blocks = (H + kBlock - 1) / kBlock;
  float peak = 0.f;
  for (int r = threadIdx.x >> 7; r < rows; r += 2)
    if (row0 + r < N && col < H) peak = fmaxf(peak, fabsf(load_f<T>(x + (row0 + r) * ld_x + col)));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) peak = fmaxf(peak, __shfl_xor_sync(0xffffffffu, peak, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = peak;
  __syncthreads();
  for (int k = 0; k < 8; ++k) peak = fmaxf(peak, red[k]);
  const float scale = e4m3_scale(peak), inv = 1.0f / scale;
  if (threadIdx.x == 0) scales[(long long)blockIdx.x * blocks + blockIdx.y] = scale;
  for (int r = threadIdx.x >> 7; r < rows; r += 2)
    if (row0 + r < N && col < H)
      codes[(row0 + r) * ld_codes + col] = (uint8_t)pack_e4m3x2(load_f<T>(x + (row0 + r) * ld_x + col) * inv, 0.f);
}

// 64 x 64 outputs per CTA of 256 threads, one block of 128 columns at a time.
template <typename T>
__global__ void __launch_bounds__(256) product_kernel(const uint8_t* __restrict__ x8, long long ld_x, const float* __restrict__ xs,
                                                      const uint8_t* __restrict__ w8, long long ld_w, const float* __restrict__ ws,
                                                      long long N, int H, int V, T* __restrict__ out, long long ld_out) {
  __shared__ float a[64][33], b[64][33];
  const long long row0 = (long long)blockIdx.y * 64;
  const long long col0 = (long long)blockIdx.x * 64;
  const int tr = threadIdx.x >> 4, tc = threadIdx.x & 15, blocks = (H + kBlock - 1) / kBlock;
  float sum[4][4] = {};
  for (int kb = 0; kb < blocks; ++kb) {
    float part[4][4] = {};
    for (int k0 = 0; k0 < kBlock; k0 += 32) {
      __syncthreads();
      for (int i = threadIdx.x; i < 64 * 32; i += 256) {
        const int r = i >> 5, k = kb * kBlock + k0 + (i & 31);
        a[r][i & 31] = row0 + r < N && k < H ? unpack_e4m3x2(x8[(row0 + r) * ld_x + k]).x : 0.f;
        b[r][i & 31] = col0 + r < V && k < H ? unpack_e4m3x2(w8[(col0 + r) * ld_w + k]).x : 0.f;
      }
      __syncthreads();
      for (int k = 0; k < 32; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) part[i][j] = fmaf(a[tr * 4 + i][k], b[tc * 4 + j][k], part[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const long long r = row0 + tr * 4 + i, c = col0 + tc * 4 + j;
        if (r < N && c < V) sum[i][j] = fmaf(xs[r * blocks + kb] * ws[(c / kBlock) * blocks + kb], part[i][j], sum[i][j]);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const long long r = row0 + tr * 4 + i, c = col0 + tc * 4 + j;
      if (r < N && c < V) store_f(out + r * ld_out + c, sum[i][j]);
    }
}

bool row_type_ok(int32_t dtype) { return dtype == MRL_BF16 || dtype == MRL_F32; }
bool on_element(const void* p, int elem) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(elem - 1)) == 0; }

}  // namespace

extern "C" int mrl_e4m3_quantize(const void* x, int64_t ld_x, int32_t dtype, int64_t N, int32_t H, int32_t block_rows, void* codes,
                                 int64_t ld_codes, float* scales, void* stream) {
  if (!row_type_ok(dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
  if (N < 0 || H < 1 || (block_rows != 1 && block_rows != kBlock) || ld_x < H || ld_codes < H) return MRL_ERR_INVALID_ARG;
  if (H > (1 << 30)) return MRL_ERR_UNSUPPORTED_SHAPE;
  if (N == 0) return MRL_OK;
  if (x == nullptr || codes == nullptr || scales == nullptr || codes == x || codes == static_cast<void*>(scales))
    return MRL_ERR_INVALID_ARG;
  if (!on_element(x, dtype == MRL_BF16 ? 2 : 4) || !on_element(scales, 4)) return MRL_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const dim3 grid((unsigned)((N + block_rows - 1) / block_rows), (unsigned)((H + kBlock - 1) / kBlock));
  mrl_profile_before(st, "quantize_kernel");
  if (dtype == MRL_BF16)
    quantize_kernel<<<grid, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(x), ld_x, N, H, block_rows, static_cast<uint8_t*>(codes),
                                          ld_codes, scales);
  else
    quantize_kernel<<<grid, 256, 0, st>>>(static_cast<const float*>(x), ld_x, N, H, block_rows, static_cast<uint8_t*>(codes), ld_codes,
                                          scales);
  mrl_profile_after(st);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
}

extern "C" int mrl_e4m3_product(const void* x8, int64_t ld_x, const float* x_scales, const void* w8, int64_t ld_w,
                                const float* w_scales, int64_t N, int32_t H, int32_t V, int32_t out_dtype, void* out, int64_t ld_out,
                                int32_t* status, void* stream) {
  if (!row_type_ok(out_dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
  if (N < 0 || H < 1 || V < 1 || ld_x < H || ld_w < H || ld_out < V) return MRL_ERR_INVALID_ARG;
  if (H > (1 << 24) || N > 0x7fffffffll) return MRL_ERR_UNSUPPORTED_SHAPE;
  if (N == 0) return MRL_OK;
  if (x8 == nullptr || x_scales == nullptr || w8 == nullptr || w_scales == nullptr || out == nullptr) return MRL_ERR_INVALID_ARG;
  if (!on_element(x8, 16) || !on_element(w8, 16) || (N > 1 && ld_x % 16 != 0) || (V > 1 && ld_w % 16 != 0)) return MRL_ERR_INVALID_ARG;
  if (!on_element(x_scales, 4) || !on_element(w_scales, 4) || !on_element(out, out_dtype == MRL_BF16 ? 2 : 4) || !on_element(status, 4))
    return MRL_ERR_INVALID_ARG;
  if (out == x8 || out == w8 || out == x_scales || out == w_scales) return MRL_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const dim3 grid((unsigned)((V + 63) / 64), (unsigned)((N + 63) / 64));
  mrl_profile_before(st, "product_kernel");
  if (out_dtype == MRL_BF16)
    product_kernel<<<grid, 256, 0, st>>>(static_cast<const uint8_t*>(x8), ld_x, x_scales, static_cast<const uint8_t*>(w8), ld_w,
                                         w_scales, N, H, V, static_cast<__nv_bfloat16*>(out), ld_out);
  else
    product_kernel<<<grid, 256, 0, st>>>(static_cast<const uint8_t*>(x8), ld_x, x_scales, static_cast<const uint8_t*>(w8), ld_w,
                                         w_scales, N, H, V, static_cast<float*>(out), ld_out);
  mrl_profile_after(st);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
}
