// Root-mean-square norm with the residual's addition (mrl_rmsnorm_residual_fwd / _bwd): the rows that enter the fused LM
// head, and the way back for its dHidden.
//
// Forward: h = x + r, rstd = 1 / sqrt(mean h^2 + eps), y = h rstd (w + o), optionally as e4m3 codes with a scale per group.
// Backward: with g = (w + o) dy and xhat = h rstd, dx = dh + rstd (g - xhat mean(g xhat)), dw = sum over rows of dy xhat.
// A few operations per element against 6 to 9 bytes: bound by HBM where rows are whole 16-byte granules (65,536 x 4,096 bf16:
// forward with residual 334-339 us, backward 340-349 us, 6.1-6.4 TB/s of the bytes that have to move; e4m3 codes beside y, 33,880
// rows: 204-209 us, 6.1 TB/s), by the instructions' issue where they are not (65,552 x 4,095: 553 and 537 us).
#include <type_traits>

#include "mrl_common.cuh"

namespace {

using namespace mrl;

constexpr int kSms = 148;
constexpr int kLoopThreads = 512;
constexpr int kWide = 32, kMiddle = 16, kNarrow = 8;      // columns of a thread of the row kernels
constexpr int kNoCodes = 0, kRowCodes = 1, kGroupCodes = 2;
constexpr int kRowMax = 16384;                            // the widest row that one CTA holds
// registers of a thread of the row kernels
constexpr int kBwdRegs = 64, kBwdRegsMore = 80;
// (wide: shared memory allows no more CTAs anyway; codes by group spill 24 to 32 bytes at 80, 8 to 12 at 96: 33,880 rows of 4,096 208 us, with 80 216; 65,536 of
// 2,048 166 and 174, but without a residual 118 and 115, and with one scale a row 170 and 167)
constexpr int fwd_regs(int cols, int codes) { return cols != kWide ? 64 : (codes == kGroupCodes ? 96 : 80); }

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
  int stages;  // rows on their way or worked on (row kernels)
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
  int stages;
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
  let_next_start();
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

__device__ __forceinline__ float abs_max(float m, f2 v) {
  const float2 u = split_f2(v);
  return fmaxf(m, fmaxf(fabsf(u.x), fabsf(u.y)));
}

// The unit of work of the row kernels: 16 adjacent bytes of a row (whole granules), or two elements 32 columns apart.
template <typename T, bool kOdd>
struct Unit {
  static constexpr int kCols = kOdd ? 2 : 16 / (int)sizeof(T);  // columns
  static constexpr int kPairs = kCols / 2;
  static constexpr int kStep = 32 * kCols;                      // columns of a warp
  f2 p[kPairs];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < kPairs; ++k) p[k] = 0ull;
  }
  // from 16 bytes
  __device__ __forceinline__ void set(uint4 q) {
    if constexpr (sizeof(T) == 4) {
      p[0] = make_f2(__uint_as_float(q.x), __uint_as_float(q.y));
      p[1] = make_f2(__uint_as_float(q.z), __uint_as_float(q.w));
    } else if constexpr (!kOdd) {
      p[0] = bf16x2_to_f2(q.x), p[1] = bf16x2_to_f2(q.y), p[2] = bf16x2_to_f2(q.z), p[3] = bf16x2_to_f2(q.w);
    }
  }
  __device__ __forceinline__ uint4 bits() const {
    if constexpr (sizeof(T) == 4) {
      const float2 a = split_f2(p[0]), b = split_f2(p[1 % kPairs]);
      return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    } else {
      return make_uint4(f2_to_bf16x2(p[0]), f2_to_bf16x2(p[1 % kPairs]), f2_to_bf16x2(p[2 % kPairs]), f2_to_bf16x2(p[3 % kPairs]));
    }
  }
  // `at`: the unit's place in shared memory; in0 / in1: its first / second half lies inside the row
  __device__ __forceinline__ void load(const char* at, bool in0, bool in1) {
    if constexpr (!kOdd) {
      if (in0) set(*reinterpret_cast<const uint4*>(at)); else zero();
    } else {
      const T* e = reinterpret_cast<const T*>(at);
      p[0] = make_f2(in0 ? load_f(e) : 0.f, in1 ? load_f(e + 32) : 0.f);
    }
  }
  // to the unit's place in a row
  __device__ __forceinline__ void store(T* to, bool in0, bool in1) const {
    if constexpr (!kOdd) {
      if (in0) *reinterpret_cast<uint4*>(to) = bits();
    } else {
      const float2 u = split_f2(p[0]);
      if (in0) store_f(to, u.x);
      if (in1) store_f(to + 32, u.y);
    }
  }
};

// The gains (weight + offset) of the unit at column c, 0 behind the row; the weight stays in L1.
template <typename U, bool kOdd, typename W>
__device__ __forceinline__ void load_gain(const W* w, float offset, int c, bool in0, bool in1, U* g) {
  const W* p = w + c;
  const f2 o2 = make_f2(offset, offset);
  if constexpr (kOdd) {
    float a = 0.f, b = 0.f;
    if constexpr (sizeof(W) == 2) {
      if (in0) a = bf16lo_to_f32(__ldg(reinterpret_cast<const uint16_t*>(p)));
      if (in1) b = bf16lo_to_f32(__ldg(reinterpret_cast<const uint16_t*>(p) + 32));
    } else {
      if (in0) a = __ldg(p);
      if (in1) b = __ldg(p + 32);
    }
    g->p[0] = make_f2(a, b);
  } else {
    g->zero();
    if (in0) {
      if constexpr (sizeof(W) == 2) {
#pragma unroll
        for (int k = 0; k < U::kPairs / 2; ++k) {
          const uint2 q = __ldg(reinterpret_cast<const uint2*>(p) + k);
          g->p[2 * k] = bf16x2_to_f2(q.x);
          g->p[2 * k + 1] = bf16x2_to_f2(q.y);
        }
      } else {
#pragma unroll
        for (int k = 0; k < U::kPairs / 2; ++k) {
          const float4 q = __ldg(reinterpret_cast<const float4*>(p) + k);
          g->p[2 * k] = make_f2(q.x, q.y);
          g->p[2 * k + 1] = make_f2(q.z, q.w);
        }
      }
    }
  }
  if (offset != 0.f) {
#pragma unroll
    for (int k = 0; k < U::kPairs; ++k) g->p[k] = add_f2(g->p[k], o2);
  }
}

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes from global to shared memory without a register; reads the first `bytes` of them, zeros for the rest
__device__ __forceinline__ void copy_async(void* dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// waits until at most `newer` of the thread's later groups are still under way
__device__ __forceinline__ void copy_wait(int newer) {
  switch (newer) {
    case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
    case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
    case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
    default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
  }
}

// Where a row's bytes lie in a copy of the 16-byte granules that hold them (rows of any alignment).
struct Image {
  const char* first;  // granule with the row's first byte
  int off, len;       // first byte inside it; bytes of the row
};
template <typename P>
__device__ __forceinline__ Image image_of(const P* base, long long element, int H) {
  const char* p = reinterpret_cast<const char*>(base + element);
  const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15);
  return Image{p - off, off, H * (int)sizeof(P)};
}
// Granules of a row into its copy.  Bytes before the row come along where it starts inside a granule, but none from before
// the tensor (the first row, or the first few of less than a granule); nothing behind the row's end is read.
template <typename T>
__device__ __forceinline__ void image_load(char* dst, const Image& im, const T* base) {
  const int end = im.off + im.len;
  const bool by_element = im.first < reinterpret_cast<const char*>(base);
  for (int k = threadIdx.x + by_element; 16 * k < end; k += blockDim.x) copy_async(dst + 16 * k, im.first + 16 * k, min(16, end - 16 * k));
  if (by_element) {
    const int b = im.off + (int)threadIdx.x * (int)sizeof(T);
    if (b < min(16, end)) *reinterpret_cast<T*>(dst + b) = *reinterpret_cast<const T*>(im.first + b);
  }
}
// A magnitude as an ordered integer, 0 for NaN.
__device__ __forceinline__ uint32_t peak_bits(float v) { return __float_as_uint(fmaxf(fabsf(v), 0.f)); }
__host__ __device__ __forceinline__ int image_bytes(int H, int elem) { return (H * elem + 30) / 16 * 16; }

// Sum / maximum of non-negative values over the CTA in a fixed order: one barrier, none for a single warp.  `red` holds 32 floats,
// 0 where there is no warp, and is not written again before another barrier.
template <bool kMax>
__device__ __forceinline__ float row_reduce(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, v, o);
    v = kMax ? fmaxf(v, u) : v + u;
  }
  if (blockDim.x == 32) {
    __syncwarp();
    return v;
  }
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  const float4* q = reinterpret_cast<const float4*>(red);
  float4 s = q[0];
  const auto more = [&](int from, int to) {
#pragma unroll
    for (int k = from; k < to; ++k) {
      const float4 u = q[k];
      s.x = kMax ? fmaxf(s.x, u.x) : s.x + u.x;
      s.y = kMax ? fmaxf(s.y, u.y) : s.y + u.y;
      s.z = kMax ? fmaxf(s.z, u.z) : s.z + u.z;
      s.w = kMax ? fmaxf(s.w, u.w) : s.w + u.w;
    }
  };
  if (blockDim.x > 128) more(1, 2);
  if (blockDim.x > 256) more(2, 4);
  if (blockDim.x > 512) more(4, 8);
  return kMax ? fmaxf(fmaxf(s.x, s.y), fmaxf(s.z, s.w)) : (s.x + s.y) + (s.z + s.w);
}

// Rows of up to kRowMax columns, each read once and written once.  A CTA walks rows blockIdx.x, + gridDim.x, ...; the rows to
// come are under way into shared memory (`stages` of them, 16-byte asynchronous copies), so the bytes in flight do not
// depend on registers.  kOdd = false: rows of 16-byte granules; a thread copies the granules whose columns it works on
// and needs no barrier to read them.  kOdd = true: rows of any alignment; the granules are copied as they lie and read by
// column after a barrier; outputs go from registers to their rows by element (32,776 x 4,095 float32: 429 us, through shared
// memory 484; bf16 of 61, 4,095, 8,191 columns: 140, 553, 610 us, 189, 563, 592).
// Columns: a warp owns 32 * kRowCols adjacent ones, unit u of a lane lies u * kStep behind its first.  A warp whose columns
// all lie inside the row runs without tests (kFull).
// kCodes: what of y8 there is (its code costs registers): nothing, one scale a row, one a group.
template <typename T, bool kOdd, int kRowCols, int kCodes>
__global__ void __maxnreg__(fwd_regs(kRowCols, kCodes)) rmsnorm_fwd_row_kernel(const __grid_constant__ NormFwdArgs a) {
  using U = Unit<T, kOdd>;
  constexpr int kUnits = kRowCols / U::kCols, kStep = U::kStep, kPairs = U::kPairs, kHalf = kOdd ? 32 : 0;
  extern __shared__ __align__(16) char smem[];
  __shared__ __align__(16) float red[2][4][32];
  __shared__ uint32_t peak[kRowMax / 32];
  const int tid = threadIdx.x, nt = blockDim.x;
  const int c0 = (tid >> 5) * (kUnits * kStep) + (tid & 31) * (kOdd ? 1 : U::kCols);
  const bool full = ((tid >> 5) + 1) * (kUnits * kStep) <= a.H;
  const int slot = kOdd ? image_bytes(a.H, sizeof(T)) : nt * kRowCols * (int)sizeof(T);
  const int stage = a.res != nullptr ? 2 * slot : slot;
  const int group = a.group > 0 ? a.group : a.H, groups = (a.H + group - 1) / group;
  // lanes whose columns share a scale sit side by side; more than a warp of them meet in shared memory
  const bool meet = kCodes == kGroupCodes && a.group > (kOdd ? 32 : kStep);
  for (int k = tid; k < 256; k += nt) (&red[0][0][0])[k] = 0.f;
  __syncthreads();

  const auto fetch = [&](long long row, int s) {
    if (row < a.N) {
      char* dst = smem + s * stage;
      const T* x = static_cast<const T*>(a.x);
      const T* r = static_cast<const T*>(a.res);
      if constexpr (kOdd) {
        image_load<T>(dst, image_of(x, row * a.ld_x, a.H), x);
        if (r != nullptr) image_load<T>(dst + slot, image_of(r, row * a.ld_res, a.H), r);
      } else {
        dst += tid * 16;
        x += row * a.ld_x + c0;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
          if (full || c0 + u * kStep < a.H) copy_async(dst + u * nt * 16, x + u * kStep, 16);
        if (r != nullptr) {
          r += row * a.ld_res + c0;
#pragma unroll
          for (int u = 0; u < kUnits; ++u)
            if (full || c0 + u * kStep < a.H) copy_async(dst + slot + u * nt * 16, r + u * kStep, 16);
        }
      }
    }
    copy_commit();
  };

  for (int s = 0; s + 1 < a.stages; ++s) fetch(blockIdx.x + (long long)s * gridDim.x, s);
  int s = 0, turn = 0;
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x, turn ^= 1) {
    if (kOdd) {
      // the copies of this row are there for all, and those of the last row have been read by all
      if (a.stages > 1) copy_wait(a.stages - 2);
      __syncthreads();
      fetch(row + (long long)(a.stages - 1) * gridDim.x, s == 0 ? a.stages - 1 : s - 1);
      if (a.stages == 1) {
        copy_wait(0);
        __syncthreads();
      }
    } else {
      fetch(row + (long long)(a.stages - 1) * gridDim.x, s == 0 ? a.stages - 1 : s - 1);
      copy_wait(a.stages - 1);
    }
    char* here = smem + s * stage;
    const char* in_x = here + (kOdd ? c0 * (int)sizeof(T) : tid * 16);
    const char* in_r = in_x + slot;
    if (kOdd) {
      in_x += image_of(static_cast<const T*>(a.x), row * a.ld_x, a.H).off;
      in_r += image_of(static_cast<const T*>(a.res), row * a.ld_res, a.H).off;
    }
    s = s + 1 == a.stages ? 0 : s + 1;
    const int unit_bytes = kOdd ? kStep * (int)sizeof(T) : nt * 16;

    U h[kUnits];
    f2 acc[2] = {0ull, 0ull};
    const auto read = [&](auto all) {
      constexpr bool kFull = decltype(all)::value;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const bool in0 = kFull || c0 + u * kStep < a.H, in1 = kFull || c0 + u * kStep + kHalf < a.H;
        h[u].load(in_x + u * unit_bytes, in0, in1);
        if (a.res != nullptr) {
          U r;
          r.load(in_r + u * unit_bytes, in0, in1);
#pragma unroll
          for (int k = 0; k < kPairs; ++k) h[u].p[k] = add_f2(h[u].p[k], r.p[k]);
        }
#pragma unroll
        for (int k = 0; k < kPairs; ++k) acc[(u * kPairs + k) & 1] = fma_f2(h[u].p[k], h[u].p[k], acc[(u * kPairs + k) & 1]);
      }
    };
    if (full) read(std::true_type{}); else read(std::false_type{});
    if (meet)
      for (int k = tid; k < groups; k += nt) peak[k] = 0;
    const float2 part = split_f2(add_f2(acc[0], acc[1]));
    const float ss = row_reduce<false>(part.x + part.y, red[turn][0]);
    float rstd = rsqrtf(fmaf(ss, a.inv_h, a.eps));
    if (ss == INFINITY) {  // the squares may have left float32 although the row has not
      float m = 0.f;
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int k = 0; k < kPairs; ++k) m = abs_max(m, h[u].p[k]);
      m = row_reduce<true>(m, red[turn][1]);
      if (m < INFINITY) {
        const float f = scalbnf(1.f, -ilogbf(m));
        float q = 0.f;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
          for (int k = 0; k < kPairs; ++k) {
            const float2 v = split_f2(h[u].p[k]);
            q = fmaf(v.x * f, v.x * f, fmaf(v.y * f, v.y * f, q));
          }
        q = row_reduce<false>(q, red[turn][2]);
        rstd = f * rsqrtf(fmaf(q, a.inv_h, a.eps * f * f));
      }
    }
    if (tid == 0 && a.rstd != nullptr) a.rstd[row] = rstd;

    const f2 rstd2 = make_f2(rstd, rstd);
    T* to_h = static_cast<T*>(a.h_out) + row * a.ld_h + c0;
    T* to_y = static_cast<T*>(a.y) + row * a.ld_y + c0;
    const auto write = [&](auto all, auto w) {
      constexpr bool kFull = decltype(all)::value;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const bool in0 = kFull || c0 + u * kStep < a.H, in1 = kFull || c0 + u * kStep + kHalf < a.H;
        if (a.h_out != nullptr) h[u].store(to_h + u * kStep, in0, in1);
        U g;
        load_gain<U, kOdd>(w, a.offset, c0 + u * kStep, in0, in1, &g);
#pragma unroll
        for (int k = 0; k < kPairs; ++k) h[u].p[k] = mul_f2(mul_f2(h[u].p[k], rstd2), g.p[k]);
        if (a.y != nullptr) h[u].store(to_y + u * kStep, in0, in1);
      }
    };
    if (a.w_bf16) {
      if (full) write(std::true_type{}, static_cast<const __nv_bfloat16*>(a.w));
      else write(std::false_type{}, static_cast<const __nv_bfloat16*>(a.w));
    } else {
      if (full) write(std::true_type{}, static_cast<const float*>(a.w));
      else write(std::false_type{}, static_cast<const float*>(a.w));
    }

    if constexpr (kCodes != kNoCodes) {
      const int shift = 31 - __clz(group);  // of a group that is a power of two
      float row_inv = 0.f;
      if constexpr (kCodes == kRowCodes) {
        float top = 0.f;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
          for (int k = 0; k < kPairs; ++k) top = abs_max(top, h[u].p[k]);
        const float scale = e4m3_scale(row_reduce<true>(top, red[turn][3]));
        if (tid == 0) a.scales[row] = scale;
        row_inv = __fdividef(1.f, scale);
      } else if (meet) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          const int c = c0 + u * kStep;
          if constexpr (kOdd) {
            const float2 v = split_f2(h[u].p[0]);
            const uint32_t m0 = __reduce_max_sync(0xffffffffu, peak_bits(v.x)), m1 = __reduce_max_sync(0xffffffffu, peak_bits(v.y));
            if ((tid & 31) == 0 && c < a.H) atomicMax(&peak[c >> shift], m0);
            if ((tid & 31) == 0 && c + 32 < a.H) atomicMax(&peak[(c + 32) >> shift], m1);
          } else {
            float m = 0.f;
#pragma unroll
            for (int k = 0; k < kPairs; ++k) m = abs_max(m, h[u].p[k]);
            const uint32_t m0 = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
            if ((tid & 31) == 0 && c < a.H) atomicMax(&peak[c >> shift], m0);
          }
        }
        __syncthreads();
      }
      float* scales = a.scales + row * groups;
      uint8_t* q = a.y8 + row * a.ld_y8 + c0;
      // unit u as codes; inv0, inv1: 1 / scale of columns c on, and in odd rows of column c + 32
      const auto put_codes = [&](int u, float inv0, float inv1) {
        const int c = c0 + u * kStep;
        if constexpr (kOdd) {
          const float2 v = split_f2(h[u].p[0]);
          const uint32_t code = pack_e4m3x2(v.x * inv0, v.y * inv1);
          if (c < a.H) q[u * kStep] = (uint8_t)code;
          if (c + 32 < a.H) q[u * kStep + 32] = (uint8_t)(code >> 8);
        } else if (full || c < a.H) {
          uint32_t o[kPairs / 2];
          const f2 i2 = make_f2(inv0, inv0);
#pragma unroll
          for (int k = 0; k < kPairs / 2; ++k) {
            const float2 v = split_f2(mul_f2(h[u].p[2 * k], i2)), w = split_f2(mul_f2(h[u].p[2 * k + 1], i2));
            o[k] = pack_e4m3x2(v.x, v.y) | pack_e4m3x2(w.x, w.y) << 16;
          }
          if constexpr (kPairs == 4)
            *reinterpret_cast<uint2*>(q + u * kStep) = make_uint2(o[0], o[1]);
          else
            *reinterpret_cast<uint32_t*>(q + u * kStep) = o[0];
        }
      };
      // all units, from the maxima of their groups (of the lane's own columns in, of the group out)
      const auto by_group = [&](auto peak_of) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          const int c = c0 + u * kStep;
          float m0 = 0.f, m1 = 0.f;
          if constexpr (kOdd) {
            const float2 v = split_f2(h[u].p[0]);
            m0 = fmaxf(fabsf(v.x), 0.f), m1 = fmaxf(fabsf(v.y), 0.f);
          } else {
#pragma unroll
            for (int k = 0; k < kPairs; ++k) m0 = abs_max(m0, h[u].p[k]);
          }
          m0 = e4m3_scale(peak_of(m0, c));
          if (kOdd) m1 = e4m3_scale(peak_of(m1, c + 32));
          if (c < a.H && (c & (group - 1)) == 0) scales[c >> shift] = m0;
          if (kOdd && c + 32 < a.H && ((c + 32) & (group - 1)) == 0) scales[(c + 32) >> shift] = m1;
          put_codes(u, __fdividef(1.f, m0), kOdd ? __fdividef(1.f, m1) : 0.f);
        }
      };
      // the lanes that share a scale with this one
      const int lanes = kOdd ? 32 : min(32, max(1, group / U::kCols));
      const uint32_t beside = (lanes < 32 ? (1u << lanes) - 1u : 0xffffffffu) << ((tid & 31) & ~(lanes - 1));
      if constexpr (kCodes == kRowCodes) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) put_codes(u, row_inv, row_inv);
      } else if (meet) {
        by_group([&](float, int c) { return c < a.H ? __uint_as_float(peak[c >> shift]) : 0.f; });
      } else if (lanes >= 16) {
        // one instruction per set of lanes (65,536 x 4,096 bf16 with groups of 256, 128 and 32 columns: 317, 332 and 379 us, by
        // shuffles 365, 358 and 350)
        by_group([&](float m, int) { return __uint_as_float(__reduce_max_sync(beside, __float_as_uint(m))); });
      } else {
        by_group([&](float m, int) {
          for (int o = lanes >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
          return m;
        });
      }
    }
    if (!kOdd && meet) {
      __syncthreads();  // the next row clears the peaks
    }
  }
}

// Backward, with rows on their way as above.  Each thread keeps the dweight sums of its columns in registers over all of
// the CTA's rows and writes them once; (w + o) dy stays there from the row's sum on, h and dh are read from shared memory
// after it.
template <typename T, bool kOdd, int kRowCols, int kRegs>
__global__ void __maxnreg__(kRegs) rmsnorm_bwd_row_kernel(const __grid_constant__ NormBwdArgs a) {
  using U = Unit<T, kOdd>;
  constexpr int kUnits = kRowCols / U::kCols, kStep = U::kStep, kPairs = U::kPairs, kHalf = kOdd ? 32 : 0;
  extern __shared__ __align__(16) char smem[];
  __shared__ __align__(16) float red[2][32];
  const int tid = threadIdx.x, nt = blockDim.x;
  const int c0 = (tid >> 5) * (kUnits * kStep) + (tid & 31) * (kOdd ? 1 : U::kCols);
  const bool full = ((tid >> 5) + 1) * (kUnits * kStep) <= a.H;
  const int slot = kOdd ? image_bytes(a.H, sizeof(T)) : nt * kRowCols * (int)sizeof(T);
  const int stage = a.dh != nullptr ? 3 * slot : 2 * slot;
  let_next_start();
  for (int k = tid; k < 64; k += nt) (&red[0][0])[k] = 0.f;
  __syncthreads();

  const auto fetch = [&](long long row, int s) {
    if (row < a.N) {
      char* dst = smem + s * stage;
      const void* const from[3] = {a.dy, a.h, a.dh};
      const long long ld[3] = {a.ld_dy, a.ld_h, a.ld_dh};
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        if (from[k] == nullptr) continue;
        const T* p = static_cast<const T*>(from[k]);
        if constexpr (kOdd) {
          image_load<T>(dst + k * slot, image_of(p, row * ld[k], a.H), p);
        } else {
          p += row * ld[k] + c0;
#pragma unroll
          for (int u = 0; u < kUnits; ++u)
            if (full || c0 + u * kStep < a.H) copy_async(dst + k * slot + (u * nt + tid) * 16, p + u * kStep, 16);
        }
      }
    }
    copy_commit();
  };

  f2 dw[kUnits][kPairs];
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int k = 0; k < kPairs; ++k) dw[u][k] = 0ull;
  for (int s = 0; s + 1 < a.stages; ++s) fetch(blockIdx.x + (long long)s * gridDim.x, s);
  int s = 0, turn = 0;
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x, turn ^= 1) {
    const float rstd = a.rstd[row];
    if (kOdd) {  // as in the forward kernel
      if (a.stages > 1) copy_wait(a.stages - 2);
      __syncthreads();
      fetch(row + (long long)(a.stages - 1) * gridDim.x, s == 0 ? a.stages - 1 : s - 1);
      if (a.stages == 1) {
        copy_wait(0);
        __syncthreads();
      }
    } else {
      fetch(row + (long long)(a.stages - 1) * gridDim.x, s == 0 ? a.stages - 1 : s - 1);
      copy_wait(a.stages - 1);
    }
    const char* in_d = smem + s * stage + (kOdd ? c0 * (int)sizeof(T) : tid * 16);
    const char *in_h = in_d + slot, *in_e = in_h + slot;
    if (kOdd) {
      in_d += image_of(static_cast<const T*>(a.dy), row * a.ld_dy, a.H).off;
      in_h += image_of(static_cast<const T*>(a.h), row * a.ld_h, a.H).off;
      in_e += image_of(static_cast<const T*>(a.dh), row * a.ld_dh, a.H).off;
    }
    s = s + 1 == a.stages ? 0 : s + 1;
    const int unit_bytes = kOdd ? kStep * (int)sizeof(T) : nt * 16;

    const f2 rstd2 = make_f2(rstd, rstd);
    f2 gd[kUnits][kPairs], acc[2] = {0ull, 0ull};  // (w + o) dy
    const auto read = [&](auto all, auto w) {
      constexpr bool kFull = decltype(all)::value;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const bool in0 = kFull || c0 + u * kStep < a.H, in1 = kFull || c0 + u * kStep + kHalf < a.H;
        U d, x, g;
        d.load(in_d + u * unit_bytes, in0, in1);
        x.load(in_h + u * unit_bytes, in0, in1);
        load_gain<U, kOdd>(w, a.offset, c0 + u * kStep, in0, in1, &g);
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
          const f2 xhat = mul_f2(x.p[k], rstd2);
          gd[u][k] = mul_f2(d.p[k], g.p[k]);
          dw[u][k] = fma_f2(d.p[k], xhat, dw[u][k]);
          acc[k & 1] = fma_f2(gd[u][k], xhat, acc[k & 1]);
        }
      }
    };
    if (a.w_bf16) {
      if (full) read(std::true_type{}, static_cast<const __nv_bfloat16*>(a.w));
      else read(std::false_type{}, static_cast<const __nv_bfloat16*>(a.w));
    } else {
      if (full) read(std::true_type{}, static_cast<const float*>(a.w));
      else read(std::false_type{}, static_cast<const float*>(a.w));
    }
    const float2 part = split_f2(add_f2(acc[0], acc[1]));
    const float mean = row_reduce<false>(part.x + part.y, red[turn]) * a.inv_h;

    T* out = static_cast<T*>(a.dx) + row * a.ld_dx + c0;
    const f2 minus2 = make_f2(-rstd * mean, -rstd * mean);
    const auto write = [&](auto all) {
      constexpr bool kFull = decltype(all)::value;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const bool in0 = kFull || c0 + u * kStep < a.H, in1 = kFull || c0 + u * kStep + kHalf < a.H;
        U d, x;
        x.load(in_h + u * unit_bytes, in0, in1);
#pragma unroll
        for (int k = 0; k < kPairs; ++k) d.p[k] = fma_f2(x.p[k], minus2, gd[u][k]);
        if (a.dh != nullptr) {
          x.load(in_e + u * unit_bytes, in0, in1);
#pragma unroll
          for (int k = 0; k < kPairs; ++k) d.p[k] = fma_f2(d.p[k], rstd2, x.p[k]);
        } else {
#pragma unroll
          for (int k = 0; k < kPairs; ++k) d.p[k] = mul_f2(d.p[k], rstd2);
        }
        d.store(out + u * kStep, in0, in1);
      }
    };
    if (full) write(std::true_type{}); else write(std::false_type{});
  }
  if (a.partial != nullptr) {
    float* to = a.partial + (size_t)blockIdx.x * a.H + c0;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int c = c0 + u * kStep;
      if constexpr (kOdd) {
        const float2 v = split_f2(dw[u][0]);
        if (c < a.H) to[u * kStep] = v.x;
        if (c + 32 < a.H) to[u * kStep + 32] = v.y;
      } else if (c < a.H) {
#pragma unroll
        for (int k = 0; k < kPairs; k += 2) {
          const float2 v = split_f2(dw[u][k]), w = split_f2(dw[u][k + 1]);
          *reinterpret_cast<float4*>(to + u * kStep + 2 * k) = make_float4(v.x, v.y, w.x, w.y);
        }
      }
    }
  }
}

// dweight[i] = sum over the CTAs' partials, in their order within each of 32 lanes and then over the lanes.
__global__ void __launch_bounds__(1024) rmsnorm_dw_kernel(const float* partial, int rows, int H, float* dw, bool accumulate) {
  __shared__ float red[32][33];
  const int x = threadIdx.x & 31, lane = threadIdx.x >> 5, col = blockIdx.x * 32 + x;
  wait_for_previous();
  float s = 0.f;
  if (col < H) {
    int k = lane;
    for (; k + 96 < rows; k += 128) {  // four loads under way
      const float a = partial[(size_t)k * H + col], b = partial[(size_t)(k + 32) * H + col];
      const float c = partial[(size_t)(k + 64) * H + col], d = partial[(size_t)(k + 96) * H + col];
      s += a, s += b, s += c, s += d;
    }
    for (; k < rows; k += 32) s += partial[(size_t)k * H + col];
  }
  red[lane][x] = s;
  __syncthreads();
  // a warp adds up one column: 32 lanes in a tree
  float t = red[x][lane];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  const int out = blockIdx.x * 32 + lane;
  if (x == 0 && out < H) dw[out] = accumulate ? dw[out] + t : t;
}

int row_threads(int H, int cols) { return (H + cols * 32 - 1) / (cols * 32) * 32; }
// Columns of a thread.  Few rows, or short ones, are spread over more threads (one row of 4,096: 2.5 us with 8 columns, 3.4
// with 32; 262,144 rows of 64: 93 us with 8, 133 with 16).  Forward, 32 columns are fastest for rows of 2 to 16 KB in 16-byte
// granules once there are many (65,536 x 4,096 bf16: 341 us with 32, 374 with 16; 32,768 x 8,192: 338, 357), 16 for wider rows
// (16,384 x 16,384: 356, 339), for fewer (1,024 x 4,096: 8.9, 7.6) and for odd ones (65,552 x 4,095: 557 us, 624 with 8).  Backward,
// whose sums take registers, 16 (65,536 x 4,096, before the registers of launch_bwd_rows: 394 with 32, 367 with 16).
bool few_or_short(long long N, int H) { return H <= 512 || (H <= 512 * kNarrow && N <= 2 * kSms); }
int fwd_cols(long long N, int H, int elem, bool odd) {
  if (few_or_short(N, H)) return kNarrow;
  return !odd && N > 2048 && H * elem >= 2048 && H * elem <= 16384 ? kWide : kMiddle;
}
int bwd_cols(long long N, int H) { return few_or_short(N, H) ? kNarrow : kMiddle; }

bool aligned(const void* p, long long ld, int elem, int bytes) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0 && (ld * elem) % bytes == 0);
}

// How a row kernel is launched.  CTAs per SM: as many as their registers allow and as leave each at least `rows` rows in shared
// memory; stages: what fits then, 4 at most.
struct RowPlan {
  int threads, ctas_per_sm, stages, smem;
};
constexpr int kSmemPerSm = 227 * 1024, kSmemCta = 227 * 1024 - 4096;  // (4 KB: the kernels' own arrays and the system's)
RowPlan plan_rows(int threads, int regs, int stage_bytes, int rows = 2) {
  RowPlan p;
  p.threads = threads;
  int c = 4 * (16384 / (regs * 32)) / (threads / 32);  // (each quarter of the SM holds whole warps)
  if (c > 32) c = 32;
  if (c < 1) c = 1;
  const int own = 4096;
  while (c > 1 && c * (rows * stage_bytes + own) > kSmemPerSm) --c;
  const int s = stage_bytes > 0 ? (kSmemPerSm / c - own) / stage_bytes : 1;
  p.stages = s > 4 ? 4 : (s < 1 ? 1 : s);
  p.ctas_per_sm = c;
  p.smem = p.stages * stage_bytes;
  return p;
}
// CTAs of the backward kernels, and rows of dweight partials; the most that any alignment and type of the rows leads to.
// Four rows a CTA at least once every SM has one: the partials cost as much as rows.
int bwd_ctas(long long N, int per_sm) {
  const long long most = (long long)kSms * per_sm, few = N / 4 > kSms ? N / 4 : kSms;
  return (int)(N < few ? N : (few < most ? few : most));
}
int bwd_ctas_most(long long N, int H) { return bwd_ctas(N, H <= kRowMax ? plan_rows(row_threads(H, kMiddle), kBwdRegs, 0).ctas_per_sm : 2); }

// Forward, two tensors in and no codes out: where a tensor does not fit L2, fewer CTAs with three rows each are faster (65,536 x
// 4,096 bf16: 352 us with two rows, 337 with three, 355 with four; 131,072 x 2,048: 364, 344, 357), but not where it does (8,192 x
// 4,096: 45.2, 46.3), nor where three rows leave less than three CTAs (49,152 x 6,144: 384, 393), nor for the others (e4m3 codes
// beside y: 335, 371; backward 343, 388).
constexpr long long kFewerBytes = 100000000;
constexpr int kFewerStage = 20480;

template <typename K>
int allow_smem(K kernel, std::atomic<uint64_t>& done) {
  return mrl_once_per_device(done, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemCta); });
}
// One row of everything that is read fits a CTA, at most: three float32 rows of kRowMax columns off the granule (image_bytes).
static_assert(3 * (kRowMax * 4 + 16) <= kSmemCta, "rows of the row kernels");
template <typename T, bool kOdd, int kCols, int kCodes>
int launch_fwd_codes(NormFwdArgs a, cudaStream_t st) {
  const int threads = row_threads(a.H, kCols);
  const int slot = kOdd ? image_bytes(a.H, sizeof(T)) : threads * kCols * (int)sizeof(T);
  const int stage = (a.res != nullptr ? 2 : 1) * slot;
  const bool fewer = !kOdd && kCodes == kNoCodes && a.res != nullptr && stage <= kFewerStage && a.N * a.H >= kFewerBytes / (int)sizeof(T);
  const RowPlan p = plan_rows(threads, fwd_regs(kCols, kCodes), stage, fewer ? 3 : 2);
  a.stages = p.stages;
  const long long most = (long long)kSms * p.ctas_per_sm;
  static std::atomic<uint64_t> done;
  const int rc = allow_smem(rmsnorm_fwd_row_kernel<T, kOdd, kCols, kCodes>, done);
  if (rc != MRL_OK) return rc;
  mrl_profile_before(st, "rmsnorm_fwd_row_kernel");
  rmsnorm_fwd_row_kernel<T, kOdd, kCols, kCodes><<<(unsigned)(a.N < most ? a.N : most), p.threads, p.smem, st>>>(a);
  mrl_profile_after(st);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
}
template <typename T, bool kOdd, int kCols>
int launch_fwd_rows(const NormFwdArgs& a, cudaStream_t st) {
  if (a.y8 == nullptr) return launch_fwd_codes<T, kOdd, kCols, kNoCodes>(a, st);
  return a.group == 0 ? launch_fwd_codes<T, kOdd, kCols, kRowCodes>(a, st) : launch_fwd_codes<T, kOdd, kCols, kGroupCodes>(a, st);
}
template <typename T, bool kOdd, int kCols, int kRegs>
int launch_bwd_regs(NormBwdArgs a, int* ctas, cudaStream_t st) {
  const int threads = row_threads(a.H, kCols);
  const int slot = kOdd ? image_bytes(a.H, sizeof(T)) : threads * kCols * (int)sizeof(T);
  const RowPlan p = plan_rows(threads, kRegs, (a.dh != nullptr ? 3 : 2) * slot);
  a.stages = p.stages;
  *ctas = bwd_ctas(a.N, p.ctas_per_sm);
  static std::atomic<uint64_t> done;
  const int rc = allow_smem(rmsnorm_bwd_row_kernel<T, kOdd, kCols, kRegs>, done);
  if (rc != MRL_OK) return rc;
  mrl_profile_before(st, "rmsnorm_bwd_row_kernel");
  rmsnorm_bwd_row_kernel<T, kOdd, kCols, kRegs><<<*ctas, p.threads, p.smem, st>>>(a);
  mrl_profile_after(st);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
}
// 16 columns a thread: with up to 256 threads 80 registers leave room for 24 warps of an SM and spare the spills of 64
// (65,536 x 4,096 bf16: 344 us, 370 with 64); beyond, too few CTAs would fit (32,768 x 8,192: 428, 375).
template <typename T, bool kOdd, int kCols>
int launch_bwd_rows(const NormBwdArgs& a, int* ctas, cudaStream_t st) {
  if constexpr (kCols == kMiddle)
    if (row_threads(a.H, kCols) <= 256) return launch_bwd_regs<T, kOdd, kCols, kBwdRegsMore>(a, ctas, st);
  return launch_bwd_regs<T, kOdd, kCols, kBwdRegs>(a, ctas, st);
}
template <typename T>
int launch_fwd(const NormFwdArgs& a, bool odd, cudaStream_t st) {
  switch (fwd_cols(a.N, a.H, sizeof(T), odd)) {
    case kNarrow: return odd ? launch_fwd_rows<T, true, kNarrow>(a, st) : launch_fwd_rows<T, false, kNarrow>(a, st);
    case kMiddle: return odd ? launch_fwd_rows<T, true, kMiddle>(a, st) : launch_fwd_rows<T, false, kMiddle>(a, st);
    default: return launch_fwd_rows<T, false, kWide>(a, st);
  }
}
template <typename T>
int launch_bwd(const NormBwdArgs& a, bool odd, int* ctas, cudaStream_t st) {
  if (bwd_cols(a.N, a.H) == kNarrow)
    return odd ? launch_bwd_rows<T, true, kNarrow>(a, ctas, st) : launch_bwd_rows<T, false, kNarrow>(a, ctas, st);
  return odd ? launch_bwd_rows<T, true, kMiddle>(a, ctas, st) : launch_bwd_rows<T, false, kMiddle>(a, ctas, st);
}

constexpr int kMaxCols = 1 << 30;
// The smallest eps: a square below the normal range is off by 2^-150, the mean too, and 2^-126 beside it keeps that at half a step.
constexpr float kEpsMin = 1.17549435e-38f;
bool on_element(const void* p, int elem) { return (reinterpret_cast<uintptr_t>(p) & (elem - 1)) == 0; }
// An output at an input's address has to have its row stride: it would lie over rows that are still to be read.
bool over_other_rows(const void* out, long long ld_out, const void* in, long long ld_in, long long N) {
  return out != nullptr && out == in && ld_out != ld_in && N > 1;
}
bool row_type_ok(int32_t dtype) { return dtype == MRL_BF16 || dtype == MRL_F32; }

}  // namespace

size_t mrl_rmsnorm_bwd_workspace_bytes(long long N, int H) {
  if (N <= 0 || H <= 0) return 0;
  return mrl_align_up((size_t)bwd_ctas_most(N, H) * (size_t)H * 4, 256);
}

extern "C" int mrl_rmsnorm_residual_fwd(const void* x, int64_t ld_x, const void* residual, int64_t ld_res, int32_t dtype,
                                        const void* weight, int32_t w_dtype, int64_t N, int32_t H,
                                        const mrl_norm_params* np, void* h_out, int64_t ld_h, void* y, int64_t ld_y,
                                        void* y8, int64_t ld_y8, float* scales, float* rstd, void* stream) {
  if (!row_type_ok(dtype) || !row_type_ok(w_dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
  if (np == nullptr || N < 0 || H < 1) return MRL_ERR_INVALID_ARG;
  if (H > kMaxCols) return MRL_ERR_UNSUPPORTED_SHAPE;
  if (!(np->eps >= kEpsMin) || np->eps > 3.4e38f || !(np->weight_offset - np->weight_offset == 0.f)) return MRL_ERR_INVALID_ARG;
  if (np->group != 0 && np->group != 32 && np->group != 64 && np->group != 128 && np->group != 256) return MRL_ERR_INVALID_ARG;
  if (N == 0) return MRL_OK;
  if (h_out == nullptr && y == nullptr && y8 == nullptr && rstd == nullptr) return MRL_ERR_INVALID_ARG;
  if (ld_x < H || (residual != nullptr && ld_res < H) || (h_out != nullptr && ld_h < H) || (y != nullptr && ld_y < H) ||
      (y8 != nullptr && (ld_y8 < H || scales == nullptr)))
    return MRL_ERR_INVALID_ARG;
  if (h_out != nullptr && h_out == y) return MRL_ERR_INVALID_ARG;
  if (y8 != nullptr && (y8 == x || y8 == residual || y8 == h_out || y8 == y)) return MRL_ERR_INVALID_ARG;
  if (over_other_rows(h_out, ld_h, x, ld_x, N) || over_other_rows(h_out, ld_h, residual, ld_res, N) ||
      over_other_rows(y, ld_y, x, ld_x, N) || over_other_rows(y, ld_y, residual, ld_res, N))
    return MRL_ERR_INVALID_ARG;
  if (x == nullptr || weight == nullptr) return MRL_ERR_INVALID_ARG;
  const bool bf16 = dtype == MRL_BF16;
  const int elem = bf16 ? 2 : 4;
  if (!on_element(x, elem) || !on_element(residual, elem) || !on_element(h_out, elem) || !on_element(y, elem) ||
      !on_element(weight, w_dtype == MRL_BF16 ? 2 : 4) || (y8 != nullptr && !on_element(scales, 4)) || !on_element(rstd, 4))
    return MRL_ERR_INVALID_ARG;
  NormFwdArgs a{x, residual, weight, h_out, y, static_cast<uint8_t*>(y8), scales, rstd, ld_x, ld_res, ld_h, ld_y, ld_y8, N,
                H, np->group, w_dtype == MRL_BF16, np->eps, np->weight_offset, 1.0f / (float)H, 0};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (H <= kRowMax) {
    const bool whole = H % (16 / elem) == 0 && aligned(x, ld_x, elem, 16) && aligned(residual, ld_res, elem, 16) &&
                       aligned(h_out, ld_h, elem, 16) && aligned(y, ld_y, elem, 16) && aligned(y8, ld_y8, 1, 16 / elem) &&
                       aligned(weight, 0, 1, 16);
    return bf16 ? launch_fwd<__nv_bfloat16>(a, !whole, st) : launch_fwd<float>(a, !whole, st);
  }
  const unsigned grid = (unsigned)(N < 0x7fffffffll ? N : 0x7fffffffll);
  mrl_profile_before(st, "rmsnorm_fwd_loop_kernel");
  if (bf16)
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
  if (H > kMaxCols) return MRL_ERR_UNSUPPORTED_SHAPE;
  if (!(np->weight_offset - np->weight_offset == 0.f)) return MRL_ERR_INVALID_ARG;
  if (ld_dy < H || ld_h < H || ld_dx < H || (dh != nullptr && ld_dh < H)) return MRL_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool accumulate = (np->flags & MRL_FLAG_ACCUMULATE_DW) != 0;
  if (N == 0) {
    if (dweight != nullptr && !accumulate) MRL_CUDA_OK(cudaMemsetAsync(dweight, 0, (size_t)H * 4, st));
    return MRL_OK;
  }
  if (dy == nullptr || h == nullptr || weight == nullptr || rstd == nullptr || dx == nullptr) return MRL_ERR_INVALID_ARG;
  if (over_other_rows(dx, ld_dx, dy, ld_dy, N) || over_other_rows(dx, ld_dx, dh, ld_dh, N) || over_other_rows(dx, ld_dx, h, ld_h, N))
    return MRL_ERR_INVALID_ARG;
  const bool bf16 = dtype == MRL_BF16;
  const int elem = bf16 ? 2 : 4;
  if (!on_element(dy, elem) || !on_element(dh, elem) || !on_element(h, elem) || !on_element(dx, elem) ||
      !on_element(weight, w_dtype == MRL_BF16 ? 2 : 4) || !on_element(rstd, 4) || !on_element(dweight, 4))
    return MRL_ERR_INVALID_ARG;
  if (dweight != nullptr) {
    if (workspace == nullptr || workspace_bytes < mrl_rmsnorm_bwd_workspace_bytes(N, H)) return MRL_ERR_WORKSPACE_TOO_SMALL;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return MRL_ERR_INVALID_ARG;
  }
  NormBwdArgs a{dy, dh, h, weight, rstd, dx, dweight != nullptr ? static_cast<float*>(workspace) : nullptr, ld_dy, ld_dh,
                ld_h, ld_dx, N, H, w_dtype == MRL_BF16, np->weight_offset, 1.0f / (float)H, 0};
  int rc, ctas = 0;
  if (H <= kRowMax) {
    const bool whole = H % (16 / elem) == 0 && aligned(dy, ld_dy, elem, 16) && aligned(dh, ld_dh, elem, 16) &&
                       aligned(h, ld_h, elem, 16) && aligned(dx, ld_dx, elem, 16) && aligned(weight, 0, 1, 16);
    rc = bf16 ? launch_bwd<__nv_bfloat16>(a, !whole, &ctas, st) : launch_bwd<float>(a, !whole, &ctas, st);
  } else {
    ctas = bwd_ctas_most(N, H);
    mrl_profile_before(st, "rmsnorm_bwd_loop_kernel");
    if (bf16)
      rmsnorm_bwd_loop_kernel<__nv_bfloat16><<<ctas, kLoopThreads, 0, st>>>(a);
    else
      rmsnorm_bwd_loop_kernel<float><<<ctas, kLoopThreads, 0, st>>>(a);
    mrl_profile_after(st);
    rc = cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
  }
  if (rc != MRL_OK) return rc;
  if (dweight != nullptr) {
    MRL_CUDA_OK(mrl_launch_behind(rmsnorm_dw_kernel, (unsigned)((H + 31) / 32), 1024, st, a.partial, ctas, H, dweight, accumulate));
  }
  return MRL_OK;
}
