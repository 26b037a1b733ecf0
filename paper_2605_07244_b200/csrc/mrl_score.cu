// Scoring in 8 bits: mrl_e4m3_quantize and mrl_e4m3_product.
#include "mrl_tensor.cuh"

namespace {

using namespace mrl;

constexpr int kBlock = MRL_SCALE_BLOCK;

__device__ __forceinline__ void store_f(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// ------------------------------------------------------------------------------------------ quantizer
// A block's elements stay in registers between its maximum and its codes: one read, one write.  Bound by HBM (151,936 x 4,096 bf16 287 us, 6.5 TB/s).
// kWide: 16 bytes of a row by one load, and their codes by one store.  Otherwise (rows off 16 bytes) four elements by single loads, and four codes by
// one store where the codes' rows allow it: bound by issue (18,223 x 9,602 bf16 168 us, half of the copy rate, 86 % of the issue slots busy).
template <typename T, bool kWide>
struct Piece {
  static constexpr int kElems = kWide ? 16 / (int)sizeof(T) : 4, kWords = kElems * (int)sizeof(T) / 4;
  uint32_t w[kWords];  // as they lie in memory
  __device__ __forceinline__ float at(int j) const {
    if (sizeof(T) == 4) return __uint_as_float(w[j & (kWords - 1)]);
    return (j & 1) ? bf16hi_to_f32(w[(j >> 1) & (kWords - 1)]) : bf16lo_to_f32(w[(j >> 1) & (kWords - 1)]);
  }
  __device__ __forceinline__ void load(const T* row, int col, int H) {
    if (kWide && col + kElems <= H) {
      const uint4 u = __ldcs(reinterpret_cast<const uint4*>(row + col));
      w[0] = u.x, w[1] = u.y;
      if constexpr (kWords == 4) w[2] = u.z, w[3] = u.w;
      return;
    }
#pragma unroll
    for (int j = 0; j < kWords; ++j) w[j] = 0;
#pragma unroll
    for (int j = 0; j < kElems; ++j)
      if (col + j < H) {
        if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(row[col + j]);
        else w[j / 2] |= (uint32_t)__bfloat16_as_ushort(row[col + j]) << (16 * (j & 1));
      }
  }
  __device__ __forceinline__ float peak() const {  // passes over NaN
    if constexpr (sizeof(T) == 2) {
      uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
      for (int j = 1; j < kWords; ++j) asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[j] & 0x7fff7fffu));
      return fmaxf(0.f, fmaxf(bf16lo_to_f32(m), bf16hi_to_f32(m)));
    } else {
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < kElems; ++j) m = fmaxf(m, fabsf(at(j)));
      return m;
    }
  }
  __device__ __forceinline__ void store(uint8_t* row, int col, int H, float inv, bool words) const {
    uint32_t c[kElems / 4];
#pragma unroll
    for (int j = 0; j < kElems; j += 4) c[j / 4] = pack_e4m3x2(at(j) * inv, at(j + 1) * inv) | pack_e4m3x2(at(j + 2) * inv, at(j + 3) * inv) << 16;
    if (words && col + kElems <= H) {
      if constexpr (kElems == 8) *reinterpret_cast<uint2*>(row + col) = make_uint2(c[0], c[1]);
      else *reinterpret_cast<uint32_t*>(row + col) = c[0];
      return;
    }
#pragma unroll
    for (int j = 0; j < kElems; ++j)
      if (col + j < H) row[col + j] = (uint8_t)(c[j / 4] >> (8 * (j & 3)));
  }
};

struct QuantizeArgs {
  const void* x;
  long long ld_x, N;
  int H;
  uint8_t* codes;
  long long ld_codes;
  float* scales;
  bool words;  // a piece's codes start on a multiple of their number
};

// One CTA per block of 128 x 128; blocks of the same rows follow one another.  (Four CTAs an SM keep 128 KB on their way; with two, and the elements
// as floats, 507 us instead of 300.)
template <typename T, bool kWide>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) quantize_block_kernel(const QuantizeArgs p) {
  using P = Piece<T, kWide>;
  __shared__ float red[8];
  constexpr int kAcross = kBlock / P::kElems, kDown = 256 / kAcross, kEach = kBlock / kDown;  // threads across and down, pieces of a thread
  const int blocks = (p.H + kBlock - 1) / kBlock, tid = threadIdx.x;
  const long long row0 = (long long)(blockIdx.x / (unsigned)blocks) * kBlock + tid / kAcross;
  const int col = (int)(blockIdx.x % (unsigned)blocks) * kBlock + tid % kAcross * P::kElems;
  const T* x = static_cast<const T*>(p.x) + row0 * p.ld_x;
  P piece[kEach];
  float peak = 0.f;
#pragma unroll
  for (int i = 0; i < kEach; ++i) piece[i].load(x + i * kDown * p.ld_x, col, row0 + i * kDown < p.N ? p.H : 0);
#pragma unroll
  for (int i = 0; i < kEach; ++i) peak = fmaxf(peak, piece[i].peak());
  peak = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(peak)));  // (not negative: in the order of its bits)
  if ((tid & 31) == 0) red[tid >> 5] = peak;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) peak = fmaxf(peak, red[k]);
  const float scale = e4m3_scale(peak), inv = 1.0f / scale;
  if (tid == 0) p.scales[blockIdx.x] = scale;
  uint8_t* out = p.codes + row0 * p.ld_codes;
#pragma unroll
  for (int i = 0; i < kEach; ++i) piece[i].store(out + i * kDown * p.ld_codes, col, row0 + i * kDown < p.N ? p.H : 0, inv, p.words);
}

// Blocks of 1 x 128, each by the lanes that hold it; a thread works on kRowPieces of them at a time.
constexpr int kRowPieces = 4;
template <typename T, bool kWide>
__global__ void __launch_bounds__(256) quantize_row_kernel(const QuantizeArgs p) {
  using P = Piece<T, kWide>;
  constexpr int kLanes = kBlock / P::kElems, kGroups = 256 / kLanes;
  const int blocks = (p.H + kBlock - 1) / kBlock, lane = threadIdx.x % kLanes;
  const long long total = p.N * blocks, first = (long long)blockIdx.x * (kGroups * kRowPieces) + threadIdx.x / kLanes;
  P piece[kRowPieces];
  long long row[kRowPieces];
  int col[kRowPieces];
#pragma unroll
  for (int i = 0; i < kRowPieces; ++i) {
    const long long b = first + i * kGroups;
    row[i] = b < total ? (total <= 0x7fffffffll ? (long long)((unsigned)b / (unsigned)blocks) : b / blocks) : 0;
    col[i] = b < total ? (int)(b - row[i] * blocks) * kBlock + lane * P::kElems : p.H;  // (no column: nothing is read)
    piece[i].load(static_cast<const T*>(p.x) + row[i] * p.ld_x, col[i], p.H);
  }
#pragma unroll
  for (int i = 0; i < kRowPieces; ++i) {
    const long long b = first + i * kGroups;
    float peak = piece[i].peak();
    if constexpr (kLanes == 32) {
      peak = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(peak)));  // (not negative: in the order of its bits)
    } else {
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) peak = fmaxf(peak, __shfl_xor_sync(0xffffffffu, peak, o));
    }
    const float scale = e4m3_scale(peak), inv = 1.0f / scale;
    if (b < total && lane == 0) p.scales[b] = scale;
    piece[i].store(p.codes + row[i] * p.ld_codes, col[i], p.H, inv, p.words);
  }
}

template <typename T, bool kWide>
int launch_quantize(const QuantizeArgs& a, int rows, cudaStream_t st) {
  const long long blocks = (a.H + kBlock - 1) / kBlock, cta_blocks = kRowPieces * 256 * Piece<T, kWide>::kElems / kBlock;
  const long long ctas = rows == 1 ? (a.N * blocks + cta_blocks - 1) / cta_blocks : (a.N + kBlock - 1) / kBlock * blocks;
  if (ctas > 0x7fffffffll) return MRL_ERR_UNSUPPORTED_SHAPE;
  mrl_profile_before(st, rows == 1 ? "quantize_row_kernel" : "quantize_block_kernel");
  if (rows == 1)
    quantize_row_kernel<T, kWide><<<(unsigned)ctas, 256, 0, st>>>(a);
  else
    quantize_block_kernel<T, kWide><<<(unsigned)ctas, 256, 0, st>>>(a);
  mrl_profile_after(st);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
}

// ------------------------------------------------------------------------------------------ product
// One CTA per SM works through tiles of 128 rows x 256 weights.  Warp 0 brings K-blocks of 128 codes (one 128-byte swizzle row) into a
// ring by TMA, one thread of warp 1 multiplies each into one of two accumulators in tensor memory -- never two blocks into the same,
// for each block has its own scale -- and eight warps add scale * accumulator to sums in registers, 128 columns (so one scale) of one
// row a thread, while the next block is multiplied.  A block takes 827 cycles (stamps; 4,096 x 151,936 x 4,096 2.6 to 2.7 ms in repeated calls, 2.3 ms alone): 512 are the tensor core's, its
// operands alone come in 715 (48 KB from L2), additions and loads out of tensor memory take the rest.  Pairs of CTAs, which share the weights' tile, 5.6 ms: each
// block waited for an arrival across the pair; sixteen warps of 64 columns 2.96.
constexpr int kBM = 128, kBN = 256;
constexpr int kStages = 4, kEpiWarps = 8, kProductThreads = 128 + 32 * kEpiWarps;
// registers of a thread: 168 at launch, moved from the first warpgroup (copies, issue) to the two that hold sums (128 x 40 + 256 x 232)
constexpr int kIssueRegs = 40, kSumRegs = 232;
constexpr uint32_t kATile = kBM * kBlock, kBTile = kBN * kBlock, kStage = kATile + kBTile;
// staging of a warp's outputs: 32 rows of 64 bytes, 16 bytes between them
constexpr uint32_t kOutRow = 80, kOutWarp = 32 * kOutRow;
constexpr size_t kProductSmem = (size_t)kStages * kStage + 1024 /* alignment */ + 256 /* barriers */ + kEpiWarps * kOutWarp;
constexpr uint32_t kIdescE4m3 = (1u << 4) /* float32 sums */ | ((uint32_t)(kBN >> 3) << 17) | ((uint32_t)(kBM >> 4) << 24);

struct ProductArgs {
  const float *x_scales, *w_scales;
  void* out;
  long long N, ld_out;
  int V, k_blocks, m_tiles, n_tiles, group_m;
  bool vector_out, vector_scales;  // rows of out, and of both scales, start on 16 bytes
  int32_t* status;
};

// sum += a * b, where it stands among the loads (left to itself the compiler gathers the additions behind the last load)
__device__ __forceinline__ void fma_f2_here(f2& sum, f2 a, f2 b) {
  asm volatile("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(sum) : "l"(a), "l"(b));
}

// D[tmem] (+)= A[smem] * B[smem]^T, one step of 32 on e4m3 codes
__device__ __forceinline__ void tc_mma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accum)
      : "memory");
}

template <typename T>
__global__ void __launch_bounds__(kProductThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const ProductArgs p) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_addr(smem_raw), tiles = (raw + 1023u) & ~1023u;
  unsigned char* after = smem_raw + (tiles - raw) + (size_t)kStages * kStage;
  uint64_t* bars = reinterpret_cast<uint64_t*>(after);
  const uint32_t bar0 = smem_addr(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * kStages + a); };
  auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * kStages + 2 + a); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int total = p.m_tiles * p.n_tiles;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(tfull_bar(a), 1);
      mbar_init(tempty_bar(a), kEpiWarps);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssueRegs));
  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
        int m, n;
        tile_coords(t, p.m_tiles, p.n_tiles, p.group_m, m, n);
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t dst = tiles + (uint32_t)stage * kStage;
          mbar_expect_tx(full_bar(stage), kStage);
          tma_load_2d(dst, &map_x, kb * kBlock, m * kBM, full_bar(stage));
          tma_load_2d(dst + kATile, &map_w, kb * kBlock, n * kBN, full_bar(stage));
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // (The whole warp goes through the loop, so that addresses and descriptors stay in uniform registers; one lane issues.  Nothing in the loop is for whole
    // warps, so a lane may leave it by itself when a wait runs out.)
    const bool issuer = elect_one();
    int stage = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
      for (int kb = 0; kb < p.k_blocks; ++kb) {
        if (!mbar_wait2(tempty_bar(acc), acc_phase ^ 1u, full_bar(stage), phase, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t src = tiles + (uint32_t)stage * kStage;
        const uint64_t a = smem_desc_k128(src), b = smem_desc_k128(src + kATile);
        if (issuer) {
#pragma unroll
          for (int k = 0; k < kBlock / 32; ++k)  // 32 codes: 32 bytes along a swizzle row
            tc_mma_e4m3(tmem + (uint32_t)acc * kBN, a + 2 * k, b + 2 * k, kIdescE4m3, k != 0);
          tc_commit(empty_bar(stage));
          tc_commit(tfull_bar(acc));
        }
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
        acc ^= 1;
        if (acc == 0) acc_phase ^= 1u;
      }
    }
  } else if (warp >= 4) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSumRegs));
    const int quad = warp & 3, half = (warp - 4) >> 2;  // lanes 32 quad .. + 31 of tensor memory, columns 128 half .. + 127 of the tile
    const uint32_t staging = smem_addr(after + 256) + (uint32_t)(warp - 4) * kOutWarp;
    const uint32_t mine = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * kBlock);
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
      int m, n;
      tile_coords(t, p.m_tiles, p.n_tiles, p.group_m, m, n);
      const long long row0 = (long long)m * kBM + quad * 32, row = row0 + lane;
      const int col0 = n * kBN + half * kBlock;
      const bool live = row < p.N && col0 < p.V;
      const float* xs = p.x_scales + (live ? row * p.k_blocks : 0);
      const float* ws = p.w_scales + (live ? (long long)(n * 2 + half) * p.k_blocks : 0);
      f2 sum[kBlock / 2];
#pragma unroll
      for (int j = 0; j < kBlock / 2; ++j) sum[j] = 0;
      // scales of four K-blocks at a time, the next four on their way (a row's scales lie in one or two lines: four single loads
      // of them cost as much of L1 as one of 16 bytes)
      float sx[4], sw[4], s4[4];
      auto load_scales = [&](int kb) {
        if (p.vector_scales) {
          const float4 x = live && kb < p.k_blocks ? *reinterpret_cast<const float4*>(xs + kb) : make_float4(0.f, 0.f, 0.f, 0.f);
          const float4 w = live && kb < p.k_blocks ? *reinterpret_cast<const float4*>(ws + kb) : make_float4(0.f, 0.f, 0.f, 0.f);
          sx[0] = x.x, sx[1] = x.y, sx[2] = x.z, sx[3] = x.w;
          sw[0] = w.x, sw[1] = w.y, sw[2] = w.z, sw[3] = w.w;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            sx[j] = live && kb + j < p.k_blocks ? xs[kb + j] : 0.f;
            sw[j] = live && kb + j < p.k_blocks ? ws[kb + j] : 0.f;
          }
        }
      };
      load_scales(0);
      if (!mbar_wait_warp(tfull_bar(acc), acc_phase, abort_flag)) { ok = false; break; }
      tc_fence_after();
      uint32_t v[2][32];  // the 32 columns that are added and the 32 on their way
      tc_ld32_start(mine + (uint32_t)(acc * kBN), v[0]);
#pragma unroll 1
      for (int kb = 0; kb < p.k_blocks; ++kb) {
        if ((kb & 3) == 0) {
#pragma unroll
          for (int j = 0; j < 4; ++j) s4[j] = sx[j] * sw[j];
          load_scales(kb + 4);
        }
        const f2 s2 = make_f2(s4[0], s4[0]);
        s4[0] = s4[1], s4[1] = s4[2], s4[2] = s4[3];
        const uint32_t src = mine + (uint32_t)(acc * kBN), last = tempty_bar(acc);
        acc ^= 1;
        if (acc == 0) acc_phase ^= 1u;
        bool ready = false;  // in all lanes alike
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          tc_ld32_wait(v[c & 1]);
          if (c < 3) {
            tc_ld32_start(src + (uint32_t)(32 * (c + 1)), v[(c & 1) ^ 1]);
            if (c == 2) ready = __all_sync(0xffffffffu, mbar_test(tfull_bar(acc), acc_phase));
          } else {  // read: the accumulator may be written again
            tc_fence_before();
            if (lane == 0) mbar_arrive(last);
            if (kb + 1 < p.k_blocks) {
              if (!ready) ok = mbar_wait_warp(tfull_bar(acc), acc_phase, abort_flag);
              if (!ok) break;
              tc_fence_after();
              tc_ld32_start(mine + (uint32_t)(acc * kBN), v[0]);
            }
          }
#pragma unroll
          for (int j = 0; j < 32; j += 2)
            fma_f2_here(sum[c * 16 + j / 2], make_f2(__uint_as_float(v[c & 1][j]), __uint_as_float(v[c & 1][j + 1])), s2);
        }
        if (!ok) break;
      }
      if (!ok) break;
      // out through shared memory, 64 bytes of 32 rows at a time
      constexpr int kCols = 64 / (int)sizeof(T);
      T* out = static_cast<T*>(p.out) + row0 * p.ld_out + col0;
      const int rows = (int)min((long long)32, p.N - row0), cols = p.V - col0;
      if (rows > 0) {
#pragma unroll
        for (int c = 0; c < kBlock; c += kCols) {
          if (c < cols) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 2) {
                  w[j] = f2_to_bf16x2(sum[c / 2 + q * 4 + j]);
                } else {
                  const float2 u = split_f2(sum[c / 2 + q * 2 + j / 2]);
                  w[j] = __float_as_uint(j & 1 ? u.y : u.x);
                }
              }
              sts_v4(staging + (uint32_t)lane * kOutRow + 16u * q, w[0], w[1], w[2], w[3]);
            }
            __syncwarp();
            if (p.vector_out && c + kCols <= cols) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int r = (lane >> 2) + 8 * i;
                const uint4 u = lds_v4(staging + (uint32_t)r * kOutRow + (uint32_t)(lane & 3) * 16u);
                if (r < rows) *reinterpret_cast<uint4*>(out + r * p.ld_out + c + (lane & 3) * (16 / sizeof(T))) = u;
              }
            } else {
              const T* staged = reinterpret_cast<const T*>(after + 256 + (warp - 4) * kOutWarp);
              const int col = lane % kCols;  // (of float32 two rows at a time)
#pragma unroll 4
              for (int r = lane / kCols; r < rows; r += 32 / kCols)
                if (c + col < cols) out[r * p.ld_out + c + col] = staged[r * (kOutRow / sizeof(T)) + col];
            }
            __syncwarp();
          }
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (threadIdx.x == 0 && p.status != nullptr) atomicOr(p.status, MRL_DEV_TIMEOUT);
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // let copies and MMAs still in flight land before the CTA goes
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------------------------------ product of few rows
// Up to 32 rows of x: bound by the weights' bytes.  The weights take the tensor core's 128 lanes here and the rows of x its columns, so that a CTA keeps a deep
// ring of weights alone on its way; a thread sums one weight row's outputs.  Tiles are as high as makes all CTAs work on the same number of
// them (151,936 rows: 9 of 115 on each of 148 SMs instead of 8 or 9 of 128).
constexpr int kFewThreads = 192, kFewAccs = 8;  // warps: copies, issue, four that sum; accumulators, one K-block each
// (with as many columns as rows, 64 of them 158 us at 64 rows against 131 with the tiles above, 32 of them 118 at 24 rows against 131)
constexpr int kMostFew = 32;
template <int kFew>
struct FewSize {
  static constexpr uint32_t kStage = kATile + kFew * kBlock;
  // (one token's 622 MB of weights, their copies in 200 KB of stages an SM 118 us, in 183 115, in 146 to 164 112, in 110 115)
  static constexpr int kStages = (int)(150 * 1024 / kStage);
  static constexpr size_t kSmem = (size_t)kStages * kStage + 1024 /* alignment */ + 512 /* barriers */ + 4 * 4 * kFew * 4 /* scales of x */;
};

struct FewArgs {
  const float *x_scales, *w_scales;
  void* out;
  long long ld_out;
  int N, V, k_blocks, tiles, height;  // height: weight rows of a tile
  int32_t* status;
};

template <typename T, int kFew>
__global__ void __launch_bounds__(kFewThreads, 1)
product_few_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const FewArgs p) {
  constexpr int kFewStages = FewSize<kFew>::kStages;
  constexpr uint32_t kFewStage = FewSize<kFew>::kStage;
  constexpr uint32_t kIdesc = (1u << 4) | ((uint32_t)(kFew >> 3) << 17) | ((uint32_t)(kBM >> 4) << 24);
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_addr(smem_raw), tiles = (raw + 1023u) & ~1023u;
  unsigned char* after = smem_raw + (tiles - raw) + (size_t)kFewStages * kFewStage;
  uint64_t* bars = reinterpret_cast<uint64_t*>(after);
  const uint32_t bar0 = smem_addr(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kFewStages + s); };
  auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * kFewStages + a); };
  auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * kFewStages + kFewAccs + a); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kFewStages + 2 * kFewAccs);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kFewStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < kFewAccs; ++a) {
      mbar_init(tfull_bar(a), 1);
      mbar_init(tempty_bar(a), 4);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x)
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag)) { ok = false; break; }
          const uint32_t dst = tiles + (uint32_t)stage * kFewStage;
          mbar_expect_tx(full_bar(stage), (uint32_t)(p.height + kFew) * kBlock);
          tma_load_2d(dst, &map_w, kb * kBlock, t * p.height, full_bar(stage));
          tma_load_2d(dst + kATile, &map_x, kb * kBlock, 0, full_bar(stage));
          if (++stage == kFewStages) { stage = 0; phase ^= 1u; }
        }
    }
  } else if (warp == 1) {
    const bool issuer = elect_one();
    int stage = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x)
      for (int kb = 0; kb < p.k_blocks; ++kb) {
        if (!mbar_wait2(tempty_bar(acc), acc_phase ^ 1u, full_bar(stage), phase, abort_flag)) { ok = false; break; }
        tc_fence_after();
        const uint32_t src = tiles + (uint32_t)stage * kFewStage;
        const uint64_t a = smem_desc_k128(src), b = smem_desc_k128(src + kATile);
        if (issuer) {
#pragma unroll
          for (int k = 0; k < kBlock / 32; ++k) tc_mma_e4m3(tmem + (uint32_t)(acc * kFew), a + 2 * k, b + 2 * k, kIdesc, k != 0);
          tc_commit(empty_bar(stage));
          tc_commit(tfull_bar(acc));
        }
        if (++stage == kFewStages) { stage = 0; phase ^= 1u; }
        if (++acc == kFewAccs) { acc = 0; acc_phase ^= 1u; }
      }
  } else {
    const int quad = warp & 3;
    float* sx = reinterpret_cast<float*>(after + 512) + (warp - 2) * 4 * kFew;  // [4 K-blocks][kFew], this warp's own
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x) {
      const int within = quad * 32 + lane, v = t * p.height + within;
      const bool live = within < p.height && v < p.V;
      const float* ws = p.w_scales + (live ? (long long)(v / kBlock) * p.k_blocks : 0);
      f2 sum[kFew / 2];
#pragma unroll
      for (int j = 0; j < kFew / 2; ++j) sum[j] = 0;
#pragma unroll 1
      for (int kb0 = 0; kb0 < p.k_blocks && ok; kb0 += 4) {
        float sw[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) sw[q] = live && kb0 + q < p.k_blocks ? ws[kb0 + q] : 0.f;
        __syncwarp();
#pragma unroll
        for (int r = lane; r < kFew; r += 32)
#pragma unroll
          for (int q = 0; q < 4; ++q) sx[q * kFew + r] = r < p.N && kb0 + q < p.k_blocks ? p.x_scales[(long long)r * p.k_blocks + kb0 + q] : 0.f;
        __syncwarp();
#pragma unroll 1
        for (int q = 0; q < 4 && kb0 + q < p.k_blocks; ++q) {
          ok = mbar_wait_warp(tfull_bar(acc), acc_phase, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const float w = q == 0 ? sw[0] : q == 1 ? sw[1] : q == 2 ? sw[2] : sw[3];
          const f2 w2 = make_f2(w, w);
          const uint32_t src = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(acc * kFew);
          const float4* s4 = reinterpret_cast<const float4*>(sx + q * kFew);
#pragma unroll
          for (int c = 0; c < kFew; c += 16) {
            uint32_t d[16];
            tc_ld16(src + (uint32_t)c, d);
            if (c + 16 == kFew) {
              tc_fence_before();
              if (lane == 0) mbar_arrive(tempty_bar(acc));
            }
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
              const float4 s = s4[(c + j) / 4];
              f2* to = sum + (c + j) / 2;
              to[0] = fma_f2(make_f2(__uint_as_float(d[j]), __uint_as_float(d[j + 1])), mul_f2(make_f2(s.x, s.y), w2), to[0]);
              to[1] = fma_f2(make_f2(__uint_as_float(d[j + 2]), __uint_as_float(d[j + 3])), mul_f2(make_f2(s.z, s.w), w2), to[1]);
            }
          }
          if (++acc == kFewAccs) { acc = 0; acc_phase ^= 1u; }
        }
      }
      if (!ok) break;
      if (live) {
        T* out = static_cast<T*>(p.out) + v;
#pragma unroll
        for (int j = 0; j < kFew; j += 2) {
          const float2 u = split_f2(sum[j / 2]);
          if (j < p.N) store_f(out + j * p.ld_out, u.x);
          if (j + 1 < p.N) store_f(out + (j + 1) * p.ld_out, u.y);
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (threadIdx.x == 0 && p.status != nullptr) atomicOr(p.status, MRL_DEV_TIMEOUT);
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // let copies and MMAs still in flight land before the CTA goes
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// Tensor map of a row-major matrix of codes [rows, cols], read in tiles of box_rows x 128; zeros beyond its ends.
int make_code_map(CUtensorMap* map, const void* base, long long rows, int cols, long long ld, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (fn == nullptr) return MRL_ERR_CUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? ld : (long long)mrl_align_up((size_t)cols, 16))};
  const cuuint32_t box[2] = {(cuuint32_t)kBlock, (cuuint32_t)box_rows};
  const cuuint32_t step[2] = {1, 1};
  const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, step,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? MRL_OK : MRL_ERR_CUDA;
}

template <typename T>
int launch_product(const CUtensorMap& mx, const CUtensorMap& mw, const ProductArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> attr_done;
  const int rc = mrl_once_per_device(attr_done, [] {
    return cudaFuncSetAttribute(product_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kProductSmem);
  });
  if (rc != MRL_OK) return rc;
  const long long total = (long long)a.m_tiles * a.n_tiles;
  const int grid = (int)(total < sm_count() ? total : sm_count());
  mrl_profile_before(st, "product_kernel");
  product_kernel<T><<<grid, kProductThreads, kProductSmem, st>>>(mx, mw, a);
  mrl_profile_after(st);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
}

template <typename T, int kFew>
int launch_few(const void* x8, long long ld_x, const void* w8, long long ld_w, int H, FewArgs a, cudaStream_t st) {
  static std::atomic<uint64_t> attr_done;
  int rc = mrl_once_per_device(attr_done, [] {
    return cudaFuncSetAttribute(product_few_kernel<T, kFew>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)FewSize<kFew>::kSmem);
  });
  if (rc != MRL_OK) return rc;
  const int sms = sm_count(), rounds = (int)(((long long)a.V + (long long)sms * kBM - 1) / ((long long)sms * kBM));
  a.height = (int)(((long long)a.V + (long long)sms * rounds - 1) / ((long long)sms * rounds));
  a.tiles = (a.V + a.height - 1) / a.height;
  CUtensorMap mx, mw;
  rc = make_code_map(&mx, x8, a.N, H, ld_x, kFew);
  if (rc == MRL_OK) rc = make_code_map(&mw, w8, a.V, H, ld_w, a.height);
  if (rc != MRL_OK) return rc;
  mrl_profile_before(st, "product_few_kernel");
  product_few_kernel<T, kFew><<<a.tiles < sms ? a.tiles : sms, kFewThreads, FewSize<kFew>::kSmem, st>>>(mx, mw, a);
  mrl_profile_after(st);
  return cudaGetLastError() == cudaSuccess ? MRL_OK : MRL_ERR_CUDA;
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
  const int elem = dtype == MRL_BF16 ? 2 : 4, vec = 16 / elem;
  auto codes_on = [&](int n) { return on_element(codes, n) && (N == 1 || ld_codes % n == 0); };
  const bool wide = on_element(x, 16) && (N == 1 || ld_x * elem % 16 == 0) && codes_on(vec);
  const QuantizeArgs a{x, ld_x, N, H, static_cast<uint8_t*>(codes), ld_codes, scales, wide || codes_on(4)};
  if (dtype == MRL_BF16)
    return wide ? launch_quantize<__nv_bfloat16, true>(a, block_rows, st) : launch_quantize<__nv_bfloat16, false>(a, block_rows, st);
  return wide ? launch_quantize<float, true>(a, block_rows, st) : launch_quantize<float, false>(a, block_rows, st);
}

extern "C" int mrl_e4m3_product(const void* x8, int64_t ld_x, const float* x_scales, const void* w8, int64_t ld_w,
                                const float* w_scales, int64_t N, int32_t H, int32_t V, int32_t out_dtype, void* out, int64_t ld_out,
                                int32_t* status, void* stream) {
  if (!row_type_ok(out_dtype)) return MRL_ERR_UNSUPPORTED_DTYPE;
  if (N < 0 || H < 1 || V < 1 || ld_x < H || ld_w < H || ld_out < V) return MRL_ERR_INVALID_ARG;
  if (H > (1 << 24) || V > (1 << 30) || N > 0x7fffffffll) return MRL_ERR_UNSUPPORTED_SHAPE;
  if (N == 0) return MRL_OK;
  if (x8 == nullptr || x_scales == nullptr || w8 == nullptr || w_scales == nullptr || out == nullptr) return MRL_ERR_INVALID_ARG;
  if (!on_element(x8, 16) || !on_element(w8, 16) || (N > 1 && ld_x % 16 != 0) || (V > 1 && ld_w % 16 != 0)) return MRL_ERR_INVALID_ARG;
  if (!on_element(x_scales, 4) || !on_element(w_scales, 4) || !on_element(out, out_dtype == MRL_BF16 ? 2 : 4) || !on_element(status, 4))
    return MRL_ERR_INVALID_ARG;
  if (out == x8 || out == w8 || out == x_scales || out == w_scales) return MRL_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int k_blocks = (H + kBlock - 1) / kBlock;
  if (N <= kMostFew) {
    const FewArgs f{x_scales, w_scales, out, ld_out, (int)N, V, k_blocks, 0, 0, status};
    if (out_dtype == MRL_BF16)
      return N <= 16 ? launch_few<__nv_bfloat16, 16>(x8, ld_x, w8, ld_w, H, f, st) : launch_few<__nv_bfloat16, 32>(x8, ld_x, w8, ld_w, H, f, st);
    return N <= 16 ? launch_few<float, 16>(x8, ld_x, w8, ld_w, H, f, st) : launch_few<float, 32>(x8, ld_x, w8, ld_w, H, f, st);
  }
  CUtensorMap mx, mw;
  int rc = make_code_map(&mx, x8, N, H, ld_x, kBM);
  if (rc == MRL_OK) rc = make_code_map(&mw, w8, V, H, ld_w, kBN);
  if (rc != MRL_OK) return rc;
  const int es = out_dtype == MRL_BF16 ? 2 : 4;
  ProductArgs a{};
  a.x_scales = x_scales;
  a.w_scales = w_scales;
  a.out = out;
  a.N = N;
  a.ld_out = ld_out;
  a.V = V;
  a.k_blocks = k_blocks;
  a.m_tiles = (int)((N + kBM - 1) / kBM);
  a.n_tiles = (V + kBN - 1) / kBN;
  a.group_m = 4096 / kBM;  // rows of x that stay in L2 while the weights pass by
  a.vector_out = on_element(out, 16) && (N == 1 || ld_out * es % 16 == 0);
  a.vector_scales = a.k_blocks % 4 == 0 && on_element(x_scales, 16) && on_element(w_scales, 16);
  a.status = status;
  if ((long long)a.m_tiles * a.n_tiles > 0x7fffffffll) return MRL_ERR_UNSUPPORTED_SHAPE;
  return out_dtype == MRL_BF16 ? launch_product<__nv_bfloat16>(mx, mw, a, st) : launch_product<float>(mx, mw, a, st);
}
