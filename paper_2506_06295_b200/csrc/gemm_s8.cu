// Products of 8-bit integers:  C[M, N] = (A W^T)[m, n] * sA[m] * sW[n],  A [M, K] rows (tokens), W [N, K] output channels.
//
// The sums are exact 32-bit integers, so neither tile nor split changes a result; a product is scaled by its row's and its
// column's scale in fp32 and rounded once to the output's type.  A product of few rows is bound by streaming W, half the
// bytes of bf16; one of many rows by the tensor cores at twice the bf16 rate.
//
// Layout, ring and roles are those of the bf16 products (gemm_tcgen05.cu): a stage holds 128 bytes of k of each row, which
// are 128 integers instead of 64 bf16, and one tcgen05.mma (kind::i8) takes 32 of them, so bytes, cycles and addresses per
// stage are the same and only the number of stages halves.  Up to 128 rows one CTA per 128 weight rows with the k range
// split until the chip streams; above that the persistent CTA pairs of gemm_pair.cuh.
#include "../../include/dllm.h"
#include "gemm_s8.cuh"
#include "tma.cuh"
#include "umma.cuh"
#include "gemm_pair.cuh"

namespace dllm {

namespace {

// Test hook (dllm_debug_skip_one_load): while non-zero, CTA (0, 0, last range of k) of every launch of the one-CTA kernel leaves
// out its first tile of A, so that its waits run into their limit.
static __device__ int g_debug_skip = 0;

constexpr int S8_K = 128;    // integers of k per stage: one 128-byte swizzle row

// W columns (rows of A) of a finished tile, TMEM lane = weight row: 128 threads, tl = 0..127 = lane, all in step.  split: the
// integers go to the slab, for the sum over the slabs.  The rows' scales of a trip are requested together, ahead of the
// accumulator's columns (one by one between the stores, which the compiler must assume to change them, they took 1700 cycles
// per trip of 16 rows: 8192 x 24576 x 4096 757 us, 505 now).  bf16: two lanes put their columns of two rows together, four
// bytes a store.
template <int W, typename T>
__device__ __forceinline__ void s8_epilogue(uint32_t tmem_d, int tl, int m0, int n0, int M, int N, const float* __restrict__ sa,
                                            const float* __restrict__ sw, T* __restrict__ out, int* __restrict__ slab) {
  const uint32_t tmem_w = tmem_d + ((uint32_t)(tl >> 5) << 21);
  const int n = n0 + tl;
  const float w = n < N ? __ldg(sw + n) : 0.f;
  const bool pairs = sizeof(T) == 2 && !(N & 1) && !((uintptr_t)out & 3);
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
  for (int c0 = 0; c0 < W; c0 += 16) {
    if (m0 + c0 >= M) break;  // uniform across the warp
    uint32_t r[16];
    tmem_ld16(tmem_w + (uint32_t)c0, r);
    float a[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) a[j] = slab ? 0.f : __ldg(sa + min(m0 + c0 + j, M - 1));
    tmem_ld16_wait(r);
    const size_t first = (size_t)(m0 + c0) * N;
    if (slab) {
      if (n < N) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (m0 + c0 + j < M) slab[first + (size_t)j * N + n] = (int)r[j];
      }
      continue;
    }
    float v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = __int2float_rn((int)r[j]) * a[j] * w;
    if (pairs) {
      const int odd = tl & 1;
      T* const dst = out + first + (size_t)odd * N + (n & ~1);
#pragma unroll
      for (int j = 0; j < 16; j += 2) {
        const float other = __shfl_xor_sync(0xffffffffu, odd ? v[j] : v[j + 1], 1);
        const __nv_bfloat162 h = __floats2bfloat162_rn(odd ? other : v[j], odd ? v[j + 1] : other);
        if (n < N && m0 + c0 + j + odd < M) *reinterpret_cast<__nv_bfloat162*>(dst + (size_t)j * N) = h;
      }
    } else if (n < N) {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (m0 + c0 + j < M) out[first + (size_t)j * N + n] = from_f32<T>(v[j]);
    }
  }
}

template <int BN>
struct S8Layout {
  static constexpr uint32_t STAGE_BYTES = (TILE_W + BN) * S8_K;
  static constexpr uint32_t total(int stages) { return (uint32_t)stages * STAGE_BYTES + 1024; }
  static constexpr int most() {
    const int fit = (227 * 1024 - 1024 - 256) / (int)STAGE_BYTES;
    return fit < MAX_STAGES ? fit : MAX_STAGES;
  }
};

// One CTA: 128 weight rows x BN rows of A x a k range (blockIdx.z).  Warp 0 requests operands, warp 1 issues the MMAs, all
// eight drain the accumulator, half of the columns per group of four.  The CTAs of a split tile are a cluster: each leaves its
// integers in its own shared memory (the drained ring), and each adds up every S-th row of the tile over all of them, scales it
// and writes it.  (3 x 4096 x 4096 in five splits with slabs in global memory and a launch that adds them: 10.5 us with the
// row quantisation, and a third launch for the host; so: 8.5.)
constexpr int S8_THREADS = 256, S8_MOST_SPLITS = 8;
__device__ __forceinline__ int4 remote4(uint32_t addr) {
  int4 r;
  asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr));
  return r;
}
template <int BN, bool ONCE, typename T>
__global__ void __launch_bounds__(S8_THREADS) gemm_s8_kernel(const __grid_constant__ CUtensorMap tmW,
                                                             const __grid_constant__ CUtensorMap tmA,
                                                             const float* __restrict__ sa, const float* __restrict__ sw,
                                                             T* __restrict__ out, int M, int N, int num_kb, int kb_per_split,
                                                             int stages, int* __restrict__ status) {
  using SL = S8Layout<BN>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[MAX_STAGES];
  __shared__ __align__(8) uint64_t empty_bar[MAX_STAGES];
  __shared__ __align__(8) uint64_t accum_bar;
  __shared__ uint32_t tmem_base_slot;
  __shared__ int abort_flag;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int m0 = blockIdx.x * BN, n0 = blockIdx.y * TILE_W;
  const int kb0 = blockIdx.z * kb_per_split, nkb = min(num_kb, kb0 + kb_per_split) - kb0;   // >= 1 by the plan
  const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int pre = min(stages, nkb);  // stages whose weight tile is requested before the dependency wait
  int dbg_skip = 0;
  if (warp == 0) {
    dbg_skip = g_debug_skip;  // read here, long before it is used: not on the path behind the dependency wait
    if (elect_one()) {
      abort_flag = 0;
      for (int s = 0; s < stages; ++s) {
        mbar_init(smem_u32(&full_bar[s]), 1);
        mbar_init(smem_u32(&empty_bar[s]), 1);
      }
      mbar_init(smem_u32(&accum_bar), 1);
      mbar_fence_init();
      prefetch_tensormap(&tmW);
      prefetch_tensormap(&tmA);
      for (int i = 0; i < pre; ++i) {   // see launch_gemm_s8: no launch this one may overlap writes W
        const uint32_t fb = smem_u32(&full_bar[i]);
        mbar_expect_tx(fb, SL::STAGE_BYTES);
        tma_load_2d_weights<ONCE>(tiles + i * SL::STAGE_BYTES, &tmW, fb, (kb0 + i) * S8_K, n0);
      }
    }
    __syncwarp();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)),
                 "r"((uint32_t)BN)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_d = tmem_base_slot;
  volatile int* abortp = &abort_flag;
  pdl_wait();
  pdl_trigger();

  if (warp == 0) {
    int s = 0;
    uint32_t ph = 0;
    for (int i = 0; i < nkb; ++i) {
      const uint32_t fb = smem_u32(&full_bar[s]), dst = tiles + s * SL::STAGE_BYTES;
      const int kc = (kb0 + i) * S8_K;
      const bool skip = i == 0 && dbg_skip != 0 && (blockIdx.x | blockIdx.y) == 0 && blockIdx.z == gridDim.z - 1;
      if (i >= pre && !mbar_wait_warp(smem_u32(&empty_bar[s]), ph ^ 1u, abortp)) {
        if (status && lane == 0) atomicCAS(status, ST_OK, ST_TIMEOUT_TMA);
        break;
      }
      if (elect_one()) {
        if (i >= pre) {
          mbar_expect_tx(fb, SL::STAGE_BYTES);
          tma_load_2d_weights<ONCE>(dst, &tmW, fb, kc, n0);
        }
        if (!skip) tma_load_2d(dst + W_STAGE_BYTES, &tmA, fb, kc, m0);
      }
      __syncwarp();
      if (++s == stages) {
        s = 0;
        ph ^= 1u;
      }
    }
  } else if (warp == 1) {
    constexpr uint32_t idesc = make_idesc_s8(TILE_W, BN);
    int s = 0;
    uint32_t ph = 0;
    bool ready = false;
    for (int i = 0; i < nkb; ++i) {
      if (!mbar_wait_warp(smem_u32(&full_bar[s]), ph, abortp, ready)) {
        if (status && lane == 0) atomicCAS(status, ST_OK, ST_TIMEOUT_MMA);
        break;
      }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t sW = tiles + s * SL::STAGE_BYTES, empty = smem_u32(&empty_bar[s]);
      if (++s == stages) {
        s = 0;
        ph ^= 1u;
      }
      ready = mbar_peek_warp(smem_u32(&full_bar[s]), ph);
      if (elect_one()) {
        const uint64_t dW = make_smem_desc(sW), dA = make_smem_desc(sW + W_STAGE_BYTES);
#pragma unroll
        for (int k = 0; k < S8_K / 32; ++k)   // 32 bytes along K inside the swizzle row
          umma_s8(tmem_d, dW + (uint64_t)(2 * k), dA + (uint64_t)(2 * k), idesc, (i > 0 || k > 0) ? 1u : 0u);
        umma_commit(empty);
        if (i == nkb - 1) umma_commit(smem_u32(&accum_bar));
      }
      __syncwarp();
    }
  }
  __syncwarp();

  const bool have = mbar_wait(smem_u32(&accum_bar), 0u, abortp);
  if (!have && threadIdx.x == 0 && status) atomicCAS(status, ST_OK, ST_TIMEOUT_EPI);
  const bool warp_ok = __all_sync(0xffffffffu, have);   // the TMEM loads are warp-collective
  constexpr int W = BN / 2;
  const int half = (int)threadIdx.x >> 7, tl = (int)threadIdx.x & 127, S = (int)gridDim.z;
  const uint32_t tmem_h = tmem_d + (uint32_t)(half * W);
  if (!warp_ok) drain_delay();
  if (S == 1) {
    if (warp_ok) s8_epilogue<W, T>(tmem_h, tl, m0 + half * W, n0, M, N, sa, sw, out, nullptr);
  } else {
    int* const ex = reinterpret_cast<int*>(smem_raw + (tiles - smem_u32(smem_raw)));   // [BN][128]
    const int rows = min(BN, M - m0);
    if (warp_ok) {
      const uint32_t tmem_w = tmem_h + ((uint32_t)(tl >> 5) << 21);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
      for (int c0 = 0; c0 < W && half * W + c0 < rows; c0 += 16) {
        uint32_t r[16];
        tmem_ld16(tmem_w + (uint32_t)c0, r);
        tmem_ld16_wait(r);
#pragma unroll
        for (int j = 0; j < 16; ++j) ex[(half * W + c0 + j) * 128 + tl] = (int)r[j];
      }
    }
    cluster_sync();
    const int rank = (int)cluster_ctarank(), n = n0 + lane * 4;   // four columns per lane, a row per warp
    const int gave_up = lane < S ? remote(&abort_flag, lane) : 0;   // one of the ranges: the tile stays as it was
    float w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = n + e < N ? sw[n + e] : 0.f;
    const bool whole = n + 4 <= N && !(N & 3) && !((uintptr_t)out & (4 * sizeof(T) - 1));
    for (int row = rank + warp * S; row < rows; row += S * (S8_THREADS / 32)) {
      const uint32_t at = tiles + (uint32_t)(row * 128 + lane * 4) * 4u;
      int4 sum = make_int4(0, 0, 0, 0);
#pragma unroll
      for (int s = 0; s < S8_MOST_SPLITS; ++s) {
        if (s >= S) break;
        const int4 x = remote4(cluster_addr(at, s));
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
      }
      if (__any_sync(0xffffffffu, gave_up != 0)) break;   // (requested together with the integers)
      const float a = sa[m0 + row], y[4] = {__int2float_rn(sum.x) * a * w[0], __int2float_rn(sum.y) * a * w[1],
                                            __int2float_rn(sum.z) * a * w[2], __int2float_rn(sum.w) * a * w[3]};
      T* const dst = out + (size_t)(m0 + row) * N + n;
      if (whole) {
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(dst) = make_float4(y[0], y[1], y[2], y[3]);
        } else {
          const __nv_bfloat162 lo = __floats2bfloat162_rn(y[0], y[1]), hi = __floats2bfloat162_rn(y[2], y[3]);
          *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < N) dst[e] = from_f32<T>(y[e]);
      }
    }
    cluster_sync();   // no CTA leaves while another one reads its integers
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_d), "r"((uint32_t)BN) : "memory");
}

// The pair kernel's form.
template <typename T>
struct S8Form {
  const float *sa, *sw;
  T* out;
  int split;
  static constexpr int GROUPS = 2;
  template <int W>
  static constexpr uint32_t ex_bytes() { return 0; }
  template <int W>
  struct Shared {};
  template <int W>
  __device__ __forceinline__ void ahead(Shared<W>&, int, int, int) const {}
  template <int W>
  __device__ __forceinline__ void drain(Shared<W>&, uint32_t tmem_d, float*, int tl, int, int m0, int n0, int, int M, int N,
                                        float* slab) const {
    s8_epilogue<W, T>(tmem_d, tl, m0, n0, M, N, sa, sw, out, split ? reinterpret_cast<int*>(slab) : nullptr);
  }
};
template <typename T>
struct PairOperands<S8Form<T>> {
  static constexpr int STAGE_K = S8_K;
  static __host__ __device__ constexpr uint32_t idesc(int m, int n) { return make_idesc_s8(m, n); }
  static __device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    umma_s8_pair(d, a, b, idesc, accumulate);
  }
};

// Sum of a split product's slabs, scaled.
template <typename T>
__global__ void __launch_bounds__(256) s8_finish_kernel(const int* __restrict__ slabs, int S, const float* __restrict__ sa,
                                                        const float* __restrict__ sw, T* __restrict__ out, int M, int N) {
  pdl_wait();
  pdl_trigger();
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= N) return;
  const size_t slab = (size_t)M * N;
  const float w = sw[n];
  for (int m = blockIdx.y; m < M; m += gridDim.y) {
    const int* p = slabs + (size_t)m * N + n;
    int sum = 0;
    for (int s = 0; s < S; ++s) sum += __ldcg(p + s * slab);
    out[(size_t)m * N + n] = from_f32<T>(__int2float_rn(sum) * sa[m] * w);
  }
}

// ---------------------------------------------------------------- rows of 8-bit integers
// A CTA per row; QS_VECS vectors of eight elements per thread stay in registers as they were loaded between the row's maximum
// and its codes, what is beyond them is read twice.  VEC: rows start on 16-byte boundaries.
constexpr int QS_VECS = 4;
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    a = make_float4(v[0], v[1], v[2], v[3]);
    b = make_float4(v[4], v[5], v[6], v[7]);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  // largest |x| as its bits: an infinity above every number, a NaN above that
  __device__ __forceinline__ uint32_t top() const {
    float v[8];
    get(v);
    uint32_t t = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) t = max(t, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    return t;
  }
};
template <>
struct Raw8<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void set(const float (&v)[8]) {   // (numbers that were bf16)
    a = make_uint4(__byte_perm(__float_as_uint(v[0]), __float_as_uint(v[1]), 0x7632),
                   __byte_perm(__float_as_uint(v[2]), __float_as_uint(v[3]), 0x7632),
                   __byte_perm(__float_as_uint(v[4]), __float_as_uint(v[5]), 0x7632),
                   __byte_perm(__float_as_uint(v[6]), __float_as_uint(v[7]), 0x7632));
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ uint32_t top() const {   // two 16-bit magnitudes per instruction
    const uint32_t t = __vmaxu2(__vmaxu2(a.x & 0x7FFF7FFFu, a.y & 0x7FFF7FFFu), __vmaxu2(a.z & 0x7FFF7FFFu, a.w & 0x7FFF7FFFu));
    return max(t << 16, t & 0xFFFF0000u);
  }
};
template <typename T, bool VEC>
__device__ __forceinline__ Raw8<T> load_upto8(const T* p, int left) {
  Raw8<T> r;
  if (VEC && left >= 8) {
    r.load(p);
  } else {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? to_f32<T>(p[i]) : 0.f;
    r.set(v);
  }
  return r;
}
template <typename T, bool VEC>
__global__ void __launch_bounds__(1024) quantize_rows_s8_kernel(const T* __restrict__ x, size_t ldx, int8_t* __restrict__ q,
                                                                size_t ldq, float* __restrict__ scale, int cols) {
  __shared__ uint32_t red[32];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, step = blockDim.x * 8;
  const T* row = x + (size_t)blockIdx.x * ldx;
  int8_t* dst = q + (size_t)blockIdx.x * ldq;
  Raw8<T> v[QS_VECS];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < QS_VECS; ++i) v[i] = load_upto8<T, VEC>(row + tid * 8 + i * step, cols - (tid * 8 + i * step));
#pragma unroll
  for (int i = 0; i < QS_VECS; ++i) top = max(top, v[i].top());
  for (int c = tid * 8 + QS_VECS * step; c < cols; c += step) top = max(top, load_upto8<T, VEC>(row + c, cols - c).top());
  top = __reduce_max_sync(0xffffffffu, top);
  if ((tid & 31) == 0) red[tid >> 5] = top;
  __syncthreads();
  top = __reduce_max_sync(0xffffffffu, (tid & 31) < (blockDim.x >> 5) ? red[tid & 31] : 0u);
  const float s = __fdiv_rn(__uint_as_float(top), 127.f);
  const bool zero = s == 0.f || top >= 0x7F800000u;   // codes 0; the scale then shows an infinity or a NaN
  if (tid == 0) scale[blockIdx.x] = s;
  // The IEEE quotient by a product with the reciprocal and two corrections: behind the first it is within a unit of its last
  // place, and with a correctly rounded reciprocal the second is then the correctly rounded quotient (Markstein, 1990; not for
  // a divisor of ones alone, nor where a remainder leaves fp32's range: those are divided).  Rounded to an integer by adding
  // 1.5 * 2^23.  (A test for near ties with divisions behind it: bf16 rows, whose maximum is a bf16 number, meet one in nearly
  // every warp; 8192 x 12288 148 us, 112 so, 57 with rows kept as they were loaded and two numbers an instruction.)
  const bool divide = s < 1e-28f || !(s < INFINITY) || (__float_as_uint(s) & 0x7FFFFFu) == 0x7FFFFFu;
  const float inv = __frcp_rn(s);
  const float2 inv2 = make_float2(inv, inv), minus = make_float2(-s, -s), up = make_float2(12582912.f, 12582912.f);
  auto put = [&](int c, const Raw8<T>& raw) {
    float u[8];
    raw.get(u);
    uint32_t code[8];
    if (!divide) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {   // two at a time, each as fp32's own operations
        const float2 x = make_float2(u[e], u[e + 1]);
        float2 p = mul2(x, inv2);
        p = fma2(fma2(p, minus, x), inv2, p);
        p = add2(fma2(fma2(p, minus, x), inv2, p), up);
        code[e] = __float_as_uint(p.x);
        code[e + 1] = __float_as_uint(p.y);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        code[e] = zero ? 0u : (uint32_t)(int)fminf(fmaxf(rintf(__fdiv_rn(u[e], s)), -127.f), 127.f);
    }
    if (c + 8 <= cols) {
      uint2 w;
      w.x = __byte_perm(__byte_perm(code[0], code[1], 0x0040), __byte_perm(code[2], code[3], 0x0040), 0x5410);
      w.y = __byte_perm(__byte_perm(code[4], code[5], 0x0040), __byte_perm(code[6], code[7], 0x0040), 0x5410);
      *reinterpret_cast<uint2*>(dst + c) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < cols) dst[c + e] = (int8_t)code[e];
    }
  };
#pragma unroll
  for (int i = 0; i < QS_VECS; ++i)
    if (tid * 8 + i * step < cols) put(tid * 8 + i * step, v[i]);
  for (int c = tid * 8 + QS_VECS * step; c < cols; c += step) put(c, load_upto8<T, VEC>(row + c, cols - c));
}

template <int BN, bool ONCE, typename T>
cudaError_t launch_one_s8(const Launch& L, const CUtensorMap& tmW, const CUtensorMap& tmA, const float* sa, const float* sw,
                          T* out, int M, int N, const GemmPlan& plan) {
  using SL = S8Layout<BN>;
  static DeviceOnce once;
  cudaError_t e0 = once.run([] {
    return cudaFuncSetAttribute(gemm_s8_kernel<BN, ONCE, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)SL::total(SL::most()));
  });
  if (e0 != cudaSuccess) return e0;
  const int stages = plan.stages < 2 ? 2 : plan.stages > SL::most() ? SL::most() : plan.stages;
  const dim3 grid(plan.m_tiles, (N + TILE_W - 1) / TILE_W, plan.S_max);
  cudaError_t e = plan.S_max == 1 ? launch_k(L, gemm_s8_kernel<BN, ONCE, T>, grid, dim3(S8_THREADS), SL::total(stages), tmW, tmA,
                                             sa, sw, out, M, N, plan.num_kb, plan.upc, stages, L.d_status)
                                  : launch_k_cluster(L, gemm_s8_kernel<BN, ONCE, T>, grid, dim3(S8_THREADS), SL::total(stages),
                                                     dim3(1, 1, plan.S_max), tmW, tmA, sa, sw, out, M, N, plan.num_kb, plan.upc,
                                                     stages, L.d_status);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T>
cudaError_t launch_as(const Launch& L, const CUtensorMap& tmW, const CUtensorMap& tmA, const float* sa, const float* sw, T* out,
                      int* slabs, int M, int N, const GemmPlan& plan) {
  int* const part = plan.S_max > 1 ? slabs : nullptr;
  const bool once = plan.w_stream && plan.m_tiles == 1;
  cudaError_t e;
  if (plan.pair) {
    const S8Form<T> form{sa, sw, out, part != nullptr};
    float* const slab = reinterpret_cast<float*>(part);
    if (plan.BN == 128)
      e = launch_pair_form<128, false>(L, tmW, tmA, slab, M, N, plan.num_kb, plan, form, false);
    else if (plan.BN == 192)
      e = once ? launch_pair_form<192, true>(L, tmW, tmA, slab, M, N, plan.num_kb, plan, form, false)
               : launch_pair_form<192, false>(L, tmW, tmA, slab, M, N, plan.num_kb, plan, form, false);
    else
      e = once ? launch_pair_form<256, true>(L, tmW, tmA, slab, M, N, plan.num_kb, plan, form, false)
               : launch_pair_form<256, false>(L, tmW, tmA, slab, M, N, plan.num_kb, plan, form, false);
  } else if (plan.BN == 32) {
    e = once ? launch_one_s8<32, true, T>(L, tmW, tmA, sa, sw, out, M, N, plan)
             : launch_one_s8<32, false, T>(L, tmW, tmA, sa, sw, out, M, N, plan);
  } else if (plan.BN == 64) {
    e = once ? launch_one_s8<64, true, T>(L, tmW, tmA, sa, sw, out, M, N, plan)
             : launch_one_s8<64, false, T>(L, tmW, tmA, sa, sw, out, M, N, plan);
  } else {
    e = launch_one_s8<128, false, T>(L, tmW, tmA, sa, sw, out, M, N, plan);
  }
  if (e != cudaSuccess || !part || !plan.pair) return e;
  Launch behind = L;
  behind.pdl = true;
  const dim3 grid((N + 255) / 256, std::min(M, 4096));
  e = launch_k(behind, s8_finish_kernel<T>, grid, dim3(256), 0, (const int*)part, plan.S_max, sa, sw, out, M, N);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// Tile, ring and split, from sweeps on B200 (products alone, bf16 out, weights not in L2, us).
//   up to 32 rows   one CTA per 128 weight rows, k split until there is one per SM: 3 x 4096 x 4096 in 3 / 4 / 5 ranges 8.3 /
//                   8.0 / 7.8
//   up to 64        tiles of 64 rows; ranges by powers of two (clusters of five or six leave SMs idle): 64 x 4096 x 4096 in 4
//                   9.5, in 5 9.7; a ring of eight stages where a CTA has its SM for itself (64 x 12288 x 4096 15.8 -> 14.6)
//   up to 128       two tiles of 64 rows where the weight tiles are few (128 x 4608 x 3584 10.5 against 11.8), one of 128
//                   otherwise (128 x 37888 x 3584 31.2 against 34.6); CTAs, two to an SM, at most nine tenths of the places:
//                   72 tiles in 2 ranges 10.5, in 4 15.3
//   up to 256       tiles of 128 rows in 2 or 4 ranges where they fit so (256 x 4096 x 4096 12.9 against 14.9 on pairs), else
//   and above       CTA pairs, by what a unit's stages take (issue or bytes, as for bf16: a stage is the same bytes and cycles)
//                   and a split's slabs with the launch that adds them: 256 x 24576 x 4096 33 against 38 in tiles of one CTA,
//                   768 x 4096 x 12288 33 against 42, 8192 x 24576 x 4096 505 against 980
GemmPlan plan_gemm_s8(int M, int N, int K) {
  GemmPlan p;
  const int sms = sm_count(), pairs = sms / 2;
  const long n_tiles = (N + TILE_W - 1) / TILE_W, n_pairs = (N + 2 * TILE_W - 1) / (2 * TILE_W), places = 2L * sms * 9 / 10;
  p.num_kb = (K + S8_K - 1) / S8_K;
  p.w_stream = (long)N * K >= 16L << 20;
  int S = 1;
  auto ranges = [&](long tiles, long room) {   // the largest power of two that fits, four stages each at least
    int s = 1;
    while (2 * s <= S8_MOST_SPLITS && tiles * 2 * s <= room && p.num_kb >= 8 * s) s *= 2;
    return s;
  };
  if (M <= 32) {
    p.BN = 32;
    S = std::max(1, std::min({(int)((sms + n_tiles - 1) / n_tiles), p.num_kb / 4, S8_MOST_SPLITS}));
  } else if (M <= 64) {
    p.BN = 64;
    S = ranges(n_tiles, sms);
  } else if (M <= 128) {
    p.BN = 2 * n_tiles <= sms ? 64 : 128;
    S = ranges(n_tiles * ((M + p.BN - 1) / p.BN), places);
  } else if (M <= 256 && 4 * n_tiles <= places) {
    p.BN = 128;
    S = ranges(2 * n_tiles, places);
  } else {
    p.pair = 1;
    double best = -1.0;
    for (int BN : {256, 192, 128}) {
      const long tiles = n_pairs * ((M + BN - 1) / BN);
      const double issue = BN == 256 ? 0.33 : BN == 192 ? 0.27 : 0.25, bytes = (TILE_W + BN / 2) * (double)S8_K;
      for (int s = 1; s == 1 || (s <= 16 && s * tiles <= pairs && s <= p.num_kb / 4); ++s) {
        const long units = tiles * s, rounds = (units + pairs - 1) / pairs;
        const double ctas = 2.0 * (units < pairs ? units : pairs), fabric = bytes * ctas / 12.0e6;
        const double us = (double)rounds * ((p.num_kb + s - 1) / s) * (issue > fabric ? issue : fabric) +
                          (s > 1 ? 3.0 + s * (double)M * N * 8.0 / 10.0e6 : 0.0);
        if (best < 0.0 || us < best) {
          best = us;
          p.BN = BN;
          S = s;
        }
      }
    }
  }
  p.m_tiles = (M + p.BN - 1) / p.BN;
  p.stages = p.pair ? MAX_STAGES : p.BN == 128 ? 3 : n_tiles * p.m_tiles * S <= sms && p.BN == 64 ? 8 : 4;
  p.upc = (p.num_kb + S - 1) / S;
  p.S_max = (p.num_kb + p.upc - 1) / p.upc;
  return p;
}

size_t gemm_s8_scratch_bytes(int M, int N, const GemmPlan& plan) {
  return plan.pair && plan.S_max > 1 ? (size_t)plan.S_max * M * N * 4 : 0;   // one-tile CTAs add up in shared memory
}

cudaError_t launch_gemm_s8(const Launch& L, const int8_t* A, size_t lda, const float* sa, const int8_t* W, size_t ldw,
                           const float* sw, void* out, int out_dtype, int M, int N, int K, const GemmPlan& plan, void* scratch,
                           const char** err) {
  CUtensorMap tmW, tmA;
  if (!make_tensor_map_s8(W, (uint64_t)N, (uint64_t)K, ldw, TILE_W, &tmW) ||
      !make_tensor_map_s8(A, (uint64_t)M, (uint64_t)K, lda, (uint32_t)(plan.pair ? plan.BN / 2 : plan.BN), &tmA)) {
    if (err) *err = "cuTensorMapEncodeTiled failed or is unavailable";
    return cudaErrorInvalidValue;
  }
  return out_dtype == DLLM_BF16 ? launch_as(L, tmW, tmA, sa, sw, (__nv_bfloat16*)out, (int*)scratch, M, N, plan)
                                : launch_as(L, tmW, tmA, sa, sw, (float*)out, (int*)scratch, M, N, plan);
}

template <typename T>
static cudaError_t quantize_as(const Launch& L, const T* x, size_t ldx, int8_t* q, size_t ldq, float* scale, int rows, int cols) {
  const int want = (cols + 8 * QS_VECS - 1) / (8 * QS_VECS), threads = std::min(1024, std::max(64, (want + 31) / 32 * 32));
  const bool vec = !((uintptr_t)x & 15) && !(ldx * sizeof(T) & 15);
  cudaError_t e = vec ? launch_k(L, quantize_rows_s8_kernel<T, true>, dim3(rows), dim3(threads), 0, x, ldx, q, ldq, scale, cols)
                      : launch_k(L, quantize_rows_s8_kernel<T, false>, dim3(rows), dim3(threads), 0, x, ldx, q, ldq, scale, cols);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_quantize_rows_s8(const Launch& L, const void* x, size_t ldx, int dtype, int8_t* q, size_t ldq, float* scale,
                                    int rows, int cols) {
  return dtype == DLLM_BF16 ? quantize_as(L, (const __nv_bfloat16*)x, ldx, q, ldq, scale, rows, cols)
                            : quantize_as(L, (const float*)x, ldx, q, ldq, scale, rows, cols);
}

}  // namespace dllm

namespace dllm {
cudaError_t set_debug_skip_gemm_s8(int enable) {
  const int v = enable != 0;
  return cudaMemcpyToSymbol(g_debug_skip, &v, sizeof v);
}
}  // namespace dllm

DLLM_WAIT_LIMIT_HOOK(gemm_s8)
