// Rows of the 4-bit K / V cache: into it, out of it, and out of the way.
//
//   store   lo = bf16(min x), step = bf16((max x - min x) / 15) or 1 where that is 0, code = rint((x - lo) / step) clamped
//           to 0..15, all in fp32 with IEEE divisions.  A row that holds an infinity or a NaN gets NaN for both, so that
//           whatever reads it shows it.
//   load    lo + step * code in one rounding.
//   evict   per (sequence, KV head): keys that stay = the first and the last ones asked for and, of the others, those with
//           the largest weights (equal ones: lowest index), moved up in their order.
//
// All three move bytes: they are bound by HBM (store and load of many rows) or by their launches (a step's rows).
#include <algorithm>

#include "kv4.cuh"

namespace dllm {

namespace {

// Eight elements of a row.  VEC: the row starts on a 16-byte boundary.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (VEC) {
    Vec8<T>::load(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32<T>(p[i]);
  }
}

// The codes of eight elements per lane, LANES lanes per row, and the row's pair.
template <int LANES>
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], uint32_t& pair) {
  float lo = x[0], hi = x[0], odd = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    odd += x[i] - x[i];   // 0, or NaN for an infinity or a NaN
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    odd += __shfl_xor_sync(0xffffffffu, odd, o);
  }
  const __nv_bfloat16 lo_b = __float2bfloat16_rn(lo);
  __nv_bfloat16 step_b = __float2bfloat16_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.f));
  if (__bfloat162float(step_b) == 0.f) step_b = __float2bfloat16_rn(1.f);
  const float lo_f = __bfloat162float(lo_b), step = __bfloat162float(step_b);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float u = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x[i], lo_f), step)), 0.f), 15.f);
    w |= (uint32_t)u << (4 * i);
  }
  pair = (uint32_t)__bfloat16_as_ushort(step_b) | ((uint32_t)__bfloat16_as_ushort(lo_b) << 16);
  // also where the spread overflows: no step stands for it
  if (odd != 0.f || !(step < INFINITY) || !(fabsf(lo_f) < INFINITY)) {
    pair = 0x7FC07FC0u;
    w = 0;
  }
  return w;
}

// A CTA takes `per` consecutive source rows (of all sequences together), LANES lanes per head of a row.  Rows whose
// position lies outside the cache are left out.  A position named twice goes to the last row that names it: a CTA looks
// through the positions behind its own rows, with a bit per position modulo 1024 in front of the exact comparison.
constexpr int ST_THREADS = 256, ST_ROWS = 32;
template <typename T, int HD, bool VEC>
__global__ void __launch_bounds__(ST_THREADS) kv4_store_kernel(Kv4 c, const T* __restrict__ k, const T* __restrict__ v,
                                                               size_t ldk, size_t ldv, int a, int rows, int per,
                                                               const int32_t* __restrict__ pos, int start) {
  constexpr int LANES = HD / 8;
  __shared__ int at[ST_ROWS];          // where row r goes, -1: nowhere
  __shared__ uint32_t bits[32];
  pdl_wait();
  pdl_trigger();
  const int r0 = blockIdx.x * per, mine = min(per, rows - r0), tid = threadIdx.x;
  if (tid < 32) bits[tid] = 0;
  __syncthreads();
  if (tid < mine) {
    const int r = r0 + tid, p = pos ? pos[r] : start + r % a;
    at[tid] = p >= 0 && p < c.cap ? p : -1;
    if (pos && at[tid] >= 0) atomicOr(&bits[(p >> 5) & 31], 1u << (p & 31));
  }
  __syncthreads();
  if (pos) {
    const int seq_end = ((r0 + mine - 1) / a + 1) * a;   // end of the last sequence this CTA has rows of
    for (int r = r0 + 1 + tid; r < seq_end; r += ST_THREADS) {
      const int p = pos[r];
      if (p < 0 || !((bits[(p >> 5) & 31] >> (p & 31)) & 1u)) continue;
      for (int i = 0; i < mine && r0 + i < r; ++i)
        if ((r0 + i) / a == r / a && pos[r0 + i] == p) at[i] = -1;
    }
    __syncthreads();
  }
  const int heads = mine * c.Hkv, lane = tid % LANES;
  // every lane of a warp takes part in the shuffles: the trips are rounded up
  for (int i0 = 0; i0 < heads; i0 += ST_THREADS / LANES) {
    const int i = i0 + tid / LANES;
    const bool live = i < heads;
    const int r = live ? i / c.Hkv : 0, h = live ? i - r * c.Hkv : 0;
    float x[8], y[8];
    load8<T, VEC>(k + (size_t)(r0 + r) * ldk + h * HD + lane * 8, x);
    load8<T, VEC>(v + (size_t)(r0 + r) * ldv + h * HD + lane * 8, y);
    uint32_t kpair, vpair;
    const uint32_t kw = encode8<LANES>(x, kpair), vw = encode8<LANES>(y, vpair);
    if (!live || at[r] < 0) continue;
    const size_t row = ((size_t)((r0 + r) / a) * c.Hkv + h) * c.cap + at[r];
    reinterpret_cast<uint32_t*>(c.k)[row * LANES + lane] = kw;
    reinterpret_cast<uint32_t*>(c.v)[row * LANES + lane] = vw;
    if (lane == 0) {
      c.kp[row] = kpair;
      c.vp[row] = vpair;
    }
  }
}

// One word of eight codes per thread and trip; blockIdx.y: K or V.
template <typename T, int HD, bool VEC>
__global__ void __launch_bounds__(256) kv4_load_kernel(Kv4 c, int n, const int32_t* __restrict__ lens, T* __restrict__ k,
                                                       T* __restrict__ v) {
  constexpr int LANES = HD / 8;
  pdl_wait();
  pdl_trigger();
  const bool of_v = blockIdx.y != 0;
  T* out = of_v ? v : k;
  if (!out) return;
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(of_v ? c.v : c.k);
  const uint32_t* pairs = of_v ? c.vp : c.kp;
  const size_t words = (size_t)c.B * n * c.Hkv * LANES;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (size_t)gridDim.x * 256) {
    const int lane = (int)(i % LANES);
    const size_t head = i / LANES, token = head / c.Hkv;
    const int h = (int)(head - token * c.Hkv), b = (int)(token / n), j = (int)(token - (size_t)b * n);
    float x[8];
    if (lens && j >= lens[b]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
    } else {
      const size_t row = ((size_t)b * c.Hkv + h) * c.cap + j;
      const uint32_t w = codes[row * LANES + lane], p = pairs[row];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = fmaf((float)((w >> (4 * e)) & 15u), kv4_step(p), kv4_lo(p));
    }
    if constexpr (VEC) {
      Vec8<T>::store(out + i * 8, x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) out[i * 8 + e] = from_f32<T>(x[e]);
    }
  }
}

// ---------------------------------------------------------------- eviction
constexpr int EV_THREADS = 1024, EV_PER = 8, EV_BINS = 2048;

// Order of the weights as unsigned numbers; a NaN comes last, -0 and 0 are equal.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int block_scan(int v, int* warps, int& total) {   // exclusive; EV_THREADS threads
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += t;
  }
  __syncthreads();
  if (lane == 31) warps[w] = s;
  __syncthreads();
  int before = 0, all = 0;
  {
    int t = warps[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += u;
    }
    all = __shfl_sync(0xffffffffu, t, 31);
    before = __shfl_sync(0xffffffffu, t, w == 0 ? 0 : w - 1);
    if (w == 0) before = 0;
  }
  total = all;
  return before + s - v;
}

// One CTA per (sequence, KV head).  The smallest weight that stays is found digit by digit (11, 11 and 10 bits of the
// ordered weight, a histogram each), then one pass in order writes the places.
__global__ void __launch_bounds__(EV_THREADS) kv4_select_kernel(const float* __restrict__ weight, int n, int cap, int Hkv,
                                                                int keep, int first, int last,
                                                                const int32_t* __restrict__ lens, int dst_cap,
                                                                float* __restrict__ dst_weight, int32_t* __restrict__ index,
                                                                int32_t* __restrict__ new_lens) {
  __shared__ int hist[EV_BINS];
  __shared__ int warps[32];
  __shared__ uint32_t s_prefix;
  __shared__ int s_need;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, bh = blockIdx.x, b = bh / Hkv;
  const float* w = weight + (size_t)bh * cap;
  const int len = lens ? min(max(lens[b], 0), n) : n, kept = min(len, keep);
  const bool choose = len > keep;                       // else every key stays
  const int lo = choose ? first : len, hi = choose ? len - last : len;   // keys lo .. hi - 1 compete
  int need = choose ? keep - first - last : 0;          // for this many places
  uint32_t prefix = 0, mask = 0;                        // digits of the threshold found so far
  if (need > 0) {
    for (int shift = 21; ; ) {
      for (int i = tid; i < EV_BINS; i += EV_THREADS) hist[i] = 0;
      __syncthreads();
      const int bins = shift == 0 ? 1024 : 2048;
      for (int j0 = lo / 4 * 4 + tid * 4; j0 < hi; j0 += EV_THREADS * 4) {
        const float4 x = *reinterpret_cast<const float4*>(w + j0);
        const float e[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t key = weight_key(e[q]);
          if (j0 + q >= lo && j0 + q < hi && (key & mask) == prefix) atomicAdd(&hist[(key >> shift) & (bins - 1)], 1);
        }
      }
      __syncthreads();
      // the bin, counted from the largest, in which the last place goes: bins in pairs per thread, largest first
      const int top = EV_BINS - 1 - 2 * tid, c0 = hist[top], c1 = hist[top - 1];
      int total;
      const int before = block_scan(c0 + c1, warps, total);
      if (before < need && need <= before + c0) {
        s_prefix = (uint32_t)top;
        s_need = need - before;
      } else if (before + c0 < need && need <= before + c0 + c1) {
        s_prefix = (uint32_t)(top - 1);
        s_need = need - before - c0;
      }
      __syncthreads();
      prefix |= s_prefix << shift;
      mask |= (uint32_t)(bins - 1) << shift;
      need = s_need;
      __syncthreads();
      if (shift == 0) break;
      shift = shift == 21 ? 10 : 0;
    }
  }
  // `need` of the keys equal to `prefix` stay, the first ones
  int32_t* idx = index + (size_t)bh * keep;
  float* dw = dst_weight + (size_t)bh * dst_cap;
  int sure_before = 0, ties_before = 0;
  for (int base = 0; base < len; base += EV_THREADS * EV_PER) {
    const int j0 = base + tid * EV_PER;
    float e[EV_PER];
    uint32_t sure = 0, tie = 0;
#pragma unroll
    for (int q = 0; q < EV_PER; q += 4) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (j0 + q < len) x = *reinterpret_cast<const float4*>(w + j0 + q);
      e[q] = x.x; e[q + 1] = x.y; e[q + 2] = x.z; e[q + 3] = x.w;
    }
#pragma unroll
    for (int q = 0; q < EV_PER; ++q) {
      const int j = j0 + q;
      if (j >= len) continue;
      const uint32_t key = weight_key(e[q]);
      const bool forced = j < lo || j >= hi;
      if (forced || (mask && key > prefix)) sure |= 1u << q;
      else if (mask && key == prefix) tie |= 1u << q;
    }
    int total;
    const int scan = block_scan((__popc(sure) << 16) | __popc(tie), warps, total);
    int s = sure_before + (scan >> 16), t = ties_before + (scan & 0xFFFF);
#pragma unroll
    for (int q = 0; q < EV_PER; ++q) {
      const bool is_sure = (sure >> q) & 1u, is_tie = (tie >> q) & 1u;
      if (is_sure || (is_tie && t < need)) {
        const int slot = s + min(t, need);
        idx[slot] = j0 + q;
        dw[slot] = e[q];
      }
      s += is_sure;
      t += is_tie;
    }
    sure_before += total >> 16;
    ties_before += total & 0xFFFF;
  }
  for (int i = kept + tid; i < dst_cap; i += EV_THREADS) {
    if (i < keep) idx[i] = -1;
    dw[i] = 0.f;
  }
  if (tid == 0 && bh % Hkv == 0) new_lens[b] = kept;
}

// The rows that stay, 16 bytes per thread: HD / 32 threads for K and as many for V, the first of each with the pair.
template <int HD>
__global__ void __launch_bounds__(256) kv4_gather_kernel(Kv4 src, Kv4 dst, const int32_t* __restrict__ index, int keep) {
  constexpr int CH = HD / 32, PER = 2 * CH;
  pdl_wait();
  pdl_trigger();
  const int bh = blockIdx.y, unit = blockIdx.x * 256 + threadIdx.x, slot = unit / PER, part = unit % PER;
  if (slot >= keep) return;
  const int j = index[(size_t)bh * keep + slot];
  if (j < 0) return;
  const size_t from = (size_t)bh * src.cap + j, to = (size_t)bh * dst.cap + slot;
  const bool of_v = part >= CH;
  const int c = of_v ? part - CH : part;
  const uint4 x = reinterpret_cast<const uint4*>(of_v ? src.v : src.k)[from * CH + c];
  reinterpret_cast<uint4*>(of_v ? dst.v : dst.k)[to * CH + c] = x;
  if (c == 0) (of_v ? dst.vp : dst.kp)[to] = (of_v ? src.vp : src.kp)[from];
}

template <typename T, int HD>
cudaError_t store_as(const Launch& L, const Kv4& c, const T* k, const T* v, size_t ldk, size_t ldv, int a, const int32_t* pos,
                     int start) {
  const int rows = c.B * a, per = std::max(1, std::min(ST_ROWS, rows / (4 * sm_count())));
  const bool vec = !(((uintptr_t)k | (uintptr_t)v) & 15) && !((ldk | ldv) * sizeof(T) & 15);
  const dim3 grid((rows + per - 1) / per);
  cudaError_t e = vec ? launch_k(L, kv4_store_kernel<T, HD, true>, grid, dim3(ST_THREADS), 0, c, k, v, ldk, ldv, a, rows, per,
                                 pos, start)
                      : launch_k(L, kv4_store_kernel<T, HD, false>, grid, dim3(ST_THREADS), 0, c, k, v, ldk, ldv, a, rows,
                                 per, pos, start);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T, int HD>
cudaError_t load_as(const Launch& L, const Kv4& c, int n, const int32_t* lens, T* k, T* v) {
  const size_t words = (size_t)c.B * n * c.Hkv * (HD / 8);
  const dim3 grid((unsigned)std::min<size_t>((words + 255) / 256, (size_t)sm_count() * 16), 2);
  const bool vec = !(((uintptr_t)k | (uintptr_t)v) & 15);
  cudaError_t e = vec ? launch_k(L, kv4_load_kernel<T, HD, true>, grid, dim3(256), 0, c, n, lens, k, v)
                      : launch_k(L, kv4_load_kernel<T, HD, false>, grid, dim3(256), 0, c, n, lens, k, v);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv4_store(const Launch& L, const Kv4& c, const void* k, const void* v, size_t ldk, size_t ldv, int dtype,
                             int a, const int32_t* pos, int start) {
  auto go = [&](auto* t, auto hd) {
    using T = std::remove_pointer_t<decltype(t)>;
    return store_as<T, decltype(hd)::value>(L, c, (const T*)k, (const T*)v, ldk, ldv, a, pos, start);
  };
  using H64 = std::integral_constant<int, 64>;
  using H128 = std::integral_constant<int, 128>;
  if (dtype == DLLM_BF16) return c.hd == 64 ? go((__nv_bfloat16*)nullptr, H64{}) : go((__nv_bfloat16*)nullptr, H128{});
  return c.hd == 64 ? go((float*)nullptr, H64{}) : go((float*)nullptr, H128{});
}

cudaError_t launch_kv4_load(const Launch& L, const Kv4& c, int n, const int32_t* lens, void* k, void* v, int dtype) {
  if (dtype == DLLM_BF16)
    return c.hd == 64 ? load_as<__nv_bfloat16, 64>(L, c, n, lens, (__nv_bfloat16*)k, (__nv_bfloat16*)v)
                      : load_as<__nv_bfloat16, 128>(L, c, n, lens, (__nv_bfloat16*)k, (__nv_bfloat16*)v);
  return c.hd == 64 ? load_as<float, 64>(L, c, n, lens, (float*)k, (float*)v)
                    : load_as<float, 128>(L, c, n, lens, (float*)k, (float*)v);
}

cudaError_t launch_kv4_evict(const Launch& L, const Kv4& src, const float* weight, int n, int keep, int first, int last,
                             const int32_t* lens, const Kv4& dst, float* dst_weight, int32_t* index, int32_t* new_lens) {
  const int heads = src.B * src.Hkv;
  cudaError_t e = launch_k(L, kv4_select_kernel, dim3(heads), dim3(EV_THREADS), 0, weight, n, src.cap, src.Hkv, keep, first,
                           last, lens, dst.cap, dst_weight, index, new_lens);
  L.count();
  if (e != cudaSuccess) return e;
  const int per = src.hd / 16;
  const dim3 grid((unsigned)(((size_t)keep * per + 255) / 256), heads);
  Launch behind = L;
  behind.pdl = true;   // its prologue overlaps the selection's tail; it waits for it before it reads anything
  e = src.hd == 64 ? launch_k(behind, kv4_gather_kernel<64>, grid, dim3(256), 0, src, dst, index, keep)
                   : launch_k(behind, kv4_gather_kernel<128>, grid, dim3(256), 0, src, dst, index, keep);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace dllm
