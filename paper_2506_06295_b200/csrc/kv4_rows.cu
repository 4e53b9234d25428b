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
#include "tma.cuh"
#include "umma.cuh"

namespace dllm {

namespace {

// Sixteen elements of a row and, over the LANES lanes that share it, the row's least and largest one (NaN where there is a
// NaN).  VEC: the row starts on a 16-byte boundary.  bf16: two numbers per instruction, and the pair (least, -largest) goes
// through the shuffles as one word.
template <int LANES, bool VEC>
__device__ __forceinline__ void load_row(const float* p, float (&x)[16], float& lo, float& hi) {
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + i);
      x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = p[i];
  }
  auto least = [](float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
  };
  float top = -x[0];
  lo = x[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) {
    lo = least(lo, x[i]);
    top = least(top, -x[i]);
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    lo = least(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    top = least(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  hi = -top;
}
template <int LANES, bool VEC>
__device__ __forceinline__ void load_row(const __nv_bfloat16* p, float (&x)[16], float& lo, float& hi) {
  uint32_t w[8];
  if constexpr (VEC) {
    const uint4 a = *reinterpret_cast<const uint4*>(p), b = *reinterpret_cast<const uint4*>(p + 8);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      w[i] = (uint32_t)__bfloat16_as_ushort(p[2 * i]) | (uint32_t)__bfloat16_as_ushort(p[2 * i + 1]) << 16;
  }
  auto as2 = [](uint32_t u) { return *reinterpret_cast<const __nv_bfloat162*>(&u); };
  __nv_bfloat162 least = as2(w[0]), most = as2(w[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    least = __hmin2_nan(least, as2(w[i]));
    most = __hmax2_nan(most, as2(w[i]));
  }
  __nv_bfloat162 both = __hmin2_nan(__lows2bfloat162(least, __hneg2(most)), __highs2bfloat162(least, __hneg2(most)));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1)
    both = __hmin2_nan(both, as2(__shfl_xor_sync(0xffffffffu, *reinterpret_cast<const uint32_t*>(&both), o)));
  lo = __low2float(both);
  hi = -__high2float(both);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// The codes of a lane's sixteen elements of a row with least `lo` and largest `hi`, and the row's pair.
__device__ __forceinline__ uint2 encode16(const float (&x)[16], float lo, float hi, uint32_t& pair) {
  const __nv_bfloat16 lo_b = __float2bfloat16_rn(lo);
  // The IEEE quotient by 15: a product with the rounded reciprocal and one correction (right for every significand there is,
  // where the product alone is off for 5.4 of 8.4 million), unless a remainder could leave fp32's range.
  const float spread = __fsub_rn(hi, lo);
  constexpr float FIFTEENTH = 1.f / 15.f;
  float q15 = __fmul_rn(spread, FIFTEENTH);
  q15 = __fmaf_rn(__fmaf_rn(-q15, 15.f, spread), FIFTEENTH, q15);
  if (spread < 1e-28f) q15 = __fdiv_rn(spread, 15.f);
  __nv_bfloat16 step_b = __float2bfloat16_rn(q15);
  if (__bfloat162float(step_b) == 0.f) step_b = __float2bfloat16_rn(1.f);
  const float lo_f = __bfloat162float(lo_b), step = __bfloat162float(step_b);
  // The quotient by a product with the reciprocal (to 2^-23) and one correction, rounded by adding 1.5 * 2^23.  The corrected
  // product is off by 2^-45 of itself before it is rounded, so it meets a tie exactly where the quotient does: half steps are
  // exact, and a step has 8 bits, so the quotient of the nearest other d is 2^-32 of itself away from where it would be rounded
  // to the tie.  This is rint of the IEEE quotient without its cost.  Rows that it does not hold for are divided: tiny and huge
  // steps, and fp32 rows whose offset was rounded by so much that quotients leave 0..15.  Four codes add up to 16 bits in fp32.
  // (Store of 16 x 1536 tokens of 32 heads, bf16, 78 us of bytes: 310 us with a division per element, 134 one element at a time,
  // 116 now.)
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(step));
  float u[16];
  if (lo >= lo_f && __fsub_rn(hi, lo_f) <= 15.4f * step && step > 1e-30f && step < 1e30f) {
    const float2 inv2 = make_float2(inv, inv), minus = make_float2(-step, -step), from = make_float2(-lo_f, -lo_f);
    const float2 up = make_float2(12582912.f, 12582912.f), down = make_float2(-12582912.f, -12582912.f);
#pragma unroll
    for (int i = 0; i < 16; i += 2) {   // two at a time, each as fp32's own operations
      const float2 d = add2(make_float2(x[i], x[i + 1]), from), p = mul2(d, inv2);
      const float2 r = add2(add2(fma2(fma2(p, minus, d), inv2, p), up), down);
      u[i] = r.x;
      u[i + 1] = r.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x[i], lo_f), step)), 0.f), 15.f);
  }
  uint32_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    q[i] = __float_as_uint(__fadd_rn(__fmaf_rn(__fmaf_rn(__fmaf_rn(u[4 * i + 3], 16.f, u[4 * i + 2]), 16.f, u[4 * i + 1]), 16.f, u[4 * i]),
                                     12582912.f));
  pair = (uint32_t)__bfloat16_as_ushort(step_b) | ((uint32_t)__bfloat16_as_ushort(lo_b) << 16);
  if (!(step < INFINITY) || !(fabsf(lo_f) < INFINITY)) {   // an infinity, a NaN, or a spread that no step stands for
    pair = 0x7FC07FC0u;
    return make_uint2(0, 0);
  }
  return make_uint2(__byte_perm(q[0], q[1], 0x5410), __byte_perm(q[2], q[3], 0x5410));
}

// A CTA takes `per` consecutive source rows (of all sequences together), LANES lanes per head of a row.  Rows whose
// position lies outside the cache are left out.  A position named twice goes to the last row that names it: a CTA looks
// through the positions behind its own rows, with a bit per position modulo 1024 in front of the exact comparison.
constexpr int ST_THREADS = 256, ST_ROWS = 32;
template <typename T, int HD, bool VEC>
__global__ void __launch_bounds__(ST_THREADS) kv4_store_kernel(Kv4 c, const T* __restrict__ k, const T* __restrict__ v,
                                                               size_t ldk, size_t ldv, int a, int rows, int per,
                                                               const int32_t* __restrict__ pos, int start) {
  constexpr int LANES = HD / 16;
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
    float x[16], y[16], x_lo, x_hi, y_lo, y_hi;
    load_row<LANES, VEC>(k + (size_t)(r0 + r) * ldk + h * HD + lane * 16, x, x_lo, x_hi);
    load_row<LANES, VEC>(v + (size_t)(r0 + r) * ldv + h * HD + lane * 16, y, y_lo, y_hi);
    uint32_t kpair, vpair;
    const uint2 kw = encode16(x, x_lo, x_hi, kpair), vw = encode16(y, y_lo, y_hi, vpair);
    if (!live || at[r] < 0) continue;
    const size_t row = ((size_t)((r0 + r) / a) * c.Hkv + h) * c.cap + at[r];
    reinterpret_cast<uint2*>(c.k)[row * LANES + lane] = kw;
    reinterpret_cast<uint2*>(c.v)[row * LANES + lane] = vw;
    if (lane == 0) {
      c.kp[row] = kpair;
      c.vp[row] = vpair;
    }
  }
}

// A thread has 16 bytes of output (four numbers in fp32, eight in bf16) of one token per trip, so that a warp's stores are
// whole lines: `per` threads lie along the units of a token (all of them, or 256 where there are more), 256 / per tokens side
// by side.  blockIdx.y: sequence, blockIdx.z: K or V.
template <typename T, int HD, bool VEC>
__global__ void __launch_bounds__(256) kv4_load_kernel(Kv4 c, int n, const int32_t* __restrict__ lens, T* __restrict__ k,
                                                       T* __restrict__ v, int per) {
  constexpr int E = 16 / sizeof(T), UNITS = HD / E, DEEP = 4;   // numbers per thread, units per head, tokens on their way
  using Codes = std::conditional_t<E == 8, uint32_t, uint16_t>;
  pdl_wait();
  pdl_trigger();
  const bool of_v = blockIdx.z != 0;
  T* const out = of_v ? v : k;
  const int side = 256 / per, mine = (int)threadIdx.x / per, units = c.Hkv * UNITS, blocks = (units + per - 1) / per;
  const int w = (int)(blockIdx.x % blocks) * per + (int)threadIdx.x - mine * per;
  if (!out || mine >= side || w >= units) return;
  const int b = blockIdx.y, len = lens ? lens[b] : n, j0 = (int)(blockIdx.x / blocks) * (DEEP * side) + mine;
  const size_t plane = ((size_t)b * c.Hkv + w / UNITS) * c.cap;
  const Codes* const src = reinterpret_cast<const Codes*>(of_v ? c.v : c.k) + plane * UNITS + w % UNITS;
  const uint32_t* const par = (of_v ? c.vp : c.kp) + plane;
  T* const dst = out + ((size_t)b * n * units + w) * E;
  uint32_t u[DEEP], p[DEEP];
#pragma unroll
  for (int i = 0; i < DEEP; ++i) {
    const int j = j0 + i * side;
    u[i] = p[i] = 0;     // code 0, step 0, lo 0
    if (j < n && j < len) {
      u[i] = src[(size_t)j * UNITS];
      p[i] = par[j];
    }
  }
#pragma unroll
  for (int i = 0; i < DEEP; ++i) {
    const int j = j0 + i * side;
    if (j >= n) break;
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = fmaf((float)((u[i] >> (4 * e)) & 15u), kv4_step(p[i]), kv4_lo(p[i]));
    T* const to = dst + (size_t)j * units * E;
    if constexpr (!VEC) {
#pragma unroll
      for (int e = 0; e < E; ++e) to[e] = from_f32<T>(x[e]);
    } else if constexpr (E == 4) {
      *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
      Vec8<T>::store(to, x);
    }
  }
}

// ---------------------------------------------------------------- eviction
constexpr int EV_THREADS = 512, EV_UNIT = 8, EV_BINS = 256, EV_CLUSTER = 8;   // EV_UNIT: a CTA's share of the keys is a multiple
constexpr int EV_SMEM_KEYS = 40 * 1024;   // ordered weights that one CTA keeps

// Order of the weights as unsigned numbers, and back; a NaN comes last (as 0), -0 is 0.  No weight has the largest number.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t EV_STAYS = 0xFFFFFFFFu;   // the number of a key that stays whatever its weight

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
  int t = lane < EV_THREADS / 32 ? warps[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, t, o);
    if (lane >= o) t += u;
  }
  total = __shfl_sync(0xffffffffu, t, 31);
  const int before = __shfl_sync(0xffffffffu, t, max(w - 1, 0));
  return (w == 0 ? 0 : before) + s - v;
}

// A cluster of one or eight CTAs per (sequence, KV head), each with its share of the keys, kept in shared memory as ordered
// numbers where they fit.  The smallest number that stays is found digit by digit (8 bits, a histogram of its own each, so that
// one barrier of the cluster is enough; every CTA adds up all of the cluster's: with digits of 11 bits the 64 KB that a CTA reads
// from the others took 7000 cycles a digit), until a digit's whole bin stays.  Then each warp counts what stays of a range of its
// own, and writes it behind what stays ahead of it, 32 keys at a time.  What is left is the latency of barriers and of code that
// runs once.  (8 x 4 heads of 65536 keys 37 us with 11-bit digits, 24 with keys compared to the forced ranges in every pass, 20
// so.)
__global__ void __launch_bounds__(EV_THREADS) kv4_select_kernel(const float* __restrict__ weight, int n, int cap, int Hkv,
                                                                int keep, int first, int last,
                                                                const int32_t* __restrict__ lens, int share, int kept_in_smem,
                                                                int dst_cap, float* __restrict__ dst_weight,
                                                                int32_t* __restrict__ index, int32_t* __restrict__ new_lens) {
  constexpr int WARPS = EV_THREADS / 32;
  extern __shared__ __align__(16) uint32_t keys[];
  __shared__ int hist[4][EV_BINS];
  __shared__ int counts[2], of_warp[2][WARPS];
  __shared__ int warps[32];
  __shared__ int found[3];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = (int)cluster_ctarank();
  const bool alone = share >= cap;
  const int bh = alone ? blockIdx.x : blockIdx.x / EV_CLUSTER, b = bh / Hkv;
  const float* w = weight + (size_t)bh * cap;
  int32_t* idx = index + (size_t)bh * keep;
  float* dw = dst_weight + (size_t)bh * dst_cap;
  const int len = lens ? min(max(lens[b], 0), n) : n, kept = min(len, keep);
  const int j_lo = min(rank * share, len), j_hi = min(j_lo + share, len);
  if (rank == 0) {
    for (int i = kept + tid; i < dst_cap; i += EV_THREADS) {
      if (i < keep) idx[i] = -1;
      dw[i] = 0.f;
    }
    if (tid == 0 && bh % Hkv == 0) new_lens[b] = kept;
  }
  if (len <= keep) {   // every key stays (the whole cluster)
    for (int j = j_lo + tid; j < j_hi; j += EV_THREADS) {
      idx[j] = j;
      dw[j] = w[j] + 0.f;   // -0 as 0
    }
    return;
  }
  // Keys j .. j + 3 (j a multiple of 4) as numbers; those behind the length have the lowest one and lie behind all others.
  auto read = [&](int j) {
    const float4 x = *reinterpret_cast<const float4*>(w + j);
    uint4 k = make_uint4(weight_key(x.x), weight_key(x.y), weight_key(x.z), weight_key(x.w));
    if (j < first || j + 3 >= len - last) {
      uint32_t* const e = &k.x;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (j + q < first || j + q >= len - last) e[q] = j + q < len ? EV_STAYS : 0u;
    }
    return k;
  };
  auto four = [&](int j) { return kept_in_smem ? *reinterpret_cast<const uint4*>(keys + (j - j_lo)) : read(j); };
  for (int i = tid; i < 4 * EV_BINS; i += EV_THREADS) hist[0][i] = 0;
  if (kept_in_smem) {
#pragma unroll 4
    for (int j = j_lo + tid * 4; j < j_hi; j += EV_THREADS * 4) *reinterpret_cast<uint4*>(keys + (j - j_lo)) = read(j);
  }
  __syncthreads();
  uint32_t prefix = 0;   // the threshold's digits so far
  int need = keep;       // of the keys that have them
#pragma unroll 1
  for (int d = 0; d < 4; ++d) {
    const int shift = 24 - 8 * d;
    const uint32_t mask = d == 0 ? 0u : 0xFFFFFFFFu << (shift + 8);
    int* const h = hist[d];
    for (int j = j_lo + tid * 4; j < j_hi; j += EV_THREADS * 4) {
      const uint4 x = four(j);
      const uint32_t k[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if ((k[q] & mask) == prefix) atomicAdd(&h[(k[q] >> shift) & (EV_BINS - 1)], 1);
    }
    if (alone) __syncthreads();
    else cluster_sync();
    // the bin, counted from the largest, in which the last place goes: a bin per thread
    const int at = EV_BINS - 1 - tid;
    int here = 0;
    if (tid < EV_BINS) {
      if (alone) {
        here = h[at];
      } else {
        int x[EV_CLUSTER];
#pragma unroll
        for (int r = 0; r < EV_CLUSTER; ++r) x[r] = remote(&h[at], r);
#pragma unroll
        for (int r = 0; r < EV_CLUSTER; ++r) here += x[r];
      }
    }
    int total;
    const int before = block_scan(here, warps, total);
    if (before < need && need <= before + here) {
      found[0] = at;
      found[1] = need - before;
      found[2] = need == before + here;
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    need = found[1];
    if (found[2]) {   // the whole bin (its lowest number is not 0, or every key would stay)
      prefix -= 1u;
      need = 0;
      break;
    }
  }
  // What is larger than `prefix` stays, and the first `need` of those equal to it.
  const int per = ((j_hi - j_lo + WARPS - 1) / WARPS + 127) / 128 * 128;   // keys of a warp
  const int w_lo = min(j_lo + warp * per, j_hi), w_hi = min(w_lo + per, j_hi);
  const uint32_t before_me = (1u << lane) - 1u;
  auto one = [&](int j) -> uint32_t {
    if (kept_in_smem) return keys[j - j_lo];
    return j < first || j >= len - last ? EV_STAYS : weight_key(w[j]);
  };
  int sures = 0, ties = 0;
#pragma unroll 4
  for (int j = w_lo + lane; j < w_hi; j += 32) {
    const uint32_t k = one(j);
    sures += k > prefix;
    ties += k == prefix;
  }
  sures = __reduce_add_sync(0xffffffffu, sures);
  ties = __reduce_add_sync(0xffffffffu, ties);
  if (lane == 0) {
    of_warp[0][warp] = sures;
    of_warp[1][warp] = ties;
  }
  __syncthreads();
  // what stays ahead: in earlier warps (a lane each), and in the CTAs with earlier keys
  const int of0 = lane < WARPS ? of_warp[0][lane] : 0, of1 = lane < WARPS ? of_warp[1][lane] : 0;
  int s = __reduce_add_sync(0xffffffffu, lane < warp ? of0 : 0), t = __reduce_add_sync(0xffffffffu, lane < warp ? of1 : 0);
  if (!alone) {
    const int all0 = __reduce_add_sync(0xffffffffu, of0), all1 = __reduce_add_sync(0xffffffffu, of1);
    if (tid == 0) {
      counts[0] = all0;
      counts[1] = all1;
    }
    cluster_sync();
    s += __reduce_add_sync(0xffffffffu, lane < rank ? remote(&counts[0], lane) : 0);
    t += __reduce_add_sync(0xffffffffu, lane < rank ? remote(&counts[1], lane) : 0);
  }
#pragma unroll 2
  for (int j0 = w_lo; j0 < w_hi; j0 += 32) {
    const int j = j0 + lane;
    const uint32_t k = j < w_hi ? one(j) : 0u;
    const bool sure = j < w_hi && k > prefix, tie = j < w_hi && k == prefix;
    const uint32_t sure_of = __ballot_sync(0xffffffffu, sure), tie_of = __ballot_sync(0xffffffffu, tie);
    const int at = t + __popc(tie_of & before_me);
    if (sure || (tie && at < need)) {
      const int slot = s + __popc(sure_of & before_me) + min(at, need);
      idx[slot] = j;
      dw[slot] = k == EV_STAYS ? w[j] + 0.f : __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
    }
    s += __popc(sure_of);
    t += __popc(tie_of);
  }
  if (!alone) cluster_sync();   // no CTA leaves while another one reads its numbers
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
  if ((uint32_t)j >= (uint32_t)src.cap) return;   // -1: no row
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
  // Rows a CTA: few where there are few, so that all SMs have some; with positions more, which looks through fewer of the rows behind
  // (1 / 2 / 4 / 8 / 16 / 32 rows, us: 64 scattered rows of 32 heads 3.3 / 4.5 / 6.9 / 11 / 20 / 37; 16 x 1536 in place 122 / 112 / 108 /
  // 106 / 111 / 126, scattered 166 / 138 / 124 / 120 / 128 / 155; 32768 in place of 4 heads 126 / 65 / 35 / 21 / 20 / 20, scattered 730 /
  // 416 / 280 / 267 / 355 / 600: the look through the positions grows with the square of a sequence's rows)
  const int rows = c.B * a, per = std::max(1, std::min(pos ? ST_ROWS : 4, rows / (16 * sm_count())));
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
  const int units = c.Hkv * (HD / (16 / (int)sizeof(T))), per = std::min(units, 256), side = 256 / per;
  const dim3 grid((unsigned)((n + 4 * side - 1) / (4 * side) * ((units + per - 1) / per)), c.B, 2);
  const bool vec = !(((uintptr_t)k | (uintptr_t)v) & 15);
  cudaError_t e = vec ? launch_k(L, kv4_load_kernel<T, HD, true>, grid, dim3(256), 0, c, n, lens, k, v, per)
                      : launch_k(L, kv4_load_kernel<T, HD, false>, grid, dim3(256), 0, c, n, lens, k, v, per);
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
  static DeviceOnce once;
  cudaError_t e = once.run([] {
    return cudaFuncSetAttribute(kv4_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, EV_SMEM_KEYS * 4);
  });
  if (e != cudaSuccess) return e;
  // One CTA per head or a cluster of eight (us, selection and gather of a sixteenth, one / eight):
  //   up to 8192 keys one, whatever the heads: 32 x 4128 10.0 / 12.0, 32 x 8192 12.6 / 12.4, 148 x 4128 12.1 / 30.5; of few heads with
  //   most keys eight are ahead by little (8 x 4128 9.8 / 9.7, 8 x 8192 11.4 / 9.6)
  //   beyond, eight where the heads are few: 8 x 16384 16.8 / 10.2, 32 x 16384 17.6 / 13.7, 48 x 32768 33.7 / 21.9, 64 x 16384 19.2 /
  //   20.0; one where clusters would come in several rounds: 80 x 16384 21.1 / 25.9, 148 x 16384 30 / 44, 296 x 32768 111 / 129 (between
  //   75 and 96 heads of 32768 keys eight are still ahead by a tenth)
  //   more keys than one CTA keeps in shared memory: eight (148 x 41024 95 / 84, 16 x 65536 127 / 20, 600 x 65536 551 / 419)
  const bool alone = n <= 8192 || (n <= EV_SMEM_KEYS && heads > sm_count() / 2);
  const int share = alone ? src.cap : (n + EV_CLUSTER * EV_UNIT - 1) / (EV_CLUSTER * EV_UNIT) * EV_UNIT;
  const int mine = alone ? (n + EV_UNIT - 1) / EV_UNIT * EV_UNIT : share, in_smem = mine <= EV_SMEM_KEYS;
  const size_t smem = in_smem ? (size_t)mine * 4 : 0;
  e = alone ? launch_k(L, kv4_select_kernel, dim3(heads), dim3(EV_THREADS), smem, weight, n, src.cap, src.Hkv, keep, first,
                       last, lens, share, in_smem, dst.cap, dst_weight, index, new_lens)
            : launch_k_cluster(L, kv4_select_kernel, dim3(heads * EV_CLUSTER), dim3(EV_THREADS), smem, dim3(EV_CLUSTER, 1, 1),
                               weight, n, src.cap, src.Hkv, keep, first, last, lens, share, in_smem, dst.cap, dst_weight, index,
                               new_lens);
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
