// Attention over the 4-bit cache on the 5th-generation tensor cores (tcgen05), for many rows.
//
// kv4_umma_kernel: two tiles of 128 rows ((query, head of the group) pairs of one KV head) x a range of keys, sixteen warps
// with fixed roles:
//   warps 9-11, 12-15  turn keys into fp16 operands in shared memory, two rounds of 64 to a tile, codes from global memory a
//                    round ahead in registers: K' = step * (code - 8), V = lo + step * code, each times a power of two
//   warp 8           issues the tcgen05.mma: S_i = Q_i K'^T + (sum of Q_i) (lo + 8 step)^T, O_i += P_i V, row tile i = 0, 1
//                    in turn
//   warps 0-3, 4-7   the softmax group of row tile 0 resp. 1, one row per thread: maximum, p = 2^(s - m + 10), l += p, P as
//                    fp16 over its scores in tensor memory
// K' is exact: a step has 8 bits and a code's distance from 8 three, fp16 holds eleven (down to 2^-21 of the largest number of
// the CTA's keys).  The offsets' share of a score is a product of its own over sixteen elements: the row's sum in three fp16
// parts (33 bits) times lo and times 8 step.  So scores are as good as fp32 sums, and the softmax needs nothing of a key but
// its score -- the steps and offsets as four numbers per key cost 2048 of a tile's 3900 cycles in shared memory reads alone (a
// uniform 16-byte read is four wavefronts).  V's offset lo + 8 step, V and P are each rounded to fp16 (2^-12 and 2^-11 of each
// term; bf16 outputs are rounded by 2^-9 and more); the powers of two keep the largest of either below 2^15.  A row's reference follows its maximum when that
// has grown by 2^4.
// The contraction's order and O's columns are free, so the eight codes of a word stay in the order kv4_word gives, Q enters in
// it and O leaves it.
#include <algorithm>
#include <type_traits>

#include "kv4.cuh"
#include "tma.cuh"
#include "umma.cuh"

namespace dllm {

namespace {

// Test hook (dllm_debug_skip_one_load): while non-zero, the issuer of CTA (0, 0, 0) waits for products that it has not issued
// instead of for Q, so that the CTA's waits run into their limit.
static __device__ int g_debug_skip = 0;

constexpr int UK_ROWS = 128, UK_KEYS = 2 * KV4_KEYS, UK_STAGES = 2, UK_THREADS = 16 * 32, UK_MMA_WARP = 8, UK_K_WARP = 9, UK_V_WARP = 12;
constexpr int UK_P_BITS = 10;   // P = p * 2^10: fp16's small numbers are further away

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
// 16 columns; the caller waits for the stores (tcgen05.wait::st)
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// D fp32, A and B fp16; mn: B MN-major
__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool mn) {
  return (1u << 4) | ((mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ __half2 as_half2(uint32_t u) { return *reinterpret_cast<const __half2*>(&u); }
__device__ __forceinline__ uint32_t as_u32(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }

template <int HD>
struct UkSmem {
  // per stage K', V, and the offsets' sixteen elements per key
  static constexpr uint32_t TILE = UK_KEYS * HD * 2, OFF = UK_KEYS * 32, STAGE = 2 * TILE + OFF;
  // per row tile Q, and the rows' sums in parts
  static constexpr uint32_t Q = UK_ROWS * HD * 2, SUM = UK_ROWS * 32;
  static constexpr uint32_t TOTAL = UK_STAGES * STAGE + 2 * (Q + SUM) + 1024;
  // tensor memory: scores S_i (P_i over their first half), outputs O_i
  static constexpr uint32_t S_COL = 0, O_COL = 2 * UK_KEYS, COLS = 512;
  static_assert(O_COL + 2 * HD <= COLS, "tensor memory holds 512 columns");
  static_assert(TOTAL <= 227 * 1024 && STAGE % 1024 == 0 && Q % 1024 == 0, "shared memory of a CTA");
};

template <int HD>
__global__ void __launch_bounds__(UK_THREADS, 1)
    kv4_umma_kernel(const __nv_bfloat16* __restrict__ q, size_t ldq, Kv4 c, const int32_t* __restrict__ lens,
                    __nv_bfloat16* __restrict__ o, float* __restrict__ lse, float* __restrict__ o_part,
                    float2* __restrict__ ml_part, int a, int n, int H, int S, float scale_log2, int* __restrict__ status) {
  using SM = UkSmem<HD>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t kv_full[UK_STAGES], kv_empty[UK_STAGES], s_full[2], p_full[2], o_full[2], q_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag, top[2];   // top: exponent fields of the largest numbers of K and V

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, q_s = base + UK_STAGES * SM::STAGE, sum_s = q_s + 2 * SM::Q;
  volatile int* abortp = &abort_flag;
  const int G = H / c.Hkv, kh = blockIdx.y, b = blockIdx.z / S, split = blockIdx.z - b * S;
  const int rows = a * G, row0 = blockIdx.x * (2 * UK_ROWS), live = row0 + UK_ROWS < rows ? 2 : 1;
  pdl_wait();
  pdl_trigger();
  const int len = lens ? min(max(lens[b], 0), n) : n;
  const int tiles_all = (len + UK_KEYS - 1) / UK_KEYS, per_split = (tiles_all + S - 1) / S;
  const int tile_lo = min(split * per_split, tiles_all), n_tiles = min(tile_lo + per_split, tiles_all) - tile_lo;
  const size_t plane = ((size_t)b * c.Hkv + kh) * c.cap, total = (size_t)gridDim.z / S * a * H;

  if (n_tiles == 0) {   // no keys: zeros and -infinity (the whole CTA)
    if (tid < 2 * UK_ROWS && row0 + tid < rows) {
      const int vr = row0 + tid, i = vr / G;
      const size_t orow = ((size_t)b * a + i) * H + kh * G + (vr - i * G);
      if (S > 1) {
        ml_part[(size_t)split * total + orow] = make_float2(-INFINITY, 0.f);
        for (int e = 0; e < HD; e += 4)
          *reinterpret_cast<float4*>(o_part + ((size_t)split * total + orow) * HD + e) = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        for (int e = 0; e < HD; e += 8) *reinterpret_cast<uint4*>(o + orow * HD + e) = make_uint4(0, 0, 0, 0);
        if (lse) lse[orow] = -INFINITY;
      }
    }
    return;
  }

  if (tid == 0) {
    abort_flag = 0;
    top[0] = top[1] = 0;
    for (int i = 0; i < UK_STAGES; ++i) {
      mbar_init(smem_u32(&kv_full[i]), UK_THREADS / 32 - UK_K_WARP);      // one arrival per converting warp
      mbar_init(smem_u32(&kv_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&s_full[i]), 1);
      mbar_init(smem_u32(&p_full[i]), 4);       // one per warp of the tile's group
      mbar_init(smem_u32(&o_full[i]), 1);
    }
    mbar_init(smem_u32(&q_bar), 8);
    mbar_fence_init();
  }
  if (warp == UK_MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(SM::COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  bool ok = true;

  const int n_keys = min(len - tile_lo * UK_KEYS, n_tiles * UK_KEYS), rounds = (n_keys + KV4_KEYS - 1) / KV4_KEYS;
  // The largest |lo| and step of the CTA's keys, by exponent field (every warp of the calling group of T threads; fields
  // outside of 30 .. 255 count as those).  A number's field f means less than 2^(f - 126).
  auto largest = [&](const uint32_t* pairs, int t, int T, int more) {
    int f = 30;
#pragma unroll 4
    for (int j = 4 * t; j < n_keys; j += 4 * T) {
      const uint4 p = *reinterpret_cast<const uint4*>(pairs + j);
      const uint32_t u[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < n_keys) f = max(f, max((int)(u[e] >> 23) & 255, ((int)(u[e] >> 7) & 255) + more));
    }
    return min((int)__reduce_max_sync(0xffffffffu, f), 255);
  };
  // ---------------- conversion of K or of V: 32 elements of a key, 16 bytes of codes, at a time ----------------
  auto convert = [&](auto of_v, auto warps) {
    constexpr bool OF_V = decltype(of_v)::value;
    constexpr int T = 32 * decltype(warps)::value, PER_ROW = HD / 32, UNITS = KV4_KEYS * PER_ROW, N = (UNITS + T - 1) / T;
    const int t = tid - (OF_V ? UK_V_WARP : UK_K_WARP) * 32;
    const uint8_t* const codes = (OF_V ? c.v : c.k) + (plane + (size_t)tile_lo * UK_KEYS) * (HD / 2);
    const uint32_t* const pairs = (OF_V ? c.vp : c.kp) + plane + (size_t)tile_lo * UK_KEYS;
    uint4 x[N];
    uint32_t pr[N];
    auto fetch = [&](int round) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[i] = make_uint4(0, 0, 0, 0);
        pr[i] = 0;
        if (i * T + t < UNITS && round < rounds) {   // (the last tile may have one round only: zeros in the other)
          x[i] = *reinterpret_cast<const uint4*>(codes + (size_t)round * (KV4_KEYS * HD / 2) + (size_t)(i * T + t) * 16);
          pr[i] = pairs[round * KV4_KEYS + (i * T + t) / PER_ROW];
        }
      }
    };
    fetch(0);   // on its way while the largest numbers are looked for
    const int f = largest(pairs, t, T, OF_V ? 4 : 3);
    if (lane == 0) atomicMax(&top[OF_V], f);
    if constexpr (OF_V) asm volatile("bar.sync 3, %0;" ::"n"(T) : "memory");
    else asm volatile("bar.sync 4, %0;" ::"n"(T) : "memory");
    // V: |lo + step * code| < 2^(f - 125), to 2^15.  K: |lo|, 8 step < 2^(f - 126), to 2^7; 2^8 times that beside the sums
    const float scale = pow2(OF_V ? 140 - top[1] : 133 - top[0]);
    for (int it = 0; it < 2 * n_tiles; ++it) {
      const int tile = it >> 1, st = tile % UK_STAGES;
      if (!(it & 1) && tile >= UK_STAGES &&
          !mbar_wait_warp(smem_u32(&kv_empty[st]), (uint32_t)(tile / UK_STAGES - 1) & 1u, abortp)) {
        ok = false;
        break;
      }
      const uint32_t stage = base + st * SM::STAGE, to = stage + (OF_V ? SM::TILE : 0u);
      uint4 now[N];
      uint32_t pair[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        now[i] = x[i];
        pair[i] = pr[i];
      }
      fetch(it + 1);   // on its way while this one is converted
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int unit = i * T + t, r = (it & 1) * KV4_KEYS + unit / PER_ROW, qd = unit % PER_ROW;   // key; which 32 elements
        if (unit >= UNITS) continue;
        const bool out = tile * UK_KEYS + r >= n_keys;   // keys behind the length count for nothing
        const float step = out ? 0.f : kv4_step(pair[i]) * scale, lo = out ? 0.f : kv4_lo(pair[i]) * scale;
        const __half2 step2 = __float2half2_rn(step), off2 = __float2half2_rn(fmaf(8.f, step, lo));
        // chunks of eight elements, in an order that puts the eight lanes that store together into eight banks
        const bool turn = HD == 128 && qd >= 2;
        const uint4 y = now[i];
        const uint32_t w[4] = {turn ? y.z : y.x, turn ? y.w : y.y, turn ? y.x : y.z, turn ? y.y : y.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int chunk = qd * 4 + (turn ? k ^ 2 : k);
          uint32_t p[4];
          kv4_word(w[k], p);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            p[e] = as_u32(OF_V ? __hfma2(as_half2(p[e]), step2, off2) : __hmul2(as_half2(p[e]), step2));
          st_shared16(to + (chunk >> 3) * (UK_KEYS * 128) + r * 128 + (((chunk & 7) ^ (r & 7)) << 4),
                      make_uint4(p[0], p[1], p[2], p[3]));
        }
        if (!OF_V && qd == 0) {   // beside the sum's parts (h, m, l, h, m, l, 0 ..): lo three times, 8 step three times
          const float lo1 = lo * 256.f, s8 = step * 2048.f;
          st_shared16(chunk_32(stage + 2 * SM::TILE, r, 0), make_uint4(half_pair(lo1, lo1), half_pair(lo1, s8), half_pair(s8, s8), 0u));
          st_shared16(chunk_32(stage + 2 * SM::TILE, r, 1), make_uint4(0u, 0u, 0u, 0u));
        }
      }
      if (it & 1) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tensor cores read what these threads wrote
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&kv_full[st]));
      }
    }
  };
  if (warp >= UK_V_WARP) {
    convert(std::true_type{}, std::integral_constant<int, UK_THREADS / 32 - UK_V_WARP>{});
  } else if (warp >= UK_K_WARP) {
    convert(std::false_type{}, std::integral_constant<int, UK_V_WARP - UK_K_WARP>{});
  } else if (warp == UK_MMA_WARP) {
    // ---------------- MMA issuer ----------------
    constexpr uint32_t idesc_s = idesc_f16(UK_ROWS, UK_KEYS, false), idesc_o = idesc_f16(UK_ROWS, HD, true);
    auto ready = [&](int t) {
      const bool r = mbar_wait_warp(smem_u32(&kv_full[t % UK_STAGES]), (uint32_t)(t / UK_STAGES) & 1u, abortp);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      return r;
    };
    auto issue_s = [&](int i, int st) {
      if (elect_one()) {
        const uint64_t dq = make_smem_desc(q_s + i * SM::Q), dk = make_smem_desc(base + st * SM::STAGE);
        const uint32_t d = tmem + SM::S_COL + (uint32_t)(i * UK_KEYS);
        // (umma_bf16 is kind::f16: the operands' type is the descriptor's)
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks)
          umma_bf16(d, dq + (uint64_t)(((ks >> 2) * (UK_ROWS * 128) + (ks & 3) * 32) >> 4),
                    dk + (uint64_t)(((ks >> 2) * (UK_KEYS * 128) + (ks & 3) * 32) >> 4), idesc_s, ks > 0 ? 1u : 0u);
        umma_bf16(d, make_smem_desc_32(sum_s + i * SM::SUM), make_smem_desc_32(base + st * SM::STAGE + 2 * SM::TILE), idesc_s, 1u);
        umma_commit(smem_u32(&s_full[i]));
      }
      __syncwarp();
    };
    const bool skip = g_debug_skip != 0 && (blockIdx.x | blockIdx.y | blockIdx.z) == 0;   // (Q takes longer than this read)
    ok = mbar_wait_warp(smem_u32(skip ? &o_full[0] : &q_bar), 0u, abortp);
    if (ok) ok = ready(0);
    for (int i = 0; i < live && ok; ++i) issue_s(i, 0);
    for (int t = 0; t < n_tiles && ok; ++t) {
      const int st = t % UK_STAGES;
      bool next = t + 1 >= n_tiles;
      for (int i = 0; i < live && ok; ++i) {
        ok = mbar_wait_warp(smem_u32(&p_full[i]), (uint32_t)t & 1u, abortp);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (elect_one()) {
          const uint64_t dv = make_smem_desc_mn(base + st * SM::STAGE + SM::TILE, UK_KEYS * 128, 1024);
#pragma unroll
          for (int ks = 0; ks < UK_KEYS / 16; ++ks)
            umma_bf16_ta(tmem + SM::O_COL + (uint32_t)(i * HD), tmem + SM::S_COL + (uint32_t)(i * UK_KEYS + ks * 8),
                         dv + (uint64_t)((ks * 16 * 128) >> 4), idesc_o, (t > 0 || ks > 0) ? 1u : 0u);
        }
        __syncwarp();
        if (t + 1 < n_tiles) {
          if (!next) {
            ok = ready(t + 1);
            if (!ok) break;
            next = true;
          }
          issue_s(i, (t + 1) % UK_STAGES);   // its commit covers O_i too: the group may then rescale O_i
        } else {
          if (elect_one()) umma_commit(smem_u32(&o_full[i]));
          __syncwarp();
        }
      }
      if (ok && elect_one()) umma_commit(smem_u32(&kv_empty[st]));
      __syncwarp();
    }
  } else {
    // ---------------- softmax groups ----------------
    const int i = warp >> 2, row = (warp & 3) * 32 + lane, vr = row0 + i * UK_ROWS + row;
    const uint32_t row_lane = ((uint32_t)((warp & 3) * 32)) << 16;
    const uint32_t s_col = tmem + row_lane + SM::S_COL + (uint32_t)(i * UK_KEYS), o_col = tmem + row_lane + SM::O_COL + (uint32_t)(i * HD);
    const bool is_live = vr < rows;
    const int qi = is_live ? vr / G : 0, g = is_live ? vr - qi * G : 0;
    float scale;    // what a score of this row has to be multiplied by
    {
      // Q times the power of two that brings the row's largest to [2^13, 2^14), as fp16 (bf16's mantissas are exact in it)
      const uint4* src = reinterpret_cast<const uint4*>(q + ((size_t)b * a + qi) * ldq + (size_t)(kh * G + g) * HD);
      uint4 x[HD / 8];
#pragma unroll
      for (int w = 0; w < HD / 8; ++w) x[w] = is_live ? src[w] : make_uint4(0, 0, 0, 0);
      float sum = 0.f, most = 0.f;
#pragma unroll
      for (int w = 0; w < HD / 8; ++w) {
        const uint32_t u[4] = {x[w].x, x[w].y, x[w].z, x[w].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float lo = __uint_as_float(u[k] << 16), hi = __uint_as_float(u[k] & 0xFFFF0000u);
          sum += lo + hi;
          most = max3(most, fabsf(lo), fabsf(hi));
        }
      }
      const int f = max((int)(__float_as_uint(most) >> 23), 20);
      const float up = pow2(140 - f);
#pragma unroll
      for (int w = 0; w < HD / 8; ++w) {   // elements (0, 4), (1, 5), (2, 6), (3, 7), as a word's codes come out
        const uint32_t u[4] = {x[w].x, x[w].y, x[w].z, x[w].w};
        uint32_t r[4];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          r[2 * k] = half_pair(__uint_as_float(u[k] << 16) * up, __uint_as_float(u[k + 2] << 16) * up);
          r[2 * k + 1] = half_pair(__uint_as_float(u[k] & 0xFFFF0000u) * up, __uint_as_float(u[k + 2] & 0xFFFF0000u) * up);
        }
        st_shared16(q_s + i * SM::Q + (w >> 3) * (UK_ROWS * 128) + row * 128 + (((w & 7) ^ (row & 7)) << 4),
                    make_uint4(r[0], r[1], r[2], r[3]));
      }
      // the sum's three parts, 2^-8 of Q's scale (the offsets beside them have 2^8 of K's)
      const float v = sum * up * 0.00390625f;
      const float h = __half2float(__float2half_rn(v)), m = __half2float(__float2half_rn(v - h)), l = v - h - m;
      st_shared16(chunk_32(sum_s + i * SM::SUM, row, 0), make_uint4(half_pair(h, m), half_pair(l, h), half_pair(m, l), 0u));
      st_shared16(chunk_32(sum_s + i * SM::SUM, row, 1), make_uint4(0u, 0u, 0u, 0u));
      scale = scale_log2 * pow2(f - 140);   // K's part follows when it is known
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&q_bar));
    }
    constexpr float RESCALE_STEP = 4.f;
    float m_ref = -INFINITY;
    float2 l2 = make_float2(0.f, 0.f);
    if (i < live) {
      // (K's scale: what a converting warp wrote ahead of its first tile)
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&kv_full[0]), 0u, abortp));
      // at least the smallest normal number: scores that small are all alike, and those behind the length stay -infinity
      scale = fmaxf(scale * pow2(top[0] - 133), 1.17549435e-38f);
      for (int t = 0; t < n_tiles && ok; ++t) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&s_full[i]), (uint32_t)t & 1u, abortp));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int valid = n_keys - t * UK_KEYS;
        // 32 scores at a time, read from tensor memory twice (the maximum, the exponentials): more at once and the compiler
        // keeps more of a thread's 128 registers in local memory (344 instead of 321 us with tiles of 64 keys, which had none there
        // then; with tiles of 128 it is 76 bytes written and 84 read for HD 128, 48 and 84 for 64)
        float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        auto scores = [&](int part, uint32_t (&r)[32]) {
          tmem_ld32(s_col + (uint32_t)(part * 32), r);
          tmem_ld32_wait(r);
          if (valid < UK_KEYS) {   // the last tile of the sequence
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (part * 32 + j >= valid) r[j] = 0xFF800000u;
          }
        };
#pragma unroll
        for (int part = 0; part < UK_KEYS / 32; ++part) {
          uint32_t r[32];
          scores(part, r);
#pragma unroll
          for (int j = 0; j < 32; j += 2)
            most[(j >> 1) & 3] = max3(most[(j >> 1) & 3], __uint_as_float(r[j]), __uint_as_float(r[j + 1]));
        }
        const float mx = max3(fmaxf(most[0], most[1]), most[2], most[3]) * scale;   // scale > 0
        const bool grow = mx > m_ref + RESCALE_STEP;
        if (__any_sync(0xffffffffu, grow)) {
          const float corr = grow ? exp2_approx(m_ref - mx) : 1.f;
          if (grow) m_ref = mx;
          l2.x *= corr;
          l2.y *= corr;
          if (t > 0) {
#pragma unroll
            for (int cc = 0; cc < HD; cc += 32) {
              uint32_t r[32];
              tmem_ld32(o_col + (uint32_t)cc, r);
              tmem_ld32_wait(r);
#pragma unroll
              for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * corr);
              tmem_st32(o_col + (uint32_t)cc, r);
            }
          }
        }
        const float ref = (m_ref == -INFINITY ? 0.f : m_ref) - (float)UK_P_BITS;
        const float2 scale2 = make_float2(scale, scale), ref2 = make_float2(-ref, -ref);
#pragma unroll
        for (int part = 0; part < UK_KEYS / 32; ++part) {
          uint32_t pk[16], r[32];
          scores(part, r);
#pragma unroll
          for (int jj = 0; jj < 16; ++jj) {
            const float2 e = fma2(make_float2(__uint_as_float(r[2 * jj]), __uint_as_float(r[2 * jj + 1])), scale2, ref2), p = make_float2(exp2_approx(e.x), exp2_approx(e.y));
            l2 = add2(l2, p);
            pk[jj] = half_pair(p.x, p.y);
          }
          tmem_st16(s_col + (uint32_t)(part * 16), pk);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&p_full[i]));
      }
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&o_full[i]), 0u, abortp));
      if (ok) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const float l = (l2.x + l2.y) * pow2(-UK_P_BITS), down = pow2(top[1] - 140 - UK_P_BITS);
        const float f = S > 1 ? down * KV4_SUM_DOWN : l == 0.f ? 0.f : down / l;
        const size_t orow = ((size_t)b * a + qi) * H + kh * G + g;
#pragma unroll
        for (int cc = 0; cc < HD; cc += 32) {
          uint32_t r[32];
          tmem_ld32(o_col + (uint32_t)cc, r);
          tmem_ld32_wait(r);
          if (!is_live) continue;
#pragma unroll
          for (int k = 0; k < 32; k += 8) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)   // column 2e + h of eight is element e + 4h
              y[(e >> 1) + 4 * (e & 1)] = __uint_as_float(r[k + e]) * f;
            if (S > 1) Vec8<float>::store(o_part + ((size_t)split * total + orow) * HD + cc + k, y);
            else Vec8<__nv_bfloat16>::store(o + orow * HD + cc + k, y);
          }
        }
        if (is_live) {
          if (S > 1) ml_part[(size_t)split * total + orow] = make_float2(m_ref, l);
          else if (lse) lse[orow] = l == 0.f ? -INFINITY : (m_ref + log2f(l)) * 0.69314718055994531f;
        }
      }
    }
  }
  ok = __syncthreads_and(ok);
  if (!ok) {   // gave up: what is on its way (products, copies) ends before memory is released
    if (tid == 0 && status) atomicCAS(status, ST_OK, ST_TIMEOUT_ATTN_UMMA);
    drain_delay();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == UK_MMA_WARP)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(SM::COLS) : "memory");
}

template <int HD>
cudaError_t umma_as(const Launch& L, const __nv_bfloat16* q, size_t ldq, const Kv4& c, __nv_bfloat16* o, float* lse, int a, int n,
                    int H, const int32_t* lens, float* o_part, float2* ml_part, int S) {
  constexpr int SMEM = (int)UkSmem<HD>::TOTAL;
  static DeviceOnce once;
  cudaError_t e = once.run([] { return cudaFuncSetAttribute(kv4_umma_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM); });
  if (e != cudaSuccess) return e;
  const dim3 grid((a * (H / c.Hkv) + 2 * UK_ROWS - 1) / (2 * UK_ROWS), c.Hkv, c.B * S);
  e = launch_k(L, kv4_umma_kernel<HD>, grid, dim3(UK_THREADS), SMEM, q, ldq, c, lens, o, lse, o_part, ml_part, a, n, H, S,
               1.4426950408889634f / sqrtf((float)HD), L.d_status);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv4_umma(const Launch& L, const void* q, size_t ldq, const Kv4& c, void* o, float* lse, int a, int n, int H,
                            const int32_t* lens, float* o_part, float2* ml_part, int S) {
  return c.hd == 64 ? umma_as<64>(L, (const __nv_bfloat16*)q, ldq, c, (__nv_bfloat16*)o, lse, a, n, H, lens, o_part, ml_part, S)
                    : umma_as<128>(L, (const __nv_bfloat16*)q, ldq, c, (__nv_bfloat16*)o, lse, a, n, H, lens, o_part, ml_part, S);
}

}  // namespace dllm

namespace dllm {
cudaError_t set_debug_skip_kv4_umma(int enable) {
  const int v = enable != 0;
  return cudaMemcpyToSymbol(g_debug_skip, &v, sizeof v);
}
}  // namespace dllm

DLLM_WAIT_LIMIT_HOOK(kv4_umma)
