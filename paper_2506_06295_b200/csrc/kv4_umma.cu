// The 4-bit cache's attention and weights on the 5th-generation tensor cores (tcgen05), for many rows.
//
// kv4_umma_kernel: two tiles of 128 rows ((query, head of the group) pairs of one KV head) x a range of keys, thirteen warps
// with fixed roles:
//   warps 9-12       turn key tiles of 64 into operands: codes from global memory (a tile ahead in registers) to v = code - 8
//                    in shared memory, K as bf16 and V as fp16 (both hold the integers exactly), and the keys' steps and
//                    offsets to four numbers each
//   warp 8           issues the tcgen05.mma: S_i = Q_i v_K^T (bf16), O_i += P~_i v_V (fp16), row tile i = 0, 1 in turn
//   warps 0-3, 4-7   the softmax group of row tile 0 resp. 1, one row per thread: s = S * step_K + off_K * sum(q), maximum,
//                    p = 2^(s - m), l += p, z += p off_V, P~ = p step_V 2^x as fp16 over its scores in tensor memory
// x brings the largest step of the CTA's keys to [2^10, 2^11), and a row's reference follows its maximum when that has grown
// by 2^4, so P~ stays below 2^15: fp16 rounds it by 2^-11 of itself down to 2^-24 of the largest weight.  The contraction's order
// and O's columns are free, so the eight codes of a word stay in the order kv4_word gives, Q enters in it and O leaves it.
// Each tile's conversion is shared by 256 rows; what a tile takes is the exponentials and the softmax's arithmetic.
#include <algorithm>

#include "kv4.cuh"
#include "tma.cuh"
#include "umma.cuh"

namespace dllm {

namespace {

constexpr int UK_ROWS = 128, UK_STAGES = 4, UK_THREADS = 13 * 32, UK_MMA_WARP = 8, UK_CONV_WARP = 9;

// (128 + u) - 136 for the nibbles 0 and 4 of a word: bf16 pairs (128 is 0x4300, its last place is 1)
__device__ __forceinline__ uint32_t kv4_bf16_lo(uint32_t w) {
  uint32_t r;
  asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(r) : "r"(w));
  const __nv_bfloat162 h = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&r), __bfloat162bfloat162(__ushort_as_bfloat16(0x4308)));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\tmul.rn.f32x2 rd, ra, rb;\n\t"
      "mov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// 16 columns; the caller waits for the stores (tcgen05.wait::st)
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// D fp32, A and B fp16, B MN-major
__host__ __device__ constexpr uint32_t idesc_f16_mn(int m, int n) {
  return (1u << 4) | (1u << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void st_shared16(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

template <int HD>
struct UkSmem {
  static constexpr uint32_t TILE = KV4_KEYS * HD * 2, STAGE = 2 * TILE;              // K then V
  // per stage two keys per entry: (step, step, off, off) of K times the softmax's scale, (w, w, off, off) of V
  static constexpr uint32_t PAR = KV4_KEYS * 16, TOTAL = UK_STAGES * (STAGE + PAR) + 1024;
  // tensor memory: Q_i as bf16 pairs, scores S_i (P~_i over their first half), outputs O_i
  static constexpr uint32_t Q_COL = 0, S_COL = HD, O_COL = S_COL + 2 * KV4_KEYS, COLS = 512;
  static_assert(O_COL + 2 * HD <= COLS, "tensor memory holds 512 columns");
};

template <int HD>
__global__ void __launch_bounds__(UK_THREADS, 1)
    kv4_umma_kernel(const __nv_bfloat16* __restrict__ q, size_t ldq, Kv4 c, const int32_t* __restrict__ lens,
                    __nv_bfloat16* __restrict__ o, float* __restrict__ lse, float* __restrict__ o_part,
                    float2* __restrict__ ml_part, int a, int n, int H, int S, float scale_log2, int* __restrict__ status) {
  using SM = UkSmem<HD>;
  constexpr int PANELS = HD / 64;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t kv_full[UK_STAGES], kv_empty[UK_STAGES], s_full[2], p_full[2], o_full[2], q_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag, v_top;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, par_s = base + UK_STAGES * SM::STAGE;
  volatile int* abortp = &abort_flag;
  const int G = H / c.Hkv, kh = blockIdx.y, b = blockIdx.z / S, split = blockIdx.z - b * S;
  const int rows = a * G, row0 = blockIdx.x * (2 * UK_ROWS), live = row0 + UK_ROWS < rows ? 2 : 1;
  pdl_wait();
  pdl_trigger();
  const int len = lens ? min(max(lens[b], 0), n) : n;
  const int tiles_all = (len + KV4_KEYS - 1) / KV4_KEYS, per_split = (tiles_all + S - 1) / S;
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
    v_top = 0;
    for (int i = 0; i < UK_STAGES; ++i) {
      mbar_init(smem_u32(&kv_full[i]), 4);      // one arrival per converting warp
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

  if (warp >= UK_CONV_WARP) {
    // ---------------- conversion: 128 threads, per tile HD / 32 words of K and of V each, a quarter of a key's row at a time --
    constexpr int V = HD / 64;                  // 16-byte vectors of K codes per thread and tile
    constexpr int PER_ROW = HD / 32;            // such vectors per key
    const int t = tid - UK_CONV_WARP * 32;
    // the largest step of V among the CTA's keys, by its exponent
    int ex = 0;
    for (int j = tile_lo * KV4_KEYS + t; j < min(len, (tile_lo + n_tiles) * KV4_KEYS); j += 128)
      ex = max(ex, (int)(c.vp[plane + j] >> 7) & 255);
    ex = __reduce_max_sync(0xffffffffu, ex);
    if (lane == 0) atomicMax(&v_top, ex);
    asm volatile("bar.sync 3, 128;" ::: "memory");
    const float up = __uint_as_float((uint32_t)(264 - max(v_top, 20)) << 23);   // 2^(137 - field): field f means 2^(f - 127)
    uint4 kc[V], vc[V];
    uint2 pc = make_uint2(0, 0);
    auto fetch = [&](int tile) {
      const size_t key = plane + (size_t)(tile_lo + tile) * KV4_KEYS;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        kc[i] = *reinterpret_cast<const uint4*>(c.k + key * (HD / 2) + (size_t)(i * 128 + t) * 16);
        vc[i] = *reinterpret_cast<const uint4*>(c.v + key * (HD / 2) + (size_t)(i * 128 + t) * 16);
      }
      if (t < KV4_KEYS) pc = make_uint2(c.kp[key + t], c.vp[key + t]);
    };
    fetch(0);
    for (int it = 0; it < n_tiles; ++it) {
      const int st = it % UK_STAGES;
      if (it >= UK_STAGES && !mbar_wait_warp(smem_u32(&kv_empty[st]), (uint32_t)(it / UK_STAGES - 1) & 1u, abortp)) {
        ok = false;
        break;
      }
      const uint32_t ks = base + st * SM::STAGE, vs = ks + SM::TILE;
      const uint4 kn[2] = {kc[0], kc[V - 1]}, vn[2] = {vc[0], vc[V - 1]};
      const uint2 pn = pc;
      if (it + 1 < n_tiles) fetch(it + 1);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int unit = i * 128 + t, r = unit / PER_ROW, qd = unit % PER_ROW;   // key; which 32 of its elements
        // chunks of eight elements, in an order that puts the eight lanes that store together into eight banks
        const bool turn = HD == 128 && qd >= 2;
#pragma unroll
        for (int of_v = 0; of_v < 2; ++of_v) {
          const uint4 x = of_v ? vn[i] : kn[i];
          const uint32_t w[4] = {turn ? x.z : x.x, turn ? x.w : x.y, turn ? x.x : x.z, turn ? x.y : x.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int chunk = qd * 4 + (turn ? k ^ 2 : k);
            uint32_t p[4];
            if (of_v) {
              kv4_word(w[k], p);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) p[e] = kv4_bf16_lo(w[k] >> (4 * e));
            }
            st_shared16((of_v ? vs : ks) + (chunk >> 3) * (KV4_KEYS * 128) + r * 128 + (((chunk & 7) ^ (r & 7)) << 4),
                        make_uint4(p[0], p[1], p[2], p[3]));
          }
        }
      }
      if (t < KV4_KEYS) {   // keys behind the length count for nothing, whatever stands there
        const bool out = (tile_lo + it) * KV4_KEYS + t >= len;
        const float ks_ = out ? 0.f : kv4_step(pn.x), ko = out ? 0.f : fmaf(8.f, ks_, kv4_lo(pn.x));
        const float vs_ = out ? 0.f : kv4_step(pn.y), vo = out ? 0.f : fmaf(8.f, vs_, kv4_lo(pn.y));
        float* par = reinterpret_cast<float*>(smem_raw + (par_s - smem_u32(smem_raw)) + st * SM::PAR) + (t >> 1) * 8 + (t & 1);
        par[0] = ks_ * scale_log2;
        par[2] = ko * scale_log2;
        par[4] = vs_ * up;
        par[6] = vo;
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tensor cores read what these threads wrote
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&kv_full[st]));
    }
  } else if (warp == UK_MMA_WARP) {
    // ---------------- MMA issuer ----------------
    constexpr uint32_t idesc_s = make_idesc(UK_ROWS, KV4_KEYS), idesc_o = idesc_f16_mn(UK_ROWS, HD);
    auto ready = [&](int t) {
      const bool r = mbar_wait_warp(smem_u32(&kv_full[t % UK_STAGES]), (uint32_t)(t / UK_STAGES) & 1u, abortp);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      return r;
    };
    auto issue_s = [&](int i, int st) {
      if (elect_one()) {
        const uint64_t dk = make_smem_desc(base + st * SM::STAGE);
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks) {
          const uint32_t off = (ks >> 2) * (KV4_KEYS * 128) + (ks & 3) * 32;
          umma_bf16_ta(tmem + SM::S_COL + (uint32_t)(i * KV4_KEYS), tmem + SM::Q_COL + (uint32_t)(i * (HD / 2) + ks * 8),
                       dk + (uint64_t)(off >> 4), idesc_s, ks > 0 ? 1u : 0u);
        }
        umma_commit(smem_u32(&s_full[i]));
      }
      __syncwarp();
    };
    ok = mbar_wait_warp(smem_u32(&q_bar), 0u, abortp);
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
          const uint64_t dv = make_smem_desc_mn(base + st * SM::STAGE + SM::TILE, KV4_KEYS * 128, 1024);
#pragma unroll
          for (int ks = 0; ks < KV4_KEYS / 16; ++ks)
            umma_bf16_ta(tmem + SM::O_COL + (uint32_t)(i * HD), tmem + SM::S_COL + (uint32_t)(i * KV4_KEYS + ks * 8),
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
    const uint32_t s_col = tmem + row_lane + SM::S_COL + (uint32_t)(i * KV4_KEYS), o_col = tmem + row_lane + SM::O_COL + (uint32_t)(i * HD);
    const bool is_live = vr < rows;
    const int qi = is_live ? vr / G : 0, g = is_live ? vr - qi * G : 0;
    float q_sum = 0.f;
    {
      const uint4* src = reinterpret_cast<const uint4*>(q + ((size_t)b * a + qi) * ldq + (size_t)(kh * G + g) * HD);
#pragma unroll
      for (int p = 0; p < PANELS; ++p) {
        uint4 x[8];
#pragma unroll
        for (int w = 0; w < 8; ++w) x[w] = is_live ? src[p * 8 + w] : make_uint4(0, 0, 0, 0);
        uint32_t r[32];
#pragma unroll
        for (int w = 0; w < 8; ++w) {   // elements (0, 4), (1, 5), (2, 6), (3, 7), as a word's codes come out
          const uint32_t u[4] = {x[w].x, x[w].y, x[w].z, x[w].w};
          r[4 * w] = __byte_perm(u[0], u[2], 0x5410);
          r[4 * w + 1] = __byte_perm(u[0], u[2], 0x7632);
          r[4 * w + 2] = __byte_perm(u[1], u[3], 0x5410);
          r[4 * w + 3] = __byte_perm(u[1], u[3], 0x7632);
#pragma unroll
          for (int k = 0; k < 4; ++k) q_sum += __uint_as_float(u[k] << 16) + __uint_as_float(u[k] & 0xFFFF0000u);
        }
        tmem_st32(tmem + row_lane + SM::Q_COL + (uint32_t)(i * (HD / 2) + p * 32), r);
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&q_bar));
    }
    constexpr float RESCALE_STEP = 4.f;
    float m_ref = -INFINITY;
    float2 l2 = make_float2(0.f, 0.f), z2 = make_float2(0.f, 0.f);
    const float2 beta2 = make_float2(q_sum, q_sum);
    if (i < live) {
      for (int t = 0; t < n_tiles; ++t) {
        ok = mbar_wait(smem_u32(&s_full[i]), (uint32_t)t & 1u, abortp);
        // (the numbers below come from the converting warps, whose tile the scores have waited for)
        if (ok) ok = mbar_wait(smem_u32(&kv_full[t % UK_STAGES]), (uint32_t)(t / UK_STAGES) & 1u, abortp);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const float4* par = reinterpret_cast<const float4*>(smem_raw + (par_s - smem_u32(smem_raw)) + (t % UK_STAGES) * SM::PAR);
        const int valid = len - (tile_lo + t) * KV4_KEYS;
        float2 s[KV4_KEYS / 2];
        {
          uint32_t r0[32], r1[32];
          tmem_ld32(s_col, r0);
          tmem_ld32(s_col + 32u, r1);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            s[j] = make_float2(__uint_as_float(r0[2 * j]), __uint_as_float(r0[2 * j + 1]));
            s[16 + j] = make_float2(__uint_as_float(r1[2 * j]), __uint_as_float(r1[2 * j + 1]));
          }
        }
#pragma unroll
        for (int j = 0; j < KV4_KEYS / 2; ++j) {
          const float4 k = par[2 * j];
          s[j] = fma2(s[j], make_float2(k.x, k.y), mul2(make_float2(k.z, k.w), beta2));
        }
        if (valid < KV4_KEYS) {   // the last tile of the sequence
#pragma unroll
          for (int j = 0; j < KV4_KEYS / 2; ++j) {
            if (2 * j >= valid) s[j].x = -INFINITY;
            if (2 * j + 1 >= valid) s[j].y = -INFINITY;
          }
        }
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < KV4_KEYS / 2; ++j) top[j & 3] = max3(top[j & 3], s[j].x, s[j].y);
        const float mx = max3(fmaxf(top[0], top[1]), top[2], top[3]);
        const bool grow = mx > m_ref + RESCALE_STEP;
        if (__any_sync(0xffffffffu, grow)) {
          const float corr = grow ? ex2(m_ref - mx) : 1.f;
          if (grow) m_ref = mx;
          l2.x *= corr; l2.y *= corr; z2.x *= corr; z2.y *= corr;
          if (t > 0) {
#pragma unroll
            for (int cc = 0; cc < HD; cc += 32) {
              uint32_t r[32];
              tmem_ld32(o_col + (uint32_t)cc, r);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * corr);
              tmem_st32(o_col + (uint32_t)cc, r);
            }
          }
        }
        const float ref = m_ref == -INFINITY ? 0.f : m_ref;
        const float2 ref2 = make_float2(-ref, -ref);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t pk[16];
#pragma unroll
          for (int jj = 0; jj < 16; ++jj) {
            const int j = half * 16 + jj;
            const float4 v = par[2 * j + 1];
            const float2 e = add2(s[j], ref2), p = make_float2(ex2(e.x), ex2(e.y));
            l2 = add2(l2, p);
            z2 = fma2(p, make_float2(v.z, v.w), z2);
            const float2 w = mul2(p, make_float2(v.x, v.y));
            const __half2 h = __floats2half2_rn(w.x, w.y);
            pk[jj] = *reinterpret_cast<const uint32_t*>(&h);
          }
          tmem_st16(s_col + (uint32_t)(half * 16), pk);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&p_full[i]));
      }
      if (ok) ok = mbar_wait(smem_u32(&o_full[i]), 0u, abortp);
      ok = __all_sync(0xffffffffu, ok);
      if (ok) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const float l = l2.x + l2.y, z = z2.x + z2.y, down = __uint_as_float((uint32_t)(max(v_top, 20) - 10) << 23);
        const float inv = S > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
        const float f = down * inv, zf = z * inv;
        const size_t orow = ((size_t)b * a + qi) * H + kh * G + g;
#pragma unroll
        for (int cc = 0; cc < HD; cc += 32) {
          uint32_t r[32];
          tmem_ld32(o_col + (uint32_t)cc, r);
          tmem_ld_wait();
          if (!is_live) continue;
          float x[32];
#pragma unroll
          for (int k = 0; k < 32; ++k)   // column 8k + 2e + h of O is element 8k + e + 4h
            x[(k & ~7) + ((k & 7) >> 1) + 4 * (k & 1)] = fmaf(__uint_as_float(r[k]), f, zf);
          if (S > 1) {
            float* dst = o_part + ((size_t)split * total + orow) * HD + cc;
#pragma unroll
            for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(dst + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
          } else {
#pragma unroll
            for (int k = 0; k < 32; k += 8) {
              float y[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] = x[k + e];
              Vec8<__nv_bfloat16>::store(o + orow * HD + cc + k, y);
            }
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
  if (!ok && tid == 0 && status) atomicCAS(status, ST_OK, ST_TIMEOUT_ATTN_UMMA);
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

DLLM_WAIT_LIMIT_HOOK(kv4_umma)
