// Attention over the 4-bit K / V cache, and what every key gets of it.
//
// kv4_attn_kernel: 16 rows ((query, head of the group) pairs of one KV head) per CTA and split of the key range.  Its four
// warps take key tiles of 64 in turn, each with a ring of its own that cp.async fills, so no warp waits for another before
// the end; what they have is merged through shared memory there, ranges of keys inside a cluster (two, four or eight) or by
// kv4_combine_kernel.  In a tile
//     S = Q v_K^T, O += P~ v_V   mma.sync m16n8k16 on fp16, v = code - 8 made from the codes in registers
// Q enters as fp16 scaled by a power of two per row (its bf16 mantissas are exact in it; what lies 2^38 below the row's
// largest element is lost), P~ = p * step_V * 2^x with x from the largest step seen, so that it uses fp16's range: rounding
// it costs 2^-12 of each term instead of bf16's 2^-9.  Maxima, sums, steps, offsets and outputs stay in fp32.
// The order of the contraction's elements is free, which lets a thread's share of K be sixteen consecutive bytes of a key
// and lets ldmatrix.trans bring pairs of keys together for V.
#include <algorithm>
#include <atomic>

#include "kv4.cuh"
#include "tma.cuh"
#include "umma.cuh"

namespace dllm {

namespace {

constexpr int KV4_WEIGHTS_ROWS = 64;   // rows per KV head above which the weights take the tcgen05 kernel
constexpr int KA_THREADS = 128, KA_ROWS = 16, KA_STAGES = 3, KA_CLUSTER = 8;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// Power of two that brings a number with exponent field `ex` to [2^13, 2^14), and its inverse.  Fields below 20 count as 20.
__device__ __forceinline__ float kv4_up(int ex) { return __uint_as_float((uint32_t)(267 - max(ex, 20)) << 23); }
__device__ __forceinline__ float kv4_down(int ex) { return __uint_as_float((uint32_t)(max(ex, 20) - 13) << 23); }

// A lane's share of a row of Q: elements [t * HD / 4, (t + 1) * HD / 4) as fp16 pairs in the order of kv4_word, scaled by
// kv4_up of the row's largest; the four lanes of a row must call it together.  alpha: what the scaled product has to be
// multiplied by, beta: the row's sum, both times scale_log2.  live: the row may be read; counts: else it is as good as zeros,
// whatever it holds.
template <int HD>
__device__ __forceinline__ void q_share(const __nv_bfloat16* row, bool live, bool counts, int t, float scale_log2,
                                        uint32_t (&w)[HD / 8], float& alpha, float& beta) {
  uint4 raw[HD / 32];
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
    raw[i] = live ? *reinterpret_cast<const uint4*>(row + t * (HD / 4) + i * 8) : make_uint4(0, 0, 0, 0);
  if (!counts) {
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) raw[i] = make_uint4(0, 0, 0, 0);
  }
  float top = 0.f, sum = 0.f;
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) {
    const uint32_t u[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float a = __uint_as_float(u[k] << 16), b = __uint_as_float(u[k] & 0xFFFF0000u);
      top = fmaxf(top, fmaxf(fabsf(a), fabsf(b)));
      sum += a + b;
    }
  }
#pragma unroll
  for (int o = 1; o <= 2; o <<= 1) {
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
  }
  const int ex = (int)(__float_as_uint(top) >> 23);
  const float up = kv4_up(ex);
  alpha = scale_log2 * kv4_down(ex);
  beta = scale_log2 * sum;
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) {
    const uint32_t u[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    float e[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      e[2 * k] = __uint_as_float(u[k] << 16) * up;
      e[2 * k + 1] = __uint_as_float(u[k] & 0xFFFF0000u) * up;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) w[4 * i + k] = half_pair(e[k], e[k + 4]);
  }
}

template <int HD>
struct KaSmem {
  static constexpr int ROW = HD / 2;                                    // bytes of a key's codes
  static constexpr int K = 0, V = KV4_KEYS * ROW, KP = 2 * V, VP = KP + KV4_KEYS * 4, STAGE = VP + KV4_KEYS * 4;
  // a warp's ring, and what it makes of a tile's pairs: (step, step, off, off) of two keys of K, the same of V
  static constexpr int PAR = KA_STAGES * STAGE, WARP = PAR + KV4_KEYS * 16, TOTAL = 4 * WARP;
  static constexpr int XS = HD + 4;                                     // floats per exchanged row
  static_assert(KA_ROWS * XS * 4 <= WARP, "a warp's outputs replace its ring");
  // place of the 16-byte chunk c of a key's V codes: eight keys' same chunks lie in eight different banks
  static __device__ __forceinline__ int v_chunk(int key, int c) {
    return key * ROW + ((HD == 128 ? c ^ ((key >> 1) & 3) : c ^ ((key >> 2) & 1)) << 4);
  }
};

template <int HD>
__global__ void __launch_bounds__(KA_THREADS) kv4_attn_kernel(const __nv_bfloat16* __restrict__ q, size_t ldq, Kv4 c,
                                                              const int32_t* __restrict__ lens,
                                                              __nv_bfloat16* __restrict__ o, float* __restrict__ lse,
                                                              float* __restrict__ o_part, float2* __restrict__ ml_part, int a,
                                                              int n, int H, int S, int clustered, float scale_log2) {
  using SM = KaSmem<HD>;
  constexpr int KS = HD / 16, CH = HD / 32;    // k-steps of Q K^T; 16-byte chunks of a row
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float x_m[4][KA_ROWS], x_l[4][KA_ROWS];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int G = H / c.Hkv, kh = blockIdx.y, b = blockIdx.z / S, split = blockIdx.z - b * S;
  const int rows = a * G, row0 = blockIdx.x * KA_ROWS;
  pdl_wait();
  pdl_trigger();
  const int len = lens ? min(max(lens[b], 0), n) : n;
  const int tiles_all = (len + KV4_KEYS - 1) / KV4_KEYS, per_split = (tiles_all + S - 1) / S;
  const int tile_lo = min(split * per_split, tiles_all), tile_hi = min(tile_lo + per_split, tiles_all);
  const size_t plane = ((size_t)b * c.Hkv + kh) * c.cap;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * SM::WARP;
  uint8_t* const ring_g = smem + warp * SM::WARP;

  auto request = [&](int tile, int stage) {
    if (tile < tile_hi) {
      const size_t key = plane + (size_t)tile * KV4_KEYS;
      const uint32_t dst = ring + stage * SM::STAGE;
      const uint8_t* ks = c.k + key * SM::ROW;
      const uint8_t* vs = c.v + key * SM::ROW;
#pragma unroll
      for (int i = 0; i < KV4_KEYS * CH / 32; ++i) {
        const int u = i * 32 + lane, r = u / CH, ch = u % CH;
        cp_async16(dst + SM::K + u * 16, ks + u * 16);
        cp_async16(dst + SM::V + SM::v_chunk(r, ch), vs + u * 16);
      }
      const uint32_t* ps = lane < 16 ? c.kp + key + lane * 4 : c.vp + key + (lane - 16) * 4;
      cp_async16(dst + (lane < 16 ? SM::KP + lane * 16 : SM::VP + (lane - 16) * 16), ps);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < KA_STAGES - 1; ++s) request(tile_lo + warp + 4 * s, s);

  // rows g and g + 8 of the CTA's
  uint32_t aq[KS][4];
  float alpha[2], beta[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = row0 + g + 8 * h, i = r / G;
    uint32_t w[HD / 8];
    q_share<HD>(q + ((size_t)b * a + i) * ldq + (size_t)(kh * G + r - i * G) * HD, r < rows, true, t, scale_log2, w, alpha[h], beta[h]);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      aq[ks][h] = w[2 * ks];
      aq[ks][2 + h] = w[2 * ks + 1];
    }
  }

  float acc[HD / 8][4];
#pragma unroll
  for (int i = 0; i < HD / 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][e] = 0.f;
  float m[2] = {-INFINITY, -INFINITY};
  float2 l[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, z[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
  int v_ex = 20;   // exponent field of the largest step of V so far

  int stage = 0;
  for (int tile = tile_lo + warp; tile < tile_hi; tile += 4) {
    request(tile + 4 * (KA_STAGES - 1), stage == 0 ? KA_STAGES - 1 : stage - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(KA_STAGES - 1) : "memory");
    __syncwarp();
    const uint8_t* kt = ring_g + stage * SM::STAGE;
    const uint32_t vt = ring + stage * SM::STAGE + SM::V;
    const int valid = len - tile * KV4_KEYS;   // >= 1

    // the pairs of two keys per lane as the four numbers that scores and weights take; keys behind the length: no V
    const uint2 kp = *reinterpret_cast<const uint2*>(kt + SM::KP + lane * 8);
    uint2 vp = *reinterpret_cast<const uint2*>(kt + SM::VP + lane * 8);
    if (2 * lane >= valid) vp.x = 0u;
    if (2 * lane + 1 >= valid) vp.y = 0u;
    const int ex = max(v_ex, (int)__reduce_max_sync(0xffffffffu, max((vp.x >> 7) & 255u, (vp.y >> 7) & 255u)));
    const float up = kv4_up(ex);
    float4* const par = reinterpret_cast<float4*>(ring_g + SM::PAR);
    par[2 * lane] = make_float4(kv4_step(kp.x), kv4_step(kp.y), fmaf(8.f, kv4_step(kp.x), kv4_lo(kp.x)),
                                fmaf(8.f, kv4_step(kp.y), kv4_lo(kp.y)));
    par[2 * lane + 1] = make_float4(kv4_step(vp.x) * up, kv4_step(vp.y) * up, fmaf(8.f, kv4_step(vp.x), kv4_lo(vp.x)) * KV4_SUM_DOWN,
                                    fmaf(8.f, kv4_step(vp.y), kv4_lo(vp.y)) * KV4_SUM_DOWN);

    float s[8][4];
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
      uint32_t w[CH];
      const uint8_t* src = kt + SM::K + (nt * 8 + g) * SM::ROW + t * (SM::ROW / 4);
      if constexpr (HD == 128) {
        const uint4 x = *reinterpret_cast<const uint4*>(src);
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(src);
        w[0] = x.x; w[1] = x.y;
      }
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        uint32_t p[4];
        kv4_word(w[i], p);
        mma_f16_16816(s[nt], aq[2 * i], p[0], p[1]);
        mma_f16_16816(s[nt], aq[2 * i + 1], p[2], p[3]);
      }
    }
    __syncwarp();
    // scores in log2 units; their maxima (two keys of a row per instruction).  The row's scale comes
    // ahead of the step: huge steps under tiny queries then stay within fp32's range.
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
      const float4 k = par[2 * (nt * 4 + t)];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float2 x = fma2(mul2(make_float2(s[nt][2 * h], s[nt][2 * h + 1]), make_float2(alpha[h], alpha[h])), make_float2(k.x, k.y),
                              mul2(make_float2(k.z, k.w), make_float2(beta[h], beta[h])));
        s[nt][2 * h] = x.x;
        s[nt][2 * h + 1] = x.y;
      }
    }
    if (valid < KV4_KEYS) {   // the last tile of the sequence
#pragma unroll
      for (int nt = 0; nt < 8; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (nt * 8 + 2 * t + (e & 1) >= valid) s[nt][e] = -INFINITY;
    }
#pragma unroll
    for (int nt = 0; nt < 8; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) top[h] = max3(top[h], s[nt][2 * h], s[nt][2 * h + 1]);
    float corr[2];
    bool same = ex == v_ex;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
      top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2));
      const float now = fmaxf(m[h], top[h]);
      corr[h] = now == m[h] ? 1.f : exp2_approx(m[h] - now);
      same = same && now == m[h];
      m[h] = now;
    }
    if (!__all_sync(0xffffffffu, same)) {
      const float shrink = up * kv4_down(v_ex);   // 2^(v_ex - ex)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h].x *= corr[h]; l[h].y *= corr[h];
        z[h].x *= corr[h]; z[h].y *= corr[h];
        corr[h] *= shrink;
      }
#pragma unroll
      for (int i = 0; i < HD / 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] *= corr[e >> 1];
      v_ex = ex;
    }
    const float2 ref[2] = {make_float2(m[0] == -INFINITY ? 0.f : -m[0], m[0] == -INFINITY ? 0.f : -m[0]),
                           make_float2(m[1] == -INFINITY ? 0.f : -m[1], m[1] == -INFINITY ? 0.f : -m[1])};
    uint32_t pw[8][2];
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
      const float4 v = par[2 * (nt * 4 + t) + 1];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float2 e = add2(make_float2(s[nt][2 * h], s[nt][2 * h + 1]), ref[h]), p = make_float2(exp2_approx(e.x), exp2_approx(e.y));
        l[h] = add2(l[h], p);
        z[h] = fma2(p, make_float2(v.z, v.w), z[h]);
        const float2 w = mul2(p, make_float2(v.x, v.y));
        pw[nt][h] = half_pair(w.x, w.y);
      }
    }
#pragma unroll
    for (int ks = 0; ks < KV4_KEYS / 16; ++ks) {
      const uint32_t ap[4] = {pw[2 * ks][0], pw[2 * ks][1], pw[2 * ks + 1][0], pw[2 * ks + 1][1]};
#pragma unroll
      for (int cb = 0; cb < CH / 2; ++cb) {
        const int key = ks * 16 + ((lane >> 3) & 1) * 8 + (lane & 7);
        uint32_t r[4];
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(vt + SM::v_chunk(key, cb * 2 + (lane >> 4)))
                     : "memory");
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          uint32_t b0[4], b1[4];
          kv4_word(r[2 * x], b0);
          kv4_word(r[2 * x + 1], b1);
#pragma unroll
          for (int e = 0; e < 4; ++e) mma_f16_16816(acc[(cb * 2 + x) * 4 + e], ap, b0[e], b1[e]);
        }
      }
    }
    __syncwarp();   // the stage is free once every lane has read it
    stage = stage == KA_STAGES - 1 ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();

  // ---- the warps' rows, unnormalised (times KV4_SUM_DOWN), one after the other in shared memory
  float* const xo = reinterpret_cast<float*>(smem + warp * SM::WARP);
  const float down = kv4_down(v_ex) * KV4_SUM_DOWN;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float lh = l[h].x + l[h].y, zh = z[h].x + z[h].y;
#pragma unroll
    for (int x = 1; x <= 2; x <<= 1) {
      lh += __shfl_xor_sync(0xffffffffu, lh, x);
      zh += __shfl_xor_sync(0xffffffffu, zh, x);
    }
    if (t == 0) {
      x_m[warp][g + 8 * h] = m[h];
      x_l[warp][g + 8 * h] = lh;
    }
    // columns 2t and 2t + 1 of block (ch, e) are elements 32 ch + 8t + e and 32 ch + 8t + 4 + e
#pragma unroll
    for (int ch = 0; ch < CH; ++ch)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float4 v;
        float* f = &v.x;
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = fmaf(acc[ch * 4 + e][2 * h + half], down, zh);
        *reinterpret_cast<float4*>(xo + (g + 8 * h) * SM::XS + ch * 32 + t * 8 + half * 4) = v;
      }
  }
  __syncthreads();
  constexpr int PER = HD * KA_ROWS / KA_THREADS;   // consecutive elements per thread
  const int r = tid / (HD / PER), col = tid % (HD / PER) * PER, vr = row0 + r;
  float top = x_m[0][r];
#pragma unroll
  for (int w = 1; w < 4; ++w) top = fmaxf(top, x_m[w][r]);
  float sum = 0.f, out[PER];
  {
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int e = 0; e < PER; ++e) out[e] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = exp2_approx(x_m[w][r] - ref);
      const float* x = reinterpret_cast<const float*>(smem + w * SM::WARP) + r * SM::XS + col;
      sum = fmaf(f, x_l[w][r], sum);
#pragma unroll
      for (int e = 0; e < PER; ++e) out[e] = fmaf(f, x[e], out[e]);
    }
  }
  if (S > 1 && clustered) {
    // the splits are a cluster: every CTA's rows in its shared memory, each CTA finishes every S-th one
    __syncthreads();   // the warps' rows have been read
    float* const mine = reinterpret_cast<float*>(smem);
    float2* const my_ml = reinterpret_cast<float2*>(smem + KA_ROWS * SM::XS * 4);
#pragma unroll
    for (int e = 0; e < PER; e += 4)
      *reinterpret_cast<float4*>(mine + r * SM::XS + col + e) = make_float4(out[e], out[e + 1], out[e + 2], out[e + 3]);
    if (col == 0) my_ml[r] = make_float2(top, sum);
    cluster_sync();
    for (int u = tid; u < KA_ROWS * (HD / 4); u += KA_THREADS) {
      const int r2 = u / (HD / 4), c4 = u % (HD / 4) * 4, vr2 = row0 + r2;
      if (r2 % S != split || vr2 >= rows) continue;
      float2 ml[KA_CLUSTER];
      float4 x[KA_CLUSTER];
#pragma unroll
      for (int k = 0; k < KA_CLUSTER; ++k) {
        ml[k] = make_float2(-INFINITY, 0.f);
        x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k < S) {
          asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(ml[k].x), "=f"(ml[k].y) : "r"(cluster_addr(smem_u32(my_ml + r2), k)));
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(x[k].x), "=f"(x[k].y), "=f"(x[k].z), "=f"(x[k].w)
                       : "r"(cluster_addr(smem_u32(mine + r2 * SM::XS + c4), k)));
        }
      }
      float t2 = ml[0].x;
#pragma unroll
      for (int k = 1; k < KA_CLUSTER; ++k) t2 = fmaxf(t2, ml[k].x);
      const float ref = t2 == -INFINITY ? 0.f : t2;
      float l2 = 0.f;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < KA_CLUSTER; ++k) {
        const float f = exp2_approx(ml[k].x - ref);
        l2 = fmaf(f, ml[k].y, l2);
        y.x = fmaf(f, x[k].x, y.x); y.y = fmaf(f, x[k].y, y.y); y.z = fmaf(f, x[k].z, y.z); y.w = fmaf(f, x[k].w, y.w);
      }
      const float inv = l2 == 0.f ? 0.f : KV4_SUM_UP / l2;
      const int i2 = vr2 / G;
      const size_t orow = ((size_t)b * a + i2) * H + kh * G + (vr2 - i2 * G);
      const __nv_bfloat162 lo = __floats2bfloat162_rn(y.x * inv, y.y * inv), hi = __floats2bfloat162_rn(y.z * inv, y.w * inv);
      *reinterpret_cast<uint2*>(o + orow * HD + c4) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      if (lse && c4 == 0) lse[orow] = l2 == 0.f ? -INFINITY : (t2 + log2f(l2)) * 0.69314718055994531f;
    }
    cluster_sync();   // no CTA leaves while another one reads its rows
    return;
  }
  if (vr >= rows) return;
  const int i = vr / G;
  const size_t orow = ((size_t)b * a + i) * H + kh * G + (vr - i * G);
  if (S > 1) {
    const size_t at = (size_t)split * ((size_t)gridDim.z / S * a * H) + orow;
    if (col == 0) ml_part[at] = make_float2(top, sum);
#pragma unroll
    for (int e = 0; e < PER; e += 4)
      *reinterpret_cast<float4*>(o_part + at * HD + col + e) = make_float4(out[e], out[e + 1], out[e + 2], out[e + 3]);
    return;
  }
  const float inv = sum == 0.f ? 0.f : KV4_SUM_UP / sum;   // a row without keys: zeros
#pragma unroll
  for (int e = 0; e < PER; e += 8) {
    float v[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = out[e + x] * inv;
    Vec8<__nv_bfloat16>::store(o + orow * HD + col + e, v);
  }
  if (lse && col == 0) lse[orow] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
}

// A warp per (row, head): the splits' parts in their order.
template <int HD>
__global__ void __launch_bounds__(256) kv4_combine_kernel(const float* __restrict__ o_part, const float2* __restrict__ ml_part,
                                                          __nv_bfloat16* __restrict__ o, float* __restrict__ lse, size_t total,
                                                          int S) {
  constexpr int PER = HD / 32;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const size_t row = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= total) return;
  // lane s has split s (and s + 32): all of a row's numbers are on their way at once
  float2 ml[2];
#pragma unroll
  for (int k = 0; k < 2; ++k)
    ml[k] = lane + 32 * k < S ? __ldcg(&ml_part[(size_t)(lane + 32 * k) * total + row]) : make_float2(-INFINITY, 0.f);
  const float top = warp_max(fmaxf(ml[0].x, ml[1].x));
  const float ref = top == -INFINITY ? 0.f : top, f0 = exp2_approx(ml[0].x - ref), f1 = exp2_approx(ml[1].x - ref);
  const float sum = warp_sum(fmaf(f0, ml[0].y, f1 * ml[1].y));
  float out[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) out[e] = 0.f;
  for (int s0 = 0; s0 < S; s0 += 8) {
    float x[8][PER];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float* p = o_part + ((size_t)min(s0 + k, S - 1) * total + row) * HD + lane * PER;
      if constexpr (PER == 4) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(p));
        x[k][0] = v.x; x[k][1] = v.y; x[k][2] = v.z; x[k][3] = v.w;
      } else {
        const float2 v = __ldcg(reinterpret_cast<const float2*>(p));
        x[k][0] = v.x; x[k][1] = v.y;
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int s = s0 + k;
      const float f = __shfl_sync(0xffffffffu, s < 32 ? f0 : f1, s & 31);
      if (s < S)
#pragma unroll
        for (int e = 0; e < PER; ++e) out[e] = fmaf(f, x[k][e], out[e]);
    }
  }
  const float inv = sum == 0.f ? 0.f : KV4_SUM_UP / sum;
  __nv_bfloat16* dst = o + row * HD + lane * PER;
#pragma unroll
  for (int e = 0; e < PER; e += 2)
    *reinterpret_cast<__nv_bfloat162*>(dst + e) = __floats2bfloat162_rn(out[e] * inv, out[e + 1] * inv);
  if (lse && lane == 0) lse[row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------- weights
// At most KW_ROWS rows per KV head: S^T = v_K Q^T with the keys along the rows.  A CTA makes fp16 operands of the rows once, in
// shared memory; its warps hold 32 keys each in registers and go over the rows, then take the next keys, whose codes are on
// their way meanwhile.  A key's probabilities add up in its threads' registers (fp32, in the order of the rows), the four
// threads of a key at the end.  No two CTAs add to the same key.
// KW_ROWS is what the operand array holds; up to there this kernel is ahead of the tcgen05 one (us, here / there: 64 rows of 32 heads
// x 4128 keys 15.7 / 16.4, 32 rows 10.0 / 15.2, 16 sequences of 64 rows x 1536 54 / 70, 64 rows of one head x 32768 6.1 / 8.1).
constexpr int KW_KEYS = 128, KW_ROWS = KV4_WEIGHTS_ROWS;
template <int HD>
__global__ void __launch_bounds__(128) kv4_weights_kernel(const __nv_bfloat16* __restrict__ q, size_t ldq, Kv4 c,
                                                          const float* __restrict__ lse, const int32_t* __restrict__ lens,
                                                          float* __restrict__ weight, int a, int n, int H, float scale_log2) {
  constexpr int KS = HD / 16, CH = HD / 32, UNITS = HD / 32;   // units: two k-steps of a lane's share of Q, 16 bytes
  __shared__ uint4 qs[UNITS][KW_ROWS][4];
  __shared__ float4 par[KW_ROWS];    // alpha, beta, lse in log2 units
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int G = H / c.Hkv, kh = blockIdx.y, b = blockIdx.z, rows = a * G;
  pdl_wait();
  pdl_trigger();
  const int len = lens ? min(max(lens[b], 0), n) : n;
  if (blockIdx.x * KW_KEYS >= len) return;
  const size_t plane = ((size_t)b * c.Hkv + kh) * c.cap;
  uint32_t w[4][CH], pr[4];      // keys of lane group g: first + 8 i
  auto fetch = [&](int first) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const size_t key = plane + min(first + 8 * i, len - 1);
      const uint8_t* src = c.k + key * (HD / 2) + t * (HD / 8);
      if constexpr (HD == 128) {
        const uint4 x = *reinterpret_cast<const uint4*>(src);
        w[i][0] = x.x; w[i][1] = x.y; w[i][2] = x.z; w[i][3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(src);
        w[i][0] = x.x; w[i][1] = x.y;
      }
      pr[i] = c.kp[key];
    }
  };
  int key0 = blockIdx.x * KW_KEYS + warp * 32 + g;
  fetch(key0);
#pragma unroll
  for (int pass = 0; pass < KW_ROWS / 32; ++pass) {
    const int r = pass * 32 + tid / 4, i = r / G, share = tid & 3;
    if (pass * 32 >= rows) break;
    const bool live = r < rows;
    const float e = live ? lse[((size_t)b * a + i) * H + kh * G + (r - i * G)] : -INFINITY;
    uint32_t x[HD / 8];
    float alpha, beta;
    q_share<HD>(q + ((size_t)b * a + i) * ldq + (size_t)(kh * G + r - i * G) * HD, live, e != -INFINITY, share, scale_log2, x, alpha, beta);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) qs[u][r][share] = make_uint4(x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]);
    // rows past the last one and rows that saw no key give nothing
    if (share == 0) par[r] = make_float4(alpha, beta, e != -INFINITY ? e * 1.4426950408889634f : INFINITY, 0.f);
  }
  __syncthreads();
  for (; key0 - warp * 32 - g < len; key0 += gridDim.x * KW_KEYS) {
    uint32_t ak[2][KS][4];
    float step[4], off[4], got[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int k = 0; k < CH; ++k) {
        uint32_t p[4];
        kv4_word(w[i][k], p);
        ak[i >> 1][2 * k][i & 1] = p[0];
        ak[i >> 1][2 * k][2 + (i & 1)] = p[1];
        ak[i >> 1][2 * k + 1][i & 1] = p[2];
        ak[i >> 1][2 * k + 1][2 + (i & 1)] = p[3];
      }
      step[i] = kv4_step(pr[i]);
      off[i] = fmaf(8.f, step[i], kv4_lo(pr[i]));
      got[i] = 0.f;
    }
    fetch(key0 + (int)gridDim.x * KW_KEYS);
#pragma unroll 2
    for (int nt = 0; nt < KW_ROWS / 8; ++nt) {
      if (nt * 8 >= rows) break;
      float s[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = 0.f;
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        const uint4 x = qs[u][nt * 8 + g][t];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mma_f16_16816(s[i], ak[i][2 * u], x.x, x.y);
          mma_f16_16816(s[i], ak[i][2 * u + 1], x.z, x.w);
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float4 p = par[nt * 8 + 2 * t + e];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          got[i] += exp2_approx(fmaf(s[i >> 1][2 * (i & 1) + e] * p.x, step[i], fmaf(off[i], p.y, -p.z)));
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int x = 1; x <= 2; x <<= 1) got[i] += __shfl_xor_sync(0xffffffffu, got[i], x);
      if (t == 0 && key0 + 8 * i < len) weight[plane + key0 + 8 * i] += got[i];
    }
  }
}

template <int HD>
cudaError_t attention_as(const Launch& L, const Kv4Plan& plan, const __nv_bfloat16* q, size_t ldq, const Kv4& c, __nv_bfloat16* o,
                         float* lse, int a, int n, int H, const int32_t* lens, float* scratch) {
  static DeviceOnce once;
  cudaError_t e = once.run([] {
    return cudaFuncSetAttribute(kv4_attn_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, KaSmem<HD>::TOTAL);
  });
  if (e != cudaSuccess) return e;
  const size_t total = (size_t)c.B * a * H;
  const int S = plan.S;
  float* const o_part = scratch;
  float2* const ml_part = reinterpret_cast<float2*>(scratch + (S > 1 && !plan.clustered ? (size_t)S * total * HD : 0));
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)HD);
  const dim3 grid((a * (H / c.Hkv) + KA_ROWS - 1) / KA_ROWS, c.Hkv, c.B * S);
  if (plan.umma) {
    e = launch_kv4_umma(L, q, ldq, c, o, lse, a, n, H, lens, o_part, ml_part, S);
  } else {
    e = plan.clustered ? launch_k_cluster(L, kv4_attn_kernel<HD>, grid, dim3(KA_THREADS), KaSmem<HD>::TOTAL, dim3(1, 1, S), q, ldq,
                                          c, lens, o, lse, o_part, ml_part, a, n, H, S, 1, scale_log2)
                       : launch_k(L, kv4_attn_kernel<HD>, grid, dim3(KA_THREADS), KaSmem<HD>::TOTAL, q, ldq, c, lens, o, lse,
                                  o_part, ml_part, a, n, H, S, 0, scale_log2);
    L.count();
  }
  if (e != cudaSuccess || S == 1 || plan.clustered) return e != cudaSuccess ? e : cudaGetLastError();
  Launch behind = L;
  behind.pdl = true;
  e = launch_k(behind, kv4_combine_kernel<HD>, dim3((unsigned)((total + 7) / 8)), dim3(256), 0, (const float*)o_part,
               (const float2*)ml_part, o, lse, total, S);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

std::atomic<int> g_plan_hook{0};   // dllm_debug_kv4_plan: kernel + 4 * splits

}  // namespace

// Which kernel, and how many ranges the keys are cut into, by what they take (us, B200):
//   few rows   16 rows a CTA, two CTAs to an SM: 4.5 at its ends, and for a tile of 64 keys of each of its four warps 1.5, 2.1
//              beside a second CTA; 4.5 more where ranges are merged, by a cluster of up to eight as by a launch (which a call's
//              host side and scratch make the dearer one)
//   tcgen05    256 rows a CTA, one to an SM: 12 at its ends, 2.3 for a tile of 128 keys (2.8 with 256 rows and 2.2 with at most 128,
//              measured over 1 to 64 tiles), 5 for a merge and its bytes
// Over 485 shapes (1 to 16 sequences, 17 to 4096 rows per KV head, 256 to 32768 keys) the choice of kernel is 0.6 % above the better
// one's time on the geometric mean, at most 22 % (with the two measured figures per tile 0.45 %, but other ranges: 12 % and 19 % lost
// on some shapes for 17 % on others).
// Measured / by this, few rows then tcgen05, each in its best number of ranges:  64 x 768 x 32 heads 8.7 / 9, 17 / 18;
// 128 x 768 x 32 12.7 / 10.8, 17.8 / 18;  256 x 768 x 32 23 / 22, 24.7 / 26;  512 x 1024 x 32 47 / 52, 33 / 30;  128 x 512 x 28 on 4
// 10.1 / 8.7, 21 / 21;  100 x 16384 x 8 48 / 43, 32 / 36;  16 sequences of 80 x 1536 x 32 158 / 154, 131 / 158;  8 of 16 x 32768 x
// 28 on 4 270 / 273, 155 / 164.
Kv4Plan plan_kv4(int B, int a, int n, int H, int Hkv) {
  const int hook = g_plan_hook.load(std::memory_order_relaxed), kernel = hook & 3, splits = hook >> 2;
  const long rows = (long)a * (H / Hkv), heads = (long)Hkv * B, tiles = (n + KV4_KEYS - 1) / KV4_KEYS, sms = sm_count();
  Kv4Plan p;
  double best = -1.0;
  const long few = (rows + KA_ROWS - 1) / KA_ROWS * heads;
  for (int S = 1; S <= 64 && S <= tiles && (long)S * B <= 65535 && kernel != 2; ++S) {
    if (S > 1 && S < KA_CLUSTER && (S & (S - 1))) continue;   // clusters of a power of two
    const long per_warp = ((tiles + S - 1) / S + 3) / 4, waves = (few * S + 2 * sms - 1) / (2 * sms);
    const double us = (double)waves * (4.5 + (few * S > sms ? 2.1 : 1.5) * (double)per_warp) + (S > 1 ? 4.5 : 0.0);
    if (best < 0.0 || us < best) {
      best = us;
      p.S = S;
    }
  }
  const long many = (rows + 255) / 256 * heads, wide = (tiles + 1) / 2;
  for (int S = 1; (rows > KA_ROWS || kernel == 2) && kernel != 1 && S <= 64 && S <= wide && (long)S * B <= 65535; ++S) {
    const long waves = (many * S + sms - 1) / sms;
    const double us = (double)waves * (12.0 + 2.3 * (double)((wide + S - 1) / S)) + (S > 1 ? 5.0 + S * (double)B * a * H * 1040.0 / 10.0e6 : 0.0);
    if (best < 0.0 || us < best) {
      best = us;
      p.S = S;
      p.umma = true;
    }
  }
  if (splits > 0) p.S = (int)std::max(1L, std::min({(long)splits, p.umma ? wide : tiles, 65535L / B}));
  p.clustered = !p.umma && p.S > 1 && p.S <= KA_CLUSTER && !(p.S & (p.S - 1));
  return p;
}

size_t kv4_attention_scratch_bytes(const Kv4Plan& plan, int B, int a, int H, int hd) {
  return plan.S > 1 && !plan.clustered ? (size_t)plan.S * B * a * H * (hd + 2) * sizeof(float) : 0;
}

cudaError_t launch_kv4_attention(const Launch& L, const Kv4Plan& plan, const void* q, size_t ldq, const Kv4& c, void* o, float* lse,
                                 int a, int n, int H, const int32_t* lens, float* scratch) {
  auto* const qb = (const __nv_bfloat16*)q;
  auto* const ob = (__nv_bfloat16*)o;
  return c.hd == 64 ? attention_as<64>(L, plan, qb, ldq, c, ob, lse, a, n, H, lens, scratch)
                    : attention_as<128>(L, plan, qb, ldq, c, ob, lse, a, n, H, lens, scratch);
}

void set_kv4_plan(int kernel, int splits) { g_plan_hook.store(kernel + 4 * splits, std::memory_order_relaxed); }

bool plan_kv4_weights(int a, int H, int Hkv) {
  return (g_plan_hook.load(std::memory_order_relaxed) & 3) == 2 || (long)a * (H / Hkv) > KV4_WEIGHTS_ROWS;
}

size_t kv4_weights_scratch_bytes(bool umma, int B, int a, int H, int Hkv) {
  return umma ? kv4_weights_umma_scratch_bytes(B, a, H, Hkv) : 0;
}

cudaError_t launch_kv4_weights(const Launch& L, bool umma, const void* q, size_t ldq, const Kv4& c, const float* lse, float* weight,
                               int a, int n, int H, const int32_t* lens, void* scratch) {
  if (umma) return launch_kv4_weights_umma(L, q, ldq, c, lse, weight, a, n, H, lens, scratch);
  // Three CTAs to an SM, each over its share of the keys (two / three / four, us: 32 rows of 32 heads x 4128 keys 10.5 / 10.0 / 9.7, 4
  // sequences of 28 rows of 4 heads x 16384 16.8 / 15.0 / 13.2, 8 of 32 rows of 8 heads x 32768 116 / 98 / 107)
  const long blocks = (n + KW_KEYS - 1) / KW_KEYS, heads = (long)c.Hkv * c.B;
  const dim3 grid((unsigned)std::max(1L, std::min(blocks, (3L * sm_count() + heads - 1) / heads)), c.Hkv, c.B);
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)c.hd);
  cudaError_t e = c.hd == 64 ? launch_k(L, kv4_weights_kernel<64>, grid, dim3(128), 0, (const __nv_bfloat16*)q, ldq, c, lse,
                                        lens, weight, a, n, H, scale_log2)
                             : launch_k(L, kv4_weights_kernel<128>, grid, dim3(128), 0, (const __nv_bfloat16*)q, ldq, c, lse,
                                        lens, weight, a, n, H, scale_log2);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace dllm
