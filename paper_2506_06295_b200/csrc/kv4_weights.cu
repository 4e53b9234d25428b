// What every key of the 4-bit cache gets of many rows' attention, on the 5th-generation tensor cores (tcgen05).
//
// kv4_weights_umma_kernel: two tiles of 128 keys of one KV head x all rows ((query, head of the group) pairs), or a share of
// them per CTA of a cluster; thirteen warps with fixed roles:
//   warps 0-3, 4-7  a thread per key of tile 0 resp. 1: turns its key's codes into an operand row once, then adds up
//                   2^(s - lse) over the rows, which are the columns of its lane of the accumulator
//   warp 8          issues the tcgen05.mma: S^T = K Q^T for 128 rows at a time, into one of two accumulators per key tile
//   warps 9-12      bring the rows in, as they are, and their sums and lse in parts (which kv4_row_parts_kernel has left: made
//                   here, by every CTA again, they took 4500 cycles per 128 rows instead of the exponentials' 2048)
// With the keys along the lanes a key's numbers are its thread's registers, and what remains is made part of the product.  With
// step = m 2^e (1 <= m < 2), v = code - 8, off = lo + 8 step and c = m log2(e) / sqrt(hd)
//     (s - lse) log2(e) = c * ( q . (v 2^e) + (off / m) sum(q) + (1 / c) (-lse log2(e)) )
// v 2^e is exact in bf16, so are the rows; the other two products are taken over sixteen more elements, both factors in three
// bf16 parts (24 bits), the six larger partial products of each.  The thread multiplies by c: a multiplication, an exponential
// and an addition per score, and the special-function unit's four results per scheduler and cycle are what it takes.
// Every key is added to by one thread, the rows in their order, the shares of a cluster in theirs.
#include <algorithm>

#include "kv4.cuh"
#include "tma.cuh"
#include "umma.cuh"

namespace dllm {

namespace {

constexpr int WK_TILE = 128, WK_KEYS = 2 * WK_TILE, WK_ROWS = 128, WK_STAGES = 2, WK_THREADS = 21 * 32, WK_MMA_WARP = 16,
              WK_Q_WARP = 17, WK_CLUSTER = 8, WK_LENS = 1024;

__device__ __forceinline__ float exp2_sfu(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void put16(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// x as three bf16 (their sum is x)
__device__ __forceinline__ void parts3(float x, float (&p)[3]) {
  p[0] = __bfloat162float(__float2bfloat16_rn(x));
  p[1] = __bfloat162float(__float2bfloat16_rn(x - p[0]));
  p[2] = x - p[0] - p[1];
}
// Sixteen bf16 per row: 32 bytes with the 32-byte swizzle, 8-row groups 256 bytes apart.
__device__ __forceinline__ uint64_t desc_rows32(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(256 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)6 << 61);
}
__device__ __forceinline__ void put_rows32(uint32_t base, int row, uint4 lo, uint4 hi) {
  const uint32_t turn = (uint32_t)((row >> 2) & 1) << 4;
  put16(base + row * 32 + turn, lo);
  put16(base + row * 32 + (16u ^ turn), hi);
}

// A row's sum and its lse in parts, 32 bytes per row: [B, Hkv, rows up to a multiple of 128].  Rows past the last one and rows
// that saw no key: so large an lse that nothing is left.  HD / 8 threads per row.
template <int HD>
__global__ void __launch_bounds__(256) kv4_row_parts_kernel(const __nv_bfloat16* __restrict__ q, size_t ldq,
                                                            const float* __restrict__ lse, uint4* __restrict__ parts, int B, int a,
                                                            int H, int Hkv, int padded) {
  constexpr int CHUNKS = HD / 8;
  pdl_wait();
  pdl_trigger();
  const int G = H / Hkv;
  const size_t unit = (size_t)blockIdx.x * 256 + threadIdx.x, record = unit / CHUNKS;
  const int ch = (int)(unit % CHUNKS), vr = (int)(record % padded);
  const size_t head = record / padded;
  const int kh = (int)(head % Hkv), b = (int)(head / Hkv), i = vr / G, g = vr - i * G;
  const bool live = b < B && vr < a * G;
  float sum = 0.f;
  if (live) {
    const uint4 x = *reinterpret_cast<const uint4*>(q + ((size_t)b * a + i) * ldq + (size_t)(kh * G + g) * HD + ch * 8);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) sum += __uint_as_float(w[k] << 16) + __uint_as_float(w[k] & 0xFFFF0000u);
  }
#pragma unroll
  for (int o = CHUNKS / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (ch != 0 || b >= B) return;
  float x = live ? lse[((size_t)b * a + i) * H + kh * G + g] : INFINITY;
  if (x == -INFINITY) x = INFINITY;
  x = x > 1e30f ? 1e30f : x < -1e30f ? -1e30f : x;   // (a NaN stays one)
  float s[3], l[3];
  parts3(sum, s);
  parts3(-1.4426950408889634f * x, l);
  parts[2 * record] = make_uint4(bf16_pair(s[0], s[1]), bf16_pair(s[2], s[0]), bf16_pair(s[1], s[0]), bf16_pair(l[0], l[1]));
  parts[2 * record + 1] = make_uint4(bf16_pair(l[2], l[0]), bf16_pair(l[1], l[0]), 0u, 0u);
}

// 16 bytes to shared memory; live == false: zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}

// A barrier of T threads that says whether all of them came with `x`
template <int ID, int T>
__device__ __forceinline__ bool all_of(bool x) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r)
               : "r"((uint32_t)x), "n"(ID), "n"(T)
               : "memory");
  return r != 0;
}

template <int HD>
struct WkSmem {
  static constexpr uint32_t OPERAND = WK_TILE * HD * 2, MORE = WK_TILE * 32;   // 128 rows; their sixteen more elements
  static constexpr uint32_t KEYS = 2 * (OPERAND + MORE), STAGE = OPERAND + MORE;
  static constexpr uint32_t TOTAL = 2 * KEYS + WK_STAGES * STAGE + 1024;
  static_assert(TOTAL <= 226 * 1024 && KEYS % 1024 == 0 && STAGE % 1024 == 0, "shared memory of a CTA");
};

template <int HD>
__global__ void __launch_bounds__(WK_THREADS, 1)
    kv4_weights_umma_kernel(const __nv_bfloat16* __restrict__ q, size_t ldq, Kv4 c, const uint4* __restrict__ parts,
                            const int32_t* __restrict__ lens, float* __restrict__ weight, int a, int n, int H, int shares,
                            float scale_log2, int* __restrict__ status) {
  using SM = WkSmem<HD>;
  constexpr int CHUNKS = HD / 8;                 // 16-byte chunks of a row
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t k_full[2], q_full[WK_STAGES], q_empty[WK_STAGES], d_full[2][2], d_empty[2][2];
  __shared__ __align__(16) float total[2][WK_KEYS];
  __shared__ int s_lens[WK_LENS];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = base + 2 * SM::KEYS;
  volatile int* abortp = &abort_flag;
  const int G = H / c.Hkv, rows = a * G, heads = c.B * c.Hkv;
  const int rank = shares > 1 ? (int)cluster_ctarank() : 0;
  const int tiles_all = (rows + WK_ROWS - 1) / WK_ROWS, per_share = (tiles_all + shares - 1) / shares;
  const int tile_lo = min(rank * per_share, tiles_all), n_tiles = min(tile_lo + per_share, tiles_all) - tile_lo;

  if (tid == 0) {
    abort_flag = 0;
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&k_full[i]), WK_MMA_WARP);   // one arrival per warp of the keys' threads
    for (int i = 0; i < WK_STAGES; ++i) {
      mbar_init(smem_u32(&q_full[i]), 4);
      mbar_init(smem_u32(&q_empty[i]), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&d_full[i >> 1][i & 1]), 1);
      mbar_init(smem_u32(&d_empty[i >> 1][i & 1]), WK_MMA_WARP / 2);
    }
    mbar_fence_init();
  }
  if (lens)
    for (int i = tid; i < min(c.B, WK_LENS); i += WK_THREADS) s_lens[i] = lens[i];
  if (warp == WK_MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  pdl_trigger();
  bool ok = true;

  // The CTA's units, each 256 keys of a head: the earlier keys of all heads first, so that what sequences of their own lengths
  // leave out lies together.  Every role walks through them alike.
  const int stride = (int)gridDim.x / shares;
  struct Unit {
    int block, b, kh, len;
  };
  auto unit_from = [&](int w) {   // unit w or the next one of the CTA's that has keys; len == 0: none
    for (;; w += stride) {
      Unit u;
      u.block = w / heads;
      const int head = w - u.block * heads;
      u.b = head / c.Hkv;
      u.kh = head - u.b * c.Hkv;
      u.len = 0;
      if (u.block * WK_KEYS >= n) return u;
      const int len = lens ? min(u.b < WK_LENS ? s_lens[u.b] : lens[u.b], n) : n;
      if (u.block * WK_KEYS < len) {
        u.len = len;
        return u;
      }
    }
  };
  auto after = [&](const Unit& u) { return unit_from(u.block * heads + u.b * c.Hkv + u.kh + stride); };
  const Unit first = unit_from((int)blockIdx.x / shares);

  if (warp >= WK_Q_WARP) {
    // ---------------- the rows: 16 (heads of 64: 8) threads per row ----------------
    constexpr int SIDE = 128 / CHUNKS;
    const int t = tid - WK_Q_WARP * 32, ch = t % CHUNKS, r0 = t / CHUNKS;
    const int di = SIDE / G, dg = SIDE - di * G;   // SIDE rows further on
    pdl_wait();   // for the rows' parts; what the others read was there before the launch that makes them
    auto landed = [&](int it) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&q_full[it % WK_STAGES]));
    };
    int it = 0;
    for (Unit w = first; w.len > 0 && ok; w = after(w)) {
      int qi = (tile_lo * WK_ROWS + r0) / G, g = tile_lo * WK_ROWS + r0 - qi * G;
      const __nv_bfloat16* const qb = q + (size_t)w.b * a * ldq + (size_t)w.kh * G * HD + ch * 8;
      const uint4* const pb = parts + 2 * (((size_t)w.b * c.Hkv + w.kh) * tiles_all + tile_lo) * WK_ROWS;
      for (int u = 0; u < n_tiles; ++u, ++it) {
        if (it > 0) landed(it - 1);
        const int st = it % WK_STAGES;
        if (it >= WK_STAGES && !mbar_wait_warp(smem_u32(&q_empty[st]), (uint32_t)(it / WK_STAGES - 1) & 1u, abortp)) {
          ok = false;
          break;
        }
        const uint32_t to = ring + st * SM::STAGE;
#pragma unroll
        for (int p = 0; p < WK_ROWS / SIDE; ++p) {
          const int r = p * SIDE + r0;
          copy16(to + (ch >> 3) * (WK_ROWS * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4), qi < a ? qb + (size_t)qi * ldq + g * HD : qb, qi < a);
          qi += di;
          g += dg;
          if (g >= G) {
            g -= G;
            ++qi;
          }
        }
        const uint32_t turn = (uint32_t)((t >> 2) & 1) << 4;
        copy16(to + SM::OPERAND + t * 32 + turn, pb + 2 * ((size_t)u * WK_ROWS + t), true);
        copy16(to + SM::OPERAND + t * 32 + (16u ^ turn), pb + 2 * ((size_t)u * WK_ROWS + t) + 1, true);
      }
    }
    if (it > 0 && ok) landed(it - 1);
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == WK_MMA_WARP) {
    // ---------------- MMA issuer ----------------
    constexpr uint32_t idesc = make_idesc(WK_TILE, WK_ROWS);
    int it = 0, j = 0;
    for (Unit w = first; w.len > 0 && ok; w = after(w), ++j) {
      ok = mbar_wait_warp(smem_u32(&k_full[j & 1]), (uint32_t)(j >> 1) & 1u, abortp);
      for (int u = 0; u < n_tiles && ok; ++u, ++it) {
        const int st = it % WK_STAGES, buf = it & 1;
        ok = mbar_wait_warp(smem_u32(&q_full[st]), (uint32_t)(it / WK_STAGES) & 1u, abortp);
        for (int i = 0; i < 2 && ok; ++i) {
          if (it >= 2) ok = mbar_wait_warp(smem_u32(&d_empty[i][buf]), (uint32_t)(it / 2 - 1) & 1u, abortp);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          if (elect_one()) {
            const uint32_t keys = base + (j & 1) * SM::KEYS + i * (SM::OPERAND + SM::MORE), row = ring + st * SM::STAGE;
            const uint32_t d = tmem + (uint32_t)((2 * i + buf) * WK_ROWS);
            const uint64_t dk = make_smem_desc(keys), dq = make_smem_desc(row);
#pragma unroll
            for (int ks = 0; ks < HD / 16; ++ks) {
              const uint64_t off = (uint64_t)(((ks >> 2) * (128 * 128) + (ks & 3) * 32) >> 4);
              umma_bf16(d, dk + off, dq + off, idesc, ks > 0 ? 1u : 0u);
            }
            umma_bf16(d, desc_rows32(keys + SM::OPERAND), desc_rows32(row + SM::OPERAND), idesc, 1u);
            umma_commit(smem_u32(&d_full[i][buf]));
          }
          __syncwarp();
        }
        if (ok && elect_one()) umma_commit(smem_u32(&q_empty[st]));
        __syncwarp();
      }
    }
  } else {
    // ---------------- the keys ----------------
    constexpr int MINE = HD / 64;   // 16 bytes of codes for each of a key's two threads
    const int i = warp >> 3, half = (warp >> 2) & 1, row = (warp & 3) * 32 + lane, mine = i * WK_TILE + row;
    const uint32_t d_lane = tmem + (((uint32_t)((warp & 3) * 32)) << 16) + (uint32_t)(2 * i * WK_ROWS + half * (WK_ROWS / 2));
    auto key_of = [&](const Unit& w) { return ((size_t)w.b * c.Hkv + w.kh) * c.cap + min(w.block * WK_KEYS + mine, w.len - 1); };
    uint4 x[MINE];
    uint32_t pair;
    auto fetch = [&](const Unit& w) {
      const size_t at = key_of(w);
#pragma unroll
      for (int k = 0; k < MINE; ++k) x[k] = *reinterpret_cast<const uint4*>(c.k + at * (HD / 2) + (half * MINE + k) * 16);
      pair = c.kp[at];
    };
    auto convert = [&](int j) {   // what was fetched becomes operand rows; the factor of its scores
      const uint32_t to = base + (j & 1) * SM::KEYS + i * (SM::OPERAND + SM::MORE);
      const float step = kv4_step(pair), off = fmaf(8.f, step, kv4_lo(pair));
      // step = m 2^e; a step of 0 (or too small for a normal bf16): no codes
      const bool none = fabsf(step) < 1.17549435e-38f;
      const uint32_t bits = __float_as_uint(step);
      const float m = none ? 1.f : !(fabsf(step) < INFINITY) ? step : __uint_as_float((bits & 0x807FFFFFu) | 0x3F800000u);
      const float unit = none || !(fabsf(step) < INFINITY) ? 0.f : __uint_as_float(bits & 0x7F800000u);
      const float mul = scale_log2 * m;
      const __nv_bfloat162 unit2 = __float2bfloat162_rn(unit);
#pragma unroll
      for (int k = 0; k < MINE; ++k) {
        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          uint32_t p[4];   // elements (0, 1), (2, 3), (4, 5), (6, 7)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t lo = (w[jj] >> (8 * e)) & 15u, hi = (w[jj] >> (8 * e + 4)) & 15u;
            const uint32_t v = 0x43004300u | lo | hi << 16;                      // 128 + code, twice
            const __nv_bfloat162 h = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v),
                                                     __bfloat162bfloat162(__ushort_as_bfloat16(0x4308))), unit2);
            p[e] = *reinterpret_cast<const uint32_t*>(&h);
          }
          const int chunk = (half * MINE + k) * 4 + jj;
          put16(to + (chunk >> 3) * (WK_TILE * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4), make_uint4(p[0], p[1], p[2], p[3]));
        }
      }
      if (half == 0) {
        float o[3], z[3];
        parts3(off / m, o);
        parts3(1.f / mul, z);
        // beside the row's (s0, s1, s2, s0, s1, s0, l0, l1, l2, l0, l1, l0, 0 ..)
        put_rows32(to + SM::OPERAND, row, make_uint4(bf16_pair(o[0], o[0]), bf16_pair(o[0], o[1]), bf16_pair(o[1], o[2]), bf16_pair(z[0], z[0])),
                   make_uint4(bf16_pair(z[0], z[1]), bf16_pair(z[1], z[2]), 0u, 0u));
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&k_full[j & 1]));
      return mul;
    };
    float mul = 0.f, next_mul = 0.f;
    if (first.len > 0) {
      fetch(first);
      mul = convert(0);
    }
    int it = 0, j = 0;
    for (Unit w = first, next; w.len > 0; w = next, mul = next_mul, ++j) {
      next = after(w);
      if (next.len > 0) fetch(next);   // on its way during this unit's first rows
      const bool mine_to_add = shares == 1 && half == 0 && w.block * WK_KEYS + mine < w.len;
      const float had = mine_to_add ? weight[key_of(w)] : 0.f;
      float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      for (int u = 0; u < n_tiles; ++u, ++it) {
        const int buf = it & 1;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&d_full[i][buf]), (uint32_t)(it >> 1) & 1u, abortp));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = d_lane + (uint32_t)(buf * WK_ROWS);
        const int left = rows - (tile_lo + u) * WK_ROWS - half * (WK_ROWS / 2);   // rows of this thread's columns
#pragma unroll
        for (int p = 0; p < WK_ROWS / 2; p += 32) {
          if (p >= left) break;
          uint32_t r[32];
          tmem_ld32(d + (uint32_t)p, r);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 y = mul2(make_float2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), make_float2(mul, mul));
            sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], make_float2(exp2_sfu(y.x), exp2_sfu(y.y)));
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&d_empty[i][buf]));
        // The other half of the keys' buffers is free: the products of the unit before this one are complete, since this warp
        // has had all of their results.
        if (u == 0 && next.len > 0) next_mul = convert(j + 1);
      }
      const float got = (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
      if (shares > 1) {
        total[half][mine] = got;
      } else {
        // the second half of the rows' sum to the first half's thread (read before the barrier of the unit after this one, which
        // the next but one waits for before it writes here); the tile's warps go on or give up together
        if (half == 1) total[j & 1][mine] = got;
        ok = i == 0 ? all_of<1, WK_MMA_WARP * 16>(ok) : all_of<2, WK_MMA_WARP * 16>(ok);
        if (ok && mine_to_add) weight[key_of(w)] = had + (got + total[j & 1][mine]);
      }
      if (!ok) break;
    }
  }
  ok = __syncthreads_and(ok);
  if (!ok && tid == 0 && status) atomicCAS(status, ST_OK, ST_TIMEOUT_ATTN_UMMA);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == WK_MMA_WARP)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  if (shares > 1) {   // the cluster has one unit, or none
    float got = tid < WK_KEYS ? total[0][tid] + total[1][tid] : 0.f;
    if (tid < WK_KEYS) total[0][tid] = got;
    cluster_sync();
    if (rank == 0 && tid < WK_KEYS && first.block * WK_KEYS + tid < first.len) {
      for (int s = 1; s < shares; ++s) {
        float x;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(cluster_addr(smem_u32(&total[0][tid]), s)));
        got += x;
      }
      weight[((size_t)first.b * c.Hkv + first.kh) * c.cap + first.block * WK_KEYS + tid] += got;
    }
    cluster_sync();   // no CTA leaves while another one reads its sums
  }
}

template <int HD>
cudaError_t weights_as(const Launch& L, const __nv_bfloat16* q, size_t ldq, const Kv4& c, const float* lse, float* weight, int a,
                       int n, int H, const int32_t* lens, uint4* parts) {
  constexpr int SMEM = (int)WkSmem<HD>::TOTAL;
  static DeviceOnce once;
  cudaError_t e = once.run(
      [] { return cudaFuncSetAttribute(kv4_weights_umma_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM); });
  if (e != cudaSuccess) return e;
  // fewer CTAs than multiprocessors: the rows in shares, a power of two of them
  const long blocks = (n + WK_KEYS - 1) / WK_KEYS, ctas = blocks * c.Hkv * c.B;
  const int tiles = (int)(((long)a * (H / c.Hkv) + WK_ROWS - 1) / WK_ROWS);
  int shares = 1;
  while (2 * shares <= WK_CLUSTER && 2 * shares <= tiles && ctas * 2 * shares <= sm_count()) shares *= 2;
  const dim3 grid((unsigned)(shares > 1 ? ctas * shares : std::min<long>(ctas, sm_count())));
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)HD);
  const size_t threads = (size_t)c.B * c.Hkv * tiles * WK_ROWS * (HD / 8);
  e = launch_k(L, kv4_row_parts_kernel<HD>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, q, ldq, lse, parts, c.B, a, H,
               c.Hkv, tiles * WK_ROWS);
  L.count();
  if (e != cudaSuccess) return e;
  Launch behind = L;
  behind.pdl = true;
  e = shares == 1 ? launch_k(behind, kv4_weights_umma_kernel<HD>, grid, dim3(WK_THREADS), SMEM, q, ldq, c,
                             (const uint4*)parts, lens, weight, a, n, H, shares, scale_log2, L.d_status)
                  : launch_k_cluster(behind, kv4_weights_umma_kernel<HD>, grid, dim3(WK_THREADS), SMEM, dim3(shares, 1, 1), q, ldq, c,
                                     (const uint4*)parts, lens, weight, a, n, H, shares, scale_log2, L.d_status);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

size_t kv4_weights_umma_scratch_bytes(int B, int a, int H, int Hkv) {
  return (size_t)B * Hkv * (((size_t)a * (H / Hkv) + WK_ROWS - 1) / WK_ROWS) * WK_ROWS * 32;
}

cudaError_t launch_kv4_weights_umma(const Launch& L, const void* q, size_t ldq, const Kv4& c, const float* lse, float* weight,
                                    int a, int n, int H, const int32_t* lens, void* scratch) {
  return c.hd == 64 ? weights_as<64>(L, (const __nv_bfloat16*)q, ldq, c, lse, weight, a, n, H, lens, (uint4*)scratch)
                    : weights_as<128>(L, (const __nv_bfloat16*)q, ldq, c, lse, weight, a, n, H, lens, (uint4*)scratch);
}

}  // namespace dllm

DLLM_WAIT_LIMIT_HOOK(kv4_weights)
