// What every key of the 4-bit cache gets of many rows' attention, on the 5th-generation tensor cores (tcgen05).
//
// kv4_weights_umma_kernel: one CTA per multiprocessor that walks through units, two tiles of 128 keys of one KV head x all of its
// rows ((query, head of the group) pairs); where the units are few, the CTAs of a cluster share a unit's rows.  Eighteen warps
// with fixed roles:
//   warps 0-7, 8-15  two threads per key of tile 0 resp. 1: turn the codes of the unit's keys into operand rows (while the rows
//                    of the unit before are on), then each adds up 2^(s - lse) over its half of the rows, which are the columns
//                    of its lane of the accumulator
//   warp 16          issues the tcgen05.mma: S^T = K Q^T for 128 rows at a time, into one of two accumulators per key tile
//   warp 17          requests the rows, as they are, by TMA (a tile is a box of the queries' tensor, see WkTiling), and their
//                    sums and lse in parts (which kv4_row_parts_kernel has left: made here, by every CTA again, they took 4500
//                    cycles per 128 rows instead of the exponentials' 2048)
// With the keys along the lanes a key's numbers are its thread's registers, and what remains is made part of the product.  With
// step = m 2^e (1 <= m < 2), v = code - 8, off = lo + 8 step and c = m log2(e) / sqrt(hd)
//     (s - lse) log2(e) = c * ( q . (v 2^e) + (off / m) sum(q) + (1 / c) (-lse log2(e)) )
// v 2^e is exact in bf16, so are the rows; the other two products are taken over sixteen more elements, both factors in three
// bf16 parts (24 bits), the six larger partial products of each.  The thread multiplies by c: a multiplication, an exponential
// and an addition per score.  The special-function unit's four results per scheduler and cycle would bound that, so a quarter of
// the exponentials are polynomials on the FMA pipe (a fifth to a third take the same time, half 12 % more).
// Every key's sum is taken by its two threads, the rows in their order, the shares of a cluster in theirs, and added once.
// Rows that saw no key are zeros by then: the issuer puts them there (by the keys' threads, a mask per tile: 112 instead of 104 us).
// 4 sequences of 192 rows, 28 heads on 4, up to 16384 keys: 104 us, with 52 bytes of a thread's registers in local memory where HD is
// 128 (112 with all exponentials on the special-function units, which is 78 at their rate; 124 with a CTA per 256 keys, whose start and end took 7 us of each; 130 with rows brought in by cp.async,
// one tile on its way at a time).  16 sequences of 512 rows x 1536 keys, 32 heads: 256 -> 183, of which 15 are the rows' parts.
#include <algorithm>

#include "kv4.cuh"
#include "tma.cuh"
#include "umma.cuh"

namespace dllm {

namespace {

// Test hook (dllm_debug_skip_one_load): while non-zero, the last CTA that shares the first unit (the first one where none is
// shared) leaves out a box of its first rows, so that its waits run into their limit.
static __device__ int g_debug_skip = 0;

constexpr int WK_TILE = 128, WK_KEYS = 2 * WK_TILE, WK_ROWS = 128, WK_STAGES = 2, WK_THREADS = 18 * 32, WK_MMA_WARP = 16,
              WK_Q_WARP = 17, WK_CLUSTER = 8;

// 2^x of two numbers on the FMA pipe: x split into an integer and the rest f of -1/2 .. 1/2, on which 1 + f P(f), P of degree 4,
// stands for 2^f.  P: least largest relative error with the constant held at 1 (Remez exchange, then the coefficients rounded to
// fp32 from the lowest on, the others fitted again each time): 2^-23.3 off, -1.7e-8 on average, 2^-22.6 with fp32's roundings.  (The
// coefficients of a fit whose constant is free are 2^-22.6 off beside a 1, and -6.9e-8 on average, which adds up in the weights.)
// Below 2^-126 zero, above 2^128 infinity, a NaN stays one.
__device__ __forceinline__ float2 exp2_fma(float2 x) {
  auto clamp = [](float v) {
    float r;
    asm("{\n\t.reg .f32 t;\n\tmax.NaN.f32 t, %1, 0fC2FE0000;\n\tmin.NaN.f32 %0, t, 0f43000000;\n\t}" : "=f"(r) : "f"(v));   // -127, 128
    return r;
  };
  auto both = [](float v) { return make_float2(v, v); };
  const float2 y = make_float2(clamp(x.x), clamp(x.y)), r = add2(y, both(12582912.f)), f = add2(y, fma2(r, both(-1.f), both(12582912.f)));
  float2 p = fma2(f, both(1.32695213e-3f), both(9.67129134e-3f));
  p = fma2(p, f, both(5.55071086e-2f));
  p = fma2(p, f, both(2.40222469e-1f));
  p = fma2(p, f, both(6.93147004e-1f));
  p = fma2(p, f, both(1.f));
  return mul2(p, make_float2(__uint_as_float((__float_as_uint(r.x) << 23) + 0x3F800000u),
                             __uint_as_float((__float_as_uint(r.y) << 23) + 0x3F800000u)));
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
__device__ __forceinline__ void put_rows32(uint32_t base, int row, uint4 lo, uint4 hi) {
  st_shared16(chunk_32(base, row, 0), lo);
  st_shared16(chunk_32(base, row, 1), hi);
}

// The rows of a KV head in tiles of 128: heads of `queries` queries, gbox of the G heads each, so that a tile is a box of the
// queries' tensor; what is left of the 128 holds nothing.  tiles: those of one KV head, `pieces` for the same queries.
struct WkTiling {
  int pieces, gbox, queries, tiles;
};
WkTiling wk_tiling(int a, int G) {
  WkTiling best{0, 0, 0, 0};
  const int least = (G + WK_ROWS - 1) / WK_ROWS;
  for (int k = least; k < least + 8 && k <= G; ++k) {
    WkTiling t;
    t.gbox = (G + k - 1) / k;
    t.pieces = (G + t.gbox - 1) / t.gbox;
    t.queries = WK_ROWS / t.gbox;
    t.tiles = (a + t.queries - 1) / t.queries * t.pieces;
    if (best.tiles == 0 || t.tiles < best.tiles) best = t;
  }
  return best;
}

// A row's sum and its lse in parts, 32 bytes per row as they lie in shared memory: [B, Hkv, tiles, 128].  Rows that are none and
// rows that saw no key: a sum of zero and so large an lse that nothing is left; the latter have a 1 in the last place, which meets a
// zero in the product, and tells the issuer to put zeros in the row's place (it may hold anything).  HD / 8 threads per row.
template <int HD>
__global__ void __launch_bounds__(256) kv4_row_parts_kernel(const __nv_bfloat16* __restrict__ q, size_t ldq,
                                                            const float* __restrict__ lse, uint4* __restrict__ parts, int B, int a,
                                                            int H, int Hkv, WkTiling til) {
  constexpr int CHUNKS = HD / 8;
  pdl_wait();
  pdl_trigger();
  const int G = H / Hkv;
  const size_t unit = (size_t)blockIdx.x * 256 + threadIdx.x, record = unit / CHUNKS;
  const int ch = (int)(unit % CHUNKS), r = (int)(record % WK_ROWS);
  const size_t tile = record / WK_ROWS, head = tile / til.tiles;
  const int t = (int)(tile % til.tiles), kh = (int)(head % Hkv), b = (int)(head / Hkv);
  const int i = t / til.pieces * til.queries + r / til.gbox, g = t % til.pieces * til.gbox + r % til.gbox;
  const bool live = b < B && r < til.queries * til.gbox && i < a && g < G;
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
  const bool saw_none = x == -INFINITY;
  if (saw_none) {
    x = INFINITY;
    sum = 0.f;
  }
  x = x > 1e30f ? 1e30f : x < -1e30f ? -1e30f : x;   // (a NaN stays one)
  float s[3], l[3];
  parts3(sum, s);
  parts3(-1.4426950408889634f * x, l);
  const size_t turn = (r >> 2) & 1;   // the 32-byte swizzle
  parts[2 * record + turn] = make_uint4(bf16_pair(s[0], s[1]), bf16_pair(s[2], s[0]), bf16_pair(s[1], s[0]), bf16_pair(l[0], l[1]));
  parts[2 * record + (turn ^ 1)] = make_uint4(bf16_pair(l[2], l[0]), bf16_pair(l[1], l[0]), 0u, saw_none ? 0x3F800000u : 0u);
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
    kv4_weights_umma_kernel(const __grid_constant__ CUtensorMap tmQ, Kv4 c, const uint4* __restrict__ parts,
                            const int32_t* __restrict__ lens, float* __restrict__ weight, int a, int n, WkTiling til, int shares,
                            float scale_log2, int* __restrict__ status) {
  using SM = WkSmem<HD>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t k_full[2], q_full[WK_STAGES], q_empty[WK_STAGES], d_full[2][2], d_empty[2][2];
  __shared__ __align__(16) float total[2][WK_KEYS];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag, complete;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, ring = base + 2 * SM::KEYS;
  volatile int* abortp = &abort_flag;
  const int rank = shares > 1 ? (int)cluster_ctarank() : 0, per_share = (til.tiles + shares - 1) / shares;
  const int tile_lo = min(rank * per_share, til.tiles), n_tiles = min(tile_lo + per_share, til.tiles) - tile_lo;

  if (tid == 0) {
    abort_flag = 0;
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&k_full[i]), WK_MMA_WARP);   // one arrival per warp of the keys' threads
    for (int i = 0; i < WK_STAGES; ++i) {
      mbar_init(smem_u32(&q_full[i]), 1);
      mbar_init(smem_u32(&q_empty[i]), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&d_full[i >> 1][i & 1]), 1);
      mbar_init(smem_u32(&d_empty[i >> 1][i & 1]), WK_MMA_WARP / 2);
    }
    mbar_fence_init();
  }
  // the rows of a stage that no box reaches: zeros
  const int used = til.queries * til.gbox;
  for (int i = tid; i < WK_STAGES * (HD / 64) * (WK_ROWS - used) * 8; i += WK_THREADS) {
    const int ch = i & 7, r = (i >> 3) % (WK_ROWS - used), part = (i >> 3) / (WK_ROWS - used);
    st_shared16(ring + (part / (HD / 64)) * SM::STAGE + (part % (HD / 64)) * (WK_ROWS * 128) + (used + r) * 128 + ch * 16, make_uint4(0, 0, 0, 0));
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  if (warp == WK_MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  bool ok = true;

  // The CTA's units, each 256 keys of a head, those of a sequence block by block; every role walks through them alike (a warp
  // together).  len == 0: none is left.
  struct Unit {
    int block, b, kh, len;
  };
  int walk = (int)blockIdx.x / shares, before = 0, group = 0;   // unit; those of the sequences ahead of this group of 32
  auto next_unit = [&]() {
    Unit u{0, 0, 0, 0};
    for (; group < c.B; group += 32) {
      const int b = group + lane, len = b >= c.B ? 0 : lens ? min(max(lens[b], 0), n) : n;
      const int units = (len + WK_KEYS - 1) / WK_KEYS * c.Hkv;
      int upto = units;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += t;
      }
      const uint32_t hit = __ballot_sync(0xffffffffu, walk < before + upto);
      if (hit) {
        const int l = __ffs(hit) - 1, into = walk - before - __shfl_sync(0xffffffffu, upto - units, l);
        u.b = group + l;
        u.len = __shfl_sync(0xffffffffu, len, l);
        u.block = into / c.Hkv;
        u.kh = into - u.block * c.Hkv;
        break;
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    walk += (int)gridDim.x / shares;
    return u;
  };
  const Unit first = next_unit();

  if (warp >= WK_Q_WARP) {
    // ---------------- the rows ----------------
    const bool skip = g_debug_skip != 0 && (int)blockIdx.x == shares - 1;
    // for the rows' parts; what the others read was there before the launch that makes them
    pdl_wait();
    pdl_trigger();
    int it = 0;
    for (Unit w = first; w.len > 0 && ok; w = next_unit()) {
      const uint4* const pb = parts + 2 * (((size_t)w.b * c.Hkv + w.kh) * til.tiles + tile_lo) * WK_ROWS;
      for (int u = 0; u < n_tiles; ++u, ++it) {
        const int st = it % WK_STAGES, t = tile_lo + u;
        if (it >= WK_STAGES && !mbar_wait_warp(smem_u32(&q_empty[st]), (uint32_t)(it / WK_STAGES - 1) & 1u, abortp)) {
          ok = false;
          break;
        }
        if (elect_one()) {
          const uint32_t to = ring + st * SM::STAGE, bar = smem_u32(&q_full[st]);
          mbar_expect_tx(bar, (uint32_t)used * HD * 2 + SM::MORE);
#pragma unroll
          for (int h = skip && it == 0 ? 1 : 0; h < HD / 64; ++h)
            tma_load_5d(to + h * (WK_ROWS * 128), &tmQ, bar, h * 64, t % til.pieces * til.gbox, w.kh, t / til.pieces * til.queries, w.b);
          bulk_load_1d(to + SM::OPERAND, pb + 2 * (size_t)u * WK_ROWS, SM::MORE, bar);
        }
        __syncwarp();
      }
    }
  } else if (warp == WK_MMA_WARP) {
    // ---------------- MMA issuer ----------------
    constexpr uint32_t idesc = make_idesc(WK_TILE, WK_ROWS);
    // Zeros in the place of rows that saw no key
    auto rows_that_count = [&](uint32_t stage) {
      uint32_t none[WK_ROWS / 32], any = 0;
#pragma unroll
      for (int k = 0; k < WK_ROWS / 32; ++k) {
        const int r = k * 32 + lane;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(none[k]) : "r"(stage + SM::OPERAND + r * 32 + (16u ^ ((uint32_t)((r >> 2) & 1) << 4)) + 12u) : "memory");
        any |= none[k];
      }
      if (!__any_sync(0xffffffffu, any != 0u)) return;
#pragma unroll
      for (int k = 0; k < WK_ROWS / 32; ++k)
        if (none[k])
#pragma unroll 1
          for (int ch = 0; ch < HD / 8; ++ch)
            st_shared16(stage + (ch >> 3) * (WK_ROWS * 128) + (k * 32 + lane) * 128 + (ch & 7) * 16, make_uint4(0, 0, 0, 0));
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tensor cores read them
      __syncwarp();
    };
    int it = 0, j = 0;
    for (Unit w = first; w.len > 0 && ok; w = next_unit(), ++j) {
      ok = mbar_wait_warp(smem_u32(&k_full[j & 1]), (uint32_t)(j >> 1) & 1u, abortp);
      for (int u = 0; u < n_tiles && ok; ++u, ++it) {
        const int st = it % WK_STAGES, buf = it & 1;
        ok = mbar_wait_warp(smem_u32(&q_full[st]), (uint32_t)(it / WK_STAGES) & 1u, abortp);
        if (ok) rows_that_count(ring + st * SM::STAGE);
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
            umma_bf16(d, make_smem_desc_32(keys + SM::OPERAND), make_smem_desc_32(row + SM::OPERAND), idesc, 1u);
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
          st_shared16(to + (chunk >> 3) * (WK_TILE * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4), make_uint4(p[0], p[1], p[2], p[3]));
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
    Unit next{0, 0, 0, 0}, third{0, 0, 0, 0};   // the unit whose codes are in registers or on their way, and the one behind it
    if (first.len > 0) {
      fetch(first);
      mul = convert(0);
      next = next_unit();
      if (next.len > 0) fetch(next);
    }
    int it = 0, j = 0;
    for (Unit w = first; w.len > 0; w = next, next = third, mul = next_mul, ++j) {
      const bool mine_to_add = shares == 1 && half == 0 && w.block * WK_KEYS + mine < w.len;
      const float had = mine_to_add ? weight[key_of(w)] : 0.f;
      float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      for (int u = 0; u < n_tiles; ++u, ++it) {
        const int buf = it & 1;
        // The next unit's keys, whose half of the buffers is free: the products of the unit before this one are complete, since
        // this warp has had all of their results.  (The four groups of warps in turn, so that the exponentials of the others go
        // on; ahead of the wait, so that the products of a unit of one tile run meanwhile.)
        if (u == min(2 * i + half, n_tiles - 1) && next.len > 0) {
          next_mul = convert(j + 1);
          third = next_unit();
          if (third.len > 0) fetch(third);
        }
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&d_full[i][buf]), (uint32_t)(it >> 1) & 1u, abortp));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = d_lane + (uint32_t)(buf * WK_ROWS);
        const int t = tile_lo + u, left = min(til.queries, a - t / til.pieces * til.queries) * til.gbox - half * (WK_ROWS / 2);   // rows
#pragma unroll
        for (int p = 0; p < WK_ROWS / 2; p += 32) {
          if (p >= left) break;
          uint32_t r[32];
          tmem_ld32(d + (uint32_t)p, r);
          tmem_ld32_wait(r);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 y = mul2(make_float2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), make_float2(mul, mul));
            sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], (e >> 1) % 4 == 3 ? exp2_fma(y) : make_float2(exp2_approx(y.x), exp2_approx(y.y)));
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&d_empty[i][buf]));
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
  if (!ok) {   // gave up: what is on its way (products, copies) ends before memory is released
    if (tid == 0 && status) atomicCAS(status, ST_OK, ST_TIMEOUT_ATTN_UMMA);
    drain_delay();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == WK_MMA_WARP)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  if (shares > 1) {   // the cluster has one unit, or none
    float got = tid < WK_KEYS ? total[0][tid] + total[1][tid] : 0.f;
    if (tid < WK_KEYS) total[0][tid] = got;
    if (tid == 0) complete = ok;
    cluster_sync();
    if (rank == 0 && tid < WK_KEYS) {
      // all shares or nothing: where one of them gave up, the weights stay as they were
      const int of = lane < shares ? remote(&complete, lane) : 1;
      const bool mine = first.block * WK_KEYS + tid < first.len;
      float* const to = weight + ((size_t)first.b * c.Hkv + first.kh) * c.cap + first.block * WK_KEYS + tid;
      const float had = mine ? *to : 0.f;
      for (int s = 1; s < shares; ++s) {
        float x;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(cluster_addr(smem_u32(&total[0][tid]), s)));
        got += x;
      }
      if (__all_sync(0xffffffffu, of != 0) && mine) *to = had + got;
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
  const int G = H / c.Hkv;
  const WkTiling til = wk_tiling(a, G);
  CUtensorMap tmQ;
  if (!make_tensor_map_heads(q, c.B, a, c.Hkv, G, HD, ldq, til.gbox, til.queries, &tmQ)) return cudaErrorInvalidValue;
  // Fewer units than multiprocessors: a unit's rows in shares, a power of two of them; otherwise each CTA walks through several.
  // (At most one / two / four / eight shares, us: 512 rows of 2 heads x 512 keys 17.0 / 13.3 / 11.0 / 10.4, 8192 rows of one head x
  // 4096 89 / 51 / 31 / 37, 2100 rows of 4 heads x 1300 30 / 21 / 16 / 16)
  const long units = (long)((n + WK_KEYS - 1) / WK_KEYS) * c.Hkv * c.B;
  int shares = 1;
  while (2 * shares <= WK_CLUSTER && 2 * shares <= til.tiles && units * 2 * shares <= sm_count()) shares *= 2;
  const dim3 grid((unsigned)(shares > 1 ? units * shares : std::min<long>(units, sm_count())));
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)HD);
  const size_t threads = (size_t)c.B * c.Hkv * til.tiles * WK_ROWS * (HD / 8);
  e = launch_k(L, kv4_row_parts_kernel<HD>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, q, ldq, lse, parts, c.B, a, H,
               c.Hkv, til);
  L.count();
  if (e != cudaSuccess) return e;
  Launch behind = L;
  behind.pdl = true;
  e = shares == 1 ? launch_k(behind, kv4_weights_umma_kernel<HD>, grid, dim3(WK_THREADS), SMEM, tmQ, c, (const uint4*)parts, lens,
                             weight, a, n, til, shares, scale_log2, L.d_status)
                  : launch_k_cluster(behind, kv4_weights_umma_kernel<HD>, grid, dim3(WK_THREADS), SMEM, dim3(shares, 1, 1), tmQ, c,
                                     (const uint4*)parts, lens, weight, a, n, til, shares, scale_log2, L.d_status);
  L.count();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

size_t kv4_weights_umma_scratch_bytes(int B, int a, int H, int Hkv) {
  return (size_t)B * Hkv * wk_tiling(a, H / Hkv).tiles * WK_ROWS * 32;
}

cudaError_t launch_kv4_weights_umma(const Launch& L, const void* q, size_t ldq, const Kv4& c, const float* lse, float* weight,
                                    int a, int n, int H, const int32_t* lens, void* scratch) {
  return c.hd == 64 ? weights_as<64>(L, (const __nv_bfloat16*)q, ldq, c, lse, weight, a, n, H, lens, (uint4*)scratch)
                    : weights_as<128>(L, (const __nv_bfloat16*)q, ldq, c, lse, weight, a, n, H, lens, (uint4*)scratch);
}

}  // namespace dllm

namespace dllm {
cudaError_t set_debug_skip_kv4_weights(int enable) {
  const int v = enable != 0;
  return cudaMemcpyToSymbol(g_debug_skip, &v, sizeof v);
}
}  // namespace dllm

DLLM_WAIT_LIMIT_HOOK(kv4_weights)
