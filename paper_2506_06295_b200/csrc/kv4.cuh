// The K / V cache held in 4 bits: its layout and the conversions the kernels share.
//
// A head's K (or V) of one token, HD numbers, is a row of HD / 2 bytes (element 2i in the low half of byte i, 2i + 1 in
// the high half) and a pair (step, lo) of bf16: code u stands for lo + step * u.  Rows of one (sequence, KV head) are
// contiguous ([B, Hkv, capacity, .]), so a tile of keys is one block of memory; capacity is a multiple of KV4_KEYS, so a
// whole tile may be read wherever a sequence ends.
//
// With v = u - 8 (a small integer, exact in fp16 and bf16)
//     q . k   = step * (q . v) + (lo + 8 step) * sum(q)
//     sum p k = sum (p step) v + sum p (lo + 8 step)
// For few rows the matrix instructions work on these exact integers, the steps and offsets stay in fp32 outside, and centring
// the codes keeps the rounding of p * step from being multiplied by the offset.  What the tcgen05 kernels make of it stands at
// kv4_umma.cu and kv4_weights.cu: exact products step * v for the scores, numbers rounded to fp16 once for the outputs.
#pragma once
#include <cuda_fp16.h>

#include "../../include/dllm.h"
#include "common.cuh"
#include "internal.h"

namespace dllm {

constexpr int KV4_KEYS = 64;  // keys per tile, and what a cache's capacity is a multiple of

// Two codes of a word -> two halves holding u - 8, without a conversion: the integer goes into the significand of a power of two
// (the way Kim et al., arXiv 2211.10017, turn 8- and 4-bit weights into fp16).  LO: nibbles 0 and 4, i.e. bits 0-3 and 16-19; HI: nibbles 1 and 5.
// 0x6400 is 1024 in fp16, whose last place is 1: or-ing a nibble in adds it (16 times it for the high one).
__device__ __forceinline__ uint32_t kv4_half_lo(uint32_t w) {
  uint32_t r;
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(r) : "r"(w));
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&r), __half2half2(__ushort_as_half(0x6408)));  // - 1032
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t kv4_half_hi(uint32_t w) {
  uint32_t r;
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(r) : "r"(w));
  const __half2 h = __hfma2(*reinterpret_cast<const __half2*>(&r), __half2half2(__ushort_as_half(0x2C00)),   // / 16
                            __half2half2(__ushort_as_half(0xD480)));                                         // - 72
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The eight codes of a word as four pairs: p[i] = elements i and i + 4.
__device__ __forceinline__ void kv4_word(uint32_t w, uint32_t (&p)[4]) {
  p[0] = kv4_half_lo(w);
  p[1] = kv4_half_hi(w);
  p[2] = kv4_half_lo(w >> 8);
  p[3] = kv4_half_hi(w >> 8);
}
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 2^x on the special-function unit, 2^-22 off
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void st_shared16(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Operand rows of sixteen 16-bit numbers: 32 bytes with the 32-byte swizzle, K-major, 8-row groups 256 bytes apart.  The
// descriptor, and the place of a row's first or second 16 bytes.
__device__ __forceinline__ uint64_t make_smem_desc_32(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(256 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)6 << 61);
}
__device__ __forceinline__ uint32_t chunk_32(uint32_t base, int row, int chunk) {
  return base + row * 32 + ((chunk ^ ((row >> 2) & 1)) << 4);
}
__device__ __forceinline__ float kv4_step(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float kv4_lo(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

// Unnormalised outputs, which are sums over up to 2^24 keys, are kept times 2^-24: a mean of numbers near the end of fp32's range
// then stays within it on its way.  (Values below 2^-102 lose bits by it: what a key adds is off by 2^-126 of its weight, fp32's
// smallest normal number.)
constexpr float KV4_SUM_DOWN = 1.f / 16777216.f, KV4_SUM_UP = 16777216.f;

// What the host hands to the kernels.
struct Kv4 {
  uint8_t* k = nullptr;      // codes [B, Hkv, cap, hd / 2]
  uint32_t* kp = nullptr;    // (step, lo) [B, Hkv, cap], step in the low half
  uint8_t* v = nullptr;
  uint32_t* vp = nullptr;
  int B = 0, Hkv = 0, cap = 0, hd = 0;
};

// kv4_rows.cu
cudaError_t launch_kv4_store(const Launch& L, const Kv4& c, const void* k, const void* v, size_t ldk, size_t ldv, int dtype,
                             int a, const int32_t* pos, int start);
cudaError_t launch_kv4_load(const Launch& L, const Kv4& c, int n, const int32_t* lens, void* k, void* v, int dtype);
cudaError_t launch_kv4_evict(const Launch& L, const Kv4& src, const float* weight, int n, int keep, int first, int last,
                             const int32_t* lens, const Kv4& dst, float* dst_weight, int32_t* index, int32_t* new_lens);
// kv4_attention.cu.  A call makes its plan once: its scratch is checked against the plan that is launched, whatever another
// thread does to the hook meanwhile.
void set_kv4_plan(int kernel, int splits);   // dllm_debug_kv4_plan
struct Kv4Plan {
  bool umma = false;
  int S = 1;                // ranges of keys
  bool clustered = false;   // they merge inside a cluster, without scratch
};
Kv4Plan plan_kv4(int B, int a, int n, int H, int Hkv);
size_t kv4_attention_scratch_bytes(const Kv4Plan& plan, int B, int a, int H, int hd);
cudaError_t launch_kv4_attention(const Launch& L, const Kv4Plan& plan, const void* q, size_t ldq, const Kv4& c, void* o, float* lse,
                                 int a, int n, int H, const int32_t* lens, float* scratch);
bool plan_kv4_weights(int a, int H, int Hkv);   // whether they take the tcgen05 kernel
size_t kv4_weights_scratch_bytes(bool umma, int B, int a, int H, int Hkv);
cudaError_t launch_kv4_weights(const Launch& L, bool umma, const void* q, size_t ldq, const Kv4& c, const float* lse, float* weight,
                               int a, int n, int H, const int32_t* lens, void* scratch);
// kv4_umma.cu
cudaError_t launch_kv4_umma(const Launch& L, const void* q, size_t ldq, const Kv4& c, void* o, float* lse, int a, int n, int H,
                            const int32_t* lens, float* o_part, float2* ml_part, int S);
cudaError_t set_wait_limit_kv4_umma(unsigned long long ns);
cudaError_t set_debug_skip_kv4_umma(int enable);   // dllm_debug_skip_one_load
// kv4_weights.cu
size_t kv4_weights_umma_scratch_bytes(int B, int a, int H, int Hkv);
cudaError_t launch_kv4_weights_umma(const Launch& L, const void* q, size_t ldq, const Kv4& c, const float* lse, float* weight,
                                    int a, int n, int H, const int32_t* lens, void* scratch);
cudaError_t set_wait_limit_kv4_weights(unsigned long long ns);
cudaError_t set_debug_skip_kv4_weights(int enable);   // dllm_debug_skip_one_load

}  // namespace dllm
