// C entry points of the 8-bit integer products and of the 4-bit K / V cache: checks, plans, launches.
#include <cstdarg>
#include <cstdio>

#include "gemm_s8.cuh"
#include "kv4.cuh"

using namespace dllm;

namespace {

dllm_status fail(dllm_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_last_error(buf);
  return st;
}
dllm_status done(cudaError_t e, const char* what, const char* why = nullptr) {
  return e == cudaSuccess ? DLLM_OK : fail(DLLM_CUDA_ERROR, "%s: %s", what, why ? why : cudaGetErrorString(e));
}
bool known_dtype(int dtype) { return dtype == DLLM_FP32 || dtype == DLLM_BF16; }
bool aligned16(const void* p) { return !((uintptr_t)p & 15); }
// float and int32 arrays, those that are there
template <typename... P>
dllm_status check_words(const P*... p) {
  if (((0 | ... | (uintptr_t)p) & 3) != 0) return fail(DLLM_INVALID_ARG, "an array of float or int32 is not aligned to 4 bytes");
  return DLLM_OK;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
Launch on(void* stream) { return Launch{(cudaStream_t)stream, kernel_status_word(), nullptr}; }

constexpr int MOST_K = 131071;        // 128 * 128 * K stays below 2^31
constexpr int MOST_N = 65535 * 128;   // weight tiles along a grid dimension
constexpr int MOST_ROWS = 1 << 30, MOST_COLS = 1 << 30, MOST_KEYS = 1 << 24;   // indices of these and of a tile behind them: 32 bits

dllm_status check_product(const void* W, size_t ldw, const float* sw, const void* C, int out_dtype, int M, int N, int K) {
  if (!W || !sw || !C || M <= 0 || N <= 0 || K <= 0) return fail(DLLM_INVALID_ARG, "bad arguments of an 8-bit product");
  if (K > MOST_K || N > MOST_N || M > MOST_ROWS)
    return fail(DLLM_UNSUPPORTED, "K must be at most %d, N at most %d and M at most %d", MOST_K, MOST_N, MOST_ROWS);
  if (!known_dtype(out_dtype)) return fail(DLLM_INVALID_ARG, "bad output dtype");
  if (ldw % 16 || ldw < (size_t)K || !aligned16(W))
    return fail(DLLM_INVALID_ARG, "rows of W must be 16-byte aligned and at least K bytes apart");
  if ((uintptr_t)C % (out_dtype == DLLM_BF16 ? 2 : 4)) return fail(DLLM_INVALID_ARG, "the output is not aligned to its type");
  return check_words(sw);
}
dllm_status check_rows(const void* x, size_t ldx, int dtype, int cols) {
  if (!x || !known_dtype(dtype)) return fail(DLLM_INVALID_ARG, "rows must be fp32 or bf16");
  if (ldx < (size_t)cols) return fail(DLLM_INVALID_ARG, "rows overlap: ldx is below their length");
  if ((uintptr_t)x % (dtype == DLLM_BF16 ? 2 : 4)) return fail(DLLM_INVALID_ARG, "rows are not aligned to their type");
  return DLLM_OK;
}

dllm_status check_cache(const dllm_kv4_cache* c, Kv4* out) {
  if (!c || !c->d_k_codes || !c->d_k_params || !c->d_v_codes || !c->d_v_params || c->B <= 0 || c->n_kv_heads <= 0 ||
      c->capacity <= 0)
    return fail(DLLM_INVALID_ARG, "bad 4-bit cache");
  if (c->head_dim != 64 && c->head_dim != 128) return fail(DLLM_UNSUPPORTED, "a 4-bit cache has head_dim 64 or 128");
  if (c->capacity % KV4_KEYS) return fail(DLLM_INVALID_ARG, "the capacity must be a multiple of %d", KV4_KEYS);
  if (c->capacity > MOST_KEYS) return fail(DLLM_UNSUPPORTED, "the capacity must be at most %d", MOST_KEYS);
  if (c->n_kv_heads > 65535 || (long)c->B * c->n_kv_heads > 65535)
    return fail(DLLM_UNSUPPORTED, "at most 65535 (sequence, KV head) pairs");
  if (!aligned16(c->d_k_codes) || !aligned16(c->d_k_params) || !aligned16(c->d_v_codes) || !aligned16(c->d_v_params))
    return fail(DLLM_INVALID_ARG, "the cache's tensors must be 16-byte aligned");
  *out = Kv4{(uint8_t*)c->d_k_codes, (uint32_t*)c->d_k_params, (uint8_t*)c->d_v_codes, (uint32_t*)c->d_v_params, c->B,
             c->n_kv_heads, c->capacity, c->head_dim};
  return DLLM_OK;
}
dllm_status check_queries(const void* q, size_t ldq, const Kv4& c, int a, int n, int H) {
  if (!q || a <= 0 || n <= 0 || n > c.cap || H <= 0 || H % c.Hkv)
    return fail(DLLM_INVALID_ARG, "bad attention arguments: a and n positive, n within the capacity, heads a multiple of KV heads");
  if (!aligned16(q) || ldq % 8 || ldq < (size_t)H * c.hd)
    return fail(DLLM_INVALID_ARG, "rows of queries must be 16-byte aligned and at least n_heads * head_dim elements apart");
  if ((long)a * H > (1L << 30) / c.B) return fail(DLLM_UNSUPPORTED, "too many query rows for one call");
  return DLLM_OK;
}

#define TRY(expr)                       \
  do {                                  \
    const dllm_status st_ = (expr);     \
    if (st_ != DLLM_OK) return st_;     \
  } while (0)

}  // namespace

extern "C" {

dllm_status dllm_quantize_rows_s8(const void* d_x, size_t ldx, int dtype, void* d_q, size_t ldq, float* d_scale, int rows,
                                  int cols, void* stream) {
  if (!d_q || !d_scale || rows <= 0 || cols <= 0) return fail(DLLM_INVALID_ARG, "bad arguments of a row quantisation");
  if (rows > MOST_ROWS || cols > MOST_COLS) return fail(DLLM_UNSUPPORTED, "at most %d rows and columns", MOST_ROWS);
  TRY(check_rows(d_x, ldx, dtype, cols));
  TRY(check_words(d_scale));
  if (ldq % 16 || ldq < (size_t)cols || !aligned16(d_q))
    return fail(DLLM_INVALID_ARG, "rows of q must be 16-byte aligned and at least `cols` bytes apart");
  return done(launch_quantize_rows_s8(on(stream), d_x, ldx, dtype, (int8_t*)d_q, ldq, d_scale, rows, cols), "row quantisation");
}

size_t dllm_gemm_s8_scratch_bytes(int M, int N, int K) {
  if (M <= 0 || N <= 0 || K <= 0 || K > MOST_K || N > MOST_N || M > MOST_ROWS) return 0;
  return gemm_s8_scratch_bytes(M, N, plan_gemm_s8(M, N, K));
}

dllm_status dllm_gemm_s8(const void* d_A, size_t lda, const float* d_sa, const void* d_W, size_t ldw, const float* d_sw,
                         void* d_C, int out_dtype, int M, int N, int K, void* d_scratch, size_t scratch_bytes, void* stream) {
  if (!d_A || !d_sa) return fail(DLLM_INVALID_ARG, "bad arguments of an 8-bit product");
  TRY(check_product(d_W, ldw, d_sw, d_C, out_dtype, M, N, K));
  TRY(check_words(d_sa));
  if (lda % 16 || lda < (size_t)K || !aligned16(d_A))
    return fail(DLLM_INVALID_ARG, "rows of A must be 16-byte aligned and at least K bytes apart");
  const GemmPlan plan = plan_gemm_s8(M, N, K);
  const size_t need = gemm_s8_scratch_bytes(M, N, plan);
  if (need && (!d_scratch || !aligned16(d_scratch) || scratch_bytes < need))
    return fail(DLLM_INVALID_ARG, "this product needs %zu bytes of 16-byte aligned scratch", need);
  const char* why = nullptr;
  const cudaError_t e = launch_gemm_s8(on(stream), (const int8_t*)d_A, lda, d_sa, (const int8_t*)d_W, ldw, d_sw, d_C, out_dtype,
                                       M, N, K, plan, d_scratch, &why);
  return done(e, "8-bit GEMM", why);
}

size_t dllm_linear_s8_scratch_bytes(int M, int N, int K) {
  if (M <= 0 || N <= 0 || K <= 0 || K > MOST_K || N > MOST_N || M > MOST_ROWS) return 0;
  const size_t ldq = ((size_t)K + 15) & ~(size_t)15;
  return up256((size_t)M * ldq) + up256((size_t)M * 4) + gemm_s8_scratch_bytes(M, N, plan_gemm_s8(M, N, K));
}

dllm_status dllm_linear_s8(const void* d_x, size_t ldx, int dtype, const void* d_W, size_t ldw, const float* d_sw, void* d_y,
                           int out_dtype, int M, int N, int K, void* d_scratch, size_t scratch_bytes, void* stream) {
  TRY(check_product(d_W, ldw, d_sw, d_y, out_dtype, M, N, K));
  TRY(check_rows(d_x, ldx, dtype, K));
  const size_t need = dllm_linear_s8_scratch_bytes(M, N, K), ldq = ((size_t)K + 15) & ~(size_t)15;
  if (!d_scratch || !aligned16(d_scratch) || scratch_bytes < need)
    return fail(DLLM_INVALID_ARG, "this call needs %zu bytes of 16-byte aligned scratch", need);
  int8_t* const q = (int8_t*)d_scratch;
  float* const sa = (float*)(q + up256((size_t)M * ldq));
  void* const slabs = (char*)sa + up256((size_t)M * 4);
  Launch L = on(stream);
  cudaError_t e = launch_quantize_rows_s8(L, d_x, ldx, dtype, q, ldq, sa, M, K);
  if (e != cudaSuccess) return done(e, "row quantisation");
  // The quantisation was launched plainly: when it runs, everything before this call has completed.  So the product may start
  // beside it and ask for its weights.
  L.pdl = true;
  const char* why = nullptr;
  e = launch_gemm_s8(L, q, ldq, sa, (const int8_t*)d_W, ldw, d_sw, d_y, out_dtype, M, N, K, plan_gemm_s8(M, N, K), slabs, &why);
  return done(e, "8-bit GEMM", why);
}

dllm_status dllm_kv4_store(const dllm_kv4_cache* cache, const void* d_k, size_t ldk, const void* d_v, size_t ldv, int dtype,
                           int a, const int32_t* d_pos, int start, void* stream) {
  Kv4 c;
  TRY(check_cache(cache, &c));
  if (a <= 0 || start < 0 || (long)a * c.B > (1L << 30)) return fail(DLLM_INVALID_ARG, "bad number of rows or start");
  if (!d_pos && (long)start + a > c.cap) return fail(DLLM_INVALID_ARG, "rows %d .. %d do not fit the capacity", start, start + a - 1);
  TRY(check_rows(d_k, ldk, dtype, c.Hkv * c.hd));
  TRY(check_rows(d_v, ldv, dtype, c.Hkv * c.hd));
  TRY(check_words(d_pos));
  return done(launch_kv4_store(on(stream), c, d_k, d_v, ldk, ldv, dtype, a, d_pos, start), "4-bit store");
}

dllm_status dllm_kv4_load(const dllm_kv4_cache* cache, int n, const int32_t* d_lens, void* d_k, void* d_v, int dtype,
                          void* stream) {
  Kv4 c;
  TRY(check_cache(cache, &c));
  if (n <= 0 || n > c.cap || (!d_k && !d_v)) return fail(DLLM_INVALID_ARG, "n must lie within the capacity, K or V be asked for");
  if (!known_dtype(dtype)) return fail(DLLM_INVALID_ARG, "bad dtype");
  if (((uintptr_t)d_k | (uintptr_t)d_v) % (dtype == DLLM_BF16 ? 2 : 4))
    return fail(DLLM_INVALID_ARG, "the outputs are not aligned to their type");
  TRY(check_words(d_lens));
  return done(launch_kv4_load(on(stream), c, n, d_lens, d_k, d_v, dtype), "4-bit load");
}

dllm_status dllm_debug_kv4_plan(int kernel, int splits) {
  if (kernel < 0 || kernel > 2 || splits < 0 || splits > 64)
    return fail(DLLM_INVALID_ARG, "dllm_debug_kv4_plan: kernel 0, 1 or 2, splits 0 to 64");
  set_kv4_plan(kernel, splits);
  return DLLM_OK;
}

size_t dllm_attention_kv4_scratch_bytes(int B, int a, int n, int n_heads, int n_kv_heads, int head_dim) {
  if (B <= 0 || a <= 0 || n <= 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads || (head_dim != 64 && head_dim != 128) ||
      (long)a * n_heads > (1L << 30) / B)
    return 0;
  return kv4_attention_scratch_bytes(plan_kv4(B, a, n, n_heads, n_kv_heads), B, a, n_heads, head_dim);
}

dllm_status dllm_attention_kv4(const void* d_q, size_t ldq, const dllm_kv4_cache* cache, void* d_o, float* d_lse, int a, int n,
                               int n_heads, const int32_t* d_lens, void* d_scratch, size_t scratch_bytes, void* stream) {
  Kv4 c;
  TRY(check_cache(cache, &c));
  TRY(check_queries(d_q, ldq, c, a, n, n_heads));
  if (!d_o || !aligned16(d_o)) return fail(DLLM_INVALID_ARG, "the output must be 16-byte aligned");
  TRY(check_words(d_lse, d_lens));
  const Kv4Plan plan = plan_kv4(c.B, a, n, n_heads, c.Hkv);
  const size_t need = kv4_attention_scratch_bytes(plan, c.B, a, n_heads, c.hd);
  if (need && (!d_scratch || !aligned16(d_scratch) || scratch_bytes < need))
    return fail(DLLM_INVALID_ARG, "this attention needs %zu bytes of 16-byte aligned scratch", need);
  return done(launch_kv4_attention(on(stream), plan, d_q, ldq, c, d_o, d_lse, a, n, n_heads, d_lens, (float*)d_scratch),
              "attention over the 4-bit cache");
}

size_t dllm_attention_weights_kv4_scratch_bytes(int B, int a, int n_heads, int n_kv_heads) {
  if (B <= 0 || a <= 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads || (long)a * n_heads > (1L << 30) / B) return 0;
  return kv4_weights_scratch_bytes(plan_kv4_weights(a, n_heads, n_kv_heads), B, a, n_heads, n_kv_heads);
}

dllm_status dllm_attention_weights_kv4(const void* d_q, size_t ldq, const dllm_kv4_cache* cache, const float* d_lse,
                                       float* d_weight, int a, int n, int n_heads, const int32_t* d_lens, void* d_scratch,
                                       size_t scratch_bytes, void* stream) {
  Kv4 c;
  TRY(check_cache(cache, &c));
  TRY(check_queries(d_q, ldq, c, a, n, n_heads));
  if (!d_lse || !d_weight) return fail(DLLM_INVALID_ARG, "lse or weight is NULL");
  TRY(check_words(d_lse, d_weight, d_lens));
  const bool umma = plan_kv4_weights(a, n_heads, c.Hkv);
  const size_t need = kv4_weights_scratch_bytes(umma, c.B, a, n_heads, c.Hkv);
  if (need && (!d_scratch || !aligned16(d_scratch) || scratch_bytes < need))
    return fail(DLLM_INVALID_ARG, "these weights need %zu bytes of 16-byte aligned scratch", need);
  return done(launch_kv4_weights(on(stream), umma, d_q, ldq, c, d_lse, d_weight, a, n, n_heads, d_lens, d_scratch), "attention weights");
}

dllm_status dllm_kv4_evict(const dllm_kv4_cache* from, const float* d_weight, int n, int keep, int first, int last,
                           const int32_t* d_lens, const dllm_kv4_cache* to, float* d_to_weight, int32_t* d_index,
                           int32_t* d_to_lens, void* stream) {
  Kv4 s, d;
  TRY(check_cache(from, &s));
  TRY(check_cache(to, &d));
  if (!d_weight || !d_to_weight || !d_index || !d_to_lens || !aligned16(d_weight))
    return fail(DLLM_INVALID_ARG, "an argument of the eviction is NULL, or its weights are not 16-byte aligned");
  TRY(check_words(d_lens, d_to_weight, d_index, d_to_lens));
  if (s.B != d.B || s.Hkv != d.Hkv || s.hd != d.hd) return fail(DLLM_INVALID_ARG, "the caches differ in batch, heads or head_dim");
  if (n <= 0 || n > s.cap || keep <= 0 || keep > d.cap || first < 0 || last < 0 || (long)first + last > keep)
    return fail(DLLM_INVALID_ARG, "eviction: n within the capacity, 0 <= first + last <= keep <= the new capacity");
  const size_t sr = (size_t)s.B * s.Hkv * s.cap, dr = (size_t)d.B * d.Hkv * d.cap;
  struct Span { const char *p; size_t n; };
  const Span in[6] = {{(const char*)s.k, sr * s.hd / 2}, {(const char*)s.v, sr * s.hd / 2}, {(const char*)s.kp, sr * 4},
                      {(const char*)s.vp, sr * 4}, {(const char*)d_weight, sr * 4}, {(const char*)d_lens, d_lens ? (size_t)s.B * 4 : 0}};
  const Span out[7] = {{(const char*)d.k, dr * d.hd / 2}, {(const char*)d.v, dr * d.hd / 2}, {(const char*)d.kp, dr * 4},
                       {(const char*)d.vp, dr * 4}, {(const char*)d_to_weight, dr * 4},
                       {(const char*)d_index, (size_t)d.B * d.Hkv * keep * 4}, {(const char*)d_to_lens, (size_t)d.B * 4}};
  auto meet = [](const Span& x, const Span& y) { return x.n && y.n && x.p < y.p + y.n && y.p < x.p + x.n; };
  for (const Span& y : out) {
    for (const Span& x : in)
      if (meet(x, y)) return fail(DLLM_INVALID_ARG, "eviction: what is written overlaps what is read");
    for (const Span* z = out; z != &y; ++z)   // (the gather reads the index back: it must hold what the selection wrote)
      if (meet(*z, y)) return fail(DLLM_INVALID_ARG, "eviction: two of the outputs overlap");
  }
  return done(launch_kv4_evict(on(stream), s, d_weight, n, keep, first, last, d_lens, d, d_to_weight, d_index, d_to_lens),
              "eviction");
}

}  // extern "C"
