// What the 8-bit serving operators share: real types, scales, descriptors.
#pragma once

#include <math.h>

#include "common.hpp"

namespace fxpq {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));

// Calls f with a value of the C++ type of a real dtype.
template <typename F>
inline hipError_t for_real(int type, F f) {
  if (type == FXPQ_F32) return f(float());
  if (type == FXPQ_F16) return f((_Float16)0);
  return f((__bf16)0);
}

inline int real_bytes(int type) { return type == FXPQ_F32 ? 4 : 2; }

// N consecutive reals, from an address aligned to N * sizeof(T) bytes (at most 16).
template <typename T, int N>
struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Reals {
  T v[N];
};

template <typename T, int N>
__device__ inline void load_reals(const T* p, float (&out)[N]) {
  const Reals<T, N> r = *reinterpret_cast<const Reals<T, N>*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = (float)r.v[i];
}

template <typename T, int N>
__device__ inline void store_reals(T* p, const float (&x)[N]) {
  Reals<T, N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = (T)x[i];
  *reinterpret_cast<Reals<T, N>*>(p) = r;
}

// Magnitudes below this count as this when a scale is chosen: 127 / a and the
// scale itself stay normal numbers.
constexpr float kScaleFloor = 0x1p-100f;

// The smallest power of two 2^-fl with rne(a * 2^fl) <= 127, for a >= kScaleFloor.
// a = m * 2^e with 1 <= m < 2: fl = 6 - e, or 5 - e where 64 m >= 127.5 (the
// tie 127.5 rounds to the even 128).
__device__ inline float dfx_scale(float a) {
  const unsigned b = __builtin_bit_cast(unsigned, a);
  const int e = (int)(b >> 23) - 127 + ((b & 0x7FFFFFu) >= 0x7F0000u ? 1 : 0);
  return __builtin_bit_cast(float, (unsigned)(e - 6 + 127) << 23);
}

// 1 / s of a power of two s.
__device__ inline float pow2_inverse(float s) {
  return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(unsigned, s));
}

__device__ inline bool finite(float x) {
  return (__builtin_bit_cast(unsigned, x) & 0x7F800000u) != 0x7F800000u;
}

__device__ inline unsigned pack4(int a, int b, int c, int d) {
  return (unsigned)(a & 0xFF) | (unsigned)(b & 0xFF) << 8 | (unsigned)(c & 0xFF) << 16 |
         (unsigned)(d & 0xFF) << 24;
}

// Blocks of one launch: 2^32 threads are a grid's limit.
constexpr int64_t kMaxBlocks = (1 << 24) - 1;

// More than 64 KB of LDS has to be asked for.
inline hipError_t allow_lds(const void* f, int bytes) {
  return bytes > 65536 ? hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}

// ---- launchers -------------------------------------------------------------
struct GemmArgs {
  int64_t M, N, K;
  const int8_t* a;
  int64_t a_count, lda;
  const float* a_scale;
  const int32_t* a_rows;   // null: rows of a in order
  const int32_t* offsets;  // null: one group of M rows
  int experts;
  const int8_t* b;
  const float* b_scale;
  const float* bias;
  void* y;
  int64_t ldy;
  int64_t share;  // of the depth, for one block (split products)
  unsigned* flags;
};

hipError_t launch_token_quantize(const Ctx& c, const void* x, int x_type, int64_t rows, int64_t cols,
                                 int64_t ldx, int rule, int8_t* codes, int64_t ldc, float* scale);
int64_t token_gemm_workspace(int64_t M, int64_t N, int64_t K);
hipError_t launch_token_gemm(const Ctx& c, const GemmArgs& a, int y_type, void* ws);
hipError_t launch_expert_gemm(const Ctx& c, const GemmArgs& a, int y_type);
hipError_t launch_cache_append(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                               const fxpq_rotary* rot, const void* k, int64_t ldk, const void* v,
                               int64_t ldv, const void* q, int64_t ldq, void* q_out, int64_t ldqo,
                               int q_heads, int type);
hipError_t launch_cache_read(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                             void* k_out, void* v_out, int type);
int64_t cache_attention_workspace(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                                  int q_heads);
hipError_t launch_cache_attention(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                                  const void* q, int64_t ldq, int q_heads, float softmax_scale,
                                  int causal, void* out, int64_t ldo, int type, void* ws);

}  // namespace fxpq
