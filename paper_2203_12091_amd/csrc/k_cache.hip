// Appending to the paged 8-bit cache (with the position rotation) and reading
// its values back.
#include <type_traits>

#include "kv.hpp"
#include "values.hpp"

namespace fxpq {
namespace {

struct AppendArgs {
  fxpq_kv_cache c;
  fxpq_kv_batch b;
  fxpq_rotary rot;  // dims 0: none
  const void *k, *v, *q;
  void* q_out;
  int64_t ldk, ldv, ldq, ldqo;
  int q_heads;
  int segs;     // pages that one sequence's new tokens can touch
  // whole-unit kernels
  int page_log2;
  int head_blocks;  // blocks along the heads
  int kv_blocks;    // blocks of a sequence for keys and values; the queries' follow
  unsigned* flags;
};

// The products and the sum of a rotation are rounded one by one (no fused
// multiply-add), so that the codes do not depend on how a compiler pairs them.
__device__ inline float rotate_first(float x1, float x2, float c, float s) {
#pragma clang fp contract(off)
  const float a = x1 * c, b = x2 * s;
  return a - b;
}
__device__ inline float rotate_second(float x1, float x2, float c, float s) {
#pragma clang fp contract(off)
  const float a = x2 * c, b = x1 * s;
  return a + b;
}

// A new token lies past the rotation's positions.
__device__ inline bool past_positions(const AppendArgs& a, const SeqDev& q) {
  return a.rot.dims && q.fresh > 0 && q.len > a.rot.positions;
}

// Dimension d of a row after the rotation of position pos.
template <typename T>
__device__ inline float rotated(const T* row, int d, const fxpq_rotary& r, int pos) {
  if (d >= r.dims) return (float)row[d];
  const int half = r.dims / 2;
  const bool second = r.interleaved ? d & 1 : d >= half;
  const int i = r.interleaved ? d >> 1 : second ? d - half : d;
  const float x1 = (float)row[r.interleaved ? 2 * i : i];
  const float x2 = (float)row[r.interleaved ? 2 * i + 1 : i + half];
  const float c = r.cos[(int64_t)pos * half + i], s = r.sin[(int64_t)pos * half + i];
  return second ? rotate_second(x1, x2, c, s) : rotate_first(x1, x2, c, s);
}

// Old code of a block whose scale grew by 1 / ratio.
__device__ inline int regrown(int code, float ratio) { return (int)rintf((float)code * ratio); }

// Rotated queries of one new token, pair by pair (in place is fine).
template <typename T>
__device__ inline void rotate_query_pairs(const AppendArgs& a, const SeqDev& q, int token) {
  if (token >= q.fresh) return;
  const int pos = q.len - q.fresh + token, D = a.c.dim, W = a.q_heads * D;
  const T* src = static_cast<const T*>(a.q) + (q.first + (int64_t)token) * a.ldq;
  T* dst = static_cast<T*>(a.q_out) + (q.first + (int64_t)token) * a.ldqo;
  const int half = a.rot.dims / 2, pairs = a.q_heads * half;
  for (int i = threadIdx.x; i < pairs; i += 256) {
    const int h = i / half, j = i % half;
    const int d1 = h * D + (a.rot.interleaved ? 2 * j : j);
    const int d2 = a.rot.interleaved ? d1 + 1 : d1 + half;
    const float x1 = (float)src[d1], x2 = (float)src[d2];
    const float c = a.rot.cos[(int64_t)pos * half + j], s = a.rot.sin[(int64_t)pos * half + j];
    dst[d1] = (T)rotate_first(x1, x2, c, s);
    dst[d2] = (T)rotate_second(x1, x2, c, s);
  }
  if (a.rot.dims < D)
    for (int i = threadIdx.x; i < W; i += 256)
      if (i % D >= a.rot.dims) dst[i] = src[i];
}

// One block per 16 new tokens' slots (x), sequence (y) and head (z).
template <typename T>
__global__ __launch_bounds__(256) void k_cache_read(fxpq_kv_cache c, fxpq_kv_batch b, T* k_out,
                                                    T* v_out, unsigned* flags) {
  const int s = blockIdx.y, head = blockIdx.z;
  const SeqDev q = seq_of(b, c.page, s);
  if (!q.ok) {
    if (blockIdx.x == 0 && head == 0 && threadIdx.x == 0) raise_flag(flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int pos0 = q.len - q.fresh;
  const int t0 = (pos0 & ~15) + blockIdx.x * 16;
  if (q.fresh == 0 || t0 >= q.len) return;
  const int page = b.table[(int64_t)s * b.table_ld + t0 / c.page], slot = t0 % c.page;
  const bool there = page >= 0 && page < c.pages;
  if (!there && threadIdx.x == 0) raise_flag(flags, FXPQ_FLAG_RANGE);
  const int64_t at = (int64_t)page * c.heads + head;
  const float ks = there ? c.k_scale[at] : 0.0f, vs = there ? c.v_scale[at] : 0.0f;
  for (int i = threadIdx.x; i < 16 * c.dim; i += 256) {
    const int t = i / c.dim, d = i % c.dim;
    if (t0 + t < pos0 || t0 + t >= q.len) continue;
    const int64_t o = ((q.first + (int64_t)(t0 + t - pos0)) * c.heads + head) * c.dim + d;
    if (k_out) k_out[o] = (T)(there ? (float)c.k[k_offset(c, page, head, slot + t) + d] * ks : 0.0f);
    if (v_out) v_out[o] = (T)(there ? (float)c.v[v_offset(c, page, head, slot + t, d)] * vs : 0.0f);
  }
}

// ---- whole units ---------------------------------------------------------------
// A unit is 16 token slots of one page and head; each of its LP lanes takes 8
// dimensions of all of them, with 16-byte loads and stores, and keeps the values in
// registers between finding the page's largest magnitude and writing the codes: one
// read of the inputs.  A block of 256 threads is 256 / LP units, whole pages of
// some heads.  What this needs of the arguments (alignment to 16 bytes, rotated
// dimensions in multiples of 16) is append_units_fit(); anything else goes through
// the element-by-element kernels above.
template <typename T>
__device__ inline void load8(const T* p, float (&x)[8]) {
  constexpr int W = 16 / sizeof(T);
#pragma unroll
  for (int k = 0; k < 8; k += W) {
    float u[W];
    load_reals<T, W>(p + k, u);
#pragma unroll
    for (int j = 0; j < W; ++j) x[k + j] = u[j];
  }
}
template <typename T>
__device__ inline void store8(T* p, const float (&x)[8]) {
  constexpr int W = 16 / sizeof(T);
#pragma unroll
  for (int k = 0; k < 8; k += W) {
    float u[W];
#pragma unroll
    for (int j = 0; j < W; ++j) u[j] = x[k + j];
    store_reals<T, W>(p + k, u);
  }
}

// Dimensions d .. d + 7 of N key rows at neighbouring positions, rotated; every
// load is issued before the first is used.  Lanes past the rotated dimensions load
// what they have in reach and keep their values.
template <typename T, int N>
__device__ inline void rotated_rows(const T* const (&row)[N], int d, const fxpq_rotary& r, const int (&pos)[N],
                                    float (&x)[N][8]) {
  if (r.dims == 0) {
#pragma unroll
    for (int t = 0; t < N; ++t) load8(row[t] + d, x[t]);
    return;
  }
  const int half = r.dims / 2;
  const bool turns = d < r.dims;
  if (r.interleaved) {
    const int i = turns ? d / 2 : 0;
    float c[N][4], s[N][4];
#pragma unroll
    for (int t = 0; t < N; ++t) {
      load8(row[t] + d, x[t]);
      load_reals<float, 4>(r.cos + (int64_t)pos[t] * half + i, c[t]);
      load_reals<float, 4>(r.sin + (int64_t)pos[t] * half + i, s[t]);
    }
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x1 = x[t][2 * k], x2 = x[t][2 * k + 1];
        x[t][2 * k] = turns ? rotate_first(x1, x2, c[t][k], s[t][k]) : x1;
        x[t][2 * k + 1] = turns ? rotate_second(x1, x2, c[t][k], s[t][k]) : x2;
      }
    return;
  }
  const bool second = d >= half;
  const int i = !turns ? 0 : second ? d - half : d, mate = !turns ? d : second ? i : i + half;
  float other[N][8], c[N][8], s[N][8];
#pragma unroll
  for (int t = 0; t < N; ++t) {
    load8(row[t] + d, x[t]);
    load8(row[t] + mate, other[t]);
    load8(r.cos + (int64_t)pos[t] * half + i, c[t]);
    load8(r.sin + (int64_t)pos[t] * half + i, s[t]);
  }
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float y = second ? rotate_second(other[t][k], x[t][k], c[t][k], s[t][k])
                             : rotate_first(x[t][k], other[t][k], c[t][k], s[t][k]);
      x[t][k] = turns ? y : x[t][k];
    }
}

// Queries of kQueryTokens new tokens from `token` on.  A thread takes 16 dimensions
// of a head and of each of the tokens: 8 pairs whole (in place is fine), or 16 that
// do not rotate, by the same instructions, with every load issued before the first
// is used.
constexpr int kQueryTokens = 2;
template <typename T>
__device__ inline void rotate_queries(const AppendArgs& a, const SeqDev& q, int token) {
  constexpr int N = kQueryTokens;
  if (token >= q.fresh) return;
  const int D = a.c.dim, half = a.rot.dims / 2, per_head = D / 16, turned = a.rot.dims / 16;
  for (int i = threadIdx.x; i < per_head * a.q_heads; i += 256) {
    const int head = i / per_head, p = i - head * per_head;
    const bool turns = p < turned;
    const int d1 = turns && !a.rot.interleaved ? 8 * p : 16 * p, d2 = turns && !a.rot.interleaved ? d1 + half : d1 + 8;
    float x[N][8], y[N][8], c[N][8], s[N][8];
#pragma unroll
    for (int t = 0; t < N; ++t) {
      const int tok = min(token + t, q.fresh - 1);
      const T* src = static_cast<const T*>(a.q) + (q.first + (int64_t)tok) * a.ldq + (int64_t)head * D;
      load8(src + d1, x[t]);
      load8(src + d2, y[t]);
      if (turned > 0) {
        const int64_t at = (int64_t)(q.len - q.fresh + tok) * half + (turns ? 8 * p : 0);
        load8(a.rot.cos + at, c[t]);
        load8(a.rot.sin + at, s[t]);
      }
    }
#pragma unroll
    for (int t = 0; t < N; ++t) {
      if (turns && a.rot.interleaved) {  // neighbours of the 16 values
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float(&v)[8] = k < 4 ? x[t] : y[t];
          const float x1 = v[2 * (k & 3)], x2 = v[2 * (k & 3) + 1];
          v[2 * (k & 3)] = rotate_first(x1, x2, c[t][k], s[t][k]);
          v[2 * (k & 3) + 1] = rotate_second(x1, x2, c[t][k], s[t][k]);
        }
      } else if (turns) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float x1 = x[t][k], x2 = y[t][k];
          x[t][k] = rotate_first(x1, x2, c[t][k], s[t][k]);
          y[t][k] = rotate_second(x1, x2, c[t][k], s[t][k]);
        }
      }
      if (token + t >= q.fresh) continue;
      T* dst = static_cast<T*>(a.q_out) + (q.first + (int64_t)(token + t)) * a.ldqo + (int64_t)head * D;
      store8(dst + d1, x[t]);
      store8(dst + d2, y[t]);
    }
  }
}

// What a block of keys or values works on.
struct PageOf {
  bool any;   // the page has new tokens of the sequence, and lies in the cache
  bool value;
  int page, nth, head0;  // of the cache, of the sequence; the block's first head
  int lo, hi;            // its new slots
};
__device__ inline PageOf page_of(const AppendArgs& a, const SeqDev& q, int heads) {
  PageOf p;
  const int pos0 = q.len - q.fresh, seg = (int)(blockIdx.x >> 1) / a.head_blocks;
  p.value = blockIdx.x & 1;
  p.head0 = ((int)(blockIdx.x >> 1) - seg * a.head_blocks) * heads;
  p.nth = (pos0 >> a.page_log2) + seg;
  p.any = q.fresh > 0 && p.nth <= (q.len - 1) >> a.page_log2;
  if (!p.any) return p;
  p.page = a.b.table[(int64_t)blockIdx.y * a.b.table_ld + p.nth];
  p.lo = max(pos0 - (p.nth << a.page_log2), 0);
  p.hi = min(q.len - (p.nth << a.page_log2), a.c.page);
  if (p.page < 0 || p.page >= a.c.pages) {
    if (threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    p.any = false;
  }
  return p;
}

// The codes of 8 dimensions in the first `old` of up to 16 slots of a block of values,
// and of up to 8 slots of keys, after their scale grew: whole words, whose loads are
// issued together (64 sequences whose pages all grow at their last slot, 8 heads of 128:
// pages of 16 tokens 7.1 us by words and 26.6 byte by byte, of 128 19.1 and 220.7;
// without growth 6.4).
__device__ inline void requantize_values(int8_t* at, int old, float ratio) {
  uint4 w[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = *reinterpret_cast<const uint4*>(at + 16 * k);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    unsigned* words = reinterpret_cast<unsigned*>(&w[k]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int c[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int was = (int8_t)(words[i] >> (8 * e));
        c[e] = 4 * i + e < old ? regrown(was, ratio) : was;
      }
      words[i] = pack4(c[0], c[1], c[2], c[3]);
    }
    *reinterpret_cast<uint4*>(at + 16 * k) = w[k];
  }
}
__device__ inline void requantize_keys(int8_t* at, int row, int old, float ratio) {
  uint2 w[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) w[t] = *reinterpret_cast<const uint2*>(at + (int64_t)min(t, old - 1) * row);
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    int c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) c[k] = regrown((int8_t)((k < 4 ? w[t].x : w[t].y) >> (8 * (k & 3))), ratio);
    if (t < old)
      *reinterpret_cast<uint2*>(at + (int64_t)t * row) = uint2{pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7])};
  }
}

constexpr int kFewTokens = 8;    // new tokens of a sequence up to which k_append_few runs

// Few new tokens: one lane group of LP lanes per head goes over the page's new
// tokens, 8 dimensions a lane, twice (the second time from the cache).  Small code
// and no register arrays: what a step of decoding waits for is latency.  VEC false:
// any alignment and any rotated dimensions, value by value.
template <typename T, int LP, bool VEC>
__global__ __launch_bounds__(256) void k_append_few(AppendArgs a) {
  constexpr int U = 256 / LP;
  const int D = a.c.dim, P = a.c.page;
  const SeqDev q = seq_of(a.b, P, blockIdx.y);
  if (!q.ok || past_positions(a, q)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  if ((int)blockIdx.x >= a.kv_blocks) {
    if constexpr (VEC) rotate_queries<T>(a, q, ((int)blockIdx.x - a.kv_blocks) * kQueryTokens);
    else rotate_query_pairs<T>(a, q, (int)blockIdx.x - a.kv_blocks);
    return;
  }
  const PageOf p = page_of(a, q, U);
  if (!p.any) return;
  const int head = p.head0 + (int)threadIdx.x / LP, d0 = (int)threadIdx.x % LP * 8;
  const bool mine = head < a.c.heads && d0 < D;
  const T* src = static_cast<const T*>(p.value ? a.v : a.k) + (int64_t)head * D;
  const int64_t ld = p.value ? a.ldv : a.ldk, row0 = q.first + (int64_t)p.nth * P - (q.len - q.fresh);
  float* scale = (p.value ? a.c.v_scale : a.c.k_scale) + (int64_t)p.page * a.c.heads + (mine ? head : 0);
  const float old = *scale;
  bool bad = false;
  auto get = [&](int slot, float(&x)[8]) {
    const T* row = src + (row0 + slot) * ld;
    if constexpr (VEC) {
      if (p.value) {
        load8(row + d0, x);
      } else {
        float y[1][8];
        rotated_rows<T, 1>({row}, d0, a.rot, {p.nth * P + slot}, y);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = y[0][k];
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = p.value ? (float)row[d0 + k] : rotated(row, d0 + k, a.rot, p.nth * P + slot);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (!finite(x[k])) {
        bad = true;
        x[k] = 0.0f;
      }
  };
  float x[8], top = 0.0f;
  if (mine)
    for (int slot = p.lo; slot < p.hi; ++slot) {
      get(slot, x);
#pragma unroll
      for (int k = 0; k < 8; ++k) top = fmaxf(top, fabsf(x[k]));
    }
#pragma unroll
  for (int d = LP / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));  // over a head's lanes, of one wave
  if (!mine) return;
  float now = dfx_scale(fmaxf(top, kScaleFloor)), ratio = 1.0f;
  if (p.lo > 0) {
    now = fmaxf(now, old);
    ratio = old / now;
  }
  if (d0 == 0) *scale = now;
  if (bad) raise_flag(a.flags, FXPQ_FLAG_NONFINITE);
  const float inv = 1.0f / now;  // exact: a power of two, unless the caller stored another old scale
  int8_t* base = p.value ? a.c.v + v_offset(a.c, p.page, head, 0, d0) : a.c.k + k_offset(a.c, p.page, head, 0) + d0;
  if (ratio < 1.0f && p.value) {
    for (int t0 = 0; t0 < p.lo; t0 += 16) requantize_values(base + (int64_t)t0 * D, p.lo - t0, ratio);
  } else if (ratio < 1.0f) {
    for (int t0 = 0; t0 < p.lo; t0 += 8) requantize_keys(base + (int64_t)t0 * D, D, p.lo - t0, ratio);
  }
  for (int slot = p.lo; slot < p.hi; ++slot) {
    if (slot != p.hi - 1 || p.hi - p.lo > 1) get(slot, x);  // a lone token is still there
    int c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) c[k] = (int)rintf(x[k] * inv);
    if (p.value) {
      int8_t* at = base + (int64_t)(slot & ~15) * D + (slot & 15);
#pragma unroll
      for (int k = 0; k < 8; ++k) at[k * 16] = (int8_t)c[k];
    } else {
      *reinterpret_cast<uint2*>(base + (int64_t)slot * D) = uint2{pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7])};
    }
  }
}

// The queries of many new tokens, in a launch of their own: with the registers of
// the keys' and values' code there would be two waves a SIMD.  11323 tokens of 32
// heads of 128: 45 us, 4.1 TB/s (by 8 dimensions a lane in two branches 72).
template <typename T>
__global__ __launch_bounds__(256) void k_rotate_queries(AppendArgs a) {
  const SeqDev q = seq_of(a.b, a.c.page, blockIdx.y);
  if (!q.ok || past_positions(a, q)) return;
  rotate_queries<T>(a, q, (int)blockIdx.x * kQueryTokens);
}

// blockIdx.x: keys or values (fastest), heads, page of the new tokens; y: sequence.
// 11323 tokens of 8 heads of 128 (f16, pages of 64): 36 us, 2 TB/s; 226 registers (256
// in fp32) leave two waves a SIMD to cover the loads.
template <typename T, int LP>
__global__ __launch_bounds__(256) void k_append_units(AppendArgs a) {
  constexpr int U = 256 / LP;
  __shared__ float tops[U];
  const int D = a.c.dim, P = a.c.page;
  const SeqDev q = seq_of(a.b, P, blockIdx.y);
  if (!q.ok || past_positions(a, q)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int subs_log2 = a.page_log2 - 4;
  const PageOf p = page_of(a, q, U >> subs_log2);
  if (!p.any) return;
  const bool value = p.value;
  const int page = p.page, nth = p.nth, lo = p.lo, hi = p.hi;
  const int unit = threadIdx.x / LP, d0 = threadIdx.x % LP * 8;
  const int head = p.head0 + (unit >> subs_log2);
  const int t0 = (unit & ((1 << subs_log2) - 1)) * 16;  // first slot of the unit
  const bool mine = head < a.c.heads && d0 < D;
  float x[16][8];
#pragma unroll
  for (int t = 0; t < 16; ++t)
#pragma unroll
    for (int k = 0; k < 8; ++k) x[t][k] = 0.0f;
  float top = 0.0f;
  bool bad = false;
  if (mine) {
    const T* src = static_cast<const T*>(value ? a.v : a.k) + (int64_t)head * D;
    const int64_t ld = value ? a.ldv : a.ldk, row0 = q.first + (int64_t)nth * P - (q.len - q.fresh);
    constexpr int N = sizeof(T) == 4 ? 4 : 8;  // rows whose loads are in flight together
#pragma unroll
    for (int g = 0; g < 16; g += N) {
      if (t0 + g >= hi || t0 + g + N <= lo) continue;
      // rows that are not new are any new row, and dropped
      const T* row[N];
      int pos[N];
      float y[N][8];
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const int slot = min(max(t0 + g + t, lo), hi - 1);
        row[t] = src + (row0 + slot) * ld;
        pos[t] = nth * P + slot;
      }
      if (value) {
#pragma unroll
        for (int t = 0; t < N; ++t) load8(row[t] + d0, y[t]);
      } else {
        rotated_rows<T, N>(row, d0, a.rot, pos, y);
      }
#pragma unroll
      for (int t = 0; t < N; ++t)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const bool fine = finite(y[t][k]), in = t0 + g + t >= lo && t0 + g + t < hi;
          bad |= in && !fine;
          x[g + t][k] = fine && in ? y[t][k] : 0.0f;
          top = fmaxf(top, fabsf(x[g + t][k]));
        }
    }
  }
#pragma unroll
  for (int d = LP / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (threadIdx.x % LP == 0) tops[unit] = top;
  float* scale = (value ? a.c.v_scale : a.c.k_scale) + (int64_t)page * a.c.heads + (mine ? head : 0);
  const float old = *scale;
  __syncthreads();
  for (int u = 0; u < 1 << subs_log2; ++u) top = fmaxf(top, tops[(unit & ~((1 << subs_log2) - 1)) + u]);
  if (!mine) return;
  float now = dfx_scale(fmaxf(top, kScaleFloor)), ratio = 1.0f;
  if (lo > 0) {
    now = fmaxf(now, old);
    ratio = old / now;
  }
  if (t0 == 0 && d0 == 0) *scale = now;
  if (bad) raise_flag(a.flags, FXPQ_FLAG_NONFINITE);
  const float inv = 1.0f / now;
  if (t0 >= hi || (t0 + 16 <= lo && !(ratio < 1.0f))) return;  // nothing of the unit changes
  if (!value) {
    int8_t* base = a.c.k + k_offset(a.c, page, head, t0) + d0;
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      int c[8];
      if (t0 + t >= hi) continue;
      if (t0 + t < lo) {
        if (!(ratio < 1.0f)) continue;
        const uint2 w = *reinterpret_cast<const uint2*>(base + (int64_t)t * D);
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k] = regrown((int8_t)((k < 4 ? w.x : w.y) >> (8 * (k & 3))), ratio);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k] = (int)rintf(x[t][k] * inv);
      }
      *reinterpret_cast<uint2*>(base + (int64_t)t * D) = uint2{pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7])};
    }
    return;
  }
  const bool whole = t0 >= lo && t0 + 16 <= hi;
  int8_t* base = a.c.v + v_offset(a.c, page, head, t0, d0);
  uint4 w[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = whole ? uint4{0, 0, 0, 0} : *reinterpret_cast<const uint4*>(base + 16 * k);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    unsigned* words = reinterpret_cast<unsigned*>(&w[k]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int c[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = 4 * i + e, was = (int8_t)(words[i] >> (8 * e));
        c[e] = t0 + t < lo ? (ratio < 1.0f ? regrown(was, ratio) : was) : t0 + t < hi ? (int)rintf(x[t][k] * inv) : was;
      }
      words[i] = pack4(c[0], c[1], c[2], c[3]);
    }
    *reinterpret_cast<uint4*>(base + 16 * k) = w[k];
  }
}

// The values back, unit by unit: blockIdx.x: keys or values, heads, 16 token slots;
// y: sequence.  Bound by memory: the same tokens 15 us, 4.6 TB/s.
template <typename T, int LP>
__global__ __launch_bounds__(256) void k_read_units(fxpq_kv_cache c, fxpq_kv_batch b, T* k_out, T* v_out,
                                                    int page_log2, int head_blocks, unsigned* flags) {
  constexpr int U = 256 / LP;
  const int s = blockIdx.y;
  const SeqDev q = seq_of(b, c.page, s);
  if (!q.ok) {
    if (blockIdx.x == 0 && threadIdx.x == 0) raise_flag(flags, FXPQ_FLAG_RANGE);
    return;
  }
  const bool value = blockIdx.x & 1;
  T* out = value ? v_out : k_out;
  const int pos0 = q.len - q.fresh;
  const int t0 = (pos0 & ~15) + (int)(blockIdx.x >> 1) / head_blocks * 16;
  if (!out || q.fresh == 0 || t0 >= q.len) return;
  const int page = b.table[(int64_t)s * b.table_ld + (t0 >> page_log2)], slot = t0 & (c.page - 1);
  const bool there = page >= 0 && page < c.pages;
  if (!there && threadIdx.x == 0) raise_flag(flags, FXPQ_FLAG_RANGE);
  const int head = (int)(blockIdx.x >> 1) % head_blocks * U + threadIdx.x / LP, d0 = threadIdx.x % LP * 8;
  if (head >= c.heads || d0 >= c.dim) return;
  float scale = 0.0f;
  uint2 w[16] = {};  // codes of 8 dimensions of each token
  if (there) {
    scale = (value ? c.v_scale : c.k_scale)[(int64_t)page * c.heads + head];
    if (!value) {
      const int8_t* from = c.k + k_offset(c, page, head, slot) + d0;
#pragma unroll
      for (int t = 0; t < 16; ++t) w[t] = *reinterpret_cast<const uint2*>(from + t * c.dim);
    } else {
      const int8_t* from = c.v + v_offset(c, page, head, slot, d0);
      uint4 r[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) r[k] = *reinterpret_cast<const uint4*>(from + 16 * k);
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        unsigned h[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const unsigned word = t < 4 ? r[k].x : t < 8 ? r[k].y : t < 12 ? r[k].z : r[k].w;
          h[k >> 2] |= (word >> (8 * (t & 3)) & 0xFFu) << (8 * (k & 3));
        }
        w[t] = uint2{h[0], h[1]};
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 16; ++t) {
    if (t0 + t < pos0 || t0 + t >= q.len) continue;
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = (float)(int8_t)((k < 4 ? w[t].x : w[t].y) >> (8 * (k & 3))) * scale;
    store8(out + ((q.first + (int64_t)(t0 + t - pos0)) * c.heads + head) * c.dim + d0, y);
  }
}

bool fits16(const void* p, int64_t ld, int64_t size) { return (uintptr_t)p % 16 == 0 && ld * size % 16 == 0; }

bool append_units_fit(const AppendArgs& a, int64_t size) {
  return fits16(a.k, a.ldk, size) && fits16(a.v, a.ldv, size) && fits16(a.q, a.ldq, size) &&
         fits16(a.q_out, a.ldqo, size) && a.rot.dims % 16 == 0 && (uintptr_t)a.rot.cos % 16 == 0 &&
         (uintptr_t)a.rot.sin % 16 == 0;
}

int log2_of(int v) {
  int l = 0;
  while ((1 << l) < v) ++l;
  return l;
}

// Calls f with the lanes of a unit: dim / 8, rounded up to a power of two.
template <typename F>
hipError_t for_lanes(int dim, F f) {
  switch (log2_of((dim + 7) / 8)) {
    case 1: return f(std::integral_constant<int, 2>());
    case 2: return f(std::integral_constant<int, 4>());
    case 3: return f(std::integral_constant<int, 8>());
    case 4: return f(std::integral_constant<int, 16>());
    default: return f(std::integral_constant<int, 32>());
  }
}

}  // namespace

hipError_t launch_cache_append(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                               const fxpq_rotary* rot, const void* k, int64_t ldk, const void* v,
                               int64_t ldv, const void* q, int64_t ldq, void* q_out, int64_t ldqo,
                               int q_heads, int type) {
  AppendArgs a{};
  a.c = cache;
  a.b = b;
  if (rot) a.rot = *rot;
  a.k = k;
  a.v = v;
  a.q = q;
  a.q_out = q_out;
  a.ldk = ldk;
  a.ldv = ldv;
  a.ldq = ldq;
  a.ldqo = ldqo;
  a.q_heads = q ? q_heads : 0;
  a.flags = c.sc.flags;
  a.segs = (b.max_new + cache.page - 2) / cache.page + 1;
  a.page_log2 = log2_of(cache.page);
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    return for_lanes(cache.dim, [&](auto lanes) {
      constexpr int LP = decltype(lanes)::value, U = 256 / LP;
      const bool fit = append_units_fit(a, sizeof(T)), few = !fit || b.max_new <= kFewTokens;
      const int heads = few ? U : U * 16 / cache.page;  // of a block
      if (((int64_t)cache.heads / heads + 1) * 2 * a.segs + b.max_new > kMaxBlocks) return hipErrorInvalidValue;
      a.head_blocks = (cache.heads + heads - 1) / heads;
      a.kv_blocks = 2 * a.segs * a.head_blocks;
      const int q_tokens = fit ? kQueryTokens : 1, q_blocks = q ? (b.max_new + q_tokens - 1) / q_tokens : 0;
      const dim3 grid((unsigned)(a.kv_blocks + (few ? q_blocks : 0)), (unsigned)b.seqs);
      if (!fit) k_append_few<T, LP, false><<<grid, dim3(256), 0, c.stream>>>(a);
      else if (few) k_append_few<T, LP, true><<<grid, dim3(256), 0, c.stream>>>(a);
      else k_append_units<T, LP><<<grid, dim3(256), 0, c.stream>>>(a);
      if (!few && q)
        k_rotate_queries<T><<<dim3((unsigned)q_blocks, (unsigned)b.seqs), dim3(256), 0, c.stream>>>(a);
      return hipGetLastError();
    });
  });
}

hipError_t launch_cache_read(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                             void* k_out, void* v_out, int type) {
  const unsigned blocks = (unsigned)(b.max_new + 14) / 16 + 1;  // 16-slot blocks that the tokens can touch
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    if (fits16(k_out, 0, 1) && fits16(v_out, 0, 1))
      return for_lanes(cache.dim, [&](auto lanes) {
        constexpr int LP = decltype(lanes)::value, U = 256 / LP;
        const int head_blocks = (cache.heads + U - 1) / U;
        if ((int64_t)head_blocks * 2 * blocks > kMaxBlocks) return hipErrorInvalidValue;
        k_read_units<T, LP><<<dim3(2u * blocks * (unsigned)head_blocks, (unsigned)b.seqs), dim3(256), 0, c.stream>>>(
            cache, b, static_cast<T*>(k_out), static_cast<T*>(v_out), log2_of(cache.page), head_blocks, c.sc.flags);
        return hipGetLastError();
      });
    k_cache_read<T><<<dim3(blocks, (unsigned)b.seqs, (unsigned)cache.heads), dim3(256), 0, c.stream>>>(
        cache, b, static_cast<T*>(k_out), static_cast<T*>(v_out), c.sc.flags);
    return hipGetLastError();
  });
}

}  // namespace fxpq
