// Appending to the paged 8-bit cache (with the position rotation) and reading
// its values back.
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

// blockIdx.x: page of the new tokens; y: sequence;
// z: head and whether keys or values.
template <typename T>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
  __shared__ float part[4];
  const int s = blockIdx.y, lane = threadIdx.x & 63;
  const SeqDev q = seq_of(a.b, a.c.page, s);
  const bool fits = q.ok && (a.rot.dims == 0 || q.len <= a.rot.positions);
  if (!fits) {
    if (blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int pos0 = q.len - q.fresh;
  const int D = a.c.dim, P = a.c.page;
  const int head = blockIdx.z >> 1;
  const bool value = blockIdx.z & 1;
  const int nth = pos0 / P + blockIdx.x;
  if (q.fresh == 0 || nth > (q.len - 1) / P) return;
  const int page = a.b.table[(int64_t)s * a.b.table_ld + nth];
  if (page < 0 || page >= a.c.pages) {
    if (threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int lo = max(pos0 - nth * P, 0), hi = min(q.len - nth * P, P);  // new slots
  const int64_t row0 = q.first + (int64_t)nth * P - pos0;               // row of slot 0
  const T* src = static_cast<const T*>(value ? a.v : a.k) + (int64_t)head * D;
  const int64_t ld = value ? a.ldv : a.ldk;
  bool bad = false;
  auto get = [&](int slot, int d) {
    const T* row = src + (row0 + slot) * ld;
    float x = value ? (float)row[d] : rotated(row, d, a.rot, nth * P + slot);
    if (!finite(x)) {
      bad = true;
      x = 0.0f;
    }
    return x;
  };
  float top = 0.0f;
  for (int i = threadIdx.x; i < (hi - lo) * D; i += 256) top = fmaxf(top, fabsf(get(lo + i / D, i % D)));
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) part[threadIdx.x >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  float* scale = (value ? a.c.v_scale : a.c.k_scale) + (int64_t)page * a.c.heads + head;
  float now = dfx_scale(fmaxf(top, kScaleFloor)), ratio = 1.0f;
  if (lo > 0) {
    const float old = *scale;
    now = fmaxf(now, old);
    ratio = old / now;
  }
  __syncthreads();  // every thread has the old scale
  if (threadIdx.x == 0) *scale = now;
  const float inv = 1.0f / now;  // exact: a power of two, unless the caller stored another old scale
  if (!value) {
    int8_t* base = a.c.k + k_offset(a.c, page, head, 0);
    if (ratio < 1.0f)
      for (int i = threadIdx.x; i < lo * D; i += 256) base[i] = (int8_t)regrown(base[i], ratio);
    for (int i = threadIdx.x; i < (hi - lo) * D; i += 256)
      base[lo * D + i] = (int8_t)rintf(get(lo + i / D, i % D) * inv);
  } else {
    // one thread per 16-token block and dimension: 16 bytes of V
    for (int i = threadIdx.x; i < P / 16 * D; i += 256) {
      const int t0 = i / D * 16, d = i % D;
      if (t0 >= hi || (t0 + 16 <= lo && ratio == 1.0f)) continue;
      int8_t* at = a.c.v + v_offset(a.c, page, head, t0, d);
      int8_t w[16];
      *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(at);
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        if (t0 + t < lo) w[t] = (int8_t)regrown(w[t], ratio);
        else if (t0 + t < hi) w[t] = (int8_t)rintf(get(t0 + t, d) * inv);
      }
      *reinterpret_cast<uint4*>(at) = *reinterpret_cast<const uint4*>(w);
    }
  }
  if (__ballot(bad) && lane == 0) raise_flag(a.flags, FXPQ_FLAG_NONFINITE);
}

// Rotated queries: one block per new token (x) of a sequence (y).
template <typename T>
__global__ __launch_bounds__(256) void k_rotate_queries(AppendArgs a) {
  const SeqDev q = seq_of(a.b, a.c.page, blockIdx.y);
  if (!q.ok || (a.rot.dims && q.len > a.rot.positions) || (int)blockIdx.x >= q.fresh) return;
  const int pos = q.len - q.fresh + blockIdx.x, D = a.c.dim, W = a.q_heads * D;
  const T* src = static_cast<const T*>(a.q) + (q.first + (int64_t)blockIdx.x) * a.ldq;
  T* dst = static_cast<T*>(a.q_out) + (q.first + (int64_t)blockIdx.x) * a.ldqo;
  const int half = a.rot.dims / 2;
  // a thread takes a pair whole: in place is fine
  const int pairs = a.q_heads * half;
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
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    k_cache_append<T><<<dim3((unsigned)a.segs, (unsigned)b.seqs, 2u * (unsigned)cache.heads), dim3(256), 0,
                        c.stream>>>(a);
    if (q)
      k_rotate_queries<T><<<dim3((unsigned)b.max_new, (unsigned)b.seqs), dim3(256), 0, c.stream>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_cache_read(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                             void* k_out, void* v_out, int type) {
  const unsigned blocks = (unsigned)(b.max_new + 14) / 16 + 1;
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    k_cache_read<T><<<dim3(blocks, (unsigned)b.seqs, (unsigned)cache.heads), dim3(256), 0, c.stream>>>(
        cache, b, static_cast<T*>(k_out), static_cast<T*>(v_out), c.sc.flags);
    return hipGetLastError();
  });
}

}  // namespace fxpq
