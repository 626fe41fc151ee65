// The paged 8-bit cache of latents: append with rotation, and reading it back.
//
// A token's latent c and its shared key r (rotated by the token's place) become int8
// codes with one scale each, by the rule and the very arithmetic of the token
// quantizer: what fxpq_latent_read hands over is an operand of the 8-bit product.
// The rotation is computed in fp64 (the products are exact there, one rounding to
// fp32 follows), so that a value next to the border of two codes has one answer.
//
// Bound by the bytes: 8 prompts of up to 2048 tokens with 32 heads' queries, f16: append 112
// MB in 27 us, 4.2 TB/s, and read of the new tokens 8 us; read of 16 contexts of up to 8192 as
// codes, scales and keys (82 MB) 18.5 us, 4.4 TB/s.  64 x 1 tokens: 4.0 and 2.8 us, mostly launch and the way from
// length to table to page.  A wave takes a token, since both maxima need all of its row;
// queries have blocks of their own beside them, so that one launch does both.
#include <type_traits>

#include "kv.hpp"
#include "values.hpp"

namespace fxpq {
namespace {

constexpr int kPairs = 4;  // rotated pairs of a lane

// Eight reals as 16- or 32-byte loads, or one by one.
template <typename T, bool VEC, int N>
__device__ inline void take(const T* p, float (&x)[N]) {
  constexpr int W = VEC ? (16 / (int)sizeof(T) < N ? 16 / (int)sizeof(T) : N) : 1;
#pragma unroll
  for (int i = 0; i < N; i += W) {
    float u[W];
    load_reals<T, W>(p + i, u);
#pragma unroll
    for (int j = 0; j < W; ++j) x[i + j] = u[j];
  }
}
template <typename T, bool VEC, int N>
__device__ inline void put(T* p, const float (&x)[N]) {
  constexpr int W = VEC ? (16 / (int)sizeof(T) < N ? 16 / (int)sizeof(T) : N) : 1;
#pragma unroll
  for (int i = 0; i < N; i += W) {
    float u[W];
#pragma unroll
    for (int j = 0; j < W; ++j) u[j] = x[i + j];
    store_reals<T, W>(p + i, u);
  }
}

// Pairs p0 .. p0 + 3 of a row of `dims` reals, rotated by place `pos`: (x1, x2) are
// elements (p, p + dims / 2), or (2 p, 2 p + 1) when interleaved.
template <typename T, bool VEC>
__device__ inline void rotated(const T* row, int p0, const fxpq_rotary& rot, int dims, int64_t pos, float (&y1)[kPairs],
                               float (&y2)[kPairs]) {
  float x1[kPairs], x2[kPairs];
  if (rot.interleaved) {
    float x[2 * kPairs];
    take<T, VEC>(row + 2 * p0, x);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      x1[i] = x[2 * i];
      x2[i] = x[2 * i + 1];
    }
  } else {
    take<T, VEC>(row + p0, x1);
    take<T, VEC>(row + p0 + dims / 2, x2);
  }
  if (!rot.dims) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      y1[i] = x1[i];
      y2[i] = x2[i];
    }
    return;
  }
  float c[kPairs], s[kPairs];
  take<float, VEC>(rot.cos + pos * (dims / 2) + p0, c);
  take<float, VEC>(rot.sin + pos * (dims / 2) + p0, s);
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const double a = x1[i], b = x2[i];
    y1[i] = (float)(a * c[i] - b * s[i]);
    y2[i] = (float)(b * c[i] + a * s[i]);
  }
}

__device__ inline unsigned wave_max(unsigned v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, d));
  return v;
}

// Non-finite values become 0 (true: there were any); the magnitudes' bits join `top`.
template <int N>
__device__ inline bool drop_bad(float (&x)[N], unsigned& top) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (!finite(x[i])) {
      x[i] = 0.0f;
      bad = true;
    }
    top = max(top, __builtin_bit_cast(unsigned, x[i]) & 0x7FFFFFFFu);
  }
  return bad;
}

struct Step {
  float scale, inv;
};
__device__ inline Step step_of(unsigned top, int rule) {
  const float a = fmaxf(__builtin_bit_cast(float, top), kScaleFloor);
  if (rule == FXPQ_SCALE_DFX) {
    const float s = dfx_scale(a);
    return Step{s, pow2_inverse(s)};
  }
  return Step{a / 127.0f, 127.0f / a};
}
__device__ inline unsigned codes4(const float* x, float inv) {
  return pack4((int)rintf(x[0] * inv), (int)rintf(x[1] * inv), (int)rintf(x[2] * inv), (int)rintf(x[3] * inv));
}

// blockIdx.x: first the keys' blocks, four waves of one token each, then the queries', one
// token each; y: sequence.  LB: latent dimensions of a lane.
template <typename T, int LB, bool VEC>
__global__ __launch_bounds__(256) void k_latent_append(LatentAppendArgs a, int key_blocks) {
  const SeqDev s = seq_of(a.b, a.c.page, blockIdx.y);
  if (!s.ok || (s.fresh > 0 && a.rot.dims && s.len > a.rot.positions)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int pos0 = s.len - s.fresh, R = a.c.rope;
  if ((int)blockIdx.x >= key_blocks) {
    const int t = (int)blockIdx.x - key_blocks, per = R / 2 / kPairs, work = a.heads * per;
    if (t >= s.fresh) return;
    const int64_t row = s.first + (int64_t)t;
    for (int i = threadIdx.x; i < work; i += 256) {
      const int head = i / per, p0 = i % per * kPairs;
      float y1[kPairs], y2[kPairs];
      rotated<T, VEC>(static_cast<const T*>(a.q) + row * a.ldq + head * a.hdq, p0, a.rot, R, pos0 + (int64_t)t, y1, y2);
      T* to = static_cast<T*>(a.q_out) + row * a.ldqo + head * a.hdqo;
      if (a.rot.interleaved) {
        float y[2 * kPairs];
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
          y[2 * k] = y1[k];
          y[2 * k + 1] = y2[k];
        }
        put<T, VEC>(to + 2 * p0, y);
      } else {
        put<T, VEC>(to + p0, y1);
        put<T, VEC>(to + p0 + R / 2, y2);
      }
    }
    return;
  }
  const int t = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= s.fresh) return;
  const int64_t row = s.first + (int64_t)t;
  const int pos = pos0 + t, page = a.b.table[(int64_t)blockIdx.y * a.b.table_ld + pos / a.c.page];
  if (page < 0 || page >= a.c.pages) {
    if (lane == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  float x[LB], y1[kPairs], y2[kPairs];
  take<T, VEC>(static_cast<const T*>(a.latent) + row * a.ldc + lane * LB, x);
  const int p0 = lane * kPairs;
  const bool turned = p0 < R / 2;
#pragma unroll
  for (int i = 0; i < kPairs; ++i) y1[i] = y2[i] = 0.0f;
  if (turned) rotated<T, VEC>(static_cast<const T*>(a.key) + row * a.ldr, p0, a.rot, R, pos, y1, y2);
  unsigned top = 0, key_top = 0;
  bool bad = drop_bad(x, top);
  bad |= drop_bad(y1, key_top);
  bad |= drop_bad(y2, key_top);
  const Step step = step_of(wave_max(top), a.rule), key_step = step_of(wave_max(key_top), a.rule);
  if (bad) raise_flag(a.flags, FXPQ_FLAG_NONFINITE);
  const int slot = pos & (a.c.page - 1);
  const int64_t at = (int64_t)page * a.c.page + slot;
  if (lane == 0) {
    a.c.scale[at] = step.scale;
    a.c.rope_scale[at] = key_step.scale;
  }
  int8_t* to = a.c.codes + latent_offset(a.c, page, slot);
#pragma unroll
  for (int i = 0; i < LB; i += 4) *reinterpret_cast<unsigned*>(to + lane * LB + i) = codes4(x + i, step.inv);
  if (!turned) return;
  to += a.c.latent;
  if (a.rot.interleaved) {
    float y[2 * kPairs];
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      y[2 * k] = y1[k];
      y[2 * k + 1] = y2[k];
    }
    *reinterpret_cast<unsigned*>(to + 2 * p0) = codes4(y, key_step.inv);
    *reinterpret_cast<unsigned*>(to + 2 * p0 + 4) = codes4(y + 4, key_step.inv);
  } else {
    *reinterpret_cast<unsigned*>(to + p0) = codes4(y1, key_step.inv);
    *reinterpret_cast<unsigned*>(to + p0 + R / 2) = codes4(y2, key_step.inv);
  }
}

constexpr int kReadTokens = 32;  // of a block

// blockIdx.x: 32 tokens; y: sequence.  A thread takes 16 codes at a time.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_latent_read(LatentReadArgs a) {
  const SeqDev s = seq_of(a.b, a.c.page, blockIdx.y);
  int64_t first = 0;
  int t0 = 0;
  bool ok = s.ok;
  if (ok && a.kv_start) {
    const int from = a.kv_start[blockIdx.y], to = a.kv_start[blockIdx.y + 1];
    ok = from >= 0 && to >= from && to - from == s.len && to <= a.kv_tokens;
    first = from;
  } else if (ok) {
    t0 = s.len - s.fresh;
    first = (int64_t)s.first - t0;
  }
  if (!ok) {
    if (blockIdx.x == 0 && threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  t0 += (int)blockIdx.x * kReadTokens;
  const int many = min(kReadTokens, s.len - t0);
  if (many <= 0) return;
  const int pieces = (a.c.latent + a.c.rope) / 16, latents = a.c.latent / 16;
  const int32_t* table = a.b.table + (int64_t)blockIdx.y * a.b.table_ld;
  for (int i = threadIdx.x; i < many * pieces; i += 256) {
    const int t = t0 + i / pieces, piece = i % pieces;
    const int page = table[t / a.c.page], slot = t & (a.c.page - 1);
    const bool there = page >= 0 && page < a.c.pages;
    uint4 w{0, 0, 0, 0};
    float scale = 0.0f;
    if (there) {
      const bool is_key = piece >= latents;
      w = *reinterpret_cast<const uint4*>(a.c.codes + latent_offset(a.c, page, slot) + piece * 16);
      scale = (is_key ? a.c.rope_scale : a.c.scale)[(int64_t)page * a.c.page + slot];
    } else if (piece == 0) {
      raise_flag(a.flags, FXPQ_FLAG_RANGE);
    }
    const int64_t row = first + t;
    if (piece == 0 && a.scale) a.scale[row] = scale;
    if (piece < latents && a.codes) *reinterpret_cast<uint4*>(a.codes + row * a.ld_codes + piece * 16) = w;
    T* to = piece < latents ? static_cast<T*>(a.latent) : static_cast<T*>(a.key);
    if (!to) continue;
    to += piece < latents ? row * a.ld_latent + piece * 16 : row * a.ld_key + (piece - latents) * 16;
    const unsigned* words = reinterpret_cast<const unsigned*>(&w);
    float y[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) y[k] = (float)(int8_t)(words[k >> 2] >> (8 * (k & 3))) * scale;
    put<T, VEC>(to, y);
  }
}

bool fits16(const void* p, int64_t a, int64_t b, int64_t size) {
  return (uintptr_t)p % 16 == 0 && a * size % 16 == 0 && b * size % 16 == 0;
}

}  // namespace

hipError_t launch_latent_append(const Ctx& c, LatentAppendArgs a, int type) {
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    const int64_t size = sizeof(T);
    const bool vec = fits16(a.latent, a.ldc, 0, size) && fits16(a.key, a.ldr, 0, size) &&
                     (!a.heads || (fits16(a.q, a.ldq, a.hdq, size) && fits16(a.q_out, a.ldqo, a.hdqo, size))) &&
                     fits16(a.rot.cos, 0, 0, 4) && fits16(a.rot.sin, 0, 0, 4);
    const int key_blocks = (a.b.max_new + 3) / 4, q_blocks = a.heads ? a.b.max_new : 0;
    if ((int64_t)key_blocks + q_blocks > kMaxBlocks) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(key_blocks + q_blocks), (unsigned)a.b.seqs);
    auto run = [&](auto lb, auto v) {
      k_latent_append<T, decltype(lb)::value, decltype(v)::value><<<grid, dim3(256), 0, c.stream>>>(a, key_blocks);
      return hipGetLastError();
    };
    using std::integral_constant;
    if (a.c.latent == 512)
      return vec ? run(integral_constant<int, 8>(), std::true_type()) : run(integral_constant<int, 8>(), std::false_type());
    return vec ? run(integral_constant<int, 4>(), std::true_type()) : run(integral_constant<int, 4>(), std::false_type());
  });
}

hipError_t launch_latent_read(const Ctx& c, LatentReadArgs a, int type) {
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    const bool vec = fits16(a.latent, a.ld_latent, 0, sizeof(T)) && fits16(a.key, a.ld_key, 0, sizeof(T));
    const int most = a.kv_start ? a.b.max_len : a.b.max_new;
    const dim3 grid((unsigned)((most + kReadTokens - 1) / kReadTokens), (unsigned)a.b.seqs);
    if (most == 0) return hipSuccess;
    if ((int64_t)grid.x > kMaxBlocks) return hipErrorInvalidValue;
    if (vec) k_latent_read<T, true><<<grid, dim3(256), 0, c.stream>>>(a);
    else k_latent_read<T, false><<<grid, dim3(256), 0, c.stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace fxpq
