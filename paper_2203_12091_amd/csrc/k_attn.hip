// Attention over the paged 8-bit cache.
//
// S = K Q^T runs on the int8 matrix cores: a query row is written as a sum of
// int8 digit planes q = s (d0 + d1 256 + ...), s a power of two, so K's codes
// go into the products as they lie in memory and every dot product is an exact
// integer.  O^T = V^T P^T runs on the bf16 matrix cores: V's codes are exact in
// bf16, the page's scale is folded into P before it is rounded.
//
// A wave takes 64 tokens of the cache at a time as four groups of 16 (a group
// never crosses a page).  Tokens are dealt to the four 16-row tiles of S so that
// the lane that holds S for a group of 16 tokens and one query column needs V of
// exactly those 16 tokens: row i of tile t is token 16 (i / 4) + 4 t + i % 4.
// P therefore goes from the first product's result registers into the second
// product's operand without leaving the lane.
#include "kv.hpp"
#include "values.hpp"

namespace fxpq {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

struct AttnArgs {
  fxpq_kv_cache c;
  fxpq_kv_batch b;
  const void* q;
  void* out;
  int64_t ldq, ldo;
  int q_heads, group;   // group: query heads of one key / value head
  int causal;
  float scale;          // softmax_scale * log2(e)
  int col_tiles;        // blocks along a sequence's query columns
  int splits;           // blocks along the cache
  int split_chunks;     // 64-token chunks of one split
  int vec;              // q and out rows are 16-byte aligned
  float* part_o;        // [splits][tokens][q_heads][dim]
  float* part_ml;       // [splits][tokens][q_heads][2]: running maximum and sum
  unsigned* flags;
};

constexpr float kNoMax = -1e30f;  // running maximum before any token

// Chunks that the query columns of one tile see: up to the last column's limit.
__device__ inline int tile_chunks(const AttnArgs& a, const SeqDev& s, int col0, int cols) {
  const int last = min(col0 + cols, s.fresh * a.group) - 1;
  if (last < col0) return 0;
  const int limit = a.causal ? s.len - s.fresh + last / a.group : s.len - 1;
  return (limit + 64) >> 6;
}

// Four code bytes as two pairs of bf16 (exact: |code| <= 128).
__device__ inline void codes_to_bf16(int w, int& lo, int& hi) {
  const float a = (float)(int8_t)w, b = (float)(int8_t)(w >> 8), c = (float)(int8_t)(w >> 16),
              d = (float)(int8_t)(w >> 24);
  lo = (int)__builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, a), 0x07060302u);
  hi = (int)__builtin_amdgcn_perm(__builtin_bit_cast(unsigned, d), __builtin_bit_cast(unsigned, c), 0x07060302u);
}

// DB: 64-dimension blocks of a head; NC: 16-column query tiles of a wave; SPLIT_Q:
// digit planes of q; SPLIT_P: bf16 terms of P; TOK: the four waves share the
// columns and deal the chunks among them (few columns), else each has its own.
template <typename T, int DB, int NC, int SPLIT_Q, int SPLIT_P, bool TOK>
__global__ __launch_bounds__(256) void k_cache_attention(AttnArgs a) {
  constexpr int DT = DB * 4;  // 16-dimension tiles of O
  extern __shared__ float smem[];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.y, D = a.c.dim, P = a.c.page;
  const SeqDev s = seq_of(a.b, P, blockIdx.z);
  if (!s.ok) {
    if (blockIdx.x == 0 && head == 0 && threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int tile = blockIdx.x % a.col_tiles, split = blockIdx.x / a.col_tiles;
  constexpr int kCols = NC * 16 * (TOK ? 1 : 4);
  const int tile0 = tile * kCols;
  if (tile0 >= s.fresh * a.group) return;
  const int total = tile_chunks(a, s, tile0, kCols);
  const int begin = split * a.split_chunks, end = min(begin + a.split_chunks, total);
  if (a.splits > 1 && begin >= end) return;
  const int col0 = tile0 + (TOK ? 0 : wave * NC * 16);
  const int pos0 = s.len - s.fresh;

  // digit planes of this lane's query columns: dimensions 64 b + 16 g + 0..15
  v4i qd[NC][DB][SPLIT_Q];
  float qscale[NC];
  int limit[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = col0 + c * 16 + n, i = col / a.group;
    const bool real = i < s.fresh;
    limit[c] = a.causal ? pos0 + i : s.len - 1;
    const T* row = static_cast<const T*>(a.q) + (s.first + (int64_t)(real ? i : 0)) * a.ldq +
                   (int64_t)(head * a.group + col % a.group) * D;
    float x[DB][16];
    float top = 0.0f;
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      const int d = b * 64 + g * 16;
      if (real && d < D) {
        if (a.vec) {
          constexpr int W = 16 / sizeof(T);
#pragma unroll
          for (int k = 0; k < 16; k += W) {
            float u[W];
            load_reals<T, W>(row + d + k, u);
#pragma unroll
            for (int j = 0; j < W; ++j) x[b][k + j] = u[j];
          }
        } else {
#pragma unroll
          for (int k = 0; k < 16; ++k) x[b][k] = (float)row[d + k];
        }
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) x[b][k] = 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 16; ++k)
        top = __builtin_bit_cast(float, max(__builtin_bit_cast(int, top), __builtin_bit_cast(int, x[b][k]) & 0x7FFFFFFF));
    }
    top = __builtin_bit_cast(float, max(__builtin_bit_cast(int, top), __shfl_xor(__builtin_bit_cast(int, top), 16)));
    top = __builtin_bit_cast(float, max(__builtin_bit_cast(int, top), __shfl_xor(__builtin_bit_cast(int, top), 32)));
    const float step = dfx_scale(fmaxf(finite(top) ? top : 1.0f, kScaleFloor));
    constexpr float kUp = SPLIT_Q == 1 ? 1.0f : SPLIT_Q == 2 ? 256.0f : SPLIT_Q == 3 ? 65536.0f : 16777216.0f;
    // the largest sum of balanced digits: 127 in every place
    constexpr float kMost = SPLIT_Q == 1 ? 127.0f : SPLIT_Q == 2 ? 32639.0f : SPLIT_Q == 3 ? 8355711.0f : 2139062016.0f;
    const float inv = pow2_inverse(step) * kUp;
    qscale[c] = finite(top) ? step * (1.0f / kUp) * a.scale : __builtin_nanf("");
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        int v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float r = rintf(x[b][4 * w + k] * inv);
          v[k] = finite(top) ? (int)fminf(fmaxf(r, -kMost), kMost) : 0;
        }
#pragma unroll
        for (int p = 0; p < SPLIT_Q; ++p) {
          int low[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            low[k] = (int8_t)v[k];
            v[k] = (v[k] - low[k]) >> 8;
          }
          qd[c][b][p][w] = (int)pack4(low[0], low[1], low[2], low[3]);
        }
      }
  }

  float m[NC], l[NC];
  v4f o[NC][DT];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = kNoMax;
    l[c] = 0.0f;
#pragma unroll
    for (int j = 0; j < DT; ++j) o[c][j] = v4f{0, 0, 0, 0};
  }
  const int first_limit = a.causal ? pos0 + col0 / a.group : s.len - 1;
  const int32_t* table = a.b.table + (int64_t)blockIdx.z * a.b.table_ld;
  const int last_nth = (s.len - 1) / P;
  const int stride = TOK ? 4 : 1;

  // page of a group of 16 tokens, 0 where it has none (then nothing is seen of it)
  auto page_of = [&](int t) {
    const int nth = t / P;
    return nth <= last_nth ? table[nth] : -1;
  };
  const int kg = n >> 2;  // group of the K rows that this lane loads
  v4i kr[4][DB], vr[DT];
  auto load_k = [&](int chunk) {
    const int t0 = chunk * 64 + kg * 16;
    int page = page_of(t0);
    page = page < 0 || page >= a.c.pages ? 0 : page;
    const int8_t* base = a.c.k + k_offset(a.c, page, head, t0 % P + (n & 3));
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const int d = min(b * 64 + g * 16, D - 16);  // past the head: any bytes, q's digits are 0
        kr[t][b] = *reinterpret_cast<const v4i*>(base + t * 4 * D + d);
      }
  };
  int chunk = begin + (TOK ? wave : 0);
  if (chunk < end) load_k(chunk);
  for (; chunk < end; chunk += stride) {
    const int t0 = chunk * 64 + g * 16;  // this lane's 16 tokens
    const int named = page_of(t0);
    const bool there = named >= 0 && named < a.c.pages;
    if (!there && t0 < s.len) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    const int page = there ? named : 0;
    const int64_t at = (int64_t)page * a.c.heads + head;
    const float ks = there ? a.c.k_scale[at] : 0.0f, vs = there ? a.c.v_scale[at] : 0.0f;
    const int8_t* vbase = a.c.v + v_offset(a.c, page, head, t0 % P, 0);
#pragma unroll
    for (int j = 0; j < DT; ++j)
      vr[j] = *reinterpret_cast<const v4i*>(vbase + min(j * 16, D - 16) * 16 + n * 16);

    float x[NC][16];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float f = ks * qscale[c];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        v4i acc[SPLIT_Q];
#pragma unroll
        for (int p = 0; p < SPLIT_Q; ++p) {
          acc[p] = v4i{0, 0, 0, 0};
#pragma unroll
          for (int b = 0; b < DB; ++b)
            acc[p] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kr[t][b], qd[c][b][p], acc[p], 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v;  // |acc| < 2^22: two planes combine exactly in an int
          if constexpr (SPLIT_Q == 1) v = (float)acc[0][r];
          else if constexpr (SPLIT_Q == 2) v = (float)(acc[1][r] * 256 + acc[0][r]);
          else if constexpr (SPLIT_Q == 3) v = fmaf((float)(acc[2][r] * 256 + acc[1][r]), 256.0f, (float)acc[0][r]);
          else v = fmaf((float)(acc[3][r] * 256 + acc[2][r]), 65536.0f, (float)(acc[1][r] * 256 + acc[0][r]));
          x[c][t * 4 + r] = v * f;
        }
      }
    }
    if (chunk + stride < end) load_k(chunk + stride);
    const bool edge = chunk * 64 + 63 > first_limit || __any(!there);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (edge) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (t0 + i > limit[c] || !there) x[c][i] = -INFINITY;
      }
      float top = x[c][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, x[c][i]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__any(top > m[c])) {
        const float now = fmaxf(m[c], top), down = __builtin_amdgcn_exp2f(m[c] - now);
        m[c] = now;
        l[c] *= down;
#pragma unroll
        for (int j = 0; j < DT; ++j) o[c][j] *= down;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[c][i] = __builtin_amdgcn_exp2f(x[c][i] - m[c]);
        l[c] += x[c][i];
        x[c][i] *= vs;
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      v8bf p[NC][SPLIT_P];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float rest = x[c][u * 8 + i];
#pragma unroll
          for (int k = 0; k < SPLIT_P; ++k) {
            p[c][k][i] = (__bf16)rest;
            rest -= (float)p[c][k][i];
          }
        }
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        v4i w;
        int lo, hi;
        codes_to_bf16(vr[j][2 * u], lo, hi);
        w[0] = lo;
        w[1] = hi;
        codes_to_bf16(vr[j][2 * u + 1], lo, hi);
        w[2] = lo;
        w[3] = hi;
        const v8bf vv = __builtin_bit_cast(v8bf, w);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int k = 0; k < SPLIT_P; ++k)
            o[c][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, p[c][k], o[c][j], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 16);
    l[c] += __shfl_xor(l[c], 32);
  }

  // lane: column n of tile c, dimensions 16 j + 4 g + 0..3
  auto emit = [&](int col, int d, float mx, float sum, const float(&v)[4]) {
    const int i = col / a.group;
    if (i >= s.fresh || d >= D) return;
    const int64_t row = s.first + (int64_t)i;
    const int hq = head * a.group + col % a.group;
    if (a.splits > 1) {
      const int64_t r = ((int64_t)split * a.b.tokens + row) * a.q_heads + hq;
      *reinterpret_cast<float4*>(a.part_o + r * D + d) = float4{v[0], v[1], v[2], v[3]};
      if (d == 0) {
        a.part_ml[2 * r] = mx;
        a.part_ml[2 * r + 1] = sum;
      }
      return;
    }
    const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
    T* to = static_cast<T*>(a.out) + row * a.ldo + (int64_t)hq * D + d;
    const float y[4] = {v[0] * f, v[1] * f, v[2] * f, v[3] * f};
    if (a.vec) {
      store_reals<T, 4>(to, y);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) to[k] = (T)y[k];
    }
  };
  if constexpr (!TOK) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        const float v[4] = {o[c][j][0], o[c][j][1], o[c][j][2], o[c][j][3]};
        emit(col0 + c * 16 + n, j * 16 + g * 4, m[c], l[c], v);
      }
  } else {
    // join the four waves: each one's statistics and sums through LDS
    constexpr int kRow = DT * 16 + 4;  // floats of a column (the pad spreads the banks)
    float* ml = smem;                  // [4][kCols][2]
    float* os = smem + 4 * kCols * 2;  // [4][kCols][kRow]
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int at = wave * kCols + c * 16 + n;
      if (g == 0) {
        ml[2 * at] = m[c];
        ml[2 * at + 1] = l[c];
      }
#pragma unroll
      for (int j = 0; j < DT; ++j) *reinterpret_cast<v4f*>(os + at * kRow + j * 16 + g * 4) = o[c][j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kCols * DT * 4; i += 256) {
      const int col = i / (DT * 4), d = i % (DT * 4) * 4;
      float mx = kNoMax, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) mx = fmaxf(mx, ml[2 * (w * kCols + col)]);
      float v[4] = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[2 * (w * kCols + col)] - mx);
        sum += f * ml[2 * (w * kCols + col) + 1];
        const v4f ow = *reinterpret_cast<const v4f*>(os + (w * kCols + col) * kRow + d);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += f * ow[k];
      }
      emit(tile0 + col, d, mx, sum, v);
    }
  }
}

// Joins the splits of each query row: one block per token and query head.
template <typename T>
__global__ __launch_bounds__(64) void k_attention_join(AttnArgs a, int kcols) {
  const SeqDev s = seq_of(a.b, a.c.page, blockIdx.z);
  const int i = blockIdx.x, hq = blockIdx.y;
  if (!s.ok || i >= s.fresh) return;
  const int col = i * a.group + hq % a.group;
  const int total = tile_chunks(a, s, col / kcols * kcols, kcols);
  const int used = (total + a.split_chunks - 1) / a.split_chunks;
  const int64_t row = s.first + (int64_t)i, stride = (int64_t)a.b.tokens * a.q_heads;
  const int64_t r = row * a.q_heads + hq;
  float mx = kNoMax, sum = 0.0f;
  for (int p = 0; p < used; ++p) mx = fmaxf(mx, a.part_ml[2 * (p * stride + r)]);
  for (int p = 0; p < used; ++p)
    sum += __builtin_amdgcn_exp2f(a.part_ml[2 * (p * stride + r)] - mx) * a.part_ml[2 * (p * stride + r) + 1];
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  T* out = static_cast<T*>(a.out) + row * a.ldo + (int64_t)hq * a.c.dim;
  for (int d = threadIdx.x; d < a.c.dim; d += 64) {
    float v = 0.0f;
    for (int p = 0; p < used; ++p)
      v += __builtin_amdgcn_exp2f(a.part_ml[2 * (p * stride + r)] - mx) * a.part_o[(p * stride + r) * a.c.dim + d];
    out[d] = (T)(v * f);
  }
}

struct AttnPlan {
  bool tok;     // few columns: the waves of a block share them
  int nc;       // 16-column tiles of a wave
  int col_tiles, splits, split_chunks;
  int64_t part, bytes;
};

AttnPlan plan_attention(const Ctx& c, const fxpq_kv_cache& k, const fxpq_kv_batch& b, int q_heads) {
  AttnPlan p{};
  const int64_t cols = (int64_t)b.max_new * (q_heads / k.heads);
  p.tok = cols <= 16;
  p.nc = p.tok || k.dim > 128 ? 1 : 2;
  const int64_t tile = (int64_t)p.nc * 16 * (p.tok ? 1 : 4);
  p.col_tiles = (int)((cols + tile - 1) / tile);
  const int64_t blocks = (int64_t)p.col_tiles * b.seqs * k.heads;
  const int64_t chunks = (b.max_len + 63) / 64;
  const int64_t want = (4 * (int64_t)c.cus + blocks - 1) / blocks;
  int64_t per = (chunks + want - 1) / want;
  if (per < 4) per = 4;
  p.split_chunks = (int)per;
  p.splits = (int)((chunks + per - 1) / per);
  if (p.splits > 1) {
    p.part = (int64_t)p.splits * b.tokens * q_heads;
    p.bytes = p.part * (k.dim + 2) * 4;
  } else {
    p.splits = 1;
  }
  return p;
}

template <typename T, int DB, int NC, bool TOK>
hipError_t run_attention(const Ctx& c, const AttnArgs& a) {
  // Digits of q and bf16 terms of P by the type that goes in and out: what they
  // drop stays below that type's own rounding.
  constexpr int SQ = sizeof(T) == 4 ? 4 : 3;
  constexpr int SP = sizeof(T) == 4 ? 3 : __is_same(T, __bf16) ? 1 : 2;
  constexpr int bytes = TOK ? 4 * NC * 16 * (2 + DB * 64 + 4) * 4 : 0;
  auto* f = k_cache_attention<T, DB, NC, SQ, SP, TOK>;
  if (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(f),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  f<<<dim3((unsigned)(a.col_tiles * a.splits), (unsigned)a.c.heads, (unsigned)a.b.seqs), dim3(256), bytes,
      c.stream>>>(a);
  if (a.splits > 1)
    k_attention_join<T><<<dim3((unsigned)a.b.max_new, (unsigned)a.q_heads, (unsigned)a.b.seqs), dim3(64), 0,
                          c.stream>>>(a, NC * 16 * (TOK ? 1 : 4));
  return hipGetLastError();
}

template <typename T, int DB>
hipError_t run_dim(const Ctx& c, const AttnArgs& a, const AttnPlan& p) {
  if (p.tok) return run_attention<T, DB, 1, true>(c, a);
  if constexpr (DB <= 2) return run_attention<T, DB, 2, false>(c, a);
  else return run_attention<T, DB, 1, false>(c, a);
}

}  // namespace

int64_t cache_attention_workspace(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                                  int q_heads) {
  return plan_attention(c, cache, b, q_heads).bytes;
}

hipError_t launch_cache_attention(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                                  const void* q, int64_t ldq, int q_heads, float softmax_scale,
                                  int causal, void* out, int64_t ldo, int type, void* ws) {
  const AttnPlan p = plan_attention(c, cache, b, q_heads);
  AttnArgs a{};
  a.c = cache;
  a.b = b;
  a.q = q;
  a.out = out;
  a.ldq = ldq;
  a.ldo = ldo;
  a.q_heads = q_heads;
  a.group = q_heads / cache.heads;
  a.causal = causal ? 1 : 0;
  a.scale = softmax_scale * 1.44269504088896340736f;
  a.col_tiles = p.col_tiles;
  a.splits = p.splits;
  a.split_chunks = p.split_chunks;
  const int64_t size = real_bytes(type);
  a.vec = (uintptr_t)q % 16 == 0 && (uintptr_t)out % 16 == 0 && ldq * size % 16 == 0 && ldo * size % 16 == 0;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = a.part_o ? a.part_o + p.part * cache.dim : nullptr;
  a.flags = c.sc.flags;
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    switch ((cache.dim + 63) / 64) {
      case 1: return run_dim<T, 1>(c, a, p);
      case 2: return run_dim<T, 2>(c, a, p);
      case 3: return run_dim<T, 3>(c, a, p);
      default: return run_dim<T, 4>(c, a, p);
    }
  });
}

}  // namespace fxpq
