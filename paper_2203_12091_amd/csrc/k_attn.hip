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
  int page_log2;
  int vec;              // q and out rows are 16-byte aligned
  float* part_o;        // [splits][tokens][q_heads][dim]
  float* part_ml;       // [splits][tokens][q_heads][2]: running maximum and sum
  unsigned* flags;
};

constexpr float kNoMax = -3.40282347e38f;  // running maximum before any token: below every finite logit
// The reference that logits are taken from is a running maximum that follows only
// when a logit passes it by more than this (base 2): weights reach 2^8 then, which
// costs no precision, and most chunks need neither a maximum over the lanes nor a
// rescaling of O.
constexpr float kSlack = 8.0f;

// A logit, rounded by itself: a multiply-add with the running maximum would leave
// the product's rounding error, which exceeds any slack where logits pass 2^31.
__device__ inline float scaled(float x, float f) {
#pragma clang fp contract(off)
  return x * f;
}
constexpr float kFar = 0x1p24f;  // references up to this leave an error below 1

// The maximum over the four 16-lane groups of a wave, lane by lane: the swaps leave
// rows (0, 0, 2, 2) and (1, 1, 3, 3), then halves (low, low) and (high, high).
// Written out, with the wait state the swap needs after a write of its operand: this
// compiler's builtins return their first result twice.
__device__ inline float over_groups(float x) {
  float y = x;
  asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(x), "+v"(y));
  x = y = fmaxf(x, y);
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));
  return fmaxf(x, y);
}

// What a block works on: part (query tile and split) of a sequence and head.
// Blocks are dealt to the 8 XCDs round-robin by id, so the heads, which have equal
// work, are the fastest index; where they are 8, a head's keys come through one
// XCD's L2.  Query tiles of a sequence run together, for the same reason (4 x 1024
// new tokens over 4000: 237 us, with the sequences in turn 279).  Splits are dealt
// across the sequences, each sequence's to another XCD: a late split is one that
// only long sequences have (64 sequences of up to 8192: 118.4 us with the splits next
// to each other, 117.7 so).
struct BlockAt {
  int head, seq, part;
};
template <bool SPREAD>
__device__ inline BlockAt block_at(const AttnArgs& a) {
  const unsigned i = blockIdx.x, rest = i / (unsigned)a.c.heads, seqs = (unsigned)a.b.seqs;
  if constexpr (SPREAD) {
    const unsigned part = rest / seqs;
    return BlockAt{(int)(i % (unsigned)a.c.heads), (int)((rest + part) % seqs), (int)part};
  }
  const unsigned parts = (unsigned)(a.col_tiles * a.splits);
  return BlockAt{(int)(i % (unsigned)a.c.heads), (int)(rest / parts), (int)(rest % parts)};
}
inline dim3 attention_grid(const AttnArgs& a) {
  return dim3((unsigned)a.c.heads * (unsigned)a.b.seqs * (unsigned)(a.col_tiles * a.splits));
}

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

// Four dimensions of one query column: the result, or its share where the cache
// is split.
template <typename T>
__device__ inline void emit(const AttnArgs& a, const SeqDev& s, int head, int split, int col, int d, float mx,
                            float sum, const float (&v)[4]) {
  const int i = col / a.group;
  if (i >= s.fresh || d >= a.c.dim) return;
  const int64_t row = s.first + (int64_t)i;
  const int hq = head * a.group + col % a.group;
  if (a.splits > 1) {
    const int64_t r = ((int64_t)split * a.b.tokens + row) * a.q_heads + hq;
    *reinterpret_cast<float4*>(a.part_o + r * a.c.dim + d) = float4{v[0], v[1], v[2], v[3]};
    if (d == 0) {
      a.part_ml[2 * r] = mx;
      a.part_ml[2 * r + 1] = sum;
    }
    return;
  }
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  T* to = static_cast<T*>(a.out) + row * a.ldo + (int64_t)hq * a.c.dim + d;
  const float y[4] = {v[0] * f, v[1] * f, v[2] * f, v[3] * f};
  if (a.vec) {
    store_reals<T, 4>(to, y);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) to[k] = (T)y[k];
  }
}

// DB: 64-dimension blocks of a head; NC: 16-column query tiles of a wave; SPLIT_Q:
// digit planes of q; SPLIT_P: bf16 terms of P; TOK: the four waves share the
// columns and deal the chunks among them (few columns), else each has its own (many
// columns of more than 128 dimensions).  Few columns are bound by memory: one token of
// 64 sequences of up to 8192, 8 heads of 128, 118 us and 4.7 TB/s in bf16, 136 and 4.0
// in fp32 (287 registers, one wave a SIMD); of 256 dimensions 227 and 4.8.  Many columns
// of 256 dimensions, 4 x 1024 new tokens over up to 4000: 711 us, one wave a SIMD and
// every wave converting all codes.
template <typename T, int DB, int NC, int SPLIT_Q, int SPLIT_P, bool TOK>
__global__ __launch_bounds__(256) void k_cache_attention(AttnArgs a) {
  static_assert(SPLIT_Q == 3 || SPLIT_Q == 4, "three digit planes (16-bit types) or four");
  constexpr int DT = DB * 4;  // 16-dimension tiles of O
  extern __shared__ float smem[];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int D = a.c.dim, P = a.c.page;
  const BlockAt at = block_at<TOK>(a);
  const int head = at.head;
  const SeqDev s = seq_of(a.b, P, at.seq);
  if (!s.ok) {
    if (at.part == 0 && head == 0 && threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int tile = at.part % a.col_tiles, split = at.part / a.col_tiles;
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
    constexpr float kUp = SPLIT_Q == 3 ? 65536.0f : 16777216.0f;
    // the largest sum of balanced digits: 127 in every place
    constexpr float kMost = SPLIT_Q == 3 ? 8355711.0f : 2139062016.0f;
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
  const int32_t* table = a.b.table + (int64_t)at.seq * a.b.table_ld;
  const int last_nth = (s.len - 1) >> a.page_log2;
  const int stride = TOK ? 4 : 1;

  // page of a token's group of 16; past the sequence's end -1 (nothing is seen of it)
  auto page_of = [&](int t) {
    const int nth = t >> a.page_log2;
    return nth <= last_nth ? table[nth] : -1;
  };
  // Page numbers are looked up two of this wave's chunks ahead, keys and scales
  // loaded one ahead, values at the chunk's start: no latency is waited for twice.
  const int kg = n >> 2;  // group of the K rows that this lane loads
  v4i kr[4][DB], vr[DT];
  int k_page, s_page;  // of the chunk to load next: of the K rows, of this lane's 16 tokens
  int next_page = 0;
  bool next_there = false;
  float next_ks = 0.0f, next_vs = 0.0f;
  auto lookup = [&](int chunk) {
    k_page = page_of(chunk * 64 + kg * 16);
    s_page = page_of(chunk * 64 + g * 16);
  };
  auto load = [&](int chunk) {
    const int page = k_page < 0 || k_page >= a.c.pages ? 0 : k_page;
    const int8_t* base = a.c.k + k_offset(a.c, page, head, ((chunk * 64 + kg * 16) & (P - 1)) + (n & 3));
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const int d = min(b * 64 + g * 16, D - 16);  // past the head: any bytes, q's digits are 0
        kr[t][b] = *reinterpret_cast<const v4i*>(base + t * 4 * D + d);
      }
    next_there = s_page >= 0 && s_page < a.c.pages;
    if (!next_there && chunk * 64 + g * 16 < s.len) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    next_page = next_there ? s_page : 0;
    const int64_t sc = (int64_t)next_page * a.c.heads + head;
    next_ks = a.c.k_scale[sc];
    next_vs = a.c.v_scale[sc];
  };
  int chunk = begin + (TOK ? wave : 0);
  if (chunk < end) {
    lookup(chunk);
    load(chunk);
    lookup(chunk + stride);
  }
  for (; chunk < end; chunk += stride) {
    const int t0 = chunk * 64 + g * 16;  // this lane's 16 tokens
    const bool there = next_there;
    const float ks = there ? next_ks : 0.0f, vs = there ? next_vs : 0.0f;
    const int8_t* vbase = a.c.v + v_offset(a.c, next_page, head, (t0 & (P - 1)), 0);
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
          if constexpr (SPLIT_Q == 3) v = fmaf((float)(acc[2][r] * 256 + acc[1][r]), 256.0f, (float)acc[0][r]);
          else v = fmaf((float)(acc[3][r] * 256 + acc[2][r]), 65536.0f, (float)(acc[1][r] * 256 + acc[0][r]));
          x[c][t * 4 + r] = scaled(v, f);
        }
      }
    }
    if (chunk + stride < end) {
      load(chunk + stride);
      lookup(chunk + 2 * stride);
    }
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
      if (__any(top > m[c] + kSlack)) {
        const float now = fmaxf(m[c], over_groups(top)), down = __builtin_amdgcn_exp2f(m[c] - now);
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
  if constexpr (!TOK) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        const float v[4] = {o[c][j][0], o[c][j][1], o[c][j][2], o[c][j][3]};
        emit<T>(a, s, head, split, col0 + c * 16 + n, j * 16 + g * 4, m[c], l[c], v);
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
      emit<T>(a, s, head, split, tile0 + col, d, mx, sum, v);
    }
  }
}

// ---- many query columns ----------------------------------------------------------
// A block of four or eight waves, 16 NC columns each, goes over the cache together: every
// thread loads its share of the next 64 tokens' codes while the waves work on the
// current ones, converts it and leaves it in LDS in the operand types, K as T's own
// matrix-core type (bf16 for f32), V as bf16 (both hold a code exactly).  q goes in
// as QT terms of that type (exact for f16 and bf16), P as PT bf16 terms.
// 4 x 1024 new tokens over up to 4000, 32 query heads of 8 of 128: 237 us in f16, 236
// in bf16, 379 in fp32.  Bound by the softmax's vector arithmetic, about twelve
// operations an element, beside the matrix products, at two waves a SIMD.
template <typename T>
struct OperandK {
  typedef __bf16 type;
};
template <>
struct OperandK<_Float16> {
  typedef _Float16 type;
};

__device__ inline v4f mfma_k(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
__device__ inline v4f mfma_k(v8h a, v8h b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Four code bytes as two pairs of f16: byte u = code + 128 in the low bits of
// 1024.0 is 1024 + u, and 1024 + u - 1152 is the code, exactly.
__device__ inline void codes_to_f16(int w, int& lo, int& hi) {
  const unsigned u = (unsigned)w ^ 0x80808080u;
  const v2h off = {(_Float16)1152.0f, (_Float16)1152.0f};
  const v2h a = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u));
  const v2h b = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u));
  lo = __builtin_bit_cast(int, a - off);
  hi = __builtin_bit_cast(int, b - off);
}
template <typename KT>
__device__ inline void codes_to(v4i w, v4i& first, v4i& second) {
  int lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (__is_same(KT, _Float16)) codes_to_f16(w[i], lo, hi);
    else codes_to_bf16(w[i], lo, hi);
    (i < 2 ? first : second)[2 * (i & 1)] = lo;
    (i < 2 ? first : second)[2 * (i & 1) + 1] = hi;
  }
}

// LDS byte of 16-byte chunk c of K row `tok` (DB * 128 bytes).  A tile's 16 rows
// are tokens 16 (i / 4) + 4 t + i % 4: the swizzle steps through those.
template <int DB>
__device__ inline int k_lds(int tok, int c) {
  const int f = DB == 1 ? ((tok >> 1) & 1) | ((tok >> 4) & 3) << 1 : (tok & 3) | ((tok >> 4) & 3) << 2;
  return tok * DB * 128 + ((c ^ f) << 4);
}
// LDS byte of chunk c of V row d: 64 tokens, 128 bytes; chunk 4 u + g has tokens
// 16 g + 8 u + 0..7 (the 16 lanes of a ds_read_b128's pass come from two groups: with
// neighbouring chunks they still cover all banks once).
__device__ inline int v_lds(int d, int c) { return d * 128 + ((c ^ ((d >> 1) & 7)) << 4); }

template <typename T, int DB, int NC, int NW, int QT, int PT>
__global__ __launch_bounds__(NW * 64, 2) void k_cache_attention_wide(AttnArgs a) {
  typedef typename OperandK<T>::type KT;
  typedef KT v8k __attribute__((ext_vector_type(8)));
  constexpr int DT = DB * 4, kSteps = DB * 2;  // 16-dimension tiles of O; 32-dimension steps of S
  constexpr int kK = 64 * DB * 128, kV = DB * 64 * 128;  // LDS bytes of a chunk's K and V
  constexpr int kCols = NC * 16 * NW, kThreads = NW * 64;
  constexpr int kShare = DB * 256 / kThreads;  // 16-byte pieces of K, and of V, of a thread
  extern __shared__ __attribute__((aligned(256))) int8_t lds[];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int D = a.c.dim, P = a.c.page;
  const BlockAt where = block_at<false>(a);
  const int head = where.head, part = where.part;
  const SeqDev s = seq_of(a.b, P, where.seq);
  if (!s.ok) {
    if (part == 0 && head == 0 && threadIdx.x == 0) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    return;
  }
  // the last columns see the most tokens: first
  const int tile = a.col_tiles - 1 - part % a.col_tiles, split = part / a.col_tiles;
  const int tile0 = tile * kCols;
  if (tile0 >= s.fresh * a.group) return;
  const int total = tile_chunks(a, s, tile0, kCols);
  const int begin = split * a.split_chunks, end = min(begin + a.split_chunks, total);
  if (a.splits > 1 && begin >= end) return;
  const int col0 = tile0 + wave * NC * 16;
  const int pos0 = s.len - s.fresh;
  // chunks that this wave's own columns see
  const int wave_end = min(end, tile_chunks(a, s, col0, NC * 16));

  v8k q[NC][kSteps][QT];
  int limit[NC];
  const float sign = a.scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = col0 + c * 16 + n, i = col / a.group;
    const bool real = i < s.fresh;
    limit[c] = a.causal ? pos0 + i : s.len - 1;
    const T* row = static_cast<const T*>(a.q) + (s.first + (int64_t)(real ? i : 0)) * a.ldq +
                   (int64_t)(head * a.group + col % a.group) * D;
#pragma unroll
    for (int b = 0; b < kSteps; ++b) {
      const int d = b * 32 + g * 8;
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = 0.0f;
      if (real && d < D) {
        if (a.vec) {
          constexpr int W = 16 / sizeof(T);
#pragma unroll
          for (int k = 0; k < 8; k += W) {
            float u[W];
            load_reals<T, W>(row + d + k, u);
#pragma unroll
            for (int j = 0; j < W; ++j) x[k + j] = u[j];
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = (float)row[d + k];
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        // the leading bits, cut, as long as a term follows; a row with an infinity
        // has no softmax: NaN, as for a NaN
        float rest = finite(x[k]) ? x[k] * sign : __builtin_nanf("");
#pragma unroll
        for (int p = 0; p < QT; ++p) {
          const float cut = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, rest) & 0xFFFF0000u);
          q[c][b][p][k] = (KT)(p + 1 < QT ? cut : rest);
          rest -= cut;
        }
      }
    }
  }

  float m[NC], l[NC];
  bool far[NC];  // the reference is too large for the fused form (same in all lanes)
  v4f o[NC][DT];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = kNoMax;
    l[c] = 0.0f;
    far[c] = false;
#pragma unroll
    for (int j = 0; j < DT; ++j) o[c][j] = v4f{0, 0, 0, 0};
  }
  const int first_limit = a.causal ? pos0 + col0 / a.group : s.len - 1;
  const int32_t* table = a.b.table + (int64_t)where.seq * a.b.table_ld;
  const int last_nth = (s.len - 1) >> a.page_log2;
  // page of a token's group of 16; past the sequence's end -1 (nothing is seen of it)
  auto page_of = [&](int t) {
    const int nth = t >> a.page_log2;
    return nth <= last_nth ? table[nth] : -1;
  };

  // This thread's share of a chunk: K pieces of 16 dimensions of a token, V pieces
  // of 16 tokens of a dimension (64 tokens x DB * 4 pieces, and DB * 64 dimensions x
  // 4 groups, over the threads).
  // A chunk's pages are looked up two chunks ahead and its codes and scales loaded
  // one ahead, so that neither of the two latencies is waited for.
  v4i kr[kShare], vr[kShare];
  int k_page[kShare], v_page[kShare], s_page;  // of the chunk to load next
  float next_ks = 0.0f, next_vs = 0.0f;        // of this lane's 16 tokens, 0 without a page
  bool next_there = false;
  auto lookup = [&](int chunk) {
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
      const int at = i * kThreads + (int)threadIdx.x;
      k_page[i] = page_of(chunk * 64 + at / (DB * 4));
      v_page[i] = page_of(chunk * 64 + at / (DB * 64) * 16);
    }
    s_page = page_of(chunk * 64 + g * 16);
  };
  auto load = [&](int chunk) {
    auto valid = [&](int page) { return page < 0 || page >= a.c.pages ? 0 : page; };
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
      const int at = i * kThreads + (int)threadIdx.x;
      const int t = chunk * 64 + at / (DB * 4), d = min(at % (DB * 4) * 16, D - 16);
      kr[i] = *reinterpret_cast<const v4i*>(a.c.k + k_offset(a.c, valid(k_page[i]), head, (t & (P - 1))) + d);
      const int t0 = chunk * 64 + at / (DB * 64) * 16, dv = min(at % (DB * 64), D - 1);
      vr[i] = *reinterpret_cast<const v4i*>(a.c.v + v_offset(a.c, valid(v_page[i]), head, (t0 & (P - 1)), dv));
    }
    next_there = s_page >= 0 && s_page < a.c.pages;
    if (!next_there && chunk * 64 + g * 16 < s.len) raise_flag(a.flags, FXPQ_FLAG_RANGE);
    const int64_t at = (int64_t)valid(s_page) * a.c.heads + head;
    next_ks = a.c.k_scale[at];
    next_vs = a.c.v_scale[at];
  };
  auto store = [&](int buf) {
    int8_t* to = lds + buf * (kK + kV);
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
      const int at = i * kThreads + (int)threadIdx.x;
      v4i lo, hi;
      const int tok = at / (DB * 4), piece = at % (DB * 4);
      codes_to<KT>(kr[i], lo, hi);
      if (piece * 16 >= D) lo = hi = v4i{0, 0, 0, 0};  // past the head: 0 times q's 0
      *reinterpret_cast<v4i*>(to + k_lds<DB>(tok, 2 * piece)) = lo;
      *reinterpret_cast<v4i*>(to + k_lds<DB>(tok, 2 * piece + 1)) = hi;
      const int grp = at / (DB * 64), d = at % (DB * 64);
      codes_to<__bf16>(vr[i], lo, hi);
      *reinterpret_cast<v4i*>(to + kK + v_lds(d, grp)) = lo;
      *reinterpret_cast<v4i*>(to + kK + v_lds(d, 4 + grp)) = hi;
    }
  };

  if (begin < end) {
    lookup(begin);
    load(begin);
    lookup(begin + 1);
    store(0);
  }
  const float to_log2 = a.scale * sign;
  for (int chunk = begin; chunk < end; ++chunk) {
    const int buf = (chunk - begin) & 1;
    __syncthreads();  // this chunk is in LDS, and the other buffer has been read
    const bool there = next_there;
    const float ks = there ? next_ks : 0.0f, vs = there ? next_vs : 0.0f;
    if (chunk + 1 < end) {
      load(chunk + 1);
      lookup(chunk + 2);
    }
    if (chunk < wave_end) {
      const int8_t* kb = lds + buf * (kK + kV);
      const int8_t* vb = kb + kK;
      // independent sums next to each other: a product need not wait for the last
      v4f sum[NC][4];
#pragma unroll
      for (int b = 0; b < kSteps; ++b) {
        v8k k[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
          k[t] = *reinterpret_cast<const v8k*>(kb + k_lds<DB>(16 * (n >> 2) + 4 * t + (n & 3), b * 4 + g));
#pragma unroll
        for (int p = 0; p < QT; ++p)
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c)
              sum[c][t] = mfma_k(k[t], q[c][b][p], b + p ? sum[c][t] : v4f{0, 0, 0, 0});
      }
      float x[NC][16];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[c][i] = sum[c][i >> 2][i & 3];
      const int t0 = chunk * 64 + g * 16;
      const bool edge = chunk * 64 + 63 > first_limit || __any(!there);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float f = ks * to_log2;  // not negative: the largest product has the largest logit
        if (edge) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            x[c][i] = t0 + i > limit[c] || !there ? -INFINITY : scaled(x[c][i], f);
          }
          f = 1.0f;
        }
        float top = x[c][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, x[c][i]);
        top *= f;
        if (__any(top > m[c] + kSlack)) {
          const float now = fmaxf(m[c], over_groups(top)), down = __builtin_amdgcn_exp2f(m[c] - now);
          m[c] = now;
          l[c] *= down;
#pragma unroll
          for (int j = 0; j < DT; ++j) o[c][j] *= down;
          far[c] = __any(fabsf(now) > kFar);
        }
        if (far[c]) {
#pragma unroll
          for (int i = 0; i < 16; ++i) x[c][i] = scaled(x[c][i], f);
          f = 1.0f;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float p = __builtin_amdgcn_exp2f(fmaf(x[c][i], f, -m[c]));
          l[c] += p;
          x[c][i] = p * vs;
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        v8bf p[NC][PT];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          float rest[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) rest[i] = x[c][8 * u + i];
#pragma unroll
          for (int k = 0; k < PT; ++k) {
            if (k + 1 < PT) {  // the leading bits, cut: the next term has the rest
              v4i w;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                w[i] = (int)__builtin_amdgcn_perm(__builtin_bit_cast(unsigned, rest[2 * i + 1]),
                                                  __builtin_bit_cast(unsigned, rest[2 * i]), 0x07060302u);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  float& r = rest[2 * i + e];
                  r -= __builtin_bit_cast(float, __builtin_bit_cast(unsigned, r) & 0xFFFF0000u);
                }
              }
              p[c][k] = __builtin_bit_cast(v8bf, w);
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) p[c][k][i] = (__bf16)rest[i];
            }
          }
        }
#pragma unroll
        for (int j = 0; j < DT; j += 2) {
          v8bf v[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) v[e] = *reinterpret_cast<const v8bf*>(vb + v_lds((j + e) * 16 + n, 4 * u + g));
#pragma unroll
          for (int k = 0; k < PT; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
              for (int c = 0; c < NC; ++c)
                o[c][j + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[e], p[c][k], o[c][j + e], 0, 0, 0);
        }
      }
    }
    if (chunk + 1 < end) store(buf ^ 1);
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 16);
    l[c] += __shfl_xor(l[c], 32);
#pragma unroll
    for (int j = 0; j < DT; ++j) {
      const float v[4] = {o[c][j][0], o[c][j][1], o[c][j][2], o[c][j][3]};
      emit<T>(a, s, head, split, col0 + c * 16 + n, j * 16 + g * 4, m[c], l[c], v);
    }
  }
}

// Joins the splits of each query row: one block per token and query head (64 of 32
// heads of 128: 7 us).
template <typename T>
__global__ __launch_bounds__(256) void k_attention_join(AttnArgs a, int kcols) {
  constexpr int kMany = 256;  // weights kept at a time
  __shared__ float weight[kMany], red[4], sums[1024];
  const SeqDev s = seq_of(a.b, a.c.page, blockIdx.z);
  const int i = blockIdx.x, hq = blockIdx.y;
  if (!s.ok || i >= s.fresh) return;
  const int col = i * a.group + hq % a.group;
  const int total = tile_chunks(a, s, col / kcols * kcols, kcols);
  const int used = (total + a.split_chunks - 1) / a.split_chunks;
  const int64_t row = s.first + (int64_t)i, stride = (int64_t)a.b.tokens * a.q_heads;
  const int64_t r = row * a.q_heads + hq;
  const int tid = threadIdx.x, lane = tid & 63;
  float mx = kNoMax;
  for (int p = tid; p < used; p += 256) mx = fmaxf(mx, a.part_ml[2 * (p * stride + r)]);
#pragma unroll
  for (int d = 32; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
  if (lane == 0) red[tid >> 6] = mx;
  __syncthreads();
  mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  // thread: dimensions 4 x .. of the splits y, y + 256 / (dim / 4), ...
  const int quads = a.c.dim / 4, ways = 256 / quads, x = tid % quads, y = tid / quads;
  float sum = 0.0f;
  v4f v = {0, 0, 0, 0};
  for (int p0 = 0; p0 < used; p0 += kMany) {
    const int many = min(kMany, used - p0);
    __syncthreads();
    if (tid < many) {
      const int64_t at = (p0 + tid) * stride + r;
      const float w = __builtin_amdgcn_exp2f(a.part_ml[2 * at] - mx);
      weight[tid] = w;
      sum += w * a.part_ml[2 * at + 1];
    }
    __syncthreads();
    if (y < ways)
      for (int p = y; p < many; p += ways)
        v += weight[p] * *reinterpret_cast<const v4f*>(a.part_o + ((p0 + p) * stride + r) * a.c.dim + 4 * x);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  __syncthreads();
  if (lane == 0) red[tid >> 6] = sum;
  *reinterpret_cast<v4f*>(sums + 4 * tid) = v;
  __syncthreads();
  if (tid >= quads) return;
  sum = red[0] + red[1] + red[2] + red[3];
  for (int w = 1; w < ways; ++w) v += *reinterpret_cast<const v4f*>(sums + 4 * (w * quads + x));
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  T* out = static_cast<T*>(a.out) + row * a.ldo + (int64_t)hq * a.c.dim + 4 * x;
#pragma unroll
  for (int k = 0; k < 4; ++k) out[k] = (T)(v[k] * f);
}

struct AttnPlan {
  bool tok;     // few columns: the waves of a block share them
  int nc;       // 16-column tiles of a wave
  int waves;    // of a block
  int col_tiles, splits, split_chunks;
  int64_t part, bytes;
};

// Chunks of a split.  With few columns a block's own cost is small, and what matters
// is that all CUs are busy at the end of a ragged batch: 32 chunks (2048 tokens),
// fewer down to 8 where that would leave CUs without a block (one token over
// 131072: 32 chunks 58.9 us, 16 63.0; over 4096: 8 chunks 12.7 us, 16 15.8).  With
// many columns a split writes and reads back all of them, and is worth it only
// where the tiles alone do not fill the CUs (16 new tokens over 8000, 4 heads: 8
// chunks 30 us, 16 49; 4 x 1024 over 4000: whole 237, in three 442).
AttnPlan plan_attention(const Ctx& c, const fxpq_kv_cache& k, const fxpq_kv_batch& b, int q_heads, int type) {
  AttnPlan p{};
  const int64_t cols = (int64_t)b.max_new * (q_heads / k.heads);
  p.tok = cols <= 16;
  p.nc = p.tok || k.dim > 128 || type == FXPQ_F32 ? 1 : 2;
  const int64_t groups = (int64_t)b.seqs * k.heads;
  auto blocks_of = [&](int waves) {
    const int64_t tile = (int64_t)p.nc * 16 * waves;
    p.col_tiles = (int)((cols + tile - 1) / tile);
    return p.col_tiles * groups;
  };
  p.waves = 4;
  int64_t blocks = blocks_of(p.tok ? 1 : 4);
  if (!p.tok && k.dim > 64 && k.dim <= 128 && cols > p.nc * 64) {
    // eight waves share one conversion of the keys and values, but a CU holds one
    // such block: for many tiles, or so few that the cache is split anyway
    // (4 x 1024 over 4000: 237 us against 240; 2 x 64 over 20000: 69 against 88; the
    // reverse where four waves just fill the chip, 4 x 1024 over 1000 with 16
    // ungrouped heads: 174 against 86)
    const int64_t eight = blocks_of(8);
    if (eight >= 2 * (int64_t)c.cus || blocks < c.cus) {
      p.waves = 8;
      blocks = eight;
    } else {
      blocks_of(4);
    }
  }
  const int64_t chunks = (b.max_len + 63) / 64;
  // Blocks that the chip holds at a time, by the kernels' registers; one a CU too for
  // few columns in fp32 of up to 64 dimensions, where two would fit and measure the same
  // (64 sequences of up to 8192: 72.6 and 72.4 us).  Eight waves: one a CU, and a
  // quarter more where there are several sequences, whose blocks end early by their
  // lengths (2 x 64 over up to 20000: 70 us so, 79 without; 4 x 64 in 4 heads 67 and 78;
  // but 123 and 82 where both are 20000 long, which the host does not know).  One
  // sequence's blocks end together, and a quarter would run alone (512 over 20000: 400
  // us so, 271 without; 48 over 100000: 249 and 157).
  const int64_t slots = p.waves == 8 ? (b.seqs > 1 ? (int64_t)c.cus * 5 / 4 : (int64_t)c.cus)
                                     : (int64_t)c.cus * (k.dim > 128 || (p.tok && type == FXPQ_F32) ? 1 : 2);
  int64_t per = (blocks * chunks + slots - 1) / slots;
  if (p.tok) per = per < 8 ? 8 : per > 32 ? 32 : per;
  else per = blocks >= slots ? chunks : per < 8 ? 8 : per;
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

template <typename T, int KCOLS>
hipError_t join_splits(const Ctx& c, const AttnArgs& a) {
  if (a.splits > 1)
    k_attention_join<T><<<dim3((unsigned)a.b.max_new, (unsigned)a.q_heads, (unsigned)a.b.seqs), dim3(256), 0,
                          c.stream>>>(a, KCOLS);
  return hipGetLastError();
}

template <typename T, int DB, int NC, bool TOK>
hipError_t run_attention(const Ctx& c, const AttnArgs& a) {
  // Digits of q and bf16 terms of P by the type that goes in and out: what they
  // drop stays far below that type's own rounding.  (bf16 by one term of P: 116.8
  // against 117.6 us for 64 tokens over up to 8192, and the whole result's relative
  // error 0.0021 in the place of 0.0017, which is that of its own rounding.)
  constexpr int SQ = sizeof(T) == 4 ? 4 : 3;
  constexpr int SP = sizeof(T) == 4 ? 3 : 2;
  constexpr int bytes = TOK ? 4 * NC * 16 * (2 + DB * 64 + 4) * 4 : 0;
  auto* f = k_cache_attention<T, DB, NC, SQ, SP, TOK>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(f), bytes);
  if (e != hipSuccess) return e;
  f<<<attention_grid(a), dim3(256), bytes, c.stream>>>(a);
  return join_splits<T, NC * 16 * (TOK ? 1 : 4)>(c, a);
}

template <typename T, int DB, int NW>
hipError_t run_wide(const Ctx& c, const AttnArgs& a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NC = F32 ? 1 : 2;
  // terms of P as with few columns, so that a sequence's prompt and its single tokens
  // have the same accuracy
  constexpr int bytes = 2 * (64 * DB * 128 + DB * 64 * 128);
  auto* f = k_cache_attention_wide<T, DB, NC, NW, F32 ? 3 : 1, F32 ? 3 : 2>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(f), bytes);
  if (e != hipSuccess) return e;
  f<<<attention_grid(a), dim3(NW * 64), bytes, c.stream>>>(a);
  return join_splits<T, NC * 16 * NW>(c, a);
}

template <typename T, int DB>
hipError_t run_dim(const Ctx& c, const AttnArgs& a, const AttnPlan& p) {
  if (p.tok) return run_attention<T, DB, 1, true>(c, a);
  if constexpr (DB == 2)
    if (p.waves == 8) return run_wide<T, DB, 8>(c, a);
  if constexpr (DB <= 2) return run_wide<T, DB, 4>(c, a);
  else return run_attention<T, DB, 1, false>(c, a);
}

}  // namespace

int64_t cache_attention_workspace(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                                  int q_heads) {
  const int64_t wide = plan_attention(c, cache, b, q_heads, FXPQ_F32).bytes;
  const int64_t narrow = plan_attention(c, cache, b, q_heads, FXPQ_BF16).bytes;
  return wide > narrow ? wide : narrow;  // whatever the type of the call
}

hipError_t launch_cache_attention(const Ctx& c, const fxpq_kv_cache& cache, const fxpq_kv_batch& b,
                                  const void* q, int64_t ldq, int q_heads, float softmax_scale,
                                  int causal, void* out, int64_t ldo, int type, void* ws) {
  const AttnPlan p = plan_attention(c, cache, b, q_heads, type);
  if ((int64_t)cache.heads * b.seqs * p.col_tiles * p.splits * (p.waves / 4) > kMaxBlocks) return hipErrorInvalidValue;
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
  while ((1 << a.page_log2) < cache.page) ++a.page_log2;
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
