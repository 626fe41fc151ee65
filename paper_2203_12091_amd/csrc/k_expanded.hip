// Expanded attention: keys and values of each head, made of the latents, and the
// rotary key that all heads share.
//
// A block of four waves takes 64 NC query rows of one head over the keys, kTok at a
// time: two LDS buffers, filled straight from memory while the other one is worked on.
// Wave by wave S = K Q^T with 16 NC rows of q in registers, then O^T = V^T P^T.  A lane
// holds S for one query row and tokens 4 g .. 4 g + 3 of each 16-token tile; two tiles of
// them are its operand of the second product as they are, so P never leaves the lane.
// V's operand is its transpose: the hardware's transposed LDS read hands a lane four
// tokens of one dimension (f32 reads them one by one).
//
// LDS holds panels of 128 bytes a token: keys' nope part, rotary part, values.  Within a
// panel's row the 16-byte pieces are swapped by the token's number, by the address that
// each lane loads from, so that reads of 16 rows cover all banks.
//
// f16 and bf16 multiply as they are, P as two terms of the same type (2^-16 of a weight and
// less; f16 with weights lifted by 2^6, so that those down to 2^-20 of the largest keep 11 bits in
// the first), which leaves the whole result the error of its own rounding alone: with one term
// it was 1.4 times that (bf16 0.0023, f16 0.00027), and single tokens, whose weights have 11
// bits, were more exact than the same tokens in a prompt.  4 x 1024 over up to 4000, bf16, 247 us,
// with one term 200; 1 x 8192, f16, 449 and 342.  f32 is on the f32 matrix instruction, whose
// products are exact.
//
// Where there are few rows the four waves take the same 16 and share the tokens of a chunk.
//
// Bound by the products: 4 x 1024 over up to 4000, 32 heads of 128 + 64 and 128, bf16: 175
// GFLOP (with the weights' second terms 245) in 247 to 252 us, 0.70 PFLOP/s, where one large
// product reaches 1.37; 1 x 8192, f16: 449 us, 0.77 PFLOP/s.  Matrix instructions take 51% of
// the cycles, vector instructions (weights, maxima, rounding) 50%; two blocks a CU overlap the
// two.  With 128 rows and values of 128 up to 62 registers spill, all in the loop of the chunks
// that some rows see in part.  (Measured with one term: of 245 us at first the loop of its own
// for chunks that all rows see took 13, the priority and order of the instructions 35; 64 rows
// a wave, one wave a SIMD, spill: 850 us.)
#include <type_traits>

#include "kv.hpp"
#include "ring.hpp"
#include "values.hpp"

namespace fxpq {
namespace {

template <typename T>
struct Operand {
  typedef T v8 __attribute__((ext_vector_type(8)));
  static constexpr int kTok = sizeof(T) == 4 ? 32 : 64;  // tokens of a wave's chunk
};
__device__ inline v4f mfma8(Operand<_Float16>::v8 a, Operand<_Float16>::v8 b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ inline v4f mfma8(Operand<__bf16>::v8 a, Operand<__bf16>::v8 b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// Step j takes element j of each lane group: the same 32 products of a row and a column.
__device__ inline v4f mfma8(Operand<float>::v8 a, Operand<float>::v8 b, v4f c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

constexpr float kNoMax = -3.40282347e38f;
constexpr float kSlack = 8.0f;   // a reference follows when a logit passes it by more than this (base 2)
// kinds of instructions in a prescribed order
constexpr int kMfma = 0x8, kDsRead = 0x100;
constexpr float kFar = 0x1p24f;  // references up to this leave an error below 1

struct ExpandedRun {
  ExpandedArgs a;
  int row_tiles, vec, vec_out;  // vec: rows are 16-byte aligned and near enough for 32-bit offsets
  unsigned* flags;
};

// A logit rounded by itself: a multiply-add would leave the product's rounding error.
__device__ inline float scaled(float x, float f) {
#pragma clang fp contract(off)
  return x * f;
}
__device__ inline bool is_far(float m) { return fabsf(m) > kFar && m != kNoMax; }
__device__ inline float over_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// Panels of 128 bytes of a token's row, and a piece's place in its row.
template <typename T, int TOK>
struct Panels {
  static constexpr int kDims = 128 / (int)sizeof(T);
  static constexpr int of(int dims) { return (dims + kDims - 1) / kDims; }
  static constexpr int kBytes = TOK * 128;  // of a panel of TOK tokens
};
__device__ inline int key_swap(int tok) { return (tok >> 1) & 7; }
template <typename T>
__device__ inline int value_swap(int tok) {
  return sizeof(T) == 4 ? ((tok >> 2) & 1) << 2 : ((tok >> 1) & 3) << 1;
}

// A thread's piece of each panel, real by real.
template <typename T, int TOK>
__device__ inline void copy_pieces(const int8_t* from, int panels, int8_t* to) {
  constexpr int kPiece = 16 / (int)sizeof(T);
#pragma unroll 1
  for (int q = 0; q < panels; ++q) {
    const T* src = reinterpret_cast<const T*>(from + q * 128);
    Reals<T, kPiece> x;
#pragma unroll
    for (int k = 0; k < kPiece; ++k) x.v[k] = src[k];
    *reinterpret_cast<Reals<T, kPiece>*>(to + q * Panels<T, TOK>::kBytes) = x;
  }
}

typedef __attribute__((address_space(3))) const int8_t* LdsAt;
__device__ inline LdsAt lds_at(const int8_t* p) { return (LdsAt)(uint32_t)(uintptr_t)p; }
template <typename V>
__device__ inline V lds_read(LdsAt p) { return *(__attribute__((address_space(3))) const V*)p; }

// A lane's first byte of values, for dimensions 16 j .. of panels' quarters j % 4 (f32:
// halves j % 2); the rest of an operand's address is a constant.
template <typename T>
__device__ inline int value_at(int j, int g, int n) {
  if constexpr (sizeof(T) == 4) return 4 * g * 128 + ((((j & 1) * 4 + (n >> 2)) ^ value_swap<T>(4 * g)) << 4) + (n & 3) * 4;
  // lane n points at token n / 4 of four, dimensions 4 (n % 4) .. + 3
  const int tok = 4 * g + (n >> 2), piece = (j & 3) * 2 + ((n >> 1) & 1);
  return tok * 128 + ((piece ^ value_swap<T>(tok)) << 4) + (n & 1) * 8;
}
// Eight tokens of one dimension: tokens 4 g + 0..3 of the 16-token tiles 2 u and 2 u + 1,
// dimension 16 j + n, from `at` = value_at of j.
template <typename T, int TOK>
__device__ inline typename Operand<T>::v8 value_operand(LdsAt at, int u, int j) {
  typename Operand<T>::v8 v;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      v[k] = lds_read<float>(at + (j >> 1) * Panels<T, TOK>::kBytes + (32 * u + 16 * (k >> 2) + (k & 3)) * 128);
  } else {
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef short v8s __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) v4s* Quad;
    v4s part[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      part[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Quad)(at + (j >> 2) * Panels<T, TOK>::kBytes + (32 * u + 16 * k) * 128));
    v = __builtin_bit_cast(typename Operand<T>::v8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
  return v;
}

// D: dimensions of a query and key (nope + rope: up to 128 64 + 32 or 64, else 128 + 32 or
// 64); VD: of a value; NC: 16-row tiles of a wave.  SPLIT: the four waves have the same 16
// rows and a quarter of each chunk's 128 tokens; what they found is joined at the end.
template <typename T, int D, int VD, int NC, bool SPLIT>
__global__ __launch_bounds__(256, 2) void k_expanded_attention(const ExpandedRun p) {
  typedef typename Operand<T>::v8 v8;
  static_assert(!SPLIT || (NC == 1 && sizeof(T) == 2), "a wave's 32 tokens are one operand");
  constexpr int kTok = SPLIT ? 128 : Operand<T>::kTok, kOwn = SPLIT ? 32 : kTok;  // of a chunk and of a wave in it
  constexpr int TT = kOwn / 16, S = sizeof(T);
  constexpr int kSteps = D / 32, DT = VD / 16;
  constexpr int kRows = SPLIT ? 16 : NC * 64;
  constexpr int kPiece = 16 / S;  // reals of a 16-byte piece
  constexpr int kTerms = S == 2 ? 2 : 1;  // of a weight
  typedef Panels<T, kTok> Pan;
  constexpr int KP = Pan::of(D), VP = Pan::of(VD), kStage = (KP + VP) * Pan::kBytes;
  extern __shared__ __attribute__((aligned(256))) int8_t lds[];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // copies of the arguments: the loads below are opaque to the compiler
  const int64_t ldk = p.a.kv.ldk, ldr = p.a.kv.ld_key, ldv = p.a.kv.ldv;
  const bool vec = p.vec;
  const float scale = p.a.scale;
  const int causal = p.a.causal;
  const unsigned heads = (unsigned)p.a.kv.heads, rest = blockIdx.x / heads;
  const int head = (int)(blockIdx.x % heads), seq = (int)(rest / (unsigned)p.row_tiles);
  const int tile = p.row_tiles - 1 - (int)(rest % (unsigned)p.row_tiles);  // the last rows see the most tokens: first
  const SeqDev s = block_seq(seq_of(p.a.b, seq));
  const int from = __builtin_amdgcn_readfirstlane(p.a.kv.start[seq]), to = __builtin_amdgcn_readfirstlane(p.a.kv.start[seq + 1]);
  if (!s.ok || from < 0 || to < from || to - from != s.len || to > p.a.kv.tokens) {
    if (tile == 0 && head == 0 && threadIdx.x == 0) raise_flag(p.flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int row0 = tile * kRows;
  if (row0 >= s.fresh) return;
  const int pos0 = s.len - s.fresh;
  const int last = min(row0 + kRows, s.fresh) - 1;
  const int end = ((causal ? pos0 + last : s.len - 1) + kTok) / kTok;
  const int wrow = SPLIT ? row0 : row0 + wave * NC * 16, wtok = SPLIT ? wave * kOwn : 0;
  const int wlast = min(wrow + NC * 16, s.fresh) - 1;
  const int wave_end = wlast < wrow ? 0 : ((causal ? pos0 + wlast : s.len - 1) + kTok) / kTok;

  // A chunk's pieces: thread tid loads piece tid % 8 of rows tid / 8 and 32 on, panel by panel.
  constexpr int nope_panels = (D > 128 ? 128 : 64) / Pan::kDims, kRope = D > 128 ? D - 128 : D - 64;
  const int8_t* keys = reinterpret_cast<const int8_t*>(static_cast<const T*>(p.a.kv.k) + from * ldk + head * p.a.kv.hdk);
  const int8_t* shared = reinterpret_cast<const int8_t*>(static_cast<const T*>(p.a.kv.key) + from * ldr);
  const int8_t* values = reinterpret_cast<const int8_t*>(static_cast<const T*>(p.a.kv.v) + from * ldv + head * p.a.kv.hdv);
  const int trow = (int)threadIdx.x >> 3;
  const int kpiece = ((int)threadIdx.x & 7) ^ key_swap(trow), vpiece = ((int)threadIdx.x & 7) ^ value_swap<T>(trow);
  // a rotary part of half a panel: its first half twice
  const int rpiece = kRope * S < 128 ? kpiece & 3 : kpiece;
  auto load = [&](int chunk, int buf) __attribute__((always_inline)) {
    int8_t* to_lds = lds + buf * kStage + wave * 1024;
    const int64_t row_at = (int64_t)chunk * kTok;
    // past the sequence's end its last row, which nobody looks at there
    const int most = s.len - 1 - chunk * kTok;
#pragma unroll
    for (int half = 0; half < kTok / 32; ++half) {
      const int r = min(trow + 32 * half, most);
      if (vec) {
        const uint32_t ko = (uint32_t)r * (uint32_t)(ldk * S) + kpiece * 16;
        const uint32_t ro = (uint32_t)r * (uint32_t)(ldr * S) + rpiece * 16;
        const uint32_t vo = (uint32_t)r * (uint32_t)(ldv * S) + vpiece * 16;
#pragma unroll
        for (int q = 0; q < KP; ++q) {
          int8_t* l = to_lds + q * Pan::kBytes + half * 4096;
          if (q < nope_panels) dma16(keys + row_at * ldk * S + q * 128, ko, l);
          else dma16(shared + row_at * ldr * S + (q - nope_panels) * 128, ro, l);
        }
#pragma unroll
        for (int q = 0; q < VP; ++q)
          dma16(values + row_at * ldv * S + q * 128, vo, to_lds + (KP + q) * Pan::kBytes + half * 4096);
      } else {
        const int64_t row = row_at + r;
        copy_pieces<T, kTok>(keys + (row * ldk * S + kpiece * 16), nope_panels, to_lds + half * 4096 + lane * 16);
        copy_pieces<T, kTok>(shared + (row * ldr * S + rpiece * 16), KP - nope_panels,
                       to_lds + nope_panels * Pan::kBytes + half * 4096 + lane * 16);
        copy_pieces<T, kTok>(values + (row * ldv * S + vpiece * 16), VP, to_lds + KP * Pan::kBytes + half * 4096 + lane * 16);
      }
    }
  };
  load(0, 0);

  const float sign = scale < 0.0f ? -1.0f : 1.0f, f_log2 = scale * sign * 1.44269504088896340736f;
  v8 q[NC][kSteps];  // lane: row n of tile c, dimensions 32 b + 8 g + 0..7
  int limit[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int row = wrow + c * 16 + n;
    limit[c] = causal ? pos0 + row : s.len - 1;
    const T* at = static_cast<const T*>(p.a.q) + (s.first + (int64_t)min(row, s.fresh - 1)) * p.a.ldq + (int64_t)head * D + 8 * g;
#pragma unroll
    for (int b = 0; b < kSteps; ++b) {
      float x[8];
      if (vec) {
#pragma unroll
        for (int k = 0; k < 8; k += kPiece) {
          float u[kPiece];
          load_reals<T, kPiece>(at + 32 * b + k, u);
#pragma unroll
          for (int j = 0; j < kPiece; ++j) x[k + j] = u[j];
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (float)at[32 * b + k];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) q[c][b][k] = (T)(x[k] * sign);
    }
  }
  float m[NC], l[NC];
  bool far = false;  // a reference is too large for the fused form
  v4f o[NC][DT];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = kNoMax;
    l[c] = 0.0f;
#pragma unroll
    for (int j = 0; j < DT; ++j) o[c][j] = v4f{0, 0, 0, 0};
  }
  const int first_limit = causal ? pos0 + wrow : s.len - 1;
  constexpr float kLift = std::is_same<T, _Float16>::value ? 6.0f : 0.0f;

  const LdsAt first = lds_at(lds) + wtok * 128;
  constexpr int kValueBases = S == 4 ? 2 : 4;
  int kat[2], vat[kValueBases];
#pragma unroll
  for (int e = 0; e < 2; ++e) kat[e] = n * 128 + ((S == 4 ? 2 * g + e : 4 * e + g) ^ key_swap(n)) * 16;
#pragma unroll
  for (int j = 0; j < kValueBases; ++j) vat[j] = KP * Pan::kBytes + value_at<T>(j, g, n);

  // One chunk; edge: some of the wave's rows do not see some of its tokens.
  auto step = [&](int chunk, auto at_edge) __attribute__((always_inline)) {
    constexpr bool edge = decltype(at_edge)::value;
    __builtin_amdgcn_s_waitcnt(0);  // this chunk is in LDS
    ring_barrier();                 // everybody's part of it, and the other buffer has been read
    const LdsAt stage = first + (chunk & 1) * kStage;
    if (chunk + 1 < end) load(chunk + 1, (chunk + 1) & 1);
    if (edge && chunk >= wave_end) return;
    v4f sum[NC][TT];
    const LdsAt kb[2] = {stage + kat[0], stage + kat[1]};
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int b = 0; b < kSteps; ++b) {
      v8 k[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const int at = b * 32 / Pan::kDims * Pan::kBytes + 16 * t * 128;
        if constexpr (S == 2) {
          k[t] = lds_read<v8>(kb[b & 1] + at);
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const v4f part = lds_read<v4f>(kb[e] + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) k[t][4 * e + i] = part[i];
          }
        }
      }
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int c = 0; c < NC; ++c) sum[c][t] = mfma8(k[t], q[c][b], b ? sum[c][t] : v4f{0, 0, 0, 0});
    }
    if constexpr (S == 2) {
      // the next step's operands are read before this one's products
      __builtin_amdgcn_sched_group_barrier(kDsRead, 2 * TT, 0);
#pragma unroll
      for (int b = 0; b < kSteps; ++b) {
        __builtin_amdgcn_sched_group_barrier(kMfma, TT * NC, 0);
        if (b + 2 < kSteps) __builtin_amdgcn_sched_group_barrier(kDsRead, TT, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    constexpr int N = 4 * TT;  // this lane's tokens: 16 (i / 4) + 4 g + i % 4 of the chunk
    const int t0 = chunk * kTok + wtok + 4 * g;
    float x[NC][N], f = f_log2;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < N; ++i) x[c][i] = sum[c][i >> 2][i & 3];
    if constexpr (edge) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < N; ++i) x[c][i] = t0 + 16 * (i >> 2) + (i & 3) > limit[c] ? -INFINITY : scaled(x[c][i], f);
      f = 1.0f;
    }
    float top[NC];
    bool over = false;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      top[c] = x[c][0];
#pragma unroll
      for (int i = 1; i < N; ++i) top[c] = fmaxf(top[c], x[c][i]);
      top[c] *= f;
      over |= top[c] > m[c] + kSlack;
    }
    if (__any(over)) {
      far = false;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        // row by row: what one row sees has no part in its neighbours' rounding
        const float row_top = over_groups(top[c]), now = row_top > m[c] + kSlack ? row_top : m[c];
        const float down = __builtin_amdgcn_exp2f(m[c] - now);
        m[c] = now;
        l[c] *= down;
#pragma unroll
        for (int j = 0; j < DT; ++j) o[c][j] *= down;
        far |= is_far(now);
      }
      far = __any(far);
    }
    float ref[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) ref[c] = kLift - m[c];
    if (far) {
      // (row by row again)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bool mine = is_far(m[c]);
#pragma unroll
        for (int i = 0; i < N; ++i) x[c][i] = mine ? scaled(x[c][i], f) - m[c] + kLift : fmaf(x[c][i], f, ref[c]);
        ref[c] = 0.0f;
      }
      f = 1.0f;
    }
    v8 w[kTerms][NC][N / 8];
    auto weigh = [&](int u, int i) __attribute__((always_inline)) {  // token i of the 8 of operand u
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float e = __builtin_amdgcn_exp2f(fmaf(x[c][8 * u + i], f, ref[c]));
        l[c] += e;
        w[0][c][u][i] = (T)e;
        if constexpr (kTerms == 2) w[1][c][u][i] = (T)(e - (float)w[0][c][u][i]);
      }
    };
    const LdsAt vb = stage;
    constexpr int kAhead = 4;  // operands read ahead
    v8 v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) v[j] = value_operand<T, kTok>(vb + vat[j % kValueBases], j / DT, j % DT);
#pragma unroll
    for (int i = 0; i < 8; ++i) weigh(0, i);
    // Where some rows do not see some tokens, a value that is not finite must not meet
    // their weight of 0: it is kept out of the product and added to the rows that see it.
    bool wild = false;
    const int8_t* vl = lds + (chunk & 1) * kStage + KP * Pan::kBytes;
    if constexpr (edge) {
#pragma unroll 1
      for (int i = lane; i < VP * kTok * 8; i += 64) {
        const Reals<T, kPiece> y = *reinterpret_cast<const Reals<T, kPiece>*>(vl + i * 16);
#pragma unroll
        for (int k = 0; k < kPiece; ++k) wild |= !finite((float)y.v[k]);
      }
      wild = __any(wild);
    }
    if (!wild) {
      // the second half's weights between the first half's products, in this order
#pragma unroll
      for (int k = 0; k < N / 8 * DT; ++k) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < kTerms; ++t)
#pragma unroll
          for (int c = 0; c < NC; ++c) o[c][k % DT] = mfma8(v[k % kAhead], w[t][c][k / DT], o[c][k % DT]);
        const int ahead = k + kAhead;
        if (ahead < N / 8 * DT) v[k % kAhead] = value_operand<T, kTok>(vb + vat[ahead % kValueBases], ahead / DT, ahead % DT);
        if (N > 8 && k < DT)
#pragma unroll
          for (int i = 0; i < 8 / DT; ++i) weigh(1, k * (8 / DT) + i);
      }
    } else {
      if (N > 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) weigh(N / 8 - 1, i);
#pragma unroll 1
      for (int u = 0; u < N / 8; ++u)
#pragma unroll
        for (int j = 0; j < DT; ++j) {
          v8 y = value_operand<T, kTok>(vb + vat[j % kValueBases], u, j);
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = finite((float)y[k]) ? y[k] : (T)0.0f;
#pragma unroll
          for (int t = 0; t < kTerms; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c) o[c][j] = mfma8(y, u ? w[t][c][N / 8 - 1] : w[t][c][0], o[c][j]);
        }
#pragma unroll 1
      for (int t = wtok; t < wtok + kOwn; ++t) {
        const int at = chunk * kTok + t;
        if (at >= s.len) break;
#pragma unroll
        for (int j = 0; j < DT; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int d = 16 * j + 4 * g + i;
            const float v = (float)*reinterpret_cast<const T*>(
                vl + d / Pan::kDims * Pan::kBytes + t * 128 +
                ((d % Pan::kDims / kPiece ^ value_swap<T>(t)) << 4) + d % kPiece * S);
#pragma unroll
            for (int c = 0; c < NC; ++c)
              if (at <= limit[c] && !finite(v)) o[c][j][i] += v;
          }
      }
    }
  };
  // the chunks that all of the wave's rows see whole come first
  const int whole = wave_end ? min((first_limit + 1) / kTok, end) : 0;
#pragma unroll 1
  for (int chunk = 0; chunk < whole; ++chunk) step(chunk, std::false_type());
#pragma unroll 1
  for (int chunk = whole; chunk < end; ++chunk) step(chunk, std::true_type());
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 16);
    l[c] += __shfl_xor(l[c], 32);
  }
  constexpr int kTiles = SPLIT ? DT / 4 : DT;  // 16-dimension tiles that a wave writes
  const int j0 = SPLIT ? wave * kTiles : 0;
  if constexpr (SPLIT) {
    v4f* parts = reinterpret_cast<v4f*>(lds);                         // [wave][tile][lane]
    float* stats = reinterpret_cast<float*>(lds + 4 * DT * 64 * 16);  // [wave][row]: reference, sum
    __syncthreads();  // the chunks have been read
#pragma unroll
    for (int j = 0; j < DT; ++j) parts[(wave * DT + j) * 64 + lane] = o[0][j];
    if (g == 0) {
      stats[(wave * 16 + n) * 2] = m[0];
      stats[(wave * 16 + n) * 2 + 1] = l[0];
    }
    __syncthreads();
    float ms[4], top = kNoMax;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      ms[w] = stats[(w * 16 + n) * 2];
      top = fmaxf(top, ms[w]);
    }
    l[0] = 0.0f;
#pragma unroll
    for (int j = 0; j < kTiles; ++j) o[0][j] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(ms[w] - top);
      l[0] += f * stats[(w * 16 + n) * 2 + 1];
#pragma unroll
      for (int j = 0; j < kTiles; ++j) o[0][j] += f * parts[(w * DT + j0 + j) * 64 + lane];
    }
  }
  if constexpr (kTerms == 2) {
    // An infinite value times a weight's second term, which may be 0 or below it, is NaN.  Where a
    // result is NaN and its weights are not, the values that are not finite are what it is made of.
    bool bad = false;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) bad |= o[c][j][i] != o[c][j][i] && l[c] == l[c];
    if (__any(bad)) {
      v4f sum[NC][kTiles];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < kTiles; ++j) sum[c][j] = v4f{0, 0, 0, 0};
#pragma unroll 1
      for (int t = 0; t < s.len; ++t) {
        const T* at = reinterpret_cast<const T*>(values) + t * ldv + 16 * j0 + 4 * g;
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = (float)at[16 * j + i];
#pragma unroll
            for (int c = 0; c < NC; ++c)
              if (t <= limit[c] && !finite(v)) sum[c][j][i] += v;
          }
      }
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[c][j][i] = sum[c][j][i] == 0.0f ? o[c][j][i] : sum[c][j][i];
    }
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int row = wrow + c * 16 + n;
    if (row >= s.fresh) continue;
    const float f = l[c] == 0.0f ? 0.0f : 1.0f / l[c];
    T* at = static_cast<T*>(p.a.out) + (s.first + (int64_t)row) * p.a.ldo + (int64_t)head * VD + 16 * j0 + 4 * g;
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      const float y[4] = {o[c][j][0] * f, o[c][j][1] * f, o[c][j][2] * f, o[c][j][3] * f};
      if (p.vec_out) {
        store_reals<T, 4>(at + 16 * j, y);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) at[16 * j + i] = (T)y[i];
      }
    }
  }
}

template <typename T, int D, int VD, int NC, bool SPLIT = false>
hipError_t run(const Ctx& c, const ExpandedRun& p) {
  typedef Panels<T, SPLIT ? 128 : Operand<T>::kTok> Pan;
  constexpr int bytes = 2 * (Pan::of(D) + Pan::of(VD)) * Pan::kBytes, rows = SPLIT ? 16 : NC * 64;
  auto* f = k_expanded_attention<T, D, VD, NC, SPLIT>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(f), bytes);
  if (e != hipSuccess) return e;
  ExpandedRun r = p;
  r.row_tiles = (p.a.b.max_new + rows - 1) / rows;
  const int64_t blocks = (int64_t)r.row_tiles * p.a.b.seqs * p.a.kv.heads;
  if (blocks > kMaxBlocks) return hipErrorInvalidValue;
  f<<<dim3((unsigned)blocks), dim3(256), bytes, c.stream>>>(r);
  return hipGetLastError();
}

template <typename T, int D, int VD>
hipError_t run_rows(const Ctx& c, const ExpandedRun& p) {
  if constexpr (sizeof(T) == 2) {
    // 128 rows of a block read half as much, 64 make twice as many blocks.  Two blocks run on
    // a CU; in us with 64 and 128 rows: 4 x 1024 over 4000, 16 heads (2 blocks of 128 rows a
    // CU) 222 and 211, 1 x 1024 over 2048, 128 heads (4) 215 and 186, 1 x 4096, 16 heads (2)
    // 138 and 145, 2 x 1024 over 2048 (1) 65 and 70, 4 x 128 over 2048 (1/4) 48 and 68
    const int64_t blocks = ((int64_t)p.a.b.max_new + 127) / 128 * p.a.b.seqs * p.a.kv.heads;
    if (blocks >= 2 * (int64_t)c.cus) return run<T, D, VD, 2>(c, p);
    // where tiles of 16 rows do not fill the chip, the waves share the tokens: 1 x 64 over 8192,
    // 16 heads, 80 us, 64 rows a block 160; 4 x 64 over 2048 32 and 48, 2 x 77 over 127 11.4 and
    // 14.2, but 16 x 16 over 300 18.5 and 15.8.  (A token of f32 takes twice the LDS.)
    const int64_t tiles = ((int64_t)p.a.b.max_new + 15) / 16 * p.a.b.seqs * p.a.kv.heads;
    if (tiles <= c.cus) return run<T, D, VD, 1, true>(c, p);
  }
  return run<T, D, VD, 1>(c, p);
}

template <typename T, int VD>
hipError_t run_dims(const Ctx& c, const ExpandedRun& p) {
  switch (p.a.kv.nope + p.a.kv.rope) {
    case 96: return run_rows<T, 96, VD>(c, p);
    case 128: return run_rows<T, 128, VD>(c, p);
    case 160: return run_rows<T, 160, VD>(c, p);
    default: return run_rows<T, 192, VD>(c, p);
  }
}

}  // namespace

hipError_t launch_expanded_attention(const Ctx& c, const ExpandedArgs& a, int type) {
  ExpandedRun p{};
  p.a = a;
  const int64_t size = real_bytes(type);
  const auto fits = [&](const void* at, int64_t ld, int64_t hd) {
    return (uintptr_t)at % 16 == 0 && ld * size % 16 == 0 && hd * size % 16 == 0;
  };
  p.vec = fits(a.kv.k, a.kv.ldk, a.kv.hdk) && fits(a.kv.v, a.kv.ldv, a.kv.hdv) && fits(a.kv.key, a.kv.ld_key, 0) &&
          fits(a.q, a.ldq, 0);
  // a chunk's rows (32 of f32, 128 of other types at most) have to lie within 32-bit offsets of each other
  constexpr int64_t kNear = int64_t(1) << 24;
  p.vec = p.vec && a.kv.ldk < kNear && a.kv.ldv < kNear && a.kv.ld_key < kNear;
  p.vec_out = fits(a.out, a.ldo, 0);
  p.flags = c.sc.flags;
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    return a.kv.vdim == 64 ? run_dims<T, 64>(c, p) : run_dims<T, 128>(c, p);
  });
}

}  // namespace fxpq
