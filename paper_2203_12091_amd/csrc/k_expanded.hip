// Expanded attention: keys and values of each head, made of the latents, and the
// rotary key that all heads share.
//
// A block of four waves takes 64 NC query rows of one head over the keys, kTok at a
// time, which it stages in LDS: a key's nope and rotary parts side by side, values
// transposed, dimension by dimension, their tokens next to each other.  Wave by wave
// S = K Q^T with 16 NC rows of q in registers, then O^T = V^T P^T.  LDS row 16 t + i of
// the keys is token 4 TT (i / 4) + 4 t + i % 4 (TT: 16-row tiles of a chunk), so that the
// lane that holds S for a query row has the 4 TT neighbouring tokens that its operand of the
// second product needs: P goes from the first product's result into it without leaving
// the lane.
//
// f16 and bf16 multiply as they are, P rounded to the same type (bf16: 2^-9 a weight, which
// leaves the whole result's error at 1.3 times that of its own rounding; f16 with weights
// lifted by 2^6, so that those down to 2^-20 of the largest keep 11 bits); f32 on the
// f32 matrix instruction, whose products are exact.
#include <type_traits>

#include "kv.hpp"
#include "values.hpp"

namespace fxpq {
namespace {

template <typename T>
struct Operand {
  typedef T v8 __attribute__((ext_vector_type(8)));
  static constexpr int kTok = sizeof(T) == 4 ? 32 : 64;  // tokens of a chunk
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
constexpr float kFar = 0x1p24f;  // references up to this leave an error below 1

struct ExpandedRun {
  ExpandedArgs a;
  int row_tiles, vec, vec_out;
  unsigned* flags;
};

// A logit rounded by itself: a multiply-add would leave the product's rounding error.
__device__ inline float scaled(float x, float f) {
#pragma clang fp contract(off)
  return x * f;
}
__device__ inline float over_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
template <typename T>
__device__ inline bool real_finite(T x) { return finite((float)x); }

// D: dimensions of a query and key (nope + rope); VD: of a value; NC: 16-row tiles of a wave.
template <typename T, int D, int VD, int NC>
__global__ __launch_bounds__(256, 2) void k_expanded_attention(ExpandedRun p) {
  typedef typename Operand<T>::v8 v8;
  constexpr int kTok = Operand<T>::kTok, TT = kTok / 16, S = sizeof(T);
  constexpr int kSteps = D / 32, DT = VD / 16;
  constexpr int kRows = NC * 64;
  constexpr int kKRow = D * S + 16, kVRow = kTok * S + 16;  // LDS bytes of a key, of a value dimension; the pads spread the banks
  constexpr int kPiece = 16 / S;                            // reals of a 16-byte piece
  constexpr int kKPieces = kTok * D / kPiece / 256;         // a thread's share of a chunk's keys
  constexpr int kVCols = VD / 32;                           // value dimensions of a thread, for 8 tokens at 256 / 32 groups
  extern __shared__ __attribute__((aligned(256))) int8_t lds[];
  int8_t* kl = lds;
  int8_t* vl = lds + kTok * kKRow;
  volatile unsigned* wild = reinterpret_cast<volatile unsigned*>(vl + VD * kVRow);  // [2]: tokens of a chunk with a NaN or an infinity in a value
  const ExpandedArgs& a = p.a;
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned heads = (unsigned)a.kv.heads, rest = blockIdx.x / heads;
  const int head = (int)(blockIdx.x % heads), seq = (int)(rest / (unsigned)p.row_tiles);
  const int tile = p.row_tiles - 1 - (int)(rest % (unsigned)p.row_tiles);  // the last rows see the most tokens: first
  const SeqDev s = seq_of(a.b, seq);
  const int from = a.kv.start[seq], to = a.kv.start[seq + 1];
  if (!s.ok || from < 0 || to < from || to - from != s.len || to > a.kv.tokens) {
    if (tile == 0 && head == 0 && threadIdx.x == 0) raise_flag(p.flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int row0 = tile * kRows;
  if (row0 >= s.fresh) return;
  const int pos0 = s.len - s.fresh;
  const int last = min(row0 + kRows, s.fresh) - 1;
  const int end = ((a.causal ? pos0 + last : s.len - 1) + kTok) / kTok;
  const int wrow = row0 + wave * NC * 16;
  const int wlast = min(wrow + NC * 16, s.fresh) - 1;
  const int wave_end = wlast < wrow ? 0 : ((a.causal ? pos0 + wlast : s.len - 1) + kTok) / kTok;
  const float sign = a.scale < 0.0f ? -1.0f : 1.0f, f_log2 = a.scale * sign * 1.44269504088896340736f;

  v8 q[NC][kSteps];  // lane: row n of tile c, dimensions 32 b + 8 g + 0..7
  int limit[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int row = wrow + c * 16 + n;
    limit[c] = a.causal ? pos0 + row : s.len - 1;
    const T* at = static_cast<const T*>(a.q) + (s.first + (int64_t)min(row, s.fresh - 1)) * a.ldq + (int64_t)head * D + 8 * g;
#pragma unroll
    for (int b = 0; b < kSteps; ++b) {
      float x[8];
      if (p.vec) {
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
  bool far[NC];
  v4f o[NC][DT];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = kNoMax;
    l[c] = 0.0f;
    far[c] = false;
#pragma unroll
    for (int j = 0; j < DT; ++j) o[c][j] = v4f{0, 0, 0, 0};
  }
  const int first_limit = a.causal ? pos0 + wrow : s.len - 1;
  const int block_limit = a.causal ? pos0 + row0 : s.len - 1;

  // This thread's share of a chunk: pieces of keys, and kVCols dimensions of tokens
  // (kTok / 8) groups of 8 (f32: 4 groups, of twice the dimensions).
  constexpr int kVGroups = kTok / 8, kVThreads = 256 / kVGroups, kCols = VD / kVThreads;
  static_assert(kCols * kVThreads == VD && kKPieces * 256 * kPiece == kTok * D, "whole shares");
  typedef Reals<T, kPiece> Piece;
  typedef Reals<T, kCols> Cols;
  Piece kr[kKPieces];
  Cols vr[8];
  const T* keys = static_cast<const T*>(a.kv.k) + (int64_t)head * a.kv.hdk;
  const T* shared = static_cast<const T*>(a.kv.key);
  const T* values = static_cast<const T*>(a.kv.v) + (int64_t)head * a.kv.hdv;
  const int vg = threadIdx.x / kVThreads, vc = threadIdx.x % kVThreads * kCols;
  auto load = [&](int chunk) {
    // past the sequence's end its last row, which nobody looks at there
#pragma unroll
    for (int i = 0; i < kKPieces; ++i) {
      const int at = i * 256 + (int)threadIdx.x, tok = at / (D / kPiece), d = at % (D / kPiece) * kPiece;
      const int64_t row = from + (int64_t)min(chunk * kTok + tok, s.len - 1);
      const T* src = d < a.kv.nope ? keys + row * a.kv.ldk + d : shared + row * a.kv.ld_key + (d - a.kv.nope);
      if (p.vec) {
        kr[i] = *reinterpret_cast<const Piece*>(src);
      } else {
#pragma unroll
        for (int k = 0; k < kPiece; ++k) kr[i].v[k] = src[k];
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t row = from + (int64_t)min(chunk * kTok + vg * 8 + j, s.len - 1);
      const T* src = values + row * a.kv.ldv + vc;
      if (p.vec) {
        vr[j] = *reinterpret_cast<const Cols*>(src);
      } else {
#pragma unroll
        for (int k = 0; k < kCols; ++k) vr[j].v[k] = src[k];
      }
    }
  };
  auto store = [&](int chunk) {
#pragma unroll
    for (int i = 0; i < kKPieces; ++i) {
      const int at = i * 256 + (int)threadIdx.x, tok = at / (D / kPiece), piece = at % (D / kPiece);
      const int r = tok & 3, t = tok / 4 % TT, i4 = tok / (4 * TT);
      *reinterpret_cast<Piece*>(kl + (16 * t + 4 * i4 + r) * kKRow + piece * 16) = kr[i];
    }
    // where some rows do not see some tokens, a value that is not finite must not meet
    // their weight of 0: it is kept out of the product and added to the rows that see it
    if (chunk * kTok + kTok - 1 > block_limit) {
      unsigned bad = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int k = 0; k < kCols; ++k)
          if (!real_finite(vr[j].v[k])) {
            bad |= 1u << j;
            vr[j].v[k] = (T)0.0f;
          }
      if (bad) {
        const int at = vg * 8;
        atomicOr(const_cast<unsigned*>(&wild[at / 32]), bad << (at % 32));
      }
    }
#pragma unroll
    for (int k = 0; k < kCols; ++k) {
      v8 x;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = vr[j].v[k];
      *reinterpret_cast<v8*>(vl + (vc + k) * kVRow + vg * 8 * S) = x;
    }
  };

  load(0);
  for (int chunk = 0; chunk < end; ++chunk) {
    __syncthreads();  // the chunk before has been read
    if (threadIdx.x < 2) wild[threadIdx.x] = 0;
    if (chunk * kTok + kTok - 1 > block_limit) __syncthreads();
    store(chunk);
    __syncthreads();
    if (chunk + 1 < end) load(chunk + 1);
    if (chunk >= wave_end) continue;
    v4f sum[NC][TT];
#pragma unroll
    for (int b = 0; b < kSteps; ++b) {
      v8 k[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) k[t] = *reinterpret_cast<const v8*>(kl + (16 * t + n) * kKRow + (32 * b + 8 * g) * S);
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int c = 0; c < NC; ++c) sum[c][t] = mfma8(k[t], q[c][b], b ? sum[c][t] : v4f{0, 0, 0, 0});
    }
    constexpr int N = 4 * TT;  // this lane's tokens: N g + 0 .. N - 1 of the chunk
    const int t0 = chunk * kTok + N * g;
    const bool edge = chunk * kTok + kTok - 1 > first_limit;
    float x[NC][N];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float f = f_log2;
#pragma unroll
      for (int i = 0; i < N; ++i) x[c][i] = sum[c][i >> 2][i & 3];
      if (edge) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[c][i] = t0 + i > limit[c] ? -INFINITY : scaled(x[c][i], f);
        f = 1.0f;
      }
      float top = x[c][0];
#pragma unroll
      for (int i = 1; i < N; ++i) top = fmaxf(top, x[c][i]);
      top *= f;
      if (__any(top > m[c] + kSlack)) {
        // row by row: what one row sees has no part in its neighbours' rounding
        const float row_top = over_groups(top), now = row_top > m[c] + kSlack ? row_top : m[c];
        const float down = __builtin_amdgcn_exp2f(m[c] - now);
        m[c] = now;
        l[c] *= down;
#pragma unroll
        for (int j = 0; j < DT; ++j) o[c][j] *= down;
        far[c] = __any(fabsf(now) > kFar);
      }
      if (far[c]) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[c][i] = scaled(x[c][i], f);
        f = 1.0f;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float w = __builtin_amdgcn_exp2f(fmaf(x[c][i], f, -m[c]));
        if constexpr (std::is_same<T, _Float16>::value) w *= 64.0f;
        l[c] += w;
        x[c][i] = w;
      }
    }
#pragma unroll
    for (int u = 0; u < N / 8; ++u) {
      v8 w[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) w[c][i] = (T)x[c][8 * u + i];
#pragma unroll
      for (int j = 0; j < DT; ++j) {
        const v8 v = *reinterpret_cast<const v8*>(vl + (16 * j + n) * kVRow + (N * g + 8 * u) * S);
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c][j] = mfma8(v, w[c], o[c][j]);
      }
    }
    if (chunk * kTok + kTok - 1 > block_limit) {
      unsigned bits[2] = {wild[0], wild[1]};
      while (bits[0] | bits[1]) {
        const int t = bits[0] ? __builtin_ctz(bits[0]) : 32 + __builtin_ctz(bits[1]);
        bits[t / 32] &= ~(1u << (t % 32));
        const int at = chunk * kTok + t;
        const T* row = values + (from + (int64_t)min(at, s.len - 1)) * a.kv.ldv;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int j = 0; j < DT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float v = (float)row[16 * j + 4 * g + i];
              if (at <= limit[c] && at < s.len && !finite(v)) o[c][j][i] += v;
            }
      }
    }
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 16);
    l[c] += __shfl_xor(l[c], 32);
    const int row = wrow + c * 16 + n;
    if (row >= s.fresh) continue;
    const float f = l[c] == 0.0f ? 0.0f : 1.0f / l[c];
    T* at = static_cast<T*>(a.out) + (s.first + (int64_t)row) * a.ldo + (int64_t)head * VD + 4 * g;
#pragma unroll
    for (int j = 0; j < DT; ++j) {
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

template <typename T, int D, int VD, int NC>
hipError_t run(const Ctx& c, const ExpandedRun& p) {
  constexpr int kTok = Operand<T>::kTok, S = sizeof(T);
  constexpr int bytes = kTok * (D * S + 16) + VD * (kTok * S + 16) + 16;
  auto* f = k_expanded_attention<T, D, VD, NC>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(f), bytes);
  if (e != hipSuccess) return e;
  ExpandedRun r = p;
  r.row_tiles = (p.a.b.max_new + NC * 64 - 1) / (NC * 64);
  const int64_t blocks = (int64_t)r.row_tiles * p.a.b.seqs * p.a.kv.heads;
  if (blocks > kMaxBlocks) return hipErrorInvalidValue;
  f<<<dim3((unsigned)blocks), dim3(256), bytes, c.stream>>>(r);
  return hipGetLastError();
}

template <typename T, int D, int VD>
hipError_t run_rows(const Ctx& c, const ExpandedRun& p) {
  if constexpr (sizeof(T) == 4) return run<T, D, VD, 1>(c, p);
  else return p.a.b.max_new <= 64 ? run<T, D, VD, 1>(c, p) : run<T, D, VD, 2>(c, p);
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
  p.vec_out = fits(a.out, a.ldo, 0);
  p.flags = c.sc.flags;
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    return a.kv.vdim == 64 ? run_dims<T, 64>(c, p) : run_dims<T, 128>(c, p);
  });
}

}  // namespace fxpq
