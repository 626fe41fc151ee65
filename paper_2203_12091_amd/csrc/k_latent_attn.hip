// Absorbed attention over the paged 8-bit cache of latents: one row of codes a token
// is key and value of every head.
//
// A sequence's query rows are its new tokens' heads (row = token * heads + head); a
// block takes 16 RT of them over the cache, 64 tokens at a time.  Wave w computes S = K Q^T
// for tokens 16 w .. 16 w + 15: it loads their codes from the cache in the operand's
// layout (lane: token lane % 16, 16 codes from 16 (lane / 16)), converts them to f16
// (exact) and multiplies them with q, which all waves hold in registers, as f16 too: q is
// scaled by a power of two of its row, so a bf16 or f16 value is exact down to 2^-27 of
// the row's largest, and f32 is two f16 terms.  The codes go to LDS as they are, P as f16
// beside them, and after one barrier every wave multiplies all 64 tokens with its own
// quarter of the latent's dimensions: O^T = C^T P^T.  The conversion there is the
// transposition: a lane reads the same 8 (or 4) dimensions of 8 tokens and pairs bytes of
// neighbouring tokens.
//
// A token's scale s_t belongs to both products.  With x_t the logit (base 2), m the
// row's reference and R a power of two above every scale seen, P_t = 2^(x_t - m) s_t / R
// goes into O and 2^(x_t - m) into the sum.  m follows max (x_t + log2(s_t / R)) only
// when a row passes it by more than kSlack, so P_t is below 2^(kSlack + kLift) and most
// chunks need neither a maximum across the waves nor a second barrier.
#include "kv.hpp"
#include "values.hpp"

namespace fxpq {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

struct LatentRun {
  LatentArgs a;
  int row_tiles, splits, split_chunks, page_log2, vec;
  float* part_o;   // [splits][tokens][heads][latent]
  float* part_ml;  // [splits][tokens][heads][2]: reference and sum
  unsigned* flags;
};

constexpr float kNoMax = -3.40282347e38f;  // reference before any token
constexpr float kSlack = 8.0f;
// P is written as f16: 2^kLift at the reference, so that weights down to 2^-20 of the
// largest keep all 11 bits and smaller ones lose at most 2^-31 of it.
constexpr float kLift = 64.0f;
constexpr float kLeastLog = -50.0f;  // of s_t / R, where it only moves the reference

__device__ inline void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4));  // LDS operations only
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Byte u = code + 128 below the exponent of 1024 is 1024 + u, and 1024 + u - 1152 the
// code, exactly.
__device__ inline unsigned halves(unsigned biased) {
  const v2h off = {(_Float16)1152.0f, (_Float16)1152.0f};
  return __builtin_bit_cast(unsigned, __builtin_bit_cast(v2h, biased) - off);
}
// 16 codes as two operands of 8.
__device__ inline void codes_to_halves(v4i w, v8h& lo, v8h& hi) {
  v4i r[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned u = (unsigned)w[i] ^ 0x80808080u;
    r[i >> 1][2 * (i & 1)] = (int)halves(__builtin_amdgcn_perm(0x64646464u, u, 0x04010400u));
    r[i >> 1][2 * (i & 1) + 1] = (int)halves(__builtin_amdgcn_perm(0x64646464u, u, 0x04030402u));
  }
  lo = __builtin_bit_cast(v8h, r[0]);
  hi = __builtin_bit_cast(v8h, r[1]);
}
// Byte `at` of two tokens' words as a pair of halves.
__device__ inline int pair_of(unsigned first, unsigned second, int at) {
  return (int)halves(__builtin_amdgcn_perm(second, first, 0x0C040C00u + (unsigned)at * 0x00010001u) ^ 0x64806480u);
}

__device__ inline v4f mfma(v8h a, v8h b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// 64-token chunks that rows row0 .. row0 + rows - 1 of a sequence see.
__device__ inline int rows_chunks(const LatentRun& p, const SeqDev& s, int row0, int rows) {
  const int last = min(row0 + rows, s.fresh * p.a.heads) - 1;
  if (last < row0) return 0;
  const int limit = p.a.causal ? s.len - s.fresh + last / p.a.heads : s.len - 1;
  return (limit + 64) >> 6;
}

// The maximum over the four 16-lane groups of a wave, lane by lane.
__device__ inline float over_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

template <int LB, int RT, int QT>
struct LatentLds {
  static constexpr int kRow = LB * 64 + 16;  // bytes of a token: the pad spreads the banks
  static constexpr int kCodes = 64 * kRow;
  static constexpr int kPRow = 144;  // bytes of a row of P: 64 halves and a pad
  static constexpr int kP = RT * 16 * kPRow;
  static constexpr int kStats = 2 * kCodes + 2 * QT * kP;
  static constexpr int kBytes = kStats + 4 * RT * 16 * 4 + 64;
};

template <typename T, int LB, int RT>
__global__ __launch_bounds__(256, RT == 1 && sizeof(T) == 2 ? 2 : 1) void k_latent_attention(LatentRun p) {
  constexpr int QT = sizeof(T) == 4 ? 2 : 1;  // f16 terms of q and of P
  constexpr int KB = LB + 1;                  // 64-byte pieces of a token: the latent's, the key's
  constexpr int kRows = RT * 16;
  typedef LatentLds<LB, RT, QT> L;
  extern __shared__ __attribute__((aligned(256))) int8_t lds[];
  float* tops = reinterpret_cast<float*>(lds + L::kStats);          // [4][kRows]
  float* scales = tops + 4 * kRows;                                 // [4]
  volatile int* raised = reinterpret_cast<volatile int*>(scales + 4);  // [2]: chunk + 1 of the last that passed its reference
  const LatentArgs& a = p.a;
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Row tiles of one part of a cache are 8 ids apart: on one XCD, whose L2 they share.
  const unsigned oct = blockIdx.x / 8, pairs = (unsigned)a.b.seqs * (unsigned)p.splits;
  const unsigned pair = oct / (unsigned)p.row_tiles * 8 + blockIdx.x % 8;
  if (pair >= pairs) return;
  const int tile = p.row_tiles - 1 - (int)(oct % (unsigned)p.row_tiles);  // the last rows see the most tokens
  const int split = (int)(pair / (unsigned)a.b.seqs), seq = (int)((pair + split) % (unsigned)a.b.seqs);
  const int P = a.c.page;
  const SeqDev s = block_seq(seq_of(a.b, P, seq));
  if (!s.ok) {
    if (split == 0 && tile == 0 && threadIdx.x == 0) raise_flag(p.flags, FXPQ_FLAG_RANGE);
    return;
  }
  const int row0 = tile * kRows, rows = s.fresh * a.heads;
  if (row0 >= rows) return;
  const int total = rows_chunks(p, s, row0, kRows);
  const int begin = split * p.split_chunks, end = min(begin + p.split_chunks, total);
  if (p.splits > 1 && begin >= end) return;
  const int pos0 = s.len - s.fresh;

  v8h q[QT][RT][2 * KB];  // lane: row n of tile r, dimensions 64 b + 16 g + 8 h + 0..7 at 2 b + h
  float qn[RT];
  int limit[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = row0 + r * 16 + n, i = row / a.heads, head = row % a.heads;
    const bool real = row < rows;
    limit[r] = a.causal ? pos0 + i : s.len - 1;
    const int64_t at = s.first + (int64_t)(real ? i : 0);
    const T* ql = static_cast<const T*>(a.q) + at * a.ldq + head * a.hdq + 16 * g;
    const T* qr = static_cast<const T*>(a.qr) + at * a.ldqr + head * a.hdqr + 16 * g;
    float x[KB][16];
    unsigned top = 0;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const bool some = real && (b < LB || 16 * g < a.c.rope);
      const T* from = b < LB ? ql + 64 * b : qr;
#pragma unroll
      for (int k = 0; k < 16; ++k) x[b][k] = 0.0f;
      if (some) {
        if (p.vec) {
          constexpr int W = 16 / sizeof(T);
#pragma unroll
          for (int k = 0; k < 16; k += W) {
            float u[W];
            load_reals<T, W>(from + k, u);
#pragma unroll
            for (int j = 0; j < W; ++j) x[b][k + j] = u[j];
          }
        } else {
#pragma unroll
          for (int k = 0; k < 16; ++k) x[b][k] = (float)from[k];
        }
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) top = max(top, __builtin_bit_cast(unsigned, x[b][k]) & 0x7FFFFFFFu);
    }
    top = max(top, (unsigned)__shfl_xor((int)top, 16));
    top = max(top, (unsigned)__shfl_xor((int)top, 32));
    const bool fine = top < 0x7F800000u;
    const float step = __builtin_bit_cast(
        float, (unsigned)__builtin_bit_cast(int, fmaxf(fine ? __builtin_bit_cast(float, top) : 1.0f, kScaleFloor)) & 0x7F800000u);
    const float up = pow2_inverse(step) * 0x1p13f;
    qn[r] = fine ? step * 0x1p-13f : __builtin_nanf("");
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        float rest = fine ? x[b][k] * up : 0.0f;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          const _Float16 h = (_Float16)rest;
          q[t][r][2 * b + (k >> 3)][k & 7] = h;
          rest -= (float)h;
        }
      }
  }

  float m[RT], l[RT], R = 0.0f;
  v4f o[RT][LB];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    m[r] = kNoMax;
    l[r] = 0.0f;
#pragma unroll
    for (int c = 0; c < LB; ++c) o[r][c] = v4f{0, 0, 0, 0};
  }
  const int first_limit = a.causal ? pos0 + row0 / a.heads : s.len - 1;
  const int32_t* table = a.b.table + (int64_t)seq * a.b.table_ld;
  const int last_nth = (s.len - 1) >> p.page_log2;
  const float to_log2 = a.scale * 1.44269504088896340736f;

  // Page numbers two chunks ahead, codes and scales one.
  v4i kr[KB];
  v4f next_s, next_rs;
  int next_page = -1;
  bool next_there = false;
  auto lookup = [&](int chunk) {
    const int nth = (chunk * 64 + wave * 16) >> p.page_log2;
    next_page = nth <= last_nth ? table[nth] : -1;
  };
  auto load = [&](int chunk) {
    const int t = chunk * 64 + wave * 16;
    next_there = next_page >= 0 && next_page < a.c.pages;
    if (!next_there && t < s.len && lane == 0) raise_flag(p.flags, FXPQ_FLAG_RANGE);
    const int page = next_there ? next_page : 0, slot = t & (P - 1);
    const int8_t* base = a.c.codes + latent_offset(a.c, page, slot + n);
#pragma unroll
    for (int b = 0; b < LB; ++b) kr[b] = *reinterpret_cast<const v4i*>(base + 64 * b + 16 * g);
    kr[LB] = *reinterpret_cast<const v4i*>(base + 64 * LB + (16 * g < a.c.rope ? 16 * g : 0));
    const int64_t at = (int64_t)page * P + slot + 4 * g;
    next_s = *reinterpret_cast<const v4f*>(a.c.scale + at);
    next_rs = *reinterpret_cast<const v4f*>(a.c.rope_scale + at);
  };
  if (begin < end) {
    lookup(begin);
    load(begin);
    lookup(begin + 1);
    if (threadIdx.x < 2) raised[threadIdx.x] = 0;
    lds_barrier();
  }
  for (int chunk = begin; chunk < end; ++chunk) {
    const int buf = (chunk - begin) & 1;
    int8_t* cb = lds + buf * L::kCodes;
    int8_t* pb = lds + 2 * L::kCodes + buf * QT * L::kP;
    const bool there = next_there;
    const int t0 = chunk * 64 + wave * 16 + 4 * g;  // this lane's four tokens of S
    // scales: 0 for what is no token of the sequence (its memory may hold anything)
    float st[4], cs[4], rs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = there && t0 + i < s.len;
      st[i] = in ? next_s[i] : 0.0f;
      cs[i] = st[i] * to_log2;
      rs[i] = (in ? next_rs[i] : 0.0f) * to_log2;
    }
#pragma unroll
    for (int b = 0; b < LB; ++b) *reinterpret_cast<v4i*>(cb + (wave * 16 + n) * L::kRow + 64 * b + 16 * g) = kr[b];
    v4f sum[RT], turned[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) sum[r] = turned[r] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      v8h k[2];
      codes_to_halves(kr[b], k[0], k[1]);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            v4f& to = b < LB ? sum[r] : turned[r];
            to = mfma(k[h], q[t][r][2 * b + h], to);
          }
    }
    if (chunk + 1 < end) {
      load(chunk + 1);
      lookup(chunk + 2);
    }
    float z[RT][4];  // logits, but for the row's power of two
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) z[r][i] = fmaf(turned[r][i], rs[i], sum[r][i] * cs[i]);
    if (chunk * 64 + 63 > first_limit || !there) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + i > limit[r] || !there) z[r][i] = -INFINITY;
    }
    float add[RT], lg[4];
    auto logs = [&]() {
      const float inv = R > 0.0f ? pow2_inverse(R) : 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) lg[i] = fmaxf(__builtin_amdgcn_logf(st[i] * inv), kLeastLog);
    };
    auto weigh = [&]() {  // P of this wave's tokens to LDS
      const float lift = pow2_inverse(R) * kLift;
      float w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = st[i] * lift;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        float rest[4];
        add[r] = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(fmaf(z[r][i], qn[r], -m[r]));
          add[r] += e;
          rest[i] = e * w[i];
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          v4h h;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            h[i] = (_Float16)rest[i];
            rest[i] -= (float)h[i];
          }
          *reinterpret_cast<v4h*>(pb + t * L::kP + (r * 16 + n) * L::kPRow + wave * 32 + g * 8) = h;
        }
      }
    };
    logs();
    bool over = chunk == begin;
    if (!over) {
      bool mine = fmaxf(fmaxf(st[0], st[1]), fmaxf(st[2], st[3])) > R;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        float y = fmaf(z[r][0], qn[r], lg[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) y = fmaxf(y, fmaf(z[r][i], qn[r], lg[i]));
        mine |= y > m[r] + kSlack;
      }
      over = __any(mine);
    }
    if (over) {
      if (lane == 0) raised[buf] = chunk + 1;
    } else {
      weigh();
    }
    lds_barrier();
    if (raised[buf] == chunk + 1) {
      // new references: the scales' first, then each row's, over all waves
      float most = fmaxf(fmaxf(st[0], st[1]), fmaxf(st[2], st[3]));
      most = over_groups(most);
      if (lane == 0) scales[wave] = most;
      lds_barrier();
      most = fmaxf(fmaxf(fmaxf(scales[0], scales[1]), fmaxf(scales[2], scales[3])), 0x1p-110f);
      // the power of two above it
      most = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, most) & 0x7F800000u) + 0x00800000u);
      const float now_r = fmaxf(R, most);
      const float ratio = R > 0.0f ? R * pow2_inverse(now_r) : 1.0f;  // at most 1
      R = now_r;
      logs();
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        float y = fmaf(z[r][0], qn[r], lg[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) y = fmaxf(y, fmaf(z[r][i], qn[r], lg[i]));
        y = over_groups(y);
        if (g == 0) tops[wave * kRows + r * 16 + n] = y;
      }
      lds_barrier();
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const int at = r * 16 + n;
        const float y = fmaxf(fmaxf(tops[at], tops[kRows + at]), fmaxf(tops[2 * kRows + at], tops[3 * kRows + at]));
        // what came before weighs `ratio` of what it did against the new R
        const float before = m[r] == kNoMax ? kNoMax : m[r] + __builtin_amdgcn_logf(ratio);
        const float now = y > before + kSlack ? y : before, down = m[r] == kNoMax ? 0.0f : __builtin_amdgcn_exp2f(m[r] - now);
        m[r] = now;
        l[r] *= down;
        const float f = down * ratio;
#pragma unroll
        for (int c = 0; c < LB; ++c) o[r][c] *= f;
      }
      weigh();
      lds_barrier();
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) l[r] += add[r];
    // lane: dimensions LB n + 0 .. LB - 1 of this wave's quarter, of tokens 32 u + 8 g + 0 .. 7
    const int8_t* cw = cb + wave * (LB * 16) + LB * n;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      unsigned w[8][LB / 4];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned* from = reinterpret_cast<const unsigned*>(cw + (32 * u + 8 * g + j) * L::kRow);
        if constexpr (LB == 8) {
          const uint2 v = *reinterpret_cast<const uint2*>(from);
          w[j][0] = v.x;
          w[j][1] = v.y;
        } else {
          w[j][0] = *from;
        }
      }
      v8h pf[QT][RT];
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int r = 0; r < RT; ++r)
          pf[t][r] = *reinterpret_cast<const v8h*>(pb + t * L::kP + (r * 16 + n) * L::kPRow + u * 64 + g * 16);
#pragma unroll
      for (int c = 0; c < LB; ++c) {
        v4i f;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = pair_of(w[2 * j][c / 4], w[2 * j + 1][c / 4], c % 4);
        const v8h v = __builtin_bit_cast(v8h, f);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int r = 0; r < RT; ++r) o[r][c] = mfma(v, pf[t][r], o[r][c]);
      }
    }
  }

  // the rows' sums over lanes and waves
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
  }
  lds_barrier();
#pragma unroll
  for (int r = 0; r < RT; ++r)
    if (g == 0) tops[wave * kRows + r * 16 + n] = l[r];
  lds_barrier();
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int at = r * 16 + n, row = row0 + at;
    if (row >= rows) continue;
    const float sum = tops[at] + tops[kRows + at] + tops[2 * kRows + at] + tops[3 * kRows + at];
    const int64_t token = s.first + (int64_t)(row / a.heads);
    const int head = row % a.heads, d0 = wave * (LB * 16) + 4 * LB * g;
    const float unit = R * (1.0f / kLift);
    if (p.splits > 1) {
      const int64_t to = ((int64_t)split * a.b.tokens + token) * a.heads + head;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < LB; c += 4)
          *reinterpret_cast<v4f*>(p.part_o + to * (LB * 64) + d0 + LB * i + c) =
              v4f{o[r][c][i], o[r][c + 1][i], o[r][c + 2][i], o[r][c + 3][i]} * unit;
      if (wave == 0 && g == 0) {
        p.part_ml[2 * to] = m[r];
        p.part_ml[2 * to + 1] = sum;
      }
      continue;
    }
    const float f = sum == 0.0f ? 0.0f : unit / sum;
    T* to = static_cast<T*>(a.out) + token * a.ldo + head * a.hdo + d0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < LB; c += 4) {
        const float y[4] = {o[r][c][i] * f, o[r][c + 1][i] * f, o[r][c + 2][i] * f, o[r][c + 3][i] * f};
        if (p.vec) {
          store_reals<T, 4>(to + LB * i + c, y);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) to[LB * i + c + k] = (T)y[k];
        }
      }
  }
}

// Joins the splits of each row: one block per new token and head.
template <typename T>
__global__ __launch_bounds__(256) void k_latent_join(LatentRun p, int tile_rows) {
  constexpr int kMany = 256;  // weights kept at a time
  __shared__ float weight[kMany], red[4], sums[1024];
  const LatentArgs& a = p.a;
  const SeqDev s = seq_of(a.b, a.c.page, blockIdx.z);
  const int i = blockIdx.x, head = blockIdx.y;
  if (!s.ok || i >= s.fresh) return;
  const int row = i * a.heads + head;
  const int total = rows_chunks(p, s, row / tile_rows * tile_rows, tile_rows);
  const int used = (total + p.split_chunks - 1) / p.split_chunks;
  const int64_t token = s.first + (int64_t)i, stride = (int64_t)a.b.tokens * a.heads, at0 = token * a.heads + head;
  const int tid = threadIdx.x, lane = tid & 63;
  float mx = kNoMax;
  for (int k = tid; k < used; k += 256) mx = fmaxf(mx, p.part_ml[2 * (k * stride + at0)]);
#pragma unroll
  for (int d = 32; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
  if (lane == 0) red[tid >> 6] = mx;
  __syncthreads();
  mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const int quads = a.c.latent / 4, ways = 256 / quads, x = tid % quads, y = tid / quads;
  float sum = 0.0f;
  v4f v = {0, 0, 0, 0};
  for (int k0 = 0; k0 < used; k0 += kMany) {
    const int many = min(kMany, used - k0);
    __syncthreads();
    if (tid < many) {
      const int64_t at = (k0 + tid) * stride + at0;
      const float w = __builtin_amdgcn_exp2f(p.part_ml[2 * at] - mx);
      weight[tid] = w;
      sum += w * p.part_ml[2 * at + 1];
    }
    __syncthreads();
    for (int k = y; k < many; k += ways)
      v += weight[k] * *reinterpret_cast<const v4f*>(p.part_o + ((k0 + k) * stride + at0) * a.c.latent + 4 * x);
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
  T* to = static_cast<T*>(a.out) + token * a.ldo + head * a.hdo + 4 * x;
#pragma unroll
  for (int k = 0; k < 4; ++k) to[k] = (T)(v[k] * f);
}

struct LatentPlan {
  int rt, row_tiles, splits, split_chunks;
  int64_t part, bytes;
};

LatentPlan plan_latent(const Ctx& c, const fxpq_latent_cache& k, const fxpq_kv_batch& b, int heads, int type) {
  LatentPlan p{};
  const int64_t rows = (int64_t)b.max_new * heads;
  p.rt = rows <= 16 || type == FXPQ_F32 ? 1 : 2;
  p.row_tiles = (int)((rows + p.rt * 16 - 1) / (p.rt * 16));
  const int64_t blocks = (int64_t)p.row_tiles * b.seqs, chunks = (b.max_len + 63) / 64;
  const int64_t slots = (int64_t)c.cus * (p.rt == 1 ? 2 : 1);
  int64_t per = (blocks * chunks + slots - 1) / slots;
  per = per < 4 ? 4 : per > 32 && blocks < 4 * slots ? 32 : per;
  if (blocks >= 4 * slots) per = chunks;
  p.split_chunks = (int)(per < 1 ? 1 : per);
  p.splits = (int)((chunks + p.split_chunks - 1) / p.split_chunks);
  if (p.splits > 1) {
    p.part = (int64_t)p.splits * b.tokens * heads;
    p.bytes = p.part * (k.latent + 2) * 4;
  } else {
    p.splits = 1;
  }
  return p;
}

template <typename T, int LB, int RT>
hipError_t run_latent(const Ctx& c, const LatentRun& p) {
  constexpr int bytes = LatentLds<LB, RT, sizeof(T) == 4 ? 2 : 1>::kBytes;
  auto* f = k_latent_attention<T, LB, RT>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(f), bytes);
  if (e != hipSuccess) return e;
  const int64_t blocks = ((int64_t)p.a.b.seqs * p.splits + 7) / 8 * 8 * p.row_tiles;
  if (blocks > kMaxBlocks) return hipErrorInvalidValue;
  f<<<dim3((unsigned)blocks), dim3(256), bytes, c.stream>>>(p);
  if (p.splits > 1)
    k_latent_join<T><<<dim3((unsigned)p.a.b.max_new, (unsigned)p.a.heads, (unsigned)p.a.b.seqs), dim3(256), 0,
                       c.stream>>>(p, RT * 16);
  return hipGetLastError();
}

template <typename T, int LB>
hipError_t run_rows(const Ctx& c, const LatentRun& p, int rt) {
  if constexpr (sizeof(T) == 2)
    if (rt == 2) return run_latent<T, LB, 2>(c, p);
  return run_latent<T, LB, 1>(c, p);
}

}  // namespace

int64_t latent_attention_workspace(const Ctx& c, const fxpq_latent_cache& cache, const fxpq_kv_batch& b, int heads) {
  const int64_t wide = plan_latent(c, cache, b, heads, FXPQ_F32).bytes;
  const int64_t narrow = plan_latent(c, cache, b, heads, FXPQ_BF16).bytes;
  return wide > narrow ? wide : narrow;  // whatever the type of the call
}

hipError_t launch_latent_attention(const Ctx& c, const LatentArgs& a, int type, void* ws) {
  const LatentPlan plan = plan_latent(c, a.c, a.b, a.heads, type);
  LatentRun p{};
  p.a = a;
  p.row_tiles = plan.row_tiles;
  p.splits = plan.splits;
  p.split_chunks = plan.split_chunks;
  while ((1 << p.page_log2) < a.c.page) ++p.page_log2;
  const int64_t size = real_bytes(type);
  const auto fits = [&](const void* at, int64_t ld, int64_t hd) {
    return (uintptr_t)at % 16 == 0 && ld * size % 16 == 0 && hd * size % 16 == 0;
  };
  p.vec = fits(a.q, a.ldq, a.hdq) && fits(a.qr, a.ldqr, a.hdqr) && fits(a.out, a.ldo, a.hdo);
  p.part_o = static_cast<float*>(ws);
  p.part_ml = p.part_o ? p.part_o + plan.part * a.c.latent : nullptr;
  p.flags = c.sc.flags;
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    return a.c.latent == 512 ? run_rows<T, 8>(c, p, plan.rt) : run_rows<T, 4>(c, p, plan.rt);
  });
}

}  // namespace fxpq
