// Absorbed attention over the paged 8-bit cache of latents: one row of codes a token
// is key and value of every head.
//
// A sequence's query rows are its new tokens' heads (row = token * heads + head); a
// block takes 16 RT of them over a part of the sequence's cache, 64 tokens (a chunk) at a
// time.  Chunks come straight from memory into a ring of two or three LDS slots.  First
// product, S = K Q^T: a wave has 16 of the tokens; it reads their codes from LDS in the
// operand's layout (lane: token lane % 16, 16 codes from 16 (lane / 16)), converts them to
// f16 (exact) and multiplies them with q in registers.  (Products with 1152 + code, whose
// sums start from what that adds, would spare an operation for every two codes, 32 x 1 over
// 4096, 128 heads in 69 us in place of 76; but where a few channels take the scale and leave
// the other codes at some steps, such sums leave logits off by 0.05.)  q is f16 too: scaled
// by a power of two of its row, so that a bf16 or f16 value is exact down to 2^-27 of the
// row's largest, and f32 is two f16 terms.  P goes to LDS as f16 (f32: two terms) and after a
// barrier every wave multiplies all 64 tokens with its own part of the latent's dimensions:
// O^T = C^T P^T.  The conversion there is the transposition: a lane reads the same 2 to 8
// dimensions of 8 tokens and pairs bytes of neighbouring tokens.
//
// One f16 term of P rounds a weight by 2^-11 at most, a quarter of bf16's own rounding.  An f16
// result's rounding is as large: where many weights are alike the error is up to 1.4 times that
// alone.  A second term would need the LDS of the second block of a CU: 64 x 1 over 8192, 16
// heads, 91 us in place of 76, 32 x 1 over 4096, 128 heads, 115 in place of 100.
//
// A token's scale s_t belongs to both products.  With x_t the logit (base 2), m the
// row's reference and R a power of two above every scale seen, P_t = 2^(x_t - m) s_t / R
// goes into O and 2^(x_t - m) into the sum.  m follows max (x_t + log2(s_t / R)) only
// when a row passes it by more than kSlack, so P_t is below 2^(kSlack + kLift) and most
// chunks need neither a maximum across the waves nor further barriers.
//
// What it costs (latents of 512 + 64, bf16): a block's start about 8 us (its part, pages, q to
// f16); a chunk 1.8 us with four waves and one row tile, two blocks a CU (64 x 1 over 4096 and
// 8192, 16 heads, 46 and 75 us), 2.1 us with eight waves and two tiles (32 x 1 over 2048 and 4096,
// 128 heads, 65 and 99).  The bytes are not the limit but the conversions: 128 heads, 32
// sequences up to 4096: vector instructions 56% of the cycles, matrix instructions 15%, the
// rest waits at the chunk's two barriers, which one block a CU does not fill.  64 x 1 over up
// to 8192, 16 heads: 158 MB in 41.5 us, 3.8 TB/s; 32 x 1 over up to 4096, 128 heads: 74 us,
// 0.25 PFLOP/s; the join 6 us more in both.
#include "kv.hpp"
#include "ring.hpp"
#include "values.hpp"

namespace fxpq {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// How the work is split.  shared: each sequence's chunks are cut into equal parts of at
// most `share` chunks (`least` or more), a block for each part and row tile; `groups` parts
// run at a time and there are blocks for `rounds` times as many.  Parts of a sequence are
// joined afterwards.  Otherwise a block takes a row tile of a sequence whole.
struct LatentRun {
  LatentArgs a;
  int row_tiles, shared, groups, rounds, least, page_log2, vec;
  unsigned heads_mul;  // row / heads = row * heads_mul >> heads_shift, for rows below 2^30
  int heads_shift;
  float* part_o;   // [groups * rounds][row_tiles][rows of a tile][latent]
  float* part_ml;  // [groups * rounds][row_tiles][rows of a tile][2]: reference and sum
  int* line;       // [seqs] each sequence's first part; [seqs]: the share
  unsigned* flags;
};
__device__ inline int token_of(const LatentRun& p, int row) {
  return (int)((uint64_t)(unsigned)row * p.heads_mul >> p.heads_shift);
}
// ceil(n / d), n below 2^24, by d's reciprocal.
__device__ inline int quotient_up(int n, int d, float inv) {
  const int q = (int)((float)n * inv);  // off by one at most
  return q + (q * d < n ? 1 : 0) - ((q - 1) * d >= n ? 1 : 0);
}
// Chunks of each of a sequence's parts, of which there are ceil(chunks / share).
__device__ inline int part_chunks(int chunks, int share) {
  const int parts = (chunks + share - 1) / share;
  return parts == 0 ? 1 : (chunks + parts - 1) / parts;
}
// Sequences of a call that is shared, four a lane.  (With 512 every call's start takes up to 1 us
// more; 400 x 1, 16 heads, over 1 to 4096 144 us in place of 166, 32 heads over 1024 159 of 105.)
constexpr int kMostSeqs = 256;

constexpr float kNoMax = -3.40282347e38f;  // reference before any token
constexpr float kSlack = 8.0f;
// P is written as f16: 2^kLift at the reference, so that weights down to 2^-20 of the
// largest keep all 11 bits and smaller ones lose at most 2^-31 of it.
constexpr float kLift = 64.0f;
constexpr float kLeastLog = -50.0f;  // of s_t / R, where it only moves the reference
// A reference follows a growing R down until the sum of its row is 2^kMostSum.  2^30 tokens add
// at most 2^(30 + kSlack - kLeastLog) to it.
constexpr float kMostSum = 96.0f;
constexpr float kFar = 0x1p24f;  // logits past this have steps above 1: s_t / R would be rounded

__device__ inline void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4));  // LDS operations only
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Byte u = code + 128 below the exponent of 1024 is 1024 + u, and 1024 + u - 1152 the
// code, exactly.
__device__ inline unsigned unbiased(unsigned biased) {
  const v2h off = {(_Float16)1152.0f, (_Float16)1152.0f};
  return __builtin_bit_cast(unsigned, __builtin_bit_cast(v2h, biased) - off);
}
// 16 codes as two operands of 8.
__device__ inline void codes_to_halves(v4i w, v8h& lo, v8h& hi) {
  v4i r[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned u = (unsigned)w[i] ^ 0x80808080u;
    r[i >> 1][2 * (i & 1)] = (int)unbiased(__builtin_amdgcn_perm(0x64646464u, u, 0x04010400u));
    r[i >> 1][2 * (i & 1) + 1] = (int)unbiased(__builtin_amdgcn_perm(0x64646464u, u, 0x04030402u));
  }
  lo = __builtin_bit_cast(v8h, r[0]);
  hi = __builtin_bit_cast(v8h, r[1]);
}
// Byte `at` of two tokens' words as a pair of halves.
__device__ inline int pair_of(unsigned first, unsigned second, int at) {
  return (int)unbiased(__builtin_amdgcn_perm(second, first, 0x0C040C00u + (unsigned)at * 0x00010001u) ^ 0x64806480u);
}

__device__ inline v4f mfma(v8h a, v8h b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Another lane of the 16 of a row, and a wave's sum and running sum.
template <int CTRL>
__device__ inline int lanes(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true); }
__device__ inline int running_sum(int v, int lane, int& all) {
  v += lanes<0x111>(v);  // from 1, 2, 4 and 8 lanes below, in the row
  v += lanes<0x112>(v);
  v += lanes<0x114>(v);
  v += lanes<0x118>(v);
  const int a = __builtin_amdgcn_readlane(v, 15), b = __builtin_amdgcn_readlane(v, 31), c = __builtin_amdgcn_readlane(v, 47);
  all = a + b + c + __builtin_amdgcn_readlane(v, 63);
  return v + (lane < 16 ? 0 : lane < 32 ? a : lane < 48 ? a + b : a + b + c);
}

// 64-token chunks that rows row0 .. row0 + rows - 1 of a sequence see.
__device__ inline int rows_chunks(const LatentRun& p, const SeqDev& s, int row0, int rows) {
  const int last = min(row0 + rows, s.fresh * p.a.heads) - 1;
  if (last < row0) return 0;
  const int limit = p.a.causal ? s.len - s.fresh + token_of(p, last) : s.len - 1;
  return (limit + 64) >> 6;
}

// The maximum over the four 16-lane groups of a wave, lane by lane.
__device__ inline float over_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// A group of 16 tokens of a chunk in LDS: rows of LB * 4 + 4 pieces of 16 bytes.  A latent's
// piece c of token t sits at c ^ (t / 4), so that reads of one piece of 16 tokens cover all
// banks; the shared key's pieces follow in order.
template <int LB, int RT, int QT>
struct LatentLds {
  static constexpr int kPieces = LB * 4 + 4, kRow = kPieces * 16;
  static constexpr int kLoads = kPieces * 16 / 64;  // 1 KB loads of a group
  static constexpr int kGroup = 16 * kRow, kSlot = 4 * kGroup;
  // one tile of a wide latent: two slots, so that two blocks fit a CU (64 x 1 over 8192, 16
  // heads: 75 us; three slots and one block 85; 1 x 1 over 131072: 33.6 and 33.1)
  static constexpr int kSlots = LB == 8 && RT * QT == 1 ? 2 : 3;
  static constexpr int kScales = kSlots * kSlot;              // [slots][4 groups][64] floats
  static constexpr int kPRow = 144;                           // bytes of a row of P: 64 halves and a pad
  static constexpr int kP = RT * 16 * kPRow;
  static constexpr int kWeights = kScales + kSlots * 4 * 256;  // [2][QT] P
  static constexpr int kStats = kWeights + 2 * QT * kP;
  static constexpr int kBytes = kStats + 2 * 4 * RT * 16 * 4 + 64;
  // q as f16 lies in the slots behind the first until the waves have taken it
  static constexpr int kQRow = (LB * 64 + 64) * 2, kQ = RT * 16 * kQRow;
  static_assert(QT * kQ <= (kSlots - 1) * kSlot, "q fits");
};

// LB: 64-dimension pieces of the latent; RT: 16-row tiles of a block; W: waves.  Four waves:
// each has one group of 16 tokens in the first product and a quarter of the latent's
// dimensions in the second.  Eight: two share a group of tokens and have half of the rows
// each, and an eighth of the dimensions, which halves what a wave holds of q and O.
template <typename T, int LB, int RT, int W>
__global__ __launch_bounds__(W * 64, W == 8 || (RT == 1 && sizeof(T) == 2) ? 2 : 1) void k_latent_attention(const LatentRun p) {
  constexpr int QT = sizeof(T) == 4 ? 2 : 1;  // f16 terms of q and of P
  constexpr int KB = LB + 1;                  // 64-byte pieces of a token: the latent's, the key's
  constexpr int kRows = RT * 16, D = LB * 64, kThreads = W * 64;
  constexpr int H = W / 4, QR = RT / H;  // row tiles of a wave in the first product
  constexpr int CB = LB / H;             // 16-dimension tiles of a wave in the second
  typedef LatentLds<LB, RT, QT> L;
  // loads of a wave: with eight, the first four waves have the first half of each group
  constexpr int kHalf = (L::kLoads + H - 1) / H, kWaveLoads = W == 8 ? kHalf : L::kLoads + 1;
  static_assert(W == 4 || L::kLoads - kHalf + 1 == kHalf, "both halves wait for as many loads");
  extern __shared__ __attribute__((aligned(256))) int8_t lds[];
  float* tops = reinterpret_cast<float*>(lds + L::kStats);          // [4][kRows]
  float* sums = tops + 4 * kRows;                                   // [4][kRows]
  float* scales = sums + 4 * kRows;                                 // [4]
  volatile int* raised = reinterpret_cast<volatile int*>(scales + 4);  // [2]: chunk + 1 of the last that passed its reference
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tg = wave & 3, half = W == 8 ? wave >> 2 : 0;
  const int heads = p.a.heads, causal = p.a.causal, rope = p.a.c.rope, pages = p.a.c.pages, page_log2 = p.page_log2;
  const int P = 1 << page_log2, seqs = p.a.b.seqs;
  const int8_t* codes = p.a.c.codes;
  const float* latent_scale = p.a.c.scale;
  const float* key_scale = p.a.c.rope_scale;
  unsigned* flags = p.flags;
  // The softmax's scale in two factors: its power of two goes to the rows with q's, the rest
  // and q's 2^13 to the tokens.  Products of either with what it meets stay in fp32's range
  // wherever the logits do, whichever of q, cache and scale is large.
  const float unit = fminf(fmaxf(__builtin_bit_cast(float, __builtin_bit_cast(unsigned, p.a.scale) & 0x7F800000u), 0x1p-126f), 0x1p126f);
  const float to_log2 = p.a.scale * pow2_inverse(unit) * (1.44269504088896340736f * 0x1p-13f);

  // Row tiles of one part of a cache are 8 ids apart: on one XCD, whose L2 they share.
  const unsigned oct = blockIdx.x / 8;
  const int group = (int)(oct / (unsigned)p.row_tiles * 8 + blockIdx.x % 8);
  const int tile = p.row_tiles - 1 - (int)(oct % (unsigned)p.row_tiles);  // the last rows see the most tokens
  if (group >= p.groups * p.rounds) return;

  // This lane's 16 bytes of each load of a group, whose tokens lie one after another in
  // their page.
  constexpr int kMine = W == 8 ? kHalf : L::kLoads;
  uint32_t from[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int at = (i + half * kHalf) * 64 + lane, t = (at / L::kPieces) & 15, c = at % L::kPieces;
    const int piece = c < LB * 4 ? c ^ (t >> 2) : c - LB * 4 < rope / 16 ? c : LB * 4;
    from[i] = (uint32_t)(t * (D + rope) + piece * 16);
  }

  const int part = group;
  int seq = part, begin = 0, size = 0;
  SeqDev s;
  if (p.shared) {
    // Every wave finds the share and the part's sequence by itself, up to four sequences a
    // lane: nothing has to run before this kernel, and lengths stay on the device.
    constexpr int kOwn = kMostSeqs / 64;
    SeqDev d[kOwn];
    int count[kOwn], all = 0;
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
      const int i = lane + 64 * e;
      count[e] = 0;
      d[e] = SeqDev{0, 0, 0, false};
      if (64 * e < seqs) {
        d[e] = seq_of(p.a.b, P, min(i, seqs - 1));
        if (!d[e].ok && blockIdx.x == 0) raise_flag(flags, FXPQ_FLAG_RANGE);
        if (i < seqs && d[e].ok) count[e] = rows_chunks(p, d[e], 0, d[e].fresh * heads);
        int sum;
        running_sum(count[e], lane, sum);
        all += sum;
      }
    }
    int parts, before[kOwn];
    auto cut = [&](int share) __attribute__((always_inline)) {
      const float inv = 1.0f / (float)share;
      parts = 0;
#pragma unroll
      for (int e = 0; e < kOwn; ++e)
        if (64 * e < seqs) {
          const int mine = quotient_up(count[e], share, inv);
          int sum;
          before[e] = parts + running_sum(mine, lane, sum) - mine;
          parts += sum;
        }
    };
    const int most = p.groups * p.rounds;
    int share;
    if (p.rounds == 1) {
      // the smallest share that leaves no more parts than run at a time (at the latest
      // where no sequence has two)
      for (share = max((all + most - 1) / most, p.least);; share += 1 + share / 16) {
        cut(share);
        if (parts <= most) break;
      }
    } else {
      // sequences no longer than the mean stay whole, or nearly: all / share + active parts
      // at most, and no share above the longest
      int active = 0, top = 0;
#pragma unroll
      for (int e = 0; e < kOwn; ++e) {
        active += __popcll(__ballot(count[e] > 0));
        top = max(top, count[e]);
      }
      top = max(top, lanes<0xB1>(top));
      top = max(top, lanes<0x4E>(top));
      top = max(top, lanes<0x141>(top));
      top = max(top, lanes<0x140>(top));
      top = max(max(__builtin_amdgcn_readlane(top, 0), __builtin_amdgcn_readlane(top, 16)),
                max(__builtin_amdgcn_readlane(top, 32), __builtin_amdgcn_readlane(top, 48)));
      share = max(min((all + most - active - 1) / (most - active), top), p.least);
      cut(share);
    }
    if (part >= parts) return;
    // the last sequence whose first part is this or an earlier one (those without parts
    // start where the next does)
    seq = -1;
#pragma unroll
    for (int e = 0; e < kOwn; ++e)
      if (64 * e < seqs) {
        const int i = lane + 64 * e;
        seq += __popcll(__ballot(i < seqs && before[e] <= part));
        if (blockIdx.x == 0 && wave == 0 && i < seqs) p.line[i] = before[e];
      }
    if (blockIdx.x == 0 && threadIdx.x == 0) p.line[seqs] = share;
    int chunks = 0, first = 0;
#pragma unroll
    for (int e = 0; e < kOwn; ++e)
      if (seq >> 6 == e) {
        const int at = seq & 63;
        s = SeqDev{__builtin_amdgcn_readlane(d[e].first, at), __builtin_amdgcn_readlane(d[e].fresh, at),
                   __builtin_amdgcn_readlane(d[e].len, at), true};
        chunks = __builtin_amdgcn_readlane(count[e], at);
        first = __builtin_amdgcn_readlane(before[e], at);
      }
    size = part_chunks(chunks, share);
    begin = (part - first) * size;
  } else {
    s = block_seq(seq_of(p.a.b, P, seq));
    if (!s.ok && tile == 0 && threadIdx.x == 0) raise_flag(flags, FXPQ_FLAG_RANGE);
  }
  const int row0 = tile * kRows, rows = s.ok ? s.fresh * heads : 0;
  const int total = row0 < rows ? rows_chunks(p, s, row0, kRows) : 0;  // this tile's
  const int end = p.shared ? min(begin + size, total) : total;
  if (begin >= end) return;
  const int pos0 = s.len - s.fresh;
  // read by scalar loads: they are not counted among the loads to LDS
  const auto* table = (const __attribute__((address_space(4))) int32_t*)(p.a.b.table + (int64_t)seq * p.a.b.table_ld);
  const int last_nth = (s.len - 1) >> page_log2;

  // Page of this wave's tokens of a chunk; past the sequence's end -1.
  auto page_of = [&](int chunk) __attribute__((always_inline)) {
    const int nth = (chunk * 64 + tg * 16) >> page_log2;
    return nth <= last_nth ? table[nth] : -1;
  };
  auto load = [&](int chunk, int slot, int page) __attribute__((always_inline)) {
    const int t = chunk * 64 + tg * 16;
    const bool there = page >= 0 && page < pages;
    if (!there && t < s.len && lane == 0) raise_flag(flags, FXPQ_FLAG_RANGE);
    const int64_t first = ((int64_t)(there ? page : 0) << page_log2) + (t & (P - 1));
    const int8_t* base = codes + first * (D + rope);
    int8_t* into = lds + slot * L::kSlot + tg * L::kGroup;
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      if (i + 1 < kMine || half == 0) dma16(base, from[i], into + (i + half * kHalf) * 1024);
    if (W == 4 || half == 1)
      dma4((g & 1 ? key_scale : latent_scale) + first + n, lds + L::kScales + (slot * 4 + tg) * 256);
  };
  // q as it is to LDS, its loads before the first chunk's
  int8_t* ql = lds + L::kSlot;
  constexpr int kQPieces = (D + 64) * (int)sizeof(T) / 16, kQAll = kRows * kQPieces;
  int page = page_of(begin), page1 = page_of(begin + 1), page2 = page_of(begin + 2);
  if (p.vec) {
#pragma unroll 1
    for (int i = wave * 64; i < kQAll; i += kThreads) {
      const int at = i + lane, r = at / kQPieces, piece = at % kQPieces * (16 / (int)sizeof(T));  // first of 4 or 8 reals
      const int row = min(row0 + r, rows - 1);  // rows behind the last: any
      const int i_token = token_of(p, row);
      const int64_t token = s.first + (int64_t)i_token, head = row - i_token * heads;
      const T* src = piece < D ? static_cast<const T*>(p.a.q) + token * p.a.ldq + head * p.a.hdq + piece
                               : static_cast<const T*>(p.a.qr) + token * p.a.ldqr + head * p.a.hdqr + (piece - D < rope ? piece - D : 0);
      if (at < kQAll) dma16(reinterpret_cast<const int8_t*>(src), ql + i * 16);
    }
  }
  load(begin, 0, page);
  if (p.vec) wait_vmcnt<kWaveLoads>();
  lds_barrier();

  // q to f16, 16 threads a row, scaled by a power of two; the waves take their operands
  // from LDS then.  rowq: the row's power of two (with the softmax scale's), NaN where it holds a NaN or an infinity.
  float* rowq = tops;
  {
    const int sub = threadIdx.x & 15;
    constexpr int V = 16 / sizeof(T), N = LB * 4 / V;  // LB * 4 latent reals and 4 of the key a thread
    static_assert(sizeof(T) == 2 || kRows * 16 == kThreads, "f32 rows are read before any is written");
#pragma unroll 1
    for (int r = threadIdx.x >> 4; r < kRows; r += kThreads / 16) {
      const int row = row0 + r;
      const bool real = row < rows;
      float x[LB * 4 + 4];
      if (p.vec) {
        const T* raw = reinterpret_cast<const T*>(ql) + r * (D + 64);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          float u[V];
          load_reals<T, V>(raw + (k * 16 + sub) * V, u);
#pragma unroll
          for (int j = 0; j < V; ++j) x[k * V + j] = u[j];
        }
        float u[4];
        load_reals<T, 4>(raw + D + 4 * sub, u);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[LB * 4 + j] = 4 * sub < rope ? u[j] : 0.0f;
      } else {
        const int i_token = real ? token_of(p, row) : 0;
        const int64_t token = s.first + (int64_t)i_token, head = real ? row - i_token * heads : 0;
        const T* ql_from = static_cast<const T*>(p.a.q) + token * p.a.ldq + head * p.a.hdq;
        const T* qr_from = static_cast<const T*>(p.a.qr) + token * p.a.ldqr + head * p.a.hdqr;
#pragma unroll
        for (int k = 0; k < LB * 4; ++k) x[k] = (float)ql_from[(k / V * 16 + sub) * V + k % V];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[LB * 4 + j] = 4 * sub < rope ? (float)qr_from[4 * sub + j] : 0.0f;
      }
      unsigned top = 0;
#pragma unroll
      for (int k = 0; k < LB * 4 + 4; ++k) {
        if (!real) x[k] = 0.0f;
        top = max(top, __builtin_bit_cast(unsigned, x[k]) & 0x7FFFFFFFu);
      }
      // (the bits of magnitudes are ordered as integers, NaN above infinity)
      top = max(top, (unsigned)lanes<0xB1>((int)top));
      top = max(top, (unsigned)lanes<0x4E>((int)top));
      top = max(top, (unsigned)lanes<0x141>((int)top));
      top = max(top, (unsigned)lanes<0x140>((int)top));
      const bool fine = top < 0x7F800000u;
      // 2^126 at most, whose inverse is a normal number: q stays below 2^15, which f16 holds
      const float step = fminf(0x1p126f, __builtin_bit_cast(
          float, __builtin_bit_cast(unsigned, fmaxf(fine ? __builtin_bit_cast(float, top) : 1.0f, kScaleFloor)) & 0x7F800000u));
      const float up = pow2_inverse(step) * 0x1p13f;
#pragma unroll
      for (int k = 0; k < LB * 4 + 4; ++k) x[k] = fine ? x[k] * up : 0.0f;
      if constexpr (sizeof(T) == 4) lds_barrier();
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        int8_t* to_lds = ql + t * L::kQ + r * L::kQRow;
#pragma unroll
        for (int k = 0; k < N + 1; ++k) {
          const int w = k < N ? V : 4, d = k < N ? (k * 16 + sub) * V : D + 4 * sub;
#pragma unroll
          for (int j = 0; j < w; j += 4) {
            v4h y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              y[e] = (_Float16)x[k * V + j + e];
              x[k * V + j + e] -= (float)y[e];
            }
            *reinterpret_cast<v4h*>(to_lds + (d + j) * 2) = y;
          }
        }
      }
      if (sub == 0) rowq[r] = fine ? fminf(fmaxf(step * unit, 0x1p-149f), 0x1p127f) : __builtin_nanf("");
    }
  }
  if (threadIdx.x < 2) raised[threadIdx.x] = 0;
  lds_barrier();
  v8h q[QT][QR][2 * KB];  // lane: row n of tile r, dimensions 64 b + 16 g + 8 h + 0..7 at 2 b + h
  float qn[QR];
  int limit[QR];
#pragma unroll
  for (int r = 0; r < QR; ++r) {
    const int row = (half * QR + r) * 16 + n;
    limit[r] = causal ? pos0 + token_of(p, row0 + row) : s.len - 1;
    qn[r] = rowq[row];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int b = 0; b < 2 * KB; ++b)
        q[t][r][b] = *reinterpret_cast<const v8h*>(lds + L::kSlot + t * L::kQ + row * L::kQRow +
                                                   (64 * (b >> 1) + 16 * g + 8 * (b & 1)) * 2);
  }
  lds_barrier();
  if (L::kSlots == 3 && begin + 1 < end) load(begin + 1, 1, page1);

  // references of all rows of the block, the same in all waves; sums of this wave's own
  float m[RT], l[QR], R = 0.0f;
  v4f o[RT][CB];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    m[r] = kNoMax;
#pragma unroll
    for (int c = 0; c < CB; ++c) o[r][c] = v4f{0, 0, 0, 0};
  }
#pragma unroll
  for (int r = 0; r < QR; ++r) l[r] = 0.0f;
  auto mine = [&](int r) __attribute__((always_inline)) { return half ? m[(H - 1) * QR + r] : m[r]; };
  const int first_limit = causal ? pos0 + token_of(p, row0) : s.len - 1;
  int slot = 0;
#pragma unroll 1
  for (int chunk = begin; chunk < end; ++chunk) {
    const int buf = (chunk - begin) & 1;
    int8_t* pb = lds + L::kWeights + buf * QT * L::kP;
    const bool there = page >= 0 && page < pages;
    // this wave's loads have landed; the next chunk's may be on their way
    if (L::kSlots == 3 && chunk + 1 < end) wait_vmcnt<kWaveLoads>();
    else wait_vmcnt<0>();
    if constexpr (W == 8) lds_barrier();  // and the other half of its tokens
    else asm volatile("" ::: "memory");
    const int8_t* own = lds + slot * L::kSlot + tg * L::kGroup;
    const int t0 = chunk * 64 + tg * 16 + 4 * g;  // this lane's four tokens of S
    float st[4], cs[4], rs[4];
    {
      const float* sc = reinterpret_cast<const float*>(lds + L::kScales + (slot * 4 + tg) * 256) + 4 * g;
      v4f a = *reinterpret_cast<const v4f*>(sc), b = *reinterpret_cast<const v4f*>(sc + 16);
      if (!there || chunk * 64 + 64 > s.len) {
        // scales: 0 for what is no token of the sequence (its memory may hold anything)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool in = there && t0 + i < s.len;
          a[i] = in ? a[i] : 0.0f;
          b[i] = in ? b[i] : 0.0f;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        st[i] = a[i];
        cs[i] = a[i] * to_log2;
        rs[i] = b[i] * to_log2;
      }
    }
    // all operands first: one wait for LDS
    v4i raw[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b)
      raw[b] = *reinterpret_cast<const v4i*>(own + n * L::kRow + (b < LB ? (4 * b + g) ^ (n >> 2) : LB * 4 + g) * 16);
    __builtin_amdgcn_sched_barrier(0);
    // two sums for the latent, so that a product need not wait for the last
    v4f part[2][QR], turned[QR];
#pragma unroll
    for (int r = 0; r < QR; ++r) part[0][r] = part[1][r] = turned[r] = v4f{0, 0, 0, 0};
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      v8h k[2];
      codes_to_halves(raw[b], k[0], k[1]);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int r = 0; r < QR; ++r) {
            v4f& acc = b < LB ? part[h][r] : turned[r];
            acc = mfma(k[h], q[t][r][2 * b + h], acc);
          }
    }
    v4f sum[QR];
#pragma unroll
    for (int r = 0; r < QR; ++r) sum[r] = part[0][r] + part[1][r];
    float z[QR][4];  // logits, but for the row's power of two
#pragma unroll
    for (int r = 0; r < QR; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) z[r][i] = fmaf(turned[r][i], rs[i], sum[r][i] * cs[i]);
    if (chunk * 64 + 63 > first_limit || !there) {
#pragma unroll
      for (int r = 0; r < QR; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + i > limit[r] || !there) z[r][i] = -INFINITY;
    }
    float add[QR], lg[4];
    auto logs = [&]() __attribute__((always_inline)) {
      const float inv = R > 0.0f ? pow2_inverse(R) : 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) lg[i] = fmaxf(__builtin_amdgcn_logf(st[i] * inv), kLeastLog);
    };
    auto top_of = [&](int r) __attribute__((always_inline)) {  // this lane's largest logit with s_t / R
      float y = fmaf(z[r][0], qn[r], lg[0]);
#pragma unroll
      for (int i = 1; i < 4; ++i) y = fmaxf(y, fmaf(z[r][i], qn[r], lg[i]));
      return y;
    };
    auto is_far = [](float y) __attribute__((always_inline)) { return fabsf(y) > kFar && y != -INFINITY; };
    auto weigh = [&]() __attribute__((always_inline)) {  // P of this wave's tokens and rows to LDS
      const float lift = pow2_inverse(R) * kLift;
      float w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = st[i] * lift;
#pragma unroll
      for (int r = 0; r < QR; ++r) {
        float rest[4];
        add[r] = 0.0f;
        const float ref = -mine(r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(fmaf(z[r][i], qn[r], ref));
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
          *reinterpret_cast<v4h*>(pb + t * L::kP + ((half * QR + r) * 16 + n) * L::kPRow + tg * 32 + g * 8) = h;
        }
      }
    };
    logs();
    bool over = chunk == begin;
    if (!over) {
      bool some = fmaxf(fmaxf(st[0], st[1]), fmaxf(st[2], st[3])) > R;
#pragma unroll
      for (int r = 0; r < QR; ++r) {
        const float y = top_of(r);
        some |= y > mine(r) + kSlack || is_far(y);
      }
      over = __any(some);
    }
    if (over) {
      if (lane == 0) raised[buf] = chunk + 1;
    } else {
      weigh();
    }
    lds_barrier();
    if (raised[buf] == chunk + 1) {
      // new references: the scales' first, then each row's, over all groups of tokens
      float most = fmaxf(fmaxf(st[0], st[1]), fmaxf(st[2], st[3]));
      most = over_groups(most);
      if (lane == 0) scales[tg] = most;
      lds_barrier();
      most = fmaxf(fmaxf(fmaxf(scales[0], scales[1]), fmaxf(scales[2], scales[3])), 0x1p-110f);
      // the power of two above it
      most = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, most) & 0x7F800000u) + 0x00800000u);
      const float now_r = fmaxf(R, most);
      // what came before has 2^fall of the weight that it had against the old R
      const int fall = R > 0.0f ? (int)(__builtin_bit_cast(unsigned, R) >> 23) - (int)(__builtin_bit_cast(unsigned, now_r) >> 23) : 0;
      R = now_r;
      // past kFar s_t / R (below 1) is left out of references: a logit's rounding would move it
      // by more than they may be off
      logs();
      bool far = false;
#pragma unroll
      for (int r = 0; r < QR; ++r) far |= is_far(top_of(r));
      if (__any(far)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) lg[i] = 0.0f;
      }
#pragma unroll
      for (int r = 0; r < QR; ++r) {
        const float y = over_groups(top_of(r));
        float sum = l[r];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (g == 0) {
          tops[tg * kRows + (half * QR + r) * 16 + n] = y;
          sums[tg * kRows + (half * QR + r) * 16 + n] = sum;
        }
      }
      lds_barrier();
      float down[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const int row = r * 16 + n;
        const float top = fmaxf(fmaxf(tops[row], tops[kRows + row]), fmaxf(tops[2 * kRows + row], tops[3 * kRows + row]));
        const float sum = sums[row] + sums[kRows + row] + sums[2 * kRows + row] + sums[3 * kRows + row];
        const float lower = fmaxf((float)fall, fminf(__builtin_amdgcn_logf(sum) - kMostSum, 0.0f));
        const float before = m[r] == kNoMax ? kNoMax : m[r] + lower;
        const float now = top > before + kSlack ? top : before;
        down[r] = m[r] == kNoMax ? 0.0f : __builtin_amdgcn_exp2f(m[r] - now);
        m[r] = now;
        const float f = __builtin_amdgcn_ldexpf(down[r], fall);
#pragma unroll
        for (int c = 0; c < CB; ++c) o[r][c] *= f;
      }
#pragma unroll
      for (int r = 0; r < QR; ++r) l[r] *= half ? down[(H - 1) * QR + r] : down[r];
      weigh();
      lds_barrier();
    }
#pragma unroll
    for (int r = 0; r < QR; ++r) l[r] += add[r];
    // all waves have left the chunk before: its slot takes the next but one, or of two
    // slots the next
    constexpr int kAhead = L::kSlots - 1;
    if (chunk + kAhead < end) load(chunk + kAhead, slot == 0 ? kAhead : slot - 1, kAhead == 2 ? page2 : page1);
    page = page1;
    page1 = page2;
    page2 = page_of(chunk + 3);
    // lane: dimensions CB n + 0 .. CB - 1 of this wave's part, of tokens 32 u + 8 g + 0 .. 7
    const int8_t* all = lds + slot * L::kSlot;
    unsigned w[2][8][(CB + 3) / 4];
    v8h pf[2][QT][RT];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // token 8 (g % 2) + j of group 2 u + g / 2
        const int byte = wave * CB * 16 + CB * n, piece = (byte >> 4) ^ (2 * (g & 1) + (j >> 2));
        const int8_t* src = all + (2 * u + (g >> 1)) * L::kGroup + (8 * (g & 1) + j) * L::kRow + piece * 16 + (byte & 15);
        if constexpr (CB == 8) {
          const uint2 v = *reinterpret_cast<const uint2*>(src);
          w[u][j][0] = v.x;
          w[u][j][1] = v.y;
        } else if constexpr (CB == 4) {
          w[u][j][0] = *reinterpret_cast<const unsigned*>(src);
        } else {
          w[u][j][0] = *reinterpret_cast<const uint16_t*>(src);
        }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int r = 0; r < RT; ++r)
          pf[u][t][r] = *reinterpret_cast<const v8h*>(pb + t * L::kP + (r * 16 + n) * L::kPRow + u * 64 + g * 16);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        v4i f;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = pair_of(w[u][2 * j][c / 4], w[u][2 * j + 1][c / 4], c % 4);
        const v8h v = __builtin_bit_cast(v8h, f);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int r = 0; r < RT; ++r) o[r][c] = mfma(v, pf[u][t][r], o[r][c]);
      }
    slot = slot == L::kSlots - 1 ? 0 : slot + 1;
  }

  // the rows' sums over lanes and waves
  lds_barrier();
#pragma unroll
  for (int r = 0; r < QR; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
    if (g == 0) tops[tg * kRows + (half * QR + r) * 16 + n] = l[r];
  }
  lds_barrier();
  const bool whole = begin == 0 && end == total;
  const int64_t place = ((int64_t)part * p.row_tiles + tile) * kRows;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int in_tile = r * 16 + n, row = row0 + in_tile;
    if (row >= rows) continue;
    const float sum = tops[in_tile] + tops[kRows + in_tile] + tops[2 * kRows + in_tile] + tops[3 * kRows + in_tile];
    const int d0 = wave * CB * 16 + 4 * CB * g;
    const float unit = R * (1.0f / kLift);
    const float f = whole ? (sum == 0.0f ? 0.0f : unit / sum) : unit;
    float y[4 * CB];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < CB; ++c) y[i * CB + c] = o[r][c][i] * f;
    if (!whole) {
      float* into = p.part_o + (place + in_tile) * D + d0;
#pragma unroll
      for (int k = 0; k < 4 * CB; k += 4) *reinterpret_cast<v4f*>(into + k) = v4f{y[k], y[k + 1], y[k + 2], y[k + 3]};
      if (wave == 0 && g == 0) {
        p.part_ml[2 * (place + in_tile)] = m[r];
        p.part_ml[2 * (place + in_tile) + 1] = sum;
      }
      continue;
    }
    const int token = token_of(p, row);
    T* into = static_cast<T*>(p.a.out) + (s.first + (int64_t)token) * p.a.ldo + (row - token * heads) * p.a.hdo + d0;
#pragma unroll
    for (int k = 0; k < 4 * CB; k += 4) {
      const float z[4] = {y[k], y[k + 1], y[k + 2], y[k + 3]};
      if (p.vec) {
        store_reals<T, 4>(into + k, z);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) into[k + e] = (T)z[e];
      }
    }
  }
}

// Joins the parts of a row, 8 of them at a time in flight.  A unit of WAYS * Q threads
// has 4 Q dimensions of one row: one wave 256 where rows are many, a block 64 dimensions
// where they are few and have many parts.  Both kernels, in us, a wave and a block for a
// unit: 8 rows of 16 heads over 8192 31.7 and 26.1, 1 over 131072 94 and 33, 20 over 2048
// 23.3 and 26.1, 60 over 2048 30.4 and 41.4.
template <typename T, int Q, int WAYS>
__global__ __launch_bounds__(256) void k_latent_join(const LatentRun p, int tile_rows) {
  constexpr int kAhead = 8, kUnits = 256 / (Q * WAYS);
  __shared__ float sums[1024], stats[512];
  const LatentArgs& a = p.a;
  const int pieces = a.c.latent / (4 * Q), tid = threadIdx.x, x = tid % Q, y = tid / Q % WAYS;
  const int unit = (int)blockIdx.x * kUnits + tid / (Q * WAYS), row = unit / pieces, d0 = unit % pieces * 4 * Q + 4 * x;
  const SeqDev s = seq_of(a.b, a.c.page, blockIdx.y);
  const int i = token_of(p, row), head = row - i * a.heads;
  bool some = s.ok && i < s.fresh;
  float mx = kNoMax, sum = 0.0f;
  v4f v = {0, 0, 0, 0};
  if (some) {
    const int tile = row / tile_rows, total = rows_chunks(p, s, tile * tile_rows, tile_rows);
    const int size = part_chunks(rows_chunks(p, s, 0, s.fresh * a.heads), p.line[a.b.seqs]);
    const int many = (total + size - 1) / size;
    some = many > 1;  // else written already
    const int64_t stride = (int64_t)p.row_tiles * tile_rows;
    const int64_t at0 = p.line[blockIdx.y] * stride + (int64_t)tile * tile_rows + row % tile_rows;
    const auto part = [&](int k) { return k * stride + at0; };
    if (some) {
      for (int k0 = y; k0 < many; k0 += WAYS * kAhead) {
        v4f in[kAhead];
        float w[kAhead], l[kAhead];
        float now = mx;
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          const int64_t at = part(min(k0 + e * WAYS, many - 1));
          in[e] = *reinterpret_cast<const v4f*>(p.part_o + at * a.c.latent + d0);
          w[e] = k0 + e * WAYS < many ? p.part_ml[2 * at] : kNoMax;
          l[e] = p.part_ml[2 * at + 1];
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) now = fmaxf(now, w[e]);
        const float down = __builtin_amdgcn_exp2f(mx - now);
        sum *= down;
        v *= down;
        mx = now;
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
          if (k0 + e * WAYS < many) {
            w[e] = __builtin_amdgcn_exp2f(w[e] - mx);
            sum += w[e] * l[e];
            v += w[e] * in[e];
          }
      }
    }
  }
  if constexpr (WAYS > 1) {
    stats[2 * tid] = mx;
    stats[2 * tid + 1] = sum;
    *reinterpret_cast<v4f*>(sums + 4 * tid) = v;
    __syncthreads();
    if (y > 0) return;
    float top = mx;
    for (int w = 1; w < WAYS; ++w) top = fmaxf(top, stats[2 * (tid + w * Q)]);
    const float down = __builtin_amdgcn_exp2f(mx - top);
    sum *= down;
    v *= down;
    for (int w = 1; w < WAYS; ++w) {
      const float f = __builtin_amdgcn_exp2f(stats[2 * (tid + w * Q)] - top);
      sum += f * stats[2 * (tid + w * Q) + 1];
      v += f * *reinterpret_cast<const v4f*>(sums + 4 * (tid + w * Q));
    }
  }
  if (!some) return;
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
  T* to = static_cast<T*>(a.out) + (s.first + (int64_t)i) * a.ldo + head * a.hdo + d0;
#pragma unroll
  for (int k = 0; k < 4; ++k) to[k] = (T)(v[k] * f);
}

struct LatentPlan {
  int rt, row_tiles, shared, groups, rounds, least;
  int64_t each;  // chunks of a block, by the bounds
  int64_t part, bytes;
};

LatentPlan plan_with(const Ctx& c, const fxpq_latent_cache& k, const fxpq_kv_batch& b, int heads, int type, int rt) {
  LatentPlan p{};
  const int64_t rows = (int64_t)b.max_new * heads, chunks = (b.max_len + 63) / 64;
  p.rt = rt;
  p.row_tiles = (int)((rows + rt * 16 - 1) / (rt * 16));
  p.rounds = 1;
  // (the kernel counts a cut's chunks in 32 bits)
  p.shared = (int64_t)p.row_tiles * b.seqs < 4 * (int64_t)c.cus && b.seqs <= kMostSeqs && p.row_tiles <= c.cus / 8 &&
             chunks * b.seqs < INT64_C(0x7FF00000);
  if (!p.shared) {
    p.groups = b.seqs;
    p.each = chunks;
    return p;
  }
  // Parts whose blocks fit the chip at a time; two for each sequence, so that few long ones
  // among many can be cut: 128 x 1, 128 heads, over 512 and one over 16384 118 us, whole
  // 645; where all have 1024 the two ways take 121 and 108 us, 200 of them 258 and 204, which
  // is why sequences are left whole from four blocks a CU on.
  const int slots = rt == 1 && type != FXPQ_F32 ? 2 * c.cus : c.cus;
  p.groups = slots / 8 / p.row_tiles * 8;
  p.rounds = (2 * b.seqs + p.groups - 1) / p.groups;
  // one chunk a part for few tiles: 1 x 1 over 300 13.6 us, two chunks 15.4; but 8 x 1 over
  // 2048 19.9 and 18.9, 64 x 1 over 300 23.4 and 19.1
  p.least = b.seqs * p.row_tiles <= 4 ? 1 : 2;
  p.each = chunks * b.seqs / p.groups;
  p.part = (int64_t)p.groups * p.rounds * p.row_tiles * rt * 16;
  p.bytes = p.part * (k.latent + 2) * 4 + (b.seqs + 1) * 4;
  return p;
}

// Row tiles of a block: more of them spare conversions of the codes, fewer make more parts
// and shorter ones.  In us with 1, 2 and 4 tiles, 128 heads, bf16, latents of 256: 32 x 1
// over 4096 (32 chunks a block with two tiles) 75, 70, 56; 8 x 1 over 4096 (8 chunks) 30.3,
// 29.3, 33.2; 16 x 1 over 1024 (4) 23.4, 23.1, 27.7.  Latents of 512: 32 x 1 over 4096 115 and
// 100, 2 x 1 rows of 16 heads over 8192 (0.5) 19 and 22; four tiles do not fit the registers
// (174 us).  f32, whose q and P are twice as large, in one and two tiles: latents of 256,
// 32 x 1 over 4096 110 and 80, 2 x 1 of 32 heads over 512 12.8 and 15.2; of 512 one only (163
// and 196).
LatentPlan plan_latent(const Ctx& c, const fxpq_latent_cache& k, const fxpq_kv_batch& b, int heads, int type) {
  const int64_t rows = (int64_t)b.max_new * heads;
  for (int rt = type == FXPQ_F32 ? k.latent == 512 ? 1 : 2 : k.latent == 512 ? 2 : 4; rt > 1; rt /= 2) {
    if (rows <= rt * 8) continue;
    const LatentPlan p = plan_with(c, k, b, heads, type, rt);
    if (p.each >= (rt == 4 ? 12 : 4)) return p;
  }
  return plan_with(c, k, b, heads, type, 1);
}

template <typename T, int LB, int RT, int W>
hipError_t run_latent(const Ctx& c, const LatentRun& p) {
  constexpr int bytes = LatentLds<LB, RT, sizeof(T) == 4 ? 2 : 1>::kBytes;
  auto* f = k_latent_attention<T, LB, RT, W>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(f), bytes);
  if (e != hipSuccess) return e;
  const int64_t blocks = ((int64_t)p.groups * p.rounds + 7) / 8 * 8 * p.row_tiles;
  if (blocks > kMaxBlocks) return hipErrorInvalidValue;
  f<<<dim3((unsigned)blocks), dim3(W * 64), bytes, c.stream>>>(p);
  if (p.shared) {
    const int64_t rows = (int64_t)p.a.b.max_new * p.a.heads;
    if (rows * p.a.b.seqs >= 256) {
      constexpr int kUnits = 4;  // 64 lanes, 256 dimensions each
      k_latent_join<T, 64, 1><<<dim3((unsigned)((rows * (LB / 4) + kUnits - 1) / kUnits), (unsigned)p.a.b.seqs), dim3(256), 0,
                                c.stream>>>(p, RT * 16);
    } else {
      k_latent_join<T, 16, 16><<<dim3((unsigned)(rows * LB), (unsigned)p.a.b.seqs), dim3(256), 0, c.stream>>>(p, RT * 16);
    }
  }
  return hipGetLastError();
}

template <typename T, int LB>
hipError_t run_rows(const Ctx& c, const LatentRun& p, int rt) {
  if constexpr (sizeof(T) == 4 && LB == 8) {
    return run_latent<T, LB, 1, 4>(c, p);
  } else {
    if (rt == 1) return run_latent<T, LB, 1, 4>(c, p);
    if constexpr (sizeof(T) == 2 && LB == 4)
      if (rt == 4) return run_latent<T, LB, 4, 8>(c, p);
    return run_latent<T, LB, 2, 8>(c, p);
  }
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
  p.shared = plan.shared;
  p.groups = plan.groups;
  p.rounds = plan.rounds;
  p.least = plan.least;
  while ((1 << p.page_log2) < a.c.page) ++p.page_log2;
  int log2 = 0;
  while ((1 << log2) < a.heads) ++log2;
  p.heads_shift = 30 + log2;
  p.heads_mul = (unsigned)(((uint64_t(1) << p.heads_shift) + a.heads - 1) / a.heads);
  const int64_t size = real_bytes(type);
  const auto fits = [&](const void* at, int64_t ld, int64_t hd) {
    return (uintptr_t)at % 16 == 0 && ld * size % 16 == 0 && hd * size % 16 == 0;
  };
  p.vec = fits(a.q, a.ldq, a.hdq) && fits(a.qr, a.ldqr, a.hdqr) && fits(a.out, a.ldo, a.hdo);
  p.part_o = static_cast<float*>(ws);
  p.part_ml = p.part_o ? p.part_o + plan.part * a.c.latent : nullptr;
  p.line = p.part_ml ? reinterpret_cast<int*>(p.part_ml + plan.part * 2) : nullptr;
  p.flags = c.sc.flags;
  return for_real(type, [&](auto zero) {
    using T = decltype(zero);
    return a.c.latent == 512 ? run_rows<T, 8>(c, p, plan.rt) : run_rows<T, 4>(c, p, plan.rt);
  });
}

}  // namespace fxpq
