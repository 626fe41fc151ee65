// Per-token quantization and the 8-bit products whose scales belong to tokens
// and output channels, plain and grouped by expert.
#include <type_traits>

#include "ring.hpp"
#include "serve.hpp"
#include "values.hpp"

namespace fxpq {
namespace {

// ---- per-token quantization ----------------------------------------------------
// One block per row: the largest magnitude, then the codes from a second read
// of the row (at most a few ten KB, from the caches).  Bound by memory: 8192 rows of
// 2048 bf16 values 12.5 us, 4.0 TB/s; one row 2 us, a launch.
// VB: bytes of a load that every row's address is aligned to (16, 8 or the type's).
template <typename T, int VB, int NT>
__global__ __launch_bounds__(NT) void k_token_quantize(const T* __restrict__ x, int64_t cols,
                                                        int64_t ldx, int rule,
                                                        int8_t* __restrict__ codes, int64_t ldc,
                                                        float* __restrict__ scale,
                                                        unsigned* flags) {
  __shared__ float part[NT / 64];
  constexpr int V = 16;  // values of one thread and step: one 16-byte store of codes
  const T* row = x + (int64_t)blockIdx.x * ldx;
  int8_t* out = codes + (int64_t)blockIdx.x * ldc;
  const int lane = threadIdx.x & 63;
  auto load = [&](int64_t c, float(&v)[V]) {
    if (VB > (int)sizeof(T) && c + V <= cols) {
      constexpr int W = VB / sizeof(T);
#pragma unroll
      for (int i = 0; i < V; i += W) {
        float u[W];
        load_reals<T, W>(row + c + i, u);
#pragma unroll
        for (int j = 0; j < W; ++j) v[i + j] = u[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = c + i < cols ? (float)row[c + i] : 0.0f;
    }
  };
  // a NaN or an infinity makes the integer maximum of the magnitudes' bits at
  // least that of infinity
  unsigned top = 0;
  for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += NT * V) {
    float v[V];
    load(c, v);
#pragma unroll
    for (int i = 0; i < V; ++i) top = max(top, __builtin_bit_cast(unsigned, v[i]) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d));
  if (lane == 0) part[threadIdx.x >> 6] = __builtin_bit_cast(float, top);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) top = max(top, __builtin_bit_cast(unsigned, part[i]));
  const bool bad = top >= 0x7F800000u;
  const float a = fmaxf(__builtin_bit_cast(float, top), kScaleFloor);
  float s, inv;
  if (rule == FXPQ_SCALE_DFX) {
    s = dfx_scale(a);
    inv = pow2_inverse(s);
  } else {
    s = a / 127.0f;
    inv = 127.0f / a;
  }
  if (threadIdx.x == 0) {
    scale[blockIdx.x] = bad ? __builtin_nanf("") : s;
    if (bad) raise_flag(flags, FXPQ_FLAG_NONFINITE);
  }
  for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += NT * V) {
    float v[V];
    load(c, v);
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int q[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] = bad ? 0 : (int)rintf(v[4 * i + j] * inv);
      w[i] = pack4(q[0], q[1], q[2], q[3]);
    }
    *reinterpret_cast<uint4*>(out + c) = uint4{w[0], w[1], w[2], w[3]};
  }
}

// ---- tiled product -----------------------------------------------------------------
// 16 zero bytes: what a tile reads past the depth.
__device__ int4 kZero16[1] = {{0, 0, 0, 0}};

// One depth step of a tile: KS bytes of every row, as 16-byte chunks.  Chunk c
// of row r sits at position c ^ f(r), f stepping once in every 256 bytes: the 16
// rows that one pass of a ds_read_b128 takes then cover all 64 banks once.
template <int KS>
__device__ inline int slab_off(int row, int chunk) {
  return row * KS + ((chunk ^ ((row / (256 / KS)) & (KS / 16 - 1))) << 4);
}

// The same for the rows of a wave's part of the output on their way to memory,
// RB bytes each.
template <int RB>
__device__ inline int out_off(int row, int chunk) {
  constexpr int per = RB < 256 ? 256 / RB : 1;
  return row * RB + ((chunk ^ ((row / per) & (RB / 16 - 1))) << 4);
}

// Output tile BM tokens x BN channels; WR x WC waves, each (BM / WR) x (BN / WC)
// in 32 x 32 matrix-core tiles.  Both operands go through an LDS ring of NS
// stages of KS bytes of depth, filled by global -> LDS loads NS - 1 steps ahead.
// Large products are bound by the matrix cores, whose clock falls under them: 8192 x
// 8192 x 4096 (rows, channels, depth) in 230 to 268 us, 2.0 to 2.4 P operations/s.
// T = int: a block takes the blockIdx.y-th share of the depth and leaves its sums
// in g.y, [share][M][ldy], for k_gemm_join.
template <int BM, int BN, int WR, int WC, int KS, int NS, bool GROUP, typename T>
__global__ __launch_bounds__(WR* WC * 64) void k_gemm_tile(GemmArgs g) {
  constexpr int NW = WR * WC, TM = BM / WR / 32, TN = BN / WC / 32;
  constexpr int kPiece = 1024 / KS;  // rows of one load (1 KB) of a wave
  constexpr int LA = BM / kPiece / NW, LB = BN / kPiece / NW;  // loads of a wave and step
  static_assert(BM % (kPiece * NW) == 0 && BN % (kPiece * NW) == 0, "whole loads for every wave");
  extern __shared__ __attribute__((aligned(1024))) int8_t smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles_n = (int)((g.N + BN - 1) / BN);
  // Blocks are dealt to the 8 XCDs round-robin by id; each XCD takes a
  // contiguous run of tiles, in bands of 8 row tiles, so that the tiles it has
  // in flight share rows and columns in its L2.
  const int block = blockIdx.x, blocks = gridDim.x;
  int tm = 0, tn = 0;
  auto place = [&](int t, int rows_all) {
    constexpr int kBand = 8;
    const int band = t / (kBand * tiles_n);
    const int in_band = t - band * kBand * tiles_n;
    const int high = min(kBand, rows_all - band * kBand);
    tm = band * kBand + in_band % high;
    tn = in_band / high;
  };
  int64_t m0, m_end;
  const int8_t* b = g.b;
  const float* b_scale = g.b_scale;
  const float* bias = g.bias;
  if constexpr (GROUP) {
    // Groups take ceil(rows / BM) row tiles each, in order.  The grid holds as many as
    // any sizes can take; the ones that these sizes take are dealt evenly to the XCDs
    // (a run of the grid's own tiles would leave the last XCDs idle: 1024 rows of 16
    // equal experts, 4096 x 2048 weights, 64 us so and 44 dealt evenly).
    __shared__ int sh_e, sh_first, sh_tm, sh_tn;
    if (threadIdx.x < 64) {
      auto tiles_of = [&](int e) {
        if (e >= g.experts) return 0;
        const int lo = g.offsets[e], hi = g.offsets[e + 1];
        if (lo < 0 || hi < lo || hi > g.M) {
          if (block == 0) raise_flag(g.flags, FXPQ_FLAG_RANGE);
          return 0;
        }
        return (int)(((int64_t)hi - lo + BM - 1) / BM);
      };
      const int most = blocks / tiles_n;  // row tiles: more only where the offsets contradict each other
      int total = 0;
      for (int e0 = 0; e0 < g.experts; e0 += 64) {
        int n = tiles_of(e0 + lane);
#pragma unroll
        for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
        total = min(total + n, most);
      }
      const int tiles = total * tiles_n, per = (tiles + 7) / 8, t = block % 8 * per + block / 8;
      int found = -1, first = 0;
      if (block / 8 < per && t < tiles) {
        place(t, total);
        int seen = 0;
        for (int e0 = 0; e0 < g.experts && found < 0; e0 += 64) {
          const int n = tiles_of(e0 + lane);
          int upto = n;  // tiles of the experts up to this one
#pragma unroll
          for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
          }
          const unsigned long long hit = __ballot(tm < seen + upto);
          if (hit) {
            const int l = __ffsll((long long)hit) - 1;
            found = e0 + l;
            first = seen + __shfl(upto, l) - __shfl(n, l);
          }
          seen += __shfl(upto, 63);
        }
      }
      if (lane == 0) {
        sh_e = found;
        sh_first = first;
        sh_tm = tm;
        sh_tn = tn;
      }
    }
    __syncthreads();
    const int e = sh_e;
    if (e < 0) return;
    tm = sh_tm;
    tn = sh_tn;
    m0 = g.offsets[e] + (int64_t)(tm - sh_first) * BM;
    m_end = g.offsets[e + 1];
    b += (int64_t)e * g.N * g.K;
    b_scale += (int64_t)e * g.N;
    if (bias) bias += (int64_t)e * g.N;
  } else {
    place(blocks % 8 == 0 ? block % 8 * (blocks / 8) + block / 8 : block, blocks / tiles_n);
    m0 = (int64_t)tm * BM;
    m_end = g.M;
  }
  const int64_t n0 = (int64_t)tn * BN;

  int64_t depth = g.K;
  const int8_t* a = g.a;
  T* y = static_cast<T*>(g.y);
  if constexpr (__is_same(T, int)) {
    const int64_t k0 = blockIdx.y * g.share;
    depth = min(g.share, g.K - k0);
    a += k0;
    b += k0;
    y += (int64_t)blockIdx.y * g.M * g.ldy;
  }

  // this lane's part of each 1 KB load: one chunk of one row
  constexpr int kChunks = KS / 16;
  const int8_t* src[LA + LB];
#pragma unroll
  for (int i = 0; i < LA + LB; ++i) {
    const bool is_a = i < LA;
    const int piece = wave + NW * (is_a ? i : i - LA);
    const int r = piece * kPiece + lane / kChunks;
    const int chunk = ((lane % kChunks) ^ ((r / (256 / KS)) & (kChunks - 1))) * 16;
    if (is_a) {
      int64_t m = min(m0 + r, m_end - 1);  // rows past the end: any row, never stored
      if (GROUP && g.a_rows) {
        const int64_t to = g.a_rows[m];
        m = to < 0 || to >= g.a_count ? 0 : to;
      }
      src[i] = a + m * g.lda + chunk;
    } else {
      src[i] = b + min(n0 + r, g.N - 1) * g.K + chunk;
    }
  }
  constexpr int kStage = (BM + BN) * KS;
  const int steps = (int)((depth + KS - 1) / KS);
  // load i of a step's LA + LB
  auto fill_one = [&](int step, int stage, int i) {
    dma16(src[i] + (int64_t)step * KS,
          smem + stage * kStage + wave * 1024 + (i < LA ? NW * i * 1024 : BM * KS + NW * (i - LA) * 1024));
  };
  auto fill = [&](int step, int stage) {
    const int64_t k0 = (int64_t)step * KS;
#pragma unroll
    for (int i = 0; i < LA + LB; ++i) {
      if (k0 + KS <= depth) {
        fill_one(step, stage, i);
      } else {  // past the depth: zeros
        const int r = (wave + NW * (i < LA ? i : i - LA)) * kPiece + lane / kChunks;
        const int chunk = ((lane % kChunks) ^ ((r / (256 / KS)) & (kChunks - 1))) * 16;
        dma16(k0 + chunk < depth ? src[i] + k0 : reinterpret_cast<const int8_t*>(kZero16),
              smem + stage * kStage + wave * 1024 + (i < LA ? NW * i * 1024 : BM * KS + NW * (i - LA) * 1024));
      }
    }
  };

  v16i acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
  const int wm = wave / WC, wn = wave % WC;
  // LDS bytes of this lane's chunk 0 or 1 of its first token and channel row (row
  // l % 32 of a 32-row tile, whose f is the same for every tile); the column kk of
  // a step is at that address ^ 32 kk
  const int sw = slab_off<KS>(lane & 31, lane >> 5);
  const int a_at = wm * (BM / WR) * KS + sw, b_at = BM * KS + wn * (BN / WC) * KS + sw;
  // The operands of one 32-byte column of the step, two sets in turn: while one
  // feeds the matrix cores the next is read.  The last column's products run
  // across the barrier, with the next stage's first operands and the loads of
  // the stage after it already under way.
  v4i af[2][TM], bf[2][TN];
  auto fetch_one = [&](int set, int stage, int kk, int i) {
    const int at = ((i < TM ? a_at : b_at) + stage * kStage) ^ (kk << 5);
    if (i < TM) af[set][i] = *reinterpret_cast<const v4i*>(smem + at + i * 32 * KS);
    else bf[set][i - TM] = *reinterpret_cast<const v4i*>(smem + at + (i - TM) * 32 * KS);
  };
  // The products of one set; between(n) runs after the n-th of kProducts: what is
  // issued there (LDS reads, loads) goes out while the matrix cores work.
  // Weights are the first operand: a lane then holds four neighbouring channels
  // of one token in neighbouring registers.
  constexpr int kProducts = TM * TN, kReads = TM + TN, kLoads = LA + LB;
  auto multiply = [&](int set, auto between) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[set][j], af[set][i], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        between(i * TN + j);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  auto sync = [&](bool more) {
    // all but the loads of the NS - 2 stages after the next one have landed
    if (more) wait_vmcnt<(NS - 2) * (LA + LB)>();
    else wait_vmcnt<0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wave's LDS reads are done
    ring_barrier();
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < steps) fill(s, s);
  sync(steps >= NS - 1);
#pragma unroll
  for (int i = 0; i < kReads; ++i) fetch_one(0, 0, 0, i);
  if (NS - 1 < steps) fill(NS - 1, NS - 1);
  constexpr int kCols = KS / 32;
  auto columns = [&](int stage) {  // all but the step's last column
#pragma unroll
    for (int kk = 0; kk < kCols - 1; ++kk)
      multiply(kk & 1, [&](int n) {
#pragma unroll
        for (int i = n * kReads / kProducts; i < (n + 1) * kReads / kProducts; ++i)
          fetch_one((kk + 1) & 1, stage, kk + 1, i);
      });
  };
  int stage = 0, s = 0;
  const int whole = (int)(depth / KS);
  for (; s + NS < whole; ++s) {  // the step that is loaded lies inside the depth
    columns(stage);
    const int next = stage + 1 == NS ? 0 : stage + 1;
    sync(true);  // the next stage has landed, and every wave has read all of this one
    multiply((kCols - 1) & 1, [&](int n) {
#pragma unroll
      for (int i = n * kReads / kProducts; i < (n + 1) * kReads / kProducts; ++i) fetch_one(0, next, 0, i);
#pragma unroll
      for (int i = n * kLoads / kProducts; i < (n + 1) * kLoads / kProducts; ++i) fill_one(s + NS, stage, i);
    });
    stage = next;
  }
  for (; s < steps; ++s) {
    columns(stage);
    const int next = stage + 1 == NS ? 0 : stage + 1;
    if (s + 1 < steps) {
      sync(s + NS <= steps);
      if (s + NS < steps) fill(s + NS, stage);
#pragma unroll
      for (int i = 0; i < kReads; ++i) fetch_one(0, next, 0, i);
    }
    multiply((kCols - 1) & 1, [](int) {});
    stage = next;
  }

  // lane l, register r: channel 8 (r / 4) + 4 (l / 32) + r % 4, token l % 32.
  // Each 32-token slab of the wave's part goes through the wave's own share of
  // the LDS (the ring is done with) and leaves as whole 16-byte pieces of rows.
  constexpr int kW = TN * 32, RB = kW * (int)sizeof(T);  // channels of a slab row, its bytes
  constexpr int E = 16 / (int)sizeof(T);
  static_assert(NW * 32 * RB <= NS * kStage, "the slabs fit the ring's LDS");
  __syncthreads();
  int8_t* slab = smem + wave * 32 * RB;
  const int64_t c0 = n0 + wn * kW;  // kW == BN / WC
  const bool vec = (uintptr_t)y % 16 == 0 && g.ldy * sizeof(T) % 16 == 0;
  float sb[TN][16], bi[TN][16];
  auto channels = [&](const float* from, float(&to)[TN][16]) {
    if ((uintptr_t)from % 16 == 0 && n0 + BN <= g.N) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const v4f v = *reinterpret_cast<const v4f*>(from + c0 + 32 * j + 8 * q + 4 * (lane >> 5));
#pragma unroll
          for (int r = 0; r < 4; ++r) to[j][4 * q + r] = v[r];
        }
    } else {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          to[j][r] = from[min(c0 + 32 * j + 8 * (r / 4) + 4 * (lane >> 5) + r % 4, g.N - 1)];
    }
  };
  if constexpr (!__is_same(T, int)) {
    channels(b_scale, sb);
    if (bias) channels(bias, bi);
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t first = m0 + wm * (BM / WR) + 32 * i;
    if (first >= m_end) break;
    const int64_t m = min(first + (lane & 31), m_end - 1);
    int64_t am = m;
    bool bad = false;
    if (GROUP && g.a_rows) {
      am = g.a_rows[m];
      bad = am < 0 || am >= g.a_count;
      if (bad) raise_flag(g.flags, FXPQ_FLAG_RANGE);
    }
    float sa = 0.0f;
    if constexpr (!__is_same(T, int)) sa = bad ? __builtin_nanf("") : g.a_scale[am];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        Reals<T, 4> v;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if constexpr (__is_same(T, int)) {
            v.v[r] = acc[i][j][4 * q + r];
          } else {
            const float p = (float)acc[i][j][4 * q + r] * sa * sb[j][4 * q + r];
            v.v[r] = (T)(bias ? p + bi[j][4 * q + r] : p);
          }
        }
        const int n = 32 * j + 8 * q + 4 * (lane >> 5);
        *reinterpret_cast<Reals<T, 4>*>(reinterpret_cast<T*>(slab + out_off<RB>(lane & 31, n / E)) + n % E) = v;
      }
    // the wave's own LDS accesses complete in order: no barrier
    constexpr int kRowChunks = RB / 16;
#pragma unroll
    for (int k = 0; k < 32 * kRowChunks / 64; ++k) {
      const int at = k * 64 + lane, row = at / kRowChunks, chunk = at % kRowChunks;
      const Reals<T, E> v = *reinterpret_cast<const Reals<T, E>*>(slab + out_off<RB>(row, chunk));
      const int64_t to = first + row, n = c0 + chunk * E;
      if (to >= m_end || n >= g.N) continue;
      T* p = y + to * g.ldy + n;
      if (vec && n + E <= g.N) {
        // the largest tiles make outputs larger than the L2s: past them, so that the
        // operands stay (8192 x 8192 x 4096: 276 -> 258 us, 16 experts 208 -> 189)
        if constexpr (BM == 256) __builtin_nontemporal_store(__builtin_bit_cast(v4i, v), reinterpret_cast<v4i*>(p));
        else *reinterpret_cast<Reals<T, E>*>(p) = v;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (n + e < g.N) p[e] = v.v[e];
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// The sums of a split depth, [shares][M][ldw] integers in any order, scaled and
// rounded: four channels of one row a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_gemm_join(GemmArgs g, const int* part, int64_t ldw, int shares) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, quads = ldw / 4;
  const int64_t m = i / quads, n = i % quads * 4;
  if (m >= g.M) return;
  v4i sum = {0, 0, 0, 0};
  for (int s = 0; s < shares; ++s) sum += *reinterpret_cast<const v4i*>(part + ((int64_t)s * g.M + m) * ldw + n);
  const float sa = g.a_scale[m];
  T* y = static_cast<T*>(g.y) + m * g.ldy + n;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (n + r < g.N) {
      const float p = (float)sum[r] * sa * g.b_scale[n + r];
      y[r] = (T)(g.bias ? p + g.bias[n + r] : p);
    }
}

// ---- at most 16 rows: the weights are the work ------------------------------------
// One block per 16 output channels; its eight waves deal the depth among them in
// 128-byte steps and read both operands straight into the matrix cores' registers
// (lane: channel or row l % 16, 16 bytes of the depth): nothing waits for a
// barrier before the end, where the eight partial sums are joined.  Bound by latency:
// one row of 1000 channels, depth 2048, 4.8 us.
constexpr int kFewRows = 16;

template <bool GROUP, typename T>
__global__ __launch_bounds__(512) void k_gemm_few(GemmArgs g) {
  constexpr int kWaves = 8, kStep = 128;
  constexpr int U = 4;  // steps whose loads are in flight together
  __shared__ v4i part[kWaves][64];
  const int lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  int64_t lo = 0, hi = g.M;
  const int8_t* b = g.b;
  const float *b_scale = g.b_scale, *bias = g.bias;
  if constexpr (GROUP) {
    const int64_t e = blockIdx.y;
    lo = g.offsets[e];
    hi = g.offsets[e + 1];
    if (lo < 0 || hi < lo || hi > g.M) {
      if (blockIdx.x == 0 && threadIdx.x == 0) raise_flag(g.flags, FXPQ_FLAG_RANGE);
      return;
    }
    if (lo == hi) return;
    b += e * g.N * g.K;
    b_scale += e * g.N;
    if (bias) bias += e * g.N;
  }
  const int64_t m = lo + n;  // this lane's row, as an operand and as a result
  int64_t am = min(m, hi - 1);
  bool bad = false;
  if (GROUP && g.a_rows) {
    am = g.a_rows[am];
    bad = am < 0 || am >= g.a_count;
    am = bad ? 0 : am;
  }
  const int8_t* a_row = g.a + am * g.lda;
  const int8_t* w_row = b + min(n0 + n, g.N - 1) * g.K;
  const int64_t steps = (g.K + kStep - 1) / kStep;
  v4i acc = {0, 0, 0, 0};
  for (int64_t s = wave; s < steps; s += kWaves * U) {
    v4i w[U][2], x[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int64_t at = (s + u * kWaves) * kStep + k * 64 + q * 16;
        const bool in = at < g.K;  // past the depth: zero weights, any codes
        w[u][k] = *reinterpret_cast<const v4i*>(in ? w_row + at : reinterpret_cast<const int8_t*>(kZero16));
        x[u][k] = *reinterpret_cast<const v4i*>(a_row + (in ? at : 0));
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < 2; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][k], x[u][k], acc, 0, 0, 0);
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0 || m >= hi) return;
  if (bad) raise_flag(g.flags, FXPQ_FLAG_RANGE);
  // lane l: channels 4 (l / 16) + 0..3 of row l % 16
#pragma unroll
  for (int w = 1; w < kWaves; ++w) acc += part[w][lane];
  const float sa = bad ? __builtin_nanf("") : g.a_scale[am];
  T* y = static_cast<T*>(g.y) + m * g.ldy;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t c = n0 + 4 * q + r;
    if (c < g.N) {
      const float p = (float)acc[r] * sa * b_scale[c];
      y[c] = (T)(bias ? p + bias[c] : p);
    }
  }
}

template <bool GROUP, typename T>
hipError_t run_few(const Ctx& c, const GemmArgs& g) {
  k_gemm_few<GROUP, T><<<dim3((unsigned)((g.N + 15) / 16), GROUP ? (unsigned)g.experts : 1u), dim3(512), 0,
                         c.stream>>>(g);
  return hipGetLastError();
}

template <int BM, int BN, int WR, int WC, int KS, int NS, bool GROUP, typename T>
hipError_t run_tile(const Ctx& c, const GemmArgs& g, int shares = 1) {
  const int64_t tiles_n = (g.N + BN - 1) / BN;
  // groups of any sizes need at most one partly filled row tile each
  const int64_t tiles_m = GROUP ? g.M / BM + g.experts : (g.M + BM - 1) / BM;
  if ((tiles_m * tiles_n + 7) * WR * WC * 64 > 0xFFFFFFFF) return hipErrorInvalidValue;
  constexpr int bytes = NS * (BM + BN) * KS;
  auto* f = k_gemm_tile<BM, BN, WR, WC, KS, NS, GROUP, T>;
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(f), bytes);
  if (e != hipSuccess) return e;
  const int64_t blocks = GROUP ? (tiles_m * tiles_n + 7) / 8 * 8 : tiles_m * tiles_n;
  f<<<dim3((unsigned)blocks, (unsigned)shares), dim3(WR * WC * 64), bytes, c.stream>>>(g);
  return hipGetLastError();
}

// A product whose depth is split among `shares` blocks of each tile.
template <int BM, int BN, int WR, int WC, int KS, int NS, typename T>
hipError_t run_split(const Ctx& c, const GemmArgs& g, int shares, void* ws) {
  GemmArgs p = g;
  p.share = ((g.K + shares - 1) / shares + KS - 1) / KS * KS;
  shares = (int)((g.K + p.share - 1) / p.share);
  p.y = ws;
  p.ldy = (g.N + 3) / 4 * 4;
  const hipError_t e = run_tile<BM, BN, WR, WC, KS, NS, false, int>(c, p, shares);
  if (e != hipSuccess) return e;
  k_gemm_join<T><<<dim3((unsigned)((g.M * (p.ldy / 4) + 255) / 256)), dim3(256), 0, c.stream>>>(
      g, static_cast<const int*>(ws), p.ldy, shares);
  return hipGetLastError();
}

// ---- which tiles ---------------------------------------------------------------------
constexpr int64_t kCus = 256;  // of an MI355X; the work space's size must not need a handle

// Time of a product by its tiles' shape, in us at a depth of 4096 (measured): the
// 256 x 256 tile has a CU to itself, the others share it with a second block, which
// costs less than twice the time of one.  Shapes are compared at that depth whatever
// the product's own, which scales all but a block's start and end: 777 x 1533 x 2064
// (rows, channels, depth) takes 18.0 us by the 128 x 64 tiles that this picks and 17.9
// by 64 x 64, 300 x 4096 x 4096 18.3 and 17.4 (with the quantization).
enum Tile { T64, T128x64, T128, T256 };
double tile_cost(Tile t, double tiles) {
  constexpr double one[] = {11.5, 16, 24, 43}, two[] = {17, 27, 41, 86};
  const double rounds = floor(tiles / (2 * kCus)), rest = tiles - rounds * 2 * kCus;
  return rounds * two[t] + (rest == 0 ? 0 : rest <= kCus ? one[t] : two[t]);
}

// Row tiles of groups: each expert fills its last one in part.
double tiles_of(double rows, int64_t N, int bm, int bn, double experts) {
  return (experts ? rows / bm + 0.75 * experts : ceil(rows / bm)) * (double)((N + bn - 1) / bn);
}

Tile best_tile(int64_t M, int64_t N, double experts, bool large) {
  const double cost[] = {tile_cost(T64, tiles_of((double)M, N, 64, 64, experts)),
                         tile_cost(T128x64, tiles_of((double)M, N, 128, 64, experts)),
                         tile_cost(T128, tiles_of((double)M, N, 128, 128, experts)),
                         tile_cost(T256, tiles_of((double)M, N, 256, 256, experts))};
  int best = T64;
  for (int t = T128x64; t <= (large ? T256 : T128); ++t)
    if (cost[t] < cost[best]) best = t;
  return (Tile)best;
}

// At most 16 rows, as long as no CU gets more than one block; wider products go by 64 x
// 64 tiles, which read a weight once for all rows (rows x channels x depth, with the
// quantization, this kernel first: 1 x 4096 x 4096 12.1 and 14.3 us, 16 x 1024 x 8192
// 13.0 and 14.3; 1 x 8192 x 4096 13.7 and 14.3, 16 x 8192 x 4096 15.3 and 14.4, 1 x
// 14336 x 4096 18.2 and 13.3, 16 x 14336 x 4096 22.3 and 13.9).
bool few_rows(int64_t M, int64_t N) { return M <= kFewRows && N <= 16 * kCus; }

// Where 64 x 64 tiles leave CUs idle and the depth is long, blocks share it: one for
// each 2048 of it at most, in whole slabs, so that the last share may be shorter (rows
// x channels x depth, with the quantization: 64 x 4096 x 9216 23.6 us whole, 18.7 in
// two, 16.7 in four; 64 x 4096 x 4112 16.0, 14.7 in two, 14.2 in four; 64 x 2048 x 1008
// 11.9 whole, 14.0 in two).  No rows, no tiles: M = 0 asks for a work space, too.
int depth_shares(int64_t M, int64_t N, int64_t K) {
  if (M == 0 || few_rows(M, N)) return 1;
  const int64_t tiles = ((M + 63) / 64) * ((N + 63) / 64);
  int64_t shares = kCus / tiles;
  if (shares > K / 2048) shares = K / 2048;
  return (int)(shares < 1 ? 1 : shares > 8 ? 8 : shares);
}

}  // namespace

hipError_t launch_token_quantize(const Ctx& c, const void* x, int x_type, int64_t rows, int64_t cols,
                                 int64_t ldx, int rule, int8_t* codes, int64_t ldc, float* scale) {
  return for_real(x_type, [&](auto zero) {
    using T = decltype(zero);
    const T* p = static_cast<const T*>(x);
    const uintptr_t at = (uintptr_t)x | (uintptr_t)(ldx * sizeof(T));
    // few rows leave most CUs without one: more threads for each (64 rows of 9216 and
    // their product 18.4 -> 17.5 us; 8192 rows of 4096 the other way, 257 -> 277)
    const auto run = [&](auto bytes) {
      constexpr int VB = decltype(bytes)::value;
      if (rows < c.cus && cols > 4096)
        k_token_quantize<T, VB, 1024><<<dim3((unsigned)rows), dim3(1024), 0, c.stream>>>(p, cols, ldx, rule, codes, ldc,
                                                                                     scale, c.sc.flags);
      else
        k_token_quantize<T, VB, 256><<<dim3((unsigned)rows), dim3(256), 0, c.stream>>>(p, cols, ldx, rule, codes, ldc,
                                                                                   scale, c.sc.flags);
    };
    if (at % 16 == 0) run(std::integral_constant<int, 16>());
    else if (at % 8 == 0) run(std::integral_constant<int, 8>());
    else run(std::integral_constant<int, sizeof(T)>());
    return hipGetLastError();
  });
}

int64_t token_gemm_workspace(int64_t M, int64_t N, int64_t K) {
  const int shares = depth_shares(M, N, K);
  return shares > 1 ? (int64_t)shares * M * ((N + 3) / 4 * 4) * 4 : 0;
}

hipError_t launch_token_gemm(const Ctx& c, const GemmArgs& g, int y_type, void* ws) {
  return for_real(y_type, [&](auto zero) {
    using T = decltype(zero);
    if (few_rows(g.M, g.N)) return run_few<false, T>(c, g);
    const int shares = depth_shares(g.M, g.N, g.K);
    if (shares > 1) return run_split<64, 64, 2, 2, 128, 4, T>(c, g, shares, ws);
    switch (best_tile(g.M, g.N, 0, true)) {
      case T64: return run_tile<64, 64, 2, 2, 128, 4, false, T>(c, g);
      case T128x64: return run_tile<128, 64, 2, 2, 128, 3, false, T>(c, g);
      case T128: return run_tile<128, 128, 2, 2, 128, 2, false, T>(c, g);
      default: return run_tile<256, 256, 2, 4, 128, 2, false, T>(c, g);
    }
  });
}

hipError_t launch_expert_gemm(const Ctx& c, const GemmArgs& g, int y_type) {
  return for_real(y_type, [&](auto zero) {
    using T = decltype(zero);
    if (few_rows(g.M, g.N)) return run_few<true, T>(c, g);
    // By the mean group, 4096 x 2048 weights, with the quantization: 128 rows of 32
    // experts 59.7 us by 32 x 64 tiles, 62.3 by 64 x 64; 1024 rows of 16 equal experts
    // 52.4 by 32 x 64, 43.4 by 64 x 64 (the costs' choice), 40.2 by 128 x 128; 2048 of
    // 16 ragged ones 62.3 by 128 x 128, 71.0 by 256 x 256 (equal ones 47.7 and 47.2);
    // 4096 of 16 74.7 and 55.0; 16384 of 16 ragged ones 240 and 186
    const int64_t mean = g.M / g.experts;
    if (mean <= 32) return run_tile<32, 64, 1, 2, 128, 4, true, T>(c, g);
    switch (best_tile(g.M, g.N, g.experts, mean >= 192)) {
      case T64: return run_tile<64, 64, 2, 2, 128, 4, true, T>(c, g);
      case T128x64: return run_tile<128, 64, 2, 2, 128, 3, true, T>(c, g);
      case T128: return run_tile<128, 128, 2, 2, 128, 2, true, T>(c, g);
      default: return run_tile<256, 256, 2, 4, 128, 2, true, T>(c, g);
    }
  });
}

}  // namespace fxpq
