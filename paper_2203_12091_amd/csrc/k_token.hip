// Per-token quantization and the 8-bit products whose scales belong to tokens
// and output channels, plain and grouped by expert.
#include "ring.hpp"
#include "serve.hpp"
#include "values.hpp"

namespace fxpq {
namespace {

// ---- per-token quantization ----------------------------------------------------
// One block per row: the largest magnitude, then the codes from a second read
// of the row (at most a few ten KB, from the caches).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_token_quantize(const T* __restrict__ x, int64_t cols,
                                                        int64_t ldx, int rule,
                                                        int8_t* __restrict__ codes, int64_t ldc,
                                                        float* __restrict__ scale,
                                                        unsigned* flags) {
  __shared__ float part[4];
  constexpr int V = 16;  // values of one thread and step: one 16-byte store of codes
  const T* row = x + (int64_t)blockIdx.x * ldx;
  int8_t* out = codes + (int64_t)blockIdx.x * ldc;
  const int lane = threadIdx.x & 63;
  auto load = [&](int64_t c, float(&v)[V]) {
    if (VEC && c + V <= cols) {
      constexpr int W = 16 / sizeof(T);
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
  for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += 256 * V) {
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
  for (int i = 0; i < 4; ++i) top = max(top, __builtin_bit_cast(unsigned, part[i]));
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
  for (int64_t c = (int64_t)threadIdx.x * V; c < cols; c += 256 * V) {
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

// One depth step of a tile: 128 bytes of every row, as eight 16-byte chunks.
// Chunk c of row r sits at position c ^ ((r >> 1) & 7): the 16 rows that one
// pass of a ds_read_b128 takes then cover all 64 banks once.
constexpr int kStep = 128;
__device__ inline int slab_off(int row, int chunk) {
  return row * kStep + ((chunk ^ ((row >> 1) & 7)) << 4);
}

// Output tile BM tokens x BN channels; WR x WC waves, each (BM / WR) x (BN / WC)
// in 32 x 32 matrix-core tiles.  Both operands go through a two-stage LDS ring
// filled by global -> LDS loads: the next step's are issued before this step's
// products, which cover their latency.
template <int BM, int BN, int WR, int WC, bool GROUP, typename T>
__global__ __launch_bounds__(WR* WC * 64) void k_gemm_tile(GemmArgs g) {
  constexpr int NW = WR * WC, TM = BM / WR / 32, TN = BN / WC / 32;
  constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW;  // 1 KB loads of a wave and step
  extern __shared__ __attribute__((aligned(1024))) int8_t smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles_n = (int)((g.N + BN - 1) / BN);
  // Blocks are dealt to the 8 XCDs round-robin by id; each XCD takes a
  // contiguous run of tiles, in bands of 8 row tiles, so that the tiles it has
  // in flight share rows and columns in its L2.
  int t = blockIdx.x;
  const int T_all = gridDim.x;
  if (T_all % 8 == 0) t = (t % 8) * (T_all / 8) + t / 8;
  const int rows_all = T_all / tiles_n;
  constexpr int kBand = 8;
  const int band = t / (kBand * tiles_n);
  const int in_band = t - band * kBand * tiles_n;
  const int high = min(kBand, rows_all - band * kBand);
  int tm = band * kBand + in_band % high;
  const int tn = in_band / high;
  int64_t m0, m_end;
  const int8_t* b = g.b;
  const float* b_scale = g.b_scale;
  const float* bias = g.bias;
  if constexpr (GROUP) {
    // the expert of this row tile: groups take ceil(rows / BM) tiles each, in order
    __shared__ int sh_e, sh_first;
    if (threadIdx.x < 64) {
      int seen = 0, found = -1, first = 0;
      for (int e0 = 0; e0 < g.experts && found < 0; e0 += 64) {
        const int e = e0 + lane;
        int n = 0;
        if (e < g.experts) {
          const int lo = g.offsets[e], hi = g.offsets[e + 1];
          if (lo < 0 || hi < lo || hi > g.M) {
            if (blockIdx.x == 0) raise_flag(g.flags, FXPQ_FLAG_RANGE);
          } else {
            n = (hi - lo + BM - 1) / BM;
          }
        }
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
      if (lane == 0) {
        sh_e = found;
        sh_first = first;
      }
    }
    __syncthreads();
    const int e = sh_e;
    if (e < 0) return;
    m0 = g.offsets[e] + (int64_t)(tm - sh_first) * BM;
    m_end = g.offsets[e + 1];
    b += (int64_t)e * g.N * g.K;
    b_scale += (int64_t)e * g.N;
    if (bias) bias += (int64_t)e * g.N;
  } else {
    m0 = (int64_t)tm * BM;
    m_end = g.M;
  }
  const int64_t n0 = (int64_t)tn * BN;

  // this lane's part of each 1 KB load: row `lane >> 3` of eight, one chunk
  const int8_t* src[LA + LB];
  int chunk[LA + LB];
#pragma unroll
  for (int i = 0; i < LA + LB; ++i) {
    const bool is_a = i < LA;
    const int piece = wave + NW * (is_a ? i : i - LA);
    const int r = piece * 8 + (lane >> 3);
    chunk[i] = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
    if (is_a) {
      int64_t m = min(m0 + r, m_end - 1);  // rows past the end: any row, never stored
      if (GROUP && g.a_rows) {
        const int64_t to = g.a_rows[m];
        m = to < 0 || to >= g.a_count ? 0 : to;
      }
      src[i] = g.a + m * g.lda;
    } else {
      src[i] = b + min(n0 + r, g.N - 1) * g.K;
    }
  }
  constexpr int kStage = (BM + BN) * kStep;
  const int64_t steps = (g.K + kStep - 1) / kStep;
  auto fill = [&](int64_t step, int stage) {
    const int64_t k0 = step * kStep;
    int8_t* sa = smem + stage * kStage;
#pragma unroll
    for (int i = 0; i < LA + LB; ++i) {
      const int piece = wave + NW * (i < LA ? i : i - LA);
      int8_t* to = sa + (i < LA ? 0 : BM * kStep) + piece * 1024;
      const int64_t k = k0 + chunk[i];
      dma16(k < g.K ? src[i] + k : reinterpret_cast<const int8_t*>(kZero16), to);
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
  const int row0 = wm * (BM / WR) + (lane & 31), col0 = wn * (BN / WC) + (lane & 31);
  fill(0, 0);
  for (int64_t s = 0; s < steps; ++s) {
    wait_vmcnt<0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the last step's LDS reads are done
    ring_barrier();  // this stage has landed for every wave, and the other one is free
    if (s + 1 < steps) fill(s + 1, (int)((s + 1) & 1));
    const int8_t* sa = smem + (int)(s & 1) * kStage;
    const int8_t* sb = sa + BM * kStep;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      v4i af[TM], bf[TN];
      const int c = kk * 2 + (lane >> 5);
#pragma unroll
      for (int i = 0; i < TM; ++i)
        af[i] = *reinterpret_cast<const v4i*>(sa + slab_off(row0 + 32 * i, c));
#pragma unroll
      for (int j = 0; j < TN; ++j)
        bf[j] = *reinterpret_cast<const v4i*>(sb + slab_off(col0 + 32 * j, c));
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(af[i], bf[j], acc[i][j], 0, 0, 0);
    }
  }

  // lane l, register r: row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32
  T* y = static_cast<T*>(g.y);
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int64_t m = m0 + wm * (BM / WR) + 32 * i + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
      if (m >= m_end) continue;
      int64_t am = m;
      bool bad = false;
      if (GROUP && g.a_rows) {
        am = g.a_rows[m];
        bad = am < 0 || am >= g.a_count;
      }
      const float sa = bad ? __builtin_nanf("") : g.a_scale[am];
      if (bad && lane == 0) raise_flag(g.flags, FXPQ_FLAG_RANGE);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int64_t n = n0 + col0 + 32 * j;
        if (n < g.N) {
          const float p = (float)acc[i][j][r] * sa * b_scale[n];
          y[m * g.ldy + n] = (T)(bias ? p + bias[n] : p);
        }
      }
    }
}

template <int BM, int BN, int WR, int WC, bool GROUP, typename T>
hipError_t run_tile(const Ctx& c, const GemmArgs& g) {
  const int64_t tiles_n = (g.N + BN - 1) / BN;
  // groups of any sizes need at most one partly filled row tile each
  const int64_t tiles_m = GROUP ? g.M / BM + g.experts : (g.M + BM - 1) / BM;
  if (tiles_m * tiles_n * WR * WC * 64 > 0xFFFFFFFF) return hipErrorInvalidValue;
  constexpr int bytes = 2 * (BM + BN) * kStep;
  auto* f = k_gemm_tile<BM, BN, WR, WC, GROUP, T>;
  // more than 64 KB of LDS has to be asked for
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(f),
                                     hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return e;
  f<<<dim3((unsigned)(tiles_m * tiles_n)), dim3(WR * WC * 64), bytes, c.stream>>>(g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_token_quantize(const Ctx& c, const void* x, int x_type, int64_t rows, int64_t cols,
                                 int64_t ldx, int rule, int8_t* codes, int64_t ldc, float* scale) {
  return for_real(x_type, [&](auto zero) {
    using T = decltype(zero);
    const T* p = static_cast<const T*>(x);
    const bool vec = (uintptr_t)x % 16 == 0 && ldx * sizeof(T) % 16 == 0;
    if (vec)
      k_token_quantize<T, true><<<dim3((unsigned)rows), dim3(256), 0, c.stream>>>(
          p, cols, ldx, rule, codes, ldc, scale, c.sc.flags);
    else
      k_token_quantize<T, false><<<dim3((unsigned)rows), dim3(256), 0, c.stream>>>(
          p, cols, ldx, rule, codes, ldc, scale, c.sc.flags);
    return hipGetLastError();
  });
}

int64_t token_gemm_workspace(int64_t M, int64_t N, int64_t K) {
  (void)M, (void)N, (void)K;
  return 0;
}

hipError_t launch_token_gemm(const Ctx& c, const GemmArgs& g, int y_type, void* ws) {
  (void)ws;
  return for_real(y_type, [&](auto zero) { return run_tile<128, 128, 2, 2, false, decltype(zero)>(c, g); });
}

hipError_t launch_expert_gemm(const Ctx& c, const GemmArgs& g, int y_type) {
  return for_real(y_type, [&](auto zero) { return run_tile<128, 128, 2, 2, true, decltype(zero)>(c, g); });
}

}  // namespace fxpq
