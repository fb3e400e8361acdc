// 16-bit projection with its epilogue: out = act(x W^T + bias) + residual, fp16 or bf16 operands, fp32 sums.
//
//   acc[m, n] = sum_k x[m, k] W[n, k]          x [M, K], W [N, K], both K-contiguous
//
// The operands go through the matrix units as they are (products of 16-bit values are exact in fp32), sums stay in
// fp32 up to the epilogue, and the result is rounded once, to the output's type.
#include <atomic>
#include <cfloat>
#include <climits>

#include "common.h"
#include "device_util.h"
#include "half_util.h"

namespace quamba {

namespace {

// What follows the sums: bias, activation, residual, one rounding.
struct LinearEpi {
  const float *bias;  // [N] or NULL
  const void *res;    // [M, ldr] of the output's type or NULL; may be the output itself
  void *out;          // [M, ldo]
  long long ldr, ldo;
  int act;
};

// 0.5 erfc(z / sqrt 2) for z >= 0: with y = z / sqrt 2 and t = 1 / (1 + 0.4 y), erfc(y) = exp(-y^2) t p(t), p of degree 8
// fitted to erfc(y) exp(y^2) / t over 0 < t <= 1 by least squares whose weights were moved towards equal errors (1.5e-7 of the
// value).  A relative error; in fp32 the rounding of z^2 in the exponent adds to it, 2e-6 up to z = 6, 7e-6 at 12.  A third of the
// instructions of erfcf.
__device__ __forceinline__ float upper_tail(float z) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.4f * 0.70710678118654752440f, z, 1.f));
  float p = 0.02512870542705059f;
  p = fmaf(p, t, -0.09144222736358643f);
  p = fmaf(p, t, 0.08453038334846497f);
  p = fmaf(p, t, -0.0027945844922214746f);
  p = fmaf(p, t, 0.07071199268102646f);
  p = fmaf(p, t, 0.08427179604768753f);
  p = fmaf(p, t, 0.10392126441001892f);
  p = fmaf(p, t, 0.11283480376005173f);
  p = fmaf(p, t, 0.11283793300390244f);
  return p * t * __builtin_amdgcn_exp2f(-0.72134752044448170368f * z * z);
}

// v sigmoid(a) for a of v's sign.  The denominator is held 2^-8 times as large, so its reciprocal is not flushed before the result
// leaves fp32's normal range (SILU(-88) = -5e-37); nothing overflows on the way.  -infinity counts as the lowest number, whose
// product with 0 is the limit 0; a NaN comes back from the exponential.
__device__ __forceinline__ float times_sigmoid(float v, float a) {
  constexpr float LOG2E = 1.44269504088896340736f, D = 0.00390625f;
  return fmaxf(v, -FLT_MAX) * (__builtin_amdgcn_rcpf(D + __builtin_amdgcn_exp2f(fmaf(-LOG2E, a, -8.f))) * D);
}

// The activation in fp32.  exp2 of a large argument is infinite and its reciprocal 0, so nothing overflows on the way.
__device__ __forceinline__ float activate(float v, int act) {
  constexpr float LOG2E = 1.44269504088896340736f;
  switch (act) {
    case QUAMBA_ACT_RELU: return v < 0.f ? 0.f : v;  // keeps NaN
    case QUAMBA_ACT_SILU: return times_sigmoid(v, v);
    case QUAMBA_ACT_GELU: {  // v Phi(v)
      const float u = upper_tail(fabsf(v)), phi = v < 0.f ? u : 1.f - u;
      return phi == 0.f ? 0.f : v * phi;
    }
    case QUAMBA_ACT_GELU_TANH: {  // 0.5 v (1 + tanh u) = v sigmoid(2 u), u = sqrt(2 / pi) (v + 0.044715 v^3)
      const float u2 = 1.59576912160573071176f * v * (1.f + 0.044715f * v * v);
      return times_sigmoid(v, u2);
    }
    case QUAMBA_ACT_SIGMOID: return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-v * LOG2E));
    default: return v;
  }
}

// One output whose bias and residual are asked for before its sum is there: at a few rows their latency is what is left to save.
struct Single {
  float bias = 0.f, res = 0.f;
  bool on = false;
};
template <typename O>
__device__ __forceinline__ Single ask1(const LinearEpi &e, int gm, int gn, int M, int N) {
  Single s;
  s.on = gm < M && gn < N;
  if (s.on && e.bias) s.bias = e.bias[gn];
  if (s.on && e.res) s.res = to_f32(static_cast<const O *>(e.res)[(size_t)gm * e.ldr + gn]);
  return s;
}
template <typename O>
__device__ __forceinline__ void put1(const LinearEpi &e, const Single &s, int gm, int gn, float v) {
  if (s.on) static_cast<O *>(e.out)[(size_t)gm * e.ldo + gn] = from_f32<O>(activate(v + s.bias, e.act) + s.res);
}

// Byte offset of 16-byte chunk `chunk` of tile row `row` for rows of BKB bytes: any 16 consecutive rows read at one
// logical chunk hit 16 different bank groups (with 64-byte rows four rows span the 64 banks, with 128-byte rows two).
template <int BKB>
__device__ __forceinline__ int swz(int row, int chunk) {
  if constexpr (BKB == 64) return row * 64 + ((chunk ^ ((row >> 2) & 3)) << 4);
  else if constexpr (BKB == 128) return row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4);
  else return row * BKB + ((chunk ^ (row & 15)) << 4);
}

// A wave's TM x TN tiles of 32 x 32 sums: register r of lane l in tile (i, j) is column n_base + 32 i + 8 (r / 4) + 4 (l / 32)
// + r % 4 of row m_base + 32 j + l % 32.  A tile gets its bias and activation in registers (after a copy, so that their code
// exists once), then a band of 32 rows and up to 64 columns goes through a region of LDS that only this wave uses (fp32, rows 16
// bytes further apart than they are long), so that residual and output are taken 16 bytes a lane along the rows (global memory
// takes such accesses at any element's address).  The residual is asked for before the sums are laid out: one trip per row after
// them cost 4 us of a 22 us call.
constexpr int kBandPitch = 64 * 4 + 16;
constexpr int kBandBytes = 32 * kBandPitch;

template <typename O>
struct Band {
  static constexpr int E = 16 / sizeof(O), IT = 32 * 64 / (64 * E);  // elements of a 16-byte access; accesses of a lane (64 columns)
  typedef O vO __attribute__((ext_vector_type(E)));
  int m0, cc, gn, r0, rows;  // the lane's columns cc .., gn .. of the output; rows r0, r0 + rows, ...
  vO res[IT];

  __device__ __forceinline__ void ask(const LinearEpi &e, int m, int n, int cols, int lane, int M, int N) {
    const int per_row = cols / E;
    m0 = m, cc = lane % per_row * E, gn = n + cc, r0 = lane / per_row, rows = 64 / per_row;
    if (e.res && gn + E <= N) {
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int r = r0 + it * rows;
        if (r < 32 && m0 + r < M) __builtin_memcpy(&res[it], static_cast<const O *>(e.res) + (size_t)(m0 + r) * e.ldr + gn, 16);
      }
    }
  }
  __device__ __forceinline__ void put(const LinearEpi &e, int M, int N, const char *band) const {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int r = r0 + it * rows, gm = m0 + r;
      if (r >= 32 || gm >= M || gn >= N) continue;
      float v[E];
#pragma unroll
      for (int i = 0; i < E; i += 4) {
        const v4f t = *reinterpret_cast<const v4f *>(band + r * kBandPitch + (cc + i) * 4);
#pragma unroll
        for (int c = 0; c < 4; ++c) v[i + c] = t[c];
      }
      O *out = static_cast<O *>(e.out) + (size_t)gm * e.ldo + gn;
      if (gn + E <= N) {
        vO t;
#pragma unroll
        for (int i = 0; i < E; ++i) t[i] = from_f32<O>(e.res ? v[i] + to_f32(res[it][i]) : v[i]);
        __builtin_memcpy(out, &t, 16);
      } else {
        const O *rp = static_cast<const O *>(e.res) + (size_t)gm * e.ldr + gn;
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (gn + i < N) out[i] = from_f32<O>(e.res ? v[i] + to_f32(rp[i]) : v[i]);
      }
    }
  }
};

template <typename O, int TM, int TN>
__device__ __forceinline__ void store_wave(const v16f (&acc)[TN][TM], int m_base, int n_base, int lane, int M, int N, const LinearEpi &e,
                                           char *band) {
  Band<O> b;
#pragma unroll 1
  for (int step = 0; step < TM * TN; ++step) {
    const int j = step / TN, i = step - j * TN;
    const bool first = (i & 1) == 0, last = !first || i + 1 == TN;
    if (first) b.ask(e, m_base + 32 * j, n_base + 32 * i, i + 1 < TN ? 64 : 32, lane, M, N);
    float v[16], bias[16];
    if (e.bias) {
#pragma unroll
      for (int r = 0; r < 16; ++r) bias[r] = e.bias[min(n_base + 32 * i + 4 * (lane >> 5) + 8 * (r / 4) + r % 4, N - 1)];
    }
#pragma unroll
    for (int s = 0; s < TM * TN; ++s)
      if (s == step) {
        asm volatile("");  // a branch: as selects these are TM TN 16 instructions a step (19 us of a 118 us call)
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = acc[s % TN][s / TN][r];
      }
    if (e.bias) {
#pragma unroll
      for (int r = 0; r < 16; ++r) v[r] += bias[r];
    }
    switch (e.act) {
#define QUAMBA_ALL(A)                                  \
  case A: {                                            \
    _Pragma("unroll") for (int r = 0; r < 16; ++r) v[r] = activate(v[r], A); \
    break;                                             \
  }
      QUAMBA_ALL(QUAMBA_ACT_RELU)
      QUAMBA_ALL(QUAMBA_ACT_SILU)
      QUAMBA_ALL(QUAMBA_ACT_GELU)
      QUAMBA_ALL(QUAMBA_ACT_GELU_TANH)
      QUAMBA_ALL(QUAMBA_ACT_SIGMOID)
#undef QUAMBA_ALL
      default: break;
    }
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<v4f *>(band + (lane & 31) * kBandPitch + ((i & 1) * 32 + 8 * g + 4 * (lane >> 5)) * 4) =
          v4f{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
    if (last) b.put(e, M, N, band);
  }
}

// Workgroup ids are dealt round-robin to the 8 XCDs; give each a contiguous run of tiles, and walk the output in bands of
// 8 tile rows: what one XCD works on at a time then shares operand rows in its L2.
__device__ __forceinline__ void tile_of(int wg, int tiles_m, int tiles_n, int *tm, int *tn) {
  const int nwg = tiles_m * tiles_n, per = nwg >> 3;
  const int id = wg < (per << 3) ? (wg & 7) * per + (wg >> 3) : wg;
  const int width = 8 * tiles_n, first = id / width * 8, rows = min(tiles_m - first, 8), r = id % width;
  *tm = first + r % rows;
  *tn = r / rows;
}

// Any strides and alignments: K in slices of 32 staged through registers (16-byte loads at element addresses, which
// global memory serves at whatever lines they touch), two LDS stages, four waves in 2 x 2.
template <typename T, typename O, int TM, int TN>
__global__ __launch_bounds__(256) void linear_any_kernel(const T *__restrict__ x, long long ldx, const T *__restrict__ W,
                                                         long long ldw, int M, int N, int K, LinearEpi epi, int tiles_m, int tiles_n) {
  constexpr int BK = 32, BM = 64 * TM, BN = 64 * TN, STAGE = (BM + BN) * BK * 2;
  constexpr int LDS = 2 * STAGE > 4 * kBandBytes ? 2 * STAGE : 4 * kBandBytes;
  __shared__ __attribute__((aligned(16))) char lds[LDS];
  int tile_m, tile_n;
  tile_of(blockIdx.x, tiles_m, tiles_n, &tile_m, &tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave & 1, wn = wave >> 1;
  const int row = tid >> 2, ch = tid & 3;
  const int nk = (K + BK - 1) / BK;

  v16f acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  // rows outside repeat the last one: multiplied, never stored
  const T *px[TM], *pw[TN];
#pragma unroll
  for (int j = 0; j < TM; ++j) px[j] = x + (size_t)min(m0 + 64 * j + row, M - 1) * ldx;
#pragma unroll
  for (int i = 0; i < TN; ++i) pw[i] = W + (size_t)min(n0 + 64 * i + row, N - 1) * ldw;
  typename Half<T>::v8 rx[TM], rw[TN];
  auto fetch = [&](int kt) {
    const int gk = kt * BK + ch * 8;
#pragma unroll
    for (int j = 0; j < TM; ++j) rx[j] = row8(px[j], gk, K);
#pragma unroll
    for (int i = 0; i < TN; ++i) rw[i] = row8(pw[i], gk, K);
  };
  auto park = [&](int buf) {
#pragma unroll
    for (int j = 0; j < TM; ++j) *reinterpret_cast<typename Half<T>::v8 *>(lds + buf * STAGE + swz<64>(64 * j + row, ch)) = rx[j];
#pragma unroll
    for (int i = 0; i < TN; ++i) *reinterpret_cast<typename Half<T>::v8 *>(lds + buf * STAGE + BM * BK * 2 + swz<64>(64 * i + row, ch)) = rw[i];
  };

  fetch(0);
  park(0);
  __syncthreads();
  for (int kt = 0; kt < nk; ++kt) {
    const char *lx = lds + (kt & 1) * STAGE, *lw = lx + BM * BK * 2;
    if (kt + 1 < nk) fetch(kt + 1);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int chunk = s * 2 + (lane >> 5);
      typename Half<T>::v8 fx[TM], fw[TN];
#pragma unroll
      for (int j = 0; j < TM; ++j) fx[j] = *reinterpret_cast<const typename Half<T>::v8 *>(lx + swz<64>((wm * TM + j) * 32 + (lane & 31), chunk));
#pragma unroll
      for (int i = 0; i < TN; ++i) fw[i] = *reinterpret_cast<const typename Half<T>::v8 *>(lw + swz<64>((wn * TN + i) * 32 + (lane & 31), chunk));
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = Half<T>::mfma32(fw[i], fx[j], acc[i][j]);
    }
    if (kt + 1 < nk) park((kt + 1) & 1);
    __syncthreads();
  }
  store_wave<O, TM, TN>(acc, m0 + wm * TM * 32, n0 + wn * TN * 32, lane, M, N, epi, lds + wave * kBandBytes);
}

// 16-byte rows: slices travel with 16-byte direct-to-LDS buffer loads (no staging registers, no LDS write instructions).  A
// wave-level load writes 64 lanes x 16 bytes of consecutive LDS, 1024 / BKB tile rows, so the swizzle is applied on the global
// side: each lane fetches the chunk that belongs in its slot; rows past M or N and chunks past K arrive as zeros.
// Ring of S stages; KG groups of waves share one tile, group g multiplying the 32-byte sub-slices s with s % KG == g.
// s_waitcnt for "at most n vector loads outstanding, nothing else waited for" (vmcnt in bits 3:0 and 15:14, expcnt 6:4,
// lgkmcnt 11:8), and with this wave's LDS reads finished as well
#define QUAMBA_VMCNT(n) (((n) & 0xF) | ((((n) >> 4) & 0x3) << 14) | (0x7 << 4) | (0xF << 8))
#define QUAMBA_VMCNT_LGKM0(n) (((n) & 0xF) | ((((n) >> 4) & 0x3) << 14) | (0x7 << 4))

template <typename T, typename O, int BM, int BN, int WGM, int WGN, int S, int BKB, int OCC, int KG>
__global__ __launch_bounds__(64 * WGM * WGN * KG, OCC) void linear_dma_kernel(const T *__restrict__ x, long long ldx, const T *__restrict__ W,
                                                                              long long ldw, int M, int N, int K, LinearEpi epi, int tiles_m,
                                                                              int tiles_n) {
  constexpr int NW = WGM * WGN * KG, WM = BM / WGM, WN = BN / WGN, TM = WM / 32, TN = WN / 32;
  constexpr int RPI = 1024 / BKB, CPR = BKB / 16, ROWS = BM + BN, NJ = ROWS / RPI, NI = NJ / NW, STAGE = ROWS * BKB;
  constexpr int NSUB = BKB / 32 / KG, BKE = BKB / 2;  // sub-slices of a group; elements of a slice
  static_assert(WM % 32 == 0 && WN % 32 == 0 && BM % RPI == 0 && BN % RPI == 0 && BKB / 32 % KG == 0, "tile");
  static_assert((S - 2) * NI <= 63 && S >= 2 && (S > 2 || (NSUB >= 2 && KG == 1)), "ring");
  static_assert(NW * kBandBytes <= S * STAGE || KG > 1, "the bands fit in the ring");
  extern __shared__ __attribute__((aligned(16))) char ring[];

  int tile_m, tile_n;
  tile_of(blockIdx.x, tiles_m, tiles_n, &tile_m, &tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int nk = (K + BKE - 1) / BKE;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wave / (WGM * WGN), wtile = wave % (WGM * WGN), wm = wtile % WGM, wn = wtile / WGM;

  // Load i of a wave takes tile rows ROWS_I i + row on: the swizzle's phase is the same for all of them, and the first BM / ROWS_I
  // loads are x's.  A lane's offset reaches past the buffer where its row or (in the last slice) its chunk does not exist.
  constexpr int ROWS_I = NW * RPI, OFF = (int)0x80000000;
  static_assert(NJ % NW == 0 && ROWS_I % 16 == 0 && BM % ROWS_I == 0, "loads");
  const int row = wave * RPI + lane / CPR, chunk = (swz<BKB>(row, lane % CPR) - row * BKB) >> 4;
  const int ox = row * (int)ldx * 2 + chunk * 16, ow = row * (int)ldw * 2 + chunk * 16;
  const int step_x = ROWS_I * (int)ldx * 2, step_w = ROWS_I * (int)ldw * 2;
  auto end_of = [](long long bytes) { return (int)(bytes < 0x7fffffff ? bytes : 0x7fffffff); };
  const auto bx = buffer_over(x + (size_t)m0 * ldx, end_of((long long)(M - m0) * ldx * 2));
  const auto bw = buffer_over(W + (size_t)n0 * ldw, end_of((long long)(N - n0) * ldw * 2));
  auto issue = [&](int stage, int slice) {
    const bool off = slice * BKE + chunk * 8 >= K;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const bool is_x = i * ROWS_I < BM;
      const int at = is_x ? ox + i * step_x : ow + (i - BM / ROWS_I) * step_w;
      load_to_lds(is_x ? bx : bw, off ? OFF : at, slice * BKB, ring + stage * STAGE + (wave + NW * i) * 1024);
    }
  };

  v16f acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  typedef typename Half<T>::v8 v8;
  // the lane's offset of the group's first chunk in row lane % 32: another sub-slice is an exclusive-or away (as the swizzle's own
  // exchange of chunks is), 32 rows a constant.  Opaque per slice, or the sums are hoisted and take the registers of the tile
  const int at_lane = swz<BKB>(lane & 31, kg * 2 + (lane >> 5));
  auto frags = [&](int stage, int sub, v8 (&fx)[TM], v8 (&fw)[TN]) {
    int at = at_lane;
    if constexpr (TM * TN > 8) asm volatile("" : "+v"(at));
    const char *lx = ring + stage * STAGE + wm * WM * BKB + (at ^ (sub * KG * 32));
    const char *lw = ring + stage * STAGE + (BM + wn * WN) * BKB + (at ^ (sub * KG * 32));
#pragma unroll
    for (int j = 0; j < TM; ++j) fx[j] = *reinterpret_cast<const v8 *>(lx + j * 32 * BKB);
#pragma unroll
    for (int i = 0; i < TN; ++i) fw[i] = *reinterpret_cast<const v8 *>(lw + i * 32 * BKB);
  };
  auto mma = [&](const v8 (&fx)[TM], const v8 (&fw)[TN]) {
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = Half<T>::mfma32(fw[i], fx[j], acc[i][j]);
  };

  if constexpr (S == 2) {
    // Ring of two: the barrier of a slice sits in front of its last sub-slice.  By then a wave holds the last fragments of
    // the slice in registers, so behind the barrier it has products to issue at once, under which the first fragments of the
    // next slice (certified by the same barrier) and the loads of the slice after that travel.
    v8 px[TM], pw[TN];  // first fragments of the slice about to start
    issue(0, 0);
    __builtin_amdgcn_s_waitcnt(QUAMBA_VMCNT(0));
    __builtin_amdgcn_s_barrier();
    if (nk > 1) issue(1, 1);
    frags(0, 0, px, pw);
    for (int kt = 0; kt + 1 < nk; ++kt) {
      const int cur = kt & 1;
      v8 fx[TM], fw[TN];
      mma(px, pw);
#pragma unroll
      for (int sub = 1; sub + 1 < NSUB; ++sub) {
        frags(cur, sub, fx, fw);
        mma(fx, fw);
      }
      frags(cur, NSUB - 1, fx, fw);
      // this wave's loads of slice kt + 1 have landed and its reads of this slice are done: behind the barrier that holds for all
      __builtin_amdgcn_s_waitcnt(QUAMBA_VMCNT_LGKM0(0));
      __builtin_amdgcn_s_barrier();
      frags(cur ^ 1, 0, px, pw);
      __builtin_amdgcn_sched_barrier(0);  // the requests first: the products below are what covers their latency
      if (kt + 2 < nk) issue(cur, kt + 2);
      mma(fx, fw);
    }
    v8 fx[TM], fw[TN];
    mma(px, pw);
#pragma unroll
    for (int sub = 1; sub < NSUB; ++sub) {
      frags((nk - 1) & 1, sub, fx, fw);
      mma(fx, fw);
    }
  } else {
    // iteration k: slice k has landed (at most the loads issued after it are outstanding), everyone is done with slice k - 1 (its LDS
    // reads are waited for here, not only by the products that use them), whose stage slice k + S - 1 takes
#pragma unroll
    for (int s = 0; s < S - 1; ++s)
      if (s < nk) issue(s, s);
    int stage = 0;
    for (int kt = 0; kt < nk; ++kt) {
      if (kt + S - 2 < nk)
        __builtin_amdgcn_s_waitcnt(QUAMBA_VMCNT_LGKM0((S - 2) * NI));
      else
        __builtin_amdgcn_s_waitcnt(QUAMBA_VMCNT_LGKM0(0));  // tail: fewer slices were issued
      __builtin_amdgcn_s_barrier();
      if (kt + S - 1 < nk) issue(stage == 0 ? S - 1 : stage - 1, kt + S - 1);
#pragma unroll
      for (int sub = 0; sub < NSUB; ++sub) {
        v8 fx[TM], fw[TN];
        frags(stage, sub, fx, fw);
        mma(fx, fw);
      }
      stage = stage + 1 == S ? 0 : stage + 1;
    }
  }

  __syncthreads();  // operand tiles are dead
  char *band = ring + wave * kBandBytes;
  if constexpr (KG > 1) {
    // groups 1 .. KG-1 park their sums lane-major (conflict-free), group 0 adds them in order and stores; its band reuses
    // region (0, tile), which it alone reads
    constexpr int PART = TM * TN * 16 * 64 * 4 > kBandBytes ? TM * TN * 16 * 64 * 4 : kBandBytes, TILES = WGM * WGN;
    static_assert(S * STAGE >= (KG - 1) * TILES * PART, "the groups' sums fit in the ring");
    if (kg > 0) {
      v4f *part = reinterpret_cast<v4f *>(ring + ((kg - 1) * TILES + wtile) * PART);
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            part[((i * TM + j) * 4 + g) * 64 + lane] = v4f{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int o = 0; o < KG - 1; ++o) {
      const v4f *part = reinterpret_cast<const v4f *>(ring + (o * TILES + wtile) * PART);
#pragma unroll
      for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const v4f v = part[((i * TM + j) * 4 + g) * 64 + lane];
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[i][j][4 * g + c] += v[c];
          }
    }
    band = ring + wtile * PART;
  }
  store_wave<O, TM, TN>(acc, m0 + wm * WM, n0 + wn * WN, lane, M, N, epi, band);
}
#undef QUAMBA_VMCNT
#undef QUAMBA_VMCNT_LGKM0

// Up to 16 rows of W and x that do not start on 16 bytes: a workgroup owns 16 columns, its 8 waves split K in contiguous
// ranges, and the fragments go straight from memory to the matrix unit, 16 rows of W against 16 of x (rows past M repeat the
// last one; their results are columns that nobody stores).  The waves' sums are added in LDS.
template <typename T, typename O>
__global__ __launch_bounds__(512) void linear_rows_kernel(const T *__restrict__ x, long long ldx, const T *__restrict__ W, long long ldw, int M,
                                                          int N, int K, LinearEpi epi) {
  constexpr int U = 8, NW = 8;  // pieces of 32 k in flight; waves
  __shared__ float part[NW][16][17];
  typedef typename Half<T>::v8 v8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, c8 = (lane >> 4) * 8;
  const int n0 = blockIdx.x * 16;
  const int pieces = (K + 31) / 32, per = (pieces + NW - 1) / NW, lo = wave * per, hi = min(pieces, lo + per);
  const T *pw = W + (size_t)min(n0 + r, N - 1) * ldw, *px = x + (size_t)min(r, M - 1) * ldx;
  v4f acc = {0.f, 0.f, 0.f, 0.f};
  const int gm = threadIdx.x >> 4, gn = n0 + (threadIdx.x & 15);
  Single one;
  if (threadIdx.x < 256) one = ask1<O>(epi, gm, gn, M, N);
  for (int p = lo; p < hi; p += U) {
    v8 fw[U], fx[U];
#pragma unroll
    for (int u = 0; u < U; ++u) fw[u] = row8(pw, p + u < hi ? (p + u) * 32 + c8 : K, K);
#pragma unroll
    for (int u = 0; u < U; ++u) fx[u] = row8(px, p + u < hi ? (p + u) * 32 + c8 : K, K);
#pragma unroll
    for (int u = 0; u < U; ++u) acc = Half<T>::mfma16(fw[u], fx[u], acc);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) part[wave][r][(lane >> 4) * 4 + e] = acc[e];
  __syncthreads();
  if (threadIdx.x < 256) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += part[w][gm][threadIdx.x & 15];
    put1<O>(epi, one, gm, gn, v);
  }
}

// One to four rows: the job is to read W once, at the rate of a copy.  LANES lanes split K of four adjacent columns in 16-byte
// pieces (64 lanes: 1 KB of a row of W at a time), products and sums in fp32 on the vector unit (at 4 rows half as long as the
// reading), then over lanes and waves in a fixed order.
template <typename T, typename O, int MR, int LANES>
__global__ __launch_bounds__(256) void linear_vec_kernel(const T *__restrict__ x, long long ldx, const T *__restrict__ W, long long ldw, int M,
                                                         int N, int K, LinearEpi epi) {
  constexpr int U = MR == 4 ? 1 : 2, GROUPS = 256 / LANES;  // pieces in flight; column groups of a workgroup
  __shared__ float part[4][MR * 4];
  typedef typename Half<T>::v8 v8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int group = LANES == 64 ? wave : 0, at = LANES == 64 ? lane : (int)threadIdx.x;
  const int n0 = (blockIdx.x * GROUPS + group) * 4;
  const T *pw[4], *px[MR];
#pragma unroll
  for (int j = 0; j < 4; ++j) pw[j] = W + (size_t)min(n0 + j, N - 1) * ldw;
#pragma unroll
  for (int m = 0; m < MR; ++m) px[m] = x + (size_t)min(m, M - 1) * ldx;
  float acc[MR][4];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[m][j] = 0.f;
  const int mine = LANES == 64 ? lane : (int)threadIdx.x, gm = mine >> 2, gn = n0 + (mine & 3);
  Single one;
  if (mine < MR * 4) one = ask1<O>(epi, gm, gn, M, N);
  for (int k = at * 8; k < K; k += LANES * 8 * U) {
    v8 w[U][4], v[U][MR];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[u][j] = row8(pw[j], k + u * LANES * 8, K);
#pragma unroll
      for (int m = 0; m < MR; ++m) v[u][m] = row8(px[m], k + u * LANES * 8, K);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[m][j] = fmaf(to_f32(v[u][m][e]), to_f32(w[u][j][e]), acc[m][j]);
  }
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v = acc[m][j];
#pragma unroll
      for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
      if (lane == 0) part[wave][m * 4 + j] = v;
    }
  __syncthreads();
  if (mine < MR * 4)
    put1<O>(epi, one, gm, gn, LANES == 64 ? part[wave][mine] : part[0][mine] + part[1][mine] + part[2][mine] + part[3][mine]);
}

// Rows of any alignment copied to rows of a multiple of 64 elements, zeros behind K: both operands in one launch (or one of them:
// the other has no chunks).  A division of 64 bits is as long as the copy, so only what needs one does it.  A launch counts its threads
// along a dimension in 32 bits, hence the second one.
constexpr long long kCopyGrid = 1 << 20;
template <typename T>
struct RowCopy {
  const T *from;
  long long ld, chunks;  // of 8 elements
  T *to;
};
template <typename T>
__global__ __launch_bounds__(256) void align_rows_kernel(RowCopy<T> a, RowCopy<T> b, int per_row, int K) {
  long long i = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  const bool second = i >= a.chunks;
  if (second) i -= a.chunks;
  const RowCopy<T> &c = second ? b : a;
  if (i >= c.chunks) return;
  const long long row = a.chunks + b.chunks <= INT_MAX ? (long long)((unsigned)i / (unsigned)per_row) : i / per_row;
  const int k = (int)(i - row * per_row) * 8;
  *reinterpret_cast<typename Half<T>::v8 *>(c.to + i * 8) = row8(c.from + row * c.ld, k, K);
}

std::atomic<int> g_linear_variant{-1};

// Which kernel:
//   0, 1 = any alignment, 64 x 64 and 128 x 128 tiles     2 = rows straight to the matrix unit (M <= 16)     10 = vector unit (M <= 4)
//   direct-to-LDS tiles: 3 = 256 x 320, 4 = 256 x 256 (8 waves, ring of 2)   5 = 128 x 128 (ring of 2, two workgroups a CU)
//   6 = 64 x 64 (ring of 3)   7 = 32 x 32, 4 K groups   8 = 64 x 64, 2 K groups   9 = 128 x 128, 2 K groups   11 = 32 x 32, 8 K groups
// The aligned ones by how many of their tiles are resident at once on 256 CUs: 11, 8, 9 and 3, 4 one to a CU, 7, 6 and 5 two.  Up to
// one round the smaller tile wins, past it the next.  us a call on both sides of each bound (M x N x K, bf16, calls of
// a captured graph):
//   one or two rows, 10 against 7 and 11, W from memory: 1 x 10240 x 2560 12.6, 13.5 and 16.4, 2 x 2560 x 5120 10.8, 17.2 and 12.7; at three
//   rows 18.7, 13.5 and 16.5, at 2 x 10240 x 2560 already 14.7, 13.5 and 16.6
//   11 against 7, 64 rows: N = 2560 K = 5120 10.9 and 12.8, K = 2048 6.5 and 7.0, K = 1024 4.4 and 4.5; 288 tiles K = 5120 20.2 and 18.9
//   7 against 8: 512 tiles (64 x 8192 x 2560) 11.4 and 12.0; 576 14.7 and 12.2
//   8 against 6: 256 tiles (256 x 4096 x 2560) 12.3 and 15.0; 288 21.8 and 19.3
//   6 against 9: 512 tiles (512 x 4096 x 2560) 21.2 and 24.5; 560 27.2 and 24.9, at K = 1280 15.4 and 16.1; 640 27.6 and 25.0
//   9 against 5: 256 tiles (1024 x 4096 x 2560) 28.6 and 33.9; 288 48.7 and 35.4
//   5 against 4: 512 tiles (2048 x 4096 x 2560) 44.1 and 60.2; 576 70.5 and 61.1
//   3, 4 and 5 past that: 2048 x 10240 x 2560 90, 144 and 128; 4096 x 4096 x 4096 122, 109 and 130; 2560 x 8192 x 4096 232, 204 and 184
// Rows off 16 bytes that are not copied: 10 against 2 at 1 x 2560 x 2561 6.2 and 8.0, at 4 x 10240 x 2561 23.4 and 19.9, at 4 x 2560 x 5121
// 11.3 and 10.8; 0 against 1 at 240 tiles of 128 x 128 (2048 x 1920 x 2561) 62 and 68, at 288 98 and 69; copied, these take 38 and 45.
constexpr int kLinearKinds = 12;

int pick_kind(int M, int N, int K, bool wide, int forced) {
  if (forced >= 0 && forced < kLinearKinds && (forced != 2 || M <= 16) && (forced != 10 || M <= 4) && (forced < 3 || forced == 10 || wide))
    return forced;
  if (M <= 2 || (M <= 4 && !wide)) return 10;
  auto tiles = [&](long long bm, long long bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  const long long t32 = tiles(32, 32), t64 = tiles(64, 64), t128 = tiles(128, 128);
  if (!wide) return M <= 16 ? 2 : (t128 >= 256 ? 1 : 0);
  if (t32 <= 256 && K >= 2048) return 11;
  if (t32 <= 512) return 7;
  if (t64 <= 256) return 8;
  if (t64 <= 560) return 6;
  if (t128 <= 256) return 9;
  if (t128 <= 512) return 5;
  // rounds of 256 CUs times the area of a tile; the 128 x 128 ones run two to a CU at 0.9 of the others' rate (8192 x 4096 x 8192, whole
  // rounds of both: 499 us and 428)
  auto rounds = [](long long t, long long n) { return (double)((t + n - 1) / n); };
  const double e3 = rounds(tiles(256, 320), 256) * (256.0 * 320.0), e4 = rounds(tiles(256, 256), 256) * (256.0 * 256.0);
  const double e5 = rounds(t128, 512) * (2.0 * 128.0 * 128.0) * 1.1;
  return e3 < e4 && e3 < e5 ? 3 : (e4 <= e5 ? 4 : 5);
}

int too_large(int M, int N) { return fail(QUAMBA_EUNSUPPORTED, "linear: %d x %d outputs are more than one launch takes", M, N); }

template <typename T, typename O, int BM, int BN, int WGM, int WGN, int S, int BKB, int OCC, int KG>
int run_dma(const T *x, long long ldx, const T *W, long long ldw, int M, int N, int K, const LinearEpi &epi, hipStream_t st) {
  constexpr int lds = S * (BM + BN) * BKB;
  // the attribute is per device: one bit per device index, set after the first successful call there
  static std::atomic<unsigned long long> attr_set{0};
  int dev = 0;
  QUAMBA_HIP(hipGetDevice(&dev));
  const unsigned long long bit = 1ull << (dev & 63);
  if (!(attr_set.load(std::memory_order_acquire) & bit)) {
    QUAMBA_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(&linear_dma_kernel<T, O, BM, BN, WGM, WGN, S, BKB, OCC, KG>),
                                   hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    attr_set.fetch_or(bit, std::memory_order_release);
  }
  const int tiles_m = (M + BM - 1) / BM, tiles_n = (N + BN - 1) / BN;
  if (!launchable((long long)tiles_m * tiles_n, 64 * WGM * WGN * KG)) return too_large(M, N);
  hipLaunchKernelGGL((linear_dma_kernel<T, O, BM, BN, WGM, WGN, S, BKB, OCC, KG>), dim3(tiles_m * tiles_n), dim3(64 * WGM * WGN * KG), lds, st,
                     x, ldx, W, ldw, M, N, K, epi, tiles_m, tiles_n);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

template <typename T, typename O, int TM, int TN>
int run_any(const T *x, long long ldx, const T *W, long long ldw, int M, int N, int K, const LinearEpi &epi, hipStream_t st) {
  const int tiles_m = (M + 64 * TM - 1) / (64 * TM), tiles_n = (N + 64 * TN - 1) / (64 * TN);
  if (!launchable((long long)tiles_m * tiles_n, 256)) return too_large(M, N);
  hipLaunchKernelGGL((linear_any_kernel<T, O, TM, TN>), dim3(tiles_m * tiles_n), dim3(256), 0, st, x, ldx, W, ldw, M, N, K, epi, tiles_m,
                     tiles_n);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

template <typename T, typename O, int MR>
int run_vec(const T *x, long long ldx, const T *W, long long ldw, int M, int N, int K, const LinearEpi &epi, hipStream_t st) {
  if (!launchable(K <= 1024 ? (N + 15) / 16 : (N + 3) / 4, 256)) return too_large(M, N);
  if (K <= 1024)
    hipLaunchKernelGGL((linear_vec_kernel<T, O, MR, 64>), dim3((N + 15) / 16), dim3(256), 0, st, x, ldx, W, ldw, M, N, K, epi);
  else
    hipLaunchKernelGGL((linear_vec_kernel<T, O, MR, 256>), dim3((N + 3) / 4), dim3(256), 0, st, x, ldx, W, ldw, M, N, K, epi);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

// Rows that the direct-to-LDS kernels take: they start on 16 bytes, and a tile's (at most 320) lie within the 2^31 bytes that a lane's
// offset reaches.
constexpr int kLongRow = 1 << 21;
bool rows_wide(const void *p, long long ld, int K) { return aligned(p, 16) && ld % 8 == 0 && K % 8 == 0 && ld < kLongRow; }
constexpr int kCopyUnit = 64;  // elements a copied row is a multiple of: whole 128-byte lines
size_t aligned_bytes(int rows, int K) { return align_up((size_t)rows * align_up(K, kCopyUnit) * 2, 256); }
// More rows than the streaming kernels take: operands of any alignment are worth copying to 16-byte rows first (17 x 2560 x 2561 with the copy
// 16 us, without 40; 16 rows without 9.6), unless the copies would again be too long for the kernels that want them.
bool copies(int M, int K) { return M > 16 && align_up(K, kCopyUnit) < kLongRow; }

struct LinearPlan {
  bool copy_x, copy_w;
  int kind;
};
LinearPlan plan_linear(int M, int N, int K, bool wide_x, bool wide_w, size_t ws_bytes) {
  const int forced = g_linear_variant.load(std::memory_order_relaxed);
  const bool copy = copies(M, K) && !(wide_x && wide_w) && (wide_x ? 0 : aligned_bytes(M, K)) + (wide_w ? 0 : aligned_bytes(N, K)) <= ws_bytes && forced < 0;
  return LinearPlan{copy && !wide_x, copy && !wide_w, pick_kind(M, N, copy ? (int)align_up(K, 8) : K, copy || (wide_x && wide_w), forced)};
}

template <typename T, typename O>
int run_linear(const T *x, long long ldx, const T *W, long long ldw, int M, int N, int K, const LinearEpi &epi, void *ws, size_t ws_bytes,
               hipStream_t st) {
  if (((M + 31LL) / 32) * ((N + 31LL) / 32) > INT_MAX) return too_large(M, N);
  if (M > 1 << 30 || N > 1 << 30 || K > 1 << 30) return fail(QUAMBA_EUNSUPPORTED, "linear: M=%d N=%d K=%d (at most 2^30 each)", M, N, K);
  const LinearPlan p = plan_linear(M, N, K, rows_wide(x, ldx, K), rows_wide(W, ldw, K), ws_bytes);
  if (p.copy_x || p.copy_w) {
    char *at = static_cast<char *>(ws);
    const int per_row = (int)align_up(K, kCopyUnit) / 8;
    const RowCopy<T> cx{x, ldx, p.copy_x ? (long long)M * per_row : 0, reinterpret_cast<T *>(at)};
    const RowCopy<T> cw{W, ldw, p.copy_w ? (long long)N * per_row : 0, reinterpret_cast<T *>(at + (p.copy_x ? aligned_bytes(M, K) : 0))};
    const long long wgs = (cx.chunks + cw.chunks + 255) / 256;
    hipLaunchKernelGGL(align_rows_kernel<T>, dim3((unsigned)(wgs < kCopyGrid ? wgs : kCopyGrid), (unsigned)((wgs + kCopyGrid - 1) / kCopyGrid)),
                       dim3(256), 0, st, cx, cw, per_row, K);
    QUAMBA_LAUNCH_CHECK();
    if (p.copy_x) x = cx.to, ldx = per_row * 8LL;
    if (p.copy_w) W = cw.to, ldw = per_row * 8LL;
    K = (int)align_up(K, 8);  // no further: the other operand may not be a copy, and what stands behind its K is not zero
  }
  switch (p.kind) {
    case 0: return run_any<T, O, 1, 1>(x, ldx, W, ldw, M, N, K, epi, st);
    case 1: return run_any<T, O, 2, 2>(x, ldx, W, ldw, M, N, K, epi, st);
    case 2:
      if (!launchable((N + 15) / 16, 512)) return too_large(M, N);
      hipLaunchKernelGGL((linear_rows_kernel<T, O>), dim3((N + 15) / 16), dim3(512), 0, st, x, ldx, W, ldw, M, N, K, epi);
      QUAMBA_LAUNCH_CHECK();
      return QUAMBA_OK;
    case 3: return run_dma<T, O, 256, 320, 4, 2, 2, 128, 2, 1>(x, ldx, W, ldw, M, N, K, epi, st);
    case 4: return run_dma<T, O, 256, 256, 4, 2, 2, 128, 2, 1>(x, ldx, W, ldw, M, N, K, epi, st);
    case 6: return run_dma<T, O, 64, 64, 2, 2, 3, 128, 2, 1>(x, ldx, W, ldw, M, N, K, epi, st);
    case 7: return run_dma<T, O, 32, 32, 1, 1, 3, 256, 2, 4>(x, ldx, W, ldw, M, N, K, epi, st);
    case 8: return run_dma<T, O, 64, 64, 2, 2, 3, 256, 2, 2>(x, ldx, W, ldw, M, N, K, epi, st);
    case 9: return run_dma<T, O, 128, 128, 2, 2, 4, 128, 2, 2>(x, ldx, W, ldw, M, N, K, epi, st);
    case 10:
      if (M <= 1) return run_vec<T, O, 1>(x, ldx, W, ldw, M, N, K, epi, st);
      if (M <= 2) return run_vec<T, O, 2>(x, ldx, W, ldw, M, N, K, epi, st);
      return run_vec<T, O, 4>(x, ldx, W, ldw, M, N, K, epi, st);
    case 11: return run_dma<T, O, 32, 32, 1, 1, 3, 512, 2, 8>(x, ldx, W, ldw, M, N, K, epi, st);
    default: return run_dma<T, O, 128, 128, 2, 2, 2, 128, 2, 1>(x, ldx, W, ldw, M, N, K, epi, st);
  }
}

}  // namespace

}  // namespace quamba

using namespace quamba;

extern "C" {

size_t quamba_linear_workspace_bytes(int M, int N, int K) {
  if (M < 0 || N <= 0 || K <= 0) {
    fail(QUAMBA_EINVAL, "linear: M=%d N=%d K=%d", M, N, K);
    return 0;
  }
  return copies(M, K) ? aligned_bytes(M, K) + aligned_bytes(N, K) : 256;
}

int quamba_linear(int type, const void *x, int ldx, const void *W, int ldw, const float *bias, const void *residual, int ldr,
                  int M, int N, int K, int act, int out_type, void *out, int ldo, void *ws, size_t ws_bytes, void *stream) {
  if (type != QUAMBA_TYPE_F16 && type != QUAMBA_TYPE_BF16) return fail(QUAMBA_EUNSUPPORTED, "linear: operand type %d", type);
  if (out_type != type && out_type != QUAMBA_TYPE_F32)
    return fail(QUAMBA_EUNSUPPORTED, "linear: output type %d for operands of type %d", out_type, type);
  if (act < QUAMBA_ACT_NONE || act > QUAMBA_ACT_SIGMOID) return fail(QUAMBA_EUNSUPPORTED, "linear: activation %d", act);
  if (M < 0 || N <= 0 || K <= 0) return fail(QUAMBA_EINVAL, "linear: M=%d N=%d K=%d", M, N, K);
  if (ldx < K || ldw < K || ldo < N || (residual && ldr < N))
    return fail(QUAMBA_EINVAL, "linear: row strides ldx=%d ldw=%d ldr=%d ldo=%d are shorter than the rows", ldx, ldw, ldr, ldo);
  if (M == 0) return QUAMBA_OK;
  if (!x || !W || !out) return fail(QUAMBA_EINVAL, "linear: NULL pointer");
  const size_t osz = out_type == QUAMBA_TYPE_F32 ? 4 : 2;
  if (!aligned(x, 2) || !aligned(W, 2) || !aligned(out, osz) || !aligned(residual, osz) || !aligned(bias, 4))
    return fail(QUAMBA_EINVAL, "linear: a buffer is not aligned to its elements");
  if (residual == out && ldr != ldo) return fail(QUAMBA_EINVAL, "linear: residual in place with ldr=%d, ldo=%d", ldr, ldo);
  if (ws && !aligned(ws, 256)) return fail(QUAMBA_EINVAL, "linear: workspace must be 256-byte aligned");
  const LinearEpi e{bias, residual, out, ldr, ldo, act};
  hipStream_t st = as_stream(stream);
  if (type == QUAMBA_TYPE_F16) {
    const auto *a = static_cast<const _Float16 *>(x), *b = static_cast<const _Float16 *>(W);
    return out_type == QUAMBA_TYPE_F32 ? run_linear<_Float16, float>(a, ldx, b, ldw, M, N, K, e, ws, ws ? ws_bytes : 0, st)
                                       : run_linear<_Float16, _Float16>(a, ldx, b, ldw, M, N, K, e, ws, ws ? ws_bytes : 0, st);
  }
  const auto *a = static_cast<const __bf16 *>(x), *b = static_cast<const __bf16 *>(W);
  return out_type == QUAMBA_TYPE_F32 ? run_linear<__bf16, float>(a, ldx, b, ldw, M, N, K, e, ws, ws ? ws_bytes : 0, st)
                                     : run_linear<__bf16, __bf16>(a, ldx, b, ldw, M, N, K, e, ws, ws ? ws_bytes : 0, st);
}

}  // extern "C"

extern "C" void quamba_debug_set_linear_variant(int v) { quamba::g_linear_variant.store(v); }

extern "C" int quamba_debug_linear_kind(int M, int N, int K, int ldx, int ldw, size_t ws_bytes) {
  if (M <= 0 || N <= 0 || K <= 0 || ldx < K || ldw < K) return -2;
  const quamba::LinearPlan p = quamba::plan_linear(M, N, K, quamba::rows_wide(nullptr, ldx, K), quamba::rows_wide(nullptr, ldw, K), ws_bytes);
  return p.kind + (p.copy_x ? 16 : 0) + (p.copy_w ? 32 : 0);
}
