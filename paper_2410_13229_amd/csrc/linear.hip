// 16-bit projection with its epilogue: out = act(x W^T + bias) + residual, fp16 or bf16 operands, fp32 sums.
//
//   acc[m, n] = sum_k x[m, k] W[n, k]          x [M, K], W [N, K], both K-contiguous
//
// The operands go through the matrix units as they are (products of 16-bit values are exact in fp32), sums stay in
// fp32 up to the epilogue, and the result is rounded once, to the output's type.
#include <atomic>
#include <climits>

#include "common.h"
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
  bool wide;  // residual and output rows start on 16 bytes
};

// The activation is evaluated in fp32.  exp2 of a large positive argument is infinite and its reciprocal 0, so the
// sigmoid needs no branch; SiLU's v * 0 at v = -inf would be NaN where the limit is -0, as v / (1 + inf) gives.
__device__ __forceinline__ float activate(float v, int act) {
  constexpr float LOG2E = 1.44269504088896340736f;
  switch (act) {
    case QUAMBA_ACT_RELU: return v < 0.f ? 0.f : v;  // keeps NaN
    case QUAMBA_ACT_SILU: return v == -INFINITY ? 0.f : v / (1.f + __builtin_amdgcn_exp2f(-v * LOG2E));
    case QUAMBA_ACT_GELU: {
      // 0.5 v erfc(-v / sqrt 2): no cancellation for negative v, 0 at -inf instead of -inf * 0
      const float e = erfcf(v * -0.70710678118654752440f);
      return e == 0.f ? 0.f : 0.5f * v * e;
    }
    case QUAMBA_ACT_GELU_TANH: {
      // 0.5 v (1 + tanh u) = v sigmoid(2 u), u = sqrt(2 / pi) (v + 0.044715 v^3)
      const float u2 = 1.59576912160573071176f * v * (1.f + 0.044715f * v * v);
      const float d = 1.f + __builtin_amdgcn_exp2f(-u2 * LOG2E);
      return d == INFINITY ? 0.f : v / d;
    }
    case QUAMBA_ACT_SIGMOID: return 1.f / (1.f + __builtin_amdgcn_exp2f(-v * LOG2E));
    default: return v;
  }
}

template <typename O>
__device__ __forceinline__ void emit1(const LinearEpi &e, int gm, int gn, float v) {
  if (e.bias) v += e.bias[gn];
  v = activate(v, e.act);
  if (e.res) v += to_f32(static_cast<const O *>(e.res)[(size_t)gm * e.ldr + gn]);
  static_cast<O *>(e.out)[(size_t)gm * e.ldo + gn] = from_f32<O>(v);
}

__device__ __forceinline__ v4f zero4() { return v4f{0.f, 0.f, 0.f, 0.f}; }

// Byte offset of 16-byte chunk `chunk` of tile row `row` for rows of BKB bytes: any 16 consecutive rows read at one
// logical chunk hit 16 different bank groups (with 64-byte rows four rows span the 64 banks, with 128-byte rows two).
template <int BKB>
__device__ __forceinline__ int swz(int row, int chunk) {
  if constexpr (BKB == 64) return row * 64 + ((chunk ^ ((row >> 2) & 3)) << 4);
  else if constexpr (BKB == 128) return row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4);
  else return row * 256 + ((chunk ^ (row & 15)) << 4);
}

// A wave's TM x TN tiles of 32 x 32 sums: register r of lane l in tile (i, j) is column n_base + 32 i + 8 (r / 4) + 4 (l / 32)
// + r % 4 of row m_base + 32 j + l % 32.  A band of 32 rows and up to 64 columns at a time goes through a region of LDS that
// only this wave uses (fp32, rows 16 bytes further apart than they are long), so that bias, residual and output are
// taken 16 bytes a lane along the rows, and the epilogue's code exists once and not per tile.
constexpr int kBandPitch = 64 * 4 + 16;
constexpr int kBandBytes = 32 * kBandPitch;

template <typename O>
__device__ __forceinline__ void store_band(const LinearEpi &e, int m0, int n0, int cols, int lane, int M, int N, const char *band) {
  constexpr int E = 16 / sizeof(O);  // elements of a 16-byte store
  const int per_row = cols / E;
  const int cc = lane % per_row * E, gn = n0 + cc;
  if (gn >= N) return;
  const bool whole = e.wide && gn + E <= N;
  float b[E];
#pragma unroll
  for (int i = 0; i < E; ++i) b[i] = e.bias && gn + i < N ? e.bias[gn + i] : 0.f;
#pragma unroll 1
  for (int r = lane / per_row; r < 32; r += 64 / per_row) {
    const int gm = m0 + r;
    if (gm >= M) return;
    float v[E];
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const v4f t = *reinterpret_cast<const v4f *>(band + r * kBandPitch + (cc + i) * 4);
#pragma unroll
      for (int c = 0; c < 4; ++c) v[i + c] = t[c] + b[i + c];
    }
    if (e.act != QUAMBA_ACT_NONE) {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = activate(v[i], e.act);
    }
    const O *res = static_cast<const O *>(e.res) + (size_t)gm * e.ldr + gn;
    O *out = static_cast<O *>(e.out) + (size_t)gm * e.ldo + gn;
    typedef O vO __attribute__((ext_vector_type(E)));
    if (whole) {
      if (e.res) {
        const vO t = *reinterpret_cast<const vO *>(res);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] += to_f32(t[i]);
      }
      vO t;
#pragma unroll
      for (int i = 0; i < E; ++i) t[i] = from_f32<O>(v[i]);
      *reinterpret_cast<vO *>(out) = t;
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (gn + i < N) out[i] = from_f32<O>(e.res ? v[i] + to_f32(res[i]) : v[i]);
    }
  }
}

// `partial`: raw sums to partial[M, N] instead (K split over the grid).
template <typename O, int TM, int TN>
__device__ __forceinline__ void store_wave(const v16f (&acc)[TN][TM], int m_base, int n_base, int lane, int M, int N, const LinearEpi &e,
                                           float *partial, char *band) {
  constexpr int PER = (TN + 1) / 2;  // bands of columns
#pragma unroll 1
  for (int step = 0; step < TM * PER; ++step) {
    const int j = step / PER, i0 = step % PER * 2;
#pragma unroll
    for (int s = 0; s < TM * PER; ++s)
      if (s == step) {
#pragma unroll
        for (int i = s % PER * 2; i < TN && i < s % PER * 2 + 2; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<v4f *>(band + (lane & 31) * kBandPitch + ((i & 1) * 32 + 8 * g + 4 * (lane >> 5)) * 4) =
                v4f{acc[i][s / PER][4 * g], acc[i][s / PER][4 * g + 1], acc[i][s / PER][4 * g + 2], acc[i][s / PER][4 * g + 3]};
      }
    const int cols = i0 + 1 < TN ? 64 : 32;
    if (partial) {
      const LinearEpi raw{nullptr, nullptr, partial, 0, N, QUAMBA_ACT_NONE, (N & 3) == 0};
      store_band<float>(raw, m_base + 32 * j, n_base + 32 * i0, cols, lane, M, N, band);
    } else {
      store_band<O>(e, m_base + 32 * j, n_base + 32 * i0, cols, lane, M, N, band);
    }
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

struct KRange {
  int slices;      // K slices of one grid.y index
  float *partial;  // [grid.y, M, N] sums when K is split, else NULL
};

// Any strides and alignments: K in slices of 32 staged through registers (16-byte loads at element addresses, which
// global memory serves at whatever lines they touch), two LDS stages, four waves in 2 x 2.
template <typename T, typename O, int TM, int TN>
__global__ __launch_bounds__(256) void linear_any_kernel(const T *__restrict__ x, long long ldx, const T *__restrict__ W,
                                                         long long ldw, int M, int N, int K, LinearEpi epi, int tiles_m, int tiles_n,
                                                         KRange kr) {
  constexpr int BK = 32, BM = 64 * TM, BN = 64 * TN, STAGE = (BM + BN) * BK * 2;
  constexpr int LDS = 2 * STAGE > 4 * kBandBytes ? 2 * STAGE : 4 * kBandBytes;
  __shared__ __attribute__((aligned(16))) char lds[LDS];
  int tile_m, tile_n;
  tile_of(blockIdx.x, tiles_m, tiles_n, &tile_m, &tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave & 1, wn = wave >> 1;
  const int row = tid >> 2, ch = tid & 3;
  const int k_lo = blockIdx.y * kr.slices * BK;
  const int nk = min((K + BK - 1) / BK - blockIdx.y * kr.slices, kr.slices);

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
    const int gk = k_lo + kt * BK + ch * 8;
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
  store_wave<O, TM, TN>(acc, m0 + wm * TM * 32, n0 + wn * TN * 32, lane, M, N, epi, kr.partial ? kr.partial + (size_t)blockIdx.y * M * N : nullptr,
                        lds + wave * kBandBytes);
}

// 16-byte rows: slices travel with the 16-byte direct-to-LDS loads (no staging registers, no LDS write instructions).  A
// wave-level load writes 64 lanes x 16 bytes at LDS base + 16 lane, 1024 / BKB consecutive tile rows, so the swizzle is applied
// on the global side: each lane fetches the chunk that belongs in its slot.  Chunks past K are fetched from a
// block of zeros, rows past M or N repeat the last row (multiplied, never stored).
// Ring of S stages; KG groups of waves share one tile, group g multiplying the 32-byte sub-slices s with s % KG == g.
__device__ __attribute__((aligned(16))) const unsigned g_zeros[4] = {0, 0, 0, 0};

// s_waitcnt for "at most n vector loads outstanding, nothing else waited for" (vmcnt in bits 3:0 and 15:14, expcnt 6:4,
// lgkmcnt 11:8), and with this wave's LDS reads finished as well
#define QUAMBA_VMCNT(n) (((n) & 0xF) | ((((n) >> 4) & 0x3) << 14) | (0x7 << 4) | (0xF << 8))
#define QUAMBA_VMCNT_LGKM0(n) (((n) & 0xF) | ((((n) >> 4) & 0x3) << 14) | (0x7 << 4))

template <typename T, typename O, int BM, int BN, int WGM, int WGN, int S, int BKB, int OCC, int KG>
__global__ __launch_bounds__(64 * WGM * WGN * KG, OCC) void linear_dma_kernel(const T *__restrict__ x, long long ldx, const T *__restrict__ W,
                                                                              long long ldw, int M, int N, int K, LinearEpi epi, int tiles_m,
                                                                              int tiles_n, KRange kr) {
  constexpr int NW = WGM * WGN * KG, WM = BM / WGM, WN = BN / WGN, TM = WM / 32, TN = WN / 32;
  constexpr int RPI = 1024 / BKB, CPR = BKB / 16, ROWS = BM + BN, NJ = ROWS / RPI, NI = (NJ + NW - 1) / NW, STAGE = ROWS * BKB;
  constexpr int NSUB = BKB / 32 / KG, BKE = BKB / 2;  // sub-slices of a group; elements of a slice
  static_assert(WM % 32 == 0 && WN % 32 == 0 && BM % RPI == 0 && BN % RPI == 0 && BKB / 32 % KG == 0, "tile");
  static_assert((S - 2) * NI <= 63 && S >= 2 && (S > 2 || (NSUB >= 2 && KG == 1)), "ring");
  static_assert(NW * kBandBytes <= S * STAGE || KG > 1, "the bands fit in the ring");
  extern __shared__ __attribute__((aligned(16))) char ring[];

  int tile_m, tile_n;
  tile_of(blockIdx.x, tiles_m, tiles_n, &tile_m, &tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int slice_lo = blockIdx.y * kr.slices;
  const int nk = min((K + BKE - 1) / BKE - slice_lo, kr.slices);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wave / (WGM * WGN), wtile = wave % (WGM * WGN), wm = wtile % WGM, wn = wtile / WGM;

  auto load_row = [&](int i) { return min(wave + NW * i, NJ - 1) * RPI + lane / CPR; };  // a short wave repeats the last group
  auto k_of = [&](int i) {  // first k of this lane's chunk of load i in slice 0; the swizzle's phase follows the row inside its operand
    const int row = load_row(i), lrow = row < BM ? row : row - BM;
    return slice_lo * BKE + ((swz<BKB>(lrow, lane % CPR) - lrow * BKB) >> 4) * 8;
  };
  const T *src[NI];
  int dst[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int row = load_row(i);
    dst[i] = min(wave + NW * i, NJ - 1) * 1024;
    src[i] = (row < BM ? x + (size_t)min(m0 + row, M - 1) * ldx : W + (size_t)min(n0 + row - BM, N - 1) * ldw) + k_of(i);
  }
  const int ragged = K % BKE ? (K / BKE) - slice_lo : -1;  // the slice that ends past K
  auto issue = [&](int stage, int slice) {
    if (slice == ragged) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const void *p = k_of(i) + slice * BKE < K ? static_cast<const void *>(src[i] + slice * BKE) : static_cast<const void *>(g_zeros);
        __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1))) *)p,
                                         (void __attribute__((address_space(3))) *)(ring + stage * STAGE + dst[i]), 16, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1))) *)(src[i] + slice * BKE),
                                         (void __attribute__((address_space(3))) *)(ring + stage * STAGE + dst[i]), 16, 0, 0);
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
  auto frags = [&](int stage, int sub, v8 (&fx)[TM], v8 (&fw)[TN]) {
    const char *lx = ring + stage * STAGE, *lw = lx + BM * BKB;
    const int chunk = (sub * KG + kg) * 2 + (lane >> 5);
#pragma unroll
    for (int j = 0; j < TM; ++j) fx[j] = *reinterpret_cast<const v8 *>(lx + swz<BKB>(wm * WM + j * 32 + (lane & 31), chunk));
#pragma unroll
    for (int i = 0; i < TN; ++i) fw[i] = *reinterpret_cast<const v8 *>(lw + swz<BKB>(wn * WN + i * 32 + (lane & 31), chunk));
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
    // iteration k: slice k has landed (at most the loads issued after it are outstanding), everyone is done with slice k - 1,
    // whose stage slice k + S - 1 takes
#pragma unroll
    for (int s = 0; s < S - 1; ++s)
      if (s < nk) issue(s, s);
    int stage = 0;
    for (int kt = 0; kt < nk; ++kt) {
      if (kt + S - 2 < nk)
        __builtin_amdgcn_s_waitcnt(QUAMBA_VMCNT((S - 2) * NI));
      else
        __builtin_amdgcn_s_waitcnt(QUAMBA_VMCNT(0));  // tail: fewer slices were issued
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
  store_wave<O, TM, TN>(acc, m0 + wm * WM, n0 + wn * WN, lane, M, N, epi, kr.partial ? kr.partial + (size_t)blockIdx.y * M * N : nullptr, band);
}
#undef QUAMBA_VMCNT
#undef QUAMBA_VMCNT_LGKM0

// Few rows: the job is to read W once.  A workgroup owns 16 columns, its NW waves split K in contiguous ranges, and the
// fragments go straight from memory to the matrix unit: 16 rows of W against MT x 16 rows of x (rows past M repeat the
// last one; their results are columns that nobody stores).  The waves' sums are added in LDS.
template <typename T, typename O, int MT, int NW>
__global__ __launch_bounds__(64 * NW) void linear_rows_kernel(const T *__restrict__ x, long long ldx, const T *__restrict__ W, long long ldw,
                                                              int M, int N, int K, LinearEpi epi) {
  constexpr int U = MT == 1 ? 8 : (MT == 2 ? 6 : 4);  // pieces of 32 k in flight
  __shared__ float part[NW][MT * 16][17];
  typedef typename Half<T>::v8 v8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, c8 = (lane >> 4) * 8;
  const int n0 = blockIdx.x * 16;
  const int pieces = (K + 31) / 32, per = (pieces + NW - 1) / NW, lo = wave * per, hi = min(pieces, lo + per);
  const T *pw = W + (size_t)min(n0 + r, N - 1) * ldw;
  const T *px[MT];
#pragma unroll
  for (int j = 0; j < MT; ++j) px[j] = x + (size_t)min(j * 16 + r, M - 1) * ldx;
  v4f acc[MT];
#pragma unroll
  for (int j = 0; j < MT; ++j) acc[j] = zero4();
  for (int p = lo; p < hi; p += U) {
    v8 fw[U], fx[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) fw[u] = row8(pw, p + u < hi ? (p + u) * 32 + c8 : K, K);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < MT; ++j) fx[u][j] = row8(px[j], p + u < hi ? (p + u) * 32 + c8 : K, K);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < MT; ++j) acc[j] = Half<T>::mfma16(fw[u], fx[u][j], acc[j]);
  }
#pragma unroll
  for (int j = 0; j < MT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[wave][j * 16 + r][(lane >> 4) * 4 + e] = acc[j][e];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 256; i += 64 * NW) {
    const int gm = i >> 4, gn = n0 + (i & 15);
    if (gm >= M || gn >= N) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += part[w][gm][i & 15];
    emit1<O>(epi, gm, gn, v);
  }
}

// Sums of a K split added in order, then the epilogue.
template <typename O>
__global__ __launch_bounds__(256) void linear_join_kernel(const float *__restrict__ partial, int splits, int M, int N, LinearEpi epi) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, n = (size_t)M * N;
  if (i >= n) return;
  float v = 0.f;
  for (int s = 0; s < splits; ++s) v += partial[s * n + i];
  emit1<O>(epi, (int)(i / N), (int)(i % N), v);
}

std::atomic<int> g_linear_variant{-1};

struct LinearPlan {
  int kind, splits, slices;
};
//   0 = any 64 x 64   1 = any 128 x 128   2 = rows (M <= 64)
//   3 = dma 256 x 320, 8 waves   4 = dma 256 x 256, 8 waves   5 = dma 128 x 128   6 = dma 64 x 64
//   7 = dma 32 x 32, four K groups   8 = dma 64 x 64, two K groups  9 = dma 128 x 128, two K groups
LinearPlan plan_linear(int M, int N, int K, bool wide, const void *ws, size_t ws_bytes) {
  int kind;
  if (M <= 64) kind = 2;
  else if (!wide) kind = (long long)M * N > 1024 * 1024 ? 1 : 0;
  else kind = 5;
  const int forced = g_linear_variant.load(std::memory_order_relaxed);
  if (forced >= 0 && forced <= 9 && (forced != 2 || M <= 64) && (forced <= 2 || wide)) kind = forced;
  const int slice = kind <= 1 ? 32 : (kind == 7 || kind == 8 ? 128 : 64), n = (K + slice - 1) / slice;
  return LinearPlan{kind, 1, n};
}

template <typename T, typename O, int BM, int BN, int WGM, int WGN, int S, int BKB, int OCC, int KG>
int run_dma(const T *x, long long ldx, const T *W, long long ldw, int M, int N, int K, const LinearEpi &epi, const LinearPlan &p, const KRange &kr,
            hipStream_t st) {
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
  hipLaunchKernelGGL((linear_dma_kernel<T, O, BM, BN, WGM, WGN, S, BKB, OCC, KG>), dim3(tiles_m * tiles_n, p.splits), dim3(64 * WGM * WGN * KG), lds, st,
                     x, ldx, W, ldw, M, N, K, epi, tiles_m, tiles_n, kr);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

template <typename T, typename O, int TM, int TN>
int run_any(const T *x, long long ldx, const T *W, long long ldw, int M, int N, int K, const LinearEpi &epi, const LinearPlan &p, const KRange &kr,
            hipStream_t st) {
  const int tiles_m = (M + 64 * TM - 1) / (64 * TM), tiles_n = (N + 64 * TN - 1) / (64 * TN);
  hipLaunchKernelGGL((linear_any_kernel<T, O, TM, TN>), dim3(tiles_m * tiles_n, p.splits), dim3(256), 0, st, x, ldx, W, ldw, M, N, K, epi, tiles_m,
                     tiles_n, kr);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

template <typename T, typename O, int MT>
int run_rows(const T *x, long long ldx, const T *W, long long ldw, int M, int N, int K, const LinearEpi &epi, hipStream_t st) {
  const dim3 grid((N + 15) / 16);
  if (K <= 1024)
    hipLaunchKernelGGL((linear_rows_kernel<T, O, MT, 4>), grid, dim3(256), 0, st, x, ldx, W, ldw, M, N, K, epi);
  else
    hipLaunchKernelGGL((linear_rows_kernel<T, O, MT, 8>), grid, dim3(512), 0, st, x, ldx, W, ldw, M, N, K, epi);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

template <typename T, typename O>
int run_linear(const T *x, long long ldx, const T *W, long long ldw, int M, int N, int K, const LinearEpi &epi, void *ws, size_t ws_bytes,
               hipStream_t st) {
  if (((M + 31LL) / 32) * ((N + 31LL) / 32) > INT_MAX)
    return fail(QUAMBA_EUNSUPPORTED, "linear: %d x %d outputs are more than one launch takes", M, N);
  const bool wide = aligned(x, 16) && aligned(W, 16) && ldx % 8 == 0 && ldw % 8 == 0 && K % 8 == 0;
  const LinearPlan p = plan_linear(M, N, K, wide, ws, ws_bytes);
  const KRange kr{p.slices, p.splits > 1 ? static_cast<float *>(ws) : nullptr};
  int rc;
  switch (p.kind) {
    case 0: rc = run_any<T, O, 1, 1>(x, ldx, W, ldw, M, N, K, epi, p, kr, st); break;
    case 1: rc = run_any<T, O, 2, 2>(x, ldx, W, ldw, M, N, K, epi, p, kr, st); break;
    case 2:
      if (M <= 16) rc = run_rows<T, O, 1>(x, ldx, W, ldw, M, N, K, epi, st);
      else if (M <= 32) rc = run_rows<T, O, 2>(x, ldx, W, ldw, M, N, K, epi, st);
      else rc = run_rows<T, O, 4>(x, ldx, W, ldw, M, N, K, epi, st);
      break;
    case 3: rc = run_dma<T, O, 256, 320, 4, 2, 2, 128, 2, 1>(x, ldx, W, ldw, M, N, K, epi, p, kr, st); break;
    case 4: rc = run_dma<T, O, 256, 256, 4, 2, 2, 128, 2, 1>(x, ldx, W, ldw, M, N, K, epi, p, kr, st); break;
    case 6: rc = run_dma<T, O, 64, 64, 2, 2, 3, 128, 2, 1>(x, ldx, W, ldw, M, N, K, epi, p, kr, st); break;
    case 7: rc = run_dma<T, O, 32, 32, 1, 1, 3, 256, 2, 4>(x, ldx, W, ldw, M, N, K, epi, p, kr, st); break;
    case 8: rc = run_dma<T, O, 64, 64, 2, 2, 3, 256, 2, 2>(x, ldx, W, ldw, M, N, K, epi, p, kr, st); break;
    case 9: rc = run_dma<T, O, 128, 128, 2, 2, 4, 128, 2, 2>(x, ldx, W, ldw, M, N, K, epi, p, kr, st); break;
    default: rc = run_dma<T, O, 128, 128, 2, 2, 2, 128, 2, 1>(x, ldx, W, ldw, M, N, K, epi, p, kr, st); break;
  }
  if (rc != QUAMBA_OK || p.splits == 1) return rc;
  const size_t n = (size_t)M * N;
  hipLaunchKernelGGL(linear_join_kernel<O>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, kr.partial, p.splits, M, N, epi);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
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
  return 256;
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
  if (ws && !aligned(ws, 16)) return fail(QUAMBA_EINVAL, "linear: workspace must be 16-byte aligned");
  const bool wide_rows = aligned(out, 16) && ldo * osz % 16 == 0 && (!residual || (aligned(residual, 16) && ldr * osz % 16 == 0));
  const LinearEpi e{bias, residual, out, ldr, ldo, act, wide_rows};
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
