// 16-bit projection with its epilogue: out = act(x W^T + bias) + residual, fp16 or bf16 operands, fp32 sums.
//
//   acc[m, n] = sum_k x[m, k] W[n, k]          x [M, K], W [N, K], both K-contiguous
//
// The operands go through the matrix units as they are (products of 16-bit values are exact in fp32), sums stay in
// fp32 up to the epilogue, and the result is rounded once, to the output's type.
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

// Byte offset of 16-byte chunk `chunk` (0..3) of row `row` of 64 bytes: any 16 consecutive rows read at one logical
// chunk hit 16 different bank groups.
__device__ __forceinline__ int swz64(int row, int chunk) { return row * 64 + ((chunk ^ ((row >> 2) & 3)) << 4); }

// Any strides and alignments: 64 x 64 tiles, K in slices of 32 staged through registers, element loads past which
// nothing is read (rows and columns outside count as zero).
template <typename T, typename O>
__global__ __launch_bounds__(256) void linear_any_kernel(const T *__restrict__ x, long long ldx, const T *__restrict__ W,
                                                         long long ldw, int M, int N, int K, LinearEpi epi, int tiles_n) {
  constexpr int BK = 32;
  __shared__ __attribute__((aligned(16))) char lds[2][128 * BK * 2];
  const int m0 = blockIdx.x / tiles_n * 64, n0 = blockIdx.x % tiles_n * 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave & 1, wn = wave >> 1;
  const int row = tid >> 2, ch = tid & 3;

  v16f acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;

  typename Half<T>::v8 rx, rw;
  auto fetch = [&](int k0) {
    const int gk = k0 + ch * 8, gm = m0 + row, gn = n0 + row;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      rx[e] = gm < M && gk + e < K ? x[(size_t)gm * ldx + gk + e] : static_cast<T>(0.f);
      rw[e] = gn < N && gk + e < K ? W[(size_t)gn * ldw + gk + e] : static_cast<T>(0.f);
    }
  };
  auto park = [&](int buf) {
    *reinterpret_cast<typename Half<T>::v8 *>(lds[buf] + swz64(row, ch)) = rx;
    *reinterpret_cast<typename Half<T>::v8 *>(lds[buf] + 64 * BK * 2 + swz64(row, ch)) = rw;
  };

  const int nk = (K + BK - 1) / BK;
  fetch(0);
  park(0);
  __syncthreads();
  for (int kt = 0; kt < nk; ++kt) {
    const int buf = kt & 1;
    if (kt + 1 < nk) fetch((kt + 1) * BK);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int chunk = s * 2 + (lane >> 5);
      const auto fx = *reinterpret_cast<const typename Half<T>::v8 *>(lds[buf] + swz64(wm * 32 + (lane & 31), chunk));
      const auto fw = *reinterpret_cast<const typename Half<T>::v8 *>(lds[buf] + 64 * BK * 2 + swz64(wn * 32 + (lane & 31), chunk));
      acc = Half<T>::mfma32(fw, fx, acc);
    }
    if (kt + 1 < nk) park(buf ^ 1);
    __syncthreads();
  }
  const int gm = m0 + wm * 32 + (lane & 31);
  if (gm >= M) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int gn = n0 + wn * 32 + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
    if (gn < N) emit1<O>(epi, gm, gn, acc[r]);
  }
}

template <typename T, typename O>
int run_linear(const T *x, long long ldx, const T *W, long long ldw, int M, int N, int K, const LinearEpi &epi, hipStream_t st) {
  const long long tiles_m = (M + 63LL) / 64, tiles_n = (N + 63LL) / 64;
  if (tiles_m * tiles_n > INT_MAX) return fail(QUAMBA_EUNSUPPORTED, "linear: %d x %d outputs are more than one launch takes", M, N);
  hipLaunchKernelGGL((linear_any_kernel<T, O>), dim3((unsigned)(tiles_m * tiles_n)), dim3(256), 0, st, x, ldx, W, ldw, M, N, K, epi,
                     (int)tiles_n);
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
  const LinearEpi e{bias, residual, out, ldr, ldo, act};
  hipStream_t st = as_stream(stream);
  if (type == QUAMBA_TYPE_F16) {
    const auto *a = static_cast<const _Float16 *>(x), *b = static_cast<const _Float16 *>(W);
    return out_type == QUAMBA_TYPE_F32 ? run_linear<_Float16, float>(a, ldx, b, ldw, M, N, K, e, st)
                                       : run_linear<_Float16, _Float16>(a, ldx, b, ldw, M, N, K, e, st);
  }
  const auto *a = static_cast<const __bf16 *>(x), *b = static_cast<const __bf16 *>(W);
  return out_type == QUAMBA_TYPE_F32 ? run_linear<__bf16, float>(a, ldx, b, ldw, M, N, K, e, st)
                                     : run_linear<__bf16, __bf16>(a, ldx, b, ldw, M, N, K, e, st);
}

}  // extern "C"
