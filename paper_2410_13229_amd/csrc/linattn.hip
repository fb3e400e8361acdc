// Linear attention with a decay per head:  S_t = a_t S_{t-1} + k_t v_t^T,  o_t = scale q_t^T S_t,  a_t = exp(min(g_t, 0)),
// S [dk, dv] in fp32 per sequence and value head.
#include <climits>

#include "common.h"
#include "half_util.h"

namespace quamba {

namespace {

struct LinAttnArgs {
  const void *q, *k, *v;
  long long ldq, ldk, ldv;  // elements between tokens
  const float *g;           // NULL: no decay
  long long ldg;            // 0: one decay per head
  const int32_t *lens;      // NULL: L tokens each
  int Bt, L, Hk, Hv, dk, dv;
  float scale;
  void *out;
  long long ldo;
  float *state;  // NULL (prompts only): from zero, not kept
};

constexpr float LOG2E = 1.44269504088896340736f;

// a = exp(min(g, 0)); NaN stays NaN, -inf gives 0
__device__ __forceinline__ float decay_of(float g) { return __builtin_amdgcn_exp2f((g > 0.f ? 0.f : g) * LOG2E); }

// Token by token: a workgroup keeps 16 columns of one head's state in registers, 16 threads with 16 rows each per
// column; every token's products with q are added over those threads.
template <typename T>
__global__ __launch_bounds__(256) void linattn_tokens_kernel(LinAttnArgs a) {
  __shared__ float sq[256], sk[256], red[16][17];
  const int tid = threadIdx.x, c = tid & 15, r0 = (tid >> 4) * 16;
  const int h = blockIdx.y, b = blockIdx.z, col = blockIdx.x * 16 + c, hk = h / (a.Hv / a.Hk);
  const int len = a.lens ? min(max(a.lens[b], 0), a.L) : a.L;
  float *st = a.state ? a.state + ((size_t)b * a.Hv + h) * a.dk * a.dv : nullptr;
  float S[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) S[i] = st && r0 + i < a.dk && col < a.dv ? st[(size_t)(r0 + i) * a.dv + col] : 0.f;
  for (int t = 0; t < len; ++t) {
    const size_t row = (size_t)b * a.L + t;
    sq[tid] = tid < a.dk ? to_f32(static_cast<const T *>(a.q)[row * a.ldq + (size_t)hk * a.dk + tid]) : 0.f;
    sk[tid] = tid < a.dk ? to_f32(static_cast<const T *>(a.k)[row * a.ldk + (size_t)hk * a.dk + tid]) : 0.f;
    __syncthreads();
    const float vv = col < a.dv ? to_f32(static_cast<const T *>(a.v)[row * a.ldv + (size_t)h * a.dv + col]) : 0.f;
    const float al = a.g ? decay_of(a.ldg ? a.g[row * a.ldg + h] : a.g[h]) : 1.f;
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      S[i] = fmaf(al, S[i], sk[r0 + i] * vv);
      o = fmaf(sq[r0 + i], S[i], o);
    }
    red[tid >> 4][c] = o;
    __syncthreads();
    if (tid < 16 && col < a.dv) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) s += red[i][c];
      static_cast<T *>(a.out)[row * a.ldo + (size_t)h * a.dv + col] = from_f32<T>(a.scale * s);
    }
  }
  if (st)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (r0 + i < a.dk && col < a.dv) st[(size_t)(r0 + i) * a.dv + col] = S[i];
}

int check(const char *what, int type, const LinAttnArgs &a) {
  if (type != QUAMBA_TYPE_F16 && type != QUAMBA_TYPE_BF16) return fail(QUAMBA_EUNSUPPORTED, "%s: operand type %d", what, type);
  if (a.Bt < 0 || a.L < 0 || a.Hk <= 0 || a.Hv <= 0 || a.dk <= 0 || a.dv <= 0)
    return fail(QUAMBA_EINVAL, "%s: Bt=%d L=%d Hk=%d Hv=%d dk=%d dv=%d", what, a.Bt, a.L, a.Hk, a.Hv, a.dk, a.dv);
  if (a.Hv % a.Hk) return fail(QUAMBA_EUNSUPPORTED, "%s: %d value heads are no multiple of %d key heads", what, a.Hv, a.Hk);
  if (a.dk > 256 || a.dv > 1024) return fail(QUAMBA_EUNSUPPORTED, "%s: dk=%d dv=%d (at most 256 and 1024)", what, a.dk, a.dv);
  if (a.Bt > 65535 || a.Hv > 65535) return fail(QUAMBA_EUNSUPPORTED, "%s: Bt=%d Hv=%d (at most 65535 each)", what, a.Bt, a.Hv);
  const long long qw = (long long)a.Hk * a.dk, vw = (long long)a.Hv * a.dv;
  if (a.ldq < qw || a.ldk < qw || a.ldv < vw || a.ldo < vw || (a.g && a.ldg != 0 && a.ldg < a.Hv))
    return fail(QUAMBA_EINVAL, "%s: token strides ldq=%lld ldk=%lld ldv=%lld ldo=%lld ldg=%lld are shorter than the rows", what, a.ldq, a.ldk,
                a.ldv, a.ldo, a.ldg);
  if (a.Bt == 0 || a.L == 0) return QUAMBA_OK;
  if (!a.q || !a.k || !a.v || !a.out) return fail(QUAMBA_EINVAL, "%s: NULL pointer", what);
  if (!aligned(a.q, 2) || !aligned(a.k, 2) || !aligned(a.v, 2) || !aligned(a.out, 2) || !aligned(a.g, 4) || !aligned(a.lens, 4))
    return fail(QUAMBA_EINVAL, "%s: a buffer is not aligned to its elements", what);
  if (!aligned(a.state, 16)) return fail(QUAMBA_EINVAL, "%s: state must be 16-byte aligned", what);
  return QUAMBA_OK;
}

}  // namespace

}  // namespace quamba

using namespace quamba;

extern "C" {

size_t quamba_linattn_workspace_bytes(int Bt, int L, int Hk, int Hv, int dk, int dv) {
  if (Bt < 0 || L < 0 || Hk <= 0 || Hv <= 0 || dk <= 0 || dv <= 0) {
    fail(QUAMBA_EINVAL, "linattn: Bt=%d L=%d Hk=%d Hv=%d dk=%d dv=%d", Bt, L, Hk, Hv, dk, dv);
    return 0;
  }
  return 256;
}

int quamba_linattn_prefill(int type, const void *q, int ldq, const void *k, int ldk, const void *v, int ldv, const float *log_decay,
                           int ldg, const int32_t *lens, int Bt, int L, int Hk, int Hv, int dk, int dv, float scale, void *out, int ldo,
                           float *state, void *ws, size_t ws_bytes, void *stream) {
  const LinAttnArgs a{q, k, v, ldq, ldk, ldv, log_decay, ldg, lens, Bt, L, Hk, Hv, dk, dv, scale, out, ldo, state};
  const int rc = check("linattn_prefill", type, a);
  if (rc != QUAMBA_OK || Bt == 0 || L == 0) return rc;
  if (ws && !aligned(ws, 256)) return fail(QUAMBA_EINVAL, "linattn_prefill: workspace must be 256-byte aligned");
  const dim3 grid((dv + 15) / 16, Hv, Bt);
  if (type == QUAMBA_TYPE_F16)
    hipLaunchKernelGGL(linattn_tokens_kernel<_Float16>, grid, dim3(256), 0, as_stream(stream), a);
  else
    hipLaunchKernelGGL(linattn_tokens_kernel<__bf16>, grid, dim3(256), 0, as_stream(stream), a);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

int quamba_linattn_step(int type, const void *q, int ldq, const void *k, int ldk, const void *v, int ldv, const float *log_decay,
                        int ldg, int Bt, int Hk, int Hv, int dk, int dv, float scale, void *out, int ldo, float *state, void *stream) {
  const LinAttnArgs a{q, k, v, ldq, ldk, ldv, log_decay, ldg, nullptr, Bt, 1, Hk, Hv, dk, dv, scale, out, ldo, state};
  const int rc = check("linattn_step", type, a);
  if (rc != QUAMBA_OK || Bt == 0) return rc;
  if (!state) return fail(QUAMBA_EINVAL, "linattn_step: state is required");
  const dim3 grid((dv + 15) / 16, Hv, Bt);
  if (type == QUAMBA_TYPE_F16)
    hipLaunchKernelGGL(linattn_tokens_kernel<_Float16>, grid, dim3(256), 0, as_stream(stream), a);
  else
    hipLaunchKernelGGL(linattn_tokens_kernel<__bf16>, grid, dim3(256), 0, as_stream(stream), a);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

}  // extern "C"
