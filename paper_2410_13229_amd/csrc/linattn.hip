// Linear attention with a decay per head:  S_t = a_t S_{t-1} + k_t v_t^T,  o_t = scale q_t^T S_t,  a_t = exp(min(g_t, 0)),
// S [dk, dv] in fp32 per sequence and value head.
#include <atomic>
#include <cfloat>
#include <climits>
#include <cstddef>
#include <type_traits>

#include "common.h"
#include "device_util.h"
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

// Below ln 2^-126 exp leaves fp32's normal range: nothing of the past remains.
__device__ __forceinline__ bool forgets(float g) { return g < -87.33654f; }

// a = exp(min(g, 0)); NaN stays NaN, -inf gives 0
__device__ __forceinline__ float decay_of(float g) { return forgets(g) ? 0.f : __builtin_amdgcn_exp2f((g > 0.f ? 0.f : g) * LOG2E); }

// One token: bound by reading and writing the state (64 sequences, 80 heads of 128 x 64: 336 MB, at the rate a copy reaches 66 us).
// A workgroup takes 64 columns of one head's state, rows in turn over its threads, V columns a thread (4: 16-byte accesses along
// the rows); all of its reads leave before anything is waited for.  Row sums of q S are added over the lanes, then over the
// waves, in a fixed order.
template <typename T, int V, int RPT>
__global__ __launch_bounds__(256) void linattn_step_kernel(LinAttnArgs a) {
  constexpr int LPR = 64 / V, RPP = 256 / LPR;  // lanes along a row, rows at a time
  typedef float vf __attribute__((ext_vector_type(V)));
  __shared__ float sq[RPT * RPP], sk[RPT * RPP], red[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r0 = tid / LPR, cc = tid % LPR * V;
  const int h = blockIdx.y, b = blockIdx.z, col = blockIdx.x * 64 + cc, hk = h / (a.Hv / a.Hk);
  float *st = a.state + ((size_t)b * a.Hv + h) * a.dk * a.dv;
  const bool in = col < a.dv;  // V = 4: dv is a multiple of 4
  vf S[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int row = r0 + i * RPP;
    S[i] = vf(0.f);
    if (in && row < a.dk) S[i] = *reinterpret_cast<const vf *>(st + (size_t)row * a.dv + col);
  }
  const T *q = static_cast<const T *>(a.q) + (size_t)b * a.ldq + (size_t)hk * a.dk, *k = static_cast<const T *>(a.k) + (size_t)b * a.ldk + (size_t)hk * a.dk;
  for (int i = tid; i < RPT * RPP; i += 256) {
    sq[i] = i < a.dk ? to_f32(q[i]) : 0.f;
    sk[i] = i < a.dk ? to_f32(k[i]) : 0.f;
  }
  float v[V], o[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    v[e] = in ? to_f32(static_cast<const T *>(a.v)[(size_t)b * a.ldv + (size_t)h * a.dv + col + e]) : 0.f;
    o[e] = 0.f;
  }
  const float al = a.g ? decay_of(a.ldg ? a.g[(size_t)b * a.ldg + h] : a.g[h]) : 1.f;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int row = r0 + i * RPP;
    const float kk = sk[row], qq = sq[row];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      S[i][e] = fmaf(al, S[i][e], kk * v[e]);
      o[e] = fmaf(qq, S[i][e], o[e]);
    }
    if (in && row < a.dk) *reinterpret_cast<vf *>(st + (size_t)row * a.dv + col) = S[i];
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
#pragma unroll
    for (int m = LPR; m < 64; m *= 2) o[e] += __shfl_xor(o[e], m);
    if (lane < LPR) red[wave][cc + e] = o[e];
  }
  __syncthreads();
  if (tid < 64 && blockIdx.x * 64 + tid < a.dv)
    static_cast<T *>(a.out)[(size_t)b * a.ldo + (size_t)h * a.dv + blockIdx.x * 64 + tid] =
        from_f32<T>(a.scale * (red[0][tid] + red[1][tid] + red[2][tid] + red[3][tid]));
}

template <typename T, int V>
int run_step(const LinAttnArgs &a, hipStream_t st) {
  constexpr int RPP = 4 * V;
  const dim3 grid((a.dv + 63) / 64, a.Hv, a.Bt);
  if (a.dk <= 4 * RPP)
    hipLaunchKernelGGL((linattn_step_kernel<T, V, 4>), grid, dim3(256), 0, st, a);
  else if (a.dk <= (V == 4 ? 8 : 32) * RPP)
    hipLaunchKernelGGL((linattn_step_kernel<T, V, V == 4 ? 8 : 32>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((linattn_step_kernel<T, V, V == 4 ? 16 : 64>), grid, dim3(256), 0, st, a);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

// ------------------------------------------------------------------------------------------------------------------
// Prompts, in blocks of 64 tokens.  With G_t the sum of the block's log2 decays up to token t,
//   o_t = scale (exp2(G_t) q_t^T S + sum_{s <= t} exp2(G_t - G_s) (q_t . k_s) v_s),   S <- exp2(G_64) S + sum_s k_s (exp2(G_64 - G_s) v_s)^T
// four products per block, all on the matrix units; no exponential has a positive argument.
//
// A workgroup of four waves takes 64 NT columns of one value head's state and walks a range of blocks; a wave keeps its 16 NT
// columns of S (all rows) in fp32 registers.  Result registers of a 16 x 16 product hold 4 rows of one column, operand
// registers 8 rows of one column, and which 8 of 32 rows a group of 16 lanes contributes is free as long as both operands
// agree: taking rows 16 a + 4 g + r turns S's result registers into operands of the next product without moving them.
//
// fp32 values go through the 16-bit matrix units in pieces, each the rounding of what the ones before left over:
//   S in front of q: two pieces (16 bits), the block's weights two bf16 pieces, the weighted v of the state's update three bf16
//   pieces (24 bits) or two fp16 ones (22).  bf16 pieces have fp32's range.  fp16 operands (k, q) need fp16 partners, so a
//   column of S or of the weighted v is first brought to the top of fp16's range by a power of two, and what is below 2^-37 of its
//   largest element is lost (S in front of q has 22 bits there); v itself splits into two bf16 pieces exactly, whose lower one meets the
//   weights' upper one only (2^-18 of a product is left out).
// These are fewer bits than fp32's in front of a product only: states, sums and their joins are fp32.  16 bits are 2^8 (bf16) or 2^5 (fp16)
// times finer than the outputs they end in; the update's have to last, hence 22 and 24.  A third piece of S costs a fifth more products.
// A decay of -infinity (or below fp32's range) is a reset: it adds nothing to G, but weights across it are 0.
//
// The exponents G_t - G_s are differences of sums that grow by up to 126 a token, and what fp32 rounds off a sum of 2000 is 2^-14 of
// a weight.  So a sum is held as a multiple of 2^-10 and a factor for the rest: with 200 for a reset (exp2 of -200 is 0) the
// multiples stay below 64 * 200, 24 bits, and their differences are exact.
// ------------------------------------------------------------------------------------------------------------------
constexpr int kBlock = 64;

struct SegArgs {
  int segments, blocks;  // of a sequence; blocks of a segment
  float *slots;          // [Bt Hv][segments][dk][dv]: a segment's own sum of updates one slot on, later the state it starts from
  float2 *decays;        // [Bt Hv][segments]: a segment's whole decay, fp32 and what that rounding left over
};

struct alignas(16) GTable {  // of a block's 64 tokens; read four floats at a time
  float d[kBlock];     // G_t to the nearest multiple of 2^-10, less 200 for each reset up to the token
  float up[kBlock];    // scale exp2 of what the rounding left over,
  float down[kBlock];  // and exp2 of its opposite: scale exp2(G_t - G_s) = exp2(d_t - d_s) up_t down_s
  float e[kBlock];     // scale exp2(G_t), 0 behind a reset
  float w[kBlock];     // exp2(G_64 - G_s), 0 in front of a reset
  double sum;          // G_64
  double carry;        // what the factors applied so far are off by (their exact product over the applied one)
  float dec;           // the factor of the state
  int resets;
};
static_assert(sizeof(GTable) % 16 == 0 && offsetof(GTable, d) % 16 == 0 && offsetof(GTable, down) % 16 == 0 && offsetof(GTable, w) % 16 == 0,
              "both tables' rows start on 16 bytes");

// A constant in scalar registers, made where it is used: as vector registers those of the polynomial below are kept through the loop,
// and where there are none left for them, in scratch memory.
__device__ __forceinline__ double literal(double c) {
  asm volatile("" : "+s"(c));
  return c;
}
// 2^x for x <= 0, to 7e-12
__device__ __forceinline__ double exp2_neg(double x) {
  if (!(x > -200.0)) return x == x ? 0.0 : x;
  const double n = __builtin_rint(x), f = (x - n) * literal(0.69314718055994530942);
  double p = literal(1.0 / 362880.0);
  p = __builtin_fma(p, f, literal(1.0 / 40320.0));
  p = __builtin_fma(p, f, literal(1.0 / 5040.0));
  p = __builtin_fma(p, f, literal(1.0 / 720.0));
  p = __builtin_fma(p, f, literal(1.0 / 120.0));
  p = __builtin_fma(p, f, literal(1.0 / 24.0));
  p = __builtin_fma(p, f, literal(1.0 / 6.0));
  p = __builtin_fma(p, f, 0.5);
  p = __builtin_fma(p, f, 1.0);
  p = __builtin_fma(p, f, 1.0);
  return __builtin_ldexp(p, (int)n);
}

// x to the nearest multiple of 2^-10
__device__ __forceinline__ double coarse(double x) { return __builtin_rint(x * 1024.0) * (1.0 / 1024.0); }

// A double moved by a DPP pattern, 0 where no lane supplies it.
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double v) {
  const long long b = __double_as_longlong(v);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, true);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, true);
  return __longlong_as_double(((long long)hi << 32) | (unsigned)lo);
}
__device__ __forceinline__ double lane_f64(double v, int lane) {
  const long long b = __double_as_longlong(v);
  return __longlong_as_double(((long long)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32) |
                              (unsigned)__builtin_amdgcn_readlane((int)b, lane));
}

// One wave, lane = token: the table of a block from the tokens' log decays (0 behind the end).  The state is multiplied by one
// fp32 factor per block, and the roundings of a hundred equal factors would add up; so each is rounded from the exact one times
// what the product so far is off by, which keeps the product over any run of blocks within two roundings.
__device__ __forceinline__ void make_table(float g, float scale, double carry, int lane, GTable &t) {
  const bool reset = forgets(g);
  const double x = reset || g > 0.f ? 0.0 : (double)g * 1.44269504088896340736;
  double d = x;  // inclusive sums inside rows of 16 lanes
  d += dpp_f64<0x111>(d);  // row_shr 1
  d += dpp_f64<0x112>(d);
  d += dpp_f64<0x114>(d);
  d += dpp_f64<0x118>(d);
  const double b1 = lane_f64(d, 15), b2 = b1 + lane_f64(d, 31), b3 = b2 + lane_f64(d, 47), all = b3 + lane_f64(d, 63);
  const double G = d + (lane < 16 ? 0.0 : (lane < 32 ? b1 : (lane < 48 ? b2 : b3)));
  const unsigned long long m = __ballot(reset);
  const int n = __popcll(m & (~0ull >> (63 - lane))), last = __popcll(m);
  const double Gc = coarse(G), W = all - G, Wc = coarse(W);
  const float up = scale * __builtin_amdgcn_exp2f((float)(G - Gc));
  t.d[lane] = (float)(Gc - 200.0 * n);
  t.up[lane] = up;
  t.down[lane] = __builtin_amdgcn_exp2f((float)(Gc - G));
  t.e[lane] = n ? 0.f : __builtin_amdgcn_exp2f((float)Gc) * up;
  t.w[lane] = n != last ? 0.f : __builtin_amdgcn_exp2f((float)Wc) * __builtin_amdgcn_exp2f((float)(W - Wc));
  const double dec = last ? 0.0 : exp2_neg(all) * carry;
  const float used = (float)dec;
  if (lane == 0) {
    t.sum = all;
    t.carry = used > 1e-30f ? dec / (double)used : 1.0;
    t.dec = used;
    t.resets = last;
  }
}

// LDS rows of 32 KT elements whose 16-byte chunks are exchanged so that nothing meets on a bank that is read at once: 16 rows at
// one chunk in 8-byte pieces; 8 rows (0-7 or 8-15) at two adjacent chunks (the transposing reads); and of 16-byte reads, whose
// quarters are lanes 0-3, 12-15, 20-27 and so on, rows 0-3 and 12-15 at one chunk with rows 4-11 at the chunk next to it (with rows
// r and r + 8 exchanged alike those met two at a time).  The exchange depends on the row modulo 16 only.
template <int KT>
__device__ __forceinline__ int swap_of(int row) {
  const int high = (row >> 3) & 1;
  return KT == 2 ? ((((row >> 1) & 3) ^ (high << 1)) << 1) | high : (((row & 7) ^ (high << 2)) << 1) | high;
}
template <int KT>
__device__ __forceinline__ int tile_at(int row, int chunk) {
  return row * (64 * KT) + ((chunk ^ swap_of<KT>(row)) << 4);
}
// A wave's own 16 NT columns of v: rows of 32 NT bytes
template <int NT>
__device__ __forceinline__ int swap_v(int row) {
  return NT == 1 ? 0 : ((row >> 2) & 1) << 1;
}
// The block's weights, tokens t x tokens s, on and below the diagonal: 32 columns s for the first 32 rows, 64 for the others
constexpr int kWeightBytes = 32 * 64 + 32 * 128;
__device__ __forceinline__ int weight_at(int t, int chunk) {
  return t < 32 ? t * 64 + ((chunk ^ ((t >> 2) & 3)) << 4) : 2048 + (t - 32) * 128 + ((chunk ^ swap_of<2>(t)) << 4);
}

typedef short v4s __attribute__((ext_vector_type(4)));
// Four elements of column `lane % 16` of a block of 16 columns, rows first + 4 (lane / 16) .. + 3: each lane points at 4 elements
// of one row, and the read exchanges them inside groups of 16 lanes.
template <typename T>
__device__ __forceinline__ typename Half<T>::v4 read_exchanged(const char *p) {
  const v4s r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4s __attribute__((address_space(3))) *)(p));
  return __builtin_bit_cast(typename Half<T>::v4, r);
}
template <typename V4>
__device__ __forceinline__ auto both(V4 lo, V4 hi) {
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
// Operand of 32 rows (tokens) of a column block, rows 32 kb + 16 a + 4 g + r in slot 4 a + r of lane group g.  Of a k tile:
// column_at is the lane's offset of block 0; a block is an exclusive-or away (the exchange moves chunks by exclusive-or too),
// 16 rows a constant.
template <int KT>
__device__ __forceinline__ int column_at(int lane) {
  const int i = lane & 15, row = 4 * (lane >> 4) + (i >> 2);
  return tile_at<KT>(row, (i & 3) >> 1) + (i & 1) * 8;
}
template <typename T, int KT>
__device__ __forceinline__ typename Half<T>::v8 column_operand(const char *tiles, int at, int kb, int block) {
  const char *p = tiles + (at ^ (block << 5)) + 32 * kb * 64 * KT;
  return both(read_exchanged<T>(p), read_exchanged<T>(p + 16 * 64 * KT));
}
template <typename T, int NT>
__device__ __forceinline__ typename Half<T>::v8 value_operand(const char *own, int kb, int n, int lane) {
  const int i = lane & 15, row = 32 * kb + 4 * (lane >> 4) + (i >> 2), chunk = 2 * n + ((i & 3) >> 1);
  const char *p = own + row * (32 * NT) + ((chunk ^ swap_v<NT>(row)) << 4) + (i & 1) * 8;
  return both(read_exchanged<T>(p), read_exchanged<T>(p + 16 * 32 * NT));  // 16 rows on: the same exchange
}
// Operand of one row, elements 32 j + 16 a + 4 g + r in slot 4 a + r.  row_at: the lane's offset in row lane % 16 for j = 0
template <int KT>
__device__ __forceinline__ int row_at(int lane) {
  const int g = lane >> 4;
  return tile_at<KT>(lane & 15, g >> 1) + (g & 1) * 8;
}
template <typename T, int KT>
__device__ __forceinline__ typename Half<T>::v8 row_operand(const char *tile, int at, int tb, int j) {
  typedef typename Half<T>::v4 v4;
  const char *p = tile + 16 * tb * 64 * KT;
  return both(*reinterpret_cast<const v4 *>(p + (at ^ (j << 6))), *reinterpret_cast<const v4 *>(p + (at ^ (j << 6) ^ 32)));
}
__device__ __forceinline__ Half<__bf16>::v8 weight_operand(const char *p, int t, int kb, int lane) {
  const int g = lane >> 4, chunk = 4 * kb + (g >> 1), off = (g & 1) * 8;
  typedef Half<__bf16>::v4 v4;
  return both(*reinterpret_cast<const v4 *>(p + weight_at(t, chunk) + off), *reinterpret_cast<const v4 *>(p + weight_at(t, chunk + 2) + off));
}

// The power of two (its exponent) that brings m to 2^12 .. 2^13, the top of fp16's range, whatever fp32 number m is (at least -116); at
// most 2^100, so that its inverse times a decay stays an ordinary number.
__device__ __forceinline__ int top_exponent(float m) {
  const int e = 127 + 12 - (int)((__float_as_uint(m) >> 23) & 0xff);
  return min(e, 100);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned)(127 + e) << 23); }
// Largest over the four lane groups (the same column)
__device__ __forceinline__ float max_over_groups(float m) {
  m = fmaxf(m, __shfl_xor(m, 16));
  return fmaxf(m, __shfl_xor(m, 32));
}

// acc + 0 w.x + 0 w.y of two 16-bit values: NaN once one of them is infinite or NaN
__device__ __forceinline__ float times_zero(unsigned w, float acc, __bf16) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, w), __builtin_bit_cast(b2, 0u), acc, false);
}
__device__ __forceinline__ float times_zero(unsigned w, float acc, _Float16) {
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, w), __builtin_bit_cast(h2, 0u), acc, false);
}
__device__ __forceinline__ int seq_len(const LinAttnArgs &a, int b) { return a.lens ? min(max(a.lens[b], 0), a.L) : a.L; }

// Two fp32 values as one word of 16-bit ones, rounded to nearest
template <typename T>
__device__ __forceinline__ unsigned pack2(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef T t2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((f2{a, b}), t2));
}
// The same, and what it leaves over.  fp16 takes its first piece by truncation, which packs
// in one instruction; the last piece of a value is always rounded to nearest (pack2).
__device__ __forceinline__ unsigned take2(float &a, float &b, __bf16) {
  const unsigned w = pack2<__bf16>(a, b);
  a -= __uint_as_float(w << 16);
  b -= __uint_as_float(w & 0xffff0000u);
  return w;
}
__device__ __forceinline__ unsigned take2(float &a, float &b, _Float16) {
  const auto h = __builtin_amdgcn_cvt_pkrtz(a, b);
  a -= static_cast<float>(h[0]);
  b -= static_cast<float>(h[1]);
  return __builtin_bit_cast(unsigned, h);
}
typedef unsigned u4 __attribute__((ext_vector_type(4)));

// 16 bytes a lane from base + off (lane) + soff (wave) to consecutive LDS from `to` on, zeros where off is negative.  Written
// out, because the compiler takes every LDS read for one of what such a load is still bringing and waits for the load first (three
// times a block; 2 x 4000, 32 heads of 64 x 64: 72 -> 67 us).  What it would know is kept by hand: nothing reads a tile before
// the barrier that waits for its loads, and the scalar operands may come straight from a vector instruction, hence the five wait states.
// m0 is declared; the warning that goes with it says that the compiler reserves m0 and would not save it, and it keeps nothing there.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void tile_load(const void *base, int off, int soff, const char *to) {
  const unsigned long long b = reinterpret_cast<unsigned long long>(base);
  const u4 rsrc = {(unsigned)b, (unsigned)(b >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
  const unsigned lds = (unsigned)reinterpret_cast<unsigned long long>((const __attribute__((address_space(3))) char *)to);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(off), "s"(rsrc), "s"(soff)
               : "m0");
}
#pragma clang diagnostic pop

// Eight elements of a row of K from element k on, zeros behind K and where the row is off, in two steps: what is in flight is 16
// bytes that end with the row at the latest, and they are moved into place when they are used.  With the last elements loaded one
// by one every load waited for its own (10 x 570, 29 heads of 85 x 176: 443 -> 338 us).
template <typename T>
__device__ __forceinline__ typename Half<T>::v8 ask8(const T *row, int k, int K) {
  typename Half<T>::v8 v = {};
  if (K >= 8) {
    __builtin_memcpy(&v, row + min(k, K - 8), 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k == 0 && e < K ? row[min(e, K - 1)] : static_cast<T>(0.f);
  }
  return v;
}
template <typename V8>
__device__ __forceinline__ V8 place8(V8 v, int k, int K, bool on) {
  typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
  u64x2 w = __builtin_bit_cast(u64x2, v);
  if (K & 7) {  // the last elements of a row stand at the end of what was loaded
    const int bits = K < 8 ? 0 : 16 * max(k - (K - 8), 0), part = bits & 63;
    const unsigned long long lo = bits & 64 ? w[1] : w[0], hi = bits & 64 ? 0 : w[1];
    w[0] = (lo >> part) | (part ? hi << (64 - part) : 0);
    w[1] = hi >> part;
  }
  if (!on || k >= K) w = u64x2{0, 0};
  return __builtin_bit_cast(V8, w);
}

// Order LDS accesses (the compiler's and the wave's own) around the hardware barrier.  VM: so many of the wave's vector memory
// operations, the youngest, may still be under way (they complete in the order of issue); 63: all.
template <int VM>
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | 0x0070);  // vmcnt in bits 3:0 and 15:14, lgkmcnt (11:8) 0
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// KT: dk <= 32 KT.  OUT: outputs and the state; otherwise only a segment's own sum of updates and its decay.  WIDE: rows and
// heads start on 16 bytes and a block's rows span less than 2^31 bytes: tiles travel by direct-to-LDS buffer loads, whose lanes
// behind the end or behind dk or dv get an offset past the buffer and leave zeros.  Otherwise they pass through registers.
//
// LDS for two workgroups on a CU (KT = 4, NT = 2: 78.2 of 80 KB): k twice, the next block's arriving while this one's is used; q
// and v once: q is done with at the barrier behind the weights, v belongs to one wave and is done with once it is in registers.
template <typename T, int KT, int NT, bool OUT, bool WIDE>
__global__ __launch_bounds__(256, KT == 8 && OUT ? 1 : 2) void linattn_blocks_kernel(LinAttnArgs a, SegArgs sg) {
  constexpr bool F16 = std::is_same<T, _Float16>::value;
  constexpr int TB = 64 * KT * kBlock, VB = 32 * NT * kBlock, QB = OUT ? TB : 0;  // bytes of a k or q tile, of a wave's v
  typedef typename Half<T>::v8 v8;
  typedef Half<__bf16>::v8 b8;
  typedef Half<__bf16>::v4 b4;
  __shared__ __attribute__((aligned(16))) char lds[QB + 2 * TB + 4 * VB + (OUT ? 2 * kWeightBytes : 0)];
  __shared__ GTable tables[2];
  char *lq = lds, *lks = lds + QB, *lvs = lks + 2 * TB, *lp = lvs + 4 * VB, *lpl = lp + kWeightBytes;

  // XCDs get contiguous runs of workgroups (ids are dealt round-robin to the 8 of them): column parts of a head, heads of a
  // segment next to one another, so what shares q and k shares an L2
  const int nwg = gridDim.x, per = nwg >> 3;
  const int id = (int)blockIdx.x < (per << 3) ? ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3) : (int)blockIdx.x;
  const int parts = (a.dv + 64 * NT - 1) / (64 * NT);
  const int part = id % parts, rest = id / parts;
  const int pairs = a.Bt * a.Hv, pair = rest % pairs, seg = rest / pairs;
  const int h = pair % a.Hv, b = pair / a.Hv, hk = h / (a.Hv / a.Hk);
  const int len = seq_len(a, b);
  const int t_lo = seg * sg.blocks * kBlock, t_hi = min(len, t_lo + sg.blocks * kBlock);
  if (t_lo >= len || (!OUT && t_hi == len)) return;  // nothing here; the last segment's sum is nobody's start

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col0 = part * 64 * NT + wave * 16 * NT;  // this wave's first column
  char *lv = lvs + wave * VB;

  const size_t row0 = (size_t)b * a.L;
  const T *pq = static_cast<const T *>(a.q) + row0 * a.ldq + (size_t)hk * a.dk;
  const T *pk = static_cast<const T *>(a.k) + row0 * a.ldk + (size_t)hk * a.dk;
  const T *pv = static_cast<const T *>(a.v) + row0 * a.ldv + (size_t)h * a.dv;
  T *po = static_cast<T *>(a.out) + row0 * a.ldo + (size_t)h * a.dv;

  // A wave-level load fills 1 KB of LDS, 16 bytes a lane: a k or q tile in NL loads of each wave, whose rows differ by PH loads in
  // multiples of 16, so that PH lane offsets serve all of them; a wave's v in NLV loads.
  constexpr int RPL = 16 / KT, NL = KT, PH = 4 * RPL >= 16 ? 1 : 16 / (4 * RPL), RPLV = 32 / NT, NLV = 2 * NT;
  auto tile_row = [&](int i) { return (i / PH) * (PH * 4 * RPL) + (i % PH) * 4 * RPL + wave * RPL + lane / (64 / RPL); };
  auto tile_chunk = [&](int i) { return (lane % (64 / RPL)) ^ swap_of<KT>(tile_row(i)); };
  const int v_row = lane / (2 * NT), v_chunk = (lane % (2 * NT)) ^ swap_v<NT>(v_row);  // of load 0; RPLV rows further with each
  constexpr int OFF = (int)0x80000000;  // past every buffer
  int oq[PH], ok[PH], ov, oo[NT];
  if constexpr (WIDE) {
#pragma unroll
    for (int i = 0; i < PH; ++i) {
      const bool in = tile_chunk(i) * 8 < a.dk;
      oq[i] = in ? (int)(tile_row(i) * a.ldq + tile_chunk(i) * 8) * 2 : OFF;
      ok[i] = in ? (int)(tile_row(i) * a.ldk + tile_chunk(i) * 8) * 2 : OFF;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) oo[n] = col0 + 16 * n + 4 * g < a.dv ? (int)(c * a.ldo + col0 + 16 * n + 4 * g) * 2 : OFF;
    ov = col0 + v_chunk * 8 < a.dv ? (int)(v_row * a.ldv + col0 + v_chunk * 8) * 2 : OFF;
  }
  v8 rq[!WIDE && OUT ? NL : 1], rk[!WIDE ? NL : 1], rv[!WIDE ? NLV : 1];
  auto load_tile = [&](const T *p, long long ld, const int (&o)[PH], v8 *r, int t0, char *tile, int i) {  // load i of the wave's NL
    const int n = t_hi - t0;  // rows that count
    if constexpr (WIDE) {
      const int off = n >= kBlock || tile_row(i) < n ? o[i % PH] : OFF;
      tile_load(p + (size_t)t0 * ld, off, (int)((i / PH) * (PH * 4 * RPL) * ld * 2), tile + ((i / PH) * PH * 4 + (i % PH) * 4 + wave) * 1024);
    } else {
      r[i] = ask8(p + (size_t)(t0 + min(tile_row(i), n - 1)) * ld, tile_chunk(i) * 8, a.dk);
    }
  };
  auto load_v = [&](int t0, int i) {  // of NLV
    const int n = t_hi - t0, row = v_row + RPLV * i;
    if constexpr (WIDE)
      tile_load(pv + (size_t)t0 * a.ldv, n >= kBlock || row < n ? ov : OFF, (int)(RPLV * i * a.ldv * 2), lv + i * 1024);
    else
      rv[i] = ask8(pv + (size_t)(t0 + min(row, n - 1)) * a.ldv, col0 + v_chunk * 8, a.dv);
  };
  auto fetch_tile = [&](const T *p, long long ld, const int (&o)[PH], v8 *r, int t0, char *tile) {
#pragma unroll
    for (int i = 0; i < NL; ++i) load_tile(p, ld, o, r, t0, tile, i);
  };
  auto fetch_v = [&](int t0) {
#pragma unroll
    for (int i = 0; i < NLV; ++i) load_v(t0, i);
  };
  auto park = [&](char *lk, int t0) {  // what came through registers
    if constexpr (!WIDE) {
      const int n = t_hi - t0;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int at = ((i / PH) * PH * 4 + (i % PH) * 4 + wave) * 1024 + lane * 16;
        const bool on = tile_row(i) < n;
        if constexpr (OUT) *reinterpret_cast<v8 *>(lq + at) = place8(rq[i], tile_chunk(i) * 8, a.dk, on);
        *reinterpret_cast<v8 *>(lk + at) = place8(rk[i], tile_chunk(i) * 8, a.dk, on);
      }
#pragma unroll
      for (int i = 0; i < NLV; ++i)
        *reinterpret_cast<v8 *>(lv + i * 1024 + lane * 16) = place8(rv[i], col0 + v_chunk * 8, a.dv, v_row + RPLV * i < n);
    }
  };
  auto log_decay = [&](int t0) {
    const int t = t0 + lane;
    return a.g && t < t_hi ? (a.ldg ? a.g[(row0 + t) * a.ldg + h] : a.g[h]) : 0.f;
  };

  fetch_tile(pk, a.ldk, ok, rk, t_lo, lks);
  if constexpr (OUT) fetch_tile(pq, a.ldq, oq, rq, t_lo, lq);
  fetch_v(t_lo);
  float gt = log_decay(t_lo);

  // S[m][n]: rows 16 m + 4 g + r of column col0 + 16 n + c
  v4f S[2 * KT][NT];
  const float *from = !OUT ? nullptr : (sg.segments > 1 ? sg.slots + ((size_t)pair * sg.segments + seg) * a.dk * a.dv
                                                        : (a.state ? a.state + (size_t)pair * a.dk * a.dv : nullptr));
#pragma unroll
  for (int m = 0; m < 2 * KT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * m + 4 * g + r, col = col0 + 16 * n + c;
        S[m][n][r] = from && row < a.dk && col < a.dv ? from[(size_t)row * a.dv + col] : 0.f;
      }

  if constexpr (OUT) {
    // the weights above the diagonal that a product of 32 tokens takes in: zero, and never written again
    if (tid < 128) {  // piece, which of two, row, chunk
      const int pr = (tid >> 1) & 1, row = 32 * pr + ((tid >> 2) & 15), chunk = 4 * pr + 2 + (tid >> 6);
      *reinterpret_cast<b8 *>((tid & 1 ? lpl : lp) + weight_at(row, chunk)) = b8{};
    }
  }
  double G = 0.0;  // of the segment
  int resets = 0;
  if (wave == 0) make_table(gt, a.scale, 1.0, lane, tables[0]);
  park(lks, t_lo);
  block_barrier<0>();

  int buf = 0;
  for (int t0 = t_lo; t0 < t_hi; t0 += kBlock, buf ^= 1) {
    const GTable &tab = tables[buf];
    // the lane's offsets in the tiles, opaque so that the exclusive-ors of the operand reads stay where they are used: hoisted out of
    // the loop they take 30 registers
    int at_row = row_at<KT>(lane), at_column = column_at<KT>(lane) + buf * TB, at_chunk = tile_at<KT>(c, g);
    asm volatile("" : "+v"(at_row), "+v"(at_column), "+v"(at_chunk));
    char *lk_next = lks + (buf ^ 1) * TB;
    const int t1 = t0 + kBlock;
    const bool more = t1 < t_hi;
    // A wave waits about 200 cycles to issue a load while all eight waves of the CU issue theirs: the next block's travel one at a
    // time between products, k's under the state's contribution, q's under the weights', v's under the update.  The wave that
    // makes the next table (they take turns) reads the decays.
    constexpr bool SPREAD = WIDE && OUT;
    const int maker = OUT ? 2 + ((t0 / kBlock) & 1) : (t0 / kBlock) & 3;
    if (more) {
      if (wave == maker) gt = log_decay(t1);
      if constexpr (!SPREAD) fetch_tile(pk, a.ldk, ok, rk, t1, lk_next);
      if constexpr (!WIDE) {
        if constexpr (OUT) fetch_tile(pq, a.ldq, oq, rq, t1, lq);
        fetch_v(t1);
      }
    }

    v4f O[4][NT];  // transposed: columns (of v) 4 g + r, token 16 tb + c
    if constexpr (OUT) {
      // weights: the 10 blocks of 16 x 16 on and below the diagonal: two with the same tokens t for each wave (sb, sb + 1 of tb: 3 3,
      // 2 and 1 for the waves), then (0, 0) and (2, 2) for waves 0 and 1, while waves 2 and 3 make the next block's table in turn
      auto weights = [&](int tb, int sb, auto blocks) {
        constexpr int B = decltype(blocks)::value;
        v4f p[B];
#pragma unroll
        for (int x = 0; x < B; ++x) p[x] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KT; ++j) {
          const int at = at_chunk ^ (j << 6);
          const v8 fq = *reinterpret_cast<const v8 *>(lq + 16 * tb * 64 * KT + at);
#pragma unroll
          for (int x = 0; x < B; ++x)
            p[x] = Half<T>::mfma16(*reinterpret_cast<const v8 *>(lks + buf * TB + 16 * (sb + x) * 64 * KT + at), fq, p[x]);  // rows s, columns t
        }
        const int t = 16 * tb + c;
        const float d_t = tab.d[t], up = tab.up[t];
#pragma unroll
        for (int x = 0; x < B; ++x) {
          const int s = 16 * (sb + x) + 4 * g;
          const v4f ds = *reinterpret_cast<const v4f *>(&tab.d[s]), down = *reinterpret_cast<const v4f *>(&tab.down[s]);
          float v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = s + r <= t ? up * p[x][r] * (down[r] * __builtin_amdgcn_exp2f(d_t - ds[r])) : 0.f;
          const int at = weight_at(t, 2 * (sb + x) + (g >> 1)) + (g & 1) * 8;
          uint2 w;
          w.x = take2(v[0], v[1], __bf16());
          w.y = take2(v[2], v[3], __bf16());
          *reinterpret_cast<uint2 *>(lp + at) = w;
          w.x = pack2<__bf16>(v[0], v[1]);
          w.y = pack2<__bf16>(v[2], v[3]);
          *reinterpret_cast<uint2 *>(lpl + at) = w;
        }
      };
      weights(wave < 2 ? 3 : 4 - wave, wave == 1 ? 2 : 0, std::integral_constant<int, 2>());
      if (wave < 2)
        weights(2 * wave, 2 * wave, std::integral_constant<int, 1>());
      else if (more && wave == maker)
        make_table(gt, a.scale, tab.carry, lane, tables[buf ^ 1]);
      // what the state contributes
#pragma unroll
      for (int tb = 0; tb < 4; ++tb)
#pragma unroll
        for (int n = 0; n < NT; ++n) O[tb][n] = v4f{0.f, 0.f, 0.f, 0.f};
      int se[NT];
      float sf[NT];
      if constexpr (F16) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float m = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * KT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) m = fmaxf(m, fabsf(S[i][n][r]));
          se[n] = top_exponent(max_over_groups(m));
          sf[n] = pow2(se[n]);
        }
      }
      // operands of step j + 1 are asked for, and its pieces of S made, under the products of step j: left to itself the compiler
      // reads each operand right before its product and waits for it
      v8 fq[2][4];
      u4 sh[2][NT], sl[2][NT];
      auto ask_q = [&](int j, v8 (&f)[4]) {
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) f[tb] = row_operand<T, KT>(lq, at_row, tb, j);
      };
      auto split = [&](int j, u4 (&hi)[NT], u4 (&lo)[NT]) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            float x = S[2 * j + (e >> 2)][n][e & 3], y = S[2 * j + (e >> 2)][n][(e & 3) + 1];
            if constexpr (F16) x *= sf[n], y *= sf[n];
            hi[n][e / 2] = take2(x, y, T());
            lo[n][e / 2] = pack2<T>(x, y);
          }
      };
      ask_q(0, fq[0]);
      split(0, sh[0], sl[0]);
#pragma unroll
      for (int j = 0; j < KT; ++j) {
        if (j + 1 < KT) ask_q(j + 1, fq[(j + 1) & 1]);
        if (SPREAD && more) load_tile(pk, a.ldk, ok, rk, t1, lk_next, j);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
          for (int n = 0; n < NT; ++n) O[tb][n] = Half<T>::mfma16(__builtin_bit_cast(v8, sh[j & 1][n]), fq[j & 1][tb], O[tb][n]);
        if (j + 1 < KT) split(j + 1, sh[(j + 1) & 1], sl[(j + 1) & 1]);
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
          for (int n = 0; n < NT; ++n) O[tb][n] = Half<T>::mfma16(__builtin_bit_cast(v8, sl[j & 1][n]), fq[j & 1][tb], O[tb][n]);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float back[4] = {1.f, 1.f, 1.f, 1.f};
        if constexpr (F16) {
#pragma unroll
          for (int r = 0; r < 4; ++r) back[r] = pow2(-__shfl(se[n], 4 * g + r));  // column 4 g + r is lane 4 g + r's
        }
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
          const float e = tab.e[16 * tb + c];
#pragma unroll
          for (int r = 0; r < 4; ++r) O[tb][n][r] *= F16 ? e * back[r] : e;
        }
      }
    }
    if constexpr (!OUT) {
      if (more && wave == maker) make_table(gt, a.scale, tab.carry, lane, tables[buf ^ 1]);
      G += tab.sum;
      resets += tab.resets;
    }
    if constexpr (OUT) {
      // The weights are in LDS, q is done with, and this wave's v is there: loads complete in order, so where a v load is under way
      // the KT k loads behind it are too (in the last block there are none).
      if (!SPREAD)
        block_barrier<63>();
      else if (more)
        block_barrier<KT>();
      else
        block_barrier<0>();
    }

    v8 fv[2][NT];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        fv[kb][n] = value_operand<T, NT>(lv, kb, n, lane);
      }
    if (WIDE && more) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int n = 0; n < NT; ++n) asm volatile("" : "+v"(fv[kb][n])::"memory");  // read before the next block's may arrive
      if constexpr (!SPREAD) fetch_v(t1);
    }
    bool any = false;
    if constexpr (OUT) {
      b8 ph[2][2], pl[2][2];
      auto ask_p = [&](int tb) {
#pragma unroll
        for (int kb = 0; kb <= tb / 2; ++kb) {
          ph[tb & 1][kb] = weight_operand(lp, 16 * tb + c, kb, lane);
          pl[tb & 1][kb] = weight_operand(lpl, 16 * tb + c, kb, lane);
        }
      };
      ask_p(0);
      // A token's NaN or infinity in v must not reach earlier outputs, and in a product it would: its weight there is 0.  Where a
      // wave finds one (rare; looking for it costs 1 %) it leaves them out of the product, and the outputs of their column are NaN from
      // the first's token on.
      float bad[2] = {0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) bad[e & 1] = times_zero(__builtin_bit_cast(u4, fv[kb][n])[e], bad[e & 1], T());
      any = __ballot(!(bad[0] + bad[1] == 0.f)) != 0;
      if (__builtin_expect(any, 0)) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          int first = kBlock;
#pragma unroll
          for (int kb = 1; kb >= 0; --kb)
#pragma unroll
            for (int e = 7; e >= 0; --e)
              if (!(fabsf(to_f32(fv[kb][n][e])) <= FLT_MAX)) {
                first = 32 * kb + 16 * (e >> 2) + 4 * g + (e & 3);
                fv[kb][n][e] = T(0.f);
              }
          first = min(first, __shfl_xor(first, 16));
          first = min(first, __shfl_xor(first, 32));
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int of = __shfl(first, 4 * g + r);
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
              if (16 * tb + c >= of) O[tb][n][r] = __builtin_nanf("");
          }
        }
      }
      b8 vh[2][NT], vl[F16 ? 2 : 1][F16 ? NT : 1];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if constexpr (F16) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              vh[kb][n][e] = from_f32<__bf16>(to_f32(fv[kb][n][e]));
              vl[kb][n][e] = from_f32<__bf16>(to_f32(fv[kb][n][e]) - to_f32(vh[kb][n][e]));
            }
          } else {
            vh[kb][n] = fv[kb][n];
          }
        }
#pragma unroll
      for (int tb = 0; tb < 4; ++tb) {
        if (tb < 3) ask_p(tb + 1);
        if (SPREAD && more) {
#pragma unroll
          for (int i = tb * KT / 4; i < (tb + 1) * KT / 4; ++i) load_tile(pq, a.ldq, oq, rq, t1, lq, i);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb <= tb / 2; ++kb)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            O[tb][n] = Half<__bf16>::mfma16(vh[kb][n], ph[tb & 1][kb], O[tb][n]);
            O[tb][n] = Half<__bf16>::mfma16(vh[kb][n], pl[tb & 1][kb], O[tb][n]);
            if constexpr (F16) O[tb][n] = Half<__bf16>::mfma16(vl[kb][n], ph[tb & 1][kb], O[tb][n]);
          }
        const int t = t0 + 16 * tb + c;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const v4f o = O[tb][n];
          if constexpr (WIDE) {
            typedef unsigned u2 __attribute__((ext_vector_type(2)));
            const u2 w = {pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
            __builtin_amdgcn_raw_buffer_store_b64(w, buffer_over(po + (size_t)t0 * a.ldo, 0x7fffffff), t < t_hi ? oo[n] : OFF,
                                                  (int)(16 * tb * a.ldo * 2), 0);
          } else if (t < t_hi) {
            const int col = col0 + 16 * n + 4 * g;
            T *to = po + (size_t)t * a.ldo + col;
            if (col + 4 <= a.dv) {
              const unsigned w[2] = {pack2<T>(o[0], o[1]), pack2<T>(o[2], o[3])};
              __builtin_memcpy(to, w, 8);
            } else {
#pragma unroll
              for (int r = 0; r < 3; ++r)
                if (col + r < a.dv) to[r] = from_f32<T>(o[r]);
            }
          }
        }
      }
    }

    // the state's update: decay, then k (weighted v)^T, with v as it is
    if constexpr (OUT)
      if (__builtin_expect(any, 0)) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            fv[kb][n] = value_operand<T, NT>(lv, kb, n, lane);
            asm volatile("" : "+v"(fv[kb][n])::"memory");  // before the next block's may arrive
          }
      }
    constexpr int VP = F16 ? 2 : 3;
    u4 wv[VP][2][NT];
    float back[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float x[2][8], m = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const v4f w = *reinterpret_cast<const v4f *>(&tab.w[32 * kb + 16 * hf + 4 * g]);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            x[kb][4 * hf + r] = w[r] * to_f32(fv[kb][n][4 * hf + r]);
            if constexpr (F16) m = fmaxf(m, fabsf(x[kb][4 * hf + r]));
          }
        }
      float up = 1.f;
      if constexpr (F16) {
        const int e = top_exponent(max_over_groups(m));
        up = pow2(e);
        back[n] = pow2(-e);
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          float v0 = x[kb][e], v1 = x[kb][e + 1];
          if constexpr (F16) v0 *= up, v1 *= up;
#pragma unroll
          for (int p = 0; p + 1 < VP; ++p) wv[p][kb][n][e / 2] = take2(v0, v1, T());
          wv[VP - 1][kb][n][e / 2] = pack2<T>(v0, v1);
        }
    }
    const float dec = tab.dec;
    v8 fk[2][2];
    auto ask_k = [&](int i) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) fk[i & 1][kb] = column_operand<T, KT>(lks, at_column, kb, i);
    };
    ask_k(0);
#pragma unroll
    for (int i = 0; i < 2 * KT; ++i) {
      if (i + 1 < 2 * KT) ask_k(i + 1);
      if (SPREAD && more && i < NLV) load_v(t1, i);
      __builtin_amdgcn_sched_barrier(0);
      v4f u[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) u[n][r] = F16 ? 0.f : S[i][n][r] * dec;
#pragma unroll
      for (int p = VP - 1; p >= 0; --p)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int n = 0; n < NT; ++n) u[n] = Half<T>::mfma16(fk[i & 1][kb], __builtin_bit_cast(v8, wv[p][kb][n]), u[n]);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[i][n][r] = F16 ? fmaf(u[n][r], back[n], S[i][n][r] * dec) : u[n][r];
    }
    if (more) park(lk_next, t1);
    // The next block's k and q are in LDS (where one of their loads is under way the NLV v loads behind it are too), this one's are
    // done with.
    block_barrier<SPREAD ? NLV : 0>();
  }

  if constexpr (!OUT) {
    if (part == 0 && tid == 0) {
      const double dec = resets ? 0.0 : exp2_neg(G);
      sg.decays[(size_t)pair * sg.segments + seg] = make_float2((float)dec, (float)(dec - (double)(float)dec));
    }
  }
  float *to = !OUT ? sg.slots + ((size_t)pair * sg.segments + seg + 1) * a.dk * a.dv
                   : (a.state && t_hi == len ? a.state + (size_t)pair * a.dk * a.dv : nullptr);
  if (to)
#pragma unroll
    for (int m = 0; m < 2 * KT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * m + 4 * g + r, col = col0 + 16 * n + c;
          if (row < a.dk && col < a.dv) to[(size_t)row * a.dv + col] = S[m][n][r];
        }
}

// The segments' sums of updates joined: slot j becomes the state segment j starts from.  A thread takes V elements through all
// segments, eight of them asked for at a time: the sums wait for one another, the reads need not.
template <int V>
__global__ __launch_bounds__(256) void linattn_join_kernel(LinAttnArgs a, SegArgs sg) {
  typedef float vf __attribute__((ext_vector_type(V)));
  constexpr int U = 8;
  const size_t n = (size_t)a.dk * a.dv, i = ((size_t)blockIdx.x * 256 + threadIdx.x) * V;
  const int pair = blockIdx.y, b = pair / a.Hv;
  if (i >= n) return;  // V = 4: n is a multiple of 4
  const int span = sg.blocks * kBlock, used = (seq_len(a, b) + span - 1) / span;
  if (used == 0) return;
  float *p = sg.slots + (size_t)pair * sg.segments * n + i;
  const float2 *d = sg.decays + (size_t)pair * sg.segments;
  vf s = vf(0.f);
  if (a.state) s = *reinterpret_cast<const vf *>(a.state + (size_t)pair * n + i);
  *reinterpret_cast<vf *>(p) = s;
  for (int j0 = 1; j0 < used; j0 += U) {
    vf u[U];
    float2 f[U];
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (j0 + j < used) {
        u[j] = *reinterpret_cast<const vf *>(p + (size_t)(j0 + j) * n);
        f[j] = d[j0 + j - 1];
      }
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (j0 + j < used) {
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] = fmaf(s[e], f[j].x, fmaf(s[e], f[j].y, u[j][e]));
        *reinterpret_cast<vf *>(p + (size_t)(j0 + j) * n) = s;
      }
  }
}

std::atomic<int> g_segment_blocks{0};  // tuning hook

struct AttnPlan {
  int kt, nt, segments, blocks;
};

size_t slots_bytes(const AttnPlan &p, int Bt, int Hv, int dk, int dv) {
  return align_up((size_t)Bt * Hv * p.segments * dk * dv * sizeof(float), 256);
}
size_t prefill_workspace(const AttnPlan &p, int Bt, int Hv, int dk, int dv) {
  return p.segments > 1 ? slots_bytes(p, Bt, Hv, dk, dv) + align_up((size_t)Bt * Hv * p.segments * sizeof(float2), 256) : 256;
}

// How many segments a sequence is cut into: the cheapest by a cost in us fitted to measured times.  One segment is one launch of
// about 5 and 0.72 c a block; more are three launches, 9, whose two passes together take c a block and 3 to start, 1.42 times that
// with two workgroups on a CU, plus the sums' way through memory and the chain that joins them.  At 32 shapes (1 to 80 heads, 128
// to 65536 tokens, dk 32 to 256) the choice is within 10 % of the best of up to 16 that were timed: 1 x 2048, 80 heads of 128 x 64,
// 6 blocks a segment 58 us, 4 66, 8 67, all in one 115; 8 x 256, 16 heads of 64 x 64, all in one 15.5, 2 blocks 21.5, single ones
// 23.7; 1 x 16384, one head of 64 x 64, 3 blocks 33, single ones 44, all in one 617.
// The constants are those of rows on 16 bytes: the workspace query, which has to plan alike, does not know the strides.  Rows off 16
// bytes run one column tile a wave also where dv > 64 (run_prefill), up to twice the workgroups that are counted here.
// What `room` does not hold is left out; one segment needs none, so a workspace that another shape asked for serves too.
AttnPlan plan_prefill(int Bt, int L, int Hv, int dk, int dv, size_t room = SIZE_MAX) {
  AttnPlan p{2, 1, 1, 1};
  if (Bt == 0 || L == 0) return p;
  p.kt = dk <= 64 ? 2 : (dk <= 128 ? 4 : 8);
  p.nt = dv > 64 && p.kt < 8 ? 2 : 1;
  const double pairs = (double)Bt * Hv, parts = (dv + 64 * p.nt - 1) / (64 * p.nt);
  const long long blocks = (L + kBlock - 1LL) / kBlock;
  const double c = p.kt == 8 ? 7.6 : (p.kt == 4 ? (p.nt == 2 ? 6.7 : 4.9) : (p.nt == 2 ? 4.6 : 3.4));
  const double on_cu = p.kt == 8 ? 1 : 2, slow = p.kt == 8 ? 1.0 : 1.42;
  auto rounds = [&](double wgs) {
    const double full = __builtin_floor(wgs / (256 * on_cu)), rest = wgs - full * 256 * on_cu;
    return full * slow + (rest == 0 ? 0.0 : (rest <= 256 ? 1.0 : slow));
  };
  double best = 5 + rounds(pairs * parts) * 0.72 * c * blocks;
  long long at = blocks;
  if (pairs <= 65535)
    for (long long b = 1; b < blocks; b = b < 4 ? b + 1 : b + b / 4) {
      const double n = (double)((blocks + b - 1) / b);
      p.segments = (int)n;
      if (prefill_workspace(p, Bt, Hv, dk, dv) > room || !launchable((long long)(pairs * parts * n), 256)) continue;
      const double t = 9 + rounds(pairs * parts * n) * (c * b + 3) + pairs * n * dk * dv * 8.0 / 4e6 + 0.12 * n;
      if (t < best) best = t, at = b;
    }
  const int forced = g_segment_blocks.load(std::memory_order_relaxed);
  if (forced > 0 && pairs <= 65535) at = forced < blocks ? forced : blocks;
  p.blocks = (int)at;
  p.segments = (int)((blocks + at - 1) / at);
  return p;
}

template <typename T, int KT, int NT, bool WIDE>
int run_blocks(const LinAttnArgs &a, const AttnPlan &p, void *ws, hipStream_t st) {
  const int parts = (a.dv + 64 * NT - 1) / (64 * NT);
  const long long one = (long long)parts * a.Bt * a.Hv;
  if (!launchable(one * p.segments, 256))
    return fail(QUAMBA_EUNSUPPORTED, "linattn_prefill: %d sequences of %d heads are more than one launch takes", a.Bt, a.Hv);
  SegArgs sg{p.segments, p.blocks, static_cast<float *>(ws), nullptr};
  if (p.segments > 1) {
    sg.decays = reinterpret_cast<float2 *>(static_cast<char *>(ws) + slots_bytes(p, a.Bt, a.Hv, a.dk, a.dv));
    hipLaunchKernelGGL((linattn_blocks_kernel<T, KT, NT, false, WIDE>), dim3((unsigned)(one * (p.segments - 1))), dim3(256), 0, st, a, sg);
    QUAMBA_LAUNCH_CHECK();
    if (a.dk * a.dv % 4 == 0)
      hipLaunchKernelGGL(linattn_join_kernel<4>, dim3((a.dk * a.dv / 4 + 255) / 256, a.Bt * a.Hv), dim3(256), 0, st, a, sg);
    else
      hipLaunchKernelGGL(linattn_join_kernel<1>, dim3((a.dk * a.dv + 255) / 256, a.Bt * a.Hv), dim3(256), 0, st, a, sg);
    QUAMBA_LAUNCH_CHECK();
  }
  hipLaunchKernelGGL((linattn_blocks_kernel<T, KT, NT, true, WIDE>), dim3((unsigned)(one * p.segments)), dim3(256), 0, st, a, sg);
  QUAMBA_LAUNCH_CHECK();
  return QUAMBA_OK;
}

// Rows that pass through registers leave too few of them for two column tiles a wave at KT = 4 (10 x 570, 29 heads of 85 x 176:
// 135 us with one, 338 with two).
template <typename T, bool WIDE>
int run_prefill(const LinAttnArgs &a, const AttnPlan &p, void *ws, hipStream_t st) {
  if (p.kt == 2) return p.nt == 1 ? run_blocks<T, 2, 1, WIDE>(a, p, ws, st) : run_blocks<T, 2, 2, WIDE>(a, p, ws, st);
  if constexpr (WIDE)
    if (p.kt == 4 && p.nt == 2) return run_blocks<T, 4, 2, WIDE>(a, p, ws, st);
  return p.kt == 4 ? run_blocks<T, 4, 1, WIDE>(a, p, ws, st) : run_blocks<T, 8, 1, WIDE>(a, p, ws, st);
}

// Rows that the direct-to-LDS loads can take: every row and head starts on 16 bytes, 64 rows lie within 2^31 bytes.
bool wide_rows(const LinAttnArgs &a) {
  const long long most = 1LL << 23;
  return aligned(a.q, 16) && aligned(a.k, 16) && aligned(a.v, 16) && aligned(a.out, 8) && a.ldq % 8 == 0 && a.ldk % 8 == 0 &&
         a.ldv % 8 == 0 && a.ldo % 4 == 0 && a.dk % 8 == 0 && a.dv % 8 == 0 && a.ldq < most && a.ldk < most && a.ldv < most && a.ldo < most;
}

int check(const char *what, int type, const LinAttnArgs &a) {
  if (type != QUAMBA_TYPE_F16 && type != QUAMBA_TYPE_BF16) return fail(QUAMBA_EUNSUPPORTED, "%s: operand type %d", what, type);
  if (a.Bt < 0 || a.L < 0 || a.Hk <= 0 || a.Hv <= 0 || a.dk <= 0 || a.dv <= 0)
    return fail(QUAMBA_EINVAL, "%s: Bt=%d L=%d Hk=%d Hv=%d dk=%d dv=%d", what, a.Bt, a.L, a.Hk, a.Hv, a.dk, a.dv);
  if (a.Hv % a.Hk) return fail(QUAMBA_EUNSUPPORTED, "%s: %d value heads are no multiple of %d key heads", what, a.Hv, a.Hk);
  if (a.dk > 256 || a.dv > 1024) return fail(QUAMBA_EUNSUPPORTED, "%s: dk=%d dv=%d (at most 256 and 1024)", what, a.dk, a.dv);
  if (a.L > 1 << 30) return fail(QUAMBA_EUNSUPPORTED, "%s: L=%d (at most 2^30)", what, a.L);
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
  if (Bt < 0 || L < 0 || Hk <= 0 || Hv <= 0 || dk <= 0 || dv <= 0 || dk > 256 || dv > 1024) {
    fail(QUAMBA_EINVAL, "linattn: Bt=%d L=%d Hk=%d Hv=%d dk=%d dv=%d", Bt, L, Hk, Hv, dk, dv);
    return 0;
  }
  return prefill_workspace(plan_prefill(Bt, L, Hv, dk, dv), Bt, Hv, dk, dv);
}

int quamba_linattn_prefill(int type, const void *q, int ldq, const void *k, int ldk, const void *v, int ldv, const float *log_decay,
                           int ldg, const int32_t *lens, int Bt, int L, int Hk, int Hv, int dk, int dv, float scale, void *out, int ldo,
                           float *state, void *ws, size_t ws_bytes, void *stream) {
  const LinAttnArgs a{q, k, v, ldq, ldk, ldv, log_decay, ldg, lens, Bt, L, Hk, Hv, dk, dv, scale, out, ldo, state};
  const int rc = check("linattn_prefill", type, a);
  if (rc != QUAMBA_OK || Bt == 0 || L == 0) return rc;
  if (ws && !aligned(ws, 256)) return fail(QUAMBA_EINVAL, "linattn_prefill: workspace must be 256-byte aligned");
  const AttnPlan p = plan_prefill(Bt, L, Hv, dk, dv, ws ? ws_bytes : 0);
  if (p.segments > 1 && (!ws || ws_bytes < prefill_workspace(p, Bt, Hv, dk, dv)))
    return fail(QUAMBA_EWORKSPACE, "linattn_prefill: workspace of %zu bytes, %zu needed", ws ? ws_bytes : (size_t)0, prefill_workspace(p, Bt, Hv, dk, dv));
  hipStream_t st = as_stream(stream);
  if (type == QUAMBA_TYPE_F16) return wide_rows(a) ? run_prefill<_Float16, true>(a, p, ws, st) : run_prefill<_Float16, false>(a, p, ws, st);
  return wide_rows(a) ? run_prefill<__bf16, true>(a, p, ws, st) : run_prefill<__bf16, false>(a, p, ws, st);
}

int quamba_linattn_step(int type, const void *q, int ldq, const void *k, int ldk, const void *v, int ldv, const float *log_decay,
                        int ldg, int Bt, int Hk, int Hv, int dk, int dv, float scale, void *out, int ldo, float *state, void *stream) {
  const LinAttnArgs a{q, k, v, ldq, ldk, ldv, log_decay, ldg, nullptr, Bt, 1, Hk, Hv, dk, dv, scale, out, ldo, state};
  const int rc = check("linattn_step", type, a);
  if (rc != QUAMBA_OK || Bt == 0) return rc;
  if (!state) return fail(QUAMBA_EINVAL, "linattn_step: state is required");
  hipStream_t st = as_stream(stream);
  if (type == QUAMBA_TYPE_F16) return dv % 4 == 0 ? run_step<_Float16, 4>(a, st) : run_step<_Float16, 1>(a, st);
  return dv % 4 == 0 ? run_step<__bf16, 4>(a, st) : run_step<__bf16, 1>(a, st);
}

}  // extern "C"

extern "C" void quamba_debug_set_linattn_blocks(int v) { quamba::g_segment_blocks.store(v); }

extern "C" int quamba_debug_linattn_blocks(int Bt, int L, int Hv, int dk, int dv, size_t ws_bytes) {
  if (Bt <= 0 || L <= 0 || Hv <= 0 || dk <= 0 || dv <= 0 || dk > 256 || dv > 1024) return -2;
  return quamba::plan_prefill(Bt, L, Hv, dk, dv, ws_bytes).blocks;
}
