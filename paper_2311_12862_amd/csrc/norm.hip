// Layer norm over the channels of each row, with the residual add and the ReLU that stand behind it in a network.
//
//   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), y = act((x - m) r w + b + res)
//
// A group of L lanes holds one row in registers, so every tensor crosses the memory once; statistics are taken in two passes
// over the registers, in fp32.  A first mean m0 is off by its sum's roundings, in units of the values' last place, which r would blow up
// where the offset is far above the spread (60000 throughout, 13 wide: y of 0.78 and not 0).  So d = mean(x - m0) goes
// with the squares, m = m0 + d, and mean((x - m)^2) = mean((x - m0)^2) - d^2: a row without variance has x - m = 0.  The correction costs
// 0 to 5 % (170k x 450 f16 73.4 us without, 75.8; 100k x 64 f16 with both checkpoints 9.0, 9.4).
// Memory bounds it: 300k rows of 256 bf16 with a residual 86 us, 5.4 TB/s; 300k of 256 f16 with both checkpoints 100, 4.7 TB/s (5 more
// where 8-bit rounding took 9 instructions an element and not 6).
#include "common.h"
#include "rows.h"

#include <algorithm>

namespace spc {
namespace {

struct FwdArgs {
  const void* x;
  const void* res;     // or null
  const float* w;      // or null: ones
  const float* b;      // or null: zeros
  void* y;
  float2* stats;       // or null
  Q8Ref kept_x, kept_y;  // q null: not kept
  long long rows;
  int C, nb, relu;
  float eps;
};

// Workgroups a CU is to hold where a lane has one vector.  Scalar registers decide it (masks of lanes, bases of nine tensors): a wave of
// eight has 80 of them, which the count of resident workgroups leaves out.  For want of 2 to 30 of them launches of eight ran as seven or
// six, with a second round (77M elements in fp16, 38M in fp32, with no checkpoint, of x, of x and y, us, before the mean was corrected: fp32 256 wide 81, 102, 110,
// bounded 58, 73, 83; fp16 450 wide 108, 133, 167, bounded 72, 95, 128; fp32 512 wide 85, 89, 103, bounded 62, 70, 83).  The price: kernels of odd widths keep some 30 scalars in lanes of vector registers, and the 16-bit
// one of 128 lanes 12 bytes a lane in scratch memory.
template <int NV, Ends E> constexpr int kFwdHeld = NV == 1 && E != kBelowVector ? 8 : 0;

// s / c rounded to nearest, inv = 1 / c rounded to nearest (P. Markstein, 1990: one step from the product).  What the correction rests
// on: c equal differences have their own value as the mean.
__device__ __forceinline__ float over(float s, float c, float inv) {
  const float q = s * inv, rest = __builtin_fmaf(-q, c, s);
  return rest == rest ? __builtin_fmaf(rest, inv, q) : q;  // (squares that overflow stay infinite)
}

template <typename T, int L, int NV, Ends E>
__global__ void __launch_bounds__(256, (kFwdHeld<NV, E> ? kFwdHeld<NV, E> : 1)) k_norm_fwd(const FwdArgs p) {
  constexpr int W = Row<T>::W, R = 256 / L;
  __shared__ float part[3][4];
  const int lane = threadIdx.x % L, rl = threadIdx.x / L;
  const int C = p.C;
  const float inv = 1.f / (float)C;
  Place at[NV];
  int element[NV], block[NV];  // behind the workgroup's first row, which all its lanes share
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    at[v] = place_in_row<W>(v * L + lane, C);
    element[v] = rl * C + at[v].col;
    block[v] = rl * p.nb + at[v].block;
  }
  for (long long r0 = (long long)blockIdx.x * R; r0 < p.rows; r0 += (long long)gridDim.x * R) {
    const bool row = rl < p.rows - r0;
    const long long e0 = r0 * C;
    float x[NV][W];
    raw16 raw[NV], res[NV];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      each_row(element[v]);
      each_row(block[v]);
      each_row(at[v].col);
      raw[v] = res[v] = raw16{0, 0, 0, 0};
      if (row && at[v].live) {
        raw[v] = Row<T>::template load<E>(behind<E>((const T*)p.x + e0, element[v]), at[v]);
        if (p.res) res[v] = Row<T>::template load<E>(behind<E>((const T*)p.res + e0, element[v]), at[v]);
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Row<T>::widen(raw[v], x[v]);
      own_only<E>(at[v], x[v]);
      if (p.kept_x.q)
        q8_keep<E, L, W>(behind<E>(p.kept_x.q + e0, element[v]), behind<E>(p.kept_x.b + r0 * p.nb, block[v]), at[v], row && at[v].live, x[v]);
#pragma unroll
      for (int i = 0; i < W; ++i) sum += x[v][i];
    }
    const float first = group_sum<L>(sum, part, 0) * inv;
    float d = 0.f, sq = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const float m = at[v].live ? first : 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) x[v][i] -= m;
      own_only<E>(at[v], x[v]);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        d += x[v][i];
        sq += x[v][i] * x[v][i];
      }
    }
    group_sums<L>(d, sq, part + 1);
    d = over(d, (float)C, inv);
    sq = over(sq, (float)C, inv);
    const float d2 = d * d, var = d2 >= sq ? 0.f : sq - d2;  // (d2 and sq may overflow together; a NaN stays one)
    // (v_rsq is good to one unit of the last place, as its argument is at best; it takes no subnormal numbers)
    const float rstd = __builtin_amdgcn_rsqf(__builtin_elementwise_maximum(var + p.eps, 0x1p-126f));
    if (p.stats && row && lane == 0) p.stats[r0 + rl] = make_float2(d == d ? first + d : first, rstd);  // (an infinite mean stays one)
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < W; ++i) x[v][i] -= d;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const bool live = row && at[v].live;
      float y[W], t[W];
#pragma unroll
      for (int i = 0; i < W; ++i) y[i] = x[v][i] * rstd;
      if (p.w) {
        if (live) load_floats<E, W>(behind<E>(p.w, at[v].col), at[v], t);
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] *= t[i];
      }
      if (p.b) {
        if (live) load_floats<E, W>(behind<E>(p.b, at[v].col), at[v], t);
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] += t[i];
      }
      if (p.res) {
        Row<T>::widen(res[v], t);
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] += t[i];
      }
      if (p.relu) {
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] = __builtin_elementwise_maximum(y[i], 0.f);  // (a NaN stays one)
      }
      const raw16 out = Row<T>::narrow(y);
      if (live) Row<T>::template store<E>(behind<E>((T*)p.y + e0, element[v]), at[v], out);
      if (p.kept_y.q) {  // of what was written
        Row<T>::widen(out, y);
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] = live && (E == kWholeVectors || i >= at[v].lo) ? y[i] : 0.f;
        q8_keep<E, L, W>(behind<E>(p.kept_y.q + e0, element[v]), behind<E>(p.kept_y.b + r0 * p.nb, block[v]), at[v], live, y);
      }
    }
  }
}

template <typename T> int launch_fwd(const FwdArgs& a, hipStream_t st) {
  return with_lanes<Row<T>::W>(a.C, [&](auto l) {
    constexpr int L = decltype(l)::L, NV = decltype(l)::NV;
    constexpr int kHeld = kFwdHeld<NV, decltype(l)::E>;
    const auto kernel = k_norm_fwd<T, L, NV, decltype(l)::E>;
    static std::atomic<int> held{0};
    // (one workgroup per 256 / L rows: 300k rows of 256 bf16 with a residual 93 us, so 85)
    const int groups = kHeld ? 256 * kHeld : resident_groups(kernel, held);
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(a.rows, 256 / L), groups);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, st, a);
    SPC_LAUNCH_CHECK();
    return (int)SPCONV_OK;
  });
}

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" {

SPCONV_API int spconv_layer_norm_fwd(const void* x, const void* residual, const float* weight, const float* bias, float eps, int relu,
                                     int64_t rows, int C, spconv_dtype dtype, void* y, float* stats, const spconv_q8* keep_x,
                                     const spconv_q8* keep_y, void* stream) {
  if (!row_shape_ok(rows, C) || !dtype_known(dtype) || !(eps >= 0.f) || relu < 0 || relu > 1) return SPCONV_EINVAL;
  if (rows == 0) return SPCONV_OK;
  if (!x || !y || (keep_x && !(keep_x->data && keep_x->exps)) || (keep_y && !(keep_y->data && keep_y->exps))) return SPCONV_EINVAL;
  if (keep_x && keep_y && (keep_x->data == keep_y->data || keep_x->exps == keep_y->exps)) return SPCONV_EINVAL;
  FwdArgs a{};
  a.x = x;
  a.res = residual;
  a.w = weight;
  a.b = bias;
  a.y = y;
  a.stats = (float2*)stats;
  if (keep_x) a.kept_x = Q8Ref{(signed char*)keep_x->data, keep_x->exps};
  if (keep_y) a.kept_y = Q8Ref{(signed char*)keep_y->data, keep_y->exps};
  a.rows = rows;
  a.C = C;
  a.nb = (C + kQ8Block - 1) / kQ8Block;
  a.relu = relu;
  a.eps = eps;
  hipStream_t st = (hipStream_t)stream;
  switch (dtype) {
    case SPCONV_F32: return launch_fwd<float>(a, st);
    case SPCONV_F16: return launch_fwd<_Float16>(a, st);
    case SPCONV_BF16: return launch_fwd<__bf16>(a, st);
  }
  return SPCONV_EINVAL;
}

}  // extern "C"
