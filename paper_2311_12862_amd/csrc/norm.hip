// Layer norm over the channels of each row, with the residual add and the ReLU that stand behind it in a network, and its
// gradients.
//
//   forward   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), y = act((x - m) r w + b + res)
//   backward  g = dy where the ReLU let it through, xh = (x - m) r, h = g w,
//             dx = r (h - mean(h) - xh mean(h xh)), dw = sum over rows of g xh, db = sum over rows of g, dres = g
//
// A group of L lanes holds one row in registers, so every tensor crosses the memory once; statistics are taken in two passes
// over the registers, in fp32.  dw and db: every lane sums its columns over the rows it visits, the groups of a workgroup
// meet in LDS, the workgroups' sums in a second kernel, each in a fixed order: the same call gives the same bits.
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

struct BwdArgs {
  const void* dout;
  const void* x;       // or null: xq
  Q8Ref xq;
  const void* gate;    // or null: gate_q, or neither
  const signed char* gate_q;
  const float* w;      // or null: ones
  const float2* stats;
  void* dx;
  void* dres;          // or null
  float* partial;      // [workgroup][2][C], or null: no dw and db
  long long rows;
  int C, nb;
};

template <typename T, int W, int L, int NV> __global__ void __launch_bounds__(256) k_norm_fwd(const FwdArgs p) {
  const int lane = threadIdx.x % L;
  const float inv = 1.f / (float)p.C;
  const long long stride = (long long)gridDim.x * (256 / L);
  // (a wave's groups leave the loop together: lanes of rows past the end take part in the maxima)
  for (long long r0 = (long long)blockIdx.x * (256 / L) + threadIdx.x / 64 * (64 / L); r0 < p.rows; r0 += stride) {
    const long long r = r0 + threadIdx.x % 64 / L;
    const bool row = r < p.rows;
    float x[NV][W];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * L + lane) * W;
      const bool live = row && col < p.C;
#pragma unroll
      for (int i = 0; i < W; ++i) x[v][i] = 0.f;
      if (live) Chunk<T, W>::load(p.x, r * p.C + col, x[v]);
      if (p.kept_x.q) q8_keep<L, W>(p.kept_x, r, p.C, p.nb, col, live, x[v]);
#pragma unroll
      for (int i = 0; i < W; ++i) sum += x[v][i];
    }
    const float mean = group_sum<L>(sum) * inv;
    float sq = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const bool live = (v * L + lane) * W < p.C;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        x[v][i] = live ? x[v][i] - mean : 0.f;
        sq += x[v][i] * x[v][i];
      }
    }
    const float rstd = 1.f / sqrtf(group_sum<L>(sq) * inv + p.eps);
    if (p.stats && row && lane == 0) p.stats[r] = make_float2(mean, rstd);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * L + lane) * W;
      const bool live = row && col < p.C;
      float y[W] = {};
      if (live) {
        float w[W], b[W], res[W] = {};
        if (p.w) Chunk<float, W>::load(p.w, col, w);
        if (p.b) Chunk<float, W>::load(p.b, col, b);
        if (p.res) Chunk<T, W>::load(p.res, r * p.C + col, res);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          y[i] = x[v][i] * rstd;
          if (p.w) y[i] *= w[i];
          if (p.b) y[i] += b[i];
          y[i] += res[i];
          if (p.relu) y[i] = y[i] < 0.f ? 0.f : y[i];  // (a NaN stays one)
        }
        Chunk<T, W>::store(p.y, r * p.C + col, y);
      }
      if (p.kept_y.q) q8_keep<L, W>(p.kept_y, r, p.C, p.nb, col, live, y);  // of what was written
    }
  }
}

template <typename T, int W, int L, int NV> __global__ void __launch_bounds__(256) k_norm_bwd(const BwdArgs p) {
  const int lane = threadIdx.x % L;
  const float inv = 1.f / (float)p.C;
  float dw[NV][W] = {}, db[NV][W] = {};
  const long long stride = (long long)gridDim.x * (256 / L);
  for (long long r = (long long)blockIdx.x * (256 / L) + threadIdx.x / L; r < p.rows; r += stride) {
    const float2 st = p.stats[r];
    float g[NV][W], xh[NV][W];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * L + lane) * W;
#pragma unroll
      for (int i = 0; i < W; ++i) g[v][i] = xh[v][i] = 0.f;
      if (col < p.C) {
        const long long at = r * p.C + col;
        Chunk<T, W>::load(p.dout, at, g[v]);
        if (p.gate) {
          float y[W];
          Chunk<T, W>::load(p.gate, at, y);
#pragma unroll
          for (int i = 0; i < W; ++i) g[v][i] = y[i] > 0.f ? g[v][i] : 0.f;
        } else if (p.gate_q) {
          int y[W];
          q8_load<W>(p.gate_q, at, y);
#pragma unroll
          for (int i = 0; i < W; ++i) g[v][i] = y[i] > 0 ? g[v][i] : 0.f;
        }
        if (p.x) {
          Chunk<T, W>::load(p.x, at, xh[v]);
        } else {
          int q[W];
          q8_load<W>(p.xq.q, at, q);
          const float s = q8_scale(p.xq.b[r * p.nb + col / kQ8Block]);
#pragma unroll
          for (int i = 0; i < W; ++i) xh[v][i] = q8_value(q[i], s);
        }
        float w[W];
        if (p.w) Chunk<float, W>::load(p.w, col, w);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          xh[v][i] = (xh[v][i] - st.x) * st.y;
          const float h = p.w ? g[v][i] * w[i] : g[v][i];
          s1 += h;
          s2 += h * xh[v][i];
          dw[v][i] += g[v][i] * xh[v][i];
          db[v][i] += g[v][i];
        }
      }
    }
    const float c1 = group_sum<L>(s1) * inv, c2 = group_sum<L>(s2) * inv;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * L + lane) * W;
      if (col < p.C) {
        const long long at = r * p.C + col;
        float w[W], dx[W];
        if (p.w) Chunk<float, W>::load(p.w, col, w);
#pragma unroll
        for (int i = 0; i < W; ++i) dx[i] = st.y * ((p.w ? g[v][i] * w[i] : g[v][i]) - c1 - xh[v][i] * c2);
        if (p.dres) Chunk<T, W>::store(p.dres, at, g[v]);
        Chunk<T, W>::store(p.dx, at, dx);
      }
    }
  }
  if (!p.partial) return;
  __shared__ float sums[2][4][L * W];
  const int wave = threadIdx.x / 64;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
#pragma unroll
      for (int o = L; o < 64; o <<= 1) {
        dw[v][i] += __shfl_xor(dw[v][i], o);
        db[v][i] += __shfl_xor(db[v][i], o);
      }
      if (threadIdx.x % 64 < L) {
        sums[0][wave][lane * W + i] = dw[v][i];
        sums[1][wave][lane * W + i] = db[v][i];
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * L * W; e += 256) {
      const int which = e / (L * W), c = e % (L * W), col = v * L * W + c;
      if (col < p.C)
        p.partial[((long long)blockIdx.x * 2 + which) * p.C + col] =
            sums[which][0][c] + sums[which][1][c] + sums[which][2][c] + sums[which][3][c];
    }
    __syncthreads();
  }
}

// dw and db: 16 columns of the workgroups' sums to a workgroup, 64 stripes, added in order
__global__ void __launch_bounds__(1024) k_norm_sum(const float* __restrict__ partial, int groups, int C, float* __restrict__ dw,
                                                   float* __restrict__ db) {
  __shared__ float part[64][17];
  const int c = threadIdx.x % 16, stripe = threadIdx.x / 16;
  const int col = blockIdx.x * 16 + c;
  float s = 0.f;
  if (col < 2 * C) {
#pragma unroll 8
    for (int g = stripe; g < groups; g += 64) s += partial[(long long)g * 2 * C + col];
  }
  part[stripe][c] = s;
  __syncthreads();
  if (threadIdx.x < 16 && col < 2 * C) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) t += part[i][threadIdx.x];
    (col < C ? dw : db)[col < C ? col : col - C] = t;
  }
}

bool aligned(const void* p, size_t n) { return ((size_t)p & (n - 1)) == 0; }

constexpr int kBwdGroups = 1024;  // workgroups at most

unsigned bwd_groups(int64_t rows, int per_group) {
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, per_group), kBwdGroups));
}

// Lanes of a row and vectors of a lane: as few lanes as hold the row with one vector each (a block of a checkpoint needs 32 / W lanes
// where the row has one), beyond 64 lanes more vectors.
template <template <typename, int, int, int> class Go, typename T, int W, typename Args> int pick(int C, const Args& a, hipStream_t st) {
  const int n = (C + W - 1) / W;
  if constexpr (W > 1) {
    if (n <= 4) return Go<T, W, 4, 1>::run(a, st);
    if (n <= 8) return Go<T, W, 8, 1>::run(a, st);
  }
  if (n <= 16) return Go<T, W, 16, 1>::run(a, st);
  if (n <= 32) return Go<T, W, 32, 1>::run(a, st);
  if (n <= 64) return Go<T, W, 64, 1>::run(a, st);
  if (n <= 128) return Go<T, W, 64, 2>::run(a, st);
  if (n <= 256) return Go<T, W, 64, 4>::run(a, st);
  if (n <= 512) return Go<T, W, 64, 8>::run(a, st);
  if constexpr (W <= 4) {
    if (n <= 1024) return Go<T, W, 64, 16>::run(a, st);
  }
  if constexpr (W == 1) {
    if (n <= 4096) return Go<T, W, 64, 64>::run(a, st);
  }
  return SPCONV_EINVAL;
}

template <typename T, int W, int L, int NV> struct Fwd {
  static int run(const FwdArgs& a, hipStream_t st) {
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(a.rows, 256 / L), 1 << 20);
    hipLaunchKernelGGL((k_norm_fwd<T, W, L, NV>), dim3(grid), dim3(256), 0, st, a);
    SPC_LAUNCH_CHECK();
    return SPCONV_OK;
  }
};
template <typename T, int W, int L, int NV> struct Bwd {
  static int run(const BwdArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((k_norm_bwd<T, W, L, NV>), dim3(bwd_groups(a.rows, 256 / L)), dim3(256), 0, st, a);
    SPC_LAUNCH_CHECK();
    return SPCONV_OK;
  }
};

template <typename T> bool fwd_vectors(const FwdArgs& a) {
  constexpr int W = 16 / sizeof(T);
  return a.C % W == 0 && aligned(a.x, 16) && aligned(a.res, 16) && aligned(a.y, 16) && aligned(a.w, 16) && aligned(a.b, 16) &&
         aligned(a.kept_x.q, W) && aligned(a.kept_y.q, W);
}
template <typename T> int launch_fwd(const FwdArgs& a, hipStream_t st) {
  constexpr int W = 16 / sizeof(T);
  return fwd_vectors<T>(a) ? pick<Fwd, T, W>(a.C, a, st) : pick<Fwd, T, 1>(a.C, a, st);
}
template <typename T> bool bwd_vectors(const BwdArgs& a) {
  constexpr int W = 16 / sizeof(T);
  return a.C % W == 0 && aligned(a.dout, 16) && aligned(a.x, 16) && aligned(a.gate, 16) && aligned(a.dx, 16) && aligned(a.dres, 16) &&
         aligned(a.w, 16) && aligned(a.xq.q, W) && aligned(a.gate_q, W);
}
template <typename T> int launch_bwd(const BwdArgs& a, float* dw, float* db, hipStream_t st) {
  constexpr int W = 16 / sizeof(T);
  const bool vectors = bwd_vectors<T>(a);
  SPC_TRY(vectors ? (pick<Bwd, T, W>(a.C, a, st)) : (pick<Bwd, T, 1>(a.C, a, st)));
  if (!a.partial) return SPCONV_OK;
  const int w = vectors ? W : 1, n = (a.C + w - 1) / w;
  const int L = n <= 4 && w > 1 ? 4 : n <= 8 && w > 1 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : 64;
  const int groups = (int)bwd_groups(a.rows, 256 / L);
  hipLaunchKernelGGL(k_norm_sum, dim3((unsigned)ceil_div(2 * a.C, 16)), dim3(1024), 0, st, a.partial, groups, a.C, dw, db);
  SPC_LAUNCH_CHECK();
  return SPCONV_OK;
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

SPCONV_API int64_t spconv_layer_norm_bwd_workspace(int64_t rows, int C) {
  if (!row_shape_ok(rows, C)) return SPCONV_EINVAL;
  return (int64_t)kBwdGroups * 2 * C * (int64_t)sizeof(float);
}

SPCONV_API int spconv_layer_norm_bwd(const void* dout, const void* x, const spconv_q8* kept_x, const void* y, const spconv_q8* kept_y,
                                     const float* weight, const float* stats, int64_t rows, int C, spconv_dtype dtype, void* dx,
                                     void* dresidual, float* dweight, float* dbias, void* workspace, int64_t workspace_bytes,
                                     void* stream) {
  if (!row_shape_ok(rows, C) || !dtype_known(dtype) || !dweight != !dbias || (x && kept_x) || (y && kept_y)) return SPCONV_EINVAL;
  if (dweight && (!workspace || workspace_bytes < spconv_layer_norm_bwd_workspace(rows, C))) return SPCONV_EINVAL;
  if (rows > 0 && (!dout || (!x && !kept_x) || !stats || !dx)) return SPCONV_EINVAL;
  if (rows > 0 && ((kept_x && !(kept_x->data && kept_x->exps)) || (kept_y && !(kept_y->data && kept_y->exps)))) return SPCONV_EINVAL;
  if (rows == 0 && !dweight) return SPCONV_OK;
  BwdArgs a{};
  a.dout = dout;
  a.x = x;
  if (kept_x) a.xq = Q8Ref{(signed char*)kept_x->data, kept_x->exps};
  a.gate = y;
  a.gate_q = kept_y ? (const signed char*)kept_y->data : nullptr;
  a.w = weight;
  a.stats = (const float2*)stats;
  a.dx = dx;
  a.dres = dresidual;
  a.partial = dweight ? (float*)workspace : nullptr;
  a.rows = rows;
  a.C = C;
  a.nb = (C + kQ8Block - 1) / kQ8Block;
  hipStream_t st = (hipStream_t)stream;
  switch (dtype) {
    case SPCONV_F32: return launch_bwd<float>(a, dweight, dbias, st);
    case SPCONV_F16: return launch_bwd<_Float16>(a, dweight, dbias, st);
    case SPCONV_BF16: return launch_bwd<__bf16>(a, dweight, dbias, st);
  }
  return SPCONV_EINVAL;
}

}  // extern "C"
