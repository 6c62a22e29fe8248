// Gradients of layer norm with the residual add and the ReLU behind it (norm.hip).
//
//   g = dy where the ReLU let it through, xh = (x - m) r, h = g w,
//   dx = r (h - mean(h) - xh mean(h xh)), dw = sum over rows of g xh, db = sum over rows of g, dres = g
//
// A group of L lanes holds one row in registers, so every tensor crosses the memory once; x and the gate come from tensors or from
// 8-bit checkpoints.  dw and db: every lane sums its columns over the rows it visits, the groups of a workgroup meet in LDS, the
// workgroups' sums in a second kernel, each in a fixed order: the same call gives the same bits.
// Memory bounds it, and its latency: the next row is loaded ahead of the current one's sums (300k rows of 256 bf16, x and gate from
// checkpoints, with the residual's gradient: 154 -> 113 us, 5.4 TB/s; 9k rows of 256 f16 8 us, the sums 3 to 5).
#include "common.h"
#include "rows.h"

#include <algorithm>

namespace spc {
namespace {

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
  float* dw;           // sums of workgroup g at dw + g * step and db + g * step, or null: none
  float* db;
  int step;
  long long rows;
  int C, nb;
};

// One row of a group, as it is in memory (x, y: in a checkpoint's case its bytes, in the first words).
template <int NV> struct BwdRow {
  raw16 d[NV], x[NV], y[NV];
  unsigned b[NV];
  float2 st;
};

template <int W> __device__ __forceinline__ typename Bytes<W>::word bytes_of(raw16 r) {
  typename Bytes<W>::word q;
#pragma unroll
  for (int j = 0; j < W / 4; ++j) q[j] = r[j];
  return q;
}
template <int W> __device__ __forceinline__ raw16 raw_of(typename Bytes<W>::word q) {
  raw16 r = {};
#pragma unroll
  for (int j = 0; j < W / 4; ++j) r[j] = q[j];
  return r;
}

template <typename T, int L, int NV, Ends E> __global__ void __launch_bounds__(256) k_norm_bwd(const BwdArgs p) {
  constexpr int W = Row<T>::W, R = 256 / L;
  constexpr bool kAhead = NV == 1;  // the next row is on its way while this one is worked on
  __shared__ float part[2][4];
  const int lane = threadIdx.x % L, rl = threadIdx.x / L;
  const int C = p.C;
  const float inv = 1.f / (float)C;
  float dw[NV][W] = {}, db[NV][W] = {}, w[NV][W];
  Place at[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    at[v] = place_in_row<W>(v * L + lane, C);
#pragma unroll
    for (int i = 0; i < W; ++i) w[v][i] = 1.f;
    if (p.w && at[v].live) load_floats<E, W>(p.w + at[v].col, at[v], w[v]);
  }
  // (the workgroup's first row r0 is the same for all its lanes: addresses are a scalar base and 32 bits per lane)
  auto load = [&](long long r0, BwdRow<NV>& a) {
    const bool row = rl < p.rows - r0;
    const long long e0 = r0 * C;
    a.st = make_float2(0.f, 0.f);
    if (row) a.st = p.stats[r0 + rl];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      a.d[v] = a.x[v] = a.y[v] = raw16{0, 0, 0, 0};
      a.b[v] = 0;
      if (row && at[v].live) {
        const int e = rl * C + at[v].col;
        a.d[v] = Row<T>::template load<E>((const T*)p.dout + e0 + e, at[v]);
        if (p.x) {
          a.x[v] = Row<T>::template load<E>((const T*)p.x + e0 + e, at[v]);
        } else {
          a.x[v] = raw_of<W>(q8_load<E, W>(p.xq.q + e0 + e, at[v]));
          a.b[v] = p.xq.b[r0 * p.nb + (rl * p.nb + at[v].block)];
        }
        if (p.gate) a.y[v] = Row<T>::template load<E>((const T*)p.gate + e0 + e, at[v]);
        else if (p.gate_q) a.y[v] = raw_of<W>(q8_load<E, W>(p.gate_q + e0 + e, at[v]));
      }
    }
  };
  const long long step = (long long)gridDim.x * R;
  long long r0 = (long long)blockIdx.x * R;
  BwdRow<NV> a;
  if (kAhead && r0 < p.rows) load(r0, a);
  for (; r0 < p.rows; r0 += step) {
    BwdRow<NV> next;
    if constexpr (kAhead) {
      if (r0 + step < p.rows) load(r0 + step, next);
    } else {
      load(r0, a);
    }
    const bool row = rl < p.rows - r0;
    const long long e0 = r0 * C;
    float g[NV][W], xh[NV][W];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Row<T>::widen(a.d[v], g[v]);
      if (p.gate) {
        float y[W];
        Row<T>::widen(a.y[v], y);
#pragma unroll
        for (int i = 0; i < W; ++i) g[v][i] = y[i] > 0.f ? g[v][i] : 0.f;
      } else if (p.gate_q) {
        const auto y = bytes_of<W>(a.y[v]);
#pragma unroll
        for (int i = 0; i < W; ++i) g[v][i] = q8_at<W>(y, i) > 0 ? g[v][i] : 0.f;
      }
      own_only<E>(at[v], g[v]);
      if (p.x) Row<T>::widen(a.x[v], xh[v]);
      else q8_widen<W>(bytes_of<W>(a.x[v]), q8_step(a.b[v]), xh[v]);
      const float m = at[v].live ? a.st.x : 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) xh[v][i] = (xh[v][i] - m) * a.st.y;
      own_only<E>(at[v], xh[v]);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float h = g[v][i] * w[v][i];
        s1 += h;
        s2 += h * xh[v][i];
        dw[v][i] += g[v][i] * xh[v][i];
        db[v][i] += g[v][i];
      }
    }
    const float c1 = group_sum<L>(s1, part, 0) * inv, c2 = group_sum<L>(s2, part, 1) * inv;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (row && at[v].live) {
        const int e = rl * C + at[v].col;
        float dx[W];
#pragma unroll
        for (int i = 0; i < W; ++i) dx[i] = a.st.y * (g[v][i] * w[v][i] - c1 - xh[v][i] * c2);
        if (p.dres) Row<T>::template store<E>((T*)p.dres + e0 + e, at[v], Row<T>::narrow(g[v]));
        Row<T>::template store<E>((T*)p.dx + e0 + e, at[v], Row<T>::narrow(dx));
      }
    }
    if constexpr (kAhead) a = next;
  }
  if (!p.dw) return;
  float* const to_w = p.dw + (long long)blockIdx.x * p.step;
  float* const to_b = p.db + (long long)blockIdx.x * p.step;
  if constexpr (L == 256) {  // a lane's columns are its own
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < W; ++i)
        if (at[v].live && i >= at[v].lo) {
          to_w[at[v].col + i] = dw[v][i];
          to_b[at[v].col + i] = db[v][i];
        }
  } else {
    static_assert(NV == 1, "");
    constexpr int M = L < 64 ? 4 : 256 / L;  // sums of a column: of four waves, or of the groups
    __shared__ float sums[2][M][L * W];
    const int m = L < 64 ? threadIdx.x / 64 : threadIdx.x / L;
#pragma unroll
    for (int i = 0; i < W; ++i) {
#pragma unroll
      for (int o = L; o < 64; o <<= 1) {
        dw[0][i] += __shfl_xor(dw[0][i], o);
        db[0][i] += __shfl_xor(db[0][i], o);
      }
      if (L >= 64 || threadIdx.x % 64 < L) {
        sums[0][m][lane * W + i] = dw[0][i];
        sums[1][m][lane * W + i] = db[0][i];
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * L * W; e += 256) {
      const int which = e / (L * W), c = e % (L * W);
      const Place of = place_in_row<W>(c / W, C);
      float t = sums[which][0][c];
#pragma unroll
      for (int k = 1; k < M; ++k) t += sums[which][k][c];
      if (of.live && c % W >= of.lo) (which ? to_b : to_w)[of.col + c % W] = t;
    }
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

// Workgroups at most, each with its row of partial sums, and no more than the GPU holds: four a CU (300k rows of 256 bf16: 512 157 us, 1024
// 113, 2048 124); five where x is a checkpoint, with fewer bytes to wait for and more to compute, and a workgroup has 16 turns or more, so
// that the longer sum is made up for.  1024 and 1280, us: from checkpoints 300k x 256 fp16 96 and 94, 170k x 448 101 and 96, x 450 fp32 191 and
// 169, 40k x 256 fp16 20.0 and 21.6, 100k x 64 15.6 and 17.4; from tensors 300k x 256 92 and 95, 170k x 450 fp32 173 and 184.
constexpr int kBwdGroups = 1280;
int bwd_groups(bool kept, int64_t blocks) { return kept && blocks >= 16 * kBwdGroups ? kBwdGroups : 1024; }

// One workgroup for so few elements (counted with the idle lanes) that a second launch - 4 us on the host with its workspace, 4 to 5 on the
// GPU - costs more than the wait for one row after the other, up to 16 turns of 0.5 to 0.9 us; it writes dw and db itself.  A call, us, one
// workgroup and more: 8k elements 11.2, 15.8; 16k f16 of 256 11.1, 15.8; fp32 of 256 12.0, 15.9; 32k fp32 of 64 20, 16.
// (Calls without dw and db have no second launch to save, and run on one workgroup all the same: 16k f16 of 32 6.5, one row more 5.5.)
constexpr int64_t kBwdAlone = 16384;
bool alone(int64_t rows, int C) {
  int wide = 32;
  while (wide < C) wide *= 2;
  return rows * wide <= kBwdAlone;
}

// a.dw, a.db: where the sums go in the end, or null
template <typename T> int launch_bwd(const BwdArgs& args, float* workspace, hipStream_t st) {
  return with_lanes<Row<T>::W>(args.C, [&](auto l) {
    constexpr int L = decltype(l)::L, NV = decltype(l)::NV;
    const auto kernel = k_norm_bwd<T, L, NV, decltype(l)::E>;
    static std::atomic<int> held{0};
    const int64_t blocks = ceil_div(args.rows, 256 / L);
    const int groups = alone(args.rows, args.C)
                           ? 1
                           : (int)std::min<int64_t>(blocks, std::min(bwd_groups(!args.x, blocks), resident_groups(kernel, held)));
    BwdArgs a = args;
    if (args.dw && !alone(args.rows, args.C)) {
      a.dw = workspace;
      a.db = workspace + args.C;
      a.step = 2 * args.C;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, st, a);
    SPC_LAUNCH_CHECK();
    if (a.dw == args.dw) return (int)SPCONV_OK;
    hipLaunchKernelGGL(k_norm_sum, dim3((unsigned)ceil_div(2 * a.C, 16)), dim3(1024), 0, st, workspace, groups, a.C, args.dw, args.db);
    SPC_LAUNCH_CHECK();
    return (int)SPCONV_OK;
  });
}

}  // namespace
}  // namespace spc

using namespace spc;

extern "C" {

SPCONV_API int64_t spconv_layer_norm_bwd_workspace(int64_t rows, int C) {
  if (!row_shape_ok(rows, C)) return SPCONV_EINVAL;
  return alone(rows, C) ? 0 : (int64_t)kBwdGroups * 2 * C * (int64_t)sizeof(float);
}

SPCONV_API int spconv_layer_norm_bwd(const void* dout, const void* x, const spconv_q8* kept_x, const void* y, const spconv_q8* kept_y,
                                     const float* weight, const float* stats, int64_t rows, int C, spconv_dtype dtype, void* dx,
                                     void* dresidual, float* dweight, float* dbias, void* workspace, int64_t workspace_bytes,
                                     void* stream) {
  if (!row_shape_ok(rows, C) || !dtype_known(dtype) || !dweight != !dbias || (x && kept_x) || (y && kept_y)) return SPCONV_EINVAL;
  const int64_t need = spconv_layer_norm_bwd_workspace(rows, C);
  if (dweight && need > 0 && (!workspace || workspace_bytes < need)) return SPCONV_EINVAL;
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
  a.dw = dweight;
  a.db = dbias;
  a.rows = rows;
  a.C = C;
  a.nb = (C + kQ8Block - 1) / kQ8Block;
  hipStream_t st = (hipStream_t)stream;
  switch (dtype) {
    case SPCONV_F32: return launch_bwd<float>(a, (float*)workspace, st);
    case SPCONV_F16: return launch_bwd<_Float16>(a, (float*)workspace, st);
    case SPCONV_BF16: return launch_bwd<__bf16>(a, (float*)workspace, st);
  }
  return SPCONV_EINVAL;
}

}  // extern "C"
