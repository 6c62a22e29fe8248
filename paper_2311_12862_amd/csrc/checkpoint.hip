// 8-bit checkpoints of activations (see rows.h for the format): tensors into checkpoints and back, and the gradient
// through a ReLU whose output was kept as one.  Bandwidth-bound streaming kernels.
#include "common.h"
#include "rows.h"

#include <algorithm>

namespace spc {
namespace {

// A group of 32 / W lanes takes one block of a row.
template <typename T, int W>
__global__ void __launch_bounds__(256) k_q8_pack(const T* __restrict__ x, Q8Ref to, long long blocks, int C, int nb) {
  constexpr int G = kQ8Block / W;
  const long long stride = (long long)gridDim.x * (256 / G);
  const int lane = threadIdx.x % G;
  for (long long i = (long long)blockIdx.x * (256 / G) + threadIdx.x / G; i < blocks; i += stride) {
    const long long r = i / nb;
    const int col = (int)(i - r * nb) * kQ8Block + lane * W;
    const bool live = col < C;
    float v[W] = {};
    if (live) Chunk<T, W>::load(x, r * C + col, v);
    q8_keep<G, W>(to, r, C, nb, col, live, v);
  }
}

template <typename T, int W>
__global__ void __launch_bounds__(256) k_q8_unpack(Q8Ref from, T* __restrict__ out, long long chunks, int C, int nb) {
  const int cpr = C / W;  // chunks of a row
  const long long stride = (long long)gridDim.x * 256;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < chunks; i += stride) {
    const long long r = i / cpr;
    const int col = (int)(i - r * cpr) * W;
    int q[W];
    q8_load<W>(from.q, r * C + col, q);
    const float s = q8_scale(from.b[r * nb + col / kQ8Block]);
    float v[W];
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = q8_value(q[j], s);
    Chunk<T, W>::store(out, r * C + col, v);
  }
}

// out[i] = q[i] > 0 ? a[i] : 0 (out may be a)
template <typename T, int W>
__global__ void __launch_bounds__(256) k_relu_bwd_q8(const T* a, const signed char* __restrict__ q, T* out, long long chunks) {
  const long long stride = (long long)gridDim.x * 256;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < chunks; i += stride) {
    float v[W];
    int y[W];
    Chunk<T, W>::load(a, i * W, v);
    q8_load<W>(q, i * W, y);
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = y[j] > 0 ? v[j] : 0.f;
    Chunk<T, W>::store(out, i * W, v);
  }
}

unsigned grid_for(long long items, int per_block) {
  return (unsigned)std::min<long long>((items + per_block - 1) / per_block, 1 << 20);
}
bool aligned(const void* p, size_t n) { return ((size_t)p & (n - 1)) == 0; }

template <typename T> int launch_pack(const void* x, int64_t rows, int C, const Q8Ref& to, hipStream_t st) {
  constexpr int W = 16 / sizeof(T);
  const int nb = (C + kQ8Block - 1) / kQ8Block;
  const long long blocks = (long long)rows * nb;
  if (C % W == 0 && aligned(x, 16) && aligned(to.q, W))
    hipLaunchKernelGGL((k_q8_pack<T, W>), dim3(grid_for(blocks, 256 / (kQ8Block / W))), dim3(256), 0, st, (const T*)x, to, blocks, C, nb);
  else
    hipLaunchKernelGGL((k_q8_pack<T, 1>), dim3(grid_for(blocks, 256 / kQ8Block)), dim3(256), 0, st, (const T*)x, to, blocks, C, nb);
  SPC_LAUNCH_CHECK();
  return SPCONV_OK;
}
template <typename T> int launch_unpack(const Q8Ref& from, int64_t rows, int C, void* out, hipStream_t st) {
  constexpr int W = 16 / sizeof(T);
  const int nb = (C + kQ8Block - 1) / kQ8Block;
  if (C % W == 0 && aligned(out, 16) && aligned(from.q, W)) {
    const long long chunks = (long long)rows * (C / W);
    hipLaunchKernelGGL((k_q8_unpack<T, W>), dim3(grid_for(chunks, 256)), dim3(256), 0, st, from, (T*)out, chunks, C, nb);
  } else {
    const long long chunks = (long long)rows * C;
    hipLaunchKernelGGL((k_q8_unpack<T, 1>), dim3(grid_for(chunks, 256)), dim3(256), 0, st, from, (T*)out, chunks, C, nb);
  }
  SPC_LAUNCH_CHECK();
  return SPCONV_OK;
}
template <typename T> int launch_relu_bwd(const void* a, const signed char* q, int64_t n, void* out, hipStream_t st) {
  constexpr int W = 16 / sizeof(T);
  if (n % W == 0 && aligned(a, 16) && aligned(out, 16) && aligned(q, W))
    hipLaunchKernelGGL((k_relu_bwd_q8<T, W>), dim3(grid_for(n / W, 256)), dim3(256), 0, st, (const T*)a, q, (T*)out, n / W);
  else
    hipLaunchKernelGGL((k_relu_bwd_q8<T, 1>), dim3(grid_for(n, 256)), dim3(256), 0, st, (const T*)a, q, (T*)out, n);
  SPC_LAUNCH_CHECK();
  return SPCONV_OK;
}

}  // namespace

int q8_unpack(const spconv_q8* from, int64_t rows, int C, spconv_dtype dtype, void* out, hipStream_t st) {
  const Q8Ref f{(signed char*)from->data, from->exps};
  switch (dtype) {
    case SPCONV_F32: return launch_unpack<float>(f, rows, C, out, st);
    case SPCONV_F16: return launch_unpack<_Float16>(f, rows, C, out, st);
    case SPCONV_BF16: return launch_unpack<__bf16>(f, rows, C, out, st);
  }
  return SPCONV_EINVAL;
}

}  // namespace spc

using namespace spc;

extern "C" {

SPCONV_API int spconv_q8_pack(const void* x, int64_t rows, int C, spconv_dtype dtype, const spconv_q8* out, void* stream) {
  if (!row_shape_ok(rows, C) || !dtype_known(dtype) || !out) return SPCONV_EINVAL;
  if (rows == 0) return SPCONV_OK;
  if (!x || !out->data || !out->exps) return SPCONV_EINVAL;
  const Q8Ref to{(signed char*)out->data, out->exps};
  hipStream_t st = (hipStream_t)stream;
  switch (dtype) {
    case SPCONV_F32: return launch_pack<float>(x, rows, C, to, st);
    case SPCONV_F16: return launch_pack<_Float16>(x, rows, C, to, st);
    case SPCONV_BF16: return launch_pack<__bf16>(x, rows, C, to, st);
  }
  return SPCONV_EINVAL;
}

SPCONV_API int spconv_q8_unpack(const spconv_q8* kept, int64_t rows, int C, spconv_dtype dtype, void* out, void* stream) {
  if (!row_shape_ok(rows, C) || !dtype_known(dtype) || !kept) return SPCONV_EINVAL;
  if (rows == 0) return SPCONV_OK;
  if (!out || !kept->data || !kept->exps) return SPCONV_EINVAL;
  return q8_unpack(kept, rows, C, dtype, out, (hipStream_t)stream);
}

SPCONV_API int spconv_relu_bwd_q8(const void* dout, const spconv_q8* kept, void* out, int64_t n, spconv_dtype dtype, void* stream) {
  if (n < 0 || n > kRowMaxElements || !dtype_known(dtype) || !kept) return SPCONV_EINVAL;
  if (n == 0) return SPCONV_OK;
  if (!dout || !out || !kept->data) return SPCONV_EINVAL;
  const signed char* q = (const signed char*)kept->data;
  hipStream_t st = (hipStream_t)stream;
  switch (dtype) {
    case SPCONV_F32: return launch_relu_bwd<float>(dout, q, n, out, st);
    case SPCONV_F16: return launch_relu_bwd<_Float16>(dout, q, n, out, st);
    case SPCONV_BF16: return launch_relu_bwd<__bf16>(dout, q, n, out, st);
  }
  return SPCONV_EINVAL;
}

}  // extern "C"
