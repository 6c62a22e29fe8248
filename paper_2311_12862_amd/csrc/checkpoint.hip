// 8-bit checkpoints of activations (see rows.h for the format): tensors into checkpoints and back, and the gradient
// through a ReLU whose output was kept as one.  Bandwidth-bound streaming kernels: 300k rows of 256 bf16 pack 46 us (5.0 TB/s), unpack
// 36 (6.5), ReLU gradient 71 (5.4); 60k rows of 45 fp32 pack 5.8, unpack 5.6.
#include "common.h"
#include "rows.h"

#include <algorithm>

namespace spc {
namespace {

// Rows of C channels, a group of L lanes each; 256 / L rows of a workgroup, whose first is the same for all its lanes (addresses are a
// scalar base and 32 bits per lane).
template <typename T, int L, int NV, Ends E>
__global__ void __launch_bounds__(256) k_q8_pack(const T* __restrict__ x, Q8Ref to, long long rows, int C, int nb) {
  constexpr int W = Row<T>::W, R = 256 / L;
  const int lane = threadIdx.x % L, rl = threadIdx.x / L;
  for (long long r0 = (long long)blockIdx.x * R; r0 < rows; r0 += (long long)gridDim.x * R) {
    const bool row = rl < rows - r0;
    const T* xr = x + r0 * C;
    signed char* q = to.q + r0 * C;
    unsigned char* b = to.b + r0 * nb;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place at = place_in_row<W>(v * L + lane, C);
      const bool live = row && at.live;
      raw16 raw = {};
      if (live) raw = Row<T>::template load<E>(xr + (rl * C + at.col), at);
      float f[W];
      Row<T>::widen(raw, f);
      own_only<E>(at, f);
      q8_keep<E, L, W>(q + (rl * C + at.col), b + (rl * nb + at.block), at, live, f);
    }
  }
}

template <typename T, int L, int NV, Ends E>
__global__ void __launch_bounds__(256) k_q8_unpack(Q8Ref from, T* __restrict__ out, long long rows, int C, int nb) {
  constexpr int W = Row<T>::W, R = 256 / L;
  const int lane = threadIdx.x % L, rl = threadIdx.x / L;
  for (long long r0 = (long long)blockIdx.x * R; r0 < rows; r0 += (long long)gridDim.x * R) {
    const signed char* q = from.q + r0 * C;
    const unsigned char* b = from.b + r0 * nb;
    T* o = out + r0 * C;
    if (rl >= rows - r0) continue;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place at = place_in_row<W>(v * L + lane, C);
      if (at.live) {
        const auto w = q8_load<E, W>(q + (rl * C + at.col), at);
        float f[W];
        q8_widen<W>(w, q8_step(b[rl * nb + at.block]), f);
        Row<T>::template store<E>(o + (rl * C + at.col), at, Row<T>::narrow(f));
      }
    }
  }
}

// out[i] = q[i] > 0 ? a[i] : 0 (out may be a)
template <typename T> __global__ void __launch_bounds__(256) k_relu_bwd_q8(const T* a, const signed char* __restrict__ q, T* out, long long n) {
  constexpr int W = Row<T>::W;
  for (long long i0 = (long long)blockIdx.x * (256 * W); i0 < n; i0 += (long long)gridDim.x * (256 * W)) {
    const T* pa = a + i0;
    const signed char* pq = q + i0;
    T* po = out + i0;
    const int i = threadIdx.x * W;
    if (i + W <= n - i0) {
      typename Row<T>::vec v = __builtin_bit_cast(typename Row<T>::vec, load_any<raw16>(pa + i));
      const auto y = load_any<typename Bytes<W>::word>(pq + i);
#pragma unroll
      for (int j = 0; j < W; ++j) v[j] = q8_at<W>(y, j) > 0 ? v[j] : (T)0.f;
      store_any(po + i, __builtin_bit_cast(raw16, v));
    } else {
      for (int j = i; j < i + W && j < n - i0; ++j) po[j] = pq[j] > 0 ? pa[j] : (T)0.f;
    }
  }
}

unsigned grid_for(long long items, int per_block) {
  return (unsigned)std::min<long long>((items + per_block - 1) / per_block, 1 << 20);
}

// Widths that are whole blocks: every block is a row (no lane idles, whatever the width).
void blocks_as_rows(long long* rows, int* C) {
  if (*C % kQ8Block == 0) {
    *rows *= *C / kQ8Block;
    *C = kQ8Block;
  }
}
template <typename T> int launch_pack(const void* x, long long rows, int C, const Q8Ref& to, hipStream_t st) {
  blocks_as_rows(&rows, &C);
  return with_lanes<Row<T>::W>(C, [&](auto l) {
    constexpr int L = decltype(l)::L, NV = decltype(l)::NV;
    hipLaunchKernelGGL((k_q8_pack<T, L, NV, decltype(l)::E>), dim3(grid_for(rows, 256 / L)), dim3(256), 0, st, (const T*)x, to, rows, C,
                       (C + kQ8Block - 1) / kQ8Block);
    SPC_LAUNCH_CHECK();
    return (int)SPCONV_OK;
  });
}
template <typename T> int launch_unpack(const Q8Ref& from, long long rows, int C, void* out, hipStream_t st) {
  blocks_as_rows(&rows, &C);
  return with_lanes<Row<T>::W>(C, [&](auto l) {
    constexpr int L = decltype(l)::L, NV = decltype(l)::NV;
    hipLaunchKernelGGL((k_q8_unpack<T, L, NV, decltype(l)::E>), dim3(grid_for(rows, 256 / L)), dim3(256), 0, st, from, (T*)out, rows, C,
                       (C + kQ8Block - 1) / kQ8Block);
    SPC_LAUNCH_CHECK();
    return (int)SPCONV_OK;
  });
}
template <typename T> int launch_relu_bwd(const void* a, const signed char* q, int64_t n, void* out, hipStream_t st) {
  hipLaunchKernelGGL((k_relu_bwd_q8<T>), dim3(grid_for(n, 256 * Row<T>::W)), dim3(256), 0, st, (const T*)a, q, (T*)out, (long long)n);
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
