// Device-side pieces shared by the kernels that work on rows of channels (norm.hip, checkpoint.hip): groups of lanes that
// share a row, vectors of a row, and the format of 8-bit checkpoints.
#pragma once
#include <hip/hip_runtime.h>

namespace spc {
namespace {

// ---- sums and maxima over aligned groups of L lanes; every lane of the group gets the result.  Lanes 1, 2, 4 and 8 apart
// (mirrored, once the halves agree) meet in the vector unit, 16 and 32 apart through the LDS crossbar.
template <int CTRL> __device__ __forceinline__ unsigned dpp(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int O> __device__ __forceinline__ unsigned lane_across(unsigned v) {  // from the other half of 2 O lanes
  if constexpr (O == 1) return dpp<0xB1>(v);        // quad_perm [1,0,3,2]
  else if constexpr (O == 2) return dpp<0x4E>(v);   // quad_perm [2,3,0,1]
  else if constexpr (O == 4) return dpp<0x141>(v);  // row_half_mirror
  else if constexpr (O == 8) return dpp<0x140>(v);  // row_mirror
  else return (unsigned)__shfl_xor((int)v, O);
}
template <int L, int O = 1> __device__ __forceinline__ float group_sum(float v) {
  if constexpr (O >= L) return v;
  else return group_sum<L, O * 2>(v + __builtin_bit_cast(float, lane_across<O>(__builtin_bit_cast(unsigned, v))));
}
template <int L, int O = 1> __device__ __forceinline__ unsigned group_max(unsigned v) {
  if constexpr (O >= L) return v;
  else return group_max<L, O * 2>(max(v, lane_across<O>(v)));
}

// ---- W consecutive elements of a row, as fp32.  W elements of T make 16 bytes and stand at a multiple of them, or W is 1.
template <typename T, int W> struct Chunk {
  typedef T vec __attribute__((ext_vector_type(W), aligned(16)));
  static __device__ __forceinline__ void load(const void* base, long long at, float (&v)[W]) {
    const vec x = *reinterpret_cast<const vec*>(reinterpret_cast<const T*>(base) + at);
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = (float)x[i];
  }
  // rounds to nearest even; v then holds what was written
  static __device__ __forceinline__ void store(void* base, long long at, float (&v)[W]) {
    vec x;
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = (T)v[i];
    *reinterpret_cast<vec*>(reinterpret_cast<T*>(base) + at) = x;
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = (float)x[i];
  }
};
template <typename T> struct Chunk<T, 1> {
  static __device__ __forceinline__ void load(const void* base, long long at, float (&v)[1]) {
    v[0] = (float)reinterpret_cast<const T*>(base)[at];
  }
  static __device__ __forceinline__ void store(void* base, long long at, float (&v)[1]) {
    const T x = (T)v[0];
    reinterpret_cast<T*>(base)[at] = x;
    v[0] = (float)x;
  }
};

// ---- 8-bit checkpoints.  A row is cut into blocks of 32 channels.  b: biased fp32 exponent of the block's largest magnitude, at
// least 1, or 255 where the block has an infinity or a NaN; a channel is q * 2^(b - 133).
// q has 8 bits and a sign, the step is a power of two: the value is exact in fp16, bf16 and fp32 alike (the step of an fp16
// block is below fp16's smallest number only where every product is a multiple of that number), so a kernel that reads a
// checkpoint sees what it would see in the unpacked tensor.
constexpr int kQ8Block = 32;

__device__ __forceinline__ unsigned q8_exponent(unsigned top) { return max(top >> 23, 1u); }  // top: bits of the largest |x|
__device__ __forceinline__ int q8_quantise(float x, unsigned b) {
  if (b >= 255u) return 0;
  // v_ldexp: exact (2^(133 - b) itself can exceed fp32).  |x| < 2^(b - 126), so the product is below 128 and rounds to at
  // most that; the clamp costs those 128 one step at most.
  const float s = ldexpf(x, 133 - (int)b);
  int q = (int)rintf(s);
  q = min(max(q, -127), 127);
  return q == 0 ? (x > 0.f) - (x < 0.f) : q;  // keeps the sign: a ReLU's gradient asks for it
}
// 2^(b - 127); infinite for b = 255, which turns q = 0 into a NaN
__device__ __forceinline__ float q8_scale(unsigned b) { return __builtin_bit_cast(float, b << 23); }
__device__ __forceinline__ float q8_value(int q, float scale) { return (float)q * 0.015625f * scale; }

template <int W> struct Bytes;
template <> struct Bytes<8> { typedef unsigned word __attribute__((ext_vector_type(2))); };
template <> struct Bytes<4> { typedef unsigned word __attribute__((ext_vector_type(1))); };

// W consecutive q of a row (a multiple of W bytes in, or W is 1)
template <int W> __device__ __forceinline__ void q8_load(const signed char* base, long long at, int (&q)[W]) {
  if constexpr (W == 1) {
    q[0] = base[at];
  } else {
    const auto w = *reinterpret_cast<const typename Bytes<W>::word*>(base + at);
#pragma unroll
    for (int i = 0; i < W; ++i) q[i] = (int)(w[i / 4] << (24 - 8 * (i % 4))) >> 24;
  }
}
template <int W> __device__ __forceinline__ void q8_store(signed char* base, long long at, const int (&q)[W]) {
  if constexpr (W == 1) {
    base[at] = (signed char)q[0];
  } else {
    typename Bytes<W>::word w;
#pragma unroll
    for (int j = 0; j < W / 4; ++j)
      w[j] = (unsigned)(q[4 * j] & 255) | (unsigned)(q[4 * j + 1] & 255) << 8 | (unsigned)(q[4 * j + 2] & 255) << 16 |
             (unsigned)q[4 * j + 3] << 24;
    *reinterpret_cast<typename Bytes<W>::word*>(base + at) = w;
  }
}

struct Q8Ref {  // a checkpoint: [rows][C] and [rows][ceil(C / 32)]
  signed char* q;
  unsigned char* b;
};

// A group of L lanes (32 / W of them, or all, make a block) writes W channels each of row r: v of columns col.., live: col < C.
// Every lane of the wave takes part.
template <int L, int W>
__device__ __forceinline__ void q8_keep(const Q8Ref& to, long long r, int C, int nb, int col, bool live, const float (&v)[W]) {
  constexpr int G = L < kQ8Block / W ? L : kQ8Block / W;
  unsigned top = 0;
  if (live) {
#pragma unroll
    for (int i = 0; i < W; ++i) top = max(top, __builtin_bit_cast(unsigned, v[i]) & 0x7FFFFFFFu);
  }
  const unsigned b = q8_exponent(group_max<G>(top));
  if (live) {
    int q[W];
#pragma unroll
    for (int i = 0; i < W; ++i) q[i] = q8_quantise(v[i], b);
    q8_store<W>(to.q, r * C + col, q);
    if (col % kQ8Block == 0) to.b[r * nb + col / kQ8Block] = (unsigned char)b;
  }
}

}  // namespace
}  // namespace spc
