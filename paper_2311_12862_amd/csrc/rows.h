// Device-side pieces shared by the kernels that work on rows of channels (norm.hip, checkpoint.hip): groups of lanes that
// share a row, vectors of a row, and the format of 8-bit checkpoints.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

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
template <int L, int O = 1> __device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (O >= L) return v;
  else return lanes_sum<L, O * 2>(v + __builtin_bit_cast(float, lane_across<O>(__builtin_bit_cast(unsigned, v))));
}
// The same for up to 256 lanes: beyond a wave through `part`, after a barrier that the whole workgroup reaches.  Two slots, used in
// turn: whoever writes a slot again has passed the other one's barrier, which everyone reaches after reading this one.
template <int L> __device__ __forceinline__ float group_sum(float v, float (*part)[4], int slot) {
  if constexpr (L <= 64) {
    return lanes_sum<L>(v);
  } else {
    v = lanes_sum<64>(v);
    if (threadIdx.x % 64 == 0) part[slot][threadIdx.x / 64] = v;
    __syncthreads();
    const int first = threadIdx.x / L * (L / 64);
    v = part[slot][first];
#pragma unroll
    for (int w = 1; w < L / 64; ++w) v += part[slot][first + w];
    return v;
  }
}
// Two sums at once, through two slots of their own and one barrier.
template <int L> __device__ __forceinline__ void group_sums(float& a, float& b, float (*part)[4]) {
  a = lanes_sum<(L < 64 ? L : 64)>(a);
  b = lanes_sum<(L < 64 ? L : 64)>(b);
  if constexpr (L > 64) {
    if (threadIdx.x % 64 == 0) {
      part[0][threadIdx.x / 64] = a;
      part[1][threadIdx.x / 64] = b;
    }
    __syncthreads();
    const int first = threadIdx.x / L * (L / 64);
    a = part[0][first];
    b = part[1][first];
#pragma unroll
    for (int w = 1; w < L / 64; ++w) {
      a += part[0][first + w];
      b += part[1][first + w];
    }
  }
}
template <int L, int O = 1> __device__ __forceinline__ unsigned group_max(unsigned v) {
  if constexpr (O >= L) return v;
  else return group_max<L, O * 2>(max(v, lane_across<O>(v)));
}

// ---- vectors of a row: W consecutive elements that make 16 bytes, held as they are in memory.  Rows of odd widths start anywhere: the
// hardware takes 16-byte accesses at any address, so one path serves every width.
typedef unsigned int raw16 __attribute__((ext_vector_type(4)));
typedef unsigned int raw8 __attribute__((ext_vector_type(2)));
typedef float float4x __attribute__((ext_vector_type(4)));
template <typename V> struct __attribute__((packed)) AnyAddress { V v; };
template <typename V> __device__ __forceinline__ V load_any(const void* p) { return reinterpret_cast<const AnyAddress<V>*>(p)->v; }
template <typename V> __device__ __forceinline__ void store_any(void* p, V v) { reinterpret_cast<AnyAddress<V>*>(p)->v = v; }

// The last n bytes of N words whose first stands at p, 1 to 4 N - S of them, a multiple of S: the last eight if n has that bit, in
// front of them four, two and one.  Every piece is the end of one of the words, so nothing is shifted by a lane's own number.  (One
// element after the other, with a mask of lanes for each: 1.7M rows of 45 fp16 forward 139 us, so 106 to 111, gradients 160, so 120.)
template <int S, typename V> __device__ __forceinline__ void store_end(char* p, int n, V w) {
  constexpr int N = sizeof(V) / 4;
  asm volatile("" : "+v"(n));  // (conditions and addresses that hold for every row would be kept in registers all along)
  if constexpr (N == 4)
    if (n & 8) store_any(p + 8, raw8{w[2], w[3]});
  if constexpr (N > 1)
    if (n & 4) store_any(p + (4 * N - (n & ~3)), N == 4 && (n & 8) ? w[1] : w[N - 1]);
  if constexpr (S < 4) {
    unsigned front = w[N - 1];  // the word that the rest ends
#pragma unroll
    for (int j = 1; j < N; ++j) front = n >> 2 == j ? w[N - 1 - j] : front;
    if (n & 2) store_any(p + (4 * N - (n & ~1)), (unsigned short)(front >> 16));
    if constexpr (S == 1)
      if (n & 1) p[4 * N - n] = (char)(n & 2 ? front >> 8 : front >> 24);
  }
}

// How a kernel takes the end of a row: widths that are multiples of W, others, and less than W.
enum Ends { kWholeVectors = 0, kOddWidth = 1, kBelowVector = 2 };

// Where a lane's vector of a row of C channels stands.  The vector that ends a row whose width is no multiple of W reaches back over
// its neighbour's channels (loaded with one access, like any other): its first `lo` elements are not its own and count as zero.
// In rows of fewer than W channels `col` is negative and elements are taken one by one (kernels of their own: the addresses of single
// elements cost the others 64 registers, 170k rows of 450 fp16 179 us for their gradients).
struct Place {
  int col;    // channel of element 0
  int lo;     // own elements are [lo, W)
  int block;  // of 32 channels, that the own elements lie in
  bool live;  // there are any
};
template <int W> __device__ __forceinline__ Place place_in_row(int vector, int C) {
  const int first = vector * W, n = C - first;
  return {n >= W ? first : C - W, n >= W ? 0 : W - n, first / 32, n > 0};
}

// Element i behind a base that all lanes of a wave share: 32 bits a lane.  (In rows of fewer than W channels a vector starts in front of
// its row, i may be negative.)
template <Ends E, typename T> __device__ __forceinline__ T* behind(T* base, int i) {
  typedef std::conditional_t<std::is_const_v<T>, const char, char> byte;
  if constexpr (E == kBelowVector) return base + i;
  else return (T*)((byte*)base + (unsigned)(i * (int)sizeof(T)));
}
// Keeps the compiler from computing what follows from v for all rows at once and holding it: addresses of 64 bits for every tensor.
__device__ __forceinline__ void each_row(int& v) { asm volatile("" : "+v"(v)); }

template <typename T> struct Row {
  static constexpr int W = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(W)));

  // p: element 0 of the vector
  template <Ends E> static __device__ __forceinline__ raw16 load(const T* p, const Place& at) {
    if constexpr (E != kBelowVector) return load_any<raw16>(p);
    vec x;
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = p[max(i, at.lo)];
    return __builtin_bit_cast(raw16, x);
  }
  template <Ends E> static __device__ __forceinline__ void store(T* p, const Place& at, raw16 r) {
    if (E == kWholeVectors || at.lo == 0) store_any(p, r);
    else store_end<sizeof(T)>((char*)p, (W - at.lo) * (int)sizeof(T), r);
  }
  static __device__ __forceinline__ void widen(raw16 r, float (&v)[W]) {
    const vec x = __builtin_bit_cast(vec, r);
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = (float)x[i];
  }
  static __device__ __forceinline__ raw16 narrow(const float (&v)[W]) {  // to nearest even
    vec x;
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = (T)v[i];
    return __builtin_bit_cast(raw16, x);
  }
};
// what stands in front of a vector's own elements becomes zero
template <Ends E, int W> __device__ __forceinline__ void own_only(const Place& at, float (&v)[W]) {
  if constexpr (E != kWholeVectors) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = i >= at.lo ? v[i] : 0.f;
  }
}
template <Ends E, int W> __device__ __forceinline__ void load_floats(const float* p, const Place& at, float (&v)[W]) {
  if constexpr (E != kBelowVector) {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const float4x r = load_any<float4x>(p + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i + j] = r[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = p[max(i, at.lo)];
  }
}

// ---- 8-bit checkpoints.  A row is cut into blocks of 32 channels.  b: biased fp32 exponent of the block's largest magnitude, at
// least 1, or 255 where the block has an infinity or a NaN; a channel is q * 2^(b - 133).
// q has 7 bits and a sign, the step is a power of two: the value is exact in fp32, in bf16 and in the tensor's own type (the step of an fp16
// block is below fp16's smallest number only where every product is a multiple of that number).  Read as fp16, a checkpoint of an fp32
// or bf16 tensor may have values that fp16 rounds or has no number for.
constexpr int kQ8Block = 32;

struct Q8Ref {  // a checkpoint: [rows][C] and [rows][ceil(C / 32)]
  signed char* q;
  unsigned char* b;
};

// 2^(b - 133) (subnormal for the smallest b); a NaN for b = 255
__device__ __forceinline__ float q8_step(unsigned b) {
  const float s = ldexpf(1.f, (int)b - 133);
  return b == 255u ? __builtin_nanf("") : s;
}
template <int W> struct Bytes;  // the q of a vector
template <> struct Bytes<8> { typedef raw8 word; };
template <> struct Bytes<4> { typedef unsigned word __attribute__((ext_vector_type(1))); };

template <Ends E, int W>
__device__ __forceinline__ typename Bytes<W>::word q8_load(const signed char* p, const Place& at) {
  typedef typename Bytes<W>::word word;
  if constexpr (E != kBelowVector) return load_any<word>(p);
  word w = {};
#pragma unroll
  for (int i = 0; i < W; ++i) w[i / 4] |= (unsigned)(unsigned char)p[max(i, at.lo)] << (8 * (i % 4));
  return w;
}
template <Ends E, int W> __device__ __forceinline__ void q8_store(signed char* p, const Place& at, typename Bytes<W>::word w) {
  if (E == kWholeVectors || at.lo == 0) store_any(p, w);
  else store_end<1>((char*)p, W - at.lo, w);
}
template <int W> __device__ __forceinline__ int q8_at(typename Bytes<W>::word w, int i) { return (signed char)(w[i / 4] >> (8 * (i % 4))); }
template <int W> __device__ __forceinline__ void q8_widen(typename Bytes<W>::word w, float step, float (&v)[W]) {
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = (float)q8_at<W>(w, i) * step;
}

// The checkpoint of a vector, one of the G that make a block (aligned groups of G lanes; every lane of the group takes part, with zeros
// where it has no elements).  What bounds a kernel that keeps two checkpoints is the vector unit as soon as an element takes more
// than about 50 instructions; this takes 6.  Rounding is that of an addition: 1.5 * 2^23 + r has r to nearest even in its
// low bits.
template <int G, int W> __device__ __forceinline__ typename Bytes<W>::word q8_quantise(const float (&v)[W], unsigned& b) {
  float most = __builtin_fabsf(v[0]);
#pragma unroll
  for (int i = 1; i < W; ++i) most = __builtin_elementwise_maximum(most, __builtin_fabsf(v[i]));  // (a NaN stays one)
  unsigned top = __builtin_bit_cast(unsigned, most) & 0x7FFFFFFFu;
  top = group_max<G>(top);
  b = max(top >> 23, 1u);
  // 2^(133 - b) is a number from b = 6 on; below (magnitudes under 2^-121) v_ldexp scales.  Products are exact, except for values so
  // far below the block's largest that they are kept for their sign alone.
  const float inv = __builtin_bit_cast(float, (260u - max(b, 6u)) << 23);
  float t[W];
#pragma unroll
  for (int i = 0; i < W; ++i) t[i] = v[i] * inv;
  if (__builtin_expect(__any(b < 6u && top != 0u), 0)) {
#pragma unroll
    for (int i = 0; i < W; ++i) t[i] = b < 6u ? ldexpf(v[i], 133 - (int)b) : t[i];
  }
  unsigned s[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    // (at most 127: 128 would be the rounding of values from 127.5 on; at least 1 where the value is not 0, whatever its size)
    const float least = __builtin_amdgcn_fmed3f(ldexpf(__builtin_fabsf(v[i]), 150), 0.f, 1.f);
    const float r = __builtin_copysignf(__builtin_amdgcn_fmed3f(__builtin_fabsf(t[i]), least, 127.f), v[i]);
    s[i] = __builtin_bit_cast(unsigned, r + 12582912.f);
  }
  typename Bytes<W>::word w;
#pragma unroll
  for (int j = 0; j < W / 4; ++j) {
    const unsigned lo = __builtin_amdgcn_perm(s[4 * j + 1], s[4 * j], 0x0C0C0400u), hi = __builtin_amdgcn_perm(s[4 * j + 3], s[4 * j + 2], 0x04000C0Cu);
    w[j] = b < 255u ? lo | hi : 0u;
  }
  return w;
}

// A group of L lanes (32 / W of them, or all, make a block) writes a vector each, its element 0 at q, its block at b.
template <Ends E, int L, int W>
__device__ __forceinline__ void q8_keep(signed char* q, unsigned char* b, const Place& at, bool live, const float (&v)[W]) {
  constexpr int G = L < kQ8Block / W ? L : kQ8Block / W;
  unsigned exponent;
  const auto w = q8_quantise<G, W>(v, exponent);
  if (live) {
    q8_store<E, W>(q, at, w);
    if (threadIdx.x % G == 0) *b = (unsigned char)exponent;
  }
}

// Workgroups of a kernel that the GPU holds at once: a kernel that loops over rows is launched with no more, or the ones that wait run as
// a second round after the others (fp16 forward with seven a CU, launched with eight: 300k x 256 88 us, with seven 64).  At most six a
// CU: the count leaves out scalar registers, and six is what is held of kernels that take all of them.  `held` caches the answer, one for
// each kernel.
template <typename K> int resident_groups(K kernel, std::atomic<int>& held) {
  int n = held.load(std::memory_order_relaxed);
  if (n == 0) {
    int per_cu = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kernel, 256, 0) != hipSuccess || per_cu < 1) {
      (void)hipGetLastError();
      per_cu = 4;
    }
    n = 256 * std::min(per_cu, 6);
    held.store(n, std::memory_order_relaxed);
  }
  return n;
}

// Lanes of a row and vectors of a lane: as few lanes as hold the row with one vector each, up to a workgroup's 256, then more
// vectors (all of a row's lanes in one wave, with 8 vectors or more each, did not fit the registers).  Rows of more than 64 vectors take the
// kernels of odd widths whether they are odd or not, and lanes idle where the number is far below 128, 256 or 512 (forward: 40k x 1024
// bf16 5.4 TB/s, 70k x 600 f16, 75 vectors on 128 lanes, 3.5).  C is 1 to 4096.  Calls go with them as constants.
template <int LANES, int VECTORS, Ends ENDS> struct Lanes {
  static constexpr int L = LANES, NV = VECTORS;
  static constexpr Ends E = ENDS;
};
template <int W, typename F> int with_lanes(int C, F go) {
  const int n = (C + W - 1) / W;
  if (C < W) return go(Lanes<4, 1, kBelowVector>{});
  if (C % W == 0) {
    if (n <= 4) return go(Lanes<4, 1, kWholeVectors>{});
    if (n <= 8) return go(Lanes<8, 1, kWholeVectors>{});
    if (n <= 16) return go(Lanes<16, 1, kWholeVectors>{});
    if (n <= 32) return go(Lanes<32, 1, kWholeVectors>{});
    if (n <= 64) return go(Lanes<64, 1, kWholeVectors>{});
  }
  if (n <= 4) return go(Lanes<4, 1, kOddWidth>{});
  if (n <= 8) return go(Lanes<8, 1, kOddWidth>{});
  if (n <= 16) return go(Lanes<16, 1, kOddWidth>{});
  if (n <= 32) return go(Lanes<32, 1, kOddWidth>{});
  if (n <= 64) return go(Lanes<64, 1, kOddWidth>{});
  if (n <= 128) return go(Lanes<128, 1, kOddWidth>{});
  if (n <= 256) return go(Lanes<256, 1, kOddWidth>{});
  if (n <= 512) return go(Lanes<256, 2, kOddWidth>{});
  if constexpr (W == 4) return go(Lanes<256, 4, kOddWidth>{});
  return SPCONV_EINVAL;
}

}  // namespace
}  // namespace spc
