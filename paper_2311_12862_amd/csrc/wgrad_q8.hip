// Weight gradients of layers whose input was kept as an 8-bit checkpoint, 16-bit types: the pair-list kernel of wgrad.hip
// (same pieces, batches and order of sums, so the same bits as on the unpacked tensor) that gathers the checkpoint itself.
//
// A pair's row of x is C_in bytes and an exponent for every 32 of them instead of 2 C_in.  Rows go straight into LDS as they are;
// every lane then turns the 16 channels that it loaded itself into the layer's type, once per batch and workgroup (fragments are
// read by several waves: turning them there would cost four times the instructions), and writes them where the transposing
// reads expect them.  x therefore runs a batch ahead of dy.  (Where C_in ends inside a piece of 16, the rest of it is the next row's or, past
// the buffer, whose range is checked by the dword, zero: channels of dW that are not there to be stored.)
//
// Up to 128 channels a workgroup's waves go through a batch together and three workgroups share a CU (one converted batch, a barrier
// before it is replaced: with two of them and two workgroups 2.45M pairs 256 -> 64 took 310 us, so 239).  The 256 x 256 tile
// has the CU to itself, and matrix instructions, LDS and gathers each take more than half of its time: two halves of
// its waves take turns instead (all eight together 436 us, in turns 360, of which the gathers alone would take 282).
//
// bf16, 2.45M pairs of 300k rows, us for both kernels of a call, unpacking first and directly: 64 -> 64 100, 89; 96 -> 96 180, 162;
// 128 -> 128 218, 178; 256 -> 64 315, 239; 64 -> 256 (x is gathered for two column tiles) 290, 292; 256 -> 256 400, 360.
// 380k pairs of 100k rows: 64 -> 64 29.5, 22.9; 96 -> 96 41.1, 41.1; 128 -> 128 47.5, 44.4; 113k pairs 32 -> 32 14.7, 11.7.
#include "wgrad.h"
#include "rows.h"

#include <atomic>

namespace spc {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void load_byte_to_lds(u32x4 rsrc, unsigned voff, unsigned lds) {  // lane l: a dword at lds + 4 l
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_ubyte %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rsrc) : "memory");
}

// 16 channels of a checkpoint, of exponent b, as T: q * 2^(b - 133), rounded where T asks for it.
template <typename T> __device__ __forceinline__ void widen16(u32x4 q, unsigned b, u32x4 (&out)[2]);
template <> __device__ __forceinline__ void widen16<_Float16>(u32x4 q, unsigned b, u32x4 (&out)[2]) {
  // A byte q + 128 as the low bits of a half in [16, 32): 16 + (q + 128) / 64; less 18 that is q / 64.  Times 2^e, e = b - 127, in two
  // factors of about half of e each, as 2^e may be beyond a half where some products are not (q = 1 of b = 143 is 1024, q = 127 of
  // b = 102 rounds to 2^-24) and q = 0 has to stay 0.  The first product, with the 18 taken off in the same operation, is exact (multiples
  // of 2^-19 below 2^12), so only the second one rounds.  Below e = -26 every product is 0, above 22 all but that of q = 0 are infinite.
  const int e = min(max((int)b - 127, -26), 22), e1 = e >> 1, e2 = e - e1;
  const auto half2 = [](unsigned bits) { return __builtin_bit_cast(f16x2, bits * 0x10001u); };
  const f16x2 s1 = half2((unsigned)(e1 + 15) << 10), less = half2(0x8000u | (unsigned)(e1 + 19) << 10 | 0x80u);  // 2^e1, -18 * 2^e1
  const f16x2 s2 = half2(b == 255u ? 0x7E00u : (unsigned)(e2 + 15) << 10);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const unsigned u = q[w] ^ 0x80808080u;
    const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x4C4C4C4Cu, u, 0x04010400u));
    const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x4C4C4C4Cu, u, 0x04030402u));
    out[w / 2][w % 2 * 2] = __builtin_bit_cast(unsigned, __builtin_elementwise_fma(lo, s1, less) * s2);
    out[w / 2][w % 2 * 2 + 1] = __builtin_bit_cast(unsigned, __builtin_elementwise_fma(hi, s1, less) * s2);
  }
}
template <int I> __device__ __forceinline__ float byte_value(unsigned w) {  // (one instruction; spelled out it came as two)
  float f;
  if constexpr (I == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(w));
  if constexpr (I == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(w));
  if constexpr (I == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(w));
  if constexpr (I == 3) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(w));
  return f;
}
template <> __device__ __forceinline__ void widen16<__bf16>(u32x4 q, unsigned b, u32x4 (&out)[2]) {
  const float step = q8_step(b);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float v[4] = {byte_value<0>(q[w]) * step, byte_value<1>(q[w]) * step, byte_value<2>(q[w]) * step, byte_value<3>(q[w]) * step};
    unsigned f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __builtin_bit_cast(unsigned, v[i]);
    out[w / 2][w % 2 * 2] = __builtin_amdgcn_perm(f[1], f[0], 0x07060302u);  // (the upper halves: the lower ones are zero)
    out[w / 2][w % 2 * 2 + 1] = __builtin_amdgcn_perm(f[3], f[2], 0x07060302u);
  }
}

// TI x TO (channels of x, of dy) per workgroup; NWI x NWO waves share a batch, or (NWK > 1) each wave has its own.  S stages.
template <int TI, int TO, int NWI, int NWO, int NWK, int S> struct WgradQ8Shape {
  static constexpr int BP = 32;                                    // pairs of a batch
  static constexpr int NW = NWI * NWO;
  static constexpr int WI = TI / NWI, WO = TO / NWO, IB = WI / 16, OB = WO / 16;
  static constexpr int CPR = TI / 16;                              // 16-channel pieces of a row of x
  static constexpr int CH = (BP * CPR + NW * 64 - 1) / (NW * 64);  // pieces of a lane
  static constexpr int LD = BP * TO * 2 / 1024, LDW = (LD + NW - 1) / NW;  // loads of dy: of a batch, of a wave
  static constexpr int P = 2 * CH + LDW + 1;                       // loads of a wave in an iteration
  static constexpr int R = S <= 3 ? 8 : 16;                        // index ring: 2 S + 1 batches or more
  static constexpr bool kTurns = NW == 8;                          // halves of the waves multiply and load in turn
  static constexpr int NC = kTurns ? 3 : 1;                        // converted batches
  static constexpr int q_stage = NW * CH * 1024, b_stage = NW * CH * 256, d_stage = NW * LDW * 1024;
  static constexpr int x_bytes = BP * TI * 2;
  static constexpr int at_b = S * q_stage, at_d = at_b + S * b_stage, at_x = at_d + S * d_stage, at_idx = at_x + NC * x_bytes;
  static constexpr int group = at_idx + R * BP * 8;                // LDS of a wave group
  static constexpr int sums = NWK > 1 ? TI * TO * 4 : 0;
  static constexpr int total = NWK * (group > sums ? group : sums);
  static constexpr int threads = NW * NWK * 64;
  static_assert(NW == 1 || NWK == 1, "");
  static_assert(S >= 3 && 2 * S + 1 <= R && (S - 2) * P < 64 && total <= 160 * 1024, "");
};

template <typename T, int TI, int TO, int NWI, int NWO, int NWK, int S>
__global__ void __launch_bounds__(NWI* NWO* NWK * 64) k_wgrad_q8(const WgradParams p) {
  typedef WgradQ8Shape<TI, TO, NWI, NWO, NWK, S> W;
  constexpr int BP = W::BP, NW = W::NW, IB = W::IB, OB = W::OB, CH = W::CH, CPR = W::CPR, LDW = W::LDW, R = W::R, P = W::P;
  constexpr int CX = TI / 8, CD = TO / 8;
  constexpr bool kWhole = BP * CPR == NW * CH * 64;  // no lane's piece is beyond the batch
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = NWK > 1 ? wave_all : 0, wave = NWK > 1 ? 0 : wave_all;
  const int wi = wave / NWO, wo = wave % NWO;
  const int fa = lane & 15, fg = lane >> 4;
  const int ci0 = blockIdx.y * TI, co0 = blockIdx.z * TO;
  unsigned char* const my = smem + grp * W::group;
  const unsigned lds = (unsigned)(size_t)(__attribute__((address_space(3))) void*)my;

  const int bound = lane <= p.V ? p.seg[lane] : 0x7FFFFFFF;  // lane k: where offset k's pairs begin
  int k, begin, end;
  {
    const Pieces pc = pieces_of(p.split, bound, p.V, lane);
    k = __popcll(__ballot(lane < p.V && pc.before + pc.count <= (int)blockIdx.x));
    if (k >= p.V) return;
    const int q = (int)blockIdx.x - __builtin_amdgcn_readlane(pc.before, k);
    const int first = __builtin_amdgcn_readlane(bound, k), all = __builtin_amdgcn_readlane(bound, k + 1) - first;
    const int count = __builtin_amdgcn_readlane(pc.count, k), length = (all + count - 1) / count;
    begin = first + q * length;
    end = max(begin, min(first + all, begin + length));  // (may be empty: the tile is then zero)
  }

  const u32x4 x_rsrc = rsrc_of(p.feats, p.feats_bytes), b_rsrc = rsrc_of(p.exps, p.exps_bytes);
  const u32x4 d_rsrc = rsrc_of(p.dout, p.dout_bytes), p_rsrc = rsrc_of(p.pairs, p.pairs_bytes);
  const unsigned x_row = (unsigned)p.C_in, b_row = (unsigned)(p.C_in + kQ8Block - 1) / kQ8Block, d_row = (unsigned)p.C_out * 2u;

  // this lane's pieces of x (pair of the batch, channels) and loads of dy; kNoRow: none
  int x_pair[CH], d_pair[LDW];
  unsigned x_off[CH], b_off[CH], d_off[LDW];
  int x_to[CH];  // where the converted piece stands
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int id = (wave * CH + i) * 64 + lane, r = id / CPR, c = id % CPR, ch = ci0 + c * 16;
    x_pair[i] = r;
    x_off[i] = r < BP && ch < p.C_in ? (unsigned)ch : kNoRow;
    b_off[i] = (unsigned)ch / kQ8Block;
    x_to[i] = r < BP ? r * TI * 2 + place_of<2, CX>(c, r) * 32 : -1;
  }
#pragma unroll
  for (int i = 0; i < LDW; ++i) {
    const int j = wave * LDW + i, q = j * 64 + lane, r = q / CD, c = q % CD;
    const int ch = (block_at<2, CD>(c / 2, r & (BP - 1)) * 2 + c % 2) * 8 + co0;
    d_pair[i] = r;
    d_off[i] = r < BP && ch < p.C_out ? (unsigned)ch * 2u : kNoRow;
  }
  // fragment addresses
  unsigned xa[IB], da[OB];
  {
    const int r = 8 * fg + (fa >> 2), in = (fa & 3) * 8;
#pragma unroll
    for (int i = 0; i < IB; ++i) xa[i] = (unsigned)(r * TI * 2 + place_of<2, CX>(wi * IB + i, r) * 32 + in);
#pragma unroll
    for (int i = 0; i < OB; ++i) da[i] = (unsigned)(r * TO * 2 + place_of<2, CD>(wo * OB + i, r) * 32 + in);
  }
  auto frag = [&](const unsigned char* at, int pitch) -> u32x4 {  // (see k_wgrad)
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 4 * pitch));
    return __builtin_bit_cast(u32x4, s16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
  };

  const int first = begin & ~1;  // (index loads are 16 bytes: two pairs)
  const int batches = max(end - first + BP - 1, 0) / BP;
  const int mine = NWK > 1 ? (batches - grp + NWK - 1) / NWK : batches;  // batches grp, grp + NWK, ...
  auto batch_pair = [&](int b) { return first + (NWK > 1 ? b * NWK + grp : b) * BP; };
  auto load_idx = [&](int b) {  // pair indices of own batch b; every wave of a group loads the same bytes
    if (lane < BP / 2)
      load_to_lds(p_rsrc, (unsigned)(batch_pair(b) + lane * 2) * 8u, 0, lds + W::at_idx + (unsigned)(b % R) * (BP * 8));
  };
  unsigned x_src[CH], b_src[CH], d_src[LDW];
  unsigned x_rows[CH], d_rows[LDW];
  auto rows_x = [&](int b) {  // the rows of x of own batch b
    const unsigned char* ring = my + W::at_idx + (b % R) * (BP * 8);
#pragma unroll
    for (int i = 0; i < CH; ++i) x_rows[i] = *reinterpret_cast<const unsigned*>(ring + (x_pair[i] & (BP - 1)) * 8 + 4);
#pragma unroll
    for (int i = 0; i < CH; ++i) asm volatile("" : "+v"(x_rows[i]));  // (else every read becomes a branch of its own)
  };
  auto rows_d = [&](int b) {
    const unsigned char* ring = my + W::at_idx + (b % R) * (BP * 8);
#pragma unroll
    for (int i = 0; i < LDW; ++i) d_rows[i] = *reinterpret_cast<const unsigned*>(ring + (d_pair[i] & (BP - 1)) * 8);
#pragma unroll
    for (int i = 0; i < LDW; ++i) asm volatile("" : "+v"(d_rows[i]));
  };
  auto address_x = [&](int b) {  // where it gathers from
    const int e0 = batch_pair(b);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const bool live = (unsigned)(e0 + x_pair[i] - begin) < (unsigned)(end - begin) && x_off[i] != kNoRow;
      const unsigned x_at = x_rows[i] * x_row + x_off[i], b_at = x_rows[i] * b_row + b_off[i];
      x_src[i] = live ? x_at : kNoRow;
      b_src[i] = live ? b_at : kNoRow;
    }
  };
  auto address_d = [&](int b) {
    const int e0 = batch_pair(b);
#pragma unroll
    for (int i = 0; i < LDW; ++i) {
      const bool live = (unsigned)(e0 + d_pair[i] - begin) < (unsigned)(end - begin) && d_off[i] != kNoRow;
      const unsigned at = d_rows[i] * d_row + d_off[i];
      d_src[i] = live ? at : kNoRow;
    }
  };
  auto read_idx_x = [&](int b) {
    rows_x(b);
    address_x(b);
  };
  auto read_idx_d = [&](int b) {
    rows_d(b);
    address_d(b);
  };
  auto load_x = [&](int slot) {
#pragma unroll
    for (int i = 0; i < CH; ++i) load_to_lds(x_rsrc, x_src[i], 0, lds + slot * W::q_stage + (wave * CH + i) * 1024);
#pragma unroll
    for (int i = 0; i < CH; ++i) load_byte_to_lds(b_rsrc, b_src[i], lds + W::at_b + slot * W::b_stage + (wave * CH + i) * 256);
  };
  auto load_d = [&](int slot) {
#pragma unroll
    for (int i = 0; i < LDW; ++i) load_to_lds(d_rsrc, d_src[i], 0, lds + W::at_d + slot * W::d_stage + (wave * LDW + i) * 1024);
  };
  // a lane converts what it loaded itself: its own loads' wait is enough
  u32x4 q[CH];
  unsigned qb[CH];
  auto take = [&](int slot) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      q[i] = *reinterpret_cast<const u32x4*>(my + slot * W::q_stage + (wave * CH + i) * 1024 + lane * 16);
      qb[i] = *reinterpret_cast<const unsigned*>(my + W::at_b + slot * W::b_stage + (wave * CH + i) * 256 + lane * 4);
    }
  };
  u32x4 wide[CH][2];
  auto widen = [&]() {
#pragma unroll
    for (int i = 0; i < CH; ++i) widen16<T>(q[i], qb[i], wide[i]);
  };
  auto put = [&](int c) {
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (kWhole || x_to[i] >= 0) {
        u32x4* to = reinterpret_cast<u32x4*>(my + W::at_x + c * W::x_bytes + x_to[i]);
        to[0] = wide[i][0];
        to[1] = wide[i][1];
      }
  };
  auto convert = [&](int c) {
    widen();
    put(c);
  };
  auto sync = [&]() {
    if constexpr (NW > 1) asm volatile("s_barrier" ::: "memory");
  };

  f32x4 acc[OB][IB];
#pragma unroll
  for (int o = 0; o < OB; ++o)
#pragma unroll
    for (int i = 0; i < IB; ++i) acc[o][i] = f32x4{0.f, 0.f, 0.f, 0.f};

  if constexpr (W::kTurns) {
    // Two halves of the waves, one of each on every SIMD, take turns: while one multiplies batch b, the other reads its fragments of
    // b or b + 1 and issues loads.  Between its matrix instructions, which leave the vector unit idle, a wave converts its
    // share of batch b + 2 (three converted batches: the other half may still read b, and reads b + 1 next).  A memory turn issues
    // x of b + S + 1 and dy of b + S - 1 and ends when what the next one reads is there.
    const bool second = wave >= NW / 2;
#pragma unroll
    for (int b = 0; b <= 2 * S; ++b) load_idx(b);
    wait_loads<0>();
    sync();
#pragma unroll
    for (int b = 0; b < S; ++b) {
      read_idx_x(b);
      load_x(b);
      if (b >= 2) {
        read_idx_d(b - 2);
        load_d(b - 2);
      }
    }
    wait_loads<(S - 2) * (P - 1)>();
    take(0);
    convert(0);
    take(1);
    convert(1);
    read_idx_x(S);
    read_idx_d(S - 2);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    load_x(0);
    load_d(S - 2);
    read_idx_x(S + 1);
    read_idx_d(S - 1);
    wait_loads<(S - 2) * (P - 1)>();
    sync();
    if (second) sync();
    int slot = 0, conv = 0;  // of batch b in the rings of S, of three
    for (int b = 0; b < mine; ++b) {
      const int slot1 = slot + 1 >= S ? slot + 1 - S : slot + 1, slot2 = slot + 2 >= S ? slot + 2 - S : slot + 2;
      const unsigned char* xs = my + W::at_x + conv * W::x_bytes;
      const unsigned char* ds = my + W::at_d + slot * W::d_stage;
      u32x4 x[IB], d[OB];
#pragma unroll
      for (int o = 0; o < OB; ++o) d[o] = frag(ds + da[o], TO * 2);
#pragma unroll
      for (int i = 0; i < IB; ++i) x[i] = frag(xs + xa[i], TI * 2);
      take(slot2);
      load_x(slot1);                        // batch b + S + 1: batch b + 1 has been taken
      load_d(slot > 0 ? slot - 1 : S - 1);  // batch b + S - 1: everyone holds batch b - 1 in registers
      load_idx(b + 2 * S + 1);
      rows_x(b + S + 2);
      rows_d(b + S);
      // dy of batch b + 1 and x of b + 3 have landed (loads of a turn: x, dy, indices; the prologue's had no indices)
      if (b < S - 2) wait_loads<(S - 2) * (P - 1)>();
      else wait_loads<(S - 2) * P>();
      sync();
      __builtin_amdgcn_sched_barrier(0);
      address_x(b + S + 2);
      address_d(b + S);
      convert(conv == 0 ? 2 : conv - 1);  // batch b + 2
#pragma unroll
      for (int i = 0; i < IB; ++i)
#pragma unroll
        for (int o = 0; o < OB; ++o) acc[o][i] = mma<T>(d[o], x[i], acc[o][i]);
#pragma unroll
      for (int i = 0; i < IB * OB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction,
        __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);  // then vector instructions in its shadow
      }
      __builtin_amdgcn_sched_barrier(0);
      sync();
      slot = slot1;
      conv = conv == 2 ? 0 : conv + 1;
    }
    if (!second) sync();
  } else {
    // indices of batches 0 .. 2 S, stages of the first S (x: S + 1, the last one in the place of the converted first)
#pragma unroll
    for (int b = 0; b <= 2 * S; ++b) load_idx(b);
    wait_loads<0>();
    sync();
#pragma unroll
    for (int b = 0; b < S; ++b) {
      read_idx_x(b);
      read_idx_d(b);
      load_x(b);
      load_d(b);
    }
    wait_loads<(S - 2) * (P - 1)>();
    take(0);
    convert(0);
    read_idx_x(S);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    sync();
    load_x(0);
    u32x4 x[IB], d[OB];
#pragma unroll
    for (int o = 0; o < OB; ++o) d[o] = frag(my + W::at_d + da[o], TO * 2);
#pragma unroll
    for (int i = 0; i < IB; ++i) x[i] = frag(my + W::at_x + xa[i], TI * 2);
    take(1);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    sync();
    convert(0);
    read_idx_x(S + 1);
    read_idx_d(S);

    int slot = 0;  // of batch b in the rings of S
    for (int b = 0; b < mine; ++b) {
      // x of batch b + 2 and dy of batch b + 1 have landed (and the indices of b + S + 2); everyone holds batch b in registers and has
      // converted b + 1.  (Loads of a wave: first x, then dy, then indices in every iteration; the prologue's had no indices.)
      if (b < S - 2) wait_loads<(S - 2) * (P - 1)>();
      else wait_loads<(S - 2) * P>();
      sync();
      const int slot1 = slot + 1 >= S ? slot + 1 - S : slot + 1, slot2 = slot + 2 >= S ? slot + 2 - S : slot + 2;
      load_x(slot1);  // batch b + S + 1
      load_d(slot);   // batch b + S
      load_idx(b + 2 * S + 1);
      slot = slot1;
      const unsigned char* xs = my + W::at_x;
      const unsigned char* ds = my + W::at_d + slot1 * W::d_stage;
      u32x4 dn[OB];
#pragma unroll
      for (int o = 0; o < OB; ++o) dn[o] = frag(ds + da[o], TO * 2);
      take(slot2);
      read_idx_x(b + S + 2);
      read_idx_d(b + S + 1);
#pragma unroll
      for (int i = 0; i < IB; ++i) {
#pragma unroll
        for (int o = 0; o < OB; ++o) acc[o][i] = mma<T>(d[o], x[i], acc[o][i]);
        x[i] = frag(xs + xa[i], TI * 2);
      }
      widen();  // batch b + 2, before everyone waits
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) asm volatile("" : "+v"(wide[i][j]));
      if constexpr (NW > 1) {  // everyone has read batch b + 1 (one wave's accesses keep their order)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        sync();
      }
      put(0);
#pragma unroll
      for (int o = 0; o < OB; ++o) d[o] = dn[o];
    }
  }
  wait_loads<0>();  // (nothing may land in LDS that is used for something else next)

  // a lane holds channels co = 4 fg .. + 3 of row ci = fa of each block
  float* dst = p.partial + (long long)blockIdx.x * p.C_in * p.C_out;
  auto store = [&](int ci, int co, f32x4 v) {
    if (ci < p.C_in && co < p.C_out) *reinterpret_cast<f32x4*>(dst + (long long)ci * p.C_out + co) = v;
  };
  if constexpr (NWK > 1) {
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(smem);  // [group][block][lane]
#pragma unroll
    for (int o = 0; o < OB; ++o)
#pragma unroll
      for (int i = 0; i < IB; ++i) sums[(grp * OB * IB + o * IB + i) * 64 + lane] = acc[o][i];
    __syncthreads();
    constexpr int Q = OB * IB / NWK;  // blocks that each group adds up
    static_assert(NWK == 1 || OB * IB % NWK == 0, "");
#pragma unroll
    for (int u = 0; u < Q; ++u) {
      const int blk = grp * Q + u, o = blk / IB, i = blk % IB;
      f32x4 v = sums[blk * 64 + lane];
#pragma unroll
      for (int g = 1; g < NWK; ++g) v += sums[(g * OB * IB + blk) * 64 + lane];
      store(ci0 + i * 16 + fa, co0 + o * 16 + fg * 4, v);
    }
  } else {
#pragma unroll
    for (int o = 0; o < OB; ++o)
#pragma unroll
      for (int i = 0; i < IB; ++i)
        store(ci0 + wi * W::WI + i * 16 + fa, co0 + wo * W::WO + o * 16 + fg * 4, acc[o][i]);
  }
}

template <typename T, int TI, int TO, int NWI, int NWO, int NWK, int S>
int launch(const WgradParams& p, dim3 grid, hipStream_t st) {
  typedef WgradQ8Shape<TI, TO, NWI, NWO, NWK, S> W;
  auto kernel = k_wgrad_q8<T, TI, TO, NWI, NWO, NWK, S>;
  static std::atomic<bool> attr_set{false};  // (set twice by racing threads at worst: the calls are idempotent)
  if (!attr_set.load(std::memory_order_acquire)) {
    SPC_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, W::total));
    attr_set.store(true, std::memory_order_release);
  }
  hipLaunchKernelGGL(kernel, grid, dim3(W::threads), W::total, st, p);
  SPC_LAUNCH_CHECK();
  return SPCONV_OK;
}

}  // namespace

int wgrad_q8_launch(const WgradParams& p, int tile, spconv_dtype dtype, dim3 grid, hipStream_t st) {
#define SPC_WGRAD_Q8(TI, TO, NWI, NWO, NWK, S)                                           \
  if (tile == TI)                                                                        \
    return dtype == SPCONV_F16 ? launch<_Float16, TI, TO, NWI, NWO, NWK, S>(p, grid, st) \
                               : launch<__bf16, TI, TO, NWI, NWO, NWK, S>(p, grid, st);
  SPC_WGRAD_Q8(32, 32, 1, 1, 4, 4)
  SPC_WGRAD_Q8(64, 64, 1, 1, 4, 3)
  SPC_WGRAD_Q8(96, 96, 2, 2, 1, 3)
  SPC_WGRAD_Q8(128, 128, 2, 2, 1, 3)
  SPC_WGRAD_Q8(256, 256, 2, 4, 1, 4)
  return SPCONV_EINVAL;
}

}  // namespace spc
