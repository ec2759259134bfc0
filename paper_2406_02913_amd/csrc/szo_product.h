// Products of 16-bit matrices in tiles of BI x BJ for a workgroup of eight waves, C[i][j] = sum over r of A(i, r) B(j, r), sums in fp32 registers.
//
// Either operand lies in memory with r contiguous ("rows": a row of A is an i) or with i (j) contiguous ("columns": a row is an r).  A step takes 64 of r.  Its
// operands go from memory to LDS without passing through registers, 16 bytes a lane and 1 KiB an instruction, two or more steps' worth held; lanes choose what they
// read, since a load puts them side by side in LDS:
//   rows     [row][64 of r]: the eight 16-byte pieces of a row are exchanged by (row / 2) mod 8, so that 16 lanes that read one piece of 16 rows touch every bank once
//   columns  [r][256 of i], two r to an instruction: 16-wide groups are exchanged in pairs in odd r, pairs of r lie 64 bytes and eights of them 128 further than they are
//            long, so that the four 32-byte pieces each of two groups of 16 lanes, which the transposing LDS read asks for together, lie in different banks
//   columns  [r][128 of i], four r to an instruction: 16-wide groups are exchanged by r mod 4 and (r / 8) mod 2, to the same end; a read forms its address
// Fragments are read from LDS a few groups of products before they are used, across the one barrier of a step.
//   256 x 256: a step takes 1.33 us, 1.28 to 1.41 PFLOP/s with the whole chip at work (4096 x 32000 x 4096; the card's own large product 1.45 there, 1.59 at 16384 cubed), bound by the matrix
// cores and, a fifth, by what stands at a step's barrier: a CU holds one workgroup, whose sums take half of its registers.  Four waves with twice the sums each, which read
// a third less from LDS: 801 -> 1119, and 300 rows in tiles of 128 x 320 90 -> 118; a wave alone on its SIMD issues too slowly.
#pragma once
#include "szo_internal.h"
#include "szo_types.h"

namespace szo {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) uint8_t* lds_at;
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));

template <int TYPE> struct Product;
template <> struct Product<SZO_BF16> {
  typedef bf16x8 vec;
  static __device__ __forceinline__ f32x4 add(vec a, vec b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Product<SZO_F16> {
  typedef f16x8 vec;
  static __device__ __forceinline__ f32x4 add(vec a, vec b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

constexpr int kStep = 64;                  // of r
constexpr int kPairBytes = 1024 + 64;      // columns: two r of 256, and what pairs are apart

// An operand as it lies in memory: `stride` elements from row to row.  rows: r runs from 0 to `length`, `count` rows from `base` on.  columns: `length` rows from `base`
// on, of which `count` elements are there (256 are read: what is behind them reaches only sums that nobody stores).
struct Operand {
  const uint16_t* base;
  int64_t stride;
  int64_t count, length;
};

template <bool COLUMNS, int SIZE> constexpr int stage_bytes() { return COLUMNS && SIZE == 256 ? 32 * kPairBytes + 8 * 128 : SIZE * kStep * 2; }

// One operand of a workgroup's tile: its loads to LDS and its reads from there.
template <bool COLUMNS, int SIZE, int PER>           // PER: 16-wide groups of a wave
struct Side {
  static constexpr int kLoads = SIZE / 64;           // of a wave and step
  static constexpr int kStage = stage_bytes<COLUMNS, SIZE>();
  static_assert(!COLUMNS || SIZE == 256 || SIZE == 128, "columns are laid out for these");
  uint32_t from, apart;                              // bytes from the step's first row or column to this lane's first 16, and from one load to the next
  uint32_t lds;                                      // where this wave's loads go, in a stage
  lds_at read[2];                                    // rows: of the two halves of a step; columns: of even and odd groups
  uint64_t base;
  uint32_t pitch;                                    // bytes of a row
  int left;                                          // bytes (rows) or rows (columns) behind `base`
  uint32_t row_bytes;                                // columns: of a row, those that are there

  // `wave_first`: first of this wave's SIZE values
  __device__ __forceinline__ Side(const Operand& o, lds_at stages, int wave, int wave_first, int lane) {
    pitch = (uint32_t)(o.stride * 2);
    base = (uint64_t)(uintptr_t)o.base;
    row_bytes = (uint32_t)(o.count * 2);
    if constexpr (COLUMNS && SIZE == 128) {
      left = (int)o.length;
      const uint32_t q = (uint32_t)lane >> 4, exchange = q | ((uint32_t)wave & 1u) << 2;       // rows 8 w + q and, of the second load, + 4
      from = (8u * (uint32_t)wave + q) * pitch + 16u * (((uint32_t)lane & 15u) ^ exchange << 1);
      apart = 4 * pitch;
      lds = (uint32_t)(uintptr_t)stages + (uint32_t)wave * 2048u;
      const int g = lane >> 4, p = lane & 15, row = 8 * g + (p >> 2);
      read[0] = read[1] = stages + (row * 256 + (p & 3) * 8 + ((((p >> 2) | (g & 1) << 2) << 5) ^ wave_first * 2));       // the group's bits are xored in
    } else if constexpr (COLUMNS) {
      left = (int)o.length;
      const uint32_t r = (uint32_t)lane >> 5, piece = ((uint32_t)lane & 31u) ^ (2u * r);
      from = (uint32_t)(2 * wave * kLoads + (int)r) * pitch + 16u * piece;
      apart = 2 * pitch;
      lds = (uint32_t)(uintptr_t)stages + (uint32_t)(wave * kLoads) * kPairBytes + (uint32_t)wave * 128u;       // kLoads is 4: pairs 4 w .. + 3
      // lane p of sixteen: 8 bytes of row 8 g + p / 4; the row's pair is 4 g + p / 8
      const int g = lane >> 4, p = lane & 15, odd = p >> 2 & 1;
      const lds_at at = stages + (4 * g + (p >> 3)) * kPairBytes + g * 128 + odd * 512 + (p & 3) * 8 + wave_first * 2;
      read[0] = at + odd * 32;
      read[1] = at - odd * 32;
    } else {
      left = (int)(((o.count - 1) * o.stride + o.length) * 2);
      // rows of an instruction: eight, the same eight of sixteen for all of a wave's
      const uint32_t first = (uint32_t)((wave >> 1) * kLoads * 16 + (wave & 1) * 8), row = first + ((uint32_t)lane >> 3);
      from = row * pitch + 16u * (((uint32_t)lane & 7u) ^ (row >> 1 & 7u));
      apart = 16 * pitch;
      lds = (uint32_t)(uintptr_t)stages + first * 128u;
      const int at = wave_first + (lane & 15), swizzle = (lane & 15) >> 1;
      read[0] = stages + at * 128 + (((lane >> 4) ^ swizzle) << 4);
      read[1] = stages + at * 128 + ((((lane >> 4) + 4) ^ swizzle) << 4);
    }
  }

  static constexpr uint32_t kApart = !COLUMNS ? 2048 : SIZE == 256 ? kPairBytes : 1024;            // in LDS, of one load and the next
  template <int N>
  __device__ __forceinline__ void issue(uint32_t to, uint32_t from, rsrc_t rsrc) const {
    uint32_t at;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    // m0 is no register that values are allocated to, which the compiler warns of; named all the same.  Wait states: a vector instruction may have written the
    // descriptor just before.
    if constexpr (N == 4) {
      asm volatile("s_mov_b32 m0, %1\n\tv_add_u32 %0, %2, %3\n\ts_nop 4\n\t"
                   "buffer_load_dwordx4 %3, %4, 0 offen lds\n\ts_add_u32 m0, m0, %5\n\ts_nop 0\n\t"
                   "buffer_load_dwordx4 %0, %4, 0 offen lds\n\ts_add_u32 m0, m0, %5\n\tv_add_u32 %0, %2, %0\n\ts_nop 0\n\t"
                   "buffer_load_dwordx4 %0, %4, 0 offen lds\n\ts_add_u32 m0, m0, %5\n\tv_add_u32 %0, %2, %0\n\ts_nop 0\n\t"
                   "buffer_load_dwordx4 %0, %4, 0 offen lds"
                   : "=&v"(at) : "s"(to), "s"(apart), "v"(from), "s"(rsrc), "i"(kApart) : "memory", "scc", "m0");
    } else if constexpr (N == 2) {
      asm volatile("s_mov_b32 m0, %1\n\tv_add_u32 %0, %2, %3\n\ts_nop 4\n\t"
                   "buffer_load_dwordx4 %3, %4, 0 offen lds\n\ts_add_u32 m0, m0, %5\n\ts_nop 0\n\t"
                   "buffer_load_dwordx4 %0, %4, 0 offen lds"
                   : "=&v"(at) : "s"(to), "s"(apart), "v"(from), "s"(rsrc), "i"(kApart) : "memory", "scc", "m0");
    } else {
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(to), "v"(from), "s"(rsrc) : "memory", "scc", "m0");
    }
#pragma clang diagnostic pop
  }

  // Loads of the next step, which is there; addresses out of bounds read as zero.  In assembly: behind the compiler's own form it waits for all of them at every LDS
  // read, and kept apart the loads' addresses would take registers that the main loop has not got.
  __device__ __forceinline__ void load(int stage) {
    const uint32_t bytes = COLUMNS ? (uint32_t)min(left - 1, kStep - 1) * pitch + row_bytes : (uint32_t)left;
    const rsrc_t rsrc = {(uint32_t)base, (uint32_t)(base >> 32), bytes, 0x00027000u};
    const uint32_t to = lds + (uint32_t)(stage * kStage);
    constexpr int kFours = kLoads / 4;
#pragma unroll
    for (int i = 0; i < kFours; ++i) issue<4>(to + i * 4 * kApart, from + (uint32_t)i * 4 * apart, rsrc);
    if constexpr (kLoads % 4 >= 2) issue<2>(to + kFours * 4 * kApart, from + (uint32_t)kFours * 4 * apart, rsrc);
    if constexpr (kLoads % 2) issue<1>(to + (kLoads - 1) * kApart, from + (uint32_t)(kLoads - 1) * apart, rsrc);
    base += COLUMNS ? (uint64_t)pitch * kStep : (uint64_t)(kStep * 2);
    left -= COLUMNS ? kStep : kStep * 2;
  }

  // Group t of 16, half h of a step: a lane's eight of r.
  template <int TYPE>
  __device__ __forceinline__ typename Product<TYPE>::vec fragment(int stage, int half, int t) const {
    typedef typename Product<TYPE>::vec vec;
    typedef __attribute__((address_space(3))) const vec* vec_at;
    if constexpr (COLUMNS) {
      typedef short short4_t __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) short4_t* four_at;
      constexpr int kFour = SIZE == 256 ? 2 * kPairBytes : 1024;           // four r further
      lds_at at;
      if constexpr (SIZE == 256) at = read[t & 1] + (stage * kStage + half * (16 * kPairBytes + 4 * 128) + t * 32);
      else at = (lds_at)(uintptr_t)((uint32_t)(uintptr_t)read[0] ^ (uint32_t)(t << 5)) + (stage * kStage + half * 8192);
      struct { uint64_t lo, hi; } both;
      both.lo = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((four_at)at));
      both.hi = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((four_at)(at + kFour)));
      return __builtin_bit_cast(vec, both);
    } else {
      return *(vec_at)(read[half] + (stage * kStage + t * 2048));
    }
  }
};

// SA and SB: steps of either operand that LDS holds.  Loads arrive in the order in which they are asked for, A's after B's of the same step, so with SA > SB a step waits for all but
// A's newest: its loads have two steps to arrive, B's, which other CUs have asked for as well, one.
// The tile's sums: a lane has C[16 ti + 4 (lane / 16) + 0..3][16 tj + lane % 16] of its wave's part.  `steps` > 0 steps.
template <int TYPE, bool A_COLUMNS, bool B_COLUMNS, int BI, int BJ, int WI, int WJ, int SA = 2, int SB = 2>
struct Tile {
  static constexpr int TI = BI / WI / 16, TJ = BJ / WJ / 16;
  static constexpr int kLds = SA * stage_bytes<A_COLUMNS, BI>() + SB * stage_bytes<B_COLUMNS, BJ>();
  static_assert(SA >= SB && SB >= 2, "A's loads come last");
  static_assert(WI * WJ == 8 && kLds <= 160 * 1024, "eight waves, one workgroup's LDS");
  typedef typename Product<TYPE>::vec vec;
  f32x4 sum[TI][TJ];

  __device__ __forceinline__ void run(const Operand& a_op, const Operand& b_op, int steps, lds_at lds, int wave, int lane) {
    Side<A_COLUMNS, BI, TI> a(a_op, lds, wave, wave / WJ * (BI / WI), lane);
    Side<B_COLUMNS, BJ, TJ> b(b_op, lds + SA * stage_bytes<A_COLUMNS, BI>(), wave, wave % WJ * (BJ / WJ), lane);
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) sum[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // A step is kGroups groups of TJ products, one fragment of A each.  A's are read kAhead groups before they are used, B's for the second half during the first; the
    // stage's last read is then issued kAhead groups before its end, where the barrier stands, and the next stage's first reads run beside the last groups.
    constexpr int kGroups = 2 * TI, kAhead = 3;
    vec x[kAhead + 1], y[2][TJ];
    auto read_a = [&](int stage, int g) { x[g % (kAhead + 1)] = a.template fragment<TYPE>(stage, g / TI, g % TI); };
    auto read_b = [&](int stage, int half, int j) { y[half][j] = b.template fragment<TYPE>(stage, half, j); };
    static_assert(kGroups % (kAhead + 1) == 0, "a step begins with the ring's first place");
    constexpr int kLoadsA = Side<A_COLUMNS, BI, TI>::kLoads, kLoadsB = Side<B_COLUMNS, BJ, TJ>::kLoads;
    auto step = [&](int in_a, int next_a, int in_b, int next_b, int at) {
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        if (g == kGroups - kAhead) {
          // every wave has read the stage, and the next one has arrived for all of them; those behind it may be on their way
          if ((SA == 2 && SB == 2) || at + SA > steps) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
          else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "i"((SA > SB ? kLoadsA : 0) + (SB - 2) * (kLoadsA + kLoadsB)) : "memory");
          if (at + SB < steps) b.load(in_b);
          if (at + SA < steps) a.load(in_a);
        }
        if (g < kGroups - kAhead) read_a(in_a, g + kAhead);
        else read_a(next_a, g + kAhead - kGroups);             // behind the last step: what lies there, for nothing
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
          if (g == j * (TI / 2) / TJ) read_b(in_b, 1, j);
          if (g == kGroups - kAhead + j * 2 / TJ) read_b(next_b, 0, j);
        }
#pragma unroll
        for (int j = 0; j < TJ; ++j) sum[g % TI][j] = Product<TYPE>::add(x[g % (kAhead + 1)], y[g / TI][j], sum[g % TI][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
#pragma unroll
    for (int i = 0; i < SA; ++i)
      if (i < steps) {
        if (i < SB) b.load(i);
        a.load(i);
      }
    if (steps >= SA) asm volatile("s_waitcnt vmcnt(%0)" :: "i"((SA - 1) * kLoadsA + (SB - 1) * kLoadsB) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    asm volatile("s_barrier" ::: "memory");
#pragma unroll
    for (int j = 0; j < TJ; ++j) read_b(0, 0, j);
#pragma unroll
    for (int g = 0; g < kAhead; ++g) read_a(0, g);
    if constexpr (SA == 2 && SB == 2) {
      int at = 0;
      for (; at + 1 < steps; at += 2) {
        step(0, 1, 0, 1, at);
        step(1, 0, 1, 0, at + 1);
      }
      if (at < steps) step(0, 1, 0, 1, at);
    } else {
      int in_a = 0, in_b = 0;
      for (int at = 0; at < steps; ++at) {
        const int next_a = in_a + 1 == SA ? 0 : in_a + 1, next_b = in_b + 1 == SB ? 0 : in_b + 1;
        step(in_a, next_a, in_b, next_b, at);
        in_a = next_a;
        in_b = next_b;
      }
    }
  }
};

// Workgroup -> tile.  Workgroups are dealt out to the 8 XCDs in turn: each gets a run of tiles of its own, in columns of eight, so that the 32 tiles that its CUs work on
// share 8 + 4 operands in its L2.
__device__ __forceinline__ void tile_of(int id, int tiles_i, int tiles_j, int& i, int& j) {
  const int all = tiles_i * tiles_j, each = all / 8, more = all % 8, xcd = id % 8, at = id / 8;
  const int n = xcd * each + min(xcd, more) + at;            // xcd < more have one more
  const int band = n / (8 * tiles_j), first = band * 8, high = min(8, tiles_i - first), within = n - band * 8 * tiles_j;
  j = within / high;
  i = first + within % high;
}

}  // namespace szo
