// What the fused attention kernels share: the tiles of 64 keys or queries in LDS, their copies and fragment reads, and the order of workgroups.
#pragma once
#include "dp_device.h"

#include <type_traits>

namespace dp {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// Layout of a streamed [64 x DHP] bf16 tile in LDS: 64 rows of DHP / 8 16-byte chunks, no padding; the chunk
// at position pos of a row is chunk pos ^ key(row).  A tile is read two ways -- by rows as an MFMA A operand
// (16 consecutive rows, one chunk each, per 256 bytes of LDS bandwidth) and through the transposing load (4
// consecutive rows x 64 bytes) -- and the key keeps both conflict-free:
//   DHP = 64 (128-byte rows, two to the 256 bytes of a bank line): key = row bits (1, 2, 3), a bijection of the 8 rows that
//     share a half of the line among 16 consecutive ones; its bit 2 is row bit 1, so the 4 rows of a transposing read lie in
//     4 different 64-byte bank groups;
//   DHP = 96 (192-byte rows): consecutive rows already start 192 bytes apart, i.e. in different 64-byte groups;
//     rows r and r + 4 share one, so key = (row >> 2) & 3 moves them apart inside the group.
template <int DHP> struct AttnTile;
template <> struct AttnTile<64> {
  static constexpr int PIECES = 2;     // 1 KB copy instructions per wave and tile (16 rows)
  static __device__ __forceinline__ int key(int row) { return ((row & 8) >> 3) | ((row & 4) >> 1) | ((row & 2) << 1); }
};
template <> struct AttnTile<96> {
  static constexpr int PIECES = 3;
  static __device__ __forceinline__ int key(int row) { return (row >> 2) & 3; }
};

// Global -> LDS copy of one tile (`buffer_load ... lds`: the wave's 64 x 16 bytes land contiguously in LDS).
// A wave owns rows 16 * wave .. + 15; each lane keeps the byte offset, inside the (batch, head) slice, of the
// chunk that belongs at its LDS position.  Chunks past d_head get an offset of 2^31, which stays outside the
// buffer descriptor's range whatever tile offset is added: they, like rows past the end of the slice, arrive
// as zeros without touching memory.
template <int DHP>
struct AttnTileCopy {
  using T = AttnTile<DHP>;
  uint32_t off[T::PIECES];
  __device__ __forceinline__ void init(int wave, int lane, int ld, int dh) {
#pragma unroll
    for (int j = 0; j < T::PIECES; ++j) {
      const int o = 1024 * j + 16 * lane;                     // byte inside the wave's 16-row block
      const int row = 16 * wave + o / (2 * DHP), pos = (o % (2 * DHP)) / 16;
      const int chunk = pos ^ T::key(row);
      off[j] = 8 * chunk < dh ? (uint32_t)(row * ld + 8 * chunk) * 2u : 0x80000000u;
    }
  }
  // rows row0 .. row0 + 63 of the slice behind r (the tile offset goes into the per-lane offset: only that
  // one is range-checked)
  __device__ __forceinline__ void issue(u32x4 r, int row0, int ld, bf16* stage, int wave) const {
#pragma unroll
    for (int j = 0; j < T::PIECES; ++j)
      async_copy_16B_raw(r, off[j] + (uint32_t)row0 * (uint32_t)ld * 2u, lds_address(stage) + 2u * (16 * wave * DHP + 512 * j));
  }
};

// Per-lane element offsets of the fragment reads, computed once.  A row fragment (rows 32 * t + l32, k-chunk
// c) is at row[c] + 32 * DHP * t.  A transposed fragment in the slot order of frag_from_mc_accorder (rows
// r0 .. r0 + 15 with r0 a multiple of 16, which leaves the keys alone; columns 32 * i .. + 31) is read as two
// halves at tr_lo[i] + DHP * r0 and tr_hi[i] + DHP * r0 (8 rows apart).
template <int DHP, int KC>
struct AttnFragOff {
  using T = AttnTile<DHP>;
  int row[KC], tr_lo[DHP / 32], tr_hi[DHP / 32];
  __device__ __forceinline__ void init(int lane) {
    const int g = lane >> 5, l32 = lane & 31;
#pragma unroll
    for (int c = 0; c < KC; ++c) row[c] = l32 * DHP + 8 * ((2 * c + g) ^ T::key(l32));
#pragma unroll
    for (int i = 0; i < DHP / 32; ++i) transposed(lane, i, tr_lo[i], tr_hi[i]);
  }
  static __device__ __forceinline__ void transposed(int lane, int i, int& lo, int& hi) {
    const int b = lane >> 4, j = lane & 15, r = 4 * (b >> 1) + (j >> 2), chunk = 4 * i + 2 * (b & 1) + ((j & 3) >> 1);
    lo = r * DHP + 8 * (chunk ^ T::key(r)) + 4 * (j & 1);
    hi = (r + 8) * DHP + 8 * (chunk ^ T::key(r + 8)) + 4 * (j & 1);
  }
  __device__ __forceinline__ bf16x8 row_frag(const bf16* tile, int t, int c) const {
    return *reinterpret_cast<const bf16x8*>(tile + row[c] + 32 * DHP * t);
  }
  __device__ __forceinline__ bf16x8 tr_frag(const bf16* tile, int r0, int i) const {
    const bf16x4 lo = lds_read_tr(tile + tr_lo[i] + DHP * r0);
    const bf16x4 hi = lds_read_tr(tile + tr_hi[i] + DHP * r0);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};
// byte extent of a (batch, head) slice of n rows with leading dimension ld (elements), d_head columns
__device__ __forceinline__ uint32_t attn_slice_bytes(int n, int ld, int dh) { return (uint32_t)(((size_t)(n - 1) * ld + dh) * 2); }

__device__ __forceinline__ bf16x8 pack8(const f32x16& v, int off) {
  bf16x8 o;
#pragma unroll
  for (int u = 0; u < 8; ++u) o[u] = (bf16)v[off + u];
  return o;
}

// Among waves of one priority a SIMD serves the oldest first, so of the workgroups a CU holds one ends early and the last runs alone, at half the
// rate.  Where all workgroups of a launch are resident at once, a wave's priority falls by one every second tile and wraps, which keeps them
// together: 80 heads of 1024 tokens, 640 workgroups, forward 33.7 -> 31.3 us, dQ 45.2 -> 42.5, dK/dV 56.5 -> 52.7.  Where more wait to be
// started, the staggered ends are what lets them start: 40 heads of 4096 tokens lose 5 % with it; one workgroup per CU has nothing to share.
__device__ __forceinline__ void take_turns(int even, int i) {
  if (even) {
    const int turn = (i >> 1) & 3;
    if (turn == 0) __builtin_amdgcn_s_setprio(3);
    else if (turn == 1) __builtin_amdgcn_s_setprio(2);
    else if (turn == 2) __builtin_amdgcn_s_setprio(1);
    else __builtin_amdgcn_s_setprio(0);
  }
}

// tile(i, stage) for i = first .. last - 1, the stages of LDS in turn and known to the compiler: the fragment reads then need no address
// arithmetic and no registers beyond the offsets of AttnFragOff.
template <class F> __device__ __forceinline__ void two_stages(int first, int last, F tile) {
  for (int i = first; i < last; i += 2) {
    tile(i, std::integral_constant<int, 0>());
    if (i + 1 < last) tile(i + 1, std::integral_constant<int, 1>());
  }
}

// Maps a linear workgroup id to (tile along the sequence, batch * head).  Hardware deals
// consecutive ids round-robin to the 8 XCDs; with this map all tiles of one (batch, head) run
// on the same XCD, so its K/V (or Q/dO) stream is fetched into one L2 only.
__device__ __forceinline__ void attn_block_map(int id, int ntiles, int BH, int& tile, int& bh) {
  const int full = (BH / 8) * 8;
  if (id < full * ntiles) {
    const int grp = id / (8 * ntiles), r = id % (8 * ntiles);
    bh = grp * 8 + (r & 7);
    tile = r >> 3;
  } else {
    const int r = id - full * ntiles;
    bh = full + r / ntiles;
    tile = r % ntiles;
  }
}

}  // namespace dp
