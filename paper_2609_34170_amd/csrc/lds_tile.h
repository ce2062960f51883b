// Tiles of rows in LDS, filled straight from global memory and read as MFMA fragments along rows or along
// columns.
//
// A tile holds rows of RB bytes (a power of two, 64 to 1024) of bf16 or 32-bit elements.  The 16-byte chunk c of row r
// lies at position c ^ swizzle(r) of the row, so that the 16 rows of a fragment along rows, and the 4 by 16 elements of
// one along columns, fall on distinct banks.
//
// MFMA 16x16 fragments (l16 = lane % 16, grp = lane / 16): operand A has row l16, operand B column l16, and either
// holds 16 bytes of the contraction, which may run in any order that both share; a result holds rows 4 grp + 0..3 of
// column l16.  One step contracts 64 bytes of a row: 32 bf16 elements in one instruction, 16 32-bit ones in
// four.  A result of 16 (two of them: 32) contraction indices of the next product is that product's operand as it
// stands, its lane's elements being indices 4 grp + 0..3 (of both results).
#pragma once

#include "common.h"

namespace ravel {

#define RAVEL_LDS __attribute__((address_space(3)))
typedef RAVEL_LDS void lds_dst_t;
typedef RAVEL_LDS const char lds_char_t;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4_t;
typedef __amdgpu_buffer_rsrc_t rsrc_t;

constexpr unsigned kOutside = 0x80000000u;  // a byte offset outside every buffer below: such loads give 0

// 2^31 - 1 readable bytes from p on (uniform); callers keep live offsets below that
RAVEL_DEV rsrc_t buffer_from(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, 0x7fffffff, 0x00020000);
}

template <typename T> struct Mat;
template <> struct Mat<bf16_t> {
  typedef bf16x8_t frag;
  static constexpr int CK = 32;  // contraction indices of a step whose operand is a result
  static RAVEL_DEV f32x4_t mma(frag a, frag b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  // results of 2 x 16 indices as an operand (rounded to bf16)
  static RAVEL_DEV frag operand(const f32x4_t* s) {
    const u32x4_t w{pack_bf16x2(s[0][0], s[0][1]), pack_bf16x2(s[0][2], s[0][3]), pack_bf16x2(s[1][0], s[1][1]),
                    pack_bf16x2(s[1][2], s[1][3])};
    return __builtin_bit_cast(frag, w);
  }
};
template <> struct Mat<float> {
  typedef f32x4_t frag;
  static constexpr int CK = 16;
  static RAVEL_DEV f32x4_t mma(frag a, frag b, f32x4_t c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
  static RAVEL_DEV frag operand(const f32x4_t* s) { return s[0]; }
};

template <typename T, int RB>
RAVEL_DEV int swizzle(int r) {
  constexpr int chunks = RB / 16 < 16 ? RB / 16 : 16, lines = RB < 256 ? 256 / RB : 1;
  const int v = (r / lines) & (chunks - 1);
  if (sizeof(T) == 4) return v;
  return ((v << 1) | (v >> (chunks == 16 ? 3 : chunks == 8 ? 2 : 1))) & (chunks - 1);
}

// A lane's addresses inside a tile.  ALIKE: columns are contracted in the order that along_row has (8 consecutive rows a
// lane in 16 bits), so that one operand may run along rows, the other along columns; otherwise in the order of a result.
template <typename T, int RB, bool ALIKE = false>
struct TileLane {
  int row, col[sizeof(T) == 4 ? 4 : 2];
  RAVEL_DEV TileLane(int lane) {
    const int l16 = lane & 15, grp = lane >> 4;
    row = l16 * RB + ((grp ^ swizzle<T, RB>(l16)) << 4);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = grp * 4 + i;
        col[i] = r * RB + (((l16 >> 2) ^ swizzle<T, RB>(r)) << 4) + (l16 & 3) * 4;
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // 16 lanes fetch 4 rows x 16 columns, each receives one column's
        const int r = (ALIKE ? grp * 8 + h * 4 : h * 16 + grp * 4) + (l16 >> 2);
        col[h] = r * RB + ((((l16 >> 1) & 1) ^ swizzle<T, RB>(r)) << 4) + (l16 & 1) * 8;
      }
    }
  }
  // to the fragments `rows` blocks of 16 rows on, along rows, and `cols` blocks of 16 columns on (a power of two's
  // multiple), along columns
  RAVEL_DEV void advance(int rows, int cols) {
    row += rows * 16 * RB;
#pragma unroll
    for (int i = 0; i < (sizeof(T) == 4 ? 4 : 2); ++i) col[i] ^= cols * (16 * (int)sizeof(T));
  }
  // The same addresses, as a value of which the compiler knows nothing: what is derived from it is formed where it is used,
  // not kept in registers from tile to tile.
  RAVEL_DEV TileLane fresh() const {
    TileLane t = *this;
    asm volatile("" : "+v"(t.row));
#pragma unroll
    for (int i = 0; i < (sizeof(T) == 4 ? 4 : 2); ++i) asm volatile("" : "+v"(t.col[i]));
    return t;
  }
  // bytes 64 step .. 64 step + 63 of rows 16 j .. 16 j + 15
  RAVEL_DEV typename Mat<T>::frag along_row(lds_char_t* tile, int j, int step) const {
    return *(RAVEL_LDS const typename Mat<T>::frag*)(tile + j * 16 * RB + (row ^ (step << 6)));
  }
  // columns 16 d .. 16 d + 15 of rows CK j .. CK j + CK - 1, the contraction running over the rows
  RAVEL_DEV typename Mat<T>::frag along_col(lds_char_t* tile, int j, int d) const {
    if constexpr (sizeof(T) == 4) {
      f32x4_t v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *(RAVEL_LDS const float*)(tile + j * 16 * RB + (col[i] ^ (d << 6)));
      return v;
    } else {
      u32x2_t w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        w[h] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                               (RAVEL_LDS s16x4_t*)(tile + j * 32 * RB + (col[h] ^ (d << 5)))));
      return __builtin_bit_cast(bf16x8_t, (u32x4_t{w[0][0], w[0][1], w[1][0], w[1][1]}));
    }
  }
};

// Filling a tile, 1024 bytes (a segment) by one wave in one instruction.  The swizzle is linear in the bits of the row, so a
// lane's byte of a row is its byte of the first segment with the segment's swizzle flipped in, and everything else that
// changes from segment to segment is the same for all lanes.
template <typename T, int RB>
struct Segments {
  static constexpr int ROWS = 1024 / RB;  // of a segment
  int row, byte;                          // of the first segment
  RAVEL_DEV Segments(int lane) {
    row = lane / (RB / 16);
    byte = ((lane % (RB / 16)) ^ swizzle<T, RB>(row)) * 16;
  }
  RAVEL_DEV Segments fresh() const {  // as TileLane::fresh
    Segments s = *this;
    asm volatile("" : "+v"(s.row), "+v"(s.byte));
    return s;
  }
  RAVEL_DEV int byte_of(int seg) const { return byte ^ (swizzle<T, RB>(seg * ROWS) << 4); }
};
RAVEL_DEV void load_segment(rsrc_t from, char* tile, int seg, unsigned offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_dst_t*)(tile + seg * 1024), 16, (int)offset, 0, 0, 0);
}
// Results of two 16 x 16 blocks that follow each other, 4 columns of a row in a lane of each: lane groups trade, the even ones
// keep v, and a lane holds the 8 columns joined_column on of its row.
RAVEL_DEV u32x4_t join_blocks(f32x4_t v, f32x4_t w) {
  const auto a = __builtin_amdgcn_permlane16_swap(pack_bf16x2(v[0], v[1]), pack_bf16x2(w[0], w[1]), false, false);
  const auto b = __builtin_amdgcn_permlane16_swap(pack_bf16x2(v[2], v[3]), pack_bf16x2(w[2], w[3]), false, false);
  return u32x4_t{a[0], b[0], a[1], b[1]};
}
RAVEL_DEV int joined_column(int lane) { return (lane & 16) + (lane >> 5) * 8; }
// `bytes` readable bytes from p on, none if negative (uniform); reads behind them give 0
RAVEL_DEV rsrc_t buffer_from(const void* p, int64_t bytes) {
  const int n = bytes > 0x7fffffff ? 0x7fffffff : bytes < 0 ? 0 : (int)bytes;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, n, 0x00020000);
}
RAVEL_DEV int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }  // (the compiler knows it uniform)

// Until at most `n` of this wave's vector memory operations are outstanding, and its LDS reads are done; then every wave.
// What the waves have loaded is then in LDS, and what they have read before may be overwritten.
template <int N>
RAVEL_DEV void tile_barrier() {
  // vmcnt(N) expcnt(7) lgkmcnt(0)
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// Sums of matrix instructions, before they are used by others behind a loop or a branch: 16 wait states, where the 16 x 16
// products need 8 (bf16) and 10 (32 bits).  The compiler leaves them itself, but has been seen to leave too few where a uniform
// branch skips a few instructions; once a block costs nothing.  What uses a result comes behind the asm that names it; copies
// that the compiler puts in front of that, as everything in a loop, are found by tests/test_machine_code.py.
template <int N, int M>
RAVEL_DEV void results_ready(f32x4_t (&acc)[N][M]) {
  asm volatile("s_nop 15" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < M; ++j) asm volatile("" : "+v"(acc[i][j]));
}

// Instructions of the region up to here in this order: N of a kind (LDS_READS, GLOBAL_LOADS), each followed by its share
// of PRODUCTS matrix instructions, so that neither waits for the other's queue.
enum { MATRIX = 0x8, GLOBAL_LOADS = 0x20, LDS_READS = 0x100 };
template <int KIND, int N, int PRODUCTS, int I = 0>
RAVEL_DEV void spread() {
  if constexpr (I < N) {
    constexpr int share = PRODUCTS * (I + 1) / N - PRODUCTS * I / N;
    __builtin_amdgcn_sched_group_barrier(KIND, 1, 0);
    if constexpr (share > 0) __builtin_amdgcn_sched_group_barrier(MATRIX, share, 0);
    spread<KIND, N, PRODUCTS, I + 1>();
  }
}

}  // namespace ravel
