// Gated MLP up to its hidden values, h = act(x Wg^T) * (x Wu^T), and its gradients.
//
// One matrix kernel serves the forward and both gradient products.  Its operands come as rows along the contraction (x
// and the weights of the forward) or as rows across it (the weights for dx, x and the hidden gradients for dw): either
// kind goes from memory to LDS as it lies and is read from there as fragments along rows or along columns (lds_tile.h),
// so nothing is transposed in memory.  The forward's blocks take the gate and up weights of the same hidden units, 16 and 16 in
// turn, so that a wave holds both products of a unit and the activation, the product and the one rounding are its
// epilogue.
#include "gemm_epilogue.h"
#include "layer.h"
#include "lds_tile.h"

namespace ravel {
namespace {

struct MatArgs {
  // C[m, n] = sum over pairs p and k < K of A[p](m, k) B[p](n, k)
  const void *A[2], *B[2];
  int64_t lda, ldb;
  int M, N, K, pairs;
  int splits, per;  // ranges of the contraction's tiles (all pairs'), and tiles of a range
  // FORWARD: B[0] gate and B[1] up weights, N = 2 hidden; C[0] h, C[1] and C[2] x Wg^T and x Wu^T or null
  // BOTH: two products C[0] = A[0] B[0], C[1] = A[1] B[0], one behind the other in the grid
  void* C[3];
  int64_t ldc, ldg;
  int act;
  float* part;  // splits > 1: [split][M][N]
};
enum { STORE = 0, FORWARD = 1, BOTH = 2 };

RAVEL_DEV float act_f(float x, int kind) { return kind == RAVEL_SILU ? silu_f(x) : gelu_tanh_f(x); }

RAVEL_DEV void put4(float* p, f32x4_t v) { *(f32x4_t*)p = v; }
RAVEL_DEV void put4(bf16_t* p, f32x4_t v) { *(u32x2_t*)p = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }
// Outputs are written in 64 (the forward's) or 128 bytes of a row: a 16 x 16 block leaves the matrix instructions with 4
// columns of row l16 in a lane, 8 bytes.  Stored so, 32 bytes of a row, the forward of 3200 rows, 1024 -> 4096, took 82 us
// instead of 72 and the gradients' products 68 and 65 instead of 64 and 60.
// Lanes l and l ^ 8 trade: afterwards p is of row l16 & 7 and q of row l16 | 8, the lower lanes' columns p's, the upper
// ones' q's.
RAVEL_DEV void trade_rows(u32x4_t& p, u32x4_t& q) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {  // row_ror:8
    const int a = (int)p[r], b = (int)q[r];
    p[r] = (uint32_t)__builtin_amdgcn_update_dpp(a, b, 0x128, 0xF, 0xC, false);
    q[r] = (uint32_t)__builtin_amdgcn_update_dpp(b, a, 0x128, 0xF, 0x3, false);
  }
}
// Rows m0 .. + 15, columns n .. of `out`, blocks that follow each other.
template <typename O>
RAVEL_DEV void put_two_rows(O* out, int64_t ld, int m, int M, int n, int N, u32x4_t p, u32x4_t q) {
  if (n < N && m < M) *(u32x4_t*)(out + m * ld + n) = p;
  if (n < N && m + 8 < M) *(u32x4_t*)(out + (m + 8) * ld + n) = q;
}
RAVEL_DEV void put_blocks(float* out, int64_t ld, int m0, int M, int n, int N, int lane, f32x4_t v, f32x4_t w) {
  u32x4_t p = __builtin_bit_cast(u32x4_t, v), q = __builtin_bit_cast(u32x4_t, w);
  trade_rows(p, q);
  put_two_rows(out, ld, m0 + (lane & 7), M, n + (lane & 8) * 2 + (lane >> 4) * 4, N, p, q);
}
RAVEL_DEV void put_blocks(bf16_t* out, int64_t ld, int m0, int M, int n, int N, int lane, f32x4_t v, f32x4_t w) {
  const u32x4_t p = join_blocks(v, w);
  const int m = m0 + (lane & 15);
  n += joined_column(lane);
  if (n < N && m < M) *(u32x4_t*)(out + m * ld + n) = p;
}
RAVEL_DEV void put_blocks(float* out, int64_t ld, int m0, int M, int n, int N, int lane, f32x4_t v0, f32x4_t v1, f32x4_t v2, f32x4_t v3) {
  put_blocks(out, ld, m0, M, n, N, lane, v0, v1);
  put_blocks(out, ld, m0, M, n + 32, N, lane, v2, v3);
}
RAVEL_DEV void put_blocks(bf16_t* out, int64_t ld, int m0, int M, int n, int N, int lane, f32x4_t v0, f32x4_t v1, f32x4_t v2, f32x4_t v3) {
  u32x4_t p = join_blocks(v0, v1), q = join_blocks(v2, v3);
  trade_rows(p, q);
  put_two_rows(out, ld, m0 + (lane & 7), M, n + (lane & 8) * 4 + joined_column(lane), N, p, q);
}

// BM x BN outputs a block of WM x WN waves.  AC, BC: A, B lie as rows across the contraction.  O: type of the outputs, G: of the
// forward's gate and up values.
//
// What bounds it: a tile of 256 x 256 outputs and 64 contraction indices takes a CU 2048 clocks of matrix instructions and
// 2048 of LDS traffic (192 KB of fragments read, 64 KB filled); the two overlap as far as the schedule below lets them, to
// 3400.  256 x 256 is the largest tile whose sums and two steps' fragments fit the registers of two waves a SIMD; four
// waves of 128 x 128 would read a third less but spill (1210 us instead of 484).  6400 rows, 2048 <-> 8192: forward 430 us
// (1.00 PFLOP/s, with its three outputs in bf16; 458 with gate and up in 32 bits; the products alone as one library call 398), dx
// 441 (0.97; 200 blocks for 256 CUs), dw 359 (1.20); 3200 rows, 1024 <-> 4096: 72 (80), 63 + 10 for the ranges' sums, and 62.
template <typename T, typename O, typename G, int BM, int BN, int WM, int WN, bool AC, bool BC, int MODE>
__global__ __launch_bounds__(64 * WM * WN) void mlp_matrix_kernel(MatArgs a) {
  typedef Mat<T> M;
  typedef typename M::frag frag;
  constexpr int E = sizeof(T), BK = 128 / E, NW = WM * WN;
  constexpr int TM = BM / (16 * WM), TN = BN / (16 * WN);
  constexpr int RA = AC ? BM * E : 128, RBB = BC ? BN * E : 128;  // bytes of a tile's row
  constexpr int SA = BM * 128 / 1024 / NW, SB = BN * 128 / 1024 / NW;
  static_assert(SA >= 1 && SB >= 1 && BM % (16 * WM) == 0 && BN % (16 * WN) == 0, "tiles");
  static_assert(TN % 2 == 0, "two blocks of outputs that follow each other, or a gate block and its up block, in one wave");
  constexpr int STEP = TN % 4 == 0 ? 4 : 2;  // blocks stored together
  // Four arrays: reads along columns of one buffer wait for the loads in flight into another unless the compiler sees
  // that they are apart.
  __shared__ __attribute__((aligned(1024))) char As0[BM * 128], As1[BM * 128], Bs0[BN * 128], Bs1[BN * 128];

  const int lane = threadIdx.x & 63, wave = wave_index(), l16 = lane & 15, grp = lane >> 4;
  const int wm = wave / WN, wn = wave % WN;
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN, tiles_k = (a.K + BK - 1) / BK;
  const int all_m = MODE == BOTH ? 2 * tiles_m : tiles_m;
  int tr, tc, z;
  item_rcz(xcd_tile(blockIdx.x, gridDim.x), all_m, tiles_n, a.splits, tr, tc, z);
  const int which = MODE == BOTH && tr >= tiles_m ? 1 : 0;
  const int m0 = (tr - which * tiles_m) * BM, n0 = tc * BN;
  const int k0 = z * a.per, k1 = min(tiles_k * a.pairs, k0 + a.per);

  // An operand's rows are its own (AC false) or the contraction's; behind its last element are zeros.  Columns
  // behind a row's end read the next row: across the contraction they are outputs that are not stored, along it (the
  // last tile) they are cut off.  So are, by their index, rows behind the contraction's end (their memory may be a live row's).
  const Segments<T, RA> sa0(lane);
  const Segments<T, RBB> sb0(lane);
  const int lda = (int)a.lda * E, ldb = (int)a.ldb * E;
  // bytes from a tile's first element to the operand's end, at k = 0, and bytes to the next tile
  const int64_t a_left = AC ? (int64_t)(a.K - 1) * lda + (a.M - m0) * E : (int64_t)(a.M - 1 - m0) * lda + a.K * E;
  const int64_t b_left = BC                ? (int64_t)(a.K - 1) * ldb + (a.N - n0) * E
                         : MODE == FORWARD ? (int64_t)((a.N - n0) / 2 - 1) * ldb + a.K * E
                                           : (int64_t)(a.N - 1 - n0) * ldb + a.K * E;
  const int64_t a_next = AC ? (int64_t)BK * lda : 128, b_next = BC ? (int64_t)BK * ldb : 128;
  const int64_t a_first = AC ? m0 * E : (int64_t)m0 * lda, b_first = BC ? n0 * E : (int64_t)(MODE == FORWARD ? n0 / 2 : n0) * ldb;
  const auto issue = [&](int t, char* Ad, char* Bd) {  // behind the last tile: zeros
    const auto sa = sa0.fresh();
    const auto sb = sb0.fresh();
    const int pair = t >= tiles_k ? 1 : 0, kt = t - pair * tiles_k, left = a.K * E - kt * 128, rows = a.K - kt * BK;
    const rsrc_t fa = buffer_from((const char*)a.A[MODE == BOTH ? which : pair] + a_first + kt * a_next, t < k1 ? a_left - kt * a_next : 0);
    const int ra = __umul24(sa.row, lda), rb = __umul24(sb.row, ldb);
#pragma unroll
    for (int i = 0; i < SA; ++i) {
      const int seg = wave * SA + i, c = sa.byte_of(seg);
      load_segment(fa, Ad, seg, (AC ? seg * sa.ROWS + sa.row < rows : c < left) ? ra + c + seg * sa.ROWS * lda : kOutside);
    }
    const rsrc_t fb = buffer_from((const char*)a.B[MODE == STORE ? pair : 0] + b_first + kt * b_next, t < k1 ? b_left - kt * b_next : 0);
    if constexpr (MODE == FORWARD) {  // rows 32 j .. + 15 of the tile: gate, the next 16: up weights of the same units
      const rsrc_t fu = buffer_from((const char*)a.B[1] + b_first + kt * b_next, t < k1 ? b_left - kt * b_next : 0);
#pragma unroll
      for (int i = 0; i < SB; ++i) {
        const int seg = wave * SB + i, c = sb.byte_of(seg), u = (seg >> 2) * 16 + (seg & 1) * 8;
        load_segment(seg & 2 ? fu : fb, Bd, seg, c < left ? rb + c + u * ldb : kOutside);
      }
    } else {
#pragma unroll
      for (int i = 0; i < SB; ++i) {
        const int seg = wave * SB + i, c = sb.byte_of(seg);
        load_segment(fb, Bd, seg, (BC ? seg * sb.ROWS + sb.row < rows : c < left) ? rb + c + seg * sb.ROWS * ldb : kOutside);
      }
    }
  };

  f32x4_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  TileLane<T, RA, true> la(lane);
  TileLane<T, RBB, true> lb(lane);
  la.advance(AC ? 0 : wm * TM, AC ? wm * TM : 0);
  lb.advance(BC ? 0 : wn * TN, BC ? wn * TN : 0);
  // The contraction's steps are pipelined by one: the fragments of a tile's second step are read under the matrix
  // instructions of its first, those of the next tile's first step under the second's.  Between the two the waves
  // meet: by then every fragment of the tile is in registers, so its buffer takes the tile after the next.
  constexpr int PRODUCTS = TM * TN * (E == 4 ? 4 : 1), READS = TM * (AC ? (E == 4 ? 4 : 2) : 1) + TN * (BC ? (E == 4 ? 4 : 2) : 1);
  frag af[2][TM], bf[2][TN];
  const auto read = [&](const char* Ad, const char* Bd, int s) {
    lds_char_t* const as = (lds_char_t*)Ad;
    lds_char_t* const bs = (lds_char_t*)Bd;
    const auto ta = la.fresh();
    const auto tb = lb.fresh();
#pragma unroll
    for (int j = 0; j < TN; ++j) bf[s][j] = BC ? tb.along_col(bs, s, j) : tb.along_row(bs, j, s);
#pragma unroll
    for (int i = 0; i < TM; ++i) af[s][i] = AC ? ta.along_col(as, s, i) : ta.along_row(as, i, s);
  };
  const auto multiply = [&](int s) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = M::mma(bf[s][j], af[s][i], acc[i][j]);
  };
  const auto tile = [&](int t, char* Ac, char* Bc, char* An, char* Bn) {
    read(Ac, Bc, 1);
    multiply(0);
    spread<LDS_READS, READS, PRODUCTS>();
    __builtin_amdgcn_sched_barrier(0);
    tile_barrier<0>();
    issue(t + 2, Ac, Bc);
    read(An, Bn, 0);                          // (what the buffer holds, not used)
    multiply(1);
    spread<GLOBAL_LOADS, SA + SB, PRODUCTS / 2>();
    spread<LDS_READS, READS, PRODUCTS - PRODUCTS / 2>();
    __builtin_amdgcn_sched_barrier(0);
  };
  if (k0 < k1) {
    issue(k0, As0, Bs0);
    tile_barrier<0>();
    issue(k0 + 1, As1, Bs1);
    read(As0, Bs0, 0);
    for (int t = k0; t < k1; t += 2) {
      tile(t, As0, Bs0, As1, Bs1);
      if (t + 1 < k1) tile(t + 1, As1, Bs1, As0, Bs0);
    }
  }
  results_ready(acc);

  // acc[i][j] is row l16, columns 4 grp .. + 3 of its 16 x 16 block
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = m0 + (wm * TM + i) * 16;
    if constexpr (MODE == FORWARD) {
#pragma unroll
      for (int j = 0; j < TN; j += STEP) {
        const int u = n0 / 2 + (wn * TN + j) * 8, units = a.N / 2;
        f32x4_t h[STEP / 2];
#pragma unroll
        for (int k = 0; k < STEP / 2; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) h[k][r] = act_f(acc[i][j + 2 * k][r], a.act) * acc[i][j + 2 * k + 1][r];
        O* const hidden = (O*)a.C[0];
        G *const gate = (G*)a.C[1], *const up = (G*)a.C[2];
        if constexpr (STEP == 4) {
          put_blocks(hidden, a.ldc, m, a.M, u, units, lane, h[0], h[1]);
          if (gate) {
            put_blocks(gate, a.ldg, m, a.M, u, units, lane, acc[i][j], acc[i][j + 2]);
            put_blocks(up, a.ldg, m, a.M, u, units, lane, acc[i][j + 1], acc[i][j + 3]);
          }
        } else if (m + l16 < a.M && u + grp * 4 < units) {
          put4(hidden + (m + l16) * a.ldc + u + grp * 4, h[0]);
          if (gate) {
            put4(gate + (m + l16) * a.ldg + u + grp * 4, acc[i][j]);
            put4(up + (m + l16) * a.ldg + u + grp * 4, acc[i][j + 1]);
          }
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < TN; j += STEP) {
        const int n = n0 + (wn * TN + j) * 16;
        float* const part = a.part + ((size_t)z * (MODE == BOTH ? 2 : 1) + which) * a.M * a.N;
        O* const out = (O*)a.C[which];
        if constexpr (STEP == 4) {
          if (a.part)
            put_blocks(part, a.N, m, a.M, n, a.N, lane, acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3]);
          else
            put_blocks(out, a.ldc, m, a.M, n, a.N, lane, acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3]);
        } else {
          if (a.part)
            put_blocks(part, a.N, m, a.M, n, a.N, lane, acc[i][j], acc[i][j + 1]);
          else
            put_blocks(out, a.ldc, m, a.M, n, a.N, lane, acc[i][j], acc[i][j + 1]);
        }
      }
    }
  }
}

// Few rows (up to 16 MT): the weights are all there is to read, once, so nothing is staged.  A block takes 16 hidden
// units, its eight waves a range of the contraction each, with every weight of the range (up to 512 bytes a row) requested
// before the first is used; the waves' sums meet in LDS.  Bound by memory: one row, 2048 -> 8192, 12.6 us for 67 MB, where a bare
// read of as much takes 10.2 (the same again and again, from cache) to 11.3 (other memory each time); 50 rows, 1024 -> 4096,
// 8.1 us, of which the chain of loads, products and join is most.
template <typename T, typename G, int MT>
__global__ __launch_bounds__(512) void mlp_rows_kernel(MatArgs a) {
  typedef Mat<T> M;
  typedef typename M::frag frag;
  constexpr int E = sizeof(T), BATCH = MT == 4 ? 4 : 8;  // steps of 64 bytes requested at once
  __shared__ f32x4_t part[8][2][MT][64];
  const int lane = threadIdx.x & 63, wave = wave_index(), l16 = lane & 15, grp = lane >> 4;
  const int hidden = a.N / 2, u0 = blockIdx.x * 16;
  const int steps = (a.K * E + 63) / 64, per = (steps + 7) / 8;
  const int s0 = wave * per, s1 = min(steps, s0 + per);
  const int unit = min(u0 + l16, hidden - 1);
  const T* const wg = (const T*)a.B[0] + unit * a.ldb;
  const T* const wu = (const T*)a.B[1] + unit * a.ldb;
  f32x4_t acc[2][MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[0][i] = acc[1][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int s = s0; s < s1; s += BATCH) {
    frag g[BATCH], u[BATCH], x[BATCH][MT];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int k = ((s + j) * 4 + grp) * (16 / E);
      const bool in = s + j < s1 && k < a.K;
      g[j] = in ? *(const frag*)(wg + k) : frag{};
      u[j] = in ? *(const frag*)(wu + k) : frag{};
#pragma unroll
      for (int i = 0; i < MT; ++i)
        x[j][i] = in && i * 16 + l16 < a.M ? *(const frag*)((const T*)a.A[0] + (i * 16 + l16) * a.lda + k) : frag{};
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        acc[0][i] = M::mma(g[j], x[j][i], acc[0][i]);
        acc[1][i] = M::mma(u[j], x[j][i], acc[1][i]);
      }
  }
  results_ready(acc);
#pragma unroll
  for (int i = 0; i < MT; ++i) part[wave][0][i][lane] = acc[0][i], part[wave][1][i][lane] = acc[1][i];
  __syncthreads();
  const int i = threadIdx.x >> 6;  // 16 rows of the sums; lane: row l16, units 4 grp .. + 3
  const int m = i * 16 + l16, n = u0 + grp * 4;
  if (i >= MT || m >= a.M || n >= hidden) return;
  f32x4_t g = part[0][0][i][lane], u = part[0][1][i][lane], h;
#pragma unroll
  for (int w = 1; w < 8; ++w) g += part[w][0][i][lane], u += part[w][1][i][lane];
#pragma unroll
  for (int r = 0; r < 4; ++r) h[r] = act_f(g[r], a.act) * u[r];
  put4((T*)a.C[0] + m * a.ldc + n, h);
  if (a.C[1]) {
    put4((G*)a.C[1] + m * a.ldg + n, g);
    put4((G*)a.C[2] + m * a.ldg + n, u);
  }
}

// Ranges of the contraction added in order, bound by HBM: 4 ranges of 3200 x 1024, 10 us, 5.9 TB/s (they lie in cache in part).
template <typename O>
__global__ __launch_bounds__(256) void mlp_sum_kernel(const float* part, int splits, int64_t range, O* c0, O* c1, int64_t ldc,
                                                      int M, int N) {
  const int n4 = N / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (int64_t)M * n4) return;
  const int64_t m = id / n4;
  const int n = (int)(id - m * n4) * 4;
  part += (size_t)blockIdx.y * M * N;
  f32x4_t s = *(const f32x4_t*)(part + m * N + n);
  for (int z = 1; z < splits; ++z) s += *(const f32x4_t*)(part + z * range + m * N + n);
  put4((blockIdx.y ? c1 : c0) + m * ldc + n, s);
}

// The hidden gradients, dg = dh u act'(g) and du = dh act(g), [rows, hidden] each.  In bf16 calls they are rounded to it: they
// are the operands of two matrix products, which take bf16, and written once instead of formed in each of the products' blocks.
// That makes 2.3e-3 against 64 bits where rounding the results alone gives 1.7e-3, and 3.1e-3 where gate and up (G) are bf16
// as well: the caller's choice.  Bound by HBM: three tensors read, two written, 6400 x 8192 in 150 us, 4.9 TB/s (with gate and
// up in bf16 95 to 102 us, 5.1 to 5.5 TB/s).
RAVEL_DEV void act_grad(float x, int kind, float& y, float& slope) {
  if (kind == RAVEL_SILU) {
    const float s = 1.f / (1.f + __expf(-x));
    y = x * s;
    slope = s * (1.f + x * (1.f - s));
  } else {
    // gelu_tanh_f's form: s = 1 / (1 + exp(-2 u)), y = x s, slope = s + x s (1 - s) 2 u'
    const float c = 0.7978845608028654f, x2 = x * x;
    const float s = 1.f / (1.f + __expf(-2.f * c * x * (1.f + 0.044715f * x2)));
    y = x * s;
    // (far out s (1 - s) is 0, and must not meet an infinite x^2)
    const float z = fminf(fmaxf(x, -64.f), 64.f);
    slope = s + z * s * (1.f - s) * (2.f * c) * (1.f + 3.f * 0.044715f * z * z);
  }
}
template <typename T> RAVEL_DEV void get8(const T* p, float (&v)[8]);
template <> RAVEL_DEV void get8<float>(const float* p, float (&v)[8]) {
  const f32x4_t a = *(const f32x4_t*)p, b = *(const f32x4_t*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i], v[i + 4] = b[i];
}
template <> RAVEL_DEV void get8<bf16_t>(const bf16_t* p, float (&v)[8]) {
  const u32x4_t w = *(const u32x4_t*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
}
RAVEL_DEV void put8(float* p, const float (&v)[8]) {
  *(f32x4_t*)p = f32x4_t{v[0], v[1], v[2], v[3]};
  *(f32x4_t*)(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
}
RAVEL_DEV void put8(bf16_t* p, const float (&v)[8]) {
  *(u32x4_t*)p = u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
template <typename T, typename G>
__global__ __launch_bounds__(256) void mlp_hidden_grad_kernel(ravel_mlp a, ravel_mlp_grad g, T* dg, T* du) {
  const int n8 = a.hidden / 8;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (int64_t)a.rows * n8) return;
  const int64_t m = id / n8;
  const int n = (int)(id - m * n8) * 8;
  float x[8], u[8], dh[8];
  get8((const G*)a.gate + m * a.gate_stride + n, x);
  get8((const G*)a.up + m * a.gate_stride + n, u);
  get8((const T*)g.dh + m * g.dh_stride + n, dh);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float y, slope;
    act_grad(x[i], a.act, y, slope);
    x[i] = dh[i] * u[i] * slope;
    u[i] = dh[i] * y;
  }
  put8(dg + m * a.hidden + n, x);
  put8(du + m * a.hidden + n, u);
}

// ---------------------------------------------------------------------------
// plans
// ---------------------------------------------------------------------------
struct MatPlan {
  int tile;  // 0: 256 x 256, 1: 128 x 128, 2: 64 x 64
  int splits, per;
  double us;  // expected
};
constexpr int kTile[3] = {256, 128, 64};
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Tile and ranges of the contraction by the time of the fullest CU: the blocks it gets, one behind the other or side by
// side, times a block's work; ranges cost the traffic of their sums.
MatPlan plan_matrix(int64_t M, int64_t N, int64_t K, int pairs, int products, int elt, bool split) {
  // Measured with 64-wide tiles of the contraction: 1.85 us a tile of 256 x 256; 0.67 of 128 x 128 with two blocks side by
  // side, 0.88 with one alone, which is worth 1.3 of them; 64 x 64 ones 0.25 side by side, the first two in the
  // time of two.
  constexpr double us[3] = {1.85, 0.67, 0.25}, alone[3] = {1.0, 1.3, 2.0};
  constexpr double ends[3] = {3, 1, 0.5};  // a block's first loads and its end (the forward's stores three outputs)
  MatPlan best{};
  for (int t = elt == 4 ? 1 : 0; t < 3; ++t) {
    const int64_t blocks = (int64_t)ceil_div(M, kTile[t]) * ceil_div(N, kTile[t]) * products;
    const int tiles = ceil_div(K, 128 / elt) * pairs;
    const double end = split ? ends[t] : 3 * ends[t];
    for (int s = 1; s <= (split ? 16 : 1); ++s) {
      if (s > 1 && tiles / s < 4) break;
      const int per = tiles ? ceil_div(tiles, s) : 1;
      const double n = (double)((blocks * s + 255) / 256);
      double cost = (n > alone[t] ? n : alone[t]) * per * us[t] * (elt == 4 ? 2.6 : 1) + n * end;
      if (s > 1) cost += 4 + (double)M * N * products * s * 8 / 4e6;       // a launch, and the sums there and back
      if (best.us == 0 || cost < best.us) best = {t, tiles ? ceil_div(tiles, per) : 1, per, cost};
    }
  }
  return best;
}

template <typename T, typename O, bool AC, bool BC, int MODE, typename G = O>
hipError_t launch_matrix(const MatArgs& a, int tile, hipStream_t s) {
  const int64_t blocks = (int64_t)ceil_div(a.M, kTile[tile]) * ceil_div(a.N, kTile[tile]) * a.splits * (MODE == BOTH ? 2 : 1);
  const dim3 grid((unsigned)blocks);
  if (tile == 0) {
    if constexpr (sizeof(T) == 2) mlp_matrix_kernel<T, O, G, 256, 256, 2, 4, AC, BC, MODE><<<grid, 512, 0, s>>>(a);
  } else if (tile == 1) {
    mlp_matrix_kernel<T, O, G, 128, 128, 2, 2, AC, BC, MODE><<<grid, 256, 0, s>>>(a);
  } else {
    mlp_matrix_kernel<T, O, G, 64, 64, 2, 2, AC, BC, MODE><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <typename T, typename G>
hipError_t forward(const ravel_mlp& m, hipStream_t s) {
  MatArgs a{};
  a.A[0] = m.x;
  a.B[0] = m.wg;
  a.B[1] = m.wu;
  a.lda = m.x_stride;
  a.ldb = m.w_stride;
  a.M = m.rows;
  a.N = 2 * m.hidden;
  a.K = m.width;
  a.pairs = 1;
  a.C[0] = m.h;
  a.C[1] = m.gate;
  a.C[2] = m.up;
  a.ldc = m.h_stride;
  a.ldg = m.gate_stride;
  a.act = m.act;
  if (a.M <= 64) {
    const dim3 grid((unsigned)ceil_div(m.hidden, 16));
    if (a.M <= 16) mlp_rows_kernel<T, G, 1><<<grid, 512, 0, s>>>(a);
    else if (a.M <= 32) mlp_rows_kernel<T, G, 2><<<grid, 512, 0, s>>>(a);
    else mlp_rows_kernel<T, G, 4><<<grid, 512, 0, s>>>(a);
    return hipGetLastError();
  }
  // Blocks of 256 x 256 run one a CU, in rounds: the rows behind the last full round go into a launch of smaller tiles where
  // that is sooner (6400 rows, 2048 -> 8192: 6 rounds and 256 rows in 128 x 128 tiles, 447 us, instead of a seventh round,
  // 465; 3200 rows, 1024 -> 4096 stay whole). 4 us: the second launch and the first one's end.
  MatPlan p = plan_matrix(a.M, a.N, a.K, 1, 1, sizeof(T), false), rest{};
  int first = a.M;
  if (p.tile == 0)
    for (int64_t full = ceil_div(a.M, 256) * (int64_t)ceil_div(a.N, 256) / 256, round = full > 4 ? full - 3 : 1; round <= full; ++round) {
      const int64_t rows = round * 256 / ceil_div(a.N, 256) * 256;
      if (rows < 1 || rows >= a.M) continue;
      const MatPlan q = plan_matrix(a.M - rows, a.N, a.K, 1, 1, sizeof(T), false);
      const MatPlan f = plan_matrix(rows, a.N, a.K, 1, 1, sizeof(T), false);
      if (f.tile != 0 || f.us + q.us + 4 >= p.us + rest.us + (rest.us > 0 ? 4 : 0)) continue;
      p = f, rest = q, first = (int)rows;
    }
  const int all = a.M;
  a.M = first;
  a.splits = p.splits;
  a.per = p.per;
  const hipError_t e = launch_matrix<T, T, false, false, FORWARD, G>(a, p.tile, s);
  if (e != hipSuccess || first == all) return e;
  a.M = all - first;
  a.per = rest.per;
  a.A[0] = (const T*)a.A[0] + first * a.lda;
  a.C[0] = (T*)a.C[0] + first * a.ldc;
  if (a.C[1]) a.C[1] = (G*)a.C[1] + first * a.ldg, a.C[2] = (G*)a.C[2] + first * a.ldg;
  return launch_matrix<T, T, false, false, FORWARD, G>(a, rest.tile, s);
}

struct GradBytes {
  size_t hidden, part;  // of one of dg and du; of the ranges' sums
};
GradBytes grad_bytes(const ravel_mlp& m, const ravel_mlp_grad& g) {
  const int e = m.dtype == RAVEL_F32 ? 4 : 2;
  GradBytes b{};
  if (!g.dx && !g.dwg) return b;
  b.hidden = ((size_t)m.rows * m.hidden * e + 255) / 256 * 256;
  if (g.dx) {
    const MatPlan p = plan_matrix(m.rows, m.width, m.hidden, 2, 1, e, true);
    if (p.splits > 1) b.part = (size_t)p.splits * m.rows * m.width * 4;
  }
  if (g.dwg) {
    const MatPlan p = plan_matrix(m.hidden, m.width, m.rows, 1, 2, e, true);
    const size_t n = p.splits > 1 ? (size_t)p.splits * 2 * m.hidden * m.width * 4 : 0;
    if (n > b.part) b.part = n;
  }
  b.part = (b.part + 255) / 256 * 256;
  return b;
}

template <typename O>
hipError_t add_ranges(const MatArgs& a, int products, hipStream_t s) {
  const dim3 grid((unsigned)ceil_div((int64_t)a.M * (a.N / 4), 256), products);
  mlp_sum_kernel<O><<<grid, 256, 0, s>>>(a.part, a.splits, (int64_t)products * a.M * a.N, (O*)a.C[0], (O*)a.C[1], a.ldc, a.M, a.N);
  return hipGetLastError();
}

template <typename T, typename G>
hipError_t gradients(const ravel_mlp& m, const ravel_mlp_grad& g, hipStream_t s) {
  const GradBytes b = grad_bytes(m, g);
  char* const ws = (char*)g.workspace;
  T *const dg = (T*)ws, *const du = (T*)(ws + b.hidden);
  float* const part = (float*)(ws + 2 * b.hidden);
  hipError_t e;
  if (m.rows > 0) {
    mlp_hidden_grad_kernel<T, G><<<ceil_div((int64_t)m.rows * (m.hidden / 8), 256), 256, 0, s>>>(m, g, dg, du);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (g.dx && m.rows > 0) {
    MatArgs a{};
    a.A[0] = dg, a.A[1] = du;
    a.B[0] = m.wg, a.B[1] = m.wu;
    a.lda = m.hidden;
    a.ldb = m.w_stride;
    a.M = m.rows, a.N = m.width, a.K = m.hidden, a.pairs = 2;
    a.C[0] = g.dx;
    a.ldc = g.dx_stride;
    const MatPlan p = plan_matrix(a.M, a.N, a.K, 2, 1, sizeof(T), true);
    a.splits = p.splits, a.per = p.per;
    a.part = p.splits > 1 ? part : nullptr;
    if ((e = launch_matrix<T, T, false, true, STORE>(a, p.tile, s)) != hipSuccess) return e;
    if (a.part && (e = add_ranges<T>(a, 1, s)) != hipSuccess) return e;
  }
  if (g.dwg) {
    MatArgs a{};
    a.A[0] = dg, a.A[1] = du;
    a.B[0] = m.x;
    a.lda = m.hidden;
    a.ldb = m.rows > 1 ? m.x_stride : m.width;  // (one row has no stride)
    a.M = m.hidden, a.N = m.width, a.K = m.rows, a.pairs = 1;
    a.C[0] = g.dwg, a.C[1] = g.dwu;
    a.ldc = g.dw_stride;
    const MatPlan p = plan_matrix(a.M, a.N, a.K, 1, 2, sizeof(T), true);
    a.splits = p.splits, a.per = p.per;
    a.part = p.splits > 1 ? part : nullptr;
    const bool wide = g.weight_dtype == RAVEL_F32;
    if ((e = wide ? launch_matrix<T, float, true, true, BOTH>(a, p.tile, s) : launch_matrix<T, T, true, true, BOTH>(a, p.tile, s)) !=
        hipSuccess)
      return e;
    if (a.part && (e = wide ? add_ranges<float>(a, 2, s) : add_ranges<T>(a, 2, s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t mlp_workspace(const ravel_mlp&) { return 0; }
hipError_t launch_gated_mlp(ravel_mlp m, hipStream_t s) {
  if (m.rows == 0) return hipSuccess;
  const bool wide = m.act & RAVEL_GATE_F32;
  m.act &= ~RAVEL_GATE_F32;
  return m.dtype == RAVEL_F32 ? forward<float, float>(m, s) : wide ? forward<bf16_t, float>(m, s) : forward<bf16_t, bf16_t>(m, s);
}
size_t mlp_grad_workspace(const ravel_mlp& m, const ravel_mlp_grad& g) {
  const GradBytes b = grad_bytes(m, g);
  return 2 * b.hidden + b.part;
}
hipError_t launch_gated_mlp_grad(ravel_mlp m, const ravel_mlp_grad& g, hipStream_t s) {
  if (!g.dx && !g.dwg) return hipSuccess;
  const bool wide = m.act & RAVEL_GATE_F32;
  m.act &= ~RAVEL_GATE_F32;
  return m.dtype == RAVEL_F32 ? gradients<float, float>(m, g, s)
         : wide               ? gradients<bf16_t, float>(m, g, s)
                              : gradients<bf16_t, bf16_t>(m, g, s);
}

}  // namespace ravel
