// Product of two 8-bit (e4m3) matrices with a scale for each block of 128 along
// the summed axis:
//   out[m, n] = sum over blocks kb of sa[kb, m] sb[kb, n] P_kb[m, n],
//   P_kb[m, n] = sum over k in block kb of a[m, k] b[n, k]
// (sb per row of b, or per 128 rows of it), then + bias[n], ReLU, one rounding.
//
// P_kb of a 32 x 32 tile is a chain of MFMAs from zero; its 16 values per lane
// are added to fp32 accumulators with the scales' product, on the vector ALU
// beside the next chain. b's rows are the MFMA's first operand: a lane then
// holds runs of 4 neighbouring n of one m, one scale of a, and writes 4 outputs
// at once.
//
// Two forms of P_kb:
//  * exact products, fp32 sums: e4m3 values become bf16 (exactly) on their way
//    from LDS to 8 v_mfma_f32_32x32x16_bf16;
//  * fast: v_mfma_f32_16x16x128_f8f6f4 on the bytes themselves, twice the rate. That instruction (like the other 8-bit ones) adds its products in
//    groups of 8 with about 13 bits below the largest of the group (measured:
//    2^16 + 2^3 is kept, 2^16 + 2^2 is not; between groups sums are fp32), so
//    a result is off by about 1.4e-5 of its size on normal data: a hundredth
//    of a bf16 output's rounding, but not fp32. The caller asks for it.
//
// Tiles of a and b pass through LDS, 128 bytes a row and block, loaded past the
// registers; the 16-byte chunk c of row r sits at position c ^ (r / 2 % 8), so
// that 16 lanes reading one chunk of 16 rows meet every bank once.
#include <algorithm>

#include "sage_encode.hpp"
#include "sage_internal.hpp"

namespace sage {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(int)))) int intx8;
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int intx4;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 mfma_bf16x8;

__device__ __forceinline__ int swz(int r) { return (r >> 1) & 7; }

// LDS[to + 16 * lane] = 16 bytes at base + off, for the lanes in `mask`; the
// second form 4 bytes. Completion is tracked with wait_all_loads. The lanes are
// masked inside the asm: the loop around it stays one basic block, whose order
// the compiler keeps. (The waves are full, so all lanes are active before and
// after.)
__device__ __forceinline__ void load16_to_lds(const void* base, uint32_t off, uint32_t to, uint64_t mask) {
  asm volatile("s_mov_b64 exec, %3\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1"
               :: "v"(off), "s"(base), "s"(to), "s"(mask) : "memory");
}
__device__ __forceinline__ void load4_to_lds(const void* base, uint32_t off, uint32_t to, uint64_t mask) {
  asm volatile("s_mov_b64 exec, %3\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1\n\ts_mov_b64 exec, -1"
               :: "v"(off), "s"(base), "s"(to), "s"(mask) : "memory");
}
__device__ __forceinline__ uint64_t uniform64(uint32_t lo, uint32_t hi) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)hi) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)lo);
}
// LDS address of a shared array; the array counts as written by the loads from here on.
__device__ __forceinline__ uint32_t lds_address(char* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)p;
}
__device__ __forceinline__ void wait_all_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// Workgroup barrier behind this wave's LDS operations.
__device__ __forceinline__ void barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("s_barrier" ::: "memory");
}

// 16 e4m3 bytes as two operands of 8 bf16 values (exact: 4 significant bits, 2^-9 to 448).
struct Operands {
  mfma_bf16x8 v[2];
};
__device__ __forceinline__ Operands to_bf16(intx4 u) {
  union { bf16x2 p[8]; Operands o; } r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], 1.0f, false);
    r.p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], 1.0f, true);
  }
  return r.o;
}
__device__ __forceinline__ floatx4 mfma_e4m3(const intx8& a, const intx8& b) {
  const floatx4 zero = {};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, zero, 0, 0, 0, 0, 0, 0);
}

// ReLU; a NaN stays one.
__device__ __forceinline__ floatx4 act(floatx4 y, bool relu) {
  if (relu) {
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = y[j] < 0.0f ? 0.0f : y[j];
  }
  return y;
}
// Bias, ReLU and the store of 4 neighbouring outputs of a row.
template <class O, bool kVec>
__device__ __forceinline__ void finish4(floatx4 y, floatx4 bias, bool relu, O* row, int n, int N) {
  y = act(y + bias, relu);
  const float v[4] = {y[0], y[1], y[2], y[3]};
  store_row<O, 4, kVec>(v, row, n, N);
}
template <bool kVec>
__device__ __forceinline__ floatx4 bias4(const float* __restrict__ bias, int n, int N) {
  floatx4 v = {};
  if (bias) {
    float f[4];
    load_row<float, 4, kVec>(f, bias, n, N);
    v = floatx4{f[0], f[1], f[2], f[3]};
  }
  return v;
}

// What a workgroup of W waves computes: BM rows of a x BN rows of b, over blocks
// [kb0, kb1) of the summed axis; and the loads of its stages in LDS.
template <int BM, int BN, int W, bool kSquare>
struct Tile {
  static constexpr int kTileBytes = (BM + BN) * kBlock;
  static constexpr int kStageBytes = kTileBytes + (BM + BN) * 4;   // rows of a and of b, then their scales
  static constexpr int kPieces = (BM + BN) / 8 / W;      // 8 rows x 128 bytes per load and wave
  static_assert((BM + BN) / 64 == W && BM == BN && kPieces == 8, "four pieces of each operand and 64 scales a wave");

  int m0, n0, kb0, kb1, split;
  const char *a_base, *b_base;                           // the tile's first rows
  const float* scale_base;                               // this wave's 64 scales come from here: row kb, entry scale_at
  uint32_t scale_at;
  int scale_ld;
  uint32_t off[kPieces];                                 // this lane's 16 bytes of each piece
  int full;                                              // whole blocks
  int tail_chunks;                                       // 16-byte chunks of a row in the block behind them
  uint64_t tail_lanes;                                   // the lanes whose chunks those are (the same in each piece)

  __device__ __forceinline__ Tile(const Fp8Product& p, int tiles_m, int tiles_n, int splits, int blocks_per_split, int w) {
    // Workgroup b runs on XCD b % 8. Each XCD takes a run of tiles, and in it
    // bands of 4 tiles of a, walked along b: the 32 tiles that its CUs work on
    // at a time are 4 x 8, whose rows its L2 holds.
    const int total = tiles_m * tiles_n * splits, per = total / 8;
    int t = blockIdx.x;
    if (t < per * 8) t = t % 8 * per + t / 8;
    split = t % splits;
    t /= splits;
    const int band = t / (4 * tiles_n), height = min(4, tiles_m - 4 * band);
    t -= band * 4 * tiles_n;
    m0 = (4 * band + t % height) * BM;
    n0 = t / height * BN;
    const int kblocks = (p.K + kBlock - 1) / kBlock;
    full = p.K / kBlock;
    kb0 = split * blocks_per_split;
    kb1 = min(kblocks, kb0 + blocks_per_split);
    tail_chunks = p.K % kBlock / 16;
    a_base = reinterpret_cast<const char*>(p.a) + (long long)m0 * p.K;
    b_base = reinterpret_cast<const char*>(p.b) + (long long)n0 * p.K;
    const int lane = (int)lane_id();
    tail_lanes = __ballot(chunk(0, w, lane) < tail_chunks);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {                  // rows past the end read the last one; their products are not stored
      const int r = (i * W + w) * 8 + lane / 8;
      const int row = r < BM ? min(r, p.M - 1 - m0) : min(r - BM, p.N - 1 - n0);
      off[i] = (uint32_t)row * (uint32_t)p.K + (uint32_t)chunk(i, w, lane) * 16u;
    }
    const int r = w * 64 + lane;
    if (w * 64 < BM) {
      scale_base = p.a_scales;
      scale_ld = p.M;
      scale_at = (uint32_t)min(m0 + r, p.M - 1) * 4u;
    } else {
      const int n = min(n0 + r - BM, p.N - 1);
      scale_base = p.b_scales;
      scale_ld = kSquare ? (p.N + kBlock - 1) / kBlock : p.N;
      scale_at = (uint32_t)(kSquare ? n / kBlock : n) * 4u;
    }
  }
  static __device__ __forceinline__ int chunk(int i, int w, int lane) {
    return (lane % 8) ^ swz((i * W + w) * 8 + lane / 8);
  }
  // Piece i (8: the scales) of block kb into stage st. Of a block that is not
  // whole only the chunks that the rows have are loaded; of kb >= kb1 nothing.
  __device__ __forceinline__ void load(uint32_t lds, int kb, int st, int w, int i) const {
    const uint32_t on = kb < kb1 ? ~0u : 0u;
    if (i < kPieces) {
      const uint32_t lo = kb < full ? on : on & (uint32_t)tail_lanes, hi = kb < full ? on : on & (uint32_t)(tail_lanes >> 32);
      load16_to_lds((i < kPieces / 2 ? a_base : b_base) + (long long)kb * kBlock, off[i],
                    lds + (uint32_t)(st * kStageBytes + (i * W + w) * 8 * kBlock), uniform64(lo, hi));
    } else {
      load4_to_lds(scale_base + (long long)kb * scale_ld, scale_at, lds + (uint32_t)(st * kStageBytes + kTileBytes + w * 256),
                   uniform64(on, on));
    }
  }
  __device__ __forceinline__ void load_all(uint32_t lds, int kb, int st, int w) const {
#pragma unroll
    for (int i = 0; i <= kPieces; ++i) load(lds, kb, st, w, i);
  }
};

// Outputs y of row m, columns n to n + 3.
template <class O, bool kVec>
__device__ __forceinline__ void put4(const Fp8Product& p, int splits, int split, float* part, int m, int n, floatx4 y,
                                     floatx4 bias) {
  if (m >= p.M || n >= p.N) return;
  if (splits > 1) finish4<float, kVec>(y, floatx4{}, false, part + ((long long)split * p.M + m) * p.N, n, p.N);
  else finish4<O, kVec>(y, bias, p.relu, static_cast<O*>(p.out) + (long long)m * p.N, n, p.N);
}

// The exact form: WM x WN waves of 32 x 32 tiles.
template <int BM, int BN, int WM, int WN, bool kSquare, class O, bool kVec>
__global__ void __launch_bounds__(64 * WM * WN, 2) matmul_exact_kernel(Fp8Product p, int tiles_m, int tiles_n, int splits,
                                                                       int blocks_per_split, float* __restrict__ part) {
  typedef Tile<BM, BN, WM * WN, kSquare> T;
  constexpr int MT = BM / WM / 32, NT = BN / WN / 32;
  static_assert(BN / WN <= kBlock, "a wave's columns share a square block's scale");
  __shared__ __attribute__((aligned(16))) char lds[2 * T::kStageBytes];
  const uint32_t to = lds_address(lds);
  const int lane = (int)lane_id();
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  const int wm = w % WM, wn = w / WM;
  const T tile(p, tiles_m, tiles_n, splits, blocks_per_split, w);
  const int l32 = lane & 31, half = lane >> 5;
  floatx16 acc[NT][MT] = {};
  // Chunk 2 t + half of row r0 + l32: the same choice for a and b, so the lanes
  // of a half hold the same k. Chunks past a row's end are zeros.
  auto piece = [&](const char* stage, int r0, int t, int chunks) {
    const intx4 v = *reinterpret_cast<const intx4*>(stage + (r0 + l32) * kBlock + (((2 * t + half) ^ swz(l32)) * 16));
    return 2 * t + half < chunks ? v : intx4{};
  };
  auto block = [&](const char* stage, int chunks) {
    const float* const sc = reinterpret_cast<const float*>(stage + T::kTileBytes);
    float sa[MT];
    Operands wa[MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      sa[i] = sc[(wm * MT + i) * 32 + l32];
#pragma unroll
      for (int t = 0; t < 4; ++t) wa[i][t] = to_bf16(piece(stage, (wm * MT + i) * 32, t, chunks));
    }
    if constexpr (kSquare) {
      const float sb = sc[BM + wn * NT * 32];
#pragma unroll
      for (int i = 0; i < MT; ++i) sa[i] *= sb;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int r0 = BM + (wn * NT + j) * 32;
      intx4 fb[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) fb[t] = piece(stage, r0, t, chunks);
      floatx16 y[MT] = {};
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const Operands wb = to_bf16(fb[t]);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int i = 0; i < MT; ++i)
            y[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb.v[k], wa[i][t].v[k], y[i], 0, 0, 0);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        floatx4 sb;
        if constexpr (!kSquare) sb = *reinterpret_cast<const floatx4*>(sc + r0 + q * 8 + half * 4);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[j][i][4 * q + e] = fmaf(y[i][4 * q + e], kSquare ? sa[i] : sa[i] * sb[e], acc[j][i][4 * q + e]);
      }
    }
  };
  tile.load_all(to, tile.kb0, 0, w);
  const int whole = min(tile.kb1, tile.full);
  int st = 0;
  for (int kb = tile.kb0; kb < whole; ++kb, st ^= 1) {
    wait_all_loads();
    barrier();                                           // this stage has landed; the other one is free
    tile.load_all(to, kb + 1, st ^ 1, w);
    block(lds + st * T::kStageBytes, 8);
  }
  if (whole < tile.kb1) {
    wait_all_loads();
    barrier();
    block(lds + st * T::kStageBytes, tile.tail_chunks);
  }
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int n = tile.n0 + (wn * NT + j) * 32 + q * 8 + half * 4;
      const floatx4 bias = bias4<kVec>(p.bias, n, p.N);
#pragma unroll
      for (int i = 0; i < MT; ++i)
        put4<O, kVec>(p, splits, tile.split, part, tile.m0 + (wm * MT + i) * 32 + l32, n,
                      floatx4{acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]}, bias);
    }
}

// ---------------------------------------------------------------------------
// The fast form: WM x WN waves of 16 x 16 tiles, one MFMA a tile and block.
// A workgroup per CU walks a list of tiles, and its loads run on from one tile
// to the next, so a tile's start waits for nothing and its outputs are written
// while the next one's first blocks arrive.
//
// A group is one 16-row tile of b against the wave's MS tiles of a. While a
// group's MFMAs run, the rows of b of the group after the next are read, and each
// result is added up kBehind MFMAs later. The block's last two groups run behind the
// barrier that frees the stage, tile of a by tile of a: a tile's registers take
// its rows of the next stage as soon as its two MFMAs are issued, so the matrix
// cores have work while the next block's first rows are read. The loads of the
// block after that go out one by one, the first MS behind the barrier and the
// others in the next block: as a burst of 9 they fill the address unit's queue,
// and the waves wait there with their MFMAs behind.
// ---------------------------------------------------------------------------
constexpr int kBehind = 3;

struct TileAt {
  int m0, n0, kb0, kb1, split;
};
// The tiles, in the order of the list: bands of 4 tiles of a, walked along b.
struct TileList {
  int tiles_m, tiles_n, splits, blocks_per_split, kblocks, bm, bn;
  __host__ __device__ int size() const { return tiles_m * tiles_n * splits; }
  __device__ __forceinline__ TileAt at(int t) const {
    TileAt r;
    r.split = t % splits;
    t /= splits;
    const int band = t / (4 * tiles_n), height = min(4, tiles_m - 4 * band);
    t -= band * 4 * tiles_n;
    r.m0 = (4 * band + t % height) * bm;
    r.n0 = t / height * bn;
    r.kb0 = r.split * blocks_per_split;
    r.kb1 = min(kblocks, r.kb0 + blocks_per_split);
    return r;
  }
};
// A block of a workgroup's list: block kb of a tile, `t` the tile's place. Workgroup
// b runs on XCD b % 8, each XCD takes a run of the list, and its workgroups every
// (gridDim / 8)th tile of the run: the 32 tiles that an XCD's CUs work on at a time
// are neighbours, whose rows its L2 holds.
struct BlockAt {
  int t, end, kb;
  TileAt tile;
  __device__ __forceinline__ BlockAt(const TileList& list) {
    const int run = (list.size() + 7) / 8, x = blockIdx.x % 8;
    t = x * run + (int)blockIdx.x / 8;
    end = min(x * run + run, list.size());
    if (on()) tile = list.at(t), kb = tile.kb0;
  }
  __device__ __forceinline__ bool on() const { return t < end; }
  __device__ __forceinline__ void advance(const TileList& list) {   // true on a new tile
    if (on() && ++kb == tile.kb1) {
      t += (int)gridDim.x / 8;
      if (on()) tile = list.at(t), kb = tile.kb0;
    }
  }
};

template <int BM, int BN, int WM, int WN, bool kSquare, class O, bool kVec>
__global__ void __launch_bounds__(64 * WM * WN) matmul_fast_kernel(Fp8Product p, TileList list, float* __restrict__ part) {
  constexpr int W = WM * WN;
  constexpr int kTileBytes = (BM + BN) * kBlock, kStageBytes = kTileBytes + (BM + BN) * 4;
  constexpr int MS = BM / WM / 16, NS = BN / WN / 16;
  constexpr int kPieces = (BM + BN) / 8 / W;             // 8 rows x 128 bytes per load and wave: a's, then b's
  constexpr int kMfmas = NS * MS, kLast = (NS - 2) * MS; // MFMAs of a block, and those before the barrier
  constexpr int kEarly = kPieces / 2, kLate = kPieces - kEarly + 1;   // a's pieces behind the barrier; b's and the scales later,
  constexpr int kGap = 2 * kLate <= kLast ? 2 : 1;       // every kGap MFMAs
  static_assert(BM == BN && kPieces == 8 && (BM + BN) / 64 == W, "four pieces of each operand and 64 scales a wave");
  static_assert(kEarly == MS && kGap * kLate <= kLast, "a piece for every two MFMAs behind the barrier, the others before the next");
  static_assert(kBehind <= MS && NS % 4 == 0, "a result is added up in the next group at the latest; the rings close with a block");
  static_assert(BN / WN <= kBlock, "a wave's columns share a square block's scale");
  __shared__ __attribute__((aligned(16))) char lds[2 * kStageBytes];
  const uint32_t lds0 = lds_address(lds);
  const int lane = (int)lane_id();
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  const int wm = w % WM, wn = w / WM;

  // ---- loads. Chunk (lane % 8) ^ swz(row) of 8 rows a piece; rows past the end
  // read the last one, and their products are not stored. Of a block that is
  // not whole only the chunks that the rows have are loaded, the others zeroed.
  const int chunk = (lane % 8) ^ swz(w * 8 + lane / 8);  // the same in each piece: they are 8 W rows apart
  static_assert(W % 2 == 0, "8 W rows apart keep swz");
  const int full = p.K / kBlock;
  const uint64_t tail_lanes = __ballot(chunk < p.K % kBlock / 16);
  uint32_t off_a[kEarly], off_b[kPieces - kEarly], scale_at;
  const bool a_scale = w * 64 < BM;
  const float* const scale_base = a_scale ? p.a_scales : p.b_scales;
  const int scale_ld = a_scale ? p.M : kSquare ? (p.N + kBlock - 1) / kBlock : p.N;
  auto set_a = [&](const TileAt& t) {
#pragma unroll
    for (int i = 0; i < kEarly; ++i)
      off_a[i] = (uint32_t)min((i * W + w) * 8 + lane / 8, p.M - 1 - t.m0) * (uint32_t)p.K + (uint32_t)chunk * 16u;
  };
  auto set_b = [&](const TileAt& t) {
#pragma unroll
    for (int i = 0; i < kPieces - kEarly; ++i)
      off_b[i] = (uint32_t)min((i * W + w) * 8 + lane / 8, p.N - 1 - t.n0) * (uint32_t)p.K + (uint32_t)chunk * 16u;
    const int r = w * 64 + lane, n = min(t.n0 + r - BM, p.N - 1);
    scale_at = (uint32_t)(a_scale ? min(t.m0 + r, p.M - 1) : kSquare ? n / kBlock : n) * 4u;
  };
  auto load = [&](const BlockAt& at, int st, int i) {    // piece i of a block, kPieces: its scales
    const uint32_t on = at.on() ? ~0u : 0u;
    const uint32_t stage = lds0 + (uint32_t)(st * kStageBytes);
    if (i < kPieces) {
      const uint32_t lo = at.kb < full ? on : on & (uint32_t)tail_lanes, hi = at.kb < full ? on : on & (uint32_t)(tail_lanes >> 32);
      const uint64_t mask = uniform64(lo, hi);
      const char* base = reinterpret_cast<const char*>(i < kEarly ? p.a : p.b) +
                         (long long)(i < kEarly ? at.tile.m0 : at.tile.n0) * p.K + (long long)at.kb * kBlock;
      load16_to_lds(base, i < kEarly ? off_a[i < kEarly ? i : 0] : off_b[i < kEarly ? 0 : i - kEarly],
                    stage + (uint32_t)((i * W + w) * 8 * kBlock), mask);
    } else {
      load4_to_lds(scale_base + (long long)at.kb * scale_ld, scale_at, stage + (uint32_t)(kTileBytes + w * 256), uniform64(on, on));
    }
  };
  // The zeros of a block that is not whole (in its own branch: one block in a tile at most).
  auto zero_tail = [&](const BlockAt& at, int st, int first, int last) {
    if (!at.on() || at.kb < full || chunk * 16 < p.K % kBlock) return;
    for (int i = first; i < last; ++i)
      *reinterpret_cast<intx4*>(lds + st * kStageBytes + (i * W + w) * 8 * kBlock + lane * 16) = intx4{};
  };

  // ---- fragments and sums
  const int l16 = lane & 15, g4 = lane >> 4;
  const int at_a = (wm * MS * 16 + l16) * kBlock, at_b = (BM + wn * NS * 16 + l16) * kBlock;
  const int lo = (g4 ^ swz(l16)) * 16, hi = ((g4 + 4) ^ swz(l16)) * 16;   // chunks g4 and g4 + 4 of a row
  auto rows = [&](const char* stage, int at) {
    const intx4 x = *reinterpret_cast<const intx4*>(stage + at + lo), y = *reinterpret_cast<const intx4*>(stage + at + hi);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  floatx4 acc[NS][MS];
  intx8 fa[MS], fb[4];                                   // of b: groups j % 4
  float sa[MS], sa_next[MS];
  floatx4 sb[4];
  floatx4 y[kBehind + 1];
  const int at_sa = kTileBytes + (wm * MS * 16 + l16) * 4, at_sb = kTileBytes + (BM + wn * NS * 16) * 4;
  auto read_b = [&](const char* stage, int j) {
    fb[j % 4] = rows(stage, at_b + j * 16 * kBlock);
    if constexpr (!kSquare) sb[j % 4] = *reinterpret_cast<const floatx4*>(stage + at_sb + j * 64 + g4 * 16);
  };
  auto read_scales = [&](const char* stage) {
#pragma unroll
    for (int i = 0; i < MS; ++i) {
      sa_next[i] = *reinterpret_cast<const float*>(stage + at_sa + i * 64);
      if constexpr (kSquare) sa_next[i] *= *reinterpret_cast<const float*>(stage + at_sb);
    }
  };
  // MFMA number t of a block is of this group and tile of a: the last two groups in the order of a's tiles.
  auto group = [](int t) { return t < kLast ? t / MS : NS - 2 + (t - kLast) % 2; };
  auto of_a = [](int t) { return t < kLast ? t % MS : (t - kLast) / 2; };
  // The empty asm statements keep the MFMAs and the additions where they stand;
  // left to the compiler, an MFMA moves down to its addition, or the additions
  // behind the block with every y alive until then.
  auto multiply = [&](int t) {
    y[t % (kBehind + 1)] = mfma_e4m3(fb[group(t) % 4], fa[of_a(t)]);
    asm volatile("" : "+v"(y[t % (kBehind + 1)]));
  };
  auto add_up = [&](int t) {
    const int j = group(t), i = of_a(t);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      acc[j][i][e] = fmaf(y[t % (kBehind + 1)][e], kSquare ? sa[i] : sa[i] * sb[j % 4][e], acc[j][i][e]);
    asm volatile("" : "+v"(acc[j][i]));
  };

  BlockAt cur(list);
  if (!cur.on()) return;
  BlockAt early = cur, late = cur;
  set_a(cur.tile);
  set_b(cur.tile);
#pragma unroll
  for (int i = 0; i <= kPieces; ++i) load(cur, 0, i);
  zero_tail(cur, 0, 0, kPieces);
  wait_all_loads();
  barrier();
  early.advance(list);
  if (early.on() && early.t != cur.t) set_a(early.tile);
#pragma unroll
  for (int i = 0; i < kEarly; ++i) load(early, 1, i);
  zero_tail(early, 1, 0, kEarly);
  read_b(lds, 0);
  read_b(lds, 1);
#pragma unroll
  for (int i = 0; i < MS; ++i) fa[i] = rows(lds, at_a + i * 16 * kBlock);
  read_scales(lds);

  for (int st = 0; cur.on();) {
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int i = 0; i < MS; ++i) acc[j][i] = floatx4{};
    for (; cur.kb < cur.tile.kb1; ++cur.kb, st ^= 1) {
      // This block is in stage st; late, the next one, goes to the other stage, and
      // early, the one after that, to this one.
      if (early.on() && early.t != late.t) set_b(early.tile);
      late = early;
      early.advance(list);
      if (early.on() && early.t != late.t) set_a(early.tile);
      zero_tail(late, st ^ 1, kEarly, kPieces);
      const char* const stage = lds + st * kStageBytes;
      const char* const next = lds + (st ^ 1) * kStageBytes;
#pragma unroll
      for (int i = 0; i < MS; ++i) sa[i] = sa_next[i];
#pragma unroll
      for (int j = 0; j < NS - 2; ++j) {
        read_b(stage, j + 2);
        __builtin_amdgcn_sched_barrier(0);               // in this order: the compiler's own waits for each result
#pragma unroll
        for (int t = j * MS; t < (j + 1) * MS; ++t) {
          multiply(t);
          if (t >= kBehind) add_up(t - kBehind);
          if (t % kGap == kGap - 1 && t / kGap < kLate) load(late, st ^ 1, kEarly + t / kGap);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      wait_all_loads();
      barrier();                                         // the next stage has landed, this one is free
#pragma unroll
      for (int t = kLast; t < kMfmas; ++t) {             // past the list's end the reads are of a stale stage, never used
        multiply(t);
        add_up(t - kBehind);
        if (t == kLast) read_b(next, 0);
        if (t == kLast + kBehind) read_b(next, 1);       // its scales' registers: group NS - 3's last result is added
        if (t % 2 == 0) load(early, st, (t - kLast) / 2);
        if ((t - kLast) % 2) fa[of_a(t)] = rows(next, at_a + of_a(t) * 16 * kBlock);
        __builtin_amdgcn_sched_barrier(0);
      }
      read_scales(next);
#pragma unroll
      for (int t = kMfmas - kBehind; t < kMfmas; ++t) add_up(t);
      zero_tail(early, st, 0, kEarly);
    }
    const TileAt done = cur.tile;
    const bool octets = sizeof(O) == 2 && p.N % 8 == 0 && list.splits == 1;
#pragma unroll
    for (int j = 0; j < NS; j += 2) {
      const int n = done.n0 + (wn * NS + j) * 16 + g4 * 4;
      const floatx4 bias0 = bias4<kVec>(p.bias, n, p.N), bias1 = bias4<kVec>(p.bias, n + 16, p.N);
#pragma unroll
      for (int i = 0; i < MS; ++i) {
        const int m = done.m0 + (wm * MS + i) * 16 + l16;
        if (octets) {
          // Neighbouring rows of 16 lanes exchange halves of tiles j and j + 1: a lane
          // then has 8 neighbouring outputs of one of them.
          const floatx4 v0 = act(acc[j][i] + bias0, p.relu), v1 = act(acc[j + 1][i] + bias1, p.relu);
          const auto x = __builtin_amdgcn_permlane16_swap(bf16_pair(v0[0], v0[1]), bf16_pair(v1[0], v1[1]), false, false);
          const auto z = __builtin_amdgcn_permlane16_swap(bf16_pair(v0[2], v0[3]), bf16_pair(v1[2], v1[3]), false, false);
          const int n8 = done.n0 + (wn * NS + j + (g4 & 1)) * 16 + (g4 >> 1) * 8;
          if (m < p.M && n8 < p.N)
            *reinterpret_cast<uint4*>(static_cast<O*>(p.out) + (long long)m * p.N + n8) = make_uint4(x[0], z[0], x[1], z[1]);
        } else {
          put4<O, kVec>(p, list.splits, done.split, part, m, n, acc[j][i], bias0);
          put4<O, kVec>(p, list.splits, done.split, part, m, n + 16, acc[j + 1][i], bias1);
        }
      }
    }
    cur.kb = cur.tile.kb1 - 1;
    cur.advance(list);
  }
}

// The splits' sums, in order.
template <class O, bool kVec>
__global__ void __launch_bounds__(256) matmul_join_kernel(Fp8Product p, int splits, const float* __restrict__ part) {
  const int quads = (p.N + 3) / 4;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long long)p.M * quads) return;
  const int m = (int)(i / quads), n = (int)(i % quads) * 4;
  floatx4 y = {};
  for (int s = 0; s < splits; ++s) {
    float v[4];
    load_row<float, 4, kVec>(v, part + ((long long)s * p.M + m) * p.N, n, p.N);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] += v[j];
  }
  finish4<O, kVec>(y, bias4<kVec>(p.bias, n, p.N), p.relu, static_cast<O*>(p.out) + (long long)m * p.N, n, p.N);
}

struct Plan {
  int tile;                  // rows of a and of b per workgroup
  int splits, blocks_per_split;
};
Plan plan_matmul(int M, int N, int K, bool fast) {
  Plan pl;
  const int kb = ceil_div(K, kBlock);
  const long long big = (long long)ceil_div(M, 256) * ceil_div(N, 256);
  pl.tile = fast && big >= 192 ? 256 : 128;
  const long long tiles = (long long)ceil_div(M, pl.tile) * ceil_div(N, pl.tile);
  int splits = 1;
  while (tiles * splits < 192 && kb / (splits * 2) >= 4) splits *= 2;
  pl.blocks_per_split = ceil_div(kb, splits);
  pl.splits = ceil_div(kb, pl.blocks_per_split);
  return pl;
}

template <int BM, int BN, int WM, int WN, bool kFast, bool kSquare, class O, bool kVec>
hipError_t run_tiles(const Fp8Product& p, const Plan& pl, float* part, hipStream_t stream) {
  const int tiles_m = ceil_div(p.M, BM), tiles_n = ceil_div(p.N, BN);
  {
    LaunchScope scope(kFast ? "matmul_fast_kernel" : "matmul_exact_kernel", stream);
    const unsigned grid = (unsigned)(tiles_m * tiles_n * pl.splits);
    if constexpr (kFast) {
      const TileList list{tiles_m, tiles_n, pl.splits, pl.blocks_per_split, ceil_div(p.K, kBlock), BM, BN};
      const unsigned most = BM == 256 ? 256 : 512;       // workgroups that the chip holds at a time (by their LDS)
      matmul_fast_kernel<BM, BN, WM, WN, kSquare, O, kVec><<<std::min((grid + 7) / 8 * 8, most), 64 * WM * WN, 0, stream>>>(p, list, part);
    } else
      matmul_exact_kernel<BM, BN, WM, WN, kSquare, O, kVec><<<grid, 64 * WM * WN, 0, stream>>>(
          p, tiles_m, tiles_n, pl.splits, pl.blocks_per_split, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.splits == 1) return e;
  }
  LaunchScope scope("matmul_join_kernel", stream);
  const long long quads = (long long)p.M * ((p.N + 3) / 4);
  matmul_join_kernel<O, kVec><<<(unsigned)((quads + 255) / 256), 256, 0, stream>>>(p, pl.splits, part);
  return hipGetLastError();
}

template <bool kSquare, class O, bool kVec>
hipError_t run_by_tile(const Fp8Product& p, float* part, hipStream_t stream) {
  const Plan pl = plan_matmul(p.M, p.N, p.K, p.fast);
  if (pl.tile == 256) return run_tiles<256, 256, 4, 2, true, kSquare, O, kVec>(p, pl, part, stream);
  return p.fast ? run_tiles<128, 128, 2, 2, true, kSquare, O, kVec>(p, pl, part, stream)
                : run_tiles<128, 128, 2, 2, false, kSquare, O, kVec>(p, pl, part, stream);
}
template <bool kSquare, class O>
hipError_t run_by_alignment(const Fp8Product& p, float* part, hipStream_t stream) {
  return p.N % 4 == 0 ? run_by_tile<kSquare, O, true>(p, part, stream) : run_by_tile<kSquare, O, false>(p, part, stream);
}

}  // namespace

size_t matmul_fp8_workspace_bytes(int M, int N, int K) {
  const int splits = max(plan_matmul(M, N, K, false).splits, plan_matmul(M, N, K, true).splits);
  return splits > 1 ? (size_t)splits * M * N * sizeof(float) : 0;
}

hipError_t launch_matmul_fp8(const Fp8Product& p, void* ws, hipStream_t stream) {
  float* part = static_cast<float*>(ws);
  if (p.out_type == kBF16)
    return p.b_square ? run_by_alignment<true, bf16>(p, part, stream) : run_by_alignment<false, bf16>(p, part, stream);
  return p.b_square ? run_by_alignment<true, float>(p, part, stream) : run_by_alignment<false, float>(p, part, stream);
}

}  // namespace sage
