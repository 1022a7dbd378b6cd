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
//  * fast: 2 v_mfma_f32_32x32x64_f8f6f4 on the bytes themselves, twice the
//    rate. That instruction (like the other 8-bit ones) adds its products in
//    groups of 8 with about 13 bits below the largest of the group (measured:
//    2^16 + 2^3 is kept, 2^16 + 2^2 is not; between groups sums are fp32), so
//    a result is off by about 1.4e-5 of its size on normal data: a hundredth
//    of a bf16 output's rounding, but not fp32. The caller asks for it.
//
// Tiles of a and b pass through LDS, 128 bytes a row and block, loaded past the
// registers; the 16-byte chunk c of row r sits at position c ^ (r / 2 % 8), so
// that 16 lanes reading one chunk of 16 rows meet every bank once.
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

// LDS[m0 + size * lane] = `size` bytes at base + off; completion is tracked with wait_loads.
__device__ __forceinline__ void load16_to_lds(const void* base, uint32_t off, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(off), "s"(base), "s"(m0) : "memory", "m0");
}
__device__ __forceinline__ void load4_to_lds(const void* base, uint32_t off, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" :: "v"(off), "s"(base), "s"(m0) : "memory", "m0");
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
__device__ __forceinline__ floatx16 mfma_e4m3(intx4 a0, intx4 a1, intx4 b0, intx4 b1, floatx16 c) {
  const intx8 a = __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7), b = __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

// Bias, ReLU (a NaN stays one) and the store of 4 neighbouring outputs of a row.
template <class O, bool kVec>
__device__ __forceinline__ void finish4(floatx4 y, const float* __restrict__ bias, bool relu, O* row, int n, int N) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (bias && n + j < N) y[j] += bias[n + j];
    if (relu) y[j] = y[j] < 0.0f ? 0.0f : y[j];
  }
  const float v[4] = {y[0], y[1], y[2], y[3]};
  store_row<O, 4, kVec>(v, row, n, N);
}

// One tile of BM rows of a x BN rows of b, over blocks [kb0, kb1) of the summed
// axis. WM x WN waves.
template <int BM, int BN, int WM, int WN, bool kFast, bool kSquare, class O, bool kVec>
__global__ void __launch_bounds__(64 * WM * WN) matmul_fp8_kernel(Fp8Product p, int tiles_m, int tiles_n, int splits,
                                                                  int blocks_per_split, float* __restrict__ part) {
  constexpr int kWaves = WM * WN;
  constexpr int kTileBytes = (BM + BN) * kBlock;
  constexpr int kStageBytes = kTileBytes + (BM + BN) * 4;
  constexpr int kPieces = (BM + BN) / 8 / kWaves;        // 8 rows x 128 bytes per load and wave
  constexpr int MT = BM / WM / 32, NT = BN / WN / 32;    // 32 x 32 tiles of a wave
  static_assert((BM + BN) / 64 == kWaves && BM % 64 == 0, "64 scales a wave");
  static_assert(BN / WN <= kBlock, "a wave's columns share a square block's scale");
  __shared__ __attribute__((aligned(16))) char lds[2 * kStageBytes];   // the only one: its byte offsets are LDS addresses
  const int lane = (int)lane_id();
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  const int wm = w % WM, wn = w / WM;

  // Workgroup b runs on XCD b % 8: each XCD takes a run of tiles, n fastest, so
  // that its L2 holds a few rows of tiles of a and all of b.
  const int total = tiles_m * tiles_n * splits;
  int t = blockIdx.x;
  {
    const int per = total / 8, x = t % 8;
    if (t < per * 8) t = x * per + t / 8;
  }
  const int split = t % splits;
  t /= splits;
  const int m0 = t / tiles_n * BM, n0 = t % tiles_n * BN;
  const int kblocks = (p.K + kBlock - 1) / kBlock;
  const int kb0 = split * blocks_per_split, kb1 = min(kblocks, kb0 + blocks_per_split);

  // This lane's source of each piece: row and chunk of a or b (rows past the
  // end read the last one; their products are not stored).
  const char* const a_base = reinterpret_cast<const char*>(p.a) + (long long)m0 * p.K;
  const char* const b_base = reinterpret_cast<const char*>(p.b) + (long long)n0 * p.K;
  uint32_t off[kPieces];
  int chunk[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int r = (i * kWaves + w) * 8 + lane / 8;       // row of the tile, a's first
    const bool of_a = r < BM;
    const int row = of_a ? min(r, p.M - 1 - m0) : min(r - BM, p.N - 1 - n0);
    chunk[i] = (lane % 8) ^ swz(r);
    off[i] = (uint32_t)row * (uint32_t)p.K + (uint32_t)chunk[i] * 16u;
  }
  const int tail_chunks = p.K % kBlock / 16;             // chunks of the last block, 0: all 8
  auto load_stage = [&](int kb, int st) {
    const char* const ak = a_base + (long long)kb * kBlock;
    const char* const bk = b_base + (long long)kb * kBlock;
    const bool tail = tail_chunks != 0 && kb == kblocks - 1;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int r0 = (i * kWaves + w) * 8;
      const uint32_t to = (uint32_t)(st * kStageBytes + r0 * kBlock);
      if (!tail || chunk[i] < tail_chunks) load16_to_lds(r0 < BM ? ak : bk, off[i], to);
      else *reinterpret_cast<intx4*>(lds + to + lane * 16) = intx4{};
    }
    {                                                    // the block's scales, 64 a wave
      const int r = w * 64 + lane;
      const bool of_a = w * 64 < BM;
      const int n = min(n0 + r - BM, p.N - 1);
      const float* src = of_a ? p.a_scales + (long long)kb * p.M
                              : p.b_scales + (long long)kb * (kSquare ? (p.N + kBlock - 1) / kBlock : p.N);
      const uint32_t at = of_a ? (uint32_t)min(m0 + r, p.M - 1) : (uint32_t)(kSquare ? n / kBlock : n);
      load4_to_lds(src, at * 4u, (uint32_t)(st * kStageBytes + kTileBytes + w * 256));
    }
  };

  const int l32 = lane & 31, half = lane >> 5;
  floatx16 acc[NT][MT] = {};
  // Chunk 2 t + half of row r: with the same choice for a and b, the lanes of a
  // half hold the same k.
  auto piece = [&](const char* stage, int r, int t) {
    return *reinterpret_cast<const intx4*>(stage + r * kBlock + (((2 * t + half) ^ swz(r)) * 16));
  };
  if (kb0 < kb1) load_stage(kb0, 0);
  for (int kb = kb0; kb < kb1; ++kb) {
    const int st = (kb - kb0) & 1;
    wait_all_loads();
    barrier();                                           // this stage has landed; the other one is free
    if (kb + 1 < kb1) load_stage(kb + 1, st ^ 1);
    const char* const stage = lds + st * kStageBytes;
    const float* const sc = reinterpret_cast<const float*>(stage + kTileBytes);
    float sa[MT];
    intx4 fa[kFast ? MT : 1][4];
    Operands wa[kFast ? 1 : MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int r = (wm * MT + i) * 32 + l32;
      sa[i] = sc[r];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if constexpr (kFast) fa[i][t] = piece(stage, r, t);
        else wa[i][t] = to_bf16(piece(stage, r, t));
      }
    }
    if constexpr (kSquare) {
      const float sb = sc[BM + wn * NT * 32];
#pragma unroll
      for (int i = 0; i < MT; ++i) sa[i] *= sb;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int r = BM + (wn * NT + j) * 32 + l32;
      intx4 fb[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) fb[t] = piece(stage, r, t);
      floatx16 y[MT] = {};
      if constexpr (kFast) {
#pragma unroll
        for (int t = 0; t < 4; t += 2)
#pragma unroll
          for (int i = 0; i < MT; ++i) y[i] = mfma_e4m3(fb[t], fb[t + 1], fa[i][t], fa[i][t + 1], y[i]);
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const Operands wb = to_bf16(fb[t]);
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < MT; ++i)
              y[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb.v[k], wa[i][t].v[k], y[i], 0, 0, 0);
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        floatx4 sb;
        if constexpr (!kSquare)
          sb = *reinterpret_cast<const floatx4*>(sc + BM + (wn * NT + j) * 32 + q * 8 + half * 4);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[j][i][4 * q + e] = fmaf(y[i][4 * q + e], kSquare ? sa[i] : sa[i] * sb[e], acc[j][i][4 * q + e]);
      }
    }
  }

#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = m0 + (wm * MT + i) * 32 + l32;
    if (m >= p.M) continue;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + (wn * NT + j) * 32 + q * 8 + half * 4;
        if (n >= p.N) continue;
        const floatx4 v = {acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]};
        if (splits > 1) finish4<float, kVec>(v, nullptr, false, part + ((long long)split * p.M + m) * p.N, n, p.N);
        else finish4<O, kVec>(v, p.bias, p.relu, static_cast<O*>(p.out) + (long long)m * p.N, n, p.N);
      }
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
  finish4<O, kVec>(y, p.bias, p.relu, static_cast<O*>(p.out) + (long long)m * p.N, n, p.N);
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
    LaunchScope scope("matmul_fp8_kernel", stream);
    matmul_fp8_kernel<BM, BN, WM, WN, kFast, kSquare, O, kVec><<<(unsigned)(tiles_m * tiles_n * pl.splits), 64 * WM * WN, 0, stream>>>(
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
