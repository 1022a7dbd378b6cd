// Embedding lookup with scaling, per token or pooled over ragged prompts, and
// the gradient of the table by sorted tokens.
//
//   out[q] = c sum over the tokens t of prompt q of E[id_t]     (mean: / #valid)
//   dE[v]  = c sum over the tokens t with id_t = v of dout[prompt(t)] (mean: / #valid)
//
// Both are the same work: an ordered list of items, each a source row, in
// consecutive segments (prompts; equal tokens of the sorted list), and a sum
// per segment. The list is cut into chunks of equal length whatever the
// segments, so that one long prompt, or the few tokens that make up most of a
// text, are spread over the chip. A wave walks a chunk, keeps the running sum
// of 16 bytes of columns per lane in fp32, and writes a segment's sum when it
// ends; a segment that crosses chunks leaves one partial sum per chunk, which
// a second kernel adds in order. No atomics on values: results do not depend
// on the order in which waves run.
#include "sage_encode.hpp"
#include "sage_internal.hpp"

namespace sage {
namespace {

constexpr int kTurn = 8;                                 // rows in flight per wave

// ------------------------------------------------------- lookup per token
// Each thread copies pieces of 8 columns; a workgroup owns kRows tokens.
template <class T, class O, bool kAligned>
__global__ void __launch_bounds__(256) embed_tokens_kernel(const int32_t* __restrict__ tokens, int T_, const T* __restrict__ table,
                                                           int V, int d, int rows, float scale, O* __restrict__ out) {
  const int pieces = (d + 7) / 8;
  const int first = blockIdx.x * rows, n = min(rows, T_ - first);
  for (int i = threadIdx.x; i < n * pieces; i += 256) {
    const int r = i / pieces, col = (i - r * pieces) * 8;
    const int id = tokens[first + r];
    float v[8];
    load_row<T, 8, kAligned>(v, table + (long long)((unsigned)id < (unsigned)V ? id : 0) * d,
                             (unsigned)id < (unsigned)V ? col : d, d);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= scale;
    store_row<O, 8, kAligned>(v, out + (long long)(first + r) * d, col, d);
  }
}

// ------------------------------------------------------------ list of items
// Item i of the list: its segment (-1: none), its source row (-1: adds
// nothing, but its segment exists) and its weight.
struct PromptItems {                                     // tokens in order, by prompt
  const int32_t *tokens, *offsets;
  int T, Q, V;
  __device__ __forceinline__ int bag(int i) const {      // last q with offsets[q] <= i
    int lo = 0, hi = Q;                                  // offsets[lo] <= i < offsets[hi], as offsets[0] = 0, offsets[Q] = T
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (offsets[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
  }
  __device__ __forceinline__ bool any(int i) const { return i >= 0 && i < T && i >= offsets[0] && i < offsets[Q]; }
  __device__ __forceinline__ int segment(int i) const { return any(i) ? bag(i) : -1; }
  __device__ __forceinline__ int source(int i) const {
    const int id = tokens[i];
    return (unsigned)id < (unsigned)V ? id : -1;
  }
  __device__ __forceinline__ float weight(int) const { return 1.0f; }
};
struct SortedItems {                                     // token positions or prompts, by token
  const uint32_t *keys, *rows;
  const int32_t* valid;                                  // valid tokens per prompt (mean), or null
  int T, V;
  __device__ __forceinline__ int segment(int i) const {
    if (i < 0 || i >= T) return -1;
    const uint32_t k = keys[i];
    return k < (uint32_t)V ? (int)k : -1;                // tokens that are none sort last, as V
  }
  __device__ __forceinline__ int source(int i) const { return (int)rows[i]; }
  __device__ __forceinline__ float weight(int i) const { return valid ? __fdiv_rn(1.0f, (float)valid[rows[i]]) : 1.0f; }
};

// The columns of a lane: V consecutive ones, or (unaligned rows) every 64th,
// so that neighbouring lanes read neighbouring elements.
template <class T, int V, bool kAligned>
__device__ __forceinline__ void load_cols(float (&v)[V], const T* row, int slice, int d) {
  const int lane = (int)lane_id();
  if constexpr (kAligned) {
    load_row<T, V, true>(v, row, slice * 64 * V + lane * V, d);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (slice * V + j) * 64 + lane;
      v[j] = c < d ? (float)row[c] : 0.0f;
    }
  }
}
template <class T, int V, bool kAligned>
__device__ __forceinline__ void store_cols(const float (&v)[V], T* row, int slice, int d) {
  const int lane = (int)lane_id();
  if constexpr (kAligned) {
    store_row<T, V, true>(v, row, slice * 64 * V + lane * V, d);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int c = (slice * V + j) * 64 + lane;
      if (c < d) row[c] = (T)v[j];
    }
  }
}

// Partial sums: two rows of d fp32 per chunk, [0] of the segment that was open
// when the chunk began, [1] of the one that began in it and goes on after it;
// and their counts of valid items. tail[c] is the segment of [1], or -1.
struct Partials {
  float* sum;
  int32_t* count;
  int32_t* tail;
};
// What a finished sum becomes: (x scale, / count for a mean) + add, rounded.
template <class O>
struct Finish {
  O* out;
  const float* add;                                      // fp32 rows like out, or null
  float scale;
  bool mean;
  int d;
  template <int V, bool kAligned>
  __device__ __forceinline__ void write(const float (&acc)[V], int count, int seg, int slice) const {
    const float c = mean && count > 0 ? __fdiv_rn(scale, (float)count) : scale;
    float v[V];
    if (add) {
      load_cols<float, V, kAligned>(v, add + (long long)seg * d, slice, d);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = fmaf(acc[j], c, v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = acc[j] * c;
    }
    store_cols<O, V, kAligned>(v, out + (long long)seg * d, slice, d);
  }
};

// One wave per (chunk of `chunk` items, slice of 64 V columns); `chunk` is a
// multiple of 64, and lane l holds item l of the 64 in work.
template <class Items, class T, class O, int V, bool kAligned>
__global__ void __launch_bounds__(256) segment_sum_kernel(Items items, const T* __restrict__ src, int d, int slices,
                                                          int chunk, int chunks, Partials part, Finish<O> fin) {
  const int lane = (int)lane_id();
  const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + threadIdx.x / 64));
  const int c = wave / slices, slice = wave % slices;
  if (c >= chunks) return;                               // whole waves, no barrier below
  const int begin = c * chunk;
  int cur = items.segment(begin - 1);                    // the open segment, if the chunk's first items are its
  bool open = true;                                      // whether the running segment began before the chunk
  {
    const int s0 = items.segment(begin);
    if (s0 != cur || s0 < 0) open = false;
    cur = s0;
  }
  float acc[V] = {};
  int count = 0;
  auto flush = [&](bool goes_on) {
    if (cur >= 0) {
      if (open || goes_on) {
        const long long slot = 2LL * c + (open ? 0 : 1);
        store_cols<float, V, kAligned>(acc, part.sum + slot * d, slice, d);
        if (lane == 0 && slice == 0) part.count[slot] = count;
      } else {
        fin.template write<V, kAligned>(acc, count, cur, slice);
      }
    }
  };
  for (int base = begin; base < begin + chunk; base += 64) {
    const int i = base + lane;
    const int seg = items.segment(i);
    const int row = seg >= 0 ? items.source(i) : -1;
    const float wgt = row >= 0 ? items.weight(i) : 0.0f;
    if (__all(seg < 0) && cur < 0) continue;
    for (int j0 = 0; j0 < 64; j0 += kTurn) {
      float v[kTurn][V];
#pragma unroll
      for (int u = 0; u < kTurn; ++u) {
        const int r = __builtin_amdgcn_readlane(row, j0 + u);
        load_cols<T, V, kAligned>(v[u], src + (long long)max(r, 0) * d, slice, d);
      }
#pragma unroll
      for (int u = 0; u < kTurn; ++u) {
        const int s = __builtin_amdgcn_readlane(seg, j0 + u);
        if (s != cur) {
          flush(false);
          cur = s;
          open = false;
          count = 0;
#pragma unroll
          for (int j = 0; j < V; ++j) acc[j] = 0.0f;
        }
        if (__builtin_amdgcn_readlane(row, j0 + u) >= 0) {
          const float x = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(wgt), j0 + u));
          ++count;
#pragma unroll
          for (int j = 0; j < V; ++j) acc[j] = fmaf(v[u][j], x, acc[j]);
        }
      }
    }
  }
  const bool goes_on = cur >= 0 && items.segment(begin + chunk) == cur;
  if (slice == 0 && lane == 0) part.tail[c] = goes_on && !open ? cur : -1;
  flush(goes_on);
}

// The segments that cross chunks: the wave of the chunk where one begins adds
// its partial sums, chunk by chunk. part.tail of a later chunk tells nothing
// about where a segment ends: the items do.
template <class Items, class T, class O, int V, bool kAligned>
__global__ void __launch_bounds__(256) segment_join_kernel(Items items, int d, int slices, int chunk, int chunks,
                                                           Partials part, Finish<O> fin) {
  const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + threadIdx.x / 64));
  const int c = wave / slices, slice = wave % slices;
  if (c >= chunks) return;
  const int seg = part.tail[c];
  if (seg < 0) return;
  float acc[V];
  load_cols<float, V, kAligned>(acc, part.sum + (2LL * c + 1) * d, slice, d);
  int count = part.count[2LL * c + 1];
  for (int k = c + 1; k < chunks && items.segment(k * chunk) == seg; ++k) {
    float v[V];
    load_cols<float, V, kAligned>(v, part.sum + 2LL * k * d, slice, d);
    count += part.count[2LL * k];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] += v[j];
  }
  fin.template write<V, kAligned>(acc, count, seg, slice);
}

// Prompts with no tokens: rows of zeros.
template <class O, int V, bool kAligned>
__global__ void __launch_bounds__(256) empty_prompts_kernel(const int32_t* __restrict__ offsets, int T, int Q, int d,
                                                            int slices, Finish<O> fin) {
  const int q = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + threadIdx.x / 64));
  if (q >= Q) return;
  const int b = max(offsets[q], 0), e = min(offsets[q + 1], T);
  if (b < e) return;
  const float zero[V] = {};
  for (int s = 0; s < slices; ++s) fin.template write<V, kAligned>(zero, 0, q, s);
}

// Tokens that the list does not have: rows of zeros, or of `add`. A wave takes
// 32 rows: lane l finds the first item of token v0 + l by a binary search.
template <int V, bool kAligned>
__global__ void __launch_bounds__(256) missing_tokens_kernel(const uint32_t* __restrict__ keys, int T, int n_rows,
                                                             int d, int slices, Finish<float> fin) {
  constexpr int kTake = 32;
  const int lane = (int)lane_id();
  const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + threadIdx.x / 64));
  const int v0 = wave * kTake;
  if (v0 >= n_rows) return;
  int lo = 0, hi = T;
  const uint32_t want = (uint32_t)min(v0 + min(lane, kTake), n_rows);
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (keys[mid] >= want) hi = mid; else lo = mid + 1;
  }
  const int next = __shfl_down(lo, 1, 64);
  uint64_t missing = __ballot(lane < kTake && v0 + lane < n_rows && lo == next);
  const float zero[V] = {};
  while (missing) {
    const int l = __builtin_ctzll(missing);
    missing &= missing - 1;
    for (int s = 0; s < slices; ++s) fin.template write<V, kAligned>(zero, 0, v0 + l, s);
  }
}

// ------------------------------------------------------------ token sort
// Stable least-significant-digit radix sort of the tokens (as unsigned keys
// below 2^bits; a token outside [0, V) has key V) with the row that each
// brings: its position, or its prompt. Digits of up to 9 bits; each pass
// counts per tile, scans, and scatters, a wave ranking its own quarter of a
// tile with ballots.
constexpr int kSortBits = 9;
constexpr int kSortBins = 1 << kSortBits;
constexpr int kSortThreads = 256;
constexpr int kSortItems = 4;
constexpr int kSortTile = kSortThreads * kSortItems;

// Key of token i: V for one outside the table or (with prompts) in none of them.
__device__ __forceinline__ uint32_t token_key(const PromptItems& p, int i) {
  const int id = p.tokens[i];
  return (unsigned)id < (unsigned)p.V && (!p.offsets || p.any(i)) ? (uint32_t)id : (uint32_t)p.V;
}

// kFirst: the keys come from the tokens, and (mean) each prompt's valid tokens
// are counted: once per wave and prompt, as one prompt may have them all.
template <bool kFirst>
__global__ void __launch_bounds__(kSortThreads) token_count_kernel(PromptItems prompts, const uint32_t* __restrict__ keys,
                                                                   int T, int shift, int tiles,
                                                                   uint32_t* __restrict__ hist, int32_t* __restrict__ valid) {
  __shared__ uint32_t cnt[kSortBins];
  for (int b = threadIdx.x; b < kSortBins; b += kSortThreads) cnt[b] = 0;
  __syncthreads();
#pragma unroll
  for (int it = 0; it < kSortItems; ++it) {
    const int i = blockIdx.x * kSortTile + it * kSortThreads + threadIdx.x;
    uint32_t k = 0;
    if (i < T) {
      k = kFirst ? token_key(prompts, i) : keys[i];
      atomicAdd(&cnt[(k >> shift) & (kSortBins - 1)], 1u);
    }
    if (kFirst && valid) {
      const int q = i < T && k < (uint32_t)prompts.V ? prompts.segment(i) : -1;
      uint64_t left = __ballot(q >= 0);
      while (left) {
        const int q0 = __builtin_amdgcn_readlane(q, __builtin_ctzll(left));
        const uint64_t same = __ballot(q == q0);
        if (lane_id() == 0) atomicAdd(&valid[q0], (int)__popcll(same));
        left &= ~same;
      }
    }
  }
  __syncthreads();
  for (int b = threadIdx.x; b < kSortBins; b += kSortThreads) hist[(size_t)b * tiles + blockIdx.x] = cnt[b];
}

// Exclusive scan over the tiles of each digit; its total goes to total[digit].
__global__ void __launch_bounds__(256) token_scan_kernel(uint32_t* __restrict__ hist, int tiles, uint32_t* __restrict__ total) {
  __shared__ uint32_t wsum[4];
  const int lane = (int)lane_id(), w = threadIdx.x / 64;
  uint32_t* row = hist + (size_t)blockIdx.x * tiles;
  uint32_t carry = 0;
  for (int base = 0; base < tiles; base += 256) {
    const int i = base + threadIdx.x;
    const uint32_t v = i < tiles ? row[i] : 0u;
    uint32_t incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = (uint32_t)__shfl_up((int)incl, o, 64);
      if (lane >= o) incl += y;
    }
    if (lane == 63) wsum[w] = incl;
    __syncthreads();
    uint32_t before = carry;
    for (int i2 = 0; i2 < w; ++i2) before += wsum[i2];
    if (i < tiles) row[i] = before + incl - v;
    carry += wsum[0] + wsum[1] + wsum[2] + wsum[3];
    __syncthreads();
  }
  if (threadIdx.x == 0) total[blockIdx.x] = carry;
}

template <bool kFirst>
__global__ void __launch_bounds__(kSortThreads) token_scatter_kernel(
    PromptItems prompts, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ rows, int T, int shift, int tiles,
    const uint32_t* __restrict__ hist, const uint32_t* __restrict__ total, uint32_t* __restrict__ keys_out, uint32_t* __restrict__ rows_out) {
  constexpr int kWaves = kSortThreads / 64;
  __shared__ uint32_t first_of[kSortBins];
  __shared__ uint32_t wtot[kWaves];
  __shared__ uint32_t cnt[kWaves][kSortBins];
  const int lane = (int)lane_id();
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  const int first = blockIdx.x * kSortTile + w * (kSortItems * 64) + lane;
  uint32_t key[kSortItems], val[kSortItems];
#pragma unroll
  for (int it = 0; it < kSortItems; ++it) {
    const int i = first + it * 64;
    key[it] = i >= T ? 0u : kFirst ? token_key(prompts, i) : keys[i];
    if (i >= T) val[it] = 0u;
    else if (!kFirst) val[it] = rows[i];
    else val[it] = prompts.offsets ? (uint32_t)max(prompts.segment(i), 0) : (uint32_t)i;
  }
  // Exclusive scan of the digit totals, two per thread, plus this tile's offset.
  {
    static_assert(kSortBins == 2 * kSortThreads, "two digits a thread");
    const int b = 2 * threadIdx.x;
    const uint32_t v0 = total[b], v1 = total[b + 1];
    uint32_t incl = v0 + v1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = (uint32_t)__shfl_up((int)incl, o, 64);
      if (lane >= o) incl += y;
    }
    if (lane == 63) wtot[w] = incl;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) cnt[i][b] = cnt[i][b + 1] = 0;
    __syncthreads();
    uint32_t before = 0;
    for (int i = 0; i < w; ++i) before += wtot[i];
    before += incl - v0 - v1;
    first_of[b] = before + hist[(size_t)b * tiles + blockIdx.x];
    first_of[b + 1] = before + v0 + hist[(size_t)(b + 1) * tiles + blockIdx.x];
  }
  const uint64_t below = (1ull << lane) - 1ull;
  uint32_t rank[kSortItems];
#pragma unroll
  for (int it = 0; it < kSortItems; ++it) {
    const bool valid = first + it * 64 < T;
    const uint32_t digit = (key[it] >> shift) & (kSortBins - 1);
    uint64_t peers = __ballot(valid);
#pragma unroll
    for (int bit = 0; bit < kSortBits; ++bit) {
      const bool on = (digit >> bit) & 1u;
      const uint64_t m = __ballot(on);
      peers &= on ? m : ~m;
    }
    const uint32_t seen = cnt[w][digit];                 // LDS operations of a wave complete in order
    rank[it] = seen + (uint32_t)__popcll(peers & below);
    __builtin_amdgcn_wave_barrier();
    if (valid && (peers & below) == 0) cnt[w][digit] = seen + (uint32_t)__popcll(peers);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  for (int b = threadIdx.x; b < kSortBins; b += kSortThreads) {
    uint32_t run = first_of[b];
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const uint32_t c = cnt[i][b];
      cnt[i][b] = run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int it = 0; it < kSortItems; ++it) {
    if (first + it * 64 >= T) continue;
    const uint32_t pos = cnt[w][(key[it] >> shift) & (kSortBins - 1)] + rank[it];
    keys_out[pos] = key[it];
    rows_out[pos] = val[it];
  }
}

__global__ void __launch_bounds__(256) clear_kernel(int32_t* __restrict__ p, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0;
}

// ------------------------------------------------------------------- plans
// Items per chunk: about eight waves per SIMD over all chunks and slices, in
// whole groups of 64.
int chunk_items(int T, int slices) {
  const long long want = (long long)T * slices / 8192;
  return (int)min(1024LL, max(64LL, (want + 63) / 64 * 64));
}
// Slices of 64 lanes x 16 bytes of source columns.
int slice_count(int d, int vec) { return ceil_div(d, 64 * vec); }

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
struct PartialLayout {
  int chunk, chunks;
  size_t sum, count, tail, bytes;
};
// For the narrower slices of fp32 sources, which have the smaller chunks' bound.
PartialLayout partial_layout(int T, int d, int vec) {
  PartialLayout l{};
  l.chunk = chunk_items(T, slice_count(d, vec));
  l.chunks = ceil_div(T, l.chunk);
  l.sum = 0;
  l.count = align256(2ull * l.chunks * d * sizeof(float));
  l.tail = l.count + align256(2ull * l.chunks * sizeof(int32_t));
  l.bytes = l.tail + align256((size_t)l.chunks * sizeof(int32_t));
  return l;
}
size_t partial_bytes(int T, int d) { return max(partial_layout(T, d, 4).bytes, partial_layout(T, d, 8).bytes); }
Partials partials_at(void* ws, const PartialLayout& l) {
  char* p = static_cast<char*>(ws);
  return Partials{reinterpret_cast<float*>(p + l.sum), reinterpret_cast<int32_t*>(p + l.count),
                  reinterpret_cast<int32_t*>(p + l.tail)};
}

template <class Items, class T, class O, int V, bool kAligned>
hipError_t sum_segments(const Items& items, int n, const T* src, int d, void* ws, const Finish<O>& fin,
                        hipStream_t stream) {
  const int slices = slice_count(d, V);
  const PartialLayout l = partial_layout(n, d, V);
  const Partials part = partials_at(ws, l);
  const unsigned grid = (unsigned)(((long long)l.chunks * slices + 3) / 4);
  {
    LaunchScope scope("segment_sum_kernel", stream);
    segment_sum_kernel<Items, T, O, V, kAligned><<<grid, 256, 0, stream>>>(items, src, d, slices, l.chunk, l.chunks, part, fin);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  LaunchScope scope("segment_join_kernel", stream);
  segment_join_kernel<Items, T, O, V, kAligned><<<grid, 256, 0, stream>>>(items, d, slices, l.chunk, l.chunks, part, fin);
  return hipGetLastError();
}

template <class T, class O, bool kAligned>
hipError_t embed_with(const int32_t* tokens, int T_, const void* table, int V, int d, float scale, Prompts p, void* out,
                      void* ws, hipStream_t stream) {
  constexpr int kVec = 16 / sizeof(T);
  const T* src = static_cast<const T*>(table);
  O* dst = static_cast<O*>(out);
  if (!p.offsets) {
    LaunchScope scope("embed_tokens_kernel", stream);
    const int rows = max(1, 2048 / ceil_div(d, 8));      // about eight pieces a thread
    embed_tokens_kernel<T, O, kAligned><<<ceil_div(T_, rows), 256, 0, stream>>>(tokens, T_, src, V, d, rows, scale, dst);
    return hipGetLastError();
  }
  const Finish<O> fin{dst, nullptr, scale, p.mean, d};
  const int slices = slice_count(d, kVec);
  {
    LaunchScope scope("empty_prompts_kernel", stream);
    empty_prompts_kernel<O, kVec, kAligned><<<ceil_div(p.Q, 4), 256, 0, stream>>>(p.offsets, T_, p.Q, d, slices, fin);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || T_ == 0) return e;
  }
  const PromptItems items{tokens, p.offsets, T_, p.Q, V};
  return sum_segments<PromptItems, T, O, kVec, kAligned>(items, T_, src, d, ws, fin, stream);
}

template <class T, class O>
hipError_t embed_by_alignment(const int32_t* tokens, int T_, const void* table, int V, int d, float scale, Prompts p,
                              void* out, void* ws, hipStream_t stream) {
  return d % 8 == 0 ? embed_with<T, O, true>(tokens, T_, table, V, d, scale, p, out, ws, stream)
                    : embed_with<T, O, false>(tokens, T_, table, V, d, scale, p, out, ws, stream);
}

int key_bits(int V) {                                    // keys are 0..V
  int b = 1;
  while (b < 31 && (V >> b) != 0) ++b;
  return b;
}
struct GradLayout {
  int tiles;
  size_t keys[2], rows[2], hist, total, valid, part, bytes;
};
GradLayout grad_layout(int T, int Q, int d) {
  GradLayout l{};
  l.tiles = ceil_div(T, kSortTile);
  size_t at = 0;
  for (int i = 0; i < 2; ++i) {
    l.keys[i] = at;
    at += align256((size_t)T * 4);
    l.rows[i] = at;
    at += align256((size_t)T * 4);
  }
  l.hist = at;
  at += align256((size_t)kSortBins * l.tiles * 4);
  l.total = at;
  at += align256(kSortBins * 4);
  l.valid = at;
  at += align256((size_t)Q * 4);
  l.part = at;
  l.bytes = at + partial_bytes(T, d);
  return l;
}

template <class T, bool kAligned>
hipError_t embed_grad_with(const int32_t* tokens, int T_, const void* grad, int V, int d, float scale, Prompts p,
                           const float* add, float* out, void* ws, hipStream_t stream) {
  constexpr int kVec = 16 / sizeof(T);
  const GradLayout l = grad_layout(T_, p.offsets ? p.Q : 0, d);
  char* base = static_cast<char*>(ws);
  uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(base + l.keys[0]), reinterpret_cast<uint32_t*>(base + l.keys[1])};
  uint32_t* rows[2] = {reinterpret_cast<uint32_t*>(base + l.rows[0]), reinterpret_cast<uint32_t*>(base + l.rows[1])};
  uint32_t* hist = reinterpret_cast<uint32_t*>(base + l.hist);
  uint32_t* total = reinterpret_cast<uint32_t*>(base + l.total);
  int32_t* valid = p.offsets && p.mean ? reinterpret_cast<int32_t*>(base + l.valid) : nullptr;
  const Finish<float> fin{out, add, scale, false, d};
  const int slices = slice_count(d, kVec);
  const PromptItems prompts{tokens, p.offsets, T_, p.Q, V};
  hipError_t e;
  if (valid && T_ > 0) {
    LaunchScope scope("clear_kernel", stream);
    clear_kernel<<<ceil_div(p.Q, 256), 256, 0, stream>>>(valid, p.Q);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  int at = 0;                                            // where the sorted list is
  const int bits = key_bits(V);
  for (int shift = 0; T_ > 0 && shift < bits; shift += kSortBits) {
    const bool first = shift == 0;
    {
      LaunchScope scope("token_count_kernel", stream);
      if (first) token_count_kernel<true><<<l.tiles, kSortThreads, 0, stream>>>(prompts, nullptr, T_, 0, l.tiles, hist, valid);
      else token_count_kernel<false><<<l.tiles, kSortThreads, 0, stream>>>(prompts, keys[at], T_, shift, l.tiles, hist, nullptr);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    {
      LaunchScope scope("token_scan_kernel", stream);
      token_scan_kernel<<<kSortBins, 256, 0, stream>>>(hist, l.tiles, total);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    LaunchScope scope("token_scatter_kernel", stream);
    if (first) {
      token_scatter_kernel<true><<<l.tiles, kSortThreads, 0, stream>>>(prompts, nullptr, nullptr, T_, 0, l.tiles, hist, total,
                                                                       keys[0], rows[0]);
      at = 0;
    } else {
      token_scatter_kernel<false><<<l.tiles, kSortThreads, 0, stream>>>(prompts, keys[at], rows[at], T_, shift, l.tiles, hist,
                                                                        total, keys[at ^ 1], rows[at ^ 1]);
      at ^= 1;
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (add != out) {                                      // in place, rows with no token stay as they are
    LaunchScope scope("missing_tokens_kernel", stream);
    missing_tokens_kernel<kVec, kAligned><<<ceil_div(ceil_div(V, 32), 4), 256, 0, stream>>>(keys[at], T_, V, d, slices, fin);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (T_ == 0) return hipSuccess;
  const SortedItems items{keys[at], rows[at], valid, T_, V};
  return sum_segments<SortedItems, T, float, kVec, kAligned>(items, T_, static_cast<const T*>(grad), d, base + l.part, fin, stream);
}

}  // namespace

size_t embed_workspace_bytes(int T, int Q, int d) { return T > 0 && Q > 0 ? partial_bytes(T, d) : 0; }

hipError_t launch_embed(const int32_t* tokens, int T, const void* table, Type table_type, int V, int d, float scale,
                        Prompts p, void* out, Type out_type, void* ws, hipStream_t stream) {
  if (table_type == kBF16)
    return out_type == kBF16 ? embed_by_alignment<bf16, bf16>(tokens, T, table, V, d, scale, p, out, ws, stream)
                             : embed_by_alignment<bf16, float>(tokens, T, table, V, d, scale, p, out, ws, stream);
  return out_type == kBF16 ? embed_by_alignment<float, bf16>(tokens, T, table, V, d, scale, p, out, ws, stream)
                           : embed_by_alignment<float, float>(tokens, T, table, V, d, scale, p, out, ws, stream);
}

size_t embed_grad_workspace_bytes(int T, int Q, int V, int d) {
  (void)V;
  return T > 0 ? grad_layout(T, Q, d).bytes : 0;
}

hipError_t launch_embed_grad(const int32_t* tokens, int T, const void* grad, Type grad_type, int V, int d, float scale,
                             Prompts p, const float* add, float* out, void* ws, hipStream_t stream) {
  const bool aligned = d % 8 == 0;
  if (grad_type == kBF16)
    return aligned ? embed_grad_with<bf16, true>(tokens, T, grad, V, d, scale, p, add, out, ws, stream)
                   : embed_grad_with<bf16, false>(tokens, T, grad, V, d, scale, p, add, out, ws, stream);
  return aligned ? embed_grad_with<float, true>(tokens, T, grad, V, d, scale, p, add, out, ws, stream)
                 : embed_grad_with<float, false>(tokens, T, grad, V, d, scale, p, add, out, ws, stream);
}

}  // namespace sage
