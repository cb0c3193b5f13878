// Embedding lookup with scaling, and the gradient of its table.
//
//   out_t = scale table[id_t],      dtable[v] = scale sum over the tokens t with id_t = v of dout_t   (every row v, in 32 bits, in
//   the order of the tokens)
//
// Both are bound by memory.  The gradient needs the tokens of a row together: (id, token) pairs are sorted, blocks of SORT_BLOCK
// in shared memory, then merged by counting, for each pair, the smaller ones in the other sorted blocks.  A row's
// sum is one warp's, 256 columns at a time, when it has up to HOT tokens.  Longer runs are cut at every HOT-th place of the
// sorted order, each piece summed by a warp of its own into scratch, and a last kernel adds the pieces in order: so a token that
// fills half of the batch does not hold up a single warp, and the sums do not depend on which warp runs first.
#include "internal.h"

namespace muloco {

namespace {

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32(float x) { return x; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16(x); }

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int SLICE = 256;                     // columns that a warp works on at a time, 8 a lane
constexpr int HOT = EMB_CHUNK;

// 8 entries of a slice in a lane: neighbours in 16-byte accesses (WIDE), or every 32nd.
template <typename T> struct alignas(16) Vec16 { T v[16 / sizeof(T)]; };

template <typename T, bool WIDE>
__device__ __forceinline__ void load8(float (&f)[8], const T* p, int col, int d, int lane) {
  if (WIDE) {
    constexpr int V = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8; i += V) {
      Vec16<T> x;
      if (col + lane * 8 < d) x = *reinterpret_cast<const Vec16<T>*>(p + col + lane * 8 + i);
#pragma unroll
      for (int k = 0; k < V; ++k) f[i + k] = col + lane * 8 < d ? to_f32(x.v[k]) : 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = col + i * 32 + lane < d ? to_f32(p[col + i * 32 + lane]) : 0.f;
  }
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store8(const float (&f)[8], T* p, int col, int d, int lane) {
  if (WIDE) {
    constexpr int V = 16 / sizeof(T);
    if (col + lane * 8 >= d) return;
#pragma unroll
    for (int i = 0; i < 8; i += V) {
      Vec16<T> x;
#pragma unroll
      for (int k = 0; k < V; ++k) x.v[k] = from_f32<T>(f[i + k]);
      *reinterpret_cast<Vec16<T>*>(p + col + lane * 8 + i) = x;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i * 32 + lane < d) p[col + i * 32 + lane] = from_f32<T>(f[i]);
  }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(THREADS)
embedding_kernel(const EmbeddingArgs a) {
  const int lane = threadIdx.x & 31;
  const int slices = (a.d + SLICE - 1) / SLICE;
  const int64_t unit = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
  grid_wait();
  grid_release();
  const int64_t token = unit / slices;
  if (token >= a.tokens) return;
  const int col = (int)(unit - token * slices) * SLICE;
  const int64_t id = a.ids[token];
  const bool ok = id >= 0 && id < a.rows;
  float f[8];
  if (ok) {
    load8<T, WIDE>(f, reinterpret_cast<const T*>(a.table) + id * a.ld, col, a.d, lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= a.scale;
  } else {
    if (lane == 0) atomicOr(a.status, ST_TOKEN);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __int_as_float(0x7fffffff);
  }
  store8<T, WIDE>(f, reinterpret_cast<T*>(a.out) + token * a.d, col, a.d, lane);
}

// ----------------------------- sorted tokens ---------------------------------
// A pair as one number, id above token; ids outside the table sort behind all others and are reported.
__device__ __forceinline__ uint64_t pair_of(const EmbeddingArgs& a, int64_t t) {
  const int64_t id = a.ids[t];
  const bool ok = id >= 0 && id < a.rows;
  if (!ok) atomicOr(a.status, ST_TOKEN);
  return ((uint64_t)(ok ? id : a.rows) << 32) | (uint64_t)t;
}

constexpr int SORT_THREADS = 1024;
static_assert(EMB_SORT_BLOCK == 2 * SORT_THREADS, "two pairs per thread");

__global__ void __launch_bounds__(SORT_THREADS)
sort_kernel(const EmbeddingArgs a, uint64_t* out) {
  __shared__ uint64_t s[EMB_SORT_BLOCK];
  grid_wait();
  grid_release();
  const int64_t first = (int64_t)blockIdx.x * EMB_SORT_BLOCK;
  const int n = (int)(a.tokens - first < EMB_SORT_BLOCK ? a.tokens - first : EMB_SORT_BLOCK);
  int size = 64;                               // power of two that holds the block's pairs
  while (size < n) size <<= 1;
  for (int i = threadIdx.x; i < size; i += SORT_THREADS) s[i] = i < n ? pair_of(a, first + i) : ~0ull;
  __syncthreads();
  // bitonic sorting network
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j; j >>= 1) {
      const int i = 2 * threadIdx.x - (threadIdx.x & (j - 1));
      if (i < size) {
        const uint64_t x = s[i], y = s[i + j];
        if ((x > y) == ((i & k) == 0)) { s[i] = y; s[i + j] = x; }
      }
      __syncthreads();
    }
  for (int i = threadIdx.x; i < n; i += SORT_THREADS) out[first + i] = s[i];
}

// How many of the n sorted pairs are below x.
__device__ __forceinline__ int64_t below(const uint64_t* p, int64_t n, uint64_t x) {
  int64_t lo = 0;
  while (n > 0) {
    const int64_t half = n >> 1;
    if (p[lo + half] < x) { lo += half + 1; n -= half + 1; } else n = half;
  }
  return lo;
}

// Merges groups of EMB_MERGE sorted blocks of `block` pairs: a pair's place is the count of smaller ones (no two are equal).
__global__ void __launch_bounds__(THREADS)
merge_kernel(const uint64_t* in, uint64_t* out, int64_t tokens, int64_t block) {
  grid_wait();
  grid_release();
  const int64_t t = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (t >= tokens) return;
  const uint64_t x = in[t];
  const int64_t first = t / (block * EMB_MERGE) * (block * EMB_MERGE), own = (t - first) / block;
  int64_t place = first + (t - first) % block;
#pragma unroll 4
  for (int b = 0; b < EMB_MERGE; ++b) {
    const int64_t at = first + b * block;
    if (b == own || at >= tokens) continue;
    place += below(in + at, tokens - at < block ? tokens - at : block, x);
  }
  out[place] = x;
}

__device__ __forceinline__ uint32_t token_of(uint64_t x) { return (uint32_t)x; }
__device__ __forceinline__ int64_t id_of(uint64_t x) { return (int64_t)(x >> 32); }

// Sum of the gradients of pairs [from, to), 8 columns a lane.
template <typename T, bool WIDE>
__device__ __forceinline__ void sum_rows(float (&f)[8], const EmbeddingArgs& a, const uint64_t* pairs, int64_t from, int64_t to, int col,
                                         int lane) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = 0.f;
#pragma unroll 4
  for (int64_t i = from; i < to; ++i) {
    float g[8];
    load8<T, WIDE>(g, reinterpret_cast<const T*>(a.dout) + (int64_t)token_of(pairs[i]) * a.ld, col, a.d, lane);
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] += g[k];
  }
}

// Rows of the gradient (blocks 0 .. row_blocks - 1, a warp has 32 rows of a slice), pieces of long runs (the others).
template <typename T, typename O, bool WIDE>
__global__ void __launch_bounds__(THREADS)
gather_kernel(const EmbeddingArgs a, const uint64_t* pairs, int64_t row_blocks) {
  const int lane = threadIdx.x & 31;
  const int slices = (a.d + SLICE - 1) / SLICE;
  grid_wait();
  grid_release();
  if (blockIdx.x < row_blocks) {
    const int64_t unit = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5);
    const int64_t first = unit / slices * 32;
    if (first >= a.rows) return;
    const int col = (int)(unit % slices) * SLICE;
    const int64_t start = below(pairs, a.tokens, (uint64_t)(first + lane) << 32);
    int64_t end = __shfl_down_sync(0xffffffffu, start, 1);
    if (lane == 31) end = below(pairs, a.tokens, (uint64_t)(first + 32) << 32);
    const int n = (int)(a.rows - first < 32 ? a.rows - first : 32);
    for (int r = 0; r < n; ++r) {
      const int64_t from = __shfl_sync(0xffffffffu, start, r), to = __shfl_sync(0xffffffffu, end, r);
      if (to - from > HOT) continue;           // its pieces are summed below
      float f[8];
      sum_rows<T, WIDE>(f, a, pairs, from, to, col, lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= a.scale;
      store8<O, WIDE>(f, reinterpret_cast<O*>(a.dtable) + (first + r) * a.d, col, a.d, lane);
    }
    return;
  }
  const int64_t unit = (blockIdx.x - row_blocks) * WARPS + (threadIdx.x >> 5);
  const int64_t chunk = unit / slices, begin = chunk * HOT;
  if (begin >= a.tokens) return;
  const int col = (int)(unit % slices) * SLICE;
  const int64_t stop = begin + HOT < a.tokens ? begin + HOT : a.tokens;
  const int64_t id0 = id_of(pairs[begin]), id1 = id_of(pairs[stop - 1]);
  // lane 0, 1: start and end of the run of the first pair; lane 2, 3: of the last one's
  const int64_t at = below(pairs, a.tokens, (uint64_t)((lane < 2 ? id0 : id1) + (lane & 1)) << 32);
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int64_t from = __shfl_sync(0xffffffffu, at, 2 * w), to = __shfl_sync(0xffffffffu, at, 2 * w + 1);
    const int64_t id = w ? id1 : id0;
    if (to - from <= HOT || id >= a.rows || (w && id1 == id0)) continue;
    float f[8];
    sum_rows<T, WIDE>(f, a, pairs, from > begin ? from : begin, to < stop ? to : stop, col, lane);
    store8<float, WIDE>(f, a.partials + (chunk * 2 + w) * a.d_pad, col, a.d, lane);
  }
}

// Long runs: the block of the chunk in which one starts adds its pieces, each warp a share of them, then the warps' sums.
template <typename O, bool WIDE>
__global__ void __launch_bounds__(THREADS)
join_kernel(const EmbeddingArgs a, const uint64_t* pairs) {
  __shared__ float sums[WARPS][SLICE];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slices = (a.d + SLICE - 1) / SLICE;
  grid_wait();
  grid_release();
  const int64_t chunk = blockIdx.x / slices, begin = chunk * HOT;
  const int col = (int)(blockIdx.x % slices) * SLICE;
  const int64_t stop = begin + HOT < a.tokens ? begin + HOT : a.tokens;
  // a long run that starts in this chunk is its first run or its last
  const int64_t id0 = id_of(pairs[begin]), id1 = id_of(pairs[stop - 1]);
#pragma unroll 1
  for (int w = 0; w < 2; ++w) {
    const int64_t id = w ? id1 : id0;
    if ((w && id1 == id0) || id >= a.rows) continue;
    if (!w && begin > 0 && id_of(pairs[begin - 1]) == id) continue;      // started before
    // too short to be a long one: it ends in this chunk, or HOT places behind its start is another
    if (!w && (id1 != id0 || stop == a.tokens)) continue;
    if (w && (stop == a.tokens || id_of(pairs[stop]) != id)) continue;
    const int64_t at = below(pairs, a.tokens, (uint64_t)(id + (lane & 1)) << 32);
    const int64_t from = __shfl_sync(0xffffffffu, at, 0), to = __shfl_sync(0xffffffffu, at, 1);
    if (to - from <= HOT) continue;
    const int64_t last = (to - 1) / HOT, n = last - chunk + 1;           // pieces
    const int64_t p0 = n * warp / WARPS, p1 = n * (warp + 1) / WARPS;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
#pragma unroll 4
    for (int64_t p = p0; p < p1; ++p) {
      // the piece in the run's own first chunk is that chunk's first or last run, every other one its chunk's first
      float g[8];
      load8<float, WIDE>(g, a.partials + ((chunk + p) * 2 + (p == 0 ? w : 0)) * a.d_pad, col, a.d, lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] += g[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[warp][i * 32 + lane] = f[i];
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) s += sums[k][i * 32 + lane];
        f[i] = s * a.scale;
      }
      store8<O, WIDE>(f, reinterpret_cast<O*>(a.dtable) + id * a.d, col, a.d, lane);
    }
  }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <typename T, typename O, bool WIDE>
cudaError_t gather(cudaStream_t st, const EmbeddingArgs& a, const uint64_t* pairs, int* launches) {
  const int64_t slices = (a.d + SLICE - 1) / SLICE;
  const int64_t row_blocks = ((a.rows + 31) / 32 * slices + WARPS - 1) / WARPS;
  // (up to HOT tokens no run is long)
  const int64_t chunks = a.tokens > HOT ? (a.tokens + HOT - 1) / HOT : 0;
  const int64_t piece_blocks = (chunks * slices + WARPS - 1) / WARPS;
  ++*launches;
  cudaError_t e = launch_dependent(gather_kernel<T, O, WIDE>, (unsigned)(row_blocks + piece_blocks), THREADS, 0, st, a, pairs, row_blocks);
  if (e != cudaSuccess || !chunks) return e;
  ++*launches;
  return launch_dependent(join_kernel<O, WIDE>, (unsigned)(chunks * slices), THREADS, 0, st, a, pairs);
}

template <typename T, typename O>
cudaError_t gather(cudaStream_t st, const EmbeddingArgs& a, const uint64_t* pairs, int* launches) {
  const bool wide = a.d % 8 == 0 && a.ld % 8 == 0 && aligned16(a.dout) && aligned16(a.dtable);
  return wide ? gather<T, O, true>(st, a, pairs, launches) : gather<T, O, false>(st, a, pairs, launches);
}

}  // namespace

cudaError_t launch_embedding(cudaStream_t st, const EmbeddingArgs& a, int is_bf16) {
  const int64_t units = a.tokens * ((a.d + SLICE - 1) / SLICE);
  const unsigned blocks = (unsigned)((units + WARPS - 1) / WARPS);
  const bool wide = a.d % 8 == 0 && a.ld % 8 == 0 && aligned16(a.table) && aligned16(a.out);
  if (is_bf16)
    return wide ? launch_dependent(embedding_kernel<__nv_bfloat16, true>, blocks, THREADS, 0, st, a)
                : launch_dependent(embedding_kernel<__nv_bfloat16, false>, blocks, THREADS, 0, st, a);
  return wide ? launch_dependent(embedding_kernel<float, true>, blocks, THREADS, 0, st, a)
              : launch_dependent(embedding_kernel<float, false>, blocks, THREADS, 0, st, a);
}

size_t embedding_scratch(int64_t tokens, int64_t d) {
  const size_t pairs = (size_t)((tokens + 1) / 2 * 2) * 8;               // (a multiple of 16 bytes)
  return 2 * pairs + (size_t)((tokens + HOT - 1) / HOT) * 2 * (size_t)((d + 3) / 4 * 4) * 4;
}

cudaError_t launch_embedding_backward(cudaStream_t st, const EmbeddingArgs& args, int in_bf16, int out_bf16, int* launches) {
  EmbeddingArgs a = args;
  const size_t pairs_bytes = (size_t)((a.tokens + 1) / 2 * 2) * 8;
  uint64_t* pairs = static_cast<uint64_t*>(a.scratch);
  uint64_t* other = reinterpret_cast<uint64_t*>(static_cast<char*>(a.scratch) + pairs_bytes);
  a.partials = reinterpret_cast<float*>(static_cast<char*>(a.scratch) + 2 * pairs_bytes);
  a.d_pad = (a.d + 3) / 4 * 4;
  cudaError_t e = launch_dependent(sort_kernel, (unsigned)((a.tokens + EMB_SORT_BLOCK - 1) / EMB_SORT_BLOCK), SORT_THREADS, 0, st, a, pairs);
  ++*launches;
  for (int64_t block = EMB_SORT_BLOCK; e == cudaSuccess && block < a.tokens; block *= EMB_MERGE) {
    e = launch_dependent(merge_kernel, (unsigned)((a.tokens + THREADS - 1) / THREADS), THREADS, 0, st, (const uint64_t*)pairs, other, a.tokens, block);
    ++*launches;
    uint64_t* t = pairs;
    pairs = other;
    other = t;
  }
  if (e != cudaSuccess) return e;
  const uint64_t* p = pairs;
  if (in_bf16) return out_bf16 ? gather<__nv_bfloat16, __nv_bfloat16>(st, a, p, launches) : gather<__nv_bfloat16, float>(st, a, p, launches);
  return out_bf16 ? gather<float, __nv_bfloat16>(st, a, p, launches) : gather<float, float>(st, a, p, launches);
}

}  // namespace muloco
