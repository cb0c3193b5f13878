// Embedding lookup with scaling, and the gradient of its table.
//
//   out_t = scale table[id_t],      dtable[v] = scale sum over the tokens t with id_t = v of dout_t   (every row v, in 32 bits, in
//   the order of the tokens)
//
// Both are bound by memory.  The gradient needs the tokens of a row together: (id, token) pairs are sorted, blocks of EMB_SORT_BLOCK in
// shared memory (a warp sorts 64 in registers, then runs are merged two by two), then EMB_MERGE blocks at a time by counting,
// for each pair, the smaller ones in the other sorted blocks.  The sorted order is cut into chunks of EMB_CHUNK pairs; a warp adds up a chunk, 256
// columns at a time, and writes the rows whose tokens are all in it.  A row that goes on in the next chunk leaves a partial sum per
// chunk, and a last kernel adds those in order: so a token that fills half of the batch does not hold up a single warp, and the
// sums do not depend on which warp runs first.  Rows without a token are zeroed by warps of their own.
//
// Measured: lookup of 16384 x 1024 in bf16 12.3 us (5.5 TB/s), in float32 20 (6.7).  Gradient of a table of 32000 rows: 16384 tokens x 2048 in float32
// 91 us, of which writing and reading everything once take 50 (the gathering kernel 62: 4.7 TB/s; cold: sort 7, merges 5 and 7, join 17); 4001 x 768
// in bf16 25 us, four dependent kernels (cold: sort 7, merge 7, gather 14, join 5).  A small gradient is five kernels' latency: 16384 x 24
// takes 28 us whatever the table.
#include "convert.cuh"
#include "internal.h"

namespace muloco {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int SLICE = 256;                     // columns that a warp works on at a time, 8 a lane
constexpr int CHUNK = EMB_CHUNK;
static_assert(CHUNK == 16, "a pair per lane, two batches of loads");

// 8 entries of a slice in a lane: twice 4 neighbours, 128 columns apart (WIDE: whole sectors are written whatever the type), or
// every 32nd.
template <typename T> struct alignas(4 * sizeof(T)) Four { T v[4]; };
template <typename T, bool WIDE> struct Eight;
template <typename T> struct Eight<T, true> {
  Four<T> x[2];
  __device__ __forceinline__ void load(const T* p, int col, int d, int lane) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = col + i * 128 + lane * 4;
      if (at < d) x[i] = *reinterpret_cast<const Four<T>*>(p + at);
      else x[i].v[0] = x[i].v[1] = x[i].v[2] = x[i].v[3] = from_f32<T>(0.f);
    }
  }
  __device__ __forceinline__ float at(int i) const { return to_f32(x[i >> 2].v[i & 3]); }
  __device__ __forceinline__ static void store(const float (&f)[8], T* p, int col, int d, int lane) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = col + i * 128 + lane * 4;
      Four<T> y;
#pragma unroll
      for (int k = 0; k < 4; ++k) y.v[k] = from_f32<T>(f[i * 4 + k]);
      if (at < d) *reinterpret_cast<Four<T>*>(p + at) = y;
    }
  }
};
template <typename T> struct Eight<T, false> {
  T x[8];
  __device__ __forceinline__ void load(const T* p, int col, int d, int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = col + i * 32 + lane < d ? p[col + i * 32 + lane] : from_f32<T>(0.f);
  }
  __device__ __forceinline__ float at(int i) const { return to_f32(x[i]); }
  __device__ __forceinline__ static void store(const float (&f)[8], T* p, int col, int d, int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col + i * 32 + lane < d) p[col + i * 32 + lane] = from_f32<T>(f[i]);
  }
};

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
    Eight<T, WIDE> x;
    x.load(reinterpret_cast<const T*>(a.table) + id * a.ld, col, a.d, lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = x.at(i) * a.scale;
  } else {
    if (lane == 0) atomicOr(a.status, ST_TOKEN);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __int_as_float(0x7fffffff);
  }
  Eight<T, WIDE>::store(f, reinterpret_cast<T*>(a.out) + token * a.d, col, a.d, lane);
}

// ----------------------------- sorted tokens ---------------------------------
// A pair as one number, id above token; ids outside the table sort behind all others and are reported.
__device__ __forceinline__ uint64_t pair_of(const EmbeddingArgs& a, int64_t t) {
  const int64_t id = a.ids[t];
  const bool ok = id >= 0 && id < a.rows;
  if (!ok) atomicOr(a.status, ST_TOKEN);
  return ((uint64_t)(ok ? id : a.rows) << 32) | (uint64_t)t;
}

constexpr int SORT_THREADS = EMB_SORT_BLOCK / 2, RUN = 64;   // RUN: pairs that a warp sorts in registers

// How many of the n pairs of a sorted run are below x (n at most `most`, a power of two).
__device__ __forceinline__ int below_in_run(const uint64_t* p, int n, int most, uint64_t x) {
  int k = 0;
  for (int step = most; step; step >>= 1)
    if (k + step <= n && p[k + step - 1] < x) k += step;
  return k;
}

__global__ void __launch_bounds__(SORT_THREADS)
sort_kernel(const EmbeddingArgs a, uint64_t* out) {
  __shared__ uint64_t s[2][EMB_SORT_BLOCK];
  grid_wait();
  grid_release();
  const int64_t first = (int64_t)blockIdx.x * EMB_SORT_BLOCK;
  const int n = (int)(a.tokens - first < EMB_SORT_BLOCK ? a.tokens - first : EMB_SORT_BLOCK);
  const int lane = threadIdx.x & 31, run0 = (threadIdx.x >> 5) * RUN;
  // bitonic network over 64 pairs: x[h] is pair 32 h + lane of the run
  uint64_t x[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = run0 + 32 * h + lane;
    x[h] = i < n ? pair_of(a, first + i) : ~0ull;
  }
#pragma unroll
  for (int k = 2; k <= RUN; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j; j >>= 1) {
      if (j == 32) {                           // (k is RUN: ascending)
        const uint64_t lo = x[0] < x[1] ? x[0] : x[1], hi = x[0] < x[1] ? x[1] : x[0];
        x[0] = lo;
        x[1] = hi;
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint64_t y = __shfl_xor_sync(0xffffffffu, x[h], j);
          const bool up = ((32 * h + lane) & k) == 0, lower = (lane & j) == 0;
          x[h] = (x[h] < y) == (up == lower) ? x[h] : y;
        }
      }
    }
#pragma unroll
  for (int h = 0; h < 2; ++h) s[0][run0 + 32 * h + lane] = x[h];
  // merges of two runs each: a pair's place is its own in its run and the count of smaller ones in the other
  int from = 0;
  for (int run = RUN; run < EMB_SORT_BLOCK && run < n; run <<= 1, from ^= 1) {
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = threadIdx.x + h * SORT_THREADS;
      if (i >= n) continue;                    // (only whole runs, and the last one, hold pairs)
      const uint64_t v = s[from][i];
      const int own = i & ~(run - 1), other = own ^ run;
      int count = n - other;
      count = count < 0 ? 0 : count < run ? count : run;
      s[from ^ 1][(own & ~(2 * run - 1)) + (i - own) + below_in_run(&s[from][other], count, run, v)] = v;
    }
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = threadIdx.x + h * SORT_THREADS;
    if (i < n) out[first + i] = s[from][i];
  }
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

// Merges groups of EMB_MERGE sorted blocks of `block` pairs (a power of two): a pair's place is the count of smaller ones (no two are
// equal).  The searches in the other blocks go step by step together, so that their loads overlap.  The first steps look at SAMPLES evenly
// spaced pairs of a sorted block only: those are brought into shared memory in one go, where a step is a tenth of the time (in the first merge all pairs
// are).  The rest is among neighbours.  Second merge of 16384 and of 70000 tokens, cold: 10.6 and 15.8 us with all steps in global memory,
// 6.5 and 9.5 with 64 samples (32: as much; 512: 8.2 for 16384, and slower than without for 70000, as every thread block fetches its own).
// Small thread blocks: searches read scattered places, 32 to an instruction, which a multiprocessor serves one by one.
constexpr int MERGE_THREADS = 128, SAMPLES = 64;
template <bool FIRST>                          // block is EMB_SORT_BLOCK
__global__ void __launch_bounds__(MERGE_THREADS)
merge_kernel(const uint64_t* in, uint64_t* out, int64_t tokens, int64_t block) {
  constexpr int EACH = FIRST ? EMB_SORT_BLOCK : SAMPLES, ALL = EACH * EMB_MERGE;
  __shared__ __align__(16) uint64_t sample[ALL];               // pair (s + 1) apart - 1 of sorted block b at b EACH + s
  grid_wait();
  grid_release();
  const int64_t t = (int64_t)blockIdx.x * MERGE_THREADS + threadIdx.x;
  const int64_t first = ((int64_t)blockIdx.x * MERGE_THREADS) & ~(block * EMB_MERGE - 1);    // (a thread block's pairs are of one group)
  const uint64_t* from = in + first;
  const int64_t left = tokens - first;
  const int64_t apart = FIRST ? 1 : block / EACH;
  uint64_t x = 0;
  if (FIRST) {
    const int n = (int)(left < ALL ? left : ALL);
#pragma unroll 8
    for (int i = threadIdx.x; 2 * i < n; i += MERGE_THREADS) {
      // (the scratch that pairs lie in has room for an even count of them)
      reinterpret_cast<ulonglong2*>(sample)[i] = reinterpret_cast<const ulonglong2*>(from)[i];
    }
  } else {
    if (t < tokens) x = in[t];
#pragma unroll 8
    for (int i = threadIdx.x; i < ALL; i += MERGE_THREADS) {
      const int64_t at = (i + 1) * apart - 1;                  // (whole blocks one after the other)
      if (at < left) sample[i] = from[at];
    }
  }
  __syncthreads();
  if (t >= tokens) return;
  if (FIRST) x = sample[t - first];
  const int own = (int)((t - first) / block);
  uint32_t k[EMB_MERGE], n[EMB_MERGE];
#pragma unroll
  for (int b = 0; b < EMB_MERGE; ++b) {
    const int64_t rest = left - b * block;
    n[b] = b == own || rest < 0 ? 0 : (uint32_t)(rest < block ? rest : block);
    k[b] = 0;
  }
  // (while step is a multiple of `apart`, so is k, and the pair that is looked at is a sample)
  const int shift = FIRST ? 0 : 63 - __clzll(apart);
  for (uint32_t step = (uint32_t)block; step; step >>= 1) {
    uint64_t y[EMB_MERGE];
    if (FIRST || step >> shift) {
#pragma unroll
      for (int b = 0; b < EMB_MERGE; ++b) y[b] = k[b] + step <= n[b] ? sample[b * EACH + ((k[b] + step) >> shift) - 1] : ~0ull;
    } else {
#pragma unroll
      for (int b = 0; b < EMB_MERGE; ++b) y[b] = k[b] + step <= n[b] ? from[b * block + (k[b] + step - 1)] : ~0ull;
    }
#pragma unroll
    for (int b = 0; b < EMB_MERGE; ++b)
      if (y[b] < x) k[b] += step;
  }
  int64_t place = first + ((t - first) & (block - 1));
#pragma unroll
  for (int b = 0; b < EMB_MERGE; ++b) place += k[b];
  out[place] = x;
}

__device__ __forceinline__ uint32_t token_of(uint64_t x) { return (uint32_t)x; }
__device__ __forceinline__ int64_t id_of(uint64_t x) { return (int64_t)(x >> 32); }

// What a chunk of the sorted order looks like from the warp that has it: a pair per lane.
struct Piece {
  int64_t begin;
  int n;                                       // pairs of the chunk
  int64_t id;                                  // of this lane's pair
  uint32_t token;
  int64_t first_id, last_id;
  bool from_before, goes_on;                   // the first row's tokens began in an earlier chunk, the last one's end in a later one
};
__device__ __forceinline__ Piece piece_of(const EmbeddingArgs& a, const uint64_t* pairs, int64_t chunk, int lane) {
  Piece c;
  c.begin = chunk * CHUNK;
  c.n = (int)(a.tokens - c.begin < CHUNK ? a.tokens - c.begin : CHUNK);
  const uint64_t x = pairs[c.begin + (lane < c.n ? lane : c.n - 1)];
  c.id = id_of(x);
  c.token = token_of(x);
  c.first_id = __shfl_sync(0xffffffffu, c.id, 0);
  c.last_id = __shfl_sync(0xffffffffu, c.id, c.n - 1);
  c.from_before = c.begin > 0 && id_of(pairs[c.begin - 1]) == c.first_id;
  c.goes_on = c.begin + c.n < a.tokens && id_of(pairs[c.begin + c.n]) == c.last_id;
  return c;
}

// Rows without tokens (units 0 .. zero_units - 1: a warp looks after 32 rows of up to zero_cols columns), then chunks of the sorted order (a chunk and
// a slice each).
constexpr int GATHER_WARPS = 4;
template <typename T, typename O, bool WIDE>
__global__ void __launch_bounds__(32 * GATHER_WARPS)
gather_kernel(const EmbeddingArgs a, const uint64_t* pairs, int zero_cols, int64_t zero_units, int64_t chunk_units) {
  const int lane = threadIdx.x & 31;
  int64_t unit = (int64_t)blockIdx.x * GATHER_WARPS + (threadIdx.x >> 5);
  grid_wait();
  grid_release();
  if (unit >= zero_units) {
    unit -= zero_units;
    if (unit >= chunk_units) return;
    const int slices = (a.d + SLICE - 1) / SLICE;
    const int64_t chunk = unit / slices;
    const int col = (int)(unit - chunk * slices) * SLICE;
    const Piece c = piece_of(a, pairs, chunk, lane);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
    bool open = c.from_before;                 // the row under way began in an earlier chunk
    for (int e0 = 0; e0 < c.n; e0 += 8) {
      Eight<T, WIDE> g[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)              // (behind the last pair: the last one's again, not used)
        g[e].load(reinterpret_cast<const T*>(a.dout) + (int64_t)__shfl_sync(0xffffffffu, c.token, e0 + e) * a.ld, col, a.d, lane);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e0 + e >= c.n) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += g[e].at(i);
        const int64_t id = __shfl_sync(0xffffffffu, c.id, e0 + e);
        const bool at_end = e0 + e + 1 == c.n;
        if (!at_end && __shfl_sync(0xffffffffu, c.id, e0 + e + 1) == id) continue;
        // the row's last pair in this chunk
        if (id < a.rows) {
          if (open || (at_end && c.goes_on)) {
            Eight<float, WIDE>::store(f, a.partials + (chunk * 2 + (open ? 0 : 1)) * a.d_pad, col, a.d, lane);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= a.scale;
            Eight<O, WIDE>::store(f, reinterpret_cast<O*>(a.dtable) + id * a.d, col, a.d, lane);
          }
        }
        open = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 0.f;
      }
    }
    return;
  }
  const int parts = (a.d + zero_cols - 1) / zero_cols;
  const int64_t first = unit / parts * 32;
  const int col0 = (int)(unit % parts) * zero_cols, col1 = col0 + zero_cols < a.d ? col0 + zero_cols : a.d;
  const int64_t start = below(pairs, a.tokens, (uint64_t)(first + lane) << 32);
  const bool none = first + lane < a.rows && (start == a.tokens || id_of(pairs[start]) != first + lane);
  const float zero[8] = {};
  for (uint32_t rows = __ballot_sync(0xffffffffu, none); rows; rows &= rows - 1) {
    O* row = reinterpret_cast<O*>(a.dtable) + (first + __ffs(rows) - 1) * a.d;
    for (int col = col0; col < col1; col += SLICE) Eight<O, WIDE>::store(zero, row, col, a.d, lane);
  }
}

// Rows whose tokens are in several chunks: the block of the chunk in which they begin adds the partial sums, each warp a share of
// them, then the warps' sums.
template <typename O, bool WIDE>
__global__ void __launch_bounds__(THREADS)
join_kernel(const EmbeddingArgs a, const uint64_t* pairs) {
  __shared__ float sums[WARPS][SLICE];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slices = (a.d + SLICE - 1) / SLICE;
  grid_wait();
  grid_release();
  const int64_t chunk = blockIdx.x / slices;
  const int col = (int)(blockIdx.x % slices) * SLICE;
  const Piece c = piece_of(a, pairs, chunk, lane);
  const int64_t id = c.last_id;
  if (!c.goes_on || id >= a.rows || (c.from_before && c.first_id == id)) return;      // (the whole block)
  // chunks of the row: this one and those behind it that begin with it, looked at 32 at a time
  int64_t n = 1;
  for (bool more = true; more;) {
    const int64_t at = (chunk + n + lane) * CHUNK;
    const uint32_t others = __ballot_sync(0xffffffffu, at >= a.tokens || id_of(pairs[at]) != id);
    more = others == 0;
    n += more ? 32 : __ffs(others) - 1;
  }
  const int64_t p0 = n * warp / WARPS, p1 = n * (warp + 1) / WARPS;
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = 0.f;
#pragma unroll 4
  for (int64_t p = p0; p < p1; ++p) {
    Eight<float, WIDE> g;                      // (where it begins the row is the chunk's last, elsewhere its first)
    g.load(a.partials + ((chunk + p) * 2 + (p == 0 ? 1 : 0)) * a.d_pad, col, a.d, lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] += g.at(i);
  }
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
    Eight<O, WIDE>::store(f, reinterpret_cast<O*>(a.dtable) + id * a.d, col, a.d, lane);
  }
}

template <typename T, typename O, bool WIDE>
cudaError_t gather(cudaStream_t st, const EmbeddingArgs& a, const uint64_t* pairs, int* launches) {
  const int64_t slices = (a.d + SLICE - 1) / SLICE;
  const int64_t chunks = (a.tokens + CHUNK - 1) / CHUNK;
  // 1024 columns to a warp (each one searches for its rows' tokens), fewer where that leaves multiprocessors without work: 4 warps each of 148
  // (4000 rows of 771 in float32, 1500 tokens: 28.1 us with 1024 columns, 20.4 with 256)
  int zero_cols = 1024;
  while (zero_cols > SLICE && (a.rows + 31) / 32 * ((a.d + zero_cols - 1) / zero_cols) < 148 * 4) zero_cols /= 2;
  const int64_t zero_units = (a.rows + 31) / 32 * ((a.d + zero_cols - 1) / zero_cols);
  ++*launches;
  cudaError_t e = launch_dependent(gather_kernel<T, O, WIDE>, (unsigned)((chunks * slices + zero_units + GATHER_WARPS - 1) / GATHER_WARPS),
                                   32 * GATHER_WARPS, 0, st, a, pairs, zero_cols, zero_units, chunks * slices);
  if (e != cudaSuccess || chunks < 2) return e;
  ++*launches;
  return launch_dependent(join_kernel<O, WIDE>, (unsigned)((chunks - 1) * slices), THREADS, 0, st, a, pairs);
}

template <typename T, typename O>
cudaError_t gather(cudaStream_t st, const EmbeddingArgs& a, const uint64_t* pairs, int* launches) {
  const bool wide = a.d % 4 == 0 && a.ld % 4 == 0 && aligned16(a.dout) && aligned16(a.dtable);
  return wide ? gather<T, O, true>(st, a, pairs, launches) : gather<T, O, false>(st, a, pairs, launches);
}

}  // namespace

cudaError_t launch_embedding(cudaStream_t st, const EmbeddingArgs& a, int is_bf16) {
  const int64_t units = a.tokens * ((a.d + SLICE - 1) / SLICE);
  const unsigned blocks = (unsigned)((units + WARPS - 1) / WARPS);
  const bool wide = a.d % 4 == 0 && a.ld % 4 == 0 && aligned16(a.table) && aligned16(a.out);
  if (is_bf16)
    return wide ? launch_dependent(embedding_kernel<__nv_bfloat16, true>, blocks, THREADS, 0, st, a)
                : launch_dependent(embedding_kernel<__nv_bfloat16, false>, blocks, THREADS, 0, st, a);
  return wide ? launch_dependent(embedding_kernel<float, true>, blocks, THREADS, 0, st, a)
              : launch_dependent(embedding_kernel<float, false>, blocks, THREADS, 0, st, a);
}

size_t embedding_scratch(int64_t tokens, int64_t d) {
  const size_t pairs = (size_t)((tokens + 1) / 2 * 2) * 8;               // (a multiple of 16 bytes)
  return 2 * pairs + (size_t)((tokens + CHUNK - 1) / CHUNK) * 2 * (size_t)((d + 3) / 4 * 4) * 4;
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
    e = launch_dependent(block == EMB_SORT_BLOCK ? merge_kernel<true> : merge_kernel<false>,
                         (unsigned)((a.tokens + MERGE_THREADS - 1) / MERGE_THREADS), MERGE_THREADS, 0, st, (const uint64_t*)pairs, other,
                         a.tokens, block);
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
