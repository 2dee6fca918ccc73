// Embedding lookup with a factor, and the gradient of its weights, summed per partition by sorted tokens.
//
// Forward: y_i = s E[t_i], one copy of a row per token.  Memory: rows cols read, rows cols written.  16384 rows of 4096 bfloat16 41 us (6.6 TB/s), one row 2 us.
//
// Backward: dE_k[v] = s sum of dy_i over the rows i of partition k with t_i = v, written straight into row k of the partition-gradient
// matrix.  Every element is written, and most of them are zeros (a partition's tokens touch few of a vocabulary's rows): the bound is
// those partitions x vocab x cols elements.  So:
//   1. one kernel sorts each partition's tokens (stable radix sort in a cluster of 1-8 CTAs, 2-3 passes of up to nine bits) and notes in a bit
//      map which tokens there are;
//   2. a second one walks the sorted tokens in blocks of 8, 16 or 32, a team of threads a block, keeps a running float32 sum of the rows of
//      one token and writes it when the token changes.  A token whose rows reach over a block's end leaves partial sums.  The other CTAs of
//      the same grid meanwhile write the zeros of the tokens that are not there;
//   3. a third one adds the partial sums up.
// The order of every sum depends on sizes and tokens alone: the same call gives the same bits.  No atomics on values.
// 15 x 2048 tokens into 15 x 32768 x 1024 float32 312 us (6.6 TB/s of what has to be moved; zeros everywhere first and rows written over them: 404);
// 32768 tokens into 50001 x 2048 bfloat16 95 us: sort 20 (a cluster of eight), sums and zeros 60 (4.7 TB/s), partial sums 11.

#include <cooperative_groups.h>

#include <algorithm>

#include "elements.cuh"
#include "solon_internal.h"
#include "token_args.h"

namespace cg = cooperative_groups;

namespace solon {

// ------------------------------------------------------------------------------------------------------------ forward

struct EmbForwardArgs {
  const void* weight;
  const int64_t* tokens;
  void* out;
  int64_t weight_pitch, out_pitch, rows, cols, vocab;
  float scale;
  int lanes;                 // threads of a row
};

// N elements an access, as many as every row's alignment allows.  Four accesses a thread are on the way at once.
template <typename T, int N>
__global__ void __launch_bounds__(256) emb_forward_kernel(EmbForwardArgs a) {
  const int per_block = 256 / a.lanes;
  const int64_t row = (int64_t)blockIdx.x * per_block + threadIdx.x / a.lanes;
  if (row >= a.rows) return;
  const int lane = threadIdx.x % a.lanes;
  const int64_t token = a.tokens[row];
  const T* src = (const T*)a.weight + token * a.weight_pitch;
  T* dst = (T*)a.out + row * a.out_pitch;
  const int64_t words = a.cols / N;
  constexpr int kUnroll = 4;
  if (token < 0 || token >= a.vocab) {
    Pack<T, N> fill;
    const T value = from_float<T>(token < 0 ? 0.0f : __int_as_float(0x7FC00000));
#pragma unroll
    for (int i = 0; i < N; i++) fill.e[i] = value;
    for (int64_t w = lane; w < words; w += a.lanes) store_pack(dst + w * N, fill);
    if (lane < a.cols - words * N) dst[words * N + lane] = value;
    return;
  }
  for (int64_t w0 = lane; w0 < words; w0 += (int64_t)kUnroll * a.lanes) {
    Pack<T, N> v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; u++)
      if (w0 + u * a.lanes < words) v[u] = load_pack<T, N>(src + (w0 + u * a.lanes) * N);
#pragma unroll
    for (int u = 0; u < kUnroll; u++)
      if (w0 + u * a.lanes < words) {
        if (a.scale != 1.0f)
#pragma unroll
          for (int i = 0; i < N; i++) v[u].e[i] = from_float<T>(to_float(v[u].e[i]) * a.scale);
        store_pack(dst + (w0 + u * a.lanes) * N, v[u]);
      }
  }
  if (lane < a.cols - words * N) {
    const T x = src[words * N + lane];
    dst[words * N + lane] = a.scale == 1.0f ? x : from_float<T>(to_float(x) * a.scale);
  }
}

// Elements of `size` bytes that every row of the given matrices may be accessed by at once: 16 bytes at most.
static int common_pack(int size, uintptr_t addresses, int64_t pitches) {
  const uintptr_t both = addresses | (uintptr_t)(pitches * size);
  int bytes = 16;
  while (bytes > size && (both & (bytes - 1))) bytes /= 2;
  return bytes / size;
}

template <typename T, int N>
static int emb_forward_n(EmbForwardArgs a, cudaStream_t stream) {
  a.lanes = 32;
  while (a.lanes < 256 && a.lanes * 4 < a.cols / N) a.lanes *= 2;
  if (a.rows < 512)                             // few rows: a thread an access, so that none waits for another's
    while (a.lanes < 256 && a.lanes < a.cols / N) a.lanes *= 2;
  const int64_t blocks = (a.rows + 256 / a.lanes - 1) / (256 / a.lanes);
  emb_forward_kernel<T, N><<<(unsigned)blocks, 256, 0, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

template <typename T>
static int emb_forward_t(const EmbForwardArgs& a, cudaStream_t stream) {
  switch (common_pack(sizeof(T), (uintptr_t)a.weight | (uintptr_t)a.out, a.weight_pitch | a.out_pitch)) {
    case 8:
      if constexpr (sizeof(T) == 2) return emb_forward_n<T, 8>(a, stream);
    case 4:
      return emb_forward_n<T, 4>(a, stream);
    case 2:
      return emb_forward_n<T, 2>(a, stream);
    default:
      return emb_forward_n<T, 1>(a, stream);
  }
}

// ------------------------------------------------------------------------------------------------------------ backward

struct EmbBackArgs {
  const void* dy;
  const int64_t* tokens;
  void* dweight;
  int64_t dy_pitch, grad_pitch, n, cols, vocab;       // n: rows of a partition
  int partitions, accumulate;
  float scale;
  // sorted (token, row of the partition) pairs, two buffers of partitions x n; a token that counts in no gradient has key `vocab`
  int2 *pairs, *other;
  // blocks of sorted pairs
  int block;                 // pairs of a block
  int64_t per_partition, blocks;
  float* partial;            // blocks x 2 x cols: sums of a block's first token where it began earlier, of its last where it goes on
  int2* list;                // [0]: how many tokens reach over a block's end, over few blocks and over many; then the blocks that they begin in, and
                             // the tokens: those over few blocks from the front on, those over many from the back
  // the sort
  int passes, bits;
  unsigned* present;         // partitions x words bits: the tokens that a partition holds
  int64_t words;
};

constexpr int kSortThreads = 1024;
constexpr int kMaxBins = 512;
constexpr int kHeld = 4;
constexpr int kFew = 8;      // a token over more blocks is added up by a whole CTA

// A cluster a partition.  A warp of the cluster owns a run of consecutive tokens; a pass counts the digits of
// every warp's run, adds the counts up over warps, CTAs (distributed shared memory) and digits, and moves each pair to its place.
// Within a warp, 32 pairs at a time find their rank among equal digits by a match: the order of equal tokens stays.
__global__ void __launch_bounds__(kSortThreads, 1) emb_sort_kernel(EmbBackArgs a) {
  extern __shared__ int sort_smem[];
  __shared__ int warp_sums[kSortThreads / 32];
  pdl_trigger();
  cg::cluster_group cluster = cg::this_cluster();
  const int ranks = cluster.num_blocks(), rank = cluster.block_rank();
  const int k = blockIdx.x / ranks;
  const int warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int bins = 1 << a.bits;
  int* hist = sort_smem;                     // warps x bins
  int* total = hist + warps * bins;          // bins: this CTA's counts
  int* place = total + bins;                 // bins: where this CTA's first pair of a digit goes
  const int64_t run = ((a.n + (int64_t)ranks * warps - 1) / ((int64_t)ranks * warps) + 31) / 32 * 32;
  const int64_t begin = min(a.n, run * (rank * warps + warp)), end = min(a.n, begin + run);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.list[0] = make_int2(0, 0);
  const int64_t base = (int64_t)k * a.n;
  unsigned* present = a.present + k * a.words;
  for (int64_t i = rank * blockDim.x + threadIdx.x; i < a.words; i += ranks * blockDim.x) present[i] = 0;
  for (int pass = 0; pass < a.passes; pass++) {
    // (the last pass writes to `pairs`)
    int2* dst = ((a.passes - 1 - pass) & 1 ? a.other : a.pairs) + base;
    const int2* src = ((a.passes - 1 - pass) & 1 ? a.pairs : a.other) + base;
    const int shift = pass * a.bits;
    auto load = [&](int64_t i) {
      if (pass) return __ldcg(src + i);
      const int64_t t = a.tokens[base + i];
      return make_int2(t < 0 || t >= a.vocab ? (int)a.vocab : (int)t, (int)i);
    };
    int2 held[kHeld];                        // a warp's next 32 kHeld pairs, all on the way at once
    auto fetch = [&](int64_t i0) {
#pragma unroll
      for (int u = 0; u < kHeld; u++)
        if (i0 + 32 * u + lane < end) held[u] = load(i0 + 32 * u + lane);
    };
    fetch(begin);
    for (int i = threadIdx.x; i < warps * bins; i += blockDim.x) hist[i] = 0;
    __syncthreads();
    for (int64_t i0 = begin; i0 < end; i0 += 32 * kHeld) {
      if (i0 > begin) fetch(i0);
#pragma unroll
      for (int u = 0; u < kHeld; u++)
        if (i0 + 32 * u + lane < end) atomicAdd(&hist[warp * bins + ((held[u].x >> shift) & (bins - 1))], 1);
    }
    __syncthreads();
    const int bin = threadIdx.x;             // (there are at least as many threads)
    if (bin < bins) {
      int sum = 0;
      for (int w0 = 0; w0 < warps; w0 += 8) {
        int c[8];
#pragma unroll
        for (int w = 0; w < 8; w++) c[w] = hist[(w0 + w) * bins + bin];
#pragma unroll
        for (int w = 0; w < 8; w++) {
          hist[(w0 + w) * bins + bin] = sum;
          sum += c[w];
        }
      }
      total[bin] = sum;
    }
    cluster.sync();
    int before = 0, all = 0;
    if (bin < bins) {
      int c[8];
#pragma unroll
      for (int r = 0; r < 8; r++) c[r] = r < ranks ? *cluster.map_shared_rank(total + bin, r) : 0;
#pragma unroll
      for (int r = 0; r < 8; r++) {
        before += r < rank ? c[r] : 0;
        all += c[r];
      }
    }
    int up = all;                            // sums over the digits up to this one: within a warp, then over the warps
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int v = __shfl_up_sync(~0u, up, o);
      if (lane >= o) up += v;
    }
    if (lane == 31) warp_sums[warp] = up;
    __syncthreads();
    if (bin < bins) {
      int lower = 0;
      for (int w = 0; w < warp; w++) lower += warp_sums[w];
      place[bin] = lower + up - all + before;
    }
    __syncthreads();
    for (int64_t i0 = begin; i0 < end; i0 += 32 * kHeld) {
      if (end - begin > 32 * kHeld) fetch(i0);
#pragma unroll
      for (int u = 0; u < kHeld; u++) {
        const bool mine = i0 + 32 * u + lane < end;
        const unsigned who = __ballot_sync(~0u, mine);
        if (mine) {
          const int2 p = held[u];
          const int d = (p.x >> shift) & (bins - 1);
          const unsigned same = __match_any_sync(who, d);
          const int ahead = __popc(same & ((1u << lane) - 1));
          int* count = &hist[warp * bins + d];
          const int at = place[d] + *count + ahead;
          __syncwarp(who);
          if (ahead == 0) *count += __popc(same);
          dst[at] = p;
          if (pass == a.passes - 1 && lane == __ffs(__match_any_sync(who, p.x)) - 1 && p.x < a.vocab) atomicOr(present + p.x / 32, 1u << (p.x & 31));
        }
        __syncwarp();
      }
    }
    cluster.sync();
  }
}

template <typename G>
__device__ __forceinline__ void put_grad(G* p, float x, int accumulate) {
  if constexpr (sizeof(G) == 8) *p = accumulate ? *p + (double)x : (double)x;
  else *p = from_float<G>(accumulate ? to_float(*p) + x : x);
}

// `bytes` bytes of zeros at p (aligned to its elements of `size` bytes), by the lanes of a warp.
__device__ __forceinline__ void zero_bytes(char* p, int64_t bytes, int size, int lane) {
  const int64_t head = min(bytes, (int64_t)((16 - ((uintptr_t)p & 15)) & 15));
  const int64_t words = (bytes - head) / 16, tail = bytes - head - words * 16;
  uint4* w = reinterpret_cast<uint4*>(p + head);
#pragma unroll 4
  for (int64_t i = lane; i < words; i += 32) w[i] = make_uint4(0, 0, 0, 0);
  const int64_t rest = (head + tail) / size;          // at most 15 bytes at either end
  if (lane < rest) {
    const int64_t at = (int64_t)lane * size;
    char* q = at < head ? p + at : p + head + words * 16 + (at - head);
    if (size == 2) *reinterpret_cast<uint16_t*>(q) = 0;
    else if (size == 4) *reinterpret_cast<uint32_t*>(q) = 0;
    else *reinterpret_cast<uint64_t*>(q) = 0;
  }
}

// Zeros for the tokens that are not there: a warp takes eight tokens of a partition at a time, runs of absent ones as one stretch.
template <typename G>
__device__ __forceinline__ void emb_zeros(const EmbBackArgs& a, int64_t warp, int64_t warps) {
  const int lane = threadIdx.x % 32;
  const int64_t groups = (a.vocab + 7) / 8;
  for (int64_t i = warp; i < groups * a.partitions; i += warps) {
    const int64_t k = i / groups, v = (i - k * groups) * 8;
    const int rows = (int)min((int64_t)8, a.vocab - v);
    unsigned absent = ~(__ldcg(a.present + k * a.words + v / 32) >> (v & 31)) & ((1u << rows) - 1);
    while (absent) {
      const int first = __ffs(absent) - 1, count = __ffs(~(absent >> first)) - 1;
      zero_bytes((char*)((G*)a.dweight + k * a.grad_pitch + (v + first) * a.cols), count * a.cols * (int64_t)sizeof(G), sizeof(G), lane);
      absent &= ~(((1u << count) - 1) << first);
    }
  }
}

// The first CTAs of the grid: N consecutive columns a thread, blockDim.x threads (whole warps) a block of sorted pairs.  All threads of a team see the
// same pairs, so its branches do not diverge.  Eight rows are on the way at once.  The others write zeros.
template <typename T, typename G, int N>
__global__ void __launch_bounds__(256) emb_sum_kernel(EmbBackArgs a, int wide_out, int slices, unsigned sum_blocks) {
  pdl_trigger();
  pdl_wait();
  if (blockIdx.x >= sum_blocks) {
    const int warp = (threadIdx.y * blockDim.x + threadIdx.x) / 32;
    emb_zeros<G>(a, (int64_t)(blockIdx.x - sum_blocks) * 8 + warp, (int64_t)(gridDim.x - sum_blocks) * 8);
    return;
  }
  const int slice = blockIdx.x % slices;
  const int64_t b = (int64_t)(blockIdx.x / slices) * blockDim.y + threadIdx.y;
  if (b >= a.blocks) return;
  const int lane = threadIdx.x % 32;
  const int64_t col = ((int64_t)slice * blockDim.x + threadIdx.x) * N;
  const bool inside = col < a.cols;          // N divides cols
  const int64_t k = b / a.per_partition, j0 = (b - k * a.per_partition) * a.block;
  const int count = (int)min((int64_t)a.block, a.n - j0);
  const int2* pairs = a.pairs + k * a.n + j0;
  const int none = (int)a.vocab;
  const int2 mine = lane < count ? __ldcg(pairs + lane) : make_int2(none, 0);
  const int earlier = j0 > 0 ? __ldcg(&pairs[-1].x) : none, later = j0 + count < a.n ? __ldcg(&pairs[count].x) : none;
  const T* dy = (const T*)a.dy + k * a.n * a.dy_pitch + (inside ? col : 0);
  G* dw = (G*)a.dweight + k * a.grad_pitch + col;
  float acc[N];
  int key = __shfl_sync(~0u, mine.x, 0);
  if (key == none) return;
  bool first = true;

  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < N; i++) acc[i] = 0.0f;
  };
  auto finish = [&](int token) {             // a token whose rows are all in this block
    if (!inside) return;
    G* p = dw + token * a.cols;
    if (wide_out && !a.accumulate && sizeof(G) * N % 16 == 0) {
      constexpr int kEach = 16 / sizeof(G) < N ? 16 / sizeof(G) : N;
#pragma unroll
      for (int i = 0; i < N; i += kEach) {
        Pack<G, kEach> v;
#pragma unroll
        for (int e = 0; e < kEach; e++) put_grad(&v.e[e], acc[i + e] * a.scale, 0);
        store_pack(p + i, v);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; i++) put_grad(p + i, acc[i] * a.scale, a.accumulate);
    }
  };
  auto leave = [&](int which) {
    float* p = a.partial + (b * 2 + which) * a.cols + col;
#pragma unroll
    for (int i = 0; i < N; i++)
      if (inside) p[i] = acc[i];
  };

  clear();
  constexpr int kUnroll = 8;
  for (int j = 0; j < count; j += kUnroll) {
    Pack<T, N> x[kUnroll];
    int keys[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
      keys[u] = __shfl_sync(~0u, mine.x, (j + u) & 31);
      const int64_t row = __shfl_sync(~0u, mine.y, (j + u) & 31);
      if (j + u >= count) keys[u] = none;
      x[u] = load_pack<T, N>(dy + row * a.dy_pitch);       // (of a pair that is not there: row 0)
    }
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
      if (keys[u] == none) continue;
      if (keys[u] != key) {
        if (first && key == earlier) leave(0);
        else finish(key);
        clear();
        key = keys[u];
        first = false;
      }
#pragma unroll
      for (int i = 0; i < N; i++) acc[i] += to_float(x[u].e[i]);
    }
  }
  if (first && key == earlier) leave(0);
  else if (key == later) {
    leave(1);
    if (threadIdx.x == 0 && slice == 0) {
      const int64_t far = (int64_t)(kFew + 1) * a.block;
      const bool many = j0 + far < a.n && __ldcg(&pairs[far].x) == key;
      const int at = many ? (int)a.blocks - atomicAdd(&a.list[0].y, 1) : 1 + atomicAdd(&a.list[0].x, 1);
      a.list[at] = make_int2((int)b, key);
    }
  } else finish(key);
}

// How many blocks from block b on hold the token, looked at 32 at a time by the lanes of a warp.
__device__ __forceinline__ int64_t blocks_of(const EmbBackArgs& a, int64_t b, int token, int lane) {
  const int64_t k = b / a.per_partition, j0 = (b - k * a.per_partition) * a.block;
  const int2* pairs = a.pairs + k * a.n;
  int64_t blocks = 2;
  for (;;) {
    const int64_t j = j0 + (blocks + lane) * a.block;
    const unsigned other = __ballot_sync(~0u, j >= a.n || __ldcg(&pairs[j < a.n ? j : 0].x) != token);
    blocks += other ? __ffs(other) - 1 : 32;
    if (other) return blocks;
  }
}

// Partial sums [from, to) of the token that begins in block b, four columns a lane, 32 apart.
__device__ __forceinline__ void add_partials(const EmbBackArgs& a, int64_t b, int64_t from, int64_t to, int64_t col, float (&acc)[4]) {
#pragma unroll 4
  for (int64_t s = from; s < to; s++) {
    const float* p = a.partial + ((b + s) * 2 + (s == 0)) * a.cols + col;
#pragma unroll
    for (int c = 0; c < 4; c++)
      if (col + 32 * c < a.cols) acc[c] += __ldcg(p + 32 * c);
  }
}

// Adds up the partial sums of the tokens that reach over a block's end, 128 columns at a time: those over many blocks by the eight warps of a CTA, each an
// eighth of the blocks in order, then their sums in order; those over few by a warp.  The order of the lists, which is not fixed, only says
// who does which token.
template <typename G>
__global__ void __launch_bounds__(256) emb_join_kernel(EmbBackArgs a) {
  __shared__ float sums[8][128];
  pdl_wait();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t slices = (a.cols + 127) / 128;
  const int2 count = __ldcg(a.list);
  for (int64_t i = blockIdx.x; i < count.y * slices; i += gridDim.x) {
    const int2 at = __ldcg(a.list + a.blocks - i / slices);
    const int64_t b = at.x, col = i % slices * 128;
    const int64_t blocks = blocks_of(a, b, at.y, lane);
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    add_partials(a, b, blocks * warp / 8, blocks * (warp + 1) / 8, col + lane, acc);
#pragma unroll
    for (int c = 0; c < 4; c++) sums[warp][lane + 32 * c] = acc[c];
    __syncthreads();
    if (threadIdx.x < 128 && col + threadIdx.x < a.cols) {
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < 8; w++) sum += sums[w][threadIdx.x];
      put_grad((G*)a.dweight + b / a.per_partition * a.grad_pitch + at.y * a.cols + col + threadIdx.x, sum * a.scale, a.accumulate);
    }
    __syncthreads();
  }
  for (int64_t i = (int64_t)blockIdx.x * 8 + warp; i < count.x * slices; i += (int64_t)gridDim.x * 8) {
    const int2 at = __ldcg(a.list + 1 + i / slices);
    const int64_t b = at.x, col = i % slices * 128 + lane;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    add_partials(a, b, 0, blocks_of(a, b, at.y, lane), col, acc);
    G* p = (G*)a.dweight + b / a.per_partition * a.grad_pitch + at.y * a.cols + col;
#pragma unroll
    for (int c = 0; c < 4; c++)
      if (col + 32 * c < a.cols) put_grad(p + 32 * c, acc[c] * a.scale, a.accumulate);
  }
}

// How the sorted pairs are cut.  Smaller blocks where there would be less than two teams an SM (148 of them): a block is gone
// through row by row, and its time is what a short call waits for.
struct EmbCut {
  int block;
  int64_t per_partition, blocks;
};
static EmbCut emb_cut(int64_t n, int64_t cols, int partitions) {
  EmbCut c;
  c.block = 32;
  const int64_t slices = (cols + 1023) / 1024;
  while (c.block > 8 && partitions * ((n + c.block - 1) / c.block) * slices < 2 * 148) c.block /= 2;
  c.per_partition = (n + c.block - 1) / c.block;
  c.blocks = c.per_partition * partitions;
  return c;
}

static int64_t up16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

static int64_t emb_words(int64_t vocab) { return (vocab + 31) / 32; }

static int64_t emb_back_workspace(int64_t rows, int64_t cols, int64_t vocab, int partitions) {
  const EmbCut c = emb_cut(rows / partitions, cols, partitions);
  return 2 * up16(rows * (int64_t)sizeof(int2)) + up16((c.blocks + 1) * (int64_t)sizeof(int2)) + up16(emb_words(vocab) * partitions * 4) +
         (c.per_partition > 1 ? c.blocks * 2 * cols * 4 : 0);
}

template <typename T, typename G, int N>
static int emb_sum_launch(const EmbBackArgs& a, int sms, cudaStream_t stream) {
  const int64_t words = (a.cols + N - 1) / N;
  int team = 32;
  while (team < 256 && team < words) team *= 2;
  const dim3 block(team, 256 / team);
  const int64_t slices_n = (words + team - 1) / team, sum_blocks = (a.blocks + block.y - 1) / block.y * slices_n;
  const int64_t groups = (a.vocab + 7) / 8 * a.partitions;
  const int64_t zero_blocks = a.accumulate ? 0 : std::min<int64_t>((groups + 7) / 8, 1 << 20);
  if (sum_blocks + zero_blocks > 0x7FFFFFFF) return SOLON_ERR_INVALID_ARG;
  if (sum_blocks + zero_blocks == 0) return SOLON_OK;
  const int wide_out = !(((uintptr_t)a.dweight | (uintptr_t)(a.grad_pitch * sizeof(G)) | (uintptr_t)(a.cols * sizeof(G))) & 15);
  const int rc = launch_dependent(emb_sum_kernel<T, G, N>, dim3((unsigned)(sum_blocks + zero_blocks)), block, 0, stream, a, wide_out, (int)slices_n,
                                  (unsigned)sum_blocks);
  if (rc || a.per_partition <= 1) return rc;
  const int64_t joins = std::min<int64_t>((a.blocks * ((a.cols + 127) / 128) + 7) / 8, 8 * sms);
  return launch_dependent(emb_join_kernel<G>, dim3((unsigned)joins), dim3(256), 0, stream, a);
}

template <typename T, typename G>
static int emb_backward_t(const EmbBackArgs& a, int sms, cudaStream_t stream) {
  switch (common_pack(sizeof(T), (uintptr_t)a.dy, a.dy_pitch | a.cols)) {
    case 8:
      if constexpr (sizeof(T) == 2) return emb_sum_launch<T, G, 8>(a, sms, stream);
    case 4:
      return emb_sum_launch<T, G, 4>(a, sms, stream);
    case 2:
      return emb_sum_launch<T, G, 2>(a, sms, stream);
    default:
      return emb_sum_launch<T, G, 1>(a, sms, stream);
  }
}

template <typename T>
static int emb_backward_g(const EmbBackArgs& a, int grad_dtype, int sms, cudaStream_t stream) {
  if (grad_dtype == SOLON_F32) return emb_backward_t<T, float>(a, sms, stream);
  if (grad_dtype == SOLON_F64) return emb_backward_t<T, double>(a, sms, stream);
  return emb_backward_t<T, __nv_bfloat16>(a, sms, stream);
}

static int emb_sort_launch(EmbBackArgs a, cudaStream_t stream) {
  // 2048 tokens a CTA, in clusters of at most eight
  int ranks = 1;
  while (ranks < 8 && (int64_t)ranks * 2048 < a.n) ranks *= 2;
  int key_bits = 1;
  while (a.vocab >> key_bits) key_bits++;                // the key of tokens that count nowhere is `vocab` itself
  a.passes = (key_bits + 8) / 9;
  a.bits = (key_bits + a.passes - 1) / a.passes;
  int threads = std::max(256, 1 << a.bits);                // a thread a digit, and a token where there are more
  while (threads < kSortThreads && (int64_t)threads * ranks < a.n) threads *= 2;
  const size_t smem = ((size_t)(threads / 32) + 2) * ((size_t)1 << a.bits) * sizeof(int);
  SOLON_SHARED_MEMORY_ONCE(emb_sort_kernel, (kSortThreads / 32 + 2) * kMaxBins * sizeof(int));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.partitions * ranks));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)ranks, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  SOLON_CUDA_TRY(cudaLaunchKernelEx(&cfg, emb_sort_kernel, a));
  return SOLON_OK;
}

static bool emb_sizes_ok(int64_t rows, int64_t cols, int64_t vocab) {
  return rows >= 0 && rows < (1ll << 31) - 64 && cols >= 1 && cols <= SOLON_MAX_WIDTH && vocab >= 1 && vocab < (1ll << 31) - 1 &&
         vocab <= (1ll << 46) / cols;
}

}  // namespace solon

using namespace solon;

extern "C" {

int solon_embedding_forward(const void* weight, int64_t weight_pitch, int dtype, const int64_t* tokens, int64_t rows, int64_t cols, int64_t vocab,
                            double scale, void* out, int64_t out_pitch, void* cuda_stream) {
  if (!token_dtype(dtype) || !emb_sizes_ok(rows, cols, vocab)) return SOLON_ERR_INVALID_ARG;
  if (rows == 0) return SOLON_OK;
  if (!matrix_ok(weight, weight_pitch, vocab, cols, dtype) || !matrix_ok(out, out_pitch, rows, cols, dtype) || !tokens || ((uintptr_t)tokens & 7))
    return SOLON_ERR_INVALID_ARG;
  const Extent to = extent(out, rows, cols, out_pitch, element_size(dtype));
  if (meet(to, extent(weight, vocab, cols, weight_pitch, element_size(dtype))) || meet(to, extent(tokens, 1, rows, rows, 8))) return SOLON_ERR_INVALID_ARG;
  const EmbForwardArgs a = {weight, tokens, out, vocab > 1 ? weight_pitch : cols, rows > 1 ? out_pitch : cols, rows, cols, vocab, (float)scale, 0};
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (dtype == SOLON_F32) return emb_forward_t<float>(a, stream);
  if (dtype == SOLON_BF16) return emb_forward_t<__nv_bfloat16>(a, stream);
  return emb_forward_t<__half>(a, stream);
}

int64_t solon_embedding_backward_workspace(int64_t rows, int64_t cols, int64_t vocab, int partitions) {
  if (!emb_sizes_ok(rows, cols, vocab) || partitions < 1 || partitions > SOLON_MAX_NODES || rows % partitions) return SOLON_ERR_INVALID_ARG;
  return emb_back_workspace(rows, cols, vocab, partitions);
}

int solon_embedding_backward(const void* dy, int64_t dy_pitch, int dtype, const int64_t* tokens, int64_t rows, int64_t cols, int64_t vocab, int partitions,
                             double scale, void* dweight, int64_t grad_pitch, int grad_dtype, int accumulate, void* workspace, int64_t workspace_bytes,
                             void* cuda_stream) {
  if (!token_dtype(dtype) || !emb_sizes_ok(rows, cols, vocab) || partitions < 1 || partitions > SOLON_MAX_NODES || rows % partitions)
    return SOLON_ERR_INVALID_ARG;
  if (grad_dtype != SOLON_F32 && grad_dtype != SOLON_F64 && grad_dtype != SOLON_BF16) return SOLON_ERR_INVALID_ARG;
  if (!matrix_ok(dweight, grad_pitch, partitions, vocab * cols, grad_dtype)) return SOLON_ERR_INVALID_ARG;
  if (rows > 0 && (!matrix_ok(dy, dy_pitch, rows, cols, dtype) || !tokens || ((uintptr_t)tokens & 7))) return SOLON_ERR_INVALID_ARG;
  const Extent to = extent(dweight, partitions, vocab * cols, grad_pitch, element_size(grad_dtype));
  if (rows > 0 && (meet(to, extent(dy, rows, cols, dy_pitch, element_size(dtype))) || meet(to, extent(tokens, 1, rows, rows, 8)))) return SOLON_ERR_INVALID_ARG;
  if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < emb_back_workspace(rows, cols, vocab, partitions)) return SOLON_ERR_INVALID_ARG;
  int sms = 0, rc;
  if ((rc = current_sms(&sms))) return rc;
  const EmbCut cut = emb_cut(rows / partitions, cols, partitions);
  EmbBackArgs a = {};                      // (without rows: all zeros, or nothing)
  a.dy = dy;
  a.tokens = tokens;
  a.dweight = dweight;
  a.dy_pitch = rows > 1 ? dy_pitch : cols;
  a.grad_pitch = partitions > 1 ? grad_pitch : vocab * cols;
  a.n = rows / partitions;
  a.cols = cols;
  a.vocab = vocab;
  a.partitions = partitions;
  a.accumulate = accumulate != 0;
  a.scale = (float)scale;
  char* at = (char*)workspace;
  a.pairs = (int2*)at;
  a.other = (int2*)(at += up16(rows * (int64_t)sizeof(int2)));
  a.list = (int2*)(at += up16(rows * (int64_t)sizeof(int2)));
  a.present = (unsigned*)(at += up16((cut.blocks + 1) * (int64_t)sizeof(int2)));
  a.words = emb_words(vocab);
  a.partial = (float*)(at + up16(a.words * partitions * 4));
  a.block = cut.block;
  a.per_partition = cut.per_partition;
  a.blocks = cut.blocks;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  if ((rc = emb_sort_launch(a, stream))) return rc;
  if (dtype == SOLON_F32) return emb_backward_g<float>(a, grad_dtype, sms, stream);
  if (dtype == SOLON_BF16) return emb_backward_g<__nv_bfloat16>(a, grad_dtype, sms, stream);
  return emb_backward_g<__half>(a, grad_dtype, sms, stream);
}

}  // extern "C"
