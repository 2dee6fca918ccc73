// Log probabilities of given tokens straight from hidden states h (rows x cols) and output matrix W (vocab x cols), and their gradient.  The
// logits z = h W^T are never in memory: a tile of them lives in tensor memory until its part of the result has been taken from it.
//
// Forward: per row M = max z, S = sum e^(z - M), A = sum e^(z - M)(z - M) by tiles of 256 tokens, joined by a second kernel; log p = (z_t - M) -
// log S, entropy log S - A / S.  Backward, in pieces of the vocabulary: the piece's logits once more, dz = g (1[t] - p) - g_H p (log p + H) from
// them into a workspace, then dh += dz W and dW_k = dz_k^T h_k by two more products.
//
// All three products run on the tensor cores (tensor_tiles.cuh).  What is multiplied is 16 bits wide:
//   bfloat16, float16  the elements themselves; sums float32.  (Rows off 16-byte boundaries are copied to a pitch that the copies can take.)
//   float32            two float16 pieces, x = 2^-s (hi + 2^-11 lo), s such that the largest lies in [2^14, 2^15): of the row for the logits, whose epilogue
//                      undoes it, so that rows and tokens are what they are whatever stands beside them; of all W for dh, of a partition for dW, which add up over them.
//                      The pieces hold 22 bits of values down to 2^-28 of the largest, and an absolute 2^-50 of it below.  (With lo not multiplied the 22 bits ended at 2^-17: a float16's steps
//                      end at 2^-24.)  A product is three: hi lo + lo hi, whose sum is taken times 2^-11 in registers, then hi hi; the lo lo left out is below
//                      2^-22 of the term.  (Three bfloat16 pieces would take six products.)
//   dz                 float16 by the power of two of its row's |g| + |g_H| (H + 1), of any states (bfloat16 states and weights are taken as float16 by a power
//                      of two for these products: eight bits of dz would put as much into a result again as its own rounding to bfloat16 does; with eleven, an
//                      eighth of that).  One piece for dh of bfloat16 states and for bfloat16 gradients (those of float32 states take the first piece of
//                      the states alone, too): 11 bits of what lies above 2^-28 of the largest, an absolute 2^-40 of it below.  Two, the second times 2^11 as above,
//                      for dh of float16 and float32 states and for float32 and float64 gradients: 22 bits, and 2^-50.  Up to 512 bfloat16 rows it is bfloat16
//                      instead, at any magnitude: two pieces (16 bits), or three (24) for dW in float32 and float64.
//
// Measured (us, the first in bursts, the second at the power limit, of 1662 and 1407 TFLOP/s): 8192 x 2048 states, 32768 tokens, bfloat16: forward 790 and 930 (1.39 and
// 1.18 PFLOP/s), backward with bfloat16 gradients 2485 and 2910 (1.33 and 1.13, of which 100 are the scan and the copy of W as float16); a library's plain products of these sizes
// take 660 to 730 each, so that with logits in memory the two passes take 2330 together where they take 3300 here: what this form saves is 0.5 GB of logits.  In float32,
// whose products the library takes without tensor cores, it saves time as well: 2047 x 1001 over 50001 tokens 2280 against 10480.  What the product is fed by and how it ends is what that came from: one
// copy for 128 rows or columns of a block (6 %), two warps that issue them (4 %), sums of 512 in registers (5 % against 256), no branch between a row's
// elements and no store of single rows in the epilogues (a third of their time).
//
// Few rows (a served token) are a matter of reading W once.  Up to 128 rows the product is taken the other way round (tokens along the tile's rows): 131072 x 2048
// bfloat16 90 us for one row (6.0 TB/s), 100 to 119 for 96.  float32 and rows off 16-byte boundaries are not brought into another form for a few rows: kernels of
// multiply-adds, here for up to 4 rows of any type and alignment, in head_rows.cu for up to 32 float32 rows.

#include <algorithm>
#include <cmath>

#include "elements.cuh"
#include "head_rows.h"
#include "head_sums.cuh"
#include "solon_internal.h"
#include "tensor_tiles.cuh"
#include "token_args.h"

namespace solon {

using namespace tiles;

constexpr int kTile = 256;               // vocabulary tokens, or rows, of a pair's tile
constexpr int kEpilogueWarps = 8;
constexpr int kFirstEpilogue = 4;        // the warps before it bring blocks and multiply, and give registers to the others
constexpr int kThreads = 32 * (kFirstEpilogue + kEpilogueWarps);

enum HeadMode { kStats, kFewRows, kDz, kDhidden, kDweight };

// ------------------------------------------------------------------------------------------------------------ scales

// Powers of two.  A float32 row of hidden states or weights has one of its own for the logits, a row's dz has one, by the largest that it can hold, and the weights
// have one for dh.  dW of a partition adds up rows: there row i of h carries what its dz lacks to the partition's exponent, so that what counts is |dz_i| |h_i|
// against the partition's largest, and partitions say nothing about one another.

// What the scan of a call leaves behind: the bits of the weights' largest finite magnitude.  Behind it a word a partition: the exponent of its largest
// |dz_i| |h_i| over that of dz (0: no row with a share).
struct HeadWords {
  unsigned weight;
};

// Set by a wait that ran out, and never cleared.
__device__ int head_wait_status;

__device__ __forceinline__ int scale_exponent(unsigned largest) {       // 2^s brings the largest magnitude into [2^14, 2^15)
  return largest ? min(126, 14 - ilogbf(__uint_as_float(largest))) : 0;
}
constexpr int kPartBias = 1024;
__device__ __forceinline__ int part_exponent(unsigned word) { return word ? 14 + kPartBias - (int)word : 0; }      // -226 to 252
__device__ __forceinline__ int exponent_of(float power) { return (__float_as_int(power) >> 23) - 127; }             // of a power of two
__device__ __forceinline__ float inverse_power(float power) { return __int_as_float(0x7F000000 - __float_as_int(power)); }
__device__ __forceinline__ float joint(float power, float other) { return fminf(power * other, 0x1p127f); }         // (finite: it may be that zeros are multiplied)
constexpr float kSecond = 2048.0f;       // what a second piece is multiplied by: at most 2^3 is left of elements below 2^15, and 2^-25 of those below 2^-14
__device__ __forceinline__ float power_of_two(int s) { return __int_as_float((s + 127) << 23); }       // -126 <= s <= 127

// ------------------------------------------------------------------------------------------------------------ arguments

struct alignas(64) HeadMaps {
  CUtensorMap a, b, out;
};

struct HeadArgs {
  // the product: slabs times m x n, in blocks of 64 inner indices, `products` pairs of pieces
  int m, n, m_tiles, n_tiles, slabs;
  uint32_t per_slab_inverse, band_inverse;             // reciprocals for the tiles' numbers
  int k_blocks, products;
  int chunk;                             // blocks of 64 that are summed in tensor memory before the sum is added to the one in registers
  int low;                               // blocks of the products with a second piece, which come first: their sum is taken times low_factor before the others join it
  float low_factor;                      // 2^-11 for float16 pieces
  int piece_a[3], piece_b[3];            // third coordinate of the tensor maps for slab 0; slab s is s further
  int slab_a, slab_b;                    // 1: the operand has slabs
  int splits;                            // the inner dimension is cut into so many parts of k_blocks, slabs of their own; what lies behind its end is zeros
  int narrow;                            // tiles of 128 columns
  int b_by_blocks;                       // B's map takes 128 columns a copy, where its rows lie across the inner dimension
  const HeadWords* words;
  int weight_scaled;                     // kDhidden: the weights carry a power of two
  const unsigned* parts;                 // kDweight: the partitions' words (NULL: nothing carries a power of two)
  const float *undo_m, *undo_n;          // what the product's rows and columns are multiplied by (NULL: nothing)
  // rows
  const int64_t* targets;
  const float *peak, *log_sum, *entropy, *grad_logp, *grad_entropy;
  const float* undo_dz;                  // kDz: what a row's dz is multiplied by where it has been used (0: the row has no share)
  // kStats, kFewRows (whose product is W h^T: tokens are rows of it)
  float* partial;                        // slots x 3 x rows
  float* target_logit;                   // rows
  // kStats, kDz: columns of the product are tokens first + n
  int64_t first, vocab;
  // kDz
  int dz_pitch;                          // this piece's tokens, zeros behind them up to a multiple of 64
  int form;                              // what is stored of dz (DzForm)
  // kDhidden, kDweight
  float* sums;                           // slabs x m x sums_pitch: where the result goes in float32 instead of to the output, if store_sums
  int64_t sums_pitch;
  int load_sums, store_sums;             // load_sums: the result is added to what is there (kDhidden, the pieces of the vocabulary before)
  // kDhidden, kDweight
  void* out;
  int64_t out_pitch, out_slab;           // elements; a slab is a partition
  int out_by_map;                        // kDweight: the output's map can be used (16-byte aligned rows)
  int out_wide;                          // rows of the output begin at multiples of 32 bytes
};

// ------------------------------------------------------------------------------------------------------------ epilogues

// 32 rows x 32 columns from a register per column of a lane's row to four consecutive columns of a row: eight lanes a row.
__device__ __forceinline__ void stage_rows(const float* v, float4* stage, int lane) {
#pragma unroll
  for (int i = 0; i < 8; i++) stage[lane * 8 + (i ^ (lane & 7))] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
}

template <typename O>
__device__ __forceinline__ void store1(O* p, float v) {
  if constexpr (sizeof(O) == 8) *p = (double)v;
  else *p = from_float<O>(v);
}

__device__ __forceinline__ void store32(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]),
               "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void load32(const float* p, float (&v)[8]) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "l"(p)
               : "memory");
}

// N columns of a lane's row to 32-byte aligned places, 32 bytes an access.  Every lane fills whole sectors of a row of its own; bringing the rows together in
// shared memory first made wider stretches, but there the tensor cores and the copies that feed them take all there is, and the warps waited.
template <typename O, int N>
__device__ __forceinline__ void store_columns(O* p, const float* v) {
  constexpr int kEach = 32 / sizeof(O);
#pragma unroll
  for (int i = 0; i < N; i += kEach) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; j++) {
      if constexpr (sizeof(O) == 4) w[j] = __float_as_uint(v[i + j]);
      else if constexpr (sizeof(O) == 2) w[j] = Word16<O>::join(v[i + 2 * j], v[i + 2 * j + 1]);
      else w[j] = j % 2 ? __double2hiint((double)v[i + j / 2]) : __double2loint((double)v[i + j / 2]);
    }
    store32(p + i, w);
  }
}

// Rows [row, row + 32) and columns [col, col + 32) of an output of m x n at any alignment, a column a lane.
template <typename O>
__device__ __forceinline__ void write_rows(const float4* stage, O* out, int64_t pitch, int row, int col, int m, int n, int lane) {
  const float* s = reinterpret_cast<const float*>(stage) + lane % 4;
  O* p = out + row * pitch + col + lane;
  const int rows = col + lane < n ? m - row : 0;
#pragma unroll 8
  for (int r = 0; r < 32; r++, p += pitch)
    if (r < rows) store1(p, s[(r * 8 + ((lane / 4) ^ (r & 7))) * 4]);
}

struct DzRow {
  float peak, log_sum, entropy, g, gh;
};

// What is stored of dz: the nearest float16; that and what it leaves, times kSecond, as a second float16; or the nearest bfloat16 and what it leaves in one or two more.
enum DzForm { kNearest, kPair, kWidePair, kWideTriple };

struct DzOut {
  const CUtensorMap* map;
  char* stage;                           // two blocks of 32 rows x 128 bytes
  int col, row, columns, lane;           // first column and row of the warp, columns that there are
  int place;                             // of the row's target (-1: not here) and its element
  float target;
};

// 64 elements of a row as 16-bit words to a block, and the target's.  Leaves what they leave of the elements, as the next piece has it, where LEAVE.
template <typename T, bool LEAVE>
__device__ __forceinline__ void dz_block(float* v, float& target, uint32_t keep, int place, int lane, char* block) {
  using Word = Word16<T>;
  constexpr float kGrow = std::is_same<T, __half>::value ? kSecond : 1.0f;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      float &x = v[8 * i + 2 * j], &y = v[8 * i + 2 * j + 1];
      w[j] = Word::join(x, y) & keep;
      if (LEAVE) {
        float wx, wy;
        Word::pair(w[j], wx, wy);
        x = (x - wx) * kGrow, y = (y - wy) * kGrow;
      }
    }
    reinterpret_cast<uint4*>(block)[lane * 8 + (i ^ (lane & 7))] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  if (place >= 0 && place < 64) {
    const T nearest = from_float<T>(target);
    reinterpret_cast<T*>(block)[(lane * 8 + ((place / 8) ^ (lane & 7))) * 8 + place % 8] = nearest;
    if (LEAVE) target = (target - to_float(nearest)) * kGrow;
  }
}

// -p (g + g_H (log p + H)) of N tokens of a row, from their logits, in blocks of 64 tokens that are
// copied from shared memory (rows of their own are 32-byte writes, which go out at a third of the rate).  `keep` 0: zeros.
// The forms are functions of their own so that no branch stands between the elements: with branches an element's chain of operations has nothing beside it.
template <bool ENTROPY, DzForm FORM, int N>
__device__ __forceinline__ void dz_row(const DzRow& r, float (&v)[N], uint32_t keep, const DzOut& out, int& turn) {
  Float2 mp = pack2(-r.peak, -r.peak);
  const Float2 ml = pack2(-r.log_sum, -r.log_sum), ml2 = pack2(-r.log_sum * kLog2e, -r.log_sum * kLog2e), l2e = pack2(kLog2e, kLog2e);
  const Float2 mg = pack2(-r.g, -r.g), mh = pack2(-r.gh, -r.gh), h2 = pack2(r.entropy, r.entropy);
#pragma unroll
  for (int c = 0; c < N; c += 64) {
    if (c >= out.columns) break;
#pragma unroll
    for (int i = c; i < c + 64; i += 2) {
      const Float2 x2 = add2(pack2(v[i], v[i + 1]), mp);
      float x, y;
      unpack2(fma2(x2, l2e, ml2), x, y);
      Float2 d = pack2(exp2_fast(x), exp2_fast(y));
      if (ENTROPY) {                         // (p = 0 where log p is -infinity, and no product with it)
        unpack2(add2(x2, ml), x, y);
        d = mul2(d, fma2(add2(pack2(fmaxf(x, kLeastLogp), fmaxf(y, kLeastLogp)), h2), mh, mg));
      } else d = mul2(d, mg);
      unpack2(d, v[i], v[i + 1]);
      if (i % 16 == 14) in_turn(mp, d);
    }
    float target = out.target;
    // the two blocks take turns: one is filled when the copy of what it held, the last but one, has read it
    auto free_block = [&] {
      if (out.lane == 0) stores_read<1>();
      __syncwarp();
      return out.stage + turn * 4096;
    };
    auto give = [&](int piece) {
      fence_async();
      __syncwarp();
      if (out.lane == 0) {
        store_block(out.map, out.col + c, out.row, piece, pipe::smem_addr(out.stage + turn * 4096));
        stores_commit();
      }
      turn ^= 1;
    };
    using T = typename std::conditional<FORM == kNearest || FORM == kPair, __half, __nv_bfloat16>::type;
    constexpr int kPieces = FORM == kNearest ? 1 : FORM == kWideTriple ? 3 : 2;
    dz_block<T, (kPieces > 1)>(v + c, target, keep, out.place - c, out.lane, free_block());
    give(0);
    if constexpr (kPieces > 1) {
      dz_block<T, (kPieces > 2)>(v + c, target, keep, out.place - c, out.lane, free_block());
      give(1);
    }
    if constexpr (kPieces > 2) {
      dz_block<T, false>(v + c, target, keep, out.place - c, out.lane, free_block());
      give(2);
    }
  }
}

// ------------------------------------------------------------------------------------------------------------ product

struct TileAt {
  int slab, m, n;                        // first row and column
};
// t / d with the reciprocal min(2^32 - 1, 2^32 / d + 1) at hand: off by one at most before the correction, and a fifth of a division's instructions.
__device__ __forceinline__ uint32_t quotient(uint32_t t, uint32_t d, uint32_t inverse) {
  uint32_t q = __umulhi(t, inverse);
  const int r = (int)(t - q * d);
  return r < 0 ? q - 1 : r >= (int)d ? q + 1 : q;
}
// Tiles of eight row tiles at a time, columns of those before the next eight: what runs at the same time shares rows of both operands in L2.
__device__ __forceinline__ TileAt tile_at(const HeadArgs& a, uint32_t t, int bn) {
  const uint32_t per_slab = (uint32_t)a.m_tiles * a.n_tiles, band = 8u * a.n_tiles;
  const uint32_t slab = quotient(t, per_slab, a.per_slab_inverse), r = t - slab * per_slab;
  const uint32_t group = quotient(r, band, a.band_inverse), in = r - group * band;
  const uint32_t high = min(8u, a.m_tiles - group * 8), column = high == 8 ? in >> 3 : in / high;
  return {(int)slab, (int)((group * 8 + in - column * high) * kTile), (int)column * bn};
}

constexpr int kLowChunk = 32;            // what is cut off of the second pieces' products lies 2^-8 or 2^-11 lower
// Where the blocks end that are summed in tensor memory together with block kb.
__device__ __forceinline__ int chunk_end(const HeadArgs& a, int kb, int blocks) {
  return kb < a.low ? min(a.low, kb + kLowChunk) : min(blocks, kb + a.chunk);
}

// stages of A and B blocks, then the epilogue warps' staging, then barriers
template <int MODE, int BN>
struct HeadShared {
  static constexpr int kStageBytes = (kRows + BN / 2) * kBlock * 2;
  static constexpr int kBlocks = MODE == kStats ? 0 : MODE == kDz || MODE == kDweight ? 8192 : 4096;     // a warp's blocks of the result
  static constexpr int kStaging = kBlocks + (MODE == kStats || MODE == kDz ? 2048 : 0);                   // and what the tile's rows and columns come with (blocks lie at multiples of 1024)
  static constexpr int kStages = (232448 - 2048 - kEpilogueWarps * kStaging) / kStageBytes > 12 ? 12 : (232448 - 2048 - kEpilogueWarps * kStaging) / kStageBytes;
  static constexpr int kBytes = 1024 + kStages * kStageBytes + kEpilogueWarps * kStaging + 512;
};

// Warps 0 and 2 of each CTA bring blocks, warp 1 of the first CTA multiplies, eight warps take finished sums from tensor memory, of which one half is read
// while the other is being filled, and keep a tile's result in registers: 128 columns of a row a thread.
// The tensor cores cut off what lies below an accumulator's last bit, which costs a sum of n steps of 16 about n / 2 units of 2^-25, always towards 0
// (measured: 1.6e-8 a step, 2e-5 for dh of 50,001 tokens).  So a result that is wanted in float32 is summed 512 inner indices at a time, and those sums are
// added in registers, rounded to nearest (256 at a time: 5 to 15 % slower; all at once: 1 % faster); logits from two pieces 256, the products with a second piece 2048.
// Persistent: a pair takes every (pairs)-th tile.
// Every wait ends after two seconds at the latest: the tiles of a CTA whose wait ran out are filled with NaN.
template <int MODE, int BN, bool BF16, typename O>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) head_product_kernel(const __grid_constant__ HeadMaps maps, const HeadArgs a) {
  constexpr bool kAlongA = MODE != kDweight, kAlongB = MODE == kStats || MODE == kFewRows || MODE == kDz;
  using Shared = HeadShared<MODE, BN>;
  constexpr int kStages = Shared::kStages, kStageBytes = Shared::kStageBytes;
  constexpr int kHalf = BN / 2;              // columns of an epilogue warp
  extern __shared__ char raw[];
  char* smem = (char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  char* staging = smem + kStages * kStageBytes;
  uint64_t* full = (uint64_t*)(staging + kEpilogueWarps * Shared::kStaging);
  uint64_t* empty = full + kStages;
  uint64_t* sum_full = empty + kStages;
  uint64_t* sum_empty = sum_full + 2;
  uint32_t* tmem_at = (uint32_t*)(sum_empty + 2);
  int* abort_flag = (int*)(tmem_at + 1);

  pdl_trigger();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  const uint32_t tiles_all = (uint32_t)a.m_tiles * a.n_tiles * a.slabs;
  const int blocks = a.products * a.k_blocks;
  int* status = &head_wait_status;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; i++) {
      pipe::mbar_init(full + i, 1);
      pipe::mbar_init(empty + i, 1);
    }
    for (int i = 0; i < 2; i++) {
      pipe::mbar_init(sum_full + i, 1);
      pipe::mbar_init(sum_empty + i, 2 * kEpilogueWarps);
    }
    *abort_flag = 0;
    pipe::fence_barrier_init();
  }
  if (warp == 1) tmem_alloc<2 * BN>(tmem_at);
  fence_before();
  __syncthreads();
  cluster_sync();
  fence_after();
  const uint32_t tmem = *tmem_at;
  pdl_wait();                            // up to here nothing of the kernels before is touched

  if (warp < kFirstEpilogue) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");        // 128 x 72 + 256 x 216 = 64512 = 384 x 168 at launch
    if ((warp == 0 || warp == 2) && lane == 0) {       // warp 0 brings A's blocks, warp 2 B's
      int s = 0;
      uint32_t phase = 0;
      bool fine = true;
      for (uint32_t t = pair; t < tiles_all && fine; t += pairs) {
        const TileAt at = tile_at(a, t, BN);
        const int row = at.m + rank * kRows, col = at.n + rank * kHalf;
        for (int p = 0; p < a.products && fine; p++) {
          const int part = a.splits > 1 ? at.slab / a.splits : at.slab, from = (at.slab - part * a.splits) * a.k_blocks * kBlock;
          const int z = warp == 0 ? a.piece_a[p] + part * a.slab_a : a.piece_b[p] + part * a.slab_b;
          for (int k = from; k < from + a.k_blocks * kBlock; k += kBlock) {
            if (!(fine = waited(empty + s, phase ^ 1, abort_flag, status))) break;
            const uint32_t dst = pipe::smem_addr(smem + s * kStageBytes);
            if (warp == 0) {
              if (rank == 0) pipe::mbar_arrive_expect_tx(full + s, 2 * kStageBytes);
              if (kAlongA) load_block(dst, &maps.a, k, row, z, full + s);
              else load_blocks(dst, &maps.a, k, row / kBlock, z, full + s);
            } else {
              if (kAlongB) load_block(dst + kRows * 128, &maps.b, k, col, z, full + s);
              else if (a.b_by_blocks) load_blocks(dst + kRows * 128, &maps.b, k, col / kBlock, z, full + s);
              else
#pragma unroll
                for (int h = 0; h < kHalf; h += kBlock) load_block(dst + kRows * 128 + h * 128, &maps.b, col + h, k, z, full + s);
            }
            if (++s == kStages) s = 0, phase ^= 1;
          }
        }
      }
      // the last products' arrivals at this CTA's barriers come before it ends
      if (warp == 0)
        for (int i = 0; i < kStages && fine; i++) {
          fine = waited(empty + s, phase ^ 1, abort_flag, status);
          if (++s == kStages) s = 0, phase ^= 1;
        }
    } else if (warp == 1 && lane == 0 && rank == 0) {
      constexpr uint32_t idesc = instruction(BF16, kAlongA, kAlongB, BN);
      int s = 0, half = 0;
      uint32_t phase = 0, sum_phase = 0;
      for (uint32_t t = pair; t < tiles_all; t += pairs) {
        for (int kb = 0; kb < blocks;) {
          if (!waited(sum_empty + half, sum_phase ^ 1, abort_flag, status)) goto products_done;
          fence_after();
          const int first = kb, end = chunk_end(a, kb, blocks);
          for (; kb < end; kb++) {
            if (!waited(full + s, phase, abort_flag, status)) goto products_done;
            fence_after();
            const uint32_t at = pipe::smem_addr(smem + s * kStageBytes);
            const uint64_t da = operand<kAlongA>(at), db = operand<kAlongB>(at + kRows * 128);
#pragma unroll
            for (int k = 0; k < kBlock / 16; k++)
              multiply(tmem + half * BN, da + k * kStep16<kAlongA>, db + k * kStep16<kAlongB>, idesc, kb > first || k > 0);
            commit_to_both(empty + s);
            if (++s == kStages) s = 0, phase ^= 1;
          }
          commit_to_both(sum_full + half);
          if ((half ^= 1) == 0) sum_phase ^= 1;
        }
      }
    products_done:;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int quarter = warp % 4, side = (warp - kFirstEpilogue) / 4;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    char* stage = staging + (warp - kFirstEpilogue) * Shared::kStaging;
    [[maybe_unused]] float undo_weight = 1.0f;
    if (MODE == kDhidden && a.weight_scaled) undo_weight = power_of_two(-scale_exponent(a.words->weight));
    uint32_t sum_phase = 0;
    int half = 0;
    [[maybe_unused]] int turn = 0;           // which of the warp's two blocks of the result is filled next
    [[maybe_unused]] RowSums rows_so_far[kHalf / 32];
    if constexpr (MODE == kFewRows) {
#pragma unroll
      for (int i = 0; i < kHalf / 32; i++) rows_so_far[i] = {-INFINITY, 0.0f, 0.0f};
    }
    for (uint32_t t = pair; t < tiles_all; t += pairs) {
      const TileAt at = tile_at(a, t, BN);
      const int row0 = at.m + rank * kRows + quarter * 32, row = row0 + lane, col = at.n + side * kHalf;
      const bool absent = row0 >= a.m || (MODE != kStats && col >= (MODE == kDz ? a.dz_pitch : a.n));     // nothing of the tile is this warp's
      // what the tile's rows come with is on the way to shared memory while the tile is being multiplied
      [[maybe_unused]] float* of_rows = reinterpret_cast<float*>(stage + Shared::kBlocks);
      [[maybe_unused]] int64_t* of_targets = reinterpret_cast<int64_t*>(of_rows + 6 * 32);
      [[maybe_unused]] const float* of_columns = of_rows + 256;
      if ((MODE == kStats || MODE == kDz) && !absent) {
        __syncwarp();
        const bool there = row < a.m;
        const int64_t at_row = there ? row : 0;
        if (a.targets) copy_async<8>(of_targets + lane, a.targets + at_row, there);
        if (a.undo_n) copy16_async(of_rows + 256 + 4 * lane, a.undo_n + a.first + col + 4 * lane);      // (there are columns enough for whole tiles)
        if constexpr (MODE == kDz) {
          copy_async<4>(of_rows + lane, a.peak + at_row, there);
          copy_async<4>(of_rows + 32 + lane, a.log_sum + at_row, there);
          copy_async<4>(of_rows + 160 + lane, a.undo_dz + at_row, there);
          if (a.grad_logp) copy_async<4>(of_rows + 64 + lane, a.grad_logp + at_row, there);
          if (a.grad_entropy) {
            copy_async<4>(of_rows + 96 + lane, a.entropy + at_row, there);
            copy_async<4>(of_rows + 128 + lane, a.grad_entropy + at_row, there);
          }
        }
        copies_commit();
      }
      float undo_row = 1.0f;
      [[maybe_unused]] float undo[2] = {1.0f, 1.0f};         // (a partition's exponent may be twice a float's)
      if (MODE != kDweight && a.undo_m && row < a.m) undo_row = a.undo_m[row];
      if (MODE == kDweight && a.parts) {
        const int exponent = part_exponent(a.parts[a.splits > 1 ? at.slab / a.splits : at.slab]);
        undo[0] = power_of_two(-(exponent / 2));
        undo[1] = power_of_two(exponent / 2 - exponent);
      }
      float v[kHalf];
#pragma unroll
      for (int i = 0; i < kHalf; i++) v[i] = 0.0f;
      for (int kb = 0; kb < blocks; kb = chunk_end(a, kb, blocks)) {
        const float so_far = kb && kb == a.low ? a.low_factor : 1.0f;
        const Float2 so_far2 = pack2(so_far, so_far);
        pipe::mbar_wait(sum_full + half, sum_phase, abort_flag, status);
        fence_after();
        if (!absent) {
        const uint32_t from = tmem + half * BN + side * kHalf + lanes;
#pragma unroll
        for (int c = 0; c < kHalf; c += 32) {
          float more[32];
          tmem_load32(from + c, more);
          tmem_wait();
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const Float2 sum = fma2(pack2(v[c + i], v[c + i + 1]), so_far2, pack2(more[i], more[i + 1]));
            unpack2(sum, v[c + i], v[c + i + 1]);
          }
        }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) arrive_at_first(sum_empty + half);
        if ((half ^= 1) == 0) sum_phase ^= 1;
      }
      if (absent) continue;
      if constexpr (MODE == kDhidden) {
        const float both = joint(undo_row, undo_weight);
#pragma unroll
        for (int i = 0; i < kHalf; i++) v[i] *= both;
      } else if constexpr (MODE == kDweight) {
#pragma unroll
        for (int i = 0; i < kHalf; i++) v[i] = v[i] * undo[0] * undo[1];
      } else {
        if (MODE != kFewRows) {
          copies_wait<0>();
          __syncwarp();
        }
        if (a.undo_n) {
          const float* columns = MODE == kFewRows ? a.undo_n + col : of_columns;
#pragma unroll
          for (int i = 0; i < kHalf; i += 4) {
            const float4 u = *reinterpret_cast<const float4*>(columns + i);
            v[i] *= joint(undo_row, u.x), v[i + 1] *= joint(undo_row, u.y), v[i + 2] *= joint(undo_row, u.z), v[i + 3] *= joint(undo_row, u.w);
          }
        }
      }
      if (*(volatile int*)abort_flag) {
#pragma unroll
        for (int i = 0; i < kHalf; i++) v[i] = __int_as_float(0x7FC00000);
      }
      if constexpr (MODE == kStats) {
        const int inside = a.n - col;
        if (inside < kHalf) {
#pragma unroll
          for (int i = 0; i < kHalf; i++)
            if (i >= inside) v[i] = -INFINITY;
        }
        if (row < a.m) {
          const int64_t token = a.targets ? of_targets[lane] - a.first - col : -1;
          if (token >= 0 && token < kHalf && token < inside) {
            float z = 0.0f;
#pragma unroll
            for (int i = 0; i < kHalf; i++) take_if(z, v[i], (int)token == i);
            a.target_logit[row] = z;
          }
          RowSums sums;
          row_sums(v, sums);
          float* p = a.partial + (int64_t)(at.n / kHalf + side) * 3 * a.m + row;
          p[0] = sums.m;
          p[a.m] = sums.s;
          p[2 * (int64_t)a.m] = sums.a;
        }
      } else if constexpr (MODE == kFewRows) {
        // lanes are tokens and columns are rows here: 32 x 32 of them are turned, so that a lane has 32 tokens of a row
        const int inside = a.m - row0;
        float4* turned = reinterpret_cast<float4*>(stage);
        const float* turned1 = reinterpret_cast<const float*>(stage);
#pragma unroll
        for (int c = 0; c < kHalf; c += 32) {
          if (col + c >= a.n || inside <= 0) break;
          __syncwarp();
          stage_rows(v + c, turned, lane);
          __syncwarp();
          float z[32];
#pragma unroll
          for (int r = 0; r < 32; r++) z[r] = turned1[(r * 8 + ((lane / 4) ^ (r & 7))) * 4 + lane % 4];
          if (inside < 32) {
#pragma unroll
            for (int r = 0; r < 32; r++)
              if (r >= inside) z[r] = -INFINITY;
          }
          const int mine = col + c + lane;
          const int64_t token = mine < a.n && a.targets ? a.targets[mine] - row0 : -1;
          if (token >= 0 && token < min(32, inside)) {
            const int r = (int)token;
            a.target_logit[mine] = turned1[(r * 8 + ((lane / 4) ^ (r & 7))) * 4 + lane % 4];
          }
          RowSums sums;
          row_sums(z, sums);
          rows_so_far[c / 32] = join(rows_so_far[c / 32], sums);
        }
      } else if constexpr (MODE == kDz) {
        const int64_t target = a.targets && row < a.m ? of_targets[lane] : -1;
        DzRow r = {of_rows[lane], of_rows[32 + lane], a.grad_entropy ? of_rows[96 + lane] : 0.0f, a.grad_logp && target >= 0 ? of_rows[64 + lane] : 0.0f,
                   a.grad_entropy ? of_rows[128 + lane] : 0.0f};
        const float undo_dz = of_rows[160 + lane];
        const bool active = undo_dz != 0.0f;
        if (a.form == kNearest || a.form == kPair) {          // (bfloat16 takes dz as it is)
          r.g *= inverse_power(undo_dz);
          r.gh *= inverse_power(undo_dz);
        }
        const uint32_t keep = active ? ~0u : 0u;
        const int64_t token = target - a.first - col, inside = a.vocab - (a.first + col);
        if (inside < kHalf) {                // (what lies beyond is multiplied by zeros and has to be a number: p = 0)
#pragma unroll
          for (int i = 0; i < kHalf; i++)
            if (i >= inside) v[i] = -INFINITY;
        }
        const bool hit = target >= 0 && token >= 0 && token < min((int64_t)kHalf, inside);
        float z = 0.0f;
        if (__any_sync(~0u, hit)) {
#pragma unroll
          for (int i = 0; i < kHalf; i++) take_if(z, v[i], (int)token == i);
        }
        float lp = 0.0f, d = 0.0f;
        if (hit) {                           // the target's element, with its g
          lp = (z - r.peak) - r.log_sum;
          d = active ? fmaf(exp2_fast(lp * kLog2e), fmaf(-r.gh, fmaxf(lp, kLeastLogp) + r.entropy, -r.g), r.g) : 0.0f;
        }
        const int place = hit ? (int)token : -1;
        const DzOut out = {&maps.out, stage, col, row0, a.dz_pitch - col, lane, place, d};
        auto rows = [&](auto entropy) {
          constexpr bool kEntropy = decltype(entropy)::value;
          if (a.form == kPair) dz_row<kEntropy, kPair>(r, v, keep, out, turn);
          else if constexpr (BF16) {
            if (a.form == kNearest) dz_row<kEntropy, kNearest>(r, v, keep, out, turn);
            else if (a.form == kWidePair) dz_row<kEntropy, kWidePair>(r, v, keep, out, turn);
            else dz_row<kEntropy, kWideTriple>(r, v, keep, out, turn);
          } else dz_row<kEntropy, kNearest>(r, v, keep, out, turn);
        };
        if (a.grad_entropy) rows(std::true_type{});
        else rows(std::false_type{});
      } else {
        // (the sums' pitch is a multiple of 128: room for all columns of a warp that has any)
        float* so_far = a.sums + ((int64_t)at.slab * a.m + row) * a.sums_pitch + col;
        const bool here = row < a.m && col < a.n;
        if (MODE == kDhidden && a.load_sums && here) {
#pragma unroll
          for (int c = 0; c < kHalf; c += 32) {
            float was[4][8];
#pragma unroll
            for (int i = 0; i < 4; i++) load32(so_far + c + 8 * i, was[i]);
#pragma unroll
            for (int i = 0; i < 32; i++) v[c + i] += was[i / 8][i % 8];
          }
        }
        O* out = (O*)a.out + (MODE == kDweight ? at.slab * a.out_slab : 0);
        if (a.store_sums) {
          if (here) store_columns<float, kHalf>(so_far, v);
        } else if (MODE == kDweight && a.out_by_map) {
          constexpr int kEach = 128 / sizeof(O);       // columns of a block
#pragma unroll
          for (int c = 0; c < kHalf; c += kEach) {
            if (col + c >= a.n || row0 >= a.m) break;
            uint4* block = reinterpret_cast<uint4*>(stage + turn * 4096);
            turn ^= 1;
            if (lane == 0) stores_read<1>();           // the block before the last one has left its place
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; i++) {
              const float* x = v + c + i * (kEach / 8);
              uint4 w;
              if constexpr (sizeof(O) == 4) w = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
              else if constexpr (sizeof(O) == 2)
                w = make_uint4(Word16<O>::join(x[0], x[1]), Word16<O>::join(x[2], x[3]), Word16<O>::join(x[4], x[5]), Word16<O>::join(x[6], x[7]));
              else
                w = make_uint4(__double2loint((double)x[0]), __double2hiint((double)x[0]), __double2loint((double)x[1]), __double2hiint((double)x[1]));
              block[lane * 8 + (i ^ (lane & 7))] = w;
            }
            fence_async();
            __syncwarp();
            if (lane == 0) {
              store_block(&maps.out, col + c, row0, at.slab, pipe::smem_addr(block));
              stores_commit();
            }
          }
        } else if (a.out_wide && col + kHalf <= a.n) {
          if (row < a.m) store_columns<O, kHalf>(out + (int64_t)row * a.out_pitch + col, v);
        } else {
          float4* rows = reinterpret_cast<float4*>(stage);
#pragma unroll
          for (int c = 0; c < kHalf; c += 32) {
            if (col + c >= a.n || row0 >= a.m) break;
            __syncwarp();
            stage_rows(v + c, rows, lane);
            __syncwarp();
            write_rows(rows, out, a.out_pitch, row0, col + c, a.m, a.n, lane);
          }
        }
      }
    }
    if constexpr (MODE == kFewRows) {
#pragma unroll
      for (int c = 0; c < kHalf; c += 32) {
        const int mine = side * kHalf + c + lane;
        if (mine < a.n) {
          float* p = a.partial + (int64_t)(blockIdx.x * 4 + quarter) * 3 * a.n + mine;
          p[0] = rows_so_far[c / 32].m;
          p[a.n] = rows_so_far[c / 32].s;
          p[2 * (int64_t)a.n] = rows_so_far[c / 32].a;
        }
      }
    }
  }
  if ((MODE == kDz || MODE == kDweight) && warp >= kFirstEpilogue && lane == 0) stores_done();
  if (*(volatile int*)abort_flag) pipe::drain_delay();
  __syncwarp();
  fence_before();
  __syncthreads();
  cluster_sync();
  fence_after();
  if (warp == 1) tmem_free<2 * BN>(tmem);
}

// ------------------------------------------------------------------------------------------------------------ few rows

struct HeadRowsArgs {
  const void *hidden, *weight;
  int64_t hidden_pitch, weight_pitch, cols, vocab;
  const int64_t* targets;
  int rows, padded;                      // padded: columns of a row of hidden in shared memory
  float *partial, *target_logit;
};

// Up to NR rows: a warp takes R rows of W at a time against the hidden rows in shared memory (float32), a lane G groups of EACH consecutive columns
// 32 EACH apart, and adds the products up over its lanes so that each lane ends with one logit, or a part of a set of lanes.  W is read once; the
// next columns are on the way while these are multiplied.
template <typename T, int NR, int R, int EACH, int G>
__global__ void __launch_bounds__(256, 2) head_rows_kernel(HeadRowsArgs a) {
  extern __shared__ __align__(16) float hidden_smem[];
  __shared__ RowSums merged[8][NR];
  pdl_trigger();
  constexpr int kCount = NR * R, kStep = 32 * EACH * G;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int n = 0; n < NR; n++)
    for (int k = threadIdx.x; k < a.padded; k += 256)
      hidden_smem[n * a.padded + k] = n < a.rows && k < a.cols ? to_float(((const T*)a.hidden)[n * a.hidden_pitch + k]) : 0.0f;
  __syncthreads();
  RowSums sums = {-INFINITY, 0.0f, 0.0f};
  constexpr int kShift = kCount == 32 ? 0 : kCount == 16 ? 1 : kCount == 8 ? 2 : 3;
  const int index = lane >> kShift, mine_row = index / R, mine_token = index % R;
  const bool counts = (lane & ((1 << kShift) - 1)) == 0 && mine_row < a.rows;
  const int64_t target = counts && a.targets ? a.targets[mine_row] : -1;
  const int64_t groups = (a.vocab + R - 1) / R;
  for (int64_t g = (int64_t)blockIdx.x * 8 + warp; g < groups; g += (int64_t)gridDim.x * 8) {
    const int64_t v0 = g * R;
    float acc[kCount];
#pragma unroll
    for (int i = 0; i < kCount; i++) acc[i] = 0.0f;
    const T* w[R];
#pragma unroll
    for (int r = 0; r < R; r++) w[r] = (const T*)a.weight + min(v0 + r, a.vocab - 1) * a.weight_pitch;
    Pack<T, EACH> x[R][G], next[R][G];
    auto fetch = [&](Pack<T, EACH> (&to)[R][G], int k0) {         // (EACH divides the number of columns)
#pragma unroll
      for (int q = 0; q < G; q++) {
        const int k = k0 + (q * 32 + lane) * EACH;
#pragma unroll
        for (int r = 0; r < R; r++) {
          to[r][q] = {};
          if (k < a.cols) to[r][q] = load_pack<T, EACH>(w[r] + k);
        }
      }
    };
    fetch(x, 0);
    for (int k0 = 0; k0 < a.cols; k0 += kStep) {
      if (k0 + kStep < a.cols) fetch(next, k0 + kStep);
#pragma unroll
      for (int q = 0; q < G; q++) {
        const int k = k0 + (q * 32 + lane) * EACH;
#pragma unroll
        for (int n = 0; n < NR; n++) {
          const Pack<float, EACH> h = load_pack<float, EACH>(hidden_smem + n * a.padded + k);
#pragma unroll
          for (int r = 0; r < R; r++)
#pragma unroll
            for (int e = 0; e < EACH; e++) acc[n * R + r] = fmaf(to_float(x[r][q].e[e]), h.e[e], acc[n * R + r]);
        }
      }
#pragma unroll
      for (int r = 0; r < R; r++)
#pragma unroll
        for (int q = 0; q < G; q++) x[r][q] = next[r][q];
    }
#pragma unroll
    for (int o = 16, half = kCount / 2; o > 0; o /= 2, half /= 2) {
      if (half > 0) {
#pragma unroll
        for (int i = 0; i < half; i++) {
          const float keep = lane & o ? acc[i + half] : acc[i], give = lane & o ? acc[i] : acc[i + half];
          acc[i] = keep + __shfl_xor_sync(~0u, give, o);
        }
      } else acc[0] += __shfl_xor_sync(~0u, acc[0], o);
    }
    const int64_t token = v0 + mine_token;
    if (counts && token < a.vocab) {
      if (token == target) a.target_logit[mine_row] = acc[0];
      sums = join(sums, {acc[0], acc[0] == -INFINITY ? 0.0f : 1.0f, 0.0f});
    }
  }
#pragma unroll
  for (int o = 1; o < 32 / NR; o *= 2)
    sums = join(sums, {__shfl_xor_sync(~0u, sums.m, o), __shfl_xor_sync(~0u, sums.s, o), __shfl_xor_sync(~0u, sums.a, o)});
  if (lane % (32 / NR) == 0) merged[warp][lane / (32 / NR)] = sums;
  __syncthreads();
  if (threadIdx.x < a.rows) {
    RowSums r = merged[0][threadIdx.x];
    for (int i = 1; i < 8; i++) r = join(r, merged[i][threadIdx.x]);
    float* p = a.partial + (int64_t)blockIdx.x * 3 * a.rows + threadIdx.x;
    p[0] = r.m;
    p[a.rows] = r.s;
    p[2 * a.rows] = r.a;
  }
}

// ------------------------------------------------------------------------------------------------------------ joining, scanning, splitting

struct HeadJoinArgs {
  const float *partial, *target_logit;
  int64_t rows, slots, vocab;
  const int64_t* targets;
  float *logp, *entropy, *peak, *log_sum;
};

// The sums of a row's parts, 256 / ROWS threads a row, joined in an order that the sizes fix.
template <int ROWS>
__global__ void __launch_bounds__(256) head_join_kernel(HeadJoinArgs a) {
  constexpr int kGroups = 256 / ROWS;
  __shared__ RowSums part[kGroups][ROWS];
  const int r = threadIdx.x % ROWS, group = threadIdx.x / ROWS;
  const int64_t row = (int64_t)blockIdx.x * ROWS + r;
  RowSums sums = {-INFINITY, 0.0f, 0.0f};
  pdl_wait();
  if (row < a.rows)
#pragma unroll 4
    for (int64_t s = group; s < a.slots; s += kGroups) {
      const float* p = a.partial + s * 3 * a.rows + row;
      sums = join(sums, {p[0], p[a.rows], p[2 * a.rows]});
    }
  part[group][r] = sums;
  for (int half = kGroups / 2; half > 0; half /= 2) {
    __syncthreads();
    if (group < half) part[group][r] = join(part[group][r], part[group + half][r]);
  }
  if (group || row >= a.rows) return;
  sums = part[0][r];
  const bool empty = sums.m == -INFINITY;
  const float log_sum = empty ? 0.0f : logf(sums.s);
  if (a.peak) a.peak[row] = sums.m;
  if (a.log_sum) a.log_sum[row] = log_sum;
  if (a.entropy) a.entropy[row] = empty ? 0.0f : log_sum - sums.a / sums.s;
  if (a.logp) {
    const int64_t t = a.targets[row];
    a.logp[row] = t < 0 ? 0.0f : t >= a.vocab ? __int_as_float(0x7FC00000) : empty ? -INFINITY : (a.target_logit[row] - sums.m) - log_sum;
  }
}

// Eight elements of a row from column c on, zeros behind its end.  WIDE: rows lie at multiples of 16 bytes.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int64_t c, int64_t cols, bool wide, float (&v)[8]) {
  if (wide && c + 8 <= cols) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(p + c);
      *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(p + c + 4);
    } else {
      Word16<T>::unpack(*reinterpret_cast<const uint4*>(p + c), v);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = c + e < cols ? to_float(p[c + e]) : 0.0f;
  }
}
// Two float16 pieces of eight elements times `scale`, `rest` elements apart.
__device__ __forceinline__ void store_pieces(const float (&v)[8], float scale, __half* out, int64_t rest) {
  Pack<__half, 8> hi, lo;
#pragma unroll
  for (int e = 0; e < 8; e++) {
    const float y = v[e] * scale;
    hi.e[e] = __float2half_rn(y);
    lo.e[e] = __float2half_rn(fabsf(y) < INFINITY ? (y - __half2float(hi.e[e])) * kSecond : 0.0f);      // (infinity and NaN: the first piece alone says so)
  }
  store_pack(out, hi);
  store_pack(out + rest, lo);
}

struct HeadScanSide {
  const void* x;                         // NULL: not wanted
  int64_t pitch, rows;
  __half* out;                           // float32: the pieces of each row by an exponent of its own, and what they are multiplied by to undo it; 16-bit hidden states: a
                                         // copy with zeros for rows without a share (NULL: not wanted)
  float* undo;
  unsigned* largest;                     // of the whole matrix (NULL: not wanted)
};
struct HeadScanArgs {
  HeadScanSide side[2];                  // hidden states, output matrix
  int64_t cols, out_pitch, rows;
  const int64_t* targets;
  const float *peak, *grad_logp, *grad_entropy, *entropy;
  float* undo_dz;                        // of each row (NULL: not wanted)
  unsigned* parts;                       // words of the partitions of n rows (NULL: not wanted)
  int64_t n;
};

// What row r's dz is multiplied by where it has been used: a power of two from |g| + |g_H| (H + 1), which no element exceeds.  0 where the row has no share: g counts only
// with a target, and nothing counts in a row of which nothing is left.
__device__ __forceinline__ float row_share(const HeadScanArgs& a, int64_t r) {
  const float g = a.grad_logp && a.targets[r] >= 0 ? fabsf(a.grad_logp[r]) : 0.0f, gh = a.grad_entropy ? fabsf(a.grad_entropy[r]) : 0.0f;
  if (a.peak[r] == -INFINITY || (g == 0.0f && gh == 0.0f)) return 0.0f;
  return power_of_two(-scale_exponent(min(__float_as_uint(gh == 0.0f ? g : g + gh * (fabsf(a.entropy[r]) + 1.0f)) & 0x7FFFFFFFu, 0x7F7FFFFFu)));
}

// Powers of two: of rows of float32 hidden states and weights, of the whole output matrix, of the rows' dz and of the partitions.
// float32 rows leave as two pieces on the way, by TEAM threads a row, which hold its first 32 TEAM elements in registers (the rest is read twice): W comes from memory once,
// where an exponent for the whole matrix took a pass of its own before the pieces (50001 x 1001: 116 us together), and no row's exponent is its neighbour's.
template <typename T, int TEAM>
__global__ void __launch_bounds__(256) head_scan_kernel(HeadScanArgs a) {
  __shared__ unsigned most[8], row_most[8];
  pdl_trigger();
  unsigned big = 0;
  auto see = [](unsigned& most, float x) {
    const unsigned u = __float_as_uint(x) & 0x7FFFFFFFu;
    if (u < 0x7F800000u) most = max(most, u);
  };
  const int warp = threadIdx.x / 32, lane = threadIdx.x % TEAM;
  unsigned* word = nullptr;
  if (blockIdx.y == 2) {
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.rows; r += (int64_t)gridDim.x * 256) a.undo_dz[r] = row_share(a, r);
  } else {
    const HeadScanSide m = blockIdx.y ? a.side[1] : a.side[0];
    if (!m.x) return;
    word = m.largest;
    const bool wide = !(((uintptr_t)m.x | (uintptr_t)(m.pitch * sizeof(T))) & 15);
    if (sizeof(T) == 4 && blockIdx.x == 0 && m.rows + threadIdx.x < (m.rows + kTile - 1) / kTile * kTile) m.undo[m.rows + threadIdx.x] = 1.0f;      // (of whole tiles)
    constexpr int kTeams = 256 / TEAM, kGroups = sizeof(T) == 4 ? 4 : 1;
    for (int64_t r = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM; r < m.rows; r += (int64_t)gridDim.x * kTeams) {
      const T* p = (const T*)m.x + r * m.pitch;
      unsigned row = 0;
      float held[kGroups][8];
#pragma unroll
      for (int q = 0; q < kGroups; q++) load8(p, (q * TEAM + lane) * 8, a.cols, wide, held[q]);
#pragma unroll
      for (int q = 0; q < kGroups; q++)
#pragma unroll
        for (int e = 0; e < 8; e++) see(row, held[q][e]);
#pragma unroll 4
      for (int64_t c = (kGroups * TEAM + lane) * 8; c < a.cols; c += TEAM * 8) {
        float v[8];
        load8(p, c, a.cols, wide, v);
#pragma unroll
        for (int e = 0; e < 8; e++) see(row, v[e]);
      }
      const bool to_part = blockIdx.y == 0 && a.parts;
      if (sizeof(T) == 4 || to_part) {
        row = __reduce_max_sync(~0u, row);
        if (TEAM > 32) {
          __syncthreads();
          if (threadIdx.x % 32 == 0) row_most[warp] = row;
          __syncthreads();
#pragma unroll
          for (int i = 0; i < 8; i++) row = max(row, row_most[i]);
        }
      }
      if (to_part && lane == 0 && row) {
        const float share = row_share(a, r);
        const unsigned there = share == 0.0f ? 0 : kPartBias + max(ilogbf(__uint_as_float(row)), -112) + exponent_of(share);
        if (there > __ldcg(a.parts + r / a.n)) atomicMax(a.parts + r / a.n, there);
      }
      if constexpr (sizeof(T) == 4) {
        const int exponent = scale_exponent(row);
        const float scale = power_of_two(exponent);
        __half* out = m.out + r * a.out_pitch;
        const int64_t rest = m.rows * a.out_pitch;
#pragma unroll
        for (int q = 0; q < kGroups; q++) {
          const int64_t c = (q * TEAM + lane) * 8;
          if (c < a.out_pitch) store_pieces(held[q], scale, out + c, rest);
        }
#pragma unroll 2
        for (int64_t c = (kGroups * TEAM + lane) * 8; c < a.out_pitch; c += TEAM * 8) {
          float v[8];
          load8(p, c, a.cols, wide, v);
          store_pieces(v, scale, out + c, rest);
        }
        if (lane == 0) m.undo[r] = power_of_two(-exponent);
      } else if (m.out) {
        const bool counts = row_share(a, r) != 0.0f;
        for (int64_t c = lane * 8; c < a.out_pitch; c += TEAM * 8) {
          float v[8];
          load8(p, c, counts ? a.cols : 0, wide, v);
          *reinterpret_cast<uint4*>(m.out + r * a.out_pitch + c) = Word16<T>::pack(v);
        }
      }
      big = max(big, row);
    }
  }
  if (!word) return;
  big = __reduce_max_sync(~0u, big);
  if (threadIdx.x % 32 == 0) most[warp] = big;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 8; i++) big = max(big, most[i]);
    if (big) atomicMax(word, big);
  }
}

// By which powers of two a matrix is taken in pieces: its own, or what each row lacks to its partition's; none for elements that stay as they are.
struct HeadScale {
  const unsigned* largest;
  const float* undo_dz;
  const unsigned* parts;
  int64_t n;
};

// Rows of a matrix at a pitch that tensor copies can take, zeros behind their ends: float32 as two float16 pieces, bfloat16 and float16 as one, 16-bit elements
// (of type uint16_t here) as they are.  Rows without a share are zeros.
template <typename T>
__global__ void __launch_bounds__(256) head_split_kernel(const T* x, int64_t pitch, int64_t rows, int64_t cols, uint16_t* out, int64_t out_pitch, HeadScale by) {
  pdl_trigger();
  pdl_wait();
  const int64_t words = out_pitch / 8;
  constexpr bool kAsIs = std::is_same<T, uint16_t>::value;
  const float whole = by.largest ? power_of_two(scale_exponent(*by.largest)) : 1.0f;
  const bool wide = !(((uintptr_t)x | (uintptr_t)(pitch * sizeof(T))) & 15);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * words; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / words, c = (i - r * words) * 8;
    if constexpr (kAsIs) {
      Pack<uint16_t, 8> v;
#pragma unroll
      for (int e = 0; e < 8; e++) v.e[e] = c + e < cols ? x[r * pitch + c + e] : (uint16_t)0;
      store_pack(out + r * out_pitch + c, v);
    } else {
      float v[8], scale = whole;
      load8(x + r * pitch, c, cols, wide, v);
      if (by.undo_dz) {
        const float undo = by.undo_dz[r];
        const int exponent = undo == 0.0f ? -127 : part_exponent(by.parts[r / by.n]) + exponent_of(undo);
        scale = exponent < -126 ? 0.0f : power_of_two(min(exponent, 126));        // (above 126 only where a row is nothing but zeros)
        if (scale == 0.0f)
#pragma unroll
          for (int e = 0; e < 8; e++) v[e] = 0.0f;
      }
      if constexpr (sizeof(T) == 4) {
        store_pieces(v, scale, (__half*)out + r * out_pitch + c, rows * out_pitch);
      } else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] *= scale;
        *reinterpret_cast<uint4*>(out + r * out_pitch + c) = Word16<__half>::pack(v);
      }
    }
  }
}

// Adds up the parts of a product whose inner dimension was cut: parts x splits x m x pitch float32 to parts x m x n elements.
struct HeadFinishArgs {
  const float* sums;
  int64_t pitch, m, n, out_pitch, out_slab;
  int parts, splits;
  void* out;
};
template <typename O>
__global__ void __launch_bounds__(256) head_finish_kernel(HeadFinishArgs a) {
  pdl_trigger();
  pdl_wait();
  const int64_t words = (a.n + 3) / 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.parts * a.m * words; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / words, c = (i - r * words) * 4, part = r / a.m, row = r - part * a.m;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int s = 0; s < a.splits; s++) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(a.sums + ((part * a.splits + s) * a.m + row) * a.pitch + c));
      sum = make_float4(sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w);
    }
    O* p = (O*)a.out + part * a.out_slab + row * a.out_pitch + c;
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
    for (int e = 0; e < 4 && c + e < a.n; e++) store1(p + e, v[e]);
  }
}

// ------------------------------------------------------------------------------------------------------------ host

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// What a call keeps where: offsets into the workspace, in bytes.
struct HeadPlan {
  // few rows
  int row_kernel;                        // 0, or the number of rows that the kernel of multiply-adds is built for
  bool few;                              // the product is taken the other way round
  int small;                             // float32: 0, or the number of rows that the kernels of head_rows.cu are built for
  int64_t turned;
  int64_t slots;
  // products
  int pieces;                            // of hidden and weight
  bool split;                            // hidden and weight are brought to a layout of their own
  int64_t pitch;                         // of theirs
  bool as_is;                            // bfloat16 states and weights go into dh and dW as they are
  int dz_pieces;
  int64_t width;                         // tokens of a piece of the vocabulary
  int h_splits, w_splits;                // parts of the inner dimensions of dh and dW
  int64_t undo_hidden, undo_weight;      // float32: what the pieces' rows are multiplied by
  int64_t undo_dz;
  int64_t hidden_w, weight_h;            // as they go into dW and, a piece of the vocabulary at a time, into dh
  int64_t words, partial, target_logit, hidden, weight, dz, sums, w_sums, total;
};

constexpr int64_t kHeadSharedRows = 200 * 1024;       // bytes of hidden rows that the kernel for few rows holds
constexpr int kRowBlocks = 148 * 2;

constexpr int kFewMost = 128;
constexpr int kFewPairs = 74;

static int64_t rows_padded(int64_t cols) { return up(cols, 256); }

static HeadPlan head_forward_plan(int64_t rows, int64_t cols, int64_t vocab, int dtype, bool aligned) {
  HeadPlan p = {};
  // W has to be read once and is all there is to read.  Up to 4 rows multiply-adds keep up with that, at any type and alignment; up to 32 float32 rows they cost
  // less than bringing W into two pieces first (65536 x 2048: 16 rows 446 us in pieces), except over a small vocabulary (9 rows of 2307 over 1702 tokens:
  // 190 us, seven tiles on seven SMs).
  if (rows <= 4 && (dtype == SOLON_F32 || !aligned)) {
    const int nr = rows == 3 ? 4 : (int)rows;
    if (nr * rows_padded(cols) * 4 <= kHeadSharedRows) p.row_kernel = nr;
  }
  if (!p.row_kernel && dtype == SOLON_F32 && rows <= kSmallForward && vocab >= kSmallVocab) p.small = small_rows(rows);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += up(bytes, 256);
    return here;
  };
  p.target_logit = take(rows * 4);
  if (p.row_kernel) {
    p.slots = kRowBlocks;
  } else if (p.small) {
    p.slots = (vocab + small_tile() - 1) / small_tile();
    p.turned = take(up(cols, 32) * p.small * 4);
  } else {
    // Up to 128 rows are the columns of tiles, not their rows: half the products of a tile that is mostly empty.
    p.few = rows <= kFewMost;
    const int64_t tiles = (vocab + kTile - 1) / kTile;
    p.slots = p.few ? 8 * std::min<int64_t>(tiles, kFewPairs) : 2 * tiles;
    p.pieces = dtype == SOLON_F32 ? 2 : 1;
    p.split = dtype == SOLON_F32 || !aligned;
    p.pitch = up(cols, kBlock);
    if (p.split) {
      p.hidden = take(p.pieces * rows * p.pitch * 2);
      p.weight = take(p.pieces * vocab * p.pitch * 2);
    }
    if (dtype == SOLON_F32) {
      p.undo_hidden = take(up(rows, kTile) * 4);
      p.undo_weight = take(up(vocab, kTile) * 4);
    }
  }
  p.partial = take(p.slots * 3 * rows * 4);
  p.total = at;
  return p;
}

// dlogits in memory at a time.  (Gradient of 16384 x 1024 over 15 x 512 rows: 1210 us with 128 MB, 1071 with 256, 1040 with 512, 992 with 1024.)
constexpr int64_t kDzBytes = 512ll << 20;

// 128 columns a tile instead of 256: where there are no more, and where that covers them with a sixth less and little is multiplied (`blocks` of 64 inner
// indices), so that writing the result is what takes time.  The tensor cores take a tile of 128 no less time than one of 256.  (Gradient of 32768 x 2048
// over 8192 rows 1374 against 716 us, of 2003 x 333 over 45 x 64 rows 54 against 73.)
static bool narrow(int64_t cols, int64_t blocks) { return cols <= 128 || (blocks <= 8 && up(cols, 128) * 6 <= up(cols, 256) * 5); }

// Into how many parts the inner dimension of a product of `slabs` times m x n is cut, where it has too few tiles for the 74 pairs of CTAs or a last round that
// is mostly empty.  A block of 64 indices takes a tile 0.3 us, a tile 1.5 us besides; parts are written and read once
// more at 5 TB/s by a launch of their own of 4 us.
static int head_splits(int64_t slabs, int64_t m, int64_t n, int64_t k, int products, int times) {
  const int64_t kb = (k + kBlock - 1) / kBlock;
  const int64_t bn = narrow(n, kb * products) ? 128 : kTile, tiles = slabs * ((m + kTile - 1) / kTile) * (up(n, bn) / bn);
  const double block = 0.3 * products, bytes = (double)slabs * m * up(n, 128) * 4;
  int best = 1;
  double least = 0.0;
  for (int s = 1; s <= 16 && (s == 1 || kb / s >= 4); s++) {
    const int64_t rounds = (tiles * s + 73) / 74;
    const double cost = times * rounds * ((kb + s - 1) / s * block + 1.5) + (s > 1 ? 4.0 + s * bytes * 2 * times / 5e6 : bytes * 2 * (times - 1) / 5e6);
    if (s == 1 || cost < 0.95 * least) best = s, least = cost;
  }
  return best;
}

// bfloat16 states: up to so many rows dh is taken from two bfloat16 pieces of dz and W as it lies, and dW from two or three of them.  Beyond, one float16 piece makes one
// product of two, and W as float16 (scan, copy: three times its size, 0.9 ps an element) costs less than the other (1.4 fs an element and row).
constexpr int kAsIsRows = 512;

// Pairs of pieces that dh and dW are the sums of.
static int dh_products(const HeadPlan& p, int dtype) { return dtype == SOLON_F32 ? 3 : dtype == SOLON_F16 || p.as_is ? 2 : 1; }
static int dw_products(const HeadPlan& p, int grad_dtype) { return p.as_is ? (grad_dtype == SOLON_BF16 ? 2 : 3) : grad_dtype == SOLON_BF16 ? 1 : p.pieces + 1; }

static HeadPlan head_backward_plan(int64_t rows, int64_t cols, int64_t vocab, int partitions, int dtype, int grad_dtype, bool aligned) {
  HeadPlan p = {};
  p.pieces = dtype == SOLON_F32 ? 2 : 1;
  p.split = dtype == SOLON_F32 || !aligned;
  p.pitch = up(cols, kBlock);
  p.as_is = dtype == SOLON_BF16 && rows <= kAsIsRows;
  p.dz_pieces = p.as_is ? (grad_dtype == SOLON_BF16 ? 2 : 3) : dtype == SOLON_BF16 && grad_dtype == SOLON_BF16 ? 1 : 2;
  p.width = std::max<int64_t>(kTile, kDzBytes / (rows * 2 * p.dz_pieces) / kTile * kTile);
  p.width = std::min(up(vocab, 64), up((vocab + (vocab + p.width - 1) / p.width - 1) / ((vocab + p.width - 1) / p.width), kTile));     // pieces of one size
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += up(bytes, 256);
    return here;
  };
  if (dtype == SOLON_F32 && rows <= kSmallBackward && vocab >= kSmallVocab) {      // (13 rows of 3456 over 37760 tokens: 755 us in pieces)
    p.small = small_rows(rows);
    p.h_splits = small_splits(cols, vocab);
    p.turned = take(up(cols, 32) * p.small * 4);
    p.dz = take((vocab + 64) * p.small * 4);
    p.sums = take(p.h_splits * rows * up(cols, 128) * 4);
    p.total = at;
    return p;
  }
  const int times = (int)((vocab + p.width - 1) / p.width);
  p.h_splits = head_splits(1, rows, cols, std::min(vocab, p.width), dh_products(p, dtype), times);
  p.w_splits = head_splits(partitions, std::min(vocab, p.width), cols, rows / partitions, dw_products(p, grad_dtype), 1);
  p.words = take(sizeof(HeadWords) + partitions * 4);
  p.undo_dz = take(rows * 4);
  if (p.split) {
    p.hidden = take(p.pieces * rows * p.pitch * 2);
    p.weight = take(p.pieces * vocab * p.pitch * 2);
  }
  if (dtype == SOLON_F32) {
    p.undo_hidden = take(up(rows, kTile) * 4);
    p.undo_weight = take(up(vocab, kTile) * 4);
  }
  p.hidden_w = take(p.pieces * rows * p.pitch * 2);
  if (dtype != SOLON_F16 && !p.as_is) p.weight_h = take(p.pieces * p.width * p.pitch * 2);
  p.dz = take(p.dz_pieces * rows * p.width * 2);
  if (times > 1 || p.h_splits > 1) p.sums = take(p.h_splits * rows * up(cols, 128) * 4);
  if (p.w_splits > 1) p.w_sums = take((int64_t)p.w_splits * partitions * std::min(vocab, p.width) * up(cols, 128) * 4);
  p.total = at;
  return p;
}

static bool aligned16(const void* p, int64_t pitch, int64_t rows, int dtype) {
  return !(((uintptr_t)p & 15) || (rows > 1 && (pitch * element_size(dtype)) & 15));
}

template <typename T, int NR, int R, int EACH, int G>
static int head_rows_launch(const HeadRowsArgs& a, cudaStream_t stream) {
  const size_t smem = (size_t)NR * a.padded * 4;
  SOLON_SHARED_MEMORY_ONCE((head_rows_kernel<T, NR, R, EACH, G>), kHeadSharedRows);
  head_rows_kernel<T, NR, R, EACH, G><<<kRowBlocks, 256, smem, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

template <typename T, int EACH, int G>
static int head_rows_e(const HeadRowsArgs& a, int nr, cudaStream_t stream) {
  switch (nr) {
    case 1: return head_rows_launch<T, 1, sizeof(T) == 4 ? 8 : 4, EACH, G>(a, stream);
    case 2: return head_rows_launch<T, 2, 4, EACH, G>(a, stream);
    default: return head_rows_launch<T, 4, 4, EACH, G>(a, stream);
  }
}

// As many consecutive columns an access as every row's alignment and the number of columns allow, 16 to 32 bytes a row of W and lane.
template <typename T>
static int head_rows_t(const HeadRowsArgs& a, int nr, cudaStream_t stream) {
  const uintptr_t both = (uintptr_t)a.weight | (uintptr_t)((a.weight_pitch | a.cols) * sizeof(T));
  if constexpr (sizeof(T) == 4) {
    if (!(both & 15)) return head_rows_e<T, 4, 1>(a, nr, stream);
    return head_rows_e<T, 1, 4>(a, nr, stream);
  } else {
    if (!(both & 3)) return head_rows_e<T, 2, 4>(a, nr, stream);
    return head_rows_e<T, 1, 8>(a, nr, stream);
  }
}

template <int MODE, int BN, bool BF16, typename O>
static int head_product_launch(const HeadMaps& maps, HeadArgs a, int sms, cudaStream_t stream) {
  auto* kernel = head_product_kernel<MODE, BN, BF16, O>;
  constexpr int bytes = HeadShared<MODE, BN>::kBytes;
  a.m_tiles = (a.m + kTile - 1) / kTile;
  a.n_tiles = (a.n + BN - 1) / BN;
  a.low = (a.products - 1) * a.k_blocks;
  if (!a.low_factor) a.low_factor = 1.0f / kSecond;
  // (what is cut off of a logit is a relative error of its probability: 256 inner indices for float32, 128 in the gradient of few rows, where memory is what takes time.
  // 45 x 64 rows x 333 float32: dW 1.7e-6 off with 512, 1.0e-6 so; 16 x 768: 1.8e-6, 6.5e-7.  One row's logits with 128: 100 us instead of 90.)
  if (MODE == kDhidden || MODE == kDweight) a.chunk = sizeof(O) == 2 ? 64 : 8;
  else a.chunk = MODE == kDz && a.m <= 512 ? 2 : a.products == 3 ? 4 : 8;
  const int64_t tiles = (int64_t)a.m_tiles * a.n_tiles * a.slabs;
  if (tiles > 0x3FFFFFFF) return SOLON_ERR_INVALID_ARG;
  auto inverse = [](int64_t d) { return (uint32_t)std::min<int64_t>(0xFFFFFFFF, (1ll << 32) / d + 1); };
  a.per_slab_inverse = inverse((int64_t)a.m_tiles * a.n_tiles);
  a.band_inverse = inverse(8ll * a.n_tiles);
  const int pairs = (int)std::min<int64_t>(tiles, MODE == kFewRows ? std::min(kFewPairs, sms / 2) : sms / 2);
  SOLON_SHARED_MEMORY_ONCE(kernel, bytes);
  return launch_dependent(kernel, dim3(2 * pairs), dim3(kThreads), bytes, stream, maps, a);
}

template <int MODE, bool BF16, typename O>
static int head_product(const HeadMaps& maps, const HeadArgs& a, int sms, cudaStream_t stream) {
  if (a.narrow) return head_product_launch<MODE, 128, BF16, O>(maps, a, sms, stream);
  return head_product_launch<MODE, 256, BF16, O>(maps, a, sms, stream);
}

// A matrix as the products take it: where its pieces lie.
struct HeadOperand {
  const char* p;
  int64_t pitch, rows;
  int pieces;
};

// The elements as they are: where they lie, or copied to a pitch that tensor copies can take.
static int head_operand(const void* x, int64_t pitch, int64_t rows, int64_t cols, const HeadPlan& plan, char* to, int sms, cudaStream_t stream, HeadOperand* out) {
  if (!plan.split) {
    *out = {(const char*)x, rows > 1 ? pitch : up(cols, 8), rows, 1};
    return SOLON_OK;
  }
  const int64_t words = rows * (plan.pitch / 8);
  *out = {to, plan.pitch, rows, 1};
  return launch_dependent(head_split_kernel<uint16_t>, dim3((unsigned)std::min<int64_t>((words + 255) / 256, 16 * sms)), dim3(256), 0, stream, (const uint16_t*)x,
                          pitch, rows, cols, (uint16_t*)to, plan.pitch, HeadScale{});
}

// Elements in as many float16 pieces as they take.
static int head_pieces(const void* x, int64_t pitch, int64_t rows, int64_t cols, int dtype, const HeadPlan& plan, char* to, const HeadScale& by, int sms,
                       cudaStream_t stream, HeadOperand* out) {
  const int64_t words = rows * (plan.pitch / 8);
  const dim3 blocks((unsigned)std::min<int64_t>((words + 255) / 256, 16 * sms)), threads(256);
  *out = {to, plan.pitch, rows, plan.pieces};
  if (dtype == SOLON_F32)
    return launch_dependent(head_split_kernel<float>, blocks, threads, 0, stream, (const float*)x, pitch, rows, cols, (uint16_t*)to, plan.pitch, by);
  if (dtype == SOLON_BF16)
    return launch_dependent(head_split_kernel<__nv_bfloat16>, blocks, threads, 0, stream, (const __nv_bfloat16*)x, pitch, rows, cols, (uint16_t*)to, plan.pitch, by);
  return launch_dependent(head_split_kernel<__half>, blocks, threads, 0, stream, (const __half*)x, pitch, rows, cols, (uint16_t*)to, plan.pitch, by);
}

// Rows wider than 8192 elements are gone through by whole CTAs.
static int head_scan(const HeadScanArgs& a, int dtype, int sms, cudaStream_t stream) {
  const bool whole = dtype == SOLON_F32 && a.cols > 8192;
  const int64_t rows = std::max(a.rows, a.side[1].x ? a.side[1].rows : 0);
  const dim3 grid((unsigned)std::min<int64_t>(whole ? rows : (rows + 7) / 8, 8 * sms), a.undo_dz ? 3 : 2);
  if (whole) head_scan_kernel<float, 256><<<grid, 256, 0, stream>>>(a);
  else if (dtype == SOLON_F32) head_scan_kernel<float, 32><<<grid, 256, 0, stream>>>(a);
  else if (dtype == SOLON_BF16) head_scan_kernel<__nv_bfloat16, 32><<<grid, 256, 0, stream>>>(a);
  else head_scan_kernel<__half, 32><<<grid, 256, 0, stream>>>(a);
  SOLON_CUDA_TRY(cudaGetLastError());
  return SOLON_OK;
}

// Pairs of pieces, the smallest products first.
static void head_pairs(HeadArgs& a, int pieces_a, int pieces_b, int step_a, int step_b) {
  a.products = 0;                          // (three pieces of one factor go with one of the other)
  auto pair = [&](int x, int y) {
    a.piece_a[a.products] = x * step_a;
    a.piece_b[a.products++] = y * step_b;
  };
  if (pieces_b == 2) pair(0, 1);
  if (pieces_a == 3) pair(2, 0);
  if (pieces_a >= 2) pair(1, 0);
  pair(0, 0);
}

static int head_finish(const HeadFinishArgs& a, int dtype, int sms, cudaStream_t stream) {
  const unsigned blocks = (unsigned)std::min<int64_t>((a.parts * a.m * ((a.n + 3) / 4) + 255) / 256, 16 * sms);
  auto* kernel = dtype == SOLON_F32 ? head_finish_kernel<float> : dtype == SOLON_F64 ? head_finish_kernel<double>
                 : dtype == SOLON_BF16 ? head_finish_kernel<__nv_bfloat16> : head_finish_kernel<__half>;
  return launch_dependent(kernel, dim3(blocks), dim3(256), 0, stream, a);
}

static bool head_sizes_ok(int64_t rows, int64_t cols, int64_t vocab) {
  return rows >= 0 && rows <= (1 << 30) && cols >= 1 && cols <= SOLON_MAX_WIDTH && vocab >= 1 && vocab <= (1 << 30) && vocab <= (1ll << 46) / cols &&
         (rows == 0 || vocab <= (1ll << 46) / rows);
}

static int head_stats(const HeadMaps& maps, const HeadArgs& a, bool few, bool bf16, int sms, cudaStream_t stream) {
  if (few && a.n <= 64 && bf16) return head_product_launch<kFewRows, 64, true, float>(maps, a, sms, stream);
  if (few && a.n <= 64) return head_product_launch<kFewRows, 64, false, float>(maps, a, sms, stream);
  if (few && bf16) return head_product_launch<kFewRows, 128, true, float>(maps, a, sms, stream);
  if (few) return head_product_launch<kFewRows, 128, false, float>(maps, a, sms, stream);
  if (bf16) return head_product_launch<kStats, 256, true, float>(maps, a, sms, stream);
  return head_product_launch<kStats, 256, false, float>(maps, a, sms, stream);
}

// dh and dW are products of float16 pieces, whatever the states' type, but for few bfloat16 rows.
static int head_dhidden(const HeadMaps& maps, const HeadArgs& a, int dtype, bool as_is, int sms, cudaStream_t stream) {
  if (as_is) return head_product<kDhidden, true, __nv_bfloat16>(maps, a, sms, stream);
  if (dtype == SOLON_F32) return head_product<kDhidden, false, float>(maps, a, sms, stream);
  if (dtype == SOLON_BF16) return head_product<kDhidden, false, __nv_bfloat16>(maps, a, sms, stream);
  return head_product<kDhidden, false, __half>(maps, a, sms, stream);
}
template <bool BF16>
static int head_dweight(const HeadMaps& maps, const HeadArgs& a, int grad_dtype, int sms, cudaStream_t stream) {
  if (grad_dtype == SOLON_F32) return head_product<kDweight, BF16, float>(maps, a, sms, stream);
  if (grad_dtype == SOLON_F64) return head_product<kDweight, BF16, double>(maps, a, sms, stream);
  return head_product<kDweight, BF16, __nv_bfloat16>(maps, a, sms, stream);
}

}  // namespace solon

using namespace solon;

extern "C" {

int solon_head_status(void* cuda_stream) {
  int status = 0;
  void* at = nullptr;
  SOLON_CUDA_TRY(cudaGetSymbolAddress(&at, head_wait_status));
  SOLON_CUDA_TRY(cudaMemcpyAsync(&status, at, sizeof(int), cudaMemcpyDeviceToHost, (cudaStream_t)cuda_stream));
  SOLON_CUDA_TRY(cudaStreamSynchronize((cudaStream_t)cuda_stream));
  return status ? SOLON_ERR_INTERNAL : SOLON_OK;
}

int64_t solon_head_logprobs_workspace(int64_t rows, int64_t cols, int64_t vocab, int dtype, int aligned) {
  if (!token_dtype(dtype) || !head_sizes_ok(rows, cols, vocab)) return SOLON_ERR_INVALID_ARG;
  return rows == 0 ? 0 : head_forward_plan(rows, cols, vocab, dtype, aligned != 0).total;
}

int solon_head_logprobs(const void* hidden, int64_t hidden_pitch, const void* weight, int64_t weight_pitch, int dtype, const int64_t* targets, int64_t rows,
                        int64_t cols, int64_t vocab, float* logp, float* entropy, float* peak, float* log_sum, void* workspace, int64_t workspace_bytes,
                        void* cuda_stream) {
  if (!token_dtype(dtype) || !head_sizes_ok(rows, cols, vocab)) return SOLON_ERR_INVALID_ARG;
  if (rows == 0) return SOLON_OK;
  if (!matrix_ok(hidden, hidden_pitch, rows, cols, dtype) || !matrix_ok(weight, weight_pitch, vocab, cols, dtype)) return SOLON_ERR_INVALID_ARG;
  if ((logp && !targets) || ((uintptr_t)targets & 7) || (((uintptr_t)logp | (uintptr_t)entropy | (uintptr_t)peak | (uintptr_t)log_sum) & 3))
    return SOLON_ERR_INVALID_ARG;
  for (const float* out : {logp, entropy, peak, log_sum})
    if (meet(extent(out, 1, rows, rows, 4), extent(targets, 1, rows, rows, 8)) || meet(extent(out, 1, rows, rows, 4), extent(hidden, rows, cols, hidden_pitch, element_size(dtype))) ||
        meet(extent(out, 1, rows, rows, 4), extent(weight, vocab, cols, weight_pitch, element_size(dtype))))
      return SOLON_ERR_INVALID_ARG;
  const bool aligned = aligned16(hidden, hidden_pitch, rows, dtype) && aligned16(weight, weight_pitch, vocab, dtype);
  const HeadPlan plan = head_forward_plan(rows, cols, vocab, dtype, aligned);
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < plan.total) return SOLON_ERR_INVALID_ARG;
  int sms = 0, rc;
  if ((rc = current_sms(&sms))) return rc;
  const int64_t slots = plan.few ? std::min<int64_t>(plan.slots, 8 * (sms / 2)) : plan.slots;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  char* ws = (char*)workspace;
  if (plan.row_kernel) {
    const HeadRowsArgs a = {hidden, weight, hidden_pitch, vocab > 1 ? weight_pitch : cols, cols, vocab, targets, (int)rows, (int)rows_padded(cols),
                            (float*)(ws + plan.partial), (float*)(ws + plan.target_logit)};
    if (dtype == SOLON_F32) rc = head_rows_t<float>(a, plan.row_kernel, stream);
    else if (dtype == SOLON_BF16) rc = head_rows_t<__nv_bfloat16>(a, plan.row_kernel, stream);
    else rc = head_rows_t<__half>(a, plan.row_kernel, stream);
    if (rc) return rc;
  } else if (plan.small) {
    HeadSmallArgs a = {};
    a.hidden = (const float*)hidden;
    a.weight = (const float*)weight;
    a.hidden_pitch = hidden_pitch;
    a.weight_pitch = vocab > 1 ? weight_pitch : cols;
    a.cols = cols;
    a.vocab = vocab;
    a.rows = (int)rows;
    a.targets = targets;
    a.turned = (float*)(ws + plan.turned);
    a.partial = (float*)(ws + plan.partial);
    a.target_logit = (float*)(ws + plan.target_logit);
    if ((rc = small_forward(a, stream))) return rc;
  } else {
    HeadOperand h, w;
    if (dtype == SOLON_F32) {
      const HeadScanArgs scan = {{{hidden, hidden_pitch, rows, (__half*)(ws + plan.hidden), (float*)(ws + plan.undo_hidden), nullptr},
                                  {weight, weight_pitch, vocab, (__half*)(ws + plan.weight), (float*)(ws + plan.undo_weight), nullptr}},
                                 cols, plan.pitch, rows, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0};
      if ((rc = head_scan(scan, dtype, sms, stream))) return rc;
      h = {ws + plan.hidden, plan.pitch, rows, 2};
      w = {ws + plan.weight, plan.pitch, vocab, 2};
    } else if ((rc = head_operand(hidden, hidden_pitch, rows, cols, plan, ws + plan.hidden, sms, stream, &h)) ||
               (rc = head_operand(weight, weight_pitch, vocab, cols, plan, ws + plan.weight, sms, stream, &w))) {
      return rc;
    }
    const bool bf16 = dtype == SOLON_BF16;
    HeadMaps maps = {};
    if (!tensor_map(&maps.a, h.p, bf16, cols, rows, h.pieces, h.pitch, rows * h.pitch, !plan.few ? kRows : rows <= 64 ? 32 : 64) ||
        !tensor_map(&maps.b, w.p, bf16, cols, vocab, w.pieces, w.pitch, vocab * w.pitch, kRows))
      return SOLON_ERR_CUDA;
    HeadArgs a = {};
    a.m = (int)rows;
    a.n = (int)vocab;
    a.slabs = a.splits = 1;
    a.k_blocks = (int)((cols + kBlock - 1) / kBlock);
    head_pairs(a, h.pieces, w.pieces, 1, 1);
    if (dtype == SOLON_F32) {
      a.undo_m = (const float*)(ws + plan.undo_hidden);
      a.undo_n = (const float*)(ws + plan.undo_weight);
    }
    a.targets = targets;
    a.partial = (float*)(ws + plan.partial);
    a.target_logit = (float*)(ws + plan.target_logit);
    a.vocab = vocab;
    if (plan.few) {
      std::swap(maps.a, maps.b);
      std::swap(a.m, a.n);
      std::swap(a.undo_m, a.undo_n);
    }
    if ((rc = head_stats(maps, a, plan.few, bf16, sms, stream))) return rc;
  }
  const HeadJoinArgs j = {(const float*)(ws + plan.partial), (const float*)(ws + plan.target_logit), rows, slots, vocab, targets, logp, entropy, peak, log_sum};
  // (eight neighbouring rows are a sector of each slot)
  if (rows <= 256) return launch_dependent(head_join_kernel<1>, dim3((unsigned)rows), dim3(256), 0, stream, j);
  if (rows <= 4096) return launch_dependent(head_join_kernel<8>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, stream, j);
  return launch_dependent(head_join_kernel<32>, dim3((unsigned)((rows + 31) / 32)), dim3(256), 0, stream, j);
}

int64_t solon_head_logprobs_backward_workspace(int64_t rows, int64_t cols, int64_t vocab, int partitions, int dtype, int grad_dtype, int aligned) {
  if (!token_dtype(dtype) || !head_sizes_ok(rows, cols, vocab) || partitions < 1 || partitions > SOLON_MAX_NODES || rows % partitions) return SOLON_ERR_INVALID_ARG;
  if (grad_dtype != SOLON_F32 && grad_dtype != SOLON_F64 && grad_dtype != SOLON_BF16) return SOLON_ERR_INVALID_ARG;
  return rows == 0 ? 0 : head_backward_plan(rows, cols, vocab, partitions, dtype, grad_dtype, aligned != 0).total;
}

int solon_head_logprobs_backward(const void* hidden, int64_t hidden_pitch, const void* weight, int64_t weight_pitch, int dtype, const int64_t* targets,
                                 int64_t rows, int64_t cols, int64_t vocab, int partitions, const float* peak, const float* log_sum, const float* entropy,
                                 const float* grad_logp, const float* grad_entropy, void* dhidden, int64_t dhidden_pitch, void* dweight, int64_t grad_pitch,
                                 int grad_dtype, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!token_dtype(dtype) || !head_sizes_ok(rows, cols, vocab) || partitions < 1 || partitions > SOLON_MAX_NODES || rows % partitions)
    return SOLON_ERR_INVALID_ARG;
  if (grad_dtype != SOLON_F32 && grad_dtype != SOLON_F64 && grad_dtype != SOLON_BF16) return SOLON_ERR_INVALID_ARG;
  if (dweight && !matrix_ok(dweight, grad_pitch, partitions, vocab * cols, grad_dtype)) return SOLON_ERR_INVALID_ARG;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  const int64_t grad_size = (int64_t)element_size(grad_dtype);
  if (rows == 0) {
    for (int k = 0; dweight && k < partitions; k++)
      SOLON_CUDA_TRY(cudaMemsetAsync((char*)dweight + k * (partitions > 1 ? grad_pitch : 0) * grad_size, 0, vocab * cols * grad_size, stream));
    return SOLON_OK;
  }
  if (!matrix_ok(hidden, hidden_pitch, rows, cols, dtype) || !matrix_ok(weight, weight_pitch, vocab, cols, dtype)) return SOLON_ERR_INVALID_ARG;
  if (dhidden && !matrix_ok(dhidden, dhidden_pitch, rows, cols, dtype)) return SOLON_ERR_INVALID_ARG;
  if (!peak || !log_sum || (grad_logp && !targets) || (grad_entropy && !entropy) || ((uintptr_t)targets & 7) ||
      (((uintptr_t)peak | (uintptr_t)log_sum | (uintptr_t)entropy | (uintptr_t)grad_logp | (uintptr_t)grad_entropy) & 3))
    return SOLON_ERR_INVALID_ARG;
  if (!dhidden && !dweight) return SOLON_OK;
  const Extent outs[2] = {extent(dhidden, rows, cols, dhidden_pitch, element_size(dtype)), extent(dweight, partitions, vocab * cols, grad_pitch, element_size(grad_dtype))};
  const Extent ins[8] = {extent(hidden, rows, cols, hidden_pitch, element_size(dtype)), extent(weight, vocab, cols, weight_pitch, element_size(dtype)),
                         extent(targets, 1, rows, rows, 8), extent(peak, 1, rows, rows, 4), extent(log_sum, 1, rows, rows, 4),
                         extent(entropy, 1, rows, rows, 4), extent(grad_logp, 1, rows, rows, 4), extent(grad_entropy, 1, rows, rows, 4)};
  for (const Extent& out : outs)
    for (const Extent& in : ins)
      if (meet(out, in)) return SOLON_ERR_INVALID_ARG;
  if (meet(outs[0], outs[1])) return SOLON_ERR_INVALID_ARG;
  const bool aligned = aligned16(hidden, hidden_pitch, rows, dtype) && aligned16(weight, weight_pitch, vocab, dtype);
  const HeadPlan plan = head_backward_plan(rows, cols, vocab, partitions, dtype, grad_dtype, aligned);
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < plan.total) return SOLON_ERR_INVALID_ARG;
  int sms = 0, rc;
  if ((rc = current_sms(&sms))) return rc;
  char* ws = (char*)workspace;
  HeadWords* words = (HeadWords*)(ws + plan.words);
  const bool f32 = dtype == SOLON_F32, bf16 = dtype == SOLON_BF16, f16 = dtype == SOLON_F16;
  if (plan.small) {
    HeadSmallArgs a = {};
    a.hidden = (const float*)hidden;
    a.weight = (const float*)weight;
    a.hidden_pitch = hidden_pitch;
    a.weight_pitch = vocab > 1 ? weight_pitch : cols;
    a.cols = cols;
    a.vocab = vocab;
    a.rows = (int)rows;
    a.partitions = partitions;
    a.targets = targets;
    a.turned = (float*)(ws + plan.turned);
    a.peak = peak;
    a.log_sum = log_sum;
    a.entropy = entropy;
    a.grad_logp = grad_logp;
    a.grad_entropy = grad_entropy;
    a.dz = (float*)(ws + plan.dz);
    a.sums = dhidden ? (float*)(ws + plan.sums) : nullptr;
    a.sums_pitch = up(cols, 128);
    a.dweight = dweight;
    a.grad_pitch = partitions > 1 ? grad_pitch : up(vocab * cols, 8);
    a.grad_dtype = grad_dtype;
    if ((rc = small_backward(a, stream)) || !dhidden) return rc;
    return head_finish({a.sums, a.sums_pitch, rows, cols, rows > 1 ? dhidden_pitch : cols, 0, 1, plan.h_splits, dhidden}, dtype, sms, stream);
  }
  const bool coarse = grad_dtype == SOLON_BF16;          // dW from the first pieces alone
  const bool as_is = plan.as_is, weight_h = !f16 && !as_is && dhidden;
  const int form = as_is ? (dweight && !coarse ? kWideTriple : kWidePair) : (dhidden && !bf16) || (dweight && !coarse) ? kPair : kNearest;
  const int dz_pieces = form == kNearest ? 1 : form == kWideTriple ? 3 : 2;
  const int64_t n = rows / partitions, sums_pitch = up(cols, 128);
  unsigned* parts = (unsigned*)(words + 1);
  float* undo_dz = (float*)(ws + plan.undo_dz);
  if (!as_is) SOLON_CUDA_TRY(cudaMemsetAsync(words, 0, sizeof(HeadWords) + partitions * sizeof(unsigned), stream));
  __half* const copy = f32 ? (__half*)(ws + plan.hidden) : as_is ? (__half*)(ws + plan.hidden_w) : nullptr;
  const HeadScanArgs scan = {{{f32 || dweight ? hidden : nullptr, hidden_pitch, rows, copy, (float*)(ws + plan.undo_hidden), nullptr},
                              {f32 || weight_h ? weight : nullptr, weight_pitch, vocab, f32 ? (__half*)(ws + plan.weight) : nullptr, (float*)(ws + plan.undo_weight),
                               weight_h ? &words->weight : nullptr}},
                             cols, plan.pitch, rows, targets, peak, grad_logp, grad_entropy, entropy, undo_dz, dweight && !as_is ? parts : nullptr, n};
  if ((rc = head_scan(scan, dtype, sms, stream))) return rc;
  HeadOperand h = {ws + plan.hidden, plan.pitch, rows, 2}, w = {ws + plan.weight, plan.pitch, vocab, 2};
  if (!f32 && ((rc = head_operand(hidden, hidden_pitch, rows, cols, plan, ws + plan.hidden, sms, stream, &h)) ||
               (rc = head_operand(weight, weight_pitch, vocab, cols, plan, ws + plan.weight, sms, stream, &w))))
    return rc;

  // as rows along the inner dimension: h and W for the logits, dz for dh; across it: W for dh, dz and h for dW
  CUtensorMap map_h, map_w, map_w_across, map_h_across, map_dz, map_dz_across, map_dz_out;
  HeadOperand hw = h, wh = w;              // as they go into dW and dh
  if (as_is) hw = {ws + plan.hidden_w, plan.pitch, rows, 1};
  else if (dweight && (rc = head_pieces(hidden, hidden_pitch, rows, cols, dtype, plan, ws + plan.hidden_w, {nullptr, undo_dz, parts, n}, sms, stream, &hw))) return rc;
  // (a map across the inner dimension goes with the tiles: copies of 128 columns need 128 of them in a CTA's tile, and whole blocks of 64 in memory)
  const bool whole = cols % kBlock == 0 || plan.split, hw_whole = whole || dweight, wh_whole = whole || weight_h;
  auto across = [&](CUtensorMap* map, const void* p, bool by_blocks, int64_t rows, int64_t slabs, int64_t pitch, int64_t slab) {
    return by_blocks ? tensor_map_by_blocks(map, p, false, cols, rows, slabs, pitch, slab) : tensor_map(map, p, false, cols, rows, slabs, pitch, slab, kBlock);
  };
  const bool w_narrow = narrow(cols, (n + kBlock - 1) / kBlock * dw_products(plan, grad_dtype));
  if (!tensor_map(&map_h, h.p, bf16, cols, rows, h.pieces, h.pitch, rows * h.pitch, kRows) ||
      !across(&map_h_across, hw.p, hw_whole && !w_narrow, n, (int64_t)hw.pieces * partitions, hw.pitch, n * hw.pitch))
    return SOLON_ERR_CUDA;
  HeadArgs base = {};
  base.slabs = base.splits = 1;
  base.words = words;
  base.targets = targets;
  base.peak = peak;
  base.log_sum = log_sum;
  base.entropy = entropy;
  base.grad_logp = grad_logp;
  base.grad_entropy = grad_entropy;
  base.vocab = vocab;
  base.undo_dz = undo_dz;
  base.parts = as_is ? nullptr : parts;
  base.low_factor = as_is ? 1.0f : 1.0f / kSecond;
  for (int64_t first = 0; first < vocab; first += plan.width) {
    const int64_t width = std::min(plan.width, vocab - first), pitch = up(width, kBlock);
    const bool h_narrow = narrow(cols, pitch / kBlock * dh_products(plan, dtype));
    if (weight_h && (rc = head_pieces((const char*)weight + first * weight_pitch * (f32 ? 4 : 2), weight_pitch, width, cols, dtype, plan, ws + plan.weight_h,
                                      {&words->weight, nullptr, nullptr, 0}, sms, stream, &wh)))
      return rc;
    const char* w_across = wh.p + (weight_h ? 0 : first * wh.pitch * 2);
    if (!tensor_map(&map_dz, ws + plan.dz, false, pitch, rows, dz_pieces, pitch, rows * pitch, kRows) ||
        !tensor_map(&map_dz_out, ws + plan.dz, false, pitch, rows, dz_pieces, pitch, rows * pitch, 32) ||
        !tensor_map_by_blocks(&map_dz_across, ws + plan.dz, false, pitch, n, (int64_t)dz_pieces * partitions, pitch, n * pitch) ||
        !tensor_map(&map_w, w.p + first * w.pitch * 2, bf16, cols, width, w.pieces, w.pitch, vocab * w.pitch, kRows) ||
        !across(&map_w_across, w_across, wh_whole && !h_narrow, width, wh.pieces, wh.pitch, wh.rows * wh.pitch))
      return SOLON_ERR_CUDA;
    HeadArgs a = base;
    a.m = (int)rows;
    a.n = (int)width;
    a.first = first;
    a.k_blocks = (int)((cols + kBlock - 1) / kBlock);
    head_pairs(a, h.pieces, w.pieces, 1, 1);
    if (f32) {
      a.undo_m = (const float*)(ws + plan.undo_hidden);
      a.undo_n = (const float*)(ws + plan.undo_weight);
    }
    a.form = form;
    a.dz_pitch = (int)pitch;
    if ((rc = bf16 ? head_product_launch<kDz, 256, true, float>({map_h, map_w, map_dz_out}, a, sms, stream)
                   : head_product_launch<kDz, 256, false, float>({map_h, map_w, map_dz_out}, a, sms, stream)))
      return rc;
    if (dhidden) {
      a = base;
      a.m = (int)rows;
      a.n = (int)cols;
      a.slabs = a.splits = plan.h_splits;
      a.narrow = h_narrow;
      a.b_by_blocks = wh_whole && !h_narrow;
      a.k_blocks = (int)((pitch / kBlock + a.splits - 1) / a.splits);
      head_pairs(a, bf16 && !as_is ? 1 : 2, wh.pieces, 1, 1);
      a.weight_scaled = weight_h;
      a.undo_m = as_is ? nullptr : undo_dz;
      a.sums = (float*)(ws + plan.sums);
      a.sums_pitch = sums_pitch;
      a.load_sums = first > 0;
      const bool last = first + width == vocab;
      a.store_sums = !last || a.splits > 1;
      a.out = dhidden;
      a.out_pitch = rows > 1 ? dhidden_pitch : cols;
      a.out_wide = !(((uintptr_t)dhidden | (uintptr_t)(a.out_pitch * element_size(dtype))) & 31);
      if ((rc = head_dhidden({map_dz, map_w_across, {}}, a, dtype, as_is, sms, stream))) return rc;
      if (last && a.splits > 1 &&
          (rc = head_finish({a.sums, sums_pitch, rows, cols, a.out_pitch, 0, 1, a.splits, dhidden}, dtype, sms, stream)))
        return rc;
    }
    if (dweight) {
      a = base;
      a.m = (int)width;
      a.n = (int)cols;
      a.splits = plan.w_splits;
      a.slabs = partitions * a.splits;
      a.slab_a = a.slab_b = 1;
      a.narrow = w_narrow;
      a.b_by_blocks = hw_whole && !w_narrow;
      a.k_blocks = (int)(((n + kBlock - 1) / kBlock + a.splits - 1) / a.splits);
      a.sums = (float*)(ws + plan.w_sums);
      a.sums_pitch = sums_pitch;
      a.store_sums = a.splits > 1;
      if (as_is) head_pairs(a, coarse ? 2 : 3, 1, partitions, partitions);
      else head_pairs(a, coarse ? 1 : 2, coarse ? 1 : hw.pieces, partitions, partitions);
      a.out = (char*)dweight + first * cols * grad_size;
      a.out_pitch = cols;
      a.out_slab = partitions > 1 ? grad_pitch : 0;
      a.out_wide = !(((uintptr_t)a.out | (uintptr_t)(cols * grad_size) | (uintptr_t)(a.out_slab * grad_size)) & 31);
      HeadMaps maps = {map_dz_across, map_h_across, {}};
      a.out_by_map = !(((uintptr_t)a.out | (uintptr_t)(cols * grad_size) | (uintptr_t)(a.out_slab * grad_size)) & 15);
      if (a.out_by_map && !output_map(&maps.out, a.out, (int)grad_size, cols, width, partitions, cols, partitions > 1 ? a.out_slab : up(width * cols, 8)))
        return SOLON_ERR_CUDA;
      if ((rc = as_is ? head_dweight<true>(maps, a, grad_dtype, sms, stream) : head_dweight<false>(maps, a, grad_dtype, sms, stream))) return rc;
      if (a.splits > 1 && (rc = head_finish({a.sums, sums_pitch, width, cols, cols, a.out_slab, partitions, a.splits, a.out}, grad_dtype, sms, stream))) return rc;
    }
  }
  return SOLON_OK;
}

}  // extern "C"
