// Softmax cross entropy over a vocabulary and its gradient, without keeping the logits: dgs_vocabulary_loss and dgs_vocabulary_loss_grad.
//
// With hidden states h [N][D], a vocabulary W [V][D] and z = h W^T:
//     loss[r] = lse[r] - z[r][target[r]],  lse[r] = log(sum over v of exp z[r][v]),
//     s[r][v] = dloss[r] (exp(z[r][v] - lse[r]) - [v = target[r]]),  dh = s W,  dW = s^T h.
// The loss keeps a maximum and a sum for each row and 64 words of a tile of logits, which stay in registers.  The gradient goes through the vocabulary in
// pieces: the logits of a piece are formed again, s of the piece goes to the workspace, and its products with W and h are formed from there.
//
// Numbers: s is kept as the sum of two fp16 numbers (22 bits) under one power of two for the call, since dW goes to a flat gradient in f32; products of fp16 need
// fp16 partners, so W and h are held beside as fp16 numbers under a power of two for each column: exact for bfloat16 and fp16 values down to 2^-29 of their column's
// largest, and below that to 2^-40 of it (s likewise: an exponential below 2^-29 keeps fewer bits).  f32 matrices are sums of two fp16 numbers each; of their four products the smallest, under 2^-22 of the whole, is left out.
// Both gradients are formed from both parts of s, so that dh is rounded once, to its type: 1.0e-3 of dh in bfloat16 differed from the f32 form's with the first part alone
// (11 bits for a result of 8) and 1.4e-4 does with both, for 8192 x 768 x 50257 at the price of 2.93 ms for 2.53.
#include "dgs_tensor.cuh"

#include <algorithm>
#include <cstring>
#include <mutex>

namespace dgs {
namespace {

// ---- copies and tiles -----------------------------------------------------------------------------
__device__ __forceinline__ void tma_load3(uint32_t to, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to), "l"(map),
               "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t to, const void* from, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar)
               : "memory");
}
// *to += v, without waiting for what is there.  The only thread that adds to it in this kernel, so the sum's order is that of the kernels.  This addition takes subnormal numbers
// for 0, so it is for sums of products that still stand under their powers of two, multiples of 2^-48, and not for the caller's numbers.
__device__ __forceinline__ void add_behind(float* to, float v) { asm volatile("red.global.add.f32 [%0], %1;" ::"l"(to), "f"(v) : "memory"); }

// What the kernel forms: maxima and sums of logits; s of a piece; the products of a piece's s with h (dW) and with W (dh's part).
enum : int { kLoss, kSlope, kGrads };

// A pair of CTAs forms tiles of 256 x 256, 128 rows and 256 columns of it in each CTA's tensor memory.  A step contracts kRows values of the operands' PA and PB
// parts; a CTA brings 128 rows (or columns) of either operand, 256 bytes a value contracted.
//   contracted dimension contiguous (h and W for the logits, s for dh): blocks of 64 values contracted, 128 rows of 128 bytes each
//   contracted dimension outermost (h and s for dW, W for dh): blocks of 64 columns, kRows rows of 128 bytes each
// Either way the 16-byte pieces of a row are exchanged by its number (128-byte swizzle).  s lies in the workspace in blocks of 128 rows and 64 columns that are in
// that order already, so both uses copy it as it is.
// kChunk: steps between two sums in registers, at most: 512 values; 256 of s and 64 of logits where each is three products, since their results are all in f32.
// Logits of few steps take half of them: an exponential takes a logit's error as it is (a logit of 15 summed over 768 values in one go is off by 7e-6), and two
// chunks a tile let the products of the next tile run to their end while one is finished.
constexpr uint32_t kBlockBytes = 128 * 128;                       // 128 rows and 64 columns of s
// Shared memory is a ring of tiles, one for each part of an operand and step: a step of the gradients takes three of the twelve (f32 four), so that four steps are on
// their way.
template <int MODE, uint32_t PA, uint32_t PB> struct Step {
  static constexpr uint32_t kRows = MODE == kLoss && PA == 1 ? 128 : 64, kTile = kRows * 256, kSlots = (MODE == kSlope ? 160 : 192) * 1024 / kTile;
  static constexpr uint32_t kAhead = kSlots / (PA + PB);   // steps under way, at most
  static constexpr uint32_t kChunk = (PA == 1 ? 512 : MODE == kGrads ? 256 : 64) / kRows, kSmem = 1024 + kSlots * kTile + (MODE == kSlope ? 64 * 1024 : 0);
};
// Sixteen warps keep the sums, 64 columns of 32 rows each; four do the rest and leave them their registers.  (With eight warps of 128 columns, two a scheduler, the
// trips to tensor memory and through the exponentials showed: 5632 words of 8192 x 768 took 105 us.)
constexpr uint32_t kSumWarps = 16, kHeadThreads = kSumWarps * 32 + 128, kHeadRegs = 96, kHeadRegsSum = 104, kHeadRegsRest = 64;
static_assert(kHeadRegsSum * kSumWarps * 32 + kHeadRegsRest * 128 <= kHeadRegs * kHeadThreads, "setmaxnreg draws on the launch's registers");
constexpr uint32_t kHeadTmem = 512;                               // two accumulators of 256 columns

// A tile's descriptor, and what the k-th sixteen of the values contracted add to it.
template <bool OUTER, uint32_t R>
__device__ __forceinline__ uint64_t tile_desc(uint32_t tile) {
  return uint64_t(tile >> 4) | uint64_t(OUTER ? R * 128 >> 4 : 1) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
template <bool OUTER>
__device__ __forceinline__ uint32_t desc_step(uint32_t k) { return (OUTER ? k * 2048 : (k / 4) * kBlockBytes + (k % 4) * 32) >> 4; }
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&v)[16]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
        "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// The power of two that takes a largest finite magnitude (its bits) to [2^14, 2^15), kept where it is a normal number, and its reciprocal.
__device__ __forceinline__ uint32_t down_exponent(uint32_t largest) { return uint32_t(max(int(largest >> 23) - 14, 1)); }   // with its bias: 1 .. 240
__device__ __forceinline__ float up_of(uint32_t largest) { return __uint_as_float((254 - down_exponent(largest)) << 23); }
__device__ __forceinline__ float down_of(uint32_t largest) { return __uint_as_float(down_exponent(largest) << 23); }
// The reciprocal as two factors of about its square root: of two reciprocals the product, and a sum under one of them, may lie outside f32's range where the result does not.
struct Down {
  float a, b;
};
__device__ __forceinline__ Down downs_of(uint32_t largest) {
  const uint32_t e = down_exponent(largest), half = e / 2;
  return {__uint_as_float((63 + half) << 23), __uint_as_float((64 + e - half) << 23)};
}
__device__ __forceinline__ Down operator*(Down x, Down y) { return {x.a * y.a, x.b * y.b}; }   // from 2^-128 on: exact
__device__ __forceinline__ float operator*(float v, Down x) { return v * x.a * x.b; }
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -__builtin_huge_valf();
constexpr float kLeastPower = 0x1p-126f, kMostPower = 0x1p127f;

// One of the two products of a piece's s.
struct Product {
  uint32_t m_tiles, n_tiles, splits, tiles, steps;   // steps over the whole contraction
  float* out;
};
struct Head {
  uint32_t rows, width, words;      // N, D, V
  uint32_t m_tiles, n_tiles, tiles, steps, chunk, skip;   // logits; skip: steps that a tile's first chunk is short of
  uint32_t first_word, piece_cols;  // of the piece (a multiple of 256 in the workspace)
  uint32_t idesc;
  uint32_t wide_targets, dloss_step;
  const void* target;
  const float *lse, *dloss;
  const uint32_t *most_h, *most_w, *most_g;     // bits of the largest magnitudes: of each column of h and of W, of dloss
  const float *row_h, *row_w;       // f32: what the rows of the logits' operands are multiplied with
  float2* partial;                  // [n_tiles * 4][rows]: maximum, sum
  float* at_target;                 // [rows]
  unsigned char* s;                 // [2][m_tiles * 2][piece_cols / 64] blocks
  uint64_t plane;                   // bytes of one part of s
  Product dw, dh;                   // out: dw or partial results [splits][piece_cols][width]; [splits][rows][width]
  uint32_t share_few, share_more;   // tiles of dh for a pair of CTAs with one more tile of dw, and for others
  uint32_t add, first_piece;
  int* status;
};

// A row's target: -1 where the row is ignored or (reported) the target is not in the vocabulary.
__device__ __forceinline__ int target_of(const Head& a, uint32_t row, bool tell) {
  const long long t = a.wide_targets ? static_cast<const long long*>(a.target)[row] : static_cast<const int*>(a.target)[row];
  if (t >= (long long)(a.words)) {
    if (tell) report(a.status, DGS_EINVAL);
    return -1;
  }
  return t < 0 ? -1 : int(t);
}

// One lane of the warp, the same one each time.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p;
}
struct HeadTile {
  uint32_t m0, n0, split, from, steps;
  bool hidden;
};
// A pair's i-th tile; false behind its last.  Logits go down the rows first, 32 tiles of them at a time: the pairs work on few words together, and on rows that the
// second cache holds.  Of the two products with s, dW's tiles are dealt out first, then dh's, more to the pairs that got fewer of the others: one launch of
// both keeps 74 pairs busy where 66 tiles of dW and 96 of dh would not (155 us for 199).
template <int MODE>
__device__ __forceinline__ bool head_tile(const Head& a, uint32_t pair, uint32_t pairs, uint32_t i, HeadTile* t) {
  t->hidden = false;
  t->split = t->from = 0;
  if constexpr (MODE != kGrads) {
    const uint32_t tile = i * pairs + pair;
    if (tile >= a.tiles) return false;
    const uint32_t group = tile / (32 * a.n_tiles), rows = min(32u, a.m_tiles - group * 32), in = tile - group * 32 * a.n_tiles;
    t->m0 = (group * 32 + in % rows) * 256;
    t->n0 = in / rows * 256;
    t->steps = a.steps;
    return true;
  } else {
    const uint32_t some = a.dw.tiles % pairs, first = a.dw.tiles / pairs + (pair < some ? 1 : 0);
    uint32_t tile = i * pairs + pair;
    if (i >= first) {
      const uint32_t j = i - first, share = pair < some ? a.share_few : a.share_more;
      tile = (pair < some ? pair * share : some * a.share_few + (pair - some) * share) + j;
      if (j >= share || tile >= a.dh.tiles) return false;
      t->hidden = true;
    }
    const Product& p = t->hidden ? a.dh : a.dw;
    t->m0 = tile % p.m_tiles * 256;
    tile /= p.m_tiles;
    t->n0 = tile % p.n_tiles * 256;
    t->split = tile / p.n_tiles;
    const uint32_t each = (p.steps + p.splits - 1) / p.splits;
    t->from = min(t->split * each, p.steps);
    t->steps = min(each, p.steps - t->from);
    return true;
  }
}

// Warps: 0 to 15 keep the sums, 16 issues products, 17 and 19 copies (one operand each), 18 passes on that copies have landed.  Accumulators go to registers every
// kChunk steps, since the tensor cores add with bits cut off, and are added up there with rounding.  One pair of CTAs per pair of SMs takes tile after tile,
// so that the products of the next run while one is finished.
// Warps 16 to 19 go through their loops with all lanes, one of which does what has to be done once: descriptors and addresses then stay in uniform registers (with
// one lane in the loops the products of a step waited for their operands to be moved there: loss of 8192 x 768 x 50257 436 us, 383 so).
template <int MODE, uint32_t PA, uint32_t PB>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kHeadThreads, 1)
k_head(const __grid_constant__ Head a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b) {
  using S = Step<MODE, PA, PB>;
  constexpr uint32_t R = S::kRows, ST = S::kAhead, SLOTS = S::kSlots, TILE = S::kTile;
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[ST], s_empty[ST], s_loaded[ST], s_sum_full[2], s_sum_empty[2], s_done;
  __shared__ uint32_t s_tmem;
  const uint32_t tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid / 32, 0), lane = tid % 32, rank = cta_rank(), pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  const uint32_t stages = (smem_at(raw) + 1023u) & ~1023u, CH = MODE == kGrads ? S::kChunk : a.chunk, SKIP = MODE == kGrads ? 0 : a.skip;

  if (warp == kSumWarps) {
    tmem_alloc(&s_tmem, kHeadTmem);
    if (lane == 0) {
      for (uint32_t s = 0; s < ST; ++s) {
        bar_init(smem_at(&s_full[s]), 2);    // that copies landed, of both CTAs
        bar_init(smem_at(&s_empty[s]), 1);
        bar_init(smem_at(&s_loaded[s]), 2);  // of both operands
      }
      for (uint32_t i = 0; i < 2; ++i) {
        bar_init(smem_at(&s_sum_full[i]), 1);
        bar_init(smem_at(&s_sum_empty[i]), 2 * kSumWarps);
      }
      bar_init(smem_at(&s_done), 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
  }
  let_next_kernel_begin();
  tmem_before();
  __syncthreads();
  pair_sync();
  tmem_after();
  const uint32_t tmem = s_tmem;
  wait_for_last_kernel();   // nothing above touches memory outside the SM
  __syncwarp();
  if (warp >= kSumWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kHeadRegsRest));
    HeadTile w;
    if (warp == kSumWarps && rank == 0) {
      bool alive = true;
      const bool one = elect_one();
      uint32_t it = 0, chunk = 0, in = 0, slot = 0;   // in: steps of the chunk
      const auto products = [&](auto outer_a, auto outer_b, uint32_t acc, bool first) {
        constexpr bool kOuterA = decltype(outer_a)::value, kOuterB = decltype(outer_b)::value;
        const uint32_t idesc = a.idesc | uint32_t(kOuterA) << 15 | uint32_t(kOuterB) << 16 | idesc_cols(256);
        uint64_t ad[PA], bd[PB];
#pragma unroll
        for (uint32_t i = 0; i < PA; ++i) ad[i] = tile_desc<kOuterA, R>(stages + slot * TILE), slot = slot + 1 == SLOTS ? 0 : slot + 1;
#pragma unroll
        for (uint32_t j = 0; j < PB; ++j) bd[j] = tile_desc<kOuterB, R>(stages + slot * TILE), slot = slot + 1 == SLOTS ? 0 : slot + 1;
        if (one) {   // products with second parts first: what is cut off as they are added is small
          bool more = !first;
#pragma unroll
          for (int i = PA - 1; i >= 0; --i)
#pragma unroll
            for (int j = PB - 1; j >= 0; --j)
#pragma unroll
              for (uint32_t k = 0; k < R / 16; ++k)
                if (i + j < 2) {
                  mma(acc, ad[i] + desc_step<kOuterA>(k), bd[j] + desc_step<kOuterB>(k), idesc, more);
                  more = true;
                }
        }
      };
      using Yes = std::true_type;
      using No = std::false_type;
      for (uint32_t i = 0; alive && head_tile<MODE>(a, pair, pairs, i, &w); ++i) {
        for (uint32_t s = 0; s < w.steps; ++s, ++it) {
          const uint32_t st = it % ST, acc = tmem + (chunk & 1) * 256;
          const bool begins = s == 0 || in == 0;
          if (s == 0) in = SKIP;
          if (begins && chunk >= 2) alive = warp_wait(smem_at(&s_sum_empty[chunk & 1]), (chunk / 2 - 1) & 1);
          alive = alive && warp_wait(smem_at(&s_full[st]), it / ST & 1);
          if (!alive) break;
          tmem_after();
          if constexpr (MODE == kGrads) {
            if (w.hidden) products(Yes{}, No{}, acc, begins);
            else products(Yes{}, Yes{}, acc, begins);
          } else {
            products(No{}, No{}, acc, begins);
          }
          if (one) mma_commit(smem_at(&s_empty[st]));
          if (++in == CH || s == w.steps - 1) {
            if (one) mma_commit(smem_at(&s_sum_full[chunk & 1]));
            ++chunk;
            in = 0;
          }
        }
      }
      if (one) mma_commit(smem_at(&s_done));   // waited for in both CTAs, at the end: nothing is under way when tensor memory is given back
      if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);
    }
    if (warp == kSumWarps + 1 || warp == kSumWarps + 3) {
      const bool one = elect_one();
      const bool second = warp == kSumWarps + 3;   // of the two operands
      bool alive = true;
      uint32_t it = 0, done = 0, slot = 0;   // steps begun, steps whose products are known to be done
      const uint32_t col_blocks = a.piece_cols / 64;
      for (uint32_t i = 0; alive && head_tile<MODE>(a, pair, pairs, i, &w); ++i) {
        const uint32_t m = w.m0 + rank * 128, n = w.n0 + rank * 128;
        for (uint32_t s = 0; s < w.steps; ++s, ++it) {
          const uint32_t st = it % ST, bar = smem_at(&s_loaded[st]), k0 = (w.from + s) * R;
          if (it - done >= ST) {
            if (!(alive = warp_wait(smem_at(&s_empty[done % ST]), done / ST & 1))) break;
            ++done;
          }
          uint32_t at[PA + PB];
#pragma unroll
          for (uint32_t p = 0; p < PA + PB; ++p) {
            at[p] = stages + slot * TILE;
            slot = slot + 1 == SLOTS ? 0 : slot + 1;
          }
          if (!one) {
          } else if (!second) {
            bar_expect(bar, PA * TILE);
#pragma unroll
            for (uint32_t p = 0; p < PA; ++p) {
              if constexpr (MODE == kGrads) {
                for (uint32_t b = 0; b < 2; ++b)
                  tma_load3(at[p] + b * R * 128, w.hidden ? &map_b : &map_a, int(m + b * 64), int(k0 + (w.hidden ? a.first_word : 0)), int(p), bar);
              } else {
                for (uint32_t b = 0; b < R / 64; ++b) tma_load3(at[p] + b * kBlockBytes, &map_a, int(k0 + b * 64), int(m), int(p), bar);
              }
            }
          } else if constexpr (MODE == kGrads) {
            bar_expect(bar, PB * TILE);
#pragma unroll
            for (uint32_t p = 0; p < PB; ++p) {
              const unsigned char* from = a.s + p * a.plane;
              if (!w.hidden) {   // rows k0 on of 128 columns
                for (uint32_t b = 0; b < 2; ++b)
                  bulk_load(at[PA + p] + b * R * 128, from + (uint64_t(k0 / 128) * col_blocks + n / 64 + b) * kBlockBytes + k0 % 128 * 128, R * 128, bar);
              } else {   // columns k0 on of 128 rows
                bulk_load(at[PA + p], from + (uint64_t(n / 128) * col_blocks + k0 / 64) * kBlockBytes, kBlockBytes, bar);
              }
            }
          } else {
            bar_expect(bar, PB * TILE);
#pragma unroll
            for (uint32_t p = 0; p < PB; ++p)
              for (uint32_t b = 0; b < R / 64; ++b) tma_load3(at[PA + p] + b * kBlockBytes, &map_b, int(k0 + b * 64), int(a.first_word + n), int(p), bar);
          }
        }
      }
      // Nothing is under way to this CTA's memory when it leaves: its copies, and the arrivals that the products' commits send to both CTAs.
      for (; done < it; ++done) {
        const bool landed = warp_wait(smem_at(&s_loaded[done % ST]), done / ST & 1);
        alive = alive && landed && warp_wait(smem_at(&s_empty[done % ST]), done / ST & 1);
      }
      if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);
    }
    if (warp == kSumWarps + 2) {
      const bool one = elect_one();
      bool alive = true;
      uint32_t it = 0;
      for (uint32_t i = 0; alive && head_tile<MODE>(a, pair, pairs, i, &w); ++i) {
        for (uint32_t s = 0; s < w.steps; ++s, ++it) {
          if (!(alive = warp_wait(smem_at(&s_loaded[it % ST]), it / ST & 1))) break;
          if (one) bar_arrive_cluster(in_leader(smem_at(&s_full[it % ST])));
        }
      }
      if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kHeadRegsSum));
    const uint32_t quarter = warp % 4, group = warp / 4, mine = rank * 128 + quarter * 32 + lane;
    bool alive = true;
    uint32_t drained = 0;
    HeadTile w;
    const float up_g = MODE == kSlope ? up_of(*a.most_g) : 0.0f;
    for (uint32_t ordinal = 0; alive && head_tile<MODE>(a, pair, pairs, ordinal, &w); ++ordinal) {
      const uint32_t chunks = (w.steps + SKIP + CH - 1) / CH, row = w.m0 + mine, col0 = w.n0 + group * 64;
      // what the end of the tile needs comes while its products are formed
      int target = -1;
      float lse = 0.0f, by = 1.0f;   // by: dloss; f32 logits: what the row is multiplied with
      if constexpr (MODE != kGrads) {
        if (row < a.rows) {
          target = target_of(a, row, false);
          if (MODE == kSlope && target >= 0) lse = a.lse[row], by = a.dloss[uint64_t(row) * a.dloss_step];
        }
      }
      float acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = 0.0f;
      for (uint32_t c = 0; c < chunks; ++c, ++drained) {
        const uint32_t buf = drained & 1;
        if (!(alive = warp_wait(smem_at(&s_sum_full[buf]), drained / 2 & 1))) break;
        tmem_after();
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
          float v[16];
          tmem_load16(tmem + (quarter * 32 << 16) + buf * 256 + group * 64 + q * 16, v);
#pragma unroll
          for (int i = 0; i < 16; i += 2) add_to(acc[q * 16 + i], acc[q * 16 + i + 1], v[i], v[i + 1]);
        }
        tmem_before();
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(in_leader(smem_at(&s_sum_empty[buf])));
      }
      if (!alive) break;

      if constexpr (MODE != kGrads) {
        if (MODE == kLoss && w.m0 + rank * 128 + quarter * 32 >= a.rows) continue;   // no row of the warp's
        const uint32_t word0 = a.first_word + col0;
        if constexpr (PA == 2) {
          const float row_by = row < a.rows ? a.row_h[row] : 0.0f;
          float word_by[2];   // of two of the warp's words a lane
#pragma unroll
          for (uint32_t i = 0; i < 2; ++i) word_by[i] = word0 + i * 32 + lane < a.words ? a.row_w[word0 + i * 32 + lane] : 0.0f;
#pragma unroll
          for (uint32_t i = 0; i < 64; ++i)   // a logit between f32's ends stays there: their product first, which neither passes them nor makes 0 of an infinity's power of two
            acc[i] *= fminf(fmaxf(row_by * __shfl_sync(0xffffffffu, word_by[i / 32], i % 32), kLeastPower), kMostPower);
        }
        if (word0 + 64 > a.words) {
#pragma unroll
          for (uint32_t i = 0; i < 64; ++i)
            if (word0 + i >= a.words) acc[i] = kNone;
        }
        const uint32_t at = uint32_t(target) - word0;   // the target's column, if it is one of the thread's
        const bool has = __any_sync(0xffffffffu, target >= 0 && at < 64);
        if constexpr (MODE == kLoss) {
          if (has) {
            float z = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < 64; ++i) z = at == i ? acc[i] : z;
            if (target >= 0 && at < 64) a.at_target[row] = z;
          }
          float most = acc[0];
#pragma unroll
          for (int i = 1; i < 64; ++i) most = fmaxf(most, acc[i]);
          const float from = most == kNone ? 0.0f : most;
          float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
          for (int i = 0; i < 64; i += 2) {
            const float2 d = mul2(add2(make_float2(acc[i], acc[i + 1]), both(-from)), both(kLog2e));
            sum = add2(sum, make_float2(hardware_exp2(d.x), hardware_exp2(d.y)));
          }
          if (row < a.rows) a.partial[uint64_t(col0 / 64) * a.rows + row] = make_float2(most, sum.x + sum.y);
        } else {
          if (target < 0) {   // whatever the row's logits are
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = kNone;
          }
          const float g = target < 0 ? 0.0f : by * up_g;
          // By way of 4 KB of shared memory for each warp, so that eight lanes write a row's 128 bytes.  Bound by these stores: 10240 words of 8192 x 768 are 336 MB and
          // 122 us, for products of 79.  (When 5632 words, 184 MB, were measured alone: 74, 60 with the first part alone, 51 without; straight from the registers, 32 bytes a lane, 78; by
          // copies from shared memory, with their fences and waits for the buffer, 88.)
          const uint32_t stage = stages + SLOTS * TILE + warp * 4096;
          const uint32_t mine_at = stage + lane * 128 + ((lane & 7) << 4);   // of a row's first 16 bytes; the q-th are at mine_at ^ q << 4
          unsigned char* const to = a.s + (uint64_t(w.m0 / 128 + rank) * (a.piece_cols / 64) + col0 / 64) * kBlockBytes + quarter * 4096 + lane * 16;
          uint32_t rest[32];
          __syncwarp();
#pragma unroll
          for (uint32_t q = 0; q < 8; ++q) {
            uint32_t first[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
              const uint32_t c = q * 8 + i * 2;
              const float2 d = mul2(add2(make_float2(acc[c], acc[c + 1]), both(-lse)), both(kLog2e));
              float2 v = mul2(make_float2(hardware_exp2(d.x), hardware_exp2(d.y)), both(g));
              if (has) {   // g is 0 in a row without a target
                if (at == c) v.x -= g;
                if (at == c + 1) v.y -= g;
              }
              const __half2 hi = __floats2half2_rn(v.x, v.y);
              const float2 f = __half22float2(hi);
              const __half2 lo = __floats2half2_rn(v.x - f.x, v.y - f.y);
              memcpy(&first[i], &hi, 4);
              memcpy(&rest[q * 4 + i], &lo, 4);
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(mine_at ^ (q << 4)), "r"(first[0]), "r"(first[1]), "r"(first[2]), "r"(first[3]) : "memory");
          }
          const auto out = [&](unsigned char* at) {
            __syncwarp();
#pragma unroll
            for (uint32_t q = 0; q < 8; ++q) {
              uint4 v;
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(stage + q * 512 + lane * 16));
              __stcg(reinterpret_cast<uint4*>(at + q * 512), v);
            }
          };
          out(to);
          __syncwarp();
#pragma unroll
          for (uint32_t q = 0; q < 8; ++q)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(mine_at ^ (q << 4)), "r"(rest[q * 4]), "r"(rest[q * 4 + 1]), "r"(rest[q * 4 + 2]),
                         "r"(rest[q * 4 + 3])
                         : "memory");
          out(to + a.plane);
        }
      } else if (row < a.width) {
        // lanes are neighbours in dW's and dh's rows
        const bool direct = !w.hidden && a.dw.splits == 1, behind = w.hidden && !a.first_piece;
        const uint32_t end = w.hidden ? a.rows : min(a.piece_cols, a.words - a.first_word), last = col0 < end ? min(64u, end - col0) : 0;   // columns of the thread's
        float* p = (w.hidden ? a.dh.out : a.dw.out) + (uint64_t(w.split) * (w.hidden ? a.rows : a.piece_cols) + (direct ? a.first_word : 0) + col0) * a.width + row;
        if (direct) {
          const Down by_both = downs_of(a.most_h[row]) * downs_of(*a.most_g);
#pragma unroll
          for (int i = 0; i < 64; ++i) acc[i] = acc[i] * by_both;
        }
        if (direct && a.add) {   // sixteen of the caller's numbers on their way together
#pragma unroll
          for (uint32_t q = 0; q < 64; q += 16) {
            float before[16];
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) before[i] = q + i < last ? __ldcg(p + uint64_t(q + i) * a.width) : 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) acc[q + i] += before[i];
          }
        }
#pragma unroll
        for (uint32_t i = 0; i < 64; ++i)
          if (i < last) {
            if (behind) add_behind(p + uint64_t(i) * a.width, acc[i]);
            else p[uint64_t(i) * a.width] = acc[i];
          }
      }
    }
    if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);
  }
  __syncwarp();
  tmem_before();
  __syncthreads();
  // the commit behind the last products arrives in both CTAs: neither leaves before its own
  if (warp == kSumWarps && lane == 0 && !bar_wait(smem_at(&s_done), 0)) report(a.status, DGS_ETIMEOUT);
  __syncwarp();
  pair_sync();
  if (warp == kSumWarps) {
    __syncwarp();
    tmem_after();
    tmem_free(tmem, kHeadTmem);
  }
}

// ---- before the products --------------------------------------------------------------------------
struct Source {
  const void* data;
  uint64_t stride;
  uint32_t rows, cols, spans;
};

// A magnitude's bits where it is finite: infinities and NaN have no say in the power of two that the numbers beside them are multiplied with.
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t m = __float_as_uint(v) & 0x7fffffffu;
  return m < 0x7f800000u ? m : 0;
}
// The bits of the largest finite magnitude of each column (of rows that are not ignored, where `rows` says which), and of dloss.
constexpr uint32_t kMostRows = 64;   // of a CTA
template <class T, bool VEC>
__device__ __forceinline__ void columns_most(const Head& a, const Source& m, bool targets, uint32_t block, uint32_t* most) {
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, col0 = block % m.spans * kSpan, row0 = block / m.spans * kMostRows;
  __shared__ uint32_t s_most[8][kSpan];
  uint32_t best[8] = {};
  const auto rows = [&](auto whole) {   // loads with a branch of their own for each lane would not be on their way together
#pragma unroll 4
    for (uint32_t r = row0 + warp; r < min(row0 + kMostRows, m.rows); r += 8) {
      Eight<T> e;
      load8<T, VEC, true, decltype(whole)::value>(static_cast<const T*>(m.data) + r * m.stride, col0, lane, m.cols, e);
      const uint32_t all = !targets || target_of(a, r, false) >= 0 ? ~0u : 0;
      float2 v[4];
      floats_of(e, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        best[2 * i] = max(best[2 * i], finite_bits(v[i].x) & all);
        best[2 * i + 1] = max(best[2 * i + 1], finite_bits(v[i].y) & all);
      }
    }
  };
  if (col0 + kSpan <= m.cols) rows(std::true_type{});
  else rows(std::false_type{});
#pragma unroll
  for (int i = 0; i < 8; ++i) s_most[warp][VEC ? lane * 8 + i : i * 32 + lane] = best[i];
  __syncthreads();
  uint32_t v = 0;
  for (uint32_t q = 0; q < 8; ++q) v = max(v, s_most[q][threadIdx.x]);
  if (v && col0 + threadIdx.x < m.cols) atomicMax(most + col0 + threadIdx.x, v);   // a maximum: no order
}
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_head_most(const __grid_constant__ Head a, const __grid_constant__ Source h, const __grid_constant__ Source w, uint32_t blocks_h,
                                                   uint32_t blocks_w, uint32_t* most_h, uint32_t* most_w, uint32_t* most_g) {
  let_next_kernel_begin();
  wait_for_last_kernel();
  if (blockIdx.x < blocks_w) {
    columns_most<T, VEC>(a, w, false, blockIdx.x, most_w);
  } else if (blockIdx.x < blocks_w + blocks_h) {
    columns_most<T, VEC>(a, h, true, blockIdx.x - blocks_w, most_h);
  } else {
    uint32_t v = 0;
    for (uint32_t r = (blockIdx.x - blocks_w - blocks_h) * 256 + threadIdx.x; r < a.rows; r += (gridDim.x - blocks_w - blocks_h) * 256)
      if (target_of(a, r, true) >= 0) v = max(v, finite_bits(a.dloss[uint64_t(r) * a.dloss_step]));
    v = __reduce_max_sync(0xffffffffu, v);
    if (v && threadIdx.x % 32 == 0) atomicMax(most_g, v);
  }
}

// The sum of two fp16 numbers.  An infinity is the second alone: it meets first parts only (the product of second parts is left out), so that its sign and whether it
// meets a zero are the formula's.  As a first part it would meet second parts, which may be 0 or of the other sign.
__device__ __forceinline__ float unless_infinite(float v) { return fabsf(v) == __builtin_huge_valf() ? 0.0f : v; }
__device__ __forceinline__ void halves(const float2 (&v)[4], Eight<__half>& hi, Eight<__half>& lo) {
  float2 rest[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) rest[i] = make_float2(unless_infinite(v[i].x), unless_infinite(v[i].y));
  of_floats(rest, hi);
  floats_of(hi, rest);
#pragma unroll
  for (int i = 0; i < 4; ++i) rest[i] = make_float2(v[i].x - rest[i].x, v[i].y - rest[i].y);
  of_floats(rest, lo);
}
// A matrix as P fp16 numbers a value under a power of two for each column: [P][rows][stride].  Ignored rows are zero, whatever they hold.
constexpr uint32_t kPlaneRows = 64;   // of a CTA
template <class T, bool VEC, uint32_t P>
__device__ __forceinline__ void by_columns(const Head& a, const Source& m, bool targets, uint32_t block, const uint32_t* most, __half* out, uint32_t stride) {
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, col0 = block % m.spans * kSpan, row0 = block / m.spans * kPlaneRows;
  float2 up[4];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t c = col0 + (VEC ? lane * 8 + i : i * 32 + lane);
    const float v = c < m.cols ? up_of(most[c]) : 1.0f;
    if (i % 2) up[i / 2].y = v;
    else up[i / 2].x = v;
  }
  const auto rows = [&](auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
#pragma unroll 4
    for (uint32_t r = row0 + warp; r < min(row0 + kPlaneRows, m.rows); r += 8) {
      Eight<__half> part[2] = {};
      Eight<T> e;
      load8<T, VEC, false, kWhole>(static_cast<const T*>(m.data) + r * m.stride, col0, lane, m.cols, e);
      if (!targets || target_of(a, r, false) >= 0) {
        float2 v[4];
        floats_of(e, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], up[i]);
        if constexpr (P == 2) halves(v, part[0], part[1]);
        else of_floats(v, part[0]);
      }
#pragma unroll
      for (uint32_t p = 0; p < P; ++p) store8<__half, VEC, kWhole>(out + (uint64_t(p) * m.rows + r) * stride, col0, lane, m.cols, part[p]);
    }
  };
  if (col0 + kSpan <= m.cols) rows(std::true_type{});
  else rows(std::false_type{});
}
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_head_columns(const __grid_constant__ Head a, const __grid_constant__ Source h, const __grid_constant__ Source w, uint32_t blocks_h,
                                                      __half* out_h, __half* out_w, uint32_t stride) {
  constexpr uint32_t P = sizeof(T) == 4 ? 2 : 1;
  let_next_kernel_begin();
  wait_for_last_kernel();
  if (blockIdx.x < blocks_h)
    by_columns<T, VEC, P>(a, h, true, blockIdx.x, a.most_h, out_h, stride);
  else
    by_columns<T, VEC, P>(a, w, false, blockIdx.x - blocks_h, a.most_w, out_w, stride);
}

// The logits' operands where TMA copies cannot take them from the caller's memory: 16-bit matrices moved onto 16 bytes, f32 ones as two fp16 numbers a value under a
// power of two for each row.  A warp a row.
template <class T, bool VEC>
__device__ __forceinline__ void by_rows(const Source& m, uint64_t r, void* out, float* scale, uint32_t stride) {
  const uint32_t lane = threadIdx.x % 32;
  if (r >= m.rows) return;
  const T* row = static_cast<const T*>(m.data) + r * m.stride;
  if constexpr (sizeof(T) == 2) {
    for (uint32_t s = 0; s < m.spans; ++s) {
      Eight<T> e;
      load8<T, VEC>(row, s * kSpan, lane, m.cols, e);
      store8<T, VEC>(static_cast<T*>(out) + r * stride, s * kSpan, lane, m.cols, e);
    }
  } else {
    uint32_t most = 0;
    for (uint32_t c = lane; c < m.cols; c += 32) most = max(most, finite_bits(row[c]));
    most = __reduce_max_sync(0xffffffffu, most);
    const float up = up_of(most);
    for (uint32_t s = 0; s < m.spans; ++s) {
      Eight<T> e;
      load8<T, VEC>(row, s * kSpan, lane, m.cols, e);
      float2 v[4];
      floats_of(e, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], both(up));
      Eight<__half> hi, lo;
      halves(v, hi, lo);
      store8<__half, VEC>(static_cast<__half*>(out) + r * stride, s * kSpan, lane, m.cols, hi);
      store8<__half, VEC>(static_cast<__half*>(out) + (m.rows + r) * stride, s * kSpan, lane, m.cols, lo);
    }
    if (lane == 0) scale[r] = down_of(most);
  }
}
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_head_rows(const __grid_constant__ Source h, const __grid_constant__ Source w, uint32_t blocks_h, void* out_h, void* out_w,
                                                   float* scale_h, float* scale_w, uint32_t stride) {
  let_next_kernel_begin();
  wait_for_last_kernel();
  if (blockIdx.x < blocks_h)
    by_rows<T, VEC>(h, uint64_t(blockIdx.x) * 8 + threadIdx.x / 32, out_h, scale_h, stride);
  else
    by_rows<T, VEC>(w, uint64_t(blockIdx.x - blocks_h) * 8 + threadIdx.x / 32, out_w, scale_w, stride);
}

// ---- behind the products --------------------------------------------------------------------------
// A row's loss from its maximum and sum.  Not lse less the logit: a loss next to 0 keeps its digits where the target is the largest.
__device__ __forceinline__ void finish_row(const Head& a, uint32_t row, float2 v, float* loss, float* lse) {
  const float rest = logf(v.y);
  const int target = target_of(a, row, true);
  lse[row] = v.x + rest;
  loss[row] = target < 0 ? 0.0f : v.x - a.at_target[row] + rest;
}
// A row's parts joined in their order: 32 rows a CTA, each eighth part a warp, eight parts on their way together.
__global__ void __launch_bounds__(256) k_head_loss(const __grid_constant__ Head a, float* loss, float* lse) {
  __shared__ float2 s_part[8][32];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, row = blockIdx.x * 32 + lane, parts = a.n_tiles * 4;
  wait_for_last_kernel();
  float2 v = make_float2(kNone, 0.0f);
  const auto join = [&](const float2 (&x)[8]) {
    float most = v.x;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, x[i].x);
    const float from = most == kNone ? 0.0f : most;
    float sum = v.y * exp2f((v.x - from) * kLog2e);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += x[i].y * exp2f((x[i].x - from) * kLog2e);
    v = make_float2(most, sum);
  };
  if (row < a.rows) {
    for (uint32_t p = warp; p < parts; p += 64) {
      float2 x[8];
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) x[i] = p + i * 8 < parts ? a.partial[uint64_t(p + i * 8) * a.rows + row] : make_float2(kNone, 0.0f);
      join(x);
    }
  }
  s_part[warp][lane] = v;
  __syncthreads();
  if (warp || row >= a.rows) return;
  v = make_float2(kNone, 0.0f);
  float2 x[8];
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) x[i] = s_part[i][lane];
  join(x);
  finish_row(a, row, v, loss, lse);
}

// Partial results of dW's piece added up in their order, a warp for 256 columns of a word.
__global__ void __launch_bounds__(256) k_head_words(const __grid_constant__ Head a, const float* parts, float* dw, uint32_t spans) {
  let_next_kernel_begin();
  wait_for_last_kernel();
  const uint32_t lane = threadIdx.x % 32, words = min(a.piece_cols, a.words - a.first_word);
  const uint64_t each = uint64_t(a.piece_cols) * a.width, units = uint64_t(words) * spans;
  const Down by_g = downs_of(*a.most_g);
  for (uint64_t u = uint64_t(blockIdx.x) * 8 + threadIdx.x / 32; u < units; u += uint64_t(gridDim.x) * 8) {
    const uint32_t word = units >> 32 ? uint32_t(u / spans) : uint32_t(u) / spans, col0 = uint32_t(u - uint64_t(word) * spans) * kSpan;
    float v[8] = {};
#pragma unroll 4
    for (uint32_t s = 0; s < a.dw.splits; ++s)
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t c = col0 + i * 32 + lane;
        if (c < a.width) v[i] += parts[s * each + uint64_t(word) * a.width + c];
      }
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      const uint32_t c = col0 + i * 32 + lane;
      if (c < a.width) {
        float* p = dw + (uint64_t(a.first_word) + word) * a.width + c;
        const float x = v[i] * (downs_of(a.most_h[c]) * by_g);
        *p = a.add ? *p + x : x;
      }
    }
  }
}
// dh from many partial results: 32 columns of a row a CTA, each eighth part a warp.  A gradient by this / by k_head_hidden, us, rows x width x words: from up to four parts 700 x 512 x 3000
// 44 / 38, 1000 x 256 x 4000 43 / 40; from six or eight 70 x 2048 x 8000 76 / 78, 1500 x 128 x 1000 49 / 47; from more 100 x 128 x 5000 31 / 45, 128 x 768 x 50257 138 / 149.
constexpr uint32_t kManyParts = 6;
template <class T>
__global__ void __launch_bounds__(256) k_head_join(const __grid_constant__ Head a, const float* parts, uint32_t count, T* dh, uint64_t stride, uint32_t spans) {
  __shared__ float s_sum[8][32];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, row = blockIdx.x / spans, c = (blockIdx.x - row * spans) * 32 + lane;
  const uint64_t each = uint64_t(a.rows) * a.width;
  wait_for_last_kernel();
  float v = 0.0f;
  if (c < a.width)
#pragma unroll 8
    for (uint32_t p = warp; p < count; p += 8) v += parts[p * each + uint64_t(row) * a.width + c];
  s_sum[warp][lane] = v;
  __syncthreads();
  if (warp || c >= a.width) return;
  for (uint32_t q = 1; q < 8; ++q) v += s_sum[q][lane];
  if (a.most_w) v = v * (downs_of(a.most_w[c]) * downs_of(*a.most_g));   // NULL: the parts are what they stand for
  dh[row * stride + c] = Elem<T>::put(target_of(a, row, false) >= 0 ? v : 0.0f);   // also where W holds infinities
}
// And from few, likewise a warp for 256 columns.
template <class T>
__global__ void __launch_bounds__(256) k_head_hidden(const __grid_constant__ Head a, const float* parts, T* dh, uint64_t stride, uint32_t spans) {
  wait_for_last_kernel();
  const uint32_t lane = threadIdx.x % 32;
  const uint64_t each = uint64_t(a.rows) * a.width, units = uint64_t(a.rows) * spans;
  const Down by_g = downs_of(*a.most_g);
  for (uint64_t u = uint64_t(blockIdx.x) * 8 + threadIdx.x / 32; u < units; u += uint64_t(gridDim.x) * 8) {
    const uint32_t row = units >> 32 ? uint32_t(u / spans) : uint32_t(u) / spans, col0 = uint32_t(u - uint64_t(row) * spans) * kSpan;
    float v[8] = {};
    for (uint32_t s = 0; s < a.dh.splits; ++s)
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t c = col0 + i * 32 + lane;
        if (c < a.width) v[i] += parts[s * each + uint64_t(row) * a.width + c];
      }
    const bool live = target_of(a, row, false) >= 0;   // others: 0, also where W holds infinities
    uint32_t most[8];   // on their way together: 2000 x 512 x 8000 10 us, 22 where each is asked for as it is needed
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) most[i] = col0 + i * 32 + lane < a.width ? a.most_w[col0 + i * 32 + lane] : 0;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
      const uint32_t c = col0 + i * 32 + lane;
      if (c < a.width) dh[row * stride + c] = Elem<T>::put(live ? v[i] * (downs_of(most[i]) * by_g) : 0.0f);
    }
  }
}

}  // namespace
}  // namespace dgs

#include "dgs_vocabulary_few.cuh"

namespace dgs {
namespace {

// ---- host side --------------------------------------------------------------------------------
uint32_t ceil_div(uint64_t a, uint64_t b) { return uint32_t((a + b - 1) / b); }
uint64_t up_to(uint64_t v, uint64_t by) { return (v + by - 1) / by * by; }

// Whether TMA copies can take the matrix where it is.
bool in_place(const dgs_matrix* m) {
  return m->type != DGS_TYPE_F32 && on_16_bytes(m) && m->stride >= m->cols && m->rows <= kMostElements / 4 / m->stride;
}

// How both products of a piece's s are split among 74 pairs of CTAs: runs of their steps, and tiles of dh for the pairs with more and with fewer tiles of dW.
struct Shares {
  uint32_t words, hidden, few, more;   // runs of steps; tiles
  double us;
};
struct Work {
  uint32_t tiles, steps;
  double step_us;
  uint64_t results;
};
constexpr double kTileUs = 3.0;   // of a tile's beginning and end
double run_us(const Work& w, uint32_t splits) { return ceil_div(w.steps, splits) * w.step_us + kTileUs; }
Shares share_out(const Work& words, uint32_t sw, const Work& hidden, uint32_t sh) {
  const uint64_t pairs = std::min<uint64_t>(kSms / 2, uint64_t(words.tiles) * sw + uint64_t(hidden.tiles) * sh);
  const uint64_t tw = uint64_t(words.tiles) * sw, th = uint64_t(hidden.tiles) * sh, some = tw % pairs, q = tw / pairs;
  const double cw = run_us(words, sw), ch = run_us(hidden, sh);
  Shares best = {sw, sh, 0, 0, 1e300};
  for (uint64_t few = 0; few <= ceil_div(th, pairs); ++few) {   // for the `some` pairs with q + 1 tiles of dW
    const uint64_t left = th - std::min(th, few * some), more = ceil_div(left, pairs - some);
    const double us = std::max(some ? (q + 1) * cw + few * ch : 0.0, q * cw + more * ch);
    if (us < best.us) best.us = us, best.few = uint32_t(few), best.more = uint32_t(more);
    if (some == 0) break;
  }
  // partial results are written and read again
  if (sw > 1) best.us += 3.0 + double(words.results) * 4e-6 * (sw + 1) / 2.5;
  best.us += double(hidden.results) * 4e-6 * sh / 2.5;
  return best;
}
Shares share_out(const Work& words, const Work& hidden) {
  constexpr uint32_t kRuns[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  Shares best = {1, 1, 0, 0, 1e300};
  for (const uint32_t sw : kRuns) {
    if (sw > 1 && (sw > words.steps || uint64_t(words.tiles) * (sw - 1) > kSms)) break;
    for (const uint32_t sh : kRuns) {
      if (sh > 1 && (sh > hidden.steps || uint64_t(hidden.tiles) * (sh - 1) > kSms)) break;
      const Shares s = share_out(words, sw, hidden, sh);
      if (s.us < best.us) best = s;
    }
  }
  return best;
}

// Of s, where one tile of words does not take more.  At 160 / 320 / 640 MB, us a gradient: 8192 x 768 x 50257 in bfloat16 2510 / 2370 / 2390 (by itself, cool), 16384 x 256 x 20000 1018 / 912 / 850,
// 1000 x 768 x 50257 363 / 352 / 352: what twice the memory would give is not worth it to a caller who keeps a model there.
constexpr uint64_t kPieceBytes = 320ull << 20;

struct HeadPlan {
  uint32_t parts, stride, piece_tiles, pieces, row_blocks;
  bool copy_h, copy_w;
  uint32_t few, few_ctas, few_words, few_tiles;   // few: rows at a time without tensor cores, 0: with them; words of a tile
  Work words, hidden;   // of a whole piece
  Shares shares;
  uint64_t inner_h, inner_w, scales, most, outer_h, outer_w, s, part_w, part_h, partial, at_target, bytes;
};

bool head_ok(const dgs_matrix* h, const dgs_matrix* w) { return matrix_ok(h, false) && matrix_ok(w, false) && h->type == w->type && h->cols == w->cols && w->rows; }

// Steps of 64 values: a product 0.40 us; two of either gradient, of f32 three.
constexpr double kProductUs = 0.40;
Work words_of(uint64_t n, uint32_t d, uint32_t tiles, uint32_t type) {
  return {tiles * ceil_div(d, 256), ceil_div(n, 64), kProductUs * (type == DGS_TYPE_F32 ? 3 : 2), uint64_t(tiles) * 256 * d};
}
Work hidden_of(uint64_t n, uint32_t d, uint32_t tiles, uint32_t type) {
  return {ceil_div(n, 256) * ceil_div(d, 256), tiles * 4, kProductUs * (type == DGS_TYPE_F32 ? 3 : 2), n * d};
}

// Few rows go without tensor cores where there are not many products in all.  Loss and gradient have borders of their own, so that between them the two form logits in different ways,
// each within its own roundings of them.  Beside the products (a wide vocabulary is read as fast either way) it counts what a warp does without tensor cores: whole spans of 256 columns, for the
// loss as much again as 1024 columns beside them, and more for each row the more rows there are, while the tensor cores take 64 rows as they take one.  A loss of up to 1000 words ends before
// that shows.  Here / with tensor cores, us a call, rows x width x words:
//   loss, 16 bits: 8 x 16 x 8000 10.4 / 10.5, 20000 18.5 / 14.6; 37 x 16 x 1000 10.4 / 10.4, 2500 14.5 / 10.3; 64 x 512 x 1000 10.4 / 12.3, 2500 16.5 / 12.4; 1 x 768 x 50257 18.6 / 30.9;
//     8 x 768 x 8000 12.2 / 14.4, 20000 24.7 / 20.6; 8 x 2048 x 5000 18.7 / 19.0, 8000 20.6 / 20.4
//   loss, f32: 16 x 16 x 50257 47.2 / 41.4; 37 x 768 x 2500 20.4 / 22.7, 5000 28.0 / 25.2; 64 x 768 x 1000 13.0 / 22.6, 2500 25.7 / 22.6; 16 x 768 x 20000 50.1 / 55.0; 8 x 2048 x 50257 112 / 271
//   gradient, 16 bits: 8 x 16 x 20000 32.9 / 40.2, 50257 60.2 / 62.8; 64 x 16 x 1000 20.6 / 26.8, 2500 48.5 / 26.9; 37 x 512 x 1000 18.6 / 24.8, 2500 42.5 / 26.8; 1 x 768 x 20000
//     57.7 / 69.9, 50257 158 / 136; 8 x 768 x 5000 32.9 / 32.9; 16 x 2048 x 1000 30.8 / 35.6; 8 x 2048 x 2500 59.5 / 39.1
//   gradient, f32: 64 x 16 x 2500 43.3 / 34.9, 5000 55.2 / 38.3; 64 x 512 x 1000 25.1 / 39.0, 2500 61.6 / 41.1; 8 x 768 x 50257 188 / 275; 16 x 2048 x 5000 119 / 116; 24 x 2048 x 5000 169 / 118
// (Over 784 such sizes, 16 to 2048 columns, the choice costs 0.3 to 0.8 % against the better of the two each time, at the worst a half; by products alone it cost 4 to 13 % and up to six times,
// by spans and rows alone 1 % and up to 2.4 times.)
bool few_rows(uint64_t n, uint64_t v, uint32_t d, uint32_t type, bool grad) {
  if (n > kFewRows) return false;
  const bool f32 = type == DGS_TYPE_F32;
  const uint64_t rows = n == 1 ? 1 : n <= 4 ? 4 : up_to(n, 8), products = rows * v * d, spans = up_to(d, 256);
  if (grad) return products <= (f32 ? 465000000 : 36000000) && rows * (f32 ? rows : rows + 16) * v * spans <= (f32 ? 3760000000 : 1330000000);
  return products <= (f32 ? 960000000 : 200000000) && (v <= 1000 || rows * rows * v * (spans + 1024) <= (f32 ? 10600000000 : 1450000000));
}

int plan_head(const dgs_matrix* h, const dgs_matrix* w, bool grad, HeadPlan* out) {
  if (!head_ok(h, w)) return DGS_EINVAL;
  const uint64_t n = h->rows, v = w->rows;
  const uint32_t d = h->cols;
  // The last plans of this thread, of a loss and of a gradient: a call and its question for bytes ask for one, and a training loop for both in turn.
  struct Key {
    uint64_t n, v, d, type, copies;
  };
  thread_local Key keys[2] = {};
  thread_local HeadPlan plans[2];
  Key& last = keys[grad];
  HeadPlan& plan = plans[grad];
  HeadPlan* const p = &plan;
  const Key key = {n, v, d, h->type, uint64_t(!in_place(h)) | uint64_t(!in_place(w)) << 1};
  if (last.d && memcmp(&key, &last, sizeof(key)) == 0) {
    *out = plan;
    return DGS_OK;
  }
  last.d = 0;
  *p = {};
  p->parts = h->type == DGS_TYPE_F32 ? 2 : 1;
  p->stride = uint32_t(up_to(d, 8));
  // rows are 31-bit coordinates of TMA copies and may be passed by a tile; strides of a plane are 40 bits
  if (d > (1u << 24) || n > (1u << 30) || v > (1u << 30) || std::max(n, v) * p->stride > kMostElements / 4 ||
      uint64_t(ceil_div(n, 256)) * ceil_div(v, 256) > 0x3fffffffu)
    return DGS_ELIMIT;
  if (n && few_rows(n, v, d, h->type, grad)) {
    p->few = n == 1 ? 1 : n <= 4 ? 4 : 8;
    if (grad) {
      // Small tiles where the words are few; their CTAs fill an SM, two of the others share one.  Here / with 32 words, us a call, rows x width x words in bfloat16 (f32 alike): 3 x 512 x 1184
      // 12.3 / 14.5, 2368 18.5 / 14.4; 37 x 512 x 1184 18.8 / 51, 2368 33 / 51, 3000 43 / 51, 6000 80 / 64; 64 x 16 x 3000 49 / 57, 6000 94 / 62; 64 x 1024 x 3000 146 / 162, 6000 314 / 215.
      p->few_words = v <= 8 * kSms * (n <= 4 ? 1 : 3) ? 8 : 32;
      p->few_tiles = ceil_div(v, p->few_words);
      p->few_ctas = std::min(p->few_tiles, kSms * 2);
      p->part_h = up_to(uint64_t(p->few_ctas) * n * d * 4, 256);
      p->bytes = p->part_h;
    } else {
      const uint32_t passes = ceil_div(v, 8 * kFewWords);   // of a CTA; all make as many
      p->few_ctas = ceil_div(passes, ceil_div(passes, kSms * 4));
      p->partial = up_to(uint64_t(p->few_ctas) * n * 8, 256);
      p->at_target = up_to(n * 4, 256);
      p->bytes = p->partial + p->at_target;
    }
    last = key;
    *out = plan;
    return DGS_OK;
  }
  if (n) {
    p->copy_h = !in_place(h);
    p->copy_w = !in_place(w);
    p->inner_h = p->copy_h ? up_to(p->parts * n * p->stride * 2, 256) : 0;
    p->inner_w = p->copy_w ? up_to(p->parts * v * p->stride * 2, 256) : 0;
    p->scales = p->parts == 2 ? up_to((n + v) * 4, 256) : 0;
    p->bytes = p->inner_h + p->inner_w + p->scales;
  }
  if (n && !grad) {
    p->partial = up_to(uint64_t(ceil_div(v, 256)) * 4 * n * 8, 256);
    p->at_target = up_to(n * 4, 256);
    p->bytes += p->partial + p->at_target;
  } else if (n) {
    // Pieces: as many as give the shortest time for the three products of them all.
    const uint32_t m_tiles = ceil_div(n, 256), v_tiles = ceil_div(v, 256);
    const uint32_t most = uint32_t(std::max<uint64_t>(1, kPieceBytes / (uint64_t(m_tiles) * 256 * 256 * 4))), least = ceil_div(v_tiles, most);
    double best = 1e300;
    for (uint32_t pieces = least; pieces < least + 12 && pieces <= v_tiles; ++pieces) {
      const uint32_t t = ceil_div(v_tiles, pieces), count = ceil_div(v_tiles, t);
      if (t == p->piece_tiles) continue;
      const Work words = words_of(n, d, t, h->type), hidden = hidden_of(n, d, t, h->type);
      const Shares shares = share_out(words, hidden);
      const double us = count * (ceil_div(uint64_t(m_tiles) * t, kSms / 2) * (ceil_div(d, 64) * kProductUs * (p->parts == 2 ? 3 : 1) + 1.0) + shares.us + 4.0);
      if (us < best) best = us, p->pieces = count, p->piece_tiles = t, p->words = words, p->hidden = hidden, p->shares = shares;
    }
    if (uint64_t(p->words.tiles) * p->shares.words > 0x3fffffffu || uint64_t(p->hidden.tiles) * p->shares.hidden > 0x3fffffffu) return DGS_ELIMIT;
    p->row_blocks = m_tiles * 2;
    p->most = up_to((2 * uint64_t(d) + 1) * 4, 256);
    p->outer_h = up_to(p->parts * n * p->stride * 2, 256);
    p->outer_w = up_to(p->parts * v * p->stride * 2, 256);
    p->s = 2ull * p->row_blocks * p->piece_tiles * 4 * kBlockBytes;
    p->part_w = p->shares.words > 1 ? up_to(p->shares.words * p->words.results * 4, 256) : 0;
    p->part_h = up_to(p->shares.hidden * p->hidden.results * 4, 256);
    p->bytes += p->most + p->outer_h + p->outer_w + p->s + p->part_w + p->part_h;
  }
  last = key;
  *out = plan;
  return DGS_OK;
}

constexpr int kMaxDevices = 64;
std::mutex g_head_mu;
bool g_head_ready[kMaxDevices];
PFN_cuTensorMapEncodeTiled_v12000 g_head_encode;   // written once, under the mutex
template <int MODE, uint32_t PA, uint32_t PB>
bool head_setup() {
  cudaFuncAttributes f;
  // the split of the registers counts on what the launch brings
  return cudaFuncGetAttributes(&f, k_head<MODE, PA, PB>) == cudaSuccess && uint32_t(f.numRegs) >= kHeadRegs &&
         cudaFuncSetAttribute(k_head<MODE, PA, PB>, cudaFuncAttributeMaxDynamicSharedMemorySize, Step<MODE, PA, PB>::kSmem) == cudaSuccess;
}
int head_ready() {   // once per device
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return DGS_ECUDA;
  std::lock_guard<std::mutex> lock(g_head_mu);
  if (!g_head_ready[dev]) {
    if (!head_setup<kLoss, 1, 1>() || !head_setup<kLoss, 2, 2>() || !head_setup<kSlope, 1, 1>() || !head_setup<kSlope, 2, 2>() ||
        !head_setup<kGrads, 1, 2>() || !head_setup<kGrads, 2, 2>())
      return DGS_ECUDA;
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess || !fn) return DGS_ECUDA;
    g_head_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    g_head_ready[dev] = true;
  }
  return DGS_OK;
}

int head_map(const void* data, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t parts, bool bf16, uint32_t box_rows, CUtensorMap* map) {
  const cuuint64_t dims[3] = {cols, rows, parts}, strides[2] = {stride * 2, rows * stride * 2};
  const cuuint32_t box[3] = {64, box_rows, 1}, each[3] = {1, 1, 1};
  return g_head_encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(data), dims, strides, box, each,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? DGS_OK
             : DGS_ECUDA;
}

// Calls f with a null pointer of the element type, whether rows begin on 16 bytes, and how many rows go together.
template <class F>
int with_few(const dgs_matrix* h, const dgs_matrix* w, uint32_t few, F&& f) {
  return with_wide(h->type, on_16_bytes(h) && on_16_bytes(w), [&](auto* t, auto vec) {
    return few == 1 ? f(t, vec, std::integral_constant<uint32_t, 1>{}) : few == 4 ? f(t, vec, std::integral_constant<uint32_t, 4>{}) : f(t, vec, std::integral_constant<uint32_t, 8>{});
  });
}

template <int MODE, uint32_t PA, uint32_t PB>
int head_launch(const Head& a, uint32_t tiles, const CUtensorMap& x, const CUtensorMap& y, bool early, cudaStream_t st) {
  EarlyLaunch l(dim3(std::min(tiles, kSms / 2) * 2), kHeadThreads, Step<MODE, PA, PB>::kSmem, st);
  if (!early) l.cfg.numAttrs = 0;
  return cudaLaunchKernelEx(&l.cfg, k_head<MODE, PA, PB>, a, x, y) == cudaSuccess ? DGS_OK : DGS_ECUDA;
}

Source source_of(const dgs_matrix* m) { return {m->data, m->stride, uint32_t(m->rows), m->cols, (m->cols + kSpan - 1) / kSpan}; }
constexpr uint32_t kIdescF32 = 1u << 4 | (256u >> 4) << 24, kIdescBf16 = 1u << 7 | 1u << 10;

// The logits' operands and their maps; `launched` is set where a kernel has been enqueued.
int inner_operands(const dgs_matrix* h, const dgs_matrix* w, const HeadPlan& p, char* work, Head* a, CUtensorMap* map_h, CUtensorMap* map_w, bool* launched, cudaStream_t st) {
  const bool bf16 = h->type == DGS_TYPE_BF16;
  const uint64_t n = h->rows, v = w->rows;
  float* const scales = reinterpret_cast<float*>(work + p.inner_h + p.inner_w);
  a->row_h = scales;
  a->row_w = scales + n;
  if (p.copy_h || p.copy_w) {
    const uint32_t blocks_h = p.copy_h ? ceil_div(n, 8) : 0, blocks_w = p.copy_w ? ceil_div(v, 8) : 0;
    // a matrix that stays where it is has no say in how the other one is read
    const bool vec = (!p.copy_h || on_16_bytes(h)) && (!p.copy_w || on_16_bytes(w));
    const int rc = with_wide(h->type, vec, [&](auto* t, auto wide) {
      using T = std::remove_pointer_t<decltype(t)>;
      EarlyLaunch l(dim3(blocks_h + blocks_w), 256, 0, st);
      if (!*launched) l.cfg.numAttrs = 0;
      return cudaLaunchKernelEx(&l.cfg, k_head_rows<T, wide.value>, source_of(h), source_of(w), blocks_h, static_cast<void*>(work), static_cast<void*>(work + p.inner_h), scales,
                                scales + n, p.stride) == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
    });
    if (rc != DGS_OK) return rc;
    *launched = true;
  }
  int rc = head_map(p.copy_h ? work : h->data, n, h->cols, p.copy_h ? p.stride : h->stride, p.parts, bf16, 128, map_h);
  if (rc == DGS_OK) rc = head_map(p.copy_w ? work + p.inner_h : w->data, v, w->cols, p.copy_w ? p.stride : w->stride, p.parts, bf16, 128, map_w);
  return rc;
}

Head head_of(const dgs_matrix* h, const dgs_matrix* w, const void* target, uint32_t flags) {
  Head a = {};
  a.rows = uint32_t(h->rows);
  a.width = h->cols;
  a.words = uint32_t(w->rows);
  a.m_tiles = ceil_div(h->rows, 256);
  a.idesc = kIdescF32 | (h->type == DGS_TYPE_BF16 ? kIdescBf16 : 0);
  a.target = target;
  a.wide_targets = flags & DGS_TARGET_I64 ? 1 : 0;
  a.status = operator_status_word();
  return a;
}

Few few_of(const dgs_matrix* h, const dgs_matrix* w, const HeadPlan& p) { return {h->data, w->data, h->stride, w->stride, (h->cols + kSpan - 1) / kSpan, p.few_tiles}; }

// Loss and gradient sum a logit the same way, bit by bit: the values of a chunk are a whole number of either's steps, and are counted in the loss', the longer ones.
template <int MODE, uint32_t P>
void logit_chunks(Head* a) {
  constexpr uint32_t kMine = Step<MODE, P, P>::kRows, kLong = Step<kLoss, P, P>::kRows;
  static_assert(kLong % kMine == 0 && Step<MODE, P, P>::kChunk * kMine == Step<kLoss, P, P>::kChunk * kLong, "the same values in loss and gradient");
  a->steps = ceil_div(a->width, kMine);
  const uint32_t steps = ceil_div(a->width, kLong), chunk = std::min(ceil_div(steps, 2), Step<kLoss, P, P>::kChunk);
  a->chunk = chunk * (kLong / kMine);
  a->skip = (ceil_div(steps, chunk) * chunk - steps) * (kLong / kMine);   // the last step's values may be few: what a chunk is short of is at the other end
}
template <int MODE>
void logit_steps(uint32_t parts, Head* a) { parts == 2 ? logit_chunks<MODE, 2>(a) : logit_chunks<MODE, 1>(a); }

}  // namespace
}  // namespace dgs

using namespace dgs;

extern "C" int dgs_vocabulary_loss_bytes(const dgs_matrix* hidden, const dgs_matrix* weight, uint64_t* out_bytes) {
  HeadPlan p;
  if (!out_bytes) return DGS_EINVAL;
  const int rc = plan_head(hidden, weight, false, &p);
  if (rc == DGS_OK) *out_bytes = p.bytes;
  return rc;
}

extern "C" int dgs_vocabulary_loss(const dgs_matrix* hidden, const dgs_matrix* weight, const void* target, uint32_t flags, float* loss, float* lse, void* workspace,
                                   uint64_t workspace_bytes, void* stream) {
  HeadPlan p;
  if (flags & ~DGS_TARGET_I64) return DGS_EINVAL;
  int rc = plan_head(hidden, weight, false, &p);
  if (rc != DGS_OK) return rc;
  const uint64_t n = hidden->rows, size = flags & DGS_TARGET_I64 ? 8 : 4;
  if (!aligned(target, size) || !aligned(loss, 4) || !aligned(lse, 4) || (n && (!target || !loss || !lse))) return DGS_EINVAL;
  if (p.bytes && (!workspace || !aligned(workspace, 256))) return DGS_EINVAL;
  if (workspace_bytes < p.bytes) return DGS_ENOMEM;
  const Span part[] = {{hidden->data, span_bytes(hidden), false}, {weight->data, span_bytes(weight), false}, {target, n * size, false},
                       {loss, n * 4, true}, {lse, n * 4, true}, {workspace, p.bytes, true}};
  if (!apart(part)) return DGS_EINVAL;
  if (n == 0) return DGS_OK;
  Head a = head_of(hidden, weight, target, flags);
  if (!a.status) return DGS_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* const work = static_cast<char*>(workspace);
  if (p.few) {
    a.partial = reinterpret_cast<float2*>(work);
    a.at_target = reinterpret_cast<float*>(work + p.partial);
    const Few f = few_of(hidden, weight, p);
    rc = with_few(hidden, weight, p.few, [&](auto* t, auto vec, auto together) {
      using T = std::remove_pointer_t<decltype(t)>;
      k_few_loss<T, vec.value, together.value><<<dim3(p.few_ctas, ceil_div(n, p.few)), 256, 0, st>>>(a, f);
      return cudaGetLastError() == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
    });
    if (rc != DGS_OK) return rc;
    const EarlyLaunch l(dim3(uint32_t(n)), 256, 0, st);
    return cudaLaunchKernelEx(&l.cfg, k_few_rows, a, p.few_ctas, loss, lse) == cudaSuccess ? DGS_OK : DGS_ECUDA;
  }
  if ((rc = head_ready()) != DGS_OK) return rc;
  CUtensorMap map_h = {}, map_w = {};
  bool launched = false;
  if ((rc = inner_operands(hidden, weight, p, work, &a, &map_h, &map_w, &launched, st)) != DGS_OK) return rc;
  a.n_tiles = ceil_div(a.words, 256);
  a.tiles = a.m_tiles * a.n_tiles;
  a.partial = reinterpret_cast<float2*>(work + p.inner_h + p.inner_w + p.scales);
  a.at_target = reinterpret_cast<float*>(work + p.inner_h + p.inner_w + p.scales + p.partial);
  logit_steps<kLoss>(p.parts, &a);
  rc = p.parts == 2 ? head_launch<kLoss, 2, 2>(a, a.tiles, map_h, map_w, launched, st) : head_launch<kLoss, 1, 1>(a, a.tiles, map_h, map_w, launched, st);
  if (rc != DGS_OK) return rc;
  const EarlyLaunch l(dim3(ceil_div(n, 32)), 256, 0, st);
  return cudaLaunchKernelEx(&l.cfg, k_head_loss, a, loss, lse) == cudaSuccess ? DGS_OK : DGS_ECUDA;
}

extern "C" int dgs_vocabulary_loss_grad_bytes(const dgs_matrix* hidden, const dgs_matrix* weight, uint64_t* out_bytes) {
  HeadPlan p;
  if (!out_bytes) return DGS_EINVAL;
  const int rc = plan_head(hidden, weight, true, &p);
  if (rc == DGS_OK) *out_bytes = p.bytes;
  return rc;
}

extern "C" int dgs_vocabulary_loss_grad(const dgs_matrix* hidden, const dgs_matrix* weight, const void* target, const float* lse, const float* dloss, uint32_t dloss_stride,
                                        const dgs_matrix* dhidden, float* dw, uint32_t flags, void* workspace, uint64_t workspace_bytes, void* stream) {
  HeadPlan p;
  if ((flags & ~(DGS_TARGET_I64 | DGS_LOSS_ADD)) || dloss_stride > 1) return DGS_EINVAL;
  int rc = plan_head(hidden, weight, true, &p);
  if (rc != DGS_OK) return rc;
  const uint64_t n = hidden->rows, v = weight->rows, size = flags & DGS_TARGET_I64 ? 8 : 4;
  if (!matrix_ok(dhidden, true) || dhidden->rows != n || dhidden->cols != hidden->cols || dhidden->type != hidden->type) return DGS_EINVAL;
  if (!aligned(target, size) || !aligned(lse, 4) || !aligned(dloss, 4) || !aligned(dw, 4) || (n && (!target || !lse || !dloss))) return DGS_EINVAL;
  if (p.bytes && (!workspace || !aligned(workspace, 256))) return DGS_EINVAL;
  if (workspace_bytes < p.bytes) return DGS_ENOMEM;
  const uint64_t dw_bytes = dw ? v * hidden->cols * 4 : 0;
  const Span part[] = {{hidden->data, span_bytes(hidden), false}, {weight->data, span_bytes(weight), false}, {target, n * size, false}, {lse, n * 4, false},
                       {dloss, n ? (dloss_stride ? n : 1) * 4 : 0, false}, {dhidden->data, span_bytes(dhidden), true}, {dw, dw_bytes, true}, {workspace, p.bytes, true}};
  if (!apart(part)) return DGS_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (n == 0) return !dw || (flags & DGS_LOSS_ADD) || cudaMemsetAsync(dw, 0, dw_bytes, st) == cudaSuccess ? DGS_OK : DGS_ECUDA;
  Head a = head_of(hidden, weight, target, flags);
  if (!a.status) return DGS_ECUDA;
  if (p.few) {
    a.lse = lse;
    a.dloss = dloss;
    a.dloss_step = dloss_stride;
    a.add = flags & DGS_LOSS_ADD ? 1 : 0;
    const Few f = few_of(hidden, weight, p);
    float* const parts = static_cast<float*>(workspace);
    return with_few(hidden, weight, p.few, [&](auto* t, auto vec, auto together) {
      using T = std::remove_pointer_t<decltype(t)>;
      if (p.few_words == 8)
        k_few_grad<T, vec.value, together.value, 8><<<p.few_ctas, kFewThreads<8>, 0, st>>>(a, f, dw, parts);
      else
        k_few_grad<T, vec.value, together.value, 32><<<p.few_ctas, kFewThreads<32>, 0, st>>>(a, f, dw, parts);
      if (cudaGetLastError() != cudaSuccess) return int(DGS_ECUDA);
      const uint32_t spans = ceil_div(a.width, 32);
      const EarlyLaunch l(dim3(spans * a.rows), 256, 0, st);
      return cudaLaunchKernelEx(&l.cfg, k_head_join<T>, a, static_cast<const float*>(parts), p.few_ctas, static_cast<T*>(dhidden->data), dhidden->stride, spans) == cudaSuccess
                 ? int(DGS_OK)
                 : int(DGS_ECUDA);
    });
  }
  if ((rc = head_ready()) != DGS_OK) return rc;
  char* at = static_cast<char*>(workspace);
  char* const inner = at;
  at += p.inner_h + p.inner_w + p.scales;
  uint32_t* const most = reinterpret_cast<uint32_t*>(at);
  at += p.most;
  __half* const outer_h = reinterpret_cast<__half*>(at);
  at += p.outer_h;
  __half* const outer_w = reinterpret_cast<__half*>(at);
  at += p.outer_w;
  a.s = reinterpret_cast<unsigned char*>(at);
  at += p.s;
  float* const part_w = reinterpret_cast<float*>(at);
  at += p.part_w;
  float* const part_h = reinterpret_cast<float*>(at);
  const uint32_t d = a.width;
  a.most_h = most;
  a.most_w = most + d;
  a.most_g = most + 2 * uint64_t(d);
  a.lse = lse;
  a.dloss = dloss;
  a.dloss_step = dloss_stride;
  a.add = flags & DGS_LOSS_ADD ? 1 : 0;
  a.piece_cols = p.piece_tiles * 256;
  a.plane = p.s / 2;

  if (cudaMemsetAsync(most, 0, p.most, st) != cudaSuccess) return DGS_ECUDA;
  const Source h = source_of(hidden), w = source_of(weight);
  const uint32_t most_h = h.spans * ceil_div(h.rows, kMostRows), most_w = w.spans * ceil_div(w.rows, kMostRows), most_g = std::min(ceil_div(n, 256), kSms);
  const uint32_t blocks_h = h.spans * ceil_div(h.rows, kPlaneRows), blocks_w = w.spans * ceil_div(w.rows, kPlaneRows);
  rc = with_wide(hidden->type, on_16_bytes(hidden) && on_16_bytes(weight), [&](auto* t, auto vec) {
    using T = std::remove_pointer_t<decltype(t)>;
    k_head_most<T, vec.value><<<most_h + most_w + most_g, 256, 0, st>>>(a, h, w, most_h, most_w, most, most + d, most + 2 * uint64_t(d));
    if (cudaGetLastError() != cudaSuccess) return int(DGS_ECUDA);
    const EarlyLaunch l(dim3(blocks_h + blocks_w), 256, 0, st);
    return cudaLaunchKernelEx(&l.cfg, k_head_columns<T, vec.value>, a, h, w, blocks_h, outer_h, outer_w, p.stride) == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
  });
  if (rc != DGS_OK) return rc;
  CUtensorMap inner_h = {}, inner_w = {}, map_h = {}, map_w = {};
  bool launched = true;
  if ((rc = inner_operands(hidden, weight, p, inner, &a, &inner_h, &inner_w, &launched, st)) != DGS_OK) return rc;
  if ((rc = head_map(outer_h, n, d, p.stride, p.parts, false, 64, &map_h)) != DGS_OK) return rc;
  if ((rc = head_map(outer_w, v, d, p.stride, p.parts, false, 64, &map_w)) != DGS_OK) return rc;

  a.dh.out = part_h;
  a.dh.splits = p.shares.hidden;
  a.dw.out = p.shares.words > 1 ? part_w : dw;
  a.dw.splits = p.shares.words;
  logit_steps<kSlope>(p.parts, &a);
  for (uint32_t piece = 0; piece < p.pieces; ++piece) {
    const uint32_t tile0 = piece * p.piece_tiles, tiles = std::min(p.piece_tiles, ceil_div(v, 256) - tile0);
    Head s = a;
    s.first_word = tile0 * 256;
    s.first_piece = piece == 0;
    s.n_tiles = tiles;
    s.tiles = s.m_tiles * tiles;
    rc = p.parts == 2 ? head_launch<kSlope, 2, 2>(s, s.tiles, inner_h, inner_w, true, st) : head_launch<kSlope, 1, 1>(s, s.tiles, inner_h, inner_w, true, st);
    if (rc != DGS_OK) return rc;
    s.idesc = kIdescF32;
    s.dw.m_tiles = s.dh.m_tiles = ceil_div(d, 256);
    s.dw.n_tiles = tiles;
    s.dw.steps = ceil_div(n, 64);
    s.dw.tiles = dw ? s.dw.m_tiles * s.dw.n_tiles * s.dw.splits : 0;
    s.dh.n_tiles = a.m_tiles;
    s.dh.steps = ceil_div(std::min<uint64_t>(tiles * 256, v - s.first_word), 64);
    s.dh.tiles = s.dh.m_tiles * s.dh.n_tiles * s.dh.splits;
    // the last piece may be shorter, and dW not wanted
    Work words = words_of(n, d, tiles, hidden->type), of_h = hidden_of(n, d, tiles, hidden->type);
    if (!dw) words.tiles = 0;
    const Shares shares = dw && tiles == p.piece_tiles ? p.shares : share_out(words, s.dw.splits, of_h, s.dh.splits);
    s.share_few = shares.few;
    s.share_more = shares.more;
    const uint32_t all = s.dw.tiles + s.dh.tiles;
    rc = p.parts == 2 ? head_launch<kGrads, 2, 2>(s, all, map_h, map_w, true, st) : head_launch<kGrads, 1, 2>(s, all, map_h, map_w, true, st);
    if (rc != DGS_OK) return rc;
    if (dw && s.dw.splits > 1) {
      const EarlyLaunch l(dim3(uint32_t(std::min<uint64_t>((uint64_t(tiles) * 256 * w.spans + 7) / 8, kSms * 16))), 256, 0, st);
      if (cudaLaunchKernelEx(&l.cfg, k_head_words, s, static_cast<const float*>(part_w), dw, w.spans) != cudaSuccess) return DGS_ECUDA;
    }
  }
  return with_type(hidden->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    T* const to = static_cast<T*>(dhidden->data);
    if (a.dh.splits >= kManyParts) {
      const uint32_t spans = ceil_div(d, 32);
      const EarlyLaunch l(dim3(spans * a.rows), 256, 0, st);
      return cudaLaunchKernelEx(&l.cfg, k_head_join<T>, a, static_cast<const float*>(part_h), a.dh.splits, to, dhidden->stride, spans) == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
    }
    const EarlyLaunch l(dim3(uint32_t(std::min<uint64_t>((n * h.spans + 7) / 8, kSms * 16))), 256, 0, st);
    return cudaLaunchKernelEx(&l.cfg, k_head_hidden<T>, a, static_cast<const float*>(part_h), to, dhidden->stride, h.spans) == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
  });
}
