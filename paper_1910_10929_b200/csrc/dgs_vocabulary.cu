// Softmax cross entropy over a vocabulary and its gradient, without keeping the logits: dgs_vocabulary_loss and dgs_vocabulary_loss_grad.
//
// With hidden states h [N][D], a vocabulary W [V][D] and z = h W^T:
//     loss[r] = lse[r] - z[r][target[r]],  lse[r] = log(sum over v of exp z[r][v]),
//     s[r][v] = dloss[r] (exp(z[r][v] - lse[r]) - [v = target[r]]),  dh = s W,  dW = s^T h.
// The loss keeps a maximum and a sum for each row and 128 words of a tile of logits, which stay in registers.  The gradient goes through the vocabulary in
// pieces: the logits of a piece are formed again, s of the piece goes to the workspace, and its products with W and h are formed from there.
//
// Numbers: s is kept as the sum of two fp16 numbers (22 bits) under one power of two for the call, since dW goes to a flat gradient in f32; products of fp16 need
// fp16 partners, so W and h are held beside as fp16 numbers under a power of two for each column: exact for bfloat16 and fp16 values down to 2^-29 of their column's
// largest, and below that to 2^-40 of it.  f32 matrices are sums of two fp16 numbers each; of their four products the smallest, under 2^-22 of the whole, is left out.
// dh of bfloat16 is formed from the first part of s alone: 12 bits where the result keeps 8.
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
__device__ __forceinline__ void bulk_store(void* to, uint32_t from, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n cp.async.bulk.commit_group;" ::"l"(to), "r"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// What the kernel forms: maxima and sums of logits; s of a piece; dW of a piece from s and h; dh's part of a piece from s and W.
enum : int { kLoss, kSlope, kWords, kHidden };
template <int MODE> constexpr bool kFromPiece = MODE == kWords || MODE == kHidden;

// A pair of CTAs forms tiles of 256 x n, 128 rows and n columns of it in each CTA's tensor memory.  A step contracts kRows values of the operands' PA and PB
// parts; a CTA brings 128 rows (or columns) of the first operand and n / 2 of the second, 256 bytes a value contracted.
//   contracted dimension contiguous (h and W for the logits, s for dh): blocks of 64 values contracted, 128 rows of 128 bytes each
//   contracted dimension outermost (h and s for dW, W for dh): blocks of 64 columns, kRows rows of 128 bytes each
// Either way the 16-byte pieces of a row are exchanged by its number (128-byte swizzle).  s lies in the workspace in blocks of 128 rows and 64 columns that are in
// that order already, so both uses copy it as it is.
template <uint32_t PA, uint32_t PB> struct Step {
  static constexpr uint32_t kRows = PA * PB == 1 ? 128 : 64, kTile = kRows * 256, kStage = (PA + PB) * kTile, kStages = 192 * 1024 / kStage;
};
// Steps between two sums in registers.  Logits: each step, since an exponential takes a logit's error as it is (a logit of 15 summed over 768 values in one go is off by
// 7e-6, a step at a time by 1.5e-6).  Sums of s: 512 rows, 256 where each is three products.
template <int MODE, uint32_t PA, uint32_t PB> constexpr uint32_t kChunkSteps = !kFromPiece<MODE> ? 1 : PA == 2 ? 4 : 512 / Step<PA, PB>::kRows;
constexpr uint32_t kBlockBytes = 128 * 128;                       // 128 rows and 64 columns of s
constexpr uint32_t kStageBytes = 32 * 1024;                       // s on its way out: 4 KB a warp
constexpr uint32_t kSmem = 1024 + 192 * 1024 + kStageBytes;
constexpr uint32_t kHeadThreads = 384, kHeadRegs = 168, kHeadRegsSum = 216, kHeadRegsRest = 72;
static_assert(kHeadRegsSum * 256 + kHeadRegsRest * 128 <= kHeadRegs * kHeadThreads, "setmaxnreg draws on the launch's registers");
constexpr uint32_t kHeadTmem = 512;                               // two accumulators of 256 columns

// k: which sixteen of the values contracted.
__device__ __forceinline__ uint64_t desc_inner(uint32_t tile, uint32_t k) {
  return uint64_t(((tile + (k / 4) * kBlockBytes + (k % 4) * 32) >> 4) & 0x3fff) | uint64_t(1) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
template <uint32_t R>
__device__ __forceinline__ uint64_t desc_outer(uint32_t tile, uint32_t k) {
  return uint64_t(((tile + k * 2048) >> 4) & 0x3fff) | uint64_t(R * 128 >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}

// The power of two that takes a largest magnitude (its bits) to [2^14, 2^15), kept where it is a normal number, and its reciprocal.  Infinities and NaN: 1.
__device__ __forceinline__ float up_of(uint32_t largest) {
  const int e = int(largest >> 23);   // biased exponent
  if (e == 0xff || largest == 0) return 1.0f;
  return __uint_as_float(uint32_t(min(127 + 14 + 127 - max(e, 1), 253)) << 23);
}
__device__ __forceinline__ float down_of(uint32_t largest) { return __uint_as_float((254u << 23) - __float_as_uint(up_of(largest))); }
constexpr float kLog2e = 1.4426950408889634f;

struct Head {
  uint32_t rows, width, words;      // N, D, V
  uint32_t m_tiles, n_tiles, n, splits, tiles;
  uint32_t steps;                   // over the whole contraction
  uint32_t first_word, piece_cols;  // of the piece (a multiple of 256 in the workspace)
  uint32_t row_blocks;              // of s
  uint32_t idesc;
  uint32_t wide_targets, dloss_step, parts;
  const void* target;
  const float *lse, *dloss;
  const uint32_t *most_h, *most_w, *most_g;     // bits of the largest magnitudes: of each column of h and of W, of dloss
  const float *row_h, *row_w;       // f32: what the rows of the logits' operands are multiplied with
  float2* partial;                  // [n_tiles * 2][rows]: maximum, sum
  float* at_target;                 // [rows]
  unsigned char* s;                 // [2][row_blocks][piece_cols / 64] blocks
  float* out;                       // dw, or partial results [splits][...]
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

struct HeadTile {
  uint32_t m0, n0, split, from, steps;
};
// Tiles go down the rows first, 32 tiles of them at a time: the pairs work on few words together, and on rows that the second cache holds.
template <int MODE>
__device__ __forceinline__ HeadTile head_tile(const Head& a, uint32_t tile) {
  HeadTile t;
  t.split = 0;
  if constexpr (kFromPiece<MODE>) {
    t.m0 = tile % a.m_tiles * 256;
    tile /= a.m_tiles;
    t.n0 = tile % a.n_tiles * a.n;
    t.split = tile / a.n_tiles;
  } else {
    const uint32_t group = tile / (32 * a.n_tiles), rows = min(32u, a.m_tiles - group * 32), in = tile - group * 32 * a.n_tiles;
    t.m0 = (group * 32 + in % rows) * 256;
    t.n0 = in / rows * a.n;
  }
  const uint32_t each = (a.steps + a.splits - 1) / a.splits;
  t.from = min(t.split * each, a.steps);
  t.steps = min(each, a.steps - t.from);
  return t;
}

// Warps: 0 to 7 keep the sums, 8 issues products, 9 copies, 10 passes on that copies have landed.  Accumulators go to registers every kChunk steps, since
// the tensor cores add with bits cut off, and are added up there with rounding.  One pair of CTAs per pair of SMs takes tile after tile, so that the
// products of the next run while one is finished.
template <int MODE, uint32_t PA, uint32_t PB>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kHeadThreads, 1)
k_head(const __grid_constant__ Head a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b) {
  using S = Step<PA, PB>;
  constexpr uint32_t R = S::kRows, ST = S::kStages, CH = kChunkSteps<MODE, PA, PB>, TILE = S::kTile;
  constexpr bool kOuterA = kFromPiece<MODE>, kOuterB = MODE == kWords;
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[ST], s_empty[ST], s_loaded[ST], s_sum_full[2], s_sum_empty[2], s_done;
  __shared__ uint32_t s_tmem;
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32, rank = cta_rank(), pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  const uint32_t stages = (smem_at(raw) + 1023u) & ~1023u, half = a.n / 2;

  if (warp == 8) {
    tmem_alloc(&s_tmem, kHeadTmem);
    if (lane == 0) {
      for (uint32_t s = 0; s < ST; ++s) {
        bar_init(smem_at(&s_full[s]), 2);    // that copies landed, of both CTAs
        bar_init(smem_at(&s_empty[s]), 1);
        bar_init(smem_at(&s_loaded[s]), 1);
      }
      for (uint32_t i = 0; i < 2; ++i) {
        bar_init(smem_at(&s_sum_full[i]), 1);
        bar_init(smem_at(&s_sum_empty[i]), 16);
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
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kHeadRegsRest));
    if (warp == 8 && lane == 0 && rank == 0) {
      bool alive = true;
      uint32_t it = 0, chunk = 0;
      const uint32_t idesc = a.idesc | uint32_t(kOuterA) << 15 | uint32_t(kOuterB) << 16 | idesc_cols(a.n);
      for (uint32_t tile = pair; tile < a.tiles && alive; tile += pairs) {
        const HeadTile w = head_tile<MODE>(a, tile);
        for (uint32_t s = 0; s < w.steps; ++s, ++it) {
          const uint32_t st = it % ST, at = stages + st * S::kStage, bt = at + PA * TILE, acc = tmem + (chunk & 1) * 256;
          if (s % CH == 0 && chunk >= 2) alive = bar_wait(smem_at(&s_sum_empty[chunk & 1]), (chunk / 2 - 1) & 1);
          alive = alive && bar_wait(smem_at(&s_full[st]), it / ST & 1);
          if (!alive) break;
          tmem_after();
#pragma unroll
          for (uint32_t k = 0; k < R / 16; ++k) {
#pragma unroll
            for (uint32_t i = 0; i < PA; ++i)
#pragma unroll
              for (uint32_t j = 0; j < PB; ++j)
                if (i + j < 2) {
                  const uint64_t ad = kOuterA ? desc_outer<R>(at + i * TILE, k) : desc_inner(at + i * TILE, k);
                  const uint64_t bd = kOuterB ? desc_outer<R>(bt + j * TILE, k) : desc_inner(bt + j * TILE, k);
                  mma(acc, ad, bd, idesc, s % CH || k || i || j);
                }
          }
          mma_commit(smem_at(&s_empty[st]));
          if (s % CH == CH - 1 || s == w.steps - 1) mma_commit(smem_at(&s_sum_full[chunk++ & 1]));
        }
      }
      mma_commit(smem_at(&s_done));   // waited for in both CTAs, at the end: nothing is under way when tensor memory is given back
      if (!alive) report(a.status, DGS_ETIMEOUT);
    }
    if (warp == 9 && lane == 0) {
      bool alive = true;
      uint32_t it = 0;
      const uint32_t col_blocks = a.piece_cols / 64;
      const uint64_t plane = uint64_t(a.row_blocks) * col_blocks * kBlockBytes;
      for (uint32_t tile = pair; tile < a.tiles && alive; tile += pairs) {
        const HeadTile w = head_tile<MODE>(a, tile);
        const uint32_t m = w.m0 + rank * 128, n = w.n0 + rank * half;
        for (uint32_t s = 0; s < w.steps; ++s, ++it) {
          const uint32_t st = it % ST, at = stages + st * S::kStage, bt = at + PA * TILE, bar = smem_at(&s_loaded[st]), k0 = (w.from + s) * R;
          if (it >= ST && !(alive = bar_wait(smem_at(&s_empty[st]), (it / ST - 1) & 1))) break;
          bar_expect(bar, PA * TILE + PB * (kFromPiece<MODE> ? R * half * 2 : TILE));
#pragma unroll
          for (uint32_t i = 0; i < PA; ++i) {
            if constexpr (kOuterA) {
              for (uint32_t b = 0; b < 2; ++b) tma_load3(at + i * TILE + b * R * 128, &map_a, int(m + b * 64), int((MODE == kHidden ? a.first_word : 0) + k0), int(i), bar);
            } else {
              for (uint32_t b = 0; b < R / 64; ++b) tma_load3(at + i * TILE + b * kBlockBytes, &map_a, int(k0 + b * 64), int(m), int(i), bar);
            }
          }
#pragma unroll
          for (uint32_t j = 0; j < PB; ++j) {
            const unsigned char* from = a.s + j * plane;
            if constexpr (MODE == kWords) {   // rows k0 on of n / 2 columns
              for (uint32_t b = 0; b < half / 64; ++b)
                bulk_load(bt + j * TILE + b * R * 128, from + (uint64_t(k0 / 128) * col_blocks + n / 64 + b) * kBlockBytes + k0 % 128 * 128, R * 128, bar);
            } else if constexpr (MODE == kHidden) {   // columns k0 on of n / 2 rows
              for (uint32_t b = 0; b < R / 64; ++b)
                bulk_load(bt + j * TILE + b * kBlockBytes, from + (uint64_t(n / 128) * col_blocks + k0 / 64 + b) * kBlockBytes + n % 128 * 128, half * 128, bar);
            } else {
              for (uint32_t b = 0; b < R / 64; ++b) tma_load3(bt + j * TILE + b * kBlockBytes, &map_b, int(k0 + b * 64), int(a.first_word + n), int(j), bar);
            }
          }
        }
      }
      // Nothing is under way to this CTA's memory when it leaves: its copies, and the arrivals that the products' commits send to both CTAs.
      for (uint32_t i = it > ST ? it - ST : 0; i < it; ++i) {
        const bool landed = bar_wait(smem_at(&s_loaded[i % ST]), i / ST & 1);
        alive = alive && landed && bar_wait(smem_at(&s_empty[i % ST]), i / ST & 1);
      }
      if (!alive) report(a.status, DGS_ETIMEOUT);
    }
    if (warp == 10 && lane == 0) {
      bool alive = true;
      uint32_t it = 0;
      for (uint32_t tile = pair; tile < a.tiles && alive; tile += pairs) {
        const uint32_t steps = head_tile<MODE>(a, tile).steps;
        for (uint32_t s = 0; s < steps; ++s, ++it) {
          if (!(alive = bar_wait(smem_at(&s_loaded[it % ST]), it / ST & 1))) break;
          bar_arrive_cluster(in_leader(smem_at(&s_full[it % ST])));
        }
      }
      if (!alive) report(a.status, DGS_ETIMEOUT);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kHeadRegsSum));
    const uint32_t quarter = warp % 4, group = warp / 4, mine = rank * 128 + quarter * 32 + lane;
    const uint32_t cols = kFromPiece<MODE> ? half : 128;   // of the tile that a thread has
    bool alive = true;
    uint32_t drained = 0;
    for (uint32_t tile = pair; tile < a.tiles && alive; tile += pairs) {
      const HeadTile w = head_tile<MODE>(a, tile);
      const uint32_t chunks = (w.steps + CH - 1) / CH, row = w.m0 + mine;
      const uint32_t col0 = w.n0 + group * cols;
      // what the end of the tile needs comes while its products are formed
      int target = -1;
      float lse = 0.0f, g = 0.0f, by = 1.0f;
      if constexpr (!kFromPiece<MODE>) {
        if (row < a.rows) {
          target = target_of(a, row, false);
          if constexpr (PA == 2) by = a.row_h[row];
          if (MODE == kSlope && target >= 0) lse = a.lse[row], g = a.dloss[uint64_t(row) * a.dloss_step] * up_of(*a.most_g);
        }
      } else if (row < a.width) {
        by = down_of(MODE == kWords ? a.most_h[row] : a.most_w[row]);
      }
      float acc[128];
#pragma unroll
      for (int i = 0; i < 128; ++i) acc[i] = 0.0f;
      for (uint32_t c = 0; c < chunks; ++c, ++drained) {
        const uint32_t buf = drained & 1;
        if (!(alive = warp_wait(smem_at(&s_sum_full[buf]), drained / 2 & 1))) break;
        tmem_after();
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
          if (!kFromPiece<MODE> || q * 32 < cols) {
            float v[32];
            tmem_load32(tmem + (quarter * 32 << 16) + buf * 256 + group * cols + q * 32, v);
#pragma unroll
            for (int i = 0; i < 32; i += 2) add_to(acc[q * 32 + i], acc[q * 32 + i + 1], v[i], v[i + 1]);
          }
        }
        tmem_before();
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(in_leader(smem_at(&s_sum_empty[buf])));
      }
      if (!alive) break;

      if constexpr (!kFromPiece<MODE>) {
        if (MODE == kLoss && w.m0 + rank * 128 + quarter * 32 >= a.rows) continue;   // no row of the warp's
        const uint32_t word0 = a.first_word + col0;
        if constexpr (PA == 2) {
#pragma unroll
          for (int i = 0; i < 128; ++i) acc[i] = acc[i] * by * (word0 + i < a.words ? a.row_w[word0 + i] : 0.0f);
        }
        if (word0 + 128 > a.words) {
#pragma unroll
          for (uint32_t i = 0; i < 128; ++i)
            if (word0 + i >= a.words) acc[i] = __uint_as_float(0xff800000u);
        }
        const uint32_t at = uint32_t(target) - word0;   // the target's column, if it is one of the thread's
        const bool has = __any_sync(0xffffffffu, target >= 0 && at < 128);
        if constexpr (MODE == kLoss) {
          if (has) {
            float z = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < 128; ++i) z = at == i ? acc[i] : z;
            if (target >= 0 && at < 128) a.at_target[row] = z;
          }
          float most = acc[0];
#pragma unroll
          for (int i = 1; i < 128; ++i) most = fmaxf(most, acc[i]);
          const float from = most == __uint_as_float(0xff800000u) ? 0.0f : most;
          float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
          for (int i = 0; i < 128; i += 2) {
            const float2 d = mul2(add2(make_float2(acc[i], acc[i + 1]), both(-from)), both(kLog2e));
            sum = add2(sum, make_float2(hardware_exp2(d.x), hardware_exp2(d.y)));
          }
          if (row < a.rows) a.partial[uint64_t(col0 / 128) * a.rows + row] = make_float2(most, sum.x + sum.y);
        } else {
          if (target < 0) {   // whatever the row's logits are
#pragma unroll
            for (int i = 0; i < 128; ++i) acc[i] = __uint_as_float(0xff800000u);
          }
#pragma unroll
          for (int i = 0; i < 128; i += 2) {
            const float2 d = mul2(add2(make_float2(acc[i], acc[i + 1]), both(-lse)), both(kLog2e));
            const float2 v = mul2(make_float2(hardware_exp2(d.x), hardware_exp2(d.y)), both(g));
            acc[i] = v.x, acc[i + 1] = v.y;
          }
          if (has) {
            const float minus = target >= 0 ? g : 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < 128; ++i)
              if (at == i) acc[i] -= minus;
          }
          // two fp16 numbers each, a pair's first parts in the place of its first number
          uint32_t* const bits = reinterpret_cast<uint32_t*>(acc);
#pragma unroll
          for (int i = 0; i < 128; i += 2) {
            const __half2 hi = __floats2half2_rn(acc[i], acc[i + 1]);
            const float2 f = __half22float2(hi);
            const __half2 lo = __floats2half2_rn(acc[i] - f.x, acc[i + 1] - f.y);
            memcpy(&bits[i], &hi, 4);
            memcpy(&bits[i + 1], &lo, 4);
          }
          // a warp's 32 rows of a block lie together: one copy of 4 KB
          const uint32_t stage = stages + 192 * 1024 + warp * 4096, col_blocks = a.piece_cols / 64;
          const uint64_t plane = uint64_t(a.row_blocks) * col_blocks * kBlockBytes;
          unsigned char* const to = a.s + (uint64_t(w.m0 / 128 + rank) * col_blocks + col0 / 64) * kBlockBytes + quarter * 4096;
#pragma unroll
          for (uint32_t b = 0; b < 2; ++b)
#pragma unroll
            for (uint32_t p = 0; p < 2; ++p) {
              if (p < a.parts) {
                if (lane == 0) bulk_stores_read();
                __syncwarp();
#pragma unroll
                for (uint32_t q = 0; q < 8; ++q)
                  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * 128 + ((q ^ (lane & 7)) << 4)), "r"(bits[b * 64 + q * 8 + p]),
                               "r"(bits[b * 64 + q * 8 + 2 + p]), "r"(bits[b * 64 + q * 8 + 4 + p]), "r"(bits[b * 64 + q * 8 + 6 + p])
                               : "memory");
                writes_to_async_proxy();
                __syncwarp();
                if (lane == 0) bulk_store(to + p * plane + b * kBlockBytes, stage, 4096);
              }
            }
        }
      } else if (row < a.width) {
        // lanes are neighbours in dW's and dh's rows
        const uint32_t last = MODE == kWords ? min(a.piece_cols, a.words - a.first_word) : a.rows;   // of the columns of the tile
        const bool direct = MODE == kWords && a.splits == 1;
        float* p = a.out + (uint64_t(w.split) * (MODE == kWords ? a.piece_cols : a.rows) + (direct ? a.first_word : 0) + col0) * a.width + row;
        const float by2 = direct ? down_of(*a.most_g) : 1.0f, by1 = direct ? by : 1.0f;
        const bool add = MODE == kWords ? direct && a.add : !a.first_piece;
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
          if (q * 32 >= cols) break;
          if (direct) {
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i) acc[q * 32 + i] = acc[q * 32 + i] * by1 * by2;
          }
          if (add) {
            float old[32];
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i) old[i] = col0 + q * 32 + i < last ? p[uint64_t(q * 32 + i) * a.width] : 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i) acc[q * 32 + i] += old[i];
          }
#pragma unroll
          for (uint32_t i = 0; i < 32; ++i)
            if (col0 + q * 32 + i < last) p[uint64_t(q * 32 + i) * a.width] = acc[q * 32 + i];
        }
      }
    }
    if (MODE == kSlope && lane == 0) bulk_stores_done();
    if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);
  }
  __syncwarp();
  tmem_before();
  __syncthreads();
  // the commit behind the last products arrives in both CTAs: neither leaves before its own
  if (warp == 8 && lane == 0 && !bar_wait(smem_at(&s_done), 0)) report(a.status, DGS_ETIMEOUT);
  __syncwarp();
  pair_sync();
  if (warp == 8) {
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

// The bits of the largest magnitude of each column (of rows that are not ignored, where `rows` says which), and of dloss.
constexpr uint32_t kMostRows = 64;   // of a CTA
template <class T, bool VEC>
__device__ __forceinline__ void columns_most(const Head& a, const Source& m, bool targets, uint32_t block, uint32_t* most) {
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, col0 = block % m.spans * kSpan, row0 = block / m.spans * kMostRows;
  __shared__ uint32_t s_most[8][kSpan];
  uint32_t best[8] = {};
#pragma unroll 2
  for (uint32_t r = row0 + warp; r < min(row0 + kMostRows, m.rows); r += 8) {
    if (targets && target_of(a, r, false) < 0) continue;
    Eight<T> e;
    load8<T, VEC>(static_cast<const T*>(m.data) + r * m.stride, col0, lane, m.cols, e);
    float2 v[4];
    floats_of(e, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      best[2 * i] = max(best[2 * i], __float_as_uint(v[i].x) & 0x7fffffffu);
      best[2 * i + 1] = max(best[2 * i + 1], __float_as_uint(v[i].y) & 0x7fffffffu);
    }
  }
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
      if (target_of(a, r, true) >= 0) v = max(v, __float_as_uint(a.dloss[uint64_t(r) * a.dloss_step]) & 0x7fffffffu);
    v = __reduce_max_sync(0xffffffffu, v);
    if (v && threadIdx.x % 32 == 0) atomicMax(most_g, v);
  }
}

__device__ __forceinline__ void halves(const float2 (&v)[4], Eight<__half>& hi, Eight<__half>& lo) {
  float2 rest[4];
  of_floats(v, hi);
  floats_of(hi, rest);
#pragma unroll
  for (int i = 0; i < 4; ++i) rest[i] = make_float2(v[i].x - rest[i].x, v[i].y - rest[i].y);
  of_floats(rest, lo);
}
// A matrix as P fp16 numbers a value under a power of two for each column: [P][rows][stride].  Ignored rows are zero, whatever they hold.
template <class T, bool VEC, uint32_t P>
__device__ __forceinline__ void by_columns(const Head& a, const Source& m, bool targets, uint64_t unit, const uint32_t* most, __half* out, uint32_t stride) {
  const uint32_t lane = threadIdx.x % 32, r = uint32_t(unit / m.spans), col0 = uint32_t(unit - uint64_t(r) * m.spans) * kSpan;
  if (r >= m.rows) return;
  Eight<__half> part[2] = {};
  if (!targets || target_of(a, r, false) >= 0) {
    Eight<T> e;
    load8<T, VEC>(static_cast<const T*>(m.data) + r * m.stride, col0, lane, m.cols, e);
    float2 v[4];
    floats_of(e, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t c = col0 + (VEC ? lane * 8 + i : i * 32 + lane);
      const float up = c < m.cols ? up_of(most[c]) : 1.0f;
      if (i % 2) v[i / 2].y *= up;
      else v[i / 2].x *= up;
    }
    halves(v, part[0], part[1]);
  }
#pragma unroll
  for (uint32_t p = 0; p < P; ++p) store8<__half, VEC>(out + (uint64_t(p) * m.rows + r) * stride, col0, lane, m.cols, part[p]);
}
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_head_columns(const __grid_constant__ Head a, const __grid_constant__ Source h, const __grid_constant__ Source w, uint32_t blocks_h,
                                                      __half* out_h, __half* out_w, uint32_t stride) {
  constexpr uint32_t P = sizeof(T) == 4 ? 2 : 1;
  let_next_kernel_begin();
  wait_for_last_kernel();
  if (blockIdx.x < blocks_h)
    by_columns<T, VEC, P>(a, h, true, uint64_t(blockIdx.x) * 8 + threadIdx.x / 32, a.most_h, out_h, stride);
  else
    by_columns<T, VEC, P>(a, w, false, uint64_t(blockIdx.x - blocks_h) * 8 + threadIdx.x / 32, a.most_w, out_w, stride);
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
    for (uint32_t c = lane; c < m.cols; c += 32) most = max(most, __float_as_uint(row[c]) & 0x7fffffffu);
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
// A row's parts joined in their order: 32 rows a CTA, each eighth part a warp.
__global__ void __launch_bounds__(256) k_head_loss(const __grid_constant__ Head a, float* loss, float* lse) {
  __shared__ float2 s_part[8][32];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, row = blockIdx.x * 32 + lane, parts = a.n_tiles * 2;
  wait_for_last_kernel();
  const auto join = [](float2 x, float2 y) {
    const float most = fmaxf(x.x, y.x), from = most == __uint_as_float(0xff800000u) ? 0.0f : most;
    return make_float2(most, x.y * exp2f((x.x - from) * kLog2e) + y.y * exp2f((y.x - from) * kLog2e));
  };
  float2 v = make_float2(__uint_as_float(0xff800000u), 0.0f);
  if (row < a.rows) {
#pragma unroll 8
    for (uint32_t p = warp; p < parts; p += 8) v = join(v, a.partial[uint64_t(p) * a.rows + row]);
  }
  s_part[warp][lane] = v;
  __syncthreads();
  if (warp || row >= a.rows) return;
  for (uint32_t p = 1; p < 8; ++p) v = join(v, s_part[p][lane]);
  const float rest = logf(v.y);
  const int target = target_of(a, row, true);
  lse[row] = v.x + rest;
  loss[row] = target < 0 ? 0.0f : v.x - a.at_target[row] + rest;   // not lse less the logit: a loss next to 0 keeps its digits where the target is the largest
}

// Partial results of dW's piece added up in their order.
__global__ void __launch_bounds__(256) k_head_words(const __grid_constant__ Head a, const float* parts, float* dw) {
  let_next_kernel_begin();
  wait_for_last_kernel();
  const uint64_t all = uint64_t(min(a.piece_cols, a.words - a.first_word)) * a.width, each = uint64_t(a.piece_cols) * a.width;
  const float by2 = down_of(*a.most_g);
  for (uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += uint64_t(gridDim.x) * 256) {
    float v = 0.0f;
    for (uint32_t s = 0; s < a.splits; ++s) v += parts[s * each + i];
    v = v * down_of(a.most_h[i % a.width]) * by2;
    float* p = dw + uint64_t(a.first_word) * a.width + i;
    *p = a.add ? *p + v : v;
  }
}
// dh from its partial results.
template <class T>
__global__ void __launch_bounds__(256) k_head_hidden(const __grid_constant__ Head a, const float* parts, T* dh, uint64_t stride) {
  wait_for_last_kernel();
  const uint64_t all = uint64_t(a.rows) * a.width;
  const float by2 = down_of(*a.most_g);
  for (uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += uint64_t(gridDim.x) * 256) {
    float v = 0.0f;
    for (uint32_t s = 0; s < a.splits; ++s) v += parts[s * all + i];
    const uint64_t r = i / a.width, c = i - r * a.width;
    dh[r * stride + c] = Elem<T>::put(v * down_of(a.most_w[c]) * by2);
  }
}

// ---- host side --------------------------------------------------------------------------------
uint32_t ceil_div(uint64_t a, uint64_t b) { return uint32_t((a + b - 1) / b); }
uint64_t up_to(uint64_t v, uint64_t by) { return (v + by - 1) / by * by; }

// Whether TMA copies can take the matrix where it is.
bool in_place(const dgs_matrix* m) {
  return m->type != DGS_TYPE_F32 && on_16_bytes(m) && m->stride >= m->cols && m->rows <= kMostElements / 4 / m->stride;
}

struct Products {
  uint32_t splits;
  double us;
};
// How a contraction of `steps` steps over `tiles` tiles is split among 74 pairs of CTAs: whatever ends soonest, with step_us a step, 4 us a tile, and partial results of
// `results` values written and read again.
Products split_steps(uint64_t tiles, uint32_t steps, double step_us, uint64_t results) {
  Products best = {1, 1e300};
  for (uint32_t s = 1; s <= 32 && s <= steps; ++s) {
    const double us = double((tiles * s + kSms / 2 - 1) / (kSms / 2)) * (ceil_div(steps, s) * step_us + 4.0) + (s > 1 ? 3.0 + double(results) * 4e-6 * (s + 1) / 2.5 : 0.0);
    if (us < best.us) best = {s, us};
  }
  best.splits = ceil_div(steps, ceil_div(steps, best.splits));   // none without steps
  return best;
}

constexpr uint64_t kPieceBytes = 256ull << 20;   // of s, where one tile of words does not take more

struct HeadPlan {
  uint32_t parts, stride, piece_tiles, pieces, word_splits, hidden_splits, row_blocks;
  bool copy_h, copy_w;
  uint64_t inner_h, inner_w, scales, most, outer_h, outer_w, s, words, hidden, partial, at_target, bytes;
};

bool head_ok(const dgs_matrix* h, const dgs_matrix* w) { return matrix_ok(h, false) && matrix_ok(w, false) && h->type == w->type && h->cols == w->cols && w->rows; }

int plan_head(const dgs_matrix* h, const dgs_matrix* w, bool grad, HeadPlan* p) {
  *p = {};
  if (!head_ok(h, w)) return DGS_EINVAL;
  const uint64_t n = h->rows, v = w->rows;
  const uint32_t d = h->cols;
  p->parts = h->type == DGS_TYPE_F32 ? 2 : 1;
  p->stride = uint32_t(up_to(d, 8));
  // rows are 31-bit coordinates of TMA copies and may be passed by a tile; strides of a plane are 40 bits
  if (d > (1u << 24) || n > (1u << 30) || v > (1u << 30) || std::max(n, v) * p->stride > kMostElements / 4 ||
      uint64_t(ceil_div(n, 256)) * ceil_div(v, 256) > 0x3fffffffu)
    return DGS_ELIMIT;
  if (n == 0) return DGS_OK;
  p->copy_h = !in_place(h);
  p->copy_w = !in_place(w);
  p->inner_h = p->copy_h ? up_to(p->parts * n * p->stride * 2, 256) : 0;
  p->inner_w = p->copy_w ? up_to(p->parts * v * p->stride * 2, 256) : 0;
  p->scales = p->parts == 2 ? up_to((n + v) * 4, 256) : 0;
  if (!grad) {
    p->partial = up_to(uint64_t(ceil_div(v, 256)) * 2 * n * 8, 256);
    p->at_target = up_to(n * 4, 256);
    p->bytes = p->inner_h + p->inner_w + p->scales + p->partial + p->at_target;
    return DGS_OK;
  }
  // Pieces: as many as give the shortest time for the three products of them all.
  const uint32_t m_tiles = ceil_div(n, 256), d_tiles = ceil_div(d, 256), v_tiles = ceil_div(v, 256), products = p->parts == 2 ? 3 : 1;
  const uint32_t most = uint32_t(std::max<uint64_t>(1, kPieceBytes / (uint64_t(m_tiles) * 256 * 256 * 4))), least = ceil_div(v_tiles, most);
  const double half_us = 0.40;   // 64 rows of a product
  double best = 1e300;
  for (uint32_t pieces = least; pieces < least + 12 && pieces <= v_tiles; ++pieces) {
    const uint32_t t = ceil_div(v_tiles, pieces), count = ceil_div(v_tiles, t);
    const Products words = split_steps(uint64_t(t) * d_tiles, ceil_div(n, 64), half_us * (products + 1) * (p->parts == 2 ? 0.75 : 1), uint64_t(t) * 256 * d);
    const Products hidden = split_steps(uint64_t(m_tiles) * d_tiles, t * 4, half_us * products, n * d);
    const double us = count * (ceil_div(uint64_t(m_tiles) * t, kSms / 2) * (ceil_div(d, 64) * half_us * products + 1.0) + words.us + hidden.us + 6.0);
    if (us < best) best = us, p->pieces = count, p->piece_tiles = t;
  }
  const Products words = split_steps(uint64_t(p->piece_tiles) * d_tiles, ceil_div(n, 64), half_us * (products + 1) * (p->parts == 2 ? 0.75 : 1), uint64_t(p->piece_tiles) * 256 * d);
  const Products hidden = split_steps(uint64_t(m_tiles) * d_tiles, p->piece_tiles * 4, half_us * products, n * d);
  p->word_splits = words.splits;
  p->hidden_splits = hidden.splits;
  p->row_blocks = m_tiles * 2;
  p->most = up_to((2 * uint64_t(d) + 1) * 4, 256);
  p->outer_h = up_to(p->parts * n * p->stride * 2, 256);
  p->outer_w = up_to(p->parts * v * p->stride * 2, 256);
  p->s = 2ull * p->row_blocks * p->piece_tiles * 4 * kBlockBytes;
  p->words = p->word_splits > 1 ? up_to(uint64_t(p->word_splits) * p->piece_tiles * 256 * d * 4, 256) : 0;
  p->hidden = up_to(uint64_t(p->hidden_splits) * n * d * 4, 256);
  p->bytes = p->inner_h + p->inner_w + p->scales + p->most + p->outer_h + p->outer_w + p->s + p->words + p->hidden;
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
         cudaFuncSetAttribute(k_head<MODE, PA, PB>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) == cudaSuccess;
}
int head_ready() {   // once per device
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return DGS_ECUDA;
  std::lock_guard<std::mutex> lock(g_head_mu);
  if (!g_head_ready[dev]) {
    if (!head_setup<kLoss, 1, 1>() || !head_setup<kLoss, 2, 2>() || !head_setup<kSlope, 1, 1>() || !head_setup<kSlope, 2, 2>() || !head_setup<kWords, 1, 2>() ||
        !head_setup<kWords, 2, 2>() || !head_setup<kHidden, 1, 1>() || !head_setup<kHidden, 1, 2>() || !head_setup<kHidden, 2, 2>())
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

template <int MODE, uint32_t PA, uint32_t PB>
int head_launch(const Head& a, const CUtensorMap& x, const CUtensorMap& y, bool early, cudaStream_t st) {
  EarlyLaunch l(dim3(std::min(a.tiles, kSms / 2) * 2), kHeadThreads, kSmem, st);
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
  a.n = 256;
  a.splits = 1;
  a.idesc = kIdescF32 | (h->type == DGS_TYPE_BF16 ? kIdescBf16 : 0);
  a.target = target;
  a.wide_targets = flags & DGS_TARGET_I64 ? 1 : 0;
  a.status = operator_status_word();
  return a;
}

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
  if ((rc = head_ready()) != DGS_OK) return rc;
  Head a = head_of(hidden, weight, target, flags);
  if (!a.status) return DGS_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* const work = static_cast<char*>(workspace);
  CUtensorMap map_h = {}, map_w = {};
  bool launched = false;
  if ((rc = inner_operands(hidden, weight, p, work, &a, &map_h, &map_w, &launched, st)) != DGS_OK) return rc;
  a.n_tiles = ceil_div(a.words, 256);
  a.tiles = a.m_tiles * a.n_tiles;
  a.partial = reinterpret_cast<float2*>(work + p.inner_h + p.inner_w + p.scales);
  a.at_target = reinterpret_cast<float*>(work + p.inner_h + p.inner_w + p.scales + p.partial);
  a.steps = ceil_div(a.width, p.parts == 2 ? Step<2, 2>::kRows : Step<1, 1>::kRows);
  rc = p.parts == 2 ? head_launch<kLoss, 2, 2>(a, map_h, map_w, launched, st) : head_launch<kLoss, 1, 1>(a, map_h, map_w, launched, st);
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
  if ((rc = head_ready()) != DGS_OK) return rc;
  Head a = head_of(hidden, weight, target, flags);
  if (!a.status) return DGS_ECUDA;
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
  at += p.words;
  float* const part_h = reinterpret_cast<float*>(at);
  const uint32_t d = a.width;
  a.most_h = most;
  a.most_w = most + d;
  a.most_g = most + 2 * uint64_t(d);
  a.lse = lse;
  a.dloss = dloss;
  a.dloss_step = dloss_stride;
  a.add = flags & DGS_LOSS_ADD ? 1 : 0;
  a.row_blocks = p.row_blocks;
  a.parts = dw || hidden->type != DGS_TYPE_BF16 ? 2 : 1;
  a.piece_cols = p.piece_tiles * 256;

  if (cudaMemsetAsync(most, 0, p.most, st) != cudaSuccess) return DGS_ECUDA;
  const Source h = source_of(hidden), w = source_of(weight);
  const uint32_t most_h = h.spans * ceil_div(h.rows, kMostRows), most_w = w.spans * ceil_div(w.rows, kMostRows), most_g = std::min(ceil_div(n, 256), kSms);
  const uint32_t blocks_h = ceil_div(uint64_t(h.rows) * h.spans, 8), blocks_w = ceil_div(uint64_t(w.rows) * w.spans, 8);
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
  const bool bf16 = hidden->type == DGS_TYPE_BF16;
  if ((rc = head_map(outer_h, n, d, p.stride, p.parts, false, 64, &map_h)) != DGS_OK) return rc;
  if ((rc = head_map(outer_w, v, d, p.stride, p.parts, false, bf16 ? 128 : 64, &map_w)) != DGS_OK) return rc;

  for (uint32_t piece = 0; piece < p.pieces; ++piece) {
    const uint32_t tile0 = piece * p.piece_tiles, tiles = std::min(p.piece_tiles, ceil_div(v, 256) - tile0);
    Head s = a;
    s.first_word = tile0 * 256;
    s.first_piece = piece == 0;
    s.n_tiles = tiles;
    s.tiles = s.m_tiles * tiles;
    s.steps = ceil_div(d, p.parts == 2 ? 64 : 128);
    rc = p.parts == 2 ? head_launch<kSlope, 2, 2>(s, inner_h, inner_w, true, st) : head_launch<kSlope, 1, 1>(s, inner_h, inner_w, true, st);
    if (rc != DGS_OK) return rc;
    s.idesc = kIdescF32;
    if (dw) {
      Head b = s;
      b.m_tiles = ceil_div(d, 256);
      b.splits = p.word_splits;
      b.tiles = b.m_tiles * b.n_tiles * b.splits;
      b.steps = ceil_div(n, 64);
      b.out = b.splits > 1 ? part_w : dw;
      rc = p.parts == 2 ? head_launch<kWords, 2, 2>(b, map_h, map_h, true, st) : head_launch<kWords, 1, 2>(b, map_h, map_h, true, st);
      if (rc != DGS_OK) return rc;
      if (b.splits > 1) {
        const EarlyLaunch l(dim3(uint32_t(std::min<uint64_t>((uint64_t(tiles) * 256 * d + 1023) / 1024, kSms * 8))), 256, 0, st);
        if (cudaLaunchKernelEx(&l.cfg, k_head_words, b, static_cast<const float*>(part_w), dw) != cudaSuccess) return DGS_ECUDA;
      }
    }
    Head b = s;
    b.m_tiles = ceil_div(d, 256);
    b.n_tiles = ceil_div(n, 256);
    b.splits = p.hidden_splits;
    b.tiles = b.m_tiles * b.n_tiles * b.splits;
    b.steps = ceil_div(std::min<uint64_t>(tiles * 256, v - s.first_word), bf16 ? 128 : 64);
    b.out = part_h;
    rc = bf16 ? head_launch<kHidden, 1, 1>(b, map_w, map_w, true, st)
              : p.parts == 2 ? head_launch<kHidden, 2, 2>(b, map_w, map_w, true, st) : head_launch<kHidden, 1, 2>(b, map_w, map_w, true, st);
    if (rc != DGS_OK) return rc;
  }
  a.splits = p.hidden_splits;
  return with_type(hidden->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    const EarlyLaunch l(dim3(uint32_t(std::min<uint64_t>((n * d + 255) / 256, kSms * 16))), 256, 0, st);
    return cudaLaunchKernelEx(&l.cfg, k_head_hidden<T>, a, static_cast<const float*>(part_h), static_cast<T*>(dhidden->data), dhidden->stride) == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
  });
}
