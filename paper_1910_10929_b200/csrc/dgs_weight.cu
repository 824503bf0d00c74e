// Weight and bias gradients from checkpoints in 8 bits: dgs_checkpoint_weight_grad.
#include "dgs_operators.cuh"

#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cstring>
#include <mutex>

namespace dgs {
namespace {

// ---- tcgen05, mbarriers, TMA: pairs of CTAs -------------------------------------------------------
__device__ __forceinline__ uint32_t smem_at(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
// The same barrier in the first CTA of the pair.
__device__ __forceinline__ uint32_t in_leader(uint32_t bar) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(bar));
  return r;
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Likewise, and what threads of this CTA have written is there for a thread that has waited and then called bar_acquire_cluster.
__device__ __forceinline__ void bar_release_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_acquire_cluster(uint32_t bar, uint32_t parity) {   // of a phase that is complete
  asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n}\n" ::"r"(bar), "r"(parity) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
constexpr uint32_t kPolls = 1u << 20;   // far above any wait that ends
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  for (uint32_t n = 0; n < kPolls; ++n) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    if (done) return true;
  }
  return false;
}
// All lanes of a warp, and whether for all of them the wait ended.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, bar_wait(bar, parity)); }
__device__ __forceinline__ void writes_to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tma_load(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to),
               "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}

__device__ __forceinline__ void tmem_alloc(uint32_t* slot, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(slot)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b),
      "r"(idesc), "r"(uint32_t(add))
      : "memory");
}
// Arrives on the barrier at this address in both CTAs once the products issued so far are done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(uint16_t(3))
               : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t at, float (&v)[32]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
      "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void add_to(float& a, float& b, float x, float y) {   // two sums at a time
  const float2 s = add2(make_float2(a, b), make_float2(x, y));
  a = s.x, b = s.y;
}

// ---- tiles in shared memory ---------------------------------------------------------------------
// Both operands are contracted over their rows, so both lie in memory with the other dimension contiguous, and stay so: a tile of
// 64 or 128 rows is cut into blocks of 64 columns, each row of them 128 bytes with its 16-byte pieces exchanged by the row's
// number (128-byte swizzle).  Descriptor: how far blocks of 64 columns lie apart, and groups of 8 rows (1024 bytes).
constexpr uint32_t kCols = 128;                // columns of either operand that a CTA brings, at most
// P: how many bfloat16 numbers add up to one value of the gradient.  Rows of a step (waits and signals cost 0.45 us a step, the products of
// 64 rows and one part 0.34); stages of shared memory; steps between two sums in registers.
template <uint32_t P> struct Shape {
  static constexpr uint32_t kRows = P == 1 ? 128 : 64, kStages = P == 2 ? 4 : 3, kChunk = P == 2 ? 8 : 4;
  static constexpr uint32_t kColBlock = kRows * 128;   // bytes of 64 columns
  static constexpr uint32_t kTile = kCols / 64 * kColBlock;
  static constexpr uint32_t kStage = kTile * (1 + P), kSmem = 1024 + kStages * kStage;
};
// Eight warps keep the sums, four do the rest and leave them their registers.  (56 for the four and 224 for the sums: 16 experts of 768 x 2048 145 us a call, 140 so.)
constexpr uint32_t kThreads = 384, kRegsLaunch = 168, kRegsSum = 216, kRegsRest = 72;
static_assert(kRegsSum * 256 + kRegsRest * 128 <= kRegsLaunch * kThreads, "setmaxnreg draws on the launch's registers");
template <uint32_t P>
__device__ __forceinline__ uint32_t tile_at(uint32_t row, uint32_t piece) {   // piece: eight columns
  return (piece >> 3) * Shape<P>::kColBlock + row * 128 + (((piece ^ row) & 7) << 4);
}
template <uint32_t P>
__device__ __forceinline__ uint64_t tile_desc(uint32_t at) {
  return uint64_t(at >> 4 & 0x3fff) | uint64_t(Shape<P>::kColBlock >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// f32 += bf16 x bf16, 256 rows in a pair, both operands with the contracted dimension outermost
constexpr uint32_t kIdesc = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (256u >> 4) << 24;
__device__ __forceinline__ uint32_t idesc_cols(uint32_t n) { return (n >> 3) << 17; }

constexpr uint32_t kTmemCols = 512;            // two accumulators of 256 columns

struct WeightArgs {
  Held h;
  const __nv_bfloat16* dy;    // [P][plane rows][stride]: parts of the gradient, rows on 16 bytes
  uint64_t dy_rows, dy_stride, plane_rows;
  uint32_t inputs, outputs, code_tiles, grad_tiles, splits, experts, rows_per;
  uint32_t n;           // columns of the operand that the pair shares out: 64 .. 256
  uint32_t in_out, bias_tiles, step_rows, tiles, scans;
  const uint32_t* offsets;
  const uint32_t* rows;
  uint32_t* order;          // experts by their number of rows, the longest first; then, for each kScanRows rows of dy, whether one is left out
  __nv_bfloat16* decoded;   // [rows][h.width]: the checkpoint's values in dy's order, an expert's from expert_at(...) on
  float* dw;          // or the splits' partial results, [splits][experts][inputs * outputs]
  float* db;          // likewise, [splits * bias_tiles][experts][outputs]; NULL: not wanted
  uint32_t add_w, add_b;
  int* status;
};

// Where an expert's decoded values begin: on a step's boundary, behind those of the expert before however long it is.
__device__ __forceinline__ uint64_t expert_at(uint64_t first, uint32_t expert, uint32_t step) {
  return (first + step - 1) / step * step + uint64_t(expert) * step;
}
inline uint64_t decoded_rows(uint64_t dy_rows, uint32_t experts, uint32_t step) { return (dy_rows + step - 1) / step * step + uint64_t(experts) * step; }
// An expert's rows of dy, whatever the offsets say.
__device__ __forceinline__ void expert_rows(const WeightArgs& a, uint32_t expert, uint64_t* first, uint64_t* last, bool tell) {
  *first = 0;
  *last = a.dy_rows;
  if (a.offsets) {
    const uint64_t x = a.offsets[expert], y = a.offsets[expert + 1];
    *first = x < a.dy_rows ? x : a.dy_rows;
    *last = y < *first ? *first : y < a.dy_rows ? y : a.dy_rows;
    if ((*first != x || *last != y) && tell) report(a.status, DGS_EINVAL);
  }
}

// Whether row j of dy, which is in a list, names no row of the checkpoint: it is left out.
__device__ __forceinline__ bool left_out(const WeightArgs& a, uint64_t j) {
  return a.rows ? a.rows[j] >= a.h.rows * a.rows_per : j >= a.h.rows;
}

// ---- the checkpoint's values as bfloat16 numbers ------------------------------------------------------
// They are that exactly, so nothing is lost.  Decoding inside the products' kernel, by the warps that keep the sums, cost more than it saved:
// every tile of 256 outputs decodes again, and eight warps (all that the sums' registers leave room for) took 1.05 us a step of 128 rows where
// the products take 0.68 (32768 x 2048 x 2048: 257 us, 174 without decoding).
constexpr uint32_t kDecodeRows = 16, kScanRows = 4096;   // of a CTA
template <bool FLOAT8>
__global__ void __launch_bounds__(256) k_weight_decode(const __grid_constant__ WeightArgs a) {
  let_next_kernel_begin();
  const uint32_t ahead = a.scans ? a.scans + 1 : 0;                       // CTAs before those that decode
  const uint64_t at = uint64_t(blockIdx.x - ahead) * kDecodeRows;   // row of the decoded values
  uint64_t first = 0, last = a.dy_rows, begin = 0;
  if (blockIdx.x < a.scans) {   // whether all of dy's rows in lists name one of the checkpoint
    uint64_t from, to, x;
    expert_rows(a, 0, &from, &x, false);
    expert_rows(a, a.experts - 1, &x, &to, false);
    from = max(from, uint64_t(blockIdx.x) * kScanRows), to = min(to, uint64_t(blockIdx.x + 1) * kScanRows);
    bool out = false;
    for (uint64_t j = from + threadIdx.x; j < to; j += 8 * 256)
#pragma unroll
      for (uint32_t k = 0; k < 8; ++k) out |= j + k * 256 < to && left_out(a, j + k * 256);
    out = __syncthreads_or(out);
    if (threadIdx.x == 0) {
      a.order[a.experts + blockIdx.x] = out;
      if (out) report(a.status, DGS_EINVAL);
    }
    return;
  }
  if (blockIdx.x < ahead) {     // who comes before whom
    __shared__ uint32_t s_rows[DGS_ROUTE_MAX_EXPERTS];
    for (uint32_t e = threadIdx.x; e < a.experts; e += 256) {
      expert_rows(a, e, &first, &last, true);
      s_rows[e] = uint32_t(last - first);
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.experts; e += 256) {
      uint32_t rank = 0;
      for (uint32_t o = 0; o < a.experts; ++o) rank += s_rows[o] > s_rows[e] || (s_rows[o] == s_rows[e] && o < e);
      a.order[rank] = e;
    }
    return;
  }
  if (a.offsets) {
    // the last expert that begins at or before this row: as many as do, since each begins behind the one before
    __shared__ uint32_t s_begun;
    if (threadIdx.x == 0) s_begun = 0;
    __syncthreads();
    uint32_t begun = 0;
    for (uint32_t e = threadIdx.x; e < a.experts; e += 256) {
      uint64_t f, l;
      expert_rows(a, e, &f, &l, false);
      begun += expert_at(f, e, a.step_rows) <= at;
    }
    if (begun) atomicAdd(&s_begun, begun);
    __syncthreads();
    if (s_begun == 0) return;
    expert_rows(a, s_begun - 1, &first, &last, false);
    begin = expert_at(first, s_begun - 1, a.step_rows);
  }
  // rows behind the expert's last are zero up to the end of its last step
  const uint64_t row0 = at - begin, rows = last - first;
  if (row0 >= (rows + a.step_rows - 1) / a.step_rows * a.step_rows) return;
  // which row of the checkpoint each of the sixteen is
  constexpr uint32_t kNone = 0xffffffffu;
  __shared__ uint32_t s_src[kDecodeRows];
  if (threadIdx.x < kDecodeRows) {
    uint32_t src = kNone;
    if (row0 + threadIdx.x < rows) {
      src = uint32_t(first + row0) + threadIdx.x;
      if (a.rows) src = a.rows[src] / a.rows_per;
      if (src >= a.h.rows) src = kNone;
    }
    s_src[threadIdx.x] = src;
  }
  __syncthreads();
  const uint32_t units = a.h.width / 8, total = kDecodeRows * units;
  // i / units as the upper half of a product: exact while i * units < 2^32
  const uint32_t magic = units > 1 && units < (1u << 14) ? 0xffffffffu / units + 1 : 0;
  for (uint32_t i0 = threadIdx.x; i0 < total; i0 += 4 * 256) {
    uint2 w[4];
    uint32_t scale[4], row[4], unit[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {   // four units on their way together
      const uint32_t i = min(i0 + k * 256, total - 1);
      row[k] = magic ? __umulhi(i, magic) : i / units;
      unit[k] = i - row[k] * units;
      const uint32_t src = s_src[row[k]];
      w[k] = make_uint2(0, 0);
      scale[k] = 0;
      if (src != kNone) {
        w[k] = __ldg(reinterpret_cast<const uint2*>(a.h.codes + uint64_t(src) * a.h.width + unit[k] * 8));
        scale[k] = __ldg(a.h.scales + uint64_t(src) * a.h.spitch + unit[k] / 4);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (i0 + k * 256 >= total) break;
      float2 v[4];
      decode8<FLOAT8>(w[k], scale_down(scale[k]), v);   // rows that are not there: codes and scale of zero
      Eight<__nv_bfloat16> e;
      of_floats(v, e);
      *reinterpret_cast<uint4*>(a.decoded + (at + row[k]) * a.h.width + unit[k] * 8) = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
    }
  }
}

// ---- gradients as bfloat16 numbers ------------------------------------------------------------------
// The bfloat16 number that a float's upper half is, and what it leaves: exact.  Infinities and NaN go into the first part alone.
__device__ __forceinline__ uint32_t upper(float v, float* rest) {
  uint32_t b = __float_as_uint(v);
  const bool finite = (b & 0x7f800000u) != 0x7f800000u;
  if (!finite && (b & 0x7fffffu)) b |= 0x400000u;
  b &= 0xffff0000u;
  *rest = finite ? v - __uint_as_float(b) : 0.0f;
  return b;
}
// Three of them hold a float's 24 bits, as far as bfloat16's last bit, 2^-133: every float of at least 2^-110.
template <class T> constexpr uint32_t kParts = std::is_same_v<T, float> ? 3 : std::is_same_v<T, __half> ? 2 : 1;

// 16 bytes from the off-th on of two words.
__device__ __forceinline__ uint4 words_from(const uint4& a, const uint4& b, uint32_t off) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (off & 8)
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  if (off & 4)
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  const uint32_t s = (off & 2) * 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], s);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Writes a gradient as kParts<T> planes of bfloat16 numbers whose sum it is exactly, with rows on 16 bytes and zeros up to `stride` and `plane_rows`.  For
// gradients of 16 and 32 bits other than bfloat16, and for bfloat16 ones whose rows begin anywhere: TMA copies start on 16 bytes, and shifting words
// into place on their way to the products took 3.0 us a step of 128 rows where the products take 0.8 (8192 x 768 x 50257: 1560 us).  Eight columns a
// thread; what a row's alignment splits is in the first cache for the neighbour.
template <class T>
__global__ void __launch_bounds__(256) k_weight_parts(const T* dy, uint64_t rows, uint32_t cols, uint64_t from_stride, __nv_bfloat16* out, uint32_t stride,
                                                      uint64_t plane_rows) {
  constexpr uint32_t P = kParts<T>;
  let_next_kernel_begin();
  const uint32_t unit = blockIdx.x * 256 + threadIdx.x, col = unit * 8;
  for (uint64_t row = blockIdx.y; row < plane_rows && col < stride; row += gridDim.y) {
    Eight<T> e;
    const T* p = dy + row * from_stride + col;
    const uint32_t left = row < rows && col < cols ? cols - col : 0;
    if (left >= 8 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
#pragma unroll
      for (uint32_t i = 0; i < sizeof(T) / 2; ++i) {
        const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p) + i);
        e.w[4 * i] = w.x, e.w[4 * i + 1] = w.y, e.w[4 * i + 2] = w.z, e.w[4 * i + 3] = w.w;
      }
    } else {
      // two-byte types: the words that the eight elements lie in, where neither reaches past an end of the matrix
      const uintptr_t at = reinterpret_cast<uintptr_t>(p), word = at & ~uintptr_t(15);
      if (sizeof(T) == 2 && left >= 8 && word >= reinterpret_cast<uintptr_t>(dy) && word + 32 <= reinterpret_cast<uintptr_t>(dy + (rows - 1) * from_stride + cols)) {
        const uint4 w = words_from(__ldg(reinterpret_cast<const uint4*>(word)), __ldg(reinterpret_cast<const uint4*>(word) + 1), uint32_t(at - word));
        e.w[0] = w.x, e.w[1] = w.y, e.w[2] = w.z, e.w[3] = w.w;
      } else {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = uint32_t(i) < left ? p[i] : Elem<T>::put(0.0f);
        memcpy(e.w, t, sizeof(t));
      }
    }
    uint4 w[P];
    if constexpr (P == 1) {
      w[0] = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
    } else {
      float2 v[4];
      floats_of(e, v);
#pragma unroll
      for (uint32_t q = 0; q < P; ++q) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = upper(v[i].x, &v[i].x) >> 16 | upper(v[i].y, &v[i].y);
        w[q] = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
#pragma unroll
    for (uint32_t q = 0; q < P; ++q) *reinterpret_cast<uint4*>(out + (q * plane_rows + row) * stride + col) = w[q];
  }
  wait_for_last_kernel();   // it runs beside the decoding, and whoever waits for this kernel waits for both
}
__device__ __forceinline__ void bias_add(const uint4& w, float (&bias)[8]) {   // eight bfloat16 numbers
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    add_to(bias[2 * i], bias[2 * i + 1], __uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
  }
}

// ---- the kernel -----------------------------------------------------------------------------------
// A pair of CTAs forms tiles of 256 x n (n <= 256), each over a run of an expert's rows, 64 or 128 rows a step.  Each CTA brings 128 columns of one
// operand and n / 2 of the other to its shared memory; the products of the pair read both (tcgen05, cta_group::2), and each CTA's tensor memory takes
// 128 rows of the result.  The dimension of dw that is contiguous in memory goes on those rows (lanes), so that a warp's stores are
// coalesced wherever the layer's slice begins: inputs for [outputs][inputs], outputs for [inputs][outputs]; only the operands' roles change.
//
// Warps: 0 to 7 keep the sums; 8 issues products, 9 TMA copies, 10 passes on that copies have landed, and 10 and 11 sum the bias from them.  The gradients of an
// expert's last rows, where the next expert's would come along with a copy, are brought by warps 0 to 7, with zeros behind them.
// Sums: the tensor cores add to their accumulator with bits cut off, which over 8192 rows leaves an error of 5.5e-6; so every kChunk steps the
// accumulators go to registers of the eight warps and are added up there with rounding (2.1e-7), while the products go on in the other half of
// tensor memory.  Each step's part of db is summed by one of the CTAs that hold the same gradients.
// One pair of CTAs per pair of SMs takes tile after tile, so that the copies and products of the next run while a tile is written out (a CTA per
// tile: 10 us around the steps of each).  Bound by what comes from the second cache: 64 KB a CTA and step of 128 rows, 0.8 us.  (8192 x 768 x 50257: 488 us,
// 0.78 of the measured rate of a product that runs alone, 0.92 of one that runs for seconds.)
struct TileOf {
  uint64_t first, held_first;   // the tile's rows of the gradient, and of the decoded values
  uint32_t i0, o0, ci, go;      // first input and output of the tile, and of what the CTA brings
  uint32_t ct, split, expert;
  uint32_t count, steps, tma_steps;
  bool bias;
};
// The tiles of a pair of CTAs: to and fro over the pairs, so that with the experts in the order of their rows all pairs get about as much
// (16 experts of 55 to 8761 rows: 111 to 126 steps for the longest pair, 166 to 178 in the experts' own order, 101 the mean).
__device__ __forceinline__ uint32_t tile_in_round(uint32_t round, uint32_t pair, uint32_t pairs) {
  return round * pairs + (round & 1 ? pairs - 1 - pair : pair);
}
template <uint32_t R, bool LISTS>
__device__ __forceinline__ TileOf tile_of(const WeightArgs& a, uint32_t tile, uint32_t rank) {
  TileOf t;
  t.ct = tile % a.code_tiles;
  tile /= a.code_tiles;
  const uint32_t gt = tile % a.grad_tiles;
  tile /= a.grad_tiles;
  t.split = tile % a.splits;
  t.expert = tile / a.splits;
  if (LISTS && a.order) t.expert = a.order[t.expert];
  t.i0 = t.ct * (a.in_out ? a.n : 256);
  t.o0 = gt * (a.in_out ? 256 : a.n);
  t.ci = t.i0 + rank * (a.in_out ? a.n / 2 : kCols);
  t.go = t.o0 + rank * (a.in_out ? kCols : a.n / 2);
  uint64_t first, last;
  if constexpr (LISTS) expert_rows(a, t.expert, &first, &last, false);
  else first = 0, last = a.dy_rows;
  t.held_first = LISTS ? expert_at(first, t.expert, R) : 0;
  const uint64_t all = (last - first + R - 1) / R, each = (all + a.splits - 1) / a.splits, from = min(first + t.split * each * R, last);
  last = min(from + each * R, last);
  t.held_first += from - first;
  t.first = from;
  t.count = uint32_t(last - from);
  t.steps = (t.count + (R - 1)) / R;
  // the last step's gradients come by TMA only where nothing but the end of the matrix follows
  t.tma_steps = !LISTS || t.count % R == 0 || last == a.dy_rows ? t.steps : t.steps - 1;
  t.bias = a.db != nullptr && t.ct < a.bias_tiles;
  return t;
}

// LISTS: with them, and the code for rows that are not brought by copies alone (8192 x 768 x 2304 without lists: 49 us a call, 55 with that code there).
template <uint32_t P, bool LISTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
k_weight_grad(const __grid_constant__ WeightArgs a, const __grid_constant__ CUtensorMap held_map, const __grid_constant__ CUtensorMap grad_map) {
  using S = Shape<P>;
  constexpr uint32_t R = S::kRows, ST = S::kStages, CH = S::kChunk, STAGE = S::kStage, TILE = S::kTile, BLOCK = S::kColBlock;
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[ST], s_empty[ST], s_loaded[ST], s_sum_full[2], s_sum_empty[2], s_free[ST], s_tail, s_bias_both, s_bias_done, s_done;
  __shared__ uint32_t s_tmem;
  __shared__ float s_bias[20 * kCols];   // rows 0 to 3: sums of the steps that came by TMA, 4 to 19: of the last step
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32, rank = cta_rank(), pair = blockIdx.x / 2, pairs = gridDim.x / 2, rounds = (a.tiles + pairs - 1) / pairs;
  const uint32_t tiles = (smem_at(raw) + 1023u) & ~1023u;
  const uint32_t code_cols = a.in_out ? a.n / 2 : kCols, grad_cols = a.in_out ? kCols : a.n / 2;

  if (warp == 8) {
    tmem_alloc(&s_tmem, kTmemCols);
    if (lane == 0) {
      for (uint32_t s = 0; s < ST; ++s) {
        bar_init(smem_at(&s_full[s]), 2);     // that copies landed, of both CTAs
        bar_init(smem_at(&s_empty[s]), 3);    // products done; the bias' warps
        bar_init(smem_at(&s_loaded[s]), 1);
        bar_init(smem_at(&s_free[s]), 1);     // the gradients of an expert's last rows may be written
      }
      for (uint32_t i = 0; i < 2; ++i) {
        bar_init(smem_at(&s_sum_full[i]), 1);
        bar_init(smem_at(&s_sum_empty[i]), 16);
      }
      bar_init(smem_at(&s_tail), 8);
      bar_init(smem_at(&s_bias_both), 2);
      bar_init(smem_at(&s_bias_done), 1);
      bar_init(smem_at(&s_done), 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
  }
  tmem_before();
  __syncthreads();
  pair_sync();
  tmem_after();
  const uint32_t tmem = s_tmem;
  wait_for_last_kernel();   // nothing above touches memory outside the SM
  bool skips = false;       // rows of the gradient become zeros on their way; the copies' warp need not know
  if (LISTS && warp != 9) {
    for (uint32_t i = lane; i < a.scans; i += 32) skips |= a.order[a.experts + i] != 0;
    skips = __any_sync(0xffffffffu, skips);
  }
  if (LISTS && a.scans == 0 && blockIdx.x == 0 && warp == 9) {   // dy without rows: nothing was decoded, and nothing looked at the lists
    uint64_t first, last;
    for (uint32_t e = lane; e < a.experts; e += 32) expert_rows(a, e, &first, &last, true);
  }

  // Every role goes through the tiles by itself; it counts steps and chunks over all of them, which is what the barriers' phases go by.
  __syncwarp();
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRest));
    if (warp == 8 && lane == 0 && rank == 0) {
      bool alive = true;
      uint32_t it = 0, chunk = 0;
      for (uint32_t round = 0; round < rounds && alive; ++round) {
        const uint32_t tile = tile_in_round(round, pair, pairs);
        if (tile >= a.tiles) break;   // in the last round only
        const TileOf w = tile_of<R, LISTS>(a, tile, rank);
        const uint32_t written = skips ? 0 : w.tma_steps;
        for (uint32_t s = 0; s < w.steps; ++s, ++it) {
          const uint32_t st = it % ST, code = tiles + st * STAGE, grad = code + TILE, acc = tmem + (chunk & 1) * 256;
          if (s % CH == 0 && chunk >= 2) alive = bar_wait(smem_at(&s_sum_empty[chunk & 1]), (chunk / 2 - 1) & 1);
          alive = alive && bar_wait(smem_at(&s_full[st]), it / ST & 1);
          if (!alive) break;
          if (s >= written) bar_acquire_cluster(smem_at(&s_full[st]), it / ST & 1);
          tmem_after();
          const uint32_t groups = min(R / 16, (w.count - s * R + 15) / 16);   // of sixteen rows: the last step may have fewer
#pragma unroll
          for (uint32_t k = 0; k < R / 16; ++k) {
            if (k >= groups) break;
            const uint64_t cd = tile_desc<P>(code + k * 2048);
#pragma unroll
            for (uint32_t p = 0; p < P; ++p) {
              const uint64_t gd = tile_desc<P>(grad + p * TILE + k * 2048);
              mma(acc, a.in_out ? gd : cd, a.in_out ? cd : gd, kIdesc | idesc_cols(a.n), s % CH || k || p);
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
      const uint32_t code_blocks = (code_cols + 63) / 64, grad_blocks = (grad_cols + 63) / 64;
      bool alive = true;
      uint32_t it = 0;
      for (uint32_t round = 0; round < rounds && alive; ++round) {
        const uint32_t tile = tile_in_round(round, pair, pairs);
        if (tile >= a.tiles) break;   // in the last round only
        const TileOf w = tile_of<R, LISTS>(a, tile, rank);
        for (uint32_t s = 0; s < w.steps; ++s, ++it) {
          const uint32_t st = it % ST, to = tiles + st * STAGE, bar = smem_at(&s_loaded[st]), grads = s < w.tma_steps ? grad_blocks : 0;
          if (it >= ST && !(alive = bar_wait(smem_at(&s_empty[st]), (it / ST - 1) & 1))) break;
          if (s >= w.tma_steps) bar_arrive(smem_at(&s_free[st]));
          bar_expect(bar, (code_blocks + P * grads) * BLOCK);
          for (uint32_t c = 0; c < code_blocks; ++c) tma_load(to + c * BLOCK, &held_map, int(w.ci + c * 64), int(w.held_first + uint64_t(s) * R), bar);
#pragma unroll
          for (uint32_t p = 0; p < P; ++p)
            for (uint32_t c = 0; c < grads; ++c)
              tma_load(to + (1 + p) * TILE + c * BLOCK, &grad_map, int(w.go + c * 64), int(p * a.plane_rows + w.first + uint64_t(s) * R), bar);
        }
      }
      // Nothing is under way to this CTA's memory when it leaves: its copies, and the arrivals that the products' commits send to both CTAs.
      for (uint32_t i = it > ST ? it - ST : 0; i < it; ++i) {
        const bool landed = bar_wait(smem_at(&s_loaded[i % ST]), i / ST & 1);
        alive = alive && landed && bar_wait(smem_at(&s_empty[i % ST]), i / ST & 1);
      }
      if (!alive) report(a.status, DGS_ETIMEOUT);
    }
    if (warp >= 10) {
      // 64 threads: eight columns of every fourth row
      const uint32_t t = tid - 320, br = t / 16, bv = t % 16;
      bool alive = true;
      uint32_t it = 0, tails = 0, met = 0;
      // Warps 10 and 11 wait for each other, and not for ever: one of them may have given up.
      const auto both = [&] {
        __syncwarp();
        if (lane == 0) bar_arrive(smem_at(&s_bias_both));
        return warp_wait(smem_at(&s_bias_both), met++ & 1);
      };
      for (uint32_t round = 0; round < rounds && alive; ++round) {
        const uint32_t tile = tile_in_round(round, pair, pairs);
        if (tile >= a.tiles) break;   // in the last round only
        const TileOf w = tile_of<R, LISTS>(a, tile, rank);
        const uint32_t written = skips ? 0 : w.tma_steps;   // from here on threads write to the stages
        float bias[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) bias[i] = 0.0f;
        for (uint32_t s = 0; s < w.steps; ++s, ++it) {
          const uint32_t st = it % ST;
          if (!(alive = warp_wait(smem_at(&s_loaded[st]), it / ST & 1))) break;
          if (s >= written) {   // rare; what threads wrote is released to the other CTA, whose thread issues the products
            if (s < w.tma_steps) {
#pragma unroll 1
              for (uint32_t r = t; r < R && s * R + r < w.count; r += 64)
                if (left_out(a, w.first + s * R + r))
#pragma unroll 1
                  for (uint32_t i = 0; i < P * 16; ++i)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tiles + st * STAGE + (1 + i / 16) * TILE + tile_at<P>(r, i % 16)), "r"(0) : "memory");
              writes_to_async_proxy();
              if (!(alive = both())) break;
            } else if (warp == 10 && !(alive = warp_wait(smem_at(&s_tail), tails & 1))) {
              break;
            }
            if (warp == 10 && lane == 0) bar_release_cluster(in_leader(smem_at(&s_full[st])));
          } else if (warp == 10 && lane == 0) {   // for copies nothing need be released (8192 x 768 x 50257: 1187 us if it is, 853 so)
            bar_arrive_cluster(in_leader(smem_at(&s_full[st])));
          }
          if (w.bias && s < w.tma_steps && s % a.bias_tiles == w.ct) {
#pragma unroll 4
            for (uint32_t r = br; r < R; r += 4) {
#pragma unroll
              for (uint32_t p = 0; p < P; ++p) {
                uint4 v;
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                             : "r"(tiles + st * STAGE + (1 + p) * TILE + tile_at<P>(r, bv)));
                bias_add(v, bias);
              }
            }
          }
          __syncwarp();
          if (lane == 0) bar_arrive(smem_at(&s_empty[st]));
        }
        if (!alive) break;
        if (w.bias) {
#pragma unroll
          for (int i = 0; i < 8; ++i) s_bias[br * kCols + bv * 8 + i] = bias[i];
          if (!(alive = both())) break;
          const uint32_t rows = w.tma_steps < w.steps && (w.steps - 1) % a.bias_tiles == w.ct ? 20 : 4;
          for (uint32_t c = t; c < grad_cols && w.go + c < a.outputs; c += 64) {
            float v = 0.0f;
            for (uint32_t i = 0; i < rows; ++i) v += s_bias[i * kCols + c];
            float* p = a.db + (uint64_t(w.split * a.bias_tiles + w.ct) * a.experts + w.expert) * a.outputs + w.go + c;
            *p = a.add_b ? *p + v : v;
          }
          if (!(alive = both())) break;
        }
        if (w.tma_steps < w.steps) {
          ++tails;
          if (warp == 10 && lane == 0) bar_arrive(smem_at(&s_bias_done));
        }
      }
      if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSum));
    const uint32_t quarter = warp % 4, group = warp / 4;
    bool alive = true;
    uint32_t it = 0, drained = 0, tails = 0, used = 0;   // tails: tiles with last rows of that kind so far; used: bit s is the phase of s_free[s] to wait for
    for (uint32_t ordinal = 0; ordinal < rounds && alive; ++ordinal) {
      const uint32_t tile = tile_in_round(ordinal, pair, pairs);
      if (tile >= a.tiles) break;
      const TileOf w = tile_of<R, LISTS>(a, tile, rank);
      const uint32_t chunks = (w.steps + CH - 1) / CH;
      float acc[128];
#pragma unroll
      for (int i = 0; i < 128; ++i) acc[i] = 0.0f;
      for (uint32_t c = 0; c < chunks; ++c, ++drained) {
        if (LISTS && c + 1 == chunks && w.tma_steps < w.steps) {
          // an expert's last rows: eight columns of every sixteenth row a thread, zeros behind them.  What is read is on its way before the stage is
          // free; sixteen rows that no product takes are left out.
          const uint32_t last = it + w.steps - 1, at = tiles + last % ST * STAGE + TILE, gr = tid / 16, gv = tid % 16, col = w.go + gv * 8;
          const uint32_t j0 = (w.steps - 1) * R + gr;
          uint32_t out = 0;   // bit u: the thread's u-th row is left out
          if (skips) {
#pragma unroll 1
            for (uint32_t u = 0; u < R / 16 && j0 + 16 * u < w.count; ++u) out |= uint32_t(left_out(a, w.first + j0 + 16 * u)) << u;
          }
          uint4 v[P][R / 16];
#pragma unroll
          for (uint32_t p = 0; p < P; ++p) {
            const __nv_bfloat16* from = a.dy + (p * a.plane_rows + w.first + j0) * a.dy_stride + col;
#pragma unroll
            for (uint32_t u = 0; u < R / 16; ++u, from += 16 * a.dy_stride) {
              v[p][u] = make_uint4(0, 0, 0, 0);
              if (j0 + 16 * u < w.count && col < a.outputs && !(out >> u & 1)) {
                if (col + 8 <= a.outputs) {
                  v[p][u] = __ldg(reinterpret_cast<const uint4*>(from));
                } else {
                  uint32_t e[8];
#pragma unroll
                  for (uint32_t i = 0; i < 8; ++i) e[i] = col + i < a.outputs ? __ldg(reinterpret_cast<const unsigned short*>(from) + i) : 0u;
                  v[p][u] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                }
              }
            }
          }
          // Not s_empty itself: waits by parity only tell neighbouring phases apart, and the sums may be two phases of s_empty ahead of the bias' warps
          // here.  The thread of the copies waits for every phase of s_empty, and a stage has no second tail before this one is read.
          if (!(alive = warp_wait(smem_at(&s_free[last % ST]), used >> last % ST & 1))) break;
          used ^= 1u << last % ST;
          // the table is free: both sides count tiles with such rows alone, so that no phase goes by without this wait
          if (tails && !(alive = warp_wait(smem_at(&s_bias_done), (tails - 1) & 1))) break;
          ++tails;
          float bias[8] = {};
#pragma unroll
          for (uint32_t p = 0; p < P; ++p)
#pragma unroll
            for (uint32_t u = 0; u < R / 16; ++u)
              if ((w.steps - 1) * R + 16 * u < w.count) {
                const uint4 q = v[p][u];
                bias_add(q, bias);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + p * TILE + tile_at<P>(gr + 16 * u, gv)), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
              }
#pragma unroll
          for (int i = 0; i < 8; ++i) s_bias[(4 + gr) * kCols + gv * 8 + i] = bias[i];
          writes_to_async_proxy();
          __syncwarp();
          if (lane == 0) bar_arrive(smem_at(&s_tail));
        }
        const uint32_t buf = drained & 1;
        if (!(alive = warp_wait(smem_at(&s_sum_full[buf]), drained / 2 & 1))) break;
        tmem_after();
#pragma unroll
        for (uint32_t g = 0; g < 4; ++g) {
          if (group * 128 + g * 32 < a.n) {
            float v[32];
            tmem_load32(tmem + (quarter * 32 << 16) + buf * 256 + group * 128 + g * 32, v);
#pragma unroll
            for (int i = 0; i < 32; i += 2) add_to(acc[g * 32 + i], acc[g * 32 + i + 1], v[i], v[i + 1]);
          }
        }
        tmem_before();
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(in_leader(smem_at(&s_sum_empty[buf])));
      }
      it += w.steps;
      // results to memory
      const uint32_t row = rank * 128 + quarter * 32 + lane;
      const uint32_t lane_at = (a.in_out ? w.o0 : w.i0) + row, lane_end = a.in_out ? a.outputs : a.inputs;
      const uint32_t col_at = (a.in_out ? w.i0 : w.o0) + group * 128, col_end = min(a.in_out ? a.inputs : a.outputs, (a.in_out ? w.i0 : w.o0) + a.n);
      if (alive && lane_at < lane_end) {
        float* p = a.dw + (uint64_t(w.split) * a.experts + w.expert) * a.inputs * a.outputs + uint64_t(col_at) * lane_end + lane_at;
#pragma unroll
        for (uint32_t g = 0; g < 4; ++g) {
          if (a.add_w) {
            float old[32];
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i) old[i] = col_at + g * 32 + i < col_end ? p[uint64_t(g * 32 + i) * lane_end] : 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i) acc[g * 32 + i] += old[i];
          }
#pragma unroll
          for (uint32_t i = 0; i < 32; ++i)
            if (col_at + g * 32 + i < col_end) p[uint64_t(g * 32 + i) * lane_end] = acc[g * 32 + i];
        }
      }
    }
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
    tmem_free(tmem, kTmemCols);
  }
}

// Adds up partial results in their order: of dw over the splits, of db over the splits and the CTAs that shared its steps.  Four results a thread
// at a time, so that their parts are on their way together.
__global__ void __launch_bounds__(256) k_weight_sum(float* dw, float* db, const float* pw, const float* pb, uint64_t nw, uint64_t nb, uint32_t parts_w,
                                                    uint32_t parts_b, uint32_t add) {
  wait_for_last_kernel();
  const bool bias = blockIdx.y != 0;
  float* out = bias ? db : dw;
  const float* p = bias ? pb : pw;
  const uint64_t n = bias ? nb : nw, step = uint64_t(gridDim.x) * 256;
  const uint32_t parts = bias ? parts_b : parts_w;
  for (uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += 4 * step) {
    float v[4], old[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = 0.0f, old[k] = add && i + k * step < n ? out[i + k * step] : 0.0f;
    for (uint32_t s = 0; s < parts; ++s)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k * step < n) v[k] += p[s * n + i + k * step];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * step < n) out[i + k * step] = old[k] + v[k];
  }
}

// ---- few rows ---------------------------------------------------------------------------------------
// Where there is little to do, the three kernels that bring operands to the tensor cores cost more than products without them: one launch, a tile of 64 x 64
// results a CTA, 4 x 4 of them a thread, sixteen rows at a time through shared memory, sums in f32 with rounding.  Bound by the trips to memory and the
// barriers of each sixteen rows, 1 us.  The rule goes by all rows and by one expert's results: a call's results are written either way.  Here / with tensor
// cores, us a call alone: 37 x 512 x 1000 15 / 25 in bfloat16, 17 / 29 in f32; 64 x 1024 x 1024 20 / 27; 128 x 1024 x 1024 26 / 27; 256 x 768 x 680 29 / 25,
// 27 / 30 in f32; 512 x 512 x 512 43 / 27, 40 / 32.  With lists: 200 rows, 8 experts of 300 x 300 22 / 31; 64, 32 of 2048 x 1024 101 / 109; 256 slots, 16 of
// 768 x 2048 71 / 62; 16, 128 of 1024 x 1024 132 / 177; 256, 64 of 2048 x 2048 410 / 440.
constexpr uint32_t kSmallRows = 256;
constexpr uint64_t kSmallProducts = 1ull << 27;
constexpr uint32_t kSmallTile = 64, kSmallStep = 16;

template <class T, bool FLOAT8>
__global__ void __launch_bounds__(256) k_weight_small(const __grid_constant__ WeightArgs a, const T* dy) {
  __shared__ __align__(16) float s_held[kSmallStep][kSmallTile + 4], s_grad[kSmallStep][kSmallTile + 4];
  const uint32_t t = threadIdx.x, i0 = blockIdx.x * kSmallTile, o0 = blockIdx.y * kSmallTile, expert = blockIdx.z;
  uint64_t first, last;
  expert_rows(a, expert, &first, &last, t == 0 && blockIdx.x == 0 && blockIdx.y == 0);
  const uint32_t count = uint32_t(last - first), row = t / 16, quad = t % 16 * 4;   // four columns of one of the sixteen rows
  const uint32_t held_col = i0 + quad, grad_col = o0 + quad;
  float acc[4][4], bias = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
  uint32_t code = 0, scale = 0;
  float grad[4];
  auto fetch = [&](uint32_t from) {
    const uint32_t j = from + row;
    code = scale = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) grad[i] = 0.0f;
    if (j >= count) return;
    uint32_t src = uint32_t(first) + j;
    const T* g = dy + (first + j) * a.dy_stride + grad_col;
    if (a.rows) src = a.rows[src] / a.rows_per;
    if (src >= a.h.rows) {   // left out
      report(a.status, DGS_EINVAL);
      return;
    }
    if (held_col < a.h.width) {
      code = *reinterpret_cast<const uint32_t*>(a.h.codes + uint64_t(src) * a.h.width + held_col);
      scale = a.h.scales[uint64_t(src) * a.h.spitch + held_col / 32];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (grad_col + i < a.outputs) grad[i] = Elem<T>::get(g[i]);
  };
  fetch(0);
  for (uint32_t from = 0; from < count; from += kSmallStep) {
    float2 v[4];
    decode8<FLOAT8>(make_uint2(code, 0), scale_down(scale), v);
    *reinterpret_cast<float4*>(&s_held[row][quad]) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    *reinterpret_cast<float4*>(&s_grad[row][quad]) = make_float4(grad[0], grad[1], grad[2], grad[3]);
    __syncthreads();
    fetch(from + kSmallStep);
    const float(*along)[kSmallTile + 4] = a.in_out ? s_grad : s_held;    // the dimension of dw that is contiguous
    const float(*across)[kSmallTile + 4] = a.in_out ? s_held : s_grad;
#pragma unroll
    for (uint32_t k = 0; k < kSmallStep; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(&along[k][quad]), y = *reinterpret_cast<const float4*>(&across[k][row * 4]);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(ys[i], xs[j], acc[i][j]);
    }
    if (a.db && blockIdx.x == 0 && t < kSmallTile)
#pragma unroll
      for (uint32_t k = 0; k < kSmallStep; ++k) bias += s_grad[k][t];
    __syncthreads();
  }
  const uint32_t along_at = (a.in_out ? o0 : i0) + quad, along_end = a.in_out ? a.outputs : a.inputs;
  const uint32_t across_at = (a.in_out ? i0 : o0) + row * 4, across_end = a.in_out ? a.inputs : a.outputs;
  float* dw = a.dw + uint64_t(expert) * a.inputs * a.outputs;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (across_at + i < across_end && along_at + j < along_end) {
        float* p = dw + uint64_t(across_at + i) * along_end + along_at + j;
        *p = a.add_w ? *p + acc[i][j] : acc[i][j];
      }
  if (a.db && blockIdx.x == 0 && t < kSmallTile && o0 + t < a.outputs) {
    float* p = a.db + uint64_t(expert) * a.outputs + o0 + t;
    *p = a.add_b ? *p + bias : bias;
  }
}

// ---- host side --------------------------------------------------------------------------------
struct WeightPlan {
  uint32_t parts, code_tiles, grad_tiles, n, splits, bias_tiles, experts, step_rows, stride;
  bool small, direct;                // one kernel without tensor cores; the gradient is read as it is
  uint64_t nw, nb, plane_rows, decoded, planes, order, bytes;
};

bool lists_ok(const dgs_row_lists* l) {
  return !l || (l->offsets && l->experts && l->experts <= DGS_ROUTE_MAX_EXPERTS && l->rows_per && aligned(l->offsets, 4) && aligned(l->rows, 4));
}

uint32_t ceil_div(uint64_t a, uint64_t b) { return uint32_t((a + b - 1) / b); }
uint32_t scans_of(uint64_t dy_rows) { return ceil_div(dy_rows, kScanRows); }

int plan_weight(const dgs_checkpoint* c, const dgs_matrix* dy, const dgs_row_lists* lists, uint32_t flags, WeightPlan* p) {
  if (!checkpoint_ok(c) || !matrix_ok(dy, false) || !lists_ok(lists) || (lists ? c->rows == 0 && dy->rows : dy->rows != c->rows))
    return DGS_EINVAL;
  p->parts = dy->type == DGS_TYPE_BF16 ? 1 : dy->type == DGS_TYPE_FP16 ? 2 : 3;
  p->step_rows = p->parts == 1 ? Shape<1>::kRows : Shape<3>::kRows;
  static_assert(Shape<2>::kRows == Shape<3>::kRows, "");
  const bool in_out = flags & DGS_WEIGHT_IN_OUT;
  p->experts = lists ? lists->experts : 1;
  // rows and columns are 31-bit coordinates of TMA copies, with all parts' rows in one
  if (uint64_t(c->cols) * dy->cols > kMostElements / p->experts || dy->rows >= (1u << 31) / p->parts - 1026 * 128 || dy->cols > (1u << 30)) return DGS_ELIMIT;
  p->nw = uint64_t(c->cols) * dy->cols * p->experts;
  p->nb = uint64_t(dy->cols) * p->experts;
  // both sides are measured at k_weight_small
  p->small = dy->rows <= kSmallRows && uint64_t(c->cols) * dy->cols <= kSmallProducts / std::max<uint64_t>(dy->rows, 1) &&
             ceil_div(dy->cols, kSmallTile) <= 65535;
  if (p->small) {
    p->splits = p->bias_tiles = 1;
    p->bytes = 0;
    return DGS_OK;
  }
  // The tile's width and the split of a tile's rows among pairs: whatever ends soonest.  74 pairs run at a time; 64 rows take 0.3 us and 0.1 by the
  // width, a tile about 4 us besides, and partial results cost their way through the second cache and another launch.  (8192 x 768 x 2304, us
  // a call: 54 tiles of 128 columns 64, 27 of 256 65, 27 of 256 in two runs of rows each 48.2, 36 of 192 in two runs, which this takes, 47.5.)  Steps are those of
  // the mean expert: where one has most of the rows, few pairs do its tiles (16384 rows, 8 experts of 768 x 2048: 73 us if even, 104 if one has half, 135 if it has all).
  const uint32_t steps = std::max(1u, ceil_div(dy->rows / p->experts, 64));
  double best = 1e300;
  for (uint32_t n = 256; n >= 64; n -= 64) {
    const uint64_t tiles = uint64_t(ceil_div(in_out ? c->cols : dy->cols, n)) * ceil_div(in_out ? dy->cols : c->cols, 256) * p->experts;
    const double step_us = p->parts * (0.30 + 0.10 * n / 256);
    for (uint32_t s = 1; s <= 32 && s <= steps; ++s) {
      const double us = double(ceil_div(tiles * s, kSms / 2)) * (ceil_div(steps, s) * step_us + 4.0) + (s > 1 ? 3.0 + double(p->nw) * 4e-6 * (s + 1) / 2.5 : 0.0);
      if (us < best) best = us, p->splits = s, p->n = n;
    }
  }
  p->code_tiles = ceil_div(c->cols, in_out ? p->n : 256);
  p->grad_tiles = ceil_div(dy->cols, in_out ? 256 : p->n);
  if (uint64_t(p->code_tiles) * p->grad_tiles * p->experts * p->splits > 0x3fffffffu) return DGS_ELIMIT;
  // few steps: the bias costs less in one CTA than another launch does
  p->bias_tiles = p->splits > 1 || steps > 8 ? p->code_tiles : 1;
  const uint32_t parts_b = p->splits * p->bias_tiles;
  p->direct = p->parts == 1 && aligned(dy->data, 16) && dy->stride % 8 == 0 && dy->stride >= dy->cols;
  p->stride = (dy->cols + 7) / 8 * 8;
  p->plane_rows = p->direct ? dy->rows : (dy->rows + p->step_rows - 1) / p->step_rows * p->step_rows + p->step_rows;   // a step may begin on the last row
  p->planes = p->direct ? 0 : p->parts * p->plane_rows * p->stride * 2;
  p->decoded = dy->rows ? decoded_rows(dy->rows, lists ? p->experts : 0, p->step_rows) * held_width(c->cols) * 2 : 0;
  p->order = lists && dy->rows ? ((p->experts + uint64_t(scans_of(dy->rows))) * 4 + 15) / 16 * 16 : 0;
  p->bytes = p->decoded + p->planes + p->order + (p->splits > 1 ? p->nw * p->splits * 4 : 0) + (parts_b > 1 ? p->nb * parts_b * 4 : 0);
  return DGS_OK;
}

constexpr int kMaxDevices = 64;
std::mutex g_weight_mu;
bool g_weight_ready[kMaxDevices];
PFN_cuTensorMapEncodeTiled_v12000 g_encode;   // written once, under the mutex
template <uint32_t P, bool LISTS>
bool weight_setup() {
  cudaFuncAttributes f;
  // the split of the registers counts on what the launch brings
  return cudaFuncGetAttributes(&f, k_weight_grad<P, LISTS>) == cudaSuccess && uint32_t(f.numRegs) >= kRegsLaunch &&
         cudaFuncSetAttribute(k_weight_grad<P, LISTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<P>::kSmem) == cudaSuccess;
}
int weight_ready() {   // once per device
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return DGS_ECUDA;
  std::lock_guard<std::mutex> lock(g_weight_mu);
  if (!g_weight_ready[dev]) {
    if (!weight_setup<1, false>() || !weight_setup<2, false>() || !weight_setup<3, false>() || !weight_setup<1, true>() || !weight_setup<2, true>() ||
        !weight_setup<3, true>())
      return DGS_ECUDA;
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess || !fn) return DGS_ECUDA;
    g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    g_weight_ready[dev] = true;
  }
  return DGS_OK;
}

int make_map(const void* data, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t box_rows, CUtensorMap* map) {
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {stride * 2};
  const cuuint32_t box[2] = {64, box_rows}, each[2] = {1, 1};
  return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(data), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? DGS_OK
             : DGS_ECUDA;
}

template <uint32_t P>
int launch(const WeightArgs& a, const CUtensorMap& held, const CUtensorMap& grad, cudaStream_t st) {
  const EarlyLaunch l(dim3(std::min(a.tiles, kSms / 2) * 2), kThreads, Shape<P>::kSmem, st);
  return cudaLaunchKernelEx(&l.cfg, a.offsets ? k_weight_grad<P, true> : k_weight_grad<P, false>, a, held, grad) == cudaSuccess ? DGS_OK : DGS_ECUDA;
}

}  // namespace
}  // namespace dgs

using namespace dgs;

extern "C" int dgs_checkpoint_weight_grad_bytes(const dgs_checkpoint* ckpt, const dgs_matrix* dy, const dgs_row_lists* lists, uint32_t flags,
                                                uint64_t* out_bytes) {
  WeightPlan p = {};
  if (!out_bytes || (flags & ~(DGS_WEIGHT_IN_OUT | DGS_WEIGHT_ADD))) return DGS_EINVAL;
  const int rc = plan_weight(ckpt, dy, lists, flags, &p);
  if (rc == DGS_OK) *out_bytes = p.bytes;
  return rc;
}

extern "C" int dgs_checkpoint_weight_grad(const dgs_checkpoint* ckpt, const dgs_matrix* dy, const dgs_row_lists* lists, float* dw, float* db,
                                          uint32_t flags, void* workspace, uint64_t workspace_bytes, void* stream) {
  WeightPlan p = {};
  if (flags & ~(DGS_WEIGHT_IN_OUT | DGS_WEIGHT_ADD)) return DGS_EINVAL;
  int rc = plan_weight(ckpt, dy, lists, flags, &p);
  if (rc != DGS_OK) return rc;
  if (!dw || !aligned(dw, 4) || !aligned(db, 4)) return DGS_EINVAL;
  if (p.bytes && (!workspace || !aligned(workspace, 16))) return DGS_EINVAL;
  if (workspace_bytes < p.bytes) return DGS_ENOMEM;
  const struct { const void* p; uint64_t n; bool out; } part[] = {
      {ckpt->data, held_bytes(ckpt->rows, ckpt->cols), false}, {dy->data, span_bytes(dy), false},
      {lists ? lists->offsets : nullptr, lists ? (lists->experts + 1) * 4ull : 0, false}, {lists ? lists->rows : nullptr, lists && lists->rows ? dy->rows * 4 : 0, false},
      {dw, p.nw * 4, true}, {db, db ? p.nb * 4 : 0, true}, {workspace, p.bytes, true}};
  for (const auto& x : part)
    for (const auto& y : part)
      if (&x != &y && x.out && overlap(x.p, x.n, y.p, y.n)) return DGS_EINVAL;
  if (!p.small && (rc = weight_ready()) != DGS_OK) return rc;
  const uint32_t parts_b = p.splits * p.bias_tiles;
  char* const work = static_cast<char*>(workspace);
  WeightArgs a = {};
  a.h = held_of(ckpt);
  a.dy = static_cast<const __nv_bfloat16*>(p.direct ? dy->data : work + p.decoded);
  a.dy_rows = dy->rows;
  a.dy_stride = p.direct ? dy->stride : p.stride;
  a.plane_rows = p.plane_rows;
  a.inputs = ckpt->cols;
  a.outputs = dy->cols;
  a.code_tiles = p.code_tiles;
  a.grad_tiles = p.grad_tiles;
  a.splits = p.splits;
  a.experts = p.experts;
  a.tiles = p.code_tiles * p.grad_tiles * p.splits * p.experts;
  a.rows_per = lists ? lists->rows_per : 1;
  a.n = p.n;
  a.in_out = flags & DGS_WEIGHT_IN_OUT ? 1 : 0;
  a.bias_tiles = p.bias_tiles;
  a.step_rows = p.step_rows;
  a.scans = p.order ? scans_of(dy->rows) : 0;
  a.offsets = lists ? lists->offsets : nullptr;
  a.rows = lists ? lists->rows : nullptr;
  a.decoded = reinterpret_cast<__nv_bfloat16*>(work);
  a.order = p.order ? reinterpret_cast<uint32_t*>(work + p.decoded + p.planes) : nullptr;
  float* const part_w = reinterpret_cast<float*>(work + p.decoded + p.planes + p.order);
  float* const part_b = part_w + (p.splits > 1 ? p.nw * p.splits : 0);
  a.dw = p.splits > 1 ? part_w : dw;
  a.db = !db ? nullptr : parts_b > 1 ? part_b : db;
  const uint32_t add = flags & DGS_WEIGHT_ADD ? 1 : 0;
  a.add_w = p.splits == 1 ? add : 0;
  a.add_b = parts_b == 1 ? add : 0;
  a.status = operator_status_word();
  if (!a.status) return DGS_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (p.small) {
    a.dy_stride = dy->stride;
    return with_type(dy->type, [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      const dim3 grid(ceil_div(a.inputs, kSmallTile), ceil_div(a.outputs, kSmallTile), a.experts);
      if (ckpt->format == DGS_FORMAT_E4M3)
        k_weight_small<T, true><<<grid, 256, 0, st>>>(a, static_cast<const T*>(dy->data));
      else
        k_weight_small<T, false><<<grid, 256, 0, st>>>(a, static_cast<const T*>(dy->data));
      return cudaGetLastError() == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
    });
  }
  CUtensorMap held = {}, grad = {};
  if (dy->rows) {
    const uint64_t rows = p.decoded / (2 * uint64_t(a.h.width));
    rc = make_map(a.decoded, rows, a.h.width, a.h.width, p.step_rows, &held);
    if (rc == DGS_OK) rc = make_map(a.dy, p.parts * p.plane_rows, dy->cols, a.dy_stride, p.step_rows, &grad);
    if (rc != DGS_OK) return rc;
    const uint32_t ctas = ceil_div(rows, kDecodeRows) + (a.scans ? a.scans + 1 : 0);
    if (ckpt->format == DGS_FORMAT_E4M3)
      k_weight_decode<true><<<ctas, 256, 0, st>>>(a);
    else
      k_weight_decode<false><<<ctas, 256, 0, st>>>(a);
    if (cudaGetLastError() != cudaSuccess) return DGS_ECUDA;
    if (!p.direct) {
      const uint32_t across = ceil_div(p.stride, 2048);
      const dim3 grid(across, uint32_t(std::min<uint64_t>(p.plane_rows, std::max(1u, kSms * 16 / across))));
      rc = with_type(dy->type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const EarlyLaunch l(grid, 256, 0, st);
        return cudaLaunchKernelEx(&l.cfg, k_weight_parts<T>, static_cast<const T*>(dy->data), dy->rows, dy->cols, dy->stride, const_cast<__nv_bfloat16*>(a.dy), p.stride,
                                  p.plane_rows) == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
      });
      if (rc != DGS_OK) return rc;
    }
  }
  rc = p.parts == 1 ? launch<1>(a, held, grad, st) : p.parts == 2 ? launch<2>(a, held, grad, st) : launch<3>(a, held, grad, st);
  const uint64_t nw = p.splits > 1 ? p.nw : 0, nb = db && parts_b > 1 ? p.nb : 0;
  if (rc != DGS_OK || nw + nb == 0) return rc;
  const EarlyLaunch l(dim3(uint32_t(std::min<uint64_t>((std::max(nw, nb) + 1023) / 1024, kSms * 8)), nb ? 2 : 1), 256, 0, st);
  return cudaLaunchKernelEx(&l.cfg, k_weight_sum, dw, db, static_cast<const float*>(part_w), static_cast<const float*>(part_b), nw, nb, p.splits, parts_b, add) == cudaSuccess
             ? DGS_OK
             : DGS_ECUDA;
}
