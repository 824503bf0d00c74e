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
// A gradient's type: how many bfloat16 numbers add up to one of its values; rows of a step (waits and signals cost 0.45 us a step, the
// products of 64 rows and one part 0.34); stages of shared memory; steps between two sums in registers; rows that a group of warps takes through
// its registers at a time.
template <class T> struct Grad;
template <> struct Grad<__nv_bfloat16> { static constexpr uint32_t kParts = 1, kRows = 128, kStages = 3, kChunk = 4, kBatch = 64; };
template <> struct Grad<__half> { static constexpr uint32_t kParts = 2, kRows = 64, kStages = 4, kChunk = 8, kBatch = 64; };
template <> struct Grad<float> { static constexpr uint32_t kParts = 3, kRows = 64, kStages = 3, kChunk = 4, kBatch = 32; };
template <class T> struct Shape {
  static constexpr uint32_t kColBlock = Grad<T>::kRows * 128;   // bytes of 64 columns
  static constexpr uint32_t kTile = kCols / 64 * kColBlock;
  static constexpr uint32_t kStage = kTile * (1 + Grad<T>::kParts), kSmem = 1024 + Grad<T>::kStages * kStage;
};
// Two groups of four warps keep the sums (and bring gradients), four warps do the rest and leave them their registers.
constexpr uint32_t kThreads = 384, kRegsLaunch = 168, kRegsSum = 232, kRegsRest = 40;
static_assert(kRegsSum * 256 + kRegsRest * 128 <= kRegsLaunch * kThreads, "setmaxnreg draws on the launch's registers");
template <class T>
__device__ __forceinline__ uint32_t tile_at(uint32_t row, uint32_t piece) {   // piece: eight columns
  return (piece >> 3) * Shape<T>::kColBlock + row * 128 + (((piece ^ row) & 7) << 4);
}
template <class T>
__device__ __forceinline__ uint64_t tile_desc(uint32_t at) {
  return uint64_t(at >> 4 & 0x3fff) | uint64_t(Shape<T>::kColBlock >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// f32 += bf16 x bf16, 256 rows in a pair, both operands with the contracted dimension outermost
constexpr uint32_t kIdesc = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (256u >> 4) << 24;
__device__ __forceinline__ uint32_t idesc_cols(uint32_t n) { return (n >> 3) << 17; }

constexpr uint32_t kTmemCols = 512;            // two accumulators of 256 columns

struct WeightArgs {
  Held h;
  const void* dy;
  uint64_t dy_rows, dy_stride;
  uint32_t inputs, outputs, code_tiles, grad_tiles, splits, experts, rows_per;
  uint32_t n;           // columns of the operand that the pair shares out: 64 .. 256
  uint32_t in_out, bias_tiles, step_rows;
  const uint32_t* offsets;
  const uint32_t* rows;
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

// ---- the checkpoint's values as bfloat16 numbers ------------------------------------------------------
// They are that exactly, so nothing is lost.  Decoding inside the products' kernel, by the warps that keep the sums, cost more than it saved:
// every tile of 256 outputs decodes again, and eight warps (all that the sums' registers leave room for) took 1.05 us a step of 128 rows where
// the products take 0.68 (32768 x 2048 x 2048: 257 us, 174 without decoding).
constexpr uint32_t kDecodeRows = 16;   // of a CTA
template <bool FLOAT8>
__global__ void __launch_bounds__(256) k_weight_decode(const __grid_constant__ WeightArgs a) {
  const uint64_t at = uint64_t(blockIdx.x) * kDecodeRows;   // row of the decoded values
  uint64_t first = 0, last = a.dy_rows, begin = 0;
  if (a.offsets) {
    // the last expert that begins at or before this row: as many as do, since each begins behind the one before
    __shared__ uint32_t s_begun;
    if (threadIdx.x == 0) s_begun = 0;
    __syncthreads();
    uint32_t begun = 0;
    for (uint32_t e = threadIdx.x; e < a.experts; e += 256) {
      uint64_t f, l;
      expert_rows(a, e, &f, &l, blockIdx.x == 0);
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
  const uint32_t units = a.h.width / 8;
#pragma unroll 4
  for (uint32_t i = threadIdx.x; i < kDecodeRows * units; i += 256) {
    const uint32_t r = i / units, unit = i - r * units;
    uint4 out = make_uint4(0, 0, 0, 0);
    if (row0 + r < rows) {
      uint64_t src = first + row0 + r;
      if (a.offsets) {
        if (a.rows) {
          const uint32_t v = a.rows[src];
          src = a.rows_per == 1 ? v : v / a.rows_per;
        }
        if (src >= a.h.rows) {
          report(a.status, DGS_EINVAL);
          src = ~0ull;
        }
      }
      if (src != ~0ull) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(a.h.codes + src * a.h.width + unit * 8));
        const float down = scale_down(__ldg(a.h.scales + src * a.h.spitch + unit / 4));
        float2 v[4];
        decode8<FLOAT8>(w, down, v);
        Eight<__nv_bfloat16> e;
        of_floats(v, e);
        out = make_uint4(e.w[0], e.w[1], e.w[2], e.w[3]);
      }
    }
    *reinterpret_cast<uint4*>(a.decoded + (at + r) * a.h.width + unit * 8) = out;
  }
}

// ---- eight gradients ------------------------------------------------------------------------------
// Rows may begin on any element.  Two-byte types read the aligned 16 bytes that the first of eight elements lies in and put them together with the
// 16 behind them; what lies at a row's end, or so near an end of the matrix that a whole word would reach past it, is read element by
// element.
__device__ __forceinline__ bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
template <class T> struct Word {
  uint4 a;
};
template <> struct Word<float> {
  uint4 a, b;
};
template <class T>
__device__ __forceinline__ uint4 grads_single(const T* p, uint32_t left) {   // two-byte types
  uint32_t v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = uint32_t(i) < left ? __ldg(reinterpret_cast<const unsigned short*>(p) + i) : 0u;
  return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}
// Whether eight elements at p can be had from whole words.
template <class T>
__device__ __forceinline__ bool grads_whole(const T* p, uint32_t left, const T* lo, const T* hi) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p), word = at & ~uintptr_t(15);
  return left >= 8 && (word == at || (word >= reinterpret_cast<uintptr_t>(lo) && word + 32 <= reinterpret_cast<uintptr_t>(hi)));
}
template <class T>
__device__ __forceinline__ void grads_load(Word<T>& r, const T* p, uint32_t left, const T* lo, const T* hi) {
  r.a = make_uint4(0, 0, 0, 0);
  if constexpr (sizeof(T) == 4) {
    r.b = make_uint4(0, 0, 0, 0);
    if (left >= 8 && aligned16(p)) {
      r.a = __ldg(reinterpret_cast<const uint4*>(p));
      r.b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
    } else if (left) {
      uint32_t v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = uint32_t(i) < left ? __ldg(reinterpret_cast<const uint32_t*>(p) + i) : 0u;
      r.a = make_uint4(v[0], v[1], v[2], v[3]);
      r.b = make_uint4(v[4], v[5], v[6], v[7]);
    }
  } else {
    if (grads_whole(p, left, lo, hi)) r.a = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(15)));
  }
}
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
// The next lane's word; the last lanes of a row's sixteen have theirs in another.
__device__ __forceinline__ uint32_t next_word(uint32_t own, uint32_t edge, uint32_t from_lane) {
  const uint32_t n = __shfl_down_sync(0xffffffffu, own, 1), e = __shfl_sync(0xffffffffu, edge, from_lane);
  return (threadIdx.x & 15u) == 15u ? e : n;
}
// Two-byte types: the eight elements.
template <class T>
__device__ __forceinline__ uint4 grads_words(const Word<T>& r, const T* p, uint32_t left, const T* lo, const T* hi) {
  if (left == 0) return make_uint4(0, 0, 0, 0);
  if (!grads_whole(p, left, lo, hi)) return grads_single(p, left);
  const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p)) & 15u;
  if (off == 0) return r.a;
  return words_from(r.a, __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(15)) + 1), off);
}
__device__ __forceinline__ void bias_add(const uint4& w, float (&bias)[8]) {   // eight bfloat16 numbers
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    add_to(bias[2 * i], bias[2 * i + 1], __uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
  }
}
// The bfloat16 number that a float's upper half is, and what it leaves: exact.  Infinities and NaN go into the first part alone.
__device__ __forceinline__ uint32_t upper(float v, float* rest) {
  uint32_t b = __float_as_uint(v);
  const bool finite = (b & 0x7f800000u) != 0x7f800000u;
  if (!finite && (b & 0x7fffffu)) b |= 0x400000u;
  b &= 0xffff0000u;
  *rest = finite ? v - __uint_as_float(b) : 0.0f;
  return b;
}
// Eight values in their parts to shared memory.
template <class T>
__device__ __forceinline__ void grads_put(float (&v)[8], uint32_t at, bool mine, float (&bias)[8]) {
  constexpr uint32_t P = Grad<T>::kParts;
  if (mine)
#pragma unroll
    for (int i = 0; i < 8; ++i) bias[i] += v[i];
#pragma unroll
  for (uint32_t p = 0; p < P; ++p) {
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = upper(v[2 * i], &v[2 * i]), y = upper(v[2 * i + 1], &v[2 * i + 1]);
      out[i] = x >> 16 | y;
    }
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + p * Shape<T>::kTile), "r"(out[0]), "r"(out[1]), "r"(out[2]), "r"(out[3]) : "memory");
  }
}
template <class T>
__device__ __forceinline__ void grads_split(const uint4& q, uint32_t at, bool mine, float (&bias)[8]) {   // two-byte types
  if constexpr (Grad<T>::kParts == 1) {
    if (mine) bias_add(q, bias);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
  } else {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __half2 h;
      memcpy(&h, &w[i], 4);
      const float2 f = __half22float2(h);
      v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
    grads_put<T>(v, at, mine, bias);
  }
}
template <class T>
__device__ __forceinline__ void grads_store(const Word<T>& r, const T* from, uint32_t left, const T* lo, const T* hi, uint32_t at, bool mine, float (&bias)[8]) {
  if constexpr (sizeof(T) == 4) {
    float v[8] = {__uint_as_float(r.a.x), __uint_as_float(r.a.y), __uint_as_float(r.a.z), __uint_as_float(r.a.w),
                  __uint_as_float(r.b.x), __uint_as_float(r.b.y), __uint_as_float(r.b.z), __uint_as_float(r.b.w)};
    grads_put<T>(v, at, mine, bias);
  } else {
    grads_split<T>(grads_words(r, from, left, lo, hi), at, mine, bias);
  }
}

// ---- the kernel -----------------------------------------------------------------------------------
// A pair of CTAs forms a tile of 256 x n (n <= 256) over a run of an expert's rows, 64 rows a step.  Each CTA brings 128 columns of one operand and
// n / 2 of the other to its shared memory; the products of the pair read both (tcgen05, cta_group::2), and each CTA's tensor memory takes
// 128 rows of the result.  The dimension of dw that is contiguous in memory goes on those rows (lanes), so that a warp's stores are
// coalesced wherever the layer's slice begins: inputs for [outputs][inputs], outputs for [inputs][outputs]; only the operands' roles change.
//
// Warps: 0 to 7 keep the sums; 8 issues products, 9 TMA copies, 10 passes on that copies have landed, and 10 and 11 sum the bias from them.
// Gradients that a TMA copy cannot bring - those of several parts, on odd addresses, and the last rows of an expert, where the next expert's
// would come along - come by warps 0 to 7 (TMA = false: all of them, in two groups that take turns, since a step's waits and signals cost a
// warp several hundred cycles whatever it does in between).
// Sums: the tensor cores add to their accumulator with bits cut off, which over 8192 rows leaves an error of 5.5e-6; so every kChunk steps the
// accumulators go to registers of the eight warps and are added up there with rounding (2.1e-7), while the products go on in the other half of
// tensor memory.  Each step's part of db is summed by one of the CTAs that hold the same gradients.
template <class T, bool TMA>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
k_weight_grad(const __grid_constant__ WeightArgs a, const __grid_constant__ CUtensorMap held_map, const __grid_constant__ CUtensorMap grad_map) {
  using G = Grad<T>;
  constexpr uint32_t P = G::kParts, R = G::kRows, ST = G::kStages, CH = G::kChunk, STAGE = Shape<T>::kStage, kTile = Shape<T>::kTile, kColBlock = Shape<T>::kColBlock;
  constexpr uint32_t SUMS = TMA ? 12 : 16;   // rows of the table that db's parts are put in
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[ST], s_empty[ST], s_loaded[ST], s_sum_full[2], s_sum_empty[2], s_tail, s_done;
  __shared__ uint32_t s_tmem;
  __shared__ float s_bias[SUMS * kCols];
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32, rank = cta_rank();
  const uint32_t tiles = (smem_at(raw) + 1023u) & ~1023u;

  uint32_t b = blockIdx.x / 2;
  const uint32_t ct = b % a.code_tiles;
  b /= a.code_tiles;
  const uint32_t gt = b % a.grad_tiles;
  b /= a.grad_tiles;
  const uint32_t split = b % a.splits, expert = b / a.splits;
  // what the pair's tile covers, and what this CTA brings of it
  const uint32_t i0 = ct * (a.in_out ? a.n : 256), o0 = gt * (a.in_out ? 256 : a.n);
  const uint32_t code_cols = a.in_out ? a.n / 2 : kCols, grad_cols = a.in_out ? kCols : a.n / 2;
  const uint32_t ci = i0 + rank * code_cols, go = o0 + rank * grad_cols;

  uint64_t first, last;
  expert_rows(a, expert, &first, &last, false);
  uint64_t held_first = a.offsets ? expert_at(first, expert, R) : 0;
  {
    const uint64_t steps = (last - first + R - 1) / R, each = (steps + a.splits - 1) / a.splits;
    const uint64_t from = min(first + split * each * R, last);
    last = min(from + each * R, last);
    held_first += from - first;
    first = from;
  }
  const uint32_t count = uint32_t(last - first), steps = (count + (R - 1)) / R, chunks = (steps + CH - 1) / CH;
  // the last step's gradients come by TMA only where nothing but the end of the matrix follows
  const uint32_t tma_steps = !TMA ? 0 : count % R == 0 || last == a.dy_rows ? steps : steps - 1;
  const bool bias_here = a.db != nullptr && ct < a.bias_tiles;

  if (warp == 8) {
    tmem_alloc(&s_tmem, kTmemCols);
    if (lane == 0) {
      for (uint32_t s = 0; s < ST; ++s) {
        bar_init(smem_at(&s_full[s]), TMA ? 2 : 2 + 8);   // that copies landed, of both CTAs; their warps that brought gradients
        bar_init(smem_at(&s_empty[s]), TMA ? 3 : 1);      // products done; the bias' warps
        bar_init(smem_at(&s_loaded[s]), 1);
      }
      for (uint32_t i = 0; i < 2; ++i) {
        bar_init(smem_at(&s_sum_full[i]), 1);
        bar_init(smem_at(&s_sum_empty[i]), 16);
      }
      bar_init(smem_at(&s_tail), 4);
      bar_init(smem_at(&s_done), 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
  }
  for (uint32_t i = tid; i < SUMS * kCols; i += kThreads) s_bias[i] = 0.0f;
  tmem_before();
  __syncthreads();
  pair_sync();
  tmem_after();
  const uint32_t tmem = s_tmem;

  __syncwarp();
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRest));
    if (warp == 8 && lane == 0 && rank == 0 && steps) {
      bool alive = true;
      for (uint32_t s = 0; s < steps; ++s) {
        const uint32_t st = s % ST, code = tiles + st * STAGE, grad = code + kTile, chunk = s / CH, acc = tmem + (chunk & 1) * 256;
        if (s % CH == 0 && chunk >= 2) alive = bar_wait(smem_at(&s_sum_empty[chunk & 1]), (chunk / 2 - 1) & 1);
        alive = alive && bar_wait(smem_at(&s_full[st]), s / ST & 1);
        if (!alive) break;
        tmem_after();
        const uint32_t groups = min(R / 16, (count - s * R + 15) / 16);   // of sixteen rows: the last step may have fewer
#pragma unroll
        for (uint32_t k = 0; k < R / 16; ++k) {
          if (k >= groups) break;
          const uint64_t cd = tile_desc<T>(code + k * 2048);
#pragma unroll
          for (uint32_t p = 0; p < P; ++p) {
            const uint64_t gd = tile_desc<T>(grad + p * kTile + k * 2048);
            mma(acc, a.in_out ? gd : cd, a.in_out ? cd : gd, kIdesc | idesc_cols(a.n), s % CH || k || p);
          }
        }
        mma_commit(smem_at(&s_empty[st]));
        if (s % CH == CH - 1 || s == steps - 1) mma_commit(smem_at(&s_sum_full[chunk & 1]));
      }
      mma_commit(smem_at(&s_done));   // nothing is under way when tensor memory is given back
      if (!(bar_wait(smem_at(&s_done), 0) && alive)) report(a.status, DGS_ETIMEOUT);
    }
    if (warp == 9 && lane == 0) {
      const uint32_t code_blocks = (code_cols + 63) / 64, grad_blocks = (grad_cols + 63) / 64;
      bool alive = true;
      uint32_t s = 0;
      for (; s < steps; ++s) {
        const uint32_t st = s % ST, to = tiles + st * STAGE, bar = smem_at(&s_loaded[st]), grads = TMA && s < tma_steps ? grad_blocks : 0;
        if (s >= ST && !(alive = bar_wait(smem_at(&s_empty[st]), (s / ST - 1) & 1))) break;
        bar_expect(bar, (code_blocks + grads) * kColBlock);
        for (uint32_t c = 0; c < code_blocks; ++c) tma_load(to + c * kColBlock, &held_map, int(ci + c * 64), int(held_first + uint64_t(s) * R), bar);
        if constexpr (TMA)
          for (uint32_t c = 0; c < grads; ++c) tma_load(to + kTile + c * kColBlock, &grad_map, int(go + c * 64), int(first + uint64_t(s) * R), bar);
      }
      if (!alive) {   // copies that nobody waits for any more
        report(a.status, DGS_ETIMEOUT);
        for (uint32_t i = s > ST ? s - ST : 0; i < s; ++i) bar_wait(smem_at(&s_loaded[i % ST]), i / ST & 1);
      }
    }
    if (warp == 10 || (TMA && warp == 11)) {
      // 64 threads: eight columns of every fourth row
      const uint32_t t = tid - 320, br = t / 16, bv = t % 16;
      float bias[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) bias[i] = 0.0f;
      bool alive = true;
      for (uint32_t s = 0; s < steps; ++s) {
        const uint32_t st = s % ST;
        if (!(alive = warp_wait(smem_at(&s_loaded[st]), s / ST & 1))) break;
        if (TMA && s >= tma_steps && !(alive = warp_wait(smem_at(&s_tail), 0))) break;
        if (warp == 10 && lane == 0) bar_arrive_cluster(in_leader(smem_at(&s_full[st])));
        if constexpr (TMA) {
          if (bias_here && s < tma_steps && s % a.bias_tiles == ct) {
#pragma unroll 4
            for (uint32_t r = br; r < R; r += 4) {
              uint4 w;
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                           : "r"(tiles + st * STAGE + kTile + tile_at<T>(r, bv)));
              bias_add(w, bias);
            }
          }
          __syncwarp();
          if (lane == 0) bar_arrive(smem_at(&s_empty[st]));
        }
      }
      if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);
      if constexpr (TMA)
#pragma unroll
        for (int i = 0; i < 8; ++i) s_bias[br * kCols + bv * 8 + i] = bias[i];
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSum));
    const T* dy = static_cast<const T*>(a.dy);
    const T* dy_end = dy + ((a.dy_rows - 1) * a.dy_stride + a.outputs);   // read where dy_rows > 0 only
    const uint32_t quarter = warp % 4, group = warp / 4, t = tid % 128;
    float acc[128];
#pragma unroll
    for (int i = 0; i < 128; ++i) acc[i] = 0.0f;
    bool alive = true;

    // Gradients: eight columns a thread, of rows that leave the same remainder by 8 in a warp (by 4, two in turn): rows 8 apart begin on the
    // same bytes of a word.  A batch of rows goes through the registers at a time.
    constexpr uint32_t BATCH = TMA ? 16 : G::kBatch, GR = BATCH / 8;
    const uint32_t gr = t / 32 + (lane / 16) * 8, gv = t % 16;
    constexpr auto grad_row = [](uint32_t u) { return u % 2 * 4 + u / 2 * 16; };
    const uint32_t grad_left = go + gv * 8 < a.outputs ? a.outputs - go - gv * 8 : 0;
    const T* const grad_at = dy + (first + gr) * a.dy_stride + go + gv * 8;
    Word<T> grad[GR];
    // Two-byte types: where every lane's eight elements lie in whole words in every row (mostly), a lane takes one word of a row and gets the next
    // from its neighbour; the seventeenth word of a row goes to one lane for each row.
    constexpr bool WORDS = sizeof(T) == 2 && !TMA;
    bool fast = false;
    uint4 edge = make_uint4(0, 0, 0, 0);
    auto fetch_grads = [&](uint32_t from) {
      const T* p = grad_at + uint64_t(from) * a.dy_stride;
      if constexpr (WORDS) {
        const uintptr_t low = reinterpret_cast<uintptr_t>(p) & ~uintptr_t(15), high = (reinterpret_cast<uintptr_t>(p + grad_row(GR - 1) * a.dy_stride) & ~uintptr_t(15)) + 32;
        fast = __all_sync(0xffffffffu, grad_left >= 8 && from + BATCH <= count && low >= reinterpret_cast<uintptr_t>(dy) && high <= reinterpret_cast<uintptr_t>(dy_end));
        if (fast) {
#pragma unroll
          for (uint32_t u = 0; u < GR; ++u)
            grad[u].a = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p + grad_row(u) * a.dy_stride) & ~uintptr_t(15)));
          if (gv < GR) edge = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p + grad_row(gv) * a.dy_stride + kCols - gv * 8) & ~uintptr_t(15)));
          return;
        }
      }
#pragma unroll
      for (uint32_t u = 0; u < GR; ++u)
        grads_load<T>(grad[u], p + grad_row(u) * a.dy_stride, from + gr + grad_row(u) < count ? grad_left : 0, dy, dy_end);
    };
    auto store_grads = [&](uint32_t from, uint32_t to, uint32_t row, bool mine, float (&bias)[8]) {
      const T* p = grad_at + uint64_t(from) * a.dy_stride;
      if constexpr (WORDS) {
        if (fast) {
#pragma unroll
          for (uint32_t u = 0; u < GR; ++u) {
            const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p + grad_row(u) * a.dy_stride)) & 15u;   // the same in all lanes
            uint4 w = grad[u].a;
            if (off) {
              uint4 next;
              const uint32_t from_lane = (lane & 16u) + u;
              next.x = next_word(w.x, edge.x, from_lane);
              next.y = next.z = next.w = 0;
              if (off > 4) next.y = next_word(w.y, edge.y, from_lane);
              if (off > 8) next.z = next_word(w.z, edge.z, from_lane), next.w = next_word(w.w, edge.w, from_lane);
              w = words_from(w, next, off);
            }
            grads_split<T>(w, to + tile_at<T>(row + gr + grad_row(u), gv), mine, bias);
          }
          return;
        }
      }
#pragma unroll
      for (uint32_t u = 0; u < GR; ++u)
        grads_store<T>(grad[u], p + grad_row(u) * a.dy_stride, from + gr + grad_row(u) < count ? grad_left : 0, dy, dy_end, to + tile_at<T>(row + gr + grad_row(u), gv), mine, bias);
    };
    uint32_t drained = 0;
    auto drain = [&]() {
      const uint32_t buf = drained & 1;
      if (!(alive = warp_wait(smem_at(&s_sum_full[buf]), drained / 2 & 1))) return;
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
      ++drained;
    };
    if constexpr (TMA) {
      while (alive && drained < chunks) {
        if (drained + 1 == chunks && tma_steps < steps && group == 0) {
          // an expert's last rows: a batch at a time, zeros behind them
          const uint32_t s = steps - 1, at = tiles + s % ST * STAGE + kTile;
          if (s >= ST && !(alive = warp_wait(smem_at(&s_empty[s % ST]), (s / ST - 1) & 1))) break;
          float bias[8] = {};
#pragma unroll 1
          for (uint32_t row = 0; row < R; row += BATCH) {
            fetch_grads(s * R + row);
            store_grads(s * R + row, at, row, bias_here && s % a.bias_tiles == ct, bias);
          }
          writes_to_async_proxy();
          __syncwarp();
          if (lane == 0) bar_arrive(smem_at(&s_tail));
#pragma unroll
          for (int i = 0; i < 8; ++i) s_bias[(4 + t / 16) * kCols + gv * 8 + i] = bias[i];   // behind the rows of the TMA steps' sums
        }
        drain();
      }
    } else {
      float bias[8] = {};
      // what follows a batch: the next of this step or the first of the group's next step
      auto after = [&](uint32_t from) { return (from / BATCH + 1) % (R / BATCH) ? from + BATCH : from / R * R + 2 * R; };
      if (steps) fetch_grads(group * R);
      for (uint32_t s = group; s < steps; s += 2) {
        const uint32_t st = s % ST, at = tiles + st * STAGE + kTile;
        if (s >= ST && !(alive = warp_wait(smem_at(&s_empty[st]), (s / ST - 1) & 1))) break;
        const bool mine = bias_here && s % a.bias_tiles == ct;
#pragma unroll 1
        for (uint32_t row = 0; row < R; row += BATCH) {
          store_grads(s * R + row, at, row, mine, bias);
          fetch_grads(after(s * R + row));
        }
        writes_to_async_proxy();
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(in_leader(smem_at(&s_full[st])));
        // the wait above said that step s - ST is done
        if (s >= ST && s - ST >= CH * (drained + 1) - 1) {
          drain();
          if (!alive) break;
        }
      }
      while (alive && drained < chunks) drain();
#pragma unroll
      for (int i = 0; i < 8; ++i) s_bias[(group * 8 + t / 16) * kCols + gv * 8 + i] = bias[i];
    }
    if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);

    // results to memory
    const uint32_t row = rank * 128 + quarter * 32 + lane;
    const uint32_t lane_at = (a.in_out ? o0 : i0) + row, lane_end = a.in_out ? a.outputs : a.inputs;
    const uint32_t col_at = (a.in_out ? i0 : o0) + group * 128, col_end = min(a.in_out ? a.inputs : a.outputs, (a.in_out ? i0 : o0) + a.n);
    if (alive && lane_at < lane_end) {
      float* p = a.dw + (uint64_t(split) * a.experts + expert) * a.inputs * a.outputs + uint64_t(col_at) * lane_end + lane_at;
#pragma unroll
      for (uint32_t g = 0; g < 8; ++g) {
        if (a.add_w) {
          float old[16];
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i) old[i] = col_at + g * 16 + i < col_end ? p[uint64_t(g * 16 + i) * lane_end] : 0.0f;
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i) acc[g * 16 + i] += old[i];
        }
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i)
          if (col_at + g * 16 + i < col_end) p[uint64_t(g * 16 + i) * lane_end] = acc[g * 16 + i];
      }
    }
  }
  tmem_before();
  __syncthreads();
  if (bias_here && tid < grad_cols && go + tid < a.outputs) {
    float v = 0.0f;
    for (uint32_t i = 0; i < SUMS; ++i) v += s_bias[i * kCols + tid];
    float* p = a.db + (uint64_t(split * a.bias_tiles + ct) * a.experts + expert) * a.outputs + go + tid;
    *p = a.add_b ? *p + v : v;
  }
  pair_sync();
  if (warp == 8) {
    __syncwarp();
    tmem_after();
    tmem_free(tmem, kTmemCols);
  }
}

// Adds up partial results in their order: of dw over the splits, of db over the splits and the CTAs that shared its steps.
__global__ void __launch_bounds__(256) k_weight_sum(float* dw, float* db, const float* pw, const float* pb, uint64_t nw, uint64_t nb, uint32_t parts_w,
                                                    uint32_t parts_b, uint32_t add) {
  const uint64_t total = nw + nb;
  for (uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += uint64_t(gridDim.x) * 256) {
    const bool w = i < nw;
    const uint64_t k = w ? i : i - nw, n = w ? nw : nb;
    const float* p = (w ? pw : pb) + k;
    float* out = (w ? dw : db) + k;
    const uint32_t parts = w ? parts_w : parts_b;
    float v = 0.0f;
    for (uint32_t s = 0; s < parts; ++s) v += p[s * n];
    *out = add ? *out + v : v;
  }
}

// ---- host side --------------------------------------------------------------------------------
struct WeightPlan {
  uint32_t code_tiles, grad_tiles, n, splits, bias_tiles, experts;
  uint32_t step_rows;
  uint64_t nw, nb, decoded, bytes;
};

bool lists_ok(const dgs_row_lists* l) {
  return !l || (l->offsets && l->experts && l->experts <= DGS_ROUTE_MAX_EXPERTS && l->rows_per && aligned(l->offsets, 4) && aligned(l->rows, 4));
}

uint32_t ceil_div(uint64_t a, uint64_t b) { return uint32_t((a + b - 1) / b); }

int plan_weight(const dgs_checkpoint* c, const dgs_matrix* dy, const dgs_row_lists* lists, uint32_t flags, WeightPlan* p) {
  if (!checkpoint_ok(c) || !matrix_ok(dy, false) || !lists_ok(lists) || (lists ? c->rows == 0 && dy->rows : dy->rows != c->rows))
    return DGS_EINVAL;
  const uint32_t parts = dy->type == DGS_TYPE_BF16 ? 1 : dy->type == DGS_TYPE_FP16 ? 2 : 3;
  const bool in_out = flags & DGS_WEIGHT_IN_OUT;
  p->experts = lists ? lists->experts : 1;
  if (uint64_t(c->cols) * dy->cols > kMostElements / p->experts || dy->rows >= (1u << 31) - 1025 * 128) return DGS_ELIMIT;
  p->nw = uint64_t(c->cols) * dy->cols * p->experts;
  p->nb = uint64_t(dy->cols) * p->experts;
  // The tile's width and the split of a tile's rows among pairs: whatever ends soonest.  74 pairs run at a time; a round takes the steps of a pair
  // and about 4 us around them, and partial results cost their way through the second cache and another launch.
  const uint32_t steps = std::max(1u, ceil_div(dy->rows / p->experts, 64));   // of 64 rows, whatever the kernel's are
  p->step_rows = dy->type == DGS_TYPE_BF16 ? Grad<__nv_bfloat16>::kRows : Grad<float>::kRows;
  static_assert(Grad<__half>::kRows == Grad<float>::kRows, "");
  double best = 1e300;
  for (uint32_t n = 256; n >= 64; n -= 64) {
    const uint64_t tiles = uint64_t(ceil_div(in_out ? c->cols : dy->cols, n)) * ceil_div(in_out ? dy->cols : c->cols, 256) * p->experts;
    const double step_us = parts * (0.10 + 0.28 * n / 256);
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
  p->decoded = dy->rows ? decoded_rows(dy->rows, lists ? p->experts : 0, p->step_rows) * held_width(c->cols) * 2 : 0;
  p->bytes = p->decoded + (p->splits > 1 ? p->nw * p->splits * 4 : 0) + (parts_b > 1 ? p->nb * parts_b * 4 : 0);
  return DGS_OK;
}

constexpr int kMaxDevices = 64;
std::mutex g_weight_mu;
bool g_weight_ready[kMaxDevices];
PFN_cuTensorMapEncodeTiled_v12000 g_encode;   // written once, under the mutex
template <class T, bool TMA>
bool weight_setup() {
  cudaFuncAttributes f;
  // the split of the registers counts on what the launch brings
  return cudaFuncGetAttributes(&f, k_weight_grad<T, TMA>) == cudaSuccess && uint32_t(f.numRegs) >= kRegsLaunch &&
         cudaFuncSetAttribute(k_weight_grad<T, TMA>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<T>::kSmem) == cudaSuccess;
}
int weight_ready() {   // once per device
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return DGS_ECUDA;
  std::lock_guard<std::mutex> lock(g_weight_mu);
  if (!g_weight_ready[dev]) {
    if (!weight_setup<float, false>() || !weight_setup<__half, false>() || !weight_setup<__nv_bfloat16, false>() || !weight_setup<__nv_bfloat16, true>())
      return DGS_ECUDA;
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess || !fn) return DGS_ECUDA;
    g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    g_weight_ready[dev] = true;
  }
  return DGS_OK;
}

// A TMA copy takes blocks of 64 columns of bfloat16 numbers from rows that begin on 16 bytes.
bool tma_fits(const dgs_matrix* dy) {
  return dy->type == DGS_TYPE_BF16 && aligned(dy->data, 16) && dy->stride % 8 == 0 && dy->stride >= dy->cols && dy->cols < (1u << 31);
}
int make_map(void* data, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t box_rows, CUtensorMap* map) {
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {stride * 2};
  const cuuint32_t box[2] = {64, box_rows}, each[2] = {1, 1};
  return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, data, dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? DGS_OK
             : DGS_ECUDA;
}

template <class T, bool TMA>
int launch(const WeightArgs& a, const CUtensorMap& held, const CUtensorMap& grad, uint32_t ctas, cudaStream_t st) {
  k_weight_grad<T, TMA><<<ctas, kThreads, Shape<T>::kSmem, st>>>(a, held, grad);
  return cudaGetLastError() == cudaSuccess ? DGS_OK : DGS_ECUDA;
}

}  // namespace
}  // namespace dgs

using namespace dgs;

extern "C" int dgs_checkpoint_weight_grad_bytes(const dgs_checkpoint* ckpt, const dgs_matrix* dy, const dgs_row_lists* lists, uint32_t flags,
                                                uint64_t* out_bytes) {
  WeightPlan p;
  if (!out_bytes || (flags & ~(DGS_WEIGHT_IN_OUT | DGS_WEIGHT_ADD))) return DGS_EINVAL;
  const int rc = plan_weight(ckpt, dy, lists, flags, &p);
  if (rc == DGS_OK) *out_bytes = p.bytes;
  return rc;
}

extern "C" int dgs_checkpoint_weight_grad(const dgs_checkpoint* ckpt, const dgs_matrix* dy, const dgs_row_lists* lists, float* dw, float* db,
                                          uint32_t flags, void* workspace, uint64_t workspace_bytes, void* stream) {
  WeightPlan p;
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
  rc = weight_ready();
  if (rc != DGS_OK) return rc;
  const uint32_t parts_b = p.splits * p.bias_tiles;
  WeightArgs a = {};
  a.h = held_of(ckpt);
  a.dy = dy->data;
  a.dy_rows = dy->rows;
  a.dy_stride = dy->stride;
  a.inputs = ckpt->cols;
  a.outputs = dy->cols;
  a.code_tiles = p.code_tiles;
  a.grad_tiles = p.grad_tiles;
  a.splits = p.splits;
  a.experts = p.experts;
  a.rows_per = lists ? lists->rows_per : 1;
  a.n = p.n;
  a.in_out = flags & DGS_WEIGHT_IN_OUT ? 1 : 0;
  a.bias_tiles = p.bias_tiles;
  a.step_rows = p.step_rows;
  a.offsets = lists ? lists->offsets : nullptr;
  a.rows = lists ? lists->rows : nullptr;
  a.decoded = static_cast<__nv_bfloat16*>(workspace);
  float* const part_w = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.decoded);
  float* const part_b = part_w + (p.splits > 1 ? p.nw * p.splits : 0);
  a.dw = p.splits > 1 ? part_w : dw;
  a.db = !db ? nullptr : parts_b > 1 ? part_b : db;
  const uint32_t add = flags & DGS_WEIGHT_ADD ? 1 : 0;
  a.add_w = p.splits == 1 ? add : 0;
  a.add_b = parts_b == 1 ? add : 0;
  a.status = operator_status_word();
  if (!a.status) return DGS_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  CUtensorMap held = {}, grad = {};
  const bool tma = dy->rows && tma_fits(dy);
  if (dy->rows) {
    const uint64_t rows = p.decoded / (2 * uint64_t(a.h.width));
    rc = make_map(a.decoded, rows, a.h.width, a.h.width, p.step_rows, &held);
    if (rc == DGS_OK && tma) rc = make_map(dy->data, dy->rows, dy->cols, dy->stride, p.step_rows, &grad);
    if (rc != DGS_OK) return rc;
    const uint32_t ctas = ceil_div(rows, kDecodeRows);
    if (ckpt->format == DGS_FORMAT_E4M3)
      k_weight_decode<true><<<ctas, 256, 0, st>>>(a);
    else
      k_weight_decode<false><<<ctas, 256, 0, st>>>(a);
    if (cudaGetLastError() != cudaSuccess) return DGS_ECUDA;
  }
  const uint32_t ctas = p.code_tiles * p.grad_tiles * p.splits * p.experts * 2;
  rc = with_type(dy->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if constexpr (std::is_same_v<T, __nv_bfloat16>)
      if (tma) return launch<T, true>(a, held, grad, ctas, st);
    return launch<T, false>(a, held, grad, ctas, st);
  });
  const uint64_t nw = p.splits > 1 ? p.nw : 0, nb = db && parts_b > 1 ? p.nb : 0;
  if (rc != DGS_OK || nw + nb == 0) return rc;
  k_weight_sum<<<uint32_t(std::min<uint64_t>((nw + nb + 255) / 256, kSms * 8)), 256, 0, st>>>(dw, db, part_w, part_b, nw, nb, p.splits, parts_b, add);
  return cudaGetLastError() == cudaSuccess ? DGS_OK : DGS_ECUDA;
}
