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
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
constexpr uint32_t kPolls = 1u << 20;   // far above any wait that ends
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  for (uint32_t n = 0; n < kPolls; ++n) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
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
__device__ __forceinline__ void tmem_load16(uint32_t at, float (&v)[16]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// ---- tiles in shared memory ---------------------------------------------------------------------
// Both operands are contracted over their rows, so both lie in memory with the other dimension contiguous, and stay so: a tile of
// 64 rows is cut into blocks of 64 columns, each 64 rows of 128 bytes with the 16-byte pieces of a row exchanged by the row's
// number (128-byte swizzle).  Descriptor: blocks of 64 columns 8192 bytes apart, groups of 8 rows 1024 bytes apart.
constexpr uint32_t kRows = 64;                 // rows of a step
constexpr uint32_t kColBlock = kRows * 128;    // bytes of 64 columns
constexpr uint32_t kCols = 128;                // columns of either operand that a CTA brings, at most
constexpr uint32_t kTile = kCols / 64 * kColBlock;
__device__ __forceinline__ uint32_t tile_at(uint32_t row, uint32_t piece) {   // piece: eight columns
  return (piece >> 3) * kColBlock + row * 128 + (((piece ^ row) & 7) << 4);
}
__device__ __forceinline__ uint64_t tile_desc(uint32_t at) {
  return uint64_t(at >> 4 & 0x3fff) | uint64_t(kColBlock >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// f32 += bf16 x bf16, 256 rows in a pair, both operands with the contracted dimension outermost
constexpr uint32_t kIdesc = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (256u >> 4) << 24;
__device__ __forceinline__ uint32_t idesc_cols(uint32_t n) { return (n >> 3) << 17; }

// A gradient's type: how many bfloat16 numbers add up to one of its values; stages of shared memory; steps between two sums in registers.
template <class T> struct Grad;
template <> struct Grad<__nv_bfloat16> { static constexpr uint32_t kParts = 1, kStages = 6, kChunk = 8; };
template <> struct Grad<__half> { static constexpr uint32_t kParts = 2, kStages = 4, kChunk = 4; };
template <> struct Grad<float> { static constexpr uint32_t kParts = 3, kStages = 3, kChunk = 3; };
template <class T> struct Shape {
  static constexpr uint32_t kStage = kTile * (1 + Grad<T>::kParts);
  static constexpr uint32_t kSmem = 1024 + Grad<T>::kStages * kStage;
};
constexpr uint32_t kTmemCols = 512;            // two accumulators of 256 columns
constexpr uint32_t kThreads = 384;             // two warpgroups bring the operands and keep the sums, one issues
constexpr uint32_t kRegsLaunch = 168, kRegsBring = 232, kRegsIssue = 40;
static_assert(kRegsBring * 256 + kRegsIssue * 128 <= kRegsLaunch * kThreads, "setmaxnreg draws on the launch's registers");

struct WeightArgs {
  Held h;
  const void* dy;
  uint64_t dy_rows, dy_stride;
  uint32_t outputs, code_tiles, grad_tiles, splits, experts, rows_per;
  uint32_t n;           // columns of the operand that the pair shares out: 64 .. 256
  uint32_t in_out, bias_tiles;
  const uint32_t* offsets;
  const uint32_t* rows;
  float* dw;          // or the splits' partial results, [splits][experts][inputs * outputs]
  float* db;          // likewise, [splits * bias_tiles][experts][outputs]; NULL: not wanted
  uint32_t add_w, add_b;
  int* status;
};

// ---- eight codes to eight bfloat16 numbers --------------------------------------------------------
__device__ __forceinline__ uint32_t bf2(uint32_t a, uint32_t b, bool mul) {
  __nv_bfloat162 x, y;
  memcpy(&x, &a, 4);
  memcpy(&y, &b, 4);
  const __nv_bfloat162 r = mul ? __hmul2(x, y) : __hsub2(x, y);
  uint32_t w;
  memcpy(&w, &r, 4);
  return w;
}
__device__ __forceinline__ uint32_t scale_bf2(uint32_t byte) { return byte == kNanScale ? 0x7fc07fc0u : byte << 7 | byte << 23; }

template <bool FLOAT8>
__device__ __forceinline__ uint32_t codes_bf2(uint32_t w, uint32_t pair, uint32_t scale) {
  if constexpr (FLOAT8) {
    // sign, 4 bits of exponent and 3 of mantissa go where a bfloat16 has them; 2^120 makes up for the exponents' different zero (for
    // the subnormal codes too, which are subnormal bfloat16 numbers until then)
    const uint32_t t = __byte_perm(w, 0, pair ? 0x3424 : 0x1404);
    const uint32_t m = (t & 0x80008000u) | (t >> 4 & 0x07f007f0u);
    return bf2(bf2(m, 0x7b807b80u, true), scale, true);
  } else {
    // 128 + the code's low 7 bits, less 128, or less 256 where the code is negative: every step is exact in 8 bits
    const uint32_t t = __byte_perm(w, 0x43434343u, pair ? 0x4342 : 0x4140);
    return bf2(bf2(t & 0xff7fff7fu, t & 0xff80ff80u, false), scale, true);
  }
}
template <bool FLOAT8>
__device__ __forceinline__ uint4 codes_bf8(uint32_t lo, uint32_t hi, uint32_t scale) {
  return make_uint4(codes_bf2<FLOAT8>(lo, 0, scale), codes_bf2<FLOAT8>(lo, 1, scale), codes_bf2<FLOAT8>(hi, 0, scale), codes_bf2<FLOAT8>(hi, 1, scale));
}

// ---- eight gradients ------------------------------------------------------------------------------
// Rows may begin on any element.  Two-byte types read the aligned 16-byte words around the eight elements and shift; what lies at a
// row's end or at an end of the matrix is read element by element.
template <class T> struct Eight {
  uint4 a, b;
  uint32_t shift;   // bytes into a:b (two-byte types)
};
template <class T>
__device__ __forceinline__ void grads_load(Eight<T>& r, const T* p, uint32_t left, const T* lo, const T* hi) {
  r.a = r.b = make_uint4(0, 0, 0, 0);
  r.shift = 0;
  if (left == 0) return;
  const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p)) & 15u;
  if constexpr (sizeof(T) == 4) {
    if (left >= 8 && off == 0) {
      r.a = __ldg(reinterpret_cast<const uint4*>(p));
      r.b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
      return;
    }
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = uint32_t(i) < left ? __ldg(reinterpret_cast<const uint32_t*>(p) + i) : 0u;
    r.a = make_uint4(v[0], v[1], v[2], v[3]);
    r.b = make_uint4(v[4], v[5], v[6], v[7]);
  } else {
    const char* base = reinterpret_cast<const char*>(p) - off;
    if (left >= 8 && (off == 0 || (base >= reinterpret_cast<const char*>(lo) && base + 32 <= reinterpret_cast<const char*>(hi)))) {
      r.a = __ldg(reinterpret_cast<const uint4*>(base));
      if (off) r.b = __ldg(reinterpret_cast<const uint4*>(base) + 1);
      r.shift = off;
      return;
    }
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = uint32_t(i) < left ? __ldg(reinterpret_cast<const unsigned short*>(p) + i) : 0u;
    r.a = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
  }
}
template <class T>
__device__ __forceinline__ uint4 grads_words(const Eight<T>& r) {   // two-byte types: the eight elements
  uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
  if (r.shift & 8)
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  if (r.shift & 4)
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  const uint32_t s = (r.shift & 2) * 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], s);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void bias_add(const uint4& w, float (&bias)[8]) {   // eight bfloat16 numbers
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bias[2 * i] += __uint_as_float(v[i] << 16);
    bias[2 * i + 1] += __uint_as_float(v[i] & 0xffff0000u);
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
template <class T>
__device__ __forceinline__ void grads_store(const Eight<T>& r, uint32_t at, uint32_t part_bytes, bool mine, float (&bias)[8]) {
  constexpr uint32_t P = Grad<T>::kParts;
  uint32_t out[P][4];
  if constexpr (P == 1) {
    const uint4 w = grads_words(r);
    out[0][0] = w.x, out[0][1] = w.y, out[0][2] = w.z, out[0][3] = w.w;
    if (mine) bias_add(w, bias);
  } else {
    float v[8];
    if constexpr (sizeof(T) == 4) {
      const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    } else {
      const uint4 q = grads_words(r);
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        __half2 h;
        memcpy(&h, &w[i], 4);
        const float2 f = __half22float2(h);
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
      }
    }
    if (mine)
#pragma unroll
      for (int i = 0; i < 8; ++i) bias[i] += v[i];
#pragma unroll
    for (uint32_t p = 0; p < P; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = upper(v[2 * i], &v[2 * i]), y = upper(v[2 * i + 1], &v[2 * i + 1]);
        out[p][i] = x >> 16 | y;
      }
  }
#pragma unroll
  for (uint32_t p = 0; p < P; ++p)
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + p * part_bytes), "r"(out[p][0]), "r"(out[p][1]), "r"(out[p][2]), "r"(out[p][3])
                 : "memory");
}

// ---- the kernel -----------------------------------------------------------------------------------
// A pair of CTAs forms a tile of 256 x n (n <= 256) over a run of an expert's rows, 64 rows a step.  Each CTA brings 128 columns of one operand and
// n / 2 of the other to its shared memory; the products of the pair read both (tcgen05, cta_group::2), and each CTA's tensor memory takes
// 128 rows of the result.  The dimension of dw that is contiguous in memory goes on those rows (lanes), so that a warp's stores are
// coalesced wherever the layer's slice begins: inputs for [outputs][inputs], outputs for [inputs][outputs]; only the operands' roles change.
//
// Eight warps decode the codes (and bring gradients that a TMA copy cannot: those of several parts, on odd addresses, and the last
// rows of an expert, where the next expert's would come along).  A ninth issues products, a tenth TMA copies.  Sums: the tensor cores
// add to their accumulator with bits cut off, which over 8192 rows leaves an error of 5.5e-6; so every kChunk steps the
// accumulators go to registers of the eight warps and are added up there with rounding, while the products go on in the other half of
// tensor memory.  db is summed by the eight warps from the tiles, each step by one of the CTAs that hold the same gradients.
template <class T, bool FLOAT8, bool TMA>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
k_weight_grad(const __grid_constant__ WeightArgs a, const __grid_constant__ CUtensorMap map) {
  constexpr uint32_t P = Grad<T>::kParts, ST = Grad<T>::kStages, CH = Grad<T>::kChunk, STAGE = Shape<T>::kStage;
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[ST], s_empty[ST], s_loaded[ST], s_sum_full[2], s_sum_empty[2], s_done;
  __shared__ uint32_t s_tmem;
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

  uint64_t first = 0, last = a.dy_rows, limit = a.dy_rows;
  if (a.offsets) {
    const uint64_t x = a.offsets[expert], y = a.offsets[expert + 1];
    first = x < a.dy_rows ? x : a.dy_rows;
    last = y < first ? first : y < a.dy_rows ? y : a.dy_rows;
    if ((first != x || last != y) && tid == 0) report(a.status, DGS_EINVAL);
  }
  {
    const uint64_t steps = (last - first + kRows - 1) / kRows, each = (steps + a.splits - 1) / a.splits;
    const uint64_t from = min(first + split * each * kRows, last);
    last = min(from + each * kRows, last);
    first = from;
  }
  const uint32_t steps = uint32_t((last - first + kRows - 1) / kRows), chunks = (steps + CH - 1) / CH;
  // the last step comes by TMA only where nothing but the end of the matrix follows
  const uint32_t tma_steps = !TMA ? 0 : (last - first) % kRows == 0 || last == limit ? steps : steps - 1;

  if (warp == 8) {
    tmem_alloc(&s_tmem, kTmemCols);
    if (lane == 0) {
      for (uint32_t s = 0; s < ST; ++s) {
        bar_init(smem_at(&s_full[s]), 16);
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
  tmem_before();
  __syncthreads();
  pair_sync();
  tmem_after();
  const uint32_t tmem = s_tmem;

  __syncwarp();
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == 8 && lane == 0 && rank == 0 && steps) {
      bool alive = true;
      for (uint32_t s = 0; s < steps; ++s) {
        const uint32_t st = s % ST, code = tiles + st * STAGE, grad = code + kTile, chunk = s / CH, acc = tmem + (chunk & 1) * 256;
        if (s % CH == 0 && chunk >= 2) alive = bar_wait(smem_at(&s_sum_empty[chunk & 1]), (chunk / 2 - 1) & 1);
        alive = alive && bar_wait(smem_at(&s_full[st]), s / ST & 1);
        if (!alive) break;
        tmem_after();
#pragma unroll
        for (uint32_t k = 0; k < kRows / 16; ++k) {
          const uint64_t cd = tile_desc(code + k * 2048);
#pragma unroll
          for (uint32_t p = 0; p < P; ++p) {
            const uint64_t gd = tile_desc(grad + p * kTile + k * 2048);
            mma(acc, a.in_out ? gd : cd, a.in_out ? cd : gd, kIdesc | idesc_cols(a.n), s % CH || k || p);
          }
        }
        mma_commit(smem_at(&s_empty[st]));
        if (s % CH == CH - 1 || s == steps - 1) mma_commit(smem_at(&s_sum_full[chunk & 1]));
      }
      mma_commit(smem_at(&s_done));   // nothing is under way when tensor memory is given back
      if (!(bar_wait(smem_at(&s_done), 0) && alive)) report(a.status, DGS_ETIMEOUT);
    }
    if (TMA && warp == 9 && lane == 0 && tma_steps) {
      const uint32_t blocks = (grad_cols + 63) / 64;
      bool alive = true;
      uint32_t s = 0;
      for (; s < tma_steps; ++s) {
        const uint32_t st = s % ST, to = tiles + st * STAGE + kTile, bar = smem_at(&s_loaded[st]);
        if (s >= ST && !(alive = bar_wait(smem_at(&s_empty[st]), (s / ST - 1) & 1))) break;
        bar_expect(bar, blocks * kColBlock);
        for (uint32_t c = 0; c < blocks; ++c) tma_load(to + c * kColBlock, &map, int(go + c * 64), int(first + uint64_t(s) * kRows), bar);
      }
      if (!alive) {   // copies that nobody waits for any more
        report(a.status, DGS_ETIMEOUT);
        for (uint32_t i = s > ST ? s - ST : 0; i < s; ++i) bar_wait(smem_at(&s_loaded[i % ST]), i / ST & 1);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsBring));
    const T* dy = static_cast<const T*>(a.dy);
    const T* dy_end = dy + ((a.dy_rows - 1) * a.dy_stride + a.outputs);   // read where dy_rows > 0 only
    const uint32_t quarter = warp % 4, half = warp / 4;
    float acc[128], bias[8];
#pragma unroll
    for (int i = 0; i < 128; ++i) acc[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) bias[i] = 0.0f;
    bool alive = true;

    // codes: 16 columns of two rows a thread.  Row numbers are taken three steps ahead, codes two.
    const uint32_t cr = tid / 8, cv = tid % 8;
    const bool cols_in = cv * 16 < code_cols && ci + cv * 16 < a.h.width;
    struct CodeStep {
      uint4 w[2];
      uint32_t scale[2];
    };
    uint64_t src[2];
    auto find = [&](uint32_t s) {
#pragma unroll
      for (uint32_t u = 0; u < 2; ++u) {
        const uint64_t j = first + uint64_t(s) * kRows + cr + 32 * u;
        src[u] = ~0ull;
        if (j < last) {
          src[u] = a.rows ? a.rows[j] / a.rows_per : j;
          if (src[u] >= a.h.rows) {
            report(a.status, DGS_EINVAL);
            src[u] = ~0ull;
          }
        }
      }
    };
    auto fetch = [&](CodeStep& c) {
#pragma unroll
      for (uint32_t u = 0; u < 2; ++u) {
        c.w[u] = make_uint4(0, 0, 0, 0);
        c.scale[u] = 0;
        if (src[u] != ~0ull && cols_in) {
          c.w[u] = __ldg(reinterpret_cast<const uint4*>(a.h.codes + src[u] * a.h.width + ci + cv * 16));
          c.scale[u] = __ldg(a.h.scales + src[u] * a.h.spitch + (ci + cv * 16) / 32);
        }
      }
    };
    // gradients: eight columns of four rows a thread
    const uint32_t gr = tid / 16, gv = tid % 16;
    Eight<T> grad[4];
    auto fetch_grads = [&](uint32_t s) {
#pragma unroll
      for (uint32_t u = 0; u < 4; ++u) {
        const uint64_t j = first + uint64_t(s) * kRows + gr + 16 * u;
        const uint32_t col = go + gv * 8;
        grads_load<T>(grad[u], dy + j * a.dy_stride + col, j < last && gv * 8 < grad_cols && col < a.outputs ? a.outputs - col : 0, dy, dy_end);
      }
    };
    uint32_t drained = 0;
    auto drain = [&]() {
      const uint32_t buf = drained & 1;
      if (!(alive = warp_wait(smem_at(&s_sum_full[buf]), drained / 2 & 1))) return;
      tmem_after();
#pragma unroll
      for (uint32_t g = 0; g < 8; ++g) {
        if (half * 128 + g * 16 < a.n) {
          float v[16];
          tmem_load16(tmem + (quarter * 32 << 16) + buf * 256 + half * 128 + g * 16, v);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[g * 16 + i] += v[i];
        }
      }
      tmem_before();
      __syncwarp();
      if (lane == 0) bar_arrive_cluster(in_leader(smem_at(&s_sum_empty[buf])));
      ++drained;
    };
    auto step = [&](uint32_t s, CodeStep& c) {
      const uint32_t st = s % ST, at = tiles + st * STAGE;
      if (s >= ST && !(alive = warp_wait(smem_at(&s_empty[st]), (s / ST - 1) & 1))) return;
#pragma unroll
      for (uint32_t u = 0; u < 2; ++u) {
        const uint32_t r = cr + 32 * u, sc = scale_bf2(c.scale[u]);
        const uint4 x = codes_bf8<FLOAT8>(c.w[u].x, c.w[u].y, sc), y = codes_bf8<FLOAT8>(c.w[u].z, c.w[u].w, sc);
        const bool swap = cv >= 4;   // the halves of a row go to the same banks: one writes its second piece first
        const uint4 p = swap ? y : x, q = swap ? x : y;
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + tile_at(r, 2 * cv + swap)), "r"(p.x), "r"(p.y), "r"(p.z), "r"(p.w) : "memory");
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + tile_at(r, 2 * cv + !swap)), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
      }
      fetch(c);       // of step s + 2
      find(s + 3);
      const bool mine = a.db && s % a.bias_tiles == ct, by_tma = s < tma_steps;
      if (!by_tma) {
        if (TMA) fetch_grads(s);
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) grads_store<T>(grad[u], at + kTile + tile_at(gr + 16 * u, gv), kTile, mine, bias);
        if (!TMA && s + 1 < steps) fetch_grads(s + 1);
      } else if (mine || warp == 0) {
        if (!(alive = warp_wait(smem_at(&s_loaded[st]), s / ST & 1))) return;
        if (mine)
#pragma unroll
          for (uint32_t u = 0; u < 4; ++u) {
            uint4 w;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at + kTile + tile_at(gr + 16 * u, gv)));
            bias_add(w, bias);
          }
      }
      writes_to_async_proxy();
      __syncwarp();
      if (lane == 0) bar_arrive_cluster(in_leader(smem_at(&s_full[st])));
      // the wait above said that step s - ST is done
      if (s >= ST && s - ST >= CH * (drained + 1) - 1) drain();
    };
    CodeStep c0, c1;
    find(0);
    fetch(c0);
    find(1);
    fetch(c1);
    find(2);
    if (!TMA && steps) fetch_grads(0);
    for (uint32_t s = 0; s < steps && alive; s += 2) {
      step(s, c0);
      if (s + 1 < steps && alive) step(s + 1, c1);
    }
    while (alive && drained < chunks) drain();
    if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);

    // results to memory
    const uint32_t inputs = a.h.cols, row = rank * 128 + quarter * 32 + lane;
    const uint32_t lane_at = (a.in_out ? o0 : i0) + row, lane_end = a.in_out ? a.outputs : inputs;
    const uint32_t col_at = (a.in_out ? i0 : o0) + half * 128, col_end = min(a.in_out ? inputs : a.outputs, (a.in_out ? i0 : o0) + a.n);
    if (alive && lane_at < lane_end) {
      float* p = a.dw + (uint64_t(split) * a.experts + expert) * inputs * a.outputs + uint64_t(col_at) * lane_end + lane_at;
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
    if (a.db && ct < a.bias_tiles) {   // sixteen threads hold the same columns: their sums in order
      float* sums = reinterpret_cast<float*>(raw + (tiles - smem_at(raw)));
      asm volatile("bar.sync 1, 256;" ::: "memory");   // nothing reads the tiles any more: every chunk has been waited for
      if (alive) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[gr * kCols + gv * 8 + i] = bias[i];
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (alive && tid < grad_cols && go + tid < a.outputs) {
        float v = 0.0f;
        for (uint32_t i = 0; i < 16; ++i) v += sums[i * kCols + tid];
        float* p = a.db + (uint64_t(split * a.bias_tiles + ct) * a.experts + expert) * a.outputs + go + tid;
        *p = a.add_b ? *p + v : v;
      }
    }
  }
  tmem_before();
  __syncthreads();
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
  uint64_t nw, nb, bytes;
};

bool lists_ok(const dgs_row_lists* l) {
  return !l || (l->offsets && l->experts && l->experts <= 65535 && l->rows_per && aligned(l->offsets, 4) && aligned(l->rows, 4));
}

uint32_t ceil_div(uint64_t a, uint64_t b) { return uint32_t((a + b - 1) / b); }

int plan_weight(const dgs_checkpoint* c, const dgs_matrix* dy, const dgs_row_lists* lists, uint32_t flags, WeightPlan* p) {
  if (!checkpoint_ok(c) || !matrix_ok(dy, false) || !lists_ok(lists) || (!lists && dy->rows != c->rows)) return DGS_EINVAL;
  const uint32_t parts = dy->type == DGS_TYPE_BF16 ? 1 : dy->type == DGS_TYPE_FP16 ? 2 : 3;
  const bool in_out = flags & DGS_WEIGHT_IN_OUT;
  p->experts = lists ? lists->experts : 1;
  if (uint64_t(c->cols) * dy->cols > kMostElements / p->experts) return DGS_ELIMIT;
  p->nw = uint64_t(c->cols) * dy->cols * p->experts;
  p->nb = uint64_t(dy->cols) * p->experts;
  // The tile's width and the split of a tile's rows among pairs: whatever ends soonest.  74 pairs run at a time; a round takes the steps of a pair
  // and about 4 us around them, and partial results cost their way through the second cache and another launch.
  const uint32_t steps = std::max(1u, ceil_div(dy->rows / p->experts, kRows));
  double best = 1e300;
  for (uint32_t n = 256; n >= 64; n -= 64) {
    const uint64_t tiles = uint64_t(ceil_div(in_out ? c->cols : dy->cols, n)) * ceil_div(in_out ? dy->cols : c->cols, 256) * p->experts;
    const double step_us = parts * (0.12 + 0.28 * n / 256);
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
  p->bytes = (p->splits > 1 ? p->nw * p->splits * 4 : 0) + (parts_b > 1 ? p->nb * parts_b * 4 : 0);
  return DGS_OK;
}

constexpr int kMaxDevices = 64;
std::mutex g_weight_mu;
bool g_weight_ready[kMaxDevices];
PFN_cuTensorMapEncodeTiled_v12000 g_encode;   // written once, under the mutex
template <class T, bool FLOAT8, bool TMA>
bool weight_setup() {
  cudaFuncAttributes f;
  // the split of the registers counts on what the launch brings
  return cudaFuncGetAttributes(&f, k_weight_grad<T, FLOAT8, TMA>) == cudaSuccess && uint32_t(f.numRegs) >= kRegsLaunch &&
         cudaFuncSetAttribute(k_weight_grad<T, FLOAT8, TMA>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<T>::kSmem) == cudaSuccess;
}
int weight_ready() {   // once per device
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return DGS_ECUDA;
  std::lock_guard<std::mutex> lock(g_weight_mu);
  if (!g_weight_ready[dev]) {
    if (!weight_setup<float, false, false>() || !weight_setup<float, true, false>() || !weight_setup<__half, false, false>() ||
        !weight_setup<__half, true, false>() || !weight_setup<__nv_bfloat16, false, false>() || !weight_setup<__nv_bfloat16, true, false>() ||
        !weight_setup<__nv_bfloat16, false, true>() || !weight_setup<__nv_bfloat16, true, true>())
      return DGS_ECUDA;
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess || !fn) return DGS_ECUDA;
    g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    g_weight_ready[dev] = true;
  }
  return DGS_OK;
}

// A TMA copy takes blocks of 64 x 64 from rows that begin on 16 bytes.
bool tma_fits(const dgs_matrix* dy) {
  return dy->type == DGS_TYPE_BF16 && dy->rows && aligned(dy->data, 16) && dy->stride % 8 == 0 && dy->stride >= dy->cols && dy->rows < (1u << 31) &&
         dy->cols < (1u << 31);
}
int make_map(const dgs_matrix* dy, CUtensorMap* map) {
  const cuuint64_t dims[2] = {dy->cols, dy->rows}, strides[1] = {dy->stride * 2};
  const cuuint32_t box[2] = {64, kRows}, each[2] = {1, 1};
  return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dy->data, dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? DGS_OK
             : DGS_ECUDA;
}

template <class T, bool FLOAT8, bool TMA>
int launch(const WeightArgs& a, const CUtensorMap& map, uint32_t ctas, cudaStream_t st) {
  k_weight_grad<T, FLOAT8, TMA><<<ctas, kThreads, Shape<T>::kSmem, st>>>(a, map);
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
  a.outputs = dy->cols;
  a.code_tiles = p.code_tiles;
  a.grad_tiles = p.grad_tiles;
  a.splits = p.splits;
  a.experts = p.experts;
  a.rows_per = lists ? lists->rows_per : 1;
  a.n = p.n;
  a.in_out = flags & DGS_WEIGHT_IN_OUT ? 1 : 0;
  a.bias_tiles = p.bias_tiles;
  a.offsets = lists ? lists->offsets : nullptr;
  a.rows = lists ? lists->rows : nullptr;
  float* const part_w = static_cast<float*>(workspace);
  float* const part_b = part_w + (p.splits > 1 ? p.nw * p.splits : 0);
  a.dw = p.splits > 1 ? part_w : dw;
  a.db = !db ? nullptr : parts_b > 1 ? part_b : db;
  const uint32_t add = flags & DGS_WEIGHT_ADD ? 1 : 0;
  a.add_w = p.splits == 1 ? add : 0;
  a.add_b = parts_b == 1 ? add : 0;
  a.status = operator_status_word();
  if (!a.status) return DGS_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const uint32_t ctas = p.code_tiles * p.grad_tiles * p.splits * p.experts * 2;
  const bool f8 = ckpt->format == DGS_FORMAT_E4M3;
  CUtensorMap map = {};
  if (tma_fits(dy)) {
    rc = make_map(dy, &map);
    if (rc == DGS_OK) rc = f8 ? launch<__nv_bfloat16, true, true>(a, map, ctas, st) : launch<__nv_bfloat16, false, true>(a, map, ctas, st);
  } else {
    rc = with_type(dy->type, [&](auto* t) {
      using T = std::remove_pointer_t<decltype(t)>;
      return f8 ? launch<T, true, false>(a, map, ctas, st) : launch<T, false, false>(a, map, ctas, st);
    });
  }
  const uint64_t nw = p.splits > 1 ? p.nw : 0, nb = db && parts_b > 1 ? p.nb : 0;
  if (rc != DGS_OK || nw + nb == 0) return rc;
  k_weight_sum<<<uint32_t(std::min<uint64_t>((nw + nb + 255) / 256, kSms * 8)), 256, 0, st>>>(dw, db, part_w, part_b, nw, nb, p.splits, parts_b, add);
  return cudaGetLastError() == cudaSuccess ? DGS_OK : DGS_ECUDA;
}
