// Weight and bias gradients from checkpoints in 8 bits: dgs_checkpoint_weight_grad.
#include "dgs_operators.cuh"

#include <algorithm>
#include <cstring>
#include <mutex>

namespace dgs {
namespace {

// ---- tcgen05, mbarriers -------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_at(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
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
__device__ __forceinline__ void writes_to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tmem_alloc(uint32_t* slot, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(slot)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b),
      "r"(idesc), "r"(uint32_t(add))
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
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
__device__ __forceinline__ float tmem_load1(uint32_t at) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
  return __uint_as_float(r);
}

// ---- tiles in shared memory ---------------------------------------------------------------------
// Both operands are contracted over their rows, so both lie in memory with the other dimension contiguous, and stay so: a tile of
// 64 rows is cut into blocks of 64 columns, each 64 rows of 128 bytes with the 16-byte pieces of a row exchanged by the row's
// number (128-byte swizzle).  Descriptor: blocks of 64 columns 8192 bytes apart, groups of 8 rows 1024 bytes apart.
constexpr uint32_t kRows = 64;                 // rows of a step
constexpr uint32_t kColBlock = kRows * 128;    // bytes of 64 columns
constexpr uint32_t kCodeCols = 128;            // inputs of a tile
__device__ __forceinline__ uint32_t tile_at(uint32_t row, uint32_t piece) {   // piece: eight columns
  return (piece >> 3) * kColBlock + row * 128 + (((piece ^ row) & 7) << 4);
}
__device__ __forceinline__ uint64_t tile_desc(uint32_t at) {
  return uint64_t(at >> 4 & 0x3fff) | uint64_t(kColBlock >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// 16 x 16 ones, no swizzle: four 8 x 8 pieces of 128 bytes
__device__ __forceinline__ uint64_t ones_desc(uint32_t at) {
  return uint64_t(at >> 4 & 0x3fff) | uint64_t(128 >> 4) << 16 | uint64_t(256 >> 4) << 32 | uint64_t(1) << 46;
}
constexpr uint32_t kIdesc = 1u << 4 | 1u << 7 | 1u << 10 | (128u >> 4) << 24;   // f32 += bf16 x bf16, 128 rows
constexpr uint32_t kIdescA = 1u << 15, kIdescB = 1u << 16;                         // that operand lies as above
__host__ __device__ constexpr uint32_t idesc_cols(uint32_t n) { return (n >> 3) << 17; }

// A gradient's type: how many bfloat16 numbers add up to one of its values, and how many outputs a tile then takes.
template <class T> struct Grad;
template <> struct Grad<__nv_bfloat16> { static constexpr uint32_t kParts = 1, kCols = 256, kStages = 4; };
template <> struct Grad<__half> { static constexpr uint32_t kParts = 2, kCols = 128, kStages = 4; };
template <> struct Grad<float> { static constexpr uint32_t kParts = 3, kCols = 128, kStages = 3; };

template <class T> struct Shape {
  static constexpr uint32_t kCodeBytes = kCodeCols / 64 * kColBlock;
  static constexpr uint32_t kPartBytes = Grad<T>::kCols / 64 * kColBlock;
  static constexpr uint32_t kStage = kCodeBytes + Grad<T>::kParts * kPartBytes;
  static constexpr uint32_t kSmem = 1024 + Grad<T>::kStages * kStage;
  static constexpr uint32_t kUnits = kRows * (Grad<T>::kCols / 8) / 256;   // pieces of the gradient's tile per thread
};
constexpr uint32_t kTmemCols = 512;

struct WeightArgs {
  Held h;
  const void* dy;
  uint64_t dy_rows, dy_stride;
  uint32_t outputs, code_tiles, grad_tiles, splits, experts, rows_per;
  const uint32_t* offsets;
  const uint32_t* rows;
  float* dw;          // or the splits' partial results, [splits][experts][inputs * outputs]
  float* db;          // likewise, [splits][experts][outputs]; NULL: not wanted
  uint32_t add;
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
__device__ __forceinline__ void grads_store(const Eight<T>& r, uint32_t at, uint32_t part_bytes) {
  constexpr uint32_t P = Grad<T>::kParts;
  uint32_t out[P][4];
  if constexpr (P == 1) {
    const uint4 w = grads_words(r);
    out[0][0] = w.x, out[0][1] = w.y, out[0][2] = w.z, out[0][3] = w.w;
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
// A CTA forms a tile of 128 inputs x 256 outputs (128 for gradients of several parts) over a run of an expert's rows, 64 rows a step.
// Eight warps bring the operands to shared memory, the codes decoded; a ninth issues the products; then the eight write the
// accumulators out.  The dimension of dw that is contiguous in memory goes on the accumulators' lanes, so that a warp's stores are
// coalesced wherever the layer's slice begins: inputs for [outputs][inputs], outputs for [inputs][outputs].  The tiles are the same for
// either, only their roles are exchanged.  db comes from products of the gradient's tile with ones, in the CTAs of the first inputs.
template <class T, bool FLOAT8>
__global__ void __launch_bounds__(288, 1) k_weight_grad(const __grid_constant__ WeightArgs a, uint32_t in_out) {
  using S = Shape<T>;
  constexpr uint32_t P = Grad<T>::kParts, GC = Grad<T>::kCols, ST = Grad<T>::kStages;
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t s_full[ST], s_empty[ST], s_done;
  __shared__ uint32_t s_tmem;
  __shared__ __align__(128) uint32_t s_ones[128];
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t tiles = (smem_at(raw) + 1023u) & ~1023u;

  uint32_t b = blockIdx.x;
  const uint32_t ct = b % a.code_tiles;
  b /= a.code_tiles;
  const uint32_t gt = b % a.grad_tiles;
  b /= a.grad_tiles;
  const uint32_t split = b % a.splits, expert = b / a.splits;
  const uint32_t i0 = ct * kCodeCols, o0 = gt * GC;

  uint64_t first = 0, last = a.dy_rows;
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
  const uint32_t steps = uint32_t((last - first + kRows - 1) / kRows);
  const bool bias = a.db != nullptr && ct == 0;

  if (warp == 8) {
    tmem_alloc(&s_tmem, kTmemCols);
    if (lane == 0) {
      for (uint32_t s = 0; s < ST; ++s) {
        bar_init(smem_at(&s_full[s]), 8);
        bar_init(smem_at(&s_empty[s]), 1);
      }
      bar_init(smem_at(&s_done), 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
  }
  if (tid < 128) s_ones[tid] = 0x3f803f80u;
  writes_to_async_proxy();
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = s_tmem;

  if (warp == 8) {
    if (lane == 0 && steps) {
      const uint32_t ones = smem_at(s_ones);
      bool alive = true;
      for (uint32_t s = 0; s < steps && alive; ++s) {
        const uint32_t st = s % ST, code = tiles + st * S::kStage, grad = code + S::kCodeBytes;
        alive = bar_wait(smem_at(&s_full[st]), s / ST & 1);
        if (!alive) break;
        tmem_after();
#pragma unroll
        for (uint32_t k = 0; k < kRows / 16; ++k) {
          const uint64_t cd = tile_desc(code + k * 2048);
#pragma unroll
          for (uint32_t p = 0; p < P; ++p) {
            const uint32_t g = grad + p * S::kPartBytes + k * 2048;
            const bool more = s || k || p;
            if (!in_out) {
              mma(tmem, cd, tile_desc(g), kIdesc | kIdescA | kIdescB | idesc_cols(GC), more);
            } else {
#pragma unroll
              for (uint32_t h = 0; h < GC / 128; ++h)
                mma(tmem + h * 128, tile_desc(g + h * 2 * kColBlock), cd, kIdesc | kIdescA | kIdescB | idesc_cols(kCodeCols), more);
            }
            if (bias)
#pragma unroll
              for (uint32_t h = 0; h < GC / 128; ++h)
                mma(tmem + GC + h * 16, tile_desc(g + h * 2 * kColBlock), ones_desc(ones), kIdesc | kIdescA | idesc_cols(16), more);
          }
        }
        mma_commit(smem_at(&s_empty[st]));
      }
      if (!alive) report(a.status, DGS_ETIMEOUT);
      mma_commit(smem_at(&s_done));
    }
  } else {
    const T* dy = static_cast<const T*>(a.dy);
    const T* dy_end = dy + ((a.dy_rows - 1) * a.dy_stride + a.outputs);   // read where dy_rows > 0 only
    uint4 code[2];
    uint32_t scale[2];
    Eight<T> grad[S::kUnits];
    auto load = [&](uint32_t s) {
      const uint64_t j0 = first + uint64_t(s) * kRows;
#pragma unroll
      for (uint32_t u = 0; u < 2; ++u) {
        const uint32_t id = tid + 256 * u, r = id / 8, v = id % 8;
        const uint64_t j = j0 + r;
        const uint32_t col = i0 + v * 16;
        code[u] = make_uint4(0, 0, 0, 0);
        scale[u] = 0;
        if (j < last && col < a.h.width) {
          uint64_t src = j;
          if (a.rows) src = a.rows[j] / a.rows_per;
          if (src < a.h.rows) {
            code[u] = __ldg(reinterpret_cast<const uint4*>(a.h.codes + src * a.h.width + col));
            scale[u] = __ldg(a.h.scales + src * a.h.spitch + col / 32);
          } else {
            report(a.status, DGS_EINVAL);
          }
        }
      }
#pragma unroll
      for (uint32_t u = 0; u < S::kUnits; ++u) {
        const uint32_t id = tid + 256 * u, r = id / (GC / 8), piece = id % (GC / 8);
        const uint64_t j = j0 + r;
        const uint32_t col = o0 + piece * 8;
        grads_load<T>(grad[u], dy + j * a.dy_stride + col, j < last && col < a.outputs ? a.outputs - col : 0, dy, dy_end);
      }
    };
    bool alive = true;
    if (steps) load(0);
    for (uint32_t s = 0; s < steps; ++s) {
      const uint32_t st = s % ST, at = tiles + st * S::kStage;
      if (s >= ST && !bar_wait(smem_at(&s_empty[st]), (s / ST - 1) & 1)) {
        alive = false;
        break;
      }
#pragma unroll
      for (uint32_t u = 0; u < 2; ++u) {
        const uint32_t id = tid + 256 * u, r = id / 8, v = id % 8;
        const uint32_t sc = scale_bf2(scale[u]);
        const uint4 x = codes_bf8<FLOAT8>(code[u].x, code[u].y, sc), y = codes_bf8<FLOAT8>(code[u].z, code[u].w, sc);
        const bool swap = v >= 4;   // the halves of a row go to the same banks: one writes its second piece first
        const uint4 p = swap ? y : x, q = swap ? x : y;
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + tile_at(r, 2 * v + swap)), "r"(p.x), "r"(p.y), "r"(p.z), "r"(p.w) : "memory");
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + tile_at(r, 2 * v + !swap)), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
      }
#pragma unroll
      for (uint32_t u = 0; u < S::kUnits; ++u) {
        const uint32_t id = tid + 256 * u, r = id / (GC / 8), piece = id % (GC / 8);
        grads_store<T>(grad[u], at + S::kCodeBytes + tile_at(r, piece), S::kPartBytes);
      }
      if (s + 1 < steps) load(s + 1);
      writes_to_async_proxy();
      __syncwarp();
      if (lane == 0) bar_arrive(smem_at(&s_full[st]));
    }
    if (alive && steps) alive = bar_wait(smem_at(&s_done), 0);
    if (!alive && lane == 0) report(a.status, DGS_ETIMEOUT);
    tmem_after();
    // accumulators to memory: warps 0-3 the first half of the columns, 4-7 the second
    const uint32_t quarter = warp % 4, half = warp / 4, row = quarter * 32 + lane;
    const uint32_t inputs = a.h.cols;
    const uint64_t one = uint64_t(inputs) * a.outputs;
    float* dw = a.dw + (uint64_t(split) * a.experts + expert) * one;
    for (uint32_t c0 = half * (GC / 2); c0 < (half + 1) * (GC / 2); c0 += 32) {
      const uint32_t lane_at = in_out ? o0 + c0 / 128 * 128 + row : i0 + row, lane_end = in_out ? a.outputs : inputs;
      const uint32_t col_at = in_out ? i0 + c0 % 128 : o0 + c0, col_end = in_out ? inputs : a.outputs;
      if (col_at >= col_end || lane_at - lane >= lane_end) continue;   // the whole warp
      float v[32];
      if (steps) {
        tmem_load32(tmem + (quarter * 32 << 16) + c0, v);
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = 0.0f;
      }
      if (lane_at < lane_end && alive) {
        float* p = dw + uint64_t(col_at) * lane_end + lane_at;
        if (a.add) {
          float old[32];
#pragma unroll
          for (uint32_t i = 0; i < 32; ++i) old[i] = col_at + i < col_end ? p[uint64_t(i) * lane_end] : 0.0f;
#pragma unroll
          for (uint32_t i = 0; i < 32; ++i) v[i] += old[i];
        }
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i)
          if (col_at + i < col_end) p[uint64_t(i) * lane_end] = v[i];
      }
    }
    if (bias && half < GC / 128) {
      const float v = steps ? tmem_load1(tmem + (quarter * 32 << 16) + GC + half * 16) : 0.0f;
      const uint32_t o = o0 + half * 128 + row;
      if (o < a.outputs && alive) {
        float* p = a.db + (uint64_t(split) * a.experts + expert) * a.outputs + o;
        *p = a.add ? *p + v : v;
      }
    }
    tmem_before();
  }
  __syncthreads();
  if (warp == 8) {
    __syncwarp();
    tmem_after();
    tmem_free(tmem, kTmemCols);
  }
}

// Adds up the splits' partial results in their order.
__global__ void __launch_bounds__(256) k_weight_sum(float* dw, float* db, const float* pw, const float* pb, uint64_t nw, uint64_t nb, uint32_t splits, uint32_t add) {
  const uint64_t total = nw + (db ? nb : 0);
  for (uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += uint64_t(gridDim.x) * 256) {
    const bool w = i < nw;
    const uint64_t k = w ? i : i - nw, n = w ? nw : nb;
    const float* p = (w ? pw : pb) + k;
    float* out = (w ? dw : db) + k;
    float v = 0.0f;
    for (uint32_t s = 0; s < splits; ++s) v += p[s * n];
    *out = add ? *out + v : v;
  }
}

// ---- host side --------------------------------------------------------------------------------
struct WeightPlan {
  uint32_t code_tiles, grad_tiles, splits, experts;
  uint64_t nw, nb, bytes;
};

bool lists_ok(const dgs_row_lists* l) {
  return !l || (l->offsets && l->experts && l->experts <= 65535 && l->rows_per && aligned(l->offsets, 4) && aligned(l->rows, 4));
}

int plan_weight(const dgs_checkpoint* c, const dgs_matrix* dy, const dgs_row_lists* lists, WeightPlan* p) {
  if (!checkpoint_ok(c) || !matrix_ok(dy, false) || !lists_ok(lists) || (!lists && dy->rows != c->rows)) return DGS_EINVAL;
  const uint32_t cols = dy->type == DGS_TYPE_BF16 ? Grad<__nv_bfloat16>::kCols : Grad<float>::kCols;
  const uint32_t parts = dy->type == DGS_TYPE_BF16 ? 1 : dy->type == DGS_TYPE_FP16 ? 2 : 3;
  p->experts = lists ? lists->experts : 1;
  p->code_tiles = (c->cols + kCodeCols - 1) / kCodeCols;
  p->grad_tiles = uint32_t((uint64_t(dy->cols) + cols - 1) / cols);
  if (uint64_t(c->cols) * dy->cols > kMostElements / p->experts) return DGS_ELIMIT;
  p->nw = uint64_t(c->cols) * dy->cols * p->experts;
  p->nb = uint64_t(dy->cols) * p->experts;
  const uint64_t tiles = uint64_t(p->code_tiles) * p->grad_tiles * p->experts;
  if (tiles > 0x7fffffffu / 64) return DGS_ELIMIT;
  // Rows of a tile are split among CTAs where that ends sooner: rounds of 148 CTAs times (steps of a CTA, 0.28 us each for one part, and about 4 us
  // around them), and the partial results' way through the second cache.
  const double steps = double((dy->rows / p->experts + kRows - 1) / kRows), step_us = 0.28 * parts * cols / 256;
  double best = 0;
  p->splits = 1;
  for (uint32_t s = 1; s <= 32 && s <= std::max(1.0, steps); ++s) {
    const double rounds = double((tiles * s + kSms - 1) / kSms);
    const double us = rounds * (std::max(1.0, double(uint64_t((steps + s - 1) / s))) * step_us + 4.0) + (s > 1 ? 3.0 + double(p->nw) * 8e-6 * s / 3.0 : 0.0);
    if (s == 1 || us < best) best = us, p->splits = s;
  }
  p->bytes = p->splits > 1 ? (p->nw + p->nb) * p->splits * 4 : 0;
  return DGS_OK;
}

constexpr int kMaxDevices = 64;
std::mutex g_weight_mu;
bool g_weight_ready[kMaxDevices];
template <class T>
bool weight_setup() {
  return cudaFuncSetAttribute(k_weight_grad<T, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<T>::kSmem) == cudaSuccess &&
         cudaFuncSetAttribute(k_weight_grad<T, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<T>::kSmem) == cudaSuccess;
}
int weight_ready() {   // once per device
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return DGS_ECUDA;
  std::lock_guard<std::mutex> lock(g_weight_mu);
  if (!g_weight_ready[dev]) {
    if (!weight_setup<float>() || !weight_setup<__nv_bfloat16>() || !weight_setup<__half>()) return DGS_ECUDA;
    g_weight_ready[dev] = true;
  }
  return DGS_OK;
}

}  // namespace
}  // namespace dgs

using namespace dgs;

extern "C" int dgs_checkpoint_weight_grad_bytes(const dgs_checkpoint* ckpt, const dgs_matrix* dy, const dgs_row_lists* lists, uint32_t flags,
                                                uint64_t* out_bytes) {
  WeightPlan p;
  if (!out_bytes || (flags & ~(DGS_WEIGHT_IN_OUT | DGS_WEIGHT_ADD))) return DGS_EINVAL;
  const int rc = plan_weight(ckpt, dy, lists, &p);
  if (rc == DGS_OK) *out_bytes = p.bytes;
  return rc;
}

extern "C" int dgs_checkpoint_weight_grad(const dgs_checkpoint* ckpt, const dgs_matrix* dy, const dgs_row_lists* lists, float* dw, float* db,
                                          uint32_t flags, void* workspace, uint64_t workspace_bytes, void* stream) {
  WeightPlan p;
  if (flags & ~(DGS_WEIGHT_IN_OUT | DGS_WEIGHT_ADD)) return DGS_EINVAL;
  int rc = plan_weight(ckpt, dy, lists, &p);
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
  a.offsets = lists ? lists->offsets : nullptr;
  a.rows = lists ? lists->rows : nullptr;
  float* const part_w = static_cast<float*>(workspace);
  float* const part_b = part_w + p.nw * p.splits;
  a.dw = p.splits > 1 ? part_w : dw;
  a.db = !db ? nullptr : p.splits > 1 ? part_b : db;
  a.add = p.splits == 1 && (flags & DGS_WEIGHT_ADD);
  a.status = operator_status_word();
  if (!a.status) return DGS_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const uint32_t ctas = uint32_t(uint64_t(p.code_tiles) * p.grad_tiles * p.splits * p.experts), in_out = flags & DGS_WEIGHT_IN_OUT ? 1 : 0;
  rc = with_type(dy->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    if (ckpt->format == DGS_FORMAT_E4M3)
      k_weight_grad<T, true><<<ctas, 288, Shape<T>::kSmem, st>>>(a, in_out);
    else
      k_weight_grad<T, false><<<ctas, 288, Shape<T>::kSmem, st>>>(a, in_out);
    return cudaGetLastError() == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
  });
  if (rc != DGS_OK || p.splits == 1) return rc;
  const uint64_t sums = p.nw + (db ? p.nb : 0);
  k_weight_sum<<<uint32_t(std::min<uint64_t>((sums + 255) / 256, kSms * 8)), 256, 0, st>>>(dw, db, part_w, part_b, p.nw, p.nb, p.splits,
                                                                                      flags & DGS_WEIGHT_ADD ? 1 : 0);
  return cudaGetLastError() == cudaSuccess ? DGS_OK : DGS_ECUDA;
}
