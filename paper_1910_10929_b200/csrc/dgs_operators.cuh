// What the operators of a worker's own computation share (dgs_route.cu, dgs_checkpoint.cu, dgs_weight.cu): matrices of the
// caller in three types, the 8-bit format, the status word, and the checks that their host sides make.
#pragma once
#include "dgs.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>
#include <type_traits>

namespace dgs {

// The lowest status that an operator's kernel has left on this device since it was last read (dgs_operator_status).
// Defined in dgs_checkpoint.cu; the other files get its address as a kernel argument.
int* operator_status_word();

constexpr uint32_t kSms = 148;    // of a B200: sizes of grids, nothing that results depend on
constexpr uint32_t kBlock = 32;   // values under one scale byte

// ---- the caller's matrices ------------------------------------------------------------------
template <class T> struct Elem;
template <> struct Elem<float> {
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<__half> {
  static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
};

inline uint32_t elem_bytes(uint32_t type) { return type == DGS_TYPE_F32 ? 4u : 2u; }

// Calls f with a null pointer of the element type.
template <class F>
int with_type(uint32_t type, F&& f) {
  switch (type) {
    case DGS_TYPE_F32: return f(static_cast<float*>(nullptr));
    case DGS_TYPE_BF16: return f(static_cast<__nv_bfloat16*>(nullptr));
    case DGS_TYPE_FP16: return f(static_cast<__half*>(nullptr));
    default: return DGS_EINVAL;
  }
}

// Bytes from the first element to behind the last one.
inline uint64_t span_bytes(const dgs_matrix* m) {
  return m->rows && m->cols ? ((m->rows - 1) * m->stride + m->cols) * elem_bytes(m->type) : 0;
}
inline bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na && nb && x < y + nb && y < x + na;
}
inline bool aligned(const void* p, uint64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

constexpr uint64_t kMostElements = 1ull << 40;   // rows * stride: keeps every byte count far inside 64 bits
// A matrix that a call reads (rows may share one row: stride 0) or writes.
inline bool matrix_ok(const dgs_matrix* m, bool written) {
  if (!m || m->type > DGS_TYPE_FP16 || m->cols == 0 || m->rows >= (1ull << 31)) return false;
  if (m->stride < m->cols && m->rows > 1 && (written || m->stride != 0)) return false;
  if (m->stride && m->rows > kMostElements / m->stride) return false;
  return m->rows == 0 || (m->data && aligned(m->data, elem_bytes(m->type)));
}
inline bool same_matrix(const dgs_matrix* a, const dgs_matrix* b) {
  return a->data == b->data && a->stride == b->stride && a->type == b->type;
}

// ---- the 8-bit format -----------------------------------------------------------------------
// A checkpoint of [rows, cols]: codes [rows][width], then scale bytes [rows][spitch]; width = cols up to a multiple of 32, spitch
// = 4 bytes for each 128 columns begun.  A scale byte is e + 127: the block's values are code * 2^e, e the smallest
// exponent for which the block's largest magnitude is at most kTop * 2^e, kept where every value is a normal bfloat16 number
// (int8: -126 .. 121, e4m3: -117 .. 119).  Power-of-two scales cost at most one bit of an int8 code against free ones;
// they make every decoded value a bfloat16 number exactly, which is what the tensor cores multiply.
struct Held {
  const uint8_t* codes;
  const uint8_t* scales;
  uint64_t rows;
  uint32_t cols, width, spitch;
};
inline uint32_t held_width(uint32_t cols) { return (cols + 31u) / 32u * 32u; }
inline uint32_t held_spitch(uint32_t cols) { return (cols + 127u) / 128u * 4u; }
inline uint64_t held_bytes(uint64_t rows, uint32_t cols) { return rows * (uint64_t(held_width(cols)) + held_spitch(cols)); }
inline Held held_of(const dgs_checkpoint* c) {
  Held h;
  h.codes = static_cast<const uint8_t*>(c->data);
  h.rows = c->rows;
  h.cols = c->cols;
  h.width = held_width(c->cols);
  h.spitch = held_spitch(c->cols);
  h.scales = h.codes + h.rows * h.width;
  return h;
}
inline bool checkpoint_ok(const dgs_checkpoint* c) {
  return c && c->format <= DGS_FORMAT_E4M3 && c->cols && c->cols <= (1u << 30) && c->rows < (1ull << 31) &&
         c->rows <= kMostElements / c->cols && (c->rows == 0 || (c->data && aligned(c->data, 16)));
}

constexpr uint32_t kNanScale = 255;   // a block that held an infinity or a NaN: all of it reads as NaN

template <bool FLOAT8> struct Code {
  static constexpr uint32_t kTopBits = FLOAT8 ? 0x43e00000u : 0x42fe0000u;   // 448 and 127
  static constexpr int kTopExp = FLOAT8 ? 8 : 6;
  static constexpr int kMin = FLOAT8 ? -117 : -126, kMax = FLOAT8 ? 119 : 121;
};

// The scale byte of a block, from the bits of its largest magnitude.
template <bool FLOAT8>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  using K = Code<FLOAT8>;
  if (amax_bits >= 0x7f800000u) return kNanScale;
  // m 2^x <= top 2^e with top = tm 2^tx: e = x - tx, one more where m > tm (subnormal magnitudes end below the clamp either way)
  int e = int(amax_bits >> 23) - 127 - K::kTopExp + ((amax_bits & 0x7fffffu) > (K::kTopBits & 0x7fffffu) ? 1 : 0);
  e = e < K::kMin ? K::kMin : e > K::kMax ? K::kMax : e;
  return uint32_t(e + 127);
}
// 2^-e and 2^e of a scale byte.  Both are normal numbers for every byte that scale_byte gives: e + 127 in 1 .. 248.
__device__ __forceinline__ float scale_up(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float scale_down(uint32_t byte) {
  return byte == kNanScale ? __uint_as_float(0x7fc00000u) : __uint_as_float(byte << 23);
}

__device__ __forceinline__ float hardware_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float hardware_reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two numbers at a time.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(r)) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(r)) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "l"(reinterpret_cast<unsigned long long&>(c)));
  return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// Eight values to eight codes.  The products with a power of two are exact (below the normal numbers they are zero's neighbours
// and round to code 0 all the same), so a code is one rounding to nearest even away from its value.
template <bool FLOAT8>
__device__ __forceinline__ uint2 encode8(const float2 (&v)[4], uint32_t byte) {
  using K = Code<FLOAT8>;
  if (byte == kNanScale) return make_uint2(0, 0);
  const float up = scale_up(byte);
  uint32_t w[2];
  if constexpr (FLOAT8) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      w[h] = __nv_cvt_float2_to_fp8x2(mul2(v[2 * h], both(up)), __NV_SATFINITE, __NV_E4M3) |
             uint32_t(__nv_cvt_float2_to_fp8x2(mul2(v[2 * h + 1], both(up)), __NV_SATFINITE, __NV_E4M3)) << 16;
  } else {
    // 1.5 * 2^23 + q: the addition rounds, and the low byte is the code
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float2 a = mul2(v[2 * h], both(up)), b = mul2(v[2 * h + 1], both(up));
      if (byte == uint32_t(K::kMax + 127)) {   // beyond the largest scale only
        a = make_float2(fminf(fmaxf(a.x, -127.0f), 127.0f), fminf(fmaxf(a.y, -127.0f), 127.0f));
        b = make_float2(fminf(fmaxf(b.x, -127.0f), 127.0f), fminf(fmaxf(b.y, -127.0f), 127.0f));
      }
      a = add2(a, both(12582912.0f));
      b = add2(b, both(12582912.0f));
      w[h] = __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040), __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
    }
  }
  return make_uint2(w[0], w[1]);
}
// Eight codes to eight values.
template <bool FLOAT8>
__device__ __forceinline__ void decode8(uint2 w, float down, float2 (&v)[4]) {
  const uint32_t c[2] = {w.x, w.y};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (FLOAT8) {
      const __half2 lo(__nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(c[h] & 0xffffu), __NV_E4M3));
      const __half2 hi(__nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(c[h] >> 16), __NV_E4M3));
      v[2 * h] = mul2(__half22float2(lo), both(down));
      v[2 * h + 1] = mul2(__half22float2(hi), both(down));
    } else {
      const uint32_t u = c[h] ^ 0x80808080u;   // code + 128 in the low bits of 2^23
      const float2 a = make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7650)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7651)));
      const float2 b = make_float2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7652)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7653)));
      v[2 * h] = mul2(add2(a, both(-8388736.0f)), both(down));
      v[2 * h + 1] = mul2(add2(b, both(-8388736.0f)), both(down));
    }
  }
}

// Eight numbers of a type, and as floats.
template <class T> struct Eight {
  uint32_t w[sizeof(T) * 2];
};
__device__ __forceinline__ void floats_of(const Eight<float>& e, float2 (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(e.w[2 * i]), __uint_as_float(e.w[2 * i + 1]));
}
__device__ __forceinline__ void floats_of(const Eight<__nv_bfloat16>& e, float2 (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(e.w[i] << 16), __uint_as_float(e.w[i] & 0xffff0000u));
}
__device__ __forceinline__ void floats_of(const Eight<__half>& e, float2 (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __half2 h;
    memcpy(&h, &e.w[i], 4);
    v[i] = __half22float2(h);
  }
}
__device__ __forceinline__ void of_floats(const float2 (&v)[4], Eight<float>& e) {
#pragma unroll
  for (int i = 0; i < 4; ++i) e.w[2 * i] = __float_as_uint(v[i].x), e.w[2 * i + 1] = __float_as_uint(v[i].y);
}
__device__ __forceinline__ void of_floats(const float2 (&v)[4], Eight<__nv_bfloat16>& e) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __float22bfloat162_rn(v[i]);
    memcpy(&e.w[i], &b, 4);
  }
}
__device__ __forceinline__ void of_floats(const float2 (&v)[4], Eight<__half>& e) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 b = __float22half2_rn(v[i]);
    memcpy(&e.w[i], &b, 4);
  }
}
// The bits of the largest magnitude as a float; infinities and NaN are larger than all others.
__device__ __forceinline__ uint32_t largest_bits(const Eight<float>& e) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, e.w[i] & 0x7fffffffu);
  return m;
}
template <class T>
__device__ __forceinline__ uint32_t largest_half(const Eight<T>& e) {
  uint32_t m = e.w[0] & 0x7fff7fffu;
#pragma unroll
  for (int i = 1; i < 4; ++i) m = __vmaxu2(m, e.w[i] & 0x7fff7fffu);
  return max(m >> 16, m & 0xffffu);
}
__device__ __forceinline__ uint32_t largest_bits(const Eight<__nv_bfloat16>& e) { return largest_half(e) << 16; }
__device__ __forceinline__ uint32_t largest_bits(const Eight<__half>& e) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)largest_half(e)))); }

// Kernels of one call follow one another with their beginnings overlapped (programmatic launches).  wait_for_last_kernel: what the kernel ahead wrote is
// there, and all before it; let_next_kernel_begin: the next may be brought onto the SMs.
__device__ __forceinline__ void wait_for_last_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
struct EarlyLaunch {
  cudaLaunchAttribute early;
  cudaLaunchConfig_t cfg;
  EarlyLaunch(dim3 grid, uint32_t threads, uint32_t smem, cudaStream_t st) {
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
  }
  EarlyLaunch(const EarlyLaunch&) = delete;
};

__device__ __forceinline__ void report(int* status, int code) { atomicMin(status, code); }

}  // namespace dgs
