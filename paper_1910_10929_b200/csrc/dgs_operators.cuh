// What the operators of a worker's own computation share (dgs_route.cu, dgs_checkpoint.cu, dgs_weight.cu): matrices of the
// caller in three types, the 8-bit format, the status word, and the checks that their host sides make.
#pragma once
#include "dgs.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>
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
  if (!m || m->type > DGS_TYPE_FP16 || m->cols == 0 || m->rows >= (1ull << 32)) return false;
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
  return c && c->format <= DGS_FORMAT_E4M3 && c->cols && c->cols <= (1u << 30) && c->rows < (1ull << 32) &&
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

// Four values to four codes.  The products with a power of two are exact (below the normal numbers they are zero's neighbours
// and round to code 0 all the same), so a code is one rounding to nearest even away from its value.
template <bool FLOAT8>
__device__ __forceinline__ uint32_t encode4(const float* v, float up) {
  if constexpr (FLOAT8) {
    const float2 a = make_float2(v[0] * up, v[1] * up), b = make_float2(v[2] * up, v[3] * up);
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(a, __NV_SATFINITE, __NV_E4M3), hi = __nv_cvt_float2_to_fp8x2(b, __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int q = __float2int_rn(v[i] * up);
      q = q > 127 ? 127 : q < -127 ? -127 : q;   // beyond e = kMax only
      w |= uint32_t(q & 255) << (8 * i);
    }
    return w;
  }
}
// Four codes to four values.
template <bool FLOAT8>
__device__ __forceinline__ void decode4(uint32_t w, float down, float* v) {
  if constexpr (FLOAT8) {
    const __half2 lo(__nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(w & 0xffffu), __NV_E4M3));
    const __half2 hi(__nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(w >> 16), __NV_E4M3));
    const float2 a = __half22float2(lo), b = __half22float2(hi);
    v[0] = a.x * down, v[1] = a.y * down, v[2] = b.x * down, v[3] = b.y * down;
  } else {
    const uint32_t u = w ^ 0x80808080u;   // code + 128 in the low bits of 2^23
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = (__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7650u + i)) - 8388736.0f) * down;
  }
}

__device__ __forceinline__ void report(int* status, int code) { atomicMin(status, code); }

}  // namespace dgs
