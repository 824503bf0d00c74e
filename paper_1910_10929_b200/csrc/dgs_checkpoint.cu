// Activations held in 8 bits: dgs_checkpoint_save, _load and _activation_grad, and the operators' status word.
#include "dgs_operators.cuh"

#include <algorithm>

namespace dgs {
namespace {

__device__ int g_operator_status;

// ---- activations and their slopes -------------------------------------------------------------
// FAST is for results of 16 bits: the exponential and division of the hardware are off by 2^-20 at most where it counts, a rounding of the
// result by 2^-9 or 2^-12.  (32768 x 2048 in bfloat16, gelu_tanh: 125 us exact, see the kernels for what it takes now.)
template <bool FAST> __device__ __forceinline__ float exponential(float x) { return FAST ? __expf(x) : expf(x); }
template <bool FAST> __device__ __forceinline__ float quotient(float a, float b) { return FAST ? __fdividef(a, b) : a / b; }
// s = 1 / (1 + e^-u) and t = 1 - s, both from e^-|u|, which does not overflow: neither loses digits to the other.
template <bool FAST> struct Sigmoid {
  float s, t;
  __device__ __forceinline__ explicit Sigmoid(float u) {
    const float q = exponential<FAST>(-fabsf(u)), r = quotient<FAST>(1.0f, 1.0f + q), p = q * r;
    s = u > 0.0f ? r : p;
    t = u > 0.0f ? p : r;
  }
};
template <int ACT, bool FAST>
__device__ __forceinline__ float act_value(float x) {
  if constexpr (ACT == DGS_ACT_RELU) return x > 0.0f ? x : (x != x ? x : 0.0f);
  if constexpr (ACT == DGS_ACT_SILU) return x * Sigmoid<FAST>(x).s;
  if constexpr (ACT == DGS_ACT_GELU) return 0.5f * x * erfcf(-x * 0.70710678f);
  if constexpr (ACT == DGS_ACT_GELU_TANH) return x * Sigmoid<FAST>(1.5957691f * x * fmaf(0.044715f * x, x, 1.0f)).s;
  return x;
}
// d act / d x.  With s = 1 / (1 + e^-u): silu u = x, slope s (1 + x (1 - s)); gelu_tanh is x s(u), u = 2 sqrt(2/pi) (x + 0.044715 x^3),
// slope s + x u' s (1 - s).
template <int ACT, bool FAST>
__device__ __forceinline__ float act_slope(float x) {
  if constexpr (ACT == DGS_ACT_RELU) return x > 0.0f ? 1.0f : (x != x ? x : 0.0f);
  if constexpr (ACT == DGS_ACT_GELU) return fmaf(0.3989422804f * x, exponential<FAST>(-0.5f * x * x), 0.5f * erfcf(-x * 0.70710678f));
  if constexpr (ACT == DGS_ACT_SILU) {
    const Sigmoid<FAST> g(x);
    return g.s * fmaf(x, g.t, 1.0f);
  }
  if constexpr (ACT == DGS_ACT_GELU_TANH) {
    x = x > 30.0f ? 30.0f : x < -30.0f ? -30.0f : x;   // from there on 0 or 1; cubes beyond would overflow
    const float x2 = x * x, u = 1.5957691f * x * fmaf(0.044715f, x2, 1.0f), du = 1.5957691f * fmaf(0.134145f, x2, 1.0f);
    const Sigmoid<FAST> g(u);
    return g.s * fmaf(x * du, g.t, 1.0f);
  }
  return 1.0f;
}

// ---- eight columns at a time ------------------------------------------------------------------
// A unit is eight columns of a row; four lanes next to one another hold a block.  VEC: rows begin on 16 bytes, so that a unit is one
// or two wide accesses; otherwise it is read and written element by element (odd lengths and strides).  Units are read some at a time, so that
// a thread has several reads under way, and stay in their type until they are used.
template <class T> struct Eight {
  T v[8];
};
template <bool VEC, class T>
__device__ __forceinline__ void read8(const T* p, uint32_t left, Eight<T>& e) {
  if (VEC && left >= 8) {
    uint4 w[sizeof(T) / 2];
#pragma unroll
    for (uint32_t i = 0; i < sizeof(T) / 2; ++i) w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    memcpy(e.v, w, sizeof(w));
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) e.v[i] = uint32_t(i) < left ? p[i] : Elem<T>::put(0.0f);
}
template <bool VEC, class T>
__device__ __forceinline__ void write8(T* p, uint32_t left, const float* v) {
  Eight<T> e;
#pragma unroll
  for (int i = 0; i < 8; ++i) e.v[i] = Elem<T>::put(v[i]);
  if (VEC && left >= 8) {
    uint4 w[sizeof(T) / 2];
    memcpy(w, e.v, sizeof(w));
#pragma unroll
    for (uint32_t i = 0; i < sizeof(T) / 2; ++i) __stcs(reinterpret_cast<uint4*>(p) + i, w[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (uint32_t(i) < left) p[i] = e.v[i];
}

struct Units {
  uint64_t rows;
  uint32_t per_row;        // units of a row: width / 8
  uint64_t step_rows;      // what one stride of the grid is in rows and units
  uint32_t step_units;
};

// Walks the units of all rows, a stride of the grid apart, N at a time: load(i, row, unit) for each, then done(i, row, unit).
template <int N, class L, class D>
__device__ __forceinline__ void each_unit(const Units& g, L&& load, D&& done) {
  const uint64_t first = uint64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  uint64_t row = first / g.per_row;
  uint32_t unit = uint32_t(first - row * g.per_row);
  while (row < g.rows) {
    uint64_t r[N];
    uint32_t u[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      r[i] = row;
      u[i] = unit;
      if (row < g.rows) load(i, row, unit);
      row += g.step_rows;
      unit += g.step_units;
      if (unit >= g.per_row) unit -= g.per_row, ++row;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (r[i] < g.rows) done(i, r[i], u[i]);
  }
}
template <class T> constexpr int kAtOnce = sizeof(T) == 2 ? 4 : 2;

template <class T, bool FLOAT8, bool VEC, int ACT>
__global__ void __launch_bounds__(256) k_checkpoint_save(Held h, uint8_t* codes, uint8_t* scales, const T* x, uint64_t xs, T* y, uint64_t ys, Units g) {
  constexpr int N = kAtOnce<T>;
  Eight<T> in[N];
  each_unit<N>(
      g,
      [&](int i, uint64_t row, uint32_t unit) {
        const uint32_t col = unit * 8;
        read8<VEC>(x + row * xs + col, col < h.cols ? h.cols - col : 0, in[i]);
      },
      [&](int i, uint64_t row, uint32_t unit) {
        const uint32_t col = unit * 8, left = col < h.cols ? h.cols - col : 0;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = Elem<T>::get(in[i].v[k]);
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(v[k]) & 0x7fffffffu);
        const uint32_t lanes = 0xfu << (threadIdx.x & 28u);   // the four lanes of the block: rows are a multiple of four units
        m = max(m, __shfl_xor_sync(lanes, m, 1));
        m = max(m, __shfl_xor_sync(lanes, m, 2));
        const uint32_t byte = scale_byte<FLOAT8>(m);
        const float up = byte == kNanScale ? 0.0f : scale_up(byte);
        uint2 w = make_uint2(encode4<FLOAT8>(v, up), encode4<FLOAT8>(v + 4, up));
        if (byte == kNanScale) w = make_uint2(0, 0);
        *reinterpret_cast<uint2*>(codes + row * h.width + col) = w;
        if (unit % 4 == 0) {
          uint8_t* s = scales + row * h.spitch + unit / 4;
          *s = uint8_t(byte);
          if (unit + 4 == g.per_row)
            for (uint32_t b = g.per_row / 4; b < h.spitch; ++b) *++s = 0;
        }
        if (y) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = act_value<ACT, sizeof(T) == 2>(v[k]);
          write8<VEC>(y + row * ys + col, left, v);
        }
      });
}

struct HeldUnit {
  uint2 w;
  uint32_t scale;
};
__device__ __forceinline__ void read_held(const Held& h, uint64_t row, uint32_t unit, HeldUnit& u) {
  u.w = __ldg(reinterpret_cast<const uint2*>(h.codes + row * h.width + unit * 8));
  u.scale = __ldg(h.scales + row * h.spitch + unit / 4);
}
template <bool FLOAT8>
__device__ __forceinline__ void decode8(const HeldUnit& u, float* v) {
  const float down = scale_down(u.scale);
  decode4<FLOAT8>(u.w.x, down, v);
  decode4<FLOAT8>(u.w.y, down, v + 4);
}

template <class T, bool FLOAT8, bool VEC>
__global__ void __launch_bounds__(256) k_checkpoint_load(Held h, T* x, uint64_t xs, Units g) {
  HeldUnit in[4];
  each_unit<4>(
      g, [&](int i, uint64_t row, uint32_t unit) { read_held(h, row, unit, in[i]); },
      [&](int i, uint64_t row, uint32_t unit) {
        const uint32_t col = unit * 8;
        if (col >= h.cols) return;
        float v[8];
        decode8<FLOAT8>(in[i], v);
        write8<VEC>(x + row * xs + col, h.cols - col, v);
      });
}

template <class T, bool FLOAT8, bool VEC, int ACT>
__global__ void __launch_bounds__(256) k_activation_grad(Held h, const T* dy, uint64_t dys, T* dx, uint64_t dxs, Units g) {
  constexpr int N = kAtOnce<T>;
  HeldUnit in[N];
  Eight<T> d[N];
  each_unit<N>(
      g,
      [&](int i, uint64_t row, uint32_t unit) {
        const uint32_t col = unit * 8;
        read_held(h, row, unit, in[i]);
        read8<VEC>(dy + row * dys + col, col < h.cols ? h.cols - col : 0, d[i]);
      },
      [&](int i, uint64_t row, uint32_t unit) {
        const uint32_t col = unit * 8;
        if (col >= h.cols) return;
        float v[8];
        decode8<FLOAT8>(in[i], v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = Elem<T>::get(d[i].v[k]) * act_slope<ACT, sizeof(T) == 2>(v[k]);
        write8<VEC>(dx + row * dxs + col, h.cols - col, v);
      });
}

// ---- host side --------------------------------------------------------------------------------
struct Plan {
  Units g;
  uint32_t ctas;
};
void plan_units(uint64_t rows, uint32_t width, Plan* p) {
  p->g.rows = rows;
  p->g.per_row = width / 8;
  const uint64_t units = rows * p->g.per_row;
  p->ctas = uint32_t(std::min<uint64_t>((units + 255) / 256, uint64_t(kSms) * 8));
  const uint64_t step = uint64_t(p->ctas) * 256;
  p->g.step_rows = step / p->g.per_row;
  p->g.step_units = uint32_t(step % p->g.per_row);
}

template <class T>
bool wide(const dgs_matrix* m) {
  return aligned(m->data, 16) && m->stride * sizeof(T) % 16 == 0;
}

template <class F>
int with_act(int act, F&& f) {
  switch (act) {
    case DGS_ACT_NONE: return f(std::integral_constant<int, DGS_ACT_NONE>());
    case DGS_ACT_RELU: return f(std::integral_constant<int, DGS_ACT_RELU>());
    case DGS_ACT_GELU: return f(std::integral_constant<int, DGS_ACT_GELU>());
    case DGS_ACT_GELU_TANH: return f(std::integral_constant<int, DGS_ACT_GELU_TANH>());
    case DGS_ACT_SILU: return f(std::integral_constant<int, DGS_ACT_SILU>());
    default: return DGS_EINVAL;
  }
}
template <class F>
int with_bool(bool b, F&& f) {
  return b ? f(std::true_type()) : f(std::false_type());
}

bool fits(const dgs_checkpoint* c, const dgs_matrix* m, bool written) {
  return matrix_ok(m, written) && m->rows == c->rows && m->cols == c->cols &&
         !overlap(m->data, span_bytes(m), c->data, held_bytes(c->rows, c->cols));
}

}  // namespace

int* operator_status_word() {
  void* p = nullptr;
  return cudaGetSymbolAddress(&p, g_operator_status) == cudaSuccess ? static_cast<int*>(p) : nullptr;
}

}  // namespace dgs

using namespace dgs;

extern "C" int dgs_checkpoint_bytes(uint64_t rows, uint32_t cols, uint64_t* out_bytes) {
  if (!out_bytes || cols == 0 || cols > (1u << 30) || rows >= (1ull << 32) || rows > kMostElements / cols) return DGS_EINVAL;
  *out_bytes = held_bytes(rows, cols);
  return DGS_OK;
}

extern "C" int dgs_checkpoint_save(const dgs_checkpoint* ckpt, const dgs_matrix* x, int act, const dgs_matrix* y, void* stream) {
  if (!checkpoint_ok(ckpt) || !x || !fits(ckpt, x, false) || act < 0 || act > DGS_ACT_SILU) return DGS_EINVAL;
  if (y && (!fits(ckpt, y, true) || y->type != x->type ||
            (!same_matrix(x, y) && overlap(x->data, span_bytes(x), y->data, span_bytes(y)))))
    return DGS_EINVAL;
  if (ckpt->rows == 0) return DGS_OK;
  const Held h = held_of(ckpt);
  Plan p;
  plan_units(h.rows, h.width, &p);
  return with_type(x->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return with_bool(ckpt->format == DGS_FORMAT_E4M3, [&](auto f8) {
      return with_bool(wide<T>(x) && (!y || wide<T>(y)), [&](auto vec) {
        return with_act(y ? act : DGS_ACT_NONE, [&](auto a) {
          k_checkpoint_save<T, f8.value, vec.value, a.value><<<p.ctas, 256, 0, static_cast<cudaStream_t>(stream)>>>(
              h, const_cast<uint8_t*>(h.codes), const_cast<uint8_t*>(h.scales), static_cast<const T*>(x->data), x->stride,
              y ? static_cast<T*>(y->data) : nullptr, y ? y->stride : 0, p.g);
          return cudaGetLastError() == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
        });
      });
    });
  });
}

extern "C" int dgs_checkpoint_load(const dgs_checkpoint* ckpt, const dgs_matrix* x, void* stream) {
  if (!checkpoint_ok(ckpt) || !x || !fits(ckpt, x, true)) return DGS_EINVAL;
  if (ckpt->rows == 0) return DGS_OK;
  const Held h = held_of(ckpt);
  Plan p;
  plan_units(h.rows, h.width, &p);
  return with_type(x->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return with_bool(ckpt->format == DGS_FORMAT_E4M3, [&](auto f8) {
      return with_bool(wide<T>(x), [&](auto vec) {
        k_checkpoint_load<T, f8.value, vec.value>
            <<<p.ctas, 256, 0, static_cast<cudaStream_t>(stream)>>>(h, static_cast<T*>(x->data), x->stride, p.g);
        return cudaGetLastError() == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
      });
    });
  });
}

extern "C" int dgs_checkpoint_activation_grad(const dgs_checkpoint* ckpt, int act, const dgs_matrix* dy, const dgs_matrix* dx, void* stream) {
  if (!checkpoint_ok(ckpt) || !dy || !dx || !fits(ckpt, dy, false) || !fits(ckpt, dx, true) || dy->type != dx->type || act < 0 || act > DGS_ACT_SILU)
    return DGS_EINVAL;
  if (!same_matrix(dy, dx) && overlap(dy->data, span_bytes(dy), dx->data, span_bytes(dx))) return DGS_EINVAL;
  if (ckpt->rows == 0) return DGS_OK;
  const Held h = held_of(ckpt);
  Plan p;
  plan_units(h.rows, h.width, &p);
  return with_type(dy->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return with_bool(ckpt->format == DGS_FORMAT_E4M3, [&](auto f8) {
      return with_bool(wide<T>(dy) && wide<T>(dx), [&](auto vec) {
        return with_act(act, [&](auto a) {
          k_activation_grad<T, f8.value, vec.value, a.value><<<p.ctas, 256, 0, static_cast<cudaStream_t>(stream)>>>(
              h, static_cast<const T*>(dy->data), dy->stride, static_cast<T*>(dx->data), dx->stride, p.g);
          return cudaGetLastError() == cudaSuccess ? int(DGS_OK) : int(DGS_ECUDA);
        });
      });
    });
  });
}

extern "C" int dgs_operator_status(void* stream, int* device_status) {
  if (!device_status) return DGS_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int word = 0, zero = 0;
  if (cudaMemcpyFromSymbolAsync(&word, g_operator_status, sizeof(word), 0, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
      cudaMemcpyToSymbolAsync(g_operator_status, &zero, sizeof(zero), 0, cudaMemcpyHostToDevice, st) != cudaSuccess)
    return DGS_ECUDA;
  if (cudaStreamSynchronize(st) != cudaSuccess) return DGS_ECUDA;
  *device_status = word;
  return DGS_OK;
}
