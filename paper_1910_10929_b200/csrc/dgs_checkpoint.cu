// Activations held in 8 bits: dgs_checkpoint_save, _load and _activation_grad, and the operators' status word.
#include "dgs_operators.cuh"

#include <algorithm>
#include <atomic>
#include <thread>

namespace dgs {
namespace {

__device__ int g_operator_status;

// Reading takes the word and clears it in one step, so that a report from another stream's kernel is returned by this reading or by a later one.
// Readings under way have a place each for what they took.
constexpr uint32_t kReadings = 64;
__device__ int g_taken[kReadings];
std::atomic<uint64_t> g_reading{0};   // bit i: place i is in use
__global__ void k_status_take(uint32_t place) { g_taken[place] = atomicExch(&g_operator_status, 0); }
struct Reading {
  uint32_t place = 0;
  Reading() {
    uint64_t used = g_reading.load();
    for (;;) {
      if (used == ~0ull) {
        std::this_thread::yield();
        used = g_reading.load();
        continue;
      }
      place = uint32_t(__builtin_ctzll(~used));
      if (g_reading.compare_exchange_weak(used, used | 1ull << place)) return;
    }
  }
  ~Reading() { g_reading.fetch_and(~(1ull << place)); }
};

// ---- activations and their slopes -------------------------------------------------------------
// silu is x s(x), gelu_tanh x s(u) with u = 2 sqrt(2/pi) (x + 0.044715 x^3), s(u) = 1 / (1 + e^-u).  Slopes: s (1 + x u' (1 - s)).
constexpr float kTanhA = 1.5957691216f, kTanhB = 0.0713548163f;   // u = x (A + B x^2)
constexpr float kLog2e = 1.4426950409f;

// For results in f32: s and t = 1 - s, both from e^-|u|, which does not overflow: neither loses digits to the other.
struct Sigmoid {
  float s, t;
  __device__ __forceinline__ explicit Sigmoid(float u) {
    const float q = expf(-fabsf(u)), r = 1.0f / (1.0f + q);
    s = u > 0.0f ? r : q * r;
    t = u > 0.0f ? q * r : r;
  }
};
template <int ACT>
__device__ __forceinline__ float act_value(float x) {
  if constexpr (ACT == DGS_ACT_RELU) return x > 0.0f ? x : (x != x ? x : 0.0f);
  if constexpr (ACT == DGS_ACT_SILU) return x * Sigmoid(x).s;
  if constexpr (ACT == DGS_ACT_GELU) return 0.5f * x * erfcf(-x * 0.70710678f);
  if constexpr (ACT == DGS_ACT_GELU_TANH) return x * Sigmoid(x * fmaf(kTanhB * x, x, kTanhA)).s;
  return x;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float x) {
  if constexpr (ACT == DGS_ACT_RELU) return x > 0.0f ? 1.0f : (x != x ? x : 0.0f);
  if constexpr (ACT == DGS_ACT_GELU) return fmaf(0.3989422804f * x, expf(-0.5f * x * x), 0.5f * erfcf(-x * 0.70710678f));
  if constexpr (ACT == DGS_ACT_SILU) {
    const Sigmoid g(x);
    return g.s * fmaf(x, g.t, 1.0f);
  }
  if constexpr (ACT == DGS_ACT_GELU_TANH) {
    x = x > 30.0f ? 30.0f : x < -30.0f ? -30.0f : x;   // from there on 0 or 1; cubes beyond would overflow
    const Sigmoid g(x * fmaf(kTanhB * x, x, kTanhA));
    return g.s * fmaf(x * fmaf(3.0f * kTanhB * x, x, kTanhA), g.t, 1.0f);
  }
  return 1.0f;
}

// silu and gelu_tanh for results of 16 bits, whose own rounding is 2^-9 or 2^-12 of them: the hardware's exponential and reciprocal, off by 2^-20 at most
// beside the exponent's own roundings (3 |u| 2^-24), two numbers at a time where there is an instruction for it.  2^-24 e^-u takes the place of e^-u: its
// reciprocal 2^24 s is not flushed to zero where x s still counts.  (32768 x 2048, gelu_tanh, with expf and divisions: 42 instructions a value, 104 us; so 22
// and 66.)  gelu keeps erfcf in all types.
__device__ __forceinline__ float clamp_nan(float x, float most) {   // NaN stays NaN
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(most));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(-most));
  return x;
}
struct Scaled {   // q = 2^-24 e^-u, r = 2^24 s: 1 - s is q r
  float2 q, r;
  __device__ __forceinline__ explicit Scaled(float2 minus_u_log2_minus_24) {
    q = make_float2(hardware_exp2(minus_u_log2_minus_24.x), hardware_exp2(minus_u_log2_minus_24.y));
    const float2 d = add2(q, both(0x1p-24f));
    r = make_float2(hardware_reciprocal(d.x), hardware_reciprocal(d.y));
  }
};
template <int ACT>
__device__ __forceinline__ float2 exponent(float2 x) {
  if constexpr (ACT == DGS_ACT_SILU) return fma2(x, both(-kLog2e), both(-24.0f));
  return fma2(x, fma2(mul2(x, x), both(-kLog2e * kTanhB), both(-kLog2e * kTanhA)), both(-24.0f));
}
template <int ACT, bool FAST>
__device__ __forceinline__ void values_of(float2 (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (FAST && (ACT == DGS_ACT_SILU || ACT == DGS_ACT_GELU_TANH))
      v[i] = mul2(v[i], mul2(Scaled(exponent<ACT>(v[i])).r, both(0x1p-24f)));   // s first: x 2^-24 of a small x would lose its digits
    else
      v[i] = make_float2(act_value<ACT>(v[i].x), act_value<ACT>(v[i].y));
  }
}
template <int ACT, bool FAST>
__device__ __forceinline__ float2 slope_of(float2 x) {
  if constexpr (FAST && (ACT == DGS_ACT_SILU || ACT == DGS_ACT_GELU_TANH)) {
    // past these magnitudes the slope is 0 or 1 to within 2^-126, and e^-u 2^-24 would overflow
    constexpr float most = ACT == DGS_ACT_SILU ? 100.0f : 10.5f;
    x = make_float2(clamp_nan(x.x, most), clamp_nan(x.y, most));
    const Scaled g(exponent<ACT>(x));
    const float2 xu = ACT == DGS_ACT_SILU ? x : mul2(x, fma2(mul2(x, x), both(3.0f * kTanhB), both(kTanhA)));
    return mul2(mul2(g.r, both(0x1p-24f)), fma2(xu, mul2(g.q, g.r), both(1.0f)));
  }
  return make_float2(act_slope<ACT>(x.x), act_slope<ACT>(x.y));
}

// ---- eight columns at a time ------------------------------------------------------------------
// A unit is eight columns of a row; four lanes next to one another hold a block.  VEC: rows begin on 16 bytes, so that a unit is one
// or two wide accesses; otherwise it is read and written element by element (odd lengths and strides).  Units are read some at a time, so that
// a thread has several reads under way, and stay in their type until they are used.
template <bool VEC, class T>
__device__ __forceinline__ void read8(const T* p, uint32_t left, Eight<T>& e) {
  if (VEC && left >= 8) {
#pragma unroll
    for (uint32_t i = 0; i < sizeof(T) / 2; ++i) {
      const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p) + i);
      e.w[4 * i] = w.x, e.w[4 * i + 1] = w.y, e.w[4 * i + 2] = w.z, e.w[4 * i + 3] = w.w;
    }
    return;
  }
  T t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = uint32_t(i) < left ? p[i] : Elem<T>::put(0.0f);
  memcpy(e.w, t, sizeof(t));
}
template <bool VEC, class T>
__device__ __forceinline__ void write8(T* p, uint32_t left, const float2 (&v)[4]) {
  Eight<T> e;
  of_floats(v, e);
  if (VEC && left >= 8) {
#pragma unroll
    for (uint32_t i = 0; i < sizeof(T) / 2; ++i)
      __stcs(reinterpret_cast<uint4*>(p) + i, make_uint4(e.w[4 * i], e.w[4 * i + 1], e.w[4 * i + 2], e.w[4 * i + 3]));
    return;
  }
  T t[8];
  memcpy(t, e.w, sizeof(t));
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (uint32_t(i) < left) p[i] = t[i];
}

struct Units {
  uint32_t rows, per_row;   // units of a row: width / 8
  uint32_t groups;          // rows that the grid takes at a time: what its threads make up of whole rows, at least one
};

// Walks the units of all rows.  A thread stays in its column and goes down the rows, N of them at a time: load(i, row, unit) for each, then
// done(i, row, unit).  (Units dealt out by number alone cost 50 instructions of addresses for 22 of decoding; a save of 32768 x 2048 72 us, so 66.)
template <int N, class L, class D>
__device__ __forceinline__ void each_unit(const Units& g, L&& load, D&& done) {
  const uint32_t t = blockIdx.x * blockDim.x + threadIdx.x, group = t / g.per_row;
  if (group >= g.groups) return;
  for (uint32_t unit = t - group * g.per_row; unit < g.per_row; unit += gridDim.x * blockDim.x) {
    uint32_t row = group;
    for (; row < g.rows && g.rows - row > (N - 1) * g.groups; row += N * g.groups) {
#pragma unroll
      for (int i = 0; i < N; ++i) load(i, row + i * g.groups, unit);
#pragma unroll
      for (int i = 0; i < N; ++i) done(i, row + i * g.groups, unit);
    }
    for (; row < g.rows; row += g.groups) {
      load(0, row, unit);
      done(0, row, unit);
    }
  }
}
constexpr int kPerSm = 4, kLoadPerSm = 6;   // CTAs on an SM
template <class T> constexpr int kAtOnce = sizeof(T) == 2 ? 4 : 2;

// 32768 x 2048 in bfloat16 with gelu_tanh, of the measured copy bandwidth: save 68 us (0.76; 22 instructions a value keep the schedulers at 0.65), load 33
// us (0.95: memory), gradient 64 us (0.81).  gelu by erfcf is bound by its instructions in every type: a save 165 us, a gradient 170 us a call (in f32 152 and 167; silu in f32 113
// and 101).  Rows that do not begin on 16 bytes go element by element, bound by their accesses: 32768 x 2047 in bfloat16 a save 184, a load 213, a gradient 190 us a call.
template <class T, bool FLOAT8, bool VEC, int ACT>
__global__ void __launch_bounds__(256, kPerSm) k_checkpoint_save(Held h, uint8_t* codes, uint8_t* scales, const T* x, uint64_t xs, T* y, uint64_t ys, Units g) {
  constexpr int N = kAtOnce<T>;
  Eight<T> in[N];
  each_unit<N>(
      g,
      [&](int i, uint32_t row, uint32_t unit) {
        const uint32_t col = unit * 8;
        read8<VEC>(x + uint64_t(row) * xs + col, col < h.cols ? h.cols - col : 0, in[i]);
      },
      [&](int i, uint32_t row, uint32_t unit) {
        const uint32_t col = unit * 8, left = col < h.cols ? h.cols - col : 0;
        float2 v[4];
        floats_of(in[i], v);
        uint32_t m = largest_bits(in[i]);
        const uint32_t lanes = 0xfu << (threadIdx.x & 28u);   // the four lanes of the block: rows are a multiple of four units
        m = max(m, __shfl_xor_sync(lanes, m, 1));
        m = max(m, __shfl_xor_sync(lanes, m, 2));
        const uint32_t byte = scale_byte<FLOAT8>(m);
        const uint2 w = encode8<FLOAT8>(v, byte);
        *reinterpret_cast<uint2*>(codes + uint64_t(row) * h.width + col) = w;
        if (unit % 4 == 0) {
          uint8_t* s = scales + uint64_t(row) * h.spitch + unit / 4;
          *s = uint8_t(byte);
          if (unit + 4 == g.per_row)
            for (uint32_t b = g.per_row / 4; b < h.spitch; ++b) *++s = 0;
        }
        if (y) {
          values_of<ACT, sizeof(T) == 2>(v);
          write8<VEC>(y + uint64_t(row) * ys + col, left, v);
        }
      });
}

struct HeldUnit {
  uint2 w;
  uint32_t scale;
};
__device__ __forceinline__ void read_held(const Held& h, uint32_t row, uint32_t unit, HeldUnit& u) {
  u.w = __ldg(reinterpret_cast<const uint2*>(h.codes + uint64_t(row) * h.width + unit * 8));
  u.scale = __ldg(h.scales + uint64_t(row) * h.spitch + unit / 4);
}
template <class T, bool FLOAT8, bool VEC>
__global__ void __launch_bounds__(256, kLoadPerSm) k_checkpoint_load(Held h, T* x, uint64_t xs, Units g) {
  HeldUnit in[4];
  each_unit<4>(
      g, [&](int i, uint32_t row, uint32_t unit) { read_held(h, row, unit, in[i]); },
      [&](int i, uint32_t row, uint32_t unit) {
        const uint32_t col = unit * 8;
        if (col >= h.cols) return;
        float2 v[4];
        decode8<FLOAT8>(in[i].w, scale_down(in[i].scale), v);
        write8<VEC>(x + uint64_t(row) * xs + col, h.cols - col, v);
      });
}

template <class T, bool FLOAT8, bool VEC, int ACT>
__global__ void __launch_bounds__(256, kPerSm) k_activation_grad(Held h, const T* dy, uint64_t dys, T* dx, uint64_t dxs, Units g) {
  constexpr int N = kAtOnce<T>;
  HeldUnit in[N];
  Eight<T> d[N];
  each_unit<N>(
      g,
      [&](int i, uint32_t row, uint32_t unit) {
        const uint32_t col = unit * 8;
        read_held(h, row, unit, in[i]);
        read8<VEC>(dy + uint64_t(row) * dys + col, col < h.cols ? h.cols - col : 0, d[i]);
      },
      [&](int i, uint32_t row, uint32_t unit) {
        const uint32_t col = unit * 8;
        if (col >= h.cols) return;
        float2 v[4], dv[4];
        decode8<FLOAT8>(in[i].w, scale_down(in[i].scale), v);
        floats_of(d[i], dv);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = mul2(dv[k], slope_of<ACT, sizeof(T) == 2>(v[k]));
        write8<VEC>(dx + uint64_t(row) * dxs + col, h.cols - col, v);
      });
}

// ---- host side --------------------------------------------------------------------------------
struct Plan {
  Units g;
  uint32_t ctas;
};
void plan_units(uint64_t rows, uint32_t width, uint32_t per_sm, Plan* p) {   // as many CTAs as run at a time: each has the same rows to do
  p->g.rows = uint32_t(rows);
  p->g.per_row = width / 8;
  p->ctas = uint32_t(std::min<uint64_t>((rows * p->g.per_row + 255) / 256, uint64_t(kSms) * per_sm));
  p->g.groups = std::max(1u, p->ctas * 256 / p->g.per_row);
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
  if (!out_bytes || cols == 0 || cols > (1u << 30) || rows >= (1ull << 31) || rows > kMostElements / cols) return DGS_EINVAL;
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
  plan_units(h.rows, h.width, kPerSm, &p);
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
  plan_units(h.rows, h.width, kLoadPerSm, &p);
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
  plan_units(h.rows, h.width, kPerSm, &p);
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
  const Reading reading;
  int word = 0;
  k_status_take<<<1, 1, 0, st>>>(reading.place);
  if (cudaGetLastError() != cudaSuccess ||
      cudaMemcpyFromSymbolAsync(&word, g_taken, sizeof(word), reading.place * sizeof(word), cudaMemcpyDeviceToHost, st) != cudaSuccess)
    return DGS_ECUDA;
  if (cudaStreamSynchronize(st) != cudaSuccess) return DGS_ECUDA;
  *device_status = word;
  return DGS_OK;
}
