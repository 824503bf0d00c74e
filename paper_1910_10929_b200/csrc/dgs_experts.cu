// Tokens' rows in the order of the experts' lists and back: dgs_experts_gather, _combine and _combine_grad.
#include "dgs_operators.cuh"

#include <algorithm>

namespace dgs {
namespace {

struct Rows {
  const uint32_t* order;
  const uint32_t* place;
  uint32_t tokens, k, cols, chunks, warps;   // chunks: of kSpan columns; warps: that share a token (combine_grad)
  uint64_t slots, in_stride, mid_stride, out_stride;
  int* status;
};

// Lane j: where the token's j-th slot stands, DGS_NO_EXPERT for an empty one, for one past the last and (reported) for one that points outside.
__device__ __forceinline__ uint32_t lane_place(const Rows& a, uint32_t token, uint32_t lane) {
  uint32_t p = lane < a.k ? a.place[uint64_t(token) * a.k + lane] : DGS_NO_EXPERT;
  if (p != DGS_NO_EXPERT && p >= a.slots) {
    report(a.status, DGS_EINVAL);
    p = DGS_NO_EXPERT;
  }
  return p;
}
// Rows behind the last list are zero: as many as there are empty slots.  A token's warp looks after the rows of its slots' numbers.
template <class T, bool VEC>
__device__ __forceinline__ void clear_rows(const Rows& a, uint32_t token, uint32_t col0, uint32_t lane, T* y, uint64_t stride) {
  uint32_t left = __ballot_sync(0xffffffffu, lane < a.k && a.order[uint64_t(token) * a.k + lane] == DGS_NO_EXPERT);
  const Eight<T> zero = {};
  for (; left; left &= left - 1) store8<T, VEC>(y + (uint64_t(token) * a.k + __ffs(left) - 1) * stride, col0, lane, a.cols, zero);
}

// y[place[t][j]] = x[t]: a row is read once and written k times.  Bound by HBM.
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_experts_gather(const __grid_constant__ Rows a, const T* x, T* y) {
  const uint32_t lane = threadIdx.x % 32;
  const uint64_t units = uint64_t(a.tokens) * a.chunks, step = uint64_t(gridDim.x) * 8;
  for (uint64_t u = uint64_t(blockIdx.x) * 8 + threadIdx.x / 32; u < units; u += step) {
    const uint32_t token = units >> 32 ? uint32_t(u / a.chunks) : uint32_t(u) / a.chunks, col0 = uint32_t(u - uint64_t(token) * a.chunks) * kSpan;
    Eight<T> e;
    load8<T, VEC>(x + token * a.in_stride, col0, lane, a.cols, e);
    const uint32_t mine = lane_place(a, token, lane);
    for (uint32_t j = 0; j < a.k; ++j) {
      const uint32_t p = __shfl_sync(0xffffffffu, mine, j);
      if (p != DGS_NO_EXPERT) store8<T, VEC>(y + p * a.out_stride, col0, lane, a.cols, e);
    }
    clear_rows<T, VEC>(a, token, col0, lane, y, a.out_stride);
  }
}

// out[t] = sum over j of weight[t][j] y[place[t][j]], slots ascending, in f32.  weight NULL: 1, which is the gather's gradient.  Bound by HBM: the
// rows of four slots (two in f32 and of rows that begin anywhere) are on their way together, in 48 warps an SM (eight slots in 24 warps: 32768 x 2048, top 8 237 us, 187 so; 48 warps that go on to the next
// token 212).  Rows of f32 that begin anywhere go in 32, which need not spill registers: 40000 x 33, top 8 27 us (31 in 48 warps), 16384 x 767, top 8 77 (80).
template <class T, bool VEC>
__global__ void __launch_bounds__(256, VEC || sizeof(T) == 2 ? 6 : 4) k_experts_combine(const __grid_constant__ Rows a, const float* weight, const T* y, T* out) {
  constexpr uint32_t J = VEC && sizeof(T) == 2 ? 4 : 2;
  const uint32_t lane = threadIdx.x % 32;
  const uint64_t units = uint64_t(a.tokens) * a.chunks, step = uint64_t(gridDim.x) * 8;
  for (uint64_t u = uint64_t(blockIdx.x) * 8 + threadIdx.x / 32; u < units; u += step) {
    const uint32_t token = units >> 32 ? uint32_t(u / a.chunks) : uint32_t(u) / a.chunks, col0 = uint32_t(u - uint64_t(token) * a.chunks) * kSpan;
    const uint32_t mine = lane_place(a, token, lane);
    const float w = weight && lane < a.k ? weight[uint64_t(token) * a.k + lane] : 1.0f;
    float2 sum[4] = {};
    for (uint32_t j0 = 0; j0 < a.k; j0 += J) {
      Eight<T> e[J];
#pragma unroll
      for (uint32_t j = 0; j < J; ++j) {
        const uint32_t p = j0 + j < a.k ? __shfl_sync(0xffffffffu, mine, j0 + j) : DGS_NO_EXPERT;
        if (p != DGS_NO_EXPERT) load8<T, VEC>(y + p * a.in_stride, col0, lane, a.cols, e[j]);
      }
#pragma unroll
      for (uint32_t j = 0; j < J; ++j) {
        const uint32_t p = j0 + j < a.k ? __shfl_sync(0xffffffffu, mine, j0 + j) : DGS_NO_EXPERT;
        if (p != DGS_NO_EXPERT) {
          const float f = __shfl_sync(0xffffffffu, w, j0 + j);
          float2 v[4];
          floats_of(e[j], v);
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] = fma2(v[i], both(f), sum[i]);
        }
      }
    }
    Eight<T> r;
    of_floats(sum, r);
    store8<T, VEC>(out + token * a.out_stride, col0, lane, a.cols, r);
  }
}

// dy[place[t][j]] = weight[t][j] dout[t] and dweight[t][j] = <dout[t], y[place[t][j]]>.  `warps` warps share a token's columns; their parts of the
// products are added in their order.  Bound by HBM: a token's dout is read once for eight slots (four in f32; two of rows that begin anywhere, in 40 warps an SM for 16 bits:
// 16384 x 767 with top 8 114 us, 172 with eight slots in 16 warps; words put together from two, which need fewer loads: 272).
template <class T, bool VEC>
__global__ void __launch_bounds__(256, VEC || sizeof(T) == 4 ? 3 : 5) k_experts_combine_grad(const __grid_constant__ Rows a, const float* weight, const T* dout, const T* y, T* dy, float* dweight) {
  constexpr uint32_t J = !VEC ? 2 : sizeof(T) == 2 ? 8 : 4;
  __shared__ float s_part[8][J];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, part = warp % a.warps, each = 8 / a.warps;
  const uint32_t rounds = (a.tokens + gridDim.x * each - 1) / (gridDim.x * each);
  for (uint32_t r = 0; r < rounds; ++r) {   // every warp of the CTA goes along: the sums meet in shared memory
    const uint64_t at = (uint64_t(r) * gridDim.x + blockIdx.x) * each + warp / a.warps;
    const bool there = at < a.tokens;
    const uint32_t token = there ? uint32_t(at) : 0;
    const uint32_t mine = there ? lane_place(a, token, lane) : DGS_NO_EXPERT;
    const float w = there && lane < a.k ? weight[uint64_t(token) * a.k + lane] : 0.0f;
    for (uint32_t j0 = 0; j0 < a.k; j0 += J) {
      float2 dot[J];
#pragma unroll
      for (uint32_t j = 0; j < J; ++j) dot[j] = make_float2(0.0f, 0.0f);
      for (uint32_t c = part; there && c < a.chunks; c += a.warps) {
        Eight<T> g, e[J];
        load8<T, VEC>(dout + token * a.mid_stride, c * kSpan, lane, a.cols, g);
#pragma unroll
        for (uint32_t j = 0; j < J; ++j) {
          const uint32_t p = j0 + j < a.k ? __shfl_sync(0xffffffffu, mine, j0 + j) : DGS_NO_EXPERT;
          if (p != DGS_NO_EXPERT) load8<T, VEC>(y + p * a.in_stride, c * kSpan, lane, a.cols, e[j]);
        }
        float2 d[4];
        floats_of(g, d);
#pragma unroll
        for (uint32_t j = 0; j < J; ++j) {
          const uint32_t p = j0 + j < a.k ? __shfl_sync(0xffffffffu, mine, j0 + j) : DGS_NO_EXPERT;
          if (p != DGS_NO_EXPERT) {
            const float f = __shfl_sync(0xffffffffu, w, j0 + j);
            float2 v[4], s[4];
            floats_of(e[j], v);
#pragma unroll
            for (int i = 0; i < 4; ++i) dot[j] = fma2(d[i], v[i], dot[j]), s[i] = mul2(d[i], both(f));
            Eight<T> o;
            of_floats(s, o);
            store8<T, VEC>(dy + p * a.out_stride, c * kSpan, lane, a.cols, o);
          }
        }
        if (j0 == 0) clear_rows<T, VEC>(a, token, c * kSpan, lane, dy, a.out_stride);
      }
#pragma unroll
      for (uint32_t j = 0; j < J; ++j) {
        float v = dot[j].x + dot[j].y;
#pragma unroll
        for (int s = 16; s; s /= 2) v += __shfl_xor_sync(0xffffffffu, v, s);
        if (lane == 0) s_part[warp][j] = v;
      }
      __syncthreads();
      if (there && part == 0 && lane < J && j0 + lane < a.k) {
        float v = 0.0f;
        for (uint32_t q = 0; q < a.warps; ++q) v += s_part[warp + q][lane];
        dweight[uint64_t(token) * a.k + j0 + lane] = v;
      }
      __syncthreads();
    }
  }
}

bool slots_ok(const uint32_t* order, const uint32_t* place, uint32_t k, uint64_t tokens) {
  return k && k <= DGS_ROUTE_MAX_K && tokens <= ((1ull << 31) - 1) / k && aligned(order, 4) && aligned(place, 4) && (tokens == 0 || place);
}
bool rows_fit(const dgs_matrix* one, const dgs_matrix* all, uint32_t k) {
  return one->cols == all->cols && one->type == all->type && one->cols <= (1u << 30) && all->rows == one->rows * k;
}
Rows rows_of(const uint32_t* order, const uint32_t* place, uint32_t k, const dgs_matrix* one) {
  Rows a = {};
  a.order = order;
  a.place = place;
  a.tokens = uint32_t(one->rows);
  a.k = k;
  a.cols = one->cols;
  a.chunks = (one->cols + kSpan - 1) / kSpan;
  a.slots = one->rows * k;
  a.status = operator_status_word();
  return a;
}
uint32_t ctas(uint64_t units) { return uint32_t(std::min<uint64_t>((units + 7) / 8, 1u << 22)); }

int launched() { return cudaGetLastError() == cudaSuccess ? DGS_OK : DGS_ECUDA; }

}  // namespace
}  // namespace dgs

using namespace dgs;

extern "C" int dgs_experts_gather(const dgs_matrix* x, const uint32_t* order, const uint32_t* place, uint32_t k, const dgs_matrix* y, void* stream) {
  if (!matrix_ok(x, false) || !matrix_ok(y, true) || !slots_ok(order, place, k, x->rows) || !rows_fit(x, y, k) || (x->rows && !order)) return DGS_EINVAL;
  const uint64_t lists = x->rows * k * 4ull;
  const Span part[] = {{x->data, span_bytes(x), false}, {order, lists, false}, {place, lists, false}, {y->data, span_bytes(y), true}};
  if (!apart(part)) return DGS_EINVAL;
  if (x->rows == 0) return DGS_OK;
  Rows a = rows_of(order, place, k, x);
  if (!a.status) return DGS_ECUDA;
  a.in_stride = x->stride;
  a.out_stride = y->stride;
  return with_wide(x->type, on_16_bytes(x) && on_16_bytes(y), [&](auto* t, auto vec) {
    using T = std::remove_pointer_t<decltype(t)>;
    k_experts_gather<T, vec.value><<<ctas(uint64_t(a.tokens) * a.chunks), 256, 0, static_cast<cudaStream_t>(stream)>>>(a, static_cast<const T*>(x->data), static_cast<T*>(y->data));
    return launched();
  });
}

extern "C" int dgs_experts_combine(const dgs_matrix* y, const float* weight, const uint32_t* place, uint32_t k, const dgs_matrix* out, void* stream) {
  if (!matrix_ok(y, false) || !matrix_ok(out, true) || !slots_ok(nullptr, place, k, out->rows) || !rows_fit(out, y, k) || !aligned(weight, 4)) return DGS_EINVAL;
  const uint64_t lists = out->rows * k * 4ull;
  const Span part[] = {{y->data, span_bytes(y), false}, {weight, weight ? lists : 0, false}, {place, lists, false}, {out->data, span_bytes(out), true}};
  if (!apart(part)) return DGS_EINVAL;
  if (out->rows == 0) return DGS_OK;
  Rows a = rows_of(nullptr, place, k, out);
  if (!a.status) return DGS_ECUDA;
  a.in_stride = y->stride;
  a.out_stride = out->stride;
  return with_wide(y->type, on_16_bytes(y) && on_16_bytes(out), [&](auto* t, auto vec) {
    using T = std::remove_pointer_t<decltype(t)>;
    k_experts_combine<T, vec.value><<<ctas(uint64_t(a.tokens) * a.chunks), 256, 0, static_cast<cudaStream_t>(stream)>>>(a, weight, static_cast<const T*>(y->data), static_cast<T*>(out->data));
    return launched();
  });
}

extern "C" int dgs_experts_combine_grad(const dgs_matrix* dout, const dgs_matrix* y, const float* weight, const uint32_t* order, const uint32_t* place, uint32_t k,
                                        const dgs_matrix* dy, float* dweight, void* stream) {
  if (!matrix_ok(dout, false) || !matrix_ok(y, false) || !matrix_ok(dy, true) || !slots_ok(order, place, k, dout->rows) || !rows_fit(dout, y, k) ||
      !rows_fit(dout, dy, k) || !aligned(weight, 4) || !aligned(dweight, 4) || (dout->rows && (!order || !weight || !dweight)))
    return DGS_EINVAL;
  const uint64_t lists = dout->rows * k * 4ull;
  const Span part[] = {{dout->data, span_bytes(dout), false}, {y->data, span_bytes(y), false}, {weight, lists, false}, {order, lists, false},
                       {place, lists, false}, {dy->data, span_bytes(dy), true}, {dweight, lists, true}};
  if (!apart(part)) return DGS_EINVAL;
  if (dout->rows == 0) return DGS_OK;
  Rows a = rows_of(order, place, k, dout);
  if (!a.status) return DGS_ECUDA;
  a.in_stride = y->stride;
  a.mid_stride = dout->stride;
  a.out_stride = dy->stride;
  // Few tokens: their columns are shared out, so that no warp makes more trips to memory than it has to.  Where 32 warps an SM are the aim / 8 / 128, us: 1000 x 8192 with top 8 in bfloat16
  // 54 / 58 / 55, 4000 x 2048 with top 8 55 / 66 / 53, 2500 x 2048 with top 2 16.5 / 16.5 / 19.6, 8000 x 1024 with top 2 24.7 / 24.7 / 30.9.
  a.warps = 1;
  while (a.warps < 8 && a.warps < a.chunks && uint64_t(a.tokens) * a.warps < kSms * 32) a.warps *= 2;
  const uint32_t grid = uint32_t(std::min<uint64_t>((uint64_t(a.tokens) * a.warps + 7) / 8, 1u << 22));
  return with_wide(y->type, on_16_bytes(dout) && on_16_bytes(y) && on_16_bytes(dy), [&](auto* t, auto vec) {
    using T = std::remove_pointer_t<decltype(t)>;
    k_experts_combine_grad<T, vec.value><<<grid, 256, 0, static_cast<cudaStream_t>(stream)>>>(a, weight, static_cast<const T*>(dout->data), static_cast<const T*>(y->data),
                                                                                              static_cast<T*>(dy->data), dweight);
    return launched();
  });
}
