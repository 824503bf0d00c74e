// The loss over a vocabulary and its gradient for few rows, without tensor cores (a part of dgs_vocabulary.cu).
//
// A warp takes four words and RB rows at a time: eight columns of each a lane, 4 RB sums of products in f32, which end one to a lane.  A word is read once for
// RB rows.  The gradient has a CTA go through tiles of TW words: s of a tile in shared memory, then a thread for each column, which forms its part of the tile's
// rows of dW and of dh in one go over the rows.  Everything is in f32, so nothing need be scaled.
#pragma once

namespace dgs {
namespace {

constexpr uint32_t kFewRows = 64, kFewWords = 4;

// V sums of every lane added up over the warp: lane l is left with sum l / (32 / V).
template <uint32_t V, uint32_t BIT = 16>
__device__ __forceinline__ float sums_to_lanes(const float (&v)[V], uint32_t lane) {
  if constexpr (V == 1) {
    float s = v[0];
#pragma unroll
    for (uint32_t b = BIT; b; b /= 2) s += __shfl_xor_sync(0xffffffffu, s, b);
    return s;
  } else {
    float half[V / 2];
#pragma unroll
    for (uint32_t i = 0; i < V / 2; ++i) {
      const float keep = lane & BIT ? v[V / 2 + i] : v[i], give = lane & BIT ? v[i] : v[V / 2 + i];
      half[i] = keep + __shfl_xor_sync(0xffffffffu, give, BIT);
    }
    return sums_to_lanes<V / 2, BIT / 2>(half, lane);
  }
}

struct Few {
  const void *h, *w;
  uint64_t h_stride, w_stride;
  uint32_t spans, tiles;   // of 256 columns; gradient: of TW words
};

// The products of rows row0 .. row0 + RB with words word0 .. word0 + 4: lane l gets row l / (32 / (4 RB)) % RB with word l / (32 / 4).
template <class T, bool VEC, uint32_t RB>
__device__ __forceinline__ float few_products(const Head& a, const Few& f, uint32_t row0, uint32_t word0, uint32_t lane) {
  constexpr int kUnroll = RB == 1 ? 3 : 1;   // of 256 columns: one row's loads are all there is to wait for
  float2 sum[kFewWords * RB];
#pragma unroll
  for (uint32_t i = 0; i < kFewWords * RB; ++i) sum[i] = make_float2(0.0f, 0.0f);
  const auto span = [&](uint32_t s, auto whole) {   // of 256 columns; loads with a branch in them would wait for one another
    constexpr bool kWhole = decltype(whole)::value;
    Eight<T> we[kFewWords];
#pragma unroll
    for (uint32_t i = 0; i < kFewWords; ++i)
      load8<T, VEC, false, kWhole>(static_cast<const T*>(f.w) + min(word0 + i, a.words - 1) * f.w_stride, s * kSpan, lane, a.width, we[i]);
#pragma unroll
    for (uint32_t r = 0; r < RB; ++r) {
      Eight<T> he;
      load8<T, VEC, true, kWhole>(static_cast<const T*>(f.h) + min(row0 + r, a.rows - 1) * f.h_stride, s * kSpan, lane, a.width, he);
      float2 hv[4];
      floats_of(he, hv);
#pragma unroll
      for (uint32_t i = 0; i < kFewWords; ++i) {
        float2 wv[4];
        floats_of(we[i], wv);
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[i * RB + r] = fma2(hv[k], wv[k], sum[i * RB + r]);
      }
    }
  };
  const uint32_t whole = a.width / kSpan;
#pragma unroll kUnroll
  for (uint32_t s = 0; s < whole; ++s) span(s, std::true_type{});
  if (whole < f.spans) span(whole, std::false_type{});
  float v[kFewWords * RB];
#pragma unroll
  for (uint32_t i = 0; i < kFewWords * RB; ++i) v[i] = sum[i].x + sum[i].y;
  return sums_to_lanes(v, lane);
}

__device__ __forceinline__ float2 join_sums(float2 x, float2 y) {
  const float most = fmaxf(x.x, y.x), from = most == kNone ? 0.0f : most;
  return make_float2(most, x.y * exp2f((x.x - from) * kLog2e) + y.y * exp2f((y.x - from) * kLog2e));
}

// Maxima and sums: partial[part][row], a part for each CTA along x.
template <class T, bool VEC, uint32_t RB>
__global__ void __launch_bounds__(256, 2) k_few_loss(const __grid_constant__ Head a, const __grid_constant__ Few f) {
  constexpr uint32_t V = kFewWords * RB, kSame = 32 / V;   // lanes with the same product
  __shared__ float2 s_part[8][RB];
  let_next_kernel_begin();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, row0 = blockIdx.y * RB, index = lane / kSame, row = row0 + index % RB;
  const int target = row < a.rows ? target_of(a, row, false) : -1;
  float2 mine = make_float2(kNone, 0.0f);
  for (uint32_t word0 = (blockIdx.x * 8 + warp) * kFewWords; word0 < a.words; word0 += gridDim.x * 8 * kFewWords) {
    const float z = few_products<T, VEC, RB>(a, f, row0, word0, lane);
    const uint32_t word = word0 + index / RB;
    if (lane % kSame == 0 && word < a.words) {
      const float most = fmaxf(mine.x, z), from = most == kNone ? 0.0f : most;
      mine = make_float2(most, mine.y * hardware_exp2((mine.x - from) * kLog2e) + hardware_exp2((z - from) * kLog2e));
      if (int(word) == target) a.at_target[row] = z;
    }
  }
#pragma unroll
  for (uint32_t b = 16; b >= RB * kSame; b /= 2) mine = join_sums(mine, make_float2(__shfl_xor_sync(0xffffffffu, mine.x, b), __shfl_xor_sync(0xffffffffu, mine.y, b)));
  if (lane % kSame == 0 && lane < RB * kSame) s_part[warp][index] = mine;
  __syncthreads();
  if (threadIdx.x < RB && row0 + threadIdx.x < a.rows) {
    float2 v = s_part[0][threadIdx.x];
    for (uint32_t q = 1; q < 8; ++q) v = join_sums(v, s_part[q][threadIdx.x]);
    a.partial[uint64_t(blockIdx.x) * a.rows + row0 + threadIdx.x] = v;
  }
}
// A CTA a row joins its parts.
__global__ void __launch_bounds__(256) k_few_rows(const __grid_constant__ Head a, uint32_t parts, float* loss, float* lse) {
  __shared__ float2 s_part[8];
  const uint32_t row = blockIdx.x;
  wait_for_last_kernel();
  float2 v = make_float2(kNone, 0.0f);
  for (uint32_t p = threadIdx.x; p < parts; p += 256) v = join_sums(v, a.partial[uint64_t(p) * a.rows + row]);
#pragma unroll
  for (uint32_t b = 16; b; b /= 2) v = join_sums(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, b), __shfl_xor_sync(0xffffffffu, v.y, b)));
  if (threadIdx.x % 32 == 0) s_part[threadIdx.x / 32] = v;
  __syncthreads();
  if (threadIdx.x) return;
  for (uint32_t q = 1; q < 8; ++q) v = join_sums(v, s_part[q]);
  finish_row(a, row, v, loss, lse);
}

// dW of the words and, in `parts` [CTAs][rows][width], each CTA's part of dh, which k_head_join adds up.
template <uint32_t TW> constexpr uint32_t kFewThreads = TW == 8 ? 512 : 256;
template <class T, bool VEC, uint32_t RB, uint32_t TW>
__global__ void __launch_bounds__(kFewThreads<TW>, TW == 8 ? 1 : 2) k_few_grad(const __grid_constant__ Head a, const __grid_constant__ Few f, float* dw, float* parts) {
  constexpr uint32_t V = kFewWords * RB, kSame = 32 / V;
  __shared__ __align__(16) float s_s[kFewRows][TW];
  __shared__ int s_target[kFewRows];
  let_next_kernel_begin();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, index = lane / kSame;
  if (threadIdx.x < a.rows) s_target[threadIdx.x] = target_of(a, threadIdx.x, blockIdx.x == 0);
  __syncthreads();
  parts += uint64_t(blockIdx.x) * a.rows * a.width;
  for (uint32_t tile = blockIdx.x; tile < f.tiles; tile += gridDim.x) {
    const uint32_t first = tile * TW, row_blocks = (a.rows + RB - 1) / RB;
    for (uint32_t u = warp; u < row_blocks * (TW / kFewWords); u += kFewThreads<TW> / 32) {
      const uint32_t row0 = u / (TW / kFewWords) * RB, word0 = first + u % (TW / kFewWords) * kFewWords;
      if (word0 >= a.words) continue;
      const float z = few_products<T, VEC, RB>(a, f, row0, word0, lane);
      const uint32_t word = word0 + index / RB, row = row0 + index % RB;
      if (lane % kSame == 0 && row < a.rows) {
        const int target = s_target[row];
        float s = 0.0f;   // also behind the last word, and in ignored rows, whatever they hold
        if (target >= 0 && word < a.words) s = (hardware_exp2((z - a.lse[row]) * kLog2e) - (int(word) == target ? 1.0f : 0.0f)) * a.dloss[uint64_t(row) * a.dloss_step];
        s_s[row][word - first] = s;
      }
    }
    __syncthreads();
    const uint32_t words = min(TW, a.words - first);
    for (uint32_t c = threadIdx.x; c < a.width; c += kFewThreads<TW>) {
      float w[TW], d[TW];
#pragma unroll
      for (uint32_t i = 0; i < TW; ++i) w[i] = i < words ? Elem<T>::get(static_cast<const T*>(f.w)[(first + i) * f.w_stride + c]) : 0.0f, d[i] = 0.0f;
      constexpr uint32_t kAtOnce = TW == 8 ? 8 : 4;   // rows whose values are on their way together
      for (uint32_t r0 = 0; r0 < a.rows; r0 += kAtOnce) {
        float x[kAtOnce];
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) {
          const uint32_t r = r0 + i;
          x[i] = r < a.rows && s_target[r] >= 0 ? Elem<T>::get(static_cast<const T*>(f.h)[r * f.h_stride + c]) : 0.0f;
        }
#pragma unroll
        for (uint32_t j = 0; j < kAtOnce; ++j) {
          const uint32_t r = r0 + j;
          if (r >= a.rows) break;
          float sum = 0.0f;   // s of an ignored row is 0
#pragma unroll
          for (uint32_t i = 0; i < TW; i += 4) {
            if (i < words) {   // s behind the last word was not written
              const float4 s = *reinterpret_cast<const float4*>(&s_s[r][i]);
              sum = fmaf(s.x, w[i], sum), d[i] = fmaf(s.x, x[j], d[i]);
              sum = fmaf(s.y, w[i + 1], sum), d[i + 1] = fmaf(s.y, x[j], d[i + 1]);
              sum = fmaf(s.z, w[i + 2], sum), d[i + 2] = fmaf(s.z, x[j], d[i + 2]);
              sum = fmaf(s.w, w[i + 3], sum), d[i + 3] = fmaf(s.w, x[j], d[i + 3]);
            }
          }
          float* p = parts + uint64_t(r) * a.width + c;
          *p = tile == blockIdx.x ? sum : *p + sum;
        }
      }
      if (dw)
#pragma unroll
        for (uint32_t i = 0; i < TW; ++i)
          if (i < words) {
            float* p = dw + (uint64_t(first) + i) * a.width + c;
            *p = a.add ? *p + d[i] : d[i];
          }
    }
    __syncthreads();
  }
}
}  // namespace
}  // namespace dgs
