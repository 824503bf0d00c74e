// The router of a model with experts: dgs_route_experts and dgs_route_experts_grad.
#include "dgs_operators.cuh"

#include <algorithm>
#include <cmath>

namespace dgs {
namespace {

constexpr uint32_t kTile = 64;           // tokens of a CTA: two words of a bit mask per expert
constexpr uint32_t kRouteWarps = 8;
constexpr uint32_t kAll = 0xffffffffu;

struct RouteArgs {
  uint64_t stride;
  uint32_t tokens, experts, k, groups, group_size, kept, best, tiles;
  bool sigmoid, renorm;
  float scale;
  const float* bias;
  uint32_t* expert;
  float* weight;
  uint32_t* offsets;
  uint32_t* order;
  uint32_t* place;
  uint32_t* counts;    // [experts + 1][tiles]: slots of a tile that belong to an expert; behind the last expert: empty slots
};

// Numbers whose unsigned order is the order of the floats; 0 stands for "not there" (below -inf).
__device__ __forceinline__ uint32_t sortable(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);   // -0 and +0 are equal keys
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned long long sortable(double v) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ float unsorted(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ double unsorted(unsigned long long k) {
  return __longlong_as_double((long long)(k >> 63 ? k & 0x7fffffffffffffffull : ~k));
}
__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(kAll, v); }
__device__ __forceinline__ unsigned long long warp_max(unsigned long long v) {
#pragma unroll
  for (int d = 16; d; d /= 2) {
    const unsigned long long o = __shfl_xor_sync(kAll, v, d);
    v = o > v ? o : v;
  }
  return v;
}
template <class R>
__device__ __forceinline__ R warp_sum(R v) {
#pragma unroll
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(kAll, v, d);
  return v;
}

// Expert 32 i + lane is element i of a lane: loads are coalesced, and ballots over the lanes give the experts' order.
// Chooses the `count` largest of the keys that are not 0, ties to the lowest index: bit i of the result is element i.
// low / next: the smallest key chosen and the largest one left.
template <int PER, class K>
__device__ __forceinline__ uint32_t choose(const K (&key)[PER], uint32_t count, K* low, K* next) {
  K border = ~K(0);
  uint32_t above = 0, level = 0;
  for (;;) {   // the distinct keys in descending order until `count` are reached: at most `count` rounds
    K m = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) m = key[i] < border && key[i] > m ? key[i] : m;
    m = warp_max(m);
    if (m == 0) break;   // fewer than `count` are there
    border = m;
    above += level;
    level = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) level += __popc(__ballot_sync(kAll, key[i] == m));
    if (above + level >= count) break;
  }
  uint32_t bits = 0, seen = 0;
  K left = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t at = __ballot_sync(kAll, key[i] == border);
    const bool mine = key[i] != 0 && (key[i] > border ||
                      (key[i] == border && above + seen + __popc(at & ((1u << (threadIdx.x & 31)) - 1)) < count));
    bits |= uint32_t(mine) << i;
    if (!mine && key[i] > left) left = key[i];
    seen += __popc(at);
  }
  *low = border;
  *next = warp_max(left);
  return bits;
}

// The keys of the groups of one token, each lane keeping group `lane` (and lane + 32 and so on: GP of them); 0: no expert left in it.
template <int PER, class R, class K>
__device__ __forceinline__ K group_key(const K (&key)[PER], const RouteArgs& a, uint32_t g) {
  const uint32_t lane = threadIdx.x & 31, lo = g * a.group_size, hi = lo + a.group_size;
  K m = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t e = 32 * i + lane;
    if (32u * i < hi && 32u * i + 32 > lo && e >= lo && e < hi && key[i] > m) m = key[i];
  }
  const K first = warp_max(m);
  if (first == 0 || a.best == 1) return first;
  uint32_t equal = 0;
  m = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t e = 32 * i + lane;
    const bool in = 32u * i < hi && 32u * i + 32 > lo && e >= lo && e < hi;
    equal += __popc(__ballot_sync(kAll, in && key[i] == first));
    if (in && key[i] != first && key[i] > m) m = key[i];
  }
  const K second = equal > 1 ? first : warp_max(m);
  return second == 0 ? first : sortable(unsorted(first) + unsorted(second));
}

// Leaves only the keys of the kept groups.  close: the border between kept and dropped groups is nearer than `slack`
// (relative to the larger key's size).
template <int PER, class R, class K>
__device__ __forceinline__ bool keep_groups(K (&key)[PER], const RouteArgs& a, R slack) {
  const uint32_t lane = threadIdx.x & 31;
  K mine[PER];   // at most as many groups as experts
#pragma unroll
  for (int i = 0; i < PER; ++i) mine[i] = 0;
  for (uint32_t g = 0; g < a.groups; ++g) {
    const K v = group_key<PER, R, K>(key, a, g);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (32u * i + lane == g) mine[i] = v;
  }
  K low, next;
  const uint32_t bits = choose<PER, K>(mine, a.kept, &low, &next);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t e = 32 * i + lane, g = e < a.experts ? e / a.group_size : 0;
    uint32_t keep = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (32u * j >= a.groups) break;
      const uint32_t b = __ballot_sync(kAll, bits >> j & 1);
      if (g / 32 == uint32_t(j)) keep = b >> (g % 32) & 1;
    }
    if (!keep) key[i] = 0;
  }
  return next != 0 && R(unsorted(low)) - R(unsorted(next)) <= slack;
}

__device__ __forceinline__ float score_exp(float v) { return expf(v); }
__device__ __forceinline__ double score_exp(double v) { return exp(v); }

// Keys of one token in R arithmetic from its logits; free: bit i, element i is an expert that the token may have.  Returns what
// no score exceeds.
template <int PER, class R, class K>
__device__ __forceinline__ R make_keys(const float (&z)[PER], uint32_t free, float top, const RouteArgs& a, K (&key)[PER]) {
  const uint32_t lane = threadIdx.x & 31;
  R s[PER];
  R sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    s[i] = 0;
    if (free >> i & 1) s[i] = a.sigmoid ? R(1) / (R(1) + score_exp(-R(z[i]))) : score_exp(R(z[i]) - R(top));
    sum += s[i];
  }
  if (!a.sigmoid) {
    sum = warp_sum(sum);
#pragma unroll
    for (int i = 0; i < PER; ++i) s[i] = s[i] / sum;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const R b = a.bias && (free >> i & 1) ? R(a.bias[32 * i + lane]) : R(0);
    key[i] = free >> i & 1 ? sortable(s[i] + b) : K(0);
  }
  return a.sigmoid ? R(1) : R(1) / sum;
}

// The same choice in 64 bits, for tokens whose border 32 bits cannot tell: rare, and kept out of line.
template <int PER>
__device__ __noinline__ uint32_t choose_exactly(const float (&z)[PER], uint32_t free, float top, const RouteArgs& a) {
  unsigned long long key[PER], low, next;
  make_keys<PER, double>(z, free, top, a, key);
  if (a.groups > 1) keep_groups<PER, double>(key, a, 0.0);
  return choose<PER>(key, a.k, &low, &next);
}

// One warp per token, a tile of 64 tokens per CTA.  The token's logits stay in registers; the experts chosen are marked in a bit
// mask per expert (bit = token of the tile), whose counts are what a later kernel needs to place the tile's slots.
template <int PER, class T>
__global__ void __launch_bounds__(kRouteWarps * 32) k_route(const T* logits, const __grid_constant__ RouteArgs a) {
  extern __shared__ uint32_t mask[];   // [experts][2]
  __shared__ uint32_t s_empty;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (a.counts) {
    for (uint32_t i = threadIdx.x; i < a.experts * 2; i += blockDim.x) mask[i] = 0;
    if (threadIdx.x == 0) s_empty = 0;
    __syncthreads();
  }
  for (uint32_t n = warp; n < kTile; n += kRouteWarps) {
    const uint64_t t = uint64_t(blockIdx.x) * kTile + n;
    if (t >= a.tokens) break;
    const T* row = logits + t * a.stride;
    float z[PER], top = -INFINITY;
    uint32_t free = 0;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t e = 32 * i + lane;
      z[i] = e < a.experts ? Elem<T>::get(row[e]) : -INFINITY;
      bad |= !(z[i] < INFINITY);
      free |= uint32_t(z[i] > -INFINITY) << i;
      top = fmaxf(top, z[i]);
    }
    bad = __any_sync(kAll, bad);
    top = unsorted(warp_max(sortable(top)));
    uint32_t bits = 0;
    if (!bad) {
      uint32_t key[PER], low, next;
      if (!a.bias && a.best == 1) {   // scores ascend with the logits: these are exact keys
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = free >> i & 1 ? sortable(z[i]) : 0;
        if (a.groups > 1) keep_groups<PER, float>(key, a, 0.0f);
        bits = choose<PER>(key, a.k, &low, &next);
      } else {
        // How far two keys, or two sums of two keys, may be off together.  A softmax score is off by at most 41 roundings of itself (37 of
        // them in the sum of up to 1024 terms), a sigmoid by 4; scores of a softmax add up to 1 at most, and a rounding is 2^-24: below
        // 2^-17 of the largest score.  The additions: 12 roundings of at most the largest key, below 2^-20 of it.
        const float most = make_keys<PER, float>(z, free, top, a, key);
        float big = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (key[i]) big = fmaxf(big, fabsf(unsorted(key[i])));
        big = unsorted(warp_max(sortable(big)));
        const float slack = (a.sigmoid ? 0x1p-19f : 0x1p-17f) * most + 0x1p-20f * big;
        bool close = false;
        if (a.groups > 1) close = keep_groups<PER, float>(key, a, slack);
        bits = choose<PER>(key, a.k, &low, &next);
        close |= next != 0 && unsorted(low) - unsorted(next) <= slack;
        if (close) bits = choose_exactly<PER>(z, free, top, a);
      }
    }
    // weights: scores of the chosen, taken relative to the largest where they are divided by their sum
    float ref = top;   // sigmoid, renormalised: the largest min(z, 0) of the chosen
    if (a.renorm) {
      ref = -INFINITY;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (bits >> i & 1) ref = fmaxf(ref, a.sigmoid ? fminf(z[i], 0.0f) : z[i]);
      ref = unsorted(warp_max(sortable(ref)));
    }
    float s[PER], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool counts = a.renorm ? bits >> i & 1 : (a.sigmoid ? bits >> i & 1 : free >> i & 1);
      s[i] = 0.0f;
      if (counts) s[i] = a.sigmoid ? expf(fminf(z[i], 0.0f) - (a.renorm ? ref : 0.0f)) / (1.0f + expf(-fabsf(z[i]))) : expf(z[i] - ref);
      sum += s[i];
    }
    const float by = a.sigmoid && !a.renorm ? 1.0f : warp_sum(sum);
    uint32_t base = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t b = __ballot_sync(kAll, bits >> i & 1);
      if (bits >> i & 1) {
        const uint32_t e = 32 * i + lane, j = base + __popc(b & ((1u << lane) - 1));
        a.expert[t * a.k + j] = e;
        a.weight[t * a.k + j] = s[i] / by * a.scale;
        if (a.counts) atomicOr(&mask[2 * e + n / 32], 1u << (n % 32));
      }
      base += __popc(b);
    }
    for (uint32_t j = base + lane; j < a.k; j += 32) {
      a.expert[t * a.k + j] = DGS_NO_EXPERT;
      a.weight[t * a.k + j] = bad ? NAN : 0.0f;
    }
    if (a.counts && lane == 0 && base < a.k) atomicAdd(&s_empty, a.k - base);
  }
  if (!a.counts) return;
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < a.experts; e += blockDim.x)
    a.counts[uint64_t(e) * a.tiles + blockIdx.x] = __popc(mask[2 * e]) + __popc(mask[2 * e + 1]);
  if (threadIdx.x == 0) a.counts[uint64_t(a.experts) * a.tiles + blockIdx.x] = s_empty;
}

// One CTA per expert (and one for the empty slots): the counts of its tiles become sums over the tiles before, the total goes to offsets[e].
__global__ void __launch_bounds__(256) k_route_sums(const __grid_constant__ RouteArgs a) {
  __shared__ uint32_t warp_total[8];
  uint32_t* c = a.counts + uint64_t(blockIdx.x) * a.tiles;
  uint32_t before = 0;
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  for (uint32_t first = 0; first < a.tiles; first += 256) {
    const uint32_t i = first + threadIdx.x, v = i < a.tiles ? c[i] : 0;
    uint32_t sum = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t o = __shfl_up_sync(kAll, sum, d);
      if (lane >= uint32_t(d)) sum += o;
    }
    if (lane == 31) warp_total[warp] = sum;
    __syncthreads();
    uint32_t base = before;
    for (uint32_t w = 0; w < 8; ++w) {
      if (w < warp) base += warp_total[w];
      before += warp_total[w];
    }
    if (i < a.tiles) c[i] = base + sum - v;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.offsets[blockIdx.x < a.experts ? blockIdx.x + 1 : 0] = before;
}

// Places a tile's slots.  A slot's place is what lies before its expert's list, before the tile in that list and before the token in
// the tile: the first from the experts' totals, the second from k_route_sums, the third from the bit mask.
__global__ void __launch_bounds__(256) k_route_place(const __grid_constant__ RouteArgs a) {
  extern __shared__ uint32_t shared[];
  uint32_t* mask = shared;                     // [experts][2]
  uint32_t* begin = shared + 2 * a.experts;    // [experts + 1]
  __shared__ uint32_t warp_total[8], s_before;
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  for (uint32_t i = threadIdx.x; i < 2 * a.experts; i += 256) mask[i] = 0;
  const uint32_t first = blockIdx.x * kTile, tokens = min(kTile, a.tokens - first), slots = tokens * a.k;
  const uint32_t* expert = a.expert + uint64_t(first) * a.k;
  // totals to sums over the experts before: offsets[e + 1] still holds the total of e, the first CTA to finish must not disturb it,
  // so the sums are written by k_route_offsets behind this kernel
  uint32_t before = 0;
  for (uint32_t e0 = 0; e0 <= a.experts; e0 += 256) {
    const uint32_t e = e0 + threadIdx.x, v = e < a.experts ? a.offsets[e + 1] : 0;
    uint32_t sum = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t o = __shfl_up_sync(kAll, sum, d);
      if (lane >= uint32_t(d)) sum += o;
    }
    if (lane == 31) warp_total[warp] = sum;
    __syncthreads();
    uint32_t base = before;
    for (uint32_t w = 0; w < 8; ++w) {
      if (w < warp) base += warp_total[w];
      before += warp_total[w];
    }
    if (e <= a.experts) begin[e] = base + sum - v;
    __syncthreads();
  }
  if (threadIdx.x == 0) s_before = begin[a.experts] + a.counts[uint64_t(a.experts) * a.tiles + blockIdx.x];
  for (uint32_t i = threadIdx.x; i < slots; i += 256) {
    const uint32_t e = expert[i], n = i / a.k;
    if (e < a.experts) atomicOr(&mask[2 * e + n / 32], 1u << (n % 32));
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < slots; i += 256) {
    const uint32_t e = expert[i], n = i / a.k;
    const uint64_t slot = uint64_t(first) * a.k + i;
    if (e < a.experts) {
      const uint32_t m0 = mask[2 * e], m1 = mask[2 * e + 1];
      const uint32_t rank = n < 32 ? __popc(m0 & ((1u << n) - 1)) : __popc(m0) + __popc(m1 & ((1u << (n - 32)) - 1));
      const uint32_t at = begin[e] + a.counts[uint64_t(e) * a.tiles + blockIdx.x] + rank;
      a.order[at] = uint32_t(slot);
      a.place[slot] = at;
    } else {
      a.place[slot] = DGS_NO_EXPERT;
    }
  }
  // order behind the last list: as many entries as the tile has empty slots
  const uint32_t from = s_before;
  const uint32_t to = begin[a.experts] + (blockIdx.x + 1 < a.tiles ? a.counts[uint64_t(a.experts) * a.tiles + blockIdx.x + 1] : a.offsets[0]);
  for (uint32_t i = from + threadIdx.x; i < to; i += 256) a.order[i] = DGS_NO_EXPERT;
}

// Totals to offsets, in place, by one CTA.
__global__ void __launch_bounds__(1024) k_route_offsets(uint32_t* offsets, uint32_t experts) {
  __shared__ uint32_t warp_total[32];
  const uint32_t e = threadIdx.x, lane = e % 32, warp = e / 32;
  uint32_t sum = e < experts ? offsets[e + 1] : 0;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint32_t o = __shfl_up_sync(kAll, sum, d);
    if (lane >= uint32_t(d)) sum += o;
  }
  if (lane == 31) warp_total[warp] = sum;
  __syncthreads();
  for (uint32_t w = 0; w < warp; ++w) sum += warp_total[w];
  if (e < experts) offsets[e + 1] = sum;
  if (e == 0) offsets[0] = 0;
}

// ---- gradient ---------------------------------------------------------------------------------
// g_j = scale * dweight_j.  softmax: dz_e = s_e ([e chosen] g_e - sum_j g_j s_j); renormalised dz_l = p_l (g_l - sum g p) on the chosen only (p the
// weights without scale); sigmoid: dz_l = g_l s_l (1 - s_l); renormalised: p_l (g_l - sum g p)(1 - s_l).
template <int PER, class T>
__global__ void __launch_bounds__(256) k_route_grad(const T* logits, T* dlogits, uint64_t dstride, const uint32_t* expert, const float* dweight,
                                                    const __grid_constant__ RouteArgs a, int* status) {
  const uint32_t lane = threadIdx.x % 32;
  for (uint64_t t = uint64_t(blockIdx.x) * 8 + threadIdx.x / 32; t < a.tokens; t += uint64_t(gridDim.x) * 8) {
    const T* row = logits + t * a.stride;
    float z[PER], g[PER], top = -INFINITY;
    bool bad = false;
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t e = 32 * i + lane;
      z[i] = e < a.experts ? Elem<T>::get(row[e]) : -INFINITY;
      bad |= !(z[i] < INFINITY);
      top = fmaxf(top, z[i]);
      g[i] = 0.0f;
    }
    bad = __any_sync(kAll, bad);
    uint32_t mine = DGS_NO_EXPERT;
    float grad = 0.0f;
    if (lane < a.k) {
      mine = expert[t * a.k + lane];
      grad = dweight[t * a.k + lane] * a.scale;
      if (mine >= a.experts && mine != DGS_NO_EXPERT) report(status, DGS_EINVAL);
    }
    for (uint32_t j = 0; j < a.k; ++j) {
      const uint32_t e = __shfl_sync(kAll, mine, j);
      const float v = __shfl_sync(kAll, grad, j);
      if (e % 32 != lane) continue;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (e / 32 == uint32_t(i) && z[i] > -INFINITY) g[i] += v, bits |= 1u << i;
    }
    __syncwarp();
    float ref = top;
    if (a.renorm) {
      ref = -INFINITY;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (bits >> i & 1) ref = fmaxf(ref, a.sigmoid ? fminf(z[i], 0.0f) : z[i]);
    }
    ref = unsorted(warp_max(sortable(ref)));
    float p[PER], sum = 0.0f, pull = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool counts = a.renorm || a.sigmoid ? bits >> i & 1 : z[i] > -INFINITY;
      p[i] = 0.0f;
      if (counts) p[i] = a.sigmoid ? expf(fminf(z[i], 0.0f) - (a.renorm ? ref : 0.0f)) / (1.0f + expf(-fabsf(z[i]))) : expf(z[i] - ref);
      sum += p[i];
      pull += g[i] * p[i];
    }
    const bool plain = a.sigmoid && !a.renorm;
    sum = plain ? 1.0f : warp_sum(sum);
    pull = plain ? 0.0f : warp_sum(pull);
    const float by = sum > 0.0f ? 1.0f / sum : 0.0f;
    pull *= by;
    T* out = dlogits + t * dstride;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t e = 32 * i + lane;
      float d = p[i] * by * (g[i] - pull);
      if (a.sigmoid && (bits >> i & 1)) {
        const float q = expf(-fabsf(z[i]));
        d *= (z[i] > 0.0f ? q : 1.0f) / (1.0f + q);
      }
      if (bad) d = NAN;
      if (e < a.experts) out[e] = Elem<T>::put(d);
    }
  }
}

// ---- host side --------------------------------------------------------------------------------
bool router_ok(const dgs_router* r, uint64_t tokens, uint32_t experts) {
  if (!r || experts == 0 || experts > DGS_ROUTE_MAX_EXPERTS || r->k == 0 || r->k > DGS_ROUTE_MAX_K || r->score > DGS_SCORE_SIGMOID ||
      r->renormalise > 1 || !std::isfinite(r->scale) || r->groups == 0 || experts % r->groups || r->groups_kept == 0 ||
      r->groups_kept > r->groups || r->group_best == 0 || r->group_best > 2)
    return false;
  return r->k <= experts / r->groups * r->groups_kept;
}
bool route_fits(const dgs_router* r, uint64_t tokens) { return tokens <= 0x7fffffffull / r->k; }

RouteArgs route_args(const dgs_router* r, const dgs_matrix* logits) {
  RouteArgs a = {};
  a.stride = logits->stride;
  a.tokens = uint32_t(logits->rows);
  a.experts = logits->cols;
  a.k = r->k;
  a.groups = r->groups;
  a.group_size = a.experts / a.groups;
  a.kept = r->groups_kept;
  a.best = r->groups > 1 ? r->group_best : 1;   // one group is kept whatever its key
  a.tiles = (a.tokens + kTile - 1) / kTile;
  a.sigmoid = r->score == DGS_SCORE_SIGMOID;
  a.renorm = r->renormalise != 0;
  a.scale = r->scale;
  return a;
}

template <class F>
int with_per(uint32_t experts, F&& f) {
  if (experts <= 32) return f(std::integral_constant<int, 1>());
  if (experts <= 64) return f(std::integral_constant<int, 2>());
  if (experts <= 128) return f(std::integral_constant<int, 4>());
  if (experts <= 256) return f(std::integral_constant<int, 8>());
  if (experts <= 512) return f(std::integral_constant<int, 16>());
  return f(std::integral_constant<int, 32>());
}

int launched() { return cudaGetLastError() == cudaSuccess ? DGS_OK : DGS_ECUDA; }

}  // namespace
}  // namespace dgs

using namespace dgs;

extern "C" int dgs_route_experts_bytes(const dgs_router* router, uint64_t tokens, uint32_t experts, uint64_t* out_bytes) {
  if (!out_bytes || !router_ok(router, tokens, experts)) return DGS_EINVAL;
  if (!route_fits(router, tokens)) return DGS_ELIMIT;
  *out_bytes = (uint64_t(experts) + 1) * ((tokens + kTile - 1) / kTile) * 4;
  return DGS_OK;
}

extern "C" int dgs_route_experts(const dgs_router* router, const dgs_matrix* logits, const float* bias, uint32_t* expert, float* weight,
                                 uint32_t* offsets, uint32_t* order, uint32_t* place, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!matrix_ok(logits, false) || !router_ok(router, logits->rows, logits->cols)) return DGS_EINVAL;
  if (!route_fits(router, logits->rows)) return DGS_ELIMIT;
  const bool lists = offsets || order || place;
  const uint64_t slots = logits->rows * router->k;
  if ((slots && (!expert || !weight)) || !aligned(expert, 4) || !aligned(weight, 4) || !aligned(bias, 4)) return DGS_EINVAL;
  if (lists && (!offsets || (slots && (!order || !place)) || !aligned(offsets, 4) || !aligned(order, 4) || !aligned(place, 4))) return DGS_EINVAL;
  uint64_t need = 0;
  dgs_route_experts_bytes(router, logits->rows, logits->cols, &need);
  if (lists && need && (!workspace || !aligned(workspace, 16))) return DGS_EINVAL;
  if (lists && workspace_bytes < need) return DGS_ENOMEM;
  const struct { const void* p; uint64_t n; bool out; } part[] = {
      {logits->data, span_bytes(logits), false}, {bias, bias ? logits->cols * 4ull : 0, false}, {expert, slots * 4, true}, {weight, slots * 4, true},
      {offsets, lists ? (logits->cols + 1) * 4ull : 0, true}, {order, lists ? slots * 4 : 0, true}, {place, lists ? slots * 4 : 0, true},
      {workspace, lists ? need : 0, true}};
  for (const auto& x : part)
    for (const auto& y : part)
      if (&x != &y && x.out && overlap(x.p, x.n, y.p, y.n)) return DGS_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  RouteArgs a = route_args(router, logits);
  if (a.tokens == 0) {
    if (!lists) return DGS_OK;
    return cudaMemsetAsync(offsets, 0, (a.experts + 1) * 4ull, st) == cudaSuccess ? DGS_OK : DGS_ECUDA;
  }
  a.bias = bias;
  a.expert = expert;
  a.weight = weight;
  a.offsets = offsets;
  a.order = order;
  a.place = place;
  a.counts = lists ? static_cast<uint32_t*>(workspace) : nullptr;
  const int rc = with_type(logits->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return with_per(a.experts, [&](auto per) {
      k_route<per.value, T><<<a.tiles, kRouteWarps * 32, a.experts * 8, st>>>(static_cast<const T*>(logits->data), a);
      return launched();
    });
  });
  if (rc != DGS_OK || !lists) return rc;
  k_route_sums<<<a.experts + 1, 256, 0, st>>>(a);
  if (launched() != DGS_OK) return DGS_ECUDA;
  k_route_place<<<a.tiles, 256, (3 * a.experts + 1) * 4, st>>>(a);
  if (launched() != DGS_OK) return DGS_ECUDA;
  k_route_offsets<<<1, 1024, 0, st>>>(offsets, a.experts);
  return launched();
}

extern "C" int dgs_route_experts_grad(const dgs_router* router, const dgs_matrix* logits, const uint32_t* expert, const float* dweight,
                                      const dgs_matrix* dlogits, void* stream) {
  if (!matrix_ok(logits, false) || !matrix_ok(dlogits, true) || !router_ok(router, logits->rows, logits->cols)) return DGS_EINVAL;
  if (!route_fits(router, logits->rows)) return DGS_ELIMIT;
  if (dlogits->rows != logits->rows || dlogits->cols != logits->cols || dlogits->type != logits->type) return DGS_EINVAL;
  if (logits->rows == 0) return DGS_OK;
  const uint64_t slots = logits->rows * router->k;
  if (!expert || !dweight || !aligned(expert, 4) || !aligned(dweight, 4)) return DGS_EINVAL;
  if ((!same_matrix(logits, dlogits) && overlap(logits->data, span_bytes(logits), dlogits->data, span_bytes(dlogits))) ||
      overlap(expert, slots * 4, dlogits->data, span_bytes(dlogits)) || overlap(dweight, slots * 4, dlogits->data, span_bytes(dlogits)))
    return DGS_EINVAL;
  int* status = operator_status_word();
  if (!status) return DGS_ECUDA;
  const RouteArgs a = route_args(router, logits);
  return with_type(logits->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return with_per(a.experts, [&](auto per) {
      const uint32_t ctas = std::min<uint32_t>((a.tokens + 7) / 8, kSms * 16);
      k_route_grad<per.value, T><<<ctas, 256, 0, static_cast<cudaStream_t>(stream)>>>(
          static_cast<const T*>(logits->data), static_cast<T*>(dlogits->data), dlogits->stride, expert, dweight, a, status);
      return launched();
    });
  });
}
