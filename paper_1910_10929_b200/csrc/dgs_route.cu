// The router of a model with experts: dgs_route_experts and dgs_route_experts_grad.
#include "dgs_operators.cuh"

#include <algorithm>
#include <cmath>

namespace dgs {
namespace {

constexpr uint32_t kTile = 64;           // tokens of a CTA: two words of a bit mask per expert
// Warps of a CTA: each takes some of the tile's tokens one after the other (8192 tokens of 60 experts: 21 us with 8 warps,
// 10 with 32; 65536 of 256: 113 and 97).  Rows beyond 256 experts need more registers than 32 warps have.
__host__ __device__ constexpr uint32_t route_warps(int per) { return per <= 8 ? 32 : 8; }
constexpr uint32_t kAll = 0xffffffffu;

struct RouteArgs {
  uint64_t stride;
  uint32_t tokens, experts, k, groups, group_size, kept, best, tiles;
  bool sigmoid, renorm, wide;
  float scale;
  const float* bias;
  uint32_t* expert;
  float* weight;
  uint32_t* offsets;
  uint32_t* order;
  uint32_t* place;
  uint32_t* counts;    // [experts + 1][tiles]: slots of a tile that belong to an expert, then those of the tiles before; behind the last
                       // expert: empty slots.  NULL: no lists, or a single tile
  uint32_t* totals;    // [experts + 1]
};

// Numbers whose unsigned order is the order of the floats; 0 stands for "not there" (below -inf).
__device__ __forceinline__ uint32_t sortable(float v) {
  const int b = __float_as_int(v + 0.0f);   // -0 and +0 are equal keys
  return uint32_t(b ^ (b >> 31 | int(0x80000000)));
}
__device__ __forceinline__ unsigned long long sortable(double v) {
  const long long b = __double_as_longlong(v + 0.0);
  return (unsigned long long)(b ^ (b >> 63 | (long long)0x8000000000000000ull));
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
// Sum over the lanes before.
__device__ __forceinline__ uint32_t lanes_before(uint32_t v) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t sum = v;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint32_t o = __shfl_up_sync(kAll, sum, d);
    if (lane >= uint32_t(d)) sum += o;
  }
  return sum - v;
}

// Lane l has experts l * PER to l * PER + PER - 1, in its registers: experts ascend with the lanes and in each.
// Which of its keys a lane holds among the `count` largest of the warp (bit i: key i), ties to the lowest index.  low / next: the
// smallest key chosen and the largest left.
// sorted: PER * 32 words of the warp's own (PER of 2 to 8).
template <int PER, class K>
__device__ __forceinline__ uint32_t choose(const K (&key)[PER], uint32_t count, uint32_t* sorted, K* low, K* next) {
  K border = ~K(0), left = 0;
  if constexpr (PER <= 8 && sizeof(K) == 4) {
    // the lane's keys in descending order; round by round the largest of the lanes' first ones are taken off.  They are kept in shared memory:
    // moved up through registers they make three times the code, and the kernel waits for instructions as it is.
    K s[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) s[i] = key[i];
#pragma unroll
    for (int size = 2; size <= PER; size *= 2)
#pragma unroll
      for (int d = size / 2; d; d /= 2)
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if ((i & d) == 0) {
            const K x = s[i], y = s[i + d];
            const bool down = (i & size) == 0;
            s[i] = down ? max(x, y) : min(x, y);
            s[i + d] = down ? min(x, y) : max(x, y);
          }
    uint32_t* behind = sorted + (threadIdx.x & 31);
    if constexpr (PER > 1) {
#pragma unroll
      for (int i = 1; i < PER; ++i) behind[i * 32 - 32] = s[i];
      behind[PER * 32 - 32] = 0;
    }
    uint32_t taken = 0;
    bool more = true;
#pragma unroll 1
    while (more) {
#pragma unroll
      for (int q = 0; q < (PER > 1 ? 4 : 2); ++q) {   // rounds without a branch: those too many change nothing
        const K m = warp_max(s[0]);
        more = taken < count && m != 0;   // 0: fewer than `count` are there
        const bool mine = more && s[0] == m;
        border = more ? m : border;
        taken += __popc(__ballot_sync(kAll, mine));
        if constexpr (PER > 1) {
          if (mine) s[0] = *behind;
          behind += mine ? 32 : 0;
        } else {
          s[0] = mine ? K(0) : s[0];
        }
      }
    }
    left = s[0];
  } else {
    uint32_t taken = 0;
    for (;;) {   // the distinct keys in descending order until `count` are reached: at most `count` rounds
      K m = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) m = key[i] < border && key[i] > m ? key[i] : m;
      m = warp_max(m);
      if (m == 0) break;
      border = m;
      uint32_t level = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) level += key[i] == m;
      taken += __reduce_add_sync(kAll, level);
      if (taken >= count) break;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) left = key[i] < border && key[i] > left ? key[i] : left;
  }
  uint32_t bits = 0, ties = 0;
  if (border != ~K(0)) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (key[i] > border) bits |= 1u << i;
      if (key[i] == border) ties |= 1u << i;
    }
  }
  *low = border;
  const uint32_t above = __reduce_add_sync(kAll, uint32_t(__popc(bits))), level = __reduce_add_sync(kAll, uint32_t(__popc(ties)));
  if (above + level <= count) {
    bits |= ties;
    *next = warp_max(left);
  } else {   // more keys of the border's size than are left to take
    const uint32_t before = above + lanes_before(__popc(ties)), take = before < count ? count - before : 0;
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if ((ties >> i & 1) && uint32_t(__popc(ties & ((1u << i) - 1))) < take) mine |= 1u << i;
    bits |= mine;
    *next = border;
  }
  return bits;
}

// A group's key from the two largest of its experts' keys; 0: no expert left in it.
template <class R, class K>
__device__ __forceinline__ K group_key(K first, K second, uint32_t best) {
  return first == 0 || best == 1 || second == 0 ? first : sortable(unsorted(first) + unsorted(second));
}

// Leaves only the keys of the kept groups; true if the border between kept and dropped groups is no wider than `slack`.
template <int PER, class R, class K>
__device__ __forceinline__ bool keep_groups(K (&key)[PER], const RouteArgs& a, R slack, uint32_t* sorted) {
  const uint32_t lane = threadIdx.x & 31;
  const uint32_t lanes = a.group_size / PER;
  K low, next;
  if (lanes && a.group_size % PER == 0 && (lanes & (lanes - 1)) == 0 && a.groups <= 32) {
    // groups of 1, 2, 4 .. lanes: the two largest by lane, then across them
    K first = 0, second = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      second = max(second, min(first, key[i]));
      first = max(first, key[i]);
    }
    for (uint32_t d = 1; d < lanes; d *= 2) {
      const K f = __shfl_xor_sync(kAll, first, d), s = __shfl_xor_sync(kAll, second, d);
      second = max(max(second, s), min(first, f));
      first = max(first, f);
    }
    // lane g takes group g's, so that their order is the lanes'
    const K mine = __shfl_sync(kAll, group_key<R, K>(first, second, a.best), (lane * lanes) & 31);
    const K one[1] = {lane < a.groups ? mine : K(0)};
    const uint32_t kept = __ballot_sync(kAll, choose<1, K>(one, a.kept, sorted, &low, &next));
    if (!(kept >> (lane / lanes) & 1))
#pragma unroll
      for (int i = 0; i < PER; ++i) key[i] = 0;
  } else {
    K mine[PER];   // lane l has groups l * PER and so on: at most as many as experts
#pragma unroll
    for (int i = 0; i < PER; ++i) mine[i] = 0;
    for (uint32_t g = 0; g < a.groups; ++g) {
      const uint32_t lo = g * a.group_size, hi = lo + a.group_size;
      K first = 0, second = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const uint32_t e = lane * PER + i;
        const K v = e >= lo && e < hi ? key[i] : K(0);
        second = max(second, min(first, v));
        first = max(first, v);
      }
      const K top = warp_max(first);
      const uint32_t at = __ballot_sync(kAll, first == top);
      if (lane == uint32_t(__ffs(at)) - 1) first = second;   // the largest leaves once
      const K v = group_key<R, K>(top, warp_max(first), a.best);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (lane * PER + i == g) mine[i] = v;
    }
    const uint32_t bits = choose<PER, K>(mine, a.kept, sorted, &low, &next);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t e = lane * PER + i, g = e < a.experts ? e / a.group_size : 0;
      const uint32_t b = __shfl_sync(kAll, bits, g / PER);
      if (!(b >> (g % PER) & 1)) key[i] = 0;
    }
  }
  return next != 0 && R(unsorted(low)) - R(unsorted(next)) <= slack;
}

template <int PER, class T>
__device__ __forceinline__ void read_logits(const T* row, const RouteArgs& a, float (&z)[PER]) {
  const uint32_t e0 = (threadIdx.x & 31) * PER;
  constexpr uint32_t bytes = PER * sizeof(T), width = bytes < 16 ? bytes : 16, each = width / sizeof(T);
  if constexpr (PER > 1) {
    if (a.wide && e0 + PER <= a.experts) {
#pragma unroll
      for (int i = 0; i < PER; i += each) {
        T t[each];
        if constexpr (width == 16) {
          const uint4 w = __ldcs(reinterpret_cast<const uint4*>(row + e0 + i));
          memcpy(t, &w, 16);
        } else if constexpr (width == 8) {
          const uint2 w = __ldcs(reinterpret_cast<const uint2*>(row + e0 + i));
          memcpy(t, &w, 8);
        } else {
          const uint32_t w = __ldcs(reinterpret_cast<const uint32_t*>(row + e0 + i));
          memcpy(t, &w, 4);
        }
#pragma unroll
        for (uint32_t q = 0; q < each; ++q) z[i + q] = Elem<T>::get(t[q]);
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) z[i] = e0 + i < a.experts ? Elem<T>::get(row[e0 + i]) : -INFINITY;
}

// The choice in 64 bits, as it is defined, for tokens whose border 32 bits cannot tell: rare, and kept out of line.
template <int PER, class T>
__device__ __noinline__ uint32_t choose_exactly(const T* row, const RouteArgs& a, float* top) {
  const uint32_t lane = threadIdx.x & 31;
  float z[PER];
  read_logits<PER>(row, a, z);
  float most = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) most = fmaxf(most, z[i]);
  *top = unsorted(warp_max(sortable(most)));
  double sum = 1.0;
  if (!a.sigmoid) {
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += exp(double(z[i]) - double(*top));
    sum = warp_sum(sum);
  }
  unsigned long long key[PER], low, next;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const double s = a.sigmoid ? 1.0 / (1.0 + exp(-double(z[i]))) : exp(double(z[i]) - double(*top)) / sum;
    key[i] = z[i] > -INFINITY ? sortable(s + (a.bias ? double(a.bias[lane * PER + i]) : 0.0)) : 0;
  }
  if (a.groups > 1) keep_groups<PER, double>(key, a, 0.0, nullptr);
  return choose<PER>(key, a.k, nullptr, &low, &next);
}

// Sums over the entries before, of n values that the threads of a CTA hold in turns: f(i, value, sum before) for each.
template <class V, class F>
__device__ __forceinline__ uint32_t sums_before(uint32_t n, V&& value, F&& f) {
  __shared__ uint32_t warp_total[32];
  uint32_t before = 0;
  const uint32_t warp = threadIdx.x / 32, warps = blockDim.x / 32;
  for (uint32_t first = 0; first < n; first += blockDim.x) {
    const uint32_t i = first + threadIdx.x, v = i < n ? value(i) : 0, sum = lanes_before(v);
    if (threadIdx.x % 32 == 31) warp_total[warp] = sum + v;
    __syncthreads();
    uint32_t base = before;
    for (uint32_t w = 0; w < warps; ++w) {
      if (w < warp) base += warp_total[w];
      before += warp_total[w];
    }
    if (i < n) f(i, v, base + sum);
    __syncthreads();
  }
  return before;
}

// Places a tile's slots.  A slot's place is what lies before its expert's list (begin), before the tile in that list (earlier) and before the
// token in the tile: the tokens that the expert's bit mask marks.
template <class B>
__device__ __forceinline__ void place_tile(const RouteArgs& a, uint32_t tile, const uint32_t* mask, B&& begin) {
  const uint32_t first = tile * kTile, slots = min(kTile, a.tokens - first) * a.k;
  const uint32_t* expert = a.expert + uint64_t(first) * a.k;
  for (uint32_t i = threadIdx.x; i < slots; i += blockDim.x) {
    const uint32_t e = expert[i], n = i / a.k;
    const uint64_t slot = uint64_t(first) * a.k + i;
    uint32_t at = DGS_NO_EXPERT;
    if (e < a.experts) {
      const uint32_t m0 = mask[2 * e], m1 = mask[2 * e + 1];
      at = begin(e) + (n < 32 ? __popc(m0 & ((1u << n) - 1)) : __popc(m0) + __popc(m1 & ((1u << (n - 32)) - 1)));
      a.order[at] = uint32_t(slot);
    }
    a.place[slot] = at;
  }
}

// One warp per token, a tile of 64 tokens per CTA.  The token's logits stay in registers.  The experts chosen are marked in a bit mask per
// expert (bit = token of the tile), whose counts are what a later kernel needs to place the tile's slots; a single tile is placed here.
// Bound by instructions: about 1000 a token of 256 experts with groups and a bias (97 us for 65536 tokens, whose reading takes 10), 530 for 60 experts
// without; a token's chain of maxima over the warp is hidden by the other warps only.
template <int PER, class T>
__global__ void __launch_bounds__(route_warps(PER) * 32, 1) k_route(const T* logits, const __grid_constant__ RouteArgs a) {
  extern __shared__ uint32_t mask[];   // [experts][2]
  __shared__ uint32_t s_empty;
  constexpr uint32_t MOST = route_warps(PER);
  const uint32_t warps = blockDim.x / 32;
  __shared__ uint32_t s_slot[MOST][DGS_ROUTE_MAX_K];   // the experts of a token's slots
  __shared__ uint32_t s_sorted[MOST][PER <= 8 ? PER * 32 : 1];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  uint32_t* const sorted = s_sorted[warp];
  const bool lists = a.offsets != nullptr;
  if (lists) {
    for (uint32_t i = threadIdx.x; i < a.experts * 2; i += blockDim.x) mask[i] = 0;
    if (threadIdx.x == 0) s_empty = 0;
    __syncthreads();
  }
  const bool exact = !a.bias && a.best == 1;   // scores ascend with the logits, which are then exact keys
  float bias[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) bias[i] = a.bias && lane * PER + i < a.experts ? a.bias[lane * PER + i] : 0.0f;
  float most_bias = 0.0f;
#pragma unroll
  for (int i = 0; i < PER; ++i) most_bias = fmaxf(most_bias, fabsf(bias[i]));
  most_bias = __uint_as_float(warp_max(__float_as_uint(most_bias)));
  // Slots, weights and marks of a token whose choice is made.
  const auto finish = [&](uint32_t n, uint64_t t, uint32_t bits, bool bad, float top, float sum) {
    // the chosen, in order, one a lane
    const uint32_t mine = __popc(bits), before = lanes_before(mine), chosen = __shfl_sync(kAll, before + mine, 31);
    uint32_t* to = s_slot[warp] + before;
    for (uint32_t left = bits; left; left &= left - 1) *to++ = lane * PER + __ffs(left) - 1;
    __syncwarp();
    const bool there = lane < chosen;
    const uint32_t slot = there ? s_slot[warp][lane] : DGS_NO_EXPERT;
    const float zs = there ? Elem<T>::get(logits[t * a.stride + slot]) : -INFINITY;   // still in the first cache
    __syncwarp();
    // weights: relative to the largest where they are divided by their sum
    float w = 0.0f;
    if (a.sigmoid) {
      float ref = 0.0f;
      if (a.renorm) ref = unsorted(warp_max(sortable(fminf(zs, 0.0f))));
      if (there) w = expf(fminf(zs, 0.0f) - ref) / (1.0f + expf(-fabsf(zs)));
      if (a.renorm) w = w / warp_sum(w);
    } else {
      const float ref = a.renorm ? unsorted(warp_max(sortable(zs))) : top;
      if (there) w = expf(zs - ref);
      w = w / (a.renorm ? warp_sum(w) : sum);
    }
    if (lane < a.k) {
      a.expert[t * a.k + lane] = slot;
      a.weight[t * a.k + lane] = there ? w * a.scale : bad ? NAN : 0.0f;
    }
    if (lists) {
      if (there) atomicOr(&mask[2 * slot + n / 32], 1u << (n % 32));
      if (lane == 0 && chosen < a.k) atomicAdd(&s_empty, a.k - chosen);
    }
  };
  uint32_t again = 0;   // the warp's tokens to be chosen for in 64 bits
  for (uint32_t n = warp; n < kTile; n += warps) {
    const uint64_t t = uint64_t(blockIdx.x) * kTile + n;
    if (t >= a.tokens) break;
    float z[PER], top = -INFINITY;
    read_logits<PER>(logits + t * a.stride, a, z);
    uint32_t free = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (z[i] > -INFINITY) free |= 1u << i;
      asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(z[i]));
    }
    const bool bad = __any_sync(kAll, !(top < INFINITY));
    const bool sums = !a.sigmoid && (!exact || !a.renorm);   // whether the softmax over all experts is needed
    if (!a.sigmoid) top = unsorted(warp_max(sortable(top)));
    float s[PER], sum = 0.0f;
    if (sums) {
#pragma unroll
      for (int i = 0; i < PER; ++i) s[i] = free >> i & 1 ? expf(z[i] - top) : 0.0f, sum += s[i];
      sum = warp_sum(sum);
    }
    uint32_t bits = 0;
    if (!bad) {
      uint32_t key[PER], low, next;
      if (exact) {
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = free >> i & 1 ? sortable(z[i]) : 0;
        if (a.groups > 1) keep_groups<PER, float>(key, a, 0.0f, sorted);
        bits = choose<PER>(key, a.k, sorted, &low, &next);
      } else {
        // Keys in 32 bits.  How far two of them, or two sums of two, may be off together, in roundings (2^-24).  Sigmoid: 2 ulp of the
        // hardware's exponential q move s by 4 s (1 - s) <= 1, its argument's roundings by 1.5 |z| s (1 - s) < 0.4, 1 + q is off by 1 s and the
        // reciprocal by 2 s: 4.4, below 2^-20 for two and 2^-19 for four of them.  Softmax: 44 of the score itself, 37 of them in the sum of up
        // to 1024 terms, and two scores are at most 1 together: below 2^-17 of the largest.  The additions: 2, or 12 for two sums, of at most 1 + the
        // largest bias.
        float most = 1.0f;
        if (a.sigmoid) {
#pragma unroll
          for (int i = 0; i < PER; ++i) s[i] = hardware_reciprocal(1.0f + hardware_exp2(z[i] * -1.4426950409f));
        } else {
          most = 1.0f / sum;
#pragma unroll
          for (int i = 0; i < PER; ++i) s[i] *= most;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = free >> i & 1 ? sortable(s[i] + bias[i]) : 0;
        const float slack = a.sigmoid ? 0x1p-20f + 0x1p-23f * (1.0f + most_bias) : 0x1p-17f * most + 0x1p-23f * (most + most_bias);
        const float group_slack = a.sigmoid ? 0x1p-19f + 0x1p-20f * (1.0f + most_bias) : 0x1p-17f * most + 0x1p-20f * (most + most_bias);
        bool groups_close = false;
        if (a.groups > 1) groups_close = keep_groups<PER, float>(key, a, group_slack, sorted);
        bits = choose<PER>(key, a.k, sorted, &low, &next);
        if (groups_close || (next != 0 && unsorted(low) - unsorted(next) <= slack)) {
          again |= 1u << (n / warps);   // afterwards: a call from here would cost every token its registers
          continue;
        }
      }
    }
    finish(n, t, bits, bad, top, sum);
  }
  for (; again; again &= again - 1) {
    const uint32_t n = (__ffs(again) - 1) * warps + warp;
    const uint64_t t = uint64_t(blockIdx.x) * kTile + n;
    float top, sum = 0.0f;
    const uint32_t bits = choose_exactly<PER, T>(logits + t * a.stride, a, &top);
    if (!a.sigmoid && !a.renorm) {
      float z[PER];
      read_logits<PER>(logits + t * a.stride, a, z);
#pragma unroll
      for (int i = 0; i < PER; ++i) sum += expf(z[i] - top);
      sum = warp_sum(sum);
    }
    finish(n, t, bits, false, top, sum);
  }
  if (!lists) return;
  __syncthreads();
  const auto count = [&](uint32_t e) { return __popc(mask[2 * e]) + __popc(mask[2 * e + 1]); };
  if (a.counts) {
    for (uint32_t e = threadIdx.x; e < a.experts; e += blockDim.x) a.counts[uint64_t(e) * a.tiles + blockIdx.x] = count(e);
    if (threadIdx.x == 0) a.counts[uint64_t(a.experts) * a.tiles + blockIdx.x] = s_empty;
  } else {
    uint32_t* begin = mask + 2 * a.experts;
    const uint32_t all = sums_before(a.experts, count, [&](uint32_t e, uint32_t, uint32_t sum) { begin[e] = a.offsets[e] = sum; });
    if (threadIdx.x == 0) a.offsets[a.experts] = all;
    __syncthreads();
    place_tile(a, 0, mask, [&](uint32_t e) { return begin[e]; });
    for (uint32_t i = all + threadIdx.x; i < a.tokens * a.k; i += blockDim.x) a.order[i] = DGS_NO_EXPERT;
  }
}

// One CTA per expert (and one for the empty slots): the counts of its tiles become sums over the tiles before.
__global__ void __launch_bounds__(256) k_route_sums(const __grid_constant__ RouteArgs a) {
  wait_for_last_kernel();
  uint32_t* c = a.counts + uint64_t(blockIdx.x) * a.tiles;
  const uint32_t all = sums_before(a.tiles, [&](uint32_t i) { return c[i]; }, [&](uint32_t i, uint32_t, uint32_t sum) { c[i] = sum; });
  if (threadIdx.x == 0) a.totals[blockIdx.x] = all;
}

__global__ void __launch_bounds__(256) k_route_place(const __grid_constant__ RouteArgs a) {
  extern __shared__ uint32_t mask[];           // [experts][2]
  uint32_t* begin = mask + 2 * a.experts;      // [experts + 1]
  for (uint32_t i = threadIdx.x; i < 2 * a.experts; i += 256) mask[i] = 0;
  wait_for_last_kernel();
  __syncthreads();
  const uint32_t tile = blockIdx.x, first = tile * kTile, slots = min(kTile, a.tokens - first) * a.k;
  const uint32_t* expert = a.expert + uint64_t(first) * a.k;
  for (uint32_t i = threadIdx.x; i < slots; i += 256) {
    const uint32_t e = expert[i], n = i / a.k;
    if (e < a.experts) atomicOr(&mask[2 * e + n / 32], 1u << (n % 32));
  }
  const uint32_t all = sums_before(a.experts, [&](uint32_t e) { return a.totals[e]; }, [&](uint32_t e, uint32_t, uint32_t sum) {
    begin[e] = sum + a.counts[uint64_t(e) * a.tiles + tile];
    if (tile == 0) a.offsets[e] = sum;
  });
  if (tile == 0 && threadIdx.x == 0) a.offsets[a.experts] = all;
  __syncthreads();
  place_tile(a, tile, mask, [&](uint32_t e) { return begin[e]; });
  // order behind the last list: as many entries as the tile has empty slots
  const uint32_t* empty = a.counts + uint64_t(a.experts) * a.tiles;
  const uint32_t from = all + empty[tile], to = all + (tile + 1 < a.tiles ? empty[tile + 1] : a.totals[a.experts]);
  for (uint32_t i = from + threadIdx.x; i < to; i += 256) a.order[i] = DGS_NO_EXPERT;
}

// ---- gradient ---------------------------------------------------------------------------------
// g_j = scale * dweight_j.  softmax: dz_e = s_e ([e chosen] g_e - sum_j g_j s_j); renormalised dz_l = p_l (g_l - sum g p) on the chosen only (p the
// weights without scale); sigmoid: dz_l = g_l s_l (1 - s_l); renormalised: p_l (g_l - sum g p)(1 - s_l).
// CTAs on an SM: as many as are launched, so that all have the same to do (65536 x 256: 36 us, 43 with sixteen that come in turns, 41 with the next
// tokens' slots and logits read ahead).
constexpr uint32_t kGradPerSm = 6;

template <int PER, class T>
__device__ __forceinline__ void write_logits(T* row, const RouteArgs& a, const float (&z)[PER]) {
  const uint32_t e0 = (threadIdx.x & 31) * PER;
  constexpr uint32_t bytes = PER * sizeof(T), width = bytes < 16 ? bytes : 16, each = width / sizeof(T);
  if constexpr (PER > 1) {
    if (a.wide && e0 + PER <= a.experts) {
#pragma unroll
      for (int i = 0; i < PER; i += each) {
        T t[each];
#pragma unroll
        for (uint32_t q = 0; q < each; ++q) t[q] = Elem<T>::put(z[i + q]);
        if constexpr (width == 16) {
          uint4 w;
          memcpy(&w, t, 16);
          __stcs(reinterpret_cast<uint4*>(row + e0 + i), w);
        } else if constexpr (width == 8) {
          uint2 w;
          memcpy(&w, t, 8);
          __stcs(reinterpret_cast<uint2*>(row + e0 + i), w);
        } else {
          uint32_t w;
          memcpy(&w, t, 4);
          __stcs(reinterpret_cast<uint32_t*>(row + e0 + i), w);
        }
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (e0 + i < a.experts) row[e0 + i] = Elem<T>::put(z[i]);
}

// 65536 x 256 in f32: 36 us, half of it writing the rows; bound by the trip from slot to logit to row of each token.
// A slot a lane, then the dense row.  Everything but a softmax without renormalising leaves a row zero outside the chosen, so only
// their logits are read; where an expert is listed twice its gradients add up.
template <int PER, class T>
__global__ void __launch_bounds__(256, PER <= 8 ? kGradPerSm : 1) k_route_grad(const T* logits, T* dlogits, uint64_t dstride, const uint32_t* expert, const float* dweight,
                                                    const __grid_constant__ RouteArgs a, int* status) {
  __shared__ float s_row[8][PER * 32 + 1];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  float* row = s_row[warp];
#pragma unroll
  for (int i = 0; i < PER; ++i) row[lane * PER + i] = 0.0f;
  __syncwarp();
  for (uint64_t t = uint64_t(blockIdx.x) * 8 + warp; t < a.tokens; t += uint64_t(gridDim.x) * 8) {
    const T* from = logits + t * a.stride;
    uint32_t e = DGS_NO_EXPERT;
    float g = 0.0f;
    if (lane < a.k) {
      e = expert[t * a.k + lane];
      g = dweight[t * a.k + lane] * a.scale;
      if (e >= a.experts && e != DGS_NO_EXPERT) report(status, DGS_EINVAL);
    }
    const float ze = e < a.experts ? Elem<T>::get(from[e]) : -INFINITY;
    const bool dense = !a.sigmoid && !a.renorm;
    float z[PER], top = -INFINITY;
    bool bad = !(ze < INFINITY);
    if (dense || !__any_sync(kAll, ze > -INFINITY)) {   // a token without experts may be one with a NaN
      read_logits<PER>(from, a, z);
#pragma unroll
      for (int i = 0; i < PER; ++i) bad |= !(z[i] < INFINITY), top = fmaxf(top, z[i]);
    }
    bad = __any_sync(kAll, bad);
    const bool there = ze > -INFINITY && !bad;
    // an expert listed twice: the first of its lanes takes the gradients of all
    const uint32_t same = __match_any_sync(kAll, there ? e : 0x80000000u + lane);
    const bool leads = there && uint32_t(__ffs(same)) - 1 == lane;
    if (__any_sync(kAll, there && !leads)) {
      float all = 0.0f;
      for (uint32_t j = 0; j < 32; ++j) {
        const float v = __shfl_sync(kAll, g, j);
        if (same >> j & 1) all += v;
      }
      g = all;
    }
    float d = 0.0f;
    if (a.sigmoid) {
      const float q = expf(-fabsf(ze)), slope = (ze > 0.0f ? q : 1.0f) / (1.0f + q);   // 1 - s
      if (a.renorm) {
        const float ref = unsorted(warp_max(sortable(leads ? fminf(ze, 0.0f) : -INFINITY)));
        float p = leads ? expf(fminf(ze, 0.0f) - ref) / (1.0f + q) : 0.0f;
        const float sum = warp_sum(p);
        p = sum > 0.0f ? p / sum : 0.0f;
        const float pull = warp_sum(leads ? g * p : 0.0f);
        d = p * (g - pull) * slope;
      } else {
        d = g * (ze > 0.0f ? 1.0f : q) / (1.0f + q) * slope;
      }
    } else if (a.renorm) {
      const float ref = unsorted(warp_max(sortable(leads ? ze : -INFINITY)));
      float p = leads ? expf(ze - ref) : 0.0f;
      const float sum = warp_sum(p);
      p = sum > 0.0f ? p / sum : 0.0f;
      const float pull = warp_sum(leads ? g * p : 0.0f);
      d = p * (g - pull);
    } else {
      top = unsorted(warp_max(sortable(top)));
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < PER; ++i) z[i] = z[i] > -INFINITY ? expf(z[i] - top) : 0.0f, sum += z[i];
      sum = warp_sum(sum);
      const float by = sum > 0.0f ? 1.0f / sum : 0.0f, p = leads ? expf(ze - top) * by : 0.0f;
      const float pull = warp_sum(leads ? g * p : 0.0f);
      d = p * g;
#pragma unroll
      for (int i = 0; i < PER; ++i) z[i] = -z[i] * by * pull;
    }
    if (leads) row[e] = d;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float v = row[lane * PER + i];
      z[i] = bad ? NAN : dense ? z[i] + v : v;
    }
    __syncwarp();
    if (leads) row[e] = 0.0f;
    __syncwarp();
    write_logits<PER>(dlogits + t * dstride, a, z);
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
  const uint64_t tiles = (tokens + kTile - 1) / kTile;
  *out_bytes = tiles > 1 ? (uint64_t(experts) + 1) * (tiles + 1) * 4 : 0;   // a single tile is placed by the kernel that routes it
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
  a.counts = need ? static_cast<uint32_t*>(workspace) : nullptr;
  a.totals = need ? a.counts + (uint64_t(a.experts) + 1) * a.tiles : nullptr;
  if (!lists) a.offsets = a.counts = nullptr;
  const int rc = with_type(logits->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return with_per(a.experts, [&](auto per) {
      constexpr uint32_t width = per.value * sizeof(T) < 16 ? per.value * sizeof(T) : 16;
      a.wide = aligned(logits->data, width) && logits->stride * sizeof(T) % width == 0;
      k_route<per.value, T><<<a.tiles, std::min(route_warps(per.value), std::max(8u, a.tokens)) * 32, (lists ? 3 * a.experts : 0) * 4, st>>>(static_cast<const T*>(logits->data), a);
      return launched();
    });
  });
  if (rc != DGS_OK || !a.counts) return rc;
  const EarlyLaunch sums(dim3(a.experts + 1), 256, 0, st), placing(dim3(a.tiles), 256, (3 * a.experts + 1) * 4, st);
  if (cudaLaunchKernelEx(&sums.cfg, k_route_sums, a) != cudaSuccess) return DGS_ECUDA;
  return cudaLaunchKernelEx(&placing.cfg, k_route_place, a) == cudaSuccess ? DGS_OK : DGS_ECUDA;
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
  RouteArgs a = route_args(router, logits);
  return with_type(logits->type, [&](auto* t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return with_per(a.experts, [&](auto per) {
      constexpr uint32_t width = per.value * sizeof(T) < 16 ? per.value * sizeof(T) : 16;
      a.wide = aligned(logits->data, width) && logits->stride * sizeof(T) % width == 0 && aligned(dlogits->data, width) &&
               dlogits->stride * sizeof(T) % width == 0;
      const uint32_t ctas = std::min<uint32_t>((a.tokens + 7) / 8, kSms * kGradPerSm);
      k_route_grad<per.value, T><<<ctas, 256, 0, static_cast<cudaStream_t>(stream)>>>(
          static_cast<const T*>(logits->data), static_cast<T*>(dlogits->data), dlogits->stride, expert, dweight, a, status);
      return launched();
    });
  });
}
