// Gating by scores, groups and a balance bias (eb_router), one token by one warp; lane i holds logits i, i+32, ...
//
//   s_e = sigmoid(z_e) or softmax(z)_e;   c_e = s_e + bias[layer][e], what the choice goes by
//   value of a group = the best c_e of its experts, or the sum of the best two; the topk_group best groups stay
//   the K best c_e of these groups; w = scale * s_e, over the sum of the chosen s_e if renormalised
//
// Order is what has to be exact: two c_e that differ by less than a rounding of 32 bits change places otherwise, and with them a
// token's experts.  Without a bias c_e orders like z_e, so the logits are compared (integers in the order of the floats), also where scores in 64 bits
// would be 1 or 0 alike.  A sum, of a
// bias or of two scores, is made and compared in 32 bits first, with a bound on how far it may be off: s_e = 1 / (1 + expf(-z)) is within 2^-21,
// expf(z - top) / sum of at most 256 terms within 2^-19 (e^-d (d + 16) 2^-24, d = top - z), and each sum adds 2^-24 of its size: c_e of its own, the
// value of a group those of its two c_e as well, which with biases of opposite sign are larger than the value.  Where neighbours of the
// order, or a group that stays and one that goes, lie nearer than both bounds, the token is done again in 64 bits.
// 65536 tokens, 256 experts in 8 groups: 389 us in 64 bits throughout, 206 to 209 this way.
#pragma once

#include <cfloat>

#include "eb_route.cuh"

namespace {

__device__ __forceinline__ float logit_value(float z) { return z; }
__device__ __forceinline__ float logit_value(bf16 z) { return __bfloat162float(z); }

// Unsigned integers in the order of the doubles; 0 stands for "no candidate".
__device__ __forceinline__ unsigned long long double_key(double v) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
  return (b >> 63) ? ~b : (b | (1ull << 63));
}
__device__ __forceinline__ double key_double(unsigned long long k) {
  return __longlong_as_double((long long)((k >> 63) ? (k & ~(1ull << 63)) : ~k));
}
__device__ __forceinline__ unsigned warp_max(unsigned k) { return __reduce_max_sync(0xffffffffu, k); }
__device__ __forceinline__ unsigned long long warp_max(unsigned long long k) {
  const unsigned hi = __reduce_max_sync(0xffffffffu, (unsigned)(k >> 32));
  const unsigned lo = __reduce_max_sync(0xffffffffu, (unsigned)(k >> 32) == hi ? (unsigned)k : 0u);
  return ((unsigned long long)hi << 32) | lo;
}
// the sum of two values as keys; of the first alone where there is no second
__device__ __forceinline__ unsigned key_sum(unsigned a, unsigned b) { return b ? float_key(key_float(a) + key_float(b)) : a; }
__device__ __forceinline__ unsigned long long key_sum(unsigned long long a, unsigned long long b) {
  return b ? double_key(key_double(a) + key_double(b)) : a;
}

// The size of the terms of such a sum, of which each lacks up to 2^-24; 0 where there is no sum.
__device__ __forceinline__ float term_size(unsigned a, unsigned b) { return b ? fabsf(key_float(a)) + fabsf(key_float(b)) : 0.f; }
__device__ __forceinline__ float term_size(unsigned long long, unsigned long long) { return 0.f; }

// Whether two values in 32 bits, the larger first, are sure to be in order: `off` is twice what either may be off by, whatever its size.
__device__ __forceinline__ bool apart(float a, float b, float off) { return a - b > off + 0x1p-20f * (fabsf(a) + fabsf(b)); }
__device__ __forceinline__ bool apart(unsigned a, unsigned b, float off) { return !b || apart(key_float(a), key_float(b), off); }
__device__ __forceinline__ bool apart(unsigned long long, unsigned long long, float) { return true; }
// Whether every group that stays is sure to be worth more than every one that goes.  value, terms: of group `lane` (0: none), its scores good to
// off / 2.  A group has two of them, its sums lack up to 2^-24 of each term and of the value; 2^-20 leaves room for the roundings here.
__device__ __forceinline__ bool groups_apart(unsigned value, float terms, bool kept, float off) {
  const float v = key_float(value), e = off + 0x1p-20f * (fabsf(v) + terms), lo = v - e, hi = v + e;
  const unsigned low = !kept ? 0xffffffffu : lo == lo ? float_key(lo) : 0u, high = kept || !value ? 0u : float_key(hi);
  return __reduce_min_sync(0xffffffffu, low) > warp_max(high);
}
__device__ __forceinline__ bool groups_apart(unsigned long long, float, bool, float) { return true; }

// Takes the best key of the warp: its value (0: none left) and, in *expert, the lowest index that has it; the holder's key is cleared.
template <int PL, typename Key>
__device__ __forceinline__ Key take_best(Key (&key)[PL], int lane, int* expert) {
  Key best = key[0];
  int at = 0;
#pragma unroll
  for (int i = 1; i < PL; ++i)
    if (key[i] > best) {   // ascending i keeps the lower index on ties
      best = key[i];
      at = i;
    }
  const Key top = warp_max(best);
  const int e = (int)__reduce_min_sync(0xffffffffu, best == top ? (unsigned)(lane + 32 * at) : 0xffffffffu);
#pragma unroll
  for (int i = 0; i < PL; ++i)
    if (lane + 32 * i == e) key[i] = 0;
  *expert = top ? e : -1;
  return top;
}

// Clears the keys of the experts whose groups are not kept.  False: keys of 32 bits, good to off / 2, leave that open.
template <int PL, typename Key>
__device__ __forceinline__ bool keep_groups(const RouterParams& rp, int E, int lane, Key (&key)[PL], float off) {
  const int size = E / rp.n_group;
  Key value = 0;       // lane g: of group g
  float terms = 0.f;   // of the sum that it is
  // a, b: the lane's best two of a group
  auto insert = [](Key k, Key& a, Key& b) {
    b = k > a ? a : k > b ? k : b;
    a = k > a ? k : a;
  };
  auto finish = [&](int g, Key a, Key b) {
    Key top = warp_max(a);
    float both = 0.f;
    if (rp.group_top == 2) {
      // the holder (one of them) offers its second best
      const unsigned holders = __ballot_sync(0xffffffffu, a == top);
      const Key second = warp_max(lane == __ffs(holders) - 1 ? b : a);
      both = term_size(top, second);
      top = top ? key_sum(top, second) : 0;
    }
    if (lane == g) {
      value = top;
      terms = both;
    }
  };
  if (size % 32 == 0) {   // whole registers of all lanes: those 65536 tokens took 265 us by the other way when they took 208 by this
    Key a = 0, b = 0;
    int g = 0, left = size;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      insert(key[i], a, b);
      left -= 32;
      if (left == 0) {
        finish(g++, a, b);
        a = b = 0;
        left = size;
      }
    }
  } else {
    for (int g = 0; g < rp.n_group; ++g) {
      Key a = 0, b = 0;
#pragma unroll
      for (int i = 0; i < PL; ++i) {
        const int e = lane + 32 * i;
        insert(e >= g * size && e < (g + 1) * size ? key[i] : 0, a, b);
      }
      finish(g, a, b);
    }
  }
  unsigned kept = 0;
  Key left_over = value;
  for (int n = 0; n < rp.topk_group; ++n) {
    const Key top = warp_max(left_over);
    if (!top) break;
    const int g = __ffs(__ballot_sync(0xffffffffu, left_over == top)) - 1;
    kept |= 1u << g;
    if (lane == g) left_over = 0;
  }
  const bool sure = off <= 0.f || groups_apart(value, terms, (kept >> lane) & 1u, off);
  if (size % 32 == 0) {   // no divisions: a register holds experts of one group
    int left = size;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      if (!(kept & 1u)) key[i] = 0;
      left -= 32;
      if (left == 0) {
        kept >>= 1;
        left = size;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < PL; ++i)
      if (!((kept >> min((lane + 32 * i) / size, 31)) & 1u)) key[i] = 0;
  }
  return sure;
}

// The K best keys: expert number `lane` in lanes below K (-1: none left).  *sure: false if keys of 32 bits leave their order open.
template <int PL, typename Key>
__device__ __forceinline__ int choose(int K, int lane, Key (&key)[PL], float off, bool* sure) {
  int my_e = -1;
  Key last = 0;
  const int rounds = off > 0.f ? K + 1 : K;   // with the first that is not chosen
  for (int k = 0; k < rounds; ++k) {
    int e;
    const Key top = take_best<PL>(key, lane, &e);
    if (off > 0.f && last && !apart(last, top, off)) {
      *sure = false;
      break;
    }
    if (!top || k == K) break;
    last = top;
    if (lane == k) my_e = e;
  }
  return my_e;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_largest(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// The choice with all sums in 64 bits.  Out of line: few tokens need it.
template <int PL>
__device__ __noinline__ int choose_exactly(const ModelParams& mp, const RouterParams& rp, const float* __restrict__ bias, int lane, const float (&z)[PL],
                                           float z_top) {
  double p[PL], sum = 0.0;
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    if (rp.sigmoid) p[i] = 1.0 / (1.0 + exp(-(double)z[i]));
    else p[i] = z[i] > -INFINITY ? exp((double)z[i] - (double)z_top) : 0.0;
    sum += p[i];
  }
  if (!rp.sigmoid) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  }
  unsigned long long key[PL];
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    const int e = lane + 32 * i;
    const double s = rp.sigmoid ? p[i] : p[i] / sum;
    const double c = s + (bias && e < mp.E ? (double)__ldg(bias + e) : 0.0);
    key[i] = z[i] > -INFINITY && c > -INFINITY ? double_key(c) : 0ull;
  }
  bool sure = true;
  if (rp.n_group > 1) keep_groups<PL>(rp, mp.E, lane, key, -1.f);
  return choose<PL>(mp.K, lane, key, 0.f, &sure);
}

// Routes token t (E <= 32 PL), whose logits are zs[0 .. E): writes its row of topk_idx and topk_w.  Returns expert number `lane` in lanes
// below K.  A logit of -inf or NaN is an expert that cannot be chosen, one above the largest float counts as that.
template <int PL, typename Z>
__device__ __forceinline__ int route_scored(const ModelParams& mp, const RouterParams& rp, int t, int layer, int lane, const Z* __restrict__ zs,
                                            int32_t* __restrict__ topk_idx, float* __restrict__ topk_w) {
  const int E = mp.E, K = mp.K;
  float z[PL];
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    const float v = lane + 32 * i < E ? logit_value(zs[lane + 32 * i]) : -INFINITY;
    z[i] = v == v ? fminf(v, FLT_MAX) : -INFINITY;
  }
  float z_top = -INFINITY;
  if (!rp.sigmoid) {
#pragma unroll
    for (int i = 0; i < PL; ++i) z_top = fmaxf(z_top, z[i]);
    z_top = warp_largest(z_top);
  }
  int my_e = -1;
  bool sure = true;
  if (!rp.bias && (rp.n_group == 1 || rp.group_top == 1)) {
    unsigned key[PL];
#pragma unroll
    for (int i = 0; i < PL; ++i) key[i] = z[i] > -INFINITY ? float_key(z[i]) : 0u;
    if (rp.n_group > 1) keep_groups<PL>(rp, E, lane, key, -1.f);
    my_e = choose<PL>(K, lane, key, 0.f, &sure);
  } else {
    const float* const bias = rp.bias ? rp.bias + (size_t)layer * E : nullptr;
    float b[PL], p[PL], sum = 0.f;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      b[i] = bias && lane + 32 * i < E ? __ldg(bias + lane + 32 * i) : 0.f;
      if (rp.sigmoid) p[i] = __fdividef(1.f, 1.f + expf(-z[i]));
      else sum += p[i] = z[i] > -INFINITY ? expf(z[i] - z_top) : 0.f;
    }
    if (!rp.sigmoid) {
      sum = warp_sum(sum);
#pragma unroll
      for (int i = 0; i < PL; ++i) p[i] = __fdividef(p[i], sum);
    }
    unsigned key[PL];
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      const float c = p[i] + b[i];
      key[i] = z[i] > -INFINITY && c > -INFINITY ? float_key(c) : 0u;
    }
    constexpr float kOff = 0x1p-18f;
    if (rp.n_group > 1) sure = keep_groups<PL>(rp, E, lane, key, kOff);
    if (sure) my_e = choose<PL>(K, lane, key, kOff, &sure);
    if (!sure) my_e = choose_exactly<PL>(mp, rp, bias, lane, z, z_top);
  }
  // weights: the scores, over their sum with the power of e that the largest chosen one holds taken out, so that no sum vanishes
  const bool there = lane < K && my_e >= 0;
  const float my_z = there ? fminf(logit_value(zs[my_e]), FLT_MAX) : 0.f;   // a line at hand; carrying it along costs more
  float w;
  if (rp.sigmoid) {
    const float shift = mp.renorm ? fminf(warp_largest(there ? my_z : -INFINITY), 0.f) : 0.f;
    w = my_z > 0.f ? 1.f / (1.f + expf(-my_z)) : expf(my_z - shift) / (1.f + expf(my_z));
  } else {
    const float shift = mp.renorm ? warp_largest(there ? my_z : -INFINITY) : z_top;
    w = expf(my_z - shift);
  }
  if (!there) w = 0.f;
  float total = 1.f;
  if (mp.renorm) {
    total = warp_sum(w);
  } else if (!rp.sigmoid) {
    total = 0.f;
#pragma unroll
    for (int i = 0; i < PL; ++i) total += z[i] > -INFINITY ? expf(z[i] - z_top) : 0.f;
    total = warp_sum(total);
  }
  if (lane < K) {
    topk_idx[(size_t)t * K + lane] = my_e;
    topk_w[(size_t)t * K + lane] = there ? rp.scale * (w / total) : 0.f;
  }
  return my_e;
}

}  // namespace
