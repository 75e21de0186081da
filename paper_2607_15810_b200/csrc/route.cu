// The router of an expert layer: scores from logits, choice of the experts, weights -- and their gradient.
//   s = softmax(l) over the experts or sigmoid(l);  choice c = s + bias;  with groups: the topk_group groups with the largest sums of their
//   group_top best c stay;  the topk largest c, ties to the lower id;  w = scale * s_j, renormalised: scale * s_j / sum of the chosen.
// An expert with a logit of -inf (or NaN), or a bias of -inf, is not there.  Without a bias the experts of the groups that stay are in the order
// of their logits, which is that of the scores and also tells those apart that round to the same.
#include "kernels.cuh"

namespace quads {
namespace {

constexpr int kRouterWarps = 8;

template <bool kBf16>
__device__ __forceinline__ float router_logit(const void* p, int64_t at) {
  const float v = kBf16 ? __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t*>(p) + at) << 16) : __ldg(static_cast<const float*>(p) + at);
  return fmaxf(v + 0.f, -INFINITY);                               // -0 counts as +0, NaN as -inf
}

// Order-preserving map to unsigned integers, which is 0x007FFFFF for -inf and more for everything above.
constexpr uint32_t kKeyNone = 0x007FFFFFu;
__device__ __forceinline__ uint32_t logit_key(float v) {
  const uint32_t b = __float_as_uint(v);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_float(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k); }
__device__ __forceinline__ float warp_max_f32(float v) { return key_float(__reduce_max_sync(0xFFFFFFFFu, logit_key(v))); }

__device__ __forceinline__ uint64_t double_key(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  return (b >> 63) ? ~b : (b | 0x8000000000000000ull);
}
// Largest of the lanes' 64-bit keys.
__device__ __forceinline__ uint64_t warp_max_key(uint64_t k) {
  const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(k >> 32));
  const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
  return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

__device__ __forceinline__ float rcp_approx(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
// a / b for a normal b: the product with the approximate reciprocal and one Newton step on what it leaves over, which takes the error from two units
// in the last place to half of one but for rare cases.  As exact as rounded division (weights of 16384 tokens, relative 2-norm error 6.2e-8; 7.2e-8 without
// the step), which would take the softmax router from 10.1 to 10.9 us; the step takes no time that can be measured.
__device__ __forceinline__ float quotient(float a, float b) {
  const float r = rcp_approx(b), q = a * r;
  return fmaf(fmaf(-q, b, a), r, q);
}
__device__ __forceinline__ float sigmoid_f32(float l) {
  const float e = expf(-fabsf(l));
  return quotient(l > 0.f ? 1.f : e, 1.f + e);
}
// Weights of the chosen experts relative to one another, from their logits (a lane each, -inf: none): s_j / sum s.  Both
// scores are scaled so that the largest is of the order of one: a sum of underflown sigmoids would be zero.
__device__ __forceinline__ float renormalised(float l, bool sigmoid) {
  const float m = warp_max_f32(l);
  if (m == -INFINITY) return 0.f;
  float s;
  if (sigmoid) {
    const float m0 = fminf(m, 0.f), e = expf(-fabsf(l));
    s = quotient(l > 0.f ? expf(-m0) : expf(l - m0), 1.f + e);
  } else {
    s = expf(l - m);
  }
  const float sum = warp_sum(s);
  return s == sum ? 1.f : quotient(s, sum);                // (one alone is exactly 1, and its gradient 0)
}

// How the lanes hold a token's experts: lane g * lanes_per_group + i the `chunk` consecutive ones from i * chunk on of group g, so that a
// group is a power of two of neighbouring lanes and the order of (lane, position) is that of the ids.
struct LaneExperts { int first, count; };
__device__ __forceinline__ LaneExperts lane_experts(const RouterParams& p, int lane) {
  const int g = lane >> p.lanes_log2, i = lane & ((1 << p.lanes_log2) - 1), per = p.per_group;
  const int at = i * p.chunk;
  return {g * per + at, g < p.n_group ? max(0, min(p.chunk, per - at)) : 0};
}

// A token's logits; kVec: NJ of them in every lane, aligned to their size or 16 bytes.
template <int NJ, bool kBf16>
__device__ __forceinline__ void load_logits(const RouterParams& p, int64_t t, const LaneExperts& x, float* l) {
  constexpr int kBytes = NJ * (kBf16 ? 2 : 4);
  const int64_t at = t * p.ld + x.first;
  if (kBytes >= 8 && p.vec) {
    uint32_t w[kBytes / 4 > 0 ? kBytes / 4 : 1];
#pragma unroll
    for (int i = 0; i < kBytes / 4; ++i) w[i] = kBf16 ? 0xFF80FF80u : 0xFF800000u;      // -inf
    if (x.count > 0) {
      const uint8_t* src = static_cast<const uint8_t*>(p.logits) + at * (kBf16 ? 2 : 4);
      if constexpr (kBytes == 8) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(src));
        w[0] = v.x; w[1] = v.y;
      } else if constexpr (kBytes >= 16) {
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) {
          const uint4 v = __ldg(reinterpret_cast<const uint4*>(src) + i);
          w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const float v = kBf16 ? __uint_as_float((j & 1) ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16) : __uint_as_float(w[j]);
      l[j] = fmaxf(v + 0.f, -INFINITY);
    }
  } else {
#pragma unroll
    for (int j = 0; j < NJ; ++j) l[j] = j < x.count ? router_logit<kBf16>(p.logits, at + j) : -INFINITY;
  }
}

__device__ __forceinline__ double key_double(uint64_t k) {
  return __longlong_as_double((long long)((k >> 63) ? (k & 0x7FFFFFFFFFFFFFFFull) : ~k));
}
__device__ __forceinline__ uint32_t warp_max_any(uint32_t k) { return __reduce_max_sync(0xFFFFFFFFu, k); }
__device__ __forceinline__ uint64_t warp_max_any(uint64_t k) { return warp_max_key(k); }

// The two largest keys of a lane's group, over its lanes.
template <typename Key>
__device__ __forceinline__ void group_best(int lanes_log2, Key& a, Key& b) {
  for (int o = 1; o < 1 << lanes_log2; o <<= 1) {
    const Key oa = __shfl_xor_sync(0xFFFFFFFFu, a, o), ob = __shfl_xor_sync(0xFFFFFFFFu, b, o);
    b = max(min(a, oa), max(b, ob));
    a = max(a, oa);
  }
}

// Bit g: group g is among the topk_group best by the keys `gk` (the same in all lanes of a group, 0: nothing in it).  `last` and `next`: the
// keys of the last one kept and of the best one left out (0: none).
template <typename Key>
__device__ __forceinline__ uint32_t best_groups(const RouterParams& p, Key gk, int lane, Key& last, Key& next) {
  const int mine = lane >> p.lanes_log2;
  uint32_t kept = 0;
  last = 0;
  for (int g = 0; g < p.topk_group; ++g) {
    const Key m = warp_max_any(gk);
    if (m == 0) break;
    last = m;
    const int w = (__ffs(__ballot_sync(0xFFFFFFFFu, gk == m)) - 1) >> p.lanes_log2;
    kept |= 1u << w;
    if (mine == w) gk = 0;
  }
  next = warp_max_any(gk);
  return kept;
}

// Below it the sigmoid is e^l to float64's last bit; e^-l is infinite from -709.8 on, where the sigmoid is not yet 0.  (By e^-|l| throughout, with no
// such border, the float64 parts make the kernel slower where they are not run: 16384 tokens, softmax, 10.15 -> 10.40 us.)
constexpr float kSmallSigmoid = -700.f;

// The choice in float64, for the tokens whose float32 scores lie too near to one another: slow and exact.  Lane s < topk gets slot s.
// keys [NJ][32], a column per lane: in shared memory and loops, because in registers, or in a function that is called, they give the
// kernel a stack, and the launch of one that has any takes 0.4 us longer.  (Unrolled so far as that leaves none: 16384 tokens, all of them near, 68 us,
// 76 with no unrolling.)
template <int NJ, bool kBf16>
__device__ __forceinline__ int choose_exact(const RouterParams& p, int64_t t, uint64_t* keys) {
  const int lane = threadIdx.x & 31;
  const LaneExperts x = lane_experts(p, lane);
  const bool sigmoid = p.score == QUADS_SCORE_SIGMOID;
  const int64_t at = t * p.ld + x.first;
  auto logit = [&](int j) { return j < x.count ? router_logit<kBf16>(p.logits, at + j) : -INFINITY; };
  keys += lane;
  float mx = 0.f;
  if (!sigmoid) {
    mx = -INFINITY;
#pragma unroll 8
    for (int j = 0; j < NJ; ++j) mx = fmaxf(mx, logit(j));
    mx = warp_max_f32(mx);
  }
  double sum = 0.0;
#pragma unroll 2
  for (int j = 0; j < NJ; ++j) {
    const float l = logit(j);
    const double e = l > -INFINITY ? exp(sigmoid ? -(double)l : (double)l - (double)mx) : 0.0;
    sum += e;
    keys[32 * j] = (uint64_t)__double_as_longlong(e);
  }
  sum = warp_sum(sum);
  uint64_t a = 0, b = 0;
#pragma unroll 1
  for (int j = 0; j < NJ; ++j) {
    const double e = __longlong_as_double((long long)keys[32 * j]);
    const float l = logit(j);
    double c = (sigmoid ? 1.0 : e) / (sigmoid ? 1.0 + e : sum);
    if (sigmoid && l < kSmallSigmoid) c = exp((double)l);
    if (p.bias && j < x.count) c += (double)__ldg(p.bias + x.first + j);
    const uint64_t k = l > -INFINITY && c > -INFINITY ? double_key(c + 0.0) : 0;
    keys[32 * j] = k;
    b = max(b, min(a, k));
    a = max(a, k);
  }
  bool in = true;
  if (p.n_group > 1) {
    group_best(p.lanes_log2, a, b);
    uint64_t last, next;
    const uint32_t kept = best_groups(p, p.group_top == 2 && b ? double_key(key_double(a) + key_double(b) + 0.0) : a, lane, last, next);
    in = (kept >> (lane >> p.lanes_log2)) & 1u;
  }
  if (!in || !p.bias) {
#pragma unroll 2
    for (int j = 0; j < NJ; ++j) keys[32 * j] = in && keys[32 * j] ? (uint64_t)logit_key(logit(j)) : 0;
  }
  int my_id = -1;
  for (int s = 0; s < p.topk; ++s) {
    uint64_t best = 0;
    int at_j = 0;                                            // the first of a lane's largest ones
#pragma unroll 8
    for (int j = 0; j < NJ; ++j) {
      const uint64_t k = keys[32 * j];
      if (k > best) { best = k; at_j = j; }
    }
    const uint64_t m = warp_max_key(best);
    if (m == 0) break;
    const int w = __ffs(__ballot_sync(0xFFFFFFFFu, best == m)) - 1;
    const int id = __shfl_sync(0xFFFFFFFFu, x.first + at_j, w);
    if (lane == w) keys[32 * at_j] = 0;
    if (lane == s) my_id = id;
  }
  return my_id;
}

// The ranks of the `total` gathered experts (lane i: the i-th, in the order of the ids) by their choice in float64.
template <int NJ, bool kBf16>
__device__ __forceinline__ int rank_exact(const RouterParams& p, int64_t t, int id, int total, uint2* scratch) {
  const int lane = threadIdx.x & 31;
  const bool sigmoid = p.score == QUADS_SCORE_SIGMOID;
  const float l = lane < total ? router_logit<kBf16>(p.logits, t * p.ld + id) : -INFINITY;
  float mx = 0.f;
  double sum = 0.0;
  if (!sigmoid) {
    const LaneExperts x = lane_experts(p, lane);
    const int64_t at = t * p.ld + x.first;
    mx = -INFINITY;
#pragma unroll 1
    for (int j = 0; j < x.count; ++j) mx = fmaxf(mx, router_logit<kBf16>(p.logits, at + j));
    mx = warp_max_f32(mx);
#pragma unroll 1
    for (int j = 0; j < x.count; ++j) sum += exp((double)router_logit<kBf16>(p.logits, at + j) - (double)mx);
    sum = warp_sum(sum);
  }
  const double e = l > -INFINITY ? exp(sigmoid ? -(double)l : (double)l - (double)mx) : 0.0;
  double c = (sigmoid ? 1.0 : e) / (sigmoid ? 1.0 + e : sum);
  if (sigmoid && l < kSmallSigmoid) c = exp((double)l);
  if (p.bias && lane < total) c += (double)__ldg(p.bias + id);
  const uint64_t mine = double_key(c + 0.0);
  uint64_t* keys = reinterpret_cast<uint64_t*>(scratch);
  keys[lane] = mine;
  __syncwarp();
  int rank = 0;
  for (int i = 0; i < total; ++i) rank += keys[i] > mine || (keys[i] == mine && i < lane) ? 1 : 0;
  __syncwarp();
  return lane < total ? rank : 32;
}

// The `slots` largest of the warp's keys (those above kKeyNone), one to a lane: its key, id and rank -- descending, equal ones in the order of the
// ids --, or rank 32.  The slots-th largest of the lanes' maxima bounds the answer from below; what is not below it (slots or a few
// more) is gathered one to a lane, in the order of the ids, and ranked by counting; what is `margin` less is gathered, too.  total:
// how many those are; more than 32 (few lanes with many keys each) are not gathered: the maximum of all keys, slot by slot.
template <int NJ>
__device__ __forceinline__ void select_largest_keys(uint32_t* key, const LaneExperts& x, int slots, int lane, float margin, uint2* gathered, uint32_t& my_key, int& my_id,
                                                    int& my_rank, int& total) {
  gathered[lane] = make_uint2(0u, 0u);
  uint32_t head = key[0];
#pragma unroll
  for (int j = 1; j < NJ; ++j) head = max(head, key[j]);
  uint32_t bound = 0;
#pragma unroll 4
  for (int s = 0; s < slots; ++s) {
    bound = __reduce_max_sync(0xFFFFFFFFu, head);
    if (head == bound) head = 0;
  }
  if (margin > 0.f && bound > kKeyNone) bound = logit_key(key_float(bound) - margin);
  bound = max(bound, kKeyNone + 1u);
  int mine = 0;
#pragma unroll
  for (int j = 0; j < NJ; ++j) mine += key[j] >= bound ? 1 : 0;
  const uint32_t below = (1u << lane) - 1u;
  int at = 0;
  total = 0;
  for (int n = 1; n <= NJ; ++n) {
    const uint32_t b = __ballot_sync(0xFFFFFFFFu, mine >= n);
    if (b == 0) break;
    at += __popc(b & below);
    total += __popc(b);
  }
  __syncwarp();
  my_rank = 32;
  if (total <= 32) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (key[j] >= bound) gathered[at++] = make_uint2(key[j], (uint32_t)(x.first + j));
    __syncwarp();
    my_key = gathered[lane].x;
    my_id = (int)gathered[lane].y;
    int rank = 0;
#pragma unroll 2
    for (int i = 0; i < total; i += 2) {
      const uint4 two = *reinterpret_cast<const uint4*>(gathered + i);           // {key, id} of i and i + 1 (0 behind the last)
      rank += two.x > my_key || (two.x == my_key && i < lane) ? 1 : 0;            // (an equal key of a lower id comes first)
      rank += two.z > my_key || (two.z == my_key && i + 1 < lane) ? 1 : 0;
    }
    if (lane < total && rank < slots) my_rank = rank;
    __syncwarp();                                            // (before the next token's are written)
  } else {
    my_key = 0;
    my_id = -1;
    for (int s = 0; s < slots; ++s) {
      uint32_t best = key[0];
#pragma unroll
      for (int j = 1; j < NJ; ++j) best = max(best, key[j]);
      const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, best);
      if (m <= kKeyNone) break;
      const int w = __ffs(__ballot_sync(0xFFFFFFFFu, best == m)) - 1;
      int id = -1;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const bool it = id < 0 && key[j] == m;
        id = it ? x.first + j : id;
        key[j] = it && lane == w ? 0 : key[j];
      }
      id = __shfl_sync(0xFFFFFFFFu, id, w);
      if (lane == s) { my_key = m; my_id = id; my_rank = s; }
    }
  }
}

__device__ __forceinline__ float ex2_approx(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

// One warp per token.  Keys are order-preserving 32-bit integers of what the experts are chosen by.  By logits they are exact.  By
// scores they are float32, off by at most d and 2^-24 of themselves (the bias' addition).  Sigmoid: the exponential is good to 2^-22
// and to 2^-23 |l| (its argument), 1 + e to 2^-24, the reciprocal to 2^-23 of themselves; s (1 - s) <= 1/4 and |l| s (1 - s) < 0.23 of the first
// two reach s: at most smax 2^-22 (2 + |l|/2) with l <= 0 the largest score's logit, i.e. d = smax 2^-20 from smax = 1/4 on and
// smax 2^-19 down to smax = 2^-9 (|l| < 6.3).  Softmax: the same for the terms, 2^-20 for the sum of 256: d = smax 2^-19.  Where two
// neighbours in rank lie nearer than twice that, those gathered are ranked in float64; where two groups do, or smax is less, the
// token is chosen in float64 from the start.
// Bound by the latency of the chain of a warp's reductions and votes, one token at a time in a warp: at many tokens 52 to 54 % of the issue slots are taken
// (some 900 instructions a token with sigmoid, bias and groups, 480 by logits), and of 16384 tokens a warp takes three or four.  Replayed from a graph: 16384
// tokens of 256 experts, sigmoid, bias and groups 19.2 to 23.7 us (more where one of the tokens that the warps take last is chosen in float64; all tokens
// in float64 75), softmax 10.1 (keys of 64 bits, a maximum of all of them per slot: 30.5); one token 3.0 and
// 2.0.  Measured on the form with calls: five CTAs on an SM 22.9 against 20.7, six 23.6; two tokens to a warp, 16 lanes each, shuffles in place of the
// warp's reduction, 256 experts 28.4 and 14.9, 128 experts 10.2 and 6.5 against 11.0 and 6.9 (not taken for few experts alone: not measured on the present form).
template <int NJ, bool kBf16>
__global__ void __launch_bounds__(kRouterWarps * 32, NJ <= 8 ? 4 : 2)
route_experts_kernel(const RouterParams p) {
  __shared__ __align__(16) uint2 s_gathered[kRouterWarps][32];
  __shared__ uint64_t s_keys[kRouterWarps][32 * NJ];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint2* gathered = s_gathered[warp];
  const LaneExperts x = lane_experts(p, lane);
  const bool sigmoid = p.score == QUADS_SCORE_SIGMOID;
  pdl_sync();
  float bias[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) bias[j] = p.bias && j < x.count ? __ldg(p.bias + x.first + j) : 0.f;
  for (int64_t t = (int64_t)blockIdx.x * kRouterWarps + warp; t < p.T; t += (int64_t)gridDim.x * kRouterWarps) {
    float l[NJ];
    load_logits<NJ, kBf16>(p, t, x, l);
    // the softmax's largest logit and sum, where they are needed; keys; d: what a score may be off by
    float mx = 0.f, inv = 0.f, d = 0.f;
    if (!sigmoid && (p.by_score || !p.renormalize)) {
      mx = l[0];
#pragma unroll
      for (int j = 1; j < NJ; ++j) mx = fmaxf(mx, l[j]);
      mx = warp_max_f32(mx);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) sum += l[j] > -INFINITY ? expf(l[j] - mx) : 0.f;
      sum = warp_sum(sum);
      inv = sum > 0.f ? quotient(1.f, sum) : 0.f;
    }
    uint32_t key[NJ];
    bool near = false;
    if (p.by_score) {
      constexpr float kLog2e = 1.4426950408889634f;
      float smax = 0.f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const float e = ex2_approx((sigmoid ? -l[j] : l[j] - mx) * kLog2e);
        const float s = sigmoid ? rcp_approx(1.f + e) : e * inv;
        smax = fmaxf(smax, s);
        key[j] = l[j] > -INFINITY ? logit_key(s + bias[j]) : 0;
      }
      smax = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(smax)));
      near = smax < 0x1p-9f;
      d = smax * (sigmoid && smax > 0.25f ? 0x1p-20f : 0x1p-19f);
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j) key[j] = logit_key(l[j]);
    }
    if (p.n_group > 1) {
      uint32_t a = 0, b = 0, last, next;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        b = max(b, min(a, key[j]));
        a = max(a, key[j]);
      }
      group_best(p.lanes_log2, a, b);
      a = a > kKeyNone ? a : 0;                              // 0: nothing in the group
      b = b > kKeyNone ? b : 0;
      const uint32_t gk = p.group_top == 2 && b ? logit_key(key_float(a) + key_float(b) + 0.f) : a;
      const uint32_t kept = best_groups(p, gk, lane, last, next);
      if (p.by_score && next) {
        // the terms are off by d and 2^-24 |c| each, their sum is rounded, 2^-24 |sum|: together by 2 d + 2^-22 max |c| at most
        const float m = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(fmaxf(a ? fabsf(key_float(a)) : 0.f, b ? fabsf(key_float(b)) : 0.f))));
        near |= !(key_float(last) - key_float(next) > 4.f * d + m * 0x1p-21f);
      }
      const bool in = (kept >> (lane >> p.lanes_log2)) & 1u;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (p.by_score && !p.bias) key[j] = logit_key(l[j]);        // within the groups kept the logits are in the scores' order
        key[j] = in ? key[j] : 0;
      }
    }
    // ---- the topk largest; with a bias one more, which the last one has to be told apart from, and what might be it
    uint32_t my_key;
    int my_id, my_rank, total;
    const float most = p.bias ? 4.f * d : 0.f;
    select_largest_keys<NJ>(key, x, p.topk + (p.bias ? 1 : 0), lane, most, gathered, my_key, my_id, my_rank, total);
    if (p.bias && !near) {
      gathered[lane] = make_uint2(0u, 0u);
      __syncwarp();
      if (my_rank < 32) gathered[my_rank].x = my_key;
      __syncwarp();
      const uint32_t next = my_rank < 31 ? gathered[my_rank + 1].x : 0u;       // the one behind
      __syncwarp();
      const float c = key_float(my_key), u = key_float(next), m = fmaxf(fabsf(u), fabsf(c)) * 0x1p-23f;
      if (__any_sync(0xFFFFFFFFu, next != 0 && !(c - u > 2.f * (d + m)))) {
        // (the gathered ones are the answer's superset while the biases' roundings are small beside d)
        if (total <= 32 && !__any_sync(0xFFFFFFFFu, next != 0 && m > d)) my_rank = rank_exact<NJ, kBf16>(p, t, my_id, total, gathered);
        else near = true;
      }
    }
    if (near) {
      my_id = choose_exact<NJ, kBf16>(p, t, s_keys[warp]);
      my_rank = my_id >= 0 ? lane : 32;
    }
    // ---- their weights, by the lane that holds them
    const bool chosen = my_rank < p.topk;
    const float my_l = chosen ? router_logit<kBf16>(p.logits, t * p.ld + my_id) : -INFINITY;
    float wgt;
    if (p.renormalize) wgt = renormalised(my_l, sigmoid);
    else if (sigmoid) wgt = sigmoid_f32(my_l);
    else wgt = expf(my_l - mx) * inv;
    const int64_t out = t * p.topk;
    if (chosen) {
      p.ids[out + my_rank] = my_id;
      p.weights[out + my_rank] = wgt * p.scale;
    }
    // (slots that stay empty)
    const int n = __popc(__ballot_sync(0xFFFFFFFFu, chosen));
    if (lane >= n && lane < p.topk) {
      p.ids[out + lane] = -1;
      p.weights[out + lane] = 0.f;
    }
  }
}

// Gradient of the weights with respect to the logits, the choice held.  One warp per token, lane s with slot s: the row is written as a whole
// (zeros, or what every logit gets from the softmax's sum), then the slots' entries over it.  Bound by the stream of the rows: 16384 x 256
// 7.2 us, 34.6 MB or 4.8 TB/s; renormalised 6.1 (the slots' entries added in registers, 16 shuffles and comparisons a slot: 14.2).
template <int NJ, bool kBf16>
__global__ void __launch_bounds__(kRouterWarps * 32)
route_experts_backward_kernel(const RouterParams p) {
  pdl_sync();
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * kRouterWarps + (threadIdx.x >> 5);
  if (t >= p.T) return;
  const bool sigmoid = p.score == QUADS_SCORE_SIGMOID;
  const bool dense = !p.renormalize && !sigmoid;
  int id = -1;
  float dw = 0.f;
  if (lane < p.topk) {
    id = __ldg(p.ids_in + t * p.topk + lane);
    if ((unsigned)id >= (unsigned)p.E) id = -1;
    dw = __ldg(p.dweights + t * p.topk + lane) * p.scale;
    if (id < 0) dw = 0.f;
  }
  // (lane i: the NJ experts from i * NJ on)
  const LaneExperts x{lane * NJ, max(0, min(NJ, p.E - lane * NJ))};
  float v[NJ];
  if (dense) {
    load_logits<NJ, kBf16>(p, t, x, v);
  } else {
#pragma unroll
    for (int j = 0; j < NJ; ++j) v[j] = 0.f;
  }
  const float l = id >= 0 ? router_logit<kBf16>(p.logits, t * p.ld + id) : -INFINITY;
  float g, base = 0.f;                                       // a slot's entry, and what stands there without it
  if (p.renormalize) {
    const float r = renormalised(l, sigmoid);
    g = r * (dw - warp_sum(r * dw));
    if (sigmoid) g *= 1.f / (1.f + expf(l));
  } else if (sigmoid) {
    g = dw * sigmoid_f32(l) * (1.f / (1.f + expf(l)));
  } else {
    float mx = v[0];
#pragma unroll
    for (int j = 1; j < NJ; ++j) mx = fmaxf(mx, v[j]);
    mx = warp_max(mx);
    if (mx == -INFINITY) mx = 0.f;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) { v[j] = expf(v[j] - mx); sum += v[j]; }
    sum = warp_sum(sum);
    const float inv = sum > 0.f ? 1.f / sum : 0.f, pl = expf(l - mx) * inv;
    g = pl * dw;
    const float all = -inv * warp_sum(g);
#pragma unroll
    for (int j = 0; j < NJ; ++j) v[j] *= all;
    base = expf(l - mx) * all;
  }
  if (id < 0) g = 0.f;
  const int64_t at = t * p.ld_d + x.first;
  constexpr int kBytes = NJ * (kBf16 ? 2 : 4);
  if (kBytes >= 8 && p.vec_d) {
    if (x.count > 0) {
      uint32_t w[kBytes / 4 > 0 ? kBytes / 4 : 1];
#pragma unroll
      for (int i = 0; i < kBytes / 4; ++i) w[i] = kBf16 ? f32x2_to_bf16x2(v[(2 * i) % NJ], v[(2 * i + 1) % NJ]) : __float_as_uint(v[i % NJ]);
      uint8_t* dst = static_cast<uint8_t*>(p.dlogits) + at * (kBf16 ? 2 : 4);
      if constexpr (kBytes == 8) {
        *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
      } else if constexpr (kBytes >= 16) {
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) reinterpret_cast<uint4*>(dst)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      if (j >= x.count) continue;
      if (kBf16) static_cast<__nv_bfloat16*>(p.dlogits)[at + j] = __float2bfloat16_rn(v[j]);
      else static_cast<float*>(p.dlogits)[at + j] = v[j];
    }
  }
  // an id that stands more than once (a lane finds another one's number in its place): its first slot takes the sum, in the order of
  // the slots
  __shared__ uint8_t s_slot[kRouterWarps][kMaxExperts];
  if (id >= 0) s_slot[threadIdx.x >> 5][id] = (uint8_t)lane;
  __syncwarp();                                              // (the row's own stores, too, come before the slots')
  if (__any_sync(0xFFFFFFFFu, id >= 0 && s_slot[threadIdx.x >> 5][id] != lane)) {
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, id < 0 ? -1 - lane : id);
    float sum = 0.f;
    for (int s = 0; s < p.topk; ++s) {
      const float a = __shfl_sync(0xFFFFFFFFu, g, s);
      if ((same >> s) & 1u) sum += a;
    }
    g = sum;
    if ((same & ((1u << lane) - 1u)) != 0) id = -1;
  }
  if (id >= 0) {
    const float r = base + g;
    if (kBf16) static_cast<__nv_bfloat16*>(p.dlogits)[t * p.ld_d + id] = __float2bfloat16_rn(r);
    else static_cast<float*>(p.dlogits)[t * p.ld_d + id] = r;
  }
}

template <int NJ>
quads_status launch_router_nj(RouterParams& p, int n_sms, cudaStream_t st) {
  const dim3 block(kRouterWarps * 32);
  dim3 grid((unsigned)((p.T + kRouterWarps - 1) / kRouterWarps));
  if (!p.dlogits) grid.x = std::min(grid.x, (unsigned)(n_sms * 4));
  // whole lanes in pieces of 8 or 16 bytes
  const int size = p.bf16 ? 2 : 4, piece = std::min(16, NJ * size);
  auto whole = [&](const void* base, int64_t ld) {
    return piece >= 8 && reinterpret_cast<uintptr_t>(base) % piece == 0 && ld * size % piece == 0;
  };
  p.vec = (p.dlogits ? p.E % NJ == 0 : p.per_group % NJ == 0 && p.chunk == NJ) && whole(p.logits, p.ld);
  p.vec_d = p.dlogits && p.E % NJ == 0 && whole(p.dlogits, p.ld_d);
  if (p.dlogits) {
    if (p.bf16) QUADS_CUDA_OK(launch_kernel(route_experts_backward_kernel<NJ, true>, grid, block, (size_t)0, st, p));
    else QUADS_CUDA_OK(launch_kernel(route_experts_backward_kernel<NJ, false>, grid, block, (size_t)0, st, p));
  } else {
    if (p.bf16) QUADS_CUDA_OK(launch_kernel(route_experts_kernel<NJ, true>, grid, block, (size_t)0, st, p));
    else QUADS_CUDA_OK(launch_kernel(route_experts_kernel<NJ, false>, grid, block, (size_t)0, st, p));
  }
  return QUADS_OK;
}

}  // namespace

quads_status launch_router(const RouterParams& args, int n_sms, cudaStream_t st) {
  RouterParams p = args;
  int n = (p.E + 31) / 32;                                    // experts in a lane
  if (!p.dlogits) {
    p.per_group = p.E / p.n_group;
    p.lanes_log2 = 0;
    while (p.n_group << (p.lanes_log2 + 1) <= 32) ++p.lanes_log2;
    n = p.chunk = (p.per_group + (1 << p.lanes_log2) - 1) >> p.lanes_log2;
  }
  if (n <= 1) return launch_router_nj<1>(p, n_sms, st);
  if (n <= 2) return launch_router_nj<2>(p, n_sms, st);
  if (n <= 4) return launch_router_nj<4>(p, n_sms, st);
  if (n <= 8) return launch_router_nj<8>(p, n_sms, st);
  return launch_router_nj<16>(p, n_sms, st);
}

}  // namespace quads
