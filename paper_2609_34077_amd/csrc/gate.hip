// Routing by scores, balance bias and expert groups (include/maskmoe.h, maskmoe_gate_forward), and
// the gradient of its gates.
//
// A token takes a segment of W lanes (16; above 64 experts 64), each of which holds V consecutive experts in
// registers, so that a row of logits is read once, in order, and lower lanes hold lower experts:
//   scores    softmax or sigmoid of the registers, row maximum and sum by lane exchanges;
//   groups    the two largest keys of a group by lane exchanges, its rank by comparing it with every other; a
//             group stays if fewer than topk_group groups beat it;
//   top-K     up to 64 experts: every lane sorts its V keys; each round takes the largest first key of the segment
//             and the lowest lane that holds it, which drops it, four tokens at once. Above: the K-th largest of
//             the lanes' largest keys is a bound that the K best keys reach; the few that do go to LDS, and
//             four tokens' candidates are ranked at once, a lane each (rounds over 64 lanes took 45 instructions each for
//             one token: 131072 tokens x 256 experts 157 us instead of 120).
// Keys travel as integers that order as the numbers do (0: no eligible expert), so that a step of an
// exchange is one instruction.
// Selection goes by real numbers: keys are compared in fp32, and where two keys (groups) that the result
// depends on come closer than fp32 can tell apart (a bound on its errors, below), the wavefront
// selects again with keys in fp64 (select_exact).
// Without bias, prior and group sums the keys are the logits, which order as their scores do and need neither.

#include <float.h>

#include <algorithm>

#include "common.hpp"
#include "gate.hpp"

namespace maskmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

// v of the lane that DPP control CTRL names: 0xB1 / 0x4E exchange lanes 1 / 2 apart, 0x141 / 0x140
// mirror 8 / 16 lanes, which exchanges their halves where the lanes of each half agree.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, true));
}
// The value of the other half of 2 S lanes, where the lanes of each half agree.
template <int S>
__device__ __forceinline__ uint32_t other(uint32_t v) {
  if constexpr (S == 1) return dpp<0xB1>(v);
  else if constexpr (S == 2) return dpp<0x4E>(v);
  else if constexpr (S == 4) return dpp<0x141>(v);
  else if constexpr (S == 8) return dpp<0x140>(v);
  else {
    // swap rows 1 and 0, 3 and 2 (or halves) of two copies: one holds the even, the other the odd rows' values
    const bool low = (threadIdx.x & S) == 0;
    if constexpr (S == 16) {
      const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
      return low ? r[1] : r[0];
    } else {
      const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
      return low ? r[1] : r[0];
    }
  }
}
template <int S>
__device__ __forceinline__ float other(float v) { return __uint_as_float(other<S>(__float_as_uint(v))); }

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t umin(uint32_t a, uint32_t b) { return a < b ? a : b; }

// Largest value and sum over the W lanes of a segment, in every lane.
template <int W, int S = 1>
__device__ __forceinline__ uint32_t seg_max(uint32_t v) {
  if constexpr (S >= W) return v;
  else if constexpr (S == 16) {   // both copies of the swap at once: no need to know which is whose
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return seg_max<W, 32>(umax(r[0], r[1]));
  } else if constexpr (S == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return umax(r[0], r[1]);
  } else return seg_max<W, 2 * S>(umax(v, other<S>(v)));
}
template <int W, int S = 1>
__device__ __forceinline__ float seg_sum(float v) {
  if constexpr (S < W) return seg_sum<W, 2 * S>(v + other<S>(v));
  else return v;
}

// fp32 numbers as integers in the same order: -0 as +0, every number above 0 (kNone).
constexpr uint32_t kNone = 0;
__device__ __forceinline__ uint32_t order(float f) {
  const uint32_t b = __float_as_uint(f + 0.0f);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number(uint32_t u) {   // kNone: NaN
  return __uint_as_float(u ^ (static_cast<uint32_t>(~static_cast<int32_t>(u) >> 31) | 0x80000000u));
}
template <int W>
__device__ __forceinline__ float seg_fmax(float v) { return number(seg_max<W>(order(v))); }

__device__ __forceinline__ void lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// e^v and 1 / v by the hardware's 2^x and reciprocal (1 ulp each): relative error (|v| + 2) 2^-23 at most,
// which kKeyTol and the gates' accuracy (fp32 to a few ulp for logits of ordinary size) allow for.
__device__ __forceinline__ float fast_exp(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504f); }
__device__ __forceinline__ float fast_rcp(float v) { return __builtin_amdgcn_rcpf(v); }
__device__ __forceinline__ float fast_sigmoid(float z) { return fast_rcp(1.0f + fast_exp(-z)); }

// Numbers in the ratio of the scores of a token's entries, of which top is the largest logit: e^z for softmax, e^z / (1 + e^z)
// for sigmoid, times e^-top where that is needed to keep them in fp32's range (a sigmoid of -90 is 0 in fp32, beside one of
// -29 it is 3e-27).
__device__ __forceinline__ float ratio_weight(bool soft, float z, float top) {
  const bool low = top < 0.0f;
  const float rel = soft || low ? fast_exp(z - top) : 1.0f;
  return soft ? rel : rel * fast_rcp(1.0f + fast_exp(low ? z : -z));
}

// +inf counts as the largest finite logit; NaN and -inf leave the row (see live below).
__device__ __forceinline__ float clamp_logit(float z) { return fminf(z, FLT_MAX); }

// Errors of an fp32 key, relative to the largest s * prior + |bias| of the row. Softmax: the exponent's
// rounding (|x| 2^-23 e^x, at most 0.37 of 2^-23 where |x| e^x is largest), 2^x and reciprocal 1 ulp each, a row sum
// of up to 256 terms 8 additions deep, product, prior and bias 3: under 1.6e-6 in all. Sigmoid: less. Two
// keys are told apart at twice that, two group sums of two keys at four times; with a margin:
constexpr float kKeyTol = 4e-6f;

// e^x for x <= 0 in fp64: x = k ln 2 + r with |r| <= ln 2 / 2, the Taylor polynomial of degree 13 in r (its
// remainder is 4e-18), times 2^k. The reduction is Cody and Waite's: ln 2 as its first 32 binary places, of which k (11 bits)
// times is exact, and the rest. Coefficients come from memory one at a time: the library's exp keeps its own in
// registers through the loops around it, which leaves room for half the wavefronts.
__constant__ double kInvFactorial[14] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040,
                                         1.0 / 40320, 1.0 / 362880, 1.0 / 3628800, 1.0 / 39916800, 1.0 / 479001600,
                                         1.0 / 6227020800.0};
__device__ __forceinline__ double exp_neg(double x) {
  x = fmax(x, -800.0);   // 0 in fp64
  constexpr double kLn2First = 0x1.62e42feep-1, kLn2Rest = 0x1.a39ef35793c76p-33, kLog2E = 0x1.71547652b82fep+0;
  const double k = rint(x * kLog2E);
  const double r = fma(-k, kLn2Rest, fma(-k, kLn2First, x));
  double p = kInvFactorial[13];
#pragma unroll 1
  for (int i = 12; i >= 0; --i) p = fma(p, r, kInvFactorial[i]);
  return ldexp(p, static_cast<int>(k));
}

// How the keys order and the groups lie: keys that are the logits; keys s * prior + bias.
enum { kByLogit = 0, kByKey = 1 };
// no groups; groups of a power of two of lanes; of another number of lanes; of no whole lanes
enum { kNoGroups = 0, kLaneGroups = 1, kOddGroups = 2, kOtherGroups = 3 };

// What a lane knows of its V experts, the same for every token.
template <int V>
struct LaneExperts {
  float bias[V], prior[V];
  bool allowed[V];
};
template <int V, int KEYS>
__device__ __forceinline__ LaneExperts<V> lane_experts(const GateArgs& a, int e0) {
  LaneExperts<V> x;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = e0 + v;
    const bool in = e < a.E;
    x.bias[v] = KEYS == kByKey && in && a.bias ? a.bias[e] : 0.0f;
    x.prior[v] = KEYS == kByKey && in && a.has_prior ? a.prior[e] : 1.0f;
    x.allowed[v] = in && (!a.has_mask || (a.mask[e >> 5] >> (e & 31) & 1));
  }
  return x;
}

template <int V, bool VEC>
__device__ __forceinline__ void load_row(const GateArgs& a, int t, int e0, float (&z)[V]) {
  const float* zr = a.logits + static_cast<size_t>(t) * a.E;
  if constexpr (VEC && V == 4) {
    f32x4 q = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (e0 < a.E) q = *reinterpret_cast<const f32x4*>(zr + e0);
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] = q[v];
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] = e0 + v < a.E ? zr[e0 + v] : -INFINITY;
  }
}

template <int S>
__device__ __forceinline__ double other(double v) {
  return __hiloint2double(static_cast<int>(other<S>(static_cast<uint32_t>(__double2hiint(v)))),
                          static_cast<int>(other<S>(static_cast<uint32_t>(__double2loint(v)))));
}
template <int W, int S = 1>
__device__ __forceinline__ double seg_max(double v) {
  if constexpr (S < W) return seg_max<W, 2 * S>(fmax(v, other<S>(v)));
  else return v;
}
template <int W, int S = 1>
__device__ __forceinline__ double seg_sum(double v) {
  if constexpr (S < W) return seg_sum<W, 2 * S>(v + other<S>(v));
  else return v;
}

// Score of a logit in fp64; softmax: relative to the row's largest logit, before the division by the sum.
__device__ __forceinline__ double exact_score(bool soft, float z, float zmax) {
  const double x = exp_neg(soft ? static_cast<double>(z) - zmax : -fabs(static_cast<double>(z)));
  return soft ? x : (z >= 0.0f ? 1.0 : x) / (1.0 + x);
}

// Selection of one segment's token t with fp64 keys: lane r < K gets the r-th expert, -1 where none is left. keys and
// leads: LDS for the segment's W * V experts (leads: of their groups). Runs where fp32 keys came too close, or for
// groups whose size is no multiple of V.
template <int W, int V, bool VEC, int KEYS, int GROUPS>
__device__ __forceinline__ int select_exact(const GateArgs& a, const LaneExperts<V>& x, int t, int seg, int sl, double* keys,
                                            double* leads) {
  const double ninf = -INFINITY;
  const bool soft = a.score == 0;
  const int e0 = sl * V;
  float z[V];
  load_row<V, VEC>(a, t, e0, z);
  float zmax = -FLT_MAX;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    z[v] = z[v] > -INFINITY ? clamp_logit(z[v]) : -INFINITY;
    zmax = fmaxf(zmax, z[v]);
  }
  zmax = seg_fmax<W>(zmax);
  double key[V], sum = 0.0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    key[v] = z[v];
    if constexpr (KEYS == kByKey) {
      key[v] = exact_score(soft, z[v], zmax);
      if (z[v] > -INFINITY) sum += key[v];
      __builtin_amdgcn_sched_barrier(0);   // one exponential's registers at a time
    }
  }
  if constexpr (KEYS == kByKey) {
    sum = soft ? seg_sum<W>(sum) : 1.0;
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = key[v] / sum * x.prior[v] + x.bias[v];
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (!(z[v] > -INFINITY) || !x.allowed[v]) key[v] = ninf;
  if constexpr (GROUPS != kNoGroups) {
    const int n = a.E / a.n_group;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (e0 + v < a.E) keys[e0 + v] = key[v];
    lds_order();
#pragma unroll 1
    for (int g = sl; g < a.n_group; g += W) {
      double t1 = ninf, t2 = ninf;
#pragma unroll 4
      for (int i = 0; i < n; ++i) {
        const double k = keys[g * n + i];
        t2 = fmax(t2, fmin(t1, k));
        t1 = fmax(t1, k);
      }
      leads[g] = a.group_rule == 1 && t2 > ninf ? t1 + t2 : t1;
    }
    lds_order();
#pragma unroll 1
    for (int g = sl; g < a.n_group; g += W) {   // a group that is beaten too often loses its experts
      const double lead = leads[g];
      int ahead = 0;
#pragma unroll 4
      for (int o = 0; o < a.n_group; ++o) ahead += leads[o] > lead || (leads[o] == lead && o < g) ? 1 : 0;
      if (ahead >= a.topk_group)
#pragma unroll 1
        for (int i = 0; i < n; ++i) keys[g * n + i] = ninf;
    }
    lds_order();
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (e0 + v < a.E) key[v] = keys[e0 + v];
  }
  const uint64_t segbits = (W == 64 ? ~0ull : (1ull << W) - 1) << (seg * W);
  int mine = -1;
#pragma unroll 1
  for (int r = 0; r < a.K; ++r) {
    double head = key[0];
    int at = e0;
#pragma unroll
    for (int v = 1; v < V; ++v)
      if (key[v] > head) head = key[v], at = e0 + v;
    const double m = seg_max<W>(head);
    const uint64_t who = __ballot(head == m && m > ninf) & segbits;
    const int first = who ? __ffsll(static_cast<unsigned long long>(who)) - 1 : seg * W;
    const int e = who ? __shfl(at, first, kWave) : -1;
    if (sl == r) mine = e;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (e0 + v == e) key[v] = ninf;
  }
  return mine;
}

// The largest value that at least `need` and, where no equal values prevent it, at most `enough` of the lanes in
// `open` reach (found by comparing all with one that is still in question; with how many reach it), for a value per
// lane of a whole wavefront; 1 where fewer lanes hold one at all (kNone: none).
__device__ __forceinline__ uint32_t reached_by(uint32_t value, uint64_t open, int need, int enough, uint32_t& reach) {
  const uint64_t all = open;
  open &= __ballot(value != kNone);
  reach = static_cast<uint32_t>(__popcll(open));
  if (static_cast<int>(reach) <= need) return 1;
  for (;;) {
    const uint32_t pivot = static_cast<uint32_t>(
        __builtin_amdgcn_readlane(static_cast<int>(value), __ffsll(static_cast<unsigned long long>(open)) - 1));
    const uint64_t upto = __ballot(value >= pivot) & all;
    reach = static_cast<uint32_t>(__popcll(upto));
    if (static_cast<int>(reach) < need) {
      open &= ~upto;
    } else {
      if (static_cast<int>(reach) <= enough) return pivot;
      const uint64_t above = __ballot(value > pivot) & all;
      if (__popcll(above) < need) return pivot;
      open &= above;
    }
  }
}

struct Row {
  float zmax, total;   // softmax: largest logit and sum of e^(z - zmax) (where the gates or keys need them)
  float tol;           // how close two keys may come
  bool close;          // group scores came too close
};

// Keys of a row's logits z (overwritten) with the experts outside the kept groups dropped.
template <int W, int V, int KEYS, int GROUPS>
__device__ __forceinline__ Row row_keys(const GateArgs& a, const LaneExperts<V>& x, int seg, int e0, float pmax, float bmax,
                                        float (&z)[V], uint32_t (&key)[V]) {
  const float ninf = -INFINITY;
  const bool soft = a.score == 0;
  Row r{-FLT_MAX, 1.0f, 0.0f, GROUPS == kOtherGroups};
  bool ok[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const bool live = z[v] > ninf;   // false for NaN too
    z[v] = live ? clamp_logit(z[v]) : ninf;
    ok[v] = live && x.allowed[v];
  }
  if (soft && (KEYS == kByKey || !a.renorm)) {   // renormalised gates need no row sum
#pragma unroll
    for (int v = 0; v < V; ++v) r.zmax = fmaxf(r.zmax, z[v]);
    r.zmax = seg_fmax<W>(r.zmax);
    r.total = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) r.total += fast_exp(z[v] - r.zmax);   // 0 for -inf
    r.total = seg_sum<W>(r.total);
  }
  if constexpr (KEYS == kByLogit) {
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = ok[v] ? order(z[v]) : kNone;
  } else {
    const float inv = fast_rcp(r.total);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float s = soft ? fast_exp(z[v] - r.zmax) * inv : fast_sigmoid(z[v]);
      key[v] = ok[v] ? order(s * x.prior[v] + x.bias[v]) : kNone;
    }
    r.tol = kKeyTol * (pmax * (soft ? inv : 1.0f) + bmax);   // inv: the largest softmax score
  }
  if constexpr (GROUPS == kLaneGroups || GROUPS == kOddGroups) {
    const int n = a.E / a.n_group, glanes = n / V, own = e0 / n;
    const bool sum2 = KEYS == kByKey && a.group_rule == 1;
    uint32_t t1 = key[0], t2 = kNone;
#pragma unroll
    for (int v = 1; v < V; ++v) {
      t2 = umax(t2, umin(t1, key[v]));
      t1 = umax(t1, key[v]);
    }
    auto join = [&](uint32_t b1, uint32_t b2) {
      t2 = umax(umin(t1, b1), umax(t2, b2));
      t1 = umax(t1, b1);
    };
    if constexpr (GROUPS == kLaneGroups) {
      if (glanes > 1) join(other<1>(t1), other<1>(t2));
      if (glanes > 2) join(other<2>(t1), other<2>(t2));
      if (glanes > 4) join(other<4>(t1), other<4>(t2));
      if (glanes > 8) join(other<8>(t1), other<8>(t2));
      if (W > 16 && glanes > 16) join(other<16>(t1), other<16>(t2));
    } else {
      const uint32_t m1 = t1, m2 = t2;
      t1 = t2 = kNone;
      for (int i = 0; i < glanes; ++i) {
        const int from = seg * W + min(own, a.n_group - 1) * glanes + i;
        join(__shfl(m1, from, kWave), __shfl(m2, from, kWave));
      }
    }
    const uint32_t lead = sum2 && t2 != kNone ? order(number(t1) + number(t2)) : t1;
    bool kept;
    if constexpr (W == 64) {   // the first lane of every group stands for it
      const int lane = threadIdx.x & 63;
      const uint64_t firsts = __ballot(lane == own * glanes && own < a.n_group);
      uint32_t most;
      const uint32_t bound = reached_by(lead, firsts, a.topk_group, a.topk_group, most);
      kept = lead >= bound && own < a.n_group;
      // equal group scores at the bound, or (the keys being rounded) scores that come too close to it
      const uint32_t low = KEYS == kByKey && bound > kNone + 1 ? umax(order(number(bound) - 2.0f * r.tol), 1u) : bound;
      r.close = most > static_cast<uint32_t>(a.topk_group) ||
                __popcll(__ballot(lead >= low) & firsts) > static_cast<int>(most);
    } else {
      int ahead = 0;
      for (int g = 0; g < a.n_group; ++g) {
        const uint32_t o = __shfl(lead, seg * W + g * glanes, kWave);
        ahead += o > lead || (o == lead && g < own) ? 1 : 0;
      }
      kept = ahead < a.topk_group && own < a.n_group;
      if constexpr (KEYS == kByKey) {
        // the last group kept and the first one left out; lanes past the last expert hold no group (a copy of the last
        // one's score among those left out sent every row that keeps it to fp64: 65536 tokens x 24 experts in 2 groups
        // 34 us instead of 17)
        const float in = number(~seg_max<W>(kept ? ~lead : 0u));
        const float out = number(seg_max<W>(kept || own >= a.n_group ? kNone : lead));
        r.close = in - out < 2.0f * r.tol;   // no group left out, or none with an expert: NaN, not close
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = kept ? key[v] : kNone;
  }
  return r;
}

// The largest prior and |bias| of the experts that have a key (for the keys' errors), over the W lanes of a segment. What
// is masked or past the last expert has none: counted, the latter's prior of 1 sent every row under small priors to fp64
// (65536 tokens x 160 experts, priors 2^-20, 121 us instead of 42), as a large bias of a masked expert did.
template <int W, int V>
__device__ __forceinline__ void key_bounds(const LaneExperts<V>& x, float& pmax, float& bmax) {
  pmax = bmax = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    pmax = fmaxf(pmax, x.allowed[v] ? x.prior[v] : 0.0f);
    bmax = fmaxf(bmax, x.allowed[v] ? fabsf(x.bias[v]) : 0.0f);
  }
  pmax = seg_fmax<W>(pmax);
  bmax = seg_fmax<W>(bmax);
}

// The W lanes of a token write its entries: this lane entry r (if r < K), expert e (-1: none), whose (clamped) logit is
// given, and its gate.
template <int W>
__device__ __forceinline__ void write_gate(const GateArgs& a, int t, bool real, int r, int e, float logit, float zmax,
                                           float total, int* hist) {
  const bool has = e >= 0, soft = a.score == 0;
  const float zs = has ? logit : -INFINITY;
  float g;
  if (a.renorm) {
    const float top = seg_fmax<W>(fmaxf(zs, -FLT_MAX));
    const float w = has ? ratio_weight(soft, zs, top) : 0.0f;
    g = a.scale * (w / seg_sum<W>(w));
  } else {
    g = a.scale * (soft ? fast_exp(zs - zmax) / total : fast_sigmoid(zs));
  }
  if (real && r < a.K) {
    a.idx[static_cast<size_t>(t) * a.K + r] = e;
    a.gate[static_cast<size_t>(t) * a.K + r] = has ? g : 0.0f;
    if (a.load && has) atomicAdd(&hist[e], 1);   // integer counts: order-independent
  }
}
__device__ __forceinline__ void clear_hist(const GateArgs& a, int* hist) {
  if (!a.load) return;
  for (int e = threadIdx.x; e < a.E; e += kThreads) hist[e] = 0;
  __syncthreads();
}
__device__ __forceinline__ void add_hist(const GateArgs& a, const int* hist) {
  if (!a.load) return;
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kThreads) {
    if (gridDim.x == 1) a.load[e] = hist[e];
    else if (hist[e]) atomicAdd(&a.load[e], hist[e]);
  }
}

// Up to 64 experts: four tokens per wavefront, 16 lanes each.
template <int V, bool VEC, int KEYS, int GROUPS>
__global__ __launch_bounds__(kThreads) void gate_kernel(const GateArgs a) {
  constexpr int W = 16, SEGS = kWave / W, PER = SEGS * kWaves;   // tokens per wavefront and workgroup
  constexpr bool EXACT = KEYS == kByKey || GROUPS == kOtherGroups;   // may select in fp64
  __shared__ uint2 sel[PER][kGateMaxK];  // selected experts and their keys
  constexpr bool GROUPED = EXACT && GROUPS != kNoGroups;
  __shared__ double rows[GROUPED ? PER : 1][W * V], leads[GROUPED ? PER : 1][W * V];
  __shared__ int hist[kGateMaxE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seg = lane / W, sl = lane % W, e0 = sl * V;
  const int slot = wave * SEGS + seg;
  float next[V];
  const int stride = gridDim.x * PER;
  load_row<V, VEC>(a, min(static_cast<int>(blockIdx.x) * PER + slot, a.T - 1), e0, next);
  const LaneExperts<V> x = lane_experts<V, KEYS>(a, e0);
  clear_hist(a, hist);
  float pmax, bmax;
  key_bounds<W>(x, pmax, bmax);
  const uint32_t below = (1u << sl) - 1;   // lower lanes of the segment
  for (int t0 = blockIdx.x * PER; t0 < a.T; t0 += stride) {
    const int t = min(t0 + slot, a.T - 1);   // segments past the last token repeat it, unwritten
    float z[V];
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] = next[v];
    load_row<V, VEC>(a, min(t0 + slot + stride, a.T - 1), e0, next);   // the next round's row, behind this one's work
    uint32_t key[V];
    Row row = row_keys<W, V, KEYS, GROUPS>(a, x, seg, e0, pmax, bmax, z, key);
    // the lane's keys by decreasing key, equal ones by increasing expert
    int id[V];
#pragma unroll
    for (int v = 0; v < V; ++v) id[v] = e0 + v;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j + 1 < V - i; ++j) {
        const bool sw = key[j + 1] > key[j];   // strict: a lower expert stays ahead of its equal
        const uint32_t k = key[j];
        const int y = id[j];
        key[j] = sw ? key[j + 1] : k;
        key[j + 1] = sw ? k : key[j + 1];
        id[j] = sw ? id[j + 1] : y;
        id[j + 1] = sw ? y : id[j + 1];
      }
    uint32_t m = seg_max<W>(key[0]);
    for (int r = 0; r < a.K; ++r) {
      const uint64_t at = __ballot(key[0] == m);
      const uint32_t half = static_cast<uint32_t>(lane < 32 ? at : at >> 32) >> (lane & 16);
      const bool mine = key[0] == m && (half & below) == 0;
      if (mine) sel[slot][r] = make_uint2(m == kNone ? 0xffffffffu : static_cast<uint32_t>(id[0]), m);
#pragma unroll
      for (int v = 0; v + 1 < V; ++v) {
        key[v] = mine ? key[v + 1] : key[v];
        id[v] = mine ? id[v + 1] : id[v];
      }
      key[V - 1] = mine ? kNone : key[V - 1];
      m = seg_max<W>(key[0]);
    }
    lds_order();
    int e = -1;
    uint32_t ke = kNone;
    if (sl < a.K) {
      const uint2 q = sel[slot][sl];
      e = static_cast<int>(q.x);
      ke = q.y;
    }
    if constexpr (EXACT) {
      if constexpr (KEYS == kByKey) {   // m: the best key left out
        uint32_t after = dpp<0x101>(ke);   // the next lane's (row_shl:1)
        after = sl == a.K - 1 ? m : after;
        row.close |= sl < a.K && number(ke) - number(after) < row.tol;   // kNone: NaN, not close
      }
      if (__any(row.close)) {
        e = select_exact<W, V, VEC, KEYS, GROUPS>(a, x, t, seg, sl, rows[GROUPED ? slot : 0], leads[GROUPED ? slot : 0]);
      }
    }
    lds_order();
    const float logit = e >= 0 ? clamp_logit(a.logits[static_cast<size_t>(t) * a.E + e]) : 0.0f;
    write_gate<W>(a, t, t0 + slot < a.T, sl, e, logit, row.zmax, row.total, hist);
  }
  add_hist(a, hist);
}

// More than 64 experts: a wavefront finds the candidates of `batch` (up to 64 / C) tokens one after the other, a row over
// its 64 lanes, and then ranks them all at once, C lanes a token, by fp64 keys of the candidates alone. Bound by the
// first part: 131072 tokens x 256 experts in 8 groups take 112 to 117 us, of which the 142 MB would be 30. Its 300 vector
// instructions a token are 64 us of issue over the chip; the rest is the chain of ballots, counts and lane reads of one token's
// bound, and a loop over tokens that the compiler does not know to be uniform (`wave` is no scalar to it), which puts
// counters and row addresses in vector registers. Six wavefronts a SIMD leave 80 registers, of which some 16 are stored and
// reloaded once a batch.
template <int V, bool VEC, int KEYS, int GROUPS, int C>
__global__ __launch_bounds__(kThreads, 6) void gate_rows_kernel(const GateArgs a, int batch) {
  constexpr int TB = kWave / C;
  constexpr bool GROUPED = GROUPS != kNoGroups;
  struct Found {
    float zmax, total, tol;
    int again;                             // select in fp64: group scores too close, or more candidates than C
  };
  struct Candidate {
    uint32_t key, expert;
    float logit, bias;
  };
  __shared__ __align__(16) Candidate cand[kWaves][TB][C];
  __shared__ double cand64[KEYS == kByKey ? kWaves : 1][TB][C];
  __shared__ Found found[kWaves][TB];
  __shared__ double rows[GROUPED ? kWaves : 1][64 * V], leads[GROUPED ? kWaves : 1][64 * V];
  __shared__ int hist[kGateMaxE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, e0 = lane * V;
  const int seg = lane / C, sl = lane % C;
  const int stride = gridDim.x * kWaves * batch;
  int t0 = (blockIdx.x * kWaves + wave) * batch;
  float next[V];
  load_row<V, VEC>(a, min(t0, a.T - 1), e0, next);
  const LaneExperts<V> x = lane_experts<V, KEYS>(a, e0);
  clear_hist(a, hist);
  float pmax, bmax;
  key_bounds<kWave>(x, pmax, bmax);
  for (; t0 < a.T; t0 += stride) {
    cand[wave][seg][sl] = Candidate{kNone, 0xffffffffu, 0.0f, 0.0f};
    lds_order();
    const int count = min(batch, a.T - t0);
    for (int k = 0; k < count; ++k) {
      float z[V];
#pragma unroll
      for (int v = 0; v < V; ++v) z[v] = next[v];
      load_row<V, VEC>(a, min(k + 1 < count ? t0 + k + 1 : t0 + stride, a.T - 1), e0, next);
      uint32_t key[V];
      const Row row = row_keys<kWave, V, KEYS, GROUPS>(a, x, 0, e0, pmax, bmax, z, key);
      uint32_t head = key[0], reach;
#pragma unroll
      for (int v = 1; v < V; ++v) head = umax(head, key[v]);
      // a bound that the heads of K lanes or two more reach: so do the K best keys, and some others
      uint32_t bound = reached_by(head, ~0ull, a.K, a.K + 2, reach);
      uint64_t at[V];
      int n;
      // The candidates: keys that reach the bound; rounded ones also where their real values might
      auto candidates = [&](uint32_t b) {
        if constexpr (KEYS == kByKey)
          if (b > 1) b = umax(order(number(b) - row.tol), 1u);
        n = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          at[v] = __ballot(key[v] >= b);
          n += __popcll(at[v]);
        }
      };
      candidates(bound);
      if (n > C) {   // several large keys in one lane: a higher bound, as long as K keys reach it
        uint32_t high = 0xffffffffu;
        for (;;) {
          const uint64_t open = __ballot(head > bound && head < high);
          if (open == 0) break;
          const uint32_t pivot = static_cast<uint32_t>(
              __builtin_amdgcn_readlane(static_cast<int>(head), __ffsll(static_cast<unsigned long long>(open)) - 1));
          int reach_all = 0;
#pragma unroll
          for (int v = 0; v < V; ++v) reach_all += __popcll(__ballot(key[v] >= pivot));
          if (reach_all < a.K) {
            high = pivot;
          } else {
            bound = pivot;
            candidates(bound);
            if (n <= C) break;
          }
        }
      }
      if (n <= C) {
        int base = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int pos = static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(at[v] >> 32),
                                                                     __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(at[v]), base)));
          if (at[v] >> lane & 1) cand[wave][k][pos] = Candidate{key[v], static_cast<uint32_t>(e0 + v), z[v], x.bias[v]};
          base += __popcll(at[v]);
        }
      }
      if (lane == 0) found[wave][k] = Found{row.zmax, row.total, row.tol, row.close || n > C ? 1 : 0};
    }
    lds_order();
    // lane (token seg, candidate sl): its rank among the token's candidates, by fp64 keys
    const int t = min(t0 + seg, a.T - 1);
    const bool real = seg < count;
    const Found f = found[wave][real ? seg : 0];
    const Candidate own = cand[wave][seg][sl];
    const bool has = own.key != kNone;
    float logit = own.logit;
    int rank = 0;
    bool close = real && f.again;
    if constexpr (KEYS == kByKey) {
      double k = -INFINITY;
      if (has) {
        k = exact_score(a.score == 0, own.logit, f.zmax);
        if (a.score == 0 && a.bias) k /= f.total;   // without bias the order does not depend on the sum
        if (a.has_prior) k *= a.prior[own.expert];
        k += own.bias;
      }
      cand64[wave][seg][sl] = k;
      lds_order();
      double gap = INFINITY;
#pragma unroll 4
      for (int j = 0; j < C; ++j) {
        const double o = cand64[wave][seg][j];
        rank += o > k || (o == k && cand[wave][seg][j].expert < own.expert) ? 1 : 0;
        gap = j == sl ? gap : fmin(gap, fabs(o - k));
      }
      // a sum in fp32 beside a bias: the keys are no better than fp32
      if (a.score == 0 && a.bias) close |= real && has && rank < a.K && gap < f.tol;
    } else {
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const uint32_t o = cand[wave][seg][j].key;
        rank += o > own.key || (o == own.key && cand[wave][seg][j].expert < own.expert) ? 1 : 0;
      }
    }
    // a selected candidate's lane writes its entry; lanes without a candidate the entries that are left over
    int r = rank, e = has && rank < a.K ? static_cast<int>(own.expert) : -1;
    if (!has) {
      const uint32_t filled = static_cast<uint32_t>(__ballot(has) >> (C * seg)) & static_cast<uint32_t>((1ull << C) - 1);
      r = __popc(filled) + __popc(~filled & ((1u << sl) - 1));
    }
    const uint64_t again = __ballot(close);
    if (again != 0) {
#pragma unroll 1
      for (int k = 0; k < count; ++k) {
        if ((again >> (C * k) & ((1ull << C) - 1)) == 0) continue;
        const int ex = select_exact<kWave, V, VEC, KEYS, GROUPS>(a, x, t0 + k, 0, lane, rows[GROUPED ? wave : 0],
                                                                 leads[GROUPED ? wave : 0]);
        const int mine = __shfl(ex, sl, kWave);   // entry sl, for the token's lanes
        if (seg == k) {
          e = sl < a.K ? mine : -1;
          r = sl;
          logit = e >= 0 ? clamp_logit(a.logits[static_cast<size_t>(t) * a.E + e]) : 0.0f;
        }
      }
    }
    lds_order();
    write_gate<C>(a, t, real, r, e, logit, f.zmax, f.total, hist);
  }
  add_hist(a, hist);
}

__global__ void gate_zero_kernel(int32_t* load, int E) {
  if (static_cast<int>(threadIdx.x) < E) load[threadIdx.x] = 0;
}

constexpr int kRowsK = 10;   // experts up to which 16 candidates of a token nearly always suffice

template <int V, bool ROWS, bool VEC, int KEYS, int GROUPS>
void launch_one(const GateArgs& a, int blocks, int batch, hipStream_t stream) {
  if constexpr (ROWS) {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, stream, a, batch); };
    if (a.K <= kRowsK) go(gate_rows_kernel<V, VEC, KEYS, GROUPS, 16>);
    else go(gate_rows_kernel<V, VEC, KEYS, GROUPS, 32>);
  } else {
    hipLaunchKernelGGL((gate_kernel<V, VEC, KEYS, GROUPS>), dim3(blocks), dim3(kThreads), 0, stream, a);
  }
}
template <int V, bool ROWS, bool VEC, int KEYS>
void launch_groups(const GateArgs& a, int blocks, int batch, hipStream_t stream) {
  const int n = a.E / a.n_group, lanes = n / V;
  if (a.n_group == 1 || a.topk_group == a.n_group) launch_one<V, ROWS, VEC, KEYS, kNoGroups>(a, blocks, batch, stream);
  else if (n % V != 0) launch_one<V, ROWS, VEC, KEYS, kOtherGroups>(a, blocks, batch, stream);
  else if ((lanes & (lanes - 1)) == 0) launch_one<V, ROWS, VEC, KEYS, kLaneGroups>(a, blocks, batch, stream);
  else launch_one<V, ROWS, VEC, KEYS, kOddGroups>(a, blocks, batch, stream);
}

template <int V, bool ROWS>
hipError_t launch_gate(const GateArgs& a, hipStream_t stream) {
  if (a.T == 0 && !a.load) return hipSuccess;
  // rows over a wavefront: one token each while the chip holds a wavefront for every token (8192), else as many as
  // are ranked at once
  const int batch = !ROWS ? 4 : a.T <= 8192 ? 1 : a.K <= kRowsK ? 4 : 2;
  const int per = batch * kWaves, blocks = std::max(1, std::min((a.T + per - 1) / per, 256 * 8));
  if (a.load && (blocks > 1 || a.T == 0)) {
    hipLaunchKernelGGL(gate_zero_kernel, dim3(1), dim3(kGateMaxE), 0, stream, a.load, a.E);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess || a.T == 0) return err;
  }
  const bool by_key = a.bias || a.has_prior || (a.n_group > 1 && a.group_rule == 1);
  const bool vec = V == 4 && a.E % 4 == 0 && (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0;
  constexpr bool VEC = V == 4;
  if (vec && by_key) launch_groups<V, ROWS, VEC, kByKey>(a, blocks, batch, stream);
  else if (vec) launch_groups<V, ROWS, VEC, kByLogit>(a, blocks, batch, stream);
  else if (by_key) launch_groups<V, ROWS, false, kByKey>(a, blocks, batch, stream);
  else launch_groups<V, ROWS, false, kByLogit>(a, blocks, batch, stream);
  return hipGetLastError();
}

// dL/dz of the gates (include/maskmoe.h, maskmoe_gate_backward), bound by the rows of d_logits that it writes.
// Entry r of a token sits in lane r of 16.
struct Entry {
  int e;          // expert, -1 for none
  float dg, zs;   // scale * d_gate, the expert's logit
};
__device__ __forceinline__ Entry load_entry(const GateBwdArgs& a, int t, int r) {
  Entry x{-1, 0.0f, -INFINITY};
  if (r < a.K) {
    const int e = a.idx[static_cast<size_t>(t) * a.K + r];
    const float dg = a.d_gate[static_cast<size_t>(t) * a.K + r];
    if (e >= 0 && e < a.E) {
      const float z = a.logits[static_cast<size_t>(t) * a.E + e];
      if (z > -INFINITY) x = {e, a.scale * dg, clamp_logit(z)};
    }
  }
  return x;
}

// Gates of a softmax that is not renormalised: every expert of the row has a gradient. A segment of W lanes per
// token, V experts a lane; every lane adds the entries that name its experts, in order of r.
template <int W, int V, bool VEC>
__global__ __launch_bounds__(kThreads) void gate_bwd_dense_kernel(const GateBwdArgs a) {
  constexpr int SEGS = kWave / W, PER = SEGS * kWaves;
  __shared__ uint2 ent[PER][kGateMaxK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seg = lane / W, sl = lane % W, e0 = sl * V;
  const int slot = wave * SEGS + seg;
  const float ninf = -INFINITY;
  for (int t0 = blockIdx.x * PER; t0 < a.T; t0 += gridDim.x * PER) {
    const int t = min(t0 + slot, a.T - 1);
    const bool real = t0 + slot < a.T;
    const float* zr = a.logits + static_cast<size_t>(t) * a.E;
    float z[V], zmax = -FLT_MAX, total = 0.0f;
    if constexpr (VEC) {
      f32x4 q = {ninf, ninf, ninf, ninf};
      if (e0 < a.E) q = *reinterpret_cast<const f32x4*>(zr + e0);
#pragma unroll
      for (int v = 0; v < V; ++v) z[v] = q[v];
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) z[v] = e0 + v < a.E ? zr[e0 + v] : ninf;
    }
    const Entry x = load_entry(a, t, sl);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      z[v] = z[v] > ninf ? clamp_logit(z[v]) : ninf;
      zmax = fmaxf(zmax, z[v]);
    }
    zmax = seg_fmax<W>(zmax);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      z[v] = fast_exp(z[v] - zmax);
      total += z[v];
    }
    total = seg_sum<W>(total);
    if (sl < a.K) ent[slot][sl] = make_uint2(static_cast<uint32_t>(x.e), __float_as_uint(x.dg));
    lds_order();
    float out[V], pd = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = 0.0f;
    for (int r = 0; r < a.K; ++r) {
      const uint2 er = ent[slot][r];
#pragma unroll
      for (int v = 0; v < V; ++v) out[v] += static_cast<int>(er.x) == e0 + v ? __uint_as_float(er.y) : 0.0f;
    }
    lds_order();
    const float inv = 1.0f / total;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      z[v] = total > 0.0f ? z[v] * inv : 0.0f;   // a row without a finite logit has no gradient
      pd += z[v] * out[v];
    }
    pd = seg_sum<W>(pd);
    if (!real) continue;
    float* o = a.d_logits + static_cast<size_t>(t) * a.E;
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = z[v] * (out[v] - pd);
    if constexpr (VEC) {
      if (e0 < a.E) *reinterpret_cast<f32x4*>(o + e0) = f32x4{out[0], out[1], out[2], out[3]};
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (e0 + v < a.E) o[e0 + v] = out[v];
    }
  }
}

// The other gates: only the entries' experts have a gradient. A wavefront takes four tokens, whose entries are its 64
// lanes; the four rows (consecutive in d_logits) are put together in LDS, where all else stays zero.
template <bool VEC>
__global__ __launch_bounds__(kThreads) void gate_bwd_sparse_kernel(const GateBwdArgs a) {
  __shared__ __align__(16) float rows[kWaves][4 * kGateMaxE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15;
  const bool soft = a.score == 0;
  float* row = rows[wave];
  for (int i = lane; i < 4 * a.E; i += kWave) row[i] = 0.0f;
  lds_order();
  const int stride = gridDim.x * kWaves * 4;
  for (int t0 = (blockIdx.x * kWaves + wave) * 4; t0 < a.T; t0 += stride) {
    const int t = t0 + (lane >> 4);
    Entry x{-1, 0.0f, -INFINITY};
    if (t < a.T) x = load_entry(a, t, l16);
    const bool has = x.e >= 0;
    float d;
    if (a.renorm) {
      const float top = seg_fmax<16>(fmaxf(x.zs, -FLT_MAX));
      float w = has ? ratio_weight(soft, x.zs, top) : 0.0f;
      const float s = seg_sum<16>(w);
      w = has ? w / s : 0.0f;
      const float mean = seg_sum<16>(w * x.dg);
      d = w * (x.dg - mean) * (soft ? 1.0f : fast_sigmoid(-x.zs));
    } else {   // s (1 - s), the second factor as the sigmoid of -z
      d = x.dg * fast_sigmoid(x.zs) * fast_sigmoid(-x.zs);
    }
    float* at = row + (lane >> 4) * a.E + x.e;
    if (has) *at = static_cast<float>(lane);
    lds_order();
    const bool twice = has && *at != static_cast<float>(lane);   // another entry names the same expert
    lds_order();
    if (__any(twice)) {   // entries in order, one at a time
      if (has) *at = 0.0f;
      lds_order();
#pragma unroll 1
      for (int r = 0; r < a.K; ++r) {
        if (has && l16 == r) *at += d;
        lds_order();
      }
    } else if (has) {
      *at = d;
    }
    lds_order();
    const int n = min(4, a.T - t0) * a.E;
    float* o = a.d_logits + static_cast<size_t>(t0) * a.E;
    if constexpr (VEC) {
      for (int i = 4 * lane; i < n; i += 4 * kWave)
        *reinterpret_cast<f32x4*>(o + i) = *reinterpret_cast<const f32x4*>(row + i);
    } else {
      for (int i = lane; i < n; i += kWave) o[i] = row[i];
    }
    lds_order();
    if (has) *at = 0.0f;
    lds_order();
  }
}

template <int W, int V>
void launch_dense(const GateBwdArgs& a, bool vec, hipStream_t stream) {
  constexpr int PER = kWave / W * kWaves;
  const dim3 grid(std::min((a.T + PER - 1) / PER, 256 * 16));
  if (V == 4 && vec) hipLaunchKernelGGL((gate_bwd_dense_kernel<W, V, V == 4>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((gate_bwd_dense_kernel<W, V, false>), grid, dim3(kThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_gate_forward(const GateArgs& a, hipStream_t stream) {
  if (a.E <= 16) return launch_gate<1, false>(a, stream);
  if (a.E <= 64) return launch_gate<4, false>(a, stream);
  if (a.E <= 128) return launch_gate<2, true>(a, stream);
  return launch_gate<4, true>(a, stream);
}

hipError_t launch_gate_backward(const GateBwdArgs& a, hipStream_t stream) {
  const bool vec = a.E % 4 == 0 && ((reinterpret_cast<uintptr_t>(a.logits) | reinterpret_cast<uintptr_t>(a.d_logits)) & 15) == 0;
  if (a.score == 0 && !a.renorm) {
    if (a.E <= 16) launch_dense<16, 1>(a, vec, stream);
    else if (a.E <= 64) launch_dense<16, 4>(a, vec, stream);
    else if (a.E <= 128) launch_dense<32, 4>(a, vec, stream);
    else launch_dense<64, 4>(a, vec, stream);
    return hipGetLastError();
  }
  const dim3 grid(std::min((a.T + 4 * kWaves - 1) / (4 * kWaves), 256 * 8));
  if (vec) hipLaunchKernelGGL(gate_bwd_sparse_kernel<true>, grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(gate_bwd_sparse_kernel<false>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace maskmoe
