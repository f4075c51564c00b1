// Routing by scores, balance bias and expert groups (include/maskmoe.h, maskmoe_gate_forward), and
// the gradient of its gates.
//
// A token takes a segment of W lanes (16, 32 or 64), each of which holds V consecutive experts in
// registers, so that a row of logits is read once, in order, and lower lanes hold lower experts:
//   scores    softmax or sigmoid of the registers, row maximum and sum by lane exchanges;
//   groups    the two largest keys of a group by lane exchanges, its rank by comparing it with every other; a
//             group stays if fewer than topk_group groups beat it;
//   top-K     every lane sorts its V keys; each round takes the largest first key of the segment and
//             the lowest lane that holds it, which drops it.
// Keys travel as integers that order as the numbers do (0: no eligible expert), so that a step of an
// exchange is one instruction.
// Selection goes by real numbers: keys are compared in fp32, and where two keys that the result
// depends on come closer than fp32 can tell apart (a bound on its errors, below), the wavefront
// selects again with keys in fp64 from LDS (select_exact, plain loops: about one token in 300 with 256 experts).
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

// +inf counts as the largest finite logit; NaN and -inf leave the row (see live below).
__device__ __forceinline__ float clamp_logit(float z) { return fminf(z, FLT_MAX); }

// Errors of an fp32 key, relative to the largest s * prior + |bias| of the row. Softmax: the exponent's
// rounding (|x| 2^-23 e^x, at most 0.37 of 2^-23 where |x| e^x is largest), 2^x and reciprocal 1 ulp each, a row sum
// of up to 256 terms 8 additions deep, product, prior and bias 3: under 1.6e-6 in all. Sigmoid: less. Two
// keys are told apart at twice that, two group sums of two keys at four times; with a margin:
constexpr float kKeyTol = 4e-6f;

// e^x for x <= 0 in fp64: x = k ln 2 + r with |r| <= ln 2 / 2, the Taylor polynomial of degree 13 in r (its
// remainder is 4e-18), times 2^k. Coefficients come from memory one at a time: the library's exp keeps its own in
// registers through the loops below, which left room for half the wavefronts (113 registers instead of 62).
__constant__ double kInvFactorial[14] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040,
                                         1.0 / 40320, 1.0 / 362880, 1.0 / 3628800, 1.0 / 39916800, 1.0 / 479001600,
                                         1.0 / 6227020800.0};
__device__ __forceinline__ double exp_neg(double x) {
  x = fmax(x, -800.0);   // 0 in fp64
  const double k = rint(x * 1.4426950408889634);
  const double r = fma(-k, 1.9082149292705877e-10, fma(-k, 0.6931471803691238, x));   // ln 2 in two parts
  double p = kInvFactorial[13];
#pragma unroll 1
  for (int i = 12; i >= 0; --i) p = fma(p, r, kInvFactorial[i]);
  return ldexp(p, static_cast<int>(k));
}

// Selection of one segment's token (logits zr) with fp64 keys, in LDS: `keys` of E experts, -inf where
// ineligible, `leads` of the groups. out receives the selected experts, -1 where none is left. Plain loops that
// read everything again and hold little: rarely run, or run for groups whose size is no multiple of V.
template <int W>
__device__ __forceinline__ void select_exact(const GateArgs& a, const float* zr, int sl, bool by_key, double* keys,
                                             double* leads, int* out) {
  const double ninf = -INFINITY;
  const bool soft = by_key && a.score == 0;
  float top = -FLT_MAX;
  double sum = 0.0;
  if (soft) {
#pragma unroll 1
    for (int e = sl; e < a.E; e += W) top = fmaxf(top, clamp_logit(zr[e] > -INFINITY ? zr[e] : -FLT_MAX));
    top = seg_fmax<W>(top);
#pragma unroll 1
    for (int e = sl; e < a.E; e += W)
      if (zr[e] > -INFINITY) sum += exp_neg(static_cast<double>(clamp_logit(zr[e])) - top);
#pragma unroll 1
    for (int m = 1; m < W; m *= 2) sum += __shfl_xor(sum, m, kWave);
  }
#pragma unroll 1
  for (int e = sl; e < a.E; e += W) {
    double k = clamp_logit(zr[e]);
    const bool ok = zr[e] > -INFINITY && (!a.has_mask || (a.mask[e >> 5] >> (e & 31) & 1));
    if (by_key) {
      const double x = exp_neg(soft ? k - top : -fabs(k));
      k = soft ? x / sum : (k >= 0 ? 1.0 : x) / (1.0 + x);
      if (a.has_prior) k *= a.prior[e];
      if (a.bias) k += a.bias[e];
    }
    keys[e] = ok ? k : ninf;
  }
  lds_order();
  if (a.n_group > 1) {
    const int n = a.E / a.n_group;
#pragma unroll 1
    for (int g = sl; g < a.n_group; g += W) {
      double t1 = ninf, t2 = ninf;
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const double k = keys[g * n + i];
        t2 = fmax(t2, fmin(t1, k));
        t1 = fmax(t1, k);
      }
      leads[g] = a.group_rule == 1 && t2 > ninf ? t1 + t2 : t1;
    }
    lds_order();
#pragma unroll 1
    for (int e = sl; e < a.E; e += W) {
      const int own = e / n;
      const double lead = leads[own];
      int ahead = 0;
#pragma unroll 1
      for (int g = 0; g < a.n_group; ++g) ahead += leads[g] > lead || (leads[g] == lead && g < own) ? 1 : 0;
      if (ahead >= a.topk_group) keys[e] = ninf;
    }
    lds_order();
  }
#pragma unroll 1
  for (int r = 0; r < a.K; ++r) {
    double best = ninf;
    int at = 0x7fffffff;
#pragma unroll 1
    for (int e = sl; e < a.E; e += W) {
      const double k = keys[e];
      if (k > best) best = k, at = e;
    }
#pragma unroll 1
    for (int m = 1; m < W; m *= 2) {
      const double ok = __shfl_xor(best, m, kWave);
      const int oe = __shfl_xor(at, m, kWave);
      if (ok > best || (ok == best && oe < at)) best = ok, at = oe;
    }
    lds_order();
    if (sl == 0) {
      out[r] = best > ninf ? at : -1;
      if (best > ninf) keys[at] = ninf;
    }
    lds_order();
  }
}

// How the keys order and the groups lie: keys that are the logits; keys s * prior + bias.
enum { kByLogit = 0, kByKey = 1 };
// no groups; groups of a power of two of lanes; of another number of lanes; of no whole lanes
enum { kNoGroups = 0, kLaneGroups = 1, kOddGroups = 2, kOtherGroups = 3 };

template <int W, int V, bool VEC, int KEYS, int GROUPS>
__global__ __launch_bounds__(kThreads) void gate_kernel(const GateArgs a) {
  constexpr int SEGS = kWave / W;        // tokens per wavefront
  constexpr int PER = SEGS * kWaves;     // tokens per workgroup and round
  constexpr bool EXACT = KEYS == kByKey || GROUPS == kOtherGroups;   // may select in fp64
  __shared__ uint2 sel[PER][kGateMaxK];  // selected experts and their keys
  __shared__ int exact_sel[EXACT ? PER : 1][kGateMaxK];
  __shared__ double rows[EXACT ? PER : 1][W * V], leads[EXACT && GROUPS != kNoGroups ? PER : 1][W * V];
  __shared__ int hist[kGateMaxE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seg = lane / W, sl = lane % W, e0 = sl * V;
  const int slot = wave * SEGS + seg;
  if (a.load) {
    for (int e = tid; e < a.E; e += kThreads) hist[e] = 0;
    __syncthreads();
  }
  float bias[V], prior[V];
  bool allowed[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = e0 + v;
    const bool in = e < a.E;
    bias[v] = KEYS == kByKey && in && a.bias ? a.bias[e] : 0.0f;
    prior[v] = KEYS == kByKey && in && a.has_prior ? a.prior[e] : 1.0f;
    allowed[v] = in && (!a.has_mask || (a.mask[e >> 5] >> (e & 31) & 1));
  }
  const bool soft = a.score == 0;
  const float ninf = -INFINITY;
  const int n = a.E / a.n_group, glanes = n / V, own = e0 / n;   // group of this lane (kLaneGroups, kOddGroups)
  const uint32_t below = (1u << (lane & (W < 32 ? W - 1 : 31))) - 1;   // W < 64: lower lanes of the segment
  auto load = [&](int t, float (&z)[V]) {
    const float* zr = a.logits + static_cast<size_t>(t) * a.E;
    if constexpr (VEC) {
      f32x4 q = {ninf, ninf, ninf, ninf};
      if (e0 < a.E) q = *reinterpret_cast<const f32x4*>(zr + e0);
#pragma unroll
      for (int v = 0; v < V; ++v) z[v] = q[v];
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) z[v] = e0 + v < a.E ? zr[e0 + v] : ninf;
    }
  };
  float next[V];
  const int stride = gridDim.x * PER;
  const int first = blockIdx.x * PER + slot;
  load(min(first, a.T - 1), next);
  for (int t0 = blockIdx.x * PER; t0 < a.T; t0 += stride) {
    const int t = min(t0 + slot, a.T - 1);   // segments past the last token repeat it, unwritten
    const bool real = t0 + slot < a.T;
    float z[V];
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] = next[v];
    load(min(t0 + slot + stride, a.T - 1), next);   // the next round's row, behind this one's work
    float zmax = -FLT_MAX, total = 1.0f;
    bool live[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      live[v] = z[v] > ninf;   // false for NaN too
      z[v] = live[v] ? clamp_logit(z[v]) : ninf;
    }
    if (soft && (KEYS == kByKey || !a.renorm)) {   // renormalised gates need no row sum
#pragma unroll
      for (int v = 0; v < V; ++v) zmax = fmaxf(zmax, z[v]);
      zmax = seg_fmax<W>(zmax);
      total = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) total += fast_exp(z[v] - zmax);   // 0 for -inf
      total = seg_sum<W>(total);
    }
    uint32_t key[V];
    float mag = 0.0f;
    if constexpr (KEYS == kByLogit) {
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = live[v] && allowed[v] ? order(z[v]) : kNone;
    } else {
      const float inv = fast_rcp(total);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const bool ok = live[v] && allowed[v];
        const float s = (soft ? fast_exp(z[v] - zmax) * inv : fast_sigmoid(z[v])) * prior[v];
        key[v] = ok ? order(s + bias[v]) : kNone;
        mag = fmaxf(mag, ok ? s + fabsf(bias[v]) : 0.0f);
      }
      mag = seg_fmax<W>(mag);
    }
    const float tol = kKeyTol * mag;
    bool close = GROUPS == kOtherGroups;
    if constexpr (GROUPS == kLaneGroups || GROUPS == kOddGroups) {
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
      int ahead = 0;
      for (int g = 0; g < a.n_group; ++g) {
        uint32_t o;
        if constexpr (W == 64) o = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(lead), g * glanes));
        else o = __shfl(lead, seg * W + g * glanes, kWave);
        ahead += o > lead || (o == lead && g < own) ? 1 : 0;
      }
      const bool kept = ahead < a.topk_group && own < a.n_group;
      if constexpr (KEYS == kByKey) {   // the last group kept and the first one left out
        const float in = number(~seg_max<W>(kept ? ~lead : 0u)), out = number(seg_max<W>(kept ? kNone : lead));
        close |= in - out < 2.0f * tol;   // no group left out, or none with an expert: NaN, not close
      }
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = kept ? key[v] : kNone;
    }
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
        const int x = id[j];
        key[j] = sw ? key[j + 1] : k;
        key[j + 1] = sw ? k : key[j + 1];
        id[j] = sw ? id[j + 1] : x;
        id[j + 1] = sw ? x : id[j + 1];
      }
    uint32_t m = seg_max<W>(key[0]);
    for (int r = 0; r < a.K; ++r) {
      bool mine;
      if constexpr (W == 64) {
        mine = lane == __ffsll(static_cast<unsigned long long>(__ballot(key[0] == m))) - 1;
      } else {
        const uint64_t at = __ballot(key[0] == m);
        const uint32_t half = static_cast<uint32_t>(lane < 32 ? at : at >> 32) >> (W == 16 ? lane & 16 : 0);
        mine = key[0] == m && (half & below) == 0;
      }
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
    // lane r of the first 16 holds the r-th selected expert (K <= 16 <= W)
    int e = -1;
    uint32_t ke = kNone;
    if (sl < a.K) {
      const uint2 x = sel[slot][sl];
      e = static_cast<int>(x.x);
      ke = x.y;
    }
    if constexpr (EXACT) {
      if constexpr (KEYS == kByKey) {   // m: the best key left out
        uint32_t after = dpp<0x101>(ke);   // the next lane's (row_shl:1)
        after = sl == a.K - 1 ? m : after;
        close |= sl < a.K && number(ke) - number(after) < tol;   // kNone: NaN, not close
      }
      if (__any(close)) {
        select_exact<W>(a, a.logits + static_cast<size_t>(t) * a.E, sl, KEYS == kByKey, rows[slot],
                        leads[GROUPS != kNoGroups ? slot : 0], exact_sel[slot]);
        if (sl < a.K) e = exact_sel[slot][sl];
      }
    }
    lds_order();
    const bool has = e >= 0;
    const float zs = has ? clamp_logit(a.logits[static_cast<size_t>(t) * a.E + e]) : ninf;
    float g;
    if (a.renorm) {
      // ratios of scores, from logits relative to the largest selected one: exp(z_k - z_max) for
      // softmax, and for sigmoid where every score is e^z to fp32's precision; no score underflows
      const float top = seg_fmax<16>(fmaxf(zs, -FLT_MAX));
      const float w = !has ? 0.0f : soft || top < -30.0f ? fast_exp(zs - top) : fast_sigmoid(zs);
      g = a.scale * (w / seg_sum<16>(w));
    } else {
      g = a.scale * (soft ? fast_exp(zs - zmax) / total : fast_sigmoid(zs));
    }
    if (real && sl < a.K) {
      a.idx[static_cast<size_t>(t) * a.K + sl] = e;
      a.gate[static_cast<size_t>(t) * a.K + sl] = has ? g : 0.0f;
      if (a.load && has) atomicAdd(&hist[e], 1);   // integer counts: order-independent
    }
  }
  if (a.load) {
    __syncthreads();
    for (int e = tid; e < a.E; e += kThreads) {
      if (gridDim.x == 1) a.load[e] = hist[e];
      else if (hist[e]) atomicAdd(&a.load[e], hist[e]);
    }
  }
}

__global__ void gate_zero_kernel(int32_t* load, int E) {
  if (static_cast<int>(threadIdx.x) < E) load[threadIdx.x] = 0;
}

template <int W, int V, bool VEC, int KEYS>
void launch_groups(const GateArgs& a, dim3 grid, hipStream_t stream) {
  const int n = a.E / a.n_group, lanes = n / V;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a); };
  if (a.n_group == 1 || a.topk_group == a.n_group) go(gate_kernel<W, V, VEC, KEYS, kNoGroups>);
  else if (n % V != 0) go(gate_kernel<W, V, VEC, KEYS, kOtherGroups>);
  else if ((lanes & (lanes - 1)) == 0) go(gate_kernel<W, V, VEC, KEYS, kLaneGroups>);
  else go(gate_kernel<W, V, VEC, KEYS, kOddGroups>);
}

template <int W, int V>
hipError_t launch_gate(const GateArgs& a, hipStream_t stream) {
  constexpr int PER = kWave / W * kWaves;
  if (a.T == 0 && !a.load) return hipSuccess;
  const int blocks = std::max(1, std::min((a.T + PER - 1) / PER, 256 * 8));
  if (a.load && (blocks > 1 || a.T == 0)) {
    hipLaunchKernelGGL(gate_zero_kernel, dim3(1), dim3(kGateMaxE), 0, stream, a.load, a.E);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess || a.T == 0) return err;
  }
  const bool by_key = a.bias || a.has_prior || (a.n_group > 1 && a.group_rule == 1);
  const bool vec = V == 4 && a.E % 4 == 0 && (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0;
  constexpr bool VEC = V == 4;
  if (vec && by_key) launch_groups<W, V, VEC, kByKey>(a, dim3(blocks), stream);
  else if (vec) launch_groups<W, V, VEC, kByLogit>(a, dim3(blocks), stream);
  else if (by_key) launch_groups<W, V, false, kByKey>(a, dim3(blocks), stream);
  else launch_groups<W, V, false, kByLogit>(a, dim3(blocks), stream);
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
      float w = !has ? 0.0f : soft || top < -30.0f ? fast_exp(x.zs - top) : fast_sigmoid(x.zs);
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
  if (a.E <= 16) return launch_gate<16, 1>(a, stream);
  if (a.E <= 64) return launch_gate<16, 4>(a, stream);
  if (a.E <= 128) return launch_gate<32, 4>(a, stream);
  return launch_gate<64, 4>(a, stream);
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
