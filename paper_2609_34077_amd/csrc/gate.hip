// Routing by scores, balance bias and expert groups (include/maskmoe.h, maskmoe_gate_forward), and
// the gradient of its gates.
//
// A token takes a segment of W lanes (16, 32 or 64), each of which holds V consecutive experts in
// registers, so that a row of logits is read once, in order, and lower lanes hold lower experts:
//   scores    softmax or sigmoid of the registers, row maximum and sum by lane exchanges;
//   groups    the two largest keys of a group by lane exchanges where a group is a power of two of
//             lanes, else from the row in LDS; a group stays if fewer than topk_group groups beat it;
//   top-K     every lane sorts its V keys; each round takes the largest first key of the segment and
//             the lowest lane that holds it, which drops it: about 18 instructions a round.
// Selection goes by real numbers: keys are compared in fp32, and where two keys that the result
// depends on come closer than fp32 can tell apart (a bound on its errors, below), the wavefront
// selects again with keys in fp64. Without bias, prior and group sums the keys are the logits, which
// order as their scores do and need neither.

#include <float.h>

#include <algorithm>

#include "common.hpp"
#include "gate.hpp"

namespace maskmoe {
namespace {

constexpr int kThreads = 256;

// v of the lane that DPP control CTRL names: 0xB1 / 0x4E exchange lanes 1 / 2 apart, 0x141 / 0x140
// mirror 8 / 16 lanes, which exchanges their halves where the lanes of each half agree.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true); }
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  return __hiloint2double(dpp<CTRL>(__double2hiint(v)), dpp<CTRL>(__double2loint(v)));
}

// v of the lane S lanes away (S = 1, 2 as exchanges, 4 and 8 mirrored, 16 and 32 as exchanges).
template <int S, typename T>
__device__ __forceinline__ T from(T v) {
  if constexpr (S == 1) return dpp<0xB1>(v);
  else if constexpr (S == 2) return dpp<0x4E>(v);
  else if constexpr (S == 4) return dpp<0x141>(v);
  else if constexpr (S == 8) return dpp<0x140>(v);
  else return __shfl_xor(v, S, kWave);
}

__device__ __forceinline__ float vmax(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double vmax(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ float vmin(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ double vmin(double a, double b) { return fmin(a, b); }

// Largest value and sum over the W lanes of a segment, in every lane.
template <int W, int S = 1, typename T>
__device__ __forceinline__ T seg_max(T v) {
  if constexpr (S < W) return seg_max<W, 2 * S>(vmax(v, from<S>(v)));
  else return v;
}
template <int W, int S = 1, typename T>
__device__ __forceinline__ T seg_sum(T v) {
  if constexpr (S < W) return seg_sum<W, 2 * S>(v + from<S>(v));
  else return v;
}

__device__ __forceinline__ void lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

__device__ __forceinline__ float score_exp(float v) { return expf(v); }
__device__ __forceinline__ double score_exp(double v) { return exp(v); }

// +inf counts as the largest finite logit; NaN and -inf leave the row (see live below).
__device__ __forceinline__ float clamp_logit(float z) { return fminf(z, FLT_MAX); }

// The two largest of the keys of S-lane-aligned lane sets, in every lane of the set.
template <int LANES, typename T>
__device__ __forceinline__ void top2_lanes(T& t1, T& t2, int lanes) {
  auto step = [&](T b1, T b2) {
    t2 = vmax(vmin(t1, b1), vmax(t2, b2));
    t1 = vmax(t1, b1);
  };
  if (LANES > 1 && lanes > 1) { const T b1 = from<1>(t1), b2 = from<1>(t2); step(b1, b2); }
  if (LANES > 2 && lanes > 2) { const T b1 = from<2>(t1), b2 = from<2>(t2); step(b1, b2); }
  if (LANES > 4 && lanes > 4) { const T b1 = from<4>(t1), b2 = from<4>(t2); step(b1, b2); }
  if (LANES > 8 && lanes > 8) { const T b1 = from<8>(t1), b2 = from<8>(t2); step(b1, b2); }
  if (LANES > 16 && lanes > 16) { const T b1 = from<16>(t1), b2 = from<16>(t2); step(b1, b2); }
  if (LANES > 32 && lanes > 32) { const T b1 = from<32>(t1), b2 = from<32>(t2); step(b1, b2); }
}

// Groups, then top-K of one segment's keys; `out` (LDS, K entries of the segment) receives the
// selected experts, -1 where none is left. Keys of ineligible experts are -inf on entry. row: LDS for E
// keys of the segment. tol: how close two keys may come in type T before they count as too close.
template <int W, int V, typename T>
__device__ __forceinline__ bool select(const GateArgs& a, T (&key)[V], int seg, int sl, T* row, int* out, T tol) {
  const T ninf = -static_cast<T>(INFINITY);
  const int e0 = sl * V;
  bool close = false;
  if (a.n_group > 1) {
    const int n = a.E / a.n_group;
    const bool sum2 = a.group_rule == 1;
    const int lanes = n / V;
    if (n % V == 0 && (lanes & (lanes - 1)) == 0) {
      T t1 = ninf, t2 = ninf;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        t2 = vmax(t2, vmin(t1, key[v]));
        t1 = vmax(t1, key[v]);
      }
      top2_lanes<W>(t1, t2, lanes);
      const T lead = sum2 && t2 > ninf ? t1 + t2 : t1;
      const int own = e0 / n;
      int ahead = 0;
      for (int g = 0; g < a.n_group; ++g) {
        const T o = __shfl(lead, seg * W + g * lanes, kWave);
        ahead += o > lead || (o == lead && g < own) ? 1 : 0;
        close |= g != own && own < a.n_group && fabs(o - lead) < 2 * tol;
      }
      if (ahead >= a.topk_group) {
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = ninf;
      }
    } else {   // any other group size: lane g looks at the keys of group g (and g + W, ...) in LDS
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (e0 + v < a.E) row[e0 + v] = key[v];
      lds_order();
      // every lane ranks the groups of its own experts; a group's lead is recomputed where needed
      auto lead_of = [&](int g) {
        T t1 = ninf, t2 = ninf;
        for (int i = 0; i < n; ++i) {
          const T k = row[g * n + i];
          t2 = vmax(t2, vmin(t1, k));
          t1 = vmax(t1, k);
        }
        return sum2 && t2 > ninf ? t1 + t2 : t1;
      };
      T lead[V];
      int ahead[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        lead[v] = e0 + v < a.E ? lead_of((e0 + v) / n) : ninf;
        ahead[v] = 0;
      }
      for (int g = 0; g < a.n_group; ++g) {
        const T o = lead_of(g);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int own = (e0 + v) / n;
          if (e0 + v >= a.E) continue;
          ahead[v] += o > lead[v] || (o == lead[v] && g < own) ? 1 : 0;
          close |= g != own && fabs(o - lead[v]) < 2 * tol;
        }
      }
      lds_order();
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (ahead[v] >= a.topk_group) key[v] = ninf;
    }
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
      const T k = key[j];
      const int x = id[j];
      key[j] = sw ? key[j + 1] : k;
      key[j + 1] = sw ? k : key[j + 1];
      id[j] = sw ? id[j + 1] : x;
      id[j + 1] = sw ? x : id[j + 1];
    }
  const uint64_t segbits = (W == 64 ? ~0ull : (1ull << W) - 1) << (seg * W);
  T last = static_cast<T>(INFINITY);
  const int rounds = min(a.K + 1, a.E);   // one more than K: the best key left out
  for (int r = 0; r < rounds; ++r) {
    const T m = seg_max<W>(key[0]);
    close |= last - m < tol;   // -inf - -inf is NaN: none
    last = m;
    if (r == a.K) break;
    const uint64_t at = __ballot(key[0] == m && m > ninf) & segbits;
    const int first = __ffsll(static_cast<unsigned long long>(at)) - 1;
    const bool mine = first == seg * W + sl;
    if (mine) out[r] = id[0];
    if (at == 0 && sl == 0) out[r] = -1;
#pragma unroll
    for (int v = 0; v + 1 < V; ++v) {
      key[v] = mine ? key[v + 1] : key[v];
      id[v] = mine ? id[v + 1] : id[v];
    }
    if (mine) key[V - 1] = ninf;
  }
  return close;
}

// Errors of an fp32 key, relative to the largest s * prior + |bias| of the row: expf and the
// difference it is taken of 2 half-steps, a row sum of up to 256 terms 8, the division, product and sum
// 3: under 1e-6 in all. Two keys are told apart at 2.5e-6, two group sums of two keys at twice that;
// with a margin:
constexpr float kKeyTol = 4e-6f;

template <int W, int V, bool VEC>
__global__ __launch_bounds__(kThreads) void gate_kernel(const GateArgs a) {
  constexpr int SEGS = kWave / W;                // tokens per wavefront
  constexpr int PER = SEGS * (kThreads / kWave);   // tokens per workgroup and round
  __shared__ int sel[PER][kGateMaxK];
  __shared__ double rows[PER][W * V];
  __shared__ int hist[kGateMaxE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seg = lane / W, sl = lane % W, e0 = sl * V;
  const int slot = wave * SEGS + seg;
  if (a.load) {
    for (int e = tid; e < a.E; e += kThreads) hist[e] = 0;
    __syncthreads();
  }
  const bool by_logit = !a.bias && !a.has_prior && !(a.n_group > 1 && a.group_rule == 1);
  float bias[V], prior[V];
  bool allowed[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = e0 + v;
    const bool in = e < a.E;
    bias[v] = in && a.bias ? a.bias[e] : 0.0f;
    prior[v] = in && a.has_prior ? a.prior[e] : 1.0f;
    allowed[v] = in && (!a.has_mask || (a.mask[e >> 5] >> (e & 31) & 1));
  }
  const float ninf = -INFINITY;
  for (int t0 = blockIdx.x * PER; t0 < a.T; t0 += gridDim.x * PER) {
    const int t = min(t0 + slot, a.T - 1);   // segments past the last token repeat it, unwritten
    const bool real = t0 + slot < a.T;
    const float* zr = a.logits + static_cast<size_t>(t) * a.E;
    float z[V];
    if constexpr (VEC && V == 4) {
      f32x4 q = {ninf, ninf, ninf, ninf};
      if (e0 < a.E) q = *reinterpret_cast<const f32x4*>(zr + e0);
#pragma unroll
      for (int v = 0; v < V; ++v) z[v] = q[v];
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) z[v] = e0 + v < a.E ? zr[e0 + v] : ninf;
    }
    bool live[V];
    float zmax = ninf;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      live[v] = z[v] > ninf;   // false for NaN too
      z[v] = live[v] ? clamp_logit(z[v]) : ninf;
      zmax = fmaxf(zmax, z[v]);
    }
    const bool soft = a.score == 0;
    float total = 1.0f;
    if (soft) {
      zmax = seg_max<W>(zmax);
      total = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) total += live[v] ? expf(z[v] - zmax) : 0.0f;
      total = seg_sum<W>(total);
    }
    float key[V];
    bool close = false;
    if (by_logit) {
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = live[v] && allowed[v] ? z[v] : ninf;
      select<W, V, float>(a, key, seg, sl, reinterpret_cast<float*>(rows[slot]), sel[slot], 0.0f);
    } else {
      float mag = 0.0f;
      const float inv = 1.0f / total;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const bool ok = live[v] && allowed[v];
        const float s = soft ? expf(z[v] - zmax) * inv : 1.0f / (1.0f + expf(-z[v]));
        key[v] = ok ? s * prior[v] + bias[v] : ninf;
        mag = fmaxf(mag, ok ? s * prior[v] + fabsf(bias[v]) : 0.0f);
      }
      close = select<W, V, float>(a, key, seg, sl, reinterpret_cast<float*>(rows[slot]), sel[slot],
                                  kKeyTol * seg_max<W>(mag));
      if (__any(close)) {
        double k64[V], sum = 0.0;
        if (soft) {
#pragma unroll
          for (int v = 0; v < V; ++v) sum += live[v] ? exp(static_cast<double>(z[v]) - zmax) : 0.0;
          sum = seg_sum<W>(sum);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const double s = soft ? exp(static_cast<double>(z[v]) - zmax) / sum : 1.0 / (1.0 + exp(-static_cast<double>(z[v])));
          k64[v] = live[v] && allowed[v] ? s * prior[v] + bias[v] : -INFINITY;
        }
        lds_order();
        select<W, V, double>(a, k64, seg, sl, rows[slot], sel[slot], 0.0);
      }
    }
    lds_order();
    // gates: lane r holds the r-th selected expert (K <= 16 <= W, so one 16-lane row holds them all)
    const int e = sl < a.K ? sel[slot][sl] : -1;
    lds_order();
    const bool has = e >= 0;
    const float zs = has ? clamp_logit(zr[e]) : ninf;
    float g;
    if (a.renorm) {
      // ratios of scores, from logits relative to the largest selected one: exp(z_k - z_max) for
      // softmax, and for sigmoid where every score is e^z to fp32's precision; no score underflows
      const float top = seg_max<16>(zs);
      float w = 0.0f;
      if (has) w = soft || top < -30.0f ? expf(zs - top) : 1.0f / (1.0f + expf(-zs));
      const float s = seg_sum<16>(w);
      g = has ? a.scale * (w / s) : 0.0f;
    } else {
      g = !has ? 0.0f : a.scale * (soft ? expf(zs - zmax) / total : 1.0f / (1.0f + expf(-zs)));
    }
    if (real && sl < a.K) {
      a.idx[static_cast<size_t>(t) * a.K + sl] = e;
      a.gate[static_cast<size_t>(t) * a.K + sl] = g;
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

template <int W, int V>
hipError_t launch_gate(const GateArgs& a, hipStream_t stream) {
  constexpr int PER = kWave / W * (kThreads / kWave);
  if (a.T == 0 && !a.load) return hipSuccess;
  const int blocks = std::max(1, std::min((a.T + PER - 1) / PER, 256 * 8));
  if (a.load && blocks > 1) {
    hipLaunchKernelGGL(gate_zero_kernel, dim3(1), dim3(kGateMaxE), 0, stream, a.load, a.E);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  const bool vec = V == 4 && a.E % 4 == 0 && (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0;
  if (vec) hipLaunchKernelGGL((gate_kernel<W, V, true>), dim3(blocks), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((gate_kernel<W, V, false>), dim3(blocks), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

// dL/dz of the gates (include/maskmoe.h, maskmoe_gate_backward). A segment of W lanes per token as
// above; lane r < K holds entry r, and every lane adds the entries that name its experts, in order of r.
template <int W, int V>
__global__ __launch_bounds__(kThreads) void gate_bwd_kernel(const GateBwdArgs a) {
  constexpr int SEGS = kWave / W, PER = SEGS * (kThreads / kWave);
  __shared__ int se[PER][kGateMaxK];
  __shared__ float sd[PER][kGateMaxK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seg = lane / W, sl = lane % W, e0 = sl * V;
  const int slot = wave * SEGS + seg;
  const bool soft = a.score == 0;
  const bool dense = soft && !a.renorm;
  const float ninf = -INFINITY;
  for (int t0 = blockIdx.x * PER; t0 < a.T; t0 += gridDim.x * PER) {
    const int t = min(t0 + slot, a.T - 1);
    const bool real = t0 + slot < a.T;
    const float* zr = a.logits + static_cast<size_t>(t) * a.E;
    int e = -1;
    float dg = 0.0f;
    if (sl < a.K) {
      e = a.idx[static_cast<size_t>(t) * a.K + sl];
      dg = a.d_gate[static_cast<size_t>(t) * a.K + sl];
    }
    if (e >= a.E) e = -1;
    float zs = e >= 0 ? zr[e] : ninf;
    const bool has = zs > ninf;
    if (!has) { e = -1; dg = 0.0f; }
    zs = has ? clamp_logit(zs) : ninf;
    dg *= a.scale;
    float z[V], zmax = ninf, total = 1.0f;
    if (dense) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        z[v] = e0 + v < a.E ? zr[e0 + v] : ninf;
        z[v] = z[v] > ninf ? clamp_logit(z[v]) : ninf;
        zmax = fmaxf(zmax, z[v]);
      }
      zmax = seg_max<W>(zmax);
      total = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        z[v] = z[v] > ninf ? expf(z[v] - zmax) : 0.0f;
        total += z[v];
      }
      total = seg_sum<W>(total);
    }
    float d = 0.0f, pd = 0.0f;   // the entry's own term; dense: <p, dp>
    if (dense) {
      d = has ? dg : 0.0f;
      pd = seg_sum<16>(has ? dg * (expf(zs - zmax) / total) : 0.0f);
      pd = __shfl(pd, seg * W, kWave);   // rows other than the first hold no entries
    } else if (a.renorm) {
      const float top = seg_max<16>(zs);
      float w = 0.0f;
      if (has) w = soft || top < -30.0f ? expf(zs - top) : 1.0f / (1.0f + expf(-zs));
      const float s = seg_sum<16>(w);
      w = has ? w / s : 0.0f;
      const float mean = seg_sum<16>(w * dg);
      d = has ? w * (dg - mean) * (soft ? 1.0f : 1.0f / (1.0f + expf(zs))) : 0.0f;
    } else {   // s (1 - s), the second factor as the sigmoid of -z
      d = has ? dg / (1.0f + expf(-zs)) / (1.0f + expf(zs)) : 0.0f;
    }
    if (sl < a.K) {
      se[slot][sl] = e;
      sd[slot][sl] = d;
    }
    lds_order();
    float out[V];
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = 0.0f;
    for (int r = 0; r < a.K; ++r) {
      const int er = se[slot][r];
      const float dr = sd[slot][r];
#pragma unroll
      for (int v = 0; v < V; ++v) out[v] += er == e0 + v ? dr : 0.0f;
    }
    lds_order();
    if (dense) {
#pragma unroll
      for (int v = 0; v < V; ++v) out[v] = z[v] / total * (out[v] - pd);
    }
    if (real) {
      float* o = a.d_logits + static_cast<size_t>(t) * a.E;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (e0 + v < a.E) o[e0 + v] = out[v];
    }
  }
}

template <int W, int V>
hipError_t launch_gate_bwd(const GateBwdArgs& a, hipStream_t stream) {
  constexpr int PER = kWave / W * (kThreads / kWave);
  const int blocks = std::min((a.T + PER - 1) / PER, 256 * 16);
  hipLaunchKernelGGL((gate_bwd_kernel<W, V>), dim3(blocks), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gate_forward(const GateArgs& a, hipStream_t stream) {
  if (a.E <= 16) return launch_gate<16, 1>(a, stream);
  if (a.E <= 64) return launch_gate<16, 4>(a, stream);
  if (a.E <= 128) return launch_gate<32, 4>(a, stream);
  return launch_gate<64, 4>(a, stream);
}

hipError_t launch_gate_backward(const GateBwdArgs& a, hipStream_t stream) {
  if (a.E <= 16) return launch_gate_bwd<16, 1>(a, stream);
  if (a.E <= 64) return launch_gate_bwd<16, 4>(a, stream);
  if (a.E <= 128) return launch_gate_bwd<32, 4>(a, stream);
  return launch_gate_bwd<64, 4>(a, stream);
}

}  // namespace maskmoe
