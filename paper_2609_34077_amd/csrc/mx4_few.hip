// Both products of experts on MX4 weights for up to 16 tokens: the time is the stream of the selected experts'
// weights, and every launch besides counts. Three launches; the first two read the routing themselves:
//   up    a workgroup per 32 columns of h of one selected expert; four wavefronts split the reduction;
//   down  a workgroup per 64 columns of y and one of `splits` parts of the reductions of all selected experts, laid end
//         to end: each expert's sum is weighed by the tokens' gates and added, so that y comes out;
//   sum   of the parts, in order.
// A wavefront multiplies 64 weight rows at a time, so that the tokens' operand, which takes as many registers as
// theirs, is used four times. It keeps no ring of steps: in 56 to 84 registers all of a small launch's wavefronts are on
// the chip at once, each with one step's loads in flight (Mixtral-shaped layer, one token: 896 and 1024 workgroups, 3.5 and 4
// wavefronts a SIMD, up / down 25.3 / 14.3 us; with rings of two steps in 156 registers 27.0 / 17.1, and rings of one, whose
// registers the compiler keeps apart, 26.4 / 16.1).
// Tokens are the 16 columns of the matrix instructions as they are; a token that an expert is not selected for
// loads nothing there. Weights go from memory straight to registers, 1 KiB of 16 rows x 128 columns a load.

#include "common.hpp"
#include "mx4.hpp"
#include "mx4_block.hpp"

#include <algorithm>

namespace maskmoe {
namespace {

constexpr int kMaxExperts = 256, kMaxSlots = 256 + 8;
constexpr int kThreads = 256;

// An offset past every buffer (fewer than 2^31 bf16 values of whole 128-byte pieces), with room for the 48 bytes that
// are added to it: reads as zeros, without a branch.
constexpr uint32_t kNowhere = 0xffffffc0u;
constexpr int kNt = 2;                       // the load's non-temporal bit: weights that one workgroup reads once

// The selected experts as bits, and the entries themselves (T * K <= 256), in LDS.
struct Routing {
  uint32_t bits[kMaxExperts / 32];
  int idx[kMx4FewT * 16];
  float gate[kMx4FewT * 16];
};
__device__ __forceinline__ void read_routing(const Mx4Args& a, Routing& r, bool gates) {
  const int tid = threadIdx.x, n = a.T * a.K;
  int e = -1;
  float g = 0.0f;
  if (tid < n) {
    e = a.idx[tid];
    if (gates) g = a.gate[tid];
  }
  if (tid < kMaxExperts / 32) r.bits[tid] = 0;
  lds_sync();
  if (tid < n) {
    if (e < 0 || e >= a.E) e = -1;
    r.idx[tid] = e;
    r.gate[tid] = g;
    if (e >= 0) atomicOr(&r.bits[e >> 5], 1u << (e & 31));
  }
  lds_sync();
}
// Selected experts; with `want` the want-th of them in increasing order (-1 if there are fewer).
__device__ __forceinline__ int selected(const Routing& r, int want, int& count) {
  int found = -1;
  count = 0;
#pragma unroll
  for (int w = 0; w < kMaxExperts / 32; ++w) {
    uint32_t b = __builtin_amdgcn_readfirstlane(r.bits[w]);
    const int c = __popc(b);
    if (want >= count && want < count + c) {
      for (int i = count; i < want; ++i) b &= b - 1;
      found = 32 * w + __ffs(b) - 1;
    }
    count += c;
  }
  return found;
}

template <bool MX>
__global__ __launch_bounds__(kThreads, 4) void mx4_few_up_kernel(const Mx4Params p) {
  __shared__ Routing rt;
  __shared__ f32x4 red[4][4][kWave];
  const Mx4Args& a = p.a;
  const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int cols = a.F / 32, slot = blockIdx.x / cols, cx = blockIdx.x % cols, KS = a.K + a.n_shared;
  read_routing(a, rt, false);
  int n_sel;
  int g = selected(rt, slot, n_sel);
  if (slot >= n_sel + a.n_shared) return;
  int row = -1;   // of h: the token's first entry that names the expert
  if (slot >= n_sel) {
    g = a.E + slot - n_sel;
    if (l16 < a.T) row = l16 * KS + a.K + slot - n_sel;
  } else if (l16 < a.T) {
    for (int k = a.K - 1; k >= 0; --k)
      if (rt.idx[l16 * a.K + k] == g) row = l16 * KS + k;
  }
  const int C = a.d, R = 2 * a.F;
  const int steps = mx4_steps(C), quads = mx4_quads(C), blocks = C / kMxBlock;
  const __amdgpu_buffer_rsrc_t codes = make_rsrc(a.gu_codes + (static_cast<size_t>(g) * (R / 16) + 4 * cx) * steps * 1024,
                                                 4 * steps * 1024);
  const __amdgpu_buffer_rsrc_t scales = make_rsrc(a.gu_scales + (static_cast<size_t>(g) * (R / 16) + 4 * cx) * quads * 256,
                                                  4 * quads * 256);
  const __amdgpu_buffer_rsrc_t x = make_rsrc(a.x, static_cast<uint32_t>(a.T) * C * 2);
  const uint32_t xoff = row < 0 ? kNowhere : static_cast<uint32_t>(l16) * C * 2 + 64 * lg;
  f32x4 acc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = f32x4{0, 0, 0, 0};
  const int s0 = steps * wave / 4, s1 = steps * (wave + 1) / 4;
  struct Step {
    u32x4 w[4], b[4];
    uint32_t ws[4];
  };
  auto load = [&](int s, Step& q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q.w[i] = __builtin_amdgcn_raw_buffer_load_b128(codes, lane * 16, (i * steps + s) * 1024, kNt);
      q.ws[i] = __builtin_amdgcn_raw_buffer_load_b32(scales, lane * 4, (i * quads + (s >> 2)) * 256, 0);
    }
    const uint32_t off = 4 * s + lg < blocks ? xoff : kNowhere;
#pragma unroll
    for (int j = 0; j < 4; ++j) q.b[j] = __builtin_amdgcn_raw_buffer_load_b128(x, off + 16 * j, kMxStep * 2 * s, 0);
  };
  auto multiply = [&](int s, const Step& q) {
    const int sh = 8 * (s & 3);
    if constexpr (MX) {
      u32x4 c;
      const uint32_t bs = mx4_block_codes(q.b, c);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = mfma_mx4(q.w[i], c, acc[i], q.ws[i] >> sh, bs);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float sc = mx4_scale(q.ws[i] >> sh & 255);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i] = mfma_16x16x32(mx4_to_bf16(q.w[i][j], sc), q.b[j], acc[i]);
      }
    }
  };
  for (int s = s0; s < s1; ++s) {
    Step q;
    load(s, q);
    multiply(s, q);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) red[wave][i][lane] = acc[i];
  lds_sync();
  if (wave != 0) return;
  f32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = red[0][i][lane] + red[1][i][lane] + red[2][i][lane] + red[3][i][lane];
  // lane: rows 4 lg + i of both 16-row halves of the 32, one token
  float h[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = silu(v[0][i]) * v[1][i];
    h[4 + i] = silu(v[2][i]) * v[3][i];
  }
  if constexpr (MX) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(h[i]) & 0x7fffffffu);
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16, kWave)));
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32, kWave)));
    const uint32_t byte = mx4_scale_byte(m);
    const uint32_t c = byte == 255 ? 0 : mx4_codes(h, mx4_scale(byte));
    if (row >= 0) {
      uint16_t* q = reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(p.h) + static_cast<size_t>(row) * (a.F / 2) + 16 * cx + 2 * lg);
      q[0] = static_cast<uint16_t>(c);
      q[4] = static_cast<uint16_t>(c >> 16);
      if (lg == 0) p.hs[static_cast<size_t>(row) * 16 * mx4_quads(a.F) + mx4_scale_at(cx)] = static_cast<uint8_t>(byte);
    }
  } else if (row >= 0) {
    uint2* q = reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.h) + static_cast<size_t>(row) * a.F + 32 * cx + 4 * lg);
    q[0] = make_uint2(f32x2_to_bf16x2(h[0], h[1]), f32x2_to_bf16x2(h[2], h[3]));
    q[4] = make_uint2(f32x2_to_bf16x2(h[4], h[5]), f32x2_to_bf16x2(h[6], h[7]));
  }
}

template <bool MX>
__global__ __launch_bounds__(kThreads, 4) void mx4_few_down_kernel(const Mx4Params p, int splits, int max_slots) {
  __shared__ Routing rt;
  __shared__ uint16_t expert[kMaxSlots];
  __shared__ uint16_t slot_of[kMaxExperts];
  __shared__ f32x4 red[4][4][kWave];
  // for each of max_slots slots and a token: the gate (the sum over the token's entries that name the expert) and the row
  // of h, -1 where none does. As large as the launch needs, so that four workgroups fit a CU.
  extern __shared__ float tables[];
  float(*gates)[kMx4FewT] = reinterpret_cast<float(*)[kMx4FewT]>(tables);
  int16_t(*hrow)[kMx4FewT] = reinterpret_cast<int16_t(*)[kMx4FewT]>(tables + max_slots * kMx4FewT);
  const Mx4Args& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int KS = a.K + a.n_shared;
  const int cx = blockIdx.x / splits, split = blockIdx.x % splits;
  read_routing(a, rt, true);
  int n_sel = 0;
#pragma unroll
  for (int w = 0; w < kMaxExperts / 32; ++w) {
    const uint32_t b = rt.bits[w];
    if (tid >> 5 == w && (b >> (tid & 31) & 1)) {
      const int s = n_sel + __popc(b & ((1u << (tid & 31)) - 1));
      slot_of[tid] = static_cast<uint16_t>(s);
      expert[s] = static_cast<uint16_t>(tid);
    }
    n_sel += __popc(b);
  }
  const int slots = n_sel + a.n_shared;
  if (tid < a.n_shared) expert[n_sel + tid] = static_cast<uint16_t>(a.E + tid);
  for (int i = tid; i < slots * kMx4FewT; i += kThreads) {
    const int s = i / kMx4FewT, t = i % kMx4FewT;
    const bool shared = s >= n_sel && t < a.T;
    gates[s][t] = shared ? 1.0f : 0.0f;
    hrow[s][t] = static_cast<int16_t>(shared ? t * KS + a.K + s - n_sel : -1);
  }
  lds_sync();
  if (tid < a.T)
    for (int k = a.K - 1; k >= 0; --k) {
      const int e = rt.idx[tid * a.K + k];
      if (e < 0) continue;
      gates[slot_of[e]][tid] += rt.gate[tid * a.K + k];
      hrow[slot_of[e]][tid] = static_cast<int16_t>(tid * KS + k);
    }
  lds_sync();
  const int C = a.F, R = a.d;
  const int steps = mx4_steps(C), quads = mx4_quads(C), blocks = C / kMxBlock;
  const uint32_t fbytes = static_cast<uint32_t>(steps) * 1024, fscales = static_cast<uint32_t>(quads) * 256;   // of a fragment
  const __amdgpu_buffer_rsrc_t h = make_rsrc(p.h, static_cast<uint32_t>(a.T * KS) * C * 2);
  const __amdgpu_buffer_rsrc_t hs = make_rsrc(p.hs, static_cast<uint32_t>(a.T * KS) * quads * 16);
  // unit: one step of one slot's expert; a wavefront takes consecutive ones (at most 264 x 2^22: F d < 2^30, d >= 64)
  const int units = slots * steps, share = split * 4 + wave, shares = splits * 4;
  const int u0 = static_cast<int>(static_cast<int64_t>(units) * share / shares);
  const int u1 = static_cast<int>(static_cast<int64_t>(units) * (share + 1) / shares);
  struct Place {
    int slot, step;
  };
  struct Unit {
    u32x4 w[4], b[4];
    uint32_t ws[4], bs;
    float gate;      // of the lane's token
    int row, step;   // row: -1 where it did not select the expert
  };
  f32x4 y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = f32x4{0, 0, 0, 0};
  auto load = [&](const Place& at, Unit& q) {
    const int s = at.step;
    const size_t f = static_cast<size_t>(__builtin_amdgcn_readfirstlane(expert[at.slot])) * (R / 16) + 4 * cx;
    const __amdgpu_buffer_rsrc_t codes = make_rsrc(a.dn_codes + f * fbytes, 4 * fbytes);
    const __amdgpu_buffer_rsrc_t scales = make_rsrc(a.dn_scales + f * fscales, 4 * fscales);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q.w[i] = __builtin_amdgcn_raw_buffer_load_b128(codes, lane * 16, i * fbytes + s * 1024, kNt);
      q.ws[i] = __builtin_amdgcn_raw_buffer_load_b32(scales, lane * 4, i * fscales + (s >> 2) * 256, 0);
    }
    q.step = s;
    q.row = hrow[at.slot][l16];
    q.gate = gates[at.slot][l16];
    const bool in = q.row >= 0 && 4 * s + lg < blocks;
    if constexpr (MX) {
      q.b[0] = __builtin_amdgcn_raw_buffer_load_b128(h, in ? static_cast<uint32_t>(q.row) * (C / 2) + 16 * lg : kNowhere, 64 * s, 0);
      q.bs = __builtin_amdgcn_raw_buffer_load_b32(hs, in ? static_cast<uint32_t>(q.row) * 16 * quads + 4 * lg : kNowhere, 16 * (s >> 2), 0);
    } else {
      const uint32_t off = in ? static_cast<uint32_t>(q.row) * (2 * C) + 64 * lg : kNowhere;
#pragma unroll
      for (int j = 0; j < 4; ++j) q.b[j] = __builtin_amdgcn_raw_buffer_load_b128(h, off + 16 * j, 256 * s, 0);
    }
  };
  auto multiply = [&](const Unit& q) {
    const int sh = 8 * (q.step & 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 acc = {0, 0, 0, 0};
      if constexpr (MX) {
        acc = mfma_mx4(q.w[i], q.b[0], acc, q.ws[i] >> sh, q.bs >> sh);
      } else {
        const float f = mx4_scale(q.ws[i] >> sh & 255);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = mfma_16x16x32(mx4_to_bf16(q.w[i][j], f), q.b[j], acc);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)   // a NaN weight of an expert that the token did not select stays out
        y[i][e] += q.row >= 0 ? q.gate * acc[e] : 0.0f;
    }
  };
  Place at{u0 / steps, u0 % steps};
  for (int u = u0; u < u1; ++u) {
    Unit q;
    load(at, q);
    multiply(q);
    const bool wrap = at.step + 1 == steps;
    at = Place{wrap ? at.slot + 1 : at.slot, wrap ? 0 : at.step + 1};
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) red[wave][i][lane] = y[i];
  lds_sync();
  // wave w joins fragment w
  const f32x4 v = red[0][wave][lane] + red[1][wave][lane] + red[2][wave][lane] + red[3][wave][lane];
  if (l16 < a.T)
    *reinterpret_cast<f32x4*>(p.o + (static_cast<size_t>(split) * a.T + l16) * a.d + 64 * cx + 16 * wave + 4 * lg) = v;
}

// y = the sum of the parts [splits, T, d] in order; four columns a thread.
__global__ __launch_bounds__(kWave) void mx4_few_sum_kernel(const Mx4Params p, int splits) {
  constexpr int U = 8;   // parts loaded together
  const int n = p.a.T * p.a.d / 4, i = blockIdx.x * kWave + threadIdx.x;
  if (i >= n) return;
  const f32x4* o = reinterpret_cast<const f32x4*>(p.o) + i;
  f32x4 s = {0, 0, 0, 0};
  for (int q = 0; q < splits; q += U) {   // splits is a multiple of U
    f32x4 v[U];
#pragma unroll
    for (int k = 0; k < U; ++k) v[k] = o[static_cast<size_t>(q + k) * n];
#pragma unroll
    for (int k = 0; k < U; ++k) s += v[k];
  }
  reinterpret_cast<uint2*>(p.a.y)[i] = make_uint2(f32x2_to_bf16x2(s[0], s[1]), f32x2_to_bf16x2(s[2], s[3]));
}

template <bool MX>
hipError_t launch(const Mx4Params& p, hipStream_t stream) {
  const Mx4Args& a = p.a;
  const int slots = std::min(a.T * a.K, a.E) + a.n_shared;
  hipLaunchKernelGGL(mx4_few_up_kernel<MX>, dim3(slots * (a.F / 32)), dim3(kThreads), 0, stream, p);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const int splits = mx4_few_splits(a.d);
  hipLaunchKernelGGL(mx4_few_down_kernel<MX>, dim3(a.d / 64 * splits), dim3(kThreads), slots * kMx4FewT * 6, stream, p,
                     splits, slots);
  err = hipGetLastError();
  if (err != hipSuccess) return err;
  const int n = a.T * a.d / 4;
  hipLaunchKernelGGL(mx4_few_sum_kernel, dim3((n + kWave - 1) / kWave), dim3(kWave), 0, stream, p, splits);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_few(const Mx4Params& p, hipStream_t stream) {
  return p.a.mx_act ? launch<true>(p, stream) : launch<false>(p, stream);
}

}  // namespace maskmoe
