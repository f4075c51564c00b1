// The experts of a layer on MX4 weights (include/maskmoe.h, maskmoe_experts_forward_mx4):
//   y_t = sum_k g_k F_{A_t[k]}(x_t) + sum_s F_s(x_t),  F(x) = W_down h,  h = SiLU(W_gate x) * (W_up x),
// with W in packed MX4 blocks and x, h in bf16 or in MX4 blocks. Launches: prepare (routing entries of
// routed and shared experts, x to blocks), permutation, gate / up, down, combine.

#include <algorithm>

#include "mx4.hpp"
#include "mx4_block.hpp"

namespace maskmoe {
namespace {

constexpr int kThreads = 256;

// Entries of routed and shared experts in one list; x in blocks (four lanes a block).
__global__ __launch_bounds__(kThreads) void mx4_prepare_kernel(const Mx4Params p, int32_t* idx, float* gate,
                                                              int entry_blocks) {
  const Mx4Args& a = p.a;
  const int KS = a.K + a.n_shared;
  if (static_cast<int>(blockIdx.x) < entry_blocks) {
    const int j = blockIdx.x * kThreads + threadIdx.x;
    if (j >= a.T * KS) return;
    const int t = j / KS, k = j % KS;
    int e = a.E + k - a.K;
    float g = 1.0f;
    if (k < a.K) {
      e = a.idx[t * a.K + k];
      if (e < 0 || e >= a.E) e = -1;
      g = a.gate[t * a.K + k];
    }
    idx[j] = e;
    gate[j] = g;
    return;
  }
  const int64_t n = static_cast<int64_t>(a.T) * a.d / 8;
  const int64_t i = static_cast<int64_t>(blockIdx.x - entry_blocks) * kThreads + threadIdx.x;
  if (i >= n) return;
  const u32x4 q = reinterpret_cast<const u32x4*>(a.x)[i];
  float v[8];
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(q[j] << 16);
    v[2 * j + 1] = __uint_as_float(q[j] & 0xffff0000u);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
  m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0xB1, 0xF, 0xF, true)));
  m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0x4E, 0xF, 0xF, true)));
  const uint32_t byte = mx4_scale_byte(m);
  reinterpret_cast<uint32_t*>(p.xq)[i] = byte == 255 ? 0 : mx4_codes(v, mx4_scale(byte));
  if ((i & 3) == 0) {
    const int blocks = a.d / kMxBlock;
    const int64_t b = i >> 2, t = b / blocks;
    p.xs[t * 16 * mx4_quads(a.d) + mx4_scale_at(static_cast<int>(b - t * blocks))] = static_cast<uint8_t>(byte);
  }
}

// y = sum of the gate-weighted expert outputs (each the sum of its parts) in entry order, fp32, rounded once; a thread
// per four columns. Bound by their bytes, with the loads of U entries in flight (DeepSeek-shaped layer, 4096 tokens, 285 MB:
// 50 us). Outputs in bf16 took half the time there and 30 us off the down projection, but left an error of half a bf16
// step in every term of the sum: y was off by 2.3e-3 (relative, RMS) instead of the 1.7e-3 of its own rounding.
__global__ __launch_bounds__(kThreads) void mx4_combine_kernel(const Mx4Params p, int splits) {
  constexpr int U = 4;
  const Mx4Args& a = p.a;
  const int KS = a.K + a.n_shared, c4 = a.d / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= static_cast<int64_t>(a.T) * c4) return;
  const int t = static_cast<int>(i / c4), c = static_cast<int>(i % c4);
  const f32x4* src = reinterpret_cast<const f32x4*>(p.o) + c;
  const size_t part = static_cast<size_t>(a.T) * KS * c4;
  f32x4 s = {0, 0, 0, 0};
  for (int k0 = 0; k0 < KS; k0 += U) {
    bool live[U];
    float g[U];
    size_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = t * KS + min(k0 + u, KS - 1);
      live[u] = k0 + u < KS && static_cast<uint32_t>(p.idx[j]) < static_cast<uint32_t>(p.G);
      g[u] = p.gate[j];
      at[u] = static_cast<size_t>(p.pb.inv[j]) * c4;
    }
    f32x4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (live[u]) o[u] = src[at[u]];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!live[u]) continue;
      for (int z = 1; z < splits; ++z) o[u] += src[at[u] + z * part];
#pragma unroll
      for (int q = 0; q < 4; ++q) s[q] += g[u] * o[u][q];
    }
  }
  reinterpret_cast<uint2*>(a.y)[i] = make_uint2(f32x2_to_bf16x2(s[0], s[1]), f32x2_to_bf16x2(s[2], s[3]));
}

// Whether the wide tiles are taken: by the rows per expert from which they are faster, averaged over all experts, and
// their number, which must cover the chip (small layers: F 512, 8 experts, bf16, 1000 / 4000 tokens 42 / 48 us, batch tiles
// 28 / 40). Whole call, batch / wide, in us; "of half": the routing leaves out every other expert, as a hard mask does, so
// that the experts it reads have twice the average rows:
//   bf16: the batch tiles' weight stream hides the widening, which the wide ones pay with the products. Mixtral-shaped
//     400 tokens (100 rows an expert) 317 / 423, 1000 (250) 680 / 740, 1300 (325) 852 / 872, 1700 (425) 1079 / 992; of half
//     1000 tokens 642 / 679, 1300 829 / 801. DeepSeek-shaped 1600 (194 with the shared experts) 285 / 319, 2500 (303)
//     405 / 387, 3500 (424) 540 / 576; of half 1600 tokens 263 / 288, 2500 391 / 370.
//   MX4: Mixtral-shaped 64 tokens (16 rows) 150 / 156, 90 (22) 160 / 159, 128 (32) 181 / 163; of half 64 tokens 92 / 111,
//     90 103 / 115, 128 173 / 124. DeepSeek-shaped 100 (12) 87 / 81, 200 (24) 99 / 84; of half 100 65 / 55.
bool mx4_takes_wide(int rows, int G, int F, bool mx_act) {
  const int64_t tiles = (static_cast<int64_t>(rows) / mx4_tile_rows(mx_act) + G / 2) * ((2 * F + 255) / 256);
  return rows >= (mx_act ? 22 : 280) * G && tiles >= 256;
}

}  // namespace

Mx4Layout mx4_layout(int T, int d, int F, int E, int K, int n_shared) {
  Mx4Layout w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) & ~static_cast<size_t>(255);
    return o;
  };
  const size_t rows = static_cast<size_t>(T) * (K + n_shared), G = static_cast<size_t>(E) + n_shared;
  w.idx = take(rows * 4);
  w.gate = take(rows * 4);
  w.offsets = take((G + 1) * 4);
  w.tile_off = take((G + 1) * 4);
  w.active = take(G * 4);
  w.n_active = take(4);
  w.perm = take(rows * 4);
  w.inv = take(rows * 4);
  w.row_tok = take(rows * 4);
  w.pcount = take(static_cast<size_t>(permute_chunks(T, K + n_shared)) * G * 4);
  w.xq = take(static_cast<size_t>(T) * d / 2);
  w.xs = take(static_cast<size_t>(T) * mx4_quads(d) * 16);
  w.h = take(rows * F * 2);
  w.hs = take(rows * mx4_quads(F) * 16);
  // rows of o: one per entry; the parts of the few-token and batch paths' reductions
  const size_t few = static_cast<size_t>(kMx4FewSplits) * std::min(T, kMx4FewT);
  const size_t batch = std::min<size_t>(kMx4BatchSplits * rows, kMx4BatchSplitRows);
  w.o = take(std::max({rows, few, batch}) * d * 4);
  w.total = off;
  return w;
}

hipError_t launch_mx4_experts(const Mx4Args& a, void* workspace, hipStream_t stream) {
  const Mx4Layout w = mx4_layout(a.T, a.d, a.F, a.E, a.K, a.n_shared);
  char* ws = static_cast<char*>(workspace);
  Mx4Params p;
  p.a = a;
  p.G = a.E + a.n_shared;
  p.idx = a.idx;
  p.gate = a.gate;
  p.pb.offsets = reinterpret_cast<int32_t*>(ws + w.offsets);
  p.pb.tile_off = reinterpret_cast<int32_t*>(ws + w.tile_off);
  p.pb.active = reinterpret_cast<int32_t*>(ws + w.active);
  p.pb.n_active = reinterpret_cast<int32_t*>(ws + w.n_active);
  p.pb.perm = reinterpret_cast<int32_t*>(ws + w.perm);
  p.pb.inv = reinterpret_cast<int32_t*>(ws + w.inv);
  p.pb.row_tok = reinterpret_cast<int32_t*>(ws + w.row_tok);
  p.xq = reinterpret_cast<uint8_t*>(ws + w.xq);
  p.xs = reinterpret_cast<uint8_t*>(ws + w.xs);
  p.h = ws + w.h;
  p.hs = reinterpret_cast<uint8_t*>(ws + w.hs);
  p.o = reinterpret_cast<float*>(ws + w.o);
  if (a.T <= kMx4FewT) return launch_mx4_few(p, stream);
  const int KS = a.K + a.n_shared, rows = a.T * KS;
  hipError_t err;
  if (a.n_shared > 0 || a.mx_act) {   // else the caller's entries are all there is
    const int entry_blocks = a.n_shared > 0 ? (rows + kThreads - 1) / kThreads : 0;
    const int64_t quant_blocks = a.mx_act ? (static_cast<int64_t>(a.T) * a.d / 8 + kThreads - 1) / kThreads : 0;
    int32_t* idx = reinterpret_cast<int32_t*>(ws + w.idx);
    float* gate = reinterpret_cast<float*>(ws + w.gate);
    hipLaunchKernelGGL(mx4_prepare_kernel, dim3(static_cast<unsigned>(entry_blocks + quant_blocks)), dim3(kThreads), 0,
                       stream, p, idx, gate, entry_blocks);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
    if (a.n_shared > 0) {
      p.idx = idx;
      p.gate = gate;
    }
  }
  const bool wide = mx4_takes_wide(rows, p.G, a.F, a.mx_act);
  const int tile_rows = wide ? mx4_tile_rows(a.mx_act) : kMx4BatchRows;
  err = launch_permute(p.idx, a.T, KS, p.G, 0, tile_rows, p.pb, reinterpret_cast<int32_t*>(ws + w.pcount), stream);
  if (err != hipSuccess) return err;
  const int max_tiles = std::min(rows, rows / tile_rows + p.G);
  int splits = 1;
  if (wide) {
    err = launch_mx4_wide(p, max_tiles, stream);
  } else {
    // two workgroups a CU for the down projection, each with eight steps or more
    const int jobs = std::min(rows, p.G) * ((a.d + 255) / 256);
    while (splits < kMx4BatchSplits && jobs * splits < 512 && mx4_steps(a.F) >= 16 * splits &&
           2 * splits * rows <= kMx4BatchSplitRows)
      splits *= 2;
    err = launch_mx4_batch(p, max_tiles, splits, stream);
  }
  if (err != hipSuccess) return err;
  const int64_t cn = static_cast<int64_t>(a.T) * a.d / 4;
  hipLaunchKernelGGL(mx4_combine_kernel, dim3(static_cast<unsigned>((cn + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                     stream, p, splits);
  return hipGetLastError();
}

}  // namespace maskmoe
