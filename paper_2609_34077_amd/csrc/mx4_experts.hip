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
__global__ __launch_bounds__(kThreads) void mx4_prepare_kernel(const Mx4Params p, int entry_blocks) {
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
    p.idx[j] = e;
    p.gate[j] = g;
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

// Group that holds row tile `tile` (tile < tile_off[G]): the groups that end at or before it, counted by
// all lanes in one round trip.
__device__ __forceinline__ int group_of_tile(const int32_t* tile_off, int G, int tile) {
  const int lane = threadIdx.x & 63;
  int g = 0;
  for (int g0 = 0; g0 < G; g0 += kWave) {
    const int i = g0 + lane;
    g += __popcll(__ballot(i < G && tile_off[i + 1] <= tile));
  }
  return g;
}

// A tile of 16 NF rows of one expert times 64 weight rows (EPI 0: 32 gate rows and their up rows, then the
// SwiGLU; EPI 1: rows of W_down). Four wavefronts split the reduction and join in LDS.
template <bool MX, int NF, int EPI>
__global__ __launch_bounds__(kThreads) void mx4_tile_kernel(const Mx4Params p) {
  __shared__ f32x4 red[4][4][NF][kWave];
  const Mx4Args& a = p.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, lg = lane >> 4;
  const int cols = EPI == 0 ? a.F / 32 : a.d / 64;
  const int tile = blockIdx.x / cols, cx = blockIdx.x % cols;
  if (tile >= p.pb.tile_off[p.G]) return;
  const int g = group_of_tile(p.pb.tile_off, p.G, tile);
  const int r0 = p.pb.offsets[g] + (tile - p.pb.tile_off[g]) * 16 * NF;
  const int nrows = min(16 * NF, p.pb.offsets[g + 1] - r0);
  const int C = EPI == 0 ? a.d : a.F, R = EPI == 0 ? 2 * a.F : a.d;
  const int steps = mx4_steps(C), quads = mx4_quads(C), blocks = C / kMxBlock;
  const uint8_t* codes = (EPI == 0 ? a.gu_codes : a.dn_codes) + static_cast<size_t>(g) * (R / 16) * steps * 1024;
  const uint8_t* scales = (EPI == 0 ? a.gu_scales : a.dn_scales) + static_cast<size_t>(g) * (R / 16) * quads * 256;
  size_t row[NF];
  bool live[NF];
#pragma unroll
  for (int n = 0; n < NF; ++n) {
    const int r = 16 * n + l16;
    live[n] = r < nrows;
    row[n] = !live[n] ? 0 : EPI == 0 ? p.pb.row_tok[r0 + r] : r0 + r;
  }
  f32x4 acc[4][NF];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int n = 0; n < NF; ++n) acc[i][n] = f32x4{0, 0, 0, 0};
  const int per = (steps + 3) / 4;
  const int s1 = min((wave + 1) * per, steps);
#pragma unroll 2
  for (int s = wave * per; s < s1; ++s) {
    const bool in = 4 * s + lg < blocks;
    u32x4 w[4];
    uint32_t ws[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const size_t f = 4 * cx + i;
      w[i] = *reinterpret_cast<const u32x4*>(codes + (f * steps + s) * 1024 + lane * 16);
      ws[i] = *reinterpret_cast<const uint32_t*>(scales + ((f * quads + (s >> 2)) * 64 + lane) * 4) >> (8 * (s & 3));
    }
    if constexpr (MX) {
      const uint8_t* xq = EPI == 0 ? p.xq : static_cast<const uint8_t*>(p.h);
      const uint8_t* xs = EPI == 0 ? p.xs : p.hs;
#pragma unroll
      for (int n = 0; n < NF; ++n) {
        u32x4 b = {0, 0, 0, 0};
        uint32_t bs = 0;
        if (live[n] && in) {
          const size_t blk = row[n] * blocks + 4 * s + lg;
          b = *reinterpret_cast<const u32x4*>(xq + blk * 16);
          bs = xs[row[n] * 16 * quads + mx4_scale_at(4 * s + lg)];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][n] = mfma_mx4(w[i], b, acc[i][n], ws[i], bs);
      }
    } else {
      const uint16_t* x = EPI == 0 ? a.x : static_cast<const uint16_t*>(p.h);
      u32x4 b[NF][4];
#pragma unroll
      for (int n = 0; n < NF; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          b[n][j] = u32x4{0, 0, 0, 0};
          if (live[n] && in)
            b[n][j] = *reinterpret_cast<const u32x4*>(x + row[n] * C + kMxStep * s + 32 * lg + 8 * j);
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float sc = mx4_scale(ws[i] & 255);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4 wa = mx4_to_bf16(w[i][j], sc);
#pragma unroll
          for (int n = 0; n < NF; ++n) acc[i][n] = mfma_16x16x32(wa, b[n][j], acc[i][n]);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int n = 0; n < NF; ++n) red[wave][i][n][lane] = acc[i][n];
  lds_sync();
  for (int n = wave; n < NF; n += 4) {
    f32x4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = red[0][i][n][lane] + red[1][i][n][lane] + red[2][i][n][lane] + red[3][i][n][lane];
    const bool ok = 16 * n + l16 < nrows;
    const size_t rr = r0 + 16 * n + l16;
    if constexpr (EPI == 1) {
      if (ok) {
        f32x4* o = reinterpret_cast<f32x4*>(p.o + rr * a.d + 64 * cx + 4 * lg);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[4 * i] = v[i];
      }
    } else {
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
        if (ok) {
          uint16_t* q = reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(p.h) + rr * (a.F / 2) + 16 * cx + 2 * lg);
          q[0] = static_cast<uint16_t>(c);
          q[4] = static_cast<uint16_t>(c >> 16);
          if (lg == 0) p.hs[rr * 16 * mx4_quads(a.F) + mx4_scale_at(cx)] = static_cast<uint8_t>(byte);
        }
      } else if (ok) {
        uint2* q = reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.h) + rr * a.F + 32 * cx + 4 * lg);
        q[0] = make_uint2(f32x2_to_bf16x2(h[0], h[1]), f32x2_to_bf16x2(h[2], h[3]));
        q[4] = make_uint2(f32x2_to_bf16x2(h[4], h[5]), f32x2_to_bf16x2(h[6], h[7]));
      }
    }
  }
}

// y = sum of the gate-weighted expert outputs in entry order, fp32, rounded once; a thread per 4 columns.
__global__ __launch_bounds__(kThreads) void mx4_combine_kernel(const Mx4Params p) {
  const Mx4Args& a = p.a;
  const int KS = a.K + a.n_shared, c4 = a.d / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= static_cast<int64_t>(a.T) * c4) return;
  const int t = static_cast<int>(i / c4), c = static_cast<int>(i % c4);
  f32x4 s = {0, 0, 0, 0};
  for (int k = 0; k < KS; ++k) {
    const int j = t * KS + k;
    if (p.idx[j] < 0) continue;
    const float g = p.gate[j];
    const f32x4 o = reinterpret_cast<const f32x4*>(p.o)[static_cast<size_t>(p.pb.inv[j]) * c4 + c];
#pragma unroll
    for (int q = 0; q < 4; ++q) s[q] += g * o[q];
  }
  reinterpret_cast<uint2*>(a.y)[i] = make_uint2(f32x2_to_bf16x2(s[0], s[1]), f32x2_to_bf16x2(s[2], s[3]));
}

template <bool MX, int NF>
hipError_t launch_tiles(const Mx4Params& p, int max_tiles, hipStream_t stream) {
  hipLaunchKernelGGL((mx4_tile_kernel<MX, NF, 0>), dim3(p.a.F / 32 * max_tiles), dim3(kThreads), 0, stream, p);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((mx4_tile_kernel<MX, NF, 1>), dim3(p.a.d / 64 * max_tiles), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
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
  w.o = take(rows * d * 4);
  w.total = off;
  return w;
}

hipError_t launch_mx4_experts(const Mx4Args& a, void* workspace, hipStream_t stream) {
  const Mx4Layout w = mx4_layout(a.T, a.d, a.F, a.E, a.K, a.n_shared);
  char* ws = static_cast<char*>(workspace);
  Mx4Params p;
  p.a = a;
  p.G = a.E + a.n_shared;
  p.idx = reinterpret_cast<int32_t*>(ws + w.idx);
  p.gate = reinterpret_cast<float*>(ws + w.gate);
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
  const int KS = a.K + a.n_shared, rows = a.T * KS;
  const int entry_blocks = (rows + kThreads - 1) / kThreads;
  const int64_t quant_blocks = a.mx_act ? (static_cast<int64_t>(a.T) * a.d / 8 + kThreads - 1) / kThreads : 0;
  hipLaunchKernelGGL(mx4_prepare_kernel, dim3(static_cast<unsigned>(entry_blocks + quant_blocks)), dim3(kThreads), 0,
                     stream, p, entry_blocks);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  const bool few = a.T <= 16;
  const bool wide = rows >= 100 * p.G;
  const int tile_rows = few ? 16 : wide ? kMx4TileRows : 64;
  err = launch_permute(p.idx, a.T, KS, p.G, 0, tile_rows, p.pb, reinterpret_cast<int32_t*>(ws + w.pcount), stream);
  if (err != hipSuccess) return err;
  const int max_tiles = std::min(rows, rows / tile_rows + p.G);
  if (wide) err = launch_mx4_wide(p, max_tiles, stream);
  else if (a.mx_act) err = few ? launch_tiles<true, 1>(p, max_tiles, stream) : launch_tiles<true, 4>(p, max_tiles, stream);
  else err = few ? launch_tiles<false, 1>(p, max_tiles, stream) : launch_tiles<false, 4>(p, max_tiles, stream);
  if (err != hipSuccess) return err;
  const int64_t cn = static_cast<int64_t>(a.T) * a.d / 4;
  hipLaunchKernelGGL(mx4_combine_kernel, dim3(static_cast<unsigned>((cn + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                     stream, p);
  return hipGetLastError();
}

}  // namespace maskmoe
