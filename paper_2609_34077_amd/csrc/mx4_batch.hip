// Both products of experts on MX4 weights for a serving-sized batch: more tokens than the few-token kernels take,
// but few enough rows per expert that the time is still the stream of the experts' weights.
//
// A workgroup of four wavefronts owns 256 weight rows of one expert (a wavefront 64, its own) and up to 64 token
// rows. Weights go from memory to the registers of the one wavefront that multiplies them, issued kDepth steps of 128
// columns ahead (4 KiB a step); tokens go straight to LDS, where all four read them, as far ahead. Token fragments
// (16 rows) that hold none are not loaded and not multiplied.
// Less is in flight than is issued ahead: the compiler knows neither the token loads, which are assembly, nor which branch's
// weight loads ran (`alone`), so it waits again before each product with 8 to 11 younger loads outstanding (bf16; 14 to
// 19 with MX4 activations), when the next step's loads and half of the one's after it have arrived too. Mixtral-shaped layer, 96
// tokens, gate / up and down 94.5 + 52.5 us: 5.2 and 4.8 TB/s of weights, where a streaming read reaches 7.
// The down projection of few experts is split over the reduction as well, so that every CU streams; the combine
// adds the parts in order.

#include "gemm_tile.hpp"
#include "mx4.hpp"
#include "mx4_block.hpp"

#include <algorithm>

namespace maskmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 64;                // token rows of a tile
constexpr int kDepth = 3;                // steps issued ahead
constexpr int kStage = 1024;             // 16-byte pieces of a stage: 64 rows x 256 bytes
constexpr uint32_t kNowhere = 0xfffffff0u;   // an offset past every buffer: reads as zeros
constexpr int kNt = 2;                   // the load's non-temporal bit

struct Job {
  int g, row0, nrows, f0, s0, s1;   // expert, rows, first weight fragment, steps
  size_t out0;                      // EPI 1: first row of this part in o
  bool alone;                       // no other workgroup reads these weights
};

template <bool MX, int EPI, int NL>
__device__ __forceinline__ void run_job(const Mx4Params& p, const Job& t, u32x4* lds) {
  const Mx4Args& a = p.a;
  const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int C = EPI == 0 ? a.d : a.F, R = EPI == 0 ? 2 * a.F : a.d;
  const int steps = mx4_steps(C), quads = mx4_quads(C);
  const uint32_t fbytes = static_cast<uint32_t>(steps) * 1024, fscales = static_cast<uint32_t>(quads) * 256;
  const int f = min(t.f0 + 4 * wave, R / 16 - 4);   // past the last row: read again, not stored (R % 64 == 0)
  const size_t fe = static_cast<size_t>(t.g) * (R / 16) + f;
  const __amdgpu_buffer_rsrc_t codes = make_rsrc((EPI == 0 ? a.gu_codes : a.dn_codes) + fe * fbytes, 4 * fbytes);
  const __amdgpu_buffer_rsrc_t scales = make_rsrc((EPI == 0 ? a.gu_scales : a.dn_scales) + fe * fscales, 4 * fscales);
  const int src_rows = EPI == 0 ? a.T : a.T * (a.K + a.n_shared);
  const void* x = EPI == 0 ? (MX ? static_cast<const void*>(p.xq) : a.x) : p.h;
  const uint32_t row_bytes = MX ? C / 2 : 2 * C;
  const i32x4 xr = buffer_rsrc(x, static_cast<uint32_t>(src_rows) * row_bytes);
  const __amdgpu_buffer_rsrc_t xsr = make_rsrc(EPI == 0 ? p.xs : p.hs, static_cast<uint32_t>(src_rows) * quads * 16);
  const uint32_t lds0 = lds_offset(lds);
  auto source = [&](int r) { return static_cast<uint32_t>(EPI == 0 ? p.pb.row_tok[t.row0 + r] : t.row0 + r); };

  // token pieces. bf16: instruction i of a wave fills rows 4 (4 i + wave) .. + 3, 256 bytes each, the piece at slot s of
  // row r being logical piece s ^ (r & 15). MX4: instruction 0 fills rows 16 wave .., 64 bytes each, s ^ (r / 4 & 3).
  constexpr int kDma = MX ? 1 : NL;
  uint32_t off[kDma];
  bool upper[kDma];
#pragma unroll
  for (int i = 0; i < kDma; ++i) {
    const int r = MX ? 16 * wave + (lane >> 2) : 4 * (4 * i + wave) + (lane >> 4);
    const int piece = MX ? (lane & 3) ^ (r >> 2 & 3) : (lane & 15) ^ (r & 15);
    off[i] = r < t.nrows ? source(r) * row_bytes + piece * 16 : kNowhere;
    upper[i] = piece >= (MX ? 2 : 8);
  }
  const int cut = C % kMxStep != 0 ? steps - 1 : -1;   // the step that holds 64 columns
  auto dma = [&](int s, int slot) {
#pragma unroll
    for (int i = 0; i < kDma; ++i) {
      const uint32_t m0v = lds0 + slot * kStage * 16 + (MX ? wave : 4 * i + wave) * 1024;
      const uint32_t o = s == cut && upper[i] ? kNowhere : off[i], so = static_cast<uint32_t>(s) * (MX ? 64 : 256);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(m0v), "v"(o), "s"(xr),
                   "s"(so)
                   : "memory", "m0");
    }
  };
  uint32_t soff[NL];   // MX4: the token scales of this lane's block
  if constexpr (MX) {
#pragma unroll
    for (int n = 0; n < NL; ++n) {
      const int r = 16 * n + l16;
      soff[n] = r < t.nrows ? source(r) * quads * 16 + 4 * lg : kNowhere;
    }
  }
  struct Step {
    u32x4 w[4];
    uint32_t ws[4], bs[NL];
  };
  Step st[kDepth];
  auto load = [&](int s, Step& q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q.w[i] = t.alone ? __builtin_amdgcn_raw_buffer_load_b128(codes, lane * 16, i * fbytes + s * 1024, kNt)
                       : __builtin_amdgcn_raw_buffer_load_b128(codes, lane * 16, i * fbytes + s * 1024, 0);
      q.ws[i] = __builtin_amdgcn_raw_buffer_load_b32(scales, lane * 4, i * fscales + (s >> 2) * 256, 0);
    }
    if constexpr (MX) {
#pragma unroll
      for (int n = 0; n < NL; ++n) q.bs[n] = __builtin_amdgcn_raw_buffer_load_b32(xsr, soff[n], 16 * (s >> 2), 0);
    }
  };
  f32x4 acc[4][NL];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int n = 0; n < NL; ++n) acc[i][n] = f32x4{0, 0, 0, 0};
  auto multiply = [&](int s, int slot, const Step& q) {
    const int sh = 8 * (s & 3);
    if constexpr (MX) {
      const u32x4* b0 = lds + slot * kStage + l16 * 4 + (lg ^ (l16 >> 2));
      u32x4 b[NL];
      uint32_t bs[NL];
#pragma unroll
      for (int n = 0; n < NL; ++n) {
        b[n] = b0[n * 64];
        bs[n] = s == cut && lg >= 2 ? 0 : q.bs[n] >> sh;   // blocks past the row's end have no scale
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int n = 0; n < NL; ++n) acc[i][n] = mfma_mx4(q.w[i], b[n], acc[i][n], q.ws[i] >> sh, bs[n]);
    } else {
      float sc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[i] = mx4_scale(q.ws[i] >> sh & 255);
      const u32x4* b0 = lds + slot * kStage + l16 * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 b[NL];
#pragma unroll
        for (int n = 0; n < NL; ++n) b[n] = b0[n * 256 + ((4 * lg + j) ^ l16)];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 wa = mx4_to_bf16(q.w[i][j], sc[i]);
#pragma unroll
          for (int n = 0; n < NL; ++n) acc[i][n] = mfma_16x16x32(wa, b[n], acc[i][n]);
        }
      }
    }
  };
  // Step s sits in LDS slot s % (kDepth + 1) and register set (s - s0) % kDepth. A step's loads are issued tokens
  // first, so that kOps of each younger step are behind them. Past the end the last step is loaded again (into a slot
  // and registers that nothing reads), so that every wait is the same.
  constexpr int kOps = kDma + 8 + (MX ? NL : 0);
  static_assert(kOps * (kDepth - 1) < 64, "the wait's counter");
  auto step = [&](int s, Step& q) {
    wait_vmcnt<kOps*(kDepth - 1)>();
    lds_sync();
    dma(min(s + kDepth, t.s1 - 1), (s + kDepth) % (kDepth + 1));
    __builtin_amdgcn_sched_barrier(0);
    if (s < t.s1) multiply(s, s % (kDepth + 1), q);
    __builtin_amdgcn_sched_barrier(0);
    load(min(s + kDepth, t.s1 - 1), q);
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int i = 0; i < kDepth; ++i) {
    dma(min(t.s0 + i, t.s1 - 1), (t.s0 + i) % (kDepth + 1));
    load(min(t.s0 + i, t.s1 - 1), st[i]);
  }
  for (int s = t.s0; s < t.s1; s += kDepth) {
#pragma unroll
    for (int i = 0; i < kDepth; ++i) step(s + i, st[i]);
  }
  wait_vmcnt<0>();   // nothing may arrive in LDS after the workgroup's end

  // acc[i][n][e]: weight row 4 lg + e of fragment i, token l16 of fragment n
  if (f != t.f0 + 4 * wave) return;
#pragma unroll
  for (int n = 0; n < NL; ++n) {
    const int r = 16 * n + l16;
    const bool ok = r < t.nrows;
    if constexpr (EPI == 1) {
      if (ok) {
        f32x4* o = reinterpret_cast<f32x4*>(p.o + (t.out0 + r) * a.d + 16 * f + 4 * lg);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[4 * i] = acc[i][n];
      }
    } else {
      const size_t row = t.row0 + r;
      const int cb = f / 4;   // the block of 32 columns of h
      float h[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        h[e] = silu(acc[0][n][e]) * acc[1][n][e];
        h[4 + e] = silu(acc[2][n][e]) * acc[3][n][e];
      }
      if constexpr (MX) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(h[e]) & 0x7fffffffu);
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16, kWave)));
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32, kWave)));
        const uint32_t byte = mx4_scale_byte(m);
        const uint32_t c = byte == 255 ? 0 : mx4_codes(h, mx4_scale(byte));
        if (ok) {
          uint16_t* o = reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(p.h) + row * (a.F / 2) + 16 * cb + 2 * lg);
          o[0] = static_cast<uint16_t>(c);
          o[4] = static_cast<uint16_t>(c >> 16);
          if (lg == 0) p.hs[row * 16 * mx4_quads(a.F) + mx4_scale_at(cb)] = static_cast<uint8_t>(byte);
        }
      } else if (ok) {
        uint2* o = reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.h) + row * a.F + 32 * cb + 4 * lg);
        o[0] = make_uint2(f32x2_to_bf16x2(h[0], h[1]), f32x2_to_bf16x2(h[2], h[3]));
        o[4] = make_uint2(f32x2_to_bf16x2(h[4], h[5]), f32x2_to_bf16x2(h[6], h[7]));
      }
    }
  }
}

template <bool MX, int EPI>
__global__ __launch_bounds__(kThreads, 2) void mx4_batch_kernel(const Mx4Params p, int splits) {
  __shared__ u32x4 lds[(kDepth + 1) * kStage];
  const int C = EPI == 0 ? p.a.d : p.a.F, R = EPI == 0 ? 2 * p.a.F : p.a.d;
  const int wt = (R + 255) / 256, per = wt * splits;   // jobs per row tile
  const int live = p.pb.tile_off[p.G] * per;
  if (static_cast<int>(blockIdx.x) >= live) return;
  // neighbours on one XCD: the row tiles of an expert at the same weights
  const int lid = xcd_tile_id(live), lane = threadIdx.x & 63;
  int g = 0;
  for (int g0 = 0; g0 < p.G; g0 += kWave) {
    const int i = g0 + lane;
    g += __popcll(__ballot(i < p.G && p.pb.tile_off[i + 1] * per <= lid));
  }
  const int mtiles = p.pb.tile_off[g + 1] - p.pb.tile_off[g], within = lid - p.pb.tile_off[g] * per;
  const int m = within % mtiles, z = within / mtiles % splits, nt = within / mtiles / splits;
  const int steps = mx4_steps(C);
  Job t;
  t.g = g;
  t.row0 = p.pb.offsets[g] + m * kRows;
  t.nrows = min(kRows, p.pb.offsets[g + 1] - t.row0);
  t.f0 = 16 * nt;
  t.s0 = steps * z / splits;
  t.s1 = steps * (z + 1) / splits;
  t.out0 = static_cast<size_t>(z) * p.a.T * (p.a.K + p.a.n_shared) + t.row0;
  t.alone = mtiles == 1;
  const int nl = __builtin_amdgcn_readfirstlane((t.nrows + 15) / 16);
  if (nl == 1) run_job<MX, EPI, 1>(p, t, lds);
  else if (nl == 2) run_job<MX, EPI, 2>(p, t, lds);
  else if (nl == 3) run_job<MX, EPI, 3>(p, t, lds);
  else run_job<MX, EPI, 4>(p, t, lds);
}

template <bool MX>
hipError_t launch(const Mx4Params& p, int max_tiles, int splits, hipStream_t stream) {
  hipLaunchKernelGGL((mx4_batch_kernel<MX, 0>), dim3(max_tiles * ((2 * p.a.F + 255) / 256)), dim3(kThreads), 0, stream, p, 1);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((mx4_batch_kernel<MX, 1>), dim3(max_tiles * ((p.a.d + 255) / 256) * splits), dim3(kThreads), 0, stream, p,
                     splits);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_batch(const Mx4Params& p, int max_tiles, int splits, hipStream_t stream) {
  return p.a.mx_act ? launch<true>(p, max_tiles, splits, stream) : launch<false>(p, max_tiles, splits, stream);
}

}  // namespace maskmoe
