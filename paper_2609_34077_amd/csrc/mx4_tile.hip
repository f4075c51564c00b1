// Both products of experts on MX4 weights for many rows per expert: 256 weight rows a workgroup on the matrix
// units' 16 x 16 tiles.
//
// Wavefronts lie two side by side along the tokens: wave w owns the weight fragments (16 rows each) of w / 2 and the
// token fragments w % 2, + 2, .., so that a last tile with few rows leaves every wavefront equally little to multiply.
// Weight rows are the instruction's row operand: a lane holds four neighbouring output columns of one token, and the
// gate and up rows of a column, which alternate in the packed layout, meet in one lane.
//   bf16 activations  256 token rows, eight wavefronts of 4 x 8 fragments, stages of 128 columns. Weights go from global
//                     memory to the registers of the two wavefronts that share them (4 bits a value: a quarter of the
//                     bytes that LDS would have to pass), a stage ahead, and are widened to bf16 there, beside the
//                     products (v_mfma_f32_16x16x32_bf16); tokens go straight to LDS, double-buffered (2 x 64 KB).
//                     Widening two values takes about as long as a product (16 cycles): with 8 x 4 fragments it was as
//                     much work as they, 4850 us for the Mixtral-shaped layer of 8192 tokens instead of 4330.
//   MX4 activations   128 token rows, four wavefronts of 8 x 4 fragments, stages of 128 columns on
//                     v_mfma_scale_f32_16x16x128_f8f6f4; both operands and their scales go straight to LDS, two stages
//                     ahead (3 x 24 KB and 6 KB), two workgroups a CU, whose starts and ends overlap. Workgroups of
//                     256 rows and eight wavefronts were slower for few steps and rows (both products, DeepSeek-shaped
//                     1200 / 4096 / 8192 tokens 128 / 290 / 479 us, these 106 / 285 / 460) and faster for many
//                     (Mixtral-shaped 1500 / 8192 tokens 373 / 1589 us, these 393 / 1632; all with expert outputs in bf16).
//                     In fp32, as they are, 109 / 278 to 301 / 499 and 400 / 1650, the latter 3.5 PFLOP/s.
// Token loads are buffer loads: rows past the tile's end and columns past a row's end read as zeros.

#include "gemm_tile.hpp"
#include "mx4.hpp"
#include "mx4_block.hpp"

namespace maskmoe {
namespace {

constexpr int kFrags = 16;               // weight fragments of a tile
constexpr int kWN = 2;                   // wavefronts side by side along the tokens
template <bool MX>
constexpr int kThreads = MX ? 256 : 512;
constexpr uint32_t kNoRow = 0xfffffff0u; // past any operand (fewer than 2^32 - 256 bytes)

// 16 bytes per lane at rsrc + voff + soff straight into LDS at m0v + 16 * lane; zeros past the buffer's end.
__device__ __forceinline__ void dma16s(uint32_t m0v, i32x4 rsrc, uint32_t voff, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(m0v), "v"(voff), "s"(rsrc),
               "s"(soff)
               : "memory", "m0");
}

constexpr uint32_t kStage = 24576;       // of MX4 operands in LDS

struct Tile {
  int g, row0, nrows, f0;   // expert, its first row and rows here, first weight fragment
};

template <bool MX, int EPI, int NL>
__device__ __forceinline__ void run_tile(const Mx4Params& p, const Tile& t, u32x4* lds) {
  const Mx4Args& a = p.a;
  const int lane = threadIdx.x & 63, l16 = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  constexpr int WN = kWN, kWF = MX ? 8 : 4;   // kWF: a wavefront's weight fragments
  const int wm = wave / WN, wn = wave % WN;
  const int C = EPI == 0 ? a.d : a.F, R = EPI == 0 ? 2 * a.F : a.d;
  const int steps = mx4_steps(C), quads = mx4_quads(C);
  const uint8_t* wc = (EPI == 0 ? a.gu_codes : a.dn_codes) + static_cast<size_t>(t.g) * (R / 16) * steps * 1024;
  const uint8_t* wsc = (EPI == 0 ? a.gu_scales : a.dn_scales) + static_cast<size_t>(t.g) * (R / 16) * quads * 256;
  const __amdgpu_buffer_rsrc_t cr = make_rsrc(wc, static_cast<uint32_t>(R / 16) * steps * 1024);
  const __amdgpu_buffer_rsrc_t sr = make_rsrc(wsc, static_cast<uint32_t>(R / 16) * quads * 256);
  uint32_t frag[kWF];   // fragments past the matrix repeat its last one and are not stored
#pragma unroll
  for (int i = 0; i < kWF; ++i) frag[i] = min(t.f0 + kWF * wm + i, R / 16 - 1);
  const int src_rows = EPI == 0 ? a.T : a.T * (a.K + a.n_shared);
  const void* x = EPI == 0 ? (MX ? static_cast<const void*>(p.xq) : a.x) : p.h;
  const uint32_t row_bytes = MX ? C / 2 : 2 * C;
  const i32x4 xr = buffer_rsrc(x, static_cast<uint32_t>(src_rows) * row_bytes);
  const uint32_t lds0 = lds_offset(lds);
  auto source = [&](int r) { return EPI == 0 ? p.pb.row_tok[t.row0 + r] : t.row0 + r; };

  f32x4 acc[kWF][NL];
#pragma unroll
  for (int i = 0; i < kWF; ++i)
#pragma unroll
    for (int n = 0; n < NL; ++n) acc[i][n] = f32x4{0, 0, 0, 0};

  if constexpr (!MX) {
    // token pieces: instruction i of this wave fills stage rows 4 (8 wave + i) .. + 3, 256 bytes each; the piece at
    // slot s of row r is logical piece s ^ (r & 15), so that 16 rows at one logical piece fall on all banks
    uint32_t off[8];
    bool upper[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = 4 * (8 * wave + i) + (lane >> 4);
      const int piece = (lane & 15) ^ (r & 15);
      off[i] = r < t.nrows ? source(r) * row_bytes + piece * 16 : kNoRow;
      upper[i] = piece >= 8;
    }
    const bool half = C % kMxStep != 0;   // the last step holds 64 columns
    auto dma = [&](int s, int buf) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (4 * (8 * wave + i) >= 16 * WN * NL) break;   // rows that no wavefront multiplies
        const uint32_t o = half && s == steps - 1 && upper[i] ? kNoRow : off[i];
        const uint32_t so = static_cast<uint32_t>(s) * 256;
        dma16s(lds0 + buf * 65536 + (8 * wave + i) * 1024, xr, o, so);
      }
    };
    u32x4 w[2][kWF];
    uint32_t ws[2][kWF];
    auto load_w = [&](int s, int set) {
#pragma unroll
      for (int i = 0; i < kWF; ++i) {
        w[set][i] = __builtin_amdgcn_raw_buffer_load_b128(cr, lane * 16, (frag[i] * steps + s) * 1024, 0);
        ws[set][i] = __builtin_amdgcn_raw_buffer_load_b32(sr, lane * 4, (frag[i] * quads + (s >> 2)) * 256, 0);
      }
    };
    // token row 16 (WN n + wn) + l16 of the stage, logical piece 4 lg + j
    auto compute = [&](int s, int set) {
      float sc[kWF];
#pragma unroll
      for (int i = 0; i < kWF; ++i) sc[i] = mx4_scale(ws[set][i] >> (8 * (s & 3)) & 255);
      const u32x4* b0 = lds + set * 4096 + (16 * wn + l16) * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 b[NL];
#pragma unroll
        for (int n = 0; n < NL; ++n) b[n] = b0[n * WN * 256 + ((4 * lg + j) ^ l16)];
#pragma unroll
        for (int i = 0; i < kWF; ++i) {
          const u32x4 wa = mx4_to_bf16(w[set][i][j], sc[i]);
#pragma unroll
          for (int n = 0; n < NL; ++n) acc[i][n] = mfma_16x16x32(wa, b[n], acc[i][n]);
        }
      }
    };
    // the stage is whole when every wavefront has waited for its part; its weights are in registers then, so that the
    // compiler does not wait again behind the next stage's loads
    auto arrive = [&](int set) {
      wait_vmcnt<0>();
#pragma unroll
      for (int i = 0; i < kWF; ++i) asm volatile("" : "+v"(w[set][i]), "+v"(ws[set][i]));
      lds_sync();
    };
    auto step = [&](int s, int set) {
      arrive(set);
      const int nx = min(s + 1, steps - 1);   // past the end: a buffer that nothing reads again
      dma(nx, set ^ 1);
      load_w(nx, set ^ 1);
      __builtin_amdgcn_sched_barrier(0);
      if (s < steps) compute(s, set);
      __builtin_amdgcn_sched_barrier(0);
    };
    dma(0, 0);
    load_w(0, 0);
    for (int s = 0; s < steps; s += 2) {
      step(s, 0);
      step(s + 1, 1);
    }
    wait_vmcnt<0>();
  } else {
    // A stage is one step: 16 fragments of weights (16 KB, operand order), 128 rows x 64 bytes of tokens (8 KB; the
    // piece at slot s of row r is logical piece s ^ (r / 4 & 3)). Three stages; the scales of four steps, a dword per
    // fragment lane and token block, in 6 KB behind them. Every wavefront issues the same number of loads a step (rows
    // past the end read as zeros), so that it can wait for the oldest alone.
    uint32_t off[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 16 * (2 * wave + i) + (lane >> 2);
      off[i] = r < t.nrows ? source(r) * row_bytes + ((lane & 3) ^ (r >> 2 & 3)) * 16 : kNoRow;
    }
    const i32x4 wr = buffer_rsrc(wc, static_cast<uint32_t>(R / 16) * steps * 1024);
    uint32_t in = 0;   // where the next stage goes
    auto dma = [&](int ahead) {
      const int s = min(ahead, steps - 1);   // past the end: a stage that nothing reads again
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int f = min(t.f0 + 4 * wave + i, R / 16 - 1);
        dma16s(lds0 + in + (4 * wave + i) * 1024, wr, lane * 16, (static_cast<uint32_t>(f) * steps + s) * 1024);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) dma16s(lds0 + in + 16384 + (2 * wave + i) * 1024, xr, off[i], static_cast<uint32_t>(s) * 64);
      in = in == 2 * kStage ? 0 : in + kStage;
    };
    // scales: a wavefront four fragments and 64 token rows (both pairs of wavefronts the same ones)
    const i32x4 wscr = buffer_rsrc(wsc, static_cast<uint32_t>(R / 16) * quads * 256);
    const i32x4 xscr = buffer_rsrc(EPI == 0 ? p.xs : p.hs, static_cast<uint32_t>(src_rows) * quads * 16);
    const uint32_t wsc_off = static_cast<uint32_t>(min(t.f0 + 4 * wave + (lane >> 4), R / 16 - 1)) * quads * 256 + (lane & 15) * 16;
    const int sr_row = 64 * (wave & 1) + lane;
    const uint32_t xsc_off = sr_row < t.nrows ? source(sr_row) * quads * 16 : kNoRow;
    auto dma_scales = [&](int ahead) {
      const uint32_t q = min(ahead, quads - 1);
      dma16s(lds0 + 3 * kStage + wave * 1024, wscr, wsc_off, q * 256);
      dma16s(lds0 + 3 * kStage + 4096 + (wave & 1) * 1024, xscr, xsc_off, q * 16);
    };
    // the last step of a C of an odd number of 64 columns: its upper blocks have no token scales
    const int cut = C % kMxStep != 0 ? steps - 1 : -1;
    uint32_t ws[kWF], ts[NL];
    int out = 0;   // the stage multiplied, in 16 bytes
    auto compute = [&](auto sub_c, int s) {
      constexpr int S = decltype(sub_c)::value;   // step within the quad
      const u32x4* wa = lds + out + kWF * wm * 64 + lane;
      const u32x4* xa = lds + out + 1024 + (16 * wn + l16) * 4 + (lg ^ (l16 >> 2));
      out = out == 2 * kStage / 16 ? 0 : out + kStage / 16;
      if constexpr (S == 0) {
        const uint32_t* sc = reinterpret_cast<const uint32_t*>(lds + 3 * kStage / 16);
#pragma unroll
        for (int i = 0; i < kWF; ++i) ws[i] = sc[(kWF * wm + i) * 64 + lane];
#pragma unroll
        for (int n = 0; n < NL; ++n) ts[n] = sc[1024 + (16 * (WN * n + wn) + l16) * 4 + lg];
      }
      u32x4 xv[NL];
      uint32_t bs[NL];
#pragma unroll
      for (int n = 0; n < NL; ++n) {
        xv[n] = xa[n * WN * 64];
        bs[n] = s == cut && lg >= 2 ? 0 : ts[n];
      }
#pragma unroll
      for (int i = 0; i < kWF; ++i) {
        const u32x4 wv = wa[i * 64];
#pragma unroll
        for (int n = 0; n < NL; ++n) acc[i][n] = mfma_mx4<S>(wv, xv[n], acc[i][n], ws[i], bs[n]);
      }
    };
    auto step = [&](auto sub_c, int s) {
      constexpr int S = decltype(sub_c)::value;
      // behind step s's loads are the next step's, and in S 2 the scales issued between them
      wait_vmcnt<S == 2 ? 8 : 6>();
      lds_sync();
      if constexpr (S == 1) dma_scales((s >> 2) + 1);   // every wavefront has read this quad's
      dma(s + 2);
      __builtin_amdgcn_sched_barrier(0);
      if (s < steps) compute(sub_c, s);
      __builtin_amdgcn_sched_barrier(0);
    };
    dma_scales(0);
    dma(0);
    dma(1);
    for (int s = 0; s < steps; s += 4) {
      step(std::integral_constant<int, 0>{}, s);
      step(std::integral_constant<int, 1>{}, s + 1);
      step(std::integral_constant<int, 2>{}, s + 2);
      step(std::integral_constant<int, 3>{}, s + 3);
    }
    wait_vmcnt<0>();   // nothing may arrive in LDS after the workgroup's end
  }

  // acc[i][n][e]: weight row 4 lg + e of fragment i, token l16 of fragment WN n + wn
#pragma unroll
  for (int n = 0; n < NL; ++n) {
    const int r = 16 * (WN * n + wn) + l16;
    const bool ok = r < t.nrows;
    const size_t row = t.row0 + r;
    if constexpr (EPI == 1) {
#pragma unroll
      for (int i = 0; i < kWF; ++i) {
        const int f = t.f0 + kWF * wm + i;
        if (ok && f < R / 16) *reinterpret_cast<f32x4*>(p.o + row * a.d + 16 * f + 4 * lg) = acc[i][n];
      }
    } else {
#pragma unroll
      for (int q = 0; q < kWF / 4; ++q) {   // 32 columns: two gate and two up fragments
        const int cb = (t.f0 + kWF * wm) / 4 + q;   // their block of h
        float h[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          h[e] = silu(acc[4 * q][n][e]) * acc[4 * q + 1][n][e];
          h[4 + e] = silu(acc[4 * q + 2][n][e]) * acc[4 * q + 3][n][e];
        }
        if constexpr (MX) {
          uint32_t m = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(h[e]) & 0x7fffffffu);
          m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16, kWave)));
          m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32, kWave)));
          const uint32_t byte = mx4_scale_byte(m);
          const uint32_t c = byte == 255 ? 0 : mx4_codes(h, mx4_scale(byte));
          // c: halves lg and 4 + lg of the block's eight. Lanes lg and lg ^ 1 share theirs: dwords lg / 2 and 2 + lg / 2
          const auto both = __builtin_amdgcn_permlane16_swap(c, c, false, false);
          const uint32_t pair = __builtin_amdgcn_perm(both[1], both[0], lg & 1 ? 0x07060302u : 0x05040100u);
          if (ok && cb < a.F / 32) {
            reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p.h) + row * (a.F / 2) + 16 * cb)[2 * (lg & 1) + (lg >> 1)] = pair;
            if (lg == 0) p.hs[row * 16 * mx4_quads(a.F) + mx4_scale_at(cb)] = static_cast<uint8_t>(byte);
          }
        } else {
          if (ok && cb < a.F / 32) {
            uint2* o = reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.h) + row * a.F + 32 * cb + 4 * lg);
            o[0] = make_uint2(f32x2_to_bf16x2(h[0], h[1]), f32x2_to_bf16x2(h[2], h[3]));
            o[4] = make_uint2(f32x2_to_bf16x2(h[4], h[5]), f32x2_to_bf16x2(h[6], h[7]));
          }
        }
      }
    }
  }
}

template <bool MX, int EPI>
__global__ __launch_bounds__(kThreads<MX>, 2) void mx4_wide_kernel(const Mx4Params p) {
  __shared__ u32x4 lds[MX ? (3 * kStage + 6144) / 16 : 8192];
  constexpr int kRows = mx4_tile_rows(MX);
  const int R = EPI == 0 ? 2 * p.a.F : p.a.d;
  const int wt = (R / 16 + kFrags - 1) / kFrags;   // weight tiles
  const int live = p.pb.tile_off[p.G] * wt;
  if (static_cast<int>(blockIdx.x) >= live) return;
  const int lid = xcd_tile_id(live);
  int mt, nt;
  grouped_tile_coords(lid, p.pb.tile_off[p.G], wt, mt, nt);
  int g = 0;
  {
    const int lane = threadIdx.x & 63;
    for (int g0 = 0; g0 < p.G; g0 += kWave) {
      const int i = g0 + lane;
      g += __popcll(__ballot(i < p.G && p.pb.tile_off[i + 1] <= mt));
    }
  }
  Tile t;
  t.g = g;
  t.row0 = p.pb.offsets[g] + (mt - p.pb.tile_off[g]) * kRows;
  t.nrows = min(kRows, p.pb.offsets[g + 1] - t.row0);
  t.f0 = nt * kFrags;
  const int quarters = __builtin_amdgcn_readfirstlane((t.nrows + kRows / 4 - 1) / (kRows / 4));   // of the tile's rows
  constexpr int Q = kRows / 4 / 16 / kWN;   // a wavefront's token fragments per quarter
  if (quarters == 4) run_tile<MX, EPI, 4 * Q>(p, t, lds);
  else if (quarters == 3) run_tile<MX, EPI, 3 * Q>(p, t, lds);
  else if (quarters == 2) run_tile<MX, EPI, 2 * Q>(p, t, lds);
  else run_tile<MX, EPI, Q>(p, t, lds);
}

template <bool MX>
hipError_t launch(const Mx4Params& p, int max_tiles, hipStream_t stream) {
  auto grid = [&](int R) { return dim3(static_cast<unsigned>(max_tiles) * ((R / 16 + kFrags - 1) / kFrags)); };
  hipLaunchKernelGGL((mx4_wide_kernel<MX, 0>), grid(2 * p.a.F), dim3(kThreads<MX>), 0, stream, p);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((mx4_wide_kernel<MX, 1>), grid(p.a.d), dim3(kThreads<MX>), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_wide(const Mx4Params& p, int max_tiles, hipStream_t stream) {
  return p.a.mx_act ? launch<true>(p, max_tiles, stream) : launch<false>(p, max_tiles, stream);
}

}  // namespace maskmoe
