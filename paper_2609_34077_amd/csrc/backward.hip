// Expert-side backward of the masked MoE layer: the SwiGLU experts' weight gradients and their
// share of dL/dx, with the routing held fixed.
//
// The routers and experts update at every step (Section 3.2, Stage 1; Stage 2 continues with
// them). By Eq. 1, routed expert e receives dL/dF = g dy on the tokens that chose it and a
// shared expert dy on every token. Through F(x) = W_down (SiLU(W_gate x) * W_up x), with
// a = x W_gate^T, b = x W_up^T, h = SiLU(a) * b kept by the training forward:
//   dh = dO W_down               da = dh * b * SiLU'(a),  db = dh * SiLU(a)
//   dX = da W_gate + db W_up     dW_down = dO^T h,  dW_gate = da^T x,  dW_up = db^T x
// per expert, over the permuted rows of the forward (one row per (token, slot), shared
// experts' rows after them).
//
// Every product is run as C = A B^T on the 256x256x64 MFMA tile of gemm_tile.hpp. Operands whose
// contraction index is strided in storage are read in place as K-major operands (loaded by rows
// of the contraction index, turned into MFMA operands by transposing LDS reads): the weights
// of the dgrads, and both operands of the weight gradients, whose contraction runs over each
// expert's own rows of dO, h, [da db] and the gathered x (rows past the group's end read as
// zeros; an expert no token chose gets zeros).
// A row group's last tile multiplies and loads only its 64-row pieces that hold rows, as in the forward (but with
// SwiGLU's backward on bf16 pre-activations, which keeps whole tiles).
// Rounding (bf16 layers): dO = g dy and [da db] are rounded to bf16 before their GEMMs;
// accumulation is fp32; dX, dW are fp32.

#include <mutex>
#include <type_traits>

#include "common.hpp"
#include "gemm_tile.hpp"
#include "kernels.hpp"
#include "mx8.hpp"
#include "train_experts.hpp"

namespace maskmoe {
namespace {

constexpr int kBwdThreads = 256;

__device__ __forceinline__ uint32_t scale_pair(uint32_t v, float w) {
  const float lo = bf16_to_f32(static_cast<uint16_t>(v & 0xffffu)) * w;
  const float hi = bf16_to_f32(static_cast<uint16_t>(v >> 16)) * w;
  return f32x2_to_bf16x2(lo, hi);
}

// dO[r, :] = bf16(w_r dy[row_tok[r], :]): w_r the gate of the (token, slot) entry at routed row
// r, 1 for shared-expert rows. One workgroup per row; d % 8 == 0.
__global__ __launch_bounds__(kBwdThreads) void build_dout_kernel(const uint16_t* __restrict__ dy,
                                                                 const float* __restrict__ gate,
                                                                 const int32_t* __restrict__ perm,
                                                                 const int32_t* __restrict__ row_tok, int TK, int d,
                                                                 uint16_t* __restrict__ dout) {
  const int r = blockIdx.x;
  const float w = r < TK ? gate[perm[r]] : 1.0f;
  const uint16_t* src = dy + static_cast<size_t>(row_tok[r]) * d;
  uint16_t* dst = dout + static_cast<size_t>(r) * d;
  for (int c = threadIdx.x * 8; c < d; c += kBwdThreads * 8) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(src + c);
    u32x4 o;
#pragma unroll
    for (int h = 0; h < 4; ++h) o[h] = scale_pair(v[h], w);
    *reinterpret_cast<u32x4*>(dst + c) = o;
  }
}

// xg[r, :] = x[row_tok[r], :] (the gathered tokens of the weight gradient of gate/up, read in
// place as a K-major operand). One workgroup per row; d % 8 == 0.
__global__ __launch_bounds__(kBwdThreads) void gather_rows_kernel(const uint16_t* __restrict__ x,
                                                                  const int32_t* __restrict__ row_tok, int d,
                                                                  uint16_t* __restrict__ xg) {
  const int r = blockIdx.x;
  const uint16_t* src = x + static_cast<size_t>(row_tok[r]) * d;
  uint16_t* dst = xg + static_cast<size_t>(r) * d;
  for (int c = threadIdx.x * 8; c < d; c += kBwdThreads * 8)
    *reinterpret_cast<u32x4*>(dst + c) = *reinterpret_cast<const u32x4*>(src + c);
}

struct NtArgs {
  const uint16_t* a;          // ROWS: [rows, K] (lda), K-contiguous; KSPLIT: K-major [rows, M] (lda)
  const uint16_t* b;          // ROWS: per routed expert K-major [K, N] matrices (ldb = N); KSPLIT: K-major [rows, N]
  const uint16_t* bs;         // ROWS: the shared experts' [K, N] matrices
  const int32_t* offsets;     // [G+1] rows of each group
  const int32_t* tile_off;    // [G+1] row tiles of each group (ROWS)
  const int32_t* active;      // KSPLIT: the non-empty groups, n_active[0] of them
  const int32_t* n_active;
  const uint16_t* ab;         // SWIGLU_BWD: saved pre-activations [rows, 2N]
  const int8_t* codes;        // SWIGLU_KEPT: 8-bit blocks of the pre-activations [rows, 2N]
  const uint8_t* scales;      // SWIGLU_KEPT: [rows, 2N / 32]
  const float* row_gate;      // SWIGLU_KEPT: gate of each row
  uint16_t* gh;               // SWIGLU_KEPT: gate times SwiGLU activation [rows, N]
  float* dgate_part;          // SWIGLU_KEPT: [rows, n_tiles] partial sums of u h
  void* c;                    // ROWS: [rows, ldc]; KSPLIT: routed groups' [M, N] matrices
  void* cs;                   // KSPLIT: shared groups' [M, N] matrices
  int32_t* next;              // wgrad_kernel: [8] tiles that each XCD has handed out, 0 at the start
  float* part;                // ROWS, fp32 output: partial tiles of split tail tiles (tile_job)
  int G, E, M, N, K, lda, ldb, ldc, mt_max, n_tiles;
  int cu_xcd;                 // workgroups an XCD runs at once
};

// ROWS with fp32 output may split each XCD's last-round tiles (see tile_job).
__host__ __device__ constexpr bool nt_tail_split(int mode, int epi, int nk) {
  return mode == 0 && epi == 1 && tail_splittable(nk);
}

// The gradients of the groups that no row reached are zero. Where they are no more than the reached
// ones, every workgroup of a weight gradient writes its share of them, slice `lid` of `live` of each
// such [M, N] matrix, behind its own tile's stores: the matrix cores bound it and leave the write
// bandwidth. Otherwise (zero_unused_kernel) they are filled on a second stream, beside dgrads that
// are then short and far from the write bandwidth. Training steps, filled / here: Mixtral-shaped,
// 4 of 8 experts chosen, 8192 tokens (2.8 GB of zeros) 15.04 / 14.90 ms, 700 tokens 2.79 / 2.63,
// 64 tokens 1.97 / 1.87; DeepSeek-shaped, 12 of 64 chosen, 1000 tokens 1.13 / 1.18, 100 tokens
// 0.79 / 0.85.
__device__ __forceinline__ bool zeros_in_wgrad(int G, int n_active) { return G - n_active <= n_active; }

constexpr int kDeadWords = (256 + 8 + 63) / 64;   // the limits on E and the shared experts

// Bit l of word w: group 64 w + l is empty.
__device__ __forceinline__ void empty_groups(const int32_t* offsets, int G, uint64_t (&dead)[kDeadWords]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int w = 0; w < kDeadWords; ++w) {
    const int g = min(64 * w + lane, G - 1);
    dead[w] = 64 * w < G ? __ballot(64 * w + lane < G && offsets[g + 1] == offsets[g]) : 0;
  }
}

// n: 16-byte pieces of a matrix.
__device__ __forceinline__ void zero_slices(const uint64_t (&dead)[kDeadWords], int E, size_t n, int lid, int live,
                                            float* c, float* cs) {
  const size_t i0 = n * lid / live, i1 = n * (lid + 1) / live;
#pragma unroll
  for (int w = 0; w < kDeadWords; ++w)
    for (uint64_t m = dead[w]; m; m &= m - 1) {
      const int g = 64 * w + __builtin_ctzll(m);
      f32x4* dst = reinterpret_cast<f32x4*>(g < E ? c : cs) + static_cast<size_t>(g < E ? g : g - E) * n;
      for (size_t i = i0 + threadIdx.x; i < i1; i += kTileThreads)
        __builtin_nontemporal_store(f32x4{0.f, 0.f, 0.f, 0.f}, dst + i);
    }
}

enum { kNtRows = 0, kNtKSplit = 1 };
enum { kEpiSwigluBwd = 0, kEpiF32 = 1, kEpiSwigluKept = 2 };

// Sum over each half of the wavefront, in its last lane.
__device__ __forceinline__ float half_wave_sum(float v) {
  auto add = [&](auto ctrl, auto rows) {
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, decltype(rows)::value,
                                                    0xF, false));
  };
  using std::integral_constant;
  add(integral_constant<int, 0xB1>{}, integral_constant<int, 0xF>{});    // lanes 1 apart
  add(integral_constant<int, 0x4E>{}, integral_constant<int, 0xF>{});    // 2 apart
  add(integral_constant<int, 0x141>{}, integral_constant<int, 0xF>{});   // mirrored within 8
  add(integral_constant<int, 0x140>{}, integral_constant<int, 0xF>{});   // mirrored within 16
  add(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});   // lane 15 of rows 0, 2 to rows 1, 3
  return v;
}

// Epilogue of u = dy W_down with the pre-activations in 8-bit blocks: da, db (bf16, [rows, 2N]), the gated SwiGLU
// activation for the weight gradient (bf16, [rows, N]) and this tile's share of every row's d_gate = <u, h>. As
// kEpiSwigluBwd's, the tile goes through LDS in parts of 128 rows, a part's blocks loaded before it is staged.
template <int TM>
__device__ __forceinline__ void swiglu_kept_epilogue(const NtArgs& p, const f32x16 (&acc)[TM][kTileTN], int row0,
                                                     int row_end, int n0, int nt, TileLds& L) {
  const int tid = threadIdx.x;
  float* stg = reinterpret_cast<float*>(&L);
  uint16_t* o = static_cast<uint16_t*>(p.c);
  const size_t N = p.N;
  row_end = min(row_end, row0 + 64 * TM);
#pragma unroll
  for (int h = 0; h < (TM + 1) / 2; ++h) {
    uint2 a8[8], b8[8];
    uint32_t sa[8], sb[8];
    float gate[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {   // 4096 pieces of 8 columns: 32 per staged row
      const int u = tid + kTileThreads * q;
      const int pr = u >> 5, col = n0 + (u & 31) * 8;
      const int row = row0 + staged_tile_row<TM>(pr, h);
      a8[q] = b8[q] = make_uint2(0, 0);
      sa[q] = sb[q] = 0;
      gate[q] = 0.0f;
      if (row < row_end && col < p.N) {
        const size_t at = row * 2 * N + col;
        a8[q] = *reinterpret_cast<const uint2*>(p.codes + at);
        b8[q] = *reinterpret_cast<const uint2*>(p.codes + at + N);
        sa[q] = p.scales[at / kMx8Block];
        sb[q] = p.scales[(at + N) / kMx8Block];
        gate[q] = p.row_gate[row];
      }
    }
    wait_lgkmcnt0();
    tile_barrier();   // the k-loop's (or the previous part's) LDS reads are done
    stage_part<TM>(stg, acc, h);
    wait_lgkmcnt0();
    tile_barrier();
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int u = tid + kTileThreads * q;
      const int pr = u >> 5, cg = (u & 31) * 8, col = n0 + cg;
      const int row = row0 + staged_tile_row<TM>(pr, h);
      const bool live = row < row_end && col < p.N;
      float v[8], av[8], bv[8], da[8], db[8], gh[8];
      *reinterpret_cast<float4*>(&v[0]) = *reinterpret_cast<const float4*>(&stg[pr * kStgPitch + cg]);
      *reinterpret_cast<float4*>(&v[4]) = *reinterpret_cast<const float4*>(&stg[pr * kStgPitch + cg + 4]);
      const float s_a = mx8_step(sa[q]), s_b = mx8_step(sb[q]);
      mx8_decode4(a8[q].x, s_a, av);
      mx8_decode4(a8[q].y, s_a, av + 4);
      mx8_decode4(b8[q].x, s_b, bv);
      mx8_decode4(b8[q].y, s_b, bv + 4);
      float dot = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float s = sigmoid(av[e]), l = av[e] * s, hv = l * bv[e], gu = gate[q] * v[e];
        dot += v[e] * hv;
        da[e] = gu * bv[e] * (s + l - l * s);   // SiLU' = s + a s (1 - s)
        db[e] = gu * l;
        gh[e] = gate[q] * hv;
      }
      dot = half_wave_sum(live ? dot : 0.0f);   // 32 lanes hold a staged row
      if ((u & 31) == 31 && row < row_end) p.dgate_part[static_cast<size_t>(row) * p.n_tiles + nt] = dot;
      if (!live) continue;
      uint16_t* dst = o + row * 2 * N + col;
      u32x4 pa, pb, pg;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        pa[e] = f32x2_to_bf16x2(da[2 * e], da[2 * e + 1]);
        pb[e] = f32x2_to_bf16x2(db[2 * e], db[2 * e + 1]);
        pg[e] = f32x2_to_bf16x2(gh[2 * e], gh[2 * e + 1]);
      }
      *reinterpret_cast<u32x4*>(dst) = pa;
      *reinterpret_cast<u32x4*>(dst + N) = pb;
      *reinterpret_cast<u32x4*>(p.gh + row * N + col) = pg;
    }
  }
}


// ROWS (dgrad): group g's rows offsets[g]..offsets[g+1] of A (K-contiguous) times its own
// K-major [K, N] matrix, row tiles enumerated by tile_off as in the forward. KSPLIT (wgrad): for
// every non-empty group g the full [M, N] product over its rows offsets[g]..offsets[g+1] of the
// K-major A [rows, M] and B [rows, N]; the grid is sized for all groups and the live tiles
// (n_active x tiles per group) are spread over the XCDs.
template <int MODE, int EPI>
__global__ __launch_bounds__(kTileThreads) void gemm_nt_kernel(const NtArgs p) {
  constexpr int TM = kTileTM, TN = kTileTN, WN = 4;
  __shared__ TileLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wn = wave % WN;
  int mt, nt, g, row0, row_end, nk;
  TileJob job{0, 0, 1, -1};
  int tm = kTileTM;
  TileOps ops{};
  TileKm akm{}, bkm{};
  uint64_t dead[kDeadWords] = {};
  int live_tiles = 0, lid = 0;   // KSPLIT
  if (MODE == kNtRows) {   // each XCD's share of the live row tiles (tile_job)
    const int mt_live = p.tile_off[p.G];
    const int live = mt_live * p.n_tiles;
    const int nkf = p.K / kTileK;
    if (!tile_job(static_cast<int>(blockIdx.x), live, p.cu_xcd, nkf, nt_tail_split(MODE, EPI, nkf), job)) return;
    grouped_tile_coords(job.lid, mt_live, p.n_tiles, mt, nt);
    int lo = 0, hi = p.G;   // tile_off[lo] <= mt < tile_off[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.tile_off[mid] <= mt) lo = mid; else hi = mid;
    }
    g = lo;
    row0 = p.offsets[g] + (mt - p.tile_off[g]) * kTileM;
    row_end = p.offsets[g + 1];
    nk = nkf / job.s;
    const int k0 = job.z * nk * kTileK;
    const int n0 = nt * kTileN;
    ops.a = reinterpret_cast<const char*>(p.a + k0);
    if (EPI != kEpiSwigluBwd && job.s == 1) tm = min((row_end - row0 + 63) / 64, kTileTM);
#pragma unroll
    for (int i = 0; i < 4; ++i)   // element offsets < 2^31 (checked by the host)
      ops.aoff[i] =
          static_cast<uint32_t>(min(row0 + tile_dma_row_a(tm, i), row_end - 1) * p.lda + tile_dma_chunk_a(tm, i) * 8) * 2u;
    const uint16_t* bm = g < p.E ? p.b + static_cast<size_t>(g) * p.N * p.K : p.bs + static_cast<size_t>(g - p.E) * p.N * p.K;
    bkm.base = reinterpret_cast<const char*>(bm + static_cast<size_t>(k0) * p.ldb + n0);
    bkm.ld = p.ldb * 2;
    bkm.krows = nk * kTileK;
    bkm.mcols = p.N - n0;
  } else {
    const int per = p.mt_max * p.n_tiles;
    live_tiles = p.n_active[0] * per;
    if (static_cast<int>(blockIdx.x) >= live_tiles) return;
    lid = xcd_tile_id(live_tiles);
    if (zeros_in_wgrad(p.G, p.n_active[0])) empty_groups(p.offsets, p.G, dead);
    g = p.active[lid / per];
    grouped_tile_coords(lid % per, p.mt_max, p.n_tiles, mt, nt);
    row0 = mt * kTileM;
    row_end = p.M;
    const int r0 = p.offsets[g], nrows = p.offsets[g + 1] - r0;
    nk = (nrows + kTileK - 1) / kTileK;
    akm.base = reinterpret_cast<const char*>(p.a + static_cast<size_t>(r0) * p.lda + row0);
    akm.ld = p.lda * 2;
    akm.krows = nrows;
    akm.mcols = p.M - row0;
    bkm.base = reinterpret_cast<const char*>(p.b + static_cast<size_t>(r0) * p.ldb + nt * kTileN);
    bkm.ld = p.ldb * 2;
    bkm.krows = nrows;
    bkm.mcols = p.N - nt * kTileN;
  }
  const int n0 = nt * kTileN;
  int bfrag[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j) bfrag[j] = wn * 64 + j * 32 + (lane & 31);
  if constexpr (MODE == kNtRows && EPI != kEpiSwigluBwd) {
    auto tile = [&](auto tm_c) {
      constexpr int M = decltype(tm_c)::value;
      f32x16 acc[M][TN];
#pragma unroll
      for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
      gemm_tile_mainloop<false, false, true, false, M>(ops, nk, bfrag, acc, lds, nullptr, &akm, &bkm);
      if constexpr (EPI == kEpiSwigluKept) {
        swiglu_kept_epilogue<M>(p, acc, row0, row_end, n0, nt, lds);
      } else {
        if constexpr (M == kTileTM) {
          if (job.s > 1) {   // a slice of a split tail tile
            tail_store_partial(p.part, job.slot, acc);
            return;
          }
        }
        tile_store_f32<M>(acc, static_cast<float*>(p.c), p.ldc, row0, row_end, n0, p.N, lds);
      }
    };
    using std::integral_constant;
    if (tm == 4) tile(integral_constant<int, 4>{});
    else if (tm == 3) tile(integral_constant<int, 3>{});
    else if (tm == 2) tile(integral_constant<int, 2>{});
    else tile(integral_constant<int, 1>{});
    return;
  }
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  gemm_tile_mainloop<false, MODE == kNtKSplit, true>(ops, nk, bfrag, acc, lds, nullptr, &akm, &bkm);

  // acc[i][j][4 jj + ii] is row wm*128 + i*32 + 8 jj + 4 (lane >> 5) + ii, column
  // wn*64 + j*32 + (lane & 31) of the tile.
  if (EPI == kEpiSwigluBwd) {
    // v = dh; da, db (bf16) into [rows, 2N]. The tile goes through LDS (free after the k-loop)
    // in two halves of 128 rows x 256 columns, so that each thread then reads a, b and writes
    // da, db eight columns at a time: 16-byte accesses instead of one 2-byte access per value
    // and operand, which kept the texture-address path busy for a fifth of the kernel. A half's
    // a and b are loaded before it is staged, all in flight together. N % 64 == 0 (checked by
    // the host), so a group of eight columns is either whole or past N.
    float* stg = reinterpret_cast<float*>(&lds);
    uint16_t* o = static_cast<uint16_t*>(p.c);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 a8[8], b8[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {   // 4096 groups of 8 columns: 32 per staged row
        const int u = tid + kTileThreads * q;
        const int pr = u >> 5, col = n0 + (u & 31) * 8;
        const int row = row0 + (pr >> 6) * 128 + 64 * h + (pr & 63);
        if (row < row_end && col < p.N) {
          const uint16_t* src = p.ab + static_cast<size_t>(row) * 2 * p.N + col;
          a8[q] = *reinterpret_cast<const u32x4*>(src);
          b8[q] = *reinterpret_cast<const u32x4*>(src + p.N);
        }
      }
      wait_lgkmcnt0();
      tile_barrier();   // the k-loop's (or the previous half's) LDS reads are done
      stage_part<kTileTM>(stg, acc, h);
      wait_lgkmcnt0();
      tile_barrier();
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int u = tid + kTileThreads * q;
        const int pr = u >> 5, cg = (u & 31) * 8, col = n0 + cg;
        const int row = row0 + (pr >> 6) * 128 + 64 * h + (pr & 63);
        if (row >= row_end || col >= p.N) continue;
        float v[8];
        *reinterpret_cast<float4*>(&v[0]) = *reinterpret_cast<const float4*>(&stg[pr * kStgPitch + cg]);
        *reinterpret_cast<float4*>(&v[4]) = *reinterpret_cast<const float4*>(&stg[pr * kStgPitch + cg + 4]);
        const uint16_t* av8 = reinterpret_cast<const uint16_t*>(&a8[q]);
        const uint16_t* bv8 = reinterpret_cast<const uint16_t*>(&b8[q]);
        uint16_t da8[8], db8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float av = bf16_to_f32(av8[e]), bv = bf16_to_f32(bv8[e]);
          const float s = sigmoid(av);
          da8[e] = f32_to_bf16(v[e] * bv * (s * (1.0f + av * (1.0f - s))));
          db8[e] = f32_to_bf16(v[e] * av * s);
        }
        uint16_t* dst = o + static_cast<size_t>(row) * 2 * p.N + col;
        *reinterpret_cast<u32x4*>(dst) = *reinterpret_cast<const u32x4*>(da8);
        *reinterpret_cast<u32x4*>(dst + p.N) = *reinterpret_cast<const u32x4*>(db8);
      }
    }
    return;
  }
  float* cf = g < p.E ? static_cast<float*>(p.c) + static_cast<size_t>(g) * p.M * p.N
                      : static_cast<float*>(p.cs) + static_cast<size_t>(g - p.E) * p.M * p.N;
  tile_store_f32<kTileTM>(acc, cf, p.N, row0, row_end, n0, p.N, lds);
  zero_slices(dead, p.E, static_cast<size_t>(p.M) * p.N / 4, lid, live_tiles, static_cast<float*>(p.c),
              static_cast<float*>(p.cs));
}

// Weight gradients in bf16: for every group with rows the [M, N] product over its rows of the K-major A [rows, M] and
// B [rows, N], p.active naming the groups by descending rows. One workgroup a CU takes tile after tile; the first k-tile
// of the next tile is loaded while this one's results go through the other 64 KB of LDS (128 rows at a time, as bf16,
// so that they leave in 16-byte stores), and the stores are not waited for. An expert's reduction is short where there
// are many (DeepSeek-shaped, 4096 tokens: six k-tiles, 10 us, of which a workgroup per tile made 20).
// After its first two tiles a workgroup takes them from its XCD's counter (which changes who computes a tile, not what
// it holds): asked for at the start of a tile, handed round during its end, used for the loads at the next one's end.
// Tile order: every XCD takes an eighth of each group (pieces of per / 8 consecutive tiles, dealt in turn), so that all
// have the same work and no long reduction starts late. With a range of consecutive tiles for each XCD instead, as for
// products whose tiles are all alike, the XCD with the shared experts' tiles decided: the two gradients of that layer
// 854 + 453 us, dealt 520 + 270.
__global__ __launch_bounds__(kTileThreads) void wgrad_kernel(const NtArgs p) {
  __shared__ TileLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / 4, wn = wave % 4;
  const int per = p.mt_max * p.n_tiles, live_tiles = p.n_active[0] * per;
  const int piece = per < 8 ? 1 : per / 8, xcd = blockIdx.x & 7, slots = gridDim.x >> 3;
  uint64_t dead[kDeadWords] = {};
  const bool zeros = zeros_in_wgrad(p.G, p.n_active[0]);
  if (zeros) empty_groups(p.offsets, p.G, dead);
  int bfrag[kTileTN];
#pragma unroll
  for (int j = 0; j < kTileTN; ++j) bfrag[j] = wn * 64 + j * 32 + (lane & 31);

  struct Job {
    int g, mt, nt, nk;
    TileKm a, b;
  };
  auto tile_of = [&](int local) { return (local / piece * 8 + xcd) * piece + local % piece; };
  auto job_of = [&](int lid) {
    Job j;
    j.g = p.active[lid / per];
    grouped_tile_coords(lid % per, p.mt_max, p.n_tiles, j.mt, j.nt);
    const int r0 = p.offsets[j.g], nrows = p.offsets[j.g + 1] - r0;
    j.nk = (nrows + kTileK - 1) / kTileK;
    j.a = TileKm{reinterpret_cast<const char*>(p.a + static_cast<size_t>(r0) * p.lda + j.mt * kTileM), p.lda * 2, nrows,
                 p.M - j.mt * kTileM};
    j.b = TileKm{reinterpret_cast<const char*>(p.b + static_cast<size_t>(r0) * p.ldb + j.nt * kTileN), p.ldb * 2, nrows,
                 p.N - j.nt * kTileN};
    return j;
  };

  int lid = tile_of(blockIdx.x >> 3), next = tile_of((blockIdx.x >> 3) + slots);
  if (lid >= live_tiles) return;
  Job job = job_of(lid);
  gemm_tile_prefetch(job.a, job.b, lds);
  wait_vmcnt<0>();
  tile_barrier();
  for (;;) {
    f32x16 acc[kTileTM][kTileTN];
#pragma unroll
    for (int i = 0; i < kTileTM; ++i)
#pragma unroll
      for (int j = 0; j < kTileTN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    const bool more = next < live_tiles;
    Job nj = job;
    if (more) nj = job_of(next);
    int taken = 0;
    if (tid == 0 && more)
      taken = __hip_atomic_fetch_add(p.next + xcd, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    gemm_tile_mainloop<false, true, true, false, kTileTM, true>(TileOps{}, job.nk, bfrag, acc, lds, nullptr, &job.a, &job.b);
    wait_lgkmcnt0();
    tile_barrier();   // every wave is past the k-loop's LDS reads, and its loads have arrived
    if (more) gemm_tile_prefetch(nj.a, nj.b, lds);
    int32_t* word = reinterpret_cast<int32_t*>(&lds.a[0][1][0]);   // A's second buffer is idle until the next mainloop
    if (tid == 0) *word = taken;
    const size_t mn = static_cast<size_t>(p.M) * p.N;
    uint16_t* out = job.g < p.E ? static_cast<uint16_t*>(p.c) + job.g * mn
                                : static_cast<uint16_t*>(p.cs) + (job.g - p.E) * mn;
    // [128 rows][256 columns], 16-byte unit u of row r at u ^ 4 (r >> 2 & 1): the two halves of a wavefront, four rows
    // apart, write different banks
    uint16_t* stg = reinterpret_cast<uint16_t*>(&lds.b[1][0]);
    int after = 0;
    static_assert(128 * kTileN * 2 <= 2 * sizeof(lds.b[0]), "128 rows fit behind B's first buffer");
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int ii = 0; ii < 2; ++ii)
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
          for (int j = 0; j < kTileTN; ++j) {
            const int row = wm * 64 + ii * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
            const int col = wn * 64 + j * 32 + (lane & 31);
            stg[row * kTileN + (col ^ (row >> 2 & 1) * 32)] = f32_to_bf16(acc[2 * h + ii][j][r]);
          }
      wait_lgkmcnt0();
      if (h == 0) wait_vmcnt<0>();   // the next tile's first operands, before any store: stores are never waited for here
      tile_barrier();
#pragma unroll
      for (int q = 0; q < 8; ++q) {   // 4096 pieces of eight columns: 32 per row
        const int u = tid + kTileThreads * q;
        const int pr = u >> 5, c = (u & 31) * 8;
        const int row = job.mt * kTileM + staged_tile_row<kTileTM>(pr, h), col = job.nt * kTileN + c;
        if (row < p.M && col < p.N)
          *reinterpret_cast<u32x4*>(out + static_cast<size_t>(row) * p.N + col) =
              *reinterpret_cast<const u32x4*>(&stg[pr * kTileN + (c ^ (pr >> 2 & 1) * 32)]);
      }
      if (h == 0) after = __builtin_amdgcn_readfirstlane(*word);
      wait_lgkmcnt0();
      tile_barrier();   // the staged rows are read
    }
    if (zeros) zero_slices(dead, p.E, mn / 8, lid, live_tiles, static_cast<float*>(p.c), static_cast<float*>(p.cs));
    if (!more) return;
    lid = next;
    job = nj;
    next = tile_of(2 * slots + after);
  }
}

// Adds the slices of each split tail tile of the ROWS fp32 product in slice order and stores
// it; kTailFixParts workgroups per possible tail tile, grid 8 x kTailSlotsPerXcd x kTailFixParts.
__global__ __launch_bounds__(kTileThreads) void nt_tail_fixup(const NtArgs p) {
  const int mt_live = p.tile_off[p.G];
  const int live = mt_live * p.n_tiles;
  const int nk = p.K / kTileK;
  const int b = blockIdx.x, xcd = b & 7, t = (b >> 3) % kTailSlotsPerXcd, part = b / (8 * kTailSlotsPerXcd);
  const XcdShare x = xcd_share(xcd, live, p.cu_xcd, nk, nt_tail_split(kNtRows, kEpiF32, nk));
  if (x.s == 1 || t >= x.r) return;
  int mt, nt;
  grouped_tile_coords(x.base + x.full + t, mt_live, p.n_tiles, mt, nt);
  int lo = 0, hi = p.G;   // tile_off[lo] <= mt < tile_off[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.tile_off[mid] <= mt) lo = mid; else hi = mid;
  }
  const int row0 = p.offsets[lo] + (mt - p.tile_off[lo]) * kTileM, row_end = p.offsets[lo + 1], n0 = nt * kTileN;
  float* out = static_cast<float*>(p.c);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 4, wn = wave % 4;
  tail_fixup_part(p.part, xcd * kTailSlotsPerXcd + t * x.s, x.s, part, [&](int i, int q, float4 a0, float4 a1) {
    const float v0[4] = {a0.x, a0.y, a0.z, a0.w}, v1[4] = {a1.x, a1.y, a1.z, a1.w};
    const int c0 = n0 + wn * 64 + (lane & 31);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int row = row0 + wm * 128 + i * 32 + 8 * q + 4 * (lane >> 5) + u;
      if (row >= row_end) continue;
      if (c0 < p.N) out[static_cast<size_t>(row) * p.ldc + c0] = v0[u];
      if (c0 + 32 < p.N) out[static_cast<size_t>(row) * p.ldc + c0 + 32] = v1[u];
    }
  });
}

// dx[t, c] = sum_k dXr[inv[t K + k], c] + sum_s dXr[T K + s T + t, c], in that order.
__global__ __launch_bounds__(kBwdThreads) void dx_combine_kernel(const float* __restrict__ dxr,
                                                                 const int32_t* __restrict__ inv, int T, int K, int S,
                                                                 int d, float* __restrict__ dx) {
  const int t = blockIdx.x;
  for (int c = threadIdx.x * 4; c < d; c += kBwdThreads * 4) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < K + S; ++k) {
      const size_t row = k < K ? static_cast<size_t>(inv[t * K + k]) : static_cast<size_t>(T) * K + (k - K) * T + t;
      const float4 v = *reinterpret_cast<const float4*>(dxr + row * d + c);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    *reinterpret_cast<float4*>(dx + static_cast<size_t>(t) * d + c) = s;
  }
}

// Zero the [M, N] gradient matrices of the groups that no row reached (offsets[g+1] ==
// offsets[g]), unless the weight gradients do it (zeros_in_wgrad). Grid (G, chunks); float4 stores; M N % 4 == 0.
__global__ __launch_bounds__(kBwdThreads) void zero_unused_kernel(const int32_t* __restrict__ offsets,
                                                                  const int32_t* __restrict__ n_active, int E,
                                                                  size_t mn, float* __restrict__ c,
                                                                  float* __restrict__ cs) {
  const int g = blockIdx.x;
  if (zeros_in_wgrad(gridDim.x, n_active[0]) || offsets[g + 1] > offsets[g]) return;
  float4* dst = reinterpret_cast<float4*>(g < E ? c + g * mn : cs + (g - E) * mn);
  const size_t n4 = mn / 4;
  for (size_t i = static_cast<size_t>(blockIdx.y) * kBwdThreads + threadIdx.x; i < n4;
       i += static_cast<size_t>(gridDim.y) * kBwdThreads)
    dst[i] = make_float4(0.f, 0.f, 0.f, 0.f);
}

#define MASKMOE_TRY(x)               \
  do {                               \
    const hipError_t e_ = (x);       \
    if (e_ != hipSuccess) return e_; \
  } while (0)

// A second stream per device (default priority, created on first use and kept until the
// process ends) on which the backward writes the zero gradients of unchosen experts while the
// GEMMs run on the caller's stream. Ordered with the caller's stream by two events created per
// call.
constexpr int kMaxDevices = 64;
hipError_t side_stream(hipStream_t* out) {
  static std::mutex mu;
  static hipStream_t streams[kMaxDevices] = {};
  int dev = 0;
  MASKMOE_TRY(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (!streams[dev]) MASKMOE_TRY(hipStreamCreateWithFlags(&streams[dev], hipStreamNonBlocking));
  *out = streams[dev];
  return hipSuccess;
}

}  // namespace

BwdLayout backward_layout(int T, int d, int F, int E, int K, int S) {
  BwdLayout w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += (bytes + 255) / 256 * 256;
    return o;
  };
  (void)E;
  const size_t R = static_cast<size_t>(T) * (K + S);
  w.dout = take(R * d * 2);
  w.dab = take(R * 2 * F * 2);
  w.dxr = take(R * d * 4);
  w.xg = take(R * d * 2);
  w.part = take(kTailPartBytes);
  w.total = off;
  return w;
}

// The ROWS grid: 8 XCDs x (their largest share of the tiles + tail slices).
static dim3 rows_grid(int mt_max, int n_tiles) {
  return dim3(static_cast<unsigned>(8 * ((static_cast<long>(mt_max) * n_tiles + 7) / 8 + kTailSlotsPerXcd)));
}

// The zero gradients of the experts no token chose depend on nothing but the routing; they are
// written on a second stream beside the GEMMs, forked after the row gathers: the fill is bound
// by HBM writes like the gathers, and next to them it slowed both (gathers 0.08 -> 0.66 ms on
// the Mixtral fine-tuning layer).
hipError_t launch_layer_backward(const BwdArgs& a, hipStream_t s) {
  const int G = a.E + a.S, T = a.T, d = a.d, F = a.F, K = a.K;
  const int R = T * (K + a.S);
  const size_t FD = static_cast<size_t>(F) * d;
  const BwdLayout& w = a.lay;
  char* ws = static_cast<char*>(a.workspace);
  uint16_t* dout = reinterpret_cast<uint16_t*>(ws + w.dout);
  uint16_t* dab = reinterpret_cast<uint16_t*>(ws + w.dab);
  float* dxr = reinterpret_cast<float*>(ws + w.dxr);
  uint16_t* xg = reinterpret_cast<uint16_t*>(ws + w.xg);

  hipStream_t side;
  MASKMOE_TRY(side_stream(&side));
  hipEvent_t fork, join;
  MASKMOE_TRY(hipEventCreateWithFlags(&fork, hipEventDisableTiming));
  hipError_t e = hipEventCreateWithFlags(&join, hipEventDisableTiming);
  if (e != hipSuccess) {
    (void)hipEventDestroy(fork);
    return e;
  }
  bool forked = false;
  auto fill = [&]() {   // fork the zero fill off the caller's stream
    if (e == hipSuccess) e = hipEventRecord(fork, s);
    if (e == hipSuccess) e = hipStreamWaitEvent(side, fork, 0);
    if (e != hipSuccess) return;
    hipLaunchKernelGGL(zero_unused_kernel, dim3(G, 512), dim3(kBwdThreads), 0, side, a.pb.offsets, a.pb.n_active, a.E, FD,
                       a.d_w_down, a.d_ws_down);
    hipLaunchKernelGGL(zero_unused_kernel, dim3(G, 512), dim3(kBwdThreads), 0, side, a.pb.offsets, a.pb.n_active, a.E, 2 * FD,
                       a.d_w_gate_up, a.d_ws_gate_up);
    e = hipGetLastError();
    if (e == hipSuccess) e = hipEventRecord(join, side);
    forked = e == hipSuccess;
  };
  auto check = [&]() {
    if (e == hipSuccess) e = hipGetLastError();
  };

  // dO and the gathered tokens
  hipLaunchKernelGGL(build_dout_kernel, dim3(R), dim3(kBwdThreads), 0, s, a.dy, a.gate, a.pb.perm, a.pb.row_tok, T * K,
                     d, dout);
  hipLaunchKernelGGL(gather_rows_kernel, dim3(R), dim3(kBwdThreads), 0, s, a.x, a.pb.row_tok, d, xg);
  check();
  fill();
  // dgrad of the down projection with the SwiGLU backward: [da db] (bf16)
  NtArgs n{};
  n.offsets = a.pb.offsets;
  n.tile_off = a.pb.tile_off;
  n.G = G; n.E = a.E;
  n.mt_max = a.max_tiles;
  n.a = dout; n.lda = d;
  n.b = a.w_down; n.bs = a.ws_down; n.N = F; n.K = d; n.ldb = F;   // W_down [d, F]: K-major
  n.ab = a.ab;
  n.c = dab;
  n.n_tiles = (F + kTileN - 1) / kTileN;
  n.cu_xcd = device_cus_per_xcd();
  n.part = reinterpret_cast<float*>(ws + w.part);
  if (e == hipSuccess) {
    hipLaunchKernelGGL((gemm_nt_kernel<kNtRows, kEpiSwigluBwd>), rows_grid(n.mt_max, n.n_tiles), dim3(kTileThreads),
                       0, s, n);
    check();
  }
  // dgrad of gate/up: dX rows = [da db] W_gate_up, then the token sums
  if (e == hipSuccess) {
    n.a = dab; n.lda = 2 * F;
    n.b = a.w_gate_up; n.bs = a.ws_gate_up; n.N = d; n.K = 2 * F; n.ldb = d;   // W_gate_up [2F, d]: K-major
    n.ab = nullptr;
    n.c = dxr; n.ldc = d;
    n.n_tiles = (d + kTileN - 1) / kTileN;
    hipLaunchKernelGGL((gemm_nt_kernel<kNtRows, kEpiF32>), rows_grid(n.mt_max, n.n_tiles), dim3(kTileThreads), 0, s,
                       n);
    if (nt_tail_split(kNtRows, kEpiF32, n.K / kTileK))
      hipLaunchKernelGGL(nt_tail_fixup, dim3(8 * kTailSlotsPerXcd * kTailFixParts), dim3(kTileThreads), 0, s, n);
    hipLaunchKernelGGL(dx_combine_kernel, dim3(T), dim3(kBwdThreads), 0, s, dxr, a.pb.inv, T, K, a.S, d, a.d_x);
    check();
  }
  // weight gradients over each expert's own rows
  NtArgs m{};
  m.offsets = a.pb.offsets;
  m.active = a.pb.active;
  m.n_active = a.pb.n_active;
  m.G = G; m.E = a.E;
  if (e == hipSuccess) {   // dW_down [d, F] = dO^T h
    m.a = dout; m.lda = d; m.b = a.h; m.ldb = F; m.M = d; m.N = F;
    m.c = a.d_w_down; m.cs = a.d_ws_down;
    m.mt_max = (d + kTileM - 1) / kTileM;
    m.n_tiles = (F + kTileN - 1) / kTileN;
    hipLaunchKernelGGL((gemm_nt_kernel<kNtKSplit, kEpiF32>), dim3(G * m.mt_max * m.n_tiles), dim3(kTileThreads), 0, s,
                       m);
    check();
  }
  if (e == hipSuccess) {   // dW_gate_up [2F, d] = [da db]^T x
    m.a = dab; m.lda = 2 * F; m.b = xg; m.ldb = d; m.M = 2 * F; m.N = d;
    m.c = a.d_w_gate_up; m.cs = a.d_ws_gate_up;
    m.mt_max = (2 * F + kTileM - 1) / kTileM;
    m.n_tiles = (d + kTileN - 1) / kTileN;
    hipLaunchKernelGGL((gemm_nt_kernel<kNtKSplit, kEpiF32>), dim3(G * m.mt_max * m.n_tiles), dim3(kTileThreads), 0, s,
                       m);
    check();
  }
  if (forked) {   // the caller's stream sees the fill done
    const hipError_t je = hipStreamWaitEvent(s, join, 0);
    if (e == hipSuccess) e = je;
  }
  (void)hipEventDestroy(fork);   // released once their waits are done
  (void)hipEventDestroy(join);
  return e;
}

// The five products of the gradient of experts whose pre-activations are kept in 8-bit blocks (train_experts.hip prepares
// the rows and sums them up).
hipError_t launch_experts_backward_products(const KeptBwdArgs& a, hipStream_t s) {
  const int G = a.G, d = a.d, F = a.F;
  const size_t FD = static_cast<size_t>(F) * d;
  NtArgs n{};
  n.offsets = a.pb.offsets;
  n.tile_off = a.pb.tile_off;
  n.G = G; n.E = a.E;
  n.mt_max = a.max_tiles;
  n.cu_xcd = device_cus_per_xcd();
  n.part = a.part;
  // u = dy W_down and its epilogue
  n.a = a.dyg; n.lda = d;
  n.b = a.w_down; n.bs = a.ws_down; n.N = F; n.K = d; n.ldb = F;   // W_down [d, F]: K-major
  n.codes = a.codes;
  n.scales = a.scales;
  n.row_gate = a.row_gate;
  n.gh = a.gh;
  n.dgate_part = a.dgate_part;
  n.c = a.dab;
  n.n_tiles = (F + kTileN - 1) / kTileN;
  hipLaunchKernelGGL((gemm_nt_kernel<kNtRows, kEpiSwigluKept>), rows_grid(n.mt_max, n.n_tiles), dim3(kTileThreads), 0, s, n);
  MASKMOE_TRY(hipGetLastError());
  // rows of d_x = [da db] W_gate_up
  n.a = a.dab; n.lda = 2 * F;
  n.b = a.w_gate_up; n.bs = a.ws_gate_up; n.N = d; n.K = 2 * F; n.ldb = d;   // W_gate_up [2F, d]: K-major
  n.c = a.dxr; n.ldc = d;
  n.n_tiles = (d + kTileN - 1) / kTileN;
  hipLaunchKernelGGL((gemm_nt_kernel<kNtRows, kEpiF32>), rows_grid(n.mt_max, n.n_tiles), dim3(kTileThreads), 0, s, n);
  if (nt_tail_split(kNtRows, kEpiF32, n.K / kTileK))
    hipLaunchKernelGGL(nt_tail_fixup, dim3(8 * kTailSlotsPerXcd * kTailFixParts), dim3(kTileThreads), 0, s, n);
  MASKMOE_TRY(hipGetLastError());
  // weight gradients over each expert's own rows; zeros for the others
  NtArgs m{};
  m.offsets = a.pb.offsets;
  m.active = a.order;
  m.n_active = a.pb.n_active;
  m.G = G; m.E = a.E;
  m.a = a.dyg; m.lda = d; m.b = a.gh; m.ldb = F; m.M = d; m.N = F;   // dW_down [d, F] = dy^T (g h)
  m.c = a.d_w_down; m.cs = a.d_ws_down;
  m.mt_max = (d + kTileM - 1) / kTileM;
  m.n_tiles = (F + kTileN - 1) / kTileN;
  m.next = a.next;
  hipLaunchKernelGGL(wgrad_kernel, dim3(8 * n.cu_xcd), dim3(kTileThreads), 0, s, m);
  m.a = a.dab; m.lda = 2 * F; m.b = a.xg; m.ldb = d; m.M = 2 * F; m.N = d;   // dW_gate_up [2F, d] = [da db]^T x
  m.c = a.d_w_gate_up; m.cs = a.d_ws_gate_up;
  m.mt_max = (2 * F + kTileM - 1) / kTileM;
  m.n_tiles = (d + kTileN - 1) / kTileN;
  m.next = a.next + 8;
  hipLaunchKernelGGL(wgrad_kernel, dim3(8 * n.cu_xcd), dim3(kTileThreads), 0, s, m);
  hipLaunchKernelGGL(zero_unused_kernel, dim3(G, 512), dim3(kBwdThreads), 0, s, a.pb.offsets, a.pb.n_active, a.E, FD / 2,
                     static_cast<float*>(a.d_w_down), static_cast<float*>(a.d_ws_down));
  hipLaunchKernelGGL(zero_unused_kernel, dim3(G, 512), dim3(kBwdThreads), 0, s, a.pb.offsets, a.pb.n_active, a.E, FD,
                     static_cast<float*>(a.d_w_gate_up), static_cast<float*>(a.d_ws_gate_up));
  return hipGetLastError();
}

}  // namespace maskmoe
