// Orthogonalisation of a batch of matrices by Newton-Schulz products, and the Muon optimiser step on it.
//
//   Z_0 = U / (|U|_F + eps);    A = Z Z^T,   D = a I + b A + c A^2,   Z <- D Z        (`steps` times)
//
// with Z on its shorter side: [S, L], S <= L (tall matrices are transposed as they enter and leave).  All matrices of one
// shape, either way round, run as one batch.
//
// Products: tcgen05 kind::f16, fp32 accumulators in tensor memory, the operands in FP16 with fixed power-of-two scales that
// keep them in the middle of the format whatever S and L are:
//   Z_d = Z / sigma, sigma = 1/kf(L) (an orthogonal Z has entries of about 1/sqrt(L));   A_d = 2^12 A;   D_d = 2^12 D.
// FP16 rather than BF16 because the products run at the same rate and its 11 bits leave an eighth of the rounding error,
// which the iteration passes on to small singular values multiplied by up to 3.4 a step.
//   gram:   A_d = (sigma^2 2^12) Z_d Z_d^T            symmetric: tiles on and above the diagonal, stored twice
//   poly:   D_d = (c 2^-12) A_d A_d^T + b A_d + 2^12 a I   likewise; b A_d + .. is added to the fp32 accumulator
//   update: Z_d <- 2^-12 D_d Z_d                       Z_d is the MN-major operand: no transposed copy
// Bound: the tensor pipe for large batches (S S L + S S S + 2 S S L flops a step); for few or small matrices the latency of
// the chain of 3 `steps` products.
#include <cuda.h>
#include <math.h>

#include "scalify_common.cuh"
#include "scalify_launch.h"
#include "tcgen05_ptx.cuh"
#include "vec8.cuh"

namespace scalify {

namespace {

constexpr int kTM = 128;          // rows of the output tile per CTA
constexpr int kTN = 256;          // columns of the output tile
constexpr int kTK = 64;           // FP16 elements per K block: one 128-byte swizzle row
constexpr int kStepK = 16;        // of one MMA
constexpr int kAccs = 2;          // accumulators of 256 TMEM columns: the epilogue overlaps the next tile's products
constexpr int kEpiWarpsM = 8;
constexpr int kNsThreads = 64 + 32 * kEpiWarpsM;
constexpr int kTile16 = 32 * 64;  // bytes of a 32 x 32 FP16 tile
constexpr float kGramScale = 4096.0f;

constexpr int kMaxInst = 96;      // matrices per batch (their descriptors travel as a kernel argument)
constexpr int kMaxParts = 64;     // partial sums of a matrix's norm
constexpr int kPreTile = 64;      // rows and columns of a tile of the element-wise passes

enum { kGram = 0, kPoly = 1, kUpdate = 2 };

// Two CTAs (an SM pair) share a 256 x 256 tile; one CTA alone takes 128 x 256 where S fits 128 rows.
template <int NCTA> struct NsCfg {
  static constexpr int kTileM = kTM * NCTA;
  static constexpr int kBRows = kTN / NCTA;  // rows (or columns of an MN-major operand) of B staged per CTA
  static constexpr int kABytes = kTM * 128;
  static constexpr int kBBytes = kBRows * 128;
  static constexpr int kStages = NCTA == 1 ? 3 : 5;
  static constexpr int kEpiBytes = kEpiWarpsM * 4 * kTile16;  // per warp: two tiles, straight and transposed
  static constexpr size_t kSmem = size_t(kStages) * (kABytes + kBBytes) + kEpiBytes + 1024 + 256;
};

struct NsParams {
  int S, N, K, batch;        // output [S, N], contraction K
  int tiles_m, tiles_n, tiles;  // tiles of one matrix (symmetric: on and above the diagonal)
  uint32_t idesc;
  float alpha, b, diag;      // out = alpha acc (+ b A_d[r, c] + diag [r == c])
  const __half* A;           // poly: A_d [batch][S][ld]
  long long ld;
  uint32_t* status;
};

__device__ __forceinline__ void umma_f16(uint32_t d_tmem, uint64_t ad, uint64_t bd, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(ad), "l"(bd), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void umma_f16_pair(uint32_t d_tmem, uint64_t ad, uint64_t bd, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(ad), "l"(bd), "r"(idesc), "r"(acc) : "memory");
}

// tile index -> matrix, tile row and column (symmetric products: row by row of the upper triangle)
template <int MODE>
__device__ __forceinline__ void ns_tile(const NsParams& p, int tile, int& b, int& mt, int& nt) {
  b = tile / p.tiles;
  int t = tile - b * p.tiles;
  if constexpr (MODE == kUpdate) {
    nt = t / p.tiles_m;
    mt = t - nt * p.tiles_m;
  } else {
    mt = 0;
    while (t >= p.tiles_n - mt) { t -= p.tiles_n - mt; ++mt; }
    nt = mt + t;
  }
}

}  // namespace

// Warp 0: TMA producer; warp 1: MMA issuer; warps 2-9: epilogue.  Persistent CTAs (pairs).  Every wait is bounded; on
// expiry the CTA records SCALIFY_DEV_TIMEOUT, drains its copies and MMAs, frees its tensor memory and returns.
template <int MODE, int NCTA>
__global__ void __launch_bounds__(kNsThreads, 1) ns_product_kernel(const __grid_constant__ CUtensorMap map_a,
                                                                  const __grid_constant__ CUtensorMap map_b,
                                                                  const __grid_constant__ CUtensorMap map_y, const NsParams p) {
  using C = NsCfg<NCTA>;
  constexpr int kStages = C::kStages;
  asm volatile("griddepcontrol.launch_dependents;");  // the next product may set up while this one runs
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw);
  const uint32_t smem_a = base, smem_b = base + kStages * C::kABytes;
  constexpr uint32_t kRing = kStages * (C::kABytes + C::kBBytes);
  uint8_t* epi_mem = smem + kRing;
  uint8_t* bar_mem = epi_mem + C::kEpiBytes;
  const uint32_t bars = base + kRing + C::kEpiBytes;
  const uint32_t full_bar = bars, empty_bar = bars + 8 * kStages, acc_full = bars + 16 * kStages, acc_empty = acc_full + 8 * kAccs,
                 drain_bar = acc_empty + 8 * kAccs;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(bar_mem + 16 * kStages + 16 * kAccs + 8);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = NCTA == 2 ? cluster_ctarank() : 0u;
  const int unit = blockIdx.x / NCTA, num_units = gridDim.x / NCTA;
  const int num_kb = (p.K + kTK - 1) / kTK, num_tiles = p.tiles * p.batch;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(full_bar + 8 * s, 1); mbar_init(empty_bar + 8 * s, 1); }
    for (int s = 0; s < kAccs; ++s) { mbar_init(acc_full + 8 * s, 1); mbar_init(acc_empty + 8 * s, kEpiWarpsM * NCTA); }
    mbar_init(drain_bar, 1);
    *abort_flag = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kAccs * kTN);
  tc_fence_before();
  __syncthreads();
  if constexpr (NCTA == 2) cluster_sync_all();
  tc_fence_after();
  asm volatile("griddepcontrol.wait;" ::: "memory");  // nothing above touches global memory
  const uint32_t tmem_base = *tmem_slot;
  bool timed_out = false;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      long long issued = 0;
      for (int tile = unit; tile < num_tiles && !timed_out; tile += num_units) {
        int b, mt, nt;
        ns_tile<MODE>(p, tile, b, mt, nt);
        const int m0 = mt * C::kTileM + static_cast<int>(rank) * kTM;
        const int n0 = nt * kTN + static_cast<int>(rank) * C::kBRows * (NCTA - 1);
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait(empty_bar + 8 * stage, phase ^ 1u, abort_flag)) { timed_out = true; break; }
          const uint32_t sa = smem_a + stage * C::kABytes, sb = smem_b + stage * C::kBBytes;
          const int kx = kb * kTK * 2;  // byte coordinate of the K block
          uint32_t fb = full_bar + 8 * stage;
          if constexpr (NCTA == 2) {
            if (rank == 0u) mbar_expect_tx(fb, 2 * (C::kABytes + C::kBBytes));
            fb = map_to_cta(fb, 0u);  // both CTAs' copies are counted on the leader's barrier
            tma_load_3d_pair(sa, &map_a, fb, kx, m0, b);
            if constexpr (MODE == kUpdate) {
#pragma unroll
              for (int j = 0; j < C::kBRows / kTK; ++j) tma_load_3d_pair(sb + j * kTK * 128, &map_b, fb, (n0 + j * kTK) * 2, kb * kTK, b);
            } else {
              tma_load_3d_pair(sb, &map_b, fb, kx, n0, b);
            }
          } else {
            mbar_expect_tx(fb, C::kABytes + C::kBBytes);
            tma_load_3d(sa, &map_a, fb, kx, m0, b);
            if constexpr (MODE == kUpdate) {
#pragma unroll
              for (int j = 0; j < C::kBRows / kTK; ++j) tma_load_3d(sb + j * kTK * 128, &map_b, fb, (n0 + j * kTK) * 2, kb * kTK, b);
            } else {
              tma_load_3d(sb, &map_b, fb, kx, n0, b);
            }
          }
          ++issued;
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if ((timed_out || *abort_flag) && rank == 0u) {
        // wait (bounded) for the last use of every ring slot, so that no copy is in flight when the CTA (pair) exits
        const int pending = issued < kStages ? static_cast<int>(issued) : kStages;
        uint32_t s = stage, ph = phase;
        for (int i = 0; i < pending; ++i) {
          if (s == 0) { s = kStages - 1; ph ^= 1u; } else { --s; }
          const unsigned long long t0 = global_timer_ns();
          while (!mbar_try_wait(full_bar + 8 * s, ph) && global_timer_ns() - t0 < kWaitLimitNs) {}
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0u) {
      uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
      // MN-major B: atoms of 64 columns x 8 rows of K; along K they are 1024 bytes apart, the next 64 columns a K block's
      // box (64 x 128 bytes) further on
      const uint64_t a_desc0 = make_smem_desc(smem_a, 0u, 1024u);
      const uint64_t b_desc0 = make_smem_desc(smem_b, MODE == kUpdate ? kTK * 128u : 0u, 1024u);
      constexpr uint32_t a_inc = kStepK * 2 >> 4, b_inc = MODE == kUpdate ? (kStepK * 128 >> 4) : (kStepK * 2 >> 4);
      for (int tile = unit; tile < num_tiles && !timed_out; tile += num_units) {
        if (!mbar_wait(acc_empty + 8 * acc, acc_phase ^ 1u, abort_flag)) { timed_out = true; break; }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + acc * kTN;
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait(full_bar + 8 * stage, phase, abort_flag)) { timed_out = true; break; }
          tc_fence_after();
          const uint64_t ad0 = a_desc0 + static_cast<uint64_t>(stage * (C::kABytes >> 4));
          const uint64_t bd0 = b_desc0 + static_cast<uint64_t>(stage * (C::kBBytes >> 4));
#pragma unroll
          for (int k = 0; k < kTK / kStepK; ++k) {
            if constexpr (NCTA == 1) umma_f16(d_tmem, ad0 + k * a_inc, bd0 + k * b_inc, p.idesc, (kb | k) != 0 ? 1u : 0u);
            else umma_f16_pair(d_tmem, ad0 + k * a_inc, bd0 + k * b_inc, p.idesc, (kb | k) != 0 ? 1u : 0u);
          }
          if constexpr (NCTA == 1) umma_commit(empty_bar + 8 * stage);
          else umma_commit_pair(empty_bar + 8 * stage);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        if (timed_out) break;
        if constexpr (NCTA == 1) umma_commit(acc_full + 8 * acc);
        else umma_commit_pair(acc_full + 8 * acc);
        if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
      }
      if (timed_out || *abort_flag) {
        if constexpr (NCTA == 1) umma_commit(drain_bar);
        else umma_commit_pair(drain_bar);
        const unsigned long long t0 = global_timer_ns();
        while (!mbar_try_wait(drain_bar, 0u) && global_timer_ns() - t0 < kWaitLimitNs) {}
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 2) / 4;  // TMEM lane quarter, half of the tile's columns
    constexpr int kChunks = kTN / 64;               // 32-column chunks per warp
    uint8_t* stage_mem = epi_mem + (warp - 2) * 4 * kTile16;
    uint32_t acc = 0, acc_phase = 0, buf = 0;
    for (int tile = unit; tile < num_tiles; tile += num_units) {
      int b, mt, nt;
      ns_tile<MODE>(p, tile, b, mt, nt);
      if (!mbar_wait(acc_full + 8 * acc, acc_phase, abort_flag)) { timed_out = true; break; }
      tc_fence_after();
      const int c_first = half * kChunks, n0 = nt * kTN;
      const int n_chunks = max(0, min(kChunks, (p.N - n0 + 31) / 32 - c_first));  // chunks inside the matrix
      const uint32_t t_addr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * kTN + c_first * 32;
      const int row0 = mt * C::kTileM + static_cast<int>(rank) * kTM + q * 32, row = row0 + lane;
      const bool mirror = MODE != kUpdate && mt != nt;
      const __half* arow = nullptr;
      if constexpr (MODE == kPoly) arow = p.A + (static_cast<long long>(b) * p.S + min(row, p.S - 1)) * p.ld;
      uint32_t r[32];
#pragma unroll 1
      for (int c = 0; c < n_chunks; ++c) {
        const int col0 = n0 + (c_first + c) * 32;
        uint32_t wa[16];
        tmem_ld32(t_addr + c * 32, r);
        if constexpr (MODE == kPoly) {  // (the row's padding makes whole chunks readable)
#pragma unroll
          for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4*>(wa + 4 * j) = *reinterpret_cast<const uint4*>(arow + col0 + 8 * j);
        }
        tmem_ld_wait();
        if (c + 1 == n_chunks) {  // the accumulator has been read: the next tile may overwrite it
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if constexpr (NCTA == 1) mbar_arrive(acc_empty + 8 * acc);
            else mbar_arrive_cluster(map_to_cta(acc_empty + 8 * acc, 0u));
          }
        }
        uint32_t o[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          float x = __uint_as_float(r[2 * j]) * p.alpha, y = __uint_as_float(r[2 * j + 1]) * p.alpha;
          if constexpr (MODE == kPoly) {
            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&wa[j]));
            x = fmaf(p.b, t.x, x) + (row == col0 + 2 * j ? p.diag : 0.f);
            y = fmaf(p.b, t.y, y) + (row == col0 + 2 * j + 1 ? p.diag : 0.f);
          }
          const __half2 hh = __floats2half2_rn(x, y);
          o[j] = *reinterpret_cast<const uint32_t*>(&hh);
        }
        if (lane == 0) bulk_wait_read<1>();  // the stores that used this buffer two chunks ago have read it
        __syncwarp();
        uint8_t* t_straight = stage_mem + buf * 2 * kTile16;
        uint8_t* t_mirror = t_straight + kTile16;
        uint4* ts = reinterpret_cast<uint4*>(t_straight);  // rows of 64 bytes, 16-byte pieces in the 64-byte swizzle
#pragma unroll
        for (int j = 0; j < 4; ++j) ts[lane * 4 + (j ^ ((lane >> 1) & 3))] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
        if (mirror) {  // element (row, col) to line col of the transposed tile
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const uint16_t v16 = static_cast<uint16_t>(o[j / 2] >> (16 * (j & 1)));
            *reinterpret_cast<uint16_t*>(t_mirror + j * 64 + (((lane >> 3) ^ ((j >> 1) & 3)) << 4) + (lane & 7) * 2) = v16;
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (row0 < p.S) tma_store_3d(&map_y, smem_u32(t_straight), col0 * 2, row0, b);
          if (mirror && row0 < p.S) tma_store_3d(&map_y, smem_u32(t_mirror), row0 * 2, col0, b);
          bulk_commit();
        }
        buf ^= 1u;
      }
      if (n_chunks == 0) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (NCTA == 1) mbar_arrive(acc_empty + 8 * acc);
          else mbar_arrive_cluster(map_to_cta(acc_empty + 8 * acc, 0u));
        }
      }
      if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
    }
    if (lane == 0) bulk_wait_all();
  }
  if (timed_out) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_TIMEOUT));
  tc_fence_before();
  __syncthreads();
  if constexpr (NCTA == 2) cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kAccs * kTN);
  }
}

// ------------------------------------------------------------------------------------------------- element-wise passes
namespace {

struct MuonTable {
  MuonTensor t[kMaxInst];
};

// What the static scale rules make of a tensor's scale words; m_s == 0: no momentum.
struct MuonFactors {
  float fm, fg;        // m'_d = fm m_d + fg g_d
  float fw, fo;        // w'_d = fw w_d - fo Z_d
  float m_s, w_s;      // the new scale words
};

struct MuonPass {
  MuonFactors* factors;   // [matrix]
  double* partial;        // [matrix][kMaxParts] sums of squares of u_d
  int parts;
  __half* Z;              // [matrix][S][ld]
  long long ld;
  float momentum, one_minus, p2_m, p2_1m;
  float eps, inv_sigma, sigma, decay;
  float lr[2], p2_lr[2];  // lr * factor of wide (and square) matrices, of tall ones
  int nesterov, S, L;
  uint32_t* status;
};

__device__ __forceinline__ MuonFactors muon_factors(const MuonTensor& t, const MuonPass& p, bool* bad) {
  MuonFactors f;
  const float gs = load_scale(t.g_scale);
  *bad = !is_pow2_scale(gs);
  if (!t.m) {
    f.fm = 0.f; f.fg = 1.0f; f.fw = 0.f; f.fo = 0.f; f.m_s = 0.f; f.w_s = p.sigma;
    return f;
  }
  const float ms = *t.m_scale, ws = *t.w_scale;
  *bad = *bad || !is_pow2_scale(ms) || !is_pow2_scale(ws);
  f.m_s = fmaxf(p.p2_m * ms, p.p2_1m * gs);
  f.fm = p.momentum * (ms / f.m_s);
  f.fg = p.one_minus * (gs / f.m_s);
  const int tall = t.rows > t.cols ? 1 : 0;
  f.w_s = fmaxf(ws, p.p2_lr[tall] * p.sigma);
  f.fw = (1.0f - p.decay) * (ws / f.w_s);
  f.fo = p.lr[tall] * (p.sigma / f.w_s);
  return f;
}

// u_d of one vector (and m'_d): u is the momentum, or its Nesterov form, in units of m'_s
__device__ __forceinline__ void muon_vec(const MuonTensor& t, const MuonPass& p, const MuonFactors& f, int64_t row, int v, int n,
                                         float* u, float* m) {
  float g[kVec];
  SCALIFY_DISPATCH_DTYPE(t.g_dt, DT, {
    uint32_t w[kVec * ElemBytes<DT>::v / 4];
    load_vec<DT>(static_cast<const char*>(t.g) + row * t.g_ld * ElemBytes<DT>::v, v, n, w);
    decode_vec<DT, kVec>(w, g);
  })
  if (!t.m) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) u[e] = g[e];
    return;
  }
  if (t.m_dt == SCALIFY_F16) {
    uint32_t w[4];
    load_vec<SCALIFY_F16>(static_cast<const char*>(t.m) + row * t.m_ld * 2, v, n, w);
    decode_vec<SCALIFY_F16, kVec>(w, m);
  } else {
    uint32_t w[8];
    load_vec<SCALIFY_F32>(static_cast<const char*>(t.m) + row * t.m_ld * 4, v, n, w);
    decode_vec<SCALIFY_F32, kVec>(w, m);
  }
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    const float gg = f.fg * g[e];
    m[e] = fmaf(f.fm, m[e], gg);
    u[e] = p.nesterov ? fmaf(p.momentum, m[e], gg) : m[e];
  }
}

}  // namespace

// |u|_F^2, one partial per block (fixed order within and between blocks), and the step's factors.
__global__ void __launch_bounds__(256) muon_norm_kernel(const __grid_constant__ MuonTable tab, const MuonPass p) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  __shared__ double s_sum[8];
  const int inst = blockIdx.y;
  const MuonTensor& t = tab.t[inst];
  bool bad;
  const MuonFactors f = muon_factors(t, p, &bad);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.factors[inst] = f;
    if (bad) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_SCALE));
  }
  const uint32_t nv = (t.cols + kVec - 1) / kVec, total = nv * static_cast<uint32_t>(t.rows);
  double sum = 0.0;
  for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < total; i += gridDim.x * 256u) {
    const uint32_t row = i / nv;
    const int v = static_cast<int>(i - row * nv);
    float u[kVec], m[kVec], ss = 0.f;
    muon_vec(t, p, f, row, v, t.cols - v * kVec, u, m);
#pragma unroll
    for (int e = 0; e < kVec; ++e) ss = fmaf(u[e], u[e], ss);
    sum += ss;
  }
  sum = warp_sum_f64(sum);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int k = 0; k < 8; ++k) sum += s_sum[k];
    p.partial[inst * kMaxParts + blockIdx.x] = sum;
  }
}

// m' (stored once rounded) and Z_0 = u / (|u| + eps) / sigma in FP16, [S, L]; a 64 x 64 tile per block, turned over in shared
// memory where the matrix is tall.  The new scale words are written here (nothing of this launch reads the old ones).
__global__ void __launch_bounds__(256) muon_momentum_kernel(const __grid_constant__ MuonTable tab, const MuonPass p) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  __shared__ __align__(16) __half s_tile[kPreTile][kPreTile + 8];
  __shared__ float s_scale;
  const int inst = blockIdx.z;
  const MuonTensor& t = tab.t[inst];
  const int tiles_x = (t.cols + kPreTile - 1) / kPreTile;
  const int r0 = blockIdx.x / tiles_x * kPreTile, c0 = blockIdx.x % tiles_x * kPreTile;
  const bool tall = t.rows > t.cols;
  if (threadIdx.x < 32) {
    double s = 0.0;
    for (int i = threadIdx.x; i < p.parts; i += 32) s += p.partial[inst * kMaxParts + i];
    s = warp_sum_f64(s);
    if (threadIdx.x == 0) s_scale = p.inv_sigma / (static_cast<float>(sqrt(s)) + p.eps);
    if (threadIdx.x == 0 && blockIdx.x == 0) {
      const MuonFactors f = p.factors[inst];
      if (t.m) *t.m_scale = f.m_s;
      if (t.w_scale) *t.w_scale = f.w_s;
      if (t.wc_scale) *t.wc_scale = f.w_s;
      if (!(sqrt(s) < 3.4e38)) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_NONFINITE_STAT));
    }
  }
  const MuonFactors f = p.factors[inst];
  __syncthreads();
  const float scale = s_scale;
  __half* Z = p.Z + static_cast<long long>(inst) * p.S * p.ld;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = threadIdx.x + k * 256, lr = i >> 3, lv = i & 7;
    const int row = r0 + lr, col = c0 + lv * kVec, n = t.cols - col;
    if (row < t.rows && n > 0) {
      float u[kVec], m[kVec];
      muon_vec(t, p, f, row, col / kVec, n, u, m);
      if (t.m) {
        if (t.m_dt == SCALIFY_F16) store_vec<SCALIFY_F16>(static_cast<char*>(t.m) + static_cast<int64_t>(row) * t.m_ld * 2, col / kVec, n, m);
        else store_vec<SCALIFY_F32>(static_cast<char*>(t.m) + static_cast<int64_t>(row) * t.m_ld * 4, col / kVec, n, m);
      }
#pragma unroll
      for (int e = 0; e < kVec; ++e) u[e] *= scale;
      if (!tall) {  // (rows of Z are padded to whole vectors)
        uint32_t w[4];
        encode_vec<SCALIFY_F16, kVec>(u, w);
        st_raw<16>(Z + row * p.ld + col, w);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) s_tile[lv * kVec + e][lr] = __float2half_rn(u[e]);
      }
    }
  }
  if (!tall) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = threadIdx.x + k * 256, lr = i >> 3, lv = i & 7;  // line lr of the turned tile: column c0 + lr
    if (c0 + lr < t.cols && r0 + lv * kVec < t.rows) {
      uint32_t w[4];
      *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(&s_tile[lr][lv * kVec]);
      st_raw<16>(Z + static_cast<long long>(c0 + lr) * p.ld + r0 + lv * kVec, w);
    }
  }
}

// w' = fw w - fo Z (and its copy), or the orthogonal matrix itself.
__global__ void __launch_bounds__(256) muon_update_kernel(const __grid_constant__ MuonTable tab, const MuonPass p) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  __shared__ __align__(16) __half s_tile[kPreTile][kPreTile + 8];
  const int inst = blockIdx.z;
  const MuonTensor& t = tab.t[inst];
  const int tiles_x = (t.cols + kPreTile - 1) / kPreTile;
  const int r0 = blockIdx.x / tiles_x * kPreTile, c0 = blockIdx.x % tiles_x * kPreTile;
  const bool tall = t.rows > t.cols;
  const MuonFactors f = p.factors[inst];
  const __half* Z = p.Z + static_cast<long long>(inst) * p.S * p.ld;
  if (tall) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = threadIdx.x + k * 256, lr = i >> 3, lv = i & 7;
      if (c0 + lr < t.cols && r0 + lv * kVec < t.rows) {
        uint32_t w[4];
        ld_raw<16>(Z + static_cast<long long>(c0 + lr) * p.ld + r0 + lv * kVec, w);
        *reinterpret_cast<uint4*>(&s_tile[lr][lv * kVec]) = *reinterpret_cast<const uint4*>(w);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = threadIdx.x + k * 256, lr = i >> 3, lv = i & 7;
    const int row = r0 + lr, col = c0 + lv * kVec, n = t.cols - col;
    if (row < t.rows && n > 0) {
      float z[kVec];
      if (!tall) {
        uint32_t w[4];
        ld_raw<16>(Z + row * p.ld + col, w);
        decode_vec<SCALIFY_F16, kVec>(w, z);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) z[e] = __half2float(s_tile[lv * kVec + e][lr]);
      }
      SCALIFY_DISPATCH_WIDE(t.w_dt, DT, {
        char* wrow = static_cast<char*>(t.w) + static_cast<int64_t>(row) * t.w_ld * ElemBytes<DT>::v;
        if (t.m) {
          uint32_t w[kVec * ElemBytes<DT>::v / 4];
          float x[kVec];
          load_vec<DT>(wrow, col / kVec, n, w);
          decode_vec<DT, kVec>(w, x);
#pragma unroll
          for (int e = 0; e < kVec; ++e) z[e] = round_through<DT>(fmaf(f.fw, x[e], -f.fo * z[e]));
        }
        store_vec<DT>(wrow, col / kVec, n, z);
      })
      if (t.wc) {
        SCALIFY_DISPATCH_DTYPE(t.wc_dt, DT, store_vec<DT>(static_cast<char*>(t.wc) + static_cast<int64_t>(row) * t.wc_ld * ElemBytes<DT>::v,
                                                          col / kVec, n, z))
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------- launches
template <int MODE, int NCTA>
static int launch_product_variant(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& y, const NsParams& p, cudaStream_t st) {
  using C = NsCfg<NCTA>;
  auto kernel = ns_product_kernel<MODE, NCTA>;
  static DeviceOnce once;
  int most = 0;  // CTAs or CTA pairs that fit the GPU
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = NCTA; attrs[1].val.clusterDim.y = 1; attrs[1].val.clusterDim.z = 1;
  int rc = device_once(once, &most, [&](int* value) {
    SCALIFY_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(C::kSmem)));
    *value = sm_count();
    if (NCTA == 2) {
      cudaLaunchConfig_t qc = {};
      qc.gridDim = dim3(unsigned(sm_count() / 2 * 2)); qc.blockDim = dim3(kNsThreads); qc.dynamicSmemBytes = C::kSmem;
      qc.attrs = attrs + 1; qc.numAttrs = 1;
      int n = 0;
      SCALIFY_CUDA_TRY(cudaOccupancyMaxActiveClusters(&n, kernel, &qc));
      if (n < 1) return int(SCALIFY_ERR_UNSUPPORTED);
      *value = n;
    }
    return int(SCALIFY_OK);
  });
  if (rc) return rc;
  const long long tiles = static_cast<long long>(p.tiles) * p.batch;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((tiles < most ? tiles : most) * NCTA));
  cfg.blockDim = dim3(kNsThreads); cfg.dynamicSmemBytes = C::kSmem; cfg.stream = st;
  cfg.attrs = attrs; cfg.numAttrs = NCTA == 2 ? 2 : 1;
  SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a, b, y, p));
  return SCALIFY_OK;
}

struct NsMatrix { __half* p; int rows, cols; long long ld; };  // [batch][rows][ld]

// Y = A B^T (gram, poly: B is [N, K]) or A B (update: B is [K, N])
template <int MODE>
static int launch_product(const NsMatrix& A, const NsMatrix& B, const NsMatrix& Y, NsParams p, cudaStream_t st) {
  const int ncta = Y.rows > kTM ? 2 : 1, tile_m = kTM * ncta;
  auto map = [&](CUtensorMap* m, const NsMatrix& x, uint32_t box_bytes, uint32_t box_rows) {
    return make_byte_map(m, x.p, static_cast<uint64_t>(x.cols) * 2, x.rows, p.batch, x.ld * 2, static_cast<uint64_t>(x.rows) * x.ld * 2,
                         box_bytes, box_rows);
  };
  CUtensorMap ma, mb, my;
  int rc = map(&ma, A, 128, kTM);
  if (!rc) rc = map(&mb, B, 128, MODE == kUpdate ? kTK : kTN / ncta);
  if (!rc) rc = map(&my, Y, 64, 32);
  if (rc) return rc;
  p.S = Y.rows; p.N = Y.cols; p.K = A.cols;
  p.tiles_m = (Y.rows + tile_m - 1) / tile_m;
  p.tiles_n = (Y.cols + kTN - 1) / kTN;
  // symmetric products: the tile is square for CTA pairs; a single CTA's tile holds the whole matrix (S <= 128)
  p.tiles = MODE == kUpdate ? p.tiles_m * p.tiles_n : p.tiles_n * (p.tiles_n + 1) / 2;
  p.idesc = (1u << 4) | (uint32_t(MODE == kUpdate) << 16) | (uint32_t(kTN >> 3) << 17) | (uint32_t(tile_m >> 4) << 24);
  if (ncta == 2) return launch_product_variant<MODE, 2>(ma, mb, my, p, st);
  return launch_product_variant<MODE, 1>(ma, mb, my, p, st);
}

static long long pad64(long long n) { return (n + 63) / 64 * 64; }
struct BatchShape { int S, L; };
static BatchShape shape_of(const MuonTensor& t) { return t.rows <= t.cols ? BatchShape{t.rows, t.cols} : BatchShape{t.cols, t.rows}; }
static size_t matrix_bytes(BatchShape s) {  // two iterates, A and D
  return 4 * static_cast<size_t>(s.S) * static_cast<size_t>(pad64(s.L) + pad64(s.S));
}
constexpr size_t kMuonFixed = kWsHeader + (kMaxInst * sizeof(MuonFactors) + 255) / 256 * 256 + kMaxInst * kMaxParts * sizeof(double);

// Matrices of the i-th one's shape among t[i..n), kMaxInst at most, starting after `skip` of them; out == nullptr: count only
static int gather(int n, const MuonTensor* t, int i, int skip, MuonTable* out) {
  const BatchShape s = shape_of(t[i]);
  int count = 0;
  for (int k = i; k < n; ++k) {
    const BatchShape o = shape_of(t[k]);
    if (o.S != s.S || o.L != s.L) continue;
    if (skip-- > 0) continue;
    if (out) out->t[count] = t[k];
    if (++count == kMaxInst) break;
  }
  return count;
}
static bool first_of_shape(const MuonTensor* t, int i) {
  const BatchShape s = shape_of(t[i]);
  for (int k = 0; k < i; ++k) {
    const BatchShape o = shape_of(t[k]);
    if (o.S == s.S && o.L == s.L) return false;
  }
  return true;
}

size_t muon_ws_bytes(int n, const MuonTensor* t) {
  size_t most = 0;
  for (int i = 0; i < n; ++i) {
    if (!first_of_shape(t, i)) continue;
    const size_t b = gather(n, t, i, 0, nullptr) * matrix_bytes(shape_of(t[i]));
    if (b > most) most = b;
  }
  return kMuonFixed + most + 256;
}

static float host_p2(double c) {
  int ex;
  frexp(c, &ex);
  return static_cast<float>(ldexp(1.0, ex - 1));
}

static int run_batch(const MuonTable& tab, int count, const MuonHyper& h, void* ws, cudaStream_t st) {
  WsView view = ws_view(ws);
  const BatchShape s = shape_of(tab.t[0]);
  char* mem = static_cast<char*>(ws) + kMuonFixed;
  const long long ldz = pad64(s.L), lda = pad64(s.S);
  NsMatrix z[2], A, D;
  for (int k = 0; k < 2; ++k) {
    z[k] = NsMatrix{reinterpret_cast<__half*>(mem), s.S, s.L, ldz};
    mem += static_cast<size_t>(count) * s.S * ldz * 2;
  }
  A = NsMatrix{reinterpret_cast<__half*>(mem), s.S, s.S, lda};
  mem += static_cast<size_t>(count) * s.S * lda * 2;
  D = NsMatrix{reinterpret_cast<__half*>(mem), s.S, s.S, lda};

  MuonPass p = {};
  p.factors = static_cast<MuonFactors*>(view.area);
  p.partial = reinterpret_cast<double*>(static_cast<char*>(ws) + kMuonFixed - kMaxInst * kMaxParts * sizeof(double));
  const long long vecs = static_cast<long long>(s.S) * ((s.L + kVec - 1) / kVec);
  long long parts = (vecs + 256 * 8 - 1) / (256 * 8);
  p.parts = static_cast<int>(parts < 1 ? 1 : parts > kMaxParts ? kMaxParts : parts);
  p.Z = z[0].p;
  p.ld = ldz;
  p.momentum = h.momentum;
  p.one_minus = static_cast<float>(1.0 - static_cast<double>(h.momentum));
  p.p2_m = h.momentum > 0.f ? host_p2(h.momentum) : 0.f;
  p.p2_1m = host_p2(1.0 - static_cast<double>(h.momentum));
  p.eps = h.eps;
  p.sigma = 1.0f / kfactor(s.L);
  p.inv_sigma = kfactor(s.L);
  p.decay = h.decay;
  p.nesterov = h.nesterov;
  p.S = s.S; p.L = s.L;
  p.status = view.status;
  for (int tall = 0; tall < 2; ++tall) {
    double kappa = 1.0;
    if (h.factor == SCALIFY_MUON_SPECTRAL && tall) kappa = sqrt(static_cast<double>(s.L) / s.S);
    else if (h.factor == SCALIFY_MUON_RMS) kappa = 0.2 * sqrt(static_cast<double>(s.L));
    p.lr[tall] = static_cast<float>(static_cast<double>(h.lr) * kappa);
    p.p2_lr[tall] = p.lr[tall] > 0.f ? host_p2(p.lr[tall]) : 0.f;
  }

  muon_norm_kernel<<<dim3(p.parts, count), 256, 0, st>>>(tab, p);
  SCALIFY_CUDA_TRY(cudaGetLastError());
  const unsigned tl = static_cast<unsigned>((s.L + kPreTile - 1) / kPreTile), ts = static_cast<unsigned>((s.S + kPreTile - 1) / kPreTile);
  const dim3 tiles(tl * ts, 1, count);
  muon_momentum_kernel<<<tiles, 256, 0, st>>>(tab, p);
  SCALIFY_CUDA_TRY(cudaGetLastError());

  NsParams np = {};
  np.batch = count;
  np.status = view.status;
  int cur = 0;
  for (int k = 0; k < h.steps; ++k) {
    NsParams q = np;
    q.alpha = p.sigma * p.sigma * kGramScale;
    int rc = launch_product<kGram>(z[cur], z[cur], A, q, st);
    if (rc) return rc;
    q.alpha = h.c / kGramScale;
    q.b = h.b;
    q.diag = h.a * kGramScale;
    q.A = A.p;
    q.ld = lda;
    rc = launch_product<kPoly>(A, A, D, q, st);
    if (rc) return rc;
    q = np;
    q.alpha = 1.0f / kGramScale;
    rc = launch_product<kUpdate>(D, z[cur], z[cur ^ 1], q, st);
    if (rc) return rc;
    cur ^= 1;
  }
  p.Z = z[cur].p;
  muon_update_kernel<<<tiles, 256, 0, st>>>(tab, p);
  SCALIFY_CUDA_TRY(cudaGetLastError());
  return SCALIFY_OK;
}

int launch_muon(int n, const MuonTensor* t, const MuonHyper& h, void* ws, cudaStream_t st) {
  MuonTable tab;
  for (int i = 0; i < n; ++i) {
    if (!first_of_shape(t, i)) continue;
    for (int done = 0;;) {
      const int count = gather(n, t, i, done, &tab);
      if (count == 0) break;
      const int rc = run_batch(tab, count, h, ws, st);
      if (rc) return rc;
      done += count;
    }
  }
  return SCALIFY_OK;
}

}  // namespace scalify
