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
// which the iteration passes on to small singular values multiplied by up to 3.4 a step: five steps turn the 2^-12 of a
// rounding into 0.1 to 0.15 of absolute error in the Frobenius norm, whatever the matrix is (768 x 2304: rank 1 0.10, rank 64
// 0.15, each of its directions at most 0.016), which is 1e-3 of a full-rank result and 0.15 of one of rank 1.  Low FP16 halves
// of Z, A and D beside the high ones take that away and cost 1.8 to 2.2 times the call (three products for one; measured).
//   gram:   A_d = (sigma^2 2^12) Z_d Z_d^T            symmetric: tiles on and above the diagonal
//   poly:   D_d = (c 2^-12) A_d A_d^T + b A_d + 2^12 a I   likewise; b A_d + .. is added to the fp32 accumulator
//   update: Z_d <- 2^-12 D_d Z_d                       Z_d is the MN-major operand: no transposed copy
// The blocks of A and D below the diagonal are not stored: they are read as MN-major operands from above it (the layout is a
// matter of each K block's copies and descriptors).  Storing them as mirror images was slower at every size, in turns on one
// GPU: 4 x 8192 x 2048 1.2 %, 96 x 1024 x 1024 2.6, 8 x 1280 x 2560 3.8, 12 x 768 x 2304 4.0, 48 x 768 x 768 6.9, 16 x 768 x 768 10.
// Bound: the tensor pipe for large batches (S S L + S S S + 2 S S L flops a step); for few or small matrices the latency of
// the chain of 3 `steps` products, which then runs as ONE launch (ns_chain_kernel).
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
constexpr float kGramScale = 4096.0f;

constexpr int kMaxInst = 96;      // matrices per batch (their descriptors travel as a kernel argument)
constexpr int kMaxParts = 256;    // partial sums of a matrix's norm
constexpr int kPreTile = 64;      // rows and columns of a tile of the element-wise passes

enum { kGram = 0, kPoly = 1, kUpdate = 2 };
template <int K> struct KindC { static constexpr int value = K; };

// Two CTAs (an SM pair) share a 256 x 256 tile; one CTA alone takes 128 x 256 where S fits 128 rows.
template <int NCTA> struct NsCfg {
  static constexpr int kTileM = kTM * NCTA;
  static constexpr int kBRows = kTN / NCTA;  // rows (or columns of an MN-major operand) of B staged per CTA
  static constexpr int kABytes = kTM * 128;
  static constexpr int kBBytes = kBRows * 128;
  static constexpr int kStages = NCTA == 1 ? 4 : 6;
  static constexpr uint32_t kRing = kStages * (kABytes + kBBytes);
  static constexpr size_t kSmem = size_t(kRing) + 1024 + 256;
};

// One product: Y = alpha A B^T (gram, poly) or alpha A B (update), of every matrix of the batch.
struct NsProduct {
  int S, N, K;               // output [S, N], contraction K
  int tiles_m, tiles_n;
  int tiles;                 // tiles of one matrix (symmetric: on and above the diagonal)
  float alpha, b, diag;      // out = alpha acc (poly: + b A_d[r, c] + diag [r == c])
  __half* Y;                 // [batch][S][ldy]
  long long ldy;
  const __half* A;           // poly: A_d, laid out like Y
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

// tile of a matrix -> tile row and column (symmetric products: row by row of the upper triangle)
template <int MODE>
__device__ __forceinline__ void ns_tile(const NsProduct& p, int t, int& mt, int& nt) {
  if constexpr (MODE == kUpdate) {
    nt = t / p.tiles_m;
    mt = t - nt * p.tiles_m;
  } else {
    mt = 0;
    while (t >= p.tiles_n - mt) { t -= p.tiles_n - mt; ++mt; }
    nt = mt + t;
  }
}

// Whether K block kb of the operand's rows in tile `rt` is read MN-major: always for the update's Z, and for a block of A or D
// below the diagonal (only their 256-wide tiles on and above it exist)
template <int MODE> __device__ __forceinline__ bool a_transposed(int kb, int rt) { return MODE != kGram && kb / (kTN / kTK) < rt; }
template <int MODE> __device__ __forceinline__ bool b_transposed(int kb, int rt) {
  return MODE == kUpdate || (MODE == kPoly && kb / (kTN / kTK) < rt);
}

// What a CTA's three roles share: shared memory, barriers, and each role's place in the ring.
// Warp 0: TMA producer; warp 1: MMA issuer; warps 2-9: epilogue.  Every wait is bounded.
template <int NCTA>
struct NsEngine {
  using C = NsCfg<NCTA>;
  uint32_t smem_a, smem_b, full_bar, empty_bar, acc_full, acc_empty, drain_bar, tmem_base;
  volatile uint32_t* tmem_slot;
  volatile uint32_t* abort_flag;
  uint32_t rank, leader;       // this CTA in its pair; the pair's leader in the cluster
  int warp, lane;
  uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
  long long issued = 0;

  __device__ __forceinline__ void set_up(uint8_t* smem_raw) {
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* bar_mem = smem_raw + (base - raw) + C::kRing;
    smem_a = base;
    smem_b = base + C::kStages * C::kABytes;
    const uint32_t bars = base + C::kRing;
    full_bar = bars;
    empty_bar = bars + 8 * C::kStages;
    acc_full = bars + 16 * C::kStages;
    acc_empty = acc_full + 8 * kAccs;
    drain_bar = acc_empty + 8 * kAccs;
    tmem_slot = reinterpret_cast<volatile uint32_t*>(bar_mem + 16 * C::kStages + 16 * kAccs + 8);
    abort_flag = tmem_slot + 1;
    warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    const uint32_t r = NCTA == 2 ? cluster_ctarank() : 0u;
    rank = r & 1u;
    leader = r & ~1u;
    if (threadIdx.x == 0) {
      for (int s = 0; s < C::kStages; ++s) { mbar_init(full_bar + 8 * s, 1); mbar_init(empty_bar + 8 * s, 1); }
      for (int s = 0; s < kAccs; ++s) { mbar_init(acc_full + 8 * s, 1); mbar_init(acc_empty + 8 * s, kEpiWarpsM * NCTA); }
      mbar_init(drain_bar, 1);
      *abort_flag = 0u;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kAccs * kTN);
    tc_fence_before();
  }
  __device__ __forceinline__ void tear_down() {
    if (warp == 1) {
      tc_fence_after();
      tmem_dealloc(tmem_base, kAccs * kTN);
    }
  }
  // commit of the MMAs issued so far to a barrier of both CTAs of the pair, which may be any pair of its cluster
  // (umma_commit_pair is for clusters of one pair)
  __device__ __forceinline__ void commit(uint32_t bar) {
    if constexpr (NCTA == 1) {
      umma_commit(bar);
    } else {
      const uint16_t mask = static_cast<uint16_t>(3u << leader);
      asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(mask) : "memory");
    }
  }

  // ---- warp 0, lane 0: the operand blocks of one tile
  template <int MODE>
  __device__ __forceinline__ bool produce(const NsProduct& p, const CUtensorMap* map_a, const CUtensorMap* map_b,
                                          const CUtensorMap* map_at, const CUtensorMap* map_bt, int b, int tile) {
    int mt, nt;
    ns_tile<MODE>(p, tile, mt, nt);
    const int num_kb = (p.K + kTK - 1) / kTK;
    const int m0 = mt * C::kTileM + static_cast<int>(rank) * kTM;
    const int n0 = nt * kTN + static_cast<int>(rank) * C::kBRows * (NCTA - 1);
    for (int kb = 0; kb < num_kb; ++kb) {
      if (!mbar_wait(empty_bar + 8 * stage, phase ^ 1u, abort_flag)) return false;
      const uint32_t sa = smem_a + stage * C::kABytes, sb = smem_b + stage * C::kBBytes;
      uint32_t fb = full_bar + 8 * stage;
      const bool a_mn = a_transposed<MODE>(kb, mt), b_mn = b_transposed<MODE>(kb, nt);
      if constexpr (NCTA == 2) {
        if (rank == 0u) mbar_expect_tx(fb, 2 * (C::kABytes + C::kBBytes));
        fb = map_to_cta(fb, leader);  // both CTAs' copies are counted on the leader's barrier
      } else {
        mbar_expect_tx(fb, C::kABytes + C::kBBytes);
      }
      auto load = [&](uint32_t dst, const CUtensorMap* m, int x, int y) {
        if constexpr (NCTA == 2) tma_load_3d_pair(dst, m, fb, x * 2, y, b);  // (the maps count bytes)
        else tma_load_3d(dst, m, fb, x * 2, y, b);
      };
      // along K: one box of 64 elements x all rows; MN-major: boxes of 64 columns x the 64 lines of this K block
      if (!a_mn) {
        load(sa, map_a, kb * kTK, m0);
      } else {
#pragma unroll
        for (int j = 0; j < kTM / kTK; ++j) load(sa + j * kTK * 128, map_at, m0 + j * kTK, kb * kTK);
      }
      if (!b_mn) {
        load(sb, map_b, kb * kTK, n0);
      } else {
#pragma unroll
        for (int j = 0; j < C::kBRows / kTK; ++j) load(sb + j * kTK * 128, map_bt, n0 + j * kTK, kb * kTK);
      }
      ++issued;
      if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
    }
    return true;
  }
  // after a timeout: wait (bounded) for the last use of every ring slot, so that no copy is in flight when the CTA exits
  __device__ __forceinline__ void drain_copies() {
    if (rank != 0u) return;
    const int pending = issued < C::kStages ? static_cast<int>(issued) : C::kStages;
    uint32_t s = stage, ph = phase;
    for (int i = 0; i < pending; ++i) {
      if (s == 0) { s = C::kStages - 1; ph ^= 1u; } else { --s; }
      const unsigned long long t0 = global_timer_ns();
      while (!mbar_try_wait(full_bar + 8 * s, ph) && global_timer_ns() - t0 < kWaitLimitNs) {}
    }
  }

  // ---- warp 1, lane 0 of the leader: the MMAs of one tile
  template <int MODE>
  __device__ __forceinline__ bool multiply(const NsProduct& p, int tile) {
    // MN-major: atoms of 64 columns x 8 lines of K; along K they are 1024 bytes apart, the next 64 columns a box
    // (64 x 128 bytes) further on
    const uint64_t a_desc_k = make_smem_desc(smem_a, 0u, 1024u), a_desc_mn = make_smem_desc(smem_a, kTK * 128u, 1024u);
    const uint64_t b_desc_k = make_smem_desc(smem_b, 0u, 1024u), b_desc_mn = make_smem_desc(smem_b, kTK * 128u, 1024u);
    constexpr uint32_t k_inc = kStepK * 2 >> 4, mn_inc = kStepK * 128 >> 4;
    constexpr uint32_t idesc0 = (1u << 4) | (uint32_t(kTN >> 3) << 17) | (uint32_t(C::kTileM >> 4) << 24);  // F16 x F16 -> fp32
    int mt, nt;
    ns_tile<MODE>(p, tile, mt, nt);
    const int num_kb = (p.K + kTK - 1) / kTK;
    if (!mbar_wait(acc_empty + 8 * acc, acc_phase ^ 1u, abort_flag)) return false;
    tc_fence_after();
    const uint32_t d_tmem = tmem_base + acc * kTN;
    for (int kb = 0; kb < num_kb; ++kb) {
      const bool a_mn = a_transposed<MODE>(kb, mt), b_mn = b_transposed<MODE>(kb, nt);
      const uint32_t idesc = idesc0 | (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16);
      const uint32_t a_inc = a_mn ? mn_inc : k_inc, b_inc = b_mn ? mn_inc : k_inc;
      const uint64_t ad0 = (a_mn ? a_desc_mn : a_desc_k) + static_cast<uint64_t>(stage * (C::kABytes >> 4));
      const uint64_t bd0 = (b_mn ? b_desc_mn : b_desc_k) + static_cast<uint64_t>(stage * (C::kBBytes >> 4));
      if (!mbar_wait(full_bar + 8 * stage, phase, abort_flag)) return false;
      tc_fence_after();
#pragma unroll
      for (int k = 0; k < kTK / kStepK; ++k) {
        if constexpr (NCTA == 1) umma_f16(d_tmem, ad0 + k * a_inc, bd0 + k * b_inc, idesc, (kb | k) != 0 ? 1u : 0u);
        else umma_f16_pair(d_tmem, ad0 + k * a_inc, bd0 + k * b_inc, idesc, (kb | k) != 0 ? 1u : 0u);
      }
      commit(empty_bar + 8 * stage);  // the slot is free (in both CTAs) once these MMAs have read it
      if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
    }
    commit(acc_full + 8 * acc);
    if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
    return true;
  }
  // after a timeout: all MMAs issued so far must retire before the tensor memory is freed
  __device__ __forceinline__ void drain_multiplies() {
    commit(drain_bar);
    const unsigned long long t0 = global_timer_ns();
    while (!mbar_try_wait(drain_bar, 0u) && global_timer_ns() - t0 < kWaitLimitNs) {}
  }

  // ---- warps 2-9: accumulator -> memory.  Results go there from registers: a lane holds 32 columns of one row, two
  // 32-byte stores.  (Staging them for the store engine in shared memory costs what the MMAs and the operand copies leave
  // none of: its bandwidth.)
  template <int MODE>
  __device__ __forceinline__ bool finish(const NsProduct& p, int b, int tile) {
    const int q = warp & 3, half = (warp - 2) / 4;  // TMEM lane quarter, half of the tile's columns
    constexpr int kChunks = kTN / 64;               // 32-column chunks per warp
    int mt, nt;
    ns_tile<MODE>(p, tile, mt, nt);
    const int c_first = half * kChunks, n0 = nt * kTN;
    const int n_chunks = max(0, min(kChunks, (p.N - n0 + 31) / 32 - c_first));  // chunks inside the matrix
    const int row = mt * C::kTileM + static_cast<int>(rank) * kTM + q * 32 + lane;
    __half* yrow = p.Y + (static_cast<long long>(b) * p.S + row) * p.ldy + n0 + c_first * 32;
    // poly: this lane's row of A, read while the products run (past the L1: it may hold an earlier step's A)
    uint4 wa[MODE == kPoly ? kChunks : 1][4];
    if constexpr (MODE == kPoly) {
      const __half* arow = p.A + (static_cast<long long>(b) * p.S + min(row, p.S - 1)) * p.ldy + n0 + c_first * 32;
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          wa[c][j] = c < n_chunks ? __ldcg(reinterpret_cast<const uint4*>(arow + c * 32 + 8 * j)) : make_uint4(0u, 0u, 0u, 0u);
    }
    if (!mbar_wait(acc_full + 8 * acc, acc_phase, abort_flag)) return false;
    tc_fence_after();
    const uint32_t t_addr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * kTN + c_first * 32;
#pragma unroll
    for (int c2 = 0; c2 < kChunks; c2 += 2) {
      uint32_t r[2][32];
      tmem_ld32(t_addr + c2 * 32, r[0]);  // (columns past the matrix hold nothing of interest)
      tmem_ld32(t_addr + (c2 + 1) * 32, r[1]);
      tmem_ld_wait();
      if (c2 + 2 == kChunks) {  // the accumulator has been read: the next tile may overwrite it
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (NCTA == 1) mbar_arrive(acc_empty + 8 * acc);
          else mbar_arrive_cluster(map_to_cta(acc_empty + 8 * acc, leader));
        }
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int c = c2 + s, col0 = n0 + (c_first + c) * 32;
        uint32_t o[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          float x = __uint_as_float(r[s][2 * j]) * p.alpha, y = __uint_as_float(r[s][2 * j + 1]) * p.alpha;
          if constexpr (MODE == kPoly) {
            const uint4 w4 = wa[c][j / 4];
            const uint32_t w = (j & 3) == 0 ? w4.x : (j & 3) == 1 ? w4.y : (j & 3) == 2 ? w4.z : w4.w;
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
            x = fmaf(p.b, v.x, x) + (row == col0 + 2 * j ? p.diag : 0.f);
            y = fmaf(p.b, v.y, y) + (row == col0 + 2 * j + 1 ? p.diag : 0.f);
          }
          const __half2 hh = __floats2half2_rn(x, y);
          o[j] = *reinterpret_cast<const uint32_t*>(&hh);
        }
        if (c < n_chunks && row < p.S) {  // (rows are padded to whole chunks)
          st_bytes<32>(reinterpret_cast<char*>(yrow + c * 32), o);
          st_bytes<32>(reinterpret_cast<char*>(yrow + c * 32 + 16), o + 8);
        }
      }
    }
    if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
    return true;
  }
};

}  // namespace

// One product of the whole batch: persistent CTAs (pairs).  On expiry of a wait the CTA records SCALIFY_DEV_TIMEOUT, drains
// its copies and MMAs, frees its tensor memory and returns.
// 12 x 768 x 2304: gram 21 us (tensor pipe active 63%), poly 14 (31%), update 33 (59%): about 8 us of each are the first
// copies, the last tile's epilogue and the hand-over to the next product.  1 x 8192 x 2048 (36, 36 and 256 tiles on 74 pairs):
// 49 us (87% on the SMs that have a tile), 23 (48%), 60 (72%).
template <int MODE, int NCTA>
__global__ void __launch_bounds__(kNsThreads, 1) ns_product_kernel(const __grid_constant__ CUtensorMap map_a,
                                                                  const __grid_constant__ CUtensorMap map_b,
                                                                  const __grid_constant__ CUtensorMap map_at,
                                                                  const __grid_constant__ CUtensorMap map_bt, const NsProduct p, int batch,
                                                                  uint32_t* status) {
  asm volatile("griddepcontrol.launch_dependents;");  // the next product may set up while this one runs
  extern __shared__ uint8_t smem_raw[];
  NsEngine<NCTA> e;
  if (threadIdx.x == 32 * 2) {  // (the maps are arguments: nothing the kernel before writes)
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_a)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_b)) : "memory");
    if constexpr (MODE != kGram) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_at)) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_bt)) : "memory");
    }
  }
  e.set_up(smem_raw);
  __syncthreads();
  if constexpr (NCTA == 2) cluster_sync_all();
  tc_fence_after();
  asm volatile("griddepcontrol.wait;" ::: "memory");  // nothing above touches what the kernel before writes
  e.tmem_base = *e.tmem_slot;
  const int unit = blockIdx.x / NCTA, num_units = gridDim.x / NCTA, num_tiles = p.tiles * batch;
  bool timed_out = false;
  if (e.warp == 0) {
    if (e.lane == 0) {
      for (int tile = unit; tile < num_tiles && !timed_out; tile += num_units)
        timed_out = !e.template produce<MODE>(p, &map_a, &map_b, &map_at, &map_bt, tile / p.tiles, tile % p.tiles);
      if (timed_out || *e.abort_flag) e.drain_copies();
    }
  } else if (e.warp == 1) {
    if (e.lane == 0 && e.rank == 0u) {
      for (int tile = unit; tile < num_tiles && !timed_out; tile += num_units) timed_out = !e.template multiply<MODE>(p, tile % p.tiles);
      if (timed_out || *e.abort_flag) e.drain_multiplies();
    }
  } else {
    for (int tile = unit; tile < num_tiles && !timed_out; tile += num_units)
      timed_out = !e.template finish<MODE>(p, tile / p.tiles, tile % p.tiles);
  }
  if (timed_out) atomicOr(status, static_cast<uint32_t>(SCALIFY_DEV_TIMEOUT));
  tc_fence_before();
  __syncthreads();
  if constexpr (NCTA == 2) cluster_sync_all();
  e.tear_down();
}

// All products of all steps in one launch, for matrices of few tiles: one cluster per matrix (so no matrix waits for
// another), its CTAs (pairs) share the matrix's tiles, and a cluster barrier takes the place of a launch between products.
struct NsMaps {
  CUtensorMap z[2], b_z[2], zt[2], a, b_a, at, d, dt;
};
struct NsChain {
  NsProduct gram, poly, update[2];  // update[k]: reads z[k], writes z[k ^ 1]
  int steps;
  uint32_t* status;
};
template <int NCTA>
__global__ void __launch_bounds__(kNsThreads, 1) ns_chain_kernel(const __grid_constant__ NsMaps maps, const __grid_constant__ NsChain c) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  extern __shared__ uint8_t smem_raw[];
  NsEngine<NCTA> e;
  e.set_up(smem_raw);
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  e.tmem_base = *e.tmem_slot;
  uint32_t cluster_size;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(cluster_size));
  const int unit = static_cast<int>(cluster_ctarank()) / NCTA, num_units = static_cast<int>(cluster_size) / NCTA;
  const int b = static_cast<int>(blockIdx.x / cluster_size);
  bool timed_out = false;  // (a role that gave up keeps taking part in the barriers)
  auto product = [&](auto mode, const NsProduct& p, const CUtensorMap* ma, const CUtensorMap* mb, const CUtensorMap* mat, const CUtensorMap* mbt) {
    constexpr int MODE = decltype(mode)::value;
    if (e.warp == 0) {
      if (e.lane == 0) {
        asm volatile("fence.proxy.async;" ::: "memory");  // the copies read what the other CTAs' stores have written
        for (int tile = unit; tile < p.tiles && !timed_out; tile += num_units)
          timed_out = !e.template produce<MODE>(p, ma, mb, mat, mbt, b, tile);
      }
      __syncwarp();
    } else if (e.warp == 1) {
      if (e.lane == 0 && e.rank == 0u)
        for (int tile = unit; tile < p.tiles && !timed_out; tile += num_units) timed_out = !e.template multiply<MODE>(p, tile);
      __syncwarp();
    } else {
      for (int tile = unit; tile < p.tiles && !timed_out; tile += num_units) timed_out = !e.template finish<MODE>(p, b, tile);
      asm volatile("fence.proxy.async;" ::: "memory");
    }
    cluster_sync_all();
  };
  for (int k = 0; k < c.steps; ++k) {
    const int z = k & 1;
    product(KindC<kGram>{}, c.gram, &maps.z[z], &maps.b_z[z], nullptr, nullptr);
    product(KindC<kPoly>{}, c.poly, &maps.a, &maps.b_a, &maps.at, &maps.at);
    product(KindC<kUpdate>{}, c.update[z], &maps.d, nullptr, &maps.dt, &maps.zt[z]);
  }
  if (e.warp == 0 && e.lane == 0 && *e.abort_flag) e.drain_copies();
  if (e.warp == 1 && e.lane == 0 && e.rank == 0u && *e.abort_flag) e.drain_multiplies();
  if (timed_out) atomicOr(c.status, static_cast<uint32_t>(SCALIFY_DEV_TIMEOUT));
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  e.tear_down();
}

// ------------------------------------------------------------------------------------------------- element-wise passes
namespace {

template <int V> struct IntC { static constexpr int value = V; };

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

// Words of one vector of a matrix (MDT < 0: no momentum), and u_d (and m'_d) from them: u is the momentum, or its Nesterov form, in units of m'_s
template <int GDT, int MDT>
struct MuonWords {
  uint32_t g[kVec * ElemBytes<GDT>::v / 4], m[kVec * (MDT < 0 ? 4 : ElemBytes<MDT < 0 ? 4 : MDT>::v) / 4];
};
template <int GDT, int MDT>
__device__ __forceinline__ void muon_load(const MuonTensor& t, int64_t row, int v, int n, MuonWords<GDT, MDT>& w) {
  load_vec<GDT>(static_cast<const char*>(t.g) + row * t.g_ld * ElemBytes<GDT>::v, v, n, w.g);
  if constexpr (MDT >= 0) load_vec<MDT>(static_cast<const char*>(t.m) + row * t.m_ld * ElemBytes<MDT>::v, v, n, w.m);
}
template <int GDT, int MDT>
__device__ __forceinline__ void muon_vec(const MuonWords<GDT, MDT>& w, const MuonPass& p, const MuonFactors& f, float* u, float* m) {
  float g[kVec];
  decode_vec<GDT, kVec>(w.g, g);
  if constexpr (MDT < 0) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) u[e] = g[e];
  } else {
    decode_vec<MDT, kVec>(w.m, m);
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float gg = f.fg * g[e];
      m[e] = fmaf(f.fm, m[e], gg);
      u[e] = p.nesterov ? fmaf(p.momentum, m[e], gg) : m[e];
    }
  }
}

}  // namespace

// |u|_F^2, one partial per block (fixed order within and between blocks), and the step's factors.  12 x 768 x 2304 with an
// E5M2 gradient and FP16 momentum: 22 us (64 MB).
template <int GDT, int MDT>
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
  constexpr int kAhead = 4;  // vectors in flight per thread
  for (uint32_t i0 = blockIdx.x * 256u * kAhead + threadIdx.x; i0 < total; i0 += gridDim.x * 256u * kAhead) {
    MuonWords<GDT, MDT> w[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint32_t i = i0 + k * 256u, row = i / nv;
      const int v = static_cast<int>(i - row * nv);
      if (i < total) muon_load<GDT, MDT>(t, row, v, t.cols - v * kVec, w[k]);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i0 + k * 256u >= total) break;
      float u[kVec], m[kVec], ss = 0.f;
      muon_vec<GDT, MDT>(w[k], p, f, u, m);
#pragma unroll
      for (int e = 0; e < kVec; ++e) ss = fmaf(u[e], u[e], ss);
      sum += ss;
    }
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
// memory where the matrix is tall (12 x 768 x 2304: 28 us, 149 MB, 5.3 TB/s; 1 x 2048 x 8192 20.1 us, the tall 1 x 8192 x 2048
// 30.0: turning a tile meets 8-way bank conflicts, 25000 of 31600 wavefronts of shared memory per SM).  The new scale
// words are written here (nothing of this launch reads the old ones).
template <int GDT, int MDT>
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
    // fp32 holds the squares of a matrix with 2^-60 <= norm <= 2^63; below that it counts as zeros, above as infinite
    const float norm = static_cast<float>(sqrt(s));
    const bool finite = norm <= 0x1p63f;
    if (threadIdx.x == 0) s_scale = !finite ? __int_as_float(0x7fc00000) : norm < 0x1p-60f ? 0.f : p.inv_sigma / (norm + p.eps);
    if (threadIdx.x == 0 && blockIdx.x == 0) {
      const MuonFactors f = p.factors[inst];
      if (t.m) *t.m_scale = f.m_s;
      if (t.w_scale) *t.w_scale = f.w_s;
      if (t.wc_scale) *t.wc_scale = f.w_s;
      if (!finite) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_NONFINITE_STAT));
    }
  }
  const MuonFactors f = p.factors[inst];
  MuonWords<GDT, MDT> w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = threadIdx.x + k * 256, row = r0 + (i >> 3), col = c0 + (i & 7) * kVec;
    if (row < t.rows && col < t.cols) muon_load<GDT, MDT>(t, row, col / kVec, t.cols - col, w[k]);
  }
  __syncthreads();
  const float scale = s_scale;
  __half* Z = p.Z + static_cast<long long>(inst) * p.S * p.ld;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = threadIdx.x + k * 256, lr = i >> 3, lv = i & 7;
    const int row = r0 + lr, col = c0 + lv * kVec, n = t.cols - col;
    if (row < t.rows && n > 0) {
      float u[kVec], m[kVec];
      muon_vec<GDT, MDT>(w[k], p, f, u, m);
      if constexpr (MDT >= 0) store_vec<MDT>(static_cast<char*>(t.m) + static_cast<int64_t>(row) * t.m_ld * ElemBytes<MDT>::v, col / kVec, n, m);
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

// w' = fw w - fo Z (and its copy), or the orthogonal matrix itself (12 x 768 x 2304, FP16 with an E4M3 copy: 25 us, 5.9 TB/s;
// 1 x 8192 x 2048 29.7 us, with the same bank conflicts as above).
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
// The most clusters of `size` CTAs of a kernel that are resident at once, found once per device and size (size is a power
// of two up to 16; more than 8 needs the kernel's consent).
template <class K>
static int max_clusters(K kernel, size_t smem, int size, DeviceOnce& once, int* value) {
  return device_once(once, value, [&](int* v) {
    SCALIFY_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    if (size > 8) SCALIFY_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    cudaLaunchConfig_t qc = {};
    qc.gridDim = dim3(static_cast<unsigned>(sm_count() / size * size)); qc.blockDim = dim3(kNsThreads); qc.dynamicSmemBytes = smem;
    cudaLaunchAttribute qa[1];
    qa[0].id = cudaLaunchAttributeClusterDimension;
    qa[0].val.clusterDim.x = static_cast<unsigned>(size); qa[0].val.clusterDim.y = 1; qa[0].val.clusterDim.z = 1;
    qc.attrs = qa; qc.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &qc) != cudaSuccess) { n = 0; cudaGetLastError(); }
    *v = n;
    return int(SCALIFY_OK);
  });
}

template <int MODE, int NCTA>
static int launch_product_variant(const CUtensorMap (&m)[4], const NsProduct& p, int batch, uint32_t* status, cudaStream_t st) {
  using C = NsCfg<NCTA>;
  auto kernel = ns_product_kernel<MODE, NCTA>;
  static DeviceOnce once;
  int most = 0;  // CTAs or CTA pairs that fit the GPU
  int rc = max_clusters(kernel, C::kSmem, NCTA, once, &most);
  if (rc) return rc;
  if (most < 1) return SCALIFY_ERR_UNSUPPORTED;
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = NCTA; attrs[1].val.clusterDim.y = 1; attrs[1].val.clusterDim.z = 1;
  const long long tiles = static_cast<long long>(p.tiles) * batch;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((tiles < most ? tiles : most) * NCTA));
  cfg.blockDim = dim3(kNsThreads); cfg.dynamicSmemBytes = C::kSmem; cfg.stream = st;
  cfg.attrs = attrs; cfg.numAttrs = 2;
  SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, m[0], m[1], m[2], m[3], p, batch, status));
  return SCALIFY_OK;
}

struct NsMatrix { __half* p; int rows, cols; long long ld; };  // [batch][rows][ld]
static int ns_map(CUtensorMap* m, const NsMatrix& x, int batch, uint32_t box_rows) {
  return make_byte_map(m, x.p, static_cast<uint64_t>(x.cols) * 2, x.rows, batch, x.ld * 2, static_cast<uint64_t>(x.rows) * x.ld * 2, 128, box_rows);
}
// CTA pairs wherever there is more than one row tile of a single CTA
static int ns_ncta(int S) { return S > kTM ? 2 : 1; }
// tiles of Y = A B^T (gram, poly: B is [N, K]) or A B (update: B is [K, N]), and the sizes
static void ns_shape(int mode, const NsMatrix& A, const NsMatrix& Y, NsProduct& p) {
  const int tile_m = kTM * ns_ncta(Y.rows);
  p.S = Y.rows; p.N = Y.cols; p.K = A.cols;
  p.Y = Y.p; p.ldy = Y.ld;
  p.tiles_m = (Y.rows + tile_m - 1) / tile_m;
  p.tiles_n = (Y.cols + kTN - 1) / kTN;
  // symmetric products: the tile is square for CTA pairs; a single CTA's tile holds the whole matrix (S <= 128)
  p.tiles = mode == kUpdate ? p.tiles_m * p.tiles_n : p.tiles_n * (p.tiles_n + 1) / 2;
}
template <int MODE>
static int launch_product(const NsMatrix& A, const NsMatrix& B, const NsProduct& p, int batch, uint32_t* status, cudaStream_t st) {
  const int ncta = ns_ncta(p.S);
  CUtensorMap m[4];  // both operands with the contraction along their lines, and MN-major
  int rc = ns_map(&m[0], A, batch, kTM);
  if (!rc) rc = ns_map(&m[1], B, batch, kTN / ncta);
  if (!rc) rc = ns_map(&m[2], A, batch, kTK);
  if (!rc) rc = ns_map(&m[3], B, batch, kTK);
  if (rc) return rc;
  if (ncta == 2) return launch_product_variant<MODE, 2>(m, p, batch, status, st);
  return launch_product_variant<MODE, 1>(m, p, batch, status, st);
}

// Clusters of 1, 2, 4 or 8 units (CTAs, or pairs) per matrix
constexpr int kChainSizes = 4;
template <int NCTA>
static int chain_clusters(int size_log, int* most) {
  static DeviceOnce once[kChainSizes];
  return max_clusters(ns_chain_kernel<NCTA>, NsCfg<NCTA>::kSmem, NCTA << size_log, once[size_log], most);
}
template <int NCTA>
static int launch_chain(const NsMatrix (&z)[2], const NsMatrix& A, const NsMatrix& D, const NsChain& c, int batch, int size_log, cudaStream_t st) {
  NsMaps maps;
  int rc = SCALIFY_OK;
  for (int k = 0; k < 2 && !rc; ++k) {
    rc = ns_map(&maps.z[k], z[k], batch, kTM);
    if (!rc) rc = ns_map(&maps.b_z[k], z[k], batch, kTN / NCTA);
    if (!rc) rc = ns_map(&maps.zt[k], z[k], batch, kTK);
  }
  if (!rc) rc = ns_map(&maps.a, A, batch, kTM);
  if (!rc) rc = ns_map(&maps.b_a, A, batch, kTN / NCTA);
  if (!rc) rc = ns_map(&maps.at, A, batch, kTK);
  if (!rc) rc = ns_map(&maps.d, D, batch, kTM);
  if (!rc) rc = ns_map(&maps.dt, D, batch, kTK);
  if (rc) return rc;
  cudaLaunchAttribute attrs[2];
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = NCTA << size_log; attrs[1].val.clusterDim.y = 1; attrs[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(batch) * (NCTA << size_log));
  cfg.blockDim = dim3(kNsThreads); cfg.dynamicSmemBytes = NsCfg<NCTA>::kSmem; cfg.stream = st;
  cfg.attrs = attrs; cfg.numAttrs = 2;
  SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&cfg, ns_chain_kernel<NCTA>, maps, c));
  return SCALIFY_OK;
}

// One launch or one per product?  The times of a step, in K blocks of a tile (about 0.3 us): a unit's share of the tiles,
// and what comes between two products: a cluster barrier with a cold start of the ring (8 blocks), or a launch (18; more
// on the host).  Five steps in one launch and in fifteen: 4 x 256 x 320 90 and 99 us, 4 x 512 x 512 115 and 125;
// 16 x 512 x 1024 229 and 166, 12 x 768 x 2304 434 and 377.  *size_log < 0: one launch per product.
template <int NCTA>
static int choose_chain(const NsChain& c, int batch, int* size_log) {
  auto blocks = [](const NsProduct& p) { return static_cast<double>((p.K + kTK - 1) / kTK); };
  const NsProduct* all[3] = {&c.gram, &c.poly, &c.update[0]};
  const double units = sm_count() / NCTA;
  double best = 0.0;
  for (const NsProduct* p : all) best += ceil(static_cast<double>(p->tiles) * batch / units) * blocks(*p) + 18.0;
  *size_log = -1;
  for (int s = 0; s < kChainSizes; ++s) {
    int most = 0;
    const int rc = chain_clusters<NCTA>(s, &most);
    if (rc) return rc;
    if (most < 1) continue;
    double cost = 0.0;
    for (const NsProduct* p : all) cost += ceil(static_cast<double>(p->tiles) / (1 << s)) * blocks(*p) + 8.0;
    cost *= ceil(static_cast<double>(batch) / most);
    if (cost < best) { best = cost; *size_log = s; }
  }
  return SCALIFY_OK;
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
    // outputs/inputs: rows/cols of a weight stored [outputs, inputs], cols/rows of one stored [inputs, outputs]
    if (h.factor == SCALIFY_MUON_SPECTRAL ? tall == 1 : h.factor == SCALIFY_MUON_SPECTRAL_IN_OUT && tall == 0) kappa = sqrt(static_cast<double>(s.L) / s.S);
    else if (h.factor == SCALIFY_MUON_RMS) kappa = 0.2 * sqrt(static_cast<double>(s.L));
    p.lr[tall] = static_cast<float>(static_cast<double>(h.lr) * kappa);
    p.p2_lr[tall] = p.lr[tall] > 0.f ? host_p2(p.lr[tall]) : 0.f;
  }

  const unsigned tl = static_cast<unsigned>((s.L + kPreTile - 1) / kPreTile), ts = static_cast<unsigned>((s.S + kPreTile - 1) / kPreTile);
  const dim3 tiles(tl * ts, 1, count);
  auto enter = [&](auto g_dt, auto m_dt) {
    muon_norm_kernel<decltype(g_dt)::value, decltype(m_dt)::value><<<dim3(p.parts, count), 256, 0, st>>>(tab, p);
    muon_momentum_kernel<decltype(g_dt)::value, decltype(m_dt)::value><<<tiles, 256, 0, st>>>(tab, p);
  };
  SCALIFY_DISPATCH_DTYPE(tab.t[0].g_dt, GDT, {
    if (!tab.t[0].m) enter(IntC<GDT>{}, IntC<-1>{});
    else if (tab.t[0].m_dt == SCALIFY_F16) enter(IntC<GDT>{}, IntC<SCALIFY_F16>{});
    else enter(IntC<GDT>{}, IntC<SCALIFY_F32>{});
  })
  SCALIFY_CUDA_TRY(cudaGetLastError());

  NsChain c = {};
  c.steps = h.steps;
  c.status = view.status;
  ns_shape(kGram, z[0], A, c.gram);
  c.gram.alpha = p.sigma * p.sigma * kGramScale;
  ns_shape(kPoly, A, D, c.poly);
  c.poly.alpha = h.c / kGramScale;
  c.poly.b = h.b;
  c.poly.diag = h.a * kGramScale;
  c.poly.A = A.p;
  for (int k = 0; k < 2; ++k) {
    ns_shape(kUpdate, D, z[k ^ 1], c.update[k]);
    c.update[k].alpha = 1.0f / kGramScale;
  }
  const bool pairs = ns_ncta(s.S) == 2;
  int size_log = -1;
  int rc = pairs ? choose_chain<2>(c, count, &size_log) : choose_chain<1>(c, count, &size_log);
  if (rc) return rc;
  if (size_log >= 0) {
    rc = pairs ? launch_chain<2>(z, A, D, c, count, size_log, st) : launch_chain<1>(z, A, D, c, count, size_log, st);
    if (rc) return rc;
  } else {
    for (int k = 0; k < h.steps; ++k) {
      const int cur = k & 1;
      rc = launch_product<kGram>(z[cur], z[cur], c.gram, count, c.status, st);
      if (!rc) rc = launch_product<kPoly>(A, A, c.poly, count, c.status, st);
      if (!rc) rc = launch_product<kUpdate>(D, z[cur], c.update[cur], count, c.status, st);
      if (rc) return rc;
    }
  }
  p.Z = z[h.steps & 1].p;
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
