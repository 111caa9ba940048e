// Losses of a language model's output layer z = H W^T, H [n, d], W [V, d], without its logits in memory: softmax cross
// entropy, and the divergence from a teacher's top logits.  Both are
//
//   loss_t = sum_i q_i log q_i - sum_i q_i z[t,i]/T + Q lse_t (+ zeta lse_t^2),   lse_t = log sum_v exp(z[t,v]/T),  Q = sum q
//   d loss_t / d z[t,v] = ((Q + 2 zeta lse_t) p[t,v] - q[t,v]) / T,               p = exp(z/T - lse)
//
// with a row's target distribution q given by few entries: one for cross entropy (q = 1), up to 256 for a teacher's.
//
// Logits kernel: tcgen05 on CTA pairs, 256 x 256 tiles, FP8 operands as kind::f8f6f4, 16-bit ones as kind::f16.  The
//   epilogue warps read the fp32 logits from tensor memory while the next tile is multiplied.
//   forward: running maximum and sum of a row over a run of tiles, in base 2 (one multiply-add and one exponential per
//     element), and the sum of q z; one partial result per row and run, joined by a small kernel in a fixed order.
// Gradient kernel: the logits again, of a PIECE of the vocabulary, now to the gradient D = g (Q p - q)/T in 16 bits; and, in
//   the same launch, the products dW = D^T H and dH += D W of the piece before (MN-major operands: nothing is transposed in
//   memory; dH's sums over the pieces are fp32).  The products' few long tiles alone leave pairs idle (8192 x 50257 x 768, pieces of
//   7424 columns: 183 tiles on 74 pairs, 357 K blocks for some where 308 are the average); the logits' short ones fill them up.
//   (A vocabulary of one piece has one launch of logits and one of products.)
//
// D has the operands' type; FP8 operands are converted to FP16, which holds them exactly, and D is FP16.  FP16 has few
// exponents, so D is stored at a scale that brings the largest row coefficient to 2^14: probabilities down to 2^-28 keep all 11
// bits in that row, entries below 2^-38 of the largest coefficient are lost.  Its rounding is at most half a step (FP16 2^-11,
// BF16 2^-8) per element, independent over the vocabulary: it adds to dH and dW about what rounding them once to that type does
// (8192 x 50257 x 768, BF16: 2.3e-3 of their norm instead of 1.6e-3).  More digits would cost more than they are worth beside that
// rounding: TF32 operands run at half the rate, two halves of D are half as much again (few rows: kFewRows), and FP16 copies of BF16
// operands would lose BF16's range.
#include <cuda.h>
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "linear_loss.h"
#include "scalify_common.cuh"
#include "scalify_launch.h"
#include "tcgen05_ptx.cuh"
#include "vec8.cuh"

namespace scalify {

namespace {

constexpr int kTM = 128;            // rows of the output tile per CTA
constexpr int kTN = 256;            // columns of the output tile
constexpr int kRowBytes = 128;      // a K block: one 128-byte swizzle row
constexpr int kK16 = 64;            // ... in 16-bit elements
constexpr int kAccs = 2;            // accumulators of 256 TMEM columns: the epilogue overlaps the next tile's products
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
// Two CTAs (an SM pair) share a tile of 256 rows, each with its own rows of A and half of B; batches of at most 128 rows leave
// the second CTA's rows empty, so one CTA alone takes a tile of 128 rows and all of B there: twice the weights per MMA.
template <int NCTA> struct Cfg {
  static constexpr int kTileM = kTM * NCTA;
  static constexpr int kABytes = kTM * kRowBytes, kBBytes = kTN / NCTA * kRowBytes;
  static constexpr uint32_t kRing = 6 * (kTM + kTN / 2) * kRowBytes;
  static constexpr size_t kSmem = size_t(kRing) + 1024 + 256;
  static constexpr size_t kStaging = size_t(kEpiWarps) * 32 * 128;  // of the distillation and the gradient kernels: 32 values per lane
};
// The operand ring.  A single CTA's logits want as many weights in flight as fit, and its batch fills few of A's 128 rows: A
// takes only those (the MMAs read on into what lies behind them, which decides rows that nobody looks at), B the tile's width.
struct Ring {
  int stages, a_bytes, b_bytes;  // of a stage: multiples of 1024
};
constexpr int kMaxStages = 12;
// K blocks (of 64 16-bit or 128 8-bit values) from which on a contraction is long in the forward call, and of its parts.  Sums of 256
// 16-bit values (a single CTA, which waits for its weights anyway) and of 768 in the tensor cores' 32 bits leave the loss with the
// error that it has from rounding the result (2 rows of 3269: 3.4e-6 with parts of 512, 7.6e-6 with parts of 1024, 1.3e-6 so);
// parts in contractions of 768 values, too, would make 37 x 50257 x 768 41 instead of 29 us, which then waits for the additions.
template <int NCTA> constexpr int kLongKb = NCTA == 1 ? 12 : 24;
template <int NCTA> constexpr int kSegmentKb = NCTA == 1 ? 4 : 12;
// K blocks of one accumulator in the gradient kernel, of the logits and of the products.  The tensor cores drop what lies below the
// running sum's last bits, of every product: by measurement 2^-25 of the sum per product and 2^-23 per addition at most, so that
// a sum of N products of one sign loses N 2^-27 of itself on average.  In one accumulator a batch of 2^22 rows left dW off by
// 2.6e-2 and a vocabulary of 2^22 dH by 1.3e-2; 256 blocks lose 1e-4, less than what rounding the result to FP16 does, and 64
// blocks of logits 2.5e-5 of a logit (128 blocks of a product would make the step 4096 x 4096, whose pieces have 252, 1.2 % slower).
// Parts cost 2000 x 32003 x 8192 3.5 % (3.51 -> 3.63 ms) and 40000 x 20000 x 768 1.5 % (5.05 -> 5.13 ms).
constexpr int kLogitKb = 64, kSumKb = 256;
constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLargest = 3.402823466e38f;  // of fp32

template <bool F8, int NCTA>
__device__ __forceinline__ void umma(uint32_t d_tmem, uint64_t ad, uint64_t bd, uint32_t idesc, uint32_t acc) {
  if constexpr (F8 && NCTA == 2) {
    umma_f8_pair(d_tmem, ad, bd, idesc, acc);
  } else if constexpr (F8) {
    umma_f8(d_tmem, ad, bd, idesc, acc);
  } else if constexpr (NCTA == 1) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(ad), "l"(bd), "r"(idesc), "r"(acc) : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem), "l"(ad), "l"(bd), "r"(idesc), "r"(acc) : "memory");
  }
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What an earlier kernel may have written, read behind the wait for it: ordinary loads, kept in order with the wait.  (Not through
// the read-only path, whose loads count as invariant.  Through the L1: four of a row's entries share a sector; past it the
// distillation step 8192 x 768 takes 1958 instead of 1934 us, 37 x 768 30.2 instead of 29.1.)
__device__ __forceinline__ int2 ld_written(const int2* p) {
  int2 v;
  asm volatile("ld.global.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ int ld_written(const int* p) {
  int v;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ int ld_written(const uint16_t* p) {
  uint16_t v;
  asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ long long ld_written(const long long* p) {
  long long v;
  asm volatile("ld.global.s64 %0, [%1];" : "=l"(v) : "l"(p));
  return v;
}

// One lane of the whole warp, the same one each time (same mask, same leader): the store engine's calls and the waits for them,
// whose groups belong to the thread that made them.  (All lanes get here together: the election waits for them.  A branch on the
// lane would be as good by the rules; compiled into an earlier form of these kernels it left tiles unwritten, for a reason that
// their source does not show.)
__device__ __forceinline__ bool elected_lane() {
  uint32_t one;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(one));
  return one != 0u;
}
// 32 values of this lane's row in shared memory, where one whose place is known at run time only can be reached: 16-byte pieces
// exchanged within a row so that the lanes' accesses meet different banks.
struct LaneRow {
  uint32_t* row;
  int lane;
  __device__ __forceinline__ uint4* piece(int j) const { return reinterpret_cast<uint4*>(row) + (j ^ (lane & 7)); }
  __device__ __forceinline__ void put(const uint32_t* r) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) *piece(j) = make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
  }
  __device__ __forceinline__ void get(uint32_t* r) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint4 v = *piece(j);
      r[4 * j] = v.x; r[4 * j + 1] = v.y; r[4 * j + 2] = v.z; r[4 * j + 3] = v.w;
    }
  }
  __device__ __forceinline__ float& at(int i) const { return reinterpret_cast<float*>(piece(i >> 2))[i & 3]; }
  // 32 16-bit values per lane -> 32 rows of memory from (x bytes, y) on, by the store engine (which leaves out what lies past
  // the matrix): a warp's own stores would meet 32 lines per instruction, beside its exponentials (distillation step 8192 x 768
  // 1920 -> 1834 us).  Two tiles in turns (`flip`); every store of the tile
  // before the last one has left shared memory before its place is taken.  All lanes of the warp.
  __device__ __forceinline__ void store(const uint32_t* o, const CUtensorMap* map, int x_bytes, int y, uint32_t& flip) const {
    if (elected_lane()) bulk_wait_read<1>();
    __syncwarp();
    uint4* tile = reinterpret_cast<uint4*>(row - lane * 32) + flip * 128;
    flip ^= 1u;
#pragma unroll
    for (int j = 0; j < 4; ++j) tile[lane * 4 + (j ^ ((lane >> 1) & 3))] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
    fence_async_smem();
    __syncwarp();
    if (elected_lane()) {
      tma_store_3d(map, smem_u32(tile), x_bytes, y, 0);
      bulk_commit();
    }
  }
};

// Shared memory, barriers and each role's place in the ring.  Warp 0: TMA producer; warp 1: MMA issuer (of the pair's first
// CTA); warps 2-9: epilogue.  Every wait is bounded.
template <int NCTA> struct Engine {
  using C = Cfg<NCTA>;
  int stages, a_bytes, b_bytes;
  uint32_t smem_a, smem_b, full_bar, empty_bar, acc_full, acc_empty, drain_bar, tmem_base;
  volatile uint32_t* tmem_slot;
  volatile uint32_t* abort_flag;
  uint8_t* stage_mem;
  uint32_t rank;
  int warp, lane;
  uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
  long long issued = 0;

  __device__ __forceinline__ void set_up(uint8_t* smem_raw, const Ring& ring, bool staging) {
    stages = NCTA == 2 ? 6 : ring.stages;  // (pairs always have whole tiles)
    a_bytes = NCTA == 2 ? C::kABytes : ring.a_bytes;
    b_bytes = NCTA == 2 ? C::kBBytes : ring.b_bytes;
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    stage_mem = smem_raw + (base - raw) + C::kRing;  // (the store engine's swizzle wants 512-byte boundaries)
    const uint32_t bar_at = C::kRing + (staging ? C::kStaging : 0);
    uint8_t* bar_mem = smem_raw + (base - raw) + bar_at;
    smem_a = base;
    smem_b = base + stages * a_bytes;
    const uint32_t bars = base + bar_at;
    full_bar = bars;
    empty_bar = bars + 8 * kMaxStages;
    acc_full = bars + 16 * kMaxStages;
    acc_empty = acc_full + 8 * kAccs;
    drain_bar = acc_empty + 8 * kAccs;
    tmem_slot = reinterpret_cast<volatile uint32_t*>(bar_mem + 16 * kMaxStages + 16 * kAccs + 8);
    abort_flag = tmem_slot + 1;
    warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    rank = NCTA == 2 ? cluster_ctarank() : 0u;
    if (threadIdx.x == 0) {
      for (int s = 0; s < stages; ++s) { mbar_init(full_bar + 8 * s, 1); mbar_init(empty_bar + 8 * s, 1); }
      for (int s = 0; s < kAccs; ++s) { mbar_init(acc_full + 8 * s, 1); mbar_init(acc_empty + 8 * s, kEpiWarps * NCTA); }
      mbar_init(drain_bar, 1);
      *abort_flag = 0u;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kAccs * kTN);
    tc_fence_before();
    __syncthreads();
    if constexpr (NCTA == 2) cluster_sync_all();
    tc_fence_after();
    tmem_base = *tmem_slot;
  }
  __device__ __forceinline__ void tear_down() {
    tc_fence_before();
    __syncthreads();
    if constexpr (NCTA == 2) cluster_sync_all();
    if (warp == 1) {
      tc_fence_after();
      tmem_dealloc(tmem_base, kAccs * kTN);
    }
  }

  // ---- warp 0, lane 0: the operand blocks of one tile.  Along K: a box of 128 bytes x 128 rows.  MN-major (16-bit only):
  // boxes of 64 columns x the 64 lines of this K block.
  __device__ __forceinline__ bool produce(const CUtensorMap* ma, const CUtensorMap* mb, int m0, int n0, int height, int width, int kb0, int num_kb, bool a_mn, bool b_mn) {
    m0 += static_cast<int>(rank) * kTM;
    n0 += static_cast<int>(rank) * (width / 2);
    for (int kb = kb0; kb < kb0 + num_kb; ++kb) {
      if (!mbar_wait(empty_bar + 8 * stage, phase ^ 1u, abort_flag)) return false;
      const uint32_t sa = smem_a + stage * a_bytes, sb = smem_b + stage * b_bytes;
      uint32_t fb = full_bar + 8 * stage;
      if (rank == 0u) mbar_expect_tx(fb, NCTA * height * kRowBytes + width * kRowBytes);
      if constexpr (NCTA == 2) fb = map_to_cta(fb, 0u);  // both CTAs' copies are counted on the first one's barrier
      auto load = [&](uint32_t dst, const CUtensorMap* m, int x_bytes, int y) {
        if constexpr (NCTA == 2) tma_load_3d_pair(dst, m, fb, x_bytes, y, 0);
        else tma_load_3d(dst, m, fb, x_bytes, y, 0);
      };
      if (!a_mn) {
        load(sa, ma, kb * kRowBytes, m0);
      } else {
#pragma unroll
        for (int j = 0; j < kTM / kK16; ++j) load(sa + j * kK16 * kRowBytes, ma, (m0 + j * kK16) * 2, kb * kK16);
      }
      if (!b_mn) {
        load(sb, mb, kb * kRowBytes, n0);
      } else {
#pragma unroll
        for (int j = 0; j < kTN / NCTA / kK16; ++j) load(sb + j * kK16 * kRowBytes, mb, (n0 + j * kK16) * 2, kb * kK16);
      }
      ++issued;
      if (++stage == stages) { stage = 0; phase ^= 1u; }
    }
    return true;
  }
  // after a timeout: wait (bounded) for the last use of every ring slot, so that no copy is in flight when the CTA exits
  __device__ __forceinline__ void drain_copies() {
    if (rank != 0u) return;
    const int pending = issued < stages ? static_cast<int>(issued) : stages;
    uint32_t s = stage, ph = phase;
    for (int i = 0; i < pending; ++i) {
      if (s == 0) { s = stages - 1; ph ^= 1u; } else { --s; }
      const unsigned long long t0 = global_timer_ns();
      while (!mbar_try_wait(full_bar + 8 * s, ph) && global_timer_ns() - t0 < kWaitLimitNs) {}
    }
  }

  __device__ __forceinline__ static void commit(uint32_t bar) {
    if constexpr (NCTA == 2) umma_commit_pair(bar);
    else umma_commit(bar);
  }
  // ---- warp 1, lane 0 of the pair's first CTA: the MMAs of one tile
  template <bool F8>
  __device__ __forceinline__ bool multiply(int num_kb, uint32_t idesc, bool a_mn, bool b_mn) {  // (idesc has the width)
    const uint64_t a_desc = make_smem_desc(smem_a, a_mn ? kK16 * kRowBytes : 0u, 1024u);
    const uint64_t b_desc = make_smem_desc(smem_b, b_mn ? kK16 * kRowBytes : 0u, 1024u);
    const uint32_t a_inc = (a_mn ? 16 * kRowBytes : 32) >> 4, b_inc = (b_mn ? 16 * kRowBytes : 32) >> 4;  // per MMA: 32 bytes of K
    idesc |= (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16);
    if (!mbar_wait(acc_empty + 8 * acc, acc_phase ^ 1u, abort_flag)) return false;
    tc_fence_after();
    const uint32_t d_tmem = tmem_base + acc * kTN;
    for (int kb = 0; kb < num_kb; ++kb) {
      const uint64_t ad0 = a_desc + static_cast<uint64_t>(stage * (a_bytes >> 4));
      const uint64_t bd0 = b_desc + static_cast<uint64_t>(stage * (b_bytes >> 4));
      if (!mbar_wait(full_bar + 8 * stage, phase, abort_flag)) return false;
      tc_fence_after();
#pragma unroll
      for (int k = 0; k < 4; ++k) umma<F8, NCTA>(d_tmem, ad0 + k * a_inc, bd0 + k * b_inc, idesc, (kb | k) != 0 ? 1u : 0u);
      commit(empty_bar + 8 * stage);  // the slot is free (in both CTAs) once these MMAs have read it
      if (++stage == stages) { stage = 0; phase ^= 1u; }
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

  __device__ __forceinline__ LaneRow staging() const { return LaneRow{reinterpret_cast<uint32_t*>(stage_mem + ((warp - 2) * 32 + lane) * 128), lane}; }
  // ---- warps 2-9: waits for the accumulator, gives it back
  __device__ __forceinline__ bool wait_accumulator() {
    if (!__all_sync(0xFFFFFFFFu, mbar_wait(acc_full + 8 * acc, acc_phase, abort_flag))) return false;
    tc_fence_after();
    return true;
  }
  // f(32 columns of this lane's row, chunk) for the chunks of this warp's half that lie inside the matrix (`cols` of them
  // from the half's first one); the next chunk is read while f works on the current one
  template <class F> __device__ __forceinline__ void each_chunk(int half, int half_cols, int cols, F f) {
    const uint32_t t_addr = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16) + acc * kTN + half * half_cols;
    const int n_chunks = max(0, min(half_cols, cols) + 31) / 32;
    uint32_t ra[32], rb[32];
    if (n_chunks > 0) tmem_ld32(t_addr, ra);
#pragma unroll 1
    for (int c = 0; c < n_chunks; c += 2) {
      tmem_ld_wait();
      if (c + 1 < n_chunks) tmem_ld32(t_addr + (c + 1) * 32, rb);
      f(ra, c);
      __syncwarp();
      if (c + 1 < n_chunks) {
        tmem_ld_wait();
        if (c + 2 < n_chunks) tmem_ld32(t_addr + (c + 2) * 32, ra);
        f(rb, c + 1);
        __syncwarp();
      }
    }
  }
  // f(32 columns of this lane's row, chunk as a constant) for every chunk of this warp's half
  template <class F> __device__ __forceinline__ void each_chunk_in_order(int half, int half_cols, F f) {
    const uint32_t t_addr = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16) + acc * kTN + half * half_cols;
    uint32_t r[32];
    auto one = [&](auto chunk) {
      constexpr int c = decltype(chunk)::value;
      if (c * 32 < half_cols) {
        tmem_ld32(t_addr + c * 32, r);
        tmem_ld_wait();
        f(r, chunk);
      }
    };
    one(std::integral_constant<int, 0>());
    one(std::integral_constant<int, 1>());
    one(std::integral_constant<int, 2>());
    one(std::integral_constant<int, 3>());
  }
  // f(32 columns of this lane's row, chunk) of one tile; SUMS: its contraction may take several accumulators, whose sums so far
  // wait in memory, of which every lane reads back only what it has written itself (`sums`: this warp's, a chunk after the other, pieces of
  // 16 bytes lane by lane).
  template <bool SUMS, class F> __device__ __forceinline__ bool tile_chunks(int num_kb, int part_kb, int half, int half_cols, int cols, float* sums, F f) {
    if constexpr (!SUMS) {
      if (!wait_accumulator()) return false;
      each_chunk(half, half_cols, cols, f);
      release_accumulator();
    } else {
      for (int kb = 0; kb < num_kb; kb += part_kb) {
        if (!wait_accumulator()) return false;
        const bool first = kb == 0, last = kb + part_kb >= num_kb;
        each_chunk(half, half_cols, cols, [&](uint32_t* r, int c) {
          char* at = reinterpret_cast<char*>(sums) + c * 4096 + lane * 16;
          if (!first) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              uint32_t before[4];
              ld_raw<16>(at + j * 512, before);
#pragma unroll
              for (int i = 0; i < 4; ++i) r[4 * j + i] = __float_as_uint(__uint_as_float(r[4 * j + i]) + __uint_as_float(before[i]));
            }
          }
          if (last) {
            f(r, c);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) st_raw<16>(at + j * 512, r + 4 * j);
          }
        });
        release_accumulator();
      }
    }
    return true;
  }
  __device__ __forceinline__ void release_accumulator() {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) {
      if constexpr (NCTA == 2) mbar_arrive_cluster(map_to_cta(acc_empty + 8 * acc, 0u));
      else mbar_arrive(acc_empty + 8 * acc);
    }
    if (++acc == kAccs) { acc = 0; acc_phase ^= 1u; }
  }
};

// ------------------------------------------------------------------------------------------------- logits kernel
struct Entry { int id; float q; };  // a row's target entries, those of the tiles' first halves first, each part sorted by id

struct LogitsParams {
  int n, cols;               // rows; columns (of this piece of the vocabulary)
  long long col0;            // the piece's first column
  int num_kb;
  Ring ring;
  int box_rows;              // rows of A that are copied
  int half_cols;             // of a tile: what one epilogue warp takes (32 to 128)
  int tiles_m, tiles_n, run; // a work item: one row tile, `run` consecutive column tiles
  long long items;
  uint32_t idesc;
  bool early;                // the kernel before writes nothing that the products read: they need not wait for it
  const float* h_scale; const float* w_scale;
  float inv_temp;
  // targets
  const long long* ids; long long padding_id, vocab;  // cross entropy
  const Entry* entries; const int2* counts; int k;    // distillation: [n][k]; entries in first halves, in both
  const uint16_t* table; int bins, bin_tiles;         // [n][2][bins]: where a bin of bin_tiles tiles begins, per half
  // forward: per run and half, and row
  float2* partial;           // maximum (base-2 units), sum
  float* dot;                // sum of q z
  long long ld_part;
  // gradient
  const float* lse;
  const float2* coef;        // of p and of q
  uint16_t* d_low; long long ldd;  // the second half of D, if it has one: rows of whole tiles
  uint32_t* status;
};

// The row's entries in this warp's half of the column tiles, in ascending order; the one after the current one is on its way.
template <bool KD> struct Targets {
  int id = INT_MAX;
  float q = 0.f;
  static constexpr int kAhead = 3;  // entries on their way: frequent tokens give a row many in a few tiles
  int2 ahead[kAhead];
  const Entry* at = nullptr;
  const Entry* end = nullptr;
  __device__ __forceinline__ int2 load(const Entry* e) const { return e < end ? ld_written(reinterpret_cast<const int2*>(e)) : make_int2(INT_MAX, 0); }
  // entries of the tile with the given first column, and of those behind it
  __device__ __forceinline__ void start(const LogitsParams& p, int row, int half, long long first) {
    id = INT_MAX;
    if constexpr (!KD) {
      if (row >= p.n) return;
      const long long t = ld_written(p.ids + row);
      if (t != p.padding_id && t >= first && t < p.vocab && (static_cast<uint32_t>(t) / p.half_cols & 1u) == static_cast<uint32_t>(half)) { id = static_cast<int>(t); q = 1.0f; }
    } else {
      at = end = nullptr;
      if (row < p.n) {
        const uint32_t bin = static_cast<uint32_t>(first) / (2 * p.half_cols * p.bin_tiles);
        const int2 c = ld_written(p.counts + row);
        const Entry* e = p.entries + static_cast<long long>(row) * p.k;
        at = e + ld_written(p.table + static_cast<long long>(row) * 2 * p.bins + half * p.bins + bin);
        end = e + (half ? c.y : c.x);
        if (p.bin_tiles > 1)
          while (at < end && ld_written(&at->id) < first) ++at;
      }
      const int2 e0 = load(at);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ahead[i] = load(at + 1 + i);
      at += 1 + kAhead;
      id = e0.x;
      q = __int_as_float(e0.y);
    }
  }
  __device__ __forceinline__ void advance() {
    if constexpr (!KD) {
      id = INT_MAX;
    } else {
      id = ahead[0].x;
      q = __int_as_float(ahead[0].y);
#pragma unroll
      for (int i = 0; i + 1 < kAhead; ++i) ahead[i] = ahead[i + 1];
      ahead[kAhead - 1] = load(at);
      ++at;
    }
  }
};

// r[i], i in 0..31 known at run time only
__device__ __forceinline__ float pick32(const uint32_t* r, int i) {
  uint32_t a[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) a[j] = (i & 16) ? r[j + 16] : r[j];
#pragma unroll
  for (int w = 8; w >= 1; w >>= 1)
#pragma unroll
    for (int j = 0; j < w; ++j) a[j] = (i & w) ? a[j + w] : a[j];
  return __uint_as_float(a[0]);
}

// LONG: the tensor cores add up with truncation, an error that grows with the number of additions and the sums' size, and the
// losses are fp32: from kLongKb K blocks on, every kSegmentKb of them go to an accumulator of their own, and the epilogue warps
// add those up in registers while the next ones are filled (4096 x 128000 x 4096, 16 bits: errors of lse and loss 1.3e-6 and 2.0e-6
// of their norm in one accumulator; 2000 x 5000 x 4096 in these parts 1.2e-7 and 1.6e-7; in the same time).  Three or four chunks of
// sums beside the work on one: 136 bytes of registers spill, 264 with a teacher's entries.
template <int NCTA, bool F8, bool KD, bool LONG>
__global__ void __launch_bounds__(kThreads, 1) logits_kernel(const __grid_constant__ CUtensorMap map_h,
                                                             const __grid_constant__ CUtensorMap map_w, const LogitsParams p) {
  asm volatile("griddepcontrol.launch_dependents;");  // the next kernel may set up while this one runs
  extern __shared__ uint8_t smem_raw[];
  Engine<NCTA> e;
  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_h)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_w)) : "memory");
  }
  e.set_up(smem_raw, p.ring, KD);
  // nothing above touches what the kernel before writes
  if (!p.early || e.warp >= 2) asm volatile("griddepcontrol.wait;" ::: "memory");
  const int unit = blockIdx.x / NCTA, num_units = gridDim.x / NCTA;
  bool timed_out = false;
  if (e.warp == 0) {
    if (e.lane == 0) {
      for (long long item = unit; item < p.items && !timed_out; item += num_units) {
        const int mt = static_cast<int>(item % p.tiles_m), nt0 = static_cast<int>(item / p.tiles_m) * p.run;
        for (int nt = nt0; nt < min(nt0 + p.run, p.tiles_n) && !timed_out; ++nt)
          timed_out = !e.produce(&map_h, &map_w, mt * Cfg<NCTA>::kTileM, nt * 2 * p.half_cols, p.box_rows, 2 * p.half_cols, 0, p.num_kb, false, false);
      }
      if (timed_out || *e.abort_flag) e.drain_copies();
    }
  } else if (e.warp == 1) {
    if (e.lane == 0 && e.rank == 0u) {
      for (long long item = unit; item < p.items && !timed_out; item += num_units) {
        const int nt0 = static_cast<int>(item / p.tiles_m) * p.run;
        for (int nt = nt0; nt < min(nt0 + p.run, p.tiles_n) && !timed_out; ++nt) {
          if constexpr (LONG) {
            for (int kb = 0; kb < p.num_kb && !timed_out; kb += kSegmentKb<NCTA>) timed_out = !e.template multiply<F8>(min(kSegmentKb<NCTA>, p.num_kb - kb), p.idesc, false, false);
          } else {
            timed_out = !e.template multiply<F8>(p.num_kb, p.idesc, false, false);
          }
        }
      }
      if (timed_out || *e.abort_flag) e.drain_multiplies();
    }
  } else {
    const int half = (e.warp - 2) >> 2, quarter = e.warp & 3;
    const float c2 = load_scale_after_wait(p.h_scale) * load_scale_after_wait(p.w_scale) * p.inv_temp * kLog2E;
    Targets<KD> target;
    const LaneRow lane_row = e.staging();
    for (long long item = unit; item < p.items && !timed_out; item += num_units) {
      const int mt = static_cast<int>(item % p.tiles_m), ng = static_cast<int>(item / p.tiles_m), nt0 = ng * p.run;
      const int row = mt * Cfg<NCTA>::kTileM + static_cast<int>(e.rank) * kTM + quarter * 32 + e.lane;
      const bool warp_rows = row - e.lane < p.n;  // whether any of this warp's rows exists
      target.start(p, row, half, static_cast<long long>(nt0) * 2 * p.half_cols);
      float top = -INFINITY, sum = 0.f, dot = 0.f;
      for (int nt = nt0; nt < min(nt0 + p.run, p.tiles_n); ++nt) {
        const int n0 = (2 * nt + half) * p.half_cols;
        auto work = [&](uint32_t* r, int c) {
          const int c0 = n0 + c * 32, valid = p.cols - c0;
          if (__any_sync(0xFFFFFFFFu, target.id < c0 + 32ll)) {
            if constexpr (KD) {
              lane_row.put(r);
              while (target.id < c0 + 32ll) {
                if (target.q != 0.f) dot = fmaf(target.q, lane_row.at(target.id - c0), dot);  // (0 times -inf is nothing)
                target.advance();
              }
              __syncwarp();
            } else {
              const float z = pick32(r, (target.id - c0) & 31);
              if (target.id < c0 + 32ll) {
                dot = z;
                target.advance();
              }
            }
          }
          if (valid < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (i >= valid) r[i] = 0xFF800000u;  // -inf
          }
          float m = __uint_as_float(r[0]);
#pragma unroll
          for (int i = 1; i < 32; ++i) m = fmaxf(m, __uint_as_float(r[i]));
          // (a row with +inf: relative to the largest finite number, to which finite exponents are nothing and infinite ones inf)
          m = fminf(m * c2, kLargest);
          if (m > top) {  // (a row of -inf so far: sum is 0)
            sum *= exp2_approx(top - m);
            top = m;
          }
          const float shift = top == -INFINITY ? 0.f : -top;
          float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 32; ++i) s[i & 3] += exp2_approx(fmaf(__uint_as_float(r[i]), c2, shift));
          sum += (s[0] + s[1]) + (s[2] + s[3]);
        };
        const int cols = warp_rows ? p.cols - n0 : 0;
        if constexpr (LONG) {
          float z[kTN / 64][32];
          for (int kb = 0; kb < p.num_kb && !timed_out; kb += kSegmentKb<NCTA>) {
            if (!e.wait_accumulator()) { timed_out = true; break; }
            e.each_chunk_in_order(half, p.half_cols, [&](const uint32_t* r, auto chunk) {
              constexpr int c = decltype(chunk)::value;
#pragma unroll
              for (int i = 0; i < 32; ++i) z[c][i] = kb == 0 ? __uint_as_float(r[i]) : z[c][i] + __uint_as_float(r[i]);
            });
            e.release_accumulator();
          }
          if (timed_out) break;
#pragma unroll
          for (int c = 0; c < kTN / 64; ++c)
            if (c * 32 < min(p.half_cols, cols)) work(reinterpret_cast<uint32_t*>(z[c]), c);
        } else {
          if (!e.wait_accumulator()) { timed_out = true; break; }
          e.each_chunk(half, p.half_cols, cols, work);
          e.release_accumulator();
        }
      }
      if (row < p.n && !timed_out) {
        const long long o = static_cast<long long>(ng * 2 + half) * p.ld_part + row;
        p.partial[o] = make_float2(top, sum);
        p.dot[o] = dot;
      }
    }
  }
  if (timed_out) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_TIMEOUT));
  e.tear_down();
}

// ------------------------------------------------------------------------------------------------- gradient kernel
// What the CTA pairs of one launch share: tiles of the products dW = D^T H and dH = D W of one piece of the vocabulary, and of
// the logits (the gradient D) of the NEXT piece, which fill the pairs up to equal loads whatever the products' tiles leave.
enum { kClassDw = 0, kClassDh = 1, kClassD = 2, kClasses = 3 };
constexpr int kSms = 148;         // of the GPU, which sizes are planned for, whatever the launch finds
constexpr int kMaxUnits = kSms;
constexpr int kWarpSums = 4 * 32 * 32;
constexpr int kListed = 48;
struct Schedule {
  int order[kClasses];               // long tiles first
  int total[kClasses];
  int quota[kClasses][kMaxUnits];    // of every pair
};
// The j-th item of a pair: numbered so that the pairs work on neighbouring items and finish together (pairs with a smaller
// quota join later): counted from the end, round b holds the pairs with a quota above b.
__device__ __forceinline__ int scheduled_item(const Schedule& s, int cls, int unit, int units, int j) {
  const int b = s.quota[cls][unit] - 1 - j;
  int behind = 0;
  for (int u = 0; u < units; ++u) {
    const int q = s.quota[cls][u];
    behind += min(q, b) + (u < unit && q > b);
  }
  return s.total[cls] - 1 - behind;
}

enum { kFinal = 0, kAccFirst = 1, kAccNext = 2, kAccLast = 3 };  // what a product does with the fp32 sums of earlier pieces
struct GradProduct {
  int M, N, num_kb;
  int tiles_n;
  int parts, part_kb;   // the contraction in parts, one plane of sums each
  void* out;
  long long ldo;
  int out_dt;
  float alpha;
  int mode;
  float* acc;           // [parts][M][ld_acc]
  long long ld_acc;
};
struct GradParams {
  Schedule schedule;
  GradProduct product[2];  // dW, dH
  LogitsParams logits;
  uint32_t idesc;          // of the products
  const float* unit;       // [0]: what D is stored times; [1]: what its products are multiplied by
  float* sums;             // per CTA and epilogue warp four chunks, where a contraction takes several accumulators
};
struct GradItem { int mt, nt, part; };  // row tile, (first) column tile, part of the contraction
__device__ __forceinline__ GradItem grad_item(const GradParams& p, int cls, int item) {
  if (cls == kClassD) return GradItem{item % p.logits.tiles_m, item / p.logits.tiles_m * p.logits.run, 0};
  // (column tiles of one row tile beside each other: they share D)
  const GradProduct& g = p.product[cls];
  const int t = item / g.parts, mt = t / g.tiles_n;
  return GradItem{mt, t - mt * g.tiles_n, item - t * g.parts};
}
struct GradMaps { CUtensorMap h, w, d_mn, h_mn, d_k, w_mn, d_out; };

// SUMS: the logits' contraction is longer than kLogitKb blocks, or a product's than kSumKb.  (A kernel of its own: the test for it in
// the epilogue costs the FP8 step 8192 x 768 3 %.)
template <int NCTA, bool F8, bool KD, bool BF, bool SUMS>
__global__ void __launch_bounds__(kThreads, 1) loss_grad_kernel(const __grid_constant__ GradMaps maps, const __grid_constant__ GradParams p) {
  asm volatile("griddepcontrol.launch_dependents;");  // the next kernel may set up while this one runs
  extern __shared__ uint8_t smem_raw[];
  Engine<NCTA> e;
  const int unit = blockIdx.x / NCTA, units = gridDim.x / NCTA;
  if (threadIdx.x < 6 && p.schedule.total[threadIdx.x < 2 ? kClassD : threadIdx.x < 4 ? kClassDw : kClassDh] > 0)  // (the others are not filled in)
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&maps.h + threadIdx.x)) : "memory");
  __shared__ GradItem s_item[kClasses][kListed];  // this pair's first items
  for (int i = threadIdx.x; i < kClasses * kListed; i += kThreads) {
    const int cls = i / kListed, j = i % kListed;
    if (j < p.schedule.quota[cls][unit]) s_item[cls][j] = grad_item(p, cls, scheduled_item(p.schedule, cls, unit, units, j));
  }
  e.set_up(smem_raw, p.logits.ring, true);
  // nothing above touches what the kernel before writes
  if (!p.logits.early || e.warp >= 2) asm volatile("griddepcontrol.wait;" ::: "memory");
  const LogitsParams& l = p.logits;
  bool timed_out = false;
  // every role walks the same items: f(class, item)
  auto each_item = [&](auto f) {
    for (int k = 0; k < kClasses && !timed_out; ++k) {
      const int cls = p.schedule.order[k], mine = p.schedule.quota[cls][unit];
      for (int j = 0; j < mine && !timed_out; ++j) f(cls, j < kListed ? s_item[cls][j] : grad_item(p, cls, scheduled_item(p.schedule, cls, unit, units, j)));
    }
  };
  auto part_kbs = [&](const GradProduct& g, int part) { return min(g.part_kb, g.num_kb - part * g.part_kb); };
  if (e.warp == 0) {
    if (e.lane == 0) {
      asm volatile("fence.proxy.async;" ::: "memory");  // the copies read what ordinary stores have written
      each_item([&](int cls, const GradItem& item) {
        if (cls == kClassD) {
          for (int nt = item.nt; nt < min(item.nt + l.run, l.tiles_n) && !timed_out; ++nt)
            timed_out = !e.produce(&maps.h, &maps.w, item.mt * Cfg<NCTA>::kTileM, nt * 2 * l.half_cols, l.box_rows, 2 * l.half_cols, 0, l.num_kb, false, false);
        } else {
          const GradProduct& g = p.product[cls];
          const int m0 = item.mt * Cfg<NCTA>::kTileM, n0 = item.nt * kTN, kbs = part_kbs(g, item.part);
          timed_out = cls == kClassDw ? !e.produce(&maps.d_mn, &maps.h_mn, m0, n0, kTM, kTN, item.part * g.part_kb, kbs, true, true)
                                      : !e.produce(&maps.d_k, &maps.w_mn, m0, n0, kTM, kTN, item.part * g.part_kb, kbs, false, true);
        }
      });
      if (timed_out || *e.abort_flag) e.drain_copies();
    }
  } else if (e.warp == 1) {
    if (e.lane == 0 && e.rank == 0u) {
      const int logit_kb = SUMS ? kLogitKb : INT_MAX / 2, sum_kb = SUMS ? kSumKb : INT_MAX / 2;
      each_item([&](int cls, const GradItem& item) {
        if (cls == kClassD) {
          for (int nt = item.nt; nt < min(item.nt + l.run, l.tiles_n); ++nt)
            for (int kb = 0; kb < l.num_kb && !timed_out; kb += logit_kb) timed_out = !e.template multiply<F8>(min(logit_kb, l.num_kb - kb), l.idesc, false, false);
        } else {
          const int kbs = part_kbs(p.product[cls], item.part);
          for (int kb = 0; kb < kbs && !timed_out; kb += sum_kb) timed_out = !e.template multiply<false>(min(sum_kb, kbs - kb), p.idesc, cls == kClassDw, true);
        }
      });
      if (timed_out || *e.abort_flag) e.drain_multiplies();
    }
  } else {
    const int half = (e.warp - 2) >> 2, quarter = e.warp & 3;
    const int own_row = static_cast<int>(e.rank) * kTM + quarter * 32 + e.lane;
    const LaneRow lane_row = e.staging();
    uint32_t flip = 0;
    float* const sums = p.sums + (static_cast<long long>(blockIdx.x) * kEpiWarps + (e.warp - 2)) * kWarpSums;
    const float c2 = load_scale_after_wait(l.h_scale) * load_scale_after_wait(l.w_scale) * l.inv_temp * kLog2E;
    const float unit_d = reinterpret_cast<const volatile float*>(p.unit)[0], factor = reinterpret_cast<const volatile float*>(p.unit)[1];
    each_item([&](int cls, const GradItem& item) {
      if (cls == kClassD) {
        const int row = item.mt * Cfg<NCTA>::kTileM + own_row, nt0 = item.nt;
        Targets<KD> target;
        target.start(l, row, half, l.col0 + static_cast<long long>(nt0) * 2 * l.half_cols);
        float2 coef = make_float2(0.f, 0.f);
        float lse2 = 0.f;
        if (row < l.n) {
          coef = __ldcg(l.coef + row);
          coef.x *= unit_d; coef.y *= unit_d;
          lse2 = __ldcg(l.lse + row) * kLog2E;
        }
        for (int nt = nt0; nt < min(nt0 + l.run, l.tiles_n); ++nt) {
          const int n0 = (2 * nt + half) * l.half_cols;
          timed_out = !e.template tile_chunks<SUMS>(l.num_kb, kLogitKb, half, l.half_cols, row - e.lane < l.n ? l.cols - n0 : 0, sums, [&](uint32_t* r, int c) {
            const int c0 = n0 + c * 32;
            const long long g0 = l.col0 + c0;
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = coef.x * exp2_approx(fmaf(__uint_as_float(r[i]), c2, -lse2));
            if (__any_sync(0xFFFFFFFFu, target.id < g0 + 32)) {
              if constexpr (KD) {
                if (elected_lane()) bulk_wait_read<0>();
                __syncwarp();
                lane_row.put(reinterpret_cast<const uint32_t*>(v));
                while (target.id < g0 + 32) {
                  lane_row.at(static_cast<int>(target.id - g0)) -= coef.y * target.q;
                  target.advance();
                }
                __syncwarp();
                lane_row.get(reinterpret_cast<uint32_t*>(v));
              } else if (target.id < g0 + 32) {
                const int at = static_cast<int>(target.id - g0);
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (i == at) v[i] -= coef.y;
                target.advance();
              }
            }
            constexpr int kD = BF ? SCALIFY_BF16 : SCALIFY_F16;
            uint32_t o[16];
            if (NCTA == 1 && l.d_low != nullptr) {
              char* low = reinterpret_cast<char*>(l.d_low + row * l.ldd + c0);  // (rows are whole tiles)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                float high[8];
                uint32_t rest[4];
                encode_vec<kD, 8>(v + 8 * j, o + 4 * j);
                decode_vec<kD, 8>(o + 4 * j, high);
#pragma unroll
                for (int i = 0; i < 8; ++i) high[i] = v[8 * j + i] - high[i];
                encode_vec<kD, 8>(high, rest);
                if (row < l.n) st_bytes<16>(low + j * 16, rest);
              }
            } else {
              encode_vec<kD, 32>(v, o);
            }
            lane_row.store(o, &maps.d_out, c0 * 2, row - e.lane, flip);
          });
          if (timed_out) break;
        }
      } else {
        const GradProduct& g = p.product[cls];
        const float alpha = g.alpha * factor;
        const int row = item.mt * Cfg<NCTA>::kTileM + own_row, n0 = item.nt * kTN + half * (kTN / 2);
        const int mode = g.mode;
        char* out_row = static_cast<char*>(g.out) + (static_cast<long long>(row) * g.ldo + n0) * 2;
        float* acc_row = g.acc + (static_cast<long long>(item.part) * g.M + row) * g.ld_acc + n0;  // (padded to whole chunks)
        timed_out = !e.template tile_chunks<SUMS>(part_kbs(g, item.part), kSumKb, half, kTN / 2, row - e.lane < g.M ? g.N - n0 : 0, sums, [&](uint32_t* r, int c) {
          float v[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
          char* acc = reinterpret_cast<char*>(acc_row + c * 32);
          if (mode >= kAccNext && row < g.M) {
            uint32_t before[32];
#pragma unroll
            for (int j = 0; j < 4; ++j) ld_bytes<32, false>(acc + j * 32, before + j * 8);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += __uint_as_float(before[i]);
          }
          if (mode == kAccFirst || mode == kAccNext) {
            if (row < g.M) {
#pragma unroll
              for (int j = 0; j < 4; ++j) st_bytes<32>(acc + j * 32, reinterpret_cast<const uint32_t*>(v) + j * 8);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= alpha;
            uint32_t o[16];
            if (g.out_dt == SCALIFY_BF16) encode_vec<SCALIFY_BF16, 32>(v, o);
            else encode_vec<SCALIFY_F16, 32>(v, o);
            // (straight from registers: where a tile is little but its store, the store engine would also have to fetch the next
            // ones' operands; 256 and 100 rows, vocabulary 50257 and 115392: 89 and 139 us so, 106 and 168 through it)
            const int left = g.N - n0 - c * 32;
            char* dst = out_row + c * 64;
            if (row < g.M) {
              if (left >= 32) {
                st_bytes<32>(dst, o);
                st_bytes<32>(dst + 32, o + 8);
              } else {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (i < left) reinterpret_cast<uint16_t*>(dst)[i] = static_cast<uint16_t>((i & 1) ? o[i / 2] >> 16 : o[i / 2]);
              }
            }
          }
        });
      }
    });
    if (elected_lane()) bulk_wait_all();  // every store of this warp has completed
  }
  if (timed_out) atomicOr(l.status, static_cast<uint32_t>(SCALIFY_DEV_TIMEOUT));
  e.tear_down();
}

// ------------------------------------------------------------------------------------------------- small kernels
// A teacher's entries: probabilities, sorted by (half of its tile, id), entries without a place in the vocabulary
// or with no probability mass at all (a logit of -inf) left out.  One warp per row; the order by counting the smaller ones.
struct TeacherParams {
  long long n, vocab;
  int k;
  const long long* ids; long long padding_id;
  const void* T; int t_dt; long long t_ld; const float* t_scale; const float* t_lse;
  float inv_temp;
  int half_cols;
  uint16_t* table; int bins, bin_tiles;
  Entry* entries; int2* counts; float2* sums;  // sums: Q, sum q log q
  uint32_t* status;
};
constexpr int kMaxBins = 256;
// TEAM warps share a row, kPer entries per lane; a block takes one row of several warps or four rows of one.
template <int kPer, int TEAM>
__global__ void __launch_bounds__(TEAM == 1 ? 128 : 32 * TEAM) teacher_kernel(const TeacherParams p) {
  constexpr int kRows = TEAM == 1 ? 4 : 1;
  __shared__ uint64_t s_entry[kRows][32 * kPer * TEAM];  // key, then place, bin after bin
  __shared__ int s_bin[kRows][2 * kMaxBins];
  __shared__ float s_part[4][TEAM];
  __shared__ int s_count[2][TEAM];
  const int warp = TEAM == 1 ? threadIdx.x >> 5 : 0, lane = threadIdx.x & 31;  // (warp: the row of the block)
  const int member = TEAM == 1 ? 0 : threadIdx.x >> 5, first = member * 32 + lane;
  const long long row = static_cast<long long>(blockIdx.x) * kRows + warp;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");  // (behind the wait: a dependent may read what was there before this kernel)
  if (row >= p.n) return;
  auto sync = [] {
    if constexpr (TEAM == 1) __syncwarp();
    else __syncthreads();
  };
  // over the row, in all its threads
  auto row_sum = [&](float x, int slot) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    if constexpr (TEAM > 1) {
      if (lane == 0) s_part[slot][member] = x;
      __syncthreads();
      x = 0.f;
      for (int i = 0; i < TEAM; ++i) x += s_part[slot][i];
    }
    return x;
  };
  const float scale = load_scale_after_wait(p.t_scale);
  if (row == 0 && first == 0 && !is_pow2_scale(scale)) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_SCALE));
  const float f = scale * p.inv_temp;
  float t[kPer];
  uint32_t key[kPer];
  float top = -INFINITY;
  bool bad = false;
  long long id[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {  // (all loads at once)
    const int i = j * 32 * TEAM + first;
    id[j] = i < p.k ? p.ids[row * p.k + i] : p.padding_id;
    const long long at = row * p.t_ld + i;
    t[j] = i >= p.k ? 0.f
           : p.t_dt == SCALIFY_F32 ? load_elem<SCALIFY_F32>(p.T, at)
           : p.t_dt == SCALIFY_BF16 ? load_elem<SCALIFY_BF16>(p.T, at) : load_elem<SCALIFY_F16>(p.T, at);
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int i = j * 32 * TEAM + first;
    const bool known = id[j] >= 0 && id[j] < p.vocab, wanted = i < p.k && id[j] != p.padding_id;
    const float x = t[j] * f;
    bad = bad || (wanted && !known);
    key[j] = 0xFFFFFFFFu;
    t[j] = -INFINITY;
    if (wanted && known && x != -INFINITY) {
      t[j] = x;
      key[j] = static_cast<uint32_t>(id[j]) | (static_cast<uint32_t>(id[j]) / p.half_cols & 1u) << 30;
      top = x > top || x != x ? x : top;
    }
  }
  if (bad) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_INDEX));
  float norm;
  if (p.t_lse) {
    norm = __ldcg(p.t_lse + row);
  } else {
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if constexpr (TEAM > 1) {
      if (lane == 0) s_part[0][member] = top;
      __syncthreads();
      for (int i = 0; i < TEAM; ++i) top = fmaxf(top, s_part[0][i]);
    }
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) s += key[j] != 0xFFFFFFFFu ? expf(t[j] - top) : 0.f;
    norm = logf(row_sum(s, 1)) + top;
  }
  for (int i = first; i < 2 * p.bins; i += 32 * TEAM) s_bin[warp][i] = 0;
  sync();
  // counted by bins; a bin's entries come after those of the bins before it, in any order at first
  int bin[kPer], slot[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const uint32_t block = (key[j] & 0x3FFFFFFFu) / static_cast<uint32_t>(p.half_cols);  // 2 tile + half
    bin[j] = static_cast<int>((block & 1u) * p.bins + (block >> 1) / p.bin_tiles);
    if (key[j] != 0xFFFFFFFFu) slot[j] = atomicAdd(&s_bin[warp][bin[j]], 1);
  }
  sync();
  int begin = 0;
  for (int i0 = 0; i0 < 2 * p.bins && member == 0; i0 += 32) {
    const int i = i0 + lane, mine = i < 2 * p.bins ? s_bin[warp][i] : 0;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += u;
    }
    if (i < 2 * p.bins) {
      p.table[row * 2 * p.bins + i] = static_cast<uint16_t>(begin + upto - mine);
      s_bin[warp][i] = (begin + upto - mine) << 16 | mine;
    }
    begin += __shfl_sync(0xFFFFFFFFu, upto, 31);
  }
  sync();
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (key[j] != 0xFFFFFFFFu)
      s_entry[warp][(s_bin[warp][bin[j]] >> 16) + slot[j]] = static_cast<uint64_t>(key[j]) << 32 | static_cast<uint32_t>(j * 32 * TEAM + first);
  sync();
  int there = 0, even = 0;
  float mass = 0.f, neg = 0.f;
  Entry* out = p.entries + row * p.k;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const bool ok = key[j] != 0xFFFFFFFFu;
    there += __popc(__ballot_sync(0xFFFFFFFFu, ok));
    even += __popc(__ballot_sync(0xFFFFFFFFu, key[j] < (1u << 30)));
    const float lq = t[j] - norm, q = ok ? expf(lq) : 0.f;
    mass += q;
    neg += ok && q != 0.f ? q * lq : 0.f;
    if (ok) {  // its place within the bin: by id, equal ones by place
      const uint64_t mine = static_cast<uint64_t>(key[j]) << 32 | static_cast<uint32_t>(j * 32 * TEAM + first);
      const int b = s_bin[warp][bin[j]], begins = b >> 16, many = b & 0xFFFF;
      int before = begins;
      for (int m = 0; m < many; ++m) before += s_entry[warp][begins + m] < mine;
      out[before] = Entry{static_cast<int>(key[j] & 0x3FFFFFFFu), q};
    }
  }
  mass = row_sum(mass, 2);
  neg = row_sum(neg, 3);
  if constexpr (TEAM > 1) {
    if (lane == 0) { s_count[0][member] = even; s_count[1][member] = there; }
    __syncthreads();
    even = there = 0;
    for (int i = 0; i < TEAM; ++i) { even += s_count[0][i]; there += s_count[1][i]; }
  }
  if (first == 0) {
    p.counts[row] = make_int2(even, there);
    p.sums[row] = make_float2(mass, neg);
  }
}

// Whether a row counts, and (distillation) its Q and sum q log q
__device__ __forceinline__ bool row_target(const long long* ids, long long padding_id, long long vocab, const int2* counts,
                                           const float2* sums, long long row, float2* qe, bool* bad) {
  if (counts) {
    *qe = __ldcg(sums + row);
    return __ldcg(counts + row).y > 0;
  }
  const long long t = __ldcg(ids + row);
  *qe = make_float2(1.f, 0.f);
  if (t == padding_id) return false;
  const bool ok = t >= 0 && t < vocab;
  *bad = *bad || !ok;
  return ok;
}

struct JoinParams {
  long long n, vocab;
  int slots;
  const float2* partial; const float* dot; long long ld_part;
  const float* h_scale; const float* w_scale;
  float inv_temp, z_loss;
  const long long* ids; long long padding_id;
  const int2* counts; const float2* sums;
  float* loss; float* lse; float* mean;
  int rows_log;            // rows per block
  double2* block_sums;     // sum of losses, rows that count
  uint32_t* ticket; uint32_t* status;
};
constexpr int kJoinThreads = 256;
__device__ __forceinline__ void warp_sums(double& x, double& y) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    y += __shfl_xor_sync(0xFFFFFFFFu, y, o);
  }
}
// Joins a row's partial results: 256 >> rows_log threads share a row (at most 32 rows a block, the first warp's).  The mean is
// the sum of the blocks' fp64 sums, in a fixed order, by the block that is done last.
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const JoinParams p) {
  asm volatile("griddepcontrol.launch_dependents;");
  __shared__ float s_top[kJoinThreads], s_sum[kJoinThreads], s_dot[kJoinThreads];
  __shared__ double s_a[kJoinThreads / 32], s_b[kJoinThreads / 32];
  __shared__ bool s_last;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int rows = 1 << p.rows_log, lr = threadIdx.x & (rows - 1), part = threadIdx.x >> p.rows_log, parts = kJoinThreads >> p.rows_log;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long row = (static_cast<long long>(blockIdx.x) << p.rows_log) + lr;
  float top = -INFINITY, sum = 0.f, dot = 0.f;
  if (row < p.n) {
    constexpr int kBatch = 8;  // loads in flight
    for (int s0 = part; s0 < p.slots; s0 += parts * kBatch) {
      float2 v[kBatch];
      float d[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int s = s0 + j * parts;
        const long long o = static_cast<long long>(s) * p.ld_part + row;
        v[j] = s < p.slots ? __ldcg(p.partial + o) : make_float2(-INFINITY, 0.f);
        d[j] = s < p.slots ? __ldcg(p.dot + o) : 0.f;
      }
      float m = top;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) m = fmaxf(m, v[j].x);
      const float shift = m == -INFINITY ? 0.f : m;
      sum *= exp2f(top - shift);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        sum = fmaf(v[j].y, exp2f(v[j].x - shift), sum);
        dot += d[j];
      }
      top = m;
    }
  }
  // a row's threads in pairs: through shared memory while they lie in different warps, then by shuffles
  auto join = [&](float top2, float sum2, float dot2) {
    const float m = fmaxf(top, top2), shift = m == -INFINITY ? 0.f : m;
    sum = sum * exp2f(top - shift) + sum2 * exp2f(top2 - shift);
    dot += dot2;
    top = m;
  };
  for (int half = parts / 2; half > 0; half /= 2) {
    if (half << p.rows_log >= 32) {
      __syncthreads();
      s_top[threadIdx.x] = top; s_sum[threadIdx.x] = sum; s_dot[threadIdx.x] = dot;
      __syncthreads();
      const int other = threadIdx.x + (half << p.rows_log);
      if (part < half) join(s_top[other], s_sum[other], s_dot[other]);
    } else {
      const float t2 = __shfl_down_sync(0xFFFFFFFFu, top, half << p.rows_log), s2 = __shfl_down_sync(0xFFFFFFFFu, sum, half << p.rows_log);
      const float d2 = __shfl_down_sync(0xFFFFFFFFu, dot, half << p.rows_log);
      if (part < half) join(t2, s2, d2);
    }
  }
  double total = 0.0, count = 0.0;
  if (warp == 0) {
    if (part == 0 && row < p.n) {
      const float lse = (top + log2f(sum)) * 0.6931471805599453f;
      const float hw = load_scale_after_wait(p.h_scale) * load_scale_after_wait(p.w_scale);
      float2 qe;
      bool bad = false;
      const bool counts = row_target(p.ids, p.padding_id, p.vocab, p.counts, p.sums, row, &qe, &bad);
      if (bad) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_INDEX));
      const float mass = qe.x != 0.f ? qe.x * lse : 0.f;  // (0 times inf is nothing)
      const float loss = counts ? qe.y + (mass - dot * (hw * p.inv_temp)) + (p.z_loss > 0.f ? p.z_loss * lse * lse : 0.f) : 0.f;
      p.loss[row] = loss;
      p.lse[row] = lse;
      total = loss;
      count = counts ? 1.0 : 0.0;
      if (row == 0 && (!is_pow2_scale(load_scale_after_wait(p.h_scale)) || !is_pow2_scale(load_scale_after_wait(p.w_scale))))
        atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_SCALE));
    }
    if (p.mean) {
      warp_sums(total, count);
      if (lane == 0) {
        if (gridDim.x == 1) {
          *p.mean = static_cast<float>(total / (count > 0.0 ? count : 1.0));
          s_last = false;
        } else {
          p.block_sums[blockIdx.x] = make_double2(total, count);
          __threadfence();
          s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
        }
      }
    }
  }
  if (!p.mean) return;
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  total = 0.0; count = 0.0;
  for (unsigned b = threadIdx.x; b < gridDim.x; b += kJoinThreads) {
    const double2 v = __ldcg(p.block_sums + b);
    total += v.x; count += v.y;
  }
  warp_sums(total, count);
  if (lane == 0) { s_a[warp] = total; s_b[warp] = count; }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kJoinThreads / 32; ++i) { total += s_a[i]; count += s_b[i]; }
    *p.mean = static_cast<float>(total / (count > 0.0 ? count : 1.0));
    *p.ticket = 0u;
  }
}

// FP8 rows -> FP16 (exact), of H and then of W; H (16-bit rows too) as often as D has halves
struct WidenParams {
  const void* src[2]; __half* dst[2];
  long long ld[2], ldd, rows[2];
  int dt[2];
  long long n;   // rows of H itself
  int d;
};
struct CoefParams {
  long long n, vocab;
  const long long* ids; long long padding_id;
  const int2* counts; const float2* sums;
  const float* lse;
  float z_loss, rest;       // rest: 1/T without its power of two
  float inv_temp_p2;
  const float* grad; const float* grad_scale;
  float mean_p2;            // without grad: 1/n rounded down to a power of two
  const float* h_scale; const float* w_scale;
  float kf_vocab, kf_n;
  float2* coef;
  uint2* block_tops;        // per block: largest coefficient (bits), rows that count
  float* unit;              // [0]: what D is stored times; [1]: what its products are multiplied by
  float* dh_scale; float* dw_scale;
  uint32_t* ticket; uint32_t* status;
  int blocks;               // of the coefficients; the blocks behind them make the FP16 copies
  WidenParams widen;
};
constexpr int kCoefThreads = 256;
constexpr int kCoefBlocks = 256;
__device__ __forceinline__ void widen_rows(const WidenParams& p, int block, int blocks) {
  const int vecs = (p.d + 15) / 16;
  const long long total = (p.rows[0] + p.rows[1]) * vecs;
  for (long long i = static_cast<long long>(block) * kCoefThreads + threadIdx.x; i < total; i += static_cast<long long>(blocks) * kCoefThreads) {
    long long row = i / vecs;
    const int v = static_cast<int>(i - row * vecs), n = p.d - v * 16;
    const int which = row >= p.rows[0];
    if (which) row -= p.rows[0];
    const long long from = which == 0 && row >= p.n ? row - p.n : row;
    uint32_t w[4] = {}, o[8] = {};
    if (p.dt[which] >= SCALIFY_F16) {
      const char* src = static_cast<const char*>(p.src[which]) + from * p.ld[which] * 2;
      load_vec<SCALIFY_F16>(src, 2 * v, n, o);
      if (n > kVec) load_vec<SCALIFY_F16>(src, 2 * v + 1, n - kVec, o + 4);
    } else {
      const char* src = static_cast<const char*>(p.src[which]) + from * p.ld[which];
      float f[16];
      if (n >= 16) {
        ld_raw<16>(src + v * 16, w);
      } else {
        load_vec<SCALIFY_E4M3>(src, 2 * v, n, w);
        if (n > kVec) load_vec<SCALIFY_E4M3>(src, 2 * v + 1, n - kVec, w + 2);
      }
      if (p.dt[which] == SCALIFY_E4M3) decode_vec<SCALIFY_E4M3, 16>(w, f);
      else decode_vec<SCALIFY_E5M2, 16>(w, f);
      encode_vec<SCALIFY_F16, 16>(f, o);
    }
    st_bytes<32>(reinterpret_cast<char*>(p.dst[which] + row * p.ldd + v * 16), o);  // (rows are padded to whole vectors)
  }
}
// Row coefficients of p and of q in units of the upstream gradient (of the mean's, if there is none); what D
// is stored times; output scales; FP16 copies of FP8 operands.
__global__ void __launch_bounds__(kCoefThreads) coef_kernel(const __grid_constant__ CoefParams p) {
  __shared__ uint32_t s_top[kCoefThreads / 32];
  __shared__ int s_count[kCoefThreads / 32];
  __shared__ bool s_last;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");  // (behind the wait: a dependent may read what was there before this kernel)
  if (static_cast<int>(blockIdx.x) >= p.blocks) return widen_rows(p.widen, blockIdx.x - p.blocks, gridDim.x - p.blocks);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  bool bad = false;
  uint32_t top = 0u;
  int count = 0;
  for (long long row = static_cast<long long>(blockIdx.x) * kCoefThreads + threadIdx.x; row < p.n; row += static_cast<long long>(p.blocks) * kCoefThreads) {
    float2 qe;
    float a = 0.f, b = 0.f;
    if (row_target(p.ids, p.padding_id, p.vocab, p.counts, p.sums, row, &qe, &bad)) {
      b = (p.grad ? __ldcg(p.grad + row) : 1.0f) * p.rest;
      a = b * (qe.x + (p.z_loss > 0.f ? 2.f * p.z_loss * __ldcg(p.lse + row) : 0.f));
      ++count;
    }
    p.coef[row] = make_float2(a, b);
    const uint32_t m = max(__float_as_uint(fabsf(a)), __float_as_uint(fabsf(b * qe.x)));
    if (m < 0x7F800000u) top = max(top, m);
  }
  if (bad) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_INDEX));
  auto block_join = [&]() {  // in the first thread
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    count = __reduce_add_sync(0xFFFFFFFFu, count);
    if (lane == 0) { s_top[warp] = top; s_count[warp] = count; }
    __syncthreads();
    if (threadIdx.x == 0)
      for (int i = 1; i < kCoefThreads / 32; ++i) { top = max(top, s_top[i]); count += s_count[i]; }
  };
  block_join();
  if (threadIdx.x == 0) {
    p.block_tops[blockIdx.x] = make_uint2(top, static_cast<uint32_t>(count));
    __threadfence();
    s_last = atomicAdd(p.ticket, 1u) == static_cast<uint32_t>(p.blocks - 1);
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  top = 0u; count = 0;
  if (static_cast<int>(threadIdx.x) < p.blocks) {
    const uint2 v = __ldcg(p.block_tops + threadIdx.x);
    top = v.x; count = static_cast<int>(v.y);
  }
  block_join();
  if (threadIdx.x == 0) {
    *p.ticket = 0u;
    // The largest coefficient goes to 2^14: |D| stays at or below 2^15.  Not by a power of two: the entries at the targets,
    // which decide the gradients' error, are that coefficient times nearly 1, rounded in steps of 2^-8 (BF16) of themselves just
    // below a power of two and of twice that just above it (22 x 675 x 112: 2.3e-3 of the norm of dH, 2.8e-3 by a power of two;
    // 1.6e-3 is the rounding of the result).
    int ex = static_cast<int>(top >> 23) - 127;
    if (top == 0u) ex = 14;
    ex = min(max(14 - ex, -100), 100);
    const float unit = __uint_as_float(static_cast<uint32_t>(127 + ex) << 23) / __uint_as_float((top & 0x7FFFFFu) | 0x3F800000u);
    p.unit[0] = unit;
    p.unit[1] = (p.grad ? 1.0f : 1.0f / static_cast<float>(max(count, 1)) / p.mean_p2) / unit;
    const float hs = load_scale_after_wait(p.h_scale), ws = load_scale_after_wait(p.w_scale);
    const float gs = p.grad ? load_scale_after_wait(p.grad_scale) : p.mean_p2;
    if (!is_pow2_scale(hs) || !is_pow2_scale(ws) || !is_pow2_scale(gs)) atomicOr(p.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_SCALE));
    const float ds = gs * p.inv_temp_p2;
    if (p.dh_scale) *p.dh_scale = ds * ws * p.kf_vocab;
    if (p.dw_scale) *p.dw_scale = ds * hs * p.kf_n;
  }
}

// The sums of dH's planes, in order -> dH
struct PlanesParams {
  const float* acc; long long ld_acc; int planes;
  int M, N;
  void* out; long long ldo; int out_dt;
  float alpha; const float* unit;
};
__global__ void __launch_bounds__(256) planes_kernel(const PlanesParams p) {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int vecs = (p.N + 3) / 4;
  const float alpha = p.alpha * *reinterpret_cast<const volatile float*>(p.unit + 1);
  const long long plane = static_cast<long long>(p.M) * p.ld_acc;
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < static_cast<long long>(p.M) * vecs; i += static_cast<long long>(gridDim.x) * 256) {
    const int row = static_cast<int>(i / vecs), c = static_cast<int>(i - static_cast<long long>(row) * vecs) * 4;
    const float* a = p.acc + row * p.ld_acc + c;  // (rows are padded to whole vectors)
    float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kBatch = 8;  // loads in flight: few rows are a matter of latency
    for (int s0 = 0; s0 < p.planes; s0 += kBatch) {
      float4 v[kBatch];
#pragma unroll
      for (int s = 0; s < kBatch; ++s)
        v[s] = s0 + s < p.planes ? __ldcg(reinterpret_cast<const float4*>(a + (s0 + s) * plane)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int s = 0; s < kBatch; ++s) { f.x += v[s].x; f.y += v[s].y; f.z += v[s].z; f.w += v[s].w; }
    }
    const float x[4] = {f.x * alpha, f.y * alpha, f.z * alpha, f.w * alpha};
    const long long o = row * p.ldo + c;
    if (c + 4 <= p.N) {
      uint32_t w[2];
      if (p.out_dt == SCALIFY_BF16) encode_vec<SCALIFY_BF16, 4>(x, w);
      else encode_vec<SCALIFY_F16, 4>(x, w);
      st_raw<8>(static_cast<uint16_t*>(p.out) + o, w);
    } else {
      for (int e = 0; e < p.N - c; ++e) {
        if (p.out_dt == SCALIFY_BF16) store_elem<SCALIFY_BF16>(p.out, o + e, x[e]);
        else store_elem<SCALIFY_F16>(p.out, o + e, x[e]);
      }
    }
  }
}

// No rows: dW is zero.
__global__ void __launch_bounds__(256) zero_rows_kernel(uint16_t* out, long long ld, long long rows, int d) {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (long long r = blockIdx.x; r < rows; r += gridDim.x)
    for (int c = threadIdx.x; c < d; c += 256) out[r * ld + c] = 0;
}

// ------------------------------------------------------------------------------------------------- host side
// CTAs per tile, and the pairs (or CTAs) of the GPU.
int ctas_of(long long n) { return n <= kTM ? 1 : 2; }
int units_of(long long n) { return kSms / ctas_of(n); }
long long row_tiles(long long rows, int ctas) { return (rows + kTM * ctas - 1) / (kTM * ctas); }
long long pad_to(long long x, long long m) { return (x + m - 1) / m * m; }
size_t pad256(size_t x) { return (x + 255) / 256 * 256; }

// Columns of a logits tile.  A batch of one row tile has the vocabulary's tiles alone to share, each CTA with few of them:
// their width is chosen for equal shares (37 rows, vocabulary 50257, 148 CTAs: two rounds of 256 columns or of 192).
int tile_columns(long long n, long long vocab) {
  if (ctas_of(n) == 2) return kTN;
  int best = kTN;
  long long least = 0;
  for (int w = kTN; w >= 64; w -= 64) {
    const long long tiles = (vocab + w - 1) / w, cost = (tiles + units_of(n) - 1) / units_of(n) * (w + 16);
    if (w == kTN || cost < least) { best = w; least = cost; }
  }
  return best;
}
// The forward call's longest run, and the items that there have to be.
constexpr int kLongestRun = 8;
int run_items(int ctas) { return 16 * (kSms / ctas); }
// Consecutive column tiles per work item: long runs write few partial results, short ones share the work evenly.
int run_length(long long tiles_m, long long tiles_n, int longest, int items) {
  for (int run = longest; run > 1; run >>= 1)
    if (tiles_m * ((tiles_n + run - 1) / run) >= items) return run;
  return 1;
}
// Few rows: D in two halves of its type, the second of what the first one's rounding left out, as rows of their own: dW's
// contraction is over both (H twice), dH's sums are added at the end.  One rounding of D adds about as much to the gradients'
// error as rounding the gradients themselves; with few rows, where a few entries of D decide, up to twice that (2 x 1646 x 136,
// BF16: 2.7e-3 of the norm where 1.6e-3 is the output's own).  Both sides, BF16, loss and gradients from a graph with cold caches,
// one half against two: 50257 x 768: 3 rows 98 and 107 us, dH off by 2.0e-3 and 1.65e-3 (three draws: 1.8e-3 to 2.0e-3); 16 rows
// 102 and 114, 1.95e-3 and 1.66e-3; 32 rows 102 and 117, 1.88e-3 and 1.66e-3; 64 rows 102 and 123, 1.86e-3 and 1.66e-3.
// 115392 x 672: 3 rows 182 and 197 us, 16 rows 186 and 201, 64 rows 188 and 207.  Beyond 16 rows the error no longer depends on the
// draw, and the cost grows.
constexpr int kFewRows = 16;
int halves_of(long long n) { return n > 0 && n <= kFewRows ? 2 : 1; }
// Columns of a piece of the vocabulary: D of at most 2^27 bytes, two pieces of which are in memory; whole tiles.
// (8192 x 50257 x 768: half and a quarter of it take 4 and 8 % longer, twice of it 2 % less.)
constexpr long long kPieceElems = 1ll << 26;
long long piece_columns(long long n, long long vocab) {
  const long long rows = pad_to(n < 1 ? 1 : n, 32);
  long long cols = kPieceElems / rows / kTN * kTN;
  if (cols < kTN) cols = kTN;
  const long long all = pad_to(vocab, kTN);
  if (cols >= all) return all;
  const long long pieces = (all + cols - 1) / cols;
  return pad_to((all + pieces - 1) / pieces, kTN);
}
// K blocks that a tile's start and end cost beside its own
constexpr int kTileCost = 3;
// Parts of dH's contraction where the whole vocabulary is one piece: few tiles of a long contraction would keep few CTA pairs
// busy; a part is at most half of a pair's load.
int dh_parts(long long n, long long vocab, long long d) {
  const int ctas = ctas_of(n);
  const double tm = static_cast<double>(row_tiles(n, ctas)), tn = static_cast<double>((d + kTN - 1) / kTN), tv = static_cast<double>(row_tiles(vocab, ctas));
  const double kb_v = static_cast<double>((vocab + kK16 - 1) / kK16), kb_n = static_cast<double>((n + kK16 - 1) / kK16);
  const double load = (tm * tn * (kb_v + kTileCost) + tv * tn * (kb_n + kTileCost)) / units_of(n);
  long long parts = static_cast<long long>(ceil(2.0 * kb_v / load)), most = static_cast<long long>(kb_v / 16);
  if (parts > 32) parts = 32;
  if (parts > most) parts = most;
  return parts < 1 ? 1 : static_cast<int>(parts);
}

// K blocks of the logits
long long row_kbs(long long d, int es) { return (d * es + kRowBytes - 1) / kRowBytes; }

struct Layout {
  size_t partial, dot, sums_blocks, entries, counts, sums, table, coef, tops, unit, h16, w16, D[2], acc, sums_long, total;
  long long ld_part, ld16, ldd, ld_acc, piece, pieces;
  int slots, run, parts, width, bins, bin_tiles, halves;
};
Layout layout_of(long long n, long long vocab, long long d, int es, int k, bool backward) {
  Layout l = {};
  size_t at = kWsHeader;
  auto take = [&](size_t bytes) { const size_t o = at; at += pad256(bytes); return o; };
  const size_t rows = static_cast<size_t>(n);
  l.width = tile_columns(n, vocab);
  if (backward) {
    l.halves = halves_of(n);
    l.piece = piece_columns(n * l.halves, vocab);
    l.pieces = (vocab + l.piece - 1) / l.piece;
    if (l.pieces > 1) l.width = kTN;  // (pieces begin with a tile)
  }
  const long long tm = row_tiles(n, ctas_of(n)), tn = (vocab + l.width - 1) / l.width;
  if (k > 0) {
    l.bin_tiles = static_cast<int>((tn + kMaxBins - 1) / kMaxBins);
    l.bins = static_cast<int>((tn + l.bin_tiles - 1) / l.bin_tiles);
    l.entries = take(rows * k * sizeof(Entry));
    l.counts = take(rows * sizeof(int2));
    l.sums = take(rows * sizeof(float2));
    l.table = take(rows * 2 * l.bins * sizeof(uint16_t));
  }
  if (!backward) {
    l.run = run_length(tm, tn, kLongestRun, run_items(ctas_of(n)));
    l.slots = static_cast<int>((tn + l.run - 1) / l.run) * 2;
    l.ld_part = pad_to(n, 32);
    l.partial = take(static_cast<size_t>(l.slots) * l.ld_part * sizeof(float2));
    l.dot = take(static_cast<size_t>(l.slots) * l.ld_part * sizeof(float));
    l.sums_blocks = take((rows / 4 + 1) * sizeof(double2));
  } else {
    l.coef = take(rows * sizeof(float2));
    l.tops = take(kCoefBlocks * sizeof(uint2));
    l.unit = take(2 * sizeof(float));
    l.ld16 = pad_to(d, 16);
    const size_t d_rows = rows * l.halves;
    if (es == 1 || l.halves > 1) l.h16 = take(d_rows * l.ld16 * 2);
    if (es == 1) l.w16 = take(static_cast<size_t>(vocab) * l.ld16 * 2);
    l.ldd = l.piece;
    // (from three pieces on as much as a piece may take, not what this batch's takes: the size must not fall as batches grow)
    size_t d_bytes = d_rows * l.ldd * 2;
    if (l.pieces > 2 && d_bytes < kPieceElems * 2) d_bytes = kPieceElems * 2;
    l.D[0] = take(d_bytes);
    l.D[1] = l.pieces > 1 ? take(d_bytes) : l.D[0];
    l.parts = l.pieces == 1 && n > 0 ? dh_parts(n, vocab, d) : 1;
    if (l.pieces > 1 || l.parts > 1 || l.halves > 1) {
      l.ld_acc = pad_to(d, 32);
      l.acc = take(l.parts * d_rows * l.ld_acc * sizeof(float));
    }
    // (the widest that as many pieces can be: the size must not fall as batches grow)
    const long long widest = l.pieces > 1 ? kPieceElems / pad_to(n > 0 ? n * l.halves : 1, 32) : l.piece;
    const long long dh_kb = (widest / kK16 + l.parts - 1) / l.parts, dw_kb = (static_cast<long long>(d_rows) + kK16 - 1) / kK16;
    if (n > 0 && (dh_kb > kSumKb || dw_kb > kSumKb || row_kbs(d, es) > kLogitKb)) l.sums_long = take(static_cast<size_t>(kSms) * kEpiWarps * kWarpSums * sizeof(float));
  }
  l.total = at < kWsMin ? kWsMin : at;
  return l;
}

template <int NCTA, bool STAGING, class K>
int unit_config(K kernel, DeviceOnce& once, long long items, cudaStream_t st, cudaLaunchConfig_t* cfg, cudaLaunchAttribute* attrs, int* units) {
  constexpr size_t kBytes = Cfg<NCTA>::kSmem + (STAGING ? Cfg<NCTA>::kStaging : 0);
  int most = 0;  // CTAs (pairs) that fit the GPU
  const int rc = device_once(once, &most, [&](int* v) {
    SCALIFY_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kBytes)));
    cudaLaunchConfig_t q = {};
    q.gridDim = dim3(static_cast<unsigned>(sm_count() / NCTA * NCTA)); q.blockDim = dim3(kThreads); q.dynamicSmemBytes = kBytes;
    cudaLaunchAttribute qa[1];
    qa[0].id = cudaLaunchAttributeClusterDimension;
    qa[0].val.clusterDim.x = NCTA; qa[0].val.clusterDim.y = 1; qa[0].val.clusterDim.z = 1;
    q.attrs = qa; q.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &q) != cudaSuccess) { n = 0; cudaGetLastError(); }
    *v = n;
    return int(SCALIFY_OK);
  });
  if (rc) return rc;
  if (most < 1) return SCALIFY_ERR_UNSUPPORTED;
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = NCTA; attrs[1].val.clusterDim.y = 1; attrs[1].val.clusterDim.z = 1;
  *cfg = {};
  *units = static_cast<int>(items < most ? items : most);
  if (*units > kSms / NCTA) *units = kSms / NCTA;
  cfg->gridDim = dim3(static_cast<unsigned>(*units * NCTA));
  cfg->blockDim = dim3(kThreads); cfg->dynamicSmemBytes = kBytes; cfg->stream = st;
  cfg->attrs = attrs; cfg->numAttrs = 2;
  return SCALIFY_OK;
}
// An ordinary kernel of this file as a programmatic dependent
template <class K, class P>
int launch_small(K kernel, long long blocks, int threads, const P& p, cudaStream_t st) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks)); cfg.blockDim = dim3(threads); cfg.stream = st;
  cfg.attrs = attr; cfg.numAttrs = 1;
  SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, p));
  return SCALIFY_OK;
}

template <int NCTA, bool F8, bool KD, bool LONG>
int launch_logits_variant(const CUtensorMap& mh, const CUtensorMap& mw, const LogitsParams& p, cudaStream_t st) {
  auto kernel = logits_kernel<NCTA, F8, KD, LONG>;
  static DeviceOnce once;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attrs[2];
  int units = 0;
  const int rc = unit_config<NCTA, KD>(kernel, once, p.items, st, &cfg, attrs, &units);
  if (rc) return rc;
  SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, mh, mw, p));
  return SCALIFY_OK;
}

template <int NCTA, bool LONG>
int launch_logits(bool f8, bool kd, const CUtensorMap& mh, const CUtensorMap& mw, const LogitsParams& p, cudaStream_t st) {
  if (f8) return kd ? launch_logits_variant<NCTA, true, true, LONG>(mh, mw, p, st) : launch_logits_variant<NCTA, true, false, LONG>(mh, mw, p, st);
  return kd ? launch_logits_variant<NCTA, false, true, LONG>(mh, mw, p, st) : launch_logits_variant<NCTA, false, false, LONG>(mh, mw, p, st);
}
template <int NCTA>
int launch_logits(bool f8, bool kd, const CUtensorMap& mh, const CUtensorMap& mw, const LogitsParams& p, cudaStream_t st) {
  return p.num_kb > kLongKb<NCTA> ? launch_logits<NCTA, true>(f8, kd, mh, mw, p, st) : launch_logits<NCTA, false>(f8, kd, mh, mw, p, st);
}

// Every class's items over the pairs, long ones first, so that the loads become as equal as whole items allow.
void fill_schedule(Schedule& s, const long long (&items)[kClasses], const double (&cost)[kClasses], int units) {
  double load[kMaxUnits] = {};
  for (int i = 0; i < kClasses; ++i) s.order[i] = i;
  for (int i = 1; i < kClasses; ++i)
    for (int j = i; j > 0 && cost[s.order[j]] > cost[s.order[j - 1]]; --j) { const int t = s.order[j]; s.order[j] = s.order[j - 1]; s.order[j - 1] = t; }
  for (int i = 0; i < kClasses; ++i) {
    const int c = s.order[i];
    s.total[c] = static_cast<int>(items[c]);
    for (int u = 0; u < units; ++u) s.quota[c][u] = 0;
    if (items[c] == 0) continue;
    // the highest level up to which whole items fit, then one more for the least loaded pairs
    double lo = 0.0, hi = 0.0;
    for (int u = 0; u < units; ++u) hi = load[u] > hi ? load[u] : hi;
    hi += cost[c] * (static_cast<double>(items[c]) / units + 2.0);
    auto fits = [&](double level) {
      long long n = 0;
      for (int u = 0; u < units; ++u) n += level > load[u] ? static_cast<long long>((level - load[u]) / cost[c]) : 0;
      return n;
    };
    for (int it = 0; it < 60; ++it) {
      const double mid = 0.5 * (lo + hi);
      if (fits(mid) <= items[c]) lo = mid; else hi = mid;
    }
    long long left = items[c];
    for (int u = 0; u < units; ++u) {
      const int q = lo > load[u] ? static_cast<int>((lo - load[u]) / cost[c]) : 0;
      s.quota[c][u] = q;
      load[u] += q * cost[c];
      left -= q;
    }
    while (left > 0) {
      int best = 0;
      for (int u = 1; u < units; ++u)
        if (load[u] < load[best]) best = u;
      ++s.quota[c][best];
      load[best] += cost[c];
      --left;
    }
  }
}

template <int NCTA, bool F8, bool KD, bool BF, bool SUMS>
int launch_grad_variant(const GradMaps& m, GradParams& p, const long long (&items)[kClasses], const double (&cost)[kClasses], cudaStream_t st) {
  auto kernel = loss_grad_kernel<NCTA, F8, KD, BF, SUMS>;
  static DeviceOnce once;
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute attrs[2];
  int units = 0;
  const int rc = unit_config<NCTA, true>(kernel, once, items[0] + items[1] + items[2], st, &cfg, attrs, &units);
  if (rc) return rc;
  fill_schedule(p.schedule, items, cost, units);
  SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, m, p));
  return SCALIFY_OK;
}
template <int NCTA, bool SUMS>
int launch_grad(bool f8, bool kd, bool bf, const GradMaps& m, GradParams& p, const long long (&items)[kClasses], const double (&cost)[kClasses], cudaStream_t st) {
  if (f8) return kd ? launch_grad_variant<NCTA, true, true, false, SUMS>(m, p, items, cost, st) : launch_grad_variant<NCTA, true, false, false, SUMS>(m, p, items, cost, st);
  if (bf) return kd ? launch_grad_variant<NCTA, false, true, true, SUMS>(m, p, items, cost, st) : launch_grad_variant<NCTA, false, false, true, SUMS>(m, p, items, cost, st);
  return kd ? launch_grad_variant<NCTA, false, true, false, SUMS>(m, p, items, cost, st) : launch_grad_variant<NCTA, false, false, false, SUMS>(m, p, items, cost, st);
}
template <int NCTA>
int launch_grad(bool f8, bool kd, bool bf, const GradMaps& m, GradParams& p, const long long (&items)[kClasses], const double (&cost)[kClasses], cudaStream_t st) {
  const bool sums = (items[kClassD] > 0 && p.logits.num_kb > kLogitKb) || (items[kClassDw] > 0 && p.product[kClassDw].part_kb > kSumKb) ||
                    (items[kClassDh] > 0 && p.product[kClassDh].part_kb > kSumKb);
  return sums ? launch_grad<NCTA, true>(f8, kd, bf, m, p, items, cost, st) : launch_grad<NCTA, false>(f8, kd, bf, m, p, items, cost, st);
}

// operand formats of the instruction descriptor: kind::f16 F16 0, BF16 1; kind::f8f6f4 E4M3 0, E5M2 1
uint32_t format_of(int dt) { return dt == SCALIFY_BF16 || dt == SCALIFY_E5M2 ? 1u : 0u; }
uint32_t idesc_of(int a_dt, int b_dt, int ctas, int width) {
  return (1u << 4) | (format_of(a_dt) << 7) | (format_of(b_dt) << 10) | (uint32_t(width >> 3) << 17) | (uint32_t(ctas * kTM >> 4) << 24);
}
// [rows][cols] of es-byte elements, rows ld apart (one row alone may have any stride), in boxes of 128 bytes x box_rows
int map_of(CUtensorMap* m, const void* base, long long rows, long long cols, long long ld, int es, uint32_t box_rows) {
  const long long bytes = rows > 1 ? ld * es : pad_to(cols * es, 16);
  return make_byte_map(m, base, static_cast<uint64_t>(cols) * es, static_cast<uint64_t>(rows), 1, static_cast<uint64_t>(bytes),
                       static_cast<uint64_t>(bytes) * rows, kRowBytes, box_rows);
}

// D [rows][cols], for stores of 32 rows x 32 columns (a ragged last 16 bytes is written whole: D's rows are padded)
int d_store_map(CUtensorMap* m, const void* base, long long rows, long long cols, long long ld) {
  return make_byte_map(m, base, static_cast<uint64_t>(cols) * 2, static_cast<uint64_t>(rows), 1, static_cast<uint64_t>(ld) * 2, static_cast<uint64_t>(ld) * 2 * rows, 64, 32);
}

int prepare_teacher(const LinearLossArgs& a, const Layout& l, char* ws, cudaStream_t st) {
  if (a.k == 0) return SCALIFY_OK;
  TeacherParams t = {};
  t.n = a.n; t.vocab = a.vocab; t.k = a.k;
  t.ids = a.ids; t.padding_id = a.padding_id;
  t.T = a.T; t.t_dt = a.t_dt; t.t_ld = a.t_ld; t.t_scale = a.t_scale; t.t_lse = a.t_lse;
  t.inv_temp = a.inv_temp;
  t.half_cols = l.width / 2;
  t.table = reinterpret_cast<uint16_t*>(ws + l.table);
  t.bins = l.bins; t.bin_tiles = l.bin_tiles;
  t.entries = reinterpret_cast<Entry*>(ws + l.entries);
  t.counts = reinterpret_cast<int2*>(ws + l.counts);
  t.sums = reinterpret_cast<float2*>(ws + l.sums);
  t.status = ws_view(ws).status;
  // (one warp per row up to 64 entries, four or eight beyond: one row of 200 takes 7 us, with one warp 22)
  if (a.k <= 32) return launch_small(teacher_kernel<1, 1>, (a.n + 3) / 4, 128, t, st);
  if (a.k <= 64) return launch_small(teacher_kernel<2, 1>, (a.n + 3) / 4, 128, t, st);
  if (a.k <= 128) return launch_small(teacher_kernel<1, 4>, a.n, 128, t, st);
  return launch_small(teacher_kernel<1, 8>, a.n, 256, t, st);
}

// (whole: a launch with tiles of the products)
Ring ring_of(int ctas, int box_rows, int width, bool whole) {
  Ring r = {0, whole ? kTM * kRowBytes : box_rows * kRowBytes, (whole ? kTN : width) / ctas * kRowBytes};
  r.stages = static_cast<int>(Cfg<1>::kRing / (r.a_bytes + r.b_bytes));
  if (r.stages > kMaxStages) r.stages = kMaxStages;
  return r;
}
LogitsParams logits_params(const LinearLossArgs& a, const Layout& l, char* ws) {
  LogitsParams p = {};
  p.box_rows = ctas_of(a.n) == 2 ? kTM : static_cast<int>(pad_to(a.n, 8));
  p.ring = ring_of(ctas_of(a.n), p.box_rows, l.width, false);
  const int es = elem_size(a.h_dt);
  p.n = static_cast<int>(a.n);
  p.num_kb = static_cast<int>(row_kbs(a.d, es));
  p.tiles_m = static_cast<int>(row_tiles(a.n, ctas_of(a.n)));
  p.idesc = idesc_of(a.h_dt, a.w_dt, ctas_of(a.n), l.width);
  p.half_cols = l.width / 2;
  p.h_scale = a.h_scale; p.w_scale = a.w_scale; p.inv_temp = a.inv_temp;
  p.ids = a.ids; p.padding_id = a.padding_id; p.vocab = a.vocab;
  if (a.k > 0) {
    p.entries = reinterpret_cast<const Entry*>(ws + l.entries);
    p.counts = reinterpret_cast<const int2*>(ws + l.counts);
    p.k = a.k;
    p.table = reinterpret_cast<const uint16_t*>(ws + l.table);
    p.bins = l.bins; p.bin_tiles = l.bin_tiles;
  }
  p.status = ws_view(ws).status;
  return p;
}

}  // namespace

size_t linear_loss_ws_need(long long n, long long vocab, long long d, int operand_bytes, int k, bool backward) {
  const size_t forward = layout_of(n, vocab, d, operand_bytes, k, false).total;
  if (!backward) return forward;
  const size_t both = layout_of(n, vocab, d, operand_bytes, k, true).total;
  return both > forward ? both : forward;
}

// The most that a batch of at most n rows needs, so that a workspace for the longest batch serves every other.  The need falls only
// where the plan changes: behind the last batch with two halves of D, with one CTA per tile, of each run length, of each number
// of parts of dH, with one piece of the vocabulary, and with pieces longer than an accumulator's sum.  Between those it grows, so
// they are what is looked at.
size_t linear_loss_ws_bytes(long long n, long long vocab, long long d, int operand_bytes, int k, bool backward) {
  size_t most = 0;
  auto look = [&](long long rows) {
    const size_t need = linear_loss_ws_need(rows < n ? rows : n, vocab, d, operand_bytes, k, backward);
    if (need > most) most = need;
  };
  look(n);
  look(kFewRows);
  look(kTM);
  const long long tiles_n = (vocab + kTN - 1) / kTN, tile_m = 2 * kTM;
  for (int run = 2; run <= kLongestRun; run *= 2) {  // the last batch with runs shorter than this
    const long long per = (tiles_n + run - 1) / run;
    look((run_items(2) + per - 1) / per * tile_m - tile_m);
  }
  if (!backward) return most;
  const long long all = pad_to(vocab, kTN), one_piece = all == kTN ? n : kPieceElems / all / 32 * 32;
  look(one_piece);
  look(kPieceElems / ((kSumKb + 1) * kK16) / 32 * 32);  // the last batch with pieces that take several accumulators
  // (parts: the same for all batches of as many K blocks; one where there are two tiles for each unit)
  const long long d_tiles = (d + kTN - 1) / kTN;
  for (long long rows = kK16; rows < n && rows < one_piece && row_tiles(rows, ctas_of(rows)) * d_tiles < 2 * units_of(rows); rows += kK16) look(rows);
  return most;
}

int launch_linear_loss(const LinearLossArgs& a, void* workspace, cudaStream_t st) {
  char* ws = static_cast<char*>(workspace);
  const int es = elem_size(a.h_dt);
  const Layout l = layout_of(a.n, a.vocab, a.d, es, a.k, false);
  if (a.n == 0) {
    if (a.mean) SCALIFY_CUDA_TRY(cudaMemsetAsync(a.mean, 0, sizeof(float), st));
    return SCALIFY_OK;
  }
  LogitsParams p = logits_params(a, l, ws);
  CUtensorMap mh, mw;
  int rc = map_of(&mh, a.H, a.n, a.d, a.h_ld, es, p.box_rows);
  if (!rc) rc = map_of(&mw, a.W, a.vocab, a.d, a.w_ld, es, l.width / ctas_of(a.n));
  if (!rc) rc = prepare_teacher(a, l, ws, st);
  if (rc) return rc;
  p.early = a.k > 0;  // (after the teacher kernel)
  p.cols = static_cast<int>(a.vocab);
  p.tiles_n = static_cast<int>((a.vocab + l.width - 1) / l.width);
  p.run = l.run;
  p.items = static_cast<long long>(p.tiles_m) * (l.slots / 2);
  p.partial = reinterpret_cast<float2*>(ws + l.partial);
  p.dot = reinterpret_cast<float*>(ws + l.dot);
  p.ld_part = l.ld_part;
  rc = ctas_of(a.n) == 2 ? launch_logits<2>(es == 1, a.k > 0, mh, mw, p, st) : launch_logits<1>(es == 1, a.k > 0, mh, mw, p, st);
  if (rc) return rc;
  JoinParams j = {};
  j.n = a.n; j.vocab = a.vocab; j.slots = l.slots;
  j.partial = p.partial; j.dot = p.dot; j.ld_part = l.ld_part;
  j.h_scale = a.h_scale; j.w_scale = a.w_scale; j.inv_temp = a.inv_temp; j.z_loss = a.z_loss;
  j.ids = a.ids; j.padding_id = a.padding_id;
  if (a.k > 0) {
    j.counts = reinterpret_cast<const int2*>(ws + l.counts);
    j.sums = reinterpret_cast<const float2*>(ws + l.sums);
  }
  j.loss = a.loss; j.lse = a.lse; j.mean = a.mean;
  while (j.rows_log < 5 && (1ll << j.rows_log) < a.n) ++j.rows_log;
  while (j.rows_log > 2 && l.slots > 8 * (kJoinThreads >> j.rows_log)) --j.rows_log;  // one round of loads where it can be
  j.block_sums = reinterpret_cast<double2*>(ws + l.sums_blocks);
  j.ticket = ws_view(ws).ticket;
  j.status = ws_view(ws).status;
  return launch_small(join_kernel, (a.n + (1ll << j.rows_log) - 1) >> j.rows_log, kJoinThreads, j, st);
}

int launch_linear_loss_bwd(const LinearLossArgs& a, void* workspace, cudaStream_t st) {
  char* ws = static_cast<char*>(workspace);
  const int es = elem_size(a.h_dt);
  const Layout l = layout_of(a.n, a.vocab, a.d, es, a.k, true);
  int rc = a.n > 0 ? prepare_teacher(a, l, ws, st) : SCALIFY_OK;
  if (rc) return rc;
  CoefParams c = {};
  c.n = a.n; c.vocab = a.vocab; c.ids = a.ids; c.padding_id = a.padding_id;
  if (a.k > 0) {
    c.counts = reinterpret_cast<const int2*>(ws + l.counts);
    c.sums = reinterpret_cast<const float2*>(ws + l.sums);
  }
  c.lse = a.lse; c.z_loss = a.z_loss; c.rest = a.inv_temp_rest; c.inv_temp_p2 = a.inv_temp_p2;
  c.grad = a.grad; c.grad_scale = a.grad_scale;
  int ex;
  frexp(1.0 / static_cast<double>(a.n > 0 ? a.n : 1), &ex);
  c.mean_p2 = static_cast<float>(ldexp(1.0, ex - 1));
  c.h_scale = a.h_scale; c.w_scale = a.w_scale;
  c.kf_vocab = kfactor(a.vocab); c.kf_n = kfactor(a.n > 0 ? a.n : 1);
  c.coef = reinterpret_cast<float2*>(ws + l.coef);
  c.block_tops = reinterpret_cast<uint2*>(ws + l.tops);
  c.unit = reinterpret_cast<float*>(ws + l.unit);
  c.dh_scale = a.dh_scale; c.dw_scale = a.dw_scale;
  c.ticket = ws_view(ws).ticket; c.status = ws_view(ws).status;
  c.blocks = static_cast<int>(a.n < kCoefThreads ? 1 : a.n > kCoefThreads * kCoefBlocks ? kCoefBlocks : (a.n + kCoefThreads - 1) / kCoefThreads);
  const char* h16 = static_cast<const char*>(a.H);
  const char* w16 = static_cast<const char*>(a.W);
  long long h16_ld = a.h_ld, w16_ld = a.w_ld, widen_blocks = 0;
  if ((es == 1 || l.halves > 1) && a.n > 0) {
    WidenParams& w = c.widen;
    w.d = a.d; w.ldd = l.ld16; w.n = a.n;
    w.src[0] = a.H; w.dst[0] = reinterpret_cast<__half*>(ws + l.h16); w.ld[0] = a.h_ld; w.rows[0] = a.dW ? a.n * l.halves : 0; w.dt[0] = a.h_dt;
    w.src[1] = a.W; w.dst[1] = reinterpret_cast<__half*>(ws + l.w16); w.ld[1] = a.w_ld; w.rows[1] = a.dH && es == 1 ? a.vocab : 0; w.dt[1] = a.w_dt;
    const long long most = 16ll * sm_count();
    widen_blocks = ((w.rows[0] + w.rows[1]) * ((a.d + 15) / 16) + kCoefThreads - 1) / kCoefThreads;
    if (widen_blocks > most) widen_blocks = most;
    h16 = ws + l.h16;
    h16_ld = l.ld16;
    if (es == 1) { w16 = ws + l.w16; w16_ld = l.ld16; }
  }
  rc = launch_small(coef_kernel, c.blocks + widen_blocks, kCoefThreads, c, st);
  if (rc) return rc;
  if (a.n == 0) {
    if (!a.dW) return SCALIFY_OK;
    zero_rows_kernel<<<static_cast<unsigned>(a.vocab < 4096 ? a.vocab : 4096), 256, 0, st>>>(static_cast<uint16_t*>(a.dW), a.dw_ld, a.vocab, a.d);
    SCALIFY_CUDA_TRY(cudaGetLastError());
    return SCALIFY_OK;
  }
  const bool bf = a.h_dt == SCALIFY_BF16;
  const int d_dt = bf ? SCALIFY_BF16 : SCALIFY_F16;
  GradParams g = {};
  GradMaps m = {};
  LogitsParams& p = g.logits;
  p = logits_params(a, l, ws);
  p.lse = a.lse; p.coef = c.coef; p.ldd = l.ldd;
  const long long d_rows = a.n * l.halves;  // (at most one row tile where there are two halves)
  const int ctas = ctas_of(a.n), n_tiles = p.tiles_m, d_tiles = static_cast<int>((a.d + kTN - 1) / kTN);
  GradProduct &dw = g.product[kClassDw], &dh = g.product[kClassDh];
  dw.N = dh.N = a.d;
  dw.tiles_n = dh.tiles_n = d_tiles;
  dw.num_kb = dw.part_kb = static_cast<int>((d_rows + kK16 - 1) / kK16);
  dw.parts = 1;
  dw.ldo = a.dw_ld; dw.out_dt = a.dw_dt; dw.alpha = 1.0f / c.kf_n; dw.mode = kFinal;
  dh.M = static_cast<int>(d_rows);
  dh.out = a.dH; dh.ldo = a.dh_ld; dh.out_dt = a.dh_dt; dh.alpha = 1.0f / c.kf_vocab;
  dh.acc = reinterpret_cast<float*>(ws + l.acc); dh.ld_acc = l.ld_acc;
  g.idesc = idesc_of(d_dt, d_dt, ctas, kTN);
  g.unit = c.unit;
  g.sums = reinterpret_cast<float*>(ws + l.sums_long);  // (not touched where the layout has none)
  rc = map_of(&m.h, a.H, a.n, a.d, a.h_ld, es, p.box_rows);
  if (!rc) rc = map_of(&m.h_mn, h16, d_rows, a.d, h16_ld, 2, kK16);
  if (rc) return rc;
  // launch i: the products of piece i - 1 and the logits of piece i
  for (long long i = 0; i <= l.pieces; ++i) {
    p.early = i == 0;  // (after the coefficients)
    p.ring = ring_of(ctas, p.box_rows, l.width, i > 0);
    long long items[kClasses] = {};
    double cost[kClasses] = {};
    if (i < l.pieces) {
      const long long v0 = i * l.piece, cols = a.vocab - v0 < l.piece ? a.vocab - v0 : l.piece;
      p.col0 = v0; p.cols = static_cast<int>(cols);
      p.tiles_n = static_cast<int>((cols + l.width - 1) / l.width);
      // distillation looks up a row's place in its entries once per item: longer ones where there are enough
      p.run = a.k > 0 ? run_length(n_tiles, p.tiles_n, 4, 8 * units_of(a.n)) : 1;
      items[kClassD] = static_cast<long long>(n_tiles) * ((p.tiles_n + p.run - 1) / p.run);
      cost[kClassD] = p.run * (p.num_kb + kTileCost);
      rc = d_store_map(&m.d_out, ws + l.D[i & 1], a.n, cols, l.ldd);
      if (l.halves > 1) p.d_low = reinterpret_cast<uint16_t*>(ws + l.D[i & 1]) + a.n * l.ldd;
      if (!rc) rc = map_of(&m.w, static_cast<const char*>(a.W) + v0 * a.w_ld * es, cols, a.d, a.w_ld, es, l.width / ctas);
    }
    if (!rc && i > 0) {
      const long long v0 = (i - 1) * l.piece, cols = a.vocab - v0 < l.piece ? a.vocab - v0 : l.piece;
      const uint16_t* D = reinterpret_cast<const uint16_t*>(ws + l.D[(i - 1) & 1]);
      dw.M = static_cast<int>(cols);
      dh.num_kb = static_cast<int>((cols + kK16 - 1) / kK16);
      dh.part_kb = (dh.num_kb + l.parts - 1) / l.parts;
      dh.parts = (dh.num_kb + dh.part_kb - 1) / dh.part_kb;
      dh.mode = i == 1 && (l.pieces > 1 || dh.parts > 1 || l.halves > 1) ? kAccFirst : i == 1 ? kFinal : i < l.pieces || l.halves > 1 ? kAccNext : kAccLast;
      if (a.dW) items[kClassDw] = row_tiles(cols, ctas) * d_tiles;
      if (a.dH) items[kClassDh] = static_cast<long long>(n_tiles) * d_tiles * dh.parts;
      cost[kClassDw] = dw.num_kb + kTileCost;
      cost[kClassDh] = dh.part_kb + kTileCost;
      dw.out = a.dW ? static_cast<char*>(a.dW) + v0 * a.dw_ld * 2 : nullptr;
      rc = map_of(&m.d_mn, D, d_rows, cols, l.ldd, 2, kK16);
      if (!rc) rc = map_of(&m.d_k, D, d_rows, cols, l.ldd, 2, kTM);
      if (!rc) rc = map_of(&m.w_mn, w16 + v0 * w16_ld * 2, cols, a.d, w16_ld, 2, kK16);
    }
    if (!rc) rc = ctas == 2 ? launch_grad<2>(es == 1, a.k > 0, bf, m, g, items, cost, st) : launch_grad<1>(es == 1, a.k > 0, bf, m, g, items, cost, st);
    if (rc) return rc;
  }
  if (!a.dH || dh.parts * l.halves == 1) return SCALIFY_OK;
  PlanesParams q = {};
  q.acc = dh.acc; q.ld_acc = dh.ld_acc; q.planes = dh.parts * l.halves;  // of a.n rows each
  q.M = static_cast<int>(a.n); q.N = dh.N; q.out = a.dH; q.ldo = a.dh_ld; q.out_dt = dh.out_dt;
  q.alpha = dh.alpha; q.unit = g.unit;
  const long long blocks = (a.n * ((a.d + 3) / 4) + 255) / 256, most = 8ll * sm_count();
  return launch_small(planes_kernel, blocks < most ? blocks : most, 256, q, st);
}

}  // namespace scalify
