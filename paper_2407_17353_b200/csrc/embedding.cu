// Embedding lookup with a constant factor, and its gradient by sorted tokens.
//
// Lookup:    Y_s = wte_s p2(c),  Y_d[i] = round(wte_d[ids[i]] c/p2(c))          (a scalar constant: Section 3.4)
// Gradient:  dwte_d[v] = c/p2(c) sum_{i: ids[i] = v} dY_d[i], scale dY_s p2(c), plus an optional addend by the add rule.
//
// Gradient, five launches:
//   1. mark sets a bit for every token that occurs.
//   2. sort: one cluster of blocks sorts (token, position) pairs by token, stably, so that the positions of a token stay
//      in ascending order (least significant digit first, 8 bits a pass, two passes for vocabularies below 2^16).
//   3. fill, on the SMs that the sort leaves free: writes the rows whose token does not occur (zeros, or the addend), most
//      of the bytes of a large vocabulary.
//   4. segment_sum: the sorted tokens are cut into chunks whatever the token frequencies are (a token that makes up a
//      twentieth of the batch is common), one warp per chunk and 256 columns.  A run of at most kShort equal tokens is
//      summed by the chunk it begins in, across the border if need be; a longer one leaves an fp32 partial row per chunk.
//   5. segment_join adds the partial rows of the long runs in chunk order.
// Every sum is fp32 in an order that the token ids alone determine: no atomics on data, the same bits every time.
// Bound: HBM (the gradient's rows once, the table once, the addend once).
#include "scalify_common.cuh"
#include "scalify_launch.h"
#include "tcgen05_ptx.cuh"
#include "vec8.cuh"

namespace scalify {

namespace {

constexpr int kSlab = 32 * kVec;      // columns one warp covers in the segment kernels
constexpr int kMinChunk = 8, kMaxChunk = 16;  // sorted tokens per work item there
constexpr int kShort = 16;            // longest run that its first chunk sums alone: chunk + run fit the 32 lanes (8: no slower)
constexpr int kSortCtas = 16;         // most blocks of the sorting cluster (8 where 16 cannot be resident together)
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxKpt = 8;            // keys per thread and tile
constexpr int kFillRows = 32;         // rows per filling block: one word of marks
constexpr size_t kMarkBytes = kEmbeddingMaxVocab / 8;

}  // namespace

// ------------------------------------------------------------------------------------------------- lookup
// One warp per row and up to 4 x 256 columns: four vectors of 8 elements per lane are in flight.
// 65536 rows of 2048, FP16 -> BF16: 60.5 us (rows that repeat come from the L2: 83 MB read from HBM, 268 MB written);
// 37 rows of 768: 2.8 us in a replayed graph, which is the launch.
constexpr int kLookupVpt = 4;
template <int WDT>
__global__ void __launch_bounds__(256) embedding_lookup_kernel(const EmbeddingArgs a, int col_parts) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  const int lane = threadIdx.x & 31;
  const int64_t item = blockIdx.x * 8ll + (threadIdx.x >> 5);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const float ws = load_scale(a.src_scale);
    if (a.out_scale) *a.out_scale = ws * a.c_pow2;
    if (a.status && !is_pow2_scale(ws)) atomicOr(a.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_SCALE));
  }
  if (item >= a.n * col_parts) return;
  const int64_t row = item / col_parts;
  const int part = static_cast<int>(item - row * col_parts);
  const long long id = a.ids[row];
  const bool known = id >= 0 && id < a.vocab && id != a.padding_id;
  if (!known && id != a.padding_id && a.status && lane == 0) atomicOr(a.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_INDEX));
  const char* src = static_cast<const char*>(a.src) + (known ? id : 0) * a.src_ld * ElemBytes<WDT>::v;
  char* dst = static_cast<char*>(a.out) + row * a.out_ld * a.out_es;
  const int n_vec = (a.d + kVec - 1) / kVec, v0 = part * 32 * kLookupVpt + lane;
  uint32_t w[kLookupVpt][kVec * ElemBytes<WDT>::v / 4];
#pragma unroll
  for (int i = 0; i < kLookupVpt; ++i) {
    const int v = v0 + i * 32;
#pragma unroll
    for (int q = 0; q < kVec * ElemBytes<WDT>::v / 4; ++q) w[i][q] = 0u;
    if (known && v < n_vec) load_vec<WDT>(src, v, a.d - v * kVec, w[i]);
  }
#pragma unroll
  for (int i = 0; i < kLookupVpt; ++i) {
    const int v = v0 + i * 32;
    if (v < n_vec) {
      float f[kVec];
      decode_vec<WDT, kVec>(w[i], f);
#pragma unroll
      for (int e = 0; e < kVec; ++e) f[e] *= a.c_rest;
      SCALIFY_DISPATCH_DTYPE(a.out_dt, ODT, store_vec<ODT>(dst, v, a.d - v * kVec, f))
    }
  }
}

// ------------------------------------------------------------------------------------------------- sort
// lanes whose 9-bit value equals this lane's: nine votes (the match instruction takes a turn per distinct value)
__device__ __forceinline__ uint32_t same_digit(uint32_t digit) {
  uint32_t same = 0xFFFFFFFFu;
#pragma unroll
  for (int b = 0; b < 9; ++b) {
    const bool bit = (digit >> b) & 1u;
    const uint32_t set = __ballot_sync(0xFFFFFFFFu, bit);
    same &= bit ? set : ~set;
  }
  return same;
}

struct SortArgs {
  const long long* ids;
  long long padding_id;
  int64_t n, vocab;
  uint2* pair[2];     // ping-pong: token (unknown ones: `vocab`, sorted to the end) and position
  int passes;
  uint32_t* mark;     // [vocab / 32] bits: the token occurs
  uint32_t* status;
};

__device__ __forceinline__ uint32_t token_key(const SortArgs& s, int64_t i) {
  const long long id = s.ids[i];
  if (id == s.padding_id) return static_cast<uint32_t>(s.vocab);
  if (id < 0 || id >= s.vocab) {
    atomicOr(s.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_INDEX));
    return static_cast<uint32_t>(s.vocab);
  }
  return static_cast<uint32_t>(id);
}

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t cluster_addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
  return v;
}

// Exclusive scan of one value per thread over the first 256 threads of the block (all threads call it).
__device__ __forceinline__ uint32_t scan256(uint32_t v, uint32_t* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
  if (warp < 8) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += t;
    }
    if (lane == 31) s_warp[warp] = incl;
  }
  __syncthreads();
  uint32_t before = 0u;
  if (warp < 8)
    for (int k = 0; k < warp; ++k) before += s_warp[k];
  __syncthreads();
  return before + incl - v;
}

// 8192 tokens: 13 us (8 blocks); 65536: 22 us (16 blocks).  Bound by latency: loads, two cluster barriers and a scatter a pass.
// The cluster's block `rank` sorts positions [rank * per, rank * per + per) of every pass's input, a tile of up to
// kSortThreads * kMaxKpt keys at a time.  A pass: rank the keys of a tile among its keys of the same digit (and with that
// count them), exchange the blocks' counts, write every key to its slot.  With more than one tile per block the counts
// are taken by a sweep of their own first.
__device__ void sort_tokens(const SortArgs& s, uint32_t rank, uint32_t ctas, uint32_t* s_hist, uint32_t* s_base, uint32_t* s_warp,
                            uint32_t (*s_wh)[256]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t per = (s.n + ctas - 1) / ctas;
  const int64_t begin = min(s.n, static_cast<int64_t>(rank) * per), end = min(s.n, begin + per);
  const int kpt = static_cast<int>(min(static_cast<int64_t>(kMaxKpt), (per + kSortThreads - 1) / kSortThreads));
  const bool one_tile = per <= static_cast<int64_t>(kSortThreads) * kMaxKpt;
  uint32_t key[kMaxKpt], pos[kMaxKpt], off[kMaxKpt];
  for (int p = 0; p < s.passes; ++p) {
    const int shift = 8 * p;
    const uint2* in_pairs = (p & 1) ? s.pair[0] : s.pair[1];
    uint2* out_pairs = (p & 1) ? s.pair[1] : s.pair[0];
    // Warp w owns 32 * kpt consecutive keys of the tile, 32 at a time in order: a key's rank among the warp's keys of
    // its digit is the count of the earlier groups plus the lanes below it in its group.
    auto load_and_rank = [&](int64_t t0) {
      for (int i = threadIdx.x; i < kSortWarps * 256; i += kSortThreads) (&s_wh[0][0])[i] = 0u;
      const int64_t w0 = t0 + static_cast<int64_t>(warp) * 32 * kpt + lane;
#pragma unroll
      for (int j = 0; j < kMaxKpt; ++j) {
        const int64_t i = w0 + j * 32;
        key[j] = pos[j] = 0u;
        if (j < kpt && i < end) {
          const uint2 kp = p == 0 ? make_uint2(token_key(s, i), static_cast<uint32_t>(i)) : __ldcg(in_pairs + i);
          key[j] = kp.x;
          pos[j] = kp.y;
        }
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kMaxKpt; ++j) {
        if (j < kpt) {
          const bool in = w0 + j * 32 < end;
          const uint32_t digit = in ? (key[j] >> shift) & 255u : 256u;
          const uint32_t same = same_digit(digit);
          const uint32_t below = same & ((1u << lane) - 1u);
          const uint32_t earlier = in ? s_wh[warp][digit] : 0u;
          __syncwarp();
          if (in && below == 0u) s_wh[warp][digit] = earlier + __popc(same);
          __syncwarp();
          off[j] = earlier + __popc(below);
        }
      }
      __syncthreads();
    };
    if (one_tile) {
      load_and_rank(begin);
      if (threadIdx.x < 256) {
        uint32_t c = 0u;
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) c += s_wh[w][threadIdx.x];
        s_hist[threadIdx.x] = c;
      }
    } else {
      if (threadIdx.x < 256) s_hist[threadIdx.x] = 0u;
      __syncthreads();
      for (int64_t i0 = begin; i0 < end; i0 += kSortThreads) {  // (equal digits of a warp: one addition)
        const int64_t i = i0 + threadIdx.x;
        const uint32_t k = i < end ? (p == 0 ? token_key(s, i) : __ldcg(in_pairs + i).x) : 0u;
        const uint32_t digit = i < end ? (k >> shift) & 255u : 256u;
        const uint32_t same = same_digit(digit);
        if (i < end && (same & ((1u << lane) - 1u)) == 0u) atomicAdd(&s_hist[digit], __popc(same));
      }
    }
    cluster_sync_all();
    // first output slot of (digit, this block): all smaller digits, then this digit's count in the blocks before
    uint32_t total = 0u, before = 0u;
    if (threadIdx.x < 256) {
      const uint32_t mine = smem_u32(s_hist + threadIdx.x);
#pragma unroll
      for (uint32_t r = 0; r < kSortCtas; ++r) {
        const uint32_t c = r < ctas ? ld_cluster_u32(map_to_cta(mine, r)) : 0u;
        total += c;
        if (r < rank) before += c;
      }
    }
    const uint32_t start = scan256(total, s_warp);
    if (threadIdx.x < 256) s_base[threadIdx.x] = start + before;
    for (int64_t t0 = begin; t0 < end; t0 += static_cast<int64_t>(kSortThreads) * kpt) {
      if (!one_tile) load_and_rank(t0);
      if (threadIdx.x < 256) {  // counts of the warps -> first slots, in warp order
        uint32_t at = s_base[threadIdx.x];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
          const uint32_t c = s_wh[w][threadIdx.x];
          s_wh[w][threadIdx.x] = at;
          at += c;
        }
        s_base[threadIdx.x] = at;
      }
      __syncthreads();
      const int64_t w0 = t0 + static_cast<int64_t>(warp) * 32 * kpt + lane;
#pragma unroll
      for (int j = 0; j < kMaxKpt; ++j) {
        if (j < kpt && w0 + j * 32 < end) {
          const uint32_t slot = s_wh[warp][(key[j] >> shift) & 255u] + off[j];
          __stcg(out_pairs + slot, make_uint2(key[j], pos[j]));
        }
      }
      __syncthreads();
    }
    // the pass's output is visible to the whole cluster, and nobody reads the counts any more
    cluster_sync_all();
  }
}

// One bit per token that occurs (the words were cleared).  A block collects the words of its tokens in a small table in
// shared memory first, so that a frequent token costs one access to the word per block and not one per occurrence; words
// that find their place in the table taken go to memory directly.
constexpr int kMarkTokens = 4, kMarkTable = 1024;
__global__ void __launch_bounds__(256) embedding_mark_kernel(const SortArgs s) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  __shared__ uint32_t s_word[kMarkTable], s_bits[kMarkTable];
  for (int i = threadIdx.x; i < kMarkTable; i += 256) {
    s_word[i] = 0xFFFFFFFFu;  // no word has this index (vocab <= 2^24)
    s_bits[i] = 0u;
  }
  __syncthreads();
  const uint32_t none = static_cast<uint32_t>(s.vocab);
  uint32_t key[kMarkTokens];
#pragma unroll
  for (int j = 0; j < kMarkTokens; ++j) {
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * kMarkTokens + j) * 256 + threadIdx.x;
    key[j] = i < s.n ? token_key(s, i) : none;
  }
#pragma unroll
  for (int j = 0; j < kMarkTokens; ++j) {
    if (key[j] == none) continue;
    const uint32_t word = key[j] >> 5, bit = 1u << (key[j] & 31u), at = word % kMarkTable;
    // (plain reads first: an atomic on an address that a whole warp shares is taken lane after lane)
    uint32_t old = *const_cast<volatile uint32_t*>(&s_word[at]);
    if (old == 0xFFFFFFFFu) old = atomicCAS(&s_word[at], 0xFFFFFFFFu, word);
    if (old == 0xFFFFFFFFu || old == word) {
      if (!(*const_cast<volatile uint32_t*>(&s_bits[at]) & bit)) atomicOr(&s_bits[at], bit);
    } else if (!(__ldcg(s.mark + word) & bit)) atomicOr(s.mark + word, bit);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kMarkTable; i += 256)
    if (s_bits[i]) atomicOr(s.mark + s_word[i], s_bits[i]);
}

__global__ void __launch_bounds__(kSortThreads) embedding_sort_kernel(const EmbeddingArgs a, const SortArgs s) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  __shared__ uint32_t s_hist[256], s_base[256], s_warp[8];
  __shared__ uint32_t s_wh[kSortWarps][256];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const float g = load_scale(a.src_scale), as = a.addend ? load_scale(a.addend_scale) : 0.f;
    if (a.out_scale) *a.out_scale = fmaxf(g * a.c_pow2, as);
    if (!is_pow2_scale(g) || (a.addend && !is_pow2_scale(as))) atomicOr(s.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_SCALE));
  }
  sort_tokens(s, blockIdx.x, gridDim.x, s_hist, s_base, s_warp, s_wh);  // the grid is one cluster
}

// ------------------------------------------------------------------------------------------------- segment sums
struct SegmentArgs {
  const uint2* pair;  // sorted (token, position)
  int64_t n, vocab, chunks;
  int chunk, slabs;
  int64_t line;         // floats per partial row
  float* partial;       // [chunk][2][line]: 0 = run that began in an earlier chunk, 1 = run that goes on in the next
};

// acc (this lane's 8 columns of a complete sum) -> the table's row
template <int ODT>
__device__ __forceinline__ void finish_row(const EmbeddingArgs& a, int64_t row, int v, float fg, float fa, const float* acc) {
  const int n = a.d - v * kVec;
  float f[kVec];
  if (a.addend) {
    uint32_t w[kVec * ElemBytes<ODT>::v / 4];
    load_vec<ODT>(static_cast<const char*>(a.addend) + row * a.addend_ld * ElemBytes<ODT>::v, v, n, w);
    decode_vec<ODT, kVec>(w, f);
#pragma unroll
    for (int e = 0; e < kVec; ++e) f[e] = fmaf(acc[e], fg, f[e] * fa);
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e) f[e] = acc[e] * fg;
  }
  store_vec<ODT>(static_cast<char*>(a.out) + row * a.out_ld * ElemBytes<ODT>::v, v, n, f);
}
__device__ __forceinline__ void output_factors(const EmbeddingArgs& a, float* fg, float* fa) {
  const float gs = load_scale(a.src_scale) * a.c_pow2, as = a.addend ? load_scale(a.addend_scale) : 0.f;
  const float os = fmaxf(gs, as);
  *fg = a.c_rest * (gs / os);
  *fa = as / os;
}

// Rows whose token does not occur: zeros, or the addend brought to the output's scale.  A block takes the 32 rows of one
// word of marks; a warp units of 32 vectors of one row, two at a time.  46 us for the 47000 absent rows of a 50257 x 768 fp32
// table with an addend (6.2 TB/s), of which the sort hides 13.
template <int ODT>
__global__ void __launch_bounds__(256, 6) embedding_fill_kernel(const EmbeddingArgs a, const uint32_t* __restrict__ mark) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  // Launched as a programmatic dependent of the sort and run beside it: the marks are complete (the sort, an ordinary
  // launch behind them, has begun), and the sort touches nothing that is read or written here.
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kFillRows;
  const int rows = static_cast<int>(min(static_cast<int64_t>(kFillRows), a.vocab - row0));
  const uint32_t absent = ~__ldcg(mark + blockIdx.x) & (rows == 32 ? 0xFFFFFFFFu : (1u << rows) - 1u);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float fg, fa;
  output_factors(a, &fg, &fa);
  const int n_vec = (a.d + kVec - 1) / kVec, parts = (n_vec + 31) / 32, units = __popc(absent) * parts;
  constexpr int OW = kVec * ElemBytes<ODT>::v / 4;
  constexpr int kUnits = 2;
  for (int u0 = warp * kUnits; u0 < units; u0 += 8 * kUnits) {
    uint32_t w[kUnits][OW];
    int64_t row[kUnits];
    int v[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int at = (u0 + u) / parts;
      v[u] = (u0 + u - at * parts) * 32 + lane;
      row[u] = u0 + u < units ? row0 + __fns(absent, 0, at + 1) : -1;  // the at-th absent row
      if (row[u] >= 0 && v[u] < n_vec && a.addend)
        load_vec<ODT, true>(static_cast<const char*>(a.addend) + row[u] * a.addend_ld * ElemBytes<ODT>::v, v[u], a.d - v[u] * kVec, w[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if (row[u] >= 0 && v[u] < n_vec) {
        float f[kVec];
        if (a.addend) {
          decode_vec<ODT, kVec>(w[u], f);
#pragma unroll
          for (int e = 0; e < kVec; ++e) f[e] *= fa;
        } else {
#pragma unroll
          for (int e = 0; e < kVec; ++e) f[e] = 0.f;
        }
        store_vec<ODT>(static_cast<char*>(a.out) + row[u] * a.out_ld * ElemBytes<ODT>::v, v[u], a.d - v[u] * kVec, f);
      }
    }
  }
  // what follows in the stream waits for this grid, and through it for the sort
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// What a warp knows of the runs that touch its chunk, from the 32 tokens that begin there and the kShort before them.
struct ChunkRuns {
  uint32_t key, pos;       // this lane's token of the 32
  int len, fwd;            // tokens of the chunk; tokens of its first run from its first token on (32 at most)
  bool from_left;          // the first run began in an earlier chunk ...
  bool left_short;         // ... which sums it alone
  uint32_t last;           // the chunk's last token
  int last_begin;          // first of the 32 that belongs to its run
  int last_count;          // how many of the 32 do
  bool crosses;            // it goes on in the next chunk
  bool last_long;          // its run is longer than kShort (exact where the run begins in this chunk)
};
__device__ __forceinline__ ChunkRuns chunk_runs(const SegmentArgs& s, int64_t chunk) {
  const int lane = threadIdx.x & 31;
  const uint32_t none = static_cast<uint32_t>(s.vocab);
  const int64_t i0 = chunk * s.chunk;
  const int64_t i = i0 + lane, j = i0 - 1 - lane;
  const uint2 kp = i < s.n ? __ldcg(s.pair + i) : make_uint2(none, 0u);
  const uint32_t before = (lane < kShort && j >= 0) ? __ldcg(&s.pair[j].x) : none;
  ChunkRuns r;
  r.key = kp.x;
  r.pos = kp.y;
  r.len = static_cast<int>(min(static_cast<int64_t>(s.chunk), s.n - i0));
  const uint32_t first = __shfl_sync(0xFFFFFFFFu, kp.x, 0);
  r.fwd = __popc(__ballot_sync(0xFFFFFFFFu, kp.x == first));  // (sorted: equal tokens are neighbours)
  const int back = __popc(__ballot_sync(0xFFFFFFFFu, before == first && first != none));
  r.from_left = back > 0;
  r.left_short = r.from_left && back + r.fwd <= kShort;
  r.last = __shfl_sync(0xFFFFFFFFu, kp.x, r.len - 1);
  const uint32_t of_last = __ballot_sync(0xFFFFFFFFu, kp.x == r.last && r.last != none);
  r.last_begin = __ffs(of_last) - 1;
  r.last_count = __popc(of_last);
  r.crosses = r.len < 32 && ((of_last >> r.len) & 1u);
  r.last_long = r.last_count > kShort;
  return r;
}

// One warp per chunk and 256 columns.  65536 rows of 1024, BF16: 34 us, 130 MB from HBM (3.8 TB/s; the look at the tokens comes
// before the first row).  Three blocks per SM with 8 rows of 16 bits in flight per warp: 72.1 us for the whole call at
// 8192 x 768 with an fp32 addend and 88.7 at 65536 x 1024; four blocks (64 registers) 78.0 and 88.0 (6 rows) to 91.1 (8),
// five 81.4 and 89.6.
template <int GDT, int ODT, bool ADD>
__global__ void __launch_bounds__(256, 3) embedding_segment_sum_kernel(const EmbeddingArgs a, const SegmentArgs s) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched as a programmatic dependent: the grid before is complete
  constexpr int GW = kVec * ElemBytes<GDT>::v / 4, OW = ADD ? kVec * ElemBytes<ODT>::v / 4 : 1;
  constexpr int kAhead = GW + (ADD ? OW : 0) <= 4 ? 8 : 4;  // rows in flight, by registers
  const int lane = threadIdx.x & 31;
  const int64_t item = blockIdx.x * 8ll + (threadIdx.x >> 5);
  if (item >= s.chunks * s.slabs) return;
  const int64_t chunk = item / s.slabs;
  const int v = static_cast<int>(item - chunk * s.slabs) * 32 + lane;  // this lane's vector of 8 columns
  const int n = a.d - v * kVec;                                        // columns from its first one to the row's end
  const uint32_t none = static_cast<uint32_t>(s.vocab);
  const ChunkRuns r = chunk_runs(s, chunk);
  // tokens [t_begin, t_end) of the 32 are this warp's; bit t of `ends`: its sum is finished, or interrupted, after token t
  const int known = __popc(__ballot_sync(0xFFFFFFFFu, r.key != none));
  const uint32_t next_key = __shfl_down_sync(0xFFFFFFFFu, r.key, 1);
  const int t_begin = r.left_short ? r.fwd : 0;
  const bool last_is_first = r.from_left && r.last_begin == 0;
  int t_end = min(r.len, known);
  if (r.crosses && !r.last_long && !last_is_first) t_end = r.last_begin + r.last_count;  // finish it beyond the border
  const uint32_t ends = __ballot_sync(0xFFFFFFFFu, lane == t_end - 1 || next_key != r.key);
  const bool open_right = r.crosses && (r.last_long || last_is_first);
  float fg, fa;
  output_factors(a, &fg, &fa);
  const char* G = static_cast<const char*>(a.src);
  float2 acc[kVec / 2];
#pragma unroll
  for (int e = 0; e < kVec / 2; ++e) acc[e] = make_float2(0.f, 0.f);
  for (int t0 = t_begin; t0 < t_end; t0 += kAhead) {
    uint32_t w[kAhead][GW], wa[ADD ? kAhead : 1][OW];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = t0 + u;
      const int64_t p = __shfl_sync(0xFFFFFFFFu, r.pos, t & 31);
      if (t < t_end && n > 0) load_vec<GDT, true>(G + p * a.src_ld * ElemBytes<GDT>::v, v, n, w[u]);
      if constexpr (ADD) {
        const int64_t row = __shfl_sync(0xFFFFFFFFu, r.key, t & 31);
        if (t < t_end && n > 0 && ((ends >> t) & 1u))
          load_vec<ODT, true>(static_cast<const char*>(a.addend) + row * a.addend_ld * ElemBytes<ODT>::v, v, n, wa[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = t0 + u;
      if (t >= t_end) break;
      float f[kVec];
      decode_vec<GDT, kVec>(w[u], f);  // (lanes past the row's end add up what is never stored)
#pragma unroll
      for (int e = 0; e < kVec / 2; ++e) acc[e] = __fadd2_rn(acc[e], make_float2(f[2 * e], f[2 * e + 1]));
      if ((ends >> t) & 1u) {
        const int64_t row = __shfl_sync(0xFFFFFFFFu, r.key, t);
        const bool open_left = r.from_left && t < r.fwd, open = open_left || (t == t_end - 1 && open_right);
        if (n > 0) {
          if (!open) {
            if constexpr (ADD) decode_vec<ODT, kVec>(wa[u], f);
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
              const float x = (e & 1) ? acc[e / 2].y : acc[e / 2].x;
              f[e] = ADD ? fmaf(x, fg, f[e] * fa) : x * fg;
            }
            store_vec<ODT>(static_cast<char*>(a.out) + row * a.out_ld * ElemBytes<ODT>::v, v, n, f);
          } else {
#pragma unroll
            for (int e = 0; e < kVec / 2; ++e) { f[2 * e] = acc[e].x; f[2 * e + 1] = acc[e].y; }
            store_vec<SCALIFY_F32>(reinterpret_cast<char*>(s.partial + (chunk * 2 + (open_left ? 0 : 1)) * s.line), v, kVec, f);
          }
        }
#pragma unroll
        for (int e = 0; e < kVec / 2; ++e) acc[e] = make_float2(0.f, 0.f);
      }
    }
  }
}

// first sorted index whose token is >= key, found by a whole warp (32 probes a step)
__device__ __forceinline__ int64_t lower_bound(const uint2* sorted, int64_t n, uint32_t key) {
  const int lane = threadIdx.x & 31;
  int64_t lo = 0, hi = n;  // the answer lies in [lo, hi]
  while (lo < hi) {
    const int64_t step = (hi - lo + 31) / 32, at = lo + lane * step;
    const uint32_t below = __ballot_sync(0xFFFFFFFFu, at < hi && __ldcg(&sorted[at < hi ? at : lo].x) < key);
    const int m = __popc(below);  // probes 0 .. m-1 lie below
    if (m == 0) return lo;
    const int64_t base = lo + (m - 1) * step;
    lo = base + 1;
    hi = min(hi, base + step);
  }
  return lo;
}

// Long runs: one warp per chunk and 256 columns looks whether such a run begins in its chunk.  A run of a few parts it adds up
// itself; one of many parts (a frequent token) is left to the whole block, whose warps take equal shares of its chunks
// (8192 x 768 with an addend: 72.3 us for the whole call, 73.8 with the block for all of them; this kernel 8.6 and 9.9).
// By chunk and not over a list of the runs alone, which brings long runs together in one block: 100.6 us against 88.5 at
// 65536 x 1024.
constexpr int kWarpParts = 8;
template <int ODT>
__global__ void __launch_bounds__(256, 3) embedding_segment_join_kernel(const EmbeddingArgs a, const SegmentArgs s) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched as a programmatic dependent: the grid before is complete
  constexpr int kAhead = 4;
  __shared__ float s_part[8][kSlab];
  __shared__ int64_t s_parts[8];
  __shared__ uint32_t s_key[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t h = static_cast<int64_t>(blockIdx.x) * 8 + warp;
  const int v = blockIdx.y * 32 + lane, n = a.d - v * kVec;
  int64_t parts = 0;  // chunks h+1 .. h+parts hold slot 0 of the run, chunk h its slot 1
  uint32_t key = 0u;
  if (h < s.chunks) {
    const ChunkRuns r = chunk_runs(s, h);
    if (r.crosses && r.last_long && !(r.from_left && r.last_begin == 0)) {
      key = r.last;
      // chunks that begin with the same token: 32 looked at together, a search only for more
      const int64_t c = (h + 1 + lane) * s.chunk;
      const uint32_t same = __ballot_sync(0xFFFFFFFFu, c < s.n && __ldcg(&s.pair[c < s.n ? c : 0].x) == key);
      parts = same != 0xFFFFFFFFu ? __popc(same) : (lower_bound(s.pair, s.n, key + 1u) - 1) / s.chunk - h;
    }
  }
  float fg, fa;
  output_factors(a, &fg, &fa);
  float acc[kVec];
  auto begin_of = [&](int64_t c) {  // slot 1 of chunk c
    uint32_t w[kVec];
    load_vec<SCALIFY_F32>(reinterpret_cast<const char*>(s.partial + (c * 2 + 1) * s.line), v, kVec, w);
#pragma unroll
    for (int e = 0; e < kVec; ++e) acc[e] = __uint_as_float(w[e]);
  };
  auto add_parts = [&](int64_t c0, int64_t c1) {  // slots 0 of chunks [c0, c1)
    for (int64_t c = c0; c < c1; c += kAhead) {
      uint32_t w[kAhead][kVec];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (c + u < c1) load_vec<SCALIFY_F32>(reinterpret_cast<const char*>(s.partial + (c + u) * 2 * s.line), v, kVec, w[u]);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (c + u < c1) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) acc[e] += __uint_as_float(w[u][e]);
        }
    }
  };
  if (parts > 0 && parts <= kWarpParts && n > 0) {
    begin_of(h);
    add_parts(h + 1, h + 1 + parts);
    finish_row<ODT>(a, key, v, fg, fa, acc);
  }
  if (lane == 0) { s_parts[warp] = parts; s_key[warp] = key; }
  if (!__syncthreads_or(parts > kWarpParts)) return;
  for (int q = 0; q < 8; ++q) {
    const int64_t count = s_parts[q];
    if (count <= kWarpParts) continue;  // the same for every thread
    const int64_t hq = static_cast<int64_t>(blockIdx.x) * 8 + q, share = (count + 7) / 8;
    const int64_t c0 = hq + 1 + warp * share;
#pragma unroll
    for (int e = 0; e < kVec; ++e) acc[e] = 0.f;
    if (n > 0) {
      if (warp == 0) begin_of(hq);
      add_parts(c0, min(hq + 1 + count, c0 + share));
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) s_part[warp][lane * kVec + e] = acc[e];
    __syncthreads();
    if (warp == 0 && n > 0) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        acc[e] = 0.f;
#pragma unroll
        for (int r = 0; r < 8; ++r) acc[e] += s_part[r][lane * kVec + e];
      }
      finish_row<ODT>(a, s_key[q], v, fg, fa, acc);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------- launches
int launch_embedding_lookup(const EmbeddingArgs& a, int w_dt, cudaStream_t st) {
  const int n_vec = (a.d + kVec - 1) / kVec, parts = (n_vec + 32 * kLookupVpt - 1) / (32 * kLookupVpt);
  const int64_t blocks = a.n > 0 ? (a.n * parts + 7) / 8 : 1;  // (an empty batch still has its scale word written)
  if (blocks > 0x7FFFFFFF) return SCALIFY_ERR_SHAPE;
  SCALIFY_DISPATCH_DTYPE(w_dt, WDT, embedding_lookup_kernel<WDT><<<static_cast<unsigned>(blocks), 256, 0, st>>>(a, parts))
  SCALIFY_CUDA_TRY(cudaGetLastError());
  return SCALIFY_OK;
}

// Sorted tokens per work item: long chunks leave fewer partial rows, short ones more loads in flight.  The number of tokens
// alone decides, so that the order of the sums does not depend on the row length or the GPU.  us with 8 and with 16:
// 64 x 768 62.3 and 65.4, 1000 x 768 67.4 and 69.5, 8192 x 768 72.0 and 73.4; 16384 x 1024 56.1 and 53.5, 20000 x 2048 95.7
// and 89.4, 32768 x 64 36.4 and 32.9, 65536 x 64 51.8 and 47.7, 65536 x 1024 100.4 and 87.4.
constexpr int64_t kLongBatch = 16384;
static int chunk_of(int64_t n) { return n < kLongBatch ? kMinChunk : kMaxChunk; }
// Chunks that a workspace has room for: those of every batch of at most n tokens (just below kLongBatch there are more of them)
static int64_t chunk_room(int64_t n) {
  const int64_t own = (n + chunk_of(n) - 1) / chunk_of(n), below = kLongBatch / kMinChunk;
  return n < kLongBatch || own > below ? own : below;
}
static int64_t pad256(int64_t n) { return (n + 255) / 256 * 256; }
size_t embedding_grad_ws_bytes(int64_t n, int64_t d) {
  if (n < 0 || d < 1 || n > 0x7FFFFFFF || d > 0x7FFFFFFF) return kWsMin;
  const int64_t slabs = (d + kSlab - 1) / kSlab;
  return kWsHeader + kMarkBytes + static_cast<size_t>(pad256(8 * n)) * 2 + static_cast<size_t>(chunk_room(n)) * 2 * slabs * kSlab * sizeof(float) + 256;
}

int launch_embedding_grad(const EmbeddingArgs& a, int g_dt, void* ws, cudaStream_t st) {
  WsView v = ws_view(ws);
  SortArgs so = {};
  so.ids = a.ids; so.padding_id = a.padding_id; so.n = a.n; so.vocab = a.vocab; so.status = v.status;
  char* p = static_cast<char*>(v.area);
  so.mark = reinterpret_cast<uint32_t*>(p); p += kMarkBytes;
  for (int i = 0; i < 2; ++i) {
    so.pair[i] = reinterpret_cast<uint2*>(p); p += pad256(8 * a.n);
  }
  so.passes = 1;
  while (so.passes < 4 && (static_cast<uint64_t>(a.vocab) >> (8 * so.passes)) != 0) ++so.passes;
  const int64_t slabs = (a.d + kSlab - 1) / kSlab;
  if (slabs > 65535 || (a.n / kMinChunk + 1) * slabs > 0x7FFFFFFFll * 8) return SCALIFY_ERR_SHAPE;
  SCALIFY_CUDA_TRY(cudaMemsetAsync(so.mark, 0, static_cast<size_t>((a.vocab + 31) / 32) * 4, st));
  if (a.n > 0) {
    const int64_t per = 256 * kMarkTokens;
    embedding_mark_kernel<<<static_cast<unsigned>((a.n + per - 1) / per), 256, 0, st>>>(so);
    SCALIFY_CUDA_TRY(cudaGetLastError());
  }
  // blocks of the sorting cluster: a thread holds a few keys, so short lists take fewer blocks (and cheaper barriers)
  static DeviceOnce once;
  int most = 8;
  int rc = device_once(once, &most, [&](int* value) {
    *value = 8;  // the portable cluster size
    if (cudaFuncSetAttribute(embedding_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
      cudaLaunchConfig_t qc = {};
      qc.gridDim = dim3(kSortCtas); qc.blockDim = dim3(kSortThreads);
      cudaLaunchAttribute qa[1];
      qa[0].id = cudaLaunchAttributeClusterDimension;
      qa[0].val.clusterDim.x = kSortCtas; qa[0].val.clusterDim.y = 1; qa[0].val.clusterDim.z = 1;
      qc.attrs = qa; qc.numAttrs = 1;
      int n = 0;
      if (cudaOccupancyMaxActiveClusters(&n, embedding_sort_kernel, &qc) == cudaSuccess && n > 0) *value = kSortCtas;
    }
    cudaGetLastError();
    return int(SCALIFY_OK);
  });
  if (rc) return rc;
  int ctas = 1;
  while (ctas < most && a.n > static_cast<int64_t>(ctas) * kSortThreads) ctas *= 2;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(kSortThreads); cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = 1;
  SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&cfg, embedding_sort_kernel, a, so));
  cudaLaunchAttribute fattr[1];
  fattr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  fattr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t fcfg = {};
  fcfg.gridDim = dim3(static_cast<unsigned>((a.vocab + kFillRows - 1) / kFillRows)); fcfg.blockDim = dim3(256);
  fcfg.stream = st; fcfg.attrs = fattr; fcfg.numAttrs = 1;
  const uint32_t* mark = so.mark;
  SCALIFY_DISPATCH_WIDE(a.out_dt, ODT, SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&fcfg, embedding_fill_kernel<ODT>, a, mark)))
  if (a.n == 0) return SCALIFY_OK;
  SegmentArgs se = {};
  se.pair = so.pair[(so.passes - 1) & 1];
  se.n = a.n; se.vocab = a.vocab;
  se.slabs = (a.d + kSlab - 1) / kSlab;
  se.chunk = chunk_of(a.n);
  se.chunks = (a.n + se.chunk - 1) / se.chunk;
  se.line = static_cast<int64_t>(se.slabs) * kSlab;
  se.partial = reinterpret_cast<float*>(p);
  const unsigned sum_blocks = static_cast<unsigned>((se.chunks * se.slabs + 7) / 8);
  SCALIFY_DISPATCH_DTYPE(g_dt, GDT, SCALIFY_DISPATCH_WIDE(a.out_dt, ODT, {
    fcfg.gridDim = dim3(sum_blocks);
    if (a.addend) SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&fcfg, embedding_segment_sum_kernel<GDT, ODT, true>, a, se));
    else SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&fcfg, embedding_segment_sum_kernel<GDT, ODT, false>, a, se));
  }))
  SCALIFY_CUDA_TRY(cudaGetLastError());
  if (a.n > kShort) {  // (else no run is long)
    fcfg.gridDim = dim3(static_cast<unsigned>((se.chunks + 7) / 8), se.slabs);
    SCALIFY_DISPATCH_WIDE(a.out_dt, ODT, SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&fcfg, embedding_segment_join_kernel<ODT>, a, se)))
  }
  return SCALIFY_OK;
}

}  // namespace scalify
