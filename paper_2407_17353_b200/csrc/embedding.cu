// Embedding lookup with a constant factor, and its gradient by sorted tokens.
//
// Lookup:    Y_s = wte_s p2(c),  Y_d[i] = round(wte_d[ids[i]] c/p2(c))          (a scalar constant: Section 3.4)
// Gradient:  dwte_d[v] = c/p2(c) sum_{i: ids[i] = v} dY_d[i], scale dY_s p2(c), plus an optional addend by the add rule.
//
// Gradient, three launches:
//   1. sort_and_fill: one cluster of eight blocks sorts (token, position) pairs by token, stably, so that the positions of
//      a token stay in ascending order (least significant digit first, 8 bits a pass, two passes for vocabularies below
//      2^16).  The other blocks of the same launch meanwhile write the rows whose token does not occur (zeros, or the
//      addend): most of the bytes of a large vocabulary, and they do not need the sort, only which tokens occur.
//   2. segment_sum: the sorted tokens are cut into chunks of kChunk whatever the token frequencies are (a token that
//      makes up a twentieth of the batch is common), one warp per chunk and 256 columns.  Runs of equal tokens that lie
//      inside a chunk are finished there; a run that crosses a chunk's border leaves an fp32 partial row.
//   3. segment_join adds the partial rows of such runs in chunk order.
// Every sum is fp32 in an order that the token ids alone determine: no atomics on data, the same bits every time.
// Bound: HBM (the gradient's rows once, the table once, the addend once).
#include "scalify_common.cuh"
#include "scalify_launch.h"
#include "tcgen05_ptx.cuh"

namespace scalify {

namespace {

constexpr int kVec = 8;
constexpr int kSlab = 32 * kVec;      // columns one warp covers
constexpr int kChunk = 32;            // sorted tokens per work item: one per lane when they are loaded
constexpr int kSortCtas = 8;          // blocks of the sorting cluster (the portable limit)
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxKpt = 8;            // keys per thread and tile
constexpr int kMaxFillRows = 32768;   // rows per filling block, at most (a bit each in shared memory)

template <int DT>
__device__ __forceinline__ void load_vec(const char* row, int64_t v, int n, uint32_t* w) {
  constexpr int ES = ElemBytes<DT>::v;
  if (n >= kVec) {
    ld_raw<kVec * ES>(row + v * (kVec * ES), w);
  } else {
    float f[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) f[e] = e < n ? load_elem<DT>(row, v * kVec + e) : 0.f;
    encode_vec<DT, kVec>(f, w);
  }
}
template <int DT>
__device__ __forceinline__ void store_vec(char* row, int64_t v, int n, const float* f) {
  constexpr int ES = ElemBytes<DT>::v;
  if (n >= kVec) {
    uint32_t w[kVec * ES / 4];
    encode_vec<DT, kVec>(f, w);
    st_raw<kVec * ES>(row + v * (kVec * ES), w);
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (e < n) store_elem<DT>(row, v * kVec + e, f[e]);
  }
}

}  // namespace

// ------------------------------------------------------------------------------------------------- lookup
// One warp per row and up to 4 x 256 columns: four vectors of 8 elements per lane are in flight.
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

// ------------------------------------------------------------------------------------------------- sort and fill
struct SortArgs {
  const long long* ids;
  long long padding_id;
  int64_t n, vocab;
  uint32_t* key[2];   // ping-pong: tokens (unknown ones: `vocab`, sorted to the end) ...
  uint32_t* pos[2];   // ... and their positions
  int passes;
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

// The cluster's block `rank` sorts positions [rank * per, rank * per + per) of every pass's input.
__device__ void sort_tokens(const SortArgs& s, uint32_t rank, uint32_t* s_hist, uint32_t* s_base, uint32_t* s_warp,
                            uint32_t (*s_wh)[256]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t per = (s.n + kSortCtas - 1) / kSortCtas;
  const int64_t begin = min(s.n, static_cast<int64_t>(rank) * per), end = min(s.n, begin + per);
  const int kpt = static_cast<int>(min(static_cast<int64_t>(kMaxKpt), (per + kSortThreads - 1) / kSortThreads));
  for (int p = 0; p < s.passes; ++p) {
    const int shift = 8 * p;
    const uint32_t* kin = s.key[(p + 1) & 1];
    const uint32_t* pin = s.pos[(p + 1) & 1];
    uint32_t* kout = s.key[p & 1];
    uint32_t* pout = s.pos[p & 1];
    // digit counts of this block's share
    if (threadIdx.x < 256) s_hist[threadIdx.x] = 0u;
    __syncthreads();
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) {
      const uint32_t key = p == 0 ? token_key(s, i) : __ldcg(kin + i);
      atomicAdd(&s_hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    cluster_sync_all();
    // first output slot of (digit, this block): all smaller digits, then this digit's count in the blocks before
    uint32_t total = 0u, before = 0u;
    if (threadIdx.x < 256) {
      const uint32_t mine = smem_u32(s_hist + threadIdx.x);
#pragma unroll
      for (uint32_t r = 0; r < kSortCtas; ++r) {
        const uint32_t c = ld_cluster_u32(map_to_cta(mine, r));
        total += c;
        if (r < rank) before += c;
      }
    }
    const uint32_t start = scan256(total, s_warp);
    if (threadIdx.x < 256) s_base[threadIdx.x] = start + before;
    // nobody clears its counts for the next pass while another block still reads them
    cluster_sync_all();
    for (int64_t t0 = begin; t0 < end; t0 += static_cast<int64_t>(kSortThreads) * kpt) {
      for (int i = threadIdx.x; i < kSortWarps * 256; i += kSortThreads) (&s_wh[0][0])[i] = 0u;
      __syncthreads();
      // warp w owns 32 * kpt consecutive keys, 32 at a time in order: a key's rank among the warp's keys of the same
      // digit is the count of earlier groups plus the lanes below it in its group
      uint32_t key[kMaxKpt], pos[kMaxKpt], off[kMaxKpt];
      const int64_t w0 = t0 + static_cast<int64_t>(warp) * 32 * kpt;
#pragma unroll
      for (int j = 0; j < kMaxKpt; ++j) {
        const int64_t i = w0 + j * 32 + lane;
        if (j < kpt && i < end) {
          key[j] = p == 0 ? token_key(s, i) : __ldcg(kin + i);
          pos[j] = p == 0 ? static_cast<uint32_t>(i) : __ldcg(pin + i);
        }
      }
#pragma unroll
      for (int j = 0; j < kMaxKpt; ++j) {
        if (j < kpt) {
          const bool in = w0 + j * 32 + lane < end;
          const uint32_t digit = in ? (key[j] >> shift) & 255u : 256u;
          const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
          const uint32_t below = same & ((1u << lane) - 1u);
          const uint32_t earlier = in ? s_wh[warp][digit] : 0u;
          __syncwarp();
          if (in && below == 0u) s_wh[warp][digit] = earlier + __popc(same);
          __syncwarp();
          off[j] = earlier + __popc(below);
        }
      }
      __syncthreads();
      if (threadIdx.x < 256) {  // counts of the warps -> first slots, in warp order
        uint32_t at = s_base[threadIdx.x];
#pragma unroll 8
        for (int w = 0; w < kSortWarps; ++w) {
          const uint32_t c = s_wh[w][threadIdx.x];
          s_wh[w][threadIdx.x] = at;
          at += c;
        }
        s_base[threadIdx.x] = at;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kMaxKpt; ++j) {
        if (j < kpt && w0 + j * 32 + lane < end) {
          const uint32_t slot = s_wh[warp][(key[j] >> shift) & 255u] + off[j];
          __stcg(kout + slot, key[j]);
          __stcg(pout + slot, pos[j]);
        }
      }
      __syncthreads();
    }
    cluster_sync_all();  // the pass's output is complete and visible to the whole cluster
  }
}

// Rows [row0, row1) whose token does not occur: zeros, or the addend brought to the output's scale.
template <int ODT>
__device__ void fill_rows(const EmbeddingArgs& a, const SortArgs& s, int64_t row0, int64_t row1, uint32_t* s_present) {
  for (int i = threadIdx.x; i < (row1 - row0 + 31) / 32; i += kSortThreads) s_present[i] = 0u;
  __syncthreads();
  for (int64_t i0 = threadIdx.x; i0 < s.n; i0 += 8 * kSortThreads) {
    long long id[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) id[u] = i0 + u * kSortThreads < s.n ? s.ids[i0 + u * kSortThreads] : -1;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (id[u] >= row0 && id[u] < row1 && id[u] != s.padding_id)
        atomicOr(&s_present[(id[u] - row0) >> 5], 1u << ((id[u] - row0) & 31));
  }
  __syncthreads();
  const float gs = load_scale(a.src_scale) * a.c_pow2, as = a.addend ? load_scale(a.addend_scale) : 0.f;
  const float fa = as / fmaxf(gs, as);
  const int n_vec = (a.d + kVec - 1) / kVec;
  const int lane = threadIdx.x & 31;
  for (int64_t row = row0 + (threadIdx.x >> 5); row < row1; row += kSortWarps) {
    if ((s_present[(row - row0) >> 5] >> ((row - row0) & 31)) & 1u) continue;
    char* dst = static_cast<char*>(a.out) + row * a.out_ld * ElemBytes<ODT>::v;
    if (a.addend) {
      const char* src = static_cast<const char*>(a.addend) + row * a.addend_ld * ElemBytes<ODT>::v;
      for (int v = lane; v < n_vec; v += 128) {
        uint32_t w[4][kVec * ElemBytes<ODT>::v / 4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (v + 32 * u < n_vec) load_vec<ODT>(src, v + 32 * u, a.d - (v + 32 * u) * kVec, w[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (v + 32 * u < n_vec) {
            float f[kVec];
            decode_vec<ODT, kVec>(w[u], f);
#pragma unroll
            for (int e = 0; e < kVec; ++e) f[e] *= fa;
            store_vec<ODT>(dst, v + 32 * u, a.d - (v + 32 * u) * kVec, f);
          }
        }
      }
    } else {
      float f[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) f[e] = 0.f;
      for (int v = lane; v < n_vec; v += 32) store_vec<ODT>(dst, v, a.d - v * kVec, f);
    }
  }
}

template <int ODT>
__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads) embedding_sort_fill_kernel(
    const EmbeddingArgs a, const SortArgs s, int fill_rows_per_block) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  __shared__ uint32_t s_hist[256], s_base[256], s_warp[8], s_present[kMaxFillRows / 32];
  __shared__ uint32_t s_wh[kSortWarps][256];
  if (blockIdx.x < kSortCtas) {
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      const float g = load_scale(a.src_scale), as = a.addend ? load_scale(a.addend_scale) : 0.f;
      if (a.out_scale) *a.out_scale = fmaxf(g * a.c_pow2, as);
      if (!is_pow2_scale(g) || (a.addend && !is_pow2_scale(as))) atomicOr(s.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_SCALE));
    }
    sort_tokens(s, cluster_ctarank(), s_hist, s_base, s_warp, s_wh);
  } else {
    const int64_t row0 = static_cast<int64_t>(blockIdx.x - kSortCtas) * fill_rows_per_block;
    if (row0 < a.vocab) fill_rows<ODT>(a, s, row0, min(a.vocab, row0 + fill_rows_per_block), s_present);
  }
}

// ------------------------------------------------------------------------------------------------- segment sums
struct SegmentArgs {
  const uint32_t* key;
  const uint32_t* pos;
  int64_t n, vocab, chunks;
  int slabs;
  float* partial;   // [chunk][2][slabs * 256]: 0 = run that began in an earlier chunk, 1 = run that goes on in the next
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

template <int GDT, int ODT>
__global__ void __launch_bounds__(256) embedding_segment_sum_kernel(const EmbeddingArgs a, const SegmentArgs s) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  constexpr int GW = kVec * ElemBytes<GDT>::v / 4;
  constexpr int kAhead = 8;  // rows in flight
  const int lane = threadIdx.x & 31;
  const int64_t item = blockIdx.x * 8ll + (threadIdx.x >> 5);
  if (item >= s.chunks * s.slabs) return;
  const int64_t chunk = item / s.slabs;
  const int v = static_cast<int>(item - chunk * s.slabs) * 32 + lane;  // this lane's vector of 8 columns
  const int64_t i0 = chunk * kChunk;
  const int len = static_cast<int>(min(static_cast<int64_t>(kChunk), s.n - i0));
  const uint32_t none = static_cast<uint32_t>(s.vocab);
  const uint32_t my_key = lane < len ? s.key[i0 + lane] : none;
  const uint32_t my_pos = lane < len ? s.pos[i0 + lane] : 0u;
  const uint32_t left = i0 > 0 ? s.key[i0 - 1] : none, right = i0 + len < s.n ? s.key[i0 + len] : none;
  const bool in = v * kVec < a.d;
  float fg, fa;
  output_factors(a, &fg, &fa);
  float acc[kVec];
#pragma unroll
  for (int e = 0; e < kVec; ++e) acc[e] = 0.f;
  const char* G = static_cast<const char*>(a.src);
  bool first_run = true;  // the run being summed holds the chunk's first token
  for (int t0 = 0; t0 < len; t0 += kAhead) {
    if (__shfl_sync(0xFFFFFFFFu, my_key, t0) == none) break;  // only unknown tokens follow
    uint32_t w[kAhead][GW];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t p = __shfl_sync(0xFFFFFFFFu, my_pos, (t0 + u) & 31);
      const uint32_t k = __shfl_sync(0xFFFFFFFFu, my_key, (t0 + u) & 31);
      if (t0 + u < len && k != none && in) load_vec<GDT>(G + p * a.src_ld * ElemBytes<GDT>::v, v, a.d - v * kVec, w[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = t0 + u;
      const uint32_t k = __shfl_sync(0xFFFFFFFFu, my_key, t & 31);
      const uint32_t next_in = __shfl_sync(0xFFFFFFFFu, my_key, (t + 1) & 31);
      if (t < len && k != none) {
        if (in) {
          float g[kVec];
          decode_vec<GDT, kVec>(w[u], g);
#pragma unroll
          for (int e = 0; e < kVec; ++e) acc[e] += g[e];
        }
        const bool at_end = t + 1 == len;
        if ((at_end ? right : next_in) != k || at_end) {  // the run ends here, or the chunk does
          const bool from_left = first_run && left == k, to_right = at_end && right == k;
          if (in) {
            if (!from_left && !to_right) {
              finish_row<ODT>(a, k, v, fg, fa, acc);
            } else {
              float* slot = s.partial + ((chunk * 2 + (from_left ? 0 : 1)) * s.slabs * 32 + v) * kVec;
              uint32_t ow[kVec];
              encode_vec<SCALIFY_F32, kVec>(acc, ow);
              st_raw<32>(slot, ow);
            }
          }
#pragma unroll
          for (int e = 0; e < kVec; ++e) acc[e] = 0.f;
          first_run = false;
        }
      }
    }
  }
}

// One block per chunk; it has work where a run begins in its chunk and goes on in the next.  Its eight warps add equal
// parts of the run's partial rows, then the parts are added in order.
template <int ODT>
__global__ void __launch_bounds__(256) embedding_segment_join_kernel(const EmbeddingArgs a, const SegmentArgs s) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  __shared__ float s_part[8][kSlab];
  __shared__ int64_t s_last;
  const int64_t h = blockIdx.x;
  const int64_t i0 = h * kChunk, i1 = i0 + kChunk;  // (a last, shorter chunk has no next one)
  if (i1 >= s.n) return;
  const uint32_t k = s.key[i1 - 1], none = static_cast<uint32_t>(s.vocab);
  if (k == none || s.key[i1] != k) return;                                  // nothing goes on
  if (i0 > 0 && s.key[i0] == k && s.key[i0 - 1] == k) return;               // it began earlier
  // the last chunk that holds a part of the run
  if (threadIdx.x == 0) s_last = s.chunks - 1;
  __syncthreads();
  for (int64_t c0 = h + 1; c0 < s.chunks; c0 += blockDim.x) {
    const int64_t c = c0 + threadIdx.x;
    const bool ends = c < s.chunks && (c + 1) * kChunk < s.n && s.key[(c + 1) * kChunk] != k;
    if (ends) atomicMin(reinterpret_cast<unsigned long long*>(&s_last), static_cast<unsigned long long>(c));
    if (__syncthreads_or(ends)) break;
  }
  __syncthreads();
  const int64_t last = s_last, parts = last - h;  // chunks h+1 .. last hold slot 0, chunk h slot 1
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t share = (parts + 7) / 8, c0 = h + 1 + warp * share, c1 = min(last + 1, c0 + share);
  float fg, fa;
  output_factors(a, &fg, &fa);
  const int64_t line = static_cast<int64_t>(s.slabs) * 32 * kVec;
  for (int slab = 0; slab < s.slabs; ++slab) {
    const int v = slab * 32 + lane;
    const bool in = v * kVec < a.d;
    float acc[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) acc[e] = 0.f;
    if (in) {
      if (warp == 0) {
        uint32_t w[kVec];
        ld_raw<32>(s.partial + (h * 2 + 1) * line + v * kVec, w);
#pragma unroll
        for (int e = 0; e < kVec; ++e) acc[e] = __uint_as_float(w[e]);
      }
      for (int64_t c = c0; c < c1; c += 4) {
        uint32_t w[4][kVec];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) w[u][e] = 0u;
          if (c + u < c1) ld_raw<32>(s.partial + (c + u) * 2 * line + v * kVec, w[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < kVec; ++e) acc[e] += __uint_as_float(w[u][e]);
      }
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) s_part[warp][lane * kVec + e] = acc[e];
    __syncthreads();
    if (warp == 0 && in) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) t += s_part[q][lane * kVec + e];
        acc[e] = t;
      }
      finish_row<ODT>(a, k, v, fg, fa, acc);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------- launches
int launch_embedding_lookup(const EmbeddingArgs& a, int w_dt, cudaStream_t st) {
  const int n_vec = (a.d + kVec - 1) / kVec, parts = (n_vec + 32 * kLookupVpt - 1) / (32 * kLookupVpt);
  const int64_t blocks = (a.n * parts + 7) / 8;
  if (blocks > 0x7FFFFFFF) return SCALIFY_ERR_SHAPE;
  SCALIFY_DISPATCH_DTYPE(w_dt, WDT, embedding_lookup_kernel<WDT><<<static_cast<unsigned>(blocks), 256, 0, st>>>(a, parts))
  SCALIFY_CUDA_TRY(cudaGetLastError());
  return SCALIFY_OK;
}

static int64_t pad256(int64_t n) { return (n + 255) / 256 * 256; }
size_t embedding_grad_ws_bytes(int64_t n, int64_t d) {
  if (n < 0 || d < 1 || n > 0x7FFFFFFF || d > 0x7FFFFFFF) return kWsMin;
  const int64_t chunks = (n + kChunk - 1) / kChunk, slabs = (d + kSlab - 1) / kSlab;
  return kWsHeader + static_cast<size_t>(pad256(4 * n)) * 4 + static_cast<size_t>(chunks) * 2 * slabs * kSlab * sizeof(float) + 256;
}

int launch_embedding_grad(const EmbeddingArgs& a, int g_dt, void* ws, cudaStream_t st) {
  WsView v = ws_view(ws);
  SortArgs so = {};
  so.ids = a.ids; so.padding_id = a.padding_id; so.n = a.n; so.vocab = a.vocab; so.status = v.status;
  char* p = static_cast<char*>(v.area);
  for (int i = 0; i < 2; ++i) {
    so.key[i] = reinterpret_cast<uint32_t*>(p); p += pad256(4 * a.n);
    so.pos[i] = reinterpret_cast<uint32_t*>(p); p += pad256(4 * a.n);
  }
  so.passes = 1;
  while (so.passes < 4 && (static_cast<uint64_t>(a.vocab) >> (8 * so.passes)) != 0) ++so.passes;
  // about one filling block per SM: each of them looks through all token ids once
  int64_t rows_per = (a.vocab + sm_count() - kSortCtas - 1) / (sm_count() - kSortCtas);
  rows_per = rows_per < 32 ? 32 : rows_per > kMaxFillRows ? kMaxFillRows : rows_per;
  const int64_t fills = (a.vocab + rows_per - 1) / rows_per;
  const int64_t blocks = (kSortCtas + fills + kSortCtas - 1) / kSortCtas * kSortCtas;
  if (blocks > 0x7FFFFFFF) return SCALIFY_ERR_SHAPE;
  SCALIFY_DISPATCH_WIDE(a.out_dt, ODT, embedding_sort_fill_kernel<ODT><<<static_cast<unsigned>(blocks), kSortThreads, 0, st>>>(a, so, static_cast<int>(rows_per)))
  SCALIFY_CUDA_TRY(cudaGetLastError());
  if (a.n == 0) return SCALIFY_OK;
  SegmentArgs se = {};
  se.key = so.key[(so.passes - 1) & 1];
  se.pos = so.pos[(so.passes - 1) & 1];
  se.n = a.n; se.vocab = a.vocab;
  se.chunks = (a.n + kChunk - 1) / kChunk;
  se.slabs = (a.d + kSlab - 1) / kSlab;
  se.partial = reinterpret_cast<float*>(p);
  const int64_t sum_blocks = (se.chunks * se.slabs + 7) / 8;
  if (sum_blocks > 0x7FFFFFFF) return SCALIFY_ERR_SHAPE;
  SCALIFY_DISPATCH_DTYPE(g_dt, GDT, SCALIFY_DISPATCH_WIDE(a.out_dt, ODT,
      embedding_segment_sum_kernel<GDT, ODT><<<static_cast<unsigned>(sum_blocks), 256, 0, st>>>(a, se)))
  SCALIFY_CUDA_TRY(cudaGetLastError());
  if (se.chunks > 1) {
    SCALIFY_DISPATCH_WIDE(a.out_dt, ODT, embedding_segment_join_kernel<ODT><<<static_cast<unsigned>(se.chunks), 256, 0, st>>>(a, se))
    SCALIFY_CUDA_TRY(cudaGetLastError());
  }
  return SCALIFY_OK;
}

}  // namespace scalify
