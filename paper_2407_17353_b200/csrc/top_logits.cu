// The largest logits of every row with their places, and the row's logsumexp: what a teacher hands to the distillation loss.
//
//   V[r][0..k) = the k largest of X[r][.], descending, ids their columns; equal ones by column.  lse = log sum exp(X_s X / T)
//
// One block per row, of 256 threads (k up to 128), 512, or 1024 (no more rows than SMs).  First pass: running maximum and sum
// (base 2) of every thread's elements, and the maxima of the threads.  The k-th largest of those bounds the row's k-th largest from
// below: k threads hold an element of at least that.  Second pass (from the L2): the elements that reach the bound are listed; of
// random ones about -m log(1 - k/m) do with m threads (k = 64 of 256: 74, k = 256 of 512: 355).  Their order: each counts those
// before it, or (over 128) a sorting network.  Rows with more ties than the list holds find the
// exact k-th value by bisection on its bits and take its first places by a scan.
// A block loads nothing while it looks for the bound, lists and orders, behind five barriers: with six blocks of 256 threads an SM
// 8192 x 50257 BF16 takes 217 us (58 % of the copy rate), and without the logsumexp, most of an element's instructions, still 190.
#include <math.h>

#include <type_traits>

#include "linear_loss.h"
#include "scalify_common.cuh"
#include "scalify_launch.h"
#include "vec8.cuh"

namespace scalify {

namespace {

constexpr int kSlots = 32;       // of vector maxima, per thread
constexpr int kTopList = 2048;   // candidates of a row
constexpr int kTopHits = 512;    // slots that hold them
constexpr int kTopCounted = 128; // candidates that are put in order by counting

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {  // two-wide fp32
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
// Order-preserving whole numbers, at least 1: -0 and 0 alike, NaN above everything.
__device__ __forceinline__ uint32_t sort_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // (-0 + 0 is 0)
  if (x != x) return 0xFFFFFFFFu;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float key_value(uint32_t key) {  // (0, and keys between those of numbers: NaN)
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// Maxima that a NaN goes through, of one fp32 or two 16-bit values.
template <int DT> __device__ __forceinline__ uint32_t word_max(uint32_t a, uint32_t b) {
  if constexpr (DT == SCALIFY_F32) {
    return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b)));
  } else {
    uint32_t y;
    if constexpr (DT == SCALIFY_BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
  }
}
// what a slot holds of it: fp32, or the larger of the two halves
template <int DT> struct SlotOf { using type = typename std::conditional<DT == SCALIFY_F32, uint32_t, uint16_t>::type; };
template <int DT> __device__ __forceinline__ uint32_t slot_max(uint32_t w) {
  return DT == SCALIFY_F32 ? w : word_max<DT>(w, w >> 16) & 0xFFFFu;
}
template <int DT> __device__ __forceinline__ float slot_value(uint32_t s) {
  return DT == SCALIFY_F32 ? __uint_as_float(s) : DT == SCALIFY_BF16 ? bf16_bits_to_float(s) : __half2float(__ushort_as_half(static_cast<unsigned short>(s)));
}
template <int DT> __device__ __forceinline__ float word_top(uint32_t w) {
  if constexpr (DT == SCALIFY_F32) {
    return __uint_as_float(w);
  } else {
    float f[2];
    decode_vec<DT, 2>(&w, f);
    return max_nan(f[0], f[1]);
  }
}
template <int DT> __device__ __forceinline__ constexpr uint32_t lowest_word() {  // -inf
  return DT == SCALIFY_F32 ? 0xFF800000u : DT == SCALIFY_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
}

template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS, 1536 / THREADS) top_logits_kernel(const TopLogitsArgs p) {
  asm volatile("griddepcontrol.launch_dependents;");
  constexpr int kWords = kVec * ElemBytes<DT>::v / 4, kWarps = THREADS / 32;
  constexpr int kBits = DT == SCALIFY_F32 ? 32 : DT == SCALIFY_BF16 ? 16 : 19;  // leading bits of a key that can differ
  using Slot = typename SlotOf<DT>::type;
  extern __shared__ __align__(16) uint32_t s_raw[];
  Slot* s_slot = reinterpret_cast<Slot*>(s_raw);                // [turns / per][THREADS]
  uint64_t* s_list = reinterpret_cast<uint64_t*>(s_raw);        // then, in their place: a candidate's key, and its place, inverted
  __shared__ float s_m[kWarps], s_s[kWarps];
  __shared__ uint32_t s_mine[THREADS], s_bound;
  __shared__ int s_hit[kTopHits], s_hits, s_count, s_scan[kWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long row = blockIdx.x;
  const char* x = static_cast<const char*>(p.X) + row * p.ld * ElemBytes<DT>::v;
  const int vocab = static_cast<int>(p.vocab), vecs = (vocab + kVec - 1) / kVec;
  const float scale = load_scale_after_wait(p.x_scale) * p.inv_temp, c2 = scale * 1.4426950408889634f;
  // ---- first pass: the thread's maximum and sum; the maxima of its vectors, `per` vectors to a slot
  const int turns = (vecs + THREADS - 1) / THREADS, per = (turns + kSlots - 1) / kSlots;
  float top = -INFINITY, sum = 0.f;  // the sum is relative to top * c2
  bool nan = false;
  Slot* slot = s_slot + threadIdx.x;
  int in_slot = 0;  // vectors in the slot so far
  constexpr int kBatch = DT == SCALIFY_F32 ? 2 : 4;
  for (int t0 = 0; t0 < turns; t0 += kBatch) {
    uint32_t w[kBatch][kWords];
    if ((t0 + kBatch) * THREADS * kVec <= vocab) {
#pragma unroll
      for (int j = 0; j < kBatch; ++j) ld_bytes<kWords * 4, false>(x + static_cast<int64_t>((t0 + j) * THREADS + threadIdx.x) * kWords * 4, w[j]);
    } else {  // the row's end: -inf behind it
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int v = (t0 + j) * THREADS + threadIdx.x, n = vocab - v * kVec;
        if (n > 0) load_vec<DT>(x, v, n, w[j]);
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
          const int first = q * kVec / kWords;
          if (first >= n) w[j][q] = lowest_word<DT>();
          else if (DT != SCALIFY_F32 && first + 1 >= n) w[j][q] = (w[j][q] & 0xFFFFu) | (lowest_word<DT>() & 0xFFFF0000u);
        }
      }
    }
    uint32_t most = lowest_word<DT>();
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      uint32_t m = w[j][0];
#pragma unroll
      for (int q = 1; q < kWords; ++q) m = word_max<DT>(m, w[j][q]);
      if (t0 + j < turns) {
        const uint32_t mine = slot_max<DT>(m);
        *slot = static_cast<Slot>(in_slot == 0 ? mine : word_max<DT>(mine, *slot));
        if (++in_slot == per) { in_slot = 0; slot += THREADS; }
      }
      most = word_max<DT>(most, m);
    }
    const float largest = word_top<DT>(most);
    nan = nan || largest != largest;
    // (+inf: relative to the largest finite number, to which finite exponents are nothing and infinite ones infinite; as a bound
    // for the selection it is only lower)
    const float m = fminf(largest, 3.402823466e38f);
    if (m > top) {
      sum *= ex2((top - m) * c2);
      top = m;
    }
    if (p.lse) {
      const float shift = top == -INFINITY ? 0.f : -top * c2;
      float2 s = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (t0 + j >= turns) break;
        float f[kVec];
        decode_vec<DT, kVec>(w[j], f);
        if (fabsf(shift) > 1024.f) {  // (rows of the type's lowest value and the like: its rounding would count, so differences first)
#pragma unroll
          for (int i = 0; i < kVec; ++i) s.x += ex2((f[i] - top) * c2);
          continue;
        }
#pragma unroll
        for (int i = 0; i < kVec; i += 2) {
          const float2 y = fma2(make_float2(f[i], f[i + 1]), make_float2(c2, c2), make_float2(shift, shift));
          s = add2(s, make_float2(ex2(y.x), ex2(y.y)));
        }
      }
      sum += s.x + s.y;
    }
  }
  s_mine[threadIdx.x] = static_cast<int>(threadIdx.x) < vecs ? nan ? 0xFFFFFFFFu : sort_key(top) : 0u;
  if (p.lse) {
    float m = top, s = sum;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float m2 = __shfl_xor_sync(0xFFFFFFFFu, m, o), s2 = __shfl_xor_sync(0xFFFFFFFFu, s, o);
      const float mm = fmaxf(m, m2), base = mm == -INFINITY ? 0.f : mm;
      s = s * ex2((m - base) * c2) + s2 * ex2((m2 - base) * c2);
      m = mm;
    }
    if (lane == 0) { s_m[warp] = m; s_s[warp] = s; }
  }
  if (threadIdx.x == 0) { s_count = 0; s_hits = 0; }
  __syncthreads();
  // ---- bound: the k-th largest of the threads' maxima, its leading 16 bits (two at a time; the rest zero, a little lower)
  if (warp == 0) {
    uint32_t key[kWarps], bound = 0u;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) key[i] = s_mine[i * 32 + lane];
    uint32_t all = 0xFFFFFFFFu, any = 0u;  // bits that every key has, and that some have: the search begins where they differ
#pragma unroll
    for (int i = 0; i < kWarps; ++i) { all &= key[i]; any |= key[i]; }
    all = __reduce_and_sync(0xFFFFFFFFu, all);
    any = __reduce_or_sync(0xFFFFFFFFu, any);
    const int first = all == any ? 14 : (31 - __clz(all ^ any)) & ~1;  // (both are even numbers of the bit pairs below)
    bound = first >= 30 ? 0u : all & (0xFFFFFFFFu << (first + 2));
#pragma unroll 1
    for (int b = first; b >= 16; b -= 2) {
      int n1 = 0, n2 = 0, n3 = 0;
      const uint32_t t1 = bound | (1u << b), t2 = bound | (2u << b), t3 = bound | (3u << b);
#pragma unroll
      for (int i = 0; i < kWarps; ++i) { n1 += key[i] >= t1; n2 += key[i] >= t2; n3 += key[i] >= t3; }
      n1 = __reduce_add_sync(0xFFFFFFFFu, n1 | n2 << 16);  // (at most 1024 each)
      n3 = __reduce_add_sync(0xFFFFFFFFu, n3);
      bound = n3 >= p.k ? t3 : n1 >> 16 >= p.k ? t2 : (n1 & 0xFFFF) >= p.k ? t1 : bound;
    }
    if (lane == 0) s_bound = bound;
  } else if (warp == 1 && p.lse) {
    float m = lane < kWarps ? s_m[lane] : -INFINITY, s = lane < kWarps ? s_s[lane] : 0.f;
    float most = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    s *= ex2((m - (most == -INFINITY ? 0.f : most)) * c2);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane == 0) p.lse[row] = fmaf(most, scale, logf(s));
  }
  __syncthreads();
  const uint32_t bound = s_bound;
  // ---- the elements that reach the bound: first the slots that do, then their vectors, all at once
  auto list_element = [&](float f, int id, uint32_t least) {
    const uint32_t key = sort_key(f);
    if (key >= least) {
      const int at = atomicAdd(&s_count, 1);
      if (at < kTopList) s_list[at] = static_cast<uint64_t>(key) << 32 | ~static_cast<uint32_t>(id);
    }
  };
  const float least_value = bound == 0u ? -INFINITY : key_value(bound);
  slot = s_slot + threadIdx.x;
  for (int t0 = 0; t0 < turns; t0 += per, slot += THREADS) {
    if (t0 * THREADS + static_cast<int>(threadIdx.x) < vecs && !(slot_value<DT>(*slot) < least_value)) {
      const int at = atomicAdd(&s_hits, 1);
      if (at < kTopHits) s_hit[at] = t0 * THREADS + threadIdx.x;
    }
  }
  __syncthreads();
  const int hits = s_hits;
  if (hits <= kTopHits) {
    for (int i = threadIdx.x; i < hits * per * kVec; i += THREADS) {
      const int v = i / kVec, h = per == 1 ? v : v / per, id = (s_hit[h] + (v - h * per) * THREADS) * kVec + i % kVec;
      if (id < vocab) list_element(load_elem<DT>(x, id), id, bound);
    }
  } else if (threadIdx.x == 0) {
    s_count = kTopList + 1;
  }
  __syncthreads();
  int count = s_count;
  if (count > kTopList) {
    // too many ties: the exact k-th value, all above it, and the first places of those equal to it
    uint32_t kth = 0u;
    for (int b = 31; b >= 32 - kBits; --b) {
      const uint32_t t = kth | (1u << b);
      int n = 0;
      for (int v = threadIdx.x; v < vecs; v += THREADS) {
        uint32_t w[kWords];
        float f[kVec];
        load_vec<DT>(x, v, vocab - v * kVec, w);
        decode_vec<DT, kVec>(w, f);
#pragma unroll
        for (int i = 0; i < kVec; ++i) n += v * kVec + i < vocab && sort_key(f[i]) >= t;
      }
      n = __reduce_add_sync(0xFFFFFFFFu, n);
      if (lane == 0) s_scan[warp] = n;
      __syncthreads();
      int total = 0;
      for (int i = 0; i < kWarps; ++i) total += s_scan[i];
      if (total >= p.k) kth = t;
      __syncthreads();
    }
    const uint32_t least = kth | (0xFFFFFFFFu >> kBits - 1 >> 1);  // (bits below the key's own are all ones or zeros)
    if (threadIdx.x == 0) s_count = 0;
    __syncthreads();
    if (least != 0xFFFFFFFFu)  // fewer than k
      for (int id = threadIdx.x; id < vocab; id += THREADS) list_element(load_elem<DT>(x, id), id, least + 1u);
    __syncthreads();
    count = s_count;
    for (int v0 = 0; v0 < vecs && count < p.k; v0 += THREADS) {  // ties, in order of place
      const int v = v0 + threadIdx.x;
      uint32_t ties = 0u;
      float f[kVec] = {};
      if (v < vecs) {
        uint32_t w[kWords];
        load_vec<DT>(x, v, vocab - v * kVec, w);
        decode_vec<DT, kVec>(w, f);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const uint32_t key = sort_key(f[i]);
          if (v * kVec + i < vocab && key >= kth && key <= least) ties |= 1u << i;
        }
      }
      int before = __popc(ties);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, before, o);
        if (lane >= o) before += u;
      }
      __syncthreads();
      if (lane == 31) s_scan[warp] = before;
      __syncthreads();
      int total = 0;
      before -= __popc(ties);
      for (int i = 0; i < kWarps; ++i) {
        if (i < warp) before += s_scan[i];
        total += s_scan[i];
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        if (ties >> i & 1u) {
          const int at = count + before;
          if (at < p.k) s_list[at] = static_cast<uint64_t>(sort_key(f[i])) << 32 | ~static_cast<uint32_t>(v * kVec + i);
          ++before;
        }
      }
      count = min(count + total, p.k);
    }
    __syncthreads();
  }
  // ---- order: few candidates count those before them, many are sorted
  auto put = [&](int rank, uint64_t c) {
    p.ids[row * p.k + rank] = static_cast<uint32_t>(~c);
    store_elem<DT>(p.V, row * p.v_ld + rank, key_value(static_cast<uint32_t>(c >> 32)));  // (exact: it was of this type)
  };
  if (count <= kTopCounted) {
    if (static_cast<int>(threadIdx.x) == count && (count & 1)) s_list[count] = 0u;
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < count) {
      const uint64_t c = s_list[threadIdx.x];
      int rank = 0;
      for (int j = 0; j < count; j += 2) {
        const ulonglong2 other = *reinterpret_cast<const ulonglong2*>(s_list + j);
        rank += (other.x > c) + (other.y > c);
      }
      if (rank < p.k) put(rank, c);
    }
  } else {
    int size = 2 * kTopCounted;
    while (size < count) size *= 2;
    for (int i = count + threadIdx.x; i < size; i += THREADS) s_list[i] = 0u;
    for (int run = 2; run <= size; run *= 2) {
      for (int gap = run / 2; gap > 0; gap /= 2) {
        __syncthreads();
        for (int i = threadIdx.x; i < size / 2; i += THREADS) {
          const int lo = 2 * i - (i & (gap - 1)), hi = lo + gap;
          const uint64_t u = s_list[lo], v = s_list[hi];
          if ((u < v) == ((lo & run) == 0)) { s_list[lo] = v; s_list[hi] = u; }
        }
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.k; i += THREADS) put(i, s_list[i]);
  }
  if (row == 0 && threadIdx.x == 0 && p.v_scale) *p.v_scale = load_scale_after_wait(p.x_scale);
}

__global__ void copy_scale_kernel(const float* from, float* to) {
  asm volatile("griddepcontrol.launch_dependents;");
  *to = load_scale(from);
}

template <int DT, int THREADS>
int launch_variant(const TopLogitsArgs& a, cudaStream_t st) {
  using Slot = typename SlotOf<DT>::type;
  constexpr int kMost = kSlots * THREADS * static_cast<int>(sizeof(Slot)) > kTopList * 8 ? kSlots * THREADS * static_cast<int>(sizeof(Slot)) : kTopList * 8;
  const long long turns = ((a.vocab + kVec - 1) / kVec + THREADS - 1) / THREADS;
  int bytes = static_cast<int>(turns < kSlots ? turns : kSlots) * THREADS * static_cast<int>(sizeof(Slot));
  if (bytes < kTopList * 8) bytes = kTopList * 8;
  auto kernel = top_logits_kernel<DT, THREADS>;
  static DeviceOnce once;
  const int rc = device_once(once, nullptr, [&](int*) {
    SCALIFY_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost));
    return int(SCALIFY_OK);
  });
  if (rc) return rc;
  kernel<<<static_cast<unsigned>(a.n), THREADS, bytes, st>>>(a);
  SCALIFY_CUDA_TRY(cudaGetLastError());
  return SCALIFY_OK;
}
// Blocks of 1024 threads where there is at most one row per SM: the row's length is what takes the time then.
template <int DT>
int launch_type(const TopLogitsArgs& a, cudaStream_t st) {
  if (a.n <= sm_count()) return launch_variant<DT, 1024>(a, st);
  return a.k <= 128 ? launch_variant<DT, 256>(a, st) : launch_variant<DT, 512>(a, st);
}

}  // namespace

int launch_top_logits(const TopLogitsArgs& a, cudaStream_t st) {
  if (a.n == 0) {
    if (a.v_scale) copy_scale_kernel<<<1, 1, 0, st>>>(a.x_scale, a.v_scale);
    SCALIFY_CUDA_TRY(cudaGetLastError());
    return SCALIFY_OK;
  }
  if (a.dt == SCALIFY_F32) return launch_type<SCALIFY_F32>(a, st);
  if (a.dt == SCALIFY_BF16) return launch_type<SCALIFY_BF16>(a, st);
  return launch_type<SCALIFY_F16>(a, st);
}

}  // namespace scalify
