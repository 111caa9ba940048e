// The largest logits of every row with their places, and the row's logsumexp: what a teacher hands to the distillation loss.
//
//   V[r][0..k) = the k largest of X[r][.], descending, ids their columns; equal ones by column.  lse = log sum exp(X_s X / T)
//
// One block per row.  First pass: running maximum and sum (base 2) of every thread's elements, and the maxima of the threads.
// The k-th largest of the 512 maxima bounds the row's k-th largest from below: k threads hold an element of at least that.
// Second pass (from the L2): the elements that reach the bound are listed; of random ones hardly more than k do (k = 64:
// 69 on average, k = 256: 355).  Their order: each counts those before it.  Rows with more ties than the list holds find the
// exact k-th value by bisection on its bits and take its first places by a scan.
// Bound by DRAM for the first pass, and by instructions: an element costs a multiply-add, an exponential, an addition and
// its share of the maximum, then one comparison.
#include <math.h>

#include "linear_loss.h"
#include "scalify_common.cuh"
#include "scalify_launch.h"
#include "vec8.cuh"

namespace scalify {

namespace {

constexpr int kTopThreads = 512;
constexpr int kTopList = 2048;   // candidates of a row

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Order-preserving whole numbers, at least 1: -0 and 0 alike, NaN above everything.
__device__ __forceinline__ uint32_t sort_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // (-0 + 0 is 0)
  if (x != x) return 0xFFFFFFFFu;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int DT>
__global__ void __launch_bounds__(kTopThreads, 2) top_logits_kernel(const TopLogitsArgs p) {
  asm volatile("griddepcontrol.launch_dependents;");
  constexpr int kWords = kVec * ElemBytes<DT>::v / 4;
  constexpr int kBits = DT == SCALIFY_F32 ? 32 : DT == SCALIFY_BF16 ? 16 : 19;  // leading bits of a key that can differ
  __shared__ uint32_t s_key[kTopList];
  __shared__ int s_id[kTopList];
  __shared__ float s_m[kTopThreads / 32], s_s[kTopThreads / 32];
  __shared__ int s_count, s_scan[kTopThreads / 32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long row = blockIdx.x;
  const char* x = static_cast<const char*>(p.X) + row * p.ld * ElemBytes<DT>::v;
  const int vocab = static_cast<int>(p.vocab), vecs = (vocab + kVec - 1) / kVec;
  const float c2 = load_scale_after_wait(p.x_scale) * p.inv_temp * 1.4426950408889634f;
  // ---- first pass
  float top = -INFINITY, sum = 0.f;  // top: of the values; the sum is relative to top * c2
  bool nan = false;
  constexpr int kBatch = DT == SCALIFY_F32 ? 2 : 4;
  for (int v0 = threadIdx.x; v0 < vecs; v0 += kTopThreads * kBatch) {
    uint32_t w[kBatch][kWords];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int v = v0 + j * kTopThreads;
      if (v < vecs) load_vec<DT>(x, v, vocab - v * kVec, w[j]);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int v = v0 + j * kTopThreads;
      if (v < vecs) {
        float f[kVec];
        decode_vec<DT, kVec>(w[j], f);
        if (vocab - v * kVec < kVec) {
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (v * kVec + i >= vocab) f[i] = -INFINITY;
        }
        float m = f[0];
#pragma unroll
        for (int i = 1; i < kVec; ++i) m = fmaxf(m, f[i]);
        if (m > top) {
          sum *= ex2((top - m) * c2);
          top = m;
        }
        const float shift = top == -INFINITY ? 0.f : -top * c2;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < kVec; ++i) s += ex2(fmaf(f[i], c2, shift));
        sum += s;
      }
    }
  }
  nan = sum != sum && !(top == INFINITY);
  if (nan || top == INFINITY) {  // (an infinity makes the sum NaN too: whether there is a NaN takes a look)
    nan = false;
    for (int v = threadIdx.x; v < vecs; v += kTopThreads)
      for (int i = 0; i < kVec && v * kVec + i < vocab; ++i) {
        const float f = load_elem<DT>(x, v * kVec + i);
        nan = nan || f != f;
      }
  }
  const bool has = static_cast<int>(threadIdx.x) < vecs;
  const uint32_t mine = !has ? 0u : nan ? 0xFFFFFFFFu : sort_key(top);
  // ---- logsumexp
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
  if (threadIdx.x == 0) s_count = 0;
  // ---- bound: the k-th largest of the threads' maxima
  uint32_t bound = 0u;
  for (int b = 31; b >= 32 - kBits; --b) {
    const uint32_t t = bound | (1u << b);
    if (__syncthreads_count(mine >= t) >= p.k) bound = t;
  }
  __syncthreads();
  if (p.lse && threadIdx.x == 0) {
    float m = -INFINITY, s = 0.f;
    for (int i = 0; i < kTopThreads / 32; ++i) m = fmaxf(m, s_m[i]);
    const float base = m == -INFINITY ? 0.f : m;
    for (int i = 0; i < kTopThreads / 32; ++i) s += s_s[i] * ex2((s_m[i] - base) * c2);
    p.lse[row] = (m * c2 + log2f(s)) * 0.6931471805599453f;
  }
  // ---- second pass: the elements that reach the bound
  auto list = [&](uint32_t least) {
    for (int v0 = threadIdx.x; v0 < vecs; v0 += kTopThreads * kBatch) {
      uint32_t w[kBatch][kWords];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int v = v0 + j * kTopThreads;
        if (v < vecs) load_vec<DT>(x, v, vocab - v * kVec, w[j]);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int v = v0 + j * kTopThreads;
        if (v < vecs) {
          float f[kVec];
          decode_vec<DT, kVec>(w[j], f);
#pragma unroll
          for (int i = 0; i < kVec; ++i) {
            const uint32_t key = sort_key(f[i]);
            if (key >= least && v * kVec + i < vocab) {
              const int at = atomicAdd(&s_count, 1);
              if (at < kTopList) { s_key[at] = key; s_id[at] = v * kVec + i; }
            }
          }
        }
      }
    }
    __syncthreads();
  };
  list(bound);
  int count = s_count;
  if (count > kTopList) {
    // too many ties: the exact k-th value, all above it, and the first places of those equal to it
    uint32_t kth = 0u;
    for (int b = 31; b >= 32 - kBits; --b) {
      const uint32_t t = kth | (1u << b);
      int n = 0;
      for (int v = threadIdx.x; v < vecs; v += kTopThreads) {
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
      for (int i = 0; i < kTopThreads / 32; ++i) total += s_scan[i];
      if (total >= p.k) kth = t;
      __syncthreads();
    }
    const uint32_t least = kth | (0xFFFFFFFFu >> kBits - 1 >> 1);  // (bits below the key's own are all ones or zeros)
    if (threadIdx.x == 0) s_count = 0;
    __syncthreads();
    if (least != 0xFFFFFFFFu) list(least + 1u);  // fewer than k
    count = s_count;
    for (int v0 = 0; v0 < vecs && count < p.k; v0 += kTopThreads) {  // ties, in order of place
      const int v = v0 + threadIdx.x;
      uint32_t ties = 0u;
      if (v < vecs) {
        uint32_t w[kWords];
        float f[kVec];
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
      for (int i = 0; i < kTopThreads / 32; ++i) {
        if (i < warp) before += s_scan[i];
        total += s_scan[i];
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        if (ties >> i & 1u) {
          const int at = count + before;
          if (at < p.k) { s_key[at] = kth; s_id[at] = v * kVec + i; }
          ++before;
        }
      }
      count = min(count + total, p.k);
    }
    __syncthreads();
  }
  // ---- order
  for (int i = threadIdx.x; i < count; i += kTopThreads) {
    const uint32_t key = s_key[i];
    const int id = s_id[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) {
      const uint32_t other = s_key[j];
      rank += other > key || (other == key && s_id[j] < id);
    }
    if (rank < p.k) {
      p.ids[row * p.k + rank] = id;
      const long long o = row * p.v_ld + rank;
      if constexpr (DT == SCALIFY_F32) static_cast<float*>(p.V)[o] = reinterpret_cast<const float*>(x)[id];
      else static_cast<uint16_t*>(p.V)[o] = reinterpret_cast<const uint16_t*>(x)[id];
    }
  }
  if (row == 0 && threadIdx.x == 0 && p.v_scale) *p.v_scale = load_scale_after_wait(p.x_scale);
}

__global__ void copy_scale_kernel(const float* from, float* to) {
  asm volatile("griddepcontrol.launch_dependents;");
  *to = load_scale(from);
}

template <int DT>
int launch_variant(const TopLogitsArgs& a, cudaStream_t st) {
  top_logits_kernel<DT><<<static_cast<unsigned>(a.n), kTopThreads, 0, st>>>(a);
  SCALIFY_CUDA_TRY(cudaGetLastError());
  return SCALIFY_OK;
}

}  // namespace

int launch_top_logits(const TopLogitsArgs& a, cudaStream_t st) {
  if (a.n == 0) {
    if (a.v_scale) copy_scale_kernel<<<1, 1, 0, st>>>(a.x_scale, a.v_scale);
    SCALIFY_CUDA_TRY(cudaGetLastError());
    return SCALIFY_OK;
  }
  if (a.dt == SCALIFY_F32) return launch_variant<SCALIFY_F32>(a, st);
  if (a.dt == SCALIFY_BF16) return launch_variant<SCALIFY_BF16>(a, st);
  return launch_variant<SCALIFY_F16>(a, st);
}

}  // namespace scalify
