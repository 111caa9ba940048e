// Rows in vectors of eight elements: 8, 16 or 32 bytes per access, with the ragged end of a row in smaller ones.
// 32 bytes (fp32) move as ONE access where the address allows it: two 16-byte accesses per lane leave every other half
// sector to a second instruction.
#pragma once

#include "scalify_common.cuh"

namespace scalify {

constexpr int kVec = 8;  // elements per vector

__device__ __forceinline__ bool aligned32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0u; }

template <int BYTES, bool STREAM>
__device__ __forceinline__ void ld_bytes(const char* p, uint32_t* w) {
  if constexpr (BYTES == 32) {
    if (aligned32(p)) {
      SCALIFY_DBG_CHECK_LOAD(p, 32, 8)
      if constexpr (STREAM)
        asm volatile("ld.global.cs.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
      else
        asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
      return;
    }
  }
  if constexpr (STREAM) ld_raw_stream<BYTES>(p, w);
  else ld_raw<BYTES>(p, w);
}
template <int BYTES>
__device__ __forceinline__ void st_bytes(char* p, const uint32_t* w) {
  if constexpr (BYTES == 32) {
    if (aligned32(p)) {
      SCALIFY_DBG_CHECK_STORE(p, 32)
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                   ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
      return;
    }
  }
  st_raw<BYTES>(p, w);
}

// One or two bytes (the last ones of a row), zero-extended.
template <typename T>
__device__ __forceinline__ uint32_t ld_small(const char* p) {
#ifdef SCALIFY_DEBUG
  if (!dbg_ok(p, sizeof(T))) return 0u;
#endif
  return *reinterpret_cast<const T*>(p);
}

// Raw words of vector v of a row (n = elements from its first one to the row's end; those past it read as zero).  The words
// of a row's last, partial vector are loads of their own, and nothing is computed from them here: a row that is loaded ahead
// is not waited for because its length is no multiple of eight (norm gradient, 4099 rows of 5004: 78 -> 60 us; BF16
// throughout: 92 -> 51).  Stores stay element by element: word by word they change nothing there and cost the 65536 x 1024
// embedding gradient 3 us.
template <int DT, bool STREAM = false>
__device__ __forceinline__ void load_vec(const char* row, int64_t v, int n, uint32_t* w) {
  constexpr int BYTES = kVec * ElemBytes<DT>::v;
  const char* p = row + v * BYTES;
  if (n >= kVec) {
    ld_bytes<BYTES, STREAM>(p, w);
  } else {
    const int bytes = n * ElemBytes<DT>::v;
#pragma unroll
    for (int q = 0; q < BYTES / 4; ++q) {
      w[q] = 0u;
      if (4 * q + 4 <= bytes) ld_raw<4>(p + 4 * q, w + q);
      else if (ElemBytes<DT>::v == 2 && 4 * q < bytes) w[q] = ld_small<uint16_t>(p + 4 * q);
      else if (ElemBytes<DT>::v == 1 && 4 * q < bytes) {
        const int rest = bytes - 4 * q;
        w[q] = rest == 1 ? ld_small<uint8_t>(p + 4 * q) : ld_small<uint16_t>(p + 4 * q);
        if (rest == 3) w[q] |= ld_small<uint8_t>(p + 4 * q + 2) << 16;
      }
    }
  }
}
template <int DT>
__device__ __forceinline__ void store_vec(char* row, int64_t v, int n, const float* f) {
  constexpr int BYTES = kVec * ElemBytes<DT>::v;
  if (n >= kVec) {
    uint32_t w[BYTES / 4];
    encode_vec<DT, kVec>(f, w);
    st_bytes<BYTES>(row + v * BYTES, w);
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (e < n) store_elem<DT>(row, v * kVec + e, f[e]);
  }
}

}  // namespace scalify
