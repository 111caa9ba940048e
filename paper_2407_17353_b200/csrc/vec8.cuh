// Rows in vectors of eight elements: 8, 16 or 32 bytes per access, with the ragged end of a row element by element.
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

// Raw words of vector v of a row (n = elements from its first one to the row's end; those past it read as zero).
template <int DT, bool STREAM = false>
__device__ __forceinline__ void load_vec(const char* row, int64_t v, int n, uint32_t* w) {
  constexpr int BYTES = kVec * ElemBytes<DT>::v;
  if (n >= kVec) {
    ld_bytes<BYTES, STREAM>(row + v * BYTES, w);
  } else {
    float f[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) f[e] = e < n ? load_elem<DT>(row, v * kVec + e) : 0.f;
    encode_vec<DT, kVec>(f, w);
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
