// Residual addition + root-mean-square norm with an 8-bit (or wide) output, and its gradient.
//
// Forward, per row of d elements (add rule of Section 3.2, normalisation rule of Section 3.2.1 / Appendix C.2):
//   H_s = max(X_s, R_s),   H_d = round(X_d X_s/H_s + R_d R_s/H_s)
//   n = H_d rinv,  rinv = (mean(H_d^2) + eps)^(-1/2)        (the data component; the result carries scale 1)
//   Y_s = gamma_s,  Y_d = round(n gamma_d);  block-scaled: round(n gamma_d 2^-e), one exponent per 32 elements
// The norm is taken of H AS STORED: the gradient, which reads H, is then the derivative of what was computed, and the
// call equals scalify_scaled_add followed by the norm of its output bit for bit.
//
// Backward, with g = G_d gamma_d:   dh = rinv (g - n mean(g n)),  scale G_s gamma_s / H_s, then the add rule with the
// gradient of H itself (residual path):  dX_s = max(G_s gamma_s / H_s, Gr_s);  dgamma = sum_rows G_d n / kf(R).
//
// Both directions are bound by HBM: every array is read or written once.  A row lives in the registers of a team: one
// warp for d <= 768 (1 to 3 vectors of 8 elements per lane, several rows per block, no barrier), otherwise one block with
// 2 vectors per thread (4 above d = 8192; gradient: 6144) and two barriers per row.
#include "scalify_common.cuh"
#include "scalify_launch.h"
#include "vec8.cuh"

namespace scalify {

namespace {

constexpr int kWarpRows = 4;     // rows (warps) per block of the warp-per-row forms: forward ...
constexpr int kBwdRows = 8;      // ... and backward (a line of column sums per block)
// Longest row one warp holds, with three vectors per lane; a fourth costs more than the block form's barriers.  8192 rows of
// BF16, us with a warp and with a block per row, forward, then backward: d = 512 7.6 and 9.6, 13.9 and 20.8; 640 10.7 and 12.3,
// 18.7 and 19.2; 704 11.3 and 12.6, 18.8 and 19.9; 768 11.9 and 12.7, 19.3 and 20.0; 776 14.0 and 12.8, 23.5 and 20.8; 896 15.3 and
// 13.4, 25.0 and 23.0; 1024 16.3 and 14.1, 26.0 and 24.4.  1000 rows with an fp32 stream: 512 3.8 both, 6.9 and 13.7; 640 4.5 and
// 4.1, 8.2 and 10.0; 768 4.8 and 4.2, 8.3 and 10.0; 776 5.5 and 4.2, 10.6 and 10.3.
constexpr int kWarpMaxD = 768;
constexpr int kPrefetchThreads = 384;  // of the backward form that loads the next row ahead (168 registers a thread)
constexpr int kBwdWarpBlocks = 2;      // resident blocks per SM of the backward warp-per-row form
constexpr int kBlockThreads = 512;  // most threads of the block-per-row forms (leaves 128 registers a thread)

// one uniform branch per vector on the output's type: a template per type would multiply the kernels by five
__device__ __forceinline__ void store_vec_dt(int dt, char* row, int v, int n, const float* f) {
  SCALIFY_DISPATCH_DTYPE(dt, DT, store_vec<DT>(row, v, n, f))
}
__device__ __forceinline__ void load_gamma(const void* gamma, int dt, int v, int n, float* f) {
  if (!gamma) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) f[e] = 1.0f;
    return;
  }
  const char* p = static_cast<const char*>(gamma);
  SCALIFY_DISPATCH_WIDE(dt, DT, {
    uint32_t w[kVec * ElemBytes<DT>::v / 4];
    load_vec<DT>(p, v, n, w);
    decode_vec<DT, kVec>(w, f);
  })
}

// sum over the team that holds a row; every thread returns it (fixed order)
template <bool BLOCK>
__device__ __forceinline__ float team_sum(float x, float* s_red) {
  x = warp_sum_f32(x);
  if constexpr (BLOCK) {
    __syncthreads();  // the previous use of s_red is over
    if ((threadIdx.x & 31) == 0) s_red[threadIdx.x >> 5] = x;
    __syncthreads();
    const int nw = blockDim.x >> 5;
    x = (threadIdx.x & 31) < nw ? s_red[threadIdx.x & 31] : 0.f;
    x = warp_sum_f32(x);
  }
  return x;
}

// max of `m` and the magnitudes of one vector's words, as DT bit patterns (16-bit formats two at a time, in both halves)
template <int DT>
__device__ __forceinline__ uint32_t max_bits(const uint32_t* w, uint32_t m) {
#pragma unroll
  for (int q = 0; q < kVec * ElemBytes<DT>::v / 4; ++q)
    m = ElemBytes<DT>::v == 2 ? __vmaxu2(m, w[q] & 0x7FFF7FFFu) : max(m, w[q] & 0x7FFFFFFFu);
  return m;
}
// ... and as the fp32 bit pattern of the value
template <int DT>
__device__ __forceinline__ uint32_t max_bits_to_f32(uint32_t m) {
  if constexpr (DT == SCALIFY_F32) return m;
  const uint32_t h = max(m & 0xFFFFu, m >> 16);
  if constexpr (DT == SCALIFY_BF16) return h << 16;
  return __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(h))));
}

}  // namespace

// ------------------------------------------------------------------------------------------------- forward
// 8192 x 768 BF16 -> E4M3: 12.0 us (44 MB; 4.2 us is what one row takes, so that 5.6 TB/s move in the rest); 10000 x 4096 with
// an fp32 stream and block scales: 73.2 us, 6.2 TB/s; 4099 x 5004: 40 us, 5.6 TB/s.
template <int XDT, int HDT, int VPT, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? kBlockThreads : 32 * kWarpRows) add_rmsnorm_kernel(const RmsNormArgs a) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  __shared__ float s_red[32];
  const int team = BLOCK ? blockDim.x : 32;
  const int lane = BLOCK ? threadIdx.x : threadIdx.x & 31;
  const int64_t row = BLOCK ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * kWarpRows + (threadIdx.x >> 5);
  const float xs = load_scale(a.x_scale), rs = a.R ? load_scale(a.r_scale) : 0.f, gs = a.gamma ? load_scale(a.gamma_scale) : 1.0f;
  const float hs = fmaxf(xs, rs);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (a.h_scale) *a.h_scale = hs;
    if (a.y_scale) *a.y_scale = gs;
    if (a.status && !(is_pow2_scale(xs) && (!a.R || is_pow2_scale(rs)) && is_pow2_scale(gs)))
      atomicOr(a.status, static_cast<uint32_t>(SCALIFY_DEV_BAD_SCALE));
  }
  const bool live = row < a.rows;
  if (!live && !a.sf) return;
  const int n_vec = (a.d + kVec - 1) / kVec;
  float h[VPT][kVec];
  if (live) {
    constexpr int XW = kVec * ElemBytes<XDT>::v / 4, HW = kVec * ElemBytes<HDT>::v / 4;
    const char* xrow = static_cast<const char*>(a.X) + row * a.x_ld * (a.R ? ElemBytes<XDT>::v : ElemBytes<HDT>::v);
    const char* rrow = a.R ? static_cast<const char*>(a.R) + row * a.r_ld * ElemBytes<HDT>::v : nullptr;
    char* hrow = a.R ? static_cast<char*>(a.H) + row * a.h_ld * ElemBytes<HDT>::v : nullptr;
    float ss = 0.f;
    if (a.R) {
      const float fx = xs / hs, fr = rs / hs;  // powers of two: exact
      uint32_t wx[VPT][XW], wr[VPT][HW];
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * team;
        if (v < n_vec) {
          load_vec<XDT, true>(xrow, v, a.d - v * kVec, wx[i]);
          load_vec<HDT, true>(rrow, v, a.d - v * kVec, wr[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * team;
        float x[kVec];
        if (v < n_vec) {
          decode_vec<XDT, kVec>(wx[i], x);
          decode_vec<HDT, kVec>(wr[i], h[i]);
#pragma unroll
          for (int e = 0; e < kVec; ++e) h[i][e] = round_through<HDT>(fmaf(x[e], fx, h[i][e] * fr));
          store_vec<HDT>(hrow, v, a.d - v * kVec, h[i]);
        } else {
#pragma unroll
          for (int e = 0; e < kVec; ++e) h[i][e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) ss = fmaf(h[i][e], h[i][e], ss);
      }
    } else {
      uint32_t wr[VPT][HW];
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * team;
        if (v < n_vec) load_vec<HDT, true>(xrow, v, a.d - v * kVec, wr[i]);
      }
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        if (lane + i * team < n_vec) decode_vec<HDT, kVec>(wr[i], h[i]);
        else {
#pragma unroll
          for (int e = 0; e < kVec; ++e) h[i][e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) ss = fmaf(h[i][e], h[i][e], ss);
      }
    }
    ss = team_sum<BLOCK>(ss, s_red);
    const float rinv = __frsqrt_rn(ss / static_cast<float>(a.d) + a.eps);
    if (lane == 0 && a.rinv) a.rinv[row] = rinv;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int v = lane + i * team;
      if (v < n_vec) {
        float g[kVec];
        load_gamma(a.gamma, a.gamma_dt, v, a.d - v * kVec, g);
#pragma unroll
        for (int e = 0; e < kVec; ++e) h[i][e] = h[i][e] * rinv * g[e];
        if (!a.sf) store_vec_dt(a.y_dt, static_cast<char*>(a.Y) + row * a.y_ld * a.y_es, v, a.d - v * kVec, h[i]);
      }
    }
  }
  if (!a.sf) return;
  // Block scales (d is a multiple of 128, so a vector is whole and the four lanes of a block of 32 act together).
  // The exponent is that of scalify_mx_quantize; sixteen lanes hold the four blocks of one 128-element tile row, whose
  // bytes are neighbours.  Rows between `rows` and the next multiple of 256 get the code 127.
  const int emax = a.y_dt == SCALIFY_E4M3 ? 8 : 15;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int v = lane + i * team;
    const bool in = v < n_vec;
    uint32_t amax = 0u;
    if (live && in) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) amax = max(amax, abs_bits(h[i][e]));
    }
    amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
    int ex = 0;
    if (amax != 0u && amax < 0x7F800000u) {
      ex = static_cast<int>(amax >> 23) - 127;
      if ((amax >> 23) == 0u) ex = -127 - __clz(amax << 9);
      ex = max(-127, min(127, ex - emax));
    }
    uint32_t code = static_cast<uint32_t>(ex + 127);
    const int l0 = threadIdx.x & 16;
    const uint32_t c1 = __shfl_sync(0xFFFFFFFFu, code, l0 + 4), c2 = __shfl_sync(0xFFFFFFFFu, code, l0 + 8),
                   c3 = __shfl_sync(0xFFFFFFFFu, code, l0 + 12);
    if (in) {
      if (live) {
        const uint32_t field = static_cast<uint32_t>(127 - ex);
        const float s = __uint_as_float(field ? field << 23 : 0x00400000u);  // 2^-ex, exact
#pragma unroll
        for (int e = 0; e < kVec; ++e) h[i][e] *= s;
        char* yrow = static_cast<char*>(a.Y) + row * a.y_ld;
        if (a.y_dt == SCALIFY_E4M3) store_vec<SCALIFY_E4M3>(yrow, v, kVec, h[i]);
        else store_vec<SCALIFY_E5M2>(yrow, v, kVec, h[i]);
      }
      if ((threadIdx.x & 15) == 0) {
        const uint32_t w = code | (c1 << 8) | (c2 << 16) | (c3 << 24);
        uint8_t* p = a.sf + (row / 128 * (a.d / 128) + v / 16) * 512 + (row % 32) * 16 + (row % 128) / 32 * 4;
        st_raw<4>(p, &w);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------- backward
// Persistent teams walk the rows (grid stride); a team keeps its columns' share of dgamma in registers over all its
// rows and leaves it in the workspace, one line per block, added in block order by the second launch: the result does
// not depend on scheduling.  The statistic of the stored dX travels the same way.
// The launch bounds leave 128 registers a thread to the warp-per-row form (two blocks of eight warps per SM, which is
// what covers the load latency there).  The block-per-row form with 2 vectors per thread holds the NEXT row's words in
// registers while it works on the current one, so that the two barriers of a row do not leave the memory idle; the form
// for very long rows has no registers left for that and asks the L2 for its next row instead (4096 rows of 8192, BF16:
// 100 us without, 90 with; the request costs the other form 1 to 4 us and gains it nothing).
// Measured (bytes of G, Gr, H, dX and its 8-bit copy): 8192 x 768 BF16 19.4 us with its second launch (57 MB, 2.9 TB/s: it waits
// for memory, 16 warps per SM without a row ahead, 0.35 instructions issued per scheduler and cycle, 3.3 of a warp's 10.4 cycles
// per instruction behind loads; 3.5 rows per warp make four rounds), 4099 x 5120 with an fp32 stream 57.8 us, 5.4 TB/s; 4099 x 5004
// 60.2 us; 4096 x 8192 BF16 90 us, 3.4 TB/s (one block of 16 warps per SM waits for its row's words from the L2, and reads gamma
// and Gr in the middle of the row: 765 MB of L2 traffic for 302 MB).
template <int GDT, int HDT, int VPT, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? (VPT == 2 ? kPrefetchThreads : kBlockThreads) : 32 * kBwdRows,
                                  BLOCK ? 1 : kBwdWarpBlocks) add_rmsnorm_bwd_kernel(const RmsNormBwdArgs a) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  extern __shared__ float s_dyn[];  // warp-per-row form: gamma [d], then [kBwdRows][d] to add up the block's warps
  __shared__ float s_red[32];
  __shared__ double s_stat[32];
  constexpr bool kPrefetch = BLOCK && VPT == 2;
  constexpr bool kLean = BLOCK && VPT == 4;  // very long rows: gamma and Gr are read where they are needed
  const int team = BLOCK ? blockDim.x : 32;
  const int lane = BLOCK ? threadIdx.x : threadIdx.x & 31;
  const int warp = threadIdx.x >> 5;
  const int64_t first = BLOCK ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * kBwdRows + warp;
  const int64_t stride = BLOCK ? gridDim.x : static_cast<int64_t>(gridDim.x) * kBwdRows;
  const float g_s = load_scale(a.g_scale), h_s = load_scale(a.h_scale), gam_s = a.gamma ? load_scale(a.gamma_scale) : 1.0f;
  const float branch_s = g_s * gam_s / h_s, res_s = a.Gr ? load_scale(a.gr_scale) : 0.f;
  const float dx_s = fmaxf(branch_s, res_s);
  const float fb = branch_s / dx_s, fr = res_s / dx_s;  // powers of two
  bool nonfinite = false;
  const float r_q = a.stat_in ? rescale_factor(__ldg(a.stat_in), &nonfinite) : 1.0f;
  const float inv_rq = 1.0f / r_q;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (a.dx_scale) *a.dx_scale = dx_s;
    if (a.dxq_scale) *a.dxq_scale = dx_s * r_q;
    if (a.dgamma_scale) *a.dgamma_scale = g_s * a.kf;
    if (a.status) {
      uint32_t bits = 0u;
      if (!(is_pow2_scale(g_s) && is_pow2_scale(h_s) && is_pow2_scale(gam_s) && (!a.Gr || is_pow2_scale(res_s))))
        bits |= SCALIFY_DEV_BAD_SCALE;
      if (nonfinite) bits |= SCALIFY_DEV_NONFINITE_STAT;
      if (bits) atomicOr(a.status, bits);
    }
  }
  const int n_vec = (a.d + kVec - 1) / kVec;
  constexpr int GW = kVec * ElemBytes<GDT>::v / 4, HW = kVec * ElemBytes<HDT>::v / 4;
  const float inv_d = 1.0f / static_cast<float>(a.d);
  float dg[VPT][kVec];
  float gam_reg[BLOCK && !kLean ? VPT : 1][kVec];  // a thread meets the same columns in every row
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int v = lane + i * team;
#pragma unroll
    for (int e = 0; e < kVec; ++e) dg[i][e] = 0.f;
    if constexpr (kLean) {
    } else if constexpr (BLOCK) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) gam_reg[i][e] = 0.f;
      if (v < n_vec) load_gamma(a.gamma, a.gamma_dt, v, a.d - v * kVec, gam_reg[i]);
    } else if (warp == 0 && v < n_vec) {
      load_gamma(a.gamma, a.gamma_dt, v, a.d - v * kVec, gam_reg[0]);
#pragma unroll
      for (int e = 0; e < kVec; e += 4)
        *reinterpret_cast<float4*>(s_dyn + v * kVec + e) = make_float4(gam_reg[0][e], gam_reg[0][e + 1], gam_reg[0][e + 2], gam_reg[0][e + 3]);
    }
  }
  if constexpr (!BLOCK) __syncthreads();
  auto gamma_of = [&](int i, int v, float* gam) {
    if constexpr (kLean) {
      load_gamma(a.gamma, a.gamma_dt, v, a.d - v * kVec, gam);
    } else if constexpr (BLOCK) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) gam[e] = gam_reg[i][e];
    } else {
#pragma unroll
      for (int e = 0; e < kVec; e += 4) {
        const float4 t = *reinterpret_cast<const float4*>(s_dyn + v * kVec + e);
        gam[e] = t.x; gam[e + 1] = t.y; gam[e + 2] = t.z; gam[e + 3] = t.w;
      }
    }
  };
  uint32_t amax = 0u;
  double ssq = 0.0;
  uint32_t wg[VPT][GW], wh[VPT][HW], wr[VPT][HW];
  float rinv = 0.f;
  // words of one row; vectors outside the row stay zero, so that they add nothing to any sum below
  auto load_row = [&](int64_t row, uint32_t (&xg)[VPT][GW], uint32_t (&xh)[VPT][HW], uint32_t (&xr)[VPT][HW], float& ri) {
    const char* grow = static_cast<const char*>(a.G) + row * a.g_ld * ElemBytes<GDT>::v;
    const char* hrow = static_cast<const char*>(a.H) + row * a.h_ld * ElemBytes<HDT>::v;
    const char* rrow = a.Gr ? static_cast<const char*>(a.Gr) + row * a.gr_ld * ElemBytes<HDT>::v : nullptr;
    ri = __ldg(a.rinv + row);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int v = lane + i * team;
      if (v < n_vec) {
        load_vec<GDT, true>(grow, v, a.d - v * kVec, xg[i]);
        load_vec<HDT, true>(hrow, v, a.d - v * kVec, xh[i]);
        if (rrow && !kLean) load_vec<HDT, true>(rrow, v, a.d - v * kVec, xr[i]);
      }
    }
  };
  auto prefetch_row = [&](int64_t row) {  // as far as the L2: one request per array
    if (lane < 3 && row < a.rows) {
      const char* p = lane == 0 ? static_cast<const char*>(a.G) + row * a.g_ld * ElemBytes<GDT>::v
                    : lane == 1 ? static_cast<const char*>(a.H) + row * a.h_ld * ElemBytes<HDT>::v
                                : static_cast<const char*>(a.Gr) + row * a.gr_ld * ElemBytes<HDT>::v;
      const uint32_t bytes = static_cast<uint32_t>(a.d * (lane == 0 ? ElemBytes<GDT>::v : ElemBytes<HDT>::v)) & ~15u;
      if (lane < 2 || a.Gr) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
    }
  };
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
#pragma unroll
    for (int q = 0; q < GW; ++q) wg[i][q] = 0u;
#pragma unroll
    for (int q = 0; q < HW; ++q) wh[i][q] = wr[i][q] = 0u;
  }
  if (kPrefetch && first < a.rows) load_row(first, wg, wh, wr, rinv);
  for (int64_t row = first; row < a.rows; row += stride) {
    if constexpr (kLean) prefetch_row(row + stride);
    uint32_t ng[VPT][GW], nh[VPT][HW], nr[VPT][HW];
    float nri = 0.f;
    if constexpr (kPrefetch) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
#pragma unroll
        for (int q = 0; q < GW; ++q) ng[i][q] = 0u;
#pragma unroll
        for (int q = 0; q < HW; ++q) nh[i][q] = nr[i][q] = 0u;
      }
      if (row + stride < a.rows) load_row(row + stride, ng, nh, nr, nri);
    } else {
      load_row(row, wg, wh, wr, rinv);
    }
    // Two elements per instruction (two-wide fp32): a row's arithmetic comes between its loads and the next row's.
    // dot = sum g gamma h;   dX = (G_s gamma_s/H_s/dX_s rinv) g gamma - (.. rinv^2 dot/d rinv) h + Gr (Gr_s/dX_s)
    float2 dot2 = make_float2(0.f, 0.f);
    const float2 rinv2 = make_float2(rinv, rinv);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int v = lane + i * team;
      if (v < n_vec) {
        float g[kVec], h[kVec];
        decode_vec<GDT, kVec>(wg[i], g);
        decode_vec<HDT, kVec>(wh[i], h);
        float gam[kVec];
        gamma_of(i, v, gam);
#pragma unroll
        for (int e = 0; e < kVec; e += 2) {
          const float2 g2 = make_float2(g[e], g[e + 1]), h2 = make_float2(h[e], h[e + 1]);
          const float2 d2 = __ffma2_rn(g2, __fmul2_rn(h2, rinv2), make_float2(dg[i][e], dg[i][e + 1]));
          dg[i][e] = d2.x;
          dg[i][e + 1] = d2.y;
          const float2 t2 = __fmul2_rn(g2, make_float2(gam[e], gam[e + 1]));
          dot2 = __ffma2_rn(t2, h2, dot2);
        }
      }
    }
    const float dot = team_sum<BLOCK>(dot2.x + dot2.y, s_red) * inv_d;  // mean of g gamma h
    const float cg = rinv * fb, ch = -cg * rinv * (rinv * dot);
    const float2 cg2 = make_float2(cg, cg), ch2 = make_float2(ch, ch), fr2 = make_float2(fr, fr), iq2 = make_float2(inv_rq, inv_rq);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int v = lane + i * team;
      if (v < n_vec) {
        const int n = a.d - v * kVec;
        float g[kVec], h[kVec], gam[kVec], x[kVec];
        decode_vec<GDT, kVec>(wg[i], g);
        decode_vec<HDT, kVec>(wh[i], h);
        gamma_of(i, v, gam);
        if (a.Gr) {
          if constexpr (kLean) load_vec<HDT, true>(static_cast<const char*>(a.Gr) + row * a.gr_ld * ElemBytes<HDT>::v, v, n, wr[0]);
          decode_vec<HDT, kVec>(wr[kLean ? 0 : i], x);
        }
#pragma unroll
        for (int e = 0; e < kVec; e += 2) {
          float2 x2 = a.Gr ? __fmul2_rn(make_float2(x[e], x[e + 1]), fr2) : make_float2(0.f, 0.f);
          x2 = __ffma2_rn(make_float2(h[e], h[e + 1]), ch2, x2);
          x2 = __ffma2_rn(__fmul2_rn(make_float2(g[e], g[e + 1]), make_float2(gam[e], gam[e + 1])), cg2, x2);
          x[e] = x2.x;
          x[e + 1] = x2.y;
        }
        uint32_t ow[HW];
        encode_vec<HDT, kVec>(x, ow);
        char* xrow = static_cast<char*>(a.dX) + row * a.dx_ld * ElemBytes<HDT>::v;
        if (n >= kVec) st_bytes<kVec * ElemBytes<HDT>::v>(xrow + static_cast<int64_t>(v) * (kVec * ElemBytes<HDT>::v), ow);
        else store_vec<HDT>(xrow, v, n, x);
        if (a.stat == SCALIFY_STAT_AMAX) amax = max_bits<HDT>(ow, amax);
        if (a.dXq || a.stat == SCALIFY_STAT_L2) {
          decode_vec<HDT, kVec>(ow, x);  // the stored values
          if (a.stat == SCALIFY_STAT_L2) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) ssq += static_cast<double>(x[e]) * x[e];
          }
          if (a.dXq) {
#pragma unroll
            for (int e = 0; e < kVec; e += 2) {
              const float2 x2 = __fmul2_rn(make_float2(x[e], x[e + 1]), iq2);
              x[e] = x2.x;
              x[e + 1] = x2.y;
            }
            char* qrow = static_cast<char*>(a.dXq) + row * a.dxq_ld;
            if (a.dxq_dt == SCALIFY_E4M3) store_vec<SCALIFY_E4M3>(qrow, v, n, x);
            else store_vec<SCALIFY_E5M2>(qrow, v, n, x);
          }
        }
      }
    }
    if constexpr (kPrefetch) {
      rinv = nri;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
#pragma unroll
        for (int q = 0; q < GW; ++q) wg[i][q] = ng[i][q];
#pragma unroll
        for (int q = 0; q < HW; ++q) { wh[i][q] = nh[i][q]; wr[i][q] = nr[i][q]; }
      }
    }
  }
  if (a.partial) {
    float* line = a.partial + static_cast<int64_t>(blockIdx.x) * a.partial_ld;
    if constexpr (BLOCK) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * team;
        if (v < n_vec) {
          uint32_t w[kVec];
          encode_vec<SCALIFY_F32, kVec>(dg[i], w);
          st_raw<32>(line + v * kVec, w);  // (the line is padded to whole vectors)
        }
      }
    } else {
      const int ld = n_vec * kVec;
      float* s_lines = s_dyn + ld;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * team;
        if (v < n_vec) {
#pragma unroll
          for (int e = 0; e < kVec; e += 4)
            *reinterpret_cast<float4*>(s_lines + warp * ld + v * kVec + e) = make_float4(dg[i][e], dg[i][e + 1], dg[i][e + 2], dg[i][e + 3]);
        }
      }
      __syncthreads();
      for (int c = threadIdx.x; c < ld; c += blockDim.x) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < kBwdRows; ++k) t += s_lines[k * ld + c];
        line[c] = t;
      }
    }
  }
  if (a.stat != SCALIFY_STAT_NONE) {
    const double mine = a.stat == SCALIFY_STAT_AMAX ? static_cast<double>(warp_max_u32(max_bits_to_f32<HDT>(amax))) : warp_sum_f64(ssq);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s_stat[warp] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
      double t = 0.0;
      for (int k = 0; k < static_cast<int>(blockDim.x >> 5); ++k) t = a.stat == SCALIFY_STAT_AMAX ? fmax(t, s_stat[k]) : t + s_stat[k];
      a.stat_partial[blockIdx.x] = t;
    }
  }
}

// Adds the blocks' lines in block order: a block takes 32 columns, each of its 32 warps every 32nd line (a handful of
// loads, all in flight together); the last block of the grid reduces the statistic instead.
constexpr int kFinishThreads = 1024;
template <int ODT>
__global__ void __launch_bounds__(kFinishThreads) add_rmsnorm_bwd_finish_kernel(
    const float* __restrict__ partial, int64_t ld, int lines, int d, void* __restrict__ dgamma, float inv_kf,
    const double* __restrict__ stat_partial, int stat, double count, float* stat_word) {
  asm volatile("griddepcontrol.launch_dependents;");  // a programmatic dependent may set up while this grid runs
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched as a programmatic dependent: the gradient is complete
  __shared__ double s[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (stat != SCALIFY_STAT_NONE && blockIdx.x == gridDim.x - 1) {
    double t = 0.0;
    for (int i = threadIdx.x; i < lines; i += kFinishThreads) t = stat == SCALIFY_STAT_AMAX ? fmax(t, __ldcg(stat_partial + i)) : t + __ldcg(stat_partial + i);
    t = stat == SCALIFY_STAT_AMAX ? static_cast<double>(warp_max_u32(static_cast<uint32_t>(t))) : warp_sum_f64(t);
    if (lane == 0) s[0][warp] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
      t = 0.0;
      for (int k = 0; k < 32; ++k) t = stat == SCALIFY_STAT_AMAX ? fmax(t, s[0][k]) : t + s[0][k];
      *stat_word = stat == SCALIFY_STAT_AMAX ? __uint_as_float(static_cast<uint32_t>(t)) : static_cast<float>(sqrt(t / count));
    }
    return;
  }
  const int col = blockIdx.x * 32 + lane;
  double t = 0.0;
  if (col < d) {
    for (int i = warp; i < lines; i += 32 * 10) {
      float p[10];
#pragma unroll
      for (int u = 0; u < 10; ++u) p[u] = i + 32 * u < lines ? __ldcg(partial + static_cast<int64_t>(i + 32 * u) * ld + col) : 0.f;
#pragma unroll
      for (int u = 0; u < 10; ++u) t += p[u];
    }
  }
  s[warp][lane] = t;
  __syncthreads();
  t = warp_sum_f64(s[lane][warp]);  // warp w adds up column w of the block's 32
  if (lane == 0 && blockIdx.x * 32 + warp < d) store_elem<ODT>(dgamma, blockIdx.x * 32 + warp, static_cast<float>(t) * inv_kf);
}

// ------------------------------------------------------------------------------------------------- launches
// backward: 2 vectors per thread while the row fits the threads of the prefetching form; forward: while it fits 512
static int block_vpt(int d, bool bwd) { return (d + kVec - 1) / kVec <= 2 * (bwd ? kPrefetchThreads : kBlockThreads) ? 2 : 4; }
static int block_threads(int d, bool bwd) {
  const int n_vec = (d + kVec - 1) / kVec, vpt = block_vpt(d, bwd);
  return ((n_vec + vpt - 1) / vpt + 31) / 32 * 32;
}
static int bwd_grid_cap(int d) {  // resident blocks, by the register budgets above
  if (d <= kWarpMaxD) return sm_count() * kBwdWarpBlocks;
  const int per_sm = (block_vpt(d, true) == 2 ? kPrefetchThreads : kBlockThreads) / block_threads(d, true);
  return sm_count() * (per_sm < 1 ? 1 : per_sm);
}
size_t rmsnorm_bwd_ws_bytes(int64_t rows, int64_t d) {
  if (d < 1 || d > kRmsNormMaxD) return kWsMin;
  const size_t cap = static_cast<size_t>(bwd_grid_cap(static_cast<int>(d)));
  return kWsHeader + cap * (static_cast<size_t>((d + kVec - 1) / kVec * kVec) * sizeof(float) + sizeof(double)) + 256;
}

#define SCALIFY_RMS_VPT(X, H, KERNEL, ...)                                  \
  do {                                                                      \
    if (block && vpt == 2) KERNEL<X, H, 2, true><<<grid, threads, smem, st>>>(__VA_ARGS__); \
    else if (block) KERNEL<X, H, 4, true><<<grid, threads, smem, st>>>(__VA_ARGS__);        \
    else if (n_vec <= 32) KERNEL<X, H, 1, false><<<grid, threads, smem, st>>>(__VA_ARGS__); \
    else if (n_vec <= 64) KERNEL<X, H, 2, false><<<grid, threads, smem, st>>>(__VA_ARGS__); \
    else KERNEL<X, H, 3, false><<<grid, threads, smem, st>>>(__VA_ARGS__);                  \
  } while (0)
#define SCALIFY_RMS_TYPES(xdt, hdt, KERNEL, ...)                                                                 \
  do {                                                                                                           \
    if (hdt == SCALIFY_F32) {                                                                                    \
      if (xdt == SCALIFY_BF16) SCALIFY_RMS_VPT(SCALIFY_BF16, SCALIFY_F32, KERNEL, __VA_ARGS__);                  \
      else if (xdt == SCALIFY_F16) SCALIFY_RMS_VPT(SCALIFY_F16, SCALIFY_F32, KERNEL, __VA_ARGS__);               \
      else SCALIFY_RMS_VPT(SCALIFY_F32, SCALIFY_F32, KERNEL, __VA_ARGS__);                                       \
    } else if (hdt == SCALIFY_BF16) SCALIFY_RMS_VPT(SCALIFY_BF16, SCALIFY_BF16, KERNEL, __VA_ARGS__);            \
    else SCALIFY_RMS_VPT(SCALIFY_F16, SCALIFY_F16, KERNEL, __VA_ARGS__);                                         \
  } while (0)

int launch_add_rmsnorm(const RmsNormArgs& a, int x_dt, int h_dt, cudaStream_t st) {
  const bool block = a.d > kWarpMaxD;
  const int n_vec = (a.d + kVec - 1) / kVec;
  const int64_t rows = a.sf ? (a.rows + 255) / 256 * 256 : a.rows > 0 ? a.rows : 1;  // (no rows: the scale words alone are written)
  const int threads = block ? block_threads(a.d, false) : 32 * kWarpRows, vpt = block_vpt(a.d, false);
  const unsigned grid = static_cast<unsigned>(block ? rows : (rows + kWarpRows - 1) / kWarpRows);
  const size_t smem = 0;
  SCALIFY_RMS_TYPES(x_dt, h_dt, add_rmsnorm_kernel, a);
  SCALIFY_CUDA_TRY(cudaGetLastError());
  return SCALIFY_OK;
}

int launch_add_rmsnorm_bwd(RmsNormBwdArgs a, int g_dt, int h_dt, void* dgamma, int dgamma_dt, void* ws, cudaStream_t st) {
  const bool block = a.d > kWarpMaxD;
  const int n_vec = (a.d + kVec - 1) / kVec;
  const int threads = block ? block_threads(a.d, true) : 32 * kBwdRows, vpt = block_vpt(a.d, true);
  const int64_t want = block ? a.rows : (a.rows + kBwdRows - 1) / kBwdRows;
  const int cap = bwd_grid_cap(a.d);
  const unsigned grid = static_cast<unsigned>(want < cap ? want : cap);
  const size_t smem = block ? 0 : static_cast<size_t>(dgamma ? 1 + kBwdRows : 1) * n_vec * kVec * sizeof(float);
  a.partial = nullptr;
  a.stat_partial = nullptr;
  float* stat_word = nullptr;
  a.partial_ld = static_cast<int64_t>(n_vec) * kVec;
  if (ws) {
    WsView v = ws_view(ws);
    a.status = v.status;
    stat_word = v.stat;
    if (dgamma) a.partial = static_cast<float*>(v.area);
    a.stat_partial = reinterpret_cast<double*>(static_cast<float*>(v.area) + static_cast<int64_t>(cap) * a.partial_ld);
  }
  SCALIFY_RMS_TYPES(g_dt, h_dt, add_rmsnorm_bwd_kernel, a);
  SCALIFY_CUDA_TRY(cudaGetLastError());
  if (!dgamma && a.stat == SCALIFY_STAT_NONE) return SCALIFY_OK;
  const unsigned blocks = (dgamma ? (a.d + 31) / 32 : 0) + (a.stat != SCALIFY_STAT_NONE ? 1 : 0);
  const double count = static_cast<double>(a.rows) * a.d;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(blocks); cfg.blockDim = dim3(kFinishThreads); cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = 1;
  const float* partial = a.partial;
  const double* stats = a.stat_partial;
  SCALIFY_DISPATCH_WIDE(dgamma_dt, ODT, SCALIFY_CUDA_TRY(cudaLaunchKernelEx(&cfg, add_rmsnorm_bwd_finish_kernel<ODT>, partial, a.partial_ld,
                                            static_cast<int>(grid), dgamma ? a.d : 0, dgamma, 1.0f / a.kf, stats, a.stat, count, stat_word)))
  return SCALIFY_OK;
}

}  // namespace scalify
