// 4-bit weights on the device: codes to bf16, a step of products, an output's end.
// Shared by the projections of few rows (k_w4.hip) and of more (k_w4_rows.hip).
#pragma once
#include "ld_w4.h"

namespace ld {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;  // of a workgroup
constexpr int kCus = 256;

// A launch takes fewer than 2^32 threads, and 2^30 rows of weights may need more: launches of
// 2^17 workgroups, one but for a million columns and more.  (The number in two dimensions, with a
// test for those past the last: one row, 4096 x 11008, 6.2 -> 6.4 us.)
constexpr int64_t kW4Wgs = 1 << 17;
template <class F>
hipError_t w4_launches(W4GemmArgs a, int64_t wgs, F launch) {
  for (int64_t first = 0; first < wgs; first += kW4Wgs) {
    a.wg0 = static_cast<int32_t>(first);
    launch(a, dim3(static_cast<uint32_t>(wgs - first < kW4Wgs ? wgs - first : kW4Wgs)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------- conversions

// The scale in byte B of w as the conversions take it: they look at a float's
// exponent alone.
__device__ __forceinline__ float scale_byte(uint32_t w, int b) {
  return __builtin_bit_cast(float, b == 0 ? w << 23 : b == 1 ? w << 15 : b == 2 ? w << 7 : w >> 1);
}

union Oct {
  bf16x8 v;
  bf16x2 p[4];
  ushortx2 u[4];
};

// Eight codes of a dword; scale: of 4-bit floats.
template <int FMT>
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t w, float scale) {
  Oct r;
  if constexpr (FMT == LD_W4_E2M1) {
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  } else {
    const uint32_t a = w & 0x87878787u, b = __builtin_amdgcn_alignbit(w, w, 4) & 0x87878787u;
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 512.f, false);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 512.f, true);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 512.f, false);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 512.f, true);
  }
  return r.v;
}

template <int FMT, int GROUP>
struct W4Scales {
  static constexpr int kPer = 128 / GROUP;                           // of a lane's row in half a chunk
};

// ------------------------------------------------------------- projections

__device__ __forceinline__ bf16x8 load8(const bf16* p) { return *reinterpret_cast<const bf16x8*>(p); }

// Zeroes what was loaded from a clamped address.
__device__ __forceinline__ void keep_if(bf16x8& v, bool keep) {
  u32x4 t = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = keep ? t[i] : 0u;
  v = __builtin_bit_cast(bf16x8, t);
}

// Element (m, n) from its sums (SwiGLU: of the gate and the up row).
__device__ __forceinline__ void w4_finish(const W4GemmArgs& a, int m, int64_t n, float s0, float s1, float scale, uint16_t resid) {
  float y;
  if (a.act == kDecActSwiglu) {
    y = swiglu_fwd_f(scale * s0, scale * s1);
  } else if (a.act == kDecActRelu2) {
    const float z = scale * s0;
    y = z < 0.f ? 0.f : z * z;  // (of NaN NaN; a maximum with 0 would drop it)
  } else {
    y = scale * s0;
    if (a.R) y += static_cast<float>(__builtin_bit_cast(bf16, resid));
  }
  static_cast<bf16*>(a.C)[m * a.ldc + n] = static_cast<bf16>(y);
}

// Scales of a lane's row in half a chunk.
template <int FMT, int GROUP>
struct W4ScaleRaw {
  typedef uint32_t type;  // four bytes, or two bf16
};
template <>
struct W4ScaleRaw<LD_W4_INT4, 32> {
  typedef uint64_t type;
};
template <>
struct W4ScaleRaw<LD_W4_INT4, 128> {
  typedef uint16_t type;
};

// acc[mb] += x[mb] (+ xl[mb], where there are low parts) times step s of the codes.
// INT4: sums of a group in `part`, which go to acc times their scale at its end.
template <int FMT, int GROUP, int MB, bool LOW>
__device__ __forceinline__ void w4_step(int s, uint32_t q, typename W4ScaleRaw<FMT, GROUP>::type sc, const bf16x8 (&x)[MB],
                                        const bf16x8 (&xl)[MB], floatx4 (&acc)[MB], floatx4 (&part)[MB]) {
  if constexpr (FMT == LD_W4_E2M1) {
    const bf16x8 w = codes_to_bf16<FMT>(q, scale_byte(sc, s));
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      acc[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[mb], w, acc[mb], 0, 0, 0);
      if constexpr (LOW) acc[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xl[mb], w, acc[mb], 0, 0, 0);
    }
  } else {
    constexpr int kSteps = GROUP / 32;
    const bf16x8 w = codes_to_bf16<FMT>(q, 1.f);
    const floatx4 zero{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      part[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[mb], w, s % kSteps ? part[mb] : zero, 0, 0, 0);
      if constexpr (LOW) part[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xl[mb], w, part[mb], 0, 0, 0);
    }
    if (s % kSteps == kSteps - 1) {
      const float f = __builtin_bit_cast(float, static_cast<uint32_t>(static_cast<uint64_t>(sc) >> (s / kSteps * 16)) << 16);
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mb][e] = __builtin_fmaf(part[mb][e], f, acc[mb][e]);
    }
  }
}

// The steps 2 p and 2 p + 1 of half a chunk's codes, integers' sums scaled once for groups
// of 64 and more.
template <int FMT, int GROUP, int MB>
__device__ __forceinline__ void w4_pair(int p, const u32x4& q, typename W4ScaleRaw<FMT, GROUP>::type sc,
                                        const bf16x8 (&x)[2][MB], floatx4 (&acc)[MB]) {
  if constexpr (FMT == LD_W4_E2M1) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const bf16x8 w = codes_to_bf16<FMT>(q[2 * p + s], scale_byte(sc, 2 * p + s));
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) acc[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[s][mb], w, acc[mb], 0, 0, 0);
    }
  } else {
    constexpr int kSums = GROUP == 32 ? 2 : 1;
    const floatx4 zero{0.f, 0.f, 0.f, 0.f};
    floatx4 part[MB];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const bf16x8 w = codes_to_bf16<FMT>(q[2 * p + s], 1.f);
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
        part[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[s][mb], w, s % (2 / kSums) ? part[mb] : zero, 0, 0, 0);
      if (s == 0 && kSums == 1) continue;
      const int at = GROUP == 32 ? 2 * p + s : GROUP == 64 ? p : 0;
      const float f = __builtin_bit_cast(float, static_cast<uint32_t>(static_cast<uint64_t>(sc) >> (16 * at)) << 16);
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[mb][e] = __builtin_fmaf(part[mb][e], f, acc[mb][e]);
    }
  }
}

}  // namespace
}  // namespace ld
