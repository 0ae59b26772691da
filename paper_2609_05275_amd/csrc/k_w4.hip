// Projections by weights in 4 bits, for the few rows of a decoding step, and what
// makes such weights.  Layout: W4View in ld_w4.h, ld_w4 in layerdrop.h.
//
// Codes become bf16 exactly: a 4-bit float by one conversion that takes its
// power-of-two scale along, an integer of sign and three bits as an 8-bit float below
// its smallest normal number (steps of 2^-9), times 2^9.  The integers' scales go on
// the float32 sums of a group's products.
#include "ld_w4.h"

namespace ld {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));
typedef unsigned short ushortx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;

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
  static constexpr int kBytes = kPer * (FMT == LD_W4_E2M1 ? 1 : 2);
};

// ---------------------------------------------------------- pack and load

// A wave takes a block of 8 rows and 256 k; lanes and dwords as the codes lie, so
// that a group's values are in lanes 16 apart and in neighbouring dwords.
template <int FMT, int GROUP>
__global__ __launch_bounds__(256) void ld_w4_pack_k(W4PackArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int C = (a.w.K + kW4Chunk - 1) / kW4Chunk, c = blockIdx.x * 4 + wave;
  if (c >= C) return;
  const int r = lane & 7, h = (lane >> 3) & 1, g = lane >> 4;
  for (int64_t t = blockIdx.y; t * kW4Rows < a.w.N; t += gridDim.y) {
    const int64_t n = t * kW4Rows + r;
    const int k0 = c * kW4Chunk + 128 * h + 8 * g;
    Oct v[4];
    uint32_t amax[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      v[s].v = static_cast<bf16>(0.f);
      if (n < a.w.N && k0 + 32 * s < a.w.K)
        v[s].v = *reinterpret_cast<const bf16x8*>(static_cast<const bf16*>(a.src) + n * a.ld + k0 + 32 * s);
      ushortx2 m2{0, 0};
#pragma unroll
      for (int e = 0; e < 4; ++e) m2 = __builtin_elementwise_max(m2, v[s].u[e] & static_cast<unsigned short>(0x7fff));
      uint32_t m = max(m2[0], m2[1]);
      m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16, 64)));
      amax[s] = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32, 64)));
    }
    const int64_t block = t * C + c;
    u32x4 out;
    if constexpr (FMT == LD_W4_E2M1) {
      uint32_t sc = 0;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        // the smallest 2^e that 6 of hold the largest, 6 = 1.5 2^2
        const int e = static_cast<int>(amax[s] >> 7) - 127 - 2 + ((amax[s] & 0x7fu) > 0x40u ? 1 : 0);
        const uint32_t sb = amax[s] >= 0x7f80u ? 255u : static_cast<uint32_t>(min(max(e, kW4MinExp), 125) + 127);
        const float scale = __builtin_bit_cast(float, sb << 23);
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, v[s].p[0], scale, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, v[s].p[1], scale, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, v[s].p[2], scale, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, v[s].p[3], scale, 3);
        out[s] = sb == 255u ? 0u : q;
        sc |= sb << (8 * s);
      }
      if (g == 0) reinterpret_cast<uint32_t*>(a.w.scales)[block * 16 + lane] = sc;
    } else {
      constexpr int kPer = W4Scales<FMT, GROUP>::kPer, kSteps = GROUP / 32;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        uint32_t m = 0;
#pragma unroll
        for (int s = i * kSteps; s < (i + 1) * kSteps; ++s) m = max(m, amax[s]);
        const float top = __builtin_bit_cast(float, m << 16);
        bf16 sc = static_cast<bf16>(fmaxf(top / 7.f, 0x1p-100f));
        const bool bad = m >= 0x7f80u;
        if (bad) sc = static_cast<bf16>(__builtin_nanf(""));
        const float sf = static_cast<float>(sc);
#pragma unroll
        for (int s = i * kSteps; s < (i + 1) * kSteps; ++s) {
          uint32_t q = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            // (the quotient of two numbers of 8 bits is no nearer than 2^-13 to a tie that it is not)
            const float x = bad ? 0.f : fminf(fmaxf(__builtin_rintf(static_cast<float>(v[s].v[e]) / sf), -7.f), 7.f);
            const uint32_t mag = static_cast<uint32_t>(fabsf(x)), neg = x < 0.f;
            const int b = e & 3;
            q |= e < 4 ? mag << (8 * b) | neg << (8 * b + 7) : mag << (8 * b + 4) | neg << ((8 * b + 11) & 31);
          }
          out[s] = q;
        }
        if (g == 0) static_cast<bf16*>(a.w.scales)[(block * 16 + lane) * kPer + i] = sc;
      }
    }
    reinterpret_cast<u32x4*>(a.w.codes)[block * 64 + lane] = out;
  }
}

template <int FMT, int GROUP>
__global__ __launch_bounds__(256) void ld_w4_load_k(W4PackArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int C = (a.w.K + kW4Chunk - 1) / kW4Chunk, c = blockIdx.x * 4 + wave;
  if (c >= C) return;
  const int r = lane & 7, h = (lane >> 3) & 1, g = lane >> 4;
  for (int64_t t = blockIdx.y; t * kW4Rows < a.w.N; t += gridDim.y) {
    const int64_t n = t * kW4Rows + r, block = t * C + c;
    const int k0 = c * kW4Chunk + 128 * h + 8 * g;
    if (n >= a.w.N) continue;
    const u32x4 q = reinterpret_cast<const u32x4*>(a.w.codes)[block * 64 + lane];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (k0 + 32 * s >= a.w.K) continue;
      bf16x8 v;
      if constexpr (FMT == LD_W4_E2M1) {
        const uint32_t sc = static_cast<const uint8_t*>(a.w.scales)[(block * 16 + (lane & 15)) * 4 + s];
        v = codes_to_bf16<FMT>(q[s], scale_byte(sc, 0));
      } else {
        constexpr int kPer = W4Scales<FMT, GROUP>::kPer;
        const float sc = static_cast<float>(static_cast<const bf16*>(a.w.scales)[(block * 16 + (lane & 15)) * kPer + s * 32 / GROUP]);
        v = codes_to_bf16<FMT>(q[s], 1.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = static_cast<bf16>(static_cast<float>(v[e]) * sc);
      }
      *reinterpret_cast<bf16x8*>(static_cast<bf16*>(a.dst) + n * a.ld + k0 + 32 * s) = v;
    }
  }
}

// ------------------------------------------------------------- projections

__device__ __forceinline__ bf16x8 load8(const bf16* p) { return *reinterpret_cast<const bf16x8*>(p); }

// Element (m, n) from its sums (SwiGLU: of the gate and the up row).
__device__ __forceinline__ void w4_finish(const W4GemmArgs& a, int m, int64_t n, float s0, float s1, float scale) {
  float y;
  if (a.act == kDecActSwiglu) {
    y = swiglu_fwd_f(scale * s0, scale * s1);
  } else if (a.act == kDecActRelu2) {
    const float z = fmaxf(scale * s0, 0.f);
    y = z * z;
  } else {
    y = scale * s0;
    if (a.R) y += static_cast<float>(static_cast<const bf16*>(a.R)[m * a.ldr + n]);
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

// A workgroup takes 8 columns of C (of W 8 rows; SwiGLU: 8 gate and 8 up rows), its
// waves every eighth chunk of 256 k.  As operands of a 16x16x32 product the rows of A
// stand twice, with the first and the last 128 k of the chunk, and so do the weights: the
// product's two diagonal 8x8 blocks are added, the others, which mix the halves, dropped.
template <int FMT, int GROUP, int MB, int NR, bool NORM>
__global__ __launch_bounds__(64 * kWaves) void ld_gemm_w4_k(W4GemmArgs a) {
  typedef typename W4ScaleRaw<FMT, GROUP>::type SRaw;
  constexpr int kWave = NR * MB * 64;
  __shared__ __align__(16) float red[kWaves * kWave];
  __shared__ float ssq[NORM ? kWaves : 1][MB * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = a.w.K, M = a.M, C = (K + kW4Chunk - 1) / kW4Chunk;
  const int r = lane & 7, lk = 128 * ((lane >> 3) & 1) + 8 * (lane >> 4);
  const int64_t tile = blockIdx.x, up = a.N / kW4Rows;
  const bf16* xr[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) xr[mb] = static_cast<const bf16*>(a.A) + static_cast<int64_t>(min(mb * 8 + r, M - 1)) * a.lda;
  floatx4 acc[NR][MB], q2[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
    for (int j = 0; j < NR; ++j) acc[j][mb] = floatx4{0.f, 0.f, 0.f, 0.f};
    q2[mb] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  for (int c = wave; c < C; c += kWaves) {
    u32x4 q[NR];
    SRaw sc[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      const int64_t block = (tile + j * up) * C + c;
      q[j] = reinterpret_cast<const u32x4*>(a.w.codes)[block * 64 + lane];
      sc[j] = static_cast<const SRaw*>(a.w.scales)[block * 16 + (lane & 15)];
    }
    floatx4 part[NR][MB];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int k = c * kW4Chunk + 32 * s + lk;
      const bool in = k < K;
      bf16x8 x[MB], xl[MB];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        x[mb] = load8(xr[mb] + (in ? k : 0));
        if (!in) x[mb] = static_cast<bf16>(0.f);
      }
      if constexpr (NORM) {
        const bf16x8 gv = load8(static_cast<const bf16*>(a.g) + (in ? k : 0));
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          q2[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[mb], x[mb], q2[mb], 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 8; ++e) {  // a product of 16 bits, in two parts
            const float y = static_cast<float>(x[mb][e]) * static_cast<float>(gv[e]);
            x[mb][e] = static_cast<bf16>(y);
            xl[mb][e] = static_cast<bf16>(y - static_cast<float>(x[mb][e]));
          }
          if (!in) x[mb] = xl[mb] = static_cast<bf16>(0.f);
        }
      }
#pragma unroll
      for (int j = 0; j < NR; ++j) w4_step<FMT, GROUP, MB, NORM>(s, q[j][s], sc[j], x, xl, acc[j], part[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < NR; ++j)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      floatx4 v = acc[j][mb];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] += __shfl_xor(v[e], 40, 64);
        if ((lane & 40) == 0) red[wave * kWave + ((j * MB + mb) * 8 + 4 * (lane >> 4) + e) * 8 + r] = v[e];
      }
    }
  if constexpr (NORM) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      // lane l: rows 4 (l / 16) + e of column l % 16
      const int e = lane & 3;
      float ss = e == 0 ? q2[mb][0] : e == 1 ? q2[mb][1] : e == 2 ? q2[mb][2] : q2[mb][3];
      ss += __shfl_xor(ss, 40, 64);
      if ((lane & 40) == 0 && (lane & 15) >> 2 == lane >> 4) ssq[wave][mb * 8 + r] = ss;
    }
  }
  __syncthreads();
  const int m = tid >> 3;
  const int64_t n = tile * kW4Rows + (tid & 7);
  if (m >= M || m >= MB * 8 || n >= a.N) return;
  float s0 = 0.f, s1 = 0.f, scale = a.alpha;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    s0 += red[w * kWave + tid];
    if constexpr (NR == 2) s1 += red[w * kWave + MB * 64 + tid];
  }
  if constexpr (NORM) {
    float tot = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) tot += ssq[w][m];
    scale *= rsqrtf(tot / static_cast<float>(K) + a.eps);
  }
  w4_finish(a, m, n, s0, s1, scale);
}

template <int FMT, int GROUP, int MB, int NR, bool NORM>
hipError_t gemm_launch(const W4GemmArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((ld_gemm_w4_k<FMT, GROUP, MB, NR, NORM>), dim3((a.N + kW4Rows - 1) / kW4Rows), dim3(64 * kWaves), 0, s, a);
  return hipGetLastError();
}

template <int FMT, int GROUP, int MB>
hipError_t gemm_mb(const W4GemmArgs& a, hipStream_t s) {
  if constexpr (MB <= 2)
    if (a.g) return a.act == kDecActSwiglu ? gemm_launch<FMT, GROUP, MB, 2, true>(a, s) : gemm_launch<FMT, GROUP, MB, 1, true>(a, s);
  if (a.g) return hipErrorInvalidValue;
  return a.act == kDecActSwiglu ? gemm_launch<FMT, GROUP, MB, 2, false>(a, s) : gemm_launch<FMT, GROUP, MB, 1, false>(a, s);
}

template <int FMT, int GROUP>
hipError_t gemm_t(const W4GemmArgs& a, hipStream_t s) {
  if (a.M < 1 || a.M > kW4MaxM) return hipErrorInvalidValue;
  return a.M <= 8 ? gemm_mb<FMT, GROUP, 1>(a, s) : a.M <= 16 ? gemm_mb<FMT, GROUP, 2>(a, s)
       : a.M <= 32 ? gemm_mb<FMT, GROUP, 4>(a, s) : gemm_mb<FMT, GROUP, 8>(a, s);
}

template <int FMT, int GROUP>
hipError_t pack_t(const W4PackArgs& a, hipStream_t s) {
  const int C = (a.w.K + kW4Chunk - 1) / kW4Chunk, T = (a.w.N + kW4Rows - 1) / kW4Rows;
  const dim3 grid((C + 3) / 4, T < 65535 ? T : 65535);
  if (a.src)
    hipLaunchKernelGGL((ld_w4_pack_k<FMT, GROUP>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((ld_w4_load_k<FMT, GROUP>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t pack_or_load(const W4PackArgs& a, hipStream_t s) {
  if (a.w.format == LD_W4_E2M1) return pack_t<LD_W4_E2M1, 32>(a, s);
  return a.w.group == 32 ? pack_t<LD_W4_INT4, 32>(a, s) : a.w.group == 64 ? pack_t<LD_W4_INT4, 64>(a, s)
                                                        : pack_t<LD_W4_INT4, 128>(a, s);
}

}  // namespace

hipError_t launch_w4_pack(const W4PackArgs& a, hipStream_t s) { return pack_or_load(a, s); }
hipError_t launch_w4_load(const W4PackArgs& a, hipStream_t s) { return pack_or_load(a, s); }

// Rows and K whose norm a projection can take in.
bool w4_gemm_fuses_norm(int64_t M, int64_t K) { return M <= 16 && K <= 8192; }

size_t w4_gemm_ws_bytes(int64_t, int64_t, int64_t, int) { return 0; }

hipError_t launch_gemm_w4(const W4GemmArgs& a, hipStream_t s) {
  if (a.w.format == LD_W4_E2M1) return gemm_t<LD_W4_E2M1, 32>(a, s);
  return a.w.group == 32 ? gemm_t<LD_W4_INT4, 32>(a, s) : a.w.group == 64 ? gemm_t<LD_W4_INT4, 64>(a, s)
                                                        : gemm_t<LD_W4_INT4, 128>(a, s);
}

}  // namespace ld
