// Projections by weights in 4 bits, for the few rows of a decoding step, and what
// makes such weights.  Layout: W4View in ld_w4.h, ld_w4 in layerdrop.h.
//
// Codes become bf16 exactly: a 4-bit float by one conversion that takes its
// power-of-two scale along, an integer of sign and three bits as an 8-bit float below
// its smallest normal number (steps of 2^-9), times 2^9.  The integers' scales go on
// the float32 sums of a group's products.
#include "w4_codes.h"

namespace ld {
namespace {

// ---------------------------------------------------------- pack and load

// A wave takes a block of 8 rows and 256 k; lanes and dwords as the codes lie, so
// that a group's values are in lanes 16 apart and in neighbouring dwords.  Done once for
// weights that are kept.  22016 x 4096, 225 MB: e2m1 49 us, 4.6 TB/s; int4 62 to 66, a division
// an element; read back 55 to 59, rows written in pieces of 64 bytes.
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

// The chunks' numbers go round the waves, and neighbouring workgroups of an XCD (every
// 8th) count from different waves, so that they do not all ask for the same lines of A
// first.  Sums go by this number: the results do not depend on it.
__device__ __forceinline__ int w4_wave() {
  return __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) + (blockIdx.x >> 3)) & (kWaves - 1);
}

// Up to 8 MB rows of up to 256 kWaves CPW: every wave holds its chunks of the rows in
// registers, as operands, for all the tiles that its workgroup takes.  A tile is 8 columns of
// C (of W 8 rows; SwiGLU: 8 gate and 8 up rows); T of them are asked for, multiplied and
// summed over the waves together, with one barrier, the next T's codes on their way.
// As operands of a 16x16x32 product the rows of A stand twice, with the first and the
// last 128 k of a chunk, and so do the weights: the product's two diagonal 8x8 blocks
// are added, the others, which mix the halves, dropped.
//
// What bounds it: up to 2048 k and a few hundred tiles the launch, one trip to memory and the
// sums (qkv of one row, 2304 x 768: 4.0 us in a graph; gate and up of 8 rows, 5504 x 2048, with
// the norm: 6.8); over more columns the codes (one row, 24000 x 4096: 13.7 us, 3.6 TB/s).
template <int FMT, int GROUP, int MB, int NR, bool NORM, int CPW>
__global__ __launch_bounds__(64 * kWaves) void ld_gemm_w4_k(W4GemmArgs a) {
  typedef typename W4ScaleRaw<FMT, GROUP>::type SRaw;
  constexpr int T = NR * CPW >= 8 ? 1 : 8 / (NR * CPW), kWave = T * NR * MB * 64;
  constexpr int kOut = T * MB * 64, kMine = (kOut + 64 * kWaves - 1) / (64 * kWaves);  // outputs of T tiles, a thread's
  __shared__ __align__(16) float red[2][kWaves * kWave];
  __shared__ float ssq[NORM ? kWaves : 1][MB * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = w4_wave();
  const int K = a.w.K, M = a.M, C = (K + kW4Chunk - 1) / kW4Chunk;
  const int r = lane & 7, lk = 128 * ((lane >> 3) & 1) + 8 * (lane >> 4);
  const int tiles = (a.N + kW4Rows - 1) / kW4Rows, up = a.N / kW4Rows, step = gridDim.x;

  struct Codes {
    u32x4 q[T][NR][CPW];
    SRaw s[T][NR][CPW];
    uint16_t resid[kMine];
  };
  // tiles past the last and chunks past K: the last ones again, not used
  auto load_w = [&](Codes& w, int first) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      if (t && first + t * step >= tiles) break;
#pragma unroll
      for (int j = 0; j < NR; ++j)
#pragma unroll
        for (int u = 0; u < CPW; ++u) {
          const int64_t block = static_cast<int64_t>(first + t * step + j * up) * C + min(wave + kWaves * u, C - 1);
          w.q[t][j][u] = reinterpret_cast<const u32x4*>(a.w.codes)[block * 64 + lane];
          w.s[t][j][u] = static_cast<const SRaw*>(a.w.scales)[block * 16 + (lane & 15)];
        }
    }
    if (a.R) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int e = tid + 64 * kWaves * i, tile = first + e / (MB * 64) * step;
        const int m = min(e / 8 % (MB * 8), M - 1), n = min(tile * kW4Rows + (e & 7), a.N - 1);
        w.resid[i] = static_cast<const uint16_t*>(a.R)[static_cast<int64_t>(m) * a.ldr + n];
      }
    }
  };
  Codes w0, w1;
  load_w(w0, blockIdx.x);

  // the wave's rows (those past M repeat the last; with a gain in two parts)
  bf16x8 x[CPW][4][MB], xl[CPW][4][MB];
#pragma unroll
  for (int u = 0; u < CPW; ++u)
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int k = (wave + kWaves * u) * kW4Chunk + 32 * s + lk;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
        x[u][s][mb] = load8(static_cast<const bf16*>(a.A) + static_cast<int64_t>(min(mb * 8 + r, M - 1)) * a.lda + (k < K ? k : 0));
    }
  bf16x8 gv[NORM ? CPW : 1][4];
  if constexpr (NORM) {
#pragma unroll
    for (int u = 0; u < CPW; ++u)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int k = (wave + kWaves * u) * kW4Chunk + 32 * s + lk;
        gv[u][s] = load8(static_cast<const bf16*>(a.g) + (k < K ? k : 0));
      }
  }
#pragma unroll
  for (int u = 0; u < CPW; ++u)
    if ((wave + kWaves * u + 1) * kW4Chunk > K) {  // wave-uniform
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) keep_if(x[u][s][mb], (wave + kWaves * u) * kW4Chunk + 32 * s + lk < K);
    }
  if constexpr (NORM) {
    // Sums of squares from the products of the rows with themselves (the diagonals of the
    // two blocks).  A row times the gain has 16 bits: two bf16 parts.
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      floatx4 q{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < CPW; ++u)
#pragma unroll
        for (int s = 0; s < 4; ++s) q = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[u][s][mb], x[u][s][mb], q, 0, 0, 0);
      // lane l: rows 4 (l / 16) + e of column l % 16
      const int e = lane & 3;
      float ss = e == 0 ? q[0] : e == 1 ? q[1] : e == 2 ? q[2] : q[3];
      ss += __shfl_xor(ss, 40, 64);
      if ((lane & 40) == 0 && (lane & 15) >> 2 == lane >> 4) ssq[wave][mb * 8 + r] = ss;
    }
#pragma unroll
    for (int u = 0; u < CPW; ++u) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float y = static_cast<float>(x[u][s][mb][e]) * static_cast<float>(gv[u][s][e]);
            x[u][s][mb][e] = static_cast<bf16>(y);
            xl[u][s][mb][e] = static_cast<bf16>(y - static_cast<float>(x[u][s][mb][e]));
          }
      if ((wave + kWaves * u + 1) * kW4Chunk > K) {  // a gain past K may be anything
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) {
            const bool in = (wave + kWaves * u) * kW4Chunk + 32 * s + lk < K;
            keep_if(x[u][s][mb], in);
            keep_if(xl[u][s][mb], in);
          }
      }
    }
  }

  auto do_tiles = [&](Codes& w, int first, int next, float* sums, Codes& wn) {
    if (next < tiles) load_w(wn, next);
#pragma unroll
    for (int t = 0; t < T; ++t) {
      if (t && first + t * step >= tiles) break;
#pragma unroll
      for (int j = 0; j < NR; ++j) {
        floatx4 acc[MB], part[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) acc[mb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < CPW; ++u) {
          if (wave + kWaves * u >= C) break;  // wave-uniform
#pragma unroll
          for (int s = 0; s < 4; ++s)
            w4_step<FMT, GROUP, MB, NORM>(s, w.q[t][j][u][s], w.s[t][j][u], x[u][s], xl[u][s], acc, part);
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          floatx4 v = acc[mb];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], 40, 64);
          if ((lane & 40) == 0)
            *reinterpret_cast<floatx4*>(sums + wave * kWave + (((t * NR + j) * MB + mb) * 8 + r) * 8 + 4 * (lane >> 4)) = v;
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int e = tid + 64 * kWaves * i, t = e / (MB * 64), m = e / 8 % (MB * 8), tile = first + t * step;
      const int64_t n = static_cast<int64_t>(tile) * kW4Rows + (e & 7);
      if (e >= kOut || m >= M || tile >= tiles || n >= a.N) continue;
      const float* at = sums + ((t * NR * MB + m / 8) * 8 + (e & 7)) * 8 + (m & 7);
      float s0 = 0.f, s1 = 0.f, scale = a.alpha;
#pragma unroll
      for (int wv = 0; wv < kWaves; ++wv) {
        s0 += at[wv * kWave];
        if constexpr (NR == 2) s1 += at[wv * kWave + MB * 64];
      }
      if constexpr (NORM) {
        float tot = 0.f;
#pragma unroll
        for (int wv = 0; wv < kWaves; ++wv) tot += ssq[wv][m];
        scale *= rsqrtf(tot / static_cast<float>(K) + a.eps);
      }
      w4_finish(a, m, n, s0, s1, scale, w.resid[i]);
    }
  };
  // (a buffer's readers are past the next barrier before it is written again)
  for (int tile = blockIdx.x; tile < tiles; tile += 2 * T * step) {
    do_tiles(w0, tile, tile + T * step, red[0], w1);
    if (tile + T * step < tiles) do_tiles(w1, tile + T * step, tile + 2 * T * step, red[1], w0);
  }
}

// Any rows and K: a workgroup takes 8 columns, its waves every eighth chunk, and reads
// rows and codes beside each other.  Bound by the codes' way from memory: one row, 4096 x
// 11008 int4 6.6 us (3.5 TB/s), 8192 x 16384 17.2 (3.9).
template <int FMT, int GROUP, int MB, int NR, bool NORM>
__global__ __launch_bounds__(64 * kWaves) void ld_gemm_w4_long(W4GemmArgs a) {
  typedef typename W4ScaleRaw<FMT, GROUP>::type SRaw;
  constexpr int kWave = NR * MB * 64;
  __shared__ __align__(16) float red[kWaves * kWave];
  __shared__ float ssq[NORM ? kWaves : 1][MB * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = a.w.K, M = a.M, C = (K + kW4Chunk - 1) / kW4Chunk;
  const int r = lane & 7, lk = 128 * ((lane >> 3) & 1) + 8 * (lane >> 4);
  const int64_t tile = a.wg0 + static_cast<int>(blockIdx.x), up = a.N / kW4Rows;
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
        keep_if(x[mb], in);
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
          keep_if(x[mb], in);
          keep_if(xl[mb], in);
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
      for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], 40, 64);
      if ((lane & 40) == 0) *reinterpret_cast<floatx4*>(red + wave * kWave + ((j * MB + mb) * 8 + r) * 8 + 4 * (lane >> 4)) = v;
    }
  if constexpr (NORM) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
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
  const float* at = red + (m / 8 * 8 + (tid & 7)) * 8 + (m & 7);
  float s0 = 0.f, s1 = 0.f, scale = a.alpha;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    s0 += at[w * kWave];
    if constexpr (NR == 2) s1 += at[w * kWave + MB * 64];
  }
  if constexpr (NORM) {
    float tot = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) tot += ssq[w][m];
    scale *= rsqrtf(tot / static_cast<float>(K) + a.eps);
  }
  w4_finish(a, m, n, s0, s1, scale, a.R ? static_cast<const uint16_t*>(a.R)[m * a.ldr + n] : 0);
}

template <int FMT, int GROUP, int MB, int NR, bool NORM, int CPW>
hipError_t gemm_held(const W4GemmArgs& a, hipStream_t s) {
  const int tiles = (a.N + kW4Rows - 1) / kW4Rows, rounds = (tiles + kCus - 1) / kCus;
  hipLaunchKernelGGL((ld_gemm_w4_k<FMT, GROUP, MB, NR, NORM, CPW>), dim3((tiles + rounds - 1) / rounds), dim3(64 * kWaves), 0, s, a);
  return hipGetLastError();
}

// At most 16 rows: held in registers where those suffice.
template <int FMT, int GROUP, int MB, int NR, bool NORM>
hipError_t gemm_few(const W4GemmArgs& a, hipStream_t s) {
  const int cpw = (a.w.K + kW4Chunk * kWaves - 1) / (kW4Chunk * kWaves);  // chunks a wave
  if (cpw <= 1) return gemm_held<FMT, GROUP, MB, NR, NORM, 1>(a, s);
  if (cpw <= 2) return gemm_held<FMT, GROUP, MB, NR, NORM, 2>(a, s);
  if constexpr (MB == 1 || NORM) {
    // One or two tiles a CU over long rows: no more is gained by holding rows than is lost by
    // taking the tiles in turn.  Us of one row, held and not: 4096 x 11008 9.2, 6.1; 2048 x 5504
    // 3.7, 3.1; 2048 x 16384 7.2, 6.3.  (22016 x 4096 14.7, 22.2; 12288 x 4096 9.6, 19.4.)
    const int tiles = (a.N + kW4Rows - 1) / kW4Rows;
    constexpr int kMost = MB > 1 ? 2 : NORM || NR == 2 ? 4 : 8;  // chunks a wave's registers hold
    if constexpr (kMost >= 4)
      if (tiles > 2 * kCus && cpw <= 4) return gemm_held<FMT, GROUP, MB, NR, NORM, 4>(a, s);
    if constexpr (kMost >= 8)
      if (tiles > 2 * kCus && cpw <= 8) return gemm_held<FMT, GROUP, MB, NR, NORM, 8>(a, s);
    return w4_launches(a, tiles, [&](const W4GemmArgs& part, dim3 grid) {
      hipLaunchKernelGGL((ld_gemm_w4_long<FMT, GROUP, MB, NR, NORM>), grid, dim3(64 * kWaves), 0, s, part);
    });
  }
  return hipErrorInvalidValue;  // more than 8 rows without a gain come here with up to 4096 k (w4_gemm_by_rows)
}

template <int FMT, int GROUP, int MB>
hipError_t gemm_mb(const W4GemmArgs& a, hipStream_t s) {
  const bool glu = a.act == kDecActSwiglu;
  if (a.g) return glu ? gemm_few<FMT, GROUP, MB, 2, true>(a, s) : gemm_few<FMT, GROUP, MB, 1, true>(a, s);
  return glu ? gemm_few<FMT, GROUP, MB, 2, false>(a, s) : gemm_few<FMT, GROUP, MB, 1, false>(a, s);
}

template <int FMT, int GROUP>
hipError_t gemm_t(const W4GemmArgs& a, hipStream_t s) {
  if (a.M < 1) return hipErrorInvalidValue;
  return a.M <= 8 ? gemm_mb<FMT, GROUP, 1>(a, s) : gemm_mb<FMT, GROUP, 2>(a, s);
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
bool w4_gemm_fuses_norm(int64_t M, int64_t K) { return M <= kW4FewRows && K <= 8192; }

// From 9 rows on reading them costs as much as the codes where they are long, and laid
// out in memory once (or not, if short) they are used for more columns.  Us of 16 rows, held and laid out: 4096
// x 11008 22.2, 10.2; 2048 x 5504 9.9, 6.6; 16384 x 8192 25.2, 21.3; 22016 x 4096 18.0, 15.4;
// 12288 x 4096 12.0, 12.3; 6144 x 2048 4.8, 6.3.  Of 8: 4096 x 11008 12.8, 10.1, 8192 x 5504 10.7,
// 11.2, 2048 x 16384 10.0, 11.8.
bool w4_gemm_by_rows(int64_t M, int64_t N, int64_t K, bool norm) {
  return M > kW4FewRows || (M > 8 && !norm && (K > 4096 || N > 16384));
}

hipError_t launch_gemm_w4(const W4GemmArgs& a, hipStream_t s) {
  if (w4_gemm_by_rows(a.M, a.w.N, a.w.K, a.g != nullptr)) return launch_gemm_w4_rows(a, s);
  if (a.w.format == LD_W4_E2M1) return gemm_t<LD_W4_E2M1, 32>(a, s);
  return a.w.group == 32 ? gemm_t<LD_W4_INT4, 32>(a, s) : a.w.group == 64 ? gemm_t<LD_W4_INT4, 64>(a, s)
                                                        : gemm_t<LD_W4_INT4, 128>(a, s);
}

}  // namespace ld
