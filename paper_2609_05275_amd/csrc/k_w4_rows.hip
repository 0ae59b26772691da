// Projections of 9 to 64 rows by 4-bit weights.  Layout: W4View in ld_w4.h.
#include "w4_codes.h"

namespace ld {
namespace {

// A block of 16 rows and 32 k as the operand that a product takes: lane 16 g + n has row n's
// k = 8 g .. 8 g + 7.  Blocks [ceil(K / 256)][2][4][MB]; rows and k past the last are zeros.
// A workgroup takes four blocks of the same rows (blockIdx.y): half a chunk.
__global__ __launch_bounds__(256) void ld_w4_rows_k(W4GemmArgs a, int mb_count) {
  const int lane = threadIdx.x & 63, kb = blockIdx.x * 4 + (threadIdx.x >> 6), b = kb * mb_count + blockIdx.y;
  const int m = blockIdx.y * 16 + (lane & 15), k = kb * 32 + 8 * (lane >> 4);
  bf16x8 x = load8(static_cast<const bf16*>(a.A) + static_cast<int64_t>(min(m, a.M - 1)) * a.lda + (k < a.w.K ? k : 0));
  keep_if(x, m < a.M && k < a.w.K);
  static_cast<bf16x8*>(a.ws)[static_cast<int64_t>(b) * 64 + lane] = x;
}

// MB blocks of 16 rows against CG groups of 16 rows of W (two tiles; SwiGLU: half the groups
// gate rows, half up rows), the workgroup's eight waves taking its chunks in turn, so that
// the rows are read once a workgroup and used for CG products.  A product's 16 columns are
// 16 rows of W with the same 32 k: lanes 0-7 of 16 read one tile, lanes 8-15 the next, the same
// half of a chunk, whole lines of 128 bytes.  A half's registers are loaded with the next
// chunk's as soon as it is used.
//
// What bounds it: with few rows the codes (16 rows, 8192 x 16384: 16.5-17.7 us, 4 TB/s).  With
// more no unit is full: two waves a SIMD wait for codes, for rows and for each other, and over
// K of 4096 a wave has two chunks between the first loads and the exchange of 72 KB of
// sums.  48 rows of gate and up, 11008 x 4096 int4 in groups of 64: 21 us, 3 of them the laying
// out, vector units 0.24 and matrix units 0.13 busy (101 with the rows in LDS, 23.2 with halves
// exchanged between lanes); 64 rows, 16384 x 16384: 54 us, 0.34 and 0.24.  Rows read as they lie, 64
// bytes a row and step, took 25.7 us for 17.4 (33 rows, 4096 x 11008 e2m1): rows far apart meet in
// few of the L2's channels.
// LAID: the rows are ld_w4_rows_k's, else A's.
template <int FMT, int GROUP, int MB, int CG, bool LAID>
__global__ __launch_bounds__(64 * kWaves) void ld_gemm_w4_rows(W4GemmArgs a) {
  typedef typename W4ScaleRaw<FMT, GROUP>::type SRaw;
  constexpr int kWave = CG * MB * 256;  // sums of a wave
  __shared__ __align__(16) float red[kWaves / 2 * kWave];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int M = a.M, C = (a.w.K + kW4Chunk - 1) / kW4Chunk, n16 = lane & 15, g = lane >> 4;
  const bool glu = a.act == kDecActSwiglu;
  const int tiles = (a.w.N + kW4Rows - 1) / kW4Rows, part_tiles = glu ? a.N / kW4Rows : tiles;
  const int groups = glu ? CG / 2 : CG;       // of columns of C
  const int first = (a.wg0 + static_cast<int>(blockIdx.x)) * groups * 2;  // tile
  floatx4 acc[CG][MB];
#pragma unroll
  for (int i = 0; i < CG; ++i)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) acc[i][mb] = floatx4{0.f, 0.f, 0.f, 0.f};

  u32x4 w[CG][2];  // halves of a chunk
  SRaw sw[CG][2];
  // a lane's bytes from the first tile's block, its rows being in this one or the next
  const uint32_t in_w = 256 * g + 16 * (n16 & 7), in_s = n16 & 7;
  const uint32_t next_w = n16 >> 3 ? C * 1024u : 0u, next_s = n16 >> 3 ? C * 16u : 0u;
  auto load_w = [&](int i, int c, int half) {
    const bool is_up = glu && i >= CG / 2;
    const int t = first + (is_up ? i - CG / 2 : i) * 2, last = part_tiles - 1;
    const int64_t block = static_cast<int64_t>(min(t, last) + (is_up ? part_tiles : 0)) * C + c;
    const bool pair = t < last;  // (past the last tile: the last again, not stored)
    w[i][half] = *reinterpret_cast<const u32x4*>(a.w.codes + block * 1024 + 128 * half + (in_w + (pair ? next_w : 0u)));
    sw[i][half] = (static_cast<const SRaw*>(a.w.scales) + block * 16 + 8 * half)[in_s + (pair ? next_s : 0u)];
  };
  const bf16x8* laid = static_cast<const bf16x8*>(a.ws) + lane;
  const bf16* rows[MB];  // (past the last row: the last again, not stored)
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
    rows[mb] = static_cast<const bf16*>(a.A) + static_cast<int64_t>(min(16 * mb + n16, M - 1)) * a.lda + 8 * g;
  bf16x8 x[2][2][MB];  // two steps, the next two
  auto load_x = [&](bf16x8 (&to)[2][MB], int pair) {  // pair of steps, four a chunk
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        if constexpr (LAID) {
          to[s][mb] = laid[(static_cast<int64_t>(pair * 2 + s) * MB + mb) * 64];
        } else {
          const int k = pair * 64 + 32 * s;
          const bool in = k + 8 * g < a.w.K;
          to[s][mb] = load8(rows[mb] + (in ? k : -8 * g));
          keep_if(to[s][mb], in);
        }
      }
  };
  if (wave < C) {
    load_x(x[0], wave * 4);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < CG; ++i) load_w(i, wave, half);
  }
  for (int c = wave; c < C; c += kWaves) {
    const int next = c + kWaves < C ? c + kWaves : c;  // (the last chunk's again, not used)
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      load_x(x[(p + 1) & 1], p < 3 ? c * 4 + p + 1 : next * 4);
      // (else the compiler moves the loads to their use: 33 rows, 4096 x 11008 e2m1, 24.5 us for
      // 17.4; the largest blocks have no registers for it)
      if constexpr (MB * CG < 18) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < CG; ++i) {
        w4_pair<FMT, GROUP, MB>(p & 1, w[i][p >> 1], sw[i][p >> 1], x[p & 1], acc[i]);
        if (p & 1) load_w(i, next, p >> 1);
      }
    }
  }
  // the last four waves' sums, then all on the first four's; lane: rows 4 g + e of column n16
  float* mine = red + (wave & 3) * kWave;
#pragma unroll
  for (int half = 1; half >= 0; --half) {
    if (wave >> 2 == half) {
#pragma unroll
      for (int i = 0; i < CG; ++i)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          floatx4* at = reinterpret_cast<floatx4*>(mine + ((i * MB + mb) * 16 + n16) * 16 + 4 * g);
          *at = half ? acc[i][mb] : acc[i][mb] + *at;
        }
    }
    __syncthreads();
  }
  const int cols = groups * 16, outs = cols * MB * 16;
  for (int e = tid; e < outs; e += 64 * kWaves) {
    // columns first: neighbouring threads store neighbouring elements
    const int col = e % cols, m = e / cols, i = col / 16;
    const int64_t n = static_cast<int64_t>(first) * kW4Rows + col;
    if (m >= M || n >= a.N) continue;
    const float* at = red + ((i * MB + m / 16) * 16 + col % 16) * 16 + m % 16;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves / 2; ++v) s0 += at[v * kWave];
    if (glu) {
#pragma unroll
      for (int v = 0; v < kWaves / 2; ++v) s1 += at[v * kWave + CG / 2 * MB * 256];
    }
    w4_finish(a, m, n, s0, s1, a.alpha, a.R ? static_cast<const uint16_t*>(a.R)[m * a.ldr + n] : 0);
  }
}

template <int FMT, int GROUP, int MB, int CG, bool LAID = true>
hipError_t rows_launch(const W4GemmArgs& a, hipStream_t s) {
  const int cols = (a.act == kDecActSwiglu ? CG / 2 : CG) * 16;
  return w4_launches(a, (a.N + cols - 1) / cols, [&](const W4GemmArgs& part, dim3 grid) {
    hipLaunchKernelGGL((ld_gemm_w4_rows<FMT, GROUP, MB, CG, LAID>), grid, dim3(64 * kWaves), 0, s, part);
  });
}

// Short rows are read where they lie, which saves a launch.  Us laid out and not, 2304 columns:
// 24 rows of 512 4.8, 4.0, of 1024 5.0, 4.5, of 2048 5.9, 6.3; 40 of 768 5.5, 5.0, of 1024 5.6, 5.7; 64 of
// 512 5.7, 5.7, of 768 5.8, 6.4; 16 of 2048, 24000 columns, 10.8, 11.8; from Python two launches
// cost 3 more.
bool w4_rows_laid(int64_t M, int64_t K) { return (M <= 32 ? 2 : (M + 15) / 16) * K > 2560; }

// Groups a workgroup: with up to 32 rows two at most, so that registers leave room for a
// second workgroup; with more rows the fewest with which one round of workgroups does, since
// the rows are then read for as many columns as possible.  Us of 1, 2, 4 and 6 groups, int4 in
// groups of 64: 24 rows, 24000 x 4096 24.2, 17.8, 22.3, 18.7, 4096 x 4096 7.2, 8.8, 11.5, 14.6; 33
// rows, 24000 x 4096 31.4, 26.1, 26.7, 21.6, 12288 x 4096 18.6, 18.6, 15.4, 19.6, 4096 x 11008
// 17.7, 19.5, 24.4, 33.7.
template <int FMT, int GROUP, int MB>
hipError_t rows_mb(const W4GemmArgs& a, hipStream_t s) {
  const int groups = (a.w.N + 15) / 16;
  if (!w4_rows_laid(a.M, a.w.K)) {
    if constexpr (MB > 1)  // (up to 16 short rows come here with many columns alone)
      if (groups <= kCus && a.act != kDecActSwiglu) return rows_launch<FMT, GROUP, MB, 1, false>(a, s);
    return rows_launch<FMT, GROUP, MB, 2, false>(a, s);
  }
  if (groups <= kCus && a.act != kDecActSwiglu) return rows_launch<FMT, GROUP, MB, 1>(a, s);
  if constexpr (MB > 2) {
    if (groups > 4 * kCus) return rows_launch<FMT, GROUP, MB, 6>(a, s);
    if (groups > 2 * kCus) return rows_launch<FMT, GROUP, MB, 4>(a, s);
  }
  return rows_launch<FMT, GROUP, MB, 2>(a, s);
}

template <int FMT, int GROUP>
hipError_t rows_t(const W4GemmArgs& a, hipStream_t s) {
  return a.M <= 16 ? rows_mb<FMT, GROUP, 1>(a, s) : a.M <= 32 ? rows_mb<FMT, GROUP, 2>(a, s) : a.M <= 48 ? rows_mb<FMT, GROUP, 3>(a, s) : rows_mb<FMT, GROUP, 4>(a, s);
}

}  // namespace

size_t w4_gemm_ws_bytes(int64_t M, int64_t N, int64_t K, bool norm) {
  if (!w4_gemm_by_rows(M, N, K, norm) || !w4_rows_laid(M, K)) return 0;
  return static_cast<size_t>((M + 15) / 16 * 16) * ((K + kW4Chunk - 1) / kW4Chunk * kW4Chunk) * 2;
}

hipError_t launch_gemm_w4_rows(const W4GemmArgs& a, hipStream_t s) {
  if (a.M < 1 || a.M > kW4MaxM || a.g || (w4_rows_laid(a.M, a.w.K) && !a.ws)) return hipErrorInvalidValue;
  if (w4_rows_laid(a.M, a.w.K)) {
    const int mb = (a.M + 15) / 16, chunks = (a.w.K + kW4Chunk - 1) / kW4Chunk;
    hipLaunchKernelGGL(ld_w4_rows_k, dim3(2 * chunks, mb), dim3(256), 0, s, a, mb);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.w.format == LD_W4_E2M1) return rows_t<LD_W4_E2M1, 32>(a, s);
  return a.w.group == 32 ? rows_t<LD_W4_INT4, 32>(a, s) : a.w.group == 64 ? rows_t<LD_W4_INT4, 64>(a, s)
                                                        : rows_t<LD_W4_INT4, 128>(a, s);
}

}  // namespace ld
