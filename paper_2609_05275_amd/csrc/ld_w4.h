// Projections by 4-bit weights, as the API calls them.  A header of its own: the
// other kernels' counter records hold for the contents of ld_internal.h.
#pragma once
#include "ld_internal.h"

namespace ld {

// Weights [N, K] in 4 bits (ld_w4).  A block of 8 rows and 256 k is 64 lanes of 16 bytes:
// lane 16 g + 8 h + r, dword s, holds row r at k = 128 h + 32 s + 8 g + e, e < 8: the B
// operand of v_mfma_f32_16x16x32_bf16 whose columns 0-7 are the rows with the first 128 k
// and 8-15 the rows with the last 128.  Blocks [ceil(N / 8)][ceil(K / 256)]; scales
// [ceil(N / 8)][ceil(K / 256)][h][r][128 / group].
struct W4View {
  uint8_t* codes;
  void* scales;
  int32_t format, group, N, K;
};
constexpr int kW4Rows = 8, kW4Chunk = 256;
constexpr int kW4MaxM = 64;
constexpr int kW4FewRows = 16;  // the most of launch_gemm_w4's own kernels; they may take a norm
constexpr int kW4MinExp = -100;

struct W4PackArgs {
  W4View w;
  const void* src;  // bf16 [N, K], ld apart; pack
  void* dst;        // load
  int64_t ld;
};

// C = act(R + alpha A' W^T), A' the RMSNorm of A's rows where g is given; act
// kDecActSwiglu: W holds the gate rows 0 .. N - 1, then the up rows.
struct W4GemmArgs {
  W4View w;
  int32_t wg0;  // a launch's first workgroup, where they go in several (w4_launches)
  const void *A, *g, *R;
  void* C;
  int64_t lda, ldc, ldr;
  int32_t M, N, act;
  float alpha, eps;
  void* ws;  // of w4_gemm_ws_bytes
};

hipError_t launch_w4_pack(const W4PackArgs& a, hipStream_t s);
hipError_t launch_w4_load(const W4PackArgs& a, hipStream_t s);
bool w4_gemm_fuses_norm(int64_t M, int64_t K);
// Whether M rows go to launch_gemm_w4_rows, N rows of W; and the scratch in which they are
// laid out then, if they are.
bool w4_gemm_by_rows(int64_t M, int64_t N, int64_t K, bool norm);
size_t w4_gemm_ws_bytes(int64_t M, int64_t N, int64_t K, bool norm);
hipError_t launch_gemm_w4(const W4GemmArgs& a, hipStream_t s);
hipError_t launch_gemm_w4_rows(const W4GemmArgs& a, hipStream_t s);  // without a gain

}  // namespace ld
