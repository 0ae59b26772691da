// Kernels of the 8-bit key/value cache: quantising writer, reader, and the
// attention of a few new rows per sequence over it.  Layout and the meaning of
// codes and scales: Kv8View in ld_internal.h, ld_kv8 in layerdrop.h.
//
// Scales are powers of two, so dividing by one and multiplying with it are
// exact: a code is one rounding of its value, a value read back is the code's
// in bf16 without another, and raising a block's scale rounds old codes by a
// whole number of bits.
#include "ld_internal.h"

namespace ld {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kKv8Waves = 8;  // of an attention workgroup
constexpr int kCus = 256;

// ------------------------------------------------------------- conversions

// 8 codes (two dwords) to bf16, exact: e4m3 has 4 significant bits, int8 seven.
template <int FMT>
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t a, uint32_t b) {
  union {
    bf16x8 v;
    bf16x2 p[4];
    uint32_t u[4];
  } r;
  if constexpr (FMT == LD_KV8_E4M3) {
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
  } else {
    // (opaque, or the loads' registers are split into bytes as they arrive)
    asm("" : "+v"(a), "+v"(b));
    const uint32_t w[2] = {a, b};
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // a float of 7 bits is its upper half
      const int x = static_cast<int>(w[i >> 1]);
      const float lo = static_cast<float>(static_cast<int8_t>(i & 1 ? x >> 16 : x));
      const float hi = static_cast<float>(static_cast<int8_t>(i & 1 ? x >> 24 : x >> 8));
      r.u[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
    }
  }
  return r.v;
}

// 4 values, already divided by their scale, to codes: nearest, ties to even.
template <int FMT>
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
  if constexpr (FMT == LD_KV8_E4M3) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true));
  } else {
    const uint32_t ia = static_cast<int>(__builtin_rintf(a)), ib = static_cast<int>(__builtin_rintf(b));
    const uint32_t ic = static_cast<int>(__builtin_rintf(c)), id = static_cast<int>(__builtin_rintf(d));
    const uint32_t ab = __builtin_amdgcn_perm(ib, ia, 0x0c0c0400u), cd = __builtin_amdgcn_perm(id, ic, 0x0c0c0400u);
    return ab | (cd << 16);
  }
}

template <int FMT>
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, float f) {
  float x[4];
  if constexpr (FMT == LD_KV8_E4M3) {
    x[0] = __builtin_amdgcn_cvt_f32_fp8(codes, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8(codes, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8(codes, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8(codes, 3);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = static_cast<float>(static_cast<int8_t>(codes >> (8 * i)));
  }
  return pack_codes<FMT>(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
}

// The scale a block needs, from the largest absolute value's bf16 bits.
template <int FMT>
__device__ __forceinline__ float scale_needed(uint32_t amax) {
  if (amax >= 0x7f80u) return __builtin_nanf("");
  constexpr int kTop = FMT == LD_KV8_E4M3 ? 8 : 6;            // Q = 1.m 2^kTop
  constexpr uint32_t kMant = FMT == LD_KV8_E4M3 ? 0x60u : 0x7eu;
  int e = static_cast<int>(amax >> 7) - 127 - kTop + ((amax & 0x7fu) > kMant ? 1 : 0);
  e = max(e, kKv8MinExp);  // zeros and subnormals too
  return __builtin_bit_cast(float, static_cast<uint32_t>(e + 127) << 23);
}

// ------------------------------------------------------------------- store

// A workgroup takes a tile of TT positions (whole blocks) of one head's keys
// or values.  Every thread holds 8 dimensions of TT DH / 2048 rows.
template <int DH, int FMT, int TT>
__global__ __launch_bounds__(256) void ld_kv8_store_k(Kv8StoreArgs a) {
  constexpr int PT = DH / 8, TPP = 256 / PT, NP = TT / TPP, TW = 64 / PT;  // threads a row, rows a pass (a wave's: TW)
  __shared__ uint32_t amax_s[NP * 4];
  __shared__ float inv_s[TT / 16], ratio_s;
  __shared__ __align__(16) uint8_t ct[TT][DH];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int part = blockIdx.y & 1, h = blockIdx.y >> 1, b = blockIdx.z;
  const Kv8View& c = a.kv;
  int p = a.pos;
  if (a.seq_pos) {
    p = a.seq_pos[b];
    if (p < 0 || p > a.pos) return;
  }
  const int lo = p, hi = p + a.n;
  const int t0 = (p / TT + static_cast<int>(blockIdx.x)) * TT;
  if (t0 >= hi) return;
  const int tr = tid / PT, d8 = (tid % PT) * 8;
  const bf16* src = static_cast<const bf16*>(a.qkv) + static_cast<int64_t>(b) * a.n * a.ld_qkv +
                    (a.H + part * c.KV + h) * static_cast<int64_t>(DH) + d8;
  const int64_t head = static_cast<int64_t>(b) * c.KV + h;
  uint8_t* codes = c.codes + (head * 2 + part) * c.s16 * DH;
  float* scales = c.scales + (head * 2 + part) * c.nb;

  bf16x8 v[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int t = t0 + i * TPP + tr;
    v[i] = static_cast<bf16>(0.f);
    if (t >= lo && t < hi) v[i] = *reinterpret_cast<const bf16x8*>(src + static_cast<int64_t>(t - lo) * a.ld_qkv);
  }
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    union {
      bf16x8 v;
      uint16_t u[8];
    } x{v[i]};
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, static_cast<uint32_t>(x.u[e] & 0x7fff));
#pragma unroll
    for (int o = 1; o < 64; o *= 2) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o, 64)));
    if (lane == 0) amax_s[i * 4 + wave] = m;
  }
  if (tid == 0) ratio_s = 1.f;
  __syncthreads();
  const int per = c.block / TW;  // entries of amax_s per block
  if (tid < TT / c.block) {
    const int s0 = t0 + tid * c.block;
    float inv = 0.f;
    if (s0 < hi && s0 + c.block > lo) {
      uint32_t m = 0;
      for (int i = 0; i < per; ++i) m = max(m, amax_s[tid * per + i]);
      float s = scale_needed<FMT>(m);
      if (s0 < lo) {  // holds earlier rows: its scale can only rise
        const float old = scales[s0 / c.block];
        if (s == s && !(old <= s)) s = old;
        if (old != s) ratio_s = old / s;
      }
      scales[s0 / c.block] = s;
      inv = 1.f / s;
    }
    inv_s[tid] = inv;
  }
  __syncthreads();
  const float ratio = ratio_s;
  const bool again = ratio < 1.f;  // never for a NaN: such a block's codes say nothing
  const int b0 = max(t0, lo / c.block * c.block);  // earlier rows to round again: b0..lo-1

  // codes: keys to the cache at once, values to LDS for their transpose
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int t = t0 + i * TPP + tr;
    if (t >= lo && t < hi) {
      const float inv = inv_s[(t - t0) / c.block];
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = inv == inv ? static_cast<float>(v[i][e]) * inv : 0.f;
      u32x2 q{pack_codes<FMT>(x[0], x[1], x[2], x[3]), pack_codes<FMT>(x[4], x[5], x[6], x[7])};
      if (part == 0)
        *reinterpret_cast<u32x2*>(codes + static_cast<int64_t>(t) * DH + d8) = q;
      else
        *reinterpret_cast<u32x2*>(&ct[t - t0][d8]) = q;
    } else if (part == 0 && again && t >= b0 && t < lo) {
      u32x2* at = reinterpret_cast<u32x2*>(codes + static_cast<int64_t>(t) * DH + d8);
      const u32x2 q = *at;
      *at = u32x2{rescale4<FMT>(q[0], ratio), rescale4<FMT>(q[1], ratio)};
    }
  }
  if (part == 0) return;
  __syncthreads();
  // 16 positions of one dimension per thread and turn
  for (int r = tid; r < TT / 16 * DH; r += 256) {
    const int tile = r / DH, d = r % DH, f = t0 + 16 * tile;
    if (f >= hi || f + 16 <= (again ? b0 : lo)) continue;
    u32x4* at = reinterpret_cast<u32x4*>(codes + static_cast<int64_t>(f) * DH + d * 16);
    union {
      u32x4 v;
      uint8_t u[16];
    } q;
    if (f < lo || f + 16 > hi) {
      q.v = *at;
      if (again) {
#pragma unroll
        for (int i = 0; i < 4; ++i) q.v[i] = rescale4<FMT>(q.v[i], ratio);
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (f + i >= lo && f + i < hi) q.u[i] = ct[16 * tile + i][d];
    *at = q.v;
  }
}

// -------------------------------------------------------------------- load

// A workgroup takes 64 positions of one head's keys or values.
template <int DH, int FMT>
__global__ __launch_bounds__(256) void ld_kv8_load_k(Kv8LoadArgs a) {
  __shared__ __align__(16) uint8_t ct[4][DH][16];
  const int tid = threadIdx.x, part = blockIdx.y & 1, h = blockIdx.y >> 1, b = blockIdx.z;
  const Kv8View& c = a.kv;
  const int t0 = (a.pos / 64 + static_cast<int>(blockIdx.x)) * 64;
  int hi = a.pos + a.n;
  if (a.seq_len) hi = min(hi, a.seq_len[b]);
  if (t0 >= hi) return;
  const int64_t head = static_cast<int64_t>(b) * c.KV + h;
  const uint8_t* codes = c.codes + (head * 2 + part) * c.s16 * DH;
  const float* scales = c.scales + (head * 2 + part) * c.nb;
  if (part) {
    for (int r = tid; r < 4 * DH; r += 256) {
      const int f = t0 + 16 * (r / DH);
      if (f < hi) *reinterpret_cast<u32x4*>(&ct[r / DH][r % DH][0]) = *reinterpret_cast<const u32x4*>(codes + static_cast<int64_t>(f) * DH + (r % DH) * 16);
    }
    __syncthreads();
  }
  bf16* out = static_cast<bf16*>(a.out) + static_cast<int64_t>(b) * a.n * 2 * c.KV * DH +
              (static_cast<int64_t>(part) * c.KV + h) * DH;
  for (int r = tid; r < 64 * (DH / 8); r += 256) {
    const int i = r / (DH / 8), d8 = r % (DH / 8) * 8, t = t0 + i;
    if (t < a.pos || t >= hi) continue;
    u32x2 q;
    if (part) {
      union {
        u32x2 v;
        uint8_t u[8];
      } x;
#pragma unroll
      for (int e = 0; e < 8; ++e) x.u[e] = ct[i / 16][d8 + e][i % 16];
      q = x.v;
    } else {
      q = *reinterpret_cast<const u32x2*>(codes + static_cast<int64_t>(t) * DH + d8);
    }
    const float s = scales[t / c.block];
    bf16x8 v = codes_to_bf16<FMT>(q[0], q[1]);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<bf16>(static_cast<float>(v[e]) * s);
    *reinterpret_cast<bf16x8*>(out + static_cast<int64_t>(t - a.pos) * 2 * c.KV * DH + d8) = v;
  }
}

// --------------------------------------------------------------- attention

// A workgroup of eight waves takes a chunk of keys of one key/value head for 16
// rows (of its query heads' new rows); a wave 32 keys at a time, with its own
// running maximum and sum; they meet once, to add up.
//
// Scores S^T = K Q^T and output O^T = V^T P^T on the matrix cores (16x16x32
// bf16).  The A rows of score product t are the keys 8 g + 4 t + r (row 4 g + r),
// so lane group g = lane / 16 of the result holds keys 8 g + 4 t + r, t < 2, r < 4, of
// its query row: 8 neighbouring keys, half a tile of the cache's values, of one
// scale.  They are the B operand of O^T as they stand, and 8 bytes of a value
// tile's row the A operand.
//
// Codes are exact in bf16.  A probability, times its value scale, is split in
// two bf16 parts, which leave 2^-16 of it.
//
// Bound by the cache stream.  A wave asks for its keys and values at once (8 KB)
// and waits; 16 waves a CU at 128 registers hold 128 KB in flight.
template <int DH, int FMT, int NQ>
__global__ __launch_bounds__(64 * kKv8Waves, 4) void ld_attn_decode_kv8_k(Kv8AttnArgs a) {
  constexpr int NS = DH / 64, MT = DH / 16, NW = kKv8Waves, TT = 2, LK = 4 * TT, WK = 16 * TT;
  __shared__ float ml[NW][NQ][2];
  __shared__ __align__(16) float red[NW][NQ][DH];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const Kv8View& c = a.kv;
  const int h = static_cast<int>(blockIdx.y) % c.KV, rt = static_cast<int>(blockIdx.y) / c.KV, b = blockIdx.z;
  // Workgroups go round the XCDs by their number: turned by the head, or a number
  // of chunks that shares a factor with the XCDs' would leave those of the last
  // chunks, which short sequences do not fill, with little to do.
  const int chunk = static_cast<int>((blockIdx.x + blockIdx.y + blockIdx.z) % gridDim.x);
  const int G = a.H / c.KV, R = G * a.n_new;
  int p = a.pos;
  if (a.seq_pos) {
    p = a.seq_pos[b];
    if (p < 0 || p > a.pos) p = -a.n_new;  // left out: no keys
  }
  const int nk = p + a.n_new, k_first = chunk * a.chunk_keys;
  const int rows = min(R - rt * 16, 16);
  const int64_t d = static_cast<int64_t>(a.H) * DH;
  if (k_first >= nk) {
    if (chunk == 0 && a.n_chunks == 1) {  // left out: its rows are zeros (the combine's else)
      for (int e = tid; e < rows * DH; e += 64 * NW) {
        const int r = rt * 16 + e / DH;
        static_cast<bf16*>(a.out)[(static_cast<int64_t>(b) * a.n_new + r % a.n_new) * d +
                                  (h * G + r / a.n_new) * static_cast<int64_t>(DH) + e % DH] = static_cast<bf16>(0.f);
      }
    }
    return;
  }
  const int k_end = min(k_first + a.chunk_keys, nk);
  const int64_t head = static_cast<int64_t>(b) * c.KV + h;
  const uint8_t* kc = c.codes + head * 2 * c.s16 * DH;
  const uint8_t* vc = kc + static_cast<int64_t>(c.s16) * DH;
  const float* ks = c.scales + head * 2 * c.nb;
  const float* vs = ks + c.nb;

  // Keys k0 .. k0 + WK - 1 (past the last key: key 0, masked later): row n of
  // product t, dimensions 64 s + 16 g + 0..15.
  const int krow = LK * (n >> 2) + (n & 3);
  typedef uint32_t VRaw __attribute__((ext_vector_type(TT)));
  u32x4 kr[TT][NS];
  VRaw vr[MT];
  float sk = 0.f, sv = 0.f;
  auto load_keys = [&](int k0) {
    if (k0 + WK <= nk) {
      const uint8_t* at = kc + static_cast<int64_t>(k0 + krow) * DH + 16 * g;
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int s = 0; s < NS; ++s) kr[t][s] = *reinterpret_cast<const u32x4*>(at + 4 * t * DH + 64 * s);
    } else {
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const int kk = k0 + krow + 4 * t;
        const uint8_t* at = kc + static_cast<int64_t>(kk < nk ? kk : 0) * DH + 16 * g;
#pragma unroll
        for (int s = 0; s < NS; ++s) kr[t][s] = *reinterpret_cast<const u32x4*>(at + 64 * s);
      }
    }
    const int f = k0 + LK * g;
    sk = ks[(f < nk ? f : 0) >> c.shift];
  };
  auto load_values = [&](int k0) {
    const int f = k0 + LK * g, fc = f < nk ? f : 0;
    const uint8_t* at = vc + static_cast<int64_t>(fc & ~15) * DH + n * 16 + (fc & 15);
#pragma unroll
    for (int i = 0; i < MT; ++i) vr[i] = *reinterpret_cast<const VRaw*>(at + 256 * i);
    sv = vs[fc >> c.shift];
  };

  int k0 = k_first + wave * WK;
  const int row = rt * 16 + min(n, rows - 1), qh = h * G + row / a.n_new, j = row % a.n_new, qpos = p + j;
  bf16x8 qf[NS][2];
  {
    const bf16* q = static_cast<const bf16*>(a.qkv) + (static_cast<int64_t>(b) * a.n_new + j) * a.ld_qkv +
                    static_cast<int64_t>(qh) * DH;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        qf[s][e] = *reinterpret_cast<const bf16x8*>(q + 64 * s + 16 * g + 8 * e);
  }
  const float al2 = a.alibi ? alibi_slope(qh, a.H) * kLog2e : 0.f, sl2 = a.scale * kLog2e;

  float m = -INFINITY, l = 0.f;
  floatx4 o[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};

  for (; k0 < k_end; k0 += WK * NW) {
    load_keys(k0);
    load_values(k0);
    __builtin_amdgcn_sched_barrier(0);
    const int f = k0 + LK * g;  // the lane's keys
    const float ss = sk * sl2;
    float x[TT][4];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      floatx4 s4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16<FMT>(kr[t][s][0], kr[t][s][1]), qf[s][0], s4, 0, 0, 0);
        s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16<FMT>(kr[t][s][2], kr[t][s][3]), qf[s][1], s4, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) x[t][r] = s4[r] * ss;
      __builtin_amdgcn_sched_barrier(0);
    }
    if (a.alibi) {
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[t][r] -= al2 * static_cast<float>(qpos - (f + 4 * t + r));
    }
    const bool cut = k0 + WK - 1 > p;  // some of the keys may be behind a row, or behind the last one
    if (cut) {
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (f + 4 * t + r > qpos) x[t][r] = -INFINITY;
    }
    float mn = m;
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mn = fmaxf(mn, x[t][r]);
    mn = fmaxf(mn, __shfl_xor(mn, 16, 64));
    mn = fmaxf(mn, __shfl_xor(mn, 32, 64));
    const float mz = mn == -INFINITY ? 0.f : mn;  // of nothing but -inf, whose weights are 0
    const float keep = __builtin_amdgcn_exp2f(m - mz);
    if (__any(mn != m)) {
      l *= keep;
#pragma unroll
      for (int i = 0; i < MT; ++i) o[i] *= keep;
    }
    m = mn;
    bf16x8 ph[TT / 2], pl[TT / 2];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = __builtin_amdgcn_exp2f(x[t][r] - mz);
        l += e;
        x[t][r] = e * sv;
      }
    if (cut) {  // nothing of a masked position, whose scale may be NaN
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (f + 4 * t + r > qpos) x[t][r] = 0.f;
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bf16 whi = static_cast<bf16>(x[t][r]);
        ph[t >> 1][4 * (t & 1) + r] = whi;
        pl[t >> 1][4 * (t & 1) + r] = static_cast<bf16>(x[t][r] - static_cast<float>(whi));
      }
    if (k0 + WK > nk) {  // codes behind the last key may be anything, NaN too
#pragma unroll
      for (int w = 0; w < TT; ++w) {
        const int have = nk - f - 4 * w;  // keys of this dword
        const uint32_t mask = have <= 0 ? 0u : have >= 4 ? ~0u : (1u << (8 * have)) - 1u;
#pragma unroll
        for (int i = 0; i < MT; ++i) vr[i][w] &= mask;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < TT / 2; ++u) {
        const bf16x8 v8 = codes_to_bf16<FMT>(vr[i][2 * u], vr[i][2 * u + 1]);
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, ph[u], o[i], 0, 0, 0);
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, pl[u], o[i], 0, 0, 0);
      }
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (lane < NQ) {
    ml[wave][lane][0] = m;
    ml[wave][lane][1] = l;
  }
  if (n < NQ)
#pragma unroll
    for (int i = 0; i < MT; ++i) *reinterpret_cast<floatx4*>(&red[wave][n][16 * i + 4 * g]) = o[i];
  __syncthreads();

  // sum over the waves, in wave order, each scaled to the chunk's maximum
  for (int e = tid; e < rows * DH; e += 64 * NW) {
    const int i = e / DH, col = e % DH, r = rt * 16 + i;
    float mw[NW], M = -INFINITY, L = 0.f, s = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      mw[w] = ml[w][i][0];
      M = fmaxf(M, mw[w]);
    }
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      // (a wave whose every score was NaN has no maximum, but NaN sums: 0 times them is NaN)
      const float wgt = mw[w] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[w] - M);
      L = __builtin_fmaf(wgt, ml[w][i][1], L);
      s = __builtin_fmaf(wgt, red[w][i][col], s);
    }
    if (a.n_chunks == 1) {
      static_cast<bf16*>(a.out)[(static_cast<int64_t>(b) * a.n_new + r % a.n_new) * d +
                                (h * G + r / a.n_new) * static_cast<int64_t>(DH) + col] = static_cast<bf16>(s * (1.f / L));
    } else {
      const int64_t pr = (head * R + r) * a.n_chunks + chunk;
      a.part_o[pr * DH + col] = s;
      if (col == 0) {
        a.part_ml[pr * 2] = M;
        a.part_ml[pr * 2 + 1] = L;
      }
    }
  }
}

// W waves per (sequence, query head, new row) merge the chunks its keys fill: each
// every W-th, 16 at once so that their partial rows are all in flight; then the
// waves' sums, in their order.
template <int DH, int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void ld_attn_decode_kv8_combine(Kv8AttnArgs a) {
  constexpr int CL = DH / 64, U = 16;
  typedef float FRow __attribute__((ext_vector_type(CL)));
  __shared__ float ml[W][2];
  __shared__ __align__(16) FRow red[W][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = W == 1 ? static_cast<int64_t>(blockIdx.x) * 4 + wave : blockIdx.x;
  if (r >= static_cast<int64_t>(a.kv.n_seq) * a.H * a.n_new) return;
  const int w = W == 1 ? 0 : wave;
  const int G = a.H / a.kv.KV, R = G * a.n_new;
  const int64_t head = r / R, b = head / a.kv.KV;
  const int i = static_cast<int>(r % R), h = static_cast<int>(head % a.kv.KV) * G + i / a.n_new, j = i % a.n_new;
  int p = a.pos;
  if (a.seq_pos) {
    p = a.seq_pos[b];
    if (p < 0 || p > a.pos) p = -a.n_new;
  }
  const int chunks = (p + a.n_new + a.chunk_keys - 1) / a.chunk_keys;
  const float* po = a.part_o + r * a.n_chunks * DH + lane * CL;
  const float* pm = a.part_ml + r * a.n_chunks * 2;
  float M = -INFINITY, L = 0.f;
  FRow acc = 0.f;
  for (int c0 = w; c0 < chunks; c0 += U * W) {
    FRow v[U];
    float mc[U], lc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // past the last chunk: the last again, dropped below
      const int64_t c = min(c0 + u * W, chunks - 1);
      v[u] = *reinterpret_cast<const FRow*>(po + c * DH);
      mc[u] = pm[c * 2];
      lc[u] = pm[c * 2 + 1];
    }
    __builtin_amdgcn_sched_barrier(0);
    float m = M;
#pragma unroll
    for (int u = 0; u < U; ++u) m = fmaxf(m, mc[u]);
    const float keep = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - m);
    L *= keep;
    acc *= keep;
    M = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = c0 + u * W < chunks;  // else selected out: 0 times an infinity in v would be NaN
      const float wgt = !in || mc[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc[u] - m);
      L = __builtin_fmaf(wgt, in ? lc[u] : 0.f, L);
      acc += wgt * (in ? v[u] : FRow(0.f));
    }
  }
  if constexpr (W > 1) {
    if (lane == 0) {
      ml[w][0] = M;
      ml[w][1] = L;
    }
    red[w][lane] = acc;
    __syncthreads();
    if (w) return;
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < W; ++u) m = fmaxf(m, ml[u][0]);
    L = 0.f;
    acc = 0.f;
#pragma unroll
    for (int u = 0; u < W; ++u) {
      const float wgt = ml[u][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[u][0] - m);
      L = __builtin_fmaf(wgt, ml[u][1], L);
      acc += wgt * red[u][lane];
    }
  }
  if (chunks > 0) acc *= 1.f / L;
  bf16* out = static_cast<bf16*>(a.out) + (b * a.n_new + j) * (static_cast<int64_t>(a.H) * DH) +
              static_cast<int64_t>(h) * DH + lane * CL;
#pragma unroll
  for (int cc = 0; cc < CL; ++cc) out[cc] = static_cast<bf16>(acc[cc]);
}

template <int DH, int FMT>
hipError_t store_t(const Kv8StoreArgs& a, hipStream_t s) {
  const int tt = a.kv.block > 64 ? 128 : 64;
  // tiles of any sequence: from the one that holds its first row
  const int64_t tiles = a.seq_pos ? (static_cast<int64_t>(a.n) + tt - 2) / tt + 1
                                  : (static_cast<int64_t>(a.pos) + a.n - 1) / tt - a.pos / tt + 1;
  const dim3 grid(tiles, 2 * a.kv.KV, a.kv.n_seq);
  if (tt == 64)
    hipLaunchKernelGGL((ld_kv8_store_k<DH, FMT, 64>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((ld_kv8_store_k<DH, FMT, 128>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int DH, int FMT>
hipError_t load_t(const Kv8LoadArgs& a, hipStream_t s) {
  const dim3 grid((static_cast<int64_t>(a.pos) + a.n - 1) / 64 - a.pos / 64 + 1, 2 * a.kv.KV, a.kv.n_seq);
  hipLaunchKernelGGL((ld_kv8_load_k<DH, FMT>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int DH, int FMT>
hipError_t attn_t(const Kv8AttnArgs& a, hipStream_t s) {
  const int R = a.H / a.kv.KV * a.n_new;
  const dim3 grid(a.n_chunks, a.kv.KV * ((R + 15) / 16), a.kv.n_seq), block(64 * kKv8Waves);
  if (R == 1)
    hipLaunchKernelGGL((ld_attn_decode_kv8_k<DH, FMT, 1>), grid, block, 0, s, a);
  else if (R <= 8)
    hipLaunchKernelGGL((ld_attn_decode_kv8_k<DH, FMT, 8>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((ld_attn_decode_kv8_k<DH, FMT, 16>), grid, block, 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_chunks == 1) return e;
  const int64_t rows = static_cast<int64_t>(a.kv.n_seq) * a.H * a.n_new;
  if (a.n_chunks > 8 && rows <= 8192)
    hipLaunchKernelGGL((ld_attn_decode_kv8_combine<DH, 8>), dim3(rows), dim3(512), 0, s, a);
  else
    hipLaunchKernelGGL((ld_attn_decode_kv8_combine<DH, 1>), dim3((rows + 3) / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv8_store(const Kv8StoreArgs& a, hipStream_t s) {
  if (a.kv.dh == 128)
    return a.kv.format == LD_KV8_E4M3 ? store_t<128, LD_KV8_E4M3>(a, s) : store_t<128, LD_KV8_INT8>(a, s);
  return a.kv.format == LD_KV8_E4M3 ? store_t<64, LD_KV8_E4M3>(a, s) : store_t<64, LD_KV8_INT8>(a, s);
}

hipError_t launch_kv8_load(const Kv8LoadArgs& a, hipStream_t s) {
  if (a.kv.dh == 128)
    return a.kv.format == LD_KV8_E4M3 ? load_t<128, LD_KV8_E4M3>(a, s) : load_t<128, LD_KV8_INT8>(a, s);
  return a.kv.format == LD_KV8_E4M3 ? load_t<64, LD_KV8_E4M3>(a, s) : load_t<64, LD_KV8_INT8>(a, s);
}

namespace {
constexpr int64_t kKv8MinChunk = 512, kKv8RaggedWgs = 16 * kCus;
}

// Keys of a chunk, for `heads` (sequence, head, 16 rows).  Lengths that the host
// knows: what costs least, rounds of one workgroup per CU, each its keys and
// about 128 more, and a second launch like 500.  Otherwise (`ragged`, keys being
// the longest a sequence can have) about 16 workgroups a CU, so that whatever the
// lengths are spreads evenly.
int64_t attn_kv8_chunk(int64_t heads, int64_t keys, bool ragged) {
  const int64_t most = keys <= 1024 ? 1 : keys / kKv8MinChunk;
  int64_t best = 1;
  if (ragged) {
    best = (kKv8RaggedWgs + heads - 1) / heads;
    if (best > most) best = most;
  } else {
    int64_t best_cost = INT64_MAX;
    for (int64_t n = 1; n <= most && (n == 1 || heads * (n - 1) < 4 * kCus); ++n) {
      const int64_t cost = (heads * n + kCus - 1) / kCus * ((keys + n - 1) / n + 128) + (n > 1 ? 500 : 0);
      if (cost < best_cost) {
        best = n;
        best_cost = cost;
      }
    }
  }
  return ((keys + best - 1) / best + 63) / 64 * 64;
}

int64_t attn_kv8_max_chunks(int64_t heads, int64_t keys) {
  const int64_t by_keys = (keys + kKv8MinChunk - 1) / kKv8MinChunk, by_wgs = (kKv8RaggedWgs + heads - 1) / heads;
  return by_keys < by_wgs ? by_keys : by_wgs;
}

hipError_t launch_attn_decode_kv8(Kv8AttnArgs a, hipStream_t s) {
  const int64_t keys = static_cast<int64_t>(a.pos) + a.n_new;
  const int64_t R = static_cast<int64_t>(a.H / a.kv.KV) * a.n_new;
  const int64_t heads = static_cast<int64_t>(a.kv.n_seq) * a.kv.KV * ((R + 15) / 16);
  a.chunk_keys = static_cast<int32_t>(attn_kv8_chunk(heads, keys, a.seq_pos != nullptr));
  a.n_chunks = static_cast<int32_t>((keys + a.chunk_keys - 1) / a.chunk_keys);
  if (a.kv.dh == 128)
    return a.kv.format == LD_KV8_E4M3 ? attn_t<128, LD_KV8_E4M3>(a, s) : attn_t<128, LD_KV8_INT8>(a, s);
  return a.kv.format == LD_KV8_E4M3 ? attn_t<64, LD_KV8_E4M3>(a, s) : attn_t<64, LD_KV8_INT8>(a, s);
}

}  // namespace ld
