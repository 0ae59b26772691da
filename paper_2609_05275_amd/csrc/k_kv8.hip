// Kernels of the 8-bit key/value cache: quantising writer, reader, and the
// attention of a few new rows per sequence over it.  Layout and the meaning of
// codes and scales: Kv8View in ld_kv8.h, ld_kv8 in layerdrop.h.
//
// Scales are powers of two, so dividing by one and multiplying with it are
// exact: a code is one rounding of its value, a value read back is the code's
// in bf16 without another, and raising a block's scale rounds old codes by a
// whole number of bits.
#include "ld_kv8.h"

namespace ld {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kKv8Waves = 8;  // of an attention workgroup
constexpr int kKv8Parts = 3;  // bf16 parts of a weight, 8 of its 24 bits each
constexpr int kCus = 256;

// ------------------------------------------------------------- conversions

// 8 codes (two dwords) to bf16, exact: e4m3 has 4 significant bits, int8 seven.
// With a scale (a power of two; e4m3 only) times it.
template <int FMT>
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t a, uint32_t b, float scale = 1.f) {
  union {
    bf16x8 v;
    bf16x2 p[4];
    uint32_t u[4];
  } r;
  if constexpr (FMT == LD_KV8_E4M3) {
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
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

// Four dwords of four bytes, transposed.
__device__ __forceinline__ void transpose4(const uint32_t (&in)[4], uint32_t (&out)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(in[1], in[0], 0x05010400u), b = __builtin_amdgcn_perm(in[1], in[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(in[3], in[2], 0x05010400u), d = __builtin_amdgcn_perm(in[3], in[2], 0x07030602u);
  out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// ---------------------------------------------------------- store and load

// A wave takes a unit of U = 16 positions (32 for heads of 64) of one head's keys or
// values.  Lane l has dimensions 8 (l % PT) .. + 7, PT = DH / 8 lanes a row, of rows
// 4 (l / PT) + i, i < 4: four neighbouring positions, so that a 4x4 byte transpose in
// registers turns between rows and the values' tiles, and a load or store
// instruction still takes whole rows.  A tile's 16 bytes of a dimension come from
// four lanes and meet in LDS (rows of 16 bytes, 16 more after each 8: the lanes'
// dwords fall on different banks).
//
// Bound by memory.  Prompts of 8 x 2048 rows, 16 heads of 128: store 34 to 37 us for
// 201 MB (5.4 to 5.9 TB/s, a large copy's rate being 4.9; units of 64 positions a wave,
// four times fewer waves, 44.9, and loads that stay in the caches 41.2), load 30 us
// (6.7 TB/s, the codes still in the memory-side cache; stores that push them out 39.9).
// Load of 4 x 4096 rows of 32 heads: 78 us for 403 MB (5.1 TB/s).  A new row of 32
// sequences: 5.9 us, its value bytes alone (16 lines a head); whole tiles read and
// written 6.9.  One row of one sequence: 3.8 us, a launch and four dependent accesses.
template <int DH>
struct Kv8Lanes {
  static constexpr int PT = DH / 8, U = 4 * 64 / PT, TILES = U / 16;  // a unit: U rows, TILES tiles
  static constexpr int TILE_LDS = DH * 16 + DH * 2;                   // bytes
  static __device__ __forceinline__ int lds_row(int d) { return d * 16 + (d >> 3) * 16; }
};

// Piece number -> (sequence, piece of it, head, part), heads and parts first:
// neighbours read neighbouring columns of the same rows.
struct Kv8Unit {
  int b, piece, h, part;
};
__device__ __forceinline__ uint32_t kv8_workgroup() { return blockIdx.y * gridDim.x + blockIdx.x; }  // see kv8_grid
__device__ __forceinline__ Kv8Unit kv8_unit(uint32_t id, uint32_t KV, uint32_t pieces) {
  const uint32_t head = id >> 1, at = head / KV;
  return Kv8Unit{static_cast<int>(at / pieces), static_cast<int>(at % pieces), static_cast<int>(head % KV),
                 static_cast<int>(id & 1)};
}

// A workgroup of W waves takes a piece of W U positions (whole blocks) of one
// head's keys or values, a wave a unit; the waves of a block exchange their maxima.
template <int DH, int FMT, int W>
__global__ __launch_bounds__(64 * W) void ld_kv8_store_k(Kv8StoreArgs a) {
  using LN = Kv8Lanes<DH>;
  constexpr int PT = LN::PT, U = LN::U, PP = U * W;
  __shared__ __align__(16) uint8_t lds[W][LN::TILES * LN::TILE_LDS];
  __shared__ uint32_t mu_s[W];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Kv8View& c = a.kv;
  const Kv8Unit w = kv8_unit(kv8_workgroup(), c.KV, a.pieces);
  if (w.b >= c.n_seq) return;
  int p = a.pos;
  if (a.seq_pos) {
    p = a.seq_pos[w.b];
    if (p < 0 || p > a.pos) return;
  }
  const int lo = p, hi = p + a.n, p0 = (p / PP + w.piece) * PP;
  if (p0 >= hi) return;
  const int f = p0 + U * wave;  // the wave's unit
  const int grp = lane / PT, d8 = lane % PT * 8;
  const int64_t head = static_cast<int64_t>(w.b) * c.KV + w.h;
  uint8_t* codes = c.codes + (head * 2 + w.part) * c.s16 * DH;
  float* scales = c.scales + (head * 2 + w.part) * c.nb;
  // the first block may hold earlier rows: its scale can only rise
  const int first = (max(lo, p0) >> c.shift) << c.shift;
  const bool goes_on = first < lo;
  const float old = goes_on ? scales[first >> c.shift] : 0.f;
  const bf16* src = static_cast<const bf16*>(a.qkv) + static_cast<int64_t>(w.b) * a.n * a.ld_qkv +
                    (a.H + w.part * c.KV + w.h) * static_cast<int64_t>(DH) + d8;

  union Row {
    bf16x8 v;
    ushortx2 u[4];
  };
  Row v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = f + 4 * grp + i;
    v[i].v = static_cast<bf16>(0.f);
    if (t >= lo && t < hi)
      v[i].v = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(src + static_cast<int64_t>(t - lo) * a.ld_qkv));
  }

  // largest absolute value of the lane's block, as bf16 bits
  ushortx2 m2{0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) m2 = __builtin_elementwise_max(m2, v[i].u[e] & static_cast<unsigned short>(0x7fff));
  uint32_t mu = max(m2[0], m2[1]);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    if (x == 32 && c.block < U) break;  // two blocks of 16 in a unit of 32: half a wave each
    mu = max(mu, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mu), x, 64)));
  }
  if (c.block > U) {
    if (lane == 0) mu_s[wave] = mu;
    __syncthreads();
    const int of = c.block / U, w0 = wave / of * of;
    mu = 0;
#pragma unroll
    for (int x = 0; x < W; ++x) mu = max(mu, x >= w0 && x < w0 + of ? mu_s[x] : 0u);
  }
  const int blk = (f + 4 * grp) >> c.shift, bf = blk << c.shift;  // the lane's block
  float s = scale_needed<FMT>(mu), ratio = 1.f;                   // ratio < 1: earlier rows are rounded again
  if (goes_on && bf == first) {
    if (s == s && !(old <= s)) s = old;
    if (old < s) ratio = old / s;
  }
  if (lane % (64 / LN::TILES) == 0 && bf == f + 16 * (lane / 32) && bf < hi && bf + c.block > lo) scales[blk] = s;
  const float inv = s == s ? 1.f / s : 0.f;  // 0 for NaN: such a block's codes are zeros
  const bool again = __any(ratio < 1.f);
  if (c.block < U) ratio = fminf(ratio, __shfl_xor(ratio, 32, 64));
  const int from = again ? first : lo;
  if (f >= hi || f + U <= from) return;

  uint32_t q[4][2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = inv != 0.f ? static_cast<float>(v[i].v[e]) * inv : 0.f;
    q[i][0] = pack_codes<FMT>(x[0], x[1], x[2], x[3]);
    q[i][1] = pack_codes<FMT>(x[4], x[5], x[6], x[7]);
  }
  if (w.part == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = f + 4 * grp + i;
      u32x2* at = reinterpret_cast<u32x2*>(codes + static_cast<int64_t>(t) * DH + d8);
      if (t >= lo && t < hi) {
        *at = u32x2{q[i][0], q[i][1]};
      } else if (t >= from && t < lo) {
        const u32x2 r = *at;
        *at = u32x2{rescale4<FMT>(r[0], ratio), rescale4<FMT>(r[1], ratio)};
      }
    }
    return;
  }
  if (!again && a.n < 16) {  // no whole tile: the new bytes alone
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = f + 4 * grp + i;
      if (t < lo || t >= hi) continue;
      uint8_t* at = codes + static_cast<int64_t>(t & ~15) * DH + d8 * 16 + (t & 15);
#pragma unroll
      for (int e = 0; e < 8; ++e) at[16 * e] = static_cast<uint8_t>(q[i][e >> 2] >> (8 * (e & 3)));
    }
    return;
  }
  uint8_t* tile = lds[wave] + (LN::TILES == 2 ? (grp >> 2) * LN::TILE_LDS : 0);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint32_t in[4] = {q[0][e], q[1][e], q[2][e], q[3][e]};
    uint32_t out[4];
    transpose4(in, out);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint32_t*>(tile + LN::lds_row(d8 + 4 * e + i) + 4 * (grp & 3)) = out[i];
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int d = (lane + 64 * i) % DH, x = (lane + 64 * i) / DH, ft = f + 16 * x;
    if (ft >= hi || ft + 16 <= from) continue;
    u32x4* at = reinterpret_cast<u32x4*>(codes + static_cast<int64_t>(ft) * DH + d * 16);
    u32x4 r = *reinterpret_cast<const u32x4*>(lds[wave] + x * LN::TILE_LDS + LN::lds_row(d));
    if (ft < lo || ft + 16 > hi) {  // the other positions' bytes stay (rounded again)
      u32x4 was = *at;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t mask = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (ft + 4 * k + e >= lo && ft + 4 * k + e < hi) mask |= 0xffu << (8 * e);
        if (again) was[k] = rescale4<FMT>(was[k], ratio);
        r[k] = (r[k] & mask) | (was[k] & ~mask);
      }
    }
    *at = r;
  }
}

// A wave takes a unit, lanes as in the store.  The rows written are not read here
// again: stored past the caches, they leave the codes in them.
template <int DH, int FMT>
__global__ __launch_bounds__(256) void ld_kv8_load_k(Kv8LoadArgs a) {
  using LN = Kv8Lanes<DH>;
  constexpr int PT = LN::PT, U = LN::U;
  __shared__ __align__(16) uint8_t lds[4][LN::TILES * LN::TILE_LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Kv8View& c = a.kv;
  const Kv8Unit w = kv8_unit(kv8_workgroup() * 4 + wave, c.KV, a.pieces);
  if (w.b >= c.n_seq) return;
  const int f = (a.pos / U + w.piece) * U;
  int hi = a.pos + a.n;
  if (a.seq_len) hi = min(hi, a.seq_len[w.b]);
  if (f >= hi) return;
  const int grp = lane / PT, d8 = lane % PT * 8, t0 = f + 4 * grp;
  const int64_t head = static_cast<int64_t>(w.b) * c.KV + w.h;
  const uint8_t* codes = c.codes + (head * 2 + w.part) * c.s16 * DH;
  const float s = t0 < hi ? c.scales[(head * 2 + w.part) * c.nb + (t0 >> c.shift)] : 0.f;
  uint32_t q[4][2];
  if (w.part == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x2 r{0, 0};
      if (t0 + i >= a.pos && t0 + i < hi) r = *reinterpret_cast<const u32x2*>(codes + static_cast<int64_t>(t0 + i) * DH + d8);
      q[i][0] = r[0];
      q[i][1] = r[1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int d = (lane + 64 * i) % DH, x = (lane + 64 * i) / DH, ft = f + 16 * x;
      u32x4 r{0, 0, 0, 0};
      if (ft < hi) r = *reinterpret_cast<const u32x4*>(codes + static_cast<int64_t>(ft) * DH + d * 16);
      *reinterpret_cast<u32x4*>(lds[wave] + x * LN::TILE_LDS + LN::lds_row(d)) = r;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const uint8_t* tile = lds[wave] + (LN::TILES == 2 ? (grp >> 2) * LN::TILE_LDS : 0);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint32_t in[4], out[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        in[i] = *reinterpret_cast<const uint32_t*>(tile + LN::lds_row(d8 + 4 * e + i) + 4 * (grp & 3));
      transpose4(in, out);
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i][e] = out[i];
    }
  }
  const int64_t ld = 2ll * c.KV * DH;
  bf16* out = static_cast<bf16*>(a.out) + static_cast<int64_t>(w.b) * a.n * ld +
              (static_cast<int64_t>(w.part) * c.KV + w.h) * DH + d8;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + i;
    if (t < a.pos || t >= hi) continue;
    bf16x8 v = codes_to_bf16<FMT>(q[i][0], q[i][1]);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<bf16>(static_cast<float>(v[e]) * s);
    __builtin_nontemporal_store(v, reinterpret_cast<bf16x8*>(out + (t - a.pos) * ld));
  }
}

// --------------------------------------------------------------- attention

// Keys of a chunk of a sequence of nk: a.chunk_keys, and where lengths are the device's
// more in a sequence that would make more than a.n_chunks of them.
__device__ __forceinline__ int kv8_chunk_keys(const Kv8AttnArgs& a, int nk) {
  if (!a.seq_pos) return a.chunk_keys;
  const uint32_t n = a.n_chunks, even = ((static_cast<uint32_t>(nk) + n - 1) / n + 63) & ~63u;
  return max(static_cast<int>(even), a.chunk_keys);
}

// A workgroup of eight waves takes a chunk of keys of one key/value head for 16
// rows (of its query heads' new rows); a wave 32 keys at a time (64 for heads of
// 64), with its own running maximum and sum; they meet once, to add up.
//
// Scores S^T = K Q^T and output O^T = V^T P^T on the matrix cores (16x16x32
// bf16).  The A rows of score product t are the keys LK g + 4 t + r (row 4 g + r), LK =
// 8 (16), so lane group g = lane / 16 of the result holds keys LK g + 4 t + r, r < 4, of
// its query row: LK neighbouring keys, half a tile (a tile) of the cache's values,
// of one scale.  They are the B operand of O^T as they stand, and LK bytes of a
// value tile's row the A operand.
//
// Codes are exact in bf16.  A probability, times its value scale, goes in as three
// bf16 parts, which are all of its 24 bits (parts below 2^-126, 2^-26 of the
// smallest scale, may be lost).  Two parts take 0.1 to 1.0 us less (a verify step
// 14.6 us against 15.2, the ragged batch below 47.1 against 48.0, 131072 keys 94.4
// against 94.9), but leave up to 2^-17 of it: seven bits of values that cancel.
//
// Bound by the cache stream.  A wave asks for its keys and values at once (8 KB)
// and waits; 16 waves a CU at 128 registers hold 128 KB in flight.  131072 keys of 8
// heads of 128, 2 sequences: 537 MB in 91 us (5.9 TB/s; reading alone reaches 6.2);
// 4096 keys of 32 heads of 8: 268 MB in 46.9 us (5.7); 16 sequences of up to 8192, 276
// MB in 51.6 us (5.3: launch, tail).  Short chunks are start and end: 256 workgroups of
// 64, 256, 512 and 753 keys (six rows, int8) 5.3, 7.8, 10.0 and 12.8 us in a graph, so
// that each 256 keys more cost 2.3 to 2.8 us (7.3 to 6.0 TB/s, the cache partly in the
// memory-side cache) after 5.3 for the first.  Tried, with weights in two parts: 16
// waves a workgroup, 1506 keys of 16 heads of 8 in two chunks 14.5 -> 14.9 us; the next
// turn's keys asked for before this one's products (the queries then in LDS), 2 to 9%
// faster where every chunk is long, the ragged batch 57.9 -> 72.8; two row tiles a
// workgroup, 8 rows of 8 query heads a head 17.1 -> 21.4.
template <int DH, int FMT, int NQ>
__global__ __launch_bounds__(64 * kKv8Waves, 4) void ld_attn_decode_kv8_k(Kv8AttnArgs a) {
  constexpr int NS = DH / 64, MT = DH / 16, NW = kKv8Waves, TT = DH == 64 ? 4 : 2, LK = 4 * TT, WK = 16 * TT;
  __shared__ float ml[NW][NQ][2];
  __shared__ __align__(16) float red[NW][NQ][DH];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const Kv8View& c = a.kv;
  // Workgroups go round the 8 XCDs by their number.  Chunks are turned by the
  // head, or a number of chunks that shares a factor with the XCDs' would leave
  // those of the last chunks, which short sequences do not fill, with little to do.
  // Several row tiles: a sequence's (head, chunk) go in sets of 8, a set's tiles one
  // after the other, so that a chunk's tiles read it through one L2 at about one time.
  const int b = blockIdx.z;
  int h = blockIdx.y, chunk = blockIdx.x, r0 = 0;  // r0: the workgroup's first row
  if (a.tiles > 1) {
    const uint32_t nc = a.n_chunks, units = c.KV * nc, set = blockIdx.x / (8 * a.tiles), of = blockIdx.x % (8 * a.tiles);
    const uint32_t n8 = min(units - 8 * set, 8u), unit = 8 * set + of % n8;
    h = __builtin_amdgcn_readfirstlane(unit / nc);
    chunk = __builtin_amdgcn_readfirstlane(unit % nc);
    r0 = __builtin_amdgcn_readfirstlane(of / n8 * 16);
  }
  chunk = (chunk + h + b) % a.n_chunks;
  const int G = a.group, R = G * a.n_new;
  int p = a.pos;
  if (a.seq_pos) {
    p = a.seq_pos[b];
    if (p < 0 || p > a.pos) p = -a.n_new;  // left out: no keys
  }
  const int nk = p + a.n_new, ck = kv8_chunk_keys(a, nk), k_first = chunk * ck;
  const int rows = min(R - r0, 16);
  const int64_t d = static_cast<int64_t>(a.H) * DH;
  // where row r of the head goes in the output
  auto out_at = [&](uint32_t r) {
    return static_cast<bf16*>(a.out) + (static_cast<int64_t>(b) * a.n_new + r % static_cast<uint32_t>(a.n_new)) * d +
           (h * G + r / static_cast<uint32_t>(a.n_new)) * static_cast<int64_t>(DH);
  };
  if (k_first >= nk) {
    if (chunk == 0)  // left out: its rows are zeros
      for (int e = tid; e < rows * DH; e += 64 * NW) out_at(r0 + e / DH)[e % DH] = static_cast<bf16>(0.f);
    return;
  }
  const int k_end = min(k_first + ck, nk);
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

  const uint32_t row = r0 + min(n, rows - 1), j = row % static_cast<uint32_t>(a.n_new);
  const int qh = h * G + row / static_cast<uint32_t>(a.n_new), qpos = p + j;
  bf16x8 qf[NS][2];
  {
    const bf16* q = static_cast<const bf16*>(a.qkv) + (static_cast<int64_t>(b) * a.n_new + j) * a.ld_qkv +
                    static_cast<int64_t>(qh) * DH;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int e = 0; e < 2; ++e) qf[s][e] = *reinterpret_cast<const bf16x8*>(q + 64 * s + 16 * g + 8 * e);
  }
  const float al2 = a.alibi ? alibi_slope(qh, a.H) * kLog2e : 0.f, sl2 = a.scale * kLog2e;

  float m = -INFINITY, l = 0.f;
  floatx4 o[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};

  for (int k0 = k_first + wave * WK; k0 < k_end; k0 += WK * NW) {
    load_keys(k0);
    load_values(k0);
    __builtin_amdgcn_sched_barrier(0);
    const int f = k0 + LK * g;  // the lane's keys
    float ss = sk * sl2;        // of a product to a base-2 score
    floatx4 x[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      x[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16<FMT>(kr[t][s][0], kr[t][s][1]), qf[s][0], x[t], 0, 0, 0);
        x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16<FMT>(kr[t][s][2], kr[t][s][3]), qf[s][1], x[t], 0, 0, 0);
      }
    }
    if (a.alibi) {
      const float far = al2 * static_cast<float>(qpos - f);
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          x[t][r] = __builtin_fmaf(x[t][r], ss, __builtin_fmaf(al2, static_cast<float>(4 * t + r), -far));
      ss = 1.f;
    }
    const bool cut = k0 + WK - 1 > p;  // some of the keys may be behind a row, or behind the last one
    if (cut) {
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (f + 4 * t + r > qpos) x[t][r] = -INFINITY;
    }
    // the largest score: of the lane's products (their scale is positive), then of all
    float mn = x[0][0];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mn = fmaxf(mn, x[t][r]);
    mn = fmaxf(m, mn * ss);
    mn = fmaxf(mn, __shfl_xor(mn, 16, 64));
    mn = fmaxf(mn, __shfl_xor(mn, 32, 64));
    const float mz = mn == -INFINITY ? 0.f : mn;  // of nothing but -inf, whose weights are 0
    if (__any(mn != m)) {
      const float keep = __builtin_amdgcn_exp2f(m - mz);
      l *= keep;
#pragma unroll
      for (int i = 0; i < MT; ++i) o[i] *= keep;
    }
    m = mn;
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        x[t][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][r], ss, -mz));  // of a NaN score NaN
    if (cut) {  // a masked position's key scale may be NaN
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (f + 4 * t + r > qpos) x[t][r] = 0.f;
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) l += x[t][r];
    // Times the value scale, which e4m3 takes with the values' conversion.  Masked
    // positions must not see NaN, nor values that become infinite by it: such a
    // scale goes with the weights.
    const bool bad = !(sv < 0x1p119f);
    const float sv1 = bad ? 1.f : sv;
    if constexpr (FMT == LD_KV8_INT8) {
#pragma unroll
      for (int t = 0; t < TT; ++t) x[t] *= sv1;
    }
    if (__any(bad)) {
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (bad && f + 4 * t + r <= qpos) x[t][r] *= sv;
    }
    bf16x8 pw[kKv8Parts][TT / 2];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        floatx2 w{x[t][r], x[t][r + 1]};
#pragma unroll
        for (int i = 0; i < kKv8Parts; ++i) {
          const bf16x2 part = __builtin_convertvector(w, bf16x2);
          const uint32_t pb = __builtin_bit_cast(uint32_t, part);
          w -= floatx2{__builtin_bit_cast(float, pb << 16), __builtin_bit_cast(float, pb & 0xffff0000u)};
          pw[i][t >> 1][4 * (t & 1) + r] = part[0];
          pw[i][t >> 1][4 * (t & 1) + r + 1] = part[1];
        }
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
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int u = 0; u < TT / 2; ++u) {
        const bf16x8 v8 = codes_to_bf16<FMT>(vr[i][2 * u], vr[i][2 * u + 1], sv1);
#pragma unroll
        for (int part = 0; part < kKv8Parts; ++part)
          o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, pw[part][u], o[i], 0, 0, 0);
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
  const bool only = nk <= ck;  // the sequence's one chunk: its rows are the result
  for (int e = tid; e < rows * DH; e += 64 * NW) {
    const int i = e / DH, col = e % DH, r = r0 + i;
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
    if (only) {
      out_at(r)[col] = static_cast<bf16>(s * (1.f / L));
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

// W (four or one) waves per (sequence, query head, new row) merge the chunks its keys
// fill, where they are several: each every W-th, U at once so that their partial
// rows are all in flight; then the waves' sums, in their order.  Bound by two
// dependent loads and, with many rows, by reading the partial rows.  A launch of its
// own, 2.5 to 3.1 us of a call in a graph (with and without it: 15.2 and 12.8, 93.5 and
// 91.0, 57.0 and 54.0); the last workgroup of a row doing it instead needs
// device-scope release and acquire, which write back and empty the XCDs' L2s (a
// verify step over 1506 keys 15.2 -> 44 us).
template <int DH, int W>
__global__ __launch_bounds__(256) void ld_attn_decode_kv8_combine(Kv8AttnArgs a) {
  constexpr int CL = DH / 64, U = 4;
  typedef float FRow __attribute__((ext_vector_type(CL)));
  __shared__ float ml[W][2];
  __shared__ __align__(16) FRow red[W][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t id = W == 1 ? blockIdx.x * 4 + wave : blockIdx.x, HN = a.H * a.n_new;
  if (id >= a.kv.n_seq * HN) return;
  const int w = W == 1 ? 0 : wave;
  const int64_t r = id, b = id / HN;
  const uint32_t h = id % HN / a.n_new, j = id % a.n_new;  // (HN is a multiple of n_new)
  int chunks = a.n_chunks;
  if (a.seq_pos) {
    const int p = a.seq_pos[b], nk = p < 0 || p > a.pos ? 0 : p + a.n_new, ck = kv8_chunk_keys(a, nk);
    chunks = (nk + ck - 1) / ck;
  }
  if (chunks <= 1) return;  // written by the attention kernel
  const float* po = a.part_o + r * a.n_chunks * DH + lane * CL;
  const floatx2* pm = reinterpret_cast<const floatx2*>(a.part_ml) + r * a.n_chunks;
  float M = -INFINITY, L = 0.f;
  FRow acc = 0.f;
  for (int c0 = w; c0 < chunks; c0 += U * W) {
    FRow v[U];
    float mc[U], lc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // past the last chunk: the last again, dropped below
      const int64_t c = min(c0 + u * W, chunks - 1);
      v[u] = *reinterpret_cast<const FRow*>(po + c * DH);
      const floatx2 x = pm[c];
      mc[u] = x[0];
      lc[u] = x[1];
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
  acc *= 1.f / L;
  bf16* out = static_cast<bf16*>(a.out) + (b * a.n_new + j) * (static_cast<int64_t>(a.H) * DH) +
              static_cast<int64_t>(h) * DH + lane * CL;
#pragma unroll
  for (int cc = 0; cc < CL; ++cc) out[cc] = static_cast<bf16>(acc[cc]);
}

// Workgroups in two dimensions: one takes 2^32 threads at most.
dim3 kv8_grid(int64_t wgs) {
  constexpr int64_t kX = 1 << 20;
  return wgs <= kX ? dim3(wgs) : dim3(kX, (wgs + kX - 1) / kX);
}

template <int DH, int FMT>
hipError_t store_t(Kv8StoreArgs a, hipStream_t s) {
  constexpr int U = Kv8Lanes<DH>::U;
  const int waves = a.kv.block > 4 * U ? 8 : 4, pp = waves * U;
  // pieces of any sequence: from the one that holds its first row
  a.pieces = static_cast<int32_t>(a.seq_pos ? (static_cast<int64_t>(a.n) + pp - 2) / pp + 1
                                            : (static_cast<int64_t>(a.pos) + a.n - 1) / pp - a.pos / pp + 1);
  const int64_t wgs = 2ll * a.kv.KV * a.kv.n_seq * a.pieces;
  if (waves == 4)
    hipLaunchKernelGGL((ld_kv8_store_k<DH, FMT, 4>), kv8_grid(wgs), dim3(256), 0, s, a);
  else if constexpr (DH == 128)
    hipLaunchKernelGGL((ld_kv8_store_k<DH, FMT, 8>), kv8_grid(wgs), dim3(512), 0, s, a);
  return hipGetLastError();
}

template <int DH, int FMT>
hipError_t load_t(Kv8LoadArgs a, hipStream_t s) {
  constexpr int U = Kv8Lanes<DH>::U;
  a.pieces = static_cast<int32_t>((static_cast<int64_t>(a.pos) + a.n - 1) / U - a.pos / U + 1);
  const int64_t units = 2ll * a.kv.KV * a.kv.n_seq * a.pieces;
  hipLaunchKernelGGL((ld_kv8_load_k<DH, FMT>), kv8_grid((units + 3) / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int DH, int FMT>
hipError_t attn_t(const Kv8AttnArgs& a, hipStream_t s) {
  const int R = a.group * a.n_new;
  const dim3 block(64 * kKv8Waves);
  const dim3 grid = a.tiles == 1 ? dim3(a.n_chunks, a.kv.KV, a.kv.n_seq)
                                 : dim3(a.kv.KV * a.n_chunks * a.tiles, 1, a.kv.n_seq);
  // rows kept for the merge: less LDS and, where workgroups are few, less time at the
  // end (16 heads over 8000 keys: 11.3 us with 1, 11.5 with 8, 12.1 with 16)
  if (R == 1)
    hipLaunchKernelGGL((ld_attn_decode_kv8_k<DH, FMT, 1>), grid, block, 0, s, a);
  else if (R <= 8)
    hipLaunchKernelGGL((ld_attn_decode_kv8_k<DH, FMT, 8>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((ld_attn_decode_kv8_k<DH, FMT, 16>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <int DH>
hipError_t combine_t(const Kv8AttnArgs& a, hipStream_t s) {
  const int64_t rows = static_cast<int64_t>(a.kv.n_seq) * a.H * a.n_new;
  // Four waves a row, or one where there is little to share or the rows fill the chip
  // by themselves.  Us of a call with one, four: 16 rows of 12 chunks 9.6, 8.4; 512 of 8
  // 14.9, 14.2; 2048 of 14 34.4, 33.6; 4096 of 8 39.8, 39.8; 512 of 4 17.3, 17.4; 2048 of 4
  // 16.2, 16.6; 10240 of 2 56.5, 58.9.
  if (a.n_chunks > 4 && rows <= 2048)
    hipLaunchKernelGGL((ld_attn_decode_kv8_combine<DH, 4>), dim3(rows), dim3(256), 0, s, a);
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

int64_t attn_kv8_heads(const Kv8View& kv, int64_t H, int64_t n_new) {
  const int64_t R = H / kv.KV * n_new;
  return static_cast<int64_t>(kv.n_seq) * kv.KV * ((R + 15) / 16);
}

namespace {

constexpr int64_t kKv8MinChunk = 256, kKv8ShortKeys = 1024, kKv8UnevenChunk = 576, kKv8FewChunk = 320,
                  kKv8UnevenWgs = 2048;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Chunks of a head's keys where the host knows the lengths: what costs least, in
// ns.  Workgroups come to the CUs in rounds of 256, and it takes 3 us to change
// over.  In a full round a CU gets its share of 6 TB/s (of twice and two and a half
// times that where two or more row tiles read a chunk through one L2); in the last,
// more the fewer there are, up to the 36 (int8: 28) bytes a ns that one workgroup
// takes in on its own.  Several chunks are a second launch, counted as 3.5 us, and as
// no less than 6 us together with the first, the host's time for two.  That floor
// keeps one chunk where a call's own time is all there is to gain (16 heads over
// 777 keys 8.1 us at 1 and at 4 chunks called one by one, but 8.3 and 7.6 in a graph).
// us at n chunks, in a graph: 24 heads of 128 over 43825 keys 48.8 at 8, 50 to 56 at 10
// to 96; 140 heads over 3682 30.3 at 1, 32 at 3 to 14; 120 over 4321, int8, 28.6 at 2, 30
// to 31 at 4 to 16; 24 over 1217, six rows, int8, 14.3 at 1, 11.5 at 2, 9.5 at 4; 16 over
// 1000, int8, 11.3 at 1, 8.0 at 4; 32 over 600 7.25 at 1, 7.7 at 3; 16 of 64 of 3
// sequences over 13181 with 40 rows 48 at 1, 36.5 at 4, 32.3 at 5.
int64_t chunks_known(const Kv8AttnArgs& a, int64_t heads, int64_t keys) {
  const int64_t most = div_up(keys, kKv8MinChunk), lone = a.kv.format == LD_KV8_INT8 ? 28 : 36;
  const int64_t host = 6000, twice = a.tiles > 2 ? 5 : 2 * a.tiles;  // 2 x tiles that share a reading
  int64_t best = 1, best_cost = INT64_MAX;
  for (int64_t n = 1; n <= most && (n == 1 || heads * (n - 1) < 4 * kCus); ++n) {
    const int64_t bytes = div_up(keys, n) * 2 * a.kv.dh, wgs = heads * n, rest = wgs % kCus;
    int64_t cost = wgs / kCus * (2 * bytes * kCus / (6000 * twice)) + (div_up(wgs, kCus) - 1) * 3000;
    if (rest) cost += bytes / (lone * rest < 3000 * twice ? lone : 3000 * twice / rest);
    if (n > 1) cost = cost + 3500 > host ? cost + 3500 : host;
    if (cost < best_cost) {
      best = n;
      best_cost = cost;
    }
  }
  return best;
}

// Where it does not (keys being the most a sequence can have): for one sequence, or
// up to 1024 keys, as many as if all had that many, of at least 256 keys.  Else chunks
// of about 576 keys, so that
// whatever the lengths are spreads evenly, shorter ones where those would be few (8
// heads of 5 sequences up to 8235, int8: 13.2 us with 384 keys, 15.7 with 1088), and at
// most 2048 workgroups, long sequences' chunks growing instead: most of a full grid
// would find nothing to do, and each costs its start.  Us without that limit and
// with it (1536 and 2560): 32 heads of 16 sequences of up to 8192 keys 58.9, 55.6 (60.9,
// 57.6), all under 900 22.8, 19.2 (15.4, 17.9); 8 heads of 64 up to 4000 47.0, 43.9 (44.3,
// 44.3); with 32 rows a head (two tiles) 32 of 16 up to 8000 82.6, 55.2 (62.4, 54.6), 16
// of 64 up to 2000 105, 71.1 (71.1, 71.1); 32 of 32 up to 3000, int8, 67.9, 70.6, the one
// that loses.
void chunks_uneven(Kv8AttnArgs& a, int64_t heads, int64_t keys) {
  int64_t n, least = kKv8MinChunk;
  if (keys <= kKv8ShortKeys || a.kv.n_seq == 1) {
    n = chunks_known(a, heads, keys);
  } else {
    const int64_t by_wgs = 4 * kCus / heads, by_keys = keys / kKv8FewChunk, few = by_wgs < by_keys ? by_wgs : by_keys;
    n = div_up(keys, kKv8UnevenChunk);
    if (n < few) n = few;
    least = div_up(div_up(keys, n), 64) * 64;
  }
  const int64_t most = heads < kKv8UnevenWgs ? kKv8UnevenWgs / heads : 1;
  a.n_chunks = static_cast<int32_t>(n < most ? n : most);
  a.chunk_keys = static_cast<int32_t>(least);
}

}  // namespace

int64_t attn_kv8_max_chunks(int64_t heads, int64_t keys) {
  const int64_t by_keys = div_up(keys, kKv8MinChunk), by_wgs = div_up(kKv8UnevenWgs, heads);
  return by_keys < by_wgs ? by_keys : by_wgs;
}

void plan_attn_decode_kv8(Kv8AttnArgs& a) {
  const int64_t keys = static_cast<int64_t>(a.pos) + a.n_new;
  a.group = a.H / a.kv.KV;
  a.tiles = (a.group * a.n_new + 15) / 16;
  const int64_t heads = attn_kv8_heads(a.kv, a.H, a.n_new);
  if (a.seq_pos) {
    chunks_uneven(a, heads, keys);
  } else {
    a.chunk_keys = static_cast<int32_t>(div_up(div_up(keys, chunks_known(a, heads, keys)), 64) * 64);
    a.n_chunks = static_cast<int32_t>(div_up(keys, a.chunk_keys));
  }
}

hipError_t launch_attn_decode_kv8(const Kv8AttnArgs& a, hipStream_t s) {
  if (a.kv.dh == 128)
    return a.kv.format == LD_KV8_E4M3 ? attn_t<128, LD_KV8_E4M3>(a, s) : attn_t<128, LD_KV8_INT8>(a, s);
  return a.kv.format == LD_KV8_E4M3 ? attn_t<64, LD_KV8_E4M3>(a, s) : attn_t<64, LD_KV8_INT8>(a, s);
}

hipError_t launch_attn_decode_kv8_combine(const Kv8AttnArgs& a, hipStream_t s) {
  return a.kv.dh == 128 ? combine_t<128>(a, s) : combine_t<64>(a, s);
}

}  // namespace ld
