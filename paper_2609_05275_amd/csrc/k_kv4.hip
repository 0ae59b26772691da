// Kernels of the 4-bit key/value cache: quantising writer, reader, the attention
// of a few new rows per sequence over it with the positions' summed weights, and
// the eviction by those.  Layout and the meaning of codes and scales: Kv4View in
// ld_kv4.h, ld_kv4 in layerdrop.h.
//
// A code is a 4-bit float (sign, two bits of exponent, one of mantissa), its scale a
// power of two for 32 neighbouring dimensions of one position.  Both are what
// v_cvt_scalef32_pk_bf16_fp4 takes: two codes to two bf16, exact, in one instruction.
#include "ld_kv4.h"

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
constexpr int kKv4Waves = 8;  // of an attention workgroup
constexpr int kKv4Turn = 32 * kKv4Waves;  // keys of a turn of an attention workgroup
constexpr int kKv4Parts = 3;  // bf16 parts of a weight, 8 of its 24 bits each
constexpr uint32_t kNanScale = 255;
constexpr int kKv4MaxExp = 125;  // 6 2^125 is finite

// ------------------------------------------------------------- conversions

// Two codes of byte B times a scale, of which the conversion looks at the exponent alone: a
// scale's byte may be shifted there with its neighbours' bits where sign and mantissa are.
template <int B>
__device__ __forceinline__ bf16x2 pair_of(uint32_t w, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B);
}

// Eight codes of one scale.
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t w, float scale) {
  union {
    bf16x8 v;
    bf16x2 p[4];
  } r;
  r.p[0] = pair_of<0>(w, scale);
  r.p[1] = pair_of<1>(w, scale);
  r.p[2] = pair_of<2>(w, scale);
  r.p[3] = pair_of<3>(w, scale);
  return r.v;
}

// Eight values divided by a scale, to codes: nearest, ties to even, 6 at most.
__device__ __forceinline__ uint32_t bf16_to_codes(bf16x8 v, float scale) {
  union {
    bf16x8 v;
    bf16x2 p[4];
  } x;
  x.v = v;
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x.p[0], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x.p[1], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x.p[2], scale, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, x.p[3], scale, 3);
  return r;
}

// The scale's byte that a largest absolute value (bf16 bits) needs.
__device__ __forceinline__ uint32_t scale_needed(uint32_t amax) {
  if (amax >= 0x7f80u) return kNanScale;
  // 6 = 1.5 2^2
  const int e = static_cast<int>(amax >> 7) - 127 - 2 + ((amax & 0x7fu) > 0x40u ? 1 : 0);
  return static_cast<uint32_t>(min(max(e, kKv4MinExp), kKv4MaxExp) + 127);  // zeros and subnormals too
}

// The low 16 bits' nibbles to bytes.
__device__ __forceinline__ uint32_t spread4(uint32_t x) {
  x = (x | (x << 8)) & 0x00ff00ffu;
  return (x | (x << 4)) & 0x0f0f0f0fu;
}
// Bytes' low nibbles to the low 16 bits.
__device__ __forceinline__ uint32_t gather4(uint32_t x) {
  x &= 0x0f0f0f0fu;
  x = (x | (x >> 4)) & 0x00ff00ffu;
  return (x | (x >> 8)) & 0xffffu;
}

// ---------------------------------------------------------- store and load

// A wave takes a unit of U = 8 positions (16 for heads of 64) of one head's keys or
// values.  Lane l has dimensions 16 (l % PT) .. + 15 of row l / PT, PT = DH / 16: half a
// scale's dimensions, so that a neighbour holds the other nibbles of its values' bytes.
// Values change places in LDS, a tile's bytes going out together where all of its positions
// are new; a token appended writes its bytes one by one.
//
// Bound by memory, in small calls by the launch: 1501 rows each of 3 sequences, 8 heads of 128,
// store 6.5 us traced (23 MB, 3.6 TB/s), both 11.7; a row each of 32 sequences of 16 heads 6.4
// together.  What the load writes goes past the caches, in whole lines (both calls 11.7 us, in
// half lines 12.9, through the caches 13.2; 131072 positions of 8 heads cut to 16384 and read
// 56.5, 64.2, 66.7); rows loaded past them by the store cost 0.7 (in whole
// lines, lanes holding dimensions DH / 2 apart, 11.6, but the appended rows 6.7).
template <int DH>
struct Kv4Lanes {
  static constexpr int PT = DH / 16, U = 64 / PT, TILES = U / 8, TB = DH * 4;  // TB: bytes of a tile of 8 values
};

struct Kv4Unit {
  int b, piece, h, part;
};
__device__ __forceinline__ uint32_t kv4_workgroup() { return blockIdx.y * gridDim.x + blockIdx.x; }  // see kv4_grid
// Piece number -> (sequence, piece of it, head, part), heads and parts first:
// neighbours read neighbouring columns of the same rows.
__device__ __forceinline__ Kv4Unit kv4_unit(uint32_t id, uint32_t KV, uint32_t pieces) {
  const uint32_t head = id >> 1, at = head / KV;
  return Kv4Unit{static_cast<int>(at / pieces), static_cast<int>(at % pieces), static_cast<int>(head % KV),
                 static_cast<int>(id & 1)};
}

template <int DH>
__global__ __launch_bounds__(256) void ld_kv4_store_k(Kv4StoreArgs a) {
  using LN = Kv4Lanes<DH>;
  constexpr int PT = LN::PT, U = LN::U, TB = LN::TB, JN = DH / 32;
  __shared__ __align__(16) uint8_t lds[4][LN::TILES * TB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Kv4View& c = a.kv;
  const Kv4Unit w = kv4_unit(kv4_workgroup() * 4 + wave, c.KV, a.pieces);
  if (w.b >= c.n_seq) return;
  int lo = a.pos;
  if (a.seq_pos) {
    lo = a.seq_pos[w.b];
    if (lo < 0 || lo > a.pos) return;
  }
  const int hi = lo + a.n, f = (lo / U + w.piece) * U;
  if (f >= hi) return;
  const int row = lane / PT, c16 = lane % PT, j = c16 >> 1, half = c16 & 1, t = f + row;
  const bool in = t >= lo && t < hi;
  const int64_t head = static_cast<int64_t>(w.b) * c.KV + w.h;
  uint8_t* codes = c.codes + (head * 2 + w.part) * c.s8 * (DH / 2);
  uint8_t* scales = c.scales + (head * 2 + w.part) * c.s8 * JN;

  union Row {
    bf16x8 v;
    ushortx2 u[4];
  } v[2];
  v[0].v = v[1].v = static_cast<bf16>(0.f);
  if (in) {
    const bf16* src = static_cast<const bf16*>(a.qkv) + (static_cast<int64_t>(w.b) * a.n + t - lo) * a.ld_qkv +
                      (a.H + w.part * c.KV + w.h) * static_cast<int64_t>(DH) + 16 * c16;
    v[0].v = *reinterpret_cast<const bf16x8*>(src);
    v[1].v = *reinterpret_cast<const bf16x8*>(src + 8);
  }
  ushortx2 m2{0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) m2 = __builtin_elementwise_max(m2, v[i].u[e] & static_cast<unsigned short>(0x7fff));
  uint32_t mu = max(m2[0], m2[1]);
  mu = max(mu, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mu), 1, 64)));
  const uint32_t sb = scale_needed(mu);
  const float s = __builtin_bit_cast(float, sb << 23);
  // (a block of NaN scale: its codes are zeros)
  uint32_t q0 = sb == kNanScale ? 0u : bf16_to_codes(v[0].v, s), q1 = sb == kNanScale ? 0u : bf16_to_codes(v[1].v, s);
  if (in && half == 0) scales[static_cast<int64_t>(t) * JN + j] = static_cast<uint8_t>(sb);
  if (w.part == 0) {
    if (in) {
      *reinterpret_cast<u32x2*>(codes + static_cast<int64_t>(t) * (DH / 2) + 8 * c16) = u32x2{q0, q1};
      if (c.sums && c16 == 0) c.sums[head * c.s_max + t] = 0.f;
    }
    return;
  }
  // bytes n = 8 half + i: the even lane's dimension in the low nibble, the odd one's in the high
  const uint32_t got = static_cast<uint32_t>(__shfl_xor(static_cast<int>(half ? q0 : q1), 1, 64));
  const uint32_t ln = half ? got : q0, hn = half ? q1 : got;
  const uint32_t b0 = spread4(ln & 0xffffu) | spread4(hn & 0xffffu) << 4, b1 = spread4(ln >> 16) | spread4(hn >> 16) << 4;
  const int at = (row & 7) + 8 * j + 8 * half * 8 * JN;  // of byte 0 in its tile
  const int tile = row >> 3, t0 = f + 8 * tile;
  uint8_t* tb = codes + static_cast<int64_t>(t0 >> 3) * TB;
  if (t0 < lo || t0 + 8 > hi) {  // no whole tile: the new bytes alone
    if (in) {
#pragma unroll
      for (int i = 0; i < 8; ++i) tb[at + i * 8 * JN] = static_cast<uint8_t>((i < 4 ? b0 : b1) >> (8 * (i & 3)));
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) lds[wave][tile * TB + at + i * 8 * JN] = static_cast<uint8_t>((i < 4 ? b0 : b1) >> (8 * (i & 3)));
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int tw = lane * 8 / TB, w0 = f + 8 * tw;  // the lane's tile of the way out
  if (w0 >= lo && w0 + 8 <= hi)
    *reinterpret_cast<u32x2*>(codes + static_cast<int64_t>(w0 >> 3) * TB + lane * 8 % TB) =
        *reinterpret_cast<const u32x2*>(&lds[wave][lane * 8]);
}

// A wave takes a unit, lanes as in the store.
template <int DH>
__global__ __launch_bounds__(256) void ld_kv4_load_k(Kv4LoadArgs a) {
  using LN = Kv4Lanes<DH>;
  constexpr int PT = LN::PT, U = LN::U, TB = LN::TB, JN = DH / 32;
  __shared__ __align__(16) uint8_t lds[4][LN::TILES * TB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Kv4View& c = a.kv;
  const Kv4Unit w = kv4_unit(kv4_workgroup() * 4 + wave, c.KV, a.pieces);
  if (w.b >= c.n_seq) return;
  const int f = (a.pos / U + w.piece) * U;
  int hi = a.pos + a.n;
  if (a.seq_len) hi = min(hi, a.seq_len[w.b]);
  if (f >= hi) return;
  const int row = lane / PT, c16 = lane % PT, j = c16 >> 1, half = c16 & 1, t = f + row;
  const bool in = t >= a.pos && t < hi;
  const int64_t head = static_cast<int64_t>(w.b) * c.KV + w.h;
  const uint8_t* codes = c.codes + (head * 2 + w.part) * c.s8 * (DH / 2);
  const uint8_t* scales = c.scales + (head * 2 + w.part) * c.s8 * JN;
  const uint32_t sb = in ? scales[static_cast<int64_t>(t) * JN + j] : 0u;
  uint32_t q0 = 0, q1 = 0;
  if (w.part == 0) {
    if (in) {
      const u32x2 r = *reinterpret_cast<const u32x2*>(codes + static_cast<int64_t>(t) * (DH / 2) + 8 * c16);
      q0 = r[0];
      q1 = r[1];
    }
  } else {
    u32x2 r{0, 0};
    if (f + 8 * (lane * 8 / TB) < hi) r = *reinterpret_cast<const u32x2*>(codes + static_cast<int64_t>(f >> 3) * TB + lane * 8);
    *reinterpret_cast<u32x2*>(&lds[wave][lane * 8]) = r;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const uint8_t* at = &lds[wave][(row >> 3) * TB + (row & 7) + 8 * j + 8 * half * 8 * JN];
    uint32_t b0 = 0, b1 = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      b0 |= static_cast<uint32_t>(at[i * 8 * JN]) << (8 * i);
      b1 |= static_cast<uint32_t>(at[(i + 4) * 8 * JN]) << (8 * i);
    }
    const uint32_t ln = gather4(b0) | gather4(b1) << 16, hn = gather4(b0 >> 4) | gather4(b1 >> 4) << 16;
    const uint32_t got = static_cast<uint32_t>(__shfl_xor(static_cast<int>(half ? ln : hn), 1, 64));
    q0 = half ? got : ln;
    q1 = half ? hn : got;
  }
  if (!in) return;
  const int64_t ld = 2ll * c.KV * DH;
  bf16* out = static_cast<bf16*>(a.out) + (static_cast<int64_t>(w.b) * a.n + t - a.pos) * ld +
              (static_cast<int64_t>(w.part) * c.KV + w.h) * DH + 8 * c16;
  // a row's lanes write its first half, then its second: whole lines
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int from = lane - c16 + i * (PT / 2) + (c16 >> 1);
    const uint32_t e0 = __shfl(static_cast<int>(q0), from, 64), e1 = __shfl(static_cast<int>(q1), from, 64);
    const float s = __builtin_bit_cast(float, static_cast<uint32_t>(__shfl(static_cast<int>(sb), from, 64)) << 23);
    __builtin_nontemporal_store(codes_to_bf16(c16 & 1 ? e1 : e0, s), reinterpret_cast<bf16x8*>(out + 8 * i * PT));
  }
}

// --------------------------------------------------------------- attention

// Keys of a chunk of a sequence of nk: a.chunk_keys, and where lengths are the device's
// a.chunk_keys at least.
__device__ __forceinline__ int kv4_chunk_keys(const Kv4AttnArgs& a, int nk) {
  if (!a.seq_pos) return a.chunk_keys;
  const uint32_t n = a.n_chunks, even = ((static_cast<uint32_t>(nk) + n - 1) / n + kKv4Turn - 1) & ~(kKv4Turn - 1u);
  return max(static_cast<int>(even), a.chunk_keys);
}

// Keys of a sequence (0: left out), and the chunks they fill.
__device__ __forceinline__ int kv4_keys(const Kv4AttnArgs& a, int64_t b) {
  if (!a.seq_pos) return a.pos + a.n_new;
  const int p = a.seq_pos[b];
  return p < 0 || p > a.pos ? 0 : p + a.n_new;
}
__device__ __forceinline__ int kv4_chunks(const Kv4AttnArgs& a, int nk) {
  const int ck = kv4_chunk_keys(a, nk);
  return (nk + ck - 1) / ck;
}

// A weight's bf16 parts, TT / 2 operands of 8 positions each.
template <int TT>
struct Kv4Parts {
  bf16x8 p[kKv4Parts][TT / 2];
  __device__ __forceinline__ void split(const floatx4 (&x)[TT]) {
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        floatx2 w{x[t][r], x[t][r + 1]};
#pragma unroll
        for (int i = 0; i < kKv4Parts; ++i) {
          const bf16x2 part = __builtin_convertvector(w, bf16x2);
          const uint32_t pb = __builtin_bit_cast(uint32_t, part);
          w -= floatx2{__builtin_bit_cast(float, pb << 16), __builtin_bit_cast(float, pb & 0xffff0000u)};
          p[i][t >> 1][4 * (t & 1) + r] = part[0];
          p[i][t >> 1][4 * (t & 1) + r + 1] = part[1];
        }
      }
  }
};

// A workgroup of eight waves takes a chunk of keys of one key/value head for 16
// rows (of its query heads' new rows); a wave 32 keys at a time, with its own running
// maximum and sum; they meet once, to add up.
//
// Scores S^T = K Q^T and output O^T = V^T P^T on the matrix cores, 16x16x32 products in bf16.
// A lane has 16 bytes of a key, one scale's 32 dimensions (heads of 64: 8 bytes): a dword becomes
// the 8 dimensions of a product's first operand, and lane group g = lane / 16 of product step s
// takes dimensions 32 g + 8 s .. + 7 (64: 32 (g & 1) + 16 (g >> 1) + 8 s .. + 7), the queries
// likewise.  (Scaled 16x16x128 products take codes and scales as they lie, but add 8 neighbouring
// products to 13 bits below the largest of them alone, where float32 sums keep 24.)  Row 4 g + r of
// score product t is key 8 g + 4 t + r, so a lane group of the results holds 8 neighbouring keys of
// its query row, whole tiles of the cache's values: they are the second operand of O^T as they
// stand.
//
// Values are converted in pairs of dimensions, which share position and scale, and put
// together over positions by byte permutes.  A probability goes in as three bf16 parts,
// which are all of its 24 bits (two: 3% less time, 2^-17 of a weight lost).
//
// What bounds it: the chain of a turn, about 260 vector and 32 matrix instructions that wait
// for each other and for memory, which the four waves of a SIMD hide in part: over the long
// case below vector units are 0.52 and matrix units 0.24 busy, a fifth fewer vector
// instructions (scaled score products) took 2% less time, and caches that the last-level cache
// holds 10% less.  So the registers are kept to four waves of a SIMD (more loads in flight with
// two were slower), the maximum is renewed only where it has to be, and NaN is looked for only in
// turns that masks cut.  2 sequences of 131072 keys, 32 heads over 8 of 128 dimensions: 58 us, 4.9
// TB/s of the cache (the sums rescaled each turn 75).  16 uneven sequences of 32 heads, 68000
// keys in all: 42 us.
template <int DH, int NQ>
__global__ __launch_bounds__(64 * kKv4Waves, 4) void ld_attn_decode_kv4_k(Kv4AttnArgs a) {
  constexpr int JN = DH / 32, MT = DH / 16, NW = kKv4Waves, TT = 2, LK = 4 * TT, WK = 16 * TT;
  constexpr int VT = LK / 8, TB = DH * 4;  // value tiles a lane group; bytes of one
  constexpr int KD = DH / 32;              // dwords of a key a lane, steps of the score product
  __shared__ float ml[NW][NQ][2];
  __shared__ __align__(16) float red[NW][NQ][DH];
  __shared__ __align__(16) bf16x8 qs[KD][64];  // the queries as operands (in registers they would not fit)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const Kv4View& c = a.kv;
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
  const int nk = kv4_keys(a, b), p = nk - a.n_new, ck = kv4_chunk_keys(a, nk), k_first = chunk * ck;
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
  const uint8_t* kc = c.codes + head * c.s8 * DH;
  const uint8_t* vc = kc + static_cast<int64_t>(c.s8) * (DH / 2);
  const uint8_t* ks = c.scales + head * 2 * c.s8 * JN;
  const uint8_t* vs = ks + static_cast<int64_t>(c.s8) * JN;

  // Keys k0 .. k0 + WK - 1 (past the last key: key 0, masked later): row n of
  // product t.
  const int krow = LK * (n >> 2) + (n & 3);
  typedef uint32_t VRaw __attribute__((ext_vector_type(4)));
  typedef uint32_t SRaw __attribute__((ext_vector_type(2 * JN)));
  typedef uint32_t KRaw __attribute__((ext_vector_type(KD)));
  KRaw kr[TT];
  uint32_t sk[TT];
  union {
    VRaw q[JN / 2];
    uint32_t d[JN][2];  // [dimensions 32 j + n and 32 j + 16 + n][positions 0-3, 4-7]
  } vr[VT];
  union {
    SRaw q;
    uint32_t d[2 * JN];
  } sv[VT];  // [position][j] bytes
  // (a wave's turn is where its scalar base is; what a lane adds does not change)
  const uint32_t kg = g & (JN - 1), kb = 16 * kg + (DH == 64 ? 8 * (g >> 1) : 0);  // the lane's scale; its bytes of a key
  const uint32_t k_at = krow * (DH / 2) + kb, ks_at = krow * JN + kg;
  const uint32_t v_at = LK / 8 * g * TB + n * (8 * JN), vs_at = LK * g * JN;
  auto load_keys = [&](int k0) {
    if (k0 + WK <= nk) {
      const uint8_t *kf = kc + static_cast<int64_t>(k0) * (DH / 2), *ksf = ks + static_cast<int64_t>(k0) * JN;
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        kr[t] = *reinterpret_cast<const KRaw*>(kf + (k_at + 4 * t * (DH / 2)));
        sk[t] = ksf[ks_at + 4 * t * JN];
      }
    } else {
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        int kk = k0 + krow + 4 * t;
        kk = kk < nk ? kk : 0;
        kr[t] = *reinterpret_cast<const KRaw*>(kc + static_cast<int64_t>(kk) * (DH / 2) + kb);
        sk[t] = ks[static_cast<int64_t>(kk) * JN + kg];
      }
    }
  };
  auto load_values = [&](int k0) {
    if (k0 + WK <= nk) {
      const uint8_t *vb = vc + static_cast<int64_t>(k0) * (DH / 2), *vsb = vs + static_cast<int64_t>(k0) * JN;
#pragma unroll
      for (int v = 0; v < VT; ++v) {
#pragma unroll
        for (int i = 0; i < JN / 2; ++i) vr[v].q[i] = *reinterpret_cast<const VRaw*>(vb + (v_at + v * TB + 16 * i));
        sv[v].q = *reinterpret_cast<const SRaw*>(vsb + (vs_at + 8 * v * JN));
      }
    } else {
#pragma unroll
      for (int v = 0; v < VT; ++v) {
        const int f = k0 + LK * g + 8 * v, fc = f < nk ? f : 0;
        const uint8_t* at = vc + static_cast<int64_t>(fc >> 3) * TB + n * (8 * JN);
#pragma unroll
        for (int i = 0; i < JN / 2; ++i) vr[v].q[i] = *reinterpret_cast<const VRaw*>(at + 16 * i);
        sv[v].q = *reinterpret_cast<const SRaw*>(vs + static_cast<int64_t>(fc) * JN);
      }
    }
  };

  const uint32_t row = r0 + min(n, rows - 1), j = row % static_cast<uint32_t>(a.n_new);
  const int qh = h * G + row / static_cast<uint32_t>(a.n_new), qpos = p + j;
  int k0 = k_first + wave * WK;
  if (k0 < k_end) {
    load_keys(k0);
    load_values(k0);
  }
  if (wave < KD)
    qs[wave][lane] = *reinterpret_cast<const bf16x8*>(static_cast<const bf16*>(a.qkv) + (static_cast<int64_t>(b) * a.n_new + j) * a.ld_qkv +
                                                      static_cast<int64_t>(qh) * DH + 2 * kb + 8 * wave);
  const float al2 = a.alibi ? alibi_slope(qh, a.H) * kLog2e : 0.f, sl2 = a.scale * kLog2e;

  // The scores are taken from a reference m, the largest score when it was last set: weights
  // stay below 2^kSlack, and sums are scaled to a new one only when a score passes that.
  constexpr float kSlack = 8.f;
  float m = -INFINITY, mz = 0.f, l = 0.f;  // mz: m, or 0 where there is none
  floatx4 o[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};

  // dimensions 32 jj .. + 31 of the output: values in pairs of dimensions, put together
  // over positions
  auto add_values = [&](int jj, const Kv4Parts<TT>& pw) {
    bf16x8 lo[VT], hi[VT];
#pragma unroll
    for (int v = 0; v < VT; ++v) {
      bf16x2 pr[8];
      auto scale = [&](int q) {  // of position q, as the conversions take it
        const uint32_t w = sv[v].d[q * JN / 4];
        const int byte = q * JN % 4 + jj;
        return __builtin_bit_cast(float, byte == 0 ? w << 23 : byte == 1 ? w << 15 : byte == 2 ? w << 7 : w >> 1);
      };
      pr[0] = pair_of<0>(vr[v].d[jj][0], scale(0));
      pr[1] = pair_of<1>(vr[v].d[jj][0], scale(1));
      pr[2] = pair_of<2>(vr[v].d[jj][0], scale(2));
      pr[3] = pair_of<3>(vr[v].d[jj][0], scale(3));
      pr[4] = pair_of<0>(vr[v].d[jj][1], scale(4));
      pr[5] = pair_of<1>(vr[v].d[jj][1], scale(5));
      pr[6] = pair_of<2>(vr[v].d[jj][1], scale(6));
      pr[7] = pair_of<3>(vr[v].d[jj][1], scale(7));
      u32x4 a0, a1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t e = __builtin_bit_cast(uint32_t, pr[2 * i]), f = __builtin_bit_cast(uint32_t, pr[2 * i + 1]);
        a0[i] = __builtin_amdgcn_perm(f, e, 0x05040100u);
        a1[i] = __builtin_amdgcn_perm(f, e, 0x07060302u);
      }
      lo[v] = __builtin_bit_cast(bf16x8, a0);
      hi[v] = __builtin_bit_cast(bf16x8, a1);
    }
#pragma unroll
    for (int v = 0; v < VT; ++v)
#pragma unroll
      for (int part = 0; part < kKv4Parts; ++part) {
        o[2 * jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo[v], pw.p[part][v], o[2 * jj], 0, 0, 0);
        o[2 * jj + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi[v], pw.p[part][v], o[2 * jj + 1], 0, 0, 0);
      }
  };

  __syncthreads();
  while (k0 < k_end) {
    asm volatile("" ::: "memory");  // the queries are read each turn
    const int f = k0 + LK * g;  // the lane's keys
    float ss = sl2;             // of a product to a base-2 score
    floatx4 x[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) x[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < KD; ++st) {
      const bf16x8 q = qs[st][lane];
#pragma unroll
      for (int t = 0; t < TT; ++t)
        x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_bf16(kr[t][st], __builtin_bit_cast(float, sk[t] << 23)), q, x[t], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (k0 + WK * NW < k_end) load_keys(k0 + WK * NW);  // (the values' when these are used)
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
#pragma unroll
      for (int v = 0; v < VT; ++v) {
        const int have = nk - f - 8 * v;  // positions of this tile; what is behind them may be anything
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int of = have - 4 * u;
          const uint32_t mask = of <= 0 ? 0u : of >= 4 ? ~0u : (1u << (8 * of)) - 1u;
#pragma unroll
          for (int i = 0; i < JN; ++i) vr[v].d[i][u] &= mask;
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          constexpr uint32_t one = JN == 4 ? 0x7f7f7f7fu : 0x7f7fu, full = JN == 4 ? ~0u : 0xffffu;
          const int at = q * JN / 4, sh = q * JN % 4 * 8;
          if (q >= have) sv[v].d[at] = (sv[v].d[at] & ~(full << sh)) | (one << sh);
        }
      }
      // Masked positions must not see NaN: here it goes to the rows that see its position,
      // and the scale becomes one.
#pragma unroll 1
      for (int jj = 0; jj < JN; ++jj) {
        int first = INT32_MAX;
#pragma unroll
        for (int v = 0; v < VT; ++v)
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int at = q * JN / 4, sh = (q * JN % 4 + jj) * 8;
            if (((sv[v].d[at] >> sh) & 255u) == kNanScale) {
              first = min(first, f + 8 * v + q);
              sv[v].d[at] ^= 0x80u << sh;
            }
          }
        if (__any(first != INT32_MAX)) {
          first = min(first, __shfl_xor(first, 16, 64));
          first = min(first, __shfl_xor(first, 32, 64));
          const float nan = first <= qpos ? __builtin_nanf("") : 0.f;
#pragma unroll
          for (int i = 0; i < MT; ++i)
            if (i >> 1 == jj) o[i] += nan;
        }
      }
    }
    if (a.scores && n < rows) {
      float* sc = a.scores + (head * R + r0 + n) * a.score_keys + f;
#pragma unroll
      for (int t = 0; t < TT; ++t) *reinterpret_cast<floatx4*>(sc + 4 * t) = x[t] * ss;
    }
    // the largest of the lane's scores (their scale is positive)
    float mx = x[0][0];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[t][r]);
    mx *= ss;
    if (__any(mx > m + kSlack)) {
      mx = fmaxf(m, mx);
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      mz = mx == -INFINITY ? 0.f : mx;  // of nothing but -inf, whose weights are 0
      const float keep = __builtin_amdgcn_exp2f(m - mz);
      l *= keep;
#pragma unroll
      for (int i = 0; i < MT; ++i) o[i] *= keep;
      m = mx;
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[t][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][r], ss, -mz));  // of a NaN score NaN
        l += x[t][r];
      }
    __builtin_amdgcn_sched_barrier(0);
    Kv4Parts<TT> pw;
    pw.split(x);
#pragma unroll
    for (int jj = 0; jj < JN; ++jj) {
      add_values(jj, pw);
      __builtin_amdgcn_sched_barrier(0);  // (else all conversions go first, and spill)
    }
    k0 += WK * NW;
    if (k0 < k_end) load_values(k0);
    __builtin_amdgcn_sched_barrier(0);
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
    const int64_t pr = (head * R + r) * a.n_chunks + chunk;
    if (only)
      out_at(r)[col] = static_cast<bf16>(s * (1.f / L));
    else
      a.part_o[pr * DH + col] = s;
    if (col == 0 && (!only || a.scores)) {
      a.part_ml[pr * 2] = M;
      a.part_ml[pr * 2 + 1] = L;
    }
  }
}

// W (four or one) waves per (sequence, query head, new row) merge the chunks its keys
// fill, where they are several: each every W-th, U at once so that their partial
// rows are all in flight; then the waves' sums, in their order.  A launch that waits: 2 to 3
// us of a call, whatever the case.
template <int DH, int W>
__device__ __forceinline__ void combine_rows(const Kv4AttnArgs& a, uint32_t block) {
  constexpr int CL = DH / 64, U = 4;
  typedef float FRow __attribute__((ext_vector_type(CL)));
  __shared__ float ml[W][2];
  __shared__ __align__(16) FRow red[W][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t id = W == 1 ? block * 4 + wave : block, HN = a.H * a.n_new;
  if (id >= a.kv.n_seq * HN) return;
  const int w = W == 1 ? 0 : wave;
  const int64_t r = id, b = id / HN;
  const uint32_t h = id % HN / a.n_new, j = id % a.n_new;  // (HN is a multiple of n_new)
  const int chunks = kv4_chunks(a, kv4_keys(a, b));
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

// sums += the weights of a head's rows, a thread four positions, rows in their order: the
// weights need the rows' norms, which are known when all chunks are done, so the scores go
// through memory.  The norms of 256 rows at a time are found first, a row by 16 lanes.
constexpr int kSumKeys = 1024;  // of a workgroup
__device__ __forceinline__ void add_sums(const Kv4AttnArgs& a, uint32_t block) {
  __shared__ float norm[256][2];
  const uint32_t tiles = (static_cast<uint32_t>(a.pos) + a.n_new + kSumKeys - 1) / kSumKeys;
  const int64_t head = block / tiles;
  if (head >= static_cast<int64_t>(a.kv.n_seq) * a.kv.KV) return;
  const int tid = threadIdx.x, b = static_cast<int>(head / a.kv.KV), R = a.group * a.n_new;
  const int nk = kv4_keys(a, b), p = nk - a.n_new, t0 = block % tiles * kSumKeys, t = t0 + 4 * tid, chunks = kv4_chunks(a, nk);
  if (t0 >= nk) return;
  const float* sc = a.scores + head * R * a.score_keys + (t < nk ? t : 0);
  floatx4 s = 0.f, next = *reinterpret_cast<const floatx4*>(sc);
  for (int r0 = 0; r0 < R; r0 += 256) {
    const int rows = min(R - r0, 256);
    if (r0) __syncthreads();
    for (int i = tid >> 4; i < rows; i += 16) {
      const floatx2* ml = reinterpret_cast<const floatx2*>(a.part_ml) + (head * R + r0 + i) * a.n_chunks;
      float M = -INFINITY, L = 0.f;
      for (int c = tid & 15; c < chunks; c += 16) {
        const floatx2 x = ml[c];
        const float m = fmaxf(M, x[0]);
        // (a part whose every score was NaN has no maximum, but a NaN sum)
        L = L * (M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - m)) +
            x[1] * (x[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[0] - m));
        M = m;
      }
      float m = M;
#pragma unroll
      for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d, 64));
      L *= M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - m);
#pragma unroll
      for (int d = 1; d < 16; d *= 2) L += __shfl_xor(L, d, 64);
      if ((tid & 15) == 0) {
        norm[i][0] = m;
        norm[i][1] = 1.f / L;
      }
    }
    __syncthreads();
    for (int i = 0; i < rows; ++i) {
      const int r = r0 + i, last = p + r % a.n_new;
      const floatx4 x = next;
      next = *reinterpret_cast<const floatx4*>(sc + min(r + 1, R - 1) * a.score_keys);
#pragma unroll
      for (int u = 0; u < 4; ++u)  // (a masked position counts nothing, whatever the row holds)
        s[u] += t + u > last ? 0.f : __builtin_amdgcn_exp2f(x[u] - norm[i][0]) * norm[i][1];
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (t + u < nk) a.kv.sums[head * a.kv.s_max + t + u] += s[u];
}

// Joins chunks, in the first `blocks` workgroups, and adds to the sums in those behind: one
// launch for both (two: 2 us more).
template <int DH, int W>
__global__ __launch_bounds__(256) void ld_attn_decode_kv4_combine(Kv4AttnArgs a, uint32_t blocks) {
  const uint32_t id = kv4_workgroup();
  if (id < blocks)
    combine_rows<DH, W>(a, id);
  else
    add_sums(a, id - blocks);
}

// Over one chunk: its rows are the result.  (6 rows of 8 sequences' 16 heads at 1506 keys, with
// the joining of two chunks: 4.6 MB of scores, 5.6 us traced.)
__global__ __launch_bounds__(256) void ld_kv4_sums_k(Kv4AttnArgs a) { add_sums(a, kv4_workgroup()); }

// ---------------------------------------------------------------- eviction

// Order of the sums: larger ones first, NaN before all.
__device__ __forceinline__ uint32_t evict_rank(float x) {
  if (x != x) return ~0u;
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);  // (-0 is 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int evict_len(const Kv4EvictArgs& a, int b) {
  if (!a.seq_len) return a.len;
  const int n = a.seq_len[b];
  return n < 0 || n > a.len ? 0 : n;
}

// A place of counts gains the lanes that are `in`: those of the same place are added
// together for the first three places of a wave, since sums are of few sizes and atomics on
// one place go one after the other.
__device__ __forceinline__ void count_places(uint32_t* counts, uint32_t place, bool in) {
  uint64_t left = __ballot(in);
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (!left) return;
    const int first = __ffsll(static_cast<unsigned long long>(left)) - 1;
    const uint32_t of = __builtin_amdgcn_readlane(place, first);
    const uint64_t same = __ballot(in && place == of) & left;
    if (lane == first) atomicAdd(&counts[of], static_cast<uint32_t>(__popcll(same)));
    left &= ~same;
  }
  if (left >> lane & 1) atomicAdd(&counts[place], 1u);
}

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kSelEach = 8, kSelMost = kSelThreads * kSelEach;  // positions a workgroup holds
// A rank's three digits, of 11, 11 and 10 bits.
constexpr int kDigit0 = 2048, kDigit1 = 2048, kDigit2 = 1024, kDigits = kDigit0 + kDigit1 + kDigit2;

struct SelShared {
  uint32_t waves[kSelWaves];
  uint32_t found[2];
  uint32_t n[2][kSelEach * kSelWaves];
};

// Of N counts, the place of the left-th largest and how many are left there: found.  By all
// threads, each N / 1024 places in falling order.
template <int N>
__device__ __forceinline__ void find_place(const uint32_t* counts, uint32_t left, SelShared& sh) {
  constexpr int PER = N / kSelThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t c[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    c[i] = counts[N - 1 - (tid * PER + i)];
    sum += c[i];
  }
  uint32_t upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t x = static_cast<uint32_t>(__shfl_up(static_cast<int>(upto), d, 64));
    if (lane >= d) upto += x;
  }
  if (lane == 63) sh.waves[wave] = upto;
  __syncthreads();
  uint32_t before = upto - sum;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) before += w < wave ? sh.waves[w] : 0;
  if (before < left && left <= before + sum) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (before < left && left <= before + c[i]) {
        sh.found[0] = N - 1 - (tid * PER + i);
        sh.found[1] = left - before;
      }
      before += c[i];
    }
  }
  __syncthreads();
}

// Writes the positions first + kSelThreads e + thread that stay, in their order, from idx
// + at on: those with a rank above `least`, and the first `ties` of those at it.
template <int EACH>
__device__ __forceinline__ void emit(const uint32_t (&rank)[EACH], int first, int end, uint32_t least, uint32_t ties,
                                     uint32_t at, int32_t* idx, SelShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const bool in = first + kSelThreads * e + tid < end;
    const uint64_t mo = __ballot(in && rank[e] > least), ms = __ballot(in && rank[e] == least);
    if (lane == 0) {
      sh.n[0][e * kSelWaves + wave] = __popcll(mo);
      sh.n[1][e * kSelWaves + wave] = __popcll(ms);
    }
  }
  __syncthreads();
  // numbers before each 64 positions: the first two waves add up, EACH / 4 of them a lane
  constexpr int PER = EACH / 4;
  if (wave < 2) {
    uint32_t c[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      c[i] = sh.n[wave][lane * PER + i];
      sum += c[i];
    }
    uint32_t upto = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t x = static_cast<uint32_t>(__shfl_up(static_cast<int>(upto), d, 64));
      if (lane >= d) upto += x;
    }
    uint32_t before = upto - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      sh.n[wave][lane * PER + i] = before;
      before += c[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int i = first + kSelThreads * e + tid;
    const bool over = i < end && rank[e] > least, same = i < end && rank[e] == least;
    const uint64_t mo = __ballot(over), ms = __ballot(same);
    const uint32_t o = sh.n[0][e * kSelWaves + wave] + __popcll(mo & below);
    const uint32_t s = sh.n[1][e * kSelWaves + wave] + __popcll(ms & below);  // ties before
    if (over || (same && s < ties)) idx[at + o + min(s, ties)] = i;
  }
}

__device__ __forceinline__ uint32_t rank_digit(uint32_t u, int pass) {
  return pass == 0 ? u >> 21 : pass == 1 ? u >> 10 & 2047 : u & 1023;
}
__device__ __forceinline__ uint32_t rank_above(uint32_t u, int pass) { return pass == 0 ? 0 : pass == 1 ? u >> 21 : u >> 10; }

// Up to kSelMost positions: a workgroup takes a head and holds their ranks; the rank of the
// last one that stays by three passes over counts of a digit.  Bound by the passes' barriers:
// 8.9 us traced for 128 heads of 2048 positions (62 us with one thread looking through the
// counts).
__global__ __launch_bounds__(kSelThreads) void ld_kv4_select_k(Kv4EvictArgs a) {
  __shared__ uint32_t counts[kDigits];
  __shared__ SelShared sh;
  const int tid = threadIdx.x;
  const int h = blockIdx.x, b = blockIdx.y, n = evict_len(a, b);
  const int64_t head = static_cast<int64_t>(b) * a.from.KV + h;
  int32_t* idx = a.idx + head * a.keep;
  if (n <= a.keep) {
    for (int i = tid; i < a.keep; i += kSelThreads) idx[i] = i < n ? i : -1;
    return;
  }
  const float* sums = a.from.sums + head * a.from.s_max;
  const int old = n - a.recent;
  for (int i = tid; i < a.recent; i += kSelThreads) idx[a.keep - a.recent + i] = old + i;
  if (a.keep == a.recent) return;
  uint32_t rank[kSelEach];
#pragma unroll
  for (int e = 0; e < kSelEach; ++e) {
    const int i = tid + kSelThreads * e;
    rank[e] = i < old ? evict_rank(sums[i]) : 0u;
  }
  for (int i = tid; i < kDigits; i += kSelThreads) counts[i] = 0;
  __syncthreads();
  uint32_t left = a.keep - a.recent, prefix = 0;  // of those with the prefix `left` stay
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    uint32_t* of = counts + (p == 0 ? 0 : p == 1 ? kDigit0 : kDigit0 + kDigit1);
#pragma unroll
    for (int e = 0; e < kSelEach; ++e) {
      if (kSelThreads * e >= old) break;  // uniform
      count_places(of, rank_digit(rank[e], p), tid + kSelThreads * e < old && rank_above(rank[e], p) == prefix);
    }
    __syncthreads();
    if (p < 2)
      find_place<2048>(of, left, sh);
    else
      find_place<kDigit2>(of, left, sh);
    prefix = prefix << (p < 2 ? 11 : 10) | sh.found[0];
    left = sh.found[1];
  }
  emit<kSelEach>(rank, 0, old, prefix, left, 0, idx, sh);
}

// More positions: workgroups of kPiece of them, a launch for each digit, whose counts meet
// in memory.  Scratch of a head: the three digits' counts; after each, the prefix so far and
// how many are left at it; each piece's numbers above the last one that stays and equal to it.
// Six launches of 4 to 6 us traced, 30 in all for 8 heads of 131072 positions (one workgroup
// a head took 320).
constexpr int kPiece = 4096, kPieceEach = kPiece / kSelThreads;
constexpr int kFound = kDigits, kPieces = kDigits + 8;

__global__ __launch_bounds__(256) void ld_kv4_select_zero_k(uint32_t* ws, int64_t stride) {
  uint32_t* counts = ws + blockIdx.y * stride;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < kDigits; i += gridDim.x * 256) counts[i] = 0;
}

// PASS 0 to 2: counts of that digit; 3: a piece's numbers; 4: places.
template <int PASS>
__global__ __launch_bounds__(kSelThreads) void ld_kv4_select_pass_k(Kv4EvictArgs a, int64_t stride) {
  __shared__ uint32_t counts[PASS < 3 ? 2048 : 1];
  __shared__ SelShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int piece = blockIdx.x, h = blockIdx.y, b = blockIdx.z, n = evict_len(a, b), pieces = gridDim.x;
  const int64_t head = static_cast<int64_t>(b) * a.from.KV + h;
  int32_t* idx = a.idx + head * a.keep;
  const int old = n - a.recent, first = piece * kPiece;
  if (n <= a.keep || a.keep == a.recent) {
    if (PASS == 4)
      for (int i = piece * kSelThreads + tid; i < a.keep; i += pieces * kSelThreads)
        idx[i] = n <= a.keep ? (i < n ? i : -1) : old + i;
    return;
  }
  if (PASS == 4)
    for (int i = piece * kSelThreads + tid; i < a.recent; i += pieces * kSelThreads) idx[a.keep - a.recent + i] = old + i;
  if (first >= old) return;
  uint32_t* ws = a.ws + head * stride;
  uint32_t* per_piece = ws + kPieces;
  const float* sums = a.from.sums + head * a.from.s_max;
  uint32_t rank[kPieceEach];
#pragma unroll
  for (int e = 0; e < kPieceEach; ++e) {
    const int i = first + tid + kSelThreads * e;
    rank[e] = i < old ? evict_rank(sums[i]) : 0u;
  }
  if constexpr (PASS < 3) {
    counts[tid] = 0;
    counts[tid + kSelThreads] = 0;
  }
  // what the pass before counted; a head's workgroups all find it, the first notes it
  uint32_t left = a.keep - a.recent, prefix = 0;
  if constexpr (PASS == 4) {
    prefix = ws[kFound + 4];
    left = ws[kFound + 5];
  } else if constexpr (PASS > 0) {
    if constexpr (PASS > 1) {
      prefix = ws[kFound + 2 * (PASS - 2)];
      left = ws[kFound + 2 * (PASS - 2) + 1];
    }
    if constexpr (PASS == 3)
      find_place<kDigit2>(ws + kDigit0 + kDigit1, left, sh);
    else
      find_place<2048>(ws + (PASS == 2 ? kDigit0 : 0), left, sh);
    prefix = prefix << (PASS == 3 ? 10 : 11) | sh.found[0];
    left = sh.found[1];
    if (piece == 0 && tid == 0) {
      ws[kFound + 2 * (PASS - 1)] = prefix;
      ws[kFound + 2 * (PASS - 1) + 1] = left;
    }
  }
  if constexpr (PASS < 3) {
    if (PASS == 0) __syncthreads();
#pragma unroll
    for (int e = 0; e < kPieceEach; ++e) {
      if (first + kSelThreads * e >= old) break;  // uniform
      count_places(counts, rank_digit(rank[e], PASS),
                   first + tid + kSelThreads * e < old && rank_above(rank[e], PASS) == prefix);
    }
    __syncthreads();
    uint32_t* to = ws + (PASS == 0 ? 0 : PASS == 1 ? kDigit0 : kDigit0 + kDigit1);
    for (int i = tid; i < (PASS == 2 ? kDigit2 : 2048); i += kSelThreads)
      if (counts[i]) atomicAdd(&to[i], counts[i]);
  } else if constexpr (PASS == 3) {
    uint32_t over = 0, same = 0;
#pragma unroll
    for (int e = 0; e < kPieceEach; ++e) {
      const bool in = first + tid + kSelThreads * e < old;
      over += __popcll(__ballot(in && rank[e] > prefix));
      same += __popcll(__ballot(in && rank[e] == prefix));
    }
    if (lane == 0) {
      sh.n[0][wave] = over;
      sh.n[1][wave] = same;
    }
    __syncthreads();
    if (tid < 2) {
      uint32_t all = 0;
      for (int w = 0; w < kSelWaves; ++w) all += sh.n[tid][w];
      per_piece[2 * piece + tid] = all;
    }
  } else {
    // numbers of the pieces before
    uint32_t over = 0, same = 0;
    for (int i = lane; i < piece; i += 64) {
      over += per_piece[2 * i];
      same += per_piece[2 * i + 1];
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      over += static_cast<uint32_t>(__shfl_xor(static_cast<int>(over), d, 64));
      same += static_cast<uint32_t>(__shfl_xor(static_cast<int>(same), d, 64));
    }
    same = min(same, left);
    emit<kPieceEach>(rank, first, old, prefix, left - same, over + same, idx, sh);
  }
}

// A wave takes a tile of 8 places of the smaller cache: their keys, values, scales
// and sums.  A position's values lie in 8 (4) lines of its tile, so that the values of a
// cache are read as a whole where few positions stay: 16384 of 131072 positions of 8 heads of
// 128 read 73 MB, 17 us traced (4.3 TB/s with 18 MB written); 512 of 2048 of 128 heads 7.5.
template <int DH>
__global__ __launch_bounds__(256) void ld_kv4_gather_k(Kv4EvictArgs a) {
  constexpr int JN = DH / 32, TB = DH * 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tiles = (a.keep + 7) / 8, id = kv4_workgroup() * 4 + wave;
  const int64_t head = id / tiles;
  if (head >= static_cast<int64_t>(a.to.n_seq) * a.to.KV) return;
  const int t0 = id % tiles * 8, n = min(evict_len(a, head / a.to.KV), a.keep);
  if (t0 >= n) return;
  const int32_t* idx = a.idx + head * a.keep + t0;
  const uint8_t* kf = a.from.codes + head * a.from.s8 * DH;
  const uint8_t* vf = kf + static_cast<int64_t>(a.from.s8) * (DH / 2);
  uint8_t* kt = a.to.codes + head * a.to.s8 * DH;
  uint8_t* vt = kt + static_cast<int64_t>(a.to.s8) * (DH / 2);
  const uint8_t* sf = a.from.scales + head * 2 * a.from.s8 * JN;
  uint8_t* st = a.to.scales + head * 2 * a.to.s8 * JN;
  const int have = min(n - t0, 8);
  // the tile's positions (past the last: the first again)
  const int mine = idx[(lane & 7) < have ? lane & 7 : 0];
  int pos[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) pos[r] = __builtin_amdgcn_readlane(mine, r);
  // values: a lane 8 bytes of a tile, one of each position
  const int e = lane * 8 % TB;  // (heads of 64: half the lanes)
  uint32_t v[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) v[r] = vf[static_cast<int64_t>(pos[r] >> 3) * TB + e + (pos[r] & 7)];
  // keys: a lane DH / 16 bytes of row lane / 8
  typedef uint32_t KRow __attribute__((ext_vector_type(DH / 64)));
  const int row = lane >> 3, src = __shfl(mine, row, 64);
  const KRow k = *reinterpret_cast<const KRow*>(kf + static_cast<int64_t>(src) * (DH / 2) + (lane & 7) * (DH / 16));
  // scales: a byte a lane, keys' then values'
  const int sr = lane / JN & 7, sj = lane % JN, sp = lane / (8 * JN);
  const int from_pos = __shfl(mine, sr, 64);
  const bool scale = sp < 2 && sr < have;
  uint8_t s = 0;
  if (scale) s = sf[(static_cast<int64_t>(sp) * a.from.s8 + from_pos) * JN + sj];
  float w = 0.f;
  const bool sum = a.to.sums && lane < have;
  if (sum) w = a.from.sums[head * a.from.s_max + mine];

  if (row < have) *reinterpret_cast<KRow*>(kt + static_cast<int64_t>(t0 + row) * (DH / 2) + (lane & 7) * (DH / 16)) = k;
  uint8_t* to = vt + static_cast<int64_t>(t0 >> 3) * TB + e;
  if (lane * 8 < TB) {
    if (have == 8) {
      *reinterpret_cast<u32x2*>(to) = u32x2{v[0] | v[1] << 8 | v[2] << 16 | v[3] << 24, v[4] | v[5] << 8 | v[6] << 16 | v[7] << 24};
    } else {
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < have) to[r] = static_cast<uint8_t>(v[r]);
    }
  }
  if (scale) st[(static_cast<int64_t>(sp) * a.to.s8 + t0 + sr) * JN + sj] = s;
  if (sum) a.to.sums[head * a.to.s_max + t0 + lane] = w;
}

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups in two dimensions: one takes 2^32 threads at most.
dim3 kv4_grid(int64_t wgs) {
  constexpr int64_t kX = 1 << 20;
  return wgs <= kX ? dim3(wgs) : dim3(kX, (wgs + kX - 1) / kX);
}

template <int DH>
hipError_t store_t(Kv4StoreArgs a, hipStream_t s) {
  constexpr int U = Kv4Lanes<DH>::U;
  // pieces of any sequence: from the one that holds its first row
  a.pieces = static_cast<int32_t>(a.seq_pos ? (static_cast<int64_t>(a.n) + U - 2) / U + 1
                                            : (static_cast<int64_t>(a.pos) + a.n - 1) / U - a.pos / U + 1);
  const int64_t units = 2ll * a.kv.KV * a.kv.n_seq * a.pieces;
  hipLaunchKernelGGL((ld_kv4_store_k<DH>), kv4_grid((units + 3) / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int DH>
hipError_t load_t(Kv4LoadArgs a, hipStream_t s) {
  constexpr int U = Kv4Lanes<DH>::U;
  a.pieces = static_cast<int32_t>((static_cast<int64_t>(a.pos) + a.n - 1) / U - a.pos / U + 1);
  const int64_t units = 2ll * a.kv.KV * a.kv.n_seq * a.pieces;
  hipLaunchKernelGGL((ld_kv4_load_k<DH>), kv4_grid((units + 3) / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int DH>
hipError_t attn_t(const Kv4AttnArgs& a, hipStream_t s) {
  const int R = a.group * a.n_new;
  const dim3 block(64 * kKv4Waves);
  const dim3 grid = a.tiles == 1 ? dim3(a.n_chunks, a.kv.KV, a.kv.n_seq)
                                 : dim3(a.kv.KV * a.n_chunks * a.tiles, 1, a.kv.n_seq);
  // rows kept for the merge: less LDS
  if (R == 1)
    hipLaunchKernelGGL((ld_attn_decode_kv4_k<DH, 1>), grid, block, 0, s, a);
  else if (R <= 8)
    hipLaunchKernelGGL((ld_attn_decode_kv4_k<DH, 8>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((ld_attn_decode_kv4_k<DH, 16>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <int DH>
hipError_t combine_t(const Kv4AttnArgs& a, hipStream_t s) {
  const int64_t rows = static_cast<int64_t>(a.kv.n_seq) * a.H * a.n_new;
  const int64_t sums = a.scores ? div_up(static_cast<int64_t>(a.pos) + a.n_new, kSumKeys) * a.kv.KV * a.kv.n_seq : 0;
  if (a.n_chunks <= 1) {
    hipLaunchKernelGGL(ld_kv4_sums_k, kv4_grid(sums), dim3(256), 0, s, a);
  } else if (a.n_chunks > 4 && rows <= 2048) {
    hipLaunchKernelGGL((ld_attn_decode_kv4_combine<DH, 4>), kv4_grid(rows + sums), dim3(256), 0, s, a, static_cast<uint32_t>(rows));
  } else {
    const int64_t blocks = div_up(rows, 4);
    hipLaunchKernelGGL((ld_attn_decode_kv4_combine<DH, 1>), kv4_grid(blocks + sums), dim3(256), 0, s, a, static_cast<uint32_t>(blocks));
  }
  return hipGetLastError();
}

// Workgroups that run at once, two on each of the 256 compute units; the most that a launch
// without row tiles makes; and the fewest keys of a chunk where lengths are the device's.
// There a sequence is cut into as many chunks as the most allows, so that long ones leave no
// tail.  Us for two, three, four and six rounds, up to 8192 keys of 16 sequences of 32 heads 41,
// 42, 43, 44; 32768 of 8 of 8 42, 41, 47, 49; 4096 of 64 of 8 39, 38, 38, 43; 100000 of 16 of 8 207, 188,
// 180, 177; 2056 of 32 of 16 22, 23, 25, 26.  (With scaled score products, 2 to 3% less.)
constexpr int64_t kKv4AtOnce = 512, kKv4Wgs = 3 * kKv4AtOnce, kKv4Uneven = 512;

}  // namespace

hipError_t launch_kv4_store(const Kv4StoreArgs& a, hipStream_t s) { return a.kv.dh == 128 ? store_t<128>(a, s) : store_t<64>(a, s); }
hipError_t launch_kv4_load(const Kv4LoadArgs& a, hipStream_t s) { return a.kv.dh == 128 ? load_t<128>(a, s) : load_t<64>(a, s); }

int64_t attn_kv4_heads(const Kv4View& kv, int64_t H, int64_t n_new) {
  const int64_t R = H / kv.KV * n_new;
  return static_cast<int64_t>(kv.n_seq) * kv.KV * ((R + 15) / 16);
}

int64_t attn_kv4_max_chunks(int64_t heads, int64_t keys) {
  const int64_t by_keys = div_up(keys, kKv4Turn), by_wgs = div_up(kKv4Wgs, heads);
  return by_keys < by_wgs ? by_keys : by_wgs;
}

// What n chunks cost a launch, in tenths of the time that a turn takes with the compute units
// full: of a workgroup alone on its unit, six; a round's start and its sums, ten; the launch
// that joins chunks, six.
static int64_t chunk_cost(int64_t heads, int64_t keys, int64_t n) {
  const int64_t wgs = heads * n, turns = div_up(div_up(keys, n), kKv4Turn);
  return div_up(wgs, kKv4AtOnce) * (turns * (2 * wgs <= kKv4AtOnce ? 6 : 10) + 10) + (n > 1 ? 6 : 0);
}

// A wave's turn writes the scores of 32 keys.
int64_t attn_kv4_score_keys(int64_t keys) { return div_up(keys, 32) * 32; }

void plan_attn_decode_kv4(Kv4AttnArgs& a) {
  const int64_t keys = static_cast<int64_t>(a.pos) + a.n_new;
  a.group = a.H / a.kv.KV;
  a.tiles = (a.group * a.n_new + 15) / 16;
  const int64_t heads = attn_kv4_heads(a.kv, a.H, a.n_new);
  const int64_t most = attn_kv4_max_chunks(heads, keys);
  if (a.seq_pos) {
    const int64_t n = div_up(keys, kKv4Uneven);
    a.n_chunks = static_cast<int32_t>(n < most ? n : most);
    a.chunk_keys = static_cast<int32_t>(kKv4Uneven);
  } else {
    int64_t best = INT64_MAX, n = 1;
    for (int64_t half = 1; half <= 2 * kKv4Wgs / kKv4AtOnce; ++half) {
      int64_t c = half * kKv4AtOnce / 2 / heads;
      c = c < 1 ? 1 : c > most ? most : c;
      const int64_t cost = chunk_cost(heads, keys, c);
      if (cost < best) best = cost, n = c;
    }
    a.chunk_keys = static_cast<int32_t>(div_up(div_up(keys, n), kKv4Turn) * kKv4Turn);
    a.n_chunks = static_cast<int32_t>(div_up(keys, a.chunk_keys));
  }
  a.score_keys = attn_kv4_score_keys(keys);
}

hipError_t launch_attn_decode_kv4(const Kv4AttnArgs& a, hipStream_t s) {
  return a.kv.dh == 128 ? attn_t<128>(a, s) : attn_t<64>(a, s);
}

hipError_t launch_attn_decode_kv4_combine(const Kv4AttnArgs& a, hipStream_t s) {
  return a.kv.dh == 128 ? combine_t<128>(a, s) : combine_t<64>(a, s);
}

namespace {
// Words of scratch a head, where its positions go in pieces.
int64_t select_stride(int64_t len) { return len <= kSelMost ? 0 : kPieces + 2 * div_up(len, kPiece); }
}  // namespace

size_t kv4_evict_ws_bytes(const Kv4View& from, int64_t len) {
  return static_cast<size_t>(from.n_seq) * from.KV * select_stride(len) * 4;
}

hipError_t launch_kv4_select(const Kv4EvictArgs& a, hipStream_t s) {
  const int64_t stride = select_stride(a.len);
  if (!stride) {
    hipLaunchKernelGGL(ld_kv4_select_k, dim3(a.from.KV, a.from.n_seq), dim3(kSelThreads), 0, s, a);
    return hipGetLastError();
  }
  const dim3 grid(div_up(a.len, kPiece), a.from.KV, a.from.n_seq), block(kSelThreads);
  const int64_t heads = static_cast<int64_t>(a.from.KV) * a.from.n_seq;
  // (a launch takes 65535 in its second dimension)
  for (int64_t h = 0; h < heads; h += 65535)
    hipLaunchKernelGGL(ld_kv4_select_zero_k, dim3(4, heads - h < 65535 ? heads - h : 65535), dim3(256), 0, s, a.ws + h * stride, stride);
  hipLaunchKernelGGL(ld_kv4_select_pass_k<0>, grid, block, 0, s, a, stride);
  hipLaunchKernelGGL(ld_kv4_select_pass_k<1>, grid, block, 0, s, a, stride);
  hipLaunchKernelGGL(ld_kv4_select_pass_k<2>, grid, block, 0, s, a, stride);
  hipLaunchKernelGGL(ld_kv4_select_pass_k<3>, grid, block, 0, s, a, stride);
  hipLaunchKernelGGL(ld_kv4_select_pass_k<4>, grid, block, 0, s, a, stride);
  return hipGetLastError();
}

hipError_t launch_kv4_gather(const Kv4EvictArgs& a, hipStream_t s) {
  const int64_t waves = static_cast<int64_t>(a.to.n_seq) * a.to.KV * div_up(a.keep, 8);
  if (a.to.dh == 128)
    hipLaunchKernelGGL((ld_kv4_gather_k<128>), kv4_grid(div_up(waves, 4)), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((ld_kv4_gather_k<64>), kv4_grid(div_up(waves, 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace ld
