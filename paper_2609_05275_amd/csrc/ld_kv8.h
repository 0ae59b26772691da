// The 8-bit key/value cache's kernels, as the API calls them.  A header of its own:
// the other kernels' counter records hold for the contents of ld_internal.h.
#pragma once
#include "ld_internal.h"

namespace ld {

// An 8-bit key/value cache (ld_kv8).  Codes of head (b, h): keys [s16][dh] from
// ((b KV + h) 2) s16 dh on, then values [s16 / 16][dh][16], so that 16 positions
// of one dimension are the 16 bytes an MFMA operand of the output product
// wants.  Scales [n_seq][KV][2][nb].
struct Kv8View {
  uint8_t* codes;
  float* scales;
  int32_t format, block, shift, n_seq, KV, dh, s16, nb;  // block = 1 << shift
};
constexpr int kKv8MinExp = -100;  // smallest scale 2^-100: a code times it stays a normal bf16

// Key/value columns of rows b n + j of qkv ([., (H + 2 KV) dh], ld_qkv apart) to
// positions pos + j (seq_pos: seq_pos[b] + j where 0 <= seq_pos[b] <= pos).
struct Kv8StoreArgs {
  Kv8View kv;
  const void* qkv;
  int64_t ld_qkv;
  int32_t H, n, pos;
  const int32_t* seq_pos;
  int32_t pieces;  // of a sequence's rows, the launch's choice
};

// Positions pos .. pos + n - 1 (below seq_len[b] where given) to bf16 rows
// [n_seq, n, 2 KV dh].
struct Kv8LoadArgs {
  Kv8View kv;
  void* out;
  int32_t pos, n;
  const int32_t* seq_len;
  int32_t pieces;
};

// Queries of rows b n_new + j of qkv over positions 0 .. p + j, p = pos or
// seq_pos[b].  n_chunks and chunk_keys are plan_attn_decode_kv8's choice.
struct Kv8AttnArgs {
  Kv8View kv;
  const void* qkv;
  int64_t ld_qkv;
  void* out;       // [n_seq * n_new, H * dh]
  float* part_o;   // [n_seq][H * n_new rows of the heads in turn][n_chunks][dh]
  float* part_ml;  // [n_seq][H * n_new][n_chunks][2]: base-2 max, sum
  int32_t H, n_new, pos, group, n_chunks, chunk_keys;  // group = H / KV; chunk_keys: the least
  uint32_t tiles;  // of 16 rows a key/value head
  const int32_t* seq_pos;
  float scale;
  int32_t alibi;
};

hipError_t launch_kv8_store(const Kv8StoreArgs& a, hipStream_t s);
hipError_t launch_kv8_load(const Kv8LoadArgs& a, hipStream_t s);
// Workgroups a chunk of an attention launch, and the most chunks of `keys` keys (it
// grows with keys).
int64_t attn_kv8_heads(const Kv8View& kv, int64_t H, int64_t n_new);
int64_t attn_kv8_max_chunks(int64_t heads, int64_t keys);
// Fills in group, tiles and the chunks; the second launch is for several chunks.
void plan_attn_decode_kv8(Kv8AttnArgs& a);
hipError_t launch_attn_decode_kv8(const Kv8AttnArgs& a, hipStream_t s);
hipError_t launch_attn_decode_kv8_combine(const Kv8AttnArgs& a, hipStream_t s);

}  // namespace ld
