// The 4-bit key/value cache's kernels, as the API calls them.  A header of its own:
// the other kernels' counter records hold for the contents of ld_internal.h.
#pragma once
#include "ld_internal.h"

namespace ld {

// A 4-bit key/value cache (ld_kv4).  Bytes of head (b, h): keys [s8][dh / 2] from
// (b KV + h) s8 dh on, then values [s8 / 8][16 (n)][dh / 32 (j)][8 (position)], whose bytes
// hold dimensions 32 j + n and 32 j + 16 + n: 8 positions of 16 such pairs are what a lane of
// the output product's operand wants, and the two halves of a byte share a scale.
// Scales [n_seq][KV][2][s8][dh / 32], a power of two's exponent + 127.
struct Kv4View {
  uint8_t* codes;
  uint8_t* scales;
  float* sums;  // null, or [n_seq][KV][s_max]
  int32_t n_seq, KV, dh, s8, s_max;
};
constexpr int kKv4MinExp = -100;  // smallest scale 2^-100: a code times it stays a normal bf16

// Key/value columns of rows b n + j of qkv ([., (H + 2 KV) dh], ld_qkv apart) to
// positions pos + j (seq_pos: seq_pos[b] + j where 0 <= seq_pos[b] <= pos).
struct Kv4StoreArgs {
  Kv4View kv;
  const void* qkv;
  int64_t ld_qkv;
  int32_t H, n, pos;
  const int32_t* seq_pos;
  int32_t pieces;  // of a sequence's rows, the launch's choice
};

// Positions pos .. pos + n - 1 (below seq_len[b] where given) to bf16 rows
// [n_seq, n, 2 KV dh].
struct Kv4LoadArgs {
  Kv4View kv;
  void* out;
  int32_t pos, n;
  const int32_t* seq_len;
  int32_t pieces;
};

// Queries of rows b n_new + j of qkv over positions 0 .. p + j, p = pos or
// seq_pos[b].  n_chunks and chunk_keys are plan_attn_decode_kv4's choice.
struct Kv4AttnArgs {
  Kv4View kv;
  const void* qkv;
  int64_t ld_qkv;
  void* out;       // [n_seq * n_new, H * dh]
  float* part_o;   // [n_seq][H * n_new rows of the heads in turn][n_chunks][dh]
  float* part_ml;  // [n_seq][H * n_new][n_chunks][2]: base-2 max, sum
  float* scores;   // null, or [n_seq][H * n_new][score_keys]: base-2 scores, for the sums
  int64_t score_keys;
  int32_t H, n_new, pos, group, n_chunks, chunk_keys;  // group = H / KV; chunk_keys: the least
  uint32_t tiles;  // of 16 rows a key/value head
  const int32_t* seq_pos;
  float scale;
  int32_t alibi;
};

// The keep positions of each head that stay: the last `recent` of the length
// (seq_len[b] or len) and the largest sums of the others; idx [n_seq][KV][keep].
struct Kv4EvictArgs {
  Kv4View from, to;
  int32_t len, keep, recent;
  const int32_t* seq_len;
  int32_t* idx;
  uint32_t* ws;
};

hipError_t launch_kv4_store(const Kv4StoreArgs& a, hipStream_t s);
hipError_t launch_kv4_load(const Kv4LoadArgs& a, hipStream_t s);
// Workgroups a chunk of an attention launch, and the most chunks of `keys` keys (it
// grows with keys).
int64_t attn_kv4_heads(const Kv4View& kv, int64_t H, int64_t n_new);
int64_t attn_kv4_max_chunks(int64_t heads, int64_t keys);
int64_t attn_kv4_score_keys(int64_t keys);
// Fills in group, tiles and the chunks; the second launch, for several chunks or with scores,
// joins the chunks and adds the weights to kv.sums.
void plan_attn_decode_kv4(Kv4AttnArgs& a);
hipError_t launch_attn_decode_kv4(const Kv4AttnArgs& a, hipStream_t s);
hipError_t launch_attn_decode_kv4_combine(const Kv4AttnArgs& a, hipStream_t s);
size_t kv4_evict_ws_bytes(const Kv4View& from, int64_t len);
hipError_t launch_kv4_select(const Kv4EvictArgs& a, hipStream_t s);
hipError_t launch_kv4_gather(const Kv4EvictArgs& a, hipStream_t s);

}  // namespace ld
