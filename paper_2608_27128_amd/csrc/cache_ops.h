// Internal declarations of the operators around the cache (norm and rotation, windowed attention, the
// 4-bit cache), shared by their host layer (cache_ops.cpp) and their kernels.  Not part of the ABI.
#pragma once

#include <cstddef>
#include <cstdint>

namespace twinkv {

// Per-sequence words of a call, in the kernel arguments for small batches (no copy to launch, nothing
// to wait for) and in the workspace for large ones.
constexpr int kTabWords = 512;
struct SeqWords {
  const int32_t* far;   // device memory, or null: near holds the words
  int32_t near[kTabWords];
};

// K6: rows are heads of tokens; q and k are two ranges of heads.
struct NormRopeSide {
  const char* in;
  char* out;
  int64_t in_head, in_token, out_head, out_token;  // bytes
  const float* weight;                             // nullable
  int heads, chunks;                               // heads, and the units per token they make
};
struct NormRopeArgs {
  NormRopeSide q, k;
  int64_t T, n_pos;
  const float* rope;     // nullable [n_pos][d]
  const int32_t* pos;    // [T]
  float eps;
  int per_unit;          // heads a unit goes through
};
int launch_norm_rope(const NormRopeArgs& a, int dtype, int d, void* stream);

// The 4-bit cache of a call.
struct Cache4 {
  uint8_t* k_codes;
  uint8_t* k_scales;
  uint8_t* v_codes;
  uint8_t* v_scales;
  int64_t C;             // rows per head
};
constexpr int kCacheTile = 32;  // sequences' parts of the cache are whole numbers of so many rows
constexpr int kCacheBlock = 8;  // rows of a block of value codes

// Words per sequence: first token, first cache row, first block of the call's block list (with one
// entry more at the end: what the sequence's ends are).
constexpr int kCacheSeqWords = 3;
struct Cache4Args {
  SeqWords seq;
  Cache4 cache;
  const char* keys;      // byte addresses and strides
  const char* values;
  int64_t head_stride, token_stride, v_head_stride, v_token_stride;
  const uint8_t* retained;  // compact
  int64_t T;
  int32_t* pos;          // compact: out; the list the rows are gathered by
  const int32_t* len_in;
  int32_t* len_out;      // (len of the rows to read)
  int32_t* status;
  const int32_t* first;  // read
  char* keys_out;
  char* values_out;
  int64_t C_out;
  int n_heads, n_seqs;
  int n_blocks;          // blocks of all sequences of a head
};
int launch_cache4_positions(const Cache4Args& a, void* stream);
int launch_cache4_gather(const Cache4Args& a, int dtype, int d, void* stream);
// max_new: the most new tokens of a sequence
int launch_cache4_append(const Cache4Args& a, int max_new, int dtype, int d, void* stream);
int launch_cache4_read(const Cache4Args& a, int dtype, int d, void* stream);

// Attention.  Rows of a problem (KV head, sequence) are its queries times its query heads: row
// r = i * group + g.  An item is a tile of rows and a range of key tiles; a problem's items are
// row tiles times splits.  Words per sequence: first query, first key, first item, splits, key tiles of a
// split, first part (the items of sequences with more than one split leave parts, numbered apart).
constexpr int kAttnSeqWords = 6;
constexpr int kAttnTile = 32;        // keys of a tile
constexpr int kAttnRows = 16;        // rows of a tile
constexpr int kAttnPairRows = 32;    // of an item whose waves take two row tiles at once (4 bits)
constexpr int kAttnWideRows = 64;    // of an item whose four waves take a tile each
constexpr int kAttnBigRows = 128;    // rows and keys of the kernel for many rows
constexpr int kAttnBigTile = 64;
constexpr int kAttnMaxKeys = 1 << 30;  // of all sequences: positions and windows add without overflow
struct AttnArgs {
  SeqWords seq;
  const char* q;
  const char* k;
  const char* v;
  char* out;
  int64_t q_head, q_token, k_head, k_token, v_head, v_token, o_head, o_token;  // bytes
  Cache4 cache;          // k, v null: keys and values in 4 bits
  const int32_t* len;    // [n_heads * n_seqs] rows in use (4 bits)
  float* lse;            // nullable
  int64_t Tq;            // queries per head of lse
  float scale_log2;      // scale * log2(e)
  int window, n_sink;    // at most kAttnMaxKeys each
  int n_heads, group, n_seqs;
  int items, parts;      // per head
  int rows;              // of an item: kAttnRows, kAttnPairRows, kAttnWideRows or kAttnBigRows
  float* part_o;         // [n_heads][parts][rows][d] unnormalised sums
  float* part_ml;        // [n_heads][parts][rows][2] maximum (log2 units) and sum
};
int launch_attn(const AttnArgs& a, int dtype, int d, void* stream);
// bf16
int launch_attn_rows(const AttnArgs& a, int d, void* stream);
int launch_attn4(const AttnArgs& a, int dtype, int d, void* stream);
int launch_attn_join(const AttnArgs& a, int dtype, int d, void* stream);

}  // namespace twinkv
