// Internal declarations of the operators around the cache (norm and rotation, windowed attention, the caches
// in 4 and 8 bits, accumulated attention weights), shared by their host layers (cache_ops.cpp, cache8_ops.cpp)
// and their kernels.  Not part of the ABI.
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
  int max_tokens;        // of a sequence
};
int launch_cache4_positions(const Cache4Args& a, void* stream);
int launch_cache4_gather(const Cache4Args& a, int dtype, int d, void* stream);
// max_new: the most new tokens of a sequence
int launch_cache4_append(const Cache4Args& a, int max_new, int dtype, int d, void* stream);
int launch_cache4_read(const Cache4Args& a, int dtype, int d, void* stream);

// Attention over 8 bits with accumulated weights: bytes of an item's scores.  Two workgroups' fill a CU's LDS.
constexpr int kAttnMostLds = 70 * 1024;
// Attention.  Rows of a problem (KV head, sequence) are its queries times its query heads: row
// r = i * group + g.  An item is a tile of rows and a range of key tiles; a problem's items are
// row tiles times splits.  Words per sequence: first query, first key, first item, splits, key tiles of a
// split, first part (the items of sequences with more than one split leave parts, numbered apart).
constexpr int kAttnSeqWords = 6;
constexpr int kAttnTile = 32;        // keys of a tile
constexpr int kAttnRows = 16;        // rows of a tile
constexpr int kAttnPairRows = 32;    // of an item whose waves take two row tiles at once (a cache, bf16)
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
  Cache4 cache;          // k, v null: keys and values in 4 or 8 bits
  const int32_t* len;    // [n_heads * n_seqs] rows in use (of a cache)
  float* lse;            // nullable
  int64_t Tq;            // queries per head of lse
  float scale_log2;      // scale * log2(e)
  int window, n_sink;    // at most kAttnMaxKeys each
  int n_heads, group, n_seqs;
  int items, parts;      // per head
  int rows;              // of an item: kAttnRows, kAttnPairRows, kAttnWideRows or kAttnBigRows
  float* part_o;         // [n_heads][parts][rows][d] unnormalised sums
  float* part_ml;        // [n_heads][parts][rows][2] maximum (log2 units) and sum
  // 8 bits, one row tile a problem: accumulated weights wanted (else all null)
  float* score;          // [n_heads][score_rows][cache.C] scores in log2 units
  int score_rows;
  int score_lds;         // scores of an item that a workgroup's LDS holds
  const float* mass;     // nullable [n_heads][cache.C]
  float* mass_out;       // [n_heads][cache.C]
};
int launch_attn(const AttnArgs& a, int dtype, int d, void* stream);
// bf16
int launch_attn_rows(const AttnArgs& a, int d, void* stream);
int launch_attn4(const AttnArgs& a, int dtype, int d, void* stream);
int launch_attn_join(const AttnArgs& a, int dtype, int d, void* stream);

// The 8-bit cache: the same four arrays (layouts in include/twinkv.h), 32 rows of which share a scale.
using Cache8 = Cache4;
constexpr int kCache8Block = 32;
struct Cache8Args : Cache4Args {
  const float* mass;     // nullable [n_heads][T] by token (compact)
  float* mass_out;       // [n_heads][C]
};
int launch_cache8_gather(const Cache8Args& a, int dtype, int d, void* stream);
int launch_cache8_append(const Cache8Args& a, int max_new, int dtype, int d, void* stream);
int launch_cache8_read(const Cache8Args& a, int dtype, int d, void* stream);
int launch_attn8(const AttnArgs& a, int dtype, int d, void* stream);

// Eviction from one cache into another.  Words per sequence: first row of `from`, first row of `to`, rows to
// keep, first block of `to`.
constexpr int kEvict8SeqWords = 4;
struct Evict8Args {
  SeqWords seq;
  Cache8 from, to;
  const int32_t* len;    // [n_heads * n_seqs]
  const float* mass;     // [n_heads][from.C]
  const int32_t* pos;    // nullable [n_heads][from.C]
  int32_t* len_out;
  float* mass_out;       // nullable [n_heads][to.C]
  int32_t* pos_out;      // [n_heads][to.C]; between the two kernels: the row of `from`, -1 where none
  int n_heads, n_seqs;
  int n_sink, n_recent;
  int n_blocks;          // of `to`, per head
  int max_rows;          // of a sequence of `from`
};
int launch_evict8_select(const Evict8Args& a, void* stream);
int launch_evict8_move(const Evict8Args& a, int d, void* stream);

// The weight that each key receives.  Rows are numbered as in the attention; an item is a tile of keys and a split of
// the rows that see one of them, counted from the first.  Words per sequence: first query, first key, first item, the
// most splits of a tile, rows of a split, full tiles, shape.  The first `full` tiles have all the splits; the others,
// by the shape's upper bits: every run of so many tiles one less than the one before, the first as many; every tile so
// many less than the one before, the first as many; each tile so many.
constexpr int kMassSeqWords = 7;
enum MassShape { kMassRuns, kMassDrops, kMassRest };
constexpr int kMassShapeBits = 28;
constexpr int kMassRowTile = 128;  // splits are whole numbers of so many rows
constexpr int kMassKeys = 128;     // of a tile; bf16: or twice as many
struct MassArgs {
  SeqWords seq;
  const char* q;
  const char* k;
  int64_t q_head, q_token, k_head, k_token;  // bytes
  Cache8 cache;            // k null: keys in 8 bits
  const int32_t* len;      // [n_heads * n_seqs] rows in use (8 bits)
  const float* lse;        // [n_heads * group][Tq]
  const float* mass;       // nullable [n_heads][Tk]: what is there already
  float* mass_out;         // [n_heads][Tk]
  int64_t Tq, Tk;
  float scale_log2;
  int window, n_sink;      // at most kAttnMaxKeys each
  int n_heads, group, n_seqs;
  int items;               // per head
  int keys;                // of a tile
  bool few;                // rows see a tile (bf16)
  float* part;             // nullable [n_heads][items][keys], where a tile has more than one split
};
// The place of a sequence's item `left`: its tile, split, the splits of that tile, and its place among the parts, which
// lie tile by tile, a tile's splits side by side.  kByRows: items come in the order of the rows, many tiles and the same
// rows together; otherwise in the order of the parts.  (constexpr: for the host and the device.)
struct MassPlace {
  int tile, split, splits, part;
};
template <bool kByRows>
constexpr MassPlace mass_place(int left, int splits, int full, int shape, int tiles) {
  const int kind = shape >> kMassShapeBits, by = shape & ((1 << kMassShapeBits) - 1);
  MassPlace p = {0, 0, splits, left};
  if (kind == kMassRest) {  // `full` tiles of `splits` splits, the others of `by`
    if (left >= full * splits) {
      left -= full * splits;
      p.splits = by;
      p.tile = full + left / by;
      p.split = left % by;
    } else if (kByRows) {
      p.tile = left % full;
      p.split = left / full;
      p.part = p.tile * splits + p.split;
    } else {
      p.tile = left / splits;
      p.split = left % splits;
    }
    return p;
  }
  // `full` tiles of `splits` splits, then runs of tiles, each run of `drop` splits less, the last ones of `least`
  const int run = kind == kMassRuns ? by : 1, drop = kind == kMassRuns ? 1 : by;
  if (!kByRows) {
    int tile0 = 0;
    if (left >= full * splits) {
      left -= full * splits;
      tile0 = full;
      while (p.splits > drop && left >= run * p.splits) {
        left -= run * p.splits;
        tile0 += run;
        p.splits -= drop;
      }
    }
    p.tile = tile0 + left / p.splits;
    p.split = left % p.splits;
    return p;
  }
  // Split i of run g begins about where split i + g drop of the full tiles does: level by level of those.
  const int runs = (splits + drop - 1) / drop, least = splits - (runs - 1) * drop;
  int level = 0, here = tiles < full + run ? tiles : full + run;  // tiles that have a split at this level
  while (level < splits) {
    const int n = (drop < splits - level ? drop : splits - level) * here;
    if (left < n) break;
    left -= n;
    level += drop;
    here = tiles < here + run ? tiles : here + run;
  }
  int g = 0;
  if (level < splits) {
    p.tile = left % here;
    p.split = level + left / here;
    if (p.tile >= full) {
      g = (p.tile - full) / run;
      p.splits = splits - g * drop;
      p.split -= g * drop;
    }
  } else {
    p.splits = least;
    p.tile = full + run * runs + left / least;
    p.split = left % least;
    g = (p.tile - full) / run;
  }
  const int m = g < runs ? g : runs;
  p.part = p.tile < full ? p.tile * splits
                         : full * splits + run * (m * splits - drop * (m * (m - 1) / 2) + (g - m) * least) +
                               (p.tile - full - run * g) * p.splits;
  p.part += p.split;
  return p;
}
int launch_mass(const MassArgs& a, int dtype, int d, void* stream);
int launch_mass_join(const MassArgs& a, void* stream);

}  // namespace twinkv
