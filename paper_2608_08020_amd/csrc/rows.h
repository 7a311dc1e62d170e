// Packed tokens of several traces: layer writes into the caches, and
// attention of rows (packed token x query head of the GQA group) over them.
// Internal interface between rows_attn.cpp (validation, planner) and the
// kernels of rows_attn.hip and rows_write.hip.
#pragma once

#include <cstdint>

#include "kernels.h"

namespace gambit {

constexpr int kRowsTile = 128;  // rows of one workgroup: four waves x 32
constexpr int kKeyTile = 64;    // cached positions a workgroup takes at a time (4 blocks)
constexpr int kMaxNodes = 64;   // drafted tokens of one trace: one key tile, one 64-bit mask
constexpr int kNoLimit = 0x7fffffff;

// One workgroup's work for one KV head: up to kRowsTile rows over a range of
// a trace's cached positions and, for draft trees, the trace's drafts.
struct RowItem {
  int32_t trace;   // the table row that lists the range's blocks
  int32_t jb0;     // first logical block
  int32_t end;     // end of the range in positions (<= 16 jb0: nothing cached to read)
  int32_t tok;     // first packed token of the rows, or their place in the token list
  int32_t ntok;    // tokens
  int32_t listed;  // 1: `tok` is a place in the token list, 0: the tokens are consecutive
  int32_t pos0;    // causal: the first token's position, token i sees up to pos0 + i; kNoLimit: all
  int32_t kidx;    // partial of these rows; -1: the whole result, written to `out`
  int32_t draft;   // first packed token of the trace's tree, -1: none
  int32_t ndraft;  // its tokens
  int32_t once;    // 1: no other item reads the range's blocks
  int32_t first[4];  // the range's first four blocks (the last one again where there are fewer)
  int32_t pad;
};
static_assert(sizeof(RowItem) == 64, "one scalar load");

struct RowsLaunch {
  const RowItem* items;
  int32_t n_items;
  const int32_t* list;     // packed tokens of the listed items
  const int32_t* off;      // [N] first partial of a packed token (in units of Hq rows)
  const int32_t* nk;       // [N] its partials
  const int32_t* merge;    // [n_merge] packed tokens of more than one item
  int32_t n_merge;
  const uint64_t* anc;     // [N] bit j: node j of the token's tree is the token or an ancestor
  const uint16_t* q;       // [N][Hq][128] bf16
  const uint16_t* k_new;   // [N][Hkv][128] bf16, the drafts
  const uint16_t* v_new;
  void* out;               // [N][Hq][128]
  int32_t out_f32;
  float c;                 // |softmax scale| x log2(e); 1 for a scale of zero
  uint32_t q_and, q_xor;   // applied to pairs of query values: sign of the scale, zero
  int32_t gshift;
  float* part_acc;         // [partial][Hq][128]
  float2* part_ml;         // [partial][Hq]
};
hipError_t launch_rows_attention(const DevPool& P, const RowsLaunch& L, hipStream_t s);

// One block's part of a layer write: rows [r0, r1) of block `blk` take the
// packed tokens src, src + 1, ...
struct WriteItem {
  int32_t blk, src;
  int16_t r0, r1;
  float floor;             // fp8: least scale when the write starts the block; 0: it keeps its scale
};
static_assert(sizeof(WriteItem) == 16, "one scalar load");

struct WriteLaunch {
  const WriteItem* items;
  int32_t n_items;
  const int32_t* at;       // [n_items] position of an item's block
  const int32_t* rows;     // [N] row of k / v (and q) of a packed token, or null: its own index
  const uint16_t* k;       // [*][Hkv][128] bf16, rows k_stride values apart
  const uint16_t* v;
  int64_t k_stride, v_stride;
  // rotated writes (table not null): keys, and the queries that go to q_out
  const float* table;      // [position][rot]: rot / 2 cosines, rot / 2 sines
  int32_t rot, pairs;      // values of a head that turn; pairs: (2i, 2i + 1), else (i, i + rot / 2)
  const uint16_t* q;       // [*][Hq][128] bf16, rows q_stride values apart, or null
  int64_t q_stride;
  uint16_t* q_out;         // [N][Hq][128]
};
hipError_t launch_rows_write(const DevPool& P, const WriteLaunch& L, hipStream_t s);

}  // namespace gambit
