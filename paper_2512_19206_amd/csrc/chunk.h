// What the attention of a chunk of new tokens shares between its host side (chunk_api.hip) and its kernels (chunk_kernels.hip).
#pragma once
#include "mixkvq_internal.h"

namespace mixkvq {

constexpr int kChunkTile = 128;        // tokens of keys and values that a workgroup holds in LDS at a time
constexpr int kChunkSeqs = 128;        // sequences of one launch (their counts go by value)
constexpr int kChunkMaxSplits = 64;    // workgroups that share one tile of query rows, each over its part of the tokens
constexpr int kChunkRecords = 4;       // most records of one tile

// One launch: up to kChunkSeqs neighbouring sequences.  A unit is one workgroup: a tile of query rows of one (sequence, KV
// head) pair over one split of its tokens.  Unit numbers run over the sequences, then the heads, then the splits, then the
// tiles of rows.
struct ChunkLaunch {
  int32_t b0, n_seq;                   // first sequence and how many
  int32_t n_units;
  int32_t tile_rec;                    // records of a tile: chunk_tile_records()
  int32_t same_units;                  // units of every sequence where all have the same number, else 0
  int32_t n_rec[kChunkSeqs];           // records of the sequence
  int32_t n_new[kChunkSeqs];           // new tokens
  uint32_t rows_splits[kChunkSeqs];    // fp16 rows in use | splits << 16
  int32_t first_unit[kChunkSeqs];
};

// The caller's tensors and the launch's constants.
struct ChunkArgs {
  const __half *q, *k, *v;
  __half* out;
  float* lse;                          // [B][Hq][n_max], or nullptr
  Strides3 qs, kvs, os;
  int32_t n_max;                       // tokens the tensors have room for
  float scale;
  float* part;                         // [unit][rows][kD], then [unit][rows][2]: partial sums, maxima and sums of weights
};

// Two kernels: the tile kernel (chunk_kernels.hip; 64, 128 or 256 query rows to a workgroup, any configuration) and the one for
// few rows (chunk_few.h; 16, 32 or 48, the record layouts that chunk_few_fits takes).
bool chunk_few_fits(const CacheView& v);
hipError_t launch_chunk(const CacheView& v, const ChunkArgs& a, const ChunkLaunch& l, bool few, int rows, bool split, hipStream_t s);
hipError_t launch_chunk_books(const CacheView& v, const ChunkArgs& a, const ChunkLaunch& l, hipStream_t s);   // |q| of the chunk
int chunk_tile_records(const CacheView& v);      // records of one tile

}  // namespace mixkvq
