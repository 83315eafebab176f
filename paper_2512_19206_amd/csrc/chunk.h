// What the attention of a chunk of new tokens shares between its host side (chunk_api.hip) and its kernels (chunk_kernels.hip: tiles of
// tokens in LDS, many query rows; chunk_few.h: wavefronts of their own, few query rows).
#pragma once
#include "mixkvq_internal.h"

namespace mixkvq {

constexpr int kChunkTile = 128;        // tokens of keys and values that a workgroup of the tile kernel holds in LDS at a time
constexpr int kChunkSeqs = 128;        // sequences of one launch whose counts differ (they go by value)
constexpr int kChunkUnits = 1024;      // (sequence, split) units of such a launch
constexpr int kChunkMaxSplits = 64;    // workgroups that share one tile of query rows, each over its part of the tokens
constexpr int kChunkRecords = 4;       // most records of one tile

// The arguments of a launch, without what its kernels have no use for: they are read in one trip at the start.  The grid is
// (units x KV heads, tiles of query rows); a unit is one split of one sequence, the splits of a sequence are neighbours.
struct ChunkArgs {
  const __half *q, *k, *v;
  __half* out;
  float* lse;                          // [B][Hq][n_max], or nullptr
  float* part;                         // [block][rows][kD], then [block][rows][2]: sums, maxima and sums of weights; block: x * tiles of rows + y
  const uint8_t* blocks;
  const int32_t* table;                // [B][NB] or nullptr
  const __half *res_k, *res_v;
  Strides3 qs, kvs, os;
  float scale;
  int32_t n_max, b0;                   // tokens the tensors have room for; first sequence
  int32_t n_rec, n_fp16, n_new, n_splits;      // of every sequence, unless the launch has ChunkCounts
  int32_t row_tiles, split;            // tiles of query rows (grid's y); is any sequence split?
  int32_t NB, RW, Hkv, Hq, g, bf16;
  int32_t R, Gk, k4, k16, rec_bytes, tile_rec;
  int32_t inv_r, inv_gk;               // x inv_r >> 16 is x / R for x <= 128, and so with Gk
  int32_t nvg_bits;                    // NVG is two to this
  int32_t NLp, Wlo, W4, NVG, interleave;
  int32_t off_idx, off_kmax, off_klo_s, off_klo_z, off_k4_s, off_k4_z, off_klo, off_k4, off_k16, off_v, off_v_s, off_v_z;
};

// Counts of sequences that differ.
struct ChunkCounts {
  int32_t n_rec[kChunkSeqs];           // records
  int32_t n_new[kChunkSeqs];           // new tokens
  uint32_t rows_splits[kChunkSeqs];    // fp16 rows in use | splits << 16
  int32_t first[kChunkSeqs];           // first unit (whole words: the compiler has split the address of a half one so that the scalar unit dropped its odd half)
  uint32_t owner[kChunkUnits / 4];     // sequence of unit u: byte u % 4 of word u / 4
};
struct NoChunkCounts {};

// The part of the work that a workgroup has.
struct ChunkPlace {
  int b, j, p;                         // sequence, KV head, pair
  int split, n_splits, n_rec, n_fp16, n_new;
  int first_block;                     // x of the pair's first split (the next ones are Hkv further each)
};

__device__ __forceinline__ ChunkPlace chunk_place(const ChunkArgs& a, const NoChunkCounts&, int x) {
  ChunkPlace w;
  const int unit = x / a.Hkv, i = unit / a.n_splits;
  w.j = x - unit * a.Hkv;
  w.b = a.b0 + i;
  w.split = unit - i * a.n_splits;
  w.n_splits = a.n_splits;
  w.n_rec = a.n_rec;
  w.n_fp16 = a.n_fp16;
  w.n_new = a.n_new;
  w.first_block = i * a.n_splits * a.Hkv + w.j;
  w.p = w.b * a.Hkv + w.j;
  return w;
}
__device__ __forceinline__ ChunkPlace chunk_place(const ChunkArgs& a, const ChunkCounts& c, int x) {
  ChunkPlace w;
  const int unit = x / a.Hkv, i = (int)(c.owner[unit >> 2] >> (8 * (unit & 3)) & 0xffu);
  const uint32_t rs = c.rows_splits[i];
  const int first = c.first[i];
  w.j = x - unit * a.Hkv;
  w.b = a.b0 + i;
  w.split = unit - first;
  w.n_splits = (int)(rs >> 16);
  w.n_rec = c.n_rec[i];
  w.n_fp16 = (int)(rs & 0xffffu);
  w.n_new = c.n_new[i];
  w.first_block = first * a.Hkv + w.j;
  w.p = w.b * a.Hkv + w.j;
  return w;
}

// rows: query rows of a workgroup (256, or with few rows 16, 32 or 48).  c == nullptr: equal counts.
hipError_t launch_chunk(const ChunkArgs& a, const ChunkCounts* c, int units, int n_seq, bool few, int rows, hipStream_t s);
hipError_t launch_chunk_books(const CacheView& v, const ChunkArgs& a, const ChunkCounts* c, int n_seq, int n_most, hipStream_t s);      // |q| of the chunk
int chunk_tile_records(const CacheView& v);      // records of one tile
// Steps of 32 channel places with codes that the kernel for few rows takes: 4 where the 4-bit words find room behind the 2-bit ones.
inline int chunk_few_steps(int NLp, int W4) { return W4 == 0 || (W4 <= 2 && NLp <= 112) ? 4 : 5; }
bool chunk_few_fits(const CacheView& v);         // does the kernel for few rows take this record layout?
int chunk_few_rows(const CacheView& v);          // and with how many rows to a workgroup at most?

}  // namespace mixkvq
