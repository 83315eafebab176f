// mixkvq_chunk_attention: argument checks, and how a launch's work is cut into workgroups.
#include <math.h>
#include "cache_state.h"
#include "chunk.h"

using namespace mixkvq;

namespace mixkvq {

constexpr int kChunkUnitsAtOnce = 256;      // one workgroup to a compute unit (its tiles fill the LDS)
constexpr int kChunkMaxNew = 1 << 20;
constexpr int kFewRows = 512;               // query rows up to which the kernel for few rows may be taken

static int div_up(int a, int b) { return (a + b - 1) / b; }

// How a call is cut: the kernel, the query rows of a workgroup, and how much of a pair's tokens one workgroup takes.
struct ChunkPlan { bool few; int rows, chain; };

static int n_new_of(const int32_t* n_seq, int n_max, int b) { return n_seq ? n_seq[b] : n_max; }

// What a workgroup without splits would do one after the other for sequence b: tiles, or with few rows slices of each of its
// eight wavefronts.
static int chunk_steps(const mixkvq_cache* c, bool few, int b, int n) {
  const SeqState& st = c->seq[b];
  const int rec = (int)(st.n_quant / c->v.cfg.R), rows = st.n_sink + st.n_res;
  if (few) return div_up(rec * (c->v.cfg.R / 32) + div_up(rows, 32) + div_up(n, 32), 8);
  return div_up(rec, chunk_tile_records(c->v)) + div_up(rows, kChunkTile) + div_up(n, kChunkTile);
}

static int splits_of(int steps, int chain) {
  const int s = div_up(steps, chain);
  return s > kChunkMaxSplits ? kChunkMaxSplits : s;
}

// The cut of a call for one kernel and tile of rows that takes the least time, and that time in microseconds.  A unit (one split of
// one tile of rows) costs its steps and a constant part.  Workgroups of one length run in rounds; of several (later rows of a
// chunk see more tokens, and the longest start first) they fill the compute units evenly until the shortest ones end.  Splits have
// to be merged, which costs a launch and their rows' traffic.  The constants fit what was measured for cuts of 1 to 258 steps, by about a
// tenth; now, a pass (28 query and 4 KV heads): 48 rows (8 sequences of 32805): 17 steps a unit 62 us, 9 steps 80, 19 steps 68; 16 rows
// (one of 32805): 5 steps 25 us, 9 steps 26, 17 steps 33; tiles (1000 after 31000 tokens): 28 steps 684 us, 14 steps 760, 126 steps 692;
// (8192 tokens, empty cache): unsplit 500 us, 32 steps 575.
static double cut_chunk(const mixkvq_cache* c, int n_max, const int32_t* n_seq, ChunkPlan* pl) {
  static const int kTry[] = {1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 14, 16, 20, 24, 28, 32, 40, 48, 56, 64};
  constexpr int kTries = sizeof kTry / sizeof kTry[0];
  static_assert(kChunkMaxSplits == 64, "the last try");
  const mixkvq_config& cfg = c->v.cfg;
  const double more = (c->v.lay.NVG > 1 ? 0.7 : 0) + (cfg.k16 ? 0.25 : 0);      // values dequantized one by one, the fp16 tier
  const double step_us = !pl->few ? 4.8 : more + (pl->rows == 16 ? 1.15 : pl->rows == 32 ? 1.65 : 2.1);
  const double fixed_us = !pl->few ? 10 : pl->rows == 16 ? 12 : pl->rows == 32 ? 16 : 22, merge_us = pl->few ? 6 : 10;
  int longest = 1, shortest = 1 << 30, chain[kTries];
  bool equal = true;      // (the longest start first only among a sequence's own row tiles)
  int64_t units[kTries] = {};
  double steps = 0;
  for (int pass = 0; pass < 2; ++pass) {
    for (int b = 0; b < cfg.B;) {
      const int n = n_new_of(n_seq, n_max, b);
      int same = 1;      // sequences with the same counts from here on
      while (b + same < cfg.B && n_new_of(n_seq, n_max, b + same) == n && c->seq[b + same] == c->seq[b]) ++same;
      if (n) {
        const int t = chunk_steps(c, pl->few, b, n);
        if (pass == 0) {
          const int t0 = chunk_steps(c, pl->few, b, 1);
          equal = equal && (longest == 1 || t == longest);
          longest = t > longest ? t : longest;
          shortest = t0 < shortest ? t0 : shortest;
        } else {
          const int64_t tiles = (int64_t)same * cfg.Hkv * div_up(n * c->v.g, pl->rows);
          const int first = pl->rows / c->v.g + 1;
          for (int i = 0; i < kTries; ++i) units[i] += tiles * splits_of(t, chain[i]);
          steps += (double)tiles * (t + (n > first ? chunk_steps(c, pl->few, b, first) : t)) / 2;
        }
      }
      b += same;
    }
    if (pass == 0)
      for (int i = 0; i < kTries; ++i) chain[i] = div_up(longest, kTry[i]);
  }
  double best = 0;
  for (int i = 0; i < kTries && kTry[i] <= longest; ++i) {
    const double rounds = (double)((units[i] + kChunkUnitsAtOnce - 1) / kChunkUnitsAtOnce) * (chain[i] * step_us + fixed_us);
    const double even = (steps * step_us + fixed_us * units[i]) / kChunkUnitsAtOnce + (equal && shortest < chain[i] ? shortest : chain[i]) * step_us + fixed_us;
    // (rounds are exact if there is one; of units of one length they are a bound from above, else hopeful)
    const bool less = units[i] <= kChunkUnitsAtOnce || (equal ? rounds < even : rounds > even);
    const double t = (less ? rounds : even) + (i ? merge_us + units[i] * pl->rows / 7000.0 : 0);
    if (i == 0 || t < best) {
      best = t;
      pl->chain = chain[i];
    }
  }
  return best;
}

// The kernel for few rows reads every record anew for each 16, 32 or 48 of them, the one with tiles of 256 rows dequantizes it once in
// LDS.  Tiles of 16 rows are the quickest ones where they leave compute units idle (35 rows: a window of 90 tokens 6.7, 8.7 and 10.9 us,
// 3000 tokens 16.1, 19.1 and 22.2, 32805 tokens 27.5, 31.8 and 37.5), of 48 where they do not (8 sequences of 32805: 85, 75 and 62 us).
// Where the tiles of 256 start to win depends on that as well: 24 sequences of 8192 tokens, 161 rows, 185 (48 rows) and 179 us; 8 of 16384,
// 161 rows, 99 and 114 us, 196 rows, 127 (32 rows) and 116 us; one of 32768, 259 rows, 54 and 80 us.
static ChunkPlan plan_chunk(const mixkvq_cache* c, int n_max, const int32_t* n_seq) {
  int most = 0;
  for (int b = 0; b < c->v.cfg.B; ++b) most = n_new_of(n_seq, n_max, b) > most ? n_new_of(n_seq, n_max, b) : most;
  const int rows = most * c->v.g;
  ChunkPlan best{false, 256, 1};
  const bool fits = chunk_few_fits(c->v);
  double us = rows > 48 || !fits ? cut_chunk(c, n_max, n_seq, &best) : 0;
  for (int r = 16; fits && rows <= kFewRows && r <= chunk_few_rows(c->v) && r - 16 < rows; r += 16) {
    ChunkPlan few{true, r, 1};
    const double t = cut_chunk(c, n_max, n_seq, &few);
    if (us == 0 || t < us) {
      us = t;
      best = few;
    }
  }
  return best;
}

// Sequences [b0, b0 + n) of the call as one launch (counts that differ in *c).  How many sequences a launch takes is up to the
// caller (next_launch).
struct ChunkLaunch { int b0, n, units, row_tiles, most; bool equal, split; };

static int units_of(const mixkvq_cache* c, const ChunkPlan& pl, int b, int n) { return n ? splits_of(chunk_steps(c, pl.few, b, n), pl.chain) : 0; }

static ChunkLaunch next_launch(const mixkvq_cache* c, const ChunkPlan& pl, int b0, int n_max, const int32_t* n_seq) {
  ChunkLaunch l{b0, 0, 0, 0, 0, true, false};
  const int B = c->v.cfg.B;
  while (b0 + l.n < B) {
    const int b = b0 + l.n, n = n_new_of(n_seq, n_max, b), u = units_of(c, pl, b, n);
    const bool equal = l.equal && c->seq[b] == c->seq[b0] && n == n_new_of(n_seq, n_max, b0);
    if (!equal && (l.n >= kChunkSeqs || l.units + u > kChunkUnits)) break;
    l.equal = equal;
    l.units += u;
    l.split = l.split || u > 1;
    l.most = n > l.most ? n : l.most;
    ++l.n;
  }
  l.row_tiles = div_up(l.most * c->v.g, pl.rows);
  return l;
}

static void fill_launch(const mixkvq_cache* c, const ChunkPlan& pl, const ChunkLaunch& l, int n_max, const int32_t* n_seq, ChunkArgs* a, ChunkCounts* counts) {
  a->b0 = l.b0;
  a->row_tiles = l.row_tiles;
  a->split = l.split;
  int units = 0;
  for (int i = 0; i < (l.equal ? 1 : l.n); ++i) {
    const SeqState& st = c->seq[l.b0 + i];
    const int n = n_new_of(n_seq, n_max, l.b0 + i), u = units_of(c, pl, l.b0 + i, n);
    const int n_rec = (int)(st.n_quant / c->v.cfg.R), n_fp16 = st.n_sink + st.n_res;
    if (l.equal) {
      a->n_rec = n_rec;
      a->n_fp16 = n_fp16;
      a->n_new = n;
      a->n_splits = u;
      return;
    }
    counts->n_rec[i] = n_rec;
    counts->n_new[i] = n;
    counts->rows_splits[i] = (uint32_t)n_fp16 | (uint32_t)u << 16;
    counts->first[i] = units;
    for (int k = 0; k < u; ++k, ++units) {
      uint32_t& word = counts->owner[units >> 2];
      word = (units & 3) ? word | (uint32_t)i << (8 * (units & 3)) : (uint32_t)i;
    }
  }
}

static size_t part_bytes(const mixkvq_cache* c, const ChunkLaunch& l, const ChunkPlan& pl) {
  return l.split ? (size_t)l.units * c->v.cfg.Hkv * l.row_tiles * pl.rows * (kD + 2) * sizeof(float) : 0;
}

static int check_counts(const mixkvq_cache* c, int n_max, const int32_t* n_seq) {
  if (!c || n_max < 0 || n_max > kChunkMaxNew) return MIXKVQ_EINVAL;
  if (n_seq)
    for (int b = 0; b < c->v.cfg.B; ++b)
      if (n_seq[b] < 0 || n_seq[b] > n_max) return MIXKVQ_EINVAL;
  // unit numbers are 32-bit
  if ((int64_t)c->v.P * ((int64_t)n_max * c->v.g / 16 + 1) * kChunkMaxSplits >= 1ll << 31) return MIXKVQ_EINVAL;
  return MIXKVQ_OK;
}

static bool rows_ok(const void* p, const int64_t* strides, int B, int heads, int n) {      // rows are moved with 16-byte accesses
  if (!p || ((uintptr_t)p & 15u) || !strides) return false;
  return (B == 1 || strides[0] % 8 == 0) && (heads == 1 || strides[1] % 8 == 0) && (n == 1 || strides[2] % 8 == 0);
}

}  // namespace mixkvq

extern "C" {

int64_t mixkvq_chunk_workspace(const mixkvq_cache* c, int32_t n_new, const int32_t* n_seq) {
  const int rc = check_counts(c, n_new, n_seq);
  if (rc != MIXKVQ_OK) return rc;
  const ChunkPlan pl = plan_chunk(c, n_new, n_seq);
  size_t most = 0;
  for (int b0 = 0; b0 < c->v.cfg.B;) {
    const ChunkLaunch l = next_launch(c, pl, b0, n_new, n_seq);
    const size_t bytes = part_bytes(c, l, pl);
    most = bytes > most ? bytes : most;
    b0 += l.n;
  }
  return (int64_t)most;
}

int mixkvq_chunk_attention(mixkvq_cache* c, const void* q, const int64_t q_strides[3], const void* k_new, const void* v_new,
                           const int64_t kv_strides[3], int32_t n_new, const int32_t* n_seq, void* out,
                           const int64_t out_strides[3], float* lse, float scale, int32_t accumulate_q, void* workspace,
                           int64_t workspace_bytes, void* stream) {
  int rc = check_counts(c, n_new, n_seq);
  if (rc != MIXKVQ_OK) return rc;
  if (n_new == 0) return MIXKVQ_OK;
  const mixkvq_config& cfg = c->v.cfg;
  if (!rows_ok(q, q_strides, cfg.B, cfg.Hq, n_new) || !rows_ok(out, out_strides, cfg.B, cfg.Hq, n_new)) return MIXKVQ_EINVAL;
  if (!rows_ok(k_new, kv_strides, cfg.B, cfg.Hkv, n_new) || !rows_ok(v_new, kv_strides, cfg.B, cfg.Hkv, n_new)) return MIXKVQ_EINVAL;
  if (!(scale > 0.f)) scale = 1.0f / sqrtf((float)kD);
  if (!(scale < INFINITY)) return MIXKVQ_EINVAL;
  if (n_new > 1 && kv_strides[2] != (int32_t)kv_strides[2]) return MIXKVQ_EINVAL;      // (row numbers times it are formed by a 32-bit multiply)
  if ((workspace && ((uintptr_t)workspace & 15u)) || workspace_bytes < 0) return MIXKVQ_EINVAL;
  const ChunkPlan pl = plan_chunk(c, n_new, n_seq);
  ChunkArgs a{};
  a.q = (const __half*)q;
  a.k = (const __half*)k_new;
  a.v = (const __half*)v_new;
  a.out = (__half*)out;
  a.lse = lse;
  a.qs = Strides3{q_strides[0], q_strides[1], q_strides[2]};
  a.kvs = Strides3{kv_strides[0], kv_strides[1], kv_strides[2]};
  a.os = Strides3{out_strides[0], out_strides[1], out_strides[2]};
  a.n_max = n_new;
  a.scale = scale;
  a.part = (float*)workspace;
  const hipStream_t s = (hipStream_t)stream;
  const CacheView& v = c->v;
  const Layout& lay = v.lay;
  a.blocks = v.blocks;
  a.table = v.table;
  a.res_k = v.res_k;
  a.res_v = v.res_v;
  a.NB = v.NB;
  a.RW = v.RW;
  a.Hkv = cfg.Hkv;
  a.Hq = cfg.Hq;
  a.g = v.g;
  a.bf16 = cfg.in_dtype != 0;
  a.R = cfg.R;
  a.Gk = cfg.Gk;
  a.inv_r = 65536 / cfg.R + 1;
  a.inv_gk = 65536 / cfg.Gk + 1;
  a.nvg_bits = 31 - __builtin_clz(lay.NVG);
  a.k4 = cfg.k4;
  a.k16 = cfg.k16;
  a.rec_bytes = lay.rec_bytes;
  a.tile_rec = chunk_tile_records(v);
  a.NLp = lay.NLp;
  a.Wlo = lay.Wlo;
  a.W4 = lay.W4;
  a.NVG = lay.NVG;
  a.interleave = lay.v_interleave;
  a.off_idx = lay.off_idx;
  a.off_kmax = lay.off_kmax;
  a.off_klo_s = lay.off_klo_s;
  a.off_klo_z = lay.off_klo_z;
  a.off_k4_s = lay.off_k4_s;
  a.off_k4_z = lay.off_k4_z;
  a.off_klo = lay.off_klo;
  a.off_k4 = lay.off_k4;
  a.off_k16 = lay.off_k16;
  a.off_v = lay.off_v;
  a.off_v_s = lay.off_v_s;
  a.off_v_z = lay.off_v_z;
  for (int b0 = 0; b0 < cfg.B;) {      // everything is checked before the first launch
    const ChunkLaunch l = next_launch(c, pl, b0, n_new, n_seq);
    const size_t bytes = part_bytes(c, l, pl);
    if (bytes && (!workspace || bytes > (size_t)workspace_bytes)) return MIXKVQ_ESCRATCH;
    b0 += l.n;
  }
  for (int b0 = 0; b0 < cfg.B;) {
    const ChunkLaunch l = next_launch(c, pl, b0, n_new, n_seq);
    b0 += l.n;
    if (l.units == 0) continue;
    ChunkCounts counts;
    fill_launch(c, pl, l, n_new, n_seq, &a, &counts);
    c->last_chunk = pl.rows;
    MIXKVQ_TRY_HIP(launch_chunk(a, l.equal ? nullptr : &counts, l.units, l.n, pl.few, pl.rows, s));
    if (accumulate_q) MIXKVQ_TRY_HIP(launch_chunk_books(v, a, l.equal ? nullptr : &counts, l.n, l.most, s));
  }
  return MIXKVQ_OK;
}

int mixkvq_chunk_path(const mixkvq_cache* c) { return c ? c->last_chunk : MIXKVQ_EINVAL; }

}  // extern "C"
