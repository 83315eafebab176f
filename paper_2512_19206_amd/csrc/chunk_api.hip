// mixkvq_chunk_attention: argument checks, and how a launch's work is cut into workgroups.
#include <math.h>
#include <stdlib.h>
#include "cache_state.h"
#include "chunk.h"

using namespace mixkvq;

namespace mixkvq {

constexpr int kChunkUnitsAtOnce = 256;      // one workgroup to a compute unit (its tiles fill the LDS)
constexpr int kChunkMaxNew = 1 << 20;

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

static ChunkPlan plan_chunk(const mixkvq_cache* c, int n_max, const int32_t* n_seq) {
  const mixkvq_config& cfg = c->v.cfg;
  int most = 0;
  for (int b = 0; b < cfg.B; ++b) most = n_new_of(n_seq, n_max, b) > most ? n_new_of(n_seq, n_max, b) : most;
  ChunkPlan pl{};
  const int rows = most * c->v.g;
  static const int few_rows = getenv("MIXKVQ_FEW") ? atoi(getenv("MIXKVQ_FEW")) : 96;
  pl.few = rows <= few_rows && chunk_few_fits(c->v);
  if (pl.few) pl.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 48;
  else pl.rows = rows <= 64 ? 64 : rows <= 128 ? 128 : 256;
  // The splits' length that takes the least time: rounds of workgroups times what one does, its steps and a constant part, and
  // more where the splits have to be merged.
  int longest = 1;
  for (int b = 0; b < cfg.B; ++b) {
    const int n = n_new_of(n_seq, n_max, b), t = n ? chunk_steps(c, pl.few, b, n) : 0;
    longest = t > longest ? t : longest;
  }
  double best = 0;
  pl.chain = longest;
  for (int s = 1; s <= kChunkMaxSplits && s <= longest; ++s) {
    const int chain = div_up(longest, s);
    if (s > 1 && chain == div_up(longest, s - 1)) continue;
    int64_t units = 0;
    for (int b = 0; b < cfg.B; ++b) {
      const int n = n_new_of(n_seq, n_max, b);
      if (n) units += (int64_t)cfg.Hkv * div_up(n * c->v.g, pl.rows) * splits_of(chunk_steps(c, pl.few, b, n), chain);
    }
    const double t = (double)((units + kChunkUnitsAtOnce - 1) / kChunkUnitsAtOnce) * (chain + 3) + (s > 1 ? 4 : 0);
    if (s == 1 || t < best) {
      best = t;
      pl.chain = chain;
    }
  }
  return pl;
}

// Sequences [b0, b0 + n) of the call as one launch.
static ChunkLaunch fill_launch(const mixkvq_cache* c, const ChunkPlan& pl, int b0, int n, int n_max, const int32_t* n_seq, bool* split) {
  ChunkLaunch l{};
  l.b0 = b0;
  l.n_seq = n;
  l.tile_rec = chunk_tile_records(c->v);
  int units = 0, same = -1;
  *split = false;
  for (int i = 0; i < n; ++i) {
    const SeqState& st = c->seq[b0 + i];
    const int nn = n_new_of(n_seq, n_max, b0 + i);
    const int splits = nn ? splits_of(chunk_steps(c, pl.few, b0 + i, nn), pl.chain) : 1;
    const int u = c->v.cfg.Hkv * div_up(nn * c->v.g, pl.rows) * splits;
    l.n_rec[i] = (int)(st.n_quant / c->v.cfg.R);
    l.n_new[i] = nn;
    l.rows_splits[i] = (uint32_t)(st.n_sink + st.n_res) | (uint32_t)splits << 16;
    l.first_unit[i] = units;
    units += u;
    same = same == -1 ? u : same == u ? u : 0;
    *split = *split || splits > 1;
  }
  l.n_units = units;
  l.same_units = same > 0 ? same : 0;
  return l;
}

static size_t launch_part_bytes(const ChunkLaunch& l, const ChunkPlan& pl) { return (size_t)l.n_units * pl.rows * (kD + 2) * sizeof(float); }

static int check_counts(const mixkvq_cache* c, int n_max, const int32_t* n_seq) {
  if (!c || n_max < 0 || n_max > kChunkMaxNew) return MIXKVQ_EINVAL;
  if (n_seq)
    for (int b = 0; b < c->v.cfg.B; ++b)
      if (n_seq[b] < 0 || n_seq[b] > n_max) return MIXKVQ_EINVAL;
  // unit numbers are 32-bit
  if ((int64_t)c->v.P * ((int64_t)n_max * c->v.g / 16 + 1) * kChunkMaxSplits >= 1ll << 31) return MIXKVQ_EINVAL;
  return MIXKVQ_OK;
}

static bool rows_ok(const void* p, const int64_t* strides) {      // rows are moved with 16-byte accesses
  if (!p || ((uintptr_t)p & 15u) || !strides) return false;
  for (int i = 0; i < 3; ++i)
    if (strides[i] % 8 != 0) return false;
  return true;
}

}  // namespace mixkvq

extern "C" {

int64_t mixkvq_chunk_workspace(const mixkvq_cache* c, int32_t n_new, const int32_t* n_seq) {
  const int rc = check_counts(c, n_new, n_seq);
  if (rc != MIXKVQ_OK) return rc;
  const ChunkPlan pl = plan_chunk(c, n_new, n_seq);
  size_t most = 0;
  for (int b0 = 0; b0 < c->v.cfg.B; b0 += kChunkSeqs) {
    const int n = c->v.cfg.B - b0 < kChunkSeqs ? c->v.cfg.B - b0 : kChunkSeqs;
    bool split;
    const ChunkLaunch l = fill_launch(c, pl, b0, n, n_new, n_seq, &split);
    const size_t bytes = split ? launch_part_bytes(l, pl) : 0;
    most = bytes > most ? bytes : most;
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
  if (!rows_ok(q, q_strides) || !rows_ok(k_new, kv_strides) || !rows_ok(v_new, kv_strides) || !rows_ok(out, out_strides)) return MIXKVQ_EINVAL;
  if (!(scale > 0.f)) scale = 1.0f / sqrtf((float)kD);
  if (!(scale < INFINITY)) return MIXKVQ_EINVAL;
  const mixkvq_config& cfg = c->v.cfg;
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
  for (int b0 = 0; b0 < cfg.B; b0 += kChunkSeqs) {      // everything is checked before the first launch
    const int n = cfg.B - b0 < kChunkSeqs ? cfg.B - b0 : kChunkSeqs;
    bool split;
    const ChunkLaunch l = fill_launch(c, pl, b0, n, n_new, n_seq, &split);
    if (split && (!workspace || launch_part_bytes(l, pl) > (size_t)workspace_bytes)) return MIXKVQ_ESCRATCH;
  }
  for (int b0 = 0; b0 < cfg.B; b0 += kChunkSeqs) {
    const int n = cfg.B - b0 < kChunkSeqs ? cfg.B - b0 : kChunkSeqs;
    bool split;
    const ChunkLaunch l = fill_launch(c, pl, b0, n, n_new, n_seq, &split);
    if (l.n_units == 0) continue;
    MIXKVQ_TRY_HIP(launch_chunk(c->v, a, l, pl.few, pl.rows, split, s));
    if (accumulate_q) MIXKVQ_TRY_HIP(launch_chunk_books(c->v, a, l, s));
  }
  return MIXKVQ_OK;
}

}  // extern "C"
