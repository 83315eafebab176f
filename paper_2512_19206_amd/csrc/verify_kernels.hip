// Verification of drafted tokens against the target's probabilities (mixkvq_verify_draft): which drafts stay, and the token
// that follows them, drawn from what the target has more than the draft.
//
// A call reads one row of the vocabulary per sequence (two with draft probabilities), so it is bound by memory for a batch and by
// latencies in line (counts, drafts, their probabilities, the row, its drawn part) for a single sequence.  The row depends on the
// verdict, which every wavefront forms for itself from at most 64 pairs of probabilities; the row is then cut into parts, one
// wavefront each, whose sums one workgroup searches for the part that holds the drawn point and goes over once more.  All sums are
// binary64: the point is compared with sums over the whole vocabulary, where binary32 would be off by the width of a token.
#include "cache_state.h"

namespace mixkvq {

constexpr int kVerifyThreads = 256, kAloneThreads = 1024;
constexpr int kVerifyMaxSpans = 64;
constexpr int kVerifyMaxV = 1 << 30;     // (token numbers behind a row's end stay 32-bit)
constexpr int kParts = kVerifyThreads / 64;      // of a span, one to a wavefront
constexpr int kVerifyMaxDraft = 64;      // a wavefront forms the verdict

struct VerifyArgs {
  const float *p, *q;                    // q: nullptr, all of a draft's probability on its token
  int64_t pb, pt, qb, qt;                // strides: sequence, position
  const int32_t *draft, *n_seq;
  const float *u, *u_next;
  int32_t *n_accepted, *tokens;
  double2* part;                         // [B][spans * kParts]: sums of the remainders, of the target's probabilities
  int32_t n, V, spans;
};

// Drafts of sequence b that stay, in every lane of a wavefront: i stays if all before it do and u_i q_i < p_i (the product
// of two binary32 numbers is exact in binary64).
__device__ __forceinline__ int accepted(const VerifyArgs& a, int b, int n) {
  const int i = threadIdx.x & 63;
  bool ok = false;
  if (i < n) {
    const int t = a.draft[(size_t)b * a.n + i];
    if (t >= 0 && t < a.V) {             // (a token outside the vocabulary is never read and never stays)
      const double q = a.q ? (double)a.q[b * a.qb + i * a.qt + t] : 1.0;
      ok = (double)a.u[(size_t)b * a.n + i] * q < (double)a.p[b * a.pb + i * a.pt + t];
    }
  }
  return __ffsll((long long)~__ballot(ok)) - 1;      // (at least one lane says no where n < 64)
}

__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int b) {
  const int n = a.n_seq ? a.n_seq[b] : a.n;
  return n < 0 ? 0 : n > a.n ? a.n : n;
}

// Weights of one position: the remainder max(p - q, 0) after a rejected draft, else the target's own.
struct Row {
  const float *p, *q;
  int token;                             // one-hot draft: the token with all of its probability, else -1
  bool rejected;
  __device__ __forceinline__ double rest(int t, float pv, float qv) const {
    const double d = (double)pv - (q ? (double)qv : t == token ? 1.0 : 0.0);
    return d > 0.0 ? d : 0.0;            // (also takes care of NaN)
  }
};

__device__ __forceinline__ Row row_of(const VerifyArgs& a, int b, int n, int stay) {
  Row r;
  r.p = a.p + b * a.pb + stay * a.pt;
  r.rejected = stay < n;
  r.q = r.rejected && a.q ? a.q + b * a.qb + stay * a.qt : nullptr;
  r.token = r.rejected && !a.q ? a.draft[(size_t)b * a.n + stay] : -1;
  return r;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// A row is cut into a.spans * kParts parts of whole quads of tokens (the last one ends at V), one to a wavefront.
__device__ __forceinline__ int part_begin(const VerifyArgs& a, int i) {
  const int64_t quads = ((int64_t)a.V + 3) / 4;
  const int64_t t = quads * i / (a.spans * kParts) * 4;
  return t < a.V ? (int)t : a.V;
}

// Four neighbouring weights from any address of a binary32 number (16-byte loads need no more).
struct __attribute__((packed, aligned(4))) Quad { float x[4]; };

// Sums of the part's tokens, eight 16-byte loads of a lane in flight (64 rows of 152064 with draft probabilities: 29 us with the second
// launch; one 4-byte load after the other took 59).
template <bool HAS_Q>
__device__ __forceinline__ double2 part_sums(const Row& row, int begin, int end) {
  double rest = 0.0, whole = 0.0;
  const int lane = threadIdx.x & 63, quads = (end - begin) >> 2;
  auto add = [&](int t, float p, float q) {
    rest += row.rest(t, p, q);
    whole += p > 0.f ? (double)p : 0.0;
  };
  const Quad* p = reinterpret_cast<const Quad*>(row.p + begin);
  const Quad* q = reinterpret_cast<const Quad*>((HAS_Q ? row.q : row.p) + begin);
  int i = lane;
  for (; i + 3 * 64 < quads; i += 4 * 64) {
    Quad x[4], y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = p[i + 64 * k];
      if constexpr (HAS_Q) y[k] = q[i + 64 * k];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) add(begin + 4 * (i + 64 * k) + e, x[k].x[e], HAS_Q ? y[k].x[e] : 0.f);
  }
  for (; i < quads; i += 64) {
    const Quad x = p[i];
    Quad y{};
    if constexpr (HAS_Q) y = q[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) add(begin + 4 * i + e, x.x[e], y.x[e]);
  }
  const int t = begin + 4 * quads + lane;
  if (t < end) add(t, row.p[t], HAS_Q ? row.q[t] : 0.f);
  return make_double2(wave_sum(rest), wave_sum(whole));
}

__device__ __forceinline__ double2 sums_of(const VerifyArgs& a, const Row& row, int part) {
  const int begin = part_begin(a, part), end = part_begin(a, part + 1);
  return row.q ? part_sums<true>(row, begin, end) : part_sums<false>(row, begin, end);
}

__device__ __forceinline__ int verdict(const VerifyArgs& a, int b, int n) {
  const int stay = __builtin_amdgcn_readfirstlane(accepted(a, b, n));
  return stay < 0 || stay > n ? n : stay;
}

__global__ void __launch_bounds__(kVerifyThreads) verify_sum_kernel(VerifyArgs a) {
  const int b = blockIdx.x / a.spans, s = blockIdx.x % a.spans, part = s * kParts + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = drafts_of(a, b), lane = threadIdx.x & 63;
  const int stay = verdict(a, b, n);      // (every wavefront for itself)
  if (s == 0 && threadIdx.x == 0) a.n_accepted[b] = stay;
  const double2 x = sums_of(a, row_of(a, b, n, stay), part);
  if (lane == 0) a.part[(size_t)b * a.spans * kParts + part] = x;
}

// ALONE: the only launch, its sixteen wavefronts form the sums of sixteen parts first.
template <bool ALONE, int kThreads>
__global__ void __launch_bounds__(kThreads) verify_pick_kernel(VerifyArgs a) {
  static_assert(!ALONE || kThreads == kAloneThreads, "sixteen parts");
  __shared__ double sBefore;
  __shared__ double sWave[kThreads / 64];
  __shared__ int sPart, sByRest, sFirst, sLast;
  __shared__ double sPoint;
  __shared__ double2 sSums[ALONE ? kThreads / 64 : 1];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, n = drafts_of(a, b), parts = a.spans * kParts;
  const int stay = ALONE ? verdict(a, b, n) : a.n_accepted[b];
  const Row row = row_of(a, b, n, stay);
  const double2* sums = a.part + (size_t)b * parts;
  if constexpr (ALONE) {
    if (tid == 0) a.n_accepted[b] = stay;
    const double2 x = sums_of(a, row, __builtin_amdgcn_readfirstlane(tid >> 6));
    if (lane == 0) sSums[tid >> 6] = x;
    __syncthreads();
    sums = sSums;
  }
  // The point u W, and the first part whose sums pass it: one wavefront, four parts to a lane.
  if (tid < 64) {
    double2 x[kVerifyMaxSpans * kParts / 64];
    double rest = 0.0, whole = 0.0;
#pragma unroll
    for (int k = 0; k < kVerifyMaxSpans * kParts / 64; ++k) {
      const int i = 4 * lane + k;
      x[k] = i < parts ? sums[i] : make_double2(0.0, 0.0);
      rest += x[k].x;
      whole += x[k].y;
    }
    double upto = rest, upto_whole = whole;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double u = __shfl_up(upto, o), v = __shfl_up(upto_whole, o);
      if (lane >= o) {
        upto += u;
        upto_whole += v;
      }
    }
    const double all = __shfl(upto, 63);
    const bool by_rest = row.rejected && all > 0.0;      // a remainder that is 0 everywhere: the target's own probabilities
    const double point = (double)a.u_next[b] * (by_rest ? all : __shfl(upto_whole, 63));
    double before = by_rest ? upto - rest : upto_whole - whole, last_before = 0.0, found_before = 0.0;
    int found = -1, last = -1;
#pragma unroll
    for (int k = 0; k < kVerifyMaxSpans * kParts / 64; ++k) {
      const double w = by_rest ? x[k].x : x[k].y;
      if (w > 0.0) {
        last = 4 * lane + k;
        last_before = before;
        if (found < 0 && before + w > point) {
          found = 4 * lane + k;
          found_before = before;
        }
      }
      before += w;
    }
    const unsigned long long hit = __ballot(found >= 0), some = __ballot(last >= 0);
    const int from = hit ? __ffsll((long long)hit) - 1 : some ? 63 - __clzll((long long)some) : 0;      // (no hit: u = 1; none: nothing above 0)
    if (lane == from) {
      sPart = hit ? found : some ? last : 0;
      sBefore = hit ? found_before : last_before;
      sPoint = point;
      sByRest = by_rest;
      sFirst = a.V;
      sLast = -1;
    }
  }
  __syncthreads();
  const bool by_rest = sByRest != 0;
  const double point = sPoint;
  double before = sBefore;
  const int begin = part_begin(a, sPart), end = part_begin(a, sPart + 1);
  // Inside the part: four neighbouring tokens to a thread, sums over the threads before it.
#pragma unroll 1
  for (int first = begin; first < end; first += 4 * kThreads) {
    const int t0 = first + 4 * tid;
    double w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = t0 + e < end ? t0 + e : end - 1;
      const float p = row.p[t], q = row.q ? row.q[t] : 0.f;
      w[e] = t0 + e >= end ? 0.0 : by_rest ? row.rest(t, p, q) : p > 0.f ? (double)p : 0.0;
    }
    const double mine = (w[0] + w[1]) + (w[2] + w[3]);
    double upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 63) sWave[tid >> 6] = upto;
    __syncthreads();
    double at = before + (upto - mine), all = 0.0;
#pragma unroll
    for (int k = 0; k < kThreads / 64; ++k) {
      if (k < tid >> 6) at += sWave[k];
      all += sWave[k];
    }
    int hit = a.V, some = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      at += w[e];
      if (w[e] > 0.0) {
        some = t0 + e;
        if (at > point && hit == a.V) hit = t0 + e;
      }
    }
    if (some >= 0) atomicMax(&sLast, some);
    if (hit < a.V) atomicMin(&sFirst, hit);
    before += all;
    __syncthreads();
    if (sFirst < a.V) break;
  }
  const int token = sFirst < a.V ? sFirst : sLast < 0 ? 0 : sLast;
  int32_t* out = a.tokens + (size_t)b * (a.n + 1);
  if (tid <= a.n) out[tid] = tid < stay ? a.draft[(size_t)b * a.n + tid] : tid == stay ? token : -1;
}

// One workgroup takes a whole row, and a call one launch, where rows are short (1 row of 1000: 9.3 us, of 16384: 11.6, of 32000: 16.0 and
// with two launches 11.0; 16 rows of 16384: 14.2 and 14.5) or many enough to fill the chip (256 rows of 32000: 31.0 and 36.5 us, of
// 65536: 35.5 and 46.8; 64 rows of 32000: 20.1 and 20.7).
static bool verify_alone(int B, int V) { return V <= 16384 || (B >= 128 && V <= 65536); }

// Spans of a row: enough workgroups for the chip, none of less than 1 024 tokens.
static int verify_spans(int B, int V) {
  if (verify_alone(B, V)) return kAloneThreads / kVerifyThreads;
  int s = (2048 + B - 1) / B;
  if (s > V / 1024) s = V / 1024;
  if (s > kVerifyMaxSpans) s = kVerifyMaxSpans;
  return s < 1 ? 1 : s;
}

}  // namespace mixkvq

using namespace mixkvq;

extern "C" {

int64_t mixkvq_verify_workspace(int32_t B, int32_t V) {
  if (B < 1 || B > (1 << 20) || V < 1 || V > kVerifyMaxV) return MIXKVQ_EINVAL;
  return (int64_t)B * verify_spans(B, V) * kParts * (int64_t)sizeof(double2);
}

int mixkvq_verify_draft(int32_t B, int32_t n_draft, int32_t V, const float* p_target, const int64_t p_target_strides[2],
                        const float* p_draft, const int64_t p_draft_strides[2], const int32_t* draft, const int32_t* n_seq,
                        const float* u_accept, const float* u_next, int32_t* n_accepted, int32_t* tokens, void* workspace,
                        int64_t workspace_bytes, void* stream) {
  if (B < 1 || B > (1 << 20) || V < 1 || V > kVerifyMaxV || n_draft < 0 || n_draft > kVerifyMaxDraft) return MIXKVQ_EINVAL;
  if (!p_target || !p_target_strides || !u_next || !n_accepted || !tokens) return MIXKVQ_EINVAL;
  if (n_draft > 0 && (!draft || !u_accept)) return MIXKVQ_EINVAL;
  if (p_draft && !p_draft_strides) return MIXKVQ_EINVAL;
  for (const void* x : {(const void*)p_target, (const void*)p_draft, (const void*)draft, (const void*)n_seq, (const void*)u_accept, (const void*)u_next, (const void*)n_accepted, (const void*)tokens})
    if ((uintptr_t)x & 3u) return MIXKVQ_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 15u)) return MIXKVQ_EINVAL;
  VerifyArgs a{};
  a.spans = verify_spans(B, V);
  if (workspace_bytes < (int64_t)B * a.spans * kParts * (int64_t)sizeof(double2)) return MIXKVQ_ESCRATCH;
  a.p = p_target;
  a.q = n_draft > 0 ? p_draft : nullptr;
  a.pb = p_target_strides[0];
  a.pt = p_target_strides[1];
  if (a.q) {
    a.qb = p_draft_strides[0];
    a.qt = p_draft_strides[1];
  }
  a.draft = draft;
  a.n_seq = n_seq;
  a.u = u_accept;
  a.u_next = u_next;
  a.n_accepted = n_accepted;
  a.tokens = tokens;
  a.part = (double2*)workspace;
  a.n = n_draft;
  a.V = V;
  const hipStream_t s = (hipStream_t)stream;
  if (verify_alone(B, V)) {
    verify_pick_kernel<true, kAloneThreads><<<B, kAloneThreads, 0, s>>>(a);
  } else {
    verify_sum_kernel<<<B * a.spans, kVerifyThreads, 0, s>>>(a);
    MIXKVQ_TRY_HIP(hipGetLastError());
    // (a part of four tokens a thread is gone over in one turn: 32000 tokens 11.0 us with 256 threads, 13.5 with 1024; 500000, with
    // parts of 1953 tokens, 17.4 and 14.8)
    if (V / (a.spans * kParts) < 1024) verify_pick_kernel<false, 256><<<B, 256, 0, s>>>(a);
    else verify_pick_kernel<false, 1024><<<B, 1024, 0, s>>>(a);
  }
  MIXKVQ_TRY_HIP(hipGetLastError());
  return MIXKVQ_OK;
}

}  // extern "C"
