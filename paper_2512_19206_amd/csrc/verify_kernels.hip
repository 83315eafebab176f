// Verification of drafted tokens against the target's probabilities (mixkvq_verify_draft): which drafts stay, and the token
// that follows them, drawn from what the target has more than the draft.
//
// A call reads one row of the vocabulary per sequence (two with draft probabilities), so it is bound by memory for a batch and by
// its two launches for a single sequence.  The row depends on the verdict, which every workgroup forms for itself from at most
// 64 pairs of probabilities; the row is then cut into spans, one workgroup each, whose sums the second launch searches for the span
// that holds the drawn point and goes over once more.  All sums are binary64: the point is compared with sums over the
// whole vocabulary, where binary32 would be off by the width of a token.
#include "cache_state.h"

namespace mixkvq {

constexpr int kVerifyThreads = 256, kPickThreads = 1024;
constexpr int kVerifyMaxSpans = 64;
constexpr int kVerifyMaxDraft = 64;      // one wavefront forms the verdict

struct VerifyArgs {
  const float *p, *q;                    // q: nullptr, all of a draft's probability on its token
  int64_t pb, pt, qb, qt;                // strides: sequence, position
  const int32_t *draft, *n_seq;
  const float *u, *u_next;
  int32_t *n_accepted, *tokens;
  double2* part;                         // [B][spans]: sums of the remainders, of the target's probabilities
  int32_t n, V, spans;
};

// Drafts of sequence b that stay, in every lane of the first wavefront: i stays if all before it do and u_i q_i < p_i (the product
// of two binary32 numbers is exact in binary64).
__device__ __forceinline__ int accepted(const VerifyArgs& a, int b, int n) {
  const int i = threadIdx.x;
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

__device__ __forceinline__ int span_begin(const VerifyArgs& a, int s) { return (int)((int64_t)a.V * s / a.spans); }

__global__ void __launch_bounds__(kVerifyThreads) verify_sum_kernel(VerifyArgs a) {
  __shared__ int sStay;
  __shared__ double2 sSum[kVerifyThreads / 64];
  const int b = blockIdx.x / a.spans, s = blockIdx.x % a.spans, tid = threadIdx.x;
  const int n = drafts_of(a, b);
  if (tid < 64) {
    int stay = accepted(a, b, n);
    stay = stay < 0 || stay > n ? n : stay;
    if (tid == 0) {
      sStay = stay;
      if (s == 0) a.n_accepted[b] = stay;
    }
  }
  __syncthreads();
  const Row row = row_of(a, b, n, sStay);
  double rest = 0.0, whole = 0.0;
  const int end = span_begin(a, s + 1);
#pragma unroll 8
  for (int t = span_begin(a, s) + tid; t < end; t += kVerifyThreads) {
    const float p = row.p[t], q = row.q ? row.q[t] : 0.f;
    rest += row.rest(t, p, q);
    whole += p > 0.f ? (double)p : 0.0;
  }
  rest = wave_sum(rest);
  whole = wave_sum(whole);
  if ((tid & 63) == 0) sSum[tid >> 6] = make_double2(rest, whole);
  __syncthreads();
  if (tid == 0) {
    double2 x = sSum[0];
    for (int w = 1; w < kVerifyThreads / 64; ++w) x = make_double2(x.x + sSum[w].x, x.y + sSum[w].y);
    a.part[(size_t)b * a.spans + s] = x;
  }
}

__global__ void __launch_bounds__(kPickThreads) verify_pick_kernel(VerifyArgs a) {
  __shared__ double2 sPart[kVerifyMaxSpans];
  __shared__ double sWave[kPickThreads / 64];
  __shared__ int sFirst, sLast;
  const int b = blockIdx.x, tid = threadIdx.x, n = drafts_of(a, b), stay = a.n_accepted[b];
  if (tid < a.spans) sPart[tid] = a.part[(size_t)b * a.spans + tid];
  if (tid == 0) {
    sFirst = a.V;
    sLast = -1;
  }
  const Row row = row_of(a, b, n, stay);
  __syncthreads();
  // the point u W, and the first span whose sums pass it (every thread for itself: at most 64 adds)
  double rest = 0.0, whole = 0.0;
  for (int s = 0; s < a.spans; ++s) {
    rest += sPart[s].x;
    whole += sPart[s].y;
  }
  const bool by_rest = row.rejected && rest > 0.0;      // a remainder that is 0 everywhere: the target's own probabilities
  const double point = (double)a.u_next[b] * (by_rest ? rest : whole);
  double before = 0.0;
  int span = -1, last = 0;
  double last_before = 0.0;
  for (int s = 0; s < a.spans; ++s) {
    const double x = by_rest ? sPart[s].x : sPart[s].y;
    if (x > 0.0) {
      last = s;
      last_before = before;
      if (before + x > point) {
        span = s;
        break;
      }
    }
    before += x;
  }
  if (span < 0) {      // (u = 1, or nothing above 0)
    span = last;
    before = last_before;
  }
  // inside the span: neighbouring tokens to a thread, sums over the threads before it
  const int begin = span_begin(a, span), len = span_begin(a, span + 1) - begin, each = (len + kPickThreads - 1) / kPickThreads;
  const int t0 = begin + tid * each < begin + len ? begin + tid * each : begin + len;
  const int t1 = t0 + each < begin + len ? t0 + each : begin + len;
  auto weight = [&](int t) {
    const float p = row.p[t];
    return by_rest ? row.rest(t, p, row.q ? row.q[t] : 0.f) : p > 0.f ? (double)p : 0.0;
  };
  double mine = 0.0;
  for (int t = t0; t < t1; ++t) mine += weight(t);
  double upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double x = __shfl_up(upto, o);
    if ((tid & 63) >= o) upto += x;
  }
  if ((tid & 63) == 63) sWave[tid >> 6] = upto;
  __syncthreads();
  double at = before;
  for (int w = 0; w < tid >> 6; ++w) at += sWave[w];
  at += upto - mine;
  for (int t = t0; t < t1; ++t) {
    const double w = weight(t);
    at += w;
    if (w > 0.0) {
      atomicMax(&sLast, t);
      if (at > point) {
        atomicMin(&sFirst, t);
        break;
      }
    }
  }
  __syncthreads();
  const int token = sFirst < a.V ? sFirst : sLast < 0 ? 0 : sLast;
  int32_t* out = a.tokens + (size_t)b * (a.n + 1);
  if (tid <= a.n) out[tid] = tid < stay ? a.draft[(size_t)b * a.n + tid] : tid == stay ? token : -1;
}

// Spans of a row: enough workgroups for the chip, none of less than 2 048 tokens.
static int verify_spans(int B, int V) {
  int s = (1024 + B - 1) / B;
  if (s > V / 2048) s = V / 2048;
  if (s > kVerifyMaxSpans) s = kVerifyMaxSpans;
  return s < 1 ? 1 : s;
}

}  // namespace mixkvq

using namespace mixkvq;

extern "C" {

int64_t mixkvq_verify_workspace(int32_t B, int32_t V) {
  if (B < 1 || B > (1 << 20) || V < 1) return MIXKVQ_EINVAL;
  return (int64_t)B * verify_spans(B, V) * (int64_t)sizeof(double2);
}

int mixkvq_verify_draft(int32_t B, int32_t n_draft, int32_t V, const float* p_target, const int64_t p_target_strides[2],
                        const float* p_draft, const int64_t p_draft_strides[2], const int32_t* draft, const int32_t* n_seq,
                        const float* u_accept, const float* u_next, int32_t* n_accepted, int32_t* tokens, void* workspace,
                        int64_t workspace_bytes, void* stream) {
  if (B < 1 || B > (1 << 20) || V < 1 || n_draft < 0 || n_draft > kVerifyMaxDraft) return MIXKVQ_EINVAL;
  if (!p_target || !p_target_strides || !u_next || !n_accepted || !tokens) return MIXKVQ_EINVAL;
  if (n_draft > 0 && (!draft || !u_accept)) return MIXKVQ_EINVAL;
  if (p_draft && !p_draft_strides) return MIXKVQ_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 15u)) return MIXKVQ_EINVAL;
  VerifyArgs a{};
  a.spans = verify_spans(B, V);
  if (workspace_bytes < (int64_t)B * a.spans * (int64_t)sizeof(double2)) return MIXKVQ_ESCRATCH;
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
  verify_sum_kernel<<<B * a.spans, kVerifyThreads, 0, s>>>(a);
  MIXKVQ_TRY_HIP(hipGetLastError());
  verify_pick_kernel<<<B, kPickThreads, 0, s>>>(a);
  MIXKVQ_TRY_HIP(hipGetLastError());
  return MIXKVQ_OK;
}

}  // extern "C"
