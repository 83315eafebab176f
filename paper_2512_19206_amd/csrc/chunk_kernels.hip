// Attention of a chunk of new tokens over the mixed-precision cache and over the chunk itself, causally (Section 3.1, Eq. 1,
// with keys and values dequantized by Eq. 3).
//
// One workgroup of eight wavefronts takes a tile of query rows (a row is one query head at one new token; the g heads of
// a KV head share its keys) and walks over the tokens in tiles of 128: packed records, then the fp16 rows of the cache, then
// the chunk's own keys and values.  Both products run on the matrix cores in the transposed form, S^T = K Q^T and
// O^T = V^T P^T, 32 tokens (channels) by 32 rows at a time: a lane then holds one row's scores, so that the softmax needs
// one exchange between the two halves of the wavefront, and the weights P go into the second product from the registers in
// which the first one left them.
#include <type_traits>
#include "chunk.h"

namespace mixkvq {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int kChunkThreads = 512;
constexpr int kRowBytes = 256;                                   // one row of a tile: 128 halves
constexpr int kKeyBytes = (kChunkTile + 1) * kRowBytes;          // keys, and a row that takes what belongs nowhere
constexpr int kValueBytes = kChunkTile * kRowBytes;
constexpr int kTileBytes = kKeyBytes + kValueBytes;
constexpr int kScaleRow = kChunkTile + 8;                        // halves per value group in the table of value scales
constexpr int kOffRaw = 2 * kTileBytes;
constexpr int kOffScale = kOffRaw + kMaxRec;                     // [8][kScaleRow] scales, then zero-points
constexpr int kOffMap = kOffScale + 2 * 8 * kScaleRow * 2;       // [2][kChunkRecords][128] rows of the tile by channel place
constexpr int kLdsBytes = kOffMap + 2 * kChunkRecords * kD * 2;
static_assert(kLdsBytes <= 160 * 1024, "LDS of a compute unit");
constexpr int kOutRow = kD + 4;                                  // floats of a row where the wavefronts' results meet
static_assert(8 * 32 * kOutRow * 4 + 8 * 32 * 8 <= kLdsBytes, "results of eight wavefronts");

// A tile is 128 rows of 16 pieces of 16 bytes; piece c of row r lies at place c ^ twist(r), so that neither eight lanes with
// neighbouring rows nor the transposing reads (four rows, two pieces) meet in a bank.
__device__ __forceinline__ int twist(int r) { return ((r & 3) << 1) | (((r >> 2) ^ (r >> 3)) & 1) | (((r >> 3) & 1) << 3); }

__device__ __forceinline__ h8 lds_h8(const unsigned char* lds, int at) { return *reinterpret_cast<const h8*>(lds + at); }
// Four halves of one column of a 16-lane group's 4 x 16 block (every lane names four neighbouring columns of one row).
__device__ __forceinline__ h4 lds_column(unsigned char* lds, int at) {
  typedef __attribute__((address_space(3))) s4* lds_s4;
  return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(lds + at)));
}
__device__ __forceinline__ h8 join(h4 a, h4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
__device__ __forceinline__ h2 as_h2(unsigned w) { return __builtin_bit_cast(h2, w); }
__device__ __forceinline__ unsigned as_u(h2 v) { return __builtin_bit_cast(unsigned, v); }

// Codes 2 i and 2 i + 1 of a word (BITS each, the even one in the low half-word) times s plus z.  A code is read as the last
// bits of a half with a fixed exponent (2^e + code, exact), 2^e is taken off (exact), and one multiply-add rounds once.
template <int BITS, int I>
__device__ __forceinline__ unsigned dequant(unsigned w, h2 s, h2 z) {
  constexpr int kShift = BITS * I;                       // of the code in its half-word; it has to stand in the ten mantissa bits
  constexpr int kUp = kShift + BITS <= 10 ? kShift : kShift - (BITS == 2 ? 10 : 8);
  constexpr unsigned kMask = ((1u << BITS) - 1u) << kUp, kMagic = (unsigned)(15 + 10 - kUp) << 10;
  static_assert(kUp >= 0 && kUp + BITS <= 10, "inside the mantissa");
  const unsigned x = kShift == kUp ? w : w >> (kShift - kUp);
  const unsigned y = (x & (kMask * 0x10001u)) | (kMagic * 0x10001u);
  const _Float16 off = (_Float16)(float)(1 << (10 - kUp));
  return as_u((as_h2(y) - h2{off, off}) * s + z);
}

// State of one wavefront: 32 query rows, one to a lane and its partner 32 lanes away.
struct Rows {
  h8 q[8];            // B operand of step i: channels 16 i + 8 half ..
  f16v o[4];          // O^T: channels 32 c + 8 (r / 4) + 4 half + r % 4, relative to m
  float m, l;         // reference of the exponents (log2 units) and this lane's share of the sum of the weights
};

// The largest score may run ahead of the reference by this much (in log2) before the sums are brought to a new reference:
// weights stay below 2^8, well inside binary16, and most tiles change nothing.
constexpr float kHeadroom = 8.f;

// One pass over NS slices of 32 tokens of a tile.  BY_CHANNEL: the key tile has a row per channel (records), else a row per
// token, and the value tile the other way round.  limit: tokens of the tile this lane's row may see; only where `masked`.
template <int NS, bool BY_CHANNEL_K, bool BY_CHANNEL_V>
__device__ __forceinline__ void attend(unsigned char* lds, int keys, int values, int slice, Rows& st, float c, bool masked, int limit) {
  const int lane = threadIdx.x & 63, half = lane >> 5, i16 = lane & 15, grp = lane >> 4;
  f16v s[NS];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[n][r] = 0.f;
  }
  // Row 8 a + 4 h + i of a slice of scores stands for token 16 (a / 2) + 8 h + 4 (a % 2) + i: a lane then holds runs of eight
  // neighbouring tokens, which is what the second product takes.
  if constexpr (BY_CHANNEL_K) {
    const int row = 8 * (grp >> 1) + (i16 >> 2), piece = 2 * (grp & 1) + (i16 & 1), sub = ((i16 >> 1) & 1) * 8;
    const int a0 = keys + row * kRowBytes + sub, x0 = (piece ^ twist(row)) << 4, x1 = (piece ^ twist(row + 4)) << 4;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int at0 = a0 + (x0 ^ ((slice + n) << 6)), at1 = a0 + 4 * kRowBytes + (x1 ^ ((slice + n) << 6));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const h8 k = join(lds_column(lds, at0 + i * 16 * kRowBytes), lds_column(lds, at1 + i * 16 * kRowBytes));
        s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, st.q[i], s[n], 0, 0, 0);
      }
    }
  } else {
    const int m = lane & 31, token = 16 * (m >> 4) + 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3);
    const int a0 = keys + token * kRowBytes, x = (half ^ twist(token)) << 4;
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const h8 k = lds_h8(lds, a0 + (slice + n) * 32 * kRowBytes + (x ^ (i << 5)));
        s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, st.q[i], s[n], 0, 0, 0);
      }
  }
  if (masked) {
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if ((slice + n) * 32 + 16 * (r >> 3) + 8 * half + (r & 7) >= limit) s[n][r] = -INFINITY;
  }
  float mx = s[0][0];
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[n][r]);
  {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * c;
  }
  if (__any(mx > st.m + kHeadroom)) {
    const float m = fmaxf(st.m, mx);
    const float f = m == st.m ? 1.f : __builtin_amdgcn_exp2f(st.m - m);
    st.m = m;
    st.l *= f;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[b][r] *= f;
  }
  const float ref = st.m == -INFINITY ? 0.f : st.m;      // (a row that has seen no token yet)
  h8 p[NS][2];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r], c, -ref)), e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r + 1], c, -ref));
      sum += e0 + e1;
      const h2 e = __builtin_convertvector(f2{e0, e1}, h2);      // nearest: a truncated weight would pull every output to zero
      p[n][r >> 3][r & 7] = e[0];
      p[n][r >> 3][(r & 7) + 1] = e[1];
    }
    st.l += sum;
  }
  if constexpr (BY_CHANNEL_V) {
    const int m = lane & 31, a0 = values + m * kRowBytes, x = (half ^ twist(m)) << 4;
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int at = a0 + (x ^ ((slice + n) << 6) ^ (t << 5));
#pragma unroll
        for (int b = 0; b < 4; ++b)
          st.o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds_h8(lds, at + b * 32 * kRowBytes), p[n][t], st.o[b], 0, 0, 0);
      }
  } else {
    const int row = 8 * (grp >> 1) + (i16 >> 2), piece = 2 * (grp & 1) + ((i16 >> 1) & 1), sub = (i16 & 1) * 8;
    const int a0 = values + row * kRowBytes + sub, x0 = (piece ^ twist(row)) << 4, x1 = (piece ^ twist(row + 4)) << 4;
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int at = a0 + ((slice + n) * 32 + t * 16) * kRowBytes;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const h8 v = join(lds_column(lds, at + (x0 ^ (b << 6))), lds_column(lds, at + 4 * kRowBytes + (x1 ^ (b << 6))));
          st.o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[n][t], st.o[b], 0, 0, 0);
        }
      }
  }
}

// Dequantizes the staged tile's keys into `keys` (a row per channel).  Threads 0 .. 255; threads 256 .. 511 do the values.
__device__ __forceinline__ void unpack_keys(unsigned char* lds, const ChunkArgs& a, int keys, const unsigned short* map, int n_tok) {
  const int Rr = a.R, tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  {  // 2-bit channels: eight tokens of the eight even or odd channels of a word
    const int odd = wave & 1, tg = (wave >> 1) * 8 + (lane & 7), w = lane >> 3, t = tg * 8;
    if (w < a.Wlo && t < n_tok) {
      const int rec = t / Rr, tin = t - rec * Rr, raw = kOffRaw + rec * a.rec_bytes;
      const int words = raw + a.off_klo + (tin * a.Wlo + w) * 4;
      const unsigned pick = odd ? 0x07060302u : 0x05040100u, twice = odd ? 0x03020302u : 0x01000100u;
      unsigned x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = __builtin_amdgcn_perm(*reinterpret_cast<const unsigned*>(lds + words + (2 * i + 1) * a.Wlo * 4),
                                     *reinterpret_cast<const unsigned*>(lds + words + 2 * i * a.Wlo * 4), pick);
      const int sc = raw + a.off_klo_s + ((tin / a.Gk) * a.NLp + 16 * w) * 2, zc = sc + a.off_klo_z - a.off_klo_s;
      const unsigned* s = reinterpret_cast<const unsigned*>(lds + sc);
      const unsigned* z = reinterpret_cast<const unsigned*>(lds + zc);
      const unsigned* at = reinterpret_cast<const unsigned*>(map + rec * kD + 16 * w);
      const int col = tg << 4;
#define MIXKVQ_CHANNEL(I)                                                                                                  \
  {                                                                                                                        \
    const h2 s2 = as_h2(__builtin_amdgcn_perm(s[I], s[I], twice)), z2 = as_h2(__builtin_amdgcn_perm(z[I], z[I], twice));   \
    const int to = keys + (((at[I] >> (16 * odd)) & 0xffffu) ^ col);                                                       \
    *reinterpret_cast<uint4*>(lds + to) = make_uint4(dequant<2, I>(x[0], s2, z2), dequant<2, I>(x[1], s2, z2),             \
                                                     dequant<2, I>(x[2], s2, z2), dequant<2, I>(x[3], s2, z2));            \
  }
      MIXKVQ_CHANNEL(0) MIXKVQ_CHANNEL(1) MIXKVQ_CHANNEL(2) MIXKVQ_CHANNEL(3)
      MIXKVQ_CHANNEL(4) MIXKVQ_CHANNEL(5) MIXKVQ_CHANNEL(6) MIXKVQ_CHANNEL(7)
#undef MIXKVQ_CHANNEL
    }
  }
  // Side tiers: their channels stand in the record's list, an unused entry (255) goes to the row that nobody reads.
  const int k4 = a.k4, k16 = a.k16;
  for (int u = tid; u < a.W4 * 32; u += 256) {      // four bits: eight tokens of the four even or odd channels of a word
    const int odd = u & 1, tg = (u >> 1) & 15, w = u >> 5, t = tg * 8;
    if (t >= n_tok) continue;
    const int rec = t / Rr, tin = t - rec * Rr, raw = kOffRaw + rec * a.rec_bytes;
    const int words = raw + a.off_k4 + (tin * a.W4 + w) * 4;
    const unsigned pick = odd ? 0x07060302u : 0x05040100u, twice = odd ? 0x03020302u : 0x01000100u;
    unsigned x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = __builtin_amdgcn_perm(*reinterpret_cast<const unsigned*>(lds + words + (2 * i + 1) * a.W4 * 4),
                                   *reinterpret_cast<const unsigned*>(lds + words + 2 * i * a.W4 * 4), pick);
    const unsigned* s = reinterpret_cast<const unsigned*>(lds + raw + a.off_k4_s + ((tin / a.Gk) * k4 + 8 * w) * 2);
    const unsigned* z = reinterpret_cast<const unsigned*>(lds + raw + a.off_k4_z + ((tin / a.Gk) * k4 + 8 * w) * 2);
    const unsigned char* list = lds + raw + a.off_idx + k16 + 8 * w + odd;
#define MIXKVQ_CHANNEL(I)                                                                                                  \
  {                                                                                                                        \
    const h2 s2 = as_h2(__builtin_amdgcn_perm(s[I], s[I], twice)), z2 = as_h2(__builtin_amdgcn_perm(z[I], z[I], twice));   \
    const int ch = list[2 * I] < kD ? list[2 * I] : kD;                                                                    \
    const int to = keys + ch * kRowBytes + ((tg ^ twist(ch)) << 4);                                                        \
    *reinterpret_cast<uint4*>(lds + to) = make_uint4(dequant<4, I>(x[0], s2, z2), dequant<4, I>(x[1], s2, z2),             \
                                                     dequant<4, I>(x[2], s2, z2), dequant<4, I>(x[3], s2, z2));            \
  }
    MIXKVQ_CHANNEL(0) MIXKVQ_CHANNEL(1) MIXKVQ_CHANNEL(2) MIXKVQ_CHANNEL(3)
#undef MIXKVQ_CHANNEL
  }
  for (int u = tid; u < k16 * 8; u += 256) {      // fp16: eight tokens of two neighbouring entries
    const int tg = u & 15, e = (u >> 4) * 2, t = tg * 8;
    if (t >= n_tok) continue;
    const int rec = t / Rr, tin = t - rec * Rr, raw = kOffRaw + rec * a.rec_bytes;
    const unsigned char* src = lds + raw + a.off_k16 + (tin * k16 + e) * 2;
    unsigned x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const unsigned*>(src + i * k16 * 2);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const unsigned pick = j ? 0x07060302u : 0x05040100u;
      const int c = lds[raw + a.off_idx + e + j], ch = c < kD ? c : kD;
      *reinterpret_cast<uint4*>(lds + keys + ch * kRowBytes + ((tg ^ twist(ch)) << 4)) =
          make_uint4(__builtin_amdgcn_perm(x[1], x[0], pick), __builtin_amdgcn_perm(x[3], x[2], pick),
                     __builtin_amdgcn_perm(x[5], x[4], pick), __builtin_amdgcn_perm(x[7], x[6], pick));
    }
  }
}

// The staged tile's values into `values` (a row per channel): threads 256 .. 511, a word of 16 tokens of one channel at a time.
// Places of tokens that the tile does not have become 0 (their weights are 0, and 0 times what the LDS held may be NaN).
__device__ __forceinline__ void unpack_values(unsigned char* lds, const ChunkArgs& a, int values, int n_tok) {
  const int tid = threadIdx.x - 256, ch = tid & (kD - 1), first = __builtin_amdgcn_readfirstlane(tid >> 7);
  const int per = a.R >> 4, inv = 256 / per + 1;      // words of a record and channel; w / per = w inv >> 8 for w < 8
  const int vg = ch / a.Gv, row = values + ch * kRowBytes, tw = twist(ch);
#pragma unroll 2
  for (int k = 0; k < 4; ++k) {
    const int w = first + 2 * k;
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    int t0 = 16 * w, t1 = t0 + 8;
    if (t0 < n_tok) {
      const int rec = w * inv >> 8, in = w - rec * per;
      const unsigned x = *reinterpret_cast<const unsigned*>(lds + kOffRaw + rec * a.rec_bytes + a.off_v + (in * kD + ch) * 4);
      if (a.interleave) {
        t0 = rec * a.R + 64 * (in >> 2) + 8 * (in & 3);
        t1 = t0 + 32;
      }
      const unsigned char* s = lds + kOffScale + vg * kScaleRow * 2;
      const unsigned char* z = s + 8 * kScaleRow * 2;
      const uint4 s0 = *reinterpret_cast<const uint4*>(s + t0 * 2), z0 = *reinterpret_cast<const uint4*>(z + t0 * 2);
      const uint4 s1 = *reinterpret_cast<const uint4*>(s + t1 * 2), z1 = *reinterpret_cast<const uint4*>(z + t1 * 2);
      lo = make_uint4(dequant<2, 0>(x, as_h2(s0.x), as_h2(z0.x)), dequant<2, 1>(x, as_h2(s0.y), as_h2(z0.y)),
                      dequant<2, 2>(x, as_h2(s0.z), as_h2(z0.z)), dequant<2, 3>(x, as_h2(s0.w), as_h2(z0.w)));
      hi = make_uint4(dequant<2, 4>(x, as_h2(s1.x), as_h2(z1.x)), dequant<2, 5>(x, as_h2(s1.y), as_h2(z1.y)),
                      dequant<2, 6>(x, as_h2(s1.z), as_h2(z1.z)), dequant<2, 7>(x, as_h2(s1.w), as_h2(z1.w)));
    }
    *reinterpret_cast<uint4*>(lds + row + (((t0 >> 3) ^ tw) << 4)) = lo;
    *reinterpret_cast<uint4*>(lds + row + (((t1 >> 3) ^ tw) << 4)) = hi;
  }
}

template <int ROW_GROUPS, class Counts>
__global__ void __launch_bounds__(kChunkThreads, 2) chunk_attention_kernel(ChunkArgs a, Counts counts) {
  __shared__ __align__(256) unsigned char lds[kLdsBytes];
  constexpr int kRows = 32 * ROW_GROUPS;
  constexpr int kShares = 8 / ROW_GROUPS;              // wavefronts that share 32 rows, each with its slices of every tile
  constexpr int kSlices = 4 / kShares;                 // of a tile
  constexpr int kStep = kSlices >= 2 ? 2 : 1;          // slices taken together
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = wave % ROW_GROUPS, share = wave / ROW_GROUPS;
  const bool bf16 = a.bf16 != 0;
  const ChunkPlace at = chunk_place(a, counts, blockIdx.x);
  const int g = a.g, Hkv = a.Hkv, b = at.b, j = at.j, p = at.p, n_rec = at.n_rec, n_fp16 = at.n_fp16;
  const int n_rows = at.n_new * g, rt = gridDim.y - 1 - blockIdx.y;      // the last tiles of rows see most tokens: first
  if (rt * kRows >= n_rows) return;
  __builtin_amdgcn_s_setreg(1 | 23 << 6, 1);           // MODE.FP16_OVFL: a dequantized value past 65504 stays there

  // ---- query rows of this wavefront ----
  const int row0 = rt * kRows + 32 * group;
  const bool active = row0 < n_rows;
  const int row = row0 + (lane & 31) < n_rows ? row0 + (lane & 31) : n_rows - 1;
  const int token = row / g, q_head = j * g + row % g;
  Rows st;
  if (active) {
    const __half* q = a.q + (int64_t)b * a.qs.b + (int64_t)q_head * a.qs.h + (int64_t)token * a.qs.t + 8 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      st.q[i] = __builtin_bit_cast(h8, as_f16x8(*reinterpret_cast<const uint4*>(q + 16 * i), bf16));
  }
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.o[c][r] = 0.f;
  st.m = -INFINITY;
  st.l = 0.f;
  const float c = a.scale * 1.4426950408889634f;      // scores in log2 units
  const int see_min = row0 / g + 1;                   // chunk tokens seen by the first and the last row
  const int last_row = row0 + 31 < n_rows ? row0 + 31 : n_rows - 1;
  const int see_max = last_row / g + 1;

  // ---- this split's tiles: records, fp16 rows of the cache, the chunk as far as the tile's last row sees it ----
  const int tile_rec = a.tile_rec;
  const int tile_last = rt * kRows + kRows < n_rows ? rt * kRows + kRows - 1 : n_rows - 1;
  const int seen = tile_last / g + 1;
  const int nt_rec = (n_rec + tile_rec - 1) / tile_rec, nt_win = (n_fp16 + kChunkTile - 1) / kChunkTile;
  const int nt = nt_rec + nt_win + (seen + kChunkTile - 1) / kChunkTile;
  const int t_first = (int)((long long)nt * at.split / at.n_splits), t_end = (int)((long long)nt * (at.split + 1) / at.n_splits);

  // ---- records ----
  const int r_end = t_end < nt_rec ? t_end : nt_rec;
  if (t_first < r_end) {
    const int pieces = a.rec_bytes >> 4;      // 16-byte pieces of a record
    int pr[3], po[3], kind[3];                  // this thread's pieces of a tile: record, byte in it, plane
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int i = tid + kChunkThreads * k;
      pr[k] = i / pieces;
      po[k] = (i - pr[k] * pieces) * 16;
      const int es = po[k] - a.off_v_s, ez = po[k] - a.off_v_z, plane = a.R * a.NVG * 2;
      kind[k] = es >= 0 && es < plane ? 1 : ez >= 0 && ez < plane ? 2 : 0;
    }
    const int32_t* table = a.table ? a.table + (size_t)b * a.NB : nullptr;
    const int nvg_bits = 31 - __builtin_clz(a.NVG);
    auto tile_count = [&](int t) { const int left = n_rec - t * tile_rec; return left < tile_rec ? left : tile_rec; };
    auto record = [&](int blk) {
      return a.blocks + (table ? (size_t)table[blk] * Hkv + j : (size_t)p * a.NB + blk) * a.rec_bytes;
    };
    uint4 raw[3];
    auto fetch = [&](int t) {
      const int cnt = tile_count(t);
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (pr[k] < cnt) raw[k] = *reinterpret_cast<const uint4*>(record(t * tile_rec + pr[k]) + po[k]);
    };
    auto stage = [&](int t) {
      const int cnt = tile_count(t);
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        if (pr[k] >= cnt) continue;
        if (kind[k] == 0) {
          *reinterpret_cast<uint4*>(lds + kOffRaw + pr[k] * a.rec_bytes + po[k]) = raw[k];
        } else {      // value scales (zero-points): [token][group] there, [group][token] here
          const int li = (po[k] - (kind[k] == 1 ? a.off_v_s : a.off_v_z)) >> 1;
          unsigned short* to = reinterpret_cast<unsigned short*>(lds + kOffScale) + (kind[k] == 1 ? 0 : 8 * kScaleRow) + pr[k] * a.R;
          const unsigned v[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int tok = (li + e) >> nvg_bits, vg = (li + e) & (a.NVG - 1);
            if (tok < a.R) to[vg * kScaleRow + tok] = (unsigned short)(v[e >> 1] >> (16 * (e & 1)));
          }
        }
      }
    };
    // Wavefront w lists record w's 2-bit channels: place -> row of the key tile (twisted), 128 for places without a channel.
    const int ks = a.k4 + a.k16;
    auto map_of = [&](int t) { return reinterpret_cast<unsigned short*>(lds + kOffMap) + (t & 1) * kChunkRecords * kD; };
    auto list_channels = [&](int t) {
      if (wave >= tile_count(t)) return;
      const uint8_t* idx = record(t * tile_rec + wave) + a.off_idx;
      unsigned long long low = ~0ull, high = ~0ull;      // channels 0 .. 63 and 64 .. 127 that are in no list
      const int e0 = lane < ks ? idx[lane] : 255, e1 = lane + 64 < ks ? idx[lane + 64] : 255;
      for (int e = 0; e < ks; ++e) {
        const int ch = e < 64 ? __builtin_amdgcn_readlane(e0, e) : __builtin_amdgcn_readlane(e1, e - 64);
        if (ch < 64) low &= ~(1ull << ch);
        else if (ch < 128) high &= ~(1ull << (ch - 64));
      }
      unsigned short* to = map_of(t) + wave * kD;
      const int n_low = __popcll(low), n = n_low + __popcll(high);
      const unsigned long long before = (1ull << lane) - 1;
      if (low >> lane & 1) to[__popcll(low & before)] = (unsigned short)(lane << 8 | twist(lane) << 4);
      if (high >> lane & 1) to[n_low + __popcll(high & before)] = (unsigned short)((lane + 64) << 8 | twist(lane + 64) << 4);
      for (int i = n + lane; i < kD; i += 64) to[i] = (unsigned short)(kD << 8);
    };

    fetch(t_first);
    list_channels(t_first);
    stage(t_first);
    if (t_first + 1 < r_end) fetch(t_first + 1);
    __syncthreads();
    if (wave < 4) unpack_keys(lds, a, 0, map_of(t_first), tile_count(t_first) * a.R);
    else unpack_values(lds, a, kKeyBytes, tile_count(t_first) * a.R);
    if (t_first + 1 < r_end) list_channels(t_first + 1);
    __syncthreads();
    for (int t = t_first; t < r_end; ++t) {
      const bool next = t + 1 < r_end;
      const int here = (t - t_first & 1) * kTileBytes, there = kTileBytes - here;
      if (next) stage(t + 1);
      __syncthreads();
      if (t + 2 < r_end) fetch(t + 2);
      // The wavefronts of a SIMD (w and w + 4) unpack the next tile at different times: one's vector instructions run beside
      // the other's matrix instructions.
      if (next && wave < 4) unpack_keys(lds, a, there, map_of(t + 1), tile_count(t + 1) * a.R);
      if (active) {
        const int n_tok = tile_count(t) * a.R;
#pragma unroll 1
        for (int s = share * kSlices; s < (share + 1) * kSlices && s * 32 < n_tok; s += kStep)
          attend<kStep, true, true>(lds, here, here + kKeyBytes, s, st, c, (s + kStep) * 32 > n_tok, n_tok);
      }
      if (next && wave >= 4) unpack_values(lds, a, there + kKeyBytes, tile_count(t + 1) * a.R);
      if (t + 2 < r_end) list_channels(t + 2);
      __syncthreads();
    }
  }

  // ---- fp16 rows: the cache's (all of them are seen), then the chunk's (causal) ----
  const int f_first = t_first > nt_rec ? t_first : nt_rec;
  if (f_first < t_end) {
    const int prow = tid >> 4, piece = tid & 15;
    const int place = prow * kRowBytes + ((piece ^ twist(prow)) << 4);      // of this thread's first piece; the others 32 rows on
    uint4 fk[4], fv[4];
    auto fetch = [&](int t) {
      const bool win = t < nt_rec + nt_win;
      const int first = (t - nt_rec - (win ? 0 : nt_win)) * kChunkTile, n = win ? n_fp16 : seen;
      const __half* k = win ? a.res_k + (size_t)p * a.RW * kD : a.k + (int64_t)b * a.kvs.b + (int64_t)j * a.kvs.h;
      const __half* v = win ? a.res_v + (size_t)p * a.RW * kD : a.v + (int64_t)b * a.kvs.b + (int64_t)j * a.kvs.h;
      const int64_t step = win ? kD : a.kvs.t;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int r = first + prow + 32 * i;
        r = r < n ? r : n - 1;      // places behind the last row hold that row once more: finite, and masked
        fk[i] = *reinterpret_cast<const uint4*>(k + r * step + piece * 8);
        fv[i] = *reinterpret_cast<const uint4*>(v + r * step + piece * 8);
      }
    };
    auto stage = [&](int t, int at) {
      const bool convert = bf16 && t >= nt_rec + nt_win;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        *reinterpret_cast<uint4*>(lds + at + place + i * 32 * kRowBytes) = as_f16x8(fk[i], convert);
        *reinterpret_cast<uint4*>(lds + at + kKeyBytes + place + i * 32 * kRowBytes) = as_f16x8(fv[i], convert);
      }
    };
    fetch(f_first);
    stage(f_first, 0);
    __syncthreads();
    for (int t = f_first; t < t_end; ++t) {
      const int here = (t - f_first & 1) * kTileBytes, there = kTileBytes - here;
      if (t + 1 < t_end) fetch(t + 1);
      if (active) {
        const bool win = t < nt_rec + nt_win;
        const int first = (t - nt_rec - (win ? 0 : nt_win)) * kChunkTile;
        const int lim_min = (win ? n_fp16 : see_min) - first, lim_max = (win ? n_fp16 : see_max) - first;
        const int limit = (win ? n_fp16 : token + 1) - first;
#pragma unroll 1
        for (int s = share * kSlices; s < (share + 1) * kSlices && s * 32 < lim_max; s += kStep)
          attend<kStep, false, false>(lds, here, here + kKeyBytes, s, st, c, (s + kStep) * 32 > lim_min, limit);
      }
      if (t + 1 < t_end) stage(t + 1, there);
      __syncthreads();
    }
  }

  // ---- the shares of a row meet in LDS; results leave in whole rows ----
  float* const meet = reinterpret_cast<float*>(lds);                       // [wavefront][32][kOutRow]
  float2* const ml = reinterpret_cast<float2*>(lds + 8 * 32 * kOutRow * 4);   // [wavefront][32]
  {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(st.l), __float_as_uint(st.l), false, false);
    st.l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    if (lane < 32) ml[wave * 32 + lane] = make_float2(st.m, st.l);
#pragma unroll
    for (int c4 = 0; c4 < 4; ++c4)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f4*>(meet + (wave * 32 + (lane & 31)) * kOutRow + 32 * c4 + 8 * q + 4 * (lane >> 5)) =
            f4{st.o[c4][4 * q], st.o[c4][4 * q + 1], st.o[c4][4 * q + 2], st.o[c4][4 * q + 3]};
  }
  __syncthreads();
  const int chan = (tid & 15) * 8;
#pragma unroll 1
  for (int r = tid >> 4; r < kRows; r += kChunkThreads / 16) {      // 16 threads to a row
    const int rr = rt * kRows + r;
    if (rr >= n_rows) break;
    const int w0 = r >> 5, in_group = r & 31;
    float m = -INFINITY;
#pragma unroll
    for (int s = 0; s < kShares; ++s) m = fmaxf(m, ml[(s * ROW_GROUPS + w0) * 32 + in_group].x);
    float sum = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kShares; ++s) {
      const int at = (s * ROW_GROUPS + w0) * 32 + in_group;
      const float2 x = ml[at];
      const float f = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - m);
      sum += f * x.y;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += f * meet[at * kOutRow + chan + e];
    }
    if (a.split) {
      const size_t slot = ((size_t)blockIdx.x * gridDim.y + rt) * kRows + r;
      float* to = a.part + slot * kD + chan;
      *reinterpret_cast<f4*>(to) = f4{o[0], o[1], o[2], o[3]};
      *reinterpret_cast<f4*>(to + 4) = f4{o[4], o[5], o[6], o[7]};
      if (chan == 0) *reinterpret_cast<float2*>(a.part + (size_t)gridDim.x * gridDim.y * kRows * kD + slot * 2) = make_float2(m, sum);
    } else {
      const int t = rr / g, h = j * g + rr % g;
      const float inv = 1.f / sum;
      unsigned w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = o[2 * e] * inv, y = o[2 * e + 1] * inv;
        w[e] = bf16 ? (unsigned)f32_to_bf16_bits(x) | (unsigned)f32_to_bf16_bits(y) << 16 : as_u(__builtin_convertvector(f2{x, y}, h2));
      }
      *reinterpret_cast<uint4*>(a.out + (int64_t)b * a.os.b + (int64_t)h * a.os.h + (int64_t)t * a.os.t + chan) = make_uint4(w[0], w[1], w[2], w[3]);
      if (a.lse && chan == 0) a.lse[((size_t)b * a.Hq + h) * a.n_max + t] = (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    }
  }
}

// The splits of a row meet: 16 threads to a row; x: workgroups of 16 rows, y: pairs of the launch's sequences (in the order of
// blockIdx.x of their first splits).
template <class Counts>
__global__ void __launch_bounds__(256) chunk_merge_kernel(ChunkArgs a, Counts counts, int rows, int blocks, int per_pair) {
  int pair = blockIdx.x / per_pair;
  const int i = pair / a.Hkv, j = pair % a.Hkv;
  ChunkPlace at;
  if constexpr (std::is_same<Counts, NoChunkCounts>::value) at = chunk_place(a, counts, i * a.n_splits * a.Hkv + j);
  else at = chunk_place(a, counts, counts.first[i] * a.Hkv + j);
  const int g = a.g, n_rows = at.n_new * g, rr = blockIdx.x % per_pair * 16 + (threadIdx.x >> 4), chan = (threadIdx.x & 15) * 8;
  if (rr >= n_rows || at.b != a.b0 + i) return;      // (a sequence without new tokens has no unit)
  const size_t first = ((size_t)at.first_block * a.row_tiles + rr / rows) * rows + rr % rows, step = (size_t)a.Hkv * a.row_tiles * rows;
  const float2* ml = reinterpret_cast<const float2*>(a.part + (size_t)blocks * rows * kD);
  float m = -INFINITY, sum = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < at.n_splits; ++s) m = fmaxf(m, ml[first + s * step].x);
#pragma unroll 4
  for (int s = 0; s < at.n_splits; ++s) {
    const size_t slot = first + s * step;
    const float2 x = ml[slot];
    const float f = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - m);
    const f4 u = *reinterpret_cast<const f4*>(a.part + slot * kD + chan), v = *reinterpret_cast<const f4*>(a.part + slot * kD + chan + 4);
    sum += f * x.y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] += f * u[e];
      o[4 + e] += f * v[e];
    }
  }
  const int t = rr / g, h = j * g + rr % g;
  const float inv = 1.f / sum;
  unsigned w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = o[2 * e] * inv, y = o[2 * e + 1] * inv;
    w[e] = a.bf16 ? (unsigned)f32_to_bf16_bits(x) | (unsigned)f32_to_bf16_bits(y) << 16 : as_u(__builtin_convertvector(f2{x, y}, h2));
  }
  *reinterpret_cast<uint4*>(a.out + (int64_t)at.b * a.os.b + (int64_t)h * a.os.h + (int64_t)t * a.os.t + chan) = make_uint4(w[0], w[1], w[2], w[3]);
  if (a.lse && chan == 0) a.lse[((size_t)at.b * a.Hq + h) * a.n_max + t] = (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// |q| of the chunk joins the accumulator: exact integer sums, so that the order of the workgroups changes nothing.
template <class Counts>
__global__ void __launch_bounds__(256) chunk_books_kernel(unsigned long long* qacc, unsigned long long* qcnt, ChunkArgs a, Counts counts, int per_pair) {
  const int pair = blockIdx.x / per_pair, i = pair / a.Hkv, j = pair % a.Hkv, g = a.g, b = a.b0 + i;
  int n_new = a.n_new;
  if constexpr (!std::is_same<Counts, NoChunkCounts>::value) n_new = counts.n_new[i];
  const int d = threadIdx.x & (kD - 1), n_rows = n_new * g, first = blockIdx.x % per_pair * 64;
  unsigned long long sum = 0;
  for (int r = first + (threadIdx.x >> 7); r < n_rows && r < first + 64; r += 2)
    sum += fix24_abs(in_bits(a.q + (int64_t)b * a.qs.b + (int64_t)(j * g + r % g) * a.qs.h + (int64_t)(r / g) * a.qs.t + d, a.bf16 != 0));
  const int p = b * a.Hkv + j;
  if (sum) atomicAdd(qacc + (size_t)p * kD + d, sum);
  if (first == 0 && threadIdx.x == 0 && n_rows) atomicAdd(qcnt + p, (unsigned long long)n_rows);
}

int chunk_tile_records(const CacheView& v) {
  int n = kChunkTile / v.cfg.R > 0 ? kChunkTile / v.cfg.R : 1;
  const int fit = kMaxRec / v.lay.rec_bytes;
  n = n < fit ? n : fit;
  return n < kChunkRecords ? n : kChunkRecords;
}

// Slices of 32 tokens inside one record and one key group; four or five steps of channel places, at most one of fp16 places.
bool chunk_few_fits(const CacheView& v) {
  return v.cfg.R % 32 == 0 && v.cfg.Gk % 32 == 0 && v.lay.NVG <= 4 && v.cfg.k16 <= 32 && v.lay.W4 <= 4;
}

// 48 where the four steps hold everything and a token has one value group; the others have no registers for as many.
int chunk_few_rows(const CacheView& v) { return v.cfg.k16 == 0 && chunk_few_steps(v.lay.NLp, v.lay.W4) == 4 && v.lay.NVG == 1 ? 48 : 32; }

hipError_t start_chunk_few_1(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s);
hipError_t start_chunk_few_2(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s);
hipError_t start_chunk_few_3(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s);

template <int ROW_GROUPS>
static hipError_t start_tiles(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s) {
  const dim3 grid(units * a.Hkv, a.row_tiles);
  if (c) chunk_attention_kernel<ROW_GROUPS, ChunkCounts><<<grid, kChunkThreads, 0, s>>>(a, *c);
  else chunk_attention_kernel<ROW_GROUPS, NoChunkCounts><<<grid, kChunkThreads, 0, s>>>(a, NoChunkCounts{});
  return hipGetLastError();
}

hipError_t launch_chunk(const ChunkArgs& a, const ChunkCounts* c, int units, int n_seq, bool few, int rows, hipStream_t s) {
  hipError_t e;
  if (few) e = rows == 16 ? start_chunk_few_1(a, c, units, s) : rows == 32 ? start_chunk_few_2(a, c, units, s) : start_chunk_few_3(a, c, units, s);
  else e = rows == 64 ? start_tiles<2>(a, c, units, s) : rows == 128 ? start_tiles<4>(a, c, units, s) : start_tiles<8>(a, c, units, s);
  if (e != hipSuccess || !a.split) return e;
  const int per_pair = (a.row_tiles * rows + 15) / 16, blocks = units * a.Hkv * a.row_tiles;
  if (c) chunk_merge_kernel<<<per_pair * n_seq * a.Hkv, 256, 0, s>>>(a, *c, rows, blocks, per_pair);
  else chunk_merge_kernel<<<per_pair * n_seq * a.Hkv, 256, 0, s>>>(a, NoChunkCounts{}, rows, blocks, per_pair);
  return hipGetLastError();
}

hipError_t launch_chunk_books(const CacheView& v, const ChunkArgs& a, const ChunkCounts* c, int n_seq, int n_most, hipStream_t s) {
  const int per_pair = (n_most * a.g + 63) / 64;
  if (c) chunk_books_kernel<<<per_pair * n_seq * a.Hkv, 256, 0, s>>>(v.qacc, v.qcnt, a, *c, per_pair);
  else chunk_books_kernel<<<per_pair * n_seq * a.Hkv, 256, 0, s>>>(v.qacc, v.qcnt, a, NoChunkCounts{}, per_pair);
  return hipGetLastError();
}

}  // namespace mixkvq
