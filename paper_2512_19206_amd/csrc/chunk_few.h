// Attention of a chunk with few query rows (speculative steps): every wavefront walks over its own run of 32-token slices with up to
// 48 query rows, nothing is shared and no barrier is passed until the results meet.
//
// A slice is two tiles of 16 tokens.  Both products are v_mfma_f32_16x16x32_f16 in the transposed form, S^T = K Q^T and
// O^T = V^T P^T; row 4 a + r of tile t stands for token 8 a + 4 t + r of the slice, so that the scores a lane ends up with are
// the eight neighbouring tokens it has to hand to the second product.
//
// Keys are never dequantized: q.(c s + z) = sum (q s) c + q.z (Eq. 3).  A word's codes become eight halves of the big operand by
// one shift and four ANDs, as the binary16 SUBNORMALS c 4^p 2^-24 (4-bit codes c 16^p 2^-24), which the matrix cores multiply
// exactly; 4^-p goes into the scales.  q s is kept in two halves, hi = fp16(q s) and the exact remainder lo = fp16(q s - hi), so
// a score carries about 22 bits of it: rounded to one half, 131 072 tokens with sharp weights had outputs 0.8 % off.  A packed
// multiply and a packed multiply-add form both halves of two products.  q.z is one matrix product per group of tokens against
// the zero-points, and starts the scores.  Values are dequantized in registers (one rounding each).
//
// The channels of a record stand in the order of its tiers.  Each wavefront keeps its rows of q in that order in LDS and moves
// them only where a record's lists differ from the record's before it.
#pragma once
#include "chunk.h"

namespace mixkvq {
namespace few {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 512, kWaves = 8;
constexpr float kHeadroom = 8.f;                  // log2 by which scores may pass the reference (see chunk_kernels.hip)

__device__ __forceinline__ h2 as_h2(unsigned w) { return __builtin_bit_cast(h2, w); }
__device__ __forceinline__ unsigned as_u(h2 v) { return __builtin_bit_cast(unsigned, v); }
__device__ __forceinline__ h8 as_h8(unsigned a, unsigned b, unsigned c, unsigned d) { return __builtin_bit_cast(h8, make_uint4(a, b, c, d)); }
__device__ __forceinline__ h8 splat8(_Float16 x) { return h8{x, x, x, x, x, x, x, x}; }

__device__ __forceinline__ float max_of_groups(float x) {      // over lanes l, l ^ 16, l ^ 32, l ^ 48
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float sum_of_groups(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Codes 2 p and 2 p + 1 of a shifted word of 2-bit codes (p < 4) times s plus z, rounded once (see chunk_kernels.hip).
template <int P>
__device__ __forceinline__ unsigned value_pair(unsigned x, unsigned s, unsigned z) {
  constexpr unsigned kMask = 0x00030003u << (2 * P), kMagic = ((unsigned)(25 - 2 * P) << 10) * 0x10001u;
  const _Float16 off = (_Float16)(float)(1 << (10 - 2 * P));
  return as_u((as_h2((x & kMask) | kMagic) - h2{off, off}) * as_h2(s) + as_h2(z));
}

__device__ __forceinline__ int twist(int r) { return ((r & 3) << 1) | (((r >> 2) ^ (r >> 3)) & 1) | (((r >> 3) & 1) << 3); }

// NB: blocks of 16 query rows.  NKC: steps of 32 channel places with codes, of which only the last may hold others than 2-bit
// ones.  HAS16: one more step with the fp16 tier.  NVG: value groups of a token.
template <int NB, int NKC, int HAS16, int NVG>
struct Kernel {
  static constexpr int kRows = 16 * NB;
  static constexpr int kPieces = 4 * (NKC + HAS16);                // 16-byte pieces of a row of q in tier order
  static constexpr int kRowBytes = 16 * kPieces;
  static constexpr int kRegion = kRows * kRowBytes > 8192 ? kRows * kRowBytes : 8192;      // of a wavefront; also 32 value rows
  static constexpr int kOffWave = kRows * 256;                     // behind the rows of q as given
  static constexpr int kOffScale = kOffWave + kWaves * kRegion;
  static constexpr int kLds = kOffScale + kRows * 4;
  static constexpr int kOutRow = kD + 4;
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
  static_assert(kWaves * 16 * kOutRow * 4 + kWaves * 16 * 8 <= kLds, "results of eight wavefronts");

  // place of piece o of row r: no two of eight neighbouring rows in one bank
  __device__ static __forceinline__ int piece(int r, int o) { return kPieces == 16 ? o ^ (r & 15) : kPieces == 20 ? o ^ ((r >> 1) & 3) : o ^ (r & 7); }

  struct State {
    f4 o[NB][8];
    float m[NB], l[NB];
  };

  // Scores x (log2 units; tile t, register r: token 8 group + 4 t + r) -> weights, and the sums brought to a new reference if need be.
  __device__ static __forceinline__ h8 weigh(State& st, int b, const float (&x)[8]) {
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
    mx = max_of_groups(mx);
    if (__any(mx > st.m[b] + kHeadroom)) {
      const float m = fmaxf(st.m[b], mx), f = m == st.m[b] ? 1.f : __builtin_amdgcn_exp2f(st.m[b] - m);
      st.m[b] = m;
      st.l[b] *= f;
#pragma unroll
      for (int c = 0; c < 8; ++c) st.o[b][c] *= f;
    }
    const float ref = st.m[b] == -INFINITY ? 0.f : st.m[b];
    h8 p;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float e0 = __builtin_amdgcn_exp2f(x[e] - ref), e1 = __builtin_amdgcn_exp2f(x[e + 1] - ref);
      sum += e0 + e1;
      const h2 w = __builtin_convertvector(f2{e0, e1}, h2);
      p[e] = w[0];
      p[e + 1] = w[1];
    }
    st.l[b] += sum;
    return p;
  }

  __device__ static __forceinline__ void run(const CacheView& cv, const ChunkArgs& a, const ChunkLaunch& l, bool split_launch, unsigned char* lds) {
    const mixkvq_config& cfg = cv.cfg;
    const Layout& lay = cv.lay;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m16 = lane & 15, grp = lane >> 4;
    const bool bf16 = cfg.in_dtype != 0;
    __builtin_amdgcn_s_setreg(1 | 23 << 6, 1);           // MODE.FP16_OVFL: what passes 65504 stays there

    // ---- which unit (neighbouring units share keys: on one XCD) ----
    int unit;
    {
      const int n = l.n_units, x = blockIdx.x & 7, y = blockIdx.x >> 3, whole = n >> 3, more = n & 7;
      unit = x * whole + (x < more ? x : more) + y;
    }
    int sb = 0, base = 0;
    if (l.same_units) {
      sb = unit / l.same_units;
      base = sb * l.same_units;
    } else {
      int hi = l.n_seq;
      while (hi - sb > 1) {
        const int mid = (sb + hi) >> 1;
        if (l.first_unit[mid] <= unit) sb = mid;
        else hi = mid;
      }
      base = l.first_unit[sb];
    }
    const int g = cv.g, Hkv = cfg.Hkv, b = l.b0 + sb;
    const int n_new = l.n_new[sb], n_rec = l.n_rec[sb];
    const int n_fp16 = (int)(l.rows_splits[sb] & 0xffffu), n_splits = (int)(l.rows_splits[sb] >> 16);
    const int n_rows = n_new * g, row_tiles = (n_rows + kRows - 1) / kRows;
    int in = unit - base;
    const int rt = row_tiles - 1 - in % row_tiles;
    in /= row_tiles;
    const int split = in % n_splits, j = in / n_splits, p = b * Hkv + j, row0 = rt * kRows;

    // ---- the rows of q, each brought to a largest element of 2^6 to 2^7 (powers of two: exact) ----
    float* const row_scale = reinterpret_cast<float*>(lds + kOffScale);
    for (int i = tid; i < kRows * 16; i += kThreads) {
      const int r = i >> 4, o = i & 15, row = row0 + r;
      uint4 w = make_uint4(0, 0, 0, 0);
      if (row < n_rows)
        w = as_f16x8(*reinterpret_cast<const uint4*>(a.q + (int64_t)b * a.qs.b + (int64_t)(j * g + row % g) * a.qs.h + (int64_t)(row / g) * a.qs.t + 8 * o), bf16);
      h8 v = __builtin_bit_cast(h8, w);
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)v[e]));
      for (int s = 8; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
      int k = top > 0.f ? 7 - __builtin_amdgcn_frexp_expf(top) : 0;      // (65504 has 16, the smallest subnormal -23)
      k = k > 14 ? 14 : k;
      v *= splat8((_Float16)ldexpf(1.f, k));
      *reinterpret_cast<h8*>(lds + r * 256 + ((o ^ (r & 15)) << 4)) = v;
      if (o == 0) row_scale[r] = ldexpf(a.scale * 1.4426950408889634f, -k);      // scores in log2 units
    }
    unsigned char* const mine = lds + kOffWave + wave * kRegion;
    for (int i = lane; i < kRegion / 16; i += 64) *reinterpret_cast<uint4*>(mine + i * 16) = make_uint4(0, 0, 0, 0);
    __syncthreads();

    State st;
#pragma unroll
    for (int r = 0; r < NB; ++r) {
      st.m[r] = -INFINITY;
      st.l[r] = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) st.o[r][c] = f4{0.f, 0.f, 0.f, 0.f};
    }
    float fl[NB];
#pragma unroll
    for (int r = 0; r < NB; ++r) fl[r] = row_scale[16 * r + m16];

    // ---- this wavefront's slices: of the records, then of the cache's fp16 rows, then of the chunk ----
    const int tile_last = row0 + kRows < n_rows ? row0 + kRows - 1 : n_rows - 1, seen = tile_last / g + 1;
    const int spr = cfg.R >> 5, u_rec = n_rec * spr, u_win = (n_fp16 + 31) >> 5, u_all = u_rec + u_win + ((seen + 31) >> 5);
    const int share = split * kWaves + wave, shares = n_splits * kWaves;
    const int u0 = (int)((long long)u_all * share / shares), u1 = (int)((long long)u_all * (share + 1) / shares);

    if (u0 < u_rec) {
      const int end = u1 < u_rec ? u1 : u_rec;
      const int32_t* table = cv.table ? cv.table + (size_t)b * cv.NB : nullptr;
      auto record = [&](int blk) {
        return cv.blocks + (table ? (size_t)table[blk] * Hkv + j : (size_t)p * cv.NB + blk) * lay.rec_bytes;
      };
      // The last step with codes: octet 4 (NKC - 1) + group of [2 bit | 4 bit] places, by lane.
      const int n_lo = lay.NLp >> 3, oct = 4 * (NKC - 1) + grp;
      const bool is_lo = oct < n_lo, is_4 = !is_lo && oct < n_lo + lay.W4;
      const int last_stride = is_4 ? lay.W4 * 4 : lay.Wlo * 4, last_off = is_4 ? lay.off_k4 + (oct - n_lo) * 4 : is_lo ? lay.off_klo + (oct >> 1) * 4 : lay.off_klo;
      const int sh0 = is_lo ? 8 * (oct & 1) : 0, sh1 = is_lo ? sh0 : 8;
      const unsigned mk[4] = {is_4 ? 0x000f000fu : is_lo ? 0x00030003u : 0u, is_4 ? 0x00f000f0u : is_lo ? 0x000c000cu : 0u,
                              is_4 ? 0x000f000fu : is_lo ? 0x00300030u : 0u, is_4 ? 0x00f000f0u : is_lo ? 0x00c000c0u : 0u};
      const int last_s = is_4 ? lay.off_k4_s + (oct - n_lo) * 16 : lay.off_klo_s + oct * 16, last_dz = is_4 ? lay.off_k4_z - lay.off_k4_s : lay.off_klo_z - lay.off_klo_s;
      const int last_gs = is_4 ? cfg.k4 * 2 : lay.NLp * 2;
      const int gps = cfg.Gk >> 5;                          // slices of a group
      const int tok0 = 8 * (m16 >> 2) + (m16 & 3);          // token of tile 0; 4 further in tile 1

      struct Keys { unsigned w[2][NKC]; uint4 raw[2]; };
      auto load_keys = [&](const uint8_t* rec, int sl, Keys& k) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int tok = sl * 32 + tok0 + 4 * t;
          const unsigned at = lay.off_klo + tok * lay.Wlo * 4 + (grp >> 1) * 4;
#pragma unroll
          for (int s = 0; s < NKC - 1; ++s) k.w[t][s] = *reinterpret_cast<const unsigned*>(rec + at + 8 * s);
          k.w[t][NKC - 1] = *reinterpret_cast<const unsigned*>(rec + (unsigned)(last_off + tok * last_stride));
          if constexpr (HAS16) {
            k.raw[t] = make_uint4(0, 0, 0, 0);
            if (8 * grp < cfg.k16) {
              const uint2* src = reinterpret_cast<const uint2*>(rec + (unsigned)(lay.off_k16 + (tok * cfg.k16 + 8 * grp) * 2));
              const uint2 x = src[0];
              k.raw[t].x = x.x;
              k.raw[t].y = x.y;
              if (8 * grp + 4 < cfg.k16) {
                const uint2 y = src[1];
                k.raw[t].z = y.x;
                k.raw[t].w = y.y;
              }
            }
          }
        }
      };

      int have0 = -1, have1 = -1;      // the lists that the rows in `mine` are ordered by (entries lane and lane + 64)
      const int ks = cfg.k4 + cfg.k16;
      auto order_rows = [&](const uint8_t* rec) {
        const int e0 = lane < ks ? rec[lay.off_idx + lane] : 255, e1 = lane + 64 < ks ? rec[lay.off_idx + lane + 64] : 255;
        if (!__any(e0 != have0 || e1 != have1)) return;
        have0 = e0;
        have1 = e1;
        unsigned long long low = ~0ull, high = ~0ull;
        int s0 = -1, s1 = -1;          // places of channels lane and lane + 64
        for (int e = 0; e < ks; ++e) {
          const int ch = e < 64 ? __builtin_amdgcn_readlane(e0, e) : __builtin_amdgcn_readlane(e1, e - 64);
          const int at = e < cfg.k16 ? 32 * NKC + e : lay.NLp + e - cfg.k16;
          if (ch < 64) low &= ~(1ull << ch);
          else if (ch < 128) high &= ~(1ull << (ch - 64));
          if (ch == lane) s0 = at;
          if (ch == lane + 64) s1 = at;
        }
        const unsigned long long before = (1ull << lane) - 1;
        if (s0 < 0) s0 = __popcll(low & before);
        if (s1 < 0) s1 = __popcll(low) + __popcll(high & before);
        const int p0 = s0 >> 3, q0 = (s0 & 7) * 2, p1 = s1 >> 3, q1 = (s1 & 7) * 2, c0 = lane >> 3, d0 = (lane & 7) * 2;
#pragma unroll 8
        for (int r = 0; r < kRows; ++r) {
          const unsigned short x = *reinterpret_cast<const unsigned short*>(lds + r * 256 + ((c0 ^ (r & 15)) << 4) + d0);
          const unsigned short y = *reinterpret_cast<const unsigned short*>(lds + r * 256 + (((c0 + 8) ^ (r & 15)) << 4) + d0);
          *reinterpret_cast<unsigned short*>(mine + r * kRowBytes + (piece(r, p0) << 4) + q0) = x;
          *reinterpret_cast<unsigned short*>(mine + r * kRowBytes + (piece(r, p1) << 4) + q1) = y;
        }
      };
      auto rows_of = [&](int r, int step) { return *reinterpret_cast<const h8*>(mine + (16 * r + m16) * kRowBytes + (piece(m16, 4 * step + grp) << 4)); };

      int blk = u0 / spr, sl = u0 - blk * spr;
      const uint8_t* rec = record(blk);
      Keys cur;
      load_keys(rec, sl, cur);
      h8 sc[NKC];                      // the group's scales at the places of this lane, with the factors of the codes
      float fg[NB], bias[NB];          // scores = codes' sums * fg + bias
      bool fresh = true;
      for (int u = u0; u < end; ++u) {
        // values of this slice: word of the lane's eight tokens in each of eight blocks of 16 channels
        const int word = lay.v_interleave ? 4 * (sl >> 1) + grp : 2 * sl + (grp >> 1);
        const int vsh = 8 * (lay.v_interleave ? sl & 1 : grp & 1);
        unsigned vw[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) vw[c] = *reinterpret_cast<const unsigned*>(rec + (unsigned)(lay.off_v + (word * kD + m16) * 4) + 64 * c);
        uint4 vs[NVG], vz[NVG];        // scales and zero-points of the lane's tokens, [token][group] as stored
        {
          const unsigned at = (unsigned)((sl * 32 + 8 * grp) * NVG * 2);
#pragma unroll
          for (int i = 0; i < NVG; ++i) {
            vs[i] = *reinterpret_cast<const uint4*>(rec + (lay.off_v_s + at) + 16 * i);
            vz[i] = *reinterpret_cast<const uint4*>(rec + (lay.off_v_z + at) + 16 * i);
          }
        }
        if (fresh) order_rows(rec);
        if (fresh || sl % gps == 0) {
          fresh = false;
          const int gr = sl / gps;
          // the largest scale becomes 2^6 to 2^7: products with q stay below 2^14, small ones keep their bits
          const float top = (float)*reinterpret_cast<const _Float16*>(rec + lay.off_kmax + 2 * gr);
          int e = top > 0.f ? 7 - __builtin_amdgcn_frexp_expf(top) : 0;
          e = __builtin_amdgcn_readfirstlane(e > 14 ? 14 : e);
          h8 z[NKC];
#pragma unroll
          for (int s = 0; s < NKC - 1; ++s) {
            const unsigned at = (unsigned)(gr * lay.NLp * 2 + (4 * s + grp) * 16);
            sc[s] = *reinterpret_cast<const h8*>(rec + (lay.off_klo_s + at));
            z[s] = *reinterpret_cast<const h8*>(rec + (lay.off_klo_z + at));
          }
          const unsigned at = (unsigned)(last_s + gr * last_gs);
          sc[NKC - 1] = splat8((_Float16)0.f);
          z[NKC - 1] = sc[NKC - 1];
          if (is_lo || is_4) {
            sc[NKC - 1] = *reinterpret_cast<const h8*>(rec + at);
            z[NKC - 1] = *reinterpret_cast<const h8*>(rec + (at + last_dz));
          }
          const float back = ldexpf(16777216.f, -e);
          const _Float16 f = (_Float16)ldexpf(1.f, e), q1 = (_Float16)0.25f, q2 = (_Float16)0.0625f, q3 = (_Float16)0.015625f;
          const h8 lo_f = h8{f, f, f * q1, f * q1, f * q2, f * q2, f * q3, f * q3}, four_f = h8{f, f, f * q2, f * q2, f, f, f * q2, f * q2};
#pragma unroll
          for (int s = 0; s < NKC - 1; ++s) sc[s] *= lo_f;
          sc[NKC - 1] *= is_4 ? four_f : lo_f;
#pragma unroll
          for (int r = 0; r < NB; ++r) {
            f4 acc = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < NKC; ++s) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(z[s], rows_of(r, s), acc, 0, 0, 0);
            fg[r] = fl[r] * back;
            bias[r] = acc[0] * fl[r];
          }
        }
        // ---- scores ----
        f4 s[NB][2], s16[HAS16 ? NB : 1][2];
#pragma unroll
        for (int r = 0; r < NB; ++r) s[r][0] = s[r][1] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NKC; ++k) {
          h8 big[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const unsigned w = cur.w[t][k];
            if (k < NKC - 1) {
              const unsigned x = w >> (8 * (grp & 1));
              big[t] = as_h8(x & 0x00030003u, x & 0x000c000cu, x & 0x00300030u, x & 0x00c000c0u);
            } else {
              const unsigned x = w >> sh0, y = w >> sh1;
              big[t] = as_h8(x & mk[0], x & mk[1], y & mk[2], y & mk[3]);
            }
          }
#pragma unroll
          for (int r = 0; r < NB; ++r) {
            const h8 q = rows_of(r, k);
            const h8 hi = q * sc[k], lo = __builtin_elementwise_fma(q, sc[k], -hi);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(big[t], hi, s[r][t], 0, 0, 0);
              s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(big[t], lo, s[r][t], 0, 0, 0);
            }
          }
        }
        if constexpr (HAS16) {
#pragma unroll
          for (int r = 0; r < NB; ++r) {
            const h8 q = rows_of(r, NKC);
#pragma unroll
            for (int t = 0; t < 2; ++t)
              s16[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, cur.raw[t]), q, f4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
          }
        }
        // keys of the next slice
        if (++sl == spr) {
          sl = 0;
          ++blk;
          fresh = true;
        }
        if (u + 1 < end) {
          if (fresh) rec = record(blk);
          load_keys(rec, sl, cur);
        }
        h8 pw[NB];
#pragma unroll
        for (int r = 0; r < NB; ++r) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float add = bias[r];
            if constexpr (HAS16) add = __builtin_fmaf(s16[r][e >> 2][e & 3], fl[r], add);
            x[e] = __builtin_fmaf(s[r][e >> 2][e & 3], fg[r], add);
          }
          pw[r] = weigh(st, r, x);
          if constexpr (NB > 2) __builtin_amdgcn_sched_barrier(0);      // one block's scores at a time: registers
        }
        // ---- values ----
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          unsigned sp[4], zp[4];       // pairs of tokens of the channel's group
          if constexpr (NVG == 1) {
            sp[0] = vs[0].x; sp[1] = vs[0].y; sp[2] = vs[0].z; sp[3] = vs[0].w;
            zp[0] = vz[0].x; zp[1] = vz[0].y; zp[2] = vz[0].z; zp[3] = vz[0].w;
          } else {
            const int vg = c * NVG / 8;
            const unsigned* ps = reinterpret_cast<const unsigned*>(vs);
            const unsigned* pz = reinterpret_cast<const unsigned*>(vz);
            const unsigned pick = vg & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int d0 = (2 * i * NVG + vg) >> 1, d1 = ((2 * i + 1) * NVG + vg) >> 1;
              sp[i] = __builtin_amdgcn_perm(ps[d1], ps[d0], pick);
              zp[i] = __builtin_amdgcn_perm(pz[d1], pz[d0], pick);
            }
          }
          const unsigned x = vw[c] >> vsh;
          const h8 v = as_h8(value_pair<0>(x, sp[0], zp[0]), value_pair<1>(x, sp[1], zp[1]), value_pair<2>(x, sp[2], zp[2]), value_pair<3>(x, sp[3], zp[3]));
#pragma unroll
          for (int r = 0; r < NB; ++r) st.o[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pw[r], st.o[r][c], 0, 0, 0);
        }
      }
    }

    // ---- fp16 rows: those of the cache, then the chunk's own ----
    for (int u = u0 > u_rec ? u0 : u_rec; u < u1; ++u) {
      const bool win = u < u_rec + u_win;
      const int first = (u - u_rec - (win ? 0 : u_win)) * 32, n = win ? n_fp16 : seen;
      const __half* k = win ? cv.res_k + (size_t)p * cv.RW * kD : a.k + (int64_t)b * a.kvs.b + (int64_t)j * a.kvs.h;
      const __half* v = win ? cv.res_v + (size_t)p * cv.RW * kD : a.v + (int64_t)b * a.kvs.b + (int64_t)j * a.kvs.h;
      const int64_t step = win ? kD : a.kvs.t;
      const bool convert = bf16 && !win;
      uint4 kr[2][4], vr[8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        int r = first + 8 * (m16 >> 2) + (m16 & 3) + 4 * t;
        r = r < n ? r : n - 1;
#pragma unroll
        for (int s = 0; s < 4; ++s) kr[t][s] = *reinterpret_cast<const uint4*>(k + r * step + 32 * s + 8 * grp);
      }
      auto load_values = [&] {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          int r = first + 4 * i + grp;
          r = r < n ? r : n - 1;
          vr[i] = *reinterpret_cast<const uint4*>(v + r * step + 8 * m16);
        }
      };
      if constexpr (NB < 3) load_values();
      f4 s[NB][2];
#pragma unroll
      for (int r = 0; r < NB; ++r) s[r][0] = s[r][1] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const h8 big = __builtin_bit_cast(h8, as_f16x8(kr[t][i], convert));
#pragma unroll
          for (int r = 0; r < NB; ++r) {
            const h8 q = *reinterpret_cast<const h8*>(lds + (16 * r + m16) * 256 + (((4 * i + grp) ^ m16) << 4));
            s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(big, q, s[r][t], 0, 0, 0);
          }
        }
      if constexpr (NB == 3) {      // (no registers for them beside the keys)
        __builtin_amdgcn_sched_barrier(0);
        load_values();
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + grp;
        *reinterpret_cast<uint4*>(mine + r * 256 + ((m16 ^ twist(r)) << 4)) = as_f16x8(vr[i], convert);
      }
      h8 pw[NB];
#pragma unroll
      for (int r = 0; r < NB; ++r) {
        int row = row0 + 16 * r + m16;
        row = row < n_rows ? row : n_rows - 1;
        const int limit = (win ? n_fp16 : row / g + 1) - first;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 8 * grp + e < limit ? s[r][e >> 2][e & 3] * fl[r] : -INFINITY;
        pw[r] = weigh(st, r, x);
      }
      const int vrow = 8 * grp + (m16 >> 2), sub = (m16 & 1) * 8;
      typedef __attribute__((address_space(3))) s4* lds_s4;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const int pc = 2 * c + ((m16 >> 1) & 1);
        const h4 lo = __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(mine + vrow * 256 + ((pc ^ twist(vrow)) << 4) + sub)));
        const h4 hi = __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(mine + (vrow + 4) * 256 + ((pc ^ twist(vrow + 4)) << 4) + sub)));
        const h8 vv = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int r = 0; r < NB; ++r) st.o[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, pw[r], st.o[r][c], 0, 0, 0);
      }
    }

    // ---- the wavefronts' results meet in LDS, 16 rows at a time ----
    float* const meet = reinterpret_cast<float*>(lds);                                 // [wavefront][16][kOutRow]
    float2* const ml = reinterpret_cast<float2*>(lds + kWaves * 16 * kOutRow * 4);     // [wavefront][16]
#pragma unroll
    for (int rb = 0; rb < NB; ++rb) {
      const float sum = sum_of_groups(st.l[rb]);
      __syncthreads();
      if (lane < 16) ml[wave * 16 + lane] = make_float2(st.m[rb], sum);
#pragma unroll
      for (int c = 0; c < 8; ++c) *reinterpret_cast<f4*>(meet + (wave * 16 + m16) * kOutRow + 16 * c + 4 * grp) = st.o[rb][c];
      __syncthreads();
      const int r = tid >> 5, chan = (tid & 31) * 4, rr = row0 + 16 * rb + r;
      if (rr < n_rows) {
        float m = -INFINITY, total = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[w * 16 + r].x);
        f4 o = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float2 x = ml[w * 16 + r];
          const float f = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - m);
          total += f * x.y;
          o += f * *reinterpret_cast<const f4*>(meet + (w * 16 + r) * kOutRow + chan);
        }
        if (split_launch) {
          const size_t slot = (size_t)unit * kRows + 16 * rb + r;
          *reinterpret_cast<f4*>(a.part + slot * kD + chan) = o;
          if (chan == 0) *reinterpret_cast<float2*>(a.part + (size_t)l.n_units * kRows * kD + slot * 2) = make_float2(m, total);
        } else {
          const int t = rr / g, h = j * g + rr % g;
          o *= 1.f / total;
          const unsigned w0 = bf16 ? (unsigned)f32_to_bf16_bits(o[0]) | (unsigned)f32_to_bf16_bits(o[1]) << 16 : as_u(__builtin_convertvector(f2{o[0], o[1]}, h2));
          const unsigned w1 = bf16 ? (unsigned)f32_to_bf16_bits(o[2]) | (unsigned)f32_to_bf16_bits(o[3]) << 16 : as_u(__builtin_convertvector(f2{o[2], o[3]}, h2));
          *reinterpret_cast<uint2*>(a.out + (int64_t)b * a.os.b + (int64_t)h * a.os.h + (int64_t)t * a.os.t + chan) = make_uint2(w0, w1);
          if (a.lse && chan == 0) a.lse[((size_t)b * cfg.Hq + h) * a.n_max + t] = (m + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
        }
      }
    }
  }
};

template <int NB, int NKC, int HAS16, int NVG>
__global__ void __launch_bounds__(kThreads, 2) chunk_few_kernel(CacheView cv, ChunkArgs a, ChunkLaunch l, int split) {
  __shared__ __align__(256) unsigned char lds[Kernel<NB, NKC, HAS16, NVG>::kLds];
  Kernel<NB, NKC, HAS16, NVG>::run(cv, a, l, split != 0, lds);
}

template <int NB, int NKC, int HAS16>
static hipError_t start(const CacheView& v, const ChunkArgs& a, const ChunkLaunch& l, bool split, hipStream_t s) {
  if (v.lay.NVG == 1) chunk_few_kernel<NB, NKC, HAS16, 1><<<l.n_units, kThreads, 0, s>>>(v, a, l, split);
  else if (v.lay.NVG == 2) chunk_few_kernel<NB, NKC, HAS16, 2><<<l.n_units, kThreads, 0, s>>>(v, a, l, split);
  else chunk_few_kernel<NB, NKC, HAS16, 4><<<l.n_units, kThreads, 0, s>>>(v, a, l, split);
  return hipGetLastError();
}

// NB is a translation unit's, the rest follows the record layout (chunk_few_fits).
template <int NB>
static hipError_t start_any(const CacheView& v, const ChunkArgs& a, const ChunkLaunch& l, bool split, hipStream_t s) {
  const bool five = v.lay.NLp / 8 + v.lay.W4 > 16;
  if (v.cfg.k16 == 0) return five ? start<NB, 5, 0>(v, a, l, split, s) : start<NB, 4, 0>(v, a, l, split, s);
  return five ? start<NB, 5, 1>(v, a, l, split, s) : start<NB, 4, 1>(v, a, l, split, s);
}

}  // namespace few
}  // namespace mixkvq
