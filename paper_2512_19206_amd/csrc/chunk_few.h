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
// the zero-points.
//
// Values are dequantized in registers, c s + z rounded once, and the sum of the weights takes them as rounded: what is left of a
// rounding is relative to the values themselves.  (sum (p s) c + sum p z, with the scales in the weights, takes 64 vector instructions
// less a slice, 2 to 6 % of the time; but the two sums cancel where one element of a group lies far from the others, and p s in one half
// was then wrong by half a step of the far element: outputs up to 4e-2 off beside elements of 512.)
//
// The channels of a record stand in the order of its tiers.  Each wavefront keeps its rows of q in that order in LDS and moves
// them only where a record's lists differ from the record's before it.  What a record begins with (lists, scales, zero-points)
// is asked for a record ahead, and the scales wait in LDS, not in registers.
//
// What bounds it: vector issue.  64 sequences of 32790 tokens with 4 new ones each (40 query and 8 KV heads, K 2-bit with 12 channels
// fp16, V 2-bit) take 567 us a pass, 2.9 TB/s, with the vector ALU issuing 68 % and the matrix cores busy 37 % of the time; 4 of 131091
// with 9 new ones 183 us.  Short runs are bound by what stands around them: of the 62 us of 8 sequences of 32805 tokens with 5 new ones a
// start of 2 us, the queries' first order 4 us, the last uneven slices and the meeting of the wavefronts 6 us, the launch that merges
// splits 6 us.
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
// The largest score's weight is 2^kBoost when the sums are brought to a new reference, and no weight passes 2^kHeadroom (log2), which
// binary16 holds: most slices change nothing, and a weight counts down to 2^-33 of the largest one (with the largest one at 1 it was
// 2^-25: a first token 2^25 ahead hid all the others, whose number makes up for that).
constexpr float kHeadroom = 15.9f, kBoost = 8.f;
constexpr float kNoToken = -1e30f;                // reference of a row that has seen no token

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

// Codes 2 p and 2 p + 1 of a shifted word of 2-bit codes (p < 4) times s plus z, rounded once (see chunk_kernels.hip).  The mask
// comes in a vector register: an instruction takes one constant, and with the mask as another one it would be two.
template <int P>
__device__ __forceinline__ unsigned value_pair(unsigned x, unsigned mask, unsigned s, unsigned z) {
  constexpr unsigned kMagic = ((unsigned)(25 - 2 * P) << 10) * 0x10001u;
  const _Float16 off = (_Float16)(float)(1 << (10 - 2 * P));
  return as_u((as_h2((x & mask) | kMagic) - h2{off, off}) * as_h2(s) + as_h2(z));
}
__device__ __forceinline__ unsigned in_vgpr(unsigned x) {
  asm("" : "+v"(x));
  return x;
}
// The same number, but what is computed from it is computed here: addresses that a record needs once would otherwise be kept in
// registers through all of its slices.
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

struct __attribute__((packed, aligned(1))) uint4_any { unsigned x, y, z, w; __device__ operator uint4() const { return make_uint4(x, y, z, w); } };

__device__ __forceinline__ int twist(int r) { return ((r & 3) << 1) | (((r >> 2) ^ (r >> 3)) & 1) | (((r >> 3) & 1) << 3); }

// NB: blocks of 16 query rows.  NKC: steps of 32 channel places with codes, of which only the last may hold others than 2-bit
// ones.  HAS16: one more step with the fp16 tier.  NVG: value groups of a token.
template <int NB, int NKC, int HAS16, int NVG>
struct Kernel {
  static constexpr int kRows = 16 * NB;
  static constexpr int kPieces = 4 * (NKC + HAS16);                // 16-byte pieces of a row of q in tier order
  static constexpr int kRowBytes = 16 * kPieces;
  static constexpr int kRegion = kRows * kRowBytes > 8192 ? kRows * kRowBytes : 8192;      // of a wavefront; also 32 value rows
  static constexpr int kGroupBytes = 2 * NKC * 64;                 // scales and zero-points of a group by place
  static constexpr int kOffWave = kRows * 256;                     // behind the rows of q as given
  static constexpr int kOffGroup = kOffWave + kWaves * kRegion;
  static constexpr int kOffScale = kOffGroup + kWaves * kGroupBytes;
  static constexpr int kLds = kOffScale + kRows * 4;
  static constexpr int kOutRow = kD + 4;                           // floats of a row where the wavefronts' results meet: sums, reference, weights
  static constexpr bool kKeysEarly = NB <= 2;                      // registers for two slices' keys
  static constexpr bool kKept = NB == 1;                           // both halves of q s stay in registers through a group
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
  static_assert(kWaves * 16 * kOutRow * 4 <= kLds, "results of eight wavefronts");

  // place of piece o of row r: no two of eight neighbouring rows in one bank
  __device__ static __forceinline__ int piece(int r, int o) { return kPieces == 16 ? o ^ (r & 15) : kPieces == 20 ? o ^ ((r >> 1) & 3) : o ^ (r & 7); }

  struct State {
    // O^T by blocks of 16 channels; the ninth is a product of the weights with ones (in row 0): their sums.
    f4 o[NB][9];
    float m[NB];      // reference of the exponents (log2 units)
  };

  // Scores s f + add in log2 units (tile t, register r: token 8 group + 4 t + r) -> weights, and the sums brought to a new reference
  // if need be (which a lane sees from its own scores; only then do the lanes of a row agree on it).
  __device__ static __forceinline__ h8 weigh(State& st, int b, const float (&s)[8], float f, float add, const h8& rows) {
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i]);
    mx = __builtin_fmaf(mx, f, add);
    if (__any(mx > st.m[b] + kHeadroom)) {
      const float m = fmaxf(st.m[b], max_of_groups(mx) - kBoost), down = __builtin_amdgcn_exp2f(st.m[b] - m);
      st.m[b] = m;
#pragma unroll
      for (int c = 0; c < 9; ++c) st.o[b][c] *= down;
    }
    const float off = add - st.m[b];
    h8 p;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const h2 w = __builtin_convertvector(f2{__builtin_amdgcn_exp2f(__builtin_fmaf(s[i], f, off)), __builtin_amdgcn_exp2f(__builtin_fmaf(s[i + 1], f, off))}, h2);
      p[i] = w[0];
      p[i + 1] = w[1];
    }
    // (the sum takes the weights as rounded: what the rounding does to a row that one token rules cancels)
    st.o[b][8] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rows, p, st.o[b][8], 0, 0, 0);
    return p;
  }

  struct Keys { uint4 w[2]; unsigned four[2]; uint4 raw[2]; };
  struct Words { uint4 w[2]; uint4 s[NVG], z[NVG]; };
  struct Head { int e0, e1; unsigned s[(NKC + 3) / 4], z[(NKC + 3) / 4]; unsigned short top; };

  template <class Counts>
  __device__ static __forceinline__ void run(const ChunkArgs& a, const Counts& counts, unsigned char* lds) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m16 = lane & 15, grp = lane >> 4;
    // The arguments in one trip: read where each is first used they are several, one behind the other.
    int Hkv = a.Hkv;
    asm("" : "+s"(Hkv) : "s"(a.n_splits), "s"(a.q), "s"(a.k), "s"(a.v), "s"(a.blocks), "s"(a.table), "s"(a.res_k), "s"(a.res_v), "s"(a.qs.b),
        "s"(a.qs.h), "s"(a.qs.t), "s"(a.g), "s"(a.bf16), "s"(a.NB), "s"(a.rec_bytes), "s"(a.R), "s"(a.off_klo), "s"(a.off_klo_s));
    const ChunkPlace at = chunk_place(a, counts, blockIdx.x);
    const int g = a.g, b = at.b, j = at.j, p = at.p, n_fp16 = at.n_fp16, rt = gridDim.y - 1 - blockIdx.y, row0 = rt * kRows;
    const int n_rows = at.n_new * g;
    const bool bf16 = a.bf16 != 0;
    if (row0 >= n_rows) return;                          // (a sequence with fewer tiles of rows than others)
    __builtin_amdgcn_s_setreg(1 | 23 << 6, 1);           // MODE.FP16_OVFL: what passes 65504 stays there

    // ---- this wavefront's slices: of the records, then of the cache's fp16 rows, then of the chunk ----
    const int tile_last = row0 + kRows < n_rows ? row0 + kRows - 1 : n_rows - 1, seen = tile_last / g + 1;
    const int spr = a.R >> 5, u_rec = at.n_rec * spr, u_win = (n_fp16 + 31) >> 5, u_all = u_rec + u_win + ((seen + 31) >> 5);
    const int share = at.split * kWaves + wave, shares = at.n_splits * kWaves;
    const int u0 = (int)((long long)u_all * share / shares), u1 = (int)((long long)u_all * (share + 1) / shares);
    const bool records = u0 < u_rec && u0 < u1;
    const int end = u1 < u_rec ? u1 : u_rec;

    // (by value: a choice between two fields of an argument would keep the whole argument in memory)
    const int off_klo = a.off_klo, off_klo_s = a.off_klo_s, off_klo_z = a.off_klo_z, off_k4 = a.off_k4, off_k4_s = a.off_k4_s,
              off_k4_z = a.off_k4_z, W4 = a.W4, Wlo = a.Wlo, NLp = a.NLp, k4 = a.k4, k16 = a.k16;
    // (the table through the scalar cache: a load of the vector unit would be waited for together with all that are under way)
    typedef __attribute__((address_space(4))) const int32_t* scalar_ptr;
    const scalar_ptr table = (scalar_ptr)(uintptr_t)(a.table ? a.table + (size_t)b * a.NB : nullptr);
    auto record = [&](int blk) __attribute__((always_inline)) {
      return a.blocks + (a.table ? (size_t)table[blk] * Hkv + j : (size_t)p * a.NB + blk) * a.rec_bytes;
    };
    // All loads below are unconditional (lanes and slices that need none repeat one that is there): behind a branch the number
    // of loads under way is unknown, and the next wait is for all of them.
    // Places of a lane, chosen so that one load of 16 bytes brings the words of a token's first four steps: step i < 4 takes half
    // grp % 2 of 2-bit word 4 (grp / 2) + i.  4-bit words come last: word grp - 2 in the third step's empty half (its 2-bit words end
    // at the seventh), or word grp in a fifth step.
    const int word0 = 4 * (grp >> 1), four = NKC == 4 ? grp - 2 : grp;
    const bool has_four = four >= 0 && four < W4;
    const int tok0 = 8 * (m16 >> 2) + (m16 & 3);          // token of tile 0; 4 further in tile 1
    // Offsets of a lane in slice 0.  The odd half of a word is read from its second byte on, which leaves its codes where the masks
    // want them.
    const unsigned key_at = (unsigned)(off_klo + (tok0 * Wlo + word0) * 4 + (grp & 1)), four_at = (unsigned)(W4 ? off_k4 + (tok0 * W4 + (has_four ? four : 0)) * 4 : off_klo);
    const unsigned raw_at = (unsigned)(a.off_k16 + (tok0 * k16 + (8 * grp < k16 ? 8 * grp : 0)) * 2);
    const unsigned word_at = (unsigned)(a.off_v + (a.interleave ? grp : grp >> 1) * kD * 4 + m16 * 16 + (a.interleave ? 0 : grp & 1));
    const unsigned scale_at = (unsigned)(a.off_v_s + 16 * grp * NVG), zero_more = (unsigned)(a.off_v_z - a.off_v_s);
    auto load_keys = [&](const uint8_t* rec, int sl, Keys& k) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int from = sl * 32 + 4 * t;
        // (what lies behind a token's last word is inside the record, and meets scales of 0)
        k.w[t] = *reinterpret_cast<const uint4_any*>(rec + from * Wlo * 4 + key_at);
        k.four[t] = *reinterpret_cast<const unsigned*>(rec + from * W4 * 4 + four_at);
        // (where the tier ends inside an octet: what follows is inside the record, and may be no number; it is dropped before its use)
        if constexpr (HAS16) k.raw[t] = *reinterpret_cast<const uint4_any*>(rec + from * k16 * 2 + raw_at);
      }
    };
    // Values of a slice: words of the lane's eight tokens.  Row m of block c stands for channel 64 (c / 4) + 4 m + c % 4: two loads of
    // 16 bytes bring a lane's words of all eight blocks.  Scales and zero-points as stored, [token][group].
    auto load_words = [&](const uint8_t* rec, int sl, Words& v) __attribute__((always_inline)) {
      const uint8_t* const w = rec + (a.interleave ? (sl >> 1) * 4 * kD * 4 + (sl & 1) : sl * 2 * kD * 4);
#pragma unroll
      for (int i = 0; i < 2; ++i) v.w[i] = *reinterpret_cast<const uint4_any*>(w + word_at + 256 * i);
      const uint8_t* const m = rec + sl * 64 * NVG;
#pragma unroll
      for (int i = 0; i < NVG; ++i) {
        v.s[i] = *reinterpret_cast<const uint4*>(m + scale_at + 16 * i);
        v.z[i] = *reinterpret_cast<const uint4*>(m + zero_more + scale_at + 16 * i);
      }
    };
    // Where the scales of the pair of places 2 ln + 128 i (in the order of the steps) stand in a record; -1: nowhere.
    struct Place { int at, step, to_zero; bool four; };
    auto place_of = [&](int ln, int i) __attribute__((always_inline)) {
      const int o = (ln >> 2) + 16 * i, gp = o & 3, st = o >> 2, w = 4 * (gp >> 1) + st, fw = NKC == 4 ? gp - 2 : gp;
      Place pl{-1, NLp * 2, off_klo_z - off_klo_s, false};
      if (st < 4 && w < Wlo) pl.at = off_klo_s + (16 * w + 8 * (gp & 1) + 2 * (ln & 3)) * 2;
      else if (st == NKC - 1 && fw >= 0 && fw < W4) pl = Place{off_k4_s + (8 * fw + 2 * (ln & 3)) * 2, k4 * 2, off_k4_z - off_k4_s, true};
      return pl;
    };
    // What a group begins with: the record's lists (entries lane and lane + 64), the group's largest scale, scales and zero-points of
    // places 2 lane and 2 lane + 1 (and 128 further).
    const int ks = k4 + k16, gps = a.Gk >> 5;      // gps: slices of a group
    auto load_head = [&](const uint8_t* rec, int gr, Head& h) __attribute__((always_inline)) {
      const int ln = here(lane), last = ks > 0 ? ks - 1 : 0;
      h.e0 = rec[a.off_idx + (ln < last ? ln : last)];
      h.e1 = rec[a.off_idx + (ln + 64 < last ? ln + 64 : last)];
      h.top = *reinterpret_cast<const unsigned short*>(rec + (unsigned)(a.off_kmax + 2 * gr));
#pragma unroll
      for (int i = 0; i < (NKC + 3) / 4; ++i) {
        const Place pl = place_of(ln, i);
        const unsigned from = (unsigned)(pl.at < 0 ? off_klo_s : pl.at + gr * pl.step);
        h.s[i] = *reinterpret_cast<const unsigned*>(rec + from);
        h.z[i] = *reinterpret_cast<const unsigned*>(rec + from + (unsigned)pl.to_zero);
      }
    };
    int blk = 0, sl = 0;
    const uint8_t* rec = nullptr;
    Keys cur;
    Words val;
    Head head;
    if (records) {                                        // asked for before q, which everything waits for
      blk = u0 / spr;
      sl = u0 - blk * spr;
      rec = record(blk);
      load_head(rec, sl / gps, head);
      load_keys(rec, sl, cur);
      load_words(rec, sl, val);
    }

    // Keys of slice u of the fp16 rows: the lane's tokens and channels as the first product takes them.  Where they come first they are
    // asked for before q as well (with more rows there are no registers for that).
    uint4 kr[2][4];
    auto load_fp16_keys = [&](int u) __attribute__((always_inline)) {
      const bool win = u < u_rec + u_win;
      const int first = (u - u_rec - (win ? 0 : u_win)) * 32, n = win ? n_fp16 : seen;
      const __half* k = win ? a.res_k + (size_t)p * a.RW * kD : a.k + (int64_t)b * a.kvs.b + (int64_t)j * a.kvs.h;
      const int step = win ? kD : (int)a.kvs.t;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        int r = first + tok0 + 4 * t;
        r = r < n ? r : n - 1;
#pragma unroll
        for (int s = 0; s < 4; ++s) kr[t][s] = *reinterpret_cast<const uint4*>(k + (int64_t)r * step + 32 * s + 8 * grp);
      }
    };
    if (NB == 1 && !records && u0 < u1) load_fp16_keys(u0);

    // ---- the rows of q, each brought to a largest element of 2^6 to 2^7 (powers of two: exact) ----
    float* const row_scale = reinterpret_cast<float*>(lds + kOffScale);
#pragma unroll 1
    for (int i = tid; i < kRows * 16; i += kThreads) {
      const int r = i >> 4, o = i & 15, row = row0 + r;
      uint4 w = make_uint4(0, 0, 0, 0);
      if (row < n_rows) {
        const int t = row / g, h = j * g + row - t * g;
        w = as_f16x8(*reinterpret_cast<const uint4*>(a.q + (int64_t)b * a.qs.b + (int64_t)h * a.qs.h + (int64_t)t * a.qs.t + 8 * o), bf16);
      }
      h8 v = __builtin_bit_cast(h8, w);
      h8 av = __builtin_elementwise_abs(v);
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, (float)av[e]);
#pragma unroll 1
      for (int s = 8; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
      int k = top > 0.f ? 7 - __builtin_amdgcn_frexp_expf(top) : 0;      // (65504 has 16, the smallest subnormal -23)
      k = k > 14 ? 14 : k;
      v *= splat8((_Float16)ldexpf(1.f, k));
      *reinterpret_cast<h8*>(lds + r * 256 + ((o ^ (r & 15)) << 4)) = v;
      if (o == 0) row_scale[r] = ldexpf(a.scale * 1.4426950408889634f, -k);      // scores in log2 units
    }
    unsigned char* const mine = lds + kOffWave + wave * kRegion;
    unsigned char* const group_lds = lds + kOffGroup + wave * kGroupBytes;
#pragma unroll 2
    for (int i = 0; i < kRegion / 1024; ++i) *reinterpret_cast<uint4*>(mine + i * 1024 + lane * 16) = make_uint4(0, 0, 0, 0);
    __syncthreads();

    State st;
#pragma unroll
    for (int r = 0; r < NB; ++r) {
      st.m[r] = kNoToken;
#pragma unroll
      for (int c = 0; c < 9; ++c) st.o[r][c] = f4{0.f, 0.f, 0.f, 0.f};
    }
    const h8 ones = m16 == 0 ? splat8((_Float16)1.f) : splat8((_Float16)0.f);
    float fl[NB];
#pragma unroll
    for (int r = 0; r < NB; ++r) fl[r] = row_scale[16 * r + m16];

    if (records) {
      const bool two = NKC == 4 && !has_four;      // what a lane's word of the last step holds
      const int sh1 = two ? 0 : 8;
      const unsigned raw_lo = 8 * grp < k16 ? ~0u : 0u, raw_hi = 8 * grp + 4 < k16 ? ~0u : 0u;
      const unsigned any4 = NKC == 4 || has_four ? ~0u : 0u;
      const unsigned mk[4] = {in_vgpr(two ? 0x00030003u : 0x000f000fu & any4), in_vgpr(two ? 0x000c000cu : 0x00f000f0u & any4),
                              in_vgpr(two ? 0x00300030u : 0x000f000fu & any4), in_vgpr(two ? 0x00c000c0u : 0x00f000f0u & any4)};
      const unsigned mask[4] = {in_vgpr(0x00030003u), in_vgpr(0x000c000cu), in_vgpr(0x00300030u), in_vgpr(0x00c000c0u)};

      int have0 = -1, have1 = -1;      // the lists that the rows in `mine` are ordered by
      auto order_rows = [&](int e0, int e1) __attribute__((always_inline)) {
        if (!__any(e0 != have0 || e1 != have1)) return;
        have0 = e0;
        have1 = e1;
        const int ln = here(lane);
        unsigned long long low = ~0ull, high = ~0ull;
        int s0 = -1, s1 = -1;          // places of channels lane and lane + 64
#pragma unroll 1
        for (int e = 0; e < ks; ++e) {
          const int ch = __builtin_amdgcn_readlane(e < 64 ? e0 : e1, e & 63);
          const int place = e < k16 ? 32 * NKC + e : (NKC == 4 ? 112 : 128) + e - k16;
          const unsigned long long bit = ch < 128 ? 1ull << (ch & 63) : 0;
          if (ch < 64) low &= ~bit;
          else high &= ~bit;
          s0 = ch == ln ? place : s0;
          s1 = ch == ln + 64 ? place : s1;
        }
        const unsigned long long before = (1ull << ln) - 1;
        // 2-bit place x: half x / 8 % 2 of word x / 16
        auto low_place = [](int x) { return ((4 * (x >> 4 & 3) + 2 * (x >> 6) + (x >> 3 & 1)) << 3) + (x & 7); };
        if (s0 < 0) s0 = low_place(__popcll(low & before));
        if (s1 < 0) s1 = low_place(__popcll(low) + __popcll(high & before));
        const int p0 = s0 >> 3, q0 = (s0 & 7) * 2, p1 = s1 >> 3, q1 = (s1 & 7) * 2, c0 = ln >> 3, d0 = (ln & 7) * 2;
#pragma unroll 1
        for (int r0 = 0; r0 < kRows; r0 += 4) {
          unsigned short x[4], y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = r0 + i;
            x[i] = *reinterpret_cast<const unsigned short*>(lds + r * 256 + ((c0 ^ (r & 15)) << 4) + d0);
            y[i] = *reinterpret_cast<const unsigned short*>(lds + r * 256 + (((c0 + 8) ^ (r & 15)) << 4) + d0);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = r0 + i;
            *reinterpret_cast<unsigned short*>(mine + r * kRowBytes + (piece(r, p0) << 4) + q0) = x[i];
            *reinterpret_cast<unsigned short*>(mine + r * kRowBytes + (piece(r, p1) << 4) + q1) = y[i];
          }
        }
      };
      auto rows_of = [&](int r, int step) __attribute__((always_inline)) {
        return *reinterpret_cast<const h8*>(mine + (16 * r + m16) * kRowBytes + (piece(m16, 4 * step + grp) << 4));
      };
      auto group_of = [&](int what, int step) __attribute__((always_inline)) {      // 0: scales, 1: zero-points
        return *reinterpret_cast<const h8*>(group_lds + what * NKC * 64 + step * 64 + grp * 16);
      };

      h8 hi[kKept ? NB : 1][kKept ? NKC : 1], lo[kKept ? NB : 1][kKept ? NKC : 1];
      float fg[NB], bias[NB], rho = 0.f;      // scores = codes' sums * fg + bias; fp16 tier's sums * rho join the codes'
      bool group = true;
      for (int u = u0; u < end; ++u) {
        // Of two wavefronts on a SIMD the older one goes first; the younger one takes every other slice ahead of it, else it is left
        // with a part of the work that nothing overlaps.
        if (wave >= kWaves / 2) {
          if (u & 1) __builtin_amdgcn_s_setprio(1);
          else __builtin_amdgcn_s_setprio(0);
        }
        if (group) {
          const int gr = sl / gps;
          order_rows(lane < ks ? head.e0 : 255, lane + 64 < ks ? head.e1 : 255);
          // the largest scale becomes 2^6 to 2^7: products with q stay below 2^14, small ones keep their bits
          const float top = (float)__builtin_bit_cast(_Float16, head.top);
          int e = top > 0.f ? 7 - __builtin_amdgcn_frexp_expf(top) : 0;
          e = __builtin_amdgcn_readfirstlane(e > 14 ? 14 : e);
          const int ln = here(lane);
#pragma unroll
          for (int i = 0; i < (NKC + 3) / 4; ++i) {
            // the codes of pair x of an octet come with 4^x (4-bit ones: 16^(x % 2))
            const Place pl = place_of(ln, i);
            const int x = ln & 3, place = 2 * ln + 128 * i, down = pl.four ? 4 * (x & 1) : 2 * x;
            const _Float16 f = (_Float16)ldexpf(1.f, e - down);
            if (place < 32 * NKC) {
              *reinterpret_cast<unsigned*>(group_lds + place * 2) = pl.at < 0 ? 0u : as_u(as_h2(head.s[i]) * h2{f, f});
              *reinterpret_cast<unsigned*>(group_lds + NKC * 64 + place * 2) = pl.at < 0 ? 0u : head.z[i];
            }
          }
          const float back = ldexpf(16777216.f, -e);
          rho = ldexpf(5.9604644775390625e-8f, e);
#pragma unroll
          for (int r = 0; r < NB; ++r) {
            f4 acc = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < NKC; ++s) {
              const h8 q = rows_of(r, s);
              acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(group_of(1, s), q, acc, 0, 0, 0);
              if constexpr (kKept) {
                hi[r][s] = q * group_of(0, s);
                lo[r][s] = __builtin_elementwise_fma(q, group_of(0, s), -hi[r][s]);
              }
            }
            fg[r] = fl[r] * back;
            bias[r] = acc[0] * fl[r];
          }
          // the next group's, a group ahead
          const int left = gps - (sl - gr * gps);
          const bool over = (gr + 1) * gps == spr;
          const bool more = u + left < end;
          load_head(over && more ? record(blk + 1) : rec, !more ? gr : over ? 0 : gr + 1, head);
        }
        // keys of the next slice
        Keys next;
        const bool turn = sl + 1 == spr, more = u + 1 < end;
        const int nsl = !more ? sl : turn ? 0 : sl + 1, nblk = turn ? blk + 1 : blk;
        const uint8_t* const nrec = turn && more ? record(nblk) : rec;
        if constexpr (kKeysEarly) load_keys(nrec, nsl, next);
        // ---- scores ----
        f4 s[NB][2], s16[HAS16 ? NB : 1][2];
#pragma unroll
        for (int r = 0; r < NB; ++r) s[r][0] = s[r][1] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NKC; ++k) {
          h8 big[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            unsigned w = k == 0 ? cur.w[t].x : k == 1 ? cur.w[t].y : k == 2 ? cur.w[t].z : k == 3 ? cur.w[t].w : cur.four[t];
            if (k < NKC - 1) {
              big[t] = as_h8(w & mask[0], w & mask[1], w & mask[2], w & mask[3]);
            } else {      // 2-bit codes in some lanes, 4-bit codes (or nothing) in others
              const unsigned v = in_vgpr(cur.four[t]);      // (in a register: a choice between two members would keep them in memory)
              w = NKC == 4 ? (has_four ? v : w) : v;
              const unsigned y = w >> sh1;
              big[t] = as_h8(w & mk[0], w & mk[1], y & mk[2], y & mk[3]);
            }
          }
          h8 f;
          if constexpr (!kKept) f = group_of(0, k);
#pragma unroll
          for (int r = 0; r < NB; ++r) {
            h8 qh, ql;
            if constexpr (kKept) {
              qh = hi[r][k];
              ql = lo[r][k];
            } else {
              const h8 q = rows_of(r, k);
              qh = q * f;
              ql = __builtin_elementwise_fma(q, f, -qh);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(big[t], qh, s[r][t], 0, 0, 0);
#pragma unroll
            for (int t = 0; t < 2; ++t) s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(big[t], ql, s[r][t], 0, 0, 0);
          }
        }
        if constexpr (HAS16) {
#pragma unroll
          for (int r = 0; r < NB; ++r)
#pragma unroll
            for (int t = 0; t < 2; ++t)
              s16[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(cur.raw[t].x & raw_lo, cur.raw[t].y & raw_lo, cur.raw[t].z & raw_hi, cur.raw[t].w & raw_hi),
                                                                 rows_of(r, NKC), f4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        }
        if constexpr (kKeysEarly) cur = next;
        else load_keys(nrec, nsl, cur);
        sl = nsl;
        blk = nblk;
        rec = nrec;
        group = sl % gps == 0;
        h8 pw[NB];
#pragma unroll
        for (int r = 0; r < NB; ++r) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[i] = s[r][i >> 2][i & 3];
            if constexpr (HAS16) x[i] = __builtin_fmaf(s16[r][i >> 2][i & 3], rho, x[i]);
          }
          pw[r] = weigh(st, r, x, fg[r], bias[r], ones);
          if constexpr (NB > 2) __builtin_amdgcn_sched_barrier(0);      // one block's scores at a time: registers
        }
        // ---- values ----
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const uint4 four_words = val.w[c >> 2];
          const unsigned x = (c & 3) == 0 ? four_words.x : (c & 3) == 1 ? four_words.y : (c & 3) == 2 ? four_words.z : four_words.w;
          unsigned sp[4], z4[4];         // pairs of tokens of the group of channel 64 (c / 4) + 4 m16 + c % 4
          const unsigned* ps = reinterpret_cast<const unsigned*>(val.s);
          const unsigned* pz = reinterpret_cast<const unsigned*>(val.z);
          const int dw = NVG == 2 ? 0 : c >> 2;
          const unsigned pick = (NVG == 2 ? c >> 2 : m16 >> 3) ? 0x07060302u : 0x05040100u;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int d0 = NVG == 1 ? i : i * NVG + dw, d1 = d0 + NVG / 2;      // of tokens 2 i and 2 i + 1
            sp[i] = NVG == 1 ? ps[i] : __builtin_amdgcn_perm(ps[d1], ps[d0], pick);
            z4[i] = NVG == 1 ? pz[i] : __builtin_amdgcn_perm(pz[d1], pz[d0], pick);
          }
          const h8 v = as_h8(value_pair<0>(x, mask[0], sp[0], z4[0]), value_pair<1>(x, mask[1], sp[1], z4[1]),
                             value_pair<2>(x, mask[2], sp[2], z4[2]), value_pair<3>(x, mask[3], sp[3], z4[3]));
#pragma unroll
          for (int r = 0; r < NB; ++r) st.o[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pw[r], st.o[r][c], 0, 0, 0);
        }
        load_words(rec, sl, val);
      }
    }

    // ---- fp16 rows: those of the cache, then the chunk's own ----
#pragma unroll 1
    for (int u = u0 > u_rec ? u0 : u_rec; u < u1; ++u) {
      const bool win = u < u_rec + u_win;
      const int first = (u - u_rec - (win ? 0 : u_win)) * 32, n = win ? n_fp16 : seen;
      const __half* v = win ? a.res_v + (size_t)p * a.RW * kD : a.v + (int64_t)b * a.kvs.b + (int64_t)j * a.kvs.h;
      const int step = win ? kD : (int)a.kvs.t;
      uint4 vr[8];
      if (NB > 1 || records || u > u0) load_fp16_keys(u);
      auto load_values = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          int r = first + 4 * i + grp;
          r = r < n ? r : n - 1;
          vr[i] = *reinterpret_cast<const uint4*>(v + (int64_t)r * step + 8 * m16);
        }
      };
      if constexpr (NB < 3) load_values();
      if (bf16 && !win) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int s = 0; s < 4; ++s) kr[t][s] = as_f16x8(kr[t][s], true);
      }
      f4 s[NB][2];
#pragma unroll
      for (int r = 0; r < NB; ++r) s[r][0] = s[r][1] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < NB; ++r) {
          const h8 q = *reinterpret_cast<const h8*>(lds + (16 * r + m16) * 256 + (((4 * i + grp) ^ m16) << 4));
#pragma unroll
          for (int t = 0; t < 2; ++t) s[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, kr[t][i]), q, s[r][t], 0, 0, 0);
        }
      if constexpr (NB == 3) {      // (no registers for them beside the keys)
        __builtin_amdgcn_sched_barrier(0);
        load_values();
      }
      if (bf16 && !win) {
#pragma unroll
        for (int i = 0; i < 8; ++i) vr[i] = as_f16x8(vr[i], true);
      }
      // into LDS in the order of the blocks: channels 8 m16 + i and 8 m16 + 4 + i are neighbours in block 4 (m16 / 8) + i
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + grp;
        const unsigned lo[2] = {vr[i].x, vr[i].y}, hi[2] = {vr[i].z, vr[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = 4 * (m16 >> 3) + e, pc = 2 * c + ((m16 >> 2) & 1);
          *reinterpret_cast<unsigned*>(mine + r * 256 + ((pc ^ twist(r)) << 4) + (m16 & 3) * 4) =
              __builtin_amdgcn_perm(hi[e >> 1], lo[e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
        }
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
        pw[r] = weigh(st, r, x, 1.f, 0.f, ones);
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

    // ---- the wavefronts' results meet in LDS, 16 rows at a time: 32 threads to a row, which sum the eight ----
    float* const meet = reinterpret_cast<float*>(lds);                                 // [wavefront][16][kOutRow]
    const int mr = tid >> 5, chan = (tid & 31) * 4;
#pragma unroll 1
    for (int rb = 0; rb < NB; ++rb) {
      __syncthreads();
      float* const to = meet + (wave * 16 + m16) * kOutRow;
#pragma unroll
      for (int r = 0; r < NB; ++r) {
        if (r != rb) continue;
        // register e of block c is channel 64 (c / 4) + 16 group + 4 e + c % 4
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<f4*>(to + 64 * (i >> 2) + 16 * grp + 4 * (i & 3)) =
              f4{st.o[r][4 * (i >> 2)][i & 3], st.o[r][4 * (i >> 2) + 1][i & 3], st.o[r][4 * (i >> 2) + 2][i & 3], st.o[r][4 * (i >> 2) + 3][i & 3]};
        if (grp == 0) *reinterpret_cast<f2*>(to + kD) = f2{st.m[r], st.o[r][8][0]};
      }
      __syncthreads();
      const int rr = row0 + 16 * rb + mr;
      if (rr >= n_rows) continue;
      f2 ml[kWaves];
      float m = kNoToken;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        ml[w] = *reinterpret_cast<const f2*>(meet + (w * 16 + mr) * kOutRow + kD);
        m = fmaxf(m, ml[w][0]);
      }
      float total = 0.f;
      f4 o = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[w][0] - m);
        total += f * ml[w][1];
        o += f * *reinterpret_cast<const f4*>(meet + (w * 16 + mr) * kOutRow + chan);
      }
      if (a.split) {
        const size_t slot = ((size_t)blockIdx.x * gridDim.y + rt) * kRows + 16 * rb + mr;
        *reinterpret_cast<f4*>(a.part + slot * kD + chan) = o;
        if (chan == 0) *reinterpret_cast<float2*>(a.part + (size_t)gridDim.x * gridDim.y * kRows * kD + slot * 2) = make_float2(m, total);
      } else {
        const int t = rr / g, h = j * g + rr - t * g;
        o *= 1.f / total;
        uint2 w;
        if (bf16) w = make_uint2((unsigned)f32_to_bf16_bits(o[0]) | (unsigned)f32_to_bf16_bits(o[1]) << 16, (unsigned)f32_to_bf16_bits(o[2]) | (unsigned)f32_to_bf16_bits(o[3]) << 16);
        else w = make_uint2(as_u(__builtin_convertvector(f2{o[0], o[1]}, h2)), as_u(__builtin_convertvector(f2{o[2], o[3]}, h2)));
        *reinterpret_cast<uint2*>(a.out + (int64_t)b * a.os.b + (int64_t)h * a.os.h + (int64_t)t * a.os.t + chan) = w;
        if (a.lse && chan == 0) a.lse[((size_t)b * a.Hq + h) * a.n_max + t] = (m + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
      }
    }
  }
};

template <int NB, int NKC, int HAS16, int NVG, class Counts>
__global__ void __launch_bounds__(kThreads, 2) chunk_few_kernel(ChunkArgs a, Counts c) {
  __shared__ __align__(256) unsigned char lds[Kernel<NB, NKC, HAS16, NVG>::kLds];
  Kernel<NB, NKC, HAS16, NVG>::run(a, c, lds);
}

template <int NB, int NKC, int HAS16, int NVG>
static hipError_t start(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s) {
  const dim3 grid(units * a.Hkv, a.row_tiles);
  if (c) chunk_few_kernel<NB, NKC, HAS16, NVG, ChunkCounts><<<grid, kThreads, 0, s>>>(a, *c);
  else chunk_few_kernel<NB, NKC, HAS16, NVG, NoChunkCounts><<<grid, kThreads, 0, s>>>(a, NoChunkCounts{});
  return hipGetLastError();
}
template <int NB, int NKC, int HAS16>
static hipError_t start_groups(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s) {
  return a.NVG == 1 ? start<NB, NKC, HAS16, 1>(a, c, units, s) : a.NVG == 2 ? start<NB, NKC, HAS16, 2>(a, c, units, s) : start<NB, NKC, HAS16, 4>(a, c, units, s);
}

// NB is a translation unit's, the rest follows the record layout (chunk_few_fits).
template <int NB>
static hipError_t start_any(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s) {
  const bool five = chunk_few_steps(a.NLp, a.W4) == 5;
  if (a.k16 == 0) return five ? start_groups<NB, 5, 0>(a, c, units, s) : start_groups<NB, 4, 0>(a, c, units, s);
  return five ? start_groups<NB, 5, 1>(a, c, units, s) : start_groups<NB, 4, 1>(a, c, units, s);
}

}  // namespace few
}  // namespace mixkvq
