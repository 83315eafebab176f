// Attention of a chunk of new tokens over the mixed-precision cache and over the chunk itself, causally (Section 3.1, Eq. 1,
// with keys and values dequantized by Eq. 3).
//
// One workgroup of eight wavefronts takes a tile of 256 query rows (a row is one query head at one new token; the g heads of
// a KV head share its keys) and walks over the tokens in tiles of 128: packed records, then the fp16 rows of the cache, then
// the chunk's own keys and values.  Both products run on the matrix cores in the transposed form, S^T = K Q^T and
// O^T = V^T P^T, 32 tokens (channels) by 32 rows at a time: a lane then holds one row's scores, so that the softmax needs
// one exchange between the two halves of the wavefront, and the weights P go into the second product from the registers in
// which the first one left them.
//
// 256 rows, because a tile is dequantized once for all of them: unpacking takes 3 500 of a wavefront's 13 000 cycles for a tile of
// records.  Keys and values stand in LDS as binary16, two tiles of each (162 KB with the record on its way): the next tile is
// unpacked while this one is used, its keys in the first half of the steps, its values in the second.  A wavefront keeps its 32
// rows of Q and O in registers.
//
// What bounds it: issue.  A step (32 tokens by 32 rows) is 16 matrix instructions of 32 cycles and about 100 vector ones, 16 of them
// exponentials; on a SIMD's two wavefronts that is 1 024 matrix and about 1 250 vector cycles, of which at best 1 320 remain
// together (a matrix instruction holds the vector issue for 8 cycles), and 1 700 were measured.  So scores of the next slice, weights
// of this one and values of the last one are interleaved by hand; with the compiler's order, or with products and exponentials
// in turn, 8192 new tokens over an empty cache (28 query and 4 KV heads) took 645 and 581 us, and 500 us a pass this way (960 TFLOP/s;
// a large library product reaches 1 171 on this card).  Barriers (two to a tile), the tile's way through LDS and the start and end
// of a workgroup take a third of the time.
// 1000 new tokens after 31000 cached ones (K 2-bit with 16 channels 4-bit, V 2-bit, bfloat16) take 682 us a pass, 662 TFLOP/s; 2 x 2048
// after 8190 (records of 32) 1105 us, 700 TFLOP/s.
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
constexpr int kOffPick = kOffMap + 2 * kChunkRecords * kD * 2;    // [9] halves: 1 in place 0 .. 7, and nowhere
constexpr int kLdsBytes = kOffPick + 9 * 16;
// What binary16 drops of the 4-bit tier's keys: a row per list entry, twice (two tiles), where records leave room for it.
constexpr int kRestRows = 16, kRestBytes = kRestRows * kRowBytes, kOffRest = kOffScale - 2 * kRestBytes;
static_assert(kLdsBytes <= 160 * 1024, "LDS of a compute unit");
constexpr int kOutRow = kD + 4;                                  // floats of a row where the wavefronts' results meet
constexpr int kRows = 256;                                        // query rows of a workgroup: 32 to a wavefront
static_assert(kRows * kOutRow * 4 + kRows * 8 <= kLdsBytes, "the results");

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
// The masks come in vector registers: an instruction takes one constant, and with the mask as another one it would be two.
template <int BITS, int I>
struct CodeAt {
  static constexpr int kShift = BITS * I;                       // of the code in its half-word; it has to stand in the ten mantissa bits
  static constexpr int kUp = kShift + BITS <= 10 ? kShift : kShift - (BITS == 2 ? 10 : 8);
  static_assert(kUp >= 0 && kUp + BITS <= 10, "inside the mantissa");
  static constexpr unsigned kMask = (((1u << BITS) - 1u) << kUp) * 0x10001u, kMagic = ((unsigned)(25 - kUp) << 10) * 0x10001u;
};
template <int BITS, int I>
__device__ __forceinline__ unsigned dequant(unsigned w, const unsigned (&mask)[5], h2 s, h2 z) {
  typedef CodeAt<BITS, I> C;
  const unsigned x = C::kShift == C::kUp ? w : w >> (C::kShift - C::kUp);
  const _Float16 off = (_Float16)(float)(1 << (10 - C::kUp));
  return as_u((as_h2((x & mask[C::kUp / BITS]) | C::kMagic) - h2{off, off}) * s + z);
}
// What `k` drops of two 4-bit codes times s plus z: exact products and sums of binary32 (15 bits, and 11 at not too far an exponent).
template <int I>
__device__ __forceinline__ unsigned dropped(unsigned w, unsigned k, h2 s, h2 z) {
  const h2 h = as_h2(k), sz = s, zz = z;
  const float c0 = (float)((w >> (4 * I)) & 15u), c1 = (float)((w >> (16 + 4 * I)) & 15u);
  const float r0 = __builtin_fmaf(c0, (float)sz[0], (float)zz[0]) - (float)h[0], r1 = __builtin_fmaf(c1, (float)sz[1], (float)zz[1]) - (float)h[1];
  return as_u(__builtin_convertvector(f2{r0, r1}, h2));
}
__device__ __forceinline__ unsigned in_vgpr(unsigned x) {
  asm("" : "+v"(x));
  return x;
}

// State of one wavefront: 32 query rows, one to a lane and its partner 32 lanes away.
struct Rows {
  h8 q[8];            // B operand of step i: channels 16 i + 8 half ..
  f16v o[4];          // O^T: channels 32 c + 8 (r / 4) + 4 half + r % 4, relative to m
  float m, l;         // reference of the exponents (log2 units) and this lane's share of the sum of the weights
};

// The kernel's arguments, read anew from where the launch put them (ChunkArgs is a kernel's first argument): what is read through this
// is not kept in scalar registers across the loop, which runs out of them.
typedef __attribute__((address_space(4))) const ChunkArgs ArgsIn;
__device__ __forceinline__ ArgsIn& args_here() {
  ArgsIn* x = (ArgsIn*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(x));
  return *x;
}

// The thread's number, found anew: what is made of it is not kept in registers from one tile to the next.
__device__ __forceinline__ int tid_here() {
  int x = threadIdx.x;
  asm volatile("" : "+v"(x));
  return x;
}

// The largest score may run ahead of the reference by kHeadroom (in log2) before the sums are brought to a new reference, kBoost (or
// up to one more) below it: weights stay inside binary16, most tiles change nothing, and a weight counts down to 2^-32 of the
// largest one (with the largest one at 1 it was 2^-25: a first token 2^25 ahead hid all the others, whose number makes up for that).
constexpr float kHeadroom = 15.9f, kBoost = 8.f;
constexpr float kNoToken = -1e30f;      // reference of a row that has seen no token

// Where a lane reads its operands: addresses that stand for a whole tile (the rest is the instructions' constant offset).  BY_CHANNEL: the
// tiles have a row per channel (records), else a row per token.
// Row 8 a + 4 h + i of a slice of 32 scores stands for token 16 (a / 2) + 8 h + 4 (a % 2) + i: a lane then holds runs of eight
// neighbouring tokens, which is what the second product takes.
template <bool BY_CHANNEL>
struct Operands {
  int k[8], v[8];
  __device__ __forceinline__ Operands() {
    const int lane = threadIdx.x & 63, half = lane >> 5, i16 = lane & 15, grp = lane >> 4, m = lane & 31;
    const int row = 8 * (grp >> 1) + (i16 >> 2);      // of a transposing read, and four rows on
    if constexpr (BY_CHANNEL) {
      const int piece = 2 * (grp & 1) + (i16 & 1), sub = ((i16 >> 1) & 1) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {                   // slice i / 2
        k[i] = (row + 4 * (i & 1)) * kRowBytes + sub + ((piece ^ twist(row + 4 * (i & 1)) ^ (i >> 1) << 2) << 4);
        v[i] = kKeyBytes + m * kRowBytes + ((half ^ twist(m) ^ i << 1) << 4);
      }
    } else {
      const int token = 16 * (m >> 4) + 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3);
      const int piece = 2 * (grp & 1) + ((i16 >> 1) & 1), sub = (i16 & 1) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {                   // channels 16 i .. of the keys, 32 (i / 2) .. of the values
        k[i] = token * kRowBytes + ((half ^ twist(token) ^ i << 1) << 4);
        v[i] = kKeyBytes + (row + 4 * (i & 1)) * kRowBytes + sub + ((piece ^ twist(row + 4 * (i & 1)) ^ (i >> 1) << 2) << 4);
      }
    }
    move(k, 0);
    move(v, 0);
  }
  // To the other of the two tiles in LDS.
  static __device__ __forceinline__ void move(int (&x)[8], int by) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] += by;
      asm volatile("" : "+v"(x[i]));
    }
  }
  // Channels 16 i .. of a slice's keys.
  __device__ __forceinline__ h8 key(unsigned char* lds, int slice, int i) const {
    if constexpr (BY_CHANNEL)
      return join(lds_column(lds, k[2 * slice] + i * 16 * kRowBytes), lds_column(lds, k[2 * slice + 1] + i * 16 * kRowBytes));
    else
      return lds_h8(lds, k[i] + slice * 32 * kRowBytes);
  }
  // Channels 32 c .. at tokens 16 t .. of a slice's values.
  __device__ __forceinline__ h8 value(unsigned char* lds, int slice, int t, int c) const {
    if constexpr (BY_CHANNEL)
      return lds_h8(lds, v[2 * slice + t] + c * 32 * kRowBytes);
    else
      return join(lds_column(lds, v[2 * c] + (slice * 32 + t * 16) * kRowBytes), lds_column(lds, v[2 * c + 1] + (slice * 32 + t * 16) * kRowBytes));
  }
};

// Tokens of the tile from `limit` on do not count for this lane's row.
__device__ __forceinline__ void hide(int slice, int limit, f16v& s) {
  const int left = limit - slice * 32 - 8 * ((threadIdx.x & 63) >> 5);
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (16 * (r >> 3) + (r & 7) >= left) s[r] = -INFINITY;
}

__device__ __forceinline__ float largest(const f16v& s) {
  float mx = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
  return mx;
}

// Brings the sums and the weights that are still to be used to a new reference if a score (mx: this lane's largest) has run too far
// ahead; only then do the two lanes of a row agree on it.  References are whole numbers: the weights' factor is a power of two, taken
// in two parts because a weight of nearly 2^16 may still count when the whole factor is below binary16.
__device__ __forceinline__ void follow(float mx, Rows& st, h8 (&p)[2]) {
  if (__any(mx > st.m + kHeadroom)) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    const float m = fmaxf(st.m, ceilf(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]))) - kBoost), back = st.m - m, f = __builtin_amdgcn_exp2f(back);
    st.m = m;
    st.l *= f;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[b][r] *= f;
    const _Float16 f0 = (_Float16)__builtin_amdgcn_exp2f(fmaxf(back, -14.f)), f1 = (_Float16)__builtin_amdgcn_exp2f(fminf(back + 14.f, 0.f));
#pragma unroll
    for (int i = 0; i < 2; ++i) p[i] = p[i] * h8{f0, f0, f0, f0, f0, f0, f0, f0} * h8{f1, f1, f1, f1, f1, f1, f1, f1};
  }
}

// What a wavefront carries from step to step.
template <bool BY_CHANNEL>
struct Pipe {
  Operands<BY_CHANNEL> at;
  h8 k[4], v[4];      // the next operands of the two products: a ring, each refilled four matrix instructions ahead
  h8 q;               // queries at the channels of the 4-bit list, entries 8 half ..
  int entry;          // this lane's entry of that list
};

// The queries at a list's channels, as the ninth operand of a slice's scores: a product with ones at (entry, channel), which is
// exact.  entry: the channel of entry 8 (m / 4 % 2) + 4 (m / 8) + m % 4 in lane m < 16 (and m + 32), no channel elsewhere.
__device__ __forceinline__ h8 pick_queries(unsigned char* lds, int entry, const Rows& st) {
  f16v d;
#pragma unroll
  for (int r = 0; r < 16; ++r) d[r] = 0.f;
  const unsigned from = entry - 8 * ((threadIdx.x & 63) >> 5);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const unsigned at = from - 16 * i;
    d = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds_h8(lds, kOffPick + (at < 8 ? at : 8) * 16), st.q[i], d, 0, 0, 0);
  }
  h8 q;
#pragma unroll
  for (int r = 0; r < 8; ++r) q[r] = (_Float16)d[r];
  return q;
}

// Entries of a staged tile's 4-bit lists for pick_queries, a byte for each slice (255: none).
__device__ __forceinline__ unsigned list_entries(const unsigned char* lds, int n_rec) {
  ArgsIn& a = args_here();
  const int m = tid_here() & 31, e = 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3);
  unsigned all = 0;
#pragma unroll
  for (int slice = 0; slice < 4; ++slice) {
    const int rec = 32 * slice * a.inv_r >> 16;
    const bool there = rec < n_rec && m < 16 && e < a.k4;
    const unsigned c = lds[kOffRaw + (there ? rec * a.rec_bytes + a.off_idx + a.k16 + e : 0)];
    all |= (there ? c : 255u) << (8 * slice);
  }
  return all;
}

__device__ __forceinline__ void take_list(unsigned char* lds, Pipe<true>& in, unsigned entries, int slice, const Rows& st) {
  const int entry = entries >> (8 * slice) & 255;
  if (__any(entry != in.entry)) {      // (lists change slowly)
    in.entry = entry;
    in.q = pick_queries(lds, entry, st);
  }
}

// One step of a wavefront, on three slices at once: the scores of slice SLICE + 1 are formed (`next`), those of slice SLICE (`cur`, hidden
// and followed) become weights (`p`), and the values of the slice before are added with its weights (`before`).  Nothing of
// this depends on anything else of it, and the order is fixed piece by piece: every matrix instruction finds its operands in
// registers and has a sixteenth of the vector instructions behind it, so that neither the LDS nor the exponentials are waited for.
// Out: the next scores, hidden and followed.  REST: the scores have a ninth product, what binary16 drops of the 4-bit tier's keys (the rows
// from rest on, less the keys' address) by the queries at its channels (entries).
template <int SLICE, bool REST, bool BY_CHANNEL>
__device__ __forceinline__ void step(unsigned char* lds, Pipe<BY_CHANNEL>& in, int move, int rest, unsigned entries, f16v& cur, f16v& next, const h8 (&before)[2], h8 (&p)[2],
                                     bool masked, int limit, float c, Rows& st) {
  float sum = 0.f, mx = 0.f;
  h8 dropped;
  if constexpr (REST) {
    constexpr int kNext = (SLICE + 1) & 3;
    take_list(lds, in, entries, kNext, st);
    dropped = join(lds_column(lds, in.at.k[2 * kNext] + rest), lds_column(lds, in.at.k[2 * kNext + 1] + rest));
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) next[r] = 0.f;
#pragma unroll
  for (int s = 0, e = 0; s < 16; ++s) {
    if (s < 12 && s % 3 != 2) {
      const int i = s - s / 3;
      next = __builtin_amdgcn_mfma_f32_32x32x16_f16(in.k[i & 3], st.q[i], next, 0, 0, 0);
      if (SLICE == 2 && i == 4) in.at.move(in.at.k, move);      // the keys that follow are the next tile's
      in.k[i & 3] = in.at.key(lds, (SLICE + (i < 4 ? 1 : 2)) & 3, (i + 4) & 7);
    } else {
      const int i = s < 12 ? s / 3 : s - 8;
      st.o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(in.v[i & 3], before[i >> 2], st.o[i & 3], 0, 0, 0);
      if (SLICE == 0 && i == 4) in.at.move(in.at.v, move);      // the values that follow are this tile's
      in.v[i & 3] = in.at.value(lds, (SLICE + (i < 4 ? 3 : 0)) & 3, i < 4, i & 3);
    }
    if (s * 2 >= e * 3 && e < 8) {
      const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(cur[2 * e], c, -st.m)), e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(cur[2 * e + 1], c, -st.m));
      const h2 w = __builtin_convertvector(f2{e0, e1}, h2);      // nearest: a truncated weight would pull every output to zero
      sum = __builtin_amdgcn_fdot2(w, h2{(_Float16)1.f, (_Float16)1.f}, sum, false);
      asm volatile("" : "+v"(sum));
      p[e >> 2][2 * (e & 3)] = w[0];
      p[e >> 2][2 * (e & 3) + 1] = w[1];
      ++e;
    }
    if (REST && s == 10) next = __builtin_amdgcn_mfma_f32_32x32x16_f16(dropped, in.q, next, 0, 0, 0);
    if (s == 14) mx = largest(next);
    __builtin_amdgcn_sched_barrier(0);
  }
  st.l += sum;
  if (masked) {
    asm volatile("");      // (a branch, and not 16 selections in every step)
    hide((SLICE + 1) & 3, limit, next);
    mx = largest(next);
  }
  follow(mx * c, st, p);
}

// What the first step takes: the first slice's scores, no weights, operands in the rings.  Rows see `limit` tokens of the tile, all of
// them `all`.
template <bool REST, bool BY_CHANNEL>
__device__ __forceinline__ void begin(unsigned char* lds, Pipe<BY_CHANNEL>& in, unsigned entries, int all, int limit, float c, f16v& s, h8 (&p)[2], Rows& st) {
#pragma unroll
  for (int i = 0; i < 4; ++i) in.k[i] = in.at.key(lds, 0, i);
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    s = __builtin_amdgcn_mfma_f32_32x32x16_f16(in.k[i & 3], st.q[i], s, 0, 0, 0);
    in.k[i & 3] = in.at.key(lds, i < 4 ? 0 : 1, (i + 4) & 7);
  }
  if constexpr (REST) {
    in.entry = -1;
    take_list(lds, in, entries, 0, st);
    s = __builtin_amdgcn_mfma_f32_32x32x16_f16(join(lds_column(lds, in.at.k[0] + kOffRest), lds_column(lds, in.at.k[1] + kOffRest)), in.q, s, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) p[i] = h8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) in.v[i] = in.at.value(lds, 3, 0, i);      // (taken times 0)
  if (32 > all) {
    asm volatile("");
    hide(0, limit, s);
  }
  follow(largest(s) * c, st, p);
}

// The last slice's values.
template <bool BY_CHANNEL>
__device__ __forceinline__ void finish(unsigned char* lds, Pipe<BY_CHANNEL>& in, const h8 (&p)[2], Rows& st) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    st.o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_f16(in.v[i & 3], p[i >> 2], st.o[i & 3], 0, 0, 0);
    if (i < 4) in.v[i] = in.at.value(lds, 3, 1, i);
  }
}

// Dequantizes the 2-bit channels of the staged tile's keys into `keys` (a row per channel): threads 0 .. 255.
__device__ __forceinline__ void unpack_low_keys(unsigned char* lds, int keys, const unsigned short* map, int n_tok) {
  ArgsIn& a = args_here();
  const int Rr = a.R, inv_r = a.inv_r, inv_gk = a.inv_gk, tid = tid_here();
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const unsigned two[5] = {in_vgpr(CodeAt<2, 0>::kMask), in_vgpr(CodeAt<2, 1>::kMask), in_vgpr(CodeAt<2, 2>::kMask), in_vgpr(CodeAt<2, 3>::kMask), in_vgpr(CodeAt<2, 4>::kMask)};
  {  // 2-bit channels: eight tokens of the eight even or odd channels of a word
    const int odd = wave & 1, tg = (wave >> 1) * 8 + (lane & 7), w = lane >> 3, t = tg * 8;
    if (w < a.Wlo && t < n_tok) {
      const int rec = t * inv_r >> 16, tin = t - rec * Rr, raw = kOffRaw + rec * a.rec_bytes;
      const int words = raw + a.off_klo + (tin * a.Wlo + w) * 4;
      const unsigned pick = odd ? 0x07060302u : 0x05040100u, twice = odd ? 0x03020302u : 0x01000100u;
      unsigned x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = __builtin_amdgcn_perm(*reinterpret_cast<const unsigned*>(lds + words + (2 * i + 1) * a.Wlo * 4),
                                     *reinterpret_cast<const unsigned*>(lds + words + 2 * i * a.Wlo * 4), pick);
      const int sc = raw + a.off_klo_s + ((tin * inv_gk >> 16) * a.NLp + 16 * w) * 2, zc = sc + a.off_klo_z - a.off_klo_s;
      const unsigned* s = reinterpret_cast<const unsigned*>(lds + sc);
      const unsigned* z = reinterpret_cast<const unsigned*>(lds + zc);
      const unsigned* at = reinterpret_cast<const unsigned*>(map + rec * kD + 16 * w);
      const int col = tg << 4;
#define MIXKVQ_CHANNEL(I)                                                                                                  \
  {                                                                                                                        \
    const h2 s2 = as_h2(__builtin_amdgcn_perm(s[I], s[I], twice)), z2 = as_h2(__builtin_amdgcn_perm(z[I], z[I], twice));   \
    const int to = keys + (((at[I] >> (16 * odd)) & 0xffffu) ^ col);                                                       \
    *reinterpret_cast<uint4*>(lds + to) = make_uint4(dequant<2, I>(x[0], two, s2, z2), dequant<2, I>(x[1], two, s2, z2),             \
                                                     dequant<2, I>(x[2], two, s2, z2), dequant<2, I>(x[3], two, s2, z2));            \
  }
      MIXKVQ_CHANNEL(0) MIXKVQ_CHANNEL(1) MIXKVQ_CHANNEL(2) MIXKVQ_CHANNEL(3)
      MIXKVQ_CHANNEL(4) MIXKVQ_CHANNEL(5) MIXKVQ_CHANNEL(6) MIXKVQ_CHANNEL(7)
#undef MIXKVQ_CHANNEL
    }
  }
}

// The other tiers, whose channels stand in the record's list (an unused entry, 255, goes to the row that nobody reads): threads
// 256 .. 511.  REST: and what binary16 drops of the 4-bit tier into `rest` (a row per list entry).
template <bool REST>
__device__ __forceinline__ void unpack_side_keys(unsigned char* lds, int keys, int rest, int n_tok) {
  ArgsIn& a = args_here();
  const int Rr = a.R, inv_r = a.inv_r, inv_gk = a.inv_gk, tid = tid_here() - 256;
  const unsigned wide[5] = {in_vgpr(CodeAt<4, 0>::kMask), in_vgpr(CodeAt<4, 1>::kMask), 0, 0, 0};
  const int k4 = a.k4, k16 = a.k16;
  for (int u = tid; u < a.W4 * 64; u += 256) {      // four bits: eight tokens of two even or odd channels of a word
    const int odd = u & 1, late = (u >> 1) & 1, tg = (u >> 2) & 15, w = u >> 6, t = tg * 8;
    if (t >= n_tok) continue;
    const int rec = t * inv_r >> 16, tin = t - rec * Rr, raw = kOffRaw + rec * a.rec_bytes;
    const int words = raw + a.off_k4 + (tin * a.W4 + w) * 4;
    const unsigned pick = odd ? 0x07060302u : 0x05040100u, twice = odd ? 0x03020302u : 0x01000100u;
    unsigned x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = __builtin_amdgcn_perm(*reinterpret_cast<const unsigned*>(lds + words + (2 * i + 1) * a.W4 * 4),
                                   *reinterpret_cast<const unsigned*>(lds + words + 2 * i * a.W4 * 4), pick) >> (8 * late);
    const int first = 8 * w + 4 * late;      // list entries first + 2 I + odd
    const unsigned* s = reinterpret_cast<const unsigned*>(lds + raw + a.off_k4_s + ((tin * inv_gk >> 16) * k4 + first) * 2);
    const unsigned* z = reinterpret_cast<const unsigned*>(lds + raw + a.off_k4_z + ((tin * inv_gk >> 16) * k4 + first) * 2);
    const unsigned char* list = lds + raw + a.off_idx + k16 + first + odd;
#define MIXKVQ_CHANNEL(I)                                                                                                  \
  {                                                                                                                        \
    const h2 s2 = as_h2(__builtin_amdgcn_perm(s[I], s[I], twice)), z2 = as_h2(__builtin_amdgcn_perm(z[I], z[I], twice));   \
    const int ch = list[2 * I] < kD ? list[2 * I] : kD;                                                                    \
    const int to = keys + ch * kRowBytes + ((tg ^ twist(ch)) << 4);                                                        \
    const uint4 k = make_uint4(dequant<4, I>(x[0], wide, s2, z2), dequant<4, I>(x[1], wide, s2, z2),                       \
                               dequant<4, I>(x[2], wide, s2, z2), dequant<4, I>(x[3], wide, s2, z2));                      \
    *reinterpret_cast<uint4*>(lds + to) = k;                                                                               \
    if constexpr (REST) {                                                                                                  \
      const int e = first + 2 * I + odd;                                                                                   \
      const bool used = ch < kD;                                                                                           \
      *reinterpret_cast<uint4*>(lds + rest + e * kRowBytes + ((tg ^ twist(e)) << 4)) =                                     \
          make_uint4(used ? dropped<I>(x[0], k.x, s2, z2) : 0, used ? dropped<I>(x[1], k.y, s2, z2) : 0,                   \
                     used ? dropped<I>(x[2], k.z, s2, z2) : 0, used ? dropped<I>(x[3], k.w, s2, z2) : 0);                  \
    }                                                                                                                      \
  }
    MIXKVQ_CHANNEL(0) MIXKVQ_CHANNEL(1)
#undef MIXKVQ_CHANNEL
  }
  for (int u = tid ^ 128; u < k16 * 8; u += 256) {      // fp16: eight tokens of two neighbouring entries
    const int tg = u & 15, e = (u >> 4) * 2, t = tg * 8;
    if (t >= n_tok) continue;
    const int rec = t * inv_r >> 16, tin = t - rec * Rr, raw = kOffRaw + rec * a.rec_bytes;
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

// Quarters from .. to - 1 of the staged tile's values into `values` (a row per channel), by 256 threads, a word of 16 tokens of one channel
// at a time.
// Places of tokens that the tile does not have become 0 (their weights are 0, and 0 times what the LDS held may be NaN).
__device__ __forceinline__ void unpack_values(unsigned char* lds, int values, int n_tok, int from, int to) {
  ArgsIn& a = args_here();
  const int tid = tid_here() & 255, ch = tid & (kD - 1), first = __builtin_amdgcn_readfirstlane(tid >> 7);
  const unsigned two[5] = {in_vgpr(CodeAt<2, 0>::kMask), in_vgpr(CodeAt<2, 1>::kMask), in_vgpr(CodeAt<2, 2>::kMask), in_vgpr(CodeAt<2, 3>::kMask), in_vgpr(CodeAt<2, 4>::kMask)};
  const int per = a.R >> 4;      // words of a record and channel
  const int vg = ch >> (7 - a.nvg_bits), row = values + ch * kRowBytes, tw = twist(ch);
#pragma unroll 2
  for (int k = from; k < to; ++k) {
    const int w = first + 2 * k;
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    int t0 = 16 * w, t1 = t0 + 8;
    if (t0 < n_tok) {
      const int rec = 16 * w * a.inv_r >> 16, in = w - rec * per;
      const unsigned x = *reinterpret_cast<const unsigned*>(lds + kOffRaw + rec * a.rec_bytes + a.off_v + (in * kD + ch) * 4);
      if (a.interleave) {
        t0 = rec * a.R + 64 * (in >> 2) + 8 * (in & 3);
        t1 = t0 + 32;
      }
      const unsigned char* s = lds + kOffScale + vg * kScaleRow * 2;
      const unsigned char* z = s + 8 * kScaleRow * 2;
      const uint4 s0 = *reinterpret_cast<const uint4*>(s + t0 * 2), z0 = *reinterpret_cast<const uint4*>(z + t0 * 2);
      const uint4 s1 = *reinterpret_cast<const uint4*>(s + t1 * 2), z1 = *reinterpret_cast<const uint4*>(z + t1 * 2);
      lo = make_uint4(dequant<2, 0>(x, two, as_h2(s0.x), as_h2(z0.x)), dequant<2, 1>(x, two, as_h2(s0.y), as_h2(z0.y)),
                      dequant<2, 2>(x, two, as_h2(s0.z), as_h2(z0.z)), dequant<2, 3>(x, two, as_h2(s0.w), as_h2(z0.w)));
      hi = make_uint4(dequant<2, 4>(x, two, as_h2(s1.x), as_h2(z1.x)), dequant<2, 5>(x, two, as_h2(s1.y), as_h2(z1.y)),
                      dequant<2, 6>(x, two, as_h2(s1.z), as_h2(z1.z)), dequant<2, 7>(x, two, as_h2(s1.w), as_h2(z1.w)));
    }
    *reinterpret_cast<uint4*>(lds + row + (((t0 >> 3) ^ tw) << 4)) = lo;
    *reinterpret_cast<uint4*>(lds + row + (((t1 >> 3) ^ tw) << 4)) = hi;
  }
}

template <bool REST, class Counts>
__global__ void __launch_bounds__(kChunkThreads, 2) chunk_attention_kernel(ChunkArgs a, Counts counts) {
  __shared__ __align__(256) unsigned char lds[kLdsBytes];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool bf16 = a.bf16 != 0;
  const ChunkPlace at = chunk_place(a, counts, blockIdx.x);
  const int g = a.g, Hkv = a.Hkv, b = at.b, j = at.j, p = at.p, n_rec = at.n_rec, n_fp16 = at.n_fp16;
  const int n_rows = at.n_new * g, rt = gridDim.y - 1 - blockIdx.y;      // the last tiles of rows see most tokens: first
  if (rt * kRows >= n_rows) return;
  __builtin_amdgcn_s_setreg(1 | 23 << 6, 1);           // MODE.FP16_OVFL: a dequantized value past 65504 stays there

  // ---- query rows of this wavefront ----
  const int row0 = rt * kRows + 32 * wave;
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
  st.m = kNoToken;
  st.l = 0.f;
  f16v sc[2];                                          // scores of this slice and of the next one, in turn
  h8 pw[2][2];                                         // weights of this slice and of the one before, in turn
  const float c = a.scale * 1.4426950408889634f;      // scores in log2 units
  const int see_min = row0 / g + 1;                   // chunk tokens seen by the first row

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
    typedef __attribute__((address_space(4))) const int32_t* scalar_ptr;      // (through the scalar cache: see chunk_few.h)
    auto tile_count = [&](int t) { const int left = n_rec - t * tile_rec; return left < tile_rec ? left : tile_rec; };
    auto record = [&](int blk) __attribute__((always_inline)) {
      ArgsIn& a = args_here();
      const scalar_ptr table = (scalar_ptr)(uintptr_t)(a.table + (size_t)b * a.NB);
      return (const unsigned char*)a.blocks + (a.table ? (size_t)table[blk] * Hkv + j : (size_t)p * a.NB + blk) * a.rec_bytes;
    };
    constexpr int kPieces = REST ? 2 : 3;
    uint4 raw[kPieces];      // this thread's 16-byte pieces of a tile on their way: pieces tid, tid + 512 .. of its records
    static_assert(kOffRest - kOffRaw == 2 * 16 * kChunkThreads, "two pieces to a thread where there are rests");
    static_assert(kMaxRec <= 3 * 16 * kChunkThreads && kChunkRecords == 4, "three pieces to a thread; record_of");
    int listed[2];     // wavefront w: entries of record w's list
    auto record_of = [](int i, int pieces) { return (i >= pieces) + (i >= 2 * pieces) + (i >= 3 * pieces); };
    auto fetch = [&](int t) __attribute__((always_inline)) {
      ArgsIn& a = args_here();
      const int cnt = tile_count(t), pieces = a.rec_bytes >> 4, tid = tid_here();
      const unsigned char* mine = record(t * tile_rec);      // wavefront w < cnt lists record w
      if (tile_rec == 1 || !a.table) {                       // one after the other
        const uint4* at = reinterpret_cast<const uint4*>(mine);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) raw[k] = at[tid + kChunkThreads * k < cnt * pieces ? tid + kChunkThreads * k : 0];
        mine += (wave < cnt ? wave : 0) * a.rec_bytes;
      } else {
        const unsigned char* from[kChunkRecords];
#pragma unroll
        for (int r = 0; r < kChunkRecords; ++r) from[r] = record(t * tile_rec + (r < cnt ? r : 0)) - r * a.rec_bytes;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {      // (pieces that the tile does not have: its first one once more)
          const int i = tid + kChunkThreads * k < cnt * pieces ? tid + kChunkThreads * k : 0;
          const unsigned char* at = i < pieces ? from[0] : i < 2 * pieces ? from[1] : i < 3 * pieces ? from[2] : from[3];
          raw[k] = *reinterpret_cast<const uint4*>(at + i * 16);
        }
        mine = record(t * tile_rec + (wave < cnt ? wave : 0));
      }
      const int ks = a.k4 + a.k16, lane = tid & 63;
      listed[0] = mine[a.off_idx + (lane < ks ? lane : 0)];
      listed[1] = mine[a.off_idx + (lane + 64 < ks ? lane + 64 : 0)];
    };
    // The planes of the keys, or of the values.
    auto stage = [&](int t, bool values) __attribute__((always_inline)) {
      ArgsIn& a = args_here();
      const int cnt = tile_count(t), nvg_bits = a.nvg_bits, pieces = a.rec_bytes >> 4, plane = a.R * 2 << nvg_bits, tid = tid_here();
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        const int i = tid + kChunkThreads * k, rec = record_of(i, pieces), po = (i - rec * pieces) << 4;
        if (i >= cnt * pieces || (po >= a.off_v) != values) continue;
        const int es = po - a.off_v_s, ez = po - a.off_v_z;
        const bool scale = es >= 0 && es < plane, zero = ez >= 0 && ez < plane;
        if (!scale && !zero) {
          *reinterpret_cast<uint4*>(lds + kOffRaw + rec * a.rec_bytes + po) = raw[k];
        } else {      // value scales (zero-points): [token][group] there, [group][token] here
          const int li = (scale ? es : ez) >> 1;
          if (nvg_bits == 0) {
            *reinterpret_cast<uint4*>(lds + kOffScale + ((scale ? 0 : 8 * kScaleRow) + rec * a.R + li) * 2) = raw[k];
            continue;
          }
          unsigned short* to = reinterpret_cast<unsigned short*>(lds + kOffScale) + (scale ? 0 : 8 * kScaleRow) + rec * a.R;
          const unsigned v[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
          if (nvg_bits == 2) {      // two tokens of four groups
#pragma unroll
            for (int vg = 0; vg < 4; ++vg)
              *reinterpret_cast<unsigned*>(to + vg * kScaleRow + (li >> 2)) = __builtin_amdgcn_perm(v[2 + (vg >> 1)], v[vg >> 1], vg & 1 ? 0x07060302u : 0x05040100u);
            continue;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int tok = (li + e) >> nvg_bits, vg = (li + e) & ((1 << nvg_bits) - 1);
            if (tok < a.R) to[vg * kScaleRow + tok] = (unsigned short)(v[e >> 1] >> (16 * (e & 1)));
          }
        }
      }
    };
    // Wavefront w lists record w's 2-bit channels: place -> row of the key tile (twisted), 128 for places without a channel.
    auto map_of = [&](int t) { return reinterpret_cast<unsigned short*>(lds + kOffMap) + (t & 1) * kChunkRecords * kD; };
    auto list_channels = [&](int t) __attribute__((always_inline)) {
      if (wave >= tile_count(t)) return;
      ArgsIn& a = args_here();
      const int ks = a.k4 + a.k16, lane = tid_here() & 63;
      volatile unsigned short* to = map_of(t) + wave * kD;      // (one wavefront's reads and writes of the LDS keep their order)
      to[lane] = 1;
      to[lane + 64] = 1;
      if (lane < ks && listed[0] < kD) to[listed[0]] = 0;
      if (lane + 64 < ks && listed[1] < kD) to[listed[1]] = 0;
      const unsigned long long low = __ballot(to[lane] != 0), high = __ballot(to[lane + 64] != 0), before = (1ull << lane) - 1;
      const int n_low = __popcll(low), n = n_low + __popcll(high);
      if (low >> lane & 1) to[__popcll(low & before)] = (unsigned short)(lane << 8 | twist(lane) << 4);
      if (high >> lane & 1) to[n_low + __popcll(high & before)] = (unsigned short)((lane + 64) << 8 | twist(lane + 64) << 4);
      for (int i = n + lane; i < kD; i += 64) to[i] = (unsigned short)(kD << 8);
    };

    auto tokens_of = [&](int t) { return tile_count(t) * a.R; };
    if constexpr (REST) {
      *reinterpret_cast<uint4*>(lds + kOffRest + tid * 16) = make_uint4(0, 0, 0, 0);      // (rows behind the list stay 0)
      if (tid < 72) *reinterpret_cast<_Float16*>(lds + kOffPick + tid * 2) = (_Float16)(tid / 8 == tid % 8 ? 1.f : 0.f);
      static_assert(2 * kRestBytes == 16 * kChunkThreads, "a piece to a thread");
    }
    fetch(t_first);
    list_channels(t_first);
    stage(t_first, false);
    stage(t_first, true);
    if (t_first + 1 < r_end) fetch(t_first + 1);
    __syncthreads();
    unsigned entries = REST ? list_entries(lds, tile_count(t_first)) : 0, entries_next = entries;      // of this tile's lists and the next one's
    if (wave < 4) unpack_low_keys(lds, 0, map_of(t_first), tokens_of(t_first));
    else unpack_side_keys<REST>(lds, 0, kOffRest, tokens_of(t_first));
    unpack_values(lds, kKeyBytes, tokens_of(t_first), wave < 4 ? 0 : 2, wave < 4 ? 2 : 4);
    __syncthreads();
    if (t_first + 1 < r_end) {
      stage(t_first + 1, false);
      list_channels(t_first + 1);
    }
    const int share = n_rows - rt * kRows > kRows / 2;      // quarters of the values that wavefronts 0 .. 3 unpack: none where the others have no rows
    Pipe<true> in;
    if (active) begin<REST>(lds, in, entries, tokens_of(t_first), tokens_of(t_first), c, sc[0], pw[1], st);
    for (int t = t_first; t < r_end; ++t) {
      const bool next = t + 1 < r_end, next2 = t + 2 < r_end;
      const int odd = t - t_first & 1, here = odd * kTileBytes, there = kTileBytes - here;
      const int rest_here = kOffRest + odd * kRestBytes, rest_there = kOffRest + kRestBytes - odd * kRestBytes;
      const int n_tok = tokens_of(t), n_next = next ? tokens_of(t + 1) : 0;
      __syncthreads();      // this tile's values are there, and the next one's keys are staged
      if (next) stage(t + 1, true);
      if (next2) fetch(t + 2);
      // The wavefronts of a SIMD (w and w + 4) unpack at different times: one's vector instructions run beside the other's matrix
      // instructions, which go first (669 and 681 us for 1000 tokens after 31000).
      if (next && wave < 4) unpack_low_keys(lds, there, map_of(t + 1), tokens_of(t + 1));
      if (REST && next) entries_next = list_entries(lds, tile_count(t + 1));
      if (active) {
        __builtin_amdgcn_s_setprio(1);
        step<0, REST>(lds, in, t == t_first ? 0 : here - there, rest_here - here, entries, sc[0], sc[1], pw[1], pw[0], 2 * 32 > n_tok, n_tok, c, st);
        step<1, REST>(lds, in, 0, rest_here - here, entries, sc[1], sc[0], pw[0], pw[1], 3 * 32 > n_tok, n_tok, c, st);
        __builtin_amdgcn_s_setprio(0);
      }
      if (next && wave >= 4) unpack_side_keys<REST>(lds, there, rest_there, tokens_of(t + 1));
      __syncthreads();      // the next tile's keys are there, and its values are staged
      if (next2) {
        stage(t + 2, false);
        list_channels(t + 2);
      }
      if (next && wave >= 4) unpack_values(lds, there + kKeyBytes, tokens_of(t + 1), share, 4);
      if (active) {         // (behind the last tile: scores of what the other tile's place holds, all of them hidden)
        __builtin_amdgcn_s_setprio(1);
        step<2, REST>(lds, in, there - here, rest_here - here, entries, sc[0], sc[1], pw[1], pw[0], 4 * 32 > n_tok, n_tok, c, st);
        step<3, REST>(lds, in, 0, rest_there - there, entries_next, sc[1], sc[0], pw[0], pw[1], 32 > n_next, n_next, c, st);
        __builtin_amdgcn_s_setprio(0);
      }
      if (next && wave < 4) unpack_values(lds, there + kKeyBytes, tokens_of(t + 1), 0, share);
      entries = entries_next;
    }
    if (active) finish(lds, in, pw[1], st);
    __syncthreads();
  }

  // ---- fp16 rows: the cache's (all of them are seen), then the chunk's (causal) ----
  const int f_first = t_first > nt_rec ? t_first : nt_rec;
  if (f_first < t_end) {
    const int prow = tid >> 4, piece = tid & 15;
    const int place = prow * kRowBytes + ((piece ^ twist(prow)) << 4);      // of this thread's first piece; the others 32 rows on
    uint4 held[4];                            // half of the next tile on its way: its keys, then its values
    auto fetch = [&](int t, bool keys) {
      const bool win = t < nt_rec + nt_win;
      const int first = (t - nt_rec - (win ? 0 : nt_win)) * kChunkTile, n = win ? n_fp16 : seen;
      const __half* from = win ? (keys ? a.res_k : a.res_v) + (size_t)p * a.RW * kD : (keys ? a.k : a.v) + (int64_t)b * a.kvs.b + (int64_t)j * a.kvs.h;
      const int step = win ? kD : (int)a.kvs.t;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int r = first + prow + 32 * i;
        r = r < n ? r : n - 1;      // places behind the last row hold that row once more: finite, and masked
        held[i] = *reinterpret_cast<const uint4*>(from + (int64_t)r * step + piece * 8);
      }
    };
    auto store = [&](int t, int at) {
      if (bf16 && t >= nt_rec + nt_win) {
#pragma unroll
        for (int i = 0; i < 4; ++i) held[i] = as_f16x8(held[i], true);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(lds + at + place + i * 32 * kRowBytes) = held[i];
    };
    fetch(f_first, true);
    store(f_first, 0);
    fetch(f_first, false);
    store(f_first, kKeyBytes);
    __syncthreads();
    Pipe<false> in;
    auto first_of = [&](int t) { return (t - nt_rec - (t < nt_rec + nt_win ? 0 : nt_win)) * kChunkTile; };
    // Tokens of the tile that a row sees, and those that all rows of the wavefront see.
    auto limit_of = [&](int t) { return (t < nt_rec + nt_win ? n_fp16 : token + 1) - first_of(t); };
    auto all_of = [&](int t) { return (t < nt_rec + nt_win ? n_fp16 : see_min) - first_of(t); };
    if (active) begin<false>(lds, in, 0u, all_of(f_first), limit_of(f_first), c, sc[0], pw[1], st);
    for (int t = f_first; t < t_end; ++t) {
      const bool next = t + 1 < t_end;
      const int here = (t - f_first & 1) * kTileBytes, there = kTileBytes - here;
      const int all = all_of(t), limit = limit_of(t);
      __syncthreads();      // this tile's values are there
      if (next) fetch(t + 1, true);
      if (active) {
        __builtin_amdgcn_s_setprio(1);
        step<0, false>(lds, in, t == f_first ? 0 : here - there, 0, 0u, sc[0], sc[1], pw[1], pw[0], 2 * 32 > all, limit, c, st);
        step<1, false>(lds, in, 0, 0, 0u, sc[1], sc[0], pw[0], pw[1], 3 * 32 > all, limit, c, st);
        __builtin_amdgcn_s_setprio(0);
      }
      if (next) {
        store(t + 1, there);
        fetch(t + 1, false);
      }
      __syncthreads();      // the next tile's keys are there
      if (active) {
        const int all_next = next ? all_of(t + 1) : 0, limit_next = next ? limit_of(t + 1) : 0;
        __builtin_amdgcn_s_setprio(1);
        step<2, false>(lds, in, there - here, 0, 0u, sc[0], sc[1], pw[1], pw[0], 4 * 32 > all, limit, c, st);
        step<3, false>(lds, in, 0, 0, 0u, sc[1], sc[0], pw[0], pw[1], 32 > all_next, limit_next, c, st);
        __builtin_amdgcn_s_setprio(0);
      }
      if (next) store(t + 1, there + kKeyBytes);
    }
    if (active) finish(lds, in, pw[1], st);
    __syncthreads();
  }

  // ---- results leave in whole rows, by way of LDS ----
  float* const meet = reinterpret_cast<float*>(lds);                       // [kRows][kOutRow]
  float2* const ml = reinterpret_cast<float2*>(lds + kRows * kOutRow * 4);    // [kRows]
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
    const float m = ml[r].x, sum = ml[r].y, *o = meet + r * kOutRow + chan;
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
  if constexpr (std::is_same<Counts, NoChunkCounts>::value) {
    at = chunk_place(a, counts, i * a.n_splits * a.Hkv + j);
  } else {
    if (counts.n_new[i] == 0) return;      // (no unit is its own; the one behind the launch's last has no place in the list)
    at = chunk_place(a, counts, counts.first[i] * a.Hkv + j);
  }
  const int g = a.g, n_rows = at.n_new * g, rr = blockIdx.x % per_pair * 16 + (threadIdx.x >> 4), chan = (threadIdx.x & 15) * 8;
  if (rr >= n_rows) return;
  const size_t first = ((size_t)at.first_block * a.row_tiles + rr / rows) * rows + rr % rows, step = (size_t)a.Hkv * a.row_tiles * rows;
  const float2* ml = reinterpret_cast<const float2*>(a.part + (size_t)blocks * rows * kD);
  float m = kNoToken, sum = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < at.n_splits; ++s) m = fmaxf(m, ml[first + s * step].x);
#pragma unroll 4
  for (int s = 0; s < at.n_splits; ++s) {
    const size_t slot = first + s * step;
    const float2 x = ml[slot];
    const float f = __builtin_amdgcn_exp2f(x.x - m);
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

// Rests of the 4-bit tier where a slice lies in one record, the list has at most 16 entries and records leave room for them.
static bool has_rest(const ChunkArgs& a) { return a.k4 > 0 && a.k4 <= kRestRows && a.R % 32 == 0 && a.tile_rec * a.rec_bytes <= kOffRest - kOffRaw; }

static hipError_t start_tiles(const ChunkArgs& a, const ChunkCounts* c, int units, hipStream_t s) {
  const dim3 grid(units * a.Hkv, a.row_tiles);
  const bool rest = has_rest(a);
  if (c && rest) chunk_attention_kernel<true, ChunkCounts><<<grid, kChunkThreads, 0, s>>>(a, *c);
  else if (c) chunk_attention_kernel<false, ChunkCounts><<<grid, kChunkThreads, 0, s>>>(a, *c);
  else if (rest) chunk_attention_kernel<true, NoChunkCounts><<<grid, kChunkThreads, 0, s>>>(a, NoChunkCounts{});
  else chunk_attention_kernel<false, NoChunkCounts><<<grid, kChunkThreads, 0, s>>>(a, NoChunkCounts{});
  return hipGetLastError();
}

hipError_t launch_chunk(const ChunkArgs& a, const ChunkCounts* c, int units, int n_seq, bool few, int rows, hipStream_t s) {
  const hipError_t e = !few ? start_tiles(a, c, units, s) : rows == 16 ? start_chunk_few_1(a, c, units, s) : rows == 32 ? start_chunk_few_2(a, c, units, s)
                                                                                                           : start_chunk_few_3(a, c, units, s);
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
