// Attention of the last few tokens of every sequence to a cache of pages, with a prefix that all sequences share.
//
// Mathematics.  A row is one query (sequence, query head, token).  The keys of a row are cut into parts: pieces of the shared
// prefix and pieces of the sequence's own keys.  A part leaves  ref, l = sum exp2(x - ref), acc = sum exp2(x - ref) v  with
// x = log2(e) / sqrt(d) q.k; parts join by
//   O = sum_i 2^(ref_i - R) acc_i / sum_i 2^(ref_i - R) l_i,   lse = ln 2 (R + log2 of that sum),   R = max ref_i.
//
// Tiles.  The rows that read the same keys are the columns of the products S^T = K Q^T and O^T = V^T P^T on
// v_mfma_f32_16x16x32_bf16, 16 to a tile: for a sequence's own keys the heads of a group times its new tokens, for the prefix
// those of all sequences, so that a prefix key is read once for up to 64 of them.  A step is 32 keys:
//   K: lane (m, g) = (lane % 16, lane / 16) loads 16 bytes of key row m of a 16-key tile: an A operand as it is.
//   V: lane (m, g) loads channels 8 m .. 8 m + 7 of 8 keys, 4 whole rows of 256 bytes per instruction.  Turning the lane's
//      8 x 8 square (v_perm, 32 instructions per step) gives the A operand of 8 products, number c of which has channel
//      8 m + c in row m.
//   The key of a tile that K's row 4 g + r holds is 4 r + g, so the score that lane (n, g) gets in register r of tile t
//   belongs to the same key, 16 t + 4 r + g, that it loads of V as number 4 t + r: the probabilities are the B operand as they
//   are.  No exchange between lanes in the loop.
// The 4 waves of a workgroup take every fourth step of its keys and join at the end through LDS.
//
// What bounds it.  A sequence's own keys: HBM, each key is read once.  8 KV heads, 4 queries each: 64 sequences of 0 .. 8000
// keys (1.05 GB) 191 us, 5.5 TB/s; 4 of 65000 .. 131072 (1.53 GB) 250 us, 6.1 TB/s, where a copy of 1 GB runs at 5.1; then 7 - 10 us
// for the join.  One sequence of 531 keys: 11 us, latency from the launch to the last of five turns.
// The prefix: the instructions of a wave, and its loads beside them.  128 sequences x 4 queries behind 32749 keys (8 KV heads, 69
// GFLOP) 83 us, 830 TFLOP/s, and the prefix is fetched once for all rows (136 MB).  32 keys for 64 rows are 64 matrix, 175 vector and 60
// scalar instructions, 16 loads and 8 reads from LDS: 1.1 us, of which 0.8 are left without the loads and reads; 11 us are the launch, the
// first loads and the join of the waves.  (8-bit pages: half the loads and 64 conversions more, 1.15 us.)  Two such waves per SIMD with 32
// rows each took 36 % longer.
#include "cache.h"

namespace sale {

namespace {

// Exponents are taken relative to ref = maximum + kRoom, so that the sum of a long row times the largest bf16 value still is
// a float: the probabilities are at most 2^-24 .. 2^-17 and as precise as others (both types of the sums have 8 exponent bits).
// ref follows a maximum only when it has risen by more than kSlack: the accumulators are scaled once or twice per row.
constexpr float kRoom = 24.0f, kSlack = 7.0f;
constexpr float kNoRef = -3.0e38f;      // of a row that has seen no key
constexpr float kLog2eByRootD = 0.08838834764831845f * 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

constexpr int kWaves = 4, kStep = 32, kTurn = kWaves * kStep;      // keys per turn of a workgroup

struct DecodeArgs {
  CacheView c;
  const uint16_t* q;
  uint16_t* o;
  float* lse;
  Strided sq, so;
  const int32_t* prefix_table;
  int prefix_len, n_seqs, n_new, group, n_kvh;
  int shares;                                   // workgroups per KV head for the own keys
  int prefix_parts, prefix_chunk, row_tiles;    // parts of the prefix, keys of each; tiles of 16 * (row tiles of the kernel) rows
  // Partial results, by slot: accumulators [8][4 (g)][row], sums [row].  Own keys: share j of sequence s in slot j + s of the KV
  // head's (from one piece to the next j or s or both go up by one); prefix: [tile][KV head][part].
  f32x4 *own_acc, *pre_acc;
  float2 *own_sum, *pre_sum;
  int2* turns;                                  // [KV head][sequence] first turn of a sequence that has one, and those of all
};

// Channels of a lane's Q operand of contraction step s: those that its K operand has.
template <bool FP8>
__device__ __forceinline__ int step_channel(int s, int g) { return FP8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g; }

// Four values of E4M3 -> bf16 pairs (exact).
__device__ __forceinline__ uint32_t bf16_pair(uint32_t w, bool high) {
  return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)
                                           : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
}

// Operands of a step as loaded.
template <bool FP8>
struct Operands {
  u32x4 k[2][FP8 ? 2 : 4];
  std::conditional_t<FP8, u32x2, u32x4> v[8];
};

// The keys that a workgroup reads.
struct Keys {
  const int32_t* table;
  int n;              // positions 0 .. n - 1 hold keys (where there is a page) ..
  int all;            // .. and from here on, not all rows see them:
  int before;         // those of new token i see keys below before + i + 1 (the prefix: all of them do)
};

template <bool FP8, int NT>
struct Rows {
  bf16x8 q[NT][4];
  int token[NT];      // new token of row lane % 16 of tile qt
  f32x4 acc[NT][8];   // channels 32 g + 8 r + c (register r of number c) of row n
  float ref[NT], l[NT];
};

// An entry of a table at an index that is the same in all lanes.  Through the constant address space, for which the compiler
// takes a scalar load: a vector load would have to wait for the keys that were requested before it.
__device__ __forceinline__ int entry_at(const int32_t* table, int i) {
  return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)table)[i];
}

// Pages of the two 16-key tiles of the step at key0 (of its last one that exists where it lies behind it); -1: no page.
struct TwoPages { int a, b; };
__device__ __forceinline__ TwoPages pages_of(const CacheView& c, const Keys& ks, int key0) {
  const int last = (ks.n - 1) & ~15;
  const int a = entry_at(ks.table, min(key0, last) >> c.page_shift), b = entry_at(ks.table, min(key0 + 16, last) >> c.page_shift);
  return {(unsigned)a < (unsigned)c.n_pages ? a : -1, (unsigned)b < (unsigned)c.n_pages ? b : -1};
}

// Token slots slot .. slot + 15 of a page of one KV head, as a buffer: a load's address is then a scalar base, a lane's offset that
// stays and a scalar or constant one, without a vector instruction.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t slots_of(const PageSide& side, const uint8_t* head, int page, int slot) {
  return operand_buffer(head + (uint64_t)(uint32_t)page * side.page + (uint32_t)slot * side.token, 0x7FFFFFF0);
}
// Offsets of a lane: of the key row and channels that it loads of K, and of V.
struct LaneOffsets { int k, v; };
template <bool FP8>
__device__ __forceinline__ LaneOffsets lane_offsets(const CacheView& c, int lane) {
  const int m = lane & 15, g = lane >> 4;
  return {(int)((4 * (m & 3) + (m >> 2)) * c.k.token) + 16 * g, (int)(g * c.v.token) + (FP8 ? 8 : 16) * m};
}
template <bool FP8>
__device__ __forceinline__ void load_k(Operands<FP8>& x, int t, int s, __amdgpu_buffer_rsrc_t from, int lane_offset, int at = 0) {
  x.k[t][s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, lane_offset + 64 * s, at, 0));
}
template <bool FP8>
__device__ __forceinline__ void load_v(Operands<FP8>& x, int j, __amdgpu_buffer_rsrc_t from, int lane_offset, int at) {
  if constexpr (FP8) x.v[j] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(from, lane_offset, at, 0));
  else x.v[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, lane_offset, at, 0));
}

template <bool FP8>
__device__ __forceinline__ void load_step(const CacheView& c, const Keys& ks, int kvh, int key0, TwoPages pg, LaneOffsets at, Operands<FP8>& x) {
  const int last = (ks.n - 1) & ~15, mask = (1 << c.page_shift) - 1;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int page = max(t == 0 ? pg.a : pg.b, 0);      // (without a page: any one, whose keys are not used)
    const int slot = min(key0 + 16 * t, last) & mask;
    const __amdgpu_buffer_rsrc_t k = slots_of(c.k, c.k.base + (long long)kvh * c.k.head, page, slot);
    const __amdgpu_buffer_rsrc_t v = slots_of(c.v, c.v.base + (long long)kvh * c.v.head, page, slot);
#pragma unroll
    for (int s = 0; s < (FP8 ? 2 : 4); ++s) load_k<FP8>(x, t, s, k, at.k);
#pragma unroll
    for (int r = 0; r < 4; ++r) load_v<FP8>(x, 4 * t + r, v, at.v, 4 * r * c.v.token);
  }
}

// A operand c of the second product: channel 8 m + c of the lane's 8 keys.  (Of 8-bit values, w is what 2 channels, c rounded
// down to even and the next, are in bf16.)
template <bool FP8>
__device__ __forceinline__ bf16x8 turned(const Operands<FP8>& x, int c) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t lo, hi;
    if constexpr (FP8) {
      lo = bf16_pair(x.v[2 * i][c >> 2], (c >> 1 & 1) != 0);
      hi = bf16_pair(x.v[2 * i + 1][c >> 2], (c >> 1 & 1) != 0);
    } else {
      lo = x.v[2 * i][c >> 1];
      hi = x.v[2 * i + 1][c >> 1];
    }
    w[i] = __builtin_amdgcn_perm(hi, lo, c & 1 ? 0x07060302u : 0x05040100u);
  }
  return __builtin_bit_cast(bf16x8, w);
}

// Whether one of the two (E4M3: four) values of a word is an infinity or a NaN.
template <bool FP8>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  if constexpr (FP8) return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;      // (E4M3: 0x7F alone, a NaN)
  else return (((w & 0x7F800000u) + 0x00800000u) | ((w << 16 & 0x7F800000u) + 0x00800000u)) & 0x80000000u;
}

// O += V p of one key, for the rows that see it.  (Rare, see step: V comes from the page again.)
template <bool FP8, int NT, bool FINE>
__device__ __forceinline__ void one_key(const CacheView& c, Rows<FP8, NT>& rows, const bf16x8 (&p)[NT], const bf16x8 (&rest)[FINE ? NT : 1],
                                        const Keys& ks, int kvh, int key, int key0, TwoPages pg, int g) {
  const int in = key - key0, page = in < 16 ? pg.a : pg.b;
  if (page < 0) return;
  const uint8_t* v = c.v.base + (long long)page * c.v.page + (long long)kvh * c.v.head +
                     (long long)(key & ((1 << c.page_shift) - 1)) * c.v.token + 32 * g * (FP8 ? 1 : 2);
  float pk[NT];      // the key's probability is in lane group key % 4
#pragma unroll
  for (int qt = 0; qt < NT; ++qt) {
    float x = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j == in >> 2) x = FINE ? (float)p[qt][j] + (float)rest[FINE ? qt : 0][j] : (float)p[qt][j];
    pk[qt] = __shfl(x, (int)(threadIdx.x & 15) + 16 * (in & 3), 64);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const std::conditional_t<FP8, u32x2, u32x4> w = ((const std::conditional_t<FP8, u32x2, u32x4>*)v)[r];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x;
      if constexpr (FP8) x = __builtin_bit_cast(float, e & 1 ? bf16_pair(w[e >> 2], (e & 2) != 0) & 0xFFFF0000u : bf16_pair(w[e >> 2], (e & 2) != 0) << 16);
      else x = __builtin_bit_cast(float, e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
#pragma unroll
      for (int qt = 0; qt < NT; ++qt)
        if (key <= ks.before + rows.token[qt]) rows.acc[qt][e][r] = __builtin_fmaf(pk[qt], x, rows.acc[qt][e][r]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// One step: its 32 keys enter acc, l and ref.  edge: some of the keys are not there, or not for all rows.  FINE: the probabilities
// enter as two bf16 each, the leading bits and the rest: where reading the keys is what takes the time, the second product and
// its operands cost nothing that shows, and O is then off by its own rounding alone.  (Where the registers suffice: not for the
// own keys of 17 rows and more, nor for 64 rows of the prefix, where the matrix unit is what takes the time.  O then is off by the
// rounding of the probabilities too: 0.0022 - 0.0023 where it is 0.0017 otherwise.)
template <bool FP8, int NT, bool FINE>
__device__ __forceinline__ void step(const CacheView& c, Operands<FP8>& x, Rows<FP8, NT>& rows, float scale, const Keys& ks, int kvh,
                                     int key0, TwoPages pg, bool edge, int g, int n_new) {
  f32x4 S[2][NT];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      bf16x8 k;
      if constexpr (FP8) {
        const u32x4 w = x.k[t][s >> 1];
        const int h = 2 * (s & 1);
        k = __builtin_bit_cast(bf16x8, u32x4{bf16_pair(w[h], false), bf16_pair(w[h], true), bf16_pair(w[h + 1], false), bf16_pair(w[h + 1], true)});
      } else {
        k = __builtin_bit_cast(bf16x8, x.k[t][s]);
      }
#pragma unroll
      for (int qt = 0; qt < NT; ++qt)
        S[t][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, rows.q[qt][s], s == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : S[t][qt], 0, 0, 0);
    }
  if (edge) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int key = key0 + 16 * (j >> 2) + 4 * (j & 3) + g;
      const bool page = (j < 4 ? pg.a : pg.b) >= 0;
#pragma unroll
      for (int qt = 0; qt < NT; ++qt)
        if (!page || key >= min(ks.before + rows.token[qt] + 1, ks.n)) S[j >> 2][qt][j & 3] = -INFINITY;
    }
  }
  bf16x8 p[NT], rest[FINE ? NT : 1];
#pragma unroll
  for (int qt = 0; qt < NT; ++qt) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = S[j >> 2][qt][j & 3] * scale;
    float top = v[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, v[j]);
    if (__builtin_amdgcn_ballot_w64(top > rows.ref[qt] - kRoom + kSlack) != 0) {
      top = max_over_rows(top);
      if (top > rows.ref[qt] - kRoom + kSlack) {
        const float to = top + kRoom, by = __builtin_amdgcn_exp2f(rows.ref[qt] - to);
        rows.ref[qt] = to;
        rows.l[qt] *= by;
#pragma unroll
        for (int e = 0; e < 8; ++e) rows.acc[qt][e] *= by;
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = __builtin_amdgcn_exp2f(v[j] - rows.ref[qt]);
      rows.l[qt] += v[j];
    }
    if constexpr (FINE) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, v[2 * i + 1]), __builtin_bit_cast(uint32_t, v[2 * i]), 0x07060302u);
      p[qt] = __builtin_bit_cast(bf16x8, w);
      // (never 0 or negative beside a p that is not 0: an infinity of V stays what it is)
#pragma unroll
      for (int j = 0; j < 8; ++j) rest[qt][j] = (__bf16)__builtin_fmaf((float)p[qt][j], 0x1p-20f, v[j] - (float)p[qt][j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) p[qt][j] = (__bf16)v[j];
    }
  }
  if (edge) {
    // What is not a key is zero.  Among the new tokens' keys, which only some rows see, an infinity or a NaN (zero times these
    // is NaN) has to be kept from the others: then these keys are taken one by one, for the rows that see them.
    uint32_t inf = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int key = key0 + 16 * (j >> 2) + 4 * (j & 3) + g;
      const bool there = key < ks.n && (j < 4 ? pg.a : pg.b) >= 0;
#pragma unroll
      for (int e = 0; e < (FP8 ? 2 : 4); ++e) {
        if (!there) x.v[j][e] = 0;
        if (key >= ks.all) inf |= not_finite<FP8>(x.v[j][e]);
      }
    }
    if (n_new > 1 && __builtin_amdgcn_ballot_w64(inf != 0) != 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < (FP8 ? 2 : 4); ++e)
          if (key0 + 16 * (j >> 2) + 4 * (j & 3) + g >= ks.all) x.v[j][e] = 0;
      for (int key = max(ks.all, key0); key < min(ks.n, key0 + kStep); ++key) one_key<FP8, NT, FINE>(c, rows, p, rest, ks, kvh, key, key0, pg, g);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bf16x8 v = turned<FP8>(x, e);
#pragma unroll
    for (int qt = 0; qt < NT; ++qt) {
      rows.acc[qt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[qt], rows.acc[qt][e], 0, 0, 0);
      if constexpr (FINE) rows.acc[qt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, rest[qt], rows.acc[qt][e], 0, 0, 0);
    }
  }
}

// Keys from .. hi - 1 for the rows, 32 of every kTurn.
template <bool FP8, int NT, bool FINE>
__device__ __forceinline__ void sweep(const CacheView& c, const Keys& ks, int kvh, int from, int hi, int lane, int n_new, float scale,
                                      Rows<FP8, NT>& rows) {
  const LaneOffsets at = lane_offsets<FP8>(c, lane);
  for (int key0 = from; key0 < hi; key0 += kTurn) {
    const TwoPages pg = pages_of(c, ks, key0);
    Operands<FP8> x;
    load_step<FP8>(c, ks, kvh, key0, pg, at, x);
    step<FP8, NT, FINE>(c, x, rows, scale, ks, kvh, key0, pg, key0 + kStep > ks.all || (pg.a | pg.b) < 0, lane >> 4, n_new);
  }
}

// The same for 64 rows and `steps` steps, an even number, of which every key is there for every row, key0, key0 + kTurn, ..: a
// software pipeline.
// Phase t
//   S(t + 1) = K(t + 1) Q^T     MFMA
//   O += V(t - 1)^T P(t - 1)^T  MFMA
//   P(t) = exp2(S(t) - ref)     VALU, its sums, the turning of V(t - 1) and the largest of the scores S(t + 1)
//   K(t + 3) to LDS, K(t + 2) from there and V(t + 1) into the registers that were just read (8-bit: K(t + 3) too)
// has no dependency between its streams; they are laid side by side by hand, an MFMA and its share of the rest at a time, for a
// wave is alone on its SIMD (64 rows: 128 accumulators, 64 registers of Q, 64 of S, 96 of K and V).
//
// K of bf16 goes through LDS, straight from memory and each wave's for itself: the operand of 16 lanes is 16 bytes of each of 16 keys,
// and a load from memory that touches 16 lines for 16 lanes keeps the CU's one load path busy four times as long as one of whole
// keys.  A load brings 1 KB of neighbouring keys; in LDS a key is a row, in which chunk c of 16 bytes lies at place c ^ m, m the row of
// the operand that the key becomes.  (128 sequences behind 32749 keys: operands straight from memory 100 us, this way 83.  Keys of
// 8 bits are half the loads, and conversions take the time: 31.2 straight, 31.9 this way.)
struct KeyBuffer { u32x4 of[kWaves][512]; };      // the keys of a step of every wave
struct KeyBuffers { KeyBuffer even, odd; };
template <bool FP8, bool ONE, class Lds>
__device__ __forceinline__ void pipeline(const CacheView& c, const Keys& ks, int kvh, int key0, int steps, int lane, int wave, float scale,
                                         Lds& lds, Rows<FP8, 4>& rows) {
  constexpr int NT = 4, kQk = 8 * NT, kPv = 8 * NT, kElems = 8 * NT, kLoads = FP8 ? 2 : 4;
  const int mask = (1 << c.page_shift) - 1;
  const LaneOffsets lane_at = lane_offsets<FP8>(c, lane);
  const uint8_t *k_head = c.k.base + (long long)kvh * c.k.head, *v_head = c.v.base + (long long)kvh * c.v.head;
  // Where the 16-key tiles of step u are: their pages (one where a step lies in a page) and first slots
  auto key_of = [&](int u) { return key0 + kTurn * min(u, steps - 1); };
  auto ids_of = [&](int u) -> TwoPages {
    const int key = key_of(u), a = entry_at(ks.table, key >> c.page_shift);
    return {a, ONE ? a : entry_at(ks.table, (key + 16) >> c.page_shift)};
  };
  struct Tiles { __amdgpu_buffer_rsrc_t a, b; };      // (the same where a step lies in a page)
  const int k_second = ONE ? 16 * (int)c.k.token : 0, v_second = ONE ? 16 * (int)c.v.token : 0;      // offset of the second tile
  auto tiles_of = [&](const PageSide& side, const uint8_t* head, int u, TwoPages id) __attribute__((always_inline)) -> Tiles {
    const int slot = key_of(u) & mask;
    if constexpr (ONE) {
      const uint8_t* at = head + (uint64_t)(uint32_t)id.a * side.page + (uint32_t)slot * side.token;
      const __amdgpu_buffer_rsrc_t both = operand_buffer(at, 0x7FFFFFF0);
      return {both, both};
    } else {
      return {slots_of(side, head, id.a, slot), slots_of(side, head, id.b, (slot + 16) & mask)};
    }
  };
  Operands<FP8> x[2];      // V: [t % 2]; K: 8-bit likewise, bf16 the next one that is needed, in x[0]
  // bf16: a lane's offset in memory in load s of a 16-key tile, which brings keys 4 s .. 4 s + 3, and in LDS of operand s
  int to_lane[4], from_lane[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int m = lane & 15, g = lane >> 4, key = 4 * s + g;      // (key 4 s + g becomes row s + 4 g)
    to_lane[s] = key * (int)c.k.token + 16 * (m ^ (s + 4 * g));
    from_lane[s] = (4 * (m & 3) + (m >> 2)) * 16 + ((4 * s + g) ^ m);
  }
  auto get_k = [&](auto parity, const Tiles& from, int t, int s) __attribute__((always_inline)) {
    constexpr int p = decltype(parity)::value;
    if constexpr (FP8) load_k<FP8>(x[p], t, s, t == 0 ? from.a : from.b, lane_at.k, t * k_second);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(t == 0 ? from.a : from.b, (__attribute__((address_space(3))) void*)&(p ? lds.keys.odd : lds.keys.even).of[wave][256 * t + 64 * s],
                                                  16, to_lane[s], t * k_second, 0, 0);
  };
  auto read_k = [&](auto parity, int t, int s) __attribute__((always_inline)) {
    if constexpr (!FP8) x[0].k[t][s] = (decltype(parity)::value ? lds.keys.odd : lds.keys.even).of[wave][256 * t + from_lane[s]];
  };
  constexpr std::integral_constant<int, 0> in_even{};
  constexpr std::integral_constant<int, 1> in_odd{};
  // What was read from LDS has arrived: its place can be written again.
  auto arrived = [&]() __attribute__((always_inline)) {
    if constexpr (FP8) return;
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
  };
  // All loads but the last `newer` have arrived.  (The compiler takes a load to LDS for a write of 16 bytes, where it writes 1 KB, and
  // does not wait for all that a read from there needs.)
  auto loaded = [&](auto newer) __attribute__((always_inline)) {
    constexpr int n = decltype(newer)::value;
    if constexpr (FP8) return;      // (registers: the compiler's waits)
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((n & 15) | (n >> 4) << 14 | 0x0F70);      // vmcnt(n)
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr std::integral_constant<int, 8> k_newer{};       // newer than what is waited for: K of a step
  constexpr std::integral_constant<int, 16> kv_newer{};     // .., and V of one
  auto get_v = [&](Operands<FP8>& to, const Tiles& from, int j) __attribute__((always_inline)) { load_v<FP8>(to, j, j < 4 ? from.a : from.b, lane_at.v, 4 * (j & 3) * c.v.token + (j < 4 ? 0 : v_second)); };
  // O += V P with the accumulators in AGPRs, where the compiler would move them back and forth: S, P and V take most of the 256
  // ordinary registers.  The compiler does not see a matrix instruction here, so its waits are this code's to keep: 2 states from
  // what writes v, p or acc to the product (in a phase 3 other products are between, elsewhere s_nop 1), and from the product to
  // what else reads acc, settle.
  auto pv = [&](auto close, int qt, int e, const bf16x8& v, const bf16x8& p) __attribute__((always_inline)) {
    f32x4& acc = rows.acc[qt][e];
    if constexpr (decltype(close)::value) asm("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(v), "v"(p));
    else asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(v), "v"(p));
  };
  auto settle = [&]() __attribute__((always_inline)) {
    asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
    for (int qt = 0; qt < NT; ++qt)
#pragma unroll
      for (int e = 0; e < 8; ++e) asm volatile("" : "+a"(rows.acc[qt][e]));
  };
  f32x4 S[2][2][NT];
  bf16x8 P[2][NT];
  auto k_operand = [&](const Operands<FP8>& from, int t, int s) __attribute__((always_inline)) -> bf16x8 {
    if constexpr (FP8) {
      const u32x4 w = from.k[t][s >> 1];
      const int h = 2 * (s & 1);
      return __builtin_bit_cast(bf16x8, u32x4{bf16_pair(w[h], false), bf16_pair(w[h], true), bf16_pair(w[h + 1], false), bf16_pair(w[h + 1], true)});
    } else {
      return __builtin_bit_cast(bf16x8, from.k[t][s]);
    }
  };
  // The rows' references follow the scores S[y]; what P holds is still to be added at the old ones: it is scaled like acc.  (ref
  // is a whole number here, so that is exact.)
  auto raise = [&](int y, bf16x8 (&pending)[NT]) __attribute__((always_inline)) {
    settle();
#pragma unroll
    for (int qt = 0; qt < NT; ++qt) {
      float top = S[y][0][qt][0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = fmaxf(top, S[y][j >> 2][qt][j & 3]);
      top = max_over_rows(top) * scale;
      if (top > rows.ref[qt] - kRoom + kSlack) {
        const float to = __builtin_ceilf(top) + kRoom, by = __builtin_amdgcn_exp2f(rows.ref[qt] - to);
        rows.ref[qt] = to;
        rows.l[qt] *= by;
#pragma unroll
        for (int e = 0; e < 8; ++e) { rows.acc[qt][e] *= by; pending[qt][e] = (__bf16)((float)pending[qt][e] * by); }
      }
    }
  };
  TwoPages id1 = ids_of(1), id2 = ids_of(2), id3 = ids_of(3);
  auto get_all_k = [&](auto parity, int u, TwoPages id) __attribute__((always_inline)) {
    const Tiles from = tiles_of(c.k, k_head, u, id);
#pragma unroll
    for (int n = 0; n < 2 * kLoads; ++n) get_k(parity, from, n / kLoads, n % kLoads);
  };
  auto read_all_k = [&](auto parity) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < 8; ++n) read_k(parity, n / 4, n % 4);
  };
  const TwoPages id0 = ids_of(0);
  get_all_k(in_even, 0, id0);
  get_all_k(in_odd, 1, id1);
  loaded(k_newer);
  read_all_k(in_even);
#pragma unroll
  for (int n = 0; n < kQk; ++n) {
    const int t = n / 16, s = n / 4 % 4, qt = n % 4;
    S[0][t][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k_operand(x[0], t, s), rows.q[qt][s], s == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : S[0][t][qt], 0, 0, 0);
  }
  arrived();
  get_all_k(in_even, 2, id2);
  {
    const Tiles from = tiles_of(c.v, v_head, 0, id0);
#pragma unroll
    for (int j = 0; j < 8; ++j) get_v(x[0], from, j);
  }
  loaded(kv_newer);
  read_all_k(in_odd);
#pragma unroll
  for (int qt = 0; qt < NT; ++qt)
#pragma unroll
    for (int e = 0; e < 8; ++e) P[1][qt][e] = (__bf16)0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[1].v[j] = 0;
  raise(0, P[1]);
  auto phase = [&](auto xc, int t) __attribute__((always_inline)) {
    constexpr int cur = decltype(xc)::value, oth = 1 - cur;
    constexpr std::integral_constant<int, cur> in_cur{};
    constexpr std::integral_constant<int, oth> in_oth{};
    arrived();
    const Tiles k_next = tiles_of(c.k, k_head, t + 3, id3), v_next = tiles_of(c.v, v_head, t + 1, id1);
    id1 = id2; id2 = id3; id3 = ids_of(t + 4);
    float E[kElems], top[NT];
    // The VALU stream, four places per score: scale k, exp2 k - 1, sum k - 2, pack the pair that ends with k - 2; then four per
    // row tile for the maxima of the next scores
    constexpr int exps = (kElems + 2) * 4, slots = exps + 4 * NT;
    auto valu = [&](int n) __attribute__((always_inline)) {
      if (n < exps) {
        const int k = n / 4, o = n % 4, e = o == 0 ? k : o == 1 ? k - 1 : k - 2;
        if (e < 0 || e >= kElems) return;
        const int qt = e / 8, j = e % 8;
        if (o == 0) E[e] = __builtin_fmaf(S[cur][j >> 2][qt][j & 3], scale, -rows.ref[qt]);
        else if (o == 1) E[e] = __builtin_amdgcn_exp2f(E[e]);
        else if (o == 2) rows.l[qt] += E[e];
        else if (e & 1) { P[cur][qt][j - 1] = (__bf16)E[e - 1]; P[cur][qt][j] = (__bf16)E[e]; }
      } else {
        const int qt = (n - exps) % NT, o = (n - exps) / NT;
        const f32x4 &a = S[oth][0][qt], &b = S[oth][1][qt];
        auto max3 = [](float p, float q, float r) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(p, q), r); };
        if (o == 0) top[qt] = max3(a[0], a[1], a[2]);
        else if (o == 1) top[qt] = max3(top[qt], a[3], b[0]);
        else if (o == 2) top[qt] = max3(top[qt], b[1], b[2]);
        else top[qt] = __builtin_elementwise_maximum(top[qt], b[3]);
      }
    };
    bf16x8 k, v[2];
    static_for<kQk + kPv>([&](auto ic) __attribute__((always_inline)) {
      constexpr int i = decltype(ic)::value;
      if constexpr (i < kQk) {
        constexpr int t2 = i / 16, s = i / 4 % 4, qt = i % 4;
        if constexpr (qt == 0) k = k_operand(x[FP8 ? oth : 0], t2, s);
        S[oth][t2][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, rows.q[qt][s], s == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : S[oth][t2][qt], 0, 0, 0);
        if constexpr (qt == 1 && !FP8) get_k(in_oth, k_next, t2, s);
        if constexpr (qt == 1 && FP8 && s % 2 == 1) get_k(in_oth, k_next, t2, s / 2);
        if constexpr (i == kQk - 4) v[0] = turned<FP8>(x[oth], 0);
      } else {
        constexpr int e = (i - kQk) / 4, qt = i % 4;
        pv(std::false_type{}, qt, e, v[e % 2], P[oth][qt]);
        if constexpr (qt == 0 && e < 7) v[(e + 1) % 2] = turned<FP8>(x[oth], e + 1);
        if constexpr (i == kQk) loaded(kv_newer);
        if constexpr (qt == 1) read_k(in_cur, e / 4, e % 4);
        if constexpr (e >= 6) get_v(x[oth], v_next, 4 * (e - 6) + qt);
      }
      constexpr int from = i * slots / (kQk + kPv), to = (i + 1) * slots / (kQk + kPv);
      static_for<to - from>([&](auto vc) __attribute__((always_inline)) { valu(from + decltype(vc)::value); });
      __builtin_amdgcn_sched_barrier(0);
    });
    uint64_t rose = 0;
#pragma unroll
    for (int qt = 0; qt < NT; ++qt) rose |= __builtin_amdgcn_ballot_w64(top[qt] * scale > rows.ref[qt] - kRoom + kSlack);
    if (__builtin_expect_with_probability(rose != 0 && t + 1 < steps, 0, 0.99)) raise(oth, P[cur]);
  };
  for (int t = 0; t < steps; t += 2) {
    phase(std::integral_constant<int, 0>{}, t);
    phase(std::integral_constant<int, 1>{}, t + 1);
  }
  settle();
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bf16x8 v = turned<FP8>(x[1], e);
#pragma unroll
    for (int qt = 0; qt < NT; ++qt) pv(std::true_type{}, qt, e, v, P[1][qt]);
  }
  settle();
  loaded(std::integral_constant<int, 0>{});      // (what was requested beyond the end arrives while the workgroup is there)
}

// The sum over the four lanes that are equal modulo 16.
__device__ __forceinline__ float sum_over_rows(float v) {
  float w = v;
  asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(v), "+v"(w));
  w = v = v + w;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(v), "+v"(w));
  return v + w;
}

// The results of the four waves, joined.  keep(qt, c, x, l): x = accumulator c of this lane in tile qt, l the sum of its row, for
// two numbers c per wave; sums(row, ref, l).
struct JoinLds {
  f32x4 acc[kWaves][8][64];
  float ref[kWaves][64], l[kWaves][64];
};
template <bool FP8, int NT, class Keep, class Sums>
__device__ __forceinline__ void join_waves(Rows<FP8, NT>& rows, JoinLds& lds, int wave, int lane, Keep keep, Sums sums) {
  const int n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int qt = 0; qt < NT; ++qt) {
    rows.l[qt] = sum_over_rows(rows.l[qt]);
    if (g == 0) { lds.ref[wave][16 * qt + n] = rows.ref[qt]; lds.l[wave][16 * qt + n] = rows.l[qt]; }
  }
  __syncthreads();
#pragma unroll
  for (int qt = 0; qt < NT; ++qt) {
    const int row = 16 * qt + n;
    float top = lds.ref[0][row];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds.ref[w][row]);
    const float by = __builtin_amdgcn_exp2f(rows.ref[qt] - top);
#pragma unroll
    for (int c = 0; c < 8; ++c) lds.acc[wave][c][lane] = rows.acc[qt][c] * by;
    float l = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) l += lds.l[w][row] * __builtin_amdgcn_exp2f(lds.ref[w][row] - top);
    if (wave == 0 && g == 0) sums(row, top, l);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int c = 2 * wave + e;
      f32x4 x = lds.acc[0][c][lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) x += lds.acc[w][c][lane];
      keep(qt, c, x, l);
    }
    if (qt + 1 < NT) __syncthreads();
  }
}

__device__ __forceinline__ float lse_of(float ref, float l) { return l == 0.0f ? -INFINITY : kLn2 * (ref + __builtin_amdgcn_logf(l)); }

// Row r of a sequence: its new token and the query head inside its group.
struct RowOf { int token, head; };
__device__ __forceinline__ RowOf row_of(int group, int r) { const int t = r / group; return {t, r - t * group}; }

__device__ __forceinline__ uint16_t* row_at(uint16_t* x, const Strided& l, int s, int head, int token) {
  return x + (size_t)s * (size_t)l.sb + (size_t)head * (size_t)l.sh + (size_t)token * (size_t)l.st;
}

template <bool FP8, int NT>
__device__ __forceinline__ void load_row(const uint16_t* q, const Strided& sq, int group, int kvh, int s, int r, int qt, int g,
                                         Rows<FP8, NT>& rows) {
  const RowOf w = row_of(group, r);
  const uint16_t* row = row_at(const_cast<uint16_t*>(q), sq, s, kvh * group + w.head, w.token);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    rows.q[qt][e] = *(const bf16x8*)(row + step_channel<FP8>(e, g));
    if constexpr (NT == 4) asm("" : "+a"(rows.q[qt][e]));      // (what only the matrix unit reads stays out of the ordinary registers)
  }
  rows.token[qt] = w.token;
  rows.ref[qt] = kNoRef;
  rows.l[qt] = 0.0f;
#pragma unroll
  for (int c = 0; c < 8; ++c) rows.acc[qt][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
}

// Sharing out the own keys.  A sequence has as many turns as workgroups need to read its keys, kTurn at a time; the turns of
// all sequences, one after the other, are dealt to the workgroups of a KV head in equal shares.
__device__ __forceinline__ int turns_of(const CacheView& c, int len) { return (min(max(len, 0), c.width << c.page_shift) + kTurn - 1) / kTurn; }
struct Share { long long first, count; };
__device__ __forceinline__ Share share_of(long long turns, int shares, int j) {
  const long long each = turns / shares, more = turns - each * shares;      // (the first `more` shares have one turn more)
  return {j * each + min((long long)j, more), each + (j < more ? 1 : 0)};
}
__device__ __forceinline__ int share_with(long long turns, int shares, long long turn) {
  const long long each = turns / shares, more = turns - each * shares, border = more * (each + 1);
  return (int)(turn < border ? turn / (each + 1) : more + (turn - border) / each);
}

// A workgroup: one share of the turns of a KV head, piece by piece (a piece: neighbouring turns of one sequence).  The only piece
// of a sequence, without a prefix, is its result.  WHOLE: workgroup j has all of sequence j, and there is nothing to join.
template <bool FP8, int NT, bool WHOLE>
__global__ __launch_bounds__(64 * kWaves, NT == 4 ? 1 : 2) void own_kernel(DecodeArgs a) {
  __shared__ JoinLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_rows = a.group * a.n_new;
  const int kvh = blockIdx.x % a.n_kvh, j = blockIdx.x / a.n_kvh;
  const float scale = FP8 ? kLog2eByRootD * a.c.k_scale[kvh] : kLog2eByRootD, v_scale = FP8 ? a.c.v_scale[kvh] : 1.0f;
  // Turns from .. from + count - 1 of sequence s; whole: they are all it has, and the result.
  auto piece = [&](int s, int from, int count, bool whole) __attribute__((always_inline)) {
    const int held = max(entry_at(a.c.lens, s), 0), n_keys = min(held, a.c.width << a.c.page_shift);
    const int lo = from * kTurn, hi = min((from + count) * kTurn, n_keys);
    const size_t slot = (size_t)kvh * (a.shares + a.n_seqs) + j + s;
    Rows<FP8, NT> rows;
    // (The addresses of the rows, and of the outputs below, are made here, from arguments that are read here: nothing of them stays
    // in registers from piece to piece or during the sweep.)
    int from_lane = lane;
    auto args = (const __attribute__((address_space(4))) DecodeArgs*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+v"(from_lane), "+s"(args));
    const Strided sq = {args->sq.sb, args->sq.sh, args->sq.st, args->sq.heads};
#pragma unroll
    for (int qt = 0; qt < NT; ++qt)
      load_row<FP8, NT>(args->q, sq, a.group, kvh, s, min(16 * qt + (from_lane & 15), n_rows - 1), qt, from_lane >> 4, rows);
    const Keys ks = {a.c.table + (size_t)s * a.c.width, n_keys, min(held - a.n_new + 1, n_keys), held - a.n_new};
    sweep<FP8, NT, NT == 1>(a.c, ks, kvh, lo + kStep * wave, hi, from_lane, a.n_new, scale, rows);
    int at_lane = from_lane;
    auto late = (const __attribute__((address_space(4))) DecodeArgs*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+v"(at_lane), "+s"(late));
    const int at_row = at_lane & 15, at_group = at_lane >> 4;
    const Strided so = {late->so.sb, late->so.sh, late->so.st, late->so.heads};
    join_waves<FP8, NT>(rows, lds, wave, at_lane,
      [&](int qt, int c, f32x4 x, float l) {
        const int r = 16 * qt + at_row;
        if (r >= n_rows) return;
        if (whole) {
          const RowOf w = row_of(a.group, r);
          uint16_t* out = row_at(late->o, so, s, kvh * a.group + w.head, w.token) + 32 * at_group + c;
          const float by = l == 0.0f ? 0.0f : v_scale / l;
#pragma unroll
          for (int e = 0; e < 4; ++e) out[8 * e] = __builtin_bit_cast(uint16_t, (__bf16)(l == 0.0f ? 0.0f : x[e] * by));
        } else {
          late->own_acc[((slot * 8 + c) * 4 + at_group) * n_rows + r] = x;
        }
      },
      [&](int r, float ref, float l) {
        if (r >= n_rows) return;
        if (whole) {
          const RowOf w = row_of(a.group, r);
          if (late->lse) late->lse[((size_t)s * so.heads + kvh * a.group + w.head) * a.n_new + w.token] = lse_of(ref, l);
        } else {
          late->own_sum[slot * n_rows + r] = make_float2(ref, l);
        }
      });
  };
  if (WHOLE) { piece(j, 0, turns_of(a.c, entry_at(a.c.lens, j)), true); return; }
  // lane i counts the turns of sequences i * per ..
  const int per = (a.n_seqs + 63) / 64;
  int mine = 0;
  for (int s = lane * per; s < min((lane + 1) * per, a.n_seqs); ++s) mine += turns_of(a.c, a.c.lens[s]);
  int upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) { const int x = __shfl_up(upto, d, 64); if (lane >= d) upto += x; }
  const int all = __builtin_amdgcn_readlane(upto, 63);
  const Share share = share_of(all, a.shares, j);
  if (share.count == 0) return;
  const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > share.first));
  int s = at * per, base = __builtin_amdgcn_readlane(upto - mine, at), left = (int)share.count;      // base: first turn of sequence s
  int turn = (int)share.first;
  for (; left > 0; ++s) {
    const int turns = turns_of(a.c, entry_at(a.c.lens, s)), from = turn - base, count = min(turns - from, left);
    if (count > 0) {
      if (from == 0 && tid == 0) a.turns[(size_t)kvh * a.n_seqs + s] = make_int2(base, all);
      piece(s, from, count, count == turns && a.prefix_len == 0);
      left -= count;
      turn += count;
    }
    base += turns;
  }
}

// A workgroup: one part of the prefix, for 16 NT rows of one KV head, of whichever sequences.
// (All LDS of the kernel is one object, of which the keys come first: a load's place there is documented as a number of 16 bits.)
struct KeysAndJoin { KeyBuffers keys; JoinLds join; };
struct JoinAlone { JoinLds join; };
static_assert(sizeof(KeyBuffers) <= 65536, "the pipeline's keys lie below 64 KB of LDS");
template <bool FP8, int NT>
__global__ __launch_bounds__(64 * kWaves, NT == 4 ? 1 : 2) void prefix_kernel(DecodeArgs a) {
  __shared__ __attribute__((aligned(1024))) std::conditional_t<NT == 4 && !FP8, KeysAndJoin, JoinAlone> lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4, n_rows = a.group * a.n_new;
  const int kvh = blockIdx.x % a.n_kvh, rest = blockIdx.x / a.n_kvh, tile = rest % a.row_tiles, part = rest / a.row_tiles;
  const size_t slot = ((size_t)tile * a.n_kvh + kvh) * a.prefix_parts + part;
  const int lo = part * a.prefix_chunk, hi = min(lo + a.prefix_chunk, a.prefix_len);
  Rows<FP8, NT> rows;
#pragma unroll
  for (int qt = 0; qt < NT; ++qt) {
    const int row = min((tile * NT + qt) * 16 + n, a.n_seqs * n_rows - 1), s = row / n_rows;
    load_row<FP8, NT>(a.q, a.sq, a.group, kvh, s, row - s * n_rows, qt, g, rows);
    rows.token[qt] = 0;
  }
  const Keys ks = {a.prefix_table, a.prefix_len, a.prefix_len, a.prefix_len - 1};
  const float scale = FP8 ? kLog2eByRootD * a.c.k_scale[kvh] : kLog2eByRootD;
  int from = lo + kStep * wave;
  if constexpr (NT == 4) {
    // whole steps of pages that are there by the pipeline
    bool missing = false;
    for (int i = (lo >> a.c.page_shift) + lane; i <= (hi - 1) >> a.c.page_shift; i += 64) missing |= (unsigned)ks.table[i] >= (unsigned)a.c.n_pages;
    const int steps = (max(hi - from, 0) / kStep + kWaves - 1) / kWaves & ~1;
    if (steps > 0 && __builtin_amdgcn_ballot_w64(missing) == 0) {
      if (a.c.page_shift >= 5) pipeline<FP8, true>(a.c, ks, kvh, from, steps, lane, wave, scale, lds, rows);
      else pipeline<FP8, false>(a.c, ks, kvh, from, steps, lane, wave, scale, lds, rows);
      from += steps * kTurn;
    }
  }
  sweep<FP8, NT, NT != 4>(a.c, ks, kvh, from, hi, lane, 1, scale, rows);
  join_waves<FP8, NT>(rows, lds.join, wave, lane,
    [&](int qt, int c, f32x4 x, float) { a.pre_acc[((slot * 8 + c) * 4 + g) * (16 * NT) + 16 * qt + n] = x; },
    [&](int row, float ref, float l) { a.pre_sum[slot * 16 * NT + row] = make_float2(ref, l); });
}

// Joins the parts of 16 rows of a sequence and KV head.  The weights of the parts first, kMostWeights at a time, in LDS; then wave
// (half, c) adds up the accumulators of number c of every part (HALVES = 2: of every other one), 4 loads in flight; the rows leave
// through LDS as whole ones.
constexpr int kMostWeights = 256;
template <int HALVES>
__global__ __launch_bounds__(512 * HALVES) void join_kernel(DecodeArgs a, int pre_rows) {
  constexpr int kSeats = 32 * HALVES;      // parts whose weights are made at a time, 16 rows each
  __shared__ __attribute__((aligned(16))) uint16_t out[16][kHeadDim + 8];
  __shared__ float weight[kMostWeights][16], most[kSeats][16], sums[kSeats][16];
  __shared__ f32x4 half_acc[HALVES == 2 ? 8 : 1][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = wave & 7, half = wave >> 3;
  const int n = lane & 15, g = lane >> 4, n_rows = a.group * a.n_new;
  const int kvh = blockIdx.x % a.n_kvh, rest = blockIdx.x / a.n_kvh, tiles = (n_rows + 15) / 16, qt = rest % tiles, s = rest / tiles;
  const int r = min(16 * qt + n, n_rows - 1);
  const int turns = turns_of(a.c, entry_at(a.c.lens, s));
  int own_parts = 0;
  size_t own = 0;      // slot of the first part of the own keys
  if (turns > 0) {
    const int2 at = a.turns[(size_t)kvh * a.n_seqs + s];
    const int first = share_with(at.y, a.shares, at.x);
    own_parts = share_with(at.y, a.shares, at.x + turns - 1) - first + 1;
    own = (size_t)kvh * (a.shares + a.n_seqs) + first + s;
    if (own_parts == 1 && a.prefix_len == 0) return;      // (already the result)
  }
  const int row = s * n_rows + r, tile = row / pre_rows, in_tile = row - tile * pre_rows;
  const size_t pre = ((size_t)tile * a.n_kvh + kvh) * a.prefix_parts;
  const int parts = a.prefix_parts + own_parts;
  // part i of this lane's row: the prefix's first
  auto sum_of = [&](int i) {
    return i < a.prefix_parts ? a.pre_sum[(pre + i) * pre_rows + in_tile] : a.own_sum[(own + i - a.prefix_parts) * n_rows + r];
  };
  const int seat = tid >> 4;      // (tid % 16 = n)
  float top = kNoRef;
  for (int i = seat; i < parts; i += kSeats) top = fmaxf(top, sum_of(i).x);
  most[seat][n] = top;
  __syncthreads();
  for (int i = 0; i < min(kSeats, parts); ++i) top = fmaxf(top, most[i][n]);
  float l = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i0 = 0; i0 < parts; i0 += kMostWeights) {
    const int here = min(kMostWeights, parts - i0);
    if (i0 > 0) __syncthreads();
    for (int i = seat; i < (here + 7 & ~7); i += kSeats) {
      const float2 x = i < here ? sum_of(i0 + i) : make_float2(kNoRef, 0.0f);
      // (a part without keys for this row: sum and accumulators are 0)
      const float w = __builtin_amdgcn_exp2f(x.x - top);
      weight[i][n] = w;
      l += w * x.y;
    }
    __syncthreads();
    for (int i = half; i < here; i += 4 * HALVES) {
      f32x4 x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at = min(i0 + i + HALVES * e, parts - 1), mine = at - a.prefix_parts;
        const f32x4* from = mine < 0 ? a.pre_acc + (((pre + at) * 8 + c) * 4 + g) * pre_rows + in_tile
                                     : a.own_acc + (((own + mine) * 8 + c) * 4 + g) * n_rows + r;
        x[e] = *from;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // (By the part's number, not by its weight: what is not finite stays so under a weight that is too small for a float, as it does
        // under the exponentials inside a part.)
        const float w = weight[i + HALVES * e][n];
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[f] += i + HALVES * e < here ? w * x[e][f] : 0.0f;
      }
    }
  }
  sums[seat][n] = l;
  if (HALVES == 2 && half == 1) half_acc[c][lane] = acc;
  __syncthreads();
  if (half == 0) {
    l = 0.0f;
    for (int i = 0; i < min(kSeats, parts); ++i) l += sums[i][n];
    if constexpr (HALVES == 2) acc += half_acc[c][lane];
    const float by = l == 0.0f ? 0.0f : (a.c.v_scale ? a.c.v_scale[kvh] : 1.0f) / l;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[n][32 * g + 8 * e + c] = __builtin_bit_cast(uint16_t, (__bf16)(l == 0.0f ? 0.0f : acc[e] * by));
    if (a.lse && c == 0 && g == 0 && 16 * qt + n < n_rows) {
      const RowOf w = row_of(a.group, r);
      a.lse[((size_t)s * a.sq.heads + kvh * a.group + w.head) * a.n_new + w.token] = lse_of(top, l);
    }
  }
  __syncthreads();
  const int line = tid >> 4, r_out = 16 * qt + line;
  if (line < 16 && r_out < n_rows) {
    const RowOf w = row_of(a.group, r_out);
    uint16_t* to = a.o + row_off(a.so, s * a.so.heads + kvh * a.group + w.head, w.token) + 8 * (tid & 15);
    *(u32x4*)to = *(const u32x4*)&out[line][8 * (tid & 15)];
  }
}

// How a call is cut, as far as its sizes say (which share has which keys follows from lens).
//
// Workgroups for the own keys: one per CU reads as fast as more of them, which only make more partial results.  bf16, us with
// 256, 512, 1024, 2048 workgroups: 64 sequences of 0 .. 8000 keys 198, 202, 202, 205; 4 of 65000 .. 131072 261, 265, 269, 275; one
// of 32000 31.0, 35.2, 40.9; 16 of 500 .. 1000 19.9, 19.0, 20.2; 128 of 1000 .. 2000 150, 150, 160.  8-bit pages have half the bytes
// in flight per workgroup and want two per CU where there is much to read: 128 of 1000 .. 2000 93.9, 83.0, 98.3; 16 of 4000 .. 8000
// 47.5, 43.5, 47.3; but one of 8000 15.1, 18.3; one of 32000 23.6, 26.3.  So do short sequences (here behind a prefix), whose pieces
// each begin with a wait that another workgroup can fill: kernel, 256, 512, 768 workgroups, 128 of 0 .. 300 keys 24.1, 17.6, 19.9;
// 0 .. 1000 48.4, 44.8, 44.1, four new tokens each 54.6, 47.1, 46.2; 32 of 0 .. 1000 17.5, 15.6, 15.1; but 0 .. 2000 101, 102, 102, and 0 .. 4000
// 188, 193, 189.
// The parts of the prefix likewise, of either type, for up to 32 rows: 4 sequences behind 32000 keys 37.9, 42.2, 49.4, on 8-bit pages
// 28.0, 31.7, 38.1.  With 64 rows a workgroup has a CU to itself, so that 256 of them are one round of the chip and a few more are two:
// the number of parts, rounded up, gives 256 where the row tiles times KV heads divide it, and otherwise up to 320.  Call, 32 / 8 heads
// behind 32749 keys, 32, 48, 64, 80, 96, 128, 160, 192 sequences of one own key: 42.2, 71.8, 57.7, 95.2, 108, 93.2, 157, 194; on 8-bit
// pages 38.9, 69.8, 55.6, 93.9, 107, 88.1, 156, 194.
// (Cut into a number of parts that each sequence had to itself, the 64 took 251: the parts of the longest ended last.)
constexpr int kCus = 256, kPlentyTurns = 2048, kShortTurns = 12;
// Without a prefix, short sequences are left whole: one launch, and nothing to join.  us, cut -> whole, 8 KV heads: one sequence of
// 531 keys 14.9 -> 11.0, 750 15.0 -> 12.7, 1000 14.8 -> 15.5; 16 x 531 16.7 -> 12.5; 32 x 0 .. 1000 22.8 -> 18.9, 0 .. 1300 24.8 ->
// 22.6; 128 x 0 .. 1300 75.6 -> 72.9.
// Short, here and above, is what the tables have room for: the launches may not depend on lens, so that a wide table of short sequences
// is cut like that of long ones.  Call, under a table as wide as the keys -> one for 32K or 128K tokens: one sequence of 531 keys
// 11.2 -> 14.1, 16 of them 12.4 -> 17.1; 128 of 0 .. 1000 48.5 -> 52.5, behind 32749 keys 143.6 -> 144.7.
constexpr int kWholeTurns = 6, kManyUnits = 256, kWholeTurnsOfMany = 10;
struct Plan {
  int own_tiles, pre_tiles;      // 16-row tiles per workgroup
  int shares, prefix_parts, prefix_chunk, row_tiles;
  bool whole;                    // a workgroup per sequence and KV head, no workspace
  size_t pre_slots;
  size_t own_acc_bytes, own_sum_bytes, pre_acc_bytes, pre_sum_bytes, turns_bytes, bytes;
};

Plan make_plan(const sale_params_t* p, const sale_cache_t* c, int prefix_len) {
  Plan w = {};
  const int n_rows = p->n_q_heads / p->n_kv_heads * p->seq_len;
  const long long all_rows = (long long)p->batch * n_rows;
  auto tiles_for = [](long long rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; };
  auto up = [](long long a, long long b) { return (a + b - 1) / b; };
  auto clamp = [](long long x, long long lo, long long hi) { return (int)(x < lo ? lo : x > hi ? hi : x); };
  w.own_tiles = tiles_for(n_rows);
  const long long units = (long long)p->batch * p->n_kv_heads;
  const long long each = up((long long)c->table_width * c->page_tokens, kTurn), turns = each * p->batch;      // at most
  w.whole = prefix_len == 0 && each <= (units >= kManyUnits ? kWholeTurnsOfMany : kWholeTurns);
  const bool two = each <= kShortTurns || (c->dtype == SALE_PAGE_FP8 && turns * p->n_kv_heads > kPlentyTurns);
  const int workgroups = two ? 2 * kCus : kCus;
  w.shares = w.whole ? p->batch : clamp(up(workgroups, p->n_kv_heads), 1, turns);
  if (w.whole) return w;
  if (prefix_len > 0) {
    w.pre_tiles = tiles_for(all_rows);
    w.row_tiles = (int)up(all_rows, 16 * w.pre_tiles);
    const long long groups = w.row_tiles * (long long)p->n_kv_heads;
    const int parts = clamp(up(kCus, groups), 1,
                            up(prefix_len, kTurn) < 128 ? up(prefix_len, kTurn) : 128);
    const int whole = w.pre_tiles == 4 ? 2 * kTurn : kTurn;      // (the pipeline takes steps by two)
    w.prefix_chunk = (int)(up(up(prefix_len, parts), whole) * whole);
    w.prefix_parts = (int)up(prefix_len, w.prefix_chunk);
    w.pre_slots = (size_t)groups * w.prefix_parts;
  }
  const size_t own_rows = (size_t)p->n_kv_heads * (w.shares + p->batch) * n_rows, pre_rows = w.pre_slots * 16 * w.pre_tiles;
  auto whole = [](size_t bytes) { return (bytes + 15) & ~(size_t)15; };
  w.own_acc_bytes = own_rows * kHeadDim * sizeof(float);
  w.pre_acc_bytes = pre_rows * kHeadDim * sizeof(float);
  w.own_sum_bytes = whole(own_rows * sizeof(float2));
  w.pre_sum_bytes = whole(pre_rows * sizeof(float2));
  w.turns_bytes = (size_t)p->n_kv_heads * p->batch * sizeof(int2);
  w.bytes = w.own_acc_bytes + w.own_sum_bytes + w.pre_acc_bytes + w.pre_sum_bytes + w.turns_bytes;
  return w;
}

// What sale.h promises, and the plan.
int plan_of(const sale_params_t* p, const sale_cache_t* c, int prefix_len, Plan& w) {
  int rc = validate_tokens(p);
  if (rc == SALE_OK) rc = validate_cache(p, c, true);
  if (rc != SALE_OK) return rc;
  if (prefix_len < 0) return SALE_ERR_BAD_SHAPE;
  if (prefix_len > 0x3FFFFFFF || p->n_seqs > 0) return SALE_ERR_UNSUPPORTED;
  if ((long long)(p->n_q_heads / p->n_kv_heads) * p->seq_len > 64) return SALE_ERR_UNSUPPORTED;
  // (workgroups, rows and turns are counted in 32 bits)
  if (((long long)c->table_width * c->page_tokens / kTurn + 1) * p->batch > 0x7FFFFFFF) return SALE_ERR_UNSUPPORTED;
  if ((long long)p->batch * p->n_q_heads * p->seq_len > 0x3FFFFFFF || (long long)p->batch * p->n_kv_heads > (0x7FFFFFFF >> 8)) return SALE_ERR_UNSUPPORTED;
  w = make_plan(p, c, prefix_len);
  // (the join has 16 rows per workgroup, of 512 threads where there are many; the prefix 64 per workgroup of 256)
  const long long join = (long long)p->batch * p->n_kv_heads * ((p->n_q_heads / p->n_kv_heads * p->seq_len + 15) / 16);
  if ((!w.whole && 2 * join > kMostWorkgroups) || w.pre_slots > (size_t)kMostWorkgroups) return SALE_ERR_UNSUPPORTED;
  return SALE_OK;
}

template <bool FP8>
void launch_decode(const DecodeArgs& a, const Plan& w, hipStream_t st) {
  const dim3 own((unsigned)(a.n_kvh * a.shares)), pre((unsigned)w.pre_slots), threads(64 * kWaves);
  if (w.pre_slots > 0) {
    if (w.pre_tiles == 1) prefix_kernel<FP8, 1><<<pre, threads, 0, st>>>(a);
    else if (w.pre_tiles == 2) prefix_kernel<FP8, 2><<<pre, threads, 0, st>>>(a);
    else prefix_kernel<FP8, 4><<<pre, threads, 0, st>>>(a);
  }
  if (w.whole) {
    if (w.own_tiles == 1) own_kernel<FP8, 1, true><<<own, threads, 0, st>>>(a);
    else if (w.own_tiles == 2) own_kernel<FP8, 2, true><<<own, threads, 0, st>>>(a);
    else own_kernel<FP8, 4, true><<<own, threads, 0, st>>>(a);
    return;
  }
  if (w.own_tiles == 1) own_kernel<FP8, 1, false><<<own, threads, 0, st>>>(a);
  else if (w.own_tiles == 2) own_kernel<FP8, 2, false><<<own, threads, 0, st>>>(a);
  else own_kernel<FP8, 4, false><<<own, threads, 0, st>>>(a);
  const int n_rows = a.group * a.n_new, tiles = (n_rows + 15) / 16;
  const dim3 join((unsigned)((size_t)a.n_seqs * a.n_kvh * tiles));
  const int pre_rows = 16 * (w.pre_tiles > 0 ? w.pre_tiles : 1);
  // (more of the large ones than fit at a time: 1024 of them, 128 sequences, 16.4 us, of the small ones 10.4)
  if (join.x > 2 * kCus) join_kernel<1><<<join, dim3(512), 0, st>>>(a, pre_rows);
  else join_kernel<2><<<join, dim3(1024), 0, st>>>(a, pre_rows);
}

}  // namespace

}  // namespace sale

using namespace sale;

extern "C" size_t sale_decode_workspace_bytes(const sale_params_t* p, const sale_cache_t* cache, int32_t prefix_len) {
  Plan w;
  return p && cache && plan_of(p, cache, prefix_len, w) == SALE_OK ? w.bytes : 0;
}

extern "C" int sale_decode_attn(const sale_params_t* p, const sale_cache_t* cache, const void* q, const int32_t* prefix_table,
                                int32_t prefix_len, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (!p || !cache || !q || !o || (prefix_len > 0 && !prefix_table)) return SALE_ERR_NULL_ARG;
  Plan w;
  const int rc = plan_of(p, cache, prefix_len, w);
  if (rc != SALE_OK) return rc;
  if (((uintptr_t)q | (uintptr_t)o) & 15) return SALE_ERR_BAD_SHAPE;
  if (w.bytes > 0 && (!ws || ws_bytes < w.bytes || ((uintptr_t)ws & 15))) return SALE_ERR_WORKSPACE;
  DecodeArgs a = {};
  a.c = cache_view(p, cache);
  if (cache->dtype != SALE_PAGE_FP8) a.c.k_scale = a.c.v_scale = nullptr;
  a.q = (const uint16_t*)q;
  a.o = (uint16_t*)o;
  a.lse = lse;
  a.sq = layout_of(p->q_stride, p->n_q_heads, p->seq_len);
  a.so = layout_of(p->o_stride, p->n_q_heads, p->seq_len);
  a.prefix_table = prefix_table;
  a.prefix_len = prefix_len;
  a.n_seqs = p->batch;
  a.n_new = p->seq_len;
  a.group = p->n_q_heads / p->n_kv_heads;
  a.n_kvh = p->n_kv_heads;
  a.shares = w.shares;
  a.prefix_parts = w.prefix_parts;
  a.prefix_chunk = w.prefix_chunk;
  a.row_tiles = w.row_tiles;
  uint8_t* at = (uint8_t*)ws;
  a.own_acc = (f32x4*)at; at += w.own_acc_bytes;
  a.pre_acc = (f32x4*)at; at += w.pre_acc_bytes;
  a.own_sum = (float2*)at; at += w.own_sum_bytes;
  a.pre_sum = (float2*)at; at += w.pre_sum_bytes;
  a.turns = (int2*)at;
  if (cache->dtype == SALE_PAGE_FP8) launch_decode<true>(a, w, (hipStream_t)stream);
  else launch_decode<false>(a, w, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? SALE_OK : SALE_ERR_HIP;
}
