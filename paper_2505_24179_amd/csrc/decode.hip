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
//   are.  No LDS, no exchange between lanes in the loop.
// The 4 waves of a workgroup take every fourth step of its keys and join at the end through LDS.
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
  int own_parts, own_least;                     // parts of a sequence's own keys, and the fewest keys that one of them takes
  int prefix_parts, prefix_chunk, row_tiles;    // parts of the prefix, keys of each; tiles of 16 * (row tiles of the kernel) rows
  f32x4* own_acc;  float2* own_sum;             // [sequence][KV head][part] partial results: [row tile][8][64], [row]
  f32x4* pre_acc;  float2* pre_sum;             // [tile][KV head][part]
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

// Pages of the two 16-key tiles of the step at key0 (of its last one that exists where it lies behind it); -1: no page.
struct TwoPages { int a, b; };
__device__ __forceinline__ TwoPages pages_of(const CacheView& c, const Keys& ks, int key0) {
  const int last = (ks.n - 1) & ~15;
  const int a = ks.table[min(key0, last) >> c.page_shift], b = ks.table[min(key0 + 16, last) >> c.page_shift];
  return {(unsigned)a < (unsigned)c.n_pages ? a : -1, (unsigned)b < (unsigned)c.n_pages ? b : -1};
}

template <bool FP8>
__device__ __forceinline__ void load_step(const CacheView& c, const Keys& ks, int kvh, int key0, TwoPages pg, int m, int g, Operands<FP8>& x) {
  const int last = (ks.n - 1) & ~15, mask = (1 << c.page_shift) - 1;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int page = t == 0 ? pg.a : pg.b;
    const int slot = min(key0 + 16 * t, last) & mask;
    const long long at = page < 0 ? 0 : page;      // (without a page: any one, whose keys are not used)
    const uint8_t* kb = c.k.base + at * c.k.page + (long long)kvh * c.k.head + (long long)slot * c.k.token;
    const uint32_t row = (uint32_t)(4 * (m & 3) + (m >> 2)) * (uint32_t)c.k.token + 16 * g;
#pragma unroll
    for (int s = 0; s < (FP8 ? 2 : 4); ++s) x.k[t][s] = *(const u32x4*)(kb + row + 64 * s);
    const uint8_t* vb = c.v.base + at * c.v.page + (long long)kvh * c.v.head + (long long)slot * c.v.token;
    const uint32_t col = (uint32_t)g * (uint32_t)c.v.token + (FP8 ? 8 : 16) * m;
#pragma unroll
    for (int r = 0; r < 4; ++r) x.v[4 * t + r] = *(const std::remove_reference_t<decltype(x.v[0])>*)(vb + (long long)(4 * r) * c.v.token + col);
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
template <bool FP8, int NT>
__device__ __forceinline__ void one_key(const CacheView& c, Rows<FP8, NT>& rows, const bf16x8 (&p)[NT], const Keys& ks, int kvh, int key,
                                        int key0, TwoPages pg, int g) {
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
      if (j == in >> 2) x = (float)p[qt][j];
    pk[qt] = __shfl(x, (int)(threadIdx.x & 15) + 16 * (in & 3), 64);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x;
      if constexpr (FP8) x = __builtin_amdgcn_cvt_f32_fp8(v[8 * r + e], 0);
      else x = bf16_bits_to_float(((const uint16_t*)v)[8 * r + e]);
#pragma unroll
      for (int qt = 0; qt < NT; ++qt)
        if (key <= ks.before + rows.token[qt]) rows.acc[qt][e][r] = __builtin_fmaf(pk[qt], x, rows.acc[qt][e][r]);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// One step: its 32 keys enter acc, l and ref.  edge: some of the keys are not there, or not for all rows.
template <bool FP8, int NT>
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
  bf16x8 p[NT];
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
      const float e = __builtin_amdgcn_exp2f(v[j] - rows.ref[qt]);
      rows.l[qt] += e;
      p[qt][j] = (__bf16)e;
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
      for (int key = max(ks.all, key0); key < min(ks.n, key0 + kStep); ++key) one_key<FP8, NT>(c, rows, p, ks, kvh, key, key0, pg, g);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bf16x8 v = turned<FP8>(x, e);
#pragma unroll
    for (int qt = 0; qt < NT; ++qt) rows.acc[qt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[qt], rows.acc[qt][e], 0, 0, 0);
  }
}

// Keys lo .. hi - 1 for the rows, by the waves of the workgroup in turn.
template <bool FP8, int NT>
__device__ __forceinline__ void sweep(const CacheView& c, const Keys& ks, int kvh, int lo, int hi, int wave, int lane, int n_new, float scale,
                                      Rows<FP8, NT>& rows) {
  const int m = lane & 15, g = lane >> 4;
  for (int key0 = lo + kStep * wave; key0 < hi; key0 += kTurn) {
    const TwoPages pg = pages_of(c, ks, key0);
    Operands<FP8> x;
    load_step<FP8>(c, ks, kvh, key0, pg, m, g, x);
    step<FP8, NT>(c, x, rows, scale, ks, kvh, key0, pg, key0 + kStep > ks.all || (pg.a | pg.b) < 0, g, n_new);
  }
}

// The results of the four waves, joined: sum (one per row) and acc (one 16-row tile after the other, 8 x 64 lanes x 4 floats).
// keep(qt, c, x): x = accumulator c of this lane in tile qt, for two numbers c per wave; sums(row, ref, l).
struct JoinLds {
  f32x4 acc[kWaves][8][64];
  float ref[kWaves][64], l[kWaves][64];
};
template <bool FP8, int NT, class Keep, class Sums>
__device__ __forceinline__ void join_waves(Rows<FP8, NT>& rows, JoinLds& lds, int wave, int lane, Keep keep, Sums sums) {
  const int n = lane & 15, g = lane >> 4;
#pragma unroll
  for (int qt = 0; qt < NT; ++qt) {
    rows.l[qt] += __shfl_xor(rows.l[qt], 16, 64);
    rows.l[qt] += __shfl_xor(rows.l[qt], 32, 64);
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
__device__ __forceinline__ RowOf row_of(const DecodeArgs& a, int r) { const int t = r / a.group; return {t, r - t * a.group}; }

template <bool FP8, int NT>
__device__ __forceinline__ void load_row(const DecodeArgs& a, int kvh, int s, int r, int qt, int g, Rows<FP8, NT>& rows) {
  const RowOf w = row_of(a, r);
  const uint16_t* row = a.q + row_off(a.sq, s * a.sq.heads + kvh * a.group + w.head, w.token);
#pragma unroll
  for (int e = 0; e < 4; ++e) rows.q[qt][e] = *(const bf16x8*)(row + step_channel<FP8>(e, g));
  rows.token[qt] = w.token;
  rows.ref[qt] = kNoRef;
  rows.l[qt] = 0.0f;
#pragma unroll
  for (int c = 0; c < 8; ++c) rows.acc[qt][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
}

// A workgroup: one part of a sequence's own keys, for the rows of one KV head.
template <bool FP8, int NT, bool DIRECT>
__global__ __launch_bounds__(64 * kWaves, NT == 4 ? 1 : 2) void own_kernel(DecodeArgs a) {
  __shared__ JoinLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4, n_rows = a.group * a.n_new;
  const int kvh = blockIdx.x % a.n_kvh, rest = blockIdx.x / a.n_kvh, part = rest % a.own_parts, s = rest / a.own_parts;
  const size_t slot = ((size_t)s * a.n_kvh + kvh) * a.own_parts + part;
  const int held = max(a.c.lens[s], 0), n_keys = min(held, a.c.width << a.c.page_shift);
  const int chunk = max(a.own_least, ((n_keys + a.own_parts - 1) / a.own_parts + kTurn - 1) / kTurn * kTurn);
  const int lo = (int)min((long long)part * chunk, (long long)n_keys), hi = min(lo + chunk, n_keys);
  if (!DIRECT && lo >= hi) {
    if (tid < 16 * NT) a.own_sum[slot * 16 * NT + tid] = make_float2(kNoRef, 0.0f);
    return;
  }
  Rows<FP8, NT> rows;
#pragma unroll
  for (int qt = 0; qt < NT; ++qt) load_row<FP8, NT>(a, kvh, s, min(16 * qt + n, n_rows - 1), qt, g, rows);
  const Keys ks = {a.c.table + (size_t)s * a.c.width, n_keys, min(held - a.n_new + 1, n_keys), held - a.n_new};
  const float scale = FP8 ? kLog2eByRootD * a.c.k_scale[kvh] : kLog2eByRootD;
  sweep<FP8, NT>(a.c, ks, kvh, lo, hi, wave, lane, a.n_new, scale, rows);
  const float v_scale = FP8 ? a.c.v_scale[kvh] : 1.0f;
  join_waves<FP8, NT>(rows, lds, wave, lane,
    [&](int qt, int c, f32x4 x, float l) {
      if constexpr (DIRECT) {
        const int r = 16 * qt + n;
        if (r >= n_rows) return;
        const RowOf w = row_of(a, r);
        uint16_t* out = a.o + row_off(a.so, s * a.so.heads + kvh * a.group + w.head, w.token) + 32 * g + c;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[8 * e] = __builtin_bit_cast(uint16_t, (__bf16)(l == 0.0f ? 0.0f : x[e] / l * v_scale));
      } else {
        a.own_acc[((slot * NT + qt) * 8 + c) * 64 + lane] = x;
      }
    },
    [&](int row, float ref, float l) {
      if constexpr (DIRECT) {
        if (row >= n_rows || !a.lse) return;
        const RowOf w = row_of(a, row);
        a.lse[((size_t)s * a.sq.heads + kvh * a.group + w.head) * a.n_new + w.token] = lse_of(ref, l);
      } else {
        a.own_sum[slot * 16 * NT + row] = make_float2(ref, l);
      }
    });
}

// A workgroup: one part of the prefix, for 16 NT rows of one KV head, of whichever sequences.
template <bool FP8, int NT>
__global__ __launch_bounds__(64 * kWaves, NT == 4 ? 1 : 2) void prefix_kernel(DecodeArgs a) {
  __shared__ JoinLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4, n_rows = a.group * a.n_new;
  const int kvh = blockIdx.x % a.n_kvh, rest = blockIdx.x / a.n_kvh, tile = rest % a.row_tiles, part = rest / a.row_tiles;
  const size_t slot = ((size_t)tile * a.n_kvh + kvh) * a.prefix_parts + part;
  const int lo = part * a.prefix_chunk, hi = min(lo + a.prefix_chunk, a.prefix_len);
  Rows<FP8, NT> rows;
#pragma unroll
  for (int qt = 0; qt < NT; ++qt) {
    const int row = min((tile * NT + qt) * 16 + n, a.n_seqs * n_rows - 1), s = row / n_rows;
    load_row<FP8, NT>(a, kvh, s, row - s * n_rows, qt, g, rows);
    rows.token[qt] = 0;
  }
  const Keys ks = {a.prefix_table, a.prefix_len, a.prefix_len, a.prefix_len - 1};
  const float scale = FP8 ? kLog2eByRootD * a.c.k_scale[kvh] : kLog2eByRootD;
  sweep<FP8, NT>(a.c, ks, kvh, lo, hi, wave, lane, 1, scale, rows);
  join_waves<FP8, NT>(rows, lds, wave, lane,
    [&](int qt, int c, f32x4 x, float) { a.pre_acc[((slot * NT + qt) * 8 + c) * 64 + lane] = x; },
    [&](int row, float ref, float l) { a.pre_sum[slot * 16 * NT + row] = make_float2(ref, l); });
}

// Joins the parts of 16 rows of a sequence and KV head.  Wave c has the accumulators of number c; the rows leave through LDS as
// whole ones.
__global__ __launch_bounds__(512) void join_kernel(DecodeArgs a, int own_tiles, int pre_tiles) {
  __shared__ __attribute__((aligned(16))) uint16_t out[16][kHeadDim + 8];
  const int tid = threadIdx.x, lane = tid & 63, c = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4, n_rows = a.group * a.n_new;
  const int kvh = blockIdx.x % a.n_kvh, rest = blockIdx.x / a.n_kvh, qt = rest % own_tiles, s = rest / own_tiles;
  const int r = min(16 * qt + n, n_rows - 1);
  const size_t own = ((size_t)s * a.n_kvh + kvh) * a.own_parts;
  const int row = s * n_rows + r, tile = row / (16 * pre_tiles), in_tile = row - tile * 16 * pre_tiles;
  const size_t pre = ((size_t)tile * a.n_kvh + kvh) * a.prefix_parts;
  float top = kNoRef;
  for (int i = 0; i < a.prefix_parts; ++i) top = fmaxf(top, a.pre_sum[(pre + i) * 16 * pre_tiles + in_tile].x);
  for (int i = 0; i < a.own_parts; ++i) top = fmaxf(top, a.own_sum[(own + i) * 16 * own_tiles + r].x);
  float l = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](float2 sum, const f32x4* from) {
    if (sum.y == 0.0f) return;      // (a part without keys for this row: its accumulators may not be there)
    const float by = __builtin_amdgcn_exp2f(sum.x - top);
    l += by * sum.y;
    acc += by * *from;
  };
  for (int i = 0; i < a.prefix_parts; ++i)
    add(a.pre_sum[(pre + i) * 16 * pre_tiles + in_tile],
        a.pre_acc + (((pre + i) * pre_tiles + in_tile / 16) * 8 + c) * 64 + 16 * g + in_tile % 16);
  for (int i = 0; i < a.own_parts; ++i)
    add(a.own_sum[(own + i) * 16 * own_tiles + r], a.own_acc + (((own + i) * own_tiles + qt) * 8 + c) * 64 + 16 * g + r % 16);
  const float by = l == 0.0f ? 0.0f : (a.c.v_scale ? a.c.v_scale[kvh] : 1.0f) / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[n][32 * g + 8 * e + c] = __builtin_bit_cast(uint16_t, (__bf16)(l == 0.0f ? 0.0f : acc[e] * by));
  if (a.lse && c == 0 && g == 0 && 16 * qt + n < n_rows) {
    const RowOf w = row_of(a, r);
    a.lse[((size_t)s * a.sq.heads + kvh * a.group + w.head) * a.n_new + w.token] = lse_of(top, l);
  }
  __syncthreads();
  const int line = tid >> 4, r_out = 16 * qt + line;
  if (line < 16 && r_out < n_rows) {
    const RowOf w = row_of(a, r_out);
    uint16_t* to = a.o + row_off(a.so, s * a.so.heads + kvh * a.group + w.head, w.token) + 8 * (tid & 15);
    *(u32x4*)to = *(const u32x4*)&out[line][8 * (tid & 15)];
  }
}

// How a call is cut, from its sizes alone.
struct Plan {
  int own_tiles, pre_tiles;      // 16-row tiles per workgroup
  int own_parts, own_least, prefix_parts, prefix_chunk, row_tiles;
  bool direct;                   // one part: the result itself
  size_t own_slots, pre_slots;
  size_t own_acc_bytes, own_sum_bytes, pre_acc_bytes, pre_sum_bytes, bytes;
};

Plan make_plan(const sale_params_t* p, const sale_cache_t* c, int prefix_len) {
  Plan w = {};
  const int n_rows = p->n_q_heads / p->n_kv_heads * p->seq_len;
  const long long units = (long long)p->batch * p->n_kv_heads, all_rows = (long long)p->batch * n_rows;
  auto tiles_for = [](long long rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; };
  auto up = [](long long a, long long b) { return (a + b - 1) / b; };
  auto clamp = [](long long x, long long lo, long long hi) { return (int)(x < lo ? lo : x > hi ? hi : x); };
  w.own_tiles = tiles_for(n_rows);
  const long long capacity = (long long)c->table_width * c->page_tokens;
  const long long most = up(capacity, kTurn) < 128 ? up(capacity, kTurn) : 128;
  const long long wanted = up(1024, units), by_length = up(capacity, 2048);
  w.own_parts = clamp(wanted > by_length ? wanted : by_length, 1, most);
  w.own_least = units < 256 ? kTurn : 4 * kTurn;
  w.direct = w.own_parts == 1 && prefix_len == 0;
  if (prefix_len > 0) {
    w.pre_tiles = tiles_for(all_rows);
    w.row_tiles = (int)up(all_rows, 16 * w.pre_tiles);
    const long long groups = (long long)w.row_tiles * p->n_kv_heads;
    const int parts = clamp(up(1024, groups), 1, up(prefix_len, kTurn) < 128 ? up(prefix_len, kTurn) : 128);
    w.prefix_chunk = (int)(up(up(prefix_len, parts), kTurn) * kTurn);
    w.prefix_parts = (int)up(prefix_len, w.prefix_chunk);
    w.pre_slots = (size_t)groups * w.prefix_parts;
  }
  w.own_slots = w.direct ? 0 : (size_t)units * w.own_parts;
  w.own_acc_bytes = w.own_slots * w.own_tiles * 8 * 64 * sizeof(f32x4);
  w.own_sum_bytes = w.own_slots * w.own_tiles * 16 * sizeof(float2);
  w.pre_acc_bytes = w.pre_slots * w.pre_tiles * 8 * 64 * sizeof(f32x4);
  w.pre_sum_bytes = w.pre_slots * w.pre_tiles * 16 * sizeof(float2);
  w.bytes = w.own_acc_bytes + w.own_sum_bytes + w.pre_acc_bytes + w.pre_sum_bytes;
  return w;
}

int validate_decode(const sale_params_t* p, const sale_cache_t* c, int prefix_len) {
  int rc = validate_tokens(p);
  if (rc == SALE_OK) rc = validate_cache(p, c, true);
  if (rc != SALE_OK) return rc;
  if (prefix_len < 0) return SALE_ERR_BAD_SHAPE;
  if (prefix_len > 0x3FFFFFFF || p->n_seqs > 0) return SALE_ERR_UNSUPPORTED;
  if ((long long)(p->n_q_heads / p->n_kv_heads) * p->seq_len > 64) return SALE_ERR_UNSUPPORTED;
  // (workgroups and rows are counted in 32 bits)
  if ((long long)p->batch * p->n_q_heads * p->seq_len > 0x3FFFFFFF || (long long)p->batch * p->n_kv_heads > (0x7FFFFFFF >> 8)) return SALE_ERR_UNSUPPORTED;
  return SALE_OK;
}

template <bool FP8>
void launch_decode(const DecodeArgs& a, const Plan& w, hipStream_t st) {
  const dim3 own((unsigned)((size_t)a.n_seqs * a.n_kvh * a.own_parts)), pre((unsigned)w.pre_slots), threads(64 * kWaves);
  if (w.pre_slots > 0) {
    if (w.pre_tiles == 1) prefix_kernel<FP8, 1><<<pre, threads, 0, st>>>(a);
    else if (w.pre_tiles == 2) prefix_kernel<FP8, 2><<<pre, threads, 0, st>>>(a);
    else prefix_kernel<FP8, 4><<<pre, threads, 0, st>>>(a);
  }
  if (w.direct) {
    if (w.own_tiles == 1) own_kernel<FP8, 1, true><<<own, threads, 0, st>>>(a);
    else if (w.own_tiles == 2) own_kernel<FP8, 2, true><<<own, threads, 0, st>>>(a);
    else own_kernel<FP8, 4, true><<<own, threads, 0, st>>>(a);
    return;
  }
  if (w.own_tiles == 1) own_kernel<FP8, 1, false><<<own, threads, 0, st>>>(a);
  else if (w.own_tiles == 2) own_kernel<FP8, 2, false><<<own, threads, 0, st>>>(a);
  else own_kernel<FP8, 4, false><<<own, threads, 0, st>>>(a);
  const int n_rows = a.group * a.n_new, tiles = (n_rows + 15) / 16;
  join_kernel<<<dim3((unsigned)((size_t)a.n_seqs * a.n_kvh * tiles)), dim3(512), 0, st>>>(a, w.own_tiles, w.pre_tiles > 0 ? w.pre_tiles : 1);
}

}  // namespace

}  // namespace sale

using namespace sale;

extern "C" size_t sale_decode_workspace_bytes(const sale_params_t* p, const sale_cache_t* cache, int32_t prefix_len) {
  if (!p || !cache || validate_decode(p, cache, prefix_len) != SALE_OK) return 0;
  return make_plan(p, cache, prefix_len).bytes;
}

extern "C" int sale_decode_attn(const sale_params_t* p, const sale_cache_t* cache, const void* q, const int32_t* prefix_table,
                                int32_t prefix_len, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (!p || !cache || !q || !o || (prefix_len > 0 && !prefix_table)) return SALE_ERR_NULL_ARG;
  const int rc = validate_decode(p, cache, prefix_len);
  if (rc != SALE_OK) return rc;
  if (((uintptr_t)q | (uintptr_t)o) & 15) return SALE_ERR_BAD_SHAPE;
  const Plan w = make_plan(p, cache, prefix_len);
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
  a.own_parts = w.own_parts;
  a.own_least = w.own_least;
  a.prefix_parts = w.prefix_parts;
  a.prefix_chunk = w.prefix_chunk;
  a.row_tiles = w.row_tiles;
  uint8_t* at = (uint8_t*)ws;
  a.own_acc = (f32x4*)at; at += w.own_acc_bytes;
  a.pre_acc = (f32x4*)at; at += w.pre_acc_bytes;
  a.own_sum = (float2*)at; at += w.own_sum_bytes;
  a.pre_sum = (float2*)at;
  if (cache->dtype == SALE_PAGE_FP8) launch_decode<true>(a, w, (hipStream_t)stream);
  else launch_decode<false>(a, w, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? SALE_OK : SALE_ERR_HIP;
}
