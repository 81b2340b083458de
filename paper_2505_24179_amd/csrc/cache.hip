// Pages of a cache: writing new tokens into them, and copying them.  Both only move bytes (8-bit pages: and round them), so
// what bounds them is HBM, or latency where a call is a few megabytes or less.
#include <stdlib.h>

#include "cache.h"

namespace sale {

int validate_cache(const sale_params_t* p, const sale_cache_t* c, bool tables) {
  if (!c->k || !c->v) return SALE_ERR_NULL_ARG;
  if (c->dtype != SALE_PAGE_BF16 && c->dtype != SALE_PAGE_FP8) return SALE_ERR_UNSUPPORTED;
  if (c->n_pages <= 0 || c->page_tokens <= 0) return SALE_ERR_BAD_SHAPE;
  if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return SALE_ERR_UNSUPPORTED;
  if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return SALE_ERR_BAD_SHAPE;
  const int unit = c->dtype == SALE_PAGE_FP8 ? 16 : 8;      // elements of 16 bytes
  const int64_t* triples[2] = {c->k_stride, c->v_stride};
  for (const int64_t* st : triples) {
    if (st[0] == 0 && st[1] == 0 && st[2] == 0) continue;
    for (int e = 0; e < 3; ++e)
      if (st[e] < 0 || st[e] % unit) return SALE_ERR_BAD_SHAPE;
    if (st[2] < kHeadDim) return SALE_ERR_BAD_SHAPE;
    if ((p->n_kv_heads > 1 && st[1] == 0) || (c->n_pages > 1 && st[0] == 0)) return SALE_ERR_BAD_SHAPE;
  }
  // (strides of pages and tokens are 32-bit numbers of bytes in the kernels, and so is a token's place in its page)
  for (const int64_t* st : triples) {
    const int64_t page = st[0] | st[1] | st[2] ? st[0] : (int64_t)p->n_kv_heads * c->page_tokens * kHeadDim;
    if (page > 0xFFFFFFFFLL / (16 / unit) || st[2] > (1 << 22)) return SALE_ERR_UNSUPPORTED;
  }
  if (c->dtype == SALE_PAGE_FP8 && tables && (!c->k_scale || !c->v_scale)) return SALE_ERR_NULL_ARG;
  if (!tables) return SALE_OK;
  if (!c->table || !c->lens) return SALE_ERR_NULL_ARG;
  if (c->table_width <= 0) return SALE_ERR_BAD_SHAPE;
  if ((long long)c->table_width * c->page_tokens > 0x3FFFFFFF) return SALE_ERR_UNSUPPORTED;      // positions are 32-bit
  return SALE_OK;
}

CacheView cache_view(const sale_params_t* p, const sale_cache_t* c) {
  const long long size = c->dtype == SALE_PAGE_FP8 ? 1 : 2;
  auto side = [&](void* base, const int64_t* st) -> PageSide {
    if (st[0] == 0 && st[1] == 0 && st[2] == 0) {
      const long long token = kHeadDim * size, head = token * c->page_tokens;
      return {(uint8_t*)base, head, (uint32_t)(head * p->n_kv_heads), (uint32_t)token};
    }
    return {(uint8_t*)base, st[1] * size, (uint32_t)(st[0] * size), (uint32_t)(st[2] * size)};
  };
  return {side(c->k, c->k_stride), side(c->v, c->v_stride), c->k_scale, c->v_scale, c->table, c->lens, c->n_pages,
          __builtin_ctz((unsigned)c->page_tokens), c->table_width};
}

namespace {

// ---- append ------------------------------------------------------------------------------------------------
// A workgroup takes up to `tile` tokens of one sequence, all KV heads, K and V: 16 bytes (8 channels) of the new token per
// thread and turn, so that a row of 256 bytes is 16 neighbouring threads'.  Where the tokens of a sequence lie among the
// packed ones travels with the launch, up to kAppendChunk sequences at a time.
// 24433 tokens of 8 heads into 8-bit pages (150 MB in and out) with 16, 32, 64, 128, 256 rows per workgroup: 47.4, 37.7, 42.0, 39.0,
// 55.8 us.
constexpr int kAppendChunk = 255, kAppendRows = 32;
struct AppendJob {
  CacheView c;
  const uint8_t *k, *v;
  Strided sk, sv;
  int n_kvh, tile, heads_first;      // heads_first: neighbouring rows are those of neighbouring heads
  int each, tiles_each;              // > 0: every sequence has that many new tokens, and workgroups; otherwise by `at`
  int first_seq, n;
  int token[kAppendChunk + 1], at[kAppendChunk + 1];      // first token and first workgroup of a sequence
};

// e4m3(x / scale), nearest, ties to even; at most 448 in size; NaN stays.  The quotient is the correctly rounded one: with
// inv = 1 / scale correctly rounded, q = x inv is next to it and one step of Newton's with the exact remainder gives it (Markstein,
// 1990), in 3 instructions where the compiler's division takes 10.  (q is limited first: from an infinite one the step would make a
// NaN; what is limited there is limited in the end.  The remainder is taken as q scale - x and subtracted: where it is zero it is
// +0, and -0 - 0 is -0, so that zero keeps its sign, which x - q scale, added, would not.)  A scale so far out that remainders could
// leave the range of a float takes the division.
struct Divisor { float scale, inv; bool far; };
__device__ __forceinline__ Divisor divisor(float scale) { return {scale, 1.0f / scale, !(scale >= 0x1p-60f && scale <= 0x1p60f)}; }
__device__ __forceinline__ float quotient448(float x, const Divisor& d) {
  float q = __builtin_amdgcn_fmed3f(x * d.inv, -1000.0f, 1000.0f);
  q = __builtin_fmaf(-__builtin_fmaf(q, d.scale, -x), d.inv, q);
  if (__builtin_expect(d.far, 0)) q = x / d.scale;
  return __builtin_elementwise_minimum(__builtin_elementwise_maximum(q, -448.0f), 448.0f);      // (a NaN passes these)
}
__device__ __forceinline__ u32x2 to_fp8(u32x4 w, const Divisor& d) {
  u32x2 out;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int r = 0;
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t word = w[2 * h + (e >> 1)];
      x[e] = quotient448(__builtin_bit_cast(float, e & 1 ? word & 0xFFFF0000u : word << 16), d);
    }
    r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], r, true);
    out[h] = (uint32_t)r;
  }
  return out;
}

template <bool FP8>
__global__ __launch_bounds__(256) void append_kernel(AppendJob a) {
  int s, t0, n_new, first;      // sequence, first token of the tile in it, its new tokens, its first packed token
  if (a.each > 0) {
    s = blockIdx.x / a.tiles_each;
    t0 = (int)(blockIdx.x - s * a.tiles_each) * a.tile;
    n_new = a.each;
    first = 0;      // (of batch entry s)
  } else {
    int lo = 0, hi = a.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.at[mid] <= (int)blockIdx.x) lo = mid; else hi = mid;
    }
    s = a.first_seq + lo;
    t0 = ((int)blockIdx.x - a.at[lo]) * a.tile;
    first = a.token[lo];
    n_new = a.token[lo + 1] - first;
  }
  const int count = min(a.tile, n_new - t0), rows = count * a.n_kvh;
  const int start = max(a.c.lens[s], 0) - n_new;      // position of the sequence's first new token
  const int32_t* table = a.c.table + (size_t)s * a.c.width;
  const int batch = a.each > 0 ? s : 0;
  // Rows come in lines: the heads of a token, or the tokens of a head.  (More than one token: 64 rows at most, and the product with
  // 2^16 / line_rows, rounded up, divides them exactly.)
  const bool by_head = a.heads_first || a.tile == 1;
  const int line_rows = by_head ? a.n_kvh : count, per_line = a.tile == 1 ? 0 : (65535 + line_rows) / line_rows;
  // (four turns at a time: their page numbers and tokens are in flight together)
  for (int id0 = threadIdx.x; id0 < 2 * rows * 16; id0 += 4 * 256) {
    u32x4 w[4];
    int page[4], pos[4], head[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int id = min(id0 + 256 * u, 2 * rows * 16 - 1);
      const bool is_v = id >= rows * 16;
      const int row = (is_v ? id - rows * 16 : id) >> 4;
      const int line = row * per_line >> 16, in_line = row - line * line_rows;
      const int h = by_head ? in_line : line, i = by_head ? line : in_line;
      head[u] = h;
      pos[u] = start + t0 + i;
      const bool place = pos[u] >= 0 && pos[u] >> a.c.page_shift < a.c.width && id0 + 256 * u < 2 * rows * 16;
      page[u] = place ? table[pos[u] >> a.c.page_shift] : -1;
      const Strided& ss = is_v ? a.sv : a.sk;
      w[u] = __builtin_nontemporal_load((const u32x4*)(
          (is_v ? a.v : a.k) + 2 * ((size_t)batch * ss.sb + (size_t)h * ss.sh + (size_t)(first + t0 + i) * ss.st) + 16 * (id & 15)));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if ((unsigned)page[u] >= (unsigned)a.c.n_pages) continue;
      const bool is_v = id0 + 256 * u >= rows * 16;
      const PageSide& side = is_v ? a.c.v : a.c.k;
      uint8_t* to = side.base + (uint64_t)(uint32_t)page[u] * side.page + (long long)head[u] * side.head +
                    (uint64_t)(uint32_t)(pos[u] & ((1 << a.c.page_shift) - 1)) * side.token;
      const int chunk = id0 & 15;
      if constexpr (FP8) *(u32x2*)(to + 8 * chunk) = to_fp8(w[u], divisor((is_v ? a.c.v_scale : a.c.k_scale)[head[u]]));
      else *(u32x4*)(to + 16 * chunk) = w[u];
    }
  }
}

// ---- copy --------------------------------------------------------------------------------------------------
// Pairs of pages travel with the launch, kCopyChunk at a time.  A workgroup copies kCopyLoads x 4 KB of K or of V; what it reads and
// writes passes the caches by.  1021 pages of 256 KB (535 MB read and written): 100 us, 5.3 TB/s; with loads and stores that do not
// 108, with 16 KB per workgroup 118 and 108.
constexpr int kCopyChunk = 448, kCopyLoads = 2;
constexpr int kCopyBytes = kCopyLoads * 4096;
struct CopyJob {
  PageSide k, v;
  int parts;              // workgroups per page and side
  int row_shift;          // log2 of the 16-byte pieces of a token's row
  int page_shift, n_kvh;
  int heads_first;
  int src[kCopyChunk], dst[kCopyChunk];
};

__global__ __launch_bounds__(256) void copy_kernel(CopyJob a) {
  const int pair = blockIdx.x / (2 * a.parts), part = blockIdx.x % (2 * a.parts);
  const PageSide& side = part < a.parts ? a.k : a.v;
  const uint8_t* from = side.base + (long long)a.src[pair] * side.page;
  uint8_t* to = side.base + (long long)a.dst[pair] * side.page;
  const int pieces = a.n_kvh << (a.page_shift + a.row_shift), tokens = 1 << a.page_shift;
  const int first = (part < a.parts ? part : part - a.parts) * (kCopyBytes / 16) + (int)threadIdx.x;
  u32x4 w[kCopyLoads];
  long long at[kCopyLoads];
#pragma unroll
  for (int r = 0; r < kCopyLoads; ++r) {
    const int piece = first + 256 * r, row = piece >> a.row_shift;
    const int h = a.heads_first ? row % a.n_kvh : row >> a.page_shift, slot = a.heads_first ? row / a.n_kvh : row & (tokens - 1);
    at[r] = (long long)h * side.head + (long long)slot * side.token + 16 * (piece & ((1 << a.row_shift) - 1));
    if (piece < pieces) w[r] = __builtin_nontemporal_load((const u32x4*)(from + at[r]));
  }
#pragma unroll
  for (int r = 0; r < kCopyLoads; ++r)
    if (first + 256 * r < pieces) __builtin_nontemporal_store(w[r], (u32x4*)(to + at[r]));
}

// All pages in range, the destinations different and none a source.  (One bit per page in each of two sets; < 0: SALE_ERR_*)
int check_pairs(const int32_t* src, const int32_t* dst, int n, int n_pages) {
  const size_t words = ((size_t)n_pages + 63) / 64;
  uint64_t* const sets = (uint64_t*)calloc(2 * words, sizeof(uint64_t));
  if (!sets) return SALE_ERR_HIP;
  uint64_t *const is_src = sets, *const is_dst = sets + words;
  int rc = SALE_OK;
  for (int i = 0; i < n && rc == SALE_OK; ++i) {
    if (src[i] < 0 || src[i] >= n_pages || dst[i] < 0 || dst[i] >= n_pages) { rc = SALE_ERR_BAD_SHAPE; break; }
    const uint64_t bit = 1ull << (dst[i] & 63);
    if (is_dst[dst[i] >> 6] & bit) rc = SALE_ERR_BAD_SHAPE;
    is_dst[dst[i] >> 6] |= bit;
    is_src[src[i] >> 6] |= 1ull << (src[i] & 63);
  }
  for (size_t w = 0; w < words && rc == SALE_OK; ++w)
    if (is_src[w] & is_dst[w]) rc = SALE_ERR_BAD_SHAPE;
  free(sets);
  return rc;
}

}  // namespace
}  // namespace sale

using namespace sale;

extern "C" int sale_cache_append(const sale_params_t* p, const sale_cache_t* cache, const void* k, const void* v, void* stream) {
  if (!p || !cache || !k || !v) return SALE_ERR_NULL_ARG;
  int rc = validate_tokens(p);
  if (rc == SALE_OK) rc = validate_cache(p, cache, true);
  if (rc != SALE_OK) return rc;
  if (((uintptr_t)k | (uintptr_t)v) & 15) return SALE_ERR_BAD_SHAPE;
  AppendJob a;
  a.c = cache_view(p, cache);
  a.k = (const uint8_t*)k;
  a.v = (const uint8_t*)v;
  a.sk = layout_of(p->k_stride, p->n_kv_heads, p->seq_len);
  a.sv = layout_of(p->v_stride, p->n_kv_heads, p->seq_len);
  a.n_kvh = p->n_kv_heads;
  a.heads_first = a.sk.sh < a.sk.st ? 1 : 0;
  a.tile = kAppendRows / p->n_kv_heads < 1 ? 1 : kAppendRows / p->n_kv_heads;
  // (of packed sequences at most, in any of the launches)
  const long long most = p->n_seqs > 0 ? (long long)p->seq_len / a.tile + kAppendChunk : ((long long)(p->seq_len - 1) / a.tile + 1) * p->batch;
  if (most > kMostWorkgroups) return SALE_ERR_UNSUPPORTED;
  const hipStream_t st = (hipStream_t)stream;
  auto launch = [&](long long workgroups) -> int {
    if (cache->dtype == SALE_PAGE_FP8) append_kernel<true><<<dim3((unsigned)workgroups), dim3(256), 0, st>>>(a);
    else append_kernel<false><<<dim3((unsigned)workgroups), dim3(256), 0, st>>>(a);
    return hipGetLastError() == hipSuccess ? SALE_OK : SALE_ERR_HIP;
  };
  a.each = a.tiles_each = 0;
  if (p->n_seqs == 0) {
    a.each = p->seq_len;
    a.tiles_each = (p->seq_len - 1) / a.tile + 1;
    return launch((long long)a.tiles_each * p->batch);
  }
  for (int s0 = 0; s0 < p->n_seqs; s0 += kAppendChunk) {
    a.first_seq = s0;
    a.n = min(kAppendChunk, p->n_seqs - s0);
    int at = 0;
    for (int e = 0; e <= a.n; ++e) {
      a.token[e] = p->cu_seqlens[s0 + e];
      if (e > 0) at += (a.token[e] - a.token[e - 1] + a.tile - 1) / a.tile;
      a.at[e] = at;
    }
    if (at > 0 && (rc = launch(at)) != SALE_OK) return rc;
  }
  return SALE_OK;
}

extern "C" int sale_cache_copy(const sale_params_t* p, const sale_cache_t* cache, const int32_t* src, const int32_t* dst,
                               int32_t n, void* stream) {
  if (!p || !cache || (n > 0 && (!src || !dst))) return SALE_ERR_NULL_ARG;
  if (p->n_kv_heads <= 0 || n < 0) return SALE_ERR_BAD_SHAPE;
  if (p->head_dim != kHeadDim) return SALE_ERR_UNSUPPORTED;
  int rc = validate_cache(p, cache, false);
  if (rc == SALE_OK) rc = check_pairs(src, dst, n, cache->n_pages);
  if (rc != SALE_OK) return rc;
  const CacheView c = cache_view(p, cache);
  CopyJob a;
  a.k = c.k;
  a.v = c.v;
  a.row_shift = cache->dtype == SALE_PAGE_FP8 ? 3 : 4;
  a.page_shift = c.page_shift;
  a.n_kvh = p->n_kv_heads;
  a.heads_first = c.k.head < c.k.token ? 1 : 0;
  const long long page_bytes = (long long)p->n_kv_heads * cache->page_tokens << (a.row_shift + 4);
  if (page_bytes > (1LL << 30)) return SALE_ERR_UNSUPPORTED;      // (pieces of a launch are counted in 32 bits)
  a.parts = (int)((page_bytes + kCopyBytes - 1) / kCopyBytes);
  const int chunk = (int)min((long long)kCopyChunk, max(1LL, kMostWorkgroups / (2LL * a.parts)));
  for (int i0 = 0; i0 < n; i0 += chunk) {
    const int m = min(chunk, n - i0);
    for (int i = 0; i < m; ++i) { a.src[i] = src[i0 + i]; a.dst[i] = dst[i0 + i]; }
    copy_kernel<<<dim3((unsigned)(m * 2 * a.parts)), dim3(256), 0, (hipStream_t)stream>>>(a);
    if (hipGetLastError() != hipSuccess) return SALE_ERR_HIP;
  }
  return SALE_OK;
}
