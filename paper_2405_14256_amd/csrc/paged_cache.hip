// The paged full-precision cache around its attention: zc_paged_tables (block tables and slot maps of a step),
// zc_paged_store (a step's new keys and values into their slots), zc_paged_load (requests' pages as [B, H, L, D]
// tensors, which the compression reads).
#include <algorithm>

#include "paged_args.hpp"

namespace zc {

// ---- zc_paged_tables ----------------------------------------------------------------------------
// Request r holds kv tokens, the last q of them new; it had ceil((kv - q) / page) pages and needs ceil(kv / page).  Every
// page that it takes has one new token at its first slot, so the tokens are all the work there is: a thread per token finds
// its request among the sums of q (in LDS, 1024 requests at a time), its page - in the table if the request had it, else
// in the list of free pages - writes the slot and, at a page's first slot, the table.  Every workgroup takes the sums of
// all requests itself (8 bytes each, from the caches): workgroups exchange nothing.  Bound by the launch and two trips to memory, lengths and
// pages: 64 requests of one token 3.6 us, 256 requests of 181 000 4.6.
struct TableArgs {
  const int32_t *q_len, *kv_len;
  int R;
  int32_t* table;
  int64_t row;                  // of the table, in elements
  int cols, shift;
  const int32_t *free, *n_free;
  int F;
  int32_t* q_start;
  int32_t* slots;
  int64_t T, share;             // rows of the slot map, of a workgroup
  int half;                     // the search's first step: half of the requests' number, rounded up to a power of two
  int32_t* taken;
};

constexpr int kTabThreads = 256, kTabEach = 4, kTabReq = kTabThreads * kTabEach, kTabTokens = 4;

__global__ __launch_bounds__(kTabThreads) void k_paged_tables(TableArgs a) {
  __shared__ int s_start[kTabReq], s_page[kTabReq], s_past[kTabReq];
  __shared__ int s_sum[2][kTabThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n_free = min(max(a.n_free ? *a.n_free : a.F, 0), a.F);
  const int64_t t_lo = blockIdx.x * a.share, t_hi = min(t_lo + a.share, a.T);      // this workgroup's tokens
  int64_t start = 0;                                                    // tokens and pages of the requests before
  int page = 0;
  for (int r0 = 0; r0 < a.R; r0 += kTabReq) {
    int q[kTabEach], need[kTabEach], past[kTabEach], sq = 0, sn = 0;
#pragma unroll
    for (int i = 0; i < kTabEach; ++i) {
      const int r = r0 + tid * kTabEach + i;
      const int kv = r < a.R ? max(a.kv_len[r], 0) : 0;
      q[i] = r < a.R ? min(max(a.q_len[r], 0), kv) : 0;
      past[i] = kv - q[i];
      need[i] = (int)(((int64_t)kv + (1 << a.shift) - 1) >> a.shift) - (int)(((int64_t)past[i] + (1 << a.shift) - 1) >> a.shift);
      sq += q[i];
      sn += need[i];
    }
    const int iq = wave_inclusive_sum(sq), in = wave_inclusive_sum(sn);
    if (r0) __syncthreads();                                            // (the sums of the requests before are read)
    if (lane == 63) { s_sum[0][w] = iq; s_sum[1][w] = in; }
    __syncthreads();
    int bq = iq - sq, bn = in - sn, tq = 0, tn = 0;
#pragma unroll
    for (int v = 0; v < kTabThreads / 64; ++v) {
      bq += v < w ? s_sum[0][v] : 0;
      bn += v < w ? s_sum[1][v] : 0;
      tq += s_sum[0][v];
      tn += s_sum[1][v];
    }
#pragma unroll
    for (int i = 0; i < kTabEach; ++i) {
      const int x = tid * kTabEach + i;
      s_start[x] = bq;
      s_page[x] = bn;
      s_past[x] = past[i];
      if (blockIdx.x == 0 && r0 + x < a.R) a.q_start[r0 + x] = (int)(start + bq);
      bq += q[i];
      bn += need[i];
    }
    __syncthreads();
    // the tokens of these requests that are this workgroup's, four a thread at a time: their searches and their loads overlap
    const int64_t lo = max(t_lo, start), hi = min(t_hi, start + tq);
    for (int64_t t0 = lo + tid; t0 < hi; t0 += kTabTokens * kTabThreads) {
      int rel[kTabTokens], x[kTabTokens], id[kTabTokens], pos[kTabTokens];
      int32_t* entry[kTabTokens];
      bool mine[kTabTokens];
#pragma unroll
      for (int i = 0; i < kTabTokens; ++i) {
        const int64_t t = t0 + i * kTabThreads;
        mine[i] = t < hi;
        rel[i] = (int)((mine[i] ? t : t0) - start);
        x[i] = 0;
      }
      for (int b = a.half; b; b >>= 1)                                  // the last request that starts at or before the token: it has tokens
#pragma unroll
        for (int i = 0; i < kTabTokens; ++i)
          if (s_start[x[i] + b] <= rel[i]) x[i] += b;
#pragma unroll
      for (int i = 0; i < kTabTokens; ++i) {
        const int past = s_past[x[i]];
        pos[i] = past + rel[i] - s_start[x[i]];
        const int col = pos[i] >> a.shift, had = (int)(((int64_t)past + (1 << a.shift) - 1) >> a.shift);
        entry[i] = nullptr;
        id[i] = -1;
        if (mine[i] && (uint32_t)col < (uint32_t)a.cols) {
          int32_t* e = a.table + (int64_t)(r0 + x[i]) * a.row + col;
          const int64_t at = (int64_t)n_free - 1 - ((int64_t)page + s_page[x[i]] + col - had);
          if (col < had) id[i] = *e;
          else if (at >= 0 && at < n_free) id[i] = a.free[at];
          if (col >= had && (pos[i] & ((1 << a.shift) - 1)) == 0) entry[i] = e;
        }
      }
#pragma unroll
      for (int i = 0; i < kTabTokens; ++i) {
        if (entry[i]) *entry[i] = id[i];
        const int64_t slot = ((int64_t)id[i] << a.shift) + (pos[i] & ((1 << a.shift) - 1));
        if (mine[i]) a.slots[t0 + i * kTabThreads] = id[i] >= 0 && slot <= 0x7fffffff ? (int)slot : -1;
      }
    }
    start += tq;
    page += tn;
  }
  for (int64_t t = max(t_lo, start) + tid; t < t_hi; t += kTabThreads) a.slots[t] = -1;    // rows behind the last request
  if (blockIdx.x == 0 && tid == 0) {
    a.q_start[a.R] = (int)start;
    *a.taken = page;
  }
}

// 16 bytes that pass through once: stored without taking a place in the caches.
typedef uint32_t piece16 __attribute__((ext_vector_type(4)));
__device__ inline void put(uint8_t* to, piece16 x) { __builtin_nontemporal_store(x, reinterpret_cast<piece16*>(to)); }
__device__ inline piece16 get(const uint8_t* from) { return *reinterpret_cast<const piece16*>(from); }

// ---- zc_paged_store -------------------------------------------------------------------------------
struct StoreArgs {
  const uint8_t *k, *v;
  uint8_t *kp, *vp;
  const int32_t* slots;
  int64_t k_sH, k_sL, v_sH, v_sL;                       // bytes
  int64_t kp_sB, kp_sH, kp_sL, vp_sB, vp_sH, vp_sL;
  int64_t T, slots_n;
  int shift, cpr;                                       // 16-byte pieces of a row (a power of two), as a shift
  int pieces, wide, tokens;                             // pieces of a token (keys and values), of a workgroup; tokens of a pass
};

// A thread copies one 16-byte piece of UNROLL tokens: pieces of a token are consecutive threads, keys and then values.
// Bound by memory; the loads of all tokens are issued before the first store.  8066 tokens of 40 heads of 128 channels, fp16,
// pages of 32: 62 us (5.3 TB/s; 73 with stores through the caches, 105 with eight tokens a thread); 64 tokens 2.0 us.
template <int UNROLL>
__global__ __launch_bounds__(256) void k_paged_store(StoreArgs a) {
  const int piece = blockIdx.y * 256 + threadIdx.x % a.wide, first = threadIdx.x / a.wide;
  if (first >= a.tokens || piece >= a.pieces) return;
  const bool value = piece >= a.pieces / 2;
  const int p = value ? piece - a.pieces / 2 : piece;
  const int64_t h = p >> a.cpr;
  const int c = (p & ((1 << a.cpr) - 1)) * 16;
  const uint8_t* src = (value ? a.v + h * a.v_sH : a.k + h * a.k_sH) + c;
  uint8_t* dst = (value ? a.vp + h * a.vp_sH : a.kp + h * a.kp_sH) + c;
  const int64_t src_t = value ? a.v_sL : a.k_sL, dst_b = value ? a.vp_sB : a.kp_sB, dst_t = value ? a.vp_sL : a.kp_sL;
  const int64_t t0 = (int64_t)blockIdx.x * a.tokens * UNROLL + first;
  piece16 x[UNROLL];
  int slot[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const int64_t t = t0 + (int64_t)u * a.tokens;
    slot[u] = t < a.T ? a.slots[t] : -1;
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u)
    if (slot[u] >= 0 && slot[u] < a.slots_n) x[u] = get(src + (t0 + (int64_t)u * a.tokens) * src_t);
#pragma unroll
  for (int u = 0; u < UNROLL; ++u)
    if (slot[u] >= 0 && slot[u] < a.slots_n)
      put(dst + (slot[u] >> a.shift) * dst_b + (slot[u] & ((1 << a.shift) - 1)) * dst_t, x[u]);
}

// ---- zc_paged_load --------------------------------------------------------------------------------
struct LoadArgs {
  const uint8_t *kp, *vp;
  uint8_t *k, *v;
  const int32_t *table, *kv_len;
  int64_t row, n_pages;
  int cols, shift, cpr, L;
  int64_t k_sB, k_sH, k_sL, v_sB, v_sH, v_sL;           // bytes
  int64_t kp_sB, kp_sH, kp_sL, vp_sB, vp_sH, vp_sL;
};

// A workgroup copies 256 * UNROLL pieces of one head of one request.  Bound by memory: 16 requests of 3500 to 4096 tokens, 40 heads
// of 128 channels, fp16, 438 us (5.6 TB/s; 467 with stores through the caches), one of 4096 tokens, 8 heads, bf16, 6.4 us.
template <int UNROLL>
__global__ __launch_bounds__(256) void k_paged_load(LoadArgs a) {
  const int r = blockIdx.z >> 1, h = blockIdx.y;
  const bool value = blockIdx.z & 1;
  const int n = min(a.kv_len[r], a.L);                  // (L: at most what a row of the table has room for)
  const int rows = 256 >> a.cpr, i0 = blockIdx.x * rows * UNROLL + (threadIdx.x >> a.cpr);
  const int c = (threadIdx.x & ((1 << a.cpr) - 1)) * 16;
  const uint8_t* src = (value ? a.vp + h * a.vp_sH : a.kp + h * a.kp_sH) + c;
  uint8_t* dst = (value ? a.v + r * a.v_sB + h * a.v_sH : a.k + r * a.k_sB + h * a.k_sH) + c;
  const int64_t src_b = value ? a.vp_sB : a.kp_sB, src_t = value ? a.vp_sL : a.kp_sL, dst_t = value ? a.v_sL : a.k_sL;
  int id[UNROLL];
  piece16 x[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const int i = i0 + u * rows, col = i >> a.shift;
    id[u] = i < n && col < a.cols ? a.table[r * a.row + col] : -1;
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    x[u] = piece16{0, 0, 0, 0};
    if (id[u] >= 0 && id[u] < a.n_pages) x[u] = get(src + id[u] * src_b + ((i0 + u * rows) & ((1 << a.shift) - 1)) * src_t);
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u)
    if (i0 + u * rows < n) put(dst + (i0 + u * rows) * dst_t, x[u]);
}

}  // namespace zc

using namespace zc;

int zc_validate_pages(const zc_tensor4* k, const zc_tensor4* v) {
  int rc = zc_validate_tensor(k);
  if (rc) return rc;
  rc = zc_validate_tensor(v);
  if (rc) return rc;
  if (k->dtype != v->dtype || k->B != v->B || k->H != v->H || k->L != v->L || k->D != v->D) return ZC_ERR_INVALID_ARG;
  if (k->L < ZC_PAGE_MIN || k->L > ZC_PAGE_MAX || (k->L & (k->L - 1))) return ZC_ERR_UNSUPPORTED;
  const int64_t eb = elem_bytes(k->dtype);
  if (k->B > 0x7fffffff / k->L || k->H > 65535) return ZC_ERR_UNSUPPORTED;
  if (k->sB < 0 || k->sH < 0 || v->sB < 0 || v->sH < 0) return ZC_ERR_INVALID_ARG;
  // offsets inside a head's rows of a page, and from a page to the next, have 32 bits
  for (const zc_tensor4* t : {k, v})
    if (t->sL > 0x7fffffff / (eb * t->L) || t->sB > 0xffffffff / eb) return ZC_ERR_UNSUPPORTED;
  return ZC_OK;
}

// Rows of new tokens [1, any number of heads, T, D] beside the pages.
int zc_validate_heads(const zc_tensor4* x, const zc_tensor4* pages) {
  if (!x) return ZC_ERR_INVALID_ARG;
  zc_tensor4 t = *x;
  if (t.L == 0 && !t.ptr) t.ptr = pages->ptr;            // (no tokens: a tensor without memory is one)
  const int rc = zc_validate_tensor(&t);
  if (rc) return rc;
  if (x->B != 1 || x->dtype != pages->dtype || x->D != pages->D || x->sH < 0) return ZC_ERR_INVALID_ARG;
  return ZC_OK;
}
bool zc_rows_apart(const zc_tensor4* x) {
  if (x->B == 0 || x->H == 0 || x->L == 0) return true;
  struct Axis { int64_t n, stride; } axes[3] = {{x->B, x->sB}, {x->H, x->sH}, {x->L, x->sL}};
  std::sort(axes, axes + 3, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
  __int128 span = x->D;
  for (const Axis& a : axes) {
    if (a.n <= 1) continue;
    if (a.stride < span) return false;
    span += (__int128)(a.n - 1) * a.stride;
  }
  return true;
}
static int validate_rows(const zc_tensor4* x, const zc_tensor4* pages) {
  const int rc = zc_validate_heads(x, pages);
  return rc ? rc : x->H != pages->H ? ZC_ERR_INVALID_ARG : ZC_OK;
}

extern "C" int zc_paged_tables(const int32_t* q_len, const int32_t* kv_len, int64_t R, int32_t* block_table, int64_t row_stride,
                               int64_t max_blocks, const int32_t* free_pages, int64_t n_list, const int32_t* n_free, int64_t page,
                               int32_t* q_start, int32_t* slot_map, int64_t T, int32_t* n_taken, void* stream) {
  if (R < 0 || T < 0 || n_list < 0 || max_blocks < 0 || row_stride < max_blocks) return ZC_ERR_INVALID_ARG;
  if (page < ZC_PAGE_MIN || page > ZC_PAGE_MAX || (page & (page - 1))) return ZC_ERR_UNSUPPORTED;
  if (!q_start || !n_taken || (T > 0 && !slot_map) || (n_list > 0 && !free_pages)) return ZC_ERR_INVALID_ARG;
  if (R > 0 && (!q_len || !kv_len || (max_blocks > 0 && !block_table))) return ZC_ERR_INVALID_ARG;
  for (const void* p : {(const void*)q_len, (const void*)kv_len, (const void*)block_table, (const void*)free_pages, (const void*)n_free,
                        (const void*)q_start, (const void*)slot_map, (const void*)n_taken})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ZC_ERR_INVALID_ARG;
  if (R > 0x7fffffff - 2 * kTabReq || T > 0x7fffffff || max_blocks > 0x7fffffff || n_list > 0x7fffffff) return ZC_ERR_UNSUPPORTED;
  TableArgs a;
  a.q_len = q_len; a.kv_len = kv_len; a.R = (int)R;
  a.table = block_table; a.row = row_stride; a.cols = (int)max_blocks; a.shift = __builtin_ctzll((unsigned long long)page);
  a.free = free_pages; a.n_free = n_free; a.F = (int)n_list;
  a.q_start = q_start; a.slots = slot_map; a.T = T; a.taken = n_taken;
  a.half = 0;
  while (2 * a.half < R && 2 * a.half < kTabReq) a.half = a.half ? 2 * a.half : 1;
  int64_t wgs = ceil_div64(T, kTabTokens * kTabThreads);
  wgs = wgs < 1 ? 1 : wgs > 2048 ? 2048 : wgs;
  a.share = ceil_div64(T, wgs);
  hipLaunchKernelGGL(k_paged_tables, dim3((unsigned)wgs), dim3(kTabThreads), 0, (hipStream_t)stream, a);
  ZC_LAUNCH_CHECK();
  return ZC_OK;
}

extern "C" int zc_paged_store(const zc_tensor4* k, const zc_tensor4* v, const int32_t* slot_map, const zc_tensor4* k_pages,
                              const zc_tensor4* v_pages, void* stream) {
  int rc = zc_validate_pages(k_pages, v_pages);
  if (rc) return rc;
  rc = validate_rows(k, k_pages);
  if (rc) return rc;
  rc = validate_rows(v, v_pages);
  if (rc) return rc;
  if (k->L != v->L) return ZC_ERR_INVALID_ARG;
  if (k->L == 0) return ZC_OK;
  if (!slot_map || (reinterpret_cast<uintptr_t>(slot_map) & 3) || !zc_rows_apart(k_pages) || !zc_rows_apart(v_pages)) return ZC_ERR_INVALID_ARG;
  const int64_t eb = elem_bytes(k->dtype), rowb = k->D * eb;
  StoreArgs a;
  a.k = (const uint8_t*)k->ptr; a.v = (const uint8_t*)v->ptr; a.kp = (uint8_t*)k_pages->ptr; a.vp = (uint8_t*)v_pages->ptr;
  a.slots = slot_map;
  a.k_sH = k->sH * eb; a.k_sL = k->sL * eb; a.v_sH = v->sH * eb; a.v_sL = v->sL * eb;
  a.kp_sB = k_pages->sB * eb; a.kp_sH = k_pages->sH * eb; a.kp_sL = k_pages->sL * eb;
  a.vp_sB = v_pages->sB * eb; a.vp_sH = v_pages->sH * eb; a.vp_sL = v_pages->sL * eb;
  a.T = k->L; a.slots_n = k_pages->B * k_pages->L;
  a.shift = __builtin_ctzll((unsigned long long)k_pages->L);
  a.cpr = __builtin_ctzll((unsigned long long)(rowb / 16));
  a.pieces = (int)(2 * k->H << a.cpr);
  a.wide = a.pieces < 256 ? a.pieces : 256;
  a.tokens = 256 / a.wide;
  const int64_t cols = ceil_div64(a.pieces, 256), passes = ceil_div64(a.T, a.tokens);
  const bool many = passes * cols >= 4096;
  const int64_t wgs = many ? ceil_div64(passes, 4) : passes;
  if (wgs > 0xffffff || cols > 65535) return ZC_ERR_UNSUPPORTED;
  hipStream_t st = (hipStream_t)stream;
  if (many) hipLaunchKernelGGL(k_paged_store<4>, dim3((unsigned)wgs, (unsigned)cols), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_paged_store<1>, dim3((unsigned)wgs, (unsigned)cols), dim3(256), 0, st, a);
  ZC_LAUNCH_CHECK();
  return ZC_OK;
}

extern "C" int zc_paged_load(const zc_tensor4* k_pages, const zc_tensor4* v_pages, const int32_t* block_table, int64_t row_stride,
                             int64_t max_blocks, const int32_t* kv_len, const zc_tensor4* k, const zc_tensor4* v, void* stream) {
  int rc = zc_validate_pages(k_pages, v_pages);
  if (rc) return rc;
  if (k && v && k->B == v->B && k->L == v->L && (k->B == 0 || k->L == 0)) return ZC_OK;
  rc = zc_validate_tensor(k);
  if (rc) return rc;
  rc = zc_validate_tensor(v);
  if (rc) return rc;
  if (k->dtype != k_pages->dtype || v->dtype != k->dtype || k->D != k_pages->D || v->D != k->D || k->H != k_pages->H || v->H != k->H ||
      k->B != v->B || k->L != v->L || k->sB < 0 || k->sH < 0 || v->sB < 0 || v->sH < 0 || !zc_rows_apart(k) || !zc_rows_apart(v))
    return ZC_ERR_INVALID_ARG;
  if (max_blocks < 0 || row_stride < max_blocks) return ZC_ERR_INVALID_ARG;
  if (!kv_len || (reinterpret_cast<uintptr_t>(kv_len) & 3) || (max_blocks > 0 && !block_table) || (reinterpret_cast<uintptr_t>(block_table) & 3))
    return ZC_ERR_INVALID_ARG;
  if (k->B > 32767 || k->L > (1 << 28) || max_blocks > 0x7fffffff) return ZC_ERR_UNSUPPORTED;
  const int64_t eb = elem_bytes(k->dtype), rowb = k->D * eb;
  LoadArgs a;
  a.k = (uint8_t*)k->ptr; a.v = (uint8_t*)v->ptr; a.kp = (const uint8_t*)k_pages->ptr; a.vp = (const uint8_t*)v_pages->ptr;
  a.table = block_table; a.kv_len = kv_len; a.row = row_stride; a.cols = (int)max_blocks; a.n_pages = k_pages->B;
  a.shift = __builtin_ctzll((unsigned long long)k_pages->L);
  a.cpr = __builtin_ctzll((unsigned long long)(rowb / 16));
  a.L = (int)(max_blocks < ceil_div64(k->L, k_pages->L) ? max_blocks * k_pages->L : k->L);
  if (a.L == 0) return ZC_OK;
  a.k_sB = k->sB * eb; a.k_sH = k->sH * eb; a.k_sL = k->sL * eb; a.v_sB = v->sB * eb; a.v_sH = v->sH * eb; a.v_sL = v->sL * eb;
  a.kp_sB = k_pages->sB * eb; a.kp_sH = k_pages->sH * eb; a.kp_sL = k_pages->sL * eb;
  a.vp_sB = v_pages->sB * eb; a.vp_sH = v_pages->sH * eb; a.vp_sL = v_pages->sL * eb;
  const int rows = 256 >> a.cpr;
  const bool many = ceil_div64(a.L, rows) * k->H * k->B * 2 >= 4096;
  const int64_t wgs = ceil_div64(a.L, many ? 2 * rows : rows);
  if (wgs > 0xffffff) return ZC_ERR_UNSUPPORTED;         // (a grid counts the threads of a dimension in 32 bits)
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid((unsigned)wgs, (unsigned)k->H, (unsigned)(2 * k->B));
  if (many) hipLaunchKernelGGL(k_paged_load<2>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_paged_load<1>, grid, dim3(256), 0, st, a);
  ZC_LAUNCH_CHECK();
  return ZC_OK;
}
