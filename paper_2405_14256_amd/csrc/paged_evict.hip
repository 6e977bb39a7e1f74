// zc_paged_evict: of every request the tokens that gathered the most weight, the newest and the first ones stay, and move to the
// front of the request's pages.
//
// Two launches (three where all heads take one choice): who stays, as an ascending list for each request and head, with the
// lengths and the pages that are left; then the rows, in place.  A token that stays never moves back: the i-th of the list lies at
// list[i] >= i.  So a wave that takes some channels of a (request, head) for itself may go through the list from its start, reading
// as far ahead as it likes, and needs no copy and no other wave: the place i that it fills was read by then, as the
// token there, if it stays, is the i-th of the list or one before.
#include "lds_dma.hpp"
#include "paged_args.hpp"

namespace zc {

struct EvictArgs {
  const uint8_t* from[2];                                // keys, values (the pools)
  uint8_t* to[2];
  float* scores;                                         // [page][head][row]
  int64_t sB[2], sH[2], sL[2];                           // bytes
  const int32_t *table, *kv_len, *keep;
  int64_t row;                                           // of the table, in entries
  int cols, shift, n_pages, cap, R, Hkv, heads;          // heads: lists of a request
  int64_t most;                                          // entries of a list
  int sinks, recent;
  int32_t *new_len, *kept, *free_pages, *n_freed;
  const int32_t* n_free;
  int64_t n_list;
  const float* sums;                                     // [R, cap], of all heads (null: every head by its own scores)
  int rowb, slice, lanes;                                // bytes of a row, of a wave's part of it; 16-byte pieces of that, as a shift
};

__device__ inline int tokens_of(const EvictArgs& a, int r) { return min(max(a.kv_len[r], 0), a.cap); }
__device__ inline int stay_of(const EvictArgs& a, int r, int kv) {
  const int keep = max(a.keep[r], 0);
  return min(kv, a.most < keep ? (int)a.most : keep);
}

// ---- one score of all heads ------------------------------------------------------------------------
// A thread a token: sums in 64 bits, rounded once (sums of 32 bits in another order would rank tokens of nearly equal weight
// differently).
__global__ __launch_bounds__(256) void k_evict_sums(EvictArgs a, float* sums) {
  const int r = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  const int kv = tokens_of(a, r);
  if (i >= kv || kv <= stay_of(a, r, kv)) return;
  const int id = a.table[r * a.row + (i >> a.shift)];
  double sum = 0.0;
  if ((uint32_t)id < (uint32_t)a.n_pages) {
    const float* s = a.scores + ((int64_t)id * a.Hkv << a.shift) + (i & ((1 << a.shift) - 1));
    for (int h = 0; h < a.Hkv; ++h) sum += (double)s[(int64_t)h << a.shift];
  }
  sums[(int64_t)r * a.cap + i] = (float)sum;
}

// ---- who stays ------------------------------------------------------------------------------------
// A workgroup a list.  The smallest score that stays is found digit by digit (11, 11 and 10 bits of the scores' order-preserving images)
// from histograms in LDS; then every thread counts what it has above and at that score, and a scan of the counts gives the places.
// A thread has consecutive tokens, so the list comes out in order and of equal scores the first ones stay.
constexpr int kPick = 1024, kEach = 8, kChunk = kPick * kEach, kBins = 2048;

// This thread's scores of chunk c, as order-preserving images (0: no candidate).
__device__ inline void images(const EvictArgs& a, int r, int h, int lo, int hi, int chunk, uint32_t (&x)[kEach]) {
  const int i0 = chunk * kChunk + threadIdx.x * kEach;
#pragma unroll
  for (int e = 0; e < kEach; ++e) x[e] = 0;
  if (i0 >= hi || i0 + kEach <= lo) return;
  float4 v[2] = {};
  if (a.sums) {
    const float* s = a.sums + (int64_t)r * a.cap + i0;   // (cap: whole pages)
    v[0] = reinterpret_cast<const float4*>(s)[0];
    v[1] = reinterpret_cast<const float4*>(s)[1];
  } else {
    const int id = a.table[r * a.row + (i0 >> a.shift)];
    if ((uint32_t)id < (uint32_t)a.n_pages) {
      const float* s = a.scores + (((int64_t)id * a.Hkv + h) << a.shift) + (i0 & ((1 << a.shift) - 1));
      v[0] = reinterpret_cast<const float4*>(s)[0];
      v[1] = reinterpret_cast<const float4*>(s)[1];
    }
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const float f = (&v[e >> 2].x)[e & 3];
    const int i = i0 + e;
    if (i >= lo && i < hi) x[e] = float_key(f + 0.f);    // (-0 ties with 0)
  }
}

// Inclusive sum over the workgroup.
__device__ inline int block_inclusive_sum(int v, int* waves) {
  const int w = threadIdx.x >> 6;
  v = wave_inclusive_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) waves[w] = v;
  __syncthreads();
  int before = 0;
  for (int u = 0; u < w; ++u) before += waves[u];
  return v + before;
}

__global__ __launch_bounds__(kPick) void k_evict_pick(EvictArgs a) {
  __shared__ int bins[kBins];
  __shared__ int waves[kPick / 64];
  __shared__ int s_digit, s_above, s_total;
  const int r = blockIdx.y, h = blockIdx.x, tid = threadIdx.x;
  const int kv = tokens_of(a, r), stay = stay_of(a, r, kv);

  if (h == 0) {
    if (tid == 0) a.new_len[r] = stay;
    if (a.free_pages || a.n_freed) {
      // pages that the requests in front of this one leave, and all of them
      int before = 0, all = 0;
      for (int q = tid; q < a.R; q += kPick) {
        const int n = tokens_of(a, q), left = stay_of(a, q, n);
        const int gone = (int)(((int64_t)n + (1 << a.shift) - 1) >> a.shift) - (int)(((int64_t)left + (1 << a.shift) - 1) >> a.shift);
        all += gone;
        if (q < r) before += gone;
      }
      before = block_inclusive_sum(before, waves);
      if (tid == kPick - 1) s_total = before;
      all = block_inclusive_sum(all, waves);
      if (r == 0 && tid == kPick - 1 && a.n_freed) *a.n_freed = all;
      const int64_t at = a.free_pages ? (int64_t)*a.n_free + s_total : 0;
      const int first = (int)(((int64_t)stay + (1 << a.shift) - 1) >> a.shift), last = (int)(((int64_t)kv + (1 << a.shift) - 1) >> a.shift);
      for (int c = first + tid; c < last; c += kPick)
        if (a.free_pages && at + c - first >= 0 && at + c - first < a.n_list) a.free_pages[at + c - first] = a.table[r * a.row + c];
    }
  }
  int32_t* list = a.kept + ((int64_t)r * a.heads + h) * a.most;
  if (stay == kv) {
    for (int i = tid; i < kv; i += kPick) list[i] = i;
    return;
  }
  const int recent = min(a.recent, stay), sinks = min(a.sinks, stay - recent);
  const int lo = sinks, hi = kv - recent, need = stay - recent - sinks;     // candidates, and how many of them stay
  const int chunks = (hi + kChunk - 1) / kChunk;
  uint32_t x[kEach];
  images(a, r, h, lo, hi, 0, x);

  // the least image that stays (`least`) and how many of its equals do (`ties`)
  uint32_t least = 0xffffffffu;
  int ties = 0;
  if (need > 0) {
    uint32_t prefix = 0;
    int rest = need;
    int shift = 32;
    for (int pass = 0; pass < 3; ++pass) {
      const int bits = pass < 2 ? 11 : 10, above_shift = shift;
      shift -= bits;
      for (int b = tid; b < kBins; b += kPick) bins[b] = 0;
      __syncthreads();
      for (int c = 0; c < chunks; ++c) {
        uint32_t y[kEach];
        if (c == 0) {
#pragma unroll
          for (int e = 0; e < kEach; ++e) y[e] = x[e];
        } else {
          images(a, r, h, lo, hi, c, y);
        }
        const int i0 = c * kChunk + tid * kEach;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const bool in = i0 + e >= lo && i0 + e < hi && (pass == 0 || (y[e] >> above_shift) == prefix);
          if (in) atomicAdd(&bins[(y[e] >> shift) & ((1u << bits) - 1)], 1);
        }
      }
      __syncthreads();
      // bins from the top: thread t has the two below the 2 t largest
      const int n = 1 << bits, top = n - 1 - 2 * tid;
      const int b0 = top >= 1 ? bins[top] : 0, b1 = top >= 1 ? bins[top - 1] : 0;
      const int upto = block_inclusive_sum(b0 + b1, waves), before = upto - b0 - b1;
      if (before < rest && upto >= rest) {
        const bool second = before + b0 < rest;
        s_digit = second ? top - 1 : top;
        s_above = second ? before + b0 : before;
      }
      __syncthreads();
      prefix = pass == 0 ? (uint32_t)s_digit : (prefix << bits) | (uint32_t)s_digit;
      rest -= s_above;
      __syncthreads();
    }
    least = prefix;
    ties = rest;
  }

  // the list: first tokens, those of the candidates that stay, newest tokens
  for (int i = tid; i < sinks; i += kPick) list[i] = i;
  for (int i = tid; i < recent; i += kPick) list[stay - recent + i] = kv - recent + i;
  if (need == 0) return;
  int placed = sinks, equal = 0;                           // so far, of the chunks before
  for (int c = 0; c < chunks; ++c) {
    if (c) images(a, r, h, lo, hi, c, x);
    const int i0 = c * kChunk + tid * kEach;
    int over = 0, same = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const bool in = i0 + e >= lo && i0 + e < hi;
      over += in && x[e] > least;
      same += in && x[e] == least;
    }
    const int same_upto = block_inclusive_sum(same, waves);
    const int first_same = equal + same_upto - same;       // equals in front of this thread's
    const int mine = over + min(max(ties - first_same, 0), same);
    const int upto = block_inclusive_sum(mine, waves);
    int at = placed + upto - mine, left = max(ties - first_same, 0);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const bool in = i0 + e >= lo && i0 + e < hi;
      const bool tie = in && x[e] == least && left > 0;
      left -= tie;
      if (tie || (in && x[e] > least)) list[at++] = i0 + e;
    }
    if (tid == kPick - 1) { s_digit = upto; s_above = same_upto; }
    __syncthreads();
    placed += s_digit;
    equal += s_above;
    __syncthreads();
  }
}

// ---- the rows -------------------------------------------------------------------------------------
typedef uint32_t piece16 __attribute__((ext_vector_type(4)));

// Where token i of request r lies, in a pool: page, row; page < 0: nowhere.
__device__ inline int page_at(const EvictArgs& a, int r, int i) {
  const int id = a.table[r * a.row + (i >> a.shift)];
  return (uint32_t)id < (uint32_t)a.n_pages ? id : -1;
}

// A wave takes `slice` bytes of every row of a (request, head, tensor), the waves of a workgroup the slices side by side.
constexpr int kMove = 8;                                  // rows a lane has on their way
__global__ __launch_bounds__(512) void k_evict_move(EvictArgs a) {
  const int r = blockIdx.z, lane = threadIdx.x & 63;
  const int kv = tokens_of(a, r), stay = stay_of(a, r, kv);
  if (stay == kv) return;
  const int head = blockIdx.y;                           // keys, values, scores of every head
  const int what = head / a.Hkv, h = head - what * a.Hkv;
  const int32_t* list = a.kept + ((int64_t)r * a.heads + (a.heads > 1 ? h : 0)) * a.most;
  const int inside = (1 << a.shift) - 1;
  if (what == 2) {
    if (blockIdx.x || threadIdx.x >= 64) return;
    for (int i0 = 0; i0 < stay; i0 += 64 * kMove) {
      float x[kMove];
      float* to[kMove];
#pragma unroll
      for (int u = 0; u < kMove; ++u) {
        const int i = i0 + 64 * u + lane;
        to[u] = nullptr;
        if (i < stay) {
          const int from = list[i], src = page_at(a, r, from), dst = page_at(a, r, i);
          x[u] = src >= 0 ? a.scores[(((int64_t)src * a.Hkv + h) << a.shift) + (from & inside)] : 0.f;
          if (dst >= 0 && from != i) to[u] = a.scores + (((int64_t)dst * a.Hkv + h) << a.shift) + (i & inside);
        }
      }
      wait_vmem<0>();
#pragma unroll
      for (int u = 0; u < kMove; ++u)
        if (to[u]) *to[u] = x[u];
    }
    return;
  }
  const int w = blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
  if (w * a.slice >= a.rowb) return;
  const int per = 64 >> a.lanes;                          // rows of a transfer
  const int64_t c = w * a.slice + (lane & ((1 << a.lanes) - 1)) * 16 + h * a.sH[what];
  const uint8_t* from_pool = a.from[what] + c;
  uint8_t* to_pool = a.to[what] + c;
  const int64_t sB = a.sB[what], sL = a.sL[what];
  for (int i0 = 0; i0 < stay; i0 += per * kMove) {
    piece16 x[kMove];
    uint8_t* to[kMove];
#pragma unroll
    for (int u = 0; u < kMove; ++u) {
      const int i = i0 + per * u + (lane >> a.lanes);
      to[u] = nullptr;
      x[u] = piece16{0, 0, 0, 0};
      if (i < stay) {
        const int from = list[i], src = page_at(a, r, from), dst = page_at(a, r, i);
        if (from != i && dst >= 0) {
          to[u] = to_pool + dst * sB + (i & inside) * sL;
          if (src >= 0) x[u] = *reinterpret_cast<const piece16*>(from_pool + src * sB + (from & inside) * sL);
        }
      }
    }
    wait_vmem<0>();
#pragma unroll
    for (int u = 0; u < kMove; ++u)
      if (to[u]) *reinterpret_cast<piece16*>(to[u]) = x[u];
  }
}

}  // namespace zc

using namespace zc;

__global__ void k_evict_none(int32_t* n_freed) { *n_freed = 0; }

extern "C" size_t zc_paged_evict_workspace(int64_t R, int64_t max_blocks, int64_t page, int32_t together) {
  if (!together || R <= 0 || max_blocks <= 0 || page <= 0 || R > 65535 || max_blocks > 0x7fff0000 / page) return 0;
  return (size_t)(R * max_blocks * page) * sizeof(float);
}

extern "C" int zc_paged_evict(const zc_tensor4* k_pages, const zc_tensor4* v_pages, float* scores, const int32_t* block_table, int64_t row_stride,
                              int64_t max_blocks, const int32_t* kv_len, const int32_t* keep, int64_t R, int64_t most, int32_t sinks,
                              int32_t recent, int32_t together, int32_t* new_len, int32_t* kept, int32_t* free_pages, int64_t n_list,
                              const int32_t* n_free, int32_t* n_freed, void* ws, size_t ws_bytes, void* stream) {
  const int rc = zc_validate_pages(k_pages, v_pages);
  if (rc) return rc;
  if (!zc_rows_apart(k_pages) || !zc_rows_apart(v_pages)) return ZC_ERR_INVALID_ARG;
  if (R < 0 || most < 0 || sinks < 0 || recent < 0 || n_list < 0 || max_blocks < 0 || row_stride < max_blocks) return ZC_ERR_INVALID_ARG;
  for (const void* p : {(const void*)block_table, (const void*)kv_len, (const void*)keep, (const void*)new_len, (const void*)kept,
                        (const void*)free_pages, (const void*)n_free, (const void*)n_freed})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ZC_ERR_INVALID_ARG;
  if (!scores || (reinterpret_cast<uintptr_t>(scores) & 15) || (free_pages && !n_free)) return ZC_ERR_INVALID_ARG;
  hipStream_t st = (hipStream_t)stream;
  if (R == 0) {
    if (n_freed) {
      hipLaunchKernelGGL(k_evict_none, dim3(1), dim3(1), 0, st, n_freed);
      ZC_LAUNCH_CHECK();
    }
    return ZC_OK;
  }
  if (!kv_len || !keep || !new_len || (most > 0 && !kept) || (max_blocks > 0 && !block_table)) return ZC_ERR_INVALID_ARG;
  const int64_t page = k_pages->L, H = k_pages->H;
  if (R > 65535 || 3 * H > 65535 || most > 0x7fffffff || max_blocks > 0x7fff0000 / page || n_list > 0x7fffffff) return ZC_ERR_UNSUPPORTED;
  for (const int32_t* p : {kv_len, keep})                // (lengths are read until the last launch)
    if (new_len < p + R && p < new_len + R) return ZC_ERR_INVALID_ARG;
  const size_t need = zc_paged_evict_workspace(R, max_blocks, page, together);
  if (need && (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 15))) return ZC_ERR_WORKSPACE;

  const int64_t eb = elem_bytes(k_pages->dtype);
  EvictArgs a;
  const zc_tensor4* pools[2] = {k_pages, v_pages};
  for (int i = 0; i < 2; ++i) {
    a.from[i] = a.to[i] = (uint8_t*)pools[i]->ptr;
    a.sB[i] = pools[i]->sB * eb; a.sH[i] = pools[i]->sH * eb; a.sL[i] = pools[i]->sL * eb;
  }
  a.scores = scores;
  a.table = block_table; a.kv_len = kv_len; a.keep = keep; a.row = row_stride;
  a.cols = (int)max_blocks; a.shift = __builtin_ctzll((unsigned long long)page); a.n_pages = (int)k_pages->B; a.cap = (int)(max_blocks * page);
  a.R = (int)R; a.Hkv = (int)H; a.heads = together ? 1 : (int)H;
  a.most = most; a.sinks = sinks; a.recent = recent;
  a.new_len = new_len; a.kept = kept; a.free_pages = free_pages; a.n_freed = n_freed; a.n_free = n_free; a.n_list = n_list;
  a.sums = nullptr;
  if (need) {
    hipLaunchKernelGGL(k_evict_sums, dim3((unsigned)ceil_div64(a.cap, 256), (unsigned)R), dim3(256), 0, st, a, (float*)ws);
    ZC_LAUNCH_CHECK();
    a.sums = (const float*)ws;
  }
  hipLaunchKernelGGL(k_evict_pick, dim3((unsigned)a.heads, (unsigned)R), dim3(kPick), 0, st, a);
  ZC_LAUNCH_CHECK();
  a.rowb = (int)(k_pages->D * eb);
  a.lanes = 2;
  a.slice = 16 << a.lanes;
  const int slices = a.rowb / a.slice, waves = slices < 8 ? slices : 8;
  hipLaunchKernelGGL(k_evict_move, dim3((unsigned)ceil_div(slices, waves), (unsigned)(3 * H), (unsigned)R), dim3(64 * waves), 0, st, a);
  ZC_LAUNCH_CHECK();
  return ZC_OK;
}
