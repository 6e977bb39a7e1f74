// zc_paged_evict: of every request the tokens that gathered the most weight, the newest and the first ones stay, and move to the
// front of the request's pages.
//
// Two launches (three where all heads take one choice, one for short lists): who stays, as an ascending list for each request
// and head, with the lengths and the pages that are left; then the rows, in place.  A token that stays never moves back: the
// i-th of the list lies at list[i] >= i.  So a workgroup that takes some channels of a (request, head) for itself may go
// through the list from its start, reading as far ahead as it likes, and needs no copy and no other workgroup: the place i
// that it fills was read by then, as the token there, if it stays, is the i-th of the list or one before.
#include <limits.h>

#include "lds_dma.hpp"
#include "paged_args.hpp"

namespace zc {

struct EvictArgs {
  uint8_t* pool[2];                                      // keys, values
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
  int* moved;                                            // [R, heads], the first of a list that lies elsewhere than it will
  int rowb, slice, lanes;                                // bytes of a row, of a workgroup's part of it; 16-byte pieces of that, as a shift
};

__device__ inline int tokens_of(const EvictArgs& a, int r) { return min(max(a.kv_len[r], 0), a.cap); }
__device__ inline int stay_of(const EvictArgs& a, int r, int kv) {
  const int keep = max(a.keep[r], 0);
  return min(kv, a.most < keep ? (int)a.most : keep);
}

// ---- one score of all heads ------------------------------------------------------------------------
// A thread four tokens: sums in 64 bits, rounded once (sums of 32 bits in another order would rank tokens of nearly equal weight
// differently).  Bound by latency: 16 requests of 4096, 40 heads, 10 MB, 7.2 us.
__global__ __launch_bounds__(64) void k_evict_sums(EvictArgs a, float* sums) {
  const int r = blockIdx.y, i = (blockIdx.x * 64 + threadIdx.x) * 4;
  const int kv = tokens_of(a, r);
  if (i >= kv || kv <= stay_of(a, r, kv)) return;
  const int id = a.table[r * a.row + (i >> a.shift)];
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  if ((uint32_t)id < (uint32_t)a.n_pages) {
    const float* s = a.scores + ((int64_t)id * a.Hkv << a.shift) + (i & ((1 << a.shift) - 1));
    constexpr int U = 8;
    for (int h0 = 0; h0 < a.Hkv; h0 += U) {
      float4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = h0 + u < a.Hkv ? *reinterpret_cast<const float4*>(s + ((int64_t)(h0 + u) << a.shift)) : float4{};
#pragma unroll
      for (int u = 0; u < U; ++u) { sum[0] += x[u].x; sum[1] += x[u].y; sum[2] += x[u].z; sum[3] += x[u].w; }
    }
  }
  *reinterpret_cast<float4*>(sums + (int64_t)r * a.cap + i) = make_float4((float)sum[0], (float)sum[1], (float)sum[2], (float)sum[3]);
}

// ---- who stays ------------------------------------------------------------------------------------
// A workgroup a list.  The smallest score that stays is found digit by digit (11, 11 and 10 bits of the scores' order-preserving images)
// from histograms in LDS, until every score with the digits so far stays; then every thread counts what it has above and at that score, and
// a scan of the counts gives the places.  A thread has consecutive tokens, so the list comes out in order and of equal scores the
// first ones stay.  Bound by latency: a trip to the table, one to the scores, a barrier or two a digit (10 bits spare a fourth digit, which
// 8 would need); 8 lists of 4096 6.5 us, 256 of up to 8192 10.3, of 131072 121 (every sweep reads again what does not fit the registers).
constexpr int kEach = 4, kBins = 2048;

// A thread's scores of four tokens from i0 on, as order-preserving images.  id: the page of i0.
struct Images { uint32_t x[kEach]; };
__device__ inline Images images(const EvictArgs& a, int r, int h, int i0, int hi, int id) {
  float4 v = {};
  const bool page = (uint32_t)id < (uint32_t)a.n_pages;
  if (i0 < hi && (a.sums || page)) {
    const float* s = a.sums ? a.sums + (int64_t)r * a.cap + i0       // (cap: whole pages)
                            : a.scores + (((int64_t)id * a.Hkv + h) << a.shift) + (i0 & ((1 << a.shift) - 1));
    v = *reinterpret_cast<const float4*>(s);
  }
  Images m;
#pragma unroll
  for (int e = 0; e < kEach; ++e) m.x[e] = float_key((&v.x)[e] + 0.f);      // (-0 ties with 0)
  return m;
}
__device__ inline int page_of(const EvictArgs& a, int r, int i) { return a.cols ? a.table[r * a.row + min(i >> a.shift, a.cols - 1)] : -1; }

// Pages that requests leave: where each one's go in the list of free ones.  A workgroup a request.
template <int THREADS>
__device__ void give_back(const EvictArgs& a, int r, int kv, int stay, int (*waves)[THREADS / 64]) {
  const int tid = threadIdx.x;
  if (tid == 0) a.new_len[r] = stay;
  if (!a.free_pages && !a.n_freed) return;
  const auto pages = [&](int n) { return (int)(((int64_t)n + (1 << a.shift) - 1) >> a.shift); };
  int before = 0, all = 0;                                 // of the requests in front of this one, and of all
  for (int q = tid; q < a.R; q += THREADS) {
    const int n = tokens_of(a, q), gone = pages(n) - pages(stay_of(a, q, n));
    all += gone;
    if (q < r) before += gone;
  }
  int total_before, total;
  block_inclusive_sum<THREADS / 64>(before, waves[0], total_before);
  block_inclusive_sum<THREADS / 64>(all, waves[1], total);
  if (r == 0 && tid == 0 && a.n_freed) *a.n_freed = total;
  if (!a.free_pages) return;
  const int first = pages(stay), last = pages(kv);
  const int64_t at = (int64_t)*a.n_free + total_before - first;
  for (int c = first + tid; c < last; c += THREADS)
    if (at + c >= 0 && at + c < a.n_list) a.free_pages[at + c] = a.table[r * a.row + c];
}

template <int THREADS>
struct PickMemory {
  int bins[3][kBins];
  int waves[5][THREADS / 64];
  int digit[3], above[3], count[3], moved;
};

// The list of a request and head, in memory and for `also`; the first place of it whose token lies elsewhere, `stay` at most.
// HELD: chunks of kEach tokens a thread that it holds; scores behind them are read again in every sweep.  id: the pages of
// those it holds.
template <int THREADS, int HELD, typename F>
__device__ __forceinline__ int pick(const EvictArgs& a, int r, int h, int kv, int stay, const int (&id)[HELD], PickMemory<THREADS>& s, F&& also) {
  constexpr int NW = THREADS / 64, CHUNK = THREADS * kEach, PER = kBins / THREADS;
  auto& bins = s.bins;
  auto& waves = s.waves;
  const int tid = threadIdx.x;
  int32_t* const kept = a.kept + ((int64_t)r * a.heads + h) * a.most;
  const auto put = [&](int at, int i) {
    kept[at] = i;
    also(at, i);
  };
  if (stay == kv) {
    for (int i = tid; i < kv; i += THREADS) kept[i] = i;
    return stay;
  }
  const int recent = min(a.recent, stay), sinks = min(a.sinks, stay - recent);
  const int lo = sinks, hi = kv - recent, need = stay - recent - sinks;     // candidates, and how many of them stay
  const int chunks = (int)(((int64_t)hi + CHUNK - 1) / CHUNK);
  for (int i = tid; i < sinks; i += THREADS) put(i, i);
  for (int i = tid; i < recent; i += THREADS) put(stay - recent + i, kv - recent + i);
  if (need == 0) return sinks;
  if (tid == 0) s.moved = stay - recent;
  Images held[HELD];
#pragma unroll
  for (int c = 0; c < HELD; ++c) held[c] = images(a, r, h, c * CHUNK + tid * kEach, hi, id[c]);
  // f(first token, images) of every chunk
  const auto sweep = [&](auto&& f) {
#pragma unroll
    for (int c = 0; c < HELD; ++c)
      if (c < chunks) f(c * CHUNK + tid * kEach, held[c]);
    if (chunks <= HELD) return;
    // (one chunk's scores and the next one's pages are on their way meanwhile)
    int i0 = HELD * CHUNK + tid * kEach;
    Images next = images(a, r, h, i0, hi, page_of(a, r, i0));
    int ahead = page_of(a, r, i0 + CHUNK);
    for (int c = HELD; c < chunks; ++c, i0 += CHUNK) {
      const Images m = next;
      next = images(a, r, h, i0 + CHUNK, hi, ahead);
      ahead = page_of(a, r, i0 + 2 * CHUNK);
      f(i0, m);
    }
  };
  const auto candidate = [&](int i) { return i >= lo && i < hi; };

  for (int b = tid; b < 3 * kBins / 4; b += THREADS) reinterpret_cast<int4*>(bins)[b] = make_int4(0, 0, 0, 0);
  __syncthreads();
  // What is above `least` stays, and the first `ties` of its equals.
  uint32_t prefix = 0, least = 0;
  int ties = need;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass < 2 ? 11 : 10, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    sweep([&](int i0, const Images& m) {
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (candidate(i0 + e) && (pass == 0 || m.x[e] >> (shift + bits) == prefix)) atomicAdd(&bins[pass][(m.x[e] >> shift) & ((1 << bits) - 1)], 1);
    });
    __syncthreads();
    // from the top: thread t has the PER bins below the PER t largest
    const int top = (1 << bits) - 1 - PER * tid;
    int n[PER], sum = 0, all;
#pragma unroll
    for (int b = 0; b < PER; ++b) {
      n[b] = top - b >= 0 ? bins[pass][top - b] : 0;
      sum += n[b];
    }
    int above = block_inclusive_sum<NW>(sum, waves[pass], all) - sum;
    if (above < ties && above + sum >= ties) {
      int b = 0;
#pragma unroll
      for (int v = 0; v < PER - 1; ++v)
        if (b == v && above + n[v] < ties) { above += n[v]; ++b; }
      int count = 0;
#pragma unroll
      for (int v = 0; v < PER; ++v) count = b == v ? n[v] : count;
      s.digit[pass] = top - b;
      s.above[pass] = above;
      s.count[pass] = count;
    }
    __syncthreads();
    prefix = pass == 0 ? (uint32_t)s.digit[pass] : prefix << bits | (uint32_t)s.digit[pass];
    ties -= s.above[pass];
    least = prefix << shift;
    if (pass < 2 && s.count[pass] == ties && least > 0) {  // (all of them stay)
      --least;
      ties = 0;
      break;
    }
  }

  int placed = sinks, equal = 0;                           // of the chunks before
  int moved = INT_MAX;                                     // the first of this wave's that moves
  sweep([&](int i0, const Images& m) {
    int over = 0, same = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      over += candidate(i0 + e) && m.x[e] > least;
      same += candidate(i0 + e) && m.x[e] == least;
    }
    int all_same, all_mine;
    int left = max(ties - equal - (block_inclusive_sum<NW>(same, waves[3], all_same) - same), 0);      // equals that stay from this thread's first on
    const int mine = over + min(left, same);
    int at = placed + block_inclusive_sum<NW>(mine, waves[4], all_mine) - mine, first = INT_MAX;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const bool tie = candidate(i0 + e) && m.x[e] == least && left > 0;
      left -= tie;
      if (tie || (candidate(i0 + e) && m.x[e] > least)) {
        if (at != i0 + e) first = min(first, at);
        put(at++, i0 + e);
      }
    }
    equal += all_same;
    placed += all_mine;
    const uint64_t any = __builtin_amdgcn_ballot_w64(first != INT_MAX);          // (places ascend with the lanes, and with the chunks)
    if (any && moved == INT_MAX) moved = __builtin_amdgcn_readlane(first, __builtin_ctzll(any));
  });
  if ((tid & 63) == 0 && moved != INT_MAX) atomicMin(&s.moved, moved);
  __syncthreads();
  return s.moved;
}

template <int THREADS, int HELD>
__device__ inline void first_pages(const EvictArgs& a, int r, int (&id)[HELD]) {
#pragma unroll
  for (int c = 0; c < HELD; ++c) id[c] = page_of(a, r, c * THREADS * kEach + threadIdx.x * kEach);
}

template <int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void k_evict_pick(EvictArgs a) {
  __shared__ __align__(16) PickMemory<THREADS> s;
  const int r = blockIdx.y, h = blockIdx.x;
  int id[HELD];
  first_pages<THREADS>(a, r, id);
  const int kv = tokens_of(a, r), stay = stay_of(a, r, kv);
  if (h == a.heads) {                                      // (beside the heads')
    give_back<THREADS>(a, r, kv, stay, s.waves);
    return;
  }
  const int moved = pick<THREADS, HELD>(a, r, h, kv, stay, id, s, [](int, int) {});
  if (threadIdx.x == 0) a.moved[r * a.heads + h] = moved;
}

// ---- the rows -------------------------------------------------------------------------------------
typedef uint32_t piece16 __attribute__((ext_vector_type(4)));

// The slot of token i of request r (< 0: none).
__device__ inline int slot_at(const EvictArgs& a, int r, int i) {
  const int id = a.table[r * a.row + (i >> a.shift)];
  return (uint32_t)id < (uint32_t)a.n_pages ? id << a.shift | (i & ((1 << a.shift) - 1)) : -1;
}

// A workgroup takes `slice` bytes of every row of a (request, head, tensor), a row's by consecutive threads, kMove rows a
// thread at a time: all of them are read before the first is stored.  Where the next ones lie is looked up meanwhile.  Bound
// by memory where lists are many (16 requests, 1024 of up to 4096, 40 heads of 128 channels 131 us, 5.1 TB/s; 32 ragged ones
// of 8 heads, fewer than half as many workgroups, 67 us, 3.8 TB/s: a step waits for its rows and for the stores of the step
// before, and nothing is on its way meanwhile), by a step's trips where they are few (one such request of 8 heads 9.2).
constexpr int kMove = 4;
struct Move { int src, dst; };                           // slots (src < 0: zeros, dst < 0: nothing to do)

template <int THREADS>
__global__ __launch_bounds__(THREADS, 4) void k_evict_move(EvictArgs a) {
  const int r = blockIdx.z;
  const int kv = tokens_of(a, r), stay = stay_of(a, r, kv);
  if (stay == kv) return;
  const int what = blockIdx.x / a.Hkv, h = blockIdx.x - what * a.Hkv;          // keys, values, scores of every head
  if (what == 2 && blockIdx.y) return;
  const int32_t* list = a.kept + ((int64_t)r * a.heads + (a.heads > 1 ? h : 0)) * a.most;
  const int inside = (1 << a.shift) - 1, lanes = what == 2 ? 0 : a.lanes;
  const int per = THREADS >> lanes, first = threadIdx.x >> lanes;         // rows of a transfer
  // Three steps of the way are under way at a time: the list's entries, their pages, the rows.
  int next[kMove];
  Move m[kMove], ahead[kMove];
  const auto entries = [&](int i0) {
#pragma unroll
    for (int u = 0; u < kMove; ++u) {
      const int i = i0 + per * u + first;
      next[u] = i < stay ? list[i] : i;
    }
  };
  const auto find = [&](int i0, Move (&x)[kMove]) {
#pragma unroll
    for (int u = 0; u < kMove; ++u) {
      const int i = i0 + per * u + first;
      x[u] = {-1, -1};
      if (next[u] != i) x[u] = {slot_at(a, r, next[u]), slot_at(a, r, i)};
    }
  };
  const int step = per * kMove, begin = a.moved[r * a.heads + (a.heads > 1 ? h : 0)];       // (what is in front of it stays where it is)
  if (begin >= stay) return;
  entries(begin);
  find(begin, m);
  entries(begin + step);
  if (what == 2) {
    const auto at = [&](int slot) { return a.scores + (((int64_t)(slot >> a.shift) * a.Hkv + h) << a.shift) + (slot & inside); };
    for (int i0 = begin; i0 < stay; i0 += step) {
      float x[kMove];
      find(i0 + step, ahead);
#pragma unroll
      for (int u = 0; u < kMove; ++u) x[u] = m[u].src >= 0 ? *at(m[u].src) : 0.f;
      entries(i0 + 2 * step);
      wait_vmem<0>();
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kMove; ++u) {
        if (m[u].dst >= 0) *at(m[u].dst) = x[u];
        m[u] = ahead[u];
      }
    }
    return;
  }
  uint8_t* pool = a.pool[what] + blockIdx.y * a.slice + (threadIdx.x & ((1 << lanes) - 1)) * 16 + h * a.sH[what];
  const int64_t sB = a.sB[what], sL = a.sL[what];
  const auto at = [&](int slot) { return reinterpret_cast<piece16*>(pool + (slot >> a.shift) * sB + (slot & inside) * sL); };
  for (int i0 = begin; i0 < stay; i0 += step) {
    piece16 x[kMove];
    find(i0 + step, ahead);
#pragma unroll
    for (int u = 0; u < kMove; ++u) {
      x[u] = piece16{0, 0, 0, 0};
      if (m[u].src >= 0) x[u] = *at(m[u].src);
    }
    entries(i0 + 2 * step);
    wait_vmem<0>();
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kMove; ++u) {
      if (m[u].dst >= 0) *at(m[u].dst) = x[u];
      m[u] = ahead[u];
    }
  }
}

// ---- short lists: who stays and their rows in one launch ---------------------------------------------
// A list whose rows a workgroup takes in one step: it moves what it has chosen.  All rows are read before the first is
// stored.  Bound by latency.  us of two launches and this one: 16 requests of 30 to 250, 64 stay (8 heads of 128 channels,
// bf16) 15.0 and 12.3, 64 of 100 to 900, 200 stay 30.0 and 23.8, 37 of 20, 10 stay (40 heads) 21.4 and 14.7, 64 of 600 to
// 3000, 500 stay (64 channels) 48.6 and 37.5, 64 of 3000 to 8192, 128 stay 43.9 and 38.0.
template <int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void k_evict_short(EvictArgs a) {
  __shared__ __align__(16) PickMemory<THREADS> s;
  __shared__ int list[kMove * THREADS / 8];                // (a row has 8 pieces or more)
  const int r = blockIdx.y, h = blockIdx.x;
  int id[HELD];
  first_pages<THREADS>(a, r, id);
  const int kv = tokens_of(a, r), stay = stay_of(a, r, kv);
  if (h == a.heads) {
    give_back<THREADS>(a, r, kv, stay, s.waves);
    return;
  }
  const int begin = pick<THREADS, HELD>(a, r, h, kv, stay, id, s, [&](int at, int i) { list[at] = i; });
  if (begin >= stay) return;
  __syncthreads();
  const int inside = (1 << a.shift) - 1, per = THREADS >> a.lanes, first = threadIdx.x >> a.lanes;
  const auto row = [&](int what, int slot) {
    return reinterpret_cast<piece16*>(a.pool[what] + (threadIdx.x & ((1 << a.lanes) - 1)) * 16 + h * a.sH[what] + (slot >> a.shift) * a.sB[what] + (slot & inside) * a.sL[what]);
  };
  const auto score = [&](int slot) { return a.scores + (((int64_t)(slot >> a.shift) * a.Hkv + h) << a.shift) + (slot & inside); };
  const auto find = [&](int i) {
    Move m = {-1, -1};
    if (i < stay && list[i] != i) m = {slot_at(a, r, list[i]), slot_at(a, r, i)};
    return m;
  };
  Move m[kMove];
  piece16 x[2][kMove];
#pragma unroll
  for (int u = 0; u < kMove; ++u) m[u] = find(begin + per * u + first);
  const Move mine = find(begin + threadIdx.x);             // (of the scores, a token a thread)
#pragma unroll
  for (int u = 0; u < kMove; ++u)
#pragma unroll
    for (int what = 0; what < 2; ++what) {
      x[what][u] = piece16{0, 0, 0, 0};
      if (m[u].src >= 0) x[what][u] = *row(what, m[u].src);
    }
  const float w = mine.src >= 0 ? *score(mine.src) : 0.f;
  wait_vmem<0>();
  __syncthreads();                                         // (everything is read)
#pragma unroll
  for (int u = 0; u < kMove; ++u)
    if (m[u].dst >= 0) {
      *row(0, m[u].dst) = x[0][u];
      *row(1, m[u].dst) = x[1][u];
    }
  if (mine.dst >= 0) *score(mine.dst) = w;
}

}  // namespace zc

using namespace zc;

__global__ void k_evict_none(int32_t* n_freed) { *n_freed = 0; }

extern "C" size_t zc_paged_evict_workspace(int64_t R, int64_t Hkv, int64_t max_blocks, int64_t page, int32_t together) {
  if (R <= 0 || Hkv <= 0 || max_blocks < 0 || page <= 0 || R > 65535 || Hkv > 65535 || max_blocks > 0x7fff0000 / page) return 0;
  return (size_t)align_up64(R * (together ? 1 : Hkv) * 4, 16) + (together ? (size_t)(R * max_blocks * page) * sizeof(float) : 0);
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
  if (n_freed && n_freed == n_free) return ZC_ERR_INVALID_ARG;       // (one workgroup writes it while others read it)
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
  const size_t need = zc_paged_evict_workspace(R, H, max_blocks, page, together);
  if ((!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 15))) return ZC_ERR_WORKSPACE;

  const int64_t eb = elem_bytes(k_pages->dtype);
  EvictArgs a;
  const zc_tensor4* pools[2] = {k_pages, v_pages};
  for (int i = 0; i < 2; ++i) {
    a.pool[i] = (uint8_t*)pools[i]->ptr;
    a.sB[i] = pools[i]->sB * eb; a.sH[i] = pools[i]->sH * eb; a.sL[i] = pools[i]->sL * eb;
  }
  a.scores = scores;
  a.table = block_table; a.kv_len = kv_len; a.keep = keep; a.row = row_stride;
  a.cols = (int)max_blocks; a.shift = __builtin_ctzll((unsigned long long)page); a.n_pages = (int)k_pages->B; a.cap = (int)(max_blocks * page);
  a.R = (int)R; a.Hkv = (int)H; a.heads = together ? 1 : (int)H;
  a.most = most; a.sinks = sinks; a.recent = recent;
  a.new_len = new_len; a.kept = kept; a.free_pages = free_pages; a.n_freed = n_freed; a.n_free = n_free; a.n_list = n_list;
  a.sums = nullptr;
  a.moved = (int*)ws;
  if (together && a.cap) {
    float* sums = (float*)((uint8_t*)ws + align_up64(R * 4, 16));
    hipLaunchKernelGGL(k_evict_sums, dim3((unsigned)ceil_div64(a.cap, 256), (unsigned)R), dim3(64), 0, st, a, sums);
    ZC_LAUNCH_CHECK();
    a.sums = sums;
  }
  const dim3 lists((unsigned)a.heads + 1, (unsigned)R);
  a.rowb = (int)(k_pages->D * eb);
  // (every head its own list, all of whose rows are one step)
  a.lanes = __builtin_ctz(a.rowb / 16);
  if (a.heads == H && (most << a.lanes) <= kMove * 1024) {
    if (a.cap <= 256 * kEach && (most << a.lanes) <= kMove * 256) hipLaunchKernelGGL((k_evict_short<256, 1>), lists, dim3(256), 0, st, a);
    else if (a.cap <= 1024 * kEach) hipLaunchKernelGGL((k_evict_short<1024, 1>), lists, dim3(1024), 0, st, a);
    else if (a.cap <= 4 * 1024 * kEach) hipLaunchKernelGGL((k_evict_short<1024, 4>), lists, dim3(1024), 0, st, a);
    else hipLaunchKernelGGL((k_evict_short<1024, 8>), lists, dim3(1024), 0, st, a);
    ZC_LAUNCH_CHECK();
    return ZC_OK;
  }
  // Threads for four tokens each; short lists in workgroups of 256, of which a CU holds more.  us with 512 threads here and
  // 1024 in the move, and with 256 in both (lists that k_evict_short takes now): 37 requests of 20 tokens, 40 heads of 128
  // channels, 39 and 21; 128 of up to 250, 8 heads, 33 and 24; one of up to 900 14.2 and 14.5.
  if (a.cap <= 256 * kEach) hipLaunchKernelGGL((k_evict_pick<256, 1>), lists, dim3(256), 0, st, a);
  else if (a.cap <= 512 * kEach) hipLaunchKernelGGL((k_evict_pick<512, 1>), lists, dim3(512), 0, st, a);
  else if (a.cap <= 1024 * kEach) hipLaunchKernelGGL((k_evict_pick<1024, 1>), lists, dim3(1024), 0, st, a);
  else if (a.cap <= 2 * 1024 * kEach) hipLaunchKernelGGL((k_evict_pick<1024, 2>), lists, dim3(1024), 0, st, a);
  else if (a.cap <= 4 * 1024 * kEach) hipLaunchKernelGGL((k_evict_pick<1024, 4>), lists, dim3(1024), 0, st, a);
  else hipLaunchKernelGGL((k_evict_pick<1024, 8>), lists, dim3(1024), 0, st, a);
  ZC_LAUNCH_CHECK();
  const int64_t chains = R * H * 2;
  // Rows are cut where that fills the chip and saves steps of the way through the list.  us of whole rows, of 128, 64 and 16
  // bytes, 8 heads, 256 bytes a row: one request of 4096, 1638 stay 39.0, 26.0, 20.2 and 18.6; of 131072, 32768 stay (64 and
  // 16) 286 and 286; 4 of up to 400, 256 stay 15.7 and 15.7 (20.2 of 32); 15 of up to 8192, 2048 stay 79 whole, 81 of 128.
  a.slice = a.rowb;
  while (a.slice > 16 && chains * (a.rowb / a.slice) < 256 && most > kMove * 1024 * 16 / a.slice) a.slice /= 2;
  a.lanes = __builtin_ctz(a.slice / 16);
  // (one step is all that short lists take: a workgroup of a quarter of the threads does.  64 of up to 900 tokens, 64 stay
  // 26.2 and 20.5, 16 of up to 250 15.0 and 15.2) (parts of a row beside each other in one L2: with the parts of a head as the
  // fastest index the request of 131072 takes 299 us of 32 bytes, 388 of 16)
  const dim3 grid((unsigned)(3 * H), (unsigned)(a.rowb / a.slice), (unsigned)R);
  if (most <= kMove * 256 * 16 / a.slice) hipLaunchKernelGGL(k_evict_move<256>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_evict_move<1024>, grid, dim3(1024), 0, st, a);
  ZC_LAUNCH_CHECK();
  return ZC_OK;
}
