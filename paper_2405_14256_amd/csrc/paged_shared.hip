// zc_paged_shared_attention: attention of a step's new tokens where groups of requests share a prefix, which lies in pages of its own.
//
// Rows (token, query head of the group) of requests that share a prefix see the same keys, so they go through it together, in
// blocks of 32 or 128 rows of many requests, each key read and multiplied once for all of them; every request's own keys
// follow, and a row's parts are joined in fp32:
//   m = max(m_p, m_o),  l = l_p e^(m_p - m) + l_o e^(m_o - m),  o = (o_p e^(m_p - m) + o_o e^(m_o - m)) / l
// A request with more than 64 rows fills blocks of its own: these take the prefix and then its own keys without a join.
//
// Lengths and groups are known to the GPU only.  What every unit of work is - a block of rows, a range of tiles of the prefix,
// one of the request's own - how far long ranges are split, and what is to be joined follows from sums over requests and
// groups, which every workgroup computes for itself, or where there are many one workgroup in front (k_shared_plan).
//
// Bound by memory where rows are few: 64 tokens with 64 to 1024 of their own after 8192 (32 heads over 8 of 128 channels,
// bf16, 135 MB) 43 us and the join 7 with cold caches, 3.1 TB/s; one after 131072 106 us, 5.1 TB/s; by the matrix cores where
// they are many: 4 chunks of 512 after 32768 1145 us, 970 TFLOP/s.
#include "paged_attention_kernel.hpp"

namespace zc {

constexpr int kGroups = 1024;                   // prefixes of a step, at most
constexpr int kSharedJoinGroups = 4;            // workgroups that join a block
constexpr int kFewRows = 64;                    // of a request that goes through a prefix together with others, at most

struct SharedArgs : PagedArgs {
  const int32_t *pre_table, *pre_len, *group_start;
  int64_t pre_row;                              // of the prefixes' table, in entries
  int pre_cols, pre_cap, P;
  int* counts;                                  // units, joins
  int4* plan;                                   // [unit][4]
  int4* joins;                                  // [block][2]
  int* tokens;                                  // the tokens that go through a prefix together, group after group
  int least;                                    // tiles, below which a block is not split (fp32)
  float worth;                                  // tiles that a shared prefix has to spare
  int far;                                      // tiles, above which a prefix is read once for 33 to 64 rows
  int places;                                   // of a head's units at a time
  int most_units, most_joins;                   // (units: partial results that there is room for)
};

// What a unit of the plan is, in words of its entry.
enum Word { kFew, kGroup, kRequest, kPart, kRow0, kPast, kOwnKeys, kPrefixKeys, kToken, kHead, kRows, kLast, kFrom, kTo, kWords = 16 };

// A unit's keys are one stream of tiles, those of the prefix in front: its keys have negative positions, -kTile * pre_tiles
// on, so that the last of its tiles, which need not be full, ends in front of the request's own first key.  The places
// between, from `hole` to -1, are hidden.
struct SharedUnit {
  static constexpr int kFirst = -1;
  static constexpr int first = 0, sink_tiles = -(1 << 30);     // (tiles follow each other)
  static constexpr uint32_t behind = 0;
  int qs, past, j0, g0, rows;   // the request's first row; tokens in front of its new ones; token and head of the block's first row, its rows
  int last;                     // rows of several requests: the block's last place in the list of tokens; -1: of one
  int token;                    // then: of this lane's row
  int part;                     // where its partial results go, -1: nothing to join
  const int32_t *pre, *own;     // rows of the tables
  int pre_tiles, hole, kv, t_lo, t_hi, p0, p1;
};
__device__ inline Row row_at(const PagedArgs& a, const SharedUnit& x, int r) { return row_at(a, x.j0, x.g0, r); }
__device__ inline Row row_of(const PagedArgs& a, const SharedUnit& x, int r) {
  Row me = row_at(a, x, r);
  if (x.last >= 0) me.j = x.token;
  return me;
}
// (rows of several requests, and a row in front of its request's first token, see all of the prefix and nothing else)
__device__ inline int position(const SharedUnit& x, int j) { return x.last >= 0 ? -1 : max(x.past + j, -1); }
__device__ inline int tile_of(const SharedUnit& x, int t) { return t - x.pre_tiles; }
__device__ inline int tile_at(const SharedUnit& x, int pos) { return (pos >> 6) + x.pre_tiles; }
static_assert(kTile == 64, "tile_at");
__device__ inline const int32_t* entry_of(const PagedArgs& args, const SharedUnit& x, int key0) {
  const SharedArgs& a = static_cast<const SharedArgs&>(args);
  const bool pre = key0 < 0;
  const int block = (pre ? key0 + x.pre_tiles * kTile : key0) >> a.shift;
  return pre ? x.pre + min(block, a.pre_cols - 1) : x.own + min(block, a.cols - 1);
}
__device__ inline int keys_read(const PagedArgs& a, const SharedUnit& x, int end, int key0, int id) {
  return keys_read(a.n_pages, 0, 0, key0 < 0 ? min(end, x.hole) : end, key0, id);
}
__device__ inline __amdgpu_buffer_rsrc_t keys_at(const PagedArgs& a, const SharedUnit& x, const uint8_t* head, uint32_t sB, uint32_t row, int key0, int id, int n) {
  return keys_at(a.shift, head, sB, row, key0 < 0 ? key0 + x.pre_tiles * kTile : key0, id, n);
}
__device__ inline Seen seen_by(const PagedArgs&, const SharedUnit& x, int p0, int) {
  Seen s;
  s.low = 0;
  s.span = max(p0 - 30, 0);
  s.sink = x.hole - 31;
  return s;
}
__device__ inline int low_of(const PagedArgs&, const SharedUnit&, int) { return -1; }
__device__ inline int sinks_of(const PagedArgs&, const SharedUnit& x) { return x.hole; }
__device__ inline bool is_whole(const SharedUnit& x) { return x.part < 0; }
__device__ inline int64_t part_of(const PagedArgs& a, const SharedUnit& x, int hk) { return part_row(a, hk, x.part); }

// ---- the plan -------------------------------------------------------------------------------------
// Entries of the plan are the requests: what their rows are, and that they go through their prefix together with others' if they are few.
struct Entry { int qs, nq, kv, group, pre, few, blocks, tiles, together; };
struct Cut { int few, blocks; };                           // blocks of 32 rows or of `many`
__device__ inline Cut cut_of(int rows, int many, int few_rows = kFewRows) {
  const bool few = rows <= few_rows || many == 32;
  return {few, few ? (rows + 31) / 32 : (rows + many - 1) / many};
}

constexpr int kListed = 130;                               // tokens that a block's rows are of, at most
template <int THREADS>
struct PlanMemory {
  int g_start[kGroups + 1], g_kv[kGroups], g_first[kGroups], g_end[kGroups], g_part[kGroups], g_parts[kGroups];
  // of the entries in hand
  int unit[THREADS], join[THREADS], part[THREADS], parts[THREADS], blocks[THREADS], qs[THREADS], nq[THREADS], kv[THREADS], group[THREADS], place[THREADS];
  int waves[3][THREADS / 64], five[5][THREADS / 64];
  float sums[2][THREADS / 64];
  int one[kWords], list[kListed];                          // of one unit: its entry, the tokens of its rows
};

// ALL: units, joins and the list of tokens go to memory.  Otherwise unit `wanted` stays in LDS (false: there is none), with
// the tokens of its rows, and what it is joined with goes to memory.
template <int THREADS, bool ALL>
__device__ bool plan(const SharedArgs& a, int many, int wanted, PlanMemory<THREADS>& s) {
  constexpr int NW = THREADS / 64;
  const int tid = threadIdx.x;
  bool share = false;                                      // (set below)
  struct Given { int from, to, kv; };
  const auto given = [&](int r) { return r < a.R ? Given{a.q_start[r], a.q_start[r + 1], a.kv_len[r]} : Given{0, 0, 0}; };
  const auto entry = [&](int r, const Given& in) {         // (g_start and g_kv are there)
    Entry x = {0, 0, 0, -1, 0, 0, 0, 0, 0};
    if (r >= a.R) return x;
    x.qs = min(max(in.from, 0), a.T);
    x.nq = max(min(in.to, a.T) - x.qs, 0);
    x.kv = min(max(in.kv, 0), a.cap);
    int lo = 0, hi = a.P + 1;                              // how many groups begin at or in front of it
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (s.g_start[mid] <= r) lo = mid + 1;
      else hi = mid;
    }
    if (lo > 0 && lo <= a.P) {
      x.group = lo - 1;
      x.pre = s.g_kv[lo - 1];
    }
    const int rows = x.nq * a.G;
    const Cut c = cut_of(rows, many);
    x.few = c.few;
    x.blocks = c.blocks;
    x.together = share && rows > 0 && rows <= kFewRows && x.pre > 0 && s.g_start[lo] - s.g_start[lo - 1] > 1;
    x.tiles = (x.kv + kTile - 1) / kTile + (x.together ? 0 : (x.pre + kTile - 1) / kTile);
    return x;
  };
  // Rows of a group that go through its prefix together (of starts that do not ascend they could be more than there are).
  const auto rows_of = [&](int g) { return min(max(s.g_end[g] - s.g_first[g], 0), a.T) * a.G; };
  const auto cut_together = [&](int g) { return cut_of(rows_of(g), many, (s.g_kv[g] + kTile - 1) / kTile > a.far ? 32 : kFewRows); };
  const Given front = given(tid);
  for (int e = tid; e <= a.P; e += THREADS) {
    s.g_start[e] = min(max(a.group_start[e], 0), a.R);
    if (e < a.P) {
      s.g_kv[e] = min(max(a.pre_len[e], 0), a.pre_cap);
      s.g_first[e] = s.g_end[e] = 0;
    }
  }
  __syncthreads();
  // Whether it pays: tiles that need not be read again, of all heads, if every request of a group has a few rows (those
  // without rows, and chunks, are counted too: there may be less to spare).
  float again = 0.f;
  for (int g = tid & 63; g < a.P; g += 64) again += (float)max(s.g_start[g + 1] - s.g_start[g] - 1, 0) * (float)((s.g_kv[g] + kTile - 1) / kTile);
  share = wave_sum(again) * (float)a.Hkv > a.worth;

  // ---- rows that go through a prefix together; all work
  int placed = 0;
  float work = 0.f, n_blocks = 0.f;                        // tiles of all blocks
  Entry held;                                              // (of the first entries)
  for (int r0 = 0; r0 < a.R; r0 += THREADS) {
    const int r = r0 + tid;
    const Entry x = entry(r, r0 ? given(r) : front);
    if (r0 == 0) held = x;
    const int n = x.together ? x.nq : 0;
    int all;
    const int upto = placed + block_inclusive_sum<NW>(n, s.waves[(r0 / THREADS) & 1], all), at = upto - n;
    if constexpr (ALL)
      for (int j = 0; j < n; ++j)
        if (at + j < a.T) a.tokens[at + j] = x.qs + j;
    if (x.group >= 0) {
      if (r == s.g_start[x.group]) s.g_first[x.group] = at;
      if (r == s.g_start[x.group + 1] - 1) s.g_end[x.group] = upto;
    }
    work += (float)x.blocks * (float)x.tiles;
    n_blocks += (float)x.blocks;
    placed += all;
  }
  __syncthreads();
  for (int g = tid; g < a.P; g += THREADS) {
    const int blocks = cut_together(g).blocks;
    work += (float)blocks * (float)((s.g_kv[g] + kTile - 1) / kTile);
    n_blocks += (float)blocks;
  }
  work = wave_sum(work);
  n_blocks = wave_sum(n_blocks);
  if ((tid & 63) == 0) { s.sums[0][tid >> 6] = work; s.sums[1][tid >> 6] = n_blocks; }
  __syncthreads();
  work = n_blocks = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) { work += s.sums[0][w]; n_blocks += s.sums[1][w]; }
  float share_of_work = fmaxf(ceilf(work / (float)a.target), 1.f);               // tiles of a part, at most
  // Blocks of about one length in a few more parts than the chip has places for: some wait for a whole round of them.  Longer
  // parts that fit, then.  us: 12 chunks of 17 and 31 tokens after 4096 (32 heads over 8 of 128 channels, bf16; 72 parts a
  // head in 64 places, then 60) 64.7 and 51.8, 74.5 and 61.5.
  const float length = work / fmaxf(n_blocks, 1.f), cuts = ceilf(length / share_of_work);
  if (cuts >= 3.f && cuts * n_blocks > (float)a.places) share_of_work = fmaxf(share_of_work, ceilf(1.04f * length / (cuts - 1.f)));
  const int per = (int)fminf(share_of_work, 1e9f);
  // (below which a part is not worth its way through memory, as for the paged attention)
  n_blocks *= (float)a.Hkv;
  const int least = many == 32 ? a.least : n_blocks >= 128.f ? 16 : n_blocks >= 64.f ? 10 : 6;
  const auto parts_of = [&](int tiles) { return tiles <= max(per, least) ? 1 : (tiles + per - 1) / per; };

  // The entry in hand that a unit belongs to: the last that begins at or in front of it.
  const auto owner = [&](int u, int n) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s.unit[mid] <= u) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  const auto put = [&](int u, int part, int4 w0, int4 w1, int4 w2, int4 w3) {
    if (u >= a.most_units) return;                         // (never of lengths that ascend)
    if (part >= a.units) w0.w = w2.z = w3.x = w3.y = 0;
    int4* d = ALL ? a.plan + (int64_t)u * (kWords / 4) : reinterpret_cast<int4*>(s.one);
    d[0] = w0; d[1] = w1; d[2] = w2; d[3] = w3;
  };
  // f(u, entry) for units u of `all` in hand, the first of which has number `first`; this thread's `count` entry has those from `begin` on.
  const auto units_in_hand = [&](int first, int all, int n, int begin, int count, auto&& f) {
    if constexpr (ALL) {
      __syncthreads();
      for (int u = tid; u < all; u += THREADS) f(u, owner(u, n));
    } else if (wanted - first >= begin && wanted - first < begin + count) {
      f(wanted - first, tid);
    }
  };

  // ---- units of the prefixes
  int units = 0, joins = 0, parts = 0;
  for (int g0 = 0; g0 < a.P; g0 += THREADS) {
    const int g = g0 + tid, rows = g < a.P ? rows_of(g) : 0, tiles = g < a.P ? (s.g_kv[g] + kTile - 1) / kTile : 0;
    const Cut c = g < a.P ? cut_together(g) : Cut{1, 0};
    const int n = parts_of(tiles), mine = c.blocks * n;
    int all;
    if (g0) __syncthreads();
    const int before = block_inclusive_sum<NW>(mine, s.waves[2], all) - mine;
    s.unit[tid] = before;
    s.parts[tid] = n;
    if (g < a.P) {
      s.g_part[g] = units + before;
      s.g_parts[g] = n;
    }
    units_in_hand(units, all, min(a.P - g0, THREADS), before, mine, [&](int u, int i) {
      const int e = g0 + i, n = s.parts[i], rest = u - s.unit[i], b = rest / n, p = rest - b * n;
      const int rows = rows_of(e), tiles = (s.g_kv[e] + kTile - 1) / kTile;
      const Cut k = cut_together(e);
      const int rb = k.few ? 32 : many, i0 = b * rb, j = i0 / a.G, q = tiles / n, rem = tiles - q * n;
      const int lo = p * q + min(p, rem), hi = lo + q + (p < rem ? 1 : 0);
      put(units + u, units + u, make_int4(k.few, e, 0, units + u), make_int4(0, 0, 0, s.g_kv[e]),
          make_int4(s.g_first[e] + j, i0 - j * a.G, min(rb, rows - i0), s.g_end[e] - 1), make_int4(lo, hi, 0, 0));
    });
    units += all;
  }
  parts = units;

  // ---- units of the requests, and what is joined
  placed = 0;
  for (int r0 = 0; r0 < a.R; r0 += THREADS) {
    const Entry x = r0 ? entry(r0 + tid, given(r0 + tid)) : held;
    const int n = parts_of(x.tiles), apart = x.together || n > 1;
    int all[5];                                            // units, joins, partial results, tokens that go together, units of long requests
    if (ALL || r0) __syncthreads();                        // (the entries before are done with)
    const int t = x.together ? x.nq : 0, mine = x.blocks * n;
    // Units that do not run all at once: requests longer than the mean of the blocks first (of those in hand), or one of them
    // begins last.  us in order and so (32 heads over 8 of 128 channels, bf16): 100 tokens of 64 to 1000 after 4096 65.1 and
    // 58.2, 64 after 8192 56.7 and 53.6; 40 of 500 to 1500 after 8192 (16 heads of 64, fp16) 52.6 and 54.9.  Where they do, it
    // costs: 32 of up to 2000 after 4096 39.0 and 40.9.
    const bool late = !ALL && (float)x.tiles <= length;
    int upto[5] = {mine, apart ? x.blocks : 0, apart ? mine : 0, t, late ? 0 : mine};
    block_inclusive_sums<NW>(upto, s.five, all);
    const int begin = ALL || units + all[0] <= a.places ? upto[0] - mine : late ? all[4] + upto[0] - upto[4] - mine : upto[4] - mine;
    s.unit[tid] = begin;
    s.join[tid] = upto[1] - (apart ? x.blocks : 0);
    s.part[tid] = apart ? upto[2] - mine : -1;
    s.parts[tid] = n;
    s.blocks[tid] = x.blocks;
    s.qs[tid] = x.qs; s.nq[tid] = x.nq; s.kv[tid] = x.kv;
    s.group[tid] = x.group;
    s.place[tid] = x.together ? placed + upto[3] - t : -1; // of its first token in the list
    units_in_hand(units, all[0], THREADS, begin, mine, [&](int u, int e) {
      const int n = s.parts[e], rest = u - s.unit[e], b0 = rest / n, p = rest - b0 * n;
      const int b = s.blocks[e] - 1 - b0;                  // (a chunk's last rows see the most keys: first)
      const int past = s.kv[e] - s.nq[e], rows = s.nq[e] * a.G, group = s.group[e], together = s.place[e] >= 0;
      const Cut k = cut_of(rows, many);
      const int rb = k.few ? 32 : many, i0 = b * rb, j0 = i0 / a.G, g0 = i0 - j0 * a.G, take = min(rb, rows - i0);
      const int p1 = past + (i0 + take - 1) / a.G;
      const int pre = group >= 0 && !together ? s.g_kv[group] : 0, tiles = (pre + kTile - 1) / kTile + (p1 < 0 ? 0 : p1 / kTile + 1);
      const int q = tiles / n, rem = tiles - q * n, lo = p * q + min(p, rem), hi = lo + q + (p < rem ? 1 : 0);
      const int part = s.part[e] >= 0 ? parts + s.part[e] + b0 * n + p : -1;
      put(units + u, part, make_int4(k.few, group < 0 ? 0 : group, r0 + e, part), make_int4(s.qs[e], past, s.kv[e], pre), make_int4(j0, g0, take, -1),
          make_int4(lo, hi, 0, 0));
      const int join = joins + s.join[e] + b0;
      if (p == 0 && part >= 0 && join < a.most_joins) {
        int4 w = make_int4(g0, 0, 0, 0);
        if (together) {
          const bool big = !cut_together(group).few;
          w = make_int4(g0, s.g_part[group], s.g_parts[group] << 1 | (big ? 1 : 0), (s.place[e] - s.g_first[group]) * a.G + i0);
        }
        a.joins[2 * join] = make_int4(part, n, take, s.qs[e] + j0);
        a.joins[2 * join + 1] = w;
      }
    });
    units += all[0];
    joins += all[1];
    parts += all[2];
    placed += all[3];
  }
  if (tid == 0 && (ALL || wanted == 0)) {
    a.counts[0] = min(units, a.most_units);
    a.counts[1] = min(joins, a.most_joins);
  }
  if constexpr (ALL) return true;
  if (wanted >= min(units, a.most_units)) return false;
  __syncthreads();
  const int last = s.one[kLast], j0 = s.one[kToken];
  if (last < 0) return true;
  // the tokens of the unit's rows, `last` and all in front of it that a block can have
  placed = 0;
  for (int r0 = 0; r0 < a.R; r0 += THREADS) {
    const Entry x = r0 ? entry(r0 + tid, given(r0 + tid)) : held;
    const int n = x.together ? x.nq : 0;
    int all;
    const int at = placed + block_inclusive_sum<NW>(n, s.waves[(r0 / THREADS) & 1], all) - n;
    for (int j = max(j0 - at, 0); j < n && at + j <= last && at + j - j0 < kListed; ++j) s.list[at + j - j0] = x.qs + j;
    placed += all;
  }
  __syncthreads();
  return true;
}

// One workgroup, a thread an entry at first, then a thread a unit.
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void k_shared_plan(SharedArgs a, int many) {
  __shared__ __align__(16) PlanMemory<kPlanThreads> s;
  plan<kPlanThreads, true>(a, many, 0, s);
}

// ---- the units ------------------------------------------------------------------------------------
// PLANNED: by k_shared_plan.  Otherwise every workgroup finds its unit itself, which spares a launch.
template <int DT, int D, bool PLANNED>
__global__ __launch_bounds__(256, DT == ZC_F32 && D == 128 ? 1 : 2) void k_shared_attention(SharedArgs a) {
  constexpr int kBytes = DT == ZC_F32 ? RowsMemory<DT, D, 4>::kBytes : kStages<D> * 2 * kTile * Tile<DT, D>::ROWB;
  static_assert(kBytes >= RowsMemory<DT, D, 4>::kBytes, "blocks of few rows find room");
  static_assert(kBytes >= (int)sizeof(PlanMemory<256>), "and the plan");
  __shared__ __align__(1024) uint8_t mem[kBytes];
  __shared__ float sum[4][2][64];
  constexpr int kMany = DT == ZC_F32 ? 32 : 128;
  const int u = unit_of_grid(), hk = blockIdx.x;
  int d[kWords];
  int token = 0;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  if constexpr (PLANNED) {
    typedef __attribute__((address_space(4))) const int* scalar;
    if (u >= ((scalar)(uintptr_t)a.counts)[0]) return;
#pragma unroll
    for (int i = 0; i < kWords; ++i) d[i] = ((scalar)(uintptr_t)(a.plan + (int64_t)u * (kWords / 4)))[i];
  } else {
    PlanMemory<256>& s = *reinterpret_cast<PlanMemory<256>*>(mem);
    if (!plan<256, false>(a, kMany, u, s)) return;
#pragma unroll
    for (int i = 0; i < kWords; ++i) d[i] = __builtin_amdgcn_readfirstlane(s.one[i]);
  }
  SharedUnit x;
  x.qs = d[kRow0]; x.past = d[kPast]; x.j0 = d[kToken]; x.g0 = d[kHead]; x.rows = d[kRows]; x.last = d[kLast]; x.part = d[kPart];
  x.pre = a.pre_table + d[kGroup] * a.pre_row;
  x.own = a.table + d[kRequest] * a.row;
  x.kv = d[kOwnKeys];
  x.pre_tiles = (d[kPrefixKeys] + kTile - 1) / kTile;
  x.hole = d[kPrefixKeys] - x.pre_tiles * kTile;
  x.t_lo = d[kFrom]; x.t_hi = d[kTo];
  x.p0 = position(x, x.j0);
  x.p1 = position(x, row_at(a, x, x.rows - 1).j);
  if (x.last >= 0) {
    const int j = min(row_at(a, x, (d[kFew] ? 0 : 32 * w) + (lane & 31)).j, x.last);
    if constexpr (PLANNED) token = a.tokens[min(j, a.T - 1)];
    else token = reinterpret_cast<PlanMemory<256>*>(mem)->list[min(max(j - x.j0, 0), kListed - 1)];
  }
  x.token = min(max(token, 0), a.T - 1);
  if constexpr (!PLANNED) __syncthreads();                 // (the plan is done with LDS)
  if constexpr (DT != ZC_F32) {
    if (!d[kFew]) {
      attend_tiles<DT, D>(a, x, hk, mem);
      return;
    }
  }
  attend_rows<DT, D, 4>(a, x, hk, mem, sum);
}

// ---- the join -------------------------------------------------------------------------------------
// As the paged attention's: four workgroups a block, D / 4 threads a row; a row's parts are its own request's and those of its place
// among the rows that went through the prefix together.
template <int DT, int D>
__global__ __launch_bounds__(256) void k_shared_join(SharedArgs a) {
  constexpr int TPR = D / 4, GROUPS = 256 / TPR;
  __shared__ __align__(16) float so[GROUPS][D];
  __shared__ float2 sml[GROUPS];
  const int turn = (int)blockIdx.x / a.Hkv, hk = blockIdx.x - turn * a.Hkv;
  const int grp = threadIdx.x / TPR, c = threadIdx.x % TPR * 4, joins = a.counts[1];
  for (int join = blockIdx.y; join < joins; join += gridDim.y) {
    const int4 w = a.joins[2 * join], v = a.joins[2 * join + 1];
    const int first = w.x, own = w.y, rows = w.z, pre = v.z >> 1, shift = v.z & 1 ? 7 : 5, parts = own + pre;
    if (first + own > a.units || pre > a.units) continue;
    const int step = min((rows + kSharedJoinGroups - 1) / kSharedJoinGroups, GROUPS);        // rows at a time: few rows are spread over the workgroups too
    for (int row0 = turn * step; row0 < rows; row0 += kSharedJoinGroups * step) {
      const int n = min(rows - row0, step);
      int ways = 1;                                          // groups to a row
      while (2 * ways * n <= GROUPS && 2 * ways <= parts) ways *= 2;
      const int way = grp & (ways - 1), row = row0 + grp / ways;
      const bool mine = row < row0 + n;
      const int i = v.w + row, pre0 = v.y + (i >> shift) * pre, pre_row = i & ((1 << shift) - 1);
      float M = kLowestLogit, l = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      if (mine && (pre == 0 || (uint32_t)pre0 <= (uint32_t)(a.units - pre))) {
        constexpr int U = 4;                                 // parts requested at a time
        for (int s0 = way; s0 < parts; s0 += U * ways) {
          float2 ml[U];
          float4 t[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int s = s0 + u * ways < parts ? s0 + u * ways : s0;
            const int64_t p = s < pre ? part_row(a, hk, pre0 + s) + pre_row : part_row(a, hk, first + s - pre) + row;
            ml[u] = *reinterpret_cast<const float2*>(a.part_ml + p * 2);
            t[u] = *reinterpret_cast<const float4*>(a.part_o + p * D + c);
          }
          float top = M;
#pragma unroll
          for (int u = 0; u < U; ++u) top = fmaxf(top, ml[u].x);
          const float f0 = __builtin_amdgcn_exp2f(M - top);
          M = top;
          l *= f0; o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const float f = s0 + u * ways < parts ? __builtin_amdgcn_exp2f(ml[u].x - M) : 0.f;
            l = fmaf(ml[u].y, f, l);
            o.x = fmaf(t[u].x, f, o.x); o.y = fmaf(t[u].y, f, o.y); o.z = fmaf(t[u].z, f, o.z); o.w = fmaf(t[u].w, f, o.w);
          }
        }
      }
      if (ways > 1) {
        if (c == 0) sml[grp] = make_float2(M, l);
        *reinterpret_cast<float4*>(&so[grp][c]) = o;
        __syncthreads();
        if (mine && way == 0) {
          for (int y = 1; y < ways; ++y) {
            const float2 ml = sml[grp + y];
            const float4 t = *reinterpret_cast<const float4*>(&so[grp + y][c]);
            const float top = fmaxf(M, ml.x), f0 = __builtin_amdgcn_exp2f(M - top), f = __builtin_amdgcn_exp2f(ml.x - top);
            M = top;
            l = fmaf(ml.y, f, l * f0);
            o.x = fmaf(t.x, f, o.x * f0); o.y = fmaf(t.y, f, o.y * f0); o.z = fmaf(t.z, f, o.z * f0); o.w = fmaf(t.w, f, o.w * f0);
          }
        }
        __syncthreads();
      }
      if (mine && way == 0) store_row<DT>(a, w.w, v.x, hk, row, c, M, l, o);
    }
  }
}

// ---- host ---------------------------------------------------------------------------------------------
// How large a step can get, of one head: units, partial results (of how many rows), joins.  (target: what splitting aims at.)
struct Most { int64_t target, units, parts, joins, slot, bytes; };
static Most most_of(int64_t P, int64_t R, int64_t T, int64_t G, int64_t Hkv, bool fp32, int64_t D) {
  Most m;
  const int64_t with = R < T ? R : T, rows = T * G, many = fp32 ? 32 : 128, groups = P < with ? P : with;
  m.slot = fp32 || rows <= 32 ? 32 : 128;
  // What the chip holds at a time: more parts cost more on their way through memory than they even out.  us at 256, 384, 512,
  // 768 and 1024 units: bf16, 32 heads over 8 of 128 channels, 64 tokens after 8192 56.8, 56.7, 56.7, 63.5 and 68.4; fp16, 16
  // over 4 of 64, 20 tokens and 7 chunks after up to 4000 35.8, 32.7, 36.7, 41.0 and 42.9; 24 over 8 of 64, 90 tokens of up to
  // 3843 after up to 2314 115, 115, 110 and 105; fp32, 16 heads of 128, 74 tokens after up to 593 91.7, 97.2, 101 and 106.
  m.target = ceil_div64(fp32 && D == 128 ? 256 : 512, Hkv);
  // (a request has one block that is not full; where blocks of 128 rows are the rule, one of 33 to 64 rows is two of 32)
  const int64_t two = rows / 33 < with ? rows / 33 : with, blocks = rows / many + with + two;
  const int64_t few = rows / 32 + with < 2 * with ? rows / 32 + with : 2 * with;
  const int64_t together = rows < kFewRows * with ? rows : kFewRows * with, pre = together / many + 2 * groups;
  // a block is cut into at most tiles / (all work / target) + 1 parts; one of many rows leaves none if it is not cut (2: sums
  // of work are rounded)
  m.units = m.target + blocks + pre + 2;
  m.parts = 2 * m.target + few + pre + 2;
  m.joins = blocks;
  m.bytes = (int64_t)Hkv * m.parts * m.slot * (D + 2) * 4 + m.units * 64 + m.joins * 32 + align_up64(T * 4, 16) + 16;
  return m;
}

template <int DT, int D>
static int launch_shared(SharedArgs& a, hipStream_t st) {
  // A workgroup finds its unit in about 2 us, a plan takes a launch of 5 to 8.  us found and planned: bf16, 32 heads over 8 of
  // 128 channels, 8 tokens after 1000 19.3 and 24.9 (one round of workgroups), 64 after 8192 56.2 and 58.8 (two); fp16, 40
  // heads, 42 tokens 47.0 and 39.3 (eight), 12 chunks after 4096 307 and 312 (five); fp32, 16 heads of 128, 21 requests 32.8
  // and 29.9 (five), 74 104.8 and 88.4 (ten); 16 over 4 of 64, 22 chunks 85.7 and 73.6 (five).
  const int64_t places = DT == ZC_F32 && D == 128 ? 256 : DT != ZC_F32 && D == 64 ? 768 : 512;
  a.places = (int)(places / a.Hkv);
  const bool planned = a.most_units * a.Hkv > 4 * places;
  const int64_t own_tiles = ceil_div64(a.cap, kTile), pre_tiles = ceil_div64(a.pre_cap, kTile);
  const bool joined = own_tiles + pre_tiles > (DT == ZC_F32 ? a.least : 6) || (float)(a.R * pre_tiles * a.Hkv) > a.worth;     // (the plan's rules)
  if (planned) {
    hipLaunchKernelGGL(k_shared_plan, dim3(1), dim3(kPlanThreads), 0, st, a, DT == ZC_F32 ? 32 : 128);
    ZC_LAUNCH_CHECK();
  }
  const auto grid = [](int64_t x, int64_t n) { return dim3((unsigned)x, (unsigned)(n < 65535 ? n : 65535), (unsigned)ceil_div64(n, 65535)); };
  if (planned) hipLaunchKernelGGL((k_shared_attention<DT, D, true>), grid(a.Hkv, a.most_units), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_shared_attention<DT, D, false>), grid(a.Hkv, a.most_units), dim3(256), 0, st, a);
  ZC_LAUNCH_CHECK();
  if (!joined) return ZC_OK;
  const int64_t turns = ceil_div64(2048, a.Hkv * kSharedJoinGroups);
  hipLaunchKernelGGL((k_shared_join<DT, D>), dim3((unsigned)(a.Hkv * kSharedJoinGroups), (unsigned)(turns < a.most_joins ? turns : a.most_joins)), dim3(256), 0, st, a);
  ZC_LAUNCH_CHECK();
  return ZC_OK;
}

}  // namespace zc

using namespace zc;

// (the larger of what fp32 and 16-bit calls take, and of what a step without a prefix does)
extern "C" size_t zc_paged_shared_attention_workspace(int64_t P, int64_t R, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
  if (P < 0 || R <= 0 || T <= 0 || Hkv <= 0 || Hq < Hkv || Hq % Hkv || D <= 0 || T > 0x7fffffff / Hq) return 0;
  const size_t none = zc_paged_attention_workspace(R, T, Hq, Hkv, D);
  if (P == 0) return none;
  const size_t x = (size_t)most_of(P, R, T, Hq / Hkv, Hkv, true, D).bytes, y = (size_t)most_of(P, R, T, Hq / Hkv, Hkv, false, D).bytes;
  const size_t more = x > y ? x : y;
  return none > more ? none : more;
}

extern "C" int zc_paged_shared_attention(const zc_tensor4* q, const zc_tensor4* k_pages, const zc_tensor4* v_pages, const int32_t* prefix_table,
                                         int64_t prefix_row_stride, int64_t prefix_max_blocks, const int32_t* prefix_len, const int32_t* group_start,
                                         int64_t P, const int32_t* block_table, int64_t row_stride, int64_t max_blocks, const int32_t* q_start,
                                         const int32_t* kv_len, int64_t R, float sm_scale, const zc_tensor4* out, float* lse, void* ws,
                                         size_t ws_bytes, void* stream) {
  int rc = zc_validate_pages(k_pages, v_pages);
  if (rc) return rc;
  rc = zc_validate_heads(q, k_pages);
  if (rc) return rc;
  rc = zc_validate_heads(out, k_pages);
  if (rc) return rc;
  if (q->H != out->H || q->L != out->L || q->H % k_pages->H || !zc_rows_apart(out)) return ZC_ERR_INVALID_ARG;
  if (P < 0 || R < 0 || !(sm_scale >= 0.f) || !(sm_scale * kLog2e <= -kLowestLogit)) return ZC_ERR_INVALID_ARG;
  if (max_blocks < 0 || row_stride < max_blocks || prefix_max_blocks < 0 || prefix_row_stride < prefix_max_blocks) return ZC_ERR_INVALID_ARG;
  if (q->L == 0 || R == 0) return ZC_OK;
  if (!q_start || !kv_len || (max_blocks > 0 && !block_table)) return ZC_ERR_INVALID_ARG;
  if (P > 0 && (!prefix_len || !group_start || (prefix_max_blocks > 0 && !prefix_table))) return ZC_ERR_INVALID_ARG;
  for (const void* p : {(const void*)block_table, (const void*)q_start, (const void*)kv_len, (const void*)lse, (const void*)prefix_table,
                        (const void*)prefix_len, (const void*)group_start})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ZC_ERR_INVALID_ARG;
  if (P > kGroups) return ZC_ERR_UNSUPPORTED;
  if (P == 0 || prefix_max_blocks == 0)                  // no prefix has a token
    return zc_paged_attention(q, k_pages, v_pages, block_table, row_stride, max_blocks, q_start, kv_len, R, 0, 0, sm_scale, out, lse, ws, ws_bytes, stream);
  const int64_t T = q->L, Hkv = k_pages->H, G = q->H / Hkv;
  if (R >= (1 << 24) || max_blocks > 0x7fffffff || prefix_max_blocks > 0x7fffffff || T > 0x7fffffff / q->H || q->H > 65535 || G > 4096)
    return ZC_ERR_UNSUPPORTED;
  const int64_t page = k_pages->L;
  const auto room = [&](int64_t blocks) { return blocks > 0x7fff0000 / page ? 0x7fff0000 : blocks * page; };
  const Most m = most_of(P, R, T, G, Hkv, q->dtype == ZC_F32, q->D);
  if (m.units * Hkv > 0xffffff) return ZC_ERR_UNSUPPORTED;
  const size_t need = zc_paged_shared_attention_workspace(P, R, T, q->H, Hkv, q->D);
  if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 15)) return ZC_ERR_WORKSPACE;

  const int64_t eb = elem_bytes(q->dtype);
  SharedArgs a;
  a.q = (const uint8_t*)q->ptr; a.k = (const uint8_t*)k_pages->ptr; a.v = (const uint8_t*)v_pages->ptr; a.o = (uint8_t*)out->ptr;
  a.q_sH = q->sH * eb; a.q_sT = q->sL * eb; a.o_sH = out->sH * eb; a.o_sT = out->sL * eb;
  a.k_sB = (uint32_t)(k_pages->sB * eb); a.k_sH = k_pages->sH * eb; a.v_sB = (uint32_t)(v_pages->sB * eb); a.v_sH = v_pages->sH * eb;
  a.k_row = (uint32_t)(k_pages->sL * eb); a.v_row = (uint32_t)(v_pages->sL * eb);
  // (a table without columns holds no token: any readable word stands for its pages)
  a.table = max_blocks ? block_table : q_start; a.q_start = q_start; a.kv_len = kv_len; a.row = max_blocks ? row_stride : 0;
  a.cols = max_blocks ? (int)max_blocks : 1; a.shift = __builtin_ctzll((unsigned long long)page); a.n_pages = (int)k_pages->B; a.cap = (int)room(max_blocks);
  a.R = (int)R; a.T = (int)T; a.Hkv = (int)Hkv; a.G = (int)G;
  a.window = a.sinks = 0;
  a.scale_log2 = (sm_scale == 0.f ? 1.0f / sqrtf((float)q->D) : sm_scale) * kLog2e;
  a.lse = lse;
  a.target = (int)m.target;
  a.units = (int)m.parts;
  a.over_G = G == 1 ? 0 : (uint32_t)(((1ull << 32) + G - 1) / G);
  a.reach = 0x7fffffff;
  a.slot = (int)m.slot;
  a.coarse = 0;
  a.todo = nullptr;
  a.pre_table = prefix_table; a.pre_len = prefix_len; a.group_start = group_start; a.pre_row = prefix_row_stride;
  a.pre_cols = (int)prefix_max_blocks; a.pre_cap = (int)room(prefix_max_blocks); a.P = (int)P;
  a.least = q->D == 64 ? 4 : 2;
  // Rows that go through their prefix together have parts to be joined, so as much has to be spared (of a group's requests but
  // one, with or without tokens in this step: counting those with a few rows would be a sweep more.  8 tokens after 1000 19.5
  // us, with 56 requests without tokens beside them 19.7; one after 4096, which then has a join for nothing, 21.0 and 22.8).
  // us together and each request by itself: 8 tokens after 1000 (32 heads over 8 of 128 channels; 29 MB spared) 19.5 and 20.3,
  // 22 after up to 1412 (8 heads of 64; 48 MB) 18.2 and 21.8, 16 chunks of up to 17 after 355 (8 of 64; 12 MB) 18.9 and 15.9,
  // 64 after 8192 (2.1 GB) 55.6 and 189.
  a.worth = 28e6f / (float)(2 * kTile * q->D * eb);
  // Two blocks of 32 rows read a prefix twice, the second time from the caches as long as these hold it (256 MB); one of 128
  // is half empty.  us of two and of one, 16 tokens (32 heads over 8 of 128 channels, bf16) after 1000 26 and 38, 16384 (67
  // MB) 36 and 40, 131072 (537 MB) 166 and 120.
  a.far = (int)(128e6f / (float)(2 * kTile * q->D * eb * Hkv));
  a.most_units = (int)m.units; a.most_joins = (int)m.joins;
  uint8_t* at = (uint8_t*)ws;
  a.counts = (int*)at; at += 16;
  a.plan = (int4*)at; at += m.units * 64;
  a.joins = (int4*)at; at += m.joins * 32;
  a.tokens = (int*)at; at += align_up64(T * 4, 16);
  a.part_o = (float*)at;
  a.part_ml = a.part_o + Hkv * m.parts * m.slot * q->D;
  hipStream_t st = (hipStream_t)stream;
#define ZC_SA(DT) (q->D == 128 ? launch_shared<DT, 128>(a, st) : launch_shared<DT, 64>(a, st))
  if (q->dtype == ZC_F32) rc = ZC_SA(ZC_F32);
  else if (q->dtype == ZC_F16) rc = ZC_SA(ZC_F16);
  else rc = ZC_SA(ZC_BF16);
#undef ZC_SA
  return rc;
}
