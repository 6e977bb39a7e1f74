// zc_paged_attention: attention of a step's new tokens - one a request or a chunk - over keys and values in pages.
//
// A unit of work is a block of rows and a part of the key tiles it sees.  The host knows neither lengths nor how the
// rows are spread over requests; every wave finds its unit from the lengths alone (find_unit), so nothing has to be
// prepared, and what is long is split by the same rule in every wave.
#include "paged_attention_kernel.hpp"

namespace zc {

struct Unit {
  static constexpr int kFirst = 0;
  int r, qs, nq, kv;            // request, its first row, new tokens, tokens
  bool few;
  int j0, g0, rows;             // token and head of the block's first row, its rows
  int p0, p1;                   // positions of its first and last row
  int first, sink_tiles;        // tile t is t of the first sink_tiles, then first + t - sink_tiles
  int t_lo, t_hi;               // tiles of this unit
  int part, parts;              // which of the parts that the block's tiles are divided into
  uint32_t behind;              // 16 keys from key0 on are behind every window of the block's if key0 - sinks, without sign, is less than this
};

__device__ inline Row row_at(const PagedArgs& a, const Unit& x, int r) { return row_at(a, x.j0, x.g0, r); }
__device__ inline Row row_of(const PagedArgs& a, const Unit& x, int r) { return row_at(a, x, r); }
__device__ inline int position(const Unit& x, int j) { return x.kv - x.nq + j; }
__device__ inline int tile_of(const Unit& x, int t) { return t < x.sink_tiles ? t : x.first + t - x.sink_tiles; }
__device__ inline int tile_at(const Unit& x, int pos) { return pos / kTile - x.first + x.sink_tiles; }
__device__ inline const int32_t* entry_of(const PagedArgs& a, const Unit& x, int key0) { return a.table + x.r * a.row + min(key0 >> a.shift, a.cols - 1); }
__device__ inline int keys_read(const PagedArgs& a, const Unit& x, int end, int key0, int id) { return keys_read(a.n_pages, a.sinks, x.behind, end, key0, id); }
__device__ inline __amdgpu_buffer_rsrc_t keys_at(const PagedArgs& a, const Unit&, const uint8_t* head, uint32_t sB, uint32_t row, int key0, int id, int n) {
  return keys_at(a.shift, head, sB, row, key0, id, n);
}
__device__ inline Seen seen_by(const PagedArgs& a, const Unit&, int p0, int p1) {
  Seen s;
  s.low = a.window ? max(max(p1, 0) - a.window + 1, 0) : 0;
  const int end = max(p0, 0) - 30;                         // (of positions in front of the first key no block is seen)
  s.span = max(end - s.low, 0);
  s.sink = a.window ? min(a.sinks - 31, end) : 0;
  return s;
}
__device__ inline int low_of(const PagedArgs& a, const Unit&, int pos) { return a.window && pos >= 0 ? pos - a.window : -1; }
__device__ inline int sinks_of(const PagedArgs& a, const Unit&) { return a.sinks; }
__device__ inline bool is_whole(const Unit& x) { return x.parts == 1; }
__device__ inline int64_t part_of(const PagedArgs& a, const Unit&, int hk) { return part_row(a, hk, unit_of_grid()); }

struct Request { int qs, nq, kv; };
__device__ inline Request request(const PagedArgs& a, int r) {
  Request x = {0, 0, 0};
  if (r < a.R) {
    const int s = a.q_start[r], e = a.q_start[r + 1], kv = a.kv_len[r];
    x.qs = min(max(s, 0), a.T);
    x.nq = max(min(e, a.T) - x.qs, 0);
    x.kv = min(max(kv, 0), a.cap);
  }
  return x;
}

// The unit with index u of a head.
template <int DT, bool FEW>
__device__ inline bool find_unit(const PagedArgs& a, int u, Unit& x) {
  using B = Blocks<DT, FEW>;
  const int lane = threadIdx.x & 63;
  struct Size { int blocks, tiles, least; };               // row blocks; tiles that one sees, at most, and that make a part
  auto size = [&](const Request& t) {
    const int rows = t.nq * a.G;
    Size s;
    s.blocks = B::few(rows) ? (rows + 31) / 32 : (rows + B::kMany - 1) / B::kMany;
    s.tiles = min((t.kv + kTile - 1) / kTile, a.reach);
    s.least = B::few(rows) ? 2 : 4;                        // (32 keys a wave)
    return s;
  };
  const Request head = request(a, lane);
  int per = INT_MAX;                                       // tiles of a part, at most
  if (a.target) {
    auto work = [&](const Request& t) {
      const Size s = size(t);
      return s.blocks * ((s.tiles + (1 << a.coarse) - 1) >> a.coarse);
    };
    int all = work(head);
    for (int r0 = 64; r0 < a.R; r0 += 64) all += work(request(a, r0 + lane));
    all = __builtin_amdgcn_readlane(wave_inclusive_sum(all), 63);
    per = (int)(((uint32_t)all + a.target - 1) / (uint32_t)a.target) << a.coarse;
  }
  int units = 0;
  for (int r0 = 0; r0 < a.R; r0 += 64) {
    const Request t = r0 ? request(a, r0 + lane) : head;
    const Size s = size(t);
    const int most = max(per, s.least);
    const int parts = s.tiles <= most ? 1 : (int)((uint32_t)(s.tiles - 1) / (uint32_t)most) + 1;
    const int cu = wave_inclusive_sum(s.blocks * parts);
    const uint64_t here = __builtin_amdgcn_ballot_w64(u < units + cu);
    if (here) {
      const int l = __builtin_ctzll(here);
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      x.r = r0 + l;
      x.qs = of(t.qs); x.nq = of(t.nq); x.kv = of(t.kv);
      const int n = of(s.blocks), all_rows = x.nq * a.G;
      x.few = B::few(all_rows);
      x.parts = of(parts);
      const int rest = u - (units + of(cu) - n * x.parts);
      int b = x.parts == 1 ? rest : (int)((uint32_t)rest / (uint32_t)x.parts);
      x.part = rest - b * x.parts;
      b = n - 1 - b;                                       // (a chunk's last rows see the most keys: first)
      const int rb = x.few ? 32 : B::kMany, i0 = b * rb;
      x.j0 = i0 == 0 ? 0 : (int)((uint32_t)i0 / (uint32_t)a.G);
      x.g0 = i0 - x.j0 * a.G;
      x.rows = min(rb, all_rows - i0);
      x.p0 = x.kv - x.nq + x.j0;
      x.p1 = x.kv - x.nq + row_at(a, x, x.rows - 1).j;
      const int low = a.window ? max(0, max(x.p0, 0) - a.window + 1) : 0;      // (a difference of positions in front of the first token may pass 32 bits)
      x.first = low / kTile;
      x.sink_tiles = min((min(a.sinks, low) + kTile - 1) / kTile, x.first);
      const int far = max(x.p0, 0) - a.window - 14;
      x.behind = a.window && far > a.sinks ? far - a.sinks : 0;
      const int tiles = x.p1 < 0 ? 0 : x.sink_tiles + x.p1 / kTile + 1 - x.first;
      x.t_lo = 0;
      x.t_hi = tiles;
      if (x.parts > 1) {
        const int q = (int)((uint32_t)tiles / (uint32_t)x.parts), rem = tiles - q * x.parts;
        x.t_lo = x.part * q + min(x.part, rem);
        x.t_hi = x.t_lo + q + (x.part < rem ? 1 : 0);
      }
      return true;
    }
    units += __builtin_amdgcn_readlane(cu, 63);
  }
  return false;
}

template <int DT, int D>
__global__ __launch_bounds__(256, DT == ZC_F32 && D == 128 ? 1 : 2) void k_paged_attention(PagedArgs a) {
  constexpr int kBytes = DT == ZC_F32 ? RowsMemory<DT, D, 4>::kBytes : kStages<D> * 2 * kTile * Tile<DT, D>::ROWB;
  static_assert(kBytes >= RowsMemory<DT, D, 4>::kBytes, "blocks of few rows find room");
  __shared__ __align__(1024) uint8_t mem[kBytes];
  __shared__ float sum[4][2][64];
  const int hk = blockIdx.x;
  Unit x;
  const bool any = find_unit<DT, false>(a, unit_of_grid(), x);
  if (a.target && threadIdx.x == 0)
    a.todo[(int64_t)hk * a.units + unit_of_grid()] = any && x.part == 0 && x.parts > 1 ? make_int4(x.parts, x.rows, x.qs + x.j0, x.g0) : make_int4(0, 0, 0, 0);
  if (!any) return;
  if constexpr (DT != ZC_F32) {
    if (!x.few) {
      attend_tiles<DT, D>(a, x, hk, mem);
      return;
    }
  }
  attend_rows<DT, D, 4>(a, x, hk, mem, sum);
}

// Eight waves, blocks of 32 rows that are not split (see wide below).
template <int DT, int D>
__global__ __launch_bounds__(512, 2) void k_paged_attention_wide(PagedArgs a) {
  __shared__ __align__(1024) uint8_t mem[RowsMemory<DT, D, 8>::kBytes];
  __shared__ float sum[8][2][64];
  Unit x;
  if (find_unit<DT, true>(a, unit_of_grid(), x)) attend_rows<DT, D, 8>(a, x, blockIdx.x, mem, sum);
}

// ---- the join of split blocks ---------------------------------------------------------------------------
// Four workgroups per unit; those of a unit that a split block begins with join it, every fourth 256 / (D / 4) rows
// each.  D / 4 threads take a row; where rows are few, several such groups share a row's parts and join what they have in LDS.  Bound by two trips to memory:
// 3 us for one token over 4096 (32 heads of 128 channels), 4 for 64 of them, 6 for 4 chunks of 250 to 500 (16 heads of 64), a launch included.
constexpr int kJoinGroups = 4;
template <int DT, int D>
__global__ __launch_bounds__(256) void k_paged_join(PagedArgs a) {
  constexpr int TPR = D / 4, GROUPS = 256 / TPR;
  __shared__ __align__(16) float so[GROUPS][D];
  __shared__ float2 sml[GROUPS];
  const int hk = blockIdx.x, unit = blockIdx.y;
  const int4 todo = a.todo[(int64_t)hk * a.units + unit];
  const int parts = todo.x, rows = todo.y;
  if (parts == 0 || unit + parts > a.units) return;
  const int grp = threadIdx.x / TPR, c = threadIdx.x % TPR * 4;
  const int64_t first = part_row(a, hk, unit);
  for (int row0 = blockIdx.z * GROUPS; row0 < rows; row0 += kJoinGroups * GROUPS) {
    const int n = min(rows - row0, GROUPS);
    int ways = 1;                                          // groups to a row
    while (2 * ways * n <= GROUPS && 2 * ways <= parts) ways *= 2;
    const int way = grp & (ways - 1), row = row0 + grp / ways;
    const bool mine = row < row0 + n;
    float M = kLowestLogit, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (mine) {
      constexpr int U = 4;                                 // parts requested at a time
      for (int s0 = way; s0 < parts; s0 += U * ways) {
        float2 ml[U];
        float4 t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int s = s0 + u * ways;
          const int64_t p = first + (int64_t)(s < parts ? s : s0) * a.slot + row;
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
        for (int v = 1; v < ways; ++v) {
          const float2 ml = sml[grp + v];
          const float4 t = *reinterpret_cast<const float4*>(&so[grp + v][c]);
          const float top = fmaxf(M, ml.x), f0 = __builtin_amdgcn_exp2f(M - top), f = __builtin_amdgcn_exp2f(ml.x - top);
          M = top;
          l = fmaf(ml.y, f, l * f0);
          o.x = fmaf(t.x, f, o.x * f0); o.y = fmaf(t.y, f, o.y * f0); o.z = fmaf(t.z, f, o.z * f0); o.w = fmaf(t.w, f, o.w * f0);
        }
      }
      __syncthreads();
    }
    if (mine && way == 0) store_row<DT>(a, todo.z, todo.w, hk, row, c, M, l, o);
  }
}

// ---- host ---------------------------------------------------------------------------------------------
// How a call's rows are cut: row blocks of a head, at most; units of a head that splitting aims at (0: nothing is split); rows of a
// unit's partial results.
struct Cut { int64_t blocks, target, slot; bool wide; };
constexpr int64_t kUnits = 2560;               // of all heads, that splitting aims at, at most
constexpr int64_t kMostUnits = 4096;           // and that there may be (their partial results, 128 rows of 128 channels: 272 MB)

// Whether rows see too few keys, or the chip has too much to do without, for parts of them to be worth a second launch.  us, split
// and whole, tables of as many tiles as the keys fill: bf16, 32 heads over 8 of 128 channels, one token each, 1 request of 256 keys 8.4 and 6.9,
// of 512 8.5 and 9.2; 16 of 512 14.0 and 10.6, of 1024 18.5 and 15.0, 24 of 100 to 4096 28 and 43; 64 of 300 to 600 33 and 26; 2 chunks of 500 tokens 28.3
// and 18.7, of 1000 45.2 and 41.7; fp32, 16 heads over 4, 4 requests of 256 keys of 64 channels 9.4 and 9.0, of 128 12.5 and 14.0.
static bool whole(int64_t blocks, int64_t tiles, int dtype, int64_t D) {
  if (dtype == ZC_F32) return tiles <= (D == 64 ? 4 : 2);
  return tiles <= (blocks >= 128 ? 16 : blocks >= 64 ? 10 : 6);
}

// Whether eight waves take a block (16-bit types, one block a request): blocks that leave CUs idle and whose keys four waves would take by turns, or that
// have 17 to 32 tiles each and fill the chip less than twice; a split and its join would cost more.  us of four waves, split where that is the rule, and of eight, 32
// heads over 8 of 128 channels, bf16: 1 request of 512 keys 8.6 and 8.1, of 1024 8.5 and 11.1; 4 of 768 9.4 and 10.0; 8 of 1024 13.8 and 12.0; 12 of 51 to 1024 12.4 and 11.7, of 76
// to 1536 12.5 and 14.3; 16 of 512 10.5 and 9.8, of 2048 28.5 and 27.8, of 150 to 3000 18.2 and 22.7; 20 of 102 to 2048 20.0 and 19.3; 32 of 256 9.5 and 10.1; 40 of 512 16.9
// and 20.2, of 1600 56.7 and 52.3, of 102 to 2048 27.3 and 28.3; 60 of 2048 86.2 and 79.5.  16 heads over 4 of 64, fp16: 16 of 512 7.6 and 6.4, of 1024 10.9 and 8.9; 32 of 2048
// 16.7 and 13.7, of 102 to 2048 12.3 and 12.5, of 204 to 4096 16.5 and 19.8; 60 of 2048 26.3 and 22.2; 80 of 1200 21.9 and 19.6, of 1024 16.6 and 17.1.  In fp32 both
// wait for the matrix cores: 2 of 512, 12 heads of 64, 9.7 and 13.4.
static bool wide(int64_t n, int64_t tiles) {
  if (n < 256) return tiles > 2 && tiles <= (n >= 128 ? 32 : n >= 64 ? 16 : 8);
  return n <= 512 && tiles > 16 && tiles <= 32;
}

// Parts of every one of n row blocks that see `tiles` tiles each.  The chip runs them in rounds of what it holds, the last of which is
// shorter where CUs are left with one workgroup or none; a part costs the way of its rows' results through memory.  Of blocks
// that fill the chip two parts at most: parts of one block read different keys at a time, which the L2s then hold fewer of.
// us at 1, 2, 3 and 4 parts, bf16, 32 heads over 8 of 128 channels: 2048 tokens over 32768 (512 blocks) 1120, 1139, 1151 and 1182, 2500 (632) 1526,
// 1353, 1418 and 1408; 1200 over 8192 (304) 220, 217, 197 and 201; 512 over 8192 (128) 163, 98, 102 and 90; 40 heads, 2048 over 16384 (640) 794, 790, 866
// and 881; fp16 of 64 channels, 20 tokens and 4 chunks of 250 to 500 over up to 4001 (202) 52, 37, 33.5 and 38.
static int64_t parts_of(int64_t n, int64_t tiles, int dtype, int64_t D) {
  // workgroups at a time; us of a tile in each of them; us that a part's results take of the memory's time
  struct Kind { int64_t places; double tile, part; int least; };
  const Kind k = dtype == ZC_F32 ? (D == 64 ? Kind{512, 3.3, 0.0033, 2} : Kind{256, 2.2, 0.0065, 2})
                                 : (D == 64 ? Kind{768, 1.7, 0.013, 4} : Kind{512, 2.0, 0.026, 4});
  const int64_t most = n >= k.places ? 2 : 256;
  int64_t best = 1;
  double least = 0.0;
  for (int64_t p = 1; p <= most && (p == 1 || (p * n <= kUnits && k.least * p <= tiles)); ++p) {
    const int64_t rounds = p * n / k.places;
    const double last = (double)(p * n % k.places) / (double)k.places;
    const double all = (double)rounds + (last == 0.0 ? 0.0 : last <= 0.5 ? 0.57 : 0.95);
    const double t = all * (double)tiles * k.tile / (double)p + (p > 1 ? 3.0 + (double)(p * n) * k.part : 0.0);
    if (p == 1) least = 0.95 * t;
    else if (t < least) { least = t; best = p; }
  }
  return best;
}

// keys: a request's, at most; INT64_MAX: as many as cost the most workspace.
static Cut cut_of(int64_t R, int64_t T, int64_t G, int64_t Hkv, int dtype, int64_t D, int64_t keys, int64_t window, int64_t sinks) {
  Cut c;
  c.wide = false;
  c.slot = dtype == ZC_F32 || T * G <= 64 ? 32 : 128;
  // (a request has one block that is not full; where blocks of 128 rows are the rule, one of 33 to 64 rows is two of 32)
  const int64_t with = R < T ? R : T, two = T * G / 33;
  c.blocks = T * G / c.slot + with + (c.slot == 32 ? 0 : two < with ? two : with);
  const bool few = T * G <= 64 * R;
  const int64_t n = few ? c.blocks * Hkv : ceil_div64(T * G, c.slot) * Hkv;
  if (few ? n > 1024 : n > kUnits / 2 || c.blocks * Hkv + kUnits > kMostUnits) { c.target = 0; return c; }
  // Single tokens: so many that, with the half part that a block has too much on average, they fill the chip once - two workgroups a CU -
  // or twice where blocks are many.  us at 512 units and here: bf16, 32 heads over 8 of 128 channels, 64 requests of 64 to 8192 tokens 108.7 and 104.3,
  // 24 of 100 to 4096 28.2 and 24.5, 6 of 500 to 16000 44.9 and 41.0, 12 of 4000 45.6 and 41.8, 16 under a window of 4096 57.5 and 52.6, 8 of
  // 8192 53.4 both, 1 of 32768 33.5 both, 48 of 3000 108.5 and 112.0; fp16, 16 heads over 4, 20 of 700 to 20000 54.5 and 49.4.
  // (1 of 32768 at 256, 768 and 1024 units 32.9, 36.0 and 39.1; 4 of 20000 to 32768 105, 82 and 84; 3 of 1000 to 9000, 16 heads, fp32 104, 83 and 89.)
  // One a CU where requests have two blocks, which read the same keys: 256 and 512 units, 16 new tokens of 4 requests of 4096 20.0 and 20.6, of 16 55.6
  // and 60.7, of one of 8192 15.8 and 19.5.
  const int64_t all = with * Hkv, single = T * G > 32 * R ? 256 : (all > 320 ? 1024 : 512) - all / 2;
  if (keys == INT64_MAX) {
    c.target = ceil_div64(few ? single : kUnits, Hkv);
    return c;
  }
  if (window && window + sinks < keys) keys = window + sinks;
  const int64_t tiles = ceil_div64(keys, kTile);
  if (dtype != ZC_F32 && T * G <= 32 * with) {
    if (wide(with * Hkv, tiles)) {
      c.blocks = T * G / 32 + with;
      c.target = 0;
      c.wide = true;
      return c;
    }
    // (so many blocks need no split either, us split and not: 90 requests of 2048 tokens, 32 heads over 8 of 128 channels 127 and 116, of 102 to 2048 61.4 and 57.8, of
    // 204 to 4096 92 and 112; 8 heads of 64 69 and 60, 36.7 and 35.5; 20 of 102 to 2048, 40 heads of 128 73.4 and 75.3, of 60 to 1200 44.3 and 39.8)
    if (with * Hkv > 512 && tiles <= 32) {
      c.target = 0;
      return c;
    }
  }
  if (whole(n, tiles, dtype, D)) {
    c.target = 0;
  } else if (few) {
    c.target = ceil_div64(single, Hkv);
  } else {
    // (blocks of a prompt that begins with this step see half of its keys on average, the longest go first: rounds even out)
    const int64_t past = keys > 2 * T ? keys - 2 * T : 0;
    const int64_t p = parts_of(n, n < 512 ? tiles : ceil_div64(past, kTile), dtype, D);
    // Of several requests one may be far longer than the others: no unit takes more than its share of a round.  us without and with:
    // 2000 new tokens of a fresh prompt and one token each of three of 1000 and one of 65536 tokens (32 heads over 8 of 128 channels) 588 and 115;
    // of 2000 over 4000 and 31 of 3000 191 and 195, 20 tokens and 4 chunks of 250 to 500 over up to 4001 (fp16) 87 and 91.
    const int64_t least = R > 1 && tiles >= 32 ? 512 : 0, units = p > 1 && p * n > least ? p * n : least;
    c.target = ceil_div64(units, Hkv);
  }
  return c;
}
static size_t workspace_of(const Cut& c, int64_t Hkv, int64_t D) {
  return c.target ? (size_t)(c.target + c.blocks) * Hkv * (c.slot * (D + 2) * sizeof(float) + sizeof(int4)) : 0;
}

template <int DT, int D>
static int launch_paged(PagedArgs& a, bool wide, hipStream_t st) {
  const auto grid = [&](int64_t n) { return dim3((unsigned)a.Hkv, (unsigned)(n < 65535 ? n : 65535), (unsigned)ceil_div64(n, 65535)); };
  if constexpr (DT != ZC_F32) {
    if (wide) {
      hipLaunchKernelGGL((k_paged_attention_wide<DT, D>), grid(a.units), dim3(512), 0, st, a);
      ZC_LAUNCH_CHECK();
      return ZC_OK;
    }
  }
  hipLaunchKernelGGL((k_paged_attention<DT, D>), grid(a.units), dim3(256), 0, st, a);
  ZC_LAUNCH_CHECK();
  if (a.target) {
    const dim3 joins((unsigned)a.Hkv, (unsigned)a.units, (unsigned)kJoinGroups);     // (units: at most kMostUnits)
    hipLaunchKernelGGL((k_paged_join<DT, D>), joins, dim3(256), 0, st, a);
    ZC_LAUNCH_CHECK();
  }
  return ZC_OK;
}

}  // namespace zc

using namespace zc;

// (the larger of what fp32 and 16-bit calls take: the types' blocks differ)
extern "C" size_t zc_paged_attention_workspace(int64_t R, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
  if (R <= 0 || T <= 0 || Hkv <= 0 || Hq < Hkv || Hq % Hkv || D <= 0) return 0;
  const int64_t G = Hq / Hkv;
  const size_t x = workspace_of(cut_of(R, T, G, Hkv, ZC_F32, D, INT64_MAX, 0, 0), Hkv, D);
  const size_t y = workspace_of(cut_of(R, T, G, Hkv, ZC_F16, D, INT64_MAX, 0, 0), Hkv, D);
  return x > y ? x : y;
}

extern "C" int zc_paged_attention(const zc_tensor4* q, const zc_tensor4* k_pages, const zc_tensor4* v_pages, const int32_t* block_table,
                                  int64_t row_stride, int64_t max_blocks, const int32_t* q_start, const int32_t* kv_len, int64_t R,
                                  int32_t window, int32_t sinks, float sm_scale, const zc_tensor4* out, float* lse,
                                  void* ws, size_t ws_bytes, void* stream) {
  int rc = zc_validate_pages(k_pages, v_pages);
  if (rc) return rc;
  rc = zc_validate_heads(q, k_pages);
  if (rc) return rc;
  rc = zc_validate_heads(out, k_pages);
  if (rc) return rc;
  if (q->H != out->H || q->L != out->L || q->H % k_pages->H || !zc_rows_apart(out)) return ZC_ERR_INVALID_ARG;
  if (R < 0 || window < 0 || sinks < 0 || !(sm_scale >= 0.f) || !(sm_scale * kLog2e <= -kLowestLogit)) return ZC_ERR_INVALID_ARG;
  if (max_blocks < 0 || row_stride < max_blocks) return ZC_ERR_INVALID_ARG;
  if (q->L == 0 || R == 0) return ZC_OK;
  if (!q_start || !kv_len || (max_blocks > 0 && !block_table)) return ZC_ERR_INVALID_ARG;
  for (const void* p : {(const void*)block_table, (const void*)q_start, (const void*)kv_len, (const void*)lse})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ZC_ERR_INVALID_ARG;
  const int64_t T = q->L, Hkv = k_pages->H, G = q->H / Hkv;
  if (R >= (1 << 24) || max_blocks > 0x7fffffff || T > 0x7fffffff / q->H || q->H > 65535 || G > 4096) return ZC_ERR_UNSUPPORTED;
  const int64_t page = k_pages->L, room = max_blocks > 0x7fff0000 / page ? 0x7fff0000 : max_blocks * page;
  if (window >= room) window = 0;                    // (every row sees all it could)
  if (sinks > room) sinks = (int32_t)room;
  const Cut cut = cut_of(R, T, G, Hkv, q->dtype, q->D, room, window, sinks);
  if ((cut.target + cut.blocks) * Hkv > 0xffffff) return ZC_ERR_UNSUPPORTED;
  const size_t need = zc_paged_attention_workspace(R, T, q->H, Hkv, q->D);
  if (workspace_of(cut, Hkv, q->D) > need) return ZC_ERR_WORKSPACE;     // (never: the size is that of the finest cut)
  if (need && (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 15))) return ZC_ERR_WORKSPACE;

  const int64_t eb = elem_bytes(q->dtype);
  PagedArgs a;
  a.q = (const uint8_t*)q->ptr; a.k = (const uint8_t*)k_pages->ptr; a.v = (const uint8_t*)v_pages->ptr; a.o = (uint8_t*)out->ptr;
  a.q_sH = q->sH * eb; a.q_sT = q->sL * eb; a.o_sH = out->sH * eb; a.o_sT = out->sL * eb;
  a.k_sB = (uint32_t)(k_pages->sB * eb); a.k_sH = k_pages->sH * eb; a.v_sB = (uint32_t)(v_pages->sB * eb); a.v_sH = v_pages->sH * eb;
  a.k_row = (uint32_t)(k_pages->sL * eb); a.v_row = (uint32_t)(v_pages->sL * eb);
  // (a table without columns holds no token: any readable word stands for its pages)
  a.table = max_blocks ? block_table : q_start; a.q_start = q_start; a.kv_len = kv_len; a.row = max_blocks ? row_stride : 0;
  a.cols = max_blocks ? (int)max_blocks : 1; a.shift = __builtin_ctzll((unsigned long long)page); a.n_pages = (int)k_pages->B; a.cap = (int)room;
  a.R = (int)R; a.T = (int)T; a.Hkv = (int)Hkv; a.G = (int)G;
  a.window = window;
  a.sinks = sinks;
  a.scale_log2 = (sm_scale == 0.f ? 1.0f / sqrtf((float)q->D) : sm_scale) * kLog2e;
  a.lse = lse;
  a.target = (int)cut.target;
  a.units = (int)(cut.target + cut.blocks);
  a.slot = (int)cut.slot;
  a.over_G = G == 1 ? 0 : (uint32_t)(((1ull << 32) + G - 1) / G);
  // (a block's rows are of slot / G + 2 tokens at most)
  a.reach = a.window ? (int)((a.window + cut.slot / G + 2 + kTile - 2) / kTile + 1 + (a.sinks + kTile - 1) / kTile) : 0x7fffffff;
  a.coarse = 0;
  while ((cut.blocks * (room / kTile + 1)) >> a.coarse > 0x3fffffff) ++a.coarse;
  const int64_t parts = (cut.target + cut.blocks) * Hkv;
  a.todo = (int4*)ws;
  a.part_o = cut.target ? (float*)((int4*)ws + parts) : nullptr;
  a.part_ml = cut.target ? a.part_o + parts * cut.slot * q->D : nullptr;
  hipStream_t st = (hipStream_t)stream;
#define ZC_PA(DT) (q->D == 128 ? launch_paged<DT, 128>(a, cut.wide, st) : launch_paged<DT, 64>(a, cut.wide, st))
  if (q->dtype == ZC_F32) rc = ZC_PA(ZC_F32);
  else if (q->dtype == ZC_F16) rc = ZC_PA(ZC_F16);
  else rc = ZC_PA(ZC_BF16);
#undef ZC_PA
  return rc;
}
