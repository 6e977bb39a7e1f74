// zc_paged_scores: the attention weight that every cached token gathers, carried on from step to step (Eq. 7 over the pages).
//
// The rows of a request and a KV head are its new tokens times the G query heads of the group, token after token.  Given their
// normalisers the weight of a token is one sum over rows of exp(logit - lse), so a sweep over the keys is all there is:
//   logits  D[row][key] = sum_c Q[row][c] K[key][c]        (A = Q rows, B = K block)
// puts a key in a lane (column lane & 31) and its rows in the accumulators: the sum over rows is lane-local.  No result is split
// over workgroups, so there are no partial sums, and the order of every sum is fixed.  Logits, weights and sums are fp32.
//
// A unit of work is a range of a request's key tiles.  As for the paged attention the host knows neither lengths nor how rows
// are spread over requests: every wave finds its unit from the lengths.
#include <limits.h>

#include <type_traits>

#include "paged_args.hpp"
#include "paged_keys.hpp"

namespace zc {

struct ScoreArgs {
  const uint8_t *q, *k;
  int64_t q_sH, q_sT, k_sH;                     // bytes
  uint32_t k_sB, k_row;                         // bytes from a page, a token to the next
  const int32_t *table, *q_start, *kv_len;
  int64_t row;                                  // of the table, in entries
  int cols, shift, n_pages, cap;                // blocks of the table; page size; pages; tokens a row of the table has room for
  int R, T, Hkv, G, window, sinks;
  float scale_log2, decay;
  const float* lse;                             // [Hq, T]
  float* scores;                                // [page][head][row]
  int near_rows;                                // the rows of the four waves' transfers at a time lie within 4 GB
  float target;                                 // units a head's keys are split into, about
  uint32_t over_G;                              // ceil(2^32 / G)
};

// A request's keys go in tiles of 128, or 64 where those are few: of up to 64 rows a wave takes every fourth 32 keys, of more
// the four waves share a tile.
constexpr int kScoreTile = 128;
// Tiles of chunks and heads below which they are halved: more workgroups, which all take every row.  us of 128 and 64 keys a
// tile (32 heads over 8 of 128 channels, bf16): a prompt of 2048 103 and 72, four of 500 42 and 28, 500 tokens over 4096 (256
// tiles) 44 and 35, 1000 that see 4096 each (328) 98 and 77, 300 over 6000 (376) 37 and 46, 500 over 8192 (512) 53 and 69;
// fp32, 500 over 4096 (16 heads over 4) 190 and 115.
constexpr float kFewTiles = 340.f;

struct Span {
  int r, qs, nq, kv;            // request, its first row, new tokens, tokens
  int first, sink_tiles;        // tile t is t of the first sink_tiles, then first + t - sink_tiles
  int t_lo, t_hi;               // tiles of this unit
  int shift;                    // of a tile's keys: 7 or 6
  uint32_t behind;              // 16 keys from key0 on are behind every window if key0 - sinks, without sign, is less than this
};
__device__ inline int tile_of(const Span& x, int t) { return t < x.sink_tiles ? t : x.first + t - x.sink_tiles; }

// A copy that the compiler knows nothing of: what is computed from it is computed where it is used, not kept in registers across a loop.
__device__ inline uint32_t opaque(uint32_t x) { asm volatile("" : "+v"(x)); return x; }

// Unit u of a head; false: there are fewer.
__device__ inline bool find_span(const ScoreArgs& a, int u, Span& x) {
  const int lane = threadIdx.x & 63;
  struct Part { int qs, nq, kv, first, sink_tiles, tiles, passes; float work; };         // passes: of 64 rows over a tile; work: of all tiles
  int shift = 7;
  const auto part = [&](int r) {
    Part p = {0, 0, 0, 0, 0, 0, 1, 0.f};
    if (r >= a.R) return p;
    const int s = a.q_start[r], e = a.q_start[r + 1], kv = a.kv_len[r];
    p.qs = min(max(s, 0), a.T);
    p.nq = max(min(e, a.T) - p.qs, 0);
    p.kv = min(max(kv, 0), a.cap);
    // (weights that fade change every token's score, seen or not)
    const int p0 = max(p.kv - p.nq, 0), reached = a.window ? max(0, p0 - a.window + 1) : 0, low = a.decay == 1.f ? reached : 0;
    const int up = (1 << shift) - 1;
    p.first = low >> shift;
    p.sink_tiles = min((min(a.sinks, low) + up) >> shift, p.first);
    if (p.nq) p.tiles = p.sink_tiles + ((p.kv + up) >> shift) - p.first;
    p.passes = (int)(((int64_t)p.nq * a.G + 63) / 64);
    const int fade = min((reached >> shift) - p.first, p.tiles);     // tiles that no window reaches
    p.work = (float)(p.tiles - fade) * (float)p.passes + (float)fade;
    return p;
  };
  Part head = part(lane);
  float all = head.work, chunks = head.passes > 1 ? (float)head.tiles : 0.f;
  for (int r0 = 64; r0 < a.R; r0 += 64) {
    const Part p = part(r0 + lane);
    all += p.work;
    chunks += p.passes > 1 ? (float)p.tiles : 0.f;
  }
  all = wave_sum(all);
  if (__builtin_amdgcn_ballot_w64(chunks > 0.f) && __builtin_amdgcn_readfirstlane(wave_sum(chunks) * (float)a.Hkv < kFewTiles)) {
    shift = 6;
    head = part(lane);
    all *= 2.f;
  }
  // Work of a unit: as many units as the chip holds twice, where work is little as it holds once.  us at 512, 1024 and 2048
  // units (single tokens in the kernel of chunks): 64 tokens over 64 to 8192 (32 heads over 8 of 128 channels, bf16) 74, 65
  // and 66, 16 over up to 1694 (8 heads of 64) 14.6, 17.2 and 23.3, 3 requests with 6 tokens over up to 3840 (12 of 64) 11.1,
  // 14.7 and 14.7, 2048 tokens over 16384 295, 295 and 298.
  const float share = all / a.target, per = fmaxf(share, fminf(2.f * share, 5.f));
  int units = 0;
  for (int r0 = 0; r0 < a.R; r0 += 64) {
    const Part p = r0 ? part(r0 + lane) : head;
    const int each = max((int)fminf(ceilf(per / (float)max(p.passes, 1)), 1e9f), 1);     // tiles
    const int parts = p.tiles ? (int)((uint32_t)(p.tiles - 1) / (uint32_t)each) + 1 : 0;
    const int cu = wave_inclusive_sum(parts);
    const uint64_t here = __builtin_amdgcn_ballot_w64(u < units + cu);
    if (here) {
      const int l = __builtin_ctzll(here);
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      const int n = of(parts), tiles = of(p.tiles), half = (int)(0.25f * a.target);
      int b = u - (units + of(cu) - n);
      // (a chunk's first keys are seen by most rows: where all units run at once, the second on a CU is one of the last; a
      // window evens that out by itself.  us of units in order and so, bf16, 32 heads over 8 of 128 channels: a prompt of 4096
      // 161 and 154, 2048 over 32768 that see 4096 each 114 and 139)
      if (!a.window && n > half && n <= 2 * half && b >= half) b = n - 1 - (b - half);
      x.r = r0 + l;
      x.qs = of(p.qs); x.nq = of(p.nq); x.kv = of(p.kv);
      x.first = of(p.first); x.sink_tiles = of(p.sink_tiles);
      const int q = (int)((uint32_t)tiles / (uint32_t)n), rem = tiles - q * n;
      x.t_lo = b * q + min(b, rem);
      x.t_hi = x.t_lo + q + (b < rem ? 1 : 0);
      x.shift = shift;
      const int far = max(x.kv - x.nq, 0) - a.window - 14;
      x.behind = a.window && far > a.sinks ? far - a.sinks : 0;
      return true;
    }
    units += __builtin_amdgcn_readlane(cu, 63);
  }
  return false;
}

// Row v (of g0 on) of a unit: its token after j0, and head.
__device__ inline int2 row_of(const ScoreArgs& a, int j0, int v) {
  const int j = a.G == 1 ? v : (int)__umulhi((uint32_t)v, a.over_G);           // (exact while v G < 2^32)
  return make_int2(j0 + j, v - j * a.G);
}

// How far from a key a row may stand that sees it, at its position or behind it.
__device__ inline uint32_t reach_of(const ScoreArgs& a, int key) { return !a.window || key < a.sinks ? 0x80000000u : (uint32_t)a.window; }

__device__ inline int2 row_of_any(const ScoreArgs& a, int v) {
  const int j = (int)((uint32_t)v / (uint32_t)a.G);
  return make_int2(j, v - j * a.G);
}

// A row's normaliser in log2 units; of one that sees nothing (-inf) so that its weights are 0.
__device__ inline float norm_of(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// The score of token `key` of request x.r and head hk (null: it has no page).
__device__ inline float* score_at(const ScoreArgs& a, const Span& x, int hk, int key) {
  const int id = a.table[x.r * a.row + (key >> a.shift)];
  return (uint32_t)id < (uint32_t)a.n_pages ? a.scores + (((int64_t)id * a.Hkv + hk) << a.shift) + (key & ((1 << a.shift) - 1)) : nullptr;
}

// Accumulator v of a 32 x 32 product that was summed in N (of fp32, four: the roundings of one chain of D products are most of
// a logit's error).
template <int N> __device__ inline float logit(const v16f (&p)[N], int v) {
  if constexpr (N == 4) return (p[0][v] + p[1][v]) + (p[2][v] + p[3][v]);
  else return p[0][v];
}

// ---- up to 64 rows: single tokens ------------------------------------------------------------------
// Bound by memory.  A wave has a place for one K block in LDS; the next is requested when it has been multiplied, and the
// rows' operands stay in registers.  64 tokens over 64 to 8192 (8 KV heads of 128 channels, bf16, 274 MB): 57 us, 4.8 TB/s.
// 33 to 64 rows as two sets over one block, against the way of chunks (16 tokens of each of 16 requests over 4096): 49 and 66
// us, 9 tokens 43 and 66.
template <int DT, int D> struct FewMemory { static constexpr int kBlock = 32 * Tile<DT, D>::ROWB, kBytes = 4 * kBlock; };
// ANY: any number of rows, 32 at a time, of which every wave has normalisers and positions for itself.
template <int DT, int D, int SETS, bool ANY>
__device__ __forceinline__ void score_rows(const ScoreArgs& a, const Span& x, int hk, uint8_t* mem, float* norms, int* where) {
  using T = Tile<DT, D>;
  constexpr int BLK = FewMemory<DT, D>::kBlock, PG = 16 / T::RPI;
  constexpr int SUMS = DT == ZC_F32 ? 4 : 1;
  const int tid = (int)opaque(threadIdx.x), lane = tid & 63, r = lane & 31, kh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint8_t* kb = a.k + hk * a.k_sH;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)mem + w * BLK;
  const int32_t* table = a.table + x.r * a.row;

  int voff[PG];
#pragma unroll
  for (int j = 0; j < PG; ++j) {
    const int row = j * T::RPI + lane / T::CPR;
    voff[j] = (int)(row * a.k_row) + (((lane % T::CPR) ^ T::swz(row)) << 4);
  }
  const int up = x.shift - 5, blocks = (x.t_hi - x.t_lo) << up;
  const auto key_of = [&](int b) { return (tile_of(x, x.t_lo + (b >> up)) << x.shift) + 32 * (b & ((1 << up) - 1)); };
  // A block's keys are requested, and this lane's score so far.
  float* to = nullptr;
  float old = 0.f;
  const auto issue = [&](int key0) {
    int id[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int k16 = key0 + 16 * g;
      id[g] = page_of(table, a.cols, a.shift, k16);
      const int n = keys_read(a.n_pages, a.sinks, x.behind, x.kv, k16, id[g]);
      move_keys<PG>(lds + g * 16 * T::ROWB, keys_at(a.shift, kb, a.k_sB, a.k_row, k16, id[g], n), voff);
    }
    const int key = key0 + r, mine = r < 16 ? id[0] : id[1];
    to = nullptr;
    old = 0.f;
    if (kh == 0 && key < x.kv && (uint32_t)mine < (uint32_t)a.n_pages) {
      to = a.scores + (((int64_t)mine * a.Hkv + hk) << a.shift) + (key & ((1 << a.shift) - 1));
      if (key < x.kv - x.nq && a.decay != 0.f) old = *to;
    }
  };
  int b = w, key0 = key_of(b);
  if (b < blocks) issue(key0);

  // the rows, straight into operand registers; their normalisers
  const int rows = x.nq * a.G;
  u32x4 qf[SETS][T::NKC];
  const auto rows_from = [&](int row0, u32x4 (&to)[T::NKC]) {      // (places behind the last row: that row once more, of no weight; zeros would make NaN of infinite keys)
    const int2 me = ANY ? row_of_any(a, min(row0 + r, rows - 1)) : row_of(a, 0, min(row0 + r, rows - 1));
    const uint8_t* qr = a.q + (int64_t)(hk * a.G + me.y) * a.q_sH + (int64_t)(x.qs + me.x) * a.q_sT + kh * 16;
#pragma unroll
    for (int kc = 0; kc < T::NKC; ++kc) to[kc] = *reinterpret_cast<const u32x4*>(qr + kc * 32);
  };
  const auto place = [&](int at, int row) {
    const int2 me = ANY ? row_of_any(a, row) : row_of(a, 0, row);
    norms[at] = row < rows ? norm_of(a.lse[(int64_t)(hk * a.G + me.y) * a.T + x.qs + me.x]) : INFINITY;
    where[at] = row < rows ? x.kv - x.nq + me.x : -1;
  };
  if constexpr (ANY) {
    norms += 32 * w;
    where += 32 * w;
  } else {
#pragma unroll
    for (int s = 0; s < SETS; ++s) rows_from(32 * s, qf[s]);
    __syncthreads();                             // (the unit before is done with the normalisers)
    if (tid < 32 * SETS) place(tid, tid);
    __syncthreads();
  }
  typedef __attribute__((address_space(3))) const uint8_t* lds_ptr;
  const uint32_t kaddr = lds + T::slot(r, kh);
  const int p0 = x.kv - x.nq, p1 = x.kv - 1;
  wait_all_loads();
  for (; b < blocks; b += 4) {
    const int key = key0 + r, next = b + 4 < blocks ? key_of(b + 4) : 0;
    const int seen_from = p1 - a.window;                                       // keys above it are in every row's window
    const uint32_t reach = reach_of(a, key);
    const bool whole = key0 + 31 <= p0 && (!a.window || key0 > seen_from || key0 + 31 < a.sinks);
    const bool any = (uint32_t)(key0 - a.sinks) >= x.behind || (uint32_t)(key0 + 16 - a.sinks) >= x.behind;      // of the block's keys a row may see some
    wait_vmem<0>();
    wait_all_loads();
    float* const put = to;
    const float before = old;
    float sum = 0.f;
    v16f acc[SETS][SUMS] = {};
    const auto multiply = [&] {
#pragma unroll
      for (int kc = 0; kc < T::NKC; ++kc) {
        const u32x4 kf = *(__attribute__((address_space(3))) const u32x4*)(lds_ptr)(uintptr_t)(kaddr ^ (32 * kc));
#pragma unroll
        for (int s = 0; s < SETS; ++s) mma_chunk<DT>(acc[s][kc % SUMS], qf[s][kc], kf);
      }
    };
    const auto weigh = [&](int there) {
#pragma unroll
      for (int v4 = 0; v4 < 4 * SETS; ++v4) {
        if (8 * v4 >= there) break;
        const float4 nv = *reinterpret_cast<const float4*>(&norms[8 * v4 + 4 * kh]);
        const int4 pv = *reinterpret_cast<const int4*>(&where[8 * v4 + 4 * kh]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float e = __builtin_amdgcn_exp2f(fmaf(logit<SUMS>(acc[v4 >> 2], 4 * (v4 & 3) + u), a.scale_log2, -(&nv.x)[u]));
          sum += whole || (uint32_t)((&pv.x)[u] - key) < reach ? e : 0.f;
        }
      }
    };
    if constexpr (ANY) {
      float total = 0.f;                         // (of the rows before these 32)
      if (any)
        for (int row0 = 0; row0 < rows; row0 += 32) {
          total += sum;
          sum = 0.f;
          rows_from(row0, qf[0]);
          if (lane < 32) place(lane, row0 + lane);
          wait_all_loads();
          __builtin_amdgcn_wave_barrier();
          multiply();
          weigh(rows - row0);
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int i = 0; i < SUMS; ++i) acc[0][i] = v16f{};
        }
      sum += total;
      dma_reuse_fence();
      if (b + 4 < blocks) issue(next);
    } else {
      if (any) multiply();
      dma_reuse_fence();
      if (b + 4 < blocks) issue(next);
      if (any) weigh(rows);
    }
    if (any) sum += __shfl_xor(sum, 32);
    if (put) *put = fmaf(before, a.decay, sum);
    key0 = next;
  }
}

// f with two conditions as types.
template <typename F> __device__ __forceinline__ void with(bool x, bool y, const F& f) {
  if (x && y) f(std::true_type{}, std::true_type{});
  else if (x) f(std::true_type{}, std::false_type{});
  else if (y) f(std::false_type{}, std::true_type{});
  else f(std::false_type{}, std::false_type{});
}

// ---- more rows: chunks -----------------------------------------------------------------------------
// The waves take half of a tile's keys and 32 of every 64 rows each: K operands stay in registers, rows stream through LDS,
// 128 (fp32 64) at a time, one tile ahead.  Bound by the matrix pipe and the exponentials beside it, which are issued between
// the products of the next 32 keys (16-bit types) or of the other half: 2048 tokens over 16384 (32 heads over 8 of 128
// channels, bf16) 294 us, 870 TFLOP/s of logits that are seen.  256 VGPRs allow two workgroups a CU; three spill.
template <int DT, int D> struct ManyMemory { static constexpr int kRows = DT == ZC_F32 ? 64 : 128, kTileB = kRows * Tile<DT, D>::ROWB, kBytes = 2 * kTileB; };
constexpr int kMostRows = 128;
template <int DT, int D, int KEYS>
__device__ __forceinline__ void score_tiles(const ScoreArgs& a, const Span& x, int hk, uint8_t* mem, float* norms, int* where, float (*sums)[kScoreTile]) {
  using T = Tile<DT, D>;
  constexpr int QT = ManyMemory<DT, D>::kRows, TILE_B = ManyMemory<DT, D>::kTileB, NI = QT / T::RPI / 4, PG = 16 / T::RPI;
  static_assert(2 * QT >= kScoreTile, "K passes through both row buffers");
  // Places of a tile's normalisers.  A wave stores those of tile n + 1 in front of the barrier behind which all are done with
  // tile n.  Of 16-bit types only its own are read until then, of fp32 those of tile n - 1 too (`pending`): with two places
  // one wave could overwrite what another still reads.
  constexpr int PLACES = 2 * kMostRows / QT;
  static_assert(PLACES >= (DT == ZC_F32 ? 3 : 2) && (PLACES & (PLACES - 1)) == 0, "nobody reads what is overwritten");
  constexpr int SUMS = DT == ZC_F32 ? 4 : 1, TILE = 64 * KEYS;
  const int tid = (int)opaque(threadIdx.x), lane = tid & 63, r = lane & 31, kh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), rw = w >> 1, kw = w & 1;       // rows 32 rw on of 64, keys 32 KEYS kw on of the tile's
  const uint8_t* kb = a.k + hk * a.k_sH;
  const uint8_t* qb = a.q + (int64_t)hk * a.G * a.q_sH + (int64_t)x.qs * a.q_sT;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)mem;
  const int32_t* table = a.table + x.r * a.row;
  const int past = x.kv - x.nq;                  // position of the first row's token
  const uint32_t rows = (uint32_t)x.nq * a.G;
  typedef __attribute__((address_space(3))) const uint8_t* lds_ptr;
  using lds_u32x4 = __attribute__((address_space(3))) const u32x4;

  for (int t = x.t_lo; t < x.t_hi; ++t) {
    const int key0 = tile_of(x, t) * TILE;
    // ---- K to registers, by way of both row buffers
    int voff[PG];
    const int kl = (int)opaque(lane);
#pragma unroll
    for (int j = 0; j < PG; ++j) {
      const int row = j * T::RPI + kl / T::CPR;
      voff[j] = (int)(row * a.k_row) + (((kl % T::CPR) ^ T::swz(row)) << 4);
    }
    __syncthreads();                             // (the tile before is done with LDS)
#pragma unroll
    for (int g = 0; g < KEYS; ++g) {
      const int at = 16 * KEYS * w + 16 * g, k16 = key0 + at, id = page_of(table, a.cols, a.shift, k16);
      move_keys<PG>(lds + at * T::ROWB, keys_at(a.shift, kb, a.k_sB, a.k_row, k16, id, keys_read(a.n_pages, a.sinks, x.behind, x.kv, k16, id)), voff);
    }
    float* to = nullptr;
    float old = 0.f;
    if (tid < TILE && key0 + tid < x.kv) {
      to = score_at(a, x, hk, key0 + tid);
      if (to && key0 + tid < past && a.decay != 0.f) old = *to;
    }
    wait_vmem<0>();
    wait_all_loads();
    __syncthreads();
    u32x4 kf[KEYS][T::NKC];
#pragma unroll
    for (int n = 0; n < KEYS; ++n)
#pragma unroll
      for (int kc = 0; kc < T::NKC; ++kc)
        kf[n][kc] = *reinterpret_cast<lds_u32x4*>((lds_ptr)(uintptr_t)((lds + T::slot(r, kh)) ^ (32 * kc)) + (32 * KEYS * kw + 32 * n) * T::ROWB);

    // ---- rows that see some of these keys: up to the last row, or the last whose window reaches them
    const int key1 = min(key0 + TILE, x.kv) - 1;
    int j_first = max(key0 - past, 0), j_end = x.nq;
    if (a.window && key0 >= a.sinks) j_end = (int)min((int64_t)x.nq, (int64_t)key1 + a.window - past);
    const uint32_t i_first = (uint32_t)j_first * a.G / QT * QT, i_end = (uint32_t)max(j_end, 0) * a.G;
    int j0 = (int)(i_first / (uint32_t)a.G), g0 = (int)(i_first - (uint32_t)j0 * a.G);     // token and head of the tile's first row
    // Rows to LDS, and this thread's normaliser to a register.  Where 16 rows are whole tokens all tiles but one that is not
    // full lie alike: a base that advances, and one offset a lane.
    constexpr bool SAME = 4 * T::RPI % 16 == 0;  // (the swizzle repeats from one of a wave's transfers to the next)
    const bool even = SAME && 16 % a.G == 0 && a.near_rows;
    uint32_t off = 0;
    if (even) {
      const int row = w * T::RPI + lane / T::CPR;
      const int2 me = row_of(a, 0, row);
      off = (uint32_t)(me.y * a.q_sH + me.x * a.q_sT) + (((lane % T::CPR) ^ T::swz(row)) << 4);
    }
    const int hop = 4 * T::RPI / a.G, tokens = QT / a.G;                       // of a transfer to the next, of a tile
    const uint8_t* base = qb + (int64_t)j0 * a.q_sT;
    const int64_t q_hop = hop * a.q_sT, q_step = tokens * a.q_sT - NI * q_hop;
    const int2 at0 = row_of(a, j0, g0 + (tid < QT ? tid : 0));
    const float* norm_from = a.lse + (int64_t)(hk * a.G + at0.y) * a.T + x.qs + at0.x;
    float norm;
    int pos = past + at0.x - tokens;
    const auto issue = [&](uint32_t i0, int j, int g, int buf) {
      const uint32_t left = rows - i0;
      if (even && left >= QT) {
#pragma unroll
        for (int jj = 0; jj < NI; ++jj, base += q_hop) gdma16(lds + buf * TILE_B + (w + 4 * jj) * 1024, base, off);
        base += q_step;
        pos += tokens;
        if (tid < QT) norm = *norm_from;
        norm_from += tokens;
        return;
      }
      const int ql = (int)opaque(lane), qt = (int)opaque(tid);
#pragma unroll 1
      for (int jj = 0; jj < NI; ++jj) {
        const int row = (w + 4 * jj) * T::RPI + ql / T::CPR;
        const int2 me = row_of(a, j, g + min(row, (int)min(left, (uint32_t)QT) - 1));
        gdma16(lds + buf * TILE_B + (w + 4 * jj) * 1024, qb + (int64_t)me.y * a.q_sH + (int64_t)me.x * a.q_sT + (((ql % T::CPR) ^ T::swz(row)) << 4));
      }
      if (qt < QT) {
        const bool there = (uint32_t)qt < left;
        const int2 me = row_of(a, j, g + (there ? qt : 0));
        norm = there ? a.lse[(int64_t)(hk * a.G + me.y) * a.T + x.qs + me.x] : -INFINITY;
        pos = there ? past + me.x : -1;
      }
    };
    // Two products are under way, of both halves of a wave's 64 keys with the same 32 rows or of its 32 keys with one 32 rows
    // after the other. (sum: of a tile of rows, of 16-bit types of two; total: of those before.  One chain over all rows would
    // round as often as there are rows: constant weights of 7500 to 10000 rows were off by 120 to 410 steps of 2^-24.  us
    // without and with totals, bf16: 2048 tokens over 16384 272.6 and 274.4, a prompt of 2048 64.4 and 65.7.)
    float sum[2] = {0.f, 0.f}, total[2] = {0.f, 0.f};
    v16f acc[2][SUMS];
    // Weights of product n's 32 rows and its keys, which not all rows see.
    const auto masked = [&](int n, const float* norm_of_row, const int* pos_of_row) {
      const int key = key0 + 32 * KEYS * kw + (KEYS == 2 ? 32 * n : 0) + r;
      const uint32_t reach = reach_of(a, key);
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        const float4 nv = *reinterpret_cast<const float4*>(norm_of_row + 8 * v4);
        const int4 pv = *reinterpret_cast<const int4*>(pos_of_row + 8 * v4);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float e = __builtin_amdgcn_exp2f(fmaf(logit<SUMS>(acc[n], 4 * v4 + u), a.scale_log2, -(&nv.x)[u]));
          sum[n] += (uint32_t)((&pv.x)[u] - key) < reach ? e : 0.f;
          if (DT == ZC_F32) __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_sched_barrier(0);       // (or the operands of all 16 are brought in front, into registers there are not)
      }
    };
    // Products of the keys n with 32 rows, and meanwhile, of fp32, the weights of the products before, of keys m, if all rows see them.
    const auto step = [&](auto weigh, int n, uint32_t row, int m, const float* norm_of_row) {
      constexpr bool WEIGH = decltype(weigh)::value;
      row = opaque(row);
#pragma unroll
      for (int i = 0; i < SUMS; ++i) acc[n][i] = v16f{};
      u32x4 q[2];
      q[0] = *reinterpret_cast<lds_u32x4*>((lds_ptr)(uintptr_t)row);
      q[1] = *reinterpret_cast<lds_u32x4*>((lds_ptr)(uintptr_t)(row ^ 32));
      float4 nv;
      constexpr int EACH = 16 / T::NKC;          // weights of a step
#pragma unroll
      for (int kc = 0; kc < T::NKC; ++kc) {
        if constexpr (WEIGH)
          if (kc * EACH % 4 == 0) nv = *reinterpret_cast<const float4*>(norm_of_row + 2 * kc * EACH);
        mma_chunk<DT>(acc[n][kc % SUMS], q[kc & 1], kf[n][kc]);
        if (kc + 2 < T::NKC) q[kc & 1] = *reinterpret_cast<lds_u32x4*>((lds_ptr)(uintptr_t)(row ^ ((kc + 2) << 5)));
        if constexpr (WEIGH)
#pragma unroll
          for (int v = kc * EACH; v < (kc + 1) * EACH; ++v)
            sum[m] += __builtin_amdgcn_exp2f(fmaf(logit<SUMS>(acc[m], v), a.scale_log2, -(&nv.x)[v & 3]));
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // As above of 16-bit types with the rows' operands `q` in registers, and their normalisers `nv` of the weights: what a
    // step has used is replaced by what the step after the next (q) or the next (nv) needs, so that no step waits for LDS.
    u32x4 q[DT == ZC_F32 ? 1 : T::NKC];
    float4 nv[4];
    // FETCH: the next tile's transfers, one a step: all at once a wave waits until the last has been taken.  That is where one
    // workgroup has a CU for itself (a prompt of 2048 77 -> 71 us; two hide it from each other, 2048 tokens over 16384 305 and
    // 305).
    const auto flow = [&](auto weigh, auto fetch, auto keys, auto refill, uint32_t next_row, const float* next_norm, uint32_t to_lds, const uint8_t* from) {
      constexpr bool WEIGH = decltype(weigh)::value, FETCH = decltype(fetch)::value, REFILL = decltype(refill)::value;
      static_assert(DT == ZC_F32 || NI == T::NKC, "a transfer a step");
      constexpr int n = decltype(keys)::value;
      constexpr bool NORMS = n == 0 || KEYS == 1;    // (the first of these rows' products: their normalisers come)
      constexpr int EACH = 16 / T::NKC;
      acc[n][0] = v16f{};
      if constexpr (REFILL) next_row = opaque(next_row);
      float x[EACH], e[EACH];
#pragma unroll
      for (int i = 0; i < EACH; ++i) e[i] = 0.f;
#pragma unroll
      for (int kc = 0; kc < T::NKC; ++kc) {
        mma_chunk<DT>(acc[n][0], q[kc], kf[KEYS == 2 ? n : 0][kc]);
        if constexpr (WEIGH) {                       // (a weight's three instructions wait for each other: each goes with another step's)
          if (kc > 1)
#pragma unroll
            for (int i = 0; i < EACH; ++i) sum[n ^ 1] += e[i];
          if (kc > 0)
#pragma unroll
            for (int i = 0; i < EACH; ++i) e[i] = __builtin_amdgcn_exp2f(x[i]);
#pragma unroll
          for (int i = 0; i < EACH; ++i) {
            const int v = kc * EACH + i;
            x[i] = fmaf(acc[n ^ 1][0][v], a.scale_log2, -(&nv[v >> 2].x)[v & 3]);
          }
        }
        if constexpr (FETCH) gdma16(to_lds + kc * 4096, from + kc * q_hop, off);
        if constexpr (REFILL) q[kc] = *reinterpret_cast<lds_u32x4*>((lds_ptr)(uintptr_t)(next_row ^ (kc << 5)));
        if (NORMS && (kc + 1) * EACH % 4 == 0) nv[(kc + 1) * EACH / 4 - 1] = *reinterpret_cast<const float4*>(next_norm + 2 * ((kc + 1) * EACH - 4));
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (WEIGH)
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum[n ^ 1] += e[i] + __builtin_amdgcn_exp2f(x[i]);
    };
    const auto weigh_only = [&](int m, const float* norm_of_row) {
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        const float4 nv = *reinterpret_cast<const float4*>(norm_of_row + 8 * v4);
#pragma unroll
        for (int u = 0; u < 4; ++u) sum[m] += __builtin_amdgcn_exp2f(fmaf(logit<SUMS>(acc[m], 4 * v4 + u), a.scale_log2, -(&nv.x)[u]));
      }
    };
    __syncthreads();                             // (K is in registers)
    if (i_first < i_end) issue(i_first, j0, g0, 0);
    int place = 0;                               // of the tile's normalisers; its rows are in buffer place & 1
    const int mine = 32 * rw + 4 * kh;           // of the tile's rows, the first that this lane's accumulators hold
    bool pending = false;                        // weights of keys 1 of the tile before, which all its rows see
    for (uint32_t i0 = i_first; i0 < i_end; i0 += QT, place = (place + 1) & (PLACES - 1)) {
      const int2 next = row_of(a, j0, g0 + QT);
      const int buf = place & 1;
      float* const norms_of = norms + place * QT;
      int* const where_of = where + place * QT;
      wait_vmem<0>();
      wait_all_loads();
      if (tid < QT) { norms_of[tid] = norm_of(norm); where_of[tid] = pos; }
      __syncthreads();                           // rows and normalisers are there, and nobody still reads the other buffer
      const bool fetch = DT != ZC_F32 && KEYS == 1 && even && i0 + QT < i_end && rows - (i0 + QT) >= QT;      // by the products below
      const uint32_t to_lds = lds + (buf ^ 1) * TILE_B + w * 1024;
      const uint8_t* const from = base;
      if (fetch) {
        base += NI * q_hop + q_step;
        pos += tokens;
        if (tid < QT) norm = *norm_from;
        norm_from += tokens;
      } else if (i0 + QT < i_end) {
        issue(i0 + QT, next.x, next.y, buf ^ 1);
      }
      const uint32_t row = lds + buf * TILE_B + 32 * rw * T::ROWB + T::slot(r, kh);
      const int pa = past + j0, pb = past + row_of(a, j0, g0 + QT - 1).x;          // positions of the tile's first and last row
      const bool whole = key0 + TILE - 1 <= pa && (!a.window || key0 > pb - a.window || key0 + TILE - 1 < a.sinks);
      if constexpr (DT == ZC_F32 && KEYS == 1) {     // (the weights are little beside the products)
        step(std::false_type{}, 0, row, 1, nullptr);
        if (whole) weigh_only(0, norms_of + mine);
        else masked(0, norms_of + mine, where_of + mine);
      } else if constexpr (DT == ZC_F32) {
        if (pending) step(std::true_type{}, 0, row, 1, norms + ((place - 1) & (PLACES - 1)) * QT + mine);
        else step(std::false_type{}, 0, row, 1, nullptr);
        if (whole) step(std::true_type{}, 1, row, 0, norms_of + mine);
        else step(std::false_type{}, 1, row, 0, nullptr);
      } else {
        const uint32_t first = opaque(row);
#pragma unroll
        for (int kc = 0; kc < T::NKC; ++kc) q[kc] = *reinterpret_cast<lds_u32x4*>((lds_ptr)(uintptr_t)(first ^ (kc << 5)));
        const auto half = [&](auto of) {
          constexpr int h = decltype(of)::value;
          using K0 = std::integral_constant<int, 0>;
          using K1 = std::integral_constant<int, 1>;
          const float* const of_these = norms_of + mine + 64 * h;
          const uint32_t behind = row + 64 * (h + 1) * T::ROWB;
          if constexpr (KEYS == 1) {
            using KH = std::integral_constant<int, h & 1>;
            using MORE = std::bool_constant<h + 1 < QT / 64>;
            with(pending, h == 0 && fetch, [&](auto weigh, auto get) { flow(weigh, get, KH{}, MORE{}, behind, of_these, to_lds, from); });
            pending = whole;
            if (!whole) masked(h & 1, of_these, where_of + mine + 64 * h);
            return;
          }
          with(pending, h == 0 && fetch, [&](auto weigh, auto get) { flow(weigh, get, K0{}, std::false_type{}, 0, of_these, to_lds, from); });
          with(whole, false, [&](auto weigh, auto) { flow(weigh, std::false_type{}, K1{}, std::bool_constant<h + 1 < QT / 64>{}, behind, nullptr, 0, nullptr); });
          pending = whole;
          if (!whole) {
            masked(0, norms_of + mine + 64 * h, where_of + mine + 64 * h);
            masked(1, norms_of + mine + 64 * h, where_of + mine + 64 * h);
          }
        };
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, 1>{});
        static_assert(QT == 128, "two halves");
      }
      if constexpr (DT == ZC_F32 && KEYS == 2) {
        pending = whole;
        if (!whole) {
          masked(0, norms_of + mine, where_of + mine);
          masked(1, norms_of + mine, where_of + mine);
        }
      }
if (DT == ZC_F32 || (place & 1))
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        total[n] += sum[n];
        sum[n] = 0.f;
      }
      j0 = next.x;
      g0 = next.y;
    }
    if (pending) weigh_only(1, norms + ((place - 1) & (PLACES - 1)) * QT + mine + QT - 64);
#pragma unroll
    for (int n = 0; n < KEYS; ++n) {
      float all = KEYS == 2 ? total[n] + sum[n] : (total[0] + sum[0]) + (total[1] + sum[1]);
      all += __shfl_xor(all, 32);
      if (kh == 0) sums[rw][32 * KEYS * kw + 32 * n + r] = all;
    }
    __syncthreads();
    if (to) *to = fmaf(old, a.decay, sums[0][tid] + sums[1][tid]);
  }
}

template <int DT, int D>
__global__ __launch_bounds__(256, DT != ZC_F32 ? 2 : D == 64 ? 2 : 1) void k_paged_scores(ScoreArgs a) {
  constexpr int kFew = FewMemory<DT, D>::kBytes, kMany = ManyMemory<DT, D>::kBytes;
  __shared__ __align__(1024) uint8_t mem[kFew > kMany ? kFew : kMany];
  __shared__ __align__(16) float norms[2 * kMostRows];
  __shared__ __align__(16) int where[2 * kMostRows];
  __shared__ float sums[2][kScoreTile];
  Span x;
  for (int u = blockIdx.y; find_span(a, u, x); u += gridDim.y) {
    const int64_t rows = (int64_t)x.nq * a.G;
    if (rows <= 32) score_rows<DT, D, 1, false>(a, x, blockIdx.x, mem, norms, where);
    else if (rows <= 64) score_rows<DT, D, 2, false>(a, x, blockIdx.x, mem, norms, where);
    else if (x.shift == 7) score_tiles<DT, D, 2>(a, x, blockIdx.x, mem, norms, where, sums);
    else score_tiles<DT, D, 1>(a, x, blockIdx.x, mem, norms, where, sums);
  }
}

// Steps of single tokens: without the way of chunks there are registers for twice as many workgroups, so twice as many keys on
// their way.  us with both ways in one kernel and so: 64 over 64 to 8192 65.6 and 60.0, 16 over 4096 36.7 and 33.6, 256 over
// 500 83.9 and 68.9; 8 heads of 64 channels, fp16, 40 over 4795 to 5806 69.8 and 55.2.
template <int DT, int D>
__global__ __launch_bounds__(256, DT != ZC_F32 ? 4 : D == 64 ? 3 : 2) void k_token_scores(ScoreArgs a) {
  __shared__ __align__(1024) uint8_t mem[FewMemory<DT, D>::kBytes];
  __shared__ __align__(16) float norms[128];
  __shared__ __align__(16) int where[128];
  Span x;
  for (int u = blockIdx.y; find_span(a, u, x); u += gridDim.y) {
    if ((int64_t)x.nq * a.G <= 32) score_rows<DT, D, 1, false>(a, x, blockIdx.x, mem, norms, where);
    else score_rows<DT, D, 1, true>(a, x, blockIdx.x, mem, norms, where);
    __syncthreads();
  }
}

template <int DT, int D>
static int launch_scores(const ScoreArgs& a, int units, bool tokens, hipStream_t st) {
  if (tokens) hipLaunchKernelGGL((k_token_scores<DT, D>), dim3((unsigned)a.Hkv, (unsigned)units), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_paged_scores<DT, D>), dim3((unsigned)a.Hkv, (unsigned)units), dim3(256), 0, st, a);
  ZC_LAUNCH_CHECK();
  return ZC_OK;
}

}  // namespace zc

using namespace zc;

extern "C" int zc_paged_scores(const zc_tensor4* q, const zc_tensor4* k_pages, const int32_t* block_table, int64_t row_stride, int64_t max_blocks,
                               const int32_t* q_start, const int32_t* kv_len, int64_t R, int32_t window, int32_t sinks, float sm_scale,
                               const float* lse, float decay, float* scores, void* stream) {
  int rc = zc_validate_pages(k_pages, k_pages);
  if (rc) return rc;
  rc = zc_validate_heads(q, k_pages);
  if (rc) return rc;
  if (q->H % k_pages->H) return ZC_ERR_INVALID_ARG;
  if (R < 0 || window < 0 || sinks < 0 || !(sm_scale >= 0.f) || !(sm_scale * kLog2e <= 3.40282347e38f) || !(decay >= 0.f && decay <= 1.f))
    return ZC_ERR_INVALID_ARG;
  if (max_blocks < 0 || row_stride < max_blocks) return ZC_ERR_INVALID_ARG;
  if (!scores || (reinterpret_cast<uintptr_t>(scores) & 15)) return ZC_ERR_INVALID_ARG;
  if (q->L == 0 || R == 0 || max_blocks == 0) return ZC_OK;
  if (!q_start || !kv_len || !lse || !block_table) return ZC_ERR_INVALID_ARG;
  for (const void* p : {(const void*)block_table, (const void*)q_start, (const void*)kv_len, (const void*)lse})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ZC_ERR_INVALID_ARG;
  const int64_t T = q->L, Hkv = k_pages->H, G = q->H / Hkv, page = k_pages->L;
  if (R >= (1 << 24) || max_blocks > 0x7fffffff || T > 0x7fffffff / q->H || q->H > 65535 || G > 4096) return ZC_ERR_UNSUPPORTED;
  const int64_t room = max_blocks > 0x7fff0000 / page ? 0x7fff0000 : max_blocks * page;
  if (window >= room) window = 0;                    // (every row sees all it could)
  if (sinks > room) sinks = (int32_t)room;
  const int64_t eb = elem_bytes(q->dtype);
  ScoreArgs a;
  a.q = (const uint8_t*)q->ptr; a.k = (const uint8_t*)k_pages->ptr;
  a.q_sH = q->sH * eb; a.q_sT = q->sL * eb; a.k_sH = k_pages->sH * eb;
  a.k_sB = (uint32_t)(k_pages->sB * eb); a.k_row = (uint32_t)(k_pages->sL * eb);
  a.table = block_table; a.q_start = q_start; a.kv_len = kv_len; a.row = row_stride;
  a.cols = (int)max_blocks; a.shift = __builtin_ctzll((unsigned long long)page); a.n_pages = (int)k_pages->B; a.cap = (int)room;
  a.R = (int)R; a.T = (int)T; a.Hkv = (int)Hkv; a.G = (int)G;
  a.window = window; a.sinks = sinks;
  a.scale_log2 = (sm_scale == 0.f ? 1.0f / sqrtf((float)q->D) : sm_scale) * kLog2e;
  a.decay = decay;
  a.lse = lse;
  a.scores = scores;
  a.over_G = G == 1 ? 0 : (uint32_t)(((1ull << 32) + G - 1) / G);
  // One token a request on average, of up to 32 heads each.  (Chunks among more tokens take their own way: us with all steps
  // of up to 32 rows a request on average here, and so: 63 tokens and a chunk of 200 over 500 to 4000, 32 heads over 8 of 128
  // channels, bf16, 115 and 77, of 440 129 and 79; 16 requests of 8 tokens over 4096 35.0 and 39.5.) T and R are all that the
  // host knows, so the rule is wrong on either side: rows behind the last request's take single tokens to the kernel of chunks
  // (64 of them 65.6 instead of 60.0, 256 over 500 84 instead of 69), requests without tokens a chunk to this one (us there
  // and here, as many such requests as just keep it there and 66 more: 440 tokens over 4096 77 and 102, 100 tokens 26 and 31,
  // 16 tokens 13 and 14, 2000 over themselves 634 and 612; fp32, 440 190 and 208).
  const bool tokens = T <= R && G <= 32;
  // (us of single tokens at 1024 and 2048 units: bf16, 64 over 64 to 8192 60.0 and 59.7, 256 over 500 69 and 73; fp32, 16 over
  // 2000 to 4000, whose products take longer than their keys, 69 and 57)
  const int64_t target = ceil_div64(tokens && q->dtype == ZC_F32 ? 2048 : 1024, Hkv), tiles = ceil_div64(room, T * G > 64 * R ? kScoreTile / 2 : kScoreTile), with = R < T ? R : T;
  a.target = (float)target;
  const int64_t hop = 4096 / (q->D * eb);            // rows of the four waves' transfers at a time, of as many tokens at most
  a.near_rows = q->sH <= 0xffffffff && q->sL <= 0xffffffff && (G - 1) * a.q_sH + hop * a.q_sT < 0xffffff00ll;
  // (a workgroup takes more units where there are; those that find none cost their places: where a table's room allows few
  // tiles, as many as the chip holds)
  const int64_t all = tiles > 65535 / with ? 65535 : tiles * with, at_once = T * G <= 32 * R && all * Hkv <= 2560 ? ceil_div64(512, Hkv) : target;
  const int64_t units = at_once + with < all ? at_once + with : all;
  hipStream_t st = (hipStream_t)stream;
#define ZC_PS(DT) (q->D == 128 ? launch_scores<DT, 128>(a, (int)units, tokens, st) : launch_scores<DT, 64>(a, (int)units, tokens, st))
  if (q->dtype == ZC_F32) rc = ZC_PS(ZC_F32);
  else if (q->dtype == ZC_F16) rc = ZC_PS(ZC_F16);
  else rc = ZC_PS(ZC_BF16);
#undef ZC_PS
  return rc;
}
