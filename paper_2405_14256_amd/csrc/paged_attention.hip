// zc_paged_attention: attention of a step's new tokens - one a request or a chunk - over keys and values in pages.
//
// The rows of a request and a KV head are its new tokens times the G query heads of the group, token after token: a block
// of them reads a key once for all its rows, whatever their number, so single tokens and chunks are the same work.
//   logits  D[key][row]     = sum_c K[key][c] Q[row][c]            (A = K block, B = Q rows in registers)
//   output  D[channel][row] = sum_key Vt[channel][key] P[row][key]  (A = V block transposed, B = P)
// Both results put a row in a lane (column r = lane & 31): its running maximum, sum and rescaling are lane-local, and the
// weights that a lane has computed are, converted in place, the B operand of the second product.
// Weights of 16-bit tensors enter it rounded to the tensors' type, which is what the matrix instructions take; sums of weights,
// references and outputs stay in fp32.  A weight is off by half a step (bf16 2^-8, fp16 2^-11 of itself) at most, and over
// many keys these errors average out under the result's own rounding.  Error of a result against 64 bits (2-norm), weights of 32 bits and here: one bf16 token
// over 4096 1.70e-3 both, 64 over 64 to 8192 1.62e-3 and 1.64e-3, 2048 over 32768 1.66e-3 and 1.72e-3; fp16, 20 tokens and 4 chunks 2.06e-4 and
// 2.10e-4.  Weights as a rounded part and a remainder would take the second product twice.
//
// A unit of work is a block of rows and a part of the key tiles it sees.  The host knows neither lengths nor how the
// rows are spread over requests; every wave finds its unit from the lengths alone (find_unit), so nothing has to be
// prepared, and what is long is split by the same rule in every wave.
#include <limits.h>
#include <stdint.h>
#include <type_traits>

#include "mfma_tiles.hpp"
#include "paged_args.hpp"

namespace zc {

struct PagedArgs {
  const uint8_t *q, *k, *v;
  uint8_t* o;
  int64_t q_sH, q_sT, o_sH, o_sT;               // bytes
  int64_t k_sH, v_sH;                           // bytes
  uint32_t k_sB, v_sB, k_row, v_row;            // bytes from a page, a token to the next (a head's rows of a page: below 2 GB)
  const int32_t *table, *q_start, *kv_len;
  int64_t row;                                  // of the table, in entries
  int cols, shift, n_pages, cap;                // blocks of the table; page size; pages; tokens a row of the table has room for
  int R, T, Hkv, G, window, sinks;
  float scale_log2;
  float* lse;                                   // [Hq, T] or null
  int target, units;                            // units a head's rows are split into, about (0: nothing is split); at most
  uint32_t over_G;                              // ceil(2^32 / G)
  int reach;                                    // tiles that a block of rows sees under the window, at most
  int slot;                                     // rows of a unit's partial results
  int coarse;                                   // tiles are added up in steps of 2^coarse (sums stay within 32 bits)
  float *part_o, *part_ml;                      // of split units: [head][unit][row][D], [head][unit][row][2] (reference, sum)
  int4* todo;                                   // [head][unit]: what the join has to do from this unit on, x = 0: nothing
};

constexpr float kLowestLogit = -3.40282347e38f; // where a reference starts: finite, so that weights of -inf are 0 whatever came before

template <int DT>
__device__ inline uint32_t pack_two(float lo, float hi) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  if constexpr (DT == ZC_F16) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, h2));
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, b2));
  }
}

// ---- the work of a wave ---------------------------------------------------------------------------
// Key tiles are of 64 keys.  A request of few rows goes in blocks of 32 rows whose keys four waves share, any other (of 16-bit
// types) in blocks of 128, 32 a wave: with one token a request the first way has four waves at work where the second has one,
// and the first waits for no barrier; with many rows the second reads a key once for four times as many.  us by 128 and by 32 rows,
// 32 heads over 8 of 128 channels, bf16: 16 requests of 4096 tokens, 9 of them new (36 rows) 58.4 and 53.8, 16 (64) 60.4 and 55.0; 1 of 8192, 16 new 29.1
// and 22.4; 8 of 200 to 500, 10 to 16 new 15.9 and 10.5; 4 of 4096, 32 new (128 rows) 29.1 and 30.3; of 64 channels, 2 of 1000 to 3000, 40 to 64 new
// (one head a group) 16.7 and 14.6.
constexpr int kTile = 64;
template <int DT, bool FEW> struct Blocks {                              // FEW: of 32 rows whatever a request has
  static constexpr int kMany = DT == ZC_F32 || FEW ? 32 : 128;            // rows of a block, of many rows
  __device__ static bool few(int rows) { return DT == ZC_F32 || FEW || rows <= 64; }
};

struct Unit {
  int r, qs, nq, kv;            // request, its first row, new tokens, tokens
  bool few;
  int j0, g0, rows;             // token and head of the block's first row, its rows
  int p0, p1;                   // positions of its first and last row
  int first, sink_tiles;        // tile t is t of the first sink_tiles, then first + t - sink_tiles
  int t_lo, t_hi;               // tiles of this unit
  int part, parts;              // which of the parts that the block's tiles are divided into
  uint32_t behind;              // 16 keys from key0 on are behind every window of the block's if key0 - sinks, without sign, is less than this
};

// Row r of a block: its token (after the block's first) and head.
struct Row { int j, g; };
__device__ inline Row row_at(const PagedArgs& a, int j0, int g0, int r) {
  const int v = g0 + r, j = a.G == 1 ? v : (int)__umulhi((uint32_t)v, a.over_G);    // (exact while v G < 2^32)
  return {j0 + j, v - j * a.G};
}
__device__ inline Row row_at(const PagedArgs& a, const Unit& x, int r) { return row_at(a, x.j0, x.g0, r); }

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

__device__ inline int tile_of(const Unit& x, int t) { return t < x.sink_tiles ? t : x.first + t - x.sink_tiles; }
__device__ inline int unit_of_grid() { return blockIdx.y + 65535 * blockIdx.z; }

// The page of 16 keys from key0 on (past the table: any, no key is read).
__device__ inline int page_of(const PagedArgs& a, const Unit& x, int key0) {
  typedef __attribute__((address_space(4))) const int32_t* scalar;
  return ((scalar)(uintptr_t)(a.table + x.r * a.row))[min(key0 >> a.shift, a.cols - 1)];
}
// Of 16 keys from key0 on, how many a unit reads: none of a missing page, of those that no row's window reaches, from `end` on.
// What is not read arrives as zeros.
__device__ inline int keys_read(const PagedArgs& a, const Unit& x, int end, int key0, int id) {
  int n = max(end - key0, 0);
  asm("" : "+s"(n));                                       // (both bounds at once would be a vector instruction, and what follows too)
  n = min(n, 16);
  if ((uint32_t)id >= (uint32_t)a.n_pages) n = 0;
  if ((uint32_t)(key0 - a.sinks) < x.behind) n = 0;
  return n;
}
// Where they are (of no keys: anywhere, nothing is read).
__device__ inline __amdgpu_buffer_rsrc_t keys_at(const PagedArgs& a, const uint8_t* head, uint32_t sB, uint32_t row, int key0, int id, int n) {
  const uint64_t at = (uint64_t)(uint32_t)id * sB + ((uint32_t)key0 & ((1u << a.shift) - 1)) * row;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(head + at), 0, n * row, kBufFlags);
}
// The blocks of 32 keys that every row from position p0 to p1 sees whole: those from `low` on, `span` of them by their first key, and
// those whose first key is below `sink`.
struct Seen {
  int low, sink;
  uint32_t span;
  __device__ Seen(const PagedArgs& a, int p0, int p1) {
    low = a.window ? max(max(p1, 0) - a.window + 1, 0) : 0;
    const int end = max(p0, 0) - 30;                       // (of positions in front of the first key no block is seen)
    span = max(end - low, 0);
    sink = a.window ? min(a.sinks - 31, end) : 0;
  }
  // Blocks of 32 + more keys.
  __device__ bool whole(int key0, int more = 0) const { return (uint32_t)(key0 - low) < (uint32_t)max((int)span - more, 0) || key0 < sink - more; }
};

// 16 keys to LDS in N transfers of 1024 bytes, to consecutive places.  The descriptor changes with every page, and the compiler may have
// brought a part of it (or the place) from a vector register the instruction before: a memory instruction must not read
// such a scalar register for five wait states, and does not see that it does inside an assembly block.
#define ZC_KEYS_NEXT(v) "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 " v ", %1, 0 offen lds\n\t"
#define ZC_KEYS_FIRST "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %1, 0 offen lds\n\t"
template <int N>
__device__ inline void move_keys(uint32_t lds, __amdgpu_buffer_rsrc_t rs, const int (&v)[N]) {
  static_assert(N == 2 || N == 4 || N == 8, "16 rows of 128, 256 or 512 bytes");
  if constexpr (N == 2)
    asm volatile(ZC_KEYS_FIRST ZC_KEYS_NEXT("%3") :: "s"(lds), "s"(rs), "v"(v[0]), "v"(v[1]) : "memory", "scc");
  else if constexpr (N == 4)
    asm volatile(ZC_KEYS_FIRST ZC_KEYS_NEXT("%3") ZC_KEYS_NEXT("%4") ZC_KEYS_NEXT("%5")
                 :: "s"(lds), "s"(rs), "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]) : "memory", "scc");
  else
    asm volatile(ZC_KEYS_FIRST ZC_KEYS_NEXT("%3") ZC_KEYS_NEXT("%4") ZC_KEYS_NEXT("%5") ZC_KEYS_NEXT("%6") ZC_KEYS_NEXT("%7") ZC_KEYS_NEXT("%8") ZC_KEYS_NEXT("%9")
                 :: "s"(lds), "s"(rs), "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "v"(v[4]), "v"(v[5]), "v"(v[6]), "v"(v[7]) : "memory", "scc");
}
#undef ZC_KEYS_NEXT
#undef ZC_KEYS_FIRST

// Chunk slot permutation of a V row of 16-bit types: the transposing load reads 64 bytes of four consecutive keys per
// half-wave; these land in different banks.
template <int DT, int D>
__device__ inline int v_slot(int key) {
  if constexpr (DT == ZC_F32) return 0;
  return D == 128 ? 4 * (key & 3) ^ (key & 2) : 2 * (key & 2) ^ 2 * (key & 1);
}

// First row of the partial results of a head's unit.
__device__ inline int64_t part_row(const PagedArgs& a, int hk, int unit) { return ((int64_t)hk * a.units + unit) * a.slot; }

// ---- blocks of 32 rows: single tokens, short chunks, fp32 ---------------------------------------------
// Four or eight waves share the keys of 32 rows, a wave every fourth or eighth 32 keys, in a place of its own in LDS for one K and one V block: a
// block's K is requested when the one before has been multiplied, its V likewise, so that a wave has one of them in flight
// at any time and waits for nobody.
//
// Bound by memory: 64 single tokens over 64 to 8192 tokens, 32 heads over 8 of 128 channels, bf16, 97 us (5.5 TB/s), the join 4 more; one over
// 4096 by its chain of lengths, pages, keys and the waves' join, 6 us.  fp32 chunks by the matrix cores: 2048 over 8192, 16 heads over 4 of 64
// channels 498 us, 121 TFLOP/s.
template <int DT, int D, int NW>
struct RowsMemory {
  static constexpr int kBlock = 32 * Tile<DT, D>::ROWB;                   // bytes of a block of keys or values
  static constexpr int kBytes = 2 * NW * kBlock;
};
template <int DT, int D, int NW>
__device__ __forceinline__ void attend_rows(const PagedArgs& a, const Unit& x, int hk, uint8_t* mem, float (*sum)[2][64]) {
  using T = Tile<DT, D>;
  constexpr int BLK = RowsMemory<DT, D, NW>::kBlock;
  constexpr int NT = BLK / 1024;                 // transfers of a block
  constexpr int PG = 16 / T::RPI;                // of 16 keys
  constexpr int CT = D / 32;
  // An fp32 logit is summed in four accumulators: the roundings of one chain of D products were most of the result's error (2-norm,
  // six channels of the keys 15 times the others: one token over 2529 keys of 128 channels 1.2e-6 and 6.3e-7, 900 over 8515 of 64 1.3e-6 and
  // 7.8e-7).  us of one chain and of four: 2048 tokens over 8192, 16 heads over 4 of 128 channels 1012 and 1051, of 64 486 and 498, one token 14.8 and 15.0.
  constexpr int SUMS = DT == ZC_F32 ? 4 : 1;
  static_assert(NW * 2 * BLK >= NW * CT * 4 * 64 * 16 && CT * 4 % NW == 0, "the waves' outputs fit where their keys were");
  typedef short s16x4 __attribute__((ext_vector_type(4)));

  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, kh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint8_t* kb = a.k + hk * a.k_sH;
  const uint8_t* vb = a.v + hk * a.v_sH;
  const uint32_t mem_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)mem;
  const uint32_t k_lds = mem_lds + w * 2 * BLK, v_lds = k_lds + BLK;

  int kvoff[PG], vvoff[PG];
#pragma unroll
  for (int j = 0; j < PG; ++j) {
    const int row = j * T::RPI + lane / T::CPR;
    kvoff[j] = (int)(row * a.k_row) + (((lane % T::CPR) ^ T::swz(row)) << 4);
    vvoff[j] = (int)(row * a.v_row) + (((lane % T::CPR) ^ v_slot<DT, D>(row)) << 4);
  }
  struct Ids { int id[2], n[2], key0; };
  auto pages = [&](int b) {                      // of the unit's block b of 32 keys, two to a tile
    Ids s;
    s.key0 = tile_of(x, x.t_lo + (b >> 1)) * kTile + 32 * (b & 1);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      s.id[g] = page_of(a, x, s.key0 + 16 * g);
      s.n[g] = keys_read(a, x, x.kv, s.key0 + 16 * g, s.id[g]);
    }
    return s;
  };
  auto issue = [&](const Ids& s, const uint8_t* head, uint32_t sB, uint32_t row, uint32_t lds, const int (&voff)[PG]) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const auto rs = keys_at(a, head, sB, row, s.key0 + 16 * g, s.id[g], s.n[g]);
      move_keys<PG>(lds + g * 16 * T::ROWB, rs, voff);
    }
  };

  // (the tile of the last row's own token may have one block only)
  int blocks = 2 * (x.t_hi - x.t_lo);
  if (blocks > 0 && tile_of(x, x.t_hi - 1) * kTile + 32 > x.p1) --blocks;
  int t = w;
  Ids at = pages(t);                             // (of no block of the unit: any page, and nothing is requested)

  // this lane's row, straight into operand registers
  const bool mine = r < x.rows;
  const Row me = row_at(a, x, r);
  const int64_t hq = hk * a.G + me.g, tok = x.qs + me.j;
  const int pos = mine ? x.kv - x.nq + me.j : -1;
  u32x4 qf[T::NKC];
#pragma unroll
  for (int kc = 0; kc < T::NKC; ++kc) qf[kc] = u32x4{0, 0, 0, 0};
  if (mine) {
    const uint8_t* qr = a.q + hq * a.q_sH + tok * a.q_sT + kh * 16;
#pragma unroll
    for (int kc = 0; kc < T::NKC; ++kc) qf[kc] = *reinterpret_cast<const u32x4*>(qr + kc * 32);
  }
  if (t < blocks) {
    issue(at, kb, a.k_sB, a.k_row, k_lds, kvoff);
    issue(at, vb, a.v_sB, a.v_row, v_lds, vvoff);
  }

  typedef __attribute__((address_space(3))) const uint8_t* lds_ptr;
  const uint32_t kaddr = k_lds + T::slot(r, kh);          // chunk 2 kc + kh sits at kaddr ^ (32 kc)
  const int vkey = 4 * kh + ((lane & 15) >> 2);
  const int vsub = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
  uint32_t vaddr[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    if constexpr (DT == ZC_F32) vaddr[ct] = v_lds + 4 * kh * T::ROWB + (32 * ct + r) * 4;
    else vaddr[ct] = v_lds + vkey * T::ROWB + (((4 * ct + vsub) ^ v_slot<DT, D>(vkey)) << 4) + (lane & 1) * 8;
  }

  v16f oacc[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) oacc[ct] = v16f{};
  float m = kLowestLogit, l = 0.f;   // running maximum (log2 units), this half-wave's share of the sum

  const Seen seen(a, x.p0, x.p1);
  wait_all_loads();                              // (the rows and the first blocks: the compiler would wait for the rows in the loop, and so for the next blocks)
  for (; t < blocks; t += NW) {
    const bool more = t + NW < blocks;
    const int key0 = at.key0;
    if (more) at = pages(t + NW);
    wait_vmem<NT>();                                       // K is there (V was requested after it)
    v16f part[SUMS] = {};
#pragma unroll
    for (int kc = 0; kc < T::NKC; ++kc) {
      const u32x4 kf = *(__attribute__((address_space(3))) const u32x4*)(lds_ptr)(uintptr_t)(kaddr ^ (32 * kc));
      mma_chunk<DT>(part[kc % SUMS], kf, qf[kc]);
    }
    v16f s = part[0];
    if constexpr (SUMS == 4)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = (part[0][v] + part[1][v]) + (part[2][v] + part[3][v]);
    dma_reuse_fence();
    if (more) issue(at, kb, a.k_sB, a.k_row, k_lds, kvoff);
    if (!seen.whole(key0)) {
      const int low = a.window && pos >= 0 ? pos - a.window : -1;          // keys up to it are seen as sinks only
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = key0 + acc_row(v, kh);
        if ((key > pos) | ((key <= low) & (key >= a.sinks))) s[v] = -INFINITY;
      }
    }
    // (the maximum is taken over the raw products - the scale is not negative - and the scale enters with the subtraction)
    float tmax = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) tmax = fmaxf(tmax, s[v]);
    tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
    const float m_new = fmaxf(m, tmax * a.scale_log2);
    if (__builtin_amdgcn_ballot_w64(m_new > m)) {
      const float alpha = __builtin_amdgcn_exp2f(m - m_new);
      l *= alpha;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[ct][e] *= alpha;
      m = m_new;
    }
    float psum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, -m));
      psum += s[v];
    }
    l += psum;
    if (more) wait_vmem<NT>();
    else wait_vmem<0>();                                   // V is there
    if constexpr (DT == ZC_F32) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const float vf = *(__attribute__((address_space(3))) const float*)((lds_ptr)(uintptr_t)vaddr[ct] + acc_row(v, 0) * T::ROWB);
          oacc[ct] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[v], oacc[ct], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 pb;
        pb.x = pack_two<DT>(s[8 * h], s[8 * h + 1]);
        pb.y = pack_two<DT>(s[8 * h + 2], s[8 * h + 3]);
        pb.z = pack_two<DT>(s[8 * h + 4], s[8 * h + 5]);
        pb.w = pack_two<DT>(s[8 * h + 6], s[8 * h + 7]);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const lds_ptr base = (lds_ptr)(uintptr_t)vaddr[ct] + 16 * h * T::ROWB;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)base);
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(base + 8 * T::ROWB));
          const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
          u32x4 vf;
          vf.x = l2.x; vf.y = l2.y; vf.z = h2.x; vf.w = h2.y;
          mma_chunk<DT>(oacc[ct], vf, pb);
        }
      }
    }
    dma_reuse_fence();
    if (more) issue(at, vb, a.v_sB, a.v_row, v_lds, vvoff);
  }

  // ---- join the waves: all outputs to LDS, each wave finishes an equal part of the channels ----
  // (a wave without keys has m = kLowestLogit, l = 0 and zeros)
  constexpr int PART = CT * 4 / NW;                        // groups of four channels of a lane
  float4* stage = reinterpret_cast<float4*>(mem);
  const float l_wave = l + __shfl_xor(l, 32);
  __syncthreads();                                         // (every wave is done with its blocks)
  if (mine) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4)
        stage[((w * CT + ct) * 4 + v4) * 64 + lane] = make_float4(oacc[ct][4 * v4], oacc[ct][4 * v4 + 1], oacc[ct][4 * v4 + 2], oacc[ct][4 * v4 + 3]);
  }
  sum[w][0][lane] = m;
  sum[w][1][lane] = l_wave;
  __syncthreads();
  if (!mine) return;
  float M = kLowestLogit, l_tot = 0.f, f[NW];
#pragma unroll
  for (int v = 0; v < NW; ++v) { f[v] = sum[v][0][lane]; M = fmaxf(M, f[v]); }
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    f[v] = __builtin_amdgcn_exp2f(f[v] - M);
    l_tot = fmaf(sum[v][1][lane], f[v], l_tot);
  }
  const bool whole = x.parts == 1;
  const int64_t prow = part_row(a, hk, unit_of_grid()) + r;
  const float inv = !whole ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
  uint8_t* orow = a.o + hq * a.o_sH + tok * a.o_sT;
#pragma unroll
  for (int u = 0; u < PART; ++u) {
    const int part = w * PART + u;                         // group part % 4 of channel tile part / 4
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float4 p = stage[((v * CT * 4) + part) * 64 + lane];
      o.x = fmaf(p.x, f[v], o.x); o.y = fmaf(p.y, f[v], o.y); o.z = fmaf(p.z, f[v], o.z); o.w = fmaf(p.w, f[v], o.w);
    }
    const int c = 32 * (part >> 2) + 8 * (part & 3) + 4 * kh;
    o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
    if (!whole) *reinterpret_cast<float4*>(a.part_o + prow * D + c) = o;
    else if constexpr (DT == ZC_F32) *reinterpret_cast<float4*>(orow + c * 4) = o;
    else *reinterpret_cast<uint2*>(orow + c * 2) = make_uint2(pack_two<DT>(o.x, o.y), pack_two<DT>(o.z, o.w));
  }
  if (w == 0 && kh == 0) {
    if (!whole) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(M, l_tot);
    else if (a.lse) a.lse[hq * a.T + tok] = l_tot == 0.f ? -INFINITY : (M + log2f(l_tot)) * kLn2;
  }
}

// ---- blocks of 128 rows, 16-bit types: chunks ------------------------------------------------------------
// Four waves of 32 rows each; 64-key tiles of K and V stream through LDS for all of them, two waves on a SIMD.  Keys go by
// halves of a tile, and no wave multiplies a half that lies behind its last row.  A wave moves 16 keys of a tile, which
// lie in one page: its address is scalar work, and a page that ends inside a tile costs nothing.
//
// Bound by the matrix cores, the vector instructions beside them and the power both draw: a half is 16 matrix instructions of 32
// cycles (128 channels) and about 600 cycles of vector instructions (16 of them exponentials at a quarter of the rate), so the two have
// to run at the same time: the logits of half h + 1 are multiplied while the exponentials of half h are taken, and the operands of
// each product are requested one phase before.  2048 tokens over 32768, 32 heads over 8 of 128 channels, bf16: 1013 to 1067 us by the card, 1.0 PFLOP/s,
// matrix cores 52 % and vector issue 65 % busy at 1.79 GHz (blocks of 32 rows: 1610 us); 8192 over 16384, 16 heads over 4 of 64, 505 us, 0.82.
//
// Of 64 channels three tiles of K and V fit (three workgroups a CU either way), and they are requested two tiles ahead: a
// tile is worth 0.2 us of matrix instructions there, less than a trip to memory.
template <int D> constexpr int kStages = D == 64 ? 3 : 2;
template <int DT, int D>
__device__ __forceinline__ void attend_tiles(const PagedArgs& a, const Unit& x, int hk, uint8_t* mem) {
  using T = Tile<DT, D>;
  constexpr int KEYS = kTile;
  constexpr int TILE_B = KEYS * T::ROWB;
  constexpr int NI = 16 / T::RPI;                // transfers per wave, tile and tensor
  constexpr int CT = D / 32;                     // 32-channel tiles of the output
  constexpr int EPS = 16 / T::NKC;               // logits per slice
  constexpr int VS = T::NKC / 4;                 // the slice that requests the first V operand
  constexpr int STAGES = kStages<D>, AHEAD = STAGES - 1;       // tiles of K and of V in LDS; how far ahead they are requested
  typedef short s16x4 __attribute__((ext_vector_type(4)));

  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, kh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint8_t* kb = a.k + hk * a.k_sH;
  const uint8_t* vb = a.v + hk * a.v_sH;
  const uint32_t ks_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)mem + w * 16 * T::ROWB;
  const uint32_t vs_lds = ks_lds + STAGES * TILE_B;

  // this wave's rows, and the halves of this unit that they see: all up to the last row's
  const int wrows = min(max(x.rows - 32 * w, 0), 32);
  const int wp0 = x.kv - x.nq + row_at(a, x, 32 * w).j, wp1 = wrows > 0 ? x.kv - x.nq + row_at(a, x, 32 * w + wrows - 1).j : -1;
  const int ntiles = x.t_hi - x.t_lo;
  const Seen seen(a, wp0, wp1);
  int nh = 0;
  if (wp1 >= 0) {
    const int t1 = wp1 / KEYS - x.first + x.sink_tiles - x.t_lo;          // the tile of the last row's own token
    nh = t1 < 0 ? 0 : t1 >= ntiles ? 2 * ntiles : 2 * t1 + ((wp1 & 32) ? 2 : 1);
  }

  // A lane's place in transfer jj: row jj * RPI + lane / CPR of 16, its chunks swizzled by the row (the swizzles repeat after 16
  // rows).  The parts are put together at every transfer: kept, they would be eight registers of a loop that has none to spare.
  int krow = (lane / T::CPR) * (int)a.k_row, kchunk = ((lane % T::CPR) ^ T::swz(lane / T::CPR)) << 4;
  int vplace = (lane / T::CPR) * (int)a.v_row + (((lane % T::CPR) ^ v_slot<DT, D>(lane / T::CPR)) << 4);
  static_assert(T::RPI % 4 == 0 && T::SW * T::RP256 == 16, "what a transfer's first row adds to the swizzles");
  struct Group { int key0, id, n; };
  // The pages of this wave's keys of 64 tiles, one a lane (of tiles that are not the unit's: any).
  int ids;
  auto pages = [&](int t) {
    const int key0 = tile_of(x, x.t_lo + t + lane) * KEYS + 16 * w;
    ids = a.table[x.r * a.row + min(key0 >> a.shift, a.cols - 1)];
  };
  const int turn = x.sink_tiles - x.t_lo;        // the tile behind the sinks'
  auto next_key = [&](int t, int key0, int off) { return t == turn ? x.first * KEYS + off : key0 + KEYS; };     // of tile t, key0 that of the one before
  auto group = [&](int t, int key0) {
    Group g;
    g.key0 = next_key(t, key0, 16 * w);
    g.id = __builtin_amdgcn_readlane(ids, t & 63);
    g.n = 0;                                     // (found when its keys are requested, known when its values are)
    return g;
  };
  // Keys behind the unit's last tile are requested as none, so that every tile has as many requests behind it.  16 keys
  // from `all` to all + all_span are read whole if they have a page.
  const int end = min(x.kv, (tile_of(x, x.t_hi - 1) + 1) * KEYS), all = x.behind ? (int)x.behind + a.sinks : 0;
  const uint32_t all_span = max(end - 15 - all, 0);
  auto k_issue = [&](int place, Group& g) {
    g.n = 16;
    if ((uint32_t)(g.key0 - all) >= all_span) g.n = keys_read(a, x, end, g.key0, g.id);
    if ((uint32_t)g.id >= (uint32_t)a.n_pages) g.n = 0;
    const auto rs = keys_at(a, kb, a.k_sB, a.k_row, g.key0, g.id, g.n);
    int v[NI];
    asm volatile("" : "+v"(krow), "+v"(kchunk));
#pragma unroll
    for (int jj = 0; jj < NI; ++jj) v[jj] = krow + jj * T::RPI * (int)a.k_row + (kchunk ^ (T::swz(jj * T::RPI) << 4));
    move_keys<NI>(ks_lds + place * TILE_B, rs, v);
  };
  auto v_issue = [&](int place, const Group& g) {
    const auto rs = keys_at(a, vb, a.v_sB, a.v_row, g.key0, g.id, g.n);
    int v[NI];
    asm volatile("" : "+v"(vplace));
#pragma unroll
    for (int jj = 0; jj < NI; ++jj) v[jj] = vplace + jj * T::RPI * (int)a.v_row;
    move_keys<NI>(vs_lds + place * TILE_B, rs, v);
  };
  pages(0);

  // this lane's row, straight into operand registers
  const int pos = r < wrows ? x.kv - x.nq + row_at(a, x, 32 * w + r).j : INT_MIN;
  u32x4 qf[T::NKC];
#pragma unroll
  for (int kc = 0; kc < T::NKC; ++kc) qf[kc] = u32x4{0, 0, 0, 0};
  if (r < wrows) {
    const Row me = row_at(a, x, 32 * w + r);
    const uint8_t* qr = a.q + (hk * a.G + me.g) * a.q_sH + (int64_t)(x.qs + me.j) * a.q_sT + kh * 16;
#pragma unroll
    for (int kc = 0; kc < T::NKC; ++kc) qf[kc] = *reinterpret_cast<const u32x4*>(qr + kc * 32);
  }
  Group g[AHEAD + 2];
#pragma unroll
  for (int t = 0; t < AHEAD + 2; ++t) g[t] = group(t, t ? g[t - 1].key0 : tile_of(x, x.t_lo) * KEYS + 16 * w - KEYS);
  if (ntiles > 0) {
    k_issue(0, g[0]);
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) {
      v_issue(t, g[t]);
      k_issue((t + 1) % STAGES, g[t + 1]);
    }
  }
  Group gv = g[AHEAD], gk = g[AHEAD + 1];        // of V(t + AHEAD) and K(t + AHEAD + 1), t the next tile

  // ---- operands from LDS -----------------------------------------------------------------
  struct KFrag { u32x4 x[T::NKC]; };
  // (LDS addresses: one register per lane and chunk pattern, tile and half in the offset of
  // the instruction; the empty assembly keeps the compiler from holding a register for each)
  typedef __attribute__((address_space(3))) const uint8_t* lds_ptr;
  uint32_t kaddr = ks_lds - w * 16 * T::ROWB + T::slot(r, kh);           // chunk 2 kc + kh sits at kaddr ^ (32 kc)
  asm volatile("" : "+v"(kaddr));
  auto k_read = [&](int half, KFrag& f) {
#pragma unroll
    for (int kc = 0; kc < T::NKC; ++kc)
      f.x[kc] = *(__attribute__((address_space(3))) const u32x4*)((lds_ptr)(uintptr_t)(kaddr ^ (32 * kc)) + half * 32 * T::ROWB);
  };
  // The transposing load: in every 16 lanes, lanes 4 i .. 4 i + 3 name the 16 channels of key i, and lane c receives channel
  // c of the four keys.  A lane's 8 k-indices of operand chunk s are the keys its logit accumulators 8 s .. 8 s + 7 stand for.
  const int vkey = 4 * kh + ((lane & 15) >> 2);
  const int vsub = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
  uint32_t vaddr[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    vaddr[ct] = vs_lds - w * 16 * T::ROWB + vkey * T::ROWB + (((4 * ct + vsub) ^ v_slot<DT, D>(vkey)) << 4) + (lane & 1) * 8;
    asm volatile("" : "+v"(vaddr[ct]));
  }
  auto v_read = [&](int half, int s, int ct, u32x4& f) {
    const lds_ptr base = (lds_ptr)(uintptr_t)vaddr[ct] + (half * 32 + 16 * s) * T::ROWB;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)base);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(base + 8 * T::ROWB));
    const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
    f.x = l2.x; f.y = l2.y; f.z = h2.x; f.w = h2.y;
  };

  v16f oacc[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) oacc[ct] = v16f{};
  float m = kLowestLogit, l = 0.f;   // running maximum (log2 units), this half-wave's share of the sum
  KFrag kf;
  v16f s0, s1;

  // Largest logit (log2 units) of a half in either half-wave, over the raw products (the scale is not negative).
  auto half_max = [&](const v16f& sc) {
    float t = sc[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) t = fmaxf(t, sc[v]);
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(t), __float_as_uint(t), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * a.scale_log2;
  };
  float tmax = 0.f;                                  // of the half whose weights are taken next

  // One half, of keys key0 on: weights of the logits sc, output += V^T P; unless it is the wave's LAST, the logits of the half
  // after it (operands in kf) meanwhile, their maximum, and the request of the operands of the half after that.
  auto step = [&](auto last_c, int half, int key0, bool seen_whole, v16f& sc, v16f& sn) {
    constexpr bool LAST = decltype(last_c)::value;
    u32x4 vf[2][CT];
    if (!seen_whole) {
      const int low = a.window && pos >= 0 ? pos - a.window : -1;          // keys up to it are seen as sinks only
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = key0 + acc_row(v, kh);
        if ((key > pos) | ((key <= low) & (key >= a.sinks))) sc[v] = -INFINITY;
      }
      tmax = half_max(sc);
    }
    const float m_new = fmaxf(m, tmax);
    if (__builtin_amdgcn_ballot_w64(m_new > m)) {
      const float alpha = __builtin_amdgcn_exp2f(m - m_new);
      l *= alpha;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[ct][e] *= alpha;
      m = m_new;
    }
    uint32_t pw[8];                                  // the weights, two to a word
    float psum = 0.f;
    const float nm = -m;
    if constexpr (!LAST) sn = v16f{};
#pragma unroll
    for (int kc = 0; kc < T::NKC; ++kc) {
      if constexpr (!LAST) mma_chunk<DT>(sn, kf.x[kc], qf[kc]);
      if (kc >= VS && kc < VS + CT) v_read(half, 0, kc - VS, vf[0][kc - VS]);     // (into registers kf has left)
#pragma unroll
      for (int e = kc * EPS; e < (kc + 1) * EPS; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[e], a.scale_log2, nm));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[e + 1], a.scale_log2, nm));
        psum += p0;
        psum += p1;
        pw[e >> 1] = pack_two<DT>(p0, p1);
      }
    }
    l += psum;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) v_read(half, 1, ct, vf[1][ct]);
    if constexpr (!LAST) k_read(half, kf);
    u32x4 pb[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) { pb[s].x = pw[4 * s]; pb[s].y = pw[4 * s + 1]; pb[s].z = pw[4 * s + 2]; pb[s].w = pw[4 * s + 3]; }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) mma_chunk<DT>(oacc[ct], vf[s][ct], pb[s]);
    if constexpr (!LAST) tmax = half_max(sn);        // (beside the second product, which leaves the vector units idle)
  };
  // Tile t's barrier: K(t + 1) and V(t) are complete in LDS, and nobody still reads K(t) (its second half was requested
  // before) or V(t - 1), whose places are filled next.
  int place = AHEAD % STAGES;                        // of V(t + AHEAD); K(t + AHEAD + 1) goes where K(t) was
  auto top = [&](int t) {
    if (((t + AHEAD + 2) & 63) == 0) {
      pages(t + AHEAD + 2);
      wait_all_loads();                              // (here, not where they are used: that would be a wait in every tile)
    }
    if constexpr (AHEAD > 1) wait_vmem<(AHEAD - 1) * 2 * NI>();
    else wait_all_loads();
    __syncthreads();
    v_issue(place, gv);
    place = place + 1 == STAGES ? 0 : place + 1;
    k_issue(place, gk);
    gv = gk;
    gk = group(t + AHEAD + 2, gk.key0);
  };
  int read_place = 0;                                // of V(t); K(t + 1) is in the next
  auto next_buffers = [&]() {                        // tile t + 1
    const int next = read_place + 1 == STAGES ? 0 : read_place + 1, after = next + 1 == STAGES ? 0 : next + 1;
    kaddr += (after - next) * TILE_B;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) vaddr[ct] += (next - read_place) * TILE_B;
    read_place = next;
  };
  wait_all_loads();                                  // (on every way to the loop: the compiler would wait for the rows in it, and so for the next tiles)
  if (ntiles > 0) {
    __syncthreads();
    k_read(0, kf);
    s0 = v16f{};
#pragma unroll
    for (int kc = 0; kc < T::NKC; ++kc) mma_chunk<DT>(s0, kf.x[kc], qf[kc]);
    k_read(1, kf);
    kaddr += TILE_B;                                 // the K operands of a step are read one tile ahead
    tmax = half_max(s0);
  }
  const int t_full = nh > 0 ? (nh - 1) / 2 : 0;      // tiles of whose halves none is the wave's last
  int t = 0, key0 = tile_of(x, x.t_lo) * KEYS;
  for (; t < t_full; ++t, key0 = next_key(t, key0, 0)) {
    const bool both = seen.whole(key0, 32);
    top(t);
    step(std::false_type{}, 0, key0, both, s0, s1);
    step(std::false_type{}, 1, key0 + 32, both, s1, s0);
    next_buffers();
  }
  if (nh > 0) {                                      // the tile of the last (t < ntiles: the wave has rows)
    top(t++);
    if (nh & 1) {
      step(std::true_type{}, 0, key0, seen.whole(key0), s0, s1);
    } else {
      step(std::false_type{}, 0, key0, seen.whole(key0), s0, s1);
      step(std::true_type{}, 1, key0 + 32, seen.whole(key0 + 32), s1, s0);
    }
  }
  for (; t < ntiles; ++t) top(t);                    // the other waves' tiles: their transfers and barriers
  wait_all_loads();                                  // (nothing is on its way to a workgroup's memory when it ends)

  // ---- normalise and store: lane = row, accumulator v of tile ct = channel 32 ct + acc_row(v, kh) ----
  const float l_tot = l + __shfl_xor(l, 32);
  if (pos == INT_MIN) return;
  const Row me = row_at(a, x, 32 * w + r);
  const bool whole = x.parts == 1;
  const float inv = !whole ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
  const int64_t prow = part_row(a, hk, unit_of_grid()) + 32 * w + r, hq = hk * a.G + me.g, tok = x.qs + me.j;
  uint8_t* orow = a.o + hq * a.o_sH + tok * a.o_sT;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int v4 = 0; v4 < 4; ++v4) {
      const int c = 32 * ct + acc_row(4 * v4, kh);        // four consecutive channels
      const float4 o = make_float4(oacc[ct][4 * v4] * inv, oacc[ct][4 * v4 + 1] * inv, oacc[ct][4 * v4 + 2] * inv, oacc[ct][4 * v4 + 3] * inv);
      if (!whole) *reinterpret_cast<float4*>(a.part_o + prow * D + c) = o;
      else *reinterpret_cast<uint2*>(orow + c * 2) = make_uint2(pack_two<DT>(o.x, o.y), pack_two<DT>(o.z, o.w));
    }
  if (kh == 0) {
    if (!whole) *reinterpret_cast<float2*>(a.part_ml + prow * 2) = make_float2(m, l_tot);
    else if (a.lse) a.lse[hq * a.T + tok] = l_tot == 0.f ? -INFINITY : (m + log2f(l_tot)) * kLn2;
  }
}

// Four channels of a row whose parts are together: reference M, sum l, weighted values o.
template <int DT>
__device__ inline void store_row(const PagedArgs& a, int tok0, int g0, int hk, int row, int c, float M, float l, float4 o) {
  const Row me = row_at(a, tok0, g0, row);
  const int64_t hq = hk * a.G + me.g, tok = me.j;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint8_t* orow = a.o + hq * a.o_sH + tok * a.o_sT;
  if constexpr (DT == ZC_F32) *reinterpret_cast<float4*>(orow + c * 4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else *reinterpret_cast<uint2*>(orow + c * 2) = make_uint2(pack_two<DT>(o.x * inv, o.y * inv), pack_two<DT>(o.z * inv, o.w * inv));
  if (a.lse && c == 0) a.lse[hq * a.T + tok] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
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
