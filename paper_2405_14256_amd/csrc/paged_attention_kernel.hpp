// Attention of a block of rows over keys and values in pages: what zc_paged_attention and zc_paged_shared_attention run on.
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
// A unit of work is a block of rows and a part of the key tiles it sees, described by an X of the kernel's own:
//   rows, kv, p0, p1        rows of the block; tokens; positions of the block's first and last row
//   kFirst                  the least position of a row that sees a key
//   t_lo, t_hi              tiles of this unit
//   first, sink_tiles       tile t is of the keys behind those of tile t - 1, tile sink_tiles of those from first * kTile on
//   qs                      token of a row: qs + row_of(a, x, r).j; where nothing is to be joined, and for its position, qs + row_at(a, x, r).j
//   behind                  16 keys from key0 on are behind every window if key0 - sinks, without sign, is less
// and by functions that are found by its type: row_at, row_of, position, tile_of and tile_at (tiles and their keys), entry_of, keys_read and keys_at
// (where keys lie), seen_by, low_of and sinks_of (who sees them: keys up to low, from sinks on, are hidden), is_whole (nothing is to be joined), part_of (where
// partial results go).
#pragma once

#include <limits.h>
#include <stdint.h>
#include <type_traits>

#include "paged_args.hpp"
#include "paged_keys.hpp"

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

// Row r of a block: its token (after the block's first) and head.
struct Row { int j, g; };
__device__ inline Row row_at(const PagedArgs& a, int j0, int g0, int r) {
  const int v = g0 + r, j = a.G == 1 ? v : (int)__umulhi((uint32_t)v, a.over_G);    // (exact while v G < 2^32)
  return {j0 + j, v - j * a.G};
}
__device__ inline int unit_of_grid() { return blockIdx.y + 65535 * blockIdx.z; }

// The page of 16 keys from key0 on (past the table: any, no key is read).
template <class X> __device__ inline int page_of(const PagedArgs& a, const X& x, int key0) {
  return *(__attribute__((address_space(4))) const int32_t*)(uintptr_t)entry_of(a, x, key0);
}
// The blocks of 32 keys that every row from position p0 to p1 sees whole: those from `low` on, `span` of them by their first key, and
// those whose first key is below `sink`.
struct Seen {
  int low, sink;
  uint32_t span;
  // Blocks of 32 + more keys.
  __device__ bool whole(int key0, int more = 0) const { return (uint32_t)(key0 - low) < (uint32_t)max((int)span - more, 0) || key0 < sink - more; }
};

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
template <int DT, int D, int NW, class X>
__device__ __forceinline__ void attend_rows(const PagedArgs& a, const X& x, int hk, uint8_t* mem, float (*sum)[2][64]) {
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
      const auto rs = keys_at(a, x, head, sB, row, s.key0 + 16 * g, s.id[g], s.n[g]);
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
  const int pos = mine ? position(x, me.j) : -1;
  u32x4 qf[T::NKC];
#pragma unroll
  for (int kc = 0; kc < T::NKC; ++kc) qf[kc] = u32x4{0, 0, 0, 0};
  if (mine) {
    const Row from = row_of(a, x, r);
    const uint8_t* qr = a.q + (hk * a.G + from.g) * a.q_sH + (int64_t)(x.qs + from.j) * a.q_sT + kh * 16;
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

  const Seen seen = seen_by(a, x, x.p0, x.p1);
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
      const int low = low_of(a, x, pos), sinks = sinks_of(a, x);           // keys up to `low` are seen as sinks only
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = key0 + acc_row(v, kh);
        if ((key > pos) | ((key <= low) & (key >= sinks))) s[v] = -INFINITY;
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
  const bool whole = is_whole(x);
  const int64_t prow = part_of(a, x, hk) + r;
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
template <int DT, int D, class X>
__device__ __forceinline__ void attend_tiles(const PagedArgs& a, const X& x, int hk, uint8_t* mem) {
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

  const int wrows = min(max(x.rows - 32 * w, 0), 32);        // this wave's rows
  // the halves of this unit that the wave's rows see: all up to the last row's
  const int wp0 = position(x, row_at(a, x, 32 * w).j), wp1 = wrows > 0 ? position(x, row_at(a, x, 32 * w + wrows - 1).j) : INT_MIN;
  const int ntiles = x.t_hi - x.t_lo;
  const Seen seen = seen_by(a, x, wp0, wp1);
  int nh = 0;
  if (wp1 >= X::kFirst) {
    const int t1 = tile_at(x, wp1) - x.t_lo;     // the tile of the last row's own token
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
    ids = *entry_of(a, x, key0);
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
    const auto rs = keys_at(a, x, kb, a.k_sB, a.k_row, g.key0, g.id, g.n);
    int v[NI];
    asm volatile("" : "+v"(krow), "+v"(kchunk));
#pragma unroll
    for (int jj = 0; jj < NI; ++jj) v[jj] = krow + jj * T::RPI * (int)a.k_row + (kchunk ^ (T::swz(jj * T::RPI) << 4));
    move_keys<NI>(ks_lds + place * TILE_B, rs, v);
  };
  auto v_issue = [&](int place, const Group& g) {
    const auto rs = keys_at(a, x, vb, a.v_sB, a.v_row, g.key0, g.id, g.n);
    int v[NI];
    asm volatile("" : "+v"(vplace));
#pragma unroll
    for (int jj = 0; jj < NI; ++jj) v[jj] = vplace + jj * T::RPI * (int)a.v_row;
    move_keys<NI>(vs_lds + place * TILE_B, rs, v);
  };
  pages(0);

  // this lane's row, straight into operand registers
  const int pos = r < wrows ? position(x, row_at(a, x, 32 * w + r).j) : INT_MIN;
  u32x4 qf[T::NKC];
#pragma unroll
  for (int kc = 0; kc < T::NKC; ++kc) qf[kc] = u32x4{0, 0, 0, 0};
  if (r < wrows) {
    const Row me = row_of(a, x, 32 * w + r);
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
      const int low = low_of(a, x, pos), sinks = sinks_of(a, x);           // keys up to `low` are seen as sinks only
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = key0 + acc_row(v, kh);
        if ((key > pos) | ((key <= low) & (key >= sinks))) sc[v] = -INFINITY;
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
  const bool whole = is_whole(x);
  const float inv = !whole ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
  const int64_t prow = part_of(a, x, hk) + 32 * w + r, hq = hk * a.G + me.g, tok = x.qs + me.j;
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

}  // namespace zc
