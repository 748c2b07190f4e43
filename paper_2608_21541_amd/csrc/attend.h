// Attention of new queries over a packed cache of any format and new rows: the kernel.
//
// For query row (t, head h G + g) of sequence b, over the unit's packed rows and the
// sequence's new rows j that mask[b][t][j] admits:
//   z_i = scale <q, k_i>,  out = sum_i softmax(z)_i v_i,  lse = log sum_i e^z_i,
// with out = 0 and lse = -inf where no row is visible.
//
// Rows are taken in tiles of 32, queries in tiles of 16:
//   S^T = K Q^T on v_mfma_f32_16x16x32_bf16 with the keys as the A operand, so that
//     lane (g, c) = (lane / 16, lane % 16) holds query c and keys 4 g + i and
//     16 + 4 g + i (i = 0..3) of the tile;
//   a running sum in log2 units against a reference, the row's maximum when it was
//     last moved: only when a weight would exceed 2^8 (and the sums are rescaled);
//   O^T += V^T P^T on the same instruction: P^T (the B operand) is the lane's own
//     eight weights, V^T (the A operand) comes from transposing LDS reads of the
//     row-major value tile along the same key order.
// A weight is three bf16 whose sum it is exactly, eight of its 24 bits in each.  (Two,
// rounded, leave an error of 2e-6 against 64 bits where fp32 sums leave 4e-7, and one
// 1e-3; a call of 128 query rows over 3.36M rows of mxfp8 takes 420 us with three, 353 with
// two, and of 4 query rows over mxfp4 87 and 83.)
// Codes become bf16 values, exactly, on the way from memory to the matrix unit: a
// conversion takes the block's scale as its operand (one instruction for two codes).
//
// A workgroup has the query rows of NQ waves, each with QT query tiles.  With up to 64 query
// rows (NQ = 1, of which QT = 2 tiles are 32) it is four such groups that take the tiles in
// turn (KS), every wave a group by itself: it reads keys straight into MFMA operands, only
// values pass through its LDS tile, and no wave waits for another until the groups are joined
// at the end.  With more rows (NQ = 4 or 8, QT = 2) its waves convert the tiles together, each
// its share, two tiles to a stage, into LDS buffers ahead of those that they multiply, with
// one barrier for a stage.
//
// Bounds (calls, the join of partials included): one to sixteen query rows, the reads (3.36M
// rows of 128 dims, mxfp4, 4 query rows of each: 459 MB in 86 us, 5.3 TB/s; mxfp8: 890 MB in
// 143, 6.2 TB/s); many, the issue of matrix and vector instructions, with little of either
// under the other (the same rows of mxfp8, 128 query rows: 413 us; 256, with 64 new rows to
// a unit: 755 us, 1.2 PFLOP/s with the weights' three parts counted, which is what a library's
// plain product of 8192^3 reaches).  One layer's kernel is latency: 6.3 us for 13.1k rows.
#pragma once

#include "mx.h"
#include "stages.h"

namespace certkv {

typedef __bf16 at_bf16x8 __attribute__((__vector_size__(8 * sizeof(__bf16))));
typedef float at_f32x4 __attribute__((__vector_size__(4 * sizeof(float))));
typedef short at_s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) at_s16x4 at_lds_s16x4;

constexpr float kAtLog2e = 1.4426950408889634f;
constexpr float kAtLn2 = 0.6931471805599453f;
constexpr float kAtSlack = 8.f;    // log2 of the weight beyond which a row's reference moves
constexpr float kAtNone = -3e38f;  // the reference of a row that has seen nothing

// The rows of all units in one order, cut into chunks of equal length, one for each
// workgroup that is resident at once: the packed rows, each unit's from a place that
// follows from its first row alone (a sum over the units before would need a pass), and
// apart from them the new rows, tn of each unit.  Places are multiples of 32, so that no
// tile straddles units; a unit's place is at least `gap` rows beyond the rows before it,
// which stand for what a piece costs beside its tiles.  A chunk that crosses from one
// unit to the next is two pieces.
__device__ __forceinline__ uint32_t at_up32(uint32_t x) { return (x + 31u) & ~31u; }
struct AtCut {
  uint32_t keys, total;
};
__device__ __forceinline__ AtCut at_cut(uint32_t total, uint32_t parts, uint32_t most,
                                        uint32_t least) {
  uint32_t k = (total + parts - 1u) / parts;
  k = min(max(k, least), (uint32_t)kAtMaxKeys);
  // (more rows than the caller's bound allows for: longer chunks, so that the partials
  // stay within the workspace)
  if (total > (uint64_t)most * k) k = (total + most - 1u) / most;
  return AtCut{(k + least - 1u) / least * least, total};
}
__device__ __forceinline__ uint32_t at_place(int64_t rows_before, uint32_t u, int32_t gap) {
  return at_up32((uint32_t)rows_before) + u * (uint32_t)gap;
}
__device__ __forceinline__ AtCut at_cut_packed(const AttendArgs& a, int64_t rows) {
  return at_cut(at_place(rows, (uint32_t)a.U, a.ck.gap), a.ck.parts, a.ck.most, kAtMinKeys);
}
__device__ __forceinline__ AtCut at_cut_new(const AttendArgs& a) {
  return at_cut((uint32_t)a.U * at_up32((uint32_t)a.tn), a.ck.parts, a.ck.most_new, kAtTile);
}

// How a lane holds W bytes of a row in format F: eight or more consecutive dims.  NT:
// loaded non-temporally.
constexpr int kAtNT = 2;  // (the instruction's bit)
template <int F, int W>
struct AtRaw;
template <int F>
struct AtRaw<F, 16> {
  uint4 x;
  template <bool NT>
  __device__ __forceinline__ void load(BufRsrc r, uint32_t off) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, NT ? kAtNT : 0);
    x = make_uint4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ uint2 codes8(int s) const {
    return F == CERTKV_CACHE_MXFP8 ? (s ? make_uint2(x.z, x.w) : make_uint2(x.x, x.y))
                                   : make_uint2((&x.x)[s], 0u);
  }
};
template <int F>
struct AtRaw<F, 8> {
  uint2 x;
  template <bool NT>
  __device__ __forceinline__ void load(BufRsrc r, uint32_t off) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b64(r, (int)off, 0, NT ? kAtNT : 0);
    x = make_uint2(v[0], v[1]);
  }
  __device__ __forceinline__ uint2 codes8(int s) const {
    return F == CERTKV_CACHE_MXFP8 ? x : make_uint2((&x.x)[s], 0u);
  }
};
template <int F>
struct AtRaw<F, 4> {
  uint32_t x;
  template <bool NT>
  __device__ __forceinline__ void load(BufRsrc r, uint32_t off) {
    x = __builtin_amdgcn_raw_buffer_load_b32(r, (int)off, 0, NT ? kAtNT : 0);
  }
  __device__ __forceinline__ uint2 codes8(int) const { return make_uint2(x, 0u); }
};
// Dims 8 s .. 8 s + 7 of a lane's piece as bf16.
template <int F, int W>
__device__ __forceinline__ uint4 at_bf16(const AtRaw<F, W>& r, int s, float scale) {
  if constexpr (F == CERTKV_CACHE_BF16)
    return r.x;
  else
    return mx_decode8<F>(r.codes8(s), scale);
}

// The upper halves of two floats, a's in the low half: bf16, cut off.
__device__ __forceinline__ uint32_t at_upper(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

// LDS tiles: 32 rows of D bf16 in natural order.  Keys are read a 16-byte chunk per
// lane, sixteen rows at a time; values by transposing reads, eight rows of 32 bytes per
// half-wave: rows padded by 16 and by 32 bytes spread either over all banks, and leave
// every access at a constant distance from one address.
template <int D>
struct AtTile {
  static constexpr int KROW = D / 8 + 1, VROW = D / 8 + 2;  // 16-byte chunks per row
  static constexpr int K = kAtTile * KROW * 8, V = kAtTile * VROW * 8;  // bf16 elements
};
template <int D>
__device__ __forceinline__ int at_key_chunk(int r, int c) {
  return r * AtTile<D>::KROW + c;
}
template <int D>
__device__ __forceinline__ int at_value_chunk(int r, int c) {
  return r * AtTile<D>::VROW + c;
}

template <int D, int NQ, int QT>
struct AtShape {
  static constexpr int KS = NQ == 1 ? 4 : 1;
  static constexpr int NT = 64 * NQ * KS;
  static constexpr int SUB = NQ == 1 ? 1 : 2;         // tiles that a group takes at a time
  static constexpr int KT = NQ == 1 ? 0 : 2 * SUB;    // key tiles of a group in LDS: half are
                                                      // read, half written
  static constexpr int VT = NQ == 1 ? 1 : 2 * SUB;    // value tiles
  static constexpr int PARTS = 3;                     // bf16 parts of a weight
  static constexpr int ROW = D + 4;                   // floats of a joined output row
  static constexpr int JOIN = KS == 1 ? 0 : 2 * KS * NQ * 16 * ROW;  // bf16 elements
  static constexpr int GROUP = KT * AtTile<D>::K + VT * AtTile<D>::V;  // bf16 elements
  static constexpr int TILES = KS * GROUP;
  static constexpr int LDS = TILES > JOIN ? TILES : JOIN;
};

// The state of a wave's query rows.
template <int D, int QT>
struct AtAcc {
  float m[QT], l[QT];
  at_f32x4 o[QT][D / 16];
};

// The largest of a lane's eight scores; NaN where one is (as the row's sum will be), which
// is one instruction for three where fmaxf first has to quiet each.
__device__ __forceinline__ float at_max8(const at_f32x4 s[2]) {
  float m = s[0][0];
#pragma unroll
  for (int i = 1; i < 8; ++i) m = __builtin_elementwise_maximum(m, s[i >> 2][i & 3]);
  return m;
}
// Before the scores become weights: where a score (raw products; a row's factor, c2 but for
// huge scores (ref_factor), turns them into log2 units) is more than 8 above its row's
// reference, as in a row's first tile, the references move to the maxima and the sums are
// rescaled.  Rows that have seen nothing keep kAtNone, under which a masked score's weight is
// zero.
template <int D, int QT>
__device__ __forceinline__ void at_reference(AtAcc<D, QT>& a, const float most[QT], float c2) {
  bool above = false;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt)
    above |= most[qt] * ref_factor(a.m[qt], c2) > a.m[qt] + kAtSlack;
  if (__builtin_amdgcn_ballot_w64(above) == 0) return;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    float mt = most[qt];
    mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
    mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
    const float mnew = fmaxf(a.m[qt], ref_of(mt, c2));
    const float alpha = __builtin_amdgcn_exp2f(a.m[qt] - mnew);
    a.m[qt] = mnew;
    a.l[qt] *= alpha;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) a.o[qt][db] *= alpha;
  }
}
// The parts of a query tile's weights, eight of a lane: the upper half of each, of the
// remainder, and so on.
template <int PARTS>
struct AtParts {
  uint4 p[PARTS];
};
// Two weights (i even) of one query tile's scores s; c: the row's factor.
template <int D, int QT, int PARTS>
__device__ __forceinline__ void at_weights2(AtAcc<D, QT>& a, int qt, int i, const at_f32x4 s[2],
                                            float c, AtParts<PARTS>& w) {
  float p0 = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], c, -a.m[qt]));
  float p1 = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][(i + 1) & 3], c, -a.m[qt]));
  a.l[qt] += p0 + p1;
#pragma unroll
  for (int k = 0; k < PARTS; ++k) {
    (&w.p[k].x)[i >> 1] = at_upper(p0, p1);
    p0 -= __uint_as_float(__float_as_uint(p0) & 0xffff0000u);
    p1 -= __uint_as_float(__float_as_uint(p1) & 0xffff0000u);
  }
}

// V^T of block db of 16 dims: lane c of group g is to hold dim c of the block at keys
// 4 g + i, 16 + 4 g + i.  In a transposing read, lane c addresses key c / 4 of the four at
// dims 4 (c % 4) .. + 3.
template <int D>
__device__ __forceinline__ at_bf16x8 at_value_block(const uint16_t* vt, int db, int lane) {
  const int g = lane >> 4, c = lane & 15;
  uint2 v[2];
#pragma unroll
  for (int rd = 0; rd < 2; ++rd) {
    const int r = 16 * rd + 4 * g + (c >> 2), dim = 16 * db + 4 * (c & 3);
    const uint16_t* src = vt + at_value_chunk<D>(r, dim >> 3) * 8 + (dim & 7);
    v[rd] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (at_lds_s16x4*)(__attribute__((address_space(3))) uint16_t*)src));
  }
  return __builtin_bit_cast(at_bf16x8, make_uint4(v[0].x, v[0].y, v[1].x, v[1].y));
}
// O^T += V^T P^T of a block.
template <int D, int QT, int PARTS>
__device__ __forceinline__ void at_value_products(AtAcc<D, QT>& a, int db, at_bf16x8 vf,
                                                  const AtParts<PARTS> w[QT]) {
#pragma unroll
  for (int k = 0; k < PARTS; ++k)
#pragma unroll
    for (int qt = 0; qt < QT; ++qt)
      a.o[qt][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          vf, __builtin_bit_cast(at_bf16x8, w[qt].p[k]), a.o[qt][db], 0, 0, 0);
}
template <int D, int QT, int PARTS>
__device__ __forceinline__ void at_values(AtAcc<D, QT>& a, const uint16_t* vt,
                                          const AtParts<PARTS> w[QT], int lane) {
#pragma unroll
  for (int db = 0; db < D / 16; ++db)
    at_value_products<D, QT, PARTS>(a, db, at_value_block<D>(vt, db, lane), w);
}

// The packed rows' offsets, as a wave reads them: those of 64 units at a time in its lanes,
// so that a unit's place, its rows and the next unit's are one load to wait for, not three
// in turn; up to 64 units the same load tells the rows in all.
struct AtOffsets {
  const int64_t* __restrict__ off;
  uint32_t U;
  uint32_t at;         // the first of the 64
  int64_t base, rows;
  int64_t first, end;  // rows of unit at + lane
  __device__ __forceinline__ AtOffsets(const int64_t* o, int64_t units, int lane)
      : off(o), U((uint32_t)units), at(0), base(0), rows(0), first(0), end(0) {
    if (units == 0) return;  // (not asked for)
    window(0, lane);
    base = lane64(first, 0);
    rows = (units <= 64 ? lane64(end, U - 1) : off[U]) - base;
  }
  __device__ __forceinline__ void window(uint32_t u, int lane) {
    at = u;
    first = off[min(u + lane, U)];
    end = off[min(u + lane + 1, U)];
  }
  static __device__ __forceinline__ int64_t lane64(int64_t x, uint32_t i) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, i);
    const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)((uint64_t)x >> 32), i);
    return (int64_t)(((uint64_t)hi << 32) | lo);
  }
  // a unit's first row and the one behind its last
  __device__ __forceinline__ void unit(uint32_t u, int lane, int64_t& p0, int64_t& p1) {
    if (u - at >= 64) window(u, lane);
    p0 = lane64(first, u - at);
    p1 = lane64(end, u - at);
  }
  // The unit whose place holds row r of the common order: 64 units' ends per step.
  __device__ __forceinline__ uint32_t find(uint32_t r, int32_t gap, int lane) {
    uint32_t lo = 0, n = U;  // the answer is one of [lo, lo + n]
    while (n > 64) {
      const uint32_t step = (n + 63) / 64, i = lo + lane * step + step - 1;
      const bool past = i >= U || at_place(off[min(i + 1, U)] - base, i + 1, gap) > r;
      lo += (uint32_t)__popcll(__ballot(!past)) * step;
      n = step;
    }
    if (lo != at) window(lo, lane);
    const uint32_t i = lo + lane;
    const uint64_t past = __ballot(i >= U || at_place(end - base, i + 1, gap) > r);
    return past ? min(lo + (uint32_t)__builtin_ctzll(past), U) : U;
  }
};

// Whether a bf16 of the eight is not finite.
__device__ __forceinline__ bool at_bad8(uint4 x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
  return bad;
}

// The packed rows of the workgroup's chunks (F: their format), or the new rows (NEW, bf16).
template <int F, int D, int NQ, int QT, bool NEW>
__device__ __forceinline__ void attend_rows(const AttendArgs& a, uint16_t* lds, float2* ml_s,
                                            uint32_t* bad_s) {
  using Shape = AtShape<D, NQ, QT>;
  constexpr int KS = Shape::KS, NT = Shape::NT, PARTS = Shape::PARTS;
  constexpr int BITS = F == CERTKV_CACHE_BF16 ? 16 : F == CERTKV_CACHE_MXFP8 ? 8 : 4;
  constexpr bool MX = F != CERTKV_CACHE_BF16;
  constexpr int RB = mx_row_bytes(F, D);  // bytes of a row
  constexpr int KSTEP = D / 32;
  // keys read straight into operands (NQ = 1): lane (g, c) holds WK bytes of row c at a
  // time, EK dims, so that the four groups read 4 WK consecutive bytes
  constexpr int WK = 32 * RB / 128 >= 16 ? 16 : 8, EK = NQ == 1 ? WK * 8 / BITS : 8;
  constexpr int SK = EK / 8, NLK = KSTEP / SK;
  // a row-major tile: W bytes of a lane, the tile in NLT pieces of a wave; alone, a wave
  // takes the values, in a group the waves take turns at the keys' and the values' pieces
  constexpr int TB = kAtTile * RB;
  constexpr int W = NQ == 1 || !MX || 2 * TB / (64 * 16) >= NQ ? 16
                    : F == CERTKV_CACHE_MXFP8 || 2 * TB / (64 * 8) >= NQ ? 8 : 4;
  constexpr int EV = W * 8 / BITS, LPR = RB / W, NLT = TB / (64 * W), RPL = 64 / LPR;
  constexpr int PER = NQ == 1 ? NLT : (2 * NLT + NQ - 1) / NQ;

  const Geo& gm = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave / NQ, qw = wave % NQ;
  const int g = lane >> 4, c = lane & 15;
  const int M = a.tq * gm.G, mp = a.ck.mp;
  const float c2 = gm.scale * kAtLog2e;
  const uint32_t U = (uint32_t)a.U;

  // Query groups (more rows than a workgroup holds) of a chunk: eight workgroups apart, on
  // the same XCD, whose L2 then serves all but the first.  New rows' chunks are dealt from
  // the other end: with few of either no workgroup has both.
  const int wgx = NEW ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
  const int qg = (wgx >> 3) % a.ck.qgroups;
  const uint32_t x0 = a.ck.qgroups == 1 ? wgx : (wgx >> 3) / a.ck.qgroups * 8 + (wgx & 7);
  const uint32_t xstep = gridDim.x / a.ck.qgroups;
  const int row0 = (qg * NQ + qw) * QT * 16;  // a wave's first query row
  const bool active = row0 < M;
  auto kdim = [&](int ks) { return (ks / SK) * 4 * EK + g * EK + 8 * (ks % SK); };

  uint16_t* const group_lds = lds + kg * Shape::GROUP;
  auto key_tile = [&](int n) { return group_lds + (n & 3) * AtTile<D>::K; };  // of tile n
  auto value_tile = [&](int buf, int j) {
    return group_lds + Shape::KT * AtTile<D>::K + (buf * Shape::SUB + j) * AtTile<D>::V;
  };

  AtOffsets off(a.cache.offsets, NEW ? 0 : a.U, lane);
  const AtCut cut = NEW ? at_cut_new(a) : at_cut_packed(a, off.rows);
  const uint32_t tnp = at_up32((uint32_t)a.tn);
  const uint32_t nch = (cut.total + cut.keys - 1) / cut.keys;
  for (uint32_t x = x0; x < nch; x += xstep) {
    const uint32_t r0 = x * cut.keys, r1 = min(cut.total, r0 + cut.keys);
    for (uint32_t u = NEW ? r0 / tnp : off.find(r0, a.ck.gap, lane); u < U; ++u) {
      int64_t p0 = 0, p1 = 0;
      if constexpr (!NEW) off.unit(u, lane, p0, p1);
      const uint32_t vs = NEW ? u * tnp : at_place(p0 - off.base, u, a.ck.gap);
      if (vs >= r1) break;
      // the piece: rows [lo, lo + np) of the unit's
      const uint32_t len = NEW ? (uint32_t)a.tn : (uint32_t)min(p1 - p0, a.cover);
      const uint32_t lo = max(r0, vs) - vs;
      const int np = (int)min(r1 - vs, len) - (int)lo;
      if (np <= 0) continue;  // (only what lies between units)
      const int ntp = (np + kAtTile - 1) / kAtTile;
      const int h = (int)(u % (uint32_t)gm.H), b = (int)(u / gm.H % (uint32_t)gm.B);
      const int l = (int)(u / gm.H / gm.B);

      // Its rows; reads past them return zero.  (New rows keep their strides; what lies past
      // the last one is not used.)
      const int64_t at = p0 + lo;
      const uint32_t kst = NEW ? (uint32_t)a.k_new.s_token * 2u : RB;
      const uint32_t vst = NEW ? (uint32_t)a.v_new.s_token * 2u : RB;
      const uint16_t* vn = static_cast<const uint16_t*>(a.v_new.ptr) + l * a.v_new.s_layer +
                           ((int64_t)b * a.tn + lo) * a.v_new.s_token + h * a.v_new.s_head;
      const uint16_t* kn = static_cast<const uint16_t*>(a.k_new.ptr) + l * a.k_new.s_layer +
                           ((int64_t)b * a.tn + lo) * a.k_new.s_token + h * a.k_new.s_head;
      const BufRsrc kr = NEW ? make_rsrc(kn, (np - 1) * kst + RB)
                             : make_rsrc(static_cast<const uint8_t*>(a.cache.k) + at * RB, np * RB);
      const BufRsrc vr = NEW ? make_rsrc(vn, (np - 1) * vst + RB)
                             : make_rsrc(static_cast<const uint8_t*>(a.cache.v) + at * RB, np * RB);
      const BufRsrc ksr = make_rsrc(a.cache.k_scales + (MX ? at * (D / 32) : 0), MX ? np * (D / 32) : 0);
      const BufRsrc vsr = make_rsrc(a.cache.v_scales + (MX ? at * (D / 32) : 0), MX ? np * (D / 32) : 0);

      AtAcc<D, QT> acc;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        acc.m[qt] = kAtNone;
        acc.l[qt] = 0.f;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) acc.o[qt][db] = (at_f32x4){0.f, 0.f, 0.f, 0.f};
      }
      uint4 q[QT][KSTEP];
      auto load_queries = [&]() {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const int row = row0 + qt * 16 + c, rc = min(row, M - 1);
          const uint16_t* src = static_cast<const uint16_t*>(a.q.ptr) + l * a.q.s_layer +
                                (int64_t)(b * a.tq + rc / gm.G) * a.q.s_token +
                                (int64_t)(h * gm.G + rc % gm.G) * a.q.s_head;
#pragma unroll
          for (int ks = 0; ks < KSTEP; ++ks) {
            q[qt][ks] = *reinterpret_cast<const uint4*>(src + kdim(ks));
            if (row >= M) q[qt][ks] = make_uint4(0u, 0u, 0u, 0u);
          }
        }
      };

      // Scores of a tile whose keys' operands are kf(kb, ks).
      auto scores = [&](auto kf, at_f32x4 s[QT][2]) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) s[qt][kb] = (at_f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KSTEP; ++ks) {
            const at_bf16x8 k = __builtin_bit_cast(at_bf16x8, kf(kb, ks));
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
              s[qt][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  k, __builtin_bit_cast(at_bf16x8, q[qt][ks]), s[qt][kb], 0, 0, 0);
          }
        }
      };
      // Which of the lane's eight keys of new tile t each query sees, a bit each.
      auto see = [&](int t, uint32_t seen[QT]) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          seen[qt] = 0;
          const int row = row0 + qt * 16 + c, tt = min(row, M - 1) / gm.G;
          const uint8_t* mrow = a.mask + ((int64_t)b * a.tq + tt) * a.tn;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = t * kAtTile + 16 * (i >> 2) + 4 * g + (i & 3), j = (int)lo + r;
            bool sees = j <= a.tn - a.tq + tt;
            if (a.mask) sees = mrow[min(j, a.tn - 1)] != 0;
            seen[qt] |= (uint32_t)(sees && r < np && row < M) << i;
          }
        }
      };
      // Scores masked: of the packed rows, those past the piece; of new rows, those that a
      // query does not see.
      auto mask_scores = [&](at_f32x4 s[QT][2], int t, const uint32_t seen[QT]) {
        if (!NEW && np - t * kAtTile >= kAtTile) return;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (NEW ? !(seen[qt] >> i & 1)
                    : 16 * (i >> 2) + 4 * g + (i & 3) >= np - t * kAtTile)
              s[qt][i >> 2][i & 3] = -INFINITY;
      };
      // New rows whose values are not all finite (rare) are zero in the tile; their bits are
      // `bad`, and they reach only the queries that see them.
      auto add_bad = [&](uint32_t bad, int t, const AtParts<PARTS> w[QT], const uint32_t seen[QT]) {
        while (bad) {
          const int r = __builtin_ctz(bad);
          bad &= bad - 1;
          const int i = 4 * (r >> 4) + (r & 3), src = ((r >> 2) & 3) * 16 + c;
          const uint16_t* vrow = vn + (int64_t)(t * kAtTile + r) * a.v_new.s_token;
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) {
            float p = 0.f;  // the weight: the sum of its parts
#pragma unroll
            for (int k = PARTS - 1; k >= 0; --k) {
              const uint4 v = w[qt].p[k];
              uint32_t x = i >> 1 == 1 ? v.y : v.x;
              x = i >> 1 == 2 ? v.z : x;
              x = i >> 1 == 3 ? v.w : x;
              p += i & 1 ? bf16_hi(x) : bf16_lo(x);
            }
            p = __shfl(p, src, 64);
            const bool see = (__shfl(seen[qt], src, 64) >> i) & 1;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
              const uint2 v = *reinterpret_cast<const uint2*>(vrow + 16 * db + 4 * g);
              const float e[4] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)};
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (see) acc.o[qt][db][k] = fmaf(p, e[k], acc.o[qt][db][k]);
            }
          }
        }
      };
      // A lane's part of the tile's row r of new values: zero past the last row, and where the
      // row holds a value that is not finite, whose rows' bits are returned.
      auto finite_rows = [&](uint4& v, int t, int n) {
        const bool past = t * kAtTile + n * RPL + lane / LPR >= np;
        const uint64_t any = __ballot(!past && at_bad8(v));
        const uint64_t own = any >> (lane / LPR * LPR) & ((1ull << LPR) - 1);
        if (own || past) v = make_uint4(0u, 0u, 0u, 0u);
        uint32_t bad = 0;
        if (any) {
#pragma unroll
          for (int i = 0; i < RPL; ++i)
            if (any >> (i * LPR) & ((1ull << LPR) - 1)) bad |= 1u << (n * RPL + i);
        }
        return bad;
      };

      if constexpr (NQ == 1) {
        uint16_t* const vt = value_tile(0, 0);
        AtRaw<F, WK> kx[2][NLK];
        AtRaw<F, W> vx[PER];
        uint32_t ksc[2] = {}, vsc[PER] = {};
        auto load_keys = [&](int t) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const uint32_t r = t * kAtTile + kb * 16 + c;
#pragma unroll
            for (int i = 0; i < NLK; ++i) kx[kb][i].template load<false>(kr, r * kst + g * WK + i * 4 * WK);
            if constexpr (MX) ksc[kb] = D == 128 ? buf_load_u32(ksr, r * 4) : buf_load_u16(ksr, r * 2);
          }
        };
        auto load_values = [&](int t) {
#pragma unroll
          for (int n = 0; n < PER; ++n) {
            const uint32_t r = t * kAtTile + n * RPL + lane / LPR;
            // (a tile is read once; 3.36M rows, one query, mxfp8: 159 us without, 144 with;
            // keys too: 143, but a second query group then takes 291 instead of 253)
            vx[n].template load<!NEW>(vr, r * vst + (lane % LPR) * W);
            if constexpr (MX)
              vsc[n] = __builtin_amdgcn_raw_buffer_load_b8(
                  vsr, (int)(r * (D / 32) + (lane % LPR) * EV / 32), 0, 0);
          }
        };
        // (new rows of 128 dims beside two query tiles: registers for either keys or values; 404k
        // packed and 26k new rows, 32 query rows: 55 us, with both ahead 56)
        constexpr bool AHEAD = !(NEW && D == 128 && QT == 2);
        if (AHEAD && kg < ntp) {
          load_keys(kg);
          load_values(kg);
        }
        load_queries();
        for (int t = kg; t < ntp; t += KS) {
          if (!AHEAD) load_keys(t);
          uint32_t seen[QT];
          if constexpr (NEW) see(t, seen);
          if (!AHEAD) load_values(t);
          at_f32x4 s[QT][2];
          scores(
              [&](int kb, int ks) {
                const int i = ks / SK;
                float f = 1.f;
                if constexpr (MX) f = mx_scale((ksc[kb] >> (8 * ((i * 4 + g) * EK / 32))) & 255u);
                return at_bf16<F, WK>(kx[kb][i], ks % SK, f);
              },
              s);
          if (AHEAD && t + KS < ntp) load_keys(t + KS);
          uint32_t bad = 0;
#pragma unroll
          for (int n = 0; n < PER; ++n) {
            const int r = n * RPL + lane / LPR;
            const float f = MX ? mx_scale(vsc[n]) : 1.f;
            if constexpr (NEW) bad |= finite_rows(vx[n].x, t, n);
#pragma unroll
            for (int e = 0; e < EV / 8; ++e)
              reinterpret_cast<uint4*>(vt)[at_value_chunk<D>(r, (lane % LPR) * (EV / 8) + e)] =
                  at_bf16<F, W>(vx[n], e, f);
          }
          __builtin_amdgcn_wave_barrier();
          if (AHEAD && t + KS < ntp) load_values(t + KS);
          mask_scores(s, t, seen);
          float most[QT];
          AtParts<PARTS> w[QT];
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) most[qt] = at_max8(s[qt]);
          at_reference<D, QT>(acc, most, c2);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) {
            const float cq = ref_factor(acc.m[qt], c2);
#pragma unroll
            for (int i = 0; i < 8; i += 2)
              at_weights2<D, QT, PARTS>(acc, qt, i, s[qt], cq, w[qt]);
          }
          at_values<D, QT, PARTS>(acc, vt, w, lane);
          if constexpr (NEW) add_bad(bad, t, w, seen);
          __builtin_amdgcn_wave_barrier();
        }
      } else {
        // The waves convert two tiles at a time together.  Tile after tile a wave multiplies
        // the next one's keys while it turns the current scores into weights, then the
        // current values.  Of a stage (two tiles, 2 t and 2 t + 1) the keys are those of the
        // tiles 2 t + 1 and 2 t + 2: four key tiles and four value tiles in LDS are two in use
        // and two being written for the stage to come; what follows those is on its way to
        // registers.
        static_assert(KS == 1 && Shape::SUB == 2, "a stage is two tiles of all waves");
        constexpr int SUB = Shape::SUB;
        AtRaw<F, W> raw[SUB][PER];
        uint32_t sc[SUB][PER] = {};
        auto load_piece = [&](AtRaw<F, W>(&x)[SUB][PER], uint32_t(&xs)[SUB][PER], int t, int j,
                              int i) {
          const int n = qw + NQ * i;
          const bool key = n < NLT;
          if (n >= 2 * NLT) return;
          const uint32_t r = (t * SUB + j + (key ? 1 : 0)) * kAtTile + (n % NLT) * RPL + lane / LPR;
          x[j][i].template load<!NEW>(key ? kr : vr, r * (key ? kst : vst) + (lane % LPR) * W);
          if constexpr (MX)
            xs[j][i] = __builtin_amdgcn_raw_buffer_load_b8(
                key ? ksr : vsr, (int)(r * (D / 32) + (lane % LPR) * EV / 32), 0, 0);
        };
        auto store_piece = [&](AtRaw<F, W>(&x)[SUB][PER], const uint32_t(&xs)[SUB][PER], int t,
                               int j, int i) {
          uint32_t bad = 0;
          const int n = qw + NQ * i;
          const bool key = n < NLT;
          if (n >= 2 * NLT) return bad;
          const int r = (n % NLT) * RPL + lane / LPR;
          const float f = MX ? mx_scale(xs[j][i]) : 1.f;
          if constexpr (NEW) {
            if (!key) bad = finite_rows(x[j][i].x, t * SUB + j, n - NLT);
          }
          uint4* dst = reinterpret_cast<uint4*>(key ? key_tile(t * SUB + j + 1) : value_tile(t & 1, j));
#pragma unroll
          for (int e = 0; e < EV / 8; ++e) {
            const int ch = (lane % LPR) * (EV / 8) + e;
            dst[key ? at_key_chunk<D>(r, ch) : at_value_chunk<D>(r, ch)] =
                at_bf16<F, W>(x[j][i], e, f);
          }
          return bad;
        };
        auto load = [&](AtRaw<F, W>(&x)[SUB][PER], uint32_t(&xs)[SUB][PER], int t) {
#pragma unroll
          for (int j = 0; j < SUB; ++j)
#pragma unroll
            for (int i = 0; i < PER; ++i) load_piece(x, xs, t, j, i);
        };
        auto store = [&](AtRaw<F, W>(&x)[SUB][PER], const uint32_t(&xs)[SUB][PER], int t) {
#pragma unroll
          for (int j = 0; j < SUB; ++j) {
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) bad |= store_piece(x, xs, t, j, i);
            if (NEW && lane == 0) bad_s[((t & 1) * SUB + j) * NQ + qw] = bad;
          }
        };
        uint4 kf[2][KSTEP];
        auto read_keys = [&](int n) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int ks = 0; ks < KSTEP; ++ks)
              kf[kb][ks] = reinterpret_cast<const uint4*>(
                  key_tile(n))[at_key_chunk<D>(kb * 16 + c, ks * 4 + g)];
        };
        const int its = (ntp + SUB - 1) / SUB;
        {
          AtRaw<F, W> x[SUB][PER];  // (the first keys; nothing else of the stage before the first)
          uint32_t xs[SUB][PER] = {};
#pragma unroll
          for (int i = 0; i < PER; ++i)
            if (qw + NQ * i < NLT) load_piece(x, xs, -1, 1, i);
          load(raw, sc, 0);
          load_queries();
#pragma unroll
          for (int i = 0; i < PER; ++i)
            if (qw + NQ * i < NLT) store_piece(x, xs, -1, 1, i);
          store(raw, sc, 0);
          load(raw, sc, 1);
        }
        __syncthreads();
        at_f32x4 s[QT][2];
        uint32_t seen[QT];
        if (NEW && active) see(0, seen);
        if (active) {
          read_keys(0);
          scores([&](int kb, int ks) { return kf[kb][ks]; }, s);
          mask_scores(s, 0, seen);
          float most[QT];
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) most[qt] = at_max8(s[qt]);
          at_reference<D, QT>(acc, most, c2);
        }
        __syncthreads();  // tile 0's keys are read: the first stage writes tile 4's over them
        for (int t = 0; t < its; ++t) {
          if (active) {
#pragma unroll
            for (int j = 0; j < SUB; ++j) {
              uint32_t bad = 0, seen_next[QT];
              if constexpr (NEW) {
#pragma unroll
                for (int w = 0; w < NQ; ++w) bad |= bad_s[((t & 1) * SUB + j) * NQ + w];
                bad = __builtin_amdgcn_readfirstlane(bad);
              }
              at_f32x4 next[QT][2];
              AtParts<PARTS> w[QT];
              at_bf16x8 vf[3];
#pragma unroll
              for (int qt = 0; qt < QT; ++qt) next[qt][0] = next[qt][1] = (at_f32x4){0.f, 0.f, 0.f, 0.f};
              // The matrix unit takes KSTEP / 2 products while the vector unit turns two scores
              // into weights (the fences keep the compiler from taking them apart).
              read_keys(t * SUB + j + 1);
              if constexpr (NEW) see(t * SUB + j + 1, seen_next);
#pragma unroll
              for (int pr = 0; pr < 4 * QT; ++pr) {
#pragma unroll
                for (int m = pr * KSTEP / 2; m < (pr + 1) * KSTEP / 2; ++m) {
                  const int kb = m / (KSTEP * QT), ks = m / QT % KSTEP, qt = m % QT;
                  next[qt][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                      __builtin_bit_cast(at_bf16x8, kf[kb][ks]),
                      __builtin_bit_cast(at_bf16x8, q[qt][ks]), next[qt][kb], 0, 0, 0);
                }
                const int qt = pr / 4;
                at_weights2<D, QT, PARTS>(acc, qt, 2 * (pr % 4), s[qt],
                                          ref_factor(acc.m[qt], c2), w[qt]);
                // (here, not behind the mask's branch)
                asm volatile("" : "+v"(acc.l[qt]));
#pragma unroll
                for (int k = 0; k < PARTS; ++k) asm volatile("" : "+v"((&w[qt].p[k].x)[pr % 4]));
                if (pr >= 4 * QT - 2)
                  vf[pr - (4 * QT - 2)] = at_value_block<D>(value_tile(t & 1, j), pr - (4 * QT - 2), lane);
                __builtin_amdgcn_sched_barrier(0);
              }
              mask_scores(next, t * SUB + j + 1, seen_next);
              // And the values' products, their operands two blocks ahead, while the wave's
              // share of the tiles to come is converted and the next scores' maxima are found;
              // ahead of the other wave's weights.
              float most[QT];
              __builtin_amdgcn_s_setprio(1);
#pragma unroll
              for (int db = 0; db < D / 16; ++db) {
                if (db + 2 < D / 16)
                  vf[(db + 2) % 3] = at_value_block<D>(value_tile(t & 1, j), db + 2, lane);
                at_value_products<D, QT, PARTS>(acc, db, vf[db % 3], w);
                if constexpr (!NEW) {
#pragma unroll
                  for (int i = 0; i < PER; ++i)
                    if (db == i * (D / 16) / PER) {
                      store_piece(raw, sc, t + 1, j, i);
                      load_piece(raw, sc, t + 2, j, i);
                    }
                }
                if (db >= D / 16 - QT) most[db - (D / 16 - QT)] = at_max8(next[db - (D / 16 - QT)]);
                __builtin_amdgcn_sched_barrier(0);
              }
              __builtin_amdgcn_s_setprio(0);
              if constexpr (NEW) add_bad(bad, t * SUB + j, w, seen);
              at_reference<D, QT>(acc, most, c2);
#pragma unroll
              for (int qt = 0; qt < QT; ++qt) {
                if constexpr (NEW) seen[qt] = seen_next[qt];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) s[qt][kb] = next[qt][kb];
              }
            }
          }
          if (NEW || !active) {
            store(raw, sc, t + 1);
            load(raw, sc, t + 2);
          }
          __syncthreads();
        }
      }

      // The piece's partial: (maximum, sum, unnormalized output) of each query row, the KS
      // groups joined in LDS.
      const int64_t slot = (NEW ? a.ck.most + a.U : 0) + x + u;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        float l_row = acc.l[qt];
        l_row += __shfl_xor(l_row, 16, 64);
        l_row += __shfl_xor(l_row, 32, 64);
        if constexpr (KS == 1) {
          const int row = row0 + qt * 16 + c;
          if (row < M) {
            const int64_t pr = slot * mp + row;
            if (g == 0) a.part_ml[pr] = make_float2(acc.m[qt], l_row);
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
              *reinterpret_cast<float4*>(a.part_o + pr * D + 16 * db + 4 * g) = make_float4(
                  acc.o[qt][db][0], acc.o[qt][db][1], acc.o[qt][db][2], acc.o[qt][db][3]);
          }
        } else {
          constexpr int ROW = Shape::ROW;
          float* join = reinterpret_cast<float*>(lds);
          __syncthreads();  // every wave is done with its tiles (and with the tile before)
          if (g == 0) ml_s[wave * 16 + c] = make_float2(acc.m[qt], l_row);
          __syncthreads();
          float mx = kAtNone;
#pragma unroll
          for (int k = 0; k < KS; ++k) mx = fmaxf(mx, ml_s[(k * NQ + qw) * 16 + c].x);
          const float w = __builtin_amdgcn_exp2f(acc.m[qt] - mx);
#pragma unroll
          for (int db = 0; db < D / 16; ++db) {
            const at_f32x4 o = acc.o[qt][db];
            *reinterpret_cast<float4*>(join + (wave * 16 + c) * ROW + 16 * db + 4 * g) =
                make_float4(o[0] * w, o[1] * w, o[2] * w, o[3] * w);
          }
          __syncthreads();
          for (int i = tid; i < NQ * 16 * (D / 4); i += NT) {
            const int r = i / (D / 4), d4 = i % (D / 4);
            const int row = (qg * NQ + r / 16) * QT * 16 + qt * 16 + r % 16;
            if (row >= M) continue;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              const float4 y = *reinterpret_cast<const float4*>(
                  join + (k * NQ * 16 + r) * ROW + 4 * d4);
              o.x += y.x, o.y += y.y, o.z += y.z, o.w += y.w;
            }
            const int64_t pr = slot * mp + row;
            reinterpret_cast<float4*>(a.part_o + pr * D)[d4] = o;
            if (d4 == 0) {
              float mm = kAtNone, sum = 0.f;
#pragma unroll
              for (int k = 0; k < KS; ++k) mm = fmaxf(mm, ml_s[k * NQ * 16 + r].x);
#pragma unroll
              for (int k = 0; k < KS; ++k) {
                const float2 ml = ml_s[k * NQ * 16 + r];
                sum += ml.y * __builtin_amdgcn_exp2f(ml.x - mm);
              }
              a.part_ml[pr] = make_float2(mm, sum);
            }
          }
        }
      }
      __syncthreads();  // the joined tiles are read before the next piece overwrites them
    }
  }
}

// TREE: with new rows.
template <int F, int D, int SHAPE, bool TREE>
__global__ __launch_bounds__((64 * attend_wg_waves(SHAPE)))
__attribute__((amdgpu_waves_per_eu(attend_waves(D, SHAPE)))) void attend_kernel(
    AttendArgs a) {
  constexpr int NQ = SHAPE <= kAtTwo ? 1 : SHAPE == kAtEight ? 4 : 8;
  constexpr int QT = SHAPE == kAtOne ? 1 : 2;
  using Shape = AtShape<D, NQ, QT>;
  static_assert(Shape::NT == 64 * attend_wg_waves(SHAPE), "the workgroup's waves");
  __shared__ __align__(16) uint16_t lds[Shape::LDS];
  __shared__ float2 ml_s[Shape::KS == 1 ? 1 : Shape::KS * NQ * 16];
  __shared__ uint32_t bad_s[TREE && NQ > 1 ? 2 * Shape::SUB * Shape::KS * NQ : 1];
  attend_rows<F, D, NQ, QT, false>(a, lds, ml_s, bad_s);
  if constexpr (TREE) attend_rows<CERTKV_CACHE_BF16, D, NQ, QT, true>(a, lds, ml_s, bad_s);
}

template <int F, int D, int SHAPE>
static certkv_status launch_attend(const AttendArgs& a, hipStream_t s) {
  const int chunks = a.tn && a.ck.most_new > a.ck.most ? a.ck.most_new : a.ck.most;
  const int wgs = chunks < a.ck.parts ? chunks : a.ck.parts;
  const int grid = a.ck.qgroups == 1 ? wgs : (wgs + 7) / 8 * 8 * a.ck.qgroups;
  constexpr int NT = 64 * attend_wg_waves(SHAPE);
  if constexpr (F != CERTKV_CACHE_BF16) {
    if (a.tn == 0) {
      CERTKV_LAUNCH("attend", (attend_kernel<F, D, SHAPE, false>), dim3(grid), dim3(NT), 0, s, a);
      return CERTKV_OK;
    }
  }
  CERTKV_LAUNCH("attend", (attend_kernel<F, D, SHAPE, true>), dim3(grid), dim3(NT), 0, s, a);
  return CERTKV_OK;
}

template <int F, int D>
static certkv_status launch_attend_d(const AttendArgs& a, hipStream_t s) {
  switch (a.ck.shape) {
    case kAtOne: return launch_attend<F, D, kAtOne>(a, s);
    case kAtTwo: return launch_attend<F, D, kAtTwo>(a, s);
    case kAtEight: return launch_attend<F, D, kAtEight>(a, s);
    default: return launch_attend<F, D, kAtSixteen>(a, s);
  }
}

}  // namespace certkv
