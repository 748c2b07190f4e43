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
//   a running maximum and sum in log2 units, the maximum moved (and the sums
//     rescaled) only when a row's grows by more than 2^8;
//   O^T += V^T P^T on the same instruction: P^T (the B operand) is the lane's own
//     eight weights, as the bf16 of each and the bf16 of the remainder (16 bits of
//     the fp32 weight: one bf16 alone would leave 2^-9), V^T (the A operand) comes from
//     transposing LDS reads of the row-major value tile along the same key order.
// Codes become bf16 values, exactly, on the way from memory to the matrix unit: a
// conversion takes the block's scale as its operand (one instruction for two codes).
//
// A workgroup is NQ waves, each with QT query tiles, times KS groups that take the
// tiles in turn.  Up to 32 query rows (NQ = 1) every wave is a group by itself and
// reads keys straight into MFMA operands; only values pass through its LDS tile, and
// no wave waits for another until the groups are joined at the end.  With more rows the waves of
// a group convert a tile together, each its share, into one of two LDS buffers while
// they work on the other.
#pragma once

#include "mx.h"
#include "stages.h"

namespace certkv {

typedef __bf16 at_bf16x8 __attribute__((__vector_size__(8 * sizeof(__bf16))));
typedef float at_f32x4 __attribute__((__vector_size__(4 * sizeof(float))));
typedef __bf16 at_bf16x2 __attribute__((ext_vector_type(2)));
typedef float at_f32x2 __attribute__((ext_vector_type(2)));
typedef short at_s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) at_s16x4 at_lds_s16x4;

constexpr int kAtTile = 32;
constexpr float kAtLog2e = 1.4426950408889634f;
constexpr float kAtLn2 = 0.6931471805599453f;
constexpr float kAtSlack = 8.f;  // log2 growth of a row maximum absorbed without rescaling

// How the rows of all units are laid out in one order and cut into chunks.  A unit
// takes the tiles of its packed rows and, after them, those of its new rows, from
// a place that follows from its first row alone (a sum over the units before would
// need a pass): at least `gap` further per unit, so that tiles never straddle units
// or formats.  The chunks are of equal length, one for each workgroup that is
// resident at once; a chunk that crosses from one unit to the next is two pieces,
// and a unit's gap also stands for what a piece costs beside its tiles.
__device__ __forceinline__ uint32_t at_up32(uint32_t x) { return (x + 31u) & ~31u; }
struct AtCut {
  uint32_t keys, total;
};
__device__ __forceinline__ AtCut at_cut(const AttendChunks& c, uint32_t rows, int64_t U) {
  AtCut cut;
  cut.total = at_up32(rows) + (uint32_t)U * (uint32_t)c.gap;
  uint32_t k = (cut.total + (uint32_t)c.parts - 1u) / (uint32_t)c.parts;
  k = min(max(k, (uint32_t)kAtMinKeys), (uint32_t)kAtMaxKeys);
  // (more rows than the caller's bound allows for: longer chunks, so that the partials
  // stay within the workspace)
  if (cut.total > (uint64_t)c.most * k) k = (cut.total + (uint32_t)c.most - 1u) / (uint32_t)c.most;
  cut.keys = (k + kAtMinKeys - 1u) / kAtMinKeys * kAtMinKeys;
  return cut;
}

// How a lane holds eight or more consecutive dims of a row in format F.
template <int F, int W>
struct AtRaw;
template <int F>
struct AtRaw<F, 16> {
  uint4 x;
  __device__ __forceinline__ void load(BufRsrc r, uint32_t off) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0);
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
  __device__ __forceinline__ void load(BufRsrc r, uint32_t off) { x = buf_load_u64(r, off); }
  __device__ __forceinline__ uint2 codes8(int s) const {
    return F == CERTKV_CACHE_MXFP8 ? x : make_uint2((&x.x)[s], 0u);
  }
};
template <int F>
struct AtRaw<F, 4> {
  uint32_t x;
  __device__ __forceinline__ void load(BufRsrc r, uint32_t off) { x = buf_load_u32(r, off); }
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

// Two floats to bf16 (round to nearest even), a in the low half.
__device__ __forceinline__ uint32_t at_pack(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((at_f32x2){a, b}, at_bf16x2));
}

// LDS tiles: 32 rows of D bf16 in natural order, 16-byte chunks swizzled within a row.
// Keys are read a chunk per lane, sixteen rows at a time; values by transposing reads,
// eight rows of 32 bytes per half-wave: each spreads over all banks.
template <int D>
__device__ __forceinline__ int at_key_chunk(int r, int c) {
  return r * (D / 8) + (c ^ ((D == 128 ? r : (r >> 1)) & (D / 8 - 1)));
}
template <int D>
__device__ __forceinline__ int at_value_chunk(int r, int c) {
  return r * (D / 8) + (c ^ (2 * ((D == 128 ? r : (r >> 1)) & (D / 16 - 1))));
}

template <int F, int D, int NQ, int QT>
struct AtShape {
  static constexpr int KS = NQ == 1 ? 4 : NQ == 2 ? 2 : 1;
  static constexpr int NT = 64 * NQ * KS;
  static constexpr int TILE = kAtTile * D;            // bf16 elements of an LDS tile
  static constexpr int KT = NQ == 1 ? 0 : 2;          // key tiles of a group in LDS
  static constexpr int VT = NQ == 1 ? 1 : 2;          // value tiles
  static constexpr int ROW = D + 4;                   // floats of a joined output row
  static constexpr int JOIN = KS == 1 ? 0 : 2 * KS * NQ * 16 * ROW;  // bf16 elements
  static constexpr int TILES = KS * (KT + VT) * TILE;
  static constexpr int LDS = TILES > JOIN ? TILES : JOIN;
};

// The state of a wave's query rows.
template <int D, int QT>
struct AtAcc {
  float m[QT], l[QT];
  at_f32x4 o[QT][D / 16];
};

// Running maximum and weights of one query tile's scores s (raw products; c2 > 0 turns
// them into log2 units), and the sums rescaled where a maximum has moved.
template <int D, int QT, bool MASKED>
__device__ __forceinline__ void at_softmax(AtAcc<D, QT>& a, int qt, const at_f32x4 s[2], float c2,
                                           uint4& hi, uint4& lo, float p[8]) {
  float mt = s[0][0];
#pragma unroll
  for (int i = 1; i < 8; ++i) mt = fmaxf(mt, s[i >> 2][i & 3]);
  mt *= c2;
  if (__builtin_amdgcn_ballot_w64(mt > a.m[qt] + kAtSlack) != 0) {
    mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
    mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
    const float mnew = fmaxf(a.m[qt], mt);
    // (a row that has seen nothing yet stays at -inf)
    const float alpha = mnew == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(a.m[qt] - mnew);
    a.m[qt] = mnew;
    a.l[qt] *= alpha;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) a.o[qt][db] *= alpha;
  }
  const float mref = MASKED && a.m[qt] == -INFINITY ? 0.f : a.m[qt];
  uint32_t h[4], r[4];
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    p[i] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], c2, -mref));
    p[i + 1] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][(i + 1) & 3], c2, -mref));
    a.l[qt] += p[i] + p[i + 1];
    h[i >> 1] = at_pack(p[i], p[i + 1]);
    r[i >> 1] = at_pack(p[i] - __uint_as_float(h[i >> 1] << 16),
                        p[i + 1] - __uint_as_float(h[i >> 1] & 0xffff0000u));
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(r[0], r[1], r[2], r[3]);
}

// O^T += V^T P^T over the value tile at vt.
template <int D, int QT>
__device__ __forceinline__ void at_values(AtAcc<D, QT>& a, const uint16_t* vt, const uint4 hi[QT],
                                          const uint4 lo[QT], int lane) {
  const int g = lane >> 4, c = lane & 15;
#pragma unroll
  for (int db = 0; db < D / 16; ++db) {
    // lane c of group g is to hold dim c of the block at keys 4 g + i, 16 + 4 g + i: in a
    // transposing read, lane c addresses key c / 4 of the four at dims 4 (c % 4) .. + 3
    uint2 v[2];
#pragma unroll
    for (int rd = 0; rd < 2; ++rd) {
      const int r = 16 * rd + 4 * g + (c >> 2), dim = 16 * db + 4 * (c & 3);
      const uint16_t* src = vt + at_value_chunk<D>(r, dim >> 3) * 8 + (dim & 7);
      v[rd] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (at_lds_s16x4*)(__attribute__((address_space(3))) uint16_t*)src));
    }
    const at_bf16x8 vf = __builtin_bit_cast(at_bf16x8, make_uint4(v[0].x, v[0].y, v[1].x, v[1].y));
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      a.o[qt][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          vf, __builtin_bit_cast(at_bf16x8, hi[qt]), a.o[qt][db], 0, 0, 0);
      a.o[qt][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          vf, __builtin_bit_cast(at_bf16x8, lo[qt]), a.o[qt][db], 0, 0, 0);
    }
  }
}


// The unit whose place holds row r of the common order (at_cut), by a wave: 64 units'
// ends per step.
__device__ __forceinline__ uint32_t at_place(const int64_t* __restrict__ off, int64_t base,
                                             int64_t u, int32_t gap) {
  return at_up32((uint32_t)(off[u] - base)) + (uint32_t)u * (uint32_t)gap;
}
__device__ __forceinline__ int64_t at_find_unit(const int64_t* __restrict__ off, int64_t base,
                                                int64_t U, int32_t gap, uint32_t r, int lane) {
  int64_t lo = 0, n = U;  // the answer is one of [lo, lo + n]
  while (true) {
    const int64_t step = (n + 63) / 64, i = lo + lane * step + step - 1;
    const bool past = i >= U || at_place(off, base, i + 1, gap) > r;
    lo += (int64_t)__popcll(__ballot(!past)) * step;
    if (step == 1) return lo < U ? lo : U;
    n = step;
  }
}

// Whether a bf16 of the eight is not finite.
__device__ __forceinline__ bool at_bad8(uint4 x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
  return bad;
}

template <int F, int D, int NQ, int QT>
__global__ __launch_bounds__((AtShape<F, D, NQ, QT>::NT)) __attribute__((amdgpu_waves_per_eu(2)))
void attend_kernel(AttendArgs a) {
  using Shape = AtShape<F, D, NQ, QT>;
  constexpr int KS = Shape::KS, NT = Shape::NT, TILE = Shape::TILE;
  constexpr int RB = mx_row_bytes(F, D), BITS = F == CERTKV_CACHE_BF16 ? 16 : F == CERTKV_CACHE_MXFP8 ? 8 : 4;
  constexpr bool MX = F != CERTKV_CACHE_BF16;
  constexpr int KSTEP = D / 32;
  // keys read straight into operands (NQ = 1): lane (g, c) holds WK bytes of row c at a
  // time, EK dims, so that the four groups read 4 WK consecutive bytes
  constexpr int WK = 32 * RB / 128 >= 16 ? 16 : 8, EK = NQ == 1 ? WK * 8 / BITS : 8;
  constexpr int SK = EK / 8, NLK = KSTEP / SK;
  // a row-major tile: W bytes of a lane, the tile in NL pieces of a wave; alone, a wave
  // takes the values, in a group the waves take turns at the keys' and the values' pieces
  constexpr int TB = kAtTile * RB;
  constexpr int W = NQ == 1 || !MX || 2 * TB / (64 * 16) >= NQ ? 16
                    : F == CERTKV_CACHE_MXFP8 || 2 * TB / (64 * 8) >= NQ ? 8 : 4;
  constexpr int EV = W * 8 / BITS, LPR = RB / W, NLT = TB / (64 * W);
  constexpr int PER = NQ == 1 ? NLT : (2 * NLT + NQ - 1) / NQ;
  // and of new rows, bf16 in 16-byte pieces
  constexpr int LPRN = D / 8, NLN = kAtTile * D * 2 / 1024;
  constexpr int PERN = NQ == 1 ? NLN : (2 * NLN + NQ - 1) / NQ;

  __shared__ __align__(16) uint16_t lds[Shape::LDS];
  __shared__ float2 ml_s[KS == 1 ? 1 : KS * NQ * 16];
  __shared__ uint32_t bad_s[NQ == 1 ? 1 : 2 * KS * NQ];

  const Geo& gm = a.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave / NQ, qw = wave % NQ;
  const int g = lane >> 4, c = lane & 15;
  const int M = a.tq * gm.G, mp = a.ck.mp;
  const float c2 = gm.scale * kAtLog2e;
  const int64_t U = a.U;
  const int64_t* __restrict__ off = a.cache.offsets;
  const int32_t gap = a.ck.gap;
  const uint32_t tnp = at_up32((uint32_t)a.tn);

  // Query groups (more rows than a workgroup holds) of a chunk: eight workgroups apart, on
  // the same XCD, whose L2 then serves all but the first.
  const int wgx = blockIdx.x;
  const int qg = (wgx >> 3) % a.ck.qgroups;
  const uint32_t x0 = a.ck.qgroups == 1 ? wgx : (wgx >> 3) / a.ck.qgroups * 8 + (wgx & 7);
  const uint32_t xstep = gridDim.x / a.ck.qgroups;
  const int row0 = (qg * NQ + qw) * QT * 16;
  const bool active = row0 < M;
  auto kdim = [&](int ks) { return (ks / SK) * 4 * EK + g * EK + 8 * (ks % SK); };

  uint16_t* const group_lds = lds + kg * (Shape::KT + Shape::VT) * TILE;
  auto key_tile = [&](int buf) { return group_lds + buf * TILE; };
  auto value_tile = [&](int buf) { return group_lds + (Shape::KT + (NQ == 1 ? 0 : buf)) * TILE; };

  const int64_t base = off[0];
  const AtCut cut = at_cut(a.ck, (uint32_t)(off[U] - base), U);
  const uint32_t nch = (cut.total + cut.keys - 1) / cut.keys;
  for (uint32_t x = x0; x < nch; x += xstep) {
    const uint32_t r0 = x * cut.keys, r1 = min(cut.total, r0 + cut.keys);
    for (int64_t u = at_find_unit(off, base, U, gap, r0, lane); u < U; ++u) {
      const uint32_t vs = at_place(off, base, u, gap);
      if (vs >= r1) break;
      const int64_t p0 = off[u];
      const uint32_t len = (uint32_t)min(off[u + 1] - p0, a.cover), pt = at_up32(len);
      const uint32_t lo = max(r0, vs) - vs, hi = r1 - vs;
      // the piece: packed rows [lo, lo + np), then new rows [n0, n0 + nn)
      const int np = (int)min(hi, len) - (int)lo;
      const uint32_t nlo = max(lo, pt) - pt, nhi = hi > pt ? min(hi - pt, (uint32_t)a.tn) : 0u;
      const int nn = (int)nhi - (int)nlo;
      if (np <= 0 && nn <= 0) continue;  // (only what lies between units)
      const int ntp = np > 0 ? (np + 31) / 32 : 0, ntn = nn > 0 ? (nn + 31) / 32 : 0;
      const int h = (int)(u % gm.H);
      const int64_t lb = u / gm.H;
      const int b = (int)(lb % gm.B);
      const int l = (int)(lb / gm.B);

      // packed rows of the piece (reads past them return zero)
      const uint32_t rows = np > 0 ? np : 0;
      const int64_t at = p0 + lo;
      const BufRsrc kr = make_rsrc(static_cast<const uint8_t*>(a.cache.k) + at * RB, rows * RB);
      const BufRsrc vr = make_rsrc(static_cast<const uint8_t*>(a.cache.v) + at * RB, rows * RB);
      const BufRsrc ksr = make_rsrc(a.cache.k_scales + (MX ? at * (D / 32) : 0), MX ? rows * (D / 32) : 0);
      const BufRsrc vsr = make_rsrc(a.cache.v_scales + (MX ? at * (D / 32) : 0), MX ? rows * (D / 32) : 0);
      // new rows of the unit
      const uint16_t* kn = static_cast<const uint16_t*>(a.k_new.ptr) + l * a.k_new.s_layer +
                           (int64_t)b * a.tn * a.k_new.s_token + h * a.k_new.s_head;
      const uint16_t* vn = static_cast<const uint16_t*>(a.v_new.ptr) + l * a.v_new.s_layer +
                           (int64_t)b * a.tn * a.v_new.s_token + h * a.v_new.s_head;

      AtAcc<D, QT> acc;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        acc.m[qt] = -INFINITY;
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

      // Scores of a tile whose keys' operands are kf(kb, ks), masked to `left` rows, or by
      // the bits seen[qt] (of the lane's eight keys).
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
      auto packed_weights = [&](at_f32x4 s[QT][2], int left, uint4 ph[QT], uint4 pl[QT]) {
        if (left < kAtTile) {
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (16 * (i >> 2) + 4 * g + (i & 3) >= left) s[qt][i >> 2][i & 3] = -INFINITY;
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          float p[8];
          at_softmax<D, QT, false>(acc, qt, s[qt], c2, ph[qt], pl[qt], p);
        }
      };
      // Weights of new rows j0 .. j0 + 31, and their values added; `bad`: rows whose values
      // are not all finite, zero in the tile, which reach only the queries that see them.
      auto new_tile = [&](at_f32x4 s[QT][2], const uint16_t* vt, int j0, uint32_t bad) {
        uint4 ph[QT], pl[QT];
        float p[QT][8];
        uint32_t seen[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const int row = row0 + qt * 16 + c, t = min(row, M - 1) / gm.G;
          const uint8_t* mrow = a.mask + ((int64_t)b * a.tq + t) * a.tn;
          seen[qt] = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int j = j0 + 16 * (i >> 2) + 4 * g + (i & 3);
            bool see = j <= a.tn - a.tq + t;
            if (a.mask) see = mrow[min(j, a.tn - 1)] != 0;
            see = see && j < a.tn && row < M;
            seen[qt] |= (uint32_t)see << i;
            if (!see) s[qt][i >> 2][i & 3] = -INFINITY;
          }
          at_softmax<D, QT, true>(acc, qt, s[qt], c2, ph[qt], pl[qt], p[qt]);
        }
        at_values<D, QT>(acc, vt, ph, pl, lane);
        while (bad) {  // (rare)
          const int r = __builtin_ctz(bad);
          bad &= bad - 1;
          const int i = 4 * (r >> 4) + (r & 3), src = ((r >> 2) & 3) * 16 + c;
          const uint16_t* vrow = vn + (int64_t)min(j0 + r, a.tn - 1) * a.v_new.s_token;
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) {
            float w = p[qt][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) w = i == e ? p[qt][e] : w;
            w = __shfl(w, src, 64);
            const bool see = (__shfl(seen[qt], src, 64) >> i) & 1;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
              const uint2 v = *reinterpret_cast<const uint2*>(vrow + 16 * db + 4 * g);
              const float e[4] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)};
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (see) acc.o[qt][db][k] = fmaf(w, e[k], acc.o[qt][db][k]);
            }
          }
        }
      };

      if constexpr (NQ == 1) {
        uint16_t* const vt = value_tile(0);
        AtRaw<F, WK> kx[2][NLK];
        AtRaw<F, W> vx[PER];
        uint32_t ksc[2] = {}, vsc[PER] = {};
        auto load_keys = [&](int t) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const uint32_t r = t * kAtTile + kb * 16 + c;
#pragma unroll
            for (int i = 0; i < NLK; ++i) kx[kb][i].load(kr, r * RB + g * WK + i * 4 * WK);
            if constexpr (MX) ksc[kb] = D == 128 ? buf_load_u32(ksr, r * 4) : buf_load_u16(ksr, r * 2);
          }
        };
        auto load_values = [&](int t) {
#pragma unroll
          for (int n = 0; n < PER; ++n) {
            const uint32_t r = t * kAtTile + n * (64 / LPR) + lane / LPR;
            vx[n].load(vr, r * RB + (lane % LPR) * W);
            if constexpr (MX)
              vsc[n] = __builtin_amdgcn_raw_buffer_load_b8(
                  vsr, (int)(r * (D / 32) + (lane % LPR) * EV / 32), 0, 0);
          }
        };
        if (kg < ntp) {
          load_keys(kg);
          load_values(kg);
        }
        load_queries();
        for (int t = kg; t < ntp; t += KS) {
          at_f32x4 s[QT][2];
          scores(
              [&](int kb, int ks) {
                const int i = ks / SK;
                float f = 1.f;
                if constexpr (MX) f = mx_scale((ksc[kb] >> (8 * ((i * 4 + g) * EK / 32))) & 255u);
                return at_bf16<F, WK>(kx[kb][i], ks % SK, f);
              },
              s);
          if (t + KS < ntp) load_keys(t + KS);
#pragma unroll
          for (int n = 0; n < PER; ++n) {
            const int r = n * (64 / LPR) + lane / LPR;
            const float f = MX ? mx_scale(vsc[n]) : 1.f;
#pragma unroll
            for (int e = 0; e < EV / 8; ++e)
              reinterpret_cast<uint4*>(vt)[at_value_chunk<D>(r, (lane % LPR) * (EV / 8) + e)] =
                  at_bf16<F, W>(vx[n], e, f);
          }
          __builtin_amdgcn_wave_barrier();
          if (t + KS < ntp) load_values(t + KS);
          uint4 ph[QT], pl[QT];
          packed_weights(s, np - t * kAtTile, ph, pl);
          at_values<D, QT>(acc, vt, ph, pl, lane);
          __builtin_amdgcn_wave_barrier();
        }
        // the new rows go on where the packed ones' turn ended
        for (int t = (kg - ntp % KS + KS) % KS; t < ntn; t += KS) {
          const int j0 = (int)nlo + t * kAtTile;
          uint4 kf[2][KSTEP], vf[NLN];
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const uint16_t* src = kn + (int64_t)min(j0 + kb * 16 + c, a.tn - 1) * a.k_new.s_token;
#pragma unroll
            for (int ks = 0; ks < KSTEP; ++ks)
              kf[kb][ks] = *reinterpret_cast<const uint4*>(src + kdim(ks));
          }
#pragma unroll
          for (int n = 0; n < NLN; ++n) {
            const int r = n * (64 / LPRN) + lane / LPRN;
            vf[n] = *reinterpret_cast<const uint4*>(
                vn + (int64_t)min(j0 + r, a.tn - 1) * a.v_new.s_token + (lane % LPRN) * 8);
          }
          at_f32x4 s[QT][2];
          scores([&](int kb, int ks) { return kf[kb][ks]; }, s);
          uint32_t bad = 0;
#pragma unroll
          for (int n = 0; n < NLN; ++n) {
            const int r = n * (64 / LPRN) + lane / LPRN;
            const uint64_t any = __ballot(j0 + r < a.tn && at_bad8(vf[n]));
            const uint64_t own = any >> (lane / LPRN * LPRN) & ((1ull << LPRN) - 1);
            if (own || j0 + r >= a.tn) vf[n] = make_uint4(0u, 0u, 0u, 0u);
            if (any) {
#pragma unroll
              for (int i = 0; i < 64 / LPRN; ++i)
                if (any >> (i * LPRN) & ((1ull << LPRN) - 1)) bad |= 1u << (n * (64 / LPRN) + i);
            }
            reinterpret_cast<uint4*>(vt)[at_value_chunk<D>(r, lane % LPRN)] = vf[n];
          }
          __builtin_amdgcn_wave_barrier();
          new_tile(s, vt, j0, bad);
          __builtin_amdgcn_wave_barrier();
        }
      } else {
        // A group's waves convert a tile together; while they compute with one pair of LDS
        // tiles, the next tile's share waits in registers or is written to the other.
        auto lds_keys = [&](int buf) {
          return [&, buf](int kb, int ks) {
            return reinterpret_cast<const uint4*>(
                key_tile(buf))[at_key_chunk<D>(kb * 16 + c, ks * 4 + g)];
          };
        };
        {
          AtRaw<F, W> raw[PER];
          uint32_t sc[PER] = {};
          auto load = [&](int t) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
              const int n = qw + NQ * i;
              if (n >= 2 * NLT) continue;
              const uint32_t r = t * kAtTile + (n % NLT) * (64 / LPR) + lane / LPR;
              raw[i].load(n < NLT ? kr : vr, r * RB + (lane % LPR) * W);
              if constexpr (MX)
                sc[i] = __builtin_amdgcn_raw_buffer_load_b8(
                    n < NLT ? ksr : vsr, (int)(r * (D / 32) + (lane % LPR) * EV / 32), 0, 0);
            }
          };
          auto store = [&](int buf) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
              const int n = qw + NQ * i;
              if (n >= 2 * NLT) continue;
              const int r = (n % NLT) * (64 / LPR) + lane / LPR;
              const float f = MX ? mx_scale(sc[i]) : 1.f;
              uint4* dst = reinterpret_cast<uint4*>(n < NLT ? key_tile(buf) : value_tile(buf));
#pragma unroll
              for (int e = 0; e < EV / 8; ++e) {
                const int ch = (lane % LPR) * (EV / 8) + e;
                dst[n < NLT ? at_key_chunk<D>(r, ch) : at_value_chunk<D>(r, ch)] =
                    at_bf16<F, W>(raw[i], e, f);
              }
            }
          };
          const int its = (ntp + KS - 1) / KS;
          if (kg < ntp) load(kg);
          load_queries();
          if (kg < ntp) store(0);
          if (kg + KS < ntp) load(kg + KS);
          __syncthreads();
          for (int it = 0; it < its; ++it) {
            const int t = it * KS + kg;
            if (t + KS < ntp) store((it + 1) & 1);
            if (t + 2 * KS < ntp) load(t + 2 * KS);
            if (active && t < ntp) {
              at_f32x4 s[QT][2];
              scores(lds_keys(it & 1), s);
              uint4 ph[QT], pl[QT];
              packed_weights(s, np - t * kAtTile, ph, pl);
              at_values<D, QT>(acc, value_tile(it & 1), ph, pl, lane);
            }
            __syncthreads();
          }
        }
        if (ntn) {
          uint4 raw[PERN];
          auto load = [&](int t) {
#pragma unroll
            for (int i = 0; i < PERN; ++i) {
              const int n = qw + NQ * i;
              if (n >= 2 * NLN) continue;
              const int r = (int)nlo + t * kAtTile + (n % NLN) * (64 / LPRN) + lane / LPRN;
              raw[i] = *reinterpret_cast<const uint4*>(
                  (n < NLN ? kn : vn) + (lane % LPRN) * 8 +
                  (int64_t)min(r, a.tn - 1) * (n < NLN ? a.k_new.s_token : a.v_new.s_token));
            }
          };
          auto store = [&](int t, int buf) {
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < PERN; ++i) {
              const int n = qw + NQ * i;
              if (n >= 2 * NLN) continue;
              const int r = (n % NLN) * (64 / LPRN) + lane / LPRN, ch = lane % LPRN;
              if (n < NLN) {
                reinterpret_cast<uint4*>(key_tile(buf))[at_key_chunk<D>(r, ch)] = raw[i];
                continue;
              }
              const bool past = (int)nlo + t * kAtTile + r >= a.tn;
              const uint64_t any = __ballot(!past && at_bad8(raw[i]));
              const uint64_t own = any >> (lane / LPRN * LPRN) & ((1ull << LPRN) - 1);
              if (own || past) raw[i] = make_uint4(0u, 0u, 0u, 0u);
              if (any) {
#pragma unroll
                for (int k = 0; k < 64 / LPRN; ++k)
                  if (any >> (k * LPRN) & ((1ull << LPRN) - 1))
                    bad |= 1u << ((n - NLN) * (64 / LPRN) + k);
              }
              reinterpret_cast<uint4*>(value_tile(buf))[at_value_chunk<D>(r, ch)] = raw[i];
            }
            if (lane == 0) bad_s[(buf * KS + kg) * NQ + qw] = bad;
          };
          const int its = (ntn + KS - 1) / KS;
          if (kg < ntn) load(kg);
          if (ntp == 0) load_queries();
          if (kg < ntn) store(kg, 0);
          if (kg + KS < ntn) load(kg + KS);
          __syncthreads();
          for (int it = 0; it < its; ++it) {
            const int t = it * KS + kg;
            if (t + KS < ntn) store(t + KS, (it + 1) & 1);
            if (t + 2 * KS < ntn) load(t + 2 * KS);
            if (active && t < ntn) {
              uint32_t bad = 0;
#pragma unroll
              for (int w = 0; w < NQ; ++w) bad |= bad_s[((it & 1) * KS + kg) * NQ + w];
              bad = __builtin_amdgcn_readfirstlane(bad);
              at_f32x4 s[QT][2];
              scores(lds_keys(it & 1), s);
              new_tile(s, value_tile(it & 1), (int)nlo + t * kAtTile, bad);
            }
            __syncthreads();
          }
        }
      }

      // The piece's partial: (maximum, sum, unnormalized output) of each query row, the KS
      // groups joined in LDS.
      const int64_t slot = (int64_t)x + u;
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
          float mx = -INFINITY;
#pragma unroll
          for (int k = 0; k < KS; ++k) mx = fmaxf(mx, ml_s[(k * NQ + qw) * 16 + c].x);
          const float w = acc.m[qt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(acc.m[qt] - mx);
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
              float mm = -INFINITY, sum = 0.f;
#pragma unroll
              for (int k = 0; k < KS; ++k) mm = fmaxf(mm, ml_s[k * NQ * 16 + r].x);
#pragma unroll
              for (int k = 0; k < KS; ++k) {
                const float2 ml = ml_s[k * NQ * 16 + r];
                if (ml.x != -INFINITY || ml.y != 0.f) sum += ml.y * __builtin_amdgcn_exp2f(ml.x - mm);
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

template <int F, int D, int NQ, int QT>
static certkv_status launch_attend(const AttendArgs& a, hipStream_t s) {
  const int wgs = a.ck.most < a.ck.parts ? a.ck.most : a.ck.parts;
  const int grid = a.ck.qgroups == 1 ? wgs : (wgs + 7) / 8 * 8 * a.ck.qgroups;
  CERTKV_LAUNCH("attend", (attend_kernel<F, D, NQ, QT>), dim3(grid),
                dim3(AtShape<F, D, NQ, QT>::NT), 0, s, a);
  return CERTKV_OK;
}

template <int F, int D>
static certkv_status launch_attend_d(const AttendArgs& a, hipStream_t s) {
  switch (a.ck.shape) {
    case kAtOne: return launch_attend<F, D, 1, 1>(a, s);
    case kAtTwo: return launch_attend<F, D, 1, 2>(a, s);
    case kAtFour: return launch_attend<F, D, 2, 2>(a, s);
    case kAtEight: return launch_attend<F, D, 4, 2>(a, s);
    default: return launch_attend<F, D, 8, 2>(a, s);
  }
}

}  // namespace certkv
