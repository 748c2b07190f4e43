// Attention of new queries over a paged cache: the kernel.
//
// For query row (t, head h G + g) of sequence b, whose unit's list holds len rows, n of the tq
// queries being the sequence's own:
//   z_j = scale <q, k_j> for j <= len - n + t (t < n; none for t >= n),
//   out = sum_j softmax(z)_j v_j,  lse = log sum_j e^z_j,
// with out = 0 and lse = -inf where no row is visible.
//
// Tiles of 32 rows, products and weights are those of attend.h: S^T = K Q^T and O^T += V^T P^T on
// v_mfma_f32_16x16x32_bf16, weights in three bf16 parts against a reference that moves only on
// overflow.  A workgroup has 16 or 32 query rows; every wave takes tiles by itself, keys straight
// into operands, values through its own LDS tile, and the waves of a unit are joined at a piece's
// end.
//
// A page is a power of two of 16 rows or more, so that the 16 rows of half a tile are consecutive
// rows of one page, and their place is scalar arithmetic.  Rows of that page behind the list's
// last are read with them: their scores are replaced and their values zero, whatever they hold.
// The table's entries of 32 tiles of a wave are one load, half a tile's to each lane.
//
// Bounds (calls, the join of partials included): one token, the reads (32 layers, 3.36M rows of 128
// dims, bf16: 1.72 GB in 267 us, 6.4 TB/s; 64 ragged sequences, 1.23 GB in 204, 6.0; 8 sequences
// over 16 layers of mxfp8, 2.1 GB in 335, 6.2), but for mxfp4, the issue of its conversions and of
// weights in three parts (3.36M rows, 457 MB in 92 us, 5.0 TB/s); short lists, latency (9 us);
// drafts, issue with little of matrix and vector instructions under each other (48 query rows over
// 378k rows of mxfp4: 48 us; over 3.0M rows 236, the vector unit 43 % busy, the matrix unit 25 %: two
// groups of 32 query rows each convert every tile).
// Tiles two ahead in registers instead of one are no faster (64 dims: 1 to 8 % slower).
#pragma once

#include <type_traits>

#include "attend.h"
#include "pages.h"
#include "places.h"

namespace certkv {

// Tiles between lists' places beside their rows': what a piece costs beside its tiles.  (48 query
// rows over 256 uneven units, 8: 53 us, 16: 46, 24: 46, 32: 48, 48: 54; one token over 1024 units,
// 4: 336 us, 8: 332, 16: 457.)
constexpr int pg_gap(int qt) { return qt == 2 ? 16 : 8; }
static_assert(kPgMaxTiles == kAtMaxKeys / kAtTile, "the longest chunk is the packed cache's");

// What a workgroup has: a piece of a unit, whose tiles its waves take in turn; whole units; or the
// same piece of four heads' units, a head for each wave.
enum { kPgPiece, kPgWhole, kPgHeads };
constexpr int pg_waves(int mode) { return mode == kPgWhole ? 8 : 4; }

// Waves per SIMD that a kernel leaves registers for, which is also how many are launched.  (128
// dims, 16 query rows, two waves and three: mxfp4 93 and 86 us, mxfp8 146 and 171, bf16 266 and 376:
// they spill.)
constexpr int pg_simd_waves(int format, int D, int qt) {
  return qt == 1 && (D == 64 || format == CERTKV_CACHE_MXFP4) ? 3 : 2;
}
// A workgroup has whole units where they are short and not many: no partials, no second launch.
// (In us, whole and in pieces: 8 units of 1024 rows of 128 dims, bf16, 17 and 15, 128 of them 19
// and 23, 512 48 and 54, 2048 194 and 181; 32 units of 100 rows 9 and 15, 2048 53 and 31; of 64
// dims 16 units of 1024 rows 10 and 14, 1024 46 and 53.  The 2 us that few long units of 128 dims
// lose have no rule of their own.)
constexpr int kPgWholeRows = 1024, kPgWholeUnits = 1024;
// Four heads' units where the heads of a row lie together: their rows share lines, which they then
// read at the same time.  (64 ragged sequences, 2.4M rows of 128 dims, a head's rows by itself and
// with three others: bf16 218 and 200 us, mxfp8 136 and 118, mxfp4 124 and 86, 4.8M rows of 64
// dims of mxfp4 237 and 147; with the heads apart in a page, bf16, 202 and 206.)
// units: by query group; s_row, s_head: the pool's strides.
inline int pg_mode(int per_head, int H, int D, int64_t units, int64_t s_row, int64_t s_head,
                   int64_t cover) {
  if (cover <= kPgWholeRows && units * (D / 64) <= kPgWholeUnits) return kPgWhole;
  return !per_head && H % 4 == 0 && s_head < s_row ? kPgHeads : kPgPiece;
}

struct PagedArgs {
  PageArgs p;
  int32_t tq;
  int32_t copies;               // units of a list: L H of a sequence's, 1 of a head's; a quarter
                                // of them where a workgroup has four heads
  int32_t cover;                // rows of a list that are attended
  int32_t qgroups, mp;          // workgroups of a chunk, query rows of a partial
  int32_t mode, gap;
  int32_t parts, most;          // chunks taken at once, and that the workspace has room for
  const int32_t* q_lens;        // [B], or NULL: tq
  uint32_t* place;              // [lists + 1]: the lists' places by their queries' groups, or NULL
  certkv_tensor q;
  float* part_o;                // [most + lists copies][mp][d], or four times as many for four heads
  float2* part_ml;
  float* out;
  float* lse;
};
certkv_status run_paged(const PagedArgs& a, int shape, hipStream_t s);
certkv_status run_paged_bf16(const PagedArgs& a, int shape, hipStream_t s);   // by format
certkv_status run_paged_mxfp8(const PagedArgs& a, int shape, hipStream_t s);
certkv_status run_paged_mxfp4(const PagedArgs& a, int shape, hipStream_t s);

// The chunks of a call whose lists have `tiles` tiles, for one copy.
__device__ __forceinline__ PgCut pg_cut(const PagedArgs& a, uint32_t tiles) {
  return pg_cut((uint32_t)a.copies, tiles, (uint32_t)a.parts, (uint32_t)a.most);
}

// Where sequences have queries of their own number, and more than a workgroup holds, the groups of
// 32 that they have differ, and so does what a list costs: its groups then stand one after another
// in the order, as copies do, and the places are a scan over the lists.
constexpr int kPgWeighed = 2048;  // lists at most
__device__ __forceinline__ int pg_list_sequence(const PagedArgs& a, uint32_t r) {
  return (int)(a.p.per_head ? r / (uint32_t)a.p.g.H % (uint32_t)a.p.g.B : r);
}
__device__ __forceinline__ int pg_own(const PagedArgs& a, int n) { return min(max(n, 0), a.tq); }
__device__ __forceinline__ int pg_queries(const PagedArgs& a, int b) {
  return a.q_lens ? pg_own(a, a.q_lens[b]) : a.tq;
}
__device__ __forceinline__ uint32_t pg_groups(const PagedArgs& a, int own) {
  return (uint32_t)(own * a.p.g.G + 31) >> 5;
}
// place_s[r]: the first tile of list r, for copies = 1; and, from the first workgroup, a.place.
// (Sums stop at kPgMostTiles.)
template <int NT>
__device__ __forceinline__ void pg_weigh(const PagedArgs& a, uint32_t* place_s, uint32_t* sum_s) {
  const int tid = threadIdx.x;
  const int64_t* off = a.p.offsets;
  const int64_t base = off[0], rows = off[a.p.lists] - base;
  uint32_t before = 0;
  for (int r0 = 0; r0 < a.p.lists; r0 += NT) {
    const int r = r0 + tid;
    uint32_t x = 0;
    if (r < a.p.lists) {
      const uint32_t tiles = pg_list_tiles(off[r] - base, off[r + 1] - base, rows);
      const uint64_t n = (uint64_t)pg_groups(a, pg_queries(a, pg_list_sequence(a, r))) * (tiles + a.gap);
      x = (uint32_t)min(n, kPgMostTiles);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t y = __shfl_up(x, d, 64);
      if ((tid & 63) >= d) x = pg_add(x, y);
    }
    if ((tid & 63) == 63) sum_s[tid >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < tid >> 6) x = pg_add(x, sum_s[w]);
    }
    x = pg_add(x, before);
    for (int w = 0; w < NT / 64; ++w) before = pg_add(before, sum_s[w]);
    if (r < a.p.lists) {
      place_s[r + 1] = x;
      if (blockIdx.x == 0) a.place[r + 1] = x;
    }
    __syncthreads();
  }
  if (tid == 0) {
    place_s[0] = 0;
    if (blockIdx.x == 0) a.place[0] = 0;
  }
  __syncthreads();
}

// The lists' offsets, as a wave reads them: those of 64 lists at a time in its lanes.
struct PgOffsets {
  const int64_t* __restrict__ off;
  uint32_t R, at;
  int64_t base, rows, first, end;
  __device__ __forceinline__ PgOffsets(const int64_t* o, int32_t lists, int lane)
      : off(o), R((uint32_t)lists), at(0), base(0), rows(0), first(0), end(0) {
    if (lists == 0) return;  // (not asked for)
    window(0, lane);
    base = AtOffsets::lane64(first, 0);
    rows = (lists <= 64 ? AtOffsets::lane64(end, R - 1) : off[R]) - base;
  }
  __device__ __forceinline__ void window(uint32_t r, int lane) {
    at = r;
    first = off[min(r + lane, R)];
    end = off[min(r + lane + 1, R)];
  }
  // a list's first row and the one behind its last
  __device__ __forceinline__ void list(uint32_t r, int lane, int64_t& p0, int64_t& p1) {
    if (r - at >= 64) window(r, lane);
    p0 = AtOffsets::lane64(first, r - at) - base;
    p1 = AtOffsets::lane64(end, r - at) - base;
  }
  // The list whose place holds tile x (of one copy): 64 lists' ends per step.
  __device__ __forceinline__ uint32_t find(uint32_t x, int gap, int lane) {
    uint32_t lo = 0, n = R;  // the answer is one of [lo, lo + n]
    while (n > 64) {
      const uint32_t step = (n + 63) / 64, i = lo + lane * step + step - 1;
      const bool past = i >= R || pg_place(off[min(i + 1, R)] - base, i + 1, gap) > x;
      lo += (uint32_t)__popcll(__ballot(!past)) * step;
      n = step;
    }
    if (lo != at) window(lo, lane);
    const uint32_t i = lo + lane;
    const uint64_t past = __ballot(i >= R || pg_place(end - base, i + 1, gap) > x);
    return past ? min(lo + (uint32_t)__builtin_ctzll(past), R) : R;
  }
};

// Four dims of query row `row` of a unit: its unnormalized output o, sum L against reference m.
__device__ __forceinline__ void pg_output(const PagedArgs& a, int l, int b, int h, int row, int d4,
                                          int D, float4 o, float m, float L) {
  const Geo& g = a.p.g;
  const int t = row / g.G, gq = row % g.G;
  const int64_t orow = ((int64_t)l * g.B * a.tq + (int64_t)b * a.tq + t) * (g.H * g.G) + h * g.G + gq;
  const float inv = L == 0.f ? 0.f : 1.f / L;  // (nothing visible: out 0, lse -inf)
  const float y[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
  bool fine = true;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    fine = fine && isfinite(y[i]);
    a.out[orow * D + 4 * d4 + i] = y[i];
  }
  if (!fine) report_nonfinite(g);
  if (a.lse && d4 == 0)
    a.lse[orow] = L == 0.f ? -INFINITY
                           : (ref_log2(m, g.scale * kAtLog2e) + __builtin_amdgcn_logf(L)) * kAtLn2;
}

// A lane's part of a row, from a place that is the wave's.  NT: non-temporally.
template <bool NT, typename T>
__device__ __forceinline__ void pg_load(T& x, const uint8_t* at, uint32_t off) {
  typedef uint32_t V __attribute__((ext_vector_type(sizeof(T) / 4)));
  const V* src = reinterpret_cast<const V*>(at + off);
  x = __builtin_bit_cast(T, NT ? __builtin_nontemporal_load(src) : *src);
}
// Two bf16, those that are not finite as zero.
__device__ __forceinline__ uint32_t pg_finite(uint32_t x) {
  if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
  if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
  return x;
}

template <int F, int D, int QT, int MODE>
__global__ __launch_bounds__(64 * pg_waves(MODE))
__attribute__((amdgpu_waves_per_eu(MODE == kPgWhole ? 2 : pg_simd_waves(F, D, QT)))) void paged_kernel(PagedArgs a) {
  constexpr bool WHOLE = MODE == kPgWhole, HEADS = MODE == kPgHeads;
  constexpr int KW = pg_waves(MODE), NT = 64 * KW, PARTS = AtShape<D, 1, QT>::PARTS;
  constexpr int KS = HEADS ? 1 : KW;  // waves that take a unit's tiles in turn
  constexpr int ROW = D + 4;  // floats of a joined output row
  constexpr int JOIN = KS > 1 ? 2 * KS * 16 * ROW : 0, TILES = KW * AtTile<D>::V;  // bf16 elements
  constexpr int BITS = F == CERTKV_CACHE_BF16 ? 16 : F == CERTKV_CACHE_MXFP8 ? 8 : 4;
  constexpr bool MX = F != CERTKV_CACHE_BF16;
  constexpr int RB = mx_row_bytes(F, D);
  constexpr int KSTEP = D / 32;
  // keys: lane (g, c) holds WK bytes of row c at a time, EK dims
  constexpr int WK = RB >= 64 ? 16 : 8, EK = WK * 8 / BITS, SK = EK / 8, NLK = KSTEP / SK;
  // values: W bytes of a lane, so that a load is at most 16 rows; a tile is NLT loads
  constexpr int W = RB >= 64 ? 16 : 8, EV = W * 8 / BITS, LPR = RB / W, RPL = 64 / LPR;
  constexpr int NLT = kAtTile / RPL;
  static_assert(RPL <= 16 && SK * NLK == KSTEP, "a load's rows are in one half");
  __shared__ __align__(16) uint16_t lds[TILES > JOIN ? TILES : JOIN];
  __shared__ float2 ml_s[KS > 1 ? KS * 16 : 1];

  const PageArgs& p = a.p;
  const Geo& gm = p.g;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int M = a.tq * gm.G, mp = a.mp;
  const float c2 = gm.scale * kAtLog2e;
  const uint32_t copies = (uint32_t)a.copies;
  // Query groups of a chunk: eight workgroups apart, on the same XCD, whose L2 then serves all
  // but the first; or, where they are weighed, in the order of the units.
  const bool weighed = QT == 2 && !WHOLE && a.place;
  const int groups = weighed ? 1 : a.qgroups, wgx = blockIdx.x;
  int qg = (wgx >> 3) % groups;
  const uint32_t x0 = groups == 1 ? wgx : (wgx >> 3) / groups * 8 + (wgx & 7);
  const uint32_t xstep = gridDim.x / groups;
  constexpr int PLACES = QT == 2 && !WHOLE ? kPgWeighed + 1 : 1;
  __shared__ uint32_t place_s[PLACES], sum_s[KW];
  if constexpr (PLACES > 1) {
    if (weighed) pg_weigh<NT>(a, place_s, sum_s);
  }
  uint16_t* const vt = lds + wave * AtTile<D>::V;
  // The units' pieces: of the chunks that the workgroup takes, or the whole units.
  PgOffsets off(p.offsets, WHOLE ? 0 : p.lists, lane);
  const PgCut cut = WHOLE ? PgCut{1, 0, true}
                          : pg_cut(a, weighed ? place_s[PLACES > 1 ? p.lists : 0] : pg_tiles(off.rows, off.R, pg_gap(QT)));
  const uint32_t nch = WHOLE ? (uint32_t)p.lists * copies : (cut.total + cut.tiles - 1) / cut.tiles;
  for (uint32_t x = x0; x < nch; x = WHOLE ? nch : x + xstep) {
    const uint32_t r0 = x * cut.tiles, r1 = min(cut.total, r0 + cut.tiles);
    uint32_t r = 0, copy = 0;
    if constexpr (WHOLE) {
      r = x / copies, copy = x - r * copies;
    } else if (weighed) {
      for (uint32_t lo = 0, hi = (uint32_t)p.lists - 1; lo < hi;) {  // the last that begins here or before
        const uint32_t mid = (lo + hi + 1) >> 1;
        if (place_s[PLACES > 1 ? mid : 0] <= r0 / copies)
          lo = mid;
        else
          hi = mid - 1;
        r = lo;
      }
      r = __builtin_amdgcn_readfirstlane(r);
    } else {
      r = off.find(r0 / copies, pg_gap(QT), lane);
    }
    bool begun = false;
    while (WHOLE ? !begun : r < off.R) {
      int64_t p0, p1;
      uint32_t u = x, lo = 0, mine = copy;
      int len, ntp;
      if constexpr (WHOLE) {
        begun = true;
        p0 = p.offsets[r], p1 = p.offsets[r + 1];
        len = min(page_rows(p, p0, p1), a.cover);
        ntp = (int)pg_up(len);
      } else {
        off.list(r, lane, p0, p1);
        if (!pg_held(p0, p1, off.rows)) {
          ++r, copy = 0;
          continue;
        }
        uint32_t place = copies * pg_place(p0, r, pg_gap(QT)), times = 1;
        const uint32_t span = pg_place(p1, r + 1, pg_gap(QT)) - pg_place(p0, r, pg_gap(QT));
        if (weighed) {
          place = copies * place_s[PLACES > 1 ? r : 0];
          times = pg_groups(a, pg_queries(a, pg_list_sequence(a, r)));
        }
        if (!begun) copy = r0 > place ? (r0 - place) / span : 0;
        begun = true;
        if (copy >= copies * times) {
          ++r, copy = 0;
          continue;
        }
        const uint32_t vs = place + copy * span;
        if (vs >= r1) break;
        // the piece: tiles [lo, lo + ntp) of the unit's
        len = min(page_rows(p, p0, p1), a.cover);
        lo = max(r0, vs) - vs;
        ntp = (int)min(r1 - vs, pg_up(len)) - (int)lo;
        mine = copy++;
        if (weighed) qg = (int)(mine % times), mine /= times;
        u = r * copies + mine;
        if (ntp <= 0) continue;  // (only what lies between units)
      }
      // (What follows from the lane is worked out for each piece: kept beyond it, it would take
      // registers from the loads in flight.)
      int lane = tid & 63;
      if constexpr (!WHOLE) asm volatile("" : "+v"(lane));
      const int g = lane >> 4, c = lane & 15;
      auto kdim = [&](int ks) { return (ks / SK) * 4 * EK + g * EK + 8 * (ks % SK); };
      // bytes from row to row and from page to page, and a lane's share of a load
      const uint32_t st = (uint32_t)p.s_row * RB;
      const uint64_t page_bytes = (uint64_t)p.s_page * RB;
      const uint32_t k_off = c * st + g * WK, v_off = (lane / LPR) * st + (lane % LPR) * W;
      const uint32_t ks_off = c * (uint32_t)p.s_row * (D / 32);
      const uint32_t vs_off = (lane / LPR) * (uint32_t)p.s_row * (D / 32) + (lane % LPR) * EV / 32;
      int l, b, h;
      if (p.per_head) {
        h = (int)(r % (uint32_t)gm.H), b = (int)(r / gm.H % (uint32_t)gm.B);
        l = (int)(r / gm.H / gm.B);
      } else {
        if constexpr (HEADS) mine = mine * 4 + wave;
        b = (int)r, l = (int)(mine / (uint32_t)gm.H), h = (int)(mine % (uint32_t)gm.H);
      }
      const int row0 = qg * QT * 16;  // the first query row
      // (Query rows that are not there are another's: nothing is kept of them.)
      uint4 q[QT][KSTEP];
      auto load_queries = [&]() {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const int rc = min(row0 + qt * 16 + c, M - 1);
          const uint16_t* src = static_cast<const uint16_t*>(a.q.ptr) + l * a.q.s_layer +
                                (int64_t)(b * a.tq + rc / gm.G) * a.q.s_token +
                                (int64_t)(h * gm.G + rc % gm.G) * a.q.s_head;
#pragma unroll
          for (int ks = 0; ks < KSTEP; ++ks) q[qt][ks] = *reinterpret_cast<const uint4*>(src + kdim(ks));
        }
      };
      // A whole unit's queries and first pages are asked for before its length is known: latency.
      int32_t first_ids = 0;
      if constexpr (WHOLE) {
        const int pi = ((wave + KS * (lane >> 1)) * kAtTile + (lane & 1) * 16) >> p.lp;
        first_ids = p.table[(int64_t)r * p.max_pages + min(pi, p.max_pages - 1)];
        load_queries();
      }
      const int own = pg_queries(a, b);
      const int64_t at0 = p.per_head ? 0 : l * p.s_layer + h * p.s_head;
      const uint8_t* const kp = p.k + at0 * RB;
      const uint8_t* const vp = p.v + at0 * RB;
      const uint8_t* const ksp = p.k_scales + (MX ? at0 * (D / 32) : 0);
      const uint8_t* const vsp = p.v_scales + (MX ? at0 * (D / 32) : 0);
      // the last row that a lane's queries see, and the first of these
      int last[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const int row = row0 + qt * 16 + c, t = min(row, M - 1) / gm.G;
        last[qt] = row < M && t < own ? len - own + t : -1;
      }
      const int t0 = row0 / gm.G;  // the first token; rows up to `whole` are seen by all
      const int whole = len - own + t0;

      // The wave's tiles are lo + turn + KS n.  Their pages, 32 at a time: half i % 2 of the one of
      // n = i / 2 in lane i.
      const int turn = HEADS ? 0 : wave;
      int32_t ids = 0, window = -1;
      auto pages = [&](int n) {
        if ((n >> 5) == window) return;
        window = n >> 5;
        // (of tiles behind the last, where 31 bits may not do)
        const uint32_t row = (lo + turn + KS * ((n & ~31) + (lane >> 1))) * kAtTile + (lane & 1) * 16;
        ids = -1;
        if (row < (uint32_t)len) {
          const int32_t id = WHOLE && n == 0 ? first_ids : p.table[(int64_t)r * p.max_pages + (row >> p.lp)];
          if ((uint32_t)id < (uint32_t)p.num_pages)
            ids = id;
          else
            report_range(gm);  // (the caller's numbers)
        }
      };
      // rows of half kb of the wave's tile n that are there, and their first byte behind kp and vp
      auto half = [&](int n, int kb, int& there) {
        const int row = (int)(lo + turn + KS * n) * kAtTile + kb * 16;
        const int32_t id = __builtin_amdgcn_readlane(ids, 2 * (n & 31) + kb);
        there = id < 0 ? 0 : min(max(len - row, 0), 16);
        return (uint32_t)max(id, 0) * page_bytes + (uint32_t)(row & ((1 << p.lp) - 1)) * (uint64_t)st;
      };

      AtAcc<D, QT> acc;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        acc.m[qt] = kAtNone;
        acc.l[qt] = 0.f;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) acc.o[qt][db] = (at_f32x4){0.f, 0.f, 0.f, 0.f};
      }
      AtRaw<F, WK> kx[2][NLK];
      AtRaw<F, W> vx[NLT];
      uint32_t ksc[2] = {}, vsc[NLT] = {};
      int kthere[2] = {};
      // Values are read non-temporally, but for rows of less than a line that four heads share.
      // (32 layers of bf16 265 us, without 295; 64 sequences, four heads, bf16 200 and 219, mxfp8
      // 117 and 127, mxfp4 94 and 87, of 64 dims 148 and 126; keys too: as without or slower.)
      constexpr bool VNT = !HEADS || RB >= 128;
      // (rows that are not there are read as well, of the same page: their scores are replaced and
      // their values zero)
      auto load_keys = [&](int n) {
        pages(n);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const uint64_t at = half(n, kb, kthere[kb]);
#pragma unroll
          for (int i = 0; i < NLK; ++i) pg_load<false>(kx[kb][i].x, kp + at + i * 4 * WK, k_off);
          if constexpr (MX) {
            const uint8_t* sp = ksp + at / (RB / (D / 32));
            if constexpr (D == 128)
              ksc[kb] = *reinterpret_cast<const uint32_t*>(sp + ks_off);
            else
              ksc[kb] = *reinterpret_cast<const uint16_t*>(sp + ks_off);
          }
        }
      };
      auto load_values = [&](int n) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          int there;
          const uint64_t at = half(n, kb, there);
#pragma unroll
          for (int i = 0; i < NLT / 2; ++i) {
            const uint64_t ati = at + (uint32_t)(i * RPL) * (uint64_t)st;
            pg_load<VNT>(vx[kb * (NLT / 2) + i].x, vp + ati, v_off);
            if constexpr (MX) vsc[kb * (NLT / 2) + i] = vsp[ati / (RB / (D / 32)) + vs_off];
          }
        }
      };
      const int own_tiles = t0 < own ? (ntp - turn + KS - 1) / KS : 0;  // of the wave
      if (own_tiles > 0) {
        load_keys(0);
        load_values(0);
      }
      if constexpr (!WHOLE) load_queries();
      // One tile, whose keys and values have been asked for; TAIL: some row of it may not be seen by
      // some query.  (Apart, so that what the few last tiles need takes no registers from the
      // others' loads in flight.)
      auto tile = [&](int n, auto tail_c) {
        constexpr bool TAIL = decltype(tail_c)::value;
        const int trow = (int)(lo + turn + KS * n) * kAtTile;
        // (its addresses by itself too)
        int ln = lane;
        if constexpr (TAIL) asm volatile("" : "+v"(ln));
        const int g = ln >> 4;
        at_f32x4 s[QT][2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) s[qt][kb] = (at_f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KSTEP; ++ks) {
            const int i = ks / SK;
            float f = 1.f;
            if constexpr (MX) f = mx_scale((ksc[kb] >> (8 * ((i * 4 + g) * EK / 32))) & 255u);
            const at_bf16x8 k = __builtin_bit_cast(at_bf16x8, at_bf16<F, WK>(kx[kb][i], ks % SK, f));
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
              s[qt][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  k, __builtin_bit_cast(at_bf16x8, q[qt][ks]), s[qt][kb], 0, 0, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        const int there[2] = {kthere[0], kthere[1]};
        if (!TAIL && n + 1 < own_tiles) load_keys(n + 1);
        // (of a tile of drafted tokens' rows: values that are not finite)
        const bool guard = TAIL && a.tq > 1;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < NLT; ++i) {
          const int rr = i * RPL + ln / LPR;
          const float f = MX ? mx_scale(vsc[i]) : 1.f;
#pragma unroll
          for (int e = 0; e < EV / 8; ++e) {
            uint4 v = at_bf16<F, W>(vx[i], e, f);
            if (guard) {
              bad |= at_bad8(v) && rr % 16 < there[rr / 16];
              v = make_uint4(pg_finite(v.x), pg_finite(v.y), pg_finite(v.z), pg_finite(v.w));
            }
            reinterpret_cast<uint4*>(vt)[at_value_chunk<D>(rr, (ln % LPR) * (EV / 8) + e)] = v;
          }
        }
        __builtin_amdgcn_wave_barrier();
        if (!TAIL && n + 1 < own_tiles) load_values(n + 1);
        if (TAIL || there[0] < 16 || there[1] < 16) {
          for (int rr = ln / (D / 8); rr < kAtTile; rr += 64 / (D / 8))
            if (rr % 16 >= there[rr / 16])
              reinterpret_cast<uint4*>(vt)[at_value_chunk<D>(rr, ln % (D / 8))] = make_uint4(0u, 0u, 0u, 0u);
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int j = 4 * g + (i & 3);
              if (j >= there[i >> 2] || (TAIL && trow + 16 * (i >> 2) + j > last[qt]))
                s[qt][i >> 2][i & 3] = -INFINITY;
            }
        }
        float most[QT];
        AtParts<PARTS> w[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) most[qt] = at_max8(s[qt]);
        at_reference<D, QT>(acc, most, c2);
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const float cq = ref_factor(acc.m[qt], c2);
#pragma unroll
          for (int i = 0; i < 8; i += 2) at_weights2<D, QT, PARTS>(acc, qt, i, s[qt], cq, w[qt]);
        }
        at_values<D, QT, PARTS>(acc, vt, w, ln);
        if (guard && __ballot(bad)) {
          // A row that a query does not see has no part in its output, whatever it holds: what is
          // not finite was left out above, and is added for the queries that see it, row by row.
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int i = 0; i < NLT; ++i) {
            const float f = MX ? mx_scale(vsc[i]) : 1.f;
#pragma unroll
            for (int e = 0; e < EV / 8; ++e)
              reinterpret_cast<uint4*>(vt)[at_value_chunk<D>(i * RPL + ln / LPR, (ln % LPR) * (EV / 8) + e)] =
                  at_bf16<F, W>(vx[i], e, f);
          }
          __builtin_amdgcn_wave_barrier();
#pragma unroll 1
          for (int rr = 0; rr < kAtTile; ++rr) {
            if (rr % 16 >= there[rr / 16]) continue;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
              const uint2 v = *reinterpret_cast<const uint2*>(vt + at_value_chunk<D>(rr, 2 * db) * 8 + 4 * g);
              const float x[4] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)};
#pragma unroll
              for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
                  acc.o[qt][db][k] += !isfinite(x[k]) && trow + rr <= last[qt] ? x[k] : 0.f;
            }
          }
        }
        __builtin_amdgcn_wave_barrier();
        if (TAIL && n + 1 < own_tiles) {
          load_keys(n + 1);
          load_values(n + 1);
        }
      };
      int n = 0;
      for (; n < own_tiles && (int)(lo + turn + KS * n + 1) * kAtTile <= whole + 1; ++n)
        tile(n, std::false_type{});
      for (; n < own_tiles; ++n) tile(n, std::true_type{});

      // The piece's partial: (maximum, sum, unnormalized output) of each query row, the waves
      // joined in LDS.
      // (of the query rows that are the sequence's)
      const int64_t slot = (int64_t)x + u;
      const int kept = WHOLE ? M : own * gm.G;
      int tid_j = tid;
      asm volatile("" : "+v"(tid_j));
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        if (last[qt] < 0) {  // (a query that is not there has seen what is seen by all)
          acc.m[qt] = kAtNone;
          acc.l[qt] = 0.f;
#pragma unroll
          for (int db = 0; db < D / 16; ++db) acc.o[qt][db] = (at_f32x4){0.f, 0.f, 0.f, 0.f};
        }
        float l_row = acc.l[qt];
        l_row += __shfl_xor(l_row, 16, 64);
        l_row += __shfl_xor(l_row, 32, 64);
        const int g = (tid_j & 63) >> 4, c = tid_j & 15;
        float* join = reinterpret_cast<float*>(lds);
        if constexpr (KS == 1) {
          const int row = row0 + qt * 16 + c;
          if (row < kept) {
            const int64_t pr = (slot * 4 + wave) * mp + row;
            if (g == 0) a.part_ml[pr] = make_float2(acc.m[qt], l_row);
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
              *reinterpret_cast<float4*>(a.part_o + pr * D + 16 * db + 4 * g) =
                  make_float4(acc.o[qt][db][0], acc.o[qt][db][1], acc.o[qt][db][2], acc.o[qt][db][3]);
          }
          continue;
        }
        __syncthreads();  // every wave is done with its tiles (and with the tile before)
        if (g == 0) ml_s[wave * 16 + c] = make_float2(acc.m[qt], l_row);
        __syncthreads();
        float mx = kAtNone;
#pragma unroll 4
        for (int k = 0; k < KS; ++k) mx = fmaxf(mx, ml_s[k * 16 + c].x);
        const float w = __builtin_amdgcn_exp2f(acc.m[qt] - mx);
#pragma unroll
        for (int db = 0; db < D / 16; ++db) {
          const at_f32x4 o = acc.o[qt][db];
          *reinterpret_cast<float4*>(join + (wave * 16 + c) * ROW + 16 * db + 4 * g) =
              make_float4(o[0] * w, o[1] * w, o[2] * w, o[3] * w);
        }
        __syncthreads();
        for (int i = tid_j; i < 16 * (D / 4); i += NT) {
          const int rr = i / (D / 4), d4 = i % (D / 4);
          const int row = row0 + qt * 16 + rr;
          if (row >= kept) continue;
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int k = 0; k < KS; ++k) {
            const float4 y = *reinterpret_cast<const float4*>(join + (k * 16 + rr) * ROW + 4 * d4);
            o.x += y.x, o.y += y.y, o.z += y.z, o.w += y.w;
          }
          float mm = kAtNone, sum = 0.f;
          if (WHOLE || d4 == 0) {
#pragma unroll 4
            for (int k = 0; k < KS; ++k) mm = fmaxf(mm, ml_s[k * 16 + rr].x);
#pragma unroll 4
            for (int k = 0; k < KS; ++k) {
              const float2 ml = ml_s[k * 16 + rr];
              sum += ml.y * __builtin_amdgcn_exp2f(ml.x - mm);
            }
          }
          if constexpr (WHOLE) {
            pg_output(a, l, b, h, row, d4, D, o, mm, sum);
          } else {
            const int64_t pr = slot * mp + row;
            reinterpret_cast<float4*>(a.part_o + pr * D)[d4] = o;
            if (d4 == 0) a.part_ml[pr] = make_float2(mm, sum);
          }
        }
      }
      if (WHOLE && tid == 0 && p.offsets[r + 1] - p.offsets[r] != len) report_range(gm);
      if constexpr (KS > 1) __syncthreads();  // the joined tiles are read before the next piece's
    }
  }
}

template <int F, int D, int QT>
static certkv_status launch_paged_d(const PagedArgs& a, hipStream_t s) {
  const int64_t U = (int64_t)a.p.lists * a.copies;
  const int64_t wgs = a.mode == kPgWhole ? U : a.most < a.parts ? a.most : a.parts;
  const bool one = a.qgroups == 1 || a.place;
  const dim3 grid((unsigned)(one ? wgs : (wgs + 7) / 8 * 8 * a.qgroups));
  const dim3 block(64 * pg_waves(a.mode));
  if (a.mode == kPgWhole)
    CERTKV_LAUNCH("paged_whole", (paged_kernel<F, D, QT, kPgWhole>), grid, block, 0, s, a);
  else if (a.mode == kPgHeads)
    CERTKV_LAUNCH("paged_heads", (paged_kernel<F, D, QT, kPgHeads>), grid, block, 0, s, a);
  else
    CERTKV_LAUNCH("paged", (paged_kernel<F, D, QT, kPgPiece>), grid, block, 0, s, a);
  return CERTKV_OK;
}

template <int F>
static certkv_status launch_paged(const PagedArgs& a, int shape, hipStream_t s) {
  if (a.p.g.D == 128)
    return shape == kAtOne ? launch_paged_d<F, 128, 1>(a, s) : launch_paged_d<F, 128, 2>(a, s);
  return shape == kAtOne ? launch_paged_d<F, 64, 1>(a, s) : launch_paged_d<F, 64, 2>(a, s);
}

}  // namespace certkv
