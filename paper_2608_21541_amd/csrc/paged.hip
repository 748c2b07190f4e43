// Attention over a paged cache: dispatch by format, and the partials joined.
#include "paged.h"

namespace certkv {

constexpr int kPgJoinThreads = 256;

// The partials of each (unit, query row) joined in row order: with m the largest of their
// maxima m_k, out = sum_k 2^(m_k - m) o_k / sum_k 2^(m_k - m) l_k.  D / 4 threads fold one row's,
// four in flight; S groups of them share the partials of a row (with few rows), or take a row
// each (S = 1).
template <int D, int S>
__global__ __launch_bounds__(kPgJoinThreads) void paged_join_kernel(PagedArgs a) {
  constexpr int C4 = D / 4, GR = kPgJoinThreads / C4, RW = GR / S;
  __shared__ float4 acc_s[GR][C4];
  __shared__ float2 ml_s[GR];
  const PageArgs& p = a.p;
  const Geo& g = p.g;
  // the unit, or of four heads' units the place in common and the head's
  const uint32_t four = a.mode == kPgHeads ? 4u : 1u, u = blockIdx.x / four, head = blockIdx.x % four;
  const uint32_t r = u / (uint32_t)a.copies, copy = u % (uint32_t)a.copies;
  const int grp = threadIdx.x / C4, c4 = threadIdx.x % C4;
  const int row = blockIdx.y * RW + grp / S, sg = grp % S;
  const int M = a.tq * g.G;
  int l, b, h;
  if (p.per_head) {
    h = (int)(r % (uint32_t)g.H), b = (int)(r / g.H % (uint32_t)g.B), l = (int)(r / g.H / g.B);
  } else {
    const uint32_t x = copy * four + head;
    b = (int)r, l = (int)(x / (uint32_t)g.H), h = (int)(x % (uint32_t)g.H);
  }
  // (all asked for at once, what is not there in the offsets' place: latency)
  const uint32_t* const places = a.place ? a.place : reinterpret_cast<const uint32_t*>(p.offsets);
  const int32_t* const q_lens = a.q_lens ? a.q_lens : reinterpret_cast<const int32_t*>(p.offsets);
  const int64_t base = p.offsets[0], p0 = p.offsets[r] - base, p1 = p.offsets[r + 1] - base;
  const int64_t rows = p.offsets[p.lists] - base;
  const uint32_t place_r = places[r], place_all = places[p.lists];
  const int32_t q_len = q_lens[b];
  const int len = pg_held(p0, p1, rows) ? min(page_rows(p, p0, p1), a.cover) : 0;
  const PgCut cut = pg_cut(a, a.place ? place_all : pg_tiles(rows, (uint32_t)p.lists, a.gap));
  if ((p1 - p0 != len || !cut.fits) && blockIdx.y == 0 && threadIdx.x == 0) report_range(g);
  float m = kAtNone, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  uint32_t group = 0, groups = 1;
  const int own = a.q_lens ? pg_own(a, q_len) : a.tq;
  if (a.place) groups = pg_groups(a, own), group = (uint32_t)row >> 5;
  if (row < own * g.G && len > 0 && cut.fits) {  // (others have no partials)
    const uint32_t span = pg_place(p1, r + 1, a.gap) - pg_place(p0, r, a.gap);
    const uint32_t place = a.place ? place_r : pg_place(p0, r, a.gap);
    const uint32_t vs = (uint32_t)a.copies * place + (copy * groups + group) * span;
    const PgPieces own_pieces = pg_pieces(vs, pg_up(len), cut.tiles);
    const uint32_t s0 = own_pieces.first, nv = own_pieces.n;
    constexpr int Q = 4;
    for (uint32_t i0 = sg; i0 < nv; i0 += Q * S) {
      float2 ml[Q];
      float4 x[Q];
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        const int64_t pr = (((int64_t)s0 + u + min(i0 + i * S, nv - 1)) * four + head) * a.mp + row;
        ml[i] = i0 + i * S < nv ? a.part_ml[pr] : make_float2(kAtNone, 0.f);
        x[i] = reinterpret_cast<const float4*>(a.part_o + pr * D)[c4];
      }
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        const float mn = fmaxf(m, ml[i].x);
        const float e = __builtin_amdgcn_exp2f(m - mn);
        const float w = __builtin_amdgcn_exp2f(ml[i].x - mn);
        m = mn;
        L = fmaf(L, e, ml[i].y * w);
        o.x = fmaf(o.x, e, x[i].x * w);
        o.y = fmaf(o.y, e, x[i].y * w);
        o.z = fmaf(o.z, e, x[i].z * w);
        o.w = fmaf(o.w, e, x[i].w * w);
      }
    }
  }
  if constexpr (S > 1) {
    acc_s[grp][c4] = o;
    if (c4 == 0) ml_s[grp] = make_float2(m, L);
    __syncthreads();
    if (sg != 0) return;
    float mx = m;
#pragma unroll
    for (int k = 1; k < S; ++k) mx = fmaxf(mx, ml_s[grp + k].x);
    const float e = __builtin_amdgcn_exp2f(m - mx);
    L *= e;
    o.x *= e, o.y *= e, o.z *= e, o.w *= e;
#pragma unroll
    for (int k = 1; k < S; ++k) {
      const float2 ml = ml_s[grp + k];
      const float w = __builtin_amdgcn_exp2f(ml.x - mx);
      const float4 x = acc_s[grp + k][c4];
      L = fmaf(ml.y, w, L);
      o.x = fmaf(x.x, w, o.x);
      o.y = fmaf(x.y, w, o.y);
      o.z = fmaf(x.z, w, o.z);
      o.w = fmaf(x.w, w, o.w);
    }
    m = mx;
  }
  if (row >= M) return;
  pg_output(a, l, b, h, row, c4, D, o, m, L);
}

template <int D>
static certkv_status launch_paged_join(const PagedArgs& a, hipStream_t s) {
  constexpr int GR = kPgJoinThreads / (D / 4);
  const int M = a.tq * a.p.g.G;
  const int64_t U = (int64_t)a.p.lists * a.copies * (a.mode == kPgHeads ? 4 : 1);
  // The partials of few rows, or of many pieces to a unit, are dealt out, others taken row by row.
  // (In us, dealt and not: 8 units of 64 pieces, 4 rows 8 and 38; 256 units of 4 rows 4 and 4; 1024
  // of 4 rows 9 and 5; 64 units of 48 rows 8 and 7.)
  const int64_t chunks = a.most < a.parts ? a.most : a.parts;
  if (U * M < 2048 || chunks >= 8 * (int64_t)a.p.lists * a.copies)
    CERTKV_LAUNCH("paged_join", (paged_join_kernel<D, GR>), dim3((unsigned)U, (unsigned)M),
                  dim3(kPgJoinThreads), 0, s, a);
  else
    CERTKV_LAUNCH("paged_join", (paged_join_kernel<D, 1>),
                  dim3((unsigned)U, (unsigned)((M + GR - 1) / GR)), dim3(kPgJoinThreads), 0, s, a);
  return CERTKV_OK;
}

certkv_status run_paged(const PagedArgs& a, int shape, hipStream_t s) {
  const certkv_status st = a.p.format == CERTKV_CACHE_MXFP8   ? run_paged_mxfp8(a, shape, s)
                           : a.p.format == CERTKV_CACHE_MXFP4 ? run_paged_mxfp4(a, shape, s)
                                                              : run_paged_bf16(a, shape, s);
  if (st != CERTKV_OK || a.mode == kPgWhole) return st;
  return a.p.g.D == 128 ? launch_paged_join<128>(a, s) : launch_paged_join<64>(a, s);
}

}  // namespace certkv
