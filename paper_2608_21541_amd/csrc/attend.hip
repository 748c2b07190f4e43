// Attention over a packed cache of any format: chunks, dispatch, and the partials joined.
#include "attend.h"

namespace certkv {

bool attend_chunks(int D, int tq, int G, int tn, int64_t rows, int64_t U, AttendChunks* c) {
  const int M = tq * G;
  // By the query rows: each shape's padded rows cost as much as real ones.  (Over 3.36M rows of
  // mxfp8: up to 64 query rows as two groups of 32, each of which reads the cache, take 288 us,
  // the second group's reads from L2, with four waves that share their tiles 338.  128 query
  // rows with eight waves, half of them idle, 476, with four 432.  256 with eight 770, as two
  // groups of 128 835.)
  c->shape = M <= 16 ? kAtOne : M <= 64 ? kAtTwo : M <= 128 ? kAtEight : kAtSixteen;
  const int held = c->shape == kAtOne ? 16 : c->shape == kAtTwo ? 32 : c->shape == kAtEight ? 128 : 256;
  c->qgroups = (M + held - 1) / held;
  c->mp = c->qgroups * held;
  // as many chunks as their workgroups stay resident: 256 compute units of four SIMDs
  c->parts = 256 * 4 * attend_waves(D, c->shape) / attend_wg_waves(c->shape);
  c->parts = (c->parts + c->qgroups - 1) / c->qgroups;
  // (What a piece costs beside its tiles, in rows; one value for all shapes, though few query
  // rows would take any.  With weights in two parts: eight ragged sequences, 192 query rows,
  // 64: 137 us, 256: 124, 512: 131; 32 query rows, mxfp8: 187, 178, 181; 4 query rows, mxfp4:
  // 75, 73, 75.)
  c->gap = 256;
  auto chunks = [&](int64_t total, int64_t least) {
    const int64_t shortest = (total + least - 1) / least;
    int64_t most = (total + kAtMaxKeys - 1) / kAtMaxKeys;
    if (most < c->parts) most = c->parts;
    if (most > shortest) most = shortest;
    return (int32_t)(most > 0 ? most : 1);
  };
  const int64_t total = (rows + 31) / 32 * 32 + U * c->gap, fresh = U * ((tn + 31) / 32 * 32);
  if (U > INT32_MAX || total > INT32_MAX || fresh > INT32_MAX) return false;
  c->most = chunks(total, kAtMinKeys);
  c->most_new = chunks(fresh, kAtTile);
  return true;
}

constexpr int kAtJoinThreads = 256;

// The partials of each (unit, query row) joined in row order: with m the largest of their
// maxima m_k, out = sum_k 2^(m_k - m) o_k / sum_k 2^(m_k - m) l_k.  D / 4 threads fold one
// row's, four in flight; S groups of them share the partials of a row (with few rows),
// or take a row each (S = 1).  Bound by the reads of the partials (256 units, 256 query rows:
// 135 MB read and written in 25 us, 5.5 TB/s; of 192 rows and three pieces to a unit 97 MB in
// 21 us); for one layer by their latency (5 us).
template <int D, int S>
__global__ __launch_bounds__(kAtJoinThreads) void attend_join_kernel(AttendArgs a) {
  constexpr int C4 = D / 4, GR = kAtJoinThreads / C4, RW = GR / S;
  __shared__ float4 acc_s[GR][C4];
  __shared__ float2 ml_s[GR];
  const Geo& g = a.g;
  const uint32_t u = blockIdx.x;
  const int grp = threadIdx.x / C4, c4 = threadIdx.x % C4;
  const int row = blockIdx.y * RW + grp / S, sg = grp % S;
  const int M = a.tq * g.G;
  const int64_t* off = a.cache.offsets;
  const int64_t full = off[u + 1] - off[u];
  if (full > a.cover && blockIdx.y == 0 && threadIdx.x == 0) report_range(g);
  float m = kAtNone, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  // nv partials from `first` on
  auto fold = [&](int64_t first, uint32_t nv) {
    constexpr int Q = 4;
    for (uint32_t i0 = sg; i0 < nv; i0 += Q * S) {
      float2 ml[Q];
      float4 x[Q];
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        const int64_t pr = (first + min(i0 + i * S, nv - 1)) * a.ck.mp + row;
        ml[i] = a.part_ml[pr];
        x[i] = reinterpret_cast<const float4*>(a.part_o + pr * D)[c4];
      }
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        if (i0 + i * S >= nv) continue;
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
  };
  if (row < M) {
    const AtCut cut = at_cut_packed(a, off[a.U] - off[0]);
    const uint32_t vs = at_place(off[u] - off[0], u, a.ck.gap), s0 = vs / cut.keys;
    const uint32_t len = (uint32_t)min(full, a.cover);
    fold((int64_t)s0 + u, len ? (vs + len - 1) / cut.keys - s0 + 1 : 0);
    if (a.tn) {
      const AtCut fresh = at_cut_new(a);
      const uint32_t ns = (uint32_t)u * at_up32((uint32_t)a.tn), n0 = ns / fresh.keys;
      fold(a.ck.most + a.U + n0 + u, (ns + a.tn - 1) / fresh.keys - n0 + 1);
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
  const int h = (int)(u % (uint32_t)g.H), b = (int)(u / g.H % (uint32_t)g.B);
  const int l = (int)(u / g.H / g.B);
  const int t = row / g.G, gq = row % g.G;
  const int64_t orow = ((int64_t)l * g.B * a.tq + (int64_t)b * a.tq + t) * (g.H * g.G) + h * g.G + gq;
  const float inv = L == 0.f ? 0.f : 1.f / L;  // (nothing visible: out 0, lse -inf)
  const float y[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
  bool fine = true;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    fine = fine && isfinite(y[i]);
    a.out[orow * D + 4 * c4 + i] = y[i];
  }
  if (!fine) report_nonfinite(g);
  if (a.lse && c4 == 0)
    a.lse[orow] = L == 0.f ? -INFINITY
                           : (ref_log2(m, g.scale * kAtLog2e) + __builtin_amdgcn_logf(L)) * kAtLn2;
}

template <int D>
static certkv_status launch_attend_join(const AttendArgs& a, hipStream_t s) {
  constexpr int GR = kAtJoinThreads / (D / 4);
  const int M = a.tq * a.g.G;
  // The partials of few rows are dealt out, of many taken row by row (in us, dealt and not:
  // 256 rows 9 and 24, 1024 7 and 10, 4096 10 and 10, 8192 15 and 10).
  if (a.U * M < 8192)
    CERTKV_LAUNCH("attend_join", (attend_join_kernel<D, GR>), dim3((unsigned)a.U, (unsigned)M),
                  dim3(kAtJoinThreads), 0, s, a);
  else
    CERTKV_LAUNCH("attend_join", (attend_join_kernel<D, 1>),
                  dim3((unsigned)a.U, (unsigned)((M + GR - 1) / GR)), dim3(kAtJoinThreads), 0, s, a);
  return CERTKV_OK;
}

certkv_status run_attend(const AttendArgs& a, hipStream_t s) {
  const certkv_status st = a.cache.format == CERTKV_CACHE_MXFP8   ? run_attend_mxfp8(a, s)
                           : a.cache.format == CERTKV_CACHE_MXFP4 ? run_attend_mxfp4(a, s)
                                                                  : run_attend_bf16(a, s);
  if (st != CERTKV_OK) return st;
  return a.g.D == 128 ? launch_attend_join<128>(a, s) : launch_attend_join<64>(a, s);
}

}  // namespace certkv
