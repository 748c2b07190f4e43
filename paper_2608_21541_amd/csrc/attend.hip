// Attention of new queries over a packed cache of any format and new rows.
//
// For query row (t, head h G + g) of sequence b, over the unit's packed rows and the
// sequence's new rows j that mask[b][t][j] admits:
//   z_i = scale <q, k_i>,  out = sum_i softmax(z)_i v_i,  lse = log sum_i e^z_i,
// with out = 0 and lse = -inf where no row is visible.
//
// A workgroup per (unit, query row): each wave takes 64 rows at a time, a row to a
// lane for the dot products, dims to lanes for the weighted sum, with a running
// maximum and sum; the four waves are joined in LDS.
#include "mx.h"
#include "stages.h"

namespace certkv {

// Dims 8 c .. 8 c + 7 of packed row r as floats.
template <int D, int F>
__device__ __forceinline__ void attend_load8(const void* codes, const uint8_t* scales, int64_t r,
                                             int c, float x[8]) {
  uint4 v;
  if constexpr (F == CERTKV_CACHE_BF16) {
    v = reinterpret_cast<const uint4*>(codes)[r * (D / 8) + c];
  } else {
    uint2 w = make_uint2(0u, 0u);
    if constexpr (F == CERTKV_CACHE_MXFP8)
      w = reinterpret_cast<const uint2*>(codes)[r * (D / 8) + c];
    else
      w.x = reinterpret_cast<const uint32_t*>(codes)[r * (D / 8) + c];
    const uint32_t b = scales[r * (D / kMxBlock) + c / 4];
    v = mx_decode8<F>(w, mx_scale(b == 255u ? 127u : b));
    if (b == 255u) v = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(w[i]);
    x[2 * i + 1] = bf16_hi(w[i]);
  }
}

template <int D, int F>
__global__ __launch_bounds__(256) void attend_kernel(
    Geo g, int32_t tq, int32_t tn, int64_t cover, const uint16_t* __restrict__ qn, int64_t q_sl,
    int64_t q_st, int64_t q_sh, certkv_cache cache, const uint16_t* __restrict__ kn, int64_t kn_sl,
    int64_t kn_st, int64_t kn_sh, const uint16_t* __restrict__ vn, int64_t vn_sl, int64_t vn_st,
    int64_t vn_sh, const uint8_t* __restrict__ mask, float* __restrict__ out,
    float* __restrict__ lse) {
  __shared__ float q_s[D];
  __shared__ float o_s[4][D];
  __shared__ float2 ml_s[4];
  const int64_t u = blockIdx.x;
  const int row = blockIdx.y;
  const int h = (int)(u % g.H);
  const int64_t lb = u / g.H;
  const int b = (int)(lb % g.B);
  const int l = (int)(lb / g.B);
  const int t = row / g.G, gq = row % g.G;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t p0 = cache.offsets[u];
  const int64_t full = cache.offsets[u + 1] - p0;
  const int64_t len = full < cover ? full : cover;
  if (full > cover && row == 0 && tid == 0) report_range(g);
  if (tid < D)
    q_s[tid] = bf16_to_f32(qn[l * q_sl + (int64_t)(b * tq + t) * q_st +
                              (int64_t)(h * g.G + gq) * q_sh + tid]) * g.scale;
  __syncthreads();
  float m = -INFINITY, sum = 0.f, o[D / 64];
  for (int i = 0; i < D / 64; ++i) o[i] = 0.f;
  for (int64_t j0 = wave * 64; j0 < len + tn; j0 += 256) {
    const int64_t j = j0 + lane;
    float z = -INFINITY;
    bool see = j < len;
    const int64_t jn = j - len;
    if (!see && jn < tn)
      see = mask ? mask[((int64_t)b * tq + t) * tn + jn] != 0 : jn <= tn - tq + t;
    if (see) {
      z = 0.f;
      for (int c = 0; c < D / 8; ++c) {
        float x[8];
        if (j < len)
          attend_load8<D, F>(cache.k, cache.k_scales, p0 + j, c, x);
        else
          for (int e = 0; e < 8; ++e)
            x[e] = bf16_to_f32(kn[l * kn_sl + (b * (int64_t)tn + jn) * kn_st + h * kn_sh + c * 8 + e]);
        for (int e = 0; e < 8; ++e) z = fmaf(q_s[c * 8 + e], x[e], z);
      }
    }
    const float mx = fmaxf(m, wave_max(z));
    if (mx == -INFINITY && !__any(z != z)) continue;
    const float a = m == -INFINITY ? 0.f : expf(m - mx), p = see ? expf(z - mx) : 0.f;
    m = mx;
    sum = sum * a + wave_sum(p);
    for (int i = 0; i < D / 64; ++i) o[i] *= a;
    for (int k = 0; k < 64; ++k) {
      const float pk = __shfl(p, k, 64);
      const int64_t jk = j0 + k;
      if (!__shfl((int)see, k, 64)) continue;
      for (int i = 0; i < D / 64; ++i) {
        const int d = i * 64 + lane;
        float v;
        if (jk < len) {
          float x[8];
          attend_load8<D, F>(cache.v, cache.v_scales, p0 + jk, d / 8, x);
          v = 0.f;
          for (int e = 0; e < 8; ++e) v = (d & 7) == e ? x[e] : v;
        } else {
          v = bf16_to_f32(vn[l * vn_sl + (b * (int64_t)tn + jk - len) * vn_st + h * vn_sh + d]);
        }
        o[i] = fmaf(pk, v, o[i]);
      }
    }
  }
  for (int i = 0; i < D / 64; ++i) o_s[wave][i * 64 + lane] = o[i];
  if (lane == 0) ml_s[wave] = make_float2(m, sum);
  __syncthreads();
  float mx = -INFINITY, tot = 0.f, x = 0.f;
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, ml_s[w].x);
  for (int w = 0; w < 4; ++w) {
    if (ml_s[w].y == 0.f) continue;
    const float a = expf(ml_s[w].x - mx);
    tot += ml_s[w].y * a;
    if (tid < D) x += o_s[w][tid] * a;
  }
  if (tid >= D) return;
  const int64_t orow = ((int64_t)l * g.B * tq + (int64_t)b * tq + t) * (g.H * g.G) + h * g.G + gq;
  const float y = tot == 0.f ? 0.f : x / tot;
  if (!isfinite(y)) report_nonfinite(g);
  out[orow * D + tid] = y;
  if (lse && tid == 0) lse[orow] = tot == 0.f ? -INFINITY : mx + logf(tot);
}

template <int D, int F>
static certkv_status launch_attend(const AttendArgs& a, hipStream_t s) {
  CERTKV_LAUNCH("attend", (attend_kernel<D, F>),
                dim3((unsigned)a.U, (unsigned)(a.tq * a.g.G)), dim3(256), 0, s, a.g, a.tq, a.tn,
                a.cover, static_cast<const uint16_t*>(a.q.ptr), a.q.s_layer, a.q.s_token,
                a.q.s_head, a.cache, static_cast<const uint16_t*>(a.k_new.ptr), a.k_new.s_layer,
                a.k_new.s_token, a.k_new.s_head, static_cast<const uint16_t*>(a.v_new.ptr),
                a.v_new.s_layer, a.v_new.s_token, a.v_new.s_head, a.mask, a.out, a.lse);
  return CERTKV_OK;
}

template <int D>
static certkv_status launch_attend_f(const AttendArgs& a, hipStream_t s) {
  switch (a.cache.format) {
    case CERTKV_CACHE_MXFP8: return launch_attend<D, CERTKV_CACHE_MXFP8>(a, s);
    case CERTKV_CACHE_MXFP4: return launch_attend<D, CERTKV_CACHE_MXFP4>(a, s);
    default: return launch_attend<D, CERTKV_CACHE_BF16>(a, s);
  }
}

certkv_status run_attend(const AttendArgs& a, hipStream_t s) {
  return a.g.D == 128 ? launch_attend_f<128>(a, s) : launch_attend_f<64>(a, s);
}

}  // namespace certkv
