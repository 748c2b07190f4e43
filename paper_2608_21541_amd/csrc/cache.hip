// The packed cache in microscaled codes: written from the kept rows, and read back.
//
// Written (certkv_compact_mx): packed row i of a unit is the kept row at position
// kept_idx[i], its last one the slot (k*, v*); each block of 32 dims is quantised
// as mx.h says, from the source's own precision (bf16, fp32, the slot's fp32).
// Bound by memory: 2 d values of a row are read, 2 d codes, d/16 scales and a
// position written (1.15M rows of 16 layers, bf16 to mxfp4: 0.75 GB in 162 us,
// 4.6 TB/s, where a large copy reaches 5.1; 173 us with other inputs each time; as many
// rows of 64 dims from fp32 0.67 GB in 162 us; 13k rows of one layer 8.2 us, latency).
// D / 8 lanes take a row, eight dims each, so that a wave reads whole rows in
// 16-byte pieces (32 for fp32) and a block's largest magnitude is two exchanges
// within four lanes.  The packed rows of all units, one after another, are cut into
// equal runs, one for each workgroup, so that the share is the same however the rows
// are spread over the units; the unit of a run's first row is found by a 64-way
// search, the next ones by stepping on.
#include "mx.h"
#include "stages.h"

namespace certkv {

constexpr int kMxThreads = 256;

// The block maximum over its four lanes (bits of magnitudes order as numbers do).
__device__ __forceinline__ uint32_t mx_max4(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));  // lanes 1 0 3 2
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));  // lanes 2 3 0 1
  return x;
}

// A lane's eight dims of a row to codes and, from the first of the block's four
// lanes, the scale byte.
template <int F>
__device__ __forceinline__ void mx_store8(const Geo& g, const float x[8], int64_t at,
                                          uint8_t* __restrict__ codes,
                                          uint8_t* __restrict__ scales) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  m = mx_max4(m);
  const bool bad = m >= 0x7f800000u;
  const int e = bad ? 0 : mx_exponent<F>(m);
  const float inv = mx_pow2(-e);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = bad ? 0.f : x[i] * inv;  // (exact, or far below a code)
  const uint2 c = mx_encode8<F>(y);
  if constexpr (F == CERTKV_CACHE_MXFP8)
    *reinterpret_cast<uint2*>(codes + at) = c;
  else
    *reinterpret_cast<uint32_t*>(codes + at / 2) = c.x;
  if ((threadIdx.x & 3) == 0) scales[at / kMxBlock] = bad ? 255u : (uint8_t)(e + 127);
  if (bad) report_nonfinite(g);
}

typedef uint32_t MxU4 __attribute__((ext_vector_type(4)));
typedef float MxF4 __attribute__((ext_vector_type(4)));
template <typename T>
struct MxRaw;  // eight values as they are loaded
template <>
struct MxRaw<uint16_t> {
  uint4 a;
  __device__ __forceinline__ void load(const uint16_t* p) {
    const MxU4 v = __builtin_nontemporal_load(reinterpret_cast<const MxU4*>(p));
    a = make_uint4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ void values(float x[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
};
template <>
struct MxRaw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    const MxF4 v = __builtin_nontemporal_load(reinterpret_cast<const MxF4*>(p));
    const MxF4 w = __builtin_nontemporal_load(reinterpret_cast<const MxF4*>(p) + 1);
    a = make_float4(v[0], v[1], v[2], v[3]);
    b = make_float4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void values(float x[8]) const {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
};

template <int D, typename T, int F>
__global__ __launch_bounds__(kMxThreads) void compact_mx_kernel(
    Geo g, SeqTab st, const T* __restrict__ kc, int64_t k_sl, int64_t k_st, int64_t k_sh,
    const T* __restrict__ vc, int64_t v_sl, int64_t v_st, int64_t v_sh,
    const int64_t* __restrict__ kept_offsets, const int32_t* __restrict__ kept_idx,
    int64_t kept_cap, int64_t row_cap, const float* __restrict__ k_star, const float* __restrict__ v_star,
    uint8_t* __restrict__ k_codes, uint8_t* __restrict__ k_scales, uint8_t* __restrict__ v_codes,
    uint8_t* __restrict__ v_scales, int32_t* __restrict__ pos_packed,
    int64_t* __restrict__ packed_offsets) {
  constexpr int LPR = D / 8;              // lanes per row
  constexpr int RPS = kMxThreads / LPR;   // rows per step of the workgroup
  // Rows of a lane in flight.  (1.15M rows of 16 layers: 4 rows 230 us, 2 205, 1 205; the
  // source rows non-temporally, 2 171: a tenth of the cache in 256-byte pieces is read at
  // 3.4 TB/s at most.)
  constexpr int UR = 2;
  const uint32_t U = (uint32_t)(g.L * g.B * g.H);
  // a unit's first packed row; the offsets are the caller's on the device, so kept rows
  // past the positions given, and packed rows past the buffers, are left out and reported
  auto seg = [&](uint32_t u) { return min(kept_offsets[u], kept_cap) + (int64_t)g.slot * u; };
  for (uint32_t u = blockIdx.x * kMxThreads + threadIdx.x; u <= U; u += gridDim.x * kMxThreads) {
    packed_offsets[u] = min(seg(u), row_cap);
    if (u == U && (kept_offsets[U] > kept_cap || seg(U) > row_cap)) report_range(g);
  }
  // (up to 63 units: their ends, the rows in all and the unit of the first from one load)
  const bool few = U < 64;
  const int lane = threadIdx.x & 63;
  const int64_t s0 = few ? seg(min((uint32_t)lane, U)) : 0;
  const int64_t base = few ? __shfl(s0, 0, 64) : seg(0);
  const int64_t rows = min(few ? __shfl(s0, (int)U, 64) : seg(U), row_cap) - base;
  const int64_t per = ((rows + gridDim.x - 1) / gridDim.x + RPS - 1) / RPS * RPS;
  const int64_t r0 = base + blockIdx.x * per, r1 = min(base + rows, r0 + per);
  if (r0 >= r1) return;
  // the unit of row r0, 64 units' ends per step
  uint32_t u = 0;
  if (few) u = (uint32_t)__popcll(__ballot(lane > 0 && lane <= (int)U && s0 <= r0));
  for (uint32_t n = few ? 0 : U; n > 0;) {
    const uint32_t step = (n + 63) / 64, i = u + lane * step + step - 1;
    const bool past = i >= U || seg(i + 1) > r0;
    u += (uint32_t)__popcll(__ballot(!past)) * step;
    if (step == 1) break;
    n = step;
  }
  u = min(u, U - 1);
  const int ri = threadIdx.x / LPR, ci = threadIdx.x % LPR;
  // The lane's current unit: the row behind its last, and where its source rows are.
  // (Worked out when the unit changes: its divisions would be the time of a row.)
  int64_t end = 0, k_at = 0, v_at = 0;
  int32_t n = 0;  // source rows; 0: another launch's sequence
  auto enter = [&](int64_t unit_end) {
    end = unit_end;
    const uint32_t h = u % (uint32_t)g.H, lb = u / (uint32_t)g.H;
    const uint32_t l = lb / (uint32_t)g.B;
    const int b = (int)(lb - l * (uint32_t)g.B) - st.first;
    const bool mine = b >= 0 && b < st.count;
    const int64_t tok = mine ? st.start[b] : 0;
    n = mine ? st.len[b] : 0;
    k_at = l * k_sl + tok * k_st + h * k_sh + ci * 8;
    v_at = l * v_sl + tok * v_st + h * v_sh + ci * 8;
  };
  enter(few ? __shfl(s0, (int)u + 1, 64) : seg(u + 1));
  for (int64_t r = r0 + ri; r < r1; r += RPS * UR) {
    // The rows' sources, then the rows, in flight together; rows past the run and other
    // launches' fetch the unit's first row (or the tensor's), unused.
    int64_t ka[UR], va[UR];
    int32_t j[UR];
    uint32_t unit[UR];
    bool slot[UR], mine[UR];
#pragma unroll
    for (int q = 0; q < UR; ++q) {
      const int64_t x = r + q * RPS;
      while (x >= end && u + 1 < U) {
        ++u;
        enter(seg(u + 1));
      }
      unit[q] = u;
      mine[q] = x < r1 && n > 0;
      slot[q] = mine[q] && g.slot && x + 1 == end;
      j[q] = mine[q] && !slot[q] ? min(max(kept_idx[x - (int64_t)g.slot * u], 0), n - 1) : 0;  // caller indices clamped
      ka[q] = k_at;
      va[q] = v_at;
    }
    MxRaw<T> kx[UR], vx[UR];
#pragma unroll
    for (int q = 0; q < UR; ++q) {
      kx[q].load(kc + ka[q] + j[q] * k_st);
      vx[q].load(vc + va[q] + j[q] * v_st);
    }
#pragma unroll
    for (int q = 0; q < UR; ++q) {
      const int64_t x = r + q * RPS;
      if (!mine[q]) continue;  // (a whole row's lanes)
      float ky[8], vy[8];
      if (slot[q]) {
        MxRaw<float> s;
        s.load(k_star + (int64_t)unit[q] * D + ci * 8);
        s.values(ky);
        s.load(v_star + (int64_t)unit[q] * D + ci * 8);
        s.values(vy);
      } else {
        kx[q].values(ky);
        vx[q].values(vy);
      }
      mx_store8<F>(g, ky, x * D + ci * 8, k_codes, k_scales);
      mx_store8<F>(g, vy, x * D + ci * 8, v_codes, v_scales);
      if (ci == 0) pos_packed[x] = slot[q] ? -1 : j[q];
    }
  }
}

template <int D, typename T, int F>
static certkv_status launch_compact_mx(const CompactMxArgs& a, const SeqTab& st, hipStream_t s) {
  // eight workgroups of four waves per compute unit fill it
  CERTKV_LAUNCH("compact_mx", (compact_mx_kernel<D, T, F>), dim3(8 * 256), dim3(kMxThreads), 0, s,
                a.g, st, static_cast<const T*>(a.k.ptr), a.k.s_layer, a.k.s_token, a.k.s_head,
                static_cast<const T*>(a.v.ptr), a.v.s_layer, a.v.s_token, a.v.s_head,
                a.kept_offsets, a.kept_idx, a.kept_cap, a.row_cap, a.k_star, a.v_star, a.k_codes, a.k_scales, a.v_codes,
                a.v_scales, a.pos_packed, a.packed_offsets);
  return CERTKV_OK;
}

template <int D, typename T>
static certkv_status launch_compact_mx_f(const CompactMxArgs& a, const SeqTab& st, hipStream_t s) {
  return a.format == CERTKV_CACHE_MXFP8 ? launch_compact_mx<D, T, CERTKV_CACHE_MXFP8>(a, st, s)
                                        : launch_compact_mx<D, T, CERTKV_CACHE_MXFP4>(a, st, s);
}

certkv_status run_compact_mx(const CompactMxArgs& a, const SeqTab& st, hipStream_t s) {
  if (a.dtype == CERTKV_BF16)
    return a.g.D == 128 ? launch_compact_mx_f<128, uint16_t>(a, st, s)
                        : launch_compact_mx_f<64, uint16_t>(a, st, s);
  return a.g.D == 128 ? launch_compact_mx_f<128, float>(a, st, s)
                      : launch_compact_mx_f<64, float>(a, st, s);
}

// Codes back to values, eight dims a lane: the rows of both arrays are contiguous,
// so an item is eight dims of either and its scale byte the item's quarter.  Bound
// by the writes (mxfp8: 1.03 bytes read for 2 written as bf16), which are made
// non-temporally (1.15M rows of mxfp4 after they were written 153 us without, 111
// with; 3.36M of mxfp8 by themselves 510 and 496, 5.3 TB/s).  blockIdx.y: keys or values.
template <int F, bool F32>
__global__ __launch_bounds__(kMxThreads) void read_mx_kernel(
    int64_t items, const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_scales,
    const uint8_t* __restrict__ v_codes, const uint8_t* __restrict__ v_scales,
    void* __restrict__ k_out, void* __restrict__ v_out) {
  const uint8_t* codes = blockIdx.y ? v_codes : k_codes;
  const uint8_t* scales = blockIdx.y ? v_scales : k_scales;
  void* out = blockIdx.y ? v_out : k_out;
  if (!out) return;
  for (int64_t i = (int64_t)blockIdx.x * kMxThreads + threadIdx.x; i < items;
       i += (int64_t)gridDim.x * kMxThreads) {
    uint2 c = make_uint2(0u, 0u);
    if constexpr (F == CERTKV_CACHE_MXFP8)
      c = reinterpret_cast<const uint2*>(codes)[i];
    else
      c.x = reinterpret_cast<const uint32_t*>(codes)[i];
    const uint32_t x = scales[i >> 2];
    uint4 v = mx_decode8<F>(c, mx_scale(x == 255u ? 127u : x));
    if (x == 255u) v = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    if constexpr (F32) {
      MxF4* o = reinterpret_cast<MxF4*>(out) + 2 * i;
      __builtin_nontemporal_store((MxF4){bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)}, o);
      __builtin_nontemporal_store((MxF4){bf16_lo(v.z), bf16_hi(v.z), bf16_lo(v.w), bf16_hi(v.w)}, o + 1);
    } else {
      __builtin_nontemporal_store((MxU4){v.x, v.y, v.z, v.w}, reinterpret_cast<MxU4*>(out) + i);
    }
  }
}

template <int F, bool F32>
static certkv_status launch_read_mx(const ReadMxArgs& a, hipStream_t s) {
  const int64_t wgs = (a.items + kMxThreads - 1) / kMxThreads;
  CERTKV_LAUNCH("read_mx", (read_mx_kernel<F, F32>),
                dim3((unsigned)(wgs < 4 * 256 ? wgs : 4 * 256), 2), dim3(kMxThreads), 0, s,
                a.items, a.k_codes, a.k_scales, a.v_codes, a.v_scales, a.k_out, a.v_out);
  return CERTKV_OK;
}

certkv_status run_read_mx(const ReadMxArgs& a, hipStream_t s) {
  if (a.format == CERTKV_CACHE_MXFP8)
    return a.f32 ? launch_read_mx<CERTKV_CACHE_MXFP8, true>(a, s)
                 : launch_read_mx<CERTKV_CACHE_MXFP8, false>(a, s);
  return a.f32 ? launch_read_mx<CERTKV_CACHE_MXFP4, true>(a, s)
               : launch_read_mx<CERTKV_CACHE_MXFP4, false>(a, s);
}

}  // namespace certkv
