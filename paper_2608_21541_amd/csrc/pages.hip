// The paged cache's tables and slots, and rows written to, copied to and read from its pages.
#include "pages.h"

namespace certkv {

constexpr int kPgThreads = 256;
constexpr int kPgScan = 1024;      // lists of a step of the scan
constexpr int kPgSmallSlots = 16384;  // slots that the scan's own workgroup fills in

// ---- tables and slots ---------------------------------------------------------
//
// Of list r: had_r rows, will_r = max(0, had_r + change_r), a page for every `page` rows.  With
// need_r = pages(will) - pages(had) where that is positive and give_r where it is negative, list
// r takes the ring's places head + sum_{i<r} need_i on and gives its last pages to the places
// behind the free ones, from sum_{i<r} give_i on; its slots stand from sum_{i<r} max(0, change_i)
// on.  Lists are refused in order, so that a list that takes pages has none that is refused for
// their number before it, and the places taken have no gap.  (Refused for its own length: need
// counts as 0.)  A scan of the lists by one workgroup, 1024 at a time, then the slots and table
// entries from the sums: by the same workgroup where they are few, else by a second launch.

// What the second part needs of each list, in the workspace or LDS.
struct PgLists {
  int32_t* had;
  int32_t* pos;   // place of the ring of its first new page, or -1: refused
  int32_t* keep;  // pages that are left to a list that gives some
  int32_t* give;  // [lists + 1] sums of the pages given
  int32_t* tail;  // place of the ring where they go, and how many
};
constexpr int64_t pg_pad(int64_t n) { return (n + 63) & ~(int64_t)63; }
__host__ __device__ static inline PgLists pg_lists(int32_t* ws, int64_t lists) {
  PgLists x;
  x.tail = ws;
  x.had = ws + 64;
  x.pos = x.had + pg_pad(lists);
  x.keep = x.pos + pg_pad(lists);
  x.give = x.keep + pg_pad(lists);
  return x;
}
size_t page_resize_ws(int64_t lists) {
  return (size_t)(64 + 3 * pg_pad(lists) + pg_pad(lists + 1)) * sizeof(int32_t);
}

template <typename T, typename F>
__device__ __forceinline__ T pg_wave_scan(T x, int lane, F add) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T y = __shfl_up(x, d, 64);
    if (lane >= d) x = add(x, y);
  }
  return x;
}

// The slot of row `row` of list r, which has `had` rows and new pages from place pos on; its new
// pages' table entries are written by the threads of their first rows.
__device__ __forceinline__ int32_t pg_slot(const PageResizeArgs& a, int64_t r, int32_t row,
                                           int32_t had, int32_t pos) {
  if (pos < 0) return -1;
  const int32_t mask = (1 << a.lp) - 1, held = (had + mask) >> a.lp, pi = row >> a.lp;
  int32_t* entry = a.table + r * a.max_pages + pi;
  int32_t id;
  if (pi < held) {
    id = *entry;
  } else {
    id = a.ring[(uint32_t)(pos + (pi - held)) % (uint32_t)a.num_pages];
    if ((row & mask) == 0) *entry = id;
  }
  if ((uint32_t)id >= (uint32_t)a.num_pages) {  // (the caller's numbers)
    report_range(a.g);
    return -1;
  }
  return (id << a.lp) + (row & mask);
}

// The last r of [lo, hi] with first(r) <= x.
template <typename F>
__device__ __forceinline__ int32_t pg_bisect(int32_t lo, int32_t hi, F first, int64_t x) {
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) >> 1;
    if (first(mid) <= x)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

template <bool SMALL>
__global__ __launch_bounds__(kPgScan) void page_resize_kernel(PageResizeArgs a) {
  constexpr int W = kPgScan / 64;
  __shared__ int32_t need_s[W], give_s[W], taken_s;
  __shared__ int64_t add_s[W], len_s[W], end_s;
  // (up to kPgScan lists)
  __shared__ int32_t had_s[SMALL ? kPgScan : 1], pos_s[SMALL ? kPgScan : 1];
  __shared__ int32_t keep_s[SMALL ? kPgScan : 1], go_s[SMALL ? kPgScan + 1 : 1];
  __shared__ int32_t so_s[SMALL ? kPgScan + 1 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t R = a.lists, N = a.num_pages, mask = (1 << a.lp) - 1;
  const int64_t most_rows = (int64_t)a.max_pages << a.lp;
  const int64_t base = a.offsets[0];
  const int32_t head = (int32_t)((uint64_t)a.free[0] % (uint64_t)N);
  const int64_t free_pages = a.free[1];
  const int32_t count = (int32_t)(free_pages < 0 ? 0 : free_pages < N ? free_pages : N);
  const PgLists ws = pg_lists(a.ws, R);
  // sums of pages stop at N + 1, more than there are
  const auto sat = [N](int32_t x, int32_t y) { return min(x + y, N + 1); };
  const auto sum = [](int64_t x, int64_t y) { return x + y; };
  int32_t need_c = 0, give_c = 0;
  int64_t add_c = 0, len_c = 0, old_end = base;
  bool refused = free_pages != count;
  if (tid == 0) taken_s = 0;
  for (int32_t r0 = 0; r0 < R; r0 += kPgScan) {
    const int32_t r = r0 + tid;
    const bool in = r < R;
    // (offsets_out may be offsets: the step before has written this one's first)
    const int64_t first = tid == 0 ? old_end : in ? a.offsets[r] : 0;
    const int64_t end = in ? a.offsets[r + 1] : 0;
    const int32_t change = in ? a.change[r] : 0;
    const int64_t n = end - first;
    const int32_t had = (int32_t)(n < 0 || !in ? 0 : n < most_rows ? n : most_rows);
    const int64_t sumrows = (int64_t)had + change, will = sumrows < 0 ? 0 : sumrows;
    const int32_t held = (had + mask) >> a.lp;
    const int64_t want = (will + mask) >> a.lp;
    const bool fits = want <= a.max_pages;
    int32_t need = 0, give = 0;
    if (want > held && fits) need = (int32_t)min(want - held, (int64_t)N + 1);
    if (want < held) give = min(held - (int32_t)want, N + 1);
    const int32_t add = change > 0 ? change : 0;
    const int32_t need_i = pg_wave_scan(need, lane, sat);
    const int32_t give_i = pg_wave_scan(give, lane, sat);
    const int64_t add_i = pg_wave_scan((int64_t)add, lane, sum);
    if (lane == 63) {
      need_s[wave] = need_i;
      give_s[wave] = give_i;
      add_s[wave] = add_i;
    }
    if (tid == kPgScan - 1) end_s = end;
    __syncthreads();
    int32_t need_b = need_c, give_b = give_c;
    int64_t add_b = add_c;
    for (int w = 0; w < W; ++w) {
      if (w < wave) {
        need_b = sat(need_b, need_s[w]);
        give_b = sat(give_b, give_s[w]);
        add_b += add_s[w];
      }
      need_c = sat(need_c, need_s[w]);
      give_c = sat(give_c, give_s[w]);
      add_c += add_s[w];
    }
    old_end = end_s;
    const int64_t add_e = add_b + add_i;  // with this list's
    const bool room = add == 0 || add_e <= a.slot_capacity;
    const bool ok = fits && room && (need == 0 || sat(need_b, need_i) <= count);
    refused |= !ok;
    if (ok && need > 0) atomicMax(&taken_s, sat(need_b, need_i));
    const int64_t len = !in ? 0 : ok ? will : had;
    const int64_t len_i = pg_wave_scan(len, lane, sum);
    if (lane == 63) len_s[wave] = len_i;
    __syncthreads();
    int64_t len_b = len_c;
    for (int w = 0; w < W; ++w) {
      if (w < wave) len_b += len_s[w];
      len_c += len_s[w];
    }
    if (in) {
      const int32_t pos = ok ? (int32_t)((uint32_t)(head + need_b + need_i - need) % (uint32_t)N) : -1;
      const int32_t go = sat(give_b, give_i);
      a.offsets_out[r + 1] = base + len_b + len_i;
      a.slot_offsets[r + 1] = add_e;
      if constexpr (SMALL) {
        had_s[r] = had;
        pos_s[r] = pos;
        keep_s[r] = (int32_t)want;
        go_s[r + 1] = go;
        so_s[r + 1] = (int32_t)min(add_e, (int64_t)kPgSmallSlots + 1);
      } else {
        ws.had[r] = had;
        ws.pos[r] = pos;
        ws.keep[r] = (int32_t)min(want, (int64_t)a.max_pages);
        ws.give[r + 1] = go;
      }
    }
  }
  if (refused) report_range(a.g);
  __syncthreads();
  const int32_t taken = taken_s;
  const int32_t given = min(give_c, N - count);  // (more: the ring's pages and the lists' overlap)
  const int32_t tail = (int32_t)((uint32_t)(head + count) % (uint32_t)N);
  if (tid == 0) {
    a.offsets_out[0] = base;
    a.slot_offsets[0] = 0;
    a.free_out[0] = (uint32_t)(head + taken) % (uint32_t)N;
    a.free_out[1] = count - taken + given;
    if (give_c > given) report_range(a.g);
    if constexpr (SMALL) {
      go_s[0] = so_s[0] = 0;
    } else {
      ws.give[0] = 0;
      ws.tail[0] = tail;
      ws.tail[1] = given;
    }
  }
  if constexpr (SMALL) {
    __syncthreads();
    const int32_t total = (int32_t)min(add_c, a.slot_capacity);
    for (int32_t j = tid; j < total; j += kPgScan) {
      const int32_t r = pg_bisect(0, R - 1, [&](int32_t i) { return (int64_t)so_s[i]; }, j);
      const int32_t row = had_s[r] + (j - so_s[r]);
      a.slots[j] = pg_slot(a, r, row, had_s[r], pos_s[r]);
    }
    for (int32_t i = tid; i < given; i += kPgScan) {
      const int32_t r = pg_bisect(0, R - 1, [&](int32_t q) { return (int64_t)go_s[q]; }, i);
      a.ring[(uint32_t)(tail + i) % (uint32_t)N] =
          a.table[(int64_t)r * a.max_pages + keep_s[r] + (i - go_s[r])];
    }
  }
}

// The last list r < R with first(r) <= x, by a wave: 64 lists' ends to a step.
template <typename F>
__device__ __forceinline__ int32_t pg_find(int32_t R, F first, int64_t x, int lane) {
  int32_t u = 0;
  for (int32_t n = R;;) {
    const int32_t step = (n + 63) / 64;
    const int64_t i = (int64_t)u + (int64_t)lane * step + step - 1;
    const bool past = i >= R || first((int32_t)i + 1) > x;
    u += (int32_t)__popcll(__ballot(!past)) * step;
    if (step == 1) break;
    n = step;
  }
  return min(u, R - 1);
}

// Slots, table entries and the pages given back, 64 at a time to a wave.
__global__ __launch_bounds__(kPgThreads) void page_slots_kernel(PageResizeArgs a) {
  const PgLists ws = pg_lists(a.ws, a.lists);
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * (kPgThreads / 64) + (threadIdx.x >> 6);
  const int64_t waves = (int64_t)gridDim.x * (kPgThreads / 64);
  const int32_t R = a.lists;
  const auto so = [&](int32_t r) { return a.slot_offsets[r]; };
  const auto go = [&](int32_t r) { return (int64_t)ws.give[r]; };
  const int64_t total = min(a.slot_offsets[R], a.slot_capacity);
  // a run of the slots for each wave
  const int64_t per = ((total + waves - 1) / waves + 63) / 64 * 64;
  const int64_t j0 = wave * per, j1 = min(total, j0 + per);
  if (j0 < j1) {
    const int32_t ra = pg_find(R, so, j0, lane), rb = pg_find(R, so, j1 - 1, lane);
    for (int64_t j = j0 + lane; j < j1; j += 64) {
      const int32_t r = pg_bisect(ra, rb, so, j);
      const int32_t had = ws.had[r];
      a.slots[j] = pg_slot(a, r, (int32_t)(had + (j - so(r))), had, ws.pos[r]);
    }
  }
  const int32_t tail = ws.tail[0], given = ws.tail[1];
  for (int64_t i = wave * 64 + lane; i < given; i += waves * 64) {
    const int32_t r = pg_bisect(0, R - 1, go, i);
    a.ring[(uint32_t)(tail + i) % (uint32_t)a.num_pages] =
        a.table[(int64_t)r * a.max_pages + ws.keep[r] + (i - go(r))];
  }
}

certkv_status run_page_resize(const PageResizeArgs& a, hipStream_t s) {
  if (a.lists <= kPgScan && a.slot_capacity <= kPgSmallSlots) {
    CERTKV_LAUNCH("page_resize", (page_resize_kernel<true>), dim3(1), dim3(kPgScan), 0, s, a);
    return CERTKV_OK;
  }
  CERTKV_LAUNCH("page_resize", (page_resize_kernel<false>), dim3(1), dim3(kPgScan), 0, s, a);
  CERTKV_LAUNCH("page_slots", page_slots_kernel, dim3(4 * 256), dim3(kPgThreads), 0, s, a);
  return CERTKV_OK;
}

// ---- rows to slots --------------------------------------------------------------

// The pool's row of a slot for (layer, head); -1: none (refused rows, and numbers that are none
// of the pool's, which are reported).
__device__ __forceinline__ int64_t pg_row(const PageArgs& a, int32_t slot, int l, int h) {
  if (slot < 0) return -1;
  const int32_t id = slot >> a.lp;
  if (id >= a.num_pages) {
    report_range(a.g);
    return -1;
  }
  return l * a.s_layer + id * a.s_page + (slot & ((1 << a.lp) - 1)) * a.s_row + h * a.s_head;
}

// Eight dims of a row, as they are held in format F, from the source's values.
template <int F, typename T>
__device__ __forceinline__ void pg_store8(const Geo& g, const MxRaw<T>& x, int64_t at, uint8_t* rows,
                                          uint8_t* scales) {
  if constexpr (F != CERTKV_CACHE_BF16) {
    float y[8];
    x.values(y);
    mx_store8<F>(g, y, at, rows, scales);
  } else if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(rows + 2 * at) = x.a;
  } else {
    float y[8];
    x.values(y);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = f32_to_bf16_rne(y[2 * i]) | (uint32_t)f32_to_bf16_rne(y[2 * i + 1]) << 16;
    *reinterpret_cast<uint4*>(rows + 2 * at) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// D / 8 lanes to a row.  blockIdx.y: the layer; rows of a layer token by token, head by head.
template <int D, typename T, int F>
__global__ __launch_bounds__(kPgThreads) void page_write_kernel(PageWriteArgs a) {
  constexpr int LPR = D / 8, RPS = kPgThreads / LPR;
  const Geo& g = a.p.g;
  const int l = blockIdx.y, ci = threadIdx.x % LPR;
  const T* ks = static_cast<const T*>(a.k.ptr) + l * a.k.s_layer + ci * 8;
  const T* vs = static_cast<const T*>(a.v.ptr) + l * a.v.s_layer + ci * 8;
  const uint32_t H = (uint32_t)g.H, rows = (uint32_t)(a.tokens * g.H);
  const int64_t total = a.slot_offsets[a.p.lists];
  for (uint32_t x = blockIdx.x * RPS + threadIdx.x / LPR; x < rows; x += gridDim.x * RPS) {
    const uint32_t tk = x / H, h = x % H;
    int64_t j = tk;  // its slot's place
    bool mine = j < total;
    if (a.tn) {
      const uint32_t b = tk / (uint32_t)a.tn, i = tk % (uint32_t)a.tn;
      const int64_t r = a.p.per_head ? unit_index(g, l, (int)b, (int)h) : b;
      j = a.slot_offsets[r] + i;
      mine = j < a.slot_offsets[r + 1];
    }
    if (!mine) continue;
    if (j < 0 || j >= a.slot_count) {
      report_range(g);
      continue;
    }
    const int64_t row = pg_row(a.p, a.slots[j], l, (int)h);
    if (row < 0) continue;
    MxRaw<T> kx, vx;
    kx.load(ks + tk * a.k.s_token + h * a.k.s_head);
    vx.load(vs + tk * a.v.s_token + h * a.v.s_head);
    pg_store8<F, T>(g, kx, row * D + ci * 8, a.p.k, a.p.k_scales);
    pg_store8<F, T>(g, vx, row * D + ci * 8, a.p.v, a.p.v_scales);
  }
}

template <int D, typename T>
static certkv_status launch_page_write(const PageWriteArgs& a, hipStream_t s) {
  const int64_t steps = (a.tokens * a.p.g.H + kPgThreads * 8 / D - 1) / (kPgThreads * 8 / D);
  const dim3 grid((unsigned)(steps < 8 * 256 ? steps : 8 * 256), (unsigned)a.p.g.L);
  switch (a.p.format) {
    case CERTKV_CACHE_MXFP8:
      CERTKV_LAUNCH("page_write", (page_write_kernel<D, T, CERTKV_CACHE_MXFP8>), grid,
                    dim3(kPgThreads), 0, s, a);
      break;
    case CERTKV_CACHE_MXFP4:
      CERTKV_LAUNCH("page_write", (page_write_kernel<D, T, CERTKV_CACHE_MXFP4>), grid,
                    dim3(kPgThreads), 0, s, a);
      break;
    default:
      CERTKV_LAUNCH("page_write", (page_write_kernel<D, T, CERTKV_CACHE_BF16>), grid,
                    dim3(kPgThreads), 0, s, a);
  }
  return CERTKV_OK;
}

certkv_status run_page_write(const PageWriteArgs& a, hipStream_t s) {
  if (a.dtype == CERTKV_BF16)
    return a.p.g.D == 128 ? launch_page_write<128, uint16_t>(a, s)
                          : launch_page_write<64, uint16_t>(a, s);
  return a.p.g.D == 128 ? launch_page_write<128, float>(a, s) : launch_page_write<64, float>(a, s);
}

// Rows of RB bytes (and SB of scales, 0 for bf16) as they are held.
template <int RB, int SB>
__global__ __launch_bounds__(kPgThreads) void page_adopt_kernel(PageAdoptArgs a) {
  constexpr int LPR = RB / 16, RPS = kPgThreads / LPR;
  const int ci = threadIdx.x % LPR;
  const int64_t total = min(min(a.slot_offsets[a.p.lists], a.rows), a.slot_count);
  if (a.slot_offsets[a.p.lists] > total && threadIdx.x == 0) report_range(a.p.g);
  for (int64_t j = (int64_t)blockIdx.x * RPS + threadIdx.x / LPR; j < total;
       j += (int64_t)gridDim.x * RPS) {
    const int64_t row = pg_row(a.p, a.slots[j], 0, 0);
    if (row < 0) continue;
    reinterpret_cast<uint4*>(a.p.k + row * RB)[ci] = reinterpret_cast<const uint4*>(a.k + j * RB)[ci];
    reinterpret_cast<uint4*>(a.p.v + row * RB)[ci] = reinterpret_cast<const uint4*>(a.v + j * RB)[ci];
    if constexpr (SB > 0) {
      using S = typename std::conditional<SB == 4, uint32_t, uint16_t>::type;
      if (ci == 0) {
        reinterpret_cast<S*>(a.p.k_scales)[row] = reinterpret_cast<const S*>(a.k_scales)[j];
        reinterpret_cast<S*>(a.p.v_scales)[row] = reinterpret_cast<const S*>(a.v_scales)[j];
      }
    }
  }
}

template <int D>
static certkv_status launch_page_adopt(const PageAdoptArgs& a, hipStream_t s) {
  const int64_t step = kPgThreads / (mx_row_bytes(a.p.format, D) / 16);
  const int64_t steps = (a.rows + step - 1) / step;
  const dim3 grid((unsigned)(steps < 8 * 256 ? steps : 8 * 256));
  switch (a.p.format) {
    case CERTKV_CACHE_MXFP8:
      CERTKV_LAUNCH("page_adopt", (page_adopt_kernel<D, D / 32>), grid, dim3(kPgThreads), 0, s, a);
      break;
    case CERTKV_CACHE_MXFP4:
      CERTKV_LAUNCH("page_adopt", (page_adopt_kernel<D / 2, D / 32>), grid, dim3(kPgThreads), 0, s, a);
      break;
    default:
      CERTKV_LAUNCH("page_adopt", (page_adopt_kernel<2 * D, 0>), grid, dim3(kPgThreads), 0, s, a);
  }
  return CERTKV_OK;
}

certkv_status run_page_adopt(const PageAdoptArgs& a, hipStream_t s) {
  return a.p.g.D == 128 ? launch_page_adopt<128>(a, s) : launch_page_adopt<64>(a, s);
}

// ---- rows out of their pages ------------------------------------------------------

// Eight dims of row `row` of the pool as bf16.
template <int F, int D>
__device__ __forceinline__ uint4 pg_load8(const uint8_t* rows, const uint8_t* scales, int64_t row,
                                          int ci) {
  if constexpr (F == CERTKV_CACHE_BF16) {
    const MxU4 v = __builtin_nontemporal_load(reinterpret_cast<const MxU4*>(rows + row * (2 * D)) + ci);
    return make_uint4(v[0], v[1], v[2], v[3]);
  } else {
    uint2 c = make_uint2(0u, 0u);
    if constexpr (F == CERTKV_CACHE_MXFP8)
      c = reinterpret_cast<const uint2*>(rows + row * D)[ci];
    else
      c.x = reinterpret_cast<const uint32_t*>(rows + row * (D / 2))[ci];
    const uint32_t x = scales[row * (D / kMxBlock) + ci / 4];
    if (x == 255u) return make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    return mx_decode8<F>(c, mx_scale(x));
  }
}

template <bool F32>
__device__ __forceinline__ void pg_put8(void* out, int64_t at, uint4 v) {
  if constexpr (F32) {
    MxF4* o = reinterpret_cast<MxF4*>(static_cast<float*>(out) + at);
    __builtin_nontemporal_store((MxF4){bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)}, o);
    __builtin_nontemporal_store((MxF4){bf16_lo(v.z), bf16_hi(v.z), bf16_lo(v.w), bf16_hi(v.w)}, o + 1);
  } else {
    __builtin_nontemporal_store((MxU4){v.x, v.y, v.z, v.w},
                                reinterpret_cast<MxU4*>(static_cast<uint16_t*>(out) + at));
  }
}

// A run of a layer's rows (tokens by heads; heads' lists: all rows) for each workgroup, D / 8
// lanes to a row; the list of the run's first row by a 64-way search, the next ones by stepping
// on.
template <int F, int D, bool F32>
__global__ __launch_bounds__(kPgThreads) void page_read_kernel(PageReadArgs a) {
  constexpr int LPR = D / 8, RPS = kPgThreads / LPR;
  const PageArgs& p = a.p;
  const int l = blockIdx.y, ci = threadIdx.x % LPR, lane = threadIdx.x & 63;
  const uint32_t H = p.per_head ? 1u : (uint32_t)p.g.H;
  const int64_t base = p.offsets[0], all = p.offsets[p.lists] - base;
  const int64_t tokens = min(all, a.rows);
  if (all > a.rows && threadIdx.x == 0 && blockIdx.x == 0) report_range(p.g);
  const int64_t rows = tokens * H;
  const int64_t per = ((rows + gridDim.x - 1) / gridDim.x + RPS - 1) / RPS * RPS;
  const int64_t x0 = blockIdx.x * per, x1 = min(rows, x0 + per);
  if (x0 >= x1) return;
  const auto first = [&](int32_t r) { return p.offsets[r] - base; };
  int32_t r = pg_find(p.lists, first, x0 / H, lane);
  int64_t start = first(r), end = first(r + 1);
  const int64_t out0 = p.per_head ? 0 : (int64_t)l * a.rows * H;
  for (int64_t x = x0 + threadIdx.x / LPR; x < x1; x += RPS) {
    const int64_t tk = x / H;
    const int h = (int)(x - tk * H);
    while (tk >= end && r + 1 < p.lists) {
      ++r;
      start = end;
      end = first(r + 1);
    }
    const int64_t i = tk - start, pi = i >> p.lp;
    int32_t id = -1;
    if (i >= 0 && pi < p.max_pages) id = p.table[(int64_t)r * p.max_pages + pi];
    if ((uint32_t)id >= (uint32_t)p.num_pages) {  // (the caller's numbers)
      report_range(p.g);
      continue;
    }
    const int64_t row = pg_row(p, (id << p.lp) + (int32_t)(i & ((1 << p.lp) - 1)), l, h);
    const int64_t at = (out0 + x) * D + ci * 8;
    if (a.k) pg_put8<F32>(a.k, at, pg_load8<F, D>(p.k, p.k_scales, row, ci));
    if (a.v) pg_put8<F32>(a.v, at, pg_load8<F, D>(p.v, p.v_scales, row, ci));
  }
}

template <int F, int D>
static certkv_status launch_page_read(const PageReadArgs& a, hipStream_t s) {
  const int64_t rows = a.rows * (a.p.per_head ? 1 : a.p.g.H), step = kPgThreads * 8 / D;
  const int64_t steps = (rows + step - 1) / step;
  const int layers = a.p.per_head ? 1 : a.p.g.L;
  const int64_t most = 8 * 256;
  const dim3 grid((unsigned)(steps < most ? steps : most), (unsigned)layers);
  if (a.f32)
    CERTKV_LAUNCH("page_read", (page_read_kernel<F, D, true>), grid, dim3(kPgThreads), 0, s, a);
  else
    CERTKV_LAUNCH("page_read", (page_read_kernel<F, D, false>), grid, dim3(kPgThreads), 0, s, a);
  return CERTKV_OK;
}

template <int D>
static certkv_status launch_page_read_f(const PageReadArgs& a, hipStream_t s) {
  return a.p.format == CERTKV_CACHE_MXFP8   ? launch_page_read<CERTKV_CACHE_MXFP8, D>(a, s)
         : a.p.format == CERTKV_CACHE_MXFP4 ? launch_page_read<CERTKV_CACHE_MXFP4, D>(a, s)
                                            : launch_page_read<CERTKV_CACHE_BF16, D>(a, s);
}

certkv_status run_page_read(const PageReadArgs& a, hipStream_t s) {
  return a.p.g.D == 128 ? launch_page_read_f<128>(a, s) : launch_page_read_f<64>(a, s);
}

}  // namespace certkv
