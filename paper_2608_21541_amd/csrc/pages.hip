// The paged cache's tables and slots, and rows written to, copied to and read from its pages.
#include "pages.h"

namespace certkv {

constexpr int kPgThreads = 256;
constexpr int kPgScan = 2048;      // lists that a workgroup scans by itself
constexpr int kPgBlock = 1024;     // of more, lists to a workgroup
// Pages of a lane that are given back at a time.  (65536 pages of 8 lists of 64, with events, one wave
// 695 us and with 16 123, eight waves 26; 131072 of 64 lists of 250, four waves 413 and 76.)
constexpr int kPgGives = 16;

// ---- tables and slots ---------------------------------------------------------
//
// Of list r: had_r rows, will_r = max(0, had_r + change_r), a page for every `page` rows.  With
// need_r = pages(will) - pages(had) where that is positive and give_r where it is negative, list
// r takes the ring's places head + sum_{i<r} need_i on and gives its last pages to the places
// behind the free ones, from sum_{i<r} give_i on; its slots stand from sum_{i<r} max(0, change_i)
// on.  Lists are refused in order, so that a list that takes pages has none that is refused for
// their number before it, and the places taken have no gap.  (Refused for its own length: need
// counts as 0.)
//
// The sums are a scan of the lists; the slots and table entries follow from them.  Up to 2048 lists
// one launch does both: few slots by one workgroup, many by workgroups that each scan all lists and
// take a share of the slots.  More lists: the sums of blocks of them, then a scan of each block
// behind those, then the slots.
// Bound by latency: a launch, loads in turn (offsets, then entries of the table or ring) and the
// scan.  64 lists that get a row each 3.5 us (a call 7.0, the host's); 1024 lists of which an
// eighth each end, begin, grow by four rows and lose three, 371k slots 11 us, in two launches 15;
// 256 empty lists that get 3.36M rows 14 us, in two launches 22, the scan alone 6; lists that get a
// row each, with events, 2048 of them 22 us (three launches 33), 16384 30, 65536 32 (a scan of all by
// one workgroup 102 and 357).

// What the second part needs of each list, in the workspace or LDS; and, of many lists, the sums of
// each block of kPgBlock.
struct PgLists {
  int32_t* had;
  int32_t* pos;   // place of the ring of its first new page, or -1: refused
  int32_t* keep;  // pages that are left to a list that gives some
  int32_t* give;  // [lists + 1] sums of the pages given
  int32_t* tail;  // place of the ring where they go, how many, first free place, free pages
  int64_t* base;  // offsets[0]
  int32_t* need_b;   // of a block: pages needed and given, the last place of the ring taken,
  int32_t* give_b;
  int32_t* taken_b;
  int64_t* add_b;    // rows appended, and rows after the step
  int64_t* len_b;
};
constexpr int64_t pg_pad(int64_t n) { return (n + 63) & ~(int64_t)63; }
__host__ __device__ constexpr int64_t pg_blocks(int64_t lists) { return (lists + kPgBlock - 1) / kPgBlock; }
__host__ __device__ static inline PgLists pg_lists(int32_t* ws, int64_t lists) {
  const int64_t nb = pg_pad(pg_blocks(lists));
  PgLists x;
  x.tail = ws;
  x.base = reinterpret_cast<int64_t*>(ws + 8);
  x.had = ws + 64;
  x.pos = x.had + pg_pad(lists);
  x.keep = x.pos + pg_pad(lists);
  x.give = x.keep + pg_pad(lists);
  x.need_b = x.give + pg_pad(lists + 1);
  x.give_b = x.need_b + nb;
  x.taken_b = x.give_b + nb;
  x.add_b = reinterpret_cast<int64_t*>(x.taken_b + nb);
  x.len_b = x.add_b + nb;
  return x;
}
size_t page_resize_ws(int64_t lists) {
  return (size_t)(64 + 3 * pg_pad(lists) + pg_pad(lists + 1) + 7 * pg_pad(pg_blocks(lists))) * sizeof(int32_t);
}

// x of the lane that a data-parallel step takes it from, 0 where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ int32_t pg_dpp(int32_t x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t pg_dpp(int64_t x) {
  const uint32_t lo = (uint32_t)pg_dpp<CTRL, ROWS>((int32_t)x);
  return (int64_t)((uint64_t)(uint32_t)pg_dpp<CTRL, ROWS>((int32_t)(x >> 32)) << 32 | lo);
}
// Sums up to and with the lane's own: within rows of 16 lanes, then of the rows before.
template <typename T, typename F>
__device__ __forceinline__ T pg_wave_scan(T x, F add) {
  x = add(x, pg_dpp<0x111, 0xf>(x));  // one lane up, two, four, eight
  x = add(x, pg_dpp<0x112, 0xf>(x));
  x = add(x, pg_dpp<0x114, 0xf>(x));
  x = add(x, pg_dpp<0x118, 0xf>(x));
  x = add(x, pg_dpp<0x142, 0xa>(x));  // the last of the row before, to rows 1 and 3
  return add(x, pg_dpp<0x143, 0xc>(x));  // the last of the first half, to the second
}

// The number of page pi of list r, which had `held` pages and has its new ones from place pos of
// the ring on; -1 for one that is none of the pool's.  first: the caller's row is the page's first,
// and writes a new page's table entry.
__device__ __forceinline__ int32_t pg_page(const PageResizeArgs& a, int64_t r, int32_t pi, int32_t held,
                                           int32_t pos, bool first) {
  int32_t* entry = a.table + r * a.max_pages + pi;
  int32_t id;
  if (pi < held) {
    id = *entry;
  } else {
    const uint32_t at = (uint32_t)(pos + (pi - held)), n = (uint32_t)a.num_pages;  // below 2 n
    id = a.ring[at < n ? at : at - n];
    if (first) *entry = id;
  }
  if ((uint32_t)id >= (uint32_t)a.num_pages) {  // (the caller's numbers)
    report_range(a.g);
    return -1;
  }
  return id;
}
// The slot of row `row` of list r, which has `had` rows and new pages from place pos on (-1: it is
// refused).
__device__ __forceinline__ int32_t pg_slot(const PageResizeArgs& a, int64_t r, int32_t row,
                                           int32_t had, int32_t pos) {
  if (pos < 0) return -1;
  const int32_t mask = (1 << a.lp) - 1, in = row & mask;
  const int32_t id = pg_page(a, r, row >> a.lp, (had + mask) >> a.lp, pos, in == 0);
  return id < 0 ? -1 : (id << a.lp) + in;
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

// Slots j .. j + 3 of those before `end`, from the lists' sums: so(r) the first of list r's,
// had(r) and pos(r) as pg_slot takes them; the lists of j and of the last are in [ra, rb].
template <typename S, typename A, typename B>
__device__ __forceinline__ void pg_slots4(const PageResizeArgs& a, int64_t j, int64_t end, int32_t ra,
                                          int32_t rb, S so, A had, B pos) {
  int32_t r = pg_bisect(ra, rb, so, j), h = had(r), p = pos(r), out[4];
  int64_t first = so(r), next = so(r + 1);
  if (j + 4 <= next && j + 4 <= end) {  // one list's: rows of one page, or of two
    const int32_t mask = (1 << a.lp) - 1, held = (h + mask) >> a.lp, row = (int32_t)(h + (j - first));
    const int32_t in = row & mask, pi = row >> a.lp;
    int32_t id = -1, id2 = -1;
    if (p >= 0) {
      id = id2 = pg_page(a, r, pi, held, p, in == 0);
      if (in + 3 > mask) id2 = pg_page(a, r, pi + 1, held, p, true);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int32_t x = in + i, of = x > mask ? id2 : id;
      out[i] = of < 0 ? -1 : (of << a.lp) + (x & mask);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i > 0 && j + i >= next && j + i < end) {
        r = pg_bisect(r + 1, rb, so, j + i);
        first = so(r), next = so(r + 1);
        h = had(r), p = pos(r);
      }
      out[i] = j + i < end ? pg_slot(a, r, (int32_t)(h + (j + i - first)), h, p) : -1;
    }
  }
  if (j + 4 <= end && ((uintptr_t)(a.slots + j) & 15u) == 0) {
    *reinterpret_cast<int4*>(a.slots + j) = make_int4(out[0], out[1], out[2], out[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (j + i < end) a.slots[j + i] = out[i];
  }
}

// What a list of rows [first, end) of the offsets asks for.
struct PgStep {
  int32_t had, need, give, add;
  int64_t will;
  bool fits;
};
__device__ __forceinline__ PgStep pg_step(const PageResizeArgs& a, int64_t first, int64_t end, int32_t change) {
  const int32_t N = a.num_pages, mask = (1 << a.lp) - 1;
  const int64_t most_rows = (int64_t)a.max_pages << a.lp, n = end - first;
  PgStep x;
  x.had = (int32_t)(n < 0 ? 0 : n < most_rows ? n : most_rows);
  x.will = max((int64_t)x.had + change, (int64_t)0);
  const int32_t held = (x.had + mask) >> a.lp;
  const int64_t want = (x.will + mask) >> a.lp;
  x.fits = want <= a.max_pages;
  x.need = want > held && x.fits ? (int32_t)min(want - held, (int64_t)N + 1) : 0;
  x.give = want < held ? min(held - (int32_t)want, N + 1) : 0;
  x.add = change > 0 ? change : 0;
  return x;
}

// The sum of a workgroup's values, to all of them.  part: W words of LDS.
template <int W, typename T, typename F>
__device__ __forceinline__ T pg_total(T x, F add, T* part) {
  x = pg_wave_scan(x, add);
  if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = x;
  __syncthreads();
  T t = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) t = add(t, part[w]);
  __syncthreads();
  return t;
}

// Many lists: the sums of a block of them.
__global__ __launch_bounds__(kPgThreads) void page_blocks_kernel(PageResizeArgs a) {
  __shared__ int32_t part[kPgThreads / 64];
  __shared__ int64_t part64[kPgThreads / 64];
  const int32_t N = a.num_pages;
  const PgLists ws = pg_lists(a.ws, a.lists);
  const auto sat = [N](int32_t x, int32_t y) { return min(x + y, N + 1); };
  int32_t need = 0, give = 0;
  int64_t add = 0;
#pragma unroll
  for (int k = 0; k < kPgBlock / kPgThreads; ++k) {
    const int64_t r = (int64_t)blockIdx.x * kPgBlock + k * kPgThreads + threadIdx.x;
    if (r >= a.lists) continue;
    const PgStep x = pg_step(a, a.offsets[r], a.offsets[r + 1], a.change[r]);
    need = sat(need, x.need);
    give = sat(give, x.give);
    add += x.add;
  }
  need = pg_total<kPgThreads / 64>(need, sat, part);
  give = pg_total<kPgThreads / 64>(give, sat, part);
  add = pg_total<kPgThreads / 64>(add, [](int64_t x, int64_t y) { return x + y; }, part64);
  if (threadIdx.x == 0) {
    ws.need_b[blockIdx.x] = need;
    ws.give_b[blockIdx.x] = give;
    ws.add_b[blockIdx.x] = add;
  }
}

// W waves scan K lists a lane at a time.  PART: 0, this is the only workgroup and does all; 1, every
// workgroup scans, the first writes the sums; 2, each scans a block behind those of
// page_blocks_kernel, for page_slots_kernel.
template <int W, int K, int PART>
__global__ __launch_bounds__(64 * W) void page_resize_kernel(PageResizeArgs a) {
  constexpr int NT = 64 * W, STEP = NT * K, HELD = PART == 2 ? 1 : STEP;
  __shared__ int32_t need_s[W], give_s[W], taken_s;
  __shared__ int64_t add_s[W], len_s[W], end_s;
  __shared__ int32_t had_s[HELD], pos_s[HELD], keep_s[HELD], go_s[HELD + 1], so_s[HELD + 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t R = a.lists, N = a.num_pages, mask = (1 << a.lp) - 1;
  const int64_t base = a.offsets[0];
  const int32_t head = (int32_t)((uint64_t)a.free[0] % (uint64_t)N);
  const int64_t free_pages = a.free[1];
  const int32_t count = (int32_t)(free_pages < 0 ? 0 : free_pages < N ? free_pages : N);
  const PgLists ws = pg_lists(a.ws, R);
  const bool tells = PART != 1 || blockIdx.x == 0;
  const int32_t begin = PART == 2 ? (int32_t)blockIdx.x * STEP : 0;
  // sums of pages stop at N + 1, more than there are
  const auto sat = [N](int32_t x, int32_t y) { return min(x + y, N + 1); };
  const auto sum = [](int64_t x, int64_t y) { return x + y; };
  int32_t need_c = 0, give_c = 0;
  int64_t add_c = 0, len_c = 0, old_end = PART == 2 ? a.offsets[begin] : base;
  bool refused = free_pages != count;
  if (tid == 0) taken_s = 0;
  if constexpr (PART == 2) {
    static_assert(STEP == kPgBlock, "a workgroup's lists");
    for (int32_t i = tid; i < (int32_t)blockIdx.x; i += NT) {
      need_c = sat(need_c, ws.need_b[i]);
      give_c = sat(give_c, ws.give_b[i]);
      add_c += ws.add_b[i];
    }
    need_c = pg_total<W>(need_c, sat, need_s);
    give_c = pg_total<W>(give_c, sat, give_s);
    add_c = pg_total<W>(add_c, sum, add_s);
  }
  for (int32_t r0 = begin; r0 < (PART == 2 ? min(R, begin + STEP) : R); r0 += STEP) {
    const int32_t r = r0 + tid * K;
    int32_t had[K], need[K], give[K], add[K];
    int64_t will[K];
    bool fits[K];
    int32_t need_t = 0, give_t = 0;
    int64_t add_t = 0;
    // (offsets_out may be offsets: the step before has written this one's first)
    int64_t first = tid == 0 ? old_end : r < R ? a.offsets[r] : 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool in = r + k < R;
      const int64_t end = in ? a.offsets[r + k + 1] : first;
      const PgStep x = pg_step(a, first, end, in ? a.change[r + k] : 0);
      if (end - first != x.had) report_range(a.g);  // (the caller's numbers)
      first = end;
      had[k] = x.had, will[k] = x.will, fits[k] = x.fits;
      need[k] = x.need, give[k] = x.give, add[k] = x.add;
      need_t = sat(need_t, need[k]);
      give_t = sat(give_t, give[k]);
      add_t += add[k];
    }
    const int32_t need_i = pg_wave_scan(need_t, sat), give_i = pg_wave_scan(give_t, sat);
    const int64_t add_i = pg_wave_scan(add_t, sum);
    if (lane == 63) {
      need_s[wave] = need_i;
      give_s[wave] = give_i;
      add_s[wave] = add_i;
    }
    if (tid == NT - 1) end_s = first;
    __syncthreads();
    int32_t need_b = need_c, give_b = give_c;
    int64_t add_b = add_c;
#pragma unroll
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
    // of the lists before the lane's (not its sums less its own: they may have stopped)
    const int32_t need_l = __shfl_up(need_i, 1, 64), give_l = __shfl_up(give_i, 1, 64);
    int32_t need_e = sat(need_b, lane ? need_l : 0), give_e = sat(give_b, lane ? give_l : 0);
    int64_t add_e = add_b + add_i - add_t, len_t = 0, len[K];
    int32_t pos[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int32_t need_n = sat(need_e, need[k]);
      add_e += add[k];
      const bool ok = fits[k] && (add[k] == 0 || add_e <= a.slot_capacity) &&
                      (need[k] == 0 || need_n <= count);
      refused |= !ok;
      if (ok && need[k] > 0) atomicMax(&taken_s, need_n);
      pos[k] = ok ? (int32_t)((uint32_t)(head + need_e) % (uint32_t)N) : -1;
      need_e = need_n;
      len[k] = r + k >= R ? 0 : ok ? will[k] : had[k];
      len_t += len[k];
    }
    const int64_t len_i = pg_wave_scan(len_t, sum);
    if (lane == 63) len_s[wave] = len_i;
    __syncthreads();
    int64_t len_b = len_c;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (w < wave) len_b += len_s[w];
      len_c += len_s[w];
    }
    len_b += len_i - len_t;
    add_e = add_b + add_i - add_t;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      add_e += add[k];
      len_b += len[k];
      give_e = sat(give_e, give[k]);
      if (r + k >= R) continue;
      if (tells) {
        if (PART != 2) a.offsets_out[r + k + 1] = base + len_b;
        a.slot_offsets[r + k + 1] = add_e;
      }
      const int32_t keep = (int32_t)min((will[k] + mask) >> a.lp, (int64_t)a.max_pages);
      if constexpr (PART != 2) {
        had_s[r + k] = had[k];
        pos_s[r + k] = pos[k];
        keep_s[r + k] = keep;
        go_s[r + k + 1] = give_e;
        so_s[r + k + 1] = (int32_t)min(add_e, (int64_t)INT32_MAX);
      } else {
        ws.had[r + k] = had[k];
        ws.pos[r + k] = pos[k];
        ws.keep[r + k] = keep;
        ws.give[r + k + 1] = give_e;
      }
    }
  }
  if (refused) report_range(a.g);
  __syncthreads();
  const int32_t taken = taken_s;
  const int32_t given = min(give_c, N - count);  // (more: the ring's pages and the lists' overlap)
  const int32_t tail = (int32_t)((uint32_t)(head + count) % (uint32_t)N);
  if (PART == 2 && tid == 0) {
    ws.taken_b[blockIdx.x] = taken;
    ws.len_b[blockIdx.x] = len_c;
    if (blockIdx.x == 0) {
      a.slot_offsets[0] = 0;
      ws.give[0] = 0;
    }
    if (blockIdx.x == gridDim.x - 1) {
      ws.tail[0] = tail, ws.tail[1] = given;
      ws.tail[2] = head, ws.tail[3] = count;
      ws.base[0] = base;
      if (give_c > given) report_range(a.g);
    }
  } else if (tid == 0) {
    if (tells) {
      a.offsets_out[0] = base;
      a.slot_offsets[0] = 0;
      a.free_out[0] = (uint32_t)(head + taken) % (uint32_t)N;
      a.free_out[1] = count - taken + given;
      if (give_c > given) report_range(a.g);
    }
    go_s[0] = so_s[0] = 0;
  }
  if constexpr (PART != 2) {
    __syncthreads();
    const uint32_t total = (uint32_t)min(add_c, a.slot_capacity);
    const uint32_t at = (PART == 1 ? blockIdx.x : 0) * NT + tid, step = (PART == 1 ? gridDim.x : 1) * NT;
    const auto so = [&](int32_t i) { return (int64_t)so_s[i]; };
    if (PART == 0 && total <= NT) {  // (a row or few to a list: a slot to a lane)
      if (at < total) {
        const int32_t r = pg_bisect(0, R - 1, so, at);
        a.slots[at] = pg_slot(a, r, had_s[r] + (int32_t)(at - so_s[r]), had_s[r], pos_s[r]);
      }
    } else {
      // a run of the slots for each wave
      const int64_t wgs = PART == 1 ? gridDim.x : 1, waves = wgs * W;
      const int64_t w = (PART == 1 ? blockIdx.x : 0) * (int64_t)W + wave;
      const int64_t per = ((int64_t)total + 256 * waves - 1) / (256 * waves) * 256;
      const int64_t j0 = w * per, j1 = min((int64_t)total, j0 + per);
      if (j0 < j1) {
        const int32_t ra = pg_find(R, so, j0, lane), rb = pg_find(R, so, j1 - 1, lane);
        for (int64_t j = j0 + 4 * lane; j < j1; j += 256)
          pg_slots4(a, j, j1, ra, rb, so, [&](int32_t r) { return had_s[r]; },
                    [&](int32_t r) { return pos_s[r]; });
      }
    }
    // Pages given back, in runs of a wave's, all of a run in flight.  The run's lists are found first:
    // mostly one (a long list that ends), else each lane searches between them.
    constexpr int GIVES = PART == 0 ? kPgGives : 1, RUN = 64 * GIVES;
    const auto go = [&](int32_t i) { return (int64_t)go_s[i]; };
    for (int64_t i0 = ((PART == 1 ? blockIdx.x : 0) * (int64_t)W + wave) * RUN; i0 < given; i0 += (int64_t)step * GIVES) {
      const int32_t end = (int32_t)min(i0 + RUN, (int64_t)given) - 1;
      const int32_t ra = pg_find(R, go, i0, lane), rb = pg_find(R, go, end, lane);
      int32_t id[GIVES];
#pragma unroll
      for (int k = 0; k < GIVES; ++k) {
        const int32_t i = min((int32_t)i0 + 64 * k + lane, end);
        const int32_t r = ra == rb ? ra : pg_bisect(ra, rb, go, i);
        id[k] = a.table[(int64_t)r * a.max_pages + keep_s[r] + (i - go_s[r])];
      }
#pragma unroll
      for (int k = 0; k < GIVES; ++k) {
        const int32_t i = (int32_t)i0 + 64 * k + lane;
        const uint32_t to = (uint32_t)(tail + i);
        if (i <= end) a.ring[to < (uint32_t)N ? to : to - (uint32_t)N] = id[k];
      }
    }
  }
}

// The sums that a launch of many workgroups left beside the offsets that they read, in their place.
__global__ __launch_bounds__(kPgThreads) void page_sums_kernel(PageResizeArgs a, const int64_t* offsets,
                                                               const int64_t* free_state) {
  for (int32_t r = threadIdx.x; r <= a.lists; r += kPgThreads) a.offsets_out[r] = offsets[r];
  if (threadIdx.x < 2) a.free_out[threadIdx.x] = free_state[threadIdx.x];
}

// The new offsets of a block of lists, behind its sums' (and the ring's new state).
__device__ __forceinline__ void pg_offsets(const PageResizeArgs& a, const PgLists& ws, int32_t block,
                                           int64_t* part) {
  constexpr int W = kPgThreads / 64, K = kPgBlock / kPgThreads;
  const int tid = threadIdx.x;
  const auto sum = [](int64_t x, int64_t y) { return x + y; };
  const int64_t base = ws.base[0];
  if (block == 0) {
    int64_t taken = 0;
    for (int32_t i = tid; i < (int32_t)pg_blocks(a.lists); i += kPgThreads)
      taken = max(taken, (int64_t)ws.taken_b[i]);
    taken = pg_total<W>(taken, [](int64_t x, int64_t y) { return max(x, y); }, part);
    if (tid == 0) {
      a.offsets_out[0] = base;
      a.free_out[0] = (uint32_t)(ws.tail[2] + (int32_t)taken) % (uint32_t)a.num_pages;
      a.free_out[1] = ws.tail[3] - taken + ws.tail[1];
    }
  }
  int64_t before = base, len[K], mine = 0;
  const int32_t r = block * kPgBlock + tid * K;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    len[k] = 0;
    if (r + k < a.lists) {
      const int32_t had = ws.had[r + k];
      len[k] = ws.pos[r + k] < 0 ? had : max((int64_t)had + a.change[r + k], (int64_t)0);
    }
    mine += len[k];
  }
  int64_t s = 0;
  for (int32_t i = tid; i < block; i += kPgThreads) s += ws.len_b[i];
  before += pg_total<W>(s, sum, part);
  s = pg_wave_scan(mine, sum);
  if ((tid & 63) == 63) part[tid >> 6] = s;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w)
    if (w < tid >> 6) before += part[w];
  __syncthreads();
  before += s - mine;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    before += len[k];
    if (r + k < a.lists) a.offsets_out[r + k + 1] = before;
  }
}

// Offsets, slots, table entries and the pages given back, the slots 256 at a time to a wave.
__global__ __launch_bounds__(kPgThreads) void page_slots_kernel(PageResizeArgs a) {
  const PgLists ws = pg_lists(a.ws, a.lists);
  __shared__ int64_t part[kPgThreads / 64];
  // (by the last workgroups, whose share of few slots is none)
  for (int64_t i = (int64_t)gridDim.x - 1 - blockIdx.x; i < pg_blocks(a.lists); i += gridDim.x)
    pg_offsets(a, ws, (int32_t)i, part);
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * (kPgThreads / 64) + (threadIdx.x >> 6);
  const int64_t waves = (int64_t)gridDim.x * (kPgThreads / 64);
  const int32_t R = a.lists;
  const auto so = [&](int32_t r) { return a.slot_offsets[r]; };
  const auto go = [&](int32_t r) { return (int64_t)ws.give[r]; };
  const int64_t total = min(a.slot_offsets[R], a.slot_capacity);
  // a run of the slots for each wave, four of one place in a row to a lane
  const int64_t per = ((total + waves - 1) / waves + 255) / 256 * 256;
  const int64_t j0 = wave * per, j1 = min(total, j0 + per);
  if (j0 < j1) {
    const int32_t ra = pg_find(R, so, j0, lane), rb = pg_find(R, so, j1 - 1, lane);
    for (int64_t j = j0 + 4 * lane; j < j1; j += 256) {
      pg_slots4(a, j, j1, ra, rb, so, [&](int32_t r) { return ws.had[r]; },
                [&](int32_t r) { return ws.pos[r]; });
    }
  }
  const int32_t tail = ws.tail[0], given = ws.tail[1];
  for (int64_t i0 = wave * 64; i0 < given; i0 += waves * 64) {
    const int64_t i = min(i0 + lane, (int64_t)given - 1);
    const int32_t ra = pg_find(R, go, i0, lane), rb = pg_find(R, go, min(i0 + 63, (int64_t)given - 1), lane);
    const int32_t r = pg_bisect(ra, rb, go, i);
    a.ring[(uint32_t)(tail + i) % (uint32_t)a.num_pages] =
        a.table[(int64_t)r * a.max_pages + ws.keep[r] + (i - go(r))];
  }
}

// Slots that the scan's own workgroup fills in: in place more, where the sums of many workgroups
// wait for a launch of their own.  (In us, one workgroup and many: 250 lists of 8 rows each 10.0 and
// 9.9, of 16 12.2 and 9.6, of 64 16.5 and 9.2, in place 12.9 and 14.8; 1000 lists of 4 14.9 and 16.4,
// of 8 17 and 16.3, of 16 19.8 and 16.6, in place 15.1 and 19.)
static int64_t pg_small_slots(int32_t lists, bool in_place) {
  return in_place ? 16384 : lists <= 256 ? 2048 : 8192;
}

// And the pages that its lists may give back, whose number only the device knows: up to these few of a
// short step one wave moves them all (3.4 us for a row to each of 64 lists, four waves 3.9, eight 4.2,
// sixteen 6.3), of more eight waves (8192 pages of one list 23 us and 11, 65536 of eight 123 and 26,
// 524288 of 64 914 and 131; a grid of workgroups 14, but 6.4 for a row to each, in place 7.9).  Where
// the sums are a grid's anyhow, it is one for each 1024 of them (2048 lists that get a row each 11.7 us
// by 2 workgroups and by 256; 400 of them that end, 204800 pages, with events, 211 and 24).
constexpr int64_t kPgFewPages = 32768;

certkv_status run_page_resize(const PageResizeArgs& a, hipStream_t s) {
  const bool in_place = a.offsets_out == a.offsets || a.free_out == a.free;
  const int64_t held = (int64_t)a.lists * a.max_pages;
  if (a.lists <= 1024 && a.slot_capacity <= pg_small_slots(a.lists, in_place)) {
    const bool few = held <= kPgFewPages || a.num_pages <= kPgFewPages;
    if (few && a.lists <= 64 && a.slot_capacity <= 256)
      CERTKV_LAUNCH("page_resize", (page_resize_kernel<1, 1, 0>), dim3(1), dim3(64), 0, s, a);
    else if (few && a.lists <= 256 && a.slot_capacity <= 4096)
      CERTKV_LAUNCH("page_resize", (page_resize_kernel<4, 1, 0>), dim3(1), dim3(256), 0, s, a);
    else if (a.lists <= 256 && a.slot_capacity <= 4096)
      CERTKV_LAUNCH("page_resize", (page_resize_kernel<8, 1, 0>), dim3(1), dim3(512), 0, s, a);
    else
      CERTKV_LAUNCH("page_resize", (page_resize_kernel<16, 1, 0>), dim3(1), dim3(1024), 0, s, a);
    return CERTKV_OK;
  }
  if (a.lists <= kPgScan) {
    // (in place, the sums would be written while others read: they wait in the workspace)
    PageResizeArgs b = a;
    if (in_place) {
      b.offsets_out = reinterpret_cast<int64_t*>(a.ws);
      b.free_out = b.offsets_out + a.lists + 1;
    }
    // (of few slots, or of room for none, as where lists only shrink: by the pages given back)
    int64_t most = held < a.num_pages ? held : a.num_pages;
    if (most > 256 * 1024) most = 256 * 1024;
    const int64_t wgs = ((most > a.slot_capacity ? most : a.slot_capacity) + 1023) / 1024;
    const dim3 grid((unsigned)(wgs < 4 * 256 ? wgs : 4 * 256));
    if (a.lists <= 256)
      CERTKV_LAUNCH("page_resize", (page_resize_kernel<4, 1, 1>), grid, dim3(256), 0, s, b);
    else if (a.lists <= 1024)
      CERTKV_LAUNCH("page_resize", (page_resize_kernel<4, 4, 1>), grid, dim3(256), 0, s, b);
    else
      CERTKV_LAUNCH("page_resize", (page_resize_kernel<8, 4, 1>), grid, dim3(512), 0, s, b);
    if (in_place)
      CERTKV_LAUNCH("page_sums", page_sums_kernel, dim3(1), dim3(kPgThreads), 0, s, a, b.offsets_out,
                    b.free_out);
    return CERTKV_OK;
  }
  const dim3 blocks((unsigned)pg_blocks(a.lists));
  CERTKV_LAUNCH("page_blocks", page_blocks_kernel, blocks, dim3(kPgThreads), 0, s, a);
  CERTKV_LAUNCH("page_resize", (page_resize_kernel<16, 1, 2>), blocks, dim3(1024), 0, s, a);
  CERTKV_LAUNCH("page_slots", page_slots_kernel, dim3(8 * 256), dim3(kPgThreads), 0, s, a);
  return CERTKV_OK;
}

// ---- rows to slots --------------------------------------------------------------

// n / d for n < 2^31, by a product: with 2^(s-1) < d <= 2^s, n / d = (n + (n m >> 32)) >> s for
// m = floor(2^32 (2^s - d) / d) + 1.  (The hardware has no integer division.)
struct PgDiv {
  uint32_t m, s;
  explicit PgDiv(uint32_t d) : m(1), s(0) {
    if (d == 0) return;  // (not asked)
    while (((uint64_t)1 << s) < d) ++s;
    m = (uint32_t)((((((uint64_t)1 << s) - d) << 32) / d) + 1);
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (n + __umulhi(n, m)) >> s; }
};

// Row r of page id of the pool (the strides but the layer's are below 2^31).
__device__ __forceinline__ int64_t pg_place_of(const PageArgs& a, uint32_t id, uint32_t r, int l,
                                               uint32_t h) {
  return l * a.s_layer + (int64_t)((uint64_t)id * (uint32_t)a.s_page + (uint64_t)r * (uint32_t)a.s_row +
                                   (uint64_t)h * (uint32_t)a.s_head);
}

// The pool's row of a slot for (layer, head); -1: none (refused rows, and numbers that are none
// of the pool's, which are reported).
__device__ __forceinline__ int64_t pg_row(const PageArgs& a, int32_t slot, int l, uint32_t h) {
  if (slot < 0) return -1;
  const int32_t id = slot >> a.lp;
  if (id >= a.num_pages) {
    report_range(a.g);
    return -1;
  }
  return pg_place_of(a, id, (uint32_t)slot & ((1u << a.lp) - 1), l, h);
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

// Rows of a lane in flight, and whether keys and values are written together: microscaled rows are
// bound by the issue of their quantisation and addresses, which keys and values share; copies by
// memory, where one array at a time keeps more of the rows that are open (3.26M rows of 8 layers,
// bf16: 557 us, together 630; mxfp8: 442, apart 448; mxfp4 419 and 426).
constexpr int page_write_rows(int format) { return format == CERTKV_CACHE_BF16 ? 1 : 2; }
constexpr int page_write_arrays(int format) { return format == CERTKV_CACHE_BF16 ? 1 : 2; }
// Written: d values of a row read, its format's bytes written, for K and for V; bound by memory
// (bf16 6.0 TB/s, mxfp8 5.7) or, mxfp4, by the issue of the quantisation.  One layer's row of 64
// sequences 3.2 us, latency (a call 8, the host's).
// D / 8 lanes to a row, UR rows of a lane in flight.  blockIdx.y: the layer, whose rows are taken
// token by token, head by head; blockIdx.z: keys or values, where they are not written together.
template <int D, typename T, int F>
__global__ __launch_bounds__(kPgThreads) void page_write_kernel(PageWriteArgs a, PgDiv by_h, PgDiv by_tn) {
  constexpr int LPR = D / 8, RPS = kPgThreads / LPR, UR = page_write_rows(F), NA = page_write_arrays(F);
  const Geo& g = a.p.g;
  const int l = blockIdx.y, ci = threadIdx.x % LPR;
  const uint32_t rows = (uint32_t)(a.tokens * g.H);
  const int64_t total = a.slot_offsets[a.p.lists];
  for (uint32_t x0 = blockIdx.x * RPS * UR; x0 < rows; x0 += gridDim.x * RPS * UR) {
    MxRaw<T> x8[UR][NA];
    int64_t row[UR];
#pragma unroll
    for (int q = 0; q < UR; ++q) {
      const uint32_t x = x0 + q * RPS + threadIdx.x / LPR;
      const uint32_t tk = by_h(min(x, rows - 1)), h = min(x, rows - 1) - tk * (uint32_t)g.H;
      int64_t j = tk;  // its slot's place
      bool mine = x < rows && j < total;
      if (a.tn) {
        const uint32_t b = by_tn(tk), i = tk - b * (uint32_t)a.tn;
        const int64_t r = a.p.per_head ? unit_index(g, l, (int)b, (int)h) : b;
        j = a.slot_offsets[r] + i;
        mine = x < rows && j < a.slot_offsets[r + 1];
      }
      if (mine && (j < 0 || j >= a.slot_count)) {
        report_range(g);
        mine = false;
      }
      row[q] = mine ? pg_row(a.p, a.slots[j], l, h) : -1;
#pragma unroll
      for (int n = 0; n < NA; ++n) {
        const certkv_tensor& t = (NA == 1 ? blockIdx.z : n) ? a.v : a.k;
        if (row[q] >= 0)
          x8[q][n].load(static_cast<const T*>(t.ptr) + l * t.s_layer + tk * t.s_token + h * t.s_head + ci * 8);
      }
    }
#pragma unroll
    for (int q = 0; q < UR; ++q)
#pragma unroll
      for (int n = 0; n < NA; ++n) {
        const bool v = NA == 1 ? blockIdx.z : n;
        if (row[q] >= 0)
          pg_store8<F, T>(g, x8[q][n], row[q] * D + ci * 8, v ? a.p.v : a.p.k,
                          v ? a.p.v_scales : a.p.k_scales);
      }
  }
  // Slots that no token fills, rows that a list counts and nobody wrote, are reported.  (By the first
  // layer's workgroups, behind their rows: a list to a thread.)
  if (blockIdx.y == 0 && blockIdx.z == 0) {
    const int32_t lists = a.tn ? a.p.lists : 1;
    for (int64_t r = (int64_t)blockIdx.x * kPgThreads + threadIdx.x; r < lists; r += (int64_t)gridDim.x * kPgThreads) {
      const int64_t n = a.tn ? a.slot_offsets[r + 1] - a.slot_offsets[r] : total;
      if (n > (a.tn ? (int64_t)a.tn : a.tokens)) report_range(g);
    }
  }
}

template <int D, typename T>
static certkv_status launch_page_write(const PageWriteArgs& a, hipStream_t s) {
  const int64_t step = page_write_rows(a.p.format) * (kPgThreads * 8 / D);
  // (no token: slots are looked at all the same)
  const int64_t steps = a.tokens > 0 ? (a.tokens * a.p.g.H + step - 1) / step : 1;
  const dim3 grid((unsigned)(steps < 64 * 256 ? steps : 64 * 256), a.tokens > 0 ? (unsigned)a.p.g.L : 1u,
                  3 - page_write_arrays(a.p.format));
  const PgDiv by_h((uint32_t)a.p.g.H), by_tn((uint32_t)a.tn);
  switch (a.p.format) {
    case CERTKV_CACHE_MXFP8:
      CERTKV_LAUNCH("page_write", (page_write_kernel<D, T, CERTKV_CACHE_MXFP8>), grid,
                    dim3(kPgThreads), 0, s, a, by_h, by_tn);
      break;
    case CERTKV_CACHE_MXFP4:
      CERTKV_LAUNCH("page_write", (page_write_kernel<D, T, CERTKV_CACHE_MXFP4>), grid,
                    dim3(kPgThreads), 0, s, a, by_h, by_tn);
      break;
    default:
      CERTKV_LAUNCH("page_write", (page_write_kernel<D, T, CERTKV_CACHE_BF16>), grid,
                    dim3(kPgThreads), 0, s, a, by_h, by_tn);
  }
  return CERTKV_OK;
}

certkv_status run_page_write(const PageWriteArgs& a, hipStream_t s) {
  if (a.dtype == CERTKV_BF16)
    return a.p.g.D == 128 ? launch_page_write<128, uint16_t>(a, s)
                          : launch_page_write<64, uint16_t>(a, s);
  return a.p.g.D == 128 ? launch_page_write<128, float>(a, s) : launch_page_write<64, float>(a, s);
}

// Rows of RB bytes (and SB of scales, 0 for bf16) as they are held, 16 bytes to a lane.  Bound by
// memory: 3.36M rows of bf16, read and written 3.4 GB, 662 to 678 us, 5.1 TB/s, where a large copy
// reaches 4.8 (with 2048 workgroups 678 to 696, with four rows of a lane in flight 703 to 720,
// keys and values in workgroups of their own 773).
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
  const int64_t steps = a.rows > 0 ? (a.rows + step - 1) / step : 1;  // (no row: slots are looked at)
  const dim3 grid((unsigned)(steps < 4 * 256 ? steps : 4 * 256));
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

// Eight dims of a row as they are held, and as bf16.
template <int F, int D>
struct PgRaw {
  uint4 c;
  uint32_t x;
  __device__ __forceinline__ void load(const uint8_t* rows, const uint8_t* scales, int64_t row, int ci) {
    if constexpr (F == CERTKV_CACHE_BF16) {
      const MxU4 v = __builtin_nontemporal_load(reinterpret_cast<const MxU4*>(rows + row * (2 * D)) + ci);
      c = make_uint4(v[0], v[1], v[2], v[3]);
    } else {
      if constexpr (F == CERTKV_CACHE_MXFP8) {
        const uint2 w = reinterpret_cast<const uint2*>(rows + row * D)[ci];
        c.x = w.x, c.y = w.y;
      } else {
        c.x = reinterpret_cast<const uint32_t*>(rows + row * (D / 2))[ci];
      }
      x = scales[row * (D / kMxBlock) + ci / 4];
    }
  }
  __device__ __forceinline__ uint4 values() const {
    if constexpr (F == CERTKV_CACHE_BF16) {
      return c;
    } else {
      if (x == 255u) return make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
      return mx_decode8<F>(make_uint2(c.x, c.y), mx_scale(x));
    }
  }
};

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

// Read back: a row's format's bytes read, d values written, for K and for V (6.4M rows of 16
// layers, bf16: 6.5 GB in 1050 us, 6.2 TB/s; 3.26M of mxfp8 500 us, 5.0; of heads' lists in pages of
// 16 rows, 3.36M of bf16, 650 us).  One array and one row at a time for a workgroup, blocks in turn
// over the workgroups: in runs of their own, keys with values, 1240 us.
// Rows of a lane in flight: 32 bytes of them.  (bf16, two rows 1050 us, eight 1180; mxfp8, one row
// 590 us, four 490; mxfp4, two rows 550 us, eight 400.)
constexpr int page_read_rows(int format) {
  return format == CERTKV_CACHE_BF16 ? 2 : format == CERTKV_CACHE_MXFP8 ? 4 : 8;
}
// D / 8 lanes to a row, rows token by token, head by head (heads' lists: row by row), in blocks that
// the workgroups of a layer take in turn; the list of a block's first row by a 64-way search, the
// next ones by stepping on.  blockIdx.z: keys or values.
template <int F, int D, bool F32>
__global__ __launch_bounds__(kPgThreads) void page_read_kernel(PageReadArgs a, PgDiv by_h) {
  constexpr int LPR = D / 8, RPS = kPgThreads / LPR, UR = page_read_rows(F), BLOCK = RPS * UR;
  const PageArgs& p = a.p;
  const uint8_t* src = blockIdx.z ? p.v : p.k;
  const uint8_t* scales = blockIdx.z ? p.v_scales : p.k_scales;
  void* out = blockIdx.z ? a.v : a.k;
  const int l = blockIdx.y, ci = threadIdx.x % LPR, lane = threadIdx.x & 63;
  const uint32_t H = p.per_head ? 1u : (uint32_t)p.g.H;
  const int64_t base = p.offsets[0], all = p.offsets[p.lists] - base;
  const int64_t tokens = min(all, a.rows);
  if (all > a.rows && threadIdx.x == 0 && blockIdx.x == 0) report_range(p.g);
  const uint32_t rows = out ? (uint32_t)max(tokens, (int64_t)0) * H : 0u;
  const auto first = [&](int32_t r) { return p.offsets[r] - base; };
  const int64_t out0 = p.per_head ? 0 : (int64_t)l * a.rows * H;
  for (uint32_t x0 = blockIdx.x * BLOCK; x0 < rows; x0 += gridDim.x * BLOCK) {
    const uint32_t t0 = by_h(x0), h0 = x0 - t0 * H;  // (the workgroup's)
    int32_t r = pg_find(p.lists, first, t0, lane);
    int64_t start = first(r), end = first(r + 1);
    {
      int64_t row[UR];
      int32_t id[UR];
      uint32_t in[UR], h[UR];
#pragma unroll
      for (int q = 0; q < UR; ++q) {
        const uint32_t y = h0 + threadIdx.x / LPR + q * RPS, t = by_h(y);
        const int64_t tk = min(t0 + t, (uint32_t)(tokens - 1));
        h[q] = y - t * H;
        while (tk >= end && r + 1 < p.lists) {
          ++r;
          start = end;
          end = first(r + 1);
        }
        const int64_t i = tk - start, pi = i >> p.lp;
        in[q] = (uint32_t)i & ((1u << p.lp) - 1);
        id[q] = i >= 0 && pi < p.max_pages ? p.table[(int64_t)r * p.max_pages + pi] : -1;
      }
      PgRaw<F, D> k[UR];
#pragma unroll
      for (int q = 0; q < UR; ++q) {
        // (the caller's numbers: page 0's row in the place of one that is none, not kept)
        const bool fine = (uint32_t)id[q] < (uint32_t)p.num_pages;
        if (!fine) report_range(p.g);
        row[q] = pg_place_of(p, fine ? (uint32_t)id[q] : 0u, in[q], l, h[q]);
        k[q].load(src, scales, row[q], ci);
        if (!fine) row[q] = -1;
      }
#pragma unroll
      for (int q = 0; q < UR; ++q) {
        const uint32_t x = x0 + threadIdx.x / LPR + q * RPS;
        if (x >= rows || row[q] < 0) continue;
        pg_put8<F32>(out, (out0 + x) * D + ci * 8, k[q].values());
      }
    }
  }
  // Lengths that are none (offsets that fall, more rows than a table has) are reported, also where no
  // row of the output is such a list's.  (Behind the rows: a list to a thread.)
  if (blockIdx.y == 0 && blockIdx.z == 0) {
    for (int64_t r = (int64_t)blockIdx.x * kPgThreads + threadIdx.x; r < p.lists; r += (int64_t)gridDim.x * kPgThreads) {
      const int64_t p0 = p.offsets[r], p1 = p.offsets[r + 1];
      if (page_rows(p, p0, p1) != p1 - p0) report_range(p.g);
    }
  }
}

template <int F, int D>
static certkv_status launch_page_read(const PageReadArgs& a, hipStream_t s) {
  const int H = a.p.per_head ? 1 : a.p.g.H, layers = a.p.per_head ? 1 : a.p.g.L;
  const int64_t rows = a.rows * H, step = page_read_rows(F) * (kPgThreads * 8 / D);
  const int64_t steps = rows > 0 ? (rows + step - 1) / step : 1;  // (no room: what is left out is told)
  const int64_t wgs = steps < 64 * 256 ? steps : 64 * 256;
  const dim3 grid((unsigned)wgs, (unsigned)layers, 2);
  const PgDiv by_h((uint32_t)H);
  if (a.f32)
    CERTKV_LAUNCH("page_read", (page_read_kernel<F, D, true>), grid, dim3(kPgThreads), 0, s, a, by_h);
  else
    CERTKV_LAUNCH("page_read", (page_read_kernel<F, D, false>), grid, dim3(kPgThreads), 0, s, a, by_h);
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
