// The paged cache: what its kernels take, and where its rows are.
//
// A pool of pages, `page` rows each (a power of two); row r of page p of layer l and KV head h is
// the pool's row l s_layer + p s_page + r s_row + h s_head, held as a packed cache holds it (mx.h).
// A list of rows is a sequence, its pages shared by all layers and heads, or a (layer, sequence,
// head) unit; table[list][i] is its i-th page, offsets[list + 1] - offsets[list] its length.  Page
// numbers and lengths are the caller's on the device: every use is checked against the pool.
#pragma once

#include "mx.h"
#include "stages.h"

namespace certkv {

struct PageArgs {
  Geo g;
  int32_t format;
  int32_t lp;                   // log2 of the page's rows
  int32_t num_pages, max_pages;
  int32_t per_head;
  int32_t lists;
  int64_t s_layer, s_page, s_row, s_head;  // rows
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_scales;
  uint8_t* v_scales;
  const int32_t* table;         // [lists][max_pages]
  const int64_t* offsets;       // [lists + 1]
};

// The rows of a list (0 for offsets that fall).
__device__ __forceinline__ int32_t page_rows(const PageArgs& a, int64_t first, int64_t end) {
  const int64_t n = end - first, most = (int64_t)a.max_pages << a.lp;
  return (int32_t)(n < 0 ? 0 : n < most ? n : most);
}

// Tables and slots of a step (certkv_page_resize).
struct PageResizeArgs {
  Geo g;
  int32_t lp, num_pages, max_pages, lists;
  int32_t* table;
  const int64_t* offsets;
  int32_t* ring;
  const int64_t* free;          // first free place of the ring, free pages
  const int32_t* change;
  int64_t* offsets_out;
  int64_t* free_out;
  int32_t* slots;
  int64_t slot_capacity;
  int64_t* slot_offsets;
  int32_t* ws;
};
size_t page_resize_ws(int64_t lists);
certkv_status run_page_resize(const PageResizeArgs& a, hipStream_t s);

// Rows written to slots.
struct PageWriteArgs {
  PageArgs p;
  int32_t dtype;                // of the source
  certkv_tensor k, v;           // [L][tokens][H][d]
  int64_t tokens;
  int32_t tn;                   // tokens of a sequence, or 0: one sequence after another
  const int32_t* slots;
  int64_t slot_count;
  const int64_t* slot_offsets;
};
certkv_status run_page_write(const PageWriteArgs& a, hipStream_t s);

// A packed cache's rows copied to slots.
struct PageAdoptArgs {
  PageArgs p;
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* k_scales;
  const uint8_t* v_scales;
  int64_t rows;
  const int32_t* slots;
  int64_t slot_count;
  const int64_t* slot_offsets;
};
certkv_status run_page_adopt(const PageAdoptArgs& a, hipStream_t s);

// The lists' rows out of their pages.
struct PageReadArgs {
  PageArgs p;
  bool f32;                     // out: fp32, or bf16
  int64_t rows;                 // that the outputs have room for (tokens, or packed rows)
  void* k;                      // [L][rows][H][d], or [rows][d]
  void* v;
};
certkv_status run_page_read(const PageReadArgs& a, hipStream_t s);

}  // namespace certkv
