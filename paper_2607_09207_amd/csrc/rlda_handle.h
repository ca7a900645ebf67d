// The handle, and what the host sources share.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "rl_decode_attn.h"
#include "rlda_params.h"

struct rlda_handle {
  rl_decode_attn_config cfg;
  int32_t group;
  int64_t stride_page, stride_head, stride_slot;   // elements
  int32_t ws_ranges;                               // work ranges the workspace is sized for
  float scale;
  int16_t q_head[rlda::kMaxQHeads];
  rlda::KvKind kind;
};

namespace rlda {

constexpr size_t kAlign = 256;

inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

inline int elem_bytes(rlda_dtype t) { return t == RLDA_F32 ? 4 : t == RLDA_BF16 ? 2 : 1; }

struct WsLayout {
  size_t flags, counters, part_ml, part_acc, total;
  size_t gprefix, pfx_ml, pfx_acc, grouped_total;   // grouped runs only
};

inline size_t counters_of(const rlda_handle* h) {
  const size_t segments = (size_t)h->cfg.max_batch * rlda::kMaxRowChunks, rows = rlda::kRowsMax;
  return (segments > rows ? segments : rows) * (size_t)h->cfg.num_kv_heads;
}

inline WsLayout layout_of(const rlda_handle* h) {
  const rl_decode_attn_config& c = h->cfg;
  WsLayout w;
  w.flags = 0;
  w.counters = align_up(sizeof(uint32_t));
  // Counters: one per (sequence, KV head) segment, or per 16-row chunk of one in
  // multi-token runs through the decode kernel, or per (query row, KV head) of up to
  // kRowsMax rows.
  w.part_ml = align_up(w.counters + sizeof(uint32_t) * counters_of(h));
  // Partial slots: two per work range, 16 rows each (G rows in decode runs, up to
  // 16 rows of a segment in multi-token runs).
  w.part_acc = align_up(w.part_ml + sizeof(float) * 4 * (size_t)h->ws_ranges * rlda::kMaxGroup * 2);
  w.total = align_up(w.part_acc + sizeof(float) * 2 * (size_t)h->ws_ranges * rlda::kMaxGroup * c.head_dim);
  w.gprefix = w.total;
  w.pfx_ml = align_up(w.gprefix + sizeof(int32_t) * (size_t)c.max_batch);
  w.pfx_acc = align_up(w.pfx_ml + sizeof(float) * 2 * (size_t)c.max_batch * c.num_q_heads);
  w.grouped_total = align_up(w.pfx_acc + sizeof(float) * (size_t)c.max_batch * c.num_q_heads * c.head_dim);
  return w;
}

// Calls that keep the pages' weights: the plain workspace, then the parts of every row's
// softmax, [rows][Hq][max_pages] and [rows][Hq], and the sequence that every row was taken as.
struct WeighedLayout {
  size_t page_lse, row_lse, row_seq, total;
};
inline WeighedLayout weighed_layout(const rlda_handle* h, int32_t rows) {
  const size_t heads = (size_t)rows * h->cfg.num_q_heads;
  WeighedLayout w;
  w.page_lse = layout_of(h).total;
  w.row_lse = align_up(w.page_lse + sizeof(float) * heads * (size_t)h->cfg.max_pages_per_seq);
  w.row_seq = align_up(w.row_lse + sizeof(float) * heads);
  w.total = align_up(w.row_seq + sizeof(int32_t) * (size_t)rows);
  return w;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace rlda
