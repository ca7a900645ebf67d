// Host side of the rotary positions and of the pages' operations: argument validation,
// launch shapes.  Nothing here throws, allocates or waits.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "rl_decode_attn.h"
#include "rlda_handle.h"
#include "rlda_params.h"

namespace {

using rlda::align_up;
using rlda::aligned16;
using rlda::elem_bytes;
using rlda::kAlign;
using rlda::PageParams;
using rlda::RotaryParams;

constexpr int32_t kMaxRows = 1 << 27;   // the rows of a call (with their launch, below)
constexpr int32_t kMaxList = 1 << 23;   // rows of a release
constexpr int64_t kMaxBlocks = (1ll << 32) / rlda::kThreads - 1;   // a launch holds fewer than 2^32 threads


bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

// floor(i / x) = umulhi(i, magic) for i < 2^17 and x <= 2^13 (the error, below i x / 2^32,
// stays under 1 / x); x >= 2.
uint32_t magic_of(int64_t x) { return (uint32_t)(((1ull << 32) + x - 1) / x); }

// Rows whose chunks of eight elements are 16-byte aligned.
bool rows_ok(const rl_decode_attn_rows* r, int eb) {
  return r && r->data && aligned16(r->data) && (r->row_stride * eb) % 16 == 0 && (r->head_stride * eb) % 16 == 0 &&
         r->row_stride >= 0 && r->head_stride >= 0;
}

// ... and no two of them share memory.
bool apart(const rl_decode_attn_rows* r, int64_t rows, int64_t heads, int64_t d) {
  const int64_t a = r->row_stride, b = r->head_stride;
  if (rows == 1 && heads == 1) return true;
  if (rows == 1) return b >= d;
  if (heads == 1) return a >= d;
  return (b >= d && a >= (heads - 1) * b + d) || (a >= d && b >= (rows - 1) * a + d);
}

bool rotary_ok(const rl_decode_attn_rotary* r, int d) {
  return r && r->freqs && ((uintptr_t)r->freqs & 7u) == 0 && r->rot_dim >= 16 && r->rot_dim % 16 == 0 && r->rot_dim <= d &&
         isfinite(r->amplitude);
}

void set_rotary(RotaryParams& p, const rl_decode_attn_rotary& r, int d, int rows, int hq, int hkv) {
  p.freqs = r.freqs;
  p.half = r.rot_dim / 2;
  p.interleaved = r.interleaved != 0;
  p.inverse = r.inverse != 0;
  p.amplitude = r.amplitude;
  p.units = p.interleaved ? d / 8 : d / 8 - p.half / 8;
  p.rows = rows;
  p.hq = hq;
  p.hkv = hkv;
  p.magic_u = magic_of(p.units);
  p.magic_qu = magic_of((int64_t)p.units * hq);
  p.magic_ku = magic_of((int64_t)p.units * std::max(hkv, 1));
  p.magic_half = magic_of(p.half);
}

int64_t rotary_blocks(const RotaryParams& p) { return ((int64_t)p.rows + p.win - 1) / p.win * (p.parts + p.page_parts); }

// Windows, and workgroups of a window.  A window doubles while it has fewer than two units
// a thread and enough windows are left: each takes its rows' sines and cosines, and
// more units to a thread than two gain nothing.  us a call, windows by 8192 workgroups alone /
// so: 8192 rows of 8 heads of 64 11.8 / 4.8, 32768 of 1 of 128 14.6 / 9.2, of 32 91.6 / 88.1.
// fp8 caches have windows of a page where sequences bring several rows, so that few of them
// hold no page's first row.  Up to kWanted workgroups turn rows, none without a unit for its
// threads.
//   Workgroups that write pages: four pages to a wave, or one while they are few.
//   Inputs beyond kStreamBytes are read past the caches, which they would only pass through,
// and written so: 32768 x 32 heads, neither 101.6 us a call, the loads 96.3, both 91.3;
// 26,237 rows into fp8 pages 144.5, 145.1, 140.2.  Smaller ones are where the projection
// left them (512 tokens, 64/8 heads: 7.8 us, and 9.4 past the caches).
constexpr int kWanted = 8192, kWindows = 1024, kPagedWindows = 128, kWantedPages = 2048;
constexpr int64_t kStreamBytes = 128ll << 20;
void set_windows(RotaryParams& p, int64_t units_a_row, int64_t jobs_a_row, int64_t bytes_a_row) {
  const bool paged = jobs_a_row > 0 && p.q_start;
  p.win = 1;
  while (p.win < rlda::kRotaryWindow && p.rows >= 2ll * p.win * (paged ? kPagedWindows : kWindows) &&
         (paged || p.win * units_a_row < 2 * rlda::kThreads))
    p.win *= 2;
  const int64_t windows = ((int64_t)p.rows + p.win - 1) / p.win, n = std::min(p.rows, p.win);
  auto most = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  p.parts = (int)std::max<int64_t>(std::min(kWanted / windows, most(n * units_a_row, rlda::kThreads)), 1);
  p.stream = p.rows * bytes_a_row > kStreamBytes;
  if (jobs_a_row > 0) {
    const int64_t jobs = (paged ? p.win / 8 + 1 : p.win) * jobs_a_row;   // (a window's pages: about)
    p.page_parts = (int)std::max(most(jobs, 4 * rlda::kWaves), std::min(kWantedPages / windows, most(jobs, rlda::kWaves)));
  }
}

}  // namespace

extern "C" {

rlda_status rl_decode_attn_rotate(rlda_dtype dtype, int32_t rows, int32_t heads, int32_t head_dim,
                                  const rl_decode_attn_rows* x, const int32_t* positions,
                                  const rl_decode_attn_rotary* rotary, const rl_decode_attn_rows* out, void* stream) {
  if (dtype != RLDA_F32 && dtype != RLDA_BF16) return dtype == RLDA_FP8_E4M3FN ? RLDA_ERR_UNSUPPORTED : RLDA_ERR_INVALID_ARG;
  if (rows < 0 || heads < 0) return RLDA_ERR_INVALID_ARG;
  if (rows > kMaxRows || heads > rlda::kMaxQHeads || head_dim < 32 || head_dim > 256 || head_dim % 8) return RLDA_ERR_UNSUPPORTED;
  if (!rotary_ok(rotary, head_dim)) return RLDA_ERR_INVALID_ARG;
  if (rows == 0 || heads == 0) return RLDA_OK;
  const int eb = elem_bytes(dtype);
  if (!rows_ok(x, eb) || !rows_ok(out, eb) || !positions || !aligned4(positions)) return RLDA_ERR_INVALID_ARG;
  if (!apart(out, rows, heads, head_dim)) return RLDA_ERR_INVALID_ARG;
  RotaryParams p;
  memset(&p, 0, sizeof p);
  set_rotary(p, *rotary, head_dim, rows, heads, 0);
  p.q = x->data;
  p.q_rs = x->row_stride;
  p.q_hs = x->head_stride;
  p.q_out = const_cast<void*>(out->data);
  p.o_rs = out->row_stride;
  p.o_hs = out->head_stride;
  p.positions = positions;
  set_windows(p, (int64_t)heads * p.units, 0, (int64_t)heads * head_dim * eb);
  if (rotary_blocks(p) > kMaxBlocks) return RLDA_ERR_UNSUPPORTED;
  return rlda::launch_rotate(dtype == RLDA_F32, p, stream) == hipSuccess ? RLDA_OK : RLDA_ERR_HIP;
}

rlda_status rl_decode_attn_append_rotary(rl_decode_attn_t h, int32_t batch, int32_t num_pages, int32_t total_q,
                                         const rl_decode_attn_rotary* rotary, const rl_decode_attn_rows* q,
                                         const rl_decode_attn_rows* k_new, const rl_decode_attn_rows* v_new,
                                         const int32_t* q_start, const int32_t* positions, void* k_cache, void* v_cache,
                                         float* k_scale, float* v_scale, const int32_t* block_table,
                                         const int32_t* seq_lens, const rl_decode_attn_rows* q_out, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  if (!h) return RLDA_ERR_INVALID_ARG;
  const rl_decode_attn_config& c = h->cfg;
  if (batch < 0 || batch > c.max_batch || num_pages < 0 || total_q < 0) return RLDA_ERR_INVALID_ARG;
  if (!q_start && total_q != batch) return RLDA_ERR_INVALID_ARG;
  if (total_q > kMaxRows) return RLDA_ERR_UNSUPPORTED;
  if (!rotary_ok(rotary, c.head_dim)) return RLDA_ERR_INVALID_ARG;
  if (batch == 0 || total_q == 0) return RLDA_OK;
  const int eb = elem_bytes(c.q_dtype);
  if (!rows_ok(q, eb) || !rows_ok(k_new, eb) || !rows_ok(v_new, eb) || !rows_ok(q_out, eb)) return RLDA_ERR_INVALID_ARG;
  if (!apart(q_out, total_q, c.num_q_heads, c.head_dim)) return RLDA_ERR_INVALID_ARG;
  if (!block_table || !seq_lens || !aligned4(block_table) || !aligned4(seq_lens) || !aligned4(q_start) || !aligned4(positions))
    return RLDA_ERR_INVALID_ARG;
  // K is turned and V is not: one cache cannot be both.
  if (num_pages > 0 && (!k_cache || !v_cache || k_cache == v_cache)) return RLDA_ERR_INVALID_ARG;
  if (!aligned16(k_cache) || !aligned16(v_cache)) return RLDA_ERR_INVALID_ARG;
  if (h->kind == rlda::KvKind::FP8 && num_pages > 0 &&
      (!k_scale || !v_scale || k_scale == v_scale || !aligned4(k_scale) || !aligned4(v_scale)))
    return RLDA_ERR_INVALID_ARG;
  const rlda::WsLayout wl = rlda::layout_of(h);
  if (!workspace || ((uintptr_t)workspace % kAlign)) return RLDA_ERR_WORKSPACE;
  if (workspace_bytes < wl.total) return RLDA_ERR_WORKSPACE;
  RotaryParams p;
  memset(&p, 0, sizeof p);
  set_rotary(p, *rotary, c.head_dim, total_q, c.num_q_heads, c.num_kv_heads);
  p.q = q->data;
  p.q_rs = q->row_stride;
  p.q_hs = q->head_stride;
  p.k_in = k_new->data;
  p.k_rs = k_new->row_stride;
  p.k_hs = k_new->head_stride;
  p.v_in = v_new->data;
  p.v_rs = v_new->row_stride;
  p.v_hs = v_new->head_stride;
  p.q_out = const_cast<void*>(q_out->data);
  p.o_rs = q_out->row_stride;
  p.o_hs = q_out->head_stride;
  p.k = k_cache;
  p.v = v_cache;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.q_start = q_start;
  p.positions = positions;
  p.flags = (uint32_t*)((char*)workspace + wl.flags);
  const int kb = elem_bytes(c.kv_dtype);
  p.stride_page = h->stride_page * kb;
  p.stride_head = h->stride_head * kb;
  p.stride_slot = (int32_t)(h->stride_slot * kb);
  p.batch = batch;
  p.num_pages = num_pages;
  p.max_pages = c.max_pages_per_seq;
  set_windows(p, (int64_t)c.num_q_heads * p.units, h->kind == rlda::KvKind::FP8 ? 2 * c.num_kv_heads : 0,
              (int64_t)(c.num_q_heads + 2 * c.num_kv_heads) * c.head_dim * eb);
  if (rotary_blocks(p) > kMaxBlocks) return RLDA_ERR_UNSUPPORTED;
  return rlda::launch_append_rotary(h->kind, c.head_dim, p, stream) == hipSuccess ? RLDA_OK : RLDA_ERR_HIP;
}

}  // extern "C"

// ---------------------------------------------------------------- pages

namespace {

struct PageWs {
  size_t flags, count, live, mask, group_free, src, dst, full, map, total;
};

PageWs page_layout(const rlda_handle* h, int32_t num_pages) {
  const size_t pairs = std::max<size_t>((size_t)h->cfg.max_batch, (size_t)num_pages / 2 + 1);
  PageWs w;
  w.flags = 0;
  w.count = 64;
  w.live = 128;
  w.mask = kAlign;
  w.group_free = align_up(w.mask + sizeof(uint64_t) * (((size_t)num_pages + 63) / 64 + 1));
  w.src = align_up(w.group_free + sizeof(int32_t) * rlda::kPageGroups);
  w.dst = align_up(w.src + sizeof(int32_t) * pairs);
  w.full = align_up(w.dst + sizeof(int32_t) * pairs);
  w.map = align_up(w.full + sizeof(int32_t) * (size_t)h->cfg.max_batch);
  w.total = align_up(w.map + sizeof(int32_t) * (size_t)num_pages);
  return w;
}

// What every page operation checks and sets.
rlda_status page_call(rl_decode_attn_t h, int32_t batch, int32_t num_pages, int32_t* refs, int32_t* block_table,
                      int32_t* seq_lens, void* workspace, size_t workspace_bytes, PageParams& p) {
  if (!h) return RLDA_ERR_INVALID_ARG;
  const rl_decode_attn_config& c = h->cfg;
  if (batch < 0 || batch > c.max_batch || num_pages < 0) return RLDA_ERR_INVALID_ARG;
  if (batch > 0 && (!block_table || !seq_lens)) return RLDA_ERR_INVALID_ARG;
  if (num_pages > 0 && !refs) return RLDA_ERR_INVALID_ARG;
  if (!aligned4(refs) || !aligned4(block_table) || !aligned4(seq_lens)) return RLDA_ERR_INVALID_ARG;
  const PageWs wl = page_layout(h, num_pages);
  if (!workspace || ((uintptr_t)workspace % kAlign)) return RLDA_ERR_WORKSPACE;
  if (workspace_bytes < wl.total) return RLDA_ERR_WORKSPACE;
  char* ws = (char*)workspace;
  memset(&p, 0, sizeof p);
  p.refs = refs;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.flags = (uint32_t*)(ws + wl.flags);
  p.count_out = (int32_t*)(ws + wl.count);
  p.live_out = (int32_t*)(ws + wl.live);
  p.mask = (uint64_t*)(ws + wl.mask);
  p.group_free = (int32_t*)(ws + wl.group_free);
  p.list_src = (int32_t*)(ws + wl.src);
  p.list_dst = (int32_t*)(ws + wl.dst);
  p.fork_full = (int32_t*)(ws + wl.full);
  p.map = (int32_t*)(ws + wl.map);
  const int eb = elem_bytes(c.kv_dtype);
  p.stride_page = h->stride_page * eb;
  p.stride_head = h->stride_head * eb;
  p.stride_slot = (int32_t)(h->stride_slot * eb);
  p.row_bytes = c.head_dim * eb;
  p.page_bytes = c.num_kv_heads * rlda::kPage * p.row_bytes;
  const int64_t d = c.head_dim, sh = h->stride_head, ss = h->stride_slot;
  p.linear = (ss == d && (c.num_kv_heads == 1 || sh == rlda::kPage * d)) || (sh == d && ss == c.num_kv_heads * d);
  p.num_pages = num_pages;
  p.num_kv_heads = c.num_kv_heads;
  p.batch = batch;
  p.max_pages = c.max_pages_per_seq;
  p.words = (int32_t)(((int64_t)num_pages + 63) / 64);
  p.group_words = std::max((p.words + rlda::kPageGroups - 1) / rlda::kPageGroups, 1);
  p.in_lds = p.group_words == 1;
  return RLDA_OK;
}

// Layers of a workgroup that copies pages: a pair of a few KiB is too little for one.
constexpr int kCopyBytes = 16 << 10;
constexpr int kMoveGrid = 32768;   // workgroups of a compaction's copies at most
constexpr int kCopyGrid = 1 << 20;   // ... of a list's copies

rlda_status check_caches(rl_decode_attn_t h, int32_t num_caches, const rl_decode_attn_cache* caches, int32_t num_pages) {
  if (num_caches < 0 || (num_caches > 0 && !caches)) return RLDA_ERR_INVALID_ARG;
  for (int i = 0; i < num_caches && num_pages > 0; ++i) {
    const rl_decode_attn_cache& c = caches[i];
    if (!c.k_cache || !c.v_cache || !aligned16(c.k_cache) || !aligned16(c.v_cache)) return RLDA_ERR_INVALID_ARG;
    if (h->kind == rlda::KvKind::FP8 && (!c.k_scale || !c.v_scale || !aligned4(c.k_scale) || !aligned4(c.v_scale)))
      return RLDA_ERR_INVALID_ARG;
  }
  return RLDA_OK;
}

// Launches f once for every kPageMaxCaches caches (once without any: tables and counts).
template <class F>
rlda_status for_caches(rl_decode_attn_t h, PageParams& p, int32_t num_caches, const rl_decode_attn_cache* caches, F f) {
  const bool fp8 = h->kind == rlda::KvKind::FP8;
  int at = 0;
  do {
    const int n = std::min(num_caches - at, rlda::kPageMaxCaches);
    for (int i = 0; i < n; ++i) {
      const rl_decode_attn_cache& c = caches[at + i];
      p.caches[i] = {(char*)c.k_cache, (char*)c.v_cache, fp8 ? c.k_scale : nullptr, fp8 ? c.v_scale : nullptr};
    }
    p.num_caches = n;
    p.block_layers = std::max(kCopyBytes / (2 * p.page_bytes), 1);
    p.layer_blocks = (n + p.block_layers - 1) / p.block_layers;
    p.share = at == 0;
    if (f() != hipSuccess) return RLDA_ERR_HIP;
    at += n;
  } while (at < num_caches);
  return RLDA_OK;
}

}  // namespace

extern "C" {

rlda_status rl_decode_attn_page_workspace_size(rl_decode_attn_t h, int32_t num_pages, size_t* bytes) {
  if (!h || !bytes || num_pages < 0) return RLDA_ERR_INVALID_ARG;
  *bytes = page_layout(h, num_pages).total;
  return RLDA_OK;
}

rlda_status rl_decode_attn_page_grow(rl_decode_attn_t h, int32_t batch, int32_t num_pages, int32_t* refs,
                                     int32_t* block_table, int32_t* seq_lens, const int32_t* add, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  PageParams p;
  const rlda_status st = page_call(h, batch, num_pages, refs, block_table, seq_lens, workspace, workspace_bytes, p);
  if (st != RLDA_OK) return st;
  if (!aligned4(add)) return RLDA_ERR_INVALID_ARG;
  if (batch == 0) return RLDA_OK;
  p.add = add;
  return rlda::launch_page_grow(p, stream) == hipSuccess ? RLDA_OK : RLDA_ERR_HIP;
}

rlda_status rl_decode_attn_page_release(rl_decode_attn_t h, int32_t batch, int32_t num_pages, int32_t* refs,
                                        int32_t* block_table, int32_t* seq_lens, int32_t count, const int32_t* rows,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  PageParams p;
  const rlda_status st = page_call(h, batch, num_pages, refs, block_table, seq_lens, workspace, workspace_bytes, p);
  if (st != RLDA_OK) return st;
  if (count < 0 || (count > 0 && (!rows || !aligned4(rows)))) return RLDA_ERR_INVALID_ARG;
  if (count > kMaxList) return RLDA_ERR_UNSUPPORTED;
  if (count == 0) return RLDA_OK;
  p.count = count;
  p.list_a = rows;
  return rlda::launch_page_release(p, stream) == hipSuccess ? RLDA_OK : RLDA_ERR_HIP;
}

rlda_status rl_decode_attn_page_fork(rl_decode_attn_t h, int32_t batch, int32_t num_pages, int32_t* refs,
                                     int32_t* block_table, int32_t* seq_lens, int32_t count, const int32_t* parents,
                                     const int32_t* children, int32_t num_caches, const rl_decode_attn_cache* caches,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  PageParams p;
  rlda_status st = page_call(h, batch, num_pages, refs, block_table, seq_lens, workspace, workspace_bytes, p);
  if (st != RLDA_OK) return st;
  if (count < 0 || count > h->cfg.max_batch) return RLDA_ERR_INVALID_ARG;
  if (count > 0 && (!parents || !children || !aligned4(parents) || !aligned4(children))) return RLDA_ERR_INVALID_ARG;
  if ((st = check_caches(h, num_caches, caches, num_pages)) != RLDA_OK) return st;
  if (count == 0) return RLDA_OK;
  p.count = count;
  p.list_a = parents;
  p.list_b = children;
  if (rlda::launch_page_fork(p, stream) != hipSuccess) return RLDA_ERR_HIP;
  return for_caches(h, p, num_caches, caches, [&] { return rlda::launch_page_fork_rows(p, stream); });
}

rlda_status rl_decode_attn_page_compact(rl_decode_attn_t h, int32_t batch, int32_t num_pages, int32_t* refs,
                                        int32_t* block_table, int32_t* seq_lens, int32_t num_caches,
                                        const rl_decode_attn_cache* caches, int32_t* live, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  PageParams p;
  rlda_status st = page_call(h, batch, num_pages, refs, block_table, seq_lens, workspace, workspace_bytes, p);
  if (st != RLDA_OK) return st;
  if (!live || !aligned4(live)) return RLDA_ERR_INVALID_ARG;
  if ((st = check_caches(h, num_caches, caches, num_pages)) != RLDA_OK) return st;
  p.live_out = live;
  if (rlda::launch_page_compact(p, stream) != hipSuccess) return RLDA_ERR_HIP;
  return for_caches(h, p, num_caches, caches, [&] {
    // One for every copy there may be (half of the pages), and some for the table's rows.
    const int64_t copies = (int64_t)num_pages / 2 * p.layer_blocks;
    return rlda::launch_page_move(p, (int)std::min<int64_t>(std::max<int64_t>(copies, 256), kMoveGrid), stream);
  });
}

rlda_status rl_decode_attn_page_copy(rl_decode_attn_t h, int32_t num_pages, int32_t count, const int32_t* src,
                                     const int32_t* dst, int32_t num_caches, const rl_decode_attn_cache* caches,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  PageParams p;
  int32_t none = 0;   // the counts are not looked at
  rlda_status st = page_call(h, 0, num_pages, &none, nullptr, nullptr, workspace, workspace_bytes, p);
  if (st != RLDA_OK) return st;
  p.refs = nullptr;
  if (count < 0 || (count > 0 && (!src || !dst || !aligned4(src) || !aligned4(dst)))) return RLDA_ERR_INVALID_ARG;
  if ((st = check_caches(h, num_caches, caches, num_pages)) != RLDA_OK) return st;
  if (count == 0 || num_caches == 0) return RLDA_OK;
  if ((int64_t)count * rlda::kPageMaxCaches > INT32_MAX) return RLDA_ERR_UNSUPPORTED;
  p.count = count;
  p.list_src = const_cast<int32_t*>(src);
  p.list_dst = const_cast<int32_t*>(dst);
  return for_caches(h, p, num_caches, caches, [&] {
    return rlda::launch_page_copy(p, std::min(count * p.layer_blocks, kCopyGrid), stream);
  });
}

}  // extern "C"

// ---------------------------------------------------------------- bounds, choice, eviction

namespace {

using rlda::SelectParams;

void set_select(rl_decode_attn_t h, SelectParams& p) {
  const rl_decode_attn_config& c = h->cfg;
  memset(&p, 0, sizeof p);
  p.max_pages = c.max_pages_per_seq;
  p.num_q_heads = c.num_q_heads;
  p.num_kv_heads = c.num_kv_heads;
  p.group = h->group;
  memcpy(p.q_head, h->q_head, sizeof p.q_head);
}

bool budget_ok(int32_t budget, int32_t sink, int32_t recent) {
  return sink >= 0 && recent >= 1 && (int64_t)sink + recent <= budget;
}

// Workgroups of a choice: several to a (row, KV head) while that leaves CUs idle, none with
// less than kPiecePages of the longest sequence there may be.
constexpr int kWantedChoices = 256, kPiecePages = 512;
constexpr int32_t kMaxBudget = 1 << 24;   // entries of a choice's list

}  // namespace

extern "C" {

rlda_status rl_decode_attn_page_bounds(rl_decode_attn_t h, int32_t batch, int32_t num_pages, const void* k_cache,
                                       const float* k_scale, const int32_t* block_table, const int32_t* seq_lens,
                                       const int32_t* first, int8_t* bounds, float* bound_scale, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  if (!h) return RLDA_ERR_INVALID_ARG;
  const rl_decode_attn_config& c = h->cfg;
  if (batch < 0 || batch > c.max_batch || num_pages < 0) return RLDA_ERR_INVALID_ARG;
  if (batch == 0) return RLDA_OK;
  if (!block_table || !seq_lens || !aligned4(block_table) || !aligned4(seq_lens) || !aligned4(first)) return RLDA_ERR_INVALID_ARG;
  if (num_pages > 0 && (!k_cache || !bounds || !bound_scale)) return RLDA_ERR_INVALID_ARG;
  if (!aligned16(k_cache) || !aligned16(bounds) || !aligned4(bound_scale)) return RLDA_ERR_INVALID_ARG;
  if (h->kind == rlda::KvKind::FP8 && num_pages > 0 && (!k_scale || !aligned4(k_scale))) return RLDA_ERR_INVALID_ARG;
  const rlda::WsLayout wl = rlda::layout_of(h);
  if (!workspace || ((uintptr_t)workspace % kAlign)) return RLDA_ERR_WORKSPACE;
  if (workspace_bytes < wl.total) return RLDA_ERR_WORKSPACE;
  SelectParams p;
  set_select(h, p);
  p.k = k_cache;
  p.k_scale = k_scale;
  p.bounds = bounds;
  p.bound_scale = bound_scale;
  p.block_table = const_cast<int32_t*>(block_table);
  p.seq_lens = const_cast<int32_t*>(seq_lens);
  p.first = first;
  p.flags = (uint32_t*)((char*)workspace + wl.flags);
  const int eb = elem_bytes(c.kv_dtype);
  p.stride_page = h->stride_page * eb;
  p.stride_head = h->stride_head * eb;
  p.stride_slot = (int32_t)(h->stride_slot * eb);
  p.batch = batch;
  p.num_pages = num_pages;
  return rlda::launch_page_bounds(h->kind, c.head_dim, p, stream) == hipSuccess ? RLDA_OK : RLDA_ERR_HIP;
}

rlda_status rl_decode_attn_select_pages(rl_decode_attn_t h, int32_t batch, int32_t num_pages, int32_t total_q, int32_t budget,
                                        int32_t sink, int32_t recent, const void* q, const int8_t* bounds,
                                        const float* bound_scale, const int32_t* block_table, const int32_t* seq_lens,
                                        const int32_t* q_start, int32_t* pages, int32_t* counts, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  if (!h) return RLDA_ERR_INVALID_ARG;
  const rl_decode_attn_config& c = h->cfg;
  if (batch < 0 || batch > c.max_batch || num_pages < 0 || total_q < 0) return RLDA_ERR_INVALID_ARG;
  if (!q_start && total_q != batch) return RLDA_ERR_INVALID_ARG;
  if (!budget_ok(budget, sink, recent)) return RLDA_ERR_INVALID_ARG;
  if (c.max_pages_per_seq > rlda::kSelectMaxPages || budget > kMaxBudget) return RLDA_ERR_UNSUPPORTED;
  if (batch == 0 || total_q == 0) return RLDA_OK;
  if (!q || !block_table || !seq_lens || !pages || !counts || !aligned16(q)) return RLDA_ERR_INVALID_ARG;
  if (!aligned4(block_table) || !aligned4(seq_lens) || !aligned4(q_start) || !aligned4(pages) || !aligned4(counts))
    return RLDA_ERR_INVALID_ARG;
  if (num_pages > 0 && (!bounds || !bound_scale)) return RLDA_ERR_INVALID_ARG;
  if (!aligned16(bounds) || !aligned4(bound_scale)) return RLDA_ERR_INVALID_ARG;
  const rlda::WsLayout wl = rlda::layout_of(h);
  if (!workspace || ((uintptr_t)workspace % kAlign)) return RLDA_ERR_WORKSPACE;
  if (workspace_bytes < wl.total) return RLDA_ERR_WORKSPACE;
  SelectParams p;
  set_select(h, p);
  p.q = q;
  p.bounds = const_cast<int8_t*>(bounds);
  p.bound_scale = const_cast<float*>(bound_scale);
  p.block_table = const_cast<int32_t*>(block_table);
  p.seq_lens = const_cast<int32_t*>(seq_lens);
  p.q_start = q_start;
  p.pages = pages;
  p.counts = counts;
  char* ws = (char*)workspace;
  p.flags = (uint32_t*)(ws + wl.flags);
  p.counters = (uint32_t*)(ws + wl.counters);
  p.keys = (uint32_t*)(ws + wl.part_acc);   // where an attention call keeps its partial results
  p.batch = batch;
  p.num_pages = num_pages;
  p.total_q = total_q;
  p.budget = budget;
  p.sink = sink;
  p.recent = recent;
  const int64_t segs = (int64_t)total_q * c.num_kv_heads;
  p.pieces = 1;
  if (segs <= (int64_t)rlda::counters_of(h) && segs * c.max_pages_per_seq * (int64_t)sizeof(uint32_t) <= (int64_t)(wl.total - wl.part_acc))
    p.pieces = (int)std::max<int64_t>(std::min<int64_t>(kWantedChoices / segs, c.max_pages_per_seq / kPiecePages), 1);
  if (segs * p.pieces * rlda::kSelectThreads > (1ll << 32) - 1) return RLDA_ERR_UNSUPPORTED;   // threads of a launch
  return rlda::launch_select_pages(c.q_dtype == RLDA_F32, c.head_dim, p, stream) == hipSuccess ? RLDA_OK : RLDA_ERR_HIP;
}

rlda_status rl_decode_attn_page_evict(rl_decode_attn_t h, int32_t batch, int32_t num_pages, int32_t* refs,
                                      int32_t* block_table, int32_t* seq_lens, float* weights, int32_t budget, int32_t sink,
                                      int32_t recent, int32_t* dropped, void* workspace, size_t workspace_bytes, void* stream) {
  PageParams pp;
  const rlda_status st = page_call(h, batch, num_pages, refs, block_table, seq_lens, workspace, workspace_bytes, pp);
  if (st != RLDA_OK) return st;
  if (!budget_ok(budget, sink, recent)) return RLDA_ERR_INVALID_ARG;
  if (h->cfg.max_pages_per_seq > rlda::kSelectMaxPages) return RLDA_ERR_UNSUPPORTED;
  if (batch == 0) return RLDA_OK;
  if (!weights || !dropped || !aligned4(weights) || !aligned4(dropped)) return RLDA_ERR_INVALID_ARG;
  SelectParams p;
  set_select(h, p);
  p.refs = refs;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.weights = weights;
  p.dropped = dropped;
  p.flags = pp.flags;
  p.batch = batch;
  p.num_pages = num_pages;
  p.budget = budget;
  p.sink = sink;
  p.recent = recent;
  return rlda::launch_page_evict(p, stream) == hipSuccess ? RLDA_OK : RLDA_ERR_HIP;
}

}  // extern "C"
