// The pages of the KV cache for gfx950: taking, sharing, returning, moving and copying them.
//
// The state of a pool is one reference count per page, refs[page] (0: free), besides the
// block table and the lengths that the caller keeps anyway.  Free pages are always taken
// lowest number first, in the order of the requests: the result depends on nothing but
// the state, and no list has to be kept in step with it.
//
// Work.  Taking pages is a prefix sum over the requests against a prefix sum over the
// pool's free pages, j-th page to j-th request: one workgroup of 1024 threads does all of
// it, because a second launch or a hand-off between workgroups costs more than it saves
// until the pool is large.  The pool's counts are read once into a bit mask (a wave's
// ballot is a word of it) with the free pages before every group of words; the j-th free
// page is a search of these, then a selection in a word.  Up to kLdsPages pages the mask
// stays in LDS; larger pools are turned into one by a launch over the whole GPU before it.
// What moves cache contents is a separate launch with one workgroup per (page, few
// layers), and is bound by bandwidth; everything else by the latency of dependent reads.
// Kernel times: taking pages 6.4 us (64 sequences, a pool of 5,600 pages) and releasing 8 rows
// 3.0; forking 32 prompts into 256 rows 6.2, and 22.5 for their tables and partial pages in 28
// layers (110 MB written); compacting 16 layers 8.0, and 165 to 182 for the moves (980 MB
// read and written, 5.4 TB/s and more; a copy of one large buffer reaches 4.9).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rlda_device.h"
#include "rlda_params.h"
#include "rlda_split.h"

namespace rlda {
namespace {

constexpr int kMgr = 1024;                          // threads of the workgroup that takes pages
constexpr int kMgrWaves = kMgr / 64;
constexpr int kGroups = kPageGroups;                // groups of mask words
constexpr int kLdsWords = kGroups;                  // mask words kept in LDS: one a group
constexpr int kPerThread = kMaxBatch / kMgr;        // requests of a thread

// Prefix sum over the workgroup: each thread's x, its sum over the threads before it; `all`
// gets the total.
__device__ __forceinline__ int block_before(int x, int* s_tmp, int* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_scan(x);
  __syncthreads();   // s_tmp may still be read from the last use
  if (lane == 63) s_tmp[wave] = incl;
  __syncthreads();
  int before = incl - x, sum = 0;
  for (int w = 0; w < kMgrWaves; ++w) {
    const int v = s_tmp[w];
    before += w < wave ? v : 0;
    sum += v;
  }
  *all = sum;
  return before;
}

// Position of the k-th set bit (k < popcount).
__device__ __forceinline__ int select_bit(uint64_t m, int k) {
  int at = 0;
#pragma unroll
  for (int w = 32; w >= 1; w >>= 1) {
    const uint64_t low = m & ((1ull << w) - 1);
    const int c = __builtin_popcountll(low);
    if (k >= c) {
      k -= c;
      m >>= w;
      at += w;
    } else {
      m = low;
    }
  }
  return at;
}

// A mask over the pool's pages in words of 64, and the set bits before each of kGroups
// groups of words.
struct Mask {
  const uint64_t* words;
  const int* before;   // [kGroups + 1]
  int per;             // words of a group
  // The page of the k-th bit that differs from `flip` (0: set bits, ~0: clear ones).
  __device__ __forceinline__ int page_of(int k) const {
    int lo = 0, hi = kGroups;   // before[lo] <= k < before[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before[mid] <= k) lo = mid; else hi = mid;
    }
    k -= before[lo];
    int w = lo * per;
    for (;; ++w) {
      const int c = __builtin_popcountll(words[w]);
      if (k < c) break;
      k -= c;
    }
    return w * 64 + select_bit(words[w], k);
  }
};

// One word of the mask per wave: pages 64 w .. of the pool that are free.
__device__ __forceinline__ uint64_t free_word(const PageParams& p, int w, int lane) {
  const int64_t page = (int64_t)w * 64 + lane;
  const bool free = page < p.num_pages && p.refs[page] == 0;
  return __builtin_amdgcn_ballot_w64(free);
}

// Large pools: the mask, and the free pages of every group, by the whole GPU.
__global__ __launch_bounds__(kThreads) void page_mask_kernel(const PageParams p) {
  const int lane = threadIdx.x & 63, wave = uni((int)(threadIdx.x >> 6));
  __shared__ int s_count[kWaves];
  int count = 0;
  const int w1 = min((int)(blockIdx.x + 1) * p.group_words, p.words);
  for (int w = blockIdx.x * p.group_words + wave; w < w1; w += kWaves) {
    const uint64_t m = free_word(p, w, lane);
    if (lane == 0) p.mask[w] = m;
    count += __builtin_popcountll(m);
  }
  if (lane == 0) s_count[wave] = count;
  __syncthreads();
  if (threadIdx.x == 0) p.group_free[blockIdx.x] = s_count[0] + s_count[1] + s_count[2] + s_count[3];
}

struct Pool {
  uint64_t words[kLdsWords];
  int before[kGroups + 1];
  int tmp[kMgrWaves];
};

// Counts of eight words of a wave's: asked for together.
struct Counts {
  int r[8];
  __device__ __forceinline__ void load(const PageParams& p, int w0) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t page = (int64_t)(w0 + i * kMgrWaves) * 64 + lane;
      r[i] = p.in_lds && page < p.num_pages ? p.refs[page] : 1;
    }
  }
};

// The mask of free pages (all threads of the workgroup); returns the free pages' number.
// `c`: the first counts, asked for by the caller ahead of its own reads.
__device__ __forceinline__ int read_pool(const PageParams& p, Pool& s, Mask& mask, Counts c) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  mask = Mask{s.words, s.before, p.group_words};
  constexpr int kPer = kGroups / kMgr;   // groups of a thread
  int n[kPer], sum = 0, all;
  if (p.in_lds) {
    for (int w0 = wave; w0 < kGroups; w0 += 8 * kMgrWaves) {
      if (w0 >= p.words) break;
      if (w0 != wave) c.load(p, w0);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint64_t m = __builtin_amdgcn_ballot_w64(c.r[i] == 0);
        const int w = w0 + i * kMgrWaves;
        if (lane == 0 && w < kLdsWords) s.words[w] = m;
      }
    }
    __syncthreads();
  } else {
    mask.words = p.mask;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int gr = tid * kPer + i;
    n[i] = gr * p.group_words >= p.words ? 0 : p.in_lds ? __builtin_popcountll(s.words[gr]) : p.group_free[gr];
    sum += n[i];
  }
  int run = block_before(sum, s.tmp, &all);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    s.before[tid * kPer + i] = run;
    run += n[i];
  }
  if (tid == kMgr - 1) s.before[kGroups] = run;
  __syncthreads();
  return all;
}

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + kPage - 1) / kPage; }

// ---------------------------------------------------------------- grow

__global__ __launch_bounds__(kMgr) void page_grow_kernel(const PageParams p) {
  __shared__ Pool s_pool;
  __shared__ int s_off[kMaxBatch + 1];   // pages asked for before each sequence
  const int tid = threadIdx.x, cap = p.max_pages * kPage;
  const int per = (p.batch + kMgr - 1) / kMgr, b0 = tid * per, b1 = min(b0 + per, p.batch);
  Counts c;
  c.load(p, uni(tid >> 6));
  // A sequence whose length or growth is out of range asks for nothing and stays.
  int len[kPerThread], add[kPerThread], sum = 0, all;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    len[i] = add[i] = 0;
    const int b = b0 + i;
    if (b >= b1) continue;
    const int L = p.seq_lens[b], a = p.add ? p.add[b] : 1;
    if (L < 0 || L > cap || a < 0 || a > cap - L) {
      bad = true;
      continue;
    }
    len[i] = L;
    add[i] = a;
    sum += pages_of(L + a) - pages_of(L);
  }
  Mask mask;
  const int nfree = read_pool(p, s_pool, mask, c);
  int run = block_before(sum, s_pool.tmp, &all);
  // Requests are served in order until one finds too few pages left.
  bool out = false;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int b = b0 + i;
    if (b >= b1) continue;
    const int need = pages_of(len[i] + add[i]) - pages_of(len[i]);
    s_off[b] = run;
    run += need;
    if (add[i] == 0) continue;
    if (need == 0 || run <= nfree)
      p.seq_lens[b] = len[i] + add[i];
    else
      out = true;
  }
  if (b0 < p.batch && b1 == p.batch) s_off[p.batch] = run;
  if (bad) atomicOr(p.flags, kFlagBadLen);
  if (out) atomicOr(p.flags, kFlagNoPages);
  __syncthreads();
  // Page j goes to the sequence that asked for it: its own j - s_off[b]-th new page.
  const int total = min(s_off[p.batch], nfree);
  for (int j = tid; j < total; j += kMgr) {
    int lo = 0, hi = p.batch;   // s_off[lo] <= j < s_off[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_off[mid] <= j) lo = mid; else hi = mid;
    }
    const int need = s_off[lo + 1] - s_off[lo];
    if (s_off[lo] + need > nfree) continue;   // not served
    // The sequence is served, so its length is the new one by now (written above, by this workgroup).
    const int L = __hip_atomic_load(p.seq_lens + lo, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    const int page = mask.page_of(j);
    p.block_table[(int64_t)lo * p.max_pages + pages_of(L) - need + (j - s_off[lo])] = page;
    p.refs[page] = 1;
  }
}

// ---------------------------------------------------------------- release

// One workgroup per row: its pages lose a reference each.  The length is taken and set to
// zero in one step, so that a row named twice is released once.
__global__ __launch_bounds__(kThreads) void page_release_kernel(const PageParams p) {
  __shared__ int s_len;
  const int row = p.list_a[blockIdx.x];
  if ((uint32_t)row >= (uint32_t)p.batch) {
    if (threadIdx.x == 0) atomicOr(p.flags, kFlagBadLen);
    return;
  }
  if (threadIdx.x == 0) s_len = atomicExch(p.seq_lens + row, 0);
  __syncthreads();
  const int L = s_len;
  if (L < 0 || L > p.max_pages * kPage) {   // not a length: the row stays as it was
    if (threadIdx.x == 0) {
      atomicExch(p.seq_lens + row, L);
      atomicOr(p.flags, kFlagBadLen);
    }
    return;
  }
  const int n = pages_of(L);
  for (int j = threadIdx.x; j < n; j += kThreads) {
    const int page = p.block_table[(int64_t)row * p.max_pages + j];
    if ((uint32_t)page >= (uint32_t)p.num_pages) {
      atomicOr(p.flags, kFlagBadPage);
    } else if (atomicSub(p.refs + page, 1) <= 0) {   // nobody held it
      atomicAdd(p.refs + page, 1);
      atomicOr(p.flags, kFlagBadPage);
    }
  }
}

// ---------------------------------------------------------------- fork

// Which forks stand, and the page of each one's partial last page: fork_full[f] = the full
// pages that are shared (-1: the fork is refused), list_src / list_dst[f] the pages to copy
// (-1: none).
__global__ __launch_bounds__(kMgr) void page_fork_kernel(const PageParams p) {
  __shared__ Pool s_pool;
  __shared__ int s_claim[kMaxBatch];   // the first fork that names a row as its child
  const int tid = threadIdx.x, cap = p.max_pages * kPage;
  const int per = (p.count + kMgr - 1) / kMgr, f0 = tid * per, f1 = min(f0 + per, p.count);
  Counts counts;
  counts.load(p, uni(tid >> 6));
  for (int i = tid; i < p.batch; i += kMgr) s_claim[i] = 0x7fffffff;
  __syncthreads();
  int parent[kPerThread], child[kPerThread], len[kPerThread];   // len -1: refused
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int f = f0 + i;
    parent[i] = child[i] = 0;
    len[i] = -1;
    if (f >= f1) continue;
    const int a = p.list_a[f], c = p.list_b[f];
    if ((uint32_t)a >= (uint32_t)p.batch || (uint32_t)c >= (uint32_t)p.batch || a == c) {
      bad = true;
      continue;
    }
    parent[i] = a;
    child[i] = c;
    const int L = p.seq_lens[a];
    // The child has to be empty, or its pages would be lost.
    if (L < 0 || L > cap || p.seq_lens[c] != 0)
      bad = true;
    else
      len[i] = L;
    atomicMin(&s_claim[c], f);
  }
  __syncthreads();   // every length has been read
  int sum = 0, all;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    if (f0 + i < f1 && len[i] >= 0 && s_claim[child[i]] != f0 + i) {
      len[i] = -1;
      bad = true;
    }
    sum += len[i] > 0 && len[i] % kPage != 0;
  }
  Mask mask;
  const int nfree = read_pool(p, s_pool, mask, counts);
  int run = block_before(sum, s_pool.tmp, &all);
  bool out = false;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int f = f0 + i;
    if (f >= f1) continue;
    int src = -1, dst = -1, full = len[i] < 0 ? -1 : len[i] / kPage;
    if (len[i] > 0 && len[i] % kPage != 0) {
      const int k = run++;
      if (k < nfree) {
        src = p.block_table[(int64_t)parent[i] * p.max_pages + full];
        dst = mask.page_of(k);
        p.block_table[(int64_t)child[i] * p.max_pages + full] = dst;
        p.refs[dst] = 1;
        if ((uint32_t)src >= (uint32_t)p.num_pages) {   // nothing to copy from
          src = -1;
          atomicOr(p.flags, kFlagBadPage);
        }
      } else {
        full = -1;
        out = true;
      }
    }
    if (full >= 0) p.seq_lens[child[i]] = len[i];
    p.fork_full[f] = full;
    p.list_src[f] = src;
    p.list_dst[f] = dst;
  }
  if (bad) atomicOr(p.flags, kFlagBadLen);
  if (out) atomicOr(p.flags, kFlagNoPages);
}

// ---------------------------------------------------------------- copies

// Copy page src over page dst in caches [first, last) by the workgroup.  A wave takes runs of
// 64 chunks of 16 bytes (a page of a cache is a multiple of that), kU of them in flight
// whichever cache they are in.  ONCE: every page is read once, past the caches too (the
// compaction below 197 us a call, 192 so; a fork's parents are read by all of their children,
// 34 and 46).  The copies are written past the caches, which would only
// hold them in the way of the pages that are read again (fork below: 44.6 us a call, 35.5 so).
template <bool ONCE>
__device__ __forceinline__ void copy_page(const PageParams& p, int src, int dst, int first, int last) {
  constexpr int kU = 4;
  const int lane = threadIdx.x & 63, wave = uni((int)(threadIdx.x >> 6));
  const int runs = p.page_bytes >> 10, per_row = p.row_bytes >> 4, total = (last - first) * 2 * runs;
  for (int r0 = wave; r0 < total; r0 += kU * kWaves) {
    u32x4 v[kU];
#pragma unroll
    for (int k = 0; k < 2 * kU; ++k) {   // kU loads, then kU stores
      const int j = k % kU, r = r0 + j * kWaves;
      if (r >= total) continue;
      const int pool = r / runs, i = (r - pool * runs) * 64 + lane;
      int64_t at = (int64_t)i * 16;
      if (!p.linear) {
        const int row = i / per_row, c = i - row * per_row, g = row / kPage, s = row - g * kPage;
        at = (int64_t)g * p.stride_head + (int64_t)s * p.stride_slot + c * 16;
      }
      const PageCache& c = p.caches[first + (pool >> 1)];
      char* base = (pool & 1 ? c.v : c.k) + at;
      if (k < kU)
        v[j] = ONCE ? __builtin_nontemporal_load((const u32x4*)(base + (int64_t)src * p.stride_page))
                    : *(const u32x4*)(base + (int64_t)src * p.stride_page);
      else
        __builtin_nontemporal_store(v[j], (u32x4*)(base + (int64_t)dst * p.stride_page));
    }
  }
  for (int l = first; l < last; ++l) {
    const PageCache& c = p.caches[l];
    if (c.k_scale && (int)threadIdx.x < p.num_kv_heads) {
      const int64_t a = (int64_t)src * p.num_kv_heads + threadIdx.x, b = (int64_t)dst * p.num_kv_heads + threadIdx.x;
      c.k_scale[b] = c.k_scale[a];
      c.v_scale[b] = c.v_scale[a];
    }
  }
}

// Pages list_src -> list_dst of `count` pairs in layers of a few, one workgroup per (pair,
// layers) up to the grid.  Pairs with a page outside the pool are skipped and reported.
__global__ __launch_bounds__(kThreads) void page_copy_kernel(const PageParams p) {
  const int64_t items = (int64_t)p.count * p.layer_blocks;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int i = (int)(it / p.layer_blocks), part = (int)(it - (int64_t)i * p.layer_blocks);
    const int src = p.list_src[i], dst = p.list_dst[i];
    if ((uint32_t)src >= (uint32_t)p.num_pages || (uint32_t)dst >= (uint32_t)p.num_pages) {
      if (threadIdx.x == 0) atomicOr(p.flags, kFlagBadPage);
    } else if (src != dst) {
      copy_page<false>(p, src, dst, part * p.block_layers, min((part + 1) * p.block_layers, p.num_caches));
    }
  }
}

// The forks' table rows and references; with part > 0, their copies.
__global__ __launch_bounds__(kThreads) void page_fork_rows_kernel(const PageParams p) {
  // Contiguous items to an XCD: the children of one parent are neighbours, and all but the
  // first read its page from the L2 (256 children of 32 parents, 28 layers: 47 us a call
  // dealt round, 44.6 so).
  const int parts = 1 + p.layer_blocks;
  const int item = share_of_block(blockIdx.x, gridDim.x), f = item / parts, part = item - f * parts;
  if (part > 0) {
    const int src = p.list_src[f], dst = p.list_dst[f];
    if (src < 0 || dst < 0) return;
    copy_page<false>(p, src, dst, (part - 1) * p.block_layers, min(part * p.block_layers, p.num_caches));
    return;
  }
  const int full = p.fork_full[f];
  if (full <= 0 || !p.share) return;
  const int32_t* from = p.block_table + (int64_t)p.list_a[f] * p.max_pages;
  int32_t* to = p.block_table + (int64_t)p.list_b[f] * p.max_pages;
  for (int j = threadIdx.x; j < full; j += kThreads) {
    const int page = from[j];
    to[j] = page;
    if ((uint32_t)page < (uint32_t)p.num_pages)
      atomicAdd(p.refs + page, 1);
    else
      atomicOr(p.flags, kFlagBadPage);
  }
}

// ---------------------------------------------------------------- compaction

// With n live pages, the live pages at or above n move to the free ones below it, both in
// ascending order: the moves (list_src / list_dst, *count_out of them), the pages' new
// numbers (map, at the moved pages) and the moved references.
__global__ __launch_bounds__(kMgr) void page_compact_kernel(const PageParams p) {
  __shared__ Pool s_pool;
  Mask mask;
  Counts c;
  c.load(p, uni((int)(threadIdx.x >> 6)));
  const int nfree = read_pool(p, s_pool, mask, c), n = p.num_pages - nfree, tid = threadIdx.x;
  // Free pages below n: those before n's word, and in it.
  const int wn = n >> 6, gn = wn / p.group_words;
  int below = s_pool.before[min(gn, kGroups)];
  for (int w = gn * p.group_words; w < wn; ++w) below += __builtin_popcountll(mask.words[w]);
  if ((n & 63) != 0) below += __builtin_popcountll(mask.words[wn] & ((1ull << (n & 63)) - 1));
  if (p.in_lds)
    for (int w = tid; w < p.words; w += kMgr) p.mask[w] = s_pool.words[w];
  if (tid == 0) {
    *p.count_out = below;
    *p.live_out = n;
  }
  // As many live pages at or above n, the j-th of them to the j-th free page.
  if (p.in_lds) {
    // Lane l of a wave has page l of a word: its rank among the free pages, or the live ones, is
    // its place in the list (7,534 pages, 1,900 moves: 11.1 us with the search below, 8.0 so).
    const int lane = tid & 63;
    for (int w = uni(tid >> 6); w < p.words; w += kMgrWaves) {
      const uint64_t m = s_pool.words[w];
      const int page = w * 64 + lane, before = s_pool.before[w] + __builtin_popcountll(m & ((1ull << lane) - 1));   // free ones
      if (m >> lane & 1) {
        if (page < n) p.list_dst[before] = page;
      } else if (page >= n && page < p.num_pages) {
        p.list_src[page - before - (n - below)] = page;
      }
    }
    __syncthreads();
    for (int j = tid; j < below; j += kMgr) {
      const int src = p.list_src[j], dst = p.list_dst[j];
      p.map[src] = dst;
      p.refs[dst] = p.refs[src];
      p.refs[src] = 0;
    }
    return;
  }
  // The j-th live one: page q where n + j + (free pages in [n, q)) = q, found among the words
  // from n's on by counting live pages.
  for (int j = tid; j < below; j += kMgr) {
    int lo = gn, hi = kGroups;   // live pages below group x: min(64 per x, num_pages) - before[x]
    const int want = (n - below) + j;   // live pages before the one looked for
    auto live_before = [&](int gr) { return (int)min((int64_t)gr * p.group_words * 64, (int64_t)p.num_pages) - s_pool.before[gr]; };
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (live_before(mid) <= want) lo = mid; else hi = mid;
    }
    int k = want - live_before(lo), w = lo * p.group_words;
    uint64_t m;
    for (;; ++w) {
      m = ~mask.words[w];
      const int64_t rest = (int64_t)p.num_pages - (int64_t)w * 64;
      if (rest < 64) m &= (1ull << rest) - 1;
      const int c = __builtin_popcountll(m);
      if (k < c) break;
      k -= c;
    }
    const int src = w * 64 + select_bit(m, k), dst = mask.page_of(j);
    p.list_src[j] = src;
    p.list_dst[j] = dst;
    p.map[src] = dst;
    p.refs[dst] = p.refs[src];
    p.refs[src] = 0;
  }
}

// The table's entries follow the moves; then the moves' copies, whose number only the
// device knows, dealt over the grid (16 layers, 980 MB read and written: 213 us a call with
// 2048 workgroups and two layers to each, 196 with one for every copy there may be and
// one layer; a copy of one buffer to another takes 198).
__global__ __launch_bounds__(kThreads) void page_move_kernel(const PageParams p) {
  const int n = *p.live_out;
  if (p.share) {
    for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
      const int L = p.seq_lens[b];
      if (L < 0 || L > p.max_pages * kPage) {
        if (threadIdx.x == 0) atomicOr(p.flags, kFlagBadLen);
        continue;
      }
      int32_t* row = p.block_table + (int64_t)b * p.max_pages;
      for (int j = threadIdx.x; j < pages_of(L); j += kThreads) {
        const int page = row[j];
        // A page out of the pool, or one that a row names and nothing counts: below n too, where
        // a moved page may just have taken its place.
        if ((uint32_t)page >= (uint32_t)p.num_pages || (p.mask[page >> 6] >> (page & 63) & 1))
          atomicOr(p.flags, kFlagBadPage);
        else if (page >= n)
          row[j] = p.map[page];
      }
    }
  }
  const int64_t items = (int64_t)*p.count_out * p.layer_blocks;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int i = (int)(it / p.layer_blocks), part = (int)(it - (int64_t)i * p.layer_blocks);
    copy_page<true>(p, p.list_src[i], p.list_dst[i], part * p.block_layers, min((part + 1) * p.block_layers, p.num_caches));
  }
}

int mask_first(const PageParams& p, hipStream_t st) {
  if (p.in_lds) return 0;
  hipLaunchKernelGGL(page_mask_kernel, dim3((p.words + p.group_words - 1) / p.group_words), dim3(kThreads), 0, st, p);
  return (int)hipGetLastError();
}

}  // namespace

int launch_page_grow(const PageParams& p, void* stream) {
  if (const int e = mask_first(p, (hipStream_t)stream)) return e;
  hipLaunchKernelGGL(page_grow_kernel, dim3(1), dim3(kMgr), 0, (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

int launch_page_release(const PageParams& p, void* stream) {
  hipLaunchKernelGGL(page_release_kernel, dim3(p.count), dim3(kThreads), 0, (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

int launch_page_fork(const PageParams& p, void* stream) {
  if (const int e = mask_first(p, (hipStream_t)stream)) return e;
  hipLaunchKernelGGL(page_fork_kernel, dim3(1), dim3(kMgr), 0, (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

int launch_page_fork_rows(const PageParams& p, void* stream) {
  hipLaunchKernelGGL(page_fork_rows_kernel, dim3(p.count * (1 + p.layer_blocks)), dim3(kThreads), 0, (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

int launch_page_compact(const PageParams& p, void* stream) {
  if (const int e = mask_first(p, (hipStream_t)stream)) return e;
  hipLaunchKernelGGL(page_compact_kernel, dim3(1), dim3(kMgr), 0, (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

int launch_page_move(const PageParams& p, int grid, void* stream) {
  hipLaunchKernelGGL(page_move_kernel, dim3(grid), dim3(kThreads), 0, (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

int launch_page_copy(const PageParams& p, int grid, void* stream) {
  hipLaunchKernelGGL(page_copy_kernel, dim3(grid), dim3(kThreads), 0, (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

}  // namespace rlda
