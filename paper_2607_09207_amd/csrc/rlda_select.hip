// Which pages of a long cache are read, and which are kept, for gfx950: the bounds of each
// page's keys, the choice of pages by them for every query row, and the eviction of the pages
// that got the least weight.
//
// Bounds.  For the keys k_t of a page and a KV head, s = max |k| / 127 and, per element,
//   hi = min(ceil(max_t k_t / s), 127),  lo = max(floor(min_t k_t / s), -127)      (8 bits each)
// so that s lo <= k_t <= s hi.  A query's score with any of these keys is then at most
// s sum_d max(q_d lo_d, q_d hi_d) = s (min(q, 0) . lo + max(q, 0) . hi): one product of length
// 2 d a page, over 1/32 of the bytes that its bf16 keys and values have.
//
// Choice.  q is rounded to 8 bits as well, q8 = rint(q / sq) with sq = max |q| / 127 a (row,
// head), so the product is one of whole numbers below 2^22: exact in whatever order the matrix
// cores add it, and the choice is the same on every run and for every cut.  (With sums rounded
// in 32 bits, pages near the border would come and go with the order.)  A page's score for a KV
// head is s max_i (u_i sq_i) over its query heads, in fp32 in that order.  The `budget` best
// pages are found by the digits of their order keys, in LDS.
//
// Eviction.  The same search over the weights that the pages got (rl_decode_attn_run_weighed).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rlda_device.h"
#include "rlda_params.h"

namespace rlda {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kSel = 512;                  // threads of a workgroup that chooses
constexpr int kSelWaves = kSel / 64;
constexpr int kSelSmall = 8192;            // order keys in LDS: four such workgroups to a CU
constexpr int kDigits = 256;

__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < __builtin_huge_valf(); }

// Unsigned keys in the order of floats, both zeros alike; NaN above all.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0xFFFFFFFFu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// ---------------------------------------------------------------- bounds

// bf16 pairs to signed 16-bit integers of their order and back.
__device__ __forceinline__ uint32_t ordered(uint32_t w) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  const s16x2 x = __builtin_bit_cast(s16x2, w);
  return w ^ (__builtin_bit_cast(uint32_t, x >> (short)15) & 0x7FFF7FFFu);
}
__device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
}
__device__ __forceinline__ uint32_t pair_min(uint32_t a, uint32_t b) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
}

// One wave a (page, KV head).  A load of the wave covers 64 / LPR rows of the page, a lane E
// elements of one; the rows' largest and smallest values meet by exchanges between the lanes
// of the same elements.  fp8 values become bf16 (exactly), and bf16 values are compared as
// integers, two at a time.  Bandwidth bounds it for whole prompts, latency for a step.
template <int D, KvKind KIND>
__global__ __launch_bounds__(kThreads) void page_bounds_kernel(const SelectParams p) {
  constexpr int EB = KIND == KvKind::F32 ? 4 : KIND == KvKind::BF16 ? 2 : 1;
  constexpr int E = 16 / EB, LPR = D / E, RPI = 64 / LPR, NI = kPage / RPI;
  const int lane = threadIdx.x & 63, wave = uni((int)(threadIdx.x >> 6));
  const int b = blockIdx.y, cap = p.max_pages * kPage;
  int L = p.seq_lens[b];
  const int first = p.first ? p.first[b] : L - 1;
  if (L < 0 || L > cap || (p.first && (first < 0 || first > L))) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.flags, kFlagBadLen);
    if (L < 0 || L > cap) return;
  }
  if (L == 0) return;
  const int j0 = min(max(first, 0), L) / kPage, npages = (L + kPage - 1) / kPage;
  const int units = (npages - j0) * p.num_kv_heads;
  const int row = lane / LPR, col = lane % LPR;
  for (int u = blockIdx.x * kWaves + wave; u < units; u += gridDim.x * kWaves) {
    const int j = j0 + (int)((uint32_t)u / (uint32_t)p.num_kv_heads), g = u - (j - j0) * p.num_kv_heads;
    const int pid = uni(p.block_table[(int64_t)b * p.max_pages + j]);
    if ((unsigned)pid >= (unsigned)p.num_pages) {
      if (lane == 0) atomicOr(p.flags, kFlagBadPage);
      continue;
    }
    const int val = min(kPage, L - j * kPage);
    const char* base = (const char*)p.k + (int64_t)pid * p.stride_page + (int64_t)g * p.stride_head;
    u32x4 x[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = min(i * RPI + row, val - 1);   // (rows past the end: the last one again)
      x[i] = __builtin_nontemporal_load((const u32x4*)(base + (int64_t)r * p.stride_slot + col * 16));
    }
    float hi[E], lo[E], amax = 0.f;
    bool odd = false;
    if constexpr (KIND == KvKind::F32) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        hi[e] = lo[e] = __uint_as_float(x[0][e]);
        odd |= !finite(hi[e]);
#pragma unroll
        for (int i = 1; i < NI; ++i) {
          const float v = __uint_as_float(x[i][e]);
          odd |= !finite(v);
          hi[e] = fmaxf(hi[e], v);
          lo[e] = fminf(lo[e], v);
        }
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) {
          hi[e] = fmaxf(hi[e], __shfl_xor(hi[e], o));
          lo[e] = fminf(lo[e], __shfl_xor(lo[e], o));
        }
        amax = fmaxf(amax, fmaxf(__builtin_fabsf(hi[e]), __builtin_fabsf(lo[e])));
      }
    } else {
      constexpr int W = E / 2;   // pairs of a lane
      uint32_t mx[W], mn[W];
      u16x2 top = {0, 0};
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int w = 0; w < W; ++w) {
          uint32_t v;
          if constexpr (KIND == KvKind::BF16)
            v = x[i][w];
          else
            v = fp8x2_to_bf16x2(x[i][w / 2], (w & 1) != 0);
          top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, v & 0x7FFF7FFFu));
          v = ordered(v);
          mx[w] = i == 0 ? v : pair_max(mx[w], v);
          mn[w] = i == 0 ? v : pair_min(mn[w], v);
        }
      odd = not_finite(top);
      const float ks = KIND == KvKind::FP8 ? p.k_scale[(int64_t)pid * p.num_kv_heads + g] : 1.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) {
          mx[w] = pair_max(mx[w], (uint32_t)__shfl_xor((int)mx[w], o));
          mn[w] = pair_min(mn[w], (uint32_t)__shfl_xor((int)mn[w], o));
        }
        const uint32_t h = ordered(mx[w]), l = ordered(mn[w]);
        hi[2 * w] = __uint_as_float(h << 16);
        hi[2 * w + 1] = __uint_as_float(h & 0xFFFF0000u);
        lo[2 * w] = __uint_as_float(l << 16);
        lo[2 * w + 1] = __uint_as_float(l & 0xFFFF0000u);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if constexpr (KIND == KvKind::FP8) {   // a key is the stored value times the page's scale
          const float a = hi[e] * ks, c = lo[e] * ks;
          hi[e] = ks < 0.f ? c : a;
          lo[e] = ks < 0.f ? a : c;
          odd |= !finite(a) || !finite(c);
        }
        amax = fmaxf(amax, fmaxf(__builtin_fabsf(hi[e]), __builtin_fabsf(lo[e])));
      }
    }
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
    odd = __builtin_amdgcn_ballot_w64(odd) != 0;
    const float s = odd ? __builtin_huge_valf() : amax / 127.f;
    // The first group of lanes writes the lower bounds, the second the upper ones.
    const int64_t at = (int64_t)pid * p.num_kv_heads + g;
    if constexpr (RPI >= 2) {
      if (row < 2) {
        uint32_t out[E / 4];
#pragma unroll
        for (int w = 0; w < E / 4; ++w) {
          uint32_t word = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = (row ? hi[4 * w + e] : lo[4 * w + e]) / s;
            const float r = row ? fminf(__builtin_ceilf(v), 127.f) : fmaxf(__builtin_floorf(v), -127.f);
            const int byte = s > 0.f && !odd ? (int)r : 0;
            word |= (uint32_t)(byte & 255) << (8 * e);
          }
          out[w] = word;
        }
        uint32_t* dst = (uint32_t*)(p.bounds + (at * 2 + row) * D + col * E);
#pragma unroll
        for (int w = 0; w < E / 4; ++w) dst[w] = out[w];
      }
    }
    static_assert(RPI >= 2, "two groups of lanes write a page's bounds");
    if (lane == 0) p.bound_scale[at] = s;
  }
}

// ---------------------------------------------------------------- the rows of a call

struct RowAt {
  int seq;      // -1: a row of no sequence
  int tokens;   // that it sees
};

// The sequence and the visible tokens of query row r (the same for all lanes of a wave): the
// last entry of q_start up to r, 64 entries a step.
__device__ __forceinline__ RowAt row_at(const SelectParams& p, int r) {
  const int lane = threadIdx.x & 63, cap = p.max_pages * kPage;
  if (!p.q_start) {
    const int L = uni(p.seq_lens[r]);
    if ((L < 0 || L > cap) && lane == 0) atomicOr(p.flags, kFlagBadLen);
    return {r, min(max(L, 0), cap)};
  }
  int lo = 0, hi = p.batch + 1;   // entries below lo are at most r
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64, at = lo + (lane + 1) * step - 1;
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(at < hi && p.q_start[min(at, p.batch)] <= r));
    lo += c * step;
    hi = min(hi, lo + step - 1);
  }
  const int seq = uni(lo) - 1;
  if (seq < 0 || seq >= p.batch) return {-1, 0};
  const int q0 = uni(p.q_start[seq]), q1 = uni(p.q_start[seq + 1]), L = uni(p.seq_lens[seq]);
  const bool ok = q0 >= 0 && r >= q0 && r < q1 && q1 <= p.total_q;
  if ((!ok || L < 0 || L > cap || q1 - q0 > L) && lane == 0) atomicOr(p.flags, kFlagBadLen);
  if (!ok) return {-1, 0};
  return {seq, max(min(max(L, 0), cap) - (q1 - 1 - r), 0)};
}

// ---------------------------------------------------------------- the best of many

// What a workgroup of kSel threads shares while it looks for the K largest keys.
struct Search {
  int hist[kDigits];
  uint32_t low[kSelWaves], high[kSelWaves];
  int sum[kSelWaves], ties[kSelWaves];
  int digit, above, in;
};

// The K-th largest of keys[lo .. hi) (0 < K < hi - lo): those above *at are taken, and the
// first *ties of those equal to it.  By digits from the highest bit in which keys differ.
__device__ __forceinline__ void kth_largest(const uint32_t* keys, int lo, int hi, int K, Search& s, uint32_t* at, int* ties) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
  for (int j = lo + tid; j < hi; j += kSel) {
    kmin = min(kmin, keys[j]);
    kmax = max(kmax, keys[j]);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    kmin = min(kmin, (uint32_t)__shfl_xor((int)kmin, o));
    kmax = max(kmax, (uint32_t)__shfl_xor((int)kmax, o));
  }
  if (lane == 0) {
    s.low[wave] = kmin;
    s.high[wave] = kmax;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    kmin = min(kmin, s.low[w]);
    kmax = max(kmax, s.high[w]);
  }
  int bits = kmin == kmax ? 0 : 32 - __builtin_clz(kmin ^ kmax);   // still undecided
  uint32_t prefix = bits == 32 ? 0u : kmin >> bits << bits;
  *ties = K;
  while (bits > 0) {
    const int shift = max(bits - 8, 0);
    if (tid < kDigits) s.hist[tid] = 0;
    __syncthreads();
    for (int j = lo + tid; j < hi; j += kSel) {
      const uint32_t k = keys[j];
      if (bits == 32 || ((k ^ prefix) >> bits) == 0) atomicAdd(&s.hist[(k >> shift) & ((1u << (bits - shift)) - 1u)], 1);
    }
    __syncthreads();
    // Counts from the largest digit down, over four waves.
    if (tid < kDigits) {
      const int n = s.hist[kDigits - 1 - tid], x = wave_scan(n);
      if (lane == 63) s.sum[wave] = x;
      s.hist[kDigits - 1 - tid] = x - n;   // of its wave's larger digits
    }
    __syncthreads();
    if (tid < kDigits) {
      int before = s.hist[kDigits - 1 - tid];
      for (int w = 0; w < wave; ++w) before += s.sum[w];
      int after = 0;   // with this digit: the next thread's count, or its wave's total
      after = __shfl_down(s.hist[kDigits - 1 - tid], 1);
      if (lane == 63) after = s.sum[wave];
      for (int w = 0; w < wave; ++w) after += s.sum[w];
      if (before < K && K <= after) {
        s.digit = kDigits - 1 - tid;
        s.above = before;
        s.in = after - before;
      }
    }
    __syncthreads();
    prefix |= (uint32_t)s.digit << shift;
    K -= s.above;
    bits = shift;
    *ties = K;
    if (s.in == K) {   // all of them: whatever their lower bits are
      *ties = 0x7FFFFFFF;
      break;
    }
  }
  *at = prefix;
}

// Calls take(j, rank) for the pages j of [0, n) that are chosen, in order, and leave(j) for the
// others: those of the first `sink` and the last `recent`, and of the rest the largest keys.
// Whatever read(j) reads is read before anything is written by take or leave of pages up to j.
template <class Read, class Take, class Leave>
__device__ __forceinline__ int choose(const uint32_t* keys, int n, int budget, int sink, int recent, Search& s, Read read,
                                      Take take, Leave leave) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int K = budget - sink - recent;
  uint32_t at = 0xFFFFFFFFu;
  int ties = 0;
  if (K > 0) kth_largest(keys, sink, n - recent, K, s, &at, &ties);
  int taken = 0, tied = 0;   // in the pages before
  for (int j0 = 0; j0 < n; j0 += kSel) {
    const int j = j0 + tid;
    const bool kept = j < n && (j < sink || j >= n - recent);
    const bool rest = j < n && !kept && K > 0;
    const uint32_t k = rest ? keys[j] : 0u;
    const bool sure = kept || (rest && k > at), tie = rest && k == at;
    const auto x = read(j);
    const uint64_t below = (1ull << lane) - 1, ms = __builtin_amdgcn_ballot_w64(sure), mt = __builtin_amdgcn_ballot_w64(tie);
    if (lane == 0) {
      s.sum[wave] = __builtin_popcountll(ms);
      s.ties[wave] = __builtin_popcountll(mt);
    }
    __syncthreads();
    // Before this wave: the sure ones, and as many ties as were wanted.
    int sures = 0, tbefore = tied, alls = 0, allt = 0;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) {
      sures += w < wave ? s.sum[w] : 0;
      tbefore += w < wave ? s.ties[w] : 0;
      alls += s.sum[w];
      allt += s.ties[w];
    }
    const int mine = tbefore + __builtin_popcountll(mt & below);   // ties before this page
    const bool chosen = sure || (tie && mine < ties);
    const int rank = taken + sures + __builtin_popcountll(ms & below) + (min(mine, ties) - min(tied, ties));
    if (chosen)
      take(j, rank, x);
    else if (j < n)
      leave(j, x);
    taken += alls + (min(tied + allt, ties) - min(tied, ties));
    tied += allt;
    __syncthreads();   // the counts are used again
  }
  return taken;
}

// ---------------------------------------------------------------- choice

template <int CTRL>
__device__ __forceinline__ float row_move(float x) {
  const int v = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, true));
}
// Maximum over the 16 lanes of a row.
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, row_move<0x128>(x));   // row_ror:8, 4, 2, 1
  x = fmaxf(x, row_move<0x124>(x));
  x = fmaxf(x, row_move<0x122>(x));
  return fmaxf(x, row_move<0x121>(x));
}

// The query heads of a KV head as the second operand of 16x16x64 products, in 8 bits: lane
// 16 qg + i holds head i's elements 64 c + 16 qg .. + 15 (min(q, 0) for the lower bounds, then
// max(q, 0) for the upper ones), and its scale.
template <int D, bool QF32>
struct QBytes {
  static constexpr int C = D / 64;
  i32x4 v[2 * C];
  float scale;   // -inf: no head

  __device__ __forceinline__ void load(const SelectParams& p, int row, int g, int lane) {
    const int i = lane & 15, qg = lane >> 4;
    float x[C][16], amax = 0.f;
    bool odd = false;
    const int qh = i < p.group ? p.q_head[g * p.group + i] : 0;
    const int64_t at = ((int64_t)row * p.num_q_heads + qh) * D + 16 * qg;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (QF32) {
#pragma unroll
        for (int e = 0; e < 16; e += 4) *(f32x4*)&x[c][e] = *(const f32x4*)((const float*)p.q + at + 64 * c + e);
      } else {
#pragma unroll
        for (int e = 0; e < 16; e += 8) {
          const u32x4 w = *(const u32x4*)((const uint16_t*)p.q + at + 64 * c + e);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            x[c][e + 2 * k] = __uint_as_float(w[k] << 16);
            x[c][e + 2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        odd |= !finite(x[c][e]);
        amax = fmaxf(amax, __builtin_fabsf(x[c][e]));
      }
    }
    amax = fmaxf(amax, __shfl_xor(amax, 16));
    amax = fmaxf(amax, __shfl_xor(amax, 32));
    int any = odd;
    any |= __shfl_xor(any, 16);
    any |= __shfl_xor(any, 32);
    const float s = any ? 0.f : amax / 127.f;   // (a query of infinities or NaN says nothing about pages)
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t neg = 0, pos = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int q = s > 0.f ? (int)__builtin_rintf(x[c][4 * w + e] / s) : 0;
          neg |= (uint32_t)(min(q, 0) & 255) << (8 * e);
          pos |= (uint32_t)(max(q, 0) & 255) << (8 * e);
        }
        v[c][w] = (int)neg;
        v[C + c][w] = (int)pos;
      }
    scale = i < p.group ? s : neg_inf();
  }
};

// Order keys of the pages [j0, j1) of a (row, KV head), by the whole workgroup: store(j, key).
// A wave takes 64 pages at a time, four tiles of 16 whose loads are in flight together.
template <int D, bool QF32, class Store>
__device__ __forceinline__ void score_pages(const SelectParams& p, const QBytes<D, QF32>& q, int seq, int g, int j0, int j1,
                                            float (*s_val)[64], Store store) {
  constexpr int NC = 2 * D / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), i = lane & 15, qg = lane >> 4;
  const int32_t* bt = p.block_table + (int64_t)seq * p.max_pages;
  for (int base = j0 + 64 * wave; base < j1; base += kSel) {
    const int j = base + lane;
    int pid = j < j1 ? bt[j] : -1;
    if (j < j1 && (unsigned)pid >= (unsigned)p.num_pages) {
      atomicOr(p.flags, kFlagBadPage);
      pid = -1;
    }
    const float scale = pid >= 0 ? p.bound_scale[(int64_t)pid * p.num_kv_heads + g] : 0.f;
    i32x4 a[4][NC];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int pt = __shfl(pid, 16 * t + i);
#pragma unroll
      for (int c = 0; c < NC; ++c) a[t][c] = i32x4{0, 0, 0, 0};
      if (pt >= 0) {
        const int8_t* src = p.bounds + ((int64_t)pt * p.num_kv_heads + g) * (2 * D) + 16 * qg;
#pragma unroll
        for (int c = 0; c < NC; ++c) a[t][c] = *(const i32x4*)(src + 64 * c);
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      i32x4 u = {0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < NC; ++c) u = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[t][c], q.v[c], u, 0, 0, 0);
      // Lane 16 qg + i: page 4 qg + r with head i.
      float m[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) m[r] = row_max(i < p.group ? (float)u[r] * q.scale : neg_inf());
      const float mine = i == 0 ? m[0] : i == 1 ? m[1] : i == 2 ? m[2] : m[3];
      if (i < 4) s_val[wave][16 * t + 4 * qg + i] = mine;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const float x = s_val[wave][lane] * scale;
    __builtin_amdgcn_wave_barrier();
    // Keys that are not finite: their page is looked at first.  A page that is not there: last.
    if (j < j1) store(j, pid < 0 ? 0u : finite(scale) ? order_key(x) : 0xFFFFFFFFu);
  }
}

// One workgroup, or p.pieces of them, a (row, KV head).  With several, the one that finishes
// last gathers the others' keys.
template <int D, bool QF32, int CAP>
__global__ __launch_bounds__(kSel) void select_pages_kernel(const SelectParams p) {
  __shared__ uint32_t s_key[CAP];
  __shared__ float s_val[kSelWaves][64];
  __shared__ Search s;
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 63;
  const int seg = (int)(blockIdx.x / (uint32_t)p.pieces), piece = blockIdx.x - seg * p.pieces;
  const int row = seg / p.num_kv_heads, g = seg - row * p.num_kv_heads;
  const RowAt at = row_at(p, row);
  if (at.seq < 0) return;
  const int n = (at.tokens + kPage - 1) / kPage;
  int32_t* out = p.pages + (int64_t)seg * p.budget;
  if (n <= p.budget) {   // all of them
    if (piece != 0) return;
    for (int j = tid; j < p.budget; j += kSel) out[j] = j < n ? j : -1;
    if (tid == 0) p.counts[seg] = n;
    return;
  }
  QBytes<D, QF32> q;
  q.load(p, row, g, lane);
  if (p.pieces == 1) {
    score_pages<D, QF32>(p, q, at.seq, g, 0, n, s_val, [&](int j, uint32_t k) { s_key[j] = k; });
  } else {
    const int per = ((n + p.pieces - 1) / p.pieces + 63) / 64 * 64;
    uint32_t* keys = p.keys + (int64_t)seg * p.max_pages;
    score_pages<D, QF32>(p, q, at.seq, g, min(piece * per, n), min((piece + 1) * per, n), s_val, [&](int j, uint32_t k) {
      __hip_atomic_store(keys + j, k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    __builtin_amdgcn_s_waitcnt(0);   // this wave's stores have completed
    __syncthreads();
    if (tid == 0) {
      const uint32_t old = atomicAdd(p.counters + seg, 1u);
      if (old >= (uint32_t)p.pieces) atomicOr(p.flags, kFlagStaleState);
      s_last = old + 1u == (uint32_t)p.pieces;
      if (s_last) atomicExch(p.counters + seg, 0u);
    }
    __syncthreads();
    if (!s_last) return;
    for (int j = tid; j < n; j += kSel) s_key[j] = __hip_atomic_load(keys + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  const int count = choose(
      s_key, n, p.budget, p.sink, p.recent, s, [](int) { return 0; }, [&](int j, int rank, int) { out[rank] = j; },
      [](int, int) {});
  if (tid == 0) p.counts[seg] = count;
}

// ---------------------------------------------------------------- eviction

// One workgroup a row.  Entries move towards the front, kSel at a time: what a step writes lies
// at or before what it has read.
template <int CAP>
__global__ __launch_bounds__(kSel) void page_evict_kernel(const SelectParams p) {
  __shared__ uint32_t s_key[CAP];
  __shared__ Search s;
  const int tid = threadIdx.x, b = blockIdx.x;
  const int L = p.seq_lens[b];
  const int n = (L + kPage - 1) / kPage;
  const bool bad = L < 0 || L > p.max_pages * kPage;
  if (bad && tid == 0) atomicOr(p.flags, kFlagBadLen);
  if (bad || n <= p.budget) {
    if (tid == 0) p.dropped[b] = 0;
    return;
  }
  int32_t* table = p.block_table + (int64_t)b * p.max_pages;
  float* w = p.weights + (int64_t)b * p.max_pages;
  for (int j = tid; j < n; j += kSel) s_key[j] = order_key(w[j]);
  __syncthreads();
  struct Entry {
    int page;
    float weight;
  };
  choose(
      s_key, n, p.budget, p.sink, p.recent, s, [&](int j) { return j < n ? Entry{table[j], w[j]} : Entry{0, 0.f}; },
      [&](int, int rank, Entry x) {
        table[rank] = x.page;
        w[rank] = x.weight;
      },
      [&](int, Entry x) {
        if ((uint32_t)x.page >= (uint32_t)p.num_pages) {
          atomicOr(p.flags, kFlagBadPage);
        } else if (atomicSub(p.refs + x.page, 1) <= 0) {   // nobody held it
          atomicAdd(p.refs + x.page, 1);
          atomicOr(p.flags, kFlagBadPage);
        }
      });
  for (int j = p.budget + tid; j < n; j += kSel) w[j] = 0.f;   // (choose ends with a barrier)
  if (tid == 0) {
    p.dropped[b] = n - p.budget;
    p.seq_lens[b] = L - kPage * (n - p.budget);
  }
}

template <int D, bool QF32>
void launch_select_t(const SelectParams& p, hipStream_t st) {
  const dim3 grid((uint32_t)p.total_q * p.num_kv_heads * p.pieces);
  if (p.max_pages <= kSelSmall)
    hipLaunchKernelGGL((select_pages_kernel<D, QF32, kSelSmall>), grid, dim3(kSel), 0, st, p);
  else
    hipLaunchKernelGGL((select_pages_kernel<D, QF32, kSelectMaxPages>), grid, dim3(kSel), 0, st, p);
}

}  // namespace

int launch_page_bounds(KvKind kind, int head_dim, const SelectParams& p, void* stream) {
  // A wave a (page, KV head): enough of them for the last pages, or, without knowing the
  // lengths, for a batch's share of the GPU.
  const int64_t most = p.first ? (int64_t)p.max_pages * p.num_kv_heads : p.num_kv_heads;
  const int64_t share = 8192 / p.batch > 1 ? 8192 / p.batch : 1;
  int64_t x = (most + kWaves - 1) / kWaves;
  if (p.first && x > share) x = share;
  const dim3 grid((uint32_t)x, (uint32_t)p.batch);
  const hipStream_t st = (hipStream_t)stream;
#define RLDA_BOUNDS(D, KIND) hipLaunchKernelGGL((page_bounds_kernel<D, KIND>), grid, dim3(kThreads), 0, st, p)
  switch (kind) {
    case KvKind::BF16:
      if (head_dim == 128) RLDA_BOUNDS(128, KvKind::BF16); else RLDA_BOUNDS(64, KvKind::BF16);
      break;
    case KvKind::FP8:
      if (head_dim == 128) RLDA_BOUNDS(128, KvKind::FP8); else RLDA_BOUNDS(64, KvKind::FP8);
      break;
    case KvKind::F32:
      if (head_dim == 128) RLDA_BOUNDS(128, KvKind::F32); else RLDA_BOUNDS(64, KvKind::F32);
      break;
  }
#undef RLDA_BOUNDS
  return (int)hipGetLastError();
}

int launch_select_pages(bool q_f32, int head_dim, const SelectParams& p, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  if (q_f32) {
    if (head_dim == 128) launch_select_t<128, true>(p, st); else launch_select_t<64, true>(p, st);
  } else {
    if (head_dim == 128) launch_select_t<128, false>(p, st); else launch_select_t<64, false>(p, st);
  }
  return (int)hipGetLastError();
}

int launch_page_evict(const SelectParams& p, void* stream) {
  if (p.max_pages <= kSelSmall)
    hipLaunchKernelGGL(page_evict_kernel<kSelSmall>, dim3(p.batch), dim3(kSel), 0, (hipStream_t)stream, p);
  else
    hipLaunchKernelGGL(page_evict_kernel<kSelectMaxPages>, dim3(p.batch), dim3(kSel), 0, (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

}  // namespace rlda
