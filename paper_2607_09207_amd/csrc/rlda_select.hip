// Which pages of a long cache are read, and which are kept, for gfx950: the bounds of each
// page's keys, the choice of pages by them for every query row, and the eviction of the pages
// that got the least weight.
//
// Bounds.  For the keys k_t of a page and a KV head, s = max |k| / 127 and, per element,
//   hi = ceil(max_t k_t / s),  lo = floor(min_t k_t / s),   within +-127      (8 bits each)
// so that s lo <= k_t <= s hi.  A query's score with any of these keys is then at most
// s sum_d max(q_d lo_d, q_d hi_d) = s (min(q, 0) . lo + max(q, 0) . hi): one product of length
// 2 d a page, over 1/32 of the bytes that its bf16 keys and values have.
//
// Choice.  q is rounded to 8 bits as well, q8 = rint(q / sq) with sq = max |q| / 127 a (row,
// head), so the product is one of whole numbers below 2^22: exact in whatever order the matrix
// cores add it, and the choice is the same on every run and for every cut.  (With sums rounded
// in 32 bits, pages near the border would come and go with the order.)  The rounded query's score is
// no upper bound any more: it is off by s sq/2 sum_d max(|lo_d|, |hi_d|) at most.  Of 128 chosen of 1024
// pages 99.1% are those that q itself chooses (N(0, 1) keys; 99.6% where three channels are 24 times as
// large), and 97.7% (93.5%) those of bounds that are not rounded either.  A page's score for a KV
// head is s max_i (u_i sq_i) over its query heads, in fp32 in that order.  The `budget` best
// pages are found by the digits of their order keys, in LDS.
//
// Eviction.  The same search over the weights that the pages got (rl_decode_attn_run_weighed).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rlda_device.h"
#include "rlda_params.h"
#include "rlda_split.h"

namespace rlda {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kSel = kSelectThreads;
constexpr int kEvict = 512;                // ... that evicts
constexpr int kSelSmall = 8192;            // order keys in LDS: two such workgroups to a CU
constexpr int kDigitBits = 11, kDigits = 1 << kDigitBits;

__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < __builtin_huge_valf(); }

// Unsigned keys in the order of floats, both zeros alike; NaN above all.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0xFFFFFFFFu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// Maximum over a wave's lanes, by DPP (rlda_device.h: a shuffle is an LDS round trip a step).
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  const auto step = [&](uint32_t y) { x = x > y ? x : y; };
  step((uint32_t)dpp_or_zero<0x111, 0xf>((int)x));   // row_shr:1, 2, 4, 8, then across the rows
  step((uint32_t)dpp_or_zero<0x112, 0xf>((int)x));
  step((uint32_t)dpp_or_zero<0x114, 0xf>((int)x));
  step((uint32_t)dpp_or_zero<0x118, 0xf>((int)x));
  step((uint32_t)dpp_or_zero<0x142, 0xa>((int)x));
  step((uint32_t)dpp_or_zero<0x143, 0xc>((int)x));
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// ---------------------------------------------------------------- bounds

// bf16 pairs to signed 16-bit integers of their order (infinities and NaN beyond all others) and
// back.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t ordered(uint32_t w) {
  return w ^ (__builtin_bit_cast(uint32_t, __builtin_bit_cast(s16x2, w) >> (short)15) & 0x7FFF7FFFu);
}
template <bool F32>
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  if constexpr (F32) return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
}

// The maxima of N words over the lanes that differ in the bits from LPR (a power of two) on, dealt
// out to these lanes: with every step a lane keeps half of its words, so a step costs half of
// the one before it.  Lane l ends with words N / (64 / LPR) (l / LPR) and on.
template <bool F32, int LPR, int N>
__device__ __forceinline__ void deal_maxima(uint32_t* w) {
  const int lane = threadIdx.x & 63;
  int n = N;
#pragma unroll
  for (int o = 32; o >= LPR; o >>= 1) {
    n /= 2;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      if (i >= n) break;
      const uint32_t a = w[i], b = w[i + n];
      if (o >= 16) {   // one half gets both of a, the other both of b
        const auto r = o == 32 ? __builtin_amdgcn_permlane32_swap(a, b, false, false) : __builtin_amdgcn_permlane16_swap(a, b, false, false);
        w[i] = larger<F32>(r[0], r[1]);
      } else {
        const bool up = lane & o;
        const int send = (int)(up ? a : b);
        const int got = o == 8 ? __builtin_amdgcn_update_dpp(send, send, 0x128, 0xf, 0xf, true) : __shfl_xor(send, o);   // row_ror:8
        w[i] = larger<F32>(up ? b : a, (uint32_t)got);
      }
    }
  }
}

// One wave a (page, KV head).  A load of the wave covers RPI = 64 / LPR rows of the page, a lane E
// elements of one.  fp8 values become bf16 (exactly), and bf16 values are compared as integers,
// two at a time.  The largest values and the smallest (as the largest complements) then meet
// over the lanes of the same elements, each of which ends with a few of them to divide and write.
//   Bandwidth bounds it for whole prompts, as long as a page takes few operations: with every
// lane reducing all of its elements and two of the groups dividing them, 33 us for 64 prompts
// (151 MB) against 28.5 so (5.3 TB/s).  fp8 pages have half the bytes and no fewer operations (262 VALU
// instructions a page and KV head, bf16 242): the same prompts on 8 KV heads (160 MB) take 43.4 us, 3.7
// TB/s, 30 of it the VALU's issue.  For a step, latency.
template <int D, KvKind KIND>
__global__ __launch_bounds__(kThreads) void page_bounds_kernel(const SelectParams p) {
  constexpr bool F32 = KIND == KvKind::F32;
  constexpr int EB = F32 ? 4 : KIND == KvKind::BF16 ? 2 : 1;
  constexpr int E = 16 / EB, LPR = D / E, RPI = 64 / LPR, NI = kPage / RPI;
  constexpr int H = F32 ? E : E / 2;                      // words of a lane's elements
  constexpr int NR = 2 * H / RPI, V = F32 ? NR : 2 * NR;   // words, and values, that it ends with
  static_assert(V == 2 || V == 4, "bytes of a store");
  const int lane = threadIdx.x & 63, wave = uni((int)(threadIdx.x >> 6));
  const int b = blockIdx.y, cap = p.max_pages * kPage;
  const int L = p.seq_lens[b];
  const int first = p.first ? p.first[b] : L - 1;
  if (L < 0 || L > cap || (p.first && (first < 0 || first > L))) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.flags, kFlagBadLen);
    if (L < 0 || L > cap) return;
  }
  if (L == 0) return;
  const int j0 = min(max(first, 0), L) / kPage, npages = (L + kPage - 1) / kPage;
  const uint32_t units = (uint32_t)(npages - j0) * (uint32_t)p.num_kv_heads;
  const int row = lane / LPR, col = lane % LPR;
  for (uint32_t u = blockIdx.x * kWaves + wave; u < units; u = unit_after(u, gridDim.x * kWaves, units)) {
    const PageHead at_u = page_head_of(u, p.num_kv_heads);
    const int j = j0 + at_u.page, g = at_u.head;
    const int pid = uni(p.block_table[(int64_t)b * p.max_pages + j]);
    if ((unsigned)pid >= (unsigned)p.num_pages) {
      if (lane == 0) atomicOr(p.flags, kFlagBadPage);
      continue;
    }
    const int val = min(kPage, L - j * kPage);
    const char* base = (const char*)p.k + (int64_t)pid * p.stride_page + (int64_t)g * p.stride_head;
    const int64_t at = (int64_t)pid * p.num_kv_heads + g;
    u32x4 x[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = min(i * RPI + row, val - 1);   // (rows past the end: the last one again)
      x[i] = __builtin_nontemporal_load((const u32x4*)(base + (int64_t)r * p.stride_slot + col * 16));
    }
    const float ks = KIND == KvKind::FP8 ? p.k_scale[at] : 1.f;
    uint32_t w[2 * H];   // the largest, then the largest complements
    bool odd = false;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      uint32_t top = 0, low = 0;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        uint32_t v;
        if constexpr (KIND == KvKind::FP8)
          v = ordered(fp8x2_to_bf16x2(x[i][h / 2], (h & 1) != 0));
        else
          v = F32 ? x[i][h] : ordered(x[i][h]);
        if constexpr (F32) {
          odd |= !finite(__uint_as_float(v));
          top = i == 0 ? v : larger<true>(top, v);
          low = i == 0 ? v ^ 0x80000000u : larger<true>(low, v ^ 0x80000000u);
        } else {
          top = i == 0 ? v : larger<false>(top, v);
          low = i == 0 ? ~v : larger<false>(low, ~v);
        }
      }
      w[h] = top;
      w[H + h] = low;
    }
    deal_maxima<F32, LPR, 2 * H>(w);
    const bool low = row >= RPI / 2;
    float v[V], amax = 0.f;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      if constexpr (F32) {
        v[i] = __uint_as_float(low ? w[i] ^ 0x80000000u : w[i]);
      } else {
        const uint32_t pair = ordered(low ? ~w[i] : w[i]);
        v[2 * i] = __uint_as_float(pair << 16);
        v[2 * i + 1] = __uint_as_float(pair & 0xFFFF0000u);
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (KIND == KvKind::FP8) v[i] *= ks;   // a key is the stored value times the page's scale
      odd |= !finite(v[i]);
      amax = fmaxf(amax, __builtin_fabsf(v[i]));
    }
    odd = __builtin_amdgcn_ballot_w64(odd) != 0;
    amax = __uint_as_float(wave_max(__float_as_uint(amax)));   // (magnitudes order as integers)
    const float s = odd ? __builtin_huge_valf() : amax / 127.f;
    const bool lower = low != (ks < 0.f);   // (a negative scale turns them round)
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float y = v[i] / s;
      // (Beyond 127 by the rounding of s, far beyond where s is subnormal.)
      const int byte = (int)fmaxf(fminf(lower ? __builtin_floorf(y) : __builtin_ceilf(y), 127.f), -127.f);
      out |= (uint32_t)(byte & 255) << (8 * i);
    }
    if (!(s > 0.f) || odd) out = 0;
    int8_t* dst = p.bounds + (2 * at + (lower ? 0 : 1)) * D + col * E + (row & (RPI / 2 - 1)) * V;
    if constexpr (V == 4)
      *(uint32_t*)dst = out;
    else
      *(uint16_t*)dst = (uint16_t)out;
    if (lane == 0) p.bound_scale[at] = s;
  }
}

// ---------------------------------------------------------------- the rows of a call

struct RowAt {
  int seq;      // -1: a row of no sequence
  int tokens;   // that it sees
};

// The sequence and the visible tokens of query row r (the same for all lanes of a wave).
// `len`: seq_lens[r], where there is no q_start.
__device__ __forceinline__ RowAt row_at(const SelectParams& p, int r, int len) {
  const int lane = threadIdx.x & 63, cap = p.max_pages * kPage;
  if (!p.q_start) {
    const int L = uni(len);
    if ((L < 0 || L > cap) && lane == 0) atomicOr(p.flags, kFlagBadLen);
    return {r, min(max(L, 0), cap)};
  }
  const RowsOf at = rows_of(p.q_start, p.seq_lens, p.batch, p.total_q, r);
  if ((at.bad || (at.seq >= 0 && (at.len < 0 || at.len > cap || at.q1 - at.q0 > at.len))) && lane == 0) atomicOr(p.flags, kFlagBadLen);
  return {at.seq, max(min(max(at.len, 0), cap) - (at.q1 - 1 - r), 0)};
}

// Offsets that run backwards need not meet a row's search: the grid looks at all of them once, a
// wave of the first workgroups at 64 each.
__device__ __forceinline__ void check_offsets(const SelectParams& p) {
  for (int b0 = (int)blockIdx.x * 64; b0 < p.batch; b0 += gridDim.x * 64) {
    const int b = min(b0 + (int)(threadIdx.x & 63), p.batch - 1), q0 = p.q_start[b], q1 = p.q_start[b + 1];
    if (q0 < 0 || q0 > q1 || q1 > p.total_q) atomicOr(p.flags, kFlagBadLen);
  }
}

// ---------------------------------------------------------------- the best of many

// What a workgroup of T threads shares while it looks for the K largest keys.
template <int T>
struct Search {
  static constexpr int kWavesOf = T / 64;
  int hist[kDigits];                 // zero when a search begins
  uint32_t low[kWavesOf], high[kWavesOf];
  int sum[kWavesOf], ties[kWavesOf];
  int digit, above, in, members;
  uint32_t list[64];
};

// Sum over the waves before this one of s[wave] (all lanes; `all`: over all of them).
template <int T>
__device__ __forceinline__ int waves_before(const int* s, int* all) {
  const int lane = threadIdx.x & 63, wave = uni((int)(threadIdx.x >> 6));
  constexpr int N = T / 64;
  const int x = wave_scan(lane < N ? s[lane] : 0);
  *all = __builtin_amdgcn_readlane(x, N - 1);
  return wave == 0 ? 0 : __builtin_amdgcn_readlane(x, max(wave - 1, 0));
}

// The K-th largest of keys[lo .. hi) (0 < K < hi - lo), of which a thread has seen kmin to kmax: those
// above *at are taken, and the first *ties of those equal to it.  Digits of 11 bits from the
// highest bit in which keys differ; the first one leaves a few keys as a rule, which every
// wave then compares with each other.  Ends with s.hist in use.
template <int T>
__device__ __forceinline__ void kth_largest(const uint32_t* keys, int lo, int hi, int K, uint32_t kmin, uint32_t kmax,
                                            Search<T>& s, uint32_t* at, int* ties) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  constexpr int N = T / 64, P = kDigits / T;   // digits of a thread
  kmin = ~wave_max(~kmin);
  kmax = wave_max(kmax);
  if (lane == 0) {
    s.low[wave] = kmin;
    s.high[wave] = kmax;
  }
  if (tid == 0) s.members = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < N; ++w) {
    kmin = min(kmin, s.low[w]);
    kmax = max(kmax, s.high[w]);
  }
  int bits = kmin == kmax ? 0 : 32 - __builtin_clz(kmin ^ kmax);   // still undecided
  uint32_t prefix = bits == 32 ? 0u : kmin >> bits << bits;
  *ties = K;
  for (bool again = false; bits > 0; again = true) {
    const int shift = max(bits - kDigitBits, 0);
    if (again) {
      for (int i = tid; i < kDigits; i += T) s.hist[i] = 0;
      __syncthreads();
    }
    for (int j = lo + tid; j < hi; j += T) {
      const uint32_t k = keys[j];
      if (bits == 32 || ((k ^ prefix) >> bits) == 0) atomicAdd(&s.hist[(k >> shift) & ((1u << (bits - shift)) - 1u)], 1);
    }
    __syncthreads();
    // Counts from the largest digit down, P a thread.
    int n[P], sum = 0, all;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      n[i] = s.hist[kDigits - 1 - (tid * P + i)];
      sum += n[i];
    }
    const int incl = wave_scan(sum);
    if (lane == 63) s.sum[wave] = incl;
    __syncthreads();
    int before = waves_before<T>(s.sum, &all) + incl - sum;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (before < K && K <= before + n[i]) {
        s.digit = kDigits - 1 - (tid * P + i);
        s.above = before;
        s.in = n[i];
      }
      before += n[i];
    }
    __syncthreads();
    prefix |= (uint32_t)s.digit << shift;
    K -= s.above;
    bits = shift;
    *ties = K;
    const int in = s.in;
    if (in == K) {   // all of them: whatever their lower bits are
      *ties = 0x7FFFFFFF;
      break;
    }
    if (bits > 0 && in <= 64) {
      for (int j = lo + tid; j < hi; j += T) {
        const uint32_t k = keys[j];
        if (((k ^ prefix) >> bits) == 0) s.list[atomicAdd(&s.members, 1)] = k;
      }
      __syncthreads();
      const uint32_t mine = lane < in ? s.list[lane] : 0u;
      int above = 0, equal = 0;
      for (int i = 0; i < in; ++i) {
        const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)mine, i);
        above += k > mine;
        equal += k == mine;
      }
      const uint64_t it = __builtin_amdgcn_ballot_w64(lane < in && above < K && K <= above + equal);
      const int l = __builtin_ctzll(it);
      prefix = (uint32_t)__builtin_amdgcn_readlane((int)mine, l);
      *ties = K - __builtin_amdgcn_readlane(above, l);
      break;
    }
  }
  *at = prefix;
}

// The same by one wave alone, with 256 counters in `hist`: digits of 8 bits.
__device__ __forceinline__ void kth_largest_wave(const uint32_t* keys, int lo, int hi, int K, int* hist, uint32_t* at, int* ties) {
  const int lane = threadIdx.x & 63;
  const auto wait = [] {   // LDS operations of a wave are done in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  // Four times 64 keys at a time: f(key, whether there is one).
  const auto each = [&](auto f) {
    for (int j = lo + lane; j - lane < hi; j += 256) {
      uint32_t k[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) k[i] = keys[min(j + 64 * i, hi - 1)];
#pragma unroll
      for (int i = 0; i < 4; ++i) f(k[i], j + 64 * i < hi);
    }
  };
  uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
  each([&](uint32_t k, bool) {   // (past the end: the last one again)
    kmin = min(kmin, k);
    kmax = max(kmax, k);
  });
  kmin = ~wave_max(~kmin);
  kmax = wave_max(kmax);
  int bits = kmin == kmax ? 0 : 32 - __builtin_clz(kmin ^ kmax);
  uint32_t prefix = bits == 32 ? 0u : kmin >> bits << bits;
  *ties = K;
  while (bits > 0) {
    const int shift = max(bits - 8, 0);
    const auto inside = [&](uint32_t k) { return bits == 32 || ((k ^ prefix) >> bits) == 0; };
    *(i32x4*)&hist[4 * lane] = i32x4{0, 0, 0, 0};
    wait();
    each([&](uint32_t k, bool is) {
      if (is && inside(k)) atomicAdd(&hist[255 - ((k >> shift) & ((1u << (bits - shift)) - 1u))], 1);
    });
    wait();
    const i32x4 n = *(const i32x4*)&hist[4 * lane];   // from the largest digit down
    wait();
    const int incl = wave_scan(n[0] + n[1] + n[2] + n[3]);
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(incl >= K));   // the first lane that reaches K
    int above = __builtin_amdgcn_readlane(incl - (n[0] + n[1] + n[2] + n[3]), l), d = 4 * l, in = __builtin_amdgcn_readlane(n[0], l);
#pragma unroll
    for (int i = 1; i < 4; ++i)
      if (above + in < K) {
        above += in;
        in = __builtin_amdgcn_readlane(n[i], l);
        d = 4 * l + i;
      }
    prefix |= (uint32_t)(255 - d) << shift;
    K -= above;
    bits = shift;
    *ties = K;
    if (in == K) {   // all of them: whatever their lower bits are
      *ties = 0x7FFFFFFF;
      break;
    }
    if (bits > 0 && in <= 64) {
      int got = 0;
      each([&](uint32_t k, bool is) {
        const bool member = is && ((k ^ prefix) >> bits) == 0;
        const uint64_t m = __builtin_amdgcn_ballot_w64(member);
        if (member) hist[got + __builtin_popcountll(m & ((1ull << lane) - 1))] = (int)k;
        got += __builtin_popcountll(m);
      });
      wait();
      const uint32_t mine = lane < in ? (uint32_t)hist[lane] : 0u;
      wait();
      int greater = 0, equal = 0;
      for (int i = 0; i < in; ++i) {
        const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)mine, i);
        greater += k > mine;
        equal += k == mine;
      }
      const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < in && greater < K && K <= greater + equal));
      prefix = (uint32_t)__builtin_amdgcn_readlane((int)mine, who);
      *ties = K - __builtin_amdgcn_readlane(greater, who);
      break;
    }
  }
  *at = prefix;
}

// Which pages of [0, n) are chosen: the first `sink`, the last `recent`, and of the others the
// largest keys.
struct Chosen {
  uint32_t at;
  int ties, sink, end;   // end: of the pages with a choice
  bool any;
  // Whether page j < n is chosen whatever its ties, and whether it is one of the ties.
  __device__ __forceinline__ bool sure(int j, uint32_t k) const { return j < sink || j >= end || (any && k > at); }
  __device__ __forceinline__ bool tie(int j, uint32_t k) const { return j >= sink && j < end && any && k == at; }
};

// ... found by one wave, or by the whole workgroup from keys in LDS, of which a thread has seen kmin to kmax.
__device__ __forceinline__ Chosen choose_wave(const uint32_t* keys, int n, int budget, int sink, int recent, int* hist) {
  Chosen c = {0xFFFFFFFFu, 0, sink, n - recent, budget > sink + recent};
  if (c.any) kth_largest_wave(keys, sink, n - recent, budget - sink - recent, hist, &c.at, &c.ties);
  return c;
}
template <int T>
__device__ __forceinline__ Chosen choose(const uint32_t* keys, int n, int budget, int sink, int recent, uint32_t kmin,
                                         uint32_t kmax, Search<T>& s) {
  Chosen c = {0xFFFFFFFFu, 0, sink, n - recent, budget > sink + recent};
  if (c.any) kth_largest<T>(keys, sink, n - recent, budget - sink - recent, kmin, kmax, s, &c.at, &c.ties);
  return c;
}

// ---------------------------------------------------------------- choice

template <int CTRL>
__device__ __forceinline__ float row_move(float x) {
  const int v = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, true));
}
// Maxima of four values over the 16 lanes of a row: lane i gets that of value i / 4.  Each
// lane hands the values on that are not its own, so there are fewer of them every step.
__device__ __forceinline__ float row_max4(const float* m) {
  const int lane = threadIdx.x & 63;
  const bool b3 = lane & 8, b2 = lane & 4;
  const float x0 = fmaxf(b3 ? m[2] : m[0], row_move<0x128>(b3 ? m[0] : m[2]));   // row_ror:8
  const float x1 = fmaxf(b3 ? m[3] : m[1], row_move<0x128>(b3 ? m[1] : m[3]));
  // The lanes of the other value are 4 before or after within the eight (row_half_mirror).
  float y = fmaxf(b2 ? x1 : x0, row_move<0x141>(b2 ? x0 : x1));
  y = fmaxf(y, row_move<0xB1>(y));          // lane ^ 1, ^ 2
  return fmaxf(y, row_move<0x4E>(y));
}

// The query heads of a KV head in 8 bits: min(q8, 0) for the lower bounds, then max(q8, 0) for
// the upper ones, and their scales.  A wave a head (every wave rounding all of them for
// itself was a third of a small call's time), rows of 16 bytes more than they hold so that
// the reads below spread over the banks.
template <int D>
struct QShared {
  int8_t bytes[kMaxGroup][2 * D + 16];
  float scale[kMaxGroup];
};
template <int D, bool QF32>
__device__ __forceinline__ void round_q(const SelectParams& p, int row, int g, QShared<D>& s) {
  constexpr int E = D / 64, N = kSel / 64, H = (kMaxGroup + N - 1) / N;   // heads of a wave: their loads in flight together
  const int lane = threadIdx.x & 63, wave = uni((int)(threadIdx.x >> 6));
  float x[H][E];
#pragma unroll
  for (int i = 0; i < H; ++i) {
    // The head map by a scalar load: the arguments lie in host memory.
    const int m = g * p.group + min(wave + i * N, p.group - 1);
    const int qh = (int)(((const uint32_t*)p.q_head)[m >> 1] >> (16 * (m & 1)) & 0xFFFFu);
    const int64_t at = ((int64_t)row * p.num_q_heads + qh) * D + lane;
#pragma unroll
    for (int e = 0; e < E; ++e)
      x[i][e] = QF32 ? ((const float*)p.q)[at + 64 * e] : __uint_as_float((uint32_t)((const uint16_t*)p.q)[at + 64 * e] << 16);
  }
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int k = wave + i * N;
    if (k >= p.group) break;
    float amax = 0.f;
    bool odd = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      odd |= !finite(x[i][e]);
      amax = fmaxf(amax, __builtin_fabsf(x[i][e]));
    }
    amax = __uint_as_float(wave_max(__float_as_uint(amax)));   // (magnitudes order as integers)
    // (A query of infinities or NaN says nothing about pages.)
    const float sq = __builtin_amdgcn_ballot_w64(odd) != 0 ? 0.f : amax / 127.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int q = sq > 0.f ? (int)fmaxf(fminf(__builtin_rintf(x[i][e] / sq), 127.f), -127.f) : 0;
      s.bytes[k][64 * e + lane] = (int8_t)min(q, 0);
      s.bytes[k][D + 64 * e + lane] = (int8_t)max(q, 0);
    }
    if (lane == 0) s.scale[k] = sq;
  }
}

// ... as the second operand of 16x16x64 products: lane 16 qg + i holds head i's elements
// 64 c + 16 qg .. + 15 (past the heads, the first one's again: the maximum is the same).
template <int D>
struct QBytes {
  static constexpr int NC = 2 * D / 64;
  i32x4 v[NC];
  float scale;
  __device__ __forceinline__ void load(const QShared<D>& s, int group) {
    const int lane = threadIdx.x & 63, i = (lane & 15) < group ? lane & 15 : 0, qg = lane >> 4;
#pragma unroll
    for (int c = 0; c < NC; ++c) v[c] = *(const i32x4*)&s.bytes[i][64 * c + 16 * qg];
    scale = s.scale[i];
  }
};

// Tiles of 16 pages go round the waves, kTiles of a wave's at a time (a step), whose loads are in
// flight together: the page whose id and key a lane holds.
constexpr int kSelWaves = kSel / 64, kTiles = 2;
__device__ __forceinline__ int page_of(int j0, int step) {
  const int lane = threadIdx.x & 63, wave = uni((int)(threadIdx.x >> 6));
  if (lane >= 16 * kTiles) return 0x7fffffff;
  return j0 + 16 * ((kTiles * step + (lane >> 4)) * kSelWaves + wave) + (lane & 15);
}

// A step's bounds.
template <int D>
struct Tiles {
  static constexpr int NC = 2 * D / 64;
  i32x4 a[kTiles][NC];
  float scale;
  bool there;

  // `id`: of the lane's page, one of the row's where `in` (lanes past the tiles: none).
  __device__ __forceinline__ void load(const SelectParams& p, int g, int id, bool in) {
    const int lane = threadIdx.x & 63, i = lane & 15, qg = lane >> 4;
    there = in && (unsigned)id < (unsigned)p.num_pages;
    if (in && !there) atomicOr(p.flags, kFlagBadPage);
    if (p.num_pages == 0) return;      // (no page is there, and none is looked at)
    const int pid = there ? id : 0;   // (page 0 for those that are not: its keys are not used)
    scale = p.bound_scale[(int64_t)pid * p.num_kv_heads + g];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int64_t page = __shfl(pid, 16 * t + i);
      const int8_t* src = p.bounds + (page * p.num_kv_heads + g) * (2 * D) + 16 * qg;
#pragma unroll
      for (int c = 0; c < NC; ++c) a[t][c] = *(const i32x4*)(src + 64 * c);
    }
  }

  // The order key of the lane's page.  Bounds that are not finite: their page is looked at first.
  // A page that is not there: last.
  __device__ __forceinline__ uint32_t key(const QBytes<D>& q, float* s_val) const {
    const int lane = threadIdx.x & 63, i = lane & 15, qg = lane >> 4;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      i32x4 u = {0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < NC; ++c) u = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[t][c], q.v[c], u, 0, 0, 0);
      // Lane 16 qg + i: page 4 qg + r with head i.
      float m[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) m[r] = (float)u[r] * q.scale;
      const float most = row_max4(m);
      if ((i & 3) == 0) s_val[16 * t + 4 * qg + (i >> 2)] = most;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const float x = s_val[lane & (16 * kTiles - 1)] * scale;
    __builtin_amdgcn_wave_barrier();
    return !there ? 0u : finite(scale) ? order_key(x) : 0xFFFFFFFFu;
  }
};

// The chosen pages of [r0, r1) in order, by one wave: `rank` chosen ones and `tied` ties lie before.
// Four times 64 pages at a time; classes(): which of them are chosen, and which are ties.
struct Classes {
  uint64_t sure[4], tie[4];
  __device__ __forceinline__ Classes(const uint32_t* keys, const Chosen& c, int at, int r1) {
    const int lane = threadIdx.x & 63;
    uint32_t k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k[i] = at + 64 * i + lane < r1 ? keys[at + 64 * i + lane] : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = at + 64 * i + lane;
      sure[i] = __builtin_amdgcn_ballot_w64(j < r1 && c.sure(j, k[i]));
      tie[i] = __builtin_amdgcn_ballot_w64(j < r1 && c.tie(j, k[i]));
    }
  }
};
__device__ __forceinline__ void write_chosen(const uint32_t* keys, const Chosen& c, int r0, int r1, int rank, int tied, int32_t* out) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = (1ull << lane) - 1;
  for (int j = r0; j < r1; j += 256) {
    const Classes k(keys, c, j, r1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool chosen = (k.sure[i] >> lane & 1) || ((k.tie[i] >> lane & 1) && tied + __builtin_popcountll(k.tie[i] & below) < c.ties);
      const uint64_t m = __builtin_amdgcn_ballot_w64(chosen);
      if (chosen) out[rank + __builtin_popcountll(m & below)] = j + 64 * i + lane;
      rank += __builtin_popcountll(m);
      tied += __builtin_popcountll(k.tie[i]);
    }
  }
}

// One workgroup, or p.pieces of them, a (row, KV head).  With several, the one that finishes last
// gathers the others' keys.
//   What a small call takes is its chain of dependent reads (the length, page ids, bounds) and
// the search, so the ids and the queries are asked for before the length is known, and up to
// kWavePages pages are searched by one wave, without barriers: 7.2 us for 8 responses of up to
// 256 pages (2 KV heads), 9.9 before.  A long one is bound by the bounds it reads: two buffers of
// tiles, one computed while the other's loads are in flight.  64 sequences of 512 to 2048
// pages, 4 KV heads (92 MB): 28.7 us, of them 3.4 until the first bounds are there, 11 (mean) to
// 17 (the longest) for the products, 4 for the search and the list.  Rows of one sequence read
// its bounds through their XCD's L2: 4 rows each of 16 sequences (8 KV heads, 82 MB in 64 rows, 21
// MB of them from memory) 21 us.  Tried: several rows of a sequence to a workgroup (the same to
// 31 us: fewer, longer chains), pieces of 512 pages for all rows (43 us: their starts under load),
// 256 and 1024 threads (32 and 29.5 against 29.9 then).
constexpr int kWavePages = 256;

template <int D, bool QF32, int CAP>
__global__ __launch_bounds__(kSel) void select_pages_kernel(const SelectParams p) {
  __shared__ uint32_t s_key[CAP];
  __shared__ float s_val[kSelWaves][16 * kTiles];
  __shared__ __align__(16) QShared<D> s_q;
  __shared__ __align__(16) Search<kSel> s;
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  // A run of rows with all their KV heads to each XCD: a page's heads lie beside each other, and
  // one head alone would use few of its L2's channels.
  const int at_block = share_of_block(blockIdx.x, gridDim.x);
  const int seg = p.pieces == 1 ? at_block : at_block / (uint32_t)p.pieces, piece = at_block - seg * p.pieces;
  const int row = seg / (uint32_t)p.num_kv_heads, g = seg - row * p.num_kv_heads;
  const bool early = !p.q_start && p.pieces == 1;   // the sequence and the first page are known
  const int len = p.q_start ? 0 : p.seq_lens[row];
  int ids[2] = {0, 0};
  if (early) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = page_of(0, k);
      ids[k] = j < p.max_pages ? p.block_table[(int64_t)row * p.max_pages + j] : 0;
    }
  }
  round_q<D, QF32>(p, row, g, s_q);
  const RowAt at = row_at(p, row, len);
  // (One wave, its arguments there by now: by all of them, before the queries, 448 us of 434 for 8000
  // rows of 4000 sequences, 441 so; 200 sequences and fewer within 0.5%.)
  if (p.q_start && wave == kSelWaves - 1) check_offsets(p);
  if (at.seq < 0) return;
  const int n = (at.tokens + kPage - 1) / kPage;
  int32_t* out = p.pages + (int64_t)seg * p.budget;
  if (n <= p.budget) {   // all of them
    if (piece != 0) return;
    for (int j = tid; j < p.budget; j += kSel) out[j] = j < n ? j : -1;
    if (tid == 0) p.counts[seg] = n;
    return;
  }
  if (tid == 0) p.counts[seg] = p.budget;
  for (int i = tid; i < kDigits; i += kSel) s.hist[i] = 0;
  const int per = ((n + p.pieces - 1) / p.pieces + 15) / 16 * 16, j0 = min(piece * per, n), j1 = min(j0 + per, n);
  const int32_t* bt = p.block_table + (int64_t)at.seq * p.max_pages;
  const auto id_of = [&](int step) {
    const int j = page_of(j0, step);
    return j < j1 ? bt[j] : 0;
  };
  if (!early) {
    ids[0] = id_of(0);
    ids[1] = id_of(1);
  }
  Tiles<D> t[2];
  t[0].load(p, g, ids[0], page_of(j0, 0) < j1);
  ids[0] = id_of(2);
  __syncthreads();
  QBytes<D> q;
  q.load(s_q, p.group);
  uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
  const auto keep = [&](int j, uint32_t k) {
    s_key[j] = k;
    if (j >= p.sink && j < n - p.recent) {
      kmin = min(kmin, k);
      kmax = max(kmax, k);
    }
  };
  uint32_t* keys = p.keys + (int64_t)seg * p.max_pages;
  // Step by step, a wave's own first page telling whether it has another.
  const auto more = [&](int step) { return j0 + 16 * (kTiles * step * kSelWaves + wave) < j1; };
  for (int step = 0; more(step); step += 2) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (!more(step + k)) break;
      if (more(step + k + 1)) {
        t[1 - k].load(p, g, ids[1 - k], page_of(j0, step + k + 1) < j1);
        ids[1 - k] = id_of(step + k + 3);
      }
      const int j = page_of(j0, step + k);
      const uint32_t key = t[k].key(q, s_val[wave]);
      if (lane < 16 * kTiles && j < j1) {
        if (p.pieces == 1)
          keep(j, key);
        else
          __hip_atomic_store(keys + j, key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
  }
  if (p.pieces > 1) {
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
    for (int j = tid; j < n; j += kSel) keep(j, __hip_atomic_load(keys + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  }
  __syncthreads();
  if (n <= kWavePages) {
    if (wave != 0) return;
    const Chosen c = choose_wave(s_key, n, p.budget, p.sink, p.recent, s.hist);
    write_chosen(s_key, c, 0, n, 0, 0, out);
    return;
  }
  const Chosen c = choose<kSel>(s_key, n, p.budget, p.sink, p.recent, kmin, kmax, s);
  // Every wave writes the chosen ones of a run of pages, behind those of the waves before.
  const int run = ((n + kSelWaves - 1) / kSelWaves + 63) / 64 * 64, r0 = min(wave * run, n), r1 = min(r0 + run, n);
  int sures = 0, ties = 0;
  for (int j = r0; j < r1; j += 256) {
    const Classes k(s_key, c, j, r1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sures += __builtin_popcountll(k.sure[i]);
      ties += __builtin_popcountll(k.tie[i]);
    }
  }
  if (lane == 0) {
    s.sum[wave] = sures;
    s.ties[wave] = ties;
  }
  __syncthreads();
  int all;
  const int rank = waves_before<kSel>(s.sum, &all), tied = waves_before<kSel>(s.ties, &all);
  write_chosen(s_key, c, r0, r1, rank + min(tied, c.ties), tied, out);
}

// ---------------------------------------------------------------- eviction

// A dropped page loses a reference.
__device__ __forceinline__ void drop_page(const SelectParams& p, int page) {
  if ((uint32_t)page >= (uint32_t)p.num_pages) {
    atomicOr(p.flags, kFlagBadPage);
  } else if (atomicSub(p.refs + page, 1) <= 0) {   // nobody held it
    atomicAdd(p.refs + page, 1);
    atomicOr(p.flags, kFlagBadPage);
  }
}

// One workgroup a row.  Up to kWavePages pages, one wave of it: the entries and weights are asked
// for with the length, stay in registers, and no barrier is met (8 rows of 65 pages, 5.3 us by
// the whole workgroup and 4.5 so; what is left is the chain of reads).  More: entries move
// towards the front, kEvict at a time: what a step writes lies at or before what it has read.
template <int CAP>
__global__ __launch_bounds__(kEvict) void page_evict_kernel(const SelectParams p) {
  __shared__ uint32_t s_key[CAP];
  __shared__ __align__(16) Search<kEvict> s;
  constexpr int R = kWavePages / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), b = blockIdx.x;
  int32_t* table = p.block_table + (int64_t)b * p.max_pages;
  float* w = p.weights + (int64_t)b * p.max_pages;
  int pages[R];
  float weights[R];
  if (wave == 0) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int j = min(64 * i + lane, p.max_pages - 1);
      pages[i] = table[j];
      weights[i] = w[j];
    }
  }
  const int L = p.seq_lens[b];
  const int n = (L + kPage - 1) / kPage;
  const bool bad = L < 0 || L > p.max_pages * kPage;
  if (bad && tid == 0) atomicOr(p.flags, kFlagBadLen);
  if (bad || n <= p.budget) {
    if (tid == 0) p.dropped[b] = 0;
    return;
  }
  if (n <= kWavePages) {
    if (wave != 0) return;
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (64 * i + lane < n) s_key[64 * i + lane] = order_key(weights[i]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const Chosen c = choose_wave(s_key, n, p.budget, p.sink, p.recent, s.hist);
    const Classes k(s_key, c, 0, n);
    const uint64_t below = (1ull << lane) - 1;
    int rank = 0, tied = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const bool chosen = (k.sure[i] >> lane & 1) || ((k.tie[i] >> lane & 1) && tied + __builtin_popcountll(k.tie[i] & below) < c.ties);
      const uint64_t m = __builtin_amdgcn_ballot_w64(chosen);
      if (chosen) {
        const int to = rank + __builtin_popcountll(m & below);
        table[to] = pages[i];
        w[to] = weights[i];
      } else if (64 * i + lane < n) {
        drop_page(p, pages[i]);
      }
      rank += __builtin_popcountll(m);
      tied += __builtin_popcountll(k.tie[i]);
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (64 * i + lane >= p.budget && 64 * i + lane < n) w[64 * i + lane] = 0.f;   // (ranks end before)
    if (lane == 0) {
      p.dropped[b] = n - p.budget;
      p.seq_lens[b] = L - kPage * (n - p.budget);
    }
    return;
  }
  for (int i = tid; i < kDigits; i += kEvict) s.hist[i] = 0;
  uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
  for (int j = tid; j < n; j += kEvict) {
    const uint32_t k = order_key(w[j]);
    s_key[j] = k;
    if (j >= p.sink && j < n - p.recent) {
      kmin = min(kmin, k);
      kmax = max(kmax, k);
    }
  }
  __syncthreads();
  const Chosen c = choose<kEvict>(s_key, n, p.budget, p.sink, p.recent, kmin, kmax, s);
  int taken = 0, tied = 0;   // in the pages before
  const uint64_t below = (1ull << lane) - 1;
  for (int j0 = 0; j0 < n; j0 += kEvict) {
    const int j = j0 + tid;
    const uint32_t k = j < n ? s_key[j] : 0u;
    const bool sure = j < n && c.sure(j, k), tie = j < n && c.tie(j, k);
    const int page = j < n ? table[j] : 0;
    const float weight = j < n ? w[j] : 0.f;
    const uint64_t ms = __builtin_amdgcn_ballot_w64(sure), mt = __builtin_amdgcn_ballot_w64(tie);
    __syncthreads();   // the counts have been read
    if (lane == 0) {
      s.sum[wave] = __builtin_popcountll(ms);
      s.ties[wave] = __builtin_popcountll(mt);
    }
    __syncthreads();   // ... and the step's entries, before any of them is written
    int alls, allt;
    const int sures = waves_before<kEvict>(s.sum, &alls) + __builtin_popcountll(ms & below);
    const int ties = tied + waves_before<kEvict>(s.ties, &allt) + __builtin_popcountll(mt & below);
    const int rank = taken + sures + min(ties, c.ties) - min(tied, c.ties);
    if (sure || (tie && ties < c.ties)) {
      table[rank] = page;
      w[rank] = weight;
    } else if (j < n) {
      drop_page(p, page);
    }
    taken += alls + min(tied + allt, c.ties) - min(tied, c.ties);
    tied += allt;
  }
  __syncthreads();
  for (int j = p.budget + tid; j < n; j += kEvict) w[j] = 0.f;
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

// Workgroups of a call with first tokens: 31.5, 29.8, 28.4 and 28.5 us for 64 prompts with 4096,
// 8192, 16384 and 32768 (the lengths differ, and a sequence's share is cut from the longest).
constexpr int kBoundsGrid = 16384;
int launch_page_bounds(KvKind kind, int head_dim, const SelectParams& p, void* stream) {
  // A wave a (page, KV head): enough of them for the last pages, or, the lengths not being known,
  // a sequence's share of what the GPU holds.
  const int64_t most = p.first ? (int64_t)p.max_pages * p.num_kv_heads : p.num_kv_heads;
  const int64_t share = kBoundsGrid / p.batch > 1 ? kBoundsGrid / p.batch : 1;
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
    hipLaunchKernelGGL(page_evict_kernel<kSelSmall>, dim3(p.batch), dim3(kEvict), 0, (hipStream_t)stream, p);
  else
    hipLaunchKernelGGL(page_evict_kernel<kSelectMaxPages>, dim3(p.batch), dim3(kEvict), 0, (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

}  // namespace rlda
