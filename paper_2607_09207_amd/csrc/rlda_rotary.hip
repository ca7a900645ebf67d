// Rotary positions for gfx950: rows turned by their positions, alone or on their way into
// the paged KV cache.
//
// A head's elements form pairs; pair j of a row at position n is turned by the angle
// t = n f_j (f_j radians a position, given in 64 bits) and scaled by the amplitude A:
//     a' = A (a cos t - b sin t),   b' = A (b cos t + a sin t),
// the inverse turning by -t, which is the transpose: a gradient's way back.  Pairs are
// (j, j + rot/2) ("half") or (2j, 2j + 1) ("interleaved") of the first `rot` elements; the
// others pass.  Arithmetic is fp32; the angle is not: n f_j of a far position has lost its
// fraction of a turn in 32 bits (2^20 positions: 0.06 radians), so it is reduced to a
// fraction of a turn, and its sine and cosine taken, in 64.
//
// Work.  A workgroup takes a window of up to 16 rows (tokens): it finds their sequences,
// positions and cache slots, and takes one sine and cosine a (row, pair) into LDS, shared
// by every head of the row (one a lane in registers would be repeated by each head).  Then
// its threads walk the window's 16-byte chunks, a pair of chunks at a time where their
// elements are turned into each other, four such units in flight, the first of them asked
// for before anything else.  Few rows take small windows, and several workgroups to a
// window with a share of the units each.
// Rows are read and written once: what bounds it is bandwidth, and latency on few rows.
// us a call: 32768 x 32 heads of 128 in bf16 89 (537 MB, 6.0 TB/s; a copy of one large
// buffer to another reaches 4.9); 26,237 rows of 40/8 heads into fp8 pages 140 (700 MB, 5.0
// TB/s), into bf16 ones 155 (752 MB, 4.8 TB/s); one token of 512 sequences, 64/8 heads, 7.5 (21 MB),
// of 8 sequences 5.2 (the launch takes 3.8).  Few rows wait: for their length, then the page
// id, then the angles, which could run beside that; bf16 and f32 caches then ask for K once
// q is stored, and for V once K is.
//
// fp8 caches hold one scale per (page, KV head) that covers every row written so far, so
// their K and V rows are written a page at a time, by workgroups of their own: one wave per
// (page, KV head, K or V) turns the page's new rows in registers, finds their largest
// magnitude, sets or raises the scale (re-encoding the rows before them) and encodes them.
// A page belongs to the window that holds its first new row; its rows reach at most 15
// past the window.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rlda_device.h"
#include "rlda_params.h"

namespace rlda {
namespace {

constexpr int kWin = kRotaryWindow;      // rows of a window at most
constexpr int kWinRows = 2 * kWin;       // ... and the rows its pages may reach to
constexpr int kUnroll = 4;               // units in flight a thread

// Eight consecutive elements.
template <bool F32>
struct Chunk;
template <>
struct Chunk<false> {
  u32x4 r;
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const void* base, int64_t e) {
    const u32x4* at = (const u32x4*)((const uint16_t*)base + e);
    r = STREAM ? __builtin_nontemporal_load(at) : *at;
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(r[i] << 16);
      x[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
    }
  }
  // fp32 results rounded once to the rows' type.
  __device__ __forceinline__ void set(const float* x) {
    r = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void store(void* p) const {
    if (STREAM) __builtin_nontemporal_store(r, (u32x4*)p);
    else *(u32x4*)p = r;
  }
};
template <>
struct Chunk<true> {
  f32x4 r[2];
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const void* base, int64_t e) {
    const f32x4* at = (const f32x4*)((const float*)base + e);
    r[0] = STREAM ? __builtin_nontemporal_load(at) : at[0];
    r[1] = STREAM ? __builtin_nontemporal_load(at + 1) : at[1];
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = r[i >> 2][i & 3];
  }
  __device__ __forceinline__ void set(const float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i >> 2][i & 3] = x[i];
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void store(void* p) const {
    f32x4* at = (f32x4*)p;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (STREAM) __builtin_nontemporal_store(r[i], at + i);
      else at[i] = r[i];
  }
};

// The cosines and sines of a row: unit u turns pairs K u .. K u + K - 1 (half pairs K = 8,
// interleaved K = 4), and neighbouring lanes turn neighbouring units, so every two pairs
// of a unit stand beside the same ones of its neighbours: pair K u + r at place
// (r / 2) 2 (half / K) + 2 u + r % 2.  (In order, eight lanes met in the same banks.)
template <bool IL>
__device__ __forceinline__ int place_of(const RotaryParams& p, int pair) {
  constexpr int K = IL ? 4 : 8;
  const int u = pair / K, r = pair % K;
  return (r >> 1) * 2 * (p.half / K) + 2 * u + (r & 1);
}

// Turn unit u of a row: chunks a and b into each other (half pairs), or chunk a in itself
// (interleaved).  cs: the row's cosines and sines.
template <bool IL>
__device__ __forceinline__ void turn(const RotaryParams& p, float* a, float* b, const float2* cs, int u) {
  constexpr int K = IL ? 4 : 8;
  const f32x4* at = (const f32x4*)cs + u;   // two pairs: (cos, sin, cos, sin)
  const int step = p.half / K;
  f32x4 f[K / 2];
#pragma unroll
  for (int j = 0; j < K / 2; ++j) f[j] = at[j * step];
  if constexpr (IL) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float c = f[j >> 1][2 * (j & 1)], s = f[j >> 1][2 * (j & 1) + 1], x = a[2 * j], y = a[2 * j + 1];
      a[2 * j] = __builtin_fmaf(x, c, -(y * s));
      a[2 * j + 1] = __builtin_fmaf(y, c, x * s);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float c = f[j >> 1][2 * (j & 1)], s = f[j >> 1][2 * (j & 1) + 1], x = a[j], y = b[j];
      a[j] = __builtin_fmaf(x, c, -(y * s));
      b[j] = __builtin_fmaf(y, c, x * s);
    }
  }
}

// Units of a head: half pairs h = rot / 16 pairs of chunks, then the chunks that pass;
// interleaved: its chunks.  Unit u's first chunk is u (half: past the pairs u + h).
template <bool IL>
__device__ __forceinline__ bool unit_turns(const RotaryParams& p, int u) {
  return u < (IL ? p.half >> 2 : p.half >> 3);
}
template <bool IL>
__device__ __forceinline__ int unit_chunk(const RotaryParams& p, int u) {
  return IL || unit_turns<IL>(p, u) ? u : u + (p.half >> 3);
}

__device__ __forceinline__ uint32_t div_by(uint32_t x, uint32_t magic) { return __umulhi(x, magic); }

// Units i, i + step, .. of `nrows` rows of `heads` heads (rows first + r, r < nrows): asked
// for, and then turned and handed to put(row, head, chunk, values) where ok[row].
// STREAM: rows too many for the caches to hold are read and written past them (set_windows).
template <bool F32, bool IL, bool STREAM>
struct Units {
  Chunk<F32> a[kUnroll], b[kUnroll];
  int row[kUnroll], head[kUnroll], unit[kUnroll];

  __device__ __forceinline__ void fetch(const RotaryParams& p, const void* x, int64_t rs, int64_t hs, int first, int total,
                                        int heads, uint32_t magic_hu, int i0, int step) {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int i = i0 + k * step;
      row[k] = -1;
      if (i >= total) continue;
      const int r = (int)div_by(i, magic_hu), rem = i - r * heads * p.units, hd = (int)div_by(rem, p.magic_u);
      row[k] = r;
      head[k] = hd;
      unit[k] = rem - hd * p.units;
      const int64_t e = (int64_t)(first + r) * rs + (int64_t)hd * hs + 8 * unit_chunk<IL>(p, unit[k]);
      a[k].template load<STREAM>(x, e);
      if (!IL && unit_turns<IL>(p, unit[k])) b[k].template load<STREAM>(x, e + p.half);
    }
  }
  template <class Put>
  __device__ __forceinline__ void finish(const RotaryParams& p, const uint8_t* ok, const float2* cs, Put put) {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      if (row[k] < 0 || !ok[row[k]]) continue;
      const int u = unit[k], c = unit_chunk<IL>(p, u);
      if (unit_turns<IL>(p, u)) {
        float xa[8], xb[8];
        a[k].get(xa);
        if (!IL) b[k].get(xb);
        turn<IL>(p, xa, xb, cs + row[k] * p.half, u);
        a[k].set(xa);
        if (!IL) {
          b[k].set(xb);
          put(row[k], head[k], c + (p.half >> 3), b[k]);
        }
      }
      put(row[k], head[k], c, a[k]);
    }
  }
};

// Cosine and sine (times the amplitude) of rows [0, n) of the window, by all threads.
template <bool IL>
__device__ __forceinline__ void angles(const RotaryParams& p, const int32_t* pos, int n, float2* cs) {
  const double turns = 0.15915494309189535;   // 1 / (2 pi)
  for (int i = threadIdx.x; i < n * p.half; i += kThreads) {
    const int r = (int)div_by(i, p.magic_half), j = i - r * p.half;
    double t = (double)pos[r] * p.freqs[j] * turns;
    t -= rint(t);
    double s, c;
    sincospi(2.0 * t, &s, &c);
    const float sn = (float)(s * (double)p.amplitude);
    cs[r * p.half + place_of<IL>(p, j)] = make_float2((float)(c * (double)p.amplitude), p.inverse ? -sn : sn);
  }
}

// ---------------------------------------------------------------- rows alone
template <bool F32, bool IL, bool STREAM>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotaryParams p) {
  extern __shared__ __align__(16) float2 s_cs[];   // [win][half]
  __shared__ int32_t s_pos[kWin];
  __shared__ uint8_t s_ok[kWin];
  const int win = blockIdx.x / p.parts, part = blockIdx.x - win * p.parts;
  const int first = win * p.win, n = min(p.win, p.rows - first);
  const int total = n * p.hq * p.units, step = p.parts * kThreads;
  int i = part * kThreads + threadIdx.x;
  Units<F32, IL, STREAM> x;
  x.fetch(p, p.q, p.q_rs, p.q_hs, first, total, p.hq, p.magic_qu, i, step);
  if (threadIdx.x < (uint32_t)n) {
    s_pos[threadIdx.x] = p.positions[first + threadIdx.x];
    s_ok[threadIdx.x] = 1;
  }
  __syncthreads();
  angles<IL>(p, s_pos, n, s_cs);
  __syncthreads();
  constexpr int E = F32 ? 4 : 2;
  for (;;) {
    x.finish(p, s_ok, s_cs, [&](int r, int hd, int c, const Chunk<F32>& v) {
      v.template store<STREAM>((char*)p.q_out + ((int64_t)(first + r) * p.o_rs + (int64_t)hd * p.o_hs + 8 * c) * E);
    });
    i += kUnroll * step;
    if (i >= total) break;
    x.fetch(p, p.q, p.q_rs, p.q_hs, first, total, p.hq, p.magic_qu, i, step);
  }
}

// ---------------------------------------------------------------- rows into the cache

// The sequence that holds row r >= 0: the last b with q_start[b] <= r (a wave-wide search,
// 64 points a step; r uniform).  q_start may hold anything: the caller checks the answer.
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int batch, int r, int lane) {
  int lo = 0, n = batch;   // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int at = lo + lane * step;
    const bool below = lane * step < n && q_start[at] <= r;
    const uint64_t m = __builtin_amdgcn_ballot_w64(below);
    // The leading run of points at or below r.
    const int k = m == ~0ull ? 64 : __builtin_ctzll(~m);
    const int j = max(k - 1, 0);
    n = min(step, n - j * step);
    lo += j * step;
  }
  return lo;
}

// E4M3 (OCP FN) encoding of two fp32 values, round to nearest even.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}

// One page of an fp8 cache, KV head and K or V, by a wave: rows r0 .. r0 + m - 1 of the
// window into slots s0 .. of the page.  Lane l: chunk l % NC of the slots l / NC, + 64 / NC, ..
// (a load or store of the wave covers whole rows); its pairs' other halves come from the
// lanes that hold them.
//   A row that sets the scale, amax / 448, is encoded from 448 x / amax, one rounding from the
// value where x / scale has two: ties of bf16 rows stay ties.
template <int D, bool IL, bool TURN>
__device__ __forceinline__ void write_page(const RotaryParams& p, const void* x, int64_t rs, int64_t hs, int first, int r0,
                                           int m, int s0, int g, char* page, float* scale, const float2* cs, int lane) {
  constexpr int NC = D / 8, kStep = 64 / NC, kN = kPage / kStep;   // chunks of a row, rows of an access, accesses
  const int c = lane % NC, t0 = lane / NC, h8 = p.half >> 3;
  Chunk<false> raw[kN];
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    const int t = t0 + kStep * j;
    raw[j].r = u32x4{0u, 0u, 0u, 0u};
    if (t >= s0 && t < s0 + m) raw[j].load(x, (int64_t)(first + r0 + t - s0) * rs + (int64_t)g * hs + 8 * c);
  }
  float s = s0 > 0 ? *scale : 0.f;
  if (!(s > 0.f) || __builtin_isinf(s)) s = 0.f;
  // Half pairs: this chunk is the first (side 0) or second half of unit u, the other half in
  // the lane `other`.
  const bool turns = TURN && c < (IL ? p.half >> 2 : 2 * h8);
  const int side = !IL && c >= h8, u = side ? c - h8 : c;
  const int other = lane + (turns && !IL ? (side ? -h8 : h8) : 0);
  float v[kN][8];
  float amax = 0.f;
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    const int t = t0 + kStep * j, r = r0 + t - s0;
    raw[j].get(v[j]);
    if constexpr (TURN) {
      Chunk<false> ob;
      if constexpr (!IL) {
#pragma unroll
        for (int i = 0; i < 4; ++i) ob.r[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * other, (int)raw[j].r[i]);
      }
      if (turns && t >= s0 && t < s0 + m) {
        const float2* f = cs + r * p.half;
        if constexpr (IL) {
          float none[8];
          turn<true>(p, v[j], none, f, u);
        } else {
          float o[8];
          ob.get(o);
          if (side)
            turn<false>(p, o, v[j], f, u);
          else
            turn<false>(p, v[j], o, f, u);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[j][e]));
  }
  // Never NaN, and not negative: as an integer in the order of its value.
  amax = __builtin_bit_cast(float, __builtin_amdgcn_readlane(wave_scan_max(__builtin_bit_cast(int, amax)), 63));
  const bool grows = s0 == 0 || amax > 448.f * s;
  const float s_new = grows ? amax / 448.f : s;
  if (grows && s0 > 0) {
    // The page's earlier rows, at the new scale: four lanes a row.
    const float ratio = s > 0.f ? s / s_new : 0.f;
    const int t = lane >> 2;
    if (t < s0) {
      constexpr int N = D / 64;   // 16-byte loads of a quarter row
      u32x4* rp = (u32x4*)(page + (int64_t)t * p.stride_slot + (lane & 3) * (D / 4));
      u32x4 w[N];
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = rp[i];
#pragma unroll
      for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x2 lo = fp8x2_to_f32(w[i][j], false), hi = fp8x2_to_f32(w[i][j], true);
          w[i][j] = s > 0.f ? e4m3x2(lo[0] * ratio, lo[1] * ratio) | e4m3x2(hi[0] * ratio, hi[1] * ratio) << 16 : 0u;
        }
        rp[i] = w[i];
      }
    }
  }
  // x num / den, correctly rounded: a quotient by the rounded reciprocal, corrected by its
  // remainder (exact with a correctly rounded reciprocal); by division where the reciprocal
  // or the remainder would leave the range, both sides of it 2^16 smaller where 448 x would
  // overflow (a magnitude beside which 2^-110 is a zero byte), and where den is infinite.
  const float den_of = grows ? amax : s;
  const bool wide = den_of > 0x1p100f, divide = den_of < 0x1p-100f || wide;
  const float num = (grows ? 448.f : 1.f) * (wide ? 0x1p-16f : 1.f), den = wide ? den_of * 0x1p-16f : den_of;
  const float inv = 1.f / den;
  auto quotient = [&](float f) {
    const float n = f * num;
    if (divide) return n / den;
    const float q = n * inv;
    return __builtin_fmaf(__builtin_fmaf(-den, q, n), inv, q);
  };
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    const int t = t0 + kStep * j;
    if (t < s0 || t >= s0 + m) continue;
    u32x2 w = {0u, 0u};
    if (s_new > 0.f) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        w[i] = e4m3x2(quotient(v[j][4 * i]), quotient(v[j][4 * i + 1])) |
               e4m3x2(quotient(v[j][4 * i + 2]), quotient(v[j][4 * i + 3])) << 16;
    }
    *(u32x2*)(page + (int64_t)t * p.stride_slot + 8 * c) = w;
  }
  if (lane == 0) *scale = s_new;
}

template <int D, KvKind KIND, bool IL, bool STREAM>
__global__ __launch_bounds__(kThreads) void append_rotary_kernel(const RotaryParams p) {
  constexpr bool F32 = KIND == KvKind::F32, FP8 = KIND == KvKind::FP8;
  constexpr int E = F32 ? 4 : 2;
  extern __shared__ __align__(16) float2 s_cs[];   // [win, fp8 caches and several rows a sequence: win + 15][half]
  __shared__ int32_t s_pos[kWinRows];   // position of the row (its angle)
  __shared__ int32_t s_tok[kWinRows];   // token of its sequence
  __shared__ int32_t s_seq[kWinRows];
  __shared__ int64_t s_off[kWinRows];   // byte offset of its slot in the pool (KV head 0), -1: not written
  __shared__ int32_t s_pid[kWinRows];
  __shared__ uint8_t s_ok[kWinRows];    // the row belongs to a sequence and has a position
  __shared__ int32_t s_n;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  // fp8 caches: a window's workgroups from p.parts on write pages, the others turn q.  They
  // run together: a token's q, k and v lie behind one another, and read far apart in time
  // they cost 10 to 20 us of 150 (26,237 rows of 40/8 heads).
  //   Blocks go round the 8 XCDs, so a window's roles move on by one from window to window:
  // fixed, they would all be on some of them where their number and 8 share a factor
  // (3 and 1 of them 174 us, 3 and 2 143).
  const int all_parts = p.parts + p.page_parts;
  const int win = blockIdx.x / all_parts, turn_part = (int)((blockIdx.x + (uint32_t)win) % (uint32_t)all_parts);
  const bool pages = FP8 && turn_part >= p.parts;
  const int part = turn_part - (pages ? p.parts : 0), parts = pages ? p.page_parts : p.parts;
  const int first = win * p.win, n = min(p.win, p.rows - first);
  const int cap = p.max_pages * kPage;
  const int span = pages && p.q_start ? min(p.win + kPage - 1, p.rows - first) : n;   // rows described here
  const int total = n * p.hq * p.units, step = parts * kThreads;
  int i = part * kThreads + tid;
  Units<F32, IL, STREAM> x;
  if (!pages) x.fetch(p, p.q, p.q_rs, p.q_hs, first, total, p.hq, p.magic_qu, i, step);

  // 1. Every row's sequence, token, position and slot.
  if (wave == 0) {
    const int r = first + lane;
    int b = r, q0 = r, q1 = r + 1;
    bool ok = lane < span;
    uint32_t bad = 0;
    if (p.q_start) {
      // The last sequence that begins at or before the row: of the next 64 (asked for together)
      // as many as begin there, and behind 64 empty ones a search of its own.
      b = sequence_of(p.q_start, p.batch, first, lane);
      const int next = b + 1 + lane < p.batch ? p.q_start[b + 1 + lane] : 0x7fffffff;
      if (uni(next) < first + span) {   // (else every row is in that one)
        int k = 0;
#pragma unroll
        for (int w = 32; w >= 1; w >>= 1) k += __shfl(next, k + w - 1) <= r ? w : 0;
        k += __shfl(next, k) <= r;
        b += k;
        if (ok && k == 64) {
          int hi = b + 1;
          for (int w = 2; hi < p.batch && p.q_start[hi] <= r; w <<= 1) {
            b = hi;
            hi = min(hi + w, p.batch);
          }
          while (hi - b > 1) {   // q_start[b] <= r < q_start[hi]
            const int mid = (b + hi) >> 1;
            if (p.q_start[mid] <= r) b = mid; else hi = mid;
          }
        }
      }
      if (ok) {
        q0 = p.q_start[b];
        q1 = p.q_start[b + 1];
        // Rows before the first sequence and behind the last are nobody's.
        if (r >= q1 && b == p.batch - 1) ok = false;
        else if (r < q0 && b == 0) ok = false;
        else if (q0 < 0 || r < q0 || r >= q1 || q1 > p.rows) {
          ok = false;
          bad = kFlagBadLen;
        }
      }
    }
    int tok = -1;
    if (ok) {
      const int L = p.seq_lens[b];
      tok = L - (q1 - q0) + (r - q0);
      if (L < 0 || L > cap || (p.q_start && tok < 0)) {
        ok = false;
        bad |= kFlagBadLen;
      } else if (tok < 0) {
        ok = false;   // an empty sequence of a one-token call
      }
    }
    int64_t off = -1;
    int pid = -1;
    if (ok) {
      pid = p.block_table[(int64_t)b * p.max_pages + tok / kPage];
      if ((uint32_t)pid < (uint32_t)p.num_pages)
        off = (int64_t)pid * p.stride_page + (int64_t)(tok % kPage) * p.stride_slot;
      else
        bad |= kFlagBadPage;
    }
    if (lane < kWinRows) {
      s_ok[lane] = ok;
      s_tok[lane] = tok;
      s_seq[lane] = b;
      s_off[lane] = off;
      s_pid[lane] = pid;
      s_pos[lane] = ok ? (p.positions ? p.positions[r] : tok) : 0;
    }
    // The rows that this window's pages reach to: a row behind the window continues a page
    // when it is in the sequence and the page of the window's last row.
    if (lane == 0) s_n = n;
    if (FP8 && span > n) {
      const int bl = __builtin_amdgcn_readlane(b, n - 1), tl = __builtin_amdgcn_readlane(tok, n - 1);
      const bool on = ok && b == bl && tl >= 0 && lane >= n && tok / kPage == tl / kPage;
      const uint64_t m = __builtin_amdgcn_ballot_w64(on);
      if (lane == 0) s_n = n + __builtin_popcountll(m);
    }
    if (lane >= n) bad = 0;   // reported by the row's own window
    if (__builtin_amdgcn_ballot_w64((bad & kFlagBadLen) != 0) && part == 0 && lane == 0) atomicOr(p.flags, kFlagBadLen);
    if (__builtin_amdgcn_ballot_w64((bad & kFlagBadPage) != 0) && part == 0 && lane == 0) atomicOr(p.flags, kFlagBadPage);
  }
  __syncthreads();
  if constexpr (FP8) {
    if (pages) {
      // 2. The pages whose first new row is in the window.  A row starts a page when its
      //    token is the page's first, or its sequence's first new one.
      const int r = lane;
      const bool here = r < n && s_ok[r];
      const bool start = here && (s_tok[r] % kPage == 0 || !p.q_start || first + r == p.q_start[s_seq[r]]);
      const uint64_t starts = __builtin_amdgcn_ballot_w64(start);
      if (starts == 0) return;
      const int jobs = __builtin_popcountll(starts) * 2 * p.hkv;
      const int all = uni(s_n);
      angles<IL>(p, s_pos, all, s_cs);
      __syncthreads();
      for (int j = part * kWaves + wave; j < jobs; j += parts * kWaves) {
        int k = j / (2 * p.hkv);
        const int gw = j - k * 2 * p.hkv, g = gw >> 1;
        uint64_t m = starts;
        for (; k > 0; --k) m &= m - 1;
        const int r0 = __builtin_ctzll(m), s0 = uni(s_tok[r0]) % kPage;
        int rows = 1;   // rows of the page: as many as follow in it
        while (r0 + rows < all && s0 + rows < kPage && s_ok[r0 + rows] && s_seq[r0 + rows] == s_seq[r0]) ++rows;
        rows = uni(rows);
        const int pid = uni(s_pid[r0]);
        if ((uint32_t)pid >= (uint32_t)p.num_pages) continue;
        const int64_t at = (int64_t)pid * p.stride_page + (int64_t)g * p.stride_head;
        const int64_t si = (int64_t)pid * p.hkv + g;
        if (gw & 1)
          write_page<D, IL, false>(p, p.v_in, p.v_rs, p.v_hs, first, r0, rows, s0, g, (char*)p.v + at, p.v_scale + si, s_cs, lane);
        else
          write_page<D, IL, true>(p, p.k_in, p.k_rs, p.k_hs, first, r0, rows, s0, g, (char*)p.k + at, p.k_scale + si, s_cs, lane);
      }
      return;
    }
  }
  angles<IL>(p, s_pos, n, s_cs);
  __syncthreads();

  // 3. q, and K and V rows of caches that hold them as they are.
  for (;;) {
    x.finish(p, s_ok, s_cs, [&](int r, int hd, int c, const Chunk<F32>& v) {
      v.template store<STREAM>((char*)p.q_out + ((int64_t)(first + r) * p.o_rs + (int64_t)hd * p.o_hs + 8 * c) * E);
    });
    i += kUnroll * step;
    if (i >= total) break;
    x.fetch(p, p.q, p.q_rs, p.q_hs, first, total, p.hq, p.magic_qu, i, step);
  }
  if constexpr (!FP8) {
    const int ktotal = n * p.hkv * p.units;
    for (i = part * kThreads + tid; i < ktotal; i += kUnroll * step) {
      x.fetch(p, p.k_in, p.k_rs, p.k_hs, first, ktotal, p.hkv, p.magic_ku, i, step);
      x.finish(p, s_ok, s_cs, [&](int r, int g, int c, const Chunk<F32>& v) {
        if (s_off[r] >= 0) v.store((char*)p.k + s_off[r] + (int64_t)g * p.stride_head + 8 * c * E);
      });
    }
    constexpr int NC = D / 8;
    const int vtotal = n * p.hkv * NC;
    for (i = part * kThreads + tid; i < vtotal; i += step) {
      const int c = i % NC, rg = i / NC, r = rg / p.hkv, g = rg - r * p.hkv;
      if (!s_ok[r] || s_off[r] < 0) continue;
      Chunk<F32> v;
      v.load(p.v_in, (int64_t)(first + r) * p.v_rs + (int64_t)g * p.v_hs + 8 * c);
      v.store((char*)p.v + s_off[r] + (int64_t)g * p.stride_head + 8 * c * E);
    }
  }
}

template <int D, KvKind KIND>
int launch_append_rotary_t(const RotaryParams& p, hipStream_t st) {
  constexpr bool FP8 = KIND == KvKind::FP8;
  const int grid = (p.rows + p.win - 1) / p.win * (p.parts + p.page_parts);
  const int rows = FP8 && p.q_start ? p.win + kPage - 1 : p.win;
  auto* const kernel = p.interleaved ? (p.stream ? append_rotary_kernel<D, KIND, true, true> : append_rotary_kernel<D, KIND, true, false>)
                                     : (p.stream ? append_rotary_kernel<D, KIND, false, true> : append_rotary_kernel<D, KIND, false, false>);
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), sizeof(float2) * p.half * rows, st, p);
  return (int)hipGetLastError();
}

template <bool F32>
int launch_rotate_t(const RotaryParams& p, hipStream_t st) {
  auto* const kernel = p.interleaved ? (p.stream ? rotate_kernel<F32, true, true> : rotate_kernel<F32, true, false>)
                                     : (p.stream ? rotate_kernel<F32, false, true> : rotate_kernel<F32, false, false>);
  hipLaunchKernelGGL(kernel, dim3((p.rows + p.win - 1) / p.win * p.parts), dim3(kThreads), sizeof(float2) * p.half * p.win, st, p);
  return (int)hipGetLastError();
}

}  // namespace

int launch_rotate(bool f32, const RotaryParams& p, void* stream) {
  return f32 ? launch_rotate_t<true>(p, (hipStream_t)stream) : launch_rotate_t<false>(p, (hipStream_t)stream);
}

int launch_append_rotary(KvKind kind, int head_dim, const RotaryParams& p, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  switch (kind) {
    case KvKind::BF16:
      return head_dim == 128 ? launch_append_rotary_t<128, KvKind::BF16>(p, st) : launch_append_rotary_t<64, KvKind::BF16>(p, st);
    case KvKind::FP8:
      return head_dim == 128 ? launch_append_rotary_t<128, KvKind::FP8>(p, st) : launch_append_rotary_t<64, KvKind::FP8>(p, st);
    case KvKind::F32:
      return head_dim == 128 ? launch_append_rotary_t<128, KvKind::F32>(p, st) : launch_append_rotary_t<64, KvKind::F32>(p, st);
  }
  return -1;
}

}  // namespace rlda
