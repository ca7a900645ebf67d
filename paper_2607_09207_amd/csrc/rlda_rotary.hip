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
// Work.  A workgroup takes a window of 16 rows (tokens): it finds their sequences,
// positions and cache slots, and takes one sine and cosine a (row, pair) into LDS, shared
// by every head of the row (one a lane in registers would be repeated by each head).  Then
// its threads walk the window's 16-byte chunks, a pair of chunks at a time where their
// elements are turned into each other, four such units in flight.  Few rows take several
// workgroups to a window (`parts`), each with a share of the units.
// Rows are read and written once: what bounds it is bandwidth, and latency on few rows.
//
// fp8 caches hold one scale per (page, KV head) that covers every row written so far, so
// their K and V rows are written a page at a time: one wave per (page, KV head, K or V)
// turns the page's new rows in registers, finds their largest magnitude, sets or raises
// the scale (re-encoding the rows before them) and encodes them.  A page belongs to the
// window that holds its first new row; its rows reach at most 15 past the window.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rlda_device.h"
#include "rlda_params.h"

namespace rlda {
namespace {

constexpr int kWin = kRotaryWindow;   // rows of a window
constexpr int kWinRows = 2 * kWin;    // ... and the rows its pages may reach to
constexpr int kUnroll = 4;            // units in flight a thread

// Eight consecutive elements.
template <bool F32>
struct Chunk;
template <>
struct Chunk<false> {
  u32x4 r;
  __device__ __forceinline__ void load(const void* base, int64_t e) { r = *(const u32x4*)((const uint16_t*)base + e); }
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
  __device__ __forceinline__ void store(void* p) const { *(u32x4*)p = r; }
};
template <>
struct Chunk<true> {
  f32x4 r[2];
  __device__ __forceinline__ void load(const void* base, int64_t e) {
    r[0] = *(const f32x4*)((const float*)base + e);
    r[1] = *(const f32x4*)((const float*)base + e + 4);
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = r[i >> 2][i & 3];
  }
  __device__ __forceinline__ void set(const float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i >> 2][i & 3] = x[i];
  }
  __device__ __forceinline__ void store(void* p) const {
    *(f32x4*)p = r[0];
    *((f32x4*)p + 1) = r[1];
  }
};

// Turn a unit: chunks a and b into each other (half pairs, cs of their eight pairs), or
// chunk a in itself (interleaved, cs of its four pairs).
template <bool IL>
__device__ __forceinline__ void turn(float* a, float* b, const float2* cs) {
  if constexpr (IL) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float c = cs[j].x, s = cs[j].y, x = a[2 * j], y = a[2 * j + 1];
      a[2 * j] = __builtin_fmaf(x, c, -(y * s));
      a[2 * j + 1] = __builtin_fmaf(y, c, x * s);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float c = cs[j].x, s = cs[j].y, x = a[j], y = b[j];
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

// Turn `nrows` rows of `heads` heads (rows[first + r], r < nrows, where ok[r]) and hand
// every chunk's result to put(row, head, chunk, values).  `part` of `parts` workgroups.
template <bool F32, bool IL, class Put>
__device__ __forceinline__ void turn_rows(const RotaryParams& p, const void* x, int64_t rs, int64_t hs, int first,
                                          int nrows, int heads, uint32_t magic_hu, int part, const uint8_t* ok,
                                          const float2* cs, Put put) {
  const int U = p.units, total = nrows * heads * U, step = p.parts * kThreads, h8 = p.half >> 3;
  for (int i0 = part * kThreads + (int)threadIdx.x; i0 < total; i0 += kUnroll * step) {
    Chunk<F32> a[kUnroll], b[kUnroll];
    int row[kUnroll], head[kUnroll], unit[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int i = i0 + k * step;
      row[k] = -1;
      if (i >= total) continue;
      const int r = (int)div_by(i, magic_hu), rem = i - r * heads * U, hd = (int)div_by(rem, p.magic_u);
      unit[k] = rem - hd * U;
      head[k] = hd;
      if (!ok[r]) continue;
      row[k] = r;
      const int64_t e = (int64_t)(first + r) * rs + (int64_t)hd * hs + 8 * unit_chunk<IL>(p, unit[k]);
      a[k].load(x, e);
      if (!IL && unit_turns<IL>(p, unit[k])) b[k].load(x, e + 8 * h8);
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      if (row[k] < 0) continue;
      const int u = unit[k], c = unit_chunk<IL>(p, u);
      if (unit_turns<IL>(p, u)) {
        float xa[8], xb[8];
        a[k].get(xa);
        if (!IL) b[k].get(xb);
        turn<IL>(xa, xb, cs + row[k] * p.half + (IL ? 4 : 8) * u);
        a[k].set(xa);
        if (!IL) {
          b[k].set(xb);
          put(row[k], head[k], c + h8, b[k]);
        }
      }
      put(row[k], head[k], c, a[k]);
    }
  }
}

// Cosine and sine (times the amplitude) of rows [0, n) of the window, by all threads.
__device__ __forceinline__ void angles(const RotaryParams& p, const int32_t* pos, int n, float2* cs) {
  const double turns = 0.15915494309189535;   // 1 / (2 pi)
  for (int i = threadIdx.x; i < n * p.half; i += kThreads) {
    const int r = (int)div_by(i, p.magic_half), j = i - r * p.half;
    double t = (double)pos[r] * p.freqs[j] * turns;
    t -= rint(t);
    double s, c;
    sincospi(2.0 * t, &s, &c);
    const float sn = (float)(s * (double)p.amplitude);
    cs[i] = make_float2((float)(c * (double)p.amplitude), p.inverse ? -sn : sn);
  }
}

// ---------------------------------------------------------------- rows alone
template <bool F32, bool IL>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotaryParams p) {
  extern __shared__ float2 s_cs[];   // [kWin][half]
  __shared__ int32_t s_pos[kWin];
  __shared__ uint8_t s_ok[kWin];
  const int win = blockIdx.x / p.parts, part = blockIdx.x - win * p.parts;
  const int first = win * kWin, n = min(kWin, p.rows - first);
  if (threadIdx.x < (uint32_t)n) {
    s_pos[threadIdx.x] = p.positions[first + threadIdx.x];
    s_ok[threadIdx.x] = 1;
  }
  __syncthreads();
  angles(p, s_pos, n, s_cs);
  __syncthreads();
  constexpr int E = F32 ? 4 : 2;
  turn_rows<F32, IL>(p, p.q, p.q_rs, p.q_hs, first, n, p.hq, p.magic_qu, part, s_ok, s_cs,
                     [&](int r, int hd, int c, const Chunk<F32>& v) {
                       v.store((char*)p.q_out + ((int64_t)(first + r) * p.o_rs + (int64_t)hd * p.o_hs + 8 * c) * E);
                     });
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
// window into slots s0 .. of the page.  Lane 4 t + c: slot t, units c, c + 4, .. of its row.
template <int D, bool IL, bool TURN>
__device__ __forceinline__ void write_page(const RotaryParams& p, const void* x, int64_t rs, int64_t hs, int first, int r0,
                                           int m, int s0, int g, char* page, float* scale, const float2* cs, int lane) {
  constexpr int NC = D / 8, MU = (NC + 3) / 4;   // chunks of a row, units of a lane at most
  const int t = lane >> 2, c = lane & 3, r = r0 + t - s0, h8 = p.half >> 3;
  const bool mine = t >= s0 && t < s0 + m;
  const int U = TURN ? p.units : NC;
  float v[MU][2][8];
  float amax = 0.f;
#pragma unroll
  for (int j = 0; j < MU; ++j) {
    const int u = c + 4 * j;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[j][0][e] = v[j][1][e] = 0.f;
    if (!mine || u >= U) continue;
    const bool turns = TURN && unit_turns<IL>(p, u);
    const int64_t at = (int64_t)(first + r) * rs + (int64_t)g * hs + 8 * (TURN ? unit_chunk<IL>(p, u) : u);
    Chunk<false> a, b;
    a.load(x, at);
    a.get(v[j][0]);
    if (turns) {
      if (!IL) {
        b.load(x, at + 8 * h8);
        b.get(v[j][1]);
      }
      turn<IL>(v[j][0], v[j][1], cs + r * p.half + (IL ? 4 : 8) * u);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fmaxf(fabsf(v[j][0][e]), fabsf(v[j][1][e])));
  }
  // Never NaN, and not negative: as an integer in the order of its value.
  amax = __builtin_bit_cast(float, __builtin_amdgcn_readlane(wave_scan_max(__builtin_bit_cast(int, amax)), 63));
  float s = s0 > 0 ? *scale : 0.f;
  if (!(s > 0.f) || __builtin_isinf(s)) s = 0.f;
  float s_new = s;
  if (s0 == 0 || amax > 448.f * s) {
    s_new = amax / 448.f;
    // The page's earlier rows, at the new scale.
    const float ratio = s > 0.f ? s / s_new : 0.f;
    if (t < s0) {
      constexpr int N = D / 64;   // 16-byte loads of a quarter row
      u32x4* rp = (u32x4*)(page + (int64_t)t * p.stride_slot + c * (D / 4));
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
  char* row = page + (int64_t)t * p.stride_slot;
  auto put = [&](int ch, const float* f) {
    u32x2 w = {0u, 0u};
    if (s_new > 0.f) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        w[i] = e4m3x2(f[4 * i] / s_new, f[4 * i + 1] / s_new) | e4m3x2(f[4 * i + 2] / s_new, f[4 * i + 3] / s_new) << 16;
    }
    *(u32x2*)(row + 8 * ch) = w;
  };
#pragma unroll
  for (int j = 0; j < MU; ++j) {
    const int u = c + 4 * j;
    if (!mine || u >= U) continue;
    const int ch = TURN ? unit_chunk<IL>(p, u) : u;
    put(ch, v[j][0]);
    if (TURN && !IL && unit_turns<IL>(p, u)) put(ch + h8, v[j][1]);
  }
  if (lane == 0) *scale = s_new;
}

template <int D, KvKind KIND, bool IL>
__global__ __launch_bounds__(kThreads) void append_rotary_kernel(const RotaryParams p) {
  constexpr bool F32 = KIND == KvKind::F32, FP8 = KIND == KvKind::FP8;
  constexpr int E = F32 ? 4 : 2;
  extern __shared__ float2 s_cs[];   // [kWin, fp8 caches and several rows a sequence: kWinRows][half]
  __shared__ int32_t s_pos[kWinRows];   // position of the row (its angle)
  __shared__ int32_t s_tok[kWinRows];   // token of its sequence
  __shared__ int32_t s_seq[kWinRows];
  __shared__ int64_t s_off[kWinRows];   // byte offset of its slot in the pool (KV head 0), -1: not written
  __shared__ int32_t s_pid[kWinRows];
  __shared__ uint8_t s_ok[kWinRows];    // the row belongs to a sequence and has a position
  __shared__ int32_t s_n;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int win = blockIdx.x / p.parts, part = blockIdx.x - win * p.parts;
  const int first = win * kWin, n = min(kWin, p.rows - first);
  const int cap = p.max_pages * kPage;
  const int span = FP8 && p.q_start ? min(kWinRows, p.rows - first) : n;   // rows described here

  // 1. Every row's sequence, token, position and slot.
  if (wave == 0) {
    const int r = first + lane;
    int b = r, q0 = r, q1 = r + 1;
    bool ok = lane < span;
    uint32_t bad = 0;
    if (p.q_start) {
      b = sequence_of(p.q_start, p.batch, first, lane);
      while (ok && b < p.batch - 1 && p.q_start[b + 1] <= r) ++b;
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
    // The rows that this window's pages reach to: row i >= 16 continues a page when it is
    // in the sequence and the page of row 15 (and so on from there).
    if (lane == 0) s_n = n;
    if (FP8 && span > kWin) {
      const int b15 = __builtin_amdgcn_readlane(b, kWin - 1), t15 = __builtin_amdgcn_readlane(tok, kWin - 1);
      const bool on = ok && b == b15 && t15 >= 0 && lane >= kWin && tok / kPage == t15 / kPage;
      const uint64_t m = __builtin_amdgcn_ballot_w64(on);
      if (lane == 0) s_n = n + __builtin_popcountll(m);
    }
    if (lane >= n) bad = 0;   // reported by the row's own window
    if (__builtin_amdgcn_ballot_w64((bad & kFlagBadLen) != 0) && part == 0 && lane == 0) atomicOr(p.flags, kFlagBadLen);
    if (__builtin_amdgcn_ballot_w64((bad & kFlagBadPage) != 0) && part == 0 && lane == 0) atomicOr(p.flags, kFlagBadPage);
  }
  __syncthreads();
  angles(p, s_pos, uni(s_n), s_cs);
  __syncthreads();

  // 2. q, and K and V rows of caches that hold them as they are.
  turn_rows<F32, IL>(p, p.q, p.q_rs, p.q_hs, first, n, p.hq, p.magic_qu, part, s_ok, s_cs,
                     [&](int r, int hd, int c, const Chunk<F32>& v) {
                       v.store((char*)p.q_out + ((int64_t)(first + r) * p.o_rs + (int64_t)hd * p.o_hs + 8 * c) * E);
                     });
  if constexpr (!FP8) {
    turn_rows<F32, IL>(p, p.k_in, p.k_rs, p.k_hs, first, n, p.hkv, p.magic_ku, part, s_ok, s_cs,
                       [&](int r, int g, int c, const Chunk<F32>& v) {
                         if (s_off[r] >= 0) v.store((char*)p.k + s_off[r] + (int64_t)g * p.stride_head + 8 * c * E);
                       });
    constexpr int NC = D / 8;
    const int total = n * p.hkv * NC;
    for (int i = part * kThreads + tid; i < total; i += p.parts * kThreads) {
      const int c = i % NC, rg = i / NC, r = rg / p.hkv, g = rg - r * p.hkv;
      if (!s_ok[r] || s_off[r] < 0) continue;
      Chunk<F32> v;
      v.load(p.v_in, (int64_t)(first + r) * p.v_rs + (int64_t)g * p.v_hs + 8 * c);
      v.store((char*)p.v + s_off[r] + (int64_t)g * p.stride_head + 8 * c * E);
    }
  } else {
    // 3. fp8: the pages whose first new row is in the window.  A row starts a page when its
    //    token is the page's first, or its sequence's first new one.
    const int r = lane;
    const bool here = r < n && s_ok[r];
    const bool start = here && (s_tok[r] % kPage == 0 || !p.q_start || first + r == p.q_start[s_seq[r]]);
    const uint64_t starts = __builtin_amdgcn_ballot_w64(start);
    const int jobs = __builtin_popcountll(starts) * 2 * p.hkv;
    const int all = uni(s_n);
    for (int j = part * kWaves + wave; j < jobs; j += p.parts * kWaves) {
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
  }
}

template <int D, KvKind KIND>
int launch_append_rotary_t(const RotaryParams& p, hipStream_t st) {
  const int grid = (p.rows + kWin - 1) / kWin * p.parts;
  const size_t lds = sizeof(float2) * p.half * (KIND == KvKind::FP8 && p.q_start ? kWinRows : kWin);
  if (p.interleaved)
    hipLaunchKernelGGL((append_rotary_kernel<D, KIND, true>), dim3(grid), dim3(kThreads), lds, st, p);
  else
    hipLaunchKernelGGL((append_rotary_kernel<D, KIND, false>), dim3(grid), dim3(kThreads), lds, st, p);
  return (int)hipGetLastError();
}

}  // namespace

int launch_rotate(bool f32, const RotaryParams& p, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  const int grid = (p.rows + kWin - 1) / kWin * p.parts;
  const size_t lds = sizeof(float2) * p.half * kWin;
  if (f32 && p.interleaved)
    hipLaunchKernelGGL((rotate_kernel<true, true>), dim3(grid), dim3(kThreads), lds, st, p);
  else if (f32)
    hipLaunchKernelGGL((rotate_kernel<true, false>), dim3(grid), dim3(kThreads), lds, st, p);
  else if (p.interleaved)
    hipLaunchKernelGGL((rotate_kernel<false, true>), dim3(grid), dim3(kThreads), lds, st, p);
  else
    hipLaunchKernelGGL((rotate_kernel<false, false>), dim3(grid), dim3(kThreads), lds, st, p);
  return (int)hipGetLastError();
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
