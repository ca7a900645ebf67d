// Decode attention over a paged KV cache for gfx950 (MI355X).
//
// One launch does the whole operation (the attention step the paper's rollout
// model charges through the history term H_dec and the per-token footprint b_kv,
// App. A.1.2):
//
//   1. Work plan.  Every workgroup scans seq_lens into page-count prefix sums in
//      LDS.  The work is the flattened list of (sequence, KV head, page) units,
//      priced one per page plus a fixed start cost per (sequence, KV head);
//      workgroup u owns the u-th of nranges equal-cost shares of it.  Long
//      sequences are therefore cut across many workgroups and short ones packed
//      together: every workgroup streams the same work however long the tail of
//      the length distribution is (Sec. 2.3 on long-tail decode).  Small calls take
//      whole segments instead, one per workgroup (see rlda_split.h).
//   2. Page gather.  Each of the 4 waves of a workgroup takes a quarter of the
//      share and walks it as one continuous stream of pages: its lanes decode 64
//      positions at a time (sequence, KV head, page id, valid tokens, segment
//      start/end flags) one chunk ahead of use, and the wave computes one page
//      while the two after it are in flight to registers, by buffer loads whose
//      range check returns zero past a page's last valid token, so masked slots
//      cost no memory traffic and never yield NaN.  A segment's Q operand is loaded with its first page.
//      Segment boundaries inside the stream cost no pipeline restart.
//   3. Scores and softmax.  All G query heads that share the KV head are packed
//      into one 16-row MFMA tile: S^T = K Q^T with v_mfma_f32_16x16x32_bf16; the
//      online softmax keeps a running reference max and sum per head in log2
//      units, and moves the reference (rescaling the accumulator) only when a
//      score exceeds it by more than 8, i.e. a probability above 2^8.
//   4. PV.  O^T += V^T P^T with v_mfma_f32_16x16x16_bf16: the score tile's output
//      registers are already the P^T operand, and V's operand is assembled from
//      4 row loads per lane, so neither operand goes through LDS.  Streams that
//      are longer than equal shares for every workgroup would make them add the
//      probabilities' bf16 remainders.
//   5. Merge.  A segment a wave covered whole is normalised and written by that
//      wave.  The cut pieces (at most 2 per wave) are merged through LDS.  A piece
//      of a segment that is split across workgroups stores its unnormalised
//      partial with device-scope (sc1) stores, which write through the XCD's L2;
//      after they complete, the workgroup bumps the segment's counter.  The
//      workgroup that completes the count reads every piece of the segment with
//      device-scope loads, merges them in piece order with log-sum-exp weights,
//      writes the output and resets the counter.  Each partial carries the
//      call's tag, so a merge that meets a piece this call did not publish (a
//      counter left non-zero in the workspace) raises a flag.  No workgroup waits
//      for another, and no device-scope fence (a whole-L2 writeback and
//      invalidate per XCD) is issued.
// fp8 (OCP E4M3FN) caches are converted exactly to bf16 for the MFMA; the K
// scale multiplies the scores and the V scale multiplies P.  fp32 caches use a
// VALU path.
// The same kernel serves multi-token rows (a few query rows per sequence, each
// masked at its causal position, up to two 16-row tiles per wave) and packed
// GRPO groups (the members of a group in the rows of one tile, the shared prompt
// pages streamed once per pack); see decode_attention_kernel.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include <mutex>

#include "rlda_decode.h"
#include "rlda_device.h"
#include "rlda_params.h"

// Flags, segment counters and partial slots of rl_decode_attn_run_noalloc, for
// callers that cannot allocate device memory (layout in rlda_params.h).  Each GPU
// the library runs on holds its own copy until the process ends.  In host code the
// name stands for a host-side handle, never a device address: the address comes
// from hipGetSymbolAddress (noalloc_scratch below).
static __device__ __align__(256) unsigned char scratch[rlda::kScratchBytes];

namespace rlda {
namespace {

// ---------------------------------------------------------------- prompt pass (grouped runs)
// One workgroup per job (group i, KV head g, member block): the job's query rows
// are the G heads of each of up to 64/G members (row = (member - first) * G +
// head index), packed into up to 4 MFMA tiles of 16 rows.  The 4 waves split the
// group's prompt pages; each page is loaded once and multiplied against every
// tile, so the group reads its prompt once per KV head instead of once per
// response.  One wave per SIMD leaves a tile's chain of products, maximum and
// exponentials uncovered, so the tiles in use go through it in lockstep (GRPO with
// 4096-token prompts: the call 122.3 us one tile after another, 120.7 so).  The 4 waves' states are merged through LDS and each row's
// unnormalised (m, l, O) is stored for the attention kernel, which continues
// every member's softmax from it.  The job of block 0 of KV head 0 also stores
// the group's clamped prompt length.
constexpr int kPromptTiles = 4;

template <int D, bool FP8>
__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads), amdgpu_waves_per_eu(1, 1)))
void prompt_kernel(const Params p) {
  using Pol = Mfma<D, FP8>;
  constexpr int R = kPromptTiles, kRows = 16 * R, kDepth = Pol::kDepth;
  __shared__ __align__(16) float s_acc[kWaves][kRows][D + 4];
  __shared__ __align__(16) float s_ml[kWaves][kRows][2];
  __shared__ int32_t s_min;

  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int Hkv = p.num_kv_heads, G = p.group, Hq = p.num_q_heads, n = p.group_size;
  const int cap = p.max_pages * kPage;
  const int job = blockIdx.x / p.pfx_splits, split = blockIdx.x - job * p.pfx_splits;
  const int mb = job % p.pfx_nblocks, ig = job / p.pfx_nblocks;
  const int g = ig % Hkv, gi = ig / Hkv;
  const int b0 = gi * n, b1 = min(b0 + n, p.batch);                        // members of group gi
  const int m0 = b0 + mb * p.pfx_mblock, m1 = min(m0 + p.pfx_mblock, b1);  // members of this job

  for (int e = tid; e < Hq; e += kThreads) s_qhead[e] = p.q_head[e];
  if (tid == 0) s_min = 0x7fffffff;
  __syncthreads();
  // Shared prompt: the requested pages, clamped to the full pages of the shortest member.
  {
    int mn = 0x7fffffff;
    for (int b = b0 + tid; b < b1; b += kThreads) mn = min(mn, min(max(p.seq_lens[b], 0), cap) / kPage);
    if (mn != 0x7fffffff) atomicMin(&s_min, mn);
  }
  __syncthreads();
  const int want = p.prefix_pages[gi];
  const int P = uni(max(0, min(want, s_min)));
  if (tid == 0 && g == 0 && mb == 0 && split == 0) {
    p.gprefix[gi] = P;
    if (want != P) atomicOr(p.flags, kFlagPrefixClamped);
  }
  const int rows = (m1 - m0) * G;
  // Workgroups per job: at least 32 pages each (8 per wave), at most the launched
  // p.pfx_splits; the others have nothing to do.  A split costs a device-scope
  // handoff, which only pays off for long prompts.
  const int S = uni(min(p.pfx_splits, max(1, (P + 31) / 32)));
  if (P == 0 || rows <= 0 || split >= S) return;
  const int nt = uni((rows + 15) / 16);   // tiles in use

  Pol t[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    t[r].setup(p, lane, p.stride_slot);
    typename Pol::QOp qo;
    Pol::load_q_rows(qo, p, g, m0, rows, 16 * r, lane);
    t[r].begin(qo, p, 0, 0, lane);
  }

  // This wave's prompt pages [j0, j1) (the job's pages cut into S * 4 ranges), read
  // from the group's first member's row.
  const int ws = split * kWaves + wave;
  const int j0 = ws * P / (S * kWaves), j1 = (ws + 1) * P / (S * kWaves);
  const int32_t* bt = p.block_table + (int64_t)b0 * p.max_pages;
  const int rec = (kPage - 1) * p.stride_slot + D * Pol::kEB;   // a full page
  auto stream = [&](auto tiles) {
    constexpr int N = decltype(tiles)::value;
    for (int cb = j0; cb < j1; cb += kChunk) {
      const int cn = min(kChunk, j1 - cb);
      int pid = bt[cb + min(lane, cn - 1)];
      typename Pol::Frag fr[kDepth];
      float skm[kDepth], svm[kDepth];
      int sval[kDepth];
      // Every step issues the same loads (past the range with descriptors of no
      // records, which read nothing), so the loads stay in flight across steps.
      auto issue = [&](typename Pol::Frag& f, int& val, float& ks, float& vs, int k) {
        int pk = -1;
        if (k < cn) {
          pk = __builtin_amdgcn_readlane(pid, k);
          if ((unsigned)pk >= (unsigned)p.num_pages) {   // not a page of the pool: contributes nothing
            if (lane == 0) atomicOr(p.flags, kFlagBadPage);
            pk = -1;
          }
        }
        val = pk >= 0 ? kPage : 0;
        const int64_t po = (pk >= 0) ? (int64_t)pk * p.stride_page + (int64_t)g * p.stride_head : 0;
        const uint32_t nrec = pk >= 0 ? (uint32_t)rec : 0u;
        ks = 1.f;
        vs = 1.f;
        if constexpr (FP8) {
          const int64_t si = (pk >= 0) ? (int64_t)pk * Hkv + g : 0;
          const uint32_t sb = (pk >= 0) ? 4u : 0u;
          ks = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(make_rsrc_uni(p.k_scale + si, sb), 0, 0, 0));
          vs = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(make_rsrc_uni(p.v_scale + si, sb), 0, 0, 0));
        }
        t[0].issue(f, make_rsrc_uni((const char*)p.k + po, nrec), make_rsrc_uni((const char*)p.v + po, nrec));
      };
#pragma unroll
      for (int k = 0; k < kDepth - 1; ++k) issue(fr[k], sval[k], skm[k], svm[k], k);
      for (int i = 0; i < cn; i += kDepth) {
#pragma unroll
        for (int k = 0; k < kDepth; ++k) {
          const int si = (k + kDepth - 1) % kDepth;
          issue(fr[si], sval[si], skm[si], svm[si], i + k + kDepth - 1);
          if (i + k < cn) Pol::template compute_tiles<N>(t, fr[k], sval[k], p.scale_log2 * skm[k], svm[k]);
        }
      }
    }
  };
  // The loop is compiled for each number of tiles in use.
  switch (nt) {
    case 1: stream(std::integral_constant<int, 1>{}); break;
    case 2: stream(std::integral_constant<int, 2>{}); break;
    case 3: stream(std::integral_constant<int, 3>{}); break;
    default: stream(std::integral_constant<int, 4>{}); break;
  }
#pragma unroll
  for (int r = 0; r < R; ++r) t[r].to_lds(s_acc[wave] + 16 * r, s_ml[wave] + 16 * r, lane);
  __syncthreads();

  // Merge the 4 waves' states: thread (row, quarter of d).
  constexpr int DQ = D / 4;
  const int row = tid >> 2, d0 = (tid & 3) * DQ;
  float M = neg_inf(), Ls = 0.f, o[DQ];
#pragma unroll
  for (int e = 0; e < DQ; ++e) o[e] = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    float v[DQ];
#pragma unroll
    for (int c = 0; c < DQ; c += 4) *(f32x4*)&v[c] = *(const f32x4*)&s_acc[w][row][d0 + c];
    lse_merge<DQ>(M, Ls, o, s_ml[w][row][0], s_ml[w][row][1], v);
  }
  if (S > 1) {
    // The job is split over S workgroups: publish this one's state in slot
    // job * S + split (device scope, rows of 64), count it, and let the workgroup
    // that completes the count merge the S states in split order.
    const __amdgpu_buffer_rsrc_t ra = make_rsrc_uni(p.part_acc, (uint32_t)p.pfx_slots * kRows * D * 4u);
    const __amdgpu_buffer_rsrc_t rm = make_rsrc_uni(p.part_ml, (uint32_t)p.pfx_slots * kRows * 8u);
    const int slot_row = (job * p.pfx_splits + split) * kRows + row;
#pragma unroll
    for (int c = 0; c < DQ; c += 4)
      __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(o[c]), __float_as_uint(o[c + 1]),
                                                   __float_as_uint(o[c + 2]), __float_as_uint(o[c + 3])},
                                             ra, (slot_row * D + d0 + c) * 4, 0, kDeviceScope);
    if ((tid & 3) == 0)
      __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(M), __float_as_uint(Ls)}, rm, slot_row * 8, 0,
                                            kDeviceScope);
    __builtin_amdgcn_s_waitcnt(0);   // this wave's device-scope stores have completed
    __syncthreads();                 // ... and every other wave's
    if (tid == 0) {
      const uint32_t old = atomicAdd(p.counters + job, 1u);
      if (old >= (uint32_t)S) atomicOr(p.flags, kFlagStaleState);   // more pieces than the job has
      s_min = (old + 1u == (uint32_t)S);
    }
    __syncthreads();
    if (!s_min) return;
    if (tid == 0) atomicExch(p.counters + job, 0u);
    M = neg_inf();
    Ls = 0.f;
#pragma unroll
    for (int e = 0; e < DQ; ++e) o[e] = 0.f;
    constexpr int kBatch = 4;
    for (int k0 = 0; k0 < S; k0 += kBatch) {
      u32x2 ml[kBatch];
      float v[kBatch][DQ];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int sr = (job * p.pfx_splits + min(k0 + i, S - 1)) * kRows + row;   // past the last split: re-read, unused
        ml[i] = __builtin_amdgcn_raw_buffer_load_b64(rm, sr * 8, 0, kDeviceScope);
#pragma unroll
        for (int c = 0; c < DQ; c += 4)
          *(u32x4*)&v[i][c] = __builtin_amdgcn_raw_buffer_load_b128(ra, (sr * D + d0 + c) * 4, 0, kDeviceScope);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (k0 + i < S) lse_merge<DQ>(M, Ls, o, __uint_as_float(ml[i][0]), __uint_as_float(ml[i][1]), v[i]);
    }
  }
  if (row >= rows) return;
  const int b = m0 + row / G, h = s_qhead[g * G + row % G];
  const int64_t orow = (int64_t)b * Hq + h;
  float* dst = p.pfx_acc + orow * D + d0;
#pragma unroll
  for (int c = 0; c < DQ; c += 4) *(f32x4*)(dst + c) = f32x4{o[c], o[c + 1], o[c + 2], o[c + 3]};
  if ((tid & 3) == 0) *(f32x2*)(p.pfx_ml + orow * 2) = f32x2{M, Ls};
}

// ---------------------------------------------------------------- KV append
// One wave per (sequence, KV head) and cache (K or V; one wave for both where they are the
// same memory, since each reads and rewrites the page): lane l owns elements
// [l * E, (l + 1) * E) of the new row, E = D / 64.  bf16 / fp32 caches copy the row into
// its slot.  fp8 caches keep the page's scale covering every row written so far: the
// first row of a page sets amax / 448; a later row with a larger amax raises the scale
// and re-encodes the earlier rows (decode, times old/new scale, round to nearest even),
// four lanes a row, all rows at once.  What bounds it is latency: length, page id and
// scale are dependent reads; the row is read beside the length.  Append and decode of 18
// to 349 short fp8 sequences: 1.4 to 1.9 us less than with K and V in turn in one wave.

// E4M3 (OCP FN) encoding of two fp32 values into the low 16 bits, round to nearest even.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}

// One sequence, KV head and cache.
template <int D, KvKind KIND>
__device__ __forceinline__ void append_row(const Params& p, int item, bool is_v, int lane) {
  constexpr int E = D / 64;
  const int b = item / p.num_kv_heads, g = item - b * p.num_kv_heads;
  char* cache = (char*)(is_v ? p.v : p.k);
  const void* in = is_v ? p.v_in : p.k_in;
  typedef typename std::conditional<KIND == KvKind::F32, float, uint16_t>::type Elem;
  Elem x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = ((const Elem*)in)[(int64_t)item * D + lane * E + e];

  const int cap = p.max_pages * kPage;
  const int L = uni(p.seq_lens[b]);
  if (L < 1 || L > cap) {
    if ((L < 0 || L > cap) && lane == 0) atomicOr(p.flags, kFlagBadLen);
    return;
  }
  const int t = L - 1, slot = t % kPage;
  const int pid = uni(p.block_table[(int64_t)b * p.max_pages + t / kPage]);
  if ((unsigned)pid >= (unsigned)p.num_pages) {
    if (lane == 0) atomicOr(p.flags, kFlagBadPage);
    return;
  }
  char* page = cache + (int64_t)pid * p.stride_page + (int64_t)g * p.stride_head;   // slot 0
  if constexpr (KIND != KvKind::FP8) {
    Elem* dst = (Elem*)(page + (int64_t)slot * p.stride_slot) + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) dst[e] = x[e];
  } else {
    float* scale = (float*)(is_v ? p.v_scale : p.k_scale) + ((int64_t)pid * p.num_kv_heads + g);
    float s = slot > 0 ? *scale : 0.f;
    if (!(s > 0.f) || __builtin_isinf(s)) s = 0.f;
    float v[E], amax = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      v[e] = __uint_as_float((uint32_t)x[e] << 16);
      amax = fmaxf(amax, fabsf(v[e]));   // never NaN; as an integer in the order of its value
    }
    amax = __builtin_bit_cast(float, __builtin_amdgcn_readlane(wave_scan_max(__builtin_bit_cast(int, amax)), 63));
    float s_new = s;
    if (slot == 0 || amax > 448.f * s) {
      s_new = amax / 448.f;
      // Earlier rows of the page (slot > 0 only): re-encode at the new scale.
      const float ratio = s > 0.f ? s / s_new : 0.f;
      if ((lane >> 2) < slot) {
        constexpr int N = D / 64;   // 16-byte loads of a quarter row
        u32x4* rp = (u32x4*)(page + (int64_t)(lane >> 2) * p.stride_slot + (lane & 3) * (D / 4));
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
    uint8_t* dst = (uint8_t*)(page + (int64_t)slot * p.stride_slot) + lane * E;
    if constexpr (E == 2)
      *(uint16_t*)dst = (uint16_t)(s_new > 0.f ? e4m3x2(v[0] / s_new, v[1] / s_new) : 0u);
    else
      *dst = (uint8_t)(s_new > 0.f ? e4m3x2(v[0] / s_new, 0.f) & 0xFFu : 0u);
    if (lane == 0) *scale = s_new;
  }
}

template <int D, KvKind KIND>
__global__ __launch_bounds__(kThreads) void append_kernel(const Params p) {
  const int lane = threadIdx.x & 63;
  const int wave = uni((int)(blockIdx.x * kWaves + (threadIdx.x >> 6)));
  const int item = wave >> 1;
  if (item >= p.batch * p.num_kv_heads) return;
  const bool is_v = wave & 1;
  // One cache (or one scale array) given as both: K, then V, in one wave.
  const bool one = p.k == p.v || (KIND == KvKind::FP8 && p.k_scale == p.v_scale);
  if (one && is_v) return;
  append_row<D, KIND>(p, item, is_v, lane);
  if (one) {
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    append_row<D, KIND>(p, item, true, lane);
  }
}

template <int D, KvKind KIND>
int launch_append_t(const Params& p, void* stream) {
  const int items = p.batch * p.num_kv_heads;
  hipLaunchKernelGGL((append_kernel<D, KIND>), dim3((items + kWaves / 2 - 1) / (kWaves / 2)), dim3(kThreads), 0,
                     (hipStream_t)stream, p);
  return (int)hipGetLastError();
}

template <int D, bool FP8>
int launch_prompt_then_decode(const Params& p, int ngroups, void* stream, void* ev_begin, void* ev_end) {
  hipStream_t st = (hipStream_t)stream;
  if (ev_begin && hipEventRecord((hipEvent_t)ev_begin, st) != hipSuccess) return -1;
  const int jobs = ngroups * p.num_kv_heads * p.pfx_nblocks;
  hipLaunchKernelGGL((prompt_kernel<D, FP8>), dim3(jobs * p.pfx_splits), dim3(kThreads), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return (int)e;
  return launch<Mfma<D, FP8>, false, 1, false, true>(p, stream, nullptr, ev_end);
}

std::mutex g_scratch_mu;
void* g_scratch_ptr[64];

}  // namespace

int noalloc_scratch(void** ptr) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return -1;
  std::lock_guard<std::mutex> lk(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    // With `dev` current: this device's copy of the array.
    void* a = nullptr;
    if (hipGetSymbolAddress(&a, HIP_SYMBOL(scratch)) != hipSuccess || !a) return -1;
    g_scratch_ptr[dev] = a;
  }
  *ptr = g_scratch_ptr[dev];
  return 0;
}

#define RLDA_DISPATCH(FN, ...)                                                  \
  switch (kind) {                                                               \
    case KvKind::BF16:                                                          \
      return head_dim == 128 ? FN<Mfma<128, false>>(__VA_ARGS__)                \
                             : FN<Mfma<64, false>>(__VA_ARGS__);                \
    case KvKind::FP8:                                                           \
      return head_dim == 128 ? FN<Mfma<128, true>>(__VA_ARGS__)                 \
                             : FN<Mfma<64, true>>(__VA_ARGS__);                 \
    case KvKind::F32:                                                           \
      if (head_dim == 128) return FN<Valu<128, 1>>(__VA_ARGS__);                \
      return group == 1 ? FN<Valu<64, 1>>(__VA_ARGS__) : FN<Valu<64, 2>>(__VA_ARGS__); \
  }                                                                             \
  return -1;

int launch_decode(KvKind kind, int head_dim, int group, const Params& p, void* stream, void* ev_begin,
                  void* ev_end) {
  RLDA_DISPATCH(launch, p, stream, ev_begin, ev_end)
}

template <class Pol>
int launch_rows(int tiles, const Params& p, void* stream, void* ev_begin, void* ev_end) {
  return tiles == 2 ? launch<Pol, true, 2>(p, stream, ev_begin, ev_end) : launch<Pol, true, 1>(p, stream, ev_begin, ev_end);
}

template <class Pol>
int launch_packed(int tiles, const Params& p, void* stream, void* ev_begin, void* ev_end) {
  return tiles == 1 ? launch<Pol, true, 1, true>(p, stream, ev_begin, ev_end) : -1;
}

int launch_decode_rows(KvKind kind, int head_dim, int tiles, const Params& p, void* stream, void* ev_begin,
                       void* ev_end) {
  switch (kind) {
    case KvKind::BF16:
      return head_dim == 128 ? launch_rows<Mfma<128, false>>(tiles, p, stream, ev_begin, ev_end)
                             : launch_rows<Mfma<64, false>>(tiles, p, stream, ev_begin, ev_end);
    case KvKind::FP8:
      return head_dim == 128 ? launch_rows<Mfma<128, true>>(tiles, p, stream, ev_begin, ev_end)
                             : launch_rows<Mfma<64, true>>(tiles, p, stream, ev_begin, ev_end);
    case KvKind::F32:
      break;
  }
  return -1;
}

int launch_decode_packed(KvKind kind, int head_dim, int tiles, const Params& p, void* stream, void* ev_begin,
                         void* ev_end) {
  switch (kind) {
    case KvKind::BF16:
      return head_dim == 128 ? launch_packed<Mfma<128, false>>(tiles, p, stream, ev_begin, ev_end)
                             : launch_packed<Mfma<64, false>>(tiles, p, stream, ev_begin, ev_end);
    case KvKind::FP8:
      return head_dim == 128 ? launch_packed<Mfma<128, true>>(tiles, p, stream, ev_begin, ev_end)
                             : launch_packed<Mfma<64, true>>(tiles, p, stream, ev_begin, ev_end);
    case KvKind::F32:
      break;
  }
  return -1;
}

int launch_decode_two(KvKind kind, int head_dim, const Params& p, void* stream, void* ev_begin, void* ev_end) {
  if (kind == KvKind::BF16)
    return head_dim == 64 ? launch<Mfma<64, false>, false, 1, false, false, 2>(p, stream, ev_begin, ev_end) : -1;
  if (kind != KvKind::FP8) return -1;
  return head_dim == 128 ? launch<Mfma<128, true>, false, 1, false, false, 2>(p, stream, ev_begin, ev_end)
                         : launch<Mfma<64, true>, false, 1, false, false, 2>(p, stream, ev_begin, ev_end);
}

int launch_append(KvKind kind, int head_dim, const Params& p, void* stream) {
  switch (kind) {
    case KvKind::BF16:
      return head_dim == 128 ? launch_append_t<128, KvKind::BF16>(p, stream) : launch_append_t<64, KvKind::BF16>(p, stream);
    case KvKind::FP8:
      return head_dim == 128 ? launch_append_t<128, KvKind::FP8>(p, stream) : launch_append_t<64, KvKind::FP8>(p, stream);
    case KvKind::F32:
      return head_dim == 128 ? launch_append_t<128, KvKind::F32>(p, stream) : launch_append_t<64, KvKind::F32>(p, stream);
  }
  return -1;
}

int launch_grouped(KvKind kind, int head_dim, int, const Params& p, int ngroups, void* stream, void* ev_begin,
                   void* ev_end) {
  switch (kind) {
    case KvKind::BF16:
      return head_dim == 128 ? launch_prompt_then_decode<128, false>(p, ngroups, stream, ev_begin, ev_end)
                             : launch_prompt_then_decode<64, false>(p, ngroups, stream, ev_begin, ev_end);
    case KvKind::FP8:
      return head_dim == 128 ? launch_prompt_then_decode<128, true>(p, ngroups, stream, ev_begin, ev_end)
                             : launch_prompt_then_decode<64, true>(p, ngroups, stream, ev_begin, ev_end);
    case KvKind::F32:
      break;
  }
  return -1;
}


}  // namespace rlda
