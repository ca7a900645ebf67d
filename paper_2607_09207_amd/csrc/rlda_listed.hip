// Decode attention whose work list has query rows as its units, for gfx950: over the pages
// that every (row, KV head) lists, and over all pages with the weight that each page gets.
// The page stream, softmax, cuts and merge are those of rlda_kernels.hip; a position's page
// is looked up in the list first (kListed), or the part of the row's sum that a page brings is
// stored beside the attention (kWeighed), 4 bytes a page and query head.
//   Reading the pages bounds both: 128 listed pages of each of 64 sequences (28/4 heads, bf16, 267
// MB) 46 us, 5.8 TB/s; 64 of each of 256 (40/8, fp8, 532 MB) 96.5, 5.5 TB/s; weights of a long-tailed
// batch of 64 (28/4, bf16, 462 MB) 86.9 of which 4.8 are the second launch, the plain call 79.6.  The
// probabilities' bf16 remainders enter every product here: the calls take the same time with
// and without, and a bf16 result's error falls from 2.4e-3 to the 1.7e-3 of its own rounding.
//   Every row reads its pages for itself, so n rows of a sequence read its cache n times: 1, 4 and 32
// rows of each of 16 long-tailed sequences (28/4, bf16, 119 MB) 35.4, 89 and 629 us with weights, and 404
// MB and 3.29 GB read for 4 and 32 rows.
//   With z = log2 of the sum of exp2(score) over a row's keys and z_j over page j's of them,
// page j's weight is exp2(z_j - z), summed over heads and rows in one order by a second, small
// launch: the attention has to have every piece of a row before z is known.
#include "rlda_decode.h"
#include "rlda_params.h"

namespace rlda {
namespace {

// A lane a page of a sequence, the rows' heads dealt out to the waves: wave w adds those of w, w +
// 4, ... in order, wave 0 the four sums.  All of a lane's loads are in flight at once (one wave
// with every head, eight at a time: 11.6 us for 64 long-tailed sequences of 28 heads).
// STARTS: with q_start.
template <bool STARTS>
__global__ __launch_bounds__(kThreads) void page_weights_kernel(const Params p) {
  __shared__ float s_sum[kWaves][64];
  constexpr int H = 8;   // heads of a wave whose parts are asked for together
  const int b = blockIdx.x, Hq = p.num_q_heads, cap = p.max_pages * kPage;
  const int lane = threadIdx.x & 63, wave = uni((int)(threadIdx.x >> 6));
  const auto load = [&](float* a, int row, int h0, int j, bool seen) {
    const float* zj = p.page_lse + (int64_t)row * Hq * p.max_pages + j;
#pragma unroll
    for (int k = 0; k < H; ++k) {
      const int h = h0 + k * kWaves;
      a[k] = seen && h < Hq ? zj[(int64_t)h * p.max_pages] : neg_inf();
    }
  };
  float* const w = p.weights + (int64_t)b * p.max_pages;
  // One row a sequence: the first pages' parts and weights, ahead of the length.
  const bool early = !STARTS && blockIdx.y == 0;
  float first[H], old = 0.f;
  if (early) {
    const int j = min(lane, p.max_pages - 1);
    load(first, b, wave, j, true);
    if (wave == 0 && p.decay != 0.f) old = w[j];
  }
  const int L = min(max(p.seq_lens[b], 0), cap), npages = (L + kPage - 1) / kPage;
  int q0 = b, n = 1;
  if constexpr (STARTS) {
    q0 = p.q_start[b];
    const int q1 = p.q_start[b + 1];
    n = q0 >= 0 && q0 <= q1 && q1 <= p.total_q ? q1 - q0 : 0;
  }
  if (n == 0) return;
  for (int j0 = blockIdx.y * 64; j0 < npages; j0 += gridDim.y * 64) {
    const int j = j0 + lane, at = min(j, npages - 1);
    const bool have = early && j0 == 0;
    if (!have && wave == 0 && p.decay != 0.f) old = w[at];
    float got = 0.f;
    bool any = !STARTS;
    for (int i = 0; i < n; ++i) {
      // (Where offsets run backwards, the attention may have taken the row as another's.)
      const bool own = !STARTS || p.row_seq[q0 + i] == b;
      any |= own;
      const bool seen = L - n + i >= kPage * at;   // by the row
      const float* z = p.row_lse + (int64_t)(q0 + i) * Hq;
      for (int h0 = wave; h0 < Hq; h0 += H * kWaves) {
        float a[H];
        if (have && h0 == wave) {
#pragma unroll
          for (int k = 0; k < H; ++k) a[k] = first[k];   // (past the pages: used by no lane that writes)
        } else {
          load(a, q0 + i, h0, at, seen);
        }
#pragma unroll
        for (int k = 0; k < H; ++k)   // (no key: nothing, whatever the row's sum is)
          if (own && a[k] != neg_inf()) got += __builtin_amdgcn_exp2f(a[k] - z[min(h0 + k * kWaves, Hq - 1)]);
      }
    }
    s_sum[wave][lane] = got;
    __syncthreads();
    if (wave == 0 && j < npages && any) {
      got = s_sum[0][lane] + s_sum[1][lane] + s_sum[2][lane] + s_sum[3][lane];
      w[j] = p.decay == 0.f ? got : __builtin_fmaf(p.decay, old, got);
    }
    __syncthreads();
  }
}

template <class Pol, RowsForm ROWS>
int launch_rows_t(bool two, const Params& p, void* stream, void* ev_begin, void* ev_end) {
  if constexpr (Pol::kHalfPages)
    if (two) return launch<Pol, false, 1, false, false, 2, false, ROWS>(p, stream, ev_begin, ev_end);
  return two ? -1 : launch<Pol, false, 1, false, false, 1, false, ROWS>(p, stream, ev_begin, ev_end);
}

template <RowsForm ROWS>
int launch_rows_form(KvKind kind, int head_dim, int group, bool two, const Params& p, void* stream, void* ev_begin,
                     void* ev_end) {
  switch (kind) {
    case KvKind::BF16:
      return head_dim == 128 ? launch_rows_t<Mfma<128, false>, ROWS>(two, p, stream, ev_begin, ev_end)
                             : launch_rows_t<Mfma<64, false>, ROWS>(two, p, stream, ev_begin, ev_end);
    case KvKind::FP8:
      return head_dim == 128 ? launch_rows_t<Mfma<128, true>, ROWS>(two, p, stream, ev_begin, ev_end)
                             : launch_rows_t<Mfma<64, true>, ROWS>(two, p, stream, ev_begin, ev_end);
    case KvKind::F32:
      return head_dim == 128 ? launch_rows_t<Valu<128, 1>, ROWS>(two, p, stream, ev_begin, ev_end)
             : group == 1    ? launch_rows_t<Valu<64, 1>, ROWS>(two, p, stream, ev_begin, ev_end)
                             : launch_rows_t<Valu<64, 2>, ROWS>(two, p, stream, ev_begin, ev_end);
  }
  return -1;
}

}  // namespace

int launch_selected(KvKind kind, int head_dim, int group, bool two, const Params& p, void* stream, void* ev_begin,
                    void* ev_end) {
  return launch_rows_form<kListed>(kind, head_dim, group, two, p, stream, ev_begin, ev_end);
}

int launch_weighed(KvKind kind, int head_dim, int group, bool two, const Params& p, void* stream, void* ev_begin,
                   void* ev_end) {
  const int e = launch_rows_form<kWeighed>(kind, head_dim, group, two, p, stream, ev_begin, nullptr);
  if (e != hipSuccess) return e;
  const int y = min((p.max_pages + 63) / 64, 256);
  if (p.q_start)
    hipLaunchKernelGGL(page_weights_kernel<true>, dim3(p.batch, y), dim3(kThreads), 0, (hipStream_t)stream, p);
  else
    hipLaunchKernelGGL(page_weights_kernel<false>, dim3(p.batch, y), dim3(kThreads), 0, (hipStream_t)stream, p);
  if (const hipError_t l = hipGetLastError(); l != hipSuccess) return (int)l;
  if (ev_end && hipEventRecord((hipEvent_t)ev_end, (hipStream_t)stream) != hipSuccess) return -1;
  return 0;
}

}  // namespace rlda
