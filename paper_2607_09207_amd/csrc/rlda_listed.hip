// Decode attention whose work list has query rows as its units, for gfx950: over the pages
// that every (row, KV head) lists, and over all pages with the weight that each page gets.
// The page stream, softmax, cuts and merge are those of rlda_kernels.hip; a position's page
// is looked up in the list first (kListed), or the part of the row's sum that a page brings is
// stored beside the attention (kWeighed), 4 bytes a page and query head.
//   With z = log2 of the sum of exp2(score) over a row's keys and z_j over page j's of them,
// page j's weight is exp2(z_j - z), summed over heads and rows in one order by a second, small
// launch: the attention has to have every piece of a row before z is known.
#include "rlda_decode.h"
#include "rlda_params.h"

namespace rlda {
namespace {

// One thread a page of a sequence; its rows' heads in order.
__global__ __launch_bounds__(kThreads) void page_weights_kernel(const Params p) {
  const int b = blockIdx.x, Hq = p.num_q_heads, cap = p.max_pages * kPage;
  const int L = min(max(p.seq_lens[b], 0), cap), npages = (L + kPage - 1) / kPage;
  int q0 = b, n = 1;
  if (p.q_start) {
    q0 = p.q_start[b];
    const int q1 = p.q_start[b + 1];
    n = q0 >= 0 && q0 <= q1 && q1 <= p.total_q ? q1 - q0 : 0;
  }
  if (n == 0) return;
  for (int j = blockIdx.y * kThreads + threadIdx.x; j < npages; j += gridDim.y * kThreads) {
    float got = 0.f;
    for (int i = 0; i < n; ++i) {
      if (L - n + i < kPage * j) continue;   // the row does not see the page
      const float* z = p.row_lse + (int64_t)(q0 + i) * Hq;
      const float* zj = p.page_lse + (int64_t)(q0 + i) * Hq * p.max_pages + j;
#pragma unroll 8
      for (int h = 0; h < Hq; ++h) {
        const float a = zj[(int64_t)h * p.max_pages];
        if (a != neg_inf()) got += __builtin_amdgcn_exp2f(a - z[h]);   // (no key: nothing, whatever z is)
      }
    }
    float* w = p.weights + (int64_t)b * p.max_pages + j;
    *w = p.decay == 0.f ? got : __builtin_fmaf(p.decay, *w, got);
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
  const int y = min((p.max_pages + kThreads - 1) / kThreads, 64);
  hipLaunchKernelGGL(page_weights_kernel, dim3(p.batch, y), dim3(kThreads), 0, (hipStream_t)stream, p);
  if (const hipError_t l = hipGetLastError(); l != hipSuccess) return (int)l;
  if (ev_end && hipEventRecord((hipEvent_t)ev_end, (hipStream_t)stream) != hipSuccess) return -1;
  return 0;
}

}  // namespace rlda
