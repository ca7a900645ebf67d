// Decode attention with modified scores for gfx950: a cap by tanh, a bias that grows with
// the distance, and for every query row the interval of keys that it sees (a window, packed
// documents, a prefix).  Same page stream, softmax and merge as rlda_kernels.hip:
//   y = scale q.k;  y = cap tanh(y / cap);  y -= slope |pos - t|;  keys outside the interval out.
// Pages that no row sees leave the list before it is cut into shares, so a window costs its
// own length.
// Reading the keys bounds it, as it does the plain kernel, and the scores' operations hide
// behind that: 64 sequences of a long-tailed cache (28/4 heads, 482 MB) with a bias 85 us, 5.6
// TB/s, without 84; 4 of up to 16384 tokens under a cap 31.5, without 31; 128 fp8 sequences, a
// window of 4096 and a cap 139 us (800 MB, 5.8 TB/s; 150 with masks and a bias of 0 computed on
// every page).
#include "rlda_decode.h"
#include "rlda_params.h"

namespace rlda {
namespace {

template <class Pol>
int launch_scored_t(bool two, const Params& p, void* stream, void* ev_begin, void* ev_end) {
  if constexpr (Pol::kHalfPages)
    if (two) return launch<Pol, false, 1, false, false, 2, true>(p, stream, ev_begin, ev_end);
  return two ? -1 : launch<Pol, false, 1, false, false, 1, true>(p, stream, ev_begin, ev_end);
}

template <class Pol>
int launch_scored_rows_t(int tiles, const Params& p, void* stream, void* ev_begin, void* ev_end) {
  return tiles == 2 ? launch<Pol, true, 2, false, false, 1, true>(p, stream, ev_begin, ev_end)
                    : launch<Pol, true, 1, false, false, 1, true>(p, stream, ev_begin, ev_end);
}

}  // namespace

#define RLDA_DISPATCH_MFMA(FN, ...)                                                                              \
  switch (kind) {                                                                                                \
    case KvKind::BF16:                                                                                           \
      return head_dim == 128 ? FN<Mfma<128, false>>(__VA_ARGS__) : FN<Mfma<64, false>>(__VA_ARGS__);             \
    case KvKind::FP8:                                                                                            \
      return head_dim == 128 ? FN<Mfma<128, true>>(__VA_ARGS__) : FN<Mfma<64, true>>(__VA_ARGS__);               \
    case KvKind::F32:                                                                                            \
      break;                                                                                                     \
  }                                                                                                              \
  return -1;

int launch_scored(KvKind kind, int head_dim, bool two, const Params& p, void* stream, void* ev_begin, void* ev_end) {
  RLDA_DISPATCH_MFMA(launch_scored_t, two, p, stream, ev_begin, ev_end)
}

int launch_scored_rows(KvKind kind, int head_dim, int tiles, const Params& p, void* stream, void* ev_begin,
                       void* ev_end) {
  RLDA_DISPATCH_MFMA(launch_scored_rows_t, tiles, p, stream, ev_begin, ev_end)
}

}  // namespace rlda
