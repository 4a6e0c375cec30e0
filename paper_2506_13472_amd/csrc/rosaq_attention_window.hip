// Attention over the quantised cache with a window: the kernels of rosaq_attend.h whose rows look back `window` tokens and to the first `sinks`.
#include "rosaq_attend.h"

namespace rosaq {

template <int D, int BITS> static void run(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  launch_own<D, BITS, true>(a, p, st);
  if (p.parts > 1) launch_join<D, true>(a, p, st);
}

void launch_attention_window(const AttendArgs& a, const AttendPlan& p, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a.dim == 128) a.bits == 4 ? run<128, 4>(a, p, st) : run<128, 8>(a, p, st);
  else a.bits == 4 ? run<64, 4>(a, p, st) : run<64, 8>(a, p, st);
}

}  // namespace rosaq
