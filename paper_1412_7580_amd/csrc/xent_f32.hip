// The linear cross entropy on f32 operands.
#include "xent_impl.hpp"

namespace fc {
hipError_t xent_fprop_f32(const XentCall &c, void *ws, hipStream_t s) { return Xent<float>(c, false, ws, s).fprop(); }
hipError_t xent_backward_f32(const XentCall &c, void *ws, hipStream_t s) { return Xent<float>(c, true, ws, s).backward(); }

size_t xent_bytes(bool backward, int dtype, long N, int D, int V, bool aligned) {
    return N ? xent_plan(backward, dtype, N, D, V, aligned).total : 0;
}
bool xent_fits(bool backward, int dtype, long N, int D, int V, int T) {
    return N == 0 || xent_launchable(xent_plan(backward, dtype, N, D, V, false), backward, N, D, T);
}
}  // namespace fc
