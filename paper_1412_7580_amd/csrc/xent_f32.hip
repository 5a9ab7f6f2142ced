// The linear cross entropy on f32 operands.
#include "xent_impl.hpp"

namespace fc {
hipError_t xent_fprop_f32(const XentCall &c, void *ws, hipStream_t s) { return Xent<float, __bf16, true>(c, false, ws, s).fprop(); }
hipError_t xent_backward_f32(const XentCall &c, void *ws, hipStream_t s) { return Xent<float, __bf16, true>(c, true, ws, s).backward(); }

// Enough for weights of any alignment.
size_t xent_bytes(bool backward, int dtype, long N, int D, int V) { return N ? xent_plan(backward, dtype, N, D, V, false).total : 0; }
}  // namespace fc
