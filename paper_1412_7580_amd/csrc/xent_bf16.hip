// The linear cross entropy on bf16 operands.
#include "xent_impl.hpp"

namespace fc {
hipError_t xent_fprop_bf16(const XentCall &c, void *ws, hipStream_t s) { return Xent<__bf16, __bf16, false>(c, false, ws, s).fprop(); }
hipError_t xent_backward_bf16(const XentCall &c, void *ws, hipStream_t s) { return Xent<__bf16, __bf16, false>(c, true, ws, s).backward(); }
}  // namespace fc
