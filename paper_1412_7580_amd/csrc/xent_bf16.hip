// The linear cross entropy on bf16 operands.
#include "xent_impl.hpp"

namespace fc {
hipError_t xent_fprop_bf16(const XentCall &c, void *ws, hipStream_t s) { return Xent<__bf16>(c, false, ws, s).fprop(); }
hipError_t xent_backward_bf16(const XentCall &c, void *ws, hipStream_t s) { return Xent<__bf16>(c, true, ws, s).backward(); }
}  // namespace fc
