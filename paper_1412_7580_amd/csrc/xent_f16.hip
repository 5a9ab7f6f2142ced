// The linear cross entropy on f16 operands.
#include "xent_impl.hpp"

namespace fc {
hipError_t xent_fprop_f16(const XentCall &c, void *ws, hipStream_t s) { return Xent<_Float16>(c, false, ws, s).fprop(); }
hipError_t xent_backward_f16(const XentCall &c, void *ws, hipStream_t s) { return Xent<_Float16>(c, true, ws, s).backward(); }
}  // namespace fc
