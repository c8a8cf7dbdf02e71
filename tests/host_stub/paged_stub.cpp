// Host-only stand-ins for the launchers of the paged operators, as launch_stub.cpp has them for
// the rest: every launch reports a device error.
#include "paged.h"

namespace aatc {

aatc_status launch_turn(const TurnArgs&, aatc_dtype, aatc_dtype, int, void*) { return AATC_E_DEVICE; }
size_t paged_workspace_bytes(int batch, int n_q_heads, int) {
  return (size_t)batch * n_q_heads * 256 + 1024;
}
aatc_status launch_paged(PagedArgs, aatc_dtype, void*, void*) { return AATC_E_DEVICE; }
aatc_status launch_decode_paged(const void*, const void*, int, int, int, const void*, aatc_dtype,
                                const void*, const uint16_t*, const void*, const uint16_t*,
                                const int32_t*, int64_t, int, int, float, float*, void*, void*,
                                const PagedArgs&, aatc_dtype, void*) {
  return AATC_E_DEVICE;
}
aatc_status launch_pages_copy(void*, int64_t, int64_t, int64_t, int64_t, const int32_t*, int64_t,
                              const int32_t*, void*) {
  return AATC_E_DEVICE;
}
aatc_status launch_pages_fork(const aatc_page_table&, const aatc_page_table&, int32_t*, int64_t,
                              const int32_t*, int64_t, void*) {
  return AATC_E_DEVICE;
}
aatc_status launch_pages_free(const aatc_page_table&, int32_t*, int64_t, const int32_t*, int64_t,
                              void*) {
  return AATC_E_DEVICE;
}
size_t pages_workspace_bytes(int64_t rows, int64_t n_pages) { return (size_t)(2 * rows + n_pages) * 4; }
aatc_status launch_pages_reserve(const aatc_page_table&, int32_t*, int64_t, int, const int32_t*,
                                 const int32_t*, int32_t*, int32_t*, void*, void*) {
  return AATC_E_DEVICE;
}
aatc_status launch_pages_compact(const aatc_page_table&, const int32_t*, int64_t,
                                 const aatc_page_table&, int32_t*, int32_t*, int32_t*, void*,
                                 void*) {
  return AATC_E_DEVICE;
}

}  // namespace aatc
