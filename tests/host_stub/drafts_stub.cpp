// Host-only stand-ins for the launchers of drafted tokens and sparse attention, as paged_stub.cpp has
// them for the other operators over pages: every launch reports a device error.
#include "drafts.h"
#include "sparse.h"

namespace aatc {

size_t tree_workspace_bytes(int batch, int drafts, int n_q_heads, int) {
  return (size_t)batch * drafts * n_q_heads * 256 + 1024;
}
bool tree_fits(int64_t, int drafts, int n_q_heads, int n_kv_heads) {
  return (int64_t)drafts * (n_q_heads / n_kv_heads) <= kMaxColumns;
}
aatc_status launch_tree(TreeArgs, aatc_dtype, void*, void*) { return AATC_E_DEVICE; }
aatc_status launch_tree_accept(const AcceptArgs&, void*) { return AATC_E_DEVICE; }

aatc_status launch_bounds(const BoundsArgs&, aatc_dtype, void*) { return AATC_E_DEVICE; }
size_t sparse_workspace_bytes(int batch, int n_q_heads, int n_kv_heads, int64_t max_pages) {
  return (size_t)batch * (n_q_heads * 256 + n_kv_heads * max_pages * 4) + 1024;
}
bool sparse_fits(int64_t batch, int n_q_heads, int n_kv_heads, int64_t max_pages) {
  return n_q_heads / n_kv_heads <= kMaxSay &&
         max_pages <= ((int64_t)1 << 30) / (batch * n_kv_heads);
}
aatc_status launch_sparse(SparseArgs, aatc_dtype, void*, void*) { return AATC_E_DEVICE; }

}  // namespace aatc
