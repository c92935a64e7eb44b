// The runtime without a device (fake_runtime.cpp), and the launchers of the kernels behind enl_attend_tree.
#include "fake_runtime.cpp"

namespace {
int g_grid, g_splits, g_box, g_deep;
}
extern "C" {
int fake_grid() { return g_grid; }
int fake_splits() { return g_splits; }
int fake_box() { return g_box; }
int fake_deep() { return g_deep; }
}
namespace enl {
cudaError_t prepare_tree(int) { return g_fail_kind == 'P' ? cudaErrorInvalidValue : cudaSuccess; }
cudaError_t launch_tree(const TreeParams &p, int, int grid, cudaStream_t)
{
    g_grid = grid;
    g_splits = p.n_splits;
    g_box = p.box_tokens;
    return note('t', p.wait_first);
}
cudaError_t launch_tree_merge(const TreeMergeParams &, int, int, bool deep, cudaStream_t)
{
    g_deep = deep;
    return note('u', 0);
}
}  // namespace enl
