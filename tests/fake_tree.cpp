// The runtime without a device (fake_runtime.cpp), and the launchers of the kernels behind enl_attend_tree.
#include "fake_runtime.cpp"

namespace {
int g_grid, g_splits, g_box, g_deep, g_tiles;
const enl::TreeSegment *g_segments;                  // of the last launch (device memory is host memory; there if the plan was copied)
const int32_t *g_segment_off;
const int2 *g_heads;
}
extern "C" {
int fake_grid() { return g_grid; }
int fake_splits() { return g_splits; }
int fake_box() { return g_box; }
int fake_groups() { return g_grid / g_tiles; }
int fake_segment_off(int i) { return g_segment_off[i]; }
int fake_segment(int i, int field) { return reinterpret_cast<const int32_t *>(g_segments + i)[field]; }
int fake_unit(int u, int field) { return field ? g_heads[u].y : g_heads[u].x; }
int fake_deep() { return g_deep; }
}
namespace enl {
cudaError_t prepare_tree(int) { return g_fail_kind == 'P' ? cudaErrorInvalidValue : cudaSuccess; }
cudaError_t launch_tree(const TreeParams &p, int, int grid, cudaStream_t)
{
    g_grid = grid;
    g_splits = p.n_splits;
    g_box = p.box_tokens;
    g_tiles = p.row_tiles;
    g_segments = p.segments;
    g_segment_off = p.segment_off;
    return note('t', p.wait_first);
}
cudaError_t launch_tree_merge(const TreeMergeParams &p, int, int, int most, cudaStream_t)
{
    g_deep = most > 4;
    g_heads = p.heads;
    return note('u', 0);
}
}  // namespace enl
