// Host side of enl_attend_tree: checks, the gather plan of the selected groups, the launch of the kernels in enl_tree_sm100.cu.
#include <cmath>
#include <cstring>

#include "enl_cache.h"

using namespace enl;

namespace {

// Steps of 64 keys that a split takes at least.
constexpr int kMinSteps = 3;

}  // namespace

extern "C" int enl_attend_tree(enl_cache_t *c, const enl_attend_tree_args_t *a, void *cuda_stream)
{
    if (!c || !a) return ENL_E_INVAL;
    const enl_cache_desc_t &d = c->d;
    if (!c->gpu) return ENL_E_CUDA;
    if (a->layer < 0 || a->layer >= d.n_layers) return ENL_E_INVAL;
    if (a->batch < 1 || a->batch > d.max_batch || a->n_max < 1 || a->n_sel < 0 || a->max_blocks < 1 || a->n_pages < 1) return ENL_E_INVAL;
    if (a->n_sel > 0 && !a->sel_ids) return ENL_E_INVAL;
    const int B = a->batch;
    if (B > 1 && !a->cu_sel) return ENL_E_INVAL;
    const int32_t one_sel[2] = {0, a->n_sel};
    const int32_t *cu_sel = a->cu_sel ? a->cu_sel : one_sel;
    if (cu_sel[0] != 0 || cu_sel[B] != a->n_sel) return ENL_E_INVAL;
    for (int b = 0; b < B; ++b)
        if (cu_sel[b + 1] < cu_sel[b]) return ENL_E_INVAL;
    if (!a->tail_len || !a->block_table || !a->q || !a->k_new || !a->v_new || !a->k_tail || !a->v_tail || !a->out) return ENL_E_INVAL;
    const uintptr_t wide = reinterpret_cast<uintptr_t>(a->q) | reinterpret_cast<uintptr_t>(a->k_new) | reinterpret_cast<uintptr_t>(a->v_new) |
                           reinterpret_cast<uintptr_t>(a->k_tail) | reinterpret_cast<uintptr_t>(a->v_tail) | reinterpret_cast<uintptr_t>(a->out);
    const uintptr_t words = reinterpret_cast<uintptr_t>(a->tail_len) | reinterpret_cast<uintptr_t>(a->n_new) | reinterpret_cast<uintptr_t>(a->block_table);
    if ((wide & 15) || (words & 3) || (reinterpret_cast<uintptr_t>(a->mask) & 7)) return ENL_E_INVAL;
    if (a->n_max > ENL_TREE_MAX_NODES) return ENL_E_LIMIT;
    // TMA coordinates, and lengths in rows, are int32
    const int groups = kPageTokens / box_rows(d.head_dim);
    if (static_cast<int64_t>(a->n_pages) * d.n_kv_heads * groups > 0x3fffffff || a->max_blocks > 0x3fffffff / kPageTokens ||
        static_cast<int64_t>(B) * a->n_max > 0x3fffffff)
        return ENL_E_LIMIT;
    const int row_tiles = ceil_div(a->n_max * c->rep, kTileRows);
    const int64_t units = static_cast<int64_t>(B) * d.n_kv_heads * row_tiles;
    if (units > 0x3fffffff) return ENL_E_LIMIT;

    // ---- gather plan: the episodes' streams; reused when nothing it was built from has changed ----
    const size_t cu_bytes = sizeof(int32_t) * (B + 1);
    bool reuse = c->plan_valid && c->plan_tree && c->plan_epoch == c->epoch && c->plan_batch == B &&
                 c->key_sel.size() == static_cast<size_t>(a->n_sel) &&
                 (a->n_sel == 0 || std::memcmp(c->key_sel.data(), a->sel_ids, sizeof(int32_t) * a->n_sel) == 0) &&
                 std::memcmp(c->key_cu.data(), cu_sel, cu_bytes) == 0;
    if (!reuse || !c->plan_layer_ok[a->layer]) {
        if (const int rc = look_over(c, a->layer, B, a->sel_ids, cu_sel)) return rc;
        reuse = reuse && c->key_len == c->sel_len;
        if (reuse) c->plan_layer_ok[a->layer] = 1;
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    DeviceGuard dg(d.device);
    if (!reuse) {
        int64_t n_entries = 0;
        for (int b = 0; b < B; ++b) {
            int64_t e = 0;
            for (int s = cu_sel[b]; s < cu_sel[b + 1]; ++s) e += std::max(1, ceil_div(c->sel_len[s], kPageTokens));
            n_entries += (e + kPagesPerTile - 1) / kPagesPerTile * kPagesPerTile;
        }
        if (n_entries > c->cap_entries) return ENL_E_NOMEM;
        if (const int rc = open_plan(c)) return rc;
        auto align16 = [](size_t x) { return (x + 15) & ~static_cast<size_t>(15); };
        c->off_eps = 0;
        c->off_stream = align16(sizeof(EpInfo) * B);
        c->off_meta = c->off_stream + align16(sizeof(int32_t) * n_entries);
        c->plan_used = c->off_meta + align16(sizeof(int32_t) * n_entries);
        int32_t ne = 0, most = 0;
        for (int b = 0; b < B; ++b) {
            EpInfo &e = c->h_eps()[b];
            std::memset(&e, 0, sizeof e);
            e.n_slots = cu_sel[b + 1] - cu_sel[b];
            ne = write_stream(c, e, a->sel_ids + cu_sel[b], c->sel_len.data() + cu_sel[b], ne);
            most = std::max(most, e.n_entries);
        }
        c->plan_entries = ne;
        c->plan_items = 0;
        c->plan_splits = 1;
        c->plan_batch = B;
        c->plan_epoch = c->epoch;
        c->plan_list_pages = most;
        c->plan_tree = true;
        c->key_obj.clear();
        c->key_sel.assign(a->sel_ids, a->sel_ids + a->n_sel);
        c->key_cu.assign(cu_sel, cu_sel + B + 1);
        c->key_len = c->sel_len;
        std::fill(c->plan_layer_ok.begin(), c->plan_layer_ok.end(), 0);
        c->plan_layer_ok[a->layer] = 1;
        c->plan_valid = true;
        c->plan_on_device = false;
        c->plan_graph = 0;
    }
    if (!c->tree_ready) {
        if (prepare_tree(d.head_dim) != cudaSuccess) { cudaGetLastError(); return ENL_E_CUDA; }
        c->tree_ready = true;
    }

    TreeParams p;
    std::memset(&p, 0, sizeof p);
    {
        const int box_tokens = std::min(kTileRows / c->rep, a->n_max);
        const cuuint64_t qd[3] = {static_cast<cuuint64_t>(d.head_dim), static_cast<cuuint64_t>(d.n_q_heads), static_cast<cuuint64_t>(B) * a->n_max};
        const cuuint64_t qs[2] = {static_cast<cuuint64_t>(d.head_dim) * 2, static_cast<cuuint64_t>(d.head_dim) * 2 * d.n_q_heads};
        const cuuint32_t qb[3] = {64, static_cast<cuuint32_t>(c->rep), static_cast<cuuint32_t>(box_tokens)};
        const KeyMapShape km(d.head_dim, d.n_kv_heads, B * a->n_max);
        const PageMapShape pm(d.head_dim, d.n_kv_heads, a->n_pages);
        if (!c->maps.get(&p.tm_q, a->q, qd, qs, qb) || !c->maps.get(&p.tm_knew, a->k_new, km.dims, km.strides, km.box, 4) ||
            !c->maps.get(&p.tm_vnew, a->v_new, km.dims, km.strides, km.box, 4) || !c->maps.get(&p.tm_ktail, a->k_tail, pm.dims, pm.strides, pm.box, 4) ||
            !c->maps.get(&p.tm_vtail, a->v_tail, pm.dims, pm.strides, pm.box, 4))
            return ENL_E_CUDA;
        p.box_tokens = box_tokens;
    }
    p.tm_kpool = c->tm_k[a->layer];
    p.tm_vpool = c->tm_v[a->layer];
    p.ep0 = c->h_eps()[0];
    p.eps = reinterpret_cast<const EpInfo *>(c->plan_dev + c->off_eps);
    p.stream_page = reinterpret_cast<const int32_t *>(c->plan_dev + c->off_stream);
    p.stream_meta = reinterpret_cast<const int32_t *>(c->plan_dev + c->off_meta);
    p.block_table = a->block_table;
    p.tail_len = a->tail_len;
    p.n_new = a->n_new;
    p.mask = reinterpret_cast<const unsigned long long *>(a->mask);
    p.out = a->out;
    p.status = c->status_dev;
    p.batch = B;
    p.n_max = a->n_max;
    p.max_blocks = a->max_blocks;
    p.n_tail_pages = a->n_pages;
    p.Hq = d.n_q_heads;
    p.Hkv = d.n_kv_heads;
    p.rep = c->rep;
    p.min_steps = kMinSteps;
    p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(d.head_dim));

    // Two CTAs per multiprocessor run at once.  The device cuts the streams (it alone knows their lengths) into as many ranges as the grid has
    // CTAs: one wave where the units leave room for splits in it, else half a wave on top of a CTA per unit, so that long streams among
    // many are cut.
    const int wave = 2 * c->n_sm;
    const int64_t slot_bytes = static_cast<int64_t>(kTileRows) * (d.head_dim + 1) * 4;
    const int64_t head_bytes = (static_cast<int64_t>(B) * sizeof(int4) + 255) / 256 * 256;
    int64_t grid = units * 4 <= wave * 3ll ? wave : units + wave / 2;
    const int64_t longest = ceil_div(c->plan_list_pages + std::min(a->max_blocks, 0x3fffffff) + ceil_div(a->n_max, kPageTokens), kStepKeys / kPageTokens);
    p.may_split = longest > kMinSteps && d.scratch_bytes >= head_bytes + (units + 1) * slot_bytes;
    if (p.may_split) grid = std::min(grid, (d.scratch_bytes - head_bytes) / slot_bytes);
    else grid = units;
    if (p.may_split) {
        uint8_t *at = reinterpret_cast<uint8_t *>(c->scratch);
        p.part_head = reinterpret_cast<int4 *>(at);
        p.part_o = reinterpret_cast<float *>(at + head_bytes);
        p.part_lse = p.part_o + grid * kTileRows * d.head_dim;
    }
    if (join_loads(c, st, a->layer) != ENL_OK) return ENL_E_CUDA;
    const unsigned long long graph = capture_of(st);
    if (send_plan(c, graph, st) != ENL_OK) return ENL_E_CUDA;
    if (launch_tree(p, d.head_dim, static_cast<int>(grid), st) != cudaSuccess) { cudaGetLastError(); return ENL_E_CUDA; }
    c->settle(graph);                                       // the kernel waits for the one before, and lets the next one start after that
    if (p.may_split) {
        TreeMergeParams mp;
        mp.part_o = p.part_o;
        mp.part_lse = p.part_lse;
        mp.part_head = p.part_head;
        mp.out = a->out;
        mp.n_max = a->n_max;
        mp.Hq = d.n_q_heads;
        mp.Hkv = d.n_kv_heads;
        mp.rep = c->rep;
        mp.row_groups = ceil_div(a->n_max * c->rep, 32);
        if (launch_tree_merge(mp, d.head_dim, B, grid > 4 * units, st) != cudaSuccess) { cudaGetLastError(); return ENL_E_CUDA; }
    }
    return ENL_OK;
}
