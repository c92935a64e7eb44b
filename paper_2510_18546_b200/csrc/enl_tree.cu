// Host side of enl_attend_tree: checks, the gather plan of the selected groups, the launch of the kernels in enl_tree_sm100.cu.
#include <cmath>
#include <cstring>

#include "enl_cache.h"

using namespace enl;

namespace {

// How many splits a request's stream of `pages` pages gets that may have `most`: the fewest that come to as few steps (of four pages) per CTA as
// `most` would, and none where that does not save what putting splits together costs, some four steps.
int splits_for(int64_t pages, int64_t most)
{
    constexpr int kStepPages = kStepKeys / kPageTokens, kMergeSteps = 4;
    auto steps_of = [&](int64_t ns) { return ((pages + ns - 1) / ns + kStepPages - 1) / kStepPages; };
    most = std::max<int64_t>(1, std::min(most, (pages + kStepPages - 1) / kStepPages));
    const int64_t steps = steps_of(most);
    if (steps_of(1) <= steps + kMergeSteps) return 1;
    return static_cast<int>((pages + steps * kStepPages - 1) / (steps * kStepPages));
}

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
    if (units > 0x3fffffff || (B > 1 && (B > 0x7fff || d.n_kv_heads > 0xffff))) return ENL_E_LIMIT;

    // ---- gather plan: the episodes' streams; reused when nothing it was built from has changed ----
    const size_t cu_bytes = sizeof(int32_t) * (B + 1);
    bool reuse = c->plan_valid && c->plan_tree && c->plan_epoch == c->epoch && c->plan_batch == B && c->tree_rows == a->n_max && c->tree_blocks == a->max_blocks &&
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
        if (n_entries > c->cap_entries || (B > 1 && units > c->cap_items)) return ENL_E_NOMEM;
        static_assert(sizeof(TreeItem) == sizeof(Item) && sizeof(int2) <= sizeof(EpInfo), "the plan buffers are made for these");

        // Splits.  The host does not know how long the tails are, so they count for what their tables hold: too many splits of a stream that
        // turns out short cost little, since all CTAs run at once.  Two of them fit a multiprocessor; every request gets splits until they fill
        // that many places (the longest streams first: ranges of as few pages as there are places for).
        std::vector<int32_t> &ns = c->tree_splits;
        ns.assign(B, 1);
        auto pages_of = [&](int b) {
            int64_t e = ceil_div(a->n_max, kPageTokens) + a->max_blocks;
            for (int s = cu_sel[b]; s < cu_sel[b + 1]; ++s) e += std::max(1, ceil_div(c->sel_len[s], kPageTokens));
            return e;
        };
        const int64_t per_request = static_cast<int64_t>(d.n_kv_heads) * row_tiles;
        const int64_t slot_bytes = static_cast<int64_t>(kTileRows) * (d.head_dim + 1) * 4;
        int64_t places = std::min<int64_t>(2 * c->n_sm, d.scratch_bytes / slot_bytes);
        places = std::min<int64_t>(places, std::min(c->cap_items, 0xfff));      // (splits are twelve bits of an item)
        if (units < places) {
            int64_t lo = 1, hi = 1;                        // pages of a split: the fewest for which all CTAs have a place
            for (int b = 0; b < B; ++b) hi = std::max(hi, pages_of(b));
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                int64_t n = 0;
                for (int b = 0; b < B; ++b) n += (pages_of(b) + mid - 1) / mid * per_request;
                if (n <= places) hi = mid; else lo = mid + 1;
            }
            for (int b = 0; b < B; ++b) ns[b] = splits_for(pages_of(b), (pages_of(b) + hi - 1) / hi);
        }
        int64_t n_items = 0;
        int most = 1;
        for (int b = 0; b < B; ++b) {
            n_items += ns[b] * per_request;
            most = std::max(most, ns[b]);
        }

        if (const int rc = open_plan(c)) return rc;
        size_t at = 0;
        auto section = [&](size_t bytes) { const size_t o = at; at += (bytes + 15) & ~static_cast<size_t>(15); return o; };
        c->off_items = section(B > 1 ? sizeof(TreeItem) * n_items : 0);
        c->off_eps = section(B > 1 ? sizeof(int2) * B : 0);
        c->off_stream = section(sizeof(int32_t) * n_entries);
        c->off_meta = section(sizeof(int32_t) * n_entries);
        c->plan_used = at;
        int32_t ne = 0;
        TreeItem *items = reinterpret_cast<TreeItem *>(c->plan_host + c->off_items);
        int2 *heads = reinterpret_cast<int2 *>(c->plan_host + c->off_eps);
        int32_t n_done = 0;
        for (int b = 0; b < B; ++b) {
            EpInfo e = {};
            e.n_slots = cu_sel[b + 1] - cu_sel[b];
            ne = write_stream(c, e, a->sel_ids + cu_sel[b], c->sel_len.data() + cu_sel[b], ne);
            c->tree_entries = e.n_entries;
            if (B == 1) break;
            heads[b] = make_int2(n_done, ns[b]);
            for (int h = 0; h < d.n_kv_heads; ++h)
                for (int s = 0; s < ns[b]; ++s) {
                    const int first = static_cast<int>(static_cast<int64_t>(e.n_entries) * s / ns[b]);
                    const int last = static_cast<int>(static_cast<int64_t>(e.n_entries) * (s + 1) / ns[b]);
                    for (int t = 0; t < row_tiles; ++t) items[n_done++] = TreeItem{b << 16 | h, t << 24 | s << 12 | ns[b], e.stream_off + first, last - first};
                }
        }
        c->plan_entries = ne;
        c->plan_items = static_cast<int32_t>(n_items);
        c->plan_splits = most;
        c->plan_batch = B;
        c->plan_epoch = c->epoch;
        c->plan_tree = true;
        c->tree_rows = a->n_max;
        c->tree_blocks = a->max_blocks;
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
    p.items = reinterpret_cast<const TreeItem *>(c->plan_dev + c->off_items);
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
    p.row_tiles = row_tiles;
    p.n_splits = c->plan_splits;
    p.n_entries = c->tree_entries;
    p.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(d.head_dim));

    p.part_o = c->scratch;
    p.part_lse = c->scratch + static_cast<int64_t>(c->plan_items) * kTileRows * d.head_dim;
    if (join_loads(c, st, a->layer) != ENL_OK) return ENL_E_CUDA;
    const unsigned long long graph = capture_of(st);
    if (send_plan(c, graph, st) != ENL_OK) return ENL_E_CUDA;
    p.wait_first = (graph ? c->settled_graph != graph : c->written || c->pool_in_graphs) ? 1 : 0;      // as in enl_attend
    if (launch_tree(p, d.head_dim, c->plan_items, st) != cudaSuccess) { cudaGetLastError(); return ENL_E_CUDA; }
    c->settle(graph);
    if (c->plan_splits > 1) {
        TreeMergeParams mp;
        mp.part_o = p.part_o;
        mp.part_lse = p.part_lse;
        mp.heads = B > 1 ? reinterpret_cast<const int2 *>(c->plan_dev + c->off_eps) : nullptr;
        mp.tail_len = p.tail_len;
        mp.n_new = p.n_new;
        mp.out = a->out;
        mp.n_splits = c->plan_splits;
        mp.n_max = a->n_max;
        mp.Hq = d.n_q_heads;
        mp.Hkv = d.n_kv_heads;
        mp.rep = c->rep;
        mp.row_tiles = row_tiles;
        mp.row_groups = ceil_div(a->n_max * c->rep, 32);
        if (launch_tree_merge(mp, d.head_dim, B, c->plan_splits > 4, st) != cudaSuccess) { cudaGetLastError(); return ENL_E_CUDA; }
    }
    return ENL_OK;
}
