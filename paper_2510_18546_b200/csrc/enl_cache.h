// The cache object, for the host files that work on it: the group tables, the pools, the current gather plan and what is known about
// work already enqueued.
#pragma once

#include <algorithm>
#include <vector>

#include "../../include/enl.h"
#include "enl_internal.h"

namespace enl {

struct Group {
    std::vector<int32_t> pages;       // shared by all layers: positions 16*i .. 16*i+15 live in pages[i]
    std::vector<int32_t> len;         // per layer, -1 = never stored
    // slow tier (Sec. 3.2): pages in the pinned host pool, and which copy is current
    std::vector<int32_t> host_pages;
    bool resident = true;             // the device pages hold the group
    bool host_current = false;        // the host pages hold what the device pages held when last written back
    uint64_t last_use = 0;            // tick of the last enl_step_prepare that selected the group
};

struct DeviceGuard {
    int prev = -1;
    bool switched = false;
    explicit DeviceGuard(int dev)
    {
        if (dev < 0) return;
        if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) {
            cudaSetDevice(dev);
            switched = true;
        }
    }
    ~DeviceGuard()
    {
        if (switched) cudaSetDevice(prev);
    }
};

inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// bf16 tensor map with 128-byte swizzle; dims/box innermost first, strides in bytes for dims 1..rank-1.
bool encode_map(CUtensorMap *tm, const void *base, int rank, const cuuint64_t *dims, const cuuint64_t *strides,
                const cuuint32_t *box);

// Tensor maps of the caller's tensors, kept by what they are made from: a planning step calls enl_attend once per layer with
// tensors that come back step after step, and encoding three maps per call is most of the host time of a call whose
// gather plan is reused.
// The key is all that a map is made from.
struct MapKey {
    const void *base;
    cuuint64_t dims[4], strides[3];
    cuuint32_t box[4];
    int rank;
    MapKey() : base(nullptr), dims{}, strides{}, box{}, rank(0) {}
    MapKey(const void *b, int r, const cuuint64_t *d, const cuuint64_t *s, const cuuint32_t *x) : MapKey()
    {
        base = b;
        rank = r;
        for (int i = 0; i < r; ++i) { dims[i] = d[i]; box[i] = x[i]; }
        for (int i = 0; i + 1 < r; ++i) strides[i] = s[i];
    }
    bool operator==(const MapKey &o) const
    {
        return base == o.base && rank == o.rank && std::equal(dims, dims + 4, o.dims) && std::equal(strides, strides + 3, o.strides) &&
               std::equal(box, box + 4, o.box);
    }
};
struct MapCache {
    static constexpr int kSlots = 256;
    MapKey key[kSlots];
    CUtensorMap map[kSlots];
    bool used[kSlots] = {};
    uint32_t turn = 0;
    // bf16 map [..][d2][d1][d0] of rank 3 or 4 with box {b0, b1, b2, ..}
    bool get(CUtensorMap *out, const void *base, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box, int rank = 3)
    {
        const MapKey k(base, rank, dims, strides, box);
        const size_t h = (reinterpret_cast<uintptr_t>(base) >> 8) * 0x9E3779B97F4A7C15ull >> 56;
        int victim = -1;                                    // the same tensor with another length (decoding), else a free slot
        for (int probe = 0; probe < 4; ++probe) {
            const int i = static_cast<int>((h + probe) % kSlots);
            if (used[i] && key[i] == k) { *out = map[i]; return true; }
            if (victim < 0 && (!used[i] || key[i].base == base)) victim = i;
        }
        if (!encode_map(out, base, rank, dims, strides, box)) return false;
        const int i = victim >= 0 ? victim : static_cast<int>((h + (turn++ & 3u)) % kSlots);
        key[i] = k;
        map[i] = *out;
        used[i] = true;
        return true;
    }
};

// a caller's [n][Hkv][D] keys or values, fetched by a few rows of a head
struct KeyMapShape {
    cuuint64_t dims[4], strides[3];
    cuuint32_t box[4];
    KeyMapShape(int D, int Hkv, int n)
        : dims{64, static_cast<cuuint64_t>(n), static_cast<cuuint64_t>(D / 64), static_cast<cuuint64_t>(Hkv)},
          strides{static_cast<cuuint64_t>(D) * 2 * Hkv, 128, static_cast<cuuint64_t>(D) * 2},
          box{64, static_cast<cuuint32_t>(box_rows(D)), static_cast<cuuint32_t>(D / 64), 1} {}
};

// What a plan of enl_attend_tree takes at most besides the streams: a segment per unit (request and kv head) and one more per CTA that runs at once.
inline size_t tree_plan_bytes(int64_t batch, int64_t n_kv_heads)
{
    const size_t units = static_cast<size_t>(batch * n_kv_heads);
    return (units + kTreeMaxPlaces) * (sizeof(TreeSegment) + sizeof(int32_t)) + units * sizeof(int2) + 256;
}

// pages of 16 rows, [n][Hkv][16][D]: a page of a head in one box
struct PageMapShape {
    cuuint64_t dims[4], strides[3];
    cuuint32_t box[4];
    PageMapShape(int D, int Hkv, int64_t n)
        : dims{64, static_cast<cuuint64_t>(box_rows(D)), static_cast<cuuint64_t>(D / 64), static_cast<cuuint64_t>(n) * Hkv * (kPageTokens / box_rows(D))},
          strides{static_cast<cuuint64_t>(D) * 2, 128, static_cast<cuuint64_t>(D) * 2 * box_rows(D)},
          box{64, static_cast<cuuint32_t>(box_rows(D)), static_cast<cuuint32_t>(D / 64), static_cast<cuuint32_t>(kPageTokens / box_rows(D))} {}
};

}  // namespace enl

struct enl_cache {
    using Group = enl::Group;
    using EpInfo = enl::EpInfo;
    using Item = enl::Item;
    using MapCache = enl::MapCache;
    using ClusterCaps = enl::ClusterCaps;
    enl_cache_desc_t d{};
    bool gpu = false;
    int rep = 1;
    int n_sm = 148;                         // multiprocessors of the device (grid sizes, split counts)
    int64_t n_pages = 0;
    size_t layer_bytes = 0;                 // one layer of one pool
    uint8_t *work = nullptr;                // the device allocation that holds all but the pools
    uint8_t *kpool = nullptr, *vpool = nullptr;
    std::vector<int32_t> free_pages;        // stack of free page ids (page 0 is never in it)
    std::vector<Group> groups;
    std::vector<CUtensorMap> tm_k, tm_v;    // per layer
    uint64_t epoch = 0;                     // bumped by every store

    // gather plan: host image (pinned when there is a GPU), device copy, capacities
    int32_t cap_entries = 0, cap_items = 0;
    uint8_t *plan_host = nullptr, *plan_dev = nullptr;
    // sections of the current plan, back to back in the order of their offsets
    size_t off_eps = 0, off_items = 0, off_stream = 0, off_meta = 0, off_rowslots = 0, off_rowobj = 0, off_chg = 0, plan_used = 0;
    size_t plan_bytes = 0;                  // capacity
    cudaEvent_t plan_copied = nullptr;
    bool plan_copying = false;              // a copy out of plan_host may be under way (until plan_copied)
    bool plan_valid = false, plan_on_device = false;
    std::vector<uint8_t> plan_layer_ok;     // layers whose group lengths have been compared with the plan's
    std::vector<int32_t> sel_len;           // working space of a call
    uint64_t plan_epoch = 0;
    int32_t plan_split_hint = 0;
    bool plan_has_mass = false;
    bool plan_mass_only = false, plan_sums = false;      // what the call wants besides or instead of outputs
    bool plan_park = false;                 // every CTA walks few slots: it parks their sums in shared memory and writes the masses itself
    bool plan_finish = false;               // else a kernel behind the attention kernel turns log-sums into masses
    std::vector<int32_t> key_obj;           // object spans the row -> object map was built from
    bool plan_tree = false;                 // the plan is for enl_attend_tree: streams, and the CTAs' shares where there are several requests
    int32_t tree_rows = 0, tree_blocks = 0, tree_entries = 0;      // ... for this n_max and max_blocks; cached pages of a single request
    std::vector<EpInfo> tree_eps;           // its episodes' streams (host only)
    int32_t tree_slots = 0;                 // partial results per tile of rows
    bool tree_ready = false;                // the kernel of enl_attend_tree has been opted in
    bool plan_decode = false;               // the plan is for the one-token decode kernel
    int32_t plan_small_blocks = 0;          // > 0: the plan is for the kernel of short calls, with this many row blocks per kv head
    int32_t plan_small_groups = 0;          // ... of this many times 16 rows
    int32_t plan_cluster = 0;               // decode: CTAs per cluster, 0 = the streaming kernel
    int32_t plan_list_pages = 0;            // decode by clusters: most pages one of the CTAs covers
    ClusterCaps cluster_caps = {};          // decode by clusters: how many run at once (none on a bookkeeping-only cache)
    // Order of launches, outside captures: a launch that writes the plan or the pool has been enqueued since the last attention
    // launch.  What a capture records runs when its graph does, so calls inside one go by what the same capture holds.
    bool written = true;
    unsigned long long settled_graph = 0;   // capture that holds an attention launch behind everything written so far
    unsigned long long plan_graph = 0;      // capture that holds the write of the current plan
    bool plan_in_graphs = false;            // some graph may write its plan over the one on the device at any time
    bool pool_in_graphs = false;            // some graph holds launches that write the pool: it may run before any call outside it
    bool plan_pair = false;                 // two splits whose CTAs merge inside the attention kernel (cluster of two)
    bool plan_halves = false;               // items of one Q tile whose steps the two halves of a CTA share
    bool pairs_ok = false;                  // the device can co-schedule two of the attention kernel's CTAs as a cluster
    std::vector<int32_t> key_sel, key_cu, key_len;   // what the current plan was built from
    int32_t plan_entries = 0, plan_items = 0, plan_splits = 1, plan_batch = 0, plan_max_slots = 0;
    MapCache maps;                          // tensor maps of the caller's q / k_new / v_new
    std::vector<int32_t> seen;              // duplicate detection stamps
    int32_t stamp = 0;

    // slow tier
    bool tier = false;
    int64_t n_host_pages = 0;
    size_t host_layer_bytes = 0;
    uint8_t *host_k = nullptr, *host_v = nullptr;           // pinned, [layer][page][kv head][16][D]
    std::vector<int32_t> free_host_pages;
    int2 *pairs_host = nullptr, *pairs_dev = nullptr;        // page moves of one enqueue (pinned staging + device copy)
    int32_t cap_pairs = 0;
    cudaEvent_t pairs_copied = nullptr;
    // loads of several megabytes run beside the caller's stream, a few layers at a time (see enqueue_loads)
    cudaStream_t load_stream[2] = {nullptr, nullptr};
    std::vector<cudaEvent_t> load_done;                     // per chunk of layers
    int load_chunks = 0, load_layers = 1;                   // chunks not known to be complete (0: none pending), layers of a chunk
    uint64_t tick = 0;

    float *scratch = nullptr;
    float *finish_lse = nullptr;            // rows' log-sum-exps for that kernel, and the splits' parts of shared slots
    float2 *finish_bnd = nullptr;
    int64_t finish_cap = 0;                 // entries of either
    int32_t *status_dev = nullptr;
    int32_t *counters_dev = nullptr;        // decode: finished splits per (episode, kv head)

    EpInfo *h_eps() { return reinterpret_cast<EpInfo *>(plan_host + off_eps); }
    Item *h_items() { return reinterpret_cast<Item *>(plan_host + off_items); }
    int32_t *h_stream() { return reinterpret_cast<int32_t *>(plan_host + off_stream); }
    int32_t *h_meta() { return reinterpret_cast<int32_t *>(plan_host + off_meta); }
    int32_t *h_rowslots() { return reinterpret_cast<int32_t *>(plan_host + off_rowslots); }
    uint8_t *h_chg() { return plan_host + off_chg; }
    // A launch that writes the pool is about to be enqueued (captured: a graph that does so is being made).
    void pool_written(bool captured)
    {
        written = true;
        settled_graph = 0;
        pool_in_graphs = pool_in_graphs || captured;
    }
    // An attention launch that leaves plan and pool behind as later ones may find them (see enl_attend) has been enqueued.
    void settle(unsigned long long graph)
    {
        if (graph) settled_graph = graph;
        else written = false;
    }
    int32_t *h_rowobj() { return reinterpret_cast<int32_t *>(plan_host + off_rowobj); }
};

namespace enl {

// The steps of a call that attends, shared by enl_attend and enl_attend_tree (in enl_host.cu).
// The capture that a stream is in, 0 = none.
unsigned long long capture_of(cudaStream_t st);
// Puts work of `st` that is about to be enqueued behind the loads that are still under way: those of one layer, or (-1) all.
int join_loads(enl_cache *c, cudaStream_t st, int layer);
// Checks a select list (ids, presence, duplicates within an episode) and leaves the groups' lengths in c->sel_len.
int look_over(enl_cache *c, int layer, int B, const int32_t *sel_ids, const int32_t *cu_sel);
// The plan is about to be rebuilt: waits until its host image may be written.
int open_plan(enl_cache *c);
// Writes the key stream of one episode (e.n_slots groups) from entry `ne` on; returns the entry behind it.
int32_t write_stream(enl_cache *c, EpInfo &e, const int32_t *ids, const int32_t *lens, int32_t ne);
// Sends the plan to the device unless what runs on `st` next finds it there.
int send_plan(enl_cache *c, unsigned long long graph, cudaStream_t st);

}  // namespace enl
