// Attention of drafted trees (and of single tokens) over selected groups and a request's growing tail, sm_100a (tcgen05 + TMEM + TMA).
//
// For node i of request b, q head h:  out = softmax(q K^T / sqrt(D)) V  over the rows of the request's selected groups (pool pages, as the
// gather plan lists them), the first tail_len[b] rows of its tail (pages that its block table names), and those nodes j of its tree
// whose bit is set in mask[b][i].  Lengths, block tables and masks are read on the device: a captured call runs on as the tail grows.
//
// A CTA takes 128 query rows (128 / rep nodes x the rep q heads of one kv head) and a range of the key stream, in steps of 64 keys =
// four pages, each fetched by a TMA box from wherever it lies; per step
//   S = Q K^T               tcgen05.mma into one of two TMEM buffers of 64 columns
//   p = exp2(S * c - m)     one thread per row, hidden keys -inf before the maximum
//   O += P V                tcgen05.mma, P (bf16) out of the TMEM columns that held the scores
// Roles (7 warps): 0-3 softmax, 4 fetches K, 5 fetches V, 6 issues the MMAs and owns the TMEM.  Softmax warps without rows do nothing.
//
// What bounds it: a tree has few rows, so the keys' bytes do (64 keys of a kv head are 32 KB, which take a multiprocessor some 1400 cycles
// of its share of the memory; the tensor pipe needs 512 of them and the special-function units 512).  Hence two CTAs per
// multiprocessor, whose chains scores -> softmax -> P V overlap, and ranges of keys (splits) that fill the device whatever the batch:
// the device itself cuts the streams, since only it knows their lengths.  Splits leave outputs normalised by their own sums, and
// log2-sum-exps, in the scratch buffer; tree_merge_kernel puts them together.
#include <cuda_bf16.h>

#include "attn_ops.cuh"
#include "enl_internal.h"
#include "tmem_ops.cuh"

namespace enl {
namespace {

constexpr int kSoftmaxWarps = 4;
constexpr int kKWarp   = 4;
constexpr int kVWarp   = 5;
constexpr int kMmaWarp = 6;
constexpr int kThreads = 7 * 32;
constexpr uint32_t kTmemCols = 256;           // two CTAs per multiprocessor
constexpr uint32_t kOCol = 128;               // S: [0, 64) and [64, 128), O: [128, 128 + D)
constexpr int kStepPages = kStepKeys / kPageTokens;
constexpr float kRescaleThreshold = 8.0f;     // log2 units: p stays below 2^8 between updates of the reference

template <int D>
struct Cfg {
    static constexpr int kBlocks     = D / 64;                // 64-channel (128-byte) column blocks
    static constexpr int kBlockBytes = 128 * 128;             // Q tile: 128 rows x 128 B
    static constexpr int kTileBytes  = kBlocks * kBlockBytes;
    static constexpr int kGroupBytes = kBlocks * 1024;        // eight rows of K or V
    static constexpr int kStepBytes  = kStepKeys / 8 * kGroupBytes;
    static constexpr int kRing       = D == 128 ? 2 : 4;      // steps whose K (and whose V) are in shared memory at once
    static constexpr int kRingOff    = kTileBytes;
    static constexpr int kBarOff     = kRingOff + 2 * kRing * kStepBytes;
    static constexpr int kSmemBytes  = kBarOff + 384 + 1024;  // + alignment slack
    static_assert(kSmemBytes <= 115712, "two CTAs per multiprocessor");
};

// What a CTA does: rows of one request and kv head, a range of steps.
struct Share {
    int b, kvh, rt;                           // request, kv head, tile of 128 rows
    int n_splits;                             // 0: nothing to do
    int j_beg, j_end;                         // steps
    int n_entries, stream_off;                // pages of the selected groups, and the first of them in the plan
    int len, n;                               // rows of the tail, nodes of the tree
};

struct Request {
    int n_entries, stream_off, len, n, steps, tiles;
};
__device__ __forceinline__ int tail_pages_of(int len) { return (len + kPageTokens - 1) / kPageTokens; }

// A request as the device finds it: a length below zero (or no nodes) leaves nothing to do; a tail is as long as its block table at most.
__device__ __forceinline__ Request request_of(const TreeParams &p, int b)
{
    Request r = {0, 0, 0, 0, 0, 0};
    if (b >= p.batch) return r;
    if (p.batch == 1) {
        r.n_entries = p.ep0.n_entries;
        r.stream_off = p.ep0.stream_off;
    } else {
        r.n_entries = __ldcg(&p.eps[b].n_entries);
        r.stream_off = __ldcg(&p.eps[b].stream_off);
    }
    const int len = __ldcg(p.tail_len + b), n = p.n_new ? __ldcg(p.n_new + b) : p.n_max;
    r.len = max(0, min(len, p.max_blocks * kPageTokens));
    r.n = len < 0 ? 0 : max(0, min(n, p.n_max));
    if (r.n > 0) {
        r.steps = (r.n_entries + tail_pages_of(r.len) + tail_pages_of(r.n) + kStepPages - 1) / kStepPages;
        r.tiles = (r.n * p.rep + kTileRows - 1) / kTileRows;
    }
    return r;
}

// Range s of ns of the steps.
__device__ __forceinline__ void cut(Share &out, int steps, int s, int ns)
{
    const int each = steps / ns, more = steps - each * ns;
    out.j_beg = each * s + min(s, more);
    out.j_end = out.j_beg + each + (s < more ? 1 : 0);
    out.n_splits = ns;
}
// The streams of all requests, kv heads and row tiles ("units") are cut into ranges of about `chunk` steps, as few steps as the grid has CTAs for.
// CTA order: request, kv head, split, row tile (the tiles of a unit read the same keys at the same time).  Every warp works it out for itself, so
// that none waits for another (by one warp, with 64-bit arithmetic and a barrier behind it, 2.1 us of a launch, 3.7 for 16 requests).  With `heads`
// the warp leaves what the merge kernel has to know: per request the first CTA, its splits, row tiles and nodes.
__device__ __forceinline__ Share find_share(const TreeParams &p, int lane, bool heads)
{
    const int grid = static_cast<int>(gridDim.x), idx = static_cast<int>(blockIdx.x);
    const Request r = request_of(p, p.batch == 1 ? 0 : lane);
    Share out = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    if (p.batch == 1) {
        if (r.n == 0) {
            if (heads && lane == 0) p.part_head[0] = make_int4(0, 0, 0, 0);
            return out;
        }
        const int units = r.tiles * p.Hkv;
        const int ns = p.may_split ? max(1, min(grid / units, r.steps / p.min_steps)) : 1;
        if (heads && lane == 0) p.part_head[0] = make_int4(0, ns, r.tiles, r.n);
        if (idx >= units * ns) return out;
        const int above = idx / r.tiles;
        out.kvh = above / ns;
        out.rt = idx - above * r.tiles;
        cut(out, r.steps, above - out.kvh * ns, ns);
        out.n_entries = r.n_entries;
        out.stream_off = r.stream_off;
        out.len = r.len;
        out.n = r.n;
        return out;
    }
    float work = 0.f;
    int units = 0, longest = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const Request q = b0 ? request_of(p, b0 + lane) : r;
        work += static_cast<float>(q.tiles * p.Hkv) * static_cast<float>(q.steps);
        units += q.tiles * p.Hkv;
        longest = max(longest, q.steps);
    }
    for (int o = 16; o > 0; o >>= 1) work += __shfl_xor_sync(kFull, work, o);
    units = __reduce_add_sync(kFull, units);
    longest = __reduce_max_sync(kFull, longest);
    // One over the steps of a range; every warp of the launch comes to the same one, and to the same number of splits of a request by it.
    auto splits_of = [](int steps, float inv) { return static_cast<int>(ceilf(static_cast<float>(steps) * inv)); };
    float chunk = static_cast<float>(max(longest, 1));
    const float floor_steps = static_cast<float>(p.min_steps);
    if (p.may_split && units < grid && longest > p.min_steps) {
        // enough for certain: sum of ceil(steps / chunk) <= work / chunk + units (and a little for the rounding of the quotients)
        const float sure = fminf(chunk, fmaxf(work * 1.001f / static_cast<float>(grid - units), floor_steps));
        if (p.batch <= 32) {
            // the shortest of 32 lengths that the grid has CTAs for, a lane each
            const float least = fminf(sure, fmaxf(work / static_cast<float>(grid), floor_steps));
            const float mine = least + (sure - least) * (static_cast<float>(lane) / 31.f), inv = 1.f / mine;
            int ctas = 0;
            for (int b = 0; b < p.batch; ++b)
                ctas += splits_of(__shfl_sync(kFull, r.steps, b), inv) * __shfl_sync(kFull, r.tiles, b);
            const unsigned fit = __ballot_sync(kFull, ctas * p.Hkv <= grid);
            chunk = __shfl_sync(kFull, lane == 31 ? sure : mine, fit ? __ffs(fit) - 1 : 31);
        } else {
            chunk = sure;
        }
    }
    const float inv = 1.f / chunk;
    int first = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const Request q = b0 ? request_of(p, b0 + lane) : r;
        const int ns = q.tiles ? max(1, splits_of(q.steps, inv)) : 0, mine = ns * q.tiles * p.Hkv;
        int upto = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(kFull, upto, o);
            if (lane >= o) upto += t;
        }
        const int before = first + upto - mine;
        if (heads && b0 + lane < p.batch) p.part_head[b0 + lane] = make_int4(before, ns, q.tiles, q.n);
        const unsigned who = __ballot_sync(kFull, idx >= before && idx < before + mine);
        first += __shfl_sync(kFull, upto, 31);
        if (!who) continue;
        const int from = __ffs(who) - 1;
        const int local = idx - __shfl_sync(kFull, before, from), n_s = __shfl_sync(kFull, ns, from), tiles = __shfl_sync(kFull, q.tiles, from);
        const int above = local / tiles;
        out.b = b0 + from;
        out.kvh = above / n_s;
        out.rt = local - above * tiles;
        cut(out, __shfl_sync(kFull, q.steps, from), above - out.kvh * n_s, n_s);
        out.n_entries = __shfl_sync(kFull, q.n_entries, from);
        out.stream_off = __shfl_sync(kFull, q.stream_off, from);
        out.len = __shfl_sync(kFull, q.len, from);
        out.n = __shfl_sync(kFull, q.n, from);
        if (!heads) break;
    }
    return out;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2) tree_kernel(const __grid_constant__ TreeParams p)
{
    using C = Cfg<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t sbase = (raw + 1023u) & ~1023u;               // 1024-B aligned (swizzle atoms)
    uint8_t *smem = smem_raw + (sbase - raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    auto k_addr = [&](int x) { return sbase + static_cast<uint32_t>(C::kRingOff + 2 * x * C::kStepBytes); };
    auto v_addr = [&](int x) { return k_addr(x) + static_cast<uint32_t>(C::kStepBytes); };
    const uint32_t bar0 = sbase + C::kBarOff;
    const uint32_t bar_q_full = bar0, bar_pv_done = bar0 + 8u, bar_o_done = bar0 + 16u;      // P V of a step, of the last one
    auto bar_s_full  = [&](int b) { return bar0 + 8u * (3 + b); };              // b: step & 1
    auto bar_p_full  = [&](int b) { return bar0 + 8u * (5 + b); };
    auto bar_k_full  = [&](int x) { return bar0 + 8u * (7 + x); };              // x: place in the ring
    auto bar_k_empty = [&](int x) { return bar0 + 8u * (7 + C::kRing + x); };
    auto bar_v_full  = [&](int x) { return bar0 + 8u * (7 + 2 * C::kRing + x); };
    auto bar_v_empty = [&](int x) { return bar0 + 8u * (7 + 3 * C::kRing + x); };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::kBarOff + 8 * (7 + 4 * C::kRing));
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    static_assert(8 * (7 + 4 * C::kRing) + 8 <= 384, "shared memory");

    // ---- set-up ----
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        mbar_init(bar_q_full, 1);
        mbar_init(bar_pv_done, 1);
        mbar_init(bar_o_done, 1);
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar_s_full(b), 1);
            mbar_init(bar_p_full(b), kSoftmaxWarps);              // (the first warp arrives for those without rows, too)
        }
        for (int x = 0; x < C::kRing; ++x) {
            mbar_init(bar_k_full(x), 1);
            mbar_init(bar_k_empty(x), 1);
            mbar_init(bar_v_full(x), 1);
            mbar_init(bar_v_empty(x), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if ((warp == kKWarp || warp == kVWarp) && lane < 4) {
        const CUtensorMap *tm = warp == kKWarp ? (lane == 0 ? &p.tm_kpool : lane == 1 ? &p.tm_ktail : lane == 2 ? &p.tm_knew : &p.tm_q)
                                               : (lane == 0 ? &p.tm_vpool : lane == 1 ? &p.tm_vtail : &p.tm_vnew);
        asm volatile("prefetch.tensormap [%0];" ::"l"(tm) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    // Everything that says what to do (plan, lengths, block tables) may come from the kernel before.  The next one may start only after
    // this wait: attention launches rely on it (see enl_attend).
    pdl_wait();
    pdl_trigger();
    const Share w = find_share(p, lane, p.part_head && blockIdx.x == 0 && warp == kMmaWarp);
    const int n_steps = w.n_splits > 0 ? w.j_end - w.j_beg : 0;     // at least one where there is anything to do
    const int tail_pages = tail_pages_of(w.len);
    bool ok = true;

    if (n_steps > 0 && (warp == kKWarp || warp == kVWarp)) {
        // ================= TMA producers =================
        const bool is_k = warp == kKWarp;
        const CUtensorMap *tm_pool = is_k ? &p.tm_kpool : &p.tm_vpool, *tm_tail = is_k ? &p.tm_ktail : &p.tm_vtail,
                          *tm_new = is_k ? &p.tm_knew : &p.tm_vnew;
        const uint32_t ring = is_k ? k_addr(0) : v_addr(0), full0 = is_k ? bar_k_full(0) : bar_v_full(0),
                       empty0 = is_k ? bar_k_empty(0) : bar_v_empty(0);
        // Where 32 pages lie, one per lane, fetched eight steps ahead: kind << 30 | page of the pool (0), of the tail (1), first row among the
        // request's nodes (2).  What fills the last step, and an entry of the block table that names no page, is the page of zeros.
        constexpr int kBatch = 32 / kStepPages;
        auto where = [&](int j) -> uint32_t {
            int g = j * kStepPages + lane;
            if (g < w.n_entries) return static_cast<uint32_t>(__ldcg(p.stream_page + w.stream_off + g));
            g -= w.n_entries;
            if (g < tail_pages) {
                const int id = __ldcg(p.block_table + static_cast<long long>(w.b) * p.max_blocks + g);
                return id >= 0 && id < p.n_tail_pages ? (1u << 30) | static_cast<uint32_t>(id) : static_cast<uint32_t>(kZeroPage);
            }
            g = (g - tail_pages) * kPageTokens;
            return g < w.n ? (2u << 30) | static_cast<uint32_t>(g) : static_cast<uint32_t>(kZeroPage);
        };
        if (is_k && lane == 0) {
            mbar_expect_tx(bar_q_full, static_cast<uint32_t>(C::kBlocks * p.box_tokens * p.rep * 128));
            for (int b = 0; b < C::kBlocks; ++b)
                tma_load_3d(sbase + b * C::kBlockBytes, &p.tm_q, b * 64, w.kvh * p.rep, w.b * p.n_max + w.rt * (kTileRows / p.rep), bar_q_full);
        }
        __syncwarp();
        uint32_t cur = 0, next = where(w.j_beg);
        int fetched = 0;
        for (int jj = 0; jj < n_steps; ++jj) {
            const int x = jj % C::kRing;
            if (jj % kBatch == 0) {
                cur = next;
                next = where(w.j_beg + jj + kBatch);
            }
            const uint32_t at = __shfl_sync(kFull, cur, jj % kBatch * kStepPages + lane % kStepPages);
            if (jj >= C::kRing) ok = mbar_wait(empty0 + 8u * x, static_cast<uint32_t>((jj / C::kRing - 1) & 1), abort_flag, p.status);
            if (!ok) break;
            const uint32_t full = full0 + 8u * x;
            if (lane == 0) mbar_expect_tx(full, static_cast<uint32_t>(C::kStepBytes));
            __syncwarp();
            if (lane < kStepPages) {
                const uint32_t dst = ring + static_cast<uint32_t>(2 * x * C::kStepBytes + lane * 2 * C::kGroupBytes);
                const int id = static_cast<int>(at & 0x3fffffffu);
                if (at >> 30 == 2u) {
#pragma unroll
                    for (int y = 0; y < kPageGroups<D>; ++y)
                        tma_load_4d(dst + static_cast<uint32_t>(y * (kBoxRows<D> * D * 2)), tm_new, 0, w.b * p.n_max + id + y * kBoxRows<D>, 0, w.kvh, full);
                } else {
                    tma_load_4d(dst, at >> 30 == 1u ? tm_tail : tm_pool, 0, 0, 0, (id * p.Hkv + w.kvh) * kPageGroups<D>, full);
                }
            }
            ++fetched;
        }
        // error path only: let the copies already in flight land before the CTA retires
        if (!ok) {
            for (int f = max(0, fetched - C::kRing); f < fetched; ++f) {
                const unsigned long long t0 = global_ns();
                while (!mbar_try_wait(full0 + 8u * (f % C::kRing), static_cast<uint32_t>((f / C::kRing) & 1)) &&
                       global_ns() - t0 < 2000000ull) { }
            }
        }
    } else if (n_steps > 0 && warp == kMmaWarp) {
        // ================= MMA issuer =================
        constexpr uint32_t idesc_qk = make_idesc(kStepKeys, false), idesc_pv = make_idesc(D, true);
        constexpr uint32_t kStepUnits = C::kStepBytes >> 4, kGroupUnits = C::kGroupBytes >> 4;
        const uint64_t dq0 = smem_desc(sbase, 16), dk0 = smem_desc(k_addr(0), 16, C::kGroupBytes), dv0 = smem_desc(v_addr(0), 1024, C::kGroupBytes);
        const uint32_t dq_lo = static_cast<uint32_t>(dq0), dq_hi = static_cast<uint32_t>(dq0 >> 32);
        const uint32_t dk_lo = static_cast<uint32_t>(dk0), dk_hi = static_cast<uint32_t>(dk0 >> 32);
        const uint32_t dv_lo = static_cast<uint32_t>(dv0), dv_hi = static_cast<uint32_t>(dv0 >> 32);
        // A commit that frees a place of the ring is made only where a later fetch waits for it: nothing may arrive after the CTA has retired.
        auto issue_qk = [&](int jj) {
            const int x = jj % C::kRing, b = jj & 1;
            const uint32_t ka = dk_lo + static_cast<uint32_t>(x) * (2u * kStepUnits), d = tmem_base + static_cast<uint32_t>(b * kStepKeys);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t in_row = static_cast<uint32_t>((kk & 3) * 2);                       // 32 bytes per 16 channels
                mma_ss2(d, dq_lo + static_cast<uint32_t>((kk >> 2) * (C::kBlockBytes >> 4)) + in_row, dq_hi,
                        ka + static_cast<uint32_t>((kk >> 2) * (1024 >> 4)) + in_row, dk_hi, idesc_qk, kk > 0 ? 1u : 0u);
            }
            tc_commit(bar_s_full(b));
            if (jj + C::kRing < n_steps) tc_commit(bar_k_empty(x));
        };
        // O (+)= P V; P of keys 2c, 2c + 1 sits in column c of the buffer that held their scores
        auto issue_pv = [&](int jj) {
            const int x = jj % C::kRing, b = jj & 1;
            const uint32_t va = dv_lo + static_cast<uint32_t>(x) * (2u * kStepUnits), a = tmem_base + static_cast<uint32_t>(b * kStepKeys);
#pragma unroll
            for (int k4 = 0; k4 < kStepPages; ++k4)                  // 16 keys = two groups of 8 rows, 8 columns of P
                mma_ts2(tmem_base + kOCol, a + static_cast<uint32_t>(k4 * 8), va + static_cast<uint32_t>(k4 * 2) * kGroupUnits, dv_hi, idesc_pv,
                        (jj == 0 && k4 == 0) ? 0u : 1u);
            if (jj + C::kRing < n_steps) tc_commit(bar_v_empty(x));
            tc_commit(jj + 1 < n_steps ? bar_pv_done : bar_o_done);
        };
        auto wait_k = [&](int jj) { return mbar_wait(bar_k_full(jj % C::kRing), static_cast<uint32_t>((jj / C::kRing) & 1), abort_flag, p.status); };
        ok = mbar_wait(bar_q_full, 0, abort_flag, p.status);
        for (int jj = 0; jj < min(2, n_steps) && ok; ++jj) {
            ok = wait_k(jj);
            if (!ok) break;
            tc_fence_after();
            issue_qk(jj);
        }
        for (int jj = 0; jj < n_steps && ok; ++jj) {
            const bool more = jj + 2 < n_steps;
            ok = mbar_wait(bar_v_full(jj % C::kRing), static_cast<uint32_t>((jj / C::kRing) & 1), abort_flag, p.status);
            if (ok && more) ok = wait_k(jj + 2);
            if (ok) ok = mbar_wait(bar_p_full(jj & 1), static_cast<uint32_t>((jj >> 1) & 1), abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();
            issue_pv(jj);
            if (more) issue_qk(jj + 2);
        }
        if (ok) ok = mbar_wait(bar_o_done, 0, abort_flag, p.status);
    } else if (n_steps > 0 && warp < kSoftmaxWarps && w.rt * kTileRows + warp * 32 < w.n * p.rep) {
        // ================= softmax: one thread per query row =================
        const int rep = p.rep, lr = 31 - __clz(rep);
        const int r = warp * 32 + lane, n_act = (min(kTileRows, w.n * rep - w.rt * kTileRows) + 31) >> 5;      // softmax warps with rows
        const int t = w.rt * (kTileRows >> lr) + (r >> lr);           // node
        const bool row_valid = t < w.n;
        const uint32_t lane_sel = static_cast<uint32_t>(warp * 32) << 16;
        const uint32_t t_s = tmem_base + lane_sel, t_o = tmem_base + lane_sel + kOCol;
        const float scale = p.scale_log2;
        // nodes that this one sees; without masks the nodes are a chain
        unsigned long long tree = 0;
        if (row_valid) {
            tree = p.mask ? __ldcg(p.mask + static_cast<long long>(w.b) * p.n_max + t) : (2ull << t) - 1ull;
            if (w.n < 64) tree &= (1ull << w.n) - 1ull;
        }
        // Keys of 32 pages, one page per lane, fetched eight steps ahead: how many of the page's rows count, or 256 | first node of a page of nodes.
        constexpr int kBatch = 32 / kStepPages;
        auto load_meta = [&](int j) -> int {
            int g = j * kStepPages + lane;
            if (g < w.n_entries) return __ldcg(p.stream_meta + w.stream_off + g) & 0xff;
            g -= w.n_entries;
            if (g < tail_pages) return min(kPageTokens, w.len - g * kPageTokens);
            g = (g - tail_pages) * kPageTokens;
            return g < w.n ? 256 | g : 0;
        };
        int meta = 0, meta_next = load_meta(w.j_beg);
        float m = kNegInf, l = 0.f;                                   // reference (log2 units), row sum
        for (int jj = 0; jj < n_steps; ++jj) {
            const int b = jj & 1;
            if (jj % kBatch == 0) {
                meta = meta_next;
                meta_next = load_meta(w.j_beg + jj + kBatch);
            }
            int pg[kStepPages];
            bool whole = true;
#pragma unroll
            for (int e = 0; e < kStepPages; ++e) {
                pg[e] = __shfl_sync(kFull, meta, jj % kBatch * kStepPages + e);
                whole = whole && pg[e] == kPageTokens;
            }
            const uint32_t t_sb = t_s + static_cast<uint32_t>(b * kStepKeys);
            ok = mbar_wait(bar_s_full(b), static_cast<uint32_t>((jj >> 1) & 1), abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();

            // the row's 64 scores
            uint32_t su[kStepKeys];
#pragma unroll
            for (int k = 0; k < kStepKeys / 32; ++k)
                tmem_ld32_issue(t_sb + static_cast<uint32_t>(k * 32), reinterpret_cast<uint32_t(&)[32]>(su[k * 32]));
            tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < kStepKeys / 32; ++k) tmem_ld32_arrived(reinterpret_cast<uint32_t(&)[32]>(su[k * 32]));
            float s[kStepKeys];
#pragma unroll
            for (int x = 0; x < kStepKeys; ++x) s[x] = __uint_as_float(su[x]);

            // Hide what does not count: rows behind the end of a page's, and nodes that are no ancestors.  By a select, not by adding -inf: keys
            // that nobody sees may hold anything.
            if (!whole) {
#pragma unroll
                for (int e = 0; e < kStepPages; ++e) {
                    const uint32_t see = pg[e] & 256 ? static_cast<uint32_t>(tree >> (pg[e] & 63)) : (1u << pg[e]) - 1u;
#pragma unroll
                    for (int x = 0; x < kPageTokens; ++x)
                        if (!((see >> x) & 1u)) s[e * kPageTokens + x] = kNegInf;
                }
            }

            // row maximum: four independent chains
            float mx4[kStepPages];
#pragma unroll
            for (int k = 0; k < kStepPages; ++k) {
                float a = fmax3(s[k * 16], s[k * 16 + 1], s[k * 16 + 2]);
#pragma unroll
                for (int x = 3; x < 15; x += 2) a = fmax3(a, s[k * 16 + x], s[k * 16 + x + 1]);
                mx4[k] = fmaxf(a, s[k * 16 + 15]);
            }
            const float m_cand = fmaxf(fmax3(mx4[0], mx4[1], mx4[2]), mx4[3]) * scale;

            // The reference moves only when the row maximum has grown by more than the threshold; then sum and accumulator are
            // rescaled, behind P V of the step before (the one before that was done when these scores were).
            // (Rows of the tile that are no nodes hold whatever lay in shared memory: they must not move the others' references, or results
            // would differ in their last bits from run to run.)
            const bool need = row_valid && m_cand > m + kRescaleThreshold;       // also true when m == -inf < m_cand
            if (__any_sync(kFull, need)) {
                const float m_new = fmaxf(m, m_cand);
                const float alpha = (m_new == kNegInf) ? 1.f : ex2(m - m_new);
                l *= alpha;
                m = m_new;
                if (jj > 0) {
                    ok = mbar_wait(bar_pv_done, static_cast<uint32_t>((jj - 1) & 1), abort_flag, p.status);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int k = 0; k < D / 32; ++k) {
                        uint32_t o[32];
                        tmem_ld32_wait(t_o + static_cast<uint32_t>(k * 32), o);
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
                        tmem_st32(t_o + static_cast<uint32_t>(k * 32), o);
                    }
                }
            }
            const float m_use = (m == kNegInf) ? 0.f : m;

            // p = exp2(s * scale - m), summed in fp32 and rounded to bf16 for the tensor cores (as every kernel of the library does)
            const uint64_t sc2 = pack2(scale, scale), nm2 = pack2(-m_use, -m_use);
            uint64_t ps2[2];
#pragma unroll
            for (int ch = 0; ch < kStepKeys / 32; ++ch) {
                uint32_t pk[16];
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    float a0, a1;
                    unpack2(fma2(pack2(s[ch * 32 + 2 * x], s[ch * 32 + 2 * x + 1]), sc2, nm2), a0, a1);
                    a0 = ex2(a0);
                    a1 = ex2(a1);
                    const uint64_t p2 = pack2(a0, a1);
                    pk[x] = pack_bf16(a0, a1);
                    ps2[ch] = x ? add2(ps2[ch], p2) : p2;
                }
                tmem_st16(t_sb + static_cast<uint32_t>(ch * 16), pk);
            }
            // V rows that no row of the tile sees are cleared: 0 times whatever lies there must stay 0.  Those of the tail's last page and
            // behind the last node (pool pages are zero behind a group's end).
            if (!whole && warp == 0) {
                const int x = jj % C::kRing;
                bool waited = false;
#pragma unroll
                for (int e = 0; e < kStepPages; ++e) {
                    const int g = (w.j_beg + jj) * kStepPages + e - w.n_entries;
                    const int rows = pg[e] & 256 ? min(kPageTokens, w.n - (pg[e] & 63)) : pg[e];
                    if (g < 0 || rows == 0 || rows == kPageTokens) continue;
                    if (!waited) ok = mbar_wait(bar_v_full(x), static_cast<uint32_t>((jj / C::kRing) & 1), abort_flag, p.status);
                    waited = true;
                    if (!ok) break;
                    uint8_t *page = smem + C::kRingOff + (2 * x + 1) * C::kStepBytes + e * 2 * C::kGroupBytes;
                    for (int i = lane; i < (kPageTokens - rows) * C::kBlocks * 8; i += 32) {    // 16-byte pieces
                        const int row = rows + i / (C::kBlocks * 8), blk = i / 8 % C::kBlocks;
                        *reinterpret_cast<uint4 *>(page + (row >> 3) * C::kGroupBytes + blk * 1024 + (row & 7) * 128 + i % 8 * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                }
                if (!ok) break;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_n(bar_p_full(b), warp == 0 ? static_cast<uint32_t>(kSoftmaxWarps + 1 - n_act) : 1u);
            float lo0, hi0, lo1, hi1;
            unpack2(ps2[0], lo0, hi0);
            unpack2(ps2[1], lo1, hi1);
            l += (lo0 + hi0) + (lo1 + hi1);
        }
        if (ok) ok = mbar_wait(bar_o_done, 0, abort_flag, p.status);
        if (ok) {
            tc_fence_after();
            const float inv = l > 0.f ? 1.f / l : 0.f;
            const bool split = w.n_splits > 1;
            if (split) p.part_lse[static_cast<long long>(blockIdx.x) * kTileRows + r] = l > 0.f ? m + lg2(l) : kNegInf;
            // partial outputs [CTA][D / 4][row][4]: a warp's store is one contiguous piece
            float4 *part = reinterpret_cast<float4 *>(p.part_o) + static_cast<long long>(blockIdx.x) * (D / 4) * kTileRows + r;
            uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) +
                         ((static_cast<long long>(w.b) * p.n_max + t) * p.Hq + w.kvh * rep + (r & (rep - 1))) * D);
#pragma unroll 1
            for (int k = 0; k < D / 32; ++k) {
                uint32_t o[32];
                tmem_ld32_wait(t_o + static_cast<uint32_t>(k * 32), o);
                float f[32];
#pragma unroll
                for (int x = 0; x < 32; ++x) f[x] = l > 0.f ? __uint_as_float(o[x]) * inv : 0.f;      // a row that sees nothing: 0
                if (split) {
#pragma unroll
                    for (int x = 0; x < 8; ++x) part[(k * 8 + x) * kTileRows] = make_float4(f[4 * x], f[4 * x + 1], f[4 * x + 2], f[4 * x + 3]);
                } else if (row_valid) {
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        dst[k * 4 + x] = make_uint4(pack_bf16(f[8 * x], f[8 * x + 1]), pack_bf16(f[8 * x + 2], f[8 * x + 3]),
                                                    pack_bf16(f[8 * x + 4], f[8 * x + 5]), pack_bf16(f[8 * x + 6], f[8 * x + 7]));
                }
            }
        }
    }

    // ---- teardown ----
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
    }
}

// Puts the splits of a row together: out = sum_s 2^(lse_s - M) o_s / sum_s 2^(lse_s - M), in the order of the splits.  A CTA takes 32 rows of a
// unit, a lane each; grid.x runs over units and groups of 32 rows, grid.y over channels.  Few registers and little shared memory: its
// CTAs find a place beside those of the attention kernel and wait there for its end (with 512 threads of 64 registers they started
// after it: 4.7 us behind it for one token of 8 kv heads, ...).
//   kDeep: four channels a CTA; its warps take every fourth split, six of them at a time, and are added up in shared memory
//   else (calls with many units, whose streams have few splits): sixteen channels a CTA, four a warp, which takes all splits
constexpr int kMergeWarps = 4;
template <int D, bool kDeep>
__global__ void __launch_bounds__(kMergeWarps * 32, 8) tree_merge_kernel(const __grid_constant__ TreeMergeParams p)
{
    __shared__ float4 sums[kMergeWarps][32];
    __shared__ float2 refs[kMergeWarps][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int lr = 31 - __clz(p.rep);
    const int row_groups = p.row_groups, b = static_cast<int>(blockIdx.x) / (p.Hkv * row_groups), at = static_cast<int>(blockIdx.x) - b * (p.Hkv * row_groups);
    const int kvh = at / row_groups, rows0 = (at - kvh * row_groups) * 32, tile = rows0 / kTileRows;
    const int quad = kDeep ? static_cast<int>(blockIdx.y) : static_cast<int>(blockIdx.y) * kMergeWarps + warp;
    pdl_trigger();
    pdl_wait();                                             // the partial results come from the previous kernel
    const int4 head = __ldcg(p.part_head + b);              // first CTA, splits, row tiles, nodes
    const int row = rows0 + lane;
    if (head.y < 2 || rows0 >= head.w << lr) return;
    const bool on = row < head.w << lr;
    const int r = row % kTileRows;
    const long long cta0 = head.x + static_cast<long long>(kvh) * head.y * head.z + tile;
    constexpr int kAhead = kDeep ? 6 : 4, kEvery = kDeep ? kMergeWarps : 1;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = kNegInf, l = 0.f;
    for (int s0 = kDeep ? warp : 0; s0 < head.y && on; s0 += kAhead * kEvery) {
        float lse[kAhead];
        float4 x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int s = s0 + u * kEvery;
            lse[u] = kNegInf;
            if (s < head.y) {
                const long long cta = cta0 + static_cast<long long>(s) * head.z;
                lse[u] = __ldcg(p.part_lse + cta * kTileRows + r);
                x[u] = __ldcg(reinterpret_cast<const float4 *>(p.part_o) + (cta * (D / 4) + quad) * kTileRows + r);
            }
        }
        float m_new = m;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) m_new = fmaxf(m_new, lse[u]);
        if (m_new == kNegInf) continue;                     // splits that saw no key
        const float alpha = ex2(m - m_new);
        l *= alpha;
        acc.x *= alpha; acc.y *= alpha; acc.z *= alpha; acc.w *= alpha;
        m = m_new;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (lse[u] == kNegInf) continue;
            const float f = ex2(lse[u] - m);
            l += f;
            acc.x = fmaf(f, x[u].x, acc.x); acc.y = fmaf(f, x[u].y, acc.y);
            acc.z = fmaf(f, x[u].z, acc.z); acc.w = fmaf(f, x[u].w, acc.w);
        }
    }
    if (kDeep) {
        sums[warp][lane] = acc;
        refs[warp][lane] = make_float2(m, l);
        __syncthreads();
        if (warp != 0) return;
        float top = kNegInf;
#pragma unroll
        for (int g = 0; g < kMergeWarps; ++g) top = fmaxf(top, refs[g][lane].x);
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
        l = 0.f;
#pragma unroll
        for (int g = 0; g < kMergeWarps; ++g) {
            const float2 ml = refs[g][lane];
            if (ml.x == kNegInf) continue;
            const float f = ex2(ml.x - top);
            const float4 x = sums[g][lane];
            l = fmaf(f, ml.y, l);
            acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
        }
    }
    if (!on) return;
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint2 *dst = reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.out) +
                 ((static_cast<long long>(b) * p.n_max + (row >> lr)) * p.Hq + kvh * p.rep + (row & (p.rep - 1))) * D + quad * 4);
    *dst = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
}

}  // namespace

cudaError_t prepare_tree(int head_dim)
{
    if (head_dim == 128) return cudaFuncSetAttribute(tree_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<128>::kSmemBytes);
    if (head_dim == 64) return cudaFuncSetAttribute(tree_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<64>::kSmemBytes);
    return cudaErrorInvalidValue;
}

cudaError_t launch_tree(const TreeParams &p, int head_dim, int grid, cudaStream_t st)
{
    cudaError_t e;
    if (head_dim == 128) e = launch_pdl(tree_kernel<128>, dim3(grid), dim3(kThreads), Cfg<128>::kSmemBytes, st, p);
    else if (head_dim == 64) e = launch_pdl(tree_kernel<64>, dim3(grid), dim3(kThreads), Cfg<64>::kSmemBytes, st, p);
    else return cudaErrorInvalidValue;
    return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_tree_merge(const TreeMergeParams &p, int head_dim, int batch, bool deep, cudaStream_t st)
{
    if (head_dim != 128 && head_dim != 64) return cudaErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(batch) * p.Hkv * p.row_groups, deep ? head_dim / 4 : head_dim / (4 * kMergeWarps)), block(kMergeWarps * 32);
    const auto kernel = head_dim == 128 ? (deep ? tree_merge_kernel<128, true> : tree_merge_kernel<128, false>)
                                        : (deep ? tree_merge_kernel<64, true> : tree_merge_kernel<64, false>);
    const cudaError_t e = launch_pdl(kernel, grid, block, 0, st, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace enl
