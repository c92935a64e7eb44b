// Attention of drafted trees (and of single tokens) over selected groups and a request's growing tail, sm_100a (tcgen05 + TMEM + TMA).
//
// For node i of request b, q head h:  out = softmax(q K^T / sqrt(D)) V  over the rows of the request's selected groups (pool pages, as the
// gather plan lists them), the first tail_len[b] rows of its tail (pages that its block table names), and those nodes j of its tree
// whose bit is set in mask[b][i].  Lengths, block tables and masks are read on the device: a captured call runs on as the tail grows.
//
// A CTA takes up to 128 query rows (nodes x the rep q heads of one kv head) and a share of the keys, in steps of 64 keys =
// four pages, each fetched by a TMA box from wherever it lies; per step
//   S = Q K^T               tcgen05.mma into one of two TMEM buffers of 64 columns
//   p = exp2(S * c - m)     one thread per row, hidden keys -inf before the maximum
//   O += P V                tcgen05.mma, P (bf16) out of the TMEM columns that held the scores
// Roles: a softmax warp per 32 rows, a warp that fetches K, one that fetches V, one that issues the MMAs and owns the TMEM.
//
// What bounds it: a tree has few rows, so the keys' bytes do (64 keys of a kv head are 32 KB, which take a multiprocessor some 1400 cycles
// of its share of the memory; the tensor pipe needs 512 of them and the special-function units 512).  Hence two CTAs per
// multiprocessor, whose chains scores -> softmax -> P V overlap, and splits that fill the device whatever the batch.
//
// Shares: the host knows the cached pages of a request, but not how long its tail is.  So it cuts the stream of a request and kv head (a "unit")
// by fractions: the part from a / E to b / E takes those pages of the C cached ones and the same part of the tail's and the nodes' pages, whose
// number the device finds.  A CTA has one part, or, where the units do not divide into equal parts (see enl_tree.cu), a run of parts of
// consecutive units that is as long as any other CTA's; the loads of a part run under the one before it.  The cached pages of the first steps are fetched before the
// kernel waits for the one before it (plan and pool are written by the library only).
// Parts of a unit leave outputs normalised by their own sums, and log2-sum-exps, in the scratch buffer; tree_merge_kernel puts them together.
#include <cuda_bf16.h>

#include "attn_ops.cuh"
#include "enl_internal.h"
#include "tmem_ops.cuh"

namespace enl {
namespace {

constexpr uint32_t kTmemCols = 256;           // two CTAs per multiprocessor
constexpr uint32_t kOCol = 128;               // S: [0, 64) and [64, 128), O: [128, 128 + D)
constexpr int kStepPages = kStepKeys / kPageTokens;
constexpr int kBatch = 32 / kStepPages;       // steps whose pages a warp's lanes hold, one each
constexpr float kRescaleThreshold = 8.0f;     // log2 units: p stays below 2^8 between updates of the reference

// kRows: 64 or 128 query rows.  The Q tile of 64 rows is half of what the MMA reads: the other rows of its operand are whatever lies behind it
// (the next block of channels, the ring), and their results are not looked at.  The 16 KB go to the ring.
template <int D, int kRows>
struct Cfg {
    static constexpr int kSoftmaxWarps = kRows / 32, kKWarp = kSoftmaxWarps, kVWarp = kKWarp + 1, kMmaWarp = kKWarp + 2;
    static constexpr int kThreads    = (kSoftmaxWarps + 3) * 32;
    static constexpr int kBlocks     = D / 64;                // 64-channel (128-byte) column blocks
    static constexpr int kBlockBytes = kRows * 128;           // of the Q tile
    static constexpr int kTileBytes  = kBlocks * kBlockBytes;
    static constexpr int kGroupBytes = kBlocks * 1024;        // eight rows of K or V
    static constexpr int kStepBytes  = kStepKeys / 8 * kGroupBytes;
    // steps whose K, and whose V, are in shared memory at once: all that two CTAs have room for (V stays until its step's softmax is done)
    static constexpr int kRingK      = D == 64 ? 6 : kRows == 64 ? 3 : 2;
    static constexpr int kRingV      = D == 64 ? 6 : 3;
    static constexpr int kKOff       = kTileBytes;
    static constexpr int kVOff       = kKOff + kRingK * kStepBytes;
    static constexpr int kBarOff     = kVOff + kRingV * kStepBytes;
    static constexpr int kBars       = 9 + 2 * (kRingK + kRingV);
    static constexpr int kSmemBytes  = kBarOff + 8 * kBars + 8;
    static_assert(kSmemBytes <= 115712, "two CTAs per multiprocessor");
};

__device__ __forceinline__ int pages_of(int rows) { return (rows + kPageTokens - 1) / kPageTokens; }

template <int D, int kRows>
__global__ void __launch_bounds__((kRows / 32 + 3) * 32, 2) tree_kernel(const __grid_constant__ TreeParams p)
{
    using C = Cfg<D, kRows>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sbase = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    const uint32_t bar0 = sbase + C::kBarOff;
    const uint32_t bar_q_full = bar0, bar_q_empty = bar0 + 8u;                   // the Q tile of a segment is there / may be overwritten
    const uint32_t bar_pv_done = bar0 + 16u, bar_o_done = bar0 + 24u;           // P V of a step / of a segment's last one
    const uint32_t bar_o_free = bar0 + 32u;                                     // the accumulator has been read
    auto bar_s_full  = [&](int b) { return bar0 + 8u * (5 + b); };              // b: step & 1
    auto bar_p_full  = [&](int b) { return bar0 + 8u * (7 + b); };
    auto bar_k_full  = [&](int x) { return bar0 + 8u * (9 + x); };              // x: place in the ring
    auto bar_k_empty = [&](int x) { return bar0 + 8u * (9 + C::kRingK + x); };
    auto bar_v_full  = [&](int x) { return bar0 + 8u * (9 + 2 * C::kRingK + x); };
    auto bar_v_empty = [&](int x) { return bar0 + 8u * (9 + 2 * C::kRingK + C::kRingV + x); };
    auto phase_of = [](int at, int places) { return static_cast<uint32_t>((at / places) & 1); };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::kBarOff + 8 * C::kBars);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    if (sbase & 1023u) {                      // (swizzled tiles need it, and dynamic shared memory starts like this)
        if (threadIdx.x == 0) atomicExch(p.status, 1);
        return;
    }
    if (p.wait_first) pdl_wait();
    // ---- what this CTA does: a tile of rows of its segments (see TreeSegment) ----
    const int group = p.row_tiles == 1 ? static_cast<int>(blockIdx.x) : static_cast<int>(blockIdx.x) / p.row_tiles;
    const int rt = p.row_tiles == 1 ? 0 : static_cast<int>(blockIdx.x) - group * p.row_tiles;
    struct Part { int b, kvh, slot, first, count, from, to, whole; };
    auto segment = [&](int i) -> Part {
        Part w;
        if (p.batch == 1) {
            w.b = 0;
            w.kvh = group / p.n_splits;
            w.from = group - w.kvh * p.n_splits;
            w.to = w.from + 1;
            w.whole = p.n_splits;
            w.slot = p.n_splits > 1 ? group : -1;
            w.first = static_cast<int>(static_cast<long long>(p.n_entries) * w.from / p.n_splits);
            w.count = static_cast<int>(static_cast<long long>(p.n_entries) * w.to / p.n_splits) - w.first;
        } else {
            const int4 *src = reinterpret_cast<const int4 *>(p.segments + i);
            const int4 x = __ldcg(src), y = __ldcg(src + 1);
            w.b = x.x >> 16; w.kvh = x.x & 0xffff; w.slot = x.y; w.first = x.z; w.count = x.w;
            w.from = y.x; w.to = y.y; w.whole = y.z;
        }
        return w;
    };
    int seg_beg = 0, seg_end = 1;
    if (p.batch > 1) {
        seg_beg = __ldcg(p.segment_off + group);
        seg_end = __ldcg(p.segment_off + group + 1);
    }
    Part it = segment(seg_beg);

    // ---- set-up ----
    if (warp == C::kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        mbar_init(bar_q_full, 1);
        mbar_init(bar_q_empty, 1);
        mbar_init(bar_o_free, C::kSoftmaxWarps);                  // (with rows or without)
        mbar_init(bar_pv_done, 1);
        mbar_init(bar_o_done, 1);
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar_s_full(b), 1);
            mbar_init(bar_p_full(b), C::kSoftmaxWarps);           // (the first warp arrives for those without rows, too)
        }
        for (int x = 0; x < C::kRingK; ++x) { mbar_init(bar_k_full(x), 1); mbar_init(bar_k_empty(x), 1); }
        for (int x = 0; x < C::kRingV; ++x) { mbar_init(bar_v_full(x), 1); mbar_init(bar_v_empty(x), 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_trigger();
    bool ok = true;

    // ---- lengths: a request that has ended, or has no nodes, leaves nothing to do; a tail is as long as its block table at most.  What comes from
    // the kernel before is read past the L1, since this one may have started while that one ran. ----
    int len = 0, n = 0, t_first = 0, t_count = 0, tail_pages = 0, n_steps = 0;
    auto read_lengths = [&]() {
        const int l0 = __ldcg(p.tail_len + it.b), n0 = p.n_new ? __ldcg(p.n_new + it.b) : p.n_max;
        len = max(0, min(l0, p.max_blocks * kPageTokens));
        n = l0 < 0 ? 0 : max(0, min(n0, p.n_max));
        tail_pages = pages_of(len);
        const int t = tail_pages + pages_of(n);
        // (rising in `at`, 0 at 0 and t at the end: the parts of a unit meet)
        auto cut = [&](int at) { return at >= it.whole ? t : min(t, static_cast<int>(static_cast<float>(t) * (static_cast<float>(at) / static_cast<float>(it.whole)))); };
        t_first = cut(it.from);
        t_count = cut(it.to) - t_first;
        n_steps = rt * kRows < n * p.rep ? (it.count + t_count + kStepPages - 1) / kStepPages : 0;
    };
    // The steps of cached pages alone that the ring has room for are fetched before the wait for the kernel before.  A first segment that turns
    // out to have no rows leaves them, and its Q tile, to be passed over.
    const int early_k = p.wait_first ? 0 : min(C::kRingK, it.count / kStepPages), early_v = p.wait_first ? 0 : min(C::kRingV, it.count / kStepPages);

    if (warp == C::kKWarp || warp == C::kVWarp) {
        // ================= TMA producers =================
        const bool is_k = warp == C::kKWarp;
        const CUtensorMap *tm_pool = is_k ? &p.tm_kpool : &p.tm_vpool, *tm_tail = is_k ? &p.tm_ktail : &p.tm_vtail,
                          *tm_new = is_k ? &p.tm_knew : &p.tm_vnew;
        const uint32_t ring = sbase + static_cast<uint32_t>(is_k ? C::kKOff : C::kVOff), full0 = is_k ? bar_k_full(0) : bar_v_full(0),
                       empty0 = is_k ? bar_k_empty(0) : bar_v_empty(0);
        const int places = is_k ? C::kRingK : C::kRingV, early = is_k ? early_k : early_v;
        // Where pages lie, one per lane, fetched eight steps ahead: kind << 30 | page of the pool (0), of the tail (1), first row among the
        // request's nodes (2).  What fills the last step, and an entry of the block table that names no page, is the page of zeros.
        auto where = [&](int i) -> uint32_t {
            if (i < it.count) return static_cast<uint32_t>(__ldcg(p.stream_page + it.first + i));
            const int g = i - it.count + t_first;
            if (i >= it.count + t_count) return static_cast<uint32_t>(kZeroPage);
            if (g < tail_pages) {
                const int id = __ldcg(p.block_table + static_cast<long long>(it.b) * p.max_blocks + g);
                return id >= 0 && id < p.n_tail_pages ? (1u << 30) | static_cast<uint32_t>(id) : static_cast<uint32_t>(kZeroPage);
            }
            return (2u << 30) | static_cast<uint32_t>((g - tail_pages) * kPageTokens);
        };
        auto fetch = [&](uint32_t at, int x) {                       // `at`: the page of lanes 0 .. 3
            const uint32_t full = full0 + 8u * x;
            if (lane == 0) mbar_expect_tx(full, static_cast<uint32_t>(C::kStepBytes));
            __syncwarp();
            if (lane < kStepPages) {
                const uint32_t dst = ring + static_cast<uint32_t>(x * C::kStepBytes + lane * 2 * C::kGroupBytes);
                const int id = static_cast<int>(at & 0x3fffffffu);
                if (at >> 30 == 2u) {
#pragma unroll
                    for (int y = 0; y < kPageGroups<D>; ++y)
                        tma_load_4d(dst + static_cast<uint32_t>(y * (kBoxRows<D> * D * 2)), tm_new, 0, it.b * p.n_max + id + y * kBoxRows<D>, 0, it.kvh, full);
                } else {
                    tma_load_4d(dst, at >> 30 == 1u ? tm_tail : tm_pool, 0, 0, 0, (id * p.Hkv + it.kvh) * kPageGroups<D>, full);
                }
            }
        };
        auto fetch_q = [&]() {
            if (is_k && lane == 0) {
                mbar_expect_tx(bar_q_full, static_cast<uint32_t>(C::kBlocks * p.box_tokens * p.rep * 128));
                for (int b = 0; b < C::kBlocks; ++b)
                    tma_load_3d(sbase + b * C::kBlockBytes, &p.tm_q, b * 64, it.kvh * p.rep, it.b * p.n_max + rt * (kRows / p.rep), bar_q_full);
            }
            __syncwarp();
        };
        static_assert(C::kRingK < kBatch && C::kRingV < kBatch, "the early steps' pages are of one batch");
        uint32_t cur = 0, next = where(lane);                        // (of the cached pages so far)
        int f = 0, qn = 1;                                           // steps fetched, Q tiles fetched
        for (; f < early; ++f) fetch(__shfl_sync(kFull, next, f * kStepPages + lane % kStepPages), f);
        pdl_wait();
        fetch_q();
        read_lengths();
        for (int si = seg_beg; ok;) {
            int jj = si == seg_beg && n_steps > 0 ? early : 0;
            if (si > seg_beg) {
                next = where(lane);
                if (is_k && n_steps > 0) {
                    ok = mbar_wait(bar_q_empty, static_cast<uint32_t>((qn - 1) & 1), abort_flag, p.status);
                    if (!ok) break;
                    fetch_q();
                    ++qn;
                }
            } else if (lane >= it.count) {
                next = where(lane);
            }
            cur = next;
            if (jj > 0) next = where(kBatch * kStepPages + lane);
            for (; jj < n_steps; ++jj) {
                const int x = f % places;
                if (jj % kBatch == 0) {
                    cur = next;
                    next = where((jj + kBatch) * kStepPages + lane);
                }
                const uint32_t at = __shfl_sync(kFull, cur, jj % kBatch * kStepPages + lane % kStepPages);
                if (f >= places) ok = mbar_wait(empty0 + 8u * x, phase_of(f, places) ^ 1u, abort_flag, p.status);
                if (!ok) break;
                fetch(at, x);
                ++f;
            }
            if (++si >= seg_end) break;
            it = segment(si);
            read_lengths();
        }
        // error path only: copies in flight land before the CTA retires
        if (!ok) {
            for (int e = max(0, f - places); e < f; ++e) {
                const unsigned long long t0 = global_ns();
                while (!mbar_try_wait(full0 + 8u * (e % places), phase_of(e, places)) && global_ns() - t0 < 2000000ull) { }
            }
        }
    } else if (warp == C::kMmaWarp) {
        // ================= MMA issuer =================
        pdl_wait();
        read_lengths();
        constexpr uint32_t idesc_qk = make_idesc(kStepKeys, false), idesc_pv = make_idesc(D, true);
        constexpr uint32_t kStepUnits = C::kStepBytes >> 4, kGroupUnits = C::kGroupBytes >> 4;
        const uint64_t dq0 = smem_desc(sbase, 16), dk0 = smem_desc(sbase + C::kKOff, 16, C::kGroupBytes), dv0 = smem_desc(sbase + C::kVOff, 1024, C::kGroupBytes);
        const uint32_t dq_lo = static_cast<uint32_t>(dq0), dq_hi = static_cast<uint32_t>(dq0 >> 32);
        const uint32_t dk_lo = static_cast<uint32_t>(dk0), dk_hi = static_cast<uint32_t>(dk0 >> 32);
        const uint32_t dv_lo = static_cast<uint32_t>(dv0), dv_hi = static_cast<uint32_t>(dv0 >> 32);
        int fk = 0, fv = 0, g = 0, qn = 0, on = 0;                  // steps whose K, whose V has been used, steps, Q tiles and accumulators so far
        auto issue_qk = [&](int at, bool last) {                     // step `at` of all
            const int x = fk % C::kRingK, b = at & 1;
            const uint32_t ka = dk_lo + static_cast<uint32_t>(x) * kStepUnits, d = tmem_base + static_cast<uint32_t>(b * kStepKeys);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t in_row = static_cast<uint32_t>((kk & 3) * 2);                       // 32 bytes per 16 channels
                mma_ss2(d, dq_lo + static_cast<uint32_t>((kk >> 2) * (C::kBlockBytes >> 4)) + in_row, dq_hi,
                        ka + static_cast<uint32_t>((kk >> 2) * (1024 >> 4)) + in_row, dk_hi, idesc_qk, kk > 0 ? 1u : 0u);
            }
            tc_commit(bar_s_full(b));
            tc_commit(bar_k_empty(x));
            if (last) tc_commit(bar_q_empty);
            ++fk;
        };
        // O (+)= P V; P of keys 2c, 2c + 1 sits in column c of the buffer that held their scores
        auto issue_pv = [&](bool first, bool last) {
            const int x = fv % C::kRingV, b = g & 1;
            const uint32_t va = dv_lo + static_cast<uint32_t>(x) * kStepUnits, a = tmem_base + static_cast<uint32_t>(b * kStepKeys);
#pragma unroll
            for (int k4 = 0; k4 < kStepPages; ++k4)                  // 16 keys = two groups of 8 rows, 8 columns of P
                mma_ts2(tmem_base + kOCol, a + static_cast<uint32_t>(k4 * 8), va + static_cast<uint32_t>(k4 * 2) * kGroupUnits, dv_hi, idesc_pv,
                        (first && k4 == 0) ? 0u : 1u);
            tc_commit(bar_v_empty(x));
            tc_commit(last ? bar_o_done : bar_pv_done);
            ++fv;
        };
        auto wait_k = [&]() { return mbar_wait(bar_k_full(fk % C::kRingK), phase_of(fk, C::kRingK), abort_flag, p.status); };
        auto wait_v = [&]() { return mbar_wait(bar_v_full(fv % C::kRingV), phase_of(fv, C::kRingV), abort_flag, p.status); };
        for (int si = seg_beg; ok;) {
            if (si == seg_beg || n_steps > 0) {
                ok = mbar_wait(bar_q_full, static_cast<uint32_t>(qn & 1), abort_flag, p.status);
                ++qn;
            }
            if (n_steps == 0 && si == seg_beg) {                     // what was fetched for nothing
                for (int e = 0; e < early_k && ok; ++e, ++fk) {
                    ok = wait_k();
                    if (lane == 0) mbar_arrive(bar_k_empty(fk % C::kRingK));
                }
                for (int e = 0; e < early_v && ok; ++e, ++fv) {
                    ok = wait_v();
                    if (lane == 0) mbar_arrive(bar_v_empty(fv % C::kRingV));
                }
                if (lane == 0) mbar_arrive(bar_q_empty);
            }
            for (int jj = 0; jj < min(2, n_steps) && ok; ++jj) {
                ok = wait_k();
                if (!ok) break;
                tc_fence_after();
                issue_qk(g + jj, jj + 1 == n_steps);
            }
            for (int jj = 0; jj < n_steps && ok; ++jj, ++g) {
                const bool more = jj + 2 < n_steps;
                ok = wait_v();
                if (ok && more) ok = wait_k();
                if (ok && jj == 0 && on > 0) ok = mbar_wait(bar_o_free, static_cast<uint32_t>((on - 1) & 1), abort_flag, p.status);
                if (ok) ok = mbar_wait(bar_p_full(g & 1), static_cast<uint32_t>((g >> 1) & 1), abort_flag, p.status);
                if (!ok) break;
                tc_fence_after();
                issue_pv(jj == 0, jj + 1 == n_steps);
                if (more) issue_qk(g + 2, jj + 3 == n_steps);
            }
            if (n_steps > 0) ++on;
            if (++si >= seg_end) break;
            it = segment(si);
            read_lengths();
        }
        // nothing may arrive after the CTA has retired
        for (int e = max(0, fk - C::kRingK); e < fk && ok; ++e) ok = mbar_wait(bar_k_empty(e % C::kRingK), phase_of(e, C::kRingK), abort_flag, p.status);
        for (int e = max(0, fv - C::kRingV); e < fv && ok; ++e) ok = mbar_wait(bar_v_empty(e % C::kRingV), phase_of(e, C::kRingV), abort_flag, p.status);
        if (ok) ok = mbar_wait(bar_q_empty, static_cast<uint32_t>((qn - 1) & 1), abort_flag, p.status);
        if (ok && on > 0) ok = mbar_wait(bar_o_done, static_cast<uint32_t>((on - 1) & 1), abort_flag, p.status);
    } else {
        // ================= softmax: one thread per query row =================
        const int rep = p.rep, lr = 31 - __clz(rep);
        const int r = warp * 32 + lane;
        const int t = rt * (kRows >> lr) + (r >> lr);                 // node
        const uint32_t lane_sel = static_cast<uint32_t>(warp * 32) << 16;
        const uint32_t t_s = tmem_base + lane_sel, t_o = tmem_base + lane_sel + kOCol;
        const float scale = p.scale_log2;
        int g0 = 0, fv0 = 0, on = 0;                                  // steps, steps whose V was fetched, accumulators of the segments before
        pdl_wait();
        read_lengths();
        for (int si = seg_beg; ok;) {
            if (n_steps == 0 && si == seg_beg) fv0 = early_v;
            if (rt * kRows + warp * 32 < n * rep) {
                const int n_act = (min(kRows, n * rep - rt * kRows) + 31) >> 5;      // softmax warps with rows
                const uint32_t arrivals = warp == 0 ? static_cast<uint32_t>(C::kSoftmaxWarps + 1 - n_act) : 1u;
                const bool row_valid = t < n;
                // nodes that this one sees; without masks the nodes are a chain
                unsigned long long tree = 0;
                if (row_valid) {
                    tree = p.mask ? __ldcg(p.mask + static_cast<long long>(it.b) * p.n_max + t) : (2ull << t) - 1ull;
                    if (n < 64) tree &= (1ull << n) - 1ull;
                }
                // Keys of 32 pages, one page per lane, fetched eight steps ahead: how many of the page's rows count, or 256 | first node of a page of nodes.
                auto load_meta = [&](int i) -> int {
                    if (i < it.count) return __ldcg(p.stream_meta + it.first + i) & 0xff;
                    const int g = i - it.count + t_first;
                    if (i >= it.count + t_count) return 0;
                    return g < tail_pages ? min(kPageTokens, len - g * kPageTokens) : 256 | (g - tail_pages) * kPageTokens;
                };
                int meta = 0, meta_next = load_meta(lane);
                float m = kNegInf, l = 0.f;                                   // reference (log2 units), row sum
                for (int jj = 0; jj < n_steps; ++jj) {
                    const int g = g0 + jj, b = g & 1;
                    if (jj % kBatch == 0) {
                        meta = meta_next;
                        meta_next = load_meta((jj + kBatch) * kStepPages + lane);
                    }
                    int pg[kStepPages];
                    bool whole = true;
#pragma unroll
                    for (int e = 0; e < kStepPages; ++e) {
                        pg[e] = __shfl_sync(kFull, meta, jj % kBatch * kStepPages + e);
                        whole = whole && pg[e] == kPageTokens;
                    }
                    const uint32_t t_sb = t_s + static_cast<uint32_t>(b * kStepKeys);
                    ok = mbar_wait(bar_s_full(b), static_cast<uint32_t>((g >> 1) & 1), abort_flag, p.status);
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
                    // rescaled, behind P V of the step before (the one before that was done when these scores were; the last of a segment counts elsewhere).
                    // (Rows of the tile that are no nodes hold whatever lay in shared memory: they must not move the others' references, or results
                    // would differ in their last bits from run to run.)
                    const bool need = row_valid && m_cand > m + kRescaleThreshold;       // also true when m == -inf < m_cand
                    if (__any_sync(kFull, need)) {
                        const float m_new = fmaxf(m, m_cand);
                        const float alpha = (m_new == kNegInf) ? 1.f : ex2(m - m_new);
                        l *= alpha;
                        m = m_new;
                        if (jj > 0) {
                            ok = mbar_wait(bar_pv_done, static_cast<uint32_t>((g - on - 1) & 1), abort_flag, p.status);
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
                        const int fv = fv0 + g, x = fv % C::kRingV;
                        bool waited = false;
#pragma unroll
                        for (int e = 0; e < kStepPages; ++e) {
                            const int rows = pg[e] & 256 ? min(kPageTokens, n - (pg[e] & 63)) : pg[e];
                            if (jj * kStepPages + e < it.count || rows == 0 || rows == kPageTokens) continue;
                            if (!waited) ok = mbar_wait(bar_v_full(x), phase_of(fv, C::kRingV), abort_flag, p.status);
                            waited = true;
                            if (!ok) break;
                            uint8_t *page = smem + C::kVOff + x * C::kStepBytes + e * 2 * C::kGroupBytes;
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
                    if (lane == 0) mbar_arrive_n(bar_p_full(b), arrivals);
                    float lo0, hi0, lo1, hi1;
                    unpack2(ps2[0], lo0, hi0);
                    unpack2(ps2[1], lo1, hi1);
                    l += (lo0 + hi0) + (lo1 + hi1);
                }
                if (n_steps == 0) {                                           // a part without a step: the rows have seen nothing of it
                    if (it.slot >= 0) p.part_lse[(static_cast<long long>(it.slot) * p.row_tiles + rt) * kTileRows + r] = kNegInf;
                } else if (ok && (ok = mbar_wait(bar_o_done, static_cast<uint32_t>(on & 1), abort_flag, p.status))) {
                    tc_fence_after();
                    const float inv = l > 0.f ? 1.f / l : 0.f;
                    const bool split = it.slot >= 0;
                    const long long slot = static_cast<long long>(it.slot) * p.row_tiles + rt;
                    if (split) p.part_lse[slot * kTileRows + r] = l > 0.f ? m + lg2(l) : kNegInf;
                    // partial outputs [slot][D / 4][row][4]: a warp's store is one contiguous piece
                    float4 *part = reinterpret_cast<float4 *>(p.part_o) + slot * (D / 4) * kTileRows + r;
                    uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) +
                                 ((static_cast<long long>(it.b) * p.n_max + t) * p.Hq + it.kvh * rep + (r & (rep - 1))) * D);
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
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_o_free);
                }
            } else if (n_steps > 0) {
                // A warp without rows in this segment may have some in the next.  It keeps step with the others: ahead of them it would take phases
                // before for those that it waits for, and arrive where the first warp has arrived for it; two segments behind it would wait for good.
                ok = mbar_wait(bar_o_done, static_cast<uint32_t>(on & 1), abort_flag, p.status);
                if (ok && lane == 0) mbar_arrive(bar_o_free);
            }
            if (n_steps > 0) ++on;
            g0 += n_steps;
            if (++si >= seg_end) break;
            it = segment(si);
            read_lengths();
        }
    }

    // ---- teardown ----
    tc_fence_before();
    __syncthreads();
    if (warp == C::kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
    }
}

// Puts the parts of a unit together: out = sum_s 2^(lse_s - M) o_s / sum_s 2^(lse_s - M).  A warp takes four channels of 32 / kLanes rows; kLanes
// lanes share a row and take every kLanes-th part, up to kAhead at a time, all of whose loads are on their way at once.  No shared memory and few
// registers, so that its CTAs find a place beside those of the attention kernel and wait there for its end; nor does a load wait for
// another (a row that turns out to be none has read what lay in the scratch buffer).  grid.x: units and groups of rows, grid.y: channels.
constexpr int kMergeWarps = 4;
template <int D, int kLanes, int kAhead>
__global__ void __launch_bounds__(kMergeWarps * 32, 8) tree_merge_kernel(const __grid_constant__ TreeMergeParams p)
{
    constexpr int kWarpRows = 32 / kLanes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, of = lane / kWarpRows;
    const int lr = 31 - __clz(p.rep);
    const int unit = static_cast<int>(blockIdx.x) / p.row_groups, quad = static_cast<int>(blockIdx.y);
    const int row = ((static_cast<int>(blockIdx.x) - unit * p.row_groups) * kMergeWarps + warp) * kWarpRows + lane % kWarpRows;
    const int b = unit / p.Hkv, kvh = unit - b * p.Hkv, tile = row / kTileRows, r = row % kTileRows;
    // (the plan is not new any more: the kernel before has waited for it before it let this one start)
    const int2 head = p.heads ? __ldcg(p.heads + unit) : make_int2(unit * p.n_splits, p.n_splits);      // first slot, parts
    pdl_trigger();
    pdl_wait();                                             // the partial results come from the previous kernel
    if (head.y < 2 || tile >= p.row_tiles) return;          // (the same for the whole warp: it has rows of one tile)
    const int len = __ldcg(p.tail_len + b), n_new = p.n_new ? __ldcg(p.n_new + b) : p.n_max;
    const long long slot0 = static_cast<long long>(head.x) * p.row_tiles + tile;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = kNegInf, l = 0.f;
    for (int s0 = of; s0 < head.y; s0 += kAhead * kLanes) {
        float lse[kAhead];
        float4 x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int s = s0 + u * kLanes;
            lse[u] = kNegInf;
            if (s < head.y) {
                const long long slot = slot0 + static_cast<long long>(s) * p.row_tiles;
                lse[u] = __ldcg(p.part_lse + slot * kTileRows + r);
                x[u] = __ldcg(reinterpret_cast<const float4 *>(p.part_o) + (slot * (D / 4) + quad) * kTileRows + r);
            }
        }
        float m_new = m;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) m_new = fmaxf(m_new, lse[u]);
        if (m_new == kNegInf) continue;                     // parts that saw no key
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
    // the lanes of a row, in a fixed order
#pragma unroll
    for (int o = kWarpRows; o < 32; o <<= 1) {
        const float m2 = __shfl_xor_sync(kFull, m, o), l2 = __shfl_xor_sync(kFull, l, o);
        const float4 x = make_float4(__shfl_xor_sync(kFull, acc.x, o), __shfl_xor_sync(kFull, acc.y, o), __shfl_xor_sync(kFull, acc.z, o), __shfl_xor_sync(kFull, acc.w, o));
        const float top = fmaxf(m, m2), a = m == kNegInf ? 0.f : ex2(m - top), c = m2 == kNegInf ? 0.f : ex2(m2 - top);
        l = l * a + l2 * c;
        acc.x = acc.x * a + x.x * c; acc.y = acc.y * a + x.y * c; acc.z = acc.z * a + x.z * c; acc.w = acc.w * a + x.w * c;
        m = top;
    }
    const int n = len < 0 ? 0 : min(n_new, p.n_max);
    if (of != 0 || row >= n << lr) return;
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint2 *dst = reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.out) +
                 ((static_cast<long long>(b) * p.n_max + (row >> lr)) * p.Hq + kvh * p.rep + (row & (p.rep - 1))) * D + quad * 4);
    *dst = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
}

}  // namespace

template <int D, int kRows>
static cudaError_t prepare()
{
    return cudaFuncSetAttribute(tree_kernel<D, kRows>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, kRows>::kSmemBytes);
}
cudaError_t prepare_tree(int head_dim)
{
    if (head_dim != 128 && head_dim != 64) return cudaErrorInvalidValue;
    const cudaError_t e = head_dim == 128 ? prepare<128, 64>() : prepare<64, 64>();
    return e != cudaSuccess ? e : head_dim == 128 ? prepare<128, 128>() : prepare<64, 128>();
}

template <int D, int kRows>
static cudaError_t launch(const TreeParams &p, int grid, cudaStream_t st)
{
    return launch_pdl(tree_kernel<D, kRows>, dim3(grid), dim3(Cfg<D, kRows>::kThreads), Cfg<D, kRows>::kSmemBytes, st, p);
}
cudaError_t launch_tree(const TreeParams &p, int head_dim, int grid, cudaStream_t st)
{
    if (head_dim != 128 && head_dim != 64) return cudaErrorInvalidValue;
    const bool few = p.n_max * p.rep <= 64;
    if (few ? p.row_tiles != 1 || p.box_tokens * p.rep > 64 : p.box_tokens * p.rep > 128) return cudaErrorInvalidValue;
    const cudaError_t e = head_dim == 128 ? (few ? launch<128, 64>(p, grid, st) : launch<128, 128>(p, grid, st))
                                          : (few ? launch<64, 64>(p, grid, st) : launch<64, 128>(p, grid, st));
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <int D>
static cudaError_t launch_merge(TreeMergeParams p, int batch, int most, cudaStream_t st)
{
    // Few parts (calls with many units): lanes side by side; many: eight lanes a row, five parts each at a time.
    const int lanes = most > 4 ? 8 : 1, rows = kMergeWarps * 32 / lanes;
    p.row_groups = (p.n_max * p.rep + rows - 1) / rows;
    const dim3 grid(static_cast<unsigned>(batch) * p.Hkv * p.row_groups, D / 4), block(kMergeWarps * 32);
    return lanes == 8 ? launch_pdl(tree_merge_kernel<D, 8, 5>, grid, block, 0, st, p) : launch_pdl(tree_merge_kernel<D, 1, 4>, grid, block, 0, st, p);
}
cudaError_t launch_tree_merge(const TreeMergeParams &p, int head_dim, int batch, int most, cudaStream_t st)
{
    if (head_dim != 128 && head_dim != 64) return cudaErrorInvalidValue;
    const cudaError_t e = head_dim == 128 ? launch_merge<128>(p, batch, most, st) : launch_merge<64>(p, batch, most, st);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace enl
