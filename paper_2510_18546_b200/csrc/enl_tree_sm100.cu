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
// Splits: the host knows the cached pages of a request, but not how long its tail is.  So it settles how many splits a request has, and split s of
// ns takes pages [C s / ns, C (s + 1) / ns) of the C cached ones and the same part of the tail's and the nodes' pages, whose number the
// device finds.  The cached pages of the first steps are fetched before the kernel waits for the one before it (plan and pool are written by the
// library only); lengths are read while they are on their way.  (With shares that the device cut from the whole stream the first
// scores were there 4.6 us after the wait for the previous kernel, for 16 requests 5.5, ...)  Splits leave outputs normalised by their own sums,
// and log2-sum-exps, in the scratch buffer; tree_merge_kernel puts them together.
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
    static constexpr int kBars       = 7 + 2 * (kRingK + kRingV);
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
    const uint32_t bar_q_full = bar0, bar_pv_done = bar0 + 8u, bar_o_done = bar0 + 16u;      // P V of a step, of the last one
    auto bar_s_full  = [&](int b) { return bar0 + 8u * (3 + b); };              // b: step & 1
    auto bar_p_full  = [&](int b) { return bar0 + 8u * (5 + b); };
    auto bar_k_full  = [&](int x) { return bar0 + 8u * (7 + x); };              // x: place in the ring
    auto bar_k_empty = [&](int x) { return bar0 + 8u * (7 + C::kRingK + x); };
    auto bar_v_full  = [&](int x) { return bar0 + 8u * (7 + 2 * C::kRingK + x); };
    auto bar_v_empty = [&](int x) { return bar0 + 8u * (7 + 2 * C::kRingK + C::kRingV + x); };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + C::kBarOff + 8 * C::kBars);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    if (sbase & 1023u) {                      // (swizzled tiles need it, and dynamic shared memory starts like this)
        if (threadIdx.x == 0) atomicExch(p.status, 1);
        return;
    }
    if (p.wait_first) pdl_wait();
    // ---- what this CTA does: request, kv head, tile of rows, split; the cached pages of that split ----
    struct { int b, kvh, rt, split, n_splits, first, count; } it;
    if (p.batch == 1) {
        const int idx = static_cast<int>(blockIdx.x), above = idx / p.row_tiles;
        it.b = 0;
        it.rt = idx - above * p.row_tiles;
        it.kvh = above / p.n_splits;
        it.split = above - it.kvh * p.n_splits;
        it.n_splits = p.n_splits;
        it.first = static_cast<int>(static_cast<long long>(p.n_entries) * it.split / p.n_splits);
        it.count = static_cast<int>(static_cast<long long>(p.n_entries) * (it.split + 1) / p.n_splits) - it.first;
    } else {
        const int4 a = __ldcg(reinterpret_cast<const int4 *>(p.items) + blockIdx.x);
        it.b = a.x >> 16; it.kvh = a.x & 0xffff;
        it.rt = a.y >> 24; it.split = a.y >> 12 & 0xfff; it.n_splits = a.y & 0xfff;
        it.first = a.z; it.count = a.w;
    }

    // ---- set-up ----
    if (warp == C::kMmaWarp) {
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
        t_first = static_cast<int>(static_cast<long long>(t) * it.split / it.n_splits);
        t_count = static_cast<int>(static_cast<long long>(t) * (it.split + 1) / it.n_splits) - t_first;
        n_steps = it.rt * kRows < n * p.rep ? (it.count + t_count + kStepPages - 1) / kStepPages : 0;
    };

    if (warp == C::kKWarp || warp == C::kVWarp) {
        // ================= TMA producers =================
        const bool is_k = warp == C::kKWarp;
        const CUtensorMap *tm_pool = is_k ? &p.tm_kpool : &p.tm_vpool, *tm_tail = is_k ? &p.tm_ktail : &p.tm_vtail,
                          *tm_new = is_k ? &p.tm_knew : &p.tm_vnew;
        const uint32_t ring = sbase + static_cast<uint32_t>(is_k ? C::kKOff : C::kVOff), full0 = is_k ? bar_k_full(0) : bar_v_full(0),
                       empty0 = is_k ? bar_k_empty(0) : bar_v_empty(0);
        const int places = is_k ? C::kRingK : C::kRingV;
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
        // the steps of cached pages alone that the ring has room for, before the wait for the kernel before
        const int early = p.wait_first ? 0 : min(places, it.count / kStepPages);
        uint32_t cur = 0, next = where(lane);                        // (of the cached pages so far)
        int jj = 0;
        for (; jj < early; ++jj) fetch(__shfl_sync(kFull, next, jj * kStepPages + lane % kStepPages), jj);
        pdl_wait();
        read_lengths();
        if (n_steps > 0 && is_k && lane == 0) {
            mbar_expect_tx(bar_q_full, static_cast<uint32_t>(C::kBlocks * p.box_tokens * p.rep * 128));
            for (int b = 0; b < C::kBlocks; ++b)
                tma_load_3d(sbase + b * C::kBlockBytes, &p.tm_q, b * 64, it.kvh * p.rep, it.b * p.n_max + it.rt * (kRows / p.rep), bar_q_full);
        }
        __syncwarp();
        if (lane >= it.count) next = where(lane);
        static_assert(C::kRingK < kBatch && C::kRingV < kBatch, "the early steps' pages are of one batch");
        cur = next;
        if (jj > 0) next = where(kBatch * kStepPages + lane);
        for (; jj < n_steps; ++jj) {
            const int x = jj % places;
            if (jj % kBatch == 0) {
                cur = next;
                next = where((jj + kBatch) * kStepPages + lane);
            }
            const uint32_t at = __shfl_sync(kFull, cur, jj % kBatch * kStepPages + lane % kStepPages);
            if (jj >= places) ok = mbar_wait(empty0 + 8u * x, static_cast<uint32_t>((jj / places - 1) & 1), abort_flag, p.status);
            if (!ok) break;
            fetch(at, x);
        }
        // Copies in flight land before the CTA retires: on the error path, and where there turned out to be nothing to do.
        if (!ok || n_steps == 0) {
            for (int f = max(0, jj - places); f < jj; ++f) {
                const unsigned long long t0 = global_ns();
                while (!mbar_try_wait(full0 + 8u * (f % places), static_cast<uint32_t>((f / places) & 1)) && global_ns() - t0 < 2000000ull) { }
            }
        }
    } else {
      pdl_wait();
      read_lengths();
      if (n_steps > 0 && warp == C::kMmaWarp) {
        // ================= MMA issuer =================
        constexpr uint32_t idesc_qk = make_idesc(kStepKeys, false), idesc_pv = make_idesc(D, true);
        constexpr uint32_t kStepUnits = C::kStepBytes >> 4, kGroupUnits = C::kGroupBytes >> 4;
        const uint64_t dq0 = smem_desc(sbase, 16), dk0 = smem_desc(sbase + C::kKOff, 16, C::kGroupBytes), dv0 = smem_desc(sbase + C::kVOff, 1024, C::kGroupBytes);
        const uint32_t dq_lo = static_cast<uint32_t>(dq0), dq_hi = static_cast<uint32_t>(dq0 >> 32);
        const uint32_t dk_lo = static_cast<uint32_t>(dk0), dk_hi = static_cast<uint32_t>(dk0 >> 32);
        const uint32_t dv_lo = static_cast<uint32_t>(dv0), dv_hi = static_cast<uint32_t>(dv0 >> 32);
        // A commit that frees a place of the ring is made only where a later fetch waits for it: nothing may arrive after the CTA has retired.
        auto issue_qk = [&](int jj) {
            const int x = jj % C::kRingK, b = jj & 1;
            const uint32_t ka = dk_lo + static_cast<uint32_t>(x) * kStepUnits, d = tmem_base + static_cast<uint32_t>(b * kStepKeys);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t in_row = static_cast<uint32_t>((kk & 3) * 2);                       // 32 bytes per 16 channels
                mma_ss2(d, dq_lo + static_cast<uint32_t>((kk >> 2) * (C::kBlockBytes >> 4)) + in_row, dq_hi,
                        ka + static_cast<uint32_t>((kk >> 2) * (1024 >> 4)) + in_row, dk_hi, idesc_qk, kk > 0 ? 1u : 0u);
            }
            tc_commit(bar_s_full(b));
            if (jj + C::kRingK < n_steps) tc_commit(bar_k_empty(x));
        };
        // O (+)= P V; P of keys 2c, 2c + 1 sits in column c of the buffer that held their scores
        auto issue_pv = [&](int jj) {
            const int x = jj % C::kRingV, b = jj & 1;
            const uint32_t va = dv_lo + static_cast<uint32_t>(x) * kStepUnits, a = tmem_base + static_cast<uint32_t>(b * kStepKeys);
#pragma unroll
            for (int k4 = 0; k4 < kStepPages; ++k4)                  // 16 keys = two groups of 8 rows, 8 columns of P
                mma_ts2(tmem_base + kOCol, a + static_cast<uint32_t>(k4 * 8), va + static_cast<uint32_t>(k4 * 2) * kGroupUnits, dv_hi, idesc_pv,
                        (jj == 0 && k4 == 0) ? 0u : 1u);
            if (jj + C::kRingV < n_steps) tc_commit(bar_v_empty(x));
            tc_commit(jj + 1 < n_steps ? bar_pv_done : bar_o_done);
        };
        auto wait_k = [&](int jj) { return mbar_wait(bar_k_full(jj % C::kRingK), static_cast<uint32_t>((jj / C::kRingK) & 1), abort_flag, p.status); };
        ok = mbar_wait(bar_q_full, 0, abort_flag, p.status);
        for (int jj = 0; jj < min(2, n_steps) && ok; ++jj) {
            ok = wait_k(jj);
            if (!ok) break;
            tc_fence_after();
            issue_qk(jj);
        }
        for (int jj = 0; jj < n_steps && ok; ++jj) {
            const bool more = jj + 2 < n_steps;
            ok = mbar_wait(bar_v_full(jj % C::kRingV), static_cast<uint32_t>((jj / C::kRingV) & 1), abort_flag, p.status);
            if (ok && more) ok = wait_k(jj + 2);
            if (ok) ok = mbar_wait(bar_p_full(jj & 1), static_cast<uint32_t>((jj >> 1) & 1), abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();
            issue_pv(jj);
            if (more) issue_qk(jj + 2);
        }
        if (ok) ok = mbar_wait(bar_o_done, 0, abort_flag, p.status);
      } else if (warp < C::kSoftmaxWarps && it.rt * kRows + warp * 32 < n * p.rep) {
        // ================= softmax: one thread per query row =================
        const int rep = p.rep, lr = 31 - __clz(rep);
        const int r = warp * 32 + lane, n_act = (min(kRows, n * rep - it.rt * kRows) + 31) >> 5;      // softmax warps with rows
        const int t = it.rt * (kRows >> lr) + (r >> lr);              // node
        const bool row_valid = t < n;
        const uint32_t lane_sel = static_cast<uint32_t>(warp * 32) << 16;
        const uint32_t t_s = tmem_base + lane_sel, t_o = tmem_base + lane_sel + kOCol;
        const float scale = p.scale_log2;
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
        int meta = 0, meta_next = n_steps > 0 ? load_meta(lane) : 0;
        float m = kNegInf, l = 0.f;                                   // reference (log2 units), row sum
        for (int jj = 0; jj < n_steps; ++jj) {
            const int b = jj & 1;
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
                const int x = jj % C::kRingV;
                bool waited = false;
#pragma unroll
                for (int e = 0; e < kStepPages; ++e) {
                    const int rows = pg[e] & 256 ? min(kPageTokens, n - (pg[e] & 63)) : pg[e];
                    if (jj * kStepPages + e < it.count || rows == 0 || rows == kPageTokens) continue;
                    if (!waited) ok = mbar_wait(bar_v_full(x), static_cast<uint32_t>((jj / C::kRingV) & 1), abort_flag, p.status);
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
            if (lane == 0) mbar_arrive_n(bar_p_full(b), warp == 0 ? static_cast<uint32_t>(C::kSoftmaxWarps + 1 - n_act) : 1u);
            float lo0, hi0, lo1, hi1;
            unpack2(ps2[0], lo0, hi0);
            unpack2(ps2[1], lo1, hi1);
            l += (lo0 + hi0) + (lo1 + hi1);
        }
        if (ok && n_steps > 0) ok = mbar_wait(bar_o_done, 0, abort_flag, p.status);
        if (ok) {
            tc_fence_after();
            // (A split without a step has seen nothing, and O holds nothing: 0, as for a row that sees no key.)
            const float inv = l > 0.f ? 1.f / l : 0.f;
            const bool split = it.n_splits > 1;
            if (split) p.part_lse[static_cast<long long>(blockIdx.x) * kTileRows + r] = l > 0.f ? m + lg2(l) : kNegInf;
            // partial outputs [CTA][D / 4][row][4]: a warp's store is one contiguous piece
            float4 *part = reinterpret_cast<float4 *>(p.part_o) + static_cast<long long>(blockIdx.x) * (D / 4) * kTileRows + r;
            uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) +
                         ((static_cast<long long>(it.b) * p.n_max + t) * p.Hq + it.kvh * rep + (r & (rep - 1))) * D);
#pragma unroll 1
            for (int k = 0; k < D / 32; ++k) {
                uint32_t o[32];
                tmem_ld32_wait(t_o + static_cast<uint32_t>(k * 32), o);
                float f[32];
#pragma unroll
                for (int x = 0; x < 32; ++x) f[x] = l > 0.f ? __uint_as_float(o[x]) * inv : 0.f;
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
    }

    // ---- teardown ----
    tc_fence_before();
    __syncthreads();
    if (warp == C::kMmaWarp) {
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
    const int kvh = at / row_groups, rows0 = (at - kvh * row_groups) * 32, tile = rows0 / kTileRows;      // (calls of fewer rows have one tile)
    const int quad = kDeep ? static_cast<int>(blockIdx.y) : static_cast<int>(blockIdx.y) * kMergeWarps + warp;
    pdl_trigger();
    pdl_wait();                                             // the partial results come from the previous kernel
    const int2 head = p.heads ? __ldcg(p.heads + b) : make_int2(0, p.n_splits);      // first CTA, splits
    const int n = __ldcg(p.tail_len + b) < 0 ? 0 : p.n_new ? min(__ldcg(p.n_new + b), p.n_max) : p.n_max;
    const int row = rows0 + lane;
    if (head.y < 2 || rows0 >= n << lr) return;
    const bool on = row < n << lr;
    const int r = row % kTileRows;
    const long long cta0 = head.x + static_cast<long long>(kvh) * head.y * p.row_tiles + tile;
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
                const long long cta = cta0 + static_cast<long long>(s) * p.row_tiles;
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
