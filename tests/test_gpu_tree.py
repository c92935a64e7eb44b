"""Drafted trees over selected groups and growing tails, on the GPU, against the plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2510_18546_b200 import enl
from tests import tree_reference as ref

pytestmark = pytest.mark.gpu

BF16, I32 = torch.bfloat16, torch.int32
NAN = float("nan")
MODELS = [(32, 8, 128), (8, 2, 64), (8, 8, 64), (4, 4, 128), (4, 2, 128), (16, 2, 128), (16, 1, 64), (32, 2, 128)]


def dev(a, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda", dtype)


def f64(t):
    return t.detach().double().cpu().numpy()


class Case:
    """A cache with groups, tails in pages that lie in no order, trees.  What does not count is NaN: rows behind a tail's end, pages that no
    request holds, nodes behind n_new."""

    def __init__(self, model, group_lens, tails, n_new, n_max, seed=0, std=1.5, parents=None, max_blocks=None, scratch_bytes=0, pages=None,
                 layers=1, spare_groups=2):
        self.n_q, self.n_kv, self.d = model
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.batch, self.n_max = len(tails), n_max
        self.tails, self.n_new = np.asarray(tails, np.int32), np.asarray(n_new, np.int32)
        self.lens = [list(x) for x in group_lens]

        def rows(*shape, s=1.0):
            return torch.randn(*shape, generator=g, device="cuda") .mul_(s).to(BF16)

        flat = [n for x in self.lens for n in x]
        self.k_group = [[rows(n, self.n_kv, self.d) for n in flat] for _ in range(layers)]
        self.v_group = [[rows(n, self.n_kv, self.d) for n in flat] for _ in range(layers)]
        self.cache = enl.enl_cache_create(layers, self.n_q, self.n_kv, self.d, max_groups=len(flat) + spare_groups, max_tokens=max(sum(flat), 1) + 64,
                                          device=0, max_batch=self.batch, scratch_bytes=scratch_bytes)
        # groups have been longer before: what is left of them behind their ends must not show
        for layer in range(layers):
            for i, n in enumerate(flat):
                enl.enl_group_store(self.cache, i, layer, self.k_group[layer][i], self.v_group[layer][i])
        self.sel = np.arange(len(flat), dtype=np.int32)
        self.cu_sel = np.concatenate([[0], np.cumsum([len(x) for x in self.lens])]).astype(np.int32)
        blocks = -(-np.maximum(self.tails, 0) // 16)
        self.max_blocks = max_blocks or int(max(blocks.max(), 1)) + 1
        n_pages = pages or int(blocks.sum()) + 3
        order = rng.permutation(n_pages).astype(np.int32)
        self.table = np.full((self.batch, self.max_blocks), -1, np.int32)
        self.k_tail = torch.full((n_pages, self.n_kv, 16, self.d), NAN, dtype=BF16, device="cuda")
        self.v_tail = torch.full((n_pages, self.n_kv, 16, self.d), NAN, dtype=BF16, device="cuda")
        self.own = []                                            # every request's tail rows
        at = 0
        for b in range(self.batch):
            t = max(int(self.tails[b]), 0)
            k, v = rows(t, self.n_kv, self.d), rows(t, self.n_kv, self.d)
            self.own.append((k, v))
            for j in range(blocks[b]):
                page, n = int(order[at]), min(16, t - 16 * j)
                at += 1
                self.table[b, j] = page
                self.k_tail[page, :, :n] = k[16 * j:16 * j + n].transpose(0, 1)
                self.v_tail[page, :, :n] = v[16 * j:16 * j + n].transpose(0, 1)
        self.q = rows(self.batch, n_max, self.n_q, self.d, s=std)
        self.k, self.v = rows(self.batch, n_max, self.n_kv, self.d), rows(self.batch, n_max, self.n_kv, self.d)
        self.see = []
        for b in range(self.batch):
            n = self.count(b)
            self.q[b, n:], self.k[b, n:], self.v[b, n:] = NAN, NAN, NAN
            parent = None
            if parents != "chain":
                parent = np.array([-1] + [int(rng.integers(-1, i)) for i in range(1, max(n, 1))])
            self.see.append(ref.ancestors(parent, n))
        self.mask = None if parents == "chain" else dev(np.stack([ref.bits(s, n_max) for s in self.see]))
        self.out = torch.full((self.batch, n_max, self.n_q, self.d), 7.0, dtype=BF16, device="cuda")
        self.d_table, self.d_tails, self.d_new = dev(self.table), dev(self.tails), dev(self.n_new)

    def count(self, b):
        return 0 if self.tails[b] < 0 else int(min(max(self.n_new[b], 0), self.n_max))

    def call(self, layer=0, **kw):
        args = dict(n_new=self.d_new, mask=self.mask, cu_sel=self.cu_sel, stream=torch.cuda.current_stream().cuda_stream)
        args.update(kw)
        enl.enl_attend_tree(self.cache, layer, self.sel, self.q, self.k, self.v, self.k_tail, self.v_tail, self.d_table, self.d_tails, self.out, **args)

    def check(self, layer=0):
        torch.cuda.synchronize()
        assert enl.enl_cache_status(self.cache) == enl.ENL_OK
        got = f64(self.out)
        for b in range(self.batch):
            n = self.count(b)
            assert (got[b, n:] == 7.0).all(), f"request {b}: rows behind the last node were written"
            if n == 0:
                continue
            g = range(self.cu_sel[b], self.cu_sel[b + 1])
            k, v = [np.concatenate([f64(x[layer][i]) for i in g] + [f64(self.own[b][at]), f64(new[b, :n])])
                    for at, (x, new) in enumerate(((self.k_group, self.k), (self.v_group, self.v)))]
            see = np.concatenate([np.ones((n, len(k) - n), bool), self.see[b]], 1)
            want, tol = ref.attend(f64(self.q[b, :n]), k, v, see)
            assert np.isfinite(got[b, :n]).all(), f"request {b}: not finite"
            off = np.abs(got[b, :n] - want)
            assert (off <= tol).all(), f"request {b}: {(off - tol).max():.3e} above the bound, max {off.max():.3e}"

    def close(self):
        torch.cuda.synchronize()
        try:
            assert enl.enl_cache_selfcheck(self.cache) == enl.ENL_OK
        finally:
            enl.enl_cache_free(self.cache)


def run(*a, **kw):
    c = Case(*a, **kw)
    try:
        c.call()
        c.check()
    finally:
        c.close()


@pytest.mark.parametrize("model", MODELS, ids=str)
@pytest.mark.parametrize("nodes", [1, 2, 7, 16, 17, 33, 64])
def test_one_request(model, nodes):
    run(model, [[40, 1, 17, 64]], [37], [nodes], nodes, seed=nodes)


@pytest.mark.parametrize("tail", [0, 1, 15, 16, 17, 31, 48, 100])
@pytest.mark.parametrize("groups", [[], [16], [5, 0, 33]], ids=str)
def test_tails_and_groups(tail, groups):
    """Pages that end inside a step, empty groups, empty lists, empty tails."""
    run((8, 2, 128), [groups], [tail], [9], 9, seed=tail)


@pytest.mark.parametrize("model", [(32, 8, 128), (8, 2, 64)], ids=str)
@pytest.mark.parametrize("batch", [2, 5, 33, 70])
def test_ragged_batches(model, batch):
    """Requests of every kind side by side: ended ones, ones without nodes, counts beyond the rows, empty tails."""
    rng = np.random.default_rng(batch)
    lens = [rng.integers(0, 60, rng.integers(0, 5)).tolist() for _ in range(batch)]
    tails = rng.integers(0, 90, batch)
    n_new = rng.integers(0, 15, batch)
    tails[::7], n_new[1::6], tails[2::9] = -1, 0, 0
    n_new[-1] = 40                                               # beyond n_max: as many as there are rows
    run(model, lens, tails, n_new, 12, seed=batch)


def test_one_long_request_among_short_ones():
    run((8, 2, 128), [[700] * 9, [20], [33], [16, 16]], [900, 3, 0, 17], [20, 20, 1, 7], 20)


@pytest.mark.parametrize("model,batch,n_max", [((8, 2, 64), 40, 5), ((16, 2, 128), 41, 12), ((32, 2, 128), 14, 24), ((8, 2, 128), 40, 30)], ids=str)
def test_runs_of_parts_across_requests(model, batch, n_max):
    """Streams that do not divide into equal parts: most CTAs take the end of one and the beginning of the next, with other counts of rows; some
    of them belong to requests that have ended or have no nodes, the first ones too."""
    rng = np.random.default_rng(n_max)
    tails, n_new = rng.integers(0, 300, batch), rng.integers(0, n_max + 1, batch)
    tails[::9], n_new[3::8] = -1, 0
    c = Case(model, [[int(rng.integers(900, 1200)) for _ in range(4)] for _ in range(batch)], tails, n_new, n_max, seed=n_max)
    try:
        c.call()
        tiles = -(-n_max * (model[0] // model[1]) // 128)
        assert enl.enl_plan_inspect(c.cache)["n_items"] == 148 // tiles * tiles, "equal parts: not what this test is for"
        c.check()
        first = c.out.clone()
        for _ in range(3):
            c.out[:] = 7.0
            c.call()
            torch.cuda.synchronize()
            assert torch.equal(first, c.out)
    finally:
        c.close()


@pytest.mark.parametrize("model,batch,n_max", [((8, 2, 64), 80, 5), ((8, 8, 128), 19, 9), ((32, 2, 128), 27, 24)], ids=str)
def test_more_streams_than_multiprocessors(model, batch, n_max):
    """More than a wave of CTAs, in whole streams or in runs."""
    rng = np.random.default_rng(n_max)
    tails, n_new = rng.integers(0, 300, batch), rng.integers(0, n_max + 1, batch)
    tails[::9], n_new[3::8] = -1, 0
    tails[-1], n_new[-1] = 100, n_max
    c = Case(model, [[int(rng.integers(500, 800)) for _ in range(4)] for _ in range(batch)], tails, n_new, n_max, seed=n_max)
    try:
        c.call()
        c.check()
    finally:
        c.close()


@pytest.mark.parametrize("model,nodes", [((32, 8, 128), 1), ((32, 8, 128), 30), ((32, 8, 128), 64), ((16, 2, 128), 40), ((32, 2, 128), 64), ((16, 1, 64), 64),
                                         ((8, 8, 64), 64)], ids=str)
def test_long_streams(model, nodes):
    """Many steps, many splits, one to eight tiles of rows."""
    run(model, [[311] * 17 + [16] * 20], [1000], [nodes], nodes, seed=3)


@pytest.mark.parametrize("batch", [1, 3])
def test_chain_without_masks(batch):
    run((32, 8, 128), [[40, 40]] * batch, [50] * batch, [13] * batch, 13, parents="chain")


def test_single_tokens_of_a_batch():
    run((32, 8, 128), [[100, 60]] * 9, list(range(0, 90, 10)), [1] * 9, 1, parents="chain")


def test_without_counts_every_row_is_a_node():
    c = Case((8, 2, 64), [[30]] * 3, [5, 20, 0], [6, 6, 6], 6)
    try:
        c.call(n_new=None)
        c.check()
    finally:
        c.close()


@pytest.mark.parametrize("d", [64, 128])
def test_masks_of_any_kind(d):
    """Masks that are no trees: nothing at all (zeros where there is nothing else), later nodes, bits behind the last node."""
    for groups, tail in (([], 0), ([], 3), ([20], 0)):
        c = Case((8, 2, d), [groups], [tail], [40], 50)
        try:
            see = np.random.default_rng(1).random((40, 40)) < 0.3
            see[[0, 31, 39]] = False
            c.see = [see]
            words = ref.bits(see, 50)
            words[:40] |= np.int64(-1) << np.int64(40)           # count for nothing
            c.mask = dev(words[None])
            c.call()
            c.check()
            if not groups and not tail:
                assert (c.out[0, [0, 31, 39]] == 0).all()
        finally:
            c.close()


@pytest.mark.parametrize("std", [0.0, 30.0, 200.0])
def test_flat_and_steep_scores(std):
    """Running maxima that jump by hundreds from step to step."""
    run((8, 2, 128), [[200, 300]], [150], [24], 24, std=std, seed=5)


def test_scores_that_grow_from_page_to_page():
    c = Case((8, 2, 64), [[16] * 40], [64], [8], 8)
    try:
        with torch.no_grad():
            c.q[:] = 1.0
            for i in range(40):
                c.k_group[0][i][:] = i / 16
                enl.enl_group_store(c.cache, i, 0, c.k_group[0][i], c.v_group[0][i])
        c.call()
        c.check()
    finally:
        c.close()


def test_infinite_scores_and_values_of_hidden_keys():
    """Keys that nobody may see (other requests' pages, rows behind a tail) are infinite here, not NaN."""
    c = Case((8, 2, 128), [[33], [40]], [21, 40], [5, 6], 9)
    try:
        for t in (c.k_tail, c.v_tail, c.k, c.v, c.q):
            t[torch.isnan(t)] = float("inf")
        c.call()
        c.check()
    finally:
        c.close()


@pytest.mark.parametrize("model,tails,n_max", [((8, 2, 64), [40], 9), ((32, 8, 128), [0], 64), ((32, 8, 128), [700], 33), ((16, 1, 64), [5, 900, 0], 20),
                                               ((4, 4, 128), [16, 3, 250, 64], 1), ((32, 2, 128), [100, 31], 50)], ids=str)
def test_values_that_are_not_finite_reach_those_who_see_them(model, tails, n_max):
    """0 x inf is NaN, but a node that is not seen does not count."""
    c = Case(model, [[100, 30]] * len(tails), tails, [n_max] * len(tails), n_max, seed=n_max)
    try:
        rng = np.random.default_rng(n_max)
        keep = c.v.clone()
        what = np.zeros((c.batch, n_max, c.n_kv, c.d))
        for _ in range(3 * c.batch):
            b, j, h = int(rng.integers(c.batch)), int(rng.integers(n_max)), int(rng.integers(c.n_kv))
            at = rng.choice(c.d, int(rng.choice([1, 5, c.d])), replace=False)
            what[b, j, h, at] = rng.choice([NAN, np.inf, -np.inf])
        odd = ~np.isfinite(what)
        c.v = torch.where(dev(odd), dev(what, BF16), c.v)
        clean = torch.where(dev(odd), torch.zeros_like(keep), keep)
        c.call()
        torch.cuda.synchronize()
        assert enl.enl_cache_status(c.cache) == enl.ENL_OK
        got, rep = f64(c.out), c.n_q // c.n_kv
        with np.errstate(invalid="ignore"):
            for b in range(c.batch):
                for i in range(n_max):
                    seen = np.nonzero(c.see[b][i])[0]
                    add = np.repeat(np.where(odd[b, seen], what[b, seen], 0.0).sum(0), rep, 0)      # 0, inf, -inf or NaN for every head and channel
                    bad = ~np.isfinite(add)
                    assert np.array_equal(got[b, i][bad], add[bad], equal_nan=True)
                    assert np.isfinite(got[b, i][~bad]).all()
                    got[b, i][bad] = 0.0
        # where they are finite, outputs are those of the same values without them
        c.v = clean
        c.call()
        torch.cuda.synchronize()
        want = f64(c.out)
        for b in range(c.batch):
            for i in range(n_max):
                seen = np.nonzero(c.see[b][i])[0]
                bad = np.repeat(odd[b, seen].any(0), rep, 0)
                assert np.array_equal(got[b, i][~bad], want[b, i][~bad])
        c.check()
    finally:
        c.close()


def test_small_scratch_means_no_splits():
    run((8, 2, 128), [[300] * 4], [200], [8], 8, scratch_bytes=4096)
    run((8, 2, 128), [[300] * 4] * 3, [200, 0, 9], [8, 1, 3], 8, scratch_bytes=200000)


def test_table_entries_that_name_no_page():
    """Zeros are read there, nothing else happens."""
    c = Case((8, 2, 64), [[20]], [40], [4], 4)
    try:
        for k, bad in enumerate((-1, c.k_tail.shape[0], 0x7fffffff)):
            c.d_table[0, k] = bad
        for x in c.own[0]:
            x[:] = 0
        c.call()
        c.check()
    finally:
        c.close()


def test_tail_beyond_its_table():
    """The tail ends where its block table does."""
    c = Case((8, 2, 64), [[20]], [64], [4], 4, max_blocks=4)
    try:
        c.d_tails[:] = 1 << 30
        c.call()
        c.check()
    finally:
        c.close()


def test_pages_far_into_a_pool():
    """Offsets beyond 32 bits, in elements and bytes."""
    n = (1 << 31) // (8 * 16 * 128) + 40
    c = Case((32, 8, 128), [[20]], [90], [5], 5)
    try:
        for name in ("k_tail", "v_tail"):
            near = getattr(c, name)
            far = torch.empty((n, 8, 16, 128), dtype=BF16, device="cuda")
            far[n - near.shape[0]:] = near
            setattr(c, name, far)
        c.d_table = torch.where(c.d_table >= 0, c.d_table + (n - near.shape[0]), -1)
        c.call()
        c.check()
    finally:
        c.close()


def test_layers_selections_and_stores_between_calls():
    """Plans are built anew when the selection, a group or the layer changes, and kept apart from enl_attend's."""
    c = Case((8, 2, 128), [[40, 17, 64]], [30], [6], 6, layers=2)
    try:
        for layer in (0, 1, 0):
            c.out[:] = 7.0
            c.call(layer)
            c.check(layer)
        # a call of enl_attend in between, over the same list
        q = torch.randn(20, 8, 128, device="cuda").to(BF16)
        k, v = torch.randn(20, 2, 128, device="cuda").to(BF16), torch.randn(20, 2, 128, device="cuda").to(BF16)
        out = torch.empty_like(q)
        first = None
        for _ in range(2):
            enl.enl_attend(c.cache, 0, c.sel, q, k, v, out, stream=torch.cuda.current_stream().cuda_stream)
            first = out.clone() if first is None else first
            assert torch.equal(out, first)
            c.out[:] = 7.0
            c.call()
            c.check()
        # another order, fewer groups
        c.sel, c.cu_sel = np.array([2, 0], np.int32), np.array([0, 2], np.int32)
        kg, vg = c.k_group, c.v_group
        c.k_group, c.v_group = [[x[2], x[0]] for x in kg], [[x[2], x[0]] for x in vg]
        c.out[:] = 7.0
        c.call()
        c.check()
        # a group grows
        more = [torch.randn(9, 2, 128, device="cuda").to(BF16) for _ in range(2)]
        enl.enl_group_store(c.cache, 2, 0, *more, mode=enl.ENL_APPEND)
        c.k_group[0][0], c.v_group[0][0] = torch.cat([c.k_group[0][0], more[0]]), torch.cat([c.v_group[0][0], more[1]])
        c.out[:] = 7.0
        c.call()
        c.check()
    finally:
        c.close()


def test_twice_the_same_bits():
    c = Case((32, 8, 128), [[311] * 9, [64] * 7], [700, 100], [30, 12], 30)
    try:
        c.call()
        torch.cuda.synchronize()
        first = c.out.clone()
        for _ in range(5):
            c.out[:] = 7.0
            c.call()
            torch.cuda.synchronize()
            assert torch.equal(first, c.out)
    finally:
        c.close()


def test_back_to_back_calls_of_different_shapes():
    """Nothing waits between the calls: scratch, plan and outputs are ordered by the stream."""
    cases = [Case((8, 2, 128), [[311] * 5], [70], [n], n, seed=n) for n in (1, 9, 40)]
    try:
        for _ in range(4):
            for c in cases:
                c.call()
        for c in cases:
            c.check()
    finally:
        for c in cases:
            c.close()


def test_another_stream():
    c = Case((8, 2, 128), [[100, 50]], [70], [9], 9)
    try:
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            c.call()
        s.synchronize()
        c.check()
    finally:
        c.close()


def test_captured_call_follows_the_lengths():
    """One graph, replayed while tail, counts, masks and block tables change under it."""
    c = Case((32, 8, 128), [[64, 40, 200]] * 2, [200, 250], [20, 20], 20)
    try:
        c.call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call()
        full = (c.own[0], c.own[1])
        for tails, n_new in (((200, 250), (20, 20)), ((0, 17), (1, 20)), ((160, 1), (20, 0)), ((-1, 250), (5, 3))):
            c.tails, c.n_new = np.asarray(tails, np.int32), np.asarray(n_new, np.int32)
            c.own = [tuple(x[:max(t, 0)] for x in full[b]) for b, t in enumerate(tails)]
            c.see = [ref.ancestors([-1] + list(range(n - 1)), c.count(b)) for b, n in enumerate(n_new)]
            c.d_tails.copy_(dev(c.tails))
            c.d_new.copy_(dev(c.n_new))
            c.mask.copy_(dev(np.stack([ref.bits(s, 20) for s in c.see])))
            c.out[:] = 7.0
            g.replay()
            c.check()
        c.out[:] = 7.0
        c.call()                                                  # and outside the graph again
        c.check()
        del g
    finally:
        c.close()


# ---- block tables, slots, positions, masks -----------------------------------------------------------------------------------
class Tails:
    def __init__(self, rng, batch, max_blocks, n_pages, used):
        order = rng.permutation(n_pages).astype(np.int32)
        self.n_blocks = np.asarray(used, np.int32)
        self.table = np.full((batch, max_blocks), -7, np.int32)
        at = 0
        for b in range(batch):
            self.table[b, :used[b]] = order[at:at + used[b]]
            at += used[b]
        self.free = np.full(n_pages, -9, np.int32)
        self.free[:n_pages - at] = order[at:]
        self.n_free = n_pages - at


def check_tables(t, tail_len, n_new, parent, pos_base, n_max, masks=True, positions=True, failed=0):
    batch = len(tail_len)
    d = {k: dev(getattr(t, k)) for k in ("table", "n_blocks", "free")}
    n_free = dev(np.array([t.n_free], np.int32))
    slot = torch.full((batch, n_max), 99, dtype=I32, device="cuda")
    pos = torch.full((batch, n_max), 99, dtype=I32, device="cuda") if positions else None
    mask = torch.full((batch, n_max), 99, dtype=torch.int64, device="cuda") if masks else None
    bad = torch.full((1,), 5, dtype=I32, device="cuda")
    opt = lambda x: None if x is None else dev(np.asarray(x, np.int32))  # noqa: E731
    enl.enl_tail_tables(dev(np.asarray(tail_len, np.int32)), d["table"], d["n_blocks"], d["free"], n_free, slot, pos, mask, n_new=opt(n_new),
                        parent=opt(parent), pos_base=opt(pos_base), failed=bad, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    want = ref.tables(np.asarray(tail_len), np.full(batch, n_max) if n_new is None else np.asarray(n_new), parent, pos_base, t.table, t.n_blocks, t.free,
                      t.n_free, n_max, masks)
    for k in ("table", "n_blocks", "free"):
        assert np.array_equal(d[k].cpu().numpy(), want[k]), k
    assert int(n_free) == want["n_free"]
    assert np.array_equal(slot.cpu().numpy(), want["slot"])
    if positions:
        assert np.array_equal(pos.cpu().numpy(), want["position"])
    if masks:
        assert np.array_equal(mask.cpu().numpy(), want["mask"])
    assert int(bad) == 5 + want["failed"] and want["failed"] >= failed
    t.table, t.n_blocks, t.free, t.n_free = want["table"], want["n_blocks"], want["free"], want["n_free"]
    return want


def random_parents(rng, batch, n_max):
    return np.stack([[int(rng.integers(-1, max(i, 1))) if i else -1 for i in range(n_max)] for _ in range(batch)]).astype(np.int32)


@pytest.mark.parametrize("batch,n_max", [(1, 1), (1, 64), (3, 17), (33, 33), (70, 2), (200, 64), (1024, 5)])
def test_tables_of_trees(batch, n_max):
    rng = np.random.default_rng(batch * 100 + n_max)
    tail = rng.integers(0, 200, batch)
    used = -(-tail // 16)
    n_new = rng.integers(0, n_max + 1, batch)
    t = Tails(rng, batch, 20, int(used.sum()) + 8 * batch + 4, used)
    check_tables(t, tail, n_new, random_parents(rng, batch, n_max), rng.integers(0, 1000, batch).astype(np.int32), n_max)
    # the next steps: tails have grown, some requests have ended
    for step in range(3):
        tail = np.where(tail >= 0, np.minimum(tail + n_new // 2 + 1, 16 * 20 - 70), tail)
        tail[rng.integers(0, batch)] = -1
        n_new = rng.integers(0, n_max + 1, batch)
        check_tables(t, tail, n_new, random_parents(rng, batch, n_max), None, n_max)


def test_tables_without_trees():
    """Rows in a chain: prompts longer than any tree, without masks, without counts."""
    rng = np.random.default_rng(1)
    for batch, n_max in ((1, 500), (5, 65), (3, 16384), (40, 130)):
        tail = rng.integers(0, 50, batch)
        t = Tails(rng, batch, 1100, batch * 1100, -(-tail // 16))
        check_tables(t, tail, None if batch == 1 else rng.integers(0, n_max + 9, batch), None, None, n_max, masks=False, positions=batch != 5)
    t = Tails(rng, 2, 9, 18, [0, 1])
    check_tables(t, [0, 9], [64, 7], None, [5, 6], 64)


def test_tables_when_pages_run_out():
    rng = np.random.default_rng(2)
    t = Tails(rng, 5, 6, 20, [1, 2, 1, 0, 3])
    t.n_free = 4
    # two pages for the first, three for the second (the list does not last), none needed by the third, the fourth gets none either
    w = check_tables(t, [16, 32, 3, 0, 40], [20, 40, 2, 9, 6], random_parents(rng, 5, 40), None, 40, failed=2)
    assert (w["slot"][1] == -1).all() and (w["slot"][2, :2] >= 0).all() and (w["slot"][3] == -1).all() and (w["slot"][4, :6] >= 0).all()
    # more pages than the table has columns
    t = Tails(rng, 2, 3, 30, [3, 0])
    check_tables(t, [48, 10], [1, 3], None, None, 8, failed=1)
    check_tables(t, [0x7ffffff0, 10], [8, 3], None, None, 8, failed=1)
    # what ended requests give back is there for the next call, not for this one
    t = Tails(rng, 3, 5, 5, [5, 0, 0])
    check_tables(t, [-1, 3, 0], [4, 4, 4], None, None, 4, failed=2)
    check_tables(t, [-1, 3, 0], [4, 4, 4], None, None, 4)


def test_tables_take_odd_counts_and_parents_for_what_they_say():
    rng = np.random.default_rng(3)
    t = Tails(rng, 3, 8, 24, [0, 0, 0])
    parent = np.array([[-1, 1, 5, 0, 2, -9], [3, 0, 1, 2, 3, 4], [-1, 0, 1, 2, 3, 4]], np.int32)
    check_tables(t, [0, 17, 3], [6, -4, 100], parent, None, 6)


# ---- accepted paths -------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("batch,n_max", [(1, 1), (1, 64), (7, 33), (300, 64), (9, 5)])
@pytest.mark.parametrize("chain", [False, True])
@pytest.mark.parametrize("first", [False, True])
def test_accepted_paths(batch, n_max, chain, first):
    rng = np.random.default_rng(batch + n_max)
    parent = None if chain else random_parents(rng, batch, n_max)
    token = rng.integers(0, 3, (batch, n_max)).astype(np.int32)         # few tokens: equal siblings, long paths
    target = rng.integers(0, 3, (batch, n_max)).astype(np.int32)
    n_new = rng.integers(-1, n_max + 3, batch).astype(np.int32)
    want_first = rng.integers(0, 3, batch).astype(np.int32) if first else None
    acc, n, nxt = (torch.full(s, 55, dtype=I32, device="cuda") for s in ((batch, n_max), (batch,), (batch,)))
    enl.enl_tree_accept(None if chain else dev(parent), dev(token), dev(target), acc, n, nxt, n_new=dev(n_new), first=dev(want_first) if first else None,
                        stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    a, c, x = ref.accept(n_new, parent, token, target, want_first, n_max)
    assert np.array_equal(acc.cpu().numpy(), a) and np.array_equal(n.cpu().numpy(), c) and np.array_equal(nxt.cpu().numpy(), x)


# ---- rows into pages --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layers,heads,d,batch,n_max", [(1, 1, 64, 1, 1), (3, 8, 128, 4, 16), (70, 2, 64, 3, 5), (2, 3, 8, 5, 130), (1, 5, 136, 2, 70)])
@pytest.mark.parametrize("path", [False, True])
def test_append(layers, heads, d, batch, n_max, path):
    rng = np.random.default_rng(layers)
    n_pages = batch * (n_max // 16 + 2)
    order = rng.permutation(n_pages * 16).astype(np.int32)
    slots = order[:batch * n_max].reshape(batch, n_max).copy()
    n = rng.integers(0, n_max + 1, batch).astype(np.int32)
    n[0] = n_max + 3 if batch > 1 else n_max
    tail = rng.integers(0, 50, batch).astype(np.int32)
    accept = np.stack([np.sort(rng.permutation(n_max)) for _ in range(batch)]).astype(np.int32)
    if batch > 2:
        tail[1] = -1                                                    # ended
        slots[2] = -1                                                   # got no pages
        if path and n_max > 2:
            accept[3 % batch, 1] = n_max                                # out of range
    ks, vs = ([torch.randn(batch, n_max, heads, d, device="cuda").to(BF16) for _ in range(layers)] for _ in range(2))
    kt, vt = ([torch.randn(n_pages, heads, 16, d, device="cuda").to(BF16) for _ in range(layers)] for _ in range(2))
    want_k, want_v, want_len = [x.clone() for x in kt], [x.clone() for x in vt], tail.copy()
    for b in range(batch):
        if tail[b] < 0:
            continue
        for k in range(min(n[b], n_max)):
            row, s = int(accept[b, k]) if path else k, int(slots[b, k])
            if s < 0 or not 0 <= row < n_max:
                continue
            want_len[b] += 1
            for l in range(layers):
                want_k[l][s // 16, :, s % 16] = ks[l][b, row]
                want_v[l][s // 16, :, s % 16] = vs[l][b, row]
    length = dev(tail)
    enl.enl_tail_append(ks, vs, kt, vt, dev(slots), length, length, accept=dev(accept) if path else None, n_accept=dev(n),
                        stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert np.array_equal(length.cpu().numpy(), want_len)
    for l in range(layers):
        assert torch.equal(kt[l], want_k[l]) and torch.equal(vt[l], want_v[l])


def test_append_without_counts_takes_every_row():
    k = torch.randn(2, 3, 2, 64, device="cuda").to(BF16)
    kt, vt = torch.zeros(2, 2, 16, 64, dtype=BF16, device="cuda"), torch.zeros(2, 2, 16, 64, dtype=BF16, device="cuda")
    out = torch.zeros(2, dtype=I32, device="cuda")
    enl.enl_tail_append([k], [k], [kt], [vt], dev(np.array([[0, 1, 2], [16, 17, 18]], np.int32)), dev(np.array([4, 5], np.int32)), out)
    torch.cuda.synchronize()
    assert out.tolist() == [7, 8] and torch.equal(kt[:, :, :3], k.transpose(1, 2)) and torch.equal(vt, kt)


# ---- a run of them together ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("captured", [False, True])
def test_drafting_steps(captured):
    """Steps of a planner that drafts: tables, rotation, attention, accepted path, append, with nothing on the host but the launches; the
    tails that come out, and every step's attention, are those of the plain forms.  Captured: one graph, replayed."""
    model, batch, n_max, steps, layers = (8, 2, 64), 3, 6, 7, 2
    n_q, n_kv, d = model
    rng = np.random.default_rng(11)
    c = Case(model, [[40, 17], [5], []], [0, 0, 0], [n_max] * batch, n_max, layers=layers, pages=40, max_blocks=8)
    try:
        st = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
        kt, vt = ([torch.full((40, n_kv, 16, d), NAN, dtype=BF16, device="cuda") for _ in range(layers)] for _ in range(2))
        tail = dev(np.zeros(batch, np.int32))
        table = torch.full((batch, 8), -1, dtype=I32, device="cuda")
        n_blocks, free, n_free = dev(np.zeros(batch, np.int32)), dev(rng.permutation(40).astype(np.int32)), dev(np.array([40], np.int32))
        parent = dev(np.stack([[-1, 0, 0, 1, 2, 2]] * batch).astype(np.int32))
        base = dev(np.array([100, 0, 7], np.int32))
        slots, pos, acc = (torch.zeros(batch, n_max, dtype=I32, device="cuda") for _ in range(3))
        mask = torch.zeros(batch, n_max, dtype=torch.int64, device="cuda")
        n_acc, nxt = (torch.zeros(batch, dtype=I32, device="cuda") for _ in range(2))
        token, target = (torch.zeros(batch, n_max, dtype=I32, device="cuda") for _ in range(2))
        raw = [[torch.zeros(batch, n_max, h, d, dtype=BF16, device="cuda") for h in (n_q, n_kv, n_kv)] for _ in range(layers)]
        qkv = [[torch.zeros_like(x) for x in r] for r in raw]
        outs = [torch.zeros(batch, n_max, n_q, d, dtype=BF16, device="cuda") for _ in range(layers)]

        def step():
            enl.enl_tail_tables(tail, table, n_blocks, free, n_free, slots, pos, mask, parent=parent, pos_base=base, stream=st())
            for l in range(layers):
                for x, y in zip(qkv[l], raw[l]):
                    x.copy_(y)
                for x in qkv[l][:2]:
                    enl.enl_rope_rotate(x.view(batch * n_max, -1, d), positions=pos.view(-1), stream=st())
                enl.enl_attend_tree(c.cache, l, c.sel, *qkv[l], kt[l], vt[l], table, tail, outs[l], mask=mask, cu_sel=c.cu_sel, stream=st())
            enl.enl_tree_accept(parent, token, target, acc, n_acc, nxt, stream=st())
            enl.enl_tail_append([x[1] for x in qkv], [x[2] for x in qkv], kt, vt, slots, tail, tail, accept=acc, n_accept=n_acc, stream=st())

        graph = None
        if captured:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                step()
        grown = [[([], []) for _ in range(batch)] for _ in range(layers)]
        see = [ref.ancestors([-1, 0, 0, 1, 2, 2], n_max)] * batch
        for i in range(steps):
            g = torch.Generator(device="cuda").manual_seed(i)
            for r in raw:
                for x in r:
                    x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
            tok, tgt = rng.integers(0, 2, (batch, n_max)).astype(np.int32), rng.integers(0, 2, (batch, n_max)).astype(np.int32)
            token.copy_(dev(tok))
            target.copy_(dev(tgt))
            before = tail.cpu().numpy().copy()
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            want_acc, want_n, want_next = ref.accept(np.full(batch, n_max), parent.cpu().numpy(), tok, tgt, None, n_max)
            assert np.array_equal(acc.cpu().numpy(), want_acc) and np.array_equal(nxt.cpu().numpy(), want_next)
            assert np.array_equal(tail.cpu().numpy(), before + want_n)
            want_pos = np.array([100, 0, 7])[:, None] + before[:, None] + np.array([0, 1, 1, 2, 2, 2])
            assert np.array_equal(pos.cpu().numpy(), want_pos)
            for l in range(layers):
                for b in range(batch):
                    gk, gv = grown[l][b]
                    parts = [[f64(x[l][j]) for j in range(c.cu_sel[b], c.cu_sel[b + 1])] + [r[None] for r in own] + [f64(new[b])]
                             for x, own, new in ((c.k_group, gk, qkv[l][1]), (c.v_group, gv, qkv[l][2]))]
                    k, v = np.concatenate(parts[0]), np.concatenate(parts[1])
                    full = np.concatenate([np.ones((n_max, len(k) - n_max), bool), see[b]], 1)
                    want, tol = ref.attend(f64(qkv[l][0][b]), k, v, full)
                    assert (np.abs(f64(outs[l][b]) - want) <= tol).all()
                    for a in want_acc[b, :want_n[b]]:
                        gk.append(f64(qkv[l][1][b, a]))
                        gv.append(f64(qkv[l][2][b, a]))
        del graph
    finally:
        c.close()


# ---- what the binding looks at ---------------------------------------------------------------------------------------------------------
def test_binding_checks_types_shapes_and_layouts():
    c = Case((8, 2, 64), [[20]], [10], [4], 4)
    try:
        good = dict(q=c.q, k=c.k, v=c.v, k_tail=c.k_tail, v_tail=c.v_tail, d_table=c.d_table, d_tails=c.d_tails, out=c.out, mask=c.mask)
        for name, bad in (("q", c.q[:, :, :4].contiguous()), ("q", c.q.float()), ("k", c.k[:, :3].contiguous()), ("v", c.v.transpose(2, 3)),
                          ("k_tail", c.k_tail[:, :, :8].contiguous()), ("v_tail", c.v_tail[1:].contiguous()), ("d_table", c.d_table.long()),
                          ("d_tails", c.d_tails.repeat(2)), ("out", c.out[:, :2].contiguous()), ("mask", c.mask.to(I32)), ("mask", c.mask.cpu()),
                          ("out", c.out.cpu()), ("q", None)):
            setattr(c, name, bad)
            with pytest.raises(ValueError):
                c.call()
            setattr(c, name, good[name])
        with pytest.raises(ValueError):
            c.call(cu_sel=np.array([0, 1, 1], np.int32))
        # tensors that gradients are kept for, and parameters, are tensors like others
        c.q, c.k = torch.nn.Parameter(c.q), c.k.clone().requires_grad_()
        c.call()
        c.q, c.k = c.q.detach(), c.k.detach()
        c.check()
    finally:
        c.close()
