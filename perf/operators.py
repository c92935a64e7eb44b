"""Verifying drafted tokens over the selected groups and a request's growing tail, as cases that can be timed.

While a planner answers, every episode (request) has a tail of its own behind the selected groups: instruction, trajectory and
the tokens answered so far, in pages of 16 rows that a block table names.  A step drafts a tree of up to 64 tokens per request
and goes through four operators:
  tables   block tables grown from a shared list of free pages, slots and positions of the new rows, ancestor masks of the tree
  attend   every drafted token over the selected groups, the tail and its ancestors in the tree
  accept   the path of drafted tokens that the model would have written itself
  append   the accepted rows' K and V, every layer, into the tail
Lengths live on the device throughout.  Scores have a standard deviation of about 1.5 before the softmax.
"""
import math

import numpy as np
import torch

own = False

BF16, I32 = torch.bfloat16, torch.int32
PAGE = 16                                                     # rows of a page
MODEL = dict(q_heads=32, kv_heads=8, head_dim=128)            # the planner model of the benchmark configurations
SMALL = dict(q_heads=8, kv_heads=2, head_dim=64)              # and the small one
SCORE_STD = 1.5


def listed():
    return [
        # the smallest verification: a small model, four short groups, an instruction, eight drafted tokens
        dict(SMALL, name="attend_tiny", kind="attend", shapes=10, batch=1, sel=4, len_lo=32, len_hi=32, tail_lo=64, tail_hi=64, nodes=8),
        # an ordinary step of a planner that drafts: the selected part of the map, 512 prompt tokens and some answered ones
        dict(MODEL, name="attend_planner", kind="attend", shapes=11, batch=1, sel=24, len_lo=40, len_hi=120, tail_lo=530, tail_hi=530, nodes=16),
        # one token, nothing drafted, over a large part of the map: the decoding form
        dict(MODEL, name="attend_token", kind="attend", shapes=12, batch=1, sel=96, len_lo=256, len_hi=426, tail_lo=64, tail_hi=64, nodes=1),
        # a drafted tree over the same
        dict(MODEL, name="attend_long", kind="attend", shapes=12, batch=1, sel=96, len_lo=256, len_hi=426, tail_lo=64, tail_hi=64, nodes=32),
        # the widest tree: two tiles of query rows per kv head
        dict(MODEL, name="attend_wide", kind="attend", shapes=13, batch=1, sel=64, len_lo=20, len_hi=200, tail_lo=1061, tail_hi=1061, nodes=64),
        # sixteen robots planned for at once, tails and trees of different sizes
        dict(MODEL, name="attend_batch", kind="attend", shapes=14, batch=16, sel=32, len_lo=40, len_hi=160, tail_lo=256, tail_hi=768, nodes=24),
        # tables of one request's step, and of a server's worth of requests
        dict(name="tables_step", kind="tables", shapes=15, batch=1, nodes=16, tail_lo=530, tail_hi=530, blocks=64),
        dict(name="tables_server", kind="tables", shapes=16, batch=512, nodes=64, tail_lo=1, tail_hi=1500, blocks=128),
        # the accepted path of one tree, and of a server's worth
        dict(name="accept_step", kind="accept", shapes=17, batch=1, nodes=16),
        dict(name="accept_server", kind="accept", shapes=18, batch=512, nodes=64),
        # the accepted rows of one tree in the 40 layers of the planner model, and whole prompts of sixteen requests
        dict(MODEL, name="append_step", kind="append", shapes=19, batch=1, nodes=16, layers=40, tail_lo=530, tail_hi=530, path=True),
        dict(MODEL, name="append_prompts", kind="append", shapes=20, batch=16, nodes=512, layers=16, tail_lo=0, tail_hi=0, path=False),
    ]


# ---- more cases of the same ranges ------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = rng.choice([(32, 8, 128)] * 4 + [(8, 2, 64), (16, 2, 128), (8, 8, 64), (8, 8, 128), (32, 2, 128), (16, 8, 64)])
    model = dict(q_heads=heads[0], kv_heads=heads[1], head_dim=heads[2])
    kind = rng.choice(["attend"] * 6 + ["tables", "accept", "append", "append"])
    shapes = rng.randrange(1 << 20)
    if kind == "attend":
        lo = _log(rng, 8, 160)
        tail = _log(rng, 1, 1200)
        case = dict(model, kind=kind, shapes=shapes, batch=1 if rng.random() < 0.5 else rng.randint(2, 32), sel=_log(rng, 1, 128), len_lo=lo,
                    len_hi=int(lo * rng.uniform(1.1, 4.0)) + 1, tail_lo=tail // 3, tail_hi=tail, nodes=_log(rng, 1, 64))
        while work(case)["bytes"] > 2.2e8 or work(case)["flops"] > 2.2e10:
            if case["batch"] > 1:
                case["batch"] = (case["batch"] + 1) // 2
            elif case["sel"] > 1:
                case["sel"] = (case["sel"] + 1) // 2
            else:
                case["nodes"] = (case["nodes"] + 1) // 2
        return case
    if kind == "tables":
        tail = _log(rng, 8, 1500)
        return dict(kind=kind, shapes=shapes, batch=_log(rng, 1, 512), nodes=_log(rng, 1, 64), tail_lo=tail // 4, tail_hi=tail, blocks=128)
    if kind == "accept":
        return dict(kind=kind, shapes=shapes, batch=_log(rng, 1, 512), nodes=_log(rng, 1, 64))
    path = rng.random() < 0.5
    tail = _log(rng, 1, 800)
    case = dict(model, kind=kind, shapes=shapes, batch=_log(rng, 1, 16), nodes=_log(rng, 1, 64) if path else _log(rng, 16, 600),
                layers=_log(rng, 1, 40), tail_lo=tail // 2, tail_hi=tail, path=path)
    while work(case)["bytes"] > 1e9:
        case["layers"] = (case["layers"] + 1) // 2
        case["batch"] = (case["batch"] + 1) // 2
    return case


# ---- shapes: lengths, trees and pages follow from the case alone ---------------------------------------------------
def _rng(case):
    return np.random.default_rng([case["shapes"], case["batch"], case["nodes"]])


def _trees(rng, batch, nodes):
    """Nodes of every request (the first request has all), and parents: -1 for the first node, else a node before, mostly a recent one."""
    n_new = rng.integers(1, nodes + 1, batch)
    n_new[0] = nodes
    back = 1 + np.minimum(rng.geometric(0.4, (batch, nodes)) - 1, np.maximum(np.arange(nodes) - 1, 0))
    parent = np.where(np.arange(nodes) > 0, np.arange(nodes) - back, -1)
    return n_new.astype(np.int32), np.where(np.arange(nodes) < n_new[:, None], parent, -1).astype(np.int32)


def _tails(rng, case):
    return rng.integers(case["tail_lo"], case["tail_hi"] + 1, case["batch"]).astype(np.int32)


def _attend_shapes(case):
    rng = _rng(case)
    n_new, parent = _trees(rng, case["batch"], case["nodes"])
    tail = _tails(rng, case)
    lens = rng.integers(case["len_lo"], case["len_hi"] + 1, (case["batch"], case["sel"])).astype(np.int64)
    return rng, n_new, parent, tail, lens


def _ancestors(parent):
    """[batch][nodes][nodes] truth values on the host: the column is the row's ancestor or itself."""
    batch, nodes = parent.shape
    anc = np.zeros((batch, nodes, nodes), bool)
    for i in range(nodes):
        anc[:, i, i] = True
        has = np.nonzero(parent[:, i] >= 0)[0]
        anc[has, i] |= anc[has, parent[has, i]]
    return anc


def _bits(anc):
    nodes = anc.shape[-1]
    words = (anc.astype(np.uint64) << np.arange(nodes, dtype=np.uint64)).sum(-1, dtype=np.uint64)
    return words.view(np.int64)


def _blocks(case, tail, n_new):
    return -(-(tail + n_new) // PAGE)


def work(case):
    b = case["batch"]
    if case["kind"] == "tables":
        rng = _rng(case)
        n_new, _ = _trees(rng, b, case["nodes"])
        tail = _tails(rng, case)
        rows = b * case["nodes"]
        # lengths, counts, bases and block counts; parents in, slots, positions and masks out; the tables that name the new rows' pages
        return {"bytes": 16 * b + rows * (4 + 4 + 4 + 8) + 4 * int(_blocks(case, tail, n_new).sum()), "flops": 0}
    if case["kind"] == "accept":
        rows = b * case["nodes"]
        return {"bytes": rows * (4 + 4 + 4 + 4) + 12 * b, "flops": 0}
    row = case["kv_heads"] * case["head_dim"] * 4                # K and V
    if case["kind"] == "append":
        rng = _rng(case)
        rows = sum(len(x) for x in _paths(rng, case)) if case["path"] else b * case["nodes"]
        return {"bytes": 2 * rows * row * case["layers"] + 8 * rows + 12 * b, "flops": 0}
    _, n_new, parent, tail, lens = _attend_shapes(case)
    keys = lens.sum(1) + tail
    seen = _ancestors(parent).sum(2)
    pairs = int((keys * n_new).sum()) + int((seen * (np.arange(case["nodes"]) < n_new[:, None])).sum())
    q_row = case["q_heads"] * case["head_dim"] * 2
    return {"bytes": int((keys + n_new).sum()) * row + int(n_new.sum()) * (2 * q_row + 8), "flops": 4 * case["q_heads"] * case["head_dim"] * pairs}


def _paths(rng, case):
    """Accepted nodes of every request: the way from a root to some node."""
    n_new, parent = _trees(rng, case["batch"], case["nodes"])
    found = []
    for b in range(case["batch"]):
        at, path = int(rng.integers(0, n_new[b])), []
        while at >= 0:
            path.append(at)
            at = int(parent[b, at])
        found.append(path[::-1])
    return found


# ---- inputs ----------------------------------------------------------------------------------------------------
class _Cache:
    """A cache of the library with every group stored, freed with the state that holds it."""

    def __init__(self, case, k_pool, v_pool, lens):
        from paper_2510_18546_b200 import enl
        self.enl = enl
        flat = lens.reshape(-1)
        self.handle = enl.enl_cache_create(1, case["q_heads"], case["kv_heads"], case["head_dim"], max_groups=flat.size, max_tokens=int(flat.sum()),
                                           device=torch.cuda.current_device(), max_batch=case["batch"])
        at = 0
        for g, n in enumerate(flat):
            enl.enl_group_store(self.handle, g, 0, k_pool[at:at + n], v_pool[at:at + n], stream=torch.cuda.current_stream().cuda_stream)
            at += int(n)

    def __del__(self):
        self.enl.enl_cache_free(self.handle)


def _dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)


def _paged(rng, blocks, max_blocks):
    """Pages in no order: a block table (-1 behind a request's blocks) and the pages that are left."""
    total = int(blocks.sum())
    order = rng.permutation(total + 8).astype(np.int32)
    table = np.full((len(blocks), max_blocks), -1, np.int32)
    ends = np.cumsum(blocks)
    for b, n in enumerate(blocks):
        table[b, :n] = order[ends[b] - n:ends[b]]
    return table, order[total:]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"kind": case["kind"], "case": case}
    batch, nodes = case["batch"], case["nodes"]

    def values(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=BF16) * std)

    if case["kind"] == "tables":
        rng = _rng(case)
        n_new, parent = _trees(rng, batch, nodes)
        tail = np.random.default_rng(seed).integers(case["tail_lo"], case["tail_hi"] + 1, batch).astype(np.int32)
        have = -(-tail // PAGE)                                  # what the committed rows lie in; the new rows may need more
        table, _ = _paged(np.random.default_rng(seed + 1), have, case["blocks"])
        spare = int((_blocks(case, tail, n_new) - have).sum()) + 5
        free = np.random.default_rng(seed + 2).permutation(np.arange(int(have.sum()) + 8, int(have.sum()) + 8 + spare)).astype(np.int32)
        s.update(tail=_dev(tail), n_new=_dev(n_new), parent=_dev(parent), base=_dev(np.random.default_rng(seed + 3).integers(0, 5000, batch).astype(np.int32)),
                 table=_dev(table), n_blocks=_dev(have.astype(np.int32)), free=_dev(free), n_free=_dev(np.asarray([spare], np.int32)),
                 slots=torch.full((batch, nodes), -1, dtype=I32, device="cuda"), positions=torch.zeros(batch, nodes, dtype=I32, device="cuda"),
                 mask=torch.zeros(batch, nodes, dtype=torch.int64, device="cuda"))
        return s
    if case["kind"] == "accept":
        rng = _rng(case)
        n_new, parent = _trees(rng, batch, nodes)
        vals = np.random.default_rng(seed)
        token = vals.integers(0, 32000, (batch, nodes)).astype(np.int32)
        target = vals.integers(0, 32000, (batch, nodes)).astype(np.int32)
        # a draft is right about three times in four
        right = (vals.random((batch, nodes)) < 0.75) & (parent >= 0)
        rows, cols = np.nonzero(right)
        target[rows, parent[rows, cols]] = token[rows, cols]
        s.update(n_new=_dev(n_new), parent=_dev(parent), token=_dev(token), target=_dev(target),
                 accept=torch.full((batch, nodes), -1, dtype=I32, device="cuda"), n_accept=torch.zeros(batch, dtype=I32, device="cuda"),
                 next=torch.zeros(batch, dtype=I32, device="cuda"))
        return s
    h, d = case["kv_heads"], case["head_dim"]
    if case["kind"] == "append":
        rng = _rng(case)
        if case["path"]:
            paths = _paths(rng, case)
            accept = np.full((batch, nodes), -1, np.int32)
            for b, p in enumerate(paths):
                accept[b, :len(p)] = p
            s.update(accept=_dev(accept), n_accept=_dev(np.asarray([len(p) for p in paths], np.int32)))
        else:
            s.update(accept=None, n_accept=torch.full((batch,), nodes, dtype=I32, device="cuda"))
        tail = _tails(rng, case)
        blocks = -(-(tail + nodes) // PAGE)
        table, _ = _paged(rng, blocks, int(blocks.max()))
        rows = tail[:, None] + np.arange(nodes)
        slots = np.take_along_axis(table, rows // PAGE, 1) * PAGE + rows % PAGE
        pages = int(blocks.sum()) + 8
        layers = case["layers"]
        s.update(k=values(layers, batch, nodes, h, d), v=values(layers, batch, nodes, h, d), k_tail=torch.zeros(layers, pages, h, PAGE, d, dtype=BF16, device="cuda"),
                 v_tail=torch.zeros(layers, pages, h, PAGE, d, dtype=BF16, device="cuda"), slots=_dev(slots, I32), tail=_dev(tail),
                 tail_out=torch.zeros(batch, dtype=I32, device="cuda"))
        s["layers"] = [list(s[x].unbind(0)) for x in ("k", "v", "k_tail", "v_tail")]
        return s
    rng, n_new, parent, tail, lens = _attend_shapes(case)
    total = int(lens.sum())
    blocks = -(-tail // PAGE)
    table, _ = _paged(rng, blocks, max(int(blocks.max()), 1) + 4)
    pages = int(blocks.sum()) + 8
    # the selected groups' rows, request by request: row numbers of the pool, -1 behind the last
    n_keys = lens.sum(1)
    keys = np.where(np.arange(n_keys.max()) < n_keys[:, None], np.arange(n_keys.max()) + (np.cumsum(n_keys) - n_keys)[:, None], -1)
    s.update(k_pool=values(total, h, d), v_pool=values(total, h, d), keys=_dev(keys), k_tail=values(pages, h, PAGE, d), v_tail=values(pages, h, PAGE, d),
             table=_dev(table), tail=_dev(tail), n_new=_dev(n_new), mask=_dev(_bits(_ancestors(parent))),
             q=values(batch, nodes, case["q_heads"], d, std=SCORE_STD), k=values(batch, nodes, h, d), v=values(batch, nodes, h, d),
             out=torch.zeros(batch, nodes, case["q_heads"], d, dtype=BF16, device="cuda"))
    if own:
        s["cache"] = _Cache(case, s["k_pool"], s["v_pool"], lens)
        s["sel"] = np.arange(lens.size, dtype=np.int32)
        s["cu_sel"] = np.arange(0, lens.size + 1, lens.shape[1], dtype=np.int32)
    return s


# ---- one pass --------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)[s["kind"]](s)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _own_tables(s):
    from paper_2510_18546_b200 import enl
    enl.enl_tail_tables(s["tail"], s["table"], s["n_blocks"], s["free"], s["n_free"], s["slots"], s["positions"], s["mask"], n_new=s["n_new"],
                        parent=s["parent"], pos_base=s["base"], stream=_stream())
    return {k: s[k] for k in ("table", "n_blocks", "n_free", "slots", "positions", "mask")}


def _own_attend(s):
    from paper_2510_18546_b200 import enl
    enl.enl_attend_tree(s["cache"].handle, 0, s["sel"], s["q"], s["k"], s["v"], s["k_tail"], s["v_tail"], s["table"], s["tail"], s["out"],
                        n_new=s["n_new"], mask=s["mask"], cu_sel=s["cu_sel"], stream=_stream())
    return s["out"]


def _own_accept(s):
    from paper_2510_18546_b200 import enl
    enl.enl_tree_accept(s["parent"], s["token"], s["target"], s["accept"], s["n_accept"], s["next"], n_new=s["n_new"], stream=_stream())
    return {k: s[k] for k in ("accept", "n_accept", "next")}


def _own_append(s):
    from paper_2510_18546_b200 import enl
    enl.enl_tail_append(*s["layers"], s["slots"], s["tail"], s["tail_out"], accept=s["accept"], n_accept=s["n_accept"], stream=_stream())
    return {k: s[k] for k in ("k_tail", "v_tail", "tail_out")}


def _closure(parent, nodes):
    """[batch][nodes][nodes] truth values: the column is the row's ancestor or itself (products of the one-step relation)."""
    at = torch.arange(nodes, device=parent.device)
    a = ((parent[:, :, None] == at) | (at[:, None] == at)).float()
    a = ((a @ a) > 0).float()
    a = ((a @ a) > 0).float()
    a = ((a @ a) > 0).float()
    a = ((a @ a) > 0).float()
    a = ((a @ a) > 0).float()
    return (a @ a) > 0


def _plain_tables(s):
    tail, n_new, parent, table, free = s["tail"].long(), s["n_new"].long(), s["parent"].long(), s["table"], s["free"].long()
    batch, nodes = parent.shape
    at = torch.arange(nodes, device="cuda")
    live = at < n_new[:, None]
    have, want = s["n_blocks"].long(), (tail + n_new + PAGE - 1) // PAGE
    take = (want - have).clamp_min(0)
    first = take.cumsum(0) - take
    block = torch.arange(table.shape[1], device="cuda")
    new = (block >= have[:, None]) & (block < want[:, None])
    place = s["n_free"].long() - 1 - (first[:, None] + block - have[:, None])
    table = torch.where(new, free[place.clamp(0, free.numel() - 1)], table.long())
    rows = tail[:, None] + at
    slots = torch.gather(table, 1, (rows // PAGE).clamp_max(table.shape[1] - 1)) * PAGE + rows % PAGE
    anc = _closure(parent, nodes) & live[:, :, None]
    bits = torch.where(anc, torch.ones((), dtype=torch.int64, device="cuda") << at, 0).sum(2)
    depth = anc.sum(2) - 1
    positions = s["base"].long()[:, None] + tail[:, None] + depth
    return {"table": table.to(I32), "n_blocks": torch.maximum(have, want).to(I32), "n_free": (s["n_free"] - take.sum()).to(I32),
            "slots": torch.where(live, slots, -1).to(I32), "positions": torch.where(live, positions, 0).to(I32), "mask": bits}


def _plain_attend(s):
    q, k_new, v_new, tail, table = s["q"].float(), s["k"].float(), s["v"].float(), s["tail"].long(), s["table"].long()
    batch, nodes, q_heads, d = q.shape
    h = k_new.shape[2]
    at = torch.arange(nodes, device="cuda")
    row = torch.arange(table.shape[1] * PAGE, device="cuda")
    page = table.clamp_min(0)[:, row // PAGE]                                               # [batch][rows]

    def keys_of(pool, pages, new):
        cached = pool[s["keys"].clamp_min(0)].float()                                       # [batch][keys][h][d]
        own_rows = pages[page, :, (row % PAGE).expand(batch, -1)].float()
        return torch.cat([cached, own_rows, new], 1)

    k, v = keys_of(s["k_pool"], s["k_tail"], k_new), keys_of(s["v_pool"], s["v_tail"], v_new)
    tree = ((s["mask"][:, :, None] >> at) & 1).bool() & (at < s["n_new"].long()[:, None])[:, None, :]
    shared = torch.cat([s["keys"] >= 0, row < tail[:, None]], 1)
    seen = torch.cat([shared[:, None, :].expand(-1, nodes, -1), tree], 2)                   # [batch][nodes][keys]
    score = torch.einsum("bnhrd,bshd->bhrns", q.view(batch, nodes, h, q_heads // h, d), k) / math.sqrt(d)
    score = torch.where(seen[:, None, None], score, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = torch.einsum("bhrns,bshd->bnhrd", p / p.sum(-1, keepdim=True), v).reshape(batch, nodes, q_heads, d)
    return torch.where((at < s["n_new"].long()[:, None])[:, :, None, None], o, 0).to(BF16)


def _plain_accept(s):
    parent, token, target, n_new = s["parent"].long(), s["token"], s["target"], s["n_new"].long()
    batch, nodes = parent.shape
    at = torch.arange(nodes, device="cuda")
    live = at < n_new[:, None]
    said = torch.gather(target, 1, parent.clamp_min(0))                                     # what the model put behind the parent
    hit = torch.where(parent < 0, at == 0, said == token) & live
    twin = (parent[:, :, None] == parent[:, None, :]) & hit[:, None, :] & (at[:, None] > at)      # an equal sibling with a lower index
    hit = hit & ~twin.any(2)
    anc = _closure(parent, nodes)
    held = (~anc | hit[:, None, :]).all(2) & live
    n = held.sum(1)
    order = torch.where(held, at, nodes).sort(1).values
    accept = torch.where(order < nodes, order, -1)
    last = torch.where(held, at, -1).amax(1)
    nxt = torch.where(last >= 0, torch.gather(target, 1, last.clamp_min(0)[:, None])[:, 0], -1)
    return {"accept": accept.to(I32), "n_accept": n.to(I32), "next": nxt.to(I32)}


def _plain_append(s):
    layers, batch, nodes, h, d = s["k"].shape
    at = torch.arange(nodes, device="cuda")
    source = at.expand(batch, -1) if s["accept"] is None else s["accept"].long()
    b, i = torch.nonzero(at < s["n_accept"].long()[:, None], as_tuple=True)
    slot, row = s["slots"].long()[b, i], source[b, i]
    s["k_tail"][:, slot // PAGE, :, slot % PAGE] = s["k"][:, b, row].transpose(0, 1)
    s["v_tail"][:, slot // PAGE, :, slot % PAGE] = s["v"][:, b, row].transpose(0, 1)
    return {"k_tail": s["k_tail"], "v_tail": s["v_tail"], "tail_out": s["tail"] + s["n_accept"]}


_run_plain = {"tables": _plain_tables, "attend": _plain_attend, "accept": _plain_accept, "append": _plain_append}
_run_own = {"tables": _own_tables, "attend": _own_attend, "accept": _own_accept, "append": _own_append}


# ---- the same from the definitions, in 64 bits, request by request ---------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"tables": _exact_tables, "attend": _exact_attend, "accept": _exact_accept, "append": _exact_append}[case["kind"]](s)


def _host(t):
    return t.cpu().numpy().copy()


def _exact_tables(s):
    tail, n_new, parent, base = (_host(s[k]) for k in ("tail", "n_new", "parent", "base"))
    table, n_blocks, free, n_free = (_host(s[k]) for k in ("table", "n_blocks", "free", "n_free"))
    batch, nodes = parent.shape
    slots, positions, mask = np.full((batch, nodes), -1, np.int32), np.zeros((batch, nodes), np.int32), np.zeros((batch, nodes), np.uint64)
    for b in range(batch):
        while n_blocks[b] * PAGE < tail[b] + n_new[b]:
            n_free[0] -= 1
            table[b, n_blocks[b]] = free[n_free[0]]
            n_blocks[b] += 1
        depth = {-1: -1}
        for i in range(n_new[b]):
            p = int(parent[b, i])
            depth[i] = depth[p] + 1
            r = int(tail[b]) + i
            slots[b, i] = table[b, r // PAGE] * PAGE + r % PAGE
            positions[b, i] = base[b] + tail[b] + depth[i]
            mask[b, i] = np.uint64(1 << i) | (mask[b, p] if p >= 0 else np.uint64(0))
    return {"table": _dev(table), "n_blocks": _dev(n_blocks), "n_free": _dev(n_free), "slots": _dev(slots), "positions": _dev(positions),
            "mask": _dev(mask.view(np.int64))}


def _exact_attend(s):
    case = s["case"]
    _, n_new, parent, tail, lens = _attend_shapes(case)
    table, d = _host(s["table"]), case["head_dim"]
    rep = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    first = 0
    for b in range(case["batch"]):
        n, m = int(lens[b].sum()), int(n_new[b])
        pages = [int(p) for p in table[b, :-(-int(tail[b]) // PAGE)]]
        see = torch.zeros(m, m, dtype=torch.bool)
        for i in range(m):
            at = i
            while at >= 0:
                see[i, at] = True
                at = int(parent[b, at])
        hidden = torch.cat([torch.zeros(m, n + int(tail[b]), dtype=torch.bool), ~see], 1).cuda()
        for h in range(case["kv_heads"]):
            rows = []
            for pool, paged, new in (("k_pool", "k_tail", "k"), ("v_pool", "v_tail", "v")):
                grown = s[paged][pages, h].reshape(-1, d)[:int(tail[b])]
                rows.append(torch.cat([s[pool][first:first + n, h], grown, s[new][b, :m, h]]).double())
            for r in range(rep):
                w = (s["q"][b, :m, h * rep + r].double() @ rows[0].T * d ** -0.5).masked_fill(hidden, -math.inf)
                out[b, :m, h * rep + r] = torch.softmax(w, 1) @ rows[1]
        first += n
    return out


def _exact_accept(s):
    n_new, parent, token, target = (_host(s[k]) for k in ("n_new", "parent", "token", "target"))
    batch, nodes = parent.shape
    accept, n_accept, nxt = np.full((batch, nodes), -1, np.int32), np.zeros(batch, np.int32), np.full(batch, -1, np.int32)
    for b in range(batch):
        at = 0 if n_new[b] > 0 else -1
        while at >= 0:
            accept[b, n_accept[b]] = at
            n_accept[b] += 1
            nxt[b] = target[b, at]
            at = next((i for i in range(n_new[b]) if parent[b, i] == at and token[b, i] == target[b, at]), -1)
    return {"accept": _dev(accept), "n_accept": _dev(n_accept), "next": _dev(nxt)}


def _exact_append(s):
    k_tail, v_tail = s["k_tail"].double(), s["v_tail"].double()
    slots, n = _host(s["slots"]), _host(s["n_accept"])
    accept = _host(s["accept"]) if s["accept"] is not None else None
    for b in range(len(n)):
        rows = list(range(n[b])) if accept is None else accept[b, :n[b]].tolist()
        to = slots[b, :n[b]]
        page, within = torch.from_numpy(to // PAGE).long().cuda(), torch.from_numpy(to % PAGE).long().cuda()
        for l in range(k_tail.shape[0]):
            k_tail[l][page, :, within] = s["k"][l, b, rows].double()
            v_tail[l][page, :, within] = s["v"][l, b, rows].double()
    return {"k_tail": k_tail, "v_tail": v_tail, "tail_out": s["tail"] + s["n_accept"]}
