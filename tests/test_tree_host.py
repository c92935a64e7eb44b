"""Drafted trees and tails without a GPU: what the calls refuse, what the binding refuses, and the host side of enl_attend_tree on a CUDA
runtime that has no device (fake_tree.cpp)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2510_18546_b200 import build as enl_build
from paper_2510_18546_b200 import enl
from tests import tree_reference as ref

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCES = ["enl_host.cu", "enl_static_scratch.cu", "enl_decode_cluster_sm100.cu", "enl_tree.cu"]
BASE = 1 << 20                                                   # of pointers that are never followed


@pytest.fixture(scope="module", autouse=True)
def _built():
    enl_build.build_library()


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("tree") / "libtree.so")
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=compute_100a", "-std=c++17", "-O1",
                    "-cudart", "none", "-Xcompiler", "-fPIC", "-shared", "-Xlinker", "-Bsymbolic", "-t", "4", "-o", path,
                    os.path.join(HERE, "fake_tree.cpp")] + [os.path.join(enl_build.CSRC, s) for s in SOURCES], check=True)
    return path


@pytest.fixture
def host(built, tmp_path):
    path = str(tmp_path / "libtree.so")
    with open(built, "rb") as f, open(path, "wb") as g:
        g.write(f.read())
    L = ctypes.CDLL(path)
    L.fake_capture.argtypes = [ctypes.c_ulonglong]
    return L


class Host:
    """A cache on the runtime without a device: four groups of 40 rows, two layers."""

    def __init__(self, L, **kw):
        d = enl.CacheDesc(2, 32, 8, 128, 0, 8, 4096, enl.ENL_BF16, 0, 4, 0, 0)
        for k, v in kw.items():
            setattr(d, k, v)
        self.L, self.h = L, ctypes.c_void_p()
        assert L.enl_cache_create(ctypes.byref(d), ctypes.byref(self.h)) == enl.ENL_OK
        for g in range(4):
            for layer in range(2):
                self.store(g, layer)
        L.fake_clear()

    def store(self, g, layer, n=40):
        assert self.L.enl_group_store(self.h, g, layer, n, ctypes.c_void_p(BASE), ctypes.c_void_p(BASE), enl.ENL_REPLACE, None) == enl.ENL_OK

    def args(self, sel=(0, 1, 2), **kw):
        a = enl.AttendTreeArgs()
        a.held = np.asarray(sel, np.int32)
        a.layer, a.batch, a.n_max, a.sel_ids, a.n_sel, a.max_blocks, a.n_pages = 0, 1, 16, a.held.ctypes.data, len(sel), 32, 100
        for i, n in enumerate(("tail_len", "n_new", "mask", "block_table", "q", "k_new", "v_new", "k_tail", "v_tail", "out")):
            setattr(a, n, BASE * (i + 1))
        for k, v in kw.items():
            if isinstance(v, np.ndarray):
                a.keep = getattr(a, "keep", []) + [v]
                v = v.ctypes.data
            setattr(a, k, v)
        return a

    def call(self, *args, **kw):
        return self.L.enl_attend_tree(self.h, ctypes.byref(self.args(*args, **kw)), None)

    def attend(self):
        a = enl.AttendArgs()
        a.batch, a.n_q, a.n_new, a.n_sel = 1, 300, 300, 3
        a.held = np.arange(3, dtype=np.int32)
        a.sel_ids = a.held.ctypes.data
        a.q = a.k_new = a.v_new = a.out = BASE
        return self.L.enl_attend(self.h, ctypes.byref(a), None)

    def kinds(self):
        got = "".join(chr(self.L.fake_kind(i)) for i in range(self.L.fake_launches()))
        self.L.fake_clear()
        return got


INVALID = [dict(layer=2), dict(layer=-1), dict(batch=0), dict(batch=5), dict(n_max=0), dict(n_sel=-1), dict(max_blocks=0), dict(n_pages=0), dict(sel_ids=None),
           dict(batch=2), dict(batch=2, cu_sel=np.array([0, 2, 4], np.int32)), dict(batch=2, cu_sel=np.array([1, 2, 3], np.int32)),
           dict(batch=3, cu_sel=np.array([0, 2, 1, 3], np.int32)), dict(sel=(0, 1, 1))] + \
          [dict([(n, None)]) for n in ("tail_len", "block_table", "q", "k_new", "v_new", "k_tail", "v_tail", "out")] + \
          [dict([(n, BASE + 8)]) for n in ("q", "k_new", "v_new", "k_tail", "v_tail", "out")] + \
          [dict([(n, BASE + 2)]) for n in ("tail_len", "block_table", "n_new")] + [dict(mask=BASE + 4)]


@pytest.mark.parametrize("kw", INVALID, ids=str)
def test_attend_tree_refuses(host, kw):
    c = Host(host)
    assert c.call(**kw) == enl.ENL_E_INVAL
    assert c.kinds() == ""
    assert c.call() == enl.ENL_OK                                # nothing was changed


def test_attend_tree_refuses_by_group_and_size(host):
    c = Host(host)
    for kw, code in ((dict(sel=(0, 5)), enl.ENL_E_NOGROUP), (dict(sel=(0, 8)), enl.ENL_E_NOGROUP), (dict(sel=(-1,)), enl.ENL_E_NOGROUP),
                     (dict(n_max=65), enl.ENL_E_LIMIT), (dict(n_pages=1 << 28), enl.ENL_E_LIMIT), (dict(max_blocks=1 << 27), enl.ENL_E_LIMIT)):
        assert c.call(**kw) == code, kw
    assert c.kinds() == ""
    assert host.enl_attend_tree(None, ctypes.byref(c.args()), None) == enl.ENL_E_INVAL
    assert host.enl_attend_tree(c.h, None, None) == enl.ENL_E_INVAL


def test_attend_tree_needs_a_device():
    cache = enl.enl_cache_create(1, 8, 2, 64, max_groups=2, max_tokens=64, device=enl.ENL_DEVICE_NONE)
    a = enl.AttendTreeArgs()
    assert enl.lib().enl_attend_tree(cache, ctypes.byref(a), None) == enl.ENL_E_CUDA
    enl.enl_cache_free(cache)


def test_evicted_groups_are_refused(host):
    c = Host(host)
    assert host.enl_tier_enable(c.h, ctypes.c_int64(4096)) == enl.ENL_OK
    assert host.enl_group_evict(c.h, 1, None) == enl.ENL_OK
    c.kinds()
    assert c.call() == enl.ENL_E_EVICTED and c.kinds() == ""
    assert c.call(sel=(0, 2)) == enl.ENL_OK


def test_plan_is_sent_once_and_again_when_something_changed(host):
    c = Host(host)
    assert c.call() == enl.ENL_OK and c.kinds() == "wtu"
    for layer in (0, 1, 1, 0):
        assert c.call(layer=layer) == enl.ENL_OK
    assert c.kinds() == "tu" * 4
    assert c.call(n_new=None, mask=None, n_pages=50) == enl.ENL_OK and c.kinds() == "tu"
    assert c.call(n_max=7) == enl.ENL_OK and c.call(max_blocks=40) == enl.ENL_OK and c.kinds() == "wtuwtu"    # what the splits go by
    assert c.call() == enl.ENL_OK and c.kinds() == "wtu"
    assert c.call(sel=(2, 1, 0)) == enl.ENL_OK and c.kinds() == "wtu"
    c.store(1, 0)
    c.kinds()
    assert c.call(sel=(2, 1, 0)) == enl.ENL_OK and c.kinds() == "wtu"
    c.store(1, 1, 50)                                             # another length in layer 1 only
    c.kinds()
    assert c.call(sel=(2, 1, 0)) == enl.ENL_OK and c.call(sel=(2, 1, 0), layer=1) == enl.ENL_OK
    assert c.kinds() == "wtu" + "wtu"
    cu = np.array([0, 1, 3], np.int32)
    assert c.call(sel=(2, 1, 0), batch=2, cu_sel=cu) == enl.ENL_OK and c.kinds() == "wtu"


def test_plans_of_the_two_attentions_are_kept_apart(host):
    c = Host(host)
    for _ in range(2):
        assert c.attend() == enl.ENL_OK
        assert c.kinds()[:2] == "wa"
        assert c.call() == enl.ENL_OK
        assert c.kinds() == "wtu"
    assert c.call() == enl.ENL_OK and c.kinds() == "tu"


def test_the_next_attention_need_not_wait_first(host):
    """Either attention leaves plan and pool behind as later ones may find them before the kernel before them has ended."""
    c = Host(host)
    assert c.attend() == enl.ENL_OK and host.fake_wait_first(1) == 1
    host.fake_clear()
    assert c.attend() == enl.ENL_OK and host.fake_wait_first(0) == 0
    c.store(3, 0)
    c.kinds()
    for first in (1, 0, 0):
        assert c.call(sel=(0, 1)) == enl.ENL_OK
        at = host.fake_launches() - 2
        assert host.fake_kind(at) == ord("t") and host.fake_wait_first(at) == first
    host.fake_clear()
    assert c.attend() == enl.ENL_OK                               # the plan is written anew: it waits
    assert host.fake_kind(0) == ord("w") and host.fake_wait_first(1) == 1


def test_plan_can_be_read_back(host):
    """The same stream as enl_attend's for the same list, and how it is split."""
    host.enl_plan_inspect.argtypes = enl.lib().enl_plan_inspect.argtypes

    def inspect(c):
        arr = [np.zeros(64, np.int32) for _ in range(4)]
        n = [ctypes.c_int32() for _ in range(4)]
        p = [x.ctypes.data_as(ctypes.c_void_p) for x in arr]
        assert host.enl_plan_inspect(c.h, 64, p[0], p[1], ctypes.byref(n[0]), 64, p[2], p[3], ctypes.byref(n[1]), ctypes.byref(n[2]), ctypes.byref(n[3])) == enl.ENL_OK
        return [x.tolist() for x in arr], [x.value for x in n]

    c = Host(host)
    assert c.attend() == enl.ENL_OK
    streams, (entries, _, _, _) = inspect(c)
    assert c.call() == enl.ENL_OK
    mine, (e, splits, items, kind) = inspect(c)
    assert mine[:2] == streams[:2] and mine[2][0] == streams[2][0] and mine[3][0] == streams[3][0] and e == entries
    assert splits == host.fake_splits() and items == host.fake_grid() and kind == 1
    assert c.call(sel=(0, 1, 2, 3), batch=2, cu_sel=np.array([0, 1, 4], np.int32)) == enl.ENL_OK
    mine, _ = inspect(c)
    assert mine[2][:2] == [0, 8] and mine[3][:2] == [1, 2]


def test_a_captured_call_takes_its_plan_along(host):
    c = Host(host)
    assert c.call() == enl.ENL_OK
    c.kinds()
    host.fake_capture(3)
    assert c.call() == enl.ENL_OK and c.call(layer=1) == enl.ENL_OK
    host.fake_capture(0)
    assert c.kinds() == "wtu" + "tu"
    assert c.call() == enl.ENL_OK and c.kinds() == "wtu"          # the graph may have run in between
    assert c.call() == enl.ENL_OK and c.kinds() == "wtu"


def test_refused_launches_are_reported(host):
    for kind in "twPe":
        c = Host(host)
        host.fake_fail(ord(kind))
        assert c.call() == enl.ENL_E_CUDA, kind
        host.fake_fail(0)
        assert c.call() == enl.ENL_OK, kind
    c = Host(host)
    host.fake_fail(ord("u"))
    assert c.call() == enl.ENL_E_CUDA


def test_plan_larger_than_its_buffers(host):
    c = Host(host, max_tokens=640, max_batch=64)
    batch = 40
    sel = np.tile(np.arange(4), batch).astype(np.int32)
    assert c.call(sel=sel, batch=batch, cu_sel=np.arange(0, 4 * batch + 1, 4, dtype=np.int32)) in (enl.ENL_OK, enl.ENL_E_NOMEM)
    assert c.call() == enl.ENL_OK


def test_grid_and_splits(host):
    """Parts until the multiprocessors have work, and none where the scratch buffer has no room for them or the stream is too short."""
    c = Host(host)
    # 9 cached pages, a table of 32, one page of nodes
    assert c.call() == enl.ENL_OK
    assert host.fake_grid() == 8 * host.fake_splits() <= 148 and 2 <= host.fake_splits() <= 11 and host.fake_box() == 16
    # 64 nodes are two tiles of rows
    assert c.call(n_max=64) == enl.ENL_OK
    assert host.fake_grid() == 16 * host.fake_splits() <= 148 and host.fake_splits() >= 2 and host.fake_box() == 32
    c.kinds()
    assert c.call(sel=(), max_blocks=1, n_max=1) == enl.ENL_OK and (host.fake_grid(), host.fake_splits()) == (8, 1) and c.kinds() == "t"        # an empty plan
    c = Host(host, scratch_bytes=100000)
    assert c.call() == enl.ENL_OK and (host.fake_grid(), host.fake_splits()) == (8, 1)
    slot = 128 * 129 * 4
    c = Host(host, scratch_bytes=24 * slot)
    assert c.call() == enl.ENL_OK and (host.fake_grid(), host.fake_splits()) == (24, 3)
    # two requests: the longer one is cut into more
    c = Host(host)
    assert c.call(sel=(0, 1, 2, 3), batch=2, cu_sel=np.array([0, 0, 4], np.int32)) == enl.ENL_OK
    assert host.fake_grid() <= 148 and host.fake_grid() % 8 == 0 and host.fake_splits() >= 2


@pytest.mark.parametrize("batch,lens,blocks,n_max,kv", [(16, (180, 230), 52, 24, 8), (16, (180, 230), 52, 64, 8), (3, (1100, 1500), 40, 16, 8), (40, (70, 140), 30, 8, 8),
                                                        (64, (40, 90), 20, 1, 8), (5, (600, 1000), 3, 33, 2)], ids=str)
def test_shares_of_several_requests(host, batch, lens, blocks, n_max, kv):
    """Every unit's parts meet from its beginning to its end and have slots and heads of their own, a run is about as long as any other,
    and CTAs find a place each."""
    rng = np.random.default_rng(batch)
    pages = rng.integers(lens[0], lens[1], batch)
    d = dict(max_groups=batch, max_tokens=int(pages.sum()) * 16 + 16 * batch, max_batch=64, n_q_heads=4 * kv, n_kv_heads=kv)
    c = Host.__new__(Host)
    desc = enl.CacheDesc(1, 32, 8, 128, 0, 8, 4096, enl.ENL_BF16, 0, 4, 0, 0)
    for k, v in d.items():
        setattr(desc, k, v)
    c.L, c.h = host, ctypes.c_void_p()
    assert host.enl_cache_create(ctypes.byref(desc), ctypes.byref(c.h)) == enl.ENL_OK
    for g in range(batch):
        c.store(g, 0, int(pages[g]) * 16)
    c.kinds()
    assert c.call(sel=np.arange(batch, dtype=np.int32), batch=batch, cu_sel=np.arange(batch + 1, dtype=np.int32), n_max=n_max, max_blocks=blocks) == enl.ENL_OK
    assert c.kinds()[0] == "p"                                    # a large plan: copied, so that it can be read here
    tiles = -(-n_max * 4 // 128)
    groups, off = host.fake_groups(), [host.fake_segment_off(i) for i in range(host.fake_groups() + 1)]
    assert off[0] == 0 and all(a < b for a, b in zip(off, off[1:])) and host.fake_grid() == groups * tiles
    seg = [[host.fake_segment(i, f) for f in range(7)] for i in range(off[-1])]
    units, slots, at = {}, set(), np.concatenate([[0], np.cumsum(-(-pages // 8) * 8)])
    for head, slot, first, count, a, b, whole in seg:
        units.setdefault((head >> 16, head & 0xffff), []).append((a, b, whole, slot, first, count))
        if slot >= 0:
            assert slot not in slots
            slots.add(slot)
    assert sorted(units) == [(r, h) for r in range(batch) for h in range(kv)] and slots == set(range(len(slots)))
    for (r, h), parts in units.items():
        assert parts[0][0] == 0 and parts[-1][1] == parts[-1][2] and all(x[1] == y[0] and x[2] == y[2] for x, y in zip(parts, parts[1:]))
        assert parts[0][4] == at[r] and sum(x[5] for x in parts) == pages[r] and all(x[4] + x[5] == y[4] for x, y in zip(parts, parts[1:]))
        assert (len(parts) == 1) == (parts[0][3] < 0)
        if len(parts) > 1:
            assert [x[3] for x in parts] == list(range(parts[0][3], parts[0][3] + len(parts)))
        if host.fake_splits() > 1:
            assert host.fake_unit(r * kv + h, 1) == len(parts) and (len(parts) == 1 or host.fake_unit(r * kv + h, 0) == parts[0][3])
    work = [sum((b - a) / whole * (pages[head >> 16] + blocks + -(-n_max // 16)) for head, _, _, _, a, b, whole in seg[i:j]) for i, j in zip(off, off[1:])]
    units_per_place = batch * kv * tiles / 148
    if units_per_place < 1:
        assert groups * tiles <= 148
        assert max(work) <= sum(work) / (148 // tiles) * 1.35 + 4 * 4, (max(work), sum(work) / (148 // tiles))


# ---- the calls without a cache: nothing is followed before everything has been looked at ---------------------------------------
def filled(cls, **kw):
    a = cls()
    for name, kind in cls._fields_:
        setattr(a, name, BASE if kind is ctypes.c_void_p else 1)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


TABLES = [(dict([(n, None)]), "INVAL") for n in ("tail_len", "block_table", "n_blocks", "free_pages", "n_free", "slot")] + \
         [(dict([(n, 0)]), "INVAL") for n in ("batch", "n_max", "max_blocks", "n_pages")] + \
         [(dict([(n, BASE + 1)]), "INVAL") for n in ("tail_len", "n_new", "parent", "pos_base", "block_table", "n_blocks", "free_pages", "n_free", "slot",
                                                     "position", "failed")] + \
         [(dict(mask=BASE + 4), "INVAL"), (dict(batch=1025), "LIMIT"), (dict(n_max=65), "LIMIT"), (dict(n_max=65, parent=None), "LIMIT"),
          (dict(n_max=65, mask=None), "LIMIT"), (dict(n_max=16385, mask=None, parent=None), "LIMIT"), (dict(n_pages=1 << 28), "LIMIT"),
          (dict(max_blocks=1 << 28), "LIMIT")]


@pytest.mark.parametrize("kw,code", TABLES, ids=str)
def test_tail_tables_refuses(kw, code):
    assert enl.lib().enl_tail_tables(ctypes.byref(filled(enl.TailTablesArgs, **kw)), None) == getattr(enl, "ENL_E_" + code)


ACCEPT = [(dict([(n, None)]), "INVAL") for n in ("token", "target", "accept", "n_accept", "next")] + [(dict(batch=0), "INVAL"), (dict(n_max=0), "INVAL")] + \
         [(dict([(n, BASE + 2)]), "INVAL") for n in ("n_new", "parent", "token", "target", "first", "accept", "n_accept", "next")] + [(dict(n_max=65), "LIMIT")]


@pytest.mark.parametrize("kw,code", ACCEPT, ids=str)
def test_tree_accept_refuses(kw, code):
    assert enl.lib().enl_tree_accept(ctypes.byref(filled(enl.TreeAcceptArgs, **kw)), None) == getattr(enl, "ENL_E_" + code)


def append_args(**kw):
    four = {n: (ctypes.c_void_p * 2)(BASE, BASE) for n in ("k_new", "v_new", "k_tail", "v_tail")}
    hole = kw.pop("hole", None)
    if hole:
        four[hole[0]][1] = hole[1]
    a = filled(enl.TailAppendArgs, n_layers=2, head_dim=64, **{n: ctypes.cast(p, ctypes.c_void_p) for n, p in four.items()})
    for k, v in kw.items():
        setattr(a, k, v)
    a.held = four
    return a


APPEND = [(dict([(n, None)]), "INVAL") for n in ("k_new", "v_new", "k_tail", "v_tail", "slot", "tail_len", "tail_len_out")] + \
         [(dict(hole=(n, x)), "INVAL") for n in ("k_new", "v_new", "k_tail", "v_tail") for x in (None, BASE + 8)] + \
         [(dict([(n, 0)]), "INVAL") for n in ("n_layers", "batch", "n_max", "n_kv_heads", "head_dim", "n_pages")] + [(dict(head_dim=12), "INVAL")] + \
         [(dict([(n, BASE + 2)]), "INVAL") for n in ("slot", "accept", "n_accept", "tail_len", "tail_len_out")] + \
         [(dict(n_max=16385), "LIMIT"), (dict(n_pages=1 << 28), "LIMIT"), (dict(n_kv_heads=1 << 20), "LIMIT")]


@pytest.mark.parametrize("kw,code", APPEND, ids=str)
def test_tail_append_refuses(kw, code):
    assert enl.lib().enl_tail_append(ctypes.byref(append_args(**kw)), None) == getattr(enl, "ENL_E_" + code)


def test_binding_refuses_what_the_library_could_not_see():
    """Types, shapes and layouts, by name; the CPU stands for every wrong device."""
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="token has to be a CUDA tensor"):
        enl.enl_tree_accept(None, i32(2, 3), i32(2, 3), i32(2, 3), i32(2), i32(2))
    with pytest.raises(ValueError, match="token has to be torch.int32, not torch.int64"):
        enl.enl_tree_accept(None, i32(2, 3).long(), i32(2, 3), i32(2, 3), i32(2), i32(2))
    with pytest.raises(ValueError, match="token has to have 2 dimensions"):
        enl.enl_tree_accept(None, i32(6), i32(2, 3), i32(2, 3), i32(2), i32(2))
    with pytest.raises(ValueError, match="token has to be contiguous"):
        enl.enl_tree_accept(None, i32(3, 2).t(), i32(2, 3), i32(2, 3), i32(2), i32(2))
    with pytest.raises(ValueError, match="slots has to be a CUDA tensor"):
        enl.enl_tail_tables(i32(2), i32(2, 4), i32(2), i32(8), i32(1), i32(2, 3))
    with pytest.raises(ValueError, match="slots has to be a CUDA tensor"):
        enl.enl_tail_append([], [], [], [], i32(2, 3), i32(2), i32(2))


# ---- the plain forms the GPU tests go by, by hand -----------------------------------------------------------------------------------
def test_reference_tree():
    see = ref.ancestors([-1, 0, 0, 1, -1, 7], 6)
    assert [np.nonzero(r)[0].tolist() for r in see] == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [5]]
    assert ref.bits(see, 8).tolist() == [1, 3, 5, 11, 16, 32, 0, 0]
    assert ref.ancestors(None, 3).tolist() == np.tril(np.ones((3, 3), bool)).tolist()


def test_reference_tables():
    table = np.full((3, 4), -1, np.int32)
    table[0, 0], table[2, :2] = 9, (4, 5)
    t = ref.tables(np.array([15, 0, -1]), np.array([3, 1, 2]), None, np.array([100, 0, 0]), table, np.array([1, 0, 2]), np.array([1, 2, 3, 8, 0, 0]), 4, 3, True)
    assert t["table"].tolist() == [[9, 8, -1, -1], [3, -1, -1, -1], [4, 5, -1, -1]] and t["n_blocks"].tolist() == [2, 1, 0]
    assert t["n_free"] == 4 and t["free"][:4].tolist() == [1, 2, 4, 5] and t["failed"] == 0
    assert t["slot"].tolist() == [[9 * 16 + 15, 8 * 16, 8 * 16 + 1], [48, -1, -1], [-1, -1, -1]]
    assert t["position"].tolist() == [[115, 116, 117], [0, 0, 0], [0, 0, 0]] and t["mask"].tolist() == [[1, 3, 7], [1, 0, 0], [0, 0, 0]]


def test_reference_accept():
    parent, token, target = np.array([[-1, 0, 0, 2, 3]]), np.array([[7, 1, 2, 2, 4]]), np.array([[2, 0, 2, 9, 5]])
    a, n, nxt = ref.accept(np.array([5]), parent, token, target, None, 5)
    assert a.tolist() == [[0, 2, 3, -1, -1]] and n.tolist() == [3] and nxt.tolist() == [9]
    a, n, nxt = ref.accept(np.array([5]), parent, token, target, np.array([6]), 5)
    assert n.tolist() == [0] and nxt.tolist() == [6]


def test_reference_attend():
    q = np.zeros((1, 1, 4))
    v = np.arange(12, dtype=float).reshape(3, 1, 4)
    out, tol = ref.attend(q, np.ones((3, 1, 4)), v, np.array([[True, False, True]]))
    assert np.allclose(out[0, 0], v[[0, 2], 0].mean(0)) and (tol >= 0).all()
    out, _ = ref.attend(q, np.ones((3, 1, 4)), v, np.zeros((1, 3), bool))
    assert (out == 0).all()
