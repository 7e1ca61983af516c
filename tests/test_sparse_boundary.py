"""Host side of the sparse attention's, the page tables' and the rotary forms' entry points
(include/ssa_sparse.h, include/ssa_pages.h, include/ssa_layer.h): what the plans cover, what
the calls refuse, the rotary tables, and the oracle against brute force.  No GPU: every
argument is checked before any HIP call."""
import ctypes

import numpy as np
import pytest

from oracle import sparse as osp
from paper_2606_05933_amd import ssa, workload

LIB = ssa.LIB
HEADER = np.dtype([("magic", "<u4"), ("block", "<i4"), ("hash", "<u8"), ("num_reqs", "<i4"),
                   ("num_tokens", "<i4"), ("hq", "<i4"), ("hkv", "<i4"), ("d", "<i4"),
                   ("page", "<i4"), ("maxp", "<i4"), ("num_pages", "<i4"), ("scale", "<f4"),
                   ("top", "<i4"), ("sink", "<i4"), ("recent", "<i4"), ("max_blocks", "<i4"),
                   ("most_blocks", "<i4"), ("num_groups", "<i4"), ("num_singles", "<i4"),
                   ("num_scores", "<i4"), ("off_rows", "<i4"), ("off_scores", "<i4"),
                   ("tiles", "<i4"), ("nsplit", "<i4"), ("entries", "<i4"), ("plan_bytes", "<i8"),
                   ("ws_bytes", "<i8")])
ROWS = np.dtype([(n, "<i4") for n in ("req", "row0", "pos0", "n")])
SCORE = np.dtype([(n, "<i4") for n in ("req", "row0", "pos0", "n", "blk0", "blk1", "p0", "p1")])
assert HEADER.itemsize == 120
NULL, SHAPE, HEAD_DIM, PAGE_SIZE, LENGTH, PAGES, PLAN_SIZE = -1, -2, -3, -4, -5, -6, -7
WORKSPACE, MISMATCH, ARG = -8, -9, -13
vp = ctypes.c_void_p


def shape_of(hq, hkv, d, lens, num_pages=1 << 20):
    return ssa.make_shape(hq, hkv, d, num_pages, max(1, -(-int(max(lens, default=1)) // 16)), 0.125)


def parse(plan):
    h = plan[:120].view(HEADER)[0]
    n = h["num_groups"] + h["num_singles"]
    return (h, plan[h["off_rows"]:h["off_rows"] + 16 * n].view(ROWS),
            plan[h["off_scores"]:h["off_scores"] + 32 * h["num_scores"]].view(SCORE))


@pytest.mark.parametrize("seed", range(40))
def test_plans_cover_every_row_and_block_once(seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(0, 9))
    c = rng.choice([0, 1, 1, 2, 3, 17, 64, 300], n)
    u = rng.choice([0, 1, 15, 16, 17, 400, 5000, 70000], n)
    hq, hkv, d = [(8, 8, 64), (32, 8, 128), (28, 4, 128), (16, 1, 64), (5, 5, 128)][seed % 5]
    block, top = int(rng.choice([16, 32, 64, 128])), int(rng.choice([2, 9, 64, 2000]))
    shape = shape_of(hq, hkv, d, c + u if n else [])
    plan, ws, most = ssa.sparse_plan(shape, c, u, block, top, 1, 1)
    h, rows, scores = parse(plan)
    assert h["plan_bytes"] == plan.nbytes and h["ws_bytes"] == ws >= 4096
    assert h["off_rows"] % 16 == 0 and h["off_scores"] % 32 == 0
    assert plan[120:120 + 8 * n].view(np.int32).reshape(n, 2).tolist() == np.stack(
        [c, u], axis=1).reshape(n, 2).tolist()
    seen = -(-(c + u)[c > 0] // block)
    assert h["most_blocks"] == max(seen, default=0)
    assert most == h["max_blocks"] == max(4, -(-max(seen, default=0) // 4) * 4)
    start = np.cumsum(c) - c
    T = int(c.sum())
    assert h["num_tokens"] == T
    mine = np.zeros(T, int)
    for i, r in enumerate(rows):
        assert 1 <= r["n"] <= 16 and (c[r["req"]] > 1) == (i < h["num_groups"])
        assert r["pos0"] - u[r["req"]] == r["row0"] - start[r["req"]]
        mine[r["row0"]:r["row0"] + r["n"]] += 1
    assert (mine == 1).all()
    covered = [np.zeros((int(u[i] + c[i] - 1) // block + 1, c[i]), int) if c[i] else None for i in range(n)]
    for s in scores:
        i = s["req"]
        j = s["row0"] - start[i]
        assert 0 <= j and j + s["n"] <= c[i] and s["pos0"] == u[i] + j
        assert 0 <= s["blk0"] < s["blk1"] <= (s["pos0"] + s["n"] - 1) // block + 1
        covered[i][s["blk0"]:s["blk1"], j:j + s["n"]] += 1
    for i in range(n):
        for j in range(c[i]):  # at least the blocks that the row sees, each once
            assert (covered[i][:(u[i] + j) // block + 1, j] == 1).all()
        assert c[i] == 0 or covered[i].max() == 1
    # pieces of the lists, and their tickets and records
    assert h["nsplit"] == -(-top // h["entries"]) <= 64
    g = hq // hkv
    tokens = min(16, 32 // g)
    units = h["num_groups"] * -(-16 // tokens) + h["num_singles"]
    if h["nsplit"] > 1:
        assert units * hkv <= 1024
        cols = tokens * g
        assert ws == 4096 + units * hkv * h["nsplit"] * 4 * (-(-2 * cols // 4) * 4 + cols * d)
    else:
        assert ws == 4096


# Batches whose score items hold more than four tiles of queries or more than one pass of 128
# blocks: heads, new tokens, cached ones, block, tiles of a chunk's item, blocks of a decode's.
LARGE_SCORES = [
    ((32, 8, 128), (550, 37, 1), (30000, 500, 4000), 32, 16, 128),
    ((8, 8, 64), (603, 1), (29990, 30), 16, 8, 128),
    ((28, 4, 128), (597, 1, 1), (30001, 16, 900), 32, 16, 128),
    ((8, 4, 128), (1030, 2), (33000, 100), 32, 8, 128),
    ((16, 1, 64), (611,), (30000,), 16, 16, 128),
    ((64, 8, 128), (1,) * 64, tuple(28000 + 31 * i for i in range(64)), 16, 16, 384),
    ((64, 8, 128), (1,) * 40 + (530,), tuple(20000 + 777 * i for i in range(40)) + (31000,), 16, 16, 256),
]


@pytest.mark.parametrize("heads,c,u,block,tiles,span", LARGE_SCORES)
def test_large_score_items_cover_every_row_and_block_once(heads, c, u, block, tiles, span):
    c, u = np.array(c), np.array(u)
    h, _, scores = parse(ssa.sparse_plan(shape_of(*heads, c + u), c, u, block, 8)[0])
    assert h["tiles"] == tiles and max(scores["blk1"] - scores["blk0"]) == span
    start = np.cumsum(c) - c
    for i in range(len(c)):
        covered = np.zeros((int(u[i] + c[i] - 1) // block + 1, c[i]), int)
        for s in scores[scores["req"] == i]:
            j = s["row0"] - start[i]
            assert 0 <= j and j + s["n"] <= c[i] and s["pos0"] == u[i] + j
            covered[s["blk0"]:s["blk1"], j:j + s["n"]] += 1
        seen = np.arange(len(covered))[:, None] <= (u[i] + np.arange(c[i])) // block
        assert (covered[seen] == 1).all() and covered.max() == 1


def test_sparse_plan_refusals():
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)

    def code(shape=shape, c=(1, 3), u=(10, 20), block=16, top=4, sink=1, recent=1):
        try:
            ssa.sparse_plan(shape, c, u, block, top, sink, recent)
        except ssa.SsaError as e:
            return e.code
        return 0

    assert code() == 0 and code(c=[], u=[]) == 0 and code(c=[0], u=[5]) == 0
    for block in (0, 8, 24, 48, 256, -16):
        assert code(block=block) == ARG
    assert code(top=0) == code(top=-1) == code(recent=0) == code(sink=-1) == ARG
    assert code(top=3, sink=2, recent=2) == code(top=32769) == ARG
    assert code(top=2 ** 31 - 1) == code(sink=2 ** 31 - 1, recent=2 ** 31 - 1, top=32768) == ARG
    assert code(top=2) == 0
    assert code(c=[-1], u=[0]) == code(c=[1], u=[-1]) == LENGTH
    assert code(c=[1], u=[320]) == PAGES and code(c=[1], u=[319]) == 0
    assert code(shape=ssa.make_shape(8, 3, 64, 100, 20, 0.125)) == SHAPE
    assert code(shape=ssa.make_shape(8, 2, 96, 100, 20, 0.125)) == HEAD_DIM
    assert code(shape=ssa.make_shape(8, 2, 64, 100, 20, 0.125, page_size=32)) == PAGE_SIZE
    wide = ssa.make_shape(8, 2, 64, 1 << 20, 1 << 20, 0.125)
    assert code(shape=wide, c=[1], u=[32768 * 16 - 1]) == 0
    assert code(shape=wide, c=[1], u=[32768 * 16]) == LENGTH
    assert code(shape=wide, c=[1], u=[32768 * 16], block=32) == 0
    assert code(shape=ssa.make_shape(1024, 1024, 64, 1 << 20, 1 << 20, 0.125), c=[1],
                u=[16384 * 16]) == LENGTH  # 1024 heads of 16388 blocks
    cfg = ssa.SsaSparseConfig(16, 4, 1, 1)
    c, u = np.array([1], np.int32), np.array([10], np.int32)
    sizes = [ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_int32()]

    def size(s=ctypes.byref(shape), g=ctypes.byref(cfg), c=c.ctypes.data, u=u.ctypes.data, n=1,
             out=tuple(ctypes.byref(x) for x in sizes)):
        return LIB.ssa_sparse_plan_size(s, g, c, u, n, *out)

    assert size() == 0 and size(n=-1) == LENGTH
    assert size(s=None) == size(g=None) == size(c=None) == size(u=None) == NULL
    for i in range(3):
        assert size(out=tuple(None if j == i else ctypes.byref(x) for j, x in enumerate(sizes))) == NULL
    buf = np.zeros(sizes[0].value, np.uint8)

    def plan(n_bytes=buf.nbytes, at=buf.ctypes.data):
        return LIB.ssa_sparse_plan(ctypes.byref(shape), ctypes.byref(cfg), c.ctypes.data,
                                   u.ctypes.data, 1, at, n_bytes)

    assert plan() == 0 and plan(buf.nbytes - 1) == PLAN_SIZE and plan(at=None) == NULL


def test_plans_of_other_configurations_differ():
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    hashes = set()
    for args in ([1], [20], 16, 4, 1, 1), ([1], [21], 16, 4, 1, 1), ([2], [19], 16, 4, 1, 1), \
                ([1], [20], 32, 4, 1, 1), ([1], [20], 16, 5, 1, 1), ([1], [20], 16, 4, 2, 1), \
                ([1], [20], 16, 4, 1, 2), ([1, 0], [20, 3], 16, 4, 1, 1):
        hashes.add(int(parse(ssa.sparse_plan(shape, *args)[0])[0]["hash"]))
    assert len(hashes) == 8


def test_sparse_calls_refuse_before_they_launch():
    """Every pointer is a small number: a launch, or a read of one, would end the process."""
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    other = ssa.make_shape(8, 4, 64, 100, 20, 0.125)
    c, u = [1, 3], [10, 20]
    batch, _ = ssa.ssa_plan(shape, c, u)
    plan, ws, _ = ssa.sparse_plan(shape, c, u, 16, 4)
    calls = {
        # name: (plan, its other arguments, which of them are refused unless 16-byte aligned)
        "ssa_block_summary": (batch, [16, 16, 16, 16], [1, 3]),
        "ssa_block_scores": (plan, [16, 16, 16, 16], [0, 1, 3]),
        "ssa_block_select": (plan, [16, 16], [0, 1]),
        "ssa_sparse_attention": (plan, [16, 16, 16, 16, 16, 16, 16, ws], [0, 1, 2, 4, 5, 6]),
    }
    for name, (p, args, aligned) in calls.items():
        f = getattr(LIB, name)

        def call(s=shape, p=p, dev=16, args=args):
            a = [x if isinstance(x, int) and i == 7 else x for i, x in enumerate(args)]
            return f(None if s is None else ctypes.byref(s), None if p is None else p.ctypes.data,
                     dev, *a, None)

        assert call(s=None) == NULL and call(p=None) == NULL and call(dev=None) == NULL
        assert call(s=other) == MISMATCH
        assert call(p=plan if p is batch else batch) == MISMATCH
        for dev in (4097, 4100, 4092):
            assert call(dev=dev) == ARG
        for i in range(len(args)):
            if name == "ssa_block_summary" and i == 0:  # block_keys
                for b in (0, 17, 256):
                    assert call(args=[b, *args[1:]]) == ARG
                continue
            if i == 7:
                assert call(args=[*args[:7], ws - 1]) == WORKSPACE
                continue
            want = WORKSPACE if name == "ssa_sparse_attention" and i == 6 else NULL
            assert call(args=[None if j == i else x for j, x in enumerate(args)]) == want, (name, i)
            if i in aligned:
                assert call(args=[24 if j == i else x for j, x in enumerate(args)]) == ARG, (name, i)
    # batches without a new token launch nothing
    for c in ([], [0, 0]):
        u = [5] * len(c)
        batch, _ = ssa.ssa_plan(shape, c, u)
        plan, ws, _ = ssa.sparse_plan(shape, c, u, 16, 4)
        s = ctypes.byref(shape)
        assert LIB.ssa_block_summary(s, batch.ctypes.data, 16, 16, None, None, None, None) == 0
        assert LIB.ssa_block_scores(s, plan.ctypes.data, 16, None, None, None, None, None) == 0
        assert LIB.ssa_block_select(s, plan.ctypes.data, 16, None, None, None) == 0
        assert LIB.ssa_sparse_attention(s, plan.ctypes.data, 16, None, None, None, None, None, None,
                                        16, ws, None) == 0


def test_pages_resize_refuses_before_it_launches():
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)

    def call(s=shape, n=3, args=(16, 16, 16, 16, 160, 320, 16, 16), rows=10):
        return LIB.ssa_pages_resize(None if s is None else ctypes.byref(s), n, *args, rows, None)

    assert call(s=None) == NULL
    assert call(n=-1) == call(n=65537) == LENGTH
    for i in range(6):
        assert call(args=[None if j == i else x for j, x in enumerate((16, 16, 16, 16, 160, 320, 16, 16))]) == NULL
    assert call(rows=-1) == ARG
    for at in (160, 148, 172):  # the new state over the old one
        assert call(args=(16, 16, 16, 16, 160, at, 16, 16)) == ARG
    assert call(s=ssa.make_shape(8, 2, 64, 0, 20, 0.125)) == PAGES
    assert call(s=ssa.make_shape(8, 2, 64, 100, 20, 0.125, page_size=8)) == PAGE_SIZE


@pytest.fixture
def host_calls(monkeypatch):
    """The binding's checks on host tensors: a list of what reaches the library, whose calls
    launch nothing here."""
    calls = []

    class Buffers(ssa._Buffers):
        __slots__ = ()

        def __init__(self):
            self.device = -1  # a host tensor's

        def stream(self, stream):
            return None

    class Lib:
        def __getattr__(self, name):
            return lambda *args: calls.append((name, args)) or 0

    monkeypatch.setattr(ssa, "_Buffers", Buffers)
    monkeypatch.setattr(ssa, "LIB", Lib())
    return calls


def test_an_empty_slot_map_is_not_one_left_out(host_calls):
    """A slot map without room for a row: the library has to see that it is there, so that
    new rows are refused and nothing changes."""
    import torch
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    for slots, rows in ((None, 0), (torch.zeros(0, dtype=torch.int64), 0),
                        (torch.zeros(7, dtype=torch.int64), 7)):
        ssa.pages_resize(shape, ints(3), ints(3), ints(3, 20), ints(100), ints(4), ints(4), None,
                         slots)
        name, args = host_calls.pop()
        assert name == "ssa_pages_resize" and args[8] is None and args[10] == rows
        assert (args[9] is None) == (slots is None) and args[9] != 0


def test_a_buffer_shorter_than_a_header_is_no_plan():
    """Refused by its size: its words would be read past its end (here from a plan that it is
    the beginning of)."""
    import torch
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    assert min(ssa.sparse_plan(shape, [], [], 16, 4)[0].nbytes, ssa.ssa_plan(shape, [], [])[0].nbytes,
               ssa.score_plan(shape, [], [])[0].nbytes,
               ssa.evict_plan(shape, [], [], 0, 0)[0].nbytes) >= 128
    plan, _, _ = ssa.sparse_plan(shape, [1], [20], 16, 4)
    fixed = plan.copy()
    fixed.flags.writeable = False
    for p in (plan, fixed, torch.from_numpy(plan)):
        at, words = ssa._header(p, ssa._SPARSE_MAGIC, "")
        assert words[ssa._SPARSE_TOKENS] == 1 and at
        for n in (0, 8, 127):
            with pytest.raises(ssa.SsaError) as e:
                ssa._header(p[:n], ssa._SPARSE_MAGIC, "")
            assert e.value.code == MISMATCH
        ssa._header(p[:128], ssa._SPARSE_MAGIC, "")
    with pytest.raises(ssa.SsaError) as e:
        ssa._header(None, ssa._SPARSE_MAGIC, "")
    assert e.value.code == NULL


def test_shifts_of_a_batch_without_requests(host_calls):
    import torch
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    plan = np.zeros(256, np.uint8)
    plan[:4].view(np.uint32)[0] = ssa._PLAN_MAGIC
    none = torch.zeros(0, dtype=torch.int32)
    pool = torch.zeros(100 * 2 * 16 * 64, dtype=torch.bfloat16)
    rows = torch.zeros(0, dtype=torch.bfloat16)
    dev = torch.from_numpy(plan)
    ssa.rope_append_as(shape, plan, dev, rows, torch.zeros(1, 64), rows, pool, pool, none,
                       shift_host=np.zeros(0, np.int32), shift_dev=none)
    _, args = host_calls.pop()
    assert args[7] and args[8], "both shift arrays are there, and empty"


def test_rotary_tables_of_other_rows(host_calls, monkeypatch):
    """A table whose rows are not the rotated dims is refused; a flat one goes by its size."""
    import torch
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    plan = np.zeros(256, np.uint8)
    plan[:4].view(np.uint32)[0] = ssa._PLAN_MAGIC
    bf = lambda n: torch.zeros(n, dtype=torch.bfloat16)  # noqa: E731
    none, shift = torch.zeros(0, dtype=torch.int32), np.zeros(0, np.int32)
    monkeypatch.setattr(ssa, "_check_dev", lambda *a: None)
    monkeypatch.setattr(ssa, "_stream", lambda s: 0)

    def positions(name, table, rotary):
        args = [shape, plan, torch.from_numpy(plan), bf(0), table]
        pools = [bf(0), bf(100 * 2 * 16 * 64), bf(100 * 2 * 16 * 64), none]
        if name == "rope_append_as":
            ssa.rope_append_as(*args, *pools, rotary_dim=rotary)
        elif name == "rope_append_shifted":
            ssa.rope_append_shifted(*args, shift, none, *pools)
        else:
            ssa.rope_append(*args, *pools)
        got, args = host_calls.pop()
        assert got == "ssa_" + name
        return args[6 if name == "rope_append_as" else 5]

    for name, rotary in (("rope_append_as", 32), ("rope_append_as", 64),
                         ("rope_append_shifted", 64), ("rope_append", 64)):
        for size in ((7, rotary), (7, 2, rotary // 2), (7 * rotary,), (1, rotary)):
            assert positions(name, torch.zeros(size), rotary) == (1 if size[0] == 1 else 7)
        for size in ((7, 2 * rotary), (14, rotary // 2), (7 * rotary + 1,), (4, rotary + 16)):
            with pytest.raises(ValueError):
                positions(name, torch.zeros(size), rotary)
            assert not host_calls


def test_rope_append_as_refuses_before_it_launches():
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    plan, _ = ssa.ssa_plan(shape, [1, 3], [10, 20])
    shift = np.array([0, 42], np.int32)

    def call(form=(0, 64), position=64, shifts=(None, None), qkv=16):
        f = None if form is None else ctypes.byref(ssa.SsaRopeForm(*form))
        return LIB.ssa_rope_append_as(ctypes.byref(shape), plan.ctypes.data, 16, f, qkv, 16, position,
                                      *shifts, 16, 16, 16, 16, None)

    assert call(form=None) == NULL
    for form in (2, 64), (-1, 64), (0, 0), (0, 8), (0, 24), (0, 80), (1, 72), (1, -16):
        assert call(form=form) == ARG, form
    assert call(position=22) == ARG
    assert call(qkv=None) == call(shifts=(shift.ctypes.data, None)) == call(shifts=(None, 16)) == NULL
    assert call(shifts=(shift.ctypes.data, 16)) == ARG  # position 64 of 64
    with pytest.raises(ValueError):
        ssa.rope_append_as(shape, plan, None, *[None] * 6, layout="quarter")


def test_a_sparse_layer_refuses_before_it_launches():
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    c, u = [1, 3], [10, 20]
    plan, _ = ssa.ssa_plan(shape, c, u)
    w = ssa.SsaLayerWeights(16, 16, 16, 16, 16, 16, 16, 256, 128, 64, 1e-5)
    good, ws, _ = ssa.sparse_plan(shape, c, u, 16, 4)

    def call(e, n=1 << 30):
        return LIB.ssa_layer_forward_sparse(
            ctypes.byref(shape), plan.ctypes.data, vp(16), ctypes.byref(w),
            None if e is None else ctypes.byref(e), *[vp(16)] * 6, n, None)

    def parts(p=good, **more):
        return ssa.SsaLayerSparse(**{**dict(
            plan_host=p.ctypes.data, plan_dev=16, summary=16, scores=16, blocks=16, workspace=16,
            ws_bytes=ws, block_keys=16), **more})

    assert call(None) == NULL
    assert call(parts(), n=256) == WORKSPACE
    for other in ([1, 3, 0], [20, 10, 5]), ([1, 2], [10, 20]), ([2, 2], [10, 20]), ([1, 3], [20, 10]):
        assert call(parts(ssa.sparse_plan(shape, *other, 16, 4)[0])) == MISMATCH
    assert call(parts(plan)) == MISMATCH
    assert call(parts(block_keys=32)) == ARG
    assert call(parts(ws_bytes=ws - 1)) == WORKSPACE and call(parts(workspace=None)) == WORKSPACE
    for name in ("summary", "plan_dev", "scores", "blocks"):
        assert call(parts(**{name: None})) == NULL, name
        assert call(parts(**{name: 8 if name != "plan_dev" else 20})) == ARG, name
    assert call(ssa.SsaLayerSparse(summary=16, block_keys=24)) == ARG
    assert call(ssa.SsaLayerSparse(summary=24, block_keys=16)) == ARG
    shift = np.array([0, 42], np.int32)
    assert call(ssa.SsaLayerSparse(shift_host=shift.ctypes.data)) == NULL
    assert call(ssa.SsaLayerSparse(shift_dev=16)) == NULL
    assert call(ssa.SsaLayerSparse(shift_host=shift.ctypes.data, shift_dev=16)) == ARG
    for form in (2, 64), (0, 24), (1, 128):
        f = ssa.SsaRopeForm(*form)
        assert call(ssa.SsaLayerSparse(rope=ctypes.pointer(f))) == ARG


@pytest.mark.parametrize("kind,more", [("none", {}), ("linear", dict(factor=4.0)),
                                       ("base", dict(factor=8.0)),
                                       ("parts", dict(factor=8.0, trained_positions=8192, low=1.0, high=4.0))])
@pytest.mark.parametrize("d,base,magnitude", [(128, 5e5, 1.0), (32, 1e4, 1.2), (96, 1e4, 1.0), (4, 10.0, 0.5)])
def test_scaled_rotary_tables(kind, more, d, base, magnitude):
    """The angle of the last position is off by a few 2^-53 of itself in either form; an entry
    is rounded once."""
    n = 3000
    got = ssa.rope_cos_sin_scaled(n, d, base, kind, magnitude=magnitude, **more)
    t = osp.angles(d, base, kind, more.get("factor", 1.0), more.get("trained_positions", 0),
                   more.get("low", 0.0), more.get("high", 0.0))
    a = np.arange(n)[:, None] * t
    want = magnitude * np.concatenate([np.cos(a), np.sin(a)], axis=1)
    assert np.abs(got - want).max() <= magnitude * (2.0 ** -24 + n * 2.0 ** -50)
    if kind == "none" and magnitude == 1.0:
        assert np.array_equal(got, ssa.rope_cos_sin(n, d, base))
    if kind == "base":  # the slowest angle is divided by the factor, the fastest is kept
        plain = osp.angles(d, base)
        assert np.isclose(t[-1], plain[-1] / 8.0, rtol=1e-12) and t[0] == 1.0
    if kind == "parts":
        plain = osp.angles(d, base)
        turns = 8192 * plain / (2 * np.pi)
        assert np.allclose(t[turns >= 4], plain[turns >= 4])
        assert np.allclose(t[turns <= 1], plain[turns <= 1] / 8)
        assert ((t <= plain * (1 + 1e-12)) & (t >= plain / 8 * (1 - 1e-12))).all()


def test_scaled_rotary_table_refusals():
    def code(n=10, d=64, base=1e4, scaling="linear", factor=2.0, trained=100, low=1.0, high=4.0, magnitude=1.0):
        try:
            ssa.rope_cos_sin_scaled(n, d, base, scaling, factor, trained, low, high, magnitude)
        except ssa.SsaError as e:
            return e.code
        return 0

    nan, inf = float("nan"), float("inf")
    for kind in ssa.ROPE_SCALINGS:
        assert code(scaling=kind) == 0
        assert code(n=0) == code(d=7) == code(base=1.0) == code(base=inf) == ARG
        for m in (0.0, -1.0, nan, inf):
            assert code(scaling=kind, magnitude=m) == ARG
        for f in (0.5, nan, inf):
            assert code(scaling=kind, factor=f) == (0 if kind == "none" else ARG)
    assert code(scaling="base", d=2) == ARG and code(scaling="linear", d=2) == 0
    assert code(scaling="base", base=1e300, factor=1e30) == ARG
    for bad in (dict(trained=0), dict(low=-1.0), dict(low=4.0), dict(high=inf), dict(low=nan), dict(high=nan)):
        assert code(scaling="parts", **bad) == ARG and code(**bad) == 0
    assert LIB.ssa_rope_table_scaled(4, 8, 1e4, None, 16) == NULL
    s = ssa.SsaRopeScaling(4, 0, 1.0, 0, 0, 1.0)
    out = np.zeros((4, 8), np.float32)
    assert LIB.ssa_rope_table_scaled(4, 8, 1e4, ctypes.byref(s), out.ctypes.data) == ARG
    s.kind = 0
    assert LIB.ssa_rope_table_scaled(4, 8, 1e4, ctypes.byref(s), None) == NULL
    with pytest.raises(ValueError):
        ssa.rope_cos_sin_scaled(4, 8, 1e4, "other")


def test_oracle_by_hand():
    f = np.float32
    assert osp.select(np.array([1, 5, 5, 2, 0], f), 3, 1, 1).tolist() == [0, 1, 4]
    assert osp.select(np.array([1, 5, np.nan, 6, 0], f), 3, 0, 1).tolist() == [2, 3, 4]
    assert osp.select(np.array([1, 2], f), 4, 1, 1).tolist() == [0, 1, -1, -1]
    assert osp.select(np.array([-np.inf, -np.inf, 0], f), 2, 0, 1).tolist() == [0, 2]
    q = np.array([[1.0, -2.0], [-1.0, 0.5]])
    hi, lo = np.array([[3.0, 1.0]]), np.array([[-1.0, -4.0]])
    assert osp.bounds(q, hi, lo)[0].tolist() == [11.0]  # 3 + 8, and 1 + 0.5
    assert osp.keys_of([1, -1, 0, 1, 9], 2, 2).tolist() == [2, 0, 1, 2]
    table = np.array([[7, -1], [3, -1]])
    ring = np.array([5, 0, 1, 2, -1, -1])
    t, r, s, rows, slots = osp.pages(table, ring, [0, 4, 0, 0], [15, 16], [18, 0], 6)
    assert t.tolist() == [[7, 5], [3, -1]] and r.tolist() == [5, 0, 1, 2, 3, -1]
    assert s.tolist() == [1, 4, 0, 0] and rows.tolist() == [0, 3, 3]
    assert slots.tolist() == [7 * 16 + 15, 5 * 16, 5 * 16 + 1]
    x = np.arange(4.0).reshape(1, 1, 4)
    c, s = np.zeros((1, 1)), np.ones((1, 1))
    assert osp.rotate(x, c, s, "half", 2).tolist() == [[[-1, 0, 2, 3]]]
    c, s = np.zeros((1, 2)), np.ones((1, 2))
    assert osp.rotate(x, c, s, "half", 4).tolist() == [[[-2, -3, 0, 1]]]
    assert osp.rotate(x, c, s, "interleaved", 4).tolist() == [[[-1, 0, -3, 2]]]


def test_oracle_attention_over_all_blocks_is_attention():
    from oracle import oracle
    b = workload.make_batch(workload.Shape(4, 2, 64), [3, 1, 0], [20, 40, 7], seed=2, spare_pages=3)
    kc, vc = oracle.batch_kv_append(b)
    lists = np.tile(np.arange(3, dtype=np.int32), (4, 2, 1))
    out, mass, _ = osp.attention(b, kc, vc, lists, 16)
    ref, _ = oracle.batch_attention(b, kc, vc)
    assert np.allclose(out, ref, rtol=1e-12, atol=1e-12) and (mass >= np.abs(out)).all()
    lists[3] = -1
    assert not osp.attention(b, kc, vc, lists, 16)[0][3].any()
