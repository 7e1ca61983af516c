"""Host side of the eviction entry points (include/ssa_evict.h): what their plans
cover, what they refuse, the table check, and the oracle against brute force.  No
GPU: every argument is checked before any HIP call."""
import ctypes

import numpy as np
import pytest

from oracle import evict as oev
from paper_2606_05933_amd import ssa, workload

LIB = ssa.LIB
LISTS = ("lse", "decode", "lse_join", "sum", "decode_join")
HEADER = np.dtype([("magic", "<u4"), ("last_rows", "<i4"), ("hash", "<u8"), ("num_reqs", "<i4"),
                   ("num_tokens", "<i4"), ("hq", "<i4"), ("hkv", "<i4"), ("d", "<i4"),
                   ("page", "<i4"), ("maxp", "<i4"), ("num_pages", "<i4"), ("scale", "<f4"),
                   ("max_q", "<i4"), ("lse_groups", "<i4"), ("sum_cols", "<i4"),
                   ("off_items", "<i4"), ("num_tickets", "<i4"), ("count", "<i4", 5), ("first", "<i4", 5),
                   ("plan_bytes", "<i8"), ("ws_bytes", "<i8")])
ITEM = np.dtype([(n, "<i4") for n in ("req", "q_row", "ticket", "rows", "len", "ctx", "col0",
                                      "cols_pad", "key0", "key1", "split", "nsplit")]
                + [("off0", "<i8"), ("off1", "<i8")])
assert HEADER.itemsize == 128 and ITEM.itemsize == 64


def shape_of(hq, hkv, d, lens, num_pages=1 << 20):
    return ssa.make_shape(hq, hkv, d, num_pages, max(1, -(-int(max(lens, default=1)) // 16)), 0.125)


def parse(plan):
    h = plan[:128].view(HEADER)[0]
    items = plan[h["off_items"]:].view(ITEM)
    return h, {n: items[h["first"][i]:h["first"][i] + h["count"][i]] for i, n in enumerate(LISTS)}


def random_batch(rng):
    n = int(rng.integers(0, 9))
    c = rng.choice([0, 1, 1, 2, 3, 17, 64, 300, 2000], n)
    u = rng.choice([0, 1, 15, 16, 17, 400, 5000, 70000], n)
    return c, u


@pytest.mark.parametrize("seed", range(40))
def test_score_plans_cover_the_batch_once_and_stay_in_the_workspace(seed):
    rng = np.random.default_rng(seed)
    c, u = random_batch(rng)
    hq, hkv, d = [(8, 8, 64), (32, 8, 128), (28, 4, 128), (16, 1, 64), (5, 5, 128)][seed % 5]
    g, last = hq // hkv, int(rng.choice([0, 0, 1, 2, 50]))
    shape = shape_of(hq, hkv, d, c + u if len(c) else [])
    plan, ws_bytes = ssa.score_plan(shape, c, u, last)
    h, items = parse(plan)
    assert h["plan_bytes"] == plan.nbytes and h["ws_bytes"] == ws_bytes >= 256
    assert h["num_tokens"] == c.sum() and h["max_q"] == max(c, default=0)
    start = np.cumsum(c) - c
    taken, tickets = [], []  # workspace ranges, in floats
    for i in range(len(c)):
        rows = min(c[i], last) if last else c[i]
        mine = {n: x[x["req"] == i] for n, x in items.items()}
        for x in mine.values():
            assert (x["q_row"] == start[i] + c[i] - rows).all() and (x["rows"] == rows).all()
            assert (x["len"] == c[i] + u[i]).all() and (x["ctx"] == u[i]).all()
            assert (x["key0"] < x["key1"]).all() or not len(x) or (x is mine["lse_join"])
        used = ("decode", "decode_join") if rows == 1 else ("lse", "lse_join", "sum")
        assert all(not len(mine[n]) for n in LISTS if c[i] == 0 or n not in used)
        if c[i] == 0:
            continue
        length = c[i] + u[i]

        def partition(x):
            x = np.sort(x, order="key0")
            assert x["key0"][0] == 0 and x["key1"][-1] == length
            assert (x["key0"][1:] == x["key1"][:-1]).all()

        if rows == 1:
            dec = mine["decode"]
            partition(dec)
            if dec["split"][0] == -1:  # the whole row in one workgroup, its logits in LDS
                assert len(dec) == 1 and not len(mine["decode_join"])
                assert dec["cols_pad"][0] * g <= 8192
                continue
            partition(mine["decode_join"])
            assert (dec["key0"] % 128 == 0).all() and (mine["decode_join"]["key0"] % 16 == 0).all()
            pad, ns = int(dec["cols_pad"][0]), int(dec["nsplit"][0])
            assert pad % 32 == 0 and pad >= length and ns == len(dec)
            assert sorted(dec["split"]) == list(range(ns))
            taken.append((int(dec["off0"][0]), hkv * g * pad))
            taken.append((int(dec["off1"][0]), hkv * ns * ((2 * g + 3) // 4 * 4 + g * d)))
            continue
        lse, cols = mine["lse"], rows * g
        pad, ns = int(lse["cols_pad"][0]), int(lse["nsplit"][0])
        width = 64 * h["lse_groups"]
        assert pad % 256 == 0 and pad >= cols
        assert sorted(set(lse["col0"])) == list(range(0, cols, width))
        for col in set(lse["col0"]):
            x = lse[lse["col0"] == col]
            partition(x)
            assert len(x) == ns and (x["key0"] % 128 == 0).all()
        sums, per = mine["sum"], int(h["sum_cols"])
        assert per % 32 == 0 and (sums["key0"] % 256 == 0).all()
        partition(sums[sums["col0"] == sums["col0"].max()])  # the last rows see every key
        pieces = -(-cols // per)
        for k in set(sums["key0"]):
            # the column ranges from the first row that sees the tile on
            x = np.sort(sums[sums["key0"] == k], order="col0")
            first = max(0, k - (length - rows)) * g // per
            assert x["col0"].tolist() == [per * p for p in range(first, pieces)]
            assert x["split"].tolist() == list(range(len(x))) and (x["nsplit"] == len(x)).all()
            assert len(set(x["key1"])) == 1 and x["key1"][0] == min(length, k + 256)
            if len(x) > 1:
                tickets += list(range(x["ticket"][0], x["ticket"][0] + hkv))
                assert len(set(x["ticket"])) == 1
        if pieces > 1:
            taken.append((int(sums["off1"][0]), pieces * hkv * -(-length // 256) * 256))
        taken.append((int(lse["off0"][0]), hkv * pad))
        if ns > 1:
            assert sorted(mine["lse_join"]["col0"]) == list(range(0, pad, 256))
            taken.append((int(lse["off1"][0]), hkv * ns * pad * 2))
        else:
            assert not len(mine["lse_join"])
    assert sorted(tickets) == list(range(h["num_tickets"]))
    taken.sort()
    assert not taken or taken[0][0] >= h["num_tickets"]
    for (a, n), (b, _) in zip(taken, taken[1:]):
        assert a + n <= b
    assert all(a % 64 == 0 for a, _ in taken)
    assert not taken or 4 * (taken[-1][0] + taken[-1][1]) <= ws_bytes


def raw_score_plan(shape, c, u, last_rows, cap=None):
    c, u = np.asarray(c, np.int32), np.asarray(u, np.int32)
    pb, wb = ctypes.c_size_t(), ctypes.c_size_t()
    rc = LIB.ssa_score_plan_size(ctypes.byref(shape), c.ctypes.data, u.ctypes.data, len(c),
                                 last_rows, ctypes.byref(pb), ctypes.byref(wb))
    if rc or cap is None:
        return rc
    out = np.zeros(pb.value, np.uint8)
    return LIB.ssa_score_plan(ctypes.byref(shape), c.ctypes.data, u.ctypes.data, len(c), last_rows,
                              out.ctypes.data, cap(pb.value))


def test_score_plan_refusals():
    shape = ssa.make_shape(8, 8, 64, 100, 4, 0.125)
    assert raw_score_plan(shape, [1, 3], [10, 20], 0, lambda n: n) == 0
    assert raw_score_plan(shape, [1, 3], [10, 20], 0, lambda n: n - 1) == -7
    assert raw_score_plan(shape, [1], [10], -1) == ssa.SSA_ERR_ARG
    assert raw_score_plan(shape, [-1], [10], 0) == -5
    assert raw_score_plan(shape, [1], [-10], 0) == -5
    assert raw_score_plan(shape, [1], [64], 0) == -6  # 65 keys, 4 pages
    assert raw_score_plan(ssa.make_shape(7, 2, 64, 100, 4, 0.1), [1], [1], 0) == -2
    assert raw_score_plan(ssa.make_shape(17, 1, 64, 100, 4, 0.1), [1], [1], 0) == -2
    assert raw_score_plan(ssa.make_shape(8, 8, 96, 100, 4, 0.1), [1], [1], 0) == -3
    assert raw_score_plan(ssa.make_shape(8, 8, 64, 100, 4, -1.0), [1], [1], 0) == -11
    big = ssa.make_shape(16, 1, 64, 1 << 27, 1 << 26, 0.1)
    assert raw_score_plan(big, [1 << 29, 1 << 29, 1], [0, 0, 0], 1) == -5
    assert raw_score_plan(big, [(1 << 24) + 1], [0], 0) == -5  # more than 2^28 columns
    assert raw_score_plan(ssa.make_shape(1 << 18, 1 << 18, 128, 9, 9, 0.1), [1], [1], 0) == -2
    pb = ctypes.c_size_t()
    assert LIB.ssa_score_plan_size(ctypes.byref(shape), None, None, 1, 0, ctypes.byref(pb),
                                   ctypes.byref(pb)) == ssa.SSA_ERR_NULL
    assert LIB.ssa_score_plan_size(ctypes.byref(shape), None, None, 0, 0, ctypes.byref(pb),
                                   None) == ssa.SSA_ERR_NULL


def call_scores(shape, plan, decay=1.0, ws=1 << 30, fill=16, dev=1, fn="ssa_key_scores", n_ptr=0):
    """Raw call with made-up pointers: it has to be refused before they are used."""
    vp = ctypes.c_void_p
    ptr = plan.ctypes.data if plan is not None else None
    if fn == "ssa_key_scores":
        return LIB.ssa_key_scores(ctypes.byref(shape), ptr, vp(dev), vp(fill), vp(fill), vp(fill),
                                  None, decay, vp(fill), vp(4096), ws, None)
    return LIB.ssa_decode_scored(ctypes.byref(shape), ptr, vp(dev), vp(fill), vp(fill), vp(n_ptr),
                                 vp(fill), None, decay, vp(fill), vp(fill), vp(4096), ws, None)


def test_scored_calls_refuse_before_they_launch():
    shape = ssa.make_shape(8, 8, 64, 100, 4, 0.125)
    other = ssa.make_shape(8, 8, 64, 101, 4, 0.125)
    plan, ws = ssa.score_plan(shape, [1, 3], [10, 20])
    assert call_scores(shape, None) == ssa.SSA_ERR_NULL
    assert call_scores(other, plan) == ssa.SSA_ERR_PLAN_MISMATCH
    attention, _ = ssa.ssa_plan(shape, [1, 3], [10, 20])
    assert call_scores(shape, attention) == ssa.SSA_ERR_PLAN_MISMATCH
    eviction, _ = ssa.evict_plan(shape, [30], [20], 0, 0)
    assert call_scores(shape, eviction) == ssa.SSA_ERR_PLAN_MISMATCH
    for decay in (-0.5, float("nan"), float("inf")):
        assert call_scores(shape, plan, decay) == ssa.SSA_ERR_ARG
    assert call_scores(shape, plan, ws=ws - 1) == ssa.SSA_ERR_WORKSPACE
    assert call_scores(shape, plan, fill=0) == ssa.SSA_ERR_NULL
    assert call_scores(shape, plan, fill=24) == ssa.SSA_ERR_ARG  # 8-byte aligned
    assert call_scores(shape, plan, dev=0) == ssa.SSA_ERR_NULL
    # a chunk has no place in the decode call
    assert call_scores(shape, plan, fn="ssa_decode_scored", n_ptr=1) == ssa.SSA_ERR_ARG
    decodes, _ = ssa.score_plan(shape, [1, 0], [10, 20])
    assert call_scores(shape, decodes, fn="ssa_decode_scored", n_ptr=0) == ssa.SSA_ERR_NULL
    # a window of one row does not make a chunk a decode
    window, _ = ssa.score_plan(shape, [3], [10], 1)
    assert call_scores(shape, window, fn="ssa_decode_scored", n_ptr=1) == ssa.SSA_ERR_ARG
    # nothing to do needs no pointers
    empty, _ = ssa.score_plan(shape, [0, 0], [10, 20])
    assert call_scores(shape, empty, fill=0) == ssa.SSA_OK


def test_evict_plan_and_its_refusals():
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    plan, ws = ssa.evict_plan(shape, [100, 0, 17, 300], [70, 5, 17, 300], 4, 8)
    i4, i8 = plan[:128].view(np.int32), plan[:128].view(np.int64)
    assert ws >= 256 and i4[3] == 4 and i8[10] == 70 + 0 + 17 + 300 and i8[11] == plan.nbytes
    reqs = plan[128:128 + 64].view(np.dtype([("len", "<i4"), ("kept", "<i4"), ("off", "<i8")]))
    assert reqs["len"].tolist() == [100, 0, 17, 300] and reqs["kept"].tolist() == [70, 0, 17, 300]
    assert reqs["off"].tolist() == [0, 70, 70, 87]
    shorts = plan[i4[16]:i4[17]].view(np.int32).reshape(-1, 6)
    assert len(shorts) == i4[13] == 3 and i4[14] == i4[19] == 0
    assert shorts[:, :5].tolist() == [[0, 100, 70, 0, 0], [2, 17, 17, 0, 70], [3, 300, 300, 0, 87]]
    items = plan[i4[18]:].view(np.int32).reshape(-1, 8)
    assert len(items) == i4[15] == 2 and items[:, :5].tolist() == [[0, 0, 64, 100, 70],
                                                                 [0, 64, 6, 100, 70]]

    def code(lens, budget, sink, recent, s=shape):
        with pytest.raises(ssa.SsaError) as e:
            ssa.evict_plan(s, lens, budget, sink, recent)
        return e.value.code

    assert code([100], [11], 4, 8) == ssa.SSA_ERR_ARG  # sinks and recent keys do not fit
    assert ssa.evict_plan(shape, [11], [11], 4, 8)     # nothing is lost: they need not
    assert ssa.evict_plan(shape, [100], [12], 4, 8)
    assert ssa.evict_plan(shape, [100], [0], 0, 0)
    assert code([100], [11], -1, 8) == ssa.SSA_ERR_ARG
    assert code([100], [11], 2 ** 31 - 1, 2 ** 31 - 1) == ssa.SSA_ERR_ARG
    assert code([-1], [11], 0, 0) == -5 and code([1], [-11], 0, 0) == -5
    assert code([321], [100], 0, 0) == -6
    with pytest.raises(ValueError):
        ssa.evict_plan(shape, [1, 2], [1], 0, 0)


def test_long_lists_are_cut_into_segments():
    hkv, lens = 3, [8192, 8193, 100000, 9000, 50000]
    shape = shape_of(3 * hkv, hkv, 64, lens)
    plan, ws = ssa.evict_plan(shape, lens, [100, 8192, 1, 9000, 0], 0, 0)
    i4, i8 = plan[:128].view(np.int32), plan[:128].view(np.int64)
    segs = plan[i4[17]:i4[18]].view(np.dtype([(n, "<i4") for n in (
        "req", "len", "kept", "key0", "seg0", "long")] + [("keep", "<i8"), ("cand", "<i8")]))
    assert i4[13] == 2 and i4[19] == 2 and len(segs) == i4[14] == 2 + 13
    for i, at, long, keep, cand in ((1, 0, 0, 100, 0), (2, 2, 1, 8292, 8193)):
        x = segs[segs["req"] == i]
        assert x["key0"].tolist() == list(range(0, lens[i], 8192)) and (x["seg0"] == at).all()
        for name, v in (("len", lens[i]), ("long", long), ("keep", keep), ("cand", cand)):
            assert (x[name] == v).all()
    # histograms and states, counts, candidates
    assert i8[13] == 2 * hkv * (4096 * 4 + 16) and i8[14] >= i8[13] + 15 * hkv * 4
    assert i8[14] % 256 == 0 and ws == i8[12] == i8[14] + (8193 + 100000) * hkv * 8


def test_evict_calls_refuse_before_they_launch():
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    plan, ws = ssa.evict_plan(shape, [100], [70], 4, 8)
    score, _ = ssa.score_plan(shape, [1], [100])
    vp, ptr = ctypes.c_void_p, plan.ctypes.data
    s = ctypes.byref(shape)

    def select(p=ptr, dev=1, scores=1, table=1, keep=1, w=1, n=ws):
        return LIB.ssa_evict_select(s, p, vp(dev), vp(scores), vp(table), vp(keep), vp(w), n, None)

    assert select(p=None) == ssa.SSA_ERR_NULL and select(dev=0) == ssa.SSA_ERR_NULL
    assert select(p=score.ctypes.data) == ssa.SSA_ERR_PLAN_MISMATCH
    for name in ("scores", "table", "keep"):
        assert select(**{name: 0}) == ssa.SSA_ERR_NULL
    assert select(w=0) == select(n=ws - 1) == ssa.SSA_ERR_WORKSPACE
    assert select(scores=24, w=16) == select(scores=16, w=8) == ssa.SSA_ERR_ARG

    def compact(p=ptr, dev=1, keep=1, table=1, new=1, k=1, v=1):
        return LIB.ssa_evict_compact(s, p, vp(dev), vp(keep), vp(table), vp(new), vp(k), vp(v),
                                     None, None)

    assert compact(p=score.ctypes.data) == ssa.SSA_ERR_PLAN_MISMATCH
    for name in ("p", "dev", "keep", "table", "new", "k", "v"):
        assert compact(**{name: None if name == "p" else 0}) == ssa.SSA_ERR_NULL
    assert compact(k=8, v=16) == compact(k=16, v=8) == ssa.SSA_ERR_ARG
    whole, _ = ssa.evict_plan(shape, [100], [100], 0, 0)
    assert LIB.ssa_evict_compact(s, whole.ctypes.data, vp(1), None, None, None, None, None, None,
                                 None) == ssa.SSA_OK  # nothing moves


def test_evict_tables_are_checked():
    shape = ssa.make_shape(8, 2, 64, 30, 5, 0.125)
    plan, _ = ssa.evict_plan(shape, [70, 33, 16], [40, 33, 8], 0, 0)
    old = np.array([[1, 2, 3, 4, 5], [6, 7, 8, -1, -1], [9, -1, -1, -1, -1]])
    new = np.array([[10, 11, 12, -1, -1], [-1] * 5, [13, -1, -1, -1, -1]])
    ssa.check_evict_tables(shape, plan, old)
    ssa.check_evict_tables(shape, plan, old, new)

    def refused(o, n):
        with pytest.raises(ssa.SsaError) as e:
            ssa.check_evict_tables(shape, plan, o, n)
        assert e.value.code == -6

    for at, page in (((0, 4), 30), ((0, 0), -1), ((2, 0), 1 << 30)):
        bad = old.copy()
        bad[at] = page
        refused(bad, None)
    for at, page in (((0, 2), 30), ((0, 0), -1), ((2, 0), 10), ((0, 0), 7), ((0, 1), 9), ((2, 0), 9)):
        bad = new.copy()  # outside the pool, named twice, or a page that is in use
        bad[at] = page
        refused(old, bad)
    with pytest.raises(ValueError):
        ssa.check_evict_tables(shape, plan, old[:2])


def test_rope_append_shifted_refuses_bad_shifts():
    shape = ssa.make_shape(8, 8, 64, 100, 4, 0.125)
    plan, _ = ssa.ssa_plan(shape, [1, 3, 0], [10, 20, 50])
    vp = ctypes.c_void_p

    def call(shift, most, dev=1):
        s = np.asarray(shift, np.int32)
        return LIB.ssa_rope_append_shifted(ctypes.byref(shape), plan.ctypes.data, vp(1), None,
                                           vp(1), most, s.ctypes.data, vp(dev), vp(1), vp(1),
                                           vp(1), vp(1), None)

    assert call([0, 0, 0], 22) == ssa.SSA_ERR_ARG       # position 22
    assert call([0, 0, 0], 23) == ssa.SSA_ERR_NULL      # the positions are fine, qkv is missing
    assert call([13, 0, 0], 23) == ssa.SSA_ERR_ARG
    assert call([12, 0, 99], 23) == ssa.SSA_ERR_NULL    # a request without new tokens
    assert call([0, -1, 0], 1000) == ssa.SSA_ERR_ARG
    assert call([2 ** 31 - 1, 0, 0], 1000) == ssa.SSA_ERR_ARG
    assert call([0, 0, 0], 1000, dev=0) == ssa.SSA_ERR_NULL


def test_an_evicting_layer_refuses_before_it_launches():
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    c, u = [1, 3], [10, 20]
    plan, _ = ssa.ssa_plan(shape, c, u)
    vp = ctypes.c_void_p
    w = ssa.SsaLayerWeights(16, 16, 16, 16, 16, 16, 16, 256, 128, 64, 1e-5)

    def call(e, position=64, ws=1 << 30):
        w.max_position = position
        return LIB.ssa_layer_forward_evicting(
            ctypes.byref(shape), plan.ctypes.data, vp(16), ctypes.byref(w),
            None if e is None else ctypes.byref(e), vp(16), vp(16), vp(16), vp(16), vp(16), vp(16),
            ws, None)

    def scored(plan, **more):
        return ssa.SsaLayerEviction(**{**dict(
            score_plan_host=plan.ctypes.data, score_plan_dev=16, scores_out=16, score_workspace=16,
            score_ws_bytes=1 << 20, decay=1.0), **more})

    assert call(None) == ssa.SSA_ERR_NULL
    good, ws = ssa.score_plan(shape, c, u)
    for other in ([1, 3, 0], [20, 10, 5]), ([1, 2], [10, 20]), ([2, 2], [10, 20]):
        bad, _ = ssa.score_plan(shape, *other)
        assert call(scored(bad)) == ssa.SSA_ERR_PLAN_MISMATCH
    assert call(scored(plan)) == ssa.SSA_ERR_PLAN_MISMATCH
    assert call(scored(good, score_ws_bytes=ws - 1)) == ssa.SSA_ERR_WORKSPACE
    assert call(scored(good, score_plan_dev=None)) == ssa.SSA_ERR_NULL
    assert call(scored(good, scores_out=None)) == ssa.SSA_ERR_NULL
    assert call(scored(good, scores_out=8)) == ssa.SSA_ERR_ARG
    assert call(scored(good, decay=-1.0)) == ssa.SSA_ERR_ARG
    assert call(scored(good), ws=256) == ssa.SSA_ERR_WORKSPACE
    shift = np.array([0, 41], np.int32)
    e = ssa.SsaLayerEviction(shift_host=shift.ctypes.data, shift_dev=16)
    assert call(e, position=63) == ssa.SSA_ERR_ARG  # position 63
    assert call(ssa.SsaLayerEviction(shift_host=shift.ctypes.data)) == ssa.SSA_ERR_NULL
    assert call(ssa.SsaLayerEviction(shift_dev=16)) == ssa.SSA_ERR_NULL
    shift[0] = -1
    assert call(e) == ssa.SSA_ERR_ARG


def test_oracle_scores_against_one_weight_at_a_time():
    """The oracle's scores of a small batch, weight by weight with Python floats."""
    import math
    shape = workload.Shape(4, 2, 64)
    b = workload.make_batch(shape, [3, 1, 0], [5, 18, 7], seed=2, spare_pages=3)
    from oracle import oracle
    kc, _ = oracle.batch_kv_append(b)
    old = np.random.default_rng(0).random((b.num_pages, 2, 16))
    got, _ = oev.key_scores(b, kc, window=2, old=old, decay=0.5)
    f = lambda bits: workload.bf16_bits_to_f32(bits).astype(float)  # noqa: E731
    for i, row0, c, u, rows in ((0, 0, 3, 5, (1, 2)), (1, 3, 1, 18, (0,))):
        for h in range(2):
            at = [(b.block_table[i, t // 16], h, t % 16) for t in range(u + c)]
            want = [0.5 * old[x] if t < u else 0.0 for t, x in enumerate(at)]
            for j in rows:
                for head in (2 * h, 2 * h + 1):
                    q = f(b.q[row0 + j, head])
                    e = [math.exp(shape.softmax_scale * float(q @ f(kc[x]))) for x in at[:u + j + 1]]
                    for t, x in enumerate(e):
                        want[t] += x / math.fsum(e)
            assert np.allclose([got[x] for x in at], want, rtol=1e-12)
    assert np.isnan(got[b.block_table[2, 0]]).all()
    used = sum(-(-n // 16) for n in (8, 19))
    assert (~np.isnan(got)).sum() == 2 * (8 + 19) and used == 3


def test_oracle_selection_by_hand():
    x = np.array([0.0, 5, 1, 7, 7, np.nan, -np.inf, 7, 2, 9], dtype=np.float32)
    assert oev.select(x, 4, 1, 1).tolist() == [0, 3, 4, 9]
    assert oev.select(x, 5, 0, 0).tolist() == [1, 3, 4, 7, 9]
    assert oev.select(x, 9, 0, 1).tolist() == [0, 1, 2, 3, 4, 5, 7, 8, 9]  # NaN before -inf by index
    assert oev.select(x, 2, 2, 0).tolist() == [0, 1]
    assert oev.select(x, 10, 0, 0).tolist() == list(range(10))


def test_an_evicting_layer_takes_a_score_plan_of_its_own_batch_only():
    """Lengths of every request count: a plan of an earlier iteration, or with two
    requests' lengths exchanged, names other pages and other keys."""
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    vp = ctypes.c_void_p
    w = ssa.SsaLayerWeights(16, 16, 16, 16, 16, 16, 16, 256, 128, 64, 1e-5)

    def call(c, u, scored_c, scored_u):
        """Past the plans' check it ends at the layer's workspace, which is too small."""
        plan, _ = ssa.ssa_plan(shape, c, u)
        score, _ = ssa.score_plan(shape, scored_c, scored_u)
        e = ssa.SsaLayerEviction(score_plan_host=score.ctypes.data, score_plan_dev=16,
                                 scores_out=16, score_workspace=16, score_ws_bytes=1 << 20,
                                 decay=1.0)
        return LIB.ssa_layer_forward_evicting(
            ctypes.byref(shape), plan.ctypes.data, vp(16), ctypes.byref(w), ctypes.byref(e), vp(16),
            vp(16), vp(16), vp(16), vp(16), vp(16), 256, None)

    def refused(*a):
        return call(*a) == ssa.SSA_ERR_PLAN_MISMATCH

    assert call([1, 1], [10, 20], [1, 1], [10, 20]) == ssa.SSA_ERR_WORKSPACE
    assert call([3, 0, 1], [9, 30, 20], [3, 0, 1], [9, 30, 20]) == ssa.SSA_ERR_WORKSPACE
    assert refused([1, 1], [10, 20], [1, 1], [9, 19])       # the iteration before
    assert refused([1, 1], [10, 20], [1, 1], [30, 20])      # before an eviction
    assert refused([1, 1], [10, 20], [1, 1], [20, 10])
    assert refused([3, 1], [10, 20], [1, 3], [10, 20])
    assert refused([3, 1], [10, 20], [1, 3], [20, 10])
    assert refused([1, 0, 1], [10, 5, 20], [1, 1, 0], [10, 5, 20])


@pytest.mark.parametrize("n", [0, 1, 7, 8, 9, 200])
def test_a_score_plan_names_its_batch(n):
    rng = np.random.default_rng(n)
    c, u = rng.integers(0, 3, n).astype(np.int32), rng.integers(0, 300, n).astype(np.int32)
    shape = shape_of(8, 2, 64, c + u if n else [])
    plan = np.full(ssa.score_plan(shape, c, u)[0].nbytes, 0xA5, np.uint8)
    ssa.score_plan(shape, c, u, out=plan)
    h, _ = parse(plan)
    assert h["off_items"] % 64 == 0 and h["off_items"] >= 128 + 8 * n
    reqs = plan[128:128 + 8 * n].view(np.int32).reshape(n, 2)
    assert np.array_equal(reqs[:, 0], c) and np.array_equal(reqs[:, 1], u)
    assert not plan[128 + 8 * n:h["off_items"]].any()


def test_misaligned_plans_are_refused():
    """plan_dev at another multiple than 8: the kernels would read another header, write
    nothing and say nothing.  Only calls with something to do look at it."""
    shape = ssa.make_shape(8, 2, 64, 100, 20, 0.125)
    s, vp = ctypes.byref(shape), ctypes.c_void_p
    score, ws = ssa.score_plan(shape, [1, 1], [10, 20])
    evict, ews = ssa.evict_plan(shape, [100], [70], 4, 8)
    plan, _ = ssa.ssa_plan(shape, [1, 1], [10, 20])
    w = ssa.SsaLayerWeights(16, 16, 16, 16, 16, 16, 16, 256, 128, 64, 1e-5)
    p = vp(16)
    for dev in (4097, 4098, 4100, 4092):
        at = vp(dev)
        assert call_scores(shape, score, dev=dev) == ssa.SSA_ERR_ARG
        assert call_scores(shape, score, dev=dev, fn="ssa_decode_scored", n_ptr=16) == ssa.SSA_ERR_ARG
        assert LIB.ssa_evict_select(s, evict.ctypes.data, at, p, p, p, p, ews, None) == ssa.SSA_ERR_ARG
        assert LIB.ssa_evict_compact(s, evict.ctypes.data, at, p, p, p, p, p, p,
                                     None) == ssa.SSA_ERR_ARG
        e = ssa.SsaLayerEviction(score_plan_host=score.ctypes.data, score_plan_dev=dev,
                                 scores_out=16, score_workspace=16, score_ws_bytes=ws, decay=1.0)
        assert LIB.ssa_layer_forward_evicting(s, plan.ctypes.data, p, ctypes.byref(w),
                                              ctypes.byref(e), p, p, p, p, p, p, 1 << 30,
                                              None) == ssa.SSA_ERR_ARG


@pytest.mark.parametrize("seed", range(10))
def test_norms_of_chunk_columns_have_room_for_two_numbers(seed):
    """A padded column's maximum and reciprocal sum per kv head: no other range of the
    workspace begins within them."""
    rng = np.random.default_rng(100 + seed)
    c, u = rng.choice([2, 17, 64, 300, 1000], 5), rng.choice([0, 40, 5000, 30000], 5)
    hq, hkv, d = [(8, 8, 64), (32, 8, 128), (28, 4, 128), (16, 1, 64), (5, 5, 128)][seed % 5]
    plan, ws = ssa.score_plan(shape_of(hq, hkv, d, c + u), c, u)
    h, items = parse(plan)
    starts = {int(x[f]) for n in LISTS for x in items[n] for f in ("off0", "off1")
              if f == "off0" or x["nsplit"] > 1} | {ws // 4}
    for x in items["lse"]:
        end = int(x["off0"]) + 2 * hkv * int(x["cols_pad"])
        assert end <= ws // 4 and not any(x["off0"] < s < end for s in starts)
