"""GPU tests of ssa_pages_resize (include/ssa_pages.h), of the rotary forms
(ssa_rope_append_as) and of a serving run of them with the sparse attention.

Whole numbers are compared bit for bit with the oracle (oracle/sparse.py).  Rotated values:
two products and their sum in fp32 (each off by 2^-24 of its value, the table's entries by
2^-24 too) and one rounding to bf16:
    |err| <= 2^-8 |ref| + 5 2^-24 (|a c| + |b s|).
"""
import numpy as np
import pytest

from test_gpu_evict import dev, say
from test_gpu_sparse import bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    return torch


class Pages:
    """Requests' tables and the free pages on the device, beside the oracle's."""

    def __init__(self, torch, n, num_pages, width, rng, rows):
        from paper_2606_05933_amd import ssa
        self.torch, self.ssa, self.n, self.num_pages = torch, ssa, n, num_pages
        self.shape = ssa.make_shape(8, 2, 64, num_pages, width, 0.1)
        self.table = np.full((n, width), -1, np.int32)
        self.ring = rng.permutation(num_pages).astype(np.int32)
        self.state = np.array([int(rng.integers(num_pages)), num_pages, 0, 0])
        self.len = np.zeros(n, np.int64)
        self.dev = {"table": dev(torch, self.table), "ring": dev(torch, self.ring)}
        self.states = [dev(torch, self.state.astype(np.int32)), dev(torch, np.zeros(4, np.int32))]
        self.row_start = torch.full((n + 2,), -3, dtype=torch.int32, device="cuda")
        self.slots = torch.full((rows,), -3, dtype=torch.int64, device="cuda")

    def call(self, new, slots=True, row_start=True):
        t = self.torch
        self.ssa.pages_resize(self.shape, dev(t, self.len.astype(np.int32)),
                              dev(t, np.asarray(new, np.int32)), self.dev["table"],
                              self.dev["ring"], *self.states,
                              self.row_start if row_start else None, self.slots if slots else None)
        self.states.reverse()

    def resize(self, new):
        from oracle import sparse
        self.row_start.fill_(-3)
        self.slots.fill_(-3)
        self.call(new)
        self.table, self.ring, self.state, starts, slots = sparse.pages(
            self.table, self.ring, self.state, self.len, new, self.num_pages)
        self.len = np.asarray(new, np.int64)
        got = self.slots.cpu().numpy()
        assert np.array_equal(got[:len(slots)], slots) and (got[len(slots):] == -3).all()
        assert np.array_equal(self.row_start.cpu().numpy(), [*starts, -3])
        self.same()

    def same(self):
        assert np.array_equal(self.dev["table"].cpu().numpy(), self.table)
        assert np.array_equal(self.dev["ring"].cpu().numpy(), self.ring)
        assert np.array_equal(self.states[0].cpu().numpy(), self.state)


@pytest.mark.parametrize("n,longest", [(1, 5), (1, 3000), (7, 100), (64, 700), (500, 300),
                                       (5000, 20)])
def test_requests_grow_shrink_and_end(torch_dev, n, longest):
    rng = np.random.default_rng(n + longest)
    say(f"[gpu pages] n={n} longest={longest}")
    width = -(-longest // 16)
    p = Pages(torch_dev, n, max(2, n * width * 3 // 4), width, rng, n * longest + 1)
    for _ in range(8):
        new = np.where(rng.random(n) < 0.3, rng.integers(0, longest + 1, n),
                       np.minimum(p.len + rng.integers(0, 3, n), longest))
        new[rng.random(n) < 0.1] = 0
        need = lambda x: -(-x // 16)  # noqa: E731
        while np.maximum(need(new) - need(p.len), 0).sum() > p.state[1]:
            i = rng.integers(n)
            new[i] = p.len[i] if rng.random() < 0.9 else 0
            new[np.flatnonzero(new > p.len)[::2]] -= 0
            over = np.flatnonzero(new > p.len)
            if len(over):
                new[over[0]] = p.len[over[0]]
        p.resize(new)
    held = [x for i in range(n) for x in p.table[i, :-(-int(p.len[i]) // 16)]]
    free = [p.ring[(p.state[0] + k) % p.num_pages] for k in range(p.state[1])]
    assert sorted(held + free) == list(range(p.num_pages)), "a page is lost or held twice"


@pytest.mark.parametrize("n", [513, 1025, 32769, 65536])
def test_more_requests_than_waves(torch_dev, n):
    rng = np.random.default_rng(n)
    p = Pages(torch_dev, n, 3 * n, 3, rng, 48 * n)
    p.resize(rng.integers(0, 49, n))
    new = rng.integers(0, 49, n)
    free = p.state[1]
    new[np.cumsum(np.maximum(-(-new // 16) - -(-p.len // 16), 0)) > free] = 0
    p.resize(new)


def test_no_requests_and_maps_left_out(torch_dev):
    rng = np.random.default_rng(0)
    p = Pages(torch_dev, 0, 9, 3, rng, 1)
    p.resize([])
    p = Pages(torch_dev, 3, 9, 3, rng, 200)
    p.call([17, 0, 16], slots=False, row_start=False)
    from oracle import sparse
    p.table, p.ring, p.state, _, _ = sparse.pages(p.table, p.ring, p.state, p.len, [17, 0, 16], 9)
    p.same()
    assert (p.slots == -3).all() and (p.row_start == -3).all()


@pytest.mark.parametrize("what", ["short", "negative", "wide", "old", "rows", "head", "count", "full"])
def test_what_the_device_refuses_changes_nothing(torch_dev, what):
    rng = np.random.default_rng(1)
    p = Pages(torch_dev, 4, 12, 5, rng, 200)
    p.resize([16, 17, 0, 40])  # 1 + 2 + 0 + 3 pages
    new, status, missing = [20, 20, 5, 41], 0, 0
    state = p.states[0]
    if what == "short":
        new, status, missing = [80, 80, 5, 40], p.ssa.PAGES_SHORT, 4 + 3 + 1 - 6
    elif what == "negative":
        new[2], status = -1, p.ssa.PAGES_LENGTH
    elif what == "wide":
        new[2], status = 81, p.ssa.PAGES_LENGTH
    elif what == "old":
        p.len[1], status = 1 << 30, p.ssa.PAGES_LENGTH
    elif what == "rows":
        p.slots, status = p.slots[:12], p.ssa.PAGES_ROWS  # 4 + 3 + 5 + 1
    elif what == "head":
        state[0], p.state[0], status = 12, 12, p.ssa.PAGES_RING
    elif what == "count":
        state[1], p.state[1], status = -1, -1, p.ssa.PAGES_RING
    else:  # more pages come back than were taken
        state[1], p.state[1], status = 12, 12, p.ssa.PAGES_RING
        new = [0, 17, 0, 40]
    p.row_start.fill_(-3)
    p.slots.fill_(-3)
    p.call(new)
    p.state = np.array([p.state[0], p.state[1], status, missing])
    p.same()
    assert (p.slots == -3).all() and (p.row_start == -3).all()


def test_a_slot_map_without_room(torch_dev):
    """Room for no row: growing requests are refused, and shrinking ones are not."""
    rng = np.random.default_rng(2)
    p = Pages(torch_dev, 2, 9, 4, rng, 0)
    p.row_start.fill_(-3)
    p.call([17, 0])
    p.state = np.array([p.state[0], p.state[1], p.ssa.PAGES_ROWS, 0])
    p.same()
    assert (p.row_start == -3).all()
    q = Pages(torch_dev, 2, 9, 4, rng, 40)
    q.resize([17, 20])
    q.slots = q.slots[:0]
    q.resize([5, 20])


FORMS = [("half", None), ("half", 32), ("half", 16), ("half", 48), ("interleaved", None),
         ("interleaved", 32), ("interleaved", 16)]


@pytest.mark.parametrize("layout,rotary", FORMS)
@pytest.mark.parametrize("hq,hkv,d,cu", [
    (8, 8, 64, [(64, 192), (1, 128), (1, 256), (0, 3)]),
    (28, 4, 128, [(100, 1000), (1, 4095), (1, 16), (33, 7)]),
    (160, 10, 64, [(3, 5), (1, 0)]),  # a row of more heads than one workgroup takes
])
@pytest.mark.parametrize("shifted", [False, True])
def test_rope_forms(torch_dev, layout, rotary, hq, hkv, d, cu, shifted):
    from oracle import sparse
    from paper_2606_05933_amd import ssa, workload
    torch = torch_dev
    r = rotary or d
    say(f"[gpu rope form] {layout} {rotary} {hq}/{hkv}/{d} shifted={shifted}")
    b = workload.make_batch(workload.Shape(hq, hkv, d), [c for c, _ in cu], [u for _, u in cu],
                            seed=r, spare_pages=3)
    T = b.num_tokens
    shift = np.arange(len(cu), dtype=np.int32) * 37 if shifted else np.zeros(len(cu), np.int32)
    most = int((b.q_len + b.ctx_len + shift).max())
    angle = np.arange(most)[:, None] * sparse.angles(r, 1e4, "parts", 4.0, 1000, 1.0, 4.0)
    table = ssa.rope_cos_sin_scaled(most, r, 1e4, "parts", 4.0, 1000, 1.0, 4.0)
    shape = ssa.make_shape(hq, hkv, d, b.num_pages, b.max_pages_per_req, 0.1)
    plan, _ = ssa.ssa_plan(shape, b.q_len, b.ctx_len)
    qkv = np.concatenate([b.q, b.k_new, b.v_new], axis=1)
    k, v = dev(torch, b.k_cache), dev(torch, b.v_cache)
    q_out = torch.full((T + 1, hq, d), 3.0, dtype=torch.bfloat16, device="cuda")
    more = dict(shift_host=shift, shift_dev=dev(torch, shift)) if shifted else {}
    args = (shape, plan, dev(torch, plan), dev(torch, qkv), dev(torch, table))
    ssa.rope_append_as(*args, q_out, k, v, dev(torch, b.block_table), layout=layout,
                       rotary_dim=rotary, **more)
    req = np.repeat(np.arange(len(cu)), b.q_len)
    t = np.concatenate([np.arange(u, u + c) for c, u in cu]).astype(int)
    x = sparse._f64(qkv[:, :hq + hkv])
    a = angle[t + shift[req]]
    ref = sparse.rotate(x, np.cos(a), np.sin(a), layout, r)
    size = sparse.rotate(np.abs(x), np.abs(np.cos(a)), np.abs(np.sin(a)), layout, r)
    size = size + 2 * np.abs(x)  # at least |a c| + |b s|, whatever the sign between them
    page, slot = b.block_table[req, t // 16], t % 16
    kc, vc = bits(k), bits(v)
    got = sparse._f64(np.concatenate([bits(q_out)[:T], kc[page, :, slot]], axis=1))
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 5 * 2.0 ** -24 * size).all()
    assert np.array_equal(got[:, :, r:], x[:, :, r:]), "dims that do not turn"
    assert (q_out[-1] == 3.0).all()
    want = b.v_cache.copy()
    want[page, :, :, slot] = b.v_new
    assert np.array_equal(vc, want)
    rest = np.ones((b.num_pages, 16), bool)
    rest[page, slot] = False
    assert np.array_equal(kc.transpose(0, 2, 1, 3)[rest], b.k_cache.transpose(0, 2, 1, 3)[rest])
    if layout == "half" and r == d and not shifted:
        k2, v2, q2 = dev(torch, b.k_cache), dev(torch, b.v_cache), torch.empty_like(q_out)
        ssa.rope_append(*args, q2, k2, v2, dev(torch, b.block_table))
        assert np.array_equal(bits(k2), kc) and np.array_equal(bits(q2)[:T], bits(q_out)[:T])


def test_a_serving_run(torch_dev):
    """Requests come, decode and end: pages from their lengths, RoPE + append, summaries,
    scores, lists and attention, each step against the oracle on the same rotated rows."""
    import types

    from oracle import sparse
    from paper_2606_05933_amd import ssa, workload
    torch = torch_dev
    hq, hkv, d, block, top = 8, 2, 64, 32, 4
    rng = np.random.default_rng(3)
    n, num_pages, width = 5, 90, 40
    p = Pages(torch, n, num_pages, width, rng, 400)
    shape = p.shape = ssa.make_shape(hq, hkv, d, num_pages, width, 0.125)
    k = torch.full((num_pages, hkv, 16, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    v = torch.full((num_pages, hkv, d, 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    summary = torch.full((num_pages, hkv, 2, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    table = dev(torch, ssa.rope_cos_sin_scaled(700, 32, 1e4, "linear", 2.0))
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    steps = [[200, 0, 37, 0, 1], [201, 130, 38, 0, 2], [0, 131, 39, 16, 3], [3, 132, 40, 17, 30],
             [4, 133, 0, 18, 31], [300, 100, 1, 19, 32], [301, 101, 2, 20, 33]]
    for new in steps:
        old = p.len
        p.resize(new)
        c = np.maximum(np.asarray(new) - old, 0)
        u = np.where(c > 0, old, 0)
        T = int(c.sum())
        qkv = workload.normal_bf16((T, (hq + 2 * hkv) * d), int(rng.integers(1 << 30)))
        plan, _ = ssa.ssa_plan(shape, c, u)
        sp, need, stride = ssa.sparse_plan(shape, c, u, block, top, 1, 1)
        assert need <= ws.numel()
        pd, sd = dev(torch, plan), dev(torch, sp)
        q = torch.zeros((T, hq, d), dtype=torch.bfloat16, device="cuda")
        scores = torch.zeros((T, hkv, stride), device="cuda")
        blocks = torch.zeros((T, hkv, top), dtype=torch.int32, device="cuda")
        out = torch.zeros((T, hq, d), dtype=torch.bfloat16, device="cuda")
        bt = p.dev["table"]
        ssa.rope_append_as(shape, plan, pd, dev(torch, qkv), table, q, k, v, bt,
                           layout="interleaved", rotary_dim=32)
        ssa.block_summary(shape, plan, pd, block, k, bt, summary)
        ssa.block_scores(shape, sp, sd, q, summary, bt, scores)
        ssa.block_select(shape, sp, sd, scores, blocks)
        ssa.sparse_attention(shape, sp, sd, q, k, v, bt, blocks, out, ws)
        b = types.SimpleNamespace(shape=workload.Shape(hq, hkv, d, scale=0.125), q_len=c, ctx_len=u,
                                  block_table=p.table, q=bits(q), num_reqs=n, num_tokens=T)
        kc, vc, lists, got = bits(k), bits(v), blocks.cpu().numpy(), scores.cpu().numpy()
        slots = p.slots[:T].cpu().numpy()
        assert np.array_equal(vc[slots // 16, :, :, slots % 16],
                              qkv.reshape(T, -1, d)[:, hq + hkv:]), "rows lie in their slots"
        row = 0
        for i in range(n):
            for j in range(c[i]):
                m = (u[i] + j) // block + 1
                for h in range(hkv):
                    keys = sparse._f64(sparse.cached(b, kc, i, h, u[i] + c[i]))
                    part = [keys[x * block:(x + 1) * block] for x in range(m)]
                    ref, size = sparse.bounds(sparse._f64(b.q[row, 4 * h:4 * h + 4]),
                                              np.stack([x.max(axis=0) for x in part]),
                                              np.stack([x.min(axis=0) for x in part]))
                    assert (np.abs(got[row, h, :m] - ref) <= 2 * d * 2.0 ** -24 * size).all()
                    assert np.array_equal(lists[row, h], sparse.select(got[row, h, :m], top, 1, 1))
                row += 1
        ref, mass, a = sparse.attention(b, kc, vc, lists, block)
        rel = 2.0 ** -24 * (2 * (2 * d * a + 8 * a + 2 * top * block / 32 + 256) + 1)
        err = np.abs(out.float().cpu().numpy() - ref)
        assert (err <= 2.0 ** -8 * np.abs(ref) + rel * mass).all()


def layer_setup(torch, hq, hkv, d, cu, hidden=256, inter=128, seed=5, **weights):
    from paper_2606_05933_amd import ssa, workload
    c, u = [p[0] for p in cu], [p[1] for p in cu]
    b = workload.make_batch(workload.Shape(hq, hkv, d), c, u, seed=seed, spare_pages=5)
    shape = ssa.make_shape(hq, hkv, d, b.num_pages, b.max_pages_per_req, d ** -0.5)
    host = workload.layer_weights(seed, hidden, inter, hq, hkv, d)
    w = ssa.LayerWeights(host, hq, hkv, d, 2048, **weights)
    plan, _ = ssa.ssa_plan(shape, b.q_len, b.ctx_len)
    x = workload.normal_bf16((b.num_tokens, hidden), seed + 1)
    ws = torch.zeros(ssa.layer_workspace_size(shape, plan, w), dtype=torch.uint8, device="cuda")
    return b, shape, host, w, plan, x, ws


def test_a_layer_without_its_sparse_parts_is_the_layer(torch_dev):
    from paper_2606_05933_amd import ssa
    torch = torch_dev
    b, shape, _, w, plan, x, ws = layer_setup(torch, 8, 2, 64, [(20, 30), (1, 100), (0, 4)])
    pd, table, xd = dev(torch, plan), dev(torch, b.block_table), dev(torch, x)
    got = []
    for sparse in (False, True):
        k, v, out = dev(torch, b.k_cache), dev(torch, b.v_cache), torch.empty_like(xd)
        call = ssa.layer_forward_sparse if sparse else ssa.layer_forward
        call(shape, plan, pd, w, xd, out, k, v, table, ws)
        got.append([bits(t) for t in (out, k, v)])
    assert all(np.array_equal(p, q) for p, q in zip(*got))


def test_a_sparse_layer_over_all_blocks_matches_the_oracle(torch_dev):
    """Lists of every block: the dense layer's bar (seven bf16 tensors between x and out, each
    at most a step apart from the oracle's)."""
    from oracle import layer as olay
    from paper_2606_05933_amd import ssa
    torch = torch_dev
    hq, hkv, d = 8, 2, 64
    b, shape, host, w, plan, x, ws = layer_setup(torch, hq, hkv, d, [(20, 30), (1, 100), (1, 5), (37, 0)])
    T = b.num_tokens
    sp, need, stride = ssa.sparse_plan(shape, b.q_len, b.ctx_len, 16, 8)
    k, v = dev(torch, b.k_cache), dev(torch, b.v_cache)
    out = torch.zeros((T, 256), dtype=torch.bfloat16, device="cuda")
    # the cached keys' summaries first
    summary = torch.zeros((b.num_pages, hkv, 2, d), dtype=torch.bfloat16, device="cuda")
    held = np.where(b.q_len > 0, b.ctx_len, 0)
    whole, _ = ssa.ssa_plan(shape, held, 0 * held)
    ssa.block_summary(shape, whole, dev(torch, whole), 16, k, dev(torch, b.block_table), summary)
    ssa.layer_forward_sparse(
        shape, plan, dev(torch, plan), w, dev(torch, x), out, k, v, dev(torch, b.block_table), ws,
        summary=summary, block_keys=16, sparse_plan_host=sp, sparse_plan_dev=dev(torch, sp),
        scores=torch.zeros((T, hkv, stride), device="cuda"),
        blocks=torch.zeros((T, hkv, 8), dtype=torch.int32, device="cuda"),
        sparse_workspace=torch.zeros(need, dtype=torch.uint8, device="cuda"))
    ref, _, _ = olay.decoder_layer(x, host, hq, hkv, d, b.q_len, b.ctx_len, b.block_table, b.k_cache,
                                   b.v_cache, eps=1e-5)
    got = out.float().cpu().numpy().astype(np.float64)
    err = np.abs(got - ref)
    say(f"    out: max_abs={err.max():.3e} mean_abs={err.mean():.3e}")
    assert (err <= 2.0 ** -5 * (np.abs(ref) + 1.0)).all() and err.mean() <= 3e-3


@pytest.mark.parametrize("selected", [False, True])
@pytest.mark.parametrize("hq,hkv,d,cu", [(8, 2, 64, [(20, 300), (1, 700), (0, 4), (1, 3)]),
                                         (4, 1, 128, [(1, 900), (1, 40)])])
def test_a_sparse_layer_is_its_calls(torch_dev, hq, hkv, d, cu, selected):
    """Bit for bit the sequence of the public calls, eagerly and replayed from a graph."""
    from paper_2606_05933_amd import ssa
    torch = torch_dev
    table = ssa.rope_cos_sin_scaled(2048, 32, 1e4, "base", 2.0)
    b, shape, _, w, plan, x, ws = layer_setup(torch, hq, hkv, d, cu, cos_sin=table)
    T, hidden, block, top = b.num_tokens, 256, 32, 5
    pd, bt, xd = dev(torch, plan), dev(torch, b.block_table), dev(torch, x)
    shift = np.arange(len(cu), dtype=np.int32) * 11
    sd = dev(torch, shift)
    sp, need, stride = ssa.sparse_plan(shape, b.q_len, b.ctx_len, block, top)
    spd = dev(torch, sp)
    sws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    held = np.where(b.q_len > 0, b.ctx_len, 0)
    whole, _ = ssa.ssa_plan(shape, held, 0 * held)
    wd = dev(torch, whole)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    state = {"k": bf(*b.k_cache.shape), "v": bf(*b.v_cache.shape), "out": bf(T, hidden),
             "summary": bf(b.num_pages, hkv, 2, d),
             "scores": torch.zeros((T, hkv, stride), device="cuda"),
             "blocks": torch.zeros((T, hkv, top), dtype=torch.int32, device="cuda")}
    first = [dev(torch, b.k_cache), dev(torch, b.v_cache)]

    def reset():
        for t in state.values():
            t.zero_()
        state["k"].copy_(first[0])
        state["v"].copy_(first[1])
        ssa.block_summary(shape, whole, wd, block, state["k"], bt, state["summary"])

    def layer():
        s = state
        more = dict(sparse_plan_host=sp, sparse_plan_dev=spd, scores=s["scores"], blocks=s["blocks"],
                    sparse_workspace=sws) if selected else {}
        ssa.layer_forward_sparse(shape, plan, pd, w, xd, s["out"], s["k"], s["v"], bt, ws,
                                 layout="interleaved", rotary_dim=32, shift_host=shift, shift_dev=sd,
                                 summary=s["summary"], block_keys=block, **more)

    def calls():
        s = state
        xn, qkv, q, a = bf(T, hidden), bf(T, (hq + 2 * hkv) * d), bf(T, hq, d), bf(T, hq, d)
        h, act = bf(T, hidden), bf(T, w.inter)
        gws = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
        ssa.rms_norm(xd, w.attn_norm, xn)
        ssa.linear(xn, w.w_qkv, qkv, workspace=gws)
        ssa.rope_append_as(shape, plan, pd, qkv, w.cos_sin, q, s["k"], s["v"], bt, "interleaved", 32,
                           shift, sd)
        ssa.block_summary(shape, plan, pd, block, s["k"], bt, s["summary"])
        if selected:
            ssa.block_scores(shape, sp, spd, q, s["summary"], bt, s["scores"])
            ssa.block_select(shape, sp, spd, s["scores"], s["blocks"])
            ssa.sparse_attention(shape, sp, spd, q, s["k"], s["v"], bt, s["blocks"], a, sws)
        else:
            _, aws = ssa.ssa_plan_size(shape, b.q_len, b.ctx_len)
            ssa.ssa_mixed_attention(shape, plan, pd, q, s["k"], s["v"], bt, a,
                                    torch.zeros(aws, dtype=torch.uint8, device="cuda"))
        ssa.linear(a.view(T, -1), w.w_o, h, ssa.EPILOGUE_RESIDUAL, residual=xd, workspace=gws)
        ssa.rms_norm(h, w.mlp_norm, xn)
        ssa.linear(xn, w.w_gate_up, act, ssa.EPILOGUE_SWIGLU, workspace=gws)
        ssa.linear(act, w.w_down, s["out"], ssa.EPILOGUE_RESIDUAL, residual=h, workspace=gws)

    reset()
    calls()
    torch.cuda.synchronize()
    want = {n: t.clone() for n, t in state.items()}
    assert want["out"].isfinite().all()

    def same(what):
        torch.cuda.synchronize()
        for n, t in state.items():
            p, q = (y.view(torch.int16) if y.dtype == torch.bfloat16 else y for y in (t, want[n]))
            assert torch.equal(p, q), (what, n)

    reset()
    layer()
    same("eager")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            layer()
    for r in range(3):
        reset()
        torch.cuda.synchronize()
        graph.replay()
        same(r)


def test_a_sparse_layer_refuses_half_given_parts(torch_dev):
    from paper_2606_05933_amd import ssa
    torch = torch_dev
    b, shape, host, w, plan, x, ws = layer_setup(torch, 8, 2, 64, [(2, 30), (1, 5)])
    k, v, xd = dev(torch, b.k_cache), dev(torch, b.v_cache), dev(torch, x)
    before = bits(k), bits(v)
    shift = np.array([7, 9], np.int32)

    def call(**parts):
        ssa.layer_forward_sparse(shape, plan, dev(torch, plan), w, xd, torch.empty_like(xd), k, v,
                                 dev(torch, b.block_table), ws, **parts)

    for parts in (dict(shift_dev=dev(torch, shift)), dict(shift_host=shift)):
        with pytest.raises(ssa.SsaError) as e:
            call(**parts)
        assert e.value.code == ssa.SSA_ERR_NULL
    some = torch.zeros((b.num_pages, 2, 16), device="cuda")
    for name in ("scores", "blocks", "sparse_workspace", "sparse_plan_dev"):
        with pytest.raises(ValueError):
            call(**{name: some})
    with pytest.raises(ValueError):
        call(rotary_dim=32)  # the weights' table has whole rows
    part = ssa.LayerWeights(host, 8, 2, 64, 2048, cos_sin=ssa.rope_cos_sin(2048, 32))
    for f in (ssa.layer_forward, ssa.layer_forward_evicting, ssa.layer_forward_sparse):
        with pytest.raises(ValueError):  # and these would read past one of 32
            f(shape, plan, dev(torch, plan), part, xd, torch.empty_like(xd), k, v,
              dev(torch, b.block_table), ws)
    assert np.array_equal(bits(k), before[0]) and np.array_equal(bits(v), before[1])
