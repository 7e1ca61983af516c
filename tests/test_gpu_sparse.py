"""GPU parity of block summaries, scores, selection and attention over selected blocks
(include/ssa_sparse.h) with the float64 oracle (oracle/sparse.py).

Bars, from the arithmetic:
* summaries, lists: bit for bit.
* scores: a sum of 2 D products of two bf16 values (exact in fp32), each addition off by
  at most 2^-24 of a partial sum, which is at most the sum A of the terms' magnitudes:
      |err| <= 2 D 2^-24 A.
* attention: logits of D products, so off by D 2^-24 A; the exponents' fma and the
  exponential add a few 2^-24 of their argument (<= 2 A log2 e) and value; sums of
  positive terms at most 2^-24 for each of the L / 32 + 128 links of their longest chain; a
  weight enters the products whole (three bf16 parts, 2^-24); the result is rounded to
  bf16:
      |err| <= 2^-8 |ref| + 2^-24 (2 (2 D A + 8 A + 2 L / 32 + 256) + 1) sum |w v|.
"""
import numpy as np
import pytest

from test_gpu_evict import HEADS, dev, say
from test_sparse_boundary import LARGE_SCORES, parse

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    return torch


def bits(t):
    """uint16 numpy array of a bf16 tensor."""
    import torch
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


class Sparse:
    """A batch on the device, its new rows appended, with its plans."""

    def __init__(self, torch, heads, c, u, block, top, sink=1, recent=1, seed=0, plan="device",
                 scale=None):
        from oracle import oracle
        from paper_2606_05933_amd import ssa, workload
        self.torch, self.ssa, self.block = torch, ssa, block
        self.top, self.sink, self.recent = top, sink, recent
        self.b = b = workload.make_batch(workload.Shape(*heads, scale=scale), c, u, seed=seed,
                                         spare_pages=5, extra_pages_per_req=2)
        say(f"[gpu sparse] heads={heads} c={list(c)[:8]} u={list(u)[:8]} block={block} top={top} "
            f"seed={seed}")
        self.kc, self.vc = oracle.batch_kv_append(b)
        s = b.shape
        self.shape = ssa.make_shape(s.hq, s.hkv, s.d, b.num_pages, b.max_pages_per_req,
                                    s.softmax_scale)
        self.batch_plan, _ = ssa.ssa_plan(self.shape, b.q_len, b.ctx_len)
        self.plan, ws, self.max_blocks = ssa.sparse_plan(self.shape, b.q_len, b.ctx_len, block, top,
                                                         sink, recent)
        if plan == "pinned":
            self.plan = self.plan_dev = torch.from_numpy(self.plan).pin_memory()
            self.batch_plan = self.batch_dev = torch.from_numpy(self.batch_plan).pin_memory()
        else:
            self.plan_dev, self.batch_dev = dev(torch, self.plan), dev(torch, self.batch_plan)
        self.upload()
        # behind the tickets the workspace holds anything
        self.ws = torch.full((ws,), 0xFF, dtype=torch.uint8, device="cuda")
        self.ws[:4096] = 0
        T, hkv = b.num_tokens, s.hkv
        self.scores = torch.full((T, hkv, self.max_blocks), -7.0, device="cuda")
        self.blocks = torch.full((T, hkv, top), -9, dtype=torch.int32, device="cuda")
        self.out = torch.full((T + 1, s.hq, s.d), 3.0, dtype=torch.bfloat16, device="cuda")
        self.summary = dev(torch, np.full((b.num_pages, hkv, 2, s.d), 0x1234, np.uint16))

    def upload(self):
        b, torch = self.b, self.torch
        self.q, self.k, self.v = dev(torch, b.q), dev(torch, self.kc), dev(torch, self.vc)
        self.table = dev(torch, b.block_table)

    def summarise(self, stream=None):
        self.ssa.block_summary(self.shape, self.batch_plan, self.batch_dev, self.block, self.k,
                               self.table, self.summary, stream)

    def score(self, stream=None):
        self.ssa.block_scores(self.shape, self.plan, self.plan_dev, self.q, self.summary, self.table,
                              self.scores, stream)

    def select(self, stream=None):
        self.ssa.block_select(self.shape, self.plan, self.plan_dev, self.scores, self.blocks, stream)

    def attend(self, stream=None):
        self.ssa.sparse_attention(self.shape, self.plan, self.plan_dev, self.q, self.k, self.v,
                                  self.table, self.blocks, self.out, self.ws, stream)

    def rows(self):
        """(request, token row, position) of every new row."""
        row = 0
        for i in range(self.b.num_reqs):
            for j in range(int(self.b.q_len[i])):
                yield i, row, int(self.b.ctx_len[i]) + j
                row += 1

    def whole_summary(self):
        """All blocks' summaries by the oracle, on the device: bits [num_pages, Hkv, 2, D]."""
        from oracle import sparse
        b = self.b
        whole = np.full((b.num_pages, b.shape.hkv, 2, b.shape.d), 0x7FC0, np.uint16)  # NaN
        length = b.q_len + b.ctx_len
        import dataclasses
        for at, x in sparse.summary(dataclasses.replace(b, q_len=np.where(b.q_len > 0, length, 0),
                                                        ctx_len=np.zeros_like(length)),
                                    self.kc, self.block).items():
            whole[at] = x
        self.summary = dev(self.torch, whole)
        return whole

    def check_scores(self, whole):
        from oracle import sparse
        b, s = self.b, self.b.shape
        g, got = s.group, self.scores.cpu().numpy().astype(np.float64)
        for i, row, pos in self.rows():
            n = pos // self.block + 1
            at = b.block_table[i, np.arange(n) * self.block // 16]
            for h in range(s.hkv):
                hl = sparse._f64(whole[at, h])
                ref, size = sparse.bounds(sparse._f64(b.q[row, h * g:(h + 1) * g]), hl[:, 0], hl[:, 1])
                err = np.abs(got[row, h, :n] - ref)
                assert (err <= 2 * s.d * 2.0 ** -24 * size).all(), (i, row, h, err.max())
                assert (got[row, h, n:] == -7.0).all(), "scores of no block were written"

    def check_lists(self):
        from oracle import sparse
        got, scores = self.blocks.cpu().numpy(), self.scores.cpu().numpy()
        for i, row, pos in self.rows():
            for h in range(self.b.shape.hkv):
                ref = sparse.select(scores[row, h, :pos // self.block + 1], self.top, self.sink,
                                    self.recent)
                assert np.array_equal(got[row, h], ref), (i, row, h, got[row, h], ref)

    def check_out(self):
        from oracle import sparse
        b = self.b
        lists = self.blocks.cpu().numpy()
        ref, mass, a = sparse.attention(b, self.kc, self.vc, lists, self.block)
        keys = self.top * self.block
        rel = 2.0 ** -24 * (2 * (2 * b.shape.d * a + 8 * a + 2 * keys / 32 + 256) + 1)
        got = self.out.float().cpu().numpy().astype(np.float64)
        assert (got[-1] == 3.0).all(), "a row behind the last one was written"
        err, tol = np.abs(got[:-1] - ref), 2.0 ** -8 * np.abs(ref) + rel * mass
        assert (err <= tol).all(), (float(np.nanmax(err)), np.argwhere(~(err <= tol))[:5])
        assert not self.ws[:4096].any(), "tickets are left"


MIXED = [((3, 1, 0, 1, 40), (0, 15, 9, 900, 333)), ((1,), (0,)), ((1, 1, 1), (16, 31, 2000)),
         ((70, 1), (1000, 4095)), ((2, 0, 1), (127, 5, 128))]


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("cu", MIXED)
@pytest.mark.parametrize("heads", [(8, 8, 64), (28, 4, 128), (5, 5, 64), (6, 6, 128)])
def test_summaries_are_the_keys_extremes(torch_dev, heads, cu, block):
    x = Sparse(torch_dev, heads, *cu, block, 4, seed=block)
    rng = np.random.default_rng(block)
    # zeros of both signs, infinities and numbers that are none, among the keys
    odd = rng.choice(np.array([0x0000, 0x8000, 0x7F80, 0xFF80, 0x7FC1, 0xFFC1], np.uint16), x.kc.shape)
    x.kc = np.where(rng.random(x.kc.shape) < 0.02, odd, x.kc)
    x.upload()
    x.summarise()
    from oracle import sparse
    got = bits(x.summary)
    want = np.full_like(got, 0x1234)
    for at, v in sparse.summary(x.b, x.kc, block).items():
        want[at] = v
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("block,cu", [(16, MIXED[0]), (64, MIXED[3]), (32, MIXED[2]), (128, MIXED[4]),
                                      (16, ((100, 1), (2500, 6000)))])
def test_scores_bound_the_blocks(torch_dev, heads, block, cu):
    x = Sparse(torch_dev, heads, *cu, block, 4, seed=1)
    whole = x.whole_summary()
    x.score()
    x.check_scores(whole)


def test_scores_bound_every_logit(torch_dev):
    """The bound is one: no <q, k> of a block is above it (by more than its rounding)."""
    from oracle import sparse
    x = Sparse(torch_dev, (8, 2, 128), (5, 1), (700, 300), 32, 4, seed=4)
    x.whole_summary()
    x.score()
    got = x.scores.cpu().numpy().astype(np.float64)
    for i, row, pos in x.rows():
        for h in range(2):
            k = sparse._f64(sparse.cached(x.b, x.kc, i, h, pos + 1))
            q = sparse._f64(x.b.q[row, 4 * h:4 * h + 4])
            size = (np.abs(q) @ np.abs(k).T).max()
            for n in range(pos // 32 + 1):
                logits = q @ k[n * 32:(n + 1) * 32].T
                assert logits.max() <= got[row, h, n] + 2 * 256 * 2.0 ** -24 * size


@pytest.mark.parametrize("heads,c,u,block,tiles,span", LARGE_SCORES)
def test_scores_of_large_batches(torch_dev, heads, c, u, block, tiles, span):
    """Only the plan, queries, summaries and scores.  Requests share pages, and the pages in which
    no block begins hold NaN."""
    from oracle import sparse
    from paper_2606_05933_amd import ssa, workload
    torch = torch_dev
    hq, hkv, d = heads
    g, c, u = hq // hkv, np.array(c), np.array(u)
    say(f"[gpu sparse scores] {heads} c={c[:4]} u={u[:4]} block={block}")
    width, pool = int(-(-(c + u).max() // 16)), 600
    shape = ssa.make_shape(hq, hkv, d, 2 * pool, width, 0.1)
    plan, _, stride = ssa.sparse_plan(shape, c, u, block, 8)
    head, _, items = parse(plan)
    assert head["tiles"] == tiles and max(items["blk1"] - items["blk0"]) == span
    rng = np.random.default_rng(block + hq)
    table = rng.integers(pool, 2 * pool, (len(c), width))
    table[:, ::block // 16] = rng.integers(0, pool, table[:, ::block // 16].shape)
    T = int(c.sum())
    q = workload.normal_bf16((T, hq, d), 1)
    summary = np.full((2 * pool, hkv, 2, d), 0x7FC0, np.uint16)
    summary[:pool] = workload.normal_bf16((pool, hkv, 2, d), 2)
    scores = torch.full((T + 1, hkv, stride), -7.0, device="cuda")
    ssa.block_scores(shape, plan, dev(torch, plan), dev(torch, q), dev(torch, summary),
                     dev(torch, table.astype(np.int32)), scores)
    got = scores.cpu().numpy()
    assert (got[-1] == -7.0).all()
    row = 0
    for i in range(len(c)):
        rows, n = slice(row, row + c[i]), -(-(c[i] + u[i]) // block)
        seen = np.arange(n) <= (u[i] + np.arange(c[i]))[:, None] // block
        at = table[i, np.arange(n) * (block // 16)]
        for h in range(hkv):
            x = sparse._f64(q[rows, h * g:(h + 1) * g]).reshape(-1, d)
            high, low = (np.ascontiguousarray(sparse._f64(summary[at, h, j]).T) for j in range(2))
            over = lambda y: y.reshape(c[i], g, n).max(axis=1)  # noqa: E731
            up, down = np.maximum(x, 0), np.minimum(x, 0)
            ref, size = over(up @ high + down @ low), over(up @ np.abs(high) - down @ np.abs(low))
            err = np.abs(got[rows, h, :n] - ref)
            assert (err <= 2 * d * 2.0 ** -24 * size)[seen].all(), (i, h, err[seen].max())
            assert (got[rows, h, :n][~seen] == -7.0).all() and (got[rows, h, n:] == -7.0).all()
        row += c[i]


@pytest.mark.parametrize("heads", [(4, 4, 64), (4, 2, 128), (6, 2, 64), (8, 2, 64), (28, 4, 128),
                                   (16, 1, 64), (13, 1, 128)])
def test_scores_of_queries_that_are_no_numbers(torch_dev, heads):
    """A NaN counts only where all heads of a group have one, and then as the highest score."""
    from oracle import sparse
    x = Sparse(torch_dev, heads, (7, 1), (400, 900), 32, 4, seed=8)
    b, s, g = x.b, x.b.shape, x.b.shape.group
    for row in range(8):
        for h in range(s.hkv):
            if (row + h) % 3 == 2:
                b.q[row, h * g:(h + 1) * g, row] = 0x7FC0
            elif g > 1:
                b.q[row, h * g + (row + h) % g, s.d - 1] = 0xFFC0
    x.upload()
    whole = x.whole_summary()
    x.score()
    got = x.scores.cpu().numpy().astype(np.float64)
    for i, row, pos in x.rows():
        n = pos // 32 + 1
        at = b.block_table[i, np.arange(n) * 2]
        for h in range(s.hkv):
            q, hl = sparse._f64(b.q[row, h * g:(h + 1) * g]), sparse._f64(whole[at, h])
            q = q[~np.isnan(q).any(axis=1)]
            if len(q) == 0:
                assert np.isnan(got[row, h, :n]).all(), (row, h)
                continue
            ref, size = sparse.bounds(q, hl[:, 0], hl[:, 1])
            assert (np.abs(got[row, h, :n] - ref) <= 2 * s.d * 2.0 ** -24 * size).all(), (row, h)
    x.select()
    x.check_lists()


@pytest.mark.parametrize("heads,c,u,block", [
    ((8, 8, 64), (1, 1, 3), (10, 600, 900), 16),
    ((28, 4, 128), (40, 1), (3000, 7000), 16),       # up to 438 blocks: one wave
    ((4, 2, 128), (1, 2), (20000, 30000), 16),       # 1876: four waves
    ((2, 2, 64), (1, 1, 1), (90000, 500, 131071), 16),  # 8192: sixteen
    ((1, 1, 64), (1, 2), (524285, 70000), 16),       # 32768: the most
])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd", "narrow"])
@pytest.mark.parametrize("top,sink,recent", [(1, 0, 1), (5, 1, 2), (64, 3, 1), (100, 50, 50)])
def test_selection(torch_dev, heads, c, u, block, kind, top, sink, recent):
    """Only the plan and the scores: no pool is touched."""
    from oracle import sparse
    from paper_2606_05933_amd import ssa
    torch = torch_dev
    say(f"[gpu sparse select] {heads} c={c} u={u} {kind} top={top}")
    hq, hkv, d = heads
    shape = ssa.make_shape(hq, hkv, d, 1 << 20, 40000, 0.1)
    plan, _, stride = ssa.sparse_plan(shape, c, u, block, top, sink, recent)
    T = sum(c)
    rng = np.random.default_rng(top)
    size = (T, hkv, stride)
    if kind == "spread":
        s = rng.lognormal(0, 3, size) * rng.choice([-1, 1], size)
    elif kind == "ties":
        s = rng.integers(0, 3, size).astype(np.float64)
    elif kind == "odd":
        s = rng.choice([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, -1e-40, 3e38], size)
    else:
        s = 1.0 + rng.integers(0, 2000, size) * 2.0 ** -23
    s = s.astype(np.float32)
    blocks = torch.full((T + 1, hkv, top), -9, dtype=torch.int32, device="cuda")
    ssa.block_select(shape, plan, dev(torch, plan), dev(torch, s), blocks)
    got, row = blocks.cpu().numpy(), 0
    assert (got[-1] == -9).all()
    for i in range(len(c)):
        for j in range(c[i]):
            for h in range(hkv):
                ref = sparse.select(s[row, h, :(u[i] + j) // block + 1], top, sink, recent)
                assert np.array_equal(got[row, h], ref), (i, j, h)
            row += 1


def stable_select(score, top, sink, recent):
    """oracle.sparse.select of a list of more than `top` blocks, by one stable sort."""
    n = len(score)
    x = np.where(np.isnan(score), np.inf, score.astype(np.float64))[sink:n - recent]
    most = np.argsort(-x, kind="stable")[:top - sink - recent] + sink
    return np.sort(np.concatenate([np.arange(sink), most, np.arange(n - recent, n)]))


@pytest.mark.parametrize("hkv,c,most", [(8, 130, 700), (8, 130, 1024), (8, 130, 1025), (16, 67, 2048),
                                        (8, 130, 2049), (2, 3, 700)])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd", "narrow"])
@pytest.mark.parametrize("top,sink,recent", [(1, 0, 1), (64, 3, 1), (100, 50, 50), (513, 0, 2)])
def test_selection_of_many_lists(torch_dev, hkv, c, most, kind, top, sink, recent):
    """1024 lists and more, which one wave each takes up to 2048 blocks; and few of 700."""
    from oracle import sparse
    from paper_2606_05933_amd import ssa
    torch = torch_dev
    u = most * 16 - c
    say(f"[gpu sparse select] {hkv} heads, {c} rows, {most} blocks {kind} top={top}")
    shape = ssa.make_shape(hkv, hkv, 64, 1 << 20, 40000, 0.1)
    plan, _, stride = ssa.sparse_plan(shape, (c, 1), (u, 9), 16, top, sink, recent)
    rng = np.random.default_rng(top + most)
    size = (c + 1, hkv, stride)
    s = {"spread": lambda: rng.lognormal(0, 3, size) * rng.choice([-1, 1], size),
         "ties": lambda: rng.integers(0, 3, size).astype(np.float64),
         "odd": lambda: rng.choice([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, -1e-40, 3e38], size),
         "narrow": lambda: 1.0 + rng.integers(0, 2000, size) * 2.0 ** -23}[kind]().astype(np.float32)
    blocks = torch.full((c + 2, hkv, top), -9, dtype=torch.int32, device="cuda")
    ssa.block_select(shape, plan, dev(torch, plan), dev(torch, s), blocks)
    got = blocks.cpu().numpy()
    assert (got[-1] == -9).all()
    for j in range(c):
        n = (u + j) // 16 + 1
        for h in range(hkv):
            ref = stable_select(s[j, h, :n], top, sink, recent)
            assert np.array_equal(got[j, h], ref), (j, h)
    for h in range(hkv):  # the oracle's own word for some of them
        assert np.array_equal(got[h % c, h], sparse.select(s[h % c, h, :(u + h % c) // 16 + 1], top, sink,
                                                           recent))
        assert np.array_equal(got[c, h], sparse.select(s[c, h, :1], top, sink, recent))


def random_lists(rng, x):
    """Lists as ssa_block_select does not make them: unordered, named twice, out of range,
    empty ones."""
    s = x.b.shape
    lists = np.full((x.b.num_tokens, s.hkv, x.top), -1, np.int32)
    for _, row, pos in x.rows():
        n = pos // x.block + 1
        for h in range(s.hkv):
            lists[row, h] = rng.integers(0, n, x.top)
            kind = rng.integers(0, 6)
            if kind == 0:
                lists[row, h] = -1
            elif kind == 1:
                lists[row, h, rng.random(x.top) < 0.7] = -1
            elif kind == 2:
                bad = rng.random(x.top) < 0.5
                lists[row, h, bad] = rng.choice([n, n + 7, -5, 2 ** 31 - 1, -2 ** 31], int(bad.sum()))
            elif kind == 3:
                lists[row, h] = n - 1  # the partial block, over and over
            elif kind == 4:
                lists[row, h] = rng.permutation(np.resize(np.arange(n), x.top))
    x.blocks.copy_(dev(x.torch, lists))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("block,top,cu", [(16, 5, MIXED[0]), (64, 3, MIXED[3]), (32, 40, MIXED[2]),
                                          (128, 2, MIXED[4]), (16, 1, MIXED[1]), (16, 600, MIXED[0])])
def test_attention_over_any_lists(torch_dev, heads, block, top, cu):
    x = Sparse(torch_dev, heads, *cu, block, top, 0, 1, seed=7)
    random_lists(np.random.default_rng(top), x)
    x.attend()
    x.check_out()
    first = bits(x.out)
    x.attend()  # the workspace as the call left it, and the same bits
    assert np.array_equal(bits(x.out), first)


@pytest.mark.parametrize("heads,u,block,top", [((8, 2, 128), 5000, 64, 64), ((16, 1, 64), 9000, 16, 500),
                                               ((4, 4, 64), 3000, 128, 20), ((13, 1, 128), 20000, 32, 33)])
def test_cut_lists_of_few_rows(torch_dev, heads, u, block, top):
    x = Sparse(torch_dev, heads, (1,), (u,), block, top, seed=11)
    assert x.ws.numel() > 4096, "the list is not cut"
    rng = np.random.default_rng(1)
    lists = np.sort(rng.permutation(u // block + 1)[:top]).astype(np.int32)
    lists = np.pad(lists, (0, top - len(lists)), constant_values=-1)
    x.blocks.copy_(dev(torch_dev, np.tile(lists, (1, heads[1], 1))))
    x.attend()
    x.check_out()
    lists[3:] = -1  # most pieces hold nothing
    x.blocks.copy_(dev(torch_dev, np.tile(lists, (1, heads[1], 1))))
    x.attend()
    x.check_out()
    x.blocks.fill_(-1)
    x.attend()
    assert not x.out[:-1].any(), "a row without keys gives zeros"


def test_all_blocks_give_the_attention_call(torch_dev):
    """Lists of every block: ssa_mixed_attention's result, to the two calls' rounding."""
    from oracle import oracle
    x = Sparse(torch_dev, (28, 4, 128), *MIXED[0], 32, 64, seed=2)
    x.blocks.copy_(torch_dev.arange(64, dtype=torch_dev.int32, device="cuda").expand(x.blocks.shape))
    x.attend()
    x.check_out()
    ref, _ = oracle.batch_attention(x.b, x.kc, x.vc)
    got = x.out[:-1].float().cpu().numpy().astype(np.float64)
    assert np.abs(got - ref).max() <= 2e-2 and np.abs(got - ref).mean() <= 2e-3


@pytest.mark.parametrize("plan", ["device", "pinned"])
@pytest.mark.parametrize("heads,block,top,cu", [((32, 8, 128), 16, 8, ((1, 1, 20), (500, 3000, 700))),
                                                ((8, 8, 64), 64, 3, ((1, 5, 0, 1), (64, 900, 3, 1)))])
def test_the_calls_in_order(torch_dev, heads, block, top, cu, plan):
    """Summaries of the whole prompt, then of the new tokens, scores, lists, attention, on a
    stream of their own."""
    torch = torch_dev
    x = Sparse(torch, heads, *cu, block, top, 1, 2, seed=5, plan=plan)
    whole = x.whole_summary()
    made = bits(x.summary)
    b = x.b
    import dataclasses
    y = dataclasses.replace(b, q_len=np.where(b.q_len > 0, b.ctx_len, 0), ctx_len=0 * b.ctx_len)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        x.summary.fill_(1.0)
        first, _ = x.ssa.ssa_plan(x.shape, y.q_len, y.ctx_len)
        x.ssa.block_summary(x.shape, first, dev(torch, first), block, x.k, x.table, x.summary)
        x.summarise()
        x.score()
        x.select()
        x.attend()
    s.synchronize()
    got = bits(x.summary)
    for i in range(b.num_reqs):
        n = int(b.q_len[i] + b.ctx_len[i])
        if b.q_len[i]:
            at = b.block_table[i, np.arange(-(-n // block)) * block // 16]
            assert np.array_equal(got[at], made[at])
    x.check_scores(whole)
    x.check_lists()
    x.check_out()


def test_calls_on_two_streams(torch_dev):
    """Two batches at once, each with buffers of its own, give what each gives alone."""
    torch = torch_dev
    batches = [Sparse(torch, (32, 8, 128), (1, 4, 1), (5000, 300, 40), 32, 20, 1, 2, seed=30),
               Sparse(torch, (16, 2, 64), (9, 1), (3000, 9000), 16, 40, 1, 1, seed=31)]
    want = []
    for x in batches:
        x.whole_summary()
        for f in (x.summarise, x.score, x.select, x.attend):
            f()
        x.check_lists()
        x.check_out()
        want.append(bits(x.out))
    streams = [torch.cuda.Stream() for _ in batches]
    for i in range(5):
        for x in batches:
            x.out[:-1] = 7.0
            x.blocks.fill_(-9)
        torch.cuda.synchronize()
        for call in ("summarise", "score", "select", "attend"):
            for x, s in zip(batches, streams):
                getattr(x, call)(s)
        torch.cuda.synchronize()
        for x, w in zip(batches, want):
            assert np.array_equal(bits(x.out), w), i
            assert not x.ws[:4096].any()


@pytest.mark.parametrize("what", ["stale", "other", "short"])
def test_another_plan_on_the_device_writes_nothing(torch_dev, what):
    """A plan of the batch before, of other rows, or a shorter one at plan_dev."""
    torch = torch_dev
    x = Sparse(torch, (16, 2, 64), (20, 1, 1), (700, 300, 40), 32, 12, 1, 1, seed=12)
    assert x.ws.numel() > 4096
    x.whole_summary()
    before = bits(x.summary)
    plans = []
    for mine, make in ((x.plan, lambda c, u: x.ssa.sparse_plan(x.shape, c, u, 32, 12, 1, 1)[0]),
                       (x.batch_plan, lambda c, u: x.ssa.ssa_plan(x.shape, c, u)[0])):
        if what == "stale":
            other = mine.copy()
            other[8] ^= 1  # its hash
        else:
            other = make(*(((20, 1, 1), (699, 300, 40)) if what == "other" else ((1,), (3,))))
        # what lies behind a shorter one is no record
        buf = np.full(mine.nbytes, 0xFF, np.uint8)
        buf[:min(len(other), len(buf))] = other[:len(buf)]
        plans.append(dev(torch, buf))
    x.plan_dev, x.batch_dev = plans
    for f in (x.summarise, x.score, x.select, x.attend):
        f()
    torch.cuda.synchronize()
    assert np.array_equal(bits(x.summary), before)
    assert (x.scores == -7.0).all() and (x.blocks == -9).all() and (x.out == 3.0).all()
    assert not x.ws[:4096].any() and (x.ws[4096:] == 0xFF).all()


def test_replayed_graph(torch_dev):
    """All calls in one graph, replayed with eager work of the same workspace between."""
    torch = torch_dev
    x = Sparse(torch, (32, 8, 128), (1, 4, 1), (5000, 300, 40), 32, 20, 1, 2, seed=9)
    assert x.ws.numel() > 4096
    x.whole_summary()

    def run():
        x.summarise()
        x.score()
        x.select()
        x.attend()

    run()
    torch.cuda.synchronize()
    want = bits(x.out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        x.out.fill_(3.0)
        x.blocks.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(bits(x.out), want), i
        x.attend()
    x.check_lists()
    x.check_out()


@pytest.mark.parametrize("scale", [0.0, 4.0])
@pytest.mark.parametrize("heads,c,u", [((16, 2, 64), (9, 1), (200, 77)), ((8, 8, 128), (1, 33), (15, 0))])
def test_scales(torch_dev, heads, c, u, scale):
    """Scale 0: the mean of the keys' values, also where a row sees a part of a page."""
    x = Sparse(torch_dev, heads, c, u, 32, 5, seed=21, scale=scale)
    random_lists(np.random.default_rng(3), x)
    x.attend()
    x.check_out()


def test_more_pages_than_lds_holds(torch_dev):
    """Lists and unions of more than 512 pages for a workgroup, and requests of more blocks
    than a union's masks have room for."""
    rng = np.random.default_rng(8)
    # one row whose list of 32768 entries names 150 blocks here and there: 64 pieces of 4096 pages
    x = Sparse(torch_dev, (4, 2, 64), (1,), (20000,), 128, 32768, seed=22)
    lists = np.full((1, 2, 32768), -1, np.int32)
    for h in range(2):
        lists[0, h, rng.permutation(32768)[:150]] = rng.permutation(157)[:150]
    lists[0, 1, :600] = rng.permutation(np.resize(np.arange(157), 600))  # a piece of 4096 pages
    x.blocks.copy_(dev(torch_dev, lists))
    x.attend()
    x.check_out()
    # 512 workgroups of 16 rows each: nothing is cut, and a union has more than 512 blocks
    x = Sparse(torch_dev, (64, 64, 64), (128,), (9000,), 16, 100, seed=23)
    assert x.ws.numel() == 4096
    lists = np.sort(np.argsort(rng.random((128, 64, 563)), axis=2)[:, :, :100], axis=2)
    x.blocks.copy_(dev(torch_dev, lists.astype(np.int32)))
    union = len(np.unique(lists[:16, 0]))
    assert union > 512, union
    x.attend()
    x.check_out()
    # rows past 8192 blocks go by their own lists
    x = Sparse(torch_dev, (2, 1, 64), (5,), (131070,), 16, 40, seed=24)
    lists = np.stack([rng.permutation(8192)[:40] for _ in range(5)])[:, None]
    lists[2:, 0, 7] = 8192
    x.blocks.copy_(dev(torch_dev, lists.astype(np.int32)))
    x.attend()
    x.check_out()


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (16, 2, 64), (16, 2, 128), (2, 2, 64)])
def test_values_that_are_no_numbers(torch_dev, hq, hkv, d):
    """NaN and infinite keys and values of named blocks show, and nothing else does: other
    blocks, later positions, and the slots behind a request's last key."""
    torch = torch_dev
    x = Sparse(torch, (hq, hkv, d), (3, 1), (200, 70), 16, 4, seed=3)
    b, g = x.b, hq // hkv
    lists = np.full((4, 2, 4), -1, np.int32)
    lists[:, :, :2] = [1, 3]
    lists[:3, :, 2] = [[12], [12], [12]]
    x.blocks.copy_(dev(torch, lists))
    x.attend()
    plain = x.out[:-1].float().cpu().numpy().reshape(4, 2, g, d)
    # request 0: NaN in block 2 (named by no one), in position 202 (seen by row 2 alone)
    x.kc[b.block_table[0, 2], :, 3] = 0x7FC0
    x.vc[b.block_table[0, 2], :, :, 5] = 0x7F80
    x.vc[b.block_table[0, 12], 0, :, 10] = 0x7FC0
    # request 1: an infinite value of a named key
    x.vc[b.block_table[1, 1], 1, 7, 2] = 0xFF80
    x.upload()
    x.attend()
    got = x.out[:-1].float().cpu().numpy().reshape(4, 2, g, d)
    bad = np.isnan(got)
    assert bad[2, 0].all() and not bad[:2].any() and not bad[2, 1].any() and not bad[3].any()
    assert (got[3, 1, :, 7] == -np.inf).all()
    got[2, 0] = plain[2, 0]
    got[3, 1, :, 7] = plain[3, 1, :, 7]
    # what went key by key agrees with what the matrix cores gave: two roundings to bf16, and
    # sums of up to 48 terms of magnitude under 5
    assert (np.abs(got - plain) <= 2.0 ** -7 * np.abs(plain) + 1e-5).all()
    # a key seen by rows 1 and 2 alone is NaN: so are they, of that kv head
    x.kc[b.block_table[0, 12], 1, 9, 5] = 0x7FC0
    x.upload()
    x.attend()
    bad = np.isnan(x.out[:-1].float().cpu().numpy().reshape(4, 2, g, d))
    assert bad[1:3, 1].all() and bad[2, 0].all() and not bad[0].any() and not bad[1, 0].any()


def test_logits_of_minus_infinity(torch_dev):
    """Keys whose logits are all -infinity have no weights: NaN, as of a softmax over them; a
    row without a key gives zeros."""
    torch = torch_dev
    x = Sparse(torch, (4, 2, 64), (2, 1), (100, 60), 16, 3, seed=6)
    b = x.b
    b.q[:, :, 0] = 0x3F80  # 1
    for i in range(2):
        x.kc[b.block_table[i, 1], :, :, 0] = 0xFF80
    x.upload()
    lists = np.full((3, 2, 3), -1, np.int32)
    lists[:, 0, 0] = 1
    lists[0, 0, 1] = 2
    x.blocks.copy_(dev(torch, lists))
    x.attend()
    got = x.out[:-1].float().cpu().numpy().reshape(3, 2, 2, 64)
    assert np.isnan(got[1:, 0]).all() and np.isfinite(got[0, 0]).all() and (got[:, 1] == 0).all()


def test_a_long_chunk(torch_dev):
    """A chunk of more than 512 rows on a context of ten times its lists, by its own scores."""
    x = Sparse(torch_dev, (8, 2, 128), (530, 1), (7000, 300), 32, 20, 1, 2, seed=17)
    whole = x.whole_summary()
    x.score()
    x.check_scores(whole)
    x.select()
    x.check_lists()
    x.attend()
    x.check_out()


def cut_decode(torch):
    """One decode row of two kv heads, and its list of 32 blocks, cut into pieces of four."""
    x = Sparse(torch, (4, 2, 64), (1,), (4000,), 64, 32, seed=13)
    x.b.q[:, :, 0] = 0x3F80  # 1
    h = parse(x.plan)[0]
    assert (h["nsplit"], h["entries"]) == (8, 4) and x.ws.numel() > 4096
    lists = np.random.default_rng(4).permutation(62)[:32].astype(np.int32)
    x.blocks.copy_(dev(torch, np.tile(lists, (1, 2, 1))))
    return x, lists


def cut_bar(x, lists):
    """Oracle of the caches as they are over `lists` (as x's, or fewer), and its bar."""
    from oracle import sparse
    ref, mass, a = sparse.attention(x.b, x.kc, x.vc, lists, x.block)
    rel = 2.0 ** -24 * (2 * (2 * 64 * a + 8 * a + 2 * x.top * x.block / 32 + 256) + 1)
    return ref[0].reshape(2, 2, 64), (2.0 ** -8 * np.abs(ref) + rel * mass)[0].reshape(2, 2, 64)


def cut_out(x):
    x.upload()
    x.attend()
    assert not x.ws[:4096].any(), "tickets are left"
    return x.out[0].float().cpu().numpy().astype(np.float64).reshape(2, 2, 64)


def test_pieces_of_minus_infinity(torch_dev):
    """Pieces of a cut list whose keys' logits are all -infinity: they weigh nothing beside others;
    all of them together are NaN; and beside pieces without a key they are too."""
    torch = torch_dev
    for dead in (range(4), range(28, 32), range(4, 32), [*range(8), 9, 17, 30]):
        x, lists = cut_decode(torch)
        left = np.tile(np.delete(lists, list(dead)), (1, 2, 1))
        left[0, 1] = lists[:left.shape[2]]  # kv head 1 is as it was
        ref, bar = cut_bar(x, left)
        ref[1], bar[1] = (y[1] for y in cut_bar(x, np.tile(lists, (1, 2, 1))))
        for b in lists[list(dead)]:
            x.kc[x.b.block_table[0, b * 4:b * 4 + 4], 0, :, 0] = 0xFF80
        got = cut_out(x)
        assert (np.abs(got - ref) <= bar).all(), list(dead)
    x, lists = cut_decode(torch)
    ref, bar = cut_bar(x, np.tile(lists, (1, 2, 1)))
    x.kc[:, 0, :, 0] = 0xFF80
    got = cut_out(x)
    assert np.isnan(got[0]).all() and (np.abs(got - ref) <= bar)[1].all()
    # one piece of them, the others without a key; kv head 1 without any
    x.blocks.fill_(-1)
    x.blocks[0, 0, 13] = int(lists[0])
    got = cut_out(x)
    assert np.isnan(got[0]).all() and (got[1] == 0).all()


def test_pieces_of_values_that_are_no_numbers(torch_dev):
    """One piece of a cut list goes key by key, the others do not."""
    torch = torch_dev
    for at in (0, 14, 31):
        x, lists = cut_decode(torch)
        ref, bar = cut_bar(x, np.tile(lists, (1, 2, 1)))
        page = x.b.block_table[0, lists[at] * 4]
        x.vc[page, 1, 7, 3] = 0x7F80
        x.vc[page, 1, 9, 5] = 0x7FC0
        got = cut_out(x)
        assert (got[1, :, 7] == np.inf).all() and np.isnan(got[1, :, 9]).all()
        ref[1, :, [7, 9]] = got[1, :, [7, 9]] = 0
        assert (np.abs(got - ref) <= bar).all(), at
        # a key that is no number, of the other kv head
        x.kc[page, 0, 2, 11] = 0x7FC0
        got = cut_out(x)
        assert np.isnan(got[0]).all()
        got[1, :, [7, 9]] = 0
        assert (np.abs(got - ref) <= bar)[1].all(), at
    # an infinite value of a key that weighs nothing: 0 times infinity
    x, lists = cut_decode(torch)
    page = x.b.block_table[0, lists[20] * 4]
    x.kc[page, 0, 4, 0] = 0xFF80
    x.vc[page, 0, 30, 4] = 0xFF80
    got = cut_out(x)
    assert np.isnan(got[0, :, 30]).all()
    got[0, :, 30] = 0
    assert np.isfinite(got).all()


def test_an_infinite_value_behind_the_first_pass(torch_dev):
    """Workgroups of more than 512 pages: the sums of all their passes are made anew, key by key."""
    from oracle import sparse
    torch = torch_dev
    rng = np.random.default_rng(18)
    x = Sparse(torch, (64, 64, 64), (128,), (9000,), 16, 100, seed=26)
    assert x.ws.numel() == 4096, "the lists are cut"
    # even rows name block 3, of the first pass, odd ones block 560, of the second
    others = np.delete(np.arange(563), [3, 560])
    lists = others[np.argsort(rng.random((128, 64, 561)), axis=2)[:, :, :100]]
    lists[0::2, :, 40], lists[1::2, :, 40] = 3, 560
    lists = np.sort(lists, axis=2).astype(np.int32)
    for h in (5, 6):
        for at in range(0, 128, 16):
            union = np.unique(lists[at:at + 16, h])
            assert list(union).index(3) < 512 <= list(union).index(560)
    x.blocks.copy_(dev(torch, lists))
    ref, mass, a = sparse.attention(x.b, x.kc, x.vc, lists, 16)
    rel = 2.0 ** -24 * (2 * (2 * 64 * a + 8 * a + 2 * 1600 / 32 + 256) + 1)
    bar = 2.0 ** -8 * np.abs(ref) + rel * mass
    for block, slot, h, d in ((3, 1, 5, 2), (560, 9, 6, 60)):
        x.vc[x.b.block_table[0, block], h, d, slot] = 0x7F80
    x.upload()
    x.attend()
    got = x.out[:-1].float().cpu().numpy().astype(np.float64)
    for first, h, d in ((0, 5, 2), (1, 6, 60)):
        assert (got[first::2, h, d] == np.inf).all()
        got[first::2, h, d] = ref[first::2, h, d]
    assert (np.abs(got - ref) <= bar).all()
    # one row that goes by its list, in pieces of eight passes: a key of the second pass
    x = Sparse(torch, (4, 2, 64), (1,), (20000,), 128, 32768, seed=27)
    lists = np.full((1, 2, 32768), -1, np.int32)
    lists[0, :, :150] = rng.permutation(156)[:150]
    x.blocks.copy_(dev(torch, lists))
    ref, mass, a = sparse.attention(x.b, x.kc, x.vc, lists, 128)
    rel = 2.0 ** -24 * (2 * (2 * 64 * a + 8 * a + 2 * 512 * 128 / 32 + 256) + 1)
    bar = 2.0 ** -8 * np.abs(ref) + rel * mass
    x.vc[x.b.block_table[0, lists[0, 1, 100] * 8 + 5], 1, 33, 2] = 0xFF80
    x.upload()
    x.attend()
    got = x.out[:-1].float().cpu().numpy().astype(np.float64)
    assert (got[0, 2:, 33] == -np.inf).all()
    got[0, 2:, 33] = ref[0, 2:, 33]
    assert (np.abs(got - ref) <= bar).all()


def test_far_offsets(torch_dev):
    """Pages whose bytes lie past 2^32 from the pools' first one."""
    torch = torch_dev
    from paper_2606_05933_amd import ssa
    hq, hkv, d = 8, 8, 128
    pages = (1 << 32) // (hkv * 16 * d * 2) * 2 + 9  # 8 GiB a pool
    shape = ssa.make_shape(hq, hkv, d, pages, 4, 0.1)
    gen = torch.Generator(device="cuda").manual_seed(0)
    k = torch.zeros((pages, hkv, 16, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros((pages, hkv, d, 16), dtype=torch.bfloat16, device="cuda")
    summary = torch.zeros((pages, hkv, 2, d), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([pages - 1, pages // 2 + 5, pages - 3], device="cuda")
    k[at] = torch.empty((3, hkv, 16, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    v[at] = torch.empty((3, hkv, d, 16), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    q = torch.empty((1, hq, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    table = torch.tensor([[*at.tolist(), 0]], dtype=torch.int32, device="cuda")
    near = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device="cuda")
    outs = []
    for t, kk, vv, n in ((table, k, v, pages), (near, k[at].clone(), v[at].clone(), 3)):
        s = ssa.make_shape(hq, hkv, d, n, 4, 0.1)
        whole, _ = ssa.ssa_plan(s, [47], [0])
        plan, ws, stride = ssa.sparse_plan(s, [1], [46], 16, 2, 0, 1)
        sm = summary[:n]
        ssa.block_summary(s, whole, dev(torch, whole), 16, kk, t, sm)
        scores = torch.zeros((1, hkv, stride), device="cuda")
        blocks = torch.zeros((1, hkv, 2), dtype=torch.int32, device="cuda")
        out = torch.zeros((1, hq, d), dtype=torch.bfloat16, device="cuda")
        pd = dev(torch, plan)
        ssa.block_scores(s, plan, pd, q, sm, t, scores)
        ssa.block_select(s, plan, pd, scores, blocks)
        ssa.sparse_attention(s, plan, pd, q, kk, vv, t, blocks, out,
                             torch.zeros(ws, dtype=torch.uint8, device="cuda"))
        outs.append((sm[t[0, :3].long()].clone(), scores, blocks, out))
    for a, c in zip(*outs):
        assert torch.equal(a, c)
    assert outs[0][3].any()
