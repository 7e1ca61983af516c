"""GPU tests of the eviction calls at the edges of their arithmetic and their masks.

The bar of each test is derived beside it from the roundings of its own inputs
(half a step: fp32 2^-24, bf16 2^-8 of the value).
"""
import numpy as np
import pytest

from test_gpu_evict import Scored, batch, dev, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    return torch


def bf16(x):
    """float64 of the bf16 values nearest to x."""
    from paper_2606_05933_amd import workload
    x = np.asarray(x, np.float32)
    return workload.bf16_bits_to_f32(workload.f32_to_bf16_bits(x)).astype(np.float64).reshape(x.shape)


def put_keys(b, cache, i, head, at, rows, values=False):
    """rows [n, D] (bf16 values) into the slots `at` of request i's pages."""
    from paper_2606_05933_amd import workload
    at = np.asarray(at)
    bits = workload.f32_to_bf16_bits(np.asarray(rows, np.float32))
    if values:
        cache[b.block_table[i, at // 16], head, :, at % 16] = bits
    else:
        cache[b.block_table[i, at // 16], head, at % 16] = bits


@pytest.mark.parametrize("heads", [(8, 8, 64), (4, 1, 128)])
@pytest.mark.parametrize("u", [2, 40, 4500])
def test_scored_decode_weighs_values_in_full(torch_dev, heads, u):
    """Two keys of weight 1 hold the first two bf16 parts of a third key's weight p, and
    that one the value -1: what is left of the output is p's bits past the 16th.

    Logits are single products (exact).  p = 2^(x c) is off by the rounding of c and of
    x c (2^-24 |x c| ln 2 each, |x c| < 1) and the exponential's (one step, 2^-23): under
    4 2^-24 p.  Three terms add with at most three roundings of sums under 2, and 1 / l
    and its product take 2^-23 of a value under 2^-8.  So, mass being sum |w v| l < 3:
    |err| <= 2^-8 |ref| + (4 + 3 * 2 + 1) 2^-24 mass / l."""
    from paper_2606_05933_amd import workload
    hq, hkv, d = heads
    g = hq // hkv
    n = 6
    b = batch(hq, hkv, d, [1] * n, [u] * n, seed=40, scale=0.125)
    x = Scored(torch_dev, b, old=False)
    scale = float(np.float32(0.125))
    rng = np.random.default_rng(41)
    q = np.zeros((n, hq, d), np.float32)
    q[:, :, 0] = 1
    want = np.zeros((n, hq, d))
    bar = np.zeros_like(want)
    for i in range(n):
        for h in range(hkv):
            keys = np.zeros((u + 1, d))
            keys[:, 0] = -1e6  # weight 0
            values = bf16(rng.standard_normal((u + 1, d)))
            one, two, third = rng.choice(u + 1, 3, replace=False)
            logit = bf16(-rng.uniform(0.5, 5.0, 100))
            p = np.exp(scale * logit)
            hi = bf16(p)
            mid = bf16(p - hi)
            best = np.argmax(np.abs(hi + mid - p))  # much to miss
            p, hi, mid = p[best], hi[best], mid[best]
            keys[[one, two], 0], keys[third, 0] = 0, logit[best]
            values[one], values[two], values[third] = hi, mid, -1
            put_keys(b, x.kc, i, h, np.arange(u + 1), keys)
            put_keys(b, x.vc, i, h, np.arange(u + 1), values, values=True)
            want[i, h * g:(h + 1) * g] = (hi + mid - p) / (2 + p)
            bar[i, h * g:(h + 1) * g] = 11 * 2.0 ** -24 * (hi + abs(mid) + p) / (2 + p)
    b.q = workload.f32_to_bf16_bits(q)
    x.q, x.k, x.v = dev(torch_dev, b.q), dev(torch_dev, x.kc), dev(torch_dev, x.vc)
    x.decode()
    torch_dev.cuda.synchronize()
    got = x.out.float().cpu().numpy().astype(np.float64)
    err = np.abs(got - want)
    assert (np.abs(want) > 2 * bar).all(), "the inputs do not show the last bits"
    assert (err <= 2.0 ** -8 * np.abs(want) + bar).all(), float((err / bar).max())


@pytest.mark.parametrize("heads", [(8, 8, 64), (28, 4, 128)])
@pytest.mark.parametrize("u", [3, 700, 5000])
def test_infinite_values_of_seen_keys_stay_infinite(torch_dev, heads, u):
    """Weights are far from underflow (logits within 20 of each other): a dim with an
    infinite value is infinite, with both signs NaN, and the others are as they were, bit
    for bit."""
    hq, hkv, d = heads
    b = batch(*heads, [1] * 3, [u, u // 2, u], seed=43)
    x = Scored(torch_dev, b, old=False)
    x.decode()
    torch_dev.cuda.synchronize()
    plain = x.out.clone()
    rng = np.random.default_rng(44)
    kind = np.zeros((3, hkv, d), int)  # 0: finite, 1: +inf, 2: -inf, 3: both
    for i in range(3):
        n = int(b.ctx_len[i]) + 1
        for h in range(hkv):
            dims = rng.choice(d, 9, replace=False)
            for dim, what in zip(dims, [1, 1, 1, 2, 2, 2, 3, 3, 3]):
                kind[i, h, dim] = what
                at = rng.choice(n, 2, replace=False)
                for t, bits in zip(at, {1: (0x7F80,), 2: (0xFF80,), 3: (0x7F80, 0xFF80)}[what]):
                    x.vc[b.block_table[i, t // 16], h, dim, t % 16] = bits
    x.v = dev(torch_dev, x.vc)
    x.out.zero_()
    x.decode()
    torch_dev.cuda.synchronize()
    x.check_scores()
    got = x.out.float().cpu().numpy()
    kind = np.repeat(kind, hq // hkv, axis=1)
    assert (got[kind == 1] == np.inf).all() and (got[kind == 2] == -np.inf).all()
    assert np.isnan(got[kind == 3]).all()
    same = kind == 0
    assert np.array_equal(got[same], plain.float().cpu().numpy()[same])


@pytest.mark.parametrize("heads", [(8, 8, 64), (8, 4, 128)])
@pytest.mark.parametrize("c,u", [([2, 2, 3], [500, 40, 300]), ([2], [9000])])
@pytest.mark.parametrize("q_scale", [1, 16, 256])
def test_weights_of_chunk_rows_add_up_to_one(torch_dev, heads, c, u, q_scale):
    """A kv head's new scores of a request add up to its c G rows, however far from zero
    the logits are: both passes form the same logits (the same products in the same
    order), so a weight is 2^r / l with the r of l's own terms, r within 40 of zero
    where it counts.  Per weight, in either pass: r's rounding 2^-24 64 ln 2, the
    exponential one step; 1 / l and its product one and a half, sums over a tile's
    rows under 8 additions; in l additions along at most (u + c) / 32 + 40 terms."""
    b = batch(*heads, c, u, seed=45)
    x = Scored(torch_dev, b, old=False, q_scale=q_scale)
    x.scores()
    torch_dev.cuda.synchronize()
    got = x.out_scores.cpu().numpy().astype(np.float64)
    worst = 0.0
    for i in range(b.num_reqs):
        n = int(b.q_len[i] + b.ctx_len[i])
        t = np.arange(n)
        sums = got[b.block_table[i, t // 16], :, t % 16].sum(axis=0)
        rows = int(b.q_len[i]) * b.shape.group
        bar = 2.0 ** -24 * (2 * 64 * np.log(2) + 2 * 2 + 3 + 8 + n / 32 + 40)
        off = np.abs(sums / rows - 1)
        worst = max(worst, float(off.max() / bar))
    say(f"    of the bar: {worst:.3f}")
    assert worst <= 1


@pytest.mark.parametrize("heads", [(8, 8, 64), (4, 4, 128), (28, 4, 128)])
@pytest.mark.parametrize("row", [0, 5, -1])
@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_rows_that_are_not_finite_reach_only_the_keys_they_see(torch_dev, heads, row, value):
    """One row of each chunk is not finite: the keys that it sees score NaN, later ones
    what the other rows give them, also where padded columns stand beside."""
    from oracle import evict
    from paper_2606_05933_amd import workload
    c, u = [20, 33, 7, 300], [0, 50, 700, 9]
    b = batch(*heads, c, u, seed=46)
    x = Scored(torch_dev, b, old=False)
    _, size = evict.key_scores(b, x.kc)
    start = np.cumsum(c) - c
    bits = workload.f32_to_bf16_bits(np.asarray([value], np.float32)).ravel()[0]
    for i in range(len(c)):
        b.q[start[i] + row % c[i], :, 3] = bits
    x.q = dev(torch_dev, b.q)
    x.scores()
    torch_dev.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        ref, _ = evict.key_scores(b, x.kc)
    got = x.out_scores.cpu().numpy().astype(np.float64)
    for i in range(len(c)):
        t = np.arange(c[i] + u[i])
        at = b.block_table[i, t // 16], slice(None), t % 16
        seen = t <= u[i] + row % c[i]
        assert np.isnan(ref[at][seen]).all() and np.isfinite(ref[at][~seen]).all()
        assert np.isnan(got[at][seen]).all()
        err, tol = np.abs(got[at] - ref[at])[~seen], (x.rel(size)[at] * ref[at])[~seen]
        assert (err <= tol).all(), (i, int(np.isnan(err).sum()), err.size)


def test_an_evicting_layer_refuses_half_given_parts(torch_dev):
    """Shifts of which only one copy is given, and buffers of the scores without their
    plan: nothing is written to the caches."""
    torch = torch_dev
    from paper_2606_05933_amd import ssa, workload
    hq, hkv, d, hidden, inter = 8, 2, 64, 256, 128
    b = batch(hq, hkv, d, [2, 1], [30, 5], seed=47)
    shape = ssa.make_shape(hq, hkv, d, b.num_pages, b.max_pages_per_req, d ** -0.5)
    w = ssa.LayerWeights(workload.layer_weights(1, hidden, inter, hq, hkv, d), hq, hkv, d, 2048)
    x = dev(torch, workload.normal_bf16((3, hidden), 5))
    plan, _ = ssa.ssa_plan(shape, b.q_len, b.ctx_len)
    k, v = dev(torch, b.k_cache), dev(torch, b.v_cache)
    before = k.clone(), v.clone()
    ws = torch.zeros(ssa.layer_workspace_size(shape, plan, w), dtype=torch.uint8, device="cuda")
    scores = torch.zeros((b.num_pages, hkv, 16), device="cuda")
    shift = np.array([7, 9], np.int32)

    def call(**parts):
        ssa.layer_forward_evicting(shape, plan, dev(torch, plan), w, x, torch.empty_like(x), k, v,
                                   dev(torch, b.block_table), ws, **parts)

    for parts in (dict(shift_dev=dev(torch, shift)), dict(shift_host=shift)):
        with pytest.raises(ssa.SsaError) as e:
            call(**parts)
        assert e.value.code == ssa.SSA_ERR_NULL
    for name in ("scores_in", "scores_out", "score_workspace", "score_plan_dev"):
        with pytest.raises(ValueError):
            call(**{name: scores})
    torch.cuda.synchronize()
    assert torch.equal(k.view(torch.int16), before[0].view(torch.int16))
    assert torch.equal(v.view(torch.int16), before[1].view(torch.int16))


@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 2, 128)])
@pytest.mark.parametrize("c", [1, 20])
@pytest.mark.parametrize("gain", [30, 3000])
def test_far_logits_give_their_weight_to_the_keys_that_have_it(torch_dev, heads, c, gain):
    """Logits up to 1e4 and more, nearly all weight on one key a row: every key's score
    by the oracle's.  A logit and the sum's logarithm are each off by D 2^-24 A, so a
    weight by a factor of at most exp(rel) (rel: the bar of the other tests); weights
    under 2^-126 may be zero."""
    from oracle import evict
    from paper_2606_05933_amd import workload
    b = batch(*heads, [c, c], [300, 3000], seed=48)
    b.q = workload.f32_to_bf16_bits(workload.bf16_bits_to_f32(b.q) * np.float32(gain))
    x = Scored(torch_dev, b, old=False)
    ref, size = evict.key_scores(b, x.kc)
    bar = np.expm1(x.rel(size)) * ref + c * b.shape.group * 2.0 ** -126
    known = ~np.isnan(ref)
    if gain == 30:  # the bar tells a row's keys from one another
        assert np.nanmax(x.rel(size)) < 0.01 and np.nanmax(ref) > 100 * np.nanmedian(ref)

    def check():
        torch_dev.cuda.synchronize()
        got = x.out_scores.cpu().numpy().astype(np.float64)
        err = np.abs(got - ref)
        assert (err <= bar)[known].all(), float(np.nanmax((err / bar)[known]))

    x.scores()
    check()
    if c == 1:
        x.out_scores.fill_(-7.0)
        x.decode()
        check()
        x.check_out()


@pytest.mark.parametrize("cu,shift", [([(20, 30), (1, 100), (1, 5), (37, 0)], [400, 77, 0, 0]),
                                      ([(1, 90), (1, 700), (1, 3)], [30, 900, 0])])
def test_an_evicting_layer_matches_the_oracle(torch_dev, cu, shift):
    """The whole shifted layer, its output included, and its scores, eagerly and replayed
    from a graph.  Between x and out lie seven bf16 tensors, each at most a step apart
    from the oracle's: the bar of the plain layer's test."""
    torch = torch_dev
    from oracle import evict, layer as olay
    from paper_2606_05933_amd import ssa, workload
    from paper_2606_05933_amd.device import bits_of
    hidden, inter, hq, hkv, d = 256, 256, 4, 2, 64
    c, u = [p[0] for p in cu], [p[1] for p in cu]
    wts = workload.layer_weights(49, hidden, inter, hq, hkv, d)
    b = batch(hq, hkv, d, c, u, seed=49)
    T = b.num_tokens
    shift = np.asarray(shift, np.int32)
    shape = ssa.make_shape(hq, hkv, d, b.num_pages, b.max_pages_per_req, d ** -0.5)
    w = ssa.LayerWeights(wts, hq, hkv, d, max_position=2048)
    plan, _ = ssa.ssa_plan(shape, c, u)
    sp, sws = ssa.score_plan(shape, c, u)
    x = workload.normal_bf16((T, hidden), 50)
    xd, k, v = dev(torch, x), dev(torch, b.k_cache), dev(torch, b.v_cache)
    out = torch.zeros((T, hidden), dtype=torch.bfloat16, device="cuda")
    scores = torch.full((b.num_pages, hkv, 16), -7.0, device="cuda")
    ws = torch.zeros(ssa.layer_workspace_size(shape, plan, w), dtype=torch.uint8, device="cuda")
    score_ws = torch.full((sws,), 0xFF, dtype=torch.uint8, device="cuda")
    held = [dev(torch, a) for a in (plan, b.block_table, sp, shift)]

    def layer():
        ssa.layer_forward_evicting(shape, plan, held[0], w, xd, out, k, v, held[1], ws, sp, held[2],
                                   None, 1.0, scores, score_ws, shift, held[3])

    layer()
    torch.cuda.synchronize()
    ref, kc_ref, vc_ref = olay.decoder_layer(x, wts, hq, hkv, d, b.q_len, b.ctx_len, b.block_table,
                                             b.k_cache, b.v_cache, eps=1e-5, shift=shift)
    got = out.float().cpu().numpy().astype(np.float64)
    err = np.abs(got - ref)
    say(f"    out: max_abs={err.max():.3e} mean_abs={err.mean():.3e}")
    assert np.isfinite(got).all()
    assert (err <= 2.0 ** -5 * (np.abs(ref) + 1.0)).all() and err.mean() <= 3e-3
    plain, _, _ = olay.decoder_layer(x, wts, hq, hkv, d, b.q_len, b.ctx_len, b.block_table, b.k_cache,
                                     b.v_cache, eps=1e-5)
    assert np.abs(plain - ref).mean() > 4 * err.mean(), "the shift does not show"
    # each row's weights add up to 1 over the keys that it sees
    sc = scores.cpu().numpy().astype(np.float64)
    for i in range(len(c)):
        t = np.arange(c[i] + u[i])
        sums = sc[b.block_table[i, t // 16], :, t % 16].sum(axis=0)
        assert np.allclose(sums, c[i] * hq // hkv, rtol=1e-5)
    want = [t.clone() for t in (out, k, v, scores)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        layer()  # warm the stream before capture
        with torch.cuda.graph(graph, stream=side):
            layer()
    for r in range(4):
        k.copy_(dev(torch, b.k_cache))
        v.copy_(dev(torch, b.v_cache))
        out.zero_()
        scores.fill_(-7.0)
        score_ws.fill_(0xA5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, e in zip((out, k, v, scores), want):
            a, e = (t.view(torch.int16) if t.dtype == torch.bfloat16 else t for t in (a, e))
            assert torch.equal(a, e), r
