"""Eviction from the paged key-value cache by accumulated attention weight: the
calls whose speed is followed, with the plain form of each.

Kinds of call, each one pass through an entry point of the package:

  key_scores     a hybrid batch's attention weights, added per key and kv head
                 into the paged scores
  decode_scored  attention of one new token per request, with the same scores
  select         which keys of each request and kv head stay
  compact        the kept keys, values and scores moved to new pages
  rope_shifted   RoPE + append of requests whose cache index is no longer the
                 position

Batch lengths are fixed by the case (``len_seed``); values and page placement
come from the seed.  Head layouts and lengths are those of the package's named
workloads (8 heads of 64, 32/8, 28/4, 64/8 and 8/1 heads of 128).
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
ROPE_BASE = 500000.0
HEADS = ((8, 8, 64), (32, 8, 128), (28, 4, 128), (64, 8, 128), (8, 1, 128), (16, 1, 64))


def _case(kind, hq, hkv, d, chunks="", decodes=0, lo=0, hi=0, len_seed=0, **more):
    """chunks: "c@u,..." (c new tokens on u cached ones); decodes: how many further
    requests, their cached lengths log-uniform over [lo, hi]."""
    return {"kind": kind, "hq": hq, "hkv": hkv, "d": d, "chunks": chunks, "decodes": decodes,
            "lo": lo, "hi": hi, "len_seed": len_seed, **more}


def listed():
    """Twelve cases."""
    named = lambda name, c: dict(c, name=name)  # noqa: E731
    return [
        # the smallest iteration: a short chunk and four decodes at D = 64, launch latency
        named("scores_tiny", _case("key_scores", 8, 8, 64, "64@192", 4, 128, 512, last_rows=0,
                                   decay=1.0, old=True, q_std=1.0)),
        # an 8B model's server, one prompt chunk among 64 decodes, the scores decaying
        named("scores_mixed_8b", _case("key_scores", 32, 8, 128, "512@2048", 64, 512, 4096,
                                       last_rows=0, decay=0.98, old=True, q_std=1.0)),
        # the end of a long prompt at the 70B head shape: only the last 64 rows vote on
        # which of 33k keys stay, and there is nothing to add to
        named("scores_window_70b", _case("key_scores", 64, 8, 128, "1024@32768", 0, 0, 0,
                                         last_rows=64, decay=1.0, old=False, q_std=2.0)),
        # four prompt chunks of ragged sizes with every row voting, 7 heads a group
        named("scores_chunks_28", _case("key_scores", 28, 4, 128, "64@5000,250@3001,512@777,1024@7168",
                                        0, 0, 0, last_rows=0, decay=1.0, old=True, q_std=1.0)),
        # four short decodes: launch latency
        named("decode_small", _case("decode_scored", 8, 8, 64, "", 4, 128, 512, decay=1.0, old=True,
                                    q_std=1.0)),
        # long-context decoding at the 70B head shape: K and V stream from memory
        named("decode_70b", _case("decode_scored", 64, 8, 128, "", 32, 8192, 32768, decay=0.99,
                                  old=True, q_std=2.0)),
        # a server's requests just over their budget, each a little ragged
        named("select_server", _case("select", 32, 8, 128, "", 64, 600, 4096, budget=1000, sink=4,
                                     recent=128)),
        # one very long request alone: few lists, each long
        named("select_long", _case("select", 64, 8, 128, "0@131071", 0, 0, 0, budget=8192, sink=4,
                                   recent=1024)),
        # that server's cache cut down
        named("compact_server", _case("compact", 32, 8, 128, "", 64, 600, 4096, budget=1000, sink=4,
                                      recent=128)),
        # long contexts cut to a quarter, gigabytes to move
        named("compact_70b", _case("compact", 64, 8, 128, "", 32, 8192, 32768, budget=8192, sink=4,
                                   recent=1024)),
        # the next decode iteration after an eviction
        named("rope_decode", _case("rope_shifted", 32, 8, 128, "", 128, 64, 1000, shift=30000)),
        # a further chunk of long prompts, some of them evicted before
        named("rope_chunks", _case("rope_shifted", 64, 8, 128, "1024@8192,777@1000,2048@0", 32, 512,
                                   8192, shift=100000)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(("key_scores", "key_scores", "decode_scored", "decode_scored", "select",
                       "compact", "rope_shifted"))
    hq, hkv, d = rng.choice(HEADS)
    seed = rng.randrange(1 << 30)
    if kind == "key_scores":
        nc = rng.choice((0, 1, 1, 2, 3))
        chunks = ",".join("%d@%d" % (_log_int(rng, 2, 600), _log_int(rng, 1, 9000) - 1)
                          for _ in range(nc))
        decodes = _log_int(rng, 1, 64) if nc == 0 or rng.random() < 0.5 else 0
        lo = _log_int(rng, 1, 4096)
        return _case(kind, hq, hkv, d, chunks, decodes, lo, _log_int(rng, lo, 8192), seed,
                     last_rows=rng.choice((0, 0, 1, 16, 50, 64)), decay=rng.choice((1.0, 0.95)),
                     old=rng.random() < 0.7, q_std=rng.choice((0.5, 1.0, 2.0)))
    if kind == "decode_scored":
        lo = _log_int(rng, 1, 16384)
        return _case(kind, hq, hkv, d, "", _log_int(rng, 1, 64), lo, _log_int(rng, lo, 16384), seed,
                     decay=rng.choice((1.0, 0.95)), old=rng.random() < 0.7,
                     q_std=rng.choice((0.5, 1.0, 2.0)))
    if kind == "rope_shifted":
        chunks = ",".join("%d@%d" % (_log_int(rng, 2, 1500), _log_int(rng, 1, 9000) - 1)
                          for _ in range(rng.choice((0, 1, 2))))
        lo = _log_int(rng, 1, 4096)
        return _case(kind, hq, hkv, d, chunks, _log_int(rng, 1, 256), lo, _log_int(rng, lo, 8192),
                     seed, shift=_log_int(rng, 1, 100000))
    n = _log_int(rng, 1, 64)
    lo = _log_int(rng, 1, 16384)
    hi = _log_int(rng, lo, 100000 if n <= 4 else 16384)
    sink, recent = rng.choice((0, 1, 4, 16)), rng.choice((0, 1, 32, 100))
    budget = sink + recent + _log_int(rng, 1, max(2, hi // 2))
    return _case(kind, hq, hkv, d, "", n, lo, hi, seed, budget=budget, sink=sink, recent=recent)


def _lengths(case):
    """(c, u) of every request: new and cached tokens (select, compact: u + 1 cached)."""
    rng = np.random.default_rng(case["len_seed"])
    pairs = [tuple(int(v) for v in part.split("@")) for part in case["chunks"].split(",") if part]
    lo, hi = max(1, case["lo"]), max(1, case["hi"])
    u = np.rint(np.exp(rng.uniform(math.log(lo), math.log(hi), case["decodes"]))).astype(np.int64)
    c = np.array([p[0] for p in pairs] + [1] * case["decodes"], dtype=np.int64)
    u = np.array([p[1] for p in pairs] + u.tolist(), dtype=np.int64)
    if case["kind"] in ("select", "compact"):  # keys in the cache
        return np.zeros_like(u), u + 1
    return c, u


def _kept(case, length):
    return np.minimum(length, case["budget"])


def _rows(case, c):
    """New rows that add their weights."""
    window = case.get("last_rows", 0)
    return np.minimum(c, window) if window else c


def work(case):
    """Bytes and operations of one pass: each input and output once."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    c, u = _lengths(case)
    length = u + c
    keys, tokens = int(length.sum()), int(c.sum())
    kind = case["kind"]
    if kind == "select":
        return {"bytes": 4 * hkv * (keys + int(_kept(case, length).sum())), "flops": 0}
    if kind == "compact":
        kept = _kept(case, length)
        moved = int(kept[kept < length].sum())
        return {"bytes": hkv * moved * (2 * (4 * d + 4) + 4), "flops": 0}
    if kind == "rope_shifted":
        row = (hq + 2 * hkv) * d * 2
        return {"bytes": tokens * (2 * row + 4 * d), "flops": 3 * tokens * (hq + hkv) * d}
    r = _rows(case, c)
    # row j of c sees u + j + 1 keys; the last r rows count
    pairs = int((r * length - r * (r - 1) // 2).sum())
    old = int(u.sum()) if case["old"] else 0
    scores = 4 * hkv * (keys + old)
    q = 2 * hq * d * int(r.sum())
    if kind == "key_scores":
        return {"bytes": 2 * hkv * d * keys + scores + q, "flops": 2 * hq * d * pairs}
    return {"bytes": 4 * hkv * d * keys + scores + 2 * q, "flops": 4 * hq * d * pairs}


def _group(index, c, u, start, rows, table):
    """What the plain forms know of some of the batch's requests."""
    t = lambda a: torch.tensor(a, dtype=torch.int64, device="cuda")  # noqa: E731
    length = u + c
    req = np.repeat(np.arange(len(index)), length[index])
    first = np.concatenate([[0], np.cumsum(length[index])])[:-1]
    pos = np.arange(len(req)) - np.repeat(first, length[index])
    return {"n": len(index), "c": t(c[index]), "u": t(u[index]), "start": t(start[index]),
            "rows": t(rows[index]), "most_rows": int(rows[index].max()),
            "most_keys": int(length[index].max()), "req": t(req), "pos": t(pos),
            "table": table[t(index)]}


def prepare(case, seed):
    kind, hq, hkv, d = case["kind"], case["hq"], case["hkv"], case["d"]
    c, u = _lengths(case)
    length = u + c
    n = len(c)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)  # noqa: E731
    pages = -(-length // PAGE)
    kept = _kept(case, length) if kind in ("select", "compact") else np.zeros(n, dtype=np.int64)
    moved = (kept < length) if kind == "compact" else np.zeros(n, dtype=bool)
    new_pages = np.where(moved, -(-kept // PAGE), 0)
    num_pages = int(pages.sum() + new_pages.sum()) + 7
    width = max(1, int(pages.max()))
    order = torch.randperm(num_pages, generator=gen, device="cuda").int()

    def table(count, first):
        at = np.full((n, width), num_pages - 1, dtype=np.int64)
        for i in range(n):
            at[i, :count[i]] = first + np.arange(count[i])
            first += int(count[i])
        return order[torch.from_numpy(at).cuda()]

    state = {"case": case, "c": c, "u": u, "num_pages": num_pages, "width": width, "kept": kept,
             "block_table": table(pages, 0), "scale": float(np.float32(1 / math.sqrt(d)))}
    T = int(c.sum())
    start = np.concatenate([[0], np.cumsum(c)])[:-1]
    if kind in ("key_scores", "decode_scored"):
        state["q"] = normal(T, hq, d) * case["q_std"]
        state["k_cache"] = normal(num_pages, hkv, PAGE, d)
        if kind == "decode_scored":
            state["v_cache"] = normal(num_pages, hkv, d, PAGE)
        state["scores_in"] = None
        if case["old"]:
            state["scores_in"] = torch.empty((num_pages, hkv, PAGE), device="cuda").log_normal_(
                -1.0, 2.0, generator=gen)
        state["scores_out"] = torch.zeros((num_pages, hkv, PAGE), device="cuda")
        rows = _rows(case, c)
        # decode rows and chunk rows apart: the plain form pads each to its longest
        parts = [np.flatnonzero(c == 1), np.flatnonzero(c > 1)]
        state["groups"] = [_group(p, c, u, start, rows, state["block_table"])
                           for p in parts if len(p)]
    elif kind == "rope_shifted":
        state["qkv"] = normal(T, (hq + 2 * hkv) * d)
        state["k_cache"] = normal(num_pages, hkv, PAGE, d)
        state["v_cache"] = normal(num_pages, hkv, d, PAGE)
        rng = np.random.default_rng(case["len_seed"] + 1)
        # a third of the requests has lost nothing
        state["shift"] = np.where(rng.random(n) < 1 / 3, 0,
                                  rng.integers(0, case["shift"] + 1, n)).astype(np.int32)
        state["shift_dev"] = torch.from_numpy(state["shift"]).cuda()
        most = int((length + state["shift"]).max())
        angle = torch.arange(most, dtype=torch.float64, device="cuda")[:, None] * torch.pow(
            torch.tensor(ROPE_BASE, dtype=torch.float64, device="cuda"),
            -torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
        state["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
        state["token_req"] = torch.from_numpy(np.repeat(np.arange(n), c)).cuda()
        state["token_index"] = torch.from_numpy(
            np.arange(T) - np.repeat(start, c) + np.repeat(u, c)).cuda()
    else:
        # accumulated weights have a long tail; some keys were never looked at
        scores = torch.empty((num_pages, hkv, PAGE), device="cuda").log_normal_(-1.0, 2.0,
                                                                                 generator=gen)
        scores *= torch.rand(scores.shape, generator=gen, device="cuda") > 0.1
        state["scores"] = scores
        state["length"] = torch.from_numpy(length).cuda()
        state["kept_dev"] = torch.from_numpy(kept).cuda()
        if kind == "compact":
            state["k_cache"] = normal(num_pages, hkv, PAGE, d)
            state["v_cache"] = normal(num_pages, hkv, d, PAGE)
            state["new_table"] = table(new_pages, int(pages.sum()))
            state["moved"] = torch.from_numpy(moved).cuda()
            r = torch.rand((n, hkv, int(length.max())), generator=gen, device="cuda")
            state["keep"] = _lists(r, state["length"], state["kept_dev"], case)
    return state


def _lists(score, length, kept, case):
    """The kept keys of [n, hkv, L] scores, flat by request, head and index: the first
    `sink`, the last `recent` and the highest others, the lowest index of equals first."""
    pos = torch.arange(score.shape[2], device="cuda")
    here = pos < length[:, None, None]
    always = here & ((pos < case["sink"]) | (pos >= length[:, None, None] - case["recent"]))
    score = torch.where(score.isnan(), -math.inf, score)
    # by score, then what has to stay before the others and what is not there last
    by = torch.sort(score, dim=2, descending=True, stable=True).indices
    level = torch.where(always, 2, here.int()).expand(score.shape).gather(2, by)
    by = by.gather(2, torch.sort(level, dim=2, descending=True, stable=True).indices)
    rank = torch.empty_like(by).scatter_(2, by, pos.expand(by.shape).contiguous())
    return (rank < kept[:, None, None]).nonzero()[:, 2].int()


def _cached(pool, group, slot_last):
    """[n, hkv, L, D] in 32 bits: the cached rows of a group's requests, zero past the end."""
    pos = torch.arange(group["most_keys"], device="cuda")
    page, slot = group["table"][:, pos // PAGE].long(), (pos % PAGE).expand(group["n"], -1)
    rows = pool[page, :, :, slot] if slot_last else pool[page, :, slot]
    here = pos < (group["u"] + group["c"])[:, None]
    return torch.where(here[:, :, None, None], rows.float(), 0.0).permute(0, 2, 1, 3)


def _weights(state, group):
    """[n, hkv, rows * G, L] attention weights of the counted rows in 32 bits, zero for the
    rows that pad shorter requests."""
    case = state["case"]
    hkv, g, d = case["hkv"], case["hq"] // case["hkv"], case["d"]
    n, most, keys = group["n"], group["most_rows"], group["most_keys"]
    back = torch.arange(most, device="cuda")
    row = group["c"][:, None] - 1 - back  # from the last one
    q = state["q"][(group["start"][:, None] + row).clamp(min=0)].float()
    q = q.view(n, most, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n * hkv, most * g, d)
    k = _cached(state["k_cache"], group, False).transpose(2, 3).reshape(n * hkv, d, keys)
    s = torch.bmm(q, k.contiguous()).mul_(state["scale"]).view(n, hkv, most, g, keys)
    seen = torch.arange(keys, device="cuda") <= (group["u"][:, None] + row)[:, :, None]
    s.masked_fill_(~seen[:, None, :, None], -math.inf)
    s.sub_(s.amax(dim=4, keepdim=True)).exp_()
    s.div_(s.sum(dim=4, keepdim=True))
    counted = (back < group["rows"][:, None])[:, None, :, None, None]
    return torch.where(counted, s, 0.0).view(n, hkv, most * g, keys)


def _add_scores(state, group, w):
    req, pos = group["req"], group["pos"]
    page, slot = group["table"][req, pos // PAGE].long(), pos % PAGE
    new = w.sum(dim=2)[req, :, pos]
    if state["scores_in"] is not None:
        old = state["scores_in"][page, :, slot] * state["case"]["decay"]
        new = new + torch.where((pos < group["u"][req])[:, None], old, 0.0)
    state["scores_out"][page, :, slot] = new


def _scored_group(state, group):
    """Scores of one group, and its rows' attention where the values are there."""
    w = _weights(state, group)
    _add_scores(state, group, w)
    if "v_cache" not in state:
        return None
    case, n = state["case"], group["n"]
    v = _cached(state["v_cache"], group, True).reshape(n * case["hkv"], -1, case["d"])
    out = torch.bmm(w.view(n * case["hkv"], -1, group["most_keys"]), v.contiguous())
    return out.view(n, case["hq"], case["d"]).to(torch.bfloat16)


def _scored(state):
    got = [_scored_group(state, g) for g in state["groups"]]
    return {"scores": state["scores_out"]} if got[0] is None else {"scores": state["scores_out"],
                                                                   "out": got[0]}


def _select(state):
    case, table = state["case"], state["block_table"]
    pos = torch.arange(int((state["u"] + state["c"]).max()), device="cuda")
    page, slot = table[:, pos // PAGE].long(), (pos % PAGE).expand(table.shape[0], -1)
    score = state["scores"][page, :, slot].permute(0, 2, 1)
    return _lists(score, state["length"], state["kept_dev"], case)


def _compact(state):
    n, hkv = len(state["kept"]), state["case"]["hkv"]
    # (request, head, rank) of each entry of the flat lists
    total = int(state["kept"].sum()) * hkv
    lists = state["kept_dev"].repeat_interleave(hkv)
    which = torch.arange(n * hkv, device="cuda").repeat_interleave(lists, output_size=total)
    rank = torch.arange(total, device="cuda") - (lists.cumsum(0) - lists)[which]
    req, head, key = which // hkv, which % hkv, state["keep"].long()
    src = state["block_table"][req, key // PAGE].long()
    dst = state["new_table"][req, rank // PAGE].long()
    # a request that keeps everything stays where it is
    dst = torch.where(state["moved"][req], dst, src)
    a, b = key % PAGE, torch.where(state["moved"][req], rank % PAGE, key % PAGE)
    k, v, s = state["k_cache"], state["v_cache"], state["scores"]
    k[dst, head, b] = k[src, head, a]
    v[dst, head, :, b] = v[src, head, :, a]
    s[dst, head, b] = s[src, head, a]
    return {"k": k, "v": v, "scores": s}


def _rope(state):
    case = state["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    x = state["qkv"].float().view(-1, hq + 2 * hkv, d)
    req, index = state["token_req"], state["token_index"]
    cs = state["cos_sin"][index + state["shift_dev"][req]][:, None]
    cos, sin = cs[..., :d // 2], cs[..., d // 2:]
    a, b = x[:, :hq + hkv, :d // 2], x[:, :hq + hkv, d // 2:]
    turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2).to(torch.bfloat16)
    page, slot = state["block_table"][req, index // PAGE].long(), index % PAGE
    state["k_cache"][page, :, slot] = turned[:, hq:]
    state["v_cache"][page, :, :, slot] = x[:, hq + hkv:].to(torch.bfloat16)
    return {"q": turned[:, :hq], "k": state["k_cache"], "v": state["v_cache"]}


def _handle(state):
    """The shape, the plan and the buffers that a serving program keeps for a batch, made on
    the first pass over it."""
    if "handle" in state:
        return state["handle"]
    from paper_2606_05933_amd import ssa
    case = state["case"]
    kind, hq, hkv, d = case["kind"], case["hq"], case["hkv"], case["d"]
    shape = ssa.make_shape(hq, hkv, d, state["num_pages"], state["width"], state["scale"])
    c, u = state["c"], state["u"]
    ws_bytes = 0
    h = {"shape": shape}
    if kind in ("key_scores", "decode_scored"):
        plan, ws_bytes = ssa.score_plan(shape, c, u, case.get("last_rows", 0))
    elif kind == "rope_shifted":
        plan, _ = ssa.ssa_plan(shape, c, u)
    else:
        plan, ws_bytes = ssa.evict_plan(shape, u, np.full(len(u), case["budget"]), case["sink"],
                                        case["recent"])
    h["plan"], h["plan_dev"] = plan, torch.from_numpy(plan).cuda()
    h["workspace"] = torch.zeros(max(ws_bytes, 256), dtype=torch.uint8, device="cuda")
    if kind == "decode_scored":
        h["out"] = torch.empty((len(c), hq, d), dtype=torch.bfloat16, device="cuda")
    if kind == "rope_shifted":
        h["q"] = torch.empty((int(c.sum()), hq, d), dtype=torch.bfloat16, device="cuda")
    if kind == "select":
        h["keep"] = torch.empty(int(state["kept"].sum()) * hkv, dtype=torch.int32, device="cuda")
    state["handle"] = h
    return h


def _own(state):
    from paper_2606_05933_amd import ssa
    h, case, kind = _handle(state), state["case"], state["case"]["kind"]
    plan = (h["shape"], h["plan"], h["plan_dev"])
    if kind == "key_scores":
        ssa.key_scores(*plan, state["q"], state["k_cache"], state["block_table"],
                       state["scores_in"], case["decay"], state["scores_out"], h["workspace"])
        return {"scores": state["scores_out"]}
    if kind == "decode_scored":
        ssa.decode_scored(*plan, state["q"], state["k_cache"], state["v_cache"],
                          state["block_table"], state["scores_in"], case["decay"],
                          state["scores_out"], h["out"], h["workspace"])
        return {"scores": state["scores_out"], "out": h["out"]}
    if kind == "select":
        ssa.evict_select(*plan, state["scores"], state["block_table"], h["keep"], h["workspace"])
        return h["keep"]
    if kind == "compact":
        ssa.evict_compact(*plan, state["keep"], state["block_table"], state["new_table"],
                          state["k_cache"], state["v_cache"], state["scores"])
        return {"k": state["k_cache"], "v": state["v_cache"], "scores": state["scores"]}
    ssa.rope_append_shifted(*plan, state["qkv"], state["cos_sin"], state["shift"],
                            state["shift_dev"], h["q"], state["k_cache"], state["v_cache"],
                            state["block_table"])
    return {"q": h["q"], "k": state["k_cache"], "v": state["v_cache"]}


def run(state):
    """One pass through the operator."""
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "select":
        return _select(state)
    if kind == "compact":
        return _compact(state)
    if kind == "rope_shifted":
        return _rope(state)
    return _scored(state)


def exact(case, seed):
    """What ``run`` returns, request by request and in 64 bits."""
    if case["kind"] == "select":
        return None  # whole numbers
    state = prepare(case, seed)
    if case["kind"] == "compact":
        first = 0
        for i, (n, kept) in enumerate(zip(state["u"].tolist(), state["kept"].tolist())):
            lists = state["keep"][first:first + case["hkv"] * kept].view(case["hkv"], kept).long()
            first += case["hkv"] * kept
            pages, to = state["block_table"][i].long(), state["new_table"][i].long()
            for h in range(case["hkv"] if kept < n else 0):
                for pool, slots_last in (("k_cache", False), ("v_cache", True), ("scores", False)):
                    x = state[pool][:, h].transpose(1, 2) if slots_last else state[pool][:, h]
                    old = x[pages[:-(-n // PAGE)]].flatten(0, 1)[lists[h]]
                    new = x[to[:-(-kept // PAGE)]].flatten(0, 1)
                    new[:kept] = old
                    x[to[:-(-kept // PAGE)]] = new.unflatten(0, (-1, PAGE))
        return {"k": state["k_cache"], "v": state["v_cache"], "scores": state["scores"]}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g = hq // hkv
    rows = _rows(case, state["c"])
    scores = state["scores_out"].double() if "scores_out" in state else None
    if case["kind"] == "rope_shifted":
        keys, values = state["k_cache"].double(), state["v_cache"].double()
    outs, at = [], 0
    for i, (c, u) in enumerate(zip(state["c"].tolist(), state["u"].tolist())):
        pages = state["block_table"][i, :-(-(u + c) // PAGE)].long()
        if case["kind"] == "rope_shifted":
            x = state["qkv"][at:at + c].double().view(c, hq + 2 * hkv, d)
            p = torch.arange(c, dtype=torch.float64, device="cuda") + (u + int(state["shift"][i]))
            turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), p[:, None] *
                               ROPE_BASE ** (-2 * torch.arange(d // 2, dtype=torch.float64,
                                                               device="cuda") / d))
            z = torch.complex(x[:, :hq + hkv, :d // 2], x[:, :hq + hkv, d // 2:]) * turn[:, None]
            z = torch.cat([z.real, z.imag], dim=2)
            outs.append(z[:, :hq])
            flat = keys[pages].transpose(1, 2).reshape(-1, hkv, d)
            flat[u:u + c] = z[:, hq:]
            keys[pages] = flat.view(-1, PAGE, hkv, d).transpose(1, 2)
            flat = values[pages].permute(0, 3, 1, 2).reshape(-1, hkv, d)
            flat[u:u + c] = x[:, hq + hkv:]
            values[pages] = flat.view(-1, PAGE, hkv, d).permute(0, 2, 3, 1)
            at += c
            continue
        k = state["k_cache"][pages].transpose(1, 2).reshape(-1, hkv, d)[:u + c].double()
        w_sum = torch.zeros((hkv, u + c), dtype=torch.float64, device="cuda")
        out = torch.zeros((hq, d), dtype=torch.float64, device="cuda")
        for h in range(hkv):
            for j0 in range(c - int(rows[i]), c, 256):
                j = torch.arange(j0, min(j0 + 256, c), device="cuda")
                q = state["q"][at + j, h * g:(h + 1) * g].double().reshape(-1, d)
                s = (q @ k[:, h].T.contiguous()).view(len(j), g, u + c) * state["scale"]
                s[(torch.arange(u + c, device="cuda") > u + j[:, None])[:, None].expand(s.shape)] = -math.inf
                w = torch.softmax(s, dim=2)
                w_sum[h] += w.sum(dim=(0, 1))
                if "v_cache" in state:
                    v = state["v_cache"][pages, h].transpose(1, 2).reshape(-1, d)[:u + c].double()
                    out[h * g:(h + 1) * g] = w[0] @ v
        if case["old"]:
            old = state["scores_in"][pages].transpose(1, 2).reshape(-1, hkv)[:u].double()
            w_sum[:, :u] += case["decay"] * old.T
        flat = scores[pages].transpose(1, 2).reshape(-1, hkv)
        flat[:u + c] = w_sum.T
        scores[pages] = flat.view(-1, PAGE, hkv).transpose(1, 2)
        outs.append(out)
        at += c
    if case["kind"] == "rope_shifted":
        return {"q": torch.cat(outs), "k": keys, "v": values}
    return {"scores": scores, "out": torch.stack(outs)} if "v_cache" in state else {"scores": scores}
