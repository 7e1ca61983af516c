"""Serving long contexts from the paged key-value cache: the calls whose speed is followed,
with the plain form of each.

Kinds of call, each one pass through an entry point of the package:

  pages      block tables, the ring of free pages, row starts and slot maps after requests
             have grown, shrunk or ended, from their lengths on the device
  rope       RoPE + append with interleaved or half pairs, of part of the head
  summary    per block of cached keys, kv head and dim the highest and the lowest value
  scores     per new row, kv head and block an upper bound of the block's logits
  select     the blocks that each row and kv head looks at
  attention  attention over those blocks

Batch lengths are fixed by the case (``len_seed``); values and page placement come from the
seed.  Head layouts and lengths are those of the package's named workloads (8 heads of 64,
32/8, 28/4, 64/8 and 8/1 heads of 128).
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
ROPE_BASE = 500000.0
HEADS = ((8, 8, 64), (32, 8, 128), (28, 4, 128), (64, 8, 128), (8, 1, 128), (16, 1, 64))
INTERLEAVED, HALF = "interleaved", "half"


def _case(kind, hq, hkv, d, chunks="", decodes=0, lo=0, hi=0, len_seed=0, **more):
    """chunks: "c@u,..." (c new tokens on u cached ones); decodes: how many further
    requests of one new token, their cached lengths log-uniform over [lo, hi]."""
    return {"kind": kind, "hq": hq, "hkv": hkv, "d": d, "chunks": chunks, "decodes": decodes,
            "lo": lo, "hi": hi, "len_seed": len_seed, **more}


def _blocks(block, top, sink=1, recent=2):
    return {"block": block, "top": top, "sink": sink, "recent": recent}


def listed():
    """Twelve cases."""
    named = lambda name, c: dict(c, name=name)  # noqa: E731
    return [
        # a decode iteration of a server: every request grows by a token, a few take a page
        named("pages_decode", _case("pages", 32, 8, 128, "", 64, 512, 4096, ended=0)),
        # long prompts come in while some long requests end
        named("pages_prompts", _case("pages", 32, 8, 128, "32768@0,16384@0,8192@4096,1000@77", 500,
                                     64, 16384, ended=40)),
        # a decode iteration of a model that turns half of each head, in neighbouring pairs
        named("rope_decode", _case("rope", 32, 8, 128, "", 128, 64, 8192, layout=INTERLEAVED,
                                   rotary=64, factor=1.0)),
        # a further chunk of long prompts beyond the trained length, three quarters of the
        # head turned at stretched positions
        named("rope_chunks", _case("rope", 64, 8, 128, "1024@80000,777@1000,2048@0", 32, 512, 8192,
                                   layout=HALF, rotary=96, factor=8.0)),
        # the blocks that a decode iteration's new keys go to
        named("summary_decode", _case("summary", 32, 8, 128, "", 64, 512, 16384, block=64)),
        # a long prompt read in one piece beside a ragged chunk
        named("summary_prompt", _case("summary", 64, 8, 128, "32768@0,1000@4001", 0, block=64)),
        # long-context decoding at the 70B head shape
        named("scores_decode", _case("scores", 64, 8, 128, "", 32, 8192, 32768,
                                     **_blocks(64, 64))),
        # a prompt chunk on a long context beside decodes
        named("scores_chunk", _case("scores", 32, 8, 128, "512@32768", 16, 4096, 16384,
                                    **_blocks(32, 64))),
        # the choice of such a decode iteration
        named("select_decode", _case("select", 64, 8, 128, "", 32, 8192, 32768,
                                     **_blocks(64, 64))),
        # and of a chunk: thousands of lists
        named("select_chunk", _case("select", 32, 8, 128, "512@32768", 16, 4096, 16384,
                                    **_blocks(32, 64))),
        # one very long request alone: few rows, launch latency and a cut list
        named("attention_one", _case("attention", 32, 8, 128, "", 1, 131071, 131071,
                                     **_blocks(64, 32))),
        # long-context decoding at the 70B head shape with a short chunk beside it
        named("attention_70b", _case("attention", 64, 8, 128, "128@32768", 32, 8192, 32768,
                                     **_blocks(64, 64))),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(("pages", "rope", "summary", "scores", "scores", "select", "attention",
                       "attention", "attention"))
    hq, hkv, d = rng.choice(HEADS)
    seed = rng.randrange(1 << 30)

    def chunks(most, longest, cached):
        return ",".join("%d@%d" % (_log_int(rng, 2, longest), _log_int(rng, 1, cached) - 1)
                        for _ in range(rng.randrange(most + 1)))

    if kind == "pages":
        lo = _log_int(rng, 1, 4096)
        n = _log_int(rng, 1, 500)
        return _case(kind, hq, hkv, d, chunks(3, 20000, 8192), n, lo, _log_int(rng, lo, 16384),
                     seed, ended=rng.randrange(n // 4 + 1))
    if kind == "rope":
        lo = _log_int(rng, 1, 4096)
        return _case(kind, hq, hkv, d, chunks(2, 1500, 60000), _log_int(rng, 1, 128), lo,
                     _log_int(rng, lo, 8192), seed, layout=rng.choice((INTERLEAVED, HALF)),
                     rotary=16 * rng.randrange(1, d // 16 + 1),
                     factor=rng.choice((1.0, 4.0, 8.0)))
    block = rng.choice((16, 32, 64, 128))
    if kind == "summary":
        lo = _log_int(rng, 1, 8192)
        return _case(kind, hq, hkv, d, chunks(2, 12000, 8192), _log_int(rng, 1, 64), lo,
                     _log_int(rng, lo, 16384), seed, block=block)
    sink, recent = rng.choice((0, 1, 2)), rng.choice((1, 2, 3))
    if kind == "attention":
        top = max(sink + recent, _log_int(rng, 4, 4096 // block))
        parts, n = chunks(1, 100, 20000), _log_int(rng, 1, 32)
    else:
        top = sink + recent + _log_int(rng, 1, 128)
        parts, n = chunks(2, 200, 20000), _log_int(rng, 1, 32)
    lo = _log_int(rng, 1, 20000)
    return _case(kind, hq, hkv, d, parts, n, lo, _log_int(rng, lo, 20000), seed,
                 **_blocks(block, top, sink, recent))


def _lengths(case):
    """(c, u) of every request: new and cached tokens."""
    rng = np.random.default_rng(case["len_seed"])
    pairs = [tuple(int(v) for v in part.split("@")) for part in case["chunks"].split(",") if part]
    lo, hi = max(1, case["lo"]), max(1, case["hi"])
    u = np.rint(np.exp(rng.uniform(math.log(lo), math.log(hi), case["decodes"]))).astype(np.int64)
    c = np.array([p[0] for p in pairs] + [1] * case["decodes"], dtype=np.int64)
    u = np.array([p[1] for p in pairs] + u.tolist(), dtype=np.int64)
    return c, u


def _old_new(case):
    """pages: the requests' lengths before and after."""
    c, u = _lengths(case)
    new = u + c
    n = len(new)
    gone = np.random.default_rng(case["len_seed"] + 1).permutation(n)[:case["ended"]]
    new[gone] = 0
    back = gone[::3]  # some lose only a part (rejected drafts, a cut context)
    new[back] = u[back] // 2
    return u, new


def _ceil(a, b):
    return -(-a // b)


def _visible(case):
    """Per new row: its request, its position, and the blocks that start no later."""
    c, u = _lengths(case)
    req = np.repeat(np.arange(len(c)), c)
    first = np.cumsum(c) - c
    pos = np.arange(len(req)) - first[req] + u[req]
    return req, pos, pos // case["block"] + 1


def _stride(case):
    """Blocks that a row of the scores has room for: those of the longest request, a
    multiple of four."""
    c, u = _lengths(case)
    return int(_ceil(_ceil((u + c)[c > 0].max(), case["block"]), 4) * 4)


def work(case):
    """Bytes and operations of one pass: each input and output once."""
    hq, hkv, d, kind = case["hq"], case["hkv"], case["d"], case["kind"]
    c, u = _lengths(case)
    tokens = int(c.sum())
    if kind == "pages":
        old, new = _old_new(case)
        p, q = _ceil(old, PAGE), _ceil(new, PAGE)
        rows = int(np.maximum(new - old, 0).sum())
        moved = int(np.abs(p - q).sum())
        return {"bytes": 8 * len(old) + 8 * moved + 4 * (len(old) + 1) + 8 * rows + 32, "flops": 0}
    if kind == "rope":
        row = (hq + 2 * hkv) * d * 2
        return {"bytes": tokens * (2 * row + 4 * case["rotary"]),
                "flops": 3 * tokens * (hq + hkv) * case["rotary"]}
    block = case["block"]
    if kind == "summary":
        first = u // block
        keys = int((u + c - first * block).sum())
        return {"bytes": 2 * hkv * d * keys + 4 * hkv * d * int((_ceil(u + c, block) - first).sum()),
                "flops": 0}
    req, pos, seen = _visible(case)
    if kind == "scores":
        blocks = int(_ceil(u + c, block)[c > 0].sum())
        return {"bytes": 4 * d * hkv * blocks + 2 * hq * d * tokens + 4 * hkv * int(seen.sum()),
                "flops": 4 * hq * d * int(seen.sum())}
    if kind == "select":
        return {"bytes": 4 * hkv * (int(seen.sum()) + tokens * case["top"]), "flops": 0}
    # every listed block is whole but the row's own one
    keys = (np.minimum(seen, case["top"]) - 1) * block + pos % block + 1
    per_req = np.minimum(np.bincount(req, keys, len(c)), u + c).sum()
    return {"bytes": int(4 * hkv * d * per_req) + 4 * hq * d * tokens + 4 * hkv * tokens * case["top"],
            "flops": int(4 * hq * d * keys.sum())}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] == "pages":
        return _prepare_pages(case, gen)
    kind, hq, hkv, d = case["kind"], case["hq"], case["hkv"], case["d"]
    c, u = _lengths(case)
    n, T, length = len(c), int(c.sum()), u + c
    normal = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)  # noqa: E731
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    pages = _ceil(length, PAGE)
    num_pages, width = int(pages.sum()) + 7, int(pages.max())
    at = np.full((n, width), num_pages - 1, dtype=np.int64)
    first = np.cumsum(pages) - pages
    for i in range(n):
        at[i, :pages[i]] = first[i] + np.arange(pages[i])
    order = torch.randperm(num_pages, generator=gen, device="cuda").int()
    req = np.repeat(np.arange(n), c)
    pos = np.arange(T) - np.repeat(np.cumsum(c) - c, c) + np.repeat(u, c)
    state = {"case": case, "c": c, "u": u, "num_pages": num_pages, "width": width,
             "block_table": order[dev(at)], "scale": float(np.float32(1 / math.sqrt(d))),
             "req": dev(req), "pos": dev(pos)}
    if kind == "rope":
        state["qkv"] = normal(T, (hq + 2 * hkv) * d)
        state["k_cache"] = normal(num_pages, hkv, PAGE, d)
        state["v_cache"] = normal(num_pages, hkv, d, PAGE)
        angle = torch.arange(int(length.max()), dtype=torch.float64, device="cuda")[:, None] * (
            _turns(case))
        state["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
        return state
    if kind == "summary":
        state["k_cache"] = normal(num_pages, hkv, PAGE, d)
        state["summary"] = normal(num_pages, hkv, 2, d)
        return state
    if kind == "scores":
        state["q"] = normal(T, hq, d)
        # the extremes of a block of normal keys
        lift = torch.tensor([1.0, -1.0], device="cuda")[:, None] * math.sqrt(2 * math.log(case["block"]))
        state["summary"] = (0.4 * normal(num_pages, hkv, 2, d) + lift).to(torch.bfloat16)
        state["scores"] = torch.zeros((T, hkv, _stride(case)), device="cuda")
        return state
    # a request's blocks matter in much the same way to its neighbouring rows
    base = torch.empty((n, hkv, _stride(case)), device="cuda").normal_(generator=gen)
    scores = torch.empty((T, hkv, _stride(case)), device="cuda").normal_(generator=gen)
    scores = scores.mul_(3.0).addcmul_(base[state["req"]], torch.tensor(8.0, device="cuda")).add_(60.0)
    state["seen"] = dev(np.asarray(pos // case["block"] + 1))
    if kind == "select":
        state["scores"] = scores
        return state
    state["blocks"] = _chosen(scores, state["seen"], case)
    state["q"] = 1.5 * normal(T, hq, d)
    state["k_cache"] = normal(num_pages, hkv, PAGE, d)
    state["v_cache"] = normal(num_pages, hkv, d, PAGE)
    return state


def _prepare_pages(case, gen):
    old, new = _old_new(case)
    n = len(old)
    held, wanted = _ceil(old, PAGE), _ceil(new, PAGE)
    spare = int(np.maximum(wanted - held, 0).sum()) + 100
    num_pages = int(held.sum()) + spare
    width = int(max(held.max(), wanted.max()))
    order = torch.randperm(num_pages, generator=gen, device="cuda").int()
    table = np.full((n, width), -1, dtype=np.int64)
    first = np.cumsum(held) - held
    for i in range(n):
        table[i, :held[i]] = first[i] + np.arange(held[i])
    table = torch.from_numpy(table).cuda()
    table = torch.where(table < 0, -1, order[table.clamp(min=0)])
    # the ring's free entries begin somewhere and may wrap
    head = int(torch.randint(num_pages, (1,), generator=gen, device="cuda"))
    ring = torch.full((num_pages,), -1, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(spare, device="cuda")) % num_pages] = order[num_pages - spare:]
    rows = int(np.maximum(new - old, 0).sum())
    return {"case": case, "num_pages": num_pages, "width": width,
            "old_len": torch.from_numpy(old).int().cuda(),
            "new_len": torch.from_numpy(new).int().cuda(), "block_table": table.int(),
            "free_pages": ring,
            "page_state": torch.tensor([head, spare, 0, 0], dtype=torch.int32, device="cuda"),
            "page_state_out": torch.zeros(4, dtype=torch.int32, device="cuda"),
            "row_start": torch.zeros(n + 1, dtype=torch.int32, device="cuda"),
            "slots": torch.zeros(rows, dtype=torch.int64, device="cuda")}


def _turns(case):
    """The pairs' angles per position, in 64 bits: full below a wavelength of 2048
    positions, divided by ``factor`` above 8192, blended in between."""
    t = torch.pow(torch.tensor(ROPE_BASE, dtype=torch.float64, device="cuda"),
                  -torch.arange(0, case["rotary"], 2, dtype=torch.float64, device="cuda") / case["rotary"])
    keep = ((8192 * t / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
    return keep * t + (1.0 - keep) * t / case["factor"]


def _chosen(score, seen, case):
    """Lists [T, hkv, top] of the blocks chosen by scores [T, hkv, stride], ascending, -1
    behind them: the first `sink`, the last `recent` and the highest others, the lowest
    index of equals first."""
    b = torch.arange(score.shape[2], device="cuda")
    last = seen[:, None, None]
    here = (b < last).expand(score.shape)
    always = here & ((b < case["sink"]) | (b >= last - case["recent"]))
    by = torch.sort(score, dim=2, descending=True, stable=True).indices
    # what has to stay before the others and what is not there last
    level = torch.where(always, 2, here.int()).gather(2, by)
    by = by.gather(2, torch.sort(level, dim=2, descending=True, stable=True).indices)
    by = by[:, :, :case["top"]]
    by = torch.where(torch.arange(by.shape[2], device="cuda") < last, by, score.shape[2])
    by = torch.sort(by, dim=2).values
    out = torch.full((*score.shape[:2], case["top"]), -1, dtype=torch.int32, device="cuda")
    out[:, :, :by.shape[2]] = torch.where(by < score.shape[2], by, -1).int()
    return out


def _pages(state):
    old, new, table = state["old_len"].long(), state["new_len"].long(), state["block_table"]
    ring, N = state["free_pages"], state["num_pages"]
    head, count = state["page_state"][0].long(), state["page_state"][1].long()
    held, wanted = (old + PAGE - 1) // PAGE, (new + PAGE - 1) // PAGE

    def spread(lo, hi):
        """(request, index) of every index in [lo, hi) of each request"""
        k = (hi - lo).clamp(min=0)
        which = torch.repeat_interleave(torch.arange(len(k), device="cuda"), k)
        return which, torch.arange(len(which), device="cuda") - (k.cumsum(0) - k)[which] + lo[which]

    req, index = spread(held, wanted)
    table[req, index] = ring[(head + torch.arange(len(req), device="cuda")) % N]
    back, at = spread(wanted, held)
    ring[(head + count + torch.arange(len(back), device="cuda")) % N] = table[back, at]
    out = state["page_state_out"]
    out.zero_()
    out[0] = (head + len(req)) % N
    out[1] = count - len(req) + len(back)
    state["row_start"][1:] = (new - old).clamp(min=0).cumsum(0)
    req, t = spread(old, new)
    state["slots"].copy_(table[req, t // PAGE].long() * PAGE + t % PAGE)
    return {k: state[k] for k in ("block_table", "free_pages", "page_state_out", "row_start", "slots")}


def _rope(state):
    case = state["case"]
    hq, hkv, d, r = case["hq"], case["hkv"], case["d"], case["rotary"]
    x = state["qkv"].float().view(-1, hq + 2 * hkv, d)
    cs = state["cos_sin"][state["pos"]][:, None]
    cos, sin = cs[..., :r // 2], cs[..., r // 2:]
    part = x[:, :hq + hkv, :r]
    if case["layout"] == HALF:
        a, b = part[..., :r // 2], part[..., r // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=3).flatten(2)
    turned = torch.cat([turned, x[:, :hq + hkv, r:]], dim=2).to(torch.bfloat16)
    page = state["block_table"][state["req"], state["pos"] // PAGE].long()
    slot = state["pos"] % PAGE
    state["k_cache"][page, :, slot] = turned[:, hq:]
    state["v_cache"][page, :, :, slot] = x[:, hq + hkv:].to(torch.bfloat16)
    return {"q": turned[:, :hq], "k": state["k_cache"], "v": state["v_cache"]}


def _summary(state):
    case, c, u = state["case"], state["c"], state["u"]
    block = case["block"]
    for i in range(len(c)):
        first, last = int(u[i]) // block, int(_ceil(u[i] + c[i], block))
        pos = torch.arange(first * block, last * block, device="cuda")
        here = pos < int(u[i] + c[i])
        pos = pos.clamp(max=int(u[i] + c[i]) - 1)
        k = state["k_cache"][state["block_table"][i, pos // PAGE].long(), :, pos % PAGE].float()
        k = k.view(last - first, block, case["hkv"], case["d"])
        here = here.view(last - first, block, 1, 1)
        hi = torch.where(here, k, -math.inf).amax(dim=1)
        lo = torch.where(here, k, math.inf).amin(dim=1)
        page = state["block_table"][i, torch.arange(first, last, device="cuda") * (block // PAGE)].long()
        state["summary"][page] = torch.stack([hi, lo], dim=2).to(torch.bfloat16)
    return state["summary"]


def _bounds(q, s):
    """q [n, hkv, rows, G, d], summaries [n, hkv, blocks, 2, d], 32 bits: the bounds of
    rows and blocks [n, hkv, rows, blocks]."""
    n, hkv, rows, g, d = q.shape
    q = q.reshape(n * hkv, rows * g, d)
    s = s.reshape(n * hkv, -1, 2, d).permute(2, 0, 3, 1)
    b = torch.bmm(q.clamp(min=0), s[0].contiguous()) + torch.bmm(q.clamp(max=0), s[1].contiguous())
    return b.view(n, hkv, rows, g, -1).amax(dim=3)


def _scores(state):
    case, c, u = state["case"], state["c"], state["u"]
    hq, hkv, d, block = case["hq"], case["hkv"], case["d"], case["block"]
    start = np.cumsum(c) - c
    ones = np.flatnonzero(c == 1)
    parts = [[i] for i in np.flatnonzero(c > 1)] + ([ones] if len(ones) else [])
    for index in parts:  # a chunk alone, all single rows together
        most = int(_ceil(u[index] + c[index], block).max())
        table = state["block_table"][torch.as_tensor(np.asarray(index), device="cuda")]
        b = torch.arange(most, device="cuda") * (block // PAGE)
        s = state["summary"][table[:, b].long()].float().permute(0, 2, 1, 3, 4)
        rows = int(c[index[0]])
        row = torch.as_tensor(start[index], device="cuda")[:, None] + torch.arange(rows, device="cuda")
        q = state["q"][row].float().view(len(index), rows, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4)
        got = _bounds(q, s).permute(0, 2, 1, 3)
        here = torch.arange(most, device="cuda") <= (state["pos"][row] // block)[:, :, None, None]
        state["scores"][row, :, :most] = torch.where(here, got, state["scores"][row, :, :most])
    return state["scores"]


def _attention(state):
    case = state["case"]
    hq, hkv, d, block, top = case["hq"], case["hkv"], case["d"], case["block"], case["top"]
    g, T, keys = hq // hkv, len(state["req"]), case["top"] * block
    out = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 28) // (hkv * keys * d))
    heads = torch.arange(hkv, device="cuda")[None, :, None]
    for at in range(0, T, step):
        rows = slice(at, min(T, at + step))
        lists = state["blocks"][rows].long()
        n = lists.shape[0]
        pos = (lists[..., None] * block + torch.arange(block, device="cuda")).view(n, hkv, keys)
        seen = (pos >= 0) & (pos <= state["pos"][rows][:, None, None])
        pos = torch.where(seen, pos, 0)
        page = state["block_table"][state["req"][rows][:, None, None], pos // PAGE].long()
        k = state["k_cache"][page, heads, pos % PAGE].float().view(n * hkv, keys, d)
        q = state["q"][rows].float().view(n * hkv, g, d)
        s = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(state["scale"])
        s.masked_fill_(~seen.view(n * hkv, 1, keys), -math.inf)
        s.sub_(s.amax(dim=2, keepdim=True)).exp_()
        s.div_(s.sum(dim=2, keepdim=True))
        v = state["v_cache"][page, heads, :, pos % PAGE].float().view(n * hkv, keys, d)
        out[rows] = torch.bmm(s, v).view(n, hq, d).to(torch.bfloat16)
    return out


def _handle(state):
    """The shape, the plans and the buffers that a serving program keeps for a batch, made
    on the first pass over it."""
    if "handle" in state:
        return state["handle"]
    from paper_2606_05933_amd import ssa
    case = state["case"]
    kind, hq, hkv, d = case["kind"], case["hq"], case["hkv"], case["d"]
    shape = ssa.make_shape(hq, hkv, d, state["num_pages"], state["width"], state.get("scale", 1.0))
    h = {"shape": shape}
    if kind == "pages":
        state["handle"] = h
        return h
    c, u = state["c"], state["u"]
    T = int(c.sum())
    ws_bytes = 0
    if kind in ("rope", "summary"):
        plan, _ = ssa.ssa_plan(shape, c, u)
    else:
        plan, ws_bytes, _ = ssa.sparse_plan(shape, c, u, case["block"], case["top"], case["sink"],
                                            case["recent"])
    h["plan"], h["plan_dev"] = plan, torch.from_numpy(plan).cuda()
    if kind == "rope":
        h["q"] = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")
    if kind == "select":
        h["blocks"] = torch.empty((T, hkv, case["top"]), dtype=torch.int32, device="cuda")
    if kind == "attention":
        h["workspace"] = torch.zeros(max(ws_bytes, 256), dtype=torch.uint8, device="cuda")
        h["out"] = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")
    state["handle"] = h
    return h


def _own(state):
    from paper_2606_05933_amd import ssa
    h, case, kind = _handle(state), state["case"], state["case"]["kind"]
    if kind == "pages":
        ssa.pages_resize(h["shape"], state["old_len"], state["new_len"], state["block_table"],
                         state["free_pages"], state["page_state"], state["page_state_out"],
                         state["row_start"], state["slots"])
        return {k: state[k] for k in ("block_table", "free_pages", "page_state_out", "row_start",
                                      "slots")}
    plan = (h["shape"], h["plan"], h["plan_dev"])
    if kind == "rope":
        ssa.rope_append_as(*plan, state["qkv"], state["cos_sin"], h["q"], state["k_cache"],
                           state["v_cache"], state["block_table"], layout=case["layout"],
                           rotary_dim=case["rotary"])
        return {"q": h["q"], "k": state["k_cache"], "v": state["v_cache"]}
    if kind == "summary":
        ssa.block_summary(*plan, case["block"], state["k_cache"], state["block_table"],
                          state["summary"])
        return state["summary"]
    if kind == "scores":
        ssa.block_scores(*plan, state["q"], state["summary"], state["block_table"], state["scores"])
        return state["scores"]
    if kind == "select":
        ssa.block_select(*plan, state["scores"], h["blocks"])
        return h["blocks"]
    ssa.sparse_attention(*plan, state["q"], state["k_cache"], state["v_cache"],
                         state["block_table"], state["blocks"], h["out"], h["workspace"])
    return h["out"]


def run(state):
    """One pass through the operator."""
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "pages":
        return _pages(state)
    if kind == "rope":
        return _rope(state)
    if kind == "summary":
        return _summary(state)
    if kind == "scores":
        return _scores(state)
    if kind == "select":
        return _chosen(state["scores"], state["seen"], state["case"])
    return _attention(state)


def exact(case, seed):
    """What ``run`` returns, request by request and in 64 bits."""
    kind = case["kind"]
    if kind in ("pages", "select"):
        return None  # whole numbers
    state = prepare(case, seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g = hq // hkv
    f64 = {"dtype": torch.float64, "device": "cuda"}
    if kind == "rope":
        keys, values = state["k_cache"].double(), state["v_cache"].double()
        turns = _turns(case)
    elif kind == "summary":
        result = state["summary"].double()
    elif kind == "scores":
        result = state["scores"].double()
    outs, row = [], 0
    for i, (c, u) in enumerate(zip(state["c"].tolist(), state["u"].tolist())):
        pages = state["block_table"][i, :_ceil(u + c, PAGE)].long()
        if kind == "rope":
            r = case["rotary"]
            x = state["qkv"][row:row + c].double().view(c, hq + 2 * hkv, d)
            p = torch.arange(c, **f64) + u
            turn = torch.polar(torch.ones((), **f64), p[:, None] * turns)[:, None]
            a = x[:, :hq + hkv, :r]
            pairs = a.unflatten(2, (2, -1)).transpose(2, 3) if case["layout"] == HALF else a.unflatten(2, (-1, 2))
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = (z.transpose(2, 3) if case["layout"] == HALF else z).flatten(2)
            z = torch.cat([z, x[:, :hq + hkv, r:]], dim=2)
            outs.append(z[:, :hq])
            flat = keys[pages].transpose(1, 2).reshape(-1, hkv, d)
            flat[u:u + c] = z[:, hq:]
            keys[pages] = flat.view(-1, PAGE, hkv, d).transpose(1, 2)
            flat = values[pages].permute(0, 3, 1, 2).reshape(-1, hkv, d)
            flat[u:u + c] = x[:, hq + hkv:]
            values[pages] = flat.view(-1, PAGE, hkv, d).permute(0, 2, 3, 1)
            row += c
            continue
        block = case["block"]
        starts = pages[::block // PAGE]
        if kind == "summary":
            k = state["k_cache"][pages].transpose(1, 2).reshape(-1, hkv, d)[:u + c].double()
            for b in range(u // block, _ceil(u + c, block)):
                part = k[b * block:(b + 1) * block]
                result[starts[b], :, 0] = part.max(dim=0).values
                result[starts[b], :, 1] = part.min(dim=0).values
            continue
        if kind == "scores":
            s = state["summary"][starts].double()
            for h in range(hkv):
                # the higher of q hi and q lo, as the mean of both and half their distance
                mid, span = (s[:, h, 0] + s[:, h, 1]) / 2, (s[:, h, 0] - s[:, h, 1]) / 2
                for j in range(c):
                    q = state["q"][row + j, h * g:(h + 1) * g].double()
                    b = (u + j) // block + 1
                    best = q @ mid[:b].T.contiguous() + q.abs() @ span[:b].abs().T.contiguous()
                    result[row + j, h, :b] = best.max(dim=0).values
            row += c
            continue
        for j in range(c):
            for h in range(hkv):
                b = state["blocks"][row + j, h].long()
                t = (b[b >= 0][:, None] * block + torch.arange(block, device="cuda")).flatten()
                t = t[t <= u + j]
                k = state["k_cache"][pages[t // PAGE], h, t % PAGE].double()
                v = state["v_cache"][pages[t // PAGE], h, :, t % PAGE].double()
                q = state["q"][row + j, h * g:(h + 1) * g].double()
                outs.append(torch.softmax(q @ k.T.contiguous() * state["scale"], dim=1) @ v)
        row += c
    if kind == "rope":
        return {"q": torch.cat(outs), "k": keys, "v": values}
    return torch.cat(outs).view(-1, hq, d) if kind == "attention" else result
