"""Sampled verification over long contexts, as cases that can be timed and checked.

Three operators of a verification step whose context is long and whose answer is sampled:

  select  which blocks of the committed cache each drafted token reads.  A block is 64 rows; of its
          keys the bounds of every channel are kept in 8 bits.  hi and lo are the largest and the
          smallest key, s = 2^(floor(log2(max |hi|, |lo|)) - 6) over all channels,
          HI = ceil(hi / s) and LO = floor(lo / s), both within -127 .. 127; a query is
          held likewise, Q = rint(q / s').  A block's score for a token is the largest over the
          query heads of the key head of s s' sum_c (max(Q, 0) HI + min(Q, 0) LO), which is exact.
          Read are the first `sinks` and the last `recent` blocks and the best of the others,
          `count` in all, the lowest index on ties.  A pass first computes the bounds of
          `fresh` blocks, the last, which became complete, or all behind a prompt; these are returned
          too, as the numbers that they stand for.
  attend  attention of the drafted tokens over the blocks that each has selected, over the committed
          rows behind the last whole block and over the drafted rows that it sees.
  accept  acceptance of drafted tokens against the target's probabilities p = softmax(logits / T)
          from given numbers u in [0, 1).  The children of an accepted node are tried in order:
          without draft probabilities x is accepted if u sum(p) < p(x), else p(x) becomes 0; with
          them if u q(x) < p(x), else p becomes max(p - q, 0) and q(x) becomes 0, both normalised.
          Where no child is accepted the next token is drawn from p with the root's u.

A selection is held as words of 64 bits, [key heads, ceil(M / 64), whole blocks]: bit i % 64 of word
i / 64 says that token i reads the block.
"""
import hashlib
import math

import torch

own = False         # False: elementary torch operations; True: the calls of paper_2505_23219_amd

BLOCK = 64          # committed rows that are selected together


def listed():
    return [
        # One token over a long context, four query heads to a key head; a block has just become whole.
        {"name": "select_decode_128k", "op": "select", "M": 1, "nh": 32, "nkv": 8, "d": 128, "kv": 131072,
         "count": 64, "sinks": 1, "recent": 2, "fresh": "last", "layout": "heads"},
        # A 64-node tree of a 7B-shaped model over a long context: every node selects for itself.
        {"name": "select_tree64_32k", "op": "select", "M": 64, "nh": 32, "nkv": 32, "d": 128, "kv": 32771,
         "count": 32, "sinks": 1, "recent": 2, "fresh": "last", "layout": "heads"},
        # A small model, five query heads to a key head, rows of all heads side by side: latency.
        {"name": "select_small_ragged", "op": "select", "M": 5, "nh": 20, "nkv": 4, "d": 64, "kv": 1931,
         "count": 7, "sinks": 0, "recent": 1, "fresh": "last", "layout": "tokens"},
        # The first step behind a prompt: the bounds of all blocks, then a 16-node tree's selection.
        {"name": "select_prompt_16k", "op": "select", "M": 16, "nh": 32, "nkv": 32, "d": 128, "kv": 16384,
         "count": 32, "sinks": 1, "recent": 1, "fresh": "all", "layout": "heads"},
        # One token's attention over 64 of 2047 blocks: long-context decoding.
        {"name": "attend_decode_128k", "op": "attend", "M": 1, "nh": 32, "nkv": 8, "d": 128, "kv": 131071,
         "count": 64, "pool": 64, "mask": "tree", "tree": "chain", "layout": "heads"},
        # The tree of the second case: nodes of one tree mostly agree on what they read.
        {"name": "attend_tree64_32k", "op": "attend", "M": 64, "nh": 32, "nkv": 32, "d": 128, "kv": 32771,
         "count": 32, "pool": 48, "mask": "tree", "tree": "random", "layout": "heads"},
        # Draft sequences side by side over a short odd context.
        {"name": "attend_small_ragged", "op": "attend", "M": 37, "nh": 20, "nkv": 4, "d": 64, "kv": 777,
         "count": 5, "pool": 9, "mask": "sequences", "tree": "random", "layout": "tokens"},
        # The widest tree over half of the 13B-shaped workload's cache.
        {"name": "attend_chain128_13b", "op": "attend", "M": 128, "nh": 40, "nkv": 40, "d": 128, "kv": 8192,
         "count": 64, "pool": 96, "mask": "tree", "tree": "chain", "layout": "heads"},
        # A small vocabulary, eight nodes, drafts without probabilities: latency.
        {"name": "accept_tiny", "op": "accept", "M": 8, "V": 1000, "tree": "random", "q": "none", "T": 1.0},
        # The benchmark's tree and vocabulary; drafting heads' best candidates, as this library drafts.
        {"name": "accept_tree64", "op": "accept", "M": 64, "V": 32000, "tree": "random", "q": "none", "T": 0.8},
        # The same with candidates drawn from the heads' distributions, one for every depth.
        {"name": "accept_heads64", "op": "accept", "M": 64, "V": 32000, "tree": "wide", "q": "depths", "T": 0.7},
        # A draft model's chain over a large vocabulary.
        {"name": "accept_chain128", "op": "accept", "M": 128, "V": 131072, "tree": "chain", "q": "rows", "T": 1.0},
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["select", "attend", "accept"])
    M, tree = _log(rng, 1, 128), rng.choice(["chain", "random", "wide"])
    if op == "accept":
        V = _log(rng, 256, 131072)
        return {"op": op, "M": M, "V": V, "tree": tree, "q": rng.choice(["none", "depths", "rows"]),
                "T": round(rng.uniform(0.3, 1.5), 3)}
    d, rep, nkv = rng.choice([64, 128, 128]), rng.choice([1, 1, 2, 4, 5, 8]), _log(rng, 1, 40)
    kv, count = _log(rng, BLOCK, 131072), _log(rng, 1, 64)
    while M * nkv * rep > 128 * 40:
        M = (M + 1) // 2
    if op == "select":
        fresh = rng.choice(["last", "last", "all"])
        while kv * nkv * d > (131072 * 8 if fresh == "last" else 16384 * 32) * 128:
            kv = kv * 3 // 4
        while M * nkv * rep * (kv // BLOCK) * d > 64 * 32 * 512 * 128:
            M = (M + 1) // 2
        sinks = rng.randint(0, min(2, count))
        return {"op": op, "M": M, "nh": nkv * rep, "nkv": nkv, "d": d, "kv": kv, "count": count, "sinks": sinks,
                "recent": rng.randint(0, min(2, count - sinks)), "fresh": fresh, "layout": rng.choice(["heads", "tokens"])}
    kv = rng.choice([kv, kv, kv, rng.randint(1, BLOCK)])
    while kv * nkv * d > 131072 * 8 * 128:
        kv = kv * 3 // 4
    pool = int(count * rng.uniform(1.0, 1.5))
    return {"op": op, "M": M, "nh": nkv * rep, "nkv": nkv, "d": d, "kv": kv, "count": count, "pool": pool,
            "mask": rng.choice(["tree", "tree", "sequences", "sparse"]), "tree": tree,
            "layout": rng.choice(["heads", "tokens"])}


# ---- inputs -------------------------------------------------------------------------
def _gen(seed, *tags):
    g = torch.Generator(device="cuda")
    g.manual_seed(int.from_bytes(hashlib.sha256(repr((int(seed),) + tags).encode()).digest()[:7], "little"))
    return g


def _normal(shape, seed, *tags):
    return torch.randn(shape, generator=_gen(seed, *tags), device="cuda", dtype=torch.float32)


def _uniform(shape, seed, *tags):
    return torch.rand(shape, generator=_gen(seed, *tags), device="cuda", dtype=torch.float32)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _parent(case, seed):
    """parent[] of the draft tree: a chain, a random tree of depth at most 5, or a wide
    shallow one (a root, M/8 children, grandchildren)."""
    M, kind = case["M"], case["tree"]
    r = torch.Generator().manual_seed(int(seed) * 7919 + M)
    parent, depth = [-1], [0]
    for i in range(1, M):
        if kind == "chain":
            p = i - 1
        elif kind == "wide":
            p = 0 if i <= (M + 7) // 8 else 1 + int(torch.randint((M + 7) // 8, (1,), generator=r))
        else:
            ok = [j for j in range(i) if depth[j] < 5]
            p = ok[int(torch.randint(len(ok), (1,), generator=r))]
        parent.append(p)
        depth.append(depth[p] + 1)
    return parent, depth


def _capacity(case):
    return (case["kv"] + case["M"] + BLOCK - 1) // BLOCK * BLOCK


def _keys(case, seed):
    """The key cache [nkv, capacity, d]: every channel with a mean and a spread of its own, and rows
    of one passage (64 of them) more alike than others."""
    nkv, d, T = case["nkv"], case["d"], _capacity(case)
    spread = torch.exp(0.5 * _normal((nkv, 1, d), seed, "k", "spread"))
    k = _normal((nkv, T, d), seed, "k")
    k.view(nkv, T // BLOCK, BLOCK, d).add_(_normal((nkv, T // BLOCK, 1, d), seed, "k", "passage"))
    k = k.mul_(spread).add_(0.5 * _normal((nkv, 1, d), seed, "k", "mean")).half()
    if case["layout"] == "tokens":      # a row of the cache holds all heads
        k = k.transpose(0, 1).contiguous().transpose(0, 1)
    return k


def _values(case, seed):
    """The value cache, channel-major: [nkv, d, capacity]."""
    return _normal((case["nkv"], case["d"], _capacity(case)), seed, "v").half()


def _queries(case, seed):
    """[M, nh, d]: the tokens of a tree have much in common."""
    M, nh, d = case["M"], case["nh"], case["d"]
    return (0.8 * _normal((1, nh, d), seed, "q", "common") + 0.6 * _normal((M, nh, d), seed, "q")).half()


def _see_lists(case, seed):
    """Per drafted token the drafted tokens that it sees, as Python ints of bits."""
    M = case["M"]
    if case["mask"] == "tree":
        parent, see = _parent(case, seed)[0], [0] * M
        for i in range(M):
            see[i] = (1 << i) | (see[parent[i]] if i else 0)
        return see
    if case["mask"] == "sequences":     # draft sequences of 8 tokens side by side
        return [sum(1 << j for j in range(i // 8 * 8, i + 1)) for i in range(M)]
    # any relation: about a third of the pairs, every fifth token sees no drafted token at all
    bits = torch.rand((M, M), generator=torch.Generator().manual_seed(int(seed) + 17)) < 0.33
    bits[::5] = False
    return [sum(1 << j for j, b in enumerate(row) if b) for row in bits.tolist()]


def _mask_words(see):
    def word(x):
        x &= (1 << 64) - 1
        return x - (1 << 64) if x >> 63 else x
    return torch.tensor([[word(s), word(s >> 64)] for s in see], dtype=torch.int64, device="cuda")


def _chosen(case, seed):
    """Truth values [nkv, M, blocks]: every token reads `count` of a head's pool of blocks."""
    nkv, M, n = case["nkv"], case["M"], case["kv"] // BLOCK
    count, pool = min(case["count"], n), min(case["pool"], n)
    if n == 0:
        return torch.zeros((nkv, M, 0), dtype=torch.bool, device="cuda")
    at = _uniform((nkv, n), seed, "pool").topk(pool, dim=1).indices
    mine = _uniform((nkv, M, pool), seed, "mine").topk(count, dim=2).indices
    sel = torch.zeros((nkv, M, n), dtype=torch.bool, device="cuda")
    return sel.scatter_(2, at[:, None].expand(nkv, M, pool).gather(2, mine), True)


def _words(sel):
    """Truth values [nkv, M, blocks] to words [nkv, ceil(M / 64), blocks]."""
    nkv, M, n = sel.shape
    W = -(-M // 64)
    bits = torch.zeros((nkv, W * 64, n), dtype=torch.int64, device=sel.device)
    bits[:, :M] = sel
    shift = torch.arange(64, device=sel.device)[None, None, :, None]
    return (bits.view(nkv, W, 64, n) << shift).sum(2)


def _logits(case, seed):
    """Target logits [M, V]: a few likely tokens in every row."""
    M, V = case["M"], case["V"]
    x = _normal((M, V), seed, "logits").mul_(1.5)
    at = (_uniform((M, 8), seed, "top", "at") * V).long().clamp_(max=V - 1)
    return x.scatter_add_(1, at, 3 + 6 * _uniform((M, 8), seed, "top"))


def _accept_inputs(case, seed):
    M, V = case["M"], case["V"]
    parent, depth = _parent(case, seed)
    logits = _logits(case, seed)
    kids = [[] for _ in range(M)]
    for i in range(1, M):
        kids[parent[i]].append(i)
    q, row = None, None
    if case["q"] == "rows":             # a draft model: the distribution behind every node
        q = logits + 0.7 * _normal((M, V), seed, "draft")
    elif case["q"] == "depths":         # drafting heads: one distribution for the children of all nodes of a depth
        first = [depth.index(t) for t in range(max(depth) + 1)]
        q = logits[first] + 0.7 * _normal((len(first), V), seed, "draft")
        row = depth
    # Candidates are drawn without replacement from q (Gumbel noise), or are the best of noisy logits.
    most = max(1, max(len(c) for c in kids))
    if q is None:
        key = logits + 0.7 * _normal((M, V), seed, "draft")
    else:
        key = q / case["T"] if row is None else (q / case["T"])[row]
        key = key - torch.log(-torch.log(_uniform((M, V), seed, "gumbel").clamp_(1e-9, 1 - 1e-7)))
    best = key.topk(min(most, V), dim=1).indices.tolist()
    tokens = [int(torch.randint(V, (1,), generator=torch.Generator().manual_seed(int(seed) + 3)))] + [0] * (M - 1)
    for p in range(M):
        for r, c in enumerate(kids[p]):
            tokens[c] = best[p][min(r, V - 1)]
    return logits, _int32(tokens), parent, kids, _uniform((M,), seed, "u"), q, row


def prepare(case, seed):
    """What a program holds before the call: cache, bounds, a selection, a tree, random numbers, buffers."""
    op, s = case["op"], {"op": case["op"], "case": case}
    if own:
        from paper_2505_23219_amd import binding as B
    if op == "accept":
        s["logits"], s["tokens"], parent, kids, s["u"], s["q"], row = _accept_inputs(case, seed)
        M = case["M"]
        s["res"] = torch.zeros(2 + M, dtype=torch.int32, device="cuda")
        s["parent"] = _int32(parent)
        s["row"] = None if row is None else _int32(row)
        if own:
            s["ws"] = B.workspace(B.ghd_accept_sampled_workspace_bytes(M, case["V"]))
        else:
            # nodes that have an r-th child, and that child
            s["rounds"] = [(_int32([p for p in range(M) if len(kids[p]) > r]).long(),
                            _int32([kids[p][r] for p in range(M) if len(kids[p]) > r]).long())
                           for r in range(max(len(c) for c in kids))]
            s["deepest"] = max(_parent(case, seed)[1])
        return s
    s["q"], s["k"] = _queries(case, seed), _keys(case, seed)
    n = case["kv"] // BLOCK
    if op == "select":
        if own:
            s["bounds"] = B.BlockBounds(case["nkv"], case["d"], _capacity(case))
            B.ghd_block_bounds(s["bounds"], s["k"], 0, n)
            s["sel"] = torch.empty((case["nkv"], -(-case["M"] // 64), n), dtype=torch.int64, device="cuda")
            s["ws"] = B.workspace(B.ghd_block_select_workspace_bytes(case["M"], case["kv"], case["nkv"]))
        else:
            s["bounds"] = _plain_bounds(case, s["k"], 0, n)
        return s
    s["v"] = _values(case, seed)
    s["sel"] = _words(_chosen(case, seed))
    s["parent"] = _int32(_parent(case, seed)[0]) if case["mask"] == "tree" else None
    s["mask"] = _mask_words(_see_lists(case, seed))
    if own:
        s["out"] = torch.empty_like(s["q"])
        s["ws"] = B.workspace(B.ghd_sparse_attention_workspace_bytes(case["M"], case["kv"], case["nh"], case["nkv"],
                                                                     case["d"]))
    return s


# ---- the operators in plain form ------------------------------------------------------
def _fresh(case):
    n = case["kv"] // BLOCK
    return (0, n) if case["fresh"] == "all" else (n - 1, 1)


def _unit(a):
    """2^(floor(log2 a) - 6) of numbers a >= 0; 0 of 0, infinity of what is not finite."""
    one = torch.ones_like(a)
    u = torch.ldexp(one, torch.frexp(torch.where(torch.isfinite(a) & (a > 0), a, one)).exponent - 7)
    return torch.where(a > 0, torch.where(torch.isfinite(a), u, a.abs() * math.inf), torch.where(a == 0, a, one * math.inf))


def _codes(x, unit, rounding):
    """x / unit as whole numbers within -127 .. 127; 0 where there is no finite unit."""
    ok = (unit > 0) & torch.isfinite(unit)
    return torch.where(ok, rounding(x / torch.where(ok, unit, torch.ones_like(unit))), torch.zeros_like(x)).clamp_(-127, 127)


def _plain_bounds(case, k, first, n):
    """HI and LO [nkv, n, d] as 32-bit numbers and their unit [nkv, n]."""
    x = k[:, first * BLOCK:(first + n) * BLOCK].float().reshape(case["nkv"], n, BLOCK, case["d"])
    hi, lo = x.amax(2), x.amin(2)
    unit = _unit(torch.maximum(hi.abs(), lo.abs()).amax(2))[..., None]
    return [_codes(hi, unit, torch.ceil), _codes(lo, unit, torch.floor), unit[..., 0]]


def _plain_select(s):
    case = s["case"]
    M, nh, nkv, d, n = case["M"], case["nh"], case["nkv"], case["d"], case["kv"] // BLOCK
    first, fresh = _fresh(case)
    for held, new in zip(s["bounds"], _plain_bounds(case, s["k"], first, fresh)):
        held[:, first:first + fresh] = new
    hi, lo, unit = s["bounds"]
    q = s["q"].float()
    a = q.abs().amax(2, keepdim=True)
    step = _unit(a)
    code = _codes(q, step, torch.round)
    step = torch.where(torch.isfinite(step), step, torch.zeros_like(step))
    score = torch.full((nkv, M, n), -math.inf, device="cuda")
    rep = nh // nkv
    for h in range(nkv):
        for g in range(h * rep, (h + 1) * rep):
            t = code[:, g].clamp(min=0) @ hi[h].t() + code[:, g].clamp(max=0) @ lo[h].t()
            score[h] = torch.maximum(score[h], t * step[:, g])
    finite = torch.isfinite(unit)
    score = torch.where(finite[:, None], score * torch.where(finite, unit, torch.ones_like(unit))[:, None],
                        torch.full_like(score, math.inf))
    lo_end, hi_end = min(case["sinks"], n), max(min(case["sinks"], n), n - case["recent"])
    sel = torch.ones((nkv, M, n), dtype=torch.bool, device="cuda")
    keep = min(case["count"], n) - lo_end - (n - hi_end)
    sel[:, :, lo_end:hi_end] = False
    if keep > 0:
        best = torch.sort(score[:, :, lo_end:hi_end], dim=2, descending=True, stable=True).indices[:, :, :keep]
        sel.scatter_(2, best + lo_end, True)
    new = slice(first, first + fresh)
    return {"sel": _words(sel), "hi": hi[:, new] * unit[:, new, None], "lo": lo[:, new] * unit[:, new, None]}


def _ancestors(parent):
    M = parent.numel()
    i = torch.arange(M, device=parent.device)
    a = torch.eye(M, device=parent.device)
    a[i[1:], parent[1:].long()] = 1.0
    for _ in range(7):                  # paths of up to 2, 4, ... 128 edges
        a = (a @ a > 0).float()
    return a > 0


def _plain_attend(s):
    case = s["case"]
    M, nh, nkv, d, kv = (case[n] for n in ("M", "nh", "nkv", "d", "kv"))
    rep, n, i = nh // nkv, kv // BLOCK, torch.arange(case["M"], device="cuda")
    tree = _ancestors(s["parent"]) if s["parent"] is not None else ((s["mask"][:, i // 64] >> (i % 64)) & 1) > 0
    sel = (s["sel"][:, i // 64] >> (i % 64)[None, :, None]) & 1 > 0                 # [nkv, M, n]
    out = torch.empty((M, nh, d), dtype=torch.float32, device="cuda")
    for h in range(nkv):
        see = torch.ones((M, kv + M), dtype=torch.bool, device="cuda")
        see[:, :n * BLOCK] = sel[h].repeat_interleave(BLOCK, dim=1)
        see[:, kv:] = tree
        k, v = s["k"][h, :kv + M].float(), s["v"][h, :, :kv + M].float()
        q = s["q"][:, h * rep:(h + 1) * rep].float().reshape(M * rep, d)
        t = (q @ k.t() * (1.0 / math.sqrt(d))).view(M, rep, kv + M)
        t = torch.where(see[:, None], t, torch.full_like(t, -math.inf))
        top = t.amax(2, keepdim=True)
        p = torch.exp(t - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = p.sum(2, keepdim=True)
        p = p / torch.where(total > 0, total, torch.ones_like(total))               # a row that sees nothing: zeros
        out[:, h * rep:(h + 1) * rep] = (p.view(M * rep, -1) @ v.t()).view(M, rep, d)
    return out.half()


def _plain_accept(s):
    """In 64 bits: a token is drawn where a long sum passes a number.  All nodes at once, their children
    one after another; the path is walked at the end."""
    case = s["case"]
    M, T = case["M"], case["T"]

    def softmax(x):
        x = x.double() / T
        w = torch.exp(x - x.amax(1, keepdim=True))
        return w / w.sum(1, keepdim=True)
    p, token, u = softmax(s["logits"]), s["tokens"].long(), s["u"].double()
    q = None
    if s["q"] is not None:
        q = softmax(s["q"])
        q = q.clone() if s["row"] is None else q[s["row"].long()]
    taken = torch.full((M,), -1, dtype=torch.long, device="cuda")
    for node, child in s["rounds"]:
        at = (node, token[child])
        px = p[at]
        ok = u[child] * p[node].sum(1) < px if q is None else u[child] * q[at] < px
        open_ = taken[node] < 0
        taken[node] = torch.where(open_ & ok, child, taken[node])
        no = (open_ & ~ok)[:, None]
        if q is None:
            p[at] = torch.where(no[:, 0], torch.zeros_like(px), px)
            continue
        rest = (p[node] - q[node]).clamp_(min=0)
        total = rest.sum(1, keepdim=True)
        p[node] = torch.where(no & (total > 0), rest / torch.where(total > 0, total, torch.ones_like(total)), p[node])
        left = q[node].scatter(1, token[child][:, None], 0.0)
        total = left.sum(1, keepdim=True)
        q[node] = torch.where(no, left / torch.where(total > 0, total, torch.ones_like(total)), q[node])
    res = s["res"].zero_()
    cur = torch.zeros(1, dtype=torch.long, device="cuda")
    length, going = torch.ones(1, dtype=torch.long, device="cuda"), torch.ones(1, dtype=torch.bool, device="cuda")
    for t in range(s["deepest"]):
        nxt = taken[cur]
        going = going & (nxt >= 0)
        cur = torch.where(going, nxt, cur)
        length = length + going
        res[3 + t:4 + t] = torch.where(going, cur, torch.zeros_like(cur)).int()
    row = p[cur[0]]
    total = row.cumsum(0)
    last = torch.where(row > 0, torch.arange(case["V"], device="cuda"), torch.zeros_like(token[:1])).amax()
    res[0:1], res[1] = length.int(), torch.minimum((total <= u[0] * total[-1]).sum(), last).int()
    return res


def run(s):
    op, case = s["op"], s["case"]
    if not own:
        return {"select": _plain_select, "attend": _plain_attend, "accept": _plain_accept}[op](s)
    from paper_2505_23219_amd import binding as B
    if op == "accept":
        return B.ghd_accept_sampled(s["logits"], s["tokens"], s["parent"], s["u"], temperature=case["T"], q_logits=s["q"],
                                    q_row=s["row"], res=s["res"], ws=s["ws"])
    if op == "select":
        B.ghd_block_bounds(s["bounds"], s["k"], *_fresh(case))
        sel = B.ghd_block_select(s["q"], s["bounds"], case["kv"], case["count"], sinks=case["sinks"],
                                 recent=case["recent"], sel=s["sel"], ws=s["ws"])
        hi, lo = B.ghd_block_bounds_read(s["bounds"], *_fresh(case))
        return {"sel": sel, "hi": hi, "lo": lo}
    if case["mask"] == "tree":
        return B.ghd_sparse_attention(s["q"], s["k"], s["v"], s["sel"], case["kv"], parent=s["parent"], ws=s["ws"],
                                      out=s["out"])
    return B.ghd_sparse_attention(s["q"], s["k"], s["v"], s["sel"], case["kv"], mask=s["mask"], ws=s["ws"], out=s["out"])


# ---- what a pass cannot do without ----------------------------------------------------
def work(case):
    op, M = case["op"], case["M"]
    if op == "accept":
        deep = {"chain": M, "random": 6, "wide": 3}[case["tree"]]
        rows = M + {"none": 0, "depths": min(deep, M), "rows": M}[case["q"]]
        return {"bytes": 4 * rows * case["V"] + 16 * M, "flops": 4 * rows * case["V"]}
    nh, nkv, d, n = case["nh"], case["nkv"], case["d"], case["kv"] // BLOCK
    if op == "select":
        fresh = _fresh(case)[1]
        return {"bytes": nkv * n * (2 * d + 4) + 2 * M * nh * d + 8 * nkv * -(-M // 64) * n
                + nkv * fresh * d * (2 * BLOCK + 2 + 8),
                "flops": 4 * M * nh * n * d + 2 * nkv * fresh * BLOCK * d}
    rest = case["kv"] - n * BLOCK + M
    pool = min(case["pool"], n) if M > 1 else min(case["count"], n)
    return {"bytes": 4 * nkv * d * (pool * BLOCK + rest) + 4 * M * nh * d + 8 * nkv * -(-M // 64) * n,
            "flops": 4 * M * nh * d * (min(case["count"], n) * BLOCK + rest)}


# ---- the same in 64 bits ----------------------------------------------------------------
def _power_below(a):
    """2^(floor(log2 a) - 6) of a positive number held exactly."""
    e = torch.floor(torch.log2(a))
    e = torch.where(torch.exp2(e) > a, e - 1, torch.where(torch.exp2(e + 1) <= a, e + 1, e))
    return torch.exp2(e - 6)


def _exact_select(case, seed):
    M, nh, nkv, n = case["M"], case["nh"], case["nkv"], case["kv"] // BLOCK
    k, q = _keys(case, seed), _queries(case, seed).double()
    picked = torch.zeros((nkv, M, n), dtype=torch.bool, device="cuda")
    first, fresh = _fresh(case)
    hi, lo = [], []
    for h in range(nkv):
        x = torch.stack(k[h, :n * BLOCK].double().split(BLOCK))         # [n, 64, d]
        top, low = x.max(1).values, x.min(1).values
        s = _power_below(torch.stack([top.abs(), low.abs()]).amax((0, 2)))[:, None]
        top, low = (top / s).ceil().clamp(-127, 127), (low / s).floor().clamp(-127, 127)
        hi.append((top * s)[first:first + fresh])
        lo.append((low * s)[first:first + fresh])
        best = None
        for g in range(h * nh // nkv, (h + 1) * nh // nkv):
            sq = _power_below(q[:, g].abs().amax(1))[:, None]
            c = (q[:, g] / sq).round().clamp(-127, 127)
            v = sq * (torch.where(c > 0, c, 0.0) @ (top * s).t() + torch.where(c < 0, c, 0.0) @ (low * s).t())
            best = v if best is None else torch.maximum(best, v)
        for m, row in enumerate(best.tolist()):
            must = [b for b in range(n) if b < case["sinks"] or b >= n - case["recent"]]
            rest = sorted((b for b in range(n) if case["sinks"] <= b < n - case["recent"]), key=lambda b: (-row[b], b))
            picked[h, m, (must + rest[:max(0, min(case["count"], n) - len(must))])] = True
    words = []
    for w in range(0, M, 64):
        x = torch.zeros((nkv, n), dtype=torch.int64, device="cuda")
        for m in range(w, min(M, w + 64)):
            x |= picked[:, m].long() << (m - w)
        words.append(x)
    return {"sel": torch.stack(words, dim=1), "hi": torch.stack(hi), "lo": torch.stack(lo)}


def _exact_attend(case, seed):
    M, nh, nkv, d, kv = (case[x] for x in ("M", "nh", "nkv", "d", "kv"))
    q, k, v = _queries(case, seed), _keys(case, seed), _values(case, seed)
    n = kv // BLOCK
    chosen = _chosen(case, seed)
    hide = torch.tensor([[not (s >> j) & 1 for j in range(M)] for s in _see_lists(case, seed)], device="cuda")
    out = torch.zeros((M, nh, d), dtype=torch.float64, device="cuda")
    for h in range(nh):
        g = h // (nh // nkv)
        some = chosen[g].any(0).repeat_interleave(BLOCK)        # keys that any token reads
        at = torch.cat([some.nonzero()[:, 0], torch.arange(n * BLOCK, kv + M, device="cuda")])
        block = torch.div(at, BLOCK, rounding_mode="floor")
        score = q[:, h].double() @ k[g, at].double().t() / math.sqrt(d)
        inside = at < n * BLOCK
        if n:
            score.masked_fill_(inside & ~chosen[g][:, block.clamp(max=n - 1)], -math.inf)
        score[:, score.shape[1] - M:].masked_fill_(hide, -math.inf)
        out[:, h] = torch.nan_to_num(torch.softmax(score, dim=1), nan=0.0) @ v[g][:, at].double().t()
    return out


def _exact_accept(case, seed):
    logits, tokens, _, kids, u, q_logits, row = _accept_inputs(case, seed)
    tokens, u = tokens.tolist(), u.double().tolist()
    node, path = 0, [0]
    while True:
        p = torch.softmax(logits[node].double().cpu() / case["T"], 0)
        q = None
        if q_logits is not None:
            q = torch.softmax(q_logits[node if row is None else row[node]].double().cpu() / case["T"], 0)
        for c in kids[node]:
            x = tokens[c]
            if q is None:
                if u[c] * p.sum().item() < p[x].item():
                    break
                p[x] = 0
            else:
                if u[c] * q[x].item() < p[x].item():
                    break
                r = torch.relu(p - q)
                if r.sum() > 0:
                    p = r / r.sum()
                q[x] = 0
                q = q / q.sum() if q.sum() > 0 else q
        else:
            break
        node = c
        path.append(c)
    run_sum = p.cumsum(0)
    later = (run_sum > u[0] * run_sum[-1]).nonzero()
    token = int(later[0]) if len(later) else int(p.nonzero()[-1])
    return _int32([len(path), token] + path + [0] * (case["M"] - len(path)))


def exact(case, seed):
    return {"select": _exact_select, "attend": _exact_attend, "accept": _exact_accept}[case["op"]](case, seed)
