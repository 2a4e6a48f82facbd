"""The 4-bit operators of the verification step, as cases that can be timed and checked.

A verification step streams its weights and its cache once; held in 4 bits both are about
a quarter of their fp16 size.  Four operators make such a step: a linear layer over 4-bit
weights with group scales, the append of a step's keys and values (rotated on the way) to
a 4-bit cache, the attention of the drafted tokens over that cache, and the commit of an
accepted path inside it.  Rows are read back as fp16 by a fifth call, which the cases of
append and commit use to return the cache rows that they change.

Formats:
  weights  codes[n, k] in 0..15 with a scale (fp16) and a whole zero point 0..15 (8 where
           none is given) for every `group` columns of a row:
           W[n, k] = (codes[n, k] - zero[n, k / group]) * scale[n, k / group]
  cache    a row of a head is cut into groups of 32 channels; a group x (fp16) is held as
           lo = min x, s = fp16((max x - lo) / 15) and codes rint((x - lo) / s) in 0..15;
           it stands for fp16(lo + code * s)
"""
import hashlib
import math

import torch

own = False         # False: elementary torch operations; True: the calls of paper_2505_23219_amd

ROPE_BASE = 10000.0
GROUP = 32          # channels that share a scale in the cache


def listed():
    return [
        # One token through the widest matrix of a 7B-shaped layer (gate and up): decoding.
        {"name": "linear_decode_gate_up", "op": "linear", "M": 1, "N": 22016, "K": 4096, "group": 128, "zeros": True,
         "out16": True, "pad": 0},
        # A small layer whose sizes divide by nothing, rows of x in a wider buffer: latency.
        {"name": "linear_small_ragged", "op": "linear", "M": 5, "N": 1003, "K": 1288, "group": 32, "zeros": False,
         "out16": False, "pad": 8},
        # A 64-node tree through the down projection of a 7B-shaped layer: few, long rows.
        {"name": "linear_tree64_down", "op": "linear", "M": 64, "N": 4096, "K": 11008, "group": 64, "zeros": True,
         "out16": False, "pad": 0},
        # The LM head of a 13B-shaped model over the widest tree.
        {"name": "linear_chain128_head", "op": "linear", "M": 128, "N": 32000, "K": 5120, "group": 128,
         "zeros": False, "out16": False, "pad": 0},
        # One token over a long context, four query heads to a key head: long-context decoding.
        {"name": "attention_decode_64k", "op": "attention", "M": 1, "nh": 32, "nkv": 8, "d": 128, "kv": 65536,
         "mask": "tree", "tree": "chain"},
        # The benchmark's attention: a 64-node tree over 2048 cached tokens, 32 heads.
        {"name": "attention_tree64_7b", "op": "attention", "M": 64, "nh": 32, "nkv": 32, "d": 128, "kv": 2048,
         "mask": "tree", "tree": "random"},
        # Draft sequences side by side, a short odd context, five query heads to a key head.
        {"name": "attention_small_ragged", "op": "attention", "M": 37, "nh": 20, "nkv": 4, "d": 64, "kv": 777,
         "mask": "sequences", "tree": "random"},
        # The widest tree over the 13B-shaped workload's cache.
        {"name": "attention_chain128_13b", "op": "attention", "M": 128, "nh": 40, "nkv": 40, "d": 128, "kv": 8192,
         "mask": "tree", "tree": "chain"},
        # A 64-node tree's rows join a 7B-shaped layer's cache at an odd row.
        {"name": "append_tree64_7b", "op": "append", "M": 64, "nh": 32, "nkv": 32, "d": 128, "kv": 2053,
         "tree": "random"},
        # A prompt's rows are written to an empty cache.
        {"name": "append_prompt_4096", "op": "append", "M": 4096, "nh": 32, "nkv": 8, "d": 128, "kv": 0,
         "tree": "prompt"},
        # Three accepted tokens of an 8-node tree in a small one-layer model.
        {"name": "commit_tiny", "op": "commit", "L": 1, "M": 8, "nkv": 4, "d": 64, "kv": 128, "len": 3},
        # Four accepted tokens of a 64-node tree in all layers of a 7B-shaped model.
        {"name": "commit_tree64_7b", "op": "commit", "L": 32, "M": 64, "nkv": 32, "d": 128, "kv": 2051, "len": 4},
    ]


def _log(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v // step * step if step > 1 else v))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "attention", "attention", "attention", "append", "commit"])
    M = _log(rng, 1, 128)
    if op == "linear":
        N, K = _log(rng, 64, 32000), _log(rng, 256, 13824, 8)
        while N * K > 32000 * 5120:
            N = N * 3 // 4
        return {"op": op, "M": M, "N": N, "K": K, "group": rng.choice([32, 64, 128]), "zeros": rng.random() < 0.5,
                "out16": rng.random() < 0.5, "pad": 8 * rng.randint(0, 4)}
    d = rng.choice([64, 128, 128])
    if op == "attention":
        nkv, rep = _log(rng, 1, 40), rng.choice([1, 1, 2, 4, 5, 8])
        nkv = max(1, min(nkv, 128 // rep))
        kv = _log(rng, 1, 65536) - 1
        while (kv + M) * nkv * d > 65537 * 8 * 128 or (kv + M) * nkv * rep * M * d > 8320 * 40 * 128 * 128:
            kv = kv * 3 // 4
        return {"op": op, "M": M, "nh": nkv * rep, "nkv": nkv, "d": d, "kv": kv,
                "mask": rng.choice(["tree", "tree", "sequences", "sparse"]),
                "tree": rng.choice(["chain", "random", "wide"])}
    if op == "append":
        nkv, rep = _log(rng, 1, 32), rng.choice([1, 2, 4])
        if rng.random() < 0.5:
            M = _log(rng, 1, 4096)
            while M * nkv * (rep + 2) * d > 4096 * 8 * 6 * 128:
                M = M * 3 // 4
            return {"op": op, "M": M, "nh": nkv * rep, "nkv": nkv, "d": d, "kv": _log(rng, 1, 8192) - 1,
                    "tree": "prompt"}
        return {"op": op, "M": M, "nh": nkv * rep, "nkv": nkv, "d": d, "kv": _log(rng, 1, 8192) - 1,
                "tree": rng.choice(["chain", "random", "wide"])}
    nkv, L = _log(rng, 1, 32), rng.randint(1, 32)
    M = min(M, 64)
    return {"op": "commit", "L": L, "M": M, "nkv": nkv, "d": d, "kv": _log(rng, 1, 2048) - 1,
            "len": rng.randint(1, max(1, min(8, (M + 1) // 2)))}


# ---- inputs -------------------------------------------------------------------------
def _gen(seed, *tags):
    g = torch.Generator(device="cuda")
    g.manual_seed(int.from_bytes(hashlib.sha256(repr((int(seed),) + tags).encode()).digest()[:7], "little"))
    return g


def _normal(shape, seed, *tags):
    return torch.randn(shape, generator=_gen(seed, *tags), device="cuda", dtype=torch.float32)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _parent(case, seed):
    """parent[] of the draft tree: a chain, a random tree of depth at most 5, or a wide
    shallow one (a root, M/2 children, grandchildren)."""
    M, kind = case["M"], case["tree"]
    r = torch.Generator().manual_seed(int(seed) * 7919 + M)
    parent, depth = [-1], [0]
    for i in range(1, M):
        if kind == "chain":
            p = i - 1
        else:
            if kind == "wide":
                ok = [0] if i <= M // 2 else list(range(1, M // 2 + 1))
            else:
                ok = [j for j in range(i) if depth[j] < 5]
            p = ok[int(torch.randint(len(ok), (1,), generator=r))]
        parent.append(p)
        depth.append(depth[p] + 1)
    return parent


def _weights(case, seed):
    """A weight matrix N(0, 0.02) as a quantised checkpoint has it: codes two to a byte (even
    column in the low half), scales and zero points of groups of columns."""
    N, K, g = case["N"], case["K"], case["group"]
    G = -(-K // g)
    W = torch.zeros((N, G * g), device="cuda")
    W[:, :K] = _normal((N, K), seed, "W").mul_(0.02)
    W = W.view(N, G, g)
    if case["zeros"]:
        lo, hi = W.amin(2), W.amax(2)
        scale = ((hi - lo) / 15).half()
        zero = (-lo / scale.float()).round_().clamp_(0, 15)
    else:
        scale = (W.abs().amax(2) / 7).half()
        zero = torch.full_like(scale, 8.0, dtype=torch.float32)
    codes = W.div_(scale.float()[:, :, None]).add_(zero[:, :, None]).round_().clamp_(0, 15).to(torch.uint8)
    codes = codes.view(N, G * g)[:, :K].contiguous()
    codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
    return codes.contiguous(), scale, zero.to(torch.uint8) if case["zeros"] else None


def _x(case, seed):
    wide = _normal((case["M"], case["K"] + case["pad"]), seed, "x").half()
    return wide[:, :case["K"]]


def _rows(shape, seed, *tags):
    """Rows of keys or values [..., heads, d] as models have them: every channel with a mean
    and a spread of its own, some spreads several times the others."""
    n, d = shape[-2:]
    spread = torch.exp(0.5 * _normal((n, d), seed, *tags, "spread"))
    mean = 0.5 * _normal((n, d), seed, *tags, "mean")
    return _normal(shape, seed, *tags, "x").mul_(spread).add_(mean).half()


def _capacity(case):
    return (case["kv"] + case["M"] + 63) // 64 * 64


def _see_lists(case, seed):
    """Per drafted token the drafted tokens that it sees, as Python ints of bits."""
    M = case["M"]
    if case["mask"] == "tree":
        parent, see = _parent(case, seed), [0] * M
        for i in range(M):
            see[i] = (1 << i) | (see[parent[i]] if i else 0)
        return see
    if case["mask"] == "sequences":     # draft sequences of 8 tokens side by side
        return [sum(1 << j for j in range(i // 8 * 8, i + 1)) for i in range(M)]
    # any relation: about a third of the pairs, every fifth token sees no drafted token at all
    # (with nothing committed its row is empty)
    bits = torch.rand((M, M), generator=torch.Generator().manual_seed(int(seed) + 17)) < 0.33
    bits[::5] = False
    return [sum(1 << j for j, b in enumerate(row) if b) for row in bits.tolist()]


def _mask_words(see):
    def word(x):
        x &= (1 << 64) - 1
        return x - (1 << 64) if x >> 63 else x
    return torch.tensor([[word(s), word(s >> 64)] for s in see], dtype=torch.int64, device="cuda")


def _attention_inputs(case, seed):
    M, nh, nkv, d, T = case["M"], case["nh"], case["nkv"], case["d"], case["kv"] + case["M"]
    return (_normal((M, nh, d), seed, "q").half(), _rows((T, nkv, d), seed, "k"), _rows((T, nkv, d), seed, "v"))


def _qkv(case, seed):
    """q, k and v side by side in a row, as a fused linear layer leaves them."""
    M, nh, nkv, d = case["M"], case["nh"], case["nkv"], case["d"]
    q = _normal((M, nh, d), seed, "q").half()
    return torch.cat([q, _rows((M, nkv, d), seed, "k"), _rows((M, nkv, d), seed, "v")], dim=1).reshape(M, -1)


def _split(case, qkv):
    M, nh, nkv, d = case["M"], case["nh"], case["nkv"], case["d"]
    return (qkv[:, :nh * d].view(M, nh, d), qkv[:, nh * d:(nh + nkv) * d].view(M, nkv, d),
            qkv[:, (nh + nkv) * d:].view(M, nkv, d))


def _commit_inputs(case, seed):
    """Drafted rows (and the up to 64 committed ones before them) of every layer, and an
    accepted path whose nodes lie behind the rows that it moves to, as in a tree with several
    candidates a level; a second commit then leaves the cache as the first did."""
    L, M, nkv, d, n = case["L"], case["M"], case["nkv"], case["d"], case["len"]
    row0 = max(0, case["kv"] - 64) // 32 * 32
    T = case["kv"] + M - row0
    r = torch.Generator().manual_seed(int(seed) + 5)
    path = [0] + sorted((torch.randperm(M - n, generator=r)[:n - 1] + n).tolist())
    k = _rows((L, T, nkv, d), seed, "k")
    v = _rows((L, T, nkv, d), seed, "v")
    return row0, k, v, [n, 1] + path + [0] * (M - n)


def _first_row(case):
    """The rows that append and commit return begin with the group of 32 that the first changed
    row is in: in the cache those lie together, and the call must leave the others alone."""
    return case["kv"] // 32 * 32


class PlainCache:
    """A 4-bit cache as plain tensors: codes a byte each, lo and scale fp16; [L, rows, heads, .]."""

    def __init__(self, L, nkv, d, capacity):
        def one():
            return (torch.zeros((L, capacity, nkv, d), dtype=torch.uint8, device="cuda"),
                    torch.zeros((L, capacity, nkv, d // GROUP), dtype=torch.float16, device="cuda"),
                    torch.zeros((L, capacity, nkv, d // GROUP), dtype=torch.float16, device="cuda"))
        self.k, self.v = one(), one()

    def put(self, layer, row, k, v):
        for held, x in ((self.k, k), (self.v, v)):
            for to, part in zip(held, _quantise(x)):
                to[layer, row:row + x.shape[0]] = part

    def rows(self, layers, lo, hi):
        return tuple(_values(*(t[layers, lo:hi] for t in held)) for held in (self.k, self.v))


def _cache(L, case):
    """The cache that the calls of `own` work on, or its plain counterpart."""
    if own:
        from paper_2505_23219_amd import binding as B
        return B.KvQ4(L, case["nkv"], case["d"], _capacity(case))
    return PlainCache(L, case["nkv"], case["d"], _capacity(case))


def _fill(cache, layer, row, k, v):
    if own:
        from paper_2505_23219_amd import binding as B
        B.ghd_kv_append_q4(cache, layer, k, v, row)
    else:
        cache.put(layer, row, k, v)


def prepare(case, seed):
    """What a program holds before the call: weights laid out, a filled cache, a tree, buffers."""
    op, s = case["op"], {"op": case["op"], "case": case}
    if own:
        from paper_2505_23219_amd import binding as B
    if op == "linear":
        s["x"] = _x(case, seed)
        codes, scale, zero = _weights(case, seed)
        if own:
            s["W"] = B.ghd_pack_weight_q4(codes, scale, zero, case["group"])
            s["y"] = torch.empty((case["M"], case["N"]), dtype=torch.float16 if case["out16"] else torch.float32,
                                 device="cuda")
            s["ws"] = B.workspace(B.ghd_linear_q4_workspace_bytes(case["M"], case["N"], case["K"]))
        else:
            s["W"] = (codes, scale, zero)
    elif op == "attention":
        s["q"], k, v = _attention_inputs(case, seed)
        s["cache"] = _cache(1, case)
        _fill(s["cache"], 0, 0, k, v)
        s["parent"] = _int32(_parent(case, seed)) if case["mask"] == "tree" else None
        s["mask"] = _mask_words(_see_lists(case, seed))
        if own:
            s["out"] = torch.empty_like(s["q"])
            s["ws"] = B.workspace(B.ghd_attention_q4_workspace_bytes(case["M"], case["kv"], case["nh"], case["nkv"],
                                                                     case["d"]))
    elif op == "append":
        s["qkv"] = _qkv(case, seed)
        s["cache"] = _cache(1, case)
        s["parent"] = None if case["tree"] == "prompt" else _int32(_parent(case, seed))
        row0 = _first_row(case)
        if row0 < case["kv"]:           # committed rows that share the first group of 32
            n = case["kv"] - row0
            _fill(s["cache"], 0, row0, _rows((n, case["nkv"], case["d"]), seed, "k0"),
                  _rows((n, case["nkv"], case["d"]), seed, "v0"))
    else:
        row0, k, v, res = _commit_inputs(case, seed)
        s["cache"] = _cache(case["L"], case)
        for layer in range(case["L"]):
            _fill(s["cache"], layer, row0, k[layer], v[layer])
        s["res"] = _int32(res)
    return s


# ---- the operators in plain form ------------------------------------------------------
def _quantise(x):
    """x fp16 [..., d] -> codes uint8 [..., d], lo fp16 and scale fp16 [..., d / 32]."""
    g = x.reshape(x.shape[:-1] + (-1, GROUP)).float()
    lo = g.amin(-1)
    s = ((g.amax(-1) - lo) / 15).half()
    # a scale is rounded down where the largest code would stand for more than fp16 holds
    s = torch.where((lo + 15 * s.float() >= 65520) & torch.isfinite(s), (s.view(torch.int16) - 1).view(torch.float16), s)
    sf = s.float()[..., None]
    code = torch.where(sf > 0, (g - lo[..., None]) / sf, torch.zeros_like(g)).round()
    code = torch.nan_to_num(code, nan=0.0, posinf=0.0, neginf=0.0).clamp(0, 15).to(torch.uint8)
    return code.reshape(x.shape), lo.half(), s


def _values(code, lo, s):
    g = code.reshape(code.shape[:-1] + (-1, GROUP)).float()
    return (lo.float()[..., None] + g * s.float()[..., None]).half().reshape(code.shape)


def _plain_linear(case, x, W):
    codes, scale, zero = W
    N, K, g = case["N"], case["K"], case["group"]
    G = scale.shape[1]
    w = torch.zeros((N, G * g), dtype=torch.float32, device=codes.device)
    w[:, 0:K:2] = (codes & 15).float()
    w[:, 1:K:2] = (codes >> 4).float()
    z = 8.0 if zero is None else zero.float()[:, :, None]
    w = ((w.view(N, G, g) - z) * scale.float()[:, :, None]).view(N, G * g)[:, :K]
    y = x.float() @ w.t()
    return y.half() if case["out16"] else y


def _plain_see(s):
    """[M, M] truth values: the ancestors-or-self of parent[], or the bits of the mask."""
    M = s["case"]["M"]
    if s["parent"] is not None:
        return _ancestors(s["parent"])
    j = torch.arange(M, device="cuda")
    return ((s["mask"][:, j // 64] >> (j % 64)) & 1) > 0


def _ancestors(parent):
    M = parent.numel()
    i = torch.arange(M, device=parent.device)
    a = torch.eye(M, device=parent.device)
    a[i[1:], parent[1:].long()] = 1.0
    for _ in range(7):                  # paths of up to 2, 4, ... 128 edges
        a = (a @ a > 0).float()
    return a > 0


def _plain_attention(s):
    case = s["case"]
    M, nh, nkv, d, kv = (case[n] for n in ("M", "nh", "nkv", "d", "kv"))
    rep = nh // nkv
    see = _plain_see(s)
    k, v = (t.float() for t in s["cache"].rows(0, 0, kv + M))             # [T, nkv, d]
    out = torch.empty((M, nh, d), dtype=torch.float32, device="cuda")
    for h in range(nkv):
        q = s["q"][:, h * rep:(h + 1) * rep].float().reshape(M * rep, d)
        t = (q @ k[:, h].t() * (1.0 / math.sqrt(d))).view(M, rep, kv + M)
        t[:, :, kv:] = torch.where(see[:, None], t[:, :, kv:], torch.full_like(t[:, :, kv:], -math.inf))
        top = t.amax(2, keepdim=True)
        p = torch.exp(t - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = p.sum(2, keepdim=True)
        p = p / torch.where(total > 0, total, torch.ones_like(total))     # a row that sees nothing: zeros
        out[:, h * rep:(h + 1) * rep] = (p.view(M * rep, -1) @ v[:, h]).view(M, rep, d)
    return out.half()


def _rotation(case, parent, M):
    """cos and sin [M, d / 2] of the rotary angles at kv + depth, worked out in 64 bits."""
    d = case["d"]
    depth = torch.arange(M, device="cuda") if parent is None else _ancestors(parent).sum(1) - 1
    j = torch.arange(d // 2, dtype=torch.float64, device="cuda")
    angle = (case["kv"] + depth).double()[:, None] * torch.exp2(-2.0 / d * math.log2(ROPE_BASE) * j)
    return angle.cos(), angle.sin()


def _rotate(x, c, s):
    a, b = x.float().chunk(2, dim=-1)
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1).half()


def _plain_append(s):
    case = s["case"]
    q, k, v = _split(case, s["qkv"])
    c, sn = (t.float()[:, None] for t in _rotation(case, s["parent"], case["M"]))
    s["cache"].put(0, case["kv"], _rotate(k, c, sn), v)
    kr, vr = s["cache"].rows(slice(0, 1), _first_row(case), case["kv"] + case["M"])
    return {"q": _rotate(q, c, sn), "k": kr, "v": vr}


def _plain_commit(s):
    case, n = s["case"], s["case"]["len"]
    src = case["kv"] + s["res"][2:2 + n].long()
    for held in (s["cache"].k, s["cache"].v):
        for t in held:
            t[:, case["kv"]:case["kv"] + n] = t[:, src]
    kr, vr = s["cache"].rows(slice(0, case["L"]), _first_row(case), case["kv"] + case["M"])
    return {"k": kr, "v": vr}


def run(s):
    op, case = s["op"], s["case"]
    if not own:
        if op == "linear":
            return _plain_linear(case, s["x"], s["W"])
        return {"attention": _plain_attention, "append": _plain_append, "commit": _plain_commit}[op](s)
    from paper_2505_23219_amd import binding as B
    M, kv = case["M"], case["kv"] if op != "linear" else 0
    if op == "linear":
        return B.ghd_linear_q4(s["x"], s["W"], case["N"], case["group"], ws=s["ws"], y=s["y"])
    if op == "attention":
        if case["mask"] == "tree":
            return B.ghd_tree_attention_q4(s["q"], s["cache"], 0, s["parent"], kv, ws=s["ws"], out=s["out"])
        return B.ghd_masked_attention_q4(s["q"], s["cache"], 0, s["mask"], kv, ws=s["ws"], out=s["out"])
    row0 = _first_row(case)
    if op == "append":
        q, k, v = _split(case, s["qkv"])
        q = B.ghd_kv_append_q4(s["cache"], 0, k, v, kv, q=q, parent=s["parent"], rope_base=ROPE_BASE)
        kr, vr = B.ghd_kv_read_q4(s["cache"], row0, kv + M - row0)
        return {"q": q, "k": kr, "v": vr}
    B.ghd_commit_path_q4(s["cache"], s["res"], M, kv)
    kr, vr = B.ghd_kv_read_q4(s["cache"], row0, kv + M - row0)
    return {"k": kr, "v": vr}


# ---- what a pass cannot do without ----------------------------------------------------
def _row_bytes(nkv, d):
    """Keys and values of one cached token: 4 bits a channel, lo and scale for every 32."""
    return 2 * nkv * (d // 2 + d // GROUP * 4)


def work(case):
    op, M = case["op"], case["M"]
    if op == "linear":
        N, K, g = case["N"], case["K"], case["group"]
        meta = N * -(-K // g) * (2.5 if case["zeros"] else 2.0)
        return {"bytes": N * K / 2 + meta + 2 * M * K + (2 if case["out16"] else 4) * M * N, "flops": 2 * M * N * K}
    nkv, d, kv = case["nkv"], case["d"], case["kv"]
    row = _row_bytes(nkv, d)
    if op == "attention":
        return {"bytes": (kv + M) * row + 4 * M * case["nh"] * d, "flops": 4 * M * case["nh"] * d * (kv + M)}
    back = kv + M - _first_row(case)        # rows read back: in 4 bits, out fp16
    if op == "append":
        H, Hkv = case["nh"] * d, nkv * d
        return {"bytes": 2 * M * (2 * H + 2 * Hkv) + M * row + back * (row + 4 * Hkv), "flops": M * (6 * H + 14 * Hkv)}
    return {"bytes": case["L"] * (2 * (case["len"] - 1) * row + back * (row + 4 * nkv * d)),
            "flops": 4 * case["L"] * back * nkv * d}


# ---- the same in 64 bits ----------------------------------------------------------------
def _held(x):
    """What a 4-bit cache stands for after taking x (fp16 [..., d]), in 64 bits: lo and scale are
    the fp16 numbers that are stored, the value is rounded to fp16 once."""
    g = x.double().unflatten(-1, (x.shape[-1] // GROUP, GROUP))
    lo, hi = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values
    s = ((hi - lo).float() / 15.0).half().double()
    code = torch.round((g - lo) / torch.where(s > 0, s, torch.ones_like(s))).clamp(0, 15)
    return (lo + code * s).half().double().flatten(-2)


def _exact_turn(case, x, depth):
    d = case["d"]
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    j = torch.arange(d // 2, dtype=torch.float64, device=x.device)
    phase = (case["kv"] + depth.double())[:, None, None] * ROPE_BASE ** (-j / (d // 2))
    z = torch.polar(torch.ones_like(phase), phase) * torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double())
    out[..., :d // 2], out[..., d // 2:] = z.real, z.imag
    return out


def exact(case, seed):
    op, M = case["op"], case["M"]
    if op == "linear":
        codes, scale, zero = _weights(case, seed)
        x = _x(case, seed).double()
        K, g = case["K"], case["group"]
        y = torch.zeros((M, case["N"]), dtype=torch.float64, device="cuda")
        for i in range(scale.shape[1]):         # group by group: scale * (x . codes - zero * sum x)
            c = codes[:, i * g // 2:min((i + 1) * g, K) // 2]
            xs = x[:, i * g:min((i + 1) * g, K)]
            t = xs[:, 0::2] @ (c & 15).double().t() + xs[:, 1::2] @ (c >> 4).double().t()
            z = torch.full_like(scale[:, i], 8).double() if zero is None else zero[:, i].double()
            y += scale[:, i].double() * (t - z * xs.sum(1, keepdim=True))
        return y
    if op == "attention":
        nh, nkv, d, kv = case["nh"], case["nkv"], case["d"], case["kv"]
        q, k, v = _attention_inputs(case, seed)
        hide = torch.tensor([[not (s >> j) & 1 for j in range(M)] for s in _see_lists(case, seed)], device="cuda")
        out = torch.zeros((M, nh, d), dtype=torch.float64, device="cuda")
        for h in range(nh):
            kh, vh = (_held(t[:, h // (nh // nkv)]) for t in (k, v))
            score = q[:, h].double() @ kh.t() / math.sqrt(d)
            score[:, kv:].masked_fill_(hide, -math.inf)
            out[:, h] = torch.nan_to_num(torch.softmax(score, dim=1), nan=0.0) @ vh
        return out
    row0 = _first_row(case)
    if op == "append":
        q, k, v = _split(case, _qkv(case, seed))
        if case["tree"] == "prompt":
            depth = torch.arange(M, device="cuda")
        else:
            depth, parent = [0] * M, _parent(case, seed)
            for i in range(1, M):
                depth[i] = depth[parent[i]] + 1
            depth = torch.tensor(depth, device="cuda")
        n = case["kv"] - row0
        before = [_rows((n, case["nkv"], case["d"]), seed, t) for t in ("k0", "v0")]
        rows = [torch.cat([b, x])[None] for b, x in zip(before, (_exact_turn(case, k, depth).half(), v))]
        return {"q": _exact_turn(case, q, depth), "k": _held(rows[0]), "v": _held(rows[1])}
    first, k, v, res = _commit_inputs(case, seed)
    n, kv = case["len"], case["kv"]
    out = {}
    for name, x in (("k", k), ("v", v)):
        to = x.clone()
        for j, node in enumerate(res[2:2 + n]):
            to[:, kv + j - first] = x[:, kv + node - first]
        out[name] = _held(to[:, row0 - first:])
    return out
