"""The sparse attention's operators and sampled acceptance in plain 64-bit arithmetic on the CPU."""
import math

import torch

BLOCK = 64


def unit_below(a):
    """2^(floor(log2 a) - 6); 0 of 0."""
    return 2.0 ** (math.frexp(a)[1] - 7) if a > 0 else 0.0


def bounds(k, n):
    """k [nkv, rows, d]: (HI, LO [nkv, n, d], unit [nkv, n]) of the first n blocks."""
    nkv, _, d = k.shape
    hi, lo, unit = torch.zeros(nkv, n, d).double(), torch.zeros(nkv, n, d).double(), torch.zeros(nkv, n).double()
    for h in range(nkv):
        for b in range(n):
            x = k[h, b * BLOCK:(b + 1) * BLOCK].double()
            if not torch.isfinite(x).all():
                unit[h, b] = math.inf
                continue
            s = unit_below(x.abs().max().item())
            unit[h, b] = s
            if s:
                hi[h, b] = torch.clamp(torch.ceil(x.max(0).values / s), -127, 127)
                lo[h, b] = torch.clamp(torch.floor(x.min(0).values / s), -127, 127)
    return hi, lo, unit


def read(b):
    hi, lo, unit = b
    u = unit[..., None].expand_as(hi)
    finite = torch.isfinite(u)
    w = torch.where(finite, u, torch.zeros_like(u))
    return torch.where(finite, hi * w, math.inf), torch.where(finite, lo * w, -math.inf)


def scores(q, b):
    """[nkv, M, n], exact."""
    hi, lo, unit = b
    M, nh, d = q.shape
    nkv, n = unit.shape
    out = torch.full((nkv, M, n), -math.inf).double()
    for i in range(M):
        for g in range(nh):
            x, h = q[i, g].double(), g // (nh // nkv)
            s = unit_below(x.abs().max().item()) if torch.isfinite(x).all() else 0.0
            c = torch.clamp(torch.round(x / s), -127, 127) if s else torch.zeros(d).double()
            t = (hi[h] @ c.clamp(min=0) + lo[h] @ c.clamp(max=0)) * s
            out[h, i] = torch.maximum(out[h, i], t)
    finite = torch.isfinite(unit)[:, None]
    return torch.where(finite, out * torch.where(torch.isfinite(unit), unit, torch.zeros_like(unit))[:, None], math.inf)


def select(score, count, sinks, recent):
    """Truth values [nkv, M, n]."""
    nkv, M, n = score.shape
    sel = torch.zeros((nkv, M, n), dtype=torch.bool)
    must = [b for b in range(n) if b < sinks or b >= n - recent]
    other = [b for b in range(n) if not (b < sinks or b >= n - recent)]
    for h in range(nkv):
        for i in range(M):
            row = score[h, i].tolist()
            best = sorted(other, key=lambda b: (-row[b], b))
            sel[h, i, must + best[:max(0, min(count, n) - len(must))]] = True
    return sel


def words(sel):
    nkv, M, n = sel.shape
    out = torch.zeros((nkv, -(-M // 64), n), dtype=torch.int64)
    for i in range(M):
        out[:, i // 64] |= sel[:, i].long() << (i % 64)
    return out


def ancestors(parent):
    see = []
    for i, p in enumerate(parent):
        see.append({i} | (see[p] if 0 <= p < i else set()))
    M = len(see)
    return torch.tensor([[j in s for j in range(M)] for s in see])


def mask_words(see):
    M = see.shape[0]
    out = torch.zeros((M, 2), dtype=torch.int64)
    for j in range(M):
        out[:, j // 64] |= see[:, j].long() << (j % 64)
    return out


def attend(q, k, v, sel, see, kv_len, scale):
    """q [M, nh, d], k [nkv, rows, d], v [nkv, d, rows]: (outputs, what their rounding is relative to: sums of p |v|)."""
    M, nh, d = q.shape
    nkv, n, total = k.shape[0], kv_len // BLOCK, kv_len + M
    out, size = torch.zeros(M, nh, d).double(), torch.zeros(M, nh, d).double()
    for g in range(nh):
        h = g // (nh // nkv)
        seen = torch.ones((M, total), dtype=torch.bool)
        seen[:, :n * BLOCK] = sel[h].repeat_interleave(BLOCK, dim=1)
        seen[:, kv_len:] = see
        kh, vh = k[h, :total].double(), v[h, :, :total].double().t()
        for i in range(M):
            at = seen[i].nonzero()[:, 0]
            if len(at) == 0:
                continue
            p = torch.softmax(kh[at] @ q[i, g].double() * scale, 0)
            out[i, g] = p @ vh[at]
            size[i, g] = p @ vh[at].abs()
    return out, size


def accept(logits, tokens, parent, u, T, q_logits=None, q_row=None, q_T=None):
    """[length, next token] + path; probabilities are kept as 64-bit softmax values, one rejection after another."""
    def softmax(x, T):
        x = torch.where(torch.isnan(x), -math.inf, x.double())
        top = x.max().item()
        if top == -math.inf:
            return torch.zeros_like(x)
        w = (x == math.inf).double() if top == math.inf else torch.exp((x - top) / T)
        return w / w.sum()
    M, V = logits.shape
    node, path = 0, [0]
    while True:
        p, q = softmax(logits[node], T), None
        if q_logits is not None:
            r = node if q_row is None else min(max(int(q_row[node]), 0), q_logits.shape[0] - 1)
            q = softmax(q_logits[r], T if q_T is None else q_T)
        for c in [c for c in range(node + 1, M) if parent[c] == node]:
            x, uc = int(tokens[c]), float(u[c])
            if not 0 <= x < V:
                continue
            if q is None:
                if uc * p.sum() < p[x]:
                    break
                p[x] = 0
                continue
            if uc * q[x] < p[x]:
                break
            rest = torch.clamp(p - q, min=0)
            if rest.sum() > 0:
                p = rest / rest.sum()
            q[x] = 0
            if q.sum() > 0:
                q = q / q.sum()
        else:
            break
        node = c
        path.append(c)
    total = p.cumsum(0)
    over = (total > float(u[0]) * total[-1]).nonzero()[:, 0]
    some = p.nonzero()[:, 0]
    token = int(over[0]) if len(over) else int(some[-1]) if len(some) else -1
    return [len(path), token] + path
