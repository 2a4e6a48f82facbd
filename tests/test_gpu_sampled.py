"""Sampled acceptance against a plain 64-bit form: whole numbers, equal."""
import math

import pytest
import torch

import sparse_plain as P
from paper_2505_23219_amd import binding as B, workloads as wl

pytestmark = pytest.mark.gpu


def _tree(kind, M, seed):
    if kind == "chain":
        return wl.tree_chain(M).tolist()
    if kind == "star":
        return wl.tree_star(M).tolist()
    return wl.tree_random(M, 5, seed).tolist()


def _case(M, V, kind, draft, seed, T=1.0, near=0.7):
    """Logits, tokens, parent, u and draft logits on the CPU; tokens as a drafter picks them."""
    g = torch.Generator().manual_seed(seed)
    parent = _tree(kind, M, seed)
    logits = 1.5 * torch.randn(M, V, generator=g)
    logits.scatter_add_(1, torch.randint(V, (M, 4), generator=g), 6 * torch.rand(M, 4, generator=g))
    q, row = None, None
    if draft == "rows":
        q = logits + near * torch.randn(M, V, generator=g)
    elif draft == "depths":
        depth = [0] * M
        for i in range(1, M):
            depth[i] = depth[parent[i]] + 1
        q, row = logits[:max(depth) + 1] + near * torch.randn(max(depth) + 1, V, generator=g), depth
    tokens = torch.zeros(M, dtype=torch.int32)
    for p in range(M):
        kids = [c for c in range(M) if parent[c] == p]
        if not kids:
            continue
        if q is None:
            best = (logits[p] + near * torch.randn(V, generator=g)).argsort(descending=True)
        else:
            of = q[p] if row is None else q[row[p]]
            best = (of / T - torch.log(-torch.log(torch.rand(V, generator=g).clamp(1e-9, 1 - 1e-7)))).argsort(descending=True)
        for r, c in enumerate(kids):
            tokens[c] = best[r % V]
    return logits, tokens, parent, torch.rand(M, generator=g), q, row


def _gpu(case, T=1.0, q_T=None, **kw):
    logits, tokens, parent, u, q, row = case
    M = len(parent)
    res = torch.full((2 + M,), -7, dtype=torch.int32, device="cuda")
    got = B.ghd_accept_sampled(logits.cuda(), tokens.cuda(), torch.tensor(parent, dtype=torch.int32, device="cuda"), u.cuda(), temperature=T,
                               q_logits=None if q is None else q.cuda(),
                               q_row=None if row is None else torch.tensor(row, dtype=torch.int32, device="cuda"), q_temperature=q_T,
                               res=res, **kw)
    assert got is res
    return res.tolist()


def _check(case, T=1.0, q_T=None, **kw):
    logits, tokens, parent, u, q, row = case
    want = P.accept(logits, tokens, parent, u, T, q, row, q_T)
    got = _gpu(case, T, q_T, **kw)
    assert got[:len(want)] == want, (got, want)
    assert all(x == -7 for x in got[len(want):])
    return want


@pytest.mark.parametrize("draft", ["none", "rows", "depths"])
@pytest.mark.parametrize("M,V,kind", [(1, 1, "chain"), (1, 7, "chain"), (2, 2, "chain"), (5, 3, "star"), (8, 1000, "random"),
                                      (16, 4095, "star"), (33, 4097, "random"), (64, 32000, "random"), (128, 2000, "chain"),
                                      (128, 999, "star"), (3, 131072, "random"), (2, 262144, "star")])
def test_accept(M, V, kind, draft):
    lengths = []
    for seed in range(12 if M * V <= 1 << 17 else 2):
        T = (1.0, 0.6, 1.4)[seed % 3]
        lengths.append(_check(_case(M, V, kind, draft, seed, T), T)[0])
    assert max(lengths) > 1 or M == 1 or len(lengths) < 12


@pytest.mark.parametrize("draft", ["none", "rows"])
def test_all_rejected_and_all_accepted(draft):
    case = _case(40, 500, "random", draft, 3)
    for u0 in (0.0, 0.25, 0.999999):
        for value in (0.0, 0.99999994):
            case[3][:] = value
            case[3][0] = u0
            want = _check(case)
            assert value > 0 or want[0] > 1
    case = _case(9, 500, "star", draft, 3)
    case[3][:] = 0.99999994
    _check(case)


@pytest.mark.parametrize("draft", ["none", "rows"])
def test_tokens_twice_and_outside(draft):
    for seed in range(20):
        case = _case(12, 30, "star", draft, seed)
        case[1][3], case[1][5], case[1][6], case[1][8] = case[1][1], case[1][1], -1, 30
        case[3][1:] = 0.9 + 0.1 * case[3][1:]
        _check(case)


@pytest.mark.parametrize("draft", ["none", "rows"])
def test_masked_and_odd_logits(draft):
    for seed in range(10):
        case = _case(6, 5000, "random", draft, seed)
        logits, q = case[0], case[4]
        logits[:, 100:4900] = -math.inf
        logits[0, 7], logits[1, 8], logits[2, 9] = math.nan, -math.inf, -3e38
        _check(case)
        logits[3], logits[4] = -math.inf, math.nan
        logits[0, 20], logits[0, 30] = math.inf, math.inf
        _check(case)
        if q is not None:
            q[:, 50:] = -math.inf
            q[1, 3] = math.nan
            q[2] = -math.inf
            q[0, 5] = math.inf
            _check(case)
    logits[:] = -math.inf
    assert _check(case)[1] == -1


def test_sharp_and_flat():
    for T in (1e-3, 0.05, 20.0, 1e30):
        for draft in ("none", "rows"):
            for seed in range(4):
                _check(_case(8, 3000, "random", draft, seed, T), T)
    for seed in range(4):
        _check(_case(8, 3000, "random", "rows", seed, 0.7), 0.7, q_T=1.3)


@pytest.mark.parametrize("T", [1e-10, 1e-15, 1e-20, 1e-38])
def test_next_to_no_temperature(T):
    """The likeliest token has all of the probability, at whatever height its logit is."""
    for draft in ("none", "rows"):
        for V in (300, 40000):
            case = _case(12, V, "random", draft, 3)
            case[0].add_(1000.0)
            want = _check(case, T)
            got = want[2:]
            assert want[1] == int(case[0][got[-1]].argmax())


def test_drafts_far_from_and_equal_to_the_target():
    for seed in range(8):
        case = _case(30, 700, "random", "rows", seed, near=8.0)
        _check(case)
        _check((case[0], case[1], case[2], case[3], case[0].clone(), None))


def test_little_left():
    """All but 1e-9 and 1e-30 of the draft's probability is its first children's."""
    for gap in (20.0, 70.0, 300.0):
        case = _case(6, 50, "star", "rows", 1)
        logits, tokens, parent, u, q, row = case
        q[0] = -torch.arange(50.0) * 0.01 - 2 * gap
        q[0, 7], q[0, 9] = 0.0, -gap
        tokens[1:] = torch.tensor([7, 9, 3, 4, 5])
        logits[0, 7] = logits[0, 9] = -50.0
        for u1 in (0.1, 0.5, 0.9):
            u[1:] = u1
            _check(case)
        case[0][0] = q[0].flip(0)
        _check((case[0], tokens, parent, u, None, None))


@pytest.mark.parametrize("V", [5, 4096, 4097, 8193, 32768, 33000, 70001, 262144])
@pytest.mark.parametrize("children", [2, 3, 19])
def test_many_rejections(V, children):
    """A root whose children are all rejected, their tokens once and twice and outside of the vocabulary; any workspace.

    The token follows from sums of p - b q of tokens not rejected.  A weight is off by 2^-24 of itself, b and the difference as much again, and
    up to eight of them are added up in 32 bits (three roundings each, at most): the running sum by less than 12 2^-24 of the
    running sum of p + b q."""
    children = min(children, V - 2)
    M, g = children + 1, torch.Generator().manual_seed(V + children)
    for turn in range(3):
        logits, q = 1.5 * torch.randn(M, V, generator=g), torch.randn(M, V, generator=g)
        tokens = torch.zeros(M, dtype=torch.int32)
        tokens[1:] = torch.randperm(V, generator=g)[:children].int()
        if V > 4096:                             # one in the last segment, in the first, at both ends
            tokens[1], tokens[2] = V - 1, 0
        if turn == 1 and children > 4:
            tokens[3], tokens[4] = tokens[1], V
        u = torch.full((M,), 0.99)
        u[0] = (0.11, 0.77, 0.0)[turn]
        at = tokens[1:].long().clamp(max=V - 1)
        logits[0, at], q[0, at] = -30.0, q[0, at] + 4.0
        p, qp = torch.softmax(logits[0].double(), 0), torch.softmax(q[0].double(), 0)
        size, beta, alpha, gone = p.clone(), 0.0, 1.0, torch.zeros(V, dtype=torch.bool)
        left, rest = p.clone(), 1.0
        for x in tokens[1:].tolist():
            if x >= V:
                continue
            beta += 1.0 / (alpha * rest)
            gone[x] = True
            left, size = (p - beta * qp).clamp(min=0).masked_fill(gone, 0), (p + beta * qp).masked_fill(gone, 0)
            alpha, rest = 1.0 / left.sum().item(), qp.masked_fill(gone, 0).sum().item()
        ws = torch.full((B.ghd_accept_sampled_workspace_bytes(M, V),), 255, dtype=torch.uint8, device="cuda")
        got = _gpu((logits, tokens, [-1] + [0] * children, u, q, None), ws=ws)
        assert got[0] == 1 and 0 <= got[1] < V and not gone[got[1]]
        upto, off = left.cumsum(0), 12 * 2.0 ** -24 * size.cumsum(0)
        goal, t = u[0].double() * left.sum(), got[1]
        assert upto[t] + off[-1] >= goal and upto[t] - left[t] - off[-1] <= goal and left[t] > -off[-1], (t, goal, upto[t], left[t])


def test_rows_of_drafts_are_clamped_and_a_parent_is_an_earlier_node():
    case = _case(10, 200, "random", "depths", 4)
    row = [r + 100 if i % 2 else r - 100 for i, r in enumerate(case[5])]
    _check(case[:5] + (row,))
    logits, tokens, parent, u, q, row = _case(8, 100, "random", "none", 2)
    odd = list(parent)
    odd[3], odd[5] = 3, 7
    got = _gpu((logits, tokens, odd, u, q, row))
    odd[3] = odd[5] = -1
    want = P.accept(logits, tokens, odd, u, 1.0)
    assert got[:len(want)] == want


def test_rows_behind_one_another_over_any_workspace():
    """Rows that begin at any 4 bytes; a workspace that held anything; nothing before or behind the result."""
    M, V = 9, 1001
    case = _case(M, V, "random", "rows", 5)
    want = _check(case)
    need = B.ghd_accept_sampled_workspace_bytes(M, V)
    room = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
    store = torch.zeros(2 * M * V + 1, device="cuda")
    logits, q = store[1:1 + M * V].view(M, V), store[1 + M * V:].view(M, V)
    logits.copy_(case[0])
    q.copy_(case[4])
    res = torch.full((4 + M,), -7, dtype=torch.int32, device="cuda")
    B.ghd_accept_sampled(logits, case[1].cuda(), torch.tensor(case[2], dtype=torch.int32, device="cuda"), case[3].cuda(), q_logits=q,
                         res=res[1:-1], ws=room[256:256 + need])
    assert res.tolist()[1:1 + len(want)] == want and res[0] == -7 and res[-1] == -7
    assert (room[:256] == 255).all() and (room[256 + need:] == 255).all()


def test_the_result_may_lie_where_the_inputs_are():
    M, V = 20, 300
    case = _case(M, V, "random", "none", 5)
    want = P.accept(case[0], case[1], case[2], case[3], 1.0)
    room = torch.cat([torch.tensor(case[2], dtype=torch.int32), case[1], torch.zeros(2, dtype=torch.int32)]).cuda()
    B.ghd_accept_sampled(case[0].cuda(), room[M:2 * M], room[:M], case[3].cuda(), res=room[M:])
    assert room[M:].tolist()[:len(want)] == want


def test_graphs_and_streams():
    M, V = 32, 3000
    cases = [_case(M, V, "random", "rows", s) for s in range(5)]
    parent = torch.tensor(cases[0][2], dtype=torch.int32, device="cuda")
    logits, tokens, u, q = (cases[0][i].cuda() for i in (0, 1, 3, 4))
    res, ws = torch.zeros(2 + M, dtype=torch.int32, device="cuda"), B.workspace(B.ghd_accept_sampled_workspace_bytes(M, V))
    other = torch.zeros_like(res)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.ghd_accept_sampled(logits, tokens, parent, u, q_logits=q, res=res, ws=ws)
    torch.cuda.synchronize()
    graphs = []
    for draft in (q, None):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.ghd_accept_sampled(logits, tokens, parent, u, q_logits=draft, res=res if draft is not None else other, ws=ws)
        graphs.append(g)
    for case in cases[1:]:
        for to, i in ((logits, 0), (tokens, 1), (u, 3), (q, 4)):
            to.copy_(case[i])
        parent.copy_(torch.tensor(case[2], dtype=torch.int32))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for to, draft in ((res, case[4]), (other, None)):
            want = P.accept(case[0], case[1], case[2], case[3], 1.0, draft)
            assert to.tolist()[:len(want)] == want


def test_what_follows_is_distributed_as_the_target():
    """u on a grid: how often each token comes next, over drafts drawn from q, is p."""
    V, n = 4, 64
    g = torch.Generator().manual_seed(1)
    logits, q = torch.randn(1, V, generator=g), torch.randn(1, V, generator=g)
    p, qp = torch.softmax(logits[0].double(), 0), torch.softmax(q[0].double(), 0)
    count = torch.zeros(V).double()
    grid = (torch.arange(n) + 0.5) / n
    rows = logits.repeat(2, 1).cuda()
    for x in range(V):
        for u1 in grid.tolist():
            for u0 in grid[::8].tolist():
                res = B.ghd_accept_sampled(rows, torch.tensor([0, x], dtype=torch.int32, device="cuda"),
                                           torch.tensor([-1, 0], dtype=torch.int32, device="cuda"), torch.tensor([u0, u1], device="cuda"),
                                           q_logits=q.cuda().repeat(2, 1)).tolist()
                count[x if res[0] == 2 else res[1]] += qp[x] / (n * n / 8)
    # a grid of n has each acceptance right to 1 / n, one of n / 8 each draw (of what is rejected) to 8 / n
    reject = (qp - torch.minimum(p, qp)).sum()
    assert ((count - p).abs() <= 1.0 / n + 8.0 / n * reject + 1e-9).all(), (count, p)
