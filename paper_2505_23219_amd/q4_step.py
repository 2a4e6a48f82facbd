"""A decoder stack with weights and cache in 4 bits, verified a token tree at a time.

    python -m paper_2505_23219_amd.q4_step [--shape tiny|7b|13b] [--layers L] [--tokens N] [--kv-heads N]

The linear layers, the cache and its attention, acceptance and commit are the library's
(ghd_linear_q4, ghd_kv_append_q4, ghd_tree_attention_q4, ghd_accept_greedy_static,
ghd_commit_path_q4, ghd_embed); the norms, the residual and the SwiGLU between them are torch
elementwise operations in fp32, each rounded once to the fp16 that the next linear layer reads.
Run as a module it decodes from random weights, one token a step and then with drafted trees, and
prints how many steps each took and whether they wrote the same tokens.  (Sums of a tree are taken in
another order than a single token's, so with random weights, whose best two logits are often alike, a
long run may part from the other at such a place.)
"""
from __future__ import annotations

import argparse
import time
from typing import Dict, List, Optional, Sequence, Tuple

import torch

from . import binding as B, workloads as wl


def quantise_weight(w: torch.Tensor, group: int) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """[N, K] -> what ghd_pack_weight_q4 takes: codes uint8 [N, K / 2], scales fp16 and zeros uint8
    [N, ceil(K / group)], with w ~ (code - zero) * scale.

    Each group's range, stretched to hold 0 (the zero is a code of its own, so 0 is exact), is cut in
    15 steps.  The fp16 scale is what the codes are taken with; a group of zeros gets scale 1."""
    N, K = w.shape
    n = -(-K // group)
    w = torch.nn.functional.pad(w.float(), (0, n * group - K)).view(N, n, group)
    lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
    scale = ((hi - lo) / 15).to(torch.float16)
    scale = torch.where(scale > 0, scale, torch.ones_like(scale))
    zero = torch.round(-lo / scale.float()).clamp(0, 15)
    codes = (torch.round(w / scale.float()[..., None]) + zero[..., None]).clamp(0, 15).to(torch.uint8)
    codes = codes.view(N, n * group)[:, :K]
    return (codes[:, 0::2] | codes[:, 1::2] << 4).contiguous(), scale, zero.to(torch.uint8)


class Q4Matrix:
    """A [N, K] matrix in 4 bits on the GPU and its product with up to 128 rows."""

    def __init__(self, w: torch.Tensor, group: int, device="cuda"):
        self.N, self.K, self.group = w.shape[0], w.shape[1], group
        self.packed = B.ghd_pack_weight_q4(*quantise_weight(w.to(device), group), group)

    def __call__(self, x: torch.Tensor, ws: torch.Tensor, out_dtype=torch.float32) -> torch.Tensor:
        return B.ghd_linear_q4(x, self.packed, self.N, self.group, out_dtype, ws=ws)


def grouped_heads(w: torch.Tensor, shape, nkv: int) -> torch.Tensor:
    """The rows of a stacked q, k, v projection with only the first nkv heads of k and v."""
    H, kept = shape.H, nkv * shape.d
    return torch.cat((w[:H], w[H:H + kept], w[2 * H:2 * H + kept]))


class Q4Stack:
    """Layers (workloads.layer_weights' names) and head of `shape` in 4 bits, nkv key/value heads, and
    the cache of `capacity` rows (a multiple of 32) that its steps fill."""

    def __init__(self, shape, nkv: int, layers: Sequence[Dict[str, torch.Tensor]], head: Dict[str, torch.Tensor],
                 capacity: int, group: int = 128, device="cuda"):
        self.shape, self.nkv, self.group = shape, nkv, group
        self.cache = B.KvQ4(len(layers), nkv, shape.d, capacity, device)
        self.layers: List[dict] = []
        for w in layers:
            layer = {g: w[g].to(device).float() for g in ("g_attn", "g_ffn")}
            layer["Wqkv"] = Q4Matrix(grouped_heads(w["Wqkv"], shape, nkv), group, device)
            for m in ("Wo", "Wgu", "Wdown"):
                layer[m] = Q4Matrix(w[m], group, device)
            self.layers.append(layer)
        self.g_final = head["g_final"].to(device).float()
        self.Wlm = Q4Matrix(head["Wlm"], group, device)
        self.ws: Optional[torch.Tensor] = None

    def workspace(self, M: int, kv_len: int) -> torch.Tensor:
        """One workspace that every call of a step shares: they follow one another on one stream."""
        s = self.shape
        need = B.ghd_attention_q4_workspace_bytes(M, kv_len, s.nh, self.nkv, s.d)
        for m in [self.layers[0][n] for n in ("Wqkv", "Wo", "Wgu", "Wdown")] + [self.Wlm]:
            need = max(need, B.ghd_linear_q4_workspace_bytes(M, m.N, m.K))
        if self.ws is None or self.ws.numel() < need:
            self.ws = B.workspace(need, self.g_final.device)
        return self.ws

    def _norm(self, x: torch.Tensor, gain: torch.Tensor) -> torch.Tensor:
        return torch.nn.functional.rms_norm(x, (self.shape.H,), gain, self.shape.rms_eps).half()

    def step(self, x16: torch.Tensor, parent: torch.Tensor, kv_len: int) -> torch.Tensor:
        """Logits fp32 [M, V] of a tree of M <= 128 tokens (embeddings x16 [M, H]) behind kv_len rows;
        the tree's keys and values are left in the rows from kv_len on."""
        s, nkv, M = self.shape, self.nkv, x16.shape[0]
        ws = self.workspace(M, kv_len)
        x = x16.float()
        for i, w in enumerate(self.layers):
            qkv = w["Wqkv"](self._norm(x, w["g_attn"]), ws, torch.float16).view(M, s.nh + 2 * nkv, s.d)
            q, k, v = qkv.split((s.nh, nkv, nkv), dim=1)
            q = B.ghd_kv_append_q4(self.cache, i, k, v, kv_len, q=q, parent=parent, rope_base=s.rope_base)
            a = B.ghd_tree_attention_q4(q, self.cache, i, parent, kv_len, ws=ws)
            x = x + w["Wo"](a.view(M, s.nh * s.d), ws)
            gate, up = w["Wgu"](self._norm(x, w["g_ffn"]), ws).chunk(2, dim=1)
            x = x + w["Wdown"]((torch.nn.functional.silu(gate) * up).half(), ws)
        return self.Wlm(self._norm(x, self.g_final), ws)

    def commit(self, res: torch.Tensor, M: int, kv_len: int) -> None:
        """Moves the accepted path's rows behind the kv_len committed ones."""
        B.ghd_commit_path_q4(self.cache, res, M, kv_len)


def decode(stack: Q4Stack, table: torch.Tensor, first: int, count: int, parent: Sequence[int], draft=None
           ) -> Tuple[List[int], int, float]:
    """At least `count` tokens behind `first`, greedily: (tokens, steps, seconds).  parent: the tree of
    every step; draft(written) -> the tokens of its nodes 1 .. M - 1 (none for a tree of one node)."""
    M = len(parent)
    tree = torch.tensor(parent, dtype=torch.int32, device=table.device)
    res = torch.empty(2 + M, dtype=torch.int32, device=table.device)
    amax = torch.empty(M, dtype=torch.int32, device=table.device)
    written: List[int] = []
    kv_len = steps = 0
    root = first
    torch.cuda.synchronize()
    start = time.perf_counter()
    while len(written) < count:
        nodes = torch.tensor([root] + (draft(written) if M > 1 else []), dtype=torch.int32, device=table.device)
        logits = stack.step(B.ghd_embed(table, nodes), tree, kv_len)
        B.ghd_accept_greedy_static(logits, nodes, tree, res, amax)
        stack.commit(res, M, kv_len)
        r = res.tolist()
        taken, root = r[0], r[1]
        path = nodes[torch.tensor(r[2:2 + taken], device=table.device)].tolist()
        written += path[1:] + [root]
        kv_len += taken
        steps += 1
    torch.cuda.synchronize()
    return written, steps, time.perf_counter() - start


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    shapes = {s.name: s for s in (wl.TINY, wl.LLAMA_7B, wl.LLAMA_13B)}
    ap.add_argument("--shape", choices=sorted(shapes), default="tiny")
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--kv-heads", type=int, default=0, help="0: as many as query heads")
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--group", type=int, choices=(32, 64, 128), default=128)
    a = ap.parse_args()
    shape = wl.with_layers(shapes[a.shape], a.layers)
    parent = wl.tree_medusa(16, (4, 2, 1, 1), 1).tolist()
    capacity = -(-(a.tokens + len(parent) + 8) // 32) * 32
    layers = [wl.layer_weights(shape, 0, i, "cuda") for i in range(shape.L)]
    stack = Q4Stack(shape, a.kv_heads or shape.nh, layers, wl.head_weights(shape, 0, "cuda"), capacity, a.group)
    del layers
    table = wl.embedding_table(shape, 0, "cuda")

    decode(stack, table, 1, 2, [-1])                       # first calls load the kernels
    plain, steps, sec = decode(stack, table, 1, a.tokens, [-1])
    print("one token a step : %d tokens in %d steps, %.2f ms a step" % (len(plain), steps, 1e3 * sec / steps))

    depth = [0] * len(parent)
    for i in range(1, len(parent)):
        depth[i] = depth[parent[i]] + 1

    def draft(written: List[int]) -> List[int]:
        """The token that comes at each node's depth, at two nodes in three: a stand-in for drafting
        heads, which need training."""
        out = []
        for i in range(1, len(parent)):
            at = len(written) + depth[i] - 1
            right = at < len(plain) and i % 3 != len(written) % 3
            out.append(plain[at] if right else (i * 7919) % shape.V)
        return out

    tree, steps, sec = decode(stack, table, 1, a.tokens, parent, draft)
    same = tree[:a.tokens] == plain[:a.tokens]
    print("trees of %d nodes: %d tokens in %d steps, %.2f ms a step, same tokens: %s"
          % (len(parent), len(tree), steps, 1e3 * sec / steps, same))


if __name__ == "__main__":
    main()
