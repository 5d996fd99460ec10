"""The attention half of a decoder layer with 2-bit projections, for prompts, single tokens and drafted trees of many requests.

    QKV projection (2-bit) [+ adapters] -> norm of q and k, rotation, K and V into the paged cache
      -> attention over the cache -> output projection (2-bit) [+ adapters]

Every step is a call of ``binding``; this module holds the weights and no memory of a step: steps may run on several streams,
from several threads and in graphs.  ``python -m paper_2508_06753_amd.attention_block`` runs a prompt, a drafted tree and single tokens.
"""
from dataclasses import dataclass
from typing import Optional

import torch

from . import binding as w2


@dataclass
class Batch:
    """Where the rows of one step belong (device tensors, see binding.qk_norm_rope, tree_attention, lora_add)."""
    positions: torch.Tensor                  # int32 [M]
    slots: torch.Tensor                      # int64 [M]: where each row's key and value go
    page_table: torch.Tensor                 # int32 [requests, pages]
    row_start: torch.Tensor                  # int32 [requests + 1]
    kv_len: torch.Tensor                     # int32 [requests], the rows of this step included
    max_rows: int
    max_len: int
    total_len: int = 0
    mask: Optional[torch.Tensor] = None      # int64 [M, words]; None: causal
    adapter: Optional[torch.Tensor] = None   # int32 [M]; None: no adapters


class AttentionBlock:
    """wqkv, wo: blobs of binding.prepack, [hidden -> (n_q + 2 n_kv) head_dim] and [n_q head_dim -> hidden], group size G."""

    def __init__(self, wqkv, wo, hidden, n_q, n_kv, head_dim, G, rope, q_weight=None, k_weight=None, eps=1e-6,
                 qkv_lora=None, o_lora=None):
        self.wqkv, self.wo, self.hidden, self.G = wqkv, wo, hidden, G
        self.n_q, self.n_kv, self.head_dim = n_q, n_kv, head_dim
        self.width = (n_q + 2 * n_kv) * head_dim
        self.rope, self.q_weight, self.k_weight, self.eps = rope, q_weight, k_weight, eps
        self.qkv_lora, self.o_lora = qkv_lora, o_lora

    def workspace_size(self, M, batch, cache):
        """Bytes of workspace of a step of M rows (a larger batch may need fewer)."""
        inner = self.n_q * self.head_dim
        sizes = [w2.workspace_size(M, self.hidden, self.width, self.G), w2.workspace_size(M, inner, self.hidden, self.G),
                 w2.tree_attention_workspace_size(batch.kv_len.shape[0], M, self.n_q, cache, batch.max_rows, batch.max_len,
                                                  batch.total_len)]
        sizes += [w2.lora_workspace_size(a, M) for a in (self.qkv_lora, self.o_lora) if a is not None]
        return max(16, max(sizes))

    def step(self, X, cache, batch, workspace=None):
        """X (fp32 or bf16 [M, hidden]) -> bf16 [M, hidden]; the rows' keys and values go into `cache` (binding.KVCache).

        `workspace`: a uint8 device tensor of workspace_size(M, batch, cache) bytes or more, which is the step's alone until it has
        run; None: allocated for the step, like the tensors between its calls, from the current stream's memory (in a graph's
        capture: from the graph's own)."""
        M = X.shape[0]
        need = self.workspace_size(M, batch, cache)
        ws = torch.empty(need, dtype=torch.uint8, device=X.device) if workspace is None else workspace
        if ws.numel() < need:
            raise ValueError(f"workspace has {ws.numel()} bytes, the step needs {need}")
        qkv = w2.matmul_a8_fused(self.wqkv, self.hidden, self.width, self.G, X, workspace=ws)
        if self.qkv_lora is not None and batch.adapter is not None:
            w2.lora_add(self.qkv_lora, X, batch.adapter, qkv, out=qkv, workspace=ws)
        q = w2.qk_norm_rope(qkv, self.n_q, self.rope, batch.positions, cache, batch.slots, q_weight=self.q_weight,
                            k_weight=self.k_weight, eps=self.eps)
        o = w2.tree_attention(q, cache, batch.page_table, batch.row_start, batch.kv_len, batch.max_rows, batch.max_len,
                              mask=batch.mask, total_len=batch.total_len, workspace=ws)
        o = o.view(M, -1)
        y = w2.matmul_a8_fused(self.wo, self.n_q * self.head_dim, self.hidden, self.G, o, workspace=ws)
        if self.o_lora is not None and batch.adapter is not None:
            w2.lora_add(self.o_lora, o, batch.adapter, y, out=y, workspace=ws)
        return y


def causal_batch(starts, counts, page_table, page_size, device, adapter=None):
    """The Batch of `counts` new tokens of each request behind `starts` committed ones: prompts, chunks, single tokens.  Built row by
    row on the host, from a copy of the page table that waits for the GPU: a program that serves keeps its own."""
    rows = [(r, starts[r] + i) for r in range(len(starts)) for i in range(counts[r])]
    i32 = dict(dtype=torch.int32, device=device)
    lens = [s + c for s, c in zip(starts, counts)]
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    table = page_table.cpu()
    slots = [int(table[r, p // page_size]) * page_size + p % page_size for r, p in rows]
    return Batch(torch.tensor([p for _, p in rows], **i32), torch.tensor(slots, dtype=torch.int64, device=device), page_table,
                 torch.tensor(at, **i32), torch.tensor(lens, **i32), max(counts), max(lens), sum(lens),
                 adapter=None if adapter is None else torch.tensor([adapter[r] for r, _ in rows], **i32))


def tree_batch(starts, parents, page_table, page_size, device, adapter=None):
    """The Batch of a drafted tree per request: parents[r][i] < i is the token that token i follows, -1 the committed context.
    A token's position is its depth behind the context; it sees the context, its ancestors and itself."""
    batch = causal_batch(starts, [len(p) for p in parents], page_table, page_size, device, adapter)
    words = (max(len(p) for p in parents) + 63) // 64
    positions, masks = [], []
    for s, par in zip(starts, parents):
        depth, seen = [], []
        for i, p in enumerate(par):
            depth.append(0 if p < 0 else depth[p] + 1)
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
            positions.append(s + depth[i])
            masks.append([((seen[i] >> 64 * w) & (1 << 64) - 1) for w in range(words)])
    batch.positions = torch.tensor(positions, dtype=torch.int32, device=device)
    batch.mask = torch.tensor([[b - (1 << 64) if b >> 63 else b for b in m] for m in masks], dtype=torch.int64, device=device)
    return batch


def main():
    """True: every row is finite, and none of zeros."""
    from . import synth
    hidden, n_q, n_kv, D, G, page, n_requests = 1024, 8, 2, 128, 128, 16, 3
    width = (n_q + 2 * n_kv) * D

    def packed(K, N, seed):
        codes, scales = synth.make_weights(K, N, G, 0, seed=seed)
        return w2.prepack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales.view("int16")).cuda(), G)

    def adapters(K, N, parts, seed, rank=16, n=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        A = torch.randn(n, len(parts) * rank, K, device="cuda", generator=g) / K ** 0.5
        B = torch.randn(n, N, rank, device="cuda", generator=g) / rank ** 0.5
        return w2.Lora(A.bfloat16(), B.bfloat16(), parts=parts)

    ones = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    block = AttentionBlock(packed(hidden, width, 1), packed(n_q * D, hidden, 2), hidden, n_q, n_kv, D, G,
                           w2.Rope(D, base=500000.0, scaling=("bands", 8.0, 8192, 1.0, 4.0)), ones, ones,
                           qkv_lora=adapters(hidden, width, [n_q * D, n_kv * D, n_kv * D], 3),
                           o_lora=adapters(n_q * D, hidden, [hidden], 4))
    k = torch.zeros(64, page, n_kv, D, dtype=torch.bfloat16, device="cuda")
    cache = w2.KVCache(k, torch.zeros_like(k))
    table = torch.randperm(60, generator=torch.Generator().manual_seed(5))[:n_requests * 16].view(n_requests, 16).int().cuda()
    adapter, lens, sound = [0, 1, -1], [37, 120, 64], True
    for what, batch in [("prompts", causal_batch([0, 0, 0], lens, table, page, "cuda", adapter)),
                        ("drafted trees", tree_batch(lens, [[-1, 0, 0, 1], [-1, 0, 1, 1, 0], [-1]], table, page, "cuda", adapter)),
                        ("single tokens", causal_batch(lens, [1, 1, 1], table, page, "cuda", adapter))]:
        X = torch.randn(batch.positions.shape[0], hidden, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6))
        y = block.step(X, cache, batch)
        finite = bool(torch.isfinite(y).all())
        sound &= finite and bool((y != 0).any(dim=1).all())
        print(f"{what}: {y.shape[0]} rows, rms {y.float().square().mean().sqrt().item():.3f}, finite {finite}")
    return sound


if __name__ == "__main__":
    main()
