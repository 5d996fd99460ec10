"""A decoder layer with 2-bit weights, for prompts, single tokens and drafted trees of many requests.

    residual, last block's output -> [norm behind it, scale] -> residual -> norm -> attention block
      -> [norm behind it, scale] -> residual -> norm -> router -> 2-bit experts (+ a shared one) -> block's output

Every step is a call of ``binding`` or of ``attention_block``; a layer holds the weights and no memory of a step.
``python -m paper_2508_06753_amd.decoder_layer`` runs two layers over a prompt and single tokens.
"""
import torch

from . import binding as w2


class MoeBlock:
    """router: binding.Router, experts: binding.Experts.  shared: None, or (gate_up blob, down blob, inter) of an expert that every
    row goes to."""

    def __init__(self, router, experts, shared=None):
        if router.K != experts.hidden or router.n_experts != experts.n_experts:
            raise ValueError("the router's K and n_experts must be the experts' hidden and n_experts")
        self.router, self.experts, self.shared = router, experts, shared

    def workspace_size(self, M):
        """Bytes of workspace of a step of M rows (a larger batch may need fewer)."""
        e = self.experts
        sizes = [w2.moe_route_workspace_size(self.router, M), w2.moe_experts_workspace_size(e, M, self.router.top_k)]
        if self.shared is not None:
            inter = self.shared[2]
            sizes += [w2.workspace_size(M, e.hidden, 2 * inter, e.G, a16=True), w2.workspace_size(M, inter, e.hidden, e.G, a16=True)]
        return max(16, max(sizes))

    def step(self, x, workspace=None):
        """x bf16 [M, hidden] -> bf16 [M, hidden].  `workspace`: as for AttentionBlock.step."""
        M, e = x.shape[0], self.experts
        need = self.workspace_size(M)
        ws = torch.empty(need, dtype=torch.uint8, device=x.device) if workspace is None else workspace
        if ws.numel() < need:
            raise ValueError(f"workspace has {ws.numel()} bytes, the step needs {need}")
        base = None
        if self.shared is not None:
            gate_up, down, inter = self.shared
            h = w2.matmul_a16_epi(gate_up, e.hidden, 2 * inter, e.G, x, act=w2.ACT_SILU_MUL, workspace=ws)
            base = w2.matmul_a16(down, inter, e.hidden, e.G, h, workspace=ws)
        ids, weights = w2.moe_route(self.router, x, workspace=ws)
        return w2.moe_experts(e, x, ids, weights, base=base, out=base, workspace=ws)


class DecoderLayer:
    """attention: attention_block.AttentionBlock, norms: two binding.Norm (what stands before either block)."""

    def __init__(self, attention, moe, attention_norm, moe_norm):
        self.attention, self.moe = attention, moe
        self.attention_norm, self.moe_norm = attention_norm, moe_norm

    def workspace_size(self, M, batch, cache):
        return max(self.attention.workspace_size(M, batch, cache), self.moe.workspace_size(M))

    def step(self, residual, y, cache, batch, workspace=None):
        """residual (fp32 or bf16 [M, hidden]) and the last block's output y (bf16, or None before the first layer) -> the same
        behind this layer: what the next one's step takes, or binding.residual_norm for the model's last norm.

        The rows' keys and values go into `cache`.  `workspace`: as for AttentionBlock.step."""
        if workspace is None:
            workspace = torch.empty(self.workspace_size(residual.shape[0], batch, cache), dtype=torch.uint8, device=residual.device)
        x, residual = w2.residual_norm(self.attention_norm, residual, y)
        a = self.attention.step(x, cache, batch, workspace=workspace)
        x, residual = w2.residual_norm(self.moe_norm, residual, a, out=x, residual_out=residual)
        return residual, self.moe.step(x, workspace=workspace)


def prepack_experts(codes, scales, G, codec=w2.CODEC_INT2):
    """Blobs of n_experts matrices, uint8 [n_experts, bytes], of codes uint8 [n_experts, K, N] and scales [n_experts, K/G, N]."""
    return torch.stack([w2.prepack(c, s, G, codec) for c, s in zip(codes, scales)])


def main():
    """True: every row is finite, and none of zeros."""
    from . import synth
    from .attention_block import AttentionBlock, causal_batch
    hidden, inter, E, top_k, n_q, n_kv, D, G, page, n_requests, layers = 1024, 512, 16, 4, 8, 2, 128, 128, 16, 2, 2
    width = (n_q + 2 * n_kv) * D
    gen = torch.Generator(device="cuda").manual_seed(1)
    scaled = lambda *shape: (torch.rand(shape, device="cuda", generator=gen) * 0.02 + 0.005).bfloat16()  # noqa: E731

    def blob(K, N, seed):
        codes, scales = synth.make_weights(K, N, G, 0, seed=seed)
        return w2.prepack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales.view("int16")).cuda(), G)

    def layer(i):
        codes = lambda K, N: torch.randint(0, 4, (E, K, N), dtype=torch.uint8, device="cuda", generator=gen)  # noqa: E731
        ones = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
        experts = w2.Experts(prepack_experts(codes(hidden, 2 * inter), scaled(E, hidden // G, 2 * inter), G),
                             prepack_experts(codes(inter, hidden), scaled(E, inter // G, hidden), G), hidden, inter, G)
        router = w2.Router(torch.randn(E, hidden, device="cuda", generator=gen).bfloat16(), top_k)
        attention = AttentionBlock(blob(hidden, width, 10 + i), blob(n_q * D, hidden, 20 + i), hidden, n_q, n_kv, D, G, w2.Rope(D))
        shared = blob(hidden, 2 * inter, 30 + i), blob(inter, hidden, 40 + i), inter
        return DecoderLayer(attention, MoeBlock(router, experts, shared), w2.Norm(ones), w2.Norm(ones, post_weight=ones))

    stack, last = [layer(i) for i in range(layers)], w2.Norm(torch.ones(hidden, dtype=torch.bfloat16, device="cuda"))
    caches = [w2.KVCache(*(torch.zeros(32, page, n_kv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))) for _ in stack]
    table = torch.arange(n_requests * 8, dtype=torch.int32, device="cuda").view(n_requests, 8)
    lens, sound = [37, 60], True
    for what, batch in [("prompts", causal_batch([0, 0], lens, table, page, "cuda")),
                        ("single tokens", causal_batch(lens, [1, 1], table, page, "cuda"))]:
        residual, y = torch.randn(batch.positions.shape[0], hidden, device="cuda", generator=gen), None
        for block, cache in zip(stack, caches):
            residual, y = block.step(residual, y, cache, batch)
        x, _ = w2.residual_norm(last, residual, y)
        finite = bool(torch.isfinite(x).all())
        sound &= finite and bool((x != 0).any(dim=1).all())
        print(f"{what}: {x.shape[0]} rows, rms {x.float().square().mean().sqrt().item():.3f}, finite {finite}")
    return sound


if __name__ == "__main__":
    main()
