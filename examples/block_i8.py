"""The last block of a Mixture-of-Experts model in 8 bits, from a residual stream to logits:

    h      = x + residual                     moe_rmsnorm_i8: bf16 rows for the router, 8-bit rows for the experts
    h'     = h + experts(norm(h))             moe_layer_forward_i8
    logits = head(norm(h'))                   moe_rmsnorm_i8, moe_gemm_i8

    python examples/block_i8.py [tokens]      shapes of the qwen3_30b_a3b preset, compared with the same block in bf16
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_17889_amd import binding as B  # noqa: E402
from paper_2605_17889_amd import synth  # noqa: E402

EPS = 1e-6


def in_8_bits(w):
    """Matrices [..., N, K] as 8-bit integers and a scale for each of their rows."""
    q = torch.empty(w.shape, dtype=torch.int8, device=w.device)
    scale = torch.empty(w.shape[:-1], dtype=torch.float32, device=w.device)
    B.moe_quantize_i8(w.reshape(-1, w.shape[-1]), q.view(-1, w.shape[-1]), scale.view(-1))
    return q, scale


class Block:
    """Weights and buffers of the block for up to T tokens; a call leaves the logits [T, vocabulary] fp32 of its tokens."""

    def __init__(self, cfg, vocabulary, device="cuda"):
        T, d = cfg.T, cfg.d_model
        self.cfg, self.vocabulary = cfg, vocabulary
        self.ctx = B.MoeContext(T, d, cfg.d_ff, cfg.E, cfg.k)
        self.router = synth.make_router(cfg, device)
        self.bf16 = synth.make_experts(cfg, device)
        self.experts = [t for w in self.bf16 for t in in_8_bits(w)]
        gen = torch.Generator(device=device).manual_seed(cfg.seed)
        self.head_bf16 = (torch.randn((vocabulary, d), generator=gen, device=device) * 0.02).bfloat16()
        self.head = in_8_bits(self.head_bf16)
        self.norms = [(1 + 0.1 * torch.randn(d, generator=gen, device=device)).bfloat16() for _ in range(2)]
        rows = lambda kind: torch.empty((T, d), dtype=kind, device=device)
        self.h, self.y, self.out, self.q = rows(torch.bfloat16), rows(torch.bfloat16), rows(torch.bfloat16), rows(torch.int8)
        self.scale = torch.empty(T, dtype=torch.float32, device=device)
        self.logits = torch.empty((T, vocabulary), dtype=torch.float32, device=device)

    def __call__(self, x, residual):
        T, d = x.shape
        h, y, out, q, scale = self.h[:T], self.y[:T], self.out[:T], self.q[:T], self.scale[:T]
        B.moe_rmsnorm_i8(x, residual, self.norms[0], EPS, h, y, q, scale)
        B.moe_layer_forward_i8(self.ctx, y, q, scale, self.router, None, *self.experts, T, out)
        B.moe_rmsnorm_i8(out, h, self.norms[1], EPS, q=q, q_scale=scale)
        B.moe_gemm_i8(self.ctx, q, scale, None, T, 1, self.vocabulary, d, *self.head, self.logits[:T])
        return self.logits[:T]

    def in_bf16(self, x, residual):
        """The same block with nothing in 8 bits, for comparison."""
        T = x.shape[0]
        norm = lambda v, w: (v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * w.float()).bfloat16()
        h = x.float() + residual.float()
        out = torch.empty_like(x)
        B.moe_layer_forward(self.ctx, norm(h, self.norms[0]), self.router, None, *self.bf16, T, out)
        return norm(out.float() + h.bfloat16().float(), self.norms[1]).float() @ self.head_bf16.float().t()


def main():
    T = int(sys.argv[1]) if len(sys.argv) > 1 else 64
    cfg = synth.PRESETS["qwen3_30b_a3b_prefill"].with_T(T)
    block = Block(cfg, 32000)
    x, residual = synth.make_tokens(cfg, "cuda"), synth.make_tokens(cfg, "cuda") * 0.5
    logits = block(x, residual)
    want = block.in_bf16(x, residual)
    error = ((logits - want).norm() / want.norm()).item()
    same = (logits.argmax(-1) == want.argmax(-1)).float().mean().item()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(20):
        block(x, residual)
    end.record()
    torch.cuda.synchronize()
    print(f"{T} tokens: {start.elapsed_time(end) / 20 * 1e3:.0f} us a block; logits differ from bf16 by {error:.2%} of their norm, "
          f"{same:.0%} of the largest ones are the same")


if __name__ == "__main__":
    main()
