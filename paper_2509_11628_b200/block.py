"""A transformer block on the library's layer calls, and a stack of them as a model for the sampler.

The scheduler takes its model from the caller. ``TransformerBlock`` is the block such models are made of -- adaptive
layer norm, projections, rotary positions with the heads' RMS norm, attention over packed samples, gated
residuals, MLP -- built from ``speca_layer_modulate``, ``speca_layer_rope`` and ``speca_layer_attention`` with plain
matrix products in between, or, with ``eight=True``, from ``speca_layer_norm8``, ``speca_layer_quantize8`` and
``speca_layer_matmul8``: weights and the products' inputs in 8 bits, bias, GELU and gated residual in their epilogues. ``BlockStack`` runs L of them with random weights as the sampler's model: a full step computes and
caches every block's output; a speculative step computes the last block alone, on the forecast of its input, which
is the fresh feature that verification compares with the forecast of its output. The layer calls skip samples that are not
active, the products in 8 bits among them; plain ones run over all rows.

    python -m paper_2509_11628_b200.block        # a sampler run over a small stack, per-step decisions and counts
    python -m paper_2509_11628_b200.block --eight-bit
"""
from __future__ import annotations

import math
from typing import Sequence

import torch

from . import binding as S


def grid_positions(text: int, frames: int, height: int, width: int, device) -> torch.Tensor:
    """fp32 [text + frames * height * width, 3]: text tokens at the origin, then (time, height, width) of every patch."""
    t, h, w = torch.meshgrid(torch.arange(frames), torch.arange(height), torch.arange(width), indexing="ij")
    pos = torch.stack([t, h, w], -1).reshape(-1, 3).float()
    return torch.cat([torch.zeros(text, 3), pos]).to(device)


class TransformerBlock:
    """One block over ``batch`` samples of ``tokens`` tokens. Weights are random; the arithmetic is the block's."""

    def __init__(self, batch: int, tokens: int, heads: int, head_dim: int, axis_dims: Sequence[int], dtype: int = S.SPECA_BF16,
                 device: str = "cuda:0", seed: int = 0, mlp_ratio: int = 4, eight: bool = False):
        self.batch, self.tokens, self.heads, self.head_dim = batch, tokens, heads, head_dim
        self.dim = dim = heads * head_dim
        self.device, tdt = torch.device(device), S._TORCH_DTYPES[dtype]
        rows = batch * tokens
        self.layer = S.SpecaLayer([tokens * b for b in range(batch + 1)], dtype, n_heads=heads, n_kv_heads=heads,
                                  head_dim=head_dim, axis_dims=axis_dims, device=device)
        g = torch.Generator(device=self.device).manual_seed(seed)

        def weight(n_in, n_out, gain=1.0):
            w = torch.randn(n_in, n_out, generator=g, device=self.device) * (gain / math.sqrt(n_in))
            return w.to(tdt)

        self.w_qkv, self.w_out = weight(dim, 3 * dim), weight(dim, dim)
        self.w_up, self.w_down = weight(dim, mlp_ratio * dim), weight(mlp_ratio * dim, dim)
        self.w_mod = weight(dim, 6 * dim, 0.3)
        self.q_norm = (1 + 0.1 * torch.randn(head_dim, generator=g, device=self.device)).to(tdt)
        self.k_norm = (1 + 0.1 * torch.randn(head_dim, generator=g, device=self.device)).to(tdt)

        def rows_of(*shape):
            return torch.zeros(rows, *shape, device=self.device, dtype=tdt)

        self.mid, self.attn = rows_of(dim), rows_of(heads, head_dim)
        self.q, self.k = rows_of(heads, head_dim), rows_of(heads, head_dim)
        self.eight = eight
        if eight:  # the products take weights as [outputs, inputs]
            for name in ("w_qkv", "w_out", "w_up", "w_down"):
                setattr(self, name, S.quantize8(getattr(self, name).T.contiguous()))
            self.norm8, self.attn8, self.up8 = (S.Matrix8.empty(rows, n, self.device) for n in (dim, dim, mlp_ratio * dim))
            self.qkv, self.branch = rows_of(3 * dim), rows_of(dim)
        else:
            self.norm, self.unit = rows_of(dim), rows_of(dim)

    def __call__(self, x: torch.Tensor, cond: torch.Tensor, positions: torch.Tensor, out: torch.Tensor, active=None) -> torch.Tensor:
        """``out`` [rows, dim] = the block's output for ``x`` [rows, dim] and the conditioning ``cond`` [batch, dim]. Rows of
        samples whose ``active`` byte is zero are left as they are in ``out``."""
        h, hd, dim = self.heads, self.head_dim, self.dim
        mod = torch.nn.functional.silu(cond) @ self.w_mod                      # [batch, 6 dim]
        shift_a, scale_a, gate_a, shift_m, scale_m, gate_m = mod.split(dim, 1)
        if self.eight:
            layer = self.layer
            layer.norm8(x, self.norm8, S.SPECA_NORM_LAYER, scale=scale_a, shift=shift_a, active=active)
            layer.matmul8(self.norm8, self.w_qkv, self.qkv, active=active)
            qkv = self.qkv.view(-1, 3 * h, hd)
            layer.rope(qkv[:, :h], self.q, qkv[:, h:2 * h], self.k, positions, self.q_norm, self.k_norm, active=active)
            layer.attention(self.q, self.k, qkv[:, 2 * h:], self.attn, active=active)
            layer.quantize8(self.attn.view(-1, dim), self.attn8, active=active)
            layer.matmul8(self.attn8, self.w_out, self.branch, active=active)
            layer.norm8(x, self.norm8, S.SPECA_NORM_LAYER, branch=self.branch, gate=gate_a, scale=scale_m, shift=shift_m, x_out=self.mid,
                        active=active)
            layer.matmul8(self.norm8, self.w_up, self.up8, activation=S.SPECA_ACT_GELU, active=active)
            layer.matmul8(self.up8, self.w_down, out, residual=self.mid, gate=gate_m, active=active)
            return out
        self.layer.modulate(x, self.norm, scale=scale_a, shift=shift_a, active=active)
        qkv = (self.norm @ self.w_qkv).view(-1, 3 * h, hd)
        self.layer.rope(qkv[:, :h], self.q, qkv[:, h:2 * h], self.k, positions, self.q_norm, self.k_norm, active=active)
        self.layer.attention(self.q, self.k, qkv[:, 2 * h:], self.attn, active=active)
        branch = self.attn.view(-1, dim) @ self.w_out
        self.layer.modulate(x, self.norm, branch=branch, gate=gate_a, scale=scale_m, shift=shift_m, x_out=self.mid, active=active)
        branch = torch.nn.functional.gelu(self.norm @ self.w_up, approximate="tanh") @ self.w_down
        # the second residual: the norm that comes with it is the next block's affair
        self.layer.modulate(self.mid, self.unit, branch=branch, gate=gate_m, x_out=out, active=active)
        return out


class BlockStack:
    """L blocks as the model of ``scheduler.run_sampler``; the cached entries are their outputs, verified on the last."""

    def __init__(self, blocks: int, batch: int, tokens: int, heads: int, head_dim: int, axis_dims: Sequence[int],
                 positions: torch.Tensor, dtype: int = S.SPECA_BF16, device: str = "cuda:0", seed: int = 0, eight: bool = False):
        if blocks < 2:
            raise ValueError("a stack needs two blocks: the last one is verified on the forecast of the one before")
        self.blocks = [TransformerBlock(batch, tokens, heads, head_dim, axis_dims, dtype, device, seed + i, eight=eight) for i in range(blocks)]
        self.batch, self.tokens, self.dim = batch, tokens, heads * head_dim
        self.device, tdt = torch.device(device), S._TORCH_DTYPES[dtype]
        self.positions = positions.repeat(batch, 1).contiguous()
        g = torch.Generator(device=self.device).manual_seed(seed + 1000)
        self.start = torch.randn(batch * tokens, self.dim, generator=g, device=self.device)
        self.drift = torch.randn(batch * tokens, self.dim, generator=g, device=self.device)
        self.phase = torch.randn(batch, self.dim, generator=g, device=self.device)
        self.outs = [torch.zeros(batch * tokens, self.dim, device=self.device, dtype=tdt) for _ in self.blocks]
        self.fresh = torch.zeros(batch * tokens, self.dim, device=self.device, dtype=tdt)
        self.tdt = tdt
        self.backend = None

    @property
    def entries(self):
        return [(self.tokens, self.dim)] * len(self.blocks)

    def _cond(self, times):
        t = torch.tensor(list(times), device=self.device)[:, None]
        return torch.cos(self.phase + t).to(self.tdt)

    def _shaped(self, x):
        return x.view(self.batch, self.tokens, self.dim)

    def full(self, step, times, mask):
        """Every block for the samples in ``mask``: the features of a reference step."""
        active = torch.tensor([1 if m else 0 for m in mask], dtype=torch.uint8, device=self.device)
        t = torch.tensor(list(times), device=self.device).repeat_interleave(self.tokens)[:, None]
        x = (self.start + t * self.drift).to(self.tdt)
        cond = self._cond(times)
        for block, out in zip(self.blocks, self.outs):
            x = block(x, cond, self.positions, out, active)
        return [self._shaped(o) for o in self.outs]

    def verify_feature(self, step, times):
        """The last block for real, on the forecast output of the one before it, for the samples that speculate."""
        x = self.backend.outs[-2].reshape(self.batch * self.tokens, self.dim)
        return self._shaped(self.blocks[-1](x, self._cond(times), self.positions, self.fresh, self.backend.active))


def main() -> None:
    import argparse

    from .scheduler import SpecaCacheBackend, run_sampler
    parser = argparse.ArgumentParser(description="A sampler run over a small stack of transformer blocks with random weights.")
    parser.add_argument("--eight-bit", action="store_true", help="weights and the products' inputs in 8 bits")
    args = parser.parse_args()
    device = "cuda:0"
    positions = grid_positions(16, 1, 16, 16, device)
    stack = BlockStack(blocks=6, batch=2, tokens=positions.shape[0], heads=6, head_dim=64, axis_dims=(16, 24, 24),
                       positions=positions, device=device, eight=args.eight_bit)
    cache = S.SpecaCache(stack.entries, stack.batch, 2, S.SPECA_BF16, device)
    stack.backend = backend = SpecaCacheBackend(cache)
    trace = run_sampler(backend, stack, [1.0 - 0.02 * i for i in range(50)], tau0=0.1, beta=0.5, period=5, warm_refs=3,
                        gamma=1.0 / len(stack.blocks))
    for b in range(stack.batch):
        full, accepted, rejected = trace.counts(b)
        print("sample %d: %s  full %d accepted %d rejected %d, speedup by cost model %.2f" % (
            b, "".join(row[b] for row in trace.steps), full, accepted, rejected, trace.speedup(b)))
    for block in stack.blocks:
        block.layer.check()
    cache.close()


if __name__ == "__main__":
    main()
