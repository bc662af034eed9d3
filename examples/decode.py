"""A decoding loop over one of the repository's linear stacks: packed products,
the 4-bit key-value cache with its attention, the residual norm and the sampler,
every step one CUDA graph.

    python examples/decode.py --stack stack131m --batch 1 --tokens 64

Weights and embeddings are random (seeded), so the tokens mean nothing; the step
is the one that a trained model of these shapes takes. Per layer:

    norm -> QKV product -> rotate, quantise, append -> attention -> O product
    -> norm -> gate-up product -> SwiGLU -> down product

then norm, head product, sample. Batch 1 runs the SwiGLU inside the down
projection (vbq_gemv_swiglu_in); batches of 2..16 run vbq_gemm_small."""

from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_02893_gb300 as vbq  # noqa: E402
import synth  # noqa: E402
from synth import gen  # noqa: E402

HEADS = {"stack131m": (12, 12, 64), "stack1b": (16, 2, 128), "stack9b": (32, 8, 128)}   # heads, kv heads, head dim


class Decoder:
    """A stack's packed weights, its caches and one step of decoding."""

    def __init__(self, stack: str, batch: int = 1, max_tokens: int = 4096, layers: int | None = None, seed: int = 0):
        self.batch, self.max_tokens = batch, max_tokens
        self.heads, self.kv_heads, self.head_dim = HEADS[stack]
        specs = synth.workload(stack + "-fused").mats
        self.layers = min(layers or len(specs), (len(specs) - 1) // 4)
        self.specs = specs[:4 * self.layers] + specs[-1:]
        self.layouts = [self._pack(s) for s in self.specs]
        self.vocab, self.width = self.specs[-1].n, self.specs[-1].k
        dev, rng = "cuda", torch.Generator(device="cuda").manual_seed(seed)
        f32 = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=dev)  # noqa: E731
        bf16 = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device=dev)  # noqa: E731
        self.embedding = torch.randn(self.vocab, self.width, generator=rng, device=dev)
        self.weights = [1 + 0.1 * torch.randn(self.width, generator=rng, device=dev) for _ in range(2 * self.layers + 1)]
        d, h, hk = self.head_dim, self.heads, self.kv_heads
        angle = torch.arange(max_tokens, device=dev, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, d, 2, device=dev, dtype=torch.float64) / d)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        pages = -(-max_tokens // 64)
        self.table = torch.arange(batch * pages, dtype=torch.int32, device=dev).reshape(batch, pages)
        self.caches = [vbq.KvCache(batch * pages, hk, d) for _ in range(self.layers)]
        self.workspace = vbq.vbq_kv_workspace(self.caches[0], batch, 1, h)
        self.pos = torch.zeros(batch, 1, dtype=torch.int32, device=dev)
        self.tokens = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.u = torch.zeros(batch, device=dev)
        full = lambda v, t=torch.float32: torch.full((batch,), v, dtype=t, device=dev)  # noqa: E731
        self.temperature, self.top_k = full(0.8), full(50, torch.int32)
        self.top_p, self.min_p = full(0.95), full(0.0)
        self.residual, self.x = f32(batch, self.width), bf16(batch, self.width)
        self.qkv, self.q = f32(batch, 1, h + 2 * hk, d), bf16(batch, 1, h, d)
        self.attended, self.y = bf16(batch, 1, h, d), f32(batch, self.width)
        self.gate_up = f32(batch, self.specs[2].n)
        self.logits, self.probs = f32(batch, self.vocab), f32(batch)

    @staticmethod
    def _pack(spec):
        inp = gen.matrix_inputs(spec, 1)
        widths = torch.from_numpy(inp["widths"]).to("cuda")
        codes = gen.codes_torch(widths, inp["key"], spec.k, device="cuda")
        scales = torch.from_numpy(inp["scales"].view(np.uint16).astype(np.int16)).to("cuda")
        return vbq.vbq_pack(codes, widths, scales)

    def _product(self, i: int, x, y):
        if self.batch == 1:
            vbq.vbq_gemv(self.layouts[i], x, y)
        else:
            vbq.vbq_gemm_small(self.layouts[i], x, y, self.batch)

    def step(self):
        """One token for every sequence: from self.tokens at self.pos to the next self.tokens."""
        h, hk = self.heads, self.kv_heads
        torch.index_select(self.embedding, 0, self.tokens, out=self.residual)
        vbq.vbq_residual_norm(self.residual, None, self.weights[0], 1e-5, out=self.x)
        for layer in range(self.layers):
            qkv, o, gate_up, down = range(4 * layer, 4 * layer + 4)
            cache = self.caches[layer]
            self._product(qkv, self.x, self.qkv)
            vbq.vbq_kv_append(cache, self.table, self.pos, self.qkv[:, :, h:h + hk], self.qkv[:, :, h + hk:], q=self.qkv[:, :, :h],
                              cos=self.cos, sin=self.sin, q_out=self.q)
            vbq.vbq_kv_attend(cache, self.table, self.pos, self.q, out=self.attended, workspace=self.workspace)
            self._product(o, self.attended, self.y)
            vbq.vbq_residual_norm(self.y, self.residual, self.weights[2 * layer + 1], 1e-5, out=self.x, residual_out=self.residual)
            self._product(gate_up, self.x, self.gate_up)
            if self.batch == 1:
                vbq.vbq_gemv_swiglu_in(self.layouts[down], self.gate_up, self.y)
            else:
                hidden = torch.nn.functional.silu(self.gate_up[:, 0::2]) * self.gate_up[:, 1::2]
                vbq.vbq_gemm_small(self.layouts[down], hidden.to(torch.bfloat16), self.y, self.batch)
            vbq.vbq_residual_norm(self.y, self.residual, self.weights[2 * layer + 2], 1e-5, out=self.x, residual_out=self.residual)
        self._product(len(self.layouts) - 1, self.x, self.logits)
        vbq.vbq_sample(self.logits, self.temperature, self.top_k, self.top_p, self.min_p, self.u, tokens=self.tokens,
                       probs=self.probs, kept=False)
        self.pos.add_(1)

    def reset(self, tokens):
        self.pos.zero_()
        self.tokens.copy_(tokens)

    def capture(self):
        """The step as a CUDA graph (the caches and self.pos move on by one step while capturing warms up)."""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step()
        return graph

    def generate(self, first, uniforms, graph=None):
        """Tokens (steps, batch) from the first token of each sequence and given random numbers (steps, batch)."""
        self.reset(first)
        out = torch.empty(uniforms.shape, dtype=torch.int32, device="cuda")
        for i in range(uniforms.shape[0]):
            self.u.copy_(uniforms[i])
            if graph is None:
                self.step()
            else:
                graph.replay()
            out[i].copy_(self.tokens)
        return out


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--stack", default="stack131m", choices=sorted(HEADS))
    ap.add_argument("--batch", type=int, default=1)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--layers", type=int, default=None)
    a = ap.parse_args()
    decoder = Decoder(a.stack, a.batch, max_tokens=max(a.tokens + 2, 64), layers=a.layers)
    graph = decoder.capture()
    u = torch.rand(a.tokens, a.batch, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    first = torch.arange(a.batch, dtype=torch.int32, device="cuda")
    decoder.generate(first, u, graph)
    torch.cuda.synchronize()
    began = time.perf_counter()
    tokens = decoder.generate(first, u, graph)
    torch.cuda.synchronize()
    spent = time.perf_counter() - began
    vbq.vbq_device_status()
    print("tokens of the first sequence:", tokens[:16, 0].tolist())
    print(f"{a.stack}, {decoder.layers} layers, batch {a.batch}: {spent / a.tokens * 1e6:.1f} us a step, "
          f"{a.tokens * a.batch / spent:.0f} tokens/s")


if __name__ == "__main__":
    main()
