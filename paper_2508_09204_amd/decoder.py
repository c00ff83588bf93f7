#!/usr/bin/env python3
"""A decoder whose sequences each run on their own quantization expert: the router chooses once a sequence (Section 3.1), then every layer goes

    norm -> fused projection of the sequence's expert -> rotary positions, keys and values into the paged 8-bit cache -> attention over the cache
         -> output projection -> residual and norm -> SILU_MLP block -> residual and norm of the next layer

with the grouped products of the library, moqe_residual_norm, moqe_kv_append and moqe_kv_attention.  A `Step` holds the buffers and marshalled calls for
S sequences of T new rows each (a prompt, or one token each); a step of one token can be captured into a graph, since lengths live on the device.  All sequences of a `Sequences` are
equally long; ragged rows, prefixes, biases by distance, gates and norms behind a block are arguments of the calls themselves (binding.KvBatch, Attention, ResidualNormCall).

    python -m paper_2508_09204_amd.decoder --prompt 512 --tokens 64

times prompts and single tokens of a few layers on seeded synthetic weights and prints one JSON line.
"""
from __future__ import annotations

import argparse
import json
import math
from dataclasses import dataclass
from typing import List, Optional

import torch

from . import binding as mq


def rope_frequencies(rot_dim: int, theta: float = 10000.0, stretch: float = 1.0, by_parts: Optional[tuple] = None, device="cuda") -> torch.Tensor:
    """inv_freq for binding.Rope: theta ** (-2 j / rot_dim), float64.  stretch > 1 divides frequencies, so that positions `stretch` times as far keep the angles that
    the model was trained with.  by_parts = (trained length, fast, slow): pairs that turn more than `fast` times within the trained length keep their frequency, those
    that turn less than `slow` times are divided, those between get a share of each that is linear in their number of turns."""
    j = torch.arange(rot_dim // 2, dtype=torch.float64)
    f = theta ** (-2.0 * j / rot_dim)
    if by_parts is not None:
        length, fast, slow = by_parts
        keep = ((length * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        f = f * keep + f / stretch * (1 - keep)
    else:
        f = f / stretch
    return f.to(device)


@dataclass
class Layer:
    """qkv and out: a packed matrix per expert, [(n_heads + 2 kv heads) * head_dim, d] and [d, n_heads * head_dim]; mlp: a SILU_MLP block on d features."""
    attn_norm: mq.Norm
    qkv: List[mq.QMat]
    out: List[mq.QMat]
    mlp_norm: mq.Norm
    mlp: mq.Block


@dataclass
class Decoder:
    layers: List[Layer]
    final_norm: mq.Norm
    router: mq.Router
    rope: mq.Rope
    n_heads: int
    kv_heads: int
    head_dim: int
    cap: float = 0.0
    window: int = 0
    residual_scale: float = 1.0


class Sequences:
    """What S sequences keep between steps: a cache for every layer, block tables, lengths, their experts and the buckets of those."""

    def __init__(self, model: Decoder, S: int, max_tokens: int, block_tokens: int = 64, device="cuda"):
        per = -(-max_tokens // block_tokens)
        self.S, self.max_tokens = S, max_tokens
        self.caches = [mq.KvCache.empty(S * per, model.kv_heads, block_tokens, model.head_dim, device) for _ in model.layers]
        self.block_table = torch.arange(S * per, dtype=torch.int32, device=device).view(S, per)
        K = len(model.layers[0].qkv)
        i32 = dict(dtype=torch.int32, device=device)
        self.kv_len, self.expert_idx, self.perm = (torch.zeros(S, **i32) for _ in range(3))
        self.offsets = torch.zeros(K + 1, **i32)
        self.tokens = 0                                       # of every sequence, as the host counts them

    def route(self, model: Decoder, x: torch.Tensor, T: int) -> None:
        """Chooses the sequences' experts from rows x [S * T, d] and buckets them, for this and all later steps."""
        mq.moqe_route(x, self.S, T, model.router, self.expert_idx)
        mq.moqe_bucket(self.expert_idx, self.S, self.offsets.numel() - 1, None, self.offsets, self.perm, None)

    def clear(self) -> None:
        self.kv_len.zero_()
        self.tokens = 0


class Step:
    """T new rows of every sequence through all layers.  Rows go into `x` (fp32 [S * T, d]); calling the step enqueues the work; `out` (bf16) has the normed rows."""

    def __init__(self, model: Decoder, seqs: Sequences, T: int, workspace: Optional[torch.Tensor] = None):
        if T < 1 or T > seqs.max_tokens:
            raise ValueError(f"a step of {T} rows for sequences of at most {seqs.max_tokens} tokens")
        first, S, M = model.layers[0], seqs.S, seqs.S * T
        dev, d, width = seqs.kv_len.device, first.qkv[0].k, first.qkv[0].n
        heads = model.n_heads * model.head_dim
        bf = dict(dtype=torch.bfloat16, device=dev)
        self.model, self.seqs, self.T = model, seqs, T
        self.x = torch.empty((M, d), dtype=torch.float32, device=dev)            # the residual, in place
        self.normed, self.qkv, self.q, self.att = (torch.empty((M, n), **bf) for n in (d, width, heads, heads))
        self.y = torch.empty((M, d), dtype=torch.float32, device=dev)
        self.out = torch.empty((M, d), **bf)
        batch = mq.KvBatch(seqs.block_table, seqs.kv_len, S, T, M)
        attn = mq.Attention(model.n_heads, model.head_dim ** -0.5, model.cap, model.window)
        need = max(max(mq.moqe_grouped_qgemm_workspace_bytes(m, S, T) for l in model.layers for m in (l.qkv, l.out)),
                   mq.moqe_kv_attention_workspace_bytes(attn, batch, seqs.caches[0]),
                   max(mq.moqe_workspace_bytes_routed(l.mlp, S, T) for l in model.layers))
        ws = workspace                                           # the calls come one after the other and share it, and so may the steps of a stream
        if ws is None:
            ws = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        elif ws.numel() < need:
            raise ValueError(f"a workspace of {ws.numel()} bytes, the step needs {need}")
        self.workspace = ws
        calls = [mq.ResidualNormCall(None, self.x, self.normed, pre=first.attn_norm)]
        for i, layer in enumerate(model.layers):
            last = i + 1 == len(model.layers)
            calls += [
                self._product(self.normed, layer.qkv, self.qkv, mq.SCATTER_OUTPUT | mq.OUTPUT_BF16, ws),
                mq.KvAppendCall(self.qkv, model.n_heads, model.rope, batch, seqs.caches[i], self.q),
                mq.KvAttentionCall(self.q, attn, batch, seqs.caches[i], self.att, ws),
                self._product(self.att, layer.out, self.y, mq.SCATTER_OUTPUT, ws),
                mq.ResidualNormCall(self.y, self.x, self.normed, self.x, scale=model.residual_scale, pre=layer.mlp_norm),
                self._mlp(layer.mlp, ws),
                mq.ResidualNormCall(self.y, self.x, self.out if last else self.normed, self.x, scale=model.residual_scale,
                                    pre=model.final_norm if last else model.layers[i + 1].attn_norm),
            ]
        self._calls = calls
        self._graph: Optional[torch.cuda.CUDAGraph] = None

    def _product(self, a, experts, y, flags, ws):
        s = self.seqs
        return lambda: mq.moqe_grouped_qgemm(a, s.offsets, s.perm, s.S, self.T, experts, y, flags, ws)

    def _mlp(self, block, ws):
        return lambda: mq.moqe_forward_routed(block, self.seqs.expert_idx, self.normed, self.seqs.S, self.T, self.y, None, ws)

    def _enqueue(self) -> None:
        self.seqs.kv_len.add_(self.T)
        for call in self._calls:
            call()

    def capture(self) -> None:
        """Records the step; later calls replay it.  `x` and `out` stay the step's buffers."""
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self._enqueue()
        self._graph = graph

    def __call__(self) -> torch.Tensor:
        if self.seqs.tokens + self.T > self.seqs.max_tokens:
            raise ValueError(f"{self.seqs.tokens} + {self.T} tokens, sequences hold {self.seqs.max_tokens}")
        self.seqs.tokens += self.T
        if self._graph is not None:
            self._graph.replay()
        else:
            self._enqueue()
        return self.out


def synthetic(layers: int, d: int, f: int, n_heads: int, kv_heads: int, head_dim: int, experts, router_hidden: int = 0, seed: int = 0, theta: float = 1e4,
              head_norms: bool = False, cap: float = 0.0, window: int = 0, device="cuda") -> Decoder:
    """A decoder of seeded normal weights; experts: (bits, group, symmetric) each, all quantized from the same weights."""
    from . import experts as ex
    gen = torch.Generator(device=device).manual_seed(seed)
    rand = lambda *shape, by=1.0: torch.randn(shape, generator=gen, device=device) * by  # noqa: E731
    norm = lambda n: mq.Norm("rms", 1e-6, 1.0 + 0.1 * rand(n))  # noqa: E731

    def matrix(n, k):
        w = rand(n, k, by=k ** -0.5)
        return [ex.quantize_and_pack(w, bits, group, sym) for bits, group, sym in experts]

    K = len(experts)
    hidden = router_hidden
    router = mq.Router(rand(hidden, d, by=d ** -0.5) if hidden else None, torch.zeros(hidden, device=device) if hidden else None,
                       rand(K, hidden or d, by=(hidden or d) ** -0.5), None, d, hidden, K)
    made = [Layer(norm(d), matrix((n_heads + 2 * kv_heads) * head_dim, d), matrix(d, n_heads * head_dim), norm(d),
                  mq.Block(kind=mq.KIND_SILU_MLP, router=router, w0=matrix(f, d), w1=matrix(f, d), w2=matrix(d, f))) for _ in range(layers)]
    gains = [1.0 + 0.1 * rand(head_dim) if head_norms else None for _ in range(2)]
    rope = mq.Rope(rope_frequencies(head_dim, theta, device=device), head_dim, q_gain=gains[0], k_gain=gains[1])
    return Decoder(made, norm(d), router, rope, n_heads, kv_heads, head_dim, cap, window, residual_scale=(2 * layers) ** -0.5)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sequences", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--layers", type=int, default=4)
    a = ap.parse_args()
    S, d, heads = a.sequences, 4096, 32
    model = synthetic(a.layers, d, 11008, heads, heads, 128, [(4, 128, False), (4, 128, False), (3, 128, False), (8, 0, True)], router_hidden=256)
    seqs = Sequences(model, S, a.prompt + a.tokens)
    prompt = Step(model, seqs, a.prompt)
    token = Step(model, seqs, 1)
    x = torch.randn((S * a.prompt, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    token.x.normal_()
    seqs.route(model, x.bfloat16(), a.prompt)
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
    for timed in (False, True):
        seqs.clear()
        prompt.x.copy_(x)
        marks[0].record()
        prompt()
        marks[1].record()
        if not timed:
            token()                                  # what a process does once is done before the capture
            token.capture()
            seqs.tokens = a.prompt
            seqs.kv_len.fill_(a.prompt)
        marks[2].record()
        for _ in range(a.tokens):
            token()
        marks[3].record()
    torch.cuda.synchronize()
    print(json.dumps({"layers": a.layers, "sequences": S, "prompt": a.prompt, "prompt_ms": round(marks[0].elapsed_time(marks[1]), 3),
                      "token_ms": round(marks[2].elapsed_time(marks[3]) / a.tokens, 4), "finite": bool(token.out.isfinite().all())}))


if __name__ == "__main__":
    main()
