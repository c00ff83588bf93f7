#!/usr/bin/env python3
"""A decoder whose sequences each run on their own quantization expert: the router chooses once a sequence (Section 3.1), then every layer goes

    norm -> fused projection of the sequence's expert -> rotary positions, keys and values into the paged 8-bit cache -> attention over the cache
         -> output projection -> residual and norm -> SILU_MLP block -> residual and norm of the next layer

with the grouped products of the library, moqe_residual_norm, moqe_kv_append and moqe_kv_attention.  Projections and MLP can be in 8-bit floating point too (binding.F8Mat, F8Mlp): then the norms
give 8-bit rows (moqe_residual_norm_f8) and products take those (moqe_f8_gemm).  A `Step` holds the buffers and marshalled calls for
S sequences of T new rows each (a prompt, or one token each); a step of one token can be captured into a graph, since lengths live on the device.  All sequences of a `Sequences` are
equally long; ragged rows, prefixes, biases by distance, gates and norms behind a block are arguments of the calls themselves (binding.KvBatch, Attention, ResidualNormCall).

A model with a `head` goes on to tokens: `Draw` is the vocabulary's product on the last row of every sequence and moqe_sample, `Generator` a prompt and single tokens, the latter captured with
embedding, layers, head and sampling in one graph.

    python -m paper_2508_09204_amd.decoder --prompt 512 --tokens 64 [--f8] [--fast-sums] [--vocabulary 32000]

times prompts and single tokens of a few layers on seeded synthetic weights and prints one JSON line.
"""
from __future__ import annotations

import argparse
import json
import math
from dataclasses import dataclass
from typing import List, Optional, Union

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
class F8Mlp:
    """A SILU_MLP block in 8-bit floating point: a gated pair [f, d] and a matrix [d, f] per expert, or one of each for all.  fast: both products with fast sums (binding.F8GemmCall)."""
    gate_up: List[mq.F8Mat]
    down: List[mq.F8Mat]
    fast: bool = False


@dataclass
class Layer:
    """qkv and out: a packed matrix per expert, [(n_heads + 2 kv heads) * head_dim, d] and [d, n_heads * head_dim], or one F8Mat for all; mlp: a block on d features.  fast: those projections that
    are in 8 bits with fast sums (binding.F8GemmCall)."""
    attn_norm: mq.Norm
    qkv: Union[List[mq.QMat], List[mq.F8Mat]]
    out: Union[List[mq.QMat], List[mq.F8Mat]]
    mlp_norm: mq.Norm
    mlp: Union[mq.Block, F8Mlp]
    fast: bool = False


@dataclass
class Decoder:
    """head: the vocabulary's matrix [V, d]; embedding: fp32 [V, d].  Only a Generator needs them."""
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
    head: Optional[mq.F8Mat] = None
    embedding: Optional[torch.Tensor] = None


def _f8(mats) -> bool:
    return isinstance(mats, F8Mlp) or isinstance(mats, list) and isinstance(mats[0], mq.F8Mat)


class Sequences:
    """What S sequences keep between steps: a cache for every layer, block tables, lengths, their experts and the buckets of those."""

    def __init__(self, model: Decoder, S: int, max_tokens: int, block_tokens: int = 64, device="cuda"):
        per = -(-max_tokens // block_tokens)
        self.S, self.max_tokens = S, max_tokens
        self.caches = [mq.KvCache.empty(S * per, model.kv_heads, block_tokens, model.head_dim, device) for _ in model.layers]
        self.block_table = torch.arange(S * per, dtype=torch.int32, device=device).view(S, per)
        K = model.router.n_experts
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
    """T new rows of every sequence through all layers.  Rows go into `x` (fp32 [S * T, d]); calling the step enqueues the work; `out` (bf16) has the normed rows, and `out8` of a model with a
    head has them in 8 bits."""

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
        self.y16 = torch.empty((M, d), **bf)                                     # results of 8-bit products
        self.out = torch.empty((M, d), **bf)
        eight = any(_f8(m) for l in model.layers for m in (l.qkv, l.out, l.mlp))
        self.normed8, self.att8 = (mq.F8Rows.empty(M, n, dev) if eight else None for n in (d, heads))
        self.out8 = mq.F8Rows.empty(M, d, dev) if model.head is not None else None
        mlps = [l.mlp for l in model.layers if _f8(l.mlp)]
        self.h8 = mq.F8Rows.empty(M, mlps[0].down[0].k, dev) if mlps else None
        batch = mq.KvBatch(seqs.block_table, seqs.kv_len, S, T, M)
        attn = mq.Attention(model.n_heads, model.head_dim ** -0.5, model.cap, model.window)
        need = [mq.moqe_kv_attention_workspace_bytes(attn, batch, seqs.caches[0])]
        for l in model.layers:
            for m in (l.qkv, l.out):
                need.append(self._f8_bytes(m, mq.TYPE_BF16) if _f8(m) else mq.moqe_grouped_qgemm_workspace_bytes(m, S, T))
            if _f8(l.mlp):
                need += [self._f8_bytes(l.mlp.gate_up, mq.TYPE_F8), self._f8_bytes(l.mlp.down, mq.TYPE_BF16)]
            else:
                need.append(mq.moqe_workspace_bytes_routed(l.mlp, S, T))
        ws = workspace                                           # the calls come one after the other and share it, and so may the steps of a stream
        if ws is None:
            ws = torch.empty(max(*need, 256), dtype=torch.uint8, device=dev)
        elif ws.numel() < max(need):
            raise ValueError(f"a workspace of {ws.numel()} bytes, the step needs {max(need)}")
        self.workspace = ws
        self._calls = self._norm(None, first.attn_norm, first.qkv)
        for i, layer in enumerate(model.layers):
            self._calls += self._product(self.normed, self.normed8, layer.qkv, self.qkv, layer.fast)
            self._calls += [mq.KvAppendCall(self.qkv, model.n_heads, model.rope, batch, seqs.caches[i], self.q),
                            mq.KvAttentionCall(self.q, attn, batch, seqs.caches[i], self.att, ws)]
            if _f8(layer.out):
                self._calls.append(mq.ResidualNormF8Call(None, self.att, self.att8))
            y = self.y16 if _f8(layer.out) else self.y
            self._calls += self._product(self.att, self.att8, layer.out, y, layer.fast)
            self._calls += self._norm(y, layer.mlp_norm, layer.mlp)
            if _f8(layer.mlp):
                y = self.y16
                self._calls += self._product(None, self.normed8, layer.mlp.gate_up, self.h8, layer.mlp.fast)
                self._calls += self._product(None, self.h8, layer.mlp.down, y, layer.mlp.fast)
            else:
                y = self.y
                self._calls.append(self._mlp(layer.mlp, ws))
            if i + 1 < len(model.layers):
                self._calls += self._norm(y, model.layers[i + 1].attn_norm, model.layers[i + 1].qkv)
            elif model.head is not None:
                self._calls.append(mq.ResidualNormF8Call(y, self.x, self.out8, self.out, self.x, scale=model.residual_scale, pre=model.final_norm))
            else:
                self._calls.append(mq.ResidualNormCall(y, self.x, self.out, self.x, scale=model.residual_scale, pre=model.final_norm))
        self._graph: Optional[torch.cuda.CUDAGraph] = None

    def _f8_bytes(self, mats, y_type) -> int:
        return mq.moqe_f8_gemm_workspace_bytes(mats, self.seqs.S, self.T, y_type)

    def _norm(self, y, norm, mats):
        """The residual with y, normed for what multiplies it."""
        kind, out = (mq.ResidualNormF8Call, self.normed8) if _f8(mats) else (mq.ResidualNormCall, self.normed)
        return [kind(y, self.x, out, residual_out=self.x if y is not None else None, scale=self.model.residual_scale if y is not None else 1.0, pre=norm)]

    def _product(self, a, a8, mats, y, fast=False):
        s, ws = self.seqs, self.workspace
        if not _f8(mats):
            flags = mq.SCATTER_OUTPUT | (mq.OUTPUT_BF16 if y.dtype == torch.bfloat16 else 0)
            return [lambda: mq.moqe_grouped_qgemm(a, s.offsets, s.perm, s.S, self.T, mats, y, flags, ws)]
        if len(mats) == 1:
            return [mq.F8GemmCall(a8, mats, y, S=s.S, T=self.T, workspace=ws, fast=fast)]
        return [mq.F8GemmCall(a8, mats, y, s.offsets, s.perm, s.S, self.T, scatter=True, workspace=ws, fast=fast)]

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


class Draw:
    """The next token of every sequence: the head's product on the last row that a step left, and moqe_sample.  `u` (fp32 [S]) holds the uniform numbers of the next call; temperature, top_k,
    top_p and min_p as in binding.SampleCall.  Calling it enqueues the work; `tokens` (int32 [S]) and `logprobs` have the result, `logits` (fp32 [S, V]) what it was drawn from."""

    def __init__(self, model: Decoder, step: Step, temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None, top_p: Optional[torch.Tensor] = None,
                 min_p: Optional[torch.Tensor] = None):
        if model.head is None:
            raise ValueError("the model has no head")
        S, T, V, dev = step.seqs.S, step.T, model.head.n, step.x.device
        self.logits = torch.empty((S, V), dtype=torch.float32, device=dev)
        self.u = torch.zeros(S, dtype=torch.float32, device=dev)
        self.tokens, self.logprobs = torch.zeros(S, dtype=torch.int32, device=dev), torch.empty(S, dtype=torch.float32, device=dev)
        last = mq.F8Rows(*(t.view(S, T, -1)[:, T - 1] for t in step.out8.tensors()), S, step.out8.d)
        self._calls = [mq.F8GemmCall(last, [model.head], self.logits),
                       mq.SampleCall(self.logits, self.u, self.tokens, temperature, top_k, top_p, min_p, self.logprobs)]

    def __call__(self) -> torch.Tensor:
        for call in self._calls:
            call()
        return self.tokens


def check_tokens(tokens: torch.Tensor, S: int, T: int, V: int) -> None:
    """Refuses what is not S sequences of T tokens below V (reads them: waits for the device)."""
    if tuple(tokens.shape) != (S, T) or tokens.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"tokens must be int32 or int64 {(S, T)}, got {tuple(tokens.shape)} of {tokens.dtype}")
    least, most = (int(v) for v in torch.aminmax(tokens))
    if least < 0 or most >= V:
        raise ValueError(f"tokens from {least} to {most}, the vocabulary has {V}")


def embed(table: torch.Tensor, tokens: torch.Tensor, x: torch.Tensor) -> None:
    """Rows of the table for tokens (below its length) into x, in place.  Where none was drawn (-1), that of token 0."""
    torch.index_select(table, 0, tokens.clamp(min=0), out=x)


class Generator:
    """Sequences continued token by token.  `start` takes the prompts' tokens (int [S, prompt]), chooses the experts and draws the first tokens; `next` draws the ones after, from the first
    call on as a replayed graph: embedding, layers, head and sampling without the host.  A sequence for which no token was left (-1: its logits are all NaN or minus
    infinity) goes on as from token 0."""

    def __init__(self, model: Decoder, S: int, prompt: int, tokens: int, block_tokens: int = 64, **how):
        if model.head is None or model.embedding is None:
            raise ValueError("the model has no head or no embedding")
        V, d = model.head.n, model.layers[0].qkv[0].k
        if tuple(model.embedding.shape) != (V, d) or model.embedding.dtype != torch.float32:
            raise ValueError(f"the embedding must be fp32 {(V, d)}, got {tuple(model.embedding.shape)} of {model.embedding.dtype}")
        dev = model.embedding.device
        self.model, self.seqs = model, Sequences(model, S, prompt + tokens, block_tokens, dev)
        self.prompt, self.token = Step(model, self.seqs, prompt), Step(model, self.seqs, 1)
        self.first, self.draw = Draw(model, self.prompt, **how), Draw(model, self.token, **how)
        self._graph: Optional[torch.cuda.CUDAGraph] = None

    def start(self, prompt: torch.Tensor, u: torch.Tensor) -> torch.Tensor:
        check_tokens(prompt, self.seqs.S, self.prompt.T, self.model.head.n)
        self.first.u.copy_(u)                            # refused, if it does not fit, while nothing has changed
        self.seqs.clear()
        embed(self.model.embedding, prompt.reshape(-1), self.prompt.x)
        self.seqs.route(self.model, self.prompt.x.bfloat16(), self.prompt.T)
        self.prompt()
        self.draw.tokens.copy_(self.first())
        return self.draw.tokens

    def _enqueue(self) -> None:
        embed(self.model.embedding, self.draw.tokens, self.token.x)
        self.token._enqueue()
        self.draw()

    def next(self, u: torch.Tensor) -> torch.Tensor:
        if self.seqs.tokens + 1 > self.seqs.max_tokens:
            raise ValueError(f"{self.seqs.tokens} tokens, sequences hold {self.seqs.max_tokens}")
        self.draw.u.copy_(u)
        self.seqs.tokens += 1
        if self._graph is None:
            self._enqueue()                              # what a process does once is done before the capture
            self._graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self._graph):
                self._enqueue()
        else:
            self._graph.replay()
        return self.draw.tokens


def synthetic(layers: int, d: int, f: int, n_heads: int, kv_heads: int, head_dim: int, experts, router_hidden: int = 0, seed: int = 0, theta: float = 1e4,
              head_norms: bool = False, cap: float = 0.0, window: int = 0, device="cuda", vocabulary: int = 0, fast: bool = False) -> Decoder:
    """A decoder of seeded normal weights; experts: (bits, group, symmetric) each, all quantized from the same weights, or a number: so many MLP blocks of their own in 8-bit floating point
    between projections in 8 bits that all share.  vocabulary: tokens of an embedding and a head, 0: none.  fast: fast sums of 8-bit products, but the head's."""
    from . import experts as ex
    gen = torch.Generator(device=device).manual_seed(seed)
    rand = lambda *shape, by=1.0: torch.randn(shape, generator=gen, device=device) * by  # noqa: E731
    norm = lambda n: mq.Norm("rms", 1e-6, 1.0 + 0.1 * rand(n))  # noqa: E731
    eight = isinstance(experts, int)

    def matrix(n, k):
        w = rand(n, k, by=k ** -0.5)
        return [ex.quantize_f8(w)] if eight else [ex.quantize_and_pack(w, bits, group, sym) for bits, group, sym in experts]

    def mlp():
        if not eight:
            return mq.Block(kind=mq.KIND_SILU_MLP, router=router, w0=matrix(f, d), w1=matrix(f, d), w2=matrix(d, f))
        return F8Mlp([ex.quantize_f8(rand(f, d, by=d ** -0.5), rand(f, d, by=d ** -0.5)) for _ in range(K)], [ex.quantize_f8(rand(d, f, by=f ** -0.5)) for _ in range(K)], fast)

    K = experts if eight else len(experts)
    hidden = router_hidden
    router = mq.Router(rand(hidden, d, by=d ** -0.5) if hidden else None, torch.zeros(hidden, device=device) if hidden else None,
                       rand(K, hidden or d, by=(hidden or d) ** -0.5), None, d, hidden, K)
    made = [Layer(norm(d), matrix((n_heads + 2 * kv_heads) * head_dim, d), matrix(d, n_heads * head_dim), norm(d), mlp(), fast) for _ in range(layers)]
    gains = [1.0 + 0.1 * rand(head_dim) if head_norms else None for _ in range(2)]
    rope = mq.Rope(rope_frequencies(head_dim, theta, device=device), head_dim, q_gain=gains[0], k_gain=gains[1])
    model = Decoder(made, norm(d), router, rope, n_heads, kv_heads, head_dim, cap, window, residual_scale=(2 * layers) ** -0.5)
    if vocabulary:
        model.head, model.embedding = ex.quantize_f8(rand(vocabulary, d, by=d ** -0.5)), rand(vocabulary, d)
    return model


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sequences", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--f8", action="store_true", help="projections and experts in 8-bit floating point")
    ap.add_argument("--fast-sums", action="store_true", help="fast sums of products in 8-bit floating point")
    ap.add_argument("--vocabulary", type=int, default=0, help="draw tokens of so many (0: rows go in and out)")
    a = ap.parse_args()
    S, d, heads = a.sequences, 4096, 32
    experts = 4 if a.f8 else [(4, 128, False), (4, 128, False), (3, 128, False), (8, 0, True)]
    model = synthetic(a.layers, d, 11008, heads, heads, 128, experts, router_hidden=256, vocabulary=a.vocabulary, fast=a.fast_sums)
    gen = torch.Generator(device="cuda").manual_seed(1)
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
    if a.vocabulary:
        full = lambda v: torch.full((S,), v, device="cuda")  # noqa: E731
        g = Generator(model, S, a.prompt, a.tokens + 1, temperature=full(0.8), top_p=full(0.95), top_k=full(100).int())
        prompt = torch.randint(0, a.vocabulary, (S, a.prompt), generator=gen, device="cuda")
        u = torch.rand((a.tokens + 1, S), generator=gen, device="cuda")
        for timed in (False, True):
            marks[0].record()
            g.start(prompt, u[0])
            marks[1].record()
            marks[2].record()
            for i in range(a.tokens if timed else 1):
                g.next(u[1 + i])
            marks[3].record()
        finite = g.draw.logprobs.isfinite().all()
    else:
        seqs = Sequences(model, S, a.prompt + a.tokens)
        prompt = Step(model, seqs, a.prompt)
        token = Step(model, seqs, 1)
        x = torch.randn((S * a.prompt, d), generator=gen, device="cuda")
        token.x.normal_()
        seqs.route(model, x.bfloat16(), a.prompt)
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
        finite = token.out.isfinite().all()
    torch.cuda.synchronize()
    print(json.dumps({"layers": a.layers, "sequences": S, "prompt": a.prompt, "prompt_ms": round(marks[0].elapsed_time(marks[1]), 3),
                      "token_ms": round(marks[2].elapsed_time(marks[3]) / a.tokens, 4), "finite": bool(finite)}))


if __name__ == "__main__":
    main()
