"""Layers of a pipeline stage on one GPU, and the planner's tables measured from them.

``Embedding``, ``AttentionBlock`` (norm, causal attention over packed sequences and a residual) and ``ExpertBlock`` (a mixture of
experts with gated activations and a residual) run a micro-batch forward and backward through the layer operators of
``layers.py``: between the two they keep activations in 8 bits, but for what attention reads again in its own 16, and
their weight gradients add up over the micro-batches of a step.  ``Layer`` is an attention block before an expert block.  ``measure`` times one layer of each kind, as the
paper's profiling module does (Sec. 4.1.3; one layer per distinct type), and ``plan_problem`` makes the
planner's tables of the times and of the bytes that S micro-batches in flight keep:

    python -m paper_2609_06086_amd.stage          # measure, then search for the best placement of the layers
"""
from __future__ import annotations

import argparse
import statistics
from dataclasses import dataclass, replace
from typing import List, Optional

import numpy as np
import torch

from . import layers as L
from . import poseidon as P
from .workloads import Problem


@dataclass
class Shape:
    """Sizes of a model: its vocabulary, width, experts (of `inner` gated values, `chosen` per token), the tokens of a
    micro-batch, and with `heads` attention before the experts: its heads, the heads of its keys (0: as many) and the
    tokens of a sequence (0: all of a micro-batch)."""
    vocab: int = 32000
    width: int = 2048
    experts: int = 16
    chosen: int = 2
    inner: int = 2048
    tokens: int = 4096
    heads: int = 0
    kv_heads: int = 0
    sequence: int = 0


class Embedding:
    """The first layer: scaled rows of a table."""

    def __init__(self, shape: Shape, device, seed: int = 0, dtype=torch.bfloat16):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.scale = shape.width ** 0.5
        self.table = (torch.randn(shape.vocab, shape.width, generator=g, device=device) * 0.02).to(dtype)
        self.grad = torch.zeros(shape.vocab, shape.width, dtype=torch.float32, device=device)

    def forward(self, ids):
        return L.poseidon_embed(ids, self.table, self.scale), ids

    def backward(self, dout, ids) -> None:
        L.poseidon_embed_backward(ids, dout, self.table.shape[0], self.scale, out=self.grad, accumulate=True)

    @property
    def weight_bytes(self) -> int:
        return self.table.numel() * self.table.element_size() + self.grad.numel() * 4


@dataclass
class KeptAttention:
    """What an AttentionBlock keeps of a micro-batch for its backward pass."""
    offsets: Optional[torch.Tensor]
    h: L.Stash                 # the norm's input
    y: L.Stash                 # its output, the projections' input
    rstd: torch.Tensor
    both: torch.Tensor         # queries, keys and values
    a: torch.Tensor            # attention's output
    lse: torch.Tensor

    @property
    def kept_bytes(self) -> int:
        plain = (self.rstd, self.both, self.a, self.lse) + (() if self.offsets is None else (self.offsets,))
        return sum(t.numel() * t.element_size() for t in plain) + self.h.nbytes + self.y.nbytes

    @property
    def plain_bytes(self) -> int:
        """The same with the activations in their own 16 bits."""
        return self.kept_bytes + sum(2 * s.rows * s.width - s.nbytes for s in (self.h, self.y))


def key_heads(shape: Shape, dtype=torch.bfloat16) -> int:
    """The heads of the keys of an attention of these sizes; ValueError for what its operators do not take."""
    d, heads, kv_heads = shape.width, shape.heads, shape.kv_heads or shape.heads
    if not 0 < heads <= L.HEADS_MAX or d > L.NORM_WIDTH_MAX:
        raise ValueError(f"{heads} heads of a width of {d}: 1 to {L.HEADS_MAX}, widths up to {L.NORM_WIDTH_MAX}")
    if d % heads or d // heads % 8 or d // heads > L.HEAD_MAX:
        raise ValueError(f"{heads} heads do not share a width of {d} in multiples of 8 up to {L.HEAD_MAX}")
    if kv_heads < 0 or heads % kv_heads:
        raise ValueError(f"{kv_heads} heads of keys do not divide {heads} heads")
    if shape.sequence < 0:
        raise ValueError(f"sequences of {shape.sequence} tokens")
    if dtype not in (torch.float16, torch.bfloat16):
        raise ValueError(f"attention in {dtype}: float16 or bfloat16")
    return kv_heads


class AttentionBlock:
    """out = x + Wo attention(Wqkv norm(x)), causal within each of the packed sequences.  float16 or bfloat16."""

    def __init__(self, shape: Shape, device, seed: int = 0, dtype=torch.bfloat16):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        d, self.heads, self.kv_heads = shape.width, shape.heads, key_heads(shape, dtype)
        self.dim = d // self.heads
        self.parts = [n * self.dim for n in (self.heads, self.kv_heads, self.kv_heads)]

        def weight(*size):
            return (torch.randn(*size, generator=g, device=device) * size[-1] ** -0.5).to(dtype)

        self.norm, self.wqkv, self.wo = torch.ones(d, dtype=dtype, device=device), weight(sum(self.parts), d), weight(d, d)
        self.dnorm, self.dwqkv, self.dwo = (torch.zeros(w.shape, dtype=torch.float32, device=device)
                                            for w in (self.norm, self.wqkv, self.wo))

    @property
    def weight_bytes(self) -> int:
        return sum(w.numel() * (w.element_size() + 4) for w in (self.norm, self.wqkv, self.wo))

    def _heads(self, both):
        """Queries, keys and values as views of one product's rows."""
        return [part.view(both.shape[0], -1, self.dim) for part in both.split(self.parts, dim=1)]

    def forward(self, x, offsets=None):
        y = L.poseidon_norm_forward(x, self.norm, keep_out=True, keep_sum=True)
        both = L.poseidon_expert_product(y.out, self.wqkv)
        a, lse = L.poseidon_attention_forward(*self._heads(both), offsets)
        out = x + L.poseidon_expert_product(a.view(x.shape), self.wo)
        return out, KeptAttention(offsets, y.kept_sum, y.kept_out, y.rstd, both, a, lse)

    def backward(self, dout, kept: KeptAttention):
        a = kept.a.view(dout.shape)    # in 8 bits for its product's gradient, as all weight gradients take rows
        L.poseidon_weight_gradient(dout, L.poseidon_stash(a), out=self.dwo, accumulate=True)
        da = L.poseidon_expert_product(dout, self.wo, transposed=True)
        dboth = torch.empty_like(kept.both)
        dq, dk, dv = self._heads(dboth)
        L.poseidon_attention_backward(da.view(kept.a.shape), *self._heads(kept.both), kept.a, kept.lse, kept.offsets,
                                      dq=dq, dk=dk, dv=dv)
        L.poseidon_weight_gradient(dboth, kept.y, out=self.dwqkv, accumulate=True)
        dy = L.poseidon_expert_product(dboth, self.wqkv, transposed=True)
        return L.poseidon_norm_backward(dy, kept.h, kept.rstd, self.norm, dout, dweight=self.dnorm, accumulate=True)[0]


@dataclass
class Kept:
    """What an ExpertBlock keeps of a micro-batch for its backward pass."""
    x: torch.Tensor            # the router's input
    probs: torch.Tensor        # the chosen experts' weights
    choice: torch.Tensor
    plan: L.ExpertPlan
    cuts: Optional[List[int]]  # in 32 bits the experts' row ranges, on the host for the library's products
    xs: L.Stash
    gate: L.Stash
    up: L.Stash
    ys: L.Stash

    @property
    def kept_bytes(self) -> int:
        plain = (self.x, self.probs, self.choice, self.plan.order, self.plan.position, self.plan.offsets)
        return sum(t.numel() * t.element_size() for t in plain) + sum(s.nbytes for s in (self.xs, self.gate, self.up, self.ys))

    @property
    def plain_bytes(self) -> int:
        """The same with the activations in their own 16 bits."""
        stashes = (self.xs, self.gate, self.up, self.ys)
        return self.kept_bytes + sum(2 * s.rows * s.width - s.nbytes for s in stashes)


class ExpertBlock:
    """out = x + sum over the chosen experts of p * W2 (silu(W1g x) * W1u x)."""

    def __init__(self, shape: Shape, device, seed: int = 0, dtype=torch.bfloat16):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        d, f, e = shape.width, shape.inner, shape.experts

        def weight(*size):
            return (torch.randn(*size, generator=g, device=device) * size[-1] ** -0.5).to(dtype)

        self.chosen, self.inner = shape.chosen, f
        self.router, self.w1, self.w2 = weight(e, d), weight(e, 2 * f, d), weight(e, d, f)
        self.drouter, self.dw1, self.dw2 = (torch.zeros(w.shape, dtype=torch.float32, device=device)
                                            for w in (self.router, self.w1, self.w2))

    @property
    def weight_bytes(self) -> int:
        return sum(w.numel() * (w.element_size() + 4) for w in (self.router, self.w1, self.w2))

    @staticmethod
    def _product(rows, weights, plan, cuts, transposed=False):
        """rows of each expert's range times its weights; in 32 bits, which the operator does not take, by the library."""
        if cuts is None:
            return L.poseidon_expert_product(rows, weights, plan.offsets, transposed=transposed)
        weights = weights if transposed else weights.transpose(1, 2)
        out = rows.new_zeros(rows.shape[0], weights.shape[2])
        for e, (a, b) in enumerate(zip(cuts, cuts[1:])):
            if b > a:
                torch.matmul(rows[a:b], weights[e], out=out[a:b])
        return out

    def forward(self, x):
        f = self.inner
        logits, choice = torch.topk((x @ self.router.t()).float(), self.chosen, dim=1)
        probs, choice = torch.softmax(logits, 1), choice.to(torch.int32)
        plan = L.poseidon_expert_sort(choice, self.w1.shape[0])
        xs, kept_xs = L.poseidon_expert_gather(x, plan, keep=True)
        cuts = plan.offsets.tolist() if xs.dtype == torch.float32 else None
        both = self._product(xs, self.w1, plan, cuts)
        act, kept_gate, kept_up = L.poseidon_gated_forward(both[:, :f], both[:, f:])
        ys = self._product(act, self.w2, plan, cuts)
        out = x + L.poseidon_expert_combine(ys, plan, probs)
        return out, Kept(x, probs, choice, plan, cuts, kept_xs, kept_gate, kept_up, L.poseidon_stash(ys))

    def backward(self, dout, kept: Kept):
        f, plan, cuts = self.inner, kept.plan, kept.cuts
        dys, dprobs = L.poseidon_expert_combine_backward(dout, L.poseidon_restore(kept.ys), plan, kept.probs)
        act = L.poseidon_gated_forward(L.poseidon_restore(kept.gate), L.poseidon_restore(kept.up), keep=False)[0]
        L.poseidon_weight_gradient(dys, L.poseidon_stash(act), offsets=plan.offsets, out=self.dw2, accumulate=True)
        dact = self._product(dys, self.w2, plan, cuts, transposed=True)
        dboth = act.new_empty(act.shape[0], 2 * f)
        L.poseidon_gated_backward(dact, kept.gate, kept.up, dgate=dboth[:, :f], dup=dboth[:, f:])
        L.poseidon_weight_gradient(dboth, kept.xs, offsets=plan.offsets, out=self.dw1, accumulate=True)
        dxs = self._product(dboth, self.w1, plan, cuts, transposed=True)
        # the router: softmax over the chosen logits, then its product
        dlogits = kept.probs * (dprobs - (kept.probs * dprobs).sum(1, keepdim=True))
        dall = torch.zeros(kept.x.shape[0], self.router.shape[0], dtype=torch.float32, device=dout.device)
        dall.scatter_(1, kept.choice.long(), dlogits)
        self.drouter += dall.t() @ kept.x.float()
        return dout + L.poseidon_expert_combine(dxs, plan) + dall.to(dout.dtype) @ self.router


@dataclass
class KeptLayer:
    """What a Layer keeps of a micro-batch: its two blocks' parts."""
    attention: KeptAttention
    experts: Kept

    @property
    def kept_bytes(self) -> int:
        return self.attention.kept_bytes + self.experts.kept_bytes

    @property
    def plain_bytes(self) -> int:
        return self.attention.plain_bytes + self.experts.plain_bytes


class Layer:
    """An attention block, then an expert block."""

    def __init__(self, shape: Shape, device, seed: int = 0, dtype=torch.bfloat16):
        self.attention = AttentionBlock(shape, device, seed, dtype)
        self.experts = ExpertBlock(shape, device, seed + 1, dtype)

    @property
    def weight_bytes(self) -> int:
        return self.attention.weight_bytes + self.experts.weight_bytes

    def forward(self, x, offsets=None):
        h, attention = self.attention.forward(x, offsets)
        out, experts = self.experts.forward(h)
        return out, KeptLayer(attention, experts)

    def backward(self, dout, kept: KeptLayer):
        return self.attention.backward(self.experts.backward(dout, kept.experts), kept.attention)


@dataclass
class LayerProfile:
    """One layer kind: times of a micro-batch, bytes of its weights and their gradients, bytes a micro-batch keeps, what
    it would keep with its activations in their own 16 bits, and the most that a pass works with besides."""
    fwd_us: float
    bwd_us: float
    weight_bytes: int
    kept_bytes: int
    plain_bytes: int = 0
    work_bytes: int = 0

    def in_16_bits(self) -> "LayerProfile":
        """The same times with the memory of 16 bits: what a plan gains by the 8 bits' memory alone."""
        return replace(self, kept_bytes=self.plain_bytes)


def _median_us(f, repeats: int) -> float:
    times = []
    for _ in range(repeats):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return statistics.median(times)


def _work_bytes(f, device) -> int:
    """The most that a call of f has allocated at a time, but for what it keeps beside its output."""
    torch.cuda.reset_peak_memory_stats(device)
    result = f()
    out = result[0] if isinstance(result, tuple) else result
    stays = torch.cuda.memory_allocated(device) - (0 if out is None else out.numel() * out.element_size())
    return max(0, torch.cuda.max_memory_allocated(device) - stays)


def measure(shape: Shape, device=None, keep_8_bits: bool = True, repeats: int = 5):
    """(profile of the embedding, profile of an expert block, or with heads of a Layer) on this GPU.  The layers run with
    their activations kept in 8 bits; keep_8_bits False gives those times with the bytes that 16 bits would keep."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    g = torch.Generator(device=device)
    g.manual_seed(1)
    ids = torch.randint(0, shape.vocab, (shape.tokens,), generator=g, device=device, dtype=torch.int32)
    first, block = Embedding(shape, device), (Layer if shape.heads else ExpertBlock)(shape, device)
    x, _ = first.forward(ids)
    args = (x,)
    if shape.heads and shape.sequence:
        cuts = list(range(0, shape.tokens, shape.sequence)) + [shape.tokens]
        args = (x, torch.tensor(cuts, dtype=torch.int32, device=device))
    out, kept = block.forward(*args)
    dout = (torch.randn(out.shape, generator=g, device=device) * 0.01).to(out.dtype)
    dx = block.backward(dout, kept)
    first.backward(dx, ids)

    def profile(layer, forward, backward, kept_bytes, plain_bytes):
        work = max(_work_bytes(forward, device), _work_bytes(backward, device))
        return LayerProfile(_median_us(forward, repeats), _median_us(backward, repeats), layer.weight_bytes, kept_bytes,
                            plain_bytes, work)

    profiles = (profile(first, lambda: first.forward(ids), lambda: first.backward(dx, ids), ids.numel() * 4, ids.numel() * 4),
                profile(block, lambda: block.forward(*args), lambda: block.backward(dout, kept), kept.kept_bytes, kept.plain_bytes))
    return profiles if keep_8_bits else tuple(p.in_16_bits() for p in profiles)


def plan_problem(first: LayerProfile, block: LayerProfile, blocks: int, stages: int, micro_batches: int, *,
                 slower=(1.0, 1.7), caps_mb=(65536, 65536), link_us: int = 100, assign: Optional[np.ndarray] = None) -> Problem:
    """The planner's tables for an embedding and `blocks` expert blocks: times on each device type (`slower`: times this
    GPU's), memory of a layer = weights, their gradients and what min(stages, micro_batches) micro-batches in flight
    keep.  A device runs one pass at a time, so its cap is less what the largest works with."""
    profiles = [first] + [block] * blocks
    flight = min(stages, micro_batches)
    fwd, bwd = (np.array([[max(1, round(getattr(p, name) * s)) for p in profiles] for s in slower], np.uint32)
                for name in ("fwd_us", "bwd_us"))
    mem = np.array([-(-(p.weight_bytes + flight * p.kept_bytes) // 10 ** 6) for p in profiles], np.uint32)
    work = -(-max(p.work_bytes for p in profiles) // 10 ** 6)
    caps = np.array([max(0, cap - work) for cap in caps_mb], np.uint32)
    comm = np.full(stages - 1, link_us, np.uint32)
    return Problem(len(profiles), stages, micro_batches, len(slower), fwd, bwd, comm, comm, mem, caps,
                   assign)


def main() -> None:
    ap = argparse.ArgumentParser(description="Measure layers on this GPU and search for the best pipeline of them.")
    ap.add_argument("--tokens", type=int, default=4096, help="tokens of a micro-batch")
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--chosen", type=int, default=2)
    ap.add_argument("--inner", type=int, default=2048)
    ap.add_argument("--heads", type=int, default=0, help="heads of attention before the experts (default: none)")
    ap.add_argument("--kv-heads", type=int, default=0, help="heads of its keys (default: as many)")
    ap.add_argument("--sequence", type=int, default=0, help="tokens of a sequence (default: all of a micro-batch)")
    ap.add_argument("--blocks", type=int, default=23)
    ap.add_argument("--stages", type=int, default=4)
    ap.add_argument("--micro-batches", type=int, default=32)
    ap.add_argument("--cap-mb", type=int, default=0,
                    help="memory of a device (default: 5%% above an even share, and what a pass works with)")
    a = ap.parse_args()
    shape = Shape(width=a.width, experts=a.experts, chosen=a.chosen, inner=a.inner, tokens=a.tokens,
                  heads=a.heads, kv_heads=a.kv_heads, sequence=a.sequence)
    if shape.heads:
        try:
            key_heads(shape)
        except ValueError as e:
            ap.error(str(e))
    first, eight = measure(shape)
    cap = a.cap_mb or int(1.05 * -(-a.blocks // a.stages) *
                          (eight.weight_bytes + min(a.stages, a.micro_batches) * eight.kept_bytes) / 1e6 +
                          eight.work_bytes / 1e6)
    for kept, block in (("8 bits", eight), ("16 bits (memory alone, times of 8 bits)", eight.in_16_bits())):
        prob = plan_problem(first, block, a.blocks, a.stages, a.micro_batches, caps_mb=(cap, cap))
        ctx = P.poseidon_load_costs(prob, torch.cuda.current_device())
        best, _ = P.poseidon_search(ctx, rows_per_chunk=64, ramp=True)
        ctx.close()
        found = f"best plan {best.index}, {best.makespan} us a step" if best.index is not None else "no plan fits"
        print(f"activations in {kept}: block {block.fwd_us:.0f} + {block.bwd_us:.0f} us, keeps "
              f"{block.kept_bytes / 1e6:.1f} MB of a micro-batch, works with "
              f"{block.work_bytes / 1e6:.1f} MB; devices of {cap} MB: {found}", flush=True)


if __name__ == "__main__":
    main()
