"""A worker that pretrains a model of the workloads' shapes: forward and backward pass on the library's operators (operators.py), every
layer's synchronisation and update overlapped with the backward pass (overlap.BackwardOverlap), the loss from the hidden states
without logits in memory.  Projections are plain matrix products (torch).

    python -m paper_2502_11058_amd.pretrain [--config small_llama | tiny_gpt2 | gpt2_small | tinyllama_1b] [--batch 4] [--tokens 256] [--iterations 8]

Tokens are synthetic: a random walk over the vocabulary that the model can learn.  The peers' buffers stand for N - 1 workers that
have drifted from this one (Gaussian, as in the benchmark).  Llama-shaped workloads: root-mean-square norm, rotary positions, shared key heads,
gated feed-forward block.  GPT-2-shaped: layer norm, learned positions, the embedding as the head: one parameter, whose gradient autograd
adds up from both uses before its hook fires, behind the last kernel that reads it.
"""
from __future__ import annotations

import argparse
import time
from dataclasses import dataclass
from typing import Callable, Dict, List

import torch
import torch.nn.functional as F

from . import operators as O
from . import workloads as W
from .harness import DeviceReplica
from .overlap import BackwardOverlap


@dataclass
class Model:
    """The dimensions that a workload's tensors have, and the norms' weights among them."""
    family: str
    blocks: int
    width: int
    heads: int
    kv_heads: int
    vocab: int
    context: int
    workload: W.Workload

    def loss(self, p: Dict[str, torch.Tensor], tokens: torch.Tensor, targets: torch.Tensor, table=None, ops=O) -> torch.Tensor:
        """Mean cross entropy of tokens [batch, tokens]; p: flat tensors by their names.  `ops`: the operators' module."""
        b, t = tokens.shape
        d, hd = self.width, self.width // self.heads
        kv = self.kv_heads * hd
        if self.family == "llama":
            x = F.embedding(tokens, p["embed_tokens"].view(-1, d))
            for i in range(self.blocks):
                q = f"layers.{i}."
                h = ops.norm(x, p[q + "input_layernorm"], kind="rms")
                query, key, value = (F.linear(h, p[q + n].view(-1, d)).view(b, t, -1, hd) for n in ("q_proj", "k_proj", "v_proj"))
                query, key = ops.rotary(query, key, table)
                x = x + F.linear(ops.attention(query, key, value).reshape(b, t, d), p[q + "o_proj"].view(d, d))
                h = ops.norm(x, p[q + "post_attention_layernorm"], kind="rms")
                gate, up = (F.linear(h, p[q + n].view(-1, d)) for n in ("gate_proj", "up_proj"))
                x = x + F.linear(F.silu(gate) * up, p[q + "down_proj"].view(d, -1))
            return ops.linear_cross_entropy(ops.norm(x, p["norm"], kind="rms"), p["lm_head"].view(-1, d), targets)
        embedding = p["wte"].view(-1, d)
        x = F.embedding(tokens, embedding) + p["wpe"].view(-1, d)[:t]
        for i in range(self.blocks):
            q = f"h.{i}."
            h = ops.norm(x, p[q + "ln_1.weight"], p[q + "ln_1.bias"])
            # queries, keys and values are parts of one projection's output
            query, key, value = F.linear(h, p[q + "attn.c_attn.weight"].view(-1, d)).view(b, t, 3, self.heads, hd).unbind(2)
            x = x + F.linear(ops.attention(query, key, value).reshape(b, t, d), p[q + "attn.c_proj.weight"].view(d, d))
            h = ops.norm(x, p[q + "ln_2.weight"], p[q + "ln_2.bias"])
            x = x + F.linear(F.gelu(F.linear(h, p[q + "mlp.c_fc.weight"].view(-1, d))), p[q + "mlp.c_proj.weight"].view(d, -1))
        return ops.linear_cross_entropy(x, embedding, targets)

    def norm_weights(self) -> List[int]:
        return [i for i, s in enumerate(self.workload.tensors) if "norm" in s.name or s.name.endswith(("ln_1.weight", "ln_2.weight"))]

    def table(self, device) -> torch.Tensor:
        return O.rotary_table(self.context, self.width // self.heads, device=device) if self.family == "llama" else None


def _llama(w: W.Workload, heads: int, kv_heads: int, context: int = 4096) -> Model:
    numel = {s.name: s.numel for s in w.tensors}
    d = numel["norm"]
    return Model("llama", sum(s.name.endswith("q_proj") for s in w.tensors), d, heads, kv_heads, numel["lm_head"] // d, context, w)


def _gpt2(w: W.Workload, heads: int) -> Model:
    numel = {s.name: s.numel for s in w.tensors}
    d = numel["h.0.ln_1.weight"]
    return Model("gpt2", sum(s.name.endswith("ln_1.weight") for s in w.tensors), d, heads, heads, numel["wte"] // d, numel["wpe"] // d, w)


def _tiny_gpt2() -> Model:
    c = dict(W.load_config("gpt2_small"), n_blocks=2, d=128, ffn=512, vocab=1009, context=256, n_replicas=4, period=2)
    return _gpt2(W.from_config("tiny_gpt2", c), 2)


def _of_config(name: str) -> Callable[[], Model]:
    def make() -> Model:
        c = W.load_config(name)
        return _llama(W.get(name), int(c["n_heads"]), int(c["n_kv"])) if c["family"] == "llama" else _gpt2(W.get(name), int(c["d"]) // 64)
    return make


MODELS: Dict[str, Callable[[], Model]] = {
    "small_llama": lambda: _llama(W.small_llama(), 8, 2),
    "tiny_gpt2": _tiny_gpt2,
    "gpt2_small": _of_config("gpt2_small"),
    "tinyllama_1b": _of_config("tinyllama_1b"),
    "llama2_7b": _of_config("llama2_7b"),
    "llama3_8b": _of_config("llama3_8b"),
}


def walk(g: torch.Generator, vocab: int, batch: int, tokens: int, device) -> torch.Tensor:
    """[batch, tokens + 1]: each token is a small step from the one before, so that there is something to learn."""
    steps = torch.randint(1, 4, (batch, tokens + 1), generator=g, device=device)
    steps[:, 0] = torch.randint(0, vocab, (batch,), generator=g, device=device)
    return steps.cumsum(1) % vocab


class Pretraining:
    """One worker: its state in HBM, the model over it, and an iteration."""

    def __init__(self, model: Model, device: int = 0, seed: int = 1234, side_cus: int = 0):
        self.model, self.rep = model, DeviceReplica(model.workload, device, placement_probe=False)
        rep = self.rep
        rep.init_params()
        for i in model.norm_weights():
            rep.sync[i].fill_(1.0)
            if rep.bf16:
                rep.model[i].fill_(1.0)
        self.overlap = BackwardOverlap(rep, side_cus=side_cus)
        self.params = {s.name: p for s, p in zip(model.workload.tensors, self.overlap.params)}
        self.table = model.table(rep.dev)
        self.generator = torch.Generator(device=rep.dev)
        self.generator.manual_seed(seed)

    def batch(self, batch: int, tokens: int):
        seq = walk(self.generator, self.model.vocab, batch, tokens, self.rep.dev)
        return seq[:, :-1].contiguous(), seq[:, 1:].contiguous()

    def peers(self, r: int) -> None:
        """The peers' buffers of iteration r's slot: this worker's parameters and a drift."""
        rep = self.rep
        slot = r % len(rep.sets)
        rep.ctx.ddp_pack(slot, rep.flat)
        rep.fill_peers_from(rep.flat, r, rep.ctx.ddp_slot_numel(slot))

    def iteration(self, r: int, tokens: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """Behind what the current stream holds (tokens, peers' buffers), on the worker's own stream; what comes on the current stream
        afterwards is behind it.  -> the loss, for the current stream."""
        ov = self.overlap
        caller = torch.cuda.current_stream(self.rep.dev)
        ov.main_stream.wait_stream(caller)
        with torch.cuda.stream(ov.main_stream):
            ov.begin(r, with_stats=False)
            loss = self.model.loss(self.params, tokens, targets, self.table)
            ov.backward(loss)
            ov.end()
        caller.wait_stream(ov.main_stream)
        loss = loss.detach()
        loss.record_stream(caller)
        return loss

    def close(self) -> None:
        self.overlap.close()
        self.rep.close()


def main() -> None:
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--config", choices=sorted(MODELS), default="small_llama")
    a.add_argument("--batch", type=int, default=4)
    a.add_argument("--tokens", type=int, default=256)
    a.add_argument("--iterations", type=int, default=8)
    a = a.parse_args()
    model = MODELS[a.config]()
    if not 0 < a.tokens <= model.context:
        raise SystemExit(f"--tokens has to be in [1, {model.context}]")
    worker = Pretraining(model)
    for r in range(a.iterations):
        tokens, targets = worker.batch(a.batch, a.tokens)
        worker.peers(r)
        torch.cuda.synchronize()
        t = time.perf_counter()
        loss = worker.iteration(r, tokens, targets)
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        print(f"iteration {r}: loss {loss.item():.4f}, {1e3 * t:.2f} ms, {a.batch * a.tokens / t:.0f} tokens/s", flush=True)
    worker.close()


if __name__ == "__main__":
    main()
