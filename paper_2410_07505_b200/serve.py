"""An attention layer served from quantized weights and a quantized cache: the serving operators as they are used together.

    python -m paper_2410_07505_b200.serve [--hidden 4096] [--heads 32] [--kv-heads 8] [--prompt 1000] [--steps 16] [--bits 8|4]

`AttentionLayer` holds two block-quantized projections (`cq.Fp8Weight`) and a paged cache (`cq.KVCache`).  The prompt
calibrates the cache: the channel factors are the CrossQuant column factors c_j^(1 - alpha) of its keys and values
(Section 4.2, `cq.absmax_cols`), fixed from then on.  `prompt` fills the cache and attends over the tokens read back from it;
`step` appends one token for every sequence and attends with the kernel that reads the codes.
"""
from __future__ import annotations

import argparse
import math
import time

import torch

from . import cq


class AttentionLayer:
    def __init__(self, w_qkv: torch.Tensor, w_out: torch.Tensor, heads: int, kv_heads: int, *, sequences: int, longest: int,
                 bits: int = 8, page_size: int = 64, alpha: float = 0.15):
        """w_qkv [(heads + 2 kv_heads) * D, hidden], w_out [hidden, heads * D], both 16-bit on the GPU.
        A sequence has room for `longest` tokens, rounded up to whole pages."""
        self.heads, self.kv_heads, self.alpha, self.bits, self.page_size = heads, kv_heads, alpha, bits, page_size
        self.head_dim = w_out.shape[1] // heads
        self.w_qkv, self.w_out = cq.fp8_quantize_weight(w_qkv), cq.fp8_quantize_weight(w_out)
        per_seq = -(-longest // page_size)
        dev = w_qkv.device
        # behind the last page stands one that is none, for positions beyond it
        self._pages = torch.full((sequences, per_seq + 1), -1, dtype=torch.int32, device=dev)
        self.page_table = self._pages[:, :per_seq]
        self.page_table.copy_(torch.arange(sequences * per_seq, dtype=torch.int32, device=dev).view(sequences, per_seq))
        self.lens = torch.zeros(sequences, dtype=torch.int32, device=dev)
        self._room, self._filled = per_seq * page_size, [0] * sequences      # tokens of each sequence, as the host knows them
        self.cache = None

    def _split(self, x: torch.Tensor):
        """(queries, keys, values) [T, heads, D] of tokens x [T, hidden]: slices of one product."""
        qkv = cq.fp8_linear(x, self.w_qkv).view(x.shape[0], self.heads + 2 * self.kv_heads, self.head_dim)
        return qkv.split((self.heads, self.kv_heads, self.kv_heads), dim=1)

    def _slots(self, seq: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
        """Slots of positions; below 0, which the cache skips, for those beyond a sequence's last page."""
        page = self._pages[seq, (pos // self.page_size).clamp_(max=self._pages.shape[1] - 1)].long()
        return page * self.page_size + pos % self.page_size

    def _calibrate(self, k: torch.Tensor, v: torch.Tensor) -> None:
        shape = (self.kv_heads, self.head_dim)
        # (c_j^(1 - alpha); 1 for a channel of which the prompt says nothing: a factor of 0 would drop what later tokens hold there)
        top = [cq.absmax_cols(x.reshape(x.shape[0], -1)).view(shape) for x in (k, v)]
        col = [torch.where((c > 0) & torch.isfinite(c), c.pow(1.0 - self.alpha), 1.0) for c in top]
        self.cache = cq.KVCache.empty(self.page_table.numel(), self.page_size, *shape, self.bits, k_col=col[0], v_col=col[1],
                                      device=k.device)

    def prompt(self, x: torch.Tensor, seq: int) -> torch.Tensor:
        """The prompt x [T, hidden] of sequence `seq`; the layer's outputs [T, hidden].  What the sequence held is replaced."""
        T, seq = x.shape[0], range(len(self._filled))[seq]
        if not 1 <= T <= self._room:
            raise ValueError(f"a prompt of {T} tokens: a sequence holds 1 to {self._room}")
        q, k, v = self._split(x)
        if self.cache is None:
            self._calibrate(k, v)
        pos = torch.arange(T, device=x.device)
        slots = self._slots(torch.full_like(pos, seq), pos)
        cq.kv_write(self.cache, k, v, slots)
        self.lens[seq] = T
        self._filled[seq] = T
        k, v = cq.kv_read(self.cache, slots, x.dtype)               # what later tokens will see of the prompt
        G = self.heads // self.kv_heads
        logits = torch.einsum("ihgd,jhd->hgij", q.view(T, self.kv_heads, G, -1).float(), k.float()) / math.sqrt(self.head_dim)
        logits = logits.masked_fill(pos[None, :] > pos[:, None], -math.inf)
        out = torch.einsum("hgij,jhd->ihgd", logits.softmax(-1), v.float()).to(x.dtype)
        return cq.fp8_linear(out.reshape(T, -1), self.w_out)

    def step(self, x: torch.Tensor) -> torch.Tensor:
        """One token for every sequence, x [sequences, hidden]; the layer's outputs [sequences, hidden]."""
        B = x.shape[0]
        if B != len(self._filled):
            raise ValueError(f"{B} tokens for {len(self._filled)} sequences")
        if self.cache is None:
            raise ValueError("a step before any prompt: the prompt calibrates the cache")
        if max(self._filled) >= self._room:
            raise ValueError(f"a sequence has its {self._room} tokens already")
        q, k, v = self._split(x)
        pos = self.lens.long()
        cq.kv_write(self.cache, k, v, self._slots(torch.arange(B, device=x.device), pos))
        self.lens += 1
        self._filled = [n + 1 for n in self._filled]
        out = cq.kv_attention(q.unsqueeze(1), self.cache, self.page_table, self.lens)
        return cq.fp8_linear(out.view(B, -1), self.w_out)


def plain_layer(x: torch.Tensor, w_qkv: torch.Tensor, w_out: torch.Tensor, heads: int, kv_heads: int) -> torch.Tensor:
    """The same layer on one whole sequence in 64 bits, nothing quantized: what the quantized one is compared with."""
    D = w_out.shape[1] // heads
    T, G = x.shape[0], heads // kv_heads
    q, k, v = (x.double() @ w_qkv.double().t()).view(T, heads + 2 * kv_heads, D).split((heads, kv_heads, kv_heads), dim=1)
    logits = torch.einsum("ihgd,jhd->hgij", q.reshape(T, kv_heads, G, D), k) / math.sqrt(D)
    pos = torch.arange(T, device=x.device)
    logits = logits.masked_fill(pos[None, :] > pos[:, None], -math.inf)
    out = torch.einsum("hgij,jhd->ihgd", logits.softmax(-1), v)
    return out.reshape(T, -1) @ w_out.double().t()


def demo(hidden: int, heads: int, kv_heads: int, prompt: int, steps: int, bits: int, sequences: int = 2, seed: int = 0) -> dict:
    """Random weights and tokens through the layer; its error against `plain_layer` and the time of a step."""
    D = hidden // heads
    gen = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    w_qkv = (draw((heads + 2 * kv_heads) * D, hidden) / math.sqrt(hidden)).bfloat16()
    w_out = (draw(hidden, heads * D) / math.sqrt(heads * D)).bfloat16()
    layer = AttentionLayer(w_qkv, w_out, heads, kv_heads, sequences=sequences, longest=prompt + steps, bits=bits)
    tokens = draw(sequences, prompt + steps, hidden).bfloat16()
    got = [[layer.prompt(tokens[b, :prompt], b)] for b in range(sequences)]
    torch.cuda.synchronize()
    began = time.perf_counter()
    for i in range(steps):
        out = layer.step(tokens[:, prompt + i].contiguous())
        for b in range(sequences):
            got[b].append(out[b:b + 1])
    torch.cuda.synchronize()
    took = time.perf_counter() - began
    if cq.serve_fault():
        raise RuntimeError("a bounded wait gave up in one of the kernels: the results are not to be used")
    err = {}
    for part, at in (("prompt", slice(0, prompt)), ("steps", slice(prompt, None))):
        off = ref = 0.0
        for b in range(sequences):
            want = plain_layer(tokens[b], w_qkv, w_out, heads, kv_heads)[at]
            off += float((torch.cat(got[b])[at].double() - want).square().sum())
            ref += float(want.square().sum())
        err[part] = math.sqrt(off / ref)
    return {"relative_error_prompt": err["prompt"], "relative_error_steps": err["steps"], "us_per_step": took / steps * 1e6}


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--bits", type=int, default=8, choices=(4, 8))
    a = ap.parse_args()
    r = demo(a.hidden, a.heads, a.kv_heads, a.prompt, a.steps, a.bits)
    print(f"INT{a.bits} cache, e4m3 weights: relative error {r['relative_error_prompt']:.4f} (prompt), {r['relative_error_steps']:.4f} (steps); "
          f"{r['us_per_step']:.0f} us a step")


if __name__ == "__main__":
    main()
