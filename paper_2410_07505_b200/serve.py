"""An attention layer served from quantized weights and a quantized cache: the serving operators as they are used together.

    python -m paper_2410_07505_b200.serve [--hidden 4096] [--heads 32] [--kv-heads 8] [--prompt 1000] [--steps 16] [--bits 8|4]
                                          [--rotate] [--adapter-rank R]

`AttentionLayer` holds two block-quantized projections (`cq.Fp8Weight`) and a paged cache (`cq.KVCache`).  The prompt
calibrates the cache: the channel factors are the CrossQuant column factors c_j^(1 - alpha) of its keys and values
(Section 4.2, `cq.absmax_cols`), fixed from then on.  `prompt` (`prompts` for several at once) fills the cache and attends over
the tokens read back from it; `step` appends one token for every sequence and attends with the kernel that reads the codes.
On request queries and keys are normalised for each head and rotated by their positions before the cache sees them
(`cq.norm_rotate`), and each sequence has a low-rank adapter of its own beside the projections (`cq.adapter_add`).
"""
from __future__ import annotations

import argparse
import math
import time

import torch

from . import cq


class AttentionLayer:
    def __init__(self, w_qkv: torch.Tensor, w_out: torch.Tensor, heads: int, kv_heads: int, *, sequences: int, longest: int,
                 bits: int = 8, page_size: int = 64, alpha: float = 0.15, freq: torch.Tensor | None = None, eps: float | None = None,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, neighbours: bool = False,
                 qkv_adapters=None, out_adapters=None, fine_prompts: bool = True):
        """w_qkv [(heads + 2 kv_heads) * D, hidden], w_out [hidden, heads * D], both 16-bit on the GPU.
        A sequence has room for `longest` tokens, rounded up to whole pages.

        `freq` (float64, `cq.rotation_freq`) turns the rotation on, `eps` the norms, with the weights if they are given; the adapters
        (`cq.Adapters` of either projection) are chosen for each prompt.  `fine_prompts` = False lets a prompt's attention round its weights to
        16 bits (the faster `cq.prompt_attention`)."""
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
        if eps is None and (q_weight is not None or k_weight is not None):
            raise ValueError("weights belong to the norms: eps is None")
        self._turn = None
        if freq is not None or eps is not None:
            if freq is None:                                            # norms alone: no channel is rotated
                freq = torch.empty(0, dtype=torch.float64, device=dev)
            self._turn = (freq, q_weight, k_weight, eps, neighbours)
        self.qkv_adapters, self.out_adapters, self.fine_prompts = qkv_adapters, out_adapters, fine_prompts
        self.adapter = torch.full((sequences,), -1, dtype=torch.int32, device=dev)      # of each sequence; below 0: none

    def _project(self, x: torch.Tensor, w, adapters, adapter: torch.Tensor) -> torch.Tensor:
        y = cq.fp8_linear(x, w)
        return y if adapters is None else cq.adapter_add(y, x, adapters, adapter, out=y)

    def _split(self, x: torch.Tensor, pos: torch.Tensor, adapter: torch.Tensor):
        """(queries, keys, values) [T, heads, D] of tokens x [T, hidden] at positions pos: slices of one product."""
        qkv = self._project(x, self.w_qkv, self.qkv_adapters, adapter).view(x.shape[0], self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), dim=1)
        if self._turn is not None:
            freq, q_weight, k_weight, eps, neighbours = self._turn
            q, k = cq.norm_rotate(q, k, pos, freq, q_weight, k_weight, eps=eps, neighbours=neighbours, out=(q, k))
        return q, k, v

    def _attend(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lengths) -> torch.Tensor:
        """Causal attention of packed prompts over their own tokens."""
        if q.is_cuda:
            ends = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
            starts = torch.cat([torch.full((1,), n, dtype=torch.int32, device=q.device) for n in ends])      # (no copy from the host)
            return cq.prompt_attention(q, k, v, starts, fine=self.fine_prompts)
        G, outs = self.heads // self.kv_heads, []                       # on the host, in elementary operations
        for q, k, v in zip(q.split(lengths), k.split(lengths), v.split(lengths)):
            T = q.shape[0]
            logits = torch.einsum("ihgd,jhd->hgij", q.reshape(T, self.kv_heads, G, -1).float(), k.float()) / math.sqrt(self.head_dim)
            logits = logits.masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), -math.inf)
            outs.append(torch.einsum("hgij,jhd->ihgd", logits.softmax(-1), v.float()).reshape(T, self.heads, -1).to(q.dtype))
        return torch.cat(outs)

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

    def prompt(self, x: torch.Tensor, seq: int, adapter: int = -1) -> torch.Tensor:
        """The prompt x [T, hidden] of sequence `seq`; the layer's outputs [T, hidden].  What the sequence held is replaced."""
        return self.prompts(x, [seq], [x.shape[0]], [adapter])

    def prompts(self, x: torch.Tensor, seqs, lengths, adapters=None) -> torch.Tensor:
        """Prompts of several sequences, packed: the first lengths[0] rows of x are that of sequence seqs[0], and so on;
        `adapters`: which adapter each sequence has from now on (outside their range, as by default: none)."""
        seqs = [range(len(self._filled))[s] for s in seqs]
        adapters = [-1] * len(seqs) if adapters is None else list(adapters)
        if len(set(seqs)) != len(seqs) or not len(seqs) == len(lengths) == len(adapters) or sum(lengths) != x.shape[0]:
            raise ValueError("prompts of different sequences, whose lengths make up the rows of x")
        if not seqs:
            raise ValueError("no prompt")
        for T in lengths:
            if not 1 <= T <= self._room:
                raise ValueError(f"a prompt of {T} tokens: a sequence holds 1 to {self._room}")
        if any(a >= 0 for a in adapters) and self.qkv_adapters is None and self.out_adapters is None:
            raise ValueError("the layer has no adapters")
        dev = x.device
        pos = torch.cat([torch.arange(T, device=dev) for T in lengths])
        of = torch.cat([torch.full((T,), s, dtype=torch.long, device=dev) for s, T in zip(seqs, lengths)])
        chosen = torch.cat([torch.full((T,), a, dtype=torch.int32, device=dev) for a, T in zip(adapters, lengths)])
        q, k, v = self._split(x, pos, chosen)
        if self.cache is None:
            self._calibrate(k, v)
        slots = self._slots(of, pos)
        cq.kv_write(self.cache, k, v, slots)
        for s, T, a in zip(seqs, lengths, adapters):
            self.lens[s].fill_(T)                                   # (no copy from the host: the call can be captured)
            self.adapter[s].fill_(a)
            self._filled[s] = T
        k, v = cq.kv_read(self.cache, slots, x.dtype)               # what later tokens will see of the prompt
        out = self._attend(q, k, v, list(lengths))
        return self._project(out.reshape(x.shape[0], -1), self.w_out, self.out_adapters, chosen)

    def step(self, x: torch.Tensor) -> torch.Tensor:
        """One token for every sequence, x [sequences, hidden]; the layer's outputs [sequences, hidden]."""
        B = x.shape[0]
        if B != len(self._filled):
            raise ValueError(f"{B} tokens for {len(self._filled)} sequences")
        if self.cache is None:
            raise ValueError("a step before any prompt: the prompt calibrates the cache")
        if max(self._filled) >= self._room:
            raise ValueError(f"a sequence has its {self._room} tokens already")
        pos = self.lens.long()
        q, k, v = self._split(x, pos, self.adapter)
        cq.kv_write(self.cache, k, v, self._slots(torch.arange(B, device=x.device), pos))
        self.lens += 1
        self._filled = [n + 1 for n in self._filled]
        out = cq.kv_attention(q.unsqueeze(1), self.cache, self.page_table, self.lens)
        return self._project(out.view(B, -1), self.w_out, self.out_adapters, self.adapter)


def plain_layer(x: torch.Tensor, w_qkv: torch.Tensor, w_out: torch.Tensor, heads: int, kv_heads: int, *, freq: torch.Tensor | None = None,
                eps: float | None = None) -> torch.Tensor:
    """The same layer on one whole sequence in 64 bits, nothing quantized: what the quantized one is compared with (an
    adapter is part of its weights here; norms without weights, channels i and i + R / 2 rotated)."""
    D = w_out.shape[1] // heads
    T, G = x.shape[0], heads // kv_heads
    q, k, v = (x.double() @ w_qkv.double().t()).view(T, heads + 2 * kv_heads, D).split((heads, kv_heads, kv_heads), dim=1)
    if eps is not None:
        q, k = (t / torch.sqrt(t.square().mean(-1, keepdim=True) + eps) for t in (q, k))
    if freq is not None:
        half = freq.shape[0]
        f = torch.arange(T, device=x.device)[:, None].double() * freq
        cos, sin = f.cos()[:, None], f.sin()[:, None]
        q, k = (torch.cat((t[..., :half] * cos - t[..., half:2 * half] * sin, t[..., :half] * sin + t[..., half:2 * half] * cos, t[..., 2 * half:]), dim=-1)
                for t in (q, k))
    logits = torch.einsum("ihgd,jhd->hgij", q.reshape(T, kv_heads, G, D), k) / math.sqrt(D)
    pos = torch.arange(T, device=x.device)
    logits = logits.masked_fill(pos[None, :] > pos[:, None], -math.inf)
    out = torch.einsum("hgij,jhd->ihgd", logits.softmax(-1), v)
    return out.reshape(T, -1) @ w_out.double().t()


def demo(hidden: int, heads: int, kv_heads: int, prompt: int, steps: int, bits: int, sequences: int = 2, seed: int = 0, rotate: bool = False,
         adapter_rank: int = 0) -> dict:
    """Random weights and tokens through the layer; its error against `plain_layer` and the time of a step.  With `rotate`
    queries and keys are normalised and rotated; with an adapter rank every sequence but the first has an adapter."""
    D = hidden // heads
    gen = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    wide = (heads + 2 * kv_heads) * D
    w_qkv = (draw(wide, hidden) / math.sqrt(hidden)).bfloat16()
    w_out = (draw(hidden, heads * D) / math.sqrt(heads * D)).bfloat16()
    more, plain = {}, {}
    if rotate:
        more = plain = dict(freq=cq.rotation_freq(D), eps=1e-6)
    tokens = draw(sequences, prompt + steps, hidden).bfloat16()
    if adapter_rank:
        pairs = [cq.Adapters((draw(sequences, adapter_rank, w.shape[1]) / math.sqrt(w.shape[1])).bfloat16(),
                             (draw(sequences, w.shape[0], adapter_rank) / math.sqrt(adapter_rank)).bfloat16(),
                             torch.full((sequences,), 0.5, device="cuda")) for w in (w_qkv, w_out)]
        more = dict(more, qkv_adapters=pairs[0], out_adapters=pairs[1])
    layer = AttentionLayer(w_qkv, w_out, heads, kv_heads, sequences=sequences, longest=prompt + steps, bits=bits, **more)
    chosen = [b - 1 if adapter_rank else -1 for b in range(sequences)]
    got = [[layer.prompt(tokens[b, :prompt], b, chosen[b])] for b in range(sequences)]
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
            w = [w_qkv.double(), w_out.double()]
            if chosen[b] >= 0:
                w = [m + float(p.scale[chosen[b]]) * (p.B[chosen[b]].double() @ p.A[chosen[b]].double()) for m, p in zip(w, pairs)]
            want = plain_layer(tokens[b], *w, heads, kv_heads, **plain)[at]
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
    ap.add_argument("--rotate", action="store_true", help="norms and position rotation of queries and keys")
    ap.add_argument("--adapter-rank", type=int, default=0, help="a low-rank adapter for every sequence but the first")
    a = ap.parse_args()
    r = demo(a.hidden, a.heads, a.kv_heads, a.prompt, a.steps, a.bits, rotate=a.rotate, adapter_rank=a.adapter_rank)
    print(f"INT{a.bits} cache, e4m3 weights: relative error {r['relative_error_prompt']:.4f} (prompt), {r['relative_error_steps']:.4f} (steps); "
          f"{r['us_per_step']:.0f} us a step")


if __name__ == "__main__":
    main()
