"""A decoder with compressed linear layers, end to end: tokens in, logits out, one new token per sequence and step.

Every layer is one of two kinds, as in the text decoders of the LLaMA-3.2 vision models: self-attention over a paged
key-value cache, or attention to the states of an image (with normalised queries and keys, and gates).  All products run on
dictionary-coded weights (tq_fused_gemv_stack; tq_fused_gemm_ws for the image's keys and values); between them are
tq_rmsnorm, tq_rope_append, tq_paged_attention and tq_cross_attention, each reading what the product before it wrote
(fp32) and writing what the next one reads (bf16).  Weights are random.

    python examples/vision_decoder.py [--model 1b|3b|11b|90b --layers N] [--steps N] [--batch N] [--check]
"""
from __future__ import annotations

import argparse
import math
import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from inputs import synth  # noqa: E402
from paper_2509_22951_b200 import binding as tq  # noqa: E402

EPS = 1e-5


@dataclass
class Config:
    hidden: int = 256
    heads: int = 8
    kv_heads: int = 2
    dim: int = 64
    ffn: int = 512
    vocab: int = 1024
    layers: str = "scs"    # s: self-attention, c: attention to the image
    page: int = 16
    max_tokens: int = 256  # per sequence
    tiles: int = 2         # of an image
    patches: int = 100     # states of a tile
    theta: float = 500000.0

    @staticmethod
    def named(model: str, layers: int) -> "Config":
        shapes = {n.split(".")[-1]: (o, i) for n, o, i in synth.llama32_linear_shapes(model, 1)}
        dim = 64 if model == "1b" else 128
        return Config(hidden=shapes["q"][1], heads=shapes["q"][0] // dim, kv_heads=shapes["k"][0] // dim, dim=dim, ffn=shapes["gate"][0],
                      vocab=shapes["lm_head"][0], layers=("sssc" * layers)[:layers], max_tokens=4096, tiles=4, patches=1601)


class Decoder:
    """Weights, cache and buffers of `batch` sequences."""

    def __init__(self, cfg: Config, batch: int, seed: int = 0):
        self.cfg, self.batch = cfg, batch
        c, h, qd, kd = cfg, cfg.hidden, cfg.heads * cfg.dim, cfg.kv_heads * cfg.dim
        names, levels, scales = [], [], []
        for n in range(len(c.layers)):
            for name, rows, cols in (("q", qd, h), ("k", kd, h), ("v", kd, h), ("o", h, qd), ("gate", c.ffn, h), ("up", c.ffn, h), ("down", h, c.ffn)):
                names.append(f"l{n}.{name}")
                lv, sc = tq.tq_quantize_rows_device(synth.weight(rows, cols, synth.matrix_seed(len(names) + 1000 * seed), device="cuda"))
                levels.append(lv), scales.append(sc)
        names.append("head")
        lv, sc = tq.tq_quantize_rows_device(synth.weight(c.vocab, h, synth.matrix_seed(999 + 1000 * seed), device="cuda"))
        levels.append(lv), scales.append(sc)
        table = tq.tq_dict_upload(tq.tq_build_dictionary_device(levels))
        self.mats = {n: tq.tq_upload_device(table, lv, sc) for n, lv, sc in zip(names, levels, scales)}
        self.dense = dict(zip(names, zip(levels, scales)))  # for the check
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.embed = torch.randn(c.vocab, h, generator=g, device="cuda").to(torch.bfloat16)
        norm = lambda n: 1 + 0.1 * torch.randn(n, generator=g, device="cuda")  # noqa: E731
        self.norms = {f"l{n}.{k}": norm(h) for n in range(len(c.layers)) for k in ("attn", "mlp")}
        self.norms |= {f"l{n}.{k}": norm(c.dim) for n in range(len(c.layers)) for k in ("qn", "kn")}
        self.norms["head"] = norm(h)
        self.gates = [0.5 + 0.1 * n for n in range(len(c.layers))]

        f = c.theta ** (-torch.arange(0, c.dim, 2, dtype=torch.float64, device="cuda") / c.dim)
        a = torch.arange(c.max_tokens, dtype=torch.float64, device="cuda")[:, None] * f
        self.rope = torch.cat([a.cos(), a.sin()], 1).float()

        per = -(-c.max_tokens // c.page)
        pages = batch * per
        self.pages = torch.randperm(pages, generator=g, device="cuda").int().view(batch, per).contiguous()
        new = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.caches = {n: tq.tq_kv_cache(new(pages, c.kv_heads, c.page, c.dim), new(pages, c.kv_heads, c.page, c.dim))
                       for n, kind in enumerate(c.layers) if kind == "s"}
        self.workspace = tq.tq_attn_workspace()
        self.image = {}  # layer -> keys, values
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.steps = 0  # tokens of every sequence, on the host
        self.tile_mask = None

        # operands of the products and the products that can run together
        f32 = lambda n: torch.empty(batch, n, device="cuda")  # noqa: E731
        bf = lambda n: torch.empty(batch, n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.x, self.a, self.act = bf(h), bf(qd), bf(c.ffn)
        self.q, self.k, self.v, self.o, self.gate, self.up, self.down = f32(qd), f32(kd), f32(kd), f32(h), f32(c.ffn), f32(c.ffn), f32(h)
        self.logits = f32(c.vocab)
        m = self.mats
        self.stacks = []
        for n, kind in enumerate(c.layers):
            first = tq.tq_stack_create([m[f"l{n}.q"], m[f"l{n}.k"], m[f"l{n}.v"]], [self.x] * 3, [self.q, self.k, self.v]) if kind == "s" else \
                tq.tq_stack_create([m[f"l{n}.q"]], [self.x], [self.q])
            self.stacks.append((first, tq.tq_stack_create([m[f"l{n}.o"]], [self.a], [self.o]),
                                tq.tq_stack_create([m[f"l{n}.gate"], m[f"l{n}.up"]], [self.x] * 2, [self.gate, self.up]),
                                tq.tq_stack_create([m[f"l{n}.down"]], [self.act], [self.down])))
        self.head = tq.tq_stack_create([m["head"]], [self.x], [self.logits])

    def see(self, states: torch.Tensor, tiles) -> None:
        """The image of each sequence: states bf16 [batch][tiles * patches][hidden], tiles[b] of them filled.  Their keys and values
        are computed once, by every layer that looks at them."""
        c, S = self.cfg, states.shape[1]
        self.image_states = states
        self.tile_mask = (torch.arange(c.tiles, device="cuda") < torch.tensor(tiles, device="cuda")[:, None])[:, None].to(torch.uint8).contiguous()
        for n, kind in enumerate(c.layers):
            if kind != "c":
                continue
            kv = []
            for name in ("k", "v"):
                mat = self.mats[f"l{n}.{name}"]
                ws = torch.empty(tq.tq_gemm_workspace_size(mat) + 256, dtype=torch.uint8, device="cuda")
                ws = ws[(-ws.data_ptr()) % 256:]
                kv.append(tq.tq_fused_gemm_ws(mat, states.reshape(-1, c.hidden), ws))
            keys = tq.tq_rmsnorm(kv[0].view(-1, c.dim), self.norms[f"l{n}.kn"], eps=EPS)
            self.image[n] = (keys.view(-1, S, c.kv_heads, c.dim), kv[1].to(torch.bfloat16).view(-1, S, c.kv_heads, c.dim))

    def step(self, tokens: torch.Tensor) -> torch.Tensor:
        """One new token per sequence -> logits, fp32 [batch][vocab] (the decoder's own buffer)."""
        c, B = self.cfg, self.batch
        if self.steps >= c.max_tokens:
            raise ValueError(f"the cache has room for {c.max_tokens} tokens of a sequence")
        self.steps += 1
        h = self.embed[tokens]
        positions = self.lens.clone()
        page = self.pages.gather(1, (positions // c.page).long()[:, None])[:, 0]
        slots = page * c.page + positions % c.page
        self.lens += 1
        delta = None
        for n, (first, out, gate_up, down) in enumerate(self.stacks):
            tq.tq_rmsnorm(h, self.norms[f"l{n}.attn"], delta, eps=EPS, out=self.x)
            tq.tq_fused_gemv_stack(first)
            a = self.a.view(B, c.heads, c.dim)
            if c.layers[n] == "s":
                q = tq.tq_rope_append(self.q, self.k, self.v, self.rope, positions, slots, self.caches[n])
                tq.tq_paged_attention(q, self.caches[n], self.pages, self.lens, self.workspace, out=a)
                tq.tq_fused_gemv_stack(out)
            else:
                q = tq.tq_rmsnorm(self.q.view(-1, c.dim), self.norms[f"l{n}.qn"], eps=EPS).view(B, 1, c.heads, c.dim)
                tq.tq_cross_attention(q, *self.image[n], self.workspace, mask=self.tile_mask, block_len=c.patches, out=a[:, None])
                tq.tq_fused_gemv_stack(out)
                self.o *= math.tanh(self.gates[n])
            tq.tq_rmsnorm(h, self.norms[f"l{n}.mlp"], self.o, eps=EPS, out=self.x)
            tq.tq_fused_gemv_stack(gate_up)
            torch.mul(torch.nn.functional.silu(self.gate), self.up, out=self.gate)
            self.act.copy_(self.gate)
            tq.tq_fused_gemv_stack(down)
            if c.layers[n] == "c":
                self.down *= math.tanh(self.gates[n])
            delta = self.down
        tq.tq_rmsnorm(h, self.norms["head"], delta, eps=EPS, out=self.x)
        tq.tq_fused_gemv_stack(self.head)
        return self.logits

    # -------------------------------------------------------------------------------------- in 64 bits
    def reference(self, history: torch.Tensor) -> torch.Tensor:
        """Logits after history ([batch][tokens]), from the formulas in 64 bits on the dequantised weights, all tokens at once."""
        c, (B, T) = self.cfg, history.shape
        w = lambda n: self.dense[n][0].double() * self.dense[n][1].double()[:, None]  # noqa: E731
        rms = lambda x, n: x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * self.norms[n].double()  # noqa: E731
        split = lambda x, n: x.view(B, -1, n, c.dim).transpose(1, 2)  # noqa: E731
        G = c.heads // c.kv_heads
        h = self.embed[history].double()
        cos, sin = self.rope.double()[:T].chunk(2, 1)

        def turn(x):
            a, b = x.chunk(2, -1)
            return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)

        def attend(q, k, v, seen):
            x = q @ k.repeat_interleave(G, 1).transpose(-1, -2) / math.sqrt(c.dim)
            return torch.softmax(x.masked_fill(~seen, -math.inf), -1) @ v.repeat_interleave(G, 1)

        for n, kind in enumerate(c.layers):
            x = rms(h, f"l{n}.attn")
            q = split(x @ w(f"l{n}.q").T, c.heads)
            if kind == "s":
                k, v = (split(x @ w(f"l{n}.{m}").T, c.kv_heads) for m in "kv")
                a = attend(turn(q), turn(k), v, torch.ones(T, T, dtype=torch.bool, device="cuda").tril())
                g = 1.0
            else:
                st = self.image_states.double()
                k, v = (split(st @ w(f"l{n}.{m}").T, c.kv_heads) for m in "kv")
                seen = self.tile_mask.bool().repeat_interleave(c.patches, -1)[:, None]
                a = attend(rms(q, f"l{n}.qn"), rms(k, f"l{n}.kn"), v, seen)
                g = math.tanh(self.gates[n])
            h = h + g * (a.transpose(1, 2).reshape(B, T, -1) @ w(f"l{n}.o").T)
            x = rms(h, f"l{n}.mlp")
            h = h + g * ((torch.nn.functional.silu(x @ w(f"l{n}.gate").T) * (x @ w(f"l{n}.up").T)) @ w(f"l{n}.down").T)
        return rms(h[:, -1], "head") @ w("head").T


def run(cfg: Config, batch: int, steps: int, seed: int = 0, check: bool = True):
    """Greedy decoding from one start token per sequence; -> (tokens [batch][steps], largest error of the last logits relative to
    their largest magnitude, us per step)."""
    if not 1 <= steps <= cfg.max_tokens:
        raise ValueError(f"1 to {cfg.max_tokens} steps, not {steps}")
    d = Decoder(cfg, batch, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    d.see(torch.randn(batch, cfg.tiles * cfg.patches, cfg.hidden, generator=g, device="cuda").to(torch.bfloat16),
          [1 + b % cfg.tiles for b in range(batch)])
    token = torch.arange(batch, device="cuda") % cfg.vocab
    history = [token]
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for n in range(steps):
        if n == min(3, steps - 1):
            start.record()
        logits = d.step(token)
        token = logits.argmax(1)
        history.append(token)
    end.record()
    torch.cuda.synchronize()
    error = None
    if check:
        ref = d.reference(torch.stack(history[:-1], 1))
        error = float(((logits.double() - ref).abs().amax(1) / ref.abs().amax(1)).max())
    status = tq.tq_attn_status(d.workspace) | max((tq.tq_kv_cache_status(x) for x in d.caches.values()), default=0)
    assert status == 0, status
    return torch.stack(history[1:], 1), error, start.elapsed_time(end) * 1e3 / (steps - min(3, steps - 1))


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--model", choices=["1b", "3b", "11b", "90b"])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--batch", type=int, default=2)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    tokens, error, us = run(Config.named(a.model, a.layers) if a.model else Config(), a.batch, a.steps, check=a.check or not a.model)
    print(f"{a.batch} sequences, {a.steps} steps, {us:.0f} us per step" + ("" if error is None else f", error of the last logits {error:.2e}"))
    print(tokens[:, :16].tolist())
