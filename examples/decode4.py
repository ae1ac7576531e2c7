"""Decode with everything in 4 bits: weights, KV cache, and a cache of bounded length.

    python examples/decode4.py [--config mini] [--tokens 48] [--budget 96] [--recent 32]

A Llama-shaped model of random weights (synth/) is rounded to 4-bit weights; its prompt and its own tokens are
run through the library's 4-bit operators: every projection is op_linear_w4, every layer writes its K and V
rows to a 4-bit paged cache (op_kv4_append), attends over it (op_attention_kv4) and adds up how
much attention each cached row draws (op_kv4_score); when a cache passes its limit, the rows that drew least
leave it (op_kv4_evict).  Norms, rotary angles and the SwiGLU product are plain torch.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2402_15758_gb300 as pkg  # noqa: E402
import synth  # noqa: E402

CHUNK = 64  # rows of one attention call


def rms_norm(x, gain, eps):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * gain.float()


def rotate(x, positions, theta):
    """Rotary embedding (rotate-half) of [rows][heads][head_dim]."""
    half = x.shape[-1] // 2
    angle = positions[:, None].double() * theta ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


class Linear4:
    """y = x W^T with W rounded to 4 bits."""

    def __init__(self, w, group):
        self.group = group
        self.codes, self.scales, self.zeros = pkg.w4_round(w, group)

    def __call__(self, x, add_to=None):
        y = torch.empty(x.shape[0], self.codes.shape[0], device="cuda") if add_to is None else add_to
        pkg.op_linear_w4(x.to(torch.bfloat16), self.codes, self.scales, y, zeros=self.zeros, group=self.group,
                         epi=0 if add_to is None else 2, out_f32=True)
        return y


class Decoder4:
    """One sequence; a cache of at most `budget` rows plus one chunk."""

    def __init__(self, cfg, weights, budget, recent, group=128):
        self.cfg, self.budget, self.recent = cfg, budget, recent
        self.w = weights
        lin = lambda name: Linear4(weights[name], group)  # noqa: E731
        self.layers = [{n: lin(f"layers.{i}.{n}") for n in ("wqkv", "wo", "w_gate", "w_up", "w_down")} for i in range(cfg["n_layers"])]
        self.lm_head = lin("lm_head")
        H, hd = cfg["n_heads"], cfg["head_dim"]
        self.slots = budget + CHUNK
        pages = (self.slots + 15) // 16
        self.pools = [pkg.kv4_pool(2 * pages, H, hd) for _ in self.layers]
        # two sets of pages: the cache is in one, an eviction writes the other
        self.table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
        self.spare = self.table + pages
        self.scores = [torch.zeros(1, H, self.slots, device="cuda") for _ in self.layers]
        self.n, self.position, self.evictions = 0, 0, 0
        self.anc = torch.from_numpy(np.array([(1 << (i + 1)) - 1 for i in range(CHUNK)], dtype=np.uint64).view(np.int64)).cuda()

    def _evict(self):
        H, hd = self.cfg["n_heads"], self.cfg["head_dim"]
        n_ctx = torch.tensor([self.n], dtype=torch.int32, device="cuda")
        kept = torch.empty(1, H, self.budget, dtype=torch.int32, device="cuda")
        n_out = torch.empty(1, dtype=torch.int32, device="cuda")
        for pool, scores in zip(self.pools, self.scores):
            sums = torch.empty(1, H, self.budget, device="cuda")
            pkg.op_kv4_evict(pool, self.table, n_ctx, scores, self.budget, self.recent, self.spare, kept, sums, n_out, hd)
            scores.zero_()
            scores[:, :, :self.budget] = sums
        self.table, self.spare = self.spare, self.table
        self.n, self.evictions = self.budget, self.evictions + 1

    def rows(self, tokens):
        """The logits of the last of up to CHUNK tokens, which join the cache."""
        cfg, r = self.cfg, len(tokens)
        H, hd, d = cfg["n_heads"], cfg["head_dim"], cfg["d_model"]
        if self.n + r > self.slots:
            self._evict()
        n_ctx = torch.tensor([self.n], dtype=torch.int32, device="cuda")
        at = torch.arange(self.position, self.position + r, device="cuda")
        x = self.w["embed"][torch.tensor(tokens, device="cuda")].float()
        for i, layer in enumerate(self.layers):
            qkv = layer["wqkv"](rms_norm(x, self.w[f"layers.{i}.attn_norm"], cfg["rms_eps"])).view(r, 3, H, hd)
            q, k = (rotate(qkv[:, j], at, cfg["rope_theta"]).reshape(r, d) for j in (0, 1))
            pkg.op_kv4_append(k, qkv[:, 2].reshape(r, d), self.pools[i], self.table, n_ctx, r, hd)
            out = torch.empty(r, d, dtype=torch.bfloat16, device="cuda")
            lse = torch.empty(r, H, device="cuda")
            args = (n_ctx, self.anc)
            pkg.op_attention_kv4(q, self.pools[i], self.table, *args, out, r, 0, r, r, H, hd, lse=lse)
            pkg.op_kv4_score(q, lse, self.pools[i], self.table, *args, self.scores[i], r, 0, r, r, H, hd)
            layer["wo"](out, add_to=x)
            h = rms_norm(x, self.w[f"layers.{i}.ffn_norm"], cfg["rms_eps"])
            layer["w_down"](torch.nn.functional.silu(layer["w_gate"](h)) * layer["w_up"](h), add_to=x)
        self.n += r
        self.position += r
        return self.lm_head(rms_norm(x[-1:], self.w["final_norm"], cfg["rms_eps"]))[0]

    def generate(self, prompt, count):
        for i in range(0, len(prompt), CHUNK):
            logits = self.rows(prompt[i:i + CHUNK])
        out = []
        for _ in range(count):
            out.append(int(logits.argmax()))
            logits = self.rows(out[-1:])
        pkg.op_sync()
        return out


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--config", default="mini", help="a bf16 configuration of synth/")
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--budget", type=int, default=96)
    ap.add_argument("--recent", type=int, default=32)
    ap.add_argument("--group", type=int, default=128)
    a = ap.parse_args()
    cfg = synth.get_config(a.config)
    weights = {k: v.cuda() for k, v in synth.make_weights(cfg).items()}
    model = Decoder4(cfg, weights, a.budget, a.recent, a.group)
    tokens = model.generate(synth.make_prompts(cfg)[0], a.tokens)
    print("tokens:", tokens)
    print(f"{model.position} positions seen, {model.n} cached rows, {model.evictions} evictions")


if __name__ == "__main__":
    main()
