"""examples/decode4.py, the 4-bit operators together, against a plain model of the same 4-bit weights whose cached rows
are rounded by the cache's rule, in 64 bits."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_2402_15758_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("decode4", os.path.join(ROOT, "examples", "decode4.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _dense(lin):
    code = torch.stack([lin.codes & 15, lin.codes >> 4], -1).view(lin.codes.shape[0], -1).double()
    per = lambda t: t.double().repeat_interleave(lin.group, 1)[:, :code.shape[1]]  # noqa: E731
    return (code - per(lin.zeros)) * per(lin.scales)


def _round4(x):
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    base, step = lo.to(torch.bfloat16).float(), ((hi - lo) / 15).to(torch.bfloat16).float()
    return (base + step * torch.round((x - base) / step).clamp(0, 15)).double()


class _Plain:
    """The same decoder in 64 bits: dense weights, a list of rounded rows and their sums per layer."""

    def __init__(self, example, model):
        self.e, self.m, self.cfg = example, model, model.cfg
        self.layers = [{k: _dense(v) for k, v in layer.items()} for layer in model.layers]
        self.head = _dense(model.lm_head)
        H, hd = self.cfg["n_heads"], self.cfg["head_dim"]
        empty = lambda: torch.zeros(H, 0, hd, dtype=torch.float64, device="cuda")  # noqa: E731
        self.k, self.v = [empty() for _ in self.layers], [empty() for _ in self.layers]
        self.sums = [torch.zeros(H, 0, dtype=torch.float64, device="cuda") for _ in self.layers]
        self.position = 0

    def _lin(self, x, w):  # the example rounds activations to bf16
        return x.to(torch.bfloat16).double() @ w.T

    def rows(self, tokens):
        cfg, r, w, e = self.cfg, len(tokens), self.m.w, self.e
        H, hd, d = cfg["n_heads"], cfg["head_dim"], cfg["d_model"]
        at = torch.arange(self.position, self.position + r, device="cuda")
        n = self.k[0].shape[1]
        if n + r > self.m.slots:
            for i in range(len(self.layers)):
                older = n - self.m.recent
                best = torch.sort(self.sums[i][:, :older], dim=-1, descending=True, stable=True).indices[:, :self.m.budget - self.m.recent]
                keep = torch.cat([best.sort(-1).values, torch.arange(older, n, device="cuda").expand(H, -1)], 1)
                take = keep[..., None].expand(-1, -1, hd)
                self.k[i], self.v[i], self.sums[i] = self.k[i].gather(1, take), self.v[i].gather(1, take), self.sums[i].gather(1, keep)
        x = w["embed"][torch.tensor(tokens, device="cuda")].double()
        for i, layer in enumerate(self.layers):
            qkv = self._lin(e.rms_norm(x, w[f"layers.{i}.attn_norm"], cfg["rms_eps"]), layer["wqkv"]).view(r, 3, H, hd)
            q, k = (e.rotate(qkv[:, j], at, cfg["rope_theta"]).transpose(0, 1) for j in (0, 1))
            self.k[i] = torch.cat([self.k[i], _round4(k)], 1)
            self.v[i] = torch.cat([self.v[i], _round4(qkv[:, 2].transpose(0, 1))], 1)
            z = q.double() @ self.k[i].transpose(1, 2) / math.sqrt(hd)
            total = z.shape[-1]
            hidden = torch.ones(r, total, dtype=torch.bool, device="cuda").triu(total - r + 1)
            p = torch.softmax(z.masked_fill(hidden, -math.inf), -1)
            self.sums[i] = torch.nn.functional.pad(self.sums[i], (0, r)) + p.sum(1)
            x = x + self._lin((p @ self.v[i]).transpose(0, 1).reshape(r, d), layer["wo"])
            h = e.rms_norm(x, w[f"layers.{i}.ffn_norm"], cfg["rms_eps"])
            x = x + self._lin(torch.nn.functional.silu(self._lin(h, layer["w_gate"])) * self._lin(h, layer["w_up"]), layer["w_down"])
        self.position += r
        return self._lin(e.rms_norm(x[-1:], w["final_norm"], cfg["rms_eps"]), self.head)[0]


def test_decode4_follows_the_plain_model(example):
    # Roundings of activations to bf16 (2^-9 each, some ten in a row of a layer) and of rows to 4 bits that fall the other
    # way next to a tie (a step is a fifth of a deviation, and takes part with its attention weight) differ between
    # the two: 4 % of the largest logit.  Both are fed the same tokens.
    cfg = synth.get_config("mini")
    weights = {k: v.cuda() for k, v in synth.make_weights(cfg).items()}
    model = example.Decoder4(cfg, weights, budget=96, recent=32)
    plain = _Plain(example, model)
    prompt = synth.make_prompts(cfg)[0]
    token = None
    for i in range(0, len(prompt), example.CHUNK):
        got, want = model.rows(prompt[i:i + example.CHUNK]), plain.rows(prompt[i:i + example.CHUNK])
    worst = 0.0
    for _ in range(80):
        worst = max(worst, float((got.double() - want).abs().max() / want.abs().max()))
        token = int(want.argmax())
        got, want = model.rows([token]), plain.rows([token])
    assert model.evictions >= 1 and model.n == plain.k[0].shape[1]
    assert worst <= 0.04


def test_decode4_runs_as_a_program(example, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["decode4.py", "--tokens", "80"])
    example.main()
    out = capsys.readouterr().out
    assert "1 evictions" in out and len(out.split("[")[1].split("]")[0].split(",")) == 80
    assert np.all(np.array([int(t) for t in out.split("[")[1].split("]")[0].split(",")]) < 2048)
