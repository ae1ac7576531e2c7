"""What the speed of the 4-bit serving operators is measured on.

One decoder layer that keeps its weights and its KV cache in 4 bits is made of four operators:
  linear     Y = epilogue(X W^T), W = scale * (code - zero) by groups along K
  append     fresh K and V rows are rounded to 4 bits, written to their slots of a paged cache,
             and read back as the values that they now stand for
  attention  tree-masked attention over the paged 4-bit cache (grouped-query heads, 1 to 64 queries)
  score      the attention weight that each cached row drew is added to its running sum
  evict      the rows with the largest sums and the most recent rows move to new pages

listed() are the measured cases, draw() gives more of the same ranges; prepare() builds what a
program holds before the call, run() is one pass, exact() the same numbers in 64 bits.  Shapes
are those of the repository's configurations (4096 and 5120 wide with 32 and 40 heads of 128 and an
FFN of 11008, 256 wide with 4 heads of 64) and generic grouped-query layouts.

The cache holds, per row and head, head_dim codes 0..15 with a step and a base in bf16:
  base = bf16(min x), step = bf16((max x - min x) / 15), code = clamp(rint((x - base) / step), 0, 15)
and the row stands for base + step * code.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # run the framework's operators instead of the plain forms


# ---------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------
def _linear(name, rows, n, k, group, zeros, epi, split, dtype, out):
    return dict(name=name, kind="linear", rows=rows, n=n, k=k, group=group, zeros=zeros, epi=epi, split=split,
                dtype=dtype, out=out)


def _cache(name, kind, batch, heads, kv_heads, head_dim, ctx_min, ctx_max, **more):
    return dict(name=name, kind=kind, batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim, ctx_min=ctx_min,
                ctx_max=ctx_max, **more)


def listed():
    return [
        # the smallest projection, at odd sizes: a few rows of a small model, latency only
        _linear("linear_ragged_5row", 5, 1000, 544, 32, True, 1, False, "bf16", "bf16"),
        # decoding one token: SwiGLU's gate and up projections of the 4096-wide model
        _linear("linear_gate_up_1row", 1, 22016, 4096, 128, True, 0, False, "bf16", "bf16"),
        # verifying a 64-node tree: the same projections, activations as hi + lo pairs, added to fp32
        _linear("linear_gate_up_64row", 64, 22016, 4096, 128, True, 2, True, "bf16", "fp32"),
        # one decoded token's K and V of one layer
        _cache("append_1row", "append", 1, 32, 32, 128, 700, 700, rows=1, dtype="fp32"),
        # a batch of prompts' K and V, ragged
        _cache("append_prompts", "append", 4, 32, 32, 128, 0, 300, rows=1000, dtype="bf16"),
        # decoding one token of a 512-token request
        _cache("attention_1query_512", "attention", 1, 32, 32, 128, 512, 512, queries=1, q_local0=0, tree=False,
               out="bf16", out_lo=False, lse=True),
        # a ragged batch of eight, grouped-query heads, four chained draft rows each
        _cache("attention_batch8_gqa", "attention", 8, 32, 8, 128, 256, 4096, queries=4, q_local0=0, tree=False,
               out="bf16", out_lo=True, lse=True),
        # verifying a 64-node tree over a long cache
        _cache("attention_tree_16k", "attention", 1, 32, 32, 128, 16384, 16384, queries=64, q_local0=0, tree=True,
               out="bf16", out_lo=False, lse=False),
        # the weight of one decoded token's attention, short and long
        _cache("score_1query_512", "score", 1, 32, 32, 128, 512, 512, queries=1, q_local0=0, tree=False),
        _cache("score_tree_16k", "score", 1, 32, 32, 128, 16384, 16384, queries=32, q_local0=0, tree=True),
        # a small model's cache at its budget, one page over it
        _cache("evict_256_of_272", "evict", 1, 4, 4, 64, 272, 272, budget=256, recent=64),
        # a ragged batch cut to half of its longest member's rows
        _cache("evict_batch2_16k", "evict", 2, 32, 32, 128, 6000, 16384, budget=8192, recent=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


LAYOUTS = [(32, 32, 128), (32, 32, 128), (40, 40, 128), (32, 8, 128), (28, 4, 128), (8, 1, 128), (4, 4, 64), (16, 2, 64)]
MOST_MACS = 64 * 22016 * 4096 * 2  # the largest listed linear
MOST_WEIGHTS = 22016 * 4096


def draw(rng):
    kind = rng.choices(["linear", "append", "attention", "score", "evict"], [6, 2, 6, 2, 3])[0]
    if kind == "linear":
        dtype = rng.choices(["bf16", "fp32"], [5, 1])[0]
        epi = rng.choice([0, 1, 2])
        split = dtype == "bf16" and rng.random() < 0.5
        rows, n, k = _log_int(rng, 1, 256), _log_int(rng, 400, 32000), 32 * _log_int(rng, 8, 384)
        n = max(1, min(n, MOST_WEIGHTS // k, MOST_MACS // (k * rows * (2 if split else 1))))
        return dict(kind=kind, rows=rows, n=n, k=k, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.7, epi=epi,
                    split=split, dtype=dtype,
                    out="fp32" if dtype == "fp32" or epi == 2 or rng.random() < 0.4 else "bf16")
    heads, kv_heads, head_dim = rng.choice(LAYOUTS)
    batch = _log_int(rng, 1, 8)
    c = dict(kind=kind, batch=batch, heads=heads, kv_heads=kv_heads, head_dim=head_dim)
    if kind == "append":
        rows = _log_int(rng, 1, 3000 // batch)
        ctx = rng.randint(0, 500)
        return dict(c, ctx_min=ctx // 2, ctx_max=ctx, rows=rows, dtype=rng.choice(["fp32", "bf16"]))
    if kind == "evict":
        ctx = _log_int(rng, 40, 16384 // batch)
        budget = max(2, int(ctx * rng.uniform(0.2, 0.9)))
        return dict(c, ctx_min=max(1, ctx // 3), ctx_max=ctx, budget=budget, recent=rng.randint(0, budget))
    ctx = _log_int(rng, 16, 16000 // batch)
    tree = rng.random() < 0.5
    queries = rng.randint(2, (64 if kind == "attention" else 32) if batch == 1 else 16) if tree else rng.randint(1, 4)
    c = dict(c, ctx_min=ctx // 3, ctx_max=ctx, queries=queries, q_local0=0 if tree else rng.randint(0, 3), tree=tree)
    if kind == "score":
        return c
    out = rng.choice(["bf16", "bf16", "fp32"])
    return dict(c, out=out, out_lo=out == "bf16" and rng.random() < 0.4, lse=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g)


def _dtype(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def _two_terms(x32):
    hi = x32.to(torch.bfloat16)
    return hi, (x32 - hi.float()).to(torch.bfloat16)


def _linear_inputs(c, seed):
    """Codes, steps and zeros of a round-to-nearest group quantisation of N(0, 0.02) weights."""
    g = _generator(seed)
    rows, n, k, group = c["rows"], c["n"], c["k"], c["group"]
    x32 = _normal(g, (rows, k))
    groups = -(-k // group)
    w = torch.zeros(n, groups * group, device="cuda")
    w[:, :k] = _normal(g, (n, k), 0.02)
    w = w.view(n, groups, group)
    lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
    if c["zeros"]:
        scale = ((hi - lo) / 15).clamp(min=1e-8).to(torch.bfloat16)
        zero = torch.round(-lo / scale.float()).clamp(0, 15)
    else:
        scale = (torch.maximum(hi, -lo) / 7.5).clamp(min=1e-8).to(torch.bfloat16)
        zero = torch.full_like(lo, 8)
    code = torch.round(w / scale.float()[..., None] + zero[..., None]).clamp(0, 15).to(torch.uint8).view(n, -1)[:, :k]
    s = dict(kind="linear", case=c, x=x32.to(_dtype(c["dtype"])), x_lo=None, scale=scale,
             w=(code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), zero=zero.to(torch.uint8) if c["zeros"] else None)
    if c["split"]:
        s["x"], s["x_lo"] = _two_terms(x32)
    s["y"] = _normal(g, (rows, n)).to(_dtype(c["out"]))  # epilogue 2 adds to it
    return s


def _round4(x):
    """Codes, step and base (in bf16) of rows of 32-bit values."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    base, step = lo.to(torch.bfloat16), ((hi - lo) / 15).to(torch.bfloat16)
    code = torch.round((x - base.float()) / step.float()).clamp(0, 15)
    code = torch.where(step > 0, code, torch.zeros_like(code))
    return code.to(torch.uint8), step, base


def _kv_rows(g, batch, length, kv_heads, head_dim):
    """Keys whose channels have offsets and sizes of their own, as trained models' do, and plain values."""
    size = torch.exp(0.5 * _normal(g, (kv_heads, head_dim)))
    mean = 0.7 * _normal(g, (kv_heads, head_dim))
    k = (_normal(g, (batch, length, kv_heads, head_dim)) + mean) * size
    return k, _normal(g, (batch, length, kv_heads, head_dim))


def _tree_masks(n, tree, r):
    """Ancestor-or-self masks: a random tree, or a chain."""
    masks = []
    for i in range(n):
        parent = (int(r.integers(0, i)) if tree else i - 1) if i else -1
        masks.append((masks[parent] if parent >= 0 else 0) | (1 << i))
    return masks


def _lengths(c, seed):
    r = np.random.default_rng(seed)
    return [c["ctx_max"]] + [int(v) for v in r.integers(c["ctx_min"], c["ctx_max"] + 1, c["batch"] - 1)]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cache_inputs(c, seed):
    g, r = _generator(seed), np.random.default_rng(seed + 1)
    batch, heads, kv_heads, head_dim = c["batch"], c["heads"], c["kv_heads"], c["head_dim"]
    ctx = _lengths(c, seed)
    s = dict(kind=c["kind"], case=c, ctx=ctx, n_ctx=_ints(ctx))
    if c["kind"] == "append":
        new = c["rows"]
        k, v = _kv_rows(g, batch, new, kv_heads, head_dim)
        dt = _dtype(c["dtype"])
        s["k"], s["v"] = k.view(batch * new, -1).to(dt), v.view(batch * new, -1).to(dt)
        s["k_back"], s["v_back"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        pages = (max(ctx) + new + 15) // 16
        filled = 0
    else:
        new = c["q_local0"] + c["queries"] if c["kind"] != "evict" else 0
        filled = max(ctx) + new
        k, v = _kv_rows(g, batch, filled, kv_heads, head_dim)
        pages = (filled + 15) // 16
    extra = (c["budget"] + 15) // 16 if c["kind"] == "evict" else 0
    blocks = batch * (pages + extra)
    order = r.permutation(blocks).astype(np.int32)
    s["table"] = torch.from_numpy(order[:batch * pages].reshape(batch, pages)).cuda()
    s["blocks"] = blocks
    if c["kind"] == "evict":
        s["dst_table"] = torch.from_numpy(order[batch * pages:].reshape(batch, extra)).cuda()
        # sums of attention weights: most rows draw little, a few draw much
        s["scores"] = torch.exp(1.5 * _normal(g, (batch, kv_heads, pages * 16)))
        s["scores_out"] = torch.zeros(batch, kv_heads, c["budget"], device="cuda")
        s["kept"] = torch.zeros(batch, kv_heads, c["budget"], dtype=torch.int32, device="cuda")
        s["n_out"] = torch.zeros(batch, dtype=torch.int32, device="cuda")
        s["k_back"] = torch.zeros(batch * c["budget"], kv_heads * head_dim, dtype=torch.bfloat16, device="cuda")
        s["v_back"] = torch.zeros_like(s["k_back"])
        s["zero_slot"] = torch.zeros(batch, dtype=torch.int32, device="cuda")
    if c["kind"] in ("attention", "score"):
        masks = _tree_masks(new, c["tree"], r)
        nq = c["queries"]
        s["masks"], s["n_local"] = masks, new
        s["anc"] = torch.from_numpy(np.array(masks, dtype=np.uint64).view(np.int64)).cuda()
        s["q"] = _normal(g, (batch * nq, heads * head_dim), 0.8)
        if c["kind"] == "attention":
            s["out"] = torch.empty(batch * nq, heads * head_dim, dtype=_dtype(c["out"]), device="cuda")
            s["out_lo"] = torch.empty_like(s["out"]) if c["out_lo"] else None
            s["lse"] = torch.empty(batch * nq, heads, device="cuda") if c["lse"] else None
        else:
            s["scores"] = torch.zeros(batch, kv_heads, pages * 16, device="cuda")
            # the rows of an accepted path count, the others do not
            s["weight"] = torch.from_numpy((r.random(batch * nq) < 0.6).astype(np.float32)).cuda() if c["tree"] else None
    if filled:
        s["codes"] = [_round4(k), _round4(v)]
    if own:
        import paper_2402_15758_gb300 as pkg
        s["pool"] = pkg.kv4_pool(blocks, kv_heads, head_dim)
        if filled:
            pkg.op_kv4_append(k.view(batch * filled, -1), v.view(batch * filled, -1), s["pool"], s["table"],
                              torch.zeros(batch, dtype=torch.int32, device="cuda"), filled, head_dim)
            del s["codes"]
    if c["kind"] == "score":
        # what the attention before it left behind: the log of each row's sum
        s["lse"] = _logits(s, _values(_round4(k)), torch.float32).logsumexp(-1)
        s["lse"] = s["lse"].permute(0, 2, 1).reshape(batch * c["queries"], heads).contiguous()
    return s


def prepare(case, seed):
    return _linear_inputs(case, seed) if case["kind"] == "linear" else _cache_inputs(case, seed)


# ---------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------
def _dense_weight(s, dt):
    c = s["case"]
    code = torch.stack([s["w"] & 15, s["w"] >> 4], -1).view(c["n"], c["k"]).to(dt)
    per_k = lambda t: t.to(dt).repeat_interleave(c["group"], 1)[:, :c["k"]]  # noqa: E731
    return (code - (per_k(s["zero"]) if s["zero"] is not None else 8)) * per_k(s["scale"])


def _linear_value(s, dt):
    x = s["x"].to(dt) if s["x_lo"] is None else s["x"].to(dt) + s["x_lo"].to(dt)
    y = x @ _dense_weight(s, dt).T
    if s["case"]["epi"] == 1:
        y = y / (1 + torch.exp(-y))
    return y


def _values(codes, dt=torch.float32):
    """What the codes stand for, [batch][kv heads][rows][head_dim]."""
    code, step, base = codes
    return (base.to(dt) + step.to(dt) * code.to(dt)).transpose(1, 2)


def _logits(s, k, dt):
    """Masked q . k / sqrt(head_dim), [batch][heads][queries][slots]; -inf where nothing is seen."""
    c = s["case"]
    batch, heads, kv_heads, head_dim, nq = c["batch"], c["heads"], c["kv_heads"], c["head_dim"], c["queries"]
    q = s["q"].to(dt).view(batch, nq, kv_heads, heads // kv_heads, head_dim).permute(0, 2, 3, 1, 4)
    z = (q.reshape(batch, kv_heads, -1, head_dim) @ k.transpose(-1, -2)).view(batch, heads, nq, -1) / math.sqrt(head_dim)
    slot = torch.arange(z.shape[-1], device="cuda")
    local = slot[None] - s["n_ctx"].long()[:, None]
    bit = (s["anc"][c["q_local0"]:c["q_local0"] + nq][None, :, None] >> local.clamp(0, 63)[:, None]) & 1
    seen = (local < 0)[:, None] | ((local >= 0) & (local < s["n_local"]))[:, None] & (bit != 0)
    return z.masked_fill(~seen[:, None], -math.inf)


def _pair(hi, lo):
    """The value that a hi + lo pair stands for: next to a tie of hi, lo alone is a matter of the last bit of the sum."""
    return hi.float() + lo


def _attention_value(s, k, v, dt):
    c = s["case"]
    batch, heads, kv_heads, head_dim, nq = c["batch"], c["heads"], c["kv_heads"], c["head_dim"], c["queries"]
    z = _logits(s, k, dt)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    o = (p / total).view(batch, kv_heads, -1, z.shape[-1]) @ v
    o = o.view(batch, heads, nq, head_dim).permute(0, 2, 1, 3).reshape(batch * nq, heads * head_dim)
    return o, (top + torch.log(total))[..., 0].permute(0, 2, 1).reshape(batch * nq, heads)


def _score_value(s, k, dt):
    """The attention weight that each slot draws from the counted rows, [batch][kv heads][slots]."""
    c = s["case"]
    batch, heads, kv_heads, nq = c["batch"], c["heads"], c["kv_heads"], c["queries"]
    lse = s["lse"].to(dt).view(batch, nq, heads).permute(0, 2, 1)[..., None]
    p = torch.exp(_logits(s, k, dt) - lse)
    if s["weight"] is not None:
        p = p * s["weight"].to(dt).view(batch, 1, nq, 1)
    return p.view(batch, kv_heads, -1, p.shape[-1]).sum(2)


def _kept_rows(s):
    """Slots that stay, ascending, -1 past the end: the most recent ones and the largest sums before them."""
    c = s["case"]
    budget, recent = c["budget"], c["recent"]
    n = s["n_ctx"].long()[:, None, None]
    slot = torch.arange(s["scores"].shape[-1], device="cuda")
    x = s["scores"].masked_fill(slot >= n - recent, math.inf)
    x = x.masked_fill(slot >= n, -math.inf)
    at = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :budget]
    last = s["scores"].shape[-1]
    at = torch.sort(at.masked_fill(at >= n, last), -1).values
    return torch.where(at < last, at, -1)


def _evict_value(s, dt):
    c = s["case"]
    kept = _kept_rows(s)
    at, there = kept.clamp(min=0), kept >= 0
    sums = torch.where(there, s["scores"].gather(-1, at), 0)
    back = []
    for codes in s["codes"]:
        rows = _values(codes, dt).gather(2, at[..., None].expand(-1, -1, -1, c["head_dim"]))
        rows = torch.where(there[..., None], rows, 0)
        back.append(rows.transpose(1, 2).reshape(c["batch"] * c["budget"], -1))
    return kept.to(torch.int32), sums, back


def _run_plain(s):
    c = s["case"]
    f32 = torch.float32
    if c["kind"] == "linear":
        y = _linear_value(s, f32)
        if c["epi"] == 2:
            return s["y"].add_(y)
        return y.to(_dtype(c["out"]))
    if c["kind"] == "append":
        back = [_values(_round4(x.to(f32).view(c["batch"], c["rows"], c["kv_heads"], -1))) for x in (s["k"], s["v"])]
        return [x.transpose(1, 2).reshape(c["batch"] * c["rows"], -1).to(_dtype(c["dtype"])) for x in back]
    if c["kind"] == "attention":
        o, lse = _attention_value(s, _values(s["codes"][0]), _values(s["codes"][1]), f32)
        out = o.to(_dtype(c["out"]))
        if c["out_lo"]:
            out = _pair(out, (o - out.float()).to(torch.bfloat16))
        return dict(out=out, lse=lse if c["lse"] else None)
    if c["kind"] == "score":
        s["scores"][..., :max(s["ctx"]) + s["n_local"]] += _score_value(s, _values(s["codes"][0]), f32)
        return s["scores"]
    kept, sums, back = _evict_value(s, f32)
    return dict(kept=kept, scores=sums, n=s["n_ctx"].clamp(max=c["budget"]), k=back[0].to(torch.bfloat16),
                v=back[1].to(torch.bfloat16))


# ---------------------------------------------------------------------------------------
# the framework's operators
# ---------------------------------------------------------------------------------------
def _run_own(s):
    import paper_2402_15758_gb300 as pkg
    c = s["case"]
    if c["kind"] == "linear":
        pkg.op_linear_w4(s["x"], s["w"], s["scale"], s["y"], zeros=s["zero"], group=c["group"], epi=c["epi"],
                         out_f32=c["out"] == "fp32", X_lo=s["x_lo"])
        return s["y"]
    if c["kind"] == "append":
        pkg.op_kv4_append(s["k"], s["v"], s["pool"], s["table"], s["n_ctx"], c["rows"], c["head_dim"])
        pkg.op_kv4_read(s["pool"], s["table"], s["n_ctx"], c["rows"], c["head_dim"], s["k_back"], s["v_back"])
        return [s["k_back"], s["v_back"]]
    if c["kind"] == "attention":
        pkg.op_attention_kv4(s["q"], s["pool"], s["table"], s["n_ctx"], s["anc"], s["out"], c["queries"], c["q_local0"],
                             s["n_local"], c["queries"], c["heads"], c["head_dim"], out_lo=s["out_lo"], lse=s["lse"])
        return dict(out=_pair(s["out"], s["out_lo"]) if c["out_lo"] else s["out"], lse=s["lse"])
    if c["kind"] == "score":
        pkg.op_kv4_score(s["q"], s["lse"], s["pool"], s["table"], s["n_ctx"], s["anc"], s["scores"], c["queries"],
                         c["q_local0"], s["n_local"], c["queries"], c["heads"], c["head_dim"], weight=s["weight"])
        return s["scores"]
    pkg.op_kv4_evict(s["pool"], s["table"], s["n_ctx"], s["scores"], c["budget"], c["recent"], s["dst_table"],
                     s["kept"], s["scores_out"], s["n_out"], c["head_dim"])
    pkg.op_kv4_read(s["pool"], s["dst_table"], s["zero_slot"], c["budget"], c["head_dim"], s["k_back"], s["v_back"],
                    counts=s["n_out"])
    return dict(kept=s["kept"], scores=s["scores_out"], n=s["n_out"], k=s["k_back"], v=s["v_back"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "linear":
        rows, n, k, terms = c["rows"], c["n"], c["k"], 2 if c["split"] else 1
        x = rows * k * (4 if c["dtype"] == "fp32" else 2) * terms
        y = rows * n * (4 if c["out"] == "fp32" else 2) * (2 if c["epi"] == 2 else 1)
        groups = n * -(-k // c["group"])
        return dict(bytes=n * k / 2 + groups * (3 if c["zeros"] else 2) + x + y, flops=2.0 * rows * n * k * terms)
    batch, kv_heads, hd = c["batch"], c["kv_heads"], c["head_dim"]
    row = kv_heads * (hd + 8)  # one cached row: K and V codes, two steps and two bases
    mean = c["ctx_max"] if batch == 1 else (c["ctx_max"] + (batch - 1) * (c["ctx_min"] + c["ctx_max"]) / 2) / batch
    if c["kind"] == "append":
        x = 2 * kv_heads * hd * (4 if c["dtype"] == "fp32" else 2)
        return dict(bytes=batch * c["rows"] * (2 * x + 2 * row), flops=batch * c["rows"] * kv_heads * hd * 10.0)
    if c["kind"] == "evict":
        keep = batch * min(c["budget"], mean)
        return dict(bytes=batch * mean * kv_heads * 4 + keep * (kv_heads * 8 + 3 * row + 4 * kv_heads * hd), flops=0.0)
    rows = batch * c["queries"]
    keys = mean + c["q_local0"] + c["queries"]
    q = rows * c["heads"] * hd
    if c["kind"] == "attention":
        out = q * ((4 if c["out"] == "fp32" else 2) + (2 if c["out_lo"] else 0)) + (4 * rows * c["heads"] if c["lse"] else 0)
        return dict(bytes=batch * keys * row + 4 * q + out, flops=4.0 * q * keys)
    return dict(bytes=batch * keys * kv_heads * (hd / 2 + 4 + 8) + 4 * q + 4 * rows * c["heads"], flops=2.0 * q * keys)


# ---------------------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------------------
def _exact_linear(s):
    c, f64 = s["case"], torch.float64
    x = s["x"].to(f64)
    if s["x_lo"] is not None:
        x = x + s["x_lo"].to(f64)
    y = torch.zeros(c["rows"], c["n"], dtype=f64, device="cuda")
    for i, k0 in enumerate(range(0, c["k"], c["group"])):  # group by group: step * (x . codes - zero * sum x)
        k1 = min(k0 + c["group"], c["k"])
        packed = s["w"][:, k0 // 2:k1 // 2]
        part = x[:, k0:k1:2] @ (packed & 15).to(f64).T + x[:, k0 + 1:k1:2] @ (packed >> 4).to(f64).T
        zero = s["zero"][:, i].to(f64) if s["zero"] is not None else torch.full((c["n"],), 8.0, dtype=f64, device="cuda")
        y += s["scale"][:, i].to(f64) * (part - zero * x[:, k0:k1].sum(1, keepdim=True))
    if c["epi"] == 1:
        y = y * torch.sigmoid(y)
    return y + s["y"].to(f64) if c["epi"] == 2 else y


def _exact_row(x):
    """The value of each row after rounding to 4 bits, from its definition."""
    x = x.double()
    lo, hi = x.min(-1).values[..., None], x.max(-1).values[..., None]
    base, step = lo.to(torch.bfloat16).double(), ((hi - lo) / 15).to(torch.bfloat16).double()
    code = torch.where(step > 0, ((x - base) / step.clamp(min=1e-300)).round(), torch.zeros_like(x))
    return base + step * torch.minimum(torch.maximum(code, torch.zeros_like(code)), torch.full_like(code, 15))


def _exact_heads(s, b, h):
    """One head of one sequence: probabilities, log of the sum and the values, over its visible slots."""
    c = s["case"]
    nq, hd, g = c["queries"], c["head_dim"], h // (c["heads"] // c["kv_heads"])
    n = s["ctx"][b] + s["n_local"]
    deq = [code[b, :n, g].double() * step[b, :n, g].double() + base[b, :n, g].double() for code, step, base in s["codes"]]
    q = s["q"][b * nq:(b + 1) * nq, h * hd:(h + 1) * hd].double()
    z = q @ deq[0].T * hd ** -0.5
    for i in range(nq):
        mask = s["masks"][c["q_local0"] + i]
        hidden = [s["ctx"][b] + j for j in range(s["n_local"]) if not mask >> j & 1]
        z[i, hidden] = -math.inf
    return z, deq[1]


def exact(case, seed):
    c = case
    if c["kind"] == "linear":
        return _exact_linear(_linear_inputs(c, seed))
    s = _cache_inputs(c, seed)
    if c["kind"] == "append":
        split = lambda x: x.view(x.shape[0], c["kv_heads"], c["head_dim"])  # noqa: E731
        return [_exact_row(split(x)).reshape(x.shape) for x in (s["k"], s["v"])]
    if c["kind"] == "evict":
        k, v = (base.double() + code.double() * step.double() for code, step, base in s["codes"])
        sums = torch.zeros_like(s["scores_out"], dtype=torch.float64)
        back = [torch.zeros(c["batch"], c["budget"], c["kv_heads"], c["head_dim"], dtype=torch.float64, device="cuda")
                for _ in range(2)]
        for b in range(c["batch"]):
            n = s["ctx"][b]
            older = max(0, n - c["recent"])
            for h in range(c["kv_heads"]):
                x = s["scores"][b, h, :n].double().cpu().numpy()
                best = np.lexsort((np.arange(older), -x[:older]))[:max(0, min(c["budget"], n) - (n - older))]
                at = np.concatenate([np.sort(best), np.arange(older, n)])[:c["budget"]]
                at = torch.from_numpy(at).cuda()
                sums[b, h, :len(at)] = s["scores"][b, h, at].double()
                back[0][b, :len(at), h], back[1][b, :len(at), h] = k[b, at, h], v[b, at, h]
        k, v = (x.reshape(c["batch"] * c["budget"], -1) for x in back)
        return dict(kept=None, scores=sums, n=None, k=k, v=v)
    heads, nq, hd = c["heads"], c["queries"], c["head_dim"]
    out = torch.zeros(c["batch"] * nq, heads * hd, dtype=torch.float64, device="cuda")
    lse = torch.zeros(c["batch"] * nq, heads, dtype=torch.float64, device="cuda")
    sums = torch.zeros(s["scores"].shape if c["kind"] == "score" else (1,), dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        at = slice(b * nq, (b + 1) * nq)
        for h in range(heads):
            z, v = _exact_heads(s, b, h)
            if c["kind"] == "attention":
                lse[at, h] = torch.logsumexp(z, 1)
                out[at, h * hd:(h + 1) * hd] = torch.softmax(z, 1) @ v
                continue
            p = torch.exp(z - s["lse"][at, h, None].double())
            if s["weight"] is not None:
                p = p * s["weight"][at, None].double()
            sums[b, h // (heads // c["kv_heads"]), :p.shape[1]] += p.sum(0)
    if c["kind"] == "score":
        return sums
    return dict(out=out, lse=lse if c["lse"] else None)
