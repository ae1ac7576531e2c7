"""The 4-bit operators (linear, cache append and read, attention, weight sums, eviction) against their
definitions in 64 bits, at the sizes and masks where they can go wrong, and their refusals.

Tolerances.  fp32 sums of exact products, in chains of at most K / 16 steps that lose at most 2^-23 of
the running sum each and mostly cancel: 4e-6 of a row's largest value.  Queries and probabilities
enter as two fp16 terms (2^-22): 1e-5 of a row's largest value for attention and for its logarithms.
One rounding to bf16: 2^-9 of a value, 4e-3 of the row's largest with what comes before it."""
import math

import numpy as np
import pytest
import torch

import paper_2402_15758_gb300 as pkg

EINVAL, ECAPACITY = -1, -3
F32_TOL, ATT_TOL, BF16_TOL = 4e-6, 1e-5, 4e-3


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2402_15758_gb300 import build
    build.build()
    pkg.load()


def _gen(*seed):
    return torch.Generator(device="cuda").manual_seed(int(np.random.default_rng(seed).integers(1 << 31)))


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rel_rows(a, ref):
    a, ref = a.double(), ref.double()
    assert a.shape == ref.shape
    return float(((a - ref).abs() / ref.abs().amax(-1, keepdim=True).clamp(min=1e-30)).max())


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------
# linear
# ---------------------------------------------------------------------------------------
def _weights(g, n, k, group, zeros):
    groups = -(-k // group)
    code = torch.randint(0, 16, (n, k), generator=g, device="cuda")
    scale = (0.001 + 0.02 * torch.rand(n, groups, generator=g, device="cuda")).to(torch.bfloat16)
    scale = scale * torch.where(torch.rand(n, groups, generator=g, device="cuda") < 0.1, -1, 1).to(torch.bfloat16)
    zero = torch.randint(0, 16, (n, groups), generator=g, device="cuda").to(torch.uint8) if zeros else None
    per = lambda t: t.double().repeat_interleave(group, 1)[:, :k]  # noqa: E731
    dense = (code.double() - (per(zero) if zeros else 8)) * per(scale)
    packed = (code[:, 0::2] | code[:, 1::2] << 4).to(torch.uint8).contiguous()
    return packed, scale.contiguous(), zero, dense


LINEARS = [(1, 1, 32, 32), (1, 16, 64, 64), (1, 4097, 4096, 128), (2, 100, 1056, 128), (5, 1000, 544, 32), (8, 333, 2080, 64),
           (9, 4100, 1024, 128), (16, 250, 11008, 128), (17, 129, 96, 64), (24, 128, 160, 32), (33, 300, 4128, 128),
           (64, 1536, 1024, 128), (64, 520, 2048, 64), (65, 400, 1504, 32), (100, 1000, 768, 128), (128, 257, 512, 32),
           (129, 130, 1120, 64), (200, 2050, 4096, 128), (256, 129, 12288, 64), (300, 700, 544, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,group", LINEARS)
@pytest.mark.parametrize("kind", ["bf16", "split", "fp32"])
def test_linear_w4(M, N, K, group, kind):
    g = _gen(M, N, K, group)
    zeros = (M + N) % 3 != 0
    W, scale, zero, dense = _weights(g, N, K, group, zeros)
    wide = torch.zeros(M, K + 32, device="cuda")
    wide[:, :K] = _normal(g, M, K)
    x, lo = wide[:, :K], None
    value = x.double()
    if kind != "fp32":
        hi = wide.to(torch.bfloat16)
        x, value = hi[:, :K], hi[:, :K].double()
        if kind == "split":
            low = (wide - hi.float()).to(torch.bfloat16)
            lo, value = low[:, :K], value + low[:, :K].double()
    ref = value @ dense.T
    Y = torch.full((M, N + 3), float("nan"), device="cuda")
    pkg.op_linear_w4(x, W, scale, Y[:, :N], zeros=zero, group=group, out_f32=True, X_lo=lo)
    first = Y.clone()
    assert _rel_rows(Y[:, :N], ref) <= F32_TOL
    assert torch.isnan(Y[:, N:]).all()
    pkg.op_linear_w4(x, W, scale, Y[:, :N], zeros=zero, group=group, out_f32=True, X_lo=lo)
    assert torch.equal(first[:, :N], Y[:, :N])  # no sum in arrival order
    Y = _normal(g, M, N)
    want = Y.double() + ref
    pkg.op_linear_w4(x, W, scale, Y, zeros=zero, group=group, epi=2, X_lo=lo)
    assert _rel_rows(Y, want) <= F32_TOL
    if kind != "fp32":
        Y = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
        pkg.op_linear_w4(x, W, scale, Y, zeros=zero, group=group, epi=1, X_lo=lo)
        assert _rel_rows(Y, ref * torch.sigmoid(ref)) <= BF16_TOL
    pkg.op_sync()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "split", "fp32"])
@pytest.mark.parametrize("M,N,K,group", [(1, 4096, 12288, 128), (3, 1028, 11488, 32), (8, 700, 2592, 64), (40, 700, 8192, 128)])
def test_linear_w4_fp32_results_keep_their_bits(M, N, K, group, kind):
    # Two fp16 terms hold an activation to 2^-22, and a chain of 16 sums that each cut off 2^-24 of a group's sum, always
    # toward zero, can add 2^-20 at worst; independent groups average that to well under 2^-21 in the norm.
    g = _gen(M, N, K, 5)
    W, scale, zero, dense = _weights(g, N, K, group, True)
    x, lo = _normal(g, M, K), None
    value = x.double()
    if kind != "fp32":
        hi = x.to(torch.bfloat16)
        lo = (x - hi.float()).to(torch.bfloat16) if kind == "split" else None
        x, value = hi, hi.double() + (lo.double() if lo is not None else 0.0)
    Y = torch.zeros(M, N, device="cuda")
    pkg.op_linear_w4(x, W, scale, Y, zeros=zero, group=group, out_f32=True, X_lo=lo)
    ref = value @ dense.T
    assert float((Y.double() - ref).norm() / ref.norm()) <= 2.0 ** -22 + 2.0 ** -21


@pytest.mark.gpu
def test_linear_w4_extreme_activations():
    # a token that is not finite spoils its own row alone; very large and very small ones keep their precision
    g = _gen(7)
    for M in (5, 40):
        W, scale, zero, dense = _weights(g, 300, 512, 64, True)
        x = _normal(g, M, 512).to(torch.bfloat16)
        x[1] *= 1e30
        x[2] *= 1e-30
        x[3, 100] = float("inf")
        Y = torch.zeros(M, 300, device="cuda")
        pkg.op_linear_w4(x, W, scale, Y, zeros=zero, group=64, out_f32=True)
        ref = x.double() @ dense.T
        rest = [i for i in range(M) if i != 3]
        assert _rel_rows(Y[rest], ref[rest]) <= F32_TOL
        assert not torch.isfinite(Y[3]).all()


@pytest.mark.gpu
def test_w4_round_is_within_half_a_step():
    w = _normal(_gen(3), 70, 416) * 0.02
    for group in (32, 64, 128):
        packed, scale, zero = pkg.w4_round(w, group)
        eye = torch.eye(416, device="cuda", dtype=torch.bfloat16)
        Y = torch.zeros(416, 70, device="cuda")
        pkg.op_linear_w4(eye, packed, scale, Y, zeros=zero, group=group, out_f32=True)
        step = scale.float().repeat_interleave(group, 1)[:, :416]
        # half a step, and at the ends of a group what rounding its step to bf16 (2^-9 of 15 steps) and its zero cuts off
        assert float(((Y.T - w).abs() / step).max()) <= 0.5 + 0.5 + 15 / 512


# ---------------------------------------------------------------------------------------
# cache
# ---------------------------------------------------------------------------------------
def _round4(x):
    """The rule, in 32 bits: codes, step, base."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    base, step = lo.to(torch.bfloat16), ((hi - lo) / 15).to(torch.bfloat16)
    code = torch.round((x - base.float()) / step.float()).clamp(0, 15)
    return torch.where(step > 0, code, torch.zeros_like(code)), step, base


def _stands_for(x):
    code, step, base = _round4(x.float())
    return base.double() + step.double() * code.double()


class Cache:
    """A pool with shuffled pages, filled with `rows[b]` rows of each sequence; the pages' other slots hold
    bytes that are no numbers as steps and bases."""

    def __init__(self, g, rows, G, hd, size=1.0, spare=0, pages=None):
        self.rows, self.G, self.hd, self.B = rows, G, hd, len(rows)
        self.pages = pages or max(1, (max(rows) + 15) // 16 + 1)
        blocks = self.B * (self.pages + spare)
        order = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
        self.table = order[:self.B * self.pages].view(self.B, self.pages).contiguous()
        self.spare = order[self.B * self.pages:].view(self.B, spare).contiguous()
        self.pool = pkg.kv4_pool(blocks, G, hd)
        self.pool.fill_(255)
        most = max(1, max(rows))
        offsets = _normal(g, G, hd)
        self.k = (_normal(g, self.B, most, G, hd) + offsets) * size
        self.v = _normal(g, self.B, most, G, hd) * torch.exp(_normal(g, self.B, most, G, 1)) * size
        pkg.op_kv4_append(self.k.view(self.B * most, -1), self.v.view(self.B * most, -1), self.pool, self.table,
                          torch.zeros(self.B, dtype=torch.int32, device="cuda"), most, hd, counts=_ints(rows))
        self.k, self.v = _stands_for(self.k), _stands_for(self.v)


@pytest.mark.gpu
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,rows,G", [(1, 1, 1), (3, 5, 2), (2, 47, 8), (1, 300, 5)])
def test_append_and_read(hd, dtype, B, rows, G):
    g = _gen(hd, B, rows, G)
    pages = rows // 16 + 4
    table = torch.randperm(B * pages, generator=g, device="cuda").to(torch.int32).view(B, pages).contiguous()
    slot0 = torch.randint(0, 30, (B,), generator=g, device="cuda").to(torch.int32)
    counts = torch.randint(0, rows + 1, (B,), generator=g, device="cuda").to(torch.int32)
    counts[0] = rows
    pool = pkg.kv4_pool(B * pages, G, hd)
    pool.fill_(255)
    k = (_normal(g, B * rows, G * hd + 8) * 3).to(dtype)
    v = (_normal(g, B * rows, G * hd) * torch.exp(3 * _normal(g, B * rows, 1))).to(dtype)
    k[0, :hd] = 1.25  # a row of equal values
    k[0, hd:2 * hd] *= 1e-20 if G > 1 else 1
    pkg.op_kv4_append(k[:, :G * hd], v, pool, table, slot0, rows, hd, counts=counts)
    before = pool.clone()
    kb = torch.full((B * rows, G * hd + 4), -7.0, device="cuda", dtype=dtype)
    vb = torch.full((B * rows, G * hd), -7.0, device="cuda", dtype=dtype)
    pkg.op_kv4_read(pool, table, slot0, rows, hd, kb[:, :G * hd], vb, counts=counts)
    pkg.op_sync()
    assert torch.equal(pool, before)
    there = (torch.arange(rows, device="cuda")[None] < counts[:, None]).view(-1, 1)
    for got, x in ((kb[:, :G * hd], k[:, :G * hd]), (vb, v)):
        want = _stands_for(x.reshape(B * rows, G, hd)).view(B * rows, -1).to(torch.float32).to(dtype)
        assert torch.equal(got, torch.where(there, want, torch.full_like(want, -7)))
    assert (kb[:, G * hd:] == -7).all()
    # the second half again, on its own: neighbours that share a word of V stay as they are
    if rows > 1:
        half = rows // 2
        at = torch.arange(half, rows, device="cuda")
        kk = k.view(B, rows, -1)[:, half:].reshape(B * len(at), -1)
        vv = v.view(B, rows, -1)[:, half:].reshape(B * len(at), -1)
        pkg.op_kv4_append(kk[:, :G * hd], vv, pool, table, slot0 + half, rows - half, hd, counts=(counts - half).clamp(min=0))
        assert torch.equal(pool, before)


@pytest.mark.gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_append_rows_that_are_not_finite(hd):
    rows = torch.zeros(6, hd, device="cuda") + 1
    rows[0, 3] = float("nan")
    rows[1, hd - 1] = float("inf")
    rows[2, 0] = -float("inf")
    rows[3, 0], rows[3, 1] = 3e38, -3e38  # its range overflows
    rows[4, 5] = 1e-42                    # the rest are 1
    rows[5] = 0
    pool, table, zero = pkg.kv4_pool(1, 1, hd), _ints([[0]]), _ints([0])
    pkg.op_kv4_append(rows, rows.flip(0).contiguous(), pool, table, zero, 6, hd)
    k, v = torch.zeros_like(rows), torch.zeros_like(rows)
    pkg.op_kv4_read(pool, table, zero, 6, hd, k, v)
    assert torch.isnan(k[:4]).all() and torch.isnan(v[2:]).all()
    assert torch.isfinite(k[4:]).all() and (k[5] == 0).all() and torch.equal(v[:2], k[4:].flip(0))


# ---------------------------------------------------------------------------------------
# attention and weight sums
# ---------------------------------------------------------------------------------------
def _masks(kind, n, r):
    out = []
    for i in range(n):
        if kind == "tree":
            parent = int(r.integers(0, i)) if i else -1
            out.append((out[parent] if parent >= 0 else 0) | 1 << i)
        elif kind == "chain":
            out.append((1 << (i + 1)) - 1)
        else:  # none: no local row is seen
            out.append(0)
    return out


def _anc(masks):
    return torch.from_numpy(np.array(masks, dtype=np.uint64).view(np.int64)).cuda()


def _probabilities(cache, q, ctx, masks, nq, q_local0, n_local, H, q_rows):
    """Per sequence: logits [H][nq][slots], -inf where nothing is seen."""
    out = []
    for b in range(cache.B):
        n = ctx[b] + n_local
        x = q[b * q_rows:b * q_rows + nq].double().view(nq, H, cache.hd).transpose(0, 1)
        k = cache.k[b, :n].transpose(0, 1).repeat_interleave(H // cache.G, 0)
        z = x @ k.transpose(1, 2) / math.sqrt(cache.hd)
        for i in range(nq):
            hidden = [ctx[b] + j for j in range(n_local) if not masks[q_local0 + i] >> j & 1]
            z[:, i, hidden] = -math.inf
        out.append(z)
    return out


#    ctx per sequence          G  H   hd   nq  ql0 n_local mask
ATTENTIONS = [
    ([0], 1, 1, 64, 1, 0, 0, "none"),                # nothing to see
    ([1], 2, 2, 128, 1, 0, 0, "none"),
    ([0, 17], 2, 4, 128, 2, 0, 2, "none"),           # the first sequence's rows see nothing
    ([15], 4, 4, 64, 1, 0, 1, "chain"),
    ([16], 3, 3, 128, 4, 0, 4, "chain"),
    ([31, 0, 5], 1, 8, 128, 3, 2, 5, "chain"),       # queries start at local row 2
    ([100], 2, 14, 128, 5, 0, 5, "tree"),            # 35 rows a group
    ([513], 4, 32, 64, 1, 0, 1, "chain"),
    ([300, 77], 8, 8, 128, 64, 0, 64, "tree"),
    ([1000], 4, 4, 128, 63, 1, 64, "chain"),
    ([5000], 2, 2, 128, 1, 0, 0, "none"),
    ([2049, 130, 900, 0, 1], 2, 4, 64, 16, 0, 16, "tree"),
]


def _setup(case, seed, size=1.0, qs=1.5):
    ctx, G, H, hd, nq, ql0, n_local, mask = case
    g, r = _gen(seed, len(ctx), G, H, nq), np.random.default_rng(seed)
    cache = Cache(g, [n + n_local for n in ctx], G, hd, size)
    masks = _masks(mask, max(ql0 + nq, n_local, 1), r)
    q_rows = nq + 1
    q = _normal(g, len(ctx) * q_rows, H * hd + 4)[:, :H * hd] * (qs / size)
    return cache, masks, q, q_rows


@pytest.mark.gpu
@pytest.mark.parametrize("case", ATTENTIONS)
@pytest.mark.parametrize("splits", [0, 1, 7])
@pytest.mark.parametrize("form", ["f32", "pair", "bf16"])
def test_attention_kv4(case, splits, form):
    ctx, G, H, hd, nq, ql0, n_local, _ = case
    cache, masks, q, q_rows = _setup(case, 11)
    if form == "bf16":
        q = q.to(torch.bfloat16)
    B, width = len(ctx), H * hd
    ref = torch.zeros(B, nq, width, dtype=torch.float64, device="cuda")
    lse_ref = torch.zeros(B, nq, H, dtype=torch.float64, device="cuda")
    for b, z in enumerate(_probabilities(cache, q, ctx, masks, nq, ql0, n_local, H, q_rows)):
        v = cache.v[b, :ctx[b] + n_local].transpose(0, 1).repeat_interleave(H // G, 0)
        p = torch.softmax(z, -1).nan_to_num(0.0)
        ref[b] = (p @ v).transpose(0, 1).reshape(nq, width)
        lse_ref[b] = torch.logsumexp(z, -1).T
    out = torch.full((B * q_rows, width + 5), -7.0, device="cuda", dtype=torch.float32 if form == "f32" else torch.bfloat16)
    lo = torch.full_like(out, -7.0) if form == "pair" else None
    lse = torch.full((B * q_rows, H), -7.0, device="cuda")
    pkg.op_attention_kv4(q, cache.pool, cache.table, _ints(ctx), _anc(masks), out[:, :width], nq, ql0, n_local, q_rows, H, hd,
                         out_lo=lo, lse=lse if form != "bf16" else None, splits=splits)
    pkg.op_sync()
    got = out[:, :width].float().view(B, q_rows, width)
    if lo is not None:
        got = got + lo[:, :width].float().view(B, q_rows, width)
    tol = BF16_TOL if form == "bf16" else ATT_TOL
    assert _rel_rows(got[:, :nq].reshape(B, nq, H, hd), ref.view(B, nq, H, hd)) <= tol
    assert (got[:, nq:] == (-14 if lo is not None else -7)).all()  # rows that are not queries
    assert (out[:, width:] == -7).all()
    if form != "bf16":
        got = lse.view(B, q_rows, H)[:, :nq].double()
        empty = torch.isinf(lse_ref)
        assert torch.equal(empty, torch.isinf(got))
        assert float((got - lse_ref)[~empty].abs().max() if (~empty).any() else 0) <= ATT_TOL * 10  # of logits up to about 20


# batches whose pages are dealt by their lengths: fewer slots of the grid than every sequence could use
RAGGED = [
    ([2049, 0, 130, 900, 1], 32, 32, 64, 1, 0, 1, "chain"),
    ([1900, 0, 17], 40, 40, 128, 2, 0, 0, "none"),        # a sequence that sees nothing
    ([700, 3, 1500, 64], 16, 16, 128, 40, 0, 40, "tree"),
    ([40 * i for i in range(32)], 8, 16, 128, 2, 0, 2, "chain"),
    ([1500] + [0] * 30 + [9], 16, 16, 64, 1, 0, 1, "chain"),
    ([30 * i for i in range(33)], 8, 8, 64, 1, 0, 1, "chain"),  # more sequences than are dealt
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", RAGGED)
@pytest.mark.parametrize("form", ["f32", "pair", "bf16"])
def test_attention_kv4_ragged(case, form):
    test_attention_kv4(case, 0, form)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [1e-12, 1e-3, 1e6])
def test_attention_kv4_any_size_of_values(size):
    case = ([200], 2, 4, 128, 3, 0, 3, "chain")
    cache, masks, q, q_rows = _setup(case, 5, size)
    out = torch.zeros(q_rows, 4 * 128, device="cuda")
    pkg.op_attention_kv4(q, cache.pool, cache.table, _ints([200]), _anc(masks), out, 3, 0, 3, q_rows, 4, 128)
    z = _probabilities(cache, q, [200], masks, 3, 0, 3, 4, q_rows)[0]
    v = cache.v[0, :203].transpose(0, 1).repeat_interleave(2, 0)
    ref = (torch.softmax(z, -1) @ v).transpose(0, 1)
    assert _rel_rows(out[:3].view(3, 4, 128), ref) <= ATT_TOL


@pytest.mark.gpu
def test_attention_kv4_peaked_rows():
    # logits of several hundred: one key takes nearly all, the running maximum is raised many times
    case = ([700], 1, 2, 128, 4, 0, 4, "chain")
    cache, masks, q, q_rows = _setup(case, 8, qs=40.0)
    out = torch.zeros(q_rows, 2 * 128, device="cuda")
    pkg.op_attention_kv4(q, cache.pool, cache.table, _ints([700]), _anc(masks), out, 4, 0, 4, q_rows, 2, 128)
    z = _probabilities(cache, q, [700], masks, 4, 0, 4, 2, q_rows)[0]
    ref = (torch.softmax(z, -1) @ cache.v[0, :704].transpose(0, 1).repeat_interleave(2, 0)).transpose(0, 1)
    # a logit of size Z is known to 2^-22 Z or so
    assert _rel_rows(out[:4].view(4, 2, 128), ref) <= ATT_TOL + float(z[z.isfinite()].abs().max()) * 2.0 ** -20


@pytest.mark.gpu
@pytest.mark.parametrize("case", ATTENTIONS)
@pytest.mark.parametrize("weighted", [False, True])
def test_score_kv4(case, weighted):
    ctx, G, H, hd, nq, ql0, n_local, _ = case
    cache, masks, q, q_rows = _setup(case, 23)
    B = len(ctx)
    lse = torch.zeros(B * q_rows, H, device="cuda")
    weight = torch.rand(B * q_rows, device="cuda", generator=_gen(4)) * (torch.rand(B * q_rows, device="cuda", generator=_gen(5)) < 0.7)
    ld = cache.pages * 16
    scores = torch.rand(B, G, ld, device="cuda", generator=_gen(6))
    want = scores.double()
    for b, z in enumerate(_probabilities(cache, q, ctx, masks, nq, ql0, n_local, H, q_rows)):
        lse[b * q_rows:b * q_rows + nq] = torch.logsumexp(z, -1).T.float()
        p = torch.exp(z - lse[b * q_rows:b * q_rows + nq].T[:, :, None].double()).nan_to_num(0.0)
        if weighted:
            p = p * weight[b * q_rows:b * q_rows + nq, None].double()
        want[b, :, :ctx[b] + n_local] += p.view(G, H // G * nq, -1).sum(1)
    if weighted:
        lse[weight == 0] = float("nan")  # rows that do not count
    pkg.op_kv4_score(q, lse, cache.pool, cache.table, _ints(ctx), _anc(masks), scores, nq, ql0, n_local, q_rows, H, hd,
                     weight=weight if weighted else None)
    pkg.op_sync()
    assert _rel_rows(scores, want) <= ATT_TOL
    for b in range(B):  # slots without a row are not touched
        assert torch.equal(scores[b, :, ctx[b] + n_local:].double(), want[b, :, ctx[b] + n_local:])


@pytest.mark.gpu
@pytest.mark.parametrize("case", RAGGED)
def test_score_kv4_ragged(case):
    test_score_kv4(case, True)


# ---------------------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------------------
EVICTIONS = [([40], 1, 64, 24, 8), ([272], 4, 64, 256, 64), ([16, 300, 0, 129], 2, 128, 128, 0), ([1000, 1], 3, 128, 37, 37),
             ([5000], 2, 128, 2500, 100), ([2048], 1, 64, 1, 0), ([3000], 2, 64, 1, 1), ([70000], 1, 64, 33000, 17)]


@pytest.mark.gpu
@pytest.mark.parametrize("ctx,G,hd,budget,recent", EVICTIONS)
@pytest.mark.parametrize("kind", ["plain", "ties", "odd"])
def test_evict(ctx, G, hd, budget, recent, kind):
    g = _gen(budget, recent, G)
    B = len(ctx)
    spare = (budget + 15) // 16
    cache = Cache(g, ctx, G, hd, spare=spare)
    ld = max(cache.pages * 16, 1)
    scores = torch.exp(2 * _normal(g, B, G, ld))
    if kind == "ties":
        scores = torch.randint(0, 3, (B, G, ld), generator=g, device="cuda").float() * torch.where(
            torch.rand(B, G, ld, generator=g, device="cuda") < 0.5, -1.0, 1.0)  # 0 and -0 are equal
    if kind == "odd":
        some = torch.rand(B, G, ld, generator=g, device="cuda")
        scores = torch.where(some < 0.1, float("nan"), torch.where(some < 0.2, float("inf"), torch.where(
            some < 0.4, -float("inf"), -scores)))
    kept = torch.full((B, G, budget), -9, dtype=torch.int32, device="cuda")
    out = torch.full((B, G, budget), -9.0, device="cuda")
    n_out = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    before = cache.pool.clone()
    pkg.op_kv4_evict(cache.pool, cache.table, _ints(ctx), scores, budget, recent, cache.spare, kept, out, n_out, hd)
    k = torch.full((B * budget, G * hd), -9.0, device="cuda")
    v = torch.full_like(k, -9.0)
    pkg.op_kv4_read(cache.pool, cache.spare, torch.zeros(B, dtype=torch.int32, device="cuda"), budget, hd, k, v, counts=n_out)
    pkg.op_sync()
    assert n_out.tolist() == [min(n, budget) for n in ctx]
    assert torch.equal(cache.pool[cache.table.view(-1).long()], before[cache.table.view(-1).long()])
    k, v = k.view(B, budget, G, hd), v.view(B, budget, G, hd)
    for b in range(B):
        n = ctx[b]
        for h in range(G):
            x = scores[b, h, :n].double().cpu().numpy() + 0.0
            older = max(0, n - recent) if n > budget else n
            rank = np.where(np.isnan(x), -np.inf, x)
            order = np.lexsort((np.arange(n), np.isnan(x), -rank))[:]
            order = order[order < older][:min(n, budget) - (n - older)]
            want = np.concatenate([np.sort(order), np.arange(older, n)])
            m = len(want)
            assert m == min(n, budget)
            got = kept[b, h].cpu().numpy()
            assert np.array_equal(got[:m], want) and (got[m:] == -1).all()
            at = torch.from_numpy(want).cuda()
            torch.testing.assert_close(out[b, h, :m], scores[b, h, at], rtol=0, atol=0, equal_nan=True)
            assert (out[b, h, m:] == 0).all()
            assert torch.equal(k[b, :m, h].double(), cache.k[b, at, h].float().double())
            assert torch.equal(v[b, :m, h].double(), cache.v[b, at, h].float().double())
            assert (k[b, m:, h] == -9).all()


# ---------------------------------------------------------------------------------------
# large offsets, streams, refusals
# ---------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_offsets_past_32_bits():
    G, hd = 32, 128
    blocks = 70000  # 4.9 GB
    pool = pkg.kv4_pool(blocks, G, hd)
    g = _gen(9)
    table = torch.arange(blocks - 4, blocks, device="cuda").to(torch.int32).view(1, 4).contiguous()
    dst = torch.arange(62000, 62002, device="cuda").to(torch.int32).view(1, 2).contiguous()
    k, v = _normal(g, 50, G * hd), _normal(g, 50, G * hd)
    zero = _ints([0])
    pkg.op_kv4_append(k, v, pool, table, zero, 50, hd)
    q = _normal(g, 1, G * hd)
    out, lse = torch.zeros(1, G * hd, device="cuda"), torch.zeros(1, G, device="cuda")
    pkg.op_attention_kv4(q, pool, table, _ints([50]), None, out, 1, 0, 0, 1, G, hd, lse=lse)
    kk, vv = _stands_for(k.view(50, G, hd)).transpose(0, 1), _stands_for(v.view(50, G, hd)).transpose(0, 1)
    z = (q.double().view(G, 1, hd) @ kk.transpose(1, 2)) / math.sqrt(hd)
    p = torch.softmax(z, -1)
    assert _rel_rows(out.view(G, hd), (p @ vv)[:, 0]) <= ATT_TOL
    scores = torch.zeros(1, G, 64, device="cuda")
    pkg.op_kv4_score(q, lse, pool, table, _ints([50]), None, scores, 1, 0, 0, 1, G, hd)
    assert _rel_rows(scores[0, :, :50], p[:, 0]) <= ATT_TOL
    kept, so, n = torch.zeros(1, G, 20, dtype=torch.int32, device="cuda"), torch.zeros(1, G, 20, device="cuda"), _ints([0])
    pkg.op_kv4_evict(pool, table, _ints([50]), scores, 20, 4, dst, kept, so, n, hd)
    kb, vb = torch.zeros(20, G * hd, device="cuda"), torch.zeros(20, G * hd, device="cuda")
    pkg.op_kv4_read(pool, dst, zero, 20, hd, kb, vb)
    pkg.op_sync()
    for h in (0, 31):
        at = kept[0, h].long()
        assert torch.equal(kb.view(20, G, hd)[:, h].double(), kk[h, at].float().double())
        assert torch.equal(vb.view(20, G, hd)[:, h].double(), vv[h, at].float().double())


@pytest.mark.gpu
def test_calls_on_two_streams():
    case = ([900], 2, 4, 128, 2, 0, 2, "chain")
    made = [_setup(case, s) for s in (31, 32)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros(q.shape[0], 512, device="cuda") for _ in range(20)] for _, _, q, _ in made]
    torch.cuda.synchronize()
    for i in range(20):
        for s, (cache, masks, q, q_rows), o in zip(streams, made, outs):
            with torch.cuda.stream(s):
                anc, n = _anc(masks), _ints([900])
                pkg.op_attention_kv4(q, cache.pool, cache.table, n, anc, o[i], 2, 0, 2, q_rows, 4, 128, splits=5, stream=s)
    torch.cuda.synchronize()
    pkg.op_sync()
    for (cache, masks, q, q_rows), o in zip(made, outs):
        z = _probabilities(cache, q, [900], masks, 2, 0, 2, 4, q_rows)[0]
        ref = (torch.softmax(z, -1) @ cache.v[0, :902].transpose(0, 1).repeat_interleave(2, 0)).transpose(0, 1)
        for x in o:
            assert torch.equal(x, o[0])
        assert _rel_rows(o[0][:2].view(2, 4, 128), ref) <= ATT_TOL


def _status(fn, *a, **k):
    with pytest.raises(pkg.ChimeraError) as e:
        fn(*a, **k)
    return e.value.status


@pytest.mark.gpu
def test_device_side_refusals():
    g = _gen(2)
    k = _normal(g, 4, 128)
    pool, zero = pkg.kv4_pool(2, 1, 128), _ints([0])
    pkg.op_kv4_append(k, k, pool, _ints([[0, 1]]), _ints([30]), 4, 128)  # slots 30..33 of 32
    assert _status(pkg.op_sync) == ECAPACITY
    pkg.op_kv4_append(k, k, pool, _ints([[2, 1]]), zero, 4, 128)  # block 2 of 2
    assert _status(pkg.op_sync) == EINVAL
    q, out = _normal(g, 1, 128), torch.zeros(1, 128, device="cuda")
    pkg.op_attention_kv4(q, pool, _ints([[0, -1]]), _ints([20]), None, out, 1, 0, 0, 1, 1, 128)
    assert _status(pkg.op_sync) == EINVAL
    pkg.op_attention_kv4(q, pool, _ints([[0, 1]]), _ints([33]), None, out, 1, 0, 0, 1, 1, 128)
    assert _status(pkg.op_sync) == ECAPACITY
    pkg.op_attention_kv4(q, pool, _ints([[0, 1]]), _ints([-1]), None, out, 1, 0, 0, 1, 1, 128)
    assert _status(pkg.op_sync) == ECAPACITY
    pkg.op_sync()


def test_host_side_refusals():
    """Every refusal comes before the GPU is touched: addresses here are numbers that nothing reads."""
    lib = pkg.load()
    a = 4096

    def linear(**kw):
        d = dict(dtype=1, epi=0, out_f32=1, M=4, N=8, K=64, group=64, X=a, X_lo=0, ldx=64, W=a, s=a, z=0, Y=a, ldy=8)
        d.update(kw)
        return lib.chimera_op_linear_w4(*d.values(), None)

    for bad in (dict(dtype=2), dict(epi=3), dict(M=0), dict(N=0), dict(K=48), dict(K=0), dict(group=16), dict(group=100), dict(X=0),
                dict(W=0), dict(s=0), dict(Y=0), dict(ldx=56), dict(ldx=65), dict(ldy=7), dict(X=a + 2), dict(W=a + 8),
                dict(X_lo=a + 2), dict(dtype=0, X_lo=a), dict(Y=a + 2)):
        assert linear(**bad) == EINVAL, bad

    def rows(fn, **kw):
        d = dict(dtype=0, batch=1, rows=1, G=1, hd=128, k=a, ldk=128, v=a, ldv=128, pool=a, blocks=1, table=a, pages=1, slot0=a,
                 counts=0)
        d.update(kw)
        return fn(*d.values(), None)

    for fn in (lib.chimera_op_kv4_append, lib.chimera_op_kv4_read):
        for bad in (dict(dtype=2), dict(batch=0), dict(rows=-1), dict(G=0), dict(hd=96), dict(k=0), dict(ldk=127), dict(ldv=100),
                    dict(pool=0), dict(pool=a + 8), dict(blocks=0), dict(table=0), dict(pages=0), dict(slot0=0), dict(v=0), dict(k=a + 2)):
            assert rows(fn, **bad) == EINVAL, bad
        assert rows(fn, rows=0) == 0  # nothing to do

    def attention(**kw):
        d = dict(qd=0, od=0, batch=1, H=4, G=2, hd=128, nq=1, ql0=0, n_local=1, q=a, ldq=512, q_rows=1, pool=a, blocks=1, table=a,
                 pages=1, n_ctx=a, anc=a, out=a, lo=0, ldo=512, lse=0, splits=0)
        d.update(kw)
        return lib.chimera_op_attention_kv4(*d.values(), None)

    for bad in (dict(qd=3), dict(od=2), dict(H=3), dict(G=0), dict(hd=32), dict(nq=0), dict(nq=65, q_rows=65), dict(ql0=-1),
                dict(n_local=65), dict(q=0), dict(ldq=511), dict(q_rows=0), dict(pool=a + 1), dict(n_ctx=0), dict(anc=0), dict(out=0),
                dict(lo=a), dict(ldo=500), dict(splits=-1), dict(splits=65), dict(batch=40000), dict(q=a + 1)):
        assert attention(**bad) == EINVAL, bad

    def score(**kw):
        d = dict(qd=0, batch=1, H=4, G=2, hd=128, nq=1, ql0=0, n_local=1, q=a, ldq=512, q_rows=1, lse=a, weight=0, pool=a, blocks=1,
                 table=a, pages=1, n_ctx=a, anc=a, scores=a, ld=16)
        d.update(kw)
        return lib.chimera_op_kv4_score(*d.values(), None)

    for bad in (dict(lse=0), dict(scores=0), dict(ld=0), dict(H=5), dict(n_ctx=0)):
        assert score(**bad) == EINVAL, bad

    def evict(**kw):
        d = dict(batch=1, G=1, hd=64, pool=a, blocks=4, table=a, pages=2, n_ctx=a, scores=a, ld=32, budget=16, recent=4, dst=a,
                 dst_pages=1, kept=a, out=a, n_out=a)
        d.update(kw)
        return lib.chimera_op_kv4_evict(*d.values(), None)

    for bad in (dict(budget=0), dict(recent=-1), dict(recent=17), dict(dst=0), dict(budget=17), dict(kept=0), dict(out=0), dict(n_out=0),
                dict(scores=0), dict(ld=0), dict(n_ctx=0)):
        assert evict(**bad) == EINVAL, bad
