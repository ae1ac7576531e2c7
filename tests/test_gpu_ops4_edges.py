"""The 4-bit operators at the edges of their range.  Tolerances are those of test_gpu_ops4.py."""
import math

import pytest
import torch

import paper_2402_15758_gb300 as pkg
from test_gpu_ops4 import BF16_TOL, Cache, _anc, _gen, _ints, _normal, _probabilities, _rel_rows, _stands_for


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2402_15758_gb300 import build
    build.build()
    pkg.load()


def _attend(cache, q, ctx, masks, nq, n_local, H, form, splits=0):
    """Output (fp32) and logsumexp (not with bf16 alone) of every query, [B][nq][H][hd] and [B][nq][H]."""
    B, width = cache.B, H * cache.hd
    out = torch.zeros(B * nq, width, device="cuda", dtype=torch.float32 if form == "f32" else torch.bfloat16)
    lo = torch.zeros_like(out) if form == "pair" else None
    lse = torch.zeros(B * nq, H, device="cuda") if form != "bf16" else None
    pkg.op_attention_kv4(q, cache.pool, cache.table, _ints(ctx), _anc(masks), out, nq, 0, n_local, nq, H, cache.hd, out_lo=lo,
                         lse=lse, splits=splits)
    pkg.op_sync()
    got = out.float() + (lo.float() if lo is not None else 0)
    return got.view(B, nq, H, cache.hd), lse.view(B, nq, H) if lse is not None else None


def _reference(cache, q, ctx, masks, nq, n_local, H):
    out, lse = [], []
    for b, z in enumerate(_probabilities(cache, q, ctx, masks, nq, 0, n_local, H, nq)):
        v = cache.v[b, :ctx[b] + n_local].transpose(0, 1).repeat_interleave(H // cache.G, 0)
        out.append((torch.softmax(z, -1).nan_to_num(0.0) @ v).transpose(0, 1))
        lse.append(torch.logsumexp(z, -1).T)
    return torch.stack(out), torch.stack(lse)


def _one_key(cache, q, at, logit, size):
    """Makes the key at slot `at` draw a logit of about `logit` from every query (queries that hardly differ), and its
    V rows `size` times the others'."""
    G, hd = cache.G, cache.hd
    mean = q.view(-1, G, q.shape[1] // (G * hd), hd).mean((0, 2))
    k = mean * (logit * math.sqrt(hd) / mean.square().sum(-1, keepdim=True))
    v = _normal(_gen(at), G, hd) * size
    pkg.op_kv4_append(k.reshape(1, -1), v.reshape(1, -1), cache.pool, cache.table, _ints([at]), 1, hd)
    cache.k[0, at], cache.v[0, at] = _stands_for(k), _stands_for(v)


def _alike(g, nq, H, G, hd):
    """Queries of one direction per kv head, which differ a little."""
    one = _normal(g, 1, G, 1, hd)
    return (one + 0.02 * _normal(g, nq, G, H // G, hd)).reshape(nq, H * hd)

@pytest.mark.gpu
@pytest.mark.parametrize("size", [1e-8, 1e-10, 1e-11, 1e-13])
@pytest.mark.parametrize("at,nq", [(3, 40), (299, 40), (150, 9)])
def test_a_small_row_of_much_weight(size, at, nq):
    # Most of the weight is its own, and the result is what that leaves of the others'.  Of the forms, the one whose weights
    # have one term (bf16 alone, more than 8 rows); the others' sums never took a rounded weight.
    G, H, hd = 2, 4, 128
    g = _gen(47, at, nq)
    cache = Cache(g, [300], G, hd)
    q = _alike(g, nq, H, G, hd)
    _one_key(cache, q, at, 14.0, size)
    ref, _ = _reference(cache, q, [300], [0] * nq, nq, 0, H)
    for splits in (0, 1):
        got, _ = _attend(cache, q, [300], [0] * nq, nq, 0, H, "bf16", splits)
        assert _rel_rows(got, ref) <= BF16_TOL
