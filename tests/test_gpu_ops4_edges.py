"""The 4-bit operators at the edges of their range.  Tolerances are those of test_gpu_ops4.py."""
import math

import numpy as np
import pytest
import torch

import paper_2402_15758_gb300 as pkg
from test_gpu_ops4 import (ATT_TOL, BF16_TOL, ECAPACITY, EINVAL, Cache, _anc, _gen, _ints, _masks, _normal, _probabilities, _rel_rows,
                           _stands_for, _status, _weights)


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


def _spoil(cache, b, slot, word):
    """The step and base (the halves of `word`) of a slot's K and V, and all of its K codes, in every head."""
    at, row = 16 * cache.hd + 4 * (slot % 16), slot % 16
    page = cache.pool[int(cache.table[b, slot // 16])]
    four = torch.from_numpy(np.array([word], dtype=np.uint32).view(np.uint8)).cuda()
    page[:, at:at + 4] = four
    page[:, at + 64:at + 68] = four
    page[:, row * cache.hd // 2:(row + 1) * cache.hd // 2] = 255


#    ctx per sequence   G   H   hd  nq  n_local
HIDDEN = [([20], 2, 4, 128, 5, 5), ([0], 1, 1, 64, 3, 3), ([513], 4, 32, 64, 1, 4), ([300, 77], 8, 8, 128, 64, 64),
          ([1000], 4, 4, 128, 33, 40), ([1900, 0, 17], 40, 40, 128, 2, 3), ([700, 3, 1500, 64], 16, 16, 64, 40, 40)]


@pytest.mark.gpu
@pytest.mark.parametrize("case", HIDDEN)
@pytest.mark.parametrize("word", [0xffffffff, 0x7f807f80, 0xff80ff80, 0x00007e00, 0x7e007e00], ids=["nan", "inf", "-inf", "step", "large"])
@pytest.mark.parametrize("form", ["f32", "pair", "bf16"])
def test_hidden_local_rows_are_no_part_of_a_result(case, word, form):
    ctx, G, H, hd, nq, n_local = case
    g, r = _gen(41, len(ctx), G, nq), np.random.default_rng(41)
    cache = Cache(g, [n + n_local for n in ctx], G, hd)
    masks = _masks("tree", n_local, r)
    q = _normal(g, len(ctx) * nq, H * hd) * 1.5
    ref, lse_ref = _reference(cache, q, ctx, masks, nq, n_local, H)
    bad = sorted({n_local - 1, n_local // 2, n_local // 3} - {0})
    for b in range(len(ctx)):
        for j in bad:
            _spoil(cache, b, ctx[b] + j, word)
    clean = [i for i in range(nq) if not any(masks[i] >> j & 1 for j in bad)]
    assert clean  # the root at least
    for splits in (0, 1, 3):
        got, lse = _attend(cache, q, ctx, masks, nq, n_local, H, form, splits)
        assert _rel_rows(got[:, clean], ref[:, clean]) <= (BF16_TOL if form == "bf16" else ATT_TOL)
        if lse is not None:
            assert float((lse.double() - lse_ref)[:, clean].abs().max()) <= ATT_TOL * 10


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["f32", "pair", "bf16"])
@pytest.mark.parametrize("nq", [3, 24])
def test_a_row_without_numbers_reaches_those_that_see_it_alone(form, nq):
    # appended as the library does it: V of local row 1 holds an infinity
    ctx, G, H, hd = [90], 2, 4, 128
    g = _gen(43, nq)
    cache = Cache(g, [90 + nq], G, hd)
    masks = [1] + [1 | 1 << i for i in range(1, nq)]  # children of the root
    q = _normal(g, nq, H * hd)
    ref, lse_ref = _reference(cache, q, ctx, masks, nq, nq, H)
    k, v = _normal(g, 1, G * hd), _normal(g, 1, G * hd)
    v[:, [5, hd + 5]] = float("inf")
    pkg.op_kv4_append(k, v, cache.pool, cache.table, _ints([91]), 1, hd)
    cache.k[0, 91] = _stands_for(k.view(G, hd))
    lse_ref[:, 1] = _reference(cache, q, ctx, masks, nq, nq, H)[1][:, 1]
    got, lse = _attend(cache, q, ctx, masks, nq, nq, H, form)
    rest = [i for i in range(nq) if i != 1]
    assert torch.isnan(got[:, 1]).all()
    assert _rel_rows(got[:, rest], ref[:, rest]) <= (BF16_TOL if form == "bf16" else ATT_TOL)
    if lse is not None:
        assert float((lse.double() - lse_ref).abs().max()) <= ATT_TOL * 10


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


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["f32", "pair", "bf16"])
@pytest.mark.parametrize("size", [1e6, 1e12, 1e15])
@pytest.mark.parametrize("at,nq", [(3, 1), (3, 40), (299, 2), (299, 40), (150, 9)])
def test_a_large_row_of_little_weight(form, size, at, nq):
    # its weight, exp(-60) of the others', times its size is nothing beside them
    G, H, hd = 2, 4, 128
    g = _gen(47, at, nq)
    cache = Cache(g, [300], G, hd)
    q = _alike(g, nq, H, G, hd)
    _one_key(cache, q, at, -60.0, size)
    ref, _ = _reference(cache, q, [300], [0] * nq, nq, 0, H)
    for splits in (0, 1):
        got, _ = _attend(cache, q, [300], [0] * nq, nq, 0, H, form, splits)
        assert _rel_rows(got, ref) <= (BF16_TOL if form == "bf16" else ATT_TOL)


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["f32", "pair", "bf16"])
@pytest.mark.parametrize("nq", [2, 40])
@pytest.mark.parametrize("size", [1e-26, 1e-9, 1.0, 1e12, 1e30])
def test_rows_of_equal_values_among_others(form, nq, size):
    # rows of equal values have step 0; a zero row, and one of 1e20 times the others' size, which all others vanish beside
    G, H, hd = 2, 4, 64
    g = _gen(53, nq)
    cache = Cache(g, [200], G, hd)
    q = _normal(g, nq, H * hd)
    v = _normal(g, 200, G, hd)
    v[::3] = v[::3, :, :1]
    v[5:40] = 0
    at = [s for s in range(200) if s % 3 == 0]
    for large in (False, True):
        if large and size > 1e15:
            continue
        x = v * size
        if large:
            x[at[-4]] = 1e20 * size
        pkg.op_kv4_append(cache.k[0].float().reshape(200, -1), x.view(200, -1), cache.pool, cache.table, _ints([0]), 200, hd)
        cache.k[0], cache.v[0] = _stands_for(cache.k[0]), _stands_for(x)
        ref, _ = _reference(cache, q, [200], [0] * nq, nq, 0, H)
        for splits in (0, 1):
            got, _ = _attend(cache, q, [200], [0] * nq, nq, 0, H, form, splits)
            assert _rel_rows(got, ref) <= (BF16_TOL if form == "bf16" else ATT_TOL)
    pkg.op_kv4_append(cache.k[0].float().reshape(200, -1), torch.zeros(200, G * hd, device="cuda"), cache.pool, cache.table, _ints([0]),
                      200, hd)
    assert (_attend(cache, q, [200], [0] * nq, nq, 0, H, form)[0] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 3, -2 ** 31, None])
@pytest.mark.parametrize("batch", [1, 12])
def test_lengths_past_the_table_are_reported(n, batch):
    # n + n_local passes 32 bits, or the table by one slot (None); the other sequences of a (dealt) batch are as they were
    G, hd, n_local = 16, 64, 4
    g = _gen(61, batch)
    cache = Cache(g, [29] + [500] * (batch - 1), G, hd, pages=3 if batch == 1 else 40)
    slots = cache.pages * 16
    ctx = [25] + [496] * (batch - 1)
    masks = _masks("chain", n_local, None)
    q = _normal(g, batch * n_local, G * hd)
    ref, _ = _reference(cache, q, ctx, masks, n_local, n_local, G)
    lengths = _ints([slots - n_local + 1 if n is None else n] + ctx[1:])
    out, lse = torch.zeros(batch * n_local, G * hd, device="cuda"), torch.zeros(batch * n_local, G, device="cuda")
    pkg.op_attention_kv4(q, cache.pool, cache.table, lengths, _anc(masks), out, n_local, 0, n_local, n_local, G, hd, lse=lse)
    assert _status(pkg.op_sync) == ECAPACITY
    if batch > 1:
        assert _rel_rows(out.view(batch, n_local, G, hd)[1:], ref[1:]) <= ATT_TOL
    scores = torch.zeros(batch, G, slots, device="cuda")
    pkg.op_kv4_score(q, lse, cache.pool, cache.table, lengths, _anc(masks), scores, n_local, 0, n_local, n_local, G, hd)
    assert _status(pkg.op_sync) == ECAPACITY


def test_tensors_of_other_types_and_strides_are_refused():
    """Before the library is called: each of these would be read or written as something that it is not."""
    f32, bf16, f16, f64, u8, i32, i64 = (torch.float32, torch.bfloat16, torch.float16, torch.float64, torch.uint8, torch.int32,
                                         torch.int64)
    z = torch.zeros

    def linear(**kw):
        d = dict(X=z(4, 64, dtype=bf16), W=z(8, 32, dtype=u8), scales=z(8, 1, dtype=bf16), Y=z(4, 8, dtype=bf16), zeros=z(8, 1, dtype=u8),
                 group=64)
        d.update(kw)
        return pkg.op_linear_w4, d

    def rows(fn=pkg.op_kv4_append, **kw):
        d = dict(k=z(3, 128), v=z(3, 128), pool=z(1, 1, 16 * 128 + 128, dtype=u8), page_table=z(1, 1, dtype=i32), slot0=z(1, dtype=i32),
                 rows=3, head_dim=128)
        d.update(kw)
        return fn, d

    def queries(fn, **kw):
        d = dict(q=z(2, 256), pool=z(1, 2, 16 * 128 + 128, dtype=u8), page_table=z(1, 1, dtype=i32), n_ctx=z(1, dtype=i32),
                 anc=z(2, dtype=i64), lse=z(2, 2), nq=2, q_local0=0, n_local=2, q_rows=2, n_heads=2, head_dim=128)
        d.update(dict(out=z(2, 256)) if fn is pkg.op_attention_kv4 else dict(scores=z(1, 2, 16)))
        d.update(kw)
        return fn, d

    def evict(**kw):
        d = dict(pool=z(2, 2, 16 * 128 + 128, dtype=u8), page_table=z(2, 1, dtype=i32), n_ctx=z(2, dtype=i32), scores=z(2, 2, 16), budget=8,
                 recent=2, dst_table=z(2, 1, dtype=i32), kept=z(2, 2, 8, dtype=i32), scores_out=z(2, 2, 8), n_out=z(2, dtype=i32),
                 head_dim=128)
        d.update(kw)
        return pkg.op_kv4_evict, d

    wide = z(4, 300, dtype=bf16)
    bad = [linear(X=z(4, 64, dtype=f16)), linear(X=z(4, 64, dtype=f64)), linear(X=z(64, 4, dtype=bf16).t()), linear(Y=z(4, 8)),
           linear(Y=z(4, 8, dtype=f16)), linear(out_f32=True), linear(epi=2), linear(X=z(4, 64)), linear(Y=z(8, 4, dtype=bf16).t()),
           linear(W=z(8, 32, dtype=f32)), linear(W=z(32, 8, dtype=u8).t()), linear(scales=z(8, 1)), linear(scales=z(8, 1, dtype=f16)),
           linear(zeros=z(8, 1, dtype=i32)), linear(X_lo=z(4, 64)), linear(X_lo=wide[:, :64])]
    for fn in (pkg.op_kv4_append, pkg.op_kv4_read):
        bad += [rows(fn, k=z(3, 128, dtype=f16), v=z(3, 128, dtype=f16)), rows(fn, k=z(3, 128, dtype=f64), v=z(3, 128, dtype=f64)),
                rows(fn, v=z(3, 128, dtype=bf16)), rows(fn, k=z(3, 128, dtype=bf16)), rows(fn, k=z(128, 3).t()),
                rows(fn, v=z(3, 256)[:, ::2]), rows(fn, page_table=z(1, 1, dtype=i64)), rows(fn, page_table=z(2, 2, dtype=i32)[:, :1]),
                rows(fn, slot0=z(1, dtype=i64)), rows(fn, counts=z(1, dtype=i64)), rows(fn, pool=z(1, 1, 16 * 128 + 128, dtype=f32))]
    for fn in (pkg.op_attention_kv4, pkg.op_kv4_score):
        bad += [queries(fn, q=z(2, 256, dtype=f16)), queries(fn, q=z(2, 256, dtype=f64)), queries(fn, q=z(256, 2).t()),
                queries(fn, lse=z(2, 2, dtype=bf16)), queries(fn, lse=z(2, 4)[:, ::2]), queries(fn, anc=z(2, dtype=i32)),
                queries(fn, n_ctx=z(1, dtype=i64)), queries(fn, page_table=z(1, 1, dtype=i64)),
                queries(fn, pool=z(1, 2, 16 * 128 + 128, dtype=i32))]
    bad += [queries(pkg.op_attention_kv4, out=z(2, 256, dtype=f16)), queries(pkg.op_attention_kv4, out=z(256, 2).t()),
            queries(pkg.op_attention_kv4, out=z(2, 256, dtype=bf16), out_lo=z(2, 256)),
            queries(pkg.op_attention_kv4, out=z(2, 256, dtype=bf16), out_lo=wide[:2, :256])]
    two = dict(q=z(4, 256), n_ctx=z(2, dtype=i32), page_table=z(2, 1, dtype=i32), lse=z(4, 2))
    bad += [queries(pkg.op_kv4_score, scores=z(1, 2, 16, dtype=f64)), queries(pkg.op_kv4_score, scores=z(1, 2, 32)[:, :, ::2]),
            queries(pkg.op_kv4_score, scores=z(2, 3, 16)[:, 1:], **two), queries(pkg.op_kv4_score, weight=z(2, dtype=f64)),
            evict(scores=z(2, 3, 16)[:, :2]), evict(scores=z(2, 2, 16, dtype=bf16)), evict(kept=z(2, 2, 8, dtype=i64)),
            evict(scores_out=z(2, 2, 8, dtype=bf16)), evict(n_out=z(2, dtype=i64)), evict(dst_table=z(2, 1, dtype=i64))]
    for fn, d in bad:
        assert _status(fn, **d) == EINVAL, (fn.__name__, {k: (v.dtype, v.stride()) if hasattr(v, "dtype") else v for k, v in d.items()})


def _calls():
    """The C entry points with arguments that they take; addresses are numbers that nothing reads."""
    lib, a = pkg.load(), 4096
    rows = dict(dtype=0, batch=1, rows=1, G=1, hd=128, k=a, ldk=128, v=a, ldv=128, pool=a, blocks=1, table=a, pages=1, slot0=a, counts=a)
    cache = dict(pool=a, blocks=1, table=a, pages=1, n_ctx=a)
    attention = dict(qd=1, od=1, batch=1, H=4, G=2, hd=128, nq=1, ql0=0, n_local=1, q=a, ldq=512, q_rows=1, **cache, anc=a, out=a, lo=a,
                     ldo=512, lse=a, splits=0)
    score = dict(qd=1, batch=1, H=4, G=2, hd=128, nq=1, ql0=0, n_local=1, q=a, ldq=512, q_rows=1, lse=a, weight=a, **cache, anc=a,
                 scores=a, ld=16)
    evict = dict(batch=1, G=1, hd=64, **cache, scores=a, ld=32, budget=16, recent=4, dst=a, dst_pages=1, kept=a, out=a, n_out=a)
    return [(lib.chimera_op_kv4_append, rows), (lib.chimera_op_kv4_read, rows), (lib.chimera_op_attention_kv4, attention),
            (lib.chimera_op_kv4_score, score), (lib.chimera_op_kv4_evict, evict)]


def test_pointers_that_are_not_aligned_are_refused():
    least = dict(k=4, v=4, pool=16, table=4, slot0=4, counts=4, n_ctx=4, q=2, anc=8, lo=2, lse=4, weight=4, scores=4, dst=4, kept=4,
                 n_out=4)
    for fn, args in _calls():
        for name in args.keys() & (least.keys() | {"out"}):
            step = least.get(name, 2 if "lo" in args else 4)
            for off in {1, step // 2}:
                assert fn(*{**args, name: args[name] + off}.values(), None) == EINVAL, (fn.__name__, name, off)


def test_a_grid_past_32_bits_is_refused():
    fn, args = _calls()[2]
    many = dict(batch=65535, H=65535, G=1, hd=64, nq=64, q_rows=64, ldq=65535 * 64, ldo=65535 * 64)
    for more in (dict(), dict(lo=0, lse=0), dict(od=0, lo=0)):
        assert fn(*{**args, **many, **more}.values(), None) == EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_eviction_skips_the_rows_of_a_bad_block_alone(hd):
    G, n, budget = 2, 64, 47
    g = _gen(71, hd)
    cache = Cache(g, [n], G, hd, spare=3)
    # kept of the older ones: slots 0 to 30 and 32 to 43, so that rows 30 and 31 of the result, a pair, are slots 30 and 32
    scores = 1 + torch.rand(1, G, cache.pages * 16, generator=g, device="cuda")
    scores[..., 31] = scores[..., 44:] = 0
    table = cache.table.clone()
    table[0, 1] = cache.pool.shape[0]  # slots 16 to 31
    kept, out, n_out = torch.zeros(1, G, budget, dtype=torch.int32, device="cuda"), torch.zeros(1, G, budget, device="cuda"), _ints([0])
    pkg.op_kv4_evict(cache.pool, table, _ints([n]), scores, budget, 4, cache.spare, kept, out, n_out, hd)
    assert _status(pkg.op_sync) == EINVAL
    k, v = torch.zeros(budget, G * hd, device="cuda"), torch.zeros(budget, G * hd, device="cuda")
    pkg.op_kv4_read(cache.pool, cache.spare, _ints([0]), budget, hd, k, v)
    pkg.op_sync()
    for h in range(G):
        at = kept[0, h].long()
        good = (at < 16) | (at >= 32)
        assert at[30:32].tolist() == [30, 32]
        for got, want in ((k, cache.k), (v, cache.v)):
            assert torch.equal(got.view(budget, G, hd)[good, h].double(), want[0, at[good], h].float().double())


@pytest.mark.gpu
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_any_size_are_rounded_by_the_rule(hd, dtype):
    # steps from subnormal numbers to 2^123 (the rounding scales those below 2^-60 and above 2^60)
    sizes = [1e-41, 1e-38, 1e-30, 3e-19, 1e-18, 1.0, 1e18, 1e19, 3e19, 1e30, 1e36, 4e37]
    g, n = _gen(67, hd), len(sizes)
    rows = (_normal(g, n, 8, hd).clamp(-4, 4) * torch.tensor(sizes, device="cuda")[:, None, None]).view(-1, hd).to(dtype)
    pages = rows.shape[0] // 16
    pool, table, zero = pkg.kv4_pool(pages, 1, hd), torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1), _ints([0])
    back = rows.flip(0).contiguous()
    k, v = torch.zeros_like(rows), torch.zeros_like(rows)
    pkg.op_kv4_append(rows, back, pool, table, zero, rows.shape[0], hd)
    pkg.op_kv4_read(pool, table, zero, rows.shape[0], hd, k, v)
    pkg.op_sync()
    assert torch.equal(k, _stands_for(rows).float().to(dtype)) and torch.equal(v, _stands_for(back).float().to(dtype))


@pytest.mark.gpu
def test_rows_that_bf16_cannot_hold_are_no_numbers():
    # a minimum that rounds to -inf in bf16, a range past fp32, and their neighbours
    hd = 64
    rows = torch.zeros(16, hd, device="cuda")
    rows[0, 3] = -3.4e38
    rows[1, 0], rows[1, 1] = 2e38, -2e38
    rows[2, 0], rows[2, 1] = 1.5e38, -1.5e38
    rows[3] = 3.38e38
    pool, table, zero = pkg.kv4_pool(1, 1, hd), _ints([[0]]), _ints([0])
    pkg.op_kv4_append(rows, rows, pool, table, zero, 16, hd)
    k, v = torch.zeros_like(rows), torch.zeros_like(rows)
    pkg.op_kv4_read(pool, table, zero, 16, hd, k, v)
    pkg.op_sync()
    for x in (k, v):
        assert torch.isnan(x[:2]).all() and torch.equal(x[2:], _stands_for(rows[2:]).float())


# A rounding to bf16 is at most 2^-8 of the value.  Before it: sums of up to 128 codes of up to 15, with their zero or before
# it is taken off, are cut toward zero at 2^-22 of what they have reached in each of up to 8 steps; of tokens that share
# a sign that adds up over the groups, to 2^-15 of a row's largest result at worst (32 groups, codes around their zero).
ROUNDED_TOL = 2.0 ** -8 + 2.0 ** -14


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,group", [(1, 1000, 4096, 128), (3, 333, 4096, 64), (8, 250, 1056, 128), (5, 300, 4096, 32),
                                         (40, 300, 4096, 128)])
@pytest.mark.parametrize("kind", ["bf16", "split"])
@pytest.mark.parametrize("zeros", [True, False])
def test_linear_w4_rounded_results(M, N, K, group, kind, zeros):
    g = _gen(73, M, N)
    W, scale, zero, dense = _weights(g, N, K, group, zeros)
    for mean in (0.0, 1.0, 30.0):  # activations around 0, and of one sign
        x = _normal(g, M, K) + mean
        hi = x.to(torch.bfloat16)
        lo = (x - hi.float()).to(torch.bfloat16) if kind == "split" else None
        ref = (hi.double() + (lo.double() if lo is not None else 0.0)) @ dense.T
        Y = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
        pkg.op_linear_w4(hi, W, scale, Y, zeros=zero, group=group, X_lo=lo)
        assert _rel_rows(Y, ref) <= ROUNDED_TOL
    pkg.op_sync()


@pytest.mark.gpu
@pytest.mark.parametrize("M,group", [(5, 64), (5, 128), (8, 128), (40, 128)])
@pytest.mark.parametrize("zeros", [True, False])
def test_linear_w4_extreme_activations_rounded(M, group, zeros):
    g = _gen(79, M)
    W, scale, zero, dense = _weights(g, 300, 512, group, zeros)
    x = _normal(g, M, 512).to(torch.bfloat16)
    x[0, 7] = 3000.0  # one outlier
    x[1] *= 1e30
    x[2] *= 1e-30
    x[3, 100] = float("inf")
    x[4] = 0
    Y = torch.full((M, 300), float("nan"), dtype=torch.bfloat16, device="cuda")
    pkg.op_linear_w4(x, W, scale, Y, zeros=zero, group=group)
    pkg.op_sync()
    ref = x.double() @ dense.T
    rest = [i for i in range(M) if i != 3]
    assert _rel_rows(Y[rest], ref[rest]) <= ROUNDED_TOL
    assert not torch.isfinite(Y[3]).all() and (Y[4] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("case", HIDDEN)
@pytest.mark.parametrize("word", [0xffffffff, 0x7f807f80, 0x7e007e00], ids=["nan", "inf", "large"])
def test_weight_sums_of_rows_that_no_counted_query_sees(case, word):
    # local rows without numbers draw nothing from queries that do not see them, and change no other row's sum
    ctx, G, H, hd, nq, n_local = case
    g, r = _gen(83, len(ctx), G, nq), np.random.default_rng(83)
    cache = Cache(g, [n + n_local for n in ctx], G, hd)
    masks = _masks("tree", n_local, r)
    q = _normal(g, len(ctx) * nq, H * hd)
    bad = sorted({n_local - 1, n_local // 2} - {0})
    counts = torch.tensor([float(not any(masks[i] >> j & 1 for j in bad)) for i in range(nq)], device="cuda").repeat(len(ctx))
    scores = torch.rand(len(ctx), G, cache.pages * 16, generator=g, device="cuda")
    want, lse = scores.double(), torch.zeros(len(ctx) * nq, H, device="cuda")
    for b, z in enumerate(_probabilities(cache, q, ctx, masks, nq, 0, n_local, H, nq)):
        lse[b * nq:(b + 1) * nq] = torch.logsumexp(z, -1).T.float()
        p = torch.exp(z - lse[b * nq:(b + 1) * nq].T[:, :, None].double()).nan_to_num(0.0) * counts[:nq, None].double()
        want[b, :, :ctx[b] + n_local] += p.view(G, H // G * nq, -1).sum(1)
        for j in bad:
            _spoil(cache, b, ctx[b] + j, word)
    pkg.op_kv4_score(q, lse, cache.pool, cache.table, _ints(ctx), _anc(masks), scores, nq, 0, n_local, nq, H, hd, weight=counts)
    pkg.op_sync()
    assert _rel_rows(scores, want) <= ATT_TOL
