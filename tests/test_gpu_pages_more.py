"""Calls around the paged 8-bit store that tests/test_gpu_pages.py does not make, against the same plain forms in 64 bits (page_forms.py);
tolerances are derived as at its head, and where a test says so."""
import math

import numpy as np
import pytest
import torch

import page_forms as pg
from test_gpu_pages import (BF16, F32, HALF, IMPLS, check, ctx, f64, fc, filled_pool, i32, numpy_pool, rand, same_pages, same_pool,  # noqa: F401
                            status_word, tables)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------ entries that nobody needs

@pytest.mark.parametrize("dtype, impl", IMPLS)
@pytest.mark.parametrize("vis, begin, sink, active", [
    ([160, 160], [20, 100], 0, [1]),                    # windows that overlap
    ([100, 160], [20, 100], 0, [1]),                    # that meet
    ([160, 150, 140], [10, 70, 133], 5, [1]),           # one inside the other, and first tokens that all see
    ([90, 150, 160], [40, 60, 100], 70, [0]),           # first tokens that reach into the others' windows
    ([33, 160, 64, 160], [0, 50, 31, 90], 3, [2, 0]),
])
def test_attention_over_a_shared_sequence_minds_what_active_chunks_see(fc, ctx, vis, begin, sink, active, dtype, impl):
    # the pages that only inactive chunks see have been let go of: nobody asks for them, nothing is reported
    H, d, page, n, W = 2, 64, 16, 160, len(vis)
    pool, status = filled_pool(fc, 10, H, page, d, 1), status_word()
    where = numpy_pool(pool)
    live = {j // page for c in active for j in pg.seen_tokens(vis[c], sink, begin[c])}
    t = [e if e in live else (-1, 77)[e % 2] for e in range(10)]
    assert any(j // page not in live for c in range(W) for j in pg.seen_tokens(vis[c], sink, begin[c]))
    off = [3 * c for c in range(W + 1)]
    Q = rand((H, off[-1], d), 2, 1.0, dtype)
    O = torch.full_like(Q, 9.0)
    ids, count = i32(active + [-1] * (W - len(active))), i32([len(active)])
    args = (None, None, off, vis, ids, count, O)
    ctx.chunk_attention_kv8(Q, pool, i32([t]), [n] * W, *args, n_sink=sink, kv_begin=begin, impl=impl, status=status)
    assert int(status) == 0
    kv = [tuple(where.rows(w, t, pg.seen_tokens(vis[c], sink, begin[c])) for w in (0, 1)) if c in active else None for c in range(W)]
    check(O, None, f64(Q), kv, off, active, d ** -0.5, dtype, impl, 9.0)
    # one that an active chunk does see is reported
    t[pg.seen_tokens(vis[active[0]], sink, begin[active[0]])[-1] // page] = -1
    ctx.chunk_attention_kv8(Q, pool, i32([t]), [n] * W, *args, n_sink=sink, kv_begin=begin, impl=impl, status=status)
    assert int(status) == fc.STATUS_BITS["bad_index"]


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_of_many_chunks_over_a_shared_sequence(fc, ctx, dtype, impl, page):
    # 64 windows, each beginning and ending at a token of its own: as many pieces as there can be; some meet, some are inside others
    H, d, n, W, sink = 2, 64, 2000, 64, 9
    rng = np.random.default_rng(3)
    begin = rng.permutation(1800)[:W].tolist()
    vis = [min(n, b + int(k)) for b, k in zip(begin, rng.integers(1, 500, W))]
    vis[7], begin[9], vis[11] = begin[8], vis[10], 5  # meeting; ending among the first tokens
    active = sorted(rng.permutation(W)[:20].tolist())
    n_pages = -(-n // page)
    pool, status = filled_pool(fc, n_pages, H, page, d, 1), status_word()
    where = numpy_pool(pool)
    seen = [pg.seen_tokens(vis[c], sink, begin[c]) for c in range(W)]
    live = {j // page for c in active for j in seen[c]}
    t = [p if e in live else -1 for e, p in enumerate(tables(n_pages, [n_pages], n_pages, 4)[0])]
    off = [2 * c for c in range(W + 1)]
    Q = rand((H, off[-1], d), 2, 1.0, dtype)
    O = torch.full_like(Q, 9.0)
    ctx.chunk_attention_kv8(Q, pool, i32([t]), [n] * W, None, None, off, vis, i32(active), i32([len(active)]), O, n_sink=sink, kv_begin=begin, impl=impl,
                            status=status)
    assert int(status) == 0
    kv = [tuple(where.rows(w, t, seen[c]) for w in (0, 1)) if c in active else None for c in range(W)]
    check(O, None, f64(Q), kv, off, active, d ** -0.5, dtype, impl, 9.0)


# ------------------------------------------------------------------------------------ numbers of any size

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", [-90, 0, 100, 114, 121])
@pytest.mark.parametrize("n, plain, rows", [(100, 0, 3), (60, 40, 11), (0, 100, 3), (0, 100, 11), (1, 0, 1), (0, 1, 1)])
def test_attention_values_of_any_size(fc, ctx, n, plain, rows, size, dtype, d):
    # values of up to 2^121 (of a single token: up to the largest that there are), a sum of whose number times their size stays below 2^128
    H, page, up = 2, 32, 127 if n + plain == 1 and size == 121 else size
    pool, t = filled_pool(fc, 4, H, page, d, 1), [2, 0, 3, 1]
    pool.v_codes[pool.v_codes.bitwise_and(0x7f) > 0x78] = 0xf8  # magnitudes up to 256
    pool.v_scales[:] = 2.0 ** (up - 8)
    K, V = rand((H, plain, d), 3, 1.0, dtype), (rand((H, plain, d), 4, 1.0, F32).clamp(-4, 4) / 4 * 1.99 * 2.0 ** (up - 1)).to(dtype)
    where = numpy_pool(pool)
    kv = [np.concatenate([where.rows(w, t, range(n)), f64(y)], 1) for w, y in ((0, K), (1, V))]
    assert np.abs(kv[1]).max() * (n + plain) < 2.0 ** 128
    Q = rand((H, rows, d), 2, 2.0, dtype)
    O, lse = torch.zeros_like(Q), torch.zeros((H, rows), device="cuda")
    ctx.chunk_attention_kv8(Q, pool, i32([t]), [n], *((K, V) if plain else (None, None)), [0, rows], [n + plain], i32([0]), i32([1]), O, lse=lse, impl=3)
    unit = 2.0 ** -up  # an exact change of scale, so that the tolerances mean what they say
    check(O.double() * unit, lse, f64(Q), [(kv[0], kv[1] * unit)], [0, rows], [0], d ** -0.5, dtype, 3)


@pytest.mark.parametrize("parts", [1, 40])
def test_attention_values_of_any_size_in_parts(fc, ctx, parts):
    # the same through the joins: of a cluster's blocks, and of chunks of very different lengths
    H, d, page, n = 1, 64, 128, 128 * 20 * parts
    pool = filled_pool(fc, 20 * parts, H, page, d, 1)
    pool.v_codes.bitwise_and_(0x7f).clamp_(max=0x78)  # of one sign, so that the sums grow
    pool.v_scales[:] = 2.0 ** (110 - 8)  # times the tokens: below 2^128
    t = list(range(20 * parts))
    for dtype in (BF16, F32):
        Q, off, vis = rand((H, 9, d), 2, 0.01, dtype), [0, 1, 9], [n, 100]  # weights that are nearly the same
        O = torch.zeros_like(Q)
        ctx.chunk_attention_kv8(Q, pool, i32([t]), vis, None, None, off, vis, i32([0, 1]), i32([2]), O, impl=3)
        kv = [tuple(numpy_pool(pool).rows(w, t, range(v)) * (1.0, 2.0 ** -110)[w] for w in (0, 1)) for v in vis]
        check(O.double() * 2.0 ** -110, None, f64(Q), kv, off, [0, 1], d ** -0.5, dtype, 3)


@pytest.mark.parametrize("d, page", [(64, 32), (128, 16), (128, 128)])
@pytest.mark.parametrize("rows", [1, 8, 13])
def test_attention_small_weights_of_fp32_rows(fc, ctx, rows, d, page):
    # in every 32 keys one of weight 1, whose value is 0, beside 31 of weight e^-L: the output is what the small weights carry
    n = 32 * 40
    pool = fc.Kv8Pool.empty(n // page, 1, page, d)
    for c in (pool.k_codes, pool.v_codes):
        c.fill_(0)
    pool.k_scales.fill_(1.0), pool.v_scales.fill_(1.0)
    token = torch.arange(n, device="cuda").view(n // page, 1, page)
    pool.k_codes[..., 0][token % 32 == 5] = 0x38            # 1
    pool.v_codes[..., : d][token % 32 != 5] = 0x3c          # 1.5
    L = torch.linspace(11, 18, rows, dtype=F32) if rows > 1 else torch.tensor([17.3])
    Q, O = torch.zeros((1, rows, d), dtype=F32, device="cuda"), torch.zeros((1, rows, d), dtype=F32, device="cuda")
    Q[0, :, 0] = L.cuda()
    ctx.chunk_attention_kv8(Q, pool, i32([list(range(n // page))]), [n], None, None, [0, rows], [n], i32([0]), i32([1]), O, scale=1.0)
    L = L.double().numpy()[:, None]
    e = 31 * np.exp(-L)
    want = 1.5 * e / (1 + e)
    # The logit is one product: Q's parts leave out 2^-23 of it, and four roundings 2^-24 each; all in the exponent.  The exponential and a weight's
    # parts 2^-22 each, the sums n 2^-24, and a weight that is small for fp16's parts 2^-43 of the largest.
    rel = L * (2.0 ** -23 + 4 * 2.0 ** -24) + 2 * 2.0 ** -22 + n * 2.0 ** -24 + 2.0 ** -24
    assert (np.abs(f64(O)[0] - want) <= rel * want + 1.5 * 31 * 2.0 ** -43).all()


# ------------------------------------------------------------------------------------ pages

def test_fork_reports_free_pages(fc, ctx):
    # as drop and compact do.  A free page is nobody's: it is not shared, and nothing is copied out of it
    H, d, page, bad = 2, 64, 16, fc.STATUS_BITS["bad_index"]
    pool, status = filled_pool(fc, 7, H, page, d, 1), status_word()
    codes = pool.k_codes.clone()
    ref, table = i32([1, 0, 1, 0, 0, 1, 1]), i32([[0, 1, 2, 5], [-1] * 4, [0, 2, 6, 3], [-1] * 4, [-1] * 4])
    ctx.pages_fork(pool, ref, table, [0, 0], [1, 3], [48, 40], status=status)  # entry 1 names page 1, which is free
    # the second fork fills entry 2 in part: page 2 is copied into the lowest free one
    assert int(status) == bad
    assert table.tolist() == [[0, 1, 2, 5], [0, -1, 2, -1], [0, 2, 6, 3], [0, -1, 1, -1], [-1] * 4]
    assert ref.tolist() == [3, 1, 2, 0, 0, 1, 1]
    codes[1] = codes[2]
    assert torch.equal(pool.k_codes, codes)
    status.zero_()
    ctx.pages_fork(pool, ref, table, [2], [4], [50], status=status)  # entry 3 names page 3, free, and is filled in part
    assert int(status) == bad and torch.equal(pool.k_codes, codes)
    assert table[4].tolist() == [0, 2, 6, 3] and ref.tolist() == [4, 1, 3, 1, 0, 1, 2]
    status.zero_()
    ctx.pages_fork(pool, ref, table, [0], [4], [16], status=status)
    assert int(status) == 0


def test_append_writes_only_to_pages_with_one_holder(fc, ctx):
    H, d, page = 2, 64, 16
    K = rand((H, 40, d), 1)
    pool, status = filled_pool(fc, 4, H, page, d, 1), status_word()
    want = numpy_pool(pool)
    ctx.kv8_append(K, K, pool, i32([[0, 1, 2]]), [0], ref=i32([1, 0, 1, 1]), status=status)  # page 1 is free
    for a, b, p in ((0, 16, 0), (32, 40, 2)):
        for which in (0, 1):
            want.append(f64(K)[:, a:b], which, [p], 0)
    same_pool(pool, want)
    assert int(status) == fc.STATUS_BITS["bad_index"]


@pytest.mark.parametrize("rows", [1, 11, 140])
@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_infinities(fc, ctx, dtype, impl, rows):
    # one in Q: NaN, of either sign.  One in K or V: what it reaches is infinite or NaN, or a token's logit is -inf and the others are left;
    # nothing else differs, and what is not seen has no effect
    H, d, n = 2, 64, 50
    Q, K, V = rand((H, rows, d), 1, 1.0, dtype), rand((H, n, d), 2, 1.0, dtype), rand((H, n, d), 3, 1.0, dtype)
    K[:, :, 0] = K[:, :, 0].abs() + 0.25
    out = {}
    for which in ("none", "q", "minus q", "k", "v", "unseen"):
        q, k, v = Q.clone(), K.clone(), V.clone()
        if which == "q":
            q[0, 0, 0] = math.inf
        elif which == "minus q":
            q[0, 0, 0] = -math.inf
        elif which == "k":
            k[0, 20, 3] = math.inf
        elif which == "v":
            v[0, 20, 3] = -math.inf
        elif which == "unseen":
            k[0, 8, 3], v[1, 9, 3] = math.inf, -math.inf
        O, lse = torch.full_like(Q, 9.0), torch.full((H, rows), 5.0, device="cuda")
        ctx.chunk_attention_span(q, k, v, [0, rows], [n], [0, n], [0], i32([0]), i32([1]), O, n_sink=5, kv_begin=[13], lse=lse, impl=impl)
        out[which] = O, lse
    O, lse = out["none"]
    assert torch.isfinite(O).all() and torch.isfinite(lse).all()
    assert torch.equal(out["unseen"][0], O) and torch.equal(out["unseen"][1], lse)
    for which in ("q", "minus q"):
        got, got_lse = out[which]
        assert torch.equal(got[1], O[1]) and torch.equal(got[0, 1:], O[0, 1:]) and torch.equal(got_lse[1], lse[1])
        assert torch.isnan(got[0, 0]).all() and torch.isnan(got_lse[0, 0])
    got = out["k"][0]  # logits of +inf or -inf: nothing else is seen, or the token is not
    assert torch.equal(got[1], O[1])
    per_row = torch.isnan(got[0]).all(1) | torch.isfinite(got[0]).all(1)
    assert per_row.all() and (dtype == BF16 or torch.isnan(got[0]).all())
    got = out["v"][0]
    keep = torch.arange(d, device="cuda") != 3
    assert torch.equal(got[1], O[1]) and torch.equal(got[0][:, keep], O[0][:, keep])
    assert (torch.isnan(got[0, :, 3]) | (got[0, :, 3] == -math.inf)).all()


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_infinities_in_queries_over_pages(fc, ctx, dtype, impl):
    H, d, page, n, rows = 1, 64, 16, 40, 4
    pool, t = filled_pool(fc, 3, H, page, d, 1), i32([[0, 1, 2]])
    pool.k_codes[..., 0] = pool.k_codes[..., 0].bitwise_and(0x7f).clamp(min=8)  # positive
    Q = rand((H, rows, d), 1, 1.0, dtype)
    want, want_lse = torch.zeros_like(Q), torch.zeros((H, rows), device="cuda")
    got, got_lse = torch.zeros_like(Q), torch.zeros((H, rows), device="cuda")
    args = (pool, t, [n], None, None, [0, rows], [n], i32([0]), i32([1]))
    ctx.chunk_attention_kv8(Q, *args, want, lse=want_lse, impl=impl)
    Q[0, 1, 0], Q[0, 2, 0] = math.inf, -math.inf
    ctx.chunk_attention_kv8(Q, *args, got, lse=got_lse, impl=impl)
    assert torch.equal(got[0, ::3], want[0, ::3]) and torch.isnan(got[0, 1:3]).all() and torch.isnan(got_lse[0, 1:3]).all()


def test_on_the_bounds_checking_build(fc):
    # the calls of this file whose stores are guarded there; every test counts its status
    import os
    import subprocess
    import sys
    from paper_2602_10825_b200 import build as fc_build
    fc_build.build(debug_bounds=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "tests/test_gpu_pages_more.py", "-m", "gpu", "-k",
                          "shared_sequence or free_pages or one_holder or captured"],
                         cwd=root, env={**os.environ, "FC_LIB": "debug"}, capture_output=True, text=True, timeout=600)
    assert run.returncode == 0, run.stdout[-3000:] + run.stderr[-2000:]


def test_pages_and_append_captured_move_the_same_bytes(fc, ctx):
    # the pool, the counts and the table are put back before each replay: all that a turn writes is the replay's own
    H, d, page = 2, 64, 16
    pool = filled_pool(fc, 20, H, page, d, 1)
    ref, table = pool.tables(3, 8)
    K, V, status = rand((H, 20, d), 1), rand((H, 20, d), 2), status_word()
    ctx.pages_take(ref, table, [0, 0, 0], [3, 0, 3])
    ctx.pages_drop(ref, table, [0, 0, 0], [0, 0, 1])  # a hole for the compaction
    state = [pool.k_codes, pool.k_scales, pool.v_codes, pool.v_scales, ref, table, status]
    start = [x.clone() for x in state]

    def turn():
        ctx.pages_fork(pool, ref, table, [0], [1], [37], status=status)
        ctx.kv8_append(K, V, pool, table[1:2], [37], ref=ref, status=status)  # its rows from 48 on have no page: reported
        ctx.pages_take(ref, table, [3, 4, 3], [4, 5, 3], status=status)
        ctx.pages_drop(ref, table, [0, 0, 1], [1, 0, 3], status=status)
        ctx.pages_compact(pool, ref, table, status=status)
    turn()
    torch.cuda.synchronize()
    want = [x.clone() for x in state]
    assert int(status) == fc.STATUS_BITS["bad_index"]
    assert not torch.equal(want[0], start[0]) and not torch.equal(want[3], start[3])
    graph = torch.cuda.CUDAGraph()
    for x, y in zip(state, start):
        x.copy_(y)
    with torch.cuda.graph(graph):
        turn()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(state, start))  # a capture runs nothing
    for _ in range(3):
        for x, y in zip(state, start):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(state, want)):
            assert torch.equal(x, y), f"tensor {i}"
