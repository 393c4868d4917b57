"""The paged 8-bit store, its pages, and attention over it and over plain rows with a sliding window, against plain forms in 64 bits
(page_forms.py), at the sizes and masks where they can go wrong.

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value, one to fp16 by 2^-11, one to fp32 by 2^-24.
  append, unpack, pages   none: codes, scales, values, counts and tables are compared as bits.
  attention  a logit is a sum of d products, exact or of parts of numbers that leave out 2^-23 of a product at most, added by tensor cores that
             may cut each sum instead of rounding it: (d + 8) 2^-23 |q||k| scale; a weight is off by twice that, its exponential by 2^-22
             or, on the tcgen05 kernel, 1e-4, and sums of n terms by n 2^-24, all relative to A = sum p |v|.  bf16: a weight is rounded to
             bf16 (2^-8 A), or to fp16 in units of 2^-25 of a weight of 2^7 (2^-11 A and n 2^-32 of the largest |v|); fp32: weights lose 2^-22 A at
             most.  Then the output's rounding.  The log of the weights' sum is off by the logit's error, the sum's n 2^-24, the exponentials',
             and its own rounding and that of the logarithm (2^-22).
"""
import math

import numpy as np
import pytest
import torch

import page_forms as pg
import workloads as wl

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


@pytest.fixture(scope="module")
def fc():
    import paper_2602_10825_b200 as fc
    from paper_2602_10825_b200 import build as fc_build
    fc_build.build()
    return fc


@pytest.fixture(scope="module")
def ctx(fc):
    c = fc.Context(0)
    yield c
    c.close()


def f64(t):
    return t.detach().double().cpu().numpy()


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def rand(shape, seed, sigma=1.0, dtype=BF16):
    return wl.normal(shape, seed, sigma, dtype).cuda()


def status_word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------ append and unpack

def filled_pool(fc, n_pages, H, page, d, seed, codes=None):
    """A pool of random codes (no NaN) and scales of four bits."""
    g = torch.Generator().manual_seed(seed)
    t = []
    for _ in range(2):
        c = torch.randint(0, 127, (n_pages, H, page, d), generator=g) + 128 * torch.randint(0, 2, (n_pages, H, page, d), generator=g)
        s = (8 + torch.randint(0, 8, (n_pages, H), generator=g)) / 8 * 2.0 ** torch.randint(-9, -6, (n_pages, H), generator=g)
        t += [c.to(torch.uint8).cuda(), s.float().cuda()]
    return fc.Kv8Pool(*t)


def numpy_pool(pool):
    return pg.Pool(*(t.cpu().numpy() for t in (pool.k_codes, pool.k_scales, pool.v_codes, pool.v_scales)))


def same_pool(pool, want):
    for i, (c, s) in enumerate(((pool.k_codes, pool.k_scales), (pool.v_codes, pool.v_scales))):
        assert np.array_equal(c.cpu().numpy(), want.codes[i]), f"codes {i}: {np.argwhere(c.cpu().numpy() != want.codes[i])[:3]}"
        assert np.array_equal(f64(s), want.scales[i])


def tables(n_pages, counts, width, seed):
    order, at = np.random.default_rng(seed).permutation(n_pages), 0
    t = np.full((len(counts), width), -1)
    for c, n in enumerate(counts):
        t[c, :n] = order[at:at + n]
        at += n
    return t


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H, d, page, pos, n", [
    (1, 64, 16, [0], [1]), (3, 128, 16, [5], [40]), (2, 64, 32, [31, 0], [1, 33]), (2, 128, 64, [63, 64, 1], [1, 130, 0]), (5, 64, 128, [100], [400]),
    (2, 128, 128, [127, 0, 300], [2, 128, 9]), (1, 128, 32, [7, 40, 3, 0], [0, 25, 29, 1]), (2, 64, 64, [10, 70], [3, 3]),
])
def test_append_and_unpack(fc, ctx, H, d, page, pos, n, dtype):
    off = np.concatenate([[2], 2 + np.cumsum(n)])  # rows before the first sequence's and behind the last's belong to nobody
    counts = [-(-(p + k) // page) for p, k in zip(pos, n)]
    n_pages = sum(counts) + 4
    t = tables(n_pages, counts, max(counts) + 1, 3)
    pool = filled_pool(fc, n_pages, H, page, d, 1)
    want = numpy_pool(pool)
    K, V = rand((H, off[-1] + 3, d), 4, 3.0, dtype), rand((H, off[-1] + 3, d), 5, 0.01, dtype)
    status = status_word()
    ctx.kv8_append(K, V, pool, i32(t), pos, off.tolist(), status=status)
    for c in range(len(pos)):
        if n[c]:
            want.append(f64(K)[:, off[c]:off[c + 1]], 0, t[c], pos[c])
            want.append(f64(V)[:, off[c]:off[c + 1]], 1, t[c], pos[c])
    same_pool(pool, want)
    assert int(status) == 0
    # read back from the middle of the first page on, and into rows of a larger tensor
    first = [min(3, p) for p in pos]
    rows = [p + k - f for p, k, f in zip(pos, n, first)]
    at = np.concatenate([[1], 1 + np.cumsum(rows)])
    for dt in (BF16, F32):
        K_dst, V_dst = torch.full((H, at[-1] + 2, d), 7.0, dtype=dt, device="cuda"), torch.full((H, at[-1] + 2, d), 7.0, dtype=dt, device="cuda")
        ctx.kv8_unpack(pool, i32(t), first, at.tolist(), K_dst=K_dst, V_dst=V_dst, status=status)
        for which, got in ((0, f64(K_dst)), (1, f64(V_dst))):
            ref = np.full(got.shape, 7.0)
            for c in range(len(pos)):
                ref[:, at[c]:at[c + 1]] = want.rows(which, t[c], range(first[c], first[c] + rows[c]))
            assert np.array_equal(got, ref)  # exact in both types
    assert int(status) == 0
    keys, none = ctx.kv8_unpack(pool, i32(t), first, [a - 1 for a in at.tolist()], keys_only=True)
    assert none is None and torch.equal(keys, K_dst[:, 1:-2].to(BF16))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_token_by_token(fc, ctx, dtype):
    # scales that grow now and then: what is there is rounded again each time
    H, d, page, n = 2, 64, 16, 37
    K, V = rand((H, n, d), 1, 1.0, dtype), rand((H, n, d), 2, 1.0, dtype)
    K *= torch.linspace(0.1, 30, n, device="cuda")[:, None].to(dtype)
    pool = filled_pool(fc, 5, H, page, d, 1)
    want, t = numpy_pool(pool), np.asarray([[4, 0, 2]])
    for i in range(n):
        ctx.kv8_append(K[:, i:i + 1], V[:, i:i + 1], pool, i32(t), [i])
        want.append(f64(K)[:, i:i + 1], 0, t[0], i)
        want.append(f64(V)[:, i:i + 1], 1, t[0], i)
    same_pool(pool, want)
    # rewound into the middle of a page: the rows before it stay, those behind count for nothing but the scale
    ctx.kv8_append(K[:, :4], V[:, :4], pool, i32(t), [20])
    want.append(f64(K)[:, :4], 0, t[0], 20)
    want.append(f64(V)[:, :4], 1, t[0], 20)
    same_pool(pool, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_ties_extremes_and_strides(fc, ctx, dtype):
    # rows out of a fused projection [tokens, k heads | v heads, d]; each block's scale is set by one element
    H, d, page = 6, 128, 16
    x = torch.zeros((page, 2 * H, d), dtype=dtype, device="cuda")
    codes = torch.from_numpy(pg.code_values(np.arange(1, 127, dtype=np.uint8)))
    ties = ((codes[1:] + codes[:-1]) / 2).to(dtype)  # five significant bits: exact in both types
    for h, size in enumerate([1.0, 1.875, 2.0 ** -117, 2.0 ** 119, 1e-38, 0.0]):
        for half in range(2):
            x[0, half * H + h, 0] = 448 * size
            x[1, half * H + h, :125] = (ties.double() * size).to(dtype).cuda() * (1 - 2 * half)
    x[2, 3, 0], x[2, H + 3, 0] = 3.3e38, -3.3e38  # above 448 2^119: cut to it
    x[1, 4, :] = 1e-40 if dtype == F32 else 0.0
    K, V = x[:, :H].transpose(0, 1), x[:, H:].transpose(0, 1)
    pool, t = filled_pool(fc, 2, H, page, d, 1), np.asarray([[1]])
    want = numpy_pool(pool)
    ctx.kv8_append(K, V, pool, i32(t), [0])
    want.append(f64(K), 0, t[0], 0)
    want.append(f64(V), 1, t[0], 0)
    same_pool(pool, want)
    assert f64(pool.k_scales)[1].tolist()[:4] == [1.0, 1.875, 2.0 ** -117, 2.0 ** 119] and f64(pool.k_scales)[1, 5] == 0


def test_append_fp32_next_to_ties(fc, ctx):
    H, d, page = 8, 64, 16
    codes = pg.code_values(np.arange(1, 127, dtype=np.uint8))
    ties = (codes[1:] + codes[:-1]) / 2
    x = np.zeros((H, page, d), np.float32)
    for h in range(H):
        s = (8 + h) / 8
        t = np.resize((ties * s).astype(np.float32), (5, d))  # the same ties, and their neighbours on both sides
        x[h, 0, 0] = 448 * s
        x[h, 1:6], x[h, 6:11], x[h, 11:16] = t, np.nextafter(t, np.float32(0)), np.nextafter(t, np.float32(1e9))
    x[:, 11:16] = np.minimum(x[:, 11:16], x[:, :1, :1])
    K = torch.from_numpy(x).cuda()
    pool, t = filled_pool(fc, 1, H, page, d, 1), np.asarray([[0]])
    want = numpy_pool(pool)
    ctx.kv8_append(K, -K, pool, i32(t), [0])
    want.append(f64(K), 0, t[0], 0)
    want.append(-f64(K), 1, t[0], 0)
    same_pool(pool, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", [2.0 ** -124, 2.0 ** -108, 2.0 ** -90, 2.0 ** -81, 1.0, 2.0 ** 100])
def test_append_rows_of_any_size(fc, ctx, size, dtype):
    # zeros of both signs among them, and next to the scale below which fp32 rows are divided
    H, d, page, n = 9, 64, 32, 32
    K = (rand((H, n, d), 1, 1.0, F32) * torch.linspace(0.5, 2.1, H, device="cuda")[:, None, None] * size).to(dtype)
    K[:, :, :2] = torch.tensor([0.0, -0.0], device="cuda")
    pool, t = filled_pool(fc, 1, H, page, d, 1), np.asarray([[0]])
    want = numpy_pool(pool)
    ctx.kv8_append(K, -K, pool, i32(t), [0])
    want.append(f64(K), 0, t[0], 0)
    want.append(-f64(K), 1, t[0], 0)
    same_pool(pool, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_nonfinite_elements(fc, ctx, dtype):
    H, d, page, n = 2, 64, 32, 20
    K, V = rand((H, n, d), 1, 1.0, dtype), rand((H, n, d), 2, 1.0, dtype)
    K[0, 3, 5], K[1, 4, 6], V[0, 0, 0] = math.nan, math.inf, -math.inf
    V[1] = 0
    V[1, 2, 2] = math.nan  # nothing finite but zeros
    pool, t, status = filled_pool(fc, 1, H, page, d, 1), np.asarray([[0]]), status_word()
    want = numpy_pool(pool)
    ctx.kv8_append(K, V, pool, i32(t), [0], status=status)
    want.append(f64(K), 0, t[0], 0)
    want.append(f64(V), 1, t[0], 0)
    same_pool(pool, want)
    assert int(status) == fc.STATUS_BITS["nonfinite"]
    got = ctx.kv8_unpack(pool, i32(t), [0], [0, n])
    assert torch.isnan(got[0]).sum() == 2 and torch.isnan(got[1]).sum() == 2
    # they stay NaN when the block is rounded again
    status.zero_()
    ctx.kv8_append(100 * K[:, 5:6], 100 * V[:, 5:6], pool, i32(t), [n], status=status)
    want.append(f64(100 * K[:, 5:6]), 0, t[0], n)
    want.append(f64(100 * V[:, 5:6]), 1, t[0], n)
    same_pool(pool, want)
    assert int(status) == 0


def test_append_leaves_pages_that_are_shared_or_not_there(fc, ctx):
    H, d, page = 2, 64, 16
    K = rand((H, 40, d), 1)
    pool, status = filled_pool(fc, 6, H, page, d, 1), status_word()
    want, ref = numpy_pool(pool), i32([1, 2, 1, 0, 1, 1])
    t = i32([[0, 1, 2]])
    ctx.kv8_append(K, K, pool, t, [0], ref=ref, status=status)  # page 1 has two holders
    for a, b, p in ((0, 16, 0), (32, 40, 2)):
        for which in (0, 1):
            want.append(f64(K)[:, a:b], which, [p], 0)
    same_pool(pool, want)
    assert int(status) == fc.STATUS_BITS["bad_index"]
    for bad in (-1, 6, 2 ** 31 - 1, -2 ** 31):
        status.zero_()
        ctx.kv8_append(K[:, :20], K[:, :20], pool, i32([[4, bad]]), [0], status=status)
        assert int(status) == fc.STATUS_BITS["bad_index"]
        for which in (0, 1):
            want.append(f64(K)[:, :16], which, [4], 0)
        same_pool(pool, want)
        status.zero_()
        got = ctx.kv8_unpack(pool, i32([[4, bad]]), [0], [0, 20], status=status)[0]
        assert int(status) == fc.STATUS_BITS["bad_index"] and (got[:, 16:] == 0).all() and np.array_equal(f64(got[:, :16]), want.rows(0, [4], range(16)))


def test_pool_of_other_orders_and_far_offsets(fc, ctx):
    # heads outermost; and pages 2.2e9 bytes apart, whose offsets pass 32 bits
    H, d, page, n = 3, 64, 16, 50
    K, V = rand((H, n, d), 1), rand((H, n, d), 2)
    by_head = [torch.zeros((H, 5, page, d), dtype=torch.uint8, device="cuda").transpose(0, 1) for _ in range(2)]
    scales = [torch.zeros((H, 5), device="cuda").transpose(0, 1) for _ in range(2)]
    far = 2_200_000_000 // 16 * 16
    buf = torch.zeros(2 * far + 2 * H * page * d, dtype=torch.uint8, device="cuda")
    apart = [torch.as_strided(buf, (3, H, page, d), (far, page * d, d, 1), i * H * page * d) for i in range(2)]
    for codes, sc, t in ((by_head, scales, [[4, 0, 2, 3]]), (apart, [torch.zeros((3, H), device="cuda") for _ in range(2)], [[2, 0, 1]])):
        m = min(n, len(t[0]) * page)
        pool = fc.Kv8Pool(codes[0], sc[0], codes[1], sc[1])
        want = numpy_pool(pool)
        ctx.kv8_append(K[:, :m], V[:, :m], pool, i32(t), [0])
        want.append(f64(K)[:, :m], 0, t[0], 0)
        want.append(f64(V)[:, :m], 1, t[0], 0)
        same_pool(pool, want)
        k, v = ctx.kv8_unpack(pool, i32(t), [0], [0, m])
        kv = [want.rows(w, t[0], range(m)) for w in (0, 1)]
        assert np.array_equal(f64(k), kv[0]) and np.array_equal(f64(v), kv[1])
        for rows, impls in ((2, (0, 3)), (200, (2, 3))):
            Q = rand((H, rows, d), 3)
            for impl in impls:
                O = torch.zeros_like(Q)
                ctx.chunk_attention_kv8(Q, pool, i32(t), [m], None, None, [0, rows], [m], i32([0]), i32([1]), O, impl=impl)
                check(O, None, f64(Q), [kv] * H, [0, rows], [0], d ** -0.5, BF16, impl)


# ------------------------------------------------------------------------------------ pages

def same_pages(ref, table, want):
    assert ref.tolist() == want.ref and table.tolist() == want.table


def test_pages_through_a_long_life(fc, ctx):
    # several tiles of counts; sequences that grow, branch, let go and close ranks
    rng, n_pages, n_seq, entries, H, d, page = np.random.default_rng(1), 9001, 20, 700, 1, 64, 16
    pool = filled_pool(fc, n_pages, H, page, d, 2)
    codes = [pool.k_codes.cpu().numpy(), pool.v_codes.cpu().numpy()]
    scales = [f64(pool.k_scales), f64(pool.v_scales)]
    ref, table = pool.tables(n_seq, entries)
    want, status, n_used = pg.Pages(ref.tolist(), table.tolist()), status_word(), status_word()
    length = [0] * n_seq

    def copied(moves):
        for x in codes + scales:
            for a, b in moves:
                x[b] = x[a]

    for turn in range(60):
        kind = rng.integers(5)
        if kind <= 1:  # grow
            more = [min(entries, n + int(rng.integers(0, 120))) if rng.random() < 0.5 else n for n in length]
            ctx.pages_take(ref, table, length, more, status=status)
            want.take(length, more)
            length = more
        elif kind == 2:  # let go of a piece, or of everything
            a = [int(rng.integers(0, n + 1)) if rng.random() < 0.4 else 0 for n in length]
            z = [int(rng.integers(x, n + 1)) if x or rng.random() < 0.2 else 0 for x, n in zip(a, length)]
            ctx.pages_drop(ref, table, a, z, status=status)
            want.drop(a, z)
            length = [x if z_ == n and x < z_ else n for x, z_, n in zip(a, z, length)]
        elif kind == 3:  # branch into sequences that were dropped first
            dst = rng.permutation(n_seq)[:3].tolist()
            src = [int(rng.choice([c for c in range(n_seq) if c not in dst])) for _ in dst]
            zero, ends = [0] * n_seq, [length[c] if c in dst else 0 for c in range(n_seq)]
            ctx.pages_drop(ref, table, zero, ends, status=status)
            want.drop(zero, ends)
            tokens = [int(rng.integers(0, length[s] * page + 1)) for s in src]
            ctx.pages_fork(pool, ref, table, src, dst, tokens, status=status)
            copied(want.fork(src, dst, tokens, page))
            for t, n in zip(dst, tokens):
                length[t] = -(-n // page)
        else:
            ctx.pages_compact(pool, ref, table, n_used=n_used, status=status)
            moves = want.compact()
            copied(moves)
            assert int(n_used) == sum(r > 0 for r in want.ref)
        same_pages(ref, table, want)
        held = np.bincount([p for row in want.table for p in row if p >= 0], minlength=n_pages)
        assert held.tolist() == want.ref  # counts and tables agree
    assert np.array_equal(pool.k_codes.cpu().numpy(), codes[0]) and np.array_equal(pool.v_codes.cpu().numpy(), codes[1])
    assert np.array_equal(f64(pool.k_scales), scales[0]) and np.array_equal(f64(pool.v_scales), scales[1])
    assert not want.bad and int(status) == (fc.STATUS_BITS["no_pages"] if want.none_left else 0)


def test_pages_run_out(fc, ctx):
    pool = filled_pool(fc, 5, 2, 16, 64, 1)
    ref, table = pool.tables(3, 4)
    want, status = pg.Pages(ref.tolist(), table.tolist()), status_word()
    ctx.pages_take(ref, table, [0, 0, 0], [3, 0, 1], status=status)
    want.take([0, 0, 0], [3, 0, 1])
    assert int(status) == 0
    before = pool.k_codes.clone()
    ctx.pages_fork(pool, ref, table, [0, 0], [1, 2], [20, 37], status=status)  # two copies, one page left
    copies = want.fork([0, 0], [1, 2], [20, 37], 16)
    same_pages(ref, table, want)
    assert copies == [(1, 4)] and table[2].tolist() == [0, 1, -1, -1] and int(status) == fc.STATUS_BITS["no_pages"]
    assert torch.equal(pool.k_codes[4], before[1]) and torch.equal(pool.k_codes[:4], before[:4])
    status.zero_()
    ctx.pages_take(ref, table, [3, 2, 2], [4, 4, 4], status=status)
    want.take([3, 2, 2], [4, 4, 4])
    same_pages(ref, table, want)
    assert int(status) == fc.STATUS_BITS["no_pages"]


def test_pages_bad_entries_are_reported(fc, ctx):
    pool = filled_pool(fc, 8, 1, 16, 64, 1)
    bad = fc.STATUS_BITS["bad_index"]
    ref, table = i32([1, 1, 0, 2, 0, 0, 1, 1]), i32([[3, 9, 2, -5], [3, 0, 1, 6], [-1, -1, -1, -1], [7, -1, -1, -1]])
    want, status = pg.Pages(ref.tolist(), table.tolist()), status_word()
    ctx.pages_fork(pool, ref, table, [0], [2], [40], status=status)  # entries 3, 9 (no page), and 2 (free) in part
    want.fork([0], [2], [40], 16)
    same_pages(ref, table, want)
    assert int(status) == bad
    status.zero_()
    ctx.pages_compact(pool, ref, table, status=status)
    want.compact()
    same_pages(ref, table, want)
    assert int(status) == bad and want.bad
    status.zero_()
    ctx.pages_drop(ref, table, [0, 0, 0, 0], [4, 0, 0, 0], status=status)
    want.drop([0, 0, 0, 0], [4, 0, 0, 0])
    same_pages(ref, table, want)
    assert int(status) == bad
    # a page that is dropped twice at once is free, not owed
    ref, table, status = i32([1, 0]), i32([[0, 0, 0]]), status_word()
    ctx.pages_drop(ref, table, [0], [3], status=status)
    assert ref.tolist() == [0, 0] and table.tolist() == [[-1, -1, -1]] and int(status) == bad


def test_pages_of_a_full_and_of_an_empty_pool(fc, ctx):
    for used in ([1] * 7, [0] * 7, [0] * 6 + [1], [1] + [0] * 6):
        pool, ref = filled_pool(fc, 7, 2, 32, 128, 1), i32(used)
        table = i32([[p for p in range(7) if used[p]] + [-1] * (7 - sum(used))])
        want, codes = pg.Pages(ref.tolist(), table.tolist()), pool.k_codes.clone()
        ctx.pages_compact(pool, ref, table)
        moves = want.compact()
        same_pages(ref, table, want)
        for a, b in moves:
            codes[b] = codes[a]
        assert torch.equal(pool.k_codes, codes)


# ------------------------------------------------------------------------------------ attention

def check(O, lse, Q, kv, q_off, active, scale, dtype, impl, O_before=0.0, n_max=None):
    """kv: per chunk (K, V) of the tokens that it sees, [H_kv, tokens, d] float64."""
    got, got_lse = f64(O), None if lse is None else f64(lse)
    H_q, d = Q.shape[0], Q.shape[2]
    written = np.zeros(Q.shape[1], bool)
    for c in active:
        r = slice(q_off[c], q_off[c + 1])
        written[r] = True
        K, V = kv[c]
        for h in range(H_q):
            hk = h * K.shape[0] // H_q
            want, want_lse, A, size = pg.attention(Q[h, r], K[hk], V[hk], scale)
            n = K.shape[1]
            rel = 2 * (d + 8) * 2.0 ** -23 * size + n * 2.0 ** -24 + 2.0 ** -20
            if dtype == BF16:
                rel += 2.0 ** -8 + 1e-4
            most = np.abs(V[hk]).max() if n else 0.0
            tol = rel * A + n * 2.0 ** -32 * most + HALF[dtype] * np.abs(want) + 1e-30
            err = np.abs(got[h, r] - want)
            assert (err <= tol).all(), f"chunk {c} head {h}: worst {np.max(err / tol)} of the tolerance"
            if lse is not None:
                lse_tol = (d + 8) * 2.0 ** -23 * size + n * 2.0 ** -24 + (1e-4 if dtype == BF16 else 2.0 ** -20) + 2.0 ** -22 * (1 + np.abs(want_lse))
                same = got_lse[h, r] == want_lse
                with np.errstate(invalid="ignore"):  # -inf less -inf, which is the same
                    assert (same | (np.abs(got_lse[h, r] - want_lse) <= lse_tol)).all()
    assert (got[:, ~written] == O_before).all()
    if lse is not None:
        assert (got_lse[:, :len(written)][:, ~written] == 5.0).all()


def run(fc, ctx, *, H_q, H_kv, d, lens, cache, vis, dtype, page=32, sink=0, begin=None, active=None, impl=0, shared=False, plain=0, first=None, cut=None,
        seed=1, scale=0.0, sigma=1.0, span=False):
    """Attention over pages and `plain` plain rows (cut: in two segments that are out of order) against the plain form.  Whatever no chunk
    sees is NaN: rows of pages behind the tokens, pages of tokens outside the windows, plain rows of no segment."""
    W = len(lens)
    off = np.concatenate([[3], 3 + np.cumsum(lens)]).tolist()
    begin_ = begin or [0] * W
    first_ = first or [0] * W
    active = list(range(W)) if active is None else active
    Q = rand((H_q, off[-1] + 2, d), seed, sigma, dtype)
    seen = [pg.seen_tokens(vis[c], sink, begin_[c]) for c in range(W)]
    K, V = (torch.full((H_kv, plain + 9, d), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    segs = ([0, cut, plain], [plain - cut + 5, 2]) if cut else ([0, plain], [4]) if plain else ([0], [])
    row = np.concatenate([np.arange(b - a) + p for a, b, p in zip(segs[0], segs[0][1:], segs[1])] + [np.zeros(0)]).astype(int)
    used = sorted({row[j - cache[c] + first_[c]] for c in range(W) for j in seen[c] if j >= cache[c]})
    K[:, used], V[:, used] = rand((H_kv, len(used), d), seed + 1, sigma, dtype), rand((H_kv, len(used), d), seed + 2, 1.0, dtype)
    kv = []
    pool, t = None, None
    if not span:
        counts = [-(-max(cache) // page)] if shared else [-(-n // page) for n in cache]
        n_pages = sum(counts) + 2
        t = tables(n_pages, counts, max(max(counts), 1), seed)
        pool = filled_pool(fc, n_pages, H_kv, page, d, seed)
        for c in range(len(counts)):  # NaN where nobody looks
            who = range(W) if shared else [c]
            live = {j for w in who for j in seen[w] if j < cache[w]}
            for j in range(counts[c] * page):
                if j not in live:
                    pool.k_codes[t[c, j // page], :, j % page] = 0x7f
                    pool.v_codes[t[c, j // page], :, j % page] = 0xff
        dead = [p for p in range(n_pages) if p not in t]
        pool.k_scales[dead], pool.v_scales[dead] = math.nan, math.nan
        where = numpy_pool(pool)
    for c in range(W):
        paged = [j for j in seen[c] if j < cache[c]]
        rest = row[[j - cache[c] + first_[c] for j in seen[c] if j >= cache[c]]]
        parts = [(f64(K)[:, rest], f64(V)[:, rest])]
        if paged:
            parts.insert(0, tuple(where.rows(w, t[0 if shared else c], paged) for w in (0, 1)))
        kv.append(tuple(np.concatenate(x, 1) for x in zip(*parts)))
    O = torch.full((H_q, off[-1] + 2, d), 9.0, dtype=dtype, device="cuda")
    lse = torch.full((H_q, off[-1] + 4), 5.0, device="cuda")
    ids = i32(list(active) + [-1] * (W - len(active)))
    status = status_word()
    kw = dict(n_sink=sink, kv_begin=begin, lse=lse, scale=scale, impl=impl, status=status)
    if span:
        ctx.chunk_attention_span(Q, K, V, off, vis, *segs, ids, i32([len(active)]), O, **kw)
    else:
        plain_args = (K, V) if plain else (None, None)
        ctx.chunk_attention_kv8(Q, pool, i32(t), cache, *plain_args, off, vis, ids, i32([len(active)]), O, window_first=first, seg_logical_off=segs[0] if plain else None,
                                seg_phys_off=segs[1] if plain else None, **kw)
    assert int(status) == 0
    check(O, lse[:, :off[-1] + 2], f64(Q), kv, off, active, scale or d ** -0.5, dtype, impl, 9.0)
    assert (lse[:, off[-1] + 2:] == 5.0).all()
    return O


IMPLS = [(BF16, 0), (BF16, 2), (BF16, 3), (F32, 0)]
CASES = [
    dict(H_q=1, H_kv=1, lens=[1], cache=[1], vis=[1]),
    dict(H_q=3, H_kv=3, lens=[1], cache=[1000], vis=[1000]),
    dict(H_q=4, H_kv=2, lens=[5], cache=[77], vis=[100], plain=23),
    dict(H_q=2, H_kv=1, lens=[17, 30], cache=[200, 200], vis=[217, 247], plain=47, shared=True, cut=20),
    dict(H_q=8, H_kv=1, lens=[1, 1, 1], cache=[33, 500, 1], vis=[34, 501, 2], plain=3, first=[0, 1, 2], page=16),
    dict(H_q=2, H_kv=2, lens=[300], cache=[513], vis=[813], plain=300, page=128),
    dict(H_q=6, H_kv=2, lens=[3, 0, 140], cache=[0, 50, 260], vis=[9, 50, 270], plain=10, page=64, active=[0, 2]),
    # first tokens and windows: inside a page, over its edge, meeting, behind the end, leaving nothing
    dict(H_q=2, H_kv=2, lens=[4], cache=[700], vis=[704], plain=4, sink=5, begin=[611]),
    dict(H_q=4, H_kv=4, lens=[2, 2, 150], cache=[300, 300, 300], vis=[302, 304, 450], plain=152, sink=40, begin=[41, 250, 333], shared=True, page=16),
    dict(H_q=2, H_kv=1, lens=[7, 7], cache=[100, 90], vis=[100, 90], sink=64, begin=[64, 30]),
    dict(H_q=2, H_kv=1, lens=[7, 130, 3], cache=[100, 100, 100], vis=[60, 0, 100], sink=0, begin=[60, 0, 200]),
    dict(H_q=1, H_kv=1, lens=[6, 6], cache=[20, 500], vis=[150, 520], sink=60, begin=[140, 510], plain=130, cut=33, page=64),
    dict(H_q=2, H_kv=2, lens=[257], cache=[1500], vis=[1757], plain=257, sink=100, begin=[1201], page=32),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype, impl", IMPLS)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c["lens"])) + f"@{c['cache'][0]}")
def test_attention_over_pages(fc, ctx, case, dtype, impl, d):
    run(fc, ctx, d=d, dtype=dtype, impl=impl, **case)


SPANS = [
    dict(H_q=2, H_kv=2, lens=[1], plain=1, vis=[1]),
    dict(H_q=4, H_kv=1, lens=[1], plain=3000, vis=[3000], sink=100, begin=[1700]),
    dict(H_q=2, H_kv=2, lens=[61, 61, 61], plain=800, vis=[678, 739, 800], sink=7, begin=[500, 561, 622], cut=333),
    dict(H_q=3, H_kv=3, lens=[200, 129], plain=1000, vis=[871, 1000], sink=130, begin=[600, 729], cut=129),
    dict(H_q=2, H_kv=1, lens=[9, 9, 9], plain=90, vis=[30, 0, 90], sink=0, begin=[30, 0, 89]),
    dict(H_q=8, H_kv=2, lens=[40], plain=500, vis=[500], sink=600, begin=[499]),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype, impl", IMPLS)
@pytest.mark.parametrize("case", SPANS, ids=lambda c: "-".join(map(str, c["lens"])) + f"@{c['plain']}")
def test_attention_of_a_span(fc, ctx, case, dtype, impl, d):
    run(fc, ctx, d=d, dtype=dtype, impl=impl, span=True, cache=[0] * len(case["lens"]), **case)


@pytest.mark.parametrize("rows", [1, 130])
@pytest.mark.parametrize("d", [64, 128])
def test_a_span_of_everything_is_chunk_attention(fc, ctx, rows, d):
    H, n = 3, 700
    Q, K, V = rand((H, rows, d), 1), rand((H, n, d), 2), rand((H, n, d), 3)
    got, want = torch.zeros_like(Q), torch.zeros_like(Q)
    args = ([0, rows], [n], [0, n], [0], i32([0]), i32([1]))
    ctx.chunk_attention_span(Q, K, V, *args, got, impl=2)
    ctx.chunk_attention(Q, K, V, *args, want, impl=2)
    check(got, None, f64(Q), [(f64(K), f64(V))], [0, rows], [0], d ** -0.5, BF16, 2)
    assert (got.float() - want.float()).abs().max() <= 2 * 2.0 ** -8 * want.float().abs().max()


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_large_logits_sizes_and_scale(fc, ctx, dtype, impl):
    run(fc, ctx, H_q=2, H_kv=1, d=128, lens=[3, 140], cache=[300, 300], vis=[310, 310], plain=10, dtype=dtype, impl=impl, sigma=8.0, scale=0.5, shared=True)


@pytest.mark.parametrize("q_size", [2.0 ** -60, 2.0 ** 60])
def test_attention_queries_of_any_size(fc, ctx, q_size):
    # queries far outside fp16's range over pages whose scales make up for it: the same logits, and the same outputs
    H, d, page, n = 2, 128, 16, 90
    pool, t = filled_pool(fc, 6, H, page, d, 1), i32([[0, 1, 2, 3, 4, 5]])
    Q, one = rand((H, 5, d), 2), (i32([0]), i32([1]))
    want = torch.zeros_like(Q)
    ctx.chunk_attention_kv8(Q, pool, t, [n], None, None, [0, 5], [n], *one, want, impl=3)
    pool.k_scales[:] = pool.k_scales / q_size
    got = torch.zeros_like(Q)
    ctx.chunk_attention_kv8((Q.float() * q_size).to(BF16), pool, t, [n], None, None, [0, 5], [n], *one, got, impl=3)
    assert torch.equal(got, want)


def test_attention_weights_of_many_sizes(fc, ctx):
    # one key of weight 1 beside very many of weight 2^-13 each, whose sum is larger: fp16's small numbers would lose them
    H, d, page, n = 1, 64, 128, 128 * 300
    pool = fc.Kv8Pool.empty(300, H, page, d)
    for c in (pool.k_codes, pool.v_codes):
        c.fill_(0)
    pool.k_scales.fill_(1.0), pool.v_scales.fill_(1.0)
    pool.k_codes[0, 0, 0, 0] = 0x38  # 1
    pool.v_codes[:, :, :, 0] = 0x3c  # 1.5
    pool.v_codes[0, 0, 0, 0] = 0xbc
    Q = torch.zeros((H, 1, d), dtype=F32, device="cuda")
    Q[0, 0, 0] = 13 * math.log(2)
    for dtype in (F32, BF16):
        O, q = torch.zeros((H, 1, d), dtype=dtype, device="cuda"), Q.to(dtype)
        e = math.exp(-float(q[0, 0, 0])) * (n - 1)
        want = 1.5 * (e - 1) / (e + 1)
        ctx.chunk_attention_kv8(q, pool, i32([list(range(300))]), [n], None, None, [0, 1], [n], i32([0]), i32([1]), O, scale=1.0)
        tol = abs(want) * HALF[dtype] + 1.5 * (n * 2.0 ** -24 + 2.0 ** -20 + 128 * 2.0 ** -22 + (2.0 ** -11 if dtype == BF16 else 0))
        assert abs(float(O[0, 0, 0]) - want) <= tol


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_nan_stays_with_who_sees_it(fc, ctx, dtype, impl):
    H, d, page, n = 2, 64, 16, 100
    pool, t = filled_pool(fc, 7, H, page, d, 1), i32([list(range(7))])
    pool.v_codes[2, 0, 3, 5] = 0x7f  # token 35, head 0, dim 5
    pool.k_codes[1, 1, 0, 0] = 0xff  # token 16, head 1
    Q = rand((H, 8, d), 2, 1.0, dtype)
    Q[0, 7, 0] = math.nan
    O = torch.zeros_like(Q)
    lse = torch.zeros((H, 8), device="cuda")
    # chunk 0 sees both tokens, chunk 1 tokens 0-9 and from 36 on, chunk 2 (row 7) the same
    ctx.chunk_attention_kv8(Q, pool, t, [n] * 3, None, None, [0, 4, 7, 8], [n] * 3, i32([0, 1, 2]), i32([3]), O, n_sink=10, kv_begin=[0, 36, 36], lse=lse, impl=impl)
    nan = torch.isnan(O)
    assert nan[0, :4, 5].all() and nan[0, :4].sum() == 4 and nan[1, :4].all() and not nan[:, 4:7].any() and nan[0, 7].all() and not nan[1, 7].any()
    assert torch.isnan(lse[1, :4]).all() and not torch.isnan(lse[0, :7]).any() and torch.isnan(lse[0, 7])


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_many_chunks_each_on_its_own_pages(fc, ctx, dtype, impl):
    W = 64
    lens, cache = [1 + c % 3 for c in range(W)], [1 + 13 * c % 170 for c in range(W)]
    rows = sum(lens)
    first = [sum(lens[:c]) for c in range(W)]
    run(fc, ctx, H_q=2, H_kv=1, d=64, lens=lens, cache=cache, vis=[c + n for c, n in zip(cache, lens)], plain=rows, first=first, page=16, dtype=dtype,
        impl=impl, sink=3, begin=[max(0, c - 60) for c in cache], active=[c for c in range(W) if c % 5])


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_active_list(fc, ctx, dtype, impl):
    # ids that are none are reported and otherwise ignored; a chunk named twice is one chunk; an empty list writes nothing
    H, d, page, n = 2, 128, 64, 150
    pool, t = filled_pool(fc, 3, H, page, d, 1), i32([[2, 0, 1]])
    Q = rand((H, 12, d), 2, 1.0, dtype)
    args = (pool, t, [n] * 3, None, None, [0, 4, 8, 12], [n] * 3)
    want = torch.full_like(Q, 9.0)
    ctx.chunk_attention_kv8(Q, *args, i32([0, 2, -1]), i32([2]), want, impl=impl)
    status, O = status_word(), torch.full_like(Q, 9.0)
    ctx.chunk_attention_kv8(Q, *args, i32([2, 2, 0]), i32([3]), O, impl=impl, status=status)
    assert torch.equal(O, want) and int(status) == 0 and (O[:, 4:8] == 9).all()
    O.fill_(9.0)
    ctx.chunk_attention_kv8(Q, *args, i32([7, 0, 2]), i32([3]), O, impl=impl, status=status)
    assert torch.equal(O, want) and int(status) == fc.STATUS_BITS["bad_index"]
    O.fill_(9.0)
    ctx.chunk_attention_kv8(Q, *args, i32([0, 1, 2]), i32([0]), O, impl=impl)
    assert (O == 9).all()


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_over_entries_that_are_no_page(fc, ctx, dtype, impl):
    # reported; keys and values of those tokens are zeros
    H, d, page, n, rows = 2, 64, 16, 64, 5
    pool, status = filled_pool(fc, 4, H, page, d, 1), status_word()
    Q, O = rand((H, rows, d), 2, 1.0, dtype), torch.zeros((H, rows, d), dtype=dtype, device="cuda")
    pool.k_codes[3], pool.v_codes[3] = 0x7f, 0x7f  # a page that nobody names
    where = numpy_pool(pool)
    for bad in (-1, 4, 2 ** 31 - 1, -2 ** 31):
        status.zero_()
        ctx.chunk_attention_kv8(Q, pool, i32([[0, bad, 2, 1]]), [n], None, None, [0, rows], [n], i32([0]), i32([1]), O, impl=impl, status=status)
        assert int(status) == fc.STATUS_BITS["bad_index"]
        kv = [where.rows(w, [0, 0, 2, 1], range(n)) for w in (0, 1)]
        for x in kv:
            x[:, 16:32] = 0
        check(O, None, f64(Q), [kv], [0, rows], [0], d ** -0.5, dtype, impl)
    status.zero_()  # and nobody minds entries that nobody needs
    ctx.chunk_attention_kv8(Q, pool, i32([[0, -1, 2, 1]]), [n], None, None, [0, rows], [n], i32([0]), i32([1]), O, impl=impl, n_sink=16, kv_begin=[32], status=status)
    assert int(status) == 0


@pytest.mark.parametrize("dtype, page", [(BF16, 16), (BF16, 128), (F32, 32)])
def test_attention_of_very_many_heads(fc, ctx, dtype, page):
    # more blocks than the device holds, each with more steps than its warps know of at a time
    H, d, n = 470, 64, 9001
    g = torch.Generator(device="cuda").manual_seed(1)
    n_pages = -(-n // page)
    codes = [torch.randint(0, 120, (n_pages, H, page, d), dtype=torch.uint8, device="cuda", generator=g) for _ in range(2)]
    codes = [c | torch.randint(0, 2, c.shape, dtype=torch.uint8, device="cuda", generator=g) << 7 for c in codes]
    scales = [(torch.rand((n_pages, H), device="cuda", generator=g) + 0.5) * s for s in (0.004, 0.01)]
    pool, t = fc.Kv8Pool(codes[0], scales[0], codes[1], scales[1]), tables(n_pages, [n_pages], n_pages, 1)
    Q = rand((H, 3, d), 2, 0.3, dtype)
    O, lse, status = torch.zeros_like(Q), torch.zeros((H, 3), device="cuda"), status_word()
    ctx.chunk_attention_kv8(Q, pool, i32(t), [n], None, None, [0, 3], [n], i32([0]), i32([1]), O, n_sink=40, kv_begin=[77], lse=lse, impl=3, status=status)
    assert int(status) == 0
    seen = np.asarray(pg.seen_tokens(n, 40, 77))
    at, row = torch.from_numpy(t[0][seen // page]).cuda(), torch.from_numpy(seen % page).cuda()
    for h in (0, 1, 233, 469):
        kv = [(pg.code_values(c[at, h, row].cpu().numpy()) * f64(z[at, h])[:, None])[None] for c, z in zip(codes, scales)]
        check(O[h:h + 1], lse[h:h + 1], f64(Q[h:h + 1]), [kv], [0, 3], [0], d ** -0.5, dtype, 3)


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_of_a_span_over_many_segments(fc, ctx, dtype, impl):
    # 62 segments in any order, some empty, some a row long, some that follow one another; what lies between them is NaN
    rng, H, d = np.random.default_rng(5), 2, 128
    lens = rng.integers(0, 40, 62)
    lens[[3, 9, 10]] = 0, 1, 1
    order, at, phys = rng.permutation(62), 1, np.zeros(62, int)
    for s in order:
        phys[s], at = at, at + lens[s] + int(rng.integers(0, 3))
    log = np.concatenate([[0], np.cumsum(lens)])
    row = np.concatenate([np.arange(n) + p for n, p in zip(lens, phys)]).astype(int)
    K, V = (torch.full((H, at + 5, d), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    K[:, row], V[:, row] = rand((H, len(row), d), 1, 1.0, dtype), rand((H, len(row), d), 2, 1.0, dtype)
    n = len(row)
    off, vis, begin = [0, 3, 143, 148], [n, n - 100, n // 2], [n - 300, 201, 90]
    Q, O = rand((H, 148, d), 3, 1.0, dtype), torch.zeros((H, 148, d), dtype=dtype, device="cuda")
    status = status_word()
    ctx.chunk_attention_span(Q, K, V, off, vis, log.tolist(), phys.tolist(), i32([0, 1, 2]), i32([3]), O, n_sink=70, kv_begin=begin, impl=impl, status=status)
    assert int(status) == 0
    kv = [tuple(f64(x)[:, row[pg.seen_tokens(v, 70, b)]] for x in (K, V)) for v, b in zip(vis, begin)]
    check(O, None, f64(Q), kv, off, [0, 1, 2], d ** -0.5, dtype, impl)


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_minds_only_entries_that_active_chunks_see(fc, ctx, dtype, impl):
    # a shared sequence of which nobody sees the middle; a batch in which a finished sequence has let go of its pages
    H, d, page, n = 2, 64, 16, 160
    pool, status = filled_pool(fc, 10, H, page, d, 1), status_word()
    where = numpy_pool(pool)
    Q = rand((H, 12, d), 2, 1.0, dtype)
    O = torch.zeros_like(Q)
    t = [0, 1, 2, 3, -1, 77, 6, 7, 8, 9]
    kw = dict(n_sink=5, kv_begin=[20, 100], impl=impl, status=status)
    ctx.chunk_attention_kv8(Q, pool, i32([t]), [64, n], None, None, [0, 6, 12], [64, n], i32([0, 1]), i32([2]), O, **kw)
    assert int(status) == 0
    kv = [tuple(where.rows(w, t, pg.seen_tokens(v, 5, b)) for w in (0, 1)) for v, b in ((64, 20), (n, 100))]
    check(O, None, f64(Q), kv, [0, 6, 12], [0, 1], d ** -0.5, dtype, impl)
    O.fill_(9.0)
    tables_ = i32([t[:4], [-1] * 4, t[6:]])
    ctx.chunk_attention_kv8(Q, pool, tables_, [64] * 3, None, None, [0, 4, 8, 12], [64] * 3, i32([2, 0]), i32([2]), O, impl=impl, status=status)
    assert int(status) == 0
    kv = [tuple(where.rows(w, r, range(64)) for w in (0, 1)) if r[0] >= 0 else None for r in tables_.tolist()]
    check(O, None, f64(Q), kv, [0, 4, 8, 12], [0, 2], d ** -0.5, dtype, impl, 9.0)


@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_strides(fc, ctx, dtype, rows):
    # Q and the plain rows out of a fused projection [tokens, heads, d], O into one, a pool inside a larger one
    H_q, H_kv, d, page, n = 4, 2, 64, 16, 100
    x = rand((rows, H_q + 2 * H_kv, d), 1, 1.0, dtype).transpose(0, 1)
    Q, K, V = x[:H_q], x[H_q:H_q + H_kv], x[H_q + H_kv:]
    O = torch.zeros((rows, H_q, d), dtype=dtype, device="cuda").transpose(0, 1)
    big = filled_pool(fc, 9, 5, page, d, 2)
    pool = fc.Kv8Pool(*(t[1:8, 2:4] for t in (big.k_codes, big.k_scales, big.v_codes, big.v_scales)))
    t = tables(7, [7], 7, 1)
    kv = [np.concatenate([numpy_pool(pool).rows(w, t[0], range(n)), f64(y)], 1) for w, y in ((0, K), (1, V))]
    ctx.chunk_attention_kv8(Q, pool, i32(t), [n], K, V, [0, rows], [n + rows], i32([0]), i32([1]), O)
    check(O, None, f64(Q), [kv], [0, rows], [0], d ** -0.5, dtype, 0)


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_is_reproducible_and_captured(fc, ctx, dtype, impl):
    # a captured call replayed on new data equals the calls one by one; another stream in between does not disturb it
    H, d, page, n = 4, 128, 64, 5000
    pool, t = filled_pool(fc, 80, H, page, d, 1), i32(tables(80, [79], 79, 1))
    Q, K, V = rand((H, 2, d), 2, 1.0, dtype), rand((H, 30, d), 3, 1.0, dtype), rand((H, 30, d), 4, 1.0, dtype)
    args = ([n], K, V, [0, 2], [n + 30], i32([0]), i32([1]))
    O = torch.zeros_like(Q)
    call = lambda q, out: ctx.chunk_attention_kv8(q, pool, t, *args, out, n_sink=70, kv_begin=[1000], impl=impl)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(Q, O)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(Q, O)
    other = torch.cuda.CUDAGraph()
    O2, Q2 = torch.zeros_like(Q), rand((H, 2, d), 9, 1.0, dtype)
    with torch.cuda.graph(other):
        call(Q2, O2)
    for seed in (5, 6, 7):
        Q.copy_(rand((H, 2, d), seed, 1.0, dtype))
        Q2.copy_(rand((H, 2, d), seed + 10, 1.0, dtype))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            other.replay()
        graph.replay()
        torch.cuda.synchronize()
        for q, o in ((Q, O), (Q2, O2)):
            want = torch.zeros_like(q)
            call(q, want)
            assert torch.equal(o, want)


def test_pages_and_append_are_captured(fc, ctx):
    H, d, page = 2, 64, 16
    pool = filled_pool(fc, 20, H, page, d, 1)
    ref, table = pool.tables(3, 8)
    K = rand((H, 20, d), 1)
    ctx.pages_take(ref, table, [0, 0, 0], [3, 0, 0])
    start = ref.clone(), table.clone()

    def turn():
        ctx.pages_fork(pool, ref, table, [0], [1], [37])
        ctx.kv8_append(K, K, pool, table[1:2], [37], ref=ref)
        ctx.pages_take(ref, table, [3, 4, 0], [4, 5, 0])
        ctx.pages_compact(pool, ref, table)
    turn()  # entries 3 of sequence 1 hold nothing yet: its rows from 48 on are dropped
    torch.cuda.synchronize()
    want = ref.clone(), table.clone(), pool.k_codes.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn()
    for _ in range(2):
        ref.copy_(start[0])
        table.copy_(start[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ref, want[0]) and torch.equal(table, want[1])


@pytest.mark.parametrize("dtype, impl", IMPLS)
def test_attention_over_nothing(fc, ctx, dtype, impl):
    # no pages, no plain rows, nothing seen: zeros, and a log-sum of nothing
    H, d, rows = 3, 64, 7
    Q, O, lse = rand((H, rows, d), 1, 1.0, dtype), torch.full((H, rows, d), 9.0, dtype=dtype, device="cuda"), torch.zeros((H, rows), device="cuda")
    args = ([0, rows], [0])
    ctx.chunk_attention_kv8(Q, fc.Kv8Pool.empty(1, H, 16, d), i32([[-1]]), [0], None, None, *args, i32([0]), i32([1]), O, lse=lse, impl=impl)
    assert (O == 0).all() and (lse == -math.inf).all()
    O.fill_(9.0)
    K = torch.full((H, 5, d), math.nan, dtype=dtype, device="cuda")
    ctx.chunk_attention_span(Q, K, K, *args, [0, 5], [0], i32([0]), i32([1]), O, n_sink=3, lse=lse, impl=impl)
    assert (O == 0).all() and (lse == -math.inf).all()


def test_compact_without_tables(fc, ctx):
    for n in (1, 2, 5):
        pool, ref = filled_pool(fc, n, 1, 16, 64, 1), i32([0] * (n - 1) + [3])
        codes, n_used = pool.k_codes.clone(), status_word()
        ctx.pages_compact(pool, ref, torch.zeros((0, 4), dtype=torch.int32, device="cuda"), n_used=n_used)
        assert ref.tolist() == [3] + [0] * (n - 1) and int(n_used) == 1 and torch.equal(pool.k_codes[0], codes[n - 1])


def test_binding_refusals(fc, ctx):
    H, d, page = 2, 64, 16
    pool = filled_pool(fc, 4, H, page, d, 1)
    ref, table = pool.tables(2, 2)
    K = rand((H, 10, d), 1)
    O, ids, one = torch.zeros_like(K), i32([0]), i32([1])
    bad = [
        lambda: ctx.kv8_append(K[:1], K, pool, table, [0]),
        lambda: ctx.kv8_append(K, K.float(), pool, table, [0]),
        lambda: ctx.kv8_append(K, K, pool, table, [30]),                      # behind the table's entries
        lambda: ctx.kv8_append(K, K, pool, table, [0], [0, 11]),
        lambda: ctx.kv8_append(K, K, pool, table.cpu(), [0]),
        lambda: ctx.kv8_append(K, K, pool, table.long(), [0]),
        lambda: ctx.kv8_append(K, K, pool, table, [0], ref=ref[:3]),
        lambda: ctx.kv8_unpack(pool, table, [25], [0, 10]),
        lambda: ctx.kv8_unpack(pool, table, [0, 0, 0], [0, 1, 2, 3]),
        lambda: ctx.pages_take(ref, table, [0], [3]),
        lambda: ctx.pages_take(ref, table, [0, 0, 0], [1, 1, 1]),
        lambda: ctx.pages_drop(ref.float(), table, [0], [1]),
        lambda: ctx.pages_fork(pool, ref, table, [0], [1], [33]),
        lambda: ctx.pages_fork(pool, ref[:2], table, [0], [1], [3]),
        lambda: ctx.pages_fork(pool, ref, table, [0], [0], [3]),
        lambda: ctx.pages_compact(pool, ref[1:], table),
        lambda: ctx.chunk_attention_kv8(K, pool, table, [33], None, None, [0, 10], [33], ids, one, O),
        lambda: ctx.chunk_attention_kv8(K, pool, table, [20], None, None, [0, 10], [21], ids, one, O),
        lambda: ctx.chunk_attention_kv8(K, pool, table, [20], K, None, [0, 10], [20], ids, one, O),
        lambda: ctx.chunk_attention_kv8(K, pool, table, [20], None, None, [0, 11], [20], ids, one, O),
        lambda: ctx.chunk_attention_kv8(K, pool, table, [20], None, None, [0, 10], [20], ids, one, O, kv_begin=[0, 0]),
        lambda: ctx.chunk_attention_kv8(K, pool, table, [20], None, None, [0, 10], [20], ids, one, O.float()),
        lambda: ctx.chunk_attention_span(K, None, None, [0, 10], [10], [0, 10], [0], ids, one, O),
        lambda: ctx.chunk_attention_span(K, K, K, [0, 10], [11], [0, 10], [0], ids, one, O),
        lambda: ctx.chunk_attention_span(K, K, K, [0, 10], [10], [0, 10], [1], ids, one, O),
        lambda: ctx.chunk_attention_span(K, K[:, ::2, ::2], K, [0, 10], [10], [0, 10], [0], ids, one, O),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(fc.FcError):
            f()
            pytest.fail(f"call {i} was taken")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_rolling_generation_that_branches(fc, ctx, dtype):
    # chunk by chunk: attend over [first tokens | window in pages | the chunk's own rows], append the chunk, let go of what has left the window; then
    # branch, go on in both, close ranks, and attend again: the same outputs as over the plain values of what was appended
    H_q, H_kv, d, page, n_c, sink, span = 4, 2, 64, 16, 43, 20, 100
    pool = fc.Kv8Pool.empty(60, H_kv, page, d)
    ref, table = pool.tables(3, 40)
    where, want = numpy_pool(pool), pg.Pages(ref.tolist(), table.tolist())
    length, dropped = [0, 0, 0], [2, 2, 2]
    ids, one = i32([0]), i32([1])

    def step(c, seed):
        Q, K, V = rand((H_q, n_c, d), seed, 1.0, dtype), rand((H_kv, n_c, d), seed + 1, 1.0, dtype), rand((H_kv, n_c, d), seed + 2, 1.0, dtype)
        n, vis = length[c], length[c] + n_c
        begin = max(0, vis - span)
        O = torch.zeros_like(Q)
        ctx.chunk_attention_kv8(Q, pool, table[c:c + 1], [n], K, V, [0, n_c], [vis], ids, one, O, n_sink=sink, kv_begin=[begin])
        tokens = [j for j in pg.seen_tokens(vis, sink, begin) if j < n]
        kv = [np.concatenate([where.rows(w, want.table[c], tokens), f64(x)], 1) for w, x in ((0, K), (1, V))]
        check(O, None, f64(Q), [kv], [0, n_c], [0], d ** -0.5, dtype, 0)
        first, last = [0] * 3, [0] * 3
        first[c], last[c] = -(-n // page), -(-vis // page)
        ctx.pages_take(ref, table, first, last)
        want.take(first, last)
        ctx.kv8_append(K, V, pool, table[c:c + 1], [n], ref=ref)
        where.append(f64(K), 0, want.table[c], n)
        where.append(f64(V), 1, want.table[c], n)
        length[c] = vis
        gone = max(0, length[c] + n_c - span) // page  # the next chunk's window begins here
        if gone > dropped[c]:
            first, last = [0] * 3, [0] * 3
            first[c], last[c] = dropped[c], gone
            ctx.pages_drop(ref, table, first, last)
            want.drop(first, last)
            dropped[c] = gone
        same_pages(ref, table, want)

    for i in range(6):
        step(0, 10 * i)
    ctx.pages_fork(pool, ref, table, [0, 0], [1, 2], [length[0], length[0] - 9])
    copies = want.fork([0, 0], [1, 2], [length[0], length[0] - 9], page)
    for x in where.codes + where.scales:
        for a, b in copies:
            x[b] = x[a]
    length[1], length[2], dropped[1], dropped[2] = length[0], length[0] - 9, dropped[0], dropped[0]
    for i in range(3):
        for c in (2, 0, 1):
            step(c, 100 + 30 * i + 10 * c)
    ctx.pages_drop(ref, table, [0, 0, 0], [0, 40, 0])
    want.drop([0, 0, 0], [0, 40, 0])
    ctx.pages_compact(pool, ref, table)
    moves = want.compact()
    for x in where.codes + where.scales:
        for a, b in moves:
            x[b] = x[a]
    same_pages(ref, table, want)
    assert moves and max(p for row in want.table for p in row) < sum(r > 0 for r in want.ref)
    step(0, 300)
    step(2, 310)
    # the keys of what is left, as the score reads them
    keep = list(range(dropped[2] * page, length[2]))
    keys = ctx.kv8_unpack(pool, table[2:3], [keep[0]], [0, len(keep)], keys_only=True, dtype=dtype)[0]
    assert np.array_equal(f64(keys), where.rows(0, want.table[2], keep))
