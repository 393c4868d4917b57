"""The calls around the 4-bit store against plain forms in 64 bits (plain_forms.py), at the sizes and masks where they can go wrong.

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value, one to fp32 by 2^-24.
  rotation   fp32 inside: the angle's turn is rounded to fp32 (2^-24 pi), sincospi adds two units (2^-23 each), the norm
             (a chain of 8 and a tree of 4 or 5 sums, a square root, a division, two products) at most 10 units, the
             two products and the sum 3: below 2e-6 of the size of the pair, plus the output's rounding.
  packing    none: codes and scales are compared as bits.
  attention  fp32: a logit is off by at most (d + 4) 2^-24 |q||k| scale (the products of parts that are left out over a window are 1 of the
             4: below 2^-24 of each product), a weight by twice that, and sums of n terms by
             n 2^-24, all relative to A = sum p |v|.  The tensor-core kernels round each weight to bf16 (2^-8 A) and take
             exponentials good to 1e-4 (A again); then the output's rounding.  The log of the weights' sum is off by the logit's
             error, the sum's n 2^-24, the exponentials' 1e-4, and its own rounding and that of the logarithm (2^-22).
"""
import math

import numpy as np
import pytest
import torch

import plain_forms as pf
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


# ------------------------------------------------------------------------------------ fc_qk_norm_rope

def check_turned(got, x, dtype, **kw):
    want, size = pf.norm_rope(f64(x), **kw)
    err = np.abs(f64(got) - want)
    tol = HALF[dtype] * np.abs(want) + 2e-6 * size + 1e-30
    assert (err <= tol).all(), f"worst {np.max(err / tol)} of the tolerance"


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d, axes", [(128, (44, 42, 42)), (64, (24, 20, 20)), (128, (16, 56, 56)), (64, (0, 32, 0)), (128, (2, 6, 22))])
@pytest.mark.parametrize("T, H_q, H_kv", [(1, 3, 1), (7, 4, 2), (333, 6, 2)])
def test_norm_rope(fc, ctx, T, H_q, H_kv, d, axes, dtype, halves):
    # inputs are slices of a fused projection [T, q | k | v]; every token has a place of its own
    x = rand((T, H_q + 2 * H_kv, d), 11 * T + d, 2.0, dtype).transpose(0, 1)
    Q, K = x[:H_q], x[H_q:H_q + H_kv]
    pos = torch.randint(-3000, 3000, (T, 3), generator=torch.Generator().manual_seed(T)).int()
    wq, wk = rand((d,), 3, 0.3, F32) + 1, rand((d,), 4, 0.3, F32) + 1
    kw = dict(axes=axes, pairing=fc.ROPE_HALVES if halves else fc.ROPE_PAIRS)
    Qo, Ko = ctx.qk_norm_rope(Q, K, pos=pos.cuda(), q_weight=wq, k_weight=wk, **kw)
    check_turned(Qo, Q, dtype, pos=pos.numpy(), axes=axes, halves=halves, weight=f64(wq))
    check_turned(Ko, K, dtype, pos=pos.numpy(), axes=axes, halves=halves, weight=f64(wk))


@pytest.mark.parametrize("dtype, halves", [(BF16, False), (F32, True)])
def test_norm_rope_grid_no_norm_no_weight(fc, ctx, dtype, halves):
    axes, grid, T = (44, 42, 42), (5, 3, 7), 50  # two whole frames and part of a third
    Q, K = rand((2, T, 128), 1, 1.0, dtype), rand((2, T, 128), 2, 1.0, dtype)
    pairing = fc.ROPE_HALVES if halves else fc.ROPE_PAIRS
    pos = pf.grid_positions(T, *grid)
    for norm in (False, True):
        Qo, Ko = ctx.qk_norm_rope(Q, K, axes=axes, grid=grid, norm=norm, pairing=pairing)
        check_turned(Qo, Q, dtype, pos=pos, axes=axes, halves=halves, norm=norm)
        check_turned(Ko, K, dtype, pos=pos, axes=axes, halves=halves, norm=norm)
    # keys alone, other frequencies, and into rows of a larger store, whose other rows stay
    freq = np.linspace(2.0, 0.001, 64)
    dst = torch.full((2, T + 9, 128), 7.0, dtype=dtype, device="cuda")
    none, Ko = ctx.qk_norm_rope(None, K, axes=axes, grid=grid, pairing=pairing, inv_freq=freq, K_out=dst[:, 4:4 + T])
    assert none is None
    check_turned(Ko, K, dtype, pos=pos, axes=axes, halves=halves, freq=freq)
    assert (dst[:, :4] == 7).all() and (dst[:, 4 + T:] == 7).all()
    # nothing turns: norms alone, without places
    Qo, _ = ctx.qk_norm_rope(Q, None, axes=(0, 0, 0), pairing=pairing)
    check_turned(Qo, Q, dtype, pos=pos, axes=(0, 0, 0))
    # neither: a copy
    assert torch.equal(ctx.qk_norm_rope(Q, None, axes=(0, 0, 0), norm=False)[0], Q)


@pytest.mark.parametrize("halves", [False, True])
def test_rope_far_positions_and_back(fc, ctx, halves):
    far = [[2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7], [-2 ** 31, 2 ** 31 - 1, 0], [1, 123456789, -987654321], [0, 0, 0]]
    pos = torch.tensor(far, dtype=torch.int32).cuda()
    K = rand((3, 4, 64), 5, 1.0, F32)
    kw = dict(axes=(24, 20, 20), norm=False, pairing=fc.ROPE_HALVES if halves else fc.ROPE_PAIRS)
    _, Y = ctx.qk_norm_rope(None, K, pos=pos, **kw)
    check_turned(Y, K, F32, pos=np.asarray(far), axes=kw["axes"], halves=halves, norm=False)
    # in place, and back again
    pos = torch.randint(-10 ** 9, 10 ** 9, (4, 3), generator=torch.Generator().manual_seed(1)).int().cuda()
    X = K.clone()
    ctx.qk_norm_rope(None, X, pos=pos, K_out=X, **kw)
    ctx.qk_norm_rope(None, X, pos=-pos, K_out=X, **kw)
    size = np.hypot(f64(K).max(), f64(K).max())
    assert np.abs(f64(X) - f64(K)).max() <= 4e-6 * size * 2


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d, axes", [(128, (2, 6, 22)), (64, (24, 20, 18)), (128, (0, 32, 64)), (64, (0, 0, 0))])
def test_rope_elements_behind_the_sections_pass_through(fc, ctx, d, axes, dtype, halves):
    t, T = sum(axes), 9
    X = rand((3, T, d), 7, 1.0, dtype)
    g = torch.Generator().manual_seed(d)
    odd = torch.tensor([math.inf, -math.inf, math.nan, -0.0, 0.0, 1e-39, -3e38])
    hit = torch.rand((3, T, d - t), generator=g) < 0.5
    X[..., t:] = torch.where(hit, odd[torch.randint(0, 7, hit.shape, generator=g)], X[..., t:].float().cpu()).to(dtype).cuda()
    pos = torch.randint(-3000, 3000, (T, 3), generator=g).int()
    kw = dict(axes=axes, pos=pos.cuda(), pairing=fc.ROPE_HALVES if halves else fc.ROPE_PAIRS)
    bits = torch.int16 if dtype == BF16 else torch.int32
    nan = torch.isnan(X)
    Y = X.clone()
    for out in (ctx.qk_norm_rope(X, None, norm=False, **kw)[0], ctx.qk_norm_rope(None, Y, norm=False, K_out=Y, **kw)[1]):
        assert torch.equal(torch.isnan(out), nan)
        same = out.contiguous().view(bits) == X.view(bits)
        assert (same | nan)[..., t:].all()
        check_turned(out[..., :t], X[..., :t], dtype, pos=pos.numpy(), axes=axes, halves=halves, norm=False)
    # normed: an element that passes through has its own weight, not its neighbour's
    X = rand((3, T, d), 8, 1.0, dtype)
    X[..., t::3] = -0.0
    w = rand((d,), 3, 0.3, F32) + 1
    w[-1] = math.inf
    out = ctx.qk_norm_rope(X, None, q_weight=w, **kw)[0]
    want, size = pf.norm_rope(f64(X), pos.numpy(), axes, halves=halves, weight=np.append(f64(w)[:-1], 1.0))
    assert (np.abs(f64(out) - want) <= HALF[dtype] * np.abs(want) + 2e-6 * size)[..., :-1].all()
    assert (torch.isinf(out[..., -1]) | torch.isnan(out[..., -1])).all()
    assert (torch.signbit(out) == torch.signbit(X))[..., t:-1].all()


def test_norm_rope_many_tokens_in_place(fc, ctx):
    # more rows than resident groups, so that a group walks over several heads; q in place
    T, H = 5000, 24
    Q, K = rand((H, T, 64), 1), rand((H, T, 64), 2)
    X = Q.clone()
    _, Ko = ctx.qk_norm_rope(X, K, axes=(24, 20, 20), grid=(0, 30, 52), Q_out=X)
    pos = pf.grid_positions(T, 0, 30, 52)
    pick = [0, 1, 1559, 1560, 3119, 4999]
    for got, src in ((X, Q), (Ko, K)):
        check_turned(got[:, pick], src[:, pick], BF16, pos=pos[pick], axes=(24, 20, 20))


def test_norm_rope_zero_row_and_nonfinite(fc, ctx):
    Q = torch.zeros((1, 3, 64), device="cuda")
    Q[0, 1, 5] = float("nan")
    Q[0, 2, 5] = float("inf")
    out = ctx.qk_norm_rope(Q, None, axes=(24, 20, 20), grid=(0, 1, 3))[0]
    assert (out[0, 0] == 0).all() and torch.isnan(out[0, 1]).all()
    assert torch.isnan(out[0, 2, 4:6]).all() or torch.isnan(out[0, 2, 5])  # inf / inf


def test_norm_of_a_row_with_an_infinity(fc, ctx):
    # the infinite element is inf / inf, which its pair takes on; every other element is x / inf
    Q = rand((1, 3, 64), 1, 1.0, F32)
    Q[0, 2, 5] = float("inf")
    for halves, pair in ((fc.ROPE_PAIRS, [4, 5]), (fc.ROPE_HALVES, [5, 17])):
        out = ctx.qk_norm_rope(Q, None, axes=(24, 20, 20), grid=(0, 1, 3), pairing=halves)[0]
        nan = torch.isnan(out)
        assert nan[0, 2].nonzero().flatten().tolist() == pair and int(nan.sum()) == 2
        assert (out[0, 2][~nan[0, 2]] == 0).all()


# ------------------------------------------------------------------------------------ fc_kv4_pack / fc_kv4_unpack

def check_packed(cache, K, V, rows=slice(None)):
    for x, codes, scales in ((K, cache.k_codes, cache.k_scales), (V, cache.v_codes, cache.v_scales)):
        want_c, want_s, _ = pf.quantise(f64(x))
        assert np.array_equal(codes[:, rows].cpu().numpy(), pf.code_bytes(want_c))
        np.testing.assert_array_equal(f64(scales[:, rows]), want_s)


def same_store(a, b):
    return all(torch.equal(getattr(a, n).contiguous().view(torch.uint8), getattr(b, n).contiguous().view(torch.uint8))
               for n in ("k_codes", "k_scales", "v_codes", "v_scales"))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H, n, d", [(1, 1, 64), (3, 33, 128), (2, 257, 64), (5, 1000, 128)])
def test_pack_and_unpack(fc, ctx, H, n, d, dtype):
    K, V = rand((H, n, d), n, 1.0, dtype), rand((H, n, d), n + 1, 0.01, dtype)
    status = status_word()
    cache = ctx.kv4_pack(K, V, fc.Kv4Cache.empty(H, n, d), status=status)
    check_packed(cache, K, V)
    assert int(status) == 0
    for out in (BF16, F32):
        Ku, Vu = ctx.kv4_unpack(cache, dtype=out)
        assert np.array_equal(f64(Ku), pf.quantise(f64(K))[2]) and np.array_equal(f64(Vu), pf.quantise(f64(V))[2])
        # packing what was unpacked changes nothing that is read back
        again = ctx.kv4_pack(Ku, Vu, fc.Kv4Cache.empty(H, n, d))
        assert np.abs(f64(ctx.kv4_unpack(again, dtype=F32)[0]) - f64(Ku)).max() <= np.abs(f64(Ku)).max() / 7
    # keys only, a part of the rows, a strided destination
    if n > 2:
        dst = torch.full((H, n + 2, d), 5.0, dtype=dtype, device="cuda")
        Ku, none = ctx.kv4_unpack(cache, row=1, n=n - 2, K_dst=dst[:, 1:n - 1], keys_only=True)
        assert none is None and np.array_equal(f64(Ku), pf.quantise(f64(K))[2][:, 1:n - 1])
        assert (dst[:, 0] == 5).all() and (dst[:, n - 1:] == 5).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H, n, d", [(2, 33, 128), (3, 257, 64)])
def test_packing_again_gives_the_same_store(fc, ctx, H, n, d, dtype):
    # rounding a scale up to five bits adds less than a sixteenth, so a group's largest code is 7 and 7 s / 7 is s again
    K, V = rand((H, n, d), n, 1.0, F32), rand((H, n, d), n + 1, 0.01, F32)
    V *= torch.exp2(torch.randint(-60, 60, (H, n, 1), generator=torch.Generator().manual_seed(3)).float()).cuda()
    K[0, 3], V[1, 5, :32] = 0.0, 0.0
    cache = ctx.kv4_pack(K, V, fc.Kv4Cache.empty(H, n, d))
    assert same_store(ctx.kv4_pack(*ctx.kv4_unpack(cache, dtype=dtype), fc.Kv4Cache.empty(H, n, d)), cache)


@pytest.mark.parametrize("d", [64, 128])
def test_slices_of_a_store(fc, ctx, d):
    # a store seen from an odd row on, rows before heads: every call takes it
    H, n, first = 3, 45, 7
    t = [torch.zeros((n + 20, H, k), dtype=dt, device="cuda").transpose(0, 1) for k, dt in 2 * ((d // 2, torch.uint8), (d // 32, BF16))]
    part = fc.Kv4Cache(*(x[:, first:first + n] for x in t))
    K, V = rand((H, n, d), 1), rand((H, n, d), 2)
    ctx.kv4_pack(K, V, part)
    check_packed(part, K, V)
    assert all((x[:, :first] == 0).all() and (x[:, first + n:] == 0).all() for x in t)
    Ku, Vu = ctx.kv4_unpack(part, row=3, n=n - 3)
    assert np.array_equal(f64(Ku), pf.quantise(f64(K))[2][:, 3:]) and np.array_equal(f64(Vu), pf.quantise(f64(V))[2][:, 3:])
    again = ctx.kv4_pack(None, None, fc.Kv4Cache.empty(H, n, d), old=part)
    assert same_store(again, part)
    for rows in (2, 300):
        Q = rand((H, rows, d), 3)
        O = torch.zeros_like(Q)
        ctx.chunk_attention_kv4(Q, part, None, None, [0, rows], [n], i32([0]), i32([1]), O)
        check_attention(O, None, *pf.attention(f64(Q), pf.quantise(f64(K))[2], pf.quantise(f64(V))[2], [0, rows], [n], [0]), BF16, True, n, d)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pack_ties_extremes_and_strides(fc, ctx, dtype):
    x = torch.zeros((2, 40, 64), dtype=F32)
    halfs = torch.arange(-7, 7).float() + 0.5
    for r, s in enumerate([1.0, 1.0625, 1.9375, 2.0 ** -100, 1.5 * 2.0 ** 100, 2.0 ** -126, 1.125 * 2.0 ** 60]):
        x[0, r, :14] = halfs * s  # every tie of the scale s, which the row's largest, 7 s, sets
        x[0, r, 31] = 7 * s
        x[1, r, :14] = halfs * s * (1 + 2.0 ** -7)  # just above, and just below
        x[1, r, 14:28] = halfs * s * (1 - 2.0 ** -7)
        x[1, r, 31] = -7 * s
    x[0, 10, :2] = torch.tensor([3.3e38, -3.3e38])  # the scale's upper end: values saturate
    x[0, 11, :3] = torch.tensor([1e-40, -3e-39, 2.0 ** -130])  # below the lower end
    x[0, 12, 40] = 1e-45
    g = torch.Generator().manual_seed(3)
    x[:, 20:] = torch.randn((2, 20, 64), generator=g) * torch.exp2(torch.randint(-60, 60, (2, 20, 1), generator=g).float())
    # heads and rows in another order than packed: [rows, heads, d] seen as [heads, rows, d]
    X = x.to(dtype).transpose(0, 1).contiguous().cuda().transpose(0, 1)
    cache = ctx.kv4_pack(X, X, fc.Kv4Cache.empty(2, 40, 64))
    check_packed(cache, X, X)


def test_pack_fp32_next_to_ties(fc, ctx):
    # values one fp32 step on either side of every tie
    s = torch.tensor([1.0, 1.0625, 1.1875, 1.3125, 1.4375, 1.5625, 1.8125, 1.9375])
    ties = (torch.arange(-7, 7).float() + 0.5) * s[:, None]
    x = torch.zeros((1, 8, 64))
    x[0, :, :14] = torch.nextafter(ties, torch.tensor(math.inf))
    x[0, :, 16:30] = torch.nextafter(ties, torch.tensor(-math.inf))
    x[0, :, 31] = 7 * s
    x[0, :, 32:46] = ties
    x[0, :, 63] = -7 * s
    X = x.cuda()
    check_packed(ctx.kv4_pack(X, X, fc.Kv4Cache.empty(1, 8, 64)), X, X)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pack_nonfinite_groups(fc, ctx, dtype):
    K, V = rand((2, 5, 128), 1, 1.0, dtype), rand((2, 5, 128), 2, 1.0, dtype)
    K[0, 1, 40], K[1, 2, 0], K[1, 2, 127] = float("nan"), float("inf"), -float("inf")
    status = status_word()
    cache = ctx.kv4_pack(K, V, fc.Kv4Cache.empty(2, 5, 128), status=status)
    check_packed(cache, K, V)
    assert int(status) == fc.STATUS_BITS["nonfinite"]
    Ku, Vu = ctx.kv4_unpack(cache, dtype=dtype)
    bad = torch.isnan(Ku)
    assert bad[0, 1, 32:64].all() and bad[1, 2, :32].all() and bad[1, 2, 96:].all() and int(bad.sum()) == 96
    assert not torch.isnan(Vu).any()


@pytest.mark.parametrize("dtype, d", [(BF16, 128), (F32, 64)])
def test_pack_append_and_compact(fc, ctx, dtype, d):
    H, n_old, n_new = 3, 301, 77
    K, V = rand((H, n_old + n_new, d), 1, 1.0, dtype), rand((H, n_old + n_new, d), 2, 1.0, dtype)
    whole = ctx.kv4_pack(K, V, fc.Kv4Cache.empty(H, n_old + n_new, d))
    # appended in two pieces, the second of one row: the same store; rows before and behind stay
    cache = fc.Kv4Cache.empty(H, n_old + n_new + 4, d)
    for t in (cache.k_codes, cache.v_codes):
        t.fill_(0x5A)
    for a, b in ((0, n_old + n_new - 1), (n_old + n_new - 1, n_old + n_new)):
        ctx.kv4_pack(K[:, a:b], V[:, a:b], cache, dst_row=2 + a)
    inner = fc.Kv4Cache(*(t[:, 2:-2] for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)))
    assert same_store(inner, whole)
    assert (cache.k_codes[:, :2] == 0x5A).all() and (cache.v_codes[:, -2:] == 0x5A).all()
    # a kept list per head over [old | new]; old rows are copied as bits, not packed again
    old = fc.Kv4Cache(*(t[:, :n_old].clone() for t in (whole.k_codes, whole.k_scales, whole.v_codes, whole.v_scales)))
    g = torch.Generator().manual_seed(5)
    kept = torch.stack([torch.randperm(n_old + n_new, generator=g)[:200].sort().values for _ in range(H)]).int().cuda()
    got = ctx.kv4_pack(K[:, n_old:], V[:, n_old:], fc.Kv4Cache.empty(H, 200, d), old=old, kept_idx=kept)
    at = kept.long()
    for n in ("k_codes", "k_scales", "v_codes", "v_scales"):
        src = getattr(whole, n)
        assert torch.equal(getattr(got, n), torch.gather(src, 1, at[..., None].expand(-1, -1, src.shape[2])))
    # old rows only; all rows without a list
    got = ctx.kv4_pack(None, None, fc.Kv4Cache.empty(H, 9, d), old=old, kept_idx=kept[:, :9].clamp(max=n_old - 1).contiguous())
    assert torch.equal(got.k_codes[0, 0], old.k_codes[0, int(kept[0, 0].clamp(max=n_old - 1))])
    assert same_store(ctx.kv4_pack(K[:, n_old:], V[:, n_old:], fc.Kv4Cache.empty(H, n_old + n_new, d), old=old), whole)


def test_pack_within_one_store(fc, ctx):
    # a store may be packed from its own rows as long as what is read and what is written lie apart
    H, n, d = 2, 40, 64
    K, V = rand((H, n, d), 1), rand((H, n, d), 2)
    store = ctx.kv4_pack(K, V, fc.Kv4Cache.empty(H, 2 * n, d))
    kept = torch.arange(n - 1, -1, -1).repeat(H, 1).int().cuda()
    ctx.kv4_pack(None, None, store, old=store, n_old=n, kept_idx=kept, dst_row=n)
    assert torch.equal(store.k_codes[:, n:].flip(1), store.k_codes[:, :n]) and torch.equal(store.v_scales[:, n:].flip(1), store.v_scales[:, :n])
    with pytest.raises(fc.FcError, match="invalid argument"):
        ctx.kv4_pack(None, None, store, old=store, n_old=n, kept_idx=kept, dst_row=n - 1)


@pytest.mark.parametrize("layout", ["heads", "rows", "scales in the rows"])
def test_pack_between_slices_that_lie_apart(fc, ctx, layout):
    H, n, d = 3, 40, 128
    if layout == "scales in the rows":  # 64 bytes of codes, then 8 of scales, 8 unused
        bufs = [torch.zeros((H, 2 * n + 3, 80), dtype=torch.uint8, device="cuda") for _ in range(2)]
        t = [x for b in bufs for x in (b[..., :64], b.view(BF16)[..., 32:36])]
    else:
        shapes = 2 * (((H, 2 * n + 3, d // 2), torch.uint8), ((H, 2 * n + 3, d // 32), BF16))
        t = [torch.zeros(s if layout == "heads" else (s[1], s[0], s[2]), dtype=dt, device="cuda") for s, dt in shapes]
        t = t if layout == "heads" else [x.transpose(0, 1) for x in t]
    part = lambda a, b: fc.Kv4Cache(*(x[:, a:b] for x in t))  # noqa: E731
    K, V = rand((H, n, d), 1), rand((H, n, d), 2)
    for a, to in ((0, n), (n, 0), (3, n + 3)):
        for x in t:
            x.zero_()
        old = ctx.kv4_pack(K, V, part(a, a + n))
        check_packed(old, K, V)
        got = ctx.kv4_pack(None, None, part(to, to + n), old=old)
        check_packed(got, K, V)
        check_packed(old, K, V)
        with pytest.raises(fc.FcError, match="invalid argument"):
            ctx.kv4_pack(None, None, part(a + 1, a + 1 + n), old=old)
        check_packed(old, K, V)


def test_pack_bad_index_leaves_the_row(fc, ctx):
    H, n, d = 2, 50, 128
    K, V = rand((H, n, d), 1), rand((H, n, d), 2)
    kept = torch.arange(n).repeat(H, 1).int()
    kept[0, 3], kept[1, 7], kept[1, 49] = -1, n, 2 ** 31 - 1
    cache = fc.Kv4Cache.empty(H, n, d)
    for t in (cache.k_codes, cache.v_codes):
        t.fill_(0x77)
    for t in (cache.k_scales, cache.v_scales):
        t.fill_(3.0)
    status = status_word()
    ctx.kv4_pack(K, V, cache, kept_idx=kept.cuda(), status=status)
    assert int(status) == fc.STATUS_BITS["bad_index"]
    want = ctx.kv4_pack(K, V, fc.Kv4Cache.empty(H, n, d))
    for h, r in ((0, 3), (1, 7), (1, 49)):
        assert (cache.k_codes[h, r] == 0x77).all() and (cache.v_scales[h, r] == 3).all()
        cache.k_codes[h, r], cache.v_codes[h, r] = want.k_codes[h, r], want.v_codes[h, r]
        cache.k_scales[h, r], cache.v_scales[h, r] = want.k_scales[h, r], want.v_scales[h, r]
    assert same_store(cache, want)


def test_store_past_32_bit_offsets(fc, ctx):
    # two heads 4.4e9 bytes of codes apart, rows 96 bytes apart
    H, n, d, far = 2, 70, 128, 4_400_000_000
    buf = torch.zeros(far + n * 96 + 64, dtype=torch.uint8, device="cuda")
    codes = torch.as_strided(buf, (H, n, d // 2), (far // 16 * 16, 96, 1))
    cache = fc.Kv4Cache(codes, torch.zeros((H, n, 4), dtype=BF16, device="cuda"), torch.as_strided(buf, codes.shape, codes.stride(), 0),
                        torch.zeros((H, n, 4), dtype=BF16, device="cuda"))
    K = rand((H, n, d), 1)
    ctx.kv4_pack(K, K, cache)
    check_packed(cache, K, K)
    assert np.array_equal(f64(ctx.kv4_unpack(cache)[0]), pf.quantise(f64(K))[2])
    Q = rand((H, 3, d), 2)
    O = torch.zeros_like(Q)
    ctx.chunk_attention_kv4(Q, cache, None, None, [0, 3], [n], i32([0]), i32([1]), O)
    kv = pf.quantise(f64(K))[2]
    check_attention(O, None, *pf.attention(f64(Q), kv, kv, [0, 3], [n], [0]), BF16, True, n, d)


# ------------------------------------------------------------------------------------ fc_chunk_attention_kv4

def check_attention(O, lse, want, want_lse, A, size, dtype, tensor_cores, n, d, rows=slice(None)):
    rel = 2 * (d + 4) * 2.0 ** -24 * size + n * 2.0 ** -24
    if tensor_cores:
        rel += 2.0 ** -8 + 1e-4
    tol = rel * A + HALF[dtype] * np.abs(want) + 1e-30
    err = np.abs(f64(O) - want)[:, rows]
    assert (err <= tol[:, rows]).all(), f"worst {np.max(err / tol[:, rows])} of the tolerance"
    if lse is not None:
        got, w = f64(lse)[:, rows], want_lse[:, rows]
        assert np.array_equal(np.isneginf(got), np.isneginf(w))
        fine = np.isfinite(w)
        tol = ((d + 4) * size + n) * 2.0 ** -24 + 1e-4 * tensor_cores + 2.0 ** -22 * np.maximum(1.0, np.abs(w[fine]))
        assert (np.abs(got[fine] - w[fine]) <= tol).all()


def packed_store(fc, ctx, H, n, d, seed, sigma=1.0, extra=0):
    """A store of n + extra rows whose last rows hold NaN: they are never to be read."""
    K, V = rand((H, n + extra, d), seed, sigma, F32), rand((H, n + extra, d), seed + 1, sigma, F32)
    if extra:
        K[:, n:], V[:, n:] = float("nan"), float("nan")
    cache = ctx.kv4_pack(K, V, fc.Kv4Cache.empty(H, n + extra, d))
    return cache, pf.quantise(f64(K[:, :n]))[2], pf.quantise(f64(V[:, :n]))[2]


def run_attention(fc, ctx, *, H_q, H_kv, d, lens, n_cache, win, active, dtype, impl=0, cut=None, seed=1, scale=0.0, sigma=1.0):
    """Chunks of `lens` rows; win: each chunk's own tokens follow the clean region, chunk-causally; cut: the chunks'
    visible lengths instead.  The window lies in two pieces in reverse order, with NaN rows around and between."""
    off = [0] + list(np.cumsum(lens))
    rows = off[-1]
    cache, Kc, Vc = packed_store(fc, ctx, H_kv, n_cache, d, seed, sigma, extra=3) if n_cache else (None, np.zeros((H_kv, 0, d)), np.zeros((H_kv, 0, d)))
    Q = rand((H_q, rows, d), seed + 2, sigma, dtype)
    vis = [n_cache + (off[c + 1] if win else 0) for c in range(len(lens))] if cut is None else cut
    K = V = None
    Kw, Vw, seg = np.zeros((H_kv, 0, d)), np.zeros((H_kv, 0, d)), {}
    if win:
        Kl, Vl = rand((H_kv, rows, d), seed + 3, sigma, dtype), rand((H_kv, rows, d), seed + 4, sigma, dtype)
        first = rows // 2 + 1 if rows > 1 else rows
        K, V = (torch.full((H_kv, rows + 12, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        at = 4 + rows - first + 3  # where the first piece lies, behind the second
        for dst, src in ((K, Kl), (V, Vl)):
            dst[:, at:at + first] = src[:, :first]
            dst[:, 4:4 + rows - first] = src[:, first:]
        seg = dict(seg_logical_off=[0, first, rows], seg_phys_off=[at, 4])
        Kw, Vw = f64(Kl), f64(Vl)
    O = torch.full((H_q, rows, d), 9.0, dtype=dtype, device="cuda")
    lse = torch.full((H_q, rows + 5), 9.0, device="cuda")
    status = status_word()
    ids = i32(list(active) + [-1] * (len(lens) - len(active)))
    ctx.chunk_attention_kv4(Q, cache, K, V, off, vis, ids, i32([len(active)]), O, lse=lse, n_cache=n_cache, impl=impl, status=status,
                            scale=scale, **seg)
    want = pf.attention(f64(Q), np.concatenate([Kc, Kw], 1), np.concatenate([Vc, Vw], 1), off, vis, active, scale)
    assert int(status) == 0
    on = np.concatenate([np.arange(off[c], off[c + 1]) for c in active] or [np.zeros(0, np.int64)]).astype(int)
    stay = np.setdiff1d(np.arange(rows), on)
    assert (f64(O)[:, stay] == 9).all() and (f64(lse)[:, stay] == 9).all() and (f64(lse)[:, rows:] == 9).all()
    check_attention(O, lse[:, :rows], *want, dtype, dtype == BF16 and impl != 1, max(vis + [1]), d, on)


CASES = [
    dict(H_q=1, H_kv=1, lens=[1], n_cache=1, win=False, active=[0]),
    dict(H_q=3, H_kv=3, lens=[1], n_cache=5000, win=True, active=[0]),
    dict(H_q=4, H_kv=1, lens=[1], n_cache=777, win=False, active=[0]),
    dict(H_q=6, H_kv=2, lens=[5], n_cache=33, win=True, active=[0]),
    dict(H_q=2, H_kv=2, lens=[17, 0, 40, 3], n_cache=129, win=True, active=[0, 1, 3]),
    dict(H_q=8, H_kv=2, lens=[50], n_cache=2500, win=True, active=[0]),
    dict(H_q=2, H_kv=1, lens=[130, 257], n_cache=255, win=True, active=[1]),
    dict(H_q=2, H_kv=2, lens=[300, 31, 200], n_cache=1000, win=True, active=[0, 2]),
    dict(H_q=2, H_kv=2, lens=[64, 64], n_cache=0, win=True, active=[0, 1]),
    dict(H_q=2, H_kv=2, lens=[20, 20, 20], n_cache=100, win=True, active=[]),
    dict(H_q=8, H_kv=2, lens=[97, 130, 33], n_cache=1500, win=True, active=[0, 2]),
    dict(H_q=6, H_kv=2, lens=[150, 10], n_cache=900, win=True, active=[0, 1]),
    dict(H_q=16, H_kv=1, lens=[70], n_cache=2000, win=False, active=[0]),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype, impl", [(BF16, 0), (BF16, 1), (BF16, 2), (BF16, 3), (F32, 0), (F32, 1)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c["lens"])) + f"@{c['n_cache']}")
def test_attention(fc, ctx, case, dtype, impl, d):
    run_attention(fc, ctx, d=d, dtype=dtype, impl=impl, **case)


@pytest.mark.parametrize("dtype, impl", [(BF16, 0), (BF16, 1), (BF16, 2), (BF16, 3), (F32, 0), (F32, 1)])
def test_attention_visible_lengths(fc, ctx, dtype, impl):
    # nothing visible, one token, inside the clean region, at its end, inside the window, at a tile's edge
    for cut in ([0, 1, 100], [128, 129, 300], [299, 301, 333], [0, 0, 0]):
        run_attention(fc, ctx, H_q=2, H_kv=2, d=128, lens=[20, 7, 33], n_cache=300, win=True, active=[0, 1, 2], cut=cut, dtype=dtype, impl=impl)
    # few rows and many keys, of which a part sees few
    run_attention(fc, ctx, H_q=2, H_kv=2, d=64, lens=[2, 2], n_cache=9000, win=False, active=[0, 1], cut=[3, 9000], dtype=dtype, impl=impl)


@pytest.mark.parametrize("case", [
    dict(H_q=40, H_kv=40, lens=[1000], n_cache=1500, win=True, active=[0]),           # 160 items: 12 are cut where 148 fill a round
    dict(H_q=80, H_kv=20, lens=[520, 30], n_cache=1300, win=True, active=[0, 1]),      # 200: the cut ones belong to both chunks
    dict(H_q=3, H_kv=3, lens=[2600, 2600], n_cache=900, win=True, active=[1]),         # 33: every item is cut
    dict(H_q=20, H_kv=20, lens=[256 * 7, 256], n_cache=1100, win=False, active=[0, 1]),  # 160, whole tiles only
], ids=lambda c: f"{c['H_q']}-{c['H_kv']}")
def test_attention_items_cut_into_parts(fc, ctx, case):
    run_attention(fc, ctx, d=64, dtype=BF16, impl=2, **case)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", [
    dict(H_q=12, H_kv=12, lens=[190, 251], n_cache=700, win=True, active=[0, 1]),
    dict(H_q=16, H_kv=4, lens=[251, 3, 130], n_cache=777, win=True, active=[0, 2]),
    dict(H_q=24, H_kv=24, lens=[257, 9, 120], n_cache=0, win=True, active=[0, 1, 2]),
    dict(H_q=24, H_kv=24, lens=[257, 40, 250], n_cache=333, win=True, active=[0, 1, 2], cut=[1, 0, 880]),
    dict(H_q=8, H_kv=8, lens=[300, 300, 300], n_cache=4001, win=True, active=[0, 2]),  # at d = 128 also in two parts
], ids=lambda c: "-".join(map(str, c["lens"])) + f"@{c['n_cache']}")
def test_attention_fp32_of_many_rows(fc, ctx, case, d):
    # enough rows that sixteen, not eight, go into a tile
    run_attention(fc, ctx, d=d, dtype=F32, **case)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_fp32_window_products(fc, ctx, d):
    """The six products that are taken of an fp32 weight w and a value v of the window miss at most 2^-24 |w v|: rounding to eight
    bits leaves at most 2^-8 of a number and then 2^-17, so that each of the two products of second and third parts is below 2^-25.

    Every row sees two keys: one of weight 1 and value 0, and one of weight w = (1 + x) / 2 whose values are 1 and numbers with
    large lower parts.  Its output is w v / (1 + w), and its ratio to the one where v is 1 is v.  In units of 2^-24 of it that is off by the
    missing products (1), what the tensor core cuts off the sum and off its smaller addend (2 each; the sums before the last are
    2^-7 of it), and the rounding of the product with the reciprocal (1, in both); w itself is the sum of its parts exactly."""
    g = torch.Generator().manual_seed(d)
    rows = 400
    x = torch.rand(rows, generator=g, dtype=torch.float64) * 2.0 ** -7
    Q, K, V = torch.zeros((1, rows, d)), torch.zeros((1, 2, d)), torch.zeros((1, 2, d))
    Q[0, :, 0] = torch.log((1 + x) / 2).float()
    K[0, 1, 0] = 1.0
    V[0, 1] = 1 + torch.randint(0, 2 ** 16, (d,), generator=g).float() * 2.0 ** -23
    V[0, 1, 0] = 1.0
    Q, K, V = (t.cuda() for t in (Q, K, V))
    O = torch.zeros_like(Q)
    ctx.chunk_attention_kv4(Q, None, K, V, [0, rows], [2], i32([0]), i32([1]), O, scale=1.0, n_cache=0)
    v = f64(V)[0, 1]
    units = (f64(O)[0] / f64(O)[0, :, :1] / v - 1) * 2.0 ** 24
    assert np.abs(units).max() <= 7, (units.min(), units.max())


@pytest.mark.parametrize("rows", [3, 700])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_strides_and_broadcast_heads(fc, ctx, dtype, rows):
    # tokens before heads, a slice of a wider row; and one q, one window for all heads (head stride 0), however many the rows
    H, d, n_cache = 4, 64, 300
    cache, Kc, Vc = packed_store(fc, ctx, H, n_cache, d, 3)
    wide = rand((rows, 3 * H, d), 5, 1.0, dtype).transpose(0, 1)
    out = torch.zeros((rows, 2, H, d), dtype=dtype, device="cuda")
    flat = rand((rows, d), 6, 1.0, dtype)
    for Q, K, V in ((wide[:H], wide[H:2 * H], wide[2 * H:]), (flat.expand(H, rows, d), flat.expand(H, rows, d), wide[2 * H:])):
        O = out[:, 1].transpose(0, 1)
        ctx.chunk_attention_kv4(Q, cache, K, V, [0, rows], [n_cache + rows], i32([0]), i32([1]), O)
        want = pf.attention(f64(Q), np.concatenate([Kc, f64(K)], 1), np.concatenate([Vc, f64(V)], 1), [0, rows], [n_cache + rows], [0])
        check_attention(O, None, *want, dtype, dtype == BF16, n_cache + rows, d)
    assert (out[:, 0] == 0).all()
    if dtype == BF16:
        with pytest.raises(fc.FcError, match="unsupported"):
            ctx.chunk_attention_kv4(flat.expand(H, rows, d), cache, None, None, [0, rows], [n_cache], i32([0]), i32([1]), O, impl=2)


@pytest.mark.parametrize("dtype, impl", [(BF16, 0), (BF16, 1), (BF16, 2), (BF16, 3), (F32, 0), (F32, 1)])
def test_attention_large_logits_and_scale(fc, ctx, dtype, impl):
    # logits up to hundreds: one key takes nearly all the weight
    run_attention(fc, ctx, H_q=2, H_kv=1, d=64, lens=[40], n_cache=700, win=True, active=[0], sigma=4.0, dtype=dtype, impl=impl)
    run_attention(fc, ctx, H_q=2, H_kv=1, d=64, lens=[3], n_cache=700, win=False, active=[0], scale=0.5, dtype=dtype, impl=impl)


@pytest.mark.parametrize("rows", [2, 200])
def test_attention_nan_query_stays_in_its_row(fc, ctx, rows):
    cache, _, _ = packed_store(fc, ctx, 2, 400, 64, 3)
    for dtype in (BF16, F32):
        Q = rand((2, rows, 64), 4, 1.0, dtype)
        Q[1, 1, 3] = float("nan")
        O = torch.zeros_like(Q)
        ctx.chunk_attention_kv4(Q, cache, None, None, [0, rows], [400], i32([0]), i32([1]), O)
        bad = torch.isnan(O)
        assert bad[1, 1].all() and int(bad.sum()) == 64


@pytest.mark.parametrize("dtype, impl", [(BF16, 0), (BF16, 1), (BF16, 2), (BF16, 3), (F32, 0), (F32, 1)])
@pytest.mark.parametrize("rows, n", [(2, 400), (200, 400), (200, 3000)])
def test_attention_log_sum_of_a_nan_row(fc, ctx, rows, n, dtype, impl):
    # -inf says that a row saw no token; a row whose logits are NaN saw some
    cache, _, _ = packed_store(fc, ctx, 2, n, 64, 3)
    Q = rand((2, rows, 64), 4, 1.0, dtype)
    Q[1, 1, 3] = float("nan")
    O, lse = torch.zeros_like(Q), torch.zeros((2, rows), device="cuda")
    ctx.chunk_attention_kv4(Q, cache, None, None, [0, rows], [n], i32([0]), i32([1]), O, lse=lse, impl=impl)
    bad = torch.isnan(lse)
    assert bad[1, 1] and int(bad.sum()) == 1 and torch.isnan(O[1, 1]).all()


@pytest.mark.parametrize("dtype, impl", [(BF16, 1), (BF16, 2), (BF16, 3), (F32, 0)])
def test_attention_many_chunks(fc, ctx, dtype, impl):
    # as many chunks as there may be, most of them short; half active, one of them named twice
    lens = [(7 * c) % 11 for c in range(64)]
    ids = list(range(0, 64, 2))
    cache, Kc, Vc = packed_store(fc, ctx, 2, 70, 64, 3)
    off = [0] + list(np.cumsum(lens))
    Q = rand((4, off[-1], 64), 4, 1.0, dtype)
    K, V = rand((2, off[-1], 64), 5, 1.0, dtype), rand((2, off[-1], 64), 6, 1.0, dtype)
    vis = [70 + o for o in off[1:]]
    O = torch.full_like(Q, 9.0)
    # the window in 63 pieces, one after the other
    cuts = off[:63] + [off[-1]]
    ctx.chunk_attention_kv4(Q, cache, K, V, off, vis, i32(ids + [ids[5]]), i32([len(ids) + 1]), O, impl=impl,
                            seg_logical_off=cuts, seg_phys_off=cuts[:-1])
    want = pf.attention(f64(Q), np.concatenate([Kc, f64(K)], 1), np.concatenate([Vc, f64(V)], 1), off, vis, ids)
    rows = np.concatenate([np.arange(off[c], off[c + 1]) for c in ids]).astype(int)
    check_attention(O, None, *want, dtype, dtype == BF16 and impl != 1, vis[-1], 64, rows)
    assert (f64(O)[:, np.setdiff1d(np.arange(off[-1]), rows)] == 9).all()


@pytest.mark.parametrize("dtype, impl", [(BF16, 0), (BF16, 1), (BF16, 2), (BF16, 3), (F32, 0)])
def test_attention_chunk_named_more_than_once(fc, ctx, dtype, impl):
    # 40 work items of 256 rows, 50 if the chunk that is named twice counted twice; 32 key tiles, so that items are cut into parts
    run_attention(fc, ctx, H_q=10, H_kv=10, d=64, lens=[512, 256, 1], n_cache=4096, win=False, active=[0, 0, 1], cut=[4096, 4000, 4000],
                  dtype=dtype, impl=impl)
    # the copies behind what they hide, and every entry the same
    run_attention(fc, ctx, H_q=4, H_kv=2, d=64, lens=[300, 20, 40], n_cache=1000, win=True, active=[1, 2, 1], dtype=dtype, impl=impl)
    run_attention(fc, ctx, H_q=4, H_kv=2, d=64, lens=[300, 20, 40], n_cache=1000, win=True, active=[2, 2, 2], dtype=dtype, impl=impl)


@pytest.mark.parametrize("dtype, impl", [(BF16, 0), (BF16, 1), (BF16, 2), (BF16, 3), (F32, 0)])
@pytest.mark.parametrize("lens, n_cache", [([1], 3000), ([3, 9], 700), ([300, 130], 1500), ([40, 0, 17], 0)])
def test_attention_rows_before_and_behind_the_chunks_stay(fc, ctx, lens, n_cache, dtype, impl):
    # the chunks are rows 5 .. of Q and O, with NaN queries around them
    H_q, H_kv, d, first, behind = 4, 2, 64, 5, 300
    off = [first] + [first + int(x) for x in np.cumsum(lens)]
    rows = off[-1] + behind
    cache, Kc, Vc = packed_store(fc, ctx, H_kv, n_cache, d, 3) if n_cache else (None, np.zeros((H_kv, 0, d)), np.zeros((H_kv, 0, d)))
    Q, K, V = rand((H_q, rows, d), 4, 1.0, dtype), rand((H_kv, 90, d), 5, 1.0, dtype), rand((H_kv, 90, d), 6, 1.0, dtype)
    Q[:, :first], Q[:, off[-1]:] = float("nan"), float("nan")
    O, lse = torch.full_like(Q, 9.0), torch.full((H_q, rows), 9.0, device="cuda")
    vis = [n_cache + 90 - c for c in range(len(lens))]
    ids = list(range(len(lens)))
    ctx.chunk_attention_kv4(Q, cache, K, V, off, vis, i32(ids), i32([len(ids)]), O, lse=lse, impl=impl)
    want = pf.attention(f64(Q), np.concatenate([Kc, f64(K)], 1), np.concatenate([Vc, f64(V)], 1), off, vis, ids)
    check_attention(O, lse, *want, dtype, dtype == BF16 and impl != 1, vis[0], d, slice(first, off[-1]))
    for t in (O, lse):
        assert (t[:, :first] == 9).all() and (t[:, off[-1]:] == 9).all()


def test_attention_bad_ids_are_reported(fc, ctx):
    for dtype, rows in ((BF16, 3), (BF16, 400), (F32, 3)):
        cache, Kc, Vc = packed_store(fc, ctx, 1, 90, 64, 3)
        Q = rand((1, 2 * rows, 64), 4, 1.0, dtype)
        O, status = torch.full_like(Q, 9.0), status_word()
        off = [0, rows, 2 * rows]
        ctx.chunk_attention_kv4(Q, cache, None, None, off, [90, 90], i32([7, 1]), i32([2]), O, status=status)
        assert int(status) == fc.STATUS_BITS["bad_index"]
        want = pf.attention(f64(Q), Kc, Vc, off, [90, 90], [1])
        check_attention(O, None, *want, dtype, dtype == BF16, 90, 64, slice(rows, None))
        assert (O[:, :rows] == 9).all()


def test_attention_is_reproducible(fc, ctx):
    cache, _, _ = packed_store(fc, ctx, 3, 6000, 128, 3)
    for rows in (1, 300):
        Q = rand((3, rows, 128), 4)
        outs = []
        for _ in range(3):
            O = torch.zeros_like(Q)
            ctx.chunk_attention_kv4(Q, cache, None, None, [0, rows], [6000], i32([0]), i32([1]), O)
            outs.append(O)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


# ------------------------------------------------------------------------------------ streams, graphs, refusals, together

def test_streams_and_captured_graphs_do_not_share_scratch(fc, ctx):
    # two graphs of the same call, captured one after the other on the same stream, replayed at once on two streams
    H, n, d = 4, 6000, 128
    cache, Kc, Vc = packed_store(fc, ctx, H, n, d, 3)
    for rows in (1, 200):
        ids, one = i32([0]), i32([1])
        Qs = [rand((H, rows, d), 10 + k) for k in range(2)]
        Os = [torch.zeros_like(q) for q in Qs]
        want = []
        for q in Qs:
            o = torch.zeros_like(q)
            ctx.chunk_attention_kv4(q, cache, None, None, [0, rows], [n], ids, one, o)
            want.append(o)
        graphs = []
        for q, o in zip(Qs, Os):
            g = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(g):
                ctx.chunk_attention_kv4(q, cache, None, None, [0, rows], [n], ids, one, o)
            graphs.append(g)
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for _ in range(20):
            for s, g in zip(streams, graphs):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        assert torch.equal(Os[0], want[0]) and torch.equal(Os[1], want[1])
        # eager calls on two streams at once
        for o in Os:
            o.zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            for s, q, o in zip(streams, Qs, Os):
                with torch.cuda.stream(s):
                    ctx.chunk_attention_kv4(q, cache, None, None, [0, rows], [n], ids, one, o)
        torch.cuda.synchronize()
        assert torch.equal(Os[0], want[0]) and torch.equal(Os[1], want[1])


def test_binding_refusals(fc, ctx):
    K = rand((2, 8, 64), 1)
    cache = fc.Kv4Cache.empty(2, 8, 64)
    ids, one = i32([0]), i32([1])
    with pytest.raises(fc.FcError, match="must be on cuda"):
        ctx.qk_norm_rope(K.cpu(), None, axes=(24, 20, 20), grid=(0, 2, 4))
    with pytest.raises(fc.FcError, match="places"):
        ctx.qk_norm_rope(K, None, axes=(24, 20, 20))
    with pytest.raises(fc.FcError, match="contiguous last dimension"):
        ctx.qk_norm_rope(K.transpose(1, 2), None, axes=(0, 0, 0))
    with pytest.raises(fc.FcError, match="pos"):
        ctx.qk_norm_rope(K, None, axes=(24, 20, 20), pos=i32([[0, 0, 0]]))
    with pytest.raises(fc.FcError, match="weight"):
        ctx.qk_norm_rope(K, None, axes=(0, 0, 0), q_weight=torch.ones(32, device="cuda"))
    with pytest.raises(fc.FcError, match="invalid argument"):
        ctx.qk_norm_rope(K, None, axes=(25, 20, 19), grid=(0, 2, 4))
    with pytest.raises(fc.FcError, match="V must be"):
        ctx.kv4_pack(K, K[:, :4], cache)
    with pytest.raises(fc.FcError, match="invalid argument"):
        ctx.kv4_pack(K, K, cache, dst_row=1)
    with pytest.raises(fc.FcError, match="share strides"):
        fc.Kv4Cache(cache.k_codes, cache.k_scales, cache.v_codes, torch.empty((2, 16, 2), dtype=BF16, device="cuda")[:, ::2])
    with pytest.raises(fc.FcError, match="codes must be"):
        fc.Kv4Cache(cache.k_codes, cache.k_scales, cache.v_codes[:, :4], cache.v_scales)
    with pytest.raises(fc.FcError, match="invalid argument"):
        ctx.kv4_unpack(cache, row=4, n=5)
    O = torch.zeros_like(K)
    with pytest.raises(fc.FcError, match="invalid argument"):
        ctx.chunk_attention_kv4(K, cache, None, None, [0, 8], [9], ids, one, O)
    with pytest.raises(fc.FcError, match="K must be"):
        ctx.chunk_attention_kv4(K, cache, K.float(), K.float(), [0, 8], [9], ids, one, O)
    with pytest.raises(fc.FcError, match="store, a window"):
        ctx.chunk_attention_kv4(K, None, None, None, [0, 8], [0], ids, one, O)
    with pytest.raises(fc.FcError, match="contiguous"):
        ctx.chunk_attention_kv4(K, cache, None, None, [0, 4, 8], [8, 8], i32([0, 1, 1, 0])[::2], one, O)
    with pytest.raises(fc.FcError, match="inside Q"):
        ctx.chunk_attention_kv4(K, cache, None, None, [0, 9], [8], ids, one, O)
    with pytest.raises(fc.FcError, match="workspace"):
        big = fc.Kv4Cache.empty(2, 9000, 64)
        ctx.chunk_attention_kv4(K[:, :1], big, None, None, [0, 1], [9000], ids, one, O[:, :1], ws=torch.empty(16, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_generation_step_over_a_packed_clean_region(fc, ctx, dtype):
    """A chunk's whole path: project (given), norm and rotate into the window, attend over [packed clean region | window], score
    the unpacked keys and the chunk's, select, and pack the next clean region; three chunks, checked at every step."""
    H, d, n_c, B, axes = 2, 64, 48, 96, (24, 20, 20)
    wk = rand((d,), 6, 0.2, F32) + 1
    cache, n_clean = fc.Kv4Cache.empty(H, B, d), 0
    for chunk in range(4):
        qkv = rand((n_c, 3 * H, d), 50 + chunk, 1.0, dtype).transpose(0, 1)
        Q, K = ctx.qk_norm_rope(qkv[:H], qkv[H:2 * H], axes=axes, grid=(2 * chunk, 4, 6), q_weight=wk, k_weight=wk)
        pos = pf.grid_positions(n_c, 2 * chunk, 4, 6)
        check_turned(K, qkv[H:2 * H], dtype, pos=pos, axes=axes, weight=f64(wk))
        V = qkv[2 * H:].contiguous()
        # attention of the chunk over what is kept and itself
        Kc, Vc = (f64(x) for x in ctx.kv4_unpack(cache, n=n_clean, dtype=F32))
        O = torch.zeros((H, n_c, d), dtype=dtype, device="cuda")
        ctx.chunk_attention_kv4(Q, cache, K, V, [0, n_c], [n_clean + n_c], i32([0]), i32([1]), O, n_cache=n_clean)
        want = pf.attention(f64(Q), np.concatenate([Kc, f64(K)], 1), np.concatenate([Vc, f64(V)], 1), [0, n_c], [n_clean + n_c], [0])
        check_attention(O, None, *want, dtype, dtype == BF16, n_clean + n_c, d)
        # the next clean region: score keys as they are held, keep the best B
        cand = torch.empty((H, n_clean + n_c, d), dtype=dtype, device="cuda")
        ctx.kv4_unpack(cache, n=n_clean, K_dst=cand[:, :n_clean], keys_only=True)
        cand[:, n_clean:] = K
        score = ctx.kv_score(Q[:, -8:].contiguous(), cand, lambda_=0.07, pool_k=7)["score"]
        kept = ctx.kv_select_compact(score, B)["kept_idx"]
        n_keep = kept.shape[1]
        new = fc.Kv4Cache.empty(H, B, d)
        ctx.kv4_pack(K, V, new, old=cache if n_clean else None, n_old=n_clean, kept_idx=kept)
        got = [f64(x) for x in ctx.kv4_unpack(new, n=n_keep, dtype=F32)]
        at = kept.long().cpu().numpy()[..., None]
        for g, old, x in zip(got, (Kc, Vc), (K, V)):
            assert np.array_equal(g, np.take_along_axis(np.concatenate([old, pf.quantise(f64(x))[2]], 1), at, 1))
        cache, n_clean = new, n_keep
    assert n_clean == B
