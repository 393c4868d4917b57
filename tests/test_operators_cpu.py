"""The calls around the 4-bit store, as far as they go without a GPU: what they refuse, what they answer for nothing to do, and
workspace sizes.  Every check is made before the first CUDA call, so a stand-in for the context and addresses
that nobody follows are enough."""
import ctypes as C
import struct

import numpy as np
import pytest

import paper_2602_10825_b200 as fc
from paper_2602_10825_b200 import binding as b
from paper_2602_10825_b200 import build as fc_build
import plain_forms as pf

INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = -1, -2, -3, -4
P = 0x7000_0000  # an address that is aligned; no call of this file gets as far as to use it


@pytest.fixture(scope="module")
def L():
    fc_build.build()
    return fc.lib()


@pytest.fixture(scope="module")
def ctx():
    # fc_ctx: device, SM count, shared memory limit, driver entry point
    buf = C.create_string_buffer(struct.pack("iii4xP", 0, 148, 232448, 0), 64)
    return C.cast(buf, C.c_void_p), buf


def store(**kw):
    f = dict(k_codes=P, k_scales=P, v_codes=P, v_scales=P, code_hs=64 * 100, code_rs=64, scale_hs=4 * 100, scale_rs=4, rows=100)
    f.update(kw)
    return b._Kv4Cache(**f)


# ------------------------------------------------------------------------------------ fc_qk_norm_rope

def rope(L, ctx, *, Q=P, K=P, Qo=P, Ko=P, dtype=b.BF16, wq=None, wk=None, pos=None, freq=None, **kw):
    f = dict(H_q=4, H_kv=2, d=128, T=10, q_hs=1280, q_rs=128, k_hs=1280, k_rs=128, qo_hs=1280, qo_rs=128, ko_hs=1280, ko_rs=128,
             axis_dim=(44, 42, 42), pairing=0, norm=1, eps=1e-6, theta=1e4, grid_t0=0, grid_h=2, grid_w=5)
    f.update(kw)
    f["axis_dim"] = (C.c_int32 * 3)(*f["axis_dim"])
    desc = b._RopeDesc(**f)
    arr = None if freq is None else np.asarray(freq, np.float64)
    return L.fc_qk_norm_rope(ctx[0], None, C.byref(desc), Q, K, dtype, wq, wk, pos, None if arr is None else arr.ctypes.data, Qo, Ko)


@pytest.mark.parametrize("kw, want", [
    (dict(dtype=7), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(T=-1), INVALID), (dict(H_q=-1), INVALID),
    (dict(Q=None), INVALID), (dict(Ko=None), INVALID), (dict(pairing=2), INVALID), (dict(norm=2), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(axis_dim=(43, 42, 42)), INVALID),
    (dict(axis_dim=(-2, 42, 42)), INVALID), (dict(axis_dim=(64, 64, 2)), INVALID), (dict(theta=0.0), INVALID),
    (dict(theta=float("inf")), INVALID), (dict(grid_h=0), INVALID), (dict(grid_w=-3), INVALID),
    (dict(grid_h=1 << 20, grid_w=1 << 20), INVALID), (dict(grid_t0=2 ** 31 - 1, grid_h=1, grid_w=1), INVALID),
    (dict(freq=[float("nan")] * 64), INVALID), (dict(Q=P + 8), MISALIGNED), (dict(q_hs=4), MISALIGNED), (dict(ko_rs=-8), MISALIGNED),
    (dict(qo_hs=64), INVALID), (dict(ko_rs=0), INVALID),
])
def test_rope_refusals(L, ctx, kw, want):
    assert rope(L, ctx, **kw) == want


def test_rope_nothing_to_do(L, ctx):
    assert rope(L, ctx, T=0, Q=None, K=None, Qo=None, Ko=None) == 0
    assert rope(L, ctx, H_q=0, H_kv=0, Q=None, K=None, Qo=None, Ko=None) == 0


def test_rope_of_no_tokens_asks_for_no_places(L, ctx):
    # an empty tensor of places has the address 0
    assert rope(L, ctx, T=0, pos=None, grid_h=0, grid_w=0) == 0


# ------------------------------------------------------------------------------------ fc_kv4_pack / unpack

def pack(L, ctx, *, K=P, V=P, dtype=b.BF16, old=None, kept=None, kept_hs=0, dst=True, **kw):
    f = dict(H=2, d=128, n_old=0, n_new=10, n_out=10, dst_row=0, k_hs=1280, k_rs=128, v_hs=1280, v_rs=128)
    f.update(kw)
    desc = b._Kv4PackDesc(**f)
    dst = store() if dst is True else dst
    return L.fc_kv4_pack(ctx[0], None, C.byref(desc), K, V, dtype, None if old is None else C.byref(old), kept, kept_hs,
                         None if dst is None else C.byref(dst), None)


@pytest.mark.parametrize("kw, want", [
    (dict(dtype=3), UNSUPPORTED), (dict(d=32), UNSUPPORTED), (dict(H=0), INVALID), (dict(H=70000), UNSUPPORTED),
    (dict(n_new=-1), INVALID), (dict(dst_row=-1), INVALID), (dict(n_old=2 ** 31 - 5, n_new=10), INVALID), (dict(K=None), INVALID),
    (dict(n_out=11), INVALID), (dict(kept=P, kept_hs=9), INVALID), (dict(k_rs=64), INVALID), (dict(k_hs=4), MISALIGNED),
    (dict(V=P + 2), MISALIGNED), (dict(n_old=5, n_out=15), INVALID), (dict(n_old=5, n_out=15, old=store(rows=4)), INVALID),
    (dict(dst=None), INVALID), (dict(dst=store(rows=9)), INVALID), (dict(dst_row=91), INVALID), (dict(dst_row=2 ** 63 - 5), INVALID),
    (dict(dst=store(k_codes=P + 4)), MISALIGNED), (dict(dst=store(code_rs=72)), MISALIGNED), (dict(dst=store(code_rs=48)), INVALID),
    (dict(dst=store(scale_rs=6)), MISALIGNED), (dict(dst=store(scale_rs=0)), INVALID), (dict(dst=store(v_scales=None)), INVALID),
    (dict(dst=store(k_scales=P + 4)), MISALIGNED), (dict(dst=store(code_hs=0)), INVALID), (dict(dst=store(scale_hs=0)), INVALID),
])
def test_pack_refusals(L, ctx, kw, want):
    assert pack(L, ctx, **kw) == want


def slice_of(row, rows_first=False, base=P, **kw):
    """Rows from `row` on of a store of two heads of 200 rows of 128, heads before rows or rows before heads."""
    c, s = ((64, 128), (4, 8)) if rows_first else ((64 * 200, 64), (4 * 200, 4))
    at = lambda n, rs: base + n * 0x10_0000 + row * rs  # noqa: E731
    f = dict(k_codes=at(0, c[1]), v_codes=at(1, c[1]), k_scales=at(2, 2 * s[1]), v_scales=at(3, 2 * s[1]), code_hs=c[0], code_rs=c[1],
             scale_hs=s[0], scale_rs=s[1], rows=200 - row)
    f.update(kw)
    return b._Kv4Cache(**f)


@pytest.mark.parametrize("rows_first", [False, True])
@pytest.mark.parametrize("old, dst, dst_row", [(0, 0, 39), (0, 8, 0), (8, 0, 0), (8, 0, 47), (0, 30, 9), (100, 61, 0), (3, 3, 0)])
def test_pack_refuses_slices_that_share_rows(L, ctx, old, dst, dst_row, rows_first):
    kw = dict(n_old=40, n_new=0, n_out=40, K=None, V=None)
    # the slices overlap by at least one row in every case
    assert old < dst + dst_row + 40 and dst + dst_row < old + 40
    assert pack(L, ctx, old=slice_of(old, rows_first), dst=slice_of(dst, rows_first), dst_row=dst_row, **kw) == INVALID


def test_pack_refuses_stores_that_share_some_memory(L, ctx):
    kw = dict(n_old=40, n_new=0, n_out=40, K=None, V=None)
    far = slice_of(0, base=P + 0x100_0000)
    old = slice_of(0)
    for own in ("k_codes", "v_codes", "k_scales", "v_scales"):  # one tensor of the two stores is the same, or K of one is V of the other
        for other in ("k" + own[1:], "v" + own[1:]):
            shared = {**{n: getattr(far, n) for n in ("k_codes", "v_codes", "k_scales", "v_scales")}, own: getattr(old, other)}
            assert pack(L, ctx, old=old, dst=slice_of(0, **shared), **kw) == INVALID
    # heads of one store between the heads of another, with other strides
    assert pack(L, ctx, old=old, dst=slice_of(100, code_hs=64 * 150, rows=100), **kw) == INVALID


def unpack(L, ctx, *, K=P, V=P, dtype=b.BF16, src=True, **kw):
    f = dict(H=2, d=128, n=10, src_row=0, k_hs=1280, k_rs=128, v_hs=1280, v_rs=128)
    f.update(kw)
    desc = b._Kv4UnpackDesc(**f)
    src = store() if src is True else src
    return L.fc_kv4_unpack(ctx[0], None, C.byref(desc), None if src is None else C.byref(src), K, V, dtype)


@pytest.mark.parametrize("kw, want", [
    (dict(dtype=3), UNSUPPORTED), (dict(d=256), UNSUPPORTED), (dict(n=-1), INVALID), (dict(src_row=-1), INVALID),
    (dict(K=None, V=None), INVALID), (dict(src=None), INVALID), (dict(n=101), INVALID), (dict(src_row=91), INVALID),
    (dict(k_rs=120), INVALID), (dict(v_rs=132), MISALIGNED), (dict(K=P + 1), MISALIGNED), (dict(v_hs=0), INVALID),
])
def test_unpack_refusals(L, ctx, kw, want):
    assert unpack(L, ctx, **kw) == want


def test_pack_and_unpack_nothing_to_do(L, ctx):
    assert pack(L, ctx, n_new=0, n_out=0, K=None, V=None, dst=None) == 0
    assert unpack(L, ctx, n=0, K=None, V=None, src=None) == 0


# ------------------------------------------------------------------------------------ fc_chunk_attention_kv4

def attn(L, ctx, *, Q=P, K=P, V=P, O=P, dtype=b.BF16, cache=True, n_cache=100, off=(0, 5, 10), vis=(105, 110), seg=((0, 10), (0,)),
         ids=P, n_active=P, lse=None, lse_hs=0, ws=None, ws_bytes=0, **kw):
    f = dict(H_q=4, H_kv=2, d=128, W=2, q_hs=1280, q_rs=128, k_hs=1280, k_rs=128, v_hs=1280, v_rs=128, o_hs=1280, o_rs=128, kv_rows=10,
             scale=0.0, impl=0)
    f.update(kw)
    desc = b._AttnDesc(**f)
    arr = lambda x: None if x is None else (C.c_int32 * len(x))(*x)  # noqa: E731
    cache = store() if cache is True else cache
    sl, sp = seg if seg else (None, None)
    return L.fc_chunk_attention_kv4(ctx[0], None, C.byref(desc), Q, None if cache is None else C.byref(cache), n_cache, K, V, dtype,
                                    arr(off), arr(vis), arr(sl), arr(sp), len(sp) if sp else 0, ids, n_active, O, lse, lse_hs, None,
                                    ws, ws_bytes)


@pytest.mark.parametrize("kw, want", [
    (dict(dtype=2), UNSUPPORTED), (dict(d=80), UNSUPPORTED), (dict(H_q=3), INVALID), (dict(W=0), INVALID), (dict(W=65), UNSUPPORTED),
    (dict(impl=-1), INVALID), (dict(impl=9), INVALID), (dict(impl=2, dtype=b.F32), UNSUPPORTED), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(off=(0, 5, 4)), INVALID), (dict(off=(-1, 5, 10)), INVALID), (dict(vis=(105, 111)), INVALID), (dict(vis=(-1, 110)), INVALID),
    (dict(n_cache=-1), INVALID), (dict(cache=None), INVALID), (dict(cache=store(rows=99)), INVALID), (dict(Q=None), INVALID),
    (dict(ids=None), INVALID), (dict(K=None), INVALID), (dict(Q=P + 8), MISALIGNED), (dict(q_hs=4), MISALIGNED), (dict(o_rs=64), INVALID),
    (dict(k_rs=100), MISALIGNED), (dict(kv_rows=9), INVALID), (dict(seg=((1, 10), (0,))), INVALID), (dict(seg=((0, 10), (-1,))), INVALID),
    (dict(seg=(tuple(range(65)), tuple(range(64)))), UNSUPPORTED), (dict(seg=None), INVALID), (dict(lse=P, lse_hs=0), INVALID),
    (dict(cache=store(k_codes=P + 8)), MISALIGNED), (dict(o_hs=0), INVALID), (dict(impl=2, q_hs=0), UNSUPPORTED),
])
def test_attention_refusals(L, ctx, kw, want):
    assert attn(L, ctx, **kw) == want


def test_attention_refuses_offsets_that_pass_32_bits(L, ctx):
    n = 2 ** 31 - 4097
    assert attn(L, ctx, n_cache=n, cache=store(rows=n), ws=None) == UNSUPPORTED  # and ten tokens of a window behind them


def test_a_store_keeps_its_tensors():
    torch = pytest.importorskip("torch")
    s = fc.Kv4Cache.empty(2, 5, 64, device="cpu")
    assert s.k_codes.shape == (2, 5, 32) and s.v_scales.shape == (2, 5, 2) and (s.H, s.rows, s.d) == (2, 5, 64)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        with pytest.raises(AttributeError):
            setattr(s, name, torch.zeros_like(getattr(s, name)))


def test_attention_no_rows_and_workspace(L, ctx):
    assert attn(L, ctx, off=(3, 3, 3), Q=None, O=None, ids=None, n_active=None) == 0
    desc = b._AttnDesc(H_q=4, H_kv=2, d=128, W=1)
    arr = lambda *x: (C.c_int32 * len(x))(*x)  # noqa: E731
    size = lambda rows, vis, n_cache, dt=b.BF16: L.fc_chunk_attention_kv4_workspace_bytes(  # noqa: E731
        ctx[0], C.byref(desc), dt, arr(0, rows), arr(vis), n_cache)
    assert size(1, 20000, 20000) > 0
    assert size(-1, 20000, 20000) == 0 and size(1, 20000, 20000, 5) == 0
    assert L.fc_chunk_attention_kv4_workspace_bytes(ctx[0], None, 0, arr(0, 1), arr(5), 5) == 0
    # a workspace one byte short is refused
    need = size(1, 20000, 20000)
    kw = dict(W=1, off=(0, 1), vis=(20000,), n_cache=20000, cache=store(rows=20000), seg=None, ws=P)
    assert attn(L, ctx, ws_bytes=need - 1, **kw) == WORKSPACE
    assert attn(L, ctx, ws_bytes=need, **{**kw, "ws": None}) == WORKSPACE
    assert attn(L, ctx, ws_bytes=need, **{**kw, "ws": P + 8}) == MISALIGNED


def test_packed_descriptors_are_the_structures():
    for fields, cls in ((b._ROPE_FIELDS, b._RopeDesc), (b._PACK_FIELDS, b._Kv4PackDesc), (b._UNPACK_FIELDS, b._Kv4UnpackDesc),
                        (b._ATTN_FIELDS, b._AttnDesc), (b._CACHE_FIELDS, b._Kv4Cache)):
        n = len(fields.unpack(bytes(fields.size)))
        raw = fields.pack(*range(1, n + 1)).ljust(C.sizeof(cls), b"\0")
        got = cls.from_buffer_copy(raw)
        values = [getattr(got, name) for name, _ in cls._fields_]
        flat = [x for v in values for x in (list(v) if hasattr(v, "__len__") else [v])]
        assert flat == list(range(1, n + 1))


# ------------------------------------------------------------------------------------ the plain forms themselves

def test_plain_format_by_hand():
    x = np.zeros(32)
    x[:4] = [7.0, -7.0, 2.5, 1.5]  # largest 7: scale 1; 2.5 and 1.5 are ties and go to the even 2
    codes, s, v = pf.quantise(x)
    assert s.tolist() == [1.0] and codes[:5].tolist() == [15, 1, 10, 10, 8] and v[:4].tolist() == [7, -7, 2, 2]
    by = pf.code_bytes(codes)
    # word 0: elements 0, 2, 4, 6 in the low half (15, 10, 8, 8), elements 1, 3, 5, 7 in the high half (1, 10, 8, 8)
    assert by[:4].tolist() == [0xAF, 0x88, 0xA1, 0x88] and by[4:].tolist() == [0x88] * 12
    assert np.array_equal(pf.values_of(by, s), v)
    # 7.5 / 7 = 1.0714 needs the next number of five bits, 1.125; the scale never falls below 2^-126 nor is above 2^122
    assert pf.quantise(np.full(32, 7.5))[1].tolist() == [1.125]
    assert pf.scale_of(1e-40) == 2.0 ** -126 and pf.scale_of(3e38) == 2.0 ** 122
    assert pf.quantise(np.zeros(32))[1].tolist() == [0.0] and np.isnan(pf.quantise(np.full(32, np.inf))[1]).all()


def test_plain_rotation_by_hand():
    x = np.zeros((1, 2, 64))
    x[0, :, 0] = 1.0  # pair 0 of axis 0 turns by one radian a position
    y, _ = pf.norm_rope(x, np.asarray([[0, 5, 5], [2, 5, 5]]), (24, 20, 20), norm=False)
    np.testing.assert_allclose(y[0, 0, :2], [1.0, 0.0])
    np.testing.assert_allclose(y[0, 1, :2], [np.cos(2.0), np.sin(2.0)])
    y, _ = pf.norm_rope(x, np.asarray([[0, 5, 5], [2, 5, 5]]), (24, 20, 20), norm=False, halves=True)
    np.testing.assert_allclose([y[0, 1, 0], y[0, 1, 12]], [np.cos(2.0), np.sin(2.0)])
