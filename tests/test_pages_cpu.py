"""The paged 8-bit store, its pages, and attention over it, as far as they go without a GPU: what the calls refuse, what they answer
for nothing to do, workspace sizes, and the format worked by hand.  Every check is made before the first CUDA call, so a stand-in for
the context and addresses that nobody follows are enough."""
import ctypes as C
import math
import struct

import numpy as np
import pytest

import paper_2602_10825_b200 as fc
from paper_2602_10825_b200 import binding as b
from paper_2602_10825_b200 import build as fc_build
import page_forms as pg

INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = -1, -2, -3, -4
P = 0x7000_0000  # an address that is aligned; no call of this file gets as far as to use it


@pytest.fixture(scope="module")
def L():
    fc_build.build()
    return fc.lib()


@pytest.fixture(scope="module")
def ctx():
    # fc_ctx: device, SM count, shared memory limit, driver entry point
    buf = C.create_string_buffer(struct.pack("iii4xP", 0, 148, 232448, 0), 512)
    return C.cast(buf, C.c_void_p), buf


def ints(x):
    return None if x is None else np.asarray(x, np.int32)


def at(a):
    return None if a is None else a.ctypes.data


def pool(**kw):
    f = dict(k_codes=P, v_codes=P, k_scales=P, v_scales=P, code_ps=4 * 64 * 128, code_hs=64 * 128, scale_ps=4, scale_hs=1, n_pages=100, page=64)
    f.update(kw)
    return b._Kv8Pool(**f)


POOL_REFUSALS = [
    (dict(k_codes=None), INVALID), (dict(v_scales=None), INVALID), (dict(n_pages=0), INVALID), (dict(n_pages=2 ** 31 - 8000), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(page=8), UNSUPPORTED),
    (dict(k_codes=P + 8), MISALIGNED), (dict(k_scales=P + 2), MISALIGNED), (dict(code_hs=64 * 128 + 8), MISALIGNED), (dict(code_ps=-16), MISALIGNED),
    (dict(scale_hs=-1), INVALID), (dict(code_hs=64 * 128 - 16), INVALID), (dict(code_ps=3 * 64 * 128), INVALID), (dict(scale_ps=3), INVALID),
    (dict(scale_hs=0), INVALID), (dict(code_ps=1 << 36), UNSUPPORTED), (dict(scale_ps=1 << 31), UNSUPPORTED),
]


# ------------------------------------------------------------------------------------ append, unpack

def rows(L, ctx, call, *, K=P, V=P, dtype=b.BF16, off=(0, 10), first=(5,), pool_=None, table=P, table_cs=9, ref=None, **kw):
    f = dict(H=4, d=128, W=len(first), k_hs=1280, k_rs=128, v_hs=1280, v_rs=128)
    f.update(kw)
    desc, o, p = b._Kv8Rows(**f), ints(off), ints(first)
    s = pool() if pool_ is None else pool_
    if call == "append":
        return L.fc_kv8_append(ctx[0], None, C.byref(desc), K, V, dtype, at(o), at(p), C.byref(s), table, table_cs, ref, None)
    return L.fc_kv8_unpack(ctx[0], None, C.byref(desc), C.byref(s), table, table_cs, at(p), at(o), K, V, dtype, None)


@pytest.mark.parametrize("call", ["append", "unpack"])
@pytest.mark.parametrize("kw, want", [
    (dict(dtype=7), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(H=0), INVALID), (dict(H=70000), UNSUPPORTED), (dict(W=0), INVALID),
    (dict(W=65), UNSUPPORTED), (dict(off=None), INVALID), (dict(first=None, W=1), INVALID), (dict(off=(3, 2)), INVALID), (dict(off=(-1, 2)), INVALID),
    (dict(first=(-1,)), INVALID), (dict(first=(2 ** 31 - 4100,)), UNSUPPORTED), (dict(table=None), INVALID), (dict(table_cs=-1), INVALID),
    (dict(K=P + 8), MISALIGNED), (dict(k_rs=132), MISALIGNED), (dict(v_hs=-128), MISALIGNED), (dict(v_rs=64), INVALID),
] + [(dict(pool_=pool(**kw)), want) for kw, want in POOL_REFUSALS])
def test_rows_refusals(L, ctx, call, kw, want):
    if kw.get("first", 0) is None:
        kw = dict(kw)
        del kw["first"]
        desc, o, s = b._Kv8Rows(H=4, d=128, W=1, k_hs=1280, k_rs=128, v_hs=1280, v_rs=128), ints((0, 10)), pool()
        rc = (L.fc_kv8_append(ctx[0], None, C.byref(desc), P, P, 0, at(o), None, C.byref(s), P, 9, None, None) if call == "append" else
              L.fc_kv8_unpack(ctx[0], None, C.byref(desc), C.byref(s), P, 9, None, at(o), P, P, 0, None))
    else:
        rc = rows(L, ctx, call, **kw)
    assert rc == want


def test_rows_of_overlapping_tables_and_destinations(L, ctx):
    # append: two sequences whose entries would lie in one another's rows of the table
    assert rows(L, ctx, "append", off=(0, 10, 20), first=(0, 60), table_cs=1) == INVALID
    # unpack: rows or heads of a destination that overlap
    assert rows(L, ctx, "unpack", k_hs=128) == INVALID
    assert rows(L, ctx, "unpack", v_hs=0) == INVALID
    assert rows(L, ctx, "append", K=None) == INVALID and rows(L, ctx, "append", V=None) == INVALID
    assert rows(L, ctx, "unpack", K=None, V=None) == INVALID


def test_no_rows_is_nothing_to_do(L, ctx):
    for call in ("append", "unpack"):
        assert rows(L, ctx, call, off=(7, 7), K=None, V=None, table=None, pool_=pool(k_codes=None)) == 0


# ------------------------------------------------------------------------------------ pages

def ranges(L, ctx, name, *, ref=P, n_pages=100, table=P, cs=9, W=2, first=(0, 3), last=(2, 9)):
    a, z = ints(first), ints(last)
    return getattr(L, name)(ctx[0], None, ref, n_pages, table, cs, W, at(a), at(z), None)


@pytest.mark.parametrize("name", ["fc_pages_take", "fc_pages_drop"])
@pytest.mark.parametrize("kw, want", [
    (dict(ref=None), INVALID), (dict(table=None), INVALID), (dict(n_pages=0), INVALID), (dict(n_pages=2 ** 31 - 8000), UNSUPPORTED), (dict(W=0), INVALID), (dict(W=65), UNSUPPORTED),
    (dict(first=(-1, 0)), INVALID), (dict(first=(3, 3)), INVALID), (dict(last=(2, 10)), INVALID), (dict(cs=-1), INVALID), (dict(first=None), INVALID),
    (dict(last=None), INVALID), (dict(ref=P + 4), MISALIGNED),
    (dict(W=1, first=(0,), last=(2 ** 31 - 1,)), UNSUPPORTED),
    (dict(first=(2, 9), last=(2, 9), ref=None, table=None), 0),  # nothing asked for
])
def test_range_refusals(L, ctx, name, kw, want):
    assert ranges(L, ctx, name, **kw) == want


def fork(L, ctx, *, H=4, d=128, ref=P, table=P, cs=9, n_seq=4, n=2, src=(0, 0), dst=(1, 2), tokens=(100, 64), ws=P, ws_bytes=None, pool_=None):
    s, x, y, t = pool() if pool_ is None else pool_, ints(src), ints(dst), ints(tokens)
    return L.fc_pages_fork(ctx[0], None, C.byref(s), H, d, ref, table, cs, n_seq, n, at(x), at(y), at(t), None, ws,
                           L.fc_pages_workspace_bytes(s.n_pages) if ws_bytes is None else ws_bytes)


@pytest.mark.parametrize("kw, want", [
    (dict(H=0), INVALID), (dict(H=70000), UNSUPPORTED), (dict(d=32), UNSUPPORTED), (dict(ref=None), INVALID), (dict(table=None), INVALID),
    (dict(n=-1), INVALID), (dict(n=65), UNSUPPORTED), (dict(n_seq=0), INVALID), (dict(src=(0, 4)), INVALID), (dict(dst=(1, -1)), INVALID),
    (dict(dst=(1, 1)), INVALID), (dict(dst=(0, 1)), INVALID), (dict(src=(0, 1), dst=(1, 2)), INVALID), (dict(tokens=(-1, 0)), INVALID),
    (dict(tokens=(9 * 64 + 1, 0)), INVALID), (dict(src=None), INVALID), (dict(tokens=None), INVALID), (dict(ref=P + 8), MISALIGNED),
    (dict(ws=None), WORKSPACE), (dict(ws_bytes=16), WORKSPACE), (dict(ws=P + 8), MISALIGNED),
    (dict(n=0, src=None, dst=None, tokens=None, ref=None, table=None, ws=None), 0),
] + [(dict(pool_=pool(**kw)), want) for kw, want in POOL_REFUSALS])
def test_fork_refusals(L, ctx, kw, want):
    assert fork(L, ctx, **kw) == want


@pytest.mark.parametrize("kw, want", [
    (dict(H=0), INVALID), (dict(d=32), UNSUPPORTED), (dict(ref=None), INVALID), (dict(n_seq=-1), INVALID), (dict(entries=-1), INVALID),
    (dict(table=None), INVALID), (dict(cs=5), INVALID), (dict(ref=P + 4), MISALIGNED), (dict(ws=None), WORKSPACE), (dict(ws=P + 4), MISALIGNED),
    (dict(ws_bytes=100), WORKSPACE),
] + [(dict(pool_=pool(**kw)), want) for kw, want in POOL_REFUSALS])
def test_compact_refusals(L, ctx, kw, want):
    f = dict(H=4, d=128, ref=P, table=P, cs=9, n_seq=3, entries=9, ws=P, ws_bytes=L.fc_pages_workspace_bytes(100), pool_=pool())
    f.update(kw)
    assert L.fc_pages_compact(ctx[0], None, C.byref(f["pool_"]), f["H"], f["d"], f["ref"], f["table"], f["cs"], f["n_seq"], f["entries"],
                              None, None, f["ws"], f["ws_bytes"]) == want


def test_pages_workspace(L):
    assert L.fc_pages_workspace_bytes(0) == L.fc_pages_workspace_bytes(-3) == 0
    # copies of half the pages (or of every fork), and the new place of each
    assert L.fc_pages_workspace_bytes(1) >= 16 + 64 * 8 + 4
    assert L.fc_pages_workspace_bytes(100_001) >= 16 + 50_001 * 8 + 100_001 * 4


# ------------------------------------------------------------------------------------ attention

def attend(L, ctx, kind, *, Q=P, O=P, K=P, V=P, pool_=None, table=P, table_cs=9, cache=(300, 300), dtype=b.BF16, off=(0, 3, 7), vis=(300, 340), sink=0,
           begin=(0, 100), first=None, seg=((0, 50), (10,)), ids=P, n=P, lse=None, lse_hs=0, ws=P, ws_bytes=1 << 40, size=False, **kw):
    f = dict(H_q=8, H_kv=4, d=128, W=2, q_hs=1280, q_rs=128, k_hs=12800, k_rs=128, v_hs=12800, v_rs=128, o_hs=1280, o_rs=128, kv_rows=60, scale=0.0, impl=0)
    f.update(kw)
    if kind == "span":
        vis = tuple(min(v, 50) for v in vis)
    desc = b._AttnDesc(**f)
    o, v, g, w, c = ints(off), ints(vis), ints(begin), ints(first), ints(cache)
    sl, sp, n_seg = (ints(seg[0]), ints(seg[1]), len(seg[1])) if seg else (None, None, 0)
    s = pool() if pool_ is None else pool_
    if kind == "span":
        if size:
            return L.fc_chunk_attention_span_workspace_bytes(ctx[0], C.byref(desc), dtype, at(o), at(v), sink, at(g), at(sl), n_seg)
        return L.fc_chunk_attention_span(ctx[0], None, C.byref(desc), Q, K, V, dtype, at(o), at(v), sink, at(g), at(sl), at(sp), n_seg, ids, n, O, lse,
                                         lse_hs, None, ws, ws_bytes)
    if size:
        return L.fc_chunk_attention_kv8_workspace_bytes(ctx[0], C.byref(desc), dtype, s.page, table_cs, at(c), at(o), at(v), sink, at(g), at(w), at(sl), n_seg)
    return L.fc_chunk_attention_kv8(ctx[0], None, C.byref(desc), Q, C.byref(s), table, table_cs, at(c), K, V, dtype, at(o), at(v), sink, at(g), at(w),
                                    at(sl), at(sp), n_seg, ids, n, O, lse, lse_hs, None, ws, ws_bytes)


@pytest.mark.parametrize("kind", ["kv8", "span"])
@pytest.mark.parametrize("kw, want", [
    (dict(dtype=5), UNSUPPORTED), (dict(d=80), UNSUPPORTED), (dict(H_q=6), INVALID), (dict(H_kv=0), INVALID), (dict(W=0), INVALID), (dict(W=65), UNSUPPORTED),
    (dict(H_q=70000, H_kv=70000), UNSUPPORTED), (dict(impl=1), INVALID), (dict(impl=4), INVALID), (dict(impl=2, dtype=b.F32), UNSUPPORTED),
    (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(sink=-1), INVALID), (dict(begin=(-1, 0)), INVALID),
    (dict(vis=(-1, 10)), INVALID), (dict(off=(0, 3, 2)), INVALID), (dict(off=(-1, 3, 7)), INVALID), (dict(off=None), INVALID), (dict(vis=None), INVALID),
    (dict(Q=None), INVALID), (dict(O=None), INVALID), (dict(K=None), INVALID), (dict(V=None), INVALID), (dict(ids=None), INVALID), (dict(n=None), INVALID),
    (dict(Q=P + 8), MISALIGNED), (dict(O=P + 4), MISALIGNED), (dict(K=P + 2), MISALIGNED), (dict(q_rs=130), MISALIGNED), (dict(k_rs=64), INVALID),
    (dict(o_hs=64), INVALID), (dict(o_rs=0), INVALID), (dict(k_hs=0), UNSUPPORTED), (dict(v_rs=1 << 37), UNSUPPORTED),
    (dict(seg=((0, 50), (11,))), INVALID), (dict(seg=((1, 50), (0,))), INVALID), (dict(seg=((0, 50, 40), (0, 0))), INVALID), (dict(seg=((0, 50), (-1,))), INVALID),
    (dict(seg=(tuple(range(64)), (0,) * 63)), UNSUPPORTED), (dict(lse=P), INVALID), (dict(ws=P + 8, impl=3), MISALIGNED), (dict(seg=((0, 2 ** 31 - 4000), (0,))), UNSUPPORTED),
])
def test_attention_refusals(L, ctx, kind, kw, want):
    if kw.get("vis", 0) is None:
        vis_free = dict(off=(0, 3, 7))
        desc = b._AttnDesc(H_q=8, H_kv=4, d=128, W=2, q_hs=1280, q_rs=128, k_hs=1, k_rs=128, v_hs=1, v_rs=128, o_hs=1280, o_rs=128, kv_rows=60)
        o = ints(vis_free["off"])
        assert L.fc_chunk_attention_span(ctx[0], None, C.byref(desc), P, P, P, 0, at(o), None, 0, None, None, None, 0, P, P, P, None, 0, None, P, 1 << 30) == want
        return
    if "ws" in kw:  # a call that is cut into parts
        kw = dict(kw, off=(0, 1, 2), vis=(30000, 30000), cache=(30000, 30000), table_cs=1000, seg=((0, 30000), (0,)), kv_rows=30000, k_hs=30000 * 128, v_hs=30000 * 128)
        if kind == "span":
            desc = b._AttnDesc(H_q=8, H_kv=4, d=128, W=2, q_hs=1280, q_rs=128, k_hs=30000 * 128, k_rs=128, v_hs=30000 * 128, v_rs=128, o_hs=1280, o_rs=128, kv_rows=30000, impl=3)
            o, v, sl, sp = ints((0, 1, 2)), ints((30000, 30000)), ints((0, 30000)), ints((0,))
            assert L.fc_chunk_attention_span(ctx[0], None, C.byref(desc), P, P, P, 0, at(o), at(v), 0, None, at(sl), at(sp), 1, P, P, P, None, 0, None, P + 8, 1 << 40) == want
            assert L.fc_chunk_attention_span(ctx[0], None, C.byref(desc), P, P, P, 0, at(o), at(v), 0, None, at(sl), at(sp), 1, P, P, P, None, 0, None, P, 16) == WORKSPACE
            return
    assert attend(L, ctx, kind, **kw) == want


@pytest.mark.parametrize("kw, want", [
    (dict(pool_=pool(**kw)), want) for kw, want in POOL_REFUSALS
] + [(dict(table=None), INVALID), (dict(table_cs=-1), INVALID), (dict(cache=(-1, 0)), INVALID), (dict(first=(0, -1)), INVALID),
     (dict(vis=(300, 351)), INVALID), (dict(first=(0, 11)), INVALID), (dict(seg=None), INVALID), (dict(cache=(2 ** 31 - 4100, 0)), UNSUPPORTED)])
def test_attention_over_pages_refusals(L, ctx, kw, want):
    assert attend(L, ctx, "kv8", **kw) == want


def test_attention_of_no_rows(L, ctx):
    for kind in ("kv8", "span"):
        assert attend(L, ctx, kind, off=(4, 4, 4), Q=None, O=None, ids=None, n=None) == 0
        assert attend(L, ctx, kind, off=(4, 4, 4), size=True) == 0


def test_attention_workspace(L, ctx):
    # refused arguments need none; one token over a long store is cut into parts
    assert attend(L, ctx, "kv8", size=True, dtype=9) == 0
    many = attend(L, ctx, "kv8", size=True, off=(0, 1, 2), cache=(30000, 30000), vis=(30000, 30000), begin=(0, 0), table_cs=500)
    assert many > 2 * 8 * 128 * 4
    # what is not seen costs nothing
    assert attend(L, ctx, "kv8", size=True, off=(0, 1, 2), cache=(30000, 30000), vis=(30000, 30000), begin=(29990, 29990), sink=3, table_cs=500) < many


# ------------------------------------------------------------------------------------ the format, by hand

def test_codes_by_hand():
    # sign, exponent with bias 7, mantissa of three bits: 0x38 = 1, 0x3c = 1.5, 0x7e = 448, 0x01 = 2^-9
    assert pg.code_values(np.uint8([0x38, 0x3c, 0x7e, 0x01, 0x08, 0xb8])).tolist() == [1, 1.5, 448, 2.0 ** -9, 2.0 ** -6, -1]
    # ties go to the even code: 1.0625 lies between 1 (0x38) and 1.125 (0x39), 1.1875 between 0x39 and 1.25 (0x3a)
    assert pg.codes_of([1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 500, -0.0, math.inf]).tolist() == [0x38, 0x3a, 0x00, 0x02, 0x7e, 0x80, 0x7f]


def test_scales_by_hand():
    # 448 s >= a with four bits: 1.125 reaches 504, so 448.1 needs it; 448 itself has the scale 1
    assert [pg.scale_of(a) for a in (448, 448.1, 504, 504.1, 0, 1e-40, 3e38)] == [1, 1.125, 1.125, 1.25, 0, 2.0 ** -117, 2.0 ** 119]


def test_pages_by_hand():
    p = pg.Pages([1, 0, 0, 1, 0], [[3, 0, -1], [-1, -1, -1]])
    p.take([2, 0], [3, 1])
    assert p.table == [[3, 0, 1], [2, -1, -1]] and p.ref == [1, 1, 1, 1, 0]
    assert p.fork([0], [1], [40], 16) == [(1, 4)] and p.table[1] == [3, 0, 4] and p.ref == [2, 1, 1, 2, 1]
    p.drop([0, 0], [3, 0])
    assert p.table[0] == [-1, -1, -1] and p.ref == [1, 0, 1, 1, 1]
    assert p.compact() == [(4, 1)] and p.table[1] == [3, 0, 1] and p.ref == [1, 1, 1, 1, 0]


def test_pool_class_refuses_tensors_that_do_not_fit():
    import torch
    codes, scales = torch.zeros((3, 2, 16, 64), dtype=torch.uint8), torch.zeros((3, 2))
    fc.Kv8Pool(codes, scales, codes.clone(), scales.clone())
    for bad in ((codes[..., :32], scales, codes[..., :32], scales), (codes, scales[:2], codes, scales[:2]), (codes.int(), scales, codes.int(), scales),
                (codes, scales.double(), codes, scales.double()), (codes[0], scales, codes[0], scales), (codes, scales, codes.transpose(0, 1), scales)):
        with pytest.raises(fc.FcError):
            fc.Kv8Pool(*bad)
    with pytest.raises(fc.FcError):
        fc.Kv8Pool.empty(2, 2, 24, 64, device="cpu")
