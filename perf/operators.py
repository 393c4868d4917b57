"""Cases that measure the operators around a 4-bit K/V store: per-head norms with the position rotation of several
axes, packing and unpacking of the store, and chunk-causal attention over it.

`run` computes each operator in its plain form (elementary torch operations), or, where `own` is set, through the
library's calls.  `exact` states the definitions again in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 32  # elements of a row that share a scale
EPS, THETA = 1e-6, 10000.0


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # --- norms of queries and keys with the rotation over (time, height, width)
        # one token of a fused q/k/v projection: the latency of a call
        {"name": "norm rope, one token", "op": "rope", "H_q": 24, "H_kv": 24, "d": 128, "T": 1, "dtype": "bf16", "norm": True,
         "fused": True, "grid": True, "halves": False},
        # a chunk of three latent frames of 30 x 52 patches, all heads, straight out of the fused projection
        {"name": "norm rope, chunk", "op": "rope", "H_q": 24, "H_kv": 24, "d": 128, "T": 4680, "dtype": "bf16", "norm": True,
         "fused": True, "grid": True, "halves": False},
        # cached keys in fp32 turned to new positions, one position per token, nothing normalised
        {"name": "rope, cached keys f32", "op": "rope", "H_q": 0, "H_kv": 8, "d": 64, "T": 18719, "dtype": "f32", "norm": False,
         "fused": False, "grid": False, "halves": True},
        # --- packing the store (and reading back what it stands for)
        # one token appended for all heads
        {"name": "pack, one token", "op": "pack", "H": 24, "d": 128, "n_old": 0, "n_new": 1, "n_keep": 0, "dtype": "bf16"},
        # a compression event of the streaming workload: 28080 packed rows and a new chunk, back to 28080
        {"name": "pack, compaction", "op": "pack", "H": 24, "d": 128, "n_old": 28080, "n_new": 4680, "n_keep": 28080, "dtype": "bf16"},
        # odd sizes, fp32 rows
        {"name": "pack, f32 odd", "op": "pack", "H": 5, "d": 64, "n_old": 1337, "n_new": 4099, "n_keep": 2051, "dtype": "f32"},
        # --- unpacking: the keys of a compression event for the score, or a layer's clean region
        {"name": "unpack, clean region", "op": "unpack", "H": 24, "d": 128, "n": 18720, "dtype": "bf16"},
        {"name": "unpack, f32 odd", "op": "unpack", "H": 3, "d": 64, "n": 2999, "dtype": "f32"},
        # --- attention over the packed store
        # one token against a full clean region
        {"name": "attention, one token", "op": "attn", "H_q": 24, "H_kv": 24, "d": 128, "n_c": 1, "W": 1, "active": "all",
         "n_cache": 28080, "win": True, "dtype": "bf16"},
        # the last fifty queries of a step with shared key heads, odd lengths
        {"name": "attention, 50 rows gqa", "op": "attn", "H_q": 16, "H_kv": 4, "d": 128, "n_c": 50, "W": 1, "active": "all",
         "n_cache": 12345, "win": True, "dtype": "bf16"},
        # two chunks in flight, the second recomputed, over a full clean region
        {"name": "attention, chunk", "op": "attn", "H_q": 24, "H_kv": 24, "d": 128, "n_c": 4680, "W": 2, "active": "last",
         "n_cache": 18720, "win": True, "dtype": "bf16"},
        # fp32, four ragged chunks
        {"name": "attention, f32 ragged", "op": "attn", "H_q": 4, "H_kv": 2, "d": 64, "n_c": 251, "W": 4, "active": "all",
         "n_cache": 511, "win": True, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "pack", "unpack", "attn", "attn"])
    d = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "rope":
        H_kv, group = rng.choice([1, 2, 4, 6, 8, 12]), rng.choice([0, 1, 1, 2])
        return {"op": op, "H_q": H_kv * group, "H_kv": H_kv, "d": d, "T": _log(rng, 1, 12000), "dtype": dtype,
                "norm": rng.random() < 0.7, "fused": rng.random() < 0.5, "grid": rng.random() < 0.5, "halves": rng.random() < 0.5}
    if op == "pack":
        n_old, n_new = rng.choice([0, _log(rng, 1, 20000)]), _log(rng, 1, 9000)
        n_keep = 0 if rng.random() < 0.4 else rng.randint(max(1, (n_old + n_new) // 3), n_old + n_new)
        return {"op": op, "H": rng.choice([1, 2, 3, 5, 8, 12]), "d": d, "n_old": n_old if n_keep else 0, "n_new": n_new,
                "n_keep": n_keep, "dtype": dtype}
    if op == "unpack":
        return {"op": op, "H": rng.choice([1, 2, 3, 5, 8, 12]), "d": d, "n": _log(rng, 1, 30000), "dtype": dtype}
    H_kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4])
    n_c, W = (_log(rng, 1, 60), rng.choice([1, 1, 2])) if rng.random() < 0.5 else (_log(rng, 60, 1500), rng.choice([1, 2, 3]))
    n_cache = _log(rng, 1, 30000) if dtype == "bf16" else _log(rng, 1, 2500)
    if dtype == "f32":
        n_c = min(n_c, 300)
    return {"op": op, "H_q": H_kv * group, "H_kv": H_kv, "d": d, "n_c": n_c, "W": W, "active": rng.choice(["all", "last"]),
            "n_cache": n_cache, "win": rng.random() < 0.7, "dtype": dtype}


def work(case):
    es = 2 if case.get("dtype") == "bf16" else 4
    d = case["d"]
    packed = d // 2 + d // GROUP * 2  # bytes of a packed row
    if case["op"] == "rope":
        rows = (case["H_q"] + case["H_kv"]) * case["T"]
        return {"bytes": 2 * rows * d * es + (0 if case["grid"] else 12 * case["T"]), "flops": rows * d * (7 if case["norm"] else 3)}
    if case["op"] == "pack":  # packed rows and values both come out
        H, n = case["H"], case["n_keep"] or case["n_new"]
        old = _kept_old(case)
        return {"bytes": 2 * H * (old * packed + (n - old) * d * es + n * packed + n * packed + n * d * es) + (4 * H * n if case["n_keep"] else 0),
                "flops": 2 * H * d * (2 * (n - old) + n)}
    if case["op"] == "unpack":
        n = 2 * case["H"] * case["n"]
        return {"bytes": n * (packed + d * es), "flops": n * d}
    chunks = _active(case)
    keys = sum(case["n_cache"] + ((c + 1) * case["n_c"] if case["win"] else 0) for c in chunks)
    far = (max(chunks) + 1) * case["n_c"] if case["win"] else 0
    return {"bytes": 2 * case["H_kv"] * (case["n_cache"] * packed + far * d * es) + 2 * case["H_q"] * len(chunks) * case["n_c"] * d * es,
            "flops": 4 * d * case["H_q"] * case["n_c"] * keys}


def _kept_old(case):
    """Kept rows that were packed already: the newest ones are kept first, as a protected tail would be."""
    return max(0, case["n_keep"] - case["n_new"]) if case["n_keep"] else 0


def _active(case):
    return [case["W"] - 1] if case["active"] == "last" else list(range(case["W"]))


def _axes(d):
    """Elements of a head that turn with time, height and width."""
    s = 2 * (d // 6)
    return d - 2 * s, s, s


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, sigma, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(dtype)


def _packed(x):
    """Codes [H, n, d/2] and scales [H, n, d/32] of rows x: in each 32-bit word of eight elements, element 2i sits at bits
    4i of the low half and element 2i + 1 at bits 4i of the high half."""
    n, s = _quantise(x)
    c = (n + 8).to(torch.int32).unflatten(-1, (-1, 4, 2))  # words, i, which half
    shift = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device=x.device, dtype=torch.int32)
    words = (c << shift).sum((-1, -2), dtype=torch.int32)
    return words.view(torch.uint8), s


def prepare(case, seed):
    g, dt, d = _gen(seed), DTYPES[case["dtype"]], case["d"]
    s = {"case": case}
    if case["op"] == "rope":
        H_q, H_kv, T = case["H_q"], case["H_kv"], case["T"]
        if case["fused"]:  # [T, q heads | k heads | v heads], as a projection leaves it
            x = _normal(g, (T, H_q + 2 * H_kv, d), 1.5, dt).transpose(0, 1)
            s["Q"], s["K"] = x[:H_q], x[H_q:H_q + H_kv]
        else:
            s["Q"], s["K"] = _normal(g, (H_q, T, d), 1.5, dt), _normal(g, (H_kv, T, d), 1.5, dt)
        s["wq"] = _normal(g, (d,), 0.2, torch.float32) + 1 if case["norm"] else None
        s["wk"] = _normal(g, (d,), 0.2, torch.float32) + 1 if case["norm"] else None
        # a chunk's tokens fill a grid of 30 x 52 patches a frame, from its first frame on; or each has its own place
        s["grid"] = (int(seed) % 40, 30, 52) if case["grid"] else None
        s["pos"] = None if case["grid"] else torch.randint(-60, 2000, (T, 3), generator=g, device=DEV, dtype=torch.int32)
        s["Q_out"] = torch.empty((H_q, T, d), dtype=dt, device=DEV)
        s["K_out"] = torch.empty((H_kv, T, d), dtype=dt, device=DEV)
        s["Q"], s["Q_out"] = (s["Q"], s["Q_out"]) if H_q else (None, None)
        return s
    if case["op"] == "pack":
        H, n_old, n_new = case["H"], case["n_old"], case["n_new"]
        s["K"], s["V"] = _normal(g, (H, n_new, d), 1.0, dt), _normal(g, (H, n_new, d), 0.5, dt)
        s["old"] = s["kept"] = None
        n = n_new
        if n_old:
            s["old"] = _packed(_normal(g, (H, n_old, d), 1.0, dt)) + _packed(_normal(g, (H, n_old, d), 0.5, dt))
        if case["n_keep"]:
            n, old = case["n_keep"], _kept_old(case)
            rank = torch.rand((H, n_old + n_new), generator=g, device=DEV)
            rank[:, :n_old] += 2.0  # old rows drop first
            s["kept"] = rank.argsort(-1)[:, :n].sort(-1).values.to(torch.int32).contiguous()
        s["out"] = tuple(torch.empty(shape, dtype=t, device=DEV) for shape, t in
                         2 * (((H, n, d // 2), torch.uint8), ((H, n, d // GROUP), torch.bfloat16)))
        s["K_dst"], s["V_dst"] = torch.empty((H, n, d), dtype=dt, device=DEV), torch.empty((H, n, d), dtype=dt, device=DEV)
        return s
    if case["op"] == "unpack":
        shape = (case["H"], case["n"], d)
        s["cache"] = _packed(_normal(g, shape, 1.0, dt)) + _packed(_normal(g, shape, 0.5, dt))
        s["K_dst"], s["V_dst"] = torch.empty(shape, dtype=dt, device=DEV), torch.empty(shape, dtype=dt, device=DEV)
        return s
    H_q, H_kv, n_c, W, n_cache = (case[k] for k in ("H_q", "H_kv", "n_c", "W", "n_cache"))
    shape, win = (H_kv, n_cache, d), (H_kv, W * n_c if case["win"] else 0, d)
    s["cache"] = _packed(_normal(g, shape, 1.0, dt)) + _packed(_normal(g, shape, 0.5, dt))
    s["Q"] = _normal(g, (H_q, W * n_c, d), 1.0, dt)
    s["K"], s["V"] = _normal(g, win, 1.0, dt), _normal(g, win, 0.5, dt)
    s["O"] = torch.zeros((H_q, W * n_c, d), dtype=dt, device=DEV)  # chunks that are not active keep what is there
    s["off"] = [c * n_c for c in range(W + 1)]
    s["vis"] = [n_cache + ((c + 1) * n_c if case["win"] else 0) for c in range(W)]
    ids = _active(case)
    s["ids"] = torch.tensor(ids + [-1] * (W - len(ids)), dtype=torch.int32, device=DEV)
    s["n_active"] = torch.tensor([len(ids)], dtype=torch.int32, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _quantise(x):
    """Whole numbers [H, n, d] in -7 .. 7 and bf16 scales [H, n, d/32]."""
    g = x.double().unflatten(-1, (-1, GROUP))
    a = (g.abs().amax(-1) / 7).float()
    s = ((a.view(torch.int32) + 0x7FFFF) & ~0x7FFFF).view(torch.float32).clamp(2.0 ** -126, 2.0 ** 122)
    s = torch.where(a > 0, s, 0)
    n = (g / s.double().unsqueeze(-1)).nan_to_num(0.0).round().clamp(-7, 7)
    return n.flatten(-2), s.to(torch.bfloat16)


def _values(codes, scales):
    """fp32 rows [H, n, d] that packed rows stand for."""
    words = codes.view(torch.int32)
    shift = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device=codes.device, dtype=torch.int32)
    n = ((words.unsqueeze(-1) >> shift) & 15).flatten(-2) - 8
    return (n.unflatten(-1, (-1, GROUP)).float() * scales.float().unsqueeze(-1)).flatten(-2)


def _positions(s, T):
    if s["pos"] is not None:
        return s["pos"].double()
    t0, h, w = s["grid"]
    n = torch.arange(T, device=DEV)
    return torch.stack([t0 + n // (h * w), n // w % h, n % w], -1).double()


def _turned(x, weight, pos, halves, dtype):
    x = x.float()
    d = x.shape[-1]
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
    a, b, c = _axes(d)
    f = torch.cat([THETA ** (-torch.arange(0, n, 2, device=DEV, dtype=torch.float64) / n) for n in (a, b, c)])
    axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor([a // 2, b // 2, c // 2], device=DEV))
    angle = pos[:, axis] * f
    cos, sin = angle.cos().float(), angle.sin().float()
    if halves:
        x0, x1 = (torch.cat([v.unflatten(-1, (2, -1))[..., k, :] for v in x.split([a, b, c], -1)], -1) for k in (0, 1))
        y0, y1 = x0 * cos - x1 * sin, x0 * sin + x1 * cos
        parts = [torch.cat(p, -1) for p in zip(y0.split([a // 2, b // 2, c // 2], -1), y1.split([a // 2, b // 2, c // 2], -1))]
        return torch.cat(parts, -1).to(dtype)
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack([x0 * cos - x1 * sin, x0 * sin + x1 * cos], -1).flatten(-2).to(dtype)


def _plain_rope(s):
    case = s["case"]
    pos, dt = _positions(s, case["T"]), DTYPES[case["dtype"]]
    Q = None if s["Q"] is None else _turned(s["Q"], s["wq"], pos, case["halves"], dt)
    return Q, _turned(s["K"], s["wk"], pos, case["halves"], dt)


def _plain_pack(s, x, codes, scales):
    n, scale = _quantise(x)
    rows = (n.unflatten(-1, (-1, GROUP)) * scale.double().unsqueeze(-1)).flatten(-2).to(x.dtype)
    if codes is not None:
        rows = torch.cat([_values(codes, scales).to(x.dtype), rows], 1)
    if s["kept"] is None:
        return rows
    return rows.gather(1, s["kept"].long().unsqueeze(-1).expand(-1, -1, rows.shape[-1]))


def _plain_attention(s):
    case = s["case"]
    H_kv, group = case["H_kv"], case["H_q"] // case["H_kv"]
    kc, ks, vc, vs = s["cache"]
    K = torch.cat([_values(kc, ks), s["K"].float()], 1)
    V = torch.cat([_values(vc, vs), s["V"].float()], 1)
    ids = _active(case)
    first, rows = ids[0] * case["n_c"], len(ids) * case["n_c"]
    q = s["Q"][:, first:first + rows].float().reshape(H_kv, group * rows, -1) / math.sqrt(case["d"])
    S = q @ K.transpose(1, 2)
    vis = torch.tensor(s["vis"], device=DEV)[ids].repeat_interleave(case["n_c"]).repeat(group)
    if len(ids) > 1 or s["vis"][ids[0]] < K.shape[1]:
        S.masked_fill_(torch.arange(K.shape[1], device=DEV) >= vis[:, None], -math.inf)
    P = S.sub_(S.amax(-1, keepdim=True)).exp_()
    out = (P @ V) / P.sum(-1, keepdim=True)
    O = s["O"].clone()
    O[:, first:first + rows] = out.view(case["H_q"], rows, -1).to(O.dtype)
    return O


# ------------------------------------------------------------------------------------------------ the library's calls

_kept = {}


def _library():
    """The package and a context of it, which a program creates once."""
    if not _kept:
        import paper_2602_10825_b200 as fc
        _kept["fc"], _kept["ctx"] = fc, fc.Context(torch.cuda.current_device())
    return _kept["fc"], _kept["ctx"]


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "rope":
            return _plain_rope(s)
        if op == "pack":
            old = s["old"] or (None, None, None, None)
            return _plain_pack(s, s["K"], old[0], old[1]), _plain_pack(s, s["V"], old[2], old[3])
        if op == "unpack":
            dt = s["K_dst"].dtype
            return _values(*s["cache"][:2]).to(dt), _values(*s["cache"][2:]).to(dt)
        return _plain_attention(s)
    fc, ctx = _library()
    case = s["case"]
    if op == "rope":
        return ctx.qk_norm_rope(s["Q"], s["K"], axes=_axes(case["d"]), norm=case["norm"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS,
                                theta=THETA, grid=s["grid"], pos=s["pos"], pairing=fc.ROPE_HALVES if case["halves"] else fc.ROPE_PAIRS,
                                Q_out=s["Q_out"], K_out=s["K_out"])
    if op == "pack":
        out = fc.Kv4Cache(*s["out"])
        ctx.kv4_pack(s["K"], s["V"], out, old=None if s["old"] is None else fc.Kv4Cache(*s["old"]), kept_idx=s["kept"])
        return ctx.kv4_unpack(out, K_dst=s["K_dst"], V_dst=s["V_dst"])
    if op == "unpack":
        return ctx.kv4_unpack(fc.Kv4Cache(*s["cache"]), K_dst=s["K_dst"], V_dst=s["V_dst"])
    K, V = (s["K"], s["V"]) if case["win"] else (None, None)
    return ctx.chunk_attention_kv4(s["Q"], fc.Kv4Cache(*s["cache"]), K, V, s["off"], s["vis"], s["ids"], s["n_active"], s["O"])


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_turned(x, weight, pos, halves):
    y = x.double().clone()
    d = y.shape[-1]
    if weight is not None:
        y = y / (y.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * weight.double()
    out, start = y.clone(), 0
    for axis, n in enumerate(_axes(d)):
        for i in range(n // 2):
            at, to = (start + i, start + i + n // 2) if halves else (start + 2 * i, start + 2 * i + 1)
            turn = pos[:, axis] * THETA ** (-2.0 * i / n)
            out[..., at] = y[..., at] * turn.cos() - y[..., to] * turn.sin()
            out[..., to] = y[..., at] * turn.sin() + y[..., to] * turn.cos()
        start += n
    return out


def _exact_packed(x):
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for k in range(0, x.shape[-1], GROUP):
        v = x[..., k:k + GROUP].double()
        m, e = torch.frexp(v.abs().max(-1, keepdim=True).values / 7)
        scale = torch.ldexp(torch.ceil(m * 32) / 32, e).clamp(2.0 ** -126, 2.0 ** 122)
        out[..., k:k + GROUP] = torch.where(m > 0, torch.round(v / scale).clamp(-7, 7) * scale, torch.zeros_like(v))
    return out


def _exact_values(codes, scales):
    b = codes.long()
    out = torch.empty((*codes.shape[:-1], 2 * codes.shape[-1]), dtype=torch.float64, device=codes.device)
    for i in range(8):  # element i of every word: two elements a byte, even ones in the word's low half
        byte = b[..., (i % 2) * 2 + i // 4::4]
        out[..., i::8] = (byte // (16 if i // 2 % 2 else 1) % 16 - 8).double()
    for k in range(scales.shape[-1]):
        out[..., k * GROUP:(k + 1) * GROUP] *= scales[..., k:k + 1].double()
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        if s["grid"] is not None:
            t0, h, w = s["grid"]
            pos = torch.tensor([[t0 + n // (h * w), n % (h * w) // w, n % w] for n in range(case["T"])], dtype=torch.float64, device=DEV)
        else:
            pos = s["pos"].double()
        return (None if s["Q"] is None else _exact_turned(s["Q"], s["wq"], pos, case["halves"]),
                _exact_turned(s["K"], s["wk"], pos, case["halves"]))
    if case["op"] == "pack":
        out = []
        for i, x in enumerate((s["K"], s["V"])):
            rows = _exact_packed(x)
            if s["old"] is not None:
                rows = torch.cat([_exact_values(*s["old"][2 * i:2 * i + 2]), rows], 1)
            out.append(rows if s["kept"] is None else torch.stack([rows[h][s["kept"][h].long()] for h in range(case["H"])]))
        return tuple(out)
    if case["op"] == "unpack":
        return _exact_values(*s["cache"][:2]), _exact_values(*s["cache"][2:])
    out = s["O"].double()
    group, n_c = case["H_q"] // case["H_kv"], case["n_c"]
    for hk in range(case["H_kv"]):
        K = torch.cat([_exact_values(*(t[hk:hk + 1] for t in s["cache"][:2]))[0], s["K"][hk].double()])
        V = torch.cat([_exact_values(*(t[hk:hk + 1] for t in s["cache"][2:]))[0], s["V"][hk].double()])
        for h in range(hk * group, (hk + 1) * group):
            for c in _active(case):
                q = s["Q"][h, c * n_c:(c + 1) * n_c].double()
                logits = q @ K[:s["vis"][c]].T * case["d"] ** -0.5
                out[h, c * n_c:(c + 1) * n_c] = torch.softmax(logits, -1) @ V[:s["vis"][c]]
    return out
