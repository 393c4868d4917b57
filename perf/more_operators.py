"""Cases that measure the operators of a rolling generation: a paged K/V store in 8 bits with a scale for each page and
head, the upkeep of its pages, attention over it, and attention of a sliding window with a few first tokens that stay.

`run` computes each operator in its plain form (elementary torch operations), or, where `own` is set, through the
library's calls.  `exact` states the definitions again in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # --- rows into the pages, and read back from the page that the first of them falls into
        # one token for each of two branches of a generation, into pages that are partly filled
        {"name": "append, one token", "op": "append", "H": 24, "d": 128, "page": 64, "W": 2, "n": 1, "pos": 18000, "dtype": "bf16"},
        # a finished chunk of three latent frames, 24 heads
        {"name": "append, chunk", "op": "append", "H": 24, "d": 128, "page": 64, "W": 1, "n": 4680, "pos": 18720, "dtype": "bf16"},
        # five sequences of odd lengths, fp32, small pages
        {"name": "append, f32 odd", "op": "append", "H": 5, "d": 64, "page": 16, "W": 5, "n": 777, "pos": 1001, "dtype": "f32"},
        # --- the pages themselves
        # a generation branches into six and lets go of what has left its window
        {"name": "pages, branch", "op": "branch", "H": 24, "d": 128, "page": 64, "n_pages": 512, "n": 18650, "W": 6},
        # half the sequences of a fragmented pool are gone: the others' pages move to its front
        {"name": "pages, compact", "op": "compact", "H": 24, "d": 128, "page": 64, "n_pages": 1024, "W": 8, "entries": 75},
        # --- attention over the pages
        # one token against a full clean region
        {"name": "kv8, one token", "op": "kv8", "H_q": 24, "H_kv": 24, "d": 128, "page": 64, "n_c": 1, "W": 1, "shared": True,
         "active": "all", "n_cache": 28080, "win": True, "sink": 0, "span": 0, "dtype": "bf16"},
        # a batch of sixteen sequences of ragged lengths, grouped heads, first tokens and a window
        {"name": "kv8, batch gqa", "op": "kv8", "H_q": 32, "H_kv": 8, "d": 128, "page": 32, "n_c": 1, "W": 16, "shared": False,
         "active": "all", "n_cache": 16000, "win": True, "sink": 16, "span": 8192, "dtype": "bf16"},
        # two chunks in flight, the second recomputed, over a full clean region
        {"name": "kv8, chunk", "op": "kv8", "H_q": 24, "H_kv": 24, "d": 128, "page": 64, "n_c": 4680, "W": 2, "shared": True,
         "active": "last", "n_cache": 18720, "win": True, "sink": 0, "span": 0, "dtype": "bf16"},
        # fp32, three branches with rows of their own
        {"name": "kv8, f32 ragged", "op": "kv8", "H_q": 4, "H_kv": 2, "d": 64, "page": 16, "n_c": 37, "W": 3, "shared": False,
         "active": "all", "n_cache": 3001, "win": True, "sink": 5, "span": 1500, "dtype": "f32"},
        # --- a sliding window with first tokens that stay, over plain rows
        # one token, a window of two chunks behind the first frame
        {"name": "span, one token", "op": "span", "H_q": 24, "H_kv": 24, "d": 128, "n_c": 1, "W": 1, "active": "all",
         "n_past": 28080, "sink": 1560, "span": 9360, "dtype": "bf16"},
        # four chunks in flight, each with its own window
        {"name": "span, chunks", "op": "span", "H_q": 24, "H_kv": 24, "d": 128, "n_c": 1560, "W": 4, "active": "all",
         "n_past": 18720, "sink": 1560, "span": 9360, "dtype": "bf16"},
        # fp32, odd everything
        {"name": "span, f32 odd", "op": "span", "H_q": 6, "H_kv": 3, "d": 64, "n_c": 61, "W": 3, "active": "all",
         "n_past": 1777, "sink": 7, "span": 801, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "branch", "compact", "kv8", "kv8", "kv8", "span", "span"])
    d, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "append":
        W = rng.choice([1, 1, 2, 5, 16])
        return {"op": op, "H": rng.choice([1, 2, 3, 5, 8, 12]), "d": d, "page": page, "W": W, "n": _log(rng, 1, 9000 // W),
                "pos": rng.choice([0, _log(rng, 1, 20000)]), "dtype": dtype}
    if op == "branch":
        n, W = _log(rng, 1, 200 * page), rng.choice([1, 2, 3, 7, 16])
        return {"op": op, "H": rng.choice([1, 2, 3, 5, 8, 12]), "d": d, "page": page, "n_pages": -(-n // page) + 3 * W + rng.randint(0, 50),
                "n": n, "W": W}
    if op == "compact":
        W, entries = rng.choice([2, 3, 5, 8, 16]), rng.randint(3, 60)
        return {"op": op, "H": rng.choice([1, 2, 3, 5, 8, 12]), "d": d, "page": page,
                "n_pages": W * entries + rng.randint(0, W * entries), "W": W, "entries": entries}
    H_kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4])
    n_c, W = (_log(rng, 1, 60), rng.choice([1, 1, 2, 6])) if rng.random() < 0.6 else (_log(rng, 60, 1200), rng.choice([1, 2, 3]))
    past = _log(rng, 1, 30000) if dtype == "bf16" else _log(rng, 1, 4000)
    if dtype == "f32":
        n_c = min(n_c, 300)
    case = {"op": op, "H_q": H_kv * group, "H_kv": H_kv, "d": d, "n_c": n_c, "W": W, "active": rng.choice(["all", "last"])}
    sink = rng.choice([0, rng.randint(1, 40), _log(rng, 1, 2000)])
    span = rng.choice([0, _log(rng, 1, 12000)])
    if op == "kv8":
        return {**case, "page": page, "shared": rng.random() < 0.5, "n_cache": past, "win": rng.random() < 0.7, "sink": sink, "span": span,
                "dtype": dtype}
    return {**case, "n_past": past, "sink": sink, "span": span or 1000, "dtype": dtype}


def _ragged(n, W):
    """Lengths of W sequences, the longest of them n."""
    return [max(1, n * (W + c + 1) // (2 * W)) for c in range(W)]


def _active(case):
    return [case["W"] - 1] if case["active"] == "last" else list(range(case["W"]))


def _layout(case):
    """Per chunk: tokens in pages, first token of the plain rows that it sees, visible tokens, and where its window begins."""
    W, n_c, span = case["W"], case["n_c"], case["span"]
    if case["op"] == "span":
        cache, first, vis = [0] * W, [0] * W, [case["n_past"] + (c + 1) * n_c for c in range(W)]
    elif case["shared"]:  # chunks in flight of one generation
        cache, first = [case["n_cache"]] * W, [0] * W
        vis = [case["n_cache"] + ((c + 1) * n_c if case["win"] else 0) for c in range(W)]
    else:  # sequences of a batch, each with plain rows of its own
        cache, first = _ragged(case["n_cache"], W), [c * n_c if case["win"] else 0 for c in range(W)]
        vis = [n + (n_c if case["win"] else 0) for n in cache]
    return cache, first, vis, [max(0, v - span) if span else 0 for v in vis]


def work(case):
    d = case["d"]
    es = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "append":  # new rows in, codes out, and the pages read back from the first row's page on
        H, n, W, page = case["H"], case["n"], case["W"], case["page"]
        rows = sum(p % page + n for p in _positions(case))
        return {"bytes": 2 * H * d * (W * n * es + rows * (1 + 1 + es)), "flops": 2 * H * d * 3 * rows}
    block = 2 * case["H"] * (case["page"] * d + 4) if "H" in case else 0
    if case["op"] == "branch":
        return {"bytes": 2 * block * sum(1 for n in _ragged(case["n"], case["W"]) if n % case["page"]) + 4 * case["n_pages"], "flops": 0}
    if case["op"] == "compact":
        used = (case["W"] + 1) // 2 * case["entries"]  # of n_pages, scattered
        return {"bytes": 2 * block * max(1, used * (case["n_pages"] - used) // case["n_pages"]) + 8 * case["n_pages"], "flops": 0}
    cache, first, vis, begin = _layout(case)
    ids, sink = _active(case), case["sink"]
    keys = sum(vis[c] - max(0, begin[c] - sink) if begin[c] > sink else vis[c] for c in ids)
    q = 2 * case["H_q"] * len(ids) * case["n_c"] * d * es

    def seen(chunks):  # tokens that some of these chunks, which share their keys, see: in pages, and plain
        lo, hi = min(begin[c] for c in chunks), max(vis[c] for c in chunks)
        n = cache[chunks[0]]
        parts = [(0, hi)] if lo <= sink else [(0, min(sink, hi)), (lo, hi)]
        return sum(max(0, min(b, n) - a) for a, b in parts), sum(max(0, b - max(a, n)) for a, b in parts)

    groups = [ids] if case["op"] == "span" or case["shared"] else [[c] for c in ids]
    paged, plain = (sum(x) for x in zip(*(seen(g) for g in groups)))
    return {"bytes": 2 * case["H_kv"] * d * (paged + plain * es) + q, "flops": 4 * d * case["H_q"] * case["n_c"] * keys}


def _positions(case):
    """Where each sequence's new rows begin."""
    return [p if case["pos"] else 0 for p in _ragged(case["pos"], case["W"])]


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, sigma, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(dtype)


def _filled_pool(g, n_pages, H, page, d):
    """(K codes, K scales, V codes, V scales) of pages full of rows; channels of K differ in size."""
    gain = _normal(g, (H, 1, d), 0.3).exp()
    K, V = _quantise(_normal(g, (n_pages, H, page, d), 1.0) * gain), _quantise(_normal(g, (n_pages, H, page, d), 0.5))
    return [K[0].view(torch.uint8), K[1], V[0].view(torch.uint8), V[1]]


def _tables(g, n_pages, counts, width):
    """Pages of a pool, in no order, for each of some sequences; -1 behind the last."""
    table = torch.full((len(counts), width), -1, dtype=torch.int32, device=DEV)
    pages, at = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32), 0
    for c, n in enumerate(counts):
        table[c, :n] = pages[at:at + n]
        at += n
    return table


def prepare(case, seed):
    g, d = _gen(seed), case["d"]
    s = {"case": case}
    if case["op"] == "append":
        H, page, W, n, dt = case["H"], case["page"], case["W"], case["n"], DTYPES[case["dtype"]]
        pos = _positions(case)
        counts = [-(-(p + n) // page) for p in pos]
        s["pool"] = _filled_pool(g, sum(counts) + 3, H, page, d)
        s["table"] = _tables(g, sum(counts) + 3, counts, max(counts))
        s["K"], s["V"] = _normal(g, (H, W * n, d), 1.3, dt), _normal(g, (H, W * n, d), 0.5, dt)
        s["pos"], s["off"] = pos, [c * n for c in range(W + 1)]
        s["first"] = [p // page * page for p in pos]
        rows = [p % page + n for p in pos]
        s["rows"] = [sum(rows[:c]) for c in range(W + 1)]
        s["K_dst"], s["V_dst"] = (torch.empty((H, s["rows"][-1], d), dtype=dt, device=DEV) for _ in range(2))
        return s
    if case["op"] in ("branch", "compact"):
        H, page, n_pages, W = case["H"], case["page"], case["n_pages"], case["W"]
        shape = (n_pages, H, page, d)
        codes = [torch.randint(0, 127, shape, generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        codes = [c | torch.randint(0, 2, shape, generator=g, device=DEV, dtype=torch.uint8) << 7 for c in codes]
        scales = [torch.rand((n_pages, H), generator=g, device=DEV) + 0.5 for _ in range(2)]
        s["pool"] = [codes[0], scales[0], codes[1], scales[1]]
        if case["op"] == "branch":  # row 0: the generation; the others: its branches to be
            n = case["n"]
            counts = [-(-n // page)] + [0] * W
            s["table0"] = _tables(g, n_pages, counts, counts[0] + 2)
            s["dst"], s["src"], s["tokens"] = list(range(1, W + 1)), [0] * W, _ragged(n, W)
            # each branch is to grow by a page; the generation itself keeps a first page and its newest third
            filled = [-(-t // page) for t in s["tokens"]]
            s["grow"] = [0] + filled, [0] + [f + 1 for f in filled]
            s["gone"] = [1] + [0] * W, [max(1, counts[0] * 2 // 3)] + [0] * W
        else:
            tables = _tables(g, n_pages, [case["entries"]] * W, case["entries"])
            s["table0"] = tables[::2].contiguous()  # every other sequence is gone
            s["table0"][-1, 0] = s["table0"][0, 0]  # a page that two sequences share
        ref = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV)
        at = s["table0"].flatten().long()
        ref.index_add_(0, torch.where(at < 0, n_pages, at), torch.ones_like(at, dtype=torch.int32))
        s["ref0"] = ref[:n_pages].clone()
        s["ref"], s["table"] = s["ref0"].clone(), s["table0"].clone()
        return s
    H_q, H_kv, n_c, W, dt = case["H_q"], case["H_kv"], case["n_c"], case["W"], DTYPES[case["dtype"]]
    cache, first, vis, begin = _layout(case)
    s["cache"], s["first"], s["vis"], s["begin"] = cache, first, vis, begin
    s["off"] = [c * n_c for c in range(W + 1)]
    if case["op"] == "kv8":
        page = case["page"]
        counts = [-(-n // page) for n in (cache[:1] if case["shared"] else cache)]
        n_pages = sum(counts) + 5
        s["pool"] = _filled_pool(g, n_pages, H_kv, page, d)
        s["table"] = _tables(g, n_pages, counts, max(counts))
        rows = W * n_c if case["win"] else 0
        s["segments"] = [0, rows], [0]
    else:  # the rows of the past lie behind those of the chunks in flight, in two pieces that are out of order
        past, rows = case["n_past"], case["n_past"] + W * n_c
        cut = past // 3
        s["segments"] = [0, cut, past, rows], [rows - cut, W * n_c, 0]
    s["Q"] = _normal(g, (H_q, W * n_c, d), 1.0, dt)
    s["K"], s["V"] = _normal(g, (H_kv, rows, d), 1.0, dt), _normal(g, (H_kv, rows, d), 0.5, dt)
    s["O"] = torch.zeros((H_q, W * n_c, d), dtype=dt, device=DEV)  # chunks that are not active keep what is there
    ids = _active(case)
    s["ids"] = torch.tensor(ids + [-1] * (W - len(ids)), dtype=torch.int32, device=DEV)
    s["n_active"] = torch.tensor([len(ids)], dtype=torch.int32, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _scale(a):
    """The least numbers with four significant bits that, 448 times, reach a."""
    q = (a.double() / 448).view(torch.int64)
    s = ((q + ((1 << 49) - 1)) & ~((1 << 49) - 1)).view(torch.float64).clamp(2.0 ** -117, 2.0 ** 119)
    return torch.where(a > 0, s, 0.0).float()


def _quantise(x, at_least=None):
    """E4M3 codes of blocks [..., rows, d], and a scale for each block."""
    s = _scale(x.abs().amax((-1, -2)))
    s = s if at_least is None else torch.maximum(s, at_least)
    return (x / torch.where(s > 0, s, 1.0)[..., None, None]).clamp(-448, 448).to(E4M3), s


def _values(codes, scales):
    return codes.view(E4M3).float() * scales[..., None, None]


def _plain_append(s, x, codes, scales, dst_type):
    case = s["case"]
    page, n, W, H, d = case["page"], case["n"], case["W"], case["H"], case["d"]
    pos = torch.tensor(s["pos"], device=DEV)
    blocks = max(-(-(p % page + n) // page) for p in s["pos"])
    t = torch.arange(blocks * page, device=DEV) - (pos % page)[:, None]  # [W, rows]: place among the new rows
    first = s["table"].gather(1, (pos // page)[:, None])[:, 0].long().clamp(min=0)
    old = _values(codes[first], scales[first])  # [W, H, page, d]
    new = x.float().unflatten(1, (W, n)).transpose(0, 1)
    rows = new.gather(2, t.clamp(0, n - 1)[:, None, :, None].expand(-1, H, -1, d))
    rows = torch.where(((t >= 0) & (t < n))[:, None, :, None], rows, 0.0)
    rows[:, :, :page] = torch.where((t[:, :page] < 0)[:, None, :, None], old, rows[:, :, :page])
    rows = rows.unflatten(2, (blocks, page)).transpose(1, 2)  # [W, blocks, H, page, d]
    least = torch.zeros((W, blocks, H), device=DEV)
    least[:, 0] = torch.where((pos % page > 0)[:, None], scales[first], 0.0)
    fresh = torch.where((t >= 0).view(W, blocks, 1, page, 1), rows, 0.0)
    scale = torch.maximum(_scale(fresh.abs().amax((-1, -2))), least)
    q = (rows / torch.where(scale > 0, scale, 1.0)[..., None, None]).clamp(-448, 448).to(E4M3)
    out = _values(q, scale).transpose(1, 2).flatten(2, 3).transpose(0, 1)  # [H, W, rows, d]
    return out[:, t < n].to(dst_type)


def _take_free(ref, n):
    return (ref == 0).nonzero()[:n, 0]


def _plain_branch(s):
    case, ref, table = s["case"], s["ref"], s["table"]
    page, W = case["page"], case["W"]
    ref.copy_(s["ref0"])
    table.copy_(s["table0"])
    tokens = torch.tensor(s["tokens"], device=DEV)
    width = table.shape[1]
    entry = torch.arange(width, device=DEV)
    full, part = tokens // page, tokens % page > 0
    parents = table[s["src"]]
    table[1:] = torch.where(entry < full[:, None], parents, -1)
    ref += torch.bincount(table[1:][table[1:] >= 0].long(), minlength=case["n_pages"]).int()
    at = part.nonzero()[:, 0]
    to, of = _take_free(ref, len(at)), parents[at, full[at]].long()
    for x in s["pool"]:
        x[to] = x[of]
    table[1 + at, full[at]] = to.int()
    ref[to] = 1
    more = _take_free(ref, W)  # a page for each branch to grow into
    table[torch.arange(1, W + 1, device=DEV), full + part] = more.int()
    ref[more] = 1
    gone = s["gone"]
    dropped = table[0, gone[0][0]:gone[1][0]]
    ref -= torch.bincount(dropped[dropped >= 0].long(), minlength=case["n_pages"]).int()
    table[0, gone[0][0]:gone[1][0]] = -1


def _plain_compact(s):
    ref, table = s["ref"], s["table"]
    ref.copy_(s["ref0"])
    table.copy_(s["table0"])
    used = ref > 0
    p = torch.arange(len(ref), device=DEV)
    n = used.sum()
    to, of = (~used & (p < n)).nonzero()[:, 0], (used & (p >= n)).nonzero()[:, 0]
    for x in s["pool"]:
        x[to] = x[of]
    place = p.int()
    place[of] = to.int()
    ref[to] = ref[of]
    ref[of] = 0
    table.copy_(torch.where(table >= 0, place[table.clamp(min=0).long()], -1))


def _plain_attention(s):
    """Keys of all chunks side by side, [chunks, H_kv, keys, d] (one entry where the chunks share them), and a mask."""
    case = s["case"]
    H_kv, group, n_c, d = case["H_kv"], case["H_q"] // case["H_kv"], case["n_c"], case["d"]
    ids = _active(case)
    log, phys = s["segments"]
    row = torch.cat([torch.arange(b - a, device=DEV) + p for a, b, p in zip(log, log[1:], phys)])
    K, V = s["K"][:, row].float()[None], s["V"][:, row].float()[None]
    cache, first, vis, begin = (torch.tensor([s[k][c] for c in ids], device=DEV)[:, None] for k in ("cache", "first", "vis", "begin"))
    t = torch.arange(len(row), device=DEV)
    place = torch.where(t >= first, cache + t - first, -1)  # [chunks, rows]: where a plain row stands in a chunk's order
    if case["op"] == "kv8":
        table = s["table"] if case["shared"] else s["table"][ids]
        width = table.shape[1] * case["page"]
        kc, ks, vc, vs = s["pool"]
        at = table.clamp(min=0).long()
        k, v = (_values(c[at], z[at]).transpose(1, 2).flatten(2, 3) for c, z in ((kc, ks), (vc, vs)))
        B = len(k)
        K, V = (torch.cat([a, b.expand(B, -1, -1, -1)], 2) for a, b in ((k, K), (v, V)))
        j = torch.arange(width, device=DEV)
        place = torch.cat([torch.where(j < cache, j, -1), place], 1)
    seen = (place >= 0) & (place < vis) & ((place < case["sink"]) | (place >= begin))
    lo, rows = ids[0] * n_c, len(ids) * n_c
    q = s["Q"][:, lo:lo + rows].float().view(H_kv, group, len(ids), n_c, d).permute(2, 0, 1, 3, 4).reshape(len(ids), H_kv, group * n_c, d)
    S = (q / math.sqrt(d)) @ K.transpose(-1, -2)
    S.masked_fill_(~seen[:, None, None], -math.inf)
    P = S.sub_(S.amax(-1, keepdim=True)).exp_()
    out = (P @ V) / P.sum(-1, keepdim=True)
    O = s["O"].clone()
    O[:, lo:lo + rows] = out.view(len(ids), H_kv, group, n_c, d).permute(1, 2, 0, 3, 4).reshape(case["H_q"], rows, d).to(O.dtype)
    return O


# ------------------------------------------------------------------------------------------------ the library's calls

_kept = {}


def _library():
    """The package and a context of it, which a program creates once."""
    if not _kept:
        import paper_2602_10825_b200 as fc
        _kept["fc"], _kept["ctx"] = fc, fc.Context(torch.cuda.current_device())
    return _kept["fc"], _kept["ctx"]


def _pages(s):
    """What a pass over the pages leaves: tables, counts, and the pool."""
    kc, ks, vc, vs = s["pool"]
    return {"table": s["table"], "ref": s["ref"], "k": kc.view(E4M3), "k_scales": ks, "v": vc.view(E4M3), "v_scales": vs}


def run(s):
    case, op = s["case"], s["case"]["op"]
    if not own:
        if op == "append":
            kc, ks, vc, vs = s["pool"]
            return _plain_append(s, s["K"], kc, ks, s["K"].dtype), _plain_append(s, s["V"], vc, vs, s["V"].dtype)
        if op in ("branch", "compact"):
            (_plain_branch if op == "branch" else _plain_compact)(s)
            return _pages(s)
        return _plain_attention(s)
    fc, ctx = _library()
    if op == "span":
        return ctx.chunk_attention_span(s["Q"], s["K"], s["V"], s["off"], s["vis"], *s["segments"], s["ids"], s["n_active"], s["O"],
                                        n_sink=case["sink"], kv_begin=s["begin"])
    pool = fc.Kv8Pool(*s["pool"])
    if op == "append":
        ctx.kv8_append(s["K"], s["V"], pool, s["table"], s["pos"], s["off"])
        return ctx.kv8_unpack(pool, s["table"], s["first"], s["rows"], K_dst=s["K_dst"], V_dst=s["V_dst"])
    if op == "branch":
        s["ref"].copy_(s["ref0"])
        s["table"].copy_(s["table0"])
        ctx.pages_fork(pool, s["ref"], s["table"], s["src"], s["dst"], s["tokens"])
        ctx.pages_take(s["ref"], s["table"], *s["grow"])
        ctx.pages_drop(s["ref"], s["table"], *s["gone"])
        return _pages(s)
    if op == "compact":
        s["ref"].copy_(s["ref0"])
        s["table"].copy_(s["table0"])
        ctx.pages_compact(pool, s["ref"], s["table"])
        return _pages(s)
    K, V = (s["K"], s["V"]) if case["win"] else (None, None)
    return ctx.chunk_attention_kv8(s["Q"], pool, s["table"], s["cache"], K, V, s["off"], s["vis"], s["ids"], s["n_active"], s["O"],
                                   n_sink=case["sink"], kv_begin=s["begin"], window_first=s["first"])


# ------------------------------------------------------------------------------------------------ 64 bits

def _exact_values(codes, scales):
    """Values of blocks [..., rows, d] from the bits of their codes: sign, exponent, three bits of a mantissa."""
    b = codes.view(torch.uint8).long()
    e, m = b // 8 % 16, b % 8
    v = torch.ldexp((m + torch.where(e > 0, 8, 0)).double(), torch.where(e > 0, e, 1) - 10)
    return torch.where(b >= 128, -v, v) * scales[..., None, None].double()


def _exact_scale(a):
    m, e = torch.frexp(a.double() / 448)
    s = torch.ldexp(torch.ceil(m * 16) / 16, e).clamp(2.0 ** -117, 2.0 ** 119)
    return torch.where(a > 0, s, torch.zeros_like(s))


def _exact_rounded(x, s):
    """x as multiples of s rounded to a number of four significant bits, none of them below 2^-9."""
    y = x / torch.where(s > 0, s, torch.ones_like(s))
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), e.clamp(min=-5) - 4)
    return (torch.round(y / step) * step).clamp(-448, 448) * s


def _exact_append(s, x, codes, scales):
    case, out = s["case"], []
    page, n = case["page"], case["n"]
    for c, p in enumerate(s["pos"]):
        rows, off = x[:, c * n:(c + 1) * n].double(), p % page
        at = int(s["table"][c, p // page])
        for r0 in range(-off, n, page):
            new = rows[:, max(r0, 0):min(r0 + page, n)]
            scale = _exact_scale(new.abs().amax((1, 2)))
            if r0 < 0:
                scale = torch.maximum(scale, scales[at].double())
                new = torch.cat([_exact_values(codes[at], scales[at])[:, :off], new], 1)
            out.append(_exact_rounded(new, scale[:, None, None]))
    return torch.cat(out, 1)


def _exact_pages(s):
    """The pages as lists: what each call does, one page after the other."""
    case, page = s["case"], s["case"]["page"]
    ref, table = s["ref0"].tolist(), s["table0"].tolist()
    moves = []
    if case["op"] == "branch":
        for c, src, n in zip(s["dst"], s["src"], s["tokens"]):
            table[c] = table[src][:n // page] + [-1] * (len(table[c]) - n // page)
            for p in table[src][:n // page]:
                ref[p] += 1
        for c, src, n in zip(s["dst"], s["src"], s["tokens"]):
            if n % page:
                moves.append((table[src][n // page], ref.index(0)))
                table[c][n // page] = moves[-1][1]
                ref[moves[-1][1]] = 1
        for c in range(1, case["W"] + 1):
            for i in range(s["grow"][0][c], s["grow"][1][c]):
                table[c][i] = ref.index(0)
                ref[table[c][i]] = 1
        for i in range(s["gone"][0][0], s["gone"][1][0]):
            if i < len(table[0]) and table[0][i] >= 0:
                ref[table[0][i]] -= 1
                table[0][i] = -1
    else:
        n = sum(r > 0 for r in ref)
        moves = list(zip([p for p in range(n, len(ref)) if ref[p]], [p for p in range(n) if not ref[p]]))
        place = dict(moves)
        table = [[place.get(p, p) for p in row] for row in table]
        for of, to in moves:
            ref[to], ref[of] = ref[of], 0
    pool = [x.clone() for x in s["pool"]]
    if moves:
        of, to = (torch.tensor(x, device=DEV) for x in zip(*moves))
        for x, y in zip(pool, s["pool"]):
            x[to] = y[of]
    one = torch.ones((1, 1), device=DEV)
    return {"table": torch.tensor(table, dtype=torch.int32, device=DEV), "ref": torch.tensor(ref, dtype=torch.int32, device=DEV),
            "k": _exact_values(pool[0], one), "k_scales": pool[1].double(), "v": _exact_values(pool[2], one), "v_scales": pool[3].double()}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s, s["K"], s["pool"][0], s["pool"][1]), _exact_append(s, s["V"], s["pool"][2], s["pool"][3])
    if case["op"] in ("branch", "compact"):
        return _exact_pages(s)
    out, n_c, group = s["O"].double(), case["n_c"], case["H_q"] // case["H_kv"]
    log, phys = s["segments"]
    for c in _active(case):
        n, first, vis, begin, sink = s["cache"][c], s["first"][c], s["vis"][c], s["begin"][c], case["sink"]
        logical = list(range(min(sink, vis))) + list(range(max(begin, sink), vis))  # the chunk's tokens, in order
        paged = [j for j in logical if j < n]
        plain = []
        for j in logical[len(paged):]:
            t = j - n + first
            i = max(k for k in range(len(phys)) if log[k] <= t)
            plain.append(phys[i] + t - log[i])
        plain = torch.tensor(plain, dtype=torch.long, device=DEV)
        if paged:
            rows = torch.tensor(paged, device=DEV)
            at = s["table"][0 if case["shared"] else c].long()[rows // case["page"]]
        for hk in range(case["H_kv"]):
            K, V = s["K"][hk, plain].double(), s["V"][hk, plain].double()
            if paged:
                kc, ks, vc, vs = s["pool"]
                k, v = (_exact_values(x[at, hk, rows % case["page"]][:, None], z[at, hk])[:, 0] for x, z in ((kc, ks), (vc, vs)))
                K, V = torch.cat([k, K]), torch.cat([v, V])
            for h in range(hk * group, (hk + 1) * group):
                logits = s["Q"][h, c * n_c:(c + 1) * n_c].double() @ K.T * case["d"] ** -0.5
                out[h, c * n_c:(c + 1) * n_c] = torch.softmax(logits, -1) @ V
    return out
