"""The operators of the 8-bit paged KV cache as cases to time and check.

The cache holds keys and values in pages of `page` token slots (a multiple of
32).  A tile is 32 slots of one page and KV head; it stores e4m3 numbers and,
for the keys and for the values, one exponent: a stored x stands for x * 2^e.
One layer's pool is four tensors,

    k      e4m3 [pages][Hkv][page / 32][dh / 16][32][16]   (chunk of 16 dims, slot, dim)
    v      e4m3 [pages][Hkv][page / 32][dh][32]            (dim, slot)
    k_exp  int8 [pages][Hkv][page / 32]
    v_exp  int8 [pages][Hkv][page / 32]

and slot s of sequence b lies in page table[b][s // page].

append: sequence b's new rows (all of them in order, or those that `path`
names) go to the slots from lengths[b] on, the keys rotated by their slot's
angle on the way.  A tile's exponent is the smallest that holds its new rows
(largest finite magnitude at most 448 * 2^e, at least -110) and is never below
the one that its earlier slots have; where it rises, those are rounded again.

attention: up to 64 query nodes per sequence see the cached slots, within a
window and the first `sinks` slots where there is a window, and the nodes of
their own root path (bits of `anc`), whose keys and values are not cached yet.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
E_MIN = -110
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}

# n_q_heads, n_kv_heads, head_dim, rotary base: the framework's model shapes
SHAPES = {
    "tiny": (4, 4, 64, 1e4),
    "small-gqa": (8, 2, 128, 5e5),
    "llama2-7b": (32, 32, 128, 1e4),
    "llama3-8b": (32, 8, 128, 5e5),
}


def listed():
    return [
        # Plain decoding of one conversation: the smallest call there is.
        dict(name="append-token", kind="append", shape="llama3-8b", batch=1, length=2077, spread=0, rows=1, path=0,
             rope=1, dtype="bf16", page=64),
        # A serving batch commits what its verified trees had accepted: up to 7 of 64 rows each, rotated before.
        dict(name="append-accepted", kind="append", shape="llama3-8b", batch=16, length=2048, spread=1, rows=7, path=64,
             rope=0, dtype="f32", page=64),
        # The chunks of eight prompts at different points, on a model with 64-wide heads.
        dict(name="append-ragged", kind="append", shape="tiny", batch=8, length=1800, spread=1, rows=777, path=0, rope=1,
             dtype="f16", page=32),
        # A long document's prompt.
        dict(name="append-prompt", kind="append", shape="llama3-8b", batch=1, length=0, spread=0, rows=30011, path=0,
             rope=1, dtype="bf16", page=64),
        # Plain decoding over a cached prompt.
        dict(name="decode-b1", kind="attention", shape="llama3-8b", batch=1, length=2077, spread=0, nodes=1, tree=0,
             window=0, sinks=0, dtype="bf16", page=64),
        # A serving batch that verifies two drafted tokens per conversation.
        dict(name="chain-b16", kind="attention", shape="llama3-8b", batch=16, length=2048, spread=1, nodes=3, tree=0,
             window=0, sinks=0, dtype="bf16", page=64),
        # Plain decoding of many long conversations: reading the cache is all there is.
        dict(name="decode-b32-long", kind="attention", shape="llama3-8b", batch=32, length=16384, spread=1, nodes=1,
             tree=0, window=0, sinks=0, dtype="bf16", page=64),
        # The paper's tree (60 drafts, depth 6) over one conversation.
        dict(name="tree", kind="attention", shape="llama3-8b", batch=1, length=2048, spread=0, nodes=61, tree=1,
             window=0, sinks=0, dtype="bf16", page=64),
        # The same tree in 32-bit activations, on a model without grouped heads.
        dict(name="tree-mha-f32", kind="attention", shape="llama2-7b", batch=1, length=1024, spread=0, nodes=61, tree=1,
             window=0, sinks=0, dtype="f32", page=128),
        # Trees over long contexts in a batch: the largest call.
        dict(name="tree-long-batch", kind="attention", shape="llama3-8b", batch=8, length=16384, spread=0, nodes=61,
             tree=1, window=0, sinks=0, dtype="bf16", page=64),
        # Plain decoding with a window and four first tokens that stay.
        dict(name="window-decode", kind="attention", shape="llama3-8b", batch=16, length=30011, spread=1, nodes=1,
             tree=0, window=4096, sinks=4, dtype="f16", page=64),
        # A smaller tree under a short window over a long conversation.
        dict(name="window-tree", kind="attention", shape="small-gqa", batch=4, length=30011, spread=1, nodes=27, tree=1,
             window=1000, sinks=4, dtype="bf16", page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    shape = rng.choice(["tiny", "small-gqa", "llama2-7b", "llama3-8b", "llama3-8b", "llama3-8b"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    page = rng.choice([32, 64, 64, 96, 128])
    hkv = SHAPES[shape][1]
    if rng.random() < 0.3:
        path = rng.choice([0, 0, 0, 64])
        batch = rng.choice([1, 1, 2, 3, 5, 8, 16])
        rows = rng.randint(1, 7) if path else _log_int(rng, 1, max(2, 30000 * 8 // (batch * max(8, hkv))))
        return dict(kind="append", shape=shape, batch=batch, length=_log_int(rng, 1, 4000) - 1,
                    spread=int(batch > 1 and rng.random() < 0.7), rows=rows, path=path, rope=int(rng.random() < 0.7),
                    dtype=dtype, page=page)
    batch = rng.choice([1, 1, 2, 3, 4, 8, 13, 16, 32])
    if batch > 8 or rng.random() < 0.4:
        nodes, tree = rng.randint(1, 7), int(rng.random() < 0.3)
    else:
        nodes, tree = rng.randint(5, 64), int(rng.random() < 0.9)
    # at most the largest listed cases' cached slots times heads, and products
    most = min(32000, 32 * 11000 * 8 // (batch * max(8, hkv)), 8 * 61 * 16384 * 8 // (batch * nodes * max(8, hkv)))
    window = rng.choice([0, 0, _log_int(rng, 64, 8000)])
    return dict(kind="attention", shape=shape, batch=batch, length=_log_int(rng, 8, most),
                spread=int(batch > 1 and rng.random() < 0.7), nodes=nodes, tree=tree, window=window,
                sinks=rng.choice([0, 4, 17]) if window else 0, dtype=dtype, page=page)


# --------------------------------------------------------------------- inputs

def _lengths(case):
    """Cached slots per sequence: all `length`, or spread over an eighth of it up to it."""
    b, n = case["batch"], case["length"]
    if not case["spread"]:
        return [n] * b
    lo = n // 8
    return [lo + (n - lo) * ((5 * i + 3) % b) // (b - 1) for i in range(b)]


def _counts(case, most):
    """Rows per sequence: all, or every third sequence's fewer."""
    return [most if not case["spread"] or i % 3 else max(1, most - 1 - i % 5) for i in range(case["batch"])]


def _capacity(case):
    """Pages of each sequence's table."""
    longest = case["length"] + (case["rows"] if case["kind"] == "append" else 0)
    return max(1, -(-longest // case["page"]))


def _pool(gen, pages, hkv, dh, page):
    """A pool in use: every tile holds numbers of its own size, rounded as the cache rounds them."""
    tiles = (pages, hkv, page // 32)

    def one(shape):
        x = torch.randn(tiles + shape, generator=gen, device=DEV)
        x *= torch.exp2(torch.rand(tiles, generator=gen, device=DEV) * 2 - 1)[..., None, None]
        e = _exponent(x.abs().flatten(3).amax(-1))
        return torch.ldexp(x, -e[..., None, None]).to(E4M3), e.to(torch.int8)

    k, ke = one((32, dh))
    k = k.view(torch.uint8).view(*tiles, 32, dh // 16, 16).transpose(-3, -2).contiguous().view(E4M3)
    v, ve = one((dh, 32))
    return k, v, ke, ve


def _exponent(amax):
    """The smallest e with amax <= 448 * 2^e (448 = 0.875 * 2^9), at least E_MIN."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.875, x - 9, x - 8)
    return torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp_min(E_MIN)


def _trees(case, seed):
    """Ancestor-or-self bits of every node: a chain, or a random tree of depth 6."""
    rng, n = np.random.default_rng(seed), case["nodes"]
    anc = np.zeros((case["batch"], n), dtype=np.uint64)
    for b in range(case["batch"]):
        parent = [-1] + [i - 1 for i in range(1, n)]
        if case["tree"] and n > 1:
            edge = sorted(1 + int(x) for x in rng.choice(n - 1, size=min(6, n - 1), replace=False))
            edge[0] = 1
            edge.append(n)
            for d in range(len(edge) - 1):
                lo, hi = (0, 1) if d == 0 else (edge[d - 1], edge[d])
                for i in range(edge[d], edge[d + 1]):
                    parent[i] = int(rng.integers(lo, hi))
        for i in range(n):
            anc[b, i] = (anc[b, parent[i]] if i else np.uint64(0)) | np.uint64(1 << i)
    return anc.view(np.int64)


def prepare(case, seed):
    hq, hkv, dh, base = SHAPES[case["shape"]]
    gen = torch.Generator(device=DEV).manual_seed(seed)
    batch, page, dtype = case["batch"], case["page"], DTYPES[case["dtype"]]
    cols = _capacity(case)
    pages = batch * cols + 3
    pool = _pool(gen, pages, hkv, dh, page)
    table = torch.randperm(pages, generator=gen, device=DEV)[:batch * cols].to(torch.int32).view(batch, cols)
    i32 = dict(dtype=torch.int32, device=DEV)
    st = dict(case=case, pool=pool, table=table, lengths=torch.tensor(_lengths(case), **i32))
    if case["kind"] == "append":
        rows = case["path"] or case["rows"]
        # the projections' output, of which k and v are the two last parts
        x = torch.randn((batch, rows, 2 * hkv, dh), generator=gen, device=DEV).to(dtype)
        st["k"], st["v"] = x[:, :, :hkv], x[:, :, hkv:]
        st["counts"] = torch.tensor(_counts(case, case["rows"]), **i32)
        st["path"] = None
        if case["path"]:
            order = torch.rand((batch, rows - 1), generator=gen, device=DEV).argsort(1)[:, :case["rows"] - 1]
            order = 1 + order.sort(1).values  # the root, then nodes further and further down
            st["path"] = torch.cat([torch.zeros_like(order[:, :1]) if case["rows"] > 1 else
                                    torch.zeros((batch, 1), dtype=torch.int64, device=DEV), order], 1).to(torch.int32)
        st["base"] = base if case["rope"] else None
        st["first"] = [n // 32 for n in _lengths(case)]
        return st
    n = case["nodes"]
    x = torch.randn((batch, n, hq + 2 * hkv, dh), generator=gen, device=DEV)
    x[:, :, :hq] *= 1.5
    x = x.to(dtype)
    st["q"], st["k"], st["v"] = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
    st["anc"] = torch.from_numpy(_trees(case, seed)).to(DEV) if case["tree"] else None
    st["counts"] = torch.tensor(_counts(case, n), **i32)
    st["out"] = torch.zeros((batch, n, hq, dh), dtype=dtype, device=DEV)
    return st


# ----------------------------------------------------------------------- runs

def run(st):
    if own:
        return _own(st)
    return _plain_append(st) if st["case"]["kind"] == "append" else _plain_attention(st)


def _own(st):
    import paper_2502_11018_amd as G

    case = st["case"]
    if case["kind"] == "append":
        G.paged_append(st["pool"], st["table"], st["lengths"], st["k"], st["v"], counts=st["counts"], path=st["path"],
                       rope_base=st["base"])
        return dict(zip(("k", "v", "k_exp", "v_exp"), st["pool"]))
    return G.paged_attention(st["pool"], st["table"], st["lengths"], st["q"], st["k"], st["v"], anc=st["anc"],
                             counts=st["counts"], window=case["window"], sinks=case["sinks"],
                             max_length=case["length"], out=st["out"])


def _plain_append(st):
    case, (pk, pv, ke, ve), table = st["case"], st["pool"], st["table"].long()
    hkv, dh = st["k"].shape[2:]
    tpp = case["page"] // 32
    n, m = st["lengths"].long()[:, None], st["counts"].long()[:, None]
    tiles = -(-case["rows"] // 32) + 1
    # the tiles that take new rows; past a sequence's last one, that one again
    t = torch.minimum(n // 32 + torch.arange(tiles, device=DEV), (n + m - 1) // 32)        # [B, T]
    slot = t[..., None] * 32 + torch.arange(32, device=DEV)                                 # [B, T, 32]
    j = slot - n[..., None]
    new, old = (j >= 0) & (j < m[..., None]), j < 0
    j = j.clamp(0, case["rows"] - 1)
    row = j if st["path"] is None else torch.gather(st["path"].long(), 1, j.flatten(1)).view_as(j)
    at = torch.arange(len(n), device=DEV)[:, None, None]
    k, v = st["k"][at, row].float(), st["v"][at, row].float()                               # [B, T, 32, Hkv, dh]
    if st["base"]:
        inv = st["base"] ** (-torch.arange(0, dh, 2, device=DEV, dtype=torch.float64) / dh)
        angle = slot[..., None].double() * inv
        c, s = angle.cos().float()[..., None, :], angle.sin().float()[..., None, :]
        a, b = k[..., :dh // 2], k[..., dh // 2:]
        k = torch.cat([a * c - b * s, b * c + a * s], -1)
    pg, tp = torch.gather(table, 1, t // tpp), t % tpp
    new, old = new[..., None, None], old[..., None, None]

    def put(x, held, exps):
        """x: new rows, held: the tiles' numbers, [B, T, 32, Hkv, dh] each; -> numbers and exponents."""
        need = _exponent(torch.where(new & x.isfinite(), x.abs(), 0.0).amax((2, 4)))        # [B, T, Hkv]
        had = torch.where(old.any(2)[..., 0], exps[pg, :, tp].int(), E_MIN)
        e = torch.maximum(need, had)
        q = torch.ldexp(x, -e[:, :, None, :, None]).clamp(-448, 448).to(E4M3).view(torch.uint8)
        h = torch.ldexp(held.float(), (had - e)[:, :, None, :, None]).to(E4M3).view(torch.uint8)
        exps[pg, :, tp] = e.to(torch.int8)
        return torch.where(new, q, torch.where(old, h, held.view(torch.uint8)))

    raw = pk.view(torch.uint8)
    held = raw[pg, :, tp].permute(0, 1, 4, 2, 3, 5).flatten(4).contiguous().view(E4M3)       # from [B, T, Hkv, dh/16, 32, 16]
    raw[pg, :, tp] = put(k, held, ke).unflatten(4, (dh // 16, 16)).permute(0, 1, 3, 4, 2, 5)
    raw = pv.view(torch.uint8)
    held = raw[pg, :, tp].permute(0, 1, 4, 2, 3).contiguous().view(E4M3)                     # from [B, T, Hkv, dh, 32]
    raw[pg, :, tp] = put(v, held, ve).permute(0, 1, 3, 4, 2)
    return dict(zip(("k", "v", "k_exp", "v_exp"), st["pool"]))


def _plain_attention(st):
    case, (pk, pv, ke, ve) = st["case"], st["pool"]
    q, k, v = (st[x].float().transpose(1, 2) for x in ("q", "k", "v"))                      # [B, heads, N, dh]
    batch, hq, nodes, dh = q.shape
    hkv = k.shape[1]
    pages = st["table"][:, :-(-case["length"] // case["page"])].long()
    # the caches as [B, Hkv, slots, dh]
    ck = pk[pages].float() * torch.exp2(ke[pages].float())[..., None, None, None]
    ck = ck.permute(0, 2, 1, 3, 5, 4, 6).reshape(batch, hkv, -1, dh)
    cv = pv[pages].float() * torch.exp2(ve[pages].float())[..., None, None]
    cv = cv.permute(0, 2, 1, 3, 5, 4).reshape(batch, hkv, -1, dh)
    anc = st["anc"]
    node = torch.arange(nodes, device=DEV)
    if anc is None:
        sees = (node[:, None] >= node).expand(batch, nodes, nodes)
    else:
        sees = (anc[..., None] >> node & 1).bool()                                          # [B, N, N]
    length = st["lengths"].long()[:, None, None]
    at = length[..., 0] + (sees & (node[:, None] != node)).sum(-1)                          # [B, N]
    slot = torch.arange(ck.shape[2], device=DEV)
    cached = (slot < length).expand(batch, nodes, -1)
    if case["window"]:
        cached = cached & ((at[..., None] - slot < case["window"]) | (slot < case["sinks"]))
        place = length + sees.cumsum(-1) - 1                                                # of a seen node
        sees = sees & ((at[..., None] - place < case["window"]) | (place < case["sinks"]))
    mask = torch.cat([cached, sees], -1)[:, None, None]                                     # [B, 1, 1, N, keys]
    q = q.reshape(batch, hkv, -1, dh)                                                       # the group's heads' rows
    s = torch.cat([q @ ck.transpose(-1, -2), q @ k.transpose(-1, -2)], -1) * dh ** -0.5
    s = s.view(batch, hkv, hq // hkv, nodes, -1).masked_fill_(~mask, -math.inf)
    s -= s.amax(-1, keepdim=True).clamp_min(-3e38)
    p = s.exp_().view(batch, hkv, -1, s.shape[-1])
    z = p.sum(-1, keepdim=True)
    o = (p[..., :len(slot)] @ cv + p[..., len(slot):] @ v) / z.clamp_min(1e-30)
    o = o.view(batch, hq, nodes, dh).transpose(1, 2).to(st["out"].dtype)
    live = node < st["counts"][:, None]
    return torch.where(live[..., None, None], o, st["out"])


# ----------------------------------------------------------- what it must move

def work(case):
    hq, hkv, dh, _ = SHAPES[case["shape"]]
    size = SIZES[case["dtype"]]
    if case["kind"] == "append":
        rows = sum(_counts(case, case["rows"]))
        tiles = sum(-(-(n % 32 + c) // 32) for n, c in zip(_lengths(case), _counts(case, case["rows"])))
        return dict(bytes=2 * rows * hkv * dh * (size + 1) + 2 * tiles * hkv, flops=(6 * case["rope"] + 4) * rows * hkv * dh)
    slots = keys = rows = 0
    depth = case["nodes"] if not case["tree"] else min(7, case["nodes"])
    for n, c in zip(_lengths(case), _counts(case, case["nodes"])):
        seen = n if not case["window"] else min(n, case["window"] + case["sinks"])
        slots += seen
        rows += c
        keys += c * (seen + (depth + 1) / 2)
    return dict(bytes=2 * slots * hkv * (dh + 1 / 32) + 2 * rows * (hq + hkv) * dh * size, flops=4 * keys * hq * dh)


# ------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return _exact_append(st) if case["kind"] == "append" else _exact_attention(st)


def _exact_append(st):
    """Every stored number before its one rounding to 8 bits, in units of its tile's exponent."""
    case, (pk, pv, ke, ve) = st["case"], st["pool"]
    dh, page = st["k"].shape[3], case["page"]
    out_k, out_v = pk.double(), pv.double()
    half = torch.arange(dh // 2, device=DEV, dtype=torch.float64)
    for b, (n, m) in enumerate(zip(_lengths(case), _counts(case, case["rows"]))):
        src = list(range(m)) if st["path"] is None else st["path"][b, :m].tolist()
        k, v = st["k"][b, src].double(), st["v"][b, src].double()
        if st["base"]:
            w = torch.arange(n, n + m, device=DEV, dtype=torch.float64)[:, None] * torch.exp(-2 * half / dh * math.log(st["base"]))
            z = torch.polar(torch.ones_like(w), w)[:, None]
            z = z * torch.complex(k[..., :dh // 2].contiguous(), k[..., dh // 2:].contiguous())
            k = torch.cat([z.real, z.imag], -1)
        table = st["table"][b].tolist()
        for t in range(n // 32, (n + m - 1) // 32 + 1):
            lo, hi = max(n, 32 * t), min(n + m, 32 * t + 32)
            page_at, tile, had, end = table[32 * t // page], t % (page // 32), max(0, n - 32 * t), hi - 32 * t
            for x, out, exps, keys in ((k, out_k, ke, True), (v, out_v, ve, False)):
                rows = x[lo - n:hi - n]                                                     # [r, Hkv, dh]
                top = rows.abs().amax((0, 2))
                e = torch.where(top > 0, torch.ceil(torch.log2(top / 448)), E_MIN).clamp_min(E_MIN)
                was = exps[page_at, :, tile].double()
                if had:
                    e = torch.maximum(e, was)
                place = out[page_at, :, tile]                                               # [Hkv, dh/16, 32, 16] or [Hkv, dh, 32]
                y = (rows * torch.exp2(-e)[:, None]).permute(1, 2, 0)                       # [Hkv, dh, r]
                shift = torch.exp2(was - e)
                if keys:
                    place[:, :, :had] *= shift[:, None, None, None]
                    place[:, :, end - len(rows):end] = y.unflatten(1, (dh // 16, 16)).transpose(-1, -2)
                else:
                    place[:, :, :had] *= shift[:, None, None]
                    place[:, :, end - len(rows):end] = y
    return dict(k=out_k, v=out_v, k_exp=None, v_exp=None)


def _exact_attention(st):
    case, (pk, pv, ke, ve) = st["case"], st["pool"]
    hq, dh = st["q"].shape[2:]
    hkv, page = st["k"].shape[2], case["page"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    anc = None if st["anc"] is None else st["anc"].cpu().numpy().view(np.uint64)
    for b, (n, count) in enumerate(zip(_lengths(case), _counts(case, case["nodes"]))):
        s = torch.arange(n, device=DEV)
        pg, tile, at = st["table"][b].long()[s // page], s % page // 32, s % 32
        seen = np.zeros((count, n + count), dtype=bool)
        for i in range(count):
            up = [j for j in range(i + 1) if anc is None or int(anc[b, i]) >> j & 1]
            pos = n + len([j for j in up if j != i])
            for r, x in [(x, x) for x in range(min(n, case["sinks"]))] + [(n + r, n + j) for r, j in enumerate(up)]:
                seen[i, x] = not case["window"] or pos - r < case["window"] or r < case["sinks"]
            seen[i, (max(0, pos - case["window"] + 1) if case["window"] else 0):n] = True
        seen = torch.from_numpy(seen).to(DEV)
        for h in range(hkv):
            key = pk[pg, h, tile, :, at].double().flatten(1) * torch.exp2(ke[pg, h, tile].double())[:, None]
            val = pv[pg, h, tile, :, at].double() * torch.exp2(ve[pg, h, tile].double())[:, None]
            key = torch.cat([key, st["k"][b, :count, h].double()])
            val = torch.cat([val, st["v"][b, :count, h].double()])
            for g in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                w = (st["q"][b, :count, g].double() @ key.T / math.sqrt(dh)).masked_fill(~seen, -math.inf)
                out[b, :count, g] = torch.softmax(w, -1) @ val
    return out
