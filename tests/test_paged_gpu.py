"""The 8-bit paged cache on the GPU against its fp64 definition
(oracle/paged.py).

Tolerances, from the number formats.  Appended numbers are exact but where the
fp64 number lies within the fp32 rounding of its computation of a border
between two e4m3 numbers (then the neighbour is right too).  Attention: each
probability is off by at most eta relative, each weighted value therefore by
eta of its magnitude in the numerator and again through the denominator, and
the output by half a step of its type:
    |o - exact| <= 2 eta sum p |v| + (eps / 2) |exact| + tiny
    eta = P + ln-scale error of a score + sums
where P is fp16's half step 2^-12 (fp32 inputs: two parts, 2^-22), a score of
dh products in fp32 is off by at most dh * 2^-24 of the sum of their
magnitudes (q enters exactly, or with 22 bits), times 2 for the base-2 factor
and its fma, exp2 by 2^-22, and sums of n terms in fp32 by at most n / 32 + 64
half steps (a lane adds tiles of 16 keys, first as a tree).
"""

import numpy as np
import pytest
import torch

import oracle.paged as OP

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def same_numbers():
    torch.manual_seed(0)


@pytest.fixture(scope="module")
def G():
    import paper_2502_11018_amd as pkg
    return pkg


def make_pool(G, pages, heads, page, dh, seed=0):
    """A pool whose every byte is taken, NaN codes included, and its oracle twin."""
    rng = np.random.default_rng(seed)
    pool = G.paged_pool(pages, heads, dh, page)
    for t in (pool.k, pool.v):
        t.view(torch.uint8).copy_(torch.from_numpy(rng.integers(0, 256, t.shape, dtype=np.uint8)))
    for t in (pool.k_exp, pool.v_exp):
        t.copy_(torch.from_numpy(rng.integers(-12, -4, t.shape).astype(np.int8)))
    return pool, twin(pool)


def twin(pool):
    k, v, ke, ve = (t.cpu() for t in pool)
    p, h, t, dh = v.shape[:4]
    kn = OP.e4m3_decode(k.view(torch.uint8).numpy()).transpose(0, 1, 2, 4, 3, 5).reshape(p, h, t * 32, dh)
    vn = OP.e4m3_decode(v.view(torch.uint8).numpy()).transpose(0, 1, 2, 4, 3).reshape(p, h, t * 32, dh)
    return dict(k=kn, v=vn, k_exp=ke.numpy().astype(np.int64), v_exp=ve.numpy().astype(np.int64))


def fill(G, pool, cache, table, lengths, seed, spread=True):
    """Cache `lengths` random slots per sequence (rotated already), in both."""
    rng = np.random.default_rng(seed)
    heads, dh = pool.v.shape[1], pool.v.shape[3]
    n = max(1, max(lengths))
    size = np.exp2(rng.uniform(-2, 2, (len(lengths), n // 32 + 1, heads, 1))) if spread else 1.0
    x = rng.standard_normal((2, len(lengths), n, heads, dh))
    if spread:
        x *= np.repeat(size, 32, 1)[None, :, :n]
    x = torch.from_numpy(x).to(torch.float32)
    zero = torch.zeros(len(lengths), dtype=torch.int32, device="cuda")
    cnt = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    G.paged_append(pool, table, zero, x[0].cuda(), x[1].cuda(), counts=cnt)
    for b, m in enumerate(lengths):
        if m:
            OP.append(cache, table[b].tolist(), 0, x[0, b, :m].double().numpy(), x[1, b, :m].double().numpy())


def tables(batch, cols, pages, seed=0):
    p = np.random.default_rng(seed).permutation(pages)[: batch * cols]
    return torch.from_numpy(p.astype(np.int32).reshape(batch, cols)).cuda()


def same_cache(pool, want, raw=(), ulps=0.0):
    """Exponents and numbers equal; `raw`: unrounded numbers by name, for
    places where a border lies within `ulps` fp32 half steps."""
    got = twin(pool)
    for name in ("k_exp", "v_exp"):
        np.testing.assert_array_equal(got[name], want[name])
    for name in ("k", "v"):
        diff = ~((got[name] == want[name]) | (np.isnan(got[name]) & np.isnan(want[name])))
        if not diff.any() or not ulps:
            assert not diff.any(), f"{name}: {diff.sum()} numbers differ"
            continue
        x, y = got[name][diff], want[name][diff]
        # a neighbour of the right number, on the other side of a border the exact value is close to
        near = raw[name][diff]
        assert (np.abs(np.abs(x - near) - np.abs(y - near)) <= ulps * 2.0**-24 * np.maximum(np.abs(near), 2.0**-6)).all()


APPENDS = [  # heads, dh, page, lengths, counts
    (2, 128, 64, [0], [1]),
    (2, 128, 64, [5, 31, 32, 33], [1, 1, 1, 1]),
    (1, 64, 32, [0, 7, 63, 64], [33, 26, 1, 100]),
    (8, 128, 96, [100, 0, 17], [0, 64, 31]),
    (3, 64, 128, [127, 1], [2, 200]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", APPENDS, ids=lambda s: "-".join(map(str, s)).replace(" ", ""))
@pytest.mark.parametrize("base", [None, 10000.0, 500000.0])
def test_append_matches_its_definition(G, dtype, shape, base):
    heads, dh, page, lengths, counts = shape
    B, rows = len(lengths), max(counts)
    cols = -(-max(n + c for n, c in zip(lengths, counts)) // page)
    pool, cache = make_pool(G, B * cols + 2, heads, page, dh, seed=1)
    table = tables(B, cols, B * cols + 2)
    fill(G, pool, cache, table, lengths, 2)
    same_cache(pool, cache)
    rng = np.random.default_rng(3)
    # sizes that raise some tiles' exponents and not others'
    x = torch.from_numpy(rng.standard_normal((B, rows, 2 * heads, dh)) * np.exp2(rng.uniform(-6, 6, (B, rows, 2 * heads, 1))))
    x = x.to(DT[dtype]).cuda()
    k, v = x[:, :, :heads], x[:, :, heads:]
    G.paged_append(pool, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), k, v,
                   counts=torch.tensor(counts, dtype=torch.int32, device="cuda"), rope_base=base)
    raw = {n: cache[n].copy() for n in ("k", "v")}
    for b in range(B):
        if counts[b]:
            pages = table[b].tolist()
            r = OP.append(cache, pages, lengths[b], k[b, :counts[b]].double().cpu().numpy(),
                          v[b, :counts[b]].double().cpu().numpy(), base)
            for j in range(counts[b]):
                s = lengths[b] + j
                for name, y in zip(("k", "v"), r):
                    raw[name][pages[s // page], :, s % page] = y[j]
    # rotated: two products and a sum of inputs whose cosine and sine are off by 2 half steps each
    same_cache(pool, cache, raw, ulps=16.0 if base else 0.0)


def test_append_takes_rows_of_a_path(G):
    """Source rows in another order, each sequence's own, one twice."""
    pool, cache = make_pool(G, 6, 2, 64, 128)
    table = tables(2, 2, 6)
    fill(G, pool, cache, table, [40, 3], 5)
    k, v = torch.randn(2, 2, 64, 2, 128, device="cuda").to(torch.bfloat16)
    path = [[0, 5, 63, 5], [0, 1, 2, 3]]
    count = [4, 2]
    G.paged_append(pool, table, torch.tensor([40, 3], dtype=torch.int32, device="cuda"), k, v,
                   counts=torch.tensor(count, dtype=torch.int32, device="cuda"),
                   path=torch.tensor(path, dtype=torch.int32, device="cuda"))
    for b, n in enumerate([40, 3]):
        rows = path[b][:count[b]]
        OP.append(cache, table[b].tolist(), n, k[b, rows].double().cpu().numpy(), v[b, rows].double().cpu().numpy())
    same_cache(pool, cache)


def test_append_takes_any_strides(G):
    """Odd strides and addresses, a broadcast sequence, and v apart from k."""
    pool, cache = make_pool(G, 4, 2, 64, 64)
    table = tables(2, 2, 4)
    big = torch.randn(1 + 70 * (2 * 64 + 3), device="cuda").to(torch.float16)
    k = big[1:].view(70, 2 * 64 + 3)[:, 3:].unflatten(1, (2, 64))[None].expand(2, 70, 2, 64)
    v = torch.randn(2, 2, 70, 64, device="cuda").to(torch.float16).transpose(1, 2)
    G.paged_append(pool, table, torch.tensor([0, 9], dtype=torch.int32, device="cuda"), k, v)
    for b, n in enumerate([0, 9]):
        OP.append(cache, table[b].tolist(), n, k[b].double().cpu().numpy(), v[b].double().cpu().numpy())
    same_cache(pool, cache)


def test_append_of_what_is_not_finite(G):
    """A NaN stays one, an infinity becomes the largest number, neither moves
    the exponent; zeros give the smallest exponent; the largest and smallest
    numbers of the types have theirs."""
    pool, cache = make_pool(G, 1, 1, 96, 64)
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    x = torch.randn(96, 1, 64)
    x[3, 0, 5], x[4, 0, 6], x[5, 0, 7] = float("nan"), float("inf"), -float("inf")
    x[32:64] = 0.0
    x[64:] = 0.0
    x[64, 0, 0], x[65, 0, 0] = 3e38, 1e-40
    x = x.cuda()
    G.paged_append(pool, table, torch.zeros(1, dtype=torch.int32, device="cuda"), x[None], x[None])
    OP.append(cache, [0], 0, x.double().cpu().numpy(), x.double().cpu().numpy())
    same_cache(pool, cache)
    assert cache["k_exp"][0, 0, 1] == -110 and cache["k_exp"][0, 0, 2] == 120


def test_append_token_by_token_is_the_cache_of_its_tokens(G):
    """Forty single tokens, each a call: every call's cache is the definition's."""
    pool, cache = make_pool(G, 2, 2, 32, 64)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(0)
    for j in range(40):
        x = torch.from_numpy(rng.standard_normal((2, 1, 1, 2, 64)) * 2.0 ** rng.integers(-8, 9)).to(torch.bfloat16).cuda()
        G.paged_append(pool, table, n, x[0], x[1])
        OP.append(cache, [1, 0], j, x[0, 0].double().cpu().numpy(), x[1, 0].double().cpu().numpy())
        n += 1
        same_cache(pool, cache)


def test_append_leaves_out_what_is_out_of_range(G):
    """Bad lengths, counts, pages and rows are told and write nothing; the
    other sequences are appended."""
    st = lambda: torch.zeros(1, dtype=torch.int32, device="cuda")  # noqa: E731
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    x = torch.randn(4, 40, 1, 64, device="cuda")
    for lengths, counts, bad in (((10, -1, 129, 100), (5, 5, 0, 40), 2), ((0, 64, 0, 0), (-1, 2, 41, 0), 2)):
        pool, cache = make_pool(G, 8, 1, 64, 64)
        table, status = tables(4, 2, 8), st()
        ok = [i for i in range(4) if lengths[i] >= 0 and 0 <= counts[i] <= 40 and lengths[i] + counts[i] <= 128]
        G.paged_append(pool, table, i32(*lengths), x, x, counts=i32(*counts), status=status)
        assert status.item() == bad
        for b in ok:
            if counts[b]:
                r = x[b, :counts[b]].double().cpu().numpy()
                OP.append(cache, table[b].tolist(), lengths[b], r, r)
        same_cache(pool, cache)
    pool, cache = make_pool(G, 8, 1, 64, 64)
    status = st()
    table = i32(3, 8, -1, 5).view(2, 2)
    G.paged_append(pool, table, i32(60, 63), x[:2], x[:2], counts=i32(10, 3), status=status)
    assert status.item() == 1
    r = x.double().cpu().numpy()
    OP.append(cache, [3], 60, r[0, :4], r[0, :4])
    OP.append(cache, [None, 5], 64, r[1, 1:3], r[1, 1:3])
    same_cache(pool, cache)
    pool, cache = make_pool(G, 2, 1, 64, 64)
    status = st()
    G.paged_append(pool, i32(1).view(1, 1), i32(0), x[:1], x[:1], path=i32(0, 40, -1, 2).view(1, 4), status=status)
    assert status.item() == 4
    tile = {n: cache[n].copy() for n in ("k", "v")}
    OP.append(cache, [1], 0, r[0, [0, 0, 0, 2]], r[0, [0, 0, 0, 2]])
    for n in ("k", "v"):
        cache[n][1, :, 1:3] = tile[n][1, :, 1:3]
    same_cache(pool, cache)


# ------------------------------------------------------------------ attention

def chain(n):
    return [(1 << (i + 1)) - 1 for i in range(n)]


def tree(n, seed):
    rng = np.random.default_rng(seed)
    anc = [1]
    for i in range(1, n):
        anc.append(anc[int(rng.integers(max(0, i - 9), i))] | 1 << i)
    return anc


def bound(o, mag, top, dh, keys, dtype):
    eps = torch.finfo(DT[dtype]).eps / 2
    p = 2.0**-22 if dtype == "f32" else 2.0**-12
    eta = p + 2 * (dh + 2) * 2.0**-24 * top + 2.0**-22 + (keys / 32 + 64) * 2.0**-24
    return 2 * eta * mag + eps * np.abs(o) + 1e-30


def check(out, want, mag, top, dh, keys, dtype):
    err, most = np.abs(out - want), bound(want, mag, top, dh, keys, dtype)
    assert np.isfinite(out).all()
    assert (err <= most).all(), f"{(err / most).max():.2f} of the bound"


def run_case(G, heads, dh, page, lengths, nodes, dtype, anc=None, counts=None, window=0, sinks=0, hq=None, seed=0,
             max_length=None, spread=True):
    hq = hq or heads
    B, cols = len(lengths), max(1, -(-max(lengths) // page))
    pool, cache = make_pool(G, B * cols + 1, heads, page, dh, seed)
    table = tables(B, cols, B * cols + 1, seed)
    fill(G, pool, cache, table, lengths, seed + 1, spread)
    x = torch.randn(B, nodes, hq + 2 * heads, dh, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))
    x[:, :, :hq] *= 2
    x = x.to(DT[dtype])
    q, k, v = x.split([hq, heads, heads], 2)
    out = torch.full((B, nodes, hq, dh), 7.0, device="cuda", dtype=DT[dtype])
    masks = None
    if anc is not None:
        masks = torch.from_numpy(np.array(anc, dtype=np.uint64).view(np.int64)).cuda().reshape(B, nodes)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    G.paged_attention(pool, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), q, k, v, anc=masks,
                      counts=None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda"),
                      window=window, sinks=sinks, max_length=max_length, out=out, status=status)
    assert status.item() == 0
    got = out.double().cpu().numpy()
    for b in range(B):
        c = nodes if counts is None else counts[b]
        m = (chain(nodes) if anc is None else anc[b])[:c]
        ck, cv = OP.read(cache, table[b].tolist(), lengths[b])
        n = lambda t: t[b, :c].double().cpu().numpy()  # noqa: E731
        o, mag, top = OP.attention(n(q), n(k), n(v), ck, cv, OP.visible(lengths[b], m, window, sinks))
        check(got[b, :c], o, mag, top, dh, lengths[b] + c, dtype)
        assert (got[b, c:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("length", [0, 1, 31, 32, 33, 127, 700])
def test_one_token(G, dtype, dh, length):
    run_case(G, 2, dh, 64, [length], 1, dtype, hq=8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,hq,dh,page", [(1, 1, 64, 32), (2, 8, 128, 64), (4, 4, 64, 96), (1, 7, 128, 128)])
@pytest.mark.parametrize("nodes", [2, 5, 16, 33, 64])
def test_trees_and_chains(G, dtype, heads, hq, dh, page, nodes):
    run_case(G, heads, dh, page, [90, 257], nodes, dtype, hq=hq, anc=[tree(nodes, 1), tree(nodes, 2)])
    run_case(G, heads, dh, page, [64, 5], nodes, dtype, hq=hq)


def test_ragged_batches(G):
    """Lengths from none to long ones, counts from none to all."""
    lengths, counts = [0, 1000, 3, 64, 333, 0, 1, 2000], [3, 1, 0, 2, 3, 1, 3, 2]
    run_case(G, 2, 128, 64, lengths, 3, "bf16", hq=8, counts=counts)
    run_case(G, 2, 64, 32, lengths, 3, "f32", hq=2, counts=counts, max_length=2000)


@pytest.mark.parametrize("dtype,dh,nodes,hq", [("bf16", 128, 1, 8), ("bf16", 64, 4, 4), ("f16", 128, 3, 10), ("f32", 128, 2, 16),
                                               ("f32", 64, 16, 2), ("f16", 64, 5, 6)])
@pytest.mark.parametrize("window", [0, 900])
def test_few_rows_in_units(G, dtype, dh, nodes, hq, window):
    """At most 16 rows a key head over sequences that are cut into units: the
    bound of the lengths asks for it, the lengths go from none to many tiles."""
    run_case(G, 2, dh, 64, [0, 8, 2049, 5000, 333], nodes, dtype, hq=hq, counts=[nodes, 1, nodes, max(1, nodes - 1), 0],
             window=window, sinks=40 if window else 0, max_length=5056)


def test_more_sequences_than_lanes(G):
    rng = np.random.default_rng(1)
    run_case(G, 1, 64, 32, [int(x) for x in rng.integers(0, 90, 130)], 1, "f16", hq=4)


def test_long_sequence(G):
    """Several rounds of a wave's 64 tiles."""
    run_case(G, 1, 64, 128, [40000], 2, "bf16", hq=2)
    run_case(G, 1, 128, 64, [17001, 40], 1, "f32", hq=2)


def on_gpu(pool, table, length, q, k, v, anc, window, sinks):
    """OP.attention's results in fp64 on the GPU, for one sequence."""
    n, hq, dh = q.shape
    s = torch.arange(length, device="cuda")
    page = pool.k.shape[2] * 32
    pg, tile, at = table.long()[s // page], s % page // 32, s % 32
    sees = torch.from_numpy(OP.visible(length, anc, window, sinks)).cuda()
    o, mag, top = torch.zeros(2, n, hq, dh, dtype=torch.float64, device="cuda").unbind() + (0.0,)
    group = hq // k.shape[1]
    for h in range(k.shape[1]):
        keys = torch.ldexp(pool.k[pg, h, tile, :, at].double().flatten(1), pool.k_exp[pg, h, tile].int()[:, None])
        vals = torch.ldexp(pool.v[pg, h, tile, :, at].double(), pool.v_exp[pg, h, tile].int()[:, None])
        keys, vals = torch.cat([keys, k[:, h].double()]), torch.cat([vals, v[:, h].double()])
        for g in range(h * group, (h + 1) * group):
            x = q[:, g].double()
            p = torch.softmax((x @ keys.T * dh**-0.5).masked_fill(~sees, -torch.inf), 1)
            o[:, g], mag[:, g] = p @ vals, p @ vals.abs()
            top = max(top, float((x.abs() @ keys.abs().T).max() * dh**-0.5))
    return o.cpu().numpy(), mag.cpu().numpy(), top


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dh,hq,heads,nodes,lengths,page,window", [
    (64, 2, 1, 64, [5, 40000, 0, 33], 128, 0),         # two waves; more tiles than lookups
    (128, 8, 2, 33, [9000, 31, 64], 64, 0),            # four waves, the last one's rows partly absent
    (128, 16, 4, 61, [30000, 1], 64, 0),
    (64, 7, 1, 64, [2049, 640], 32, 0),                # several row blocks
    (128, 2, 1, 50, [12000, 100, 700], 32, 3000),
    (64, 4, 1, 61, [12000, 65, 20000], 64, 9000),
    (128, 4, 2, 45, [700, 8000, 0], 64, 0),            # four waves of 128 dims
    (128, 4, 2, 20, [5000, 33, 64], 64, 0),            # two row tiles and less: one to a workgroup
    (64, 3, 1, 17, [31, 2049, 4000], 32, 0),
    (128, 32, 16, 20, [2500, 100, 5000, 3000], 32, 1800),  # a window
    (64, 1, 1, 64, [1, 3000, 190], 64, 1000),
])
def test_many_rows(G, dtype, dh, hq, heads, nodes, lengths, page, window):
    """More rows a key head than 16, under a launch for long sequences:
    units from one tile to hundreds, full and partial, against fp64 on the GPU."""
    B, used = len(lengths), [-(-n // page) for n in lengths]
    pages = sum(used) + 1
    gen = torch.Generator("cuda").manual_seed(3)
    pool = G.paged_pool(pages, heads, dh, page)
    for t in pool[:2]:
        t.copy_((torch.randn(t.shape, generator=gen, device="cuda") * 40).clamp(-448, 448).to(t.dtype))
    for t in pool[2:]:
        t.copy_(torch.randint(-8, -4, t.shape, generator=gen, device="cuda"))
    # a table of a megaslot, whose unused entries name no page
    table = torch.full((B, (1 << 20) // page), -1, dtype=torch.int32, device="cuda")
    perm, at = torch.randperm(pages, generator=gen, device="cuda").int(), 0
    for b, n in enumerate(used):
        table[b, :n] = perm[at:at + n]
        at += n
    x = torch.randn(B, nodes, hq + 2 * heads, dh, generator=gen, device="cuda")
    x[:, :, :hq] *= 2
    q, k, v = x.to(DT[dtype]).split([hq, heads, heads], 2)
    anc = [tree(nodes, b) for b in range(B)]
    masks = torch.from_numpy(np.array(anc, dtype=np.uint64).view(np.int64)).cuda()
    counts = [nodes - 3 * b for b in range(B)]
    out = torch.full((B, nodes, hq, dh), 7.0, device="cuda", dtype=DT[dtype])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = dict(anc=masks, counts=torch.tensor(counts, dtype=torch.int32, device="cuda"), window=window, sinks=37 if window else 0)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    G.paged_attention(pool, table, lens, q, k, v, out=out, status=status, **args)
    assert status.item() == 0
    again = torch.full_like(out, 7.0)
    assert torch.equal(G.paged_attention(pool, table, lens, q, k, v, out=again, **args), out)
    got = out.double().cpu().numpy()
    for b, c in enumerate(counts):
        o, mag, top = on_gpu(pool, table[b], lengths[b], q[b, :c], k[b, :c], v[b, :c], anc[b][:c], window, args["sinks"])
        check(got[b, :c], o, mag, top, dh, lengths[b] + c, dtype)
        assert (got[b, c:] == 7.0).all()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (2, 0), (33, 0), (64, 4), (100, 40), (100, 300), (5000, 4), (7, 33)])
@pytest.mark.parametrize("nodes,dtype", [(1, "bf16"), (9, "f32"), (64, "f16")])
def test_windows(G, window, sinks, nodes, dtype):
    run_case(G, 2, 64, 32, [0, 5, 64, 301], nodes, dtype, hq=4, window=window, sinks=sinks,
             anc=[tree(nodes, s) for s in range(4)])


def test_masks_that_leave_rows_empty(G):
    """Nodes that see no node, with nothing cached and with a cache; bits
    beyond the nodes mean nothing."""
    anc = [[0, 1 << 60, 0b100, 0b11], [0, 0b1, 0b100, 0]]
    run_case(G, 1, 64, 32, [0, 40], 4, "f32", hq=2, anc=[[a & 15 for a in r] for r in anc])
    pool, _ = make_pool(G, 1, 1, 32, 64)
    x = torch.randn(1, 4, 1, 64, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    masks = torch.tensor([[0, 1 << 60, 4, 3]], device="cuda")
    for cols in (1, 2000):
        table = torch.zeros(1, cols, dtype=torch.int32, device="cuda")
        out = G.paged_attention(pool, table, zero, x, x, x, anc=masks)
        assert (out[0, :2] == 0).all() and torch.equal(out[0, 2], x[0, 2]) and out.isfinite().all()


def test_large_and_small_scores(G):
    """Scores from far below to far above one another, and values from tiny to
    huge, over several tiles: the references follow them."""
    for seed, (qs, order) in enumerate([(0.0, 1), (30.0, 1), (30.0, -1), (1e-30, 1), (1e4, 1)]):
        pool, cache = make_pool(G, 8, 1, 64, 64)
        table = tables(1, 8, 8)
        rng = np.random.default_rng(seed)
        size = np.exp2(np.linspace(-10, 6, 512))[::order, None, None]
        k = torch.from_numpy(rng.standard_normal((512, 1, 64)) * size).float().cuda()
        v = torch.from_numpy(rng.standard_normal((512, 1, 64)) * size[::-1] ** 2).float().cuda()
        zero = torch.zeros(1, dtype=torch.int32, device="cuda")
        G.paged_append(pool, table, zero, k[None], v[None])
        OP.append(cache, table[0].tolist(), 0, k.double().cpu().numpy(), v.double().cpu().numpy())
        for dtype in ("f32", "bf16"):
            x = (torch.randn(3, 1, 5, 1, 64, device="cuda") * torch.tensor([qs, 1, 1], device="cuda").view(3, 1, 1, 1, 1)).to(DT[dtype])
            out = G.paged_attention(pool, table, zero + 512, *x)
            ck, cv = OP.read(cache, table[0].tolist(), 512)
            q, k5, v5 = (t[0].double().cpu().numpy() for t in x)
            o, mag, top = OP.attention(q, k5, v5, ck, cv, OP.visible(512, chain(5)))
            check(out[0].double().cpu().numpy(), o, mag, top, 64, 517, dtype)


FORMS = [(5, 1, 1, 300), (12, 4, 1, 900), (24, 2, 1, 900), (64, 2, 1, 7000), (64, 4, 4, 16400)]  # nodes, group, batch, slots


def winner(G, nodes, group, batch, length, dtype, q0, k, v):
    """Slot 0's score far above the others': scores q0 k / 8, exact."""
    heads = 4
    pool, _ = make_pool(G, batch * -(-length // 64), heads, 64, 64)
    table = tables(batch, -(-length // 64), batch * -(-length // 64))
    zero = torch.zeros(batch, dtype=torch.int32, device="cuda")
    keys = torch.zeros(batch, length, heads, 64, device="cuda")
    keys[..., 0] = -k
    keys[:, 0, :, 0] = k
    G.paged_append(pool, table, zero, keys, v.view(1, -1, 1, 64).expand(batch, length, heads, 64).contiguous())
    q = torch.zeros(batch, nodes, heads * group, 64, device="cuda")
    own = torch.zeros(batch, nodes, heads, 64, device="cuda")
    q[..., 0] = q0
    own[..., 0] = -8 * k
    out = G.paged_attention(pool, table, zero + length, q.to(DT[dtype]), own.to(DT[dtype]), torch.zeros_like(own).to(DT[dtype]))
    return out.double().cpu()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nodes,group,batch,length", FORMS)
def test_many_small_probabilities(G, nodes, group, batch, length, dtype):
    """Weights of 2^-26 beside one of 1 still count: they stand at 2^-18 or
    above in fp16, whose steps of 2^-24 round them by 2^-7, their scores' terms
    by far less."""
    v = torch.full((length, 64), 64.0, device="cuda")
    v[0] = 0
    out = winner(G, nodes, group, batch, length, dtype, 9.0, 8.0, v)
    part = (length - 1) * np.exp(-18.0)
    tol = 2.0**-7 + 2.0**-12 + torch.finfo(DT[dtype]).eps / 2 + (2.0**-25 / (64 * part) if dtype == "f16" else 0)
    assert (out / (64 * part / (1 + part)) - 1).abs().max().item() <= tol


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes,group,batch,length", FORMS)
@pytest.mark.parametrize("spread", [20, 21])
def test_small_values_beside_large_ones(G, nodes, group, batch, length, dtype, spread):
    """The row of a slot whose tile's values are 2^-20 of other tiles' is that
    slot's: its bytes times powers of two, its weight over a sum of weights
    whose exponents near 29 are rounded by 2^-20."""
    v = torch.full((length, 64), 1.75, device="cuda")
    v[:32] = 1.75 * 2.0**-20
    i = torch.arange(64, device="cuda")  # four bits each, down to e4m3's last: exact at the tile's exponent of -28
    v[0] = (i % 16) * 2.0**-26 * torch.tensor([1, 2.0**-4, 2.0**-8, 2.0**-11], device="cuda")[i // 16]
    v[32 * (length // 64):] *= 2.0**(spread - 20)
    out = winner(G, nodes, group, batch, length, dtype, 20.0, 8.0, v)
    want = v[0].double().cpu()
    # the others' weights: exp(-40) each, values up to 3.5
    assert ((out - want).abs() <= want * (2.0**-19 + torch.finfo(DT[dtype]).eps / 2) + 3.5 * length * np.exp(-40.0)).all()


def roomy(table, cols):
    """The table with entries that name no page behind its own: the launch is
    planned for what it could hold, which chooses the kernel."""
    return torch.cat([table, table.new_full((table.shape[0], cols - table.shape[1]), -1)], 1)


@pytest.mark.parametrize("nodes,group,cols,batch", [(10, 1, 4, 1), (10, 1, 1000, 1), (10, 1, 4, 300), (40, 1, 4, 1), (40, 1, 1500, 1),
                                                    (40, 1, 4, 400), (40, 2, 5000, 1), (40, 2, 4, 2800)])
def test_nan_in_masked_places(G, nodes, group, cols, batch):
    """NaN in slots behind the cached ones, in pages outside the window, and in
    nodes that are not ancestors reaches no row; a NaN inside reaches exactly
    the rows that see it."""
    pool, cache = make_pool(G, 4, 1, 64, 64)
    table = tables(1, 4, 4)
    n, window = 200, 50
    fill(G, pool, cache, table, [n], 3, False)
    pages = table[0].tolist()
    clean = [t.clone() for t in pool]
    lens = torch.full((batch,), n, dtype=torch.int32, device="cuda")
    table = roomy(table, cols).repeat(batch, 1)  # many sequences that read the same pages
    q, k, v = torch.randn(1, nodes, group + 2, 64, device="cuda").to(torch.bfloat16).repeat(batch, 1, 1, 1).split([group, 1, 1], 2)
    want = G.paged_attention(pool, table, lens, q, k, v, window=window, sinks=2)
    # keys and values that no node sees: [2, n - window + 1) and [n, ..)
    for s in list(range(2, n - window + 1)) + list(range(n, 256)):
        pg, at = pages[s // 64], s % 64
        pool.k.view(torch.uint8)[pg, :, at // 32, :, at % 32] = 0x7f
        pool.v.view(torch.uint8)[pg, :, at // 32, :, at % 32] = 0xff
    got = G.paged_attention(pool, table, lens, q, k, v, window=window, sinks=2)
    assert torch.equal(got, want) and (got == got[:1]).all()
    # a slot that the first five nodes see
    s = n - window + 5
    pg, at = pages[s // 64], s % 64
    pool.v.view(torch.uint8)[pg, :, at // 32, 17, at % 32] = 0x7f
    got = G.paged_attention(pool, table, lens, q, k, v, window=window, sinks=2)
    assert got[:, :5, :, 17].isnan().all() and torch.equal(got[:, 5:], want[:, 5:])
    assert torch.equal(got[:, :5, :, :17], want[:, :5, :, :17])
    # nodes that are not ancestors
    for t, c in zip(pool, clean):
        t.copy_(c)
    kn, vn = k.clone(), v.clone()
    kn[:, 3] = vn[:, 3] = float("nan")
    anc = torch.tensor([[(1 << (i + 1)) - 1 & ~8 if i != 3 else 15 for i in range(nodes)]], device="cuda").repeat(batch, 1)
    ok = G.paged_attention(pool, table, lens, q, k, v, anc=anc)
    got = G.paged_attention(pool, table, lens, q, kn, vn, anc=anc)
    assert got[:, 3].isnan().all()
    keep = [i for i in range(nodes) if i != 3]
    assert torch.equal(got[:, keep], ok[:, keep])


@pytest.mark.parametrize("nodes,group,cols", [(2, 1, 3), (2, 1, 400), (20, 1, 3), (20, 1, 1500), (40, 2, 2000)])
def test_attention_tells_what_is_out_of_range(G, nodes, group, cols):
    """Bad pages and lengths give NaN rows and a status bit, for their
    sequences alone; entries of pages that no node sees are not read."""
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pool, cache = make_pool(G, 9, 1, 64, 64)
    table = tables(3, 3, 9)
    fill(G, pool, cache, table, [190, 190, 190], 0)
    table, past = roomy(table, cols), 64 * cols + 1
    x = torch.randn(3, nodes, group + 2, 64, device="cuda").split([group, 1, 1], 2)
    want = G.paged_attention(pool, table, i32(190, 190, 190), *x)
    status = i32(0)
    got = G.paged_attention(pool, table, i32(190, past, -4), *x, status=status)
    assert status.item() == 2 and torch.equal(got[0], want[0]) and got[1:].isnan().all()
    status, bad = i32(0), table.clone()
    bad[1, 1], bad[2, 2] = 9, -1
    got = G.paged_attention(pool, bad, i32(190, 190, 190), *x, status=status)
    assert status.item() == 1 and torch.equal(got[0], want[0]) and got[1:].isnan().all()
    status = i32(0)
    got = G.paged_attention(pool, table, i32(190, 190, 190), *x, counts=i32(nodes, nodes + 1, -1), status=status)
    assert status.item() == 2 and torch.equal(got[0], want[0]) and got[1].isnan().all()
    want = G.paged_attention(pool, table, i32(190, 190, 190), *x, window=20)
    bad = table.clone()
    bad[:, :2] = -7
    status = i32(0)
    assert torch.equal(G.paged_attention(pool, bad, i32(190, 190, 190), *x, window=20, status=status), want)
    assert status.item() == 0


@pytest.mark.parametrize("nodes,cols", [(5, 2), (5, 3000), (25, 2), (25, 3000), (64, 5000)])
def test_attention_takes_any_strides(G, nodes, cols):
    pool, cache = make_pool(G, 4, 2, 64, 64)
    table = tables(2, 2, 4)
    fill(G, pool, cache, table, [100, 65], 0)
    table = roomy(table, cols)
    lens = torch.tensor([100, 65], dtype=torch.int32, device="cuda")
    for dt in (torch.bfloat16, torch.float32):
        raw = torch.randn(1 + 2 * nodes * (8 * 64 + 7), device="cuda").to(dt)
        x = raw[1:].view(2, nodes, 8 * 64 + 7)[:, :, 5:5 + 8 * 64].unflatten(2, (8, 64))
        q, k, v = x[:, :, :4], x[:, :, 4:6], x[:, :, 6:]
        want = G.paged_attention(pool, table, lens, q.contiguous(), k.contiguous(), v.contiguous())
        assert torch.equal(G.paged_attention(pool, table, lens, q, k, v), want)
        wide = torch.full((2, 4, nodes, 65), 7.0, dtype=dt, device="cuda")
        out = wide[..., 1:].transpose(1, 2)
        assert torch.equal(G.paged_attention(pool, table, lens, q, k, v, out=out), want) and (wide[..., 0] == 7).all()
        two = torch.stack([table, table], 1).flatten(1)[:, :cols]  # a table with a row stride of its own
        assert torch.equal(G.paged_attention(pool, two, lens, q, k, v), want)
    # heads that share one key head's rows, and a broadcast query
    q = torch.randn(1, 1, 1, 64, device="cuda").expand(2, nodes, 4, 64)
    k = torch.randn(2, nodes, 1, 64, device="cuda").expand(2, nodes, 2, 64)
    want = G.paged_attention(pool, table, lens, q.contiguous(), k.contiguous(), k.contiguous())
    assert torch.equal(G.paged_attention(pool, table, lens, q, k, k), want)


def test_offsets_past_32_bits(G):
    """Pages whose bytes lie beyond 4 GiB of the pool."""
    heads, dh, page = 8, 128, 64
    pages = (5 << 30) // (heads * dh * page)
    pool = G.paged_pool(pages, heads, dh, page)
    small, cache = make_pool(G, 4, heads, page, dh)
    small_table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    table = torch.tensor([[pages - 1, 3], [pages - 2, pages // 2]], dtype=torch.int32, device="cuda")
    k, v = torch.randn(2, 2, 100, heads, dh, device="cuda")
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    x = torch.randn(2, 3, 16, dh, device="cuda")
    y = torch.randn(2, 2, 3, heads, dh, device="cuda")
    got = []
    for p, t in ((pool, table), (small, small_table)):
        G.paged_append(p, t, zero, k, v)
        got.append(G.paged_attention(p, t, zero + 100, x, *y))
    assert torch.equal(got[0], got[1])
    assert torch.equal(G.paged_read(pool, table[0], 100)[0], G.paged_read(small, small_table[0], 100)[0])


def test_the_same_call_gives_the_same_bits(G):
    pool, cache = make_pool(G, 40, 2, 64, 128)
    table = tables(4, 10, 40)
    fill(G, pool, cache, table, [600, 20, 333, 512], 0)
    lens = torch.tensor([600, 20, 333, 512], dtype=torch.int32, device="cuda")
    x = torch.randn(4, 30, 12, 128, device="cuda").to(torch.bfloat16)
    call = lambda: G.paged_attention(pool, table, lens, x[:, :, :8], x[:, :, 8:10], x[:, :, 10:])  # noqa: E731
    want = call()
    assert all(torch.equal(call(), want) for _ in range(5))


def decode_loop(G, pool, table, steps, prompt, x, dtype, base, window=0, sinks=0):
    """A prompt, then tokens one by one: attention, then append."""
    hq, heads = x.shape[2] - 2 * pool.k.shape[1], pool.k.shape[1]
    q, k, v = x.split([hq, heads, heads], 2)
    n = torch.zeros(x.shape[0], dtype=torch.int32, device="cuda")
    G.paged_append(pool, table, n, k[:, :prompt], v[:, :prompt], rope_base=base)
    n += prompt
    outs = []
    for j in range(prompt, prompt + steps):
        at = slice(j, j + 1)
        outs.append(G.paged_attention(pool, table, n, q[:, at], k[:, at], v[:, at], window=window, sinks=sinks))
        G.paged_append(pool, table, n, k[:, at], v[:, at], rope_base=base)
        n += 1
    return torch.cat(outs, 1)


@pytest.mark.parametrize("dtype,window", [("bf16", 0), ("f32", 0), ("f16", 48)])
def test_prompt_and_decoding_together(G, dtype, window):
    """Prompt and single tokens as they are used, every step against fp64 over
    the same 8-bit cache."""
    B, prompt, steps, heads, hq, dh = 2, 70, 30, 2, 4, 64
    pool, cache = make_pool(G, 8, heads, 32, dh)
    table = tables(B, 4, 8)
    x = torch.randn(B, prompt + steps, hq + 2 * heads, dh, device="cuda").to(DT[dtype])
    out = decode_loop(G, pool, table, steps, prompt, x, dtype, None, window, 4).double().cpu().numpy()
    q, k, v = (t.double().cpu().numpy() for t in x.split([hq, heads, heads], 2))
    for b in range(B):
        pages = table[b].tolist()
        OP.append(cache, pages, 0, k[b, :prompt], v[b, :prompt])
        for j in range(prompt, prompt + steps):
            ck, cv = OP.read(cache, pages, j)
            o, mag, top = OP.attention(q[b, j:j + 1], k[b, j:j + 1], v[b, j:j + 1], ck, cv,
                                       OP.visible(j, [1], window, 4 if window else 0))
            check(out[b, j - prompt][None], o, mag, top, dh, j, dtype)
            OP.append(cache, pages, j, k[b, j:j + 1], v[b, j:j + 1])
    same_cache(pool, cache)


def test_temporaries_on_another_stream(G):
    """What only a call on another stream still needs is not given to the next
    tensor of the caller's."""
    pool, cache = make_pool(G, 8, 2, 64, 128)
    table = tables(2, 4, 8)
    fill(G, pool, cache, table, [30, 100], 0)
    n = torch.tensor([30, 100], dtype=torch.int32, device="cuda")
    x = torch.randn(2, 16, 8, 128, device="cuda").to(torch.bfloat16)
    q, k, v = (t.contiguous() for t in x.split([4, 2, 2], 2))
    want = G.paged_attention(pool, table, n, q, k, v)
    raw = [t.view(torch.uint8) for t in pool]
    before = [t.clone() for t in raw]
    G.paged_append(pool, table, n, k, v)
    full = [t.clone() for t in raw]
    for s, t in zip(raw, before):
        s.copy_(t)
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy * 1e-3
    out = G.paged_attention(pool, table.clone(), n.clone(), q.clone(), k.clone(), v.clone(), stream=side)
    G.paged_append(pool, table.clone(), n.clone(), k.clone(), v.clone(), stream=side)
    over = [torch.zeros_like(t) for t in (table, n, q, k, v, out) for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(out, want) and not any(t.any() for t in over)
    assert all(torch.equal(s, t) for s, t in zip(raw, full))


def test_other_stream_and_captured(G):
    """The calls on a stream of their own, and captured: replays follow the
    lengths and rows that changed in place, with eager work between them."""
    pool, cache = make_pool(G, 8, 2, 64, 128)
    table = tables(2, 4, 8)
    fill(G, pool, cache, table, [30, 100], 0)
    twin_pool = G.PagedPool(*(t.clone() for t in pool))
    n = torch.tensor([30, 100], dtype=torch.int32, device="cuda")
    m = n.clone()
    x = torch.randn(2, 1, 8, 128, device="cuda").to(torch.bfloat16)
    q, k, v = x.split([4, 2, 2], 2)

    def step(p, lens):
        o = G.paged_attention(p, table, lens, q, k, v)
        G.paged_append(p, table, lens, k, v, rope_base=10000.0)
        return o

    side = torch.cuda.Stream()
    a = G.paged_attention(pool, table, n, q, k, v, stream=side)
    side.synchronize()
    assert torch.equal(a, G.paged_attention(pool, table, n, q, k, v))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(pool, n)
        n += 1
    for i in range(6):
        x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = step(twin_pool, m)
        m += 1
        assert torch.equal(got, want)
        for s, t in zip(pool, twin_pool):
            assert torch.equal(s.view(torch.uint8), t.view(torch.uint8))
