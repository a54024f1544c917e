"""The 8-bit paged cache on the CPU: its fp64 definition against hand-worked
values, and what the entry points refuse (nothing is launched)."""

import struct

import numpy as np
import pytest
import torch

import oracle.paged as OP


def test_e4m3_numbers_and_rounding():
    assert OP.E4M3[-1] == 448.0 and OP.E4M3[1] == 2.0**-9 and len(OP.E4M3) == 127
    x = np.array([448.0, 1e9, -1e9, 17.0, 19.0, 17.001, 2.0**-10, 2.0**-10 * 1.01, np.nan, np.inf])
    want = [448.0, 448.0, -448.0, 16.0, 20.0, 18.0, 0.0, 2.0**-9, np.nan, 448.0]
    np.testing.assert_array_equal(OP.e4m3_round(x), want)
    z = torch.randn(4096) * 50
    np.testing.assert_array_equal(OP.e4m3_round(z.double().numpy()), z.to(torch.float8_e4m3fn).double().numpy())


def test_tile_exponents():
    e = lambda *x: OP.tile_exponent(np.array(x))  # noqa: E731
    assert e(448.0) == 0 and e(448.0001) == 1 and e(224.0) == -1 and e(0.0) == -110 and e(np.nan, -3.5, np.inf) == -7


def test_append_keeps_and_raises_exponents():
    c = OP.empty(2, 1, 32, 2)
    OP.append(c, [1, 0], 0, np.array([[[1.0, 2.0]]]), np.array([[[1.0, 1.0]]]))
    assert c["k_exp"][1, 0, 0] == -7 and list(c["k"][1, 0, 0]) == [128.0, 256.0]
    OP.append(c, [1, 0], 1, np.array([[[0.5, 14.0]]]), np.array([[[1.0, 1.0]]]))
    assert c["k_exp"][1, 0, 0] == -5 and list(c["k"][1, 0, 0]) == [32.0, 64.0] and list(c["k"][1, 0, 1]) == [16.0, 448.0]
    OP.append(c, [1, 0], 2, np.full((31, 1, 2), 0.25), np.zeros((31, 1, 2)))
    assert c["k_exp"][1, 0, 0] == -5 and c["k_exp"][0, 0, 0] == -10 and c["v_exp"][0, 0, 0] == -110
    k, _ = OP.read(c, [1, 0], 33)
    np.testing.assert_array_equal(k[0, :3], [[1.0, 2.0], [0.5, 14.0], [0.25, 0.25]])
    assert list(k[0, 32]) == [0.25, 0.25]


def test_visible_slots_of_a_window():
    sees = OP.visible(10, [0b1, 0b11, 0b101], window=4, sinks=2)
    at = lambda i: [int(x) for x in np.nonzero(sees[i])[0]]  # noqa: E731
    assert at(0) == [0, 1, 7, 8, 9, 10] and at(1) == [0, 1, 8, 9, 10, 11] and at(2) == [0, 1, 8, 9, 10, 12]
    assert OP.visible(3, [0, 0b11]).tolist() == [[True] * 3 + [False] * 2, [True] * 5]


def test_attention_is_the_verify_passes():
    """Without a window it is the tree attention of the target's pass."""
    from oracle.verify import ancestor_matrix, tree_attention
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 5, 4, 16))
    k, v = k[:, :2], v[:, :2]
    ck, cv = rng.standard_normal((2, 2, 7, 16))
    vis = ancestor_matrix(np.array([-1, 0, 0, 1, 3]))
    anc = [sum(1 << j for j in range(5) if vis[i, j]) for i in range(5)]
    o, mag, top = OP.attention(q, k, v, ck, cv, OP.visible(7, anc))
    full = np.concatenate([np.ones((5, 7), dtype=bool), vis], 1)
    np.testing.assert_allclose(o, tree_attention(q, k, v, ck, cv, full), rtol=1e-12)
    assert (mag >= np.abs(o) - 1e-12).all() and top > 0


# -------------------------------------------------------------- what is refused

def _lib():
    from paper_2502_11018_amd import _native as N
    return N


POOL = dict(k=64, v=64, ke=1, ve=1, n=4, page=64, heads=2, dh=128)


def append_args(**kw):
    from paper_2502_11018_amd.paged import _APPEND
    a = dict(POOL, table=4, lens=4, counts=0, path=0, status=0, kd=64, ks=(512, 256, 128), vd=64, vs=(512, 256, 128),
             base=0.0, stride=2, cols=2, pstride=0, b=1, rows=2, new=2, dtype=0)
    a.update(kw)
    return _APPEND(*(a[x] for x in ("k", "v", "ke", "ve", "n", "page", "heads", "dh", "table", "lens", "counts", "path", "status")),
                   a["kd"], *a["ks"], a["vd"], *a["vs"], a["base"],
                   *(a[x] for x in ("stride", "cols", "pstride", "b", "rows", "new", "dtype")))


@pytest.mark.parametrize("code,kw", [
    ("EINVAL", dict(k=0)), ("EINVAL", dict(v=8)), ("EINVAL", dict(table=0)), ("EINVAL", dict(lens=0)), ("EINVAL", dict(kd=0)),
    ("EINVAL", dict(vd=3)), ("EINVAL", dict(dtype=3)), ("EINVAL", dict(dtype=-1)), ("EINVAL", dict(b=0)),
    ("EINVAL", dict(rows=0)), ("EINVAL", dict(new=3)), ("EINVAL", dict(new=-1)), ("EINVAL", dict(path=4, pstride=1)),
    ("EINVAL", dict(base=-1.0)), ("EINVAL", dict(base=float("nan"))), ("EINVAL", dict(base=float("inf"))),
    ("EINVAL", dict(stride=1)), ("EINVAL", dict(cols=0)), ("EINVAL", dict(ks=(-512, 256, 128))),
    ("ESHAPE", dict(dh=96)), ("ESHAPE", dict(page=48)), ("ESHAPE", dict(page=0)), ("ESHAPE", dict(n=0)), ("ESHAPE", dict(heads=0)),
    ("ESHAPE", dict(n=1 << 30)), ("ESHAPE", dict(cols=1 << 26, stride=1 << 26)),
    ("ESHAPE", dict(b=1 << 30, new=2)),
])
def test_append_refuses(code, kw):
    N = _lib()
    assert N.lib.griffin_paged_append(append_args(**kw), None) == N.CODES["GRIFFIN_" + code]


def test_append_of_nothing_launches_nothing():
    N = _lib()
    assert N.lib.griffin_paged_append(append_args(new=0), None) == 0
    assert N.lib.griffin_paged_append(None, None) == N.CODES["GRIFFIN_EINVAL"]


def attention_args(**kw):
    from paper_2502_11018_amd.paged import _ATTENTION
    a = dict(POOL, table=4, lens=4, counts=0, anc=0, status=0, q=64, k_=64, v_=64, out=64, strides=(1024, 512, 128), scale=0.1,
             stride=2, cols=2, most=-1, b=1, nodes=2, hq=4, dtype=0, window=0, sinks=0)
    a.update(kw)
    return _ATTENTION(*(a[x] for x in ("k", "v", "ke", "ve", "n", "page", "heads", "dh", "table", "lens", "counts", "anc", "status")),
                      a["q"], *a["strides"], a["k_"], *a["strides"], a["v_"], *a["strides"], a["out"], *a["strides"], a["scale"],
                      *(a[x] for x in ("stride", "cols", "most", "b", "nodes", "hq", "dtype", "window", "sinks")))


@pytest.mark.parametrize("code,kw", [
    ("EINVAL", dict(k=0)), ("EINVAL", dict(ke=0)), ("EINVAL", dict(table=0)), ("EINVAL", dict(lens=0)), ("EINVAL", dict(q=0)),
    ("EINVAL", dict(k_=0)), ("EINVAL", dict(v_=1)), ("EINVAL", dict(out=0)), ("EINVAL", dict(dtype=7)), ("EINVAL", dict(b=0)),
    ("EINVAL", dict(window=-1)), ("EINVAL", dict(sinks=-1)), ("EINVAL", dict(scale=0.0)), ("EINVAL", dict(scale=float("nan"))),
    ("EINVAL", dict(scale=float("inf"))), ("EINVAL", dict(strides=(1024, -512, 128))), ("EINVAL", dict(stride=1)),
    ("ETREE", dict(nodes=0)), ("ETREE", dict(nodes=65)), ("ESHAPE", dict(hq=3)), ("ESHAPE", dict(hq=0)), ("ESHAPE", dict(dh=32)),
    ("ESHAPE", dict(n=0)), ("ESHAPE", dict(page=33)), ("ECAPACITY", dict(most=129)), ("ESHAPE", dict(b=1 << 24)),
    ("ESHAPE", dict(hq=1 << 20)), ("ESHAPE", dict(cols=1 << 26, stride=1 << 26)),
    ("ESHAPE", dict(b=1 << 22)), ("ESHAPE", dict(hq=1 << 18)), ("ESHAPE", dict(b=1 << 20, heads=8, hq=8)),
    ("ESHAPE", dict(b=1 << 15, nodes=64, hq=4096, heads=1, most=32)),
])
def test_attention_refuses(code, kw):
    N = _lib()
    args = attention_args(**kw)
    assert N.lib.griffin_paged_attention(args, 256, 1 << 40, None) == N.CODES["GRIFFIN_" + code]
    if not set(kw) & {"q", "k_", "v_", "out", "strides"}:
        assert N.lib.griffin_paged_attention_workspace(args) == 0


def test_attention_wants_its_workspace():
    N = _lib()
    assert N.lib.griffin_paged_attention_workspace(attention_args(most=100)) == 0  # whole sequences: none
    # 5 nodes of 4 heads on each of 2 key heads: 20 rows, which units share
    args = attention_args(most=100, nodes=5, hq=8)
    need = N.lib.griffin_paged_attention_workspace(args)
    # one unit of at most eight tiles of 32 slots: 40 rows of 128 outputs and 2 sums, and the unit's place
    assert need == 40 * 130 * 4 + 8
    assert N.lib.griffin_paged_attention(args, 256, need - 1, None) == N.CODES["GRIFFIN_ENOMEM"]
    assert N.lib.griffin_paged_attention(args, 0, need, None) == N.CODES["GRIFFIN_EINVAL"]
    assert N.lib.griffin_paged_attention(args, 264, need, None) == N.CODES["GRIFFIN_EINVAL"]
    assert N.lib.griffin_paged_attention(None, 256, need, None) == N.CODES["GRIFFIN_EINVAL"]


def test_paged_context_refuses():
    """griffin_verify_init_paged and griffin_set_pages, before any device work."""
    from ctypes import byref, c_void_p
    N = _lib()
    ctx, w = c_void_p(), N.Weights()
    desc = N.ModelDesc(2, 256, 4, 4, 64, 688, 1024, 1, 1, 1e-6, 1e4, 1, 16, 4, 192)
    init = lambda pool, window=0, sinks=0: N.lib.griffin_verify_init_paged(  # noqa: E731
        byref(desc), byref(w), byref(pool) if pool else None, window, sinks, None, byref(ctx))
    assert init(None) == N.CODES["GRIFFIN_EINVAL"]
    assert init(N.Pool(16, 16, 16, 16, 4, 64, 4, 64)) == N.CODES["GRIFFIN_EINVAL"]      # null weights
    assert N.lib.griffin_verify_init_paged(None, byref(w), byref(N.Pool(16, 16, 16, 16, 4, 64, 4, 64)), 0, 0, None,
                                           byref(ctx)) == N.CODES["GRIFFIN_EINVAL"]
    # every weight pointer set (never followed): the pool's own checks
    ptrs = (c_void_p * 2)(16, 16)
    import ctypes
    cast = ctypes.cast(ptrs, ctypes.POINTER(c_void_p))
    w = N.Weights(16, 16, 16, cast, cast, cast, cast, cast, cast, None)
    for pool, window, sinks, code in [
            (N.Pool(16, 16, 16, 16, 4, 64, 2, 64), 0, 0, "ESHAPE"),      # heads
            (N.Pool(16, 16, 16, 16, 4, 64, 4, 128), 0, 0, "ESHAPE"),     # head_dim
            (N.Pool(16, 16, 16, 16, 4, 128, 4, 64), 0, 0, "ESHAPE"),     # 192 slots are no whole pages
            (N.Pool(16, 16, 16, 16, 4, 40, 4, 64), 0, 0, "ESHAPE"),
            (N.Pool(16, 16, 16, 16, 0, 64, 4, 64), 0, 0, "ESHAPE"),
            (N.Pool(16, 8, 16, 16, 4, 64, 4, 64), 0, 0, "EINVAL"),       # alignment
            (N.Pool(16, 16, None, 16, 4, 64, 4, 64), 0, 0, "EINVAL"),
            (N.Pool(16, 16, 16, 16, 4, 64, 4, 64), -1, 0, "EINVAL"),
            (N.Pool(16, 16, 16, 16, 4, 64, 4, 64), 5, -1, "EINVAL")]:
        assert init(pool, window, sinks) == N.CODES["GRIFFIN_" + code]
        assert not ctx.value
    assert N.lib.griffin_set_pages(None, 0, 0, 0, None) == N.CODES["GRIFFIN_EINVAL"]


def test_binding_checks_tensors():
    """The Python calls refuse tensors before the library sees an address."""
    import paper_2502_11018_amd as G
    pool = G.paged_pool(2, 1, 64, 32, device="cpu")
    i32 = torch.zeros(1, dtype=torch.int32)
    table = torch.zeros(1, 2, dtype=torch.int32)
    x = torch.zeros(1, 1, 1, 64)
    with pytest.raises(ValueError, match="CUDA"):
        G.paged_append(pool, table, i32, x, x)
    with pytest.raises(ValueError, match="CUDA"):
        G.paged_attention(pool, table, i32, x, x, x)
    with pytest.raises(ValueError, match="pool"):
        G.paged_append((pool.k.view(torch.uint8),) + tuple(pool[1:]), table, i32, x, x)
    with pytest.raises(ValueError, match="contiguous and of the same"):
        G.paged_append((pool.k, pool.v[:1], pool.k_exp, pool.v_exp), table, i32, x, x)
    for bad in (dict(n_pages=0), dict(head_dim=80), dict(page=40), dict(n_kv_heads=0)):
        with pytest.raises(ValueError):
            G.paged_pool(**dict(dict(n_pages=1, n_kv_heads=1, head_dim=64, page=32, device="cpu"), **bad))


def test_struct_layouts():
    """The packed arguments have the sizes of the C structs (192 and 256 bytes)."""
    assert len(append_args()) == 192 and len(attention_args()) == 256 and struct.calcsize("@P") == 8


def test_read_refuses_what_the_table_does_not_hold():
    import torch
    from paper_2502_11018_amd import paged_pool, paged_read
    pool = paged_pool(2, 1, 64, 32, device="cpu")
    for pages, n in ([0, 1], 65), ([0, 2], 64), ([-1], 1), ([0], -1):
        with pytest.raises(ValueError):
            paged_read(pool, torch.tensor(pages, dtype=torch.int32), n)
    k, v = paged_read(pool, torch.tensor([1, 5], dtype=torch.int32), 32)  # the second page is not read
    assert k.shape == v.shape == (1, 32, 64)
    assert paged_read(pool, torch.tensor([], dtype=torch.int32), 0)[0].shape == (1, 0, 64)
