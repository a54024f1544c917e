"""Verify contexts over an 8-bit paged cache, through the C ABI, against the
fp64 oracle over the same cache: oracle/paged.py rounds the prefix, and the
nodes that a commit appends, by the cache's definition; logits, predictions and
walks are held to the gates of the other parity tests (tests/harness.py)."""

import numpy as np
import pytest
import torch

import oracle
import oracle.paged as OP
from oracle.verify import ancestor_matrix
from tests import harness as H
from workloads import gen
from workloads.configs import get_workload

pytestmark = pytest.mark.gpu

PAGE = 32


def say(msg):
    print(f"[gpu-case] {msg}", flush=True)


class Paged:
    """A target over a paged cache whose sequences' pages are scattered, and
    the oracle's caches of it."""

    def __init__(self, name, window=0, sinks=0, prefixes=None, extra=64, stream=None, max_tree=64, batch=None):
        import paper_2502_11018_amd as G
        self.G, self.w = G, get_workload(name)
        m = self.m = self.w.model
        self.prefix = list(prefixes or self.w.prefixes())[:batch]
        self.B = len(self.prefix)
        self.window, self.sinks = window, sinks
        self.mw = gen.make_weights(m, self.w.weight_seed)
        self.ow = oracle.OracleWeights(self.mw)
        cap = (max(self.prefix) + max_tree + extra + 63) // 64 * 64
        self.cols, pages = cap // PAGE, self.B * (cap // PAGE) + 3
        self.pool = G.paged_pool(pages, m.n_kv_heads, m.head_dim, PAGE, layers=m.n_layers)
        for t in self.pool[:2]:  # whatever lies in unused slots
            t.view(torch.uint8).fill_(0x7f)
        self.table = np.random.default_rng(1).permutation(pages)[: self.B * self.cols].reshape(self.B, -1)
        self.caches = [[OP.empty(pages, m.n_kv_heads, PAGE, m.head_dim) for _ in range(m.n_layers)]]
        self.stream = stream
        say(f"paged {name}: prefixes {self.prefix} window {window} cap {cap}")
        self.v = G.TreeVerifier(m, self.mw.to("cuda"), max_batch=self.B, max_tree=max_tree, max_depth=max_tree - 1,
                                kv_capacity=cap, pool=self.pool, window=window, sinks=sinks, stream=stream)
        for b, n in enumerate(self.prefix):
            self.v.set_pages(b, self.table[b])
            kv = H.prefix_kv_prefill(self.ow, np.random.default_rng(100 + b).integers(0, m.vocab, n))
            for l in range(m.n_layers):
                self.v.write_prefix(l, b, torch.from_numpy(kv.K[l]).to(torch.bfloat16).cuda(),
                                    torch.from_numpy(kv.V[l]).to(torch.bfloat16).cuda())
                OP.append(self.caches[0][l], self.table[b], 0, kv.K[l].transpose(1, 0, 2), kv.V[l].transpose(1, 0, 2))
        torch.cuda.synchronize()

    def kv(self, b):
        """The oracle's cached prefix of sequence b, per layer (K, V)."""
        return [OP.read(self.caches[0][l], self.table[b], self.prefix[b]) for l in range(self.m.n_layers)]

    def reference(self, b, tree):
        kv = self.kv(b)
        visible = None
        if self.window:
            vis = ancestor_matrix(tree.parents)
            anc = [sum(1 << j for j in range(tree.n) if vis[i, j]) for i in range(tree.n)]
            visible = OP.visible(self.prefix[b], anc, self.window, self.sinks)
        return oracle.verify_tree(self.ow, lambda l: kv[l], tree, self.prefix[b], visible)

    def commit(self, b, res, path):
        for l in range(self.m.n_layers):
            rows = [0] + list(path)
            OP.append(self.caches[0][l], self.table[b], self.prefix[b], res.tree_k[l][rows], res.tree_v[l][rows])

    def step(self, trees, logits=True):
        out = torch.full((self.B * self.v.max_tree, self.m.vocab), float("nan"), device="cuda") if logits else None
        self.v.step(self.prefix, trees, out)
        acc = self.v.accept()
        pred = self.v.predictions()
        return (out.view(self.B, self.v.max_tree, -1).cpu().numpy() if logits else None), pred, acc


def seq(tree, res):
    pred = oracle.argmax_first(res.logits)
    return H.OracleSeq(H.SeqCase(None, None, tree, [], [], []), res.logits, pred, oracle.top2_margin(res.logits),
                       oracle.accept_dfs(tree, pred), res.router_logits, res.hidden)


@pytest.mark.parametrize("name", ["tiny", "small-gqa", "small-mha", "small-moe", "small-chain2"])
def test_step_matches_oracle(name):
    p = Paged(name, max_tree=get_workload(name).max_tree)
    try:
        before = [t.view(torch.uint8).clone() for t in p.pool]
        trees = [gen.random_tree(p.w.widths_of(b), p.m.vocab, 70 + b)[0] for b in range(p.B)]
        lg, pred, acc = p.step(trees)
        for b, tree in enumerate(trees):
            o = seq(tree, p.reference(b, tree))
            skip = frozenset()
            if o.router_logits is not None:
                _, _, skip, _ = H.router_check(o, p.v.router_logits()[:, b], p.m.top_k)
            H.check_parity(o, lg[b, : tree.n], pred[b, : tree.n], acc.sequence(b), exclude=skip)
            assert np.isnan(lg[b, tree.n:]).all()
        assert all(torch.equal(t.view(torch.uint8), x) for t, x in zip(p.pool, before)), "a step wrote to the cache"
    finally:
        p.v.close()


@pytest.mark.parametrize("name,window", [("small-gqa", 0), ("small-gqa", 40), ("small-mha", 0)])
def test_steps_of_few_and_many_nodes(name, window):
    """One context's steps of 1 to max_tree nodes, mixed in a batch, on both
    sides of the launches' bounds, each against the oracle."""
    p = Paged(name, window, 4 if window else 0, max_tree=23)
    try:
        sizes = [(1,), (2,), (4,), (5,), (16,), (17,), (23,), (1, 3), (2, 20), (1,), (7, 1)]
        for k, ns in enumerate(sizes):
            trees = []
            for b in range(p.B):
                rng = np.random.default_rng(10 * k + b)
                n = ns[b % len(ns)]
                parents = sorted([int(rng.integers(max(0, i - 4), i)) for i in range(1, n)])
                t = gen.chain_tree(int(rng.integers(p.m.vocab)), rng.integers(0, p.m.vocab, n - 1).tolist())
                trees.append(type(t)(t.tokens, np.array([-1] + parents, dtype=t.parents.dtype)))
            lg, pred, acc = p.step(trees)
            for b, tree in enumerate(trees):
                H.check_parity(seq(tree, p.reference(b, tree)), lg[b, : tree.n], pred[b, : tree.n], acc.sequence(b))
                assert np.isnan(lg[b, tree.n:]).all()
    finally:
        p.v.close()


@pytest.mark.parametrize("window,sinks", [(40, 0), (70, 4), (33, 40), (4096, 4)])
def test_windowed_step_matches_oracle(window, sinks):
    """Pages that no node of the step sees are not set, and hold NaN."""
    p = Paged("small-gqa", window, sinks)
    try:
        trees = [gen.random_tree(p.w.widths_of(b), p.m.vocab, 80 + b)[0] for b in range(p.B)]
        for b in range(p.B):
            first = max(0, p.prefix[b] - window + 1) // PAGE
            kept = -(-min(sinks, p.prefix[b]) // PAGE)
            if first > kept:
                p.v.set_pages(b, [-1] * (first - kept), first=kept)
                for pg in p.table[b][kept:first]:
                    for t in p.pool[:2]:
                        t.view(torch.uint8)[:, pg] = 0x7f
        lg, pred, acc = p.step(trees)
        for b, tree in enumerate(trees):
            H.check_parity(seq(tree, p.reference(b, tree)), lg[b, : tree.n], pred[b, : tree.n], acc.sequence(b))
    finally:
        p.v.close()


@pytest.mark.parametrize("name,window", [("tiny", 0), ("small-gqa", 0), ("tiny", 90)])
def test_loop_commits_what_was_accepted(name, window):
    """Cycles of step / accept / commit on trees planted with the oracle's own
    continuation over its 8-bit cache: every cycle's logits and walk match, and
    the committed pages hold what the definition says, up to numbers that lie
    on a border between two e4m3 numbers for fp32 and fp64."""
    p = Paged(name, window, 4 if window else 0)
    try:
        rng = np.random.default_rng(5)
        roots = [7 + b for b in range(p.B)]
        moved = 0
        for cycle in range(8):
            trees, refs = [], []
            for b in range(p.B):
                tree, _ = gen.random_tree(p.w.widths_of(b), p.m.vocab, 9000 + 97 * cycle + b)
                tree.tokens[0] = roots[b]
                depth = tree.depths()
                deepest = [i for i in range(1, tree.n) if depth[i] == depth.max()]
                path = tree.root_path(deepest[int(rng.integers(len(deepest)))])
                # plant the target's own choices down the path, one node after another
                for step, node in enumerate(path[: int(rng.integers(1, len(path) + 1))]):
                    up = 0 if step == 0 else path[step - 1]
                    tree = gen.apply_plant(tree, path[: step + 1],
                                           [int(tree.tokens[x]) for x in path[:step]] +
                                           [int(oracle.argmax_first(p.reference(b, tree).logits)[up])])
                trees.append(tree)
                refs.append(p.reference(b, tree))
            say(f"{name}: cycle {cycle} prefix {p.prefix}")
            lg, pred, acc = p.step(trees)
            p.v.commit()
            for b, (tree, res) in enumerate(zip(trees, refs)):
                H.check_parity(seq(tree, res), lg[b, : tree.n], pred[b, : tree.n], acc.sequence(b))
                L, toks, path = acc.sequence(b)
                p.commit(b, res, path)
                p.prefix[b] += L + 1
                roots[b] = toks[-1]
                moved += L
        assert moved > 4
        torch.cuda.synchronize()
        for l in range(p.m.n_layers):
            for b in range(p.B):
                n = p.prefix[b]
                table = torch.from_numpy(p.table[b].astype(np.int32)).cuda()
                got = [t.double().cpu().numpy() for t in p.G.paged_read(p.G.layer_pool(p.pool, l), table, n)]
                np.testing.assert_array_equal(p.v.read_v(l, b, n).cpu().numpy(), got[1])
                for x, y in zip(got, OP.read(p.caches[0][l], p.table[b], n)):
                    # a neighbouring number, at most; few of them
                    assert (np.abs(x - y) <= np.maximum(np.abs(y) / 8, np.abs(y).max() / 448 / 64)).all()
                    assert (x != y).mean() < 0.01
    finally:
        p.v.close()


def test_commit_follows_either_acceptance():
    """After a sampled acceptance the commit appends its path."""
    p = Paged("tiny")
    try:
        tree, _ = gen.random_tree((3, 4, 2), p.m.vocab, 3)
        out = torch.empty((p.v.max_tree, p.m.vocab), device="cuda")
        p.v.step(p.prefix, [tree], out)
        u = np.full((1, p.v.max_tree), 0.0, dtype=np.float32)
        acc = p.v.accept_sampled(out, None, u, u, 1.0)   # u = 0 accepts every first child with mass
        L, _, path = acc.sequence(0)
        first, at = [], 0                                # the path of first children, down to a leaf
        while (at := next((i for i in range(1, tree.n) if int(tree.parents[i]) == at), 0)) > 0:
            first.append(at)
        assert list(path) == first and L > 0
        res = p.reference(0, tree)
        p.v.commit()
        p.commit(0, res, path)
        torch.cuda.synchronize()
        table = torch.from_numpy(p.table[0].astype(np.int32)).cuda()
        for l in range(p.m.n_layers):
            got = p.G.paged_read(p.G.layer_pool(p.pool, l), table, p.prefix[0] + L + 1)
            for x, y in zip(got, OP.read(p.caches[0][l], p.table[0], p.prefix[0] + L + 1)):
                x = x.double().cpu().numpy()
                assert (np.abs(x - y) <= np.maximum(np.abs(y) / 8, np.abs(y).max() / 448 / 64)).all()
    finally:
        p.v.close()


def test_graphs_streams_and_lengths():
    """Replayed steps equal plain launches bit for bit, on a stream of the
    context's own, over prefixes on both sides of the launches' bounds."""
    p = Paged("tiny", prefixes=[200], extra=400, stream=torch.cuda.Stream())
    try:
        trees = [gen.random_tree((3, 4, 2), p.m.vocab, 40 + i)[0] for i in range(3)]
        lens = [200, 120, 200, 57, 0]
        for n in (257, 300, 600):  # slots behind the prefix, filled through the operator
            lens.append(n)
        fill = torch.randn(1, 450, p.m.n_kv_heads, p.m.head_dim, device="cuda")
        table = torch.from_numpy(p.table[:1].astype(np.int32)).cuda()
        for l in range(p.m.n_layers):
            p.G.paged_append(p.G.layer_pool(p.pool, l), table, torch.tensor([200], dtype=torch.int32, device="cuda"), fill, fill)
        torch.cuda.synchronize()
        out = torch.empty((p.v.max_tree, p.m.vocab), device="cuda")
        got = {}
        for graphs in (True, True, False):
            p.v.set_graphs(graphs)
            for n in lens:
                for i, tree in enumerate(trees):
                    p.v.step([n], [tree], out)
                    p.v.accept()
                    lg = out[: tree.n].clone()
                    torch.cuda.synchronize()
                    assert lg.isfinite().all()
                    assert torch.equal(got.setdefault((n, i), lg), lg)
    finally:
        p.v.close()


def test_cycle_over_pages():
    """SpeculativeCycle over a paged target with a draft equal to it: it emits
    what single steps emit from a copy of the same pages, as far as the target's
    choices are no near ties (the same tokens cached in other portions may be
    rounded otherwise), and accepts drafts."""
    from tests.test_cycle_gpu import self_draft
    import paper_2502_11018_amd as G
    ds, mw, dw = self_draft()
    m, n, cap = ds.target, 90, 256
    ow = oracle.OracleWeights(mw)
    kv = H.prefix_kv_prefill(ow, np.random.default_rng(100).integers(0, m.vocab, n))
    k, v = (torch.from_numpy(x[0]).to(torch.bfloat16).cuda() for x in (kv.K, kv.V))
    mg = mw.to("cuda")
    vs = []
    for _ in range(2):
        pool = G.paged_pool(cap // 64 + 1, m.n_kv_heads, m.head_dim, 64, layers=1)
        x = G.TreeVerifier(m, mg, max_batch=1, max_tree=64, max_depth=63, kv_capacity=cap, pool=pool)
        x.set_pages(0, np.arange(cap // 64)[::-1].copy())
        x.write_prefix(0, 0, k, v)
        vs.append(x)
    d = G.DraftModel(ds, dw.to("cuda"), mg, max_batch=1, max_tree=64, max_depth=63, kv_capacity=cap)
    try:
        d.write_prefix(0, k, v)
        torch.cuda.synchronize()
        cyc = G.SpeculativeCycle(vs[0], d, ds.k, ds.depth, ds.n_total)
        cyc.start([n], [5], torch.zeros(1, m.d_model, device="cuda"))
        out, accepted = [], 0
        while len(out) < 30:
            say(f"cycle over pages: {len(out)} tokens")
            out += cyc.cycle()[0]
            accepted += sum(cyc.last_accepted)
        root, at, compared = 5, n, 0
        for tok in out[:30]:
            vs[1].step([at], [gen.chain_tree(root, [])])
            acc = vs[1].accept()
            if vs[1].margins()[0, 0] < 0.05:
                break
            assert int(acc.tokens[0, 0]) == tok, f"token {compared}"
            vs[1].commit()
            root, at, compared = tok, at + 1, compared + 1
        say(f"cycle over pages: {compared} tokens compared, {accepted} drafts accepted")
        assert compared >= 8 and accepted >= 8
    finally:
        d.close()
        for x in vs:
            x.close()


def test_refusals():
    """Pages that are not set, tables that are too short, and a window without
    a pool."""
    p = Paged("tiny", extra=0)
    G, N = p.G, __import__("paper_2502_11018_amd._native", fromlist=["x"])
    code = lambda f, *a: pytest.raises(G.GriffinError, f, *a).value.name  # noqa: E731
    try:
        tree = gen.chain_tree(1, [2, 3])
        n, cap = p.prefix[0], p.cols * PAGE
        before = [t.view(torch.uint8).clone() for t in p.pool]
        assert code(p.v.step, [cap - 2], [tree]) == "GRIFFIN_ECAPACITY"
        p.v.set_pages(0, [-1], first=1)
        assert code(p.v.step, [n], [tree]) == "GRIFFIN_ECAPACITY"
        p.v.set_pages(0, p.table[0][1:2], first=1)
        p.v.set_pages(0, [-1], first=n // PAGE)        # the page that the commit would write
        assert code(p.v.step, [n], [tree]) == "GRIFFIN_ECAPACITY"
        p.v.set_pages(0, p.table[0][n // PAGE:][:1], first=n // PAGE)
        assert code(p.v.set_pages, 0, [len(p.pool.k[0])]) == "GRIFFIN_EINVAL"
        assert code(p.v.set_pages, 0, [-2]) == "GRIFFIN_EINVAL"
        assert code(p.v.set_pages, 1, [0]) == "GRIFFIN_EINVAL"
        assert code(p.v.set_pages, 0, [0, 0], p.cols - 1) == "GRIFFIN_ECAPACITY"
        assert code(p.v.commit) == "GRIFFIN_EORDER"
        assert all(torch.equal(t.view(torch.uint8), x) for t, x in zip(p.pool, before))
        p.v.step([n], [tree])
        p.v.accept()
        p.v.commit()
        mw = p.mw.to("cuda")
        args = dict(max_batch=1, max_tree=16, max_depth=15, kv_capacity=128)
        rows = torch.zeros(p.m.n_kv_heads, cap + 1, p.m.head_dim, dtype=torch.bfloat16, device="cuda")
        with pytest.raises(ValueError):
            p.v.write_prefix(0, 0, rows, rows)
        with pytest.raises(ValueError):
            G.TreeVerifier(p.m, mw, window=64, **args)
        with pytest.raises(ValueError):
            G.TreeVerifier(p.m, mw, pool=G.paged_pool(4, p.m.n_kv_heads, 64, 96, layers=p.m.n_layers), **args)
        with pytest.raises(ValueError):
            G.TreeVerifier(p.m, mw, pool=G.paged_pool(4, p.m.n_kv_heads, 64, 64, layers=1), **args)
        with pytest.raises(G.GriffinError):
            G.TreeVerifier(p.m, mw, pool=G.paged_pool(4, 1, 64, 64, layers=p.m.n_layers), **args)
        plain = G.TreeVerifier(p.m, mw, **args)
        assert code(plain.set_pages, 0, [0]) == "GRIFFIN_EINVAL"
        plain.close()
    finally:
        p.v.close()
