"""Drafted trees on the GPU (tkv_attend_tree, tkv_verify_tree, tkv_accept_tree, tkv_commit_tree) against the 64-bit oracle.

Tolerances.  A binary32 logit is off by at most (D + 8) * 2^-24 * sum |q k| * scale, A below being the largest such sum; a weight, and
the sum it is divided by, by twice that relative to it; the weighted sum of N rows by another N / 4 + 64 roundings (16 rows to an
instruction, splits, the running maximum's corrections).  So an output is off by at most (4 (D + 8) A + N / 4 + 64) * 2^-24 of
sum w |v|.  That is a bound for errors that all fall the same way; over many outputs they do not: rms sqrt(D) * 2^-24 of a logit of four
or so, 3e-6, is what the 2-norm may be off.  16-bit outputs add half a step of the output and, with one 16-bit term per weight, half a
step of the row type of sum w |v|."""
import numpy as np
import pytest
import torch

import paper_2605_09490_amd as tkv
from oracle import tree_oracle as T

pytestmark = pytest.mark.gpu
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def tree(rng, B, n, kind):
    """Parents [B, n]."""
    p = np.full((B, n), -1, np.int32)
    for b in range(B):
        for i in range(1, n):
            p[b, i] = i - 1 if kind == "line" else 0 if kind == "star" else -1 if kind == "forest" and i % 3 == 0 else rng.integers(max(0, i - 6), i)
    if kind == "holes":
        for b in range(B):
            for i in rng.choice(np.arange(1, n), max(1, n // 6), replace=False) if n > 1 else []:
                p[b, i] = rng.choice([-2, n, i, 2**31 - 1, -2**31])
    if kind == "none":
        p[:] = -2
        p[-1, 0] = -1
    return p


class Both:
    """A GPU cache and an oracle with the same rows: context, forced tiers, then whatever the test does."""

    def __init__(self, seed, L=2, B=2, Hq=10, Hkv=2, D=128, ctx=300, room=200, dtype="bf16", t2="int8_row", out="f32", tiers=True, share=(.5, .2, .2, .1),
                 mode="lazy", scorer="attention", **kw):
        self.rng = np.random.default_rng(seed)
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.L, self.B, self.Hq, self.Hkv, self.D, self.dtype, self.out = L, B, Hq, Hkv, D, dtype, out
        kw = dict(dict(k_sink=2, k_window=8), **kw)
        self.gpu = tkv.TieredKV(L, B, Hq, Hkv, D, ctx + room, kv_dtype=dtype, t2_format=t2, out_dtype=out, prefetch_mode=mode, scorer=scorer, bounce_bytes=1 << 20, **kw)
        self.orc = T.TreeOracleCache(L, B, Hq, Hkv, D, ctx + room, kv_dtype=dtype, t2_format=t2, scorer=scorer, k_sink=2, k_window=8)
        if ctx:
            self.append_all(ctx)
        if tiers and ctx:
            t = self.rng.choice(4, size=(B, ctx), p=share).astype(np.uint8)
            t[:, -8:] = 0
            self.force(t)

    def force(self, t):
        for c in (self.gpu, self.orc):
            c.set_tiers(t)
            c.migrate()

    def rows(self, n, heads):
        return torch.randn((self.B, n, heads, self.D), generator=self.g, device="cuda").to(DT[self.dtype])

    def append(self, l, k, v):
        self.gpu.append(l, k, v)
        self.orc.append(l, f64(k), f64(v))

    def append_all(self, n):
        for l in range(self.L):
            self.append(l, self.rows(n, self.Hkv), self.rows(n, self.Hkv))

    def attend(self, parents, check=True):
        """Rows and queries of a tree for every layer; outputs compared.  Returns the queries [L, B, n, Hq, D]."""
        n = parents.shape[1]
        pd = torch.from_numpy(parents).cuda()
        q = torch.stack([self.rows(n, self.Hq) for _ in range(self.L)])
        for l in range(self.L):
            self.append(l, self.rows(n, self.Hkv), self.rows(n, self.Hkv))
            got = self.gpu.attend_tree(l, q[l], pd)
            if check:
                self.compare(l, f64(got), f64(q[l]), parents)
            else:
                self.orc.attend_tree(l, f64(q[l]), parents)
        return q

    def compare(self, l, got, q, parents):
        ref = self.orc.attend_tree(l, q, parents)
        w = self.orc.tree_weights[l]                                                     # [B, n, Hq, N]
        N, G = w.shape[-1], self.Hq // self.Hkv
        K, V = (np.abs(np.repeat(x[l][:, :, :N], G, 1)) for x in (self.orc.K, self.orc.V))   # [B, Hq, N, D]
        A = np.where(w > 0, np.einsum("bnhd,bhkd->bnhk", np.abs(q), K), 0).max() / np.sqrt(self.D)
        wv = np.einsum("bnhk,bhkd->bnhd", w, V)
        tol = (4 * (self.D + 8) * A + N / 4 + 64) * 2.0 ** -24 * wv
        if self.out != "f32":
            tol += HALF_STEP[self.out] * (np.abs(ref) + tol) + HALF_STEP[self.dtype] * wv + 2.0 ** -24
        bad = np.abs(got - ref) > tol
        assert not bad.any(), f"layer {l}: {bad.sum()} outputs off, worst {(np.abs(got - ref) / np.maximum(tol, 1e-300)).max():.2f} of the bound"
        if self.out == "f32":
            assert np.linalg.norm(got - ref) <= 3e-6 * np.linalg.norm(ref)
        here = np.array([[x is not None for x in T.ancestors(p)] for p in parents])
        assert not got[~here].any()

    def check_scores(self):
        n = self.gpu.layer_length(0)
        got, ref = self.gpu.get_scores().astype(np.float64), self.orc.score
        # weights as above, 1e-4 for the largest logits here; sums of positive numbers; weights below 2^-126 are lost
        assert np.all(np.abs(got - ref) <= 1e-4 * ref + 1e-12), np.abs(got - ref).max()
        assert not got[:, n:].any() and not ref[:, n:].any()
        assert np.array_equal(self.gpu.get_tiers()[:, :n], self.orc.tier[:, :n])

    def close(self):
        self.gpu.close()


SHAPES = [
    # dtype, t2, heads, D, B, context, nodes, kind
    ("bf16", "int8_row", (10, 2), 128, 2, 300, 7, "tree"),
    ("bf16", "int4_g32", (28, 4), 128, 1, 517, 25, "holes"),
    ("bf16", "int8_row", (40, 8), 128, 2, 260, 33, "tree"),
    ("bf16", "int4_g32", (8, 1), 64, 3, 200, 64, "forest"),
    ("bf16", "int8_row", (5, 1), 64, 1, 100, 128, "tree"),
    ("bf16", "int8_row", (4, 4), 128, 2, 90, 1, "line"),
    ("f16", "int8_row", (10, 2), 128, 2, 400, 13, "tree"),
    ("f16", "int4_g32", (12, 2), 64, 1, 333, 40, "holes"),
    ("f16", "int4_g32", (7, 1), 128, 1, 150, 100, "line"),
    ("f32", "int8_row", (6, 2), 64, 2, 257, 9, "tree"),
    ("f32", "int4_g32", (8, 1), 128, 1, 140, 30, "star"),
    ("f32", "int8_row", (3, 3), 128, 2, 65, 64, "holes"),
]


@pytest.mark.parametrize("dtype,t2,heads,D,B,ctx,n,kind", SHAPES)
def test_attend_and_accept(dtype, t2, heads, D, B, ctx, n, kind):
    """Outputs of a tree over all tiers; then a path is kept, its weights enter the scores, and a second tree goes on from there."""
    p = Both(n * 7 + D, Hq=heads[0], Hkv=heads[1], D=D, B=B, ctx=ctx, dtype=dtype, t2=t2, room=2 * n + 4)
    for _ in range(2):
        parents = tree(p.rng, B, n, kind)
        q = p.attend(parents)
        paths = []
        for b in range(B):
            lines = [x for x in T.ancestors(parents[b]) if x is not None]
            paths.append(lines[p.rng.integers(len(lines))][:6])
        path = np.full((B, 6), -1, np.int32)
        for b, x in enumerate(paths):
            path[b, :len(x)] = x
        assert p.gpu.accept_tree(n, torch.from_numpy(path).cuda(), q) == p.orc.accept_tree(n, paths)
        p.check_scores()
    p.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("out", ["bf16", "f16"])
def test_outputs_of_16_bits(dtype, out):
    p = Both(3, dtype=dtype, out=out, ctx=350, L=1)
    p.attend(tree(p.rng, 2, 21, "tree"))
    p.close()


@pytest.mark.parametrize("share,kind", [((0, 1, 0, 0), "tree"), ((0, 0, 1, 0), "tree"), ((0, 0, 0, 1), "tree"), ((.01, 0, .98, .01), "none"), ((1, 0, 0, 0), "none")])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_contexts_in_one_tier(share, kind, dtype):
    """Everything staged, compressed, evicted; trees of which nothing is there but one root."""
    p = Both(11, dtype=dtype, share=share, ctx=130, L=1, t2="int4_g32")
    p.attend(tree(p.rng, 2, 10, kind))
    p.close()


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "f32")])
def test_no_context_at_all(D, dtype):
    """The tree is all there is: the first positions of the cache; then everything is taken back, and it begins again."""
    p = Both(13, dtype=dtype, D=D, ctx=0, L=2)
    for _ in range(2):
        q = p.attend(tree(p.rng, 2, 18, "forest"))
        assert p.gpu.accept_tree(18, None, q) == 0 and p.orc.accept_tree(18, [[], []]) == 0
        assert p.gpu.layer_length(1) == 0
    q = p.attend(tree(p.rng, 2, 5, "line"))
    assert p.gpu.accept_tree(5, torch.tensor([[0, 1], [0, -1]], dtype=torch.int32, device="cuda"), q) == p.orc.accept_tree(5, [[0, 1], [0]])
    p.check_scores()
    p.close()


@pytest.mark.parametrize("dtype,D,Hkv,ctx", [("bf16", 128, 2, 2500), ("f16", 64, 1, 5000), ("f32", 64, 2, 1300)])
def test_longer_lists(dtype, D, Hkv, ctx):
    """Many splits, the tree's rows across a tile's edge, lists that end inside one."""
    p = Both(17, dtype=dtype, D=D, Hq=4 * Hkv, Hkv=Hkv, B=1, L=1, ctx=ctx, share=(.7, .0, .3, .0), t2="int4_g32")
    p.attend(tree(p.rng, 1, 37, "tree"))
    p.close()


@pytest.mark.parametrize("scale", [1e-4, 1.0, 3e3])
def test_values_of_other_sizes_in_binary16(scale):
    """T2's scales beside weights in binary16: values far from one, alone and beside ordinary rows."""
    p = Both(19, dtype="f16", ctx=200, L=1, tiers=False, t2="int8_row")
    k, v = p.rows(150, 2), p.rows(150, 2)
    p.append(0, k, (v.float() * scale).half())
    t = np.zeros((2, 350), np.uint8)
    t[:, 200:300] = 2
    t[1, :200] = 2
    p.force(t)
    p.attend(tree(p.rng, 2, 6, "tree"))
    p.close()


def test_rows_of_nodes_that_are_not_there_may_hold_anything():
    p = Both(23, ctx=100, L=1)
    parents = np.array([[-1, 0, -2, 2, 1], [-1, 0, 0, 1, 3]], np.int32)
    k, v, q = p.rows(5, 2), p.rows(5, 2), p.rows(5, 10)
    p.orc.append(0, np.nan_to_num(f64(k)), np.nan_to_num(f64(v)))
    for x in (k, v, q):
        x[0, 2:4] = float("nan")
        x[0, 3, :, ::2] = float("inf")
    p.gpu.append(0, k, v)
    p.compare(0, f64(p.gpu.attend_tree(0, q, torch.from_numpy(parents).cuda())), np.nan_to_num(f64(q), posinf=0), parents)
    p.close()


def test_a_kept_path_leaves_the_cache_of_a_plain_decode():
    """What follows a kept path has the bits that follow the same tokens decoded one by one; classify and migrate work on it."""
    a, b = (Both(29, B=2, ctx=280, room=60, scorer="vatp") for _ in range(2))
    parents, path = np.array([[-1, 0, 0, 2, 2, 4, 4]] * 2, np.int32), [0, 2, 4, 6]
    n = parents.shape[1]
    rows = [(a.rows(n, 2), a.rows(n, 2), a.rows(n, 10)) for _ in range(2)]
    for l, (k, v, q) in enumerate(rows):
        a.append(l, k, v)
        a.compare(l, f64(a.gpu.attend_tree(l, q, torch.from_numpy(parents).cuda())), f64(q), parents)
    kept = a.gpu.accept_tree(n, torch.tensor([path] * 2, dtype=torch.int32, device="cuda"), torch.stack([q for _, _, q in rows]))
    assert kept == 4 == a.orc.accept_tree(n, [path] * 2)
    for j in path:
        for l, (k, v, q) in enumerate(rows):
            b.append(l, k[:, j:j + 1].contiguous(), v[:, j:j + 1].contiguous())
            b.gpu.attend_and_score(l, q[:, j].contiguous())
    a.check_scores()
    assert np.allclose(a.gpu.get_scores(), b.gpu.get_scores(), rtol=2e-4, atol=1e-9)
    for l in range(2):
        for pos in range(280, 284):
            for which in (0, 1):
                assert np.array_equal(a.gpu.get_row(l, 1, 1, pos, which), b.gpu.get_row(l, 1, 1, pos, which))
    same = a.gpu.get_scores()
    b.gpu.set_scores(same)
    for step in range(3):
        for l in range(2):
            k, v, q = a.rows(1, 2), a.rows(1, 2), a.rows(1, 10)[:, 0].contiguous()
            a.gpu.append(l, k, v)
            b.gpu.append(l, k, v)
            assert torch.equal(a.gpu.attend_and_score(l, q), b.gpu.attend_and_score(l, q))
        assert np.array_equal(a.gpu.get_scores(), b.gpu.get_scores())
        for c in (a, b):
            c.gpu.classify((300_000, 300_000, 300_000, 100_000))
            c.gpu.migrate()
        assert np.array_equal(a.gpu.get_tiers(), b.gpu.get_tiers())
        for t in range(4):
            assert np.array_equal(a.gpu.get_index_list(t, 1), b.gpu.get_index_list(t, 1))
    a.close()
    b.close()


def test_gaps_of_sequences_that_keep_less():
    """Sequences that keep different numbers of nodes, step after step, across plans: outputs, scores, tiers, lists; T3 keeps the gaps."""
    p = Both(31, B=3, ctx=200, room=120, L=2, t2="int4_g32", mode="wait")
    for step in range(5):
        parents = tree(p.rng, 3, 9, "tree")
        q = p.attend(parents)
        paths = [T.ancestors(parents[b])[p.rng.integers(9)][:p.rng.integers(1, 6)] for b in range(3)]
        path = np.full((3, 9), -1, np.int32)
        for b, x in enumerate(paths):
            path[b, :len(x)] = x
        assert p.gpu.accept_tree(9, torch.from_numpy(path).cuda(), q) == p.orc.accept_tree(9, paths)
        p.check_scores()
        n = p.gpu.layer_length(0)
        for b in range(3):
            for t, ref in enumerate(p.orc.index_lists(b)):
                assert np.array_equal(p.gpu.get_index_list(t, b), ref)
        if step % 2:
            p.gpu.classify((400_000, 200_000, 300_000, 100_000))
            plan = p.gpu.get_pending_tiers()[:, :n]
            want = p.orc.classify((400_000, 200_000, 300_000, 100_000), score_f32=p.gpu.get_scores())[:, :n]
            assert np.array_equal(plan, want)
            p.gpu.migrate()
            p.orc.migrate()
        # one token on top of the gaps, on the decode path
        for l in range(2):
            p.append(l, p.rows(1, 2), p.rows(1, 2))
            x = p.rows(1, 10)[:, 0].contiguous()
            got, ref = f64(p.gpu.attend_and_score(l, x)), p.orc.attend_and_score(l, f64(x))
            assert np.linalg.norm(got - ref) <= 3e-6 * np.linalg.norm(ref)
    st = p.gpu.get_stats()
    t = p.gpu.get_tiers()[:, :p.gpu.layer_length(0)]
    assert st["tier_count"] == [int((t == k).sum()) for k in range(4)]
    p.close()


def test_taking_positions_back_over_gaps():
    """n_path = 0 over a range with gaps, and paths within one; slots come back, and as many as before can be appended."""
    p = Both(37, B=2, ctx=64, room=12, L=1, tiers=False)
    for _ in range(30):
        q = p.attend(tree(p.rng, 2, 6, "line"), check=False)
        assert p.gpu.accept_tree(6, torch.tensor([[0, 1, 2, -1], [0, -1, -1, -1]], dtype=torch.int32, device="cuda"), q) == 3 == p.orc.accept_tree(6, [[0, 1, 2], [0]])
        with pytest.raises(tkv.TkvError) as e:             # a node of the second sequence that is a gap
            p.gpu.accept_tree(3, torch.tensor([[0, 1], [0, 1]], dtype=torch.int32, device="cuda"))
        assert e.value.status == tkv.TKV_EINVAL
        assert p.gpu.accept_tree(3, torch.tensor([[1], [0]], dtype=torch.int32, device="cuda")) == 1 == p.orc.accept_tree(3, [[1], [0]], scored=False)
        p.check_scores()
        assert p.gpu.accept_tree(1) == 0 == p.orc.accept_tree(1, [[], []], scored=False)
        p.check_scores()
        assert p.gpu.layer_length(0) == 64
    p.append_all(12)
    with pytest.raises(tkv.TkvError):
        p.append_all(1)
    p.close()


def test_scores_without_queries_do_not_change():
    p = Both(41, ctx=90, L=1)
    p.gpu.set_scores(np.arange(2 * 290, dtype=np.float32).reshape(2, 290))
    p.attend(tree(p.rng, 2, 4, "line"), check=False)
    before = p.gpu.get_scores()
    p.gpu.accept_tree(4, torch.tensor([[0, 2], [1, 3]], dtype=torch.int32, device="cuda"))
    after = p.gpu.get_scores()
    assert np.array_equal(after[:, :90], before[:, :90]) and not after[:, 92:94].any() and np.array_equal(after[:, 94:], before[:, 94:])
    assert np.array_equal(after[:, 90:92], [[before[0, 90], before[0, 92]], [before[1, 91], before[1, 93]]])
    p.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_t1_placement_is_bit_invisible(dtype):
    """Prop. 1: staged rows give the bits of rows that never left, while their copies are under way too."""
    outs = []
    for mode, share in (("wait", 0), ("wait", 1), ("lazy", 1)):
        p = Both(43, dtype=dtype, mode=mode, ctx=600, L=3, tiers=False, Hq=14)
        t = np.zeros((2, 600), np.uint8)
        t[:, 100:300] = share
        t[:, 300:400] = 2
        p.gpu.set_tiers(t)
        p.gpu.migrate()
        parents = tree(np.random.default_rng(1), 2, 20, "tree")
        q = p.attend(parents, check=False)
        res = [p.gpu.attend_tree(l, q[l], torch.from_numpy(parents).cuda()) for l in range(3)]
        p.gpu.accept_tree(20, torch.tensor([[0, 1], [0, -1]], dtype=torch.int32, device="cuda"), q)
        outs.append((torch.stack(res).cpu(), p.gpu.get_scores()))
        p.close()
    for o, s in outs[1:]:
        assert torch.equal(o, outs[0][0]) and np.array_equal(s, outs[0][1])


def test_trees_of_growing_size_and_a_step_begun_again():
    """Scratch of larger trees; a tree attended in part, then another; q of layers that do not belong to this tree is refused."""
    p = Both(47, ctx=150, L=2, B=1)
    for n in (3, 17, 65, 128, 2):
        q = p.attend(tree(p.rng, 1, n, "tree"))
        assert p.gpu.accept_tree(n, torch.tensor([[0]], dtype=torch.int32, device="cuda"), q) == 1 == p.orc.accept_tree(n, [[0]])
        p.check_scores()
    parents = tree(p.rng, 1, 5, "line")
    for l in range(2):
        p.append(l, p.rows(5, 2), p.rows(5, 2))
    q = torch.stack([p.rows(5, 10) for _ in range(2)])
    one = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    p.gpu.attend_tree(0, q[0], torch.from_numpy(parents).cuda())
    with pytest.raises(tkv.TkvError) as e:
        p.gpu.accept_tree(5, one, q)
    assert e.value.status == tkv.TKV_ESTATE and p.gpu.layer_length(0) == p.orc.length[0]
    p.gpu.attend_tree(1, q[1, :, 1:].contiguous(), torch.from_numpy(parents[:, :4]).contiguous().cuda())   # four nodes
    with pytest.raises(tkv.TkvError):
        p.gpu.accept_tree(5, one, q)
    for l in range(2):
        p.compare(l, f64(p.gpu.attend_tree(l, q[l], torch.from_numpy(parents).cuda())), f64(q[l]), parents)
    assert p.gpu.accept_tree(5, one, q) == 2 == p.orc.accept_tree(5, [[0, 1]])
    p.check_scores()
    p.close()


def test_refusals():
    p = Both(53, ctx=100, L=2, B=1)
    pd = lambda n: torch.zeros((1, n), dtype=torch.int32, device="cuda") - 1

    def refused(status, f):
        before = p.gpu.layer_length(0), p.gpu.get_scores().tobytes(), p.gpu.get_tiers().tobytes()
        with pytest.raises(tkv.TkvError) as e:
            f()
        assert e.value.status == status, e.value
        assert before == (p.gpu.layer_length(0), p.gpu.get_scores().tobytes(), p.gpu.get_tiers().tobytes())

    refused(tkv.TKV_ESTATE, lambda: p.gpu.attend_tree(0, p.rows(1, 10), pd(1)))             # nothing appended since the plan
    p.append(0, p.rows(4, 2), p.rows(4, 2))
    refused(tkv.TKV_ESTATE, lambda: p.gpu.attend_tree(1, p.rows(4, 10), pd(4)))             # the layer has not been appended to
    refused(tkv.TKV_ESTATE, lambda: p.gpu.accept_tree(4))                                   # layers differ in length
    p.append(1, p.rows(4, 2), p.rows(4, 2))
    refused(tkv.TKV_ESTATE, lambda: p.gpu.attend_tree(0, p.rows(5, 10), pd(5)))
    refused(tkv.TKV_EINVAL, lambda: p.gpu.attend_tree(2, p.rows(4, 10), pd(4)))
    refused(tkv.TKV_ESTATE, lambda: p.gpu.accept_tree(5))
    refused(tkv.TKV_EINVAL, lambda: p.gpu.accept_tree(129))
    for bad in ([[1, 0]], [[0, 0]], [[0, 4]], [[-2]], [[0, 2, 1]], [[2**31 - 1]]):
        refused(tkv.TKV_EINVAL, lambda: p.gpu.accept_tree(4, torch.tensor(bad, dtype=torch.int32, device="cuda")))
    p.gpu.classify((500_000, 300_000, 200_000, 0))
    refused(tkv.TKV_ESTATE, lambda: p.gpu.accept_tree(4))
    p.close()
    for kw in (dict(mode="stream"), dict(scorer="redundancy"), dict(scorer="combined")):
        c = tkv.TieredKV(1, 1, 8, 2, 64, 64, prefetch_mode=kw.get("mode", "wait"), scorer=kw.get("scorer", "attention"))
        x = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16, device="cuda")
        c.append(0, x, x)
        for f in (lambda: c.attend_tree(0, torch.zeros((1, 4, 8, 64), dtype=torch.bfloat16, device="cuda"), pd(4)), lambda: c.accept_tree(4)):
            with pytest.raises(tkv.TkvError) as e:
                f()
            assert e.value.status == tkv.TKV_EINVAL
        c.close()


def test_a_chunk_over_gaps_is_refused():
    p = Both(59, ctx=40, L=1, tiers=False)
    p.append_all(4)
    p.gpu.accept_tree(4, torch.tensor([[0, 1], [0, -1]], dtype=torch.int32, device="cuda"))
    p.gpu.append(0, p.rows(2, 2), p.rows(2, 2))
    p.gpu.attend_and_score_chunk(0, p.rows(2, 10))
    for f in (lambda: p.gpu.attend_and_score_chunk(0, p.rows(3, 10)), lambda: p.gpu.attend_tree(0, p.rows(3, 10), torch.zeros((2, 3), dtype=torch.int32, device="cuda"))):
        with pytest.raises(tkv.TkvError) as e:
            f()
        assert e.value.status == tkv.TKV_ESTATE
    p.close()


# ---- the walk ----------------------------------------------------------------------------------------------------------------
def _walk_inputs(seed, B, n, V, kind, dtype, drawn, pad=0):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    parents = tree(rng, B, n, kind)
    logits = 2.0 * torch.randn((B, n, V), generator=g, device="cuda")
    tokens = torch.randint(0, V, (B, n), generator=g, device="cuda")
    up = torch.from_numpy(np.where((parents >= 0) & (parents < n), parents, 0)).long().cuda()
    b = torch.arange(B, device="cuda")[:, None]
    logits[b, up, tokens] += np.log(V) + 1
    wide = torch.full((2, B, n, V + pad), float("nan"), dtype=DT[dtype], device="cuda")
    wide[0, :, :, :V] = torch.softmax(logits, -1).to(DT[dtype])
    wide[1, :, :, :V] = torch.softmax(logits + 0.7 * torch.randn(logits.shape, generator=g, device="cuda"), -1).to(DT[dtype])
    p, q = wide[0, :, :, :V], wide[1, :, :, :V] if drawn else None
    u = torch.rand((B, n), generator=g, device="cuda")
    return torch.from_numpy(parents).cuda(), tokens.int(), p, u, torch.rand(B, generator=g, device="cuda"), q


def _walk_check(args, got):
    parents, tokens, p, u, ud, q = args
    path, count, nxt = (x.cpu().numpy() for x in got)
    for b in range(parents.shape[0]):
        line, token = T.walk(parents[b].cpu().numpy(), tokens[b].cpu().numpy(), f64(p[b]), None if q is None else f64(q[b]), u[b].cpu().numpy(), ud[b].item())
        assert list(path[b]) == line + [-1] * (len(path[b]) - len(line)) and count[b] == len(line) and nxt[b] == token, (b, path[b], line, nxt[b], token)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("B,n,V,kind,dtype,pad", [
    (1, 1, 1, "line", "f32", 0), (1, 6, 32000, "line", "f32", 0), (5, 30, 1001, "tree", "bf16", 7), (3, 128, 517, "tree", "f16", 1), (2, 64, 40009, "star", "f32", 3),
    (70, 9, 129, "holes", "bf16", 0), (300, 4, 33, "forest", "f32", 0), (2, 128, 70001, "line", "bf16", 5)])
def test_walk(B, n, V, kind, dtype, pad, drawn):
    c = tkv.TieredKV(1, B, 1, 1, 64, 8, bounce_bytes=1 << 16)
    for seed in range(3):
        args = _walk_inputs(seed, B, n, V, kind, dtype, drawn, pad)
        _walk_check(args, c.verify_tree(*args))
    c.close()


def test_walk_at_the_edges():
    """Random numbers 0 and the largest below 1; residuals with nothing in them; a token outside the vocabulary; rows of one token."""
    c = tkv.TieredKV(1, 2, 1, 1, 64, 8, bounce_bytes=1 << 16)
    top = float(np.nextafter(np.float32(1), np.float32(0)))
    parents = torch.tensor([[-1, 0, 0, 0, 1]] * 2, dtype=torch.int32, device="cuda")
    for V in (3, 5000):
        hot = torch.zeros((2, 5, V), device="cuda")
        hot[..., V - 1] = 1.0
        flat = torch.full((2, 5, V), 1.0 / V, device="cuda")
        for p, q in ((hot, None), (flat, None), (flat, flat), (hot, flat), (flat, hot), (hot, hot), (torch.zeros_like(hot), flat), (torch.zeros_like(hot), None)):
            for tok in ([V - 1, V - 1, V - 1, V - 1], [0, 1, 2, V - 1], [-1, V, 2**31 - 1, V - 1]):
                for u in (0.0, top):
                    tokens = torch.tensor([[7, *tok]] * 2, dtype=torch.int32, device="cuda")
                    args = (parents, tokens, p, torch.full((2, 5), u, device="cuda"), torch.full((2,), u, device="cuda"), q)
                    _walk_check(args, c.verify_tree(*args))
    with pytest.raises(AssertionError):
        c.verify_tree(parents, tokens, flat.transpose(0, 1).contiguous().transpose(0, 1), *args[3:5])
    c.close()


def test_commit_is_verify_and_accept():
    a, b = (Both(61, B=2, ctx=120, L=2) for _ in range(2))
    args = _walk_inputs(5, 2, 12, 700, "tree", "bf16", False)
    parents = args[0].cpu().numpy()
    qs = [x.attend(parents) for x in (a, b)]
    kept, path, count, token = a.gpu.commit_tree(*args, q_all=qs[0])
    path2, count2, token2 = b.gpu.verify_tree(*args)
    _walk_check(args, (path, count, token))
    assert torch.equal(path, path2) and torch.equal(count, count2) and torch.equal(token, token2)
    assert b.gpu.accept_tree(12, path2, qs[1]) == kept == int(count.max())
    a.orc.accept_tree(12, [[i for i in r if i >= 0] for r in path.cpu().tolist()])
    a.check_scores()
    assert np.array_equal(a.gpu.get_scores(), b.gpu.get_scores()) and np.array_equal(a.gpu.get_tiers(), b.gpu.get_tiers())
    a.close()
    b.close()


# ---- streams and graphs --------------------------------------------------------------------------------------------------------
def test_on_another_stream_and_in_a_graph():
    """A tree's attention and walk captured once and replayed, with new queries, other work and eager calls between the replays."""
    p = Both(67, B=2, ctx=700, L=2, Hq=8)
    parents = tree(p.rng, 2, 12, "holes")
    pd = torch.from_numpy(parents).cuda()
    for l in range(2):
        p.append(l, p.rows(12, 2), p.rows(12, 2))
    p.gpu.wait_prefetch()
    args = _walk_inputs(9, 2, 12, 3001, "tree", "f32", True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q = torch.zeros((2, 2, 12, 8, 128), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros(q.shape, device="cuda")
    with torch.cuda.stream(s):
        for l in range(2):
            p.gpu.attend_tree(l, q[l], pd, out[l])          # (allocates)
        p.gpu.verify_tree(*args)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        for l in range(2):
            p.gpu.attend_tree(l, q[l], pd, out[l])
        walked = p.gpu.verify_tree(*args)
    for seed in range(5):
        q.copy_(torch.randn(q.shape, generator=p.g, device="cuda"))
        args[3].uniform_(generator=p.g)
        g.replay()
        torch.cuda.synchronize()
        for l in range(2):
            p.compare(l, f64(out[l]), f64(q[l]), parents)
            assert torch.equal(out[l], p.gpu.attend_tree(l, q[l], pd))
        _walk_check(args, walked)
        assert all(torch.equal(x, y) for x, y in zip(walked, p.gpu.verify_tree(*args)))
    q1 = q.clone()
    torch.cuda.synchronize()
    assert p.gpu.accept_tree(12, torch.tensor([[0], [0]], dtype=torch.int32, device="cuda"), q1, stream=s) == 1
    p.orc.accept_tree(12, [[0], [0]])
    p.check_scores()
    p.close()


def test_two_handles_at_once():
    """Two caches on two streams, without a wait between them."""
    ps = [Both(71 + i, ctx=500, L=2, B=1) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in ps]
    parents = [tree(p.rng, 1, 20, "tree") for p in ps]
    qs, pds = [], [torch.from_numpy(x).cuda() for x in parents]
    for p in ps:
        for l in range(2):
            p.append(l, p.rows(20, 2), p.rows(20, 2))
        qs.append(torch.stack([p.rows(20, 10) for _ in range(2)]))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(4):
        for i, p in enumerate(ps):
            with torch.cuda.stream(streams[i]):
                outs[i].append([p.gpu.attend_tree(l, qs[i][l], pds[i]) for l in range(2)])
    torch.cuda.synchronize()
    for i, p in enumerate(ps):
        for l in range(2):
            p.compare(l, f64(outs[i][0][l]), f64(qs[i][l]), parents[i])
            assert all(torch.equal(o[l], outs[i][0][l]) for o in outs[i])
        p.close()


@pytest.mark.parametrize("dtype,t2,D,full,coded", [
    ("bf16", "int8_row", 128, 1e30, 1e30), ("bf16", "int8_row", 128, 1e-30, 1e-30), ("bf16", "int8_row", 64, 1e25, 1e-25), ("bf16", "int8_row", 128, 1e-25, 1e25),
    ("bf16", "int4_g32", 128, 1e-3, 1e3), ("bf16", "int4_g32", 64, 1e20, 1.0), ("f16", "int8_row", 128, 1e4, 1e-4), ("f16", "int8_row", 64, 1e-4, 1e4),
    ("f16", "int4_g32", 128, 1e-3, 1e3), ("f32", "int8_row", 64, 1e25, 1e-25)])
def test_values_of_any_size(dtype, t2, D, full, coded):
    """V rows far apart in size by tier: what a weight is multiplied with must neither overflow nor lose it.  To the bound of the 2-norm
    above comes what is lost below 2^-126: with weights of at least 2^-4 for a column's largest, 3 products (a weight's terms) of each of
    N rows lose less than 2^-126 each, so an output less than 3 N 2^-122."""
    p = Both(91, Hq=10, Hkv=2, D=D, B=1, ctx=0, dtype=dtype, t2=t2, room=260, L=1)
    n, N = 12, 200
    tiers = np.where(np.arange(N) % 3 == 0, 2, 0).astype(np.uint8)[None]
    tiers[:, -8:] = 0
    size = torch.from_numpy(np.where(tiers[0] == 2, coded, full)).cuda()[None, :, None, None]
    p.append(0, p.rows(N, 2), (p.rows(N, 2).double() * size).to(DT[dtype]))
    p.force(tiers)
    p.append(0, p.rows(n, 2), (p.rows(n, 2).double() * full).to(DT[dtype]))
    parents, q = tree(p.rng, 1, n, "tree"), p.rows(n, 10)
    got, ref = f64(p.gpu.attend_tree(0, q, torch.from_numpy(parents).cuda())), p.orc.attend_tree(0, f64(q), parents)
    assert np.isfinite(got).all()
    assert np.linalg.norm(got - ref) <= 3e-6 * np.linalg.norm(ref) + np.sqrt(ref.size) * 3 * (N + n) * 2.0 ** -122
    p.close()


@pytest.mark.parametrize("offset", [1, 4])
def test_queries_that_begin_between_16_byte_boundaries(offset):
    p = Both(73, ctx=80, L=1)
    parents = tree(p.rng, 2, 6, "tree")
    p.append(0, p.rows(6, 2), p.rows(6, 2))
    q = torch.empty(2 * 6 * 10 * 128 + offset, dtype=torch.bfloat16, device="cuda")[offset:].view(2, 6, 10, 128)
    q.copy_(p.rows(6, 10))
    p.compare(0, f64(p.gpu.attend_tree(0, q, torch.from_numpy(parents).cuda())), f64(q), parents)
    one = torch.empty((1 * 2 * 6 * 10 * 128) + offset, dtype=torch.bfloat16, device="cuda")[offset:].view(1, 2, 6, 10, 128)
    one.copy_(q[None])
    p.gpu.accept_tree(6, torch.tensor([[0, 1], [0, -1]], dtype=torch.int32, device="cuda"), one)
    line = [0, 1] if parents[0, 1] == 0 else [0]
    assert line == [0, 1]
    p.orc.accept_tree(6, [[0, 1], [0]])
    p.check_scores()
    p.close()
