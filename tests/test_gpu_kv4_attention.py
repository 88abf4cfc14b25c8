"""Verify attention over a 4-bit cache against the float64 oracle, within a
bound derived from its arithmetic (tests/kv4_cases.py)."""

import numpy as np
import pytest
import torch

from oracle.tree import build_tree
from tests.gpu_cases import d2sd
from tests.kv4_cases import check_request, dev, gather, page_tables, random_cache

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class OneNode:
    """The tree of plain decoding: one token."""
    N = 1

    def visible(self):
        return np.ones((1, 1), bool)


class Rows:
    """A tree given by its visibility matrix."""

    def __init__(self, vis):
        self.vis, self.N = vis, len(vis)

    def visible(self):
        return self.vis


def mask_of(trees, W):
    out = np.zeros((sum(t.N for t in trees), W * 32), np.uint8)
    r = 0
    for t in trees:
        out[r:r + t.N, :t.N] = t.visible()
        r += t.N
    return np.packbits(out, axis=1, bitorder="little").view(np.int32)


class Batch:
    def __init__(self, trees, ctx, hq, hkv, dtype, seed=0, pad_pages=0):
        rng = np.random.default_rng(seed)
        self.trees, self.ctx, self.dtype, self.hq, self.hkv = trees, np.asarray(ctx, np.int32), dtype, hq, hkv
        self.table, pages = page_tables(self.ctx, rng)
        if pad_pages:
            self.table = np.concatenate([self.table, np.zeros((len(ctx), pad_pages), np.int32)], 1)
        self.cache, self.host = random_cache(pages, hkv, rng)
        # rows past a context hold NaN blocks, which must not be seen
        for b, c in enumerate(self.ctx):
            if c % 16:
                page = self.table[b, c // 16]
                for n in ("k_scale", "v_scale"):
                    self.host[n][page, :, c % 16:] = 255
        for n in ("k_scale", "v_scale"):
            getattr(self.cache, n).copy_(dev(self.host[n]))
        self.ip = np.concatenate([[0], np.cumsum([t.N for t in trees])]).astype(np.int32)
        self.total, self.most = int(self.ip[-1]), max(t.N for t in trees)
        self.W = (self.most + 31) // 32
        self.mask = dev(mask_of(trees, self.W))
        f = lambda h: dev(rng.standard_normal((self.total, h, 128)).astype(np.float32)).to(TYPES[dtype])
        self.q, self.kt, self.vt = f(hq), f(hkv), f(hkv)
        self.d = [dev(x) for x in (self.table, self.ctx, self.ip)]

    def run(self, **kw):
        table, ctx, ip = self.d
        kw = {"max_ctx_len": int(self.ctx.max()), **kw}
        return d2sd().cascade_verify_attention_kv4(self.q, self.cache, table, ctx, self.kt, self.vt, ip, self.mask,
                                                   total_nodes=self.total, max_nodes=self.most, **kw)

    def check(self, out, lse, stage="cascade", requests=None):
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for b in range(len(self.trees)) if requests is None else requests:
            s, e = self.ip[b], self.ip[b + 1]
            if s == e:
                continue
            x = [t[s:e].double().cpu().numpy() for t in (self.q, self.kt, self.vt)]
            c = [gather(self.host, n, self.table[b], 0, int(self.ctx[b])) for n in ("k", "v")]
            check_request(out[s:e], lse[s:e], x[0], c[0], c[1], x[1], x[2], self.trees[b], self.dtype, stage)


def tokens(n):
    return [OneNode() for _ in range(n)]


def canonical(B, rows):
    return [build_tree(B, r) for r in rows]


# contexts: empty, one key, around a tile's and a page's ends
CTX = [0, 1, 15, 16, 17, 63, 64, 65, 127, 129, 300]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq, hkv", [(4, 1), (8, 2), (3, 3), (40, 8)])
def test_single_tokens(hq, hkv, dtype):
    b = Batch(tokens(len(CTX)), CTX, hq, hkv, dtype, seed=1)
    b.check(*b.run())
    b.check(*b.run(kv_split=64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_split", [0, 64, 128])
def test_trees(kv_split, dtype):
    """One to four row tiles and more per request, tree sizes on both sides of a key tile, an empty context."""
    trees = canonical(16, [[3, 9], [], list(range(1, 16)), [1], [15]])
    b = Batch(trees, [130, 0, 333, 64, 1], 8, 2, dtype, seed=2)
    b.check(*b.run(kv_split=kv_split, node_indptr_host=b.ip))
    b.check(*b.run(kv_split=kv_split))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G, B, p", [(1, 2, [1]), (8, 8, [2, 5]), (16, 16, [4]), (5, 33, [7, 30]), (64, 3, [])])
def test_group_sizes(G, B, p, dtype):
    b = Batch(canonical(B, [p, []]), [77, 210], G, 1, dtype, seed=[3, G])
    b.check(*b.run())


def test_long_tree():
    """2080 nodes: every re-anchor position of the largest block."""
    b = Batch(canonical(64, [list(range(1, 64))]), [40], 2, 1, "bf16", seed=4)
    assert b.total == 2080
    b.check(*b.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("stage", ["prefix", "tree"])
def test_stages(stage, dtype):
    b = Batch(canonical(16, [[3, 9], [], [5]]), [130, 0, 17], 8, 2, dtype, seed=5)
    m = d2sd()
    for split in (0, 64):
        b.check(*b.run(stage=m.STAGE_PREFIX if stage == "prefix" else m.STAGE_TREE, kv_split=split), stage)


def test_a_request_without_nodes_and_rows_behind_the_last():
    trees = [Rows(np.zeros((0, 0), bool)), OneNode(), Rows(np.zeros((0, 0), bool))]
    b = Batch(trees, [50, 20, 0], 4, 1, "bf16", seed=6)
    q = b.q
    out = torch.full((b.total + 3, 4, 128), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((b.total + 3, 4), 7.0, device="cuda")
    b.run(out=out[:b.total], lse=lse[:b.total])
    b.check(out[:b.total], lse[:b.total])
    assert (out[b.total:] == 7).all() and (lse[b.total:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx", [0, 70])
def test_rows_that_see_no_tree_key(ctx, dtype):
    """An empty mask row: the context alone, or nothing (out 0, lse -inf)."""
    vis = np.tril(np.ones((70, 70), bool))
    vis[[3, 65]] = False
    b = Batch([Rows(vis)], [ctx], 4, 2, dtype, seed=7)
    b.check(*b.run())
    b.check(*b.run(kv_split=64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("wild", [float("inf"), float("-inf"), float("nan")])
def test_wild_tree_values_and_keys_reach_those_who_see_them(wild, dtype):
    """A branch whose last node's value (one dim) and another whose key is not
    finite: rows that do not see the node keep their bits."""
    trees = canonical(16, [[3, 9]])
    b = Batch(trees, [100], 4, 2, dtype, seed=8)
    ref, ref_lse = (t.clone() for t in b.run())
    vis, node, key_node = trees[0].visible(), trees[0].N - 1, 16 + 12
    b.vt[node, 1, 37] = wild
    sees = dev(vis[:, node])
    out, lse = b.run()
    assert torch.equal(lse, ref_lse)
    touched = torch.zeros_like(ref, dtype=torch.bool)
    touched[:, 2:, 37] = sees[:, None]
    assert torch.equal(out[~touched], ref[~touched])
    got = out[touched].float()
    assert got.isnan().all() if np.isnan(wild) else (got == wild).all()
    b.vt[node, 1, 37] = 0.0
    ref, ref_lse = (t.clone() for t in b.run())
    b.kt[key_node, 0, 5] = float("nan")
    out, lse = b.run()
    unseen = ~dev(vis[:, key_node])
    assert torch.equal(out[unseen], ref[unseen]) and torch.equal(lse[unseen], ref_lse[unseen])
    assert torch.equal(out[:, 2:], ref[:, 2:])
    assert out[~unseen][:, :2].isnan().all() and lse[~unseen][:, :2].isnan().all()


def test_nan_blocks_and_queries_are_not_hidden():
    b = Batch(tokens(3), [100, 100, 100], 4, 1, "bf16", seed=9)
    ref, _ = (t.clone() for t in b.run())
    b.cache.v_scale[int(b.table[1, 2]), 0, 5, 1] = 255
    b.q[2, 3, 0] = float("nan")
    for kw in ({}, dict(kv_split=64)):
        out, lse = b.run(**kw)
        assert out[1, :, 32:64].isnan().all() and out[2, 3].isnan().all() and lse[2, 3].isnan()
        assert torch.isfinite(out[0].float()).all() and torch.isfinite(out[1, :, :32].float()).all()
        assert torch.isfinite(out[2, :3].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_far_apart(dtype):
    """Key and value blocks from 2^-60 to 2^3, queries from tiny to large, a zero query."""
    b = Batch(canonical(8, [[3]]), [200], 4, 1, dtype, seed=10)
    rng = np.random.default_rng(11)
    for n, lo in (("k_scale", -60), ("v_scale", -60)):
        b.host[n][:] = np.where(b.host[n] == 255, 255, 127 + rng.choice([lo, -20, -3, -1, 0], b.host[n].shape))
        getattr(b.cache, n).copy_(dev(b.host[n]))
    f = torch.tensor([2.0 ** -110, 2.0 ** -30, 1.0, 4.0], device="cuda")[:, None]
    b.q.copy_((b.q.float() * f).to(b.q.dtype))
    b.q[0, 1] = 0
    b.check(*b.run())


def test_custom_softmax_scale_and_large_scores():
    """Scores of some hundreds: one key takes all."""
    b = Batch(canonical(8, [[3]]), [150], 4, 2, "f32", seed=12)
    o1, l1 = b.run(sm_scale=0.25)
    b.q.mul_(0.25 * np.sqrt(128))
    o2, l2 = b.run()
    assert torch.allclose(o1, o2, atol=2e-5) and torch.allclose(l1, l2, atol=2e-4)
    b.q.mul_(20.0)
    b.check(*b.run())
    b.check(*b.run(kv_split=64))


def test_padded_maximum_context_and_wider_tables():
    """max_ctx_len far above the contexts, as under capture: more splits than any context has."""
    b = Batch(canonical(16, [[3], [5, 9]]), [130, 40], 8, 2, "bf16", seed=13, pad_pages=300)
    b.check(*b.run(max_ctx_len=4800))


def test_one_long_context():
    b = Batch(tokens(2), [33001, 7], 8, 2, "bf16", seed=14)
    b.check(*b.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_every_time_and_on_another_stream(dtype):
    b = Batch(canonical(16, [[3, 9], [1], [2, 4, 8]]), [1000, 517, 64], 8, 2, dtype, seed=15)
    out, lse = (t.clone() for t in b.run())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        o, l = b.run(stream=side)
        side.synchronize()
        assert torch.equal(o, out) and torch.equal(l, lse)


def test_inconsistent_device_arrays_stay_inside():
    from tests.test_gpu_robustness import garbage_i32, guard_intact, guarded
    m, rng = d2sd(), np.random.default_rng(16)
    b = Batch(canonical(16, [[3, 9], [1], [], [2, 4, 8]]), [1000, 517, 64, 0], 8, 2, "bf16", seed=17)
    ref, ref_lse = (t.clone() for t in b.run())
    for split in (0, 64, 256):
        obuf, out = guarded(tuple(b.q.shape), b.q.dtype, 7.0)
        lbuf, lse = guarded(tuple(b.q.shape[:2]), torch.float32, 7.0)
        table, ctx, ip = garbage_i32(rng, b.table.size).view(b.table.shape), garbage_i32(rng, 4), garbage_i32(rng, 5)
        kw = dict(total_nodes=b.total, max_nodes=b.most, max_ctx_len=1000, kv_split=split)
        a = m.attn_args_kv4(b.q, b.cache, table, ctx, b.kt, b.vt, ip, b.mask, out, lse, **kw)
        wbuf, ws = guarded((max(1, m.cascade_workspace_size_kv4(a)),), torch.uint8, 0x5A)
        m.cascade_verify_attention_kv4(b.q, b.cache, table, ctx, b.kt, b.vt, ip, b.mask, out=out, lse=lse, workspace=ws, **kw)
        torch.cuda.synchronize()
        assert guard_intact(obuf, out.shape, 7.0) and guard_intact(lbuf, lse.shape, 7.0) and guard_intact(wbuf, ws.shape, 0x5A)
    out, lse = b.run()
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
