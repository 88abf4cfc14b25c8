"""Logit adjustment on the GPU against the float64 oracle. Evaluated in fp32
and rounded once: an fp32 result is off by the few roundings of its formula,
each at most 2^-24 of the largest term; bf16 adds half a step of the result,
which is 2^-8 of it: bf16 holds 8 significant bits, so its values in [1, 2) are
2^-7 apart and rounding moves one by at most half of that."""

import numpy as np
import pytest
import torch

from oracle import logits as oracle
from oracle.tree import build_tree
from tests.gpu_cases import d2sd
from tests.kv4_cases import dev

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class Batch:
    def __init__(self, trees, V, dtype, seed=0, hist=40, bias=6, masks=3, few=None):
        rng = np.random.default_rng(seed)
        self.trees, self.V, self.dtype = trees, V, dtype
        n = len(trees)
        self.ip = np.concatenate([[0], np.cumsum([t.N for t in trees])]).astype(np.int32)
        self.total, self.most = int(self.ip[-1]), max(t.N for t in trees)
        W = (self.most + 31) // 32
        self.mask = np.concatenate([t.packed_mask(W) for t in trees]).view(np.int32)
        self.depth = np.concatenate([t.position for t in trees]).astype(np.int32)
        few = min(V, 12) if few is None else few
        pool = rng.integers(0, V, few)
        pick = lambda shape: np.where(rng.random(shape) < 0.7, rng.choice(pool, shape), rng.integers(0, V, shape)).astype(np.int32)
        self.draft = pick(self.total)
        self.x = dev((rng.standard_normal((self.total, V)) * 3).astype(np.float32)).to(TYPES[dtype])
        self.kw = {}
        if hist:
            self.kw.update(history=pick((n, hist)), history_len=rng.integers(0, hist + 1, n).astype(np.int32))
            self.kw["prompt_len"] = (self.kw["history_len"] * rng.random(n)).astype(np.int32)
        u = lambda lo, hi: rng.uniform(lo, hi, n).astype(np.float32)
        self.kw.update(repetition=u(0.8, 1.6), presence=u(-1, 1), frequency=u(-0.5, 0.5))
        if bias:
            self.kw.update(bias_token=pick((n, bias)), bias_value=rng.normal(0, 3, (n, bias)).astype(np.float32),
                           bias_len=rng.integers(0, bias + 1, n).astype(np.int32))
        if masks:
            w = rng.integers(0, 1 << 32, (masks, (V + 31) // 32), dtype=np.uint32)
            w[masks - 1] = 0                                  # leaves nothing
            self.kw.update(token_mask=w.view(np.int32), mask_row=rng.integers(-1, masks, self.total).astype(np.int32))

    def run(self, x=None, **over):
        kw = {**self.kw, **over}
        kw = {k: dev(v) if isinstance(v, np.ndarray) else v for k, v in kw.items()}
        return d2sd().adjust_logits(dev(self.ip), self.total, self.most, dev(self.depth), dev(self.mask), dev(self.draft),
                                    self.x if x is None else x, **kw)

    def check(self, got, **over):
        kw = {**self.kw, **over}
        x, got = self.x.double().cpu().numpy(), got.double().cpu().numpy()
        for b, t in enumerate(self.trees):
            of = lambda name, none: none if kw.get(name) is None else kw[name][b]
            h = of("history", np.zeros(0, int))[:of("history_len", 0)]
            p = of("prompt_len", 0)
            nb = of("bias_len", None)
            pairs = list(zip(of("bias_token", ())[:nb], of("bias_value", ())[:nb].astype(float))) if kw.get("bias_token") is not None else []
            r, o, f = float(of("repetition", 1.0)), float(of("presence", 0.0)), float(of("frequency", 0.0))
            for n in range(t.N):
                g = self.ip[b] + n
                allowed = None
                if kw.get("token_mask") is not None and kw["mask_row"][g] >= 0:
                    allowed = np.unpackbits(kw["token_mask"][kw["mask_row"][g]].view(np.uint8), bitorder="little")[:self.V]
                path = oracle.path_tokens(t.parent, self.draft[self.ip[b]:self.ip[b + 1]], n)
                want = oracle.adjust_row(x[g], h[:p], h[p:], path, r, o, f, pairs, allowed)
                wild = ~np.isfinite(want)
                assert np.array_equal(wild, ~np.isfinite(got[g]))
                assert np.array_equal(got[g][wild], want[wild], equal_nan=True)
                # terms: x and its product, count * frequency, presence, the biases
                size = np.abs(x[g]) * 2 + (len(h) + len(path)) * abs(f) + abs(o) + sum(abs(v) for _, v in pairs)
                tol = 2.0 ** -24 * (8 + len(pairs)) * size + (np.abs(want) * 2.0 ** -8 * 1.001 if self.dtype == "bf16" else 0)
                off = np.abs(got[g][~wild] - want[~wild])
                assert (off <= tol[~wild]).all(), (b, n, (off / tol[~wild]).max())


SMALL = [[3, 7], [], [1, 2, 3, 4, 5, 6, 7]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 7, 31, 33, 1000, 4096, 4097, 8200])
def test_vocabularies(V, dtype):
    b = Batch([build_tree(8, p) for p in SMALL], V, dtype, seed=V)
    b.check(b.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left_out", [("history", "history_len", "prompt_len"), ("prompt_len",), ("repetition",), ("presence", "frequency"),
                                      ("bias_token", "bias_value", "bias_len"), ("bias_len",), ("token_mask", "mask_row")])
def test_parts_left_out(left_out, dtype):
    b = Batch([build_tree(8, p) for p in SMALL], 300, dtype, seed=20)
    none = {k: None for k in left_out}
    b.check(b.run(**none), **none)


def test_nothing_to_adjust_is_a_copy():
    b = Batch([build_tree(8, p) for p in SMALL], 5001, "bf16", seed=21, hist=0, bias=0, masks=0)
    none = dict(repetition=None, presence=None, frequency=None)
    assert torch.equal(b.run(**none), b.x)


def test_the_same_token_again_and_again():
    """One token through the history, the drafts of a whole chain, and the bias list."""
    b = Batch([build_tree(16, [5, 9])], 50, "f32", seed=22, hist=30, bias=12, masks=0, few=1)
    b.draft[:] = b.draft[0]
    b.kw["bias_token"][:] = b.draft[0]
    b.kw["bias_len"][:] = 12
    b.check(b.run())


def test_many_drafts_of_one_thread():
    """2080 nodes of two neighbouring tokens."""
    b = Batch([build_tree(64, list(range(1, 64)))], 40, "f32", seed=23, hist=5, bias=0, masks=0, few=2)
    assert b.total == 2080
    b.draft[:] = np.where(np.arange(2080) % 3 == 0, 16, 17)
    b.check(b.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(dtype):
    b = Batch([build_tree(8, p) for p in SMALL], 4099, dtype, seed=24)
    want = b.run()
    x = b.x.clone()
    got = b.run(x=x, out=x)
    assert got.data_ptr() == x.data_ptr() and torch.equal(got, want)


def test_ids_out_of_range_and_long_lengths():
    b = Batch([build_tree(8, p) for p in SMALL], 100, "f32", seed=25)
    want = b.run(history_len=np.full(3, 40, np.int32), prompt_len=np.full(3, 10, np.int32))
    b.kw["history"] = np.concatenate([b.kw["history"], np.full((3, 3), -1, np.int32), np.full((3, 2), 100, np.int32),
                                      np.full((3, 2), 2 ** 31 - 1, np.int32), np.full((3, 1), -2 ** 31, np.int32)], 1)
    got = b.run(history_len=np.full(3, 2 ** 30, np.int32), prompt_len=np.full(3, 10, np.int32))
    assert torch.equal(got, want)
    got = b.run(history_len=np.full(3, -5, np.int32))
    b.check(got, history_len=np.zeros(3, np.int32), prompt_len=np.zeros(3, np.int32))
    rows = b.kw["mask_row"].copy()
    assert torch.equal(b.run(mask_row=np.where(rows == 2, 77, rows).astype(np.int32)), b.run())


def test_infinite_biases_and_logits():
    b = Batch([build_tree(8, [])], 64, "f32", seed=26, masks=2)
    b.kw["bias_value"][0, :2] = [-np.inf, np.inf]
    b.kw["bias_token"][0, :3] = [3, 4, 5]
    b.kw["bias_len"][:] = 3
    b.x[:, 10] = float("-inf")
    b.x[2, 11] = float("nan")
    b.x[3, 12] = float("inf")
    b.check(b.run())


def test_rows_behind_the_last_and_garbage():
    from tests.test_gpu_robustness import garbage_i32, guard_intact, guarded
    b = Batch([build_tree(8, p) for p in SMALL], 333, "bf16", seed=27)
    want = b.run()
    buf, out = guarded((b.total, 333), torch.bfloat16, 7.0)
    assert torch.equal(b.run(out=out), want) and guard_intact(buf, out.shape, 7.0)
    rng = np.random.default_rng(28)
    m = d2sd()
    for _ in range(3):
        g = lambda t: garbage_i32(rng, t.size).view(t.shape)
        kw = {k: (g(v) if v.dtype == np.int32 else dev(v)) for k, v in b.kw.items()}
        m.adjust_logits(garbage_i32(rng, 4), b.total, b.most, g(b.depth), g(b.mask), g(b.draft), b.x, out=out, **kw)
        torch.cuda.synchronize()
        assert guard_intact(buf, out.shape, 7.0)
    assert torch.equal(b.run(), want)
