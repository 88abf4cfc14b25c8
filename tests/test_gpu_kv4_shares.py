"""How the work of an attention over a 4-bit cache is cut: batches of more
requests than a wave has lanes, every number of row tiles, streams of many
pieces, a workspace that an earlier call has used, calls on two streams."""

import numpy as np
import pytest
import torch

from tests.gpu_cases import d2sd
from tests.kv4_cases import gather
from tests.test_gpu_kv4_attention import Batch, Rows, canonical, tokens

pytestmark = pytest.mark.gpu


def chain(n):
    return Rows(np.tril(np.ones((n, n), bool)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_split", [0, 128])
def test_more_requests_than_lanes(kv_split, dtype):
    """150 requests, of which some have no nodes or no context, with the first and the last ones empty."""
    rng = np.random.default_rng(40)
    nodes = rng.integers(0, 30, 150)
    nodes[[0, 63, 64, 127, 128, 149]] = 0
    ctx = rng.integers(0, 400, 150)
    ctx[rng.random(150) < 0.2] = 0
    b = Batch([chain(int(n)) for n in nodes], ctx, 4, 1, dtype, seed=41)
    b.check(*b.run(kv_split=kv_split))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_split", [0, 64, 256])
def test_every_number_of_row_tiles(kv_split, dtype):
    """One to nine tiles of 32 rows: groups of four, two and one, full and ragged."""
    trees = [chain(8 * t - 3 * (t % 2)) for t in range(1, 10)]
    ctx = [300, 129, 0, 513, 64, 128, 700, 1, 257]
    b = Batch(trees, ctx, 8, 2, dtype, seed=42)
    b.check(*b.run(kv_split=kv_split))
    b.check(*b.run(kv_split=kv_split, node_indptr_host=b.ip))


@pytest.mark.parametrize("kv_split", [0, 64, 704])
def test_streams_of_many_pieces(kv_split):
    """One stream over all workgroups: up to 264 pieces."""
    b = Batch([chain(5)], [33700], 4, 1, "bf16", seed=43)
    b.check(*b.run(kv_split=kv_split))


def test_a_used_workspace_and_its_need():
    """Larger and smaller calls in turn on one workspace, which holds junk at first; with a byte too few it is refused."""
    m = d2sd()
    calls = [Batch(canonical(16, [[3, 9], [1], [2, 4, 8]]), [1000, 517, 64], 8, 2, "bf16", seed=44),
             Batch(tokens(3), [2000, 40, 333], 8, 2, "bf16", seed=45),
             Batch([chain(70)], [129], 8, 2, "bf16", seed=46)]
    ws = torch.randint(0, 256, (1 << 24,), dtype=torch.uint8, device="cuda")
    want = [[t.clone() for t in b.run()] for b in calls]
    for i in (0, 1, 2, 1, 0, 2):
        out, lse = calls[i].run(workspace=ws)
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
    b = calls[0]
    a = m.attn_args_kv4(b.q, b.cache, b.d[0], b.d[1], b.kt, b.vt, b.d[2], b.mask, torch.empty_like(b.q), None,
                        total_nodes=b.total, max_nodes=b.most, max_ctx_len=1000)
    need = m.cascade_workspace_size_kv4(a)
    out, _ = b.run(workspace=ws[:need])
    assert torch.equal(out, want[0][0])
    with pytest.raises(m.D2SDError):
        b.run(workspace=ws[:need - 1])


def test_calls_on_two_streams():
    """Two calls at once, each with its own workspace."""
    calls = [Batch(canonical(16, [[3, 9], [1], [2, 4, 8]]), [3000, 1517, 64], 8, 2, t, seed=47) for t in ("bf16", "f32")]
    want = [[t.clone() for t in b.run()] for b in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(4):
        got = [b.run(stream=s) for b, s in zip(calls, streams)]
        torch.cuda.synchronize()
        for (o, l), (x, y) in zip(got, want):
            assert torch.equal(o, x) and torch.equal(l, y)


def test_kernel_timing_counts_the_calls():
    m = d2sd()
    b = Batch(canonical(16, [[3, 9], [1]]), [3000, 517], 8, 2, "bf16", seed=48)
    m.kernel_timing_enable(True)
    try:
        m.kernel_timing_collect()
        b.run()
        b.run(stage=m.STAGE_TREE)
        b.run()
        kernel, merge = m.kernel_timing_collect_parts()
    finally:
        m.kernel_timing_enable(False)
    assert len(kernel) == 3 and min(kernel) > 0
    assert merge[0] > 0 and merge[1] == 0 and merge[2] > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_beyond_32_bit_offsets(dtype):
    """A cache whose codes pass 4 GiB, its context on the last pages: the bits of the same context in a small cache."""
    m = d2sd()
    b = Batch([chain(9), chain(3)], [700, 50], 16, 8, dtype, seed=49)
    small, n = b.cache, b.cache.num_pages
    want = [t.clone() for t in b.run()]
    pages = (1 << 32) // (8 * 1024) + 1000
    big = m.Kv4Cache(*(torch.empty((pages, *t.shape[1:]), dtype=torch.uint8, device="cuda")
                       for t in (small.k, small.v, small.k_scale, small.v_scale)))
    for x, y in ((big.k, small.k), (big.v, small.v), (big.k_scale, small.k_scale), (big.v_scale, small.v_scale)):
        x[:n] = 255                                    # the same ids without the offset: NaN blocks
        x[pages - n:] = y
    b.cache = big
    b.d[0] = b.d[0] + (pages - n)
    for kw in ({}, dict(kv_split=128)):
        out, lse = b.run(**kw)
        assert torch.equal(out, want[0]) or kw
        assert torch.isfinite(out.float()).all() and torch.allclose(lse, want[1], atol=1e-5)


def test_tensors_of_another_device_are_refused(monkeypatch):
    """Before any launch; another device is simulated by what the current one is said to be."""
    m = d2sd()
    b = Batch(tokens(2), [40, 20], 4, 1, "bf16", seed=53)
    one = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    monkeypatch.setattr(m, "_current_device", lambda: 7)
    x = b.kt[:2]
    for call in (b.run, lambda: m.append_kv4(one, 2, 1, x, x, b.d[0], b.d[1], b.cache, 40),
                 lambda: m.commit_accepted_kv4(2, one, 2, one, one, x, x, b.d[0], b.d[1], b.cache, 40),
                 lambda: m.read_kv4(one, 2, 1, b.d[0], b.cache),
                 lambda: m.adjust_logits(one, 2, 1, one, b.mask, one, torch.zeros((2, 8), device="cuda"))):
        with pytest.raises(ValueError, match="current device"):
            call()
    monkeypatch.undo()
    b.check(*b.run())


@pytest.mark.parametrize("kv_split", [0, 64])
@pytest.mark.parametrize("ctx", [1, 2, 17, 100, 512])
def test_lse_of_short_contexts(ctx, kv_split):
    """bf16 queries over short contexts lose nothing that an lse in 32 bits would show.

    Four E2M3 terms leave at most 2^-20 of the power of two above a block's
    largest element, itself at most twice that, per element; products and sums
    are fp32: a score is a sum of 128 products through a chain of at most 16
    accumulations, the lse one of its keys."""
    m = d2sd()
    b = Batch([chain(1)] * 8, [ctx] * 8, 8, 2, "bf16", seed=[54, ctx])
    _, lse = b.run(stage=m.STAGE_PREFIX, kv_split=kv_split)
    q, lse = b.q.double().cpu().numpy(), lse.double().cpu().numpy()
    for r in range(8):
        k = gather(b.host, "k", b.table[r], 0, ctx)
        for h in range(8):
            key = k[:, h // 4]
            s = key @ q[r, h] / np.sqrt(128.0)
            want = s.max() + np.log(np.exp(s - s.max()).sum())
            top = np.abs(q[r, h]).reshape(4, 32).max(1)
            cut = (2.0 ** -19 * top * np.abs(key).reshape(ctx, 4, 32).sum(2)).sum(1).max() / np.sqrt(128.0)
            size = (np.abs(key) @ np.abs(q[r, h])).max() / np.sqrt(128.0)
            tol = cut + 2.0 ** -24 * (18 * size + (ctx + 16) + 4 * abs(want))
            assert abs(lse[r, h] - want) <= tol, (r, h, lse[r, h] - want, tol)
