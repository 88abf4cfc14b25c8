"""The 4-bit cache on the GPU: every byte against the float64 oracle, written
and untouched ones, and the values read back, which are exact."""

import numpy as np
import pytest
import torch

from oracle import kv4
from tests.gpu_cases import d2sd
from tests.kv4_cases import bytes_of, dev, gather, page_tables, random_cache

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def same_bytes(got, want):
    """Codes and scales, except the codes of blocks that read as NaN."""
    for n in ("k", "v"):
        assert np.array_equal(got[n + "_scale"], want[n + "_scale"]), n
        nan = np.repeat(want[n + "_scale"] == 255, 16, axis=-1)
        assert np.array_equal(np.where(nan, 0, got[n]), np.where(nan, 0, want[n])), n


def hard_rows(rng, n, hkv):
    """Rows of ordinary, tiny, huge, zero, tied and non-finite values."""
    x = rng.standard_normal((n, hkv, 128)).astype(np.float32)
    x *= (2.0 ** rng.integers(-30, 30, (n, hkv, 4))).repeat(32, -1).astype(np.float32)
    kind = rng.integers(0, 12, (n, hkv, 4)).repeat(32, -1)
    ties = rng.choice([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, -0.25, -0.75, -5, -7, -0.0], x.shape)
    x = np.where(kind == 0, ties, x)
    x = np.where(kind == 1, 0.0, x)
    x = np.where(kind == 2, x * np.float32(2.0 ** -140), x)
    with np.errstate(over="ignore"):
        x = np.where(kind == 3, np.clip(x.astype(np.float64) * 2.0 ** 110, -3e38, 3e38), x)
    x = x.astype(np.float32)
    x[rng.random(x.shape) < 3e-4] = np.inf
    x[rng.random(x.shape) < 3e-4] = np.nan
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hkv, ctx, lens", [(2, [0], [1]), (1, [15, 0, 31], [1, 16, 17]), (3, [5, 0, 16, 100, 7], [0, 40, 16, 3, 33]),
                                            (8, [0, 13], [300, 1]), (5, [1], [64])])
def test_append_then_read(hkv, ctx, lens, dtype):
    m, rng = d2sd(), np.random.default_rng([1, hkv, len(lens)])
    ctx, lens = np.array(ctx, np.int32), np.array(lens, np.int32)
    table, pages = page_tables(ctx + lens, rng)
    cache, host = random_cache(pages, hkv, rng)
    ip = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    total, most = int(ip[-1]), int(lens.max())
    k, v = (dev(hard_rows(rng, total, hkv)).to(TYPES[dtype]) for _ in range(2))
    d_ctx = dev(ctx)
    m.append_kv4(dev(ip), total, most, k, v, dev(table), d_ctx, cache, int(ctx.max()))
    for b in range(len(lens)):
        for n, x in (("k", k), ("v", v)):
            kv4.write_tokens((host[n], host[n + "_scale"]), x[ip[b]:ip[b + 1]].double().cpu().numpy(), table[b], int(ctx[b]))
    assert np.array_equal(d_ctx.cpu().numpy(), ctx + lens)
    same_bytes(bytes_of(cache), host)
    host = bytes_of(cache)
    for out in TYPES.values():           # the values, exactly, in both types
        rk, rv = m.read_kv4(dev(ip), total, most, dev(table), cache, start=dev(ctx), dtype=out)
        for n, r in (("k", rk), ("v", rv)):
            want = np.concatenate([gather(host, n, table[b], int(ctx[b]), int(lens[b])) for b in range(len(lens))])
            assert np.array_equal(r.double().cpu().numpy(), want, equal_nan=True)


def test_read_without_start_any_scale_byte():
    m, rng = d2sd(), np.random.default_rng(3)
    table, pages = page_tables([70, 33], rng)
    cache, host = random_cache(pages, 2, rng)
    for n in ("k_scale", "v_scale"):      # 2 .. 252 hold normal numbers in fp32, 255 is NaN
        host[n][:] = rng.choice(np.r_[np.arange(2, 253), 255], host[n].shape)
        getattr(cache, n).copy_(dev(host[n]))
    ip = np.array([0, 70, 103], np.int32)
    k, v = m.read_kv4(dev(ip), 103, 70, dev(table), cache, dtype=torch.float32)
    for n, r in (("k", k), ("v", v)):
        want = np.concatenate([gather(host, n, table[b], 0, int(ip[b + 1] - ip[b])) for b in range(2)])
        assert np.array_equal(r.double().cpu().numpy(), want, equal_nan=True)


def test_tokens_past_the_page_table_are_left_out():
    m, rng = d2sd(), np.random.default_rng(5)
    table = np.array([[2, 0]], np.int32)
    cache, host = random_cache(3, 2, rng)
    x = dev(rng.standard_normal((30, 2, 128)).astype(np.float32))
    ctx = dev(np.array([20], np.int32))
    m.append_kv4(dev(np.array([0, 30], np.int32)), 30, 30, x, x, dev(table), ctx, cache, 20)
    for n in ("k", "v"):
        kv4.write_tokens((host[n], host[n + "_scale"]), x[:12].double().cpu().numpy(), table[0], 20)
    assert ctx.item() == 32
    same_bytes(bytes_of(cache), host)


def test_append_in_parts_equals_append_at_once():
    m, rng = d2sd(), np.random.default_rng(4)
    lens = np.array([50, 23], np.int32)
    table, pages = page_tables(lens, rng)
    k, v = (torch.randn((73, 4, 128), device="cuda").bfloat16() for _ in range(2))
    whole, parts = m.Kv4Cache.empty(pages, 4), m.Kv4Cache.empty(pages, 4)
    ctx = dev(np.zeros(2, np.int32))
    m.append_kv4(dev(np.array([0, 50, 73], np.int32)), 73, 50, k, v, dev(table), ctx, whole, 0)
    ctx.zero_()
    at = np.zeros(2, np.int32)
    for a, b in ((7, 1), (1, 0), (30, 22), (12, 0)):
        pick = np.concatenate([np.arange(at[0], at[0] + a), 50 + np.arange(at[1], at[1] + b)])
        ip = np.array([0, a, a + b], np.int32)
        idx = dev(pick.astype(np.int64))
        m.append_kv4(dev(ip), a + b, max(a, b), k[idx], v[idx], dev(table), ctx, parts, 60 if at.any() else 0)
        at += [a, b]
        assert ctx.cpu().tolist() == at.tolist()
    for n in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(whole, n), getattr(parts, n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hkv", [1, 3, 8])
def test_commit(hkv, dtype):
    """Accepted lengths 0 and B - 1, contexts empty, mid-page and at a page's end."""
    m, rng = d2sd(), np.random.default_rng([6, hkv])
    B = 16
    ctx, L = np.array([0, 15, 16, 100], np.int32), np.array([0, B - 1, 3, 7], np.int32)
    nodes = [16, 30, 20, 41]
    ip = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    path = np.full((4, B), -1, np.int32)
    for b in range(4):
        path[b, :L[b] + 1] = np.sort(rng.permutation(nodes[b])[:L[b] + 1])
    table, pages = page_tables(ctx + B, rng)
    cache, host = random_cache(pages, hkv, rng)
    k, v = (dev(hard_rows(rng, int(ip[-1]), hkv)).to(TYPES[dtype]) for _ in range(2))
    d_ctx = dev(ctx)
    m.commit_accepted_kv4(B, dev(ip), int(ip[-1]), dev(path), dev(L), k, v, dev(table), d_ctx, cache, 100)
    for b in range(4):
        for n, x in (("k", k), ("v", v)):
            rows = x[torch.from_numpy(ip[b] + path[b, :L[b] + 1]).cuda().long()].double().cpu().numpy()
            kv4.write_tokens((host[n], host[n + "_scale"]), rows, table[b], int(ctx[b]))
    assert np.array_equal(d_ctx.cpu().numpy(), ctx + L + 1)
    same_bytes(bytes_of(cache), host)


def test_pages_beyond_32_bit_offsets():
    """A cache whose byte offsets pass 2^32: pages at its end are written and read."""
    m = d2sd()
    hkv, pages = 8, (1 << 32) // (8 * 1024) + 40
    k = torch.zeros((pages, hkv, 16, 64), dtype=torch.uint8, device="cuda")
    cache = m.Kv4Cache(k, torch.zeros_like(k), torch.zeros((pages, hkv, 16, 4), dtype=torch.uint8, device="cuda"),
                       torch.zeros((pages, hkv, 16, 4), dtype=torch.uint8, device="cuda"))
    table = dev(np.array([[pages - 1, 3, pages - 30]], np.int32))
    x = torch.randn((40, hkv, 128), device="cuda").bfloat16()
    ip, ctx = dev(np.array([0, 40], np.int32)), dev(np.zeros(1, np.int32))
    m.append_kv4(ip, 40, 40, x, -x, table, ctx, cache, 0)
    rk, rv = m.read_kv4(ip, 40, 40, table, cache, dtype=torch.float32)
    want = kv4.values(*kv4.quantise(x.double().cpu().numpy()))
    assert np.array_equal(rk.double().cpu().numpy(), want) and np.array_equal(rv.double().cpu().numpy(), -want)
    assert int(cache.k[4:pages - 30].max()) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_inconsistent_device_arrays_stay_inside(dtype):
    """Garbage offsets, lengths, pages and path nodes: nothing behind a buffer changes."""
    from tests.test_gpu_robustness import garbage_i32, guard_intact, guarded
    m, rng = d2sd(), np.random.default_rng(8)
    hkv, pages, B, total, batch = 3, 9, 16, 50, 4
    bufs = [guarded((pages, hkv, 16, n), torch.uint8, 0x5A) for n in (64, 64, 4, 4)]
    cache = m.Kv4Cache(*(t for _, t in bufs))
    k, v = (torch.randn((total, hkv, 128), device="cuda").to(TYPES[dtype]) for _ in range(2))
    table = garbage_i32(rng, batch * 20).view(batch, 20)
    for _ in range(3):
        ip, ctx = garbage_i32(rng, batch + 1), garbage_i32(rng, batch)
        m.append_kv4(ip, total, 30, k, v, table, ctx, cache, 200)
        m.commit_accepted_kv4(B, ip, total, garbage_i32(rng, batch * B).view(batch, B), garbage_i32(rng, batch), k, v, table,
                              garbage_i32(rng, batch), cache, 200)
        outs = [guarded((total, hkv, 128), TYPES[dtype], 7.0) for _ in range(2)]
        m.read_kv4(ip, total, 30, table, cache, start=garbage_i32(rng, batch), k_out=outs[0][1], v_out=outs[1][1])
        torch.cuda.synchronize()
        for buf, t in outs:
            assert guard_intact(buf, t.shape, 7.0)
        for buf, t in bufs:
            assert guard_intact(buf, t.shape, 0x5A)
