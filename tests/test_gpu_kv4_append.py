"""Appending to a 4-bit cache on both sides of the size from which a workgroup
per page takes over from one per request: the same bytes, the same clamps."""

import numpy as np
import pytest
import torch

from oracle import kv4
from tests.gpu_cases import d2sd
from tests.kv4_cases import bytes_of, dev, page_tables, random_cache

pytestmark = pytest.mark.gpu
SIZES = [(8, 24), (8, 25), (1, 192), (1, 193), (3, 64), (3, 65)]      # KV heads, most tokens: 192 rows and more


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hkv, most", SIZES)
def test_both_sides_of_the_size(hkv, most, dtype):
    m, rng = d2sd(), np.random.default_rng([60, hkv, most])
    ctx, lens = np.array([0, 17, 5, 31], np.int32), np.array([most, 0, 1, most - 1], np.int32)
    table, pages = page_tables(ctx + lens, rng)
    cache, host = random_cache(pages, hkv, rng)
    ip = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    k, v = (dev(rng.standard_normal((int(ip[-1]), hkv, 128)).astype(np.float32)).to(dtype) for _ in range(2))
    at = dev(ctx)
    m.append_kv4(dev(ip), int(ip[-1]), most, k, v, dev(table), at, cache, 31)
    for b in range(4):
        for n, x in (("k", k), ("v", v)):
            kv4.write_tokens((host[n], host[n + "_scale"]), x[ip[b]:ip[b + 1]].double().cpu().numpy(), table[b], int(ctx[b]))
    got = bytes_of(cache)
    for n in host:
        assert np.array_equal(got[n], host[n]), n
    assert np.array_equal(at.cpu().numpy(), ctx + lens)


@pytest.mark.parametrize("hkv, most", SIZES)
def test_past_the_table_and_garbage(hkv, most):
    """Tokens behind the last page are left out; garbage in the device arrays stays inside the cache."""
    from tests.test_gpu_robustness import garbage_i32, guard_intact, guarded
    m, rng = d2sd(), np.random.default_rng([61, hkv, most])
    pages = 20
    parts = {n: guarded((pages, hkv, 16, w), torch.uint8, 0x5A) for n, w in (("k", 64), ("v", 64), ("k_scale", 4), ("v_scale", 4))}
    cache = m.Kv4Cache(*(parts[n][1] for n in ("k", "v", "k_scale", "v_scale")))
    for _, t in parts.values():
        t.zero_()
    x = torch.randn((2 * most, hkv, 128), device="cuda").bfloat16()
    table = dev(np.arange(20, dtype=np.int32).reshape(2, 10)[:, :(most + 15) // 16 if most < 160 else 10])
    room = table.shape[1] * 16
    most_in = min(most, room)
    ip, ctx = dev(np.array([0, most_in, 2 * most_in], np.int32)), dev(np.array([room - 3, 0], np.int32))
    m.append_kv4(ip, 2 * most_in, most_in, x[:2 * most_in], x[:2 * most_in], table, ctx, cache, room)
    assert ctx.cpu().tolist() == [room, most_in]
    k, v = m.read_kv4(dev(np.array([0, 3], np.int32)), 3, 3, table[:1], cache, start=dev(np.array([room - 3], np.int32)))
    want = torch.from_numpy(kv4.values(*kv4.quantise(x[:3].double().cpu().numpy())))
    assert torch.equal(k.double().cpu(), want) and torch.equal(v.double().cpu(), want)
    for _ in range(3):
        m.append_kv4(garbage_i32(rng, 3), 2 * most_in, most_in, x[:2 * most_in], x[:2 * most_in],
                     garbage_i32(rng, table.numel()).view(table.shape), garbage_i32(rng, 2), cache, room)
    torch.cuda.synchronize()
    for buf, t in parts.values():
        assert guard_intact(buf, t.shape, 0x5A)
