"""Shared set-up of the GPU tests of the 4-bit cache."""

from __future__ import annotations

import numpy as np
import torch

from oracle import kv4
from oracle.attention import request_attention
from tests.gpu_cases import d2sd


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def page_tables(lengths, rng, spare=2):
    """A table over a permuted pool with pages for `lengths` positions, and the pool's size."""
    n = [max(1, (int(c) + 15) // 16) for c in lengths]
    pool = rng.permutation(sum(n) + spare)
    table = np.zeros((len(n), max(n)), np.int32)
    for b, k in enumerate(n):
        table[b, :k] = pool[sum(n[:b]):sum(n[:b + 1])]
    return table, sum(n) + spare


def random_cache(pages, hkv, rng, spread=1):
    """A cache of random codes whose scales are near 2^-2 (unit values); returns (Kv4Cache, host arrays)."""
    u = lambda n: rng.integers(0, 256, (pages, hkv, 16, n), dtype=np.uint8)
    s = lambda: rng.integers(125 - spread, 126 + spread, (pages, hkv, 16, 4)).astype(np.uint8)
    host = dict(k=u(64), v=u(64), k_scale=s(), v_scale=s())
    return d2sd().Kv4Cache(*(dev(host[n]) for n in ("k", "v", "k_scale", "v_scale"))), host


def bytes_of(cache):
    return {n: getattr(cache, n).cpu().numpy() for n in ("k", "v", "k_scale", "v_scale")}


def gather(host, name, table_row, start, n):
    """float64 values [n, hkv, 128] of positions start .. start + n - 1."""
    at = np.arange(start, start + n)
    pages = table_row[at // 16]
    return kv4.values(host[name][pages, :, at % 16], host[name + "_scale"][pages, :, at % 16])


def tolerance(q, keys, vals, out_abs, scale, dtype, n_keys):
    """Bound of an output element's and of lse's error by the arithmetic used.

    A score is off by at most delta: three (bf16) or five (fp32) query terms
    leave, per element, half a unit of the last term, and a unit is at most
    2^-(4 + 5 (n - 1)) of the power of two above the block's largest, itself at
    most twice that. The sums over 128 dims and over the keys are fp32. A
    weight is off by delta relatively, plus 2^-8 from its rounding to bf16 (8
    significant bits: values in [1, 2) are 2^-7 apart; fp32: 2^-24 per term), and
    the output's own rounding is 2^-8 or 2^-24 of it; out_abs is sum p |v| >= |out|."""
    terms = 3 if dtype == "bf16" else 5
    blocks = np.abs(q).reshape(*q.shape[:-1], 4, 32).max(-1)
    cut = 2 * 2.0 ** -(5 * terms - 1) * 0.5
    key = np.abs(keys).reshape(-1, 4, 32).sum(-1).max(0) if len(keys) else np.zeros(4)
    # fp32 sums: each product and partial sum relative to sum |q k|
    size = (blocks * key).sum(-1).max(initial=0.0) * scale
    delta = cut * size + 2.0 ** -24 * 16 * size
    eps = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    sums = (n_keys + 64) * 2.0 ** -24
    out = out_abs * ((2 * delta + sums) * 1.01 + 2 * eps * 1.01) + 1e-30
    return out, delta + sums + 2.0 ** -21 * 12


def check_request(got, lse, q, kc, vc, kt, vt, tree, dtype, stage="cascade"):
    """One request's outputs against the float64 oracle within the derived bound."""
    scale = 1.0 / np.sqrt(q.shape[-1])
    want, want_lse = request_attention(q, kc, vc, kt, vt, tree, stage)
    mag, _ = request_attention(q, kc, np.abs(vc), kt, np.abs(vt), tree, stage)
    G = q.shape[1] // kt.shape[1]
    for h in range(q.shape[1]):
        keys = np.concatenate([kc[:, h // G], kt[:, h // G]]) if stage != "prefix" else kc[:, h // G]
        tol, tol_lse = tolerance(q[:, h], keys, None, mag[:, h], scale, dtype, len(keys))
        off = np.abs(got[:, h] - want[:, h])
        assert (off <= tol).all(), (h, (off / tol).max())
        empty = np.isneginf(want_lse[:, h])
        assert np.array_equal(empty, np.isneginf(lse[:, h]))
        off = np.abs(lse[~empty, h] - want_lse[~empty, h])
        assert (off <= tol_lse).all(), (h, off.max(), tol_lse)
        assert (got[empty, h] == 0).all()
