"""Refusals of the 4-bit cache and logit entry points (CPU: nothing is launched)."""

import ctypes

import pytest
import torch

from tests.test_abi import FAKE, d2sd, good_args

lib = d2sd._lib
P = ctypes.c_void_p
INVALID, UNSUPPORTED, SMALL = d2sd.ERR_INVALID_ARG, d2sd.ERR_UNSUPPORTED, d2sd.ERR_WORKSPACE_TOO_SMALL


def cache(**kw):
    f = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE)
    f.update(kw)
    return d2sd.Kv4Pointers(f["k"], f["v"], f["k_scale"], f["v_scale"])


def fill(defaults, kw):
    unknown = set(kw) - set(defaults)
    assert not unknown, unknown
    return {**defaults, **kw}


def append(**kw):
    a = fill(dict(batch=2, hkv=8, head_dim=128, page=16, dtype=d2sd.BF16, pages=64, max_pages=32, max_ctx=100, indptr=FAKE,
                  total=40, most=30, k=FAKE, v=FAKE, table=FAKE, ctx=FAKE, cache=cache()), kw)
    c = None if a["cache"] is None else ctypes.byref(a["cache"])
    return lib.d2sd_append_kv4(a["batch"], a["hkv"], a["head_dim"], a["page"], a["dtype"], a["pages"], a["max_pages"],
                               a["max_ctx"], a["indptr"], a["total"], a["most"], a["k"], a["v"], a["table"], a["ctx"], c, None)


def commit(**kw):
    a = fill(dict(batch=2, B=16, hkv=8, head_dim=128, page=16, dtype=d2sd.BF16, pages=64, max_pages=32, max_ctx=100,
                  indptr=FAKE, total=40, path=FAKE, length=FAKE, k=FAKE, v=FAKE, table=FAKE, ctx=FAKE, cache=cache()), kw)
    c = None if a["cache"] is None else ctypes.byref(a["cache"])
    return lib.d2sd_commit_accepted_kv4(a["batch"], a["B"], a["hkv"], a["head_dim"], a["page"], a["dtype"], a["pages"],
                                        a["max_pages"], a["max_ctx"], a["indptr"], a["total"], a["path"], a["length"], a["k"],
                                        a["v"], a["table"], a["ctx"], c, None)


def read(**kw):
    a = fill(dict(batch=2, hkv=8, head_dim=128, page=16, dtype=d2sd.BF16, pages=64, max_pages=32, indptr=FAKE, total=40,
                  most=30, start=None, table=FAKE, cache=cache(), k=FAKE, v=FAKE), kw)
    c = None if a["cache"] is None else ctypes.byref(a["cache"])
    return lib.d2sd_read_kv4(a["batch"], a["hkv"], a["head_dim"], a["page"], a["dtype"], a["pages"], a["max_pages"],
                             a["indptr"], a["total"], a["most"], a["start"], a["table"], c, a["k"], a["v"], None)


SIZES = [(dict(batch=0), INVALID), (dict(hkv=0), INVALID), (dict(hkv=70000), UNSUPPORTED), (dict(head_dim=64), UNSUPPORTED),
         (dict(page=32), UNSUPPORTED), (dict(dtype=2), INVALID), (dict(pages=0), INVALID), (dict(max_pages=0), INVALID),
         (dict(max_pages=1 << 27), UNSUPPORTED), (dict(total=-1), INVALID), (dict(indptr=None), INVALID),
         (dict(table=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(cache=None), INVALID),
         (dict(k=FAKE + 8), INVALID), (dict(v=FAKE + 2), INVALID), (dict(cache=cache(k=None)), INVALID),
         (dict(cache=cache(v_scale=None)), INVALID), (dict(cache=cache(v=FAKE + 8)), INVALID),
         (dict(cache=cache(k_scale=FAKE + 2)), INVALID)]
TOKENS = [(dict(most=-1), INVALID), (dict(most=41), INVALID), (dict(most=0), INVALID), (dict(total=600, most=513), INVALID)]


@pytest.mark.parametrize("kw, status", SIZES + TOKENS + [
    (dict(ctx=None), INVALID), (dict(max_ctx=-1), INVALID), (dict(max_ctx=513), INVALID)])
def test_append_refuses(kw, status):
    assert append(**kw) == status and d2sd.last_error()


@pytest.mark.parametrize("kw, status", SIZES + [
    (dict(B=1), INVALID), (dict(B=65), INVALID), (dict(ctx=None), INVALID), (dict(path=None), INVALID),
    (dict(length=None), INVALID), (dict(max_ctx=-1), INVALID), (dict(max_ctx=512 - 15), INVALID)])
def test_commit_refuses(kw, status):
    assert commit(**kw) == status and d2sd.last_error()


@pytest.mark.parametrize("kw, status", SIZES + TOKENS)
def test_read_refuses(kw, status):
    assert read(**kw) == status and d2sd.last_error()


def test_calls_without_tokens_launch_nothing():
    assert append(total=0, most=0, k=None, v=None) == d2sd.OK
    assert read(total=0, most=0, k=None, v=None) == d2sd.OK


def test_too_many_pages_for_one_call():
    assert read(batch=1 << 20, total=1 << 20, most=500) == UNSUPPORTED


def attn(**kw):
    return good_args(**{"k_cache": None, "v_cache": None, **kw})


def call(a, c=None, ws=None, n=0):
    c = cache() if c is None else c
    return lib.d2sd_cascade_verify_attention_kv4(ctypes.byref(a), ctypes.byref(c), ws, n, None)


def need(a):
    n = ctypes.c_size_t(7)
    return lib.d2sd_cascade_workspace_size_kv4(ctypes.byref(a), ctypes.byref(n)), n.value


@pytest.mark.parametrize("kw, status", [
    (dict(k_cache=FAKE), INVALID), (dict(v_cache=FAKE), INVALID), (dict(row_group=128), INVALID), (dict(packed=1), INVALID),
    (dict(head_dim=64), UNSUPPORTED), (dict(page_size=32), UNSUPPORTED), (dict(dtype=3), INVALID), (dict(stage=3), INVALID),
    (dict(kv_split=63), INVALID), (dict(kv_split=32832), INVALID), (dict(batch=0), INVALID), (dict(num_qo_heads=12), INVALID),
    (dict(mask_words=1, max_nodes=60), INVALID)])
def test_attention_sizes_are_refused(kw, status):
    assert need(attn(**kw))[0] == status
    assert call(attn(**kw), ws=FAKE, n=1 << 40) == status


@pytest.mark.parametrize("name", ["q", "page_table", "ctx_len", "k_tree", "v_tree", "node_indptr", "anc_mask", "out"])
def test_attention_pointers_are_refused(name):
    assert call(attn(**{name: None}), ws=FAKE, n=1 << 40) == INVALID
    if name in ("q", "k_tree", "v_tree", "out"):
        assert call(attn(**{name: FAKE + 8}), ws=FAKE, n=1 << 40) == INVALID


def test_attention_cache_and_workspace_are_refused():
    a = attn()
    assert lib.d2sd_cascade_verify_attention_kv4(ctypes.byref(a), None, FAKE, 1 << 40, None) == INVALID
    assert call(a, cache(v=None), FAKE, 1 << 40) == INVALID
    assert call(a, cache(k_scale=FAKE + 1), FAKE, 1 << 40) == INVALID
    a = attn(kv_split=64)
    st, n = need(a)
    assert st == d2sd.OK and n > 0
    assert call(a, ws=FAKE, n=n - 1) == SMALL
    assert call(a, ws=None, n=n) == SMALL
    assert call(a, ws=FAKE + 4, n=n + 64) == INVALID


def test_calls_without_rows_or_context_need_no_workspace():
    assert need(attn(total_nodes=0, max_nodes=0)) == (d2sd.OK, 0)
    assert need(attn(max_ctx_len=0)) == (d2sd.OK, 0)
    assert need(attn(stage=d2sd.STAGE_TREE)) == (d2sd.OK, 0)
    assert call(attn(total_nodes=0, max_nodes=0)) == d2sd.OK


def logits_args(**kw):
    f = dict(batch=2, total_nodes=20, max_nodes=12, mask_words=1, vocab=100, dtype=d2sd.F32, max_history=5, max_bias=3,
             num_masks=2)
    f.update({n: FAKE for n, _ in d2sd.LogitsArgs._fields_ if n not in f})
    f.update(kw)
    return d2sd.LogitsArgs(*[f[n] for n, _ in d2sd.LogitsArgs._fields_])


@pytest.mark.parametrize("kw, status", [
    (dict(batch=0), INVALID), (dict(total_nodes=-1), INVALID), (dict(max_nodes=0), INVALID), (dict(max_nodes=2081, mask_words=66), INVALID),
    (dict(mask_words=0), INVALID), (dict(max_nodes=33), INVALID), (dict(vocab=0), INVALID), (dict(vocab=(1 << 20) + 1), INVALID),
    (dict(dtype=2), INVALID), (dict(max_history=-1), INVALID), (dict(max_bias=-1), INVALID), (dict(num_masks=-1), INVALID),
    (dict(node_indptr=None), INVALID), (dict(depth=None), INVALID), (dict(anc_mask=None), INVALID),
    (dict(draft_tokens=None), INVALID), (dict(logits=None), INVALID), (dict(out=None), INVALID), (dict(history=None), INVALID),
    (dict(history_len=None), INVALID), (dict(bias_token=None), INVALID), (dict(bias_value=None), INVALID),
    (dict(token_mask=None), INVALID), (dict(mask_row=None), INVALID), (dict(logits=FAKE + 4), INVALID),
    (dict(out=FAKE + 8), INVALID), (dict(batch=1 << 20, vocab=1 << 20), UNSUPPORTED)])
def test_adjust_logits_refuses(kw, status):
    assert lib.d2sd_adjust_logits(ctypes.byref(logits_args(**kw)), None) == status and d2sd.last_error()


def test_adjust_logits_null_args_and_no_rows():
    assert lib.d2sd_adjust_logits(None, None) == INVALID
    assert lib.d2sd_adjust_logits(ctypes.byref(logits_args(total_nodes=0)), None) == d2sd.OK


def test_binding_refuses_before_the_library():
    u8 = torch.uint8
    k, s = torch.zeros((3, 2, 16, 64), dtype=u8), torch.zeros((3, 2, 16, 4), dtype=u8)
    for bad in ((k[:, :, :8], k, s, s), (k, k[:2], s, s), (k, k, s[..., :2], s), (k, k, s, k)):
        with pytest.raises(ValueError):
            d2sd.Kv4Cache(*bad)
    with pytest.raises(ValueError, match="device"):
        d2sd.Kv4Cache(k, k, s, s)                          # host tensors
    with pytest.raises(ValueError, match="dtype"):
        d2sd.adjust_logits(torch.zeros(2), 1, 1, None, None, None, torch.zeros((1, 8), dtype=torch.float16))
    with pytest.raises(ValueError, match="logits must be"):
        d2sd.adjust_logits(torch.zeros(2), 4, 1, None, None, None, torch.zeros((1, 8)))
