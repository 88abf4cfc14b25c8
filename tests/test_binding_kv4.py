"""What the binding of the 4-bit cache refuses, and what it hands to the library:
device tensors are stood in for by their sizes, and the library by a recorder, so
that nothing is launched."""

import pytest
import torch

from paper_2606_04446_amd import d2sd

I32, U8, BF16, F32 = torch.int32, torch.uint8, torch.bfloat16, torch.float32


class Tensor:
    """A contiguous device tensor without data."""

    is_cuda = True

    def __init__(self, *shape, dtype=I32, at=0):
        self.shape, self.dtype, self.at = torch.Size(shape), dtype, at
        self.device = torch.device("cuda", at)

    def get_device(self):
        return self.at

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return torch.empty((), dtype=self.dtype).element_size()

    def dim(self):
        return len(self.shape)

    def size(self, i):
        return self.shape[i]

    def data_ptr(self):
        return 1 << 20


def cache(pages=9, heads=2, at=0):
    k = lambda n: Tensor(pages, heads, 16, n, dtype=U8, at=at)
    return d2sd.Kv4Cache(k(64), k(64), k(4), k(4))


@pytest.fixture
def calls(monkeypatch):
    """Arguments of the library calls that get through."""
    got = []
    for name in ("_append_kv4", "_commit_kv4", "_read_kv4", "_cascade_kv4", "_ws_size_kv4", "_adjust"):
        monkeypatch.setattr(d2sd, name, lambda *a: got.append(a) or d2sd.OK)
    monkeypatch.setattr(d2sd, "_current_device", lambda: 0)
    monkeypatch.setattr(d2sd, "_stream", lambda s: 0)
    return got


def read(**kw):
    a = dict(token_indptr=Tensor(4), total_tokens=20, max_tokens=9, page_table=Tensor(3, 5), cache=cache(), start=None,
             k_out=Tensor(20, 2, 128, dtype=BF16), v_out=Tensor(20, 2, 128, dtype=BF16))
    return d2sd.read_kv4(**{**a, **kw})


@pytest.mark.parametrize("kw", [dict(), dict(page_table=Tensor(8, 5)), dict(start=Tensor(3)), dict(start=Tensor(8))])
def test_read_counts_the_requests_by_their_offsets(calls, kw):
    """A page table with rows to spare asks for no more requests than token_indptr has."""
    read(**kw)
    assert len(calls) == 1 and calls[0][0] == 3 and calls[0][6] == 5


@pytest.mark.parametrize("kw, what", [
    (dict(page_table=Tensor(2, 5)), "page_table"), (dict(page_table=Tensor(15)), "page_table"),
    (dict(start=Tensor(2)), "start"), (dict(k_out=Tensor(19, 2, 128, dtype=BF16)), "k_out"),
    (dict(v_out=Tensor(20, 1, 128, dtype=BF16)), "v_out"), (dict(v_out=Tensor(20, 2, 128, dtype=F32)), "v_out")])
def test_read_refuses_short_tensors(calls, kw, what):
    with pytest.raises(ValueError, match=what):
        read(**kw)
    assert not calls


def append(**kw):
    a = dict(token_indptr=Tensor(4), total_tokens=20, max_tokens=9, k=Tensor(20, 2, 128, dtype=BF16),
             v=Tensor(20, 2, 128, dtype=BF16), page_table=Tensor(3, 5), ctx_len=Tensor(3), cache=cache(), max_ctx_len=70)
    return d2sd.append_kv4(**{**a, **kw})


@pytest.mark.parametrize("kw", [dict(), dict(page_table=Tensor(8, 5)), dict(token_indptr=Tensor(9))])
def test_append_takes_longer_tensors(calls, kw):
    append(**kw)
    assert len(calls) == 1 and calls[0][0] == 3 and calls[0][6] == 5


@pytest.mark.parametrize("kw, what", [
    (dict(token_indptr=Tensor(3)), "token_indptr"), (dict(page_table=Tensor(2, 5)), "page_table"),
    (dict(page_table=Tensor(15)), "page_table"), (dict(k=Tensor(19, 2, 128, dtype=BF16)), "k must"),
    (dict(v=Tensor(20, 2, 64, dtype=BF16)), "v must"), (dict(v=Tensor(20, 2, 128, dtype=F32)), "v dtype")])
def test_append_refuses_short_tensors(calls, kw, what):
    with pytest.raises(ValueError, match=what):
        append(**kw)
    assert not calls


def commit(**kw):
    a = dict(B=4, node_indptr=Tensor(4), total_nodes=20, path_nodes=Tensor(3, 4), accept_len=Tensor(3),
             k_tree=Tensor(20, 2, 128, dtype=F32), v_tree=Tensor(20, 2, 128, dtype=F32), page_table=Tensor(3, 5),
             ctx_len=Tensor(3), cache=cache(), max_ctx_len=70)
    return d2sd.commit_accepted_kv4(**{**a, **kw})


@pytest.mark.parametrize("kw", [
    dict(), dict(page_table=Tensor(8, 5)), dict(node_indptr=Tensor(9)), dict(accept_len=Tensor(4)), dict(path_nodes=Tensor(6, 4)),
    dict(k_tree=Tensor(32, 2, 128, dtype=F32)), dict(v_tree=Tensor(21, 2, 128, dtype=F32))])
def test_commit_takes_longer_tensors(calls, kw):
    """As a captured step's buffers are."""
    commit(**kw)
    assert len(calls) == 1 and calls[0][0] == 3 and calls[0][7] == 5 and calls[0][10] == 20


@pytest.mark.parametrize("kw, what", [
    (dict(node_indptr=Tensor(3)), "node_indptr"), (dict(page_table=Tensor(2, 5)), "page_table"),
    (dict(path_nodes=Tensor(3, 3)), "path_nodes"), (dict(path_nodes=Tensor(3, 5)), "path_nodes"), (dict(accept_len=Tensor(2)), "accept_len"),
    (dict(k_tree=Tensor(19, 2, 128, dtype=F32)), "k_tree"), (dict(k_tree=Tensor(20, 8, 128, dtype=F32)), "k_tree"),
    (dict(v_tree=Tensor(19, 2, 128, dtype=F32)), "v_tree"), (dict(v_tree=Tensor(20, 2, 64, dtype=F32)), "v_tree"),
    (dict(v_tree=Tensor(20, 2, 128, dtype=BF16)), "v_tree"), (dict(k_tree=Tensor(20, 2, 128, dtype=torch.float16)), "k_tree")])
def test_commit_refuses_short_tensors(calls, kw, what):
    with pytest.raises(ValueError, match=what):
        commit(**kw)
    assert not calls


def attend(**kw):
    a = dict(q=Tensor(20, 8, 128, dtype=BF16), cache=cache(), page_table=Tensor(3, 5), ctx_len=Tensor(3),
             k_tree=Tensor(20, 2, 128, dtype=BF16), v_tree=Tensor(20, 2, 128, dtype=BF16), node_indptr=Tensor(4),
             anc_mask=Tensor(20, 1), total_nodes=20, max_nodes=9, max_ctx_len=70, out=Tensor(20, 8, 128, dtype=BF16),
             lse=Tensor(20, 8, dtype=F32), workspace=Tensor(64, dtype=U8))
    return d2sd.cascade_verify_attention_kv4(**{**a, **kw})


@pytest.mark.parametrize("kw", [
    dict(), dict(page_table=Tensor(8, 5)), dict(node_indptr=Tensor(9)), dict(q=Tensor(32, 8, 128, dtype=BF16)),
    dict(k_tree=Tensor(32, 2, 128, dtype=BF16)), dict(v_tree=Tensor(21, 2, 128, dtype=BF16)), dict(anc_mask=Tensor(32, 1)),
    dict(out=Tensor(32, 8, 128, dtype=BF16)), dict(lse=Tensor(400, dtype=F32)), dict(lse=None, want_lse=False),
    dict(stage=d2sd.STAGE_PREFIX, k_tree=Tensor(1, dtype=BF16), v_tree=Tensor(1, dtype=BF16), anc_mask=None)])
def test_attention_takes_longer_tensors(calls, kw):
    attend(**kw)
    a = calls[0][0]._obj
    assert len(calls) == 1 and (a.batch, a.num_qo_heads, a.num_kv_heads, a.max_pages, a.total_nodes) == (3, 8, 2, 5, 20)


@pytest.mark.parametrize("kw, what", [
    (dict(q=Tensor(19, 8, 128, dtype=BF16)), "q must"), (dict(q=Tensor(20, 8, 64, dtype=BF16)), "q must"),
    (dict(q=Tensor(20, 8, 128, dtype=torch.float16)), "q dtype"),
    (dict(out=Tensor(19, 8, 128, dtype=BF16)), "out"), (dict(out=Tensor(20, 4, 128, dtype=BF16)), "out"),
    (dict(out=Tensor(20, 8, 128, dtype=F32)), "out"), (dict(lse=Tensor(20, 4, dtype=F32)), "lse"),
    (dict(lse=Tensor(20, 8, dtype=BF16)), "lse"), (dict(k_tree=Tensor(19, 2, 128, dtype=BF16)), "k_tree"),
    (dict(k_tree=Tensor(20, 8, 128, dtype=BF16)), "k_tree"), (dict(v_tree=Tensor(20, 1, 128, dtype=BF16)), "v_tree"),
    (dict(v_tree=Tensor(20, 2, 128, dtype=F32)), "v_tree"), (dict(page_table=Tensor(2, 5)), "page_table"),
    (dict(node_indptr=Tensor(3)), "node_indptr"), (dict(anc_mask=Tensor(19, 1)), "anc_mask"),
    (dict(stage=d2sd.STAGE_TREE, anc_mask=Tensor(19, 1)), "anc_mask"),
    (dict(stage=d2sd.STAGE_PREFIX, q=Tensor(19, 8, 128, dtype=BF16)), "q must")])
def test_attention_refuses_short_tensors(calls, kw, what):
    with pytest.raises(ValueError, match=what):
        attend(**kw)
    assert not calls


def adjust(**kw):
    i, f = Tensor(3), Tensor(3, dtype=F32)
    a = dict(node_indptr=Tensor(4), total_nodes=20, max_nodes=9, depth=Tensor(20), anc_mask=Tensor(20, 1), draft_tokens=Tensor(20),
             logits=Tensor(20, 100, dtype=F32), history=Tensor(3, 7), history_len=i, prompt_len=i, repetition=f, presence=f,
             frequency=f, bias_token=Tensor(3, 2), bias_value=Tensor(3, 2, dtype=F32), bias_len=i, token_mask=Tensor(5, 4),
             mask_row=Tensor(20), out=Tensor(20, 100, dtype=F32))
    a = {**a, **kw}
    first = [a.pop(n) for n in ("node_indptr", "total_nodes", "max_nodes", "depth", "anc_mask", "draft_tokens", "logits")]
    return d2sd.adjust_logits(*first, **a)


CALLS = {"append": append, "commit": commit, "read": read, "attend": attend, "adjust": adjust}


@pytest.mark.parametrize("call, name, shape, dtype", [
    (call, name, shape, dtype) for call, names in {
        "append": [("token_indptr", (4,), I32), ("k", (20, 2, 128), BF16), ("v", (20, 2, 128), BF16), ("page_table", (3, 5), I32),
                   ("ctx_len", (3,), I32)],
        "commit": [("node_indptr", (4,), I32), ("path_nodes", (3, 4), I32), ("accept_len", (3,), I32), ("k_tree", (20, 2, 128), F32),
                   ("v_tree", (20, 2, 128), F32), ("page_table", (3, 5), I32), ("ctx_len", (3,), I32)],
        "read": [("token_indptr", (4,), I32), ("start", (3,), I32), ("page_table", (3, 5), I32), ("k_out", (20, 2, 128), BF16),
                 ("v_out", (20, 2, 128), BF16)],
        "attend": [("q", (20, 8, 128), BF16), ("page_table", (3, 5), I32), ("ctx_len", (3,), I32), ("k_tree", (20, 2, 128), BF16),
                   ("v_tree", (20, 2, 128), BF16), ("node_indptr", (4,), I32), ("anc_mask", (20, 1), I32),
                   ("out", (20, 8, 128), BF16), ("lse", (20, 8), F32), ("workspace", (64,), U8)],
        "adjust": [("node_indptr", (4,), I32), ("depth", (20,), I32), ("anc_mask", (20, 1), I32), ("draft_tokens", (20,), I32),
                   ("logits", (20, 100), F32), ("history", (3, 7), I32), ("history_len", (3,), I32), ("prompt_len", (3,), I32),
                   ("repetition", (3,), F32), ("presence", (3,), F32), ("frequency", (3,), F32), ("bias_token", (3, 2), I32),
                   ("bias_value", (3, 2), F32), ("bias_len", (3,), I32), ("token_mask", (5, 4), I32), ("mask_row", (20,), I32),
                   ("out", (20, 100), F32)]}.items() for name, shape, dtype in names])
def test_a_tensor_of_another_device_is_refused(calls, call, name, shape, dtype):
    with pytest.raises(ValueError, match="current device"):
        CALLS[call](**{name: Tensor(*shape, dtype=dtype, at=1)})
    assert not calls
    CALLS[call]()
    assert len(calls) == 1


@pytest.mark.parametrize("call", ["append", "commit", "read", "attend"])
def test_a_cache_of_another_device_is_refused(calls, call):
    with pytest.raises(ValueError, match="current device"):
        CALLS[call](cache=cache(at=1))
    assert not calls


@pytest.mark.parametrize("kw", [dict(), dict(anc_mask=Tensor(32, 1)), dict(depth=Tensor(32)), dict(mask_row=Tensor(21)),
                                dict(logits=Tensor(24, 100, dtype=F32), out=Tensor(24, 100, dtype=F32))])
def test_adjust_takes_longer_tensors(calls, kw):
    adjust(**kw)
    a = calls[0][0]._obj
    assert len(calls) == 1 and (a.batch, a.total_nodes, a.vocab, a.num_masks, a.max_history) == (3, 20, 100, 5, 7)


@pytest.mark.parametrize("kw, what", [
    (dict(anc_mask=Tensor(19, 1)), "anc_mask"), (dict(anc_mask=Tensor(20)), "anc_mask"), (dict(depth=Tensor(19)), "depth"),
    (dict(draft_tokens=Tensor(19)), "draft_tokens"), (dict(mask_row=Tensor(19)), "mask_row"), (dict(token_mask=Tensor(5, 3)), "token_mask"),
    (dict(token_mask=Tensor(20)), "token_mask"), (dict(history=Tensor(2, 7)), "history"), (dict(history_len=Tensor(2)), "history_len"),
    (dict(prompt_len=Tensor(2)), "prompt_len"), (dict(repetition=Tensor(2, dtype=F32)), "repetition"),
    (dict(presence=Tensor(2, dtype=F32)), "presence"), (dict(frequency=Tensor(2, dtype=F32)), "frequency"),
    (dict(bias_len=Tensor(2)), "bias_len"), (dict(bias_value=Tensor(3, 1, dtype=F32)), "bias_value"), (dict(bias_value=None), "bias_value"),
    (dict(bias_token=Tensor(2, 2)), "bias_token"), (dict(logits=Tensor(19, 100, dtype=F32)), "logits"),
    (dict(out=Tensor(20, 99, dtype=F32)), "out"), (dict(out=Tensor(20, 100, dtype=BF16)), "out")])
def test_adjust_refuses_short_tensors(calls, kw, what):
    with pytest.raises(ValueError, match=what):
        adjust(**kw)
    assert not calls


def test_adjust_refuses_host_tensors_where_there_is_no_device(monkeypatch):
    def none():
        raise RuntimeError("no device")
    monkeypatch.setattr(d2sd, "_current_device", none)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="logits must be a device tensor"):
        d2sd.adjust_logits(i, 1, 1, i, torch.zeros((1, 1), dtype=torch.int32), i, torch.zeros((1, 8)))
