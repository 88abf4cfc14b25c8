"""Decoding cycles on a 4-bit cache: the prompt appended, then per cycle the
tree, the attention, adjusted logits, drawn targets, the accepted path, its
commit; eager against the oracles, and captured in a HIP graph."""

import numpy as np
import pytest
import torch

from oracle import kv4, logits as oracle_logits
from oracle.accept import accept_by_paths
from oracle.tree import build_tree
from tests.gpu_cases import d2sd
from tests.kv4_cases import check_request, dev, page_tables

pytestmark = pytest.mark.gpu
B, V, HQ, HKV = 8, 500, 8, 2


class Loop:
    def __init__(self, dtype, seed):
        rng = self.rng = np.random.default_rng(seed)
        self.m, self.dtype = d2sd(), dtype
        self.t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        self.prompt = np.array([37, 1, 64], np.int32)
        n = len(self.prompt)
        self.rows = [[2, 5], [], [1, 3, 4]]
        self.trees = [build_tree(B, r) for r in self.rows]
        K = np.array([len(r) for r in self.rows], np.int32)
        p = np.zeros((n, 3), np.int32)
        for b, r in enumerate(self.rows):
            p[b, :len(r)] = r
        self.ip, self.W = self.m.tree_plan(B, K, p)
        self.total, self.most = int(self.ip[-1]), int(np.diff(self.ip).max())
        self.K, self.p, self.d_ip = dev(K), dev(p), dev(self.ip)
        self.max_ctx = int(self.prompt.max()) + 4 * B
        self.table, self.pages = page_tables(np.full(n, self.max_ctx + B), rng)
        self.d_table = dev(self.table)
        self.cache = self.m.Kv4Cache.empty(self.pages, HKV)
        self.ctx = dev(np.zeros(n, np.int32))
        tip = np.concatenate([[0], np.cumsum(self.prompt)]).astype(np.int32)
        k, v = self.draw(int(tip[-1]), HKV), self.draw(int(tip[-1]), HKV)
        self.m.append_kv4(dev(tip), int(tip[-1]), int(self.prompt.max()), k, v, self.d_table, self.ctx, self.cache, 0)
        val = lambda x, b: kv4.values(*kv4.quantise(x[tip[b]:tip[b + 1]].double().cpu().numpy()))
        self.context = [[val(k, b), val(v, b)] for b in range(n)]         # what the cache should stand for
        self.history = rng.integers(0, V, (n, 200)).astype(np.int32)
        self.hist_len = self.prompt + 1                                   # the prompt and the first token

    def draw(self, n, h):
        return dev(self.rng.standard_normal((n, h, 128)).astype(np.float32)).to(self.t)

    def inputs(self):
        x = dict(q=self.draw(self.total, HQ), kt=self.draw(self.total, HKV), vt=self.draw(self.total, HKV))
        x["logits"] = dev((self.rng.standard_normal((self.total, V)) * 2).astype(np.float32))
        x["draft"] = dev(self.rng.integers(0, V, self.total).astype(np.int32))
        x["history"], x["hist_len"] = dev(self.history), dev(self.hist_len)
        return x

    def cycle(self, x, keep=None):
        m, keep = self.m, {} if keep is None else keep
        tree = m.tree_build(B, self.K, self.p, self.d_ip, self.total, self.W, out=keep.get("tree"))
        out, lse = m.cascade_verify_attention_kv4(
            x["q"], self.cache, self.d_table, self.ctx, x["kt"], x["vt"], self.d_ip, tree["anc_mask"], total_nodes=self.total,
            max_nodes=self.most, max_ctx_len=self.max_ctx, out=keep.get("out"), lse=keep.get("lse"), workspace=keep.get("ws"),
            kv_split=64)
        adj = m.adjust_logits(self.d_ip, self.total, self.most, tree["depth"], tree["anc_mask"], x["draft"], x["logits"],
                              history=x["history"], history_len=x["hist_len"], prompt_len=x["prompt_len"], repetition=x["rep"],
                              presence=x["pres"], out=keep.get("adj"))
        tok, _ = m.sample_targets(self.d_ip, self.total, self.most, tree["parent"], x["draft"], adj, 0.0, out=keep.get("tok"))
        acc = m.accept_path(B, self.d_ip, self.total, tree["parent"], tree["depth"], tree["path_id"], x["draft"], tok,
                            out=keep.get("acc"))
        m.commit_accepted_kv4(B, self.d_ip, self.total, acc["path_nodes"], acc["accept_len"], x["kt"], x["vt"], self.d_table,
                              self.ctx, self.cache, self.max_ctx)
        return dict(tree=tree, out=out, lse=lse, adj=adj, tok=tok, acc=acc)

    def penalties(self, x):
        x["rep"], x["pres"] = dev(np.array([1.3, 1.0, 1.1], np.float32)), dev(np.array([0.4, 0.0, -0.2], np.float32))
        x["prompt_len"] = dev(self.prompt)
        return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cycles(dtype):
    loop = Loop(dtype, 30)
    for _ in range(3):
        x = loop.penalties(loop.inputs())
        # the targets of a first pass become the drafts, so that paths are accepted
        adj = loop.m.adjust_logits(loop.d_ip, loop.total, loop.most, *(lambda t: (t["depth"], t["anc_mask"]))(
            loop.m.tree_build(B, loop.K, loop.p, loop.d_ip, loop.total, loop.W)), x["draft"], x["logits"], history=x["history"],
            history_len=x["hist_len"], prompt_len=x["prompt_len"], repetition=x["rep"], presence=x["pres"])
        top = adj.argmax(1).int().cpu().numpy()
        draft = x["draft"].cpu().numpy()
        for b, t in enumerate(loop.trees):
            for n in range(1, t.N):
                if loop.rng.random() < 0.8:
                    draft[loop.ip[b] + n] = top[loop.ip[b] + t.parent[n]]
        x["draft"] = dev(draft)
        r = loop.cycle(x)
        out, lse = r["out"].double().cpu().numpy(), r["lse"].double().cpu().numpy()
        for b, t in enumerate(loop.trees):
            s, e = loop.ip[b], loop.ip[b + 1]
            q, kt, vt = (x[n][s:e].double().cpu().numpy() for n in ("q", "kt", "vt"))
            check_request(out[s:e], lse[s:e], q, *loop.context[b], kt, vt, t, dtype)
            h, np_ = loop.history[b, :loop.hist_len[b]], loop.prompt[b]
            want = np.stack([oracle_logits.adjust_row(x["logits"][s + n].double().cpu().numpy(), h[:np_], h[np_:],
                                                      oracle_logits.path_tokens(t.parent, draft[s:e], n),
                                                      float(x["rep"][b]), float(x["pres"][b])) for n in range(t.N)])
            assert np.abs(r["adj"][s:e].double().cpu().numpy() - want).max() < 1e-5
            tok = want.argmax(1)
            rep = [next(m for m in range(n + 1) if oracle_logits.path_tokens(t.parent, draft[s:e], m) ==
                        oracle_logits.path_tokens(t.parent, draft[s:e], n)) for n in range(t.N)]
            tok = tok[rep]
            assert np.array_equal(r["tok"][s:e].cpu().numpy(), tok)
            a = accept_by_paths(t, draft[s:e], tok)
            assert int(r["acc"]["accept_len"][b]) == a.L
            new = r["acc"]["out_tokens"][b, :a.L + 1].cpu().numpy()
            assert new.tolist() == list(a.tokens)
            at = loop.hist_len[b]
            loop.history[b, at:at + a.L + 1] = new
            loop.hist_len[b] += a.L + 1
            for i, y in enumerate((kt, vt)):
                loop.context[b][i] = np.concatenate([loop.context[b][i], kv4.values(*kv4.quantise(y[list(a.path_nodes)]))])
        assert loop.ctx.cpu().tolist() == [len(c[0]) for c in loop.context]
        n = loop.ctx.cpu().numpy()
        tip = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        k, v = loop.m.read_kv4(dev(tip), int(tip[-1]), int(n.max()), loop.d_table, loop.cache, dtype=torch.float32)
        for i, y in enumerate((k, v)):
            assert np.array_equal(y.double().cpu().numpy(), np.concatenate([c[i] for c in loop.context]))


def test_captured_cycle():
    """Replays with eager work and synchronisations between them, each against the eager cycle."""
    loop = Loop("bf16", 31)
    x = loop.penalties(loop.inputs())
    ctx0 = loop.ctx.clone()
    held = ("k", "v", "k_scale", "v_scale")
    cache0 = [getattr(loop.cache, n).clone() for n in held]

    def reset():
        loop.ctx.copy_(ctx0)
        for n, t in zip(held, cache0):
            getattr(loop.cache, n).copy_(t)

    def flat(r):
        return [r["out"], r["lse"], r["adj"], r["tok"], *r["acc"].values(), loop.ctx, *(getattr(loop.cache, n) for n in held)]

    keep = loop.cycle(x)
    reset()
    keep["ws"] = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    keep["tok"] = torch.empty(loop.total, dtype=torch.int32, device="cuda")
    keep = {**keep, **{k: v for k, v in loop.cycle(x, keep).items() if k != "tok"}}
    torch.cuda.synchronize()
    want = [t.clone() for t in flat(keep)]
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loop.cycle(x, keep)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.cycle(x, keep)
    for _ in range(3):
        reset()
        keep["out"].fill_(float("nan"))
        keep["adj"].fill_(float("nan"))
        junk = torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(flat(keep), want):
            assert torch.equal(a, b)
        assert torch.isfinite(junk)
    reset()
    x["q"].mul_(0.5)                      # the graph reads the live inputs
    want = [t.clone() for t in flat({**keep, **loop.cycle(x, keep)})]
    reset()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(flat(keep), want):
        assert torch.equal(a, b)
