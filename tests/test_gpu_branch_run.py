"""The branching operators together, as a decoding program uses them: trees verified by a model's step or by the operators
alone, accepted paths kept, sequences forked; captured calls, streams and the binding's refusals."""
import numpy as np
import pytest

import synth
from branch_util import ancestors, trees
from gpu_util import build_pair, dev_i32, tol
from test_gpu_batch_step import Batch, PAGE
from test_gpu_branch import attn_case, i32, logits_of, random_sets, run_tree, sets_to_mask

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dl():
    import paper_2606_13740_amd as pkg
    return pkg


def apart(a, b):
    """Differences of logits; the MASK id's -inf is on both sides."""
    assert np.array_equal(np.isfinite(a), np.isfinite(b))
    return abs(a[np.isfinite(a)] - b[np.isfinite(b)])


def paths_of(parents):
    """Each row's path from the text: its ancestors in order, itself last."""
    return [sorted(s) for s in ancestors(parents)]


class TreeBatch(Batch):
    """A batch whose steps draft trees."""

    def tree_step(self, toks, parents, logits, out=True):
        """One step over a tree a sequence (rows not committed) -> (ids, log probabilities of the drafts' own tokens given their parents)."""
        import torch
        dl, new = self.dl, np.array([len(p) for p in parents])
        R, ld = int(new.sum()), max(1, -(-int(new.max()) // 32))
        z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
        p = dict(row0=z(self.B + 1), pos=z(R), slot=z(R), seq=z(R), lim=z(R), status=z(3))
        owned, n_free = z(self.B), z(1)
        dl.dllm_batch_plan(dev_i32(self.len), dev_i32(new), self.owned, owned, self.table, self.free, self.n_free, n_free, PAGE,
                           self.shared // PAGE, p["row0"], p["pos"], p["slot"], p["seq"], p["lim"], p["status"])
        assert p["status"][2].item() == 0
        self.owned, self.n_free = owned, n_free
        total, pos, mask = self.len + new, z(R), z(R, ld)
        dl.dllm_tree_plan(dev_i32(np.concatenate(parents)), p["row0"], dev_i32(total), pos, mask)
        ids, conf = z(R), torch.zeros(R, device="cuda")
        control = dict(mask_id=self.model.shape.mask_id)
        dl.dllm_batch_step_tree(self.model.handle, self.pages, self.n_pages, PAGE, dev_i32(np.concatenate(toks)), None, mask, self.table,
                                p["row0"], pos, p["slot"], dev_i32(total), int(max(new)), int(max(total)), ids if out else None,
                                conf if out else None, shared_len=self.shared, logits=logits if out else None, control=control if out else None)
        return ids

    def cache(self):
        """The pages as [layers][2][n_pages][kv_heads][page * head_dim]."""
        import torch
        sh = self.model.shape
        t = self.pages.view(torch.float32 if self.model.dtype == "f32" else torch.float16)
        return t.view(sh.n_layers, 2, self.n_pages, getattr(sh, "kv_heads", sh.n_heads), PAGE * sh.head_dim)


@pytest.mark.parametrize("shape,dtype", [(synth.TINY, "f32"), (synth.TINY_GQA, "f32"), (synth.SMALL_BF16, "bf16"), (synth.SMALL_MQA, "q4")])
def test_a_tree_step_is_the_step_of_every_path(dl, shape, dtype):
    """Logits of a tree's rows against steps over each path as a window of its own: in a bidirectional window a row would see
    its descendants, so the windows run with causal limits; then the accepted path's K/V, compacted, serve the next step
    as if it had been appended."""
    import torch
    model, _, _ = build_pair(shape, dtype, oracle_too=False)
    rng = np.random.default_rng(0)
    prompt = synth.prompt_ids(shape, 75)
    rows = [9, 0, 13]
    parents = [np.array(p, dtype=int) for p in trees(rng, rows, back=4)]
    toks = [rng.integers(0, shape.mask_id, n).astype(np.int32) for n in rows]
    own = np.concatenate([rng.integers(0, shape.mask_id, n).astype(np.int32) for n in (20, 3, 40)])
    bt = TreeBatch(dl, model, 3, prompt)
    bt.step(own, None, np.array([20, 3, 40]))
    T = sum(rows)
    logits = torch.zeros(T, shape.vocab, device="cuda")
    bt.tree_step(toks, parents, logits)
    logits = logits.cpu().numpy().astype(np.float64)
    # every path as a causal window
    at = 0
    paths = {b: paths_of(parents[b]) for b in range(3)}
    for b, n in enumerate(rows):
        for i in range(n):
            path = paths[b][i]
            ref = TreeBatch(dl, model, 3, prompt)
            ref.step(own, None, np.array([20, 3, 40]))
            out = torch.zeros(len(path), shape.vocab, device="cuda")
            new = np.zeros(3, int)
            new[b] = len(path)
            chain = [np.arange(-1, k - 1) for k in new]
            ref.tree_step([toks[b][path] if k == b else toks[k][:0] for k in range(3)], chain, out)
            d = apart(logits[at + i], out[-1].double().cpu().numpy())
            assert d.max() <= tol(dtype) * 2, (b, i, d.max())          # (two sides, each within tol of the formula)
        at += n
    # keep the deepest path of sequences 0 and 2, and go on
    best = {b: max(paths[b], key=len) for b in (0, 2)}
    path = np.full((3, 16), -1)
    n_acc = np.zeros(3, int)
    for b, p in best.items():
        path[b, :len(p)], n_acc[b] = p, len(p)
    dl.dllm_cache_compact(bt.cache(), PAGE, bt.table, dev_i32(bt.len), dev_i32(path), dev_i32(n_acc))
    bt.len = bt.len + n_acc
    ref = TreeBatch(dl, model, 3, prompt)
    ref.step(own, None, np.array([20, 3, 40]))
    ref.tree_step([toks[b][best[b]] if b in best else toks[b][:0] for b in range(3)], [np.arange(-1, k - 1) for k in n_acc], None, out=False)
    ref.len = ref.len + n_acc
    win = rng.integers(0, shape.mask_id, 24).astype(np.int32)
    mask = (rng.random(24) < 0.5).astype(np.uint8)
    outs = []
    for x in (bt, ref):
        lg = torch.zeros(24, shape.vocab, device="cuda")
        x.step(win, mask, np.array([8, 8, 8]), commit=False, out=True, logits=lg, control=dict(mask_id=shape.mask_id))
        outs.append(lg.double().cpu().numpy())
    assert apart(outs[0], outs[1]).max() <= tol(dtype) * 2


def test_a_forked_sequence_goes_on_as_its_source(dl):
    """Three candidates of sequence 0, one sequence ended: the same steps afterwards give the same logits, while each writes on
    pages of its own."""
    import torch
    shape = synth.TINY_GQA
    model, _, _ = build_pair(shape, "f32", oracle_too=False)
    rng = np.random.default_rng(1)
    bt = TreeBatch(dl, model, 4, synth.prompt_ids(shape, 64))
    own = [rng.integers(0, shape.mask_id, n).astype(np.int32) for n in (45, 7, 3, 20)]
    bt.step(np.concatenate(own), None, np.array([45, 7, 3, 20]))
    z = lambda *n: torch.full(n, -5, dtype=torch.int32, device="cuda")  # noqa: E731
    src, keep = np.array([0, 0, 0, 3]), np.array([64 + 45, 64 + 45, 64 + 45, 0])
    owned, table, n_free, status = z(4), z(4, bt.ld), z(1), z(3)
    before = bt.n_free.item()
    dl.dllm_batch_fork(dev_i32(src), dev_i32(keep), bt.owned, owned, bt.table, table, bt.free, bt.n_free, n_free, 2, bt.cache(), PAGE, status)
    assert status.tolist() == [2, 0, 0]
    # the page of 45 - 32 = 13 positions twice more; the pages of the old 1, 2 and 3 given back
    assert n_free.item() == before + 1 + 1 + 1 - 2
    bt.owned, bt.table, bt.n_free, bt.len = owned, table, n_free, keep.copy()
    assert len({table[b, 3].item() for b in range(3)}) == 3 and len({table[b, 2].item() for b in range(3)}) == 1
    win = [rng.integers(0, shape.mask_id, 5).astype(np.int32) for _ in range(3)]
    logits = torch.zeros(15, shape.vocab, device="cuda")
    bt.step(np.concatenate(win), np.zeros(15, np.uint8), np.array([5, 5, 5, 0]), commit=False, out=True, logits=logits,
            control=dict(mask_id=shape.mask_id))
    for i in range(3):
        ref = TreeBatch(dl, model, 4, synth.prompt_ids(shape, 64))
        ref.step(np.concatenate(own), None, np.array([45, 7, 3, 20]))
        lg = torch.zeros(5, shape.vocab, device="cuda")
        ref.step(win[i], np.zeros(5, np.uint8), np.array([5, 0, 0, 0]), commit=False, out=True, logits=lg, control=dict(mask_id=shape.mask_id))
        assert apart(logits[5 * i:5 * i + 5].double().cpu().numpy(), lg.double().cpu().numpy()).max() <= 2 * tol("f32")


# ---------------------------------------------------------------------------- the operators' run, captured


def run_case(dl, dtype, seed):
    """Buffers of one run over trees, without a model: plan, attention, log probabilities of the next tokens, the accepted
    path's move, a fork."""
    import torch
    rng = np.random.default_rng(seed)
    rows, cached, H, Hk, D, page = [20, 40, 7], [100, 33, 64], 4, 2, 64, 32
    c = attn_case(rng, dtype, rows, cached, H, Hk, D, page, 0)
    T, V = c["T"], 9000
    par = np.zeros(T, int)
    parents = trees(rng, rows)
    par[:sum(rows)] = np.concatenate(parents)
    z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    path = np.zeros((3, 8))
    best = [max(paths_of(p), key=len)[:8] for p in parents]
    for b, p in enumerate(best):
        path[b, :len(p)] = p
    n_pages = c["k"].shape[0]
    pages = torch.stack([c["k"].reshape(n_pages, Hk, -1), c["v"].reshape(n_pages, Hk, -1)])[None].contiguous()
    owned = [-(-int(n) // page) for n in c["lens"]]
    free = np.full(n_pages, -1)
    unused = sorted(set(range(n_pages)) - {int(x) for x in c["table"].ravel()})
    free[:len(unused)] = unused
    f = dict(par=i32(par), row0=i32(c["row0"]), lens=i32(c["lens"]), pos=z(T), mask=z(T, 2), out=torch.zeros_like(c["q"]),
             logits=logits_of(rng, T, V, dtype).cuda(), tok=i32(rng.integers(0, V, 30)), tok_row=i32(rng.integers(0, T, 30)),
             logp=torch.zeros(30, device="cuda"), ent=torch.zeros(T, device="cuda"), top_id=z(T, 5), top_lp=torch.zeros(T, 5, device="cuda"),
             table=i32(c["table"]), base=i32(cached), path=i32(path), n=i32([len(p) for p in best]), pages=pages,
             src=i32([0, 0, 2]), keep=i32([cached[0] + len(best[0])] * 2 + [cached[2] + len(best[2])]), owned=i32(owned), owned_out=z(3),
             table_out=z(*c["table"].shape) - 1, free=i32(free), n_free=i32([len(unused)]), n_free_out=z(1), status=z(3))
    return c, f


def run_all(dl, c, f, ws=None):
    ws = ws or {}
    k, v = f["pages"][0, 0].view(c["k"].shape), f["pages"][0, 1].view(c["v"].shape)
    dl.dllm_tree_plan(f["par"], f["row0"], f["lens"], f["pos"], f["mask"])
    dl.dllm_attention_tree(c["q"], k, v, f["table"], f["row0"], f["lens"], f["mask"], f["out"], 40, 164, ws=ws.get("attn"))
    dl.dllm_logprobs(f["logits"], f["tok"], f["tok_row"], f["logp"], f["ent"], f["top_id"], f["top_lp"], ws=ws.get("logp"))
    dl.dllm_cache_compact(f["pages"], c["page"], f["table"], f["base"], f["path"], f["n"])
    dl.dllm_batch_fork(f["src"], f["keep"], f["owned"], f["owned_out"], f["table"], f["table_out"], f["free"], f["n_free"], f["n_free_out"], 0,
                       f["pages"], c["page"], f["status"], ws=ws.get("fork"))


OUT = ("pos", "mask", "out", "logp", "ent", "top_id", "top_lp", "pages", "owned_out", "table_out", "free", "n_free_out", "status")
IN = ("par", "row0", "lens", "logits", "tok", "tok_row", "table", "base", "path", "n", "src", "keep", "owned", "n_free")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_run_captured_and_replayed_with_other_data(dl, dtype):
    """One graph over the whole run, replayed with the inputs of other seeds copied into its buffers (their number of pages
    differs by none: the same rows and lengths), eager calls between: every replay equals the eager run to the bit."""
    import torch
    c, f = run_case(dl, dtype, 0)
    assert f["status"].tolist() == [0, 0, 0]
    ws = {n: torch.empty(1 << 22, dtype=torch.uint8, device="cuda") for n in ("attn", "logp", "fork")}
    first = {k: f[k].clone() for k in ("pages", "free")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run_all(dl, c, f, ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run_all(dl, c, f, ws)
    for seed in (0, 1, 2, 3, 1):
        c2, f2 = run_case(dl, dtype, seed)
        for k in IN:
            f[k].copy_(f2[k])
        c["q"].copy_(c2["q"])
        f["pages"].copy_(f2["pages"])
        f["free"].copy_(f2["free"])
        for k in OUT:
            if k not in ("pages", "free", "table_out", "pos", "mask"):
                f[k].fill_(7)
        f["out"].zero_()
        f["table_out"].fill_(-1)
        f["pos"].zero_(), f["mask"].zero_()
        g.replay()
        torch.cuda.synchronize()
        run_all(dl, c2, f2)
        torch.cuda.synchronize()
        for k in OUT:
            assert torch.equal(f[k].view(torch.uint8), f2[k].view(torch.uint8)), (seed, k)
        assert f["status"].tolist()[1:] == [0, 0] and f["status"][0].item() == 1
    assert not torch.equal(first["pages"], f["pages"])


def test_two_streams_at_once(dl):
    """The same calls on two streams with workspaces of their own, and the current device's default: the results of each alone."""
    import torch
    cases = [run_case(dl, "bf16", s) for s in (0, 1)]
    want = [run_case(dl, "bf16", s) for s in (0, 1)]
    for c, f in want:
        run_all(dl, c, f)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [{n: torch.empty(1 << 22, dtype=torch.uint8, device="cuda") for n in ("attn", "logp", "fork")} for _ in range(2)]
    torch.cuda.synchronize()
    for s, (c, f), w in zip(streams, cases, ws):
        k, v = f["pages"][0, 0].view(c["k"].shape), f["pages"][0, 1].view(c["v"].shape)
        dl.dllm_tree_plan(f["par"], f["row0"], f["lens"], f["pos"], f["mask"], stream=s)
        dl.dllm_attention_tree(c["q"], k, v, f["table"], f["row0"], f["lens"], f["mask"], f["out"], 40, 164, ws=w["attn"], stream=s)
        dl.dllm_logprobs(f["logits"], f["tok"], f["tok_row"], f["logp"], f["ent"], f["top_id"], f["top_lp"], ws=w["logp"], stream=s)
        dl.dllm_cache_compact(f["pages"], c["page"], f["table"], f["base"], f["path"], f["n"], stream=s)
        dl.dllm_batch_fork(f["src"], f["keep"], f["owned"], f["owned_out"], f["table"], f["table_out"], f["free"], f["n_free"],
                           f["n_free_out"], 0, f["pages"], c["page"], f["status"], ws=w["fork"], stream=s)
    torch.cuda.synchronize()
    for (_, f), (_, w) in zip(cases, want):
        for k in OUT:
            assert torch.equal(f[k].view(torch.uint8), w[k].view(torch.uint8)), k


def test_repeated_calls_give_the_same_bits(dl):
    import torch
    rng = np.random.default_rng(5)
    c = attn_case(rng, "bf16", [64, 33, 50], [3000, 100, 700], 28, 4, 128, 64, 0)
    mask = sets_to_mask(c, random_sets(rng, c["rows"], c["row0"]), 2)
    a = run_tree(dl, c, mask)
    x = logits_of(rng, 40, 60001, "bf16").cuda()
    o = [[torch.zeros(40, device="cuda"), torch.zeros(40, 20, dtype=torch.int32, device="cuda"), torch.zeros(40, 20, device="cuda")] for _ in range(2)]
    for _ in range(5):
        assert torch.equal(run_tree(dl, c, mask), a)
    for ent, ids, lp in o:
        dl.dllm_logprobs(x, entropy=ent, top_id=ids, top_logp=lp)
    assert all(torch.equal(p, q) for p, q in zip(*o))


# ---------------------------------------------------------------------------- refusals of the binding


def test_tensors_that_do_not_fit_are_refused(dl):
    import torch
    c, f = run_case(dl, "f16", 0)
    k, v = f["pages"][0, 0].view(c["k"].shape), f["pages"][0, 1].view(c["v"].shape)
    wide = torch.zeros(f["mask"].shape[0], 4, dtype=torch.int32, device="cuda")[:, :2]
    tree = lambda **kw: dl.dllm_tree_plan(**dict(dict(parent=f["par"], row0=f["row0"], length=f["lens"], pos=f["pos"], mask=f["mask"]), **kw))  # noqa: E731
    attn = lambda **kw: dl.dllm_attention_tree(**dict(dict(q=c["q"], k_pages=k, v_pages=v, table=f["table"], row0=f["row0"], length=f["lens"],  # noqa: E731
                                                           mask=f["mask"], out=f["out"], max_rows=40, max_len=164), **kw))
    logp = lambda **kw: dl.dllm_logprobs(**dict(dict(logits=f["logits"], tok=f["tok"], tok_row=f["tok_row"], logp=f["logp"], entropy=f["ent"],  # noqa: E731
                                                     top_id=f["top_id"], top_logp=f["top_lp"]), **kw))
    comp = lambda **kw: dl.dllm_cache_compact(**dict(dict(pages=f["pages"], page=32, table=f["table"], base=f["base"], path=f["path"], n=f["n"]), **kw))  # noqa: E731
    fork = lambda **kw: dl.dllm_batch_fork(**dict(dict(src=f["src"], keep=f["keep"], owned=f["owned"], owned_out=f["owned_out"], table=f["table"],  # noqa: E731
                                                       table_out=f["table_out"], free=f["free"], n_free=f["n_free"], n_free_out=f["n_free_out"],
                                                       shared_pages=0, pages=f["pages"], page=32, status=f["status"]), **kw))
    cpu = lambda t: t.cpu()  # noqa: E731
    bad = [(tree, dict(parent=f["par"][:5])), (tree, dict(mask=f["mask"][:, 0])), (tree, dict(mask=wide)), (tree, dict(row0=f["row0"][:3])),
           (tree, dict(parent=f["par"].long())), (tree, dict(pos=cpu(f["pos"]))), (tree, dict(mask=torch.zeros(69, 33, dtype=torch.int32, device="cuda"))),
           (attn, dict(mask=f["mask"][:9])), (attn, dict(mask=wide)), (attn, dict(mask=None)), (attn, dict(mask=f["mask"].float())),
           (attn, dict(out=f["out"][:9])), (attn, dict(mask=f["mask"].reshape(-1))), (attn, dict(max_len=2 ** 40)),
           (logp, dict(logp=None)), (logp, dict(tok=None)), (logp, dict(top_id=f["top_id"][:4])), (logp, dict(top_logp=None)), (logp, dict(logp=f["logp"][:3])),
           (logp, dict(entropy=f["ent"][:3])), (logp, dict(logits=f["logits"][0])), (logp, dict(logits=f["logits"].t())), (logp, dict(mask_id=2 ** 33)),
           (logp, dict(tok_row=f["tok_row"][:2])), (logp, dict(logits=f["logits"].double())),
           (logp, dict(top_id=torch.zeros(69, 65, dtype=torch.int32, device="cuda"), top_logp=torch.zeros(69, 65, device="cuda"))),
           (comp, dict(pages=f["pages"][0])), (comp, dict(page=33)), (comp, dict(page=16)), (comp, dict(n=f["n"][:2])), (comp, dict(path=f["path"][:2])),
           (comp, dict(path=f["path"][0])), (comp, dict(pages=f["pages"].double())), (comp, dict(pages=f["pages"][:, :, ::2])), (comp, dict(table=f["table"][:2])),
           (fork, dict(keep=f["keep"][:2])), (fork, dict(free=f["free"][:2])), (fork, dict(table_out=f["table_out"][:, :2])), (fork, dict(table_out=f["table"])),
           (fork, dict(owned_out=f["owned"])), (fork, dict(shared_pages=-1)), (fork, dict(shared_pages=2 ** 35)), (fork, dict(status=f["status"][:2])),
           (fork, dict(ws=torch.empty(16, dtype=torch.uint8, device="cuda"))), (fork, dict(pages=cpu(f["pages"]))), (fork, dict(src=f["src"].short()))]
    before = {n: t.clone() for n, t in f.items()}
    for call, kw in bad:
        try:
            call(**kw)
        except dl.DllmError:
            continue
        pytest.fail(f"not refused: {[n for n, fn in dict(tree=tree, attn=attn, logp=logp, comp=comp, fork=fork).items() if fn is call]} {list(kw)}")
    stream = torch.cuda.Stream()
    for call in (logp, fork):
        with pytest.raises(dl.DllmError):              # a given stream needs a workspace of the caller's
            call(stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(t, before[n]) for n, t in f.items())
    # no rows, no tokens
    tree(mask=f["mask"][:0])
    attn(q=c["q"][:0], out=f["out"][:0], mask=f["mask"][:0])
    dl.dllm_logprobs(f["logits"][:0])
    logp(tok=f["tok"][:0], logp=f["logp"][:0], tok_row=None)
