"""dllm_batch_step and the heads' norm against the oracle: several sequences behind one prompt, over a paged cache."""
import contextlib
import dataclasses

import numpy as np
import pytest

import oracle
import oracle.model
import synth
from batch_util import select
from gpu_util import (assert_ids_match_where_decided, assert_logits_close, build_pair, dev_i32, dev_u8, gpu_logits, tol)

pytestmark = pytest.mark.gpu

PAGE = 32


@pytest.fixture(scope="module")
def dl():
    import paper_2606_13740_amd as pkg
    return pkg


class Batch:
    """A serving program's side of a batch: tables, lengths and free pages through dllm_batch_plan."""

    def __init__(self, dl, model, n_seqs, prompt, max_rows=256, ld=16, n_pages=60):
        import torch
        self.dl, self.model, self.B, self.ld, self.n_pages, self.R = dl, model, n_seqs, ld, n_pages, max_rows
        self.pages = torch.full((dl.dllm_batch_bytes(model.handle, n_pages, PAGE),), 0x7F, dtype=torch.uint8, device="cuda")
        self.table = torch.full((n_seqs, ld), -1, dtype=torch.int32, device="cuda")
        self.free, self.n_free = dev_i32(np.random.default_rng(1).permutation(n_pages)), dev_i32([n_pages])
        self.len, self.owned = np.zeros(n_seqs, int), dev_i32(np.zeros(n_seqs))
        self.shared = len(prompt) // PAGE * PAGE
        # the prompt through sequence 0, then its whole pages into every table
        new = np.zeros(n_seqs, int)
        new[0] = len(prompt)
        self.step(prompt, None, new)
        sp = self.shared // PAGE
        self.table[1:, :sp] = self.table[0, :sp]
        self.owned[1:] = sp
        self.len[:] = self.shared
        if len(prompt) > self.shared:        # the rest of the prompt in pages of each sequence's own
            rest = np.tile(prompt[self.shared:], n_seqs)
            self.step(rest, None, np.full(n_seqs, len(prompt) - self.shared))

    def step(self, tok, mask, new, commit=True, out=False, pad=0, **kw):
        """One planned step; commit: the rows become part of the sequences.  Rows of all sequences one after another."""
        import torch
        dl, R = self.dl, len(tok) + pad
        z = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
        p = dict(row0=z(self.B + 1), pos=z(R), slot=z(R), seq=z(R), lim=z(R), status=z(3))
        owned, n_free = z(self.B), z(1)
        dl.dllm_batch_plan(dev_i32(self.len), dev_i32(new), self.owned, owned, self.table, self.free, self.n_free, n_free,
                           PAGE, self.shared // PAGE if self.len[0] else 0, p["row0"], p["pos"], p["slot"], p["seq"],
                           p["lim"], p["status"])
        assert p["status"][2].item() == 0, p["status"]
        self.owned, self.n_free = owned, n_free
        total = self.len + new
        ids, conf = (z(R), torch.zeros(R, device="cuda")) if out else (None, None)
        t = torch.cat([dev_i32(tok), z(pad)])
        m = None if mask is None else torch.cat([dev_u8(mask), torch.zeros(pad, dtype=torch.uint8, device="cuda")])
        args = (self.model.handle, self.pages, self.n_pages, PAGE, t, m, self.table, p["row0"], p["pos"], p["slot"],
                dev_i32(total), int(max(new)), int(max(total)), ids, conf)
        kw = dict(shared_len=self.shared if self.len[0] else 0, lim=p["lim"], **kw)
        dl.dllm_batch_step(*args, **kw)
        torch.cuda.synchronize()
        self.last = (args, kw)
        if commit:
            self.len = total
        return (ids.cpu().numpy(), conf.cpu().numpy().astype(np.float64)) if out else None


def scene(shape, n_prompt, blocks, windows, seed=0):
    """A prompt, each sequence's own committed ids, and its window (ids, mask)."""
    rng = np.random.default_rng(seed)
    prompt = synth.prompt_ids(shape, n_prompt)
    own = [rng.integers(0, shape.mask_id, n).astype(np.int32) for n in blocks]
    win = [(rng.integers(0, shape.mask_id, n).astype(np.int32), (rng.random(n) < 0.7).astype(np.uint8)) for n in windows]
    return prompt, own, win


def oracle_steps(om, shape, prompt, own, win, fp16):
    """The oracle's step of each sequence over a cache of its own."""
    base = oracle.OracleKV(shape, 400, fp16=fp16)
    oracle.prefill(om, base, prompt)
    outs = []
    for o, (tok, mask) in zip(own, win):
        kv = base.copy()
        if len(o):
            oracle.append_block(om, kv, o)
        outs.append(oracle.denoise_step(om, kv, tok, mask) if len(tok) else None)
    return outs


def check(shape, dtype, outs, win, ids, conf, logits):
    at, worst = 0, 0.0
    for (tok, _), ref in zip(win, outs):
        n = len(tok)
        if not n:
            continue
        got = logits[at:at + n].astype(np.float64)
        err = assert_logits_close(got, ref.logits, tol(dtype))
        worst = max(worst, err)
        assert_ids_match_where_decided(ids[at:at + n], ref.logits, err)
        same = ids[at:at + n] == ref.ids
        # a logit off by e moves a softmax probability by at most a factor exp(2 e)
        assert (abs(conf[at:at + n] - ref.conf)[same] <= ref.conf[same] * (np.exp(2 * err) - 1) + 1e-6).all()
        at += n
    return worst


@pytest.mark.parametrize("shape,dtype", [(synth.TINY, "f32"), (synth.TINY_GQA, "f32"), (synth.MICRO, "f32"), (synth.SMALL_BF16, "bf16"),
                                         (synth.SMALL_MQA, "bf16"), (synth.SMALL_BF16, "w8"), (synth.SMALL_MQA, "q4")])
@pytest.mark.parametrize("n_prompt", [64, 75])
def test_batch_step_is_the_step_of_every_sequence(dl, shape, dtype, n_prompt):
    import torch
    model, om, _ = build_pair(shape, dtype)
    prompt, own, win = scene(shape, n_prompt, [32, 5, 0, 64], [32, 7, 20, 0])
    bt = Batch(dl, model, 4, prompt)
    bt.step(np.concatenate(own), None, np.array([len(o) for o in own]))
    T, pad = sum(len(t) for t, _ in win), 3
    logits = torch.zeros(T + pad, shape.vocab, device="cuda")
    ids, conf = bt.step(np.concatenate([t for t, _ in win]), np.concatenate([m for _, m in win]), np.array([len(t) for t, _ in win]),
                        commit=False, out=True, pad=pad, logits=logits, control=dict(mask_id=shape.mask_id))
    outs = oracle_steps(om, shape, prompt, own, win, dtype != "f32")
    check(shape, dtype, outs, win, ids, conf, logits.cpu().numpy())
    # without the control the LM head's own reduction gives the same ids
    ids2, conf2 = bt.step(np.concatenate([t for t, _ in win]), np.concatenate([m for _, m in win]),
                          np.array([len(t) for t, _ in win]), commit=False, out=True, pad=pad)
    assert np.array_equal(ids[:T], ids2[:T]) and np.allclose(conf[:T], conf2[:T], rtol=1e-4)


def test_batch_step_many_rows_and_a_second_block(dl):
    """More than 64 rows (tiled GEMMs, K slices), windows committed and stepped on from."""
    import torch
    shape, dtype = synth.SMALL_BF16, "bf16"
    model, om, _ = build_pair(shape, dtype, max_window=256)
    prompt, own, win = scene(shape, 96, [64, 33, 40, 31, 0, 90], [32, 32, 32, 32, 32, 32], seed=3)
    bt = Batch(dl, model, 6, prompt)
    bt.step(np.concatenate(own), None, np.array([len(o) for o in own]))
    logits = torch.zeros(192, shape.vocab, device="cuda")
    toks, masks = np.concatenate([t for t, _ in win]), np.concatenate([m for _, m in win])
    ids, conf = bt.step(toks, masks, np.full(6, 32), commit=False, out=True, logits=logits, control=dict(mask_id=shape.mask_id))
    check(shape, dtype, oracle_steps(om, shape, prompt, own, win, True), win, ids, conf, logits.cpu().numpy())


def test_batch_step_controlled_outputs(dl):
    """Penalties, biases and masks on a step's logits: dllm_select's definition on the logits that the step leaves."""
    import torch
    shape = synth.TINY
    model, _, _ = build_pair(shape, "f32", oracle_too=False)
    prompt, own, win = scene(shape, 64, [10, 20], [9, 5], seed=5)
    bt = Batch(dl, model, 2, prompt)
    bt.step(np.concatenate(own), None, np.array([10, 20]))
    rng, V = np.random.default_rng(7), shape.vocab
    hist = [np.concatenate([prompt, o]) for o in own]
    hist0, n_prompt = np.array([0, len(hist[0]), len(hist[0]) + len(hist[1])]), np.array([64, 64])
    rep, pres, freq = (np.array(x, np.float32) for x in ([1.3, 1.1], [0.5, 0.2], [0.1, 0.3]))
    allow = rng.integers(-2 ** 31, 2 ** 31, (2, V // 32)).astype(np.int32)
    allow_row = np.array([0, 1, -1] * 4 + [0, 1])
    row0 = np.array([0, 9, 14])
    raw = torch.zeros(14, V, device="cuda")
    f = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    control = dict(mask_id=shape.mask_id, row0=dev_i32(row0), hist=dev_i32(np.concatenate(hist)), hist0=dev_i32(hist0),
                   n_prompt=dev_i32(n_prompt), repetition=f(rep), presence=f(pres), frequency=f(freq), allow=f(allow),
                   allow_row=dev_i32(allow_row))
    toks, masks = np.concatenate([t for t, _ in win]), np.concatenate([m for _, m in win])
    ids, conf = bt.step(toks, masks, np.array([9, 5]), commit=False, out=True, logits=raw, control=control)
    _, rid, rconf = select(raw.cpu().numpy(), V, shape.mask_id, row0, np.concatenate(hist), hist0, n_prompt, rep, pres, freq,
                           None, None, None, allow, allow_row)
    assert np.array_equal(ids, rid)
    assert np.allclose(conf, rconf, rtol=(V / 16 + 256) * 2.0 ** -24, atol=0)


def test_batch_step_captured(dl):
    import torch
    shape = synth.SMALL_BF16
    model, _, _ = build_pair(shape, "bf16", oracle_too=False)
    prompt, own, win = scene(shape, 64, [40, 8], [32, 32], seed=6)
    bt = Batch(dl, model, 2, prompt)
    bt.step(np.concatenate(own), None, np.array([40, 8]))
    toks, masks = np.concatenate([t for t, _ in win]), np.concatenate([m for _, m in win])
    ids, conf = bt.step(toks, masks, np.array([32, 32]), commit=False, out=True)
    args, kw = bt.last
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dl.dllm_batch_step(*args, **kw)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dl.dllm_batch_step(*args, **kw)
    for i in range(4):
        args[-2].fill_(-5)
        args[-1].fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(args[-2].cpu().numpy(), ids) and np.array_equal(args[-1].cpu().numpy().astype(np.float64), conf)
        dl.dllm_batch_step(*args, **kw)      # eager work between the replays
        torch.cuda.synchronize()


def test_captured_calls_keep_their_workspaces(dl):
    """Graphs of a single-sequence step and of a batch step, replayed after calls that needed larger workspaces: the first
    batch step at all, then a prompt of many rows, then the heads' norm's rows."""
    import torch
    shape = synth.SMALL_BF16
    model, _, _ = build_pair(shape, "bf16", oracle_too=False)
    kv = dl.KVCache(model, 128)
    dl.dllm_prefill(model.handle, kv.handle, dev_i32(synth.prompt_ids(shape, 40)), 40)
    tok, mask = synth.window(shape, 32, range(8, 32))
    step = (model.handle, kv.handle, dev_i32(tok), dev_u8(mask), 32, torch.zeros(32, dtype=torch.int32, device="cuda"),
            torch.zeros(32, device="cuda"))
    graphs = []

    def record(call, args, kw):
        call(*args, **kw)
        torch.cuda.synchronize()
        outs = [x for x in args if isinstance(x, torch.Tensor)][-2:]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(*args, **kw)
        graphs.append((g, outs, [o.clone() for o in outs]))

    def replay_all():
        junk = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(64)]       # into what has been freed, if anything
        for _ in range(3):
            for g, outs, want in graphs:
                for o in outs:
                    o.fill_(7)
                g.replay()
                torch.cuda.synchronize()
                assert all(torch.equal(o, w) for o, w in zip(outs, want))
        del junk

    record(dl.dllm_denoise_step, step, {})
    prompt, own, win = scene(shape, 64, [40, 8], [32, 32], seed=9)
    bt = Batch(dl, model, 2, prompt, n_pages=60)
    replay_all()
    bt.step(np.concatenate(own), None, np.array([40, 8]))
    bt.step(np.concatenate([t for t, _ in win]), np.concatenate([m for _, m in win]), np.array([32, 32]), commit=False, out=True)
    record(dl.dllm_batch_step, *bt.last)
    replay_all()
    many = np.random.default_rng(10).integers(0, shape.mask_id, 700).astype(np.int32)
    other = Batch(dl, model, 2, many[:288], n_pages=80)
    other.step(many[:348], None, np.array([148, 200]), commit=False)
    replay_all()


# ---------------------------------------------------------------------------- the heads' norm


@contextlib.contextmanager
def normed_oracle(shape, gq, gk):
    """The oracle's rotation with the heads' norm before it: called for q, then for k, layer by layer."""
    plain, calls = oracle.model.rope, [0]

    def rope(u, pos, base):
        l, is_k = calls[0] // 2 % shape.n_layers, calls[0] % 2
        calls[0] += 1
        u = u / np.sqrt((u * u).mean(-1, keepdims=True) + shape.eps) * (gk if is_k else gq)[l].astype(np.float64)
        return plain(u, pos, base)

    oracle.model.rope = rope
    try:
        yield
    finally:
        oracle.model.rope = plain


def gains(shape, seed=11):
    import torch
    rng = np.random.default_rng(seed)
    g = [rng.normal(1.0, 0.2, (shape.n_layers, shape.head_dim)).astype(np.float32) for _ in range(2)]
    return g, [[torch.from_numpy(r).cuda() for r in x] for x in g]


@pytest.mark.parametrize("shape,dtype", [(synth.TINY, "f32"), (synth.TINY_GQA, "f32"), (synth.SMALL_BF16, "bf16"), (synth.SMALL_MQA, "q4")])
def test_heads_norm_single_sequence(dl, shape, dtype):
    """Prompt, step, append, refresh and the no-allocation step of a model with the heads' norm."""
    import torch
    model, om, _ = build_pair(shape, dtype)
    (gq, gk), (tq, tk) = gains(shape)
    dl.dllm_model_set_qk_norm(model.handle, tq, tk)
    kv = dl.KVCache(model, 256)
    okv = oracle.OracleKV(shape, 256, fp16=dtype != "f32")
    prompt = synth.prompt_ids(shape, 75)
    dl.dllm_prefill(model.handle, kv.handle, dev_i32(prompt), 75)
    tok, mask = synth.window(shape, 32, range(8, 32))
    block = np.arange(32, dtype=np.int32) % (shape.mask_id - 1)
    with normed_oracle(shape, gq, gk):
        oracle.prefill(om, okv, prompt)
        ref = oracle.denoise_step(om, okv, tok, mask)
        got, ids, conf = gpu_logits(model, kv, tok, mask)
        assert_ids_match_where_decided(ids, ref.logits, assert_logits_close(got, ref.logits, tol(dtype)))
        rid, rconf = torch.zeros(32, dtype=torch.int32, device="cuda"), torch.zeros(32, device="cuda")
        dl.dllm_denoise_step_noalloc(model.handle, kv.handle, dev_i32(tok), dev_u8(mask), 32, rid, rconf)
        assert np.array_equal(rid.cpu().numpy(), ids)
        dl.dllm_append_prefix_kv(model.handle, kv.handle, dev_i32(block), 32)
        oracle.append_block(om, okv, block)
        dl.dllm_refresh_kv(model.handle, kv.handle, dev_i32([3, 80, 101]), dev_i32([5, 6, 7]), 3)
        oracle.refresh(om, okv, [3, 80, 101], [5, 6, 7])
        ref = oracle.denoise_step(om, okv, tok, mask)
        got, ids, conf = gpu_logits(model, kv, tok, mask)
        assert_ids_match_where_decided(ids, ref.logits, assert_logits_close(got, ref.logits, tol(dtype)))


def test_heads_norm_batch_and_a_long_prompt(dl):
    """The heads' norm in batch steps; a prompt of tiled GEMMs with K slices through both paths."""
    import torch
    shape, dtype = dataclasses.replace(synth.SMALL_MQA, n_layers=2), "bf16"
    model, om, _ = build_pair(shape, dtype)
    (gq, gk), (tq, tk) = gains(shape, 12)
    dl.dllm_model_set_qk_norm(model.handle, tq, tk)
    prompt, own, win = scene(shape, 224, [32, 9], [32, 11], seed=8)
    bt = Batch(dl, model, 2, prompt)
    bt.step(np.concatenate(own), None, np.array([32, 9]))
    logits = torch.zeros(43, shape.vocab, device="cuda")
    ids, conf = bt.step(np.concatenate([t for t, _ in win]), np.concatenate([m for _, m in win]), np.array([32, 11]),
                        commit=False, out=True, logits=logits, control=dict(mask_id=shape.mask_id))
    with normed_oracle(shape, gq, gk):
        outs = oracle_steps(om, shape, prompt, own, win, True)
        check(shape, dtype, outs, win, ids, conf, logits.cpu().numpy())
        kv = dl.KVCache(model, 320)
        dl.dllm_prefill(model.handle, kv.handle, dev_i32(prompt), 224)
        okv = oracle.OracleKV(shape, 320, fp16=True)
        oracle.prefill(om, okv, prompt)
        got, _, _ = gpu_logits(model, kv, *win[0])
        assert_logits_close(got, oracle.denoise_step(om, okv, *win[0]).logits, tol(dtype))
