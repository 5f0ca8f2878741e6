"""A model's step over candidate windows side by side: every row of a candidate sees the text and its own candidate, MASK rows
among them, as if the candidate were the sequence's only window."""
import numpy as np
import pytest

import synth
from branch_util import words
from gpu_util import assert_ids_match_where_decided, assert_logits_close, build_pair, dev_i32, dev_u8, gpu_logits, tol
from test_gpu_batch_step import PAGE, Batch, check, gains, oracle_steps

pytestmark = pytest.mark.gpu


def candidates(rng, shape, counts):
    """counts[b]: rows of each of sequence b's candidates -> their (ids, mask), about 70% of the rows MASK."""
    return [[(rng.integers(0, shape.mask_id, n).astype(np.int32), (rng.random(n) < 0.7).astype(np.uint8)) for n in ns] for ns in counts]


def candidate_step(bt, win, logits):
    """One step over all candidates -> (ids, conf), rows of a sequence's candidates one after another."""
    import torch
    dl, flat = bt.dl, [c for cs in win for c in cs]
    new = np.array([sum(len(t) for t, _ in cs) for cs in win])
    R, ld = int(new.sum()), max(1, -(-int(new.max()) // 32))
    z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    p = dict(row0=z(bt.B + 1), pos=z(R), slot=z(R), seq=z(R), lim=z(R), status=z(3))
    owned, n_free = z(bt.B), z(1)
    dl.dllm_batch_plan(dev_i32(bt.len), dev_i32(new), bt.owned, owned, bt.table, bt.free, bt.n_free, n_free, PAGE, bt.shared // PAGE,
                       p["row0"], p["pos"], p["slot"], p["seq"], p["lim"], p["status"])
    assert p["status"][2].item() == 0
    bt.owned, bt.n_free = owned, n_free
    pos, sets = [], []
    for b, cs in enumerate(win):
        at = 0
        for t, _ in cs:
            pos += [bt.len[b] + i for i in range(len(t))]
            sets += [set(range(at, at + len(t)))] * len(t)
            at += len(t)
    total, ids, conf = bt.len + new, z(R), torch.zeros(R, device="cuda")
    bt.last = (bt.model.handle, bt.pages, bt.n_pages, PAGE, dev_i32(np.concatenate([t for t, _ in flat])),
               dev_u8(np.concatenate([m for _, m in flat])), dev_i32(words(sets, ld)), bt.table, p["row0"], dev_i32(pos), p["slot"],
               dev_i32(total), int(max(new)), int(max(total)), ids, conf), dict(shared_len=bt.shared, lim=p["lim"])
    dl.dllm_batch_step_tree(*bt.last[0], **bt.last[1], logits=logits, control=None if logits is None else dict(mask_id=bt.model.shape.mask_id))
    torch.cuda.synchronize()
    return ids.cpu().numpy(), conf.cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("shape,dtype", [(synth.TINY, "f32"), (synth.TINY_GQA, "f32"), (synth.MICRO, "f32"), (synth.SMALL_BF16, "bf16"),
                                         (synth.SMALL_MQA, "bf16"), (synth.SMALL_BF16, "w8"), (synth.SMALL_MQA, "q4")])
def test_candidates_are_windows_of_their_own(shape, dtype):
    """Three candidates of one sequence, one, none, and two of 32 rows, against the oracle's step over each alone."""
    import paper_2606_13740_amd as dl
    import torch
    rng = np.random.default_rng(3)
    model, om, _ = build_pair(shape, dtype, max_window=128)
    prompt, blocks = synth.prompt_ids(shape, 75), [32, 5, 0, 40]
    own = [rng.integers(0, shape.mask_id, n).astype(np.int32) for n in blocks]
    win = candidates(rng, shape, [[9, 20, 4], [7], [], [32, 32]])
    bt = Batch(dl, model, 4, prompt, n_pages=80)
    bt.step(np.concatenate(own), None, np.array(blocks))
    flat = [c for cs in win for c in cs]
    logits = torch.zeros(sum(len(t) for t, _ in flat), shape.vocab, device="cuda")
    ids, conf = candidate_step(bt, win, logits)
    outs = oracle_steps(om, shape, prompt, [own[b] for b, cs in enumerate(win) for _ in cs], flat, dtype != "f32")
    check(shape, dtype, outs, flat, ids, conf, logits.cpu().numpy())
    model.close()


def test_candidates_captured_and_replayed():
    """A captured step, replayed with other tokens after an eager step that needs larger workspaces: the eager results to the bit."""
    import paper_2606_13740_amd as dl
    import torch
    shape, rng = synth.SMALL_BF16, np.random.default_rng(7)
    model, _, _ = build_pair(shape, "bf16", max_window=256, oracle_too=False)
    bt = Batch(dl, model, 3, synth.prompt_ids(shape, 75), n_pages=100, ld=24)
    small, large = [[[5, 8], [9], [3, 3, 3]], [[32, 32, 32], [20], [32, 32]]]
    scenes, want = [candidates(rng, shape, small) for _ in range(3)], []
    for win in scenes:
        want.append(candidate_step(bt, win, None))
    args, kw = bt.last
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dl.dllm_batch_step_tree(*args, **kw)
    for i in (0, 2, 1):
        candidate_step(bt, candidates(rng, shape, large), None)
        args[4].copy_(dev_i32(np.concatenate([t for cs in scenes[i] for t, _ in cs])))
        args[5].copy_(dev_u8(np.concatenate([m for cs in scenes[i] for _, m in cs])))
        args[-2].fill_(-5), args[-1].fill_(9.0)
        # (the large step has taken pages behind the small one's: its table entries are the same)
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(args[-2].cpu().numpy(), want[i][0]) and np.array_equal(args[-1].cpu().numpy().astype(np.float64), want[i][1])
    model.close()


@pytest.mark.parametrize("shape,dtype,n_prompt,blocks,counts,normed", [
    (synth.LLADA_8B, "bf16", 1056, [0, 40, 5], [[32, 32], [7, 1, 20], []], False),
    (synth.LLADA_8B, "w8", 600, [10, 40], [[9, 20], [32]], True),
    (synth.DREAM_7B, "q4", 1500, [64, 0, 17], [[32, 32, 32, 32], [1], [30, 5]], True)],
    ids=["LLaDA-8B bf16", "LLaDA-8B w8 normed", "Dream-7B q4 normed"])
def test_candidates_at_full_width(shape, dtype, n_prompt, blocks, counts, normed):
    """Two layers at the full widths, against the single-sequence step over each candidate."""
    import paper_2606_13740_amd as dl
    import torch
    shape = shape.with_layers(2)
    layers, glob = [synth.layer_weights(shape, l, "bf16") for l in range(2)], synth.global_weights(shape, "bf16")
    model = dl.Model(shape, dtype, glob, lambda l: layers[l], max_window=192, max_pos=n_prompt + 200)
    print(f"case: {dtype}, {counts} behind {n_prompt}", flush=True)
    if normed:
        dl.dllm_model_set_qk_norm(model.handle, *gains(shape)[1])
    rng = np.random.default_rng(5)
    prompt, own = synth.prompt_ids(shape, n_prompt), [rng.integers(0, shape.mask_id, n).astype(np.int32) for n in blocks]
    win = candidates(rng, shape, counts)
    bt = Batch(dl, model, len(blocks), prompt, ld=n_prompt // 32 + 8, n_pages=n_prompt // 32 + 9 * len(blocks))
    bt.step(np.concatenate(own), None, np.array(blocks))
    logits = torch.zeros(sum(len(t) for cs in win for t, _ in cs), shape.vocab, device="cuda")
    ids, conf = candidate_step(bt, win, logits)
    at = 0
    for o, cs in zip(own, win):
        kv = dl.KVCache(model, n_prompt + 160)
        dl.dllm_prefill(model.handle, kv.handle, dev_i32(prompt), n_prompt)
        if len(o):
            dl.dllm_append_prefix_kv(model.handle, kv.handle, dev_i32(o), len(o))
        for tok, mask in cs:
            want, wid, wconf = gpu_logits(model, kv, tok, mask)
            err = assert_logits_close(logits[at:at + len(tok)].double().cpu().numpy(), want, tol(dtype))
            got = ids[at:at + len(tok)]
            assert_ids_match_where_decided(got, want, err)
            same = got == wid
            # a logit off by e moves a softmax probability by at most a factor exp(2 e)
            assert (abs(conf[at:at + len(tok)] - wconf)[same] <= wconf[same] * (np.exp(2 * err) - 1) + 1e-6).all()
            at += len(tok)
    model.close()
