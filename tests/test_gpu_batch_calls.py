"""Batch calls that are refused, and what they leave behind."""
import dataclasses

import numpy as np
import pytest

import synth
from gpu_util import GLOBALS, build_pair, dev_i32, dev_u8, gpu_logits
from test_gpu_batch_step import Batch, gains, scene

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dl():
    import paper_2606_13740_amd as pkg
    return pkg


def wide_batch(dl, V=5000):
    """A batch of two sequences of a small model whose logits take a selection with a workspace, and a step's rows."""
    shape = dataclasses.replace(synth.TINY, vocab=V, mask_id=V - 1)
    model, _, _ = build_pair(shape, "f32", oracle_too=False)
    prompt, own, win = scene(shape, 64, [10, 20], [9, 5], seed=5)
    bt = Batch(dl, model, 2, prompt)
    bt.step(np.concatenate(own), None, np.array([10, 20]))
    return shape, model, bt, np.concatenate([t for t, _ in win]), np.concatenate([m for _, m in win])


def test_a_step_with_a_refused_selection_does_nothing(dl):
    """Every refusal of the selection comes before the step's first launch: no K/V, no outputs, no logits."""
    import torch
    shape, model, bt, tok, mask = wide_batch(dl)
    logits = torch.full((14, shape.vocab), 3.0, device="cuda")
    bt.step(tok, mask, np.array([9, 5]), commit=False, out=True, logits=logits, control=dict(mask_id=shape.mask_id))
    args, kw = bt.last
    args[-2].fill_(-5), args[-1].fill_(9.0), logits.fill_(3.0)
    bt.pages.fill_(0x11)
    before = bt.pages.clone()
    ws = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    for bad in (dict(ws=ws[8:]), dict(ws=ws[:64]), dict(mask_id=5), dict(allow=dev_i32([[0] * 200])), dict(allow=dev_i32([[0] * 9] * 20))):
        with pytest.raises(dl.DllmError):
            dl.dllm_batch_step(*args, **dict(kw, control=dict(dict(mask_id=shape.mask_id), **bad)))
        torch.cuda.synchronize()
        assert args[-2].eq(-5).all() and args[-1].eq(9.0).all() and logits.eq(3.0).all() and torch.equal(bt.pages, before), bad


def test_a_batch_step_takes_nothing_from_the_static_scratch(dl):
    """A 256-row step that just fits the no-allocation step's 64 MiB (249 KB a row) fits them after a batch step too, whose
    Q/K/V rows (24 KB a row) are in the model's own workspace."""
    import torch
    shape = dataclasses.replace(synth.SMALL_BF16, n_layers=1, d_model=2048, n_heads=16, d_ff=4096)
    model, _, _ = build_pair(shape, "bf16", max_window=256, oracle_too=False)
    kv = dl.KVCache(model, 512)
    dl.dllm_prefill(model.handle, kv.handle, dev_i32(synth.prompt_ids(shape, 64)), 64)
    tok, mask = (f(a) for f, a in zip((dev_i32, dev_u8), synth.window(shape, 256, range(8, 256))))
    outs = []
    for i in range(2):
        ids, conf = torch.zeros(256, dtype=torch.int32, device="cuda"), torch.zeros(256, device="cuda")
        dl.dllm_denoise_step_noalloc(model.handle, kv.handle, tok, mask, 256, ids, conf)
        outs += [ids, conf]
        if i == 0:
            Batch(dl, model, 2, synth.prompt_ids(shape, 64))
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3]) and outs[1].gt(0).all()


def test_a_step_too_large_for_the_card_leaves_the_model_usable(dl):
    """A workspace of more bytes than the card has (4 Mi rows of about 80 KB) is refused, and the next calls are what they
    were before."""
    import torch
    shape = dataclasses.replace(synth.SMALL_BF16, n_layers=1, d_model=2048, n_heads=16, d_ff=4096)
    model, _, _ = build_pair(shape, "bf16", oracle_too=False)
    bt = Batch(dl, model, 2, synth.prompt_ids(shape, 64))
    tok = np.arange(40, dtype=np.int32)
    want = bt.step(tok, None, np.array([30, 10]), commit=False, out=True)
    n = 1 << 22
    z = torch.zeros(n, dtype=torch.int32, device="cuda")
    row0, length = dev_i32([0, n, n]), dev_i32([0, 0])
    for _ in range(2):
        with pytest.raises(dl.DllmError) as e:
            dl.dllm_batch_step(model.handle, bt.pages, bt.n_pages, 32, z, None, bt.table, row0, z, z, length, 1, 1)
        assert e.value.code == dl.DLLM_E_NOMEM
        kv = dl.KVCache(model, 128)
        dl.dllm_prefill(model.handle, kv.handle, dev_i32(synth.prompt_ids(shape, 40)), 40)
        got = bt.step(tok, None, np.array([30, 10]), commit=False, out=True)
        assert all(np.array_equal(a, b) for a, b in zip(got, want))


def test_workspaces_kept_for_graphs_stay_few(dl):
    """Prompts that get longer 64 rows at a time after a capture: what is kept for the graph and the workspace in use take less
    than four times the workspace that the longest prompt needs, and the graph gives the same ids."""
    import torch
    shape = dataclasses.replace(synth.SMALL_BF16, n_layers=1, d_model=1024, n_heads=8, d_ff=2048)
    top, taken = 1536, []

    def used():
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        free, total = torch.cuda.mem_get_info()
        return total - free

    ids = dev_i32(synth.prompt_ids(shape, top))
    for lengths in ([top], range(64, top + 64, 64)):
        model, _, _ = build_pair(shape, "bf16", max_pos=2048, oracle_too=False)
        bt = Batch(dl, model, 2, synth.prompt_ids(shape, 64), n_pages=140)
        want = bt.step(np.arange(40, dtype=np.int32), None, np.array([30, 10]), commit=False, out=True)
        args, kw = bt.last
        g = torch.cuda.CUDAGraph()
        if len(lengths) > 1:
            with torch.cuda.graph(g):
                dl.dllm_batch_step(*args, **kw)
        before = used()
        for n in lengths:
            kv = dl.KVCache(model, top)
            dl.dllm_prefill(model.handle, kv.handle, ids[:n], n)
            del kv
        taken.append(used() - before)
        if len(lengths) > 1:
            for _ in range(3):
                args[-2].fill_(-5)
                g.replay()
                torch.cuda.synchronize()
                assert np.array_equal(args[-2].cpu().numpy(), want[0])
    print(f"  longest prompt alone {taken[0] >> 20} MiB, grown to it {taken[1] >> 20} MiB", flush=True)
    assert 0 < taken[0] and taken[1] < 4 * taken[0]


def test_allocations_on_a_stream_of_its_own(dl):
    """Model, heads' gains, first prompt and first batch step (each allocates zeroed memory) on a stream that does not wait for
    the default one: the results of the default stream."""
    import torch
    shape = dataclasses.replace(synth.SMALL_BF16, n_layers=1, d_model=1024, n_heads=8, d_ff=2048)
    tok = np.arange(40, dtype=np.int32)

    def life():
        model, _, _ = build_pair(shape, "bf16", oracle_too=False)
        dl.dllm_model_set_qk_norm(model.handle, *gains(shape)[1])
        kv = dl.KVCache(model, 512)
        dl.dllm_prefill(model.handle, kv.handle, dev_i32(synth.prompt_ids(shape, 300)), 300)
        ids, conf = torch.zeros(32, dtype=torch.int32, device="cuda"), torch.zeros(32, device="cuda")
        dl.dllm_denoise_step(model.handle, kv.handle, dev_i32(tok[:32]), None, 32, ids, conf)
        bt = Batch(dl, model, 2, synth.prompt_ids(shape, 400))
        out = bt.step(tok, None, np.array([30, 10]), commit=False, out=True)
        return [ids.cpu().numpy(), conf.cpu().numpy(), *out]

    want = life()
    assert (want[1] > 0).all()
    for _ in range(3):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = life()
        side.synchronize()
        assert all(np.array_equal(a, b) for a, b in zip(got, want))


def test_a_control_that_could_not_act_is_refused(dl):
    """Logits without ids to write, and a control without logits (it was dropped without a word)."""
    import torch
    shape, model, bt, tok, mask = wide_batch(dl)
    bt.step(tok, mask, np.array([9, 5]), commit=False, out=True)
    args, kw = bt.last
    logits, control = torch.zeros(14, shape.vocab, device="cuda"), dict(mask_id=shape.mask_id)
    for a, more in ((args[:-2], dict(logits=logits, control=control)), (args[:-2], dict(logits=logits)), (args, dict(control=control)),
                    (args[:-1], dict(logits=logits, control=control)), (args[:-2], dict(control=control))):
        with pytest.raises(dl.DllmError):
            dl.dllm_batch_step(*a, **dict(kw, **more))


def test_tensors_of_other_ranks_and_lists_without_their_parts_are_refused(dl):
    """A refusal that says so, not an error of the unpacking, and no list that is silently dropped."""
    import torch
    z = lambda *s, dt=torch.float16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    i = lambda *s: z(*s, dt=torch.int32)  # noqa: E731
    q, k, v, kp, vp = z(2, 4, 64), z(2, 2, 64), z(2, 2, 64), z(3, 2, 32, 64), z(3, 2, 64, 32)
    rope = z(8, 32, 2, dt=torch.float32)
    for a in ((q, k, v, rope, i(2), i(2), q.clone(), kp[0], vp), (q[0, 0, 0], k, v, rope, i(2), i(2), q.clone(), kp, vp),
              (q, k, v, rope, i(2), i(2), z(64), kp, vp), (q, k, v, rope, i(2), i(2), q.view(2, 256).clone(), kp[..., :0], vp)):
        with pytest.raises(dl.DllmError):
            dl.dllm_qk_norm_rope(*a)
    for a in ((q, kp[0], vp, i(1, 2), i(2), i(1), q.clone()), (z(64), kp, vp, i(1, 2), i(2), i(1), q.clone()),
              (q, kp, vp, i(1, 2)[0, 0], i(2), i(1), q.clone()), (q.view(2, 256), kp[..., :0], vp, i(1, 2), i(2), i(1), q.clone())):
        with pytest.raises(dl.DllmError):
            dl.dllm_attention_paged(*a, 2, 32)
    x, ids, conf = z(2, 50, dt=torch.float32), i(2), z(2, dt=torch.float32)
    w = z(3, dt=torch.float32)
    for control in (dict(hist=i(3)), dict(bias=w), dict(bias_id=i(3)), dict(bias0=i(2)), dict(bias=w, bias_id=i(3)),
                    dict(bias_id=i(3), bias0=i(2)), dict(allow=i(2))):
        with pytest.raises(dl.DllmError):
            dl.dllm_select(x, ids, conf, **control)
    for bad in (x[0], x[0, 0], x[None]):
        with pytest.raises(dl.DllmError):
            dl.dllm_select(bad, ids, conf)


def test_numbers_past_32_bits_are_refused(dl):
    """Not cut to their low 32 bits, in the calls that do not go through the packed structs either."""
    import torch
    shape, model, bt, tok, mask = wide_batch(dl)
    for n_pages, page in ((2 ** 32 + 1, 32), (4, 2 ** 32 + 32), (-2 ** 32 + 4, 32), (4.5, 32), ("4", 32)):
        with pytest.raises(dl.DllmError):
            dl.dllm_batch_bytes(model.handle, n_pages, page)
    bt.step(tok, mask, np.array([9, 5]), commit=False, out=True)
    args, kw = bt.last
    for at, bad in ((2, 2 ** 32 + bt.n_pages), (3, 2 ** 32 + 32), (11, 2 ** 32 + 9), (12, 2 ** 32 + 100)):
        with pytest.raises(dl.DllmError):
            dl.dllm_batch_step(*args[:at], bad, *args[at + 1:], **kw)
    with pytest.raises(dl.DllmError):
        dl.dllm_batch_step(*args, **dict(kw, shared_len=2 ** 32))
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    for page, shared in ((2 ** 32 + 32, 0), (32, 2 ** 32), (32, -2 ** 32)):
        with pytest.raises(dl.DllmError):
            dl.dllm_batch_plan(i(2), i(2), i(2), i(2), i(2, 4), i(8), i(1), i(1), page, shared, i(3), i(5), i(5), i(5), i(5), i(3))
    for head_dim in (0, -64, 2 ** 32 + 64):
        with pytest.raises(dl.DllmError):
            dl.dllm_rope_table(torch.zeros(4, 32, 2, device="cuda"), head_dim, 10000.0)


def test_gains_of_another_number_or_size_are_refused(dl):
    """The library reads a pointer a layer and head_dim floats behind each: fewer of either must not reach it."""
    import torch
    model, _, _ = build_pair(synth.TINY, "f32", oracle_too=False)
    n, d = synth.TINY.n_layers, synth.TINY.head_dim
    one = lambda size: torch.ones(size, device="cuda")  # noqa: E731
    good = [one(d)] * n
    for q, k in ((good[1:], good), (good, good[1:]), (good[1:], good[1:]), ([], []), (good + good, good + good),
                 (good, [one(d - 1)] * n), ([one(d)] * (n - 1) + [one(1)], good), (good, [one(2 * d)] * n)):
        with pytest.raises(dl.DllmError):
            dl.dllm_model_set_qk_norm(model.handle, q, k)
    dl.dllm_model_set_qk_norm(model.handle, good, good)


def test_attention_rows_reach_the_projection_unrounded(dl):
    """With W_k = 0 every key weighs the same: Q's and the probabilities' roundings do nothing, and a batch step differs from the
    single sequence's only in how the attention's rows reach the O projection.  W_o times 16, so that the logits follow
    them: rows rounded to fp16 would be off by 2^-11 / sqrt(12) RMS, about 2^-13 of the largest logit; as pairs of
    bf16 of the fp32 sums (half a step 2^-17, in both calls, beside sums of 96 values in two orders) by 2^-17."""
    import torch
    shape = dataclasses.replace(synth.SMALL_BF16, n_layers=1)
    w = synth.all_weights(shape, "bf16", 0)
    layer = dict(w["layers"][0])
    layer["wk"] = np.zeros_like(layer["wk"])
    layer["wo"] = layer["wo"] + np.uint16(4 << 7)                       # bf16: four steps of the exponent
    model = dl.Model(shape, "bf16", {k: w[k] for k in GLOBALS}, lambda l: layer, max_window=64, max_pos=256)
    prompt = synth.prompt_ids(shape, 64)
    tok, mask = synth.window(shape, 32, range(8, 32))
    kv = dl.KVCache(model, 128)
    dl.dllm_prefill(model.handle, kv.handle, dev_i32(prompt), 64)
    want, _, _ = gpu_logits(model, kv, tok, mask)
    bt = Batch(dl, model, 1, prompt)
    logits = torch.zeros(32, shape.vocab, device="cuda")
    bt.step(tok, mask, np.array([32]), commit=False, out=True, logits=logits, control=dict(mask_id=shape.mask_id))
    got, fin = logits.double().cpu().numpy(), np.isfinite(want)
    off, top = abs(got[fin] - want[fin]).max(), abs(want[fin]).max()
    print(f"  off by 2^{np.log2(off / top + 1e-30):.1f} of the largest logit", flush=True)
    assert off <= 2.0 ** -15 * top


@pytest.mark.parametrize("shape,dtype,rtol", [(synth.TINY_GQA, "f32", 1e-3), (synth.SMALL_BF16, "bf16", 0.1)])
def test_heads_norm_in_the_merged_and_the_windowed_step(dl, shape, dtype, rtol):
    """Refresh, append and step in one pass, and a window behind kept positions with selective outputs: what the calls one by one
    give for a model with the heads' norm (confidences as closely as the merged step's own test asks)."""
    import torch
    model, _, _ = build_pair(shape, dtype, oracle_too=False)
    rng, W, P = np.random.default_rng(3), 20, 40
    block, pos, new = (dev_i32(a) for a in (rng.integers(0, 900, 32), [3, 17, 39], [5, 6, 7]))
    tok, mask = (f(a) for f, a in zip((dev_i32, dev_u8), synth.window(shape, W, range(4, W))))

    def life(merged):
        kv = dl.KVCache(model, 160)
        dl.dllm_prefill(model.handle, kv.handle, dev_i32(synth.prompt_ids(shape, P)), P)
        ids, conf = torch.zeros(W, dtype=torch.int32, device="cuda"), torch.zeros(W, device="cuda")
        if merged:
            dl.dllm_step_merged(model.handle, kv.handle, pos, new, 3, block, 32, tok, mask, W, ids, conf)
        else:
            dl.dllm_refresh_kv(model.handle, kv.handle, pos, new, 3)
            dl.dllm_append_prefix_kv(model.handle, kv.handle, block, 32)
            dl.dllm_denoise_step(model.handle, kv.handle, tok, mask, W, ids, conf)
        need = torch.ones(W, dtype=torch.uint8, device="cuda")
        wid, wconf = torch.zeros_like(ids), torch.zeros_like(conf)
        (dl.dllm_denoise_window_sls(model.handle, kv.handle, P + 32, tok, mask, need, W, W, wid, wconf) if merged else
         dl.dllm_denoise_window(model.handle, kv.handle, P + 32, tok, mask, W, wid, wconf))
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in (conf, wconf)]

    plain = life(False)
    dl.dllm_model_set_qk_norm(model.handle, *gains(shape)[1])
    one, all_ = life(False), life(True)
    for a, b, c in zip(one, all_, plain):
        np.testing.assert_allclose(b, a, rtol=rtol)
        assert not np.allclose(a, c, rtol=1e-6)
