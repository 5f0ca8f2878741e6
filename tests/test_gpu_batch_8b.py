"""dllm_batch_step at the full widths: every sequence's rows against the single-sequence step over a cache of its own (which is
compared with the oracle at these widths elsewhere).  Two layers: the launches depend on the widths and rows alone."""
import numpy as np
import pytest

import synth
from gpu_util import assert_ids_match_where_decided, assert_logits_close, dev_i32, gpu_logits, tol
from test_gpu_batch_step import Batch, gains, scene

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,dtype,n_prompt,blocks,windows,normed", [
    (synth.LLADA_8B, "bf16", 1056, [0, 40, 5, 64], [32, 32, 7, 0], False),
    (synth.LLADA_8B, "w8", 600, [10, 40], [9, 20], True),
    (synth.DREAM_7B, "q4", 1500, [64, 0, 17, 5], [32, 1, 32, 32], True)], ids=["LLaDA-8B bf16", "LLaDA-8B w8 normed", "Dream-7B q4 normed"])
def test_batch_step_at_full_width(shape, dtype, n_prompt, blocks, windows, normed):
    import paper_2606_13740_amd as dl
    import torch
    shape = shape.with_layers(2)
    layers, glob = [synth.layer_weights(shape, l, "bf16") for l in range(2)], synth.global_weights(shape, "bf16")
    model = dl.Model(shape, dtype, glob, lambda l: layers[l], max_window=128, max_pos=n_prompt + 200)
    print(f"case: {dtype}, {len(windows)} windows behind {n_prompt}", flush=True)
    if normed:
        dl.dllm_model_set_qk_norm(model.handle, *gains(shape)[1])
    prompt, own, win = scene(shape, n_prompt, blocks, windows, seed=2)
    bt = Batch(dl, model, len(windows), prompt, ld=n_prompt // 32 + 8, n_pages=n_prompt // 32 + 8 * len(windows))
    bt.step(np.concatenate(own), None, np.array(blocks))
    logits = torch.zeros(sum(windows), shape.vocab, device="cuda")
    ids, conf = bt.step(np.concatenate([t for t, _ in win]), np.concatenate([m for _, m in win]), np.array(windows), commit=False,
                        out=True, logits=logits, control=dict(mask_id=shape.mask_id))
    at = 0
    for o, (tok, mask) in zip(own, win):
        if not len(tok):
            continue
        kv = dl.KVCache(model, n_prompt + 160)
        dl.dllm_prefill(model.handle, kv.handle, dev_i32(prompt), n_prompt)
        if len(o):
            dl.dllm_append_prefix_kv(model.handle, kv.handle, dev_i32(o), len(o))
        want, wid, wconf = gpu_logits(model, kv, tok, mask)
        err = assert_logits_close(logits[at:at + len(tok)].double().cpu().numpy(), want, tol(dtype))
        got = ids[at:at + len(tok)]
        assert_ids_match_where_decided(got, want, err)
        same = got == wid
        # a logit off by e moves a softmax probability by at most a factor exp(2 e)
        assert (abs(conf[at:at + len(tok)] - wconf)[same] <= wconf[same] * (np.exp(2 * err) - 1) + 1e-6).all()
        at += len(tok)
    model.close()
