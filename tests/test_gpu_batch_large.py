"""The batch operators at sizes that take their other launches (tests/batch_large.py), against references in 64 bits."""
import numpy as np
import pytest

from batch_large import ATTN, LEAD, ODD, QK, SELECT, attn_inputs, attn_reference, limits
from batch_util import EPS, rounded, tdtype, to_gpu, turned
from test_gpu_batch_ops import check_select, i32, select_case
from test_gpu_batch_ops import test_attention_infinities_and_nans_that_only_some_rows_see as check_infinities

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dl():
    import paper_2606_13740_amd as pkg
    return pkg


def call(dl, c, x, lim):
    import torch
    out = torch.full_like(x["q"], 7.0)
    dl.dllm_attention_paged(x["q"], x["k"], x["v"], i32(x["table"]), i32(x["row0"]), i32(x["lens"]), out, max(c.rows), max(c.lens),
                            shared_len=c.prefix, lim=None if lim is None else i32(lim))
    torch.cuda.synchronize()
    return out


def check(c, x, dtype, lim, out):
    got, worst = out.double().cpu().numpy(), 0.0
    for r, (o, bound) in attn_reference(c, x, dtype, lim).items():
        err = abs(got[r] - o)
        assert np.isfinite(got[r]).all() and (err <= bound + 1e-30).all(), (r, float(err.max()), float(bound.max()))
        worst = max(worst, float((err / (bound + 1e-30)).max()))
    T = LEAD + sum(c.rows)
    assert (got[:LEAD] == 7.0).all() and (got[T:] == 7.0).all()
    print(f"  worst error / bound = {worst:.2f}", flush=True)


CASES = [pytest.param(c, t, id=f"{c.name} {t}") for c in ATTN for t in c.dtypes]


@pytest.mark.parametrize("c,dtype", CASES)
def test_attention(dl, c, dtype):
    """Ragged rows from row 3 on, a waiting sequence, sequences that end inside the prefix and with it; the same bits twice."""
    import torch
    x = attn_inputs(c, dtype, 1, 0.0)
    out = call(dl, c, x, None)
    check(c, x, dtype, None, out)
    assert torch.equal(out, call(dl, c, x, None))


@pytest.mark.parametrize("c,dtype", CASES)
def test_attention_limits_over_junk(dl, c, dtype):
    """Causal rows, rows that see nothing or end inside the prefix; NaN wherever no sequence has a position."""
    x = attn_inputs(c, dtype, 2, float("nan"))
    lim = limits(c)
    check(c, x, dtype, lim, call(dl, c, x, lim))


@pytest.mark.parametrize("c,dtype", CASES)
def test_attention_holes(dl, c, dtype):
    """Table entries that are no pages, in the prefix (of every sequence) and behind it: their keys are not there."""
    x = attn_inputs(c, dtype, 3, float("inf"))
    sp, n_pages = c.prefix // c.page, x["k"].shape[0]
    for at, bad in ((0, -1), (sp // 2, n_pages), (max(sp - 1, 0), 2 ** 31 - 1)):
        if sp:
            x["table"][:, at] = bad
    for b, n in enumerate(c.own):
        if n > c.page:
            x["table"][b, sp] = (-1, n_pages + 5)[b % 2]
    check(c, x, dtype, None, call(dl, c, x, None))
    lim = limits(c)
    check(c, x, dtype, lim, call(dl, c, x, lim))


@pytest.mark.parametrize("dtype,rows,lens,H,Hk,D,prefix,tile", ODD)
def test_attention_infinities_and_nans_that_only_some_rows_see(dl, dtype, rows, lens, H, Hk, D, prefix, tile):
    check_infinities(dl, dtype, list(rows), list(lens), H, Hk, D, prefix)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,V,hist,bias,allow,per,four", SELECT)
def test_select(dl, dtype, rows, V, hist, bias, allow, per, four):
    """Tables, masks, kept logits and sequences that change inside a workgroup's rows, at more workgroups than the chip holds."""
    rng = np.random.default_rng(V + len(rows))
    check_select(dl, select_case(rng, dtype, list(rows), V, hist, bias, allow), dtype)


def test_select_rows_of_nobody_stay(dl):
    rng = np.random.default_rng(5)
    check_select(dl, select_case(rng, "bf16", [900, 0, 601], 4099, 200, 9, 2, gap=7), "bf16")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,H,Hk,D,page,heads", QK)
@pytest.mark.parametrize("gains", [True, False])
def test_qk_norm_rope(dl, dtype, T, H, Hk, D, page, heads, gains):
    """Several heads a lane group, a group of fewer at the end; also in place."""
    import torch
    rng = np.random.default_rng(T + H)
    width = (H + 2 * Hk) * D
    x, xt = rounded(rng, (T, width + 16), dtype, 2.0)
    n_pages, max_pos = T // page + 5, T + 50
    kt, vt = (torch.zeros(s, dtype=tdtype(dtype), device="cuda") for s in ((n_pages, Hk, page, D), (n_pages, Hk, D, page)))
    gq, gk = (rng.normal(1, 0.1, D).astype(np.float32) for _ in range(2))
    rope = torch.empty(max_pos, D // 2, 2, device="cuda")
    dl.dllm_rope_table(rope, D, 10000.0)
    pos, slot = rng.permutation(T) + 7, rng.permutation(n_pages * page)[:T]
    slot[5], slot[-2] = -1, n_pages * page
    q_out = torch.full((T, H, D), 7.0, dtype=tdtype(dtype), device="cuda")
    q, k, v = xt[:, :width].split([H * D, Hk * D, Hk * D], 1)
    args = (k, v, rope, i32(pos), i32(slot))
    g = (to_gpu(gq), to_gpu(gk)) if gains else (None, None)
    dl.dllm_qk_norm_rope(q, *args, q_out, kt, vt, *g, 1e-6)
    same = q.reshape(T, H, D).contiguous()
    dl.dllm_qk_norm_rope(same, *args, same, kt, vt, *g, 1e-6)
    torch.cuda.synchronize()
    assert torch.equal(same, q_out)
    cs = rope.double().cpu().numpy()[pos]
    x = x[:, :width].reshape(T, H + 2 * Hk, D)
    wide = lambda a: a.astype(np.float64) if gains else None  # noqa: E731
    (rq, sq), (rk, sk) = turned(x[:, :H], wide(gq), 1e-6, cs), turned(x[:, H:H + Hk], wide(gk), 1e-6, cs)
    half = EPS[dtype] / 2
    # the roundings of the smaller test: norm, two products and a sum in fp32, then the type's
    bound = lambda r, s: 12 * 2.0 ** -24 * s + half * abs(r) * (1 + 2.0 ** -10) + 2.0 ** -25  # noqa: E731
    assert (abs(q_out.double().cpu().numpy() - rq) <= bound(rq, sq)).all()
    ok = (slot >= 0) & (slot < n_pages * page)
    kg = kt.double().cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, Hk, D)
    vg = vt.double().cpu().numpy().transpose(0, 3, 1, 2).reshape(-1, Hk, D)
    assert (abs(kg[slot[ok]] - rk[ok]) <= bound(rk, sk)[ok]).all()
    assert np.array_equal(vg[slot[ok]], x[ok, H + Hk:])
    rest = np.setdiff1d(np.arange(n_pages * page), slot[ok])
    assert not kg[rest].any() and not vg[rest].any()
