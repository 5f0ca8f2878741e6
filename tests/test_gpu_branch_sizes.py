"""The branching operators at the sizes whose launches smaller calls do not get: long token lists, many rows, several blocks a
wave, several heads a workgroup."""
import numpy as np
import pytest

from test_gpu_branch import check_logprobs, i32, logits_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dl():
    import paper_2606_13740_amd as pkg
    return pkg


# ---------------------------------------------------------------------------- given tokens


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V,n,top", [(1, 1, 1025, 1), (5, 40001, 1500, 4), (300, 700, 5000, 0), (1500, 300, 701, 2), (2100, 64, 2100, 0)])
def test_long_lists_of_tokens(dl, dtype, T, V, n, top):
    """Lists that get a launch of their own: tokens that are none, of rows that there are not, the MASK id, rows of -inf and NaN."""
    rng = np.random.default_rng(T + n)
    x = logits_of(rng, T, V, dtype)
    if T > 3:
        x[0], x[1], x[2, ::2] = -np.inf, float("nan"), float("inf")
    tok, row = rng.integers(-2, V + 2, n), rng.integers(-2, T + 2, n)
    tok[:5], row[:5] = [-2 ** 31, 2 ** 31 - 1, 0, 0, 0], [0, 0, -2 ** 31, 2 ** 31 - 1, T]
    check_logprobs(dl, x, dtype, mask_id=V // 2 if V > 1 else -1, tok=tok, tok_row=row, top=top, ld=V + 5)
    check_logprobs(dl, x, dtype, mask_id=V // 2 if V > 1 else -1, tok=tok, tok_row=row, top=top, entropy=False)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_token_is_its_rows_without_a_list_of_rows(dl, dtype):
    """As many tokens as rows, fewer, and one; with one part a row and with several."""
    rng = np.random.default_rng(5)
    for T, V in ((1100, 90), (600, 3000), (40, 20011)):
        x = logits_of(rng, T, V, dtype)
        x[T // 2] = -np.inf
        for n in (T, T - 3, 1):
            check_logprobs(dl, x, dtype, mask_id=3, tok=rng.integers(-1, V + 1, n), top=2)


@pytest.mark.parametrize("n", [1 << 20, 3])
@pytest.mark.parametrize("named", [True, False])
def test_a_million_rows(dl, n, named):
    """The work is that of the logits and the tokens, whatever their product.  Bounds as in branch_util.logprobs."""
    import torch
    T, V, u = 1 << 20, 8, 2.0 ** -24
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.empty(T, V, device="cuda").normal_(0, 3, generator=g)
    tok = torch.randint(0, V, (n,), dtype=torch.int32, device="cuda", generator=g)
    row = torch.randint(0, T, (n,), dtype=torch.int32, device="cuda", generator=g)
    lp, ent = torch.full((n,), 77.0, device="cuda"), torch.full((T,), 77.0, device="cuda")
    dl.dllm_logprobs(x, tok, row if named else None, lp, ent)
    d = x.double() - x.double().amax(1, keepdim=True)
    lse = d.exp().sum(1, keepdim=True).log()
    p = (d - lse).exp()
    ed, ed2 = (p * -d).sum(1), (p * d * d).sum(1)
    chain = (V / 64 + 72) * u + (V / 2048 + 20) * 4 * u + 4 * u
    b_lse = chain + 3 * u * ed + 2 * u * lse[:, 0] + u
    want = lse[:, 0] + ed
    assert ((ent.double() - want).abs() <= b_lse + ed * 2 * chain + 3 * u * ed2 + u * (ed + want) + 2 * u).all()
    r = row.long() if named else torch.arange(n, device="cuda")
    at = d[r, tok.long()]
    assert ((lp.double() - (at - lse[r, 0])).abs() <= b_lse[r] + u * at.abs() + u * (at - lse[r, 0]).abs() + u).all()


def test_long_lists_captured_and_replayed(dl):
    """One graph, replayed with other logits and tokens, equals the eager calls to the bit."""
    import torch
    rng = np.random.default_rng(9)
    T, V, n = 40, 20011, 3000
    cases = [(logits_of(rng, T, V, "bf16").cuda(), i32(rng.integers(0, V, n)), i32(rng.integers(0, T, n))) for _ in range(3)]
    z = lambda: [torch.zeros(n, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, 5, dtype=torch.int32, device="cuda"),  # noqa: E731
                 torch.zeros(T, 5, device="cuda")]
    x, tok, row = (t.clone() for t in cases[0])
    out, ws = z(), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    dl.dllm_logprobs(x, tok, row, *out, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dl.dllm_logprobs(x, tok, row, *out, ws=ws)
    for k in (1, 2, 0, 1):
        for t, s in zip((x, tok, row), cases[k]):
            t.copy_(s)
        for t in out:
            t.fill_(7)
        g.replay()
        ref = z()
        dl.dllm_logprobs(*cases[k], *ref)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
