"""The branching operators at the sizes whose launches smaller calls do not get: long token lists, many rows, several blocks a
wave, several heads a workgroup."""
import numpy as np
import pytest

import test_gpu_branch
from batch_util import tdtype
from branch_util import logprobs, tree_attention
from test_gpu_branch import attn_case, check_logprobs, check_out, i32, logits_of, random_sets, run_tree, sets_to_mask

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


# ---------------------------------------------------------------------------- several blocks a wave


def special_rows(rng, V, dtype, mask_id):
    """Rows whose best ids, largest logits, ties, NaN and infinities lie in one of a wave's later blocks, or in several."""
    import torch
    t = tdtype(dtype)
    i, top, inf = torch.arange(V), float(torch.finfo(t).max), float("inf")
    blk = i.div(2048, rounding_mode="floor")
    noise = torch.from_numpy(rng.normal(0, 3, V).astype(np.float32))
    rows = [torch.zeros(V), torch.from_numpy(rng.integers(0, 3, V).astype(np.float32)), blk.float(), -blk.float(),      # ties
            torch.where(i % 7 == 0, 0.0, -0.0), (blk == blk.max() - 1).float() * 5,
            torch.where(i % 2048 == 5, 4.0, noise.clamp(max=3.9)), torch.where((i % 2048 < 3) & (blk % 4 == 2), 9.0, noise.clamp(max=8)),
            torch.linspace(-20, 30, V), torch.linspace(30, -20, V), torch.linspace(-1000, 1000, V),                     # sorted
            noise + 5.0 * blk, noise - 5.0 * blk, noise + 60.0 * (blk % 3 == 1)]                                       # the largest moves
    odd = noise.clone()
    odd[blk >= 5], odd[V - 100:] = float("nan"), 2.5
    rows.append(odd)
    odd = torch.where(i % 2 == 0, float("nan"), noise)
    odd[: 6 * 2048] = -inf
    rows.append(odd)
    odd = noise.clone()
    odd[7 * 2048 + 3], odd[V - 2], odd[9 * 2048] = inf, inf, top
    rows.append(odd)
    odd = torch.full((V,), -inf)
    odd[V - 5] = 1.5                                   # one id left, in the last block
    rows.append(odd)
    odd = torch.full((V,), -top)
    odd[5 * 2048: 5 * 2048 + 70], odd[V - 1] = 3.0, 3.0
    rows.append(odd)
    odd = torch.full((V,), -inf)
    odd[mask_id] = 4.0
    rows += [odd, torch.full((V,), float("nan")), torch.full((V,), -top)]
    odd = noise.clone()
    odd[3000::2048] = -inf
    rows.append(odd)
    return torch.stack(rows).to(t)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,V", [(256, 70001), (1100, 70001), (300, 152064)])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_logprobs_several_blocks_a_wave(dl, dtype, T, V, top):
    """A wave's list, its bound, what waits and its reference carried from block to block, with several parts a row and one:
    special rows at several places among T, all copies alike to the bit, one of each against 64 bits."""
    import torch
    mask_id = 11 * 2048 + 7
    rng = np.random.default_rng(top)
    x = special_rows(rng, V, dtype, mask_id)
    n = len(x)
    rows = torch.arange(T) % n
    g = x.cuda()[rows.cuda()]
    tok = np.concatenate([rng.integers(0, V, 300), [mask_id, 0, V - 1, V - 2, V - 5, 5 * 2048] * 20])
    of = rng.integers(0, T, len(tok))
    z = lambda *s: torch.full(s, 77.0, device="cuda")  # noqa: E731
    lp, ent, tl, ids = z(len(tok)), z(T), z(T, top), torch.full((T, top), -77, dtype=torch.int32, device="cuda")
    dl.dllm_logprobs(g, i32(tok), i32(of), lp, ent, ids, tl, mask_id)
    for out in (ent, ids, tl):
        assert torch.equal(out, out[:n][rows.cuda()])
    want = logprobs(x.double().numpy(), mask_id, tok, of % n, top)
    far = lambda got, ref: np.where(np.isneginf(ref) & np.isneginf(got), 0, abs(got - ref))  # noqa: E731
    with np.errstate(invalid="ignore"):
        assert np.array_equal(ids[:n].cpu().numpy(), want[2])
        assert (far(tl[:n].double().cpu().numpy(), want[3]) <= want[6]).all()
        assert (far(lp.double().cpu().numpy(), want[0]) <= want[4]).all()
        assert (abs(ent[:n].double().cpu().numpy() - want[1]) <= want[5]).all()


# ---------------------------------------------------------------------------- several heads a workgroup


@pytest.mark.parametrize("dtype,B,W,P,L,Hk,D,page", [
    ("f16", 64, 20, 9, 7, 7, 32, 32), ("f32", 64, 20, 9, 7, 7, 32, 32), ("bf16", 60, 33, 16, 4, 13, 64, 32), ("f16", 34, 64, 20, 13, 7, 128, 32),
    ("f16", 96, 20, 9, 7, 7, 32, 32), ("f32", 96, 20, 9, 7, 7, 32, 32), ("f16", 96, 20, 9, 11, 12, 32, 32), ("f16", 100, 20, 17, 11, 13, 32, 32),
    ("f32", 100, 20, 9, 11, 13, 32, 32)])
def test_cache_compact_several_heads_a_workgroup(dl, dtype, B, W, P, L, Hk, D, page):
    """Two, three and eight heads of V^T a workgroup, the last one with fewer, even and odd."""
    test_gpu_branch.test_cache_compact(dl, dtype, B, W, P, L, Hk, D, page)


# ---------------------------------------------------------------------------- row bounds that are none


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shared", [0, 64])
def test_attention_tree_writes_rows_of_its_sequences_only(dl, dtype, shared):
    """Row bounds past the call's rows, negative and falling: guard rows around the output and rows that are neither a
    sequence's nor in [row0[0], row0[B]) stay, and where bounds cut to the call are those of whole sequences, so are the results."""
    import torch
    rng = np.random.default_rng(21)
    c = attn_case(rng, dtype, [20, 33], [100, 70], 4, 2, 64, 32, shared)
    T, G = c["T"], 64
    c["table"] = np.where(c["table"] < 0, 0, c["table"])          # (whatever is read is a page)
    ld = 2
    mask = sets_to_mask(c, random_sets(rng, c["rows"], c["row0"]), ld)
    bits = mask.cpu().numpy().view(np.uint32)
    seen_of = lambda r: {j for j in range(32 * ld) if bits[r, j // 32] >> np.uint32(j % 32) & 1}  # noqa: E731
    lo, hi = -2 ** 31, 2 ** 31 - 1
    for row0 in ([-5, 20, hi], [0, 20, 40], [lo, lo, lo], [hi, hi, hi], [0, lo, 40], [hi, 3, 9], [30, 10, 50], [7, 7, 7], [0, 0, hi], [lo, 20, 53]):
        for ln in ([120, 103], [120, 40], [lo, hi], [0, -1]):
            big = torch.full((T + 2 * G, 4, 64), 77.0, dtype=c["q"].dtype, device="cuda")
            out = big[G:G + T]
            dl.dllm_attention_tree(c["q"], c["k"], c["v"], i32(c["table"]), i32(row0), i32(ln), mask, out, T, 120, shared_len=shared)
            cut = [min(max(r, 0), T) for r in row0]
            inside = torch.zeros(T + 2 * G, dtype=torch.bool, device="cuda")
            for a, e in ((cut[0], cut[2]), (cut[0], cut[1]), (cut[1], cut[2])):       # all rows (the parts' merge), each sequence's
                inside[G + a:G + max(a, e)] = True
            assert big[~inside].eq(77).all(), (row0, ln)
            if cut == sorted(cut) and all(0 <= n <= 120 and n >= max(shared, e - a) for n, a, e in zip(ln, cut, cut[1:])):
                seen = {cut[b] + i: {j for j in seen_of(cut[b] + i) if j < cut[b + 1] - cut[b]} for b in range(2) for i in range(cut[b + 1] - cut[b])}
                for rows, want, bound in tree_attention(c["q"].double(), c["k"].double(), c["v"].double(), c["table"], cut, ln, None, seen, shared,
                                                        32, 64 ** -0.5, dtype):
                    assert ((out[rows].double() - want).abs() <= bound).all(), (row0, ln, rows)


# ---------------------------------------------------------------------------- the same bits


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,cached,H,Hk,shared", [([128] * 4, [2000] * 4, 32, 32, 0), ([64, 0, 33, 64, 5, 64], [8192 + 900] * 6, 28, 4, 8192)])
def test_attention_tree_repeats_itself(dl, dtype, rows, cached, H, Hk, shared):
    """Candidates of 32 rows and trees behind a shared prefix: equal bits on repeated calls, and, as the formula's bound has it, off by
    no more than the roundings of probabilities and output."""
    import torch
    rng = np.random.default_rng(4)
    c = attn_case(rng, dtype, rows, cached, H, Hk, 128, 64, shared)
    seen = {int(c["row0"][b]) + i: set(range(i // 32 * 32, i // 32 * 32 + 32)) & set(range(n)) for b, n in enumerate(rows) for i in range(n)}
    mask = sets_to_mask(c, seen, 4)
    out = run_tree(dl, c, mask)
    check_out(c, out, seen)
    for _ in range(10):
        assert torch.equal(run_tree(dl, c, mask), out)
