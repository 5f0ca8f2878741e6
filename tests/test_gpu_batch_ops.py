"""The batch operators against plain 64-bit implementations: sizes, masks and strides where they can go wrong."""
import numpy as np
import pytest

from batch_util import EPS, attention, gather, plan, rounded, select, tdtype, to_gpu, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dl():
    import paper_2606_13740_amd as pkg
    return pkg


def i32(a):
    return to_gpu(np.asarray(a, dtype=np.int32))


# ---------------------------------------------------------------------------- plan


def plan_case(rng, B, ld, page, rows, spare, shared=0):
    length = rng.integers(0, (ld - 1) * page - rows, B)
    new = rng.integers(0, rows + 1, B)
    owned = np.minimum(ld, -(-length // page) + (rng.random(B) < 0.3) * rng.integers(0, 4, B))
    if shared:
        owned = np.maximum(owned, rng.integers(0, shared + 1, B))
    owned = np.minimum(owned, ld)
    n_pages = int(owned.sum() + np.maximum(0, -(-(length + new) // page) - owned).sum() + spare)
    n_pages = max(n_pages, 1)
    perm = rng.permutation(n_pages)
    table, at = np.full((B, ld), -7), 0
    for b in range(B):
        table[b, :owned[b]] = perm[at:at + owned[b]]
        at += owned[b]
    free = np.full(n_pages, -9)
    free[:n_pages - at] = perm[at:]
    return length, new, owned, table, free, n_pages - at, n_pages


def run_plan(dl, length, new, owned, table, free, n_free, n_pages, page, shared, R):
    import torch
    B = len(length)
    z = lambda n: torch.full((n,), 77, dtype=torch.int32, device="cuda")  # noqa: E731
    t, fr = i32(table), i32(free)
    o = dict(owned_out=z(B), n_free_out=z(1), row0=z(B + 1), pos=z(R), slot=z(R), seq=z(R), lim=z(R), status=z(3))
    dl.dllm_batch_plan(i32(length), i32(new), i32(owned), o["owned_out"], t, fr, i32([n_free]), o["n_free_out"], page,
                       shared, o["row0"], o["pos"], o["slot"], o["seq"], o["lim"], o["status"])
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in o.items()}, t.cpu().numpy(), fr.cpu().numpy()


def check_plan(dl, length, new, owned, table, free, n_free, n_pages, page, shared, R):
    got, t, fr = run_plan(dl, length, new, owned, table, free, n_free, n_pages, page, shared, R)
    rt, rf = table.copy(), free.copy()
    ref = plan(length, new, owned, rt, rf, n_free, page, shared, R, n_pages)
    for k, v in ref.items():
        assert np.array_equal(got[k], np.atleast_1d(v)), k
    assert np.array_equal(t, rt) and np.array_equal(fr, rf)
    return ref


@pytest.mark.parametrize("B,ld,page,rows,spare", [(1, 4, 32, 1, 0), (3, 8, 64, 40, 2), (64, 16, 32, 32, 5),
                                                  (513, 9, 128, 70, 0), (1500, 20, 32, 33, 11), (4096, 5, 256, 3, 1)])
def test_plan_matches_a_list(dl, B, ld, page, rows, spare):
    rng = np.random.default_rng(B + ld)
    length, new, owned, table, free, n_free, n_pages = plan_case(rng, B, ld, page, rows, spare)
    ref = check_plan(dl, length, new, owned, table, free, n_free, n_pages, page, 0, int(new.sum()) + 5)
    assert ref["status"][2] == 0


def test_plan_takes_pages_that_the_same_call_gives_back(dl):
    # one sequence finishes with all pages, nothing is free, the others need exactly those
    table = np.full((3, 6), -1)
    table[0, :4] = [5, 2, 7, 1]
    table[1, :1], table[2, :1] = 0, 3
    free = np.array([-9] * 8)
    ref = check_plan(dl, np.array([0, 32, 30]), np.array([0, 64, 40]), np.array([4, 1, 1]), table, free, 0, 8, 32, 0, 104)
    assert ref["status"].tolist() == [104, 0, 0] and ref["n_free_out"] == 0


def test_plan_keeps_shared_pages(dl):
    rng = np.random.default_rng(5)
    length, new, owned, table, free, n_free, n_pages = plan_case(rng, 9, 12, 32, 32, 40, shared=3)
    length[2], new[2] = 0, 0
    check_plan(dl, length, new, owned, table, free, n_free, n_pages, 32, 3, 400)


@pytest.mark.parametrize("what", ["pages", "rows", "table", "negative length", "negative count"])
def test_plan_refused_as_a_whole(dl, what):
    rng = np.random.default_rng(3)
    length, new, owned, table, free, n_free, n_pages = plan_case(rng, 6, 8, 32, 32, 0)
    length = np.minimum(length, 100)
    new = new.copy()
    new[1] = 32
    R = 400
    if what == "pages":
        new[3], length[3] = 32, owned[3] * 32
        n_free, owned = 0, -(-length // 32)
    elif what == "rows":
        R = int(new.sum()) - 1
    elif what == "table":
        new[0] = 8 * 32
        R = 2000
        length[0] = 40
        owned[0] = 2
        n_free = len(free)
        free[:] = np.arange(len(free))
    elif what == "negative length":
        length[4] = -1
    else:
        new[4] = -3
    got, t, fr = run_plan(dl, length, new, owned, table, free, n_free, n_pages, 32, 0, R)
    assert got["status"][2] == 1
    assert np.array_equal(t, table) and np.array_equal(fr, free)
    assert np.array_equal(got["owned_out"], owned) and got["n_free_out"][0] == n_free
    assert not got["row0"].any() and (got["slot"] == -1).all() and (got["seq"] == -1).all() and not got["lim"].any()


def test_plan_bad_table_entry_gives_no_slot(dl):
    table = np.array([[99, -1, 0]])
    got, _, _ = run_plan(dl, np.array([31]), np.array([34]), np.array([3]), table, np.full(4, -9), 0, 4, 32, 0, 34)
    assert got["slot"].tolist() == [-1] * 33 + [0] and got["pos"].tolist() == list(range(31, 65))


# ---------------------------------------------------------------------------- norm, rotation, cache write


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("H,Hk,D,page,T,gains", [(4, 2, 64, 32, 1, True), (28, 4, 128, 64, 37, True),
                                                 (3, 3, 32, 128, 70, True), (4, 1, 128, 32, 131, False),
                                                 (2, 2, 64, 256, 300, True)])
def test_qk_norm_rope(dl, dtype, H, Hk, D, page, T, gains):
    import torch
    rng = np.random.default_rng(T + H)
    width = (H + 2 * Hk) * D
    x, xt = rounded(rng, (T, width + 16), dtype, 2.0)         # a row stride wider than the row
    n_pages, max_pos = T // page + 5, 500
    kp, kt = rounded(rng, (n_pages, Hk, page, D), dtype)
    vp, vt = rounded(rng, (n_pages, Hk, D, page), dtype)
    gq, gk = (rng.normal(1, 0.1, D).astype(np.float32) for _ in range(2))
    rope = torch.empty(max_pos, D // 2, 2, device="cuda")
    dl.dllm_rope_table(rope, D, 10000.0)
    # a run of slots from the middle of a page on, a hole, and rows that have none
    slot = np.arange(T) + page - 3
    slot[T // 2:] += 5
    if T > 4:
        slot[2], slot[-1] = -1, n_pages * page
    pos = rng.integers(0, max_pos, T)
    if T > 4:
        pos[0], pos[1] = -4, max_pos + 10                     # read as the nearest entries
    q_out = torch.full((T, H, D), 7.0, dtype=tdtype(dtype), device="cuda")
    q, k, v = xt[:, :width].split([H * D, Hk * D, Hk * D], 1)
    dl.dllm_qk_norm_rope(q, k, v, rope, i32(pos), i32(slot), q_out, kt, vt, to_gpu(gq) if gains else None,
                         to_gpu(gk) if gains else None, 1e-6)
    torch.cuda.synchronize()
    cs = rope.double().cpu().numpy()[np.clip(pos, 0, max_pos - 1)]
    x = x[:, :width].reshape(T, H + 2 * Hk, D)
    rq, sq = turned(x[:, :H], gq.astype(np.float64) if gains else None, 1e-6, cs)
    rk, sk = turned(x[:, H:H + Hk], gk.astype(np.float64) if gains else None, 1e-6, cs)
    half = EPS[dtype] / 2
    # fp32: the sum of squares, its root and its quotient (8 roundings of the norm), two products and a sum
    bound = lambda r, s: 12 * 2.0 ** -24 * s + half * abs(r) * (1 + 2.0 ** -10) + 2.0 ** -25  # noqa: E731
    assert (abs(q_out.double().cpu().numpy() - rq) <= bound(rq, sq)).all()
    bk = np.zeros_like(kp)
    for r in range(T):
        if 0 <= slot[r] < n_pages * page:
            p, o = slot[r] // page, slot[r] % page
            kp[p, :, o], bk[p, :, o] = rk[r], bound(rk[r], sk[r])
            vp[p, :, :, o] = x[r, H + Hk:]
    assert (abs(kt.double().cpu().numpy() - kp) <= bk).all()  # untouched entries stay as they were
    assert np.array_equal(vt.double().cpu().numpy(), vp)


def test_qk_norm_rope_in_place_and_fp16_saturation(dl):
    import torch
    T, H, D = 5, 2, 64
    q = torch.full((T, H, D), 60000.0, dtype=torch.float16, device="cuda")
    k, v = q[:, :1].contiguous(), q[:, :1].contiguous()
    rope = torch.empty(8, D // 2, 2, device="cuda")
    dl.dllm_rope_table(rope, D, 10000.0)
    kp = torch.zeros(2, 1, 32, D, dtype=torch.float16, device="cuda")
    vp = torch.zeros(2, 1, D, 32, dtype=torch.float16, device="cuda")
    dl.dllm_qk_norm_rope(q, k, v, rope, i32([1] * T), i32(range(T)), q, kp, vp)      # cos 1 - sin 1 < 1 < cos 1 + sin 1
    assert q[:, :, D // 2].eq(65504).all() and torch.isfinite(q).all()
    assert kp[0, 0, :T, D // 2].eq(65504).all() and vp[0, 0, :, :T].eq(60000).all()


# ---------------------------------------------------------------------------- attention


def attn_case(rng, dtype, rows, lens, H, Hk, D, page, shared, extra_rows=2, q_std=2.0):
    B, T = len(rows), sum(rows)
    counts = [-(-n // page) for n in lens]
    sp = shared // page
    n_pages = sp + sum(max(0, c - sp) for c in counts) + 2
    perm = rng.permutation(n_pages)
    ld = max(max(counts), sp) + 1
    table, at = np.full((B, ld), -1), sp
    for b in range(B):
        table[b, :sp] = perm[:sp]
        for p in range(sp, counts[b]):
            table[b, p] = perm[at]
            at += 1
    q, qt = rounded(rng, (T + extra_rows, H, D), dtype, q_std)
    kp, kt = rounded(rng, (n_pages, Hk, page, D), dtype)
    vp, vt = rounded(rng, (n_pages, Hk, D, page), dtype)
    return dict(q=q, qt=qt, kp=kp, kt=kt, vp=vp, vt=vt, table=table, row0=np.concatenate([[0], np.cumsum(rows)]),
                lens=np.array(lens), page=page, shared=shared, rows=rows, n_pages=n_pages)


def check_attn(dl, c, dtype, lim=None, scale=None, max_len=None):
    import torch
    T, (R, H, D) = int(c["row0"][-1]), c["q"].shape
    out = torch.full((R, H, D), 7.0, dtype=tdtype(dtype), device="cuda")
    dl.dllm_attention_paged(c["qt"], c["kt"], c["vt"], i32(c["table"]), i32(c["row0"]), i32(c["lens"]), out,
                            max(c["rows"]), int(max(c["lens"])) if max_len is None else max_len, shared_len=c["shared"],
                            lim=None if lim is None else i32(lim), scale=scale)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    ref = attention(c["q"], c["kp"], c["vp"], c["table"], c["row0"], c["lens"], lim, c["shared"], c["page"],
                    D ** -0.5 if scale is None else scale, dtype)
    worst = 0.0
    for r, (o, bound) in ref.items():
        err = abs(got[r] - o)
        assert np.isfinite(got[r]).all() and (err <= bound + 1e-30).all(), (r, float(err.max()), float(bound.max()))
        worst = max(worst, float((err / (bound + 1e-30)).max()))
    assert (got[T:] == 7.0).all()
    print(f"  worst error / bound = {worst:.2f}", flush=True)
    return out


SHAPES = [  # rows, lens, H, Hk, D, page, shared
    ([1], [1], 4, 4, 64, 32, 0),
    ([1, 1, 1], [70, 33, 300], 4, 1, 128, 32, 0),
    ([32, 5, 0, 17], [200, 129, 64, 96], 4, 2, 64, 32, 64),
    ([7, 40], [512, 431], 7, 1, 128, 64, 384),
    ([33, 1, 64], [350, 257, 320], 2, 2, 128, 128, 256),
    ([3], [700], 6, 2, 64, 256, 512),
    ([100, 130], [260, 300], 2, 1, 128, 32, 32),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_paged(dl, dtype, shape):
    check_attn(dl, attn_case(np.random.default_rng(7), dtype, *shape), dtype)


@pytest.mark.parametrize("shape", [SHAPES[2], ([5, 9], [90, 40], 3, 3, 32, 32, 32)])
def test_attention_small_heads_fp32(dl, shape):
    check_attn(dl, attn_case(np.random.default_rng(8), "f32", *shape), "f32")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_row_limits(dl, dtype):
    """Causal rows, rows that see nothing, rows that end inside the shared part, limits past the length."""
    rng = np.random.default_rng(9)
    rows, lens = [40, 6, 3, 20], [230, 140, 65, 400]
    c = attn_case(rng, dtype, rows, lens, 4, 2, 128, 32, 64)
    lim = np.concatenate([np.arange(n - w + 1, n + 1) for w, n in zip(rows, lens)])
    lim[0], lim[1], lim[41], lim[42], lim[44], lim[50] = 0, -5, 1, 63, 64, 10 ** 6
    lim = np.concatenate([lim, [5, 5]])                                 # an entry per row of q, rows of nobody too
    check_attn(dl, c, dtype, lim=lim)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_ignores_what_it_must_not_see(dl, dtype):
    """NaN and infinities past a sequence's end, in pages of nobody, and tables with entries that are no pages."""
    import torch
    rng = np.random.default_rng(10)
    c = attn_case(rng, dtype, [20, 33, 4], [171, 97, 200], 4, 2, 64, 32, 64)
    used = np.zeros((c["n_pages"], 32), bool)
    for b, n in enumerate(c["lens"]):
        for p in range(n):
            used[c["table"][b, p // 32], p % 32] = True
    junk = torch.tensor(~used, device="cuda")
    for i, bad in enumerate((float("nan"), float("inf"))):
        c["kt"][junk[:, None, :, None].expand_as(c["kt"])] = bad
        c["vt"][junk[:, None, None, :].expand_as(c["vt"])] = bad
        check_attn(dl, c, dtype)
    c["table"][0, 3], c["table"][1, 2], c["table"][2, 5] = -1, c["n_pages"], 2 ** 31 - 1     # holes: their keys are not there
    check_attn(dl, c, dtype)


def run_attn(dl, c, lim):
    import torch
    out = torch.full_like(c["qt"], 7.0)
    dl.dllm_attention_paged(c["qt"], c["kt"], c["vt"], i32(c["table"]), i32(c["row0"]), i32(c["lens"]), out, max(c["rows"]),
                            int(max(c["lens"])), shared_len=c["shared"], lim=i32(lim))
    torch.cuda.synchronize()
    return out.float().cpu().numpy()


@pytest.mark.parametrize("dtype,rows,lens,H,Hk,D,shared", [
    ("f32", [1, 9, 30], [40, 70, 131], 4, 2, 32, 0), ("f32", [20, 25], [300, 250], 2, 1, 128, 64),
    ("f16", [1, 8], [64, 200], 2, 2, 64, 0), ("f16", [40, 33, 5], [300, 271, 100], 4, 2, 128, 128),
    ("bf16", [30], [190], 4, 4, 128, 0), ("bf16", [20, 64, 3], [130, 400, 60], 8, 2, 64, 128),
    ("f16", [64] * 8, [4200] * 7 + [4100], 28, 4, 128, 4096), ("bf16", [64] * 8, [4200] * 7 + [1500], 56, 8, 64, 4096)])
def test_attention_infinities_and_nans_that_only_some_rows_see(dl, dtype, rows, lens, H, Hk, D, shared):
    """Causal rows over V with a few infinities and NaNs (the last two cases: 128-row tiles).  Rows that see such a value
    get what a sum with it is; everything else keeps the bits it has with zeros in these places."""
    rng = np.random.default_rng(21)
    c = attn_case(rng, dtype, rows, lens, H, Hk, D, 32, shared)
    lim = np.concatenate([np.arange(n - w + 1, n + 1) for w, n in zip(rows, lens)] + [[1, 1]])
    spots = []                                          # (sequences, position, K/V head, dim, value)
    for b, (w, n) in enumerate(zip(rows, lens)):
        for p in rng.integers(max(n - w - 3, min(shared, n - 1)), n, 5):
            spots.append(([b], int(p), int(rng.integers(Hk)), int(rng.integers(D)), [np.inf, -np.inf, np.nan][rng.integers(3)]))
        spots += [([b], n - 1, 0, 3, np.inf), ([b], max(n - 2, 0), 0, 3, -np.inf)]
    if shared:                                          # sequences that end inside the shared part see less of it
        short = min(lens)
        spots += [([b for b in range(len(rows))], p, 0, 1, -np.inf) for p in (shared - 1, min(short, shared - 1), 0)]
    want_class = np.zeros((3, sum(rows), H, D), bool)   # +inf, -inf, NaN
    for clean in (True, False):
        for seqs, p, hk, d, x in spots:
            b = seqs[0] if p >= shared else 0
            if p < lens[b] or p < shared:
                page = c["table"][b, p // 32] if p >= shared else c["table"][0, p // 32]
                c["vt"][int(page), hk, d, p % 32] = 0.0 if clean else x
        if clean:
            base = run_attn(dl, c, lim)
    got = run_attn(dl, c, lim)
    for seqs, p, hk, d, x in spots:
        for b in seqs if p >= shared else range(len(rows)):
            for r in range(c["row0"][b], c["row0"][b + 1]):
                if p < min(lim[r], lens[b]):
                    cls = 2 if np.isnan(x) else int(x < 0)
                    want_class[cls, r, hk * (H // Hk):(hk + 1) * (H // Hk), d] = True
    pos, neg, nan = want_class
    nan = nan | (pos & neg)
    T = sum(rows)
    assert np.isfinite(base).all() and pos.any() and neg.any()
    assert (np.isnan(got[:T]) == nan).all()
    assert (got[:T][pos & ~nan] == np.inf).all() and (got[:T][neg & ~nan] == -np.inf).all()
    plain = ~(pos | neg | nan)
    assert plain.any() and (got[:T][plain] == base[:T][plain]).all() and (got[T:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_nan_keys(dl, dtype):
    """A NaN in K: NaN for the rows that see the key, in one part of the keys or all, and nothing for the others."""
    rng = np.random.default_rng(22)
    rows, lens = [30, 20], [230, 1100]
    c = attn_case(rng, dtype, rows, lens, 4, 2, 64, 32, 0)
    lim = np.concatenate([np.arange(n - w + 1, n + 1) for w, n in zip(rows, lens)] + [[1, 1]])
    ref = attention(c["q"], c["kp"], c["vp"], c["table"], c["row0"], c["lens"], lim, 0, 32, 64 ** -0.5, dtype)
    for b, p in ((0, 215), (1, 1090)):
        c["kt"][int(c["table"][b, p // 32]), 0, p % 32, 5] = float("nan")
    got = run_attn(dl, c, lim)
    for r, (o, bound) in ref.items():
        sees = lim[r] > (215 if r < 30 else 1090)
        for h in range(4):
            if sees and h < 2:
                assert np.isnan(got[r, h]).all(), (r, h)
            else:
                assert (abs(got[r, h] - o[h]) <= bound[h] + 1e-30).all(), (r, h)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_no_keys_at_all(dl, dtype):
    c = attn_case(np.random.default_rng(11), dtype, [3, 2], [0, 40], 2, 2, 64, 32, 0)
    out = check_attn(dl, c, dtype)
    assert not out[:3].any()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_attention_large_scores_and_scale(dl, dtype):
    """Scores whose maximum grows along the keys, far beyond what exp holds unshifted."""
    rng = np.random.default_rng(12)
    c = attn_case(rng, dtype, [9, 30], [310, 290], 4, 4, 64, 32, 128, q_std=6.0)
    check_attn(dl, c, dtype, scale=2.0)
    check_attn(dl, c, dtype, scale=-0.5)
    check_attn(dl, c, dtype, scale=0.0)


def test_attention_strided_rows_longer_bounds_and_repeats(dl):
    """q and out as slices of wider rows; max_len beyond every length; the same bits every time."""
    import torch
    rng = np.random.default_rng(13)
    c = attn_case(rng, "bf16", [32, 32, 11], [800, 700, 650], 4, 2, 128, 32, 608)
    plain = check_attn(dl, c, "bf16", max_len=(c["table"].shape[1] - 1) * 32)
    R, H, D = c["q"].shape
    wide = torch.zeros(R, 3 * H * D + 8, dtype=torch.bfloat16, device="cuda")
    wide[:, H * D:2 * H * D] = c["qt"].view(R, H * D)
    out = torch.full((R, 2 * H * D), 7.0, dtype=torch.bfloat16, device="cuda")
    args = (c["kt"], c["vt"], i32(c["table"]), i32(c["row0"]), i32(c["lens"]))
    for _ in range(3):
        dl.dllm_attention_paged(wide[:, H * D:2 * H * D], *args, out[:, H * D:], 32, (c["table"].shape[1] - 1) * 32,
                                shared_len=608)
        torch.cuda.synchronize()
        assert torch.equal(out[:, H * D:].reshape(R, H, D), plain) and out[:, :H * D].eq(7.0).all()


@pytest.mark.parametrize("shared", [0, 64])
def test_attention_rows_before_the_first_sequence(dl, shared):
    """row0 that does not begin at 0: the rows before it, like those behind the last, are left as they were."""
    import torch
    c = attn_case(np.random.default_rng(15), "f16", [20, 9], [210, 190], 4, 2, 64, 32, shared, extra_rows=5)
    args = (c["kt"], c["vt"], i32(c["table"]))
    out, moved = (torch.full_like(c["qt"], 7.0) for _ in range(2))
    dl.dllm_attention_paged(c["qt"], *args, i32(c["row0"]), i32(c["lens"]), out, 20, 210, shared_len=shared)
    dl.dllm_attention_paged(c["qt"].roll(3, 0), *args, i32(c["row0"] + 3), i32(c["lens"]), moved, 20, 210, shared_len=shared)
    torch.cuda.synchronize()
    assert torch.equal(moved[3:32], out[:29]) and moved[:3].eq(7.0).all() and moved[32:].eq(7.0).all()


def test_attention_on_another_stream_with_a_workspace(dl):
    """Two calls at once, each on its own stream with a workspace of its own."""
    import ctypes
    import torch
    cs = [attn_case(np.random.default_rng(16 + i), "bf16", [32, 32, 32], [1500, 1300, 900], 4, 2, 128, 32, 640) for i in range(2)]
    calls = [(c["qt"], c["kt"], c["vt"], i32(c["table"]), i32(c["row0"]), i32(c["lens"])) for c in cs]
    want = [torch.full_like(c["qt"], 7.0) for c in cs]
    for x, o in zip(calls, want):
        dl.dllm_attention_paged(*x, o, 32, 1500, shared_len=640)
    a, n = dl.dllm_attn_args(4, 98, 3, 4, 2, 128, 32, cs[0]["n_pages"], cs[0]["table"].shape[1], 640, 32, 1500, 0.1), ctypes.c_size_t()
    assert dl.lib().dllm_attention_paged_ws(ctypes.byref(a), ctypes.byref(n)) == 0
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.full((n.value,), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    got = [torch.full_like(w, 7.0) for w in want]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, o, st, ws in zip(calls, got, streams, spaces):
            dl.dllm_attention_paged(*x, o, 32, 1500, shared_len=640, ws=ws, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("bad", [dict(max_len=2 ** 32 + 8), dict(max_rows=2 ** 31), dict(scale=1e300), dict(shared_len="64")])
def test_attention_arguments_that_do_not_fit(dl, bad):
    """Numbers past their field's range are refused, not cut to 32 bits."""
    c = attn_case(np.random.default_rng(23), "f16", [4], [40], 2, 2, 64, 32, 0)
    args = dict(dict(max_rows=4, max_len=40), **bad)
    with pytest.raises(dl.DllmError):
        dl.dllm_attention_paged(c["qt"], c["kt"], c["vt"], i32(c["table"]), i32(c["row0"]), i32(c["lens"]), c["qt"].clone(), **args)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,lens,H,Hk,shared", [
    ([3, 5, 0, 7], [90, 40, 64, 130], 2, 2, 0), ([3, 5, 0, 7], [90, 40, 64, 130], 4, 2, 0), ([20, 33, 17], [300, 250, 90], 7, 1, 64),
    ([1] * 33, [540] * 32 + [500], 1, 1, 512)])
def test_attention_without_a_bound_of_rows(dl, dtype, rows, lens, H, Hk, shared):
    """max_rows = 2^31 - 1, no bound at all: the results of the tight one, and the rows behind the last as they were."""
    import torch
    c = attn_case(np.random.default_rng(24), dtype, rows, lens, H, Hk, 128, 32, shared, extra_rows=40)
    want = check_attn(dl, c, dtype)
    for bound in (max(rows) + 1, len(want), 2 ** 31 - max(rows), 2 ** 31 - 1):
        out = torch.full((len(want) + 64, H, 128), 7.0, dtype=tdtype(dtype), device="cuda")
        dl.dllm_attention_paged(c["qt"], c["kt"], c["vt"], i32(c["table"]), i32(c["row0"]), i32(c["lens"]), out[:len(want)], bound,
                                int(max(lens)), shared_len=shared)
        torch.cuda.synchronize()
        T = sum(rows)
        assert out[T:].eq(7.0).all(), bound
        # (another bound may choose another tile: two results inside the same bound of the reference)
        ref = attention(c["q"], c["kp"], c["vp"], c["table"], c["row0"], c["lens"], None, shared, 32, 128 ** -0.5, dtype)
        got = out.double().cpu().numpy()
        assert all((abs(got[r] - o) <= b + 1e-30).all() for r, (o, b) in ref.items()), bound


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_negative_lengths_are_empty(dl, dtype):
    """A sequence of a negative length sees nothing; the others are not touched by it."""
    import torch
    c = attn_case(np.random.default_rng(25), dtype, [3, 20, 4], [500, 430, 90], 4, 2, 64, 32, 64)
    want = check_attn(dl, c, dtype)
    for n in (-1, -2 ** 31):
        got = torch.full_like(c["qt"], 7.0)
        dl.dllm_attention_paged(c["qt"], c["kt"], c["vt"], i32(c["table"]), i32(c["row0"]), i32([500, n, 90]), got, 20, 500,
                                shared_len=64)
        torch.cuda.synchronize()
        assert not got[3:23].any() and torch.equal(got[:3], want[:3]) and torch.equal(got[23:], want[23:])


def test_offsets_past_32_bits(dl):
    """A pool of more than 2^31 elements a plane: the same bits from its last pages as from a small pool's."""
    import torch
    H, Hk, D, page, T = 8, 4, 128, 64, 70
    per = Hk * page * D
    n_big = 2 ** 31 // per + 8
    shift = n_big - 8                                        # page p of the small pool is page p + shift of the large one
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    mk = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(generator=g)  # noqa: E731
    small = (mk(8, Hk, page, D), mk(8, Hk, D, page))
    big = (torch.empty(n_big, Hk, page, D, dtype=torch.bfloat16, device="cuda"),
           torch.empty(n_big, Hk, D, page, dtype=torch.bfloat16, device="cuda"))
    for b, s in zip(big, small):
        b[shift:] = s
    qkv, rope = mk(T, (H + 2 * Hk) * D), torch.empty(400, D // 2, 2, device="cuda")
    dl.dllm_rope_table(rope, D, 10000.0)
    q, k, v = qkv.split([H * D, Hk * D, Hk * D], 1)
    pos = np.arange(300, 300 + T)
    table = np.array([[3, 0, 5, 1, 7, 2]])
    slot = table[0][pos // page] * page + pos % page
    outs = []
    for (kp, vp), s in ((small, 0), (big, shift)):
        qo, out = (torch.zeros(T, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        dl.dllm_qk_norm_rope(q, k, v, rope, i32(pos), i32(slot + s * page), qo, kp, vp)
        dl.dllm_attention_paged(qo, kp, vp, i32(table + s), i32([0, T]), i32([300 + T]), out, T, 6 * page)
        outs.append((qo, out))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert all(torch.equal(b[shift:], s) for b, s in zip(big, small))
    del big, small
    V, R = 152064, 2 ** 31 // 152064 + 60                    # logits of more than 2^31 elements
    x = torch.empty(R, V, dtype=torch.bfloat16, device="cuda")
    x[-50:] = mk(50, V)
    x[:-50] = x[-1]
    ids, conf = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, device="cuda")
    dl.dllm_select(x, ids, conf, mask_id=5)
    last = torch.zeros(50, dtype=torch.int32, device="cuda"), torch.zeros(50, device="cuda")
    dl.dllm_select(x[-50:].clone(), *last, mask_id=5)
    torch.cuda.synchronize()
    assert torch.equal(ids[-50:], last[0]) and torch.allclose(conf[-50:], last[1], rtol=1e-6, atol=0)
    assert ids[:-50].eq(last[0][-1]).all()


# ---------------------------------------------------------------------------- select


def select_case(rng, dtype, rows, V, hist, bias, n_allow, gap=0):
    B, T = len(rows), sum(rows)
    row0 = gap + np.concatenate([[0], np.cumsum(rows)])
    x, xt = rounded(rng, (T + 2 * gap, V), dtype, 3.0)
    c = dict(x=x, xt=xt, row0=row0, V=V, hist=None, hist0=None, n_prompt=None, rep=None, pres=None, freq=None,
             bias_id=None, bias=None, bias0=None, allow=None, allow_row=None, mask_id=V - 1)
    if hist:
        n = rng.integers(0, hist + 1, B)
        c["hist0"] = np.concatenate([[0], np.cumsum(n)])
        c["hist"] = rng.integers(-2, V + 2, n.sum() + 1)      # some outside the vocabulary
        c["n_prompt"] = rng.integers(0, n + 1)
        c["rep"], c["pres"], c["freq"] = (rng.uniform(a, b, B).astype(np.float32) for a, b in ((0.8, 1.6), (-1, 1), (-0.3, 0.5)))
    if bias:
        n = rng.integers(0, bias + 1, B)
        c["bias0"] = np.concatenate([[0], np.cumsum(n)])
        c["bias_id"] = rng.integers(-1, min(V, 40) + 1, n.sum() + 1)       # many twice
        c["bias"] = rng.normal(0, 4, n.sum() + 1).astype(np.float32)
    if n_allow:
        c["allow"] = rng.integers(-2 ** 31, 2 ** 31, (n_allow, (V + 31) // 32 + 1)).astype(np.int32)
        c["allow_row"] = rng.integers(-1, n_allow, T + 2 * gap)
    return c


def check_select(dl, c, dtype, out=True, gap=0):
    import torch
    R, V = c["x"].shape
    ids = torch.full((R,), 77, dtype=torch.int32, device="cuda")
    conf = torch.full((R,), 7.0, device="cuda")
    ol = torch.full((R, V), 7.0, dtype=tdtype(dtype), device="cuda") if out else None
    g = lambda k, f=i32: None if c[k] is None else f(c[k])  # noqa: E731
    dl.dllm_select(c["xt"], ids, conf, mask_id=c["mask_id"], row0=i32(c["row0"]), hist=g("hist"), hist0=g("hist0"),
                   n_prompt=g("n_prompt"), repetition=g("rep", to_gpu), presence=g("pres", to_gpu),
                   frequency=g("freq", to_gpu), bias_id=g("bias_id"), bias=g("bias", to_gpu), bias0=g("bias0"),
                   allow=g("allow"), allow_row=g("allow_row"), out_logits=ol)
    torch.cuda.synchronize()
    x, rid, rconf = select(c["x"], V, c["mask_id"], c["row0"], c["hist"], c["hist0"], c["n_prompt"], c["rep"], c["pres"],
                           c["freq"], c["bias_id"], c["bias"], c["bias0"], c["allow"], c["allow_row"])
    a, e = int(c["row0"][0]), int(c["row0"][-1])
    assert np.array_equal(ids.cpu().numpy()[a:e], rid[a:e])
    # a sum of V positive terms, each exp off by a few roundings of an exponent of at most ~100
    tol = (V / 16 + 256) * 2.0 ** -24
    got = conf.double().cpu().numpy()
    assert (abs(got[a:e] - rconf[a:e]) <= tol * rconf[a:e] + 1e-37).all()
    if out:
        want = torch.from_numpy(x).to(tdtype(dtype))
        assert torch.equal(ol.cpu()[a:e], want[a:e])
        assert ol[:a].eq(7.0).all() and ol[e:].eq(7.0).all()
    assert ids[:a].eq(77).all() and ids[e:].eq(77).all() and conf[e:].eq(7.0).all()
    return ids, conf


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,V,hist,bias,allow", [([1], 1, 3, 2, 0), ([5], 37, 30, 9, 2), ([32, 1, 0, 9], 1000, 200, 30, 3),
                                                    ([3, 4], 4099, 0, 0, 1), ([2, 2], 16411, 900, 0, 0),
                                                    ([17], 50001, 64, 5, 2)])
def test_select(dl, dtype, rows, V, hist, bias, allow):
    rng = np.random.default_rng(V + len(rows))
    check_select(dl, select_case(rng, dtype, rows, V, hist, bias, allow), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select_rows_of_nobody_stay(dl, dtype):
    rng = np.random.default_rng(3)
    check_select(dl, select_case(rng, dtype, [4, 3], 777, 20, 5, 2, gap=3), dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_select_ties_nan_and_infinities(dl, dtype):
    import torch
    rng = np.random.default_rng(4)
    c = select_case(rng, dtype, [9], 3001, 0, 0, 2)
    c["allow_row"] = np.array([-1, -1, -1, 0, 1, 2, -7, -1, -1])       # 2 and -7 are no masks: nothing is allowed
    c["allow"][0], c["allow"][1] = 0, 0
    c["allow"][1, 7] = 1 << 5                                           # a single id
    x = c["x"]
    x[0, [100, 2000, 2999]] = 64.0                                      # a tie far apart
    x[1, 5], x[1, 2000] = np.inf, np.inf
    x[2, :] = -np.inf
    x[4, 0] = np.inf                                                    # where the mask hides it
    x[4, 7 * 32 + 5] = -3.0
    x[7, :] = np.nan
    x[7, 11] = -1.0
    x[8, 3000] = np.inf                                                 # the MASK id's column
    c["xt"] = torch.from_numpy(x).to(tdtype(dtype)).cuda()
    ids, conf = check_select(dl, c, dtype, out=False)
    assert ids[:8].tolist()[:3] == [100, 5, -1] and ids[3:8].tolist() == [-1, 229, -1, -1, 11]
    assert conf[[2, 3, 5, 6]].eq(0).all() and conf[1] == 0.5 and conf[4] == 1


def test_select_strides_in_place_and_no_sequences(dl):
    """Rows that start at odd elements, logits adjusted in place, one sequence without row0, a mask per row."""
    import torch
    rng = np.random.default_rng(6)
    for dtype, V in (("f16", 1003), ("f32", 517), ("bf16", 2050)):
        c = select_case(rng, dtype, [6], V, 50, 6, 6)
        c["allow_row"] = np.arange(6)
        wide = torch.zeros(6, V + 7, dtype=tdtype(dtype), device="cuda")
        x = wide[:, 3:3 + V]
        x.copy_(c["xt"])
        ids, conf = torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(6, device="cuda")
        dl.dllm_select(x, ids, conf, mask_id=c["mask_id"], hist=i32(c["hist"]), hist0=i32(c["hist0"]),
                       n_prompt=i32(c["n_prompt"]), repetition=to_gpu(c["rep"]), presence=to_gpu(c["pres"]),
                       frequency=to_gpu(c["freq"]), bias_id=i32(c["bias_id"]), bias=to_gpu(c["bias"]), bias0=i32(c["bias0"]),
                       allow=i32(c["allow"]), out_logits=x)
        want, rid, _ = select(c["x"], V, c["mask_id"], c["row0"], c["hist"], c["hist0"], c["n_prompt"], c["rep"], c["pres"],
                              c["freq"], c["bias_id"], c["bias"], c["bias0"], c["allow"], c["allow_row"])
        assert ids.tolist() == rid.tolist()
        assert torch.equal(x.cpu(), torch.from_numpy(want).to(tdtype(dtype)))
        assert wide[:, :3].eq(0).all() and wide[:, 3 + V:].eq(0).all()


# ---------------------------------------------------------------------------- together, and captured


def test_select_with_histories_and_biases_that_are_empty(dl):
    """The first step of a batch: penalties are set, but no sequence has a history yet."""
    import torch
    x = torch.randn(5, 300, generator=torch.Generator().manual_seed(3)).cuda()
    e, two = i32([]), torch.full((2,), 2.0, device="cuda")
    outs = []
    for control in ({}, dict(hist=e, hist0=i32([0, 0, 0]), repetition=two, presence=two, frequency=two, n_prompt=i32([0, 0]),
                             bias_id=e, bias=torch.empty(0, device="cuda"), bias0=i32([0, 0, 0]))):
        outs.append((torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(5, device="cuda")))
        dl.dllm_select(x, *outs[-1], row0=i32([0, 3, 5]), **control)
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], x.argmax(1).int()) and all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("n_prompt", [2 ** 31 - 1, 2 ** 30, 5, 0, -1, -2 ** 31])
def test_select_with_prompts_of_any_length(dl, n_prompt):
    """More prompt entries than the history has: nothing was generated.  Fewer than none: everything was."""
    rng = np.random.default_rng(8)
    c = select_case(rng, "f32", [3, 4], 700, 300, 0, 0)
    c["hist0"] = np.array([0, 120, 250])
    c["hist"] = rng.integers(0, 40, 250)
    c["n_prompt"] = np.array([7, n_prompt])
    c["pres"], c["freq"] = np.array([0.5, 0.75], np.float32), np.array([0.25, 0.5], np.float32)
    check_select(dl, c, "f32")


def test_select_lists_that_end_at_the_last_index(dl):
    """A history and a bias list in the last entries of arrays of 2^31 - 1."""
    import torch
    rng, V, T, n, last = np.random.default_rng(10), 900, 4, 700, 2 ** 31 - 1
    c = select_case(rng, "f32", [T], V, 30, 9, 0)
    c["hist"], c["bias_id"], c["bias"] = rng.integers(-2, V + 2, n), rng.integers(0, V, n), rng.normal(0, 4, n).astype(np.float32)
    c["hist0"], c["bias0"], c["n_prompt"] = np.array([0, n]), np.array([0, n]), np.array([300])
    res = check_select(dl, c, "f32")
    far = {}
    for k, dt in (("hist", torch.int32), ("bias_id", torch.int32), ("bias", torch.float32)):
        far[k] = torch.empty(last, dtype=dt, device="cuda")
        far[k][last - n:] = to_gpu(c[k]).to(dt)
    ids, conf = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, device="cuda")
    at = i32([last - n, last])
    dl.dllm_select(c["xt"], ids, conf, mask_id=V - 1, row0=i32(c["row0"]), hist=far["hist"], hist0=at, n_prompt=i32(c["n_prompt"]),
                   repetition=to_gpu(c["rep"]), presence=to_gpu(c["pres"]), frequency=to_gpu(c["freq"]), bias_id=far["bias_id"],
                   bias=far["bias"], bias0=at)
    torch.cuda.synchronize()
    assert torch.equal(ids, res[0]) and torch.equal(conf, res[1])


REPETITIONS = [float("inf"), -float("inf"), float("nan"), 0.0, -0.0, 1e-40, 2.0 ** -126, 2.0 ** -125, 1e-30, 1e30, 2.0 ** 126,
               2.0 ** 127, 3.4e38, -1.7, 1.0000001, 0.9999999]


def test_select_repetition_of_any_size(dl):
    """Quotients and products by any float, rounded once; where the quotient is below 2^-100 its last bits may differ.  A
    subnormal factor counts as 0."""
    import torch
    rng = np.random.default_rng(9)
    B, V = len(REPETITIONS), 600
    c = select_case(rng, "f32", [2] * B, V, 40, 0, 0)
    n = 300
    c["hist0"], c["hist"] = np.arange(B + 1) * n, rng.integers(0, V, B * n)
    c["n_prompt"], c["pres"], c["freq"] = np.full(B, n), np.zeros(B, np.float32), np.zeros(B, np.float32)
    c["rep"] = np.array(REPETITIONS, np.float32)
    x = c["x"]
    x *= np.exp2(rng.integers(-20, 20, x.shape))
    x[:, ::50], x[:, 1::50], x[:, 2::50], x[:, 3::50], x[:, 4::50], x[:, 5::50] = 0.0, np.inf, -np.inf, 3e38, -3e38, 1e-44
    c["xt"] = torch.from_numpy(x.astype(np.float32)).cuda()
    c["x"] = x.astype(np.float32).astype(np.float64)
    ids, conf, out = (torch.zeros(s, dtype=t, device="cuda") for s, t in ((2 * B, torch.int32), (2 * B, torch.float32), ((2 * B, V), torch.float32)))
    dl.dllm_select(c["xt"], ids, conf, mask_id=V - 1, row0=i32(c["row0"]), hist=i32(c["hist"]), hist0=i32(c["hist0"]),
                   n_prompt=i32(c["n_prompt"]), repetition=to_gpu(c["rep"]), out_logits=out)
    torch.cuda.synchronize()
    with np.errstate(divide="ignore"):
        rep = np.where(abs(c["rep"]) < np.finfo(np.float32).tiny, np.copysign(0, c["rep"]), c["rep"]).astype(np.float32)
        want, rid, _ = select(c["x"], V, V - 1, c["row0"], c["hist"], c["hist0"], c["n_prompt"], rep, None, None, None, None, None,
                              None, None)
    got = out.cpu().numpy()
    with np.errstate(invalid="ignore"):                                 # (-inf - -inf, which the first term has)
        fine = (got == want) | ((abs(want) < 2.0 ** -100) & (abs(got - want) <= 2.0 ** -148))
    assert fine.all(), [(REPETITIONS[r // 2], float(c["x"][r, v]), float(got[r, v]), float(want[r, v])) for r, v in np.argwhere(~fine)[:8]]
    assert np.array_equal(ids.cpu().numpy(), rid)


def test_calls_without_rows(dl):
    import torch
    z = lambda *s, dt=torch.float16: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    kp, vp = z(3, 2, 32, 64), z(3, 2, 64, 32)
    dl.dllm_qk_norm_rope(z(0, 4, 64), z(0, 2, 64), z(0, 2, 64), z(8, 32, 2, dt=torch.float32), i32([]), i32([]), z(0, 4, 64), kp, vp)
    dl.dllm_attention_paged(z(0, 4, 64), kp, vp, i32([[0, 1]]), i32([0, 0]), i32([40]), z(0, 4, 64), 1, 40)
    dl.dllm_select(z(0, 100), i32([]), z(0, dt=torch.float32))
    torch.cuda.synchronize()
    assert not kp.any() and not vp.any()


def test_operators_of_a_step_together_and_captured(dl):
    """plan -> norm, rotation, cache write -> attention -> select, eagerly and replayed from a graph whose lengths change."""
    import torch
    rng = np.random.default_rng(14)
    B, page, ld, H, Hk, D, V, shared = 3, 32, 12, 4, 2, 64, 515, 64
    length, new = np.array([150, 64, 97]), np.array([32, 20, 0])
    R, n_pages = 96, 40
    perm = rng.permutation(n_pages)
    table, at = np.full((B, ld), -1), 2
    owned = -(-length // page)
    for b in range(B):
        table[b, :2] = perm[:2]
        table[b, 2:owned[b]] = perm[at:at + owned[b] - 2]
        at += owned[b] - 2
    free = np.concatenate([perm[at:], np.full(at, -9)])
    d = dict(len=i32(length), new=i32(new), owned=i32(owned), table=i32(table), free=i32(free), n_free=i32([n_pages - at]))
    z = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    p = dict(owned_out=z(B), n_free_out=z(1), row0=z(B + 1), pos=z(R), slot=z(R), seq=z(R), lim=z(R), status=z(3))
    x, xt = rounded(rng, (R, (H + 2 * Hk) * D), "bf16", 2.0)
    kp, kt = rounded(rng, (n_pages, Hk, page, D), "bf16")
    vp, vt = rounded(rng, (n_pages, Hk, D, page), "bf16")
    lg, lt = rounded(rng, (R, V), "f32", 3.0)
    gain = torch.ones(D, device="cuda")
    rope = torch.empty(512, D // 2, 2, device="cuda")
    dl.dllm_rope_table(rope, D, 10000.0)
    qo, out = (torch.zeros(R, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    total = d["len"] + d["new"]
    ids, conf = z(R), torch.zeros(R, device="cuda")

    def step():
        dl.dllm_batch_plan(d["len"], d["new"], d["owned"], p["owned_out"], d["table"], d["free"], d["n_free"], p["n_free_out"],
                           page, shared // page, p["row0"], p["pos"], p["slot"], p["seq"], p["lim"], p["status"])
        torch.add(d["len"], d["new"], out=total)
        q, k, v = xt.split([H * D, Hk * D, Hk * D], 1)
        dl.dllm_qk_norm_rope(q, k, v, rope, p["pos"], p["slot"], qo, kt, vt, gain, gain, 1e-6)
        dl.dllm_attention_paged(qo, kt, vt, d["table"], p["row0"], total, out, 32, ld * page, shared_len=shared, lim=p["lim"])
        dl.dllm_select(lt, ids, conf, row0=p["row0"])

    def check(length, new, owned, table, free, n_free):
        torch.cuda.synchronize()
        ref = plan(length, new, owned, table, free, n_free, page, shared // page, R, n_pages)
        for k in ("row0", "pos", "slot", "owned_out"):
            assert np.array_equal(p[k].cpu().numpy(), ref[k]), k
        assert np.array_equal(d["table"].cpu().numpy(), table)
        kg, vg = kt.double().cpu().numpy(), vt.double().cpu().numpy()
        T = int(ref["row0"][-1])
        xs = x.reshape(R, H + 2 * Hk, D)
        rk, sk = turned(xs[:T, H:H + Hk], np.ones(D), 1e-6, rope.double().cpu().numpy()[ref["pos"][:T]])
        for b in range(B):
            n = int(length[b] + new[b])
            K, V_ = gather(kg, table[b], n, page, False), gather(vg, table[b], n, page, True)
            a, e = ref["row0"][b], ref["row0"][b + 1]
            assert (abs(K[length[b]:] - rk[a:e]) <= 2.0 ** -8 * 1.01 * abs(rk[a:e]) + 2.0 ** -20 * sk[a:e]).all()
            assert np.array_equal(V_[length[b]:], xs[a:e, H + Hk:])
        res = attention(qo.double().cpu().numpy(), kg, vg, table, ref["row0"], length + new, ref["lim"], shared, page, D ** -0.5, "bf16")
        og = out.double().cpu().numpy()
        for r, (o, bound) in res.items():
            assert (abs(og[r] - o) <= bound).all()
        assert np.array_equal(ids.cpu().numpy()[:T], lg[:T].argmax(-1))
        return ref

    step()
    ref = check(length, new, owned, table, free, n_pages - at)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                              # the same plan again: the tables already hold its pages
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    owned, n_free = ref["owned_out"], int(ref["n_free_out"])
    for new2 in ([32, 0, 31], [1, 1, 1], [0, 32, 32], [32, 32, 32]):
        length, new = length + new, np.array(new2)
        for k, v in (("len", length), ("new", new), ("owned", owned)):
            d[k].copy_(i32(v))
        d["n_free"].fill_(n_free)
        for t in (qo, out, ids, conf):
            t.fill_(3)
        torch.cuda.synchronize()
        g.replay()
        ref = check(length, new, owned, table, free, n_free)
        owned, n_free = ref["owned_out"], int(ref["n_free_out"])
