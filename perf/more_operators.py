"""Performance cases of the branching operators: a serving step whose sequences draft trees of tokens or several candidate
windows at once, over a paged K/V cache, apart from its matrix products.

A program that decodes so does five things around a model's step:

  tree     parents of the drafted tokens -> their positions and the rows that each of them sees
  attn     attention of all drafted rows: the cached positions, and of the drafted ones those that the row's mask has
  logp     log probabilities of the drafted tokens, the rows' entropies and the best alternatives, from the logits
  compact  K and V of the accepted path moved behind the sequence's cached positions, in every layer
  fork     sequences that go on as copies of others, or end: block tables, free pages, and copies of shared last pages

A case is a dict of plain values; "kind" is one of the five.  The plain forms below are elementary torch operations in 32
bits; with `own` the same inputs go through the library's calls.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ESIZE = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # a few small trees: the smallest step there is
        {"name": "tree_s8_r16", "kind": "tree", "seqs": 8, "rows": 16, "ragged": True},
        # many sequences with wide trees
        {"name": "tree_s64_r256", "kind": "tree", "seqs": 64, "rows": 256, "ragged": True},
        # fp32 model, small heads, ragged small trees
        {"name": "attn_f32_s4_r24", "kind": "attn", "dtype": "f32", "seqs": 4, "rows": 24, "heads": 4, "kv_heads": 2,
         "head_dim": 64, "shared": 0, "own": 900, "page": 32, "ragged": True, "branch": 0},
        # four sequences, each with four candidates of a 32-row window, behind 4000 positions of their own
        {"name": "attn_f16_s4_b4x32", "kind": "attn", "dtype": "f16", "seqs": 4, "rows": 128, "heads": 32,
         "kv_heads": 32, "head_dim": 128, "shared": 0, "own": 4000, "page": 64, "ragged": False, "branch": 32},
        # the largest: sixteen trees of up to 64 rows behind a shared document and texts of their own
        {"name": "attn_bf16_s16_r64", "kind": "attn", "dtype": "bf16", "seqs": 16, "rows": 64, "heads": 28,
         "kv_heads": 4, "head_dim": 128, "shared": 8192, "own": 3000, "page": 64, "ragged": True, "branch": 0},
        # a small fp32 model's tree
        {"name": "logp_f32_r16_v1024", "kind": "logp", "dtype": "f32", "rows": 16, "vocab": 1024, "tokens": 15, "top": 4},
        # one 32-row window of the 8B vocabulary: every row's own prediction, its alternatives as the next drafts
        {"name": "logp_f32_r32_v126464", "kind": "logp", "dtype": "f32", "rows": 32, "vocab": 126464, "tokens": 32,
         "top": 8},
        # a server's step: 256 rows, 16-bit logits, as many alternatives as interfaces usually offer
        {"name": "logp_bf16_r256_v152064", "kind": "logp", "dtype": "bf16", "rows": 256, "vocab": 152064,
         "tokens": 240, "top": 20},
        # two small trees of an fp32 model
        {"name": "compact_f32_s2_r16", "kind": "compact", "dtype": "f32", "seqs": 2, "rows": 16, "path": 5, "layers": 2,
         "kv_heads": 2, "head_dim": 64, "page": 32},
        # 32 trees of 64 rows, up to 16 of them accepted, all layers of a model with grouped heads
        {"name": "compact_f16_s32_r64", "kind": "compact", "dtype": "f16", "seqs": 32, "rows": 64, "path": 16,
         "layers": 28, "kv_heads": 4, "head_dim": 128, "page": 64},
        # a search over eight candidates: the best of them go on twice, the others end
        {"name": "fork_f16_s8", "kind": "fork", "dtype": "f16", "seqs": 8, "len": 400, "layers": 28, "kv_heads": 4,
         "head_dim": 128, "page": 64, "shared": 2, "table_ld": 16},
        # many sequences of a small model: tables and free pages count
        {"name": "fork_f32_s512", "kind": "fork", "dtype": "f32", "seqs": 512, "len": 1500, "layers": 2, "kv_heads": 1,
         "head_dim": 64, "page": 32, "shared": 0, "table_ld": 64},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(int(hi), int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    """A pass's rough time in seconds, for draws: what it cannot do without at 5 TB/s and 0.8 PFLOP/s (fp32: 0.1)."""
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / (1e14 if case.get("dtype") == "f32" else 8e14)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        if _cost(case) <= most:
            return case


def _draw(rng):
    kind = rng.choice(["tree", "attn", "attn", "attn", "logp", "logp", "compact", "fork"])
    if kind == "tree":
        seqs = _log_int(rng, 1, 256)
        return {"kind": kind, "seqs": seqs, "rows": _log_int(rng, 1, min(1024, 4 * int((4 << 18) / seqs) ** 0.5)),
                "ragged": rng.random() < 0.7}
    if kind == "logp":
        rows, vocab = _log_int(rng, 1, 256), _log_int(rng, 500, 152064)
        return {"kind": kind, "dtype": rng.choice(["f32", "f16", "bf16"]) if rows * vocab < 20_000_000 else "bf16",
                "rows": rows, "vocab": vocab, "tokens": rng.choice([0, rows, _log_int(rng, 1, 2 * rows)]),
                "top": rng.choice([0, 1, _log_int(rng, 2, 32)])}
    heads, kv, dh = rng.choice([(32, 32, 128), (28, 4, 128), (4, 4, 64), (4, 2, 64), (16, 2, 64), (4, 1, 128)])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    page = rng.choice([32, 64, 128])
    if kind == "attn":
        small = dtype == "f32"
        branch = rng.choice([0, 0, 8, 32])
        seqs = _log_int(rng, 1, 6 if small else 16)
        rows = branch * rng.randint(1, 3) if branch else _log_int(rng, 1, 64)
        return {"kind": kind, "dtype": dtype, "seqs": seqs, "rows": min(rows, max(branch, 96 if small else 1024 // seqs)),
                "heads": heads, "kv_heads": kv, "head_dim": dh,
                "shared": page * rng.choice([0, _log_int(rng, 1, (1024 if small else 6144) // page)]),
                "own": _log_int(rng, 1, 1000 if small else 3000), "page": page, "ragged": not branch and rng.random() < 0.7,
                "branch": branch}
    # a cache of at most 400 MB
    per = ESIZE[dtype] * 2 * kv * dh * page
    if kind == "compact":
        rows, seqs = _log_int(rng, 1, 128), _log_int(rng, 1, 64)
        layers = max(1, min(_log_int(rng, 1, 32), 400_000_000 // (per * seqs * (2 + rows // page + 1))))
        return {"kind": kind, "dtype": dtype, "seqs": seqs, "rows": rows, "path": _log_int(rng, 1, rows), "layers": layers,
                "kv_heads": kv, "head_dim": dh, "page": page}
    seqs, ld = _log_int(rng, 1, 128), rng.choice([16, 40, 64])
    length = _log_int(rng, 20, min(ld * page, max(40, page * (300_000_000 // per // seqs))))
    layers = max(1, min(_log_int(rng, 1, 32), 400_000_000 // (per * seqs * (length // page + 2))))
    return {"kind": kind, "dtype": dtype, "seqs": seqs, "len": length, "layers": layers, "kv_heads": kv, "head_dim": dh,
            "page": page, "shared": rng.choice([0, 0, 1]), "table_ld": ld}


# ----------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------


def _rand(case):
    """The case's own numbers, whatever the seed."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _rows(case):
    """Drafted rows of each sequence."""
    r, B, W = _rand(case), case["seqs"], case["rows"]
    rows = [r.randint(1, W) if case["ragged"] else W for _ in range(B)]
    if case["ragged"] and B >= 4:
        rows[1] = 0                          # a sequence that waits in this step
    return rows


def _cached(case):
    """Cached positions of each sequence behind the shared ones."""
    r, top = _rand(case), case["own"]
    return [r.randint((top + 1) // 2, top) if case["ragged"] else top for _ in range(case["seqs"])]


def _dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _gen(seed, stream=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + stream)
    return g


def _randn(shape, dtype, g, std=1.0):
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=g)


def _starts(counts):
    s = [0]
    for n in counts:
        s.append(s[-1] + n)
    return s


def prepare(case, seed):
    return {"tree": _prepare_tree, "attn": _prepare_attn, "logp": _prepare_logp, "compact": _prepare_compact,
            "fork": _prepare_fork}[case["kind"]](case, seed)


def _parents(rows, r):
    """Trees as drafting makes them, level by level: a row's parent is one of the few rows before it, or the cached text."""
    return [-1 if i == 0 or r.random() < 0.1 else r.randint(max(0, i - 6), i - 1) for n in rows for i in range(n)]


def _prepare_tree(case, seed):
    rows = _rows(case)
    r = random.Random(seed)
    T, ld = sum(rows), max(1, -(-max(rows) // 32))
    return {"kind": "tree", "rows": T, "mask_ld": ld, "row0": _dev(_starts(rows)),
            "len": _dev([n + r.randint(0, 8000) for n in rows]), "parent": _dev(_parents(rows, r) or [0]),
            "pos": torch.zeros(max(T, 1), dtype=torch.int32, device="cuda"),
            "mask": torch.zeros((max(T, 1), ld), dtype=torch.int32, device="cuda")}


def _words(masks, ld):
    """Masks (whole numbers of any size) as rows of ld 32-bit words."""
    w = [[(m >> 32 * i) & 0xFFFFFFFF for i in range(ld)] for m in masks]
    return _dev(w, torch.int64).to(torch.int32)


def _prepare_attn(case, seed):
    dt, page, B, S = DTYPES[case["dtype"]], case["page"], case["seqs"], case["shared"]
    H, Hk, Dh = case["heads"], case["kv_heads"], case["head_dim"]
    rows, cached = _rows(case), _cached(case)
    lens = [S + c + n for c, n in zip(cached, rows)]
    counts = [-(-n // page) for n in lens]
    sp = S // page
    n_pages, T = sp + sum(counts) - B * sp + 3, sum(rows)
    perm = torch.randperm(n_pages, device="cuda", generator=_gen(seed, 7)).to(torch.int32)
    c = _dev(counts, torch.int64) - sp
    first = sp + torch.cumsum(c, 0) - c
    ld = max(counts) + 2
    j = torch.arange(ld, device="cuda")
    at = torch.where(j < sp, j.expand(B, ld), first[:, None] + j - sp)
    table = torch.where(j < (c + sp)[:, None], perm[at.clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    masks = []
    if case["branch"]:                       # candidates of a window: a row sees all of its own candidate
        nb = case["branch"]
        masks = [((1 << nb) - 1) << (i // nb * nb) for n in rows for i in range(n)]
    else:                                    # trees: a row sees itself and its ancestors
        par, at0 = _parents(rows, random.Random(seed)), 0
        for n in rows:
            for i in range(n):
                p = par[at0 + i]
                masks.append((1 << i) | (masks[at0 + p] if p >= 0 else 0))
            at0 += n
    g = _gen(seed)
    R = T + 2                                # two rows behind the last sequence
    return {"kind": "attn", "page": page, "heads": H, "kv_heads": Hk, "head_dim": Dh, "shared": S, "rows": T,
            "max_rows": max(rows), "max_len": max(lens), "row0": _dev(_starts(rows)), "len": _dev(lens), "table": table,
            "mask": _words(masks + [0, 0], max(1, -(-max(rows) // 32))), "q": _randn((R, H, Dh), dt, g, 2.0),
            "k": _randn((n_pages, Hk, page, Dh), dt, g), "v": _randn((n_pages, Hk, Dh, page), dt, g),
            "out": torch.zeros((R, H, Dh), dtype=dt, device="cuda")}


def _prepare_logp(case, seed):
    T, V, n, k = case["rows"], case["vocab"], case["tokens"], case["top"]
    g = _gen(seed)
    f = lambda *sh: torch.zeros(sh, device="cuda")  # noqa: E731
    logits = _randn((T, V), DTYPES[case["dtype"]], g, 3.0)
    # a few tokens stand out, as a model's do
    best = torch.randint(0, V, (T, 4), device="cuda", generator=g)
    logits.scatter_add_(1, best, torch.rand((T, 4), device="cuda", generator=g).to(logits.dtype) * 16)
    row = torch.randint(0, T, (max(n, 1),), device="cuda", generator=g)
    tok = torch.where(torch.rand(row.shape, device="cuda", generator=g) < 0.7, best[row, 0], torch.randint(0, V, row.shape, device="cuda", generator=g))
    return {"kind": "logp", "mask_id": V - 1, "logits": logits, "tok": tok.to(torch.int32) if n else None,
            "tok_row": row.to(torch.int32) if n else None, "logp": f(n) if n else None, "entropy": f(T),
            "top_id": torch.zeros((T, k), dtype=torch.int32, device="cuda") if k else None, "top_logp": f(T, k) if k else None}


def _cache(case, n_pages, seed):
    """Every layer's K plane [n_pages][kv_heads][page][head_dim] and V^T plane [n_pages][kv_heads][head_dim][page]."""
    return _randn((case["layers"], 2, n_pages, case["kv_heads"], case["page"] * case["head_dim"]), DTYPES[case["dtype"]], _gen(seed))


def _paths(case):
    """(cached positions, accepted rows in order) of each sequence."""
    r, B, W = _rand(case), case["seqs"], case["rows"]
    return [(r.randint(0, 2 * case["page"] - 1), sorted(r.sample(range(W), r.randint(min(1, b), min(case["path"], W))))) for b in range(B)]


def _prepare_compact(case, seed):
    B, page, W = case["seqs"], case["page"], case["rows"]
    base, path = zip(*_paths(case))
    ld = (2 * page + W) // page + 1
    counts = [-(-(b + W) // page) for b in base]
    n_pages = sum(counts) + 2
    perm = torch.randperm(n_pages, device="cuda", generator=_gen(seed, 7)).to(torch.int32)
    c = _dev(counts, torch.int64)
    j = torch.arange(ld, device="cuda")
    at = (torch.cumsum(c, 0) - c)[:, None] + j
    return {"kind": "compact", "page": page, "head_dim": case["head_dim"], "pages": _cache(case, n_pages, seed),
            "table": torch.where(j < c[:, None], perm[at.clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous(),
            "base": _dev(base), "path": _dev([p + [0] * (case["path"] - len(p)) for p in path]), "n": _dev([len(p) for p in path])}


def _families(case):
    """(pages of the cache, lengths, page lists by number, sources, kept positions) of a batch before a fork."""
    r, B, page, sp, ld = _rand(case), case["seqs"], case["page"], case["shared"], case["table_ld"]
    lens = [max(sp * page, r.randint(case["len"] // 2, case["len"])) for _ in range(B)]
    lens = [min(n, ld * page) for n in lens]
    held, n_pages = [], sp
    for b, n in enumerate(lens):
        need = -(-n // page)
        # some sequences came from the one before them and still share its whole pages
        same = min(n, lens[b - 1]) // page if b and r.random() < 0.3 else sp
        held.append(list(range(sp)) + (held[b - 1][sp:same] if same > sp else []))
        n_new = need - len(held[b])
        held[b] += range(n_pages, n_pages + max(0, n_new))
        n_pages += max(0, n_new)
    src, keep = [], []
    for b in range(B):
        x = r.random()
        s = b if x < 0.5 else r.randrange(B)
        n = lens[s]
        src.append(s)
        # most go on where their source stands; some are cut, some end
        keep.append(n if x < 0.8 else (0 if x < 0.9 else r.randint(min(n, sp * page), n)))
    return n_pages + B + 4, lens, held, src, keep


def _prepare_fork(case, seed):
    B, page, ld = case["seqs"], case["page"], case["table_ld"]
    n_pages, lens, held, src, keep = _families(case)
    perm = torch.randperm(n_pages, device="cuda", generator=_gen(seed, 7)).to(torch.int32)
    ids = _dev([h + [-1] * (ld - len(h)) for h in held], torch.int64)
    used = max(max(h, default=-1) for h in held) + 1
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[:n_pages - used] = perm[used:]
    i32 = lambda *sh: torch.zeros(sh, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"kind": "fork", "page": page, "head_dim": case["head_dim"], "shared": case["shared"],
            "pages": _cache(case, n_pages, seed), "src": _dev(src), "keep": _dev(keep),
            "owned": _dev([len(h) for h in held]), "owned_out": i32(B),
            "table": torch.where(ids >= 0, perm[ids.clamp(min=0)], -1).to(torch.int32).contiguous(), "table_out": i32(B, ld) - 1,
            "free": free, "n_free": _dev([n_pages - used]), "n_free_out": i32(1), "status": i32(3)}


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------


def run(state):
    k = state["kind"]
    if own:
        return _own(state)
    return {"tree": _plain_tree, "attn": _plain_attn, "logp": _plain_logp, "compact": _plain_compact, "fork": _plain_fork}[k](state)


def _own(s):
    import paper_2606_13740_amd as dl

    if s["kind"] == "tree":
        dl.dllm_tree_plan(s["parent"], s["row0"], s["len"], s["pos"], s["mask"])
        return {"pos": s["pos"], "mask": s["mask"]}
    if s["kind"] == "attn":
        dl.dllm_attention_tree(s["q"], s["k"], s["v"], s["table"], s["row0"], s["len"], s["mask"], s["out"], s["max_rows"],
                               s["max_len"], shared_len=s["shared"])
        return {"out": s["out"]}
    if s["kind"] == "logp":
        dl.dllm_logprobs(s["logits"], tok=s["tok"], tok_row=s["tok_row"], logp=s["logp"], entropy=s["entropy"],
                         top_id=s["top_id"], top_logp=s["top_logp"], mask_id=s["mask_id"])
        return {k: s[k] for k in ("logp", "entropy", "top_id", "top_logp")}
    if s["kind"] == "compact":
        dl.dllm_cache_compact(s["pages"], s["page"], s["table"], s["base"], s["path"], s["n"])
        return {"pages": s["pages"]}
    dl.dllm_batch_fork(s["src"], s["keep"], s["owned"], s["owned_out"], s["table"], s["table_out"], s["free"], s["n_free"],
                       s["n_free_out"], s["shared"], s["pages"], s["page"], s["status"])
    return {k: s[k] for k in ("owned_out", "table_out", "free", "n_free_out", "pages", "status")}


def _row_seq(row0, T):
    """(sequence, index in it) of rows 0 .. T - 1."""
    r0 = row0.to(torch.int64)
    r = torch.arange(T, device=row0.device)
    b = torch.searchsorted(r0[1:].contiguous(), r, right=True)
    return b, r - r0[b]


def _plain_tree(s):
    T, ld = s["rows"], s["mask_ld"]
    B, W = s["len"].numel(), 32 * ld
    b, i = _row_seq(s["row0"], T)
    n = (s["row0"][1:] - s["row0"][:-1]).to(torch.int64)
    par = torch.full((B, W), -1, dtype=torch.int64, device=b.device)
    par[b, i] = s["parent"][:T].to(torch.int64)
    j = torch.arange(W, device=b.device)
    par = torch.where((par >= 0) & (par < j), par, -1)
    # paths of up to 1, 2, 4 ... edges: products of the matrix of single edges (and of standing still)
    reach = ((par[:, :, None] == j) | (j[:, None] == j)).to(torch.float32)
    for _ in range((W - 1).bit_length()):
        reach = torch.matmul(reach, reach).clamp(max=1)
    bits = (reach.view(B, W, ld, 32) > 0).to(torch.int64) << torch.arange(32, device=b.device)
    depth = reach.sum(-1).to(torch.int64) - 1
    s["mask"][:T] = bits.sum(-1)[b, i].to(torch.int32)
    s["pos"][:T] = (s["len"].to(torch.int64) - n)[b].add(depth[b, i]).to(torch.int32)
    return {"pos": s["pos"], "mask": s["mask"]}


def _pages(pool, ids, keys_last):
    """The K (or V^T) pages of `ids` [..., n] as [..., kv_heads, n * page, Dh] in 32 bits."""
    x = pool[ids.clamp(min=0)].to(torch.float32)
    x = x.transpose(-1, -2) if keys_last else x
    x = x.transpose(-4, -3)
    return x.reshape(*x.shape[:-3], -1, x.shape[-1]).contiguous()


def _plain_attn(s):
    T, W, S, page = s["rows"], s["max_rows"], s["shared"], s["page"]
    H, Hk, Dh = s["heads"], s["kv_heads"], s["head_dim"]
    G, B = H // Hk, s["table"].shape[0]
    dev = s["q"].device
    tab, row0, ln = (s[k].to(torch.int64) for k in ("table", "row0", "len"))
    seq, at = _row_seq(s["row0"], T)
    base = (ln - (row0[1:] - row0[:-1]))                        # cached positions
    q = (s["q"][:T].to(torch.float32) * (1.0 / math.sqrt(Dh))).view(T, Hk, G, Dh)
    # the sequences' own keys, rows padded to the longest tree
    ids = tab[:, S // page:S // page + -(-(s["max_len"] - S) // page)]
    idx = (row0[:-1, None] + torch.arange(W, device=dev)).clamp(max=T - 1)
    qp = q[idx].permute(0, 2, 1, 3, 4).reshape(B, Hk, W * G, Dh).contiguous()
    so = torch.matmul(qp, _pages(s["k"], ids, False).transpose(-1, -2).contiguous()).view(B, Hk, W, G, -1)
    key = S + torch.arange(so.shape[-1], device=dev)
    j = key - base[:, None]                                     # [B, keys]: which drafted row a key is
    jw = j.clamp(0, 32 * s["mask"].shape[1] - 1)
    words = s["mask"][idx]                                      # [B, W, mask_ld]
    bit = torch.gather(words, 2, (jw >> 5)[:, None].expand(B, W, -1)) >> (jw & 31).to(torch.int32)[:, None] & 1
    sees = ((j < 0)[:, None] | (bit != 0)) & (key < ln[:, None])[:, None]
    so = torch.where(sees[:, None, :, None, :], so, -math.inf)
    m = so.amax(-1)[seq, :, at]                                 # [T, Hk, G]
    if S:
        ks = _pages(s["k"], tab[0, :S // page], False)
        ss = torch.matmul(q.permute(1, 0, 2, 3).reshape(Hk, T * G, Dh).contiguous(), ks.transpose(-1, -2).contiguous()).view(Hk, T, G, S)
        m = torch.maximum(m, ss.amax(-1).permute(1, 0, 2))
    m0 = torch.where(m == -math.inf, 0, m)
    po = torch.exp(so - m0[idx].permute(0, 2, 1, 3)[..., None])
    oo = torch.matmul(po.view(B, Hk, W * G, -1), _pages(s["v"], ids, True)).view(B, Hk, W, G, Dh)
    o, den = oo[seq, :, at], po.sum(-1)[seq, :, at]             # [T, Hk, G, Dh], [T, Hk, G]
    if S:
        ps = torch.exp(ss - m0.permute(1, 0, 2)[..., None])
        o = o + torch.matmul(ps.view(Hk, T * G, S), _pages(s["v"], tab[0, :S // page], True)).view(Hk, T, G, Dh).permute(1, 0, 2, 3)
        den = den + ps.sum(-1).permute(1, 0, 2)
    o = torch.where(den[..., None] > 0, o / den[..., None], 0)
    s["out"][:T] = o.reshape(T, H, Dh).to(s["out"].dtype)
    return {"out": s["out"]}


def _plain_logp(s):
    x = s["logits"].to(torch.float32)
    T, V = x.shape
    x = torch.where(torch.isnan(x), -math.inf, x).clamp(max=torch.finfo(torch.float32).max)
    ids = torch.arange(V, device=x.device)
    x = torch.where(ids == s["mask_id"], -math.inf, x)
    m = x.amax(-1, keepdim=True)
    d = x - torch.where(m > -math.inf, m, 0)
    e = torch.exp(d)
    S = e.sum(-1)
    lse = torch.log(S)
    s["entropy"].copy_(torch.where(S > 0, lse - torch.where(e > 0, e * d, 0).sum(-1) / S, 0))
    if s["tok"] is not None:
        r, t = s["tok_row"].to(torch.int64), s["tok"].to(torch.int64)
        s["logp"].copy_(torch.where(S[r] > 0, d[r, t] - lse[r], -math.inf))
    if s["top_id"] is not None:
        # the order of (logit, then lower id first) as one whole number
        u = (x + 0.0).view(torch.int32).to(torch.int64)
        u = torch.where(u < 0, -2147483648 - u, u)
        key = (u << 32) + (V - 1 - ids)
        i = V - 1 - (torch.topk(key, s["top_id"].shape[1], dim=-1).values & 0xFFFFFFFF)
        lp = torch.gather(d, 1, i) - lse[:, None]
        s["top_id"].copy_(torch.where(lp > -math.inf, i, -1))
        s["top_logp"].copy_(lp)
    return {k: s[k] for k in ("logp", "entropy", "top_id", "top_logp")}


def _planes(s):
    """(K as [layers, n_pages, kv_heads, page, Dh], V^T as [layers, n_pages, kv_heads, Dh, page]), views of the cache."""
    p, Dh = s["pages"], s["head_dim"]
    L, _, n, Hk, _ = p.shape
    return p[:, 0].view(L, n, Hk, s["page"], Dh), p[:, 1].view(L, n, Hk, Dh, s["page"])


def _plain_compact(s):
    k, v = _planes(s)
    page = s["page"]
    tab, base, path = (s[x].to(torch.int64) for x in ("table", "base", "path"))
    i = torch.arange(path.shape[1], device=path.device)
    b, i = (i < s["n"][:, None]).nonzero(as_tuple=True)
    src, dst = base[b] + path[b, i], base[b] + i
    sp, so, dp, do = tab[b, src // page], src % page, tab[b, dst // page], dst % page
    k[:, dp, :, do] = k[:, sp, :, so]
    v[:, dp, :, :, do] = v[:, sp, :, :, so]
    return {"pages": s["pages"]}


def _plain_fork(s):
    k, v = _planes(s)
    page, sp, n_pages = s["page"], s["shared"], k.shape[1]
    src, keep, owned, n_free = (s[x].to(torch.int64) for x in ("src", "keep", "owned", "n_free"))
    tab = s["table"].to(torch.int64)
    B, ld = tab.shape
    dev = tab.device
    j, b = torch.arange(ld, device=dev), torch.arange(B, device=dev)
    need = (keep + page - 1) // page
    new = tab[src]
    last = (need - 1).clamp(min=0)
    part = (keep % page != 0) & (need > sp)                     # a last page that is not full
    held = (j < need[:, None]) & (j >= sp)
    full = held & ~(part[:, None] & (j == last[:, None]))
    one = lambda x: torch.zeros(n_pages + 1, dtype=torch.int64, device=dev).scatter(0, torch.where(x[0], x[1], n_pages).reshape(-1), 1)[:n_pages] > 0  # noqa: E731
    is_full, was = one((full, new)), one(((j < owned[:, None]) & (j >= sp), tab))
    mine = new[b, last]
    first = torch.full((n_pages + 1,), B, dtype=torch.int64, device=dev).scatter_reduce(0, torch.where(part, mine, n_pages), b, "amin")[:n_pages]
    at = mine.clamp(0, n_pages - 1)
    copy = part & (is_full[at] | (first[at] != b))
    gone = was & ~is_full & (first == B)
    n_gone, n_copy = gone.sum(), copy.sum()
    n_stack = n_free + n_gone
    short = (n_copy - n_stack).clamp(min=0)
    ok = (short == 0) & (need <= owned[src]).all()
    i = torch.arange(n_pages, device=dev)
    stack = torch.cat([s["free"], s["free"][:1]]).scatter(0, torch.where(gone, n_free + torch.cumsum(gone, 0) - 1, n_pages), i.to(torch.int32))
    fresh = stack[(n_stack - torch.cumsum(copy, 0)).clamp(0, n_pages - 1)].to(torch.int64)
    left = torch.where(ok, n_stack - n_copy, n_free)
    new = torch.where(copy[:, None] & (j == last[:, None]), fresh[:, None], new)
    s["table_out"].copy_(torch.where((j < torch.where(ok, need, owned)[:, None]), torch.where(ok, new, tab), s["table_out"]))
    s["free"].copy_(torch.where((i >= n_free) & (i < left), stack[:-1], s["free"]))
    c = (copy & ok).nonzero(as_tuple=True)[0]
    there = torch.arange(page, device=dev) < (keep % page)[c][:, None]
    f, m = fresh[c], mine[c]
    k[:, f] = torch.where(there[:, None, :, None], k[:, m], k[:, f])
    v[:, f] = torch.where(there[:, None, None, :], v[:, m], v[:, f])
    return {"owned_out": torch.where(ok, need, owned).to(torch.int32), "table_out": s["table_out"], "free": s["free"],
            "n_free_out": left.to(torch.int32), "pages": s["pages"],
            "status": torch.stack([n_copy, short[0], (~ok[0]).to(torch.int64)]).to(torch.int32)}


# ----------------------------------------------------------------------------
# What a pass cannot do without
# ----------------------------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "tree":
        rows = _rows(case)
        return {"bytes": 4.0 * (2 * len(rows) + sum(rows) * (2 + max(1, -(-max(rows) // 32)))), "flops": 0.0}
    if kind == "logp":
        T, V = case["rows"], case["vocab"]
        return {"bytes": 1.0 * T * V * ESIZE[case["dtype"]] + 12.0 * case["tokens"] + T * (4 + 8.0 * case["top"]), "flops": 5.0 * T * V}
    Hk, Dh, es = case["kv_heads"], case["head_dim"], ESIZE[case["dtype"]]
    if kind == "attn":
        H, rows, S = case["heads"], _rows(case), case["shared"]
        cached = _cached(case)
        keys = S + sum(c + n for c, n in zip(cached, rows))
        seen = sum(n * (S + c + (case["branch"] or 1)) for c, n in zip(cached, rows))
        return {"bytes": 2.0 * keys * Hk * Dh * es + 2.0 * sum(rows) * H * Dh * es, "flops": 4.0 * seen * H * Dh}
    per = 4.0 * case["layers"] * Hk * Dh * es                   # a position's K and V, read and written
    if kind == "compact":
        moved = sum(p != i for _, path in _paths(case) for i, p in enumerate(path))
        return {"bytes": per * moved + 4.0 * sum(len(p) + 2 for _, p in _paths(case)), "flops": 0.0}
    _, _, held, src, keep = _families(case)
    copied = sum(n for _, n in _copies(case, held, src, keep))
    return {"bytes": per * copied + 4.0 * (sum(len(h) for h in held) + sum(-(-n // case["page"]) for n in keep) + 5 * case["seqs"]), "flops": 0.0}


def _copies(case, held, src, keep):
    """(sequence, positions) of the last pages that a fork copies."""
    page, sp = case["page"], case["shared"]
    full, first = set(), {}
    for b, (s, n) in enumerate(zip(src, keep)):
        whole = n // page
        full.update(held[s][sp:whole])
        if n % page and whole >= sp:
            first.setdefault(held[s][whole], b)
    return [(b, n % page) for b, (s, n) in enumerate(zip(src, keep))
            if n % page and n // page >= sp and (held[s][n // page] in full or first[held[s][n // page]] != b)]


# ----------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# ----------------------------------------------------------------------------


def exact(case, seed):
    kind = case["kind"]
    if kind == "tree":
        return None                          # whole numbers only
    s = prepare(case, seed)
    f = torch.float64
    if kind == "logp":
        x = s["logits"].to(f)
        x[:, s["mask_id"]] = -math.inf
        lp = torch.log_softmax(x, -1)
        return {"logp": lp[s["tok_row"].long(), s["tok"].long()] if s["tok"] is not None else None,
                "entropy": torch.special.entr(lp.exp()).sum(-1), "top_id": None,
                "top_logp": lp.sort(-1, descending=True).values[:, :case["top"]].contiguous() if case["top"] else None}
    page, Dh = s["page"], s["head_dim"]
    if kind == "attn":
        H, Hk = s["heads"], s["kv_heads"]
        out = s["out"].to(f)
        start, lens = s["row0"].tolist(), s["len"].tolist()
        for b, n in enumerate(lens):
            a, e = start[b], start[b + 1]
            if a == e:
                continue
            ids = s["table"][b, :-(-n // page)].long()
            k = s["k"][ids].permute(1, 0, 2, 3).reshape(Hk, -1, Dh)[:, :n].to(f)
            v = s["v"][ids].permute(1, 0, 3, 2).reshape(Hk, -1, Dh)[:, :n].to(f)
            q = s["q"][a:e].to(f).view(e - a, Hk, -1, Dh).permute(1, 2, 0, 3).reshape(Hk, -1, Dh)
            hide = torch.zeros((e - a, n), dtype=torch.bool, device=k.device)
            for i, words in enumerate(s["mask"][a:e].tolist()):
                m = sum((w & 0xFFFFFFFF) << (32 * t) for t, w in enumerate(words))
                hide[i, n - (e - a):] = torch.tensor([not m >> t & 1 for t in range(e - a)])
            p = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(Dh)
            p = torch.softmax(p.view(Hk, -1, e - a, n).masked_fill(hide, -math.inf), -1).view(Hk, -1, n)
            out[a:e] = torch.bmm(p, v).view(Hk, H // Hk, e - a, Dh).permute(2, 0, 1, 3).reshape(e - a, H, Dh)
        return {"out": out}
    pages = s["pages"].to(f)
    L, _, n_pages, Hk, _ = pages.shape
    k, v = pages[:, 0].view(L, n_pages, Hk, page, Dh), pages[:, 1].view(L, n_pages, Hk, Dh, page)
    table = s["table"].tolist()
    if kind == "compact":
        for b, (base, path) in enumerate(_paths(case)):
            # one position after the other: an accepted row lies behind those that are written before it
            for i, p in enumerate(path):
                (sp, so), (dp, do) = ((table[b][x // page], x % page) for x in (base + p, base + i))
                k[:, dp, :, do], v[:, dp, :, :, do] = k[:, sp, :, so].clone(), v[:, sp, :, :, so].clone()
        return {"pages": pages}
    _, _, held, src, keep = _families(case)
    going = {p for b, n in enumerate(keep) for p in held[src[b]][case["shared"]:-(-n // page)]}
    name = {p: table[b][j] for b, h in enumerate(held) for j, p in enumerate(h)}
    gone = sorted(name[p] for h in held for p in set(h[case["shared"]:]) - going)
    stack = s["free"].tolist()[:int(s["n_free"])] + sorted(set(gone))
    for b, n in _copies(case, held, src, keep):
        a, d = table[src[b]][keep[b] // page], stack.pop()
        k[:, d, :, :n], v[:, d, :, :, :n] = k[:, a, :, :n].clone(), v[:, a, :, :, :n].clone()
    return {"owned_out": None, "table_out": None, "free": None, "n_free_out": None, "pages": pages, "status": None}
