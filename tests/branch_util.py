"""Plain implementations of the branching operators, from their definitions (64 bits, lists), and inputs for their tests."""
import numpy as np

from batch_util import EPS


def trees(rng, rows, back=6, roots=0.1):
    """Parents of `rows[b]` rows each: one of the `back` rows before, or -1."""
    return [[-1 if i == 0 or rng.random() < roots else int(rng.integers(max(0, i - back), i)) for i in range(n)] for n in rows]


def ancestors(parents):
    """A list of each row's set: itself and its ancestors (a parent that is no earlier row counts as none)."""
    res = []
    for i, p in enumerate(parents):
        res.append({i} | (res[p] if 0 <= p < i else set()))
    return res


def words(sets, ld):
    """int32 words [rows][ld] of the sets (numbers past them left out)."""
    out = np.zeros((len(sets), ld), np.uint32)
    for r, s in enumerate(sets):
        for j in s:
            if j < 32 * ld:
                out[r, j // 32] |= np.uint32(1 << j % 32)
    return out.view(np.int32)


def tree_attention(q, kp, vp, table, row0, length, lim, seen, shared, page, scale, dtype, part=None):
    """[(rows, out [rows, H, D], bound)] of every sequence, in 64 bits on the inputs' device.  q, kp, vp: float64 tensors;
    seen: {row: set of its sequence's rows}; lim: a limit per row or None.

    The bound: a score's D products in an fp32 chain are off by D * 2^-24 * sum |q k|, its scaling and the exponent by 4
    roundings, 4 * 2^-24 * (|s| + 1); an error of d in every score moves the output by at most 2 d max|v|.  The
    probabilities are off by half a step of `dtype` relative, in fp16 also half its smallest step (2^-25) absolute, sums over n
    keys by n * 2^-24 max|v| in numerator and denominator, and the output is rounded once."""
    import torch
    half = EPS[dtype] / 2
    H, D = q.shape[1:]
    n_pages, Hk = kp.shape[:2]
    res = []
    for b in range(len(row0) - 1):
        a, e, n = int(row0[b]), int(row0[b + 1]), int(length[b])
        if a == e:
            continue
        W, base = e - a, n - (e - a)
        ids = np.where(np.arange(table.shape[1]) < shared // page, table[0], table[b])[:-(-n // page)]
        ok = np.repeat((ids >= 0) & (ids < n_pages), page)[:n]
        at = torch.from_numpy(np.where((ids >= 0) & (ids < n_pages), ids, 0).astype(np.int64)).to(q.device)
        K = kp[at].permute(1, 0, 2, 3).reshape(Hk, -1, D)[:, :n]
        V = vp[at].permute(1, 0, 3, 2).reshape(Hk, -1, D)[:, :n]
        sees = np.zeros((W, n), bool)
        for i in range(W):
            sees[i, :base] = True
            for j in seen[a + i]:
                if 0 <= base + j < n:
                    sees[i, base + j] = True
            if lim is not None:
                sees[i, max(0, int(lim[a + i])):] = False
        sees &= ok
        m = torch.from_numpy(sees).to(q.device)[:, None, :]                      # [W, 1, n]
        G = H // Hk
        qs = q[a:e]
        kk, vv = K.repeat_interleave(G, 0), V.repeat_interleave(G, 0)            # [H, n, D]
        s = torch.matmul(qs.transpose(0, 1).contiguous(), kk.transpose(1, 2).contiguous()).transpose(0, 1) * scale
        mag = torch.matmul(qs.abs().transpose(0, 1).contiguous(), kk.abs().transpose(1, 2).contiguous()).transpose(0, 1) * abs(scale)
        zero = torch.zeros((), dtype=q.dtype, device=q.device)
        d = torch.where(m, (D * mag + 4 * (s.abs() + 1)) * 2.0 ** -24, zero).amax(-1)      # [W, H]
        s = torch.where(m, s, -torch.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.where(m, torch.exp(s - torch.where(top > -torch.inf, top, zero)), zero)
        den = p.sum(-1, keepdim=True)
        p, some = p / torch.where(den > 0, den, zero + 1), den[..., 0] > 0
        anyone = m.any(1).any(0) if m.shape[0] else m
        vv = torch.where(anyone[None, :, None], vv, zero)                          # (what no row sees may be anything)
        out = torch.matmul(p.transpose(0, 1).contiguous(), vv).transpose(0, 1)
        pa = torch.matmul(p.transpose(0, 1).contiguous(), vv.abs()).transpose(0, 1)
        vmax = vv.abs().amax(1)[None].amax(-1)                                     # [1, H]
        cnt = m[:, 0].sum(-1)[:, None].to(q.dtype)                                 # [W, 1]
        bound = (2 * d * vmax + 2 * cnt * 2.0 ** -24 * vmax)[..., None] + half * pa + half * out.abs()
        if dtype == "f16":
            # (the probabilities before the division by their sum, den >= 1)
            bound = bound + (cnt * 2.0 ** -25 * vmax / torch.where(den[..., 0] > 0, den[..., 0], zero + 1))[..., None]
        res.append((slice(a, e), torch.where(some[..., None], out, zero), torch.where(some[..., None], bound, zero)))
    return res


def logprobs(x, mask_id, tok, tok_row, top):
    """(logp, entropy, top ids, top logp, and bounds of the three) in 64 bits of the clamped logits x [T, V] (float64).

    Bounds.  A lane adds at most V / 64 + 32 terms and its sum is joined with others in at most 40 steps, each an fp32
    rounding; its largest logit moves at most V / 2048 + 20 times, each an exponential (2^-22, and 3 * 2^-24 |d| of an
    argument d, which the terms carry).  A term e^d is off by 3 * 2^-24 |d| + 2^-22 relative.  The logarithm and the
    differences round once each, the logarithm within two steps."""
    T, V = x.shape
    x = x.copy()
    u = 2.0 ** -24
    x[np.isnan(x)] = -np.inf
    x = np.minimum(x, float(np.finfo(np.float32).max))
    if mask_id >= 0:
        x[:, mask_id] = -np.inf
    m = x.max(1)
    some = m > -np.inf
    ref = np.where(some, m, 0)
    with np.errstate(invalid="ignore"):
        d = x - ref[:, None]
        e = np.exp(d)
        p = e / np.where(some, e.sum(1), 1)[:, None]
        ed = np.where(p > 0, p * -d, 0).sum(1)
        ed2 = np.where(p > 0, p * d * d, 0).sum(1)
    lse = np.log(np.where(some, e.sum(1), 1))
    chain = (V / 64 + 72) * u + (V / 2048 + 20) * 4 * u + 4 * u
    b_lse = chain + 3 * u * ed + 2 * u * abs(lse) + u
    entropy = np.where(some, lse + ed, 0.0)
    b_ent = b_lse + ed * 2 * chain + 3 * u * ed2 + u * (ed + entropy) + 2 * u
    lp = d - lse[:, None]
    lp[~some] = -np.inf
    b_of = lambda r, v: b_lse[r] + u * abs(d[r, v]) + u * abs(lp[r, v]) + u  # noqa: E731
    logp = b_logp = None
    if tok is not None:
        logp, b_logp = np.full(len(tok), -np.inf), np.zeros(len(tok))
        for i, v in enumerate(tok):
            r = i if tok_row is None else tok_row[i]
            if 0 <= r < T and 0 <= v < V and lp[r, v] > -np.inf:
                logp[i], b_logp[i] = lp[r, v], b_of(r, v)
    ids, tlp, b_t = np.full((T, top), -1), np.full((T, top), -np.inf), np.zeros((T, top))
    for r in range(T):
        order = np.lexsort((np.arange(V), -x[r]))[:top]
        order = order[x[r, order] > -np.inf]
        ids[r, :len(order)], tlp[r, :len(order)], b_t[r, :len(order)] = order, lp[r, order], b_of(r, order)
    return logp, entropy, ids, tlp, b_logp, b_ent, b_t


def valid_path(path, n, base, top):
    """The entries of a path that count."""
    res, before = [], -1
    for p in path[:max(0, min(n, len(path)))]:
        if p <= before or base + p >= top:
            break
        res.append(int(p))
        before = p
    return res


def compact(pages, page, D, table, base, path, n):
    """dllm_cache_compact on an array [layers][2][n_pages][heads][page * D], position by position."""
    L, _, n_pages, Hk, _ = pages.shape
    k, v = pages[:, 0].reshape(L, n_pages, Hk, page, D).copy(), pages[:, 1].reshape(L, n_pages, Hk, D, page).copy()
    for b in range(len(base)):
        if base[b] < 0:
            continue
        for i, p in enumerate(valid_path(path[b], n[b], base[b], table.shape[1] * page)):
            (s, so), (t, to) = ((int(table[b, x // page]), x % page) for x in (base[b] + p, base[b] + i))
            if 0 <= s < n_pages and 0 <= t < n_pages:
                k[:, t, :, to], v[:, t, :, :, to] = k[:, s, :, so].copy(), v[:, s, :, :, so].copy()
    return np.stack([k.reshape(L, n_pages, Hk, -1), v.reshape(L, n_pages, Hk, -1)], 1)


def fork(src, keep, owned, table, table_out, free, n_free, shared, page, pages, D):
    """dllm_batch_fork with sets and a list; pages [layers][2][n_pages][heads][page * D] is updated in place."""
    B, ld = table.shape
    n_pages = pages.shape[2]
    table_out, free = table_out.copy(), free.copy()

    def refused(copies, short):
        for b in range(B):
            n = min(max(int(owned[b]), 0), ld)
            table_out[b, :n] = table[b, :n]
        return dict(owned_out=np.array(owned), table_out=table_out, free=free, n_free_out=np.array([n_free]),
                    status=np.array([copies, short, 1]))

    need = [-(-int(k) // page) for k in keep]
    if not 0 <= n_free <= n_pages or any(not 0 <= s < B for s in src) or any(k < 0 for k in keep) or any(
            not 0 <= o <= ld for o in owned) or any(n > owned[s] for n, s in zip(need, src)):
        return refused(0, 0)
    is_page = lambda p: 0 <= p < n_pages  # noqa: E731
    whole, part = set(), {}
    for b in range(B):
        full = int(keep[b]) // page
        whole |= {int(p) for p in table[src[b], shared:full] if is_page(p)}
        if keep[b] % page and full >= shared and is_page(table[src[b], full]):
            part.setdefault(int(table[src[b], full]), b)
    held = {int(p) for b in range(B) for p in table[b, shared:owned[b]] if is_page(p)}
    stack = list(free[:n_free]) + sorted(held - whole - set(part))
    copies = []
    for b in range(B):
        full = int(keep[b]) // page
        if keep[b] % page and full >= shared and is_page(table[src[b], full]):
            p = int(table[src[b], full])
            if p in whole or part[p] != b:
                copies.append((b, p, int(keep[b]) % page))
    if len(copies) > len(stack):
        return refused(len(copies), len(copies) - len(stack))
    for b in range(B):
        table_out[b, :need[b]] = table[src[b], :need[b]]
    L, _, _, Hk, _ = pages.shape
    k, v = pages[:, 0].reshape(L, n_pages, Hk, page, D), pages[:, 1].reshape(L, n_pages, Hk, D, page)
    for b, p, n in copies:
        t = int(stack.pop())
        table_out[b, need[b] - 1] = t
        k[:, t, :, :n], v[:, t, :, :, :n] = k[:, p, :, :n], v[:, p, :, :, :n]
    free[n_free:len(stack)] = stack[n_free:]
    return dict(owned_out=np.array(need), table_out=table_out, free=free, n_free_out=np.array([len(stack)]),
                status=np.array([len(copies), 0, 0]))
