"""Plain 64-bit implementations of the batch operators, from their definitions, and inputs for their tests."""
import numpy as np

EPS = {"f32": 2.0 ** -23, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}      # torch.finfo(t).eps


def tdtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def to_gpu(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def rounded(rng, shape, dtype, std=1.0):
    """Normal values that `dtype` holds exactly, as float64 and as a GPU tensor."""
    import torch
    t = torch.from_numpy(rng.normal(0.0, std, shape).astype(np.float32)).to(tdtype(dtype))
    return t.double().numpy(), t.cuda()


def plan(length, new, owned, table, free, n_free, page, shared, max_rows, n_pages):
    """dllm_batch_plan with a list for the stack; table and free are updated in place."""
    B, ld = table.shape
    need = [-(-(int(a) + int(b)) // page) for a, b in zip(length, new)]
    keep = [max(n, min(shared, int(o))) for n, o in zip(need, owned)]
    row0 = np.concatenate([[0], np.cumsum(new)])
    stack = list(free[:n_free])
    for b in range(B):
        stack += list(table[b, keep[b]:owned[b]]) if owned[b] > keep[b] else []
    take = sum(max(0, n - int(o)) for n, o in zip(need, owned))
    short = max(0, take - len(stack))
    bad = any(x < 0 for x in list(length) + list(new)) or any(n > ld for n in need)
    refused = bool(short or bad or row0[-1] > max_rows)
    out = dict(pos=np.zeros(max_rows, int), slot=np.full(max_rows, -1), seq=np.full(max_rows, -1),
               lim=np.zeros(max_rows, int), row0=np.zeros(B + 1, int), owned_out=np.array(owned), n_free_out=n_free,
               status=np.array([row0[-1], short, int(refused)]))
    if refused:
        return out
    for b in range(B):
        for p in range(int(owned[b]), need[b]):
            table[b, p] = stack.pop()
        out["owned_out"][b] = need[b] if need[b] >= owned[b] else keep[b]
    for i in range(n_free, len(stack)):
        free[i] = stack[i]
    out["n_free_out"], out["row0"] = len(stack), row0
    for b in range(B):
        for i in range(int(new[b])):
            r, p = row0[b] + i, int(length[b]) + i
            e = int(table[b, p // page])
            out["pos"][r], out["seq"][r], out["lim"][r] = p, b, length[b] + new[b]
            out["slot"][r] = e * page + p % page if 0 <= e < n_pages else -1
    return out


def turned(x, gain, eps, cs):
    """(rotated, error scale): RMSNorm and rotate-half of x [T, heads, D] in 64 bits, cs [T, D / 2, 2]."""
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    D = x.shape[-1]
    a, b, c, s = x[..., :D // 2], x[..., D // 2:], cs[:, None, :, 0], cs[:, None, :, 1]
    out = np.concatenate([a * c - b * s, b * c + a * s], -1)
    return out, np.concatenate([abs(a) + abs(b)] * 2, -1)


def gather(pool, table_row, n, page, v):
    """Positions [0, n) of one sequence as [n, kv_heads, D] (NaN where the table has no page)."""
    n_pages = pool.shape[0]
    D = pool.shape[2] if v else pool.shape[3]
    out = np.full((n, pool.shape[1], D), np.nan)
    for p in range(n):
        e = int(table_row[p // page])
        if 0 <= e < n_pages:
            out[p] = pool[e, :, :, p % page] if v else pool[e, :, p % page, :]
    return out


def attention(q, kp, vp, table, row0, length, lim, shared, page, scale, dtype):
    """{row: (out [H, D], bound [H, D])}: attention in 64 bits and how far a kernel that keeps fp32 scores and sums and
    rounds the probabilities and the output to `dtype` may be off.

    A score's error: D products in an fp32 chain, D * 2^-24 * sum |q k|, and four roundings of the scaled score and
    of the exponent (4 * 2^-24 * (|s| + 1)).  An error of d in every score moves the output by at most 2 d max|v|.
    Probabilities: half a step of dtype relative, and half of fp16's smallest step (2^-25) absolute.  Sums over n keys:
    n * 2^-24 * max|v|, for numerator and denominator."""
    H, D = q.shape[1:]
    G = H // kp.shape[1]
    half = EPS[dtype] / 2
    res = {}
    for b in range(len(row0) - 1):
        n = int(length[b])
        row_t = np.where(np.arange(table.shape[1]) < shared // page, table[0], table[b])
        K, V = gather(kp, row_t, n, page, False), gather(vp, row_t, n, page, True)
        for r in range(int(row0[b]), int(row0[b + 1])):
            e = n if lim is None else max(0, min(n, int(lim[r])))
            out, bound = np.zeros((H, D)), np.zeros((H, D))
            for h in range(H):
                k, v = K[:e, h // G], V[:e, h // G]
                there = ~np.isnan(k).any(-1) & ~np.isnan(v).any(-1)
                k, v = k[there], v[there]
                if len(k) == 0:
                    continue
                s = k @ q[r, h] * scale
                d = (D * abs(k * q[r, h]).sum(-1) * abs(scale) + 4 * (abs(s) + 1)).max() * 2.0 ** -24
                p = np.exp(s - s.max())
                out[h] = p @ v / p.sum()
                top = abs(v).max()
                prob = half * (p @ abs(v)) / p.sum() + (len(k) * 2.0 ** -25 * top / p.sum() if dtype == "f16" else 0)
                bound[h] = 2 * d * top + prob + 2 * len(k) * 2.0 ** -24 * top + half * abs(out[h])
            res[r] = (out, bound)
    return res


def select(x, V, mask_id, row0, hist, hist0, n_prompt, rep, pres, freq, bias_id, bias, bias0, allow, allow_row):
    """(adjusted logits in fp32 with each operation rounded once, ids, confidences in 64 bits)."""
    f = np.float32
    x = x.astype(f).copy()
    ids, conf = np.full(len(x), -1), np.zeros(len(x))
    with np.errstate(invalid="ignore", over="ignore"):
        for b in range(len(row0) - 1):
            seen, made = np.zeros(V, bool), np.zeros(V, np.int64)
            if hist is not None:
                for i in range(hist0[b], hist0[b + 1]):
                    if 0 <= hist[i] < V:
                        seen[hist[i]] = True
                        made[hist[i]] += i - hist0[b] >= (0 if n_prompt is None else n_prompt[b])
            d = {}
            if bias is not None:
                d = {int(bias_id[i]): f(bias[i]) for i in range(bias0[b], bias0[b + 1]) if 0 <= bias_id[i] < V}
            for r in range(row0[b], row0[b + 1]):
                l = x[r]
                if rep is not None:
                    l = np.where(seen, np.where(l > 0, l / f(rep[b]), l * f(rep[b])), l).astype(f)
                if freq is not None:
                    l = (l - (f(freq[b]) * made.astype(f)).astype(f)).astype(f)
                if pres is not None:
                    l = np.where(made > 0, l - f(pres[b]), l).astype(f)
                for v, w in d.items():
                    l[v] = l[v] + w
                l = np.minimum(np.where(np.isnan(l), -np.inf, l), np.finfo(f).max).astype(f)
                if mask_id >= 0:
                    l[mask_id] = -np.inf
                if allow is not None and allow_row[r] != -1:
                    a = int(allow_row[r])
                    ok = np.zeros(V, bool)
                    if 0 <= a < len(allow):
                        w = allow[a].astype(np.uint32)
                        ok = (w[np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1 == 1
                    l = np.where(ok, l, -np.inf).astype(f)
                x[r] = l
                if l.max() > -np.inf:
                    ids[r] = int(np.argmax(l))
                    conf[r] = 1.0 / np.exp(l.astype(np.float64) - float(l.max())).sum()
    return x, ids, conf
