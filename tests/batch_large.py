"""Calls of the batch operators that are large enough for the launches that small ones do not get: the shared prefix as a part of
its own, 32 x 32 tiles, selections of more than a chip's workgroups, several heads a lane group.

Each case names the launch that it is there for; the CPU tests hold the launch rules to it, the GPU tests run it."""
import dataclasses

import numpy as np

from batch_util import EPS, tdtype

LEAD, TAIL = 3, 5          # rows before the first sequence's and behind the last one's


@dataclasses.dataclass(frozen=True)
class Attn:
    name: str
    dtypes: tuple
    rows: tuple             # of each sequence
    own: tuple              # positions behind the prefix (negative: the sequence ends inside it)
    H: int
    Hk: int
    D: int
    page: int
    prefix: int
    tile: int               # rows of a workgroup
    shared: bool            # the prefix is a part of its own

    @property
    def lens(self):
        return [self.prefix + n for n in self.own]

    def plan_args(self, dtype):
        """(dtype code, n_rows, n_seqs, n_heads, n_kv_heads, head_dim, page, table_ld, shared_len, max_rows, max_len)"""
        return ({"f32": 0, "bf16": 1, "f16": 4}[dtype], LEAD + sum(self.rows) + TAIL, len(self.rows), self.H, self.Hk, self.D,
                self.page, self.table_ld, self.prefix, max(self.rows), max(self.lens))

    @property
    def table_ld(self):
        return max(-(-max(self.lens) // self.page), self.prefix // self.page) + 1


def ragged(n, most, seed):
    """Own positions of n sequences: one that ends inside the prefix, one that ends with it, the others ragged."""
    r = np.random.default_rng(seed).integers(1, most, n)
    r[1 % n], r[2 % n], r[-1] = -133, 0, most
    return tuple(int(x) for x in r)


H16, F32, ALL = ("f16", "bf16"), ("f32",), ("f32", "f16", "bf16")
ATTN = [
    Attn("16 rows", H16, (1, 1, 0, 1, 1, 1, 1, 1, 1), ragged(9, 300, 0), 1, 1, 128, 32, 2048, 16, True),
    Attn("16 rows, D 64", H16, (2, 1, 0, 1), ragged(4, 90, 1), 2, 2, 64, 64, 5504, 16, True),
    Attn("32 rows", H16, (1,) * 5 + (0,) + (1,) * 6, ragged(12, 200, 2), 1, 1, 128, 32, 1504, 32, True),
    Attn("32 rows, D 64", H16, (4, 0, 2, 3, 5), ragged(5, 400, 3), 1, 1, 64, 256, 8448, 32, True),
    Attn("64 rows", H16, (5, 32, 0, 17, 1, 33, 40, 2, 64), ragged(9, 333, 4), 4, 2, 128, 64, 1024, 64, True),
    Attn("64 rows, odd group", H16, (3,) * 7 + (9, 0, 20), ragged(10, 150, 5), 7, 1, 128, 32, 1856, 64, True),
    Attn("64 rows, D 64", H16, (8, 30, 1, 0, 16), ragged(5, 700, 6), 16, 8, 64, 128, 1024, 64, True),
    Attn("128 rows", H16, (20, 20, 0, 7) + (20,) * 15, ragged(19, 1500, 7), 28, 4, 128, 64, 4096, 128, True),
    Attn("128 rows, D 64", H16, (64, 64, 0, 5) + (64,) * 13, ragged(17, 900, 8), 16, 8, 64, 32, 2304, 128, True),
    Attn("128 rows, own keys", H16, (600, 333), (1400, 1111), 32, 8, 128, 32, 0, 128, False),
    Attn("128 rows, own keys, D 64", H16, (1101, 500), (1500, 1333), 16, 8, 64, 128, 0, 128, False),
    Attn("prompt rows", ALL, (700, 0, 511), (900, 40, 511), 4, 2, 128, 64, 0, 64, False),
    Attn("fp32, 16 rows", F32, (1, 1, 0, 1, 5), ragged(5, 300, 9), 3, 1, 128, 32, 2048, 16, True),
    Attn("fp32, 32 rows", F32, (9, 32, 0, 5), ragged(4, 200, 10), 2, 2, 64, 64, 2752, 32, True),
    Attn("fp32, 64 rows", F32, (9, 12, 0, 16, 1), ragged(5, 500, 11), 28, 4, 128, 64, 1024, 64, True),
    Attn("fp32, D 32", F32, (9, 70, 0, 33, 1), ragged(5, 100, 12), 4, 4, 32, 256, 2304, 64, True),
]


# Calls with a shared part for the infinities in V: type, rows, lengths, heads, K/V heads, head_dim, prefix, tile
ODD = [("f16", (2, 1, 3), (4200, 4150, 4111), 2, 2, 128, 4096, 16), ("bf16", (4, 3, 4, 2, 4), (4200, 4150, 3000, 4097, 4300), 1, 1, 128, 4096, 32),
       ("f16", (20, 9, 30), (4200, 4150, 4000), 4, 2, 128, 4096, 64), ("bf16", (20, 9, 30), (4200, 4150, 4099), 8, 4, 64, 4096, 64),
       ("f32", (20, 9), (4200, 3900), 4, 2, 128, 4096, 64), ("f32", (9, 5), (4200, 4120), 4, 4, 64, 4096, 16)]


def odd_plan_args(dtype, rows, lens, H, Hk, D, prefix):
    ld = max(-(-max(lens) // 32), prefix // 32) + 1
    return ({"f32": 0, "bf16": 1, "f16": 4}[dtype], sum(rows) + 2, len(rows), H, Hk, D, 32, ld, prefix, max(rows), max(lens))


def attn_inputs(c, dtype, seed, junk):
    """q, pages, tables and row bounds on the GPU.  junk: what stands where no sequence has a position."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt, B, sp = tdtype(dtype), len(c.rows), c.prefix // c.page
    counts = [max(-(-n // c.page), 0) for n in c.lens]
    n_pages = sp + sum(max(0, k - sp) for k in counts) + 2
    perm = rng.permutation(n_pages)
    table, at = np.full((B, c.table_ld), -1), sp
    table[:, :sp] = perm[:sp]
    for b in range(B):
        for p in range(sp, counts[b]):
            table[b, p] = perm[at]
            at += 1
    mk = lambda std, *s: torch.empty(s, device="cuda").normal_(0.0, std, generator=g).to(dt)  # noqa: E731
    R = LEAD + sum(c.rows) + TAIL
    q, k, v = mk(2.0, R, c.H, c.D), mk(1.0, n_pages, c.Hk, c.page, c.D), mk(1.0, n_pages, c.Hk, c.D, c.page)
    used = np.zeros((n_pages, c.page), bool)
    for b in range(B):
        for p in range(0, max(c.lens[b], c.prefix if b == 0 else 0), c.page):
            used[table[b, p // c.page], :max(0, max(c.lens[b], c.prefix) - p)] = True
    hole = torch.from_numpy(~used).cuda()
    k.masked_fill_(hole[:, None, :, None], junk)
    v.masked_fill_(hole[:, None, None, :], junk)
    return dict(q=q, k=k, v=v, table=table, row0=LEAD + np.concatenate([[0], np.cumsum(c.rows)]), lens=np.array(c.lens))


def limits(c):
    """Causal limits, with rows that see nothing, that end inside the prefix, and with limits past the length."""
    lim = np.concatenate([[9] * LEAD] + [np.arange(n - w + 1, n + 1) for w, n in zip(c.rows, c.lens)] + [[9] * TAIL])
    first = LEAD
    for i, n in enumerate((0, -5, 1, 63, 64, 10 ** 6, c.prefix - 7, c.prefix, c.prefix + 1)):
        at = first + 2 * i
        if at < len(lim) - TAIL:
            lim[at] = n
    return lim


def attn_reference(c, x, dtype, lim):
    """{row: (out, bound)} as batch_util.attention gives it (the bound is derived there), in 64 bits on the GPU."""
    import torch
    f = torch.float64
    half, scale, res, G = EPS[dtype] / 2, c.D ** -0.5, {}, c.H // c.Hk
    n_pages, sp = x["k"].shape[0], c.prefix // c.page
    for b in range(len(c.rows)):
        a, e, n = int(x["row0"][b]), int(x["row0"][b + 1]), int(x["lens"][b])
        if a == e:
            continue
        if n <= 0:
            res.update({r: (np.zeros((c.H, c.D)), np.zeros((c.H, c.D))) for r in range(a, e)})
            continue
        pages = -(-n // c.page)
        ids = np.where(np.arange(pages) < sp, x["table"][0, :pages], x["table"][b, :pages])
        there = torch.from_numpy(np.repeat((ids >= 0) & (ids < n_pages), c.page)[:n]).cuda()
        ids = torch.from_numpy(np.where((ids >= 0) & (ids < n_pages), ids, 0)).cuda()
        K = x["k"][ids].to(f).permute(1, 0, 2, 3).reshape(c.Hk, -1, c.D)[:, :n]
        V = x["v"][ids].to(f).permute(1, 0, 3, 2).reshape(c.Hk, -1, c.D)[:, :n]
        K, V = (torch.where(there[None, :, None], t, 0.0).contiguous() for t in (K, V))
        q = x["q"][a:e].to(f).view(e - a, c.Hk, G, c.D).permute(1, 0, 2, 3).reshape(c.Hk, -1, c.D).contiguous()
        KT = K.transpose(1, 2).contiguous()
        s = torch.bmm(q, KT) * scale
        top_n = torch.full((e - a,), n, device="cuda") if lim is None else torch.from_numpy(np.minimum(lim[a:e], n)).cuda()
        sees = (torch.arange(n, device="cuda")[None, :] < top_n[:, None]) & there[None, :]
        sees = sees.repeat_interleave(G, 0)[None]                                   # [1, w * G, n]
        d = torch.where(sees, c.D * torch.bmm(q.abs(), KT.abs()) * scale + 4 * (s.abs() + 1), 0.0).amax(-1) * 2.0 ** -24
        s = torch.where(sees, s, -float("inf"))
        m = s.amax(-1, keepdim=True)
        p = torch.where(sees, torch.exp(s - torch.where(m > -float("inf"), m, 0.0)), 0.0)
        den, count = p.sum(-1, keepdim=True), sees.sum(-1)[..., None].to(f)
        some = den > 0
        den = torch.where(some, den, 1.0)
        out = torch.bmm(p, V) / den
        top = torch.stack([torch.where(sees[0].T[:, :, None], V[h].abs()[:, None, :].amax(-1, keepdim=True), 0.0).amax(0) for h in range(c.Hk)])
        prob = half * torch.bmm(p, V.abs()) / den + (count * 2.0 ** -25 * top / den if dtype == "f16" else 0.0)
        bound = 2 * d[..., None] * top + prob + 2 * count * 2.0 ** -24 * top + half * out.abs()
        shape = lambda t: torch.where(some, t, 0.0).view(c.Hk, e - a, G, c.D).permute(1, 0, 2, 3).reshape(e - a, c.H, c.D)  # noqa: E731
        out, bound = shape(out).cpu().numpy(), shape(bound).cpu().numpy()
        for r in range(a, e):
            res[r] = (out[r - a], bound[r - a])
    return res


# rows of each sequence, vocabulary, longest history, biases, masks; rows of a workgroup, whether all fit at four waves a SIMD
SELECT = [
    ((700, 0, 301, 450), 4099, 900, 30, 3, 4, False),
    ((1000, 900, 1, 0, 931), 4099, 500, 9, 2, 8, False),
    ((2000, 17, 1900, 1633), 4100, 300, 60, 5, 16, False),
    ((250, 6, 400, 40), 4097, 200, 20, 2, 4, True),
]

# rows, heads, K/V heads, head_dim, page; heads of a lane group
QK = [(4100, 28, 4, 128, 64, 8), (4200, 7, 1, 64, 32, 2), (8200, 5, 1, 32, 128, 3), (2050, 33, 11, 128, 32, 5)]
