"""Plain 64-bit forms of the paged cache's operators, and caches to try them on: sequences scattered over shuffled pages, rows and
pages nobody owns filled with NaN, table entries nobody reads filled with nonsense."""
import math

import numpy as np
import torch


class Cache:
    """A cache on the host: K, V [pages, H, page, d] in the cache's type, table, len; dev() puts it on the GPU."""

    def __init__(self, lens, H, d, page, dtype, seed, per_seq=None, key=1.0, spare=2):
        gen = torch.Generator().manual_seed(seed)
        S = len(lens)
        used = [-(-max(n, 0) // page) for n in lens]
        self.per_seq = max(max(used), 1) if per_seq is None else per_seq
        pages = sum(used) + spare
        order = torch.randperm(pages, generator=gen)
        self.table = torch.full((S, self.per_seq), -77, dtype=torch.int32)
        self.table[:, 1::2] = 2_000_000_000
        self.K = torch.full((pages, H, page, d), math.nan, dtype=dtype)
        self.V = torch.full((pages, H, page, d), math.nan, dtype=dtype)
        at = 0
        for s, n in enumerate(lens):
            for i in range(used[s]):
                p = int(order[at])
                at += 1
                self.table[s, i] = p
                rows = min(page, n - i * page)
                self.K[p, :, :rows] = (key * torch.randn((H, rows, d), generator=gen)).to(dtype)
                self.V[p, :, :rows] = torch.randn((H, rows, d), generator=gen).to(dtype)
        self.len = torch.tensor(lens, dtype=torch.int32)
        self.lens, self.H, self.d, self.page, self.dtype, self.S = list(lens), H, d, page, dtype, S
        self.rows = self.per_seq * page
        self.gen = gen

    def dev(self, ws):
        return ws.PagedCache(self.K.cuda(), self.V.cuda(), self.table.cuda(), self.len.cuda())

    def head(self, pool, s, h, n):
        """Rows 0..n-1 of head h of sequence s, in 64 bits."""
        r = torch.arange(n)
        return pool[self.table[s].long()[r // self.page], h, r % self.page].double()


def attend(c, Q, scale=0.0, lens=None, K=None, V=None):
    """(O, lse, weights, size, dz): `weights` [S][H] -> [n] summed over the head's queries, `size` [S,Hq,d] = sum_r p |V|, and dz
    [S,Hq], a bound of the error of a logit formed in 32 bits."""
    K, V = c.K if K is None else K, c.V if V is None else V
    S, Hq, d = Q.shape
    g = Hq // c.H
    scale = scale if scale > 0 else d ** -0.5
    O = torch.zeros((S, Hq, d), dtype=torch.float64)
    size = torch.zeros_like(O)
    lse = torch.full((S, Hq), -math.inf, dtype=torch.float64)
    dz = torch.zeros((S, Hq), dtype=torch.float64)
    weights = [[None] * c.H for _ in range(S)]
    for s, n in enumerate(c.lens if lens is None else lens):
        if n == 0:
            continue
        for h in range(c.H):
            k, v, q = c.head(K, s, h, n), c.head(V, s, h, n), Q[s, h * g:(h + 1) * g].double()
            z = q @ k.T * scale
            p = torch.softmax(z, dim=1)
            O[s, h * g:(h + 1) * g] = p @ v
            size[s, h * g:(h + 1) * g] = p @ v.abs()
            lse[s, h * g:(h + 1) * g] = torch.logsumexp(z, dim=1)
            # d products added in fp32 in any order, the product with the scale, and the difference to the maximum
            big = (q.abs() @ k.abs().T * scale).amax(dim=1)
            dz[s, h * g:(h + 1) * g] = (d + 4) * 2.0 ** -24 * big
            weights[s][h] = p.sum(dim=0)
    return O, lse, weights, size, dz


def check_attention(O, lse, want, n_max):
    """O and lse against attend()'s answer.  A weight is off by a factor exp(2 dz) (its logit and the sum's) and 2^-20 for the
    exponential; as operand of the second product it has at least 16 bits, 2^-17; n_max terms are added in fp32, 2^-24 each at
    the very worst, in runs of at most 4096 before they are joined (runs are shorter wherever n_max is longer than that)."""
    ref, ref_lse, _, size, dz = want
    rel = 2 * dz + 2.0 ** -20 + 2.0 ** -17 + min(n_max, 4096) * 2.0 ** -24
    err = (O.double().cpu() - ref).abs()
    assert torch.isfinite(O).all()
    assert (err <= rel[:, :, None] * size + 1e-37).all(), float((err / (size + 1e-37)).max())
    if lse is not None:
        lse = lse.double().cpu()
        empty = torch.isinf(ref_lse)
        assert torch.equal(torch.isneginf(lse), empty)
        bound = dz + 2.0 ** -20 + min(n_max, 4096) * 2.0 ** -24 + ref_lse.abs().masked_fill(empty, 0.0) * 2.0 ** -22
        assert ((lse - ref_lse).abs().masked_fill(empty, 0.0) <= bound).all()
    assert (O.cpu()[torch.isinf(ref_lse)] == 0).all()


def check_weights(mass, before, decay, want, lens, n_max):
    """mass [S,H,rows] against decay * before + weights; rows behind the last one as they were (NaN planted there)."""
    _, _, weights, _, dz = want
    mass = mass.cpu().double()
    g = dz.shape[1] // len(weights[0])
    for s, n in enumerate(lens):
        assert torch.isnan(mass[s, :, n:]).all()
        for h in range(len(weights[s])):
            if n == 0:
                continue
            old = 0.0 if before is None else decay * before[s, h, :n].double()
            # every weight: its logit, the sum's, the exponential, the sum of g of them and of the account
            rel = 2 * float(dz[s, h * g:(h + 1) * g].max()) + 2.0 ** -20 + (g + 2 + min(n_max, 4096)) * 2.0 ** -24
            ref = old + weights[s][h]
            # logits are kept in units of log2: their size times 2^-24 comes to the exponent as well, for the largest of them
            assert ((mass[s, h, :n] - ref).abs() <= rel * ref + 1e-36).all(), (s, h, float(((mass[s, h, :n] - ref).abs() / (ref + 1e-36)).max()), rel)


def evict(n, keep, sinks, recent, seen, mass, stamp):
    """(came, moves) of one head: the row each row below min(n, keep) was before, and how many moved."""
    if n <= keep:
        return list(range(n)), 0
    def order(r):
        guarded = stamp[r] < sinks or stamp[r] >= seen - recent
        m = float(mass[r])
        # a NaN is less than every number, -infinity included
        return (0, 0.0, r) if guarded else (2, 0.0, r) if math.isnan(m) else (1, -m, r)
    stays = sorted(sorted(range(n), key=order)[:keep])
    movers = [r for r in stays if r >= keep]
    there = set(stays)
    came = list(range(keep))
    free = [r for r in range(keep) if r not in there]
    assert len(free) == len(movers)
    for to, src in zip(free, movers):
        came[to] = src
    return came, len(free)


def rotate(x, pos, pairs, base):
    """x [T, heads, d] (64-bit) turned by its positions, pos [axes, T]."""
    d = x.shape[2]
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    c = np.arange(d // 2)
    ang = torch.from_numpy(pos.numpy().astype(np.float64)[axis].T * float(base) ** (-2.0 * c / d))[:, None]
    a, b = x[:, :, :d // 2], x[:, :, d // 2:]
    return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], dim=2)
