"""Bounds of the paged attention's results row by row and sequence by sequence, from the roundings that the arithmetic cannot avoid:
fp32 logits, a hardware exponential, fp32 sums, nothing in fewer bits.  They know nothing of the other rows' or sequences' sizes,
so that a row left out, counted twice, or a weight held in too few bits shows.

With eps = 2^-24 (half a step of fp32):
  logit        d products added in any order, the scale (three roundings: log2 e, its product with the scale, 1/sqrt(d) twice rounded)
               and the product with it, and the difference in the exponent: (d + 7) eps sum |q k| scale; where all products and sums
               are exact, 7 eps |z|
  exponential  2^-22 of itself (the hardware's is good to a step, 2^-23)
  sum of weights   its longest chain of additions, see chain()
  log of it    2^-22 (hardware), the sum with the maximum eps |lse| / ln 2
  output       sum p V: additions one after the other in a wave, matrix instructions in any order, three parts of a weight: 3 a row
"""
import math

import torch

EPS = 2.0 ** -24
WHOLE = 2048           # no workgroup has more rows of a head than this where it has not an equal share of all rows


def chain(lens, H, g, bf16):
    """Per sequence: (additions one behind the other in the sum of its weights, additions of the product with V).  A workgroup takes
    ceil(T / groups) of all T tiles, four tiles at least, or all of a head of up to WHOLE rows; four waves share them, and four
    groups of lanes a tile.  Then the lanes, the waves, the workgroups: 2 + 4 + (at most 512 / 256 + 6 + 4); rescalings: 8.  The
    workgroups' parts of V are added by four waves."""
    tr = 32 if bf16 else 16
    tiles = [-(-n // tr) for n in lens]
    run = max(4, -(-sum(tiles) * H * (-(-g // 16)) // 256) + 1)
    out = []
    for n, t in zip(lens, tiles):
        wave = -(-min(t, max(run, -(-WHOLE // tr))) // 4) if n <= WHOLE else -(-min(t, run) // 4)
        parts = min(t, 512)
        out.append((wave * tr // 4 + 26, wave * tr * (3 if bf16 else 1) + 16 + parts // 4))
    return out


def attend(c, Q, scale=0.0, exact=False, lens=None):
    """64-bit answer with bounds: lists [S][H] of dicts O, dO [g,d]; lse, dlse [g]; w, dw [n] (None for an empty sequence)."""
    S, Hq, d = Q.shape
    g = Hq // c.H
    # the scale that reaches the library is a float
    scale = float(torch.tensor(scale, dtype=torch.float32)) if scale > 0 else d ** -0.5
    lens = c.lens if lens is None else lens
    chains = chain(lens, c.H, g, c.dtype is torch.bfloat16)
    out = [[None] * c.H for _ in range(S)]
    for s, n in enumerate(lens):
        if n == 0:
            continue
        cl, cv = chains[s]
        for h in range(c.H):
            k, v, q = c.head(c.K, s, h, n), c.head(c.V, s, h, n), Q[s, h * g:(h + 1) * g].double()
            z = q @ k.T * scale
            dz = 7 * EPS * z.abs() if exact else (d + 7) * EPS * (q.abs() @ k.abs().T * scale)
            p, lse = torch.softmax(z, dim=1), torch.logsumexp(z, dim=1)
            dsum = (p * dz).sum(1) + 2.0 ** -22 + cl * EPS                        # of the sum of weights, relative
            dlse = dsum + 2.0 ** -22 * (1 + math.log(n + 1)) + 2 * EPS * lse.abs()
            # where V is zero nothing is rounded: the additions that count are those of rows with something in them
            adds = torch.minimum(3.0 * (v != 0).sum(0) + 8, torch.tensor(float(cv)))
            dO = (p * dz) @ v.abs() + (p @ v.abs()) * (dsum[:, None] + 2.0 ** -22 + (adds + 4) * EPS)
            x = (z - lse[:, None]).abs()
            dw = (p * (dz + dlse[:, None] + 2.0 ** -22 + EPS * x)).sum(0) + g * EPS * p.sum(0)
            out[s][h] = dict(O=p @ v, dO=dO, lse=lse, dlse=dlse, w=p.sum(0), dw=dw)
    return out


def check_outputs(O, lse, want):
    """None, or what is wrong."""
    O, lse = O.double().cpu(), None if lse is None else lse.double().cpu()
    for s, heads in enumerate(want):
        for h, e in enumerate(heads):
            g = O.shape[1] // len(heads)
            got = O[s, h * g:(h + 1) * g]
            if e is None:
                if (got != 0).any() or (lse is not None and not torch.isneginf(lse[s, h * g:(h + 1) * g]).all()):
                    return f"sequence {s} has no rows"
                continue
            err = (got - e["O"]).abs()
            if not (err <= e["dO"] + 1e-36).all():
                return f"O of sequence {s} head {h}: {float((err / (e['dO'] + 1e-36)).max()):.3g} of its bound"
            if lse is not None and not ((lse[s, h * g:(h + 1) * g] - e["lse"]).abs() <= e["dlse"]).all():
                return f"lse of sequence {s} head {h}"
    return None


def check_accounts(mass, before, decay, want, lens):
    """None, or what is wrong with mass [S,H,rows] as decay * before + weights.  The old account adds its own roundings only: that of
    the decay to a float, and the sum's."""
    mass = mass.double().cpu()
    for s, n in enumerate(lens):
        if not torch.isnan(mass[s, :, n:]).all():
            return f"accounts behind the last row of sequence {s}"
        for h, e in enumerate(want[s]):
            if e is None:
                continue
            old = torch.zeros(n, dtype=torch.float64) if before is None else decay * before[s, h, :n].double()
            err = (mass[s, h, :n] - old - e["w"]).abs()
            bound = e["dw"] + 2 * EPS * (old + e["w"]) + 1e-36
            if not (err <= bound).all():
                r = int((err / bound).argmax())
                return f"account {r} of sequence {s} head {h}: {float(err[r] / bound[r]):.3g} of its bound"
    return None


# ---- data whose logits are exact and whose weights, if held in 8 or 16 bits, are all off the same way ------------------------------
def telling_scale():
    """A scale s for which e^-s, in (1/2, 1), is as far from the sum of two bf16 numbers as it can be: 2^-17 of itself, nearly."""
    s = torch.linspace(0.60, 0.693, 20001, dtype=torch.float32).double()
    p = torch.exp(-s).float()
    rest = p - p.bfloat16().float()
    rest = (rest - rest.bfloat16().float()).abs() / p
    i = int(rest.argmax())
    assert rest[i] > 0.9 * 2.0 ** -17
    return float(s[i])


def one_hot(c, g):
    """Fills the cache c: every fourth row's key is 0, the others' -1 in the first dimension; value row r_e has a one in dimension e and
    nothing else, r_e spread over the sequence.  With queries of a one in the first dimension the logits are 0 and -scale, every
    output is one row's weight, and nothing is added up but the sum of weights.  Returns Q."""
    for s, n in enumerate(c.lens):
        r = torch.arange(n)
        page, row = c.table[s].long()[r // c.page], r % c.page
        c.K[page, :, row] = 0.0
        c.V[page, :, row] = 0.0
        c.K[page, :, row, 0] = torch.where(r % 4 == 0, 0.0, -1.0).to(c.dtype)[:, None].expand(n, c.H)
        low = [x for x in range(n) if x % 4]
        for e in range(min(c.d, len(low))):
            x = low[e * (len(low) - 1) // max(1, min(c.d, len(low)) - 1)]
            c.V[c.table[s].long()[x // c.page], :, x % c.page, e] = 1.0
    Q = torch.zeros((c.S, c.H * g, c.d), dtype=c.dtype)
    Q[:, :, 0] = 1.0
    return Q
