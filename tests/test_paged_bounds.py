"""What the bounds of the paged attention's tests let through: answers planted on the CPU, right ones and wrong ones."""
import math

import pytest
import torch

import _paged as plain
import _paged_bounds as bounds

BF16 = torch.bfloat16


def rounded(c, want, before, decay):
    """The right answer in the outputs' type: (O, lse, accounts)."""
    S, H = c.S, c.H
    some = next(e for heads in want for e in heads if e is not None)
    g, d = some["O"].shape
    O, lse = torch.zeros((S, H * g, d)), torch.full((S, H * g), -math.inf)
    mass = torch.full((S, H, c.rows), math.nan)
    for s, heads in enumerate(want):
        for h, e in enumerate(heads):
            if e is not None:
                O[s, h * g:(h + 1) * g], lse[s, h * g:(h + 1) * g] = e["O"].float(), e["lse"].float()
                old = 0.0 if before is None else decay * before[s, h, :c.lens[s]].double()
                mass[s, h, :c.lens[s]] = (old + e["w"]).float()
    return O, lse, mass


@pytest.mark.parametrize("accounts", ["none", "rand"])
@pytest.mark.parametrize("n,d,H,g", [(40000, 64, 1, 1), (9000, 64, 1, 5), (20011, 128, 1, 2), (33, 64, 2, 3)])
def test_a_row_left_out_or_counted_twice_shows(n, d, H, g, accounts):
    c = plain.Cache([n, 0, 17], H, d, 64, BF16, seed=n)
    Q = torch.randn((3, H * g, d), generator=c.gen).to(BF16)
    before = torch.rand((3, H, c.rows), generator=c.gen) if accounts == "rand" else None
    want = bounds.attend(c, Q)
    O, lse, mass = rounded(c, want, before, 0.75)
    assert bounds.check_outputs(O, lse, want) is None
    assert bounds.check_accounts(mass, before, 0.75, want, c.lens) is None
    w = want[0][0]["w"]
    # beside an old account of up to 1 a weight of less than a step of it cannot be seen
    floor = 0.0 if before is None else 2.0 ** -21
    seen = {}
    for name, off in (("missing", -1.0), ("doubled", 1.0), ("a fifth off", 0.2)):
        tried = found = 0
        for r in sorted({x for b in (0, 16, 32, 1024, 4096, 8192, n - n % 32, n - 1) for x in (b - 1, b, b + 1) if 0 <= x < n}):
            if abs(off) * float(w[r]) <= floor:
                continue
            bad = mass.clone()
            bad[0, 0, r] = (0.0 if before is None else 0.75 * float(before[0, 0, r])) + (1.0 + off) * float(w[r])
            tried += 1
            found += bounds.check_accounts(bad, before, 0.75, want, c.lens) is not None
        assert tried >= 4 and found == tried, (name, tried, found)


def emulated(c, Q, scale, parts):
    """O of one_hot's data with each weight as the sum of `parts` bf16 numbers (0: as it is), the rest in 64 bits."""
    S, Hq, d = Q.shape
    g = Hq // c.H
    O = torch.zeros((S, Hq, d))
    for s, n in enumerate(c.lens):
        for h in range(c.H):
            k, v, q = c.head(c.K, s, h, n), c.head(c.V, s, h, n), Q[s, h * g:(h + 1) * g].double()
            p = torch.exp(q @ k.T * scale).float()
            held, rest = p.double(), p
            if parts:
                held = torch.zeros_like(p, dtype=torch.float64)
                for _ in range(parts):
                    held += rest.bfloat16().double()
                    rest = rest - rest.bfloat16().float()
            O[s, h * g:(h + 1) * g] = (held @ v / p.double().sum(1, keepdim=True)).float()
    return O


@pytest.mark.parametrize("lens,d,g", [([2, 5, 20, 33], 64, 1), ([64, 200, 640, 1000], 128, 4), ([70001], 128, 1), ([3000, 41], 64, 17)])
def test_weights_in_too_few_bits_show(lens, d, g):
    c = plain.Cache(lens, 1, d, 64, BF16, seed=1)
    scale = bounds.telling_scale()
    Q = bounds.one_hot(c, g)
    for s, n in enumerate(lens):
        # one sequence at a time, so that each is seen to tell
        want = bounds.attend(c, Q, scale, exact=True)
        only = lambda O: bounds.check_outputs(O[s:s + 1], None, want[s:s + 1])
        assert only(emulated(c, Q, scale, 0)) is None
        assert only(emulated(c, Q, scale, 3)) is None
        assert only(emulated(c, Q, scale, 2)) is not None, n
        assert only(emulated(c, Q, scale, 1)) is not None, n
