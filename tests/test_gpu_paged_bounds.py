"""The paged attention against bounds that see a row left out or counted twice, and a weight held in too few bits, on every path: a
workgroup per head, equal runs with joins, and the accounts' pass over 1024 rows at a time."""
import math

import numpy as np
import pytest
import torch

import _paged as plain
import _paged_bounds as bounds

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ws():
    from paper_2601_01298_amd import binding
    binding.lib()
    return binding


def check(ws, c, Q, scale=0.0, exact=False, accounts=("none", "rand")):
    """Attention with and without accounts; `before` none, or old ones in [0, 1)."""
    want = bounds.attend(c, Q, scale, exact)
    cache, Qd = c.dev(ws), Q.cuda()
    lse = torch.full(Q.shape[:2], 7.0, device="cuda")
    O = ws.ws_synapse_paged_attend(cache, Qd, scale=scale, lse=lse)
    assert bounds.check_outputs(O, lse, want) is None
    for how in accounts:
        old = torch.rand((c.S, c.H, c.rows), generator=c.gen) if how == "rand" else None
        out = torch.full((c.S, c.H, c.rows), math.nan, device="cuda")
        lse.fill_(7.0)
        O = ws.ws_synapse_paged_attend(cache, Qd, scale=scale, lse=lse, decay=0.75, mass_in=None if old is None else old.cuda(), mass_out=out)
        assert bounds.check_outputs(O, lse, want) is None, how
        assert bounds.check_accounts(out, old, 0.75, want, c.lens) is None, how


def random(ws, lens, H, g, d, page, dtype, seed, per_seq=None, **kw):
    c = plain.Cache(lens, H, d, page, dtype, seed, per_seq)
    check(ws, c, torch.randn((c.S, H * g, d), generator=c.gen).to(dtype), **kw)


@pytest.mark.parametrize("dtype,d,n,H,g", [(BF16, 128, 70001, 1, 4), (BF16, 64, 40000, 2, 1), (F32, 128, 20011, 1, 2), (F32, 64, 9000, 3, 5)])
def test_long_sequences(ws, dtype, d, n, H, g):
    random(ws, [n], H, g, d, 64, dtype, n)
    random(ws, [17, n // 2, 3, n], H, g, d, 128, dtype, n + 1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_every_length_round_the_tiles(ws, dtype, d):
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 511]
    random(ws, lens, 2, 3, d, 32, dtype, d)                          # a workgroup per head
    random(ws, lens + [1023, 1024, 1025, 2049], 2, 3, d, 16, dtype, d)   # equal runs
    random(ws, lens, 1, 1, d, 256, dtype, d, per_seq=25)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_wide_tables(ws, dtype):
    random(ws, [700, 0, 1, 3000], 3, 2, 64, 256, dtype, 11, per_seq=80)
    random(ws, [5], 2, 1, 128, 256, dtype, 11, per_seq=512)
    random(ws, [1500] * 40, 8, 1, 64, 64, dtype, 12, per_seq=256)


@pytest.mark.parametrize("S", [65, 200, 1500])
def test_many_sequences(ws, S):
    rng = np.random.default_rng(S)
    lens = [int(n) for n in np.exp(rng.uniform(0, math.log(400), S)).astype(int)]
    lens[S // 2] = 0
    random(ws, lens, 1, 3, 64, 16, BF16, S, per_seq=400)
    random(ws, lens, 1, 3, 64, 16, BF16, S)


@pytest.mark.parametrize("dtype,g", [(BF16, 17), (BF16, 64), (F32, 33), (BF16, 261)])
def test_many_query_heads(ws, dtype, g):
    random(ws, [70, 0, 300, 1, 129], 2, g, 64, 64, dtype, g)
    random(ws, [1100, 5], 1, g, 128, 16, dtype, g)


@pytest.mark.parametrize("dtype,d,g,S", [(BF16, 64, 1, 70), (BF16, 128, 4, 70), (F32, 64, 3, 70), (BF16, 128, 1, 70)])
def test_as_many_heads_as_fill_the_chip(ws, dtype, d, g, S):
    rng = np.random.default_rng(g)
    random(ws, [int(n) for n in rng.integers(0, 1217, S - 1)] + [1216], 8, g, d, 32, dtype, g)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,d,g,per_seq", [([2, 5, 20, 33], 64, 1, None), ([2, 5, 20, 33], 64, 3, 25), ([64, 200, 640, 1000], 128, 4, None),
                                              ([64, 200, 500], 128, 1, None), ([70001], 128, 1, None), ([3000, 41], 64, 17, None)])
def test_weights_keep_all_their_bits(ws, dtype, lens, d, g, per_seq):
    """Exact logits, one weight to an output: a weight in two bf16 numbers would be 2^-17 off, more than the bound."""
    c = plain.Cache(lens, 1, d, 64, dtype, seed=1, per_seq=per_seq)
    check(ws, c, bounds.one_hot(c, g), bounds.telling_scale(), exact=True)
