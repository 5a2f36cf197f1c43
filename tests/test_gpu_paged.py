"""The paged cache's operators against plain 64-bit forms: append with rotary positions, attention of one new token, eviction by
attention weight, and a run of them together."""
import math

import numpy as np
import pytest
import torch

import _paged as plain

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ws():
    from paper_2601_01298_amd import binding
    binding.lib()
    return binding


def nan_like(shape):
    return torch.full(shape, math.nan)


# ---- attention ------------------------------------------------------------------------------------------------------------
EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 0, 63, 64, 65, 127, 128, 129, 255, 257, 511, 640, 1001]


def run_attend(ws, c, g, seed=0, qscale=1.0, scale=0.0, weights=True, decay=0.75, before="rand", lens=None):
    gen = torch.Generator().manual_seed(seed)
    lens = c.lens if lens is None else lens
    Q = (qscale * torch.randn((c.S, c.H * g, c.d), generator=gen)).to(c.dtype)
    want = plain.attend(c, Q, scale, lens)
    cache = c.dev(ws)
    lse = torch.full((c.S, c.H * g), 7.0, device="cuda")
    mass_out = mass_in = old = None
    if weights:
        mass_out = nan_like((c.S, c.H, c.rows)).cuda()
        if before == "rand":
            old = torch.rand((c.S, c.H, c.rows), generator=gen)
            mass_in = old.cuda()
        elif before == "same":
            old = torch.rand((c.S, c.H, c.rows), generator=gen)
            for s, n in enumerate(lens):
                old[s, :, n:] = math.nan
            mass_in = mass_out = old.cuda()
    O = ws.ws_synapse_paged_attend(cache, Q.cuda(), scale=scale, lse=lse, decay=decay, mass_in=mass_in, mass_out=mass_out)
    plain.check_attention(O, lse, want, max(lens))
    if weights:
        plain.check_weights(mass_out, old, decay, want, lens, max(lens))
    return O, lse, mass_out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("H,g", [(1, 1), (2, 3), (3, 8), (1, 16)])
def test_attend_at_the_edges_of_tiles_and_pages(ws, dtype, d, page, H, g):
    run_attend(ws, plain.Cache(EDGES, H, d, page, dtype, seed=d + page + g), g)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("g", [17, 32, 71])
def test_attend_with_many_query_heads(ws, dtype, g):
    run_attend(ws, plain.Cache([70, 0, 300, 1, 129], 2, 64, 64, dtype, seed=g), g)
    run_attend(ws, plain.Cache([70, 0, 300, 1, 129], 1, 128, 16, dtype, seed=g), g, weights=False)


def test_attend_with_hundreds_of_query_heads_per_key_head(ws):
    run_attend(ws, plain.Cache([70, 0, 600, 1], 1, 64, 64, BF16, seed=3), 261)


@pytest.mark.parametrize("dtype,d,g", [(BF16, 64, 1), (BF16, 128, 4), (F32, 64, 3)])
def test_attend_with_as_many_heads_as_fill_the_chip(ws, dtype, d, g):
    """512 and more (sequence, head) pairs whose logits fit LDS: a workgroup each, rows up to 1216."""
    rng = np.random.default_rng(g)
    lens = [int(n) for n in rng.integers(0, 1217, 69)] + [1216]
    run_attend(ws, plain.Cache(lens, 8, d, 32, dtype, seed=g), g)
    run_attend(ws, plain.Cache([3 * n for n in lens], 8, d, 32, dtype, seed=g), g, weights=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("before", ["rand", "none", "same"])
def test_attend_accounts(ws, dtype, before):
    for decay in (1.0, 0.0, 0.9):
        run_attend(ws, plain.Cache([300, 0, 41, 1000], 2, 64, 32, dtype, seed=5), 4, before=before, decay=decay)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("S", [1, 63, 64, 65, 200])
def test_attend_with_many_sequences(ws, dtype, S):
    rng = np.random.default_rng(S)
    lens = [int(n) for n in np.exp(rng.uniform(0, math.log(400), S)).astype(int)]
    lens[S // 2] = 0
    run_attend(ws, plain.Cache(lens, 2, 64, 16, dtype, seed=S), 2)
    # tables of 6400 rows: the rows of all sequences are shared out over the workgroups
    run_attend(ws, plain.Cache(lens, 2, 64, 16, dtype, seed=S, per_seq=400), 2)
    run_attend(ws, plain.Cache(lens, 1, 128, 256, dtype, seed=S, per_seq=25), 1, weights=False)


def test_attend_with_very_many_sequences(ws):
    rng = np.random.default_rng(7)
    lens = [int(n) for n in rng.integers(0, 90, 1500)]
    run_attend(ws, plain.Cache(lens, 1, 64, 16, BF16, seed=7, per_seq=400), 3)
    run_attend(ws, plain.Cache([0] * 1499 + [5000], 1, 64, 16, BF16, seed=7), 3)


@pytest.mark.parametrize("dtype,d,n,H,g", [(BF16, 128, 70001, 1, 4), (BF16, 64, 40000, 2, 1), (F32, 128, 20011, 1, 2), (F32, 64, 9000, 3, 5)])
def test_attend_over_long_sequences(ws, dtype, d, n, H, g):
    run_attend(ws, plain.Cache([n], H, d, 64, dtype, seed=n), g)
    run_attend(ws, plain.Cache([17, n // 2, 3, n], H, d, 128, dtype, seed=n), g)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attend_with_maxima_far_apart(ws, dtype):
    """Logits of hundreds; ones that rise all along the sequence, so that the maximum moves at every step; ones that fall."""
    for sign in (0, 1, -1):
        c = plain.Cache([900, 257, 5], 2, 64, 32, dtype, seed=3, key=4.0)
        gen = torch.Generator().manual_seed(1)
        Q = (6 * torch.randn((3, 4, 64), generator=gen)).to(dtype)
        if sign:
            Q[:, :, 0] = 8.0
            for s, n in enumerate(c.lens):
                r = torch.arange(n)
                c.K[c.table[s].long()[r // c.page], :, r % c.page, 0] = (sign * r / 3.0)[:, None].to(dtype)
        want = plain.attend(c, Q)
        lse = torch.empty((3, 4), device="cuda")
        mass = nan_like((3, 2, c.rows)).cuda()
        O = ws.ws_synapse_paged_attend(c.dev(ws), Q.cuda(), lse=lse, mass_out=mass)
        plain.check_attention(O, lse, want, 900)
        plain.check_weights(mass, None, 1.0, want, c.lens, 900)


def test_attend_scale_and_equal_rows(ws):
    run_attend(ws, plain.Cache([100, 33], 2, 64, 16, BF16, seed=1), 2, scale=0.3)
    c = plain.Cache([640], 1, 128, 32, BF16, seed=2)
    r = torch.arange(640)
    c.K[c.table[0].long()[r // 32], 0, r % 32] = 0.5
    O, lse, mass = run_attend(ws, c, 2, before="none")
    assert (mass[0, 0, :640] - 2.0 / 640).abs().max() <= 2.0 ** -16 * 2.0 / 640


@pytest.mark.parametrize("lens", [[300, 41], [3000, 2999]])
def test_attend_accounts_that_are_not_aligned(ws, lens):
    """Accounts that start at an odd multiple of four bytes: the same bits as aligned ones."""
    c = plain.Cache(lens, 2, 64, 16, BF16, seed=21)
    cache = c.dev(ws)
    Q = torch.randn((2, 6, 64), generator=c.gen).to(BF16).cuda()
    old = torch.rand((2, 2, c.rows), generator=c.gen).cuda()
    odd = lambda: torch.zeros(old.numel() + 1, device="cuda")[1:].view(old.shape)
    want, got, start = torch.zeros_like(old), odd(), odd()
    start.copy_(old)
    assert got.data_ptr() % 16 == 4
    ws.ws_synapse_paged_attend(cache, Q, decay=0.5, mass_in=old, mass_out=want)
    ws.ws_synapse_paged_attend(cache, Q, decay=0.5, mass_in=start, mass_out=got)
    assert torch.equal(got, want) and (want[0, :, :lens[0]] > 0).all()
    with pytest.raises(ws.WsError):
        ws.ws_synapse_paged_attend(cache, Q, O=torch.zeros(2 * 6 * 64 + 1, device="cuda")[1:].view(2, 6, 64))


def test_attend_lengths_and_pages_out_of_range(ws):
    """Lengths outside the table are clamped into it; a page number outside the pool reads as page 0."""
    c = plain.Cache([64, 64, 64], 2, 64, 16, BF16, seed=4)
    c.len = torch.tensor([-5, 1 << 30, 64], dtype=torch.int32)
    run_attend(ws, c, 2, lens=[0, 64, 64])
    c = plain.Cache([64, 50], 2, 64, 16, BF16, seed=4)
    c.K[0] = torch.randn(c.K[0].shape, generator=c.gen).to(BF16)
    c.V[0] = torch.randn(c.V[0].shape, generator=c.gen).to(BF16)
    bad = c.table.clone()
    c.table[0, 1], c.table[1, 3] = 0, 0
    want_table = c.table
    bad[0, 1], bad[1, 3] = c.K.shape[0], -1
    Q = torch.randn((2, 4, 64), generator=c.gen).to(BF16)
    want = plain.attend(c, Q)
    c.table = bad
    O = ws.ws_synapse_paged_attend(c.dev(ws), Q.cuda())
    c.table = want_table
    plain.check_attention(O, None, want, 64)


def test_attend_shared_pages(ws):
    """Sequences whose tables name the same pages: one prefix for all, and one page twice in a sequence."""
    c = plain.Cache([128, 128, 128], 2, 64, 16, BF16, seed=6)
    c.table[1, :4] = c.table[0, :4]
    c.table[2, :4] = c.table[0, :4]
    c.table[2, 5] = c.table[2, 4]
    run_attend(ws, c, 4)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attend_tables_with_room_for_far_more(ws, dtype):
    """Tables of 20 480 and of 131 072 rows of which a few are in use: the rows counted are those there are."""
    run_attend(ws, plain.Cache([700, 0, 1, 3000], 3, 64, 256, dtype, seed=11, per_seq=80), 2)
    run_attend(ws, plain.Cache([5], 2, 128, 256, dtype, seed=11, per_seq=512), 1)
    run_attend(ws, plain.Cache([1500] * 40, 8, 64, 64, dtype, seed=12, per_seq=2048), 1)


def test_attend_repeats_its_bits(ws):
    c = plain.Cache([5000, 17, 300, 0, 2222], 4, 128, 64, BF16, seed=8)
    a, b = run_attend(ws, c, 4), run_attend(ws, c, 4)
    for x, y in zip(a, b):
        assert torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0))


def test_attend_behind_4_gib(ws):
    """Pages whose rows lie more than 2^32 bytes into the pools."""
    H, d, page, pages = 8, 128, 256, 9000
    K = torch.empty((pages, H, page, d), dtype=BF16, device="cuda")
    V = torch.empty_like(K)
    assert K.nbytes > 2 ** 32
    c = plain.Cache([700], H, d, page, BF16, seed=9, spare=1)
    table = torch.tensor([[8999, 4097, 8998]], dtype=torch.int32)
    for i, p in enumerate(table[0].tolist()):
        K[p], V[p] = c.K[c.table[0, i]].cuda(), c.V[c.table[0, i]].cuda()
    Q = torch.randn((1, 2 * H, d), generator=c.gen).to(BF16)
    cache = ws.PagedCache(K, V, table.cuda(), c.len.cuda())
    O = ws.ws_synapse_paged_attend(cache, Q.cuda())
    plain.check_attention(O, None, plain.attend(c, Q), 700)
    # one more row, and an eviction, out there
    k, v = torch.randn((1, H, d), generator=c.gen).to(BF16), torch.randn((1, H, d), generator=c.gen).to(BF16)
    cache.len.add_(1)
    ws.ws_synapse_paged_append(cache, k.cuda(), v.cuda(), torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(K[8998, :, 700 - 512].cpu(), k[0]) and torch.equal(V[8998, :, 700 - 512].cpu(), v[0])
    mass = torch.arange(768, device="cuda", dtype=torch.float32).expand(1, H, 768).contiguous()
    stamp = torch.arange(768, device="cuda", dtype=torch.int32).expand(1, H, 768).contiguous()
    ws.ws_synapse_paged_evict(cache, 256, cache.len.clone(), mass, stamp)
    assert cache.len.item() == 256
    assert torch.equal(K[8999, :, 255].cpu(), k[0]) and torch.equal(V[8999, :, 255].cpu(), v[0])


# ---- append ---------------------------------------------------------------------------------------------------------------
def run_append(ws, dtype, d, H, g, page, lens, news, pairs, base=1e6, fused=False, padding=0, big=False, rotary=True, queries=True, accounts=True,
               in_place=False, seed=0):
    c = plain.Cache(lens, H, d, page, dtype, seed)
    gen, S, T, Hq = c.gen, len(lens), sum(news) + padding, H * g
    if fused:
        both = torch.randn((T, Hq + 2 * H, d), generator=gen).to(dtype).cuda()
        q, k, v = both[:, :Hq], both[:, Hq:Hq + H], both[:, Hq + H:]
    else:
        q, k, v = (torch.randn((T, n, d), generator=gen).to(dtype).cuda() for n in (Hq, H, H))
    axes = len(pairs)
    top = 2 ** 31 - 1 if big else 9000
    pos = torch.randint(-top - 1 if big else 0, top, (axes, T), generator=gen).to(torch.int32)
    if big:
        pos[:, 0] = -2 ** 31
    first = torch.tensor(np.concatenate([[0], np.cumsum(news)]).astype(np.int32))
    seen = (c.len + torch.randint(0, 100, (S,), generator=gen)).to(torch.int32)
    stamp, mass = torch.full((S, H, c.rows), -9, dtype=torch.int32), torch.full((S, H, c.rows), 3.5)
    cache = c.dev(ws)
    q_out = q if in_place else torch.full((T, Hq, d), 5.0, dtype=dtype, device="cuda")
    q_host, k_host, v_host = q.cpu(), k.cpu(), v.cpu()
    sd, md = stamp.cuda(), mass.cuda()
    kw = dict(pos=pos.cuda(), pairs=pairs, base=base) if rotary else {}
    if queries:
        kw.update(q=q, q_out=q_out)
    if accounts:
        kw.update(seen=seen.cuda(), stamp=sd, mass=md)
    ws.ws_synapse_paged_append(cache, k, v, first.cuda(), **kw)
    rk, rq = k_host.double(), q_host.double()
    if rotary:
        rk, rq = plain.rotate(rk, pos, pairs, base), plain.rotate(rq, pos, pairs, base)
    # one rounding to the type (half a step of the result), fp32 sines and products on rows of size sqrt(x0^2 + x1^2), and, at
    # positions of 2^31, their product with a frequency in float64: 2^31 * 2^-53 of a radian
    half = torch.finfo(dtype).eps / 2

    def near(got, want, rows):
        size = rows.abs().amax()
        return ((got.double() - want).abs() <= want.abs() * half * 1.01 + float(size) * (4 * 2.0 ** -23 + (2.0 ** -22 if big else 2.0 ** -34))).all()

    K, V = c.K.clone(), c.V.clone()
    Kd, Vd = cache.K.cpu(), cache.V.cpu()
    for s in range(S):
        for i in range(news[s]):
            t, row = int(first[s]) + i, lens[s] - news[s] + i
            p, r = int(c.table[s, row // page]), row % page
            if rotary:
                assert near(Kd[p, :, r], rk[t], k_host), (s, i)
            else:
                assert torch.equal(Kd[p, :, r], k_host[t])
            assert torch.equal(Vd[p, :, r], v_host[t])
            K[p, :, r], V[p, :, r] = Kd[p, :, r], Vd[p, :, r]
            if accounts:
                stamp[s, :, row] = int(seen[s]) - news[s] + i
                mass[s, :, row] = 0.0
    # everything else is as it was
    assert torch.equal(torch.nan_to_num(K.float(), 9e9), torch.nan_to_num(Kd.float(), 9e9))
    assert torch.equal(torch.nan_to_num(V.float(), 9e9), torch.nan_to_num(Vd.float(), 9e9))
    assert torch.equal(sd.cpu(), stamp) and torch.equal(md.cpu(), mass)
    if queries:
        n = sum(news)
        got = q_out.cpu()
        assert near(got[:n], rq[:n], q_host) if rotary else torch.equal(got[:n], q_host[:n])
        assert torch.equal(got[n:], q_host[n:] if in_place else torch.full_like(got[n:], 5.0))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("axes", [1, 2, 3, 4])
def test_append(ws, dtype, d, page, axes):
    half = d // 2
    pairs = [[half], [half - 7, 7], [8, 12, half - 20], [1, 0, half - 3, 2]][axes - 1]
    run_append(ws, dtype, d, 2, 3, page, [40, 1, 17, 300, 16], [40, 0, 1, 129, 16], pairs, seed=axes)
    run_append(ws, dtype, d, 3, 1, page, [40, 1, 17, 300, 16], [1, 1, 1, 1, 1], pairs, fused=True, seed=axes)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_variants(ws, dtype):
    one = dict(ws=ws, dtype=dtype, d=64, H=2, g=2, page=16, lens=[33, 5, 18], news=[3, 0, 18], pairs=[32])
    run_append(**one, padding=7)
    run_append(**one, padding=7, fused=True, rotary=False)
    run_append(**one, queries=False)
    run_append(**one, accounts=False)
    run_append(**one, in_place=True, padding=2)
    run_append(**one, big=True)
    run_append(**one, base=10000.0)
    run_append(**{**one, "d": 128, "pairs": [16, 24, 24], "g": 40, "H": 1}, big=True)


def test_append_many_sequences(ws):
    rng = np.random.default_rng(0)
    lens = [int(n) for n in rng.integers(1, 40, 300)]
    news = [int(rng.integers(0, n + 1)) for n in lens]
    run_append(ws, BF16, 64, 1, 2, 16, lens, news, [32])


def test_append_leaves_out_what_has_no_place(ws):
    """Rows before the first, rows behind the table, pages that do not exist: nothing is written, the queries still rotate."""
    c = plain.Cache([16, 16, 16, 16], 1, 64, 16, BF16, seed=1)
    c.len = torch.tensor([1, 18, 16, -3], dtype=torch.int32)          # two new rows each: rows -1 0 | 16 17 | bad page | -5 -4
    c.table[2, 0] = c.K.shape[0]
    k, v = (torch.randn((8, 1, 64), generator=c.gen).to(BF16).cuda() for _ in range(2))
    q = torch.randn((8, 2, 64), generator=c.gen).to(BF16).cuda()
    stamp = torch.full((4, 1, 16), -9, dtype=torch.int32, device="cuda")
    mass = torch.full((4, 1, 16), 2.0, device="cuda")
    cache = c.dev(ws)
    out = ws.ws_synapse_paged_append(cache, k, v, torch.tensor([0, 2, 4, 6, 8], dtype=torch.int32, device="cuda"), q=q,
                                     seen=cache.len.clone(), stamp=stamp, mass=mass)
    K, V = c.K.clone(), c.V.clone()
    K[c.table[0, 0], 0, 0], V[c.table[0, 0], 0, 0] = k[1, 0].cpu(), v[1, 0].cpu()
    assert torch.equal(cache.K.cpu().nan_to_num(9e9), K.nan_to_num(9e9)) and torch.equal(cache.V.cpu().nan_to_num(9e9), V.nan_to_num(9e9))
    assert torch.equal(out, q)
    assert stamp[0, 0, 0].item() == 0 and mass[0, 0, 0].item() == 0 and int((stamp == -9).sum()) == 63 and int((mass == 2.0).sum()) == 63


# ---- eviction -------------------------------------------------------------------------------------------------------------
def run_evict(ws, lens, H, d, page, dtype, keep, sinks=0, recent=0, mass="rand", in_place=False, want_kept=True, seed=0, per_seq=None):
    c = plain.Cache(lens, H, d, page, dtype, seed, per_seq)
    gen, S = c.gen, len(lens)
    m = torch.rand((S, H, c.rows), generator=gen)
    if mass == "ties":
        m = torch.randint(0, 4, m.shape, generator=gen).float()
    elif mass == "zero":
        m.zero_()
    elif mass == "odd":
        m = torch.exp(20 * torch.randn(m.shape, generator=gen)) * torch.where(torch.rand(m.shape, generator=gen) < 0.3, -1.0, 1.0)
        m[torch.rand(m.shape, generator=gen) < 0.1] = math.inf
        m[torch.rand(m.shape, generator=gen) < 0.1] = math.nan
        m[torch.rand(m.shape, generator=gen) < 0.1] = 0.0
        m[torch.rand(m.shape, generator=gen) < 0.1] = -0.0
        m[torch.rand(m.shape, generator=gen) < 0.1] = -math.inf
        m[torch.rand(m.shape, generator=gen) < 0.05] = 1e-42
    seen = torch.tensor([n + 50 for n in lens], dtype=torch.int32)
    stamp = torch.stack([torch.stack([torch.randperm(c.rows + 50, generator=gen)[:c.rows] for _ in range(H)]) for _ in lens]).to(torch.int32)
    cache = c.dev(ws)
    md, sd = m.cuda(), stamp.cuda()
    mo, so, lo = (md, sd, cache.len) if in_place else (torch.full_like(md, -7.0), torch.full_like(sd, -7), torch.full_like(cache.len, -7))
    kept = torch.full((S, H, keep), -7, dtype=torch.int32, device="cuda") if want_kept else None
    first = None
    for again in range(1 if in_place else 2):
        ws.ws_synapse_paged_evict(cache, keep, seen.cuda(), md, sd, sinks, recent, mass_out=mo, stamp_out=so, len_out=lo, kept=kept)
        got = [cache.K.cpu(), cache.V.cpu(), mo.cpu(), so.cpu()]
        if first is not None:                       # made again with the same inputs: the same
            assert all(torch.equal(x.nan_to_num(9e9) if x.is_floating_point() else x, y.nan_to_num(9e9) if y.is_floating_point() else y)
                       for x, y in zip(first, got))
        first = got
    Kd, Vd, mo, so = first
    K, V = c.K.clone(), c.V.clone()
    mr, sr = (m.clone(), stamp.clone()) if in_place else (torch.full_like(m, -7.0), torch.full_like(stamp, -7))
    for s, n in enumerate(lens):
        assert int(lo[s]) == min(n, keep)
        for h in range(H):
            came, _ = plain.evict(n, keep, sinks, recent, int(seen[s]), m[s, h].tolist(), stamp[s, h].tolist())
            if want_kept:
                assert kept[s, h, :len(came)].tolist() == came, (s, h)
                assert (kept[s, h, len(came):] == -7).all()
            to = torch.arange(len(came))
            src = torch.tensor(came, dtype=torch.long)
            mr[s, h, :len(came)], sr[s, h, :len(came)] = m[s, h, src], stamp[s, h, src]
            for pool, ref in ((c.K, K), (c.V, V)):
                ref[c.table[s].long()[to // page], h, to % page] = pool[c.table[s].long()[src // page], h, src % page]
    same = lambda x, y: torch.equal(x.float().nan_to_num(9e9), y.float().nan_to_num(9e9))
    assert same(Kd, K) and same(Vd, V) and same(mo, mr) and same(so, sr)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 128)])
@pytest.mark.parametrize("keep", [1, 16, 100, 129, 700])
@pytest.mark.parametrize("mass", ["rand", "ties", "zero", "odd"])
def test_evict(ws, dtype, d, keep, mass):
    lens = [0, 1, 15, 99, 100, 101, 128, 130, 511, 700, 701]
    run_evict(ws, lens, 2, d, 16, dtype, keep, sinks=min(keep // 4, 3), recent=keep // 3, mass=mass, seed=keep)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("keep,sinks,recent", [(40, 0, 0), (40, 40, 0), (40, 0, 40), (40, 13, 27), (5000, 10, 20)])
def test_evict_protects(ws, in_place, keep, sinks, recent):
    run_evict(ws, [300, 41, 40, 77], 3, 64, 32, BF16, keep, sinks, recent, "ties", in_place, want_kept=not in_place)


@pytest.mark.parametrize("n,keep,mass", [(1023, 512, "rand"), (1024, 1000, "ties"), (1025, 3, "rand"), (5000, 4900, "zero"), (20000, 5000, "rand"),
                                         (70001, 50000, "ties"), (140000, 100, "rand")])
def test_evict_lengths(ws, n, keep, mass):
    run_evict(ws, [n, n // 2], 1, 64, 128, BF16, keep, 4, min(keep - 4, 64) if keep > 4 else 0, mass) if keep > 4 else \
        run_evict(ws, [n, n // 2], 1, 64, 128, BF16, keep, 1, 1, mass)


@pytest.mark.parametrize("keep", [100, 5000])
def test_evict_tables_with_room_for_far_more(ws, keep):
    """Tables of 131 072 rows of which a few are in use: one chunk or two of each head, more heads than workgroups for every chunk."""
    run_evict(ws, [0, 99, 101, 4097, 8200], 2, 64, 256, BF16, keep, 3, 20, "ties", per_seq=512)
    run_evict(ws, [130] * 70, 4, 64, 256, BF16, keep, 3, 20, "rand", in_place=True, want_kept=False, per_seq=512)


def test_evict_long_heads_with_fewer_workgroups_than_chunks(ws):
    run_evict(ws, [16500] + [90] * 41, 24, 64, 256, BF16, 2500, 3, 20, "rand")


def test_evict_many_heads(ws):
    run_evict(ws, [70] * 33, 16, 64, 16, BF16, 60, 2, 5, "ties")


def test_evict_leaves_out_pages_that_do_not_exist(ws):
    c = plain.Cache([64], 1, 64, 16, BF16, seed=2)
    good = c.table.clone()
    c.table[0, 0] = -1
    cache = c.dev(ws)
    mass = torch.arange(64, device="cuda", dtype=torch.float32)[None, None].contiguous()
    stamp = torch.arange(64, device="cuda", dtype=torch.int32)[None, None].contiguous()
    ws.ws_synapse_paged_evict(cache, 32, cache.len.clone(), mass, stamp)
    # rows 32..63 would fill rows 0..31; of these 0..15 have no page
    K = c.K.clone()
    K[good[0, 1]] = c.K[good[0, 3]]
    assert torch.equal(cache.K.cpu().float().nan_to_num(9e9), K.float().nan_to_num(9e9)) and cache.len.item() == 32


# ---- together ---------------------------------------------------------------------------------------------------------------
def test_agents_decode_over_a_shared_synapse(ws):
    """select -> gather -> the synapse into shared pages -> agents append, attend and evict for 60 tokens, against 64 bits."""
    H, g, d, page, N, L, k, budget, steps = 2, 2, 64, 16, 5, 1000, 40, 48, 60
    gen = torch.Generator().manual_seed(0)
    Kctx, Vctx = (torch.randn((H, L, d), generator=gen).to(BF16).cuda() for _ in range(2))
    rho = ws.ws_synapse_density(Kctx, [5.0] * H)
    Ks, Vs = ws.ws_synapse_gather(Kctx, Vctx, ws.ws_synapse_select(Kctx, rho, k, 0.5))
    # whole pages of the synapse only: a page that is shared must not be written again
    shared, own = k // page, 4
    k_used = shared * page
    per_seq = shared + own
    pages = shared + N * own
    K = torch.full((pages, H, page, d), math.nan, dtype=BF16, device="cuda")
    V = torch.full_like(K, math.nan)
    perm = torch.randperm(pages, generator=gen).to(torch.int32)
    table = torch.cat([perm[:shared].expand(N, shared), perm[shared:].view(N, own)], dim=1).contiguous().cuda()
    lens = torch.full((N,), k_used, dtype=torch.int32, device="cuda")
    cache = ws.PagedCache(K, V, table, lens)
    first = torch.zeros((N + 1,), dtype=torch.int32, device="cuda")
    first[1:] = k_used
    ws.ws_synapse_paged_append(cache, Ks[:, :k_used].transpose(0, 1), Vs[:, :k_used].transpose(0, 1), first)
    seen = lens.clone()
    stamp = torch.zeros((N, H, cache.rows), dtype=torch.int32, device="cuda")
    stamp[:, :, :k_used] = torch.arange(k_used, dtype=torch.int32, device="cuda")
    mass = torch.zeros((N, H, cache.rows), device="cuda")
    # the 64-bit side: per agent and head a list of (key, value, stamp, account)
    ref = [[[(Ks[h, r].double().cpu(), Vs[h, r].double().cpu(), r, 0.0) for r in range(k_used)] for h in range(H)] for _ in range(N)]
    each = torch.arange(N + 1, dtype=torch.int32, device="cuda")
    evictions = 0
    for step in range(steps):
        q, kn, vn = (torch.randn((N, n, d), generator=gen).to(BF16) for n in (H * g, H, H))
        lens.add_(1)
        seen.add_(1)
        pos = seen - 1
        qr = ws.ws_synapse_paged_append(cache, kn.cuda(), vn.cuda(), each, pos=pos, q=q.cuda(), seen=seen, stamp=stamp, mass=mass)
        lse = torch.empty((N, H * g), device="cuda")
        O = ws.ws_synapse_paged_attend(cache, qr, lse=lse, decay=0.9, mass_in=mass, mass_out=mass)
        n = int(lens[0])
        qh, Kh = qr.cpu().double(), cache.K.cpu()
        rk = plain.rotate(kn.double(), pos.cpu()[None], [d // 2], 1e6)
        for a in range(N):
            for h in range(H):
                row = (Kh[int(table[a, (n - 1) // page]), h, (n - 1) % page].double())
                # (one rounding of the rotated key: 2^-8 of bf16, and the fp32 sines)
                assert ((row - rk[a, h]).abs() <= rk[a, h].abs() * 2.0 ** -8 + 1e-5).all()
                ref[a][h].append((row, vn[a, h].double(), int(seen[a]) - 1, 0.0))
                keys, values = torch.stack([x[0] for x in ref[a][h]]), torch.stack([x[1] for x in ref[a][h]])
                z = qh[a, h * g:(h + 1) * g] @ keys.T / 8.0
                p = torch.softmax(z, dim=1)
                assert ((O[a, h * g:(h + 1) * g].cpu().double() - p @ values).abs() <= 3e-5 * (p @ values.abs()) + 1e-30).all()
                assert (lse[a, h * g:(h + 1) * g].cpu().double() - torch.logsumexp(z, dim=1)).abs().max() < 1e-4
                w = p.sum(dim=0)
                ref[a][h] = [(x[0], x[1], x[2], 0.9 * x[3] + float(w[i])) for i, x in enumerate(ref[a][h])]
                acc = torch.tensor([x[3] for x in ref[a][h]], dtype=torch.float64)
                # every step adds 3e-5 of a weight at most, and the account is rounded once a step
                assert ((mass[a, h, :n].cpu().double() - acc).abs() <= 1e-4 * acc).all()
                assert stamp[a, h, :n].tolist() == [x[2] for x in ref[a][h]]
        if n >= budget + 8:
            before = mass.cpu(), stamp.cpu()
            ws.ws_synapse_paged_evict(cache, budget, seen, mass, stamp, sinks=k_used, recent=10)
            evictions += 1
            assert (lens == budget).all()
            for a in range(N):
                for h in range(H):
                    # which rows go is decided by the library's own accounts (they are right to 1e-4, see above)
                    came, _ = plain.evict(n, budget, k_used, 10, int(seen[a]), before[0][a, h].tolist(), before[1][a, h].tolist())
                    ref[a][h] = [ref[a][h][r] for r in came]
                    assert stamp[a, h, :budget].tolist() == [x[2] for x in ref[a][h]]
                    assert came[:k_used] == list(range(k_used))
    assert evictions >= 4


def test_two_batches_at_once_on_two_streams(ws):
    """Two caches, two streams, a workspace each: attention and eviction of both in flight together, the same bits as one after the
    other (long enough for the calls to overlap: splits, joins, long heads over chunks)."""
    torch.manual_seed(0)
    sets = []
    for i in range(2):
        H, d, page, rows = 8, 128, 64, 20480
        K = torch.randn((2 * rows // page, H, page, d), device="cuda").to(BF16)
        V = torch.randn_like(K)
        table = torch.randperm(2 * rows // page, device="cuda").to(torch.int32).view(2, -1).contiguous()
        cache = ws.PagedCache(K, V, table, torch.tensor([rows - 37 * i, rows - 1000], dtype=torch.int32, device="cuda"))
        mass = torch.rand((2, H, rows), device="cuda")
        sets.append(dict(cache=cache, Q=torch.randn((2, 32, d), device="cuda").to(BF16), mass=mass, out=torch.zeros_like(mass),
                         O=torch.zeros((2, 32, d), device="cuda"), seen=cache.len + 5, mass2=torch.zeros_like(mass),
                         stamp=torch.arange(rows, dtype=torch.int32, device="cuda").expand(2, H, rows).contiguous(),
                         stamp2=torch.zeros((2, H, rows), dtype=torch.int32, device="cuda"), len2=torch.zeros_like(cache.len), K0=K.clone(), V0=V.clone(),
                         wa=ws.ws_synapse_paged_workspace(cache, "attend", 32, True), we=ws.ws_synapse_paged_workspace(cache, "evict", keep=9000)))

    def go(s, stream=None):
        ws.ws_synapse_paged_attend(s["cache"], s["Q"], O=s["O"], decay=0.5, mass_in=s["mass"], mass_out=s["out"], workspace=s["wa"], stream=stream)
        ws.ws_synapse_paged_evict(s["cache"], 9000, s["seen"], s["out"], s["stamp"], 4, 100, mass_out=s["mass2"], stamp_out=s["stamp2"],
                                  len_out=s["len2"], workspace=s["we"], stream=stream)

    results = lambda s: [s[n].clone() for n in ("O", "out", "mass2", "stamp2", "len2")] + [s["cache"].K.clone(), s["cache"].V.clone()]
    want = []
    for s in sets:
        go(s)
        torch.cuda.synchronize()
        want.append(results(s))
        assert s["len2"].tolist() == [9000, 9000]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for again in range(3):
        for s in sets:
            s["cache"].K.copy_(s["K0"])
            s["cache"].V.copy_(s["V0"])
            for n in ("O", "out", "mass2", "stamp2", "len2"):
                s[n].zero_()
        torch.cuda.synchronize()
        for s, stream in zip(sets, streams):
            go(s, stream)
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            assert all(torch.equal(a, b) for a, b in zip(results(s), w))


def test_a_step_in_a_graph_and_on_another_stream(ws):
    """append -> attend -> evict captured once and replayed on new inputs, with eager work between, equals the eager calls; and the
    same on a stream that is not the current one."""
    H, g, d, page, S = 2, 4, 128, 32, 9
    c = plain.Cache([90 + 13 * s for s in range(S)], H, d, page, BF16, seed=1)
    cache = c.dev(ws)
    cache.K.nan_to_num_(0.0)
    cache.V.nan_to_num_(0.0)
    K0, V0, len0 = cache.K.clone(), cache.V.clone(), cache.len.clone()
    q, k, v = (torch.zeros((S, n, d), dtype=BF16, device="cuda") for n in (H * g, H, H))
    qr = torch.zeros_like(q)
    O, lse = torch.zeros((S, H * g, d), device="cuda"), torch.zeros((S, H * g), device="cuda")
    mass = torch.zeros((S, H, cache.rows), device="cuda")
    stamp = torch.arange(cache.rows, dtype=torch.int32, device="cuda").expand(S, H, cache.rows).contiguous()
    first = torch.arange(S + 1, dtype=torch.int32, device="cuda")
    pos, seen = cache.len - 1, cache.len.clone()
    mass_out, stamp_out, len_out = torch.zeros_like(mass), torch.zeros_like(stamp), torch.zeros_like(cache.len)
    wa = ws.ws_synapse_paged_workspace(cache, "attend", H * g, True)
    we = ws.ws_synapse_paged_workspace(cache, "evict", keep=100)
    outs = (cache.K, cache.V, qr, O, lse, mass, stamp, mass_out, stamp_out, len_out)

    def step(stream=None):
        ws.ws_synapse_paged_append(cache, k, v, first, pos=pos, q=q, q_out=qr, seen=seen, stamp=stamp, mass=mass, stream=stream)
        ws.ws_synapse_paged_attend(cache, qr, O=O, lse=lse, decay=0.5, mass_in=mass, mass_out=mass, workspace=wa, stream=stream)
        ws.ws_synapse_paged_evict(cache, 100, seen, mass, stamp, 2, 8, mass_out=mass_out, stamp_out=stamp_out, len_out=len_out,
                                  workspace=we, stream=stream)

    def load(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        cache.K.copy_(K0)
        cache.V.copy_(V0)
        for t in (q, k, v):
            t.normal_(generator=gen)
        mass.uniform_(generator=gen)
        for t in (O, lse, mass_out, stamp_out, len_out):
            t.zero_()

    load(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for seed in (1, 2, 1, 3):
        load(seed)
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for how in ("graph", "stream"):
            load(seed)
            torch.cuda.synchronize()
            if how == "graph":
                graph.replay()
            else:
                step(side)
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(outs, want)):
                assert torch.equal(a, b), (how, seed, i)
