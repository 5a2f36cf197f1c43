"""Host-only checks of the paged cache's entry points: what they refuse before anything is enqueued, and what workspace they ask for."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2601_01298_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    binding.lib()
    return binding


FAKE, ODD, BIG = 0x1000, 0x1004, 1 << 45


def cache(b, **kw):
    f = dict(K=FAKE, V=FAKE, table=FAKE, len=FAKE, dt=b.WS_BF16, pages=100, Hkv=4, page=16, d=64, S=3, per_seq=20)
    f.update(kw)
    return b._PagedCache(*[f[n] for n, _ in b._PagedCache._fields_])


BAD_CACHES = [
    (dict(K=None), "INVALID_ARG"), (dict(V=None), "INVALID_ARG"), (dict(table=None), "INVALID_ARG"), (dict(len=None), "INVALID_ARG"),
    (dict(K=ODD), "INVALID_ARG"), (dict(V=ODD), "INVALID_ARG"), (dict(table=FAKE + 2), "INVALID_ARG"), (dict(len=FAKE + 1), "INVALID_ARG"),
    (dict(pages=0), "INVALID_ARG"), (dict(Hkv=0), "INVALID_ARG"), (dict(S=0), "INVALID_ARG"), (dict(per_seq=0), "INVALID_ARG"),
    (dict(S=-1), "INVALID_ARG"), (dict(dt=2), "UNSUPPORTED"), (dict(dt=-1), "UNSUPPORTED"), (dict(d=96), "UNSUPPORTED"), (dict(d=0), "UNSUPPORTED"),
    (dict(page=8), "UNSUPPORTED"), (dict(page=48), "UNSUPPORTED"), (dict(page=512), "UNSUPPORTED"), (dict(page=0), "UNSUPPORTED"),
    (dict(per_seq=1 << 20), "UNSUPPORTED"), (dict(per_seq=2147483647, page=256), "UNSUPPORTED"),
    (dict(S=1 << 20), "UNSUPPORTED"), (dict(S=2147483647, Hkv=2147483647), "UNSUPPORTED"),
]


def append(b, c, **kw):
    rows = lambda x=FAKE, token=256, head=64: b._Rows(x, token, head)
    a = dict(k=rows(), v=rows(), T=5, first=FAKE, pos=FAKE, axes=1, pairs=[32], base=1e6, q=rows(), Hq=8, q_out=FAKE, seen=FAKE, stamp=FAKE, mass=FAKE)
    for name, value in kw.items():
        a[name] = rows(**value) if name in ("k", "v", "q") and isinstance(value, dict) else value
    by = lambda r: None if r is None else ctypes.byref(r)
    pairs = None if a["pairs"] is None else (ctypes.c_int * len(a["pairs"]))(*a["pairs"])
    return b.lib().ws_synapse_paged_append(by(c), by(a["k"]), by(a["v"]), a["T"], a["first"], a["pos"], a["axes"], pairs, a["base"], by(a["q"]), a["Hq"],
                                           a["q_out"], a["seen"], a["stamp"], a["mass"], None)


def attend(b, c, Q=FAKE, Hq=8, scale=0.0, O=FAKE, lse=FAKE, decay=1.0, mass_in=FAKE, mass_out=FAKE, space=FAKE, size=BIG):
    return b.lib().ws_synapse_paged_attend(None if c is None else ctypes.byref(c), Q, Hq, scale, O, lse, decay, mass_in, mass_out, space, size, None)


def evict(b, c, keep=50, sinks=4, recent=10, seen=FAKE, mass_in=FAKE, mass_out=FAKE, stamp_in=FAKE, stamp_out=FAKE, len_out=FAKE, kept=FAKE, space=FAKE,
          size=BIG):
    return b.lib().ws_synapse_paged_evict(None if c is None else ctypes.byref(c), keep, sinks, recent, seen, mass_in, mass_out, stamp_in, stamp_out,
                                          len_out, kept, space, size, None)


@pytest.mark.parametrize("fields,why", BAD_CACHES)
def test_bad_caches(b, fields, why):
    for call in (append, attend, evict):
        assert call(b, cache(b, **fields)) == getattr(b, "WS_ERR_" + why), (call.__name__, fields)


def test_no_cache(b):
    for call in (append, attend, evict):
        assert call(b, None) == b.WS_ERR_INVALID_ARG


@pytest.mark.parametrize("kw,why", [
    (dict(k=None), "INVALID_ARG"), (dict(v=None), "INVALID_ARG"), (dict(k=dict(x=None)), "INVALID_ARG"), (dict(v=dict(x=ODD)), "INVALID_ARG"),
    (dict(k=dict(token=-64)), "INVALID_ARG"), (dict(k=dict(token=68)), "INVALID_ARG"), (dict(v=dict(head=4)), "INVALID_ARG"),
    (dict(q=dict(head=-8)), "INVALID_ARG"), (dict(q=dict(x=None)), "INVALID_ARG"), (dict(Hq=0), "INVALID_ARG"), (dict(q_out=None), "INVALID_ARG"),
    (dict(q_out=ODD), "INVALID_ARG"), (dict(Hq=1 << 20), "UNSUPPORTED"), (dict(T=0), "INVALID_ARG"), (dict(T=-3), "INVALID_ARG"),
    (dict(T=1 << 24), "UNSUPPORTED"), (dict(first=None), "INVALID_ARG"), (dict(first=FAKE + 2), "INVALID_ARG"), (dict(pos=FAKE + 1), "INVALID_ARG"),
    (dict(axes=0, pairs=[]), "UNSUPPORTED"), (dict(axes=5, pairs=[8, 8, 8, 4, 4]), "UNSUPPORTED"), (dict(pairs=None), "INVALID_ARG"),
    (dict(pairs=[31]), "INVALID_ARG"), (dict(pairs=[33]), "INVALID_ARG"), (dict(axes=2, pairs=[40, -8]), "INVALID_ARG"),
    (dict(axes=2, pairs=[2147483647, 2147483647]), "INVALID_ARG"), (dict(base=0.0), "INVALID_ARG"), (dict(base=-1.0), "INVALID_ARG"),
    (dict(base=float("nan")), "INVALID_ARG"), (dict(base=float("inf")), "INVALID_ARG"), (dict(seen=None), "INVALID_ARG"),
    (dict(stamp=FAKE + 2), "INVALID_ARG"), (dict(mass=FAKE + 3), "INVALID_ARG"),
])
def test_append_refuses(b, kw, why):
    assert append(b, cache(b), **kw) == getattr(b, "WS_ERR_" + why)


@pytest.mark.parametrize("kw,why", [
    (dict(Q=None), "INVALID_ARG"), (dict(Q=ODD), "INVALID_ARG"), (dict(O=None), "INVALID_ARG"), (dict(O=ODD), "INVALID_ARG"), (dict(Hq=6), "INVALID_ARG"),
    (dict(Hq=0), "INVALID_ARG"), (dict(Hq=-4), "INVALID_ARG"), (dict(scale=float("inf")), "INVALID_ARG"), (dict(scale=float("nan")), "INVALID_ARG"),
    (dict(lse=FAKE + 2), "INVALID_ARG"), (dict(decay=-0.5), "INVALID_ARG"), (dict(decay=float("nan")), "INVALID_ARG"), (dict(decay=float("inf")), "INVALID_ARG"),
    (dict(mass_out=None), "INVALID_ARG"), (dict(mass_in=FAKE + 1), "INVALID_ARG"), (dict(mass_out=FAKE + 1), "INVALID_ARG"), (dict(Hq=1 << 20), "UNSUPPORTED"),
    (dict(space=None), "WORKSPACE"), (dict(space=0x1010), "WORKSPACE"), (dict(size=16), "WORKSPACE"),
])
def test_attend_refuses(b, kw, why):
    assert attend(b, cache(b, per_seq=200), **kw) == getattr(b, "WS_ERR_" + why)


@pytest.mark.parametrize("kw,why", [
    (dict(keep=0), "INVALID_ARG"), (dict(keep=-1), "INVALID_ARG"), (dict(sinks=-1), "INVALID_ARG"), (dict(recent=-1), "INVALID_ARG"),
    (dict(sinks=41), "INVALID_ARG"), (dict(sinks=2147483647, recent=2147483647), "INVALID_ARG"), (dict(keep=1 << 24), "UNSUPPORTED"),
    *((dict([(n, v)]), "INVALID_ARG") for n in ("seen", "mass_in", "mass_out", "stamp_in", "stamp_out", "len_out") for v in (None, FAKE + 2)),
    (dict(kept=FAKE + 2), "INVALID_ARG"), (dict(space=None), "WORKSPACE"), (dict(space=0x1010), "WORKSPACE"), (dict(size=16), "WORKSPACE"),
])
def test_evict_refuses(b, kw, why):
    assert evict(b, cache(b), **kw) == getattr(b, "WS_ERR_" + why)


def test_workspaces(b):
    size = lambda op, **kw: b.ws_synapse_workspace_bytes(op, b.WS_BF16, kw.pop("H", 8), kw.pop("L", 4096), kw.pop("d", 128), **kw)
    plain, weights = (size(b.WS_OP_PAGED_ATTEND, k=w, N=16, Hq=32) for w in (0, 1))
    assert 0 < plain < weights <= plain + 16 * 32 * 4096 * 4 + 4096
    # short caches are one workgroup's and need nothing
    assert size(b.WS_OP_PAGED_ATTEND, k=0, N=16, Hq=32, L=512) == 0 < size(b.WS_OP_PAGED_ATTEND, k=0, N=16, Hq=32, L=528)
    assert size(b.WS_OP_PAGED_ATTEND, k=1, N=100, Hq=8, L=1200) == 0
    assert size(b.WS_OP_PAGED_EVICT, k=100, N=16) >= 16 * 8 * 100 * 8
    for op, kw in ((b.WS_OP_PAGED_ATTEND, dict(N=16, Hq=30)), (b.WS_OP_PAGED_ATTEND, dict(N=0, Hq=32)), (b.WS_OP_PAGED_ATTEND, dict(N=16, Hq=0)),
                   (b.WS_OP_PAGED_ATTEND, dict(N=1 << 20, Hq=32)), (b.WS_OP_PAGED_ATTEND, dict(N=1, Hq=8, L=1 << 24)), (b.WS_OP_PAGED_ATTEND, dict(N=1, Hq=8, d=96)),
                   (b.WS_OP_PAGED_EVICT, dict(N=16, k=0)), (b.WS_OP_PAGED_EVICT, dict(N=0, k=5)), (b.WS_OP_PAGED_EVICT, dict(N=1 << 20, k=5)),
                   (b.WS_OP_PAGED_EVICT, dict(N=1, k=5, L=1 << 24))):
        with pytest.raises(b.WsError):
            size(op, **kw)


def test_the_binding_checks_tensors_before_any_pointer_is_taken(b):
    import torch
    K = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        b.PagedCache(K, K, torch.zeros((1, 4), dtype=torch.int32), torch.zeros((1,), dtype=torch.int32))       # not on a device
