"""What the paged cache's binding does with arguments before any pointer reaches the library; no GPU needed: a cache object whose
tensors lie on the host stands in for one."""
import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2601_01298_amd import binding
    return binding


def host_cache(b, S=3, H=2, page=16, d=64, per_seq=4):
    """A PagedCache without its constructor's demand for device tensors."""
    c = object.__new__(b.PagedCache)
    K = torch.zeros((S * per_seq, H, page, d), dtype=torch.bfloat16)
    c.K, c.V, c.table, c.len = K, K.clone(), torch.zeros((S, per_seq), dtype=torch.int32), torch.zeros((S,), dtype=torch.int32)
    c.device, c.dtype, c._index = K.device, K.dtype, K.get_device()
    c.pages, c.Hkv, c.page, c.d, c.S, c.per_seq, c.rows = S * per_seq, H, page, d, S, per_seq, per_seq * page
    c._per_seq, c._per_row, c._pairs, c._ref = (S,), (S, H, c.rows), {}, None
    return c


@pytest.mark.parametrize("shape", [(), (64,), (3, 64), (3, 2, 1, 64)])
def test_rows_with_another_number_of_dimensions(b, shape):
    """ValueError as for any other wrong shape, never an IndexError from inside."""
    c, odd, good = host_cache(b), torch.zeros(shape, dtype=torch.bfloat16), torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    first = torch.zeros((4,), dtype=torch.int32)
    for kw in (dict(k=odd, v=good), dict(k=good, v=odd), dict(k=good, v=good, q=odd)):
        with pytest.raises(ValueError):
            b.ws_synapse_paged_append(c, first=first, **kw)
    with pytest.raises(ValueError):
        b.ws_synapse_paged_attend(c, odd)


@pytest.mark.parametrize("shape", [(), (1, 1, 3)])
def test_positions_with_another_number_of_dimensions(b, shape):
    c, good = host_cache(b), torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        b.ws_synapse_paged_append(c, good, good, torch.zeros((4,), dtype=torch.int32), pos=torch.zeros(shape, dtype=torch.int32))


class Recorder:
    """Stands in for the loaded library: keeps what a call was given and answers as told."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def recorded(b, monkeypatch):
    r = Recorder()
    monkeypatch.setattr(b, "lib", lambda: r)
    monkeypatch.setattr(b, "_device", lambda: -1)
    monkeypatch.setattr(b, "_raw_stream", lambda device: 0)
    return r


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32 + 8, 2 ** 64 + 8, -2 ** 32 + 8, -2 ** 31 - 1])
def test_numbers_of_more_than_32_bits_do_not_wrap(b, recorded, n):
    """A ctypes int keeps the low 32 bits: 2^32 + 8 rows to keep would be 8, and the rest of the cache given up.  What reaches the
    library is out of its range on the same side, so that it refuses the call."""
    c = host_cache(b)
    per_row = lambda t: torch.zeros(c._per_row, dtype=t)
    for name in ("keep", "sinks", "recent"):
        kw = {"keep": 8, "sinks": 0, "recent": 0, name: n}
        b.ws_synapse_paged_evict(c, kw["keep"], torch.zeros((3,), dtype=torch.int32), per_row(torch.float32), per_row(torch.int32), sinks=kw["sinks"],
                                 recent=kw["recent"], workspace=torch.zeros(256, dtype=torch.uint8))
        got = dict(zip(("keep", "sinks", "recent"), recorded.calls[-1][1][1:4]))
        assert all(-2 ** 31 <= x < 2 ** 31 for x in got.values()), got
        assert got[name] >= 2 ** 24 if n > 0 else got[name] < 0
        assert all(got[o] == kw[o] for o in got if o != name)
    b.ws_synapse_workspace_bytes(b.WS_OP_PAGED_EVICT, b.WS_BF16, 2, 64, 64, k=n, N=3)
    assert recorded.calls[-1][1][5] == (2 ** 31 - 1 if n > 0 else -2 ** 31)


def test_more_tokens_than_32_bits_count(b, recorded):
    c = host_cache(b)
    k = torch.zeros((1, 2, 64), dtype=torch.bfloat16).expand(2 ** 32 + 1, 2, 64)
    b.ws_synapse_paged_append(c, k, k, torch.zeros((4,), dtype=torch.int32))
    T = recorded.calls[-1][1][3]
    assert recorded.calls[-1][0] == "ws_synapse_paged_append" and 2 ** 24 <= T < 2 ** 31


@pytest.mark.parametrize("pairs", [(2 ** 32 + 32,), (2 ** 32 + 16, -2 ** 32 + 16)])
def test_numbers_of_pairs_do_not_wrap(b, recorded, pairs):
    c, good = host_cache(b), torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    b.ws_synapse_paged_append(c, good, good, torch.zeros((4,), dtype=torch.int32), pos=torch.zeros((len(pairs), 3), dtype=torch.int32), pairs=pairs)
    assert list(recorded.calls[-1][1][7]) == [2 ** 31 - 1 if n > 0 else -2 ** 31 for n in pairs]


def test_memory_for_a_stream_given_by_its_handle_belongs_to_that_stream(b, monkeypatch):
    """A workspace made by the call is free again when the call returns.  Allocated on the current stream it would be given to that
    stream's next work while the kernels on the other one still use it."""
    entered = []

    class Stream:
        def __init__(self, handle):
            self.cuda_stream = handle

    class on:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            entered.append(self.stream.cuda_stream)

        def __exit__(self, *a):
            pass

    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: Stream(0))
    monkeypatch.setattr(torch.cuda, "stream", on)
    for make in (lambda s: b._workspace(512, "cpu", None, s), lambda s: b._new((3,), torch.float32, "cpu", s)):
        for stream, want in ((None, []), (0x5550, [0x5550]), (0, [0]), (Stream(0x7770), [0x7770])):
            entered.clear()
            make(stream)
            assert entered == want, stream


def test_a_stream_of_another_device_is_refused(b, recorded):
    from types import SimpleNamespace
    c = host_cache(b)
    good = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    stream = lambda index: SimpleNamespace(cuda_stream=0x40, device=torch.device("cuda", index), device_index=index)
    with pytest.raises(ValueError, match="stream"):
        b.ws_synapse_paged_append(c, good, good, torch.zeros((4,), dtype=torch.int32), stream=stream(1))
    assert not recorded.calls
    c._index = 0
    b._device = lambda: 0                                # (put back by the fixture)
    assert c._stream(stream(0)) == 0x40
    with pytest.raises(ValueError, match="stream"):
        c._stream(stream(1))


def test_wide_tables_are_shared_out_however_many_heads_there_are(b):
    """A workgroup per head (no workspace) only where the longest head there may be is short: the lengths are on the device, and one
    head of 5000 rows among short ones would take 72 us by itself where equal runs take 19."""
    size = lambda L, weights, N=64, H=8, Hq=8: b.ws_synapse_workspace_bytes(b.WS_OP_PAGED_ATTEND, b.WS_BF16, H, L, 128, k=weights, N=N, Hq=Hq)
    assert size(1536, 0) == 0 < size(1552, 0) and size(5120, 0) > 0 and size(4096, 0, N=512) > 0
    assert size(2048, 1) == 0 < size(2064, 1) and size(4096, 1) > 0
    assert size(1536, 0, N=63) > 0 and size(1216, 1, Hq=32) == 0 < size(1536, 1, Hq=32)
