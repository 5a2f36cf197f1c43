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
