"""The paged cache's calls as a program makes them: streams, sizes at the borders of the choices between kernels."""
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


def test_a_stream_given_by_its_handle(ws):
    """The same bits as on the stream object, and the workspace that the call made for itself is not handed to the current stream while
    the other one may still use it."""
    c = plain.Cache([3000, 700, 0, 41], 2, 64, 16, BF16, seed=31)
    cache = c.dev(ws)
    Q = torch.randn((4, 6, 64), generator=c.gen).to(BF16).cuda()
    want = ws.ws_synapse_paged_attend(cache, Q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ws.ws_synapse_paged_attend(cache, Q, stream=side.cuda_stream)
    zero = ws.ws_synapse_paged_attend(cache, Q, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(zero, want)
    size = 37 << 20
    w = ws._workspace(size, cache.device, None, side.cuda_stream)
    at = w.data_ptr()
    del w
    here = torch.empty(size, dtype=torch.uint8, device="cuda")
    with torch.cuda.stream(side):
        there = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert here.data_ptr() != at and there.data_ptr() == at
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,weights", [(1536, False), (1552, False), (2048, True), (2064, True)])
def test_one_long_sequence_among_short_ones(ws, dtype, rows, weights):
    """512 heads, on both sides of the widths up to which each has a workgroup of its own."""
    lens = [5 + i for i in range(64)]
    lens[17], lens[40] = rows, 0
    c = plain.Cache(lens, 8, 64, 16, dtype, seed=rows)
    Q = torch.randn((64, 8, 64), generator=c.gen).to(dtype)
    want = plain.attend(c, Q)
    cache = c.dev(ws)
    none = ws.ws_synapse_workspace_bytes(ws.WS_OP_PAGED_ATTEND, ws._dtype_code(cache.K), 8, cache.rows, 64, k=int(weights), N=64, Hq=8) == 0
    assert none == (rows in (1536, 2048))
    lse = torch.empty((64, 8), device="cuda")
    mass = torch.full((64, 8, cache.rows), float("nan"), device="cuda") if weights else None
    O = ws.ws_synapse_paged_attend(cache, Q.cuda(), lse=lse, mass_out=mass)
    plain.check_attention(O, lse, want, rows)
    if weights:
        plain.check_weights(mass, None, 1.0, want, lens, rows)
