"""What the binding checks of workspaces (where they are, and that they are dense) and of tables.  Nothing is called."""
import pytest
import torch


@pytest.fixture(scope="module")
def biq():
    import paper_2005_09904_amd as biq
    from paper_2005_09904_amd import build

    if build.is_stale():
        build.build_library()
    biq.load_library()
    return biq


def attention(biq, workspace):
    page = biq.biq_cache_page_bytes(32, 2, 64)
    cache = biq.KvCache(torch.zeros((5, page), dtype=torch.uint8), torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 32, 2, 64)
    q = torch.zeros((2, 4, 64))
    return biq.PreparedAttention(cache, q, torch.zeros_like(q), workspace=workspace, stream=Stream())


def verify(biq, workspace):
    p = torch.zeros((2, 4, 50))
    return biq.PreparedVerify(p, None, torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 4)), torch.zeros((2, 4), dtype=torch.int32),
                              torch.zeros(2, dtype=torch.int32), workspace=workspace, stream=Stream())


class Stream:
    cuda_stream = 0x7000


@pytest.mark.parametrize("call", [attention, verify])
def test_workspace(biq, call):
    for bad in (torch.empty(4096, dtype=torch.uint8, device="meta"), torch.empty(1, dtype=torch.uint8).expand(4096),
                torch.empty(8192, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="workspace"):
            call(biq, bad)
    for good in (None, torch.empty(4096, dtype=torch.uint8), torch.empty((4, 64))):
        call(biq, good)                                         # (prepared, not called)


@pytest.mark.parametrize("shape", [(0, 4), (2, 0), (0, 0)])
def test_a_table_without_sequences_or_pages(biq, shape):
    page = biq.biq_cache_page_bytes(32, 2, 64)
    with pytest.raises(ValueError, match="table"):
        biq.KvCache(torch.zeros((5, page), dtype=torch.uint8), torch.zeros(shape, dtype=torch.int32), torch.zeros(shape[0], dtype=torch.int32), 32, 2, 64)
