"""What the calls about pages keep in a context is what the header says."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("call", ["compact", "extend"])
def test_scratch_of_pages(call):
    """n_pages / 4 bytes beyond a few words a sequence; memory is given out in pieces of 2 MB."""
    from paper_1509_05194_amd import hclae
    n_pages, page = 2 ** 27, 1
    ctx = hclae.Context(1, 4, 1, 1)
    tables = torch.tensor([[n_pages - 1, 5, 5, 7]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([3], dtype=torch.int32, device="cuda")
    src, dst = (torch.full((n_pages // 2,), 9, dtype=torch.int32, device="cuda") for _ in range(2))
    one = [torch.full((1,), 9, dtype=torch.int32, device="cuda") for _ in range(4)]
    slots = torch.full((1,), 9, dtype=torch.int64, device="cuda")
    starts = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    ctx.cache_compact(tables.clone(), lengths, page, 70000, src[:35000], dst[:35000])      # the kernels are loaded
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    if call == "compact":
        ctx.cache_compact(tables, lengths, page, n_pages, src, dst, used=one[0])
    else:
        ctx.cache_extend(tables, lengths, starts, page, n_pages, slots, one[1], one[2], one[3])
    torch.cuda.synchronize()
    assert free - torch.cuda.mem_get_info()[0] <= n_pages // 4 + 2 ** 22
    if call == "compact":                          # two pages in use go to the two lowest
        assert one[0].item() == 2 and tables[0].tolist() == [1, 0, 0, 7]
        assert src[:3].tolist() == [5, n_pages - 1, -1] and dst[:3].tolist() == [0, 1, -1]
    else:
        assert tables[0].tolist() == [n_pages - 1, 5, 5, 0] and lengths.item() == 4 and slots.item() == 0
    ctx.close()
