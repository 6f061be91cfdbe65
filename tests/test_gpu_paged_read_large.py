"""Reading back more than one launch can have threads for."""
import pytest
import torch

from paper_2411_09909_amd import binding
from tests.test_gpu_paged import make_pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,heads", [(torch.bfloat16, 17), (torch.float32, 9)])
def test_read_of_more_elements_than_a_launch_has_threads_for(dtype, heads):
    """2^24 rows (the most) of 17 heads of 128 are 2^32 runs of 8 elements, a thread each, and a sixteenth more, 73 GB each of keys and of values;
    with float32 two launches' worth. The slots come round every 4111 rows (odd, so that no launch begins with a round): each round equals
    what a small call reads."""
    rows, dim, period = 1 << 24, 128, 4111
    need = 2 * rows * heads * dim * dtype.itemsize
    if torch.cuda.mem_get_info()[0] < need + (20 << 30):
        pytest.skip("not enough free memory for the outputs")
    fmt = binding.make_format()
    pool = make_pool(fmt, 65, heads, dim, 64, seed=3)
    for s in (pool[1], pool[3]):
        s.copy_(s % 0x78)  # finite scales
    few = torch.randperm(65 * 64, generator=torch.Generator().manual_seed(1))[:period].to(torch.int32).cuda()
    want = binding.paged_read(fmt, pool, few, dtype=dtype)
    slots = few.repeat(-(-rows // period))[:rows].contiguous()
    k, v = (torch.full((rows, heads, dim), 3.0, dtype=dtype, device="cuda") for _ in range(2))
    binding.paged_read(fmt, pool, slots, k=k, v=v)
    whole = rows // period
    for got, w in zip((k, v), want):
        word = torch.int16 if dtype == torch.bfloat16 else torch.int32
        got, w = got.view(word), w.view(word)
        for i in range(0, whole, 200):
            n = min(200, whole - i)
            assert torch.equal(got[i * period:(i + n) * period].view(n, -1), w.view(1, -1).expand(n, -1)), i
        assert torch.equal(got[whole * period:], w[:rows - whole * period])
    del k, v, got, slots
    torch.cuda.empty_cache()
