"""sr_attn_prefill at more work items than one dimension of a grid holds (2^32)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_more_work_items_than_one_dimension_holds(gpu):
    """256 sequences of one token with 65535 heads: 258 x 65535 workgroups of 256 lanes.  A row that sees one key gives its value."""
    n, heads, d = 256, 65535, 64
    print("case prefill", n, heads, d, flush=True)
    assert (n // 128 + n) * heads * 256 > 1 << 32
    x = torch.empty((n, heads * d), dtype=torch.float16, device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(0))
    cu = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    got = gpu.sr_attn_prefill(x, x, x, cu, cu, d)
    torch.cuda.synchronize()
    assert torch.equal(got, x)
