"""What the gated block and the AdamW step hold of memory."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_closed_block_holds_no_workspace():
    """Also while the object is still there; a call on it is refused."""
    import torch
    import paper_2312_08728_amd as B
    p, f, c, r = 64, 128, 72, 20
    x, gate, up, down, y = (torch.randn(s, device="cuda").bfloat16() for s in ((r, p), (p, f), (p, f), (f, c), (r, c)))
    before = torch.cuda.memory_allocated()
    block = B.GatedBlock(p, f, c, r)
    assert torch.cuda.memory_allocated() > before
    block.forward(x, gate, up, down, y)
    block.close()
    assert torch.cuda.memory_allocated() == before
    with pytest.raises(B.BmgdError) as e:
        block.forward(x, gate, up, down, y)
    assert e.value.code == B.BMGD_EINVAL
    block.close()
