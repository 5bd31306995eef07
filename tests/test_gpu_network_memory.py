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


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_follow_tensors_that_are_given_other_memory(bits):
    """`t.data = ...` and tensors replaced in their lists: the step reads and writes where they are now, nothing where they were."""
    import torch
    import paper_2312_08728_amd as B
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    masters, sizes = [new(700), new(33)], (700, 33)
    grads = [[new(n) for n in sizes] for _ in range(2)]
    want, copies_want = [t.clone() for t in masters], [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes]
    ref = B.AdamW(want, grads[0], copies_want, state_bits=bits)
    thetas, copies, mine = [t.clone() for t in masters], [torch.zeros_like(t) for t in copies_want], [t.clone() for t in grads[0]]
    opt = B.AdamW(thetas, mine, copies, state_bits=bits)
    for o in (ref, opt):
        o.step()
    old = [t.data for t in (*thetas, *copies, *mine, *opt.state[0])]
    for t in (*thetas, *copies):
        t.data = t.data.clone()
    mine[0].data = grads[1][0].clone()
    opt.grads[1] = grads[1][1].clone()
    opt.state[0] = tuple(t.clone() for t in opt.state[0])
    before = [t.clone() for t in old]
    ref.set_grads(grads[1])
    for o in (ref, opt):
        o.step()
    assert all(torch.equal(a, b) for a, b in zip((*thetas, *copies), (*want, *copies_want)))
    assert all(torch.equal(a, b) for a, b in zip(old, before))
    for a, b in zip(opt.moments(), ref.moments()):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    thetas[0].data = thetas[0].data[:600]
    with pytest.raises(ValueError, match="theta"):
        opt.step()
    thetas[0].data = want[0].double()
    with pytest.raises(ValueError, match="theta"):
        opt.step()
    assert opt.steps == 2


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_that_overlap_are_refused(bits):
    """What a step writes it writes once: a tensor listed twice, or one that lies in another or in a gradient, would be updated in no order."""
    import torch
    import paper_2312_08728_amd as B
    flat, grads = torch.zeros(2000, device="cuda"), [torch.ones(600, device="cuda") for _ in range(2)]
    half = torch.zeros(2000, dtype=torch.bfloat16, device="cuda")

    def state(n):
        kinds = (torch.float32,) * 2 if bits == 32 else (torch.int8, torch.uint8, torch.float32, torch.float32)
        return tuple(torch.zeros(n if i < 2 else 3, dtype=k, device="cuda") for i, k in enumerate(kinds))

    one, two = state(600), state(600)
    apart = [flat[:600], flat[600:1200]]
    bad = [dict(thetas=[flat[:600]] * 2), dict(thetas=[flat[:600], flat[599:1199]]), dict(copies=[half[:600], half[500:1100]]), dict(state=[one, one]),
           dict(state=[one, (*two[:-1], one[-1])]), dict(grads=[grads[0], flat[1199:1799]]), dict(copies=[half[:600], flat[300:900].view(torch.bfloat16)[:600]])]
    for kw in bad:
        opt = B.AdamW(**{**dict(thetas=apart, grads=grads, state_bits=bits), **kw})
        with pytest.raises(B.BmgdError, match="overlap") as e:
            opt.step()
        assert e.value.code == B.BMGD_EINVAL and opt.steps == 0 and (flat == 0).all()
    opt = B.AdamW(apart, [grads[0]] * 2, [half[:600], half[600:1200]], state_bits=bits)              # gradients are read only: these may be one
    opt.step()
    assert (flat[:1200] != 0).all() and torch.equal(flat[:600], flat[600:1200])
    opt.thetas[1].data = flat[100:700]
    with pytest.raises(B.BmgdError, match="overlap"):
        opt.step()
    B.AdamW([flat[:0], flat[:0], flat[:5]], [flat[:0], flat[:0], flat[5:10]], state_bits=bits).step()    # nothing overlaps with no elements


def test_autograd_notices_what_the_calls_write():
    """A value that a graph of torch's has kept, overwritten by the block or by a step, is refused in its backward pass."""
    import torch
    import paper_2312_08728_amd as B
    p, f, c, r = 16, 24, 8, 4
    x, gate, up, down = (torch.randn(s, device="cuda").bfloat16() for s in ((r, p), (p, f), (p, f), (f, c)))
    y, g, u = (torch.zeros(r, n, device="cuda", dtype=torch.bfloat16) for n in (c, f, f))
    theta = torch.ones(50, device="cuda", requires_grad=True)
    opt = B.AdamW([theta], [torch.ones(50, device="cuda")])
    w = torch.ones(r, c, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    with B.GatedBlock(p, f, c, r) as block:
        kept = (w * y).sum()
        block.forward(x, gate, up, down, y, g, u)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            kept.backward()
        dx = torch.zeros_like(x)
        before = [t._version for t in (x, gate, up, down, g, u, y, dx)]
        block.backward(y, x, gate, up, down, g, u, dx=dx)
        assert [t._version for t in (x, gate, up, down, g, u, y, dx)] == [*before[:-1], before[-1] + 1]
    kept = (theta * theta).sum()
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward()
