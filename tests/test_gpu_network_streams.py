"""Work of the gated block and of the AdamW step on streams: what follows what."""
import pytest

from test_gpu_gated import _check_forward, _data, _empty, _types

pytestmark = pytest.mark.gpu


def _busy(stream, times=100):
    """Keeps a stream at work for some hundred milliseconds."""
    import torch
    with torch.cuda.stream(stream):
        m = torch.randn(4096, 4096, device="cuda")
        for _ in range(times):
            m = m @ m * 1e-3


def _marker(stream):
    import torch
    e = torch.cuda.Event()
    e.record(stream)
    return e


def test_a_captured_call_does_not_come_between_the_calls_around_it():
    """A call behind a busy stream, one captured on a second stream, one on a third: the third ends after the first, and the graph gives the right results too."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    r, p, f, c = 200, 1500, 64, 100                            # (several workgroups share a tile's sum)
    s1, s2, s3 = (torch.cuda.Stream() for _ in range(3))
    with B.GatedBlock(p, f, c, r, dtype=code) as block:
        sets = [_data(r, p, f, c, dtype, seed) for seed in (1, 2, 3)]
        ys = [_empty(r, c, dtype) for _ in sets]
        block.forward(*sets[2], ys[2], stream=s2)
        torch.cuda.synchronize()
        ys[2].fill_(7.0)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        _busy(s1)
        block.forward(*sets[0], ys[0], stream=s1)
        first = _marker(s1)
        with torch.cuda.stream(s2):
            graph.capture_begin(capture_error_mode="relaxed")
            block.forward(*sets[2], ys[2], stream=s2)
            graph.capture_end()
        block.forward(*sets[1], ys[1], stream=s3)
        _marker(s3).synchronize()
        assert first.query()
        torch.cuda.synchronize()
        assert (ys[2] == 7.0).all()
        graph.replay()
        torch.cuda.synchronize()
        for data, y in zip(sets, ys):
            _check_forward("bf16", "silu", *data, y)


def test_a_call_on_another_stream_ends_after_the_one_before():
    """The first call stands behind a busy stream, the second reads what it writes, on a stream that has nothing else to wait for."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    r, n, f = 300, 64, 512
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    with B.GatedBlock(n, f, n, r, dtype=code) as block:
        x, gate, up, down = _data(r, n, f, n, dtype, 1)
        y, z = _empty(r, n, dtype), _empty(r, n, dtype)
        torch.cuda.synchronize()
        _busy(s1)
        block.forward(x, gate, up, down, y, stream=s1)
        first = _marker(s1)
        block.forward(y, gate, up, down, z, stream=s2)
        _marker(s2).synchronize()
        assert first.query()
        torch.cuda.synchronize()
        _check_forward("bf16", "silu", x, gate, up, down, y)
        _check_forward("bf16", "silu", y, gate, up, down, z)


def test_calls_run_on_the_current_stream():
    """Operands are made on a busy stream that is current; what is called there without a stream follows, and what comes behind reads its results."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    r, p, f, c = 100, 64, 128, 72
    x, gate, up, down = _data(r, p, f, c, dtype, 1)
    late, y, g, u = torch.zeros_like(x), _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
    out = _empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)
    want = [t.clone() for t in (y, g, u, *out)]
    masters, grads = [[torch.randn(1000, device="cuda"), torch.randn(30, device="cuda")] for _ in range(2)]
    zeros = [torch.zeros_like(t) for t in grads]
    thetas, refs = [t.clone() for t in masters], [t.clone() for t in masters]
    s = torch.cuda.Stream()
    with B.GatedBlock(p, f, c, r, dtype=code) as block:
        opts = [B.AdamW(t, z, state_bits=8) for t, z in ((thetas, zeros), (refs, grads))]
        block.forward(x, gate, up, down, *want[:3])
        block.backward(want[0], x, gate, up, down, *want[1:])
        opts[1].step()
        moments = opts[1].moments()
        torch.cuda.synchronize()
        _busy(s)
        with torch.cuda.stream(s):
            late.copy_(x)
            for z, t in zip(zeros, grads):
                z.copy_(t)
            block.forward(late, gate, up, down, y, g, u)
            block.backward(y, late, gate, up, down, g, u, *out)
            opts[0].step()
            values = [tuple(torch.full_like(t, 7.0) for _ in range(2)) for t in thetas]
            opts[0].moments(out=values)
            found = [t.clone() for t in (y, g, u, *out, *thetas, *sum(values, ()))]
        torch.cuda.synchronize()
    for a, b in zip(found, (*want, *refs, *sum(moments, ()))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_that_the_optimizer_makes_are_there_for_steps_on_any_stream(bits):
    """The constructor's fills stand behind a busy stream: it returns when they are done, and a step on another stream finds zeros."""
    import torch
    import paper_2312_08728_amd as B
    home, other = torch.cuda.Stream(), torch.cuda.Stream()
    theta, grad = torch.randn(100_000, device="cuda"), torch.randn(100_000, device="cuda")
    want = theta.clone()
    B.AdamW([want], [grad], state_bits=bits).step()
    torch.cuda.synchronize()
    _busy(home)
    with torch.cuda.stream(home):
        opt = B.AdamW([theta], [grad], state_bits=bits)
    assert home.query()
    opt.step(stream=other)
    torch.cuda.synchronize()
    assert torch.equal(theta, want)


def test_moments_that_the_optimizer_made_are_not_given_away_under_a_step():
    """The optimizer is dropped while its step stands behind a busy stream: the moments' memory is not free yet for the stream that they were made on."""
    import torch
    import paper_2312_08728_amd as B
    other, n = torch.cuda.Stream(), 3_000_000
    theta, grad = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    opt = B.AdamW([theta], [grad])
    torch.cuda.synchronize()
    _busy(other)
    opt.step(stream=other)
    end = _marker(other)
    places = {t.data_ptr() for t in opt.state[0]}
    del opt
    new = [torch.empty(n, device="cuda") for _ in range(4)]
    assert not end.query() and not places & {t.data_ptr() for t in new}
    torch.cuda.synchronize()


def test_values_of_moments_go_to_memory_that_nothing_else_uses():
    """New results of a call on another stream lie where work of the current one may still write: they wait for it, and their memory stays theirs until they are made."""
    import torch
    import paper_2312_08728_amd as B
    home, other, n = torch.cuda.Stream(), torch.cuda.Stream(), 3_000_000
    theta, grad = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    opt = B.AdamW([theta], [grad], state_bits=8)
    opt.step()
    want = opt.moments()
    torch.cuda.synchronize()
    with torch.cuda.stream(home):
        late = [torch.empty(n, device="cuda") for _ in range(2)]
        _busy(home)
        for t in late:
            t.fill_(3.0)
        filled = _marker(home)
        del late, t                                            # (their memory is free for what is made on this stream next)
        found = opt.moments(stream=other)
        _marker(other).synchronize()
        assert filled.query()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(found[0], want[0]))
    _busy(other)
    with torch.cuda.stream(home):
        dropped = opt.moments(stream=other)
        end = _marker(other)
        places = {t.data_ptr() for t in dropped[0]}
        del dropped
        new = [torch.empty(n, device="cuda") for _ in range(4)]
    assert not end.query() and not places & {t.data_ptr() for t in new}
    torch.cuda.synchronize()
