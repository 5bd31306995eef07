"""Operands of the gated block that are copied before the products: rows far apart."""
import ctypes

import numpy as np
import pytest

from test_gpu_gated import _check_backward, _check_forward, _data, _dev, _empty, _types

pytestmark = pytest.mark.gpu


def test_copies_of_rows_so_far_apart_that_offsets_pass_32_bits():
    """X and dY, 40 rows of 5.4 GB each that begin at odd places, and a kind of tile that cannot read these: element offsets beyond 2^31 in the kernel that copies."""
    import torch
    import paper_2312_08728_amd as B
    dtype, code = _types()["bf16"]
    r, p, f, c, stride = 40, 64, 72, 24, (1 << 26) + 3
    x, gate, up, down = _data(r, p, f, c, dtype, 3)
    dy = _dev(np.random.default_rng(4).standard_normal((r, c)), dtype)
    far = [torch.empty(39 * stride + n, dtype=dtype, device="cuda").as_strided((r, n), (stride, 1)) for n in (p, c)]
    far[0].copy_(x)
    far[1].copy_(dy)
    with B.GatedBlock(p, f, c, r, dtype=code) as block:
        assert B.lib.bmgd_internal_gated_tile(ctypes.c_void_p(block.h), 0, 1) == B.BMGD_OK        # the largest, which has no form for operands at any address
        y, g, u = _empty(r, c, dtype), _empty(r, f, dtype), _empty(r, f, dtype)
        block.forward(far[0], gate, up, down, y, g, u)
        _check_forward("bf16", "silu", x, gate, up, down, y, g, u)
        out = _empty(r, p, dtype), _empty(p, f, dtype), _empty(p, f, dtype), _empty(f, c, dtype)
        block.backward(far[1], far[0], gate, up, down, g, u, *out)
        _check_backward("bf16", "silu", dy, x, gate, up, down, g, u, *out)
    del far
    torch.cuda.empty_cache()
