"""What the gated block and the AdamW step refuse before they touch a GPU."""
import ctypes
import os
import re

import pytest

import paper_2312_08728_amd as B

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "bmgd.h")


@pytest.mark.parametrize("name", ["bmgd_gated_config", "bmgd_gated_tensors", "bmgd_adamw_tensor", "bmgd_adamw_config", "bmgd_matrix"])
def test_struct_layouts_match_header_order(name):
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), open(HEADER).read(), flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    assert re.findall(r"\b(\w+);", body) == [f[0] for f in getattr(B, name)._fields_]


def _cfg(**kw):
    c = B.bmgd_gated_config(100, 200, 30, 50, B.BMGD_BF16, B.BMGD_ACT_SILU, None, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_block_sizes_and_arguments():
    base = B.bmgd_gated_workspace_bytes(_cfg())
    assert base > 0 and base % 256 == 0 and B.bmgd_gated_workspace_bytes(_cfg(max_rows=5000)) > base + 4950 * 3 * 2 * 200
    bad = [dict(p=0), dict(hidden=0), dict(out_n=0), dict(max_rows=0), dict(max_rows=1 << 30), dict(p=(1 << 20) + 1), dict(hidden=-5), dict(dtype=B.BMGD_F32),
           dict(dtype=9), dict(activation=3), dict(activation=-1), dict(max_rows=(1 << 30) - 1, p=1 << 20)]
    for kw in bad:
        assert B.bmgd_gated_workspace_bytes(_cfg(**kw)) == 0, kw
        rc, h = B.bmgd_gated_create(_cfg(**kw))
        assert rc == B.BMGD_EINVAL and h is None and "bmgd_gated_create" in B.bmgd_last_error(None), kw
    assert B.bmgd_gated_create(_cfg(workspace=8, workspace_bytes=1 << 40))[0] == B.BMGD_EINVAL
    assert B.bmgd_gated_create(_cfg(workspace=256, workspace_bytes=base - 1))[0] == B.BMGD_ENOMEM
    assert B.lib.bmgd_gated_create(None, None) == B.BMGD_EINVAL
    t = B.bmgd_gated_tensors()
    assert B.bmgd_gated_forward(None, 1, t) == B.BMGD_EINVAL and B.bmgd_gated_backward(None, 1, t) == B.BMGD_EINVAL
    assert "block must not be NULL" in B.bmgd_gated_last_error(None)
    B.bmgd_gated_destroy(None)                  # ignored


def test_no_block_without_a_gpu():
    import torch
    if torch.cuda.is_available():
        return
    rc, h = B.bmgd_gated_create(_cfg())
    assert rc == B.BMGD_EHIP and h is None


def test_step_arguments():
    t = (B.bmgd_adamw_tensor * 1)()
    t[0].n = 0
    ok = B.bmgd_adamw_default_config()
    assert (ok.lr, ok.beta1, ok.beta2, ok.eps, ok.weight_decay, ok.grad_scale, ok.state_bits) == (1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0, 32)
    assert B.bmgd_adamw_step(ok, t, 1, 1) == B.BMGD_OK and B.bmgd_adamw_step(ok, None, 0, 1) == B.BMGD_OK      # nothing to do
    for kw in (dict(lr=-1.0), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=float("nan")), dict(eps=-1e-9), dict(weight_decay=-1.0),
               dict(grad_scale=float("nan")), dict(grad_dtype=3), dict(copy_dtype=B.BMGD_F32), dict(state_bits=16), dict(state_bits=8, eps=0.0),
               dict(state_bits=8, eps=1e-60)):
        cfg = B.bmgd_adamw_default_config()
        for k, v in kw.items():
            setattr(cfg, k, v)
        assert B.bmgd_adamw_step(cfg, t, 1, 1) == B.BMGD_EINVAL and B.bmgd_last_error(None), kw
    assert B.bmgd_adamw_step(ok, t, 1, 0) == B.BMGD_EINVAL
    assert B.bmgd_adamw_step(ok, t, -1, 1) == B.BMGD_EINVAL and B.bmgd_adamw_step(ok, None, 1, 1) == B.BMGD_EINVAL
    assert B.lib.bmgd_adamw_step(None, t, 1, 1, None) == B.BMGD_EINVAL
    good = dict(theta=64, grad=64, copy=0, m=64, s=64, m_scale=64, s_scale=64, n=10)
    for bits, kw in ((32, dict(n=-1)), (32, dict(n=(1 << 38) + 1)), (32, dict(theta=0)), (32, dict(grad=0)), (32, dict(m=0)), (32, dict(s=0)), (32, dict(theta=66)),
                     (32, dict(grad=65)), (32, dict(copy=65)), (8, dict(m=65)), (8, dict(s=66)), (8, dict(m_scale=0)), (8, dict(s_scale=66))):
        cfg = B.bmgd_adamw_default_config()
        cfg.state_bits = bits
        for k, v in dict(good, **kw).items():
            setattr(t[0], k, v)
        assert B.bmgd_adamw_step(cfg, t, 1, 1) == B.BMGD_EINVAL and "tensor 0" in B.bmgd_last_error(None), kw
    for k, v in good.items():
        setattr(t[0], k, v)
    one = (ctypes.c_void_p * 1)(64)
    for m, s in ((None, one), (one, None), ((ctypes.c_void_p * 1)(0), one), (one, (ctypes.c_void_p * 1)(66))):
        assert B.bmgd_adamw_moments(t, 1, m, s) == B.BMGD_EINVAL


def test_an_internal_tile_is_checked():
    assert B.lib.bmgd_internal_gated_tile(None, 0, 1) == B.BMGD_EINVAL


def test_what_is_read_of_tensors():
    """Addresses and strides of matrices and of pairs, and the index of the first tensor that is not what was asked for."""
    import struct
    import torch
    from paper_2312_08728_amd import _tensors as T
    bf16 = torch.bfloat16
    a, b = torch.zeros(5, 8, dtype=bf16)[:, 1:4], torch.zeros(7, 1, dtype=bf16).expand(7, 1)
    one = torch.zeros(1, 6, dtype=bf16)
    got = T.matrices((a, None, b, one), ((5, 3), (1, 1), (7, 1), (1, 6)), bf16, -1)
    assert struct.unpack("8q", got) == (a.data_ptr(), 8, 0, 0, b.data_ptr(), b.stride(0), one.data_ptr(), one.stride(0))
    assert T.matrices((a, torch.zeros(4, 8, dtype=bf16).t()), ((5, 3), (8, 4)), bf16, -1) == 1             # elements of a row apart
    column = torch.zeros(4, 8, dtype=bf16)[:, :1]
    assert struct.unpack("2q", T.matrices((column,), ((4, 1),), bf16, -1)) == (column.data_ptr(), 8)
    for wrong in (a.float(), a[:4], a[0], a.reshape(3, 5), "no tensor", a.to("meta"), torch.zeros(5, 3, dtype=bf16).to_sparse()):
        assert T.matrices((one, wrong), ((1, 6), (5, 3)), bf16, -1) == 1
    assert T.matrices((a,), ((5, 3),), bf16, 0) == 0                                                          # of another device
    m, s = torch.zeros(10), torch.zeros(2, 5)
    assert T.pairs([(m, s), [s, m]], struct.pack("2q", 10, 10), torch.float32, -1) == (struct.pack("2q", m.data_ptr(), s.data_ptr()), struct.pack("2q", s.data_ptr(), m.data_ptr()))
    assert T.pairs([], b"", torch.float32, -1) == (b"", b"")
    for wrong in ((m, s[:1]), (m, s.t()), (m.double(), s), (m,), (m, s, s), m, None, (m, None)):
        assert T.pairs([(m, s), wrong], struct.pack("2q", 10, 10), torch.float32, -1) == 1
    assert T.vectors([m, s], struct.pack("2q", 10, 10), torch.float32, -1) == struct.pack("2q", m.data_ptr(), s.data_ptr()) and T.vectors([], b"", torch.float32, -1) == b""
    for wrong in (m[:9], s.t(), m.double(), m.to("meta"), None, (m,)):
        assert T.vectors([m, wrong, s], struct.pack("3q", 10, 10, 10), torch.float32, -1) == 1
    for call in (lambda: T.vectors((m,), bytes(8), torch.float32, -1), lambda: T.vectors([m], b"", torch.float32, -1), lambda: T.vectors([m], bytes(8), 3, -1)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: T.matrices((a,), (), bf16, -1), lambda: T.matrices([a], [(5, 3)], bf16, -1), lambda: T.matrices((a,), ((5, 3),), "bf16", -1), lambda: T.matrices((a,), (5,), bf16, -1),
                 lambda: T.matrices((a,), (("5", 3),), bf16, -1), lambda: T.matrices((a,)), lambda: T.pairs([(m, s)], b"", torch.float32, -1), lambda: T.pairs([(m, s)], bytes(8), torch.float32, None)):
        with pytest.raises(TypeError):
            call()
