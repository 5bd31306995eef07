"""What the norm, the 8-bit product and the log probabilities refuse before they touch a GPU."""
import ctypes as C
import os
import re

import pytest

import paper_2312_08728_amd as B

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "bmgd.h")
FAR = 1 << 32                                  # addresses that nothing reads


@pytest.mark.parametrize("name", ["bmgd_norm_config", "bmgd_norm_tensors", "bmgd_product_config", "bmgd_product_tensors", "bmgd_logprobs_config", "bmgd_logprobs_tensors"])
def test_struct_layouts_match_header_order(name):
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), open(HEADER).read(), flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    assert re.findall(r"\b(\w+);", body) == [f[0] for f in getattr(B, name)._fields_]


def _filled(kind, cols, vectors=(), **kw):
    """A call's tensors, each at an address of its own."""
    t = kind()
    for i, (name, of) in enumerate(kind._fields_):
        if name in kw:
            setattr(t, name, kw[name])
        elif of is B.bmgd_matrix:
            setattr(t, name, B.bmgd_matrix((i + 1) * FAR, cols))
        elif of is C.c_void_p:
            setattr(t, name, (i + 1) * FAR)
        else:
            setattr(t, name, 1 << 40)
    return t


def _at(n, stride=64):
    return B.bmgd_matrix(n, stride)


NONE = B.bmgd_matrix(0, 0)


def _refused(rc, *words, code=B.BMGD_EINVAL):
    assert rc == code, rc
    for w in words:
        assert w in B.bmgd_last_error(None), B.bmgd_last_error(None)


@pytest.mark.parametrize("call", [B.bmgd_norm_forward, B.bmgd_norm_backward])
def test_norm(call):
    ok = lambda **kw: B.bmgd_norm_config(kw.get("n", 64), kw.get("eps", 1e-6), kw.get("dtype", B.BMGD_BF16), 0)  # noqa: E731
    new = lambda **kw: _filled(B.bmgd_norm_tensors, 64, **kw)  # noqa: E731
    for kw in (dict(n=0), dict(n=-3), dict(n=(1 << 20) + 1), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=1e300), dict(dtype=3), dict(dtype=-1)):
        _refused(call(ok(**kw), 4, new()))
        assert B.bmgd_norm_workspace_bytes(ok(**kw), 4) == 0
    _refused(call(None, 4, new()), "NULL")
    _refused(call(ok(), 4, None), "NULL")
    _refused(call(ok(), -1, new()), "rows")
    _refused(call(ok(), 1 << 30, new()), "rows")
    _refused(call(ok(), 4, new(x=NONE)), "x:", "NULL")
    _refused(call(ok(), 4, new(x=_at(FAR + 1))), "x:", "multiple")
    _refused(call(ok(), 4, new(x=_at(FAR, 63))), "x:", "stride")
    _refused(call(ok(), 1 << 29, new(x=_at(FAR, 1 << 40))), "x:", "stride")
    _refused(call(ok(), 4, new(weight=FAR + 1)), "weight")
    _refused(call(ok(), 4, new(rstd=FAR + 2)), "rstd")
    assert call(ok(), 0, B.bmgd_norm_tensors()) == B.BMGD_OK


def test_norm_results_that_meet():
    cfg = B.bmgd_norm_config(64, 1e-6, B.BMGD_F16, 0)
    new = lambda **kw: _filled(B.bmgd_norm_tensors, 64, **kw)  # noqa: E731
    forward = lambda **kw: B.bmgd_norm_forward(cfg, 4, new(**kw))  # noqa: E731
    _refused(forward(y=NONE, codes=NONE), "wanted")
    _refused(forward(scales=None), "scales")
    _refused(forward(sum=_at(FAR), y=_at(FAR)), "sum")
    _refused(forward(codes=_at(FAR), x=_at(FAR)), "codes")
    _refused(forward(sum=_at(FAR, 65), x=_at(FAR, 64)), "stride")
    for kw in (dict(scales=50 * FAR, rstd=50 * FAR), dict(y=_at(50 * FAR), weight=50 * FAR), dict(sum=_at(50 * FAR), rstd=50 * FAR), dict(codes=_at(50 * FAR), scales=50 * FAR),
               dict(x=_at(50 * FAR), rstd=50 * FAR), dict(residual=_at(50 * FAR), scales=50 * FAR), dict(weight=50 * FAR, rstd=50 * FAR)):
        _refused(forward(**kw), "written")
    rows = 5000
    backward = lambda **kw: B.bmgd_norm_backward(cfg, rows, new(**kw))  # noqa: E731
    _refused(backward(dx=_at(FAR), x=_at(FAR)), "dx")
    _refused(backward(dx=_at(50 * FAR, 65), dy=_at(50 * FAR, 64)), "dx", "stride")
    _refused(backward(dweight=FAR, weight=FAR), "dweight")
    _refused(backward(dweight=50 * FAR, rstd=50 * FAR), "dweight")
    _refused(backward(rstd=None), "rstd")
    _refused(backward(workspace=None), "workspace")
    _refused(backward(workspace=FAR + 128), "workspace")
    need = B.bmgd_norm_workspace_bytes(cfg, rows)
    assert need and need % 256 == 0 and B.bmgd_norm_workspace_bytes(cfg, 1 << 29) >= need and B.bmgd_norm_workspace_bytes(cfg, 4) == 0
    _refused(backward(workspace_bytes=need - 1), "workspace", code=B.BMGD_ENOMEM)


def test_product():
    ok = lambda **kw: B.bmgd_product_config(kw.get("p", 64), kw.get("out_n", 64), kw.get("dtype", B.BMGD_BF16), 0)  # noqa: E731
    new = lambda **kw: _filled(B.bmgd_product_tensors, 64, **kw)  # noqa: E731
    call = B.bmgd_product_forward
    for kw in (dict(p=0), dict(p=131_072), dict(out_n=0), dict(out_n=(1 << 20) + 1), dict(dtype=9)):
        _refused(call(ok(**kw), 4, new()))
        _refused(B.bmgd_product_quantize(ok(**kw), _at(FAR), _at(2 * FAR), 3 * FAR))
    _refused(call(None, 4, new()), "NULL")
    _refused(call(ok(), 4, None), "NULL")
    _refused(call(ok(), -1, new()), "rows")
    for name in ("x", "w", "y"):
        _refused(call(ok(), 4, new(**{name: NONE})), name + ":", "NULL")
        _refused(call(ok(), 4, new(**{name: _at(FAR, 63)})), name + ":", "stride")
    for name in ("x_scales", "w_scales"):
        _refused(call(ok(), 4, new(**{name: None})), name)
        _refused(call(ok(), 4, new(**{name: FAR + 2})), name)
    _refused(call(ok(), 4, new(y=_at(FAR + 1))), "y:")
    _refused(call(ok(), 4, new(y=_at(FAR), x=_at(FAR))), "y:")
    _refused(call(ok(out_n=1 << 20), (1 << 30) - 1, _filled(B.bmgd_product_tensors, 1 << 20)), "tiles")
    assert call(ok(), 0, B.bmgd_product_tensors()) == B.BMGD_OK
    for args in ((NONE, _at(2 * FAR), 3 * FAR), (_at(FAR), NONE, 3 * FAR), (_at(FAR), _at(2 * FAR), 0), (_at(FAR), _at(FAR), 3 * FAR), (_at(FAR + 1), _at(2 * FAR), 3 * FAR),
                 (_at(FAR, 63), _at(2 * FAR), 3 * FAR), (_at(FAR), _at(2 * FAR, 63), 3 * FAR)):
        _refused(B.bmgd_product_quantize(ok(), *args), "bmgd_product_quantize")
    good = (4, 64, _at(FAR), 2 * FAR, _at(3 * FAR), B.BMGD_F32)
    for i, bad in ((0, -1), (0, 1 << 30), (1, 0), (1, (1 << 20) + 1), (2, NONE), (2, _at(FAR, 63)), (3, 0), (3, FAR + 1), (4, NONE), (4, _at(FAR)), (4, _at(2 * FAR)), (4, _at(3 * FAR + 2)), (5, 3)):
        _refused(B.bmgd_product_values(*good[:i], bad, *good[i + 1:]), "bmgd_product_values")
    assert B.bmgd_product_values(0, 64, NONE, 0, NONE, B.BMGD_F32) == B.BMGD_OK


@pytest.mark.parametrize("call", [B.bmgd_logprobs_forward, B.bmgd_logprobs_backward])
def test_logprobs(call):
    ok = lambda **kw: B.bmgd_logprobs_config(kw.get("classes", 64), kw.get("dtype", B.BMGD_BF16), kw.get("top", 4))  # noqa: E731
    new = lambda **kw: _filled(B.bmgd_logprobs_tensors, 64, **kw)  # noqa: E731
    for kw in (dict(classes=0), dict(classes=(1 << 24) + 1), dict(dtype=3), dict(top=-1), dict(top=65, classes=100), dict(classes=3)):
        _refused(call(ok(**kw), 4, new()))
        assert B.bmgd_logprobs_workspace_bytes(ok(**kw), 4) == 0
    _refused(call(None, 4, new()), "NULL")
    _refused(call(ok(), 4, None), "NULL")
    _refused(call(ok(), -1, new()), "rows")
    _refused(call(ok(), 4, new(logits=NONE)), "logits:")
    _refused(call(ok(), 4, new(logits=_at(FAR + 1))), "logits:")
    _refused(call(ok(), 4, new(logits=_at(FAR, 63))), "logits:")
    _refused(call(ok(), 4, new(labels=None)), "labels")
    _refused(call(ok(), 4, new(kept=FAR + 1)), "kept")
    assert call(ok(), 0, B.bmgd_logprobs_tensors()) == B.BMGD_OK


def test_logprobs_results():
    cfg = B.bmgd_logprobs_config(64, B.BMGD_F32, 4)
    new = lambda **kw: _filled(B.bmgd_logprobs_tensors, 64, **kw)  # noqa: E731
    for kw in (dict(top_classes=None), dict(top_logprobs=None), dict(top_classes=5 * FAR, top_logprobs=5 * FAR), dict(logprob=FAR, logits=_at(FAR)), dict(entropy=FAR + 2)):
        _refused(B.bmgd_logprobs_forward(cfg, 4, new(**kw)))
    for kw in (dict(dlogits=NONE), dict(kept=None), dict(dlogits=_at(50 * FAR, 65), logits=_at(50 * FAR)), dict(dlogits=_at(FAR), kept=FAR)):
        _refused(B.bmgd_logprobs_backward(cfg, 4, new(**kw)))
    wide = B.bmgd_logprobs_config(1 << 20, B.BMGD_F32, 64)
    need = B.bmgd_logprobs_workspace_bytes(wide, 2)
    assert need and need % 256 == 0 and B.bmgd_logprobs_workspace_bytes(wide, 100_000) == 0 and B.bmgd_logprobs_workspace_bytes(cfg, 2) == 0
    big = _filled(B.bmgd_logprobs_tensors, 1 << 20)
    for kw, code in ((dict(workspace=None), B.BMGD_EINVAL), (dict(workspace=FAR + 64), B.BMGD_EINVAL), (dict(workspace_bytes=need - 1), B.BMGD_ENOMEM)):
        for k, v in kw.items():
            setattr(big, k, v)
        _refused(B.bmgd_logprobs_forward(wide, 2, big), "workspace", code=code)
        big = _filled(B.bmgd_logprobs_tensors, 1 << 20)


def test_objects_refuse_sizes_and_types():
    for bad in (lambda: B.RMSNorm(0), lambda: B.RMSNorm(1 << 21), lambda: B.RMSNorm(8, dtype=7), lambda: B.RMSNorm(8, eps=-1.0), lambda: B.RMSNorm(8, eps=float("nan")),
                lambda: B.RMSNorm(8, eps=1e39), lambda: B.RMSNorm(8.5), lambda: B.Int8Product(131_072, 8), lambda: B.Int8Product(8, 0), lambda: B.Int8Product(8, 8, dtype="bf16"),
                lambda: B.LogProbs(0), lambda: B.LogProbs(10, top=11), lambda: B.LogProbs(100, top=65), lambda: B.LogProbs(100, top=-1), lambda: B.LogProbs(10, dtype=None)):
        with pytest.raises(ValueError):
            bad()


def test_tensors_on_the_host_are_refused():
    import torch
    x = torch.zeros(3, 8, dtype=torch.bfloat16)
    for call in (lambda: B.RMSNorm(8).forward(x, y=x), lambda: B.RMSNorm(8).backward(x, x, x, x, x), lambda: B.Int8Product(8, 8).forward(x, x, x, x, x), lambda: B.LogProbs(8).forward(x),
                 lambda: B.LogProbs(8).backward(x, x, x), lambda: B.RMSNorm(8).values(x, x, x), lambda: B.Int8Product(8, 8).quantize(x, x, x), lambda: B.LogProbs(8).forward(None)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_places_of_operands():
    """Addresses and strides as the calls take them; the first tensor that is another one is named; those written are told so."""
    import struct
    import torch
    from paper_2312_08728_amd import _tensors as T
    f, b = torch.float32, torch.int8
    m, v, c = torch.zeros(5, 10)[:, 2:9], torch.zeros(5), torch.zeros(5, 7, dtype=b)
    ask = lambda t, k=(f, f, b), s=((5, 7), (5,), (5, 7)), how=b"mvM": T.operands(t, k, s, how, -1)  # noqa: E731
    assert struct.unpack("5q", ask((m, v, c))) == (m.data_ptr(), 10, v.data_ptr(), c.data_ptr(), 7) and (m._version, v._version) == (0, 0) and c._version == 1
    assert struct.unpack("5q", ask((None, v, None))) == (0, 0, v.data_ptr(), 0, 0)
    for i, other in ((0, m.t()), (0, m.double()), (0, m[:4]), (0, m[0]), (1, torch.zeros(10)[::2]), (1, torch.zeros(5, 1)), (1, "v"), (2, v), (2, c.t().contiguous().t())):
        assert ask(tuple(other if i == k else t for k, t in enumerate((m, v, c)))) == i
    assert c._version == 1                                                                       # (nothing is written by a call that is refused)
    for bad in (lambda: ask([m, v, c]), lambda: ask((m, v)), lambda: ask((m, v, c), how=b"mv"), lambda: ask((m, v, c), s=((5, 7), 5, (5, 7))), lambda: ask((m, v, c), k=(f, f, "b")),
                lambda: T.operands((m,), (f,))):
        with pytest.raises(TypeError):
            bad()
