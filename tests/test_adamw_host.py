"""What ll_grad_norm and ll_adamw refuse, before anything touches the GPU (no GPU needed)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.test_learn_host import ROOT, fake

AT = 1 << 20


def tensors(**kw):
    t = dict(param=AT, grad=AT, m=AT, v=AT, m_scale=None, v_scale=None, copy=None, n=100, flags=0)
    t.update(kw)
    return (LL.ll_tensor * 2)(LL.ll_tensor(*[dict(t, flags=0)[n] for n, _ in LL.ll_tensor._fields_]) if not kw else LL.ll_tensor(),
                              LL.ll_tensor(*[t[n] for n, _ in LL.ll_tensor._fields_]))


def options(**kw):
    o = dict(rate=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.01, max_norm=1.0, step=1, seed=0)
    o.update(kw)
    return LL.ll_adamw_options(*[o[n] for n, _ in LL.ll_adamw_options._fields_])


def at(x):
    return None if x is None else ctypes.addressof(x)


def step(list_=None, count=2, opt=None, norm=None, clock=None, device_rate=None):
    return LL.lib().ll_adamw(at(list_), count, at(opt), norm, clock, device_rate, None)


def test_the_structs_are_the_headers():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ll.h")).read(), flags=re.S)
    for name, struct in (("ll_tensor", LL.ll_tensor), ("ll_adamw_options", LL.ll_adamw_options)):
        body = re.search(r"typedef struct " + name + r" \{(.*?)\} " + name, text, re.S).group(1)
        names = [n.strip(" *") for line in body.split(";") if line.strip() for n in re.sub(r"^\s*(const\s+)?\w+", "", line, count=1).split(",")]
        assert names == [n for n, _ in struct._fields_], names
    assert int(re.search(r"#define\s+LL_STATE_BLOCK\s+(\d+)", text).group(1)) == LL.LL_STATE_BLOCK
    for n in ("PARAM_BF16", "GRAD_BF16", "STATE_8BIT"):
        assert int(re.search(rf"#define\s+LL_TENSOR_{n}\s+(\d+)u", text).group(1)) == getattr(LL, "LL_TENSOR_" + n)


@pytest.mark.parametrize("kw", [dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param=AT + 8), dict(grad=AT + 8), dict(m=AT + 4),
                                dict(v=AT + 8), dict(copy=AT + 8), dict(n=-1), dict(n=2 ** 33 + 1), dict(flags=8), dict(flags=1 << 31), dict(m_scale=AT),
                                dict(v_scale=AT), dict(flags=4), dict(flags=4, m_scale=AT), dict(flags=4, v_scale=AT),
                                dict(flags=4, m_scale=AT + 2, v_scale=AT), dict(flags=1, copy=AT)])
def test_tensors(kw):
    assert step(tensors(**kw), opt=options()) == LL.LL_EINVAL


def test_arguments():
    nan, inf = float("nan"), float("inf")
    good = tensors()
    for bad in (dict(rate=-1.0), dict(rate=nan), dict(rate=inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=nan), dict(beta2=1.0), dict(beta2=nan),
                dict(eps=0.0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(eps=1e-60), dict(decay=-1.0), dict(decay=nan), dict(decay=inf),
                dict(step=0), dict(step=-3)):
        assert step(good, opt=options(**bad)) == LL.LL_EINVAL, bad
    assert step(None, opt=options()) == step(good) == step(good, count=-1, opt=options()) == LL.LL_EINVAL
    assert step(good, opt=options(), device_rate=fake()) == LL.LL_EINVAL                # needs a clock
    assert step(good, opt=options(), clock=fake(AT + 4)) == step(good, opt=options(), norm=fake(AT + 2)) == LL.LL_EINVAL
    assert step(good, opt=options(), clock=fake(), device_rate=fake(AT + 2)) == LL.LL_EINVAL
    for most in (0.0, -1.0, nan):
        assert step(good, opt=options(max_norm=most), norm=fake()) == LL.LL_EINVAL
    assert step(None, count=0, opt=options()) == LL.LL_OK
    assert step(tensors(n=0, param=None, grad=None, m=None, v=None), opt=options()) == LL.LL_OK     # nothing in it


def test_norm():
    call = lambda list_, *a: LL.lib().ll_grad_norm(at(list_), *a)  # noqa: E731
    need = LL.lib().ll_grad_norm_workspace_bytes(2)
    assert need > 0 and need % 256 == 0 and LL.lib().ll_grad_norm_workspace_bytes(-1) == 0
    assert LL.lib().ll_grad_norm_workspace_bytes(1000) > need
    good = tensors()
    assert call(good, 2, fake(), need, None, None) == call(good, 2, fake(), need, fake(AT + 2), None) == call(None, 2, fake(), need, fake(), None) == LL.LL_EINVAL
    assert call(good, -1, fake(), need, fake(), None) == LL.LL_EINVAL
    for kw in (dict(grad=None), dict(grad=AT + 8), dict(n=-1), dict(flags=64)):
        assert call(tensors(**kw), 2, fake(), need, fake(), None) == LL.LL_EINVAL, kw
    assert call(good, 2, None, need, fake(), None) == call(good, 2, fake(), need - 1, fake(), None) == call(good, 2, fake(AT + 128), need, fake(), None) == LL.LL_EWORKSPACE


def test_the_binding_checks_before_it_calls():
    x = torch.zeros((4, 4))
    with pytest.raises(TypeError):
        LL.TensorList([x])
    with pytest.raises(TypeError):
        LL.ll_adamw([x], 1)
    with pytest.raises(ValueError):
        LL.TensorList([], params=[x])
    assert ctypes.sizeof(LL.ll_tensor) == 72
