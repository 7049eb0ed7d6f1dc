"""What the operators that learn through the lens refuse, before anything touches the GPU (no GPU needed)."""
import ctypes
import os
import re

import pytest

from paper_2604_06483_amd import binding as LL

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def fake(n=1 << 20):
    return ctypes.c_void_p(n)        # a non-null, 256-byte aligned address that is never dereferenced


def refuser(fn, names, ok):
    def call(**kw):
        a = dict(ok, **kw)
        return fn(*[a[n] for n in names])
    return call


NORM = "shape hidden y gate gate_rows scale gamma_y gamma eps out_hidden out_normed stream".split()
NORM_GRAD = ("shape ws wsb hidden y gate gate_rows scale gamma_y gamma eps g_hidden g_normed d_hidden d_y d_gate d_gamma_y d_gamma "
             "stream").split()
LOGP = "shape ws wsb rows W temperature k ids logp lse entropy stream".split()
LOGP_GRAD = "shape ws wsb rows W temperature k ids lse entropy g_logp g_entropy grad stream".split()
DISTILL = "shape ws wsb rows W temperature k ids scores weight loss grad stream".split()


def norm_ok():
    ok = {n: fake() for n in NORM_GRAD + NORM}
    ok.update(shape=LL.ll_shape(16, 64, 0), wsb=1 << 40, gate_rows=0, scale=1.0, eps=1e-5, stream=None)
    return ok


def lens_ok():
    ok = {n: fake() for n in LOGP + LOGP_GRAD + DISTILL}
    ok.update(shape=LL.ll_shape(16, 64, 300), wsb=1 << 40, temperature=1.0, k=4, stream=None)
    return ok


def test_block_norm():
    call = refuser(LL.lib().ll_block_norm, NORM, norm_ok())
    for n in ("shape", "hidden", "y", "gamma", "out_hidden", "out_normed"):
        assert call(**{n: None}) == LL.LL_EINVAL, n
    for n in ("hidden", "y", "gate", "gamma_y", "gamma", "out_hidden", "out_normed"):
        assert call(**{n: fake((1 << 20) + 8)}) == LL.LL_EINVAL, n
    for N, d in ((-1, 64), (2 ** 31, 64), (16, 0), (16, 60), (16, -64), (16, 16392)):
        assert call(shape=LL.ll_shape(N, d, 0)) == LL.LL_EINVAL, (N, d)
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(gate_rows=2), dict(gate=None, gate_rows=1)):
        assert call(**bad) == LL.LL_EINVAL, bad
    assert call(shape=LL.ll_shape(0, 64, 0), hidden=None, y=None, out_hidden=None) == LL.LL_OK


def test_block_norm_grad():
    call = refuser(LL.lib().ll_block_norm_grad, NORM_GRAD, norm_ok())
    for n in ("shape", "hidden", "y", "gamma", "g_normed", "d_hidden", "d_y", "d_gamma", "d_gate", "d_gamma_y"):
        assert call(**{n: None}) == LL.LL_EINVAL, n
    for n in ("gate", "gamma_y"):           # a gradient of what is not there
        assert call(**{n: None}) == LL.LL_EINVAL, n
    for n in ("hidden", "y", "gate", "gamma_y", "gamma", "g_hidden", "g_normed", "d_hidden", "d_y", "d_gate", "d_gamma_y", "d_gamma"):
        assert call(**{n: fake((1 << 20) + 8)}) == LL.LL_EINVAL, n
    need = LL.ll_block_norm_grad_workspace_bytes(16, 64)
    assert need > 0 and need % 256 == 0
    assert call(ws=None) == call(wsb=need - 1) == call(ws=fake((1 << 20) + 128)) == LL.LL_EWORKSPACE
    assert LL.ll_block_norm_grad_workspace_bytes(16, 60) == LL.ll_block_norm_grad_workspace_bytes(-1, 64) == 0
    # no more for a million rows than for as many as there are workgroups
    assert LL.ll_block_norm_grad_workspace_bytes(10 ** 6, 64) == LL.ll_block_norm_grad_workspace_bytes(10 ** 7, 64)


@pytest.mark.parametrize("name,names,required,aligned", [
    ("ll_logp", LOGP, "rows W ids logp lse entropy", "rows W"),
    ("ll_logp_grad", LOGP_GRAD, "rows W ids lse entropy g_logp grad", "rows W grad"),
    ("ll_distill", DISTILL, "rows W ids scores loss", "rows W grad"),
])
def test_lens_calls(name, names, required, aligned):
    call = refuser(getattr(LL.lib(), name), names, lens_ok())
    for n in ["shape"] + required.split():
        assert call(**{n: None}) == LL.LL_EINVAL, n
    for n in aligned.split():
        assert call(**{n: fake((1 << 20) + 8)}) == LL.LL_EINVAL, n
    for n in set(names) - {"shape", "ws", "wsb", "temperature", "k", "stream"}:
        assert call(**{n: fake((1 << 20) + 2)}) == LL.LL_EINVAL, n
    for N, d, V in ((-1, 64, 300), (2 ** 31, 64, 300), (16, 0, 300), (16, 60, 300), (16, 65544, 300), (16, 64, 0), (16, 64, -5), (16, 64, 2 ** 22 + 1), (16, 64, 2 ** 31 - 1)):
        assert call(shape=LL.ll_shape(N, d, V)) == LL.LL_EINVAL, (N, d, V)
        assert getattr(LL, name + "_workspace_bytes")(N, d, V, 4) == 0
    for k in (0, -1, LL.LL_LIST_MAX + 1):
        assert call(k=k) == LL.LL_EINVAL
        assert getattr(LL, name + "_workspace_bytes")(16, 64, 300, k) == 0
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        assert call(temperature=t) == LL.LL_EINVAL, t
    need = getattr(LL, name + "_workspace_bytes")(16, 64, 300, 4)
    assert need > 0 and need % 256 == 0
    assert call(ws=None) == call(wsb=need - 1) == call(ws=fake((1 << 20) + 128)) == LL.LL_EWORKSPACE
    assert call(shape=LL.ll_shape(0, 64, 300), rows=None, W=None, ws=None, wsb=0) == LL.LL_OK


def test_workspaces_do_not_grow_past_a_pass():
    for size in (LL.ll_logp_workspace_bytes, LL.ll_logp_grad_workspace_bytes, LL.ll_distill_workspace_bytes):
        assert size(10 ** 6, 4096, 128256, 20) <= 1.01 * max(size(n, 4096, 128256, 20) for n in (1024, 1500, 1536, 2000, 2048))
        assert size(1, 4096, 128256, 20) < size(2048, 4096, 128256, 20)


def test_the_binding_checks_before_it_calls():
    import torch
    cpu = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        LL.ll_block_norm(cpu, cpu, cpu[0], 1e-5)
    with pytest.raises(TypeError):
        LL.ll_logp(cpu, cpu, torch.zeros((4, 2), dtype=torch.int32))
    with pytest.raises(TypeError):
        LL.ll_distill(cpu, cpu, torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)))


def test_header_constant_matches_binding():
    text = open(os.path.join(ROOT, "include", "ll.h")).read()
    assert int(re.search(r"#define\s+LL_LIST_MAX\s+(\d+)", text).group(1)) == LL.LL_LIST_MAX
