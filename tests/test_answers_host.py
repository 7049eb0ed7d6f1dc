"""What the calls that learn from answers refuse, before anything touches the GPU (no GPU needed)."""
import os
import re

import pytest

from paper_2604_06483_amd import binding as LL
from tests.test_learn_host import ROOT, fake, refuser

POLICY = "shape ws wsb rows W temperature ids advantage old ref weight low high kl loss logp grad stream".split()
PREFERENCE = "shape ws wsb rows W temperature ids offsets pairs ref weight form mean beta smoothing loss score logp grad stream".split()
SCALARS = {"shape", "ws", "wsb", "temperature", "low", "high", "kl", "stream", "pairs", "form", "mean", "beta", "smoothing"}


def ok():
    a = {n: fake() for n in POLICY + PREFERENCE}
    a.update(shape=LL.ll_shape(16, 64, 300), wsb=1 << 40, temperature=1.0, low=0.2, high=0.2, kl=0.1, stream=None, pairs=3, form=0, mean=0,
             beta=0.1, smoothing=0.0)
    return a


@pytest.mark.parametrize("name,names,required,size", [
    ("ll_policy", POLICY, "rows W ids advantage loss logp", lambda N, d, V: LL.ll_policy_workspace_bytes(N, d, V)),
    ("ll_preference", PREFERENCE, "rows W ids offsets loss score logp", lambda N, d, V: LL.ll_preference_workspace_bytes(N, d, V, 3)),
])
def test_answer_calls(name, names, required, size):
    call = refuser(getattr(LL.lib(), name), names, ok())
    for n in ["shape"] + required.split():
        assert call(**{n: None}) == LL.LL_EINVAL, n
    for n in ("rows", "W", "grad"):
        assert call(**{n: fake((1 << 20) + 8)}) == LL.LL_EINVAL, n
    for n in set(names) - SCALARS:
        assert call(**{n: fake((1 << 20) + 2)}) == LL.LL_EINVAL, n
    for N, d, V in ((-1, 64, 300), (2 ** 31, 64, 300), (16, 0, 300), (16, 60, 300), (16, 65544, 300), (16, 64, 0), (16, 64, 2 ** 22 + 1)):
        assert call(shape=LL.ll_shape(N, d, V)) == LL.LL_EINVAL, (N, d, V)
        assert size(N, d, V) == 0
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        assert call(temperature=t) == LL.LL_EINVAL, t
    need = size(16, 64, 300)
    assert need > 0 and need % 256 == 0
    assert call(ws=None) == call(wsb=need - 1) == call(ws=fake((1 << 20) + 128)) == LL.LL_EWORKSPACE
    # without a gradient a smaller one does
    assert call(grad=None, wsb=LL.ll_logp_workspace_bytes(16, 64, 300, 1) - 1) == LL.LL_EWORKSPACE


def test_policy_arguments():
    call = refuser(LL.lib().ll_policy, POLICY, ok())
    nan, inf = float("nan"), float("inf")
    for bad in (dict(low=-0.1), dict(low=1.1), dict(low=nan), dict(high=-0.1), dict(high=nan), dict(kl=-0.1), dict(kl=nan), dict(kl=inf), dict(ref=None)):
        assert call(**bad) == LL.LL_EINVAL, bad
    assert call(shape=LL.ll_shape(0, 64, 300), rows=None, W=None, ids=None, ws=None, wsb=0) == LL.LL_OK


def test_preference_arguments():
    call = refuser(LL.lib().ll_preference, PREFERENCE, ok())
    nan, inf = float("nan"), float("inf")
    for bad in (dict(pairs=-1), dict(form=3), dict(form=-1), dict(mean=2), dict(beta=0.0), dict(beta=-1.0), dict(beta=nan), dict(beta=inf),
                dict(smoothing=-0.1), dict(smoothing=0.6), dict(smoothing=nan), dict(form=1, smoothing=0.1), dict(form=2, smoothing=0.1)):
        assert call(**bad) == LL.LL_EINVAL, bad
    assert call(shape=LL.ll_shape(0, 64, 300), rows=None, W=None, ids=None, ws=None, wsb=0, pairs=0, offsets=None, loss=None, score=None) == LL.LL_OK
    assert LL.ll_preference_workspace_bytes(16, 64, 300, -1) == 0


def test_the_sums_that_pairs_keep_grow_with_the_rows():
    """Past one pass of 2048 rows every pass's fp32 sums are kept, and nothing else grows but 16 bytes a row."""
    d, V = 4096, 128256
    one, four = LL.ll_preference_workspace_bytes(2048, d, V, 4), LL.ll_preference_workspace_bytes(8192, d, V, 4)
    assert LL.ll_policy_workspace_bytes(2048, d, V) == one
    assert LL.ll_policy_workspace_bytes(8192, d, V) - one == 16 * (8192 - 2048)
    assert (four - one - 16 * (8192 - 2048)) % ((8192 - 2048) * d * 4) == 0 and four >= one + (8192 - 2048) * d * 4


def test_the_binding_checks_before_it_calls():
    import torch
    cpu = torch.zeros((4, 64), dtype=torch.bfloat16)
    ids = torch.zeros((4,), dtype=torch.int32)
    with pytest.raises(TypeError):
        LL.ll_policy(cpu, cpu, ids, torch.zeros((4,)))
    with pytest.raises(TypeError):
        LL.ll_preference(cpu, cpu, ids, torch.zeros((3,), dtype=torch.int32))
    with pytest.raises(ValueError):
        LL.ll_preference(cpu, cpu, ids, torch.zeros((3,), dtype=torch.int32), form="other")


def test_header_constants_match_the_binding():
    text = open(os.path.join(ROOT, "include", "ll.h")).read()
    for name, value in LL.LL_PREFERENCE.items():
        assert int(re.search(rf"#define\s+LL_PREFERENCE_{name.upper()}\s+(\d+)", text).group(1)) == value
