"""Checks on the compiled kernels of answers and of a training step: nothing goes to scratch, loads and stores of a step are past the caches, and
the 8-bit states are rounded by the hardware's own stochastic conversions."""
import re

import pytest

from tests import test_isa_checks as T
from tests.test_isa_learn import metadata

pytestmark = T.pytestmark


@pytest.fixture(scope="module")
def step(tmp_path_factory):
    return T.assembly("ll_adamw", tmp_path_factory.mktemp("isa"))


def test_step(step):
    kernels = {n: m for n, m in metadata(step).items() if "ll_adamw_kernel" in n}
    assert len(kernels) == 8
    for name, m in kernels.items():
        assert m["vgpr"] <= 64 and m["scratch"] == 0 and m["spill"] == 0, (name, m)      # eight wavefronts a SIMD
        body = step[step.index(f"\n{name}:"):]
        body = body[:body.index(".Lfunc_end")]
        wide = re.findall(r"global_(?:load|store)_dwordx4.*", body)
        fp32, eight = "ILb0E" in name, name.split("ll_adamw_kernel")[1].startswith(("ILb0ELb0ELb1", "ILb0ELb1ELb1", "ILb1ELb0ELb1", "ILb1ELb1ELb1"))
        if fp32 or not eight:
            assert wide and all(" nt" in x for x in wide), (name, wide)
        assert not re.search(r"v_pk_(add|mul|fma)_f32", body)
        assert len(re.findall(r"v_cvt_sr_fp8_f32", body)) % 4 == 0 and bool(re.search("v_cvt_sr_fp8_f32", body)) == bool(re.search("v_cvt_sr_bf8_f32", body)) == eight


def test_norm(step):
    kernels = {n: m for n, m in metadata(step).items() if "ll_grad_norm" in n}
    assert len(kernels) == 3
    for name, m in kernels.items():
        assert m["vgpr"] <= 128 and m["scratch"] == 0 and m["spill"] == 0, (name, m)


def test_answers(tmp_path):
    kernels = {n: m for n, m in metadata(T.assembly("ll_answers", tmp_path)).items() if "ll_answers" in n or "ll_preference" in n}
    assert len(kernels) == 7 + 12                 # (16, 32 and 64 ids with one to four tiles of rows)
    for name, m in kernels.items():
        assert m["vgpr"] <= (256 if "logits" in name else 128) and m["scratch"] == 0 and m["spill"] == 0, (name, m)


def test_products_that_keep_the_others_sum(tmp_path):
    kernels = {n: m for n, m in metadata(T.assembly("ll_learn_gemm", tmp_path)).items() if "ll_learn_others_kernel" in n}
    assert len(kernels) == 12                     # one to four row tiles, of whole stages through and past the caches and of ragged ones
    for name, m in kernels.items():
        assert m["vgpr"] <= 512 and m["scratch"] == 0 and m["spill"] == 0, (name, m)
    kernels = {n: m for n, m in metadata(T.assembly("ll_learn_few", tmp_path)).items() if "ll_learn_few_others_kernel" in n}
    assert len(kernels) == 6 + 6 + 5
    for name, m in kernels.items():
        assert m["vgpr"] <= 256 and m["scratch"] == 0 and m["spill"] == 0, (name, m)
