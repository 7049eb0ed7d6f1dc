"""The checks of test_isa_checks.py on the kernels that learn through the lens: M0 is the LDS base setter's alone, nothing goes to scratch."""
import re

import pytest

from tests import test_isa_checks as T

pytestmark = T.pytestmark


@pytest.fixture(scope="module")
def gemm(tmp_path_factory):
    return T.assembly("ll_learn_gemm", tmp_path_factory.mktemp("isa"))


def metadata(asm):
    found = {}
    for m in re.finditer(r"\.name:\s+(\S+)\n(.*?)\.wavefront_size", asm, re.S):
        get = lambda key: int(re.search(r"\." + key + r":\s+(\d+)", m.group(2)).group(1))
        found[m.group(1)] = dict(vgpr=get("vgpr_count"), scratch=get("private_segment_fixed_size"), spill=get("vgpr_spill_count"))
    return found


# statistics, exponentials and the logits' gradient, for one to four row tiles, of whole stages through and past the caches and of ragged
# ones; the product backwards for the row tiles, through and past the caches
@pytest.mark.parametrize("kernel,count", [("ll_learn_logits_kernel", 36), ("ll_learn_back_kernel", 8)])
def test_products(gemm, kernel, count):
    parts = gemm.split(".Lfunc_end")
    bodies = T.kernel_bodies("\n\ts_endpgm\n.Lfunc_end".join(x.replace("s_endpgm", "s_nop 0") for x in parts), kernel)   # (whole functions)
    assert len(bodies) == count, sorted(bodies)
    for name, ins in bodies.items():
        ins = [l for l in (l.split(";")[0].strip() for l in ins) if l]
        assert sum(l.startswith("global_load_lds_dwordx4") for l in ins) >= 20 + 2 * 8
        for i, l in enumerate(ins):
            if "m0" in l:
                assert re.fullmatch(r"s_mov_b32 m0, s\d+", l) and ins[i + 1].startswith("s_nop"), (name, l)
            assert not l.split()[0].startswith(("v_movrel", "s_movrel", "s_sendmsg", "ds_gws", "s_set_gpr_idx")), (name, l)
    kernels = {n: m for n, m in metadata(gemm).items() if kernel in n}
    assert len(kernels) == count
    for name, m in kernels.items():
        assert m["vgpr"] <= 512 and m["scratch"] == 0 and m["spill"] == 0, (name, m)


def test_the_product_backwards_reads_its_fragments_transposed(gemm):
    """A stage's 32 fragments of W are two transposed reads each, in the first stage and in the loop, and eight more ahead of them; of A come
    two fragments a row tile and half."""
    bodies = T.kernel_bodies(gemm, "ll_learn_back_kernelILi4E")
    assert len(bodies) == 2
    for name, ins in bodies.items():
        assert sum(l.startswith("ds_read_b64_tr_b16") for l in ins) == 2 * (2 * 32 + 8), name
        assert sum(l.startswith("v_mfma_f32_16x16x32_bf16") for l in ins) == 2 * 128, name


def test_few_rows(tmp_path):
    kernels = {n: m for n, m in metadata(T.assembly("ll_learn_few", tmp_path)).items() if "ll_learn_few_kernel" in n}
    # statistics for one, two, four and eight rows, the others for up to four: the groups of small d, and one, two and four chunks
    assert len(kernels) == (6 + 6 + 5 + 2) + 2 * (6 + 6 + 5)
    for name, m in kernels.items():
        assert m["vgpr"] <= 256 and m["scratch"] == 0 and m["spill"] == 0, (name, m)
