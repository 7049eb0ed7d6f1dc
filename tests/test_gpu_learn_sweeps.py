"""The products that learn through the lens where a workgroup sweeps several vocabulary tiles, for every number of row tiles."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.conftest import kernels_of, say
from tests.test_gpu_learn import check_distill, check_logp, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def splits_of(N, d, V, k):
    """Slices of the vocabulary, by the size of ll_logp's workspace: a row has 16 bytes for each, its k logits, a reference and the padded row."""
    up = lambda n: (n + 255) // 256 * 256
    rest = LL.ll_logp_workspace_bytes(N, d, V, k) - up(4 * N * k) - up(4 * N) - (up(2 * N * ((d + 63) // 64 * 64)) if d % 64 else 0)
    splits = rest // (16 * N)
    assert up(16 * N * splits) == rest
    return splits


# N, d, V, row tiles a wavefront; one to three row blocks, whole and ragged K stages
SWEEPS = [(40, 128, 140000, 1), (50, 136, 70000, 1), (100, 128, 140000, 2), (100, 136, 70000, 2), (180, 128, 70000, 3), (180, 136, 100000, 3), (250, 128, 70000, 4),
          (250, 136, 140000, 4), (348, 136, 70000, 3), (600, 128, 70000, 4), (600, 136, 40000, 4)]


@pytest.mark.parametrize("N,d,V,row_tiles", SWEEPS)
def test_several_tiles_a_workgroup(N, d, V, row_tiles):
    say(f"several tiles a workgroup N={N} d={d} V={V}")
    k = 6
    assert (V + 255) // 256 / splits_of(N, d, V, k) > 1.9
    a, W, ids, g = inputs(N, d, V, k)
    check_logp(a, W, ids, g, 0.7)
    scores, weight = 3 * torch.randn((N, k), generator=g), torch.rand((N,), generator=g)
    check_distill(a, W, ids, scores, weight, 2.0)
    cut = [x.to(DEV) for x in (a, W, ids, scores)]
    found = [n.split("(")[0] for n in kernels_of(lambda: (LL.ll_logp(*cut[:3]), LL.ll_distill(*cut)))]
    tail = "true" if d % 64 else "false"
    assert {n for n in found if "logits_kernel" in n or "back_kernel" in n} == {
        f"ll_learn_logits_kernel<{what}, {tail}, {row_tiles}, false>" for what in (0, 1)} | {f"ll_learn_back_kernel<{row_tiles}, false>"}, found


@pytest.mark.parametrize("N,d,V", [(60, 128, 140000), (100, 128, 140000), (180, 136, 140000), (348, 128, 70000), (600, 128, 70000)])
@pytest.mark.parametrize("gap", [60.0, 300.0])
def test_references_move_between_a_workgroups_tiles(N, d, V, gap):
    """A third of the rows have their probability on a token in a later tile of a workgroup's, another third first a third of the gap on one in the
    tile before it: what was added up before is brought to the new reference, and a row's tiles of one slice have different ones."""
    say(f"references move between tiles N={N} d={d} V={V} gap={gap}")
    k = 5
    splits, tiles = splits_of(N, d, V, k), (V + 255) // 256
    split = splits // 2
    first = split * tiles // splits
    assert (split + 1) * tiles // splits - first >= 2
    low, top = 256 * first + 37, 256 * (first + 1) + 101
    a, W, ids, g = inputs(N, d, V, k, spread=1.0)
    ids = torch.where((ids == top) | (ids == low) | (ids < 0) | (ids >= V), (ids.abs() + 1) % (V // 4), ids).to(torch.int32)
    for v in (low, top):
        W[v] = (0.02 * torch.sign(W[v].float())).to(torch.bfloat16)       # of length 0.02 sqrt(d)
    a = a.float()
    a[::3] += gap / (0.0004 * d) * W[top].float()
    a[1::3] += gap / (0.0004 * d) * W[top].float() + gap / 3 / (0.0004 * d) * W[low].float()
    a = a.to(torch.bfloat16)
    check_distill(a, W, ids, torch.randn((N, k), generator=g), torch.rand((N,), generator=g) + 0.1, 1.0)
    check_logp(a, W, ids, g, 1.0)
